"""The 4-bit operators and the quantized cache on streams of their own and in captured graphs."""
import pytest
import torch

import paper_2501_07161_b200 as q

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = q.Context(0)
    yield c
    c.close()


@pytest.fixture
def own():
    c = q.Context(0, stream=torch.cuda.Stream())
    yield c
    c.close()


def normal(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


# ---------------------------------------------------------------------------------------- another stream
@pytest.mark.parametrize("call", ["quantize", "linear", "grouped"])
def test_input_that_the_call_has_to_copy(ctx, own, call):
    """[s, b, c].transpose(0, 1) cannot be viewed as rows.  The copy that the call makes of it must be there before the
    context's stream reads it, whatever torch's own stream is busy with."""
    x = normal(5, 40, 256).transpose(0, 1)
    dense = x.contiguous()
    w = ctx.mx_quantize(normal(64, 256, seed=1))
    w3 = q.MxMatrix(w.codes.view(2, 32, -1), w.scales.unflatten(0, (2, 32)), 256)
    offsets = torch.tensor([0, 70, 200], device="cuda")
    run = {"quantize": lambda c, t: c.mx_quantize(t, want_values=True), "linear": lambda c, t: c.mx_linear(t, w),
           "grouped": lambda c, t: c.mx_linear_grouped(t, offsets, w3)}[call]
    want = run(ctx, dense)
    junk = torch.full_like(dense, 7)                       # what the copy's memory holds until it is written
    torch.cuda.synchronize()
    del junk
    torch.cuda._sleep(100_000_000)                         # torch's stream comes to nothing for a while
    got = run(own, x)
    own.stream.synchronize()
    if call == "quantize":
        assert torch.equal(got.codes, want.codes) and torch.equal(got.scales, want.scales) and torch.equal(got.values, want.values)
    else:
        assert got.shape == (40, 5, want.shape[-1]) and torch.equal(got, want)
    torch.cuda.synchronize()
