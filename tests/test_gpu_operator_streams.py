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


# ---------------------------------------------------------------------------------------- captured calls
def captured(c, fn):
    """fn(), captured on the context's stream."""
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(c.stream):
        with torch.cuda.graph(g, stream=c.stream):
            fn()
    return g


def replay(c, g):
    with torch.cuda.stream(c.stream):
        g.replay()
    c.stream.synchronize()


def test_replays_after_the_scratch_has_grown(ctx, own):
    """Decoding steps are captured, prompts follow as ordinary calls and need a larger scratch, steps are replayed."""
    w, w2 = ctx.mx_quantize(normal(300, 256, seed=2)), ctx.mx_quantize(normal(40, 2048, seed=3))
    x, y = normal(9, 256, seed=1), torch.empty(9, 300, dtype=torch.bfloat16, device="cuda")
    x2, y2 = normal(70, 2048, seed=4), torch.empty(70, 40, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    own.mx_linear(x, w, out=y)
    own.stream.synchronize()
    graphs = [(captured(own, lambda: own.mx_linear(x, w, out=y)), x, y, w)]
    for i, rows in enumerate((500, 3000, 20000)):          # each outgrows the last one's block
        big = normal(rows, 2048, seed=rows)
        torch.cuda.synchronize()
        got = own.mx_linear(big, w2)
        own.stream.synchronize()
        assert torch.equal(got, ctx.mx_linear(big, w2))
        if i == 0:                                          # a second graph holds the block that the first prompt needed
            graphs.append((captured(own, lambda: own.mx_linear(x2, w2, out=y2)), x2, y2, w2))
        junk = [torch.full((1 << k,), 255, dtype=torch.uint8, device="cuda") for k in range(10, 28)]
        for g, xs, ys, ws in graphs:
            xs.copy_(normal(*xs.shape, seed=50 + i))
            ys.fill_(0)
            torch.cuda.synchronize()
            replay(own, g)
            assert torch.equal(ys, ctx.mx_linear(xs, ws))
        assert all(bool((t == 255).all()) for t in junk)
        del junk
    torch.cuda.synchronize()
    del graphs, g


def test_scratch_cannot_grow_under_capture(ctx, own):
    """A call that would have to allocate says so, and the capture goes on without it."""
    w = ctx.mx_quantize(normal(300, 256, seed=2))
    x, big = normal(9, 256, seed=1), normal(4000, 256, seed=2)
    y, ybig = torch.zeros(9, 300, dtype=torch.bfloat16, device="cuda"), torch.zeros(4000, 300, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    own.mx_linear(x, w, out=y)
    own.stream.synchronize()
    said = []

    def calls():
        with pytest.raises(q.binding.Qv2Error) as e:
            own.mx_linear(big, w, out=ybig)
        said.append(e.value.status)
        own.mx_linear(x, w, out=y)
    g = captured(own, calls)
    assert said == [-8]
    y.zero_()
    torch.cuda.synchronize()
    replay(own, g)
    assert torch.equal(y, ctx.mx_linear(x, w)) and not bool(ybig.any())
    own.mx_linear(big, w, out=ybig)                         # outside of a capture it grows
    replay(own, g)
    assert torch.equal(ybig, ctx.mx_linear(big, w))
    torch.cuda.synchronize()
    del g


# ---------------------------------------------------------------------------------------- a kernel that gave up
def test_a_failed_product_is_reported_once(own):
    """The word that a kernel sets when it gives up is set from the host: whatever comes next says so and does nothing, the call
    after that works; asking needs no further call."""
    import ctypes as C
    c, L = own, q.lib()
    with torch.cuda.stream(c.stream):
        x = normal(4, 64)
        w = c.mx_quantize(x)
        y, marked = torch.full((4, 4), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((4, 4), 7.0, dtype=torch.bfloat16, device="cuda")
        cache = c.kv_empty(1, 4, 1, 64, q.KV_I8)
        cache.k_codes.fill_(3)
        kept = cache.k_codes.clone()
        kv, slots = x.view(4, 1, 64), torch.arange(4, device="cuda")
        table, starts = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.tensor([0, 4], device="cuda")
        calls = [lambda: c.mx_quantize(x), lambda: c.mx_dequantize(w), lambda: c.mx_matmul(w, w, out=y, out_dtype=torch.bfloat16), lambda: c.mx_linear(x, w, out=y),
                 lambda: c.kv_write(cache, kv, kv, slots), lambda: c.kv_write(cache, kv[:0], kv[:0], slots[:0]), lambda: c.kv_read(cache, table, starts, 4),
                 lambda: c.kv_read(cache, table, starts, 0), c.check_waits]
        for call in calls:
            assert L.qv2_debug_fail_wait(c._h) == 0
            before = c.launches
            with pytest.raises(q.binding.Qv2Error) as e:
                call()
            assert e.value.status == -9 and c.launches == before
        c.stream.synchronize()
        assert torch.equal(y, marked) and torch.equal(cache.k_codes, kept)
        for call in calls:                                  # told once
            call()
        c.stream.synchronize()
        assert not torch.equal(y, marked) and not torch.equal(cache.k_codes, kept)
        # arguments that are refused leave the report to the next call
        assert L.qv2_debug_fail_wait(c._h) == 0
        assert L.qv2_mx_dequantize(c._h, None, None, q.IN_F32, 0) == -2
        syncs = c.syncs
        assert L.qv2_check_waits(c._h) == -9 and L.qv2_check_waits(c._h) == 0 and c.syncs == syncs + 2
    assert L.qv2_check_waits(None) == -2 and L.qv2_debug_fail_wait(None) == -2


def test_asking_under_capture(own):
    w = own.mx_quantize(normal(300, 256, seed=2))
    x, y = normal(9, 256, seed=1), torch.zeros(9, 300, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    own.mx_linear(x, w, out=y)
    own.stream.synchronize()
    want, said = y.clone(), []

    def calls():
        said.append(q.lib().qv2_check_waits(own._h))
        own.mx_linear(x, w, out=y)
    g = captured(own, calls)
    assert said == [-8]
    y.zero_()
    torch.cuda.synchronize()
    replay(own, g)
    own.check_waits()
    assert torch.equal(y, want)
    del g
