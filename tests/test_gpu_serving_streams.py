"""Page planning, norm with rotation and attention over the cache together, on streams of their own and in captured graphs."""
import numpy as np
import pytest
import torch

import serving_reference as ref
import paper_2501_07161_b200 as q

pytestmark = pytest.mark.gpu

HEADS, KV, DIM, PAGE = 8, 2, 64, 16


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


class Server:
    """What a served layer keeps between its steps."""

    def __init__(self, c, seqs, fmt, width=12, seed=0):
        with torch.cuda.stream(c.stream):
            self.c, self.seqs = c, seqs
            self.cache = c.kv_empty(seqs * width, PAGE, KV, DIM, fmt)
            for t in (self.cache.k_codes, self.cache.k_scales, self.cache.v_codes, self.cache.v_scales):
                t.zero_()
            self.table = torch.full((seqs, width), -1, dtype=torch.int32, device="cuda")
            self.free = torch.randperm(seqs * width, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(torch.int32)
            self.freqs = 10000.0 ** (-torch.arange(0, DIM, 2, device="cuda") / DIM)
            self.w = torch.rand(DIM, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)) + 0.5
            z = lambda n: torch.zeros(n, dtype=torch.int64, device="cuda")
            self.lens, self.count = z(seqs), torch.tensor([seqs * width], device="cuda")
        c.stream.synchronize()

    def plan(self, total):
        z = lambda n: torch.zeros(n, dtype=torch.int64, device="cuda")
        return q.PagePlan(self.lens, z(self.seqs + 1), z(self.seqs + 1), z(total), z(total), self.count, z(1))

    def step(self, qkv, fresh, out, plan, max_new=None, lse=None):
        """qkv [tokens, HEADS + 2 KV, DIM] -> the attention's results in out."""
        c = self.c
        c.kv_plan(self.lens, fresh, PAGE, self.table, self.free, self.count, qkv.shape[0], out=plan)
        qs, ks = qkv[:, :HEADS], qkv[:, HEADS: HEADS + KV]
        c.norm_rotate(qs, ks, plan.positions, self.freqs, self.w, self.w, out=(qs, ks))
        c.kv_write(self.cache, ks, qkv[:, HEADS + KV:], plan.slots)
        return c.kv_attend(self.cache, qs, plan.q_starts, plan.lens, self.table, max_new=max_new, out=out)


def plain(server, history, news):
    """The last step's results in 64 bits from what the cache holds, queries as they went in."""
    c = server.cache
    i8 = c.format == q.KV_I8
    k, v = (ref.rows_of(a.cpu().numpy(), b.cpu().numpy(), DIM, i8) for a, b in ((c.k_codes, c.k_scales), (c.v_codes, c.v_scales)))
    want, _, off, _ = ref.attend(history, k, v, server.lens.tolist(), np.concatenate([[0], np.cumsum(news)]), server.table.cpu().numpy().astype(np.int64), PAGE, DIM ** -0.5)
    return want, off


@pytest.mark.parametrize("fmt", [q.KV_MX4, q.KV_I8])
def test_prompt_then_steps(ctx, fmt):
    """A prompt, ragged chunks, single tokens and a padded batch through plan, rotation, cache and attention, against plain steps."""
    s = Server(ctx, 3, fmt)
    keys = [np.zeros((0, KV, DIM)) for _ in range(3)]
    for i, (news, pad) in enumerate((([40, 1, 17], 0), ([1, 1, 1], 0), ([9, 0, 30], 5), ([1, 1, 0], 2))):
        total = sum(news) + pad
        qkv = normal(total, HEADS + 2 * KV, DIM, seed=i)
        before = qkv.double().cpu().numpy()
        out = torch.full((total, HEADS, DIM), 5.0, dtype=torch.bfloat16, device="cuda")
        plan = s.plan(total)
        old = s.lens.tolist()
        s.step(qkv, torch.tensor(news, device="cuda"), out, plan)
        assert s.lens.tolist() == [a + b for a, b in zip(old, news)] and plan.missing.item() == 0
        pos = np.concatenate([np.arange(a, a + b) for a, b in zip(old, news)])
        assert plan.positions.tolist() == pos.tolist() + [0] * pad and plan.slots.tolist()[sum(news):] == [-1] * pad
        n = sum(news)
        turned = ref.norm_rotate(before[:n, : HEADS + KV], s.w.double().cpu().numpy(), pos, s.freqs.double().cpu().numpy(), 1e-6, False)
        got = qkv.double().cpu().numpy()
        assert (np.abs(got[:n, : HEADS + KV] - turned) <= 2.0 ** -8 * np.abs(turned) + 2.0 ** -17 * (1 + np.abs(turned))).all()
        want, off = plain(s, got[:, :HEADS], news)
        y = out.double().cpu().numpy()
        assert (np.abs(y - want)[:n] <= (off + 2.0 ** -8 * (np.abs(want) + off))[:n]).all()
        assert (y[n:] == 5).all()                                   # rows behind the last sequence
        # the keys that the cache holds are those that were written
        slots = plan.slots.cpu().numpy()[:n]
        c = s.cache
        held = ref.rows_of(c.k_codes.cpu().numpy(), c.k_scales.cpu().numpy(), DIM, fmt == q.KV_I8).reshape(-1, KV, DIM)[slots]
        step = 2.0 ** -2 if fmt == q.KV_MX4 else 2.0 ** -7          # half a step of the largest element at most
        assert (np.abs(held - got[:n, HEADS: HEADS + KV]) <= step * np.abs(got[:n, HEADS: HEADS + KV]).max(-1, keepdims=True)).all()


def captured(c, fn):
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(c.stream):
        with torch.cuda.graph(g, stream=c.stream):
            fn()
    return g


@pytest.mark.parametrize("fmt", [q.KV_MX4, q.KV_I8])
@pytest.mark.parametrize("tokens", [1, 20])
def test_a_captured_step_replayed_over_pages(own, ctx, fmt, tokens):
    """One step for three sequences, captured with its bookkeeping in place, replayed until the sequences have crossed pages: the same
    bits as ordinary calls give.  (20 tokens of 8 query heads take the form for many rows.)"""
    steps, seqs = 6, 3
    a, b = Server(own, seqs, fmt), Server(ctx, seqs, fmt)
    fresh = torch.full((seqs,), tokens, device="cuda")
    qkv, out = torch.empty(seqs * tokens, HEADS + 2 * KV, DIM, dtype=torch.bfloat16, device="cuda"), torch.empty(seqs * tokens, HEADS, DIM, dtype=torch.bfloat16, device="cuda")
    plan = a.plan(seqs * tokens)
    torch.cuda.synchronize()
    warm = Server(own, seqs, fmt)                                   # the scratch is there before the capture
    qkv.copy_(normal(*qkv.shape, seed=99))
    torch.cuda.synchronize()
    warm.step(qkv, fresh, out, warm.plan(seqs * tokens), max_new=tokens)
    own.stream.synchronize()
    g = captured(own, lambda: a.step(qkv, fresh, out, plan, max_new=tokens))
    for i in range(steps):
        x = normal(*qkv.shape, seed=i)
        qkv.copy_(x)
        torch.cuda.synchronize()
        with torch.cuda.stream(own.stream):
            g.replay()
        own.stream.synchronize()
        want = torch.empty_like(out)
        b.step(x, fresh, want, b.plan(seqs * tokens), max_new=tokens)
        torch.cuda.synchronize()
        assert a.lens.tolist() == b.lens.tolist() == [tokens * (i + 1)] * seqs and torch.equal(a.table, b.table) and a.count.item() == b.count.item()
        assert torch.equal(out, want) and bool(out.isfinite().all())
    own.check_waits()
    del g


def test_replays_after_the_scratch_has_grown(own, ctx):
    """Two captured attentions of one context, one of few rows and one of many, and between their replays an ordinary call that needs more scratch."""
    cache = ctx.kv_empty(64, PAGE, KV, DIM, q.KV_I8)
    ctx.kv_write(cache, normal(64 * PAGE, KV, DIM), normal(64 * PAGE, KV, DIM, seed=1), torch.arange(64 * PAGE, device="cuda"))
    table = torch.arange(64, dtype=torch.int32, device="cuda").view(1, 64)
    lens = torch.tensor([1000], device="cuda")
    cases = []
    torch.cuda.synchronize()
    for n in (1, 100):
        x, starts = normal(n, HEADS, DIM, seed=n), torch.tensor([0, n], device="cuda")
        out = torch.zeros_like(x)
        torch.cuda.synchronize()
        call = lambda x=x, starts=starts, out=out, n=n: own.kv_attend(cache, x, starts, lens, table, max_new=n, out=out)
        call()
        own.stream.synchronize()
        cases.append((captured(own, call), x, out, starts, n))
    big = normal(900, 16 * KV, DIM, seed=5)
    torch.cuda.synchronize()
    got = own.kv_attend(cache, big, torch.tensor([0, 900], device="cuda"), lens, table)
    own.stream.synchronize()
    assert torch.equal(got, ctx.kv_attend(cache, big, torch.tensor([0, 900], device="cuda"), lens, table))
    junk = [torch.full((1 << k,), 255, dtype=torch.uint8, device="cuda") for k in range(10, 27)]
    for g, x, out, starts, n in cases:
        out.fill_(0)
        torch.cuda.synchronize()
        with torch.cuda.stream(own.stream):
            g.replay()
        own.stream.synchronize()
        assert torch.equal(out, ctx.kv_attend(cache, x, starts, lens, table, max_new=n))
    assert all(bool((t == 255).all()) for t in junk)
    del cases, g, call


def test_scratch_cannot_grow_under_capture(own, ctx):
    cache = ctx.kv_empty(8, PAGE, KV, DIM, q.KV_MX4)
    x = normal(50, HEADS, DIM)
    table, lens, starts = torch.zeros(1, 8, dtype=torch.int32, device="cuda"), torch.tensor([100], device="cuda"), torch.tensor([0, 50], device="cuda")
    out = torch.zeros_like(x)
    torch.cuda.synchronize()
    said = []

    def call():
        with pytest.raises(q.binding.Qv2Error) as e:
            own.kv_attend(cache, x, starts, lens, table, out=out)
        said.append(e.value.status)
        out.zero_()
    captured(own, call)
    assert said == [-8]


def test_on_a_stream_that_is_not_the_contexts(own, ctx):
    """Results belong to the context's stream; inputs are not handed out again before it has read them."""
    torch.cuda.synchronize()
    x, pos, f = normal(300, HEADS, DIM), torch.arange(300, device="cuda"), torch.rand(DIM // 2, device="cuda")
    want, _ = ctx.norm_rotate(x, None, pos, f)
    torch.cuda.synchronize()
    with torch.cuda.stream(own.stream):
        torch.cuda._sleep(50_000_000)
    got, _ = own.norm_rotate(x.clone(), None, pos, f)       # the clone is freed at once ...
    torch.cuda.synchronize()                                # (its copy was made on torch's stream, which nobody else waited for)
    again, _ = own.norm_rotate(x, None, pos, f)
    own.stream.synchronize()
    assert torch.equal(again, want)


def test_a_failed_kernel_is_reported_by_the_new_calls(own):
    import ctypes as C
    c, L = own, q.lib()
    with torch.cuda.stream(c.stream):
        cache = c.kv_empty(2, PAGE, KV, DIM, q.KV_I8)
        x, one, table = normal(1, HEADS, DIM), torch.tensor([1], device="cuda"), torch.zeros(1, 2, dtype=torch.int32, device="cuda")
        calls = [lambda: c.kv_plan(one, one, PAGE, table, table[0], one, 1), lambda: c.norm_rotate(x, None, one, None),
                 lambda: c.kv_attend(cache, x, torch.tensor([0, 1], device="cuda"), one, table)]
        for call in calls:
            assert L.qv2_debug_fail_wait(c._h) == 0
            before = c.launches
            with pytest.raises(q.binding.Qv2Error) as e:
                call()
            assert e.value.status == -9 and c.launches == before
            call()
        c.stream.synchronize()


def test_two_contexts_at_once(own, ctx):
    """Attentions of two contexts on two streams over one cache do not disturb each other."""
    cache = ctx.kv_empty(80, PAGE, KV, DIM, q.KV_MX4)
    ctx.kv_write(cache, normal(80 * PAGE, KV, DIM), normal(80 * PAGE, KV, DIM, seed=1), torch.arange(80 * PAGE, device="cuda"))
    table, lens = torch.arange(80, dtype=torch.int32, device="cuda").view(2, 40), torch.tensor([640, 501], device="cuda")
    xs = [(normal(2, HEADS, DIM, seed=3), torch.tensor([0, 1, 2], device="cuda")), (normal(300, HEADS, DIM, seed=4), torch.tensor([0, 200, 300], device="cuda"))]
    torch.cuda.synchronize()
    want = [ctx.kv_attend(cache, x, s, lens, table) for x, s in xs]
    torch.cuda.synchronize()
    for _ in range(20):
        got = [c.kv_attend(cache, x, s, lens, table) for c, (x, s) in ((own, xs[0]), (ctx, xs[1]))] + [c.kv_attend(cache, x, s, lens, table) for c, (x, s) in ((own, xs[1]), (ctx, xs[0]))]
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got[2], want[1]) and torch.equal(got[3], want[0])
