"""Page planning, norm with rotation and attention over the quantized cache on the GPU against numpy in 64 bits."""
import numpy as np
import pytest
import torch

import serving_reference as ref
import paper_2501_07161_b200 as q

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}          # half a step, relative
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -24, "bf16": 2.0 ** -126}
FORMATS = {"mx4": q.KV_MX4, "i8": q.KV_I8}


@pytest.fixture(scope="module")
def ctx():
    c = q.Context(0)
    yield c
    c.close()


def f64(t):
    return t.double().cpu().numpy()


def randn(*shape, seed=0, dtype="f32", gain=1.0):
    return (gain * torch.randn(*shape, generator=torch.Generator().manual_seed(seed))).to(DTYPES[dtype])


def ints(values):
    return torch.tensor(values, dtype=torch.int64, device="cuda")


# ---------------------------------------------------------------------------------------- planning
def check_plan(ctx, lens, fresh, page, width, free, count, total, table=None, out=None, alias=False):
    rng = np.random.RandomState(len(lens) + page)
    if table is None:
        table = np.full((len(lens), width), -1, dtype=np.int64)
        for s, h in enumerate(lens):
            have = min(-(-max(h, 0) // page), width)
            table[s, :have] = rng.randint(0, 1 << 20, have)
    want = ref.plan(lens, fresh, page, table, free, count, total)
    dt = torch.from_numpy(table.astype(np.int32)).cuda()
    a, b, f, c = ints(lens), ints(fresh), torch.tensor(free, dtype=torch.int32, device="cuda"), ints([count])
    if alias:
        out = q.PagePlan(a, *(torch.empty(n, dtype=torch.int64, device="cuda") for n in (len(lens) + 1, len(lens) + 1, total, total)), c, ints([0]))
    p = ctx.kv_plan(a, b, page, dt, f, c, total, out=out)
    if alias:
        assert p.lens is a and p.free_count is c
    got = [dt, p.lens, p.q_starts, p.starts, p.slots, p.positions, p.free_count, p.missing]
    for name, g, w in zip(("table", "lens", "q_starts", "starts", "slots", "positions", "left", "missing"), got, want):
        assert np.array_equal(g.cpu().numpy().reshape(-1), np.asarray(w, dtype=np.int64).reshape(-1)), name


@pytest.mark.parametrize("seqs,page,longest,new,spare", [(1, 16, 1, 1, 0), (1, 1, 5, 3, 2), (3, 7, 40, 20, 5), (64, 64, 2000, 1, 0), (257, 16, 300, 70, 99),
                                                        (1025, 32, 500, 9, 1), (2500, 16, 100, 50, 3000), (5, 128, 10, 4000, 0)])
def test_plan(ctx, seqs, page, longest, new, spare):
    rng = np.random.RandomState(seqs)
    lens = (rng.randint(0, longest + 1, seqs) * (rng.rand(seqs) < 0.8)).tolist()
    fresh = (rng.randint(0, new + 1, seqs) * (rng.rand(seqs) < 0.9)).tolist()
    width = max(-(-(h + m) // page) for h, m in zip(lens, fresh)) + 2
    need = sum(-(-(h + m) // page) - -(-h // page) for h, m in zip(lens, fresh))
    free = rng.permutation(need + 9).tolist()
    check_plan(ctx, lens, fresh, page, width, free, need + 4, sum(fresh) + spare)


def test_plan_in_place_repeatedly(ctx):
    """Steps of one token for every sequence, lengths and count updated where they lie, as a captured step does it."""
    page, seqs, steps = 4, 37, 11
    free = np.random.RandomState(0).permutation(400)
    table = np.full((seqs, 6), -1, dtype=np.int64)
    lens, count = [i % 9 for i in range(seqs)], 400
    table, lens0, *_, count, _ = ref.plan([0] * seqs, lens, page, table, free, count, 0)
    a, c, dt = ints(lens), ints([count]), torch.from_numpy(table.astype(np.int32)).cuda()
    f, one = torch.tensor(free, dtype=torch.int32, device="cuda"), ints([1] * seqs)
    out = q.PagePlan(a, ints([0] * (seqs + 1)), ints([0] * (seqs + 1)), ints([0] * seqs), ints([0] * seqs), c, ints([0]))
    for _ in range(steps):
        ctx.kv_plan(a, one, page, dt, f, c, seqs, out=out)
        table, lens, q_starts, starts, slots, positions, count, missing = ref.plan(lens, [1] * seqs, page, table, free, count, seqs)
        assert np.array_equal(dt.cpu().numpy(), table) and a.tolist() == lens and c.item() == count and missing == 0 == out.missing.item()
        assert out.slots.tolist() == slots and out.positions.tolist() == positions and out.starts.tolist() == starts


def test_plan_list_runs_out_and_rows_run_out(ctx):
    check_plan(ctx, [5, 0, 17, 3], [20, 9, 30, 0], 4, 9, list(range(100, 107)), 7, 70)
    check_plan(ctx, [5, 0, 17, 3], [20, 9, 30, 0], 4, 9, list(range(100, 107)), 50, 70)      # a count past the list
    check_plan(ctx, [5, 0, 17, 3], [20, 9, 30, 0], 4, 9, list(range(100, 107)), -3, 70)
    check_plan(ctx, [50, 0, 36], [3, 60, 1], 4, 9, list(range(40)), 40, 64)                  # more tokens than a row has pages for
    check_plan(ctx, [-5, 2, 1], [4, -7, 3], 4, 3, list(range(40)), 40, 7)                    # negative lengths are none
    check_plan(ctx, [3, 4], [5, 6], 2, 8, [9] * 20, 20, 6)                                   # total too small for the new tokens
    check_plan(ctx, [3, 4], [0, 0], 2, 8, [], 0, 0)


@pytest.mark.parametrize("seqs,total", [(3, 10), (700, 5000)])
def test_plan_aliased_outputs(ctx, seqs, total):
    rng = np.random.RandomState(3)
    lens, fresh = rng.randint(0, 90, seqs).tolist(), rng.randint(0, 8, seqs).tolist()
    check_plan(ctx, lens, fresh, 16, 8, rng.permutation(5000).tolist(), 4321, total, alias=True)


def test_plan_no_sequences(ctx):
    p = ctx.kv_plan(ints([]), ints([]), 16, torch.empty(0, 4, dtype=torch.int32, device="cuda"), torch.arange(3, dtype=torch.int32, device="cuda"), ints([3]), 5)
    assert p.q_starts.tolist() == [0] and p.starts.tolist() == [0] and p.slots.tolist() == [-1] * 5 and p.positions.tolist() == [0] * 5
    assert p.free_count.tolist() == [3] and p.missing.tolist() == [0]


# ---------------------------------------------------------------------------------------- norm and rotation
def check_rotate(got, x, weight, positions, freqs, eps, pairs, dtype):
    want = ref.norm_rotate(f64(x), None if weight is None else f64(weight), positions.cpu().numpy(), f64(freqs), eps, pairs)
    # mean of squares and its root: dim + 4 roundings, each of size 2^-24 and half of it in the root; product with r and w, sine and cosine to
    # 2^-22, two products and a sum; then one rounding to the type
    mate = np.abs(ref.norm_rotate(f64(x), None if weight is None else f64(weight), np.zeros(x.shape[0]), f64(freqs), eps, pairs))
    half = len(freqs)
    size = mate.copy()
    i = np.arange(half)
    a, b = (2 * i, 2 * i + 1) if pairs else (i, i + half)
    size[..., a] += mate[..., b]
    size[..., b] += mate[..., a]
    off = 2.0 ** -24 * (x.shape[-1] / 2 + 16) * size + 2.0 ** -21 * size
    bound = off + HALF[dtype] * (np.abs(want) + off) + TINY[dtype]
    assert (np.abs(f64(got) - want) <= bound).all(), float((np.abs(f64(got) - want) / bound).max())


ROTATIONS = [(1, 1, 1, 2, 2), (3, 4, 2, 64, 64), (5, 32, 8, 128, 128), (7, 3, 1, 80, 80), (2, 5, 5, 80, 32), (9, 2, 2, 96, 48), (4, 12, 4, 256, 256), (3, 2, 1, 33, 20),
             (6, 1, 3, 200, 10), (1300, 8, 2, 128, 64), (2400, 3, 2, 64, 64), (2, 2, 2, 8, 0)]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("tokens,heads,kv,dim,rot", ROTATIONS)
def test_norm_rotate(ctx, tokens, heads, kv, dim, rot, pairs, dtype):
    x = randn(tokens, heads + 2 * kv, dim, seed=dim, dtype=dtype).cuda()
    qq, kk = x[:, :heads], x[:, heads: heads + kv]
    freqs = (10000.0 ** (-torch.arange(0, rot, 2) / max(rot, 1))).float().cuda()
    pos = torch.randint(0, 1 << 20, (tokens,), generator=torch.Generator().manual_seed(1)).cuda()
    wq, wk = (1 + randn(dim, seed=2, gain=0.2)).cuda(), (1 + randn(dim, seed=3, gain=0.2)).cuda()
    for a, b in ((wq, wk), (None, None), (wq, None)):
        y, z = ctx.norm_rotate(qq, kk, pos, freqs if rot else None, a, b, eps=1e-5, pairs=pairs)
        assert y.dtype == x.dtype and y.shape == qq.shape and z.shape == kk.shape
        check_rotate(y, qq, a, pos, freqs, 1e-5, pairs, dtype)
        check_rotate(z, kk, b, pos, freqs, 1e-5, pairs, dtype)
    alone, none = ctx.norm_rotate(qq, None, pos, freqs if rot else None, wq, eps=1e-5, pairs=pairs)
    assert none is None and torch.equal(alone, ctx.norm_rotate(qq, kk, pos, freqs if rot else None, wq, wk, eps=1e-5, pairs=pairs)[0])


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("offset,pad", [(0, 8), (1, 3), (4, 1)])
def test_norm_rotate_strides_and_in_place(ctx, offset, pad, dtype):
    tokens, heads, dim = 21, 5, 64
    ld = heads * (dim + pad)
    buf = randn(tokens * ld + offset, seed=pad, dtype=dtype).cuda()
    x = buf[offset:].as_strided((tokens, heads, dim), (ld, dim + pad, 1))
    gap = buf.clone()
    freqs, pos, w = torch.rand(32, device="cuda"), torch.arange(tokens, device="cuda") * 1001, torch.rand(dim, device="cuda")
    want, _ = ctx.norm_rotate(x.clone(), None, pos, freqs, w)
    check_rotate(want, x, w, pos, freqs, 1e-6, False, dtype)
    got, _ = ctx.norm_rotate(x, None, pos, freqs, w, out=(x, None))
    assert got is x and torch.equal(x, want)
    gap[offset:].as_strided((tokens, heads, dim), (ld, dim + pad, 1)).copy_(want)
    assert torch.equal(buf, gap)                                              # nothing between the rows has changed


def test_norm_rotate_far_positions_and_poison(ctx):
    x = randn(4, 2, 64, seed=1).cuda()
    pos = ints([(1 << 31) + 5, 123456789, 0, -77])
    freqs = (10000.0 ** (-torch.arange(0, 64, 2) / 64)).float().cuda()
    y, _ = ctx.norm_rotate(x, None, pos, freqs)
    check_rotate(y, x, None, pos, freqs, 1e-6, False, "f32")
    x[1, 0, 5] = float("nan")
    x[2, 1, 3] = float("inf")
    y, _ = ctx.norm_rotate(x, None, pos, freqs, torch.ones(64, device="cuda"))
    bad = torch.isnan(y).any(-1)
    assert bad[1, 0] and bad[2, 1] and bad.sum() == 2
    zero, _ = ctx.norm_rotate(torch.zeros(3, 1, 64, device="cuda"), None, pos[:3], freqs, torch.ones(64, device="cuda"), eps=1e-6)
    assert (zero == 0).all()


def test_norm_rotate_no_tokens(ctx):
    x = torch.empty(0, 3, 64, device="cuda")
    y, z = ctx.norm_rotate(x, x, ints([]), torch.ones(32, device="cuda"))
    assert y.shape == x.shape and z.shape == x.shape


# ---------------------------------------------------------------------------------------- attention
class Held:
    """A cache filled through kv_write, its sequences in shuffled pages, and the values that it holds."""

    def __init__(self, ctx, fmt, lens, heads, dim, page, seed=0, extra=3, gain=1.0, write=None):
        self.lens, self.page, self.dim = list(lens), page, dim
        rng = np.random.RandomState(seed)
        pages = [-(-max(c, 0) // page) for c in lens]
        ids = rng.permutation(sum(pages) + extra)
        self.table = np.full((len(lens), max(pages + [1]) + 1), -1, dtype=np.int64)
        for s, n in enumerate(pages):
            self.table[s, :n] = ids[sum(pages[:s]): sum(pages[:s]) + n]
        total = (sum(pages) + extra) * page
        k = randn(total, heads, dim, seed=seed + 1, gain=gain) * torch.exp(0.5 * randn(total, heads, 1, seed=seed + 2))
        v = randn(total, heads, dim, seed=seed + 3) * torch.exp(1.0 * randn(total, heads, 1, seed=seed + 4))
        if write:
            write(k, v, self)
        self.cache = ctx.kv_empty(sum(pages) + extra, page, heads, dim, FORMATS[fmt])
        ctx.kv_write(self.cache, k.cuda(), v.cuda(), torch.arange(total, device="cuda"))
        c = self.cache
        self.k, self.v = (ref.rows_of(a.cpu().numpy(), b.cpu().numpy(), dim, fmt == "i8") for a, b in ((c.k_codes, c.k_scales), (c.v_codes, c.v_scales)))

    def slot(self, s, j):
        return self.table[s, j // self.page] * self.page + j % self.page


def check_attend(ctx, held, x, news, dtype, window=0, cap=0.0, slopes=None, scale=None, max_new=None, starts=None, out=None):
    starts = np.concatenate([[0], np.cumsum(news)]) if starts is None else starts
    scale = held.dim ** -0.5 if scale is None else scale
    want, lse, off, off_lse = ref.attend(f64(x), held.k, held.v, held.lens, starts, held.table, held.page, scale, window, cap,
                                         None if slopes is None else f64(slopes), 22 if dtype == "f32" else 11)
    args = (held.cache, x, ints(starts.tolist()), ints(held.lens), torch.from_numpy(held.table.astype(np.int32)).cuda())
    kw = dict(scale=scale, window=window, cap=cap, slopes=slopes, max_new=max_new)
    got, got_lse = ctx.kv_attend(*args, want_lse=True, out=out, **kw)
    assert got.dtype == x.dtype and got.shape == x.shape
    covered = np.zeros(x.shape[0], bool)
    for a, b in zip(starts[:-1], starts[1:]):
        covered[max(a, 0): max(b, 0)] = True
    g, w, o = f64(got)[covered], want[covered], off[covered]
    assert np.array_equal(np.isnan(g), np.isnan(w))
    fine = ~np.isnan(w)
    bound = o + HALF[dtype] * (np.abs(w) + o) + TINY[dtype]
    assert (np.abs(g - w)[fine] <= bound[fine]).all(), float((np.abs(g - w) / bound)[fine].max())
    gl, wl = f64(got_lse)[covered], lse[covered]
    rows = ~np.isnan(w).any(-1)
    assert np.array_equal(np.isneginf(gl[rows]), np.isneginf(wl[rows]))
    some = rows & np.isfinite(wl)
    assert (np.abs(gl[some] - wl[some]) <= off_lse[covered][some]).all(), float(np.abs(gl[some] - wl[some]).max())
    again = ctx.kv_attend(*args, **kw)
    assert torch.equal(again[torch.from_numpy(covered).cuda()].nan_to_num(7), got[torch.from_numpy(covered).cuda()].nan_to_num(7))
    return got, got_lse


STEPS = [([1], [1], 1, 1, 64, 16), ([5], [1], 4, 1, 128, 16), ([33, 1, 70], [1, 1, 1], 8, 2, 128, 16), ([200, 150, 31, 32], [1] * 4, 32, 8, 128, 16),
         ([1000, 3], [1, 1], 6, 3, 80, 7), ([129, 64, 65], [1] * 3, 16, 1, 64, 64), ([500], [1], 12, 4, 96, 32), ([77, 300], [1, 1], 5, 5, 256, 16),
         ([90, 41], [1, 1], 40, 1, 128, 16), ([18, 45], [1, 1], 3, 3, 33, 5), ([60, 61], [1, 1], 2, 1, 1, 1), ([100, 20], [1, 1], 24, 12, 200, 8)]


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("lens,news,q_heads,heads,dim,page", STEPS)
def test_attend_single_tokens(ctx, lens, news, q_heads, heads, dim, page, dtype, fmt):
    held = Held(ctx, fmt, lens, heads, dim, page, seed=dim)
    fused = randn(sum(news), q_heads + 3, dim, seed=9, dtype=dtype, gain=2.0).cuda()
    check_attend(ctx, held, fused[:, 1: 1 + q_heads], news, dtype, max_new=1)


CHUNKS = [([1], [1], 1, 1, 64, 16), ([40, 9], [40, 9], 4, 2, 128, 16), ([130], [130], 2, 1, 128, 32), ([300, 65, 1, 129], [17, 65, 1, 100], 8, 2, 128, 16),
          ([257, 140], [3, 140], 6, 2, 80, 7), ([150], [60], 16, 1, 64, 64), ([90, 200], [90, 2], 3, 3, 256, 16), ([64, 70], [33, 70], 5, 1, 33, 5), ([300], [300], 1, 1, 96, 128)]


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("lens,news,q_heads,heads,dim,page", CHUNKS)
def test_attend_chunks(ctx, lens, news, q_heads, heads, dim, page, dtype, fmt):
    held = Held(ctx, fmt, lens, heads, dim, page, seed=dim + 1)
    x = randn(sum(news), q_heads, dim, seed=8, dtype=dtype, gain=2.0).cuda()
    check_attend(ctx, held, x, news, dtype)


OPTIONS = [dict(window=1), dict(window=17), dict(window=64, cap=5.0), dict(cap=30.0), dict(slopes=True), dict(window=100, cap=2.0, slopes=True), dict(scale=0.0), dict(scale=-0.3)]


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news", [[1, 1, 1], [9, 1, 4], [200, 60, 1]])
@pytest.mark.parametrize("options", OPTIONS, ids=str)
def test_attend_options(ctx, options, news, dtype, fmt):
    held = Held(ctx, fmt, [300, 61, 128], 2, 64, 16, seed=4)
    x = randn(sum(news), 8, 64, seed=5, dtype=dtype, gain=2.0).cuda()
    options = dict(options)
    if options.get("slopes"):
        options["slopes"] = torch.exp2(-torch.arange(1.0, 9.0)).cuda()
    check_attend(ctx, held, x, news, dtype, **options)


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("news", [[1, 1, 1, 1], [20, 40, 150, 3]])
def test_attend_rows_that_see_nothing(ctx, news, fmt):
    """No tokens at all, more queries than tokens, pages that do not exist; rows of no sequence keep what they held."""
    held = Held(ctx, fmt, [0, 30, 160, 50], 2, 64, 16, seed=6)
    held.table[3] = [-1, 1 << 20, held.cache.k_codes.shape[0], -5, 7] + held.table[3, 5:].tolist()
    held.table[2, 1] = -1
    rows = sum(news)
    x = randn(rows + 9, 4, 64, seed=5, dtype="bf16", gain=2.0).cuda()
    starts = np.concatenate([[0], np.cumsum(news)]) + 4
    out = torch.full_like(x, 3.0)
    check_attend(ctx, held, x, news, "bf16", starts=starts, out=out)
    assert (out[:4] == 3).all() and (out[rows + 4:] == 3).all() and (out[4: 4 + news[0]] == 0).all()


@pytest.mark.parametrize("fmt", list(FORMATS))
def test_attend_starts_are_held_to_the_rows(ctx, fmt):
    held = Held(ctx, fmt, [30, 20], 1, 64, 16, seed=6)
    x = randn(12, 2, 64, seed=5, dtype="f16").cuda()
    check_attend(ctx, held, x, None, "f16", starts=np.array([-5, 7, 40]))


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("news", [[1, 1], [6, 5], [70, 100]])
def test_attend_poison_reaches_those_who_see_it(ctx, news, fmt):
    """A NaN in a key or a value, and what lies in slots that nobody sees: behind the end, before the window, later than the query."""
    def write(k, v, held):
        k[held.slot(0, 3), 0, 5] = float("nan")                       # head 0 of sequence 0
        v[held.slot(1, 117), 1, 40] = float("inf")                    # head 1 of sequence 1, near its end
        k[held.slot(0, 90) + 1] = float("nan")                        # slots behind the ends
        v[held.slot(1, 119) + 1] = float("nan")
    held = Held(ctx, fmt, [91, 120], 2, 64, 16, seed=7, write=write)
    x = randn(sum(news), 4, 64, seed=5, dtype="bf16").cuda()
    got, _ = check_attend(ctx, held, x, news, "bf16")
    bad = torch.isnan(got).any(-1)
    assert bad[: news[0], :2][min(news[0], 91) - 1].all() and not bad[:, 2:][: news[0]].any() and bad[-1, 2:].all()
    got, _ = check_attend(ctx, held, x, news, "bf16", window=20)
    assert not torch.isnan(got[news[0] - 1]).any()
    x[0, 1, 9] = float("nan")
    x[news[0], 0, 2] = float("inf")
    check_attend(ctx, held, x, news, "bf16", window=20)


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("news", [[1], [40]])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_attend_scales_far_apart(ctx, news, dtype, fmt):
    """Rows of zeros, values of very different size, blocks of a row of different size, a token that outweighs the rest."""
    def write(k, v, held):
        for j in range(0, 90, 3):
            v[held.slot(0, j)] *= 2.0 ** (-(j % 9))
        k[held.slot(0, 11)], v[held.slot(0, 12)] = 0, 0
        v[held.slot(0, 20), :, :32] *= 2.0 ** -6
        k[held.slot(0, 30), :, 32:] *= 2.0 ** -8
        k[held.slot(0, 40)] *= 30
    held = Held(ctx, fmt, [90], 2, 64, 16, seed=8, write=write)
    x = randn(news[0], 4, 64, seed=5, dtype=dtype).cuda()
    x[0, 0] *= 2.0 ** -9
    x[0, 1] *= 100
    x[0, 2] = 0
    check_attend(ctx, held, x, news, dtype)


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("max_new", [1, 5, 70, 100, 1 << 40])
def test_attend_whatever_most_is_said(ctx, max_new, fmt):
    """max_new chooses kernels; results do not depend on its being right."""
    held = Held(ctx, fmt, [150, 40, 130], 2, 64, 16, seed=12)
    check_attend(ctx, held, randn(111, 4, 64, seed=9, dtype="f16").cuda(), [100, 1, 10], "f16", max_new=max_new)


@pytest.mark.parametrize("fmt", list(FORMATS))
def test_attend_thousands_of_sequences(ctx, fmt):
    """More sequences than threads, many without new tokens, some of them in chunks."""
    lens = [(7 * s) % 23 for s in range(2600)]
    news = [40 if s in (700, 2599) else (0 if s % 5 == 0 else 1 + (s % 97 == 0)) for s in range(2600)]
    lens[700], lens[2599] = 60, 40
    held = Held(ctx, fmt, lens, 1, 32, 8, seed=13)
    check_attend(ctx, held, randn(sum(news), 2, 32, seed=9, dtype="bf16").cuda(), news, "bf16")


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("options", [dict(), dict(cap=5.0)], ids=str)
@pytest.mark.parametrize("lens,news", [([4, 8], [9, 12]), ([4, 70], [40, 75])])
def test_attend_poisoned_queries_that_see_nothing(ctx, lens, news, options, fmt):
    """They give zeros, like any that see nothing (padding may hold anything); those that see a token give NaN."""
    held = Held(ctx, fmt, lens, 2, 64, 16, seed=10)
    x = randn(sum(news), 4, 64, seed=7, dtype="bf16")
    x[0, 0, 3], x[1, 1, 0], x[2, :, 63] = float("nan"), float("inf"), -float("inf")
    x[news[0] - 1, 2, 5], x[news[0], 3, 7], x[news[0] + 6, 0, 1] = float("inf"), float("nan"), float("nan")
    check_attend(ctx, held, x.cuda(), news, "bf16", **options)


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("tokens,news,q_heads", [(32000, [4], 32), (3000, [31, 33, 1], 8)])
def test_attend_pieces_of_many_rows(ctx, tokens, news, q_heads, fmt):
    """Few sequences cut into many pieces, of which each has many rows of results to add up."""
    held = Held(ctx, fmt, [tokens] * len(news), 8, 64, 64, seed=11)
    check_attend(ctx, held, randn(sum(news), q_heads, 64, seed=8, dtype="bf16").cuda(), news, "bf16")


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,news", [([300], [1]), ([300], [40]), ([700, 30], [1, 30])])
@pytest.mark.parametrize("power", [90, -90])
def test_attend_values_far_from_one(ctx, power, lens, news, dtype, fmt):
    """Values times 2^90 and 2^-90: weights are held against the largest scale of a value, whatever that is."""
    def write(k, v, held):
        v *= 2.0 ** power
    held = Held(ctx, fmt, lens, 2, 128, 16, seed=9, write=write)
    check_attend(ctx, held, randn(sum(news), 4, 128, seed=6, dtype=dtype).cuda(), news, dtype)


@pytest.mark.parametrize("new", [1, 60])
def test_attend_cache_past_32_bits(ctx, new):
    """Rows of one head whose byte offsets pass 2^32; the pages in between are never touched."""
    heads, dim, page = 8, 128, 64
    pages = (1 << 32) // (page * heads * dim) + 9
    cache = ctx.kv_empty(pages, page, heads, dim, q.KV_I8)
    used = [pages - 1, 0, pages - 2]
    k, v = randn(3 * page, heads, dim, seed=1), randn(3 * page, heads, dim, seed=2)
    slots = torch.cat([torch.arange(page) + page * i for i in used]).cuda()
    ctx.kv_write(cache, k.cuda(), v.cuda(), slots)
    x = randn(new, 16, dim, seed=3, dtype="bf16").cuda()
    small = ctx.kv_empty(3, page, heads, dim, q.KV_I8)
    ctx.kv_write(small, k.cuda(), v.cuda(), torch.arange(3 * page, device="cuda"))
    args = (ints([0, new]), ints([3 * page - 5]))
    big = ctx.kv_attend(cache, x, *args, torch.tensor([used], dtype=torch.int32, device="cuda"))
    assert torch.equal(big, ctx.kv_attend(small, x, *args, torch.tensor([[0, 1, 2]], dtype=torch.int32, device="cuda")))


def test_attend_long_axis_in_many_parts(ctx):
    """One sequence of 20 K tokens among short ones."""
    lens = [20001, 3, 700, 1]
    held = Held(ctx, "mx4", lens, 1, 64, 64, seed=3)
    for dtype, news in (("f32", [1, 1, 1, 1]), ("bf16", [2, 1, 1, 1]), ("f16", [40, 3, 30, 1])):
        x = randn(sum(news), 8, 64, seed=5, dtype=dtype, gain=2.0).cuda()
        check_attend(ctx, held, x, news, dtype, max_new=max(news))


def test_attend_no_rows_no_pages(ctx):
    cache = ctx.kv_empty(0, 16, 2, 64, q.KV_MX4)
    x = torch.ones(3, 4, 64, device="cuda")
    y, lse = ctx.kv_attend(cache, x, ints([0, 1, 3]), ints([5, 9]), torch.zeros(2, 3, dtype=torch.int32, device="cuda"), want_lse=True)
    assert (y == 0).all() and torch.isneginf(lse).all()
    assert ctx.kv_attend(cache, x[:0], ints([0, 0, 0]), ints([5, 9]), torch.zeros(2, 3, dtype=torch.int32, device="cuda")).shape == (0, 4, 64)
    y, lse = ctx.kv_attend(cache, x, ints([0, 1, 3]), ints([5, 9]), torch.zeros(2, 0, dtype=torch.int32, device="cuda"), want_lse=True)
    assert (y == 0).all() and torch.isneginf(lse).all()


# ---------------------------------------------------------------------------------------- refusals
def test_refusals(ctx):
    cache = ctx.kv_empty(4, 16, 2, 64, q.KV_I8)
    x, s, n, t = torch.ones(3, 4, 64, device="cuda"), ints([0, 1, 3]), ints([5, 9]), torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    for bad, err in (((x.double(), s, n, t), TypeError), ((x[..., :60], s, n, t), ValueError), ((x.transpose(1, 2), s, n, t), ValueError), ((x, s[:2], n, t), ValueError),
                     ((x, s.int(), n, t), ValueError), ((x, s, n[:1], t), ValueError), ((x, s, n, t.long()), ValueError), ((x, s, n, t[:, ::2]), ValueError),
                     ((x.cpu(), s, n, t), ValueError)):
        with pytest.raises(err):
            ctx.kv_attend(cache, *bad)
    for kw in (dict(max_new=0), dict(window=-1), dict(slopes=torch.ones(3, device="cuda")), dict(out=torch.ones(3, 4, 63, device="cuda")), dict(out=x.half())):
        with pytest.raises(ValueError):
            ctx.kv_attend(cache, x, s, n, t, **kw)
    for kw in (dict(cap=-1.0), dict(cap=float("nan")), dict(scale=float("inf")), dict(cap=float("inf"))):
        with pytest.raises(q.binding.Qv2Error) as e:
            ctx.kv_attend(cache, x, s, n, t, **kw)
        assert e.value.status == -1
    with pytest.raises(q.binding.Qv2Error) as e:
        ctx.kv_attend(cache, x[:, :3], s, n, t)                               # three heads cannot share two
    assert e.value.status == -1
    with pytest.raises(q.binding.Qv2Error) as e:
        ctx.kv_attend(ctx.kv_empty(1, 1, 1, 257, q.KV_I8), torch.ones(3, 4, 257, device="cuda"), s, n, t)
    assert e.value.status == -4
    pos, f = ints([0, 1, 2]), torch.ones(32, device="cuda")
    for args, kw, err in (((x.double(), None, pos, f), {}, TypeError), ((x, x[:2], pos, f), {}, ValueError), ((x, None, pos[:2], f), {}, ValueError),
                          ((x, None, pos, f.double()), {}, ValueError), ((x, None, pos, f, f), {}, ValueError), ((x, x.half(), pos, f), {}, ValueError),
                          ((x, None, pos, f), dict(out=(x[:2], None)), ValueError), ((x.transpose(1, 2), None, pos, f), {}, ValueError)):
        with pytest.raises(err):
            ctx.norm_rotate(*args, **kw)
    for args, kw, status in (((x, None, pos, torch.ones(33, device="cuda")), {}, -1), ((x, None, pos, f), dict(eps=-1.0), -1), ((x, None, pos, f), dict(eps=float("nan")), -1),
                             ((torch.ones(3, 1, 260, device="cuda"), None, pos, f), {}, -4)):
        with pytest.raises(q.binding.Qv2Error) as e:
            ctx.norm_rotate(*args, **kw)
        assert e.value.status == status
    free, one = torch.arange(9, dtype=torch.int32, device="cuda"), ints([9])
    for args in ((n.int(), n, 16, t, free, one, 5), (n, n[:1], 16, t, free, one, 5), (n, n, 16, t.long(), free, one, 5), (n, n, 16, t[:1], free, one, 5),
                 (n, n, 16, t, free.long(), one, 5), (n, n, 16, t, free, n, 5)):
        with pytest.raises(ValueError):
            ctx.kv_plan(*args)
    for page, status in ((0, -1), (1 << 30, -4)):
        with pytest.raises(q.binding.Qv2Error) as e:
            ctx.kv_plan(n, n, page, t, free, one, 5)
        assert e.value.status == status
