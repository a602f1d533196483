"""The microscaled 4-bit operators and the quantized cache on the GPU against numpy in 64 bits: codes and scales bit for
bit, products within the bound of their sums, every size class, stride, mask and refusal."""
import numpy as np
import pytest
import torch

import mx_reference as ref
import paper_2501_07161_b200 as q

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = {"f32": 2.0 ** -23, "f16": 2.0 ** -10, "bf16": 2.0 ** -7}


@pytest.fixture(scope="module")
def ctx():
    c = q.Context(0)
    yield c
    c.close()


def randn(*shape, seed=0, dtype="f32"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(*shape, generator=g) * torch.exp(torch.randn(shape[-1], generator=g))
    return x.to(DTYPES[dtype])


def f64(t):
    return t.double().cpu().numpy()


def pack(x64, device="cuda", pad=0):
    """A reference-quantized matrix on the device; pad: extra bytes between rows (codes: 16 per unit)."""
    codes, scales, v = ref.quantize(x64)
    c = torch.zeros(codes.shape[0], codes.shape[1] + 16 * pad, dtype=torch.uint8)
    s = torch.full((scales.shape[0], scales.shape[1] + pad), 255, dtype=torch.uint8)       # NaN scales in the gap
    c[:, : codes.shape[1]], s[:, : scales.shape[1]] = torch.from_numpy(codes), torch.from_numpy(scales)
    if pad:
        c[:, codes.shape[1]:] = 0x77
    c, s = c.to(device), s.to(device)
    return q.MxMatrix(c[:, : codes.shape[1]], s[:, : scales.shape[1]], x64.shape[1]), v


# ---------------------------------------------------------------------------------------- rounding
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (3, 32), (2, 33), (5, 64), (7, 100), (4, 255), (33, 1000), (1, 25088), (257, 4104), (0, 64), (3, 0)])
def test_quantize_sizes(ctx, rows, cols, dtype):
    x = randn(rows, cols, seed=rows + cols, dtype=dtype) if rows * cols else torch.zeros(rows, cols, dtype=DTYPES[dtype])
    m = ctx.mx_quantize(x.cuda(), want_values=True)
    codes, scales, v = ref.quantize(f64(x))
    assert np.array_equal(m.codes.cpu().numpy(), codes) and np.array_equal(m.scales.cpu().numpy(), scales)
    assert m.values.dtype == x.dtype and np.array_equal(f64(m.values), v)


def test_quantize_many_rows_use_the_wide_kernel(ctx):
    x = randn(3001, 520, seed=5, dtype="bf16")
    m = ctx.mx_quantize(x.cuda())
    codes, scales, _ = ref.quantize(f64(x))
    assert np.array_equal(m.codes.cpu().numpy(), codes) and np.array_equal(m.scales.cpu().numpy(), scales)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("offset,ld", [(0, 300), (1, 296), (3, 301), (8, 304)])
def test_quantize_strides_and_alignment(ctx, offset, ld, dtype):
    buf = randn(20 * ld + offset, seed=ld, dtype=dtype).cuda()
    x = buf[offset:].as_strided((20, 290), (ld, 1))
    m = ctx.mx_quantize(x, want_values=True)
    codes, scales, v = ref.quantize(f64(x))
    assert np.array_equal(m.codes.cpu().numpy(), codes) and np.array_equal(m.scales.cpu().numpy(), scales)
    assert np.array_equal(f64(m.values), v)


def test_quantize_ties_and_saturation(ctx):
    # amax 4 keeps the scale at 1: every midpoint and its neighbours in bfloat16 and binary32
    mids = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5])
    up, down = np.nextafter(mids.astype(np.float32), np.float32(9)), np.nextafter(mids.astype(np.float32), np.float32(0))
    row = np.concatenate([mids, -mids, up, down, [4.0, -0.0, 0.0, 1e-30]]).astype(np.float32)
    sat = np.concatenate([[7.9, 5.0, 4.999, 5.001, 6.5, -7.5, 7.0], np.zeros(21)]).astype(np.float32)
    x = torch.from_numpy(np.stack([row, sat]))
    m = ctx.mx_quantize(x.cuda(), want_values=True)
    codes, scales, v = ref.quantize(f64(x))
    assert np.array_equal(m.codes.cpu().numpy(), codes) and np.array_equal(m.scales.cpu().numpy(), scales)
    assert v[0, 0] == 0.0 and v[0, 1] == 1.0 and v[0, 2] == 1.0 and v[0, 3] == 2.0 and v[0, 4] == 2.0 and v[0, 5] == 4.0
    assert v[1, 0] == 6.0 and v[1, 1] == 4.0


def test_quantize_range_ends_and_poison(ctx):
    top = float(np.finfo(np.float32).max)
    x = torch.zeros(12, 64)
    x[0, 3] = top; x[1, 3] = -1.5 * 2.0 ** -126; x[2, 40] = 2.0 ** -149; x[3, :] = 3 * 2.0 ** -127
    x[4, 5] = float("nan"); x[5, 6] = float("inf"); x[6, 33] = -float("inf"); x[7, :] = -0.0
    x[8, :32] = 2.0 ** -126; x[9, :32] = 2.0 ** -124; x[10, :] = torch.linspace(0.9, 1.1, 64) * 2.0 ** -125; x[11, 1] = 2.0 ** 127
    m = ctx.mx_quantize(x.cuda(), want_values=True)
    codes, scales, v = ref.quantize(f64(x))
    assert np.array_equal(m.scales.cpu().numpy(), scales) and np.array_equal(m.codes.cpu().numpy(), codes)
    assert np.array_equal(f64(m.values), v, equal_nan=True)
    assert scales[4, 0] == 255 and scales[4, 1] == 0 and np.isnan(v[4, :32]).all() and (v[4, 32:] == 0).all()
    h = torch.tensor([[2.0 ** -24 * k for k in range(32)], [65504.0 - 32 * k for k in range(32)]], dtype=torch.float16)
    h[1, 31] = float("inf")
    m = ctx.mx_quantize(h.cuda(), want_values=True)
    codes, scales, v = ref.quantize(f64(h))
    assert np.array_equal(m.codes.cpu().numpy(), codes) and np.array_equal(m.scales.cpu().numpy(), scales)
    assert np.array_equal(f64(m.values), v, equal_nan=True)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("groups,rows,cols", [(1, 5, 70), (3, 7, 96), (4, 1, 33)])
def test_dequantize(ctx, groups, rows, cols, dtype):
    x = f64(randn(groups * rows, cols, seed=cols))
    codes, scales, v = ref.quantize(x)
    scales[0, 0], v[0, :32] = 255, np.nan
    c = torch.from_numpy(codes).cuda().reshape(groups, rows, -1)
    s = torch.from_numpy(scales).cuda().reshape(groups, rows, -1)
    m = q.MxMatrix(c, s, cols) if groups > 1 else q.MxMatrix(c[0], s[0], cols)
    y = ctx.mx_dequantize(m, DTYPES[dtype])
    assert y.shape[-2:] == (rows, cols)
    want = torch.from_numpy(v).to(torch.float32).to(DTYPES[dtype]).double().numpy().reshape(f64(y).shape)
    assert np.array_equal(f64(y), want, equal_nan=True)


# ---------------------------------------------------------------------------------------- products
def check_product(y, av, wv, bias, dtype):
    want = av @ wv.T + (0 if bias is None else bias)
    got = f64(y)
    nan = np.isnan(av).any(1)[:, None] | np.isnan(wv).any(1)[None, :]
    assert np.array_equal(np.isnan(got), nan)
    bound = ref.product_bound(av, wv, EPS[dtype], want) + (0 if bias is None else 2.0 ** -23 * np.abs(bias))
    assert (np.abs(got - want)[~nan] <= bound[~nan]).all(), float((np.abs(got - want) / bound)[~nan].max())


SIZES = [(1, 1, 1), (1, 8, 32), (2, 3, 33), (1, 1000, 4096), (5, 130, 100), (16, 128, 256), (17, 127, 288), (33, 257, 512),
         (64, 513, 1024), (128, 256, 256), (129, 255, 1056), (200, 300, 25), (333, 1000, 2080), (1, 4096, 25088), (65, 4000, 260),
         (512, 768, 640), (1000, 520, 800), (2050, 300, 100), (3, 2, 0)]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("m,n,k", SIZES)
def test_matmul_sizes(ctx, m, n, k, dtype):
    a, av = pack(f64(randn(m, k, seed=m)) if k else np.zeros((m, 0)))
    w, wv = pack(f64(randn(n, k, seed=n + 1)) if k else np.zeros((n, 0)))
    bias = torch.randn(n, generator=torch.Generator().manual_seed(3)).cuda() if (m + n) % 2 else None
    if dtype == "f16":                                    # keep the sums inside binary16's range
        w = q.MxMatrix(w.codes, (w.scales.int() - 6).clamp(min=0).to(torch.uint8), k)
        wv = ref.values(w.codes.cpu().numpy(), w.scales.cpu().numpy(), k)
    y = ctx.mx_matmul(a, w, bias=bias, out_dtype=DTYPES[dtype])
    check_product(y, av, wv, None if bias is None else f64(bias), dtype)
    assert torch.equal(y, ctx.mx_matmul(a, w, bias=bias, out_dtype=DTYPES[dtype]))


@pytest.mark.parametrize("m,n,k", [(1, 200, 300), (40, 200, 300), (300, 520, 1100)])
def test_matmul_strides_out_and_poisoned_blocks(ctx, m, n, k):
    ax, wx = f64(randn(m, k, seed=1)), f64(randn(n, k, seed=2))
    ax[m // 2, k - 1] = np.nan
    wx[3, 0] = np.inf
    a, av = pack(ax, pad=3)
    w, wv = pack(wx, pad=1)
    big = torch.full((m, n + 5), 7.0, device="cuda")
    y = ctx.mx_matmul(a, w, out=big[:, 2: n + 2])
    check_product(y, av, wv, None, "f32")
    assert (big[:, :2] == 7).all() and (big[:, n + 2:] == 7).all()


@pytest.mark.parametrize("m,n,k", [(1, 64, 128), (130, 300, 512)])
def test_scale_extremes(ctx, m, n, k):
    """Scales at both ends of their range meet so that the products stay finite."""
    a, av = pack(f64(randn(m, k, seed=1)))
    w, wv = pack(f64(randn(n, k, seed=2)))
    lo = q.MxMatrix(a.codes, torch.full_like(a.scales, 1), k)
    hi = q.MxMatrix(w.codes, torch.full_like(w.scales, 252), k)
    check_product(ctx.mx_matmul(lo, hi), ref.values(lo.codes.cpu().numpy(), lo.scales.cpu().numpy(), k),
                  ref.values(hi.codes.cpu().numpy(), hi.scales.cpu().numpy(), k), None, "f32")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("shape,n", [((1, 4096), 1000), ((7, 100), 33), ((2, 9, 256), 130), ((260, 384), 512)])
def test_linear_is_quantize_then_matmul(ctx, shape, n, dtype):
    x = randn(*shape, seed=n, dtype=dtype).cuda()
    w, wv = pack(f64(randn(n, shape[-1], seed=4)) / shape[-1])
    bias = torch.randn(n, device="cuda")
    y = ctx.mx_linear(x, w, bias=bias)
    assert y.shape == (*shape[:-1], n) and y.dtype == x.dtype
    assert torch.equal(y.reshape(-1, n), ctx.mx_matmul(ctx.mx_quantize(x), w, bias=bias, out_dtype=x.dtype))
    _, _, av = ref.quantize(f64(x.reshape(-1, shape[-1])))
    check_product(y.reshape(-1, n), av, wv, f64(bias), dtype)
    assert ctx.mx_linear(x, w, out_dtype=torch.float32).dtype == torch.float32


def experts(groups, n, k, seed=0):
    x = f64(randn(groups * n, k, seed=seed)) / np.sqrt(k)
    codes, scales, v = ref.quantize(x)
    w = q.MxMatrix(torch.from_numpy(codes).cuda().reshape(groups, n, -1), torch.from_numpy(scales).cuda().reshape(groups, n, -1), k)
    return w, v.reshape(groups, n, k)


GROUPS = [([3, 0, 5], 64, 64), ([0, 0, 1], 100, 33), ([1] * 9, 130, 256), ([200, 0, 77, 130, 1], 300, 288), ([0, 700, 0], 256, 512),
          ([16, 17, 0, 31, 64, 2, 9, 0], 1000, 1056), ([1300, 3, 900], 516, 256), ([2] * 40, 40, 96), ([300, 301, 299, 298], 512, 1024)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,n,k", GROUPS)
def test_grouped(ctx, counts, n, k, dtype):
    rows = sum(counts)
    x = randn(rows, k, seed=rows, dtype=dtype).cuda()
    w, wv = experts(len(counts), n, k, seed=n)
    bias = torch.randn(len(counts), n, generator=torch.Generator().manual_seed(1)).cuda()
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), device="cuda")
    y = ctx.mx_linear_grouped(x, offsets, w, bias=bias)
    assert torch.equal(y, ctx.mx_linear_grouped(x, offsets, w, bias=bias))
    _, _, av = ref.quantize(f64(x))
    at = 0
    for g, c in enumerate(counts):
        if c:
            check_product(y[at: at + c], av[at: at + c], wv[g], f64(bias[g]), dtype)
        at += c


@pytest.mark.parametrize("m,n", [(40, 72), (900, 600)])
def test_grouped_rows_outside_and_odd_offsets(ctx, m, n):
    """Rows of no group keep what they held; offsets outside 0..m and decreasing ones are clamped."""
    k = 160
    w, wv = experts(4, n, k)
    x = randn(m, k, seed=9).cuda()
    _, _, av = ref.quantize(f64(x))
    for given, used in (([5, 5, 12, 20, 30], [5, 5, 12, 20, 30]), ([-3, 4, 2, 9, m + 50], [0, 4, 4, 9, m]), ([m, m, m, m, m], [m] * 5), ([m + 7, 0, 1, 2, 3], [m] * 5)):
        out = torch.full((m, n), 3.5, device="cuda")
        ctx.mx_linear_grouped(x, torch.tensor(given, device="cuda"), w, out=out)
        covered = np.zeros(m, bool)
        for g in range(4):
            lo, hi = used[g], used[g + 1]
            covered[lo:hi] = True
            if hi > lo:
                check_product(out[lo:hi], av[lo:hi], wv[g], None, "f32")
        assert (out.cpu().numpy()[~covered] == 3.5).all()


def test_grouped_many_groups(ctx):
    counts = [(i * 7) % 5 for i in range(q.MX_MAX_GROUPS)]
    w, wv = experts(len(counts), 8, 32)
    x = randn(sum(counts), 32, seed=2).cuda()
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), device="cuda")
    y = ctx.mx_linear_grouped(x, offsets, w)
    _, _, av = ref.quantize(f64(x))
    want = np.concatenate([av[o: o + c] @ wv[g].T for g, (o, c) in enumerate(zip(np.concatenate([[0], np.cumsum(counts)]), counts))])
    assert np.abs(f64(y) - want).max() <= 33 * 2.0 ** -23 * (np.abs(av).sum(1).max() * np.abs(wv).max())


# ---------------------------------------------------------------------------------------- cache
def gathered(seqs, table, page):
    return [np.array([table[s][i // page] * page + i % page for i in range(c)], dtype=np.int64) for s, c in enumerate(seqs)]


@pytest.mark.parametrize("fmt", [q.KV_MX4, q.KV_I8])
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("dim,heads,page", [(128, 8, 16), (64, 1, 64), (80, 3, 7), (1, 2, 1), (33, 5, 16), (256, 2, 32), (300, 1, 5), (576, 2, 16)])
def test_cache_round_trip(ctx, dim, heads, page, dtype, fmt):
    seqs = [1, 5 * page + 3, 0, page, 2 * page - 1]
    rng = np.random.RandomState(dim)
    need = [-(-c // page) for c in seqs]
    ids = rng.permutation(sum(need) + 2).astype(np.int32)
    table = np.full((len(seqs), max(need)), -1, np.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = ids[at: at + n]
        at += n
    slots = np.concatenate([x for x in gathered(seqs, table, page) if len(x)])
    T = len(slots)
    fused = randn(T, 3 * heads, dim, seed=dim, dtype=dtype)
    if T > 4:
        fused[2, 1, 0] = 0; fused[3] = 0
        fused[4, heads, dim - 1] = float("nan")
    fused = fused.cuda()
    k, v = fused[:, heads: 2 * heads], fused[:, 2 * heads:]
    cache = ctx.kv_empty(sum(need) + 2, page, heads, dim, fmt)
    for t in (cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales):
        t.fill_(1)
    order = rng.permutation(T)
    ctx.kv_write(cache, k[torch.from_numpy(order).cuda()], v[torch.from_numpy(order).cuda()], torch.from_numpy(slots[order]).cuda())
    starts = torch.tensor(np.concatenate([[0], np.cumsum(seqs)]), device="cuda")
    got = ctx.kv_read(cache, torch.from_numpy(table).cuda(), starts, T, DTYPES[dtype])
    untouched = np.ones(cache.k_codes.shape[0] * page, bool)
    untouched[slots] = False
    for new, codes, scales, y in ((k, cache.k_codes, cache.k_scales, got[0]), (v, cache.v_codes, cache.v_scales, got[1])):
        x = f64(new).reshape(T * heads, dim)
        flat_c, flat_s = codes.flatten(0, 1).cpu().numpy(), scales.flatten(0, 1).cpu().numpy()
        if fmt == q.KV_MX4:
            wc, ws, wv = ref.quantize(x)
            assert np.array_equal(flat_c[slots].reshape(T * heads, -1), wc) and np.array_equal(flat_s[slots].reshape(T * heads, -1), ws)
        else:
            wc, ws = ref.quantize_i8(x)
            assert np.array_equal(flat_c[slots].reshape(T * heads, -1), wc)
            assert np.array_equal(flat_s[slots].reshape(-1), ws, equal_nan=True)
            wv = (wc.astype(np.float32) * ws[:, None]).astype(np.float64)
        want = torch.from_numpy(wv).float().to(DTYPES[dtype]).double().numpy()
        assert np.array_equal(f64(y).reshape(T * heads, dim), want, equal_nan=True)
        assert (flat_c[untouched] == 1).all() and (flat_s[untouched] == 1).all()


@pytest.mark.parametrize("fmt", [q.KV_MX4, q.KV_I8])
def test_cache_skips_and_fills(ctx, fmt):
    """Negative and too large slots are not written; pages out of range, tables too short and rows past the last sequence read as zeros."""
    heads, dim, page, pages = 2, 96, 4, 3
    cache = ctx.kv_empty(pages, page, heads, dim, fmt)
    for t in (cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales):
        t.fill_(2)
    x = randn(5, heads, dim, seed=1, dtype="bf16").cuda()
    ctx.kv_write(cache, x, x, torch.tensor([-1, 12, 3, -(1 << 40), 1 << 40], device="cuda"))
    c = cache.k_codes.flatten(0, 1)
    keep = torch.ones(12, dtype=torch.bool, device="cuda")
    keep[3] = False
    assert (c[keep] == 2).all() and not (c[3] == 2).all()
    table = torch.tensor([[0, 9], [-5, 1]], dtype=torch.int32, device="cuda")
    starts = torch.tensor([2, 12, 17], device="cuda")              # rows 0..1 before, 17..19 behind every sequence
    k, v = ctx.kv_read(cache, table, starts, 20)
    zero = (k == 0).flatten(1).all(1).cpu().numpy()
    # sequence 0: tokens 0..3 in page 0, 4..7 in page 9 (none), 8..9 past the table's row; sequence 1: page -5 (none), then page 1
    assert zero.tolist() == [True] * 2 + [False] * 4 + [True] * 4 + [True] * 2 + [True] * 4 + [False] + [True] * 3
    assert torch.equal(k, v)
    assert ctx.kv_read(cache, table, starts, 0)[0].shape == (0, heads, dim)


def test_cache_past_32_bits(ctx):
    """Slots whose byte offset passes 2^32: a cache of 4.4 GB of key codes (and as much for the values)."""
    heads, dim, page = 8, 128, 64
    pages = (1 << 32) // (heads * dim * page) + 4000
    cache = ctx.kv_empty(pages, page, heads, dim, q.KV_I8)
    x = randn(3, heads, dim, seed=3, dtype="bf16").cuda()
    slots = torch.tensor([pages * page - 1, 5, (pages - 7) * page], device="cuda")
    cache.k_codes[0].zero_()
    ctx.kv_write(cache, x, x, slots)
    table = torch.tensor([[pages - 1], [pages - 7], [0]], dtype=torch.int32, device="cuda")
    k, v = ctx.kv_read(cache, table, torch.tensor([0, page, page + 1, page + 7], device="cuda"), page + 7)
    codes, step = ref.quantize_i8(f64(x).reshape(3 * heads, dim))
    want = torch.from_numpy(codes.astype(np.float32) * step[:, None]).bfloat16().reshape(3, heads, dim).cuda()
    assert torch.equal(k[page - 1], want[0]) and torch.equal(k[page], want[2]) and torch.equal(v[page + 6], want[1])


def test_other_stream(ctx):
    """A context on its own stream: inputs made on torch's stream, results read after the context's stream is waited for."""
    s = torch.cuda.Stream()
    c = q.Context(0, stream=s)
    x = randn(64, 512, seed=1, dtype="bf16").cuda()
    w, _ = pack(f64(randn(256, 512, seed=2)))
    want = ctx.mx_linear(x, w)
    torch.cuda.current_stream().synchronize()
    y = c.mx_linear(x, w)
    m = c.mx_quantize(x, want_values=True)
    s.synchronize()
    assert torch.equal(y, want) and torch.equal(m.codes, ctx.mx_quantize(x).codes)
    c.close()


def test_captured_in_a_graph(ctx):
    """Calls whose scratch is sized can be captured and replayed on new inputs."""
    s = torch.cuda.Stream()
    c = q.Context(0, stream=s)
    w, _ = pack(f64(randn(300, 256, seed=2)))
    with torch.cuda.stream(s):
        x = randn(9, 256, seed=1, dtype="bf16").cuda()
        y = torch.empty(9, 300, dtype=torch.bfloat16, device="cuda")
        c.mx_linear(x, w, out=y)
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            c.mx_linear(x, w, out=y)
        x.copy_(randn(9, 256, seed=7, dtype="bf16"))
        g.replay()
        s.synchronize()
    assert torch.equal(y, ctx.mx_linear(x, w))
    del g
    c.close()


# ---------------------------------------------------------------------------------------- refusals
def status(fn):
    with pytest.raises(q.binding.Qv2Error) as e:
        fn()
    return e.value.status


def test_refusals(ctx):
    import ctypes as C
    L, B = q.lib(), q.binding
    x = torch.zeros(4, 64, device="cuda")
    m = ctx.mx_empty(4, 64)
    w3 = ctx.mx_empty(8, 64, groups=2)
    raw = lambda **kw: B.MxMatrixC(**{**{f: getattr(m._c, f) for f, _ in B.MxMatrixC._fields_}, **kw})
    quant = lambda mat, xp=x.data_ptr(), t=q.IN_F32, ld=64, vp=None, vld=64: L.qv2_mx_quantize(ctx._h, xp, t, ld, mat, vp, vld)
    assert quant(m._c) == 0
    assert quant(None) == -2 and quant(m._c, xp=None) == -2 and quant(raw(codes=None)) == -2
    assert quant(m._c, t=7) == -1 and quant(m._c, ld=63) == -1 and quant(raw(groups=2)) == -4 and quant(raw(groups=0)) == -1
    assert quant(raw(codes=m._c.codes + 8)) == -3 and quant(raw(codes_ld=40)) == -3 and quant(raw(codes_ld=16)) == -1
    assert quant(raw(scales_ld=1)) == -1 and quant(m._c, xp=x.data_ptr() + 2) == -3 and quant(raw(cols=1 << 27)) == -4
    assert quant(m._c, vp=x.data_ptr() + 2) == -3 and quant(m._c, vp=x.data_ptr(), vld=3) == -1
    y = torch.zeros(4, 8, device="cuda")
    prod = lambda a=m._c, w=m._c, b=None, o=None, yp=y.data_ptr(), t=q.IN_F32, ld=8: L.qv2_mx_matmul(ctx._h, a, w, b, o, yp, t, ld)
    assert prod() == 0 and prod(a=None) == -2 and prod(w=None) == -2 and prod(yp=None) == -2
    assert prod(w=w3._c) == -1 and prod(a=w3._c) == -4 and prod(a=raw(cols=32)) == -1 and prod(ld=3) == -1 and prod(t=1) == -1
    assert prod(b=y.data_ptr() + 2) == -3 and prod(o=y.data_ptr() + 4) == -3 and prod(yp=y.data_ptr() + 1) == -3
    assert prod(w=raw(groups=1025), o=y.data_ptr()) == -4 and prod(a=raw(rows=(1 << 30) + 1)) == -4
    assert prod(w=raw(groups=2, codes_gs=16, scales_gs=64), o=y.data_ptr()) == -1
    assert L.qv2_mx_linear(ctx._h, None, q.IN_F32, 64, 4, m._c, None, None, y.data_ptr(), q.IN_F32, 8) == -2
    assert L.qv2_mx_linear(None, x.data_ptr(), q.IN_F32, 64, 4, m._c, None, None, y.data_ptr(), q.IN_F32, 8) == -2
    assert L.qv2_mx_dequantize(ctx._h, m._c, y.data_ptr(), q.IN_F32, 8) == -1
    cache = ctx.kv_empty(2, 4, 2, 32, q.KV_MX4)
    kraw = lambda **kw: B.KvCacheC(**{**{f: getattr(cache._c, f) for f, _ in B.KvCacheC._fields_}, **kw})
    slots = torch.zeros(1, dtype=torch.int64, device="cuda")
    wr = lambda c=cache._c, k=x.data_ptr(), t=q.IN_F32, s=slots.data_ptr(): L.qv2_kv_write(ctx._h, c, k, 64, 32, x.data_ptr(), 64, 32, t, 1, s)
    assert wr() == 0 and wr(c=None) == -2 and wr(k=None) == -2 and wr(s=None) == -2 and wr(t=5) == -1 and wr(s=slots.data_ptr() + 4) == -3
    assert wr(c=kraw(format=2)) == -1 and wr(c=kraw(page_size=0)) == -1 and wr(c=kraw(head_dim=5000)) == -4 and wr(c=kraw(k_codes=cache._c.k_codes + 4)) == -3
    assert wr(c=kraw(pages=1 << 31)) == -4 and wr(c=kraw(v_scales=None)) == -2
    out = torch.zeros(4, 2, 32, device="cuda")
    rd = lambda c=cache._c, st=slots.data_ptr(), n=4, k=out.data_ptr(), t=q.IN_F32: L.qv2_kv_read(ctx._h, c, None, 0, 0, st, n, k, None, t)
    assert rd() == 0 and rd(st=None) == -2 and rd(k=None) == -2 and rd(n=1 << 31) == -4 and rd(t=9) == -1
    torch.cuda.synchronize()


def test_python_refusals(ctx):
    x = torch.zeros(4, 64, device="cuda")
    w = ctx.mx_empty(8, 64)
    w3 = ctx.mx_empty(8, 64, groups=2)
    off = torch.zeros(3, dtype=torch.int64, device="cuda")
    for fn, err in ((lambda: ctx.mx_quantize(x.int()), TypeError), (lambda: ctx.mx_quantize(x.cpu()), ValueError),
                    (lambda: ctx.mx_linear(x[:, :32], w), ValueError), (lambda: ctx.mx_linear(x, w3), ValueError),
                    (lambda: ctx.mx_linear(x, w, bias=x[0]), ValueError), (lambda: ctx.mx_linear(x, w, out_dtype=torch.int32), TypeError),
                    (lambda: ctx.mx_linear_grouped(x, off, w), ValueError), (lambda: ctx.mx_linear_grouped(x, off[:2], w3), ValueError),
                    (lambda: ctx.mx_linear_grouped(x, off.int(), w3), ValueError), (lambda: ctx.mx_linear(x, w, out=torch.zeros(4, 7, device="cuda")), ValueError),
                    (lambda: ctx.mx_quantize(torch.zeros(64, 4, device="cuda").t()), ValueError),
                    (lambda: q.MxMatrix(w.codes, w.scales, 96), ValueError), (lambda: q.MxMatrix(w.codes.int(), w.scales, 64), TypeError)):
        with pytest.raises(err):
            fn()
    cache = ctx.kv_empty(2, 4, 2, 32, q.KV_I8)
    k, slots = torch.zeros(1, 2, 32, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    for fn, err in ((lambda: ctx.kv_write(cache, k, k.half(), slots), TypeError), (lambda: ctx.kv_write(cache, k, k[:, :1], slots), ValueError),
                    (lambda: ctx.kv_write(cache, k, k, slots.int()), ValueError), (lambda: ctx.kv_read(cache, slots, slots, 1), ValueError),
                    (lambda: q.KvCache(5, 32, cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales), ValueError),
                    (lambda: q.KvCache(q.KV_I8, 33, cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales), ValueError)):
        with pytest.raises(err):
            fn()


# ---------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("m,n,k", [(3000, 1001, 96), (2600, 1302, 300), (2500, 1304, 100)])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_many_rows_with_unaligned_results(ctx, m, n, k, dtype):
    """The many-row form where rows of the result start at multiples of 2, 4, 8 and 16 bytes."""
    a, av = pack(f64(randn(m, k, seed=m)))
    w, wv = pack(f64(randn(n, k, seed=n)) / 64)
    check_product(ctx.mx_matmul(a, w, out_dtype=DTYPES[dtype]), av, wv, None, dtype)


def test_strided_keys_on_odd_addresses(ctx):
    buf = randn(9 * 3 * 70 + 1, seed=1, dtype="bf16").cuda()
    k = buf[1:].as_strided((9, 3, 67), (210, 70, 1))
    for fmt in (q.KV_MX4, q.KV_I8):
        cache = ctx.kv_empty(1, 9, 3, 67, fmt)
        ctx.kv_write(cache, k, k, torch.arange(9, device="cuda"))
        one = ctx.kv_empty(1, 9, 3, 67, fmt)
        ctx.kv_write(one, k.contiguous(), k.contiguous(), torch.arange(9, device="cuda"))
        assert torch.equal(cache.k_codes, one.k_codes) and torch.equal(cache.v_scales, one.v_scales)


@pytest.mark.parametrize("fmt", [q.KV_MX4, q.KV_I8])
def test_example_block(ctx, fmt):
    """The example's block: every layer's 4-bit weights and outputs stay near FP32 (rounding to 4 bits with a scale per
    32 leaves 17 to 19 dB per operand of normal values, two operands and a chain of layers some dB less)."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "narrow_block.py")
    spec = importlib.util.spec_from_file_location("narrow_block", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    stages, block = ex.run(ctx, fmt)
    w, x, order = ex.report(ctx, stages, block)
    assert all(v > 15 for v in w) and all(v > 8 for v in x), (w, x)
    assert sorted(order) == list(range(len(stages)))
