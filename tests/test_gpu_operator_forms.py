"""Every form that the 4-bit operators and the cache can take on this device, at sizes that make each of them turn its
rings, its second accumulator and its tables over: which form a size takes is asked of the library, so that a changed
rule cannot leave a form untested unnoticed.  Plain references in 64 bits."""
import numpy as np
import pytest
import torch

import mx_reference as ref
import paper_2501_07161_b200 as q

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = {"f32": 2.0 ** -23, "f16": 2.0 ** -10, "bf16": 2.0 ** -7}
GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], dtype=torch.float64)


@pytest.fixture(scope="module")
def ctx():
    c = q.Context(0)
    yield c
    c.close()


def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def values(m):
    """What a packed matrix stands for, float64 on its device (plain torch)."""
    codes, scales = m.codes.long(), m.scales.double()
    v = GRID.to(codes.device)[torch.stack((codes & 15, codes >> 4), -1).flatten(-2)]
    return (v.unflatten(-1, (-1, 32)) * torch.exp2(scales - 127).unsqueeze(-1)).flatten(-2)[..., : m.cols]


def packed(rows, cols, seed, groups=0):
    """Random codes, scales 2^-3 .. 2^0; codes behind the last column are zero, as rounding leaves them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    lead, blocks = ((groups,) if groups else ()), -(-cols // 32)
    codes = torch.randint(0, 256, (*lead, rows, 16 * blocks), dtype=torch.uint8, device="cuda", generator=g)
    if cols % 32:
        codes[..., cols // 2 + cols % 2:] = 0
        if cols % 2:
            codes[..., cols // 2] &= 15
    scales = torch.randint(124, 128, (*lead, rows, blocks), dtype=torch.uint8, device="cuda", generator=g)
    return q.MxMatrix(codes, scales, cols)


def check(got, a, w, bias, dtype):
    """got [m, n] against a w^T + bias in 64 bits, within the bound of binary32 sums (mx_reference.product_bound)."""
    y, mag = a @ w.T, a.abs() @ w.abs().T
    if bias is not None:
        y = y + bias.double()
    bound = (a.shape[1] + 1) * 2.0 ** -23 * mag + EPS[dtype] / 2 * y.abs() + 2.0 ** -25 + (0 if bias is None else 2.0 ** -23 * bias.double().abs())
    off = (got.double() - y).abs()
    assert bool((off <= bound).all()), float((off / bound).max())


def activations(rows, cols, seed, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(rows, cols, device="cuda", generator=g) * torch.exp(0.5 * torch.randn(cols, device="cuda", generator=g)) / 8).to(DTYPES[dtype])


def rounded(x):
    """The 4-bit values of x by the reference, float64 on the device."""
    parts = [torch.from_numpy(ref.quantize(p.double().cpu().numpy())[2]) for p in x.split(512)]
    return torch.cat(parts).cuda()


# ---------------------------------------------------------------------------------------- products
# 20 x 9 tiles of 256 x 256: more than two for each of 74 pairs of CTAs; 6, 7 and 2 steps of 256 columns beside 5 stages
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("k,with_bias", [(1536, True), (1700, True), (1700, False), (300, True)])
def test_many_rows_dense(ctx, k, with_bias, dtype):
    m, n = 5000, 2100
    form, tiles = q.mx_form(m, n, 1, sms())
    assert form == 256 and tiles > 2 * (sms() // 2)
    a, w = packed(m, k, 1), packed(n, k, 2)
    bias = torch.randn(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)) if with_bias else None
    y = ctx.mx_matmul(a, w, bias=bias, out_dtype=DTYPES[dtype])
    check(y, values(a), values(w), bias, dtype)
    assert torch.equal(y, ctx.mx_matmul(a, w, bias=bias, out_dtype=DTYPES[dtype]))


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_many_rows_linear(ctx, dtype):
    """The product begins while the activations are being rounded."""
    m, n, k = 5000, 2104, 1700
    assert q.mx_form(m, n, 1, sms())[0] == 256
    x, w = activations(m, k, 1, dtype), packed(n, k, 2)
    bias = torch.randn(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(4))
    y = ctx.mx_linear(x, w, bias=bias)
    check(y, rounded(x), values(w), bias, dtype)
    assert torch.equal(y, ctx.mx_matmul(ctx.mx_quantize(x), w, bias=bias, out_dtype=x.dtype))
    out = torch.empty_like(y)
    for _ in range(20):                                    # back to back: each rounds into the scratch that the last one read
        assert ctx.mx_linear(x, w, bias=bias, out=out) is out
        assert torch.equal(out, y)


# more than 8 row tiles in a group (bands), groups that end inside a tile, empty ones and one of a single row
MANY = [2305, 0, 1, 700, 333, 256, 0, 900]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("call", ["matmul", "linear"])
@pytest.mark.parametrize("n,k,with_bias", [(2100, 1536, True), (2104, 1700, True), (2101, 700, False)])
def test_many_rows_grouped(ctx, n, k, with_bias, call, dtype):
    m, groups = sum(MANY), len(MANY)
    form, tiles = q.mx_form(m, n, groups, sms())
    assert form == 256 and sum(-(-c // 256) for c in MANY) * -(-n // 256) > 2 * (sms() // 2)
    w = packed(n, k, 5, groups)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(MANY)]), device="cuda")
    bias = torch.randn(groups, n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(6)) if with_bias else None
    if call == "matmul":
        a = packed(m, k, 7)
        av, y = values(a), ctx.mx_matmul(a, w, bias=bias, offsets=offsets, out_dtype=DTYPES[dtype])
    else:
        x = activations(m, k, 8, dtype)
        av, y = rounded(x), ctx.mx_linear_grouped(x, offsets, w, bias=bias)
    wv, at = values(w), 0
    for g, c in enumerate(MANY):
        check(y[at: at + c], av[at: at + c], wv[g], None if bias is None else bias[g], dtype)
        at += c


def test_many_rows_with_poisoned_blocks(ctx):
    m, n, k = 5000, 2100, 1536
    a, w = packed(m, k, 1), packed(n, k, 2)
    clean = ctx.mx_matmul(a, w)
    rows, cols = [0, 255, 256, 2600, 4999], [3, 191, 192, 255, 2099]
    a.scales[rows, 7], w.scales[cols, 40] = 255, 255
    y = ctx.mx_matmul(a, w)
    bad = torch.zeros(m, n, dtype=torch.bool, device="cuda")
    bad[rows], bad[:, cols] = True, True
    assert torch.equal(y.isnan(), bad) and torch.equal(y[~bad], clean[~bad])


# dense and grouped, narrow forms: more columns than the ring has stages (9, 8, 7, 5), with the columns whole and cut, one
# tile and several to a CTA
DENSE = [(3, 300, 2600, 16), (20, 700, 2300, 32), (40, 600, 2100, 64), (100, 500, 2600, 32), (333, 1000, 4096, 32), (640, 1700, 2500, 64),
         (1200, 1100, 1700, 128), (1250, 1100, 1536, 128), (1280, 1152, 2816, 128)]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("m,n,k,form", DENSE)
def test_narrow_forms_dense(ctx, m, n, k, form, dtype):
    assert q.mx_form(m, n, 1, sms())[0] == form
    x, w = activations(m, k, m, dtype), packed(n, k, n)
    bias = torch.randn(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    a = ctx.mx_quantize(x)
    y = ctx.mx_matmul(a, w, bias=bias, out_dtype=DTYPES[dtype])
    check(y, values(a), values(w), bias, dtype)
    assert torch.equal(y, ctx.mx_linear(x, w, bias=bias))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("counts,n,k,form", [([5, 0, 30, 16, 1, 17, 9, 0, 40, 2, 3, 33], 2000, 2600, 16), ([31, 0, 64, 33, 1, 17, 40, 60], 2500, 2300, 32),
                                             ([64, 65, 0, 128, 1, 90, 30, 100], 2500, 2100, 64), ([300, 0, 1, 250], 1500, 1700, 128)])
def test_narrow_forms_grouped(ctx, counts, n, k, form, dtype):
    groups, m = len(counts), sum(counts)
    assert q.mx_form(m, n, groups, sms())[0] == form
    x, w = activations(m, k, m, dtype), packed(n, k, n, groups)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), device="cuda")
    bias = torch.randn(groups, n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    a = ctx.mx_quantize(x)
    y = ctx.mx_linear_grouped(x, offsets, w, bias=bias)
    av, wv, at = values(a), values(w), 0
    for g, c in enumerate(counts):
        check(y[at: at + c], av[at: at + c], wv[g], bias[g], dtype)
        at += c
    assert torch.equal(y, ctx.mx_matmul(a, w, bias=bias, offsets=offsets, out_dtype=DTYPES[dtype]))


# ---------------------------------------------------------------------------------------- rounding
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("cols,offset", [(1000, 0), (999, 0), (1000, 1)])
def test_rounding_of_many_rows(ctx, cols, offset, dtype):
    """Enough chunks of eight for the form with four loads in flight per thread; aligned rows, odd lengths, odd addresses."""
    rows = sms() * 8 * 256 // (4 * -(-cols // 32)) + 1003
    x = activations(1, rows * cols + offset, 1, dtype)[0, offset:].reshape(rows, cols)
    want = [ref.quantize(p.double().cpu().numpy()) for p in x.split(512)]
    for want_values in (False, True):
        m = ctx.mx_quantize(x, want_values=want_values)
        assert np.array_equal(m.codes.cpu().numpy(), np.concatenate([w[0] for w in want]))
        assert np.array_equal(m.scales.cpu().numpy(), np.concatenate([w[1] for w in want]))
        if want_values:
            v = torch.from_numpy(np.concatenate([w[2] for w in want])).float().to(x.dtype)
            assert torch.equal(m.values.cpu(), v)
    for back in DTYPES.values():
        assert torch.equal(ctx.mx_dequantize(m, back), torch.from_numpy(np.concatenate([w[2] for w in want])).float().to(back).cuda())


def test_rounding_past_32_bits(ctx):
    """A matrix of 8.6 thousand million elements: the rows are taken in two slices, and offsets pass 2^32 elements."""
    cols, per = 64, 1 << 27                                # 2^30 chunks to a slice, 8 to a row
    rows = per + 70
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 5, (1 << 26) - 1, (1 << 26) + 1, per - 1, per, per + 1, rows - 1], device="cuda")
    x[at] = activations(8, cols, 1, "bf16")
    m = ctx.mx_quantize(x)
    codes, scales, v = ref.quantize(x[at].double().cpu().numpy())
    assert np.array_equal(m.codes[at].cpu().numpy(), codes) and np.array_equal(m.scales[at].cpu().numpy(), scales)
    assert int((m.scales != 0).sum()) == int((scales != 0).sum())
    del x
    y = ctx.mx_dequantize(m, torch.bfloat16)
    assert np.array_equal(y[at].double().cpu().numpy(), v)
    y[at] = 0
    assert not bool(y.any())


# ---------------------------------------------------------------------------------------- cache
@pytest.mark.parametrize("fmt", [q.KV_MX4, q.KV_I8])
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("dim,heads", [(64, 8), (128, 4), (256, 2), (300, 3), (80, 5), (67, 2), (576, 1)])
def test_cache_written_by_many_rows(ctx, dim, heads, dtype, fmt):
    """Enough rows for the forms with several in flight per thread, every width of row, keys and values strided and (odd dims)
    on any address, a few tokens without a slot."""
    page = 16
    tokens = sms() * 8 * 128 // (-(-dim // 8) * heads) + 517
    pages = -(-tokens // page) + 3
    g = torch.Generator(device="cuda").manual_seed(dim)
    fused = activations(tokens, 3 * heads * dim, dim, dtype).view(tokens, 3 * heads, dim)
    k, v = fused[:, heads: 2 * heads], fused[:, 2 * heads:]
    cache = ctx.kv_empty(pages, page, heads, dim, fmt)
    for t in (cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales):
        t.fill_(1)
    slots = torch.randperm(pages * page, device="cuda", generator=g)[:tokens]
    slots[::97] = -1
    ctx.kv_write(cache, k, v, slots)
    live = slots >= 0
    untouched = torch.ones(pages * page, dtype=torch.bool, device="cuda")
    untouched[slots[live]] = False
    for new, codes, scales in ((k, cache.k_codes.flatten(0, 1), cache.k_scales.flatten(0, 1)), (v, cache.v_codes.flatten(0, 1), cache.v_scales.flatten(0, 1))):
        x = new[live].reshape(-1, dim)
        if fmt == q.KV_MX4:
            parts = [ref.quantize(p.double().cpu().numpy()) for p in x.split(4096)]
            wc, ws = (np.concatenate([p[i] for p in parts]) for i in (0, 1))
        else:
            wc, ws = ref.quantize_i8(x.float().cpu().numpy())
        assert np.array_equal(codes[slots[live]].reshape(x.shape[0], -1).cpu().numpy(), wc)
        assert np.array_equal(scales[slots[live]].reshape(ws.shape).cpu().numpy(), ws)
        assert bool((codes[untouched] == 1).all()) and bool((scales[untouched] == 1).all())


@pytest.mark.parametrize("fmt", [q.KV_MX4, q.KV_I8])
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("dim,heads,page", [(64, 1, 16), (16, 1, 5), (33, 1, 7), (128, 2, 64), (40, 3, 16)])
def test_cache_read_in_long_runs(ctx, dim, heads, page, dtype, fmt):
    """Enough tokens for runs of more than 32 per CTA, over many short, some empty and a few long sequences; rows before the
    first sequence and behind the last one."""
    rng = np.random.RandomState(dim)
    lens = rng.randint(0, 40, 6000)
    lens[rng.rand(6000) < 0.3] = 0
    lens[100:140] = 0
    lens[50], lens[3000], lens[5999] = 3001, 129, 0
    before, after = 45, 77
    total = before + int(lens.sum()) + after
    cpr = dim // 32 if dim % 32 == 0 else dim // 16 if dim % 16 == 0 else -(-dim // 8)
    assert total // (4 * sms()) > 64 and 131072 // 32 // (cpr * heads) > 32          # tokens of a CTA
    starts = before + np.concatenate([[0], np.cumsum(lens)])
    need = -(-lens // page)
    pages = int(need.sum()) + 2
    ids = rng.permutation(pages)
    table = np.full((len(lens), need.max()), -1, np.int32)
    slot, at = np.full(total, -1, np.int64), 0
    for s, n in enumerate(need):
        table[s, :n] = ids[at: at + n]
        at += n
        i = np.arange(lens[s])
        slot[starts[s]: starts[s] + lens[s]] = table[s, i // page].astype(np.int64) * page + i % page
    g = torch.Generator(device="cuda").manual_seed(dim)
    cache = ctx.kv_empty(pages, page, heads, dim, fmt)
    for codes, scales in ((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales)):
        codes.copy_(torch.randint(-127, 128, codes.shape, device="cuda", generator=g).to(codes.dtype))
        scales.copy_(torch.randint(120, 130, scales.shape, device="cuda", generator=g) if fmt == q.KV_MX4 else torch.rand(scales.shape, device="cuda", generator=g))
    got = ctx.kv_read(cache, torch.from_numpy(table).cuda(), torch.from_numpy(starts).cuda(), total, DTYPES[dtype])
    at = torch.from_numpy(np.maximum(slot, 0)).cuda()
    none = torch.from_numpy(slot < 0).cuda()
    for codes, scales, y in ((cache.k_codes, cache.k_scales, got[0]), (cache.v_codes, cache.v_scales, got[1])):
        if fmt == q.KV_MX4:
            v = values(q.MxMatrix(codes.flatten(0, 2), scales.flatten(0, 2), dim)).float().view(-1, heads, dim)[at]
        else:
            v = codes.flatten(0, 1)[at].float() * scales.flatten(0, 1)[at].unsqueeze(-1)
        v[none] = 0
        assert torch.equal(y, v.to(DTYPES[dtype]))


@pytest.mark.parametrize("m", [3, 100, 700])
@pytest.mark.parametrize("k", [33, 1000, 2101])
def test_weights_may_hold_anything_behind_their_last_column(ctx, m, k):
    """The activations' codes are zero there, so a weight from elsewhere need not be; dequantizing does not look there."""
    w = packed(200, k, 1)
    g = torch.Generator(device="cuda").manual_seed(2)
    dirty = torch.randint(0, 256, w.codes.shape, dtype=torch.uint8, device="cuda", generator=g)
    full, half = k // 2, k % 2
    dirty[:, :full] = w.codes[:, :full]
    if half:
        dirty[:, full] = (w.codes[:, full] & 15) | (dirty[:, full] & 240)
    other = q.MxMatrix(dirty, w.scales, k)
    assert not torch.equal(dirty, w.codes)
    x = activations(m, k, 3, "bf16")
    assert torch.equal(ctx.mx_linear(x, other), ctx.mx_linear(x, w))
    assert torch.equal(ctx.mx_matmul(ctx.mx_quantize(x), other), ctx.mx_matmul(ctx.mx_quantize(x), w))
    assert torch.equal(ctx.mx_dequantize(other), ctx.mx_dequantize(w))


def test_grouped_product_without_offsets_is_refused(ctx):
    with pytest.raises(ValueError):
        ctx.mx_linear_grouped(activations(4, 64, 1, "bf16"), None, packed(8, 64, 2, groups=2))
