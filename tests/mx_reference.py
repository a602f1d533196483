"""The microscaled 4-bit format and the quantized cache in numpy, 64 bits, straight from their definitions: every grid
point is tried, nothing is computed by bit tricks."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize(x):
    """x float64 [rows, cols] -> codes uint8 [rows, 16*blocks], scales uint8 [rows, blocks], values float64 [rows, cols]."""
    rows, cols = x.shape
    blocks = -(-cols // 32)
    pad = np.zeros((rows, blocks * 32))
    pad[:, :cols] = x
    b = pad.reshape(rows, blocks, 32)
    bad = ~np.isfinite(b).all(-1)
    top = np.where(bad, 1.0, np.abs(np.where(np.isfinite(b), b, 0)).max(-1))
    _, ex = np.frexp(np.where(top > 0, top, 1.0))            # top = m * 2^ex, 1/2 <= m < 1
    e = np.where(top > 0, np.clip(ex - 1 - 2, -127, 127), -127)
    t = np.abs(np.where(bad[..., None], 0, b)) / np.exp2(e)[..., None]
    dist = np.abs(t[..., None] - GRID)
    near = dist == dist.min(-1, keepdims=True)
    first, last = near.argmax(-1), 7 - near[..., ::-1].argmax(-1)
    code = np.where((first != last) & (first % 2 == 1), last, first)
    sign = np.signbit(b) & ~bad[..., None]
    value = np.where(sign, -1.0, 1.0) * GRID[code] * np.exp2(e)[..., None]
    value = np.where(bad[..., None], np.nan, value).reshape(rows, blocks * 32)[:, :cols]
    nib = (code + 8 * sign).astype(np.uint8).reshape(rows, blocks * 32)
    return nib[:, 0::2] | (nib[:, 1::2] << 4), np.where(bad, 255, e + 127).astype(np.uint8), value


def values(codes, scales, cols):
    """What packed codes and scale bytes stand for, float64 [..., cols]."""
    nib = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    v = np.where(nib >= 8, -1.0, 1.0) * GRID[nib & 7]
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (v.reshape(*scales.shape, 32) * s[..., None]).reshape(*codes.shape[:-1], -1)[..., :cols]


def quantize_i8(x):
    """x float32 [..., dim] -> int8 codes, float32 steps: the symmetric quantizer, one binary32 rounding per operation."""
    x = x.astype(np.float32)
    finite = np.isfinite(x).all(-1)
    R = np.abs(np.where(finite[..., None], x, 0)).max(-1).astype(np.float32)
    with np.errstate(all="ignore"):
        step, inv = R / np.float32(127), np.float32(127) / R
    ok = (R > 0) & np.isfinite(inv) & (step > 0)
    step, inv = np.where(ok, step, np.float32(1)), np.where(ok, inv, np.float32(1))
    q = np.clip(np.rint(np.where(finite[..., None], x, 0) * inv[..., None]), -127, 127).astype(np.int8)
    return q, np.where(finite, step, np.float32("nan")).astype(np.float32)


def product_bound(av, wv, out_eps, y):
    """How far a product of exact terms may be from float64's: each of at most cols + 1 additions in binary32 loses at
    most 2^-23 of the running magnitude (an adder that truncates; one that rounds loses half), and the result is
    rounded once to a type of relative step out_eps (half of it per rounding)."""
    k = av.shape[1]
    mag = np.abs(np.nan_to_num(av)) @ np.abs(np.nan_to_num(wv)).T
    return (k + 1) * 2.0 ** -23 * mag + out_eps / 2 * np.abs(np.nan_to_num(y)) + 2.0 ** -25
