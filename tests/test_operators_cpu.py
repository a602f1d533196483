"""CPU-side checks of the 4-bit operators and the quantized cache: struct layouts, the division rule of their kernels, and the
reference they are tested against (numpy, no GPU)."""
import ctypes as C
import random

import numpy as np
import pytest
import torch

import mx_reference as ref
import paper_2501_07161_b200 as q
from paper_2501_07161_b200 import binding as B


def test_struct_layouts():
    assert C.sizeof(B.MxMatrixC) == 72 and B.MxMatrixC.groups.offset == 16 and B.MxMatrixC.scales_gs.offset == 64
    assert C.sizeof(B.KvCacheC) == 56 and B.KvCacheC.pages.offset == 32 and B.KvCacheC.format.offset == 52
    assert q.lib().qv2_status_string(-9).startswith(b"QV2_ERR_TIMEOUT")


def fast_div(n, d):
    """The kernels' division: one wide product and a shift."""
    k = 0
    while (1 << k) < d:
        k += 1
    s = 31 + k
    m = ((1 << s) + d - 1) // d
    assert m < 1 << 32
    return (n * m) >> s


def test_fast_division_is_exact_below_2_31():
    rng = random.Random(1)
    divisors = list(range(1, 70)) + [(1 << k) + e for k in range(7, 31) for e in (-1, 0, 1)] + [rng.randrange(1, 1 << 30) for _ in range(200)]
    for d in divisors:
        top = (1 << 31) - 1
        for n in {0, 1, d - 1, d, d + 1, top, top - 1, top // d * d, max(0, top // d * d - 1), *(rng.randrange(1 << 31) for _ in range(20))}:
            assert fast_div(n, d) == n // d, (n, d)


def test_reference_rounds_to_the_nearest_grid_point():
    rng = np.random.RandomState(0)
    x = rng.randn(20, 70) * np.exp(rng.randn(20, 70))
    codes, scales, v = ref.quantize(x)
    assert np.array_equal(ref.values(codes, scales, 70), v)
    step = np.exp2(scales.astype(np.float64) - 127).repeat(32, 1)[:, :70]
    t = np.abs(x) / step
    gap = np.where(t < 2, 0.25, np.where(t < 4, 0.5, 1.0))           # half the distance between neighbours
    inside = t <= 6
    assert (np.abs(np.abs(v) / step - t)[inside] <= gap[inside]).all() and (np.abs(v) / step)[~inside].min() == 6
    top = np.abs(np.pad(x, ((0, 0), (0, 26)))).reshape(20, 3, 32).max(-1) / np.exp2(scales.astype(np.float64) - 127)
    assert (top >= 4).all() and (top < 8).all()


def test_reference_on_hand_worked_blocks():
    x = np.zeros((4, 32))
    x[0, :8] = [4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -0.25]           # scale 1: ties go to the even code
    x[1, :3] = [7.9, 5.0, -6.5]                                        # saturation, and the tie between 4 and 6
    x[2, 0] = np.nan
    codes, scales, v = ref.quantize(x)
    assert v[0, :8].tolist() == [4, 0, 1, 1, 2, 2, 4, 0] and np.signbit(v[0, 7])
    assert v[1, :3].tolist() == [6, 4, -6] and scales[1, 0] == 127
    assert scales[2, 0] == 255 and np.isnan(v[2]).all() and (codes[2] == 0).all()
    assert scales[3, 0] == 0 and (v[3] == 0).all()
    assert codes[0, :4].tolist() == [6 | 0 << 4, 2 | 2 << 4, 4 | 4 << 4, 6 | 8 << 4]


def test_handles_check_their_parts():
    codes, scales = torch.zeros(5, 32, dtype=torch.uint8), torch.zeros(5, 2, dtype=torch.uint8)
    m = q.MxMatrix(codes, scales, 40)
    assert (m.rows, m.groups) == (5, 1) and m._c.codes_ld == 32 and m._c.scales_ld == 2
    padded = q.MxMatrix(torch.zeros(3, 5, 64, dtype=torch.uint8)[..., :32], torch.zeros(3, 5, 16, dtype=torch.uint8)[..., :2], 64)
    assert (padded._c.groups, padded._c.codes_ld, padded._c.codes_gs, padded._c.scales_ld, padded._c.scales_gs) == (3, 64, 320, 16, 80)
    for args, err in (((codes, scales, 65), ValueError), ((codes, scales[:4], 40), ValueError), ((codes.int(), scales, 40), TypeError),
                      ((codes[None, None], scales[None, None], 40), ValueError), ((codes.repeat(1, 2)[:, ::2], scales, 40), ValueError)):
        with pytest.raises(err):
            q.MxMatrix(*args)
    k, s = torch.zeros(2, 4, 3, 8, dtype=torch.int8), torch.zeros(2, 4, 3)
    c = q.KvCache(q.KV_I8, 8, k, s, k, s)
    assert (c._c.pages, c._c.page_size, c._c.heads, c._c.head_dim) == (2, 4, 3, 8)
    with pytest.raises(ValueError):
        q.KvCache(q.KV_I8, 8, k, s, k[:1], s)
    with pytest.raises(TypeError):
        q.KvCache(q.KV_MX4, 8, k, s, k, s)
    with pytest.raises(ValueError):
        q.KvCache(q.KV_I8, 8, k.transpose(1, 2), s.transpose(1, 2), k, s)
