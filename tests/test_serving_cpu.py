"""CPU: struct layouts of the calls around the cache, and the reference that they are tested against on worked examples."""
import ctypes as C
import math
import os
import re

import numpy as np
import pytest

import serving_reference as ref
from paper_2501_07161_b200 import binding as B


def test_struct_layouts():
    assert C.sizeof(B.PagePlanC) == 136 and B.PagePlanC.free_pages.offset == 40 and B.PagePlanC.lens_out.offset == 64 and B.PagePlanC.seqs.offset == 128
    assert C.sizeof(B.HeadRowsC) == 64 and B.HeadRowsC.weight.offset == 48 and B.HeadRowsC.heads.offset == 56
    assert C.sizeof(B.AttendCfgC) == 32 and B.AttendCfgC.window.offset == 8 and B.AttendCfgC.max_new.offset == 24


def test_null_arguments_are_errors():
    L = B.lib()
    assert L.qv2_kv_plan(None, None) == -2 and L.qv2_norm_rotate(None, None, None, 0, 64, 64, 0, 1e-6, 0, None, None) == -2
    assert L.qv2_kv_attend(None, None, None, 0, 0, 1, 0, 0, None, None, 0, None, 0, None, None, None) == -2


def test_reference_plan_by_hand():
    table = np.full((3, 3), -1)
    table[0, 0], table[2, :2] = 40, [41, 42]
    got = ref.plan([3, 0, 8], [3, 0, 1], 4, table, [7, 8, 9], 3, 5)
    assert got[0].tolist() == [[40, 9, -1], [-1, -1, -1], [41, 42, 8]]
    assert got[1:] == ([6, 0, 9], [0, 3, 3, 4], [0, 6, 6, 15], [40 * 4 + 3, 36, 37, 32, -1], [3, 4, 5, 8, 0], 1, 0)


def test_reference_rotation_by_hand():
    x = np.array([[[3.0, 0.0, 4.0, 0.0]]])
    y = ref.norm_rotate(x, np.ones(4), np.array([1]), np.array([math.pi / 2, 0.0]), 0.0, False)
    assert np.allclose(y, [[[-1.6, 0.0, 1.2, 0.0]]])
    y = ref.norm_rotate(x, None, np.array([2]), np.array([math.pi / 2, math.pi / 4]), 0.0, True)
    assert np.allclose(y, [[[-3.0, 0.0, 0.0, 4.0]]])


def test_reference_attention_by_hand():
    k = np.zeros((2, 2, 1, 2))
    v = np.arange(8.0).reshape(2, 2, 1, 2)
    out, lse, _, _ = ref.attend(np.ones((2, 1, 2)), k, v, [3], [0, 2], np.array([[1, 0]]), 2, 1.0)
    assert np.allclose(out[:, 0], [[5, 6], [10 / 3, 13 / 3]]) and np.allclose(lse[:, 0], np.log([2, 3]))
    out, lse, _, _ = ref.attend(np.ones((2, 1, 2)), k, v, [3], [0, 2], np.array([[1, -1]]), 2, 1.0, window=1)
    assert np.allclose(out[0, 0], [6, 7]) and (out[1, 0] == 0).all() and lse[1, 0] == -np.inf


CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2501_07161_b200", "csrc")


@pytest.mark.parametrize("name", ["qv2_pages.cu", "qv2_rotate.cu", "qv2_attend.cuh", "qv2_attend.cu", "qv2_attend_chunk.cu"])
def test_global_loads_stay_behind_the_wait_for_the_kernel_before(name):
    """As for the other operators: inline loads and copies are volatile, every kernel waits for the one before it, and multicast
    loads are not used."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    loads = re.findall(r"\basm\b(\s*volatile)?\s*\(\s*\"[^\"]*\b(?:ld\.(?:global|shared)|cp\.async)", text)
    assert all(loads) and "ld_stream" not in text and "multicast::cluster" not in text
    assert text.count("__global__") == len(re.findall(r"dependency_wait\(\);", text))
