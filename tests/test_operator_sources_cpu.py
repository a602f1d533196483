"""CPU: rules that the sources of the 4-bit operators and the cache keep and that no run can show."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2501_07161_b200", "csrc")


@pytest.mark.parametrize("name", ["qv2_mx.cuh", "qv2_mx_quant.cu", "qv2_mx_matmul.cu", "qv2_kv.cu"])
def test_global_loads_stay_behind_the_wait_for_the_kernel_before(name):
    """A kernel may start while the one before it still writes; what it loads must not be moved ahead of
    dependency_wait().  Inline loads are volatile (as __ldg is), and the sweep's ld_stream* helpers, which are not, are
    not used."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    loads = re.findall(r"\basm\b(\s*volatile)?\s*\(\s*\"[^\"]*\bld\.(?:global|shared)", text)
    assert all(loads), f"{name}: an inline load without volatile"
    assert "ld_stream" not in text
    if name == "qv2_mx.cuh":
        assert len(loads) >= 2
