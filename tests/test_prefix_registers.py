"""What the compiler made of the kernels over shared caches, from the build's own metadata: registers, scratch and LDS."""
import os
import re

import pytest

import paper_2407_11550_amd.binding as B
from test_register_budget import TOOLS, _kernel_metadata


@pytest.fixture(scope="module")
def kernels(lib):
    if not all(os.path.exists(t) for t in TOOLS):
        pytest.skip("ROCm LLVM tools not installed")
    out = {}
    for name, md in _kernel_metadata(B._LIB_PATH).items():
        m = re.search(r"prefix_attn_kernelI.*?(BF16|FP16|FP32)ELi(\d+)ELi(\d+)EE", name or "")
        if m:
            out[m.group(1), int(m.group(2)), int(m.group(3))] = md
    return out


def test_which_there_are(kernels):
    """By type, d, and wavefronts that share 32 query rows (32 bits, 8: those of 16 rows)."""
    sixteen = {(t, d, ks) for t in ("BF16", "FP16") for d in (64, 128) for ks in (1, 2)} | {(t, 64, 4) for t in ("BF16", "FP16")}
    assert set(kernels) == sixteen | {("FP32", d, ks) for d in (64, 128) for ks in (1, 2, 8)}


def test_two_workgroups_fit_on_a_compute_unit(kernels):
    """Own segments run beside shared ones, but for two fp32 tiles of 64 rows of 128 columns, which fill LDS."""
    for key, md in kernels.items():
        if key in (("FP32", 128, 2), ("FP32", 128, 8)):
            assert md["lds"] <= 160 * 1024, (key, md)
            continue
        assert md["vgpr"] + md["agpr"] <= 256 and md["lds"] <= 80 * 1024, (key, md)


def test_no_spills(kernels):
    for key, md in kernels.items():
        assert md["scratch"] == 0, (key, md)
