"""The sizes up to which the calls around a served cache go, on the host: an argument that is missing is found only after
the sizes, so that neither side of a limit launches anything."""
import ctypes

import pytest
import torch

import paper_2407_11550_amd as adakv

ONE = ctypes.c_void_p(1 << 20)      # never dereferenced


@pytest.mark.parametrize("h_q, rows, status", [
    (32, [1 << 26], -2),                         # 2^31 rows times heads
    (32, [(1 << 26) - 128], -1),
    (32, [(1 << 26) - 127], -2),                 # (rows are counted in 128s)
    (1, [1 << 28] * 8, -2),
    (1, [1 << 28] * 7 + [(1 << 28) - 128], -1),
    (1, [(1 << 28) + 1], -2),                    # a single sequence
    (64, [1 << 19] * 63 + [(1 << 19) - 128], -1),
    (64, [1 << 19] * 64, -2),
])
def test_prompts_fit_into_one_launch(lib, h_q, rows, status):
    w = 2
    layer = adakv.Layer(torch.bfloat16, h_q, 1, 64, w, 7, 0.2, [n - w for n in rows], [w for _ in rows])
    got = lib.adakv_window_attn(ctypes.byref(layer.c), None, 64 * h_q, 64, ONE, ONE, 16, 0, ONE, None, None)
    assert got == status


@pytest.mark.parametrize("rows, status", [(10 ** 9, -1), (10 ** 9 + 1, -2)])
def test_an_8_bit_cache_is_built_by_one_launch(lib, rows, status):
    layer = adakv.Layer(torch.bfloat16, 8, 8, 64, 1, 7, 0.2, [130_000_000], [rows])
    assert lib.adakv_cache_build_q8(ctypes.byref(layer.c), None, ONE, ONE, ONE, 0, ONE, ONE, ONE, ONE, ONE, None) == status
