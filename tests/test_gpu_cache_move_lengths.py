"""Lengths that no cache has, moved: what is taken of them, and that it is reported."""
import pytest
import torch

import paper_2407_11550_amd as adakv
from serve_util import DEV
from test_gpu_cache_move import source

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("held, headroom_out, moved, over", [
    ([10, 24], 3, [10, 23], 1),                  # beyond the source's capacity of 23, as much room there
    ([10, 24], 9, [10, 23], 1),                  # more room there
    ([10, 1 << 30], 0, [10, 20], 1),
    ([-5, 23], 9, [0, 23], 0),
    ([-(1 << 31), 2 ** 31 - 1], 9, [0, 23], 1),
    ([13, 23], 3, [13, 23], 0),                  # full, and no more
])
def test_a_length_beyond_the_capacity_is_reported(q8, held, headroom_out, moved, over):
    print(q8, held, headroom_out, flush=True)
    layer, cache, cu, seg_len = source(BF, 2, 64, [10, 20], 3, held, q8)
    overflow = torch.zeros(1, dtype=torch.int32, device=DEV)
    if q8:
        _, _, out, lens = adakv.cache_move_q8(layer, [0], cu, 3, cache, seg_len, headroom_out, overflow=overflow)
    else:
        _, _, *out, lens = adakv.cache_move(layer, [0], cu, 3, *cache, seg_len, headroom_out, overflow=overflow)
    torch.cuda.synchronize()
    assert lens.tolist() == moved and int(overflow) == over
    for src, dst in zip(cache[:2], out[:2]):
        for a, b, n in ((0, 0, moved[0]), (13, 10 + headroom_out, moved[1])):
            assert torch.equal(src.view(torch.uint8)[a:a + n], dst.view(torch.uint8)[b:b + n])
