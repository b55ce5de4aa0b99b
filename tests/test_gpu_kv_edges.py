"""mxkv_attention and mxkv_append where scales, windows, bounds and places go to their ends.

Tolerances are those of test_gpu_kv.py, whose helpers are used, unless a test says otherwise."""
import pytest
import torch

from tests.test_gpu_kv import check, mx  # noqa: F401  (mx is the fixture)

pytestmark = pytest.mark.gpu


def value_scales(low, high, seed=9):
    """Value scales of 2^low and 2^high by chance, a draw for each block.  Codes below 1 in magnitude become 1, so that no
    sum hangs on the tokens that are 2^(high - low) smaller."""
    def setup(cache, q, table):
        vc, vs = cache.parts[2:]
        g = torch.Generator(device="cuda").manual_seed(seed)
        for row in table:
            for pg in row:
                if 0 <= pg < vc.shape[0]:
                    pick = torch.randint(0, 2, vs[pg].shape, generator=g, device="cuda")
                    vs[pg] = (127 + torch.where(pick == 1, high, low)).to(torch.uint8)
                    held = vc[pg] != 0x7F
                    vc[pg] = torch.where(held & ((vc[pg] & 0x7F) < 0x38), (vc[pg] & 0x80) | 0x38, vc[pg])
    return setup


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("qh,h,nq,lens,window", [
    (1, 1, [100], [100], 10), (2, 1, [150, 90], [400, 60], 33), (1, 1, [300], [300], 1), (8, 2, [40, 64], [600, 64], 20), (4, 1, [2], [300], 10),
])
def test_value_scales_far_apart_with_rows_that_have_seen_nothing(mx, dim, qh, h, nq, lens, window):  # noqa: F811
    """Value scales fifty binades apart while some rows of a warp see a tile's keys and others none yet."""
    check(mx, qh, h, dim, 16, 16, nq, lens, window=window, seed=dim + qh, setup=value_scales(-56, -6))
