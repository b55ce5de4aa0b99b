"""Attention with a scale of the scores far below 1 / sqrt(dim), over keys that are larger by as much, against 64 bits."""
import pytest
import torch

from tests import keep_ref as kr
from tests.test_gpu_kv import dev, mx  # noqa: F401
from tests.test_gpu_kv_masks import compare, job

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("qh,h,dim,nq", [(4, 2, 64, 3), (8, 2, 128, 12), (8, 2, 64, 130)])
@pytest.mark.parametrize("binades", [-116, -100, 0, 100])
def test_small_scales(mx, qh, h, dim, nq, binades):  # noqa: F811
    """The factor that takes small queries back, times the scale, has to keep its bits."""
    scale = 2.0 ** -10
    cu, table, cache, q, buf, out, lse, max_q, max_len, ws = job(mx, qh, h, dim, 32, 16, [nq], [400], 5)
    q.copy_((q.double() * 2.0 ** binades).to(torch.bfloat16))
    scales = cache.parts[1]
    scales.copy_(torch.where(scales == 255, scales, (scales.int() + 7 - binades).to(torch.uint8)))
    args = (q, dev(cu), dev([400]), dev(table), *cache.parts, out, max_q, max_len, scale)
    compare(mx, lambda: mx.mxkv_attention(*args, lse=lse, workspace=ws), q, cu, [400], table, cache, scale, [kr.sinks_mask(nq, 400, 0, 0, device="cuda")], out, lse,
            buf)
