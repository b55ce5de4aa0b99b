"""Trees of many rows with workspaces of every size that they take, on the GPU against 64 bits."""
import random

import pytest
import torch

from tests import keep_ref as kr
from tests.test_gpu_kv import dev, mx  # noqa: F401
from tests.test_gpu_kv_masks import compare, job, random_tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("qh,h,dim,nq,lens", [
    (8, 1, 64, [9, 0, 13, 10], [4000, 70, 13, 900]), (4, 1, 128, [64, 17], [3000, 100]), (4, 2, 128, [40] * 6, [5000, 40, 300, 2048, 41, 1500]),
    (8, 2, 64, [33], [9000]), (2, 2, 128, [300], [2500]),
])
@pytest.mark.parametrize("size", ["full", "between", "least", "one chunk"])
def test_tree_in_workspaces_of_any_size(mx, qh, h, dim, nq, lens, size):  # noqa: F811
    """The full one, one with room for half of the chunks and a few bytes over, the other masks' and one that is barely larger than it.  Nothing behind it
    is written."""
    pick = random.Random(dim + len(nq))
    rows = [random_tree(n, pick) for n in nq]
    cu, table, cache, q, buf, out, lse, max_q, max_len, _ = job(mx, qh, h, dim, 32, 16, nq, lens, 4)
    sizes = (q.shape[0], len(nq), max_q, max_len, qh, h, dim)
    full, least = mx.mxkv_attention_tree_workspace_bytes(*sizes), mx.mxkv_attention_workspace_bytes(*sizes)
    chunk = q.shape[0] * qh * (dim + 1) * 4
    assert full % chunk == 0 and full >= 4 * chunk
    nbytes = {"full": full, "between": max(least, full // chunk // 2 * chunk + 12), "least": least, "one chunk": least + 8}[size]
    room = torch.full((nbytes + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    ws = room[:nbytes] if nbytes else None
    scale = dim ** -0.5
    mask = kr.words([r for sequence in rows for r in sequence] + [0] * 3, -(-max(nq) // 32)).cuda()
    masks = [kr.tree_mask(sequence, length, device="cuda") for sequence, length in zip(rows, lens)]
    compare(mx, lambda: mx.mxkv_attention_tree(q, dev(cu), dev(lens), dev(table), *cache.parts, out, max_q, max_len, scale, mask, lse=lse, workspace=ws),
            q, cu, lens, table, cache, scale, masks, out, lse, buf)
    assert bool((room[nbytes:] == 0xFF).all())
