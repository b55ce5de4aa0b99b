"""Eviction and an accepted tree, captured once and replayed over poisoned outputs: every output of the replay has the eager run's bits."""
import pytest
import torch

from tests import keep_ref as kr
from tests.test_gpu_kv import dev, make_table, mx  # noqa: F401

pytestmark = pytest.mark.gpu


def replayed(step, start, written):
    """step() leaves its results in `written`; start() brings those that it also reads back to what they were.  Returns the eager run's."""
    start()
    step()
    torch.cuda.synchronize()
    want = {name: t.clone() for name, t in written.items()}
    graph = torch.cuda.CUDAGraph()
    start()
    with torch.cuda.graph(graph):
        step()
    for _ in range(2):
        for t in written.values():
            t.view(torch.uint8).fill_(0x5A)
        start()
        graph.replay()
        torch.cuda.synchronize()
        for name, t in written.items():
            assert torch.equal(t.view(torch.uint8), want[name].view(torch.uint8)), name
    return want


@pytest.mark.parametrize("new", [400, 7])
@pytest.mark.parametrize("to_other_pages", [False, True])
def test_eviction(mx, new, to_other_pages):  # noqa: F811
    """Append, attention, summed weights, choice, move: codes, scales, sums, lists and lengths."""
    heads, qh, dim, page, block, length, keep = 2, 8, 128, 64, 16, 400, 130
    table, pool = make_table([length], 8, page, 1)
    cache = mx.alloc_kv_cache(pool + 3, heads, page, dim, block)
    g = torch.Generator().manual_seed(4)
    x = torch.randn(length, qh + 2 * heads, dim, generator=g).to(torch.bfloat16).cuda()
    empty = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    sums, out, lse = empty(pool + 3, heads, page), empty(new, qh, dim, dtype=torch.bfloat16), empty(new, qh)
    kept, new_lens = empty(1, heads, keep, dtype=torch.int32), empty(1, dtype=torch.int32)
    ws = empty(max(16, mx.mxkv_attention_workspace_bytes(new, 1, new, length, qh, heads, dim)), dtype=torch.uint8)
    cws = empty(mx.mxkv_compact_workspace_bytes(1, heads, keep), dtype=torch.uint8)
    lens, pages = dev([length]), dev(table)
    out_pages = dev([[pool, pool + 1, pool + 2]]) if to_other_pages else None
    old = torch.rand(sums.shape, generator=g).cuda()

    def start():
        for c in cache:
            c.zero_()
        sums.copy_(old)
        if new < length:
            mx.mxkv_append(x[:-new, qh:qh + heads], x[:-new, qh + heads:], dev([0, length - new]), dev([length - new]), pages, *cache)

    cu = dev([0, new])

    def step():
        q = x[length - new:]
        mx.mxkv_append(q[:, qh:qh + heads], q[:, qh + heads:], cu, lens, pages, *cache)
        mx.mxkv_attention(q[:, :qh], cu, lens, pages, *cache, out, new, length, dim ** -0.5, lse=lse, workspace=ws)
        mx.mxkv_attention_weights(q[:, :qh], cu, lens, pages, cache[0], cache[1], lse, sums, new, length, dim ** -0.5, earlier=sums)
        mx.mxkv_select(sums, lens, pages, kept, new_lens, length, sinks=4, recent=32)
        mx.mxkv_compact(kept, new_lens, lens, pages, *cache, out_page_table=out_pages, weights=sums, workspace=None if to_other_pages else cws)

    names = ("k codes", "k scales", "v codes", "v scales")
    want = replayed(step, start, dict(zip(names, cache), sums=sums, kept=kept, new_lens=new_lens, out=out, lse=lse))
    assert want["new_lens"].tolist() == [keep] and bool(want["k scales"][out_pages[0] if to_other_pages else pages[0, :2]].any())
    assert mx.device_timeouts() == 0 and mx.device_bad_indices() == 0


def test_accepted_tree(mx):  # noqa: F811
    """Drafts appended, attended as a tree, a path of them moved together."""
    heads, qh, dim, page, block, front, n = 2, 8, 64, 32, 16, 1000, 20
    table, pool = make_table([front + n], 33, page, 1)
    cache = mx.alloc_kv_cache(pool, heads, page, dim, block)
    g = torch.Generator().manual_seed(4)
    x = torch.randn(front + n, qh + 2 * heads, dim, generator=g).to(torch.bfloat16).cuda()
    path = [0, 2, 5, 9, 19]
    mask = kr.words([1 << i | sum(1 << p for p in path if p < i) for i in range(n)], 1).cuda()
    out, lse = torch.empty(n, qh, dim, dtype=torch.bfloat16, device="cuda"), torch.empty(n, qh, device="cuda")
    ws = torch.empty(max(16, mx.mxkv_attention_tree_workspace_bytes(n, 1, n, front + n, qh, heads, dim)), dtype=torch.uint8, device="cuda")
    cws = torch.empty(mx.mxkv_compact_workspace_bytes(1, heads, len(path)), dtype=torch.uint8, device="cuda")
    cu, lens, pages, first = dev([0, n]), dev([front + n]), dev(table), dev([front])
    kept, new_lens = dev([[[front + p for p in path]]]), dev([front + len(path)])
    before = (dev([0, front]), dev([front]))

    def start():
        for c in cache:
            c.zero_()
        mx.mxkv_append(x[:front, qh:qh + heads], x[:front, qh + heads:], *before, pages, *cache)

    def step():
        mx.mxkv_append(x[front:, qh:qh + heads], x[front:, qh + heads:], cu, lens, pages, *cache)
        mx.mxkv_attention_tree(x[front:, :qh], cu, lens, pages, *cache, out, n, front + n, dim ** -0.5, mask, lse=lse, workspace=ws)
        mx.mxkv_compact(kept, new_lens, lens, pages, *cache, first=first, workspace=cws)

    replayed(step, start, dict(zip(("k codes", "k scales", "v codes", "v scales"), cache), out=out, lse=lse))
    assert mx.device_timeouts() == 0 and mx.device_bad_indices() == 0
