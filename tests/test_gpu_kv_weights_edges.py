"""Summed weights at the ends of binary32's range, on both sides of 64 query rows for a key head, on the GPU against 64 bits."""
import math

import pytest
import torch

from tests import keep_ref as kr
from tests.test_gpu_kv import Cache, cumulative, dev, fill, make_table, mx  # noqa: F401

pytestmark = pytest.mark.gpu
FEW, MANY = (4, 2, 3), (8, 2, 130)   # query heads, key heads, new queries


def setting(qh, h, dim, nq, length, page=32, block=16, seed=0, binades=0):
    """Queries times 2^binades over keys times 2^-binades."""
    table, pool = make_table([length], -(-length // page) + 1, page, seed)
    cache = Cache(pool, h, page, dim, block)
    fill(cache, [length], table, page, block, seed)
    scales = cache.parts[1]
    scales.copy_(torch.where(scales == 255, scales, (scales.int() - binades).to(torch.uint8)))
    q = 2 * torch.randn(nq, qh, dim, generator=torch.Generator().manual_seed(seed + 1)).to(torch.bfloat16).double()
    return table, cache, (q * 2.0 ** binades).to(torch.bfloat16).cuda()


def summed(mx, q, lse, table, cache, length, earlier=None, causal=True):  # noqa: F811
    out = torch.full(cache.parts[1].shape[:2] + cache.parts[0].shape[2:3], 7.0, device="cuda")
    mx.mxkv_attention_weights(q, dev([0, q.shape[0]]), dev([length]), dev(table), cache.parts[0], cache.parts[1], lse, out, q.shape[0], length,
                              q.shape[2] ** -0.5, earlier=earlier, causal=causal)
    torch.cuda.synchronize()
    assert mx.device_timeouts() == 0 and cache.guards_intact()
    return out


def of_tokens(sums, table, length):
    key = torch.arange(length, device="cuda")
    page = sums.shape[2]
    return sums[torch.tensor(table[0], device="cuda")[key // page], :, key % page]   # [length, heads]


@pytest.mark.parametrize("qh,h,nq", [FEW, MANY])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("binades", [118, 60, -60, -118, -124])
@pytest.mark.parametrize("mixed", [False, True])
def test_queries_of_any_size(mx, qh, h, nq, dim, binades, mixed):  # noqa: F811
    """Very large queries over very small keys and the other way round: the scores are ordinary ones.  Mixed: every other query is an ordinary one, whose
    scores are next to nothing (over small keys; over large ones it would have to see one key only)."""
    length, scale = 400, dim ** -0.5
    table, cache, q = setting(qh, h, dim, nq, length, seed=dim + nq, binades=binades)
    if mixed:
        q[::2] = (q[::2].double() * 2.0 ** -max(binades, 0)).to(torch.bfloat16) if binades > 0 else 0.0
    masks = [kr.sinks_mask(nq, length, 0, 0, device="cuda")]
    lse = kr.attention(q, [0, nq], [length], table, *cache.parts[:2], *cache.parts[:2], scale, masks)[1].float()
    sums = summed(mx, q, lse, table, cache, length)
    want = torch.full_like(sums, 7.0).double()
    slack = kr.weights(q, lse, [0, nq], [length], table, *cache.parts[:2], scale, masks, want, None)
    err = (sums.double() - want).abs()
    assert bool((err <= slack).all()), f"off by {float((err / slack.clamp(min=1e-30)).nan_to_num(math.inf).max()):.3g} tolerances"


@pytest.mark.parametrize("qh,h,nq", [FEW, MANY, (6, 1, 90), (3, 1, 200), (7, 1, 8), (1, 1, 300)])
@pytest.mark.parametrize("lse_of_all", [-math.inf, 300.0])
@pytest.mark.parametrize("causal", [True, False])
def test_nothing_is_exactly_nothing(mx, qh, h, nq, lse_of_all, causal):  # noqa: F811
    """Rows that saw nothing, and weights below 2^-400: exactly 0, and exactly the earlier sums, whatever rows a tile of queries has."""
    length = 500
    table, cache, q = setting(qh, h, 64, nq, length, seed=nq)
    q = (q.double() / 16).to(torch.bfloat16)   # scores below some 20
    lse = torch.full((nq, qh), lse_of_all, device="cuda")
    assert bool((of_tokens(summed(mx, q, lse, table, cache, length, causal=causal), table, length) == 0).all())
    shape = cache.parts[1].shape[:2] + (32,)
    before = torch.exp(torch.randn(shape, generator=torch.Generator().manual_seed(1)) - 85).cuda()   # some 2^-123
    got, old = (of_tokens(x, table, length) for x in (summed(mx, q, lse, table, cache, length, earlier=before, causal=causal), before))
    assert torch.equal(got[:length - nq], old[:length - nq]) and bool((got[length - nq:] == 0).all())


@pytest.mark.parametrize("qh,h,nq", [(2, 2, 5), (2, 2, 128)])
def test_nan_that_gives_nothing(mx, qh, h, nq):  # noqa: F811
    """A row whose lse is -infinity gives nothing, a NaN in it or not."""
    length = 300
    table, cache, q = setting(qh, h, 64, nq, length, seed=nq)
    lse = torch.full((nq, qh), -math.inf, device="cuda")
    q[nq // 2] = math.nan
    assert bool((of_tokens(summed(mx, q, lse, table, cache, length, causal=False), table, length) == 0).all())
    q[0] = math.inf
    assert bool((of_tokens(summed(mx, q, lse, table, cache, length, causal=False), table, length) == 0).all())


@pytest.mark.parametrize("qh,h,nq", [(2, 2, 5), (2, 2, 128)])
@pytest.mark.parametrize("where", ["query", "lse"])
def test_nan_in_any_row(mx, qh, h, nq, where):  # noqa: F811
    """A NaN in a query or in its lse alone (the attention gives such a query an lse of NaN) makes the sums of its head's keys NaN and no other,
    whichever row it is."""
    length = 300
    table, cache, q = setting(qh, h, 64, nq, length, seed=nq)
    masks = [kr.sinks_mask(nq, length, 0, 0, causal=False, device="cuda")]
    lse = kr.attention(q, [0, nq], [length], table, *cache.parts[:2], *cache.parts[:2], 0.125, masks)[1].float()
    for row in range(nq):
        x, y = q.clone(), lse.clone()
        if where == "query":
            x[row, 1, 7 * row % 64] = math.nan
        else:
            y[row, 1] = math.nan
        got = of_tokens(summed(mx, x, y, table, cache, length, causal=False), table, length)
        assert bool(got[:, 1].isnan().all()) and not bool(got[:, 0].isnan().any()), row


@pytest.mark.parametrize("qh,h,nq", [FEW, (8, 2, 12), MANY])
@pytest.mark.parametrize("binades", [-116, -100, 0, 100])
def test_small_scales_of_the_scores(mx, qh, h, nq, binades):  # noqa: F811
    """The scores' scale far below 1 / sqrt(dim), over keys that are larger by as much: a factor of small queries and the scale has to keep its bits."""
    length, dim, scale = 400, 64, 2.0 ** -10
    table, cache, q = setting(qh, h, dim, nq, length, seed=nq, binades=binades)
    scales = cache.parts[1]
    scales.copy_(torch.where(scales == 255, scales, scales + 7))
    masks = [kr.sinks_mask(nq, length, 0, 0, device="cuda")]
    lse = kr.attention(q, [0, nq], [length], table, *cache.parts[:2], *cache.parts[:2], scale, masks)[1].float()
    sums = torch.full(cache.parts[1].shape[:2] + (32,), 7.0, device="cuda")
    mx.mxkv_attention_weights(q, dev([0, nq]), dev([length]), dev(table), cache.parts[0], cache.parts[1], lse, sums, nq, length, scale)
    want = torch.full_like(sums, 7.0).double()
    slack = kr.weights(q, lse, [0, nq], [length], table, *cache.parts[:2], scale, masks, want, None)
    err = (sums.double() - want).abs()
    assert bool((err <= slack).all()), f"off by {float((err / slack.clamp(min=1e-30)).nan_to_num(math.inf).max()):.3g} tolerances"


@pytest.mark.parametrize("qh,h,nq", [(2, 2, 5), (2, 2, 128), (6, 2, 100)])
def test_nan_in_a_key(mx, qh, h, nq):  # noqa: F811
    """A NaN code makes its own key's sum NaN and no other, with an lse that knows nothing of it."""
    length = 300
    table, cache, q = setting(qh, h, 64, nq, length, seed=nq)
    masks = [kr.sinks_mask(nq, length, 0, 0, causal=False, device="cuda")]
    lse = kr.attention(q, [0, nq], [length], table, *cache.parts[:2], *cache.parts[:2], 0.125, masks)[1].float()
    bad = [0, 31, 128, 255, 299]
    for t in bad:
        cache.parts[0][table[0][t // 32], 1, t % 32, t % 64] = 0x7F
    got = of_tokens(summed(mx, q, lse, table, cache, length, causal=False), table, length)
    assert got[:, 1].isnan().nonzero().flatten().tolist() == bad and not bool(got[:, 0].isnan().any())
