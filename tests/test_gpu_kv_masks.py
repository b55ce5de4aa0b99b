"""mxkv_attention_sinks and mxkv_attention_tree on the GPU against 64 bits, with the tolerances of mxkv_attention (tests/test_gpu_kv.py): the
products and sums are the same, only which keys a row sees differs."""
import math
import random

import pytest
import torch

from tests import keep_ref as kr
from tests.test_gpu_kv import NAN_CODE, Cache, cumulative, dev, fill, make_table, mx  # noqa: F401

pytestmark = pytest.mark.gpu


def compare(mx, call, q, cu, lens, table, cache, scale, masks, out, lse, buf):
    call()
    torch.cuda.synchronize()
    assert mx.device_timeouts() == 0
    n = cu[-1]
    want, want_lse, mag, big = kr.attention(q[:n], cu, lens, table, *cache.parts, scale, masks)
    got = out[:n].double()
    err, tol = (got - want).abs(), 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -10) * mag + 1e-30
    assert bool((err <= tol).all()), f"out: off by {float((err / tol).nan_to_num(1e9).max()):.3g} tolerances"
    live = want_lse > -math.inf
    assert bool((lse[:n][~live] == -math.inf).all()) and not bool(got[~live].any())
    e = (lse[:n].double() - want_lse)[live].abs()
    t = (16 * 2.0 ** -23 * big + 2.0 ** -19 + 5 * 2.0 ** -23 * want_lse.abs())[live]
    assert bool((e <= t).all()), f"lse: off by {float((e / t).max()):.3g} tolerances"
    assert bool((lse[n:] == 7).all()) and bool((buf[n:] == 7).all()) and bool((buf[:, -1] == 7).all()), "rows that are not the call's were written"
    assert cache.guards_intact()
    first = out.clone()
    call()
    assert torch.equal(first, out), "not repeatable"


def job(mx, qh, h, dim, page, block, nq, lens, seed, max_q=None, max_len=None):
    cu, n = cumulative(nq), sum(nq)
    max_len = max(max(lens), 1) if max_len is None else max_len
    table, pool = make_table(lens, -(-max_len // page) + 1, page, seed, junk=-7 if seed % 2 else 2 ** 30)
    cache = Cache(pool, h, page, dim, block)
    fill(cache, lens, table, page, block, seed)
    x = (2 * torch.randn(n + 3, (qh + 2) * dim, generator=torch.Generator().manual_seed(seed + 1))).to(torch.bfloat16).cuda()
    q = x[:, dim:(qh + 1) * dim].view(-1, qh, dim)
    buf = torch.full((n + 3, qh + 1, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n + 3, qh), 7.0, device="cuda")
    max_q = max(max(nq), 1) if max_q is None else max_q
    nbytes = mx.mxkv_attention_workspace_bytes(n + 3, len(lens), max_q, max_len, qh, h, dim)
    ws = torch.full((nbytes,), 0xFF, dtype=torch.uint8, device="cuda") if nbytes else None
    return cu, table, cache, q, buf, buf[:, :qh], lse, max_q, max_len, ws


def check_sinks(mx, qh, h, dim, page, block, nq, lens, window, sinks, seed=0, **kw):
    cu, table, cache, q, buf, out, lse, max_q, max_len, ws = job(mx, qh, h, dim, page, block, nq, lens, seed, **kw)
    scale = dim ** -0.5
    masks = [kr.sinks_mask(b - a, length, window, sinks, device="cuda") for a, b, length in zip(cu, cu[1:], lens)]
    compare(mx, lambda: mx.mxkv_attention_sinks(q, dev(cu), dev(lens), dev(table), *cache.parts, out, max_q, max_len, scale, window, sinks, lse=lse,
                                                workspace=ws), q, cu, lens, table, cache, scale, masks, out, lse, buf)
    return cache, table


SINKS = [  # query heads, key heads, dim, page, block, new queries, lengths
    (1, 1, 64, 16, 16, [1], [1]), (32, 8, 128, 64, 16, [1] * 5, [1, 63, 64, 65, 1300]), (8, 1, 64, 128, 64, [1, 1], [127, 2049]),
    (14, 2, 64, 16, 16, [1, 1, 0], [15, 700, 50]), (6, 2, 64, 32, 16, [2, 3, 4, 1], [2, 70, 1000, 5]), (8, 2, 128, 16, 16, [8, 5, 7], [8, 9, 429]),
    (16, 2, 64, 128, 32, [3, 6], [1, 2000]), (1, 1, 128, 64, 16, [1], [20000]), (32, 4, 64, 16, 16, [4, 4], [900, 4100]),
    (4, 1, 128, 64, 16, [100], [700]), (8, 2, 64, 32, 32, [129, 17, 64], [729, 400, 64]), (5, 1, 64, 16, 16, [200, 40], [150, 1040]),
    (2, 2, 64, 64, 16, [1000], [1500]), (8, 1, 128, 128, 64, [128, 256], [128, 2031]),
]


@pytest.mark.parametrize("qh,h,dim,page,block,nq,lens", SINKS)
@pytest.mark.parametrize("window,sinks", [(1, 1), (50, 4), (300, 33), (128, 128), (40, 500), (5000, 4), (200, 0)])
def test_sinks(mx, qh, h, dim, page, block, nq, lens, window, sinks):  # noqa: F811
    check_sinks(mx, qh, h, dim, page, block, nq, lens, window, sinks, seed=dim + page + window)


@pytest.mark.parametrize("nq", [1, 3, 150])
@pytest.mark.parametrize("page,sinks", [(16, 4), (64, 4), (64, 70), (128, 1)])
def test_sinks_pages_between_may_be_released(mx, nq, page, sinks):  # noqa: F811
    """Pages that hold neither first tokens nor the window's: out of range in the table; what stands beside the seen tokens in their pages is NaN."""
    window, length = 100, 1500

    lens = [length]
    mx.device_bad_indices_reset()
    cu, table, cache, q, buf, out, lse, max_q, max_len, ws = job(mx, 8, 2, 128, page, 16, [nq], lens, 4)
    masks = [kr.sinks_mask(nq, length, window, sinks, device="cuda")]
    want, want_lse, mag, _ = kr.attention(q[:nq], cu, lens, table, *cache.parts, 128 ** -0.5, masks)
    left = [list(table[0])]
    low = length - nq - window + 1   # the first key in the first query's window
    for p in range(-(-length // page)):
        if p * page >= sinks and (p + 1) * page <= low:
            left[0][p] = -5 if p % 2 else 2 ** 30
        for o in range(page):
            if sinks <= p * page + o < low:
                cache.parts[0][table[0][p], :, o] = NAN_CODE
                cache.parts[2][table[0][p], :, o] = NAN_CODE
    mx.mxkv_attention_sinks(q, dev(cu), dev(lens), dev(left), *cache.parts, out, max_q, max_len, 128 ** -0.5, window, sinks, lse=lse, workspace=ws)
    assert bool(((out[:nq].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -10) * mag).all())
    assert bool(((lse[:nq].double() - want_lse).abs() < 1e-4).all())
    assert mx.device_bad_indices() == 0


@pytest.mark.parametrize("nq", [1, 100])
def test_sinks_equal_the_window_or_all(mx, nq):  # noqa: F811
    """Without first tokens the call has the bits of mxkv_attention with the window; with a window over everything those without one."""
    cu, table, cache, q, buf, out, lse, max_q, max_len, ws = job(mx, 8, 2, 64, 32, 16, [nq], [900], 6)
    args = (q, dev(cu), dev([900]), dev(table), *cache.parts)
    other = torch.empty_like(out)
    mx.mxkv_attention_sinks(*args, out, max_q, max_len, 0.125, 77, 0, lse=lse, workspace=ws)
    mx.mxkv_attention(*args, other, max_q, max_len, 0.125, window=77, workspace=ws)
    assert torch.equal(out[:nq], other[:nq])
    mx.mxkv_attention_sinks(*args, out, max_q, max_len, 0.125, 2 ** 31 - 1, 2 ** 31 - 1, lse=lse, workspace=ws)
    mx.mxkv_attention(*args, other, max_q, max_len, 0.125, workspace=ws)
    assert torch.equal(out[:nq], other[:nq])


@pytest.mark.parametrize("nq,max_len", [(1, 300), (1, 64), (100, 300), (100, 700)])
def test_sinks_lengths_above_the_bound(mx, nq, max_len):  # noqa: F811
    """Keys past max_kv_len are not seen; the first tokens and the places stay."""
    length, window, sinks = 1000, 400, 40
    cu, table, cache, q, buf, out, lse, max_q, _, ws = job(mx, 4, 2, 64, 32, 16, [nq], [length], 8, max_len=1000)
    scale = 0.125
    masks = [kr.sinks_mask(nq, length, window, sinks, device="cuda") & (torch.arange(length, device="cuda") < max_len)]
    compare(mx, lambda: mx.mxkv_attention_sinks(q, dev(cu), dev([length]), dev(table), *cache.parts, out, max_q, max_len, scale, window, sinks, lse=lse,
                                                workspace=ws), q, cu, [length], table, cache, scale, masks, out, lse, buf)


# ---- trees -----------------------------------------------------------------------------------------------------------

def random_tree(n, pick, back=5):
    seen = []
    for i in range(n):
        up = i - pick.randint(1, back)
        seen.append((seen[up] if up >= 0 else 0) | 1 << i)
    return seen


def check_tree(mx, qh, h, dim, page, block, nq, lens, rows, seed=0, count=None, **kw):
    cu, table, cache, q, buf, out, lse, max_q, max_len, ws = job(mx, qh, h, dim, page, block, nq, lens, seed, **kw)
    scale = dim ** -0.5
    count = -(-max(nq) // 32) if count is None else count
    flat = [r for sequence in rows for r in sequence] + [-1] * 3
    mask = kr.words(flat, count).cuda()
    cut = (1 << 32 * count) - 1
    masks = [kr.tree_mask([r & cut for r in sequence], length, device="cuda") for sequence, length in zip(rows, lens)]
    compare(mx, lambda: mx.mxkv_attention_tree(q, dev(cu), dev(lens), dev(table), *cache.parts, out, max_q, max_len, scale, mask, lse=lse, workspace=ws),
            q, cu, lens, table, cache, scale, masks, out, lse, buf)


TREES = [  # query heads, key heads, dim, page, block, drafts, lengths with them
    (4, 1, 128, 64, 16, [12], [12]), (32, 8, 128, 64, 16, [12, 16, 1], [700, 16, 65]), (32, 4, 64, 16, 16, [8, 5, 0, 7], [500, 37, 9, 131]),
    (8, 8, 64, 32, 32, [33, 64], [129, 2000]), (2, 1, 128, 16, 16, [31, 32], [5000, 47]), (8, 2, 128, 64, 16, [40, 64, 17], [700, 64, 1031]),
    (6, 1, 64, 128, 64, [100, 128, 33], [300, 129, 700]), (1, 1, 64, 64, 64, [200], [333]), (4, 2, 128, 16, 16, [300, 9], [300, 1009]),
]


@pytest.mark.parametrize("qh,h,dim,page,block,nq,lens", TREES)
@pytest.mark.parametrize("form", ["tree", "chain", "any", "empty"])
def test_tree(mx, qh, h, dim, page, block, nq, lens, form):  # noqa: F811
    """Trees; chains (the causal mask); any bits, those of tokens that do not exist among them; rows that see no draft at all, not even themselves."""
    pick = random.Random(dim + page)
    make = {"tree": lambda n: random_tree(n, pick), "chain": lambda n: [(2 << i) - 1 for i in range(n)],
            "any": lambda n: [pick.getrandbits(32 * -(-max(nq) // 32)) for _ in range(n)], "empty": lambda n: [0] * n}[form]
    check_tree(mx, qh, h, dim, page, block, nq, lens, [make(n) for n in nq], seed=dim + page + 3)


@pytest.mark.parametrize("nq,count", [([40, 70], 1), ([40, 70], 9), ([5, 9], 4)])
def test_tree_fewer_and_more_words(mx, nq, count):  # noqa: F811
    pick = random.Random(count)
    check_tree(mx, 2, 1, 64, 32, 16, nq, [100, 500], [[pick.getrandbits(32 * count) for _ in range(n)] for n in nq], seed=count, count=count)


@pytest.mark.parametrize("qh", [4, 40])
def test_tree_more_drafts_than_the_cache_has(mx, qh):  # noqa: F811
    """Drafts whose places lie in front of the first key: the mask's bits still go by their number among the sequence's."""
    check_tree(mx, qh, 1, 64, 16, 16, [12], [7], [random_tree(12, random.Random(3))], seed=2)


def test_a_chain_has_the_causal_masks_bits(mx):  # noqa: F811
    # (few rows; many rows in calls whose keys neither of the two entry points shares out)
    for qh, h, nq, length in ((4, 1, 6, 900), (320, 40, 40, 800)):
        cu, table, cache, q, buf, out, lse, max_q, max_len, ws = job(mx, qh, h, 128, 64, 16, [nq], [length], 1)
        args = (q, dev(cu), dev([length]), dev(table), *cache.parts)
        other = torch.empty_like(out)
        mask = kr.words([(2 << i) - 1 for i in range(nq)] + [0] * 3, 2).cuda()
        mx.mxkv_attention_tree(*args, out, max_q, max_len, 0.1, mask, lse=lse, workspace=ws)
        mx.mxkv_attention(*args, other, max_q, max_len, 0.1, workspace=ws)
        assert torch.equal(out[:nq], other[:nq])


@pytest.mark.parametrize("qh,h,dim,nq,lens", [
    (16, 1, 64, [9] * 40, [1 + 37 * i for i in range(40)]), (8, 2, 128, [0, 40, 3, 0, 64], [5, 3000, 700, 9000, 64]),
    (20, 4, 64, [20, 70], [20, 5000]), (32, 2, 128, [5] * 70, [500] * 70), (5, 1, 128, [50, 20], [0, 4000]),
])
@pytest.mark.parametrize("max_q,max_len", [(None, None), (33, 900)])
def test_trees_shared_out_by_length(mx, qh, h, dim, nq, lens, max_q, max_len):  # noqa: F811
    """Many sequences of very different lengths, sequences without drafts, drafts without keys, bounds below the lists: rows past max_q_len are
    undefined, all others as ever."""
    pick = random.Random(len(nq))
    rows = [random_tree(n, pick) for n in nq]
    cu, table, cache, q, buf, out, lse, _, _, ws = job(mx, qh, h, dim, 32, 16, nq, lens, 3)
    scale, count = dim ** -0.5, -(-max(nq) // 32)
    max_q = max(nq) if max_q is None else max_q
    max_len = max(lens) if max_len is None else min(max_len, max(lens))
    mask = kr.words([r for sequence in rows for r in sequence] + [0] * 3, count).cuda()
    masks = [kr.tree_mask(sequence, length, device="cuda") & (torch.arange(length, device="cuda") < max_len) for sequence, length in zip(rows, lens)]
    need = mx.mxkv_attention_workspace_bytes(q.shape[0], len(lens), max_q, max_len, qh, h, dim)
    ws = torch.full((max(16, need),), 0xFF, dtype=torch.uint8, device="cuda")
    mx.mxkv_attention_tree(q, dev(cu), dev(lens), dev(table), *cache.parts, out, max_q, max_len, scale, mask, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    want, want_lse, mag, big = kr.attention(q[:cu[-1]], cu, lens, table, *cache.parts, scale, masks)
    done = torch.cat([torch.arange(n) < max_q for n in nq]).cuda()
    got, want, mag = out[:cu[-1]][done].double(), want[done], mag[done]
    assert bool(((got - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -10) * mag + 1e-30).all())
    e, live = (lse[:cu[-1]][done].double() - want_lse[done]), want_lse[done] > -math.inf
    assert bool((lse[:cu[-1]][done][~live] == -math.inf).all())
    assert bool((e[live].abs() <= (16 * 2.0 ** -23 * big[done] + 2.0 ** -19 + 5 * 2.0 ** -23 * want_lse[done].abs())[live]).all())
    assert bool((lse[cu[-1]:] == 7).all()) and bool((buf[cu[-1]:] == 7).all()) and bool((buf[:, -1] == 7).all())
    assert mx.device_timeouts() == 0 and cache.guards_intact()


def test_masks_on_streams_and_in_graphs(mx):  # noqa: F811
    """Calls with workspaces of their own on two streams and as graphs: the bits of a call alone."""
    jobs = []
    for seed, (nq, lens) in enumerate((([1, 1], [6000, 900]), ([70, 7], [700, 3000]), ([9], [5000]))):
        cu, table, cache, q, buf, out, lse, max_q, max_len, ws = job(mx, 8, 4, 128, 64, 16, nq, lens, seed)
        mask = kr.words([r for n in nq for r in random_tree(n, random.Random(n))] + [0] * 3, 3).cuda()
        fixed = (q, dev(cu), dev(lens), dev(table), *cache.parts)
        if seed == 0:
            call = lambda to, f=fixed, a=(max_q, max_len), w=ws: mx.mxkv_attention_sinks(*f, to, *a, 0.1, 500, 20, workspace=w)  # noqa: E731
        else:
            call = lambda to, f=fixed, a=(max_q, max_len), w=ws, m=mask: mx.mxkv_attention_tree(*f, to, *a, 0.1, m, workspace=w)  # noqa: E731
        alone, again = torch.zeros_like(q), torch.zeros_like(q)
        call(alone)
        jobs.append((call, alone, again, torch.cuda.Stream(), cache))
    torch.cuda.synchronize()
    for _ in range(10):
        for call, _, again, stream, _ in jobs:
            with torch.cuda.stream(stream):
                call(again)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for _, a, b, _, _ in jobs)
    graphs = []
    for call, _, again, stream, _ in jobs:
        again.zero_()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            call(again)
    for _ in range(10):
        for graph, (_, _, _, stream, _) in zip(graphs, jobs):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for _, a, b, _, _ in jobs)
    assert mx.device_timeouts() == 0


@pytest.mark.parametrize("dim,block", [(64, 16), (128, 64)])
@pytest.mark.parametrize("length", [1030, 1100, 2047, 4096, 5000])
def test_trees_of_up_to_128_rows(mx, dim, block, length):  # noqa: F811
    """Up to 128 rows for a key head, in chunks: odd and even numbers of tiles, value scales far apart within and between tiles, runs of zero values."""
    qh, h, nq = 16, 2, [16, 9, 12]
    lens = [length, 1025, 300]
    pick = random.Random(length)
    rows = [random_tree(n, pick) for n in nq]
    for spread in (0, 40):
        cu, table, cache, q, buf, out, lse, max_q, max_len, ws = job(mx, qh, h, dim, 64, block, nq, lens, 5)
        if spread:
            g = torch.Generator(device="cuda").manual_seed(length)
            for s, n in enumerate(lens):
                for i in range(-(-n // 64)):
                    v = cache.parts[3][table[s][i]]
                    v.copy_(torch.randint(90, 90 + spread, v.shape, generator=g, device="cuda").to(torch.uint8))
                    if i % 3 == 1:
                        v.zero_()
                        cache.parts[2][table[s][i]].zero_()
        scale, mask = dim ** -0.5, kr.words([r for sequence in rows for r in sequence] + [0] * 3, 1).cuda()
        masks = [kr.tree_mask(sequence, n, device="cuda") for sequence, n in zip(rows, lens)]
        # weights are rounded beside the largest product of weight and value scale of their tile: the bound goes by the softmax |v| as ever
        compare(mx, lambda: mx.mxkv_attention_tree(q, dev(cu), dev(lens), dev(table), *cache.parts, out, max_q, max_len, scale, mask, lse=lse, workspace=ws),
                q, cu, lens, table, cache, scale, masks, out, lse, buf)
