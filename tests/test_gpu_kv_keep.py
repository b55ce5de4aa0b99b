"""Summed weights of the keys, the choice of tokens that stay and moving them together, on the GPU against 64 bits.

A weight's exponent is a score minus lse: the score is off by at most 16 roundings of its sum of magnitudes and a few of itself, lse * log2 e by
one; the exponential adds 2^-21, a sum over N rows at most N / 8 roundings (eight partial sums each) of the whole.  Choices and moves have to be exact."""
import math
import random

import pytest
import torch

from tests import keep_ref as kr
from tests import qkv_ref as ref
from tests.test_gpu_kv import Cache, cumulative, dev, fill, make_table, mx  # noqa: F401

pytestmark = pytest.mark.gpu


def sums_buffer(pool, heads, page, value=7.0):
    full = torch.full((pool * heads * page + 128,), -3.0, device="cuda")
    part = full[64:-64].view(pool, heads, page)
    part.fill_(value)
    return full, part


def check_weights(mx, qh, h, dim, page, block, nq, lens, causal=True, window=0, sinks=0, earlier="other", seed=0, max_q=None, max_len=None, edit=None,
                  align=0):
    cu, n = cumulative(nq), sum(nq)
    bound = max(max(lens), 1) if max_len is None else max_len
    table, pool = make_table(lens, -(-max(lens + [1]) // page) + 1, page, seed, junk=-7 if seed % 2 else 2 ** 30)
    cache = Cache(pool, h, page, dim, block)
    fill(cache, lens, table, page, block, seed)
    kc, ks = cache.parts[0], cache.parts[1]
    if align:   # codes that are no more than 16-byte aligned
        room = torch.empty(kc.numel() + 64, dtype=torch.uint8, device="cuda")
        at = (align - room.data_ptr()) % 32
        moved = room[at:at + kc.numel()].view(kc.shape)
        moved.copy_(kc)
        kc = moved
    x = (2 * torch.randn(n + 3, (qh + 2) * dim, generator=torch.Generator().manual_seed(seed + 1))).to(torch.bfloat16).cuda()
    q = x[:, dim:(qh + 1) * dim].view(-1, qh, dim)
    masks = [kr.sinks_mask(b - a, length, window, sinks, causal, device="cuda") for a, b, length in zip(cu, cu[1:], lens)]
    if max_len is not None:
        masks = [m & (torch.arange(m.shape[1], device="cuda") < max_len) for m in masks]
    scale = dim ** -0.5
    lse = torch.full((n + 3, qh), math.nan, device="cuda")
    lse[:n] = kr.attention(q[:n], cu, lens, table, kc, ks, kc, ks, scale, masks)[1].float()
    if edit is not None:
        edit(q, lse)
    full, sums = sums_buffer(pool, h, page)
    before = torch.exp(torch.randn(pool, h, page, generator=torch.Generator().manual_seed(seed + 2))).cuda() if earlier else None
    if earlier == "same":
        sums.copy_(before)
    if max_q is not None:
        keep_rows = [torch.arange(b - a, device="cuda") < max_q for a, b in zip(cu, cu[1:])]
        masks = [m & k[:, None] for m, k in zip(masks, keep_rows)]
    want = sums.double().clone()
    # (rows that nothing is asked of give nothing: their lse is of no use here)
    slack = kr.weights(q[:n], lse, cu, lens, table, kc, ks, scale, masks, want, before)
    if max_len is not None:
        for s, length in enumerate(lens):
            for t in range(max_len, length):
                pg, o = table[s][t // page], t % page
                want[pg, :, o], slack[pg, :, o] = sums[pg, :, o].double(), 0
    call = lambda to: mx.mxkv_attention_weights(q, dev(cu), dev(lens), dev(table), kc, ks, lse, to, max(max(nq), 1) if max_q is None else max_q, bound,  # noqa: E731
                                                scale, earlier=to if earlier == "same" else before, causal=causal, window=window, sinks=sinks)
    again = sums.clone()
    call(sums)
    torch.cuda.synchronize()
    assert mx.device_timeouts() == 0
    nan = want.isnan()
    assert bool((sums.isnan() == nan).all())
    err = (sums.double() - want).abs()[~nan]
    assert bool((err <= slack[~nan]).all()), f"off by {float((err / slack[~nan].clamp(min=1e-30)).max()):.3g} tolerances"
    assert bool((full[:64] == -3).all()) and bool((full[-64:] == -3).all()) and cache.guards_intact()
    call(again)
    assert torch.equal(sums.nan_to_num(-1), again.nan_to_num(-1)), "not repeatable"
    return sums, table, pool


FEW = [  # query heads, key heads, dim, page, block, new queries, lengths
    (1, 1, 64, 16, 16, [1], [1]), (32, 8, 128, 64, 16, [1] * 5, [1, 63, 64, 65, 700]), (8, 1, 64, 128, 64, [1, 1], [127, 2049]),
    (16, 1, 128, 64, 32, [1, 0], [300, 17]), (14, 2, 64, 16, 16, [1, 1, 1], [15, 16, 500]), (64, 2, 64, 64, 64, [1], [129]),
    (6, 2, 64, 32, 16, [2, 3, 4, 1], [2, 70, 1000, 5]), (8, 2, 128, 16, 16, [8, 5, 7], [8, 9, 129]), (4, 4, 128, 16, 16, [1] * 40, list(range(1, 41))),
    (2, 1, 128, 64, 16, [1], [20000]),
]
MANY = [
    (4, 1, 128, 64, 16, [100], [100]), (8, 2, 64, 32, 32, [129, 17, 64], [129, 400, 64]), (4, 4, 128, 16, 16, [33], [2000]),
    (6, 1, 128, 128, 64, [257, 1, 300], [300, 77, 300]), (2, 2, 64, 64, 16, [1000], [1500]), (8, 1, 128, 64, 16, [128, 256], [128, 1031]),
    (5, 1, 64, 16, 16, [200, 40], [150, 40]), (3, 1, 128, 64, 16, [255, 0, 86], [255, 300, 257]), (160, 1, 64, 64, 16, [3, 1], [300, 260]),
    (300, 1, 128, 32, 32, [2], [258]), (16, 1, 64, 256, 64, [1040], [1040]),
]


@pytest.mark.parametrize("qh,h,dim,page,block,nq,lens", FEW + MANY)
@pytest.mark.parametrize("causal,window,sinks", [(True, 0, 0), (False, 0, 0), (True, 70, 0), (False, 200, 0), (True, 50, 5), (True, 130, 140)])
def test_weights(mx, qh, h, dim, page, block, nq, lens, causal, window, sinks):  # noqa: F811
    check_weights(mx, qh, h, dim, page, block, nq, lens, causal, window, sinks, seed=dim + page + window, earlier=["other", "same", None][window // 50 % 3])


@pytest.mark.parametrize("nq", [1, 90])
def test_weights_codes_of_other_alignment(mx, nq):  # noqa: F811
    check_weights(mx, 4, 2, 128, 64, 16, [nq, nq], [400, 333], align=16, seed=nq)


@pytest.mark.parametrize("nq,max_q,max_len", [([4, 2], 2, None), ([100, 30], 40, None), ([1, 1], None, 100), ([80, 90], None, 150)])
def test_weights_beyond_the_bounds(mx, nq, max_q, max_len):  # noqa: F811
    """Rows past max_q_len give nothing; tokens past max_kv_len are neither read nor written."""
    check_weights(mx, 8, 2, 64, 32, 16, nq, [300, 160], max_q=max_q, max_len=max_len, seed=3)


@pytest.mark.parametrize("nq", [3, 80])
def test_weights_nan_and_rows_that_saw_nothing(mx, nq):  # noqa: F811
    """A NaN in one row reaches the keys it sees and no other; a row whose lse is -infinity gives nothing."""
    def edit(q, lse):
        q[1, 0, 5] = math.nan
        lse[1, 0] = math.nan
        lse[2, 1] = -math.inf
    sums, table, _ = check_weights(mx, 2, 2, 64, 32, 16, [nq], [200], edit=edit, seed=5)
    key = torch.arange(200, device="cuda")
    pages = torch.tensor(table[0], device="cuda")[key // 32]
    assert bool((sums[pages, 0, key % 32].isnan() == (key <= 200 - nq + 1)).all()) and not bool(sums[pages, 1, key % 32].isnan().any())


def test_weights_add_up_to_the_rows(mx):  # noqa: F811
    """Each row's softmax weights sum to 1, so all keys' sums add up to the number of rows that see something; over calls too."""
    heads, dim, page, block, qh = 2, 128, 64, 16, 8
    table, pool = make_table([700], 12, page, 1)
    cache = mx.alloc_kv_cache(pool, heads, page, dim, block)
    g = torch.Generator().manual_seed(9)
    sums = torch.zeros(pool, heads, page, device="cuda")
    done = rows = 0
    for new in (500, 1, 1, 70, 3, 125):
        done += new
        x = torch.randn(new, qh + 2 * heads, dim, generator=g).to(torch.bfloat16).cuda()
        lists = (dev([0, new]), dev([done]), dev(table))
        mx.mxkv_append(x[:, qh:qh + heads], x[:, qh + heads:], *lists, *cache)
        q, out, lse = x[:, :qh], torch.empty(new, qh, dim, dtype=torch.bfloat16, device="cuda"), torch.empty(new, qh, device="cuda")
        ws = torch.empty(max(16, mx.mxkv_attention_workspace_bytes(new, 1, new, done, qh, heads, dim)), dtype=torch.uint8, device="cuda")
        mx.mxkv_attention(q, *lists, *cache, out, new, done, dim ** -0.5, lse=lse, workspace=ws)
        mx.mxkv_attention_weights(q, *lists, cache[0], cache[1], lse, sums, new, done, dim ** -0.5, earlier=sums)
        rows += new
        # lse and the exponents are off by at most 16 * 2^-23 of sum |q k| (about 7) and 2^-19 each: below 1e-4 a row
        assert float((sums.double().sum((0, 2)) - rows * qh // heads).abs().max()) < 1e-4 * rows * qh // heads + 1e-3


# ---- choice ----------------------------------------------------------------------------------------------------------

def run_select(mx, w, lens, table, heads, keep, sinks, recent, max_len):
    kept = torch.full((len(lens), heads, keep), -9, dtype=torch.int32, device="cuda")
    new_lens = torch.full((len(lens),), -9, dtype=torch.int32, device="cuda")
    mx.mxkv_select(w, dev(lens), dev(table), kept, new_lens, max_len, sinks=sinks, recent=recent)
    return kept.cpu(), new_lens.cpu()


@pytest.mark.parametrize("heads,page,lens,keep,sinks,recent", [
    (1, 16, [1], 1, 0, 0), (1, 16, [2], 1, 0, 0), (2, 64, [100, 0, 33, 34], 33, 4, 8), (8, 32, [1000, 999, 64, 5000], 512, 4, 100),
    (3, 128, [20000], 7000, 16, 1000), (1, 64, [70000, 12], 20000, 0, 0), (2, 16, [600] * 5, 599, 1, 1), (2, 16, [500, 90], 90, 40, 50),
    (1, 256, [5000], 1, 0, 1), (1, 256, [5000], 1, 1, 0), (40, 64, [300] * 9, 100, 4, 20), (1, 64, [300000], 100000, 5, 7),
])
@pytest.mark.parametrize("form", ["spread", "ties", "special"])
def test_select(mx, heads, page, lens, keep, sinks, recent, form):  # noqa: F811
    """Weights spread over many binades; a few values only, so that places decide; infinities, NaN, both zeros and negative ones."""
    table, pool = make_table(lens, -(-max(lens) // page) + 1, page, 3, junk=2 ** 30)
    g = torch.Generator().manual_seed(len(lens) + keep)
    w = torch.exp(6 * torch.randn(pool, heads, page, generator=g))
    if form == "ties":
        w = torch.randint(0, 4, w.shape, generator=g).float()
    if form == "special":
        pick = torch.randint(0, 9, w.shape, generator=g)
        for i, v in enumerate((math.inf, -math.inf, math.nan, 0.0, -0.0, 1e-45)):
            w[pick == i] = v
        w[pick == 6] *= -1
    kept, new_lens = run_select(mx, w.cuda(), lens, table, heads, keep, sinks, recent, max(lens))
    rows = []
    for s, length in enumerate(lens):
        key = torch.arange(length)
        pages = torch.tensor(table[s])[key // page]
        rows.append([w[pages, h, key % page] for h in range(heads)])
    want = kr.select(rows, lens, keep, sinks, recent)
    assert new_lens.tolist() == [min(x, keep) for x in lens]
    for s in range(len(lens)):
        for h in range(heads):
            assert kept[s, h].tolist() == want[s][h] + [-1] * (keep - len(want[s][h])), (s, h)
    assert mx.device_bad_indices() == 0


def test_select_bad_pages_and_bounds(mx):  # noqa: F811
    """A page out of range: its tokens come last (after a NaN's place among equals) and are counted; tokens past the bound do not exist."""
    mx.device_bad_indices_reset()
    w = torch.rand(4, 2, 16, generator=torch.Generator().manual_seed(1)).cuda()
    kept, _ = run_select(mx, w, [64], [[0, -1, 2, 99]], 2, 32, 0, 0, 64)
    assert kept[0].tolist() == [list(range(16)) + list(range(32, 48))] * 2 and mx.device_bad_indices() > 0
    mx.device_bad_indices_reset()
    kept, n = run_select(mx, w, [64], [[0, 1, 2, 3]], 2, 20, 0, 5, 17)
    assert kept[0].tolist() == [list(range(17)) + [-1] * 3] * 2 and n.tolist() == [17]


# ---- moving ----------------------------------------------------------------------------------------------------------

def check_compact(mx, heads, dim, page, block, lens, lists, first=None, new_lens=None, out=False, seed=0, edit=None, width=None):
    """lists[s][h or 0]; the result bit for bit that of the plain statement."""
    table, pool = make_table(lens, width or -(-max(lens) // page) + 1, page, seed, junk=2 ** 30)
    new_lens = [(first[s] if first else 0) + len(lists[s][0]) for s in range(len(lens))] if new_lens is None else new_lens
    out_table, extra = table, 0
    if out:
        out_table, extra = make_table([max(1, x) for x in new_lens], -(-max(new_lens) // page) + 1, page, seed + 1, junk=-1)
        out_table = [[p + pool if 0 <= p < extra else p for p in row] for row in out_table]
    cache = Cache(pool + extra, heads, page, dim, block, code=9, scale=100)
    fill(cache, lens, table, page, block, seed, k_spread=6, v_spread=6)
    if edit is not None:
        edit(cache, table)
    full, sums = sums_buffer(pool + extra, heads, page)
    sums.copy_(torch.rand(sums.shape, generator=torch.Generator().manual_seed(seed)))
    want, want_sums = cache.cpu(), sums.cpu().clone()
    for i in (0, 2):
        kr.compact(want[i], want[i + 1], lists, first, new_lens, table, out_table, page, block)
    was = want_sums.clone()
    for s, end in enumerate(new_lens):
        f = first[s] if first else 0
        for h in range(heads):
            kept = lists[s][h if len(lists[s]) > 1 else 0]
            for p in range(f, end):
                want_sums[out_table[s][p // page], h, p % page] = was[table[s][kept[p - f] // page], h, kept[p - f] % page]
    n = max(max(len(x) for row in lists for x in row), 1)
    kept = torch.full((len(lens), len(lists[0]), n), -4, dtype=torch.int32)
    for s, row in enumerate(lists):
        for h, x in enumerate(row):
            kept[s, h, :len(x)] = torch.tensor(x, dtype=torch.int32)
    ws = torch.full((mx.mxkv_compact_workspace_bytes(len(lens), heads, n),), 0xFF, dtype=torch.uint8, device="cuda")
    mx.mxkv_compact(kept.cuda(), dev(new_lens), dev(lens), dev(table), *cache.parts, out_page_table=dev(out_table) if out else None,
                    first=dev(first) if first else None, weights=sums, workspace=None if out else ws)
    torch.cuda.synchronize()
    assert mx.device_timeouts() == 0
    for name, got, w in zip(("k codes", "k scales", "v codes", "v scales"), cache.parts, want):
        got = got.cpu()
        if "codes" in name:   # a NaN's sign says nothing
            got, w = (torch.where((t & 0x7F) == 0x7F, torch.full_like(t, 0x7F), t) for t in (got, w))
        assert torch.equal(got, w), name
    assert torch.equal(sums.cpu(), want_sums) and cache.guards_intact() and bool((full[:64] == -3).all()) and bool((full[-64:] == -3).all())
    return cache


def rising(pick, length, n):
    return sorted(pick.sample(range(length), n))


MOVES = [  # heads, dim, page, block, lengths, tokens that stay
    (1, 64, 16, 16, [1], [1]), (1, 128, 16, 16, [40], [7]), (2, 128, 64, 16, [100, 33, 700], [60, 33, 200]), (3, 64, 32, 32, [500, 64, 65], [100, 1, 64]),
    (8, 128, 64, 64, [1000, 130], [999, 65]), (2, 64, 256, 64, [3000], [2000]), (4, 128, 128, 32, [2000, 1], [130, 1]), (2, 128, 16, 16, [20000], [9000]),
    (1, 64, 64, 16, [300] * 30, list(range(1, 300, 10))),
]


@pytest.mark.parametrize("heads,dim,page,block,lens,n", MOVES)
@pytest.mark.parametrize("out", [False, True])
@pytest.mark.parametrize("shared", [False, True])
def test_compact(mx, heads, dim, page, block, lens, n, out, shared):  # noqa: F811
    pick = random.Random(dim + page)
    lists = [[rising(pick, length, k) for _ in range(1 if shared else heads)] for length, k in zip(lens, n)]
    check_compact(mx, heads, dim, page, block, lens, lists, out=out, seed=page + block)


@pytest.mark.parametrize("dim,page,block", [(64, 16, 16), (128, 64, 16), (128, 64, 64), (64, 128, 32)])
@pytest.mark.parametrize("out", [False, True])
def test_compact_a_path_of_a_tree(mx, dim, page, block, out):  # noqa: F811
    """One list for all heads behind a part that stays: lengths in front at, before and behind the ends of blocks and pages."""
    front = [0, 1, 15, 16, 63, 64, 65, 100, 127, 640]
    lens = [f + 24 for f in front]
    pick = random.Random(page)
    lists = [[[f + t for t in rising(pick, 24, 1 + f % 9)]] for f in front]
    # (to other pages: what stands in front of the list in its first block is what these pages hold)
    check_compact(mx, 2, dim, page, block, lens, lists, first=front, out=out, seed=block)


def test_compact_far_scales_zeros_and_nan(mx):  # noqa: F811
    """Blocks whose scales lie up to 200 binades apart, zeros, NaN codes, subnormal codes and scales at both ends."""
    def edit(cache, table):
        g = torch.Generator(device="cuda").manual_seed(2)
        for i in (0, 2):
            c, sc = cache.parts[i], cache.parts[i + 1]
            c.copy_(torch.randint(0, 256, c.shape, generator=g, device="cuda").to(torch.uint8))
            c[:, :, ::5] = 0
            c[:, :, 1::7] &= 0x87
            sc.copy_(torch.tensor([0, 1, 5, 17, 40, 110, 120, 121, 122, 130, 200, 240], dtype=torch.uint8, device="cuda")[
                torch.randint(0, 12, sc.shape, generator=g, device="cuda")])
    pick = random.Random(1)
    for dim, page, block in ((128, 64, 16), (64, 64, 32), (128, 64, 64)):
        check_compact(mx, 2, dim, page, block, [900, 64], [[rising(pick, 900, 300) for _ in range(2)], [rising(pick, 64, 20) for _ in range(2)]], seed=7,
                      edit=edit)


def test_compact_to_other_pages_in_any_order(mx):  # noqa: F811
    pick = random.Random(4)
    lists = [[[pick.randrange(500) for _ in range(700)] for _ in range(2)]]
    check_compact(mx, 2, 128, 32, 16, [500], lists, out=True, seed=3)


def test_compact_what_stays_is_left_alone(mx):  # noqa: F811
    """Blocks in front of the first gap keep their bits, scales larger than needed among them."""
    check_compact(mx, 2, 128, 64, 16, [500], [[list(range(200)) + list(range(230, 400))] * 2], seed=1)
    check_compact(mx, 2, 128, 64, 16, [500], [[list(range(500))] * 2], seed=1)
    check_compact(mx, 1, 64, 64, 16, [500, 90], [[list(range(300))], [list(range(10))]], new_lens=[300, 0], seed=2)


def test_compact_bad_entries(mx):  # noqa: F811
    """Blocks with an entry out of range, below its place or out of order, or a page out of range, are left as they are; others move."""
    heads, dim, page, block = 1, 128, 32, 16
    for kept, table, bad in (([5] + list(range(20, 35)) + [99] + list(range(40, 50)), [[0, 1]], 1), ([3, 4, -1] + list(range(10, 40)), [[0, 1]], 0),
                             ([2, 1] + list(range(10, 40)), [[0, 1]], 0), (list(range(20, 50)), [[0, 7]], 0)):
        cache = Cache(3, heads, page, dim, block, code=9, scale=100)
        g = torch.Generator(device="cuda").manual_seed(1)
        for i in (0, 2):
            cache.parts[i].copy_(torch.randint(0, 100, cache.parts[i].shape, generator=g, device="cuda").to(torch.uint8))
        before = cache.cpu()
        n = len(kept)
        ws = torch.empty(mx.mxkv_compact_workspace_bytes(1, heads, n), dtype=torch.uint8, device="cuda")
        mx.device_bad_indices_reset()
        mx.mxkv_compact(dev([[kept]]), dev([n]), dev([64]), dev(table), *cache.parts, workspace=ws)
        assert mx.device_bad_indices() > 0 and mx.device_timeouts() == 0 and cache.guards_intact()
        after = cache.cpu()
        assert torch.equal(after[0][0, 0, 16 * bad:16 * bad + 16], before[0][0, 0, 16 * bad:16 * bad + 16])
        assert torch.equal(after[0][2], before[0][2])
    for first, new_len in ((-1, 5), (70, 75), (2 ** 31 - 1, -2 ** 31), (0, 2 ** 31 - 1)):
        cache = Cache(3, heads, page, dim, block, code=9, scale=100)
        before = cache.cpu()
        kept = dev([[[0, 1, 2]]])
        ws = torch.empty(mx.mxkv_compact_workspace_bytes(1, heads, 3), dtype=torch.uint8, device="cuda")
        mx.device_bad_indices_reset()
        mx.mxkv_compact(kept, dev([new_len]), dev([64]), dev([[0, 1]]), *cache.parts, first=dev([first]), workspace=ws)
        assert mx.device_bad_indices() > 0
        assert all(torch.equal(a, b) for a, b in zip(before, cache.cpu()))
    mx.device_bad_indices_reset()


def test_compact_past_32_bits(mx):  # noqa: F811
    """Pages more than 2^32 bytes into the pool: the bits that a small pool gives."""
    heads, dim, page, block, length = 8, 128, 64, 16, 250
    pages = 2 ** 32 // (heads * dim * page) + 9
    pick = random.Random(2)
    lists = torch.tensor([[rising(pick, length, 100) for _ in range(heads)]], dtype=torch.int32).cuda()
    g = torch.Generator().manual_seed(3)
    x = torch.randn(length, 2 * heads, dim, generator=g).to(torch.bfloat16).cuda()
    results = []
    for pool, table in ((5, [[2, 0, 3, 1]]), (pages, [[pages - 2, pages - 4, pages - 1, pages - 3]])):
        cache = mx.alloc_kv_cache(pool, heads, page, dim, block)
        mx.mxkv_append(x[:, :heads], x[:, heads:], dev([0, length]), dev([length]), dev(table), *cache)
        ws = torch.empty(mx.mxkv_compact_workspace_bytes(1, heads, 100), dtype=torch.uint8, device="cuda")
        mx.mxkv_compact(lists, dev([100]), dev([length]), dev(table), *cache, workspace=ws)
        results.append([c[torch.tensor(table[0], device="cuda")] for c in cache])
        del cache
    assert all(torch.equal(a, b) for a, b in zip(*results)) and bool(results[0][0].any())


def test_evict_and_go_on(mx):  # noqa: F811
    """As a model runs them, captured once and replayed: append, attention, summed weights; then choice and move in place; then attention over what
    stayed, each head its own tokens, against 64 bits on the tokens that the plain statement keeps."""
    heads, qh, dim, page, block, length, keep = 2, 8, 128, 64, 16, 400, 130
    table, pool = make_table([length + 8], 8, page, 1)
    cache = mx.alloc_kv_cache(pool, heads, page, dim, block)
    g = torch.Generator().manual_seed(4)
    sums = torch.zeros(pool, heads, page, device="cuda")
    x = torch.randn(length, qh + 2 * heads, dim, generator=g).to(torch.bfloat16).cuda()
    out, lse = torch.empty(length, qh, dim, dtype=torch.bfloat16, device="cuda"), torch.empty(length, qh, device="cuda")
    ws = torch.empty(max(16, mx.mxkv_attention_workspace_bytes(length, 1, length, length, qh, heads, dim)), dtype=torch.uint8, device="cuda")
    kept = torch.empty(1, heads, keep, dtype=torch.int32, device="cuda")
    new_lens = torch.empty(1, dtype=torch.int32, device="cuda")
    lists = (dev([0, length]), dev([length]), dev(table))
    cws = torch.empty(mx.mxkv_compact_workspace_bytes(1, heads, keep), dtype=torch.uint8, device="cuda")

    def step():
        mx.mxkv_append(x[:, qh:qh + heads], x[:, qh + heads:], *lists, *cache)
        mx.mxkv_attention(x[:, :qh], *lists, *cache, out, length, length, dim ** -0.5, lse=lse, workspace=ws)
        mx.mxkv_attention_weights(x[:, :qh], *lists, cache[0], cache[1], lse, sums, length, length, dim ** -0.5)
        mx.mxkv_select(sums, lists[1], lists[2], kept, new_lens, length, sinks=4, recent=32)

    def move():
        mx.mxkv_compact(kept, new_lens, lists[1], lists[2], *cache, weights=sums, workspace=cws)

    step()
    torch.cuda.synchronize()
    full = [c.cpu().clone() for c in cache]
    chosen, w = kept.cpu(), sums.cpu().clone()
    key = torch.arange(length)
    pages = torch.tensor(table[0])[key // page]
    want = kr.select([[w[pages, h, key % page] for h in range(heads)]], [length], keep, 4, 32)
    assert chosen[0].tolist() == want[0] and new_lens.tolist() == [keep]
    move()
    torch.cuda.synchronize()
    moved = [c.cpu().clone() for c in cache]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
        move()
    for c in (*cache, sums, kept):
        c.zero_()
    graph.replay()
    torch.cuda.synchronize()
    slots = torch.arange(keep)
    at = torch.tensor(table[0])[slots // page]
    for a, b in zip((moved[0], moved[2]), (cache[0].cpu(), cache[2].cpu())):
        assert torch.equal(a[at, :, slots % page], b[at, :, slots % page])
    # two more tokens see what stayed
    for which in (0, 2):
        full_k = [ref.dequantise(full[which], full[which + 1], torch.tensor(table[0][:-(-length // page)]), block, h, length) for h in range(heads)]
        new_k = [ref.dequantise(moved[which], moved[which + 1], torch.tensor(table[0][:-(-keep // page)]), block, h, keep) for h in range(heads)]
        for h in range(heads):
            old = full_k[h][chosen[0, h].long()]
            # exact but for codes that become subnormal: half of E4M3's smallest step on a scale that lies 2^8 below the block's largest
            assert bool(((new_k[h] - old).abs() <= 2.0 ** -10 * 2.0 ** -7 * old.abs().amax()).all())
    y = torch.randn(2, qh + 2 * heads, dim, generator=g).to(torch.bfloat16).cuda()
    late = (dev([0, 2]), new_lens + 2, dev(table))
    mx.mxkv_append(y[:, qh:qh + heads], y[:, qh + heads:], *late, *cache)
    out2 = torch.empty(2, qh, dim, dtype=torch.bfloat16, device="cuda")
    ws2 = torch.empty(max(16, mx.mxkv_attention_workspace_bytes(2, 1, 2, length, qh, heads, dim)), dtype=torch.uint8, device="cuda")
    mx.mxkv_attention(y[:, :qh], *late, *cache, out2, 2, length, dim ** -0.5, workspace=ws2)
    want_out, _, mag, _ = ref.attention(y[:, :qh], [0, 2], [keep + 2], table, *cache, dim ** -0.5)
    assert bool(((out2.double() - want_out).abs() <= 2.0 ** -8 * want_out.abs() + (2.0 ** -8 + 2.0 ** -10) * mag).all())
    assert mx.device_timeouts() == 0 and mx.device_bad_indices() == 0


def test_tree_accepted_and_go_on(mx):  # noqa: F811
    """Drafts of a tree are appended, attended, a path of them accepted and moved together: what follows sees the same as if the path alone had been
    appended."""
    heads, qh, dim, page, block, front = 2, 8, 64, 32, 16, 40
    table, pool = make_table([120], 4, page, 1)
    g = torch.Generator().manual_seed(4)
    path, tree = [0, 2, 5, 9], 12
    base = torch.randn(front, 2 * heads, dim, generator=g).to(torch.bfloat16).cuda()
    drafts = torch.randn(tree, 2 * heads, dim, generator=g).to(torch.bfloat16).cuda()
    caches = []
    for rows in (drafts, drafts[path]):
        cache = mx.alloc_kv_cache(pool, heads, page, dim, block)
        mx.mxkv_append(base[:, :heads], base[:, heads:], dev([0, front]), dev([front]), dev(table), *cache)
        n = rows.shape[0]
        mx.mxkv_append(rows[:, :heads], rows[:, heads:], dev([0, n]), dev([front + n]), dev(table), *cache)
        caches.append(cache)
    kept = dev([[[front + t for t in path]]])
    ws = torch.empty(mx.mxkv_compact_workspace_bytes(1, heads, len(path)), dtype=torch.uint8, device="cuda")
    mx.mxkv_compact(kept, dev([front + len(path)]), dev([front + tree]), dev(table), *caches[0], first=dev([front]), workspace=ws)
    pages = torch.tensor(table[0][:2])
    for i in (0, 2):
        for h in range(heads):
            a, b = (ref.dequantise(c[i].cpu(), c[i + 1].cpu(), pages, block, h, front + len(path)) for c in caches)
            # the same mantissas, but for codes that are subnormal on one of the two scales (half a step: 2^-10 of a scale, each)
            assert bool(((a - b).abs() <= 2.0 ** -9 * 2.0 ** -7 * b.abs().amax() * 2).all())
    assert mx.device_timeouts() == 0 and mx.device_bad_indices() == 0


def test_compact_many_at_once_in_place(mx):  # noqa: F811
    """Calls in place on two streams, each with a workspace of its own, again and again from the same cache: the same bits each time."""
    heads, dim, page, block = 8, 128, 64, 16
    jobs = []
    for seed, lens in enumerate(([9000, 300], [4000] * 6)):
        table, pool = make_table(lens, 150, page, seed)
        cache = Cache(pool, heads, page, dim, block)
        fill(cache, lens, table, page, block, seed)
        w = torch.rand(pool, heads, page, generator=torch.Generator().manual_seed(seed)).cuda()
        kept = torch.empty(len(lens), heads, 2500, dtype=torch.int32, device="cuda")
        new_lens = torch.empty(len(lens), dtype=torch.int32, device="cuda")
        mx.mxkv_select(w, dev(lens), dev(table), kept, new_lens, max(lens), sinks=4, recent=64)
        ws = torch.empty(mx.mxkv_compact_workspace_bytes(len(lens), heads, 2500), dtype=torch.uint8, device="cuda")
        jobs.append(([c.clone() for c in cache.parts], cache, (kept, new_lens, dev(lens), dev(table)), ws, torch.cuda.Stream(), []))
    torch.cuda.synchronize()
    for _ in range(15):
        for was, cache, args, ws, stream, got in jobs:
            with torch.cuda.stream(stream):
                for c, w in zip(cache.parts, was):
                    c.copy_(w)
                mx.mxkv_compact(*args, *cache.parts, workspace=ws)
                got.append([c.clone() for c in cache.parts])
    torch.cuda.synchronize()
    for _, cache, _, _, _, got in jobs:
        assert all(torch.equal(a, b) for other in got[1:] for a, b in zip(got[0], other)) and cache.guards_intact()
    assert mx.device_timeouts() == 0


def test_weights_without_rows(mx):  # noqa: F811
    """No new tokens at all, or none in some sequences: earlier sums are passed on; sequences without tokens; nothing else is written."""
    heads, dim, page = 2, 64, 32
    lens = [70, 0, 5]
    table, pool = make_table(lens, 4, page, 2)
    cache = Cache(pool, heads, page, dim, 16)
    fill(cache, lens, table, page, 16, 1)
    before = torch.rand(pool, heads, page, generator=torch.Generator().manual_seed(1)).cuda()
    full, sums = sums_buffer(pool, heads, page)
    q, lse = torch.empty(0, 4, dim, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 4, device="cuda")
    want = sums.clone()
    for s, length in enumerate(lens):
        for t in range(length):
            want[table[s][t // page], :, t % page] = before[table[s][t // page], :, t % page]
    for max_q in (1, 500):
        mx.mxkv_attention_weights(q, dev([0, 0, 0, 0]), dev(lens), dev(table), cache.parts[0], cache.parts[1], lse, sums, max_q, 70, 0.1, earlier=before)
        assert torch.equal(sums, want) and bool((full[:64] == -3).all())
        sums.fill_(7.0)
    # one sequence has a row, by the kernels for few and for many rows
    for max_q in (1, 500):
        q = torch.zeros(1, 4, dim, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((1, 4), math.log(70.0), device="cuda")   # scores of zero: 1 / 70 for each of 70 keys and head
        mx.mxkv_attention_weights(q, dev([0, 1, 1, 1]), dev(lens), dev(table), cache.parts[0], cache.parts[1], lse, sums, max_q, 70, 0.1, earlier=before)
        key = torch.arange(70, device="cuda")
        pages = torch.tensor(table[0], device="cuda")[key // page]
        old = torch.where(key < 69, 1.0, 0.0)[:, None] * before[pages, :, key % page]
        assert bool(((sums[pages, :, key % page] - old - 2 / 70).abs() < 1e-6).all())
        assert torch.equal(sums[table[2][0], :, :5], before[table[2][0], :, :5])
        sums.fill_(7.0)


@pytest.mark.parametrize("offset", [1, 2, 3])
def test_select_weights_of_any_alignment(mx, offset):  # noqa: F811
    lens, heads, page = [900, 64], 2, 32
    table, pool = make_table(lens, 30, page, 5)
    room = torch.rand(pool * heads * page + 8, generator=torch.Generator().manual_seed(3)).cuda()
    w = room[offset:offset + pool * heads * page].view(pool, heads, page)
    kept, new_lens = run_select(mx, w, lens, table, heads, 100, 4, 20, 900)
    other, _ = run_select(mx, w.clone(), lens, table, heads, 100, 4, 20, 900)
    assert torch.equal(kept, other) and new_lens.tolist() == [100, 64]


def test_keeping_on_streams(mx):  # noqa: F811
    """Summed weights (few rows, prompts in both head sizes), choice and attention on four streams at once: the bits of a call alone."""
    jobs = []
    for seed, (qh, heads, dim, nq, lens) in enumerate(((8, 2, 128, [1, 1], [9000, 400]), (8, 2, 128, [700, 90], [2000, 700]), (8, 4, 64, [600], [3000]),
                                                       (16, 2, 64, [9, 9], [700, 300]))):
        cu, n = cumulative(nq), sum(nq)
        table, pool = make_table(lens, 150, 64, seed)
        cache = Cache(pool, heads, 64, dim, 16)
        fill(cache, lens, table, 64, 16, seed)
        q = torch.randn(n, qh, dim, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda()
        lists = (dev(cu), dev(lens), dev(table))
        out, lse = torch.empty_like(q), torch.empty(n, qh, device="cuda")
        ws = torch.empty(max(16, mx.mxkv_attention_workspace_bytes(n, len(nq), max(nq), max(lens), qh, heads, dim)), dtype=torch.uint8, device="cuda")

        def call(sums, kept, q=q, lists=lists, cache=cache, out=out, lse=lse, ws=ws, a=(max(nq), max(lens), dim ** -0.5)):
            mx.mxkv_attention(q, *lists, *cache.parts, out, *a, lse=lse, workspace=ws)
            mx.mxkv_attention_weights(q, *lists, cache.parts[0], cache.parts[1], lse, sums, *a)
            mx.mxkv_select(sums, lists[1], lists[2], kept[0], kept[1], a[1], sinks=2, recent=9)
        new = lambda n=len(nq), h=heads, p=pool: (torch.zeros(p, h, 64, device="cuda"),  # noqa: E731
                                                  (torch.zeros(n, h, 100, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")))
        alone, again = new(), new()
        call(*alone)
        jobs.append((call, alone, again, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(10):
        for call, _, again, stream in jobs:
            with torch.cuda.stream(stream):
                call(*again)
    torch.cuda.synchronize()
    for _, alone, again, _ in jobs:
        assert torch.equal(alone[0], again[0]) and torch.equal(alone[1][0], again[1][0])
    assert mx.device_timeouts() == 0


def test_compact_a_list_for_each_head_behind_a_part_that_stays(mx):  # noqa: F811
    """Different tokens for each head, in place, with a first place inside a block; lists as long as the row of the table allows."""
    pick = random.Random(8)
    first = [37, 64, 500]
    lens = [400, 64 + 300, 501]
    n = [90, 299, 1]
    lists = [[[f + t for t in rising(pick, length - f, k)] for _ in range(3)] for f, length, k in zip(first, lens, n)]
    for dim, page, block in ((128, 64, 16), (64, 32, 32), (128, 64, 64)):
        check_compact(mx, 3, dim, page, block, lens, lists, first=first, seed=dim + block)
