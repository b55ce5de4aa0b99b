"""mxkv_attention and mxkv_append where scales, windows, bounds and places go to their ends.

Tolerances are those of test_gpu_kv.py, whose helpers are used, unless a test says otherwise."""
import math

import pytest
import torch

from tests import qkv_ref as ref
from tests.test_gpu_kv import Cache, check, cumulative, dev, fill, make_table, mx  # noqa: F401  (mx is the fixture)

pytestmark = pytest.mark.gpu


def dense(q, place, k, v, scale, causal, window, limit):
    """(out, lse, sum of softmax |v|, largest sum of |scale q k|) of one head in 64 bits: queries q [n, D] at `place` [n] over keys and
    values [length, D], of which those from `limit` on are not seen."""
    key = torch.arange(k.shape[0], device=k.device)[None]
    seen = (key < limit) & ((key <= place[:, None]) if causal else (key >= 0))
    if window:
        seen = seen & (key > place[:, None] - window)
    z = (q.double() @ k.T * scale).masked_fill(~seen, -math.inf)
    p = torch.nan_to_num(torch.softmax(z, -1), 0.0)
    big = ((q.double().abs() @ k.abs().T) * abs(scale)).masked_fill(~seen, 0).amax(-1)
    return p @ v, torch.logsumexp(z, -1), p @ v.abs(), big


WIDE = 2.0 ** -8 + 2.0 ** -10


def near(out, lse, want, want_lse, mag, big, weight=WIDE):
    tol = 2.0 ** -8 * want.abs() + weight * mag + 1e-30
    assert bool(((out.double() - want).abs() <= tol).all()), f"out: {float(((out.double() - want).abs() / tol).max()):.3g} tolerances"
    live = want_lse > -math.inf
    assert bool((lse[~live] == -math.inf).all()) and not bool(out[~live].any())
    t = (16 * 2.0 ** -23 * big + 2.0 ** -19 + 5 * 2.0 ** -23 * want_lse.abs())[live]
    e = (lse.double() - want_lse).abs()[live]
    assert bool((e <= t).all()), f"lse: {float((e / t).max()):.3g} tolerances"


def attend(mx, q, cu, lens, table, cache, max_q, max_len, scale, **options):  # noqa: F811
    """(out, lse) with rows that the call leaves alone at 7."""
    n, q_heads, dim = q.shape
    out, lse = torch.full_like(q, 7.0, memory_format=torch.contiguous_format), torch.full((n, q_heads), 7.0, device="cuda")
    nbytes = mx.mxkv_attention_workspace_bytes(n, len(lens), max_q, max_len, q_heads, cache.parts[0].shape[1], dim)
    ws = torch.full((max(16, nbytes),), 0xFF, dtype=torch.uint8, device="cuda")
    mx.mxkv_attention(q, dev(cu), dev(lens), dev(table), *cache.parts, out, max_q, max_len, scale, lse=lse, workspace=ws, **options)
    torch.cuda.synchronize()
    assert mx.device_timeouts() == 0
    return out, lse


def agrees(mx, nq, lens, heads, group, dim, page, max_len, rows=None, seed=3, scale=None, q_std=1.0, weight=WIDE, **options):  # noqa: F811
    """The call against `dense`, sequence by sequence; `rows`: rows of q that there are (the last sequence may go on behind them)."""
    block, cu = 16, cumulative(nq)
    rows = cu[-1] if rows is None else rows
    table, pool = make_table(lens, -(-max(lens) // page), page, seed)
    cache = Cache(pool, heads, page, dim, block)
    fill(cache, lens, table, page, block, seed)
    q = (q_std * torch.randn(rows, heads * group, dim, generator=torch.Generator().manual_seed(seed))).to(torch.bfloat16).cuda()
    scale = dim ** -0.5 if scale is None else scale
    out, lse = attend(mx, q, cu, lens, table, cache, max(nq), max_len, scale, **options)
    for s, length in enumerate(lens):
        a, b = cu[s], min(cu[s + 1], rows)
        place = length - nq[s] + torch.arange(b - a, device="cuda")
        pages = torch.tensor(table[s][:-(-length // page)], device="cuda")
        for h in range(heads * group):
            k, v = (ref.dequantise(c, sc, pages, block, h // group, length) for c, sc in (cache.parts[:2], cache.parts[2:]))
            near(out[a:b, h], lse[a:b, h],
                 *dense(q[a:b, h], place, k, v, scale, options.get("causal", True), options.get("window", 0), max_len), weight)
    assert cache.guards_intact()


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


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nq,lens,max_len", [
    ([10], [100], 90), ([1, 4, 3], [500, 90, 333], 320), ([70], [300], 250), ([200, 90], [400, 130], 256), ([40, 1], [1300, 2000], 1290),
])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 25), (False, 0), (False, 100), (True, 400)])
def test_lengths_above_the_bound(mx, dim, nq, lens, max_len, causal, window):  # noqa: F811
    """Keys past max_kv_len are not seen; the queries stand where kv_lens puts them all the same."""
    agrees(mx, nq, lens, 2, 2, dim, 32, max_len, causal=causal, window=window)


@pytest.mark.parametrize("nq,lens,rows", [([3, 8], [40, 100], 7), ([5, 300], [64, 500], 180), ([2, 4], [9, 3000], 4)])
@pytest.mark.parametrize("window", [0, 30])
def test_rows_end_before_the_last_sequence(mx, nq, lens, rows, window):  # noqa: F811
    """cu_q goes on behind the rows that there are: those that are there keep their places."""
    agrees(mx, nq, lens, 2, 4, 64, 16, max(lens), rows=rows, window=window)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nq,lens", [([8], [3]), ([6, 5, 40], [2, 5, 30]), ([100], [60]), ([300, 200], [100, 190])])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 5, 2 ** 30])
@pytest.mark.parametrize("causal", [True, False])
def test_windows_without_end(mx, dim, nq, lens, window, causal):  # noqa: F811
    """A window as large as it may be hides nothing, with queries that stand before the first key among the rows."""
    agrees(mx, nq, lens, 2, 3, dim, 32, max(lens), window=window, causal=causal)


def zero_values(length, zeros, key_zero, key_rest):
    """Pages of 32 tokens, all sequences alike: tokens zeros[0] .. zeros[1] - 1 have values of zero (scale 0, as the append leaves them)
    and keys of the one code, the others the other; all queries are ones."""
    def setup(cache, q, table):
        kc, ks, vc, vs = cache.parts
        q.fill_(1.0)
        key = torch.tensor([key_zero, key_rest]).to(torch.float8_e4m3fn).view(torch.uint8).tolist()
        pages = torch.tensor(table, device="cuda")
        for t in range(0, length, 16):
            pg, at, zero = pages[:, t // 32], t % 32, zeros[0] <= t < zeros[1]
            end = at + min(16, length - t)
            kc[pg, :, at:end] = key[0] if zero else key[1]
            kc[pg, 0, at:end, 0] ^= (torch.arange(end - at, device="cuda") % 2 * 0x80).to(torch.uint8)   # not all the same score
            ks[pg, :, at // 16] = 121
            if zero:
                vc[pg, :, at:end] = 0
                vs[pg, :, at // 16] = 0
    return setup


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nq,length", [(1, 1100), (4, 1100), (100, 1100), (1, 6000), (60, 1100)])
@pytest.mark.parametrize("zeros", [(0, 16), (0, 32), (0, 64), (0, 128), (0, 1008), (48, 208), (496, 1100)])
@pytest.mark.parametrize("key_zero,key_rest", [(0.0, 0.0), (0.0, 40.0), (40.0, 0.0), (-448.0, 448.0), (448.0, -208.0)])
def test_runs_of_zero_values(mx, dim, nq, length, zeros, key_zero, key_rest):  # noqa: F811
    """Zero values with scores as large as the others', far below or far above: they count in the softmax's sum, whatever the scale."""
    check(mx, 4, 2, dim, 32, 16, [nq], [length], seed=dim, setup=zero_values(length, zeros, key_zero, key_rest))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nq", [1, 4])
@pytest.mark.parametrize("zeros", [(0, 32), (0, 128), (48, 208)])
@pytest.mark.parametrize("key_zero,key_rest", [(0.0, 0.0), (0.0, 40.0), (448.0, -208.0)])
def test_runs_of_zero_values_in_long_chunks(mx, dim, nq, zeros, key_zero, key_rest):  # noqa: F811
    """The same where many sequences leave each warp several tiles one after another."""
    check(mx, 16, 8, dim, 32, 16, [nq] * 80, [400] * 80, seed=dim, setup=zero_values(400, zeros, key_zero, key_rest))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nq,lens", [([1, 3], [700, 5000]), ([16], [900]), ([50, 100], [300, 2000])])
@pytest.mark.parametrize("low,high", [(-127, 0), (-127, 100), (-60, 60), (-25, -4), (60, 110)])
@pytest.mark.parametrize("window", [0, 300])
def test_value_scales_over_all_of_their_range(mx, dim, nq, lens, low, high, window):  # noqa: F811
    check(mx, 8, 2, dim, 32, 16, nq, lens, window=window, seed=dim + high, setup=value_scales(low, high))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page,block", [(16, 16), (32, 16), (64, 32), (128, 64), (256, 16)])
@pytest.mark.parametrize("nq,lens,window", [
    ([1], [121], 4), ([1, 1, 4], [1000, 300, 2500], 100), ([4], [9000], 700), ([70], [500], 10), ([90, 200], [800, 3000], 300), ([300], [2000], 1),
    ([40, 1], [1500, 1400], 33),
])
@pytest.mark.parametrize("causal", [True, False])
def test_pages_behind_the_window(mx, dim, page, block, nq, lens, window, causal):  # noqa: F811
    """Pages that lie before every query's window: released (no page of the pool) or full of NaN, they change nothing, and no bad
    index is counted; the same for NaN values before the window in the page that it begins in."""
    heads, group = 2, 2
    table, pool = make_table(lens, -(-max(lens) // page), page, page + dim)
    cache = Cache(pool, heads, page, dim, block)
    fill(cache, lens, table, page, block, dim)
    q = torch.randn(sum(nq), heads * group, dim, generator=torch.Generator().manual_seed(page)).to(torch.bfloat16).cuda()
    cu = cumulative(nq)
    call = lambda t: attend(mx, q, cu, lens, t, cache, max(nq), max(lens), dim ** -0.5, causal=causal, window=window)  # noqa: E731
    mx.device_bad_indices_reset()
    want = call(table)
    released = []
    for s, length in enumerate(lens):
        first = max(0, length - nq[s] - window + 1)
        row = list(table[s])
        for i in range(first // page):
            cache.parts[0][row[i]] = cache.parts[2][row[i]] = 0x7F
            cache.parts[1][row[i]] = cache.parts[3][row[i]] = 0xFF
            row[i] = -1 if i % 2 else pool + i
        # the page in which the window begins: its tokens before the window, in blocks that are all before it with their scales
        pg, n = row[first // page], first % page
        cache.parts[0][pg, :, :n] = cache.parts[2][pg, :, :n] = 0x7F
        released.append(row)
    assert all(torch.equal(a, b) for a, b in zip(want, call(table))), "NaN behind the window"
    assert all(torch.equal(a, b) for a, b in zip(want, call(released))), "released pages behind the window"
    assert mx.device_bad_indices() == 0
    assert bool(want[0].isfinite().all())


# what test_gpu_kv.py asks of the kernel for few rows, asked of the one for many

@pytest.mark.parametrize("size", [2.0 ** -100, 2.0 ** -20, 2.0 ** 100])
@pytest.mark.parametrize("dim", [64, 128])
def test_prompt_query_sizes(mx, size, dim):  # noqa: F811
    """Queries far from one, against key scales as far the other way."""
    def setup(cache, q, table):
        q.mul_(size)
        ks = cache.parts[1]
        shift = int(-math.log2(size))
        ks.copy_(torch.where(ks != 0xFF, (ks.int() + shift).clamp(0, 254), ks.int()).to(torch.uint8))
    check(mx, 8, 2, dim, 32, 16, [100, 40], [200, 100], seed=12, setup=setup)


@pytest.mark.parametrize("dim", [64, 128])
def test_prompt_zero_queries(mx, dim):  # noqa: F811
    def setup(cache, q, table):
        q[:50] = 0
        q[50:, :, 3:] = 0
    check(mx, 8, 2, dim, 32, 16, [100, 20], [200, 100], seed=13, setup=setup)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nq,height", [(100, 150.0), (100, 20.0), (200, 448.0)])
def test_prompt_one_token_far_above_the_rest(mx, dim, nq, height):  # noqa: F811
    """The first key's score above all others', so that the reference comes down by as much as it may afterwards, and the output so far is
    corrected."""
    def setup(cache, q, table):
        kc = cache.parts[0]
        for h in range(kc.shape[1]):
            d = q[:, h * (q.shape[1] // kc.shape[1])].float().mean(0)
            kc[table[0][0], h, 0] = (d * (height / d.abs().max())).to(torch.float8_e4m3fn).view(torch.uint8)
    check(mx, 2, 2, dim, 64, 16, [nq], [6000], seed=11, q_std=0.3, setup=setup)


@pytest.mark.parametrize("dim", [64, 128])
def test_prompt_without_keys(mx, dim):  # noqa: F811
    """Sequences of length zero and queries before the first key: zeros and -infinity."""
    check(mx, 4, 2, dim, 16, 16, [100, 50, 70], [0, 1, 30], seed=6)
    check(mx, 4, 2, dim, 16, 16, [100, 50], [0, 0], seed=7)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nq,lens", [([1], [300]), ([4, 3], [900, 50]), ([100, 30], [150, 700])])
@pytest.mark.parametrize("scale", [-0.1, 0.0, 3.0])
def test_scales_of_the_scores(mx, dim, nq, lens, scale):  # noqa: F811
    agrees(mx, nq, lens, 2, 4, dim, 32, max(lens), scale=scale)


# The error of the weights as they are documented: half a step of binary16, 2^-11 each.  The rest, relative to the sum of the weights'
# magnitudes: a score's binary32 sum, 16 2^-23 of its magnitudes (below 8 here: 2^-16); scale, reference and exponential 2^-19; the binary32
# sums over up to 2100 tokens in steps of 16, 132 2^-23 < 2^-15; the last product 2^-23: below 2^-14 together, 2^-13 with what
# the prompt kernel's pair of E4M3 numbers leaves of q's smallest elements (2^-18 of the row's largest, some of 128: below 2^-16).
# q_std = 0.3 keeps scores and value scales within 13 binades, so that no weight is below binary16's normal range.
SHARP = 2.0 ** -11 + 2.0 ** -13


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nq,lens", [([1], [2100]), ([1, 1, 1], [17, 500, 2000]), ([4, 8], [1000, 300]), ([65], [700]), ([150, 300], [2000, 333])])
@pytest.mark.parametrize("options", [{}, {"window": 200}, {"causal": False}])
def test_weights_are_as_sharp_as_stated(mx, dim, nq, lens, options):  # noqa: F811
    agrees(mx, nq, lens, 2, 2, dim, 64, max(lens), q_std=0.3, weight=SHARP, **options)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("nq,length,window", [(1, 2000, 0), (4, 2000, 0), (1, 700, 300), (100, 2000, 0), (100, 700, 0), (200, 900, 250), (4, 20000, 0)])
def test_each_token_counts_once(mx, dim, page, nq, length, window):  # noqa: F811
    """Equal scores; one token's value in each dimension, at the ends of runs of 16 tokens (tiles, pages, chunks): its share is one
    over the number of keys seen."""
    heads, group = 2, 1
    table, pool = make_table([length], -(-length // page), page, 1)
    cache = Cache(pool, heads, page, dim, 16, code=0, scale=121)
    lo = max(0, length - nq - window + 1) if window else 0
    ends = [t for t in range(lo, length) if t % 16 in (0, 15) or t >= length - 2]
    at = [ends[round(i * (len(ends) - 1) / (dim - 1))] for i in range(dim)]
    for d, t in enumerate(at):
        cache.parts[2][table[0][t // page], :, t % page, d] = 0x70   # 128 * 2^-6
    q = torch.zeros(nq, heads * group, dim, dtype=torch.bfloat16, device="cuda")
    out, lse = attend(mx, q, [0, nq], [length], table, cache, nq, length, 1.0, window=window)
    place = length - nq + torch.arange(nq, device="cuda")[:, None]
    key = torch.tensor(at, device="cuda")[None]
    seen = (key <= place) & (key > place - window if window else key >= 0)
    count = torch.minimum(place + 1, torch.full_like(place, window)) if window else place + 1
    want = torch.where(seen, 2.0 / count.double(), 0.0)[:, None].expand(nq, heads, dim)
    assert bool(((out.double() - want).abs() <= (2.0 ** -8 + SHARP) * want).all())
    assert bool(((lse.double() - count.double().log()).abs() <= 2.0 ** -19 + 5 * 2.0 ** -23 * count.double().log()).all())


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("seqs,nq", [(1, 1), (40, 1), (40, 4), (1, 100), (2, 150)])
@pytest.mark.parametrize("regions", [(227, 121), (121, 227), (121, 0, 121, 227, 121), (0, 121, 0, 121), (60, 121, 187), (1, 247, 1), (121, 100, 121, 140)])
@pytest.mark.parametrize("width", [32, 144])
def test_value_scales_by_region(mx, dim, seqs, nq, regions, width):  # noqa: F811
    """Regions of tokens whose value scales lie far from their neighbours', and back: each token counts in the softmax's sum.  247 is the
    largest byte that finite values have; with 254, codes of about 60 are values of 2^133, whose mean no bf16 holds."""
    length = 900

    def setup(cache, q, table):
        vc, vs = cache.parts[2:]
        vc.copy_(torch.where((vc != 0x7F) & ((vc & 0x7F) < 0x38), (vc & 0x80) | 0x38, vc))   # no code below 1: see value_scales
        pages = torch.tensor(table, device="cuda")[:, :-(-length // 32)]
        for b in range(-(-length // 16)):
            vs[pages[:, b // 2], :, b % 2] = regions[16 * b // width % len(regions)]
    check(mx, 16 if seqs > 2 else 4, 8 if seqs > 2 else 2, dim, 32, 16, [nq] * seqs, [length] * seqs, seed=dim + nq, setup=setup)
