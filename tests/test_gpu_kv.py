"""mxkv_append and mxkv_attention on the GPU: the append bit for bit against its contract, the attention against 64 bits.

Tolerances of the attention.  out: a weight is off by at most 2^-8 of itself (in binary16 it is 2^-11), or 2^-15 of the tile's
largest where it is so far below that it rounds to nothing, binary32 sums; then one rounding to bf16:
2^-8 |out| + (2^-8 + 2^-10) sum of softmax |v|, where 2^-10 covers the 32 small weights of a tile (32 * 2^-15).
lse: a score is the binary32 sum of at most 128 exact products, added in a few steps of the tensor cores: 16 roundings of 2^-23 of
the sum of magnitudes (`big`) and four of the score itself; exp2 and log2 add 2^-21 and the sum over tiles 2^-20 of relative
error each, i.e. the same in absolute terms in the logarithm; the multiplication by ln 2 another 2^-23 of lse."""
import math

import pytest
import torch

from tests import qkv_ref as ref

pytestmark = pytest.mark.gpu
NAN_CODE = 0x7F


@pytest.fixture(scope="module")
def mx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2603_13180_b200 import binding
    return binding


def cumulative(n):
    cu = [0]
    for x in n:
        cu.append(cu[-1] + x)
    return cu


def dev(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def make_table(lens, width, page, seed, junk=-1):
    """A shuffled page table (list) and the pool's size; entries behind a sequence's last page are junk."""
    need = [-(-x // page) for x in lens]
    pool = sum(need) + 3
    order = torch.randperm(pool, generator=torch.Generator().manual_seed(seed)).tolist()
    table, at = [], 0
    for n in need:
        table.append(order[at:at + n] + [junk] * (width - n))
        at += n
    return table, pool


class Cache:
    """A cache with guard bytes around each of its four tensors, filled with `code` and `scale`."""

    def __init__(self, pool, heads, page, dim, block, code=NAN_CODE, scale=0xFF):
        self.full, self.parts = [], []
        for shape, fill in (((pool, heads, page, dim), code), ((pool, heads, page // block), scale)) * 2:
            n = math.prod(shape)
            full = torch.full((256 + n + 256,), 0xA5, dtype=torch.uint8, device="cuda")
            full[256:256 + n] = fill
            self.full.append((full, n))
            self.parts.append(full[256:256 + n].view(shape))

    def guards_intact(self):
        return all(bool((f[:256] == 0xA5).all()) and bool((f[256 + n:] == 0xA5).all()) for f, n in self.full)

    def cpu(self):
        return [p.cpu().clone() for p in self.parts]


APPENDS = [  # heads, dim, page, block, rotated, pairs, lengths before, new tokens
    (1, 64, 16, 16, 0, False, [0], [1]),
    (2, 128, 64, 16, 128, False, [0, 5, 15, 16, 17, 63, 64], [1, 1, 1, 1, 1, 1, 1]),
    (8, 128, 64, 16, 128, False, [0, 100, 31], [200, 3, 129]),
    (3, 64, 32, 32, 32, True, [0, 31, 32, 40, 7], [1, 2, 33, 0, 90]),
    (4, 96, 128, 64, 96, False, [1, 64, 127, 0], [70, 1, 130, 300]),
    (5, 16, 16, 16, 16, True, [3, 0], [40, 17]),
    (1, 256, 256, 32, 64, False, [250, 0, 255], [20, 513, 1]),
    (9, 32, 32, 16, 16, False, [0] * 40, list(range(1, 41))),
]


@pytest.mark.parametrize("heads,dim,page,block,rot,pairs,old,new", APPENDS)
def test_append_is_bit_exact(mx, heads, dim, page, block, rot, pairs, old, new):
    """Earlier tokens in one call, new ones in a second: codes and scales equal the contract's, all else is untouched."""
    g = torch.Generator().manual_seed(dim + page)
    lens = [a + b for a, b in zip(old, new)]
    width = max(-(-x // page) for x in lens) + 1
    table, pool = make_table(lens, width, page, seed=dim)
    cache = Cache(pool, heads, page, dim, block)
    want = cache.cpu()
    rope = ref.rope_table(max(lens) + 1, rot) if rot else None
    for counts, ends in ((old, old), (new, lens)):
        cu = cumulative(counts)
        n = cu[-1]
        if n == 0:
            continue
        # rows of very different size, so that later tokens raise their block's scale; zeros among them; rows behind the last sequence
        x = torch.randn(n + 5, 2 * heads * dim, generator=g) * torch.exp(2 * torch.randn(n + 5, 1, generator=g))
        x[torch.rand(n + 5, generator=g) < 0.1] = 0
        x = x.to(torch.bfloat16)
        xd = x.cuda()
        k, v = xd[:, :heads * dim].view(-1, heads, dim), xd[:, heads * dim:].view(-1, heads, dim)
        mx.mxkv_append(k, v, dev(cu), dev(ends), dev(table), *cache.parts, cos_sin=None if rope is None else rope.cuda(), interleaved=pairs)
        kx, vx = x[:n, :heads * dim].reshape(n, heads, dim).float(), x[:n, heads * dim:].reshape(n, heads, dim).float()
        pos = torch.cat([torch.arange(e - c, e) for c, e in zip(counts, ends)])
        kx = ref.rotate(kx, rope, pos, pairs)
        ref.append(kx, want[0], want[1], cu, ends, table, page, block)
        ref.append(vx, want[2], want[3], cu, ends, table, page, block)
        for name, got, w in zip(("k codes", "k scales", "v codes", "v scales"), cache.parts, want):
            assert torch.equal(got.cpu(), w), name
        before = cache.cpu()
        mx.mxkv_append(k, v, dev(cu), dev(ends), dev(table), *cache.parts, cos_sin=None if rope is None else rope.cuda(), interleaved=pairs)
        assert all(torch.equal(a, b) for a, b in zip(before, cache.cpu())), "the same append again changed something"
    assert cache.guards_intact()


def test_append_token_by_token_keeps_the_largest_scale(mx):
    """One token a call, growing by powers of two: the block's scale follows, earlier codes are exact while they stay normal."""
    heads, dim, page, block = 2, 64, 32, 16
    cache = Cache(1, heads, page, dim, block, code=0, scale=0)
    want = cache.cpu()
    base = torch.randn(1, heads, dim, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16)
    for t in range(20):
        x = base * 2.0 ** (t - 10)
        mx.mxkv_append(x.cuda(), x.cuda(), dev([0, 1]), dev([t + 1]), dev([[0]]), *cache.parts)
        for i in (0, 2):
            ref.append(x.float(), want[i], want[i + 1], [0, 1], [t + 1], [[0]], page, block)
    assert all(torch.equal(a.cpu(), b) for a, b in zip(cache.parts, want))


def test_append_leaves_bad_places_out(mx):
    heads, dim, page, block = 2, 64, 32, 16
    cache = Cache(2, heads, page, dim, block, code=3, scale=4)
    before = cache.cpu()
    x = torch.randn(40, heads, dim, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    mx.device_bad_indices_reset()
    # a page below and one above the pool; a length shorter than the new tokens; a place behind the table's last column
    mx.mxkv_append(x[:3], x[:3], dev([0, 1, 2, 3]), dev([1, 1, 0]), dev([[-1], [2], [0]]), *cache.parts)
    mx.mxkv_append(x[:1], x[:1], dev([0, 1]), dev([33]), dev([[0]]), *cache.parts)
    assert mx.device_bad_indices() > 0
    assert all(torch.equal(a, b) for a, b in zip(before, cache.cpu()))
    # places outside the rotation's table: the keys are left out, the values (not rotated) are written
    mx.device_bad_indices_reset()
    mx.mxkv_append(x[:1], x[:1], dev([0, 1]), dev([20]), dev([[1]]), *cache.parts, cos_sin=ref.rope_table(10, 64).cuda())
    assert mx.device_bad_indices() > 0
    after = cache.cpu()
    assert torch.equal(before[0], after[0]) and torch.equal(before[1], after[1]) and not torch.equal(before[2], after[2])
    # lists that do not rise, or that end behind the rows: nothing out of bounds
    mx.mxkv_append(x[:4], x[:4], dev([0, 9, 2]), dev([9, 2]), dev([[0], [1]]), *cache.parts)
    mx.mxkv_append(x[:4], x[:4], dev([2, 2, 99]), dev([9, 97]), dev([[0, 0, 0, 0], [1, 1, 1, 1]]), *cache.parts)
    torch.cuda.synchronize()
    assert cache.guards_intact()
    mx.device_bad_indices_reset()


def fill(cache, lens, table, page, block, seed, k_spread=3, v_spread=3):
    """Random finite codes and scales at the places that tokens hold; NaN codes and scales stay everywhere else."""
    kc, ks, vc, vs = cache.parts
    g = torch.Generator(device="cuda").manual_seed(seed)
    for s, length in enumerate(lens):
        for i in range(-(-length // page)):
            pg, n = table[s][i], min(page, length - i * page)
            for c, sc, spread in ((kc, ks, k_spread), (vc, vs, v_spread)):
                h, d = c.shape[1], c.shape[3]
                c[pg, :, :n] = (60 * torch.randn(h, n, d, generator=g, device="cuda")).clamp(-256, 256).to(torch.float8_e4m3fn).view(torch.uint8)
                nb = -(-n // block)
                sc[pg, :, :nb] = torch.randint(121 - spread, 122, (h, nb), generator=g, device="cuda").to(torch.uint8)


def check(mx, q_heads, heads, dim, page, block, nq, lens, causal=True, window=0, seed=0, q_std=2.0, max_q=None, max_len=None, setup=None,
          workspace_fill=0xFF, with_lse=True):
    cu = cumulative(nq)
    n = cu[-1]
    top = max(max(lens), 1)
    max_len = top if max_len is None else max_len
    width = -(-max_len // page) + 1
    table, pool = make_table(lens, width, page, seed, junk=-7 if seed % 2 else 2 ** 30)
    cache = Cache(pool, heads, page, dim, block)
    fill(cache, lens, table, page, block, seed)
    g = torch.Generator().manual_seed(seed + 1)
    x = (q_std * torch.randn(n + 3, (q_heads + 2) * dim, generator=g)).to(torch.bfloat16).cuda()
    q = x[:, dim:(q_heads + 1) * dim].view(-1, q_heads, dim)     # strided, with rows behind the last sequence
    if setup is not None:
        setup(cache, q, table)
    buf = torch.full((n + 3, q_heads + 1, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    out = buf[:, :q_heads]
    lse = torch.full((n + 3, q_heads), 7.0, device="cuda") if with_lse else None
    max_q = max(max(nq), 1) if max_q is None else max_q
    nbytes = mx.mxkv_attention_workspace_bytes(n + 3, len(lens), max_q, max_len, q_heads, heads, dim)
    ws = torch.full((nbytes,), workspace_fill, dtype=torch.uint8, device="cuda") if nbytes else None
    scale = 1 / math.sqrt(dim)
    args = (q, dev(cu), dev(lens), dev(table), *cache.parts, out, max_q, max_len, scale)
    mx.mxkv_attention(*args, causal=causal, window=window, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    assert mx.device_timeouts() == 0
    want, want_lse, mag, big = ref.attention(q[:n], cu, lens, table, *cache.parts, scale, causal, window)
    got = out[:n].double()
    err, tol = (got - want).abs(), 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -10) * mag + 1e-30
    assert bool((err <= tol).all()), f"out: off by {float((err / tol.clamp(min=1e-30)).nan_to_num(1e9).max()):.3g} tolerances"
    if with_lse:
        live = want_lse > -math.inf
        assert bool((lse[:n][~live] == -math.inf).all()) and not bool(got[~live].any())
        e = (lse[:n].double() - want_lse)[live].abs()
        t = (16 * 2.0 ** -23 * big + 2.0 ** -19 + 5 * 2.0 ** -23 * want_lse.abs())[live]
        assert bool((e <= t).all()), f"lse: off by {float((e / t).max()):.3g} tolerances"
        assert bool((lse[n:] == 7).all())
    assert bool((buf[n:] == 7).all()) and bool((buf[:, q_heads] == 7).all()), "rows or heads that are not the call's were written"
    assert cache.guards_intact()
    first = out.clone()
    mx.mxkv_attention(*args, causal=causal, window=window, lse=lse, workspace=ws)
    assert torch.equal(first, out), "not repeatable"
    return cache, q, table


DECODE = [  # query heads, key heads, dim, page, block, new queries, lengths
    (1, 1, 64, 16, 16, [1], [1]), (1, 1, 128, 16, 16, [1], [1]),
    (32, 8, 128, 64, 16, [1], [1000]), (32, 8, 128, 64, 16, [1] * 5, [1, 63, 64, 65, 700]),
    (8, 8, 128, 32, 32, [1, 1, 1], [31, 32, 33]), (8, 1, 64, 128, 64, [1, 1], [127, 2049]),
    (16, 1, 128, 64, 32, [1, 1], [300, 17]), (14, 2, 64, 16, 16, [1, 1, 1], [15, 16, 500]),
    (3, 1, 128, 256, 16, [1, 0, 1], [4000, 50, 257]), (64, 2, 64, 64, 64, [1], [129]),
    (4, 4, 128, 16, 16, [1] * 70, list(range(1, 71))),
    (6, 2, 64, 32, 16, [2, 3, 4, 1], [2, 70, 1000, 5]), (32, 4, 128, 64, 16, [4, 4, 4], [4, 100, 3000]),
    (8, 2, 128, 16, 16, [8, 5, 7], [8, 9, 129]), (16, 2, 64, 128, 32, [3, 6], [1, 2000]),
]


@pytest.mark.parametrize("qh,h,dim,page,block,nq,lens", DECODE)
@pytest.mark.parametrize("window", [0, 1, 50, 600])
def test_attention_few_rows(mx, qh, h, dim, page, block, nq, lens, window):
    check(mx, qh, h, dim, page, block, nq, lens, window=window, seed=dim + page + window)


PROMPT = [
    (4, 1, 128, 64, 16, [100], [100]), (8, 2, 64, 32, 32, [129, 17, 64], [129, 400, 64]), (4, 4, 128, 16, 16, [33], [2000]),
    (6, 1, 128, 128, 64, [257, 1, 300], [300, 77, 300]), (2, 2, 64, 64, 16, [1000], [1500]), (8, 1, 128, 64, 16, [128, 256], [128, 1031]),
    (5, 1, 64, 16, 16, [200, 40], [150, 40]),
]


@pytest.mark.parametrize("qh,h,dim,page,block,nq,lens", PROMPT)
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 70), (False, 200)])
def test_attention_prompts(mx, qh, h, dim, page, block, nq, lens, causal, window):
    check(mx, qh, h, dim, page, block, nq, lens, causal=causal, window=window, seed=dim + page + 1)


@pytest.mark.parametrize("qh,h,dim,page,block,nq,lens", [
    (64, 64, 64, 64, 16, [650], [700]), (40, 40, 128, 64, 16, [800], [1000]), (80, 40, 64, 32, 16, [400], [300]),
])
def test_attention_prompts_in_halves(mx, qh, h, dim, page, block, nq, lens):
    """More blocks of 256 rows than SMs: those of the last round are halved.  Odd ends, and queries before the first key."""
    check(mx, qh, h, dim, page, block, nq, lens, seed=dim + qh)


@pytest.mark.parametrize("qh,h,dim,nq,lens", [
    (1, 1, 128, [1], [20000]), (8, 2, 64, [4], [9000]), (4, 1, 128, [16], [5000]),              # more than eight chunks
    (2, 1, 64, [1, 1], [1300, 3]), (32, 4, 64, [4, 3, 0], [1500, 4, 9]), (8, 4, 128, [8], [1100]),  # a few
])
@pytest.mark.parametrize("window", [0, 700])
def test_attention_in_chunks(mx, qh, h, dim, nq, lens, window):
    check(mx, qh, h, dim, 64, 16, nq, lens, window=window, seed=dim + window + qh)


@pytest.mark.parametrize("nq", [1, 150])
def test_cache_past_32_bits(mx, nq):
    """Pages whose codes lie more than 2^32 bytes into the pool: the bits that a small pool gives."""
    heads, dim, page, block, length = 8, 128, 64, 16, 200
    pages = 2 ** 32 // (heads * dim * page) + 9
    g = torch.Generator().manual_seed(nq)
    x = torch.randn(length, 4 * heads, dim, generator=g).to(torch.bfloat16).cuda()
    results = []
    for pool, table in ((4, [[2, 0, 3, 1]]), (pages, [[pages - 2, pages - 4, pages - 1, pages - 3]])):
        cache = mx.alloc_kv_cache(pool, heads, page, dim, block)
        mx.mxkv_append(x[:, :heads], x[:, heads:2 * heads], dev([0, length]), dev([length]), dev(table), *cache)
        q = x[length - nq:, 2 * heads:]
        out = torch.empty_like(q)
        nbytes = mx.mxkv_attention_workspace_bytes(nq, 1, nq, length, 2 * heads, heads, dim)
        ws = torch.empty(max(16, nbytes), dtype=torch.uint8, device="cuda")
        mx.mxkv_attention(q, dev([0, nq]), dev([length]), dev(table), *cache, out, nq, length, dim ** -0.5, workspace=ws)
        results.append([c[torch.tensor(table[0], device="cuda")] for c in cache] + [out])
        assert all(not bool(c[1 if pool > 4 else 4:pool - 4].any()) for c in cache)
        del cache
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert bool(results[0][-1].isfinite().all()) and bool(results[0][0].any())


def test_calls_at_the_same_time(mx):
    """Two streams with a workspace each, and graphs of both that run side by side: every result has the bits of a call alone."""
    heads, dim, page, block = 4, 128, 64, 16
    jobs = []
    for seed, (nq, lens) in enumerate((([1, 1], [6000, 900]), ([130, 7], [700, 3000]), ([2], [12000]))):
        table, pool = make_table(lens, 200, page, seed)
        cache = Cache(pool, heads, page, dim, block)
        fill(cache, lens, table, page, block, seed)
        q = torch.randn(sum(nq), 8, dim, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda()
        nbytes = mx.mxkv_attention_workspace_bytes(sum(nq), len(nq), max(nq), max(lens), 8, heads, dim)
        ws = torch.empty(max(16, nbytes), dtype=torch.uint8, device="cuda")
        fixed = (dev(cumulative(nq)), dev(lens), dev(table), *cache.parts)
        alone, out = torch.empty_like(q), torch.zeros_like(q)
        call = lambda to, q=q, fixed=fixed, nq=nq, lens=lens, ws=ws: mx.mxkv_attention(  # noqa: E731
            q, *fixed, to, max(nq), max(lens), dim ** -0.5, workspace=ws)
        call(alone)
        jobs.append((call, alone, out, torch.cuda.Stream(), cache))
    torch.cuda.synchronize()
    for _ in range(20):
        for call, _, out, stream, _ in jobs:
            with torch.cuda.stream(stream):
                call(out)
    torch.cuda.synchronize()
    assert all(torch.equal(alone, out) for _, alone, out, _, _ in jobs)
    graphs = []
    for call, _, out, stream, _ in jobs:
        out.zero_()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            call(out)
    torch.cuda.synchronize()
    for _ in range(20):
        for graph, (_, _, _, stream, _) in zip(graphs, jobs):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(alone, out) for _, alone, out, _, _ in jobs)
    assert mx.device_timeouts() == 0


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("qh,nq", [(8, 8), (13, 5), (1, 64), (1, 65)])
@pytest.mark.parametrize("longest", [150, 300])
def test_attention_around_64_rows(mx, qh, nq, dim, longest):
    """64 and 65 query rows for a key head: the last of the one kernel, the first of the other; a few chunks and more."""
    check(mx, qh, 1, dim, 64, 16, [nq, nq - 1, 1], [longest, nq, 77], seed=qh + nq)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nq,length", [(1, 90), (1, 1500), (4, 30000), (40, 300), (90, 200), (200, 3000)])
def test_attention_infinities_and_nan(mx, dim, nq, length):
    """A row with an infinity or NaN among its queries, and rows that see a NaN key, are NaN; the others keep their bits."""
    table, pool = make_table([length], -(-length // 32), 32, 7)
    cache = Cache(pool, 2, 32, dim, 16)
    fill(cache, [length], table, 32, 16, 7)
    g = torch.Generator().manual_seed(nq)
    q = torch.randn(nq, 4, dim, generator=g).to(torch.bfloat16).cuda()
    nbytes = mx.mxkv_attention_workspace_bytes(nq, 1, nq, length, 4, 2, dim)
    ws = torch.empty(max(16, nbytes), dtype=torch.uint8, device="cuda")

    def run():
        out, lse = torch.empty_like(q), torch.empty(nq, 4, device="cuda")
        mx.mxkv_attention(q, dev([0, nq]), dev([length]), dev(table), *cache.parts, out, nq, length, dim ** -0.5, lse=lse, workspace=ws)
        return out, lse

    clean, clean_lse = run()
    assert bool(clean.isfinite().all())
    for value in (float("inf"), float("-inf"), float("nan")):
        keep = q.clone()
        q[nq // 2, 1, 5] = value
        out, lse = run()
        assert bool(out[nq // 2, 1].isnan().all()) and bool(lse[nq // 2, 1].isnan())
        out[nq // 2, 1], lse[nq // 2, 1] = clean[nq // 2, 1], clean_lse[nq // 2, 1]
        assert torch.equal(out, clean) and torch.equal(lse, clean_lse)
        q.copy_(keep)
    # a NaN key of one head, among the new tokens' places: rows before it do not see it
    for back in sorted({0, min(nq - 1, 1), nq // 2}):
        at = length - 1 - back
        place = (table[0][at // 32], 1, at % 32, 3)
        code = int(cache.parts[0][place])
        cache.parts[0][place] = NAN_CODE
        out, lse = run()
        sees = nq - 1 - back
        assert bool(out[sees:, 2:].isnan().all()) and bool(lse[sees:, 2:].isnan().all())
        assert torch.equal(out[:sees], clean[:sees]) and torch.equal(out[:, :2], clean[:, :2])
        cache.parts[0][place] = code


def test_attention_over_its_queries(mx):
    """out may be q itself: every row is read before it is written, whatever the chunks."""
    for nq, length, window in (([1], 2000, 0), ([4], 20000, 0), ([70], 500, 0), ([300], 900, 100)):
        table, pool = make_table([length], -(-length // 64), 64, 5)
        cache = Cache(pool, 2, 64, 128, 16)
        fill(cache, [length], table, 64, 16, 5)
        q = torch.randn(nq[0], 8, 128, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
        nbytes = mx.mxkv_attention_workspace_bytes(nq[0], 1, nq[0], length, 8, 2, 128)
        ws = torch.empty(max(16, nbytes), dtype=torch.uint8, device="cuda")
        fixed = (dev([0] + nq), dev([length]), dev(table), *cache.parts)
        out = torch.empty_like(q)
        mx.mxkv_attention(q, *fixed, out, nq[0], length, 0.1, window=window, workspace=ws)
        mx.mxkv_attention(q, *fixed, q, nq[0], length, 0.1, window=window, workspace=ws)
        assert torch.equal(q, out)


def test_attention_bounds_larger_than_the_lengths(mx):
    check(mx, 8, 2, 128, 64, 16, [1, 1], [5, 90], max_q=4, max_len=20000, seed=4)
    check(mx, 8, 2, 64, 64, 16, [3, 40], [500, 90], max_q=64, max_len=5000, seed=5, with_lse=False)


def test_attention_without_keys(mx):
    """Sequences of length zero and queries before the first key: zeros and -infinity."""
    check(mx, 4, 2, 64, 16, 16, [1, 2, 5], [0, 1, 3], seed=6)
    check(mx, 4, 2, 128, 16, 16, [1], [0], seed=7)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nq", [1, 60])
def test_attention_scales_far_apart(mx, dim, nq):
    """Scales over forty binades, blocks of zeros with scale 0, a first token that takes most of the weight and holds a zero value."""
    def setup(cache, q, table):
        kc, ks, vc, vs = cache.parts
        g = torch.Generator(device="cuda").manual_seed(9)
        for row in table:
            for pg in row:
                if 0 <= pg < vc.shape[0]:
                    vs[pg] = torch.randint(100, 141, vs[pg].shape, generator=g, device="cuda").to(torch.uint8)
        vc[table[0][0], :, :16] = 0
        vs[table[0][0], :, 0] = 0
        kc[table[0][1], :, 16:32] = 0
        ks[table[0][1], :, 1] = 0
    check(mx, 8, 2, dim, 32, 16, [nq, nq], [900, 333], seed=10, setup=setup)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nq", [1, 40])
def test_attention_one_token_far_above_the_rest(mx, dim, nq):
    """A key with a score some 15 above the others', so that most of the weight sits in thousands of tiny ones."""
    def setup(cache, q, table):
        kc, ks, vc, vs = cache.parts
        for h in range(kc.shape[1]):
            d = q[:, h * (q.shape[1] // kc.shape[1])].float().mean(0)
            kc[table[0][0], h, 0] = (d * (150 / d.abs().max())).to(torch.float8_e4m3fn).view(torch.uint8)
    check(mx, 2, 2, dim, 64, 16, [nq], [6000], seed=11, q_std=0.3, setup=setup)


@pytest.mark.parametrize("size", [2.0 ** -100, 2.0 ** -20, 2.0 ** 100])
def test_attention_query_sizes(mx, size):
    """Queries far from one, against key scales as far the other way."""
    def setup(cache, q, table):
        q.mul_(size)
        ks = cache.parts[1]
        shift = int(-math.log2(size))
        cache.parts[1].copy_(torch.where(ks != 0xFF, (ks.int() + shift).clamp(0, 254), ks.int()).to(torch.uint8))
    check(mx, 4, 2, 64, 32, 16, [1, 20], [200, 100], seed=12, setup=setup)


def test_attention_zero_queries(mx):
    def setup(cache, q, table):
        q[:1] = 0
        q[1:, :, 3:] = 0
    check(mx, 4, 2, 128, 32, 16, [1, 2], [200, 100], seed=13, setup=setup)


def test_attention_leaves_bad_pages_out(mx):
    """A page out of range among the visible ones: the result is that of the other keys; the pool is not left."""
    heads, dim, page, block, length = 2, 128, 32, 16, 150
    for nq in (1, 70):
        table, pool = make_table([length], 6, page, 3)
        cache = Cache(pool, heads, page, dim, block)
        fill(cache, [length], table, page, block, 3)
        q = torch.randn(nq, 4, dim, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
        broken = [list(table[0])]
        broken[0][1], broken[0][3] = -1, pool
        out = torch.empty_like(q)
        nbytes = mx.mxkv_attention_workspace_bytes(nq, 1, nq, length, 4, heads, dim)
        ws = torch.empty(max(16, nbytes), dtype=torch.uint8, device="cuda")
        mx.device_bad_indices_reset()
        mx.mxkv_attention(q, dev([0, nq]), dev([length]), dev(broken), *cache.parts, out, nq, length, 0.1, causal=False, workspace=ws)
        assert mx.device_bad_indices() > 0
        mx.device_bad_indices_reset()
        keep = torch.tensor([t for t in range(length) if t // page not in (1, 3)], device="cuda")
        pages = torch.tensor(table[0][:5], device="cuda")
        for j in range(4):
            k, v = (ref.dequantise(c, s, pages, block, j // 2, length)[keep] for c, s in (cache.parts[:2], cache.parts[2:]))
            p = torch.softmax(q[:, j].double() @ k.T * 0.1, -1)
            tol = 2.0 ** -8 * (p @ v).abs() + (2.0 ** -8 + 2.0 ** -10) * (p @ v.abs())
            assert bool(((out[:, j].double() - p @ v).abs() <= tol).all())


def test_norm_append_attend_as_a_model_runs_them(mx):
    """A prompt, then single tokens: norm and rotation of the projections, append, attention; against all of it in 64 bits on the
    cache's own codes, and on another stream and in a captured graph with the same bits."""
    hq, hk, dim, page, block, S = 8, 2, 128, 64, 16, 3
    g = torch.Generator().manual_seed(21)
    prompt, steps = [70, 5, 130], 4
    final = [p + steps for p in prompt]
    table, pool = make_table(final, 4, page, 2)
    rope = ref.rope_table(400, dim)
    gains = [(1 + 0.1 * torch.randn(dim, generator=g)).to(torch.bfloat16).cuda() for _ in range(2)]
    inputs = [torch.randn(sum(prompt), (hq + 2 * hk) * dim, generator=g).to(torch.bfloat16).cuda()]
    inputs += [torch.randn(S, (hq + 2 * hk) * dim, generator=g).to(torch.bfloat16).cuda() for _ in range(steps)]
    rope_d, table_d = rope.cuda(), dev(table)

    def step(cache, x, cu, lens, pos, bufs, max_q):
        q, k = x[:, :hq * dim].view(-1, hq, dim), x[:, hq * dim:(hq + hk) * dim].view(-1, hk, dim)
        v = x[:, (hq + hk) * dim:].view(-1, hk, dim)
        qn, kn, out, ws = bufs
        mx.rmsnorm_rope_fwd(q, k, gains[0], gains[1], rope_d, pos, qn, kn, eps=1e-6)
        mx.mxkv_append(kn, v, cu, lens, table_d, *cache.parts)
        mx.mxkv_attention(qn, cu, lens, table_d, *cache.parts, out, max_q, 4 * page, dim ** -0.5, workspace=ws)

    def buffers(n, max_q):
        e = lambda h: torch.empty(n, h, dim, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        nbytes = mx.mxkv_attention_workspace_bytes(n, S, max_q, 4 * page, hq, hk, dim)
        return e(hq), e(hk), e(hq), torch.empty(max(16, nbytes), dtype=torch.uint8, device="cuda")

    plans = []
    for i, x in enumerate(inputs):
        counts = prompt if i == 0 else [1] * S
        lens = [p + i for p in prompt]
        pos = torch.cat([torch.arange(e - c, e) for c, e in zip(counts, lens)]).to(torch.int32).cuda()
        plans.append((x, dev(cumulative(counts)), dev(lens), pos, max(counts), cumulative(counts), lens))
    results = []
    for mode in ("eager", "stream", "graph"):
        cache = Cache(pool, hk, page, dim, block)
        outs = []
        for x, cu, lens, pos, max_q, cu_l, lens_l in plans:
            bufs = buffers(x.shape[0], max_q)
            if mode == "stream":
                side = torch.cuda.Stream()
                side.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(side):
                    step(cache, x, cu, lens, pos, bufs, max_q)
                torch.cuda.current_stream().wait_stream(side)
            elif mode == "graph":
                graph = torch.cuda.CUDAGraph()
                torch.cuda.synchronize()
                with torch.cuda.graph(graph):
                    step(cache, x, cu, lens, pos, bufs, max_q)
                graph.replay()
                graph.replay()
            else:
                step(cache, x, cu, lens, pos, bufs, max_q)
                qn = bufs[0]
                want, _, mag, _ = ref.attention(qn, cu_l, lens_l, table, *cache.parts, dim ** -0.5)
                u = ref.norm_fwd(x[:, :hq * dim].view(-1, hq, dim), gains[0], 1e-6)
                near = ref.rotate(u, rope_d.double(), pos, False)
                assert bool(((qn.double() - near).abs() <= 2.0 ** -8 * near.abs() + 2.0 ** -19 * u.abs().amax(-1, keepdim=True)).all())
                assert bool(((bufs[2].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -10) * mag).all())
            torch.cuda.synchronize()
            outs.append(bufs[2].clone())
        assert cache.guards_intact()
        results.append((outs, cache.cpu()))
    for outs, parts in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs, results[0][0]))
        assert all(torch.equal(a, b) for a, b in zip(parts, results[0][1]))
    assert mx.device_bad_indices() == 0 and mx.device_timeouts() == 0
