"""Attention over the 8-bit paged cache with more masks, and keeping that cache short: measured cases.

The cache is that of ``mxkv_append`` and ``mxkv_attention``: E4M3 codes in pages, one E8M0 scale for each block of tokens and head.

* ``sinks``   - attention with a sliding window beside a sequence's first tokens, which stay visible;
* ``tree``    - attention of a tree of drafted tokens: each sees what is in front of the tree and its own ancestors;
* ``weights`` - the softmax weight that each key has been given by all queries of a call, added up for each key head;
* ``evict``   - the tokens with the largest such sums are chosen for each key head, beside the first and the latest ones, and moved
  together (codes, scales, sums).

``run`` computes the operators in elementary torch operations where ``own`` is false and calls the library where it is true.
"""
import math

import torch

own = False

binding = None    # the library, imported by the first call that needs it

DEV = "cuda"
EMAX = 8          # log2 of the largest power of two of E4M3


def _binding():
    global binding
    if binding is None:
        from paper_2603_13180_b200 import binding as b
        binding = b
    return binding


# ---- cases ---------------------------------------------------------------------------------------------------------

def _sinks(seqs, q_max, len_max, q_heads, kv_heads, dim, page, block, window, sinks):
    return {"op": "sinks", "seqs": seqs, "q_max": q_max, "len_max": len_max, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "page": page, "block": block, "window": window, "sinks": sinks}


def _tree(seqs, q_max, len_max, q_heads, kv_heads, dim, page, block):
    return {"op": "tree", "seqs": seqs, "q_max": q_max, "len_max": len_max, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "page": page, "block": block}


def _weights(seqs, q_max, len_max, q_heads, kv_heads, dim, page, block, add):
    return {"op": "weights", "seqs": seqs, "q_max": q_max, "len_max": len_max, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "page": page, "block": block, "add": add}


def _evict(seqs, len_max, keep, sinks, recent, kv_heads, dim, page, block):
    return {"op": "evict", "seqs": seqs, "len_max": len_max, "keep": keep, "sinks": sinks, "recent": recent, "kv_heads": kv_heads,
            "dim": dim, "page": page, "block": block}


def listed():
    return [
        # a single user of a streaming model: one token, a short window, a few first tokens: latency
        dict(_sinks(1, 1, 1000, 32, 8, 128, 64, 16, 512, 4), name="sinks one short"),
        # a serving batch far behind its window: 32 query and 8 key heads of 128 (hidden size 4096)
        dict(_sinks(64, 1, 8192, 32, 8, 128, 64, 16, 2048, 4), name="sinks batch 64"),
        # a prompt's second half in a model that was trained with a window and first tokens
        dict(_sinks(1, 4096, 8192, 32, 8, 128, 64, 16, 1024, 64), name="sinks prompt"),
        # a single user with a small tree of drafted tokens
        dict(_tree(1, 12, 1500, 32, 8, 128, 64, 16), name="tree one"),
        # trees of different sizes in heads of 64, small pages
        dict(_tree(16, 13, 4100, 32, 4, 64, 16, 16), name="tree batch odd"),
        # wide trees for a few users with long histories
        dict(_tree(8, 64, 8192, 32, 8, 128, 64, 16), name="tree wide"),
        # after a decode step: the weights of one token's attention are added to those of the steps before
        dict(_weights(64, 1, 8192, 32, 8, 128, 64, 16, True), name="weights batch 64"),
        # the weights that a prompt gives its keys
        dict(_weights(1, 4096, 8192, 32, 8, 128, 64, 16, False), name="weights prompt"),
        # several short prompts together in heads of 64
        dict(_weights(8, 1000, 1500, 32, 4, 64, 32, 32, False), name="weights prompts ragged"),
        # a few short sequences brought back to their budget: latency
        dict(_evict(4, 700, 512, 4, 64, 4, 64, 16, 16), name="evict few short"),
        # a serving batch brought back to its budget
        dict(_evict(32, 8192, 2048, 4, 256, 8, 128, 64, 16), name="evict batch 32"),
        # a quarter of one very long history
        dict(_evict(1, 131072, 32768, 16, 1024, 8, 128, 64, 16), name="evict one long"),
    ]


def _between(rng, lo, hi):
    """A whole number from lo to hi, spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["sinks", "tree", "weights", "evict"])
    dim = rng.choice([64, 128])
    page = rng.choice([16, 32, 64, 128])
    block = rng.choice([b for b in (16, 32, 64) if b <= page])
    kv = rng.choice([1, 2, 4, 8])
    if op == "evict":
        seqs = _between(rng, 1, 32)
        length = _between(rng, 200, max(200, min(131072, 32 * 8192 * 8 * 128 // (seqs * kv * dim))))
        keep = max(32, int(length * rng.uniform(0.1, 0.9)))
        sinks = rng.choice([0, 1, 4, 16])
        return _evict(seqs, length, keep, sinks, rng.randint(0, keep - sinks), kv, dim, page, block)
    group = rng.choice([1, 2, 3, 4, 6, 8, 16])
    heads = kv * group
    if op == "tree":
        seqs = _between(rng, 1, 32)
        q = _between(rng, 2, 128)
        most = min(64 * 8192 * 8 * 128 // (seqs * kv * dim), 8 * 64 * 8192 * 32 * 128 // (seqs * q * heads * dim), 32768)
        return _tree(seqs, q, q + _between(rng, 1, max(2, most)), heads, kv, dim, page, block)
    form = rng.choice(["one", "few", "prompt"])
    if form == "prompt":
        seqs = _between(rng, 1, 8)
        room = 4096 * 8192 * 32 * 128 // (heads * dim * seqs)     # query tokens times length
        q = _between(rng, 16, max(16, min(4096, int(math.sqrt(room / 2)))))
        length = min(q + _between(rng, 1, 4096), max(q, room // q))
    else:
        seqs = _between(rng, 1, 64)
        q = 1 if form == "one" else rng.randint(2, 8)
        length = max(q, _between(rng, 1, max(1, min(131072, 64 * 8192 * 8 * 128 // (seqs * kv * dim)))))
    if op == "weights":
        return _weights(seqs, q, length, heads, kv, dim, page, block, rng.random() < 0.5)
    return _sinks(seqs, q, length, heads, kv, dim, page, block, _between(rng, 16, 4000), rng.choice([1, 4, 16, 70]))


# ---- inputs --------------------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 2654435761 % (1 << 62) + 29)
    return g


def _sizes(n, most, least, turn):
    """n whole numbers from least to most on the host: the first is `most`, the rest are spread over its upper three quarters.
    They go by the case alone; `turn` tells the lists of one case apart."""
    i = torch.arange(n, dtype=torch.float64)
    u = (i * 0.6180339887498949 + 0.37 * turn) % 1.0
    s = (most * (0.25 + 0.75 * u)).long().clamp_(least, most)
    s[0] = most
    return s


def _lengths(c):
    """(new tokens, length with them) of each sequence."""
    lens = _sizes(c["seqs"], c["len_max"], 1, 1)
    if c["op"] == "evict":
        return torch.zeros_like(lens), lens
    q = _sizes(c["seqs"], c["q_max"], 1, 0) if c["q_max"] > 8 else torch.full((c["seqs"],), c["q_max"])
    return torch.minimum(q, lens), lens


def _cum(n):
    return torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]).to(torch.int32)


def _tables(seed, page, *lists):
    """Page tables, one for each list of lengths, with pages of their own in one shuffled pool, -1 behind each sequence's last page;
    and the pool's size."""
    need = [(lens + page - 1) // page for lens in lists]
    total = sum(int(n.sum()) for n in need)
    pool = total + total // 16 + 1
    order = torch.randperm(pool, generator=torch.Generator().manual_seed(seed + 1)).to(torch.int32)
    tables, used = [], 0
    for n in need:
        table = torch.full((len(n), max(1, int(n.max()))), -1, dtype=torch.int32)
        table[torch.arange(table.shape[1])[None, :] < n[:, None]] = order[used:used + int(n.sum())]
        used += int(n.sum())
        tables.append(table.to(DEV))
    return tables, pool


def _cache(g, pool, heads, page, dim, block):
    """Codes and scales of a cache in use: E4M3 bytes of normal values, scales a few binades apart."""
    codes = torch.empty(pool, heads, page, dim, dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 27) // (heads * page * dim))
    for a in range(0, pool, step):
        n = min(step, pool - a)
        r = torch.randn(n, heads, page, dim, generator=g, device=DEV)
        codes[a:a + n] = (r * 56).clamp_(-256, 256).to(torch.float8_e4m3fn).view(torch.uint8)
    scales = torch.randint(119, 123, (pool, heads, page // block), generator=g, device=DEV, dtype=torch.int32).to(torch.uint8)
    return codes, scales


def _drafts(seed, counts, words):
    """int32 [tokens, words]: bit i of a drafted token's row tells whether it sees drafted token i of its sequence.  A token hangs from one
    of the few before it, or from the last token in front of the tree, and sees its ancestors and itself."""
    pick = torch.Generator().manual_seed(seed + 3)
    rows = []
    for n in counts.tolist():
        back = torch.randint(1, 6, (n,), generator=pick).tolist()
        seen = []
        for i in range(n):
            up = i - back[i]
            seen.append((seen[up] if up >= 0 else 0) | 1 << i)
        rows += seen
    cells = [[(r >> 32 * w & 0xFFFFFFFF) - (1 << 32 if r >> 32 * w & 1 << 31 else 0) for w in range(words)] for r in rows]
    return torch.tensor(cells, dtype=torch.int32).to(DEV)


def prepare(case, seed):
    c = dict(case)
    g = _gen(seed)
    h, d, page, block = c["kv_heads"], c["dim"], c["page"], c["block"]
    new, lens = _lengths(c)
    c["lens"] = lens.to(torch.int32).to(DEV)
    if c["op"] == "evict":
        # the shortened sequences get pages of their own: those in front may be shared with other sequences
        (c["page_table"], c["out_table"]), pool = _tables(seed, page, lens, lens.clamp(max=c["keep"]))
        # sums of softmax weights: a few large ones, many small ones, some of nothing
        w = torch.exp(2 * torch.randn(pool, h, page, generator=g, device=DEV))
        w[torch.rand(pool, h, page, generator=g, device=DEV) < 0.05] = 0
        c["weights"] = w
        c["kept"] = torch.empty(c["seqs"], h, c["keep"], dtype=torch.int32, device=DEV)
        c["new_lens"] = torch.empty(c["seqs"], dtype=torch.int32, device=DEV)
    else:
        (c["page_table"],), pool = _tables(seed, page, lens)
        c["n"] = int(new.sum())
        c["cu"] = _cum(new).to(DEV)
        c["q"] = (2 * torch.randn(c["n"], c["q_heads"], d, generator=g, device=DEV)).to(torch.bfloat16)
        c["scale"] = 1.0 / math.sqrt(d)
    c["k_codes"], c["k_scales"] = _cache(g, pool, h, page, d, block)
    if c["op"] == "weights":
        c["lse"] = _attend_plain(c, False)[0]
        c["weights"] = torch.zeros(pool, h, page, device=DEV)
        c["earlier"] = torch.exp(2 * torch.randn(pool, h, page, generator=g, device=DEV)) if c["add"] else None
        return c
    c["v_codes"], c["v_scales"] = _cache(g, pool, h, page, d, block)
    if c["op"] != "evict":
        c["out"] = torch.empty(c["n"], c["q_heads"], d, dtype=torch.bfloat16, device=DEV)
        c["lse"] = torch.empty(c["n"], c["q_heads"], dtype=torch.float32, device=DEV)
    if c["op"] == "tree":
        c["mask"] = _drafts(seed, new, (c["q_max"] + 31) // 32)
    return c


# ---- plain forms: elementary torch operations in binary32 ------------------------------------------------------------

def _dense(codes, scales, c):
    """[S, L, H, D] binary32 values of every sequence, whatever stands behind its length."""
    t = c["page_table"].long().clamp(min=0)
    x = codes[t].view(torch.float8_e4m3fn).float()                               # [S, P, H, page, D]
    s = torch.exp2(scales[t].float() - 127).repeat_interleave(c["block"], -1)    # [S, P, H, page]
    return (x * s[..., None]).transpose(2, 3).flatten(1, 2)[:, :c["len_max"]]


def _slots(c):
    """Sequence and number within it of each of the new tokens."""
    cu = c["cu"].long()
    row = torch.arange(c["n"], device=DEV)
    seq = torch.searchsorted(cu[1:].contiguous(), row, right=True)
    return seq, row - cu[seq]


def _scores(c, seq, slot):
    """(scores [S, H, G, m, L] with -infinity where a row sees nothing, visible [S, 1, 1, m, L])."""
    hq, h, d, s, m = c["q_heads"], c["kv_heads"], c["dim"], c["seqs"], c["q_max"]
    cu, lens = c["cu"].long(), c["lens"].long()
    front = lens - (cu[1:] - cu[:-1])                                            # tokens in front of the new ones
    q = torch.zeros(s, m, hq, d, device=DEV)
    q[seq, slot] = c["q"].float()
    j = torch.arange(c["len_max"], device=DEV)
    if c["op"] == "tree":
        bits = torch.zeros(s, m, 32 * c["mask"].shape[1], dtype=torch.bool, device=DEV)
        bits[seq, slot] = ((c["mask"][:, :, None] >> torch.arange(32, device=DEV)) & 1).flatten(1).bool()
        at = (j - front[:, None])[:, None].expand(s, m, -1)
        seen = (at < 0) | ((at < (lens - front)[:, None, None]) & bits.gather(2, at.clamp(0, bits.shape[2] - 1)))
        exists = torch.zeros(s, m, 1, dtype=torch.bool, device=DEV)
        exists[seq, slot] = True
        seen &= exists
    else:
        at = torch.full((s, m, 1), -1, dtype=torch.int64, device=DEV)
        at[seq, slot] = (front[seq] + slot)[:, None]
        seen = j <= at
        if c["op"] == "sinks":
            seen &= (j > at - c["window"]) | (j < c["sinks"])
    k = _dense(c["k_codes"], c["k_scales"], c)
    q = q.view(s, m, h, hq // h, d).permute(0, 2, 3, 1, 4).flatten(2, 3)          # [S, H, G*m, D]
    score = (torch.matmul(q, k.permute(0, 2, 3, 1)) * c["scale"]).view(s, h, hq // h, m, -1)
    seen = seen[:, None, None]
    return score.masked_fill_(~seen, -math.inf), seen


def _attend_plain(c, values):
    seq, slot = _slots(c)
    score, _ = _scores(c, seq, slot)
    top = score.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(score.sub_(top))
    total = p.sum(-1, keepdim=True)
    lse = (top + torch.log(total))[..., 0].permute(0, 3, 1, 2).flatten(2, 3)[seq, slot]
    if not values:
        return [lse]
    v = _dense(c["v_codes"], c["v_scales"], c)
    o = torch.matmul(p.flatten(2, 3), v.transpose(1, 2)).view(*p.shape[:4], -1)
    o = o / torch.where(total > 0, total, torch.ones_like(total))
    return [o.permute(0, 3, 1, 2, 4).flatten(2, 3)[seq, slot].to(torch.bfloat16), lse]


def _cells(c, table, at):
    """(page, head, place within the page) of the tokens `at` [S, H, n] of each sequence and head."""
    page = table.long().gather(1, (at // c["page"]).flatten(1)).view(at.shape)
    return page, torch.arange(at.shape[1], device=DEV)[:, None].expand_as(at), at % c["page"]


def _weights_plain(c):
    seq, slot = _slots(c)
    score, seen = _scores(c, seq, slot)
    s, h, m, length = c["seqs"], c["kv_heads"], c["q_max"], c["len_max"]
    lse = torch.zeros(s, m, c["q_heads"], device=DEV)
    lse[seq, slot] = c["lse"]
    lse = lse.view(s, m, h, -1).permute(0, 2, 3, 1)[..., None]                    # [S, H, G, m, 1]
    p = torch.exp(score.sub_(lse))                                               # (0 where a row sees nothing)
    w = p.sum((2, 3))                                                            # [S, H, L]
    lens, cu = c["lens"].long(), c["cu"].long()
    j = torch.arange(length, device=DEV).expand(s, h, length)
    here = j < lens[:, None, None]
    cells = _cells(c, c["page_table"].clamp(min=0), j)
    if c["earlier"] is not None:
        old = j < (lens - (cu[1:] - cu[:-1]))[:, None, None]
        w = w + torch.where(old, c["earlier"][cells], torch.zeros_like(w))
    c["weights"][tuple(x[here] for x in cells)] = w[here]
    return [c["weights"]]


def _select_plain(c):
    s, h, keep = c["seqs"], c["kv_heads"], c["keep"]
    lens = c["lens"].long()
    length = c["len_max"]
    j = torch.arange(length, device=DEV).expand(s, h, length)
    lim = lens[:, None, None]
    w = c["weights"][_cells(c, c["page_table"].clamp(min=0), j)]
    sure = (j < c["sinks"]) | (j >= lim - c["recent"])
    w = torch.where(sure, torch.full_like(w, math.inf), w)
    w = torch.where(j < lim, w, torch.full_like(w, -math.inf))
    order = w.sort(dim=-1, descending=True, stable=True).indices
    order = torch.nn.functional.pad(order, (0, max(0, keep - length)), value=length)
    kept = order[..., :keep]
    kept = torch.where(kept < lim, kept, torch.full_like(kept, 1 << 30)).sort(dim=-1).values
    c["kept"].copy_(torch.where(kept < lim, kept, torch.full_like(kept, -1)))
    c["new_lens"].copy_(lens.clamp(max=keep))


def _move_plain(codes, scales, c, source, target, real):
    """Tokens at the cells `source` [S, H, n] to the cells `target`, each block with the scale that its largest value asks for."""
    n, block = real.shape[2], c["block"]
    x = codes[source].view(torch.float8_e4m3fn).float()                          # [S, H, n, D]
    x *= torch.exp2(scales[source[0], source[1], source[2] // block].float() - 127)[..., None]
    m, e = torch.frexp(x.abs().amax(-1))
    asks = torch.where(m > 0.5, e, e - 1) - EMAX + 127
    asks = torch.where((m == 0) | ~real, torch.zeros_like(asks), asks).clamp(min=0)
    scale = torch.nn.functional.pad(asks, (0, -n % block)).unflatten(-1, (-1, block)).amax(-1).repeat_interleave(block, -1)[..., :n]
    x *= torch.exp2(127 - scale.float())[..., None]
    at = tuple(t[real] for t in target)
    codes[at] = x[real].to(torch.float8_e4m3fn).view(torch.uint8)
    scales[at[0], at[1], at[2] // block] = scale[real].to(torch.uint8)


def _evict_plain(c):
    _select_plain(c)
    kept = c["kept"].long()
    real = kept >= 0
    source = _cells(c, c["page_table"], kept.clamp(min=0))
    slot = torch.arange(c["keep"], device=DEV).expand_as(kept)
    target = _cells(c, c["out_table"], slot.clamp(max=c["out_table"].shape[1] * c["page"] - 1))
    _move_plain(c["k_codes"], c["k_scales"], c, source, target, real)
    _move_plain(c["v_codes"], c["v_scales"], c, source, target, real)
    c["weights"][tuple(t[real] for t in target)] = c["weights"][source][real]
    return _evicted(c)


def _evicted(c):
    return [c["kept"], c["new_lens"], c["k_codes"].view(torch.float8_e4m3fn), c["k_scales"].view(torch.float8_e8m0fnu),
            c["v_codes"].view(torch.float8_e4m3fn), c["v_scales"].view(torch.float8_e8m0fnu), c["weights"]]


def _run_plain(c):
    if c["op"] == "weights":
        return _weights_plain(c)
    if c["op"] == "evict":
        return _evict_plain(c)
    return _attend_plain(c, True)


# ---- the library's calls ---------------------------------------------------------------------------------------------

def _workspace(c, nbytes):
    if "workspace" not in c:
        c["workspace"] = torch.empty(max(16, nbytes()), dtype=torch.uint8, device=DEV)
    return c["workspace"]


def _run_own(c):
    b = _binding()
    if c["op"] == "weights":
        b.mxkv_attention_weights(c["q"], c["cu"], c["lens"], c["page_table"], c["k_codes"], c["k_scales"], c["lse"], c["weights"],
                                 c["q_max"], c["len_max"], c["scale"], earlier=c["earlier"])
        return [c["weights"]]
    if c["op"] == "evict":
        b.mxkv_select(c["weights"], c["lens"], c["page_table"], c["kept"], c["new_lens"], c["len_max"], sinks=c["sinks"],
                      recent=c["recent"])
        b.mxkv_compact(c["kept"], c["new_lens"], c["lens"], c["page_table"], c["k_codes"], c["k_scales"], c["v_codes"], c["v_scales"],
                       out_page_table=c["out_table"], weights=c["weights"])
        return _evicted(c)
    size = b.mxkv_attention_tree_workspace_bytes if c["op"] == "tree" else b.mxkv_attention_workspace_bytes
    ws = _workspace(c, lambda: size(c["n"], c["seqs"], c["q_max"], c["len_max"], c["q_heads"], c["kv_heads"], c["dim"]))
    cache = (c["k_codes"], c["k_scales"], c["v_codes"], c["v_scales"])
    if c["op"] == "sinks":
        b.mxkv_attention_sinks(c["q"], c["cu"], c["lens"], c["page_table"], *cache, c["out"], c["q_max"], c["len_max"], c["scale"],
                               c["window"], c["sinks"], lse=c["lse"], workspace=ws)
    else:
        b.mxkv_attention_tree(c["q"], c["cu"], c["lens"], c["page_table"], *cache, c["out"], c["q_max"], c["len_max"], c["scale"],
                              c["mask"], lse=c["lse"], workspace=ws)
    return [c["out"], c["lse"]]


def run(state):
    if own:
        return _run_own(state)
    return _run_plain(state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------

def work(case):
    c = case
    new, lens = (t.tolist() for t in _lengths(c))
    h, d, block = c["kv_heads"], c["dim"], c["block"]
    if c["op"] == "evict":
        kept = sum(min(n, c["keep"]) for n in lens)
        # the sums of all tokens read; codes, scales, sums of the kept ones read and written, their places written
        return {"bytes": h * (4.0 * sum(lens) + kept * (4 * d + 4 / block + 12)), "flops": 0}
    hq = c["q_heads"]
    pairs = used = 0.0
    for n, length in zip(new, lens):
        front = length - n
        if c["op"] == "tree":
            pairs += n * (front + 1.0)       # at least itself in the tree
            used += length
            continue
        full, reach = n * front + n * (n + 1) / 2, float(length)
        if c["op"] == "sinks":
            w, s = c["window"], c["sinks"]
            # the query at place p sees min(p + 1, window + min(sinks, p + 1 - window)) keys
            all_of = max(0, min(n, w + s - front))                        # queries that still see everything before them
            full = all_of * front + all_of * (all_of + 1) / 2 + (n - all_of) * (w + s)
            reach = float(min(length, w + n - 1 + s))
        pairs += full
        used += reach
    rows = float(sum(new)) * hq
    if c["op"] == "weights":
        fronts = float(sum(a - b for a, b in zip(lens, new)))
        return {"bytes": used * h * (d + 1 / block + 4) + (fronts * h * 4 if c["add"] else 0) + rows * (2 * d + 4), "flops": 2 * pairs * hq * d}
    mask = float(sum(new)) * ((c["q_max"] + 31) // 32 * 4) if c["op"] == "tree" else 0.0
    return {"bytes": used * h * (2 * d + 2 / block) + rows * (4 * d + 4) + mask, "flops": 4 * pairs * hq * d}


# ---- the same from the definitions in 64 bits ----------------------------------------------------------------------------

def _e4m3_values():
    return torch.arange(256, dtype=torch.int32, device=DEV).to(torch.uint8).view(torch.float8_e4m3fn).double()


def _exact_hidden(c, s, n, length):
    """[n, length]: what the queries of sequence s may not see."""
    place = length - n + torch.arange(n, device=DEV)[:, None]
    key = torch.arange(length, device=DEV)[None, :]
    if c["op"] == "tree":
        a = int(c["cu"][s])
        rows = c["mask"][a:a + n].tolist()
        bits = [[(row[i // 32] >> (i % 32)) & 1 for i in range(n)] for row in rows]
        hidden = torch.zeros(n, length, dtype=torch.bool, device=DEV)
        hidden[:, length - n:] = ~torch.tensor(bits, dtype=torch.bool, device=DEV)
        return hidden
    hidden = key > place
    if c["op"] == "sinks":
        hidden |= (key <= place - c["window"]) & (key >= c["sinks"])
    return hidden


def _exact_rows(codes, scales, c, pages, head, length):
    """[length, D] values of a sequence's tokens."""
    val = _e4m3_values()
    return (val[codes[pages, head].int()].view(-1, c["dim"])[:length]
            * torch.exp2(scales[pages, head].double() - 127).flatten().repeat_interleave(c["block"])[:length, None])


def _exact_evict(c):
    page, block, keep, sinks, recent = c["page"], c["block"], c["keep"], c["sinks"], c["recent"]
    val = _e4m3_values()
    outs = []
    for codes, scales in ((c["k_codes"], c["k_scales"]), (c["v_codes"], c["v_scales"])):
        outs += [val[codes.int()], torch.exp2(scales.double() - 127)]
    weights = c["weights"].double()
    kept_all = torch.full((c["seqs"], c["kv_heads"], keep), -1, dtype=torch.int32, device=DEV)
    lens = c["lens"].tolist()
    for s, length in enumerate(lens):
        pages = c["page_table"][s, :-(-length // page)].long()
        n = min(length, keep)
        slot = torch.arange(n, device=DEV)
        to_page, to_at = c["out_table"][s].long()[slot // page], slot % page
        for h in range(c["kv_heads"]):
            w = c["weights"][pages, h].flatten()[:length].double()
            if length <= keep:
                kept = slot
            else:
                # ranks by (weight falling, place rising), from a sort by place of equal weights
                middle = torch.arange(sinks, length - recent, device=DEV)
                value, where = torch.sort(-w[middle], stable=True)
                best = middle[where[:keep - sinks - recent]]
                kept = torch.cat([torch.arange(sinks, device=DEV), best, torch.arange(length - recent, length, device=DEV)]).sort().values
            kept_all[s, h, :n] = kept.to(torch.int32)
            weights[to_page, h, to_at] = w[kept]
            for i, (codes, scales) in enumerate(((c["k_codes"], c["k_scales"]), (c["v_codes"], c["v_scales"]))):
                x = _exact_rows(codes, scales, c, pages, h, length)[kept]
                top = torch.zeros(-(-n // block) * block, dtype=torch.float64, device=DEV)
                top[:n] = x.abs().amax(-1)
                top = top.view(-1, block).amax(-1)
                scale = torch.exp2((torch.ceil(torch.log2(top)) - EMAX).clamp(min=-127))
                each = scale.repeat_interleave(block)[:n]
                outs[2 * i][to_page, h, to_at] = x / each[:, None]
                outs[2 * i + 1][to_page, h, to_at // block] = each
    return [kept_all, torch.tensor(lens, device=DEV).clamp(max=keep).to(torch.int32), *outs, weights]


def exact(case, seed):
    c = prepare(case, seed)
    if c["op"] == "evict":
        return _exact_evict(c) if c["seqs"] * c["kv_heads"] <= 512 else None
    cu, lens = c["cu"].tolist(), c["lens"].tolist()
    hq, h, d, page = c["q_heads"], c["kv_heads"], c["dim"], c["page"]
    out = torch.zeros(c["n"], hq, d, dtype=torch.float64, device=DEV)
    lse = torch.zeros(c["n"], hq, dtype=torch.float64, device=DEV)
    sums = torch.zeros_like(c["weights"], dtype=torch.float64) if c["op"] == "weights" else None
    for s in range(c["seqs"]):
        n, length = cu[s + 1] - cu[s], lens[s]
        pages = c["page_table"][s, :-(-length // page)].long()
        hidden = _exact_hidden(c, s, n, length)
        for i in range(h):
            k = _exact_rows(c["k_codes"], c["k_scales"], c, pages, i, length)
            v = None if sums is not None else _exact_rows(c["v_codes"], c["v_scales"], c, pages, i, length)
            given = torch.zeros(length, dtype=torch.float64, device=DEV)
            for j in range(i * (hq // h), (i + 1) * (hq // h)):
                z = (c["q"][cu[s]:cu[s + 1], j].double() @ k.T * c["scale"]).masked_fill_(hidden, -math.inf)
                if sums is not None:
                    given += torch.exp(z - c["lse"][cu[s]:cu[s + 1], j, None].double()).sum(0)
                    continue
                lse[cu[s]:cu[s + 1], j] = torch.logsumexp(z, -1)
                out[cu[s]:cu[s + 1], j] = torch.softmax(z, -1) @ v
            if sums is not None:
                if c["earlier"] is not None:
                    given[:length - n] += c["earlier"][pages, i].flatten()[:length - n].double()
                key = torch.arange(length, device=DEV)
                sums[pages[key // page], i, key % page] = given
    return [sums] if sums is not None else [out, lse]
