"""Per-head norm with rotation, append to an 8-bit paged cache and attention over that cache: measured cases.

The path of queries, keys and values around attention, in the order in which a model runs it:

* ``norm`` / ``norm_bwd`` - RMS norm of every query and key head with the position rotation in the same pass, and its gradient;
* ``append`` - keys (rotated on the way) and values of new tokens written into a paged cache of E4M3 codes with one E8M0
  scale for each block of tokens and head;
* ``attend`` - attention of new queries (one token a sequence, a few, or a prompt) over that cache.

``run`` computes the operators in elementary torch operations where ``own`` is false and calls the library where it is true.
"""
import math

import torch

own = False

binding = None    # the library, imported by the first call that needs it

DEV = "cuda"
EMAX = 8          # log2 of the largest power of two of E4M3
THETA = 500000.0  # base of the rotation's angles


def _binding():
    global binding
    if binding is None:
        from paper_2603_13180_b200 import binding as b
        binding = b
    return binding


# ---- cases ---------------------------------------------------------------------------------------------------------

def _norm(kind, tokens, q_heads, k_heads, dim, rot, interleaved, table):
    return {"op": kind, "tokens": tokens, "q_heads": q_heads, "k_heads": k_heads, "dim": dim, "rot": rot,
            "interleaved": interleaved, "table": table}


def _append(seqs, new_max, len_max, kv_heads, dim, page, block, rot, interleaved):
    return {"op": "append", "seqs": seqs, "new_max": new_max, "len_max": len_max, "kv_heads": kv_heads, "dim": dim, "page": page,
            "block": block, "rot": rot, "interleaved": interleaved}


def _attend(seqs, q_max, len_max, q_heads, kv_heads, dim, page, block, window):
    return {"op": "attend", "seqs": seqs, "q_max": q_max, "len_max": len_max, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "page": page, "block": block, "window": window}


def listed():
    return [
        # one decode step of 64 sequences at hidden size 4096 (32 query and 8 key heads of 128): a launch-bound call
        dict(_norm("norm", 64, 32, 8, 128, 128, False, 8192), name="norm decode 64"),
        # the training batch of the benchmark, 16384 tokens at hidden size 4096
        dict(_norm("norm", 16384, 32, 8, 128, 128, False, 8192), name="norm train 16384"),
        # its backward, with the gradients of both gains
        dict(_norm("norm_bwd", 16384, 32, 8, 128, 128, False, 8192), name="norm backward 16384"),
        # hidden size 2048 in heads of 64, an odd token count, interleaved pairs and a rotation of half the head
        dict(_norm("norm_bwd", 4099, 32, 4, 64, 32, True, 131072), name="norm backward odd"),
        # one token for each of 64 running sequences
        dict(_append(64, 1, 2048, 8, 128, 64, 16, 128, False), name="append decode 64"),
        # prompts of several lengths, some behind an earlier part of the same sequence
        dict(_append(6, 4096, 8192, 8, 128, 64, 16, 128, False), name="append prompts"),
        # a single user with a short history: latency
        dict(_attend(1, 1, 1000, 32, 8, 128, 64, 16, 0), name="attend one short"),
        # a serving batch of ragged lengths
        dict(_attend(64, 1, 8192, 32, 8, 128, 64, 16, 0), name="attend batch 64"),
        # a single user with a very long history
        dict(_attend(1, 1, 131072, 32, 8, 128, 64, 16, 0), name="attend one long"),
        # four drafted tokens a sequence in heads of 64, small pages, a sliding window
        dict(_attend(32, 4, 4100, 32, 4, 64, 16, 16, 1024), name="attend drafts window"),
        # a prompt's second half over the whole prompt
        dict(_attend(1, 4096, 8192, 32, 8, 128, 64, 16, 0), name="attend prompt"),
        # several short prompts together in heads of 64
        dict(_attend(8, 1000, 1500, 32, 4, 64, 32, 32, 0), name="attend prompts ragged"),
    ]


def _between(rng, lo, hi):
    """A whole number from lo to hi, spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm_bwd", "append", "attend", "attend", "attend"])
    dim = rng.choice([64, 128])
    page = rng.choice([16, 32, 64, 128])
    block = rng.choice([b for b in (16, 32, 64) if b <= page])
    kv = rng.choice([1, 2, 4, 8])
    if kind in ("norm", "norm_bwd"):
        dim = rng.choice([64, 96, 128, 256])
        heads = kv * rng.choice([1, 2, 4])
        most = max(1, min(16384, 16384 * 40 * 128 // ((heads + kv) * dim)))
        return _norm(kind, _between(rng, 1, most), heads, kv, dim, rng.choice([dim, dim // 2]), rng.random() < 0.5,
                     rng.choice([4096, 32768, 131072]))
    if kind == "append":
        seqs = _between(rng, 1, 64)
        new = _between(rng, 1, max(1, 16384 // seqs))
        return _append(seqs, new, new + _between(rng, 1, 4096), kv, dim, page, block, rng.choice([0, dim // 2, dim]),
                       rng.random() < 0.5)
    group = rng.choice([1, 2, 3, 4, 6, 8, 16])
    form = rng.choice(["one", "one", "few", "prompt"])
    window = rng.choice([0, 0, _between(rng, 16, 2000)])
    if form == "prompt":
        heads = kv * group
        seqs = _between(rng, 1, 8)
        room = 4096 * 8192 * 32 * 128 // (heads * dim * seqs)     # query tokens times length
        q = _between(rng, 16, max(16, min(4096, int(math.sqrt(room / 2)))))
        return _attend(seqs, q, min(q + _between(rng, 1, 4096), max(q, room // q)), heads, kv, dim, page, block, window)
    seqs = _between(rng, 1, 64)
    length = _between(rng, 1, max(1, min(131072, 64 * 8192 * 8 * 128 // (seqs * kv * dim))))
    q = 1 if form == "one" else rng.randint(2, 8)
    return _attend(seqs, q, max(q, length), kv * group, kv, dim, page, block, window)


# ---- inputs --------------------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 2654435761 % (1 << 62) + 17)
    return g


def _table(rows, rot):
    """[rows, rot] binary32: rot/2 cosines, then rot/2 sines, of pos * THETA^(-2i/rot), from angles in 64 bits."""
    inv = THETA ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    ang = torch.arange(rows, dtype=torch.float64, device=DEV)[:, None] * inv
    return torch.cat([ang.cos(), ang.sin()], dim=1).float().contiguous()


def _hidden(g, rows, width):
    """bf16 activations as projections give them: normal, a scale for each row, a few channels far larger."""
    x = torch.randn(rows, width, generator=g, device=DEV)
    x *= torch.exp(0.5 * torch.randn(rows, 1, generator=g, device=DEV))
    x[:, torch.randint(0, width, (max(1, width // 1000),), generator=g, device=DEV)] *= 8
    return x.to(torch.bfloat16)


def _sizes(n, most, least, turn):
    """n whole numbers from least to most on the host: the first is `most`, the rest are spread over its upper three quarters.
    They go by the case alone; `turn` tells the lists of one case apart."""
    i = torch.arange(n, dtype=torch.float64)
    u = (i * 0.6180339887498949 + 0.37 * turn) % 1.0
    s = (most * (0.25 + 0.75 * u)).long().clamp_(least, most)
    s[0] = most
    return s


def _lengths(c):
    """(new tokens, length with them) of each sequence of an append or attend case."""
    if c["op"] == "append":
        new = _sizes(c["seqs"], c["new_max"], 1, 0)
        return new, _sizes(c["seqs"], c["len_max"] - c["new_max"], 0, 1) + new
    lens = _sizes(c["seqs"], c["len_max"], 1, 1)
    q = _sizes(c["seqs"], c["q_max"], 1, 0) if c["q_max"] > 8 else torch.full((c["seqs"],), c["q_max"])
    return torch.minimum(q, lens), lens


def _cum(n):
    return torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]).to(torch.int32)


def _pages(g, lens, width, page):
    """Page table [seqs, width] in a shuffled pool, -1 behind each sequence's last page, and the pool's size."""
    need = (lens + page - 1) // page
    total = int(need.sum())
    pool = total + total // 16 + 1
    order = torch.randperm(pool, generator=torch.Generator().manual_seed(g + 1))[:total].to(torch.int32)
    table = torch.full((len(lens), width), -1, dtype=torch.int32)
    at = torch.arange(width)[None, :] < need[:, None]
    table[at] = order
    return table.to(DEV), pool


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


def prepare(case, seed):
    c = dict(case)
    g = _gen(seed)
    if c["op"] in ("norm", "norm_bwd"):
        t, hq, hk, d = c["tokens"], c["q_heads"], c["k_heads"], c["dim"]
        # the fused projection's output: queries, keys and values of a token side by side
        x = _hidden(g, t, (hq + 2 * hk) * d)
        c["q"] = x[:, :hq * d].view(t, hq, d)
        c["k"] = x[:, hq * d:(hq + hk) * d].view(t, hk, d)
        c["q_gain"] = (1 + 0.1 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16)
        c["k_gain"] = (1 + 0.1 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16)
        c["cos_sin"] = _table(c["table"], c["rot"])
        first = torch.randint(0, max(1, c["table"] - t), (1,), generator=g, device=DEV, dtype=torch.int32)
        c["positions"] = ((torch.arange(t, device=DEV, dtype=torch.int32) + first) % c["table"]).to(torch.int32)
        c["q_out"] = torch.empty(t, hq, d, dtype=torch.bfloat16, device=DEV)
        c["k_out"] = torch.empty(t, hk, d, dtype=torch.bfloat16, device=DEV)
        if c["op"] == "norm_bwd":
            c["gq"] = (1e-2 * torch.randn(t, hq, d, generator=g, device=DEV)).to(torch.bfloat16)
            c["gk"] = (1e-2 * torch.randn(t, hk, d, generator=g, device=DEV)).to(torch.bfloat16)
            c["dq_gain"] = torch.empty(d, dtype=torch.float32, device=DEV)
            c["dk_gain"] = torch.empty(d, dtype=torch.float32, device=DEV)
        return c
    h, d, page, block, s = c["kv_heads"], c["dim"], c["page"], c["block"], c["seqs"]
    if c["op"] == "append":
        new, lens = _lengths(c)
        c["n"] = int(new.sum())
        x = _hidden(g, c["n"], 2 * h * d)
        c["k"] = x[:, :h * d].view(-1, h, d)
        c["v"] = x[:, h * d:].view(-1, h, d)
        c["cu"] = _cum(new).to(DEV)
        c["cos_sin"] = _table(c["len_max"], c["rot"]) if c["rot"] else None
    else:
        q, lens = _lengths(c)
        c["n"] = int(q.sum())
        c["cu"] = _cum(q).to(DEV)
        hq = c["q_heads"]
        c["q"] = (2 * torch.randn(c["n"], hq, d, generator=g, device=DEV)).to(torch.bfloat16)
        c["scale"] = 1.0 / math.sqrt(d)
        c["out"] = torch.empty(c["n"], hq, d, dtype=torch.bfloat16, device=DEV)
        c["lse"] = torch.empty(c["n"], hq, dtype=torch.float32, device=DEV)
    c["lens"] = lens.to(torch.int32).to(DEV)
    c["page_table"], pool = _pages(seed, lens, -(-c["len_max"] // page), page)
    c["k_codes"], c["k_scales"] = _cache(g, pool, h, page, d, block)
    c["v_codes"], c["v_scales"] = _cache(g, pool, h, page, d, block)
    return c


# ---- plain forms: elementary torch operations in binary32 ------------------------------------------------------------

def _rotate(x, table, pos, interleaved, back=False):
    """x [T, H, D] binary32: the first rot elements of each head turned in pairs by the token's angles."""
    rot = table.shape[1]
    row = table[pos.long()]
    cos, sin = row[:, None, :rot // 2], row[:, None, rot // 2:]
    if back:
        sin = -sin
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([turned, x[..., rot:]], dim=-1)


EPS = 1e-6


def _norm_plain(x, gain, c):
    x = x.float()
    u = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain.float()
    return _rotate(u, c["cos_sin"], c["positions"], c["interleaved"]).to(torch.bfloat16)


def _norm_bwd_plain(x, grad, gain, c):
    x = x.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    n = x * r
    du = _rotate(grad.float(), c["cos_sin"], c["positions"], c["interleaved"], back=True)
    h = du * gain.float()
    dx = r * (h - n * (h * n).mean(-1, keepdim=True))
    return dx.to(torch.bfloat16), (du * n).sum((0, 1))


def _where(c):
    """Sequence and position of each of the c["n"] rows of new tokens."""
    cu = c["cu"].long()
    row = torch.arange(c["n"], device=DEV)
    seq = torch.searchsorted(cu[1:].contiguous(), row, right=True)
    return seq, c["lens"].long()[seq] - cu[seq + 1] + row


def _append_one(x, codes, scales, c, seq, pos):
    """x [N, H, D] binary32 into codes / scales, in place."""
    page, block = c["page"], c["block"]
    table, cu, lens = c["page_table"].long(), c["cu"].long(), c["lens"].long()
    # the scale exponent each token asks for: ceil(log2 absmax) - 8
    m, e = torch.frexp(x.abs().amax(-1))
    asks = torch.where(m > 0.5, e, e - 1) - EMAX + 127
    asks = torch.where(m == 0, torch.zeros_like(asks), asks).clamp(min=0)
    new = torch.full(scales.shape, -1, dtype=torch.int32, device=DEV)
    # blocks that hold earlier tokens keep at least their scale
    start = lens - (cu[1:] - cu[:-1])
    kept = start % block != 0
    at = (table.gather(1, (start // page).clamp(max=table.shape[1] - 1)[:, None])[:, 0].clamp(min=0), (start % page) // block)
    old = scales[at[0], :, at[1]].int()                                          # [S, H]
    per = scales.shape[2]
    heads = torch.arange(scales.shape[1], device=DEV)
    flat = new.view(-1)
    cell = (at[0][:, None] * scales.shape[1] + heads) * per + at[1][:, None]     # [S, H]
    flat.scatter_reduce_(0, cell.flatten(), torch.where(kept[:, None], old, torch.full_like(old, -1)).flatten(), "amax")
    pg, off = table[seq, pos // page], pos % page
    mine = (pg[:, None] * scales.shape[1] + heads) * per + (off // block)[:, None]
    flat.scatter_reduce_(0, mine.flatten(), asks.int().flatten(), "amax")
    scales.copy_(torch.where(new >= 0, new.to(torch.uint8), scales))
    # earlier tokens of a shared block: their codes on the new scale
    within = torch.arange(block, device=DEV)
    first = (start % page) // block * block
    o = first[:, None] + within                                                  # [S, block] offsets in the page
    was = codes[at[0][:, None], :, o].view(torch.float8_e4m3fn).float()          # [S, block, H, D]
    by = torch.exp2((old - scales[at[0], :, at[1]].int()).float())               # [S, H]
    again = (was * by[:, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    mine_before = kept[:, None] & (o < (start % page)[:, None])
    keep = codes[at[0][:, None], :, o]
    codes[at[0][:, None], :, o] = torch.where(mine_before[:, :, None, None], again, keep)
    # the new tokens' codes
    sb = flat[mine].float()                                                      # [N, H]
    codes[pg, :, off] = (x * torch.exp2(127 - sb)[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)


def _append_plain(c):
    seq, pos = _where(c)
    k = c["k"].float()
    if c["cos_sin"] is not None:
        k = _rotate(k, c["cos_sin"], pos, c["interleaved"])
    _append_one(k, c["k_codes"], c["k_scales"], c, seq, pos)
    _append_one(c["v"].float(), c["v_codes"], c["v_scales"], c, seq, pos)


def _cache_out(c):
    return [c["k_codes"].view(torch.float8_e4m3fn), c["k_scales"].view(torch.float8_e8m0fnu),
            c["v_codes"].view(torch.float8_e4m3fn), c["v_scales"].view(torch.float8_e8m0fnu)]


def _dense(codes, scales, c):
    """[S, L, H, D] binary32 values of every sequence, whatever stands behind its length."""
    t = c["page_table"].long().clamp(min=0)
    x = codes[t].view(torch.float8_e4m3fn).float()                               # [S, P, H, page, D]
    s = torch.exp2(scales[t].float() - 127).repeat_interleave(c["block"], -1)    # [S, P, H, page]
    return (x * s[..., None]).transpose(2, 3).flatten(1, 2)[:, :c["len_max"]]


def _attend_plain(c):
    hq, h, d, s, m = c["q_heads"], c["kv_heads"], c["dim"], c["seqs"], c["q_max"]
    cu, lens = c["cu"].long(), c["lens"].long()
    seq, pos = _where(c)
    slot = torch.arange(c["n"], device=DEV) - cu[seq]
    q = torch.zeros(s, m, hq, d, device=DEV)
    q[seq, slot] = c["q"].float()
    at = torch.full((s, m), -1, dtype=torch.int64, device=DEV)
    at[seq, slot] = pos
    k = _dense(c["k_codes"], c["k_scales"], c)
    q = q.view(s, m, h, hq // h, d).permute(0, 2, 3, 1, 4).flatten(2, 3)          # [S, H, G*m, D]
    score = torch.matmul(q, k.permute(0, 2, 3, 1)) * c["scale"]                   # [S, H, G*m, L]
    del k
    j = torch.arange(score.shape[-1], device=DEV)
    seen = (j <= at[..., None]) & (j < lens[:, None, None])
    if c["window"]:
        seen &= j > at[..., None] - c["window"]
    score = score.view(s, h, hq // h, m, -1)
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(score.sub_(top))
    total = p.sum(-1, keepdim=True)
    lse = (top + torch.log(total))[..., 0]                                        # [S, H, G, m]
    v = _dense(c["v_codes"], c["v_scales"], c)
    o = torch.matmul(p.flatten(2, 3), v.transpose(1, 2)).view(s, h, hq // h, m, d)
    o = o / torch.where(total > 0, total, torch.ones_like(total))
    o = o.permute(0, 3, 1, 2, 4).flatten(2, 3)[seq, slot]
    return [o.to(torch.bfloat16), lse.permute(0, 3, 1, 2).flatten(2, 3)[seq, slot]]


def _run_plain(c):
    if c["op"] == "norm":
        return [_norm_plain(c["q"], c["q_gain"], c), _norm_plain(c["k"], c["k_gain"], c)]
    if c["op"] == "norm_bwd":
        dq, dqg = _norm_bwd_plain(c["q"], c["gq"], c["q_gain"], c)
        dk, dkg = _norm_bwd_plain(c["k"], c["gk"], c["k_gain"], c)
        return [dq, dk, dqg, dkg]
    if c["op"] == "append":
        _append_plain(c)
        return _cache_out(c)
    return _attend_plain(c)


# ---- the library's calls ---------------------------------------------------------------------------------------------

def _workspace(c, nbytes):
    if "workspace" not in c:
        c["workspace"] = torch.empty(max(16, nbytes), dtype=torch.uint8, device=DEV)
    return c["workspace"]


def _run_own(c):
    b = _binding()
    if c["op"] == "norm":
        b.rmsnorm_rope_fwd(c["q"], c["k"], c["q_gain"], c["k_gain"], c["cos_sin"], c["positions"], c["q_out"], c["k_out"], eps=EPS,
                            interleaved=c["interleaved"])
        return [c["q_out"], c["k_out"]]
    if c["op"] == "norm_bwd":
        ws = c.get("workspace")
        if ws is None:
            ws = _workspace(c, b.rmsnorm_rope_bwd_workspace_bytes(c["tokens"], c["q_heads"], c["k_heads"], c["dim"]))
        b.rmsnorm_rope_bwd(c["q"], c["k"], c["gq"], c["gk"], c["q_gain"], c["k_gain"], c["cos_sin"], c["positions"], c["q_out"],
                            c["k_out"], c["dq_gain"], c["dk_gain"], ws, eps=EPS, interleaved=c["interleaved"])
        return [c["q_out"], c["k_out"], c["dq_gain"], c["dk_gain"]]
    if c["op"] == "append":
        b.mxkv_append(c["k"], c["v"], c["cu"], c["lens"], c["page_table"], c["k_codes"], c["k_scales"], c["v_codes"], c["v_scales"],
                      cos_sin=c["cos_sin"], interleaved=c["interleaved"])
        return _cache_out(c)
    ws = c.get("workspace")
    if ws is None:
        ws = _workspace(c, b.mxkv_attention_workspace_bytes(c["n"], c["seqs"], c["q_max"], c["len_max"], c["q_heads"], c["kv_heads"],
                                                            c["dim"]))
    b.mxkv_attention(c["q"], c["cu"], c["lens"], c["page_table"], c["k_codes"], c["k_scales"], c["v_codes"], c["v_scales"], c["out"],
                     c["q_max"], c["len_max"], c["scale"], lse=c["lse"], window=c["window"], workspace=ws)
    return [c["out"], c["lse"]]


def run(state):
    if own:
        return _run_own(state)
    return _run_plain(state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------

def work(case):
    c = case
    if c["op"] in ("norm", "norm_bwd"):
        t, e = c["tokens"], c["tokens"] * (c["q_heads"] + c["k_heads"]) * c["dim"]
        rows = min(t, c["table"])
        small = rows * c["rot"] * 4 + 4 * t + 4 * c["dim"]
        if c["op"] == "norm":
            return {"bytes": 4 * e + small, "flops": 8 * e}
        return {"bytes": 6 * e + small + 8 * c["dim"], "flops": 16 * e}
    new, lens = (t.double() for t in _lengths(c))
    if c["op"] == "append":
        n = float(new.sum())
        e = n * c["kv_heads"] * c["dim"]
        return {"bytes": 2 * e * 3 + n * c["rot"] * 4 + 2 * n * c["kv_heads"] / c["block"], "flops": 8 * e}
    hq, h, d, w = c["q_heads"], c["kv_heads"], c["dim"], c["window"]
    pairs = used = 0.0
    for n, length in zip(new.tolist(), lens.tolist()):
        # the query at place p sees p + 1 keys, or as many of them as its window holds
        full = n * (length - n) + n * (n + 1) / 2
        if w:
            short = max(0.0, min(w, length) - (length - n))   # queries that see fewer keys than the window holds
            full = (n - short) * w + short * (length - n) + short * (short + 1) / 2
        pairs += full
        used += min(length, w + n - 1) if w else length
    return {"bytes": used * h * (2 * d + 2 / c["block"]) + float(new.sum()) * hq * (4 * d + 4), "flops": 4 * pairs * hq * d}


# ---- the same from the definitions in 64 bits ----------------------------------------------------------------------------

def _turn64(x, c, pos, sign):
    """Rotation as a product of complex numbers, with the table's own cosines and sines."""
    rot = c["rot"]
    if not rot:
        return x
    row = c["cos_sin"].double().index_select(0, pos.long())
    w = torch.complex(row[:, :rot // 2], sign * row[:, rot // 2:])[:, None, :]
    y = x.clone()
    if c["interleaved"]:
        z = torch.view_as_complex(x[..., :rot].reshape(*x.shape[:-1], rot // 2, 2).contiguous()) * w
        y[..., :rot] = torch.view_as_real(z).flatten(-2)
    else:
        z = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:rot].contiguous()) * w
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    return y


def _e4m3_values():
    return torch.arange(256, dtype=torch.int32, device=DEV).to(torch.uint8).view(torch.float8_e4m3fn).double()


def _exact_append(x, codes, scales, c):
    """Codes as the unrounded quotients by the block's scale, scales as powers of two; the earlier codes as they stand."""
    val = _e4m3_values()
    out, sc = val[codes.int()], torch.exp2(scales.double() - 127)
    cu, lens, table = c["cu"].tolist(), c["lens"].tolist(), c["page_table"].tolist()
    page, block = c["page"], c["block"]
    for s in range(c["seqs"]):
        n = cu[s + 1] - cu[s]
        p, end = lens[s] - n, lens[s]
        while p < end:
            stop = min(end, (p // block + 1) * block)
            pg, b, o = table[s][p // page], (p % page) // block, p % page
            new = x[cu[s + 1] - end + p:cu[s + 1] - end + stop].transpose(0, 1)            # [H, n, D]
            top = new.abs().amax((1, 2))
            want = torch.exp2(torch.ceil(torch.log2(top)) - EMAX)
            if p % block:
                was = sc[pg, :, b].clone()
                want = torch.maximum(want, was)
                out[pg, :, b * block:o] *= (was / want)[:, None, None]
            sc[pg, :, b] = want
            out[pg, :, o:o + stop - p] = new / want[:, None, None]
            p = stop
    return out, sc


def exact(case, seed):
    c = prepare(case, seed)
    if c["op"] in ("norm", "norm_bwd"):
        res, gains = [], []
        for x, g, gain in ((c["q"], c.get("gq"), c["q_gain"]), (c["k"], c.get("gk"), c["k_gain"])):
            x, gain = x.double(), gain.double()
            rms = torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS)
            if g is None:
                res.append(_turn64(x / rms * gain, c, c["positions"], 1.0))
                continue
            back = _turn64(g.double(), c, c["positions"], -1.0)
            gains.append((back * x / rms).sum((0, 1)))
            h = back * gain
            res.append(h / rms - x * (h * x).sum(-1, keepdim=True) / (x.shape[-1] * rms ** 3))
        return res + gains
    if c["op"] == "append":
        if c["n"] // c["block"] + c["seqs"] > 6000:
            return None
        cu, lens = c["cu"].tolist(), c["lens"].tolist()
        pos = torch.cat([torch.arange(lens[s] - (cu[s + 1] - cu[s]), lens[s]) for s in range(c["seqs"])]).to(DEV)
        k, ks = _exact_append(_turn64(c["k"].double(), c, pos, 1.0), c["k_codes"], c["k_scales"], c)
        v, vs = _exact_append(c["v"].double(), c["v_codes"], c["v_scales"], c)
        return [k, ks, v, vs]
    val = _e4m3_values()
    cu, lens = c["cu"].tolist(), c["lens"].tolist()
    hq, h, d, page, block = c["q_heads"], c["kv_heads"], c["dim"], c["page"], c["block"]
    out = torch.zeros(c["n"], hq, d, dtype=torch.float64, device=DEV)
    lse = torch.zeros(c["n"], hq, dtype=torch.float64, device=DEV)
    for s in range(c["seqs"]):
        n, L = cu[s + 1] - cu[s], lens[s]
        pages = c["page_table"][s, :-(-L // page)].long()
        place = L - n + torch.arange(n, device=DEV)
        key = torch.arange(L, device=DEV)
        hidden = key[None, :] > place[:, None]
        if c["window"]:
            hidden |= key[None, :] <= place[:, None] - c["window"]
        for i in range(h):
            kk, vv = (val[codes[pages, i].int()].view(-1, d)[:L]
                      * torch.exp2(sc[pages, i].double() - 127).flatten().repeat_interleave(block)[:L, None]
                      for codes, sc in ((c["k_codes"], c["k_scales"]), (c["v_codes"], c["v_scales"])))
            for j in range(i * (hq // h), (i + 1) * (hq // h)):
                z = (c["q"][cu[s]:cu[s + 1], j].double() @ kk.T * c["scale"]).masked_fill_(hidden, -math.inf)
                lse[cu[s]:cu[s + 1], j] = torch.logsumexp(z, -1)
                out[cu[s]:cu[s + 1], j] = torch.softmax(z, -1) @ vv
    return [out, lse]
