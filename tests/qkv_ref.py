"""Plain statements of the per-head norm with rotation, the cache append and the attention over the cache, for the tests: 64 bits
throughout, except where the contract itself fixes binary32 operations (the rotation in front of the cache's cast)."""
import math

import torch


def rope_table(rows, rot, base=10000.0):
    inv = base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    ang = torch.arange(rows, dtype=torch.float64)[:, None] * inv
    return torch.cat([ang.cos(), ang.sin()], 1).float()


def rotate(x, table, pos, pairs, sign=1.0):
    """x [T, H, D] in any precision, table [P, rot]; products and sums are rounded to x's type one by one."""
    if table is None:
        return x
    rot = table.shape[1]
    row = table[pos.long()].to(x.dtype)
    c, s = row[:, None, :rot // 2], sign * row[:, None, rot // 2:]
    y = x.clone()
    ia, ib = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x[..., ia], x[..., ib]
    y[..., ia] = a * c - b * s
    y[..., ib] = b * c + a * s
    return y


def norm_fwd(x, gain, eps, normalise=True):
    """u = x / rms * gain in 64 bits."""
    x = x.double()
    if not normalise:
        return x
    ms = (x * x).mean(-1, keepdim=True) + eps
    r = torch.where(ms > 0, 1 / torch.sqrt(ms), torch.zeros_like(ms))
    return x * r * (1.0 if gain is None else gain.double())


def norm_bwd(x, du, gain, eps):
    """(dx, dgain, bound on |dx| before cancellation, sum of |du n|), 64 bits; du is already turned back."""
    x = x.double()
    ms = (x * x).mean(-1, keepdim=True) + eps
    r = torch.where(ms > 0, 1 / torch.sqrt(ms), torch.zeros_like(ms))
    n, h = x * r, du * (1.0 if gain is None else gain.double())
    m = (h * n).mean(-1, keepdim=True)
    size = r * (h.abs().amax(-1, keepdim=True) + n.abs().amax(-1, keepdim=True) * (h * n).abs().mean(-1, keepdim=True))
    return r * (h - n * m), (du * n).sum((0, 1)), size, (du * n).abs().sum((0, 1))


def ceil_log2(x):
    m, e = math.frexp(x)
    return e - 1 if m == 0.5 else e


def append(x, codes, scales, cu, lens, table, page, block):
    """x [n, H, D] binary32 (rotated) on the CPU into codes / scales (CPU, in place), token by token of each block."""
    heads = codes.shape[1]
    for s in range(len(lens)):
        n = cu[s + 1] - cu[s]
        p, end = lens[s] - n, lens[s]
        while p < end:
            stop = min(end, (p // block + 1) * block)
            pg, b, o = table[s][p // page], (p % page) // block, p % page
            for h in range(heads):
                new = x[cu[s + 1] - end + p:cu[s + 1] - end + stop, h]
                top = float(new.abs().max())
                sb = 0 if top < 2.0 ** -126 else max(0, ceil_log2(top) - 8 + 127)
                if p % block:
                    old = int(scales[pg, h, b])
                    if old > sb:
                        sb = old
                    elif old < sb:
                        was = codes[pg, h, b * block:o].view(torch.float8_e4m3fn).double() * 2.0 ** (old - sb)
                        codes[pg, h, b * block:o] = was.float().to(torch.float8_e4m3fn).view(torch.uint8)
                scales[pg, h, b] = sb
                codes[pg, h, o:o + stop - p] = (new.double() * 2.0 ** (127 - sb)).float().to(torch.float8_e4m3fn).view(torch.uint8)
            p = stop


def dequantise(codes, scales, pages, block, head, length):
    """[length, D] binary64 keys (or values) of one head of a sequence with the given pages."""
    c = codes[pages, head].view(torch.float8_e4m3fn).double().flatten(0, 1)
    s = torch.exp2(scales[pages, head].double() - 127).flatten().repeat_interleave(block)
    return (c * s[:, None])[:length]


def attention(q, cu, lens, table, kc, ks, vc, vs, scale, causal=True, window=0):
    """(out, lse, sum of softmax |v|, largest sum of |scale q k|), all binary64, rows of no sequence NaN."""
    n, hq, d = q.shape
    heads, page = kc.shape[1], kc.shape[2]
    block = page // ks.shape[2]
    g = hq // heads
    out = torch.full((n, hq, d), math.nan, dtype=torch.float64, device=q.device)
    mag, lse, big = out.clone(), out[..., 0].clone(), out[..., 0].clone()
    for s in range(len(lens)):
        a, b, length = cu[s], cu[s + 1], lens[s]
        if a == b:
            continue
        pages = torch.tensor(table[s][:-(-length // page)], dtype=torch.long, device=q.device)
        place = length - (b - a) + torch.arange(b - a, device=q.device)
        key = torch.arange(length, device=q.device)
        seen = torch.ones(b - a, length, dtype=torch.bool, device=q.device)
        if causal:
            seen &= key[None] <= place[:, None]
        if window:
            seen &= key[None] > place[:, None] - window
        for h in range(heads):
            k, v = (dequantise(c, sc, pages, block, h, length) for c, sc in ((kc, ks), (vc, vs)))
            for j in range(h * g, (h + 1) * g):
                x = q[a:b, j].double()
                z = (x @ k.T * scale).masked_fill(~seen, -math.inf)
                lse[a:b, j] = torch.logsumexp(z, -1) if length else -math.inf
                p = torch.nan_to_num(torch.softmax(z, -1), 0.0)
                out[a:b, j], mag[a:b, j] = p @ v, p @ v.abs()
                big[a:b, j] = ((x.abs() @ k.abs().T) * abs(scale)).masked_fill(~seen, 0).amax(-1) if length else 0.0
    return out, lse, mag, big
