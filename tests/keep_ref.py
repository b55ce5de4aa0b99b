"""Plain statements, in 64 bits, of attention over the cache under any mask, of the keys' summed weights, of the choice of tokens that stay and of
moving them, for the tests."""
import math

import torch

from tests import qkv_ref as ref


def sinks_mask(n, length, window, sinks, causal=True, device="cpu"):
    """[n, length]: which keys the last n tokens of a sequence see."""
    place = length - n + torch.arange(n, device=device)[:, None]
    key = torch.arange(length, device=device)[None]
    seen = key <= place if causal else torch.ones(n, length, dtype=torch.bool, device=device)
    if window:
        seen &= (key > place - window) | (key < sinks)
    return seen


def tree_mask(rows, length, device="cpu"):
    """[n, length]: all in front of the n new tokens, and those whose bit the row (a whole number) has."""
    n = len(rows)
    seen = torch.ones(n, length, dtype=torch.bool, device=device)
    front = length - n
    for i, row in enumerate(rows):
        for j in range(n):
            if front + j >= 0:
                seen[i, front + j] = bool(row >> j & 1)
    return seen


def words(rows, count):
    """int32 [rows, count] of whole numbers."""
    out = [[(r >> 32 * w & 0xFFFFFFFF) for w in range(count)] for r in rows]
    return torch.tensor([[v - (1 << 32) if v >> 31 else v for v in row] for row in out], dtype=torch.int32).reshape(-1, count)


def attention(q, cu, lens, table, kc, ks, vc, vs, scale, masks):
    """(out, lse, sum of softmax |v|, largest sum of |scale q k|) under masks[s] [n, length]."""
    n, hq, d = q.shape
    heads, page = kc.shape[1], kc.shape[2]
    block, g = page // ks.shape[2], hq // heads
    out = torch.full((n, hq, d), math.nan, dtype=torch.float64, device=q.device)
    mag, lse, big = out.clone(), out[..., 0].clone(), out[..., 0].clone()
    for s, length in enumerate(lens):
        a, b = cu[s], cu[s + 1]
        if a == b:
            continue
        pages = torch.tensor(table[s][:-(-length // page)], dtype=torch.long, device=q.device)
        for h in range(heads):
            k, v = (ref.dequantise(c, sc, pages, block, h, length) for c, sc in ((kc, ks), (vc, vs)))
            for j in range(h * g, (h + 1) * g):
                x = q[a:b, j].double()
                z = (x @ k.T * scale).masked_fill(~masks[s], -math.inf)
                lse[a:b, j] = torch.logsumexp(z, -1) if length else -math.inf
                p = torch.nan_to_num(torch.softmax(z, -1), 0.0)
                out[a:b, j], mag[a:b, j] = p @ v, p @ v.abs()
                big[a:b, j] = ((x.abs() @ k.abs().T) * abs(scale)).masked_fill(~masks[s], 0).amax(-1) if length else 0.0
    return out, lse, mag, big


def weights(q, lse, cu, lens, table, kc, ks, scale, masks, sums, earlier):
    """sums [pages, heads, page] binary64 in place, and a bound of each sum's relative error that comes from its exponents."""
    hq = q.shape[1]
    heads, page = kc.shape[1], kc.shape[2]
    block, g = page // ks.shape[2], hq // heads
    slack = torch.zeros_like(sums)
    for s, length in enumerate(lens):
        a, b = cu[s], cu[s + 1]
        pages = torch.tensor(table[s][:-(-length // page)], dtype=torch.long, device=q.device)
        key = torch.arange(length, device=q.device)
        at = (pages[key // page], key % page)
        old = max(0, length - (b - a))
        for h in range(heads):
            k = ref.dequantise(kc, ks, pages, block, h, length)
            w = torch.zeros(length, dtype=torch.float64, device=q.device)
            big = w.clone()
            if earlier is not None:
                w[:old] += earlier[at[0][:old], h, at[1][:old]].double()
            for j in range(h * g, (h + 1) * g):
                x = q[a:b, j].double()
                l = lse[a:b, j, None].double()
                z = (x @ k.T * scale - l).masked_fill(~masks[s] | (l == -math.inf), -math.inf)
                p = torch.exp(z)
                w += p.sum(0)
                # an exponent is off by 16 roundings of the sum of magnitudes and four of itself and of lse
                big += (p * (16 * 2.0 ** -23 * (x.abs() @ k.abs().T) * abs(scale) + 6 * 2.0 ** -23 * l.abs().nan_to_num(0, 0, 0) + 2.0 ** -21)).nan_to_num(0).sum(0)
            sums[at[0], h, at[1]] = w
            slack[at[0], h, at[1]] = big + 2.0 ** -24 * (b - a) * g / 8 * w.nan_to_num(0) + 2.0 ** -22 * w.nan_to_num(0) + 1e-37
    return slack


def select(weights_of, lens, keep, sinks, recent):
    """kept (list of lists of lists): weights_of(s, h) [length] binary32."""
    kept = []
    for s, length in enumerate(lens):
        row = []
        for w in weights_of[s]:
            if length <= keep:
                row.append(list(range(length)))
                continue
            w = [-math.inf if math.isnan(x) else x for x in w.tolist()]
            nan = [math.isnan(x) for x in weights_of[s][len(row)].tolist()]
            middle = sorted(range(sinks, length - recent), key=lambda t: (nan[t], -w[t], t))[:keep - sinks - recent]
            row.append(list(range(sinks)) + sorted(middle) + list(range(length - recent, length)))
        kept.append(row)
    return kept


def compact(codes, scales, lists, first, new_lens, table, out_table, page, block):
    """Moves tokens on the CPU, in place: lists[s][h]; reads everything before it writes anything."""
    was_codes, was_scales = codes.clone(), scales.clone()
    value = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double()
    for s, end in enumerate(new_lens):
        f = first[s] if first is not None else 0
        for h in range(codes.shape[1]):
            kept = lists[s][h if len(lists[s]) > 1 else 0]
            where = {}
            for p in range(f // block * block, end):
                if p < f:
                    where[p] = (out_table[s][p // page], p % page)
                else:
                    t = kept[p - f]
                    where[p] = (table[s][t // page], t % page)
            for b0 in range(f // block * block, end, block):
                places = [p for p in range(b0, min(b0 + block, end))]
                target = [(out_table[s][p // page], p % page) for p in places]
                if all(where[p] == t for p, t in zip(places, target)):
                    continue
                rows = torch.stack([value[was_codes[where[p][0], h, where[p][1]].int()] for p in places])
                sc = torch.tensor([int(was_scales[where[p][0], h, where[p][1] // block]) for p in places])
                size = rows.abs().nan_to_num(0.0).amax(1)
                asks = [0 if m == 0 else max(0, ref.ceil_log2(float(m)) - 8 + int(e)) for m, e in zip(size, sc)]
                sb = min(254, max(asks))
                codes_new = (rows * torch.exp2((sc - sb).double())[:, None]).float().to(torch.float8_e4m3fn).view(torch.uint8)
                for (pg, o), c in zip(target, codes_new):
                    codes[pg, h, o] = c
                    scales[pg, h, o // block] = sb
