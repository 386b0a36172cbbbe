"""Plain implementations of the rules on logits and of the cache's weights and evictions, and the tolerances their tests
use. Written from the definitions, in 64 bits, token by token and head by head.
"""
import math

import torch

PROMPT = -2 ** 31


def words_of(bits):
    """bool [..., V] -> int32 [..., ceil(V / 32)]."""
    V = bits.shape[-1]
    n = -(-V // 32)
    full = torch.zeros(*bits.shape[:-1], 32 * n, dtype=torch.int64)
    full[..., :V] = bits.long()
    w = (full.view(*bits.shape[:-1], n, 32) << torch.arange(32)).sum(-1)
    return (w - ((w >> 31) << 32)).to(torch.int32)


def step(x):
    """One operation's result rounded to 32 bits. The operands are 32-bit numbers, so that the 64-bit operation before
    it has more than twice their bits and this rounds as the operation in 32 bits would."""
    return x.float().double()


def changed(z, draft, marked, seen, bias, repetition, frequency, presence, allow):
    """The logits of one request [R, V] (any type) under its rules, as 32-bit values in 64 bits.

    marked bool [V], seen int [V] (PROMPT or times said), bias [V]; draft: a list of R - 1 ids, or []; allow bool [R,
    V] or None. Penalties are numbers or None."""
    z = z.double()
    R, V = z.shape
    seen = torch.where(marked, seen.long(), torch.zeros_like(seen.long()))
    out = torch.empty_like(z)
    for j in range(R):
        times = seen & 0x7fffffff
        for x in draft[:j]:
            if 0 <= x < V:
                times[x] += 1
        x = z[j].clone()
        if repetition is not None:
            rho = torch.tensor(repetition).double()
            known = (times > 0) | (seen < 0)
            x = torch.where(known, torch.where(x > 0, step(x / rho), step(x * rho)), x)
        if frequency is not None:
            x = torch.where(times > 0, step(x - step(times.double() * torch.tensor(frequency).double())), x)
        if presence is not None:
            x = torch.where(times > 0, step(x - torch.tensor(presence).double()), x)
        x = torch.where(marked, step(x + bias.double()), x)
        if allow is not None:
            x = torch.where(allow[j], x, torch.full_like(x, -math.inf))
        out[j] = x
    return out


def weighed(q, lse, k, table, kv_len, new_len, path, scale, decay, before):
    """q [B, T, Hq, D], k [pages, page, Hkv, D], before [B, Hkv, width]. Returns the weights in 64 bits (NaN where
    nothing is written) and the bound on what 32-bit arithmetic is off by.

    A score is a sum of D products in 32 bits, each within D + 2 units of the products' sizes; it is scaled and the lse
    taken off in numbers no larger than theirs (four roundings); the exponential has two units of its own (2^-22); a sum
    of n terms adds n units; the weight before is scaled and added with a rounding each."""
    B, T, Hq, D = q.shape
    page, Hkv = k.shape[1], k.shape[2]
    G, u = Hq // Hkv, 2.0 ** -24
    out = torch.full(before.shape, math.nan, dtype=torch.float64)
    tol = torch.zeros_like(out)
    for b in range(B):
        ctx = int(kv_len[b])
        rows = T if path is None else path.shape[1]
        n = rows if new_len is None else int(new_len[b])
        if n == 0:
            continue
        slots = torch.arange(ctx + n)
        keys = k[table[b].long()[slots // page], slots % page].double()  # [slots, Hkv, D]
        for h in range(Hkv):
            total, off = torch.zeros(ctx + n, dtype=torch.float64), torch.zeros(ctx + n, dtype=torch.float64)
            for i in range(n):
                t = i if path is None else int(path[b, i])
                if not 0 <= t < T:
                    continue
                for g in range(h * G, (h + 1) * G):
                    x, sees = q[b, t, g].double(), ctx + i + 1
                    ref = float(lse[b, t, g])
                    if math.isinf(ref):
                        continue
                    z = keys[:sees, h] @ x * scale
                    reach = keys[:sees, h].abs() @ x.abs() * abs(scale)
                    p = torch.exp(z - ref)
                    total[:sees] += p
                    off[:sees] += p * ((D + 2) * u * reach + 4 * u * (z.abs() + abs(ref)) + 2.0 ** -22)
            was = torch.zeros(ctx + n, dtype=torch.float64)
            if decay:
                was[:ctx] = before[b, h, :ctx].double() * decay
            out[b, h, :ctx + n] = total + was
            tol[b, h, :ctx + n] = 1.01 * off + (n * G + 2) * u * (total + was.abs()) + 1e-37
    return out, tol


def evicted(k, v, table, kv_len, weight, keep, first, last):
    """k, v [layers, pages, page, heads, D], weight [layers, B, heads, width]: copies after the eviction, and the new
    lengths. weight past the new end is left."""
    k, v, weight = k.clone(), v.clone(), weight.clone()
    layers, page, heads = k.shape[0], k.shape[2], k.shape[3]
    new = []
    for b in range(table.shape[0]):
        ctx = int(kv_len[b])
        n = min(int(keep[b]), ctx)
        f = min(first, n)
        r = min(last, n - f)
        new.append(n)

        def place(slot):
            return int(table[b, slot // page]), slot % page
        for layer in range(layers):
            for h in range(heads):
                w = [float(x) for x in weight[layer, b, h, :ctx]]
                middle = sorted(range(f, ctx - r), key=lambda s: (-math.inf if math.isnan(w[s]) else w[s], -s),
                                reverse=True)
                stay = set(range(f)) | set(range(ctx - r, ctx)) | set(middle[:n - f - r])
                src = [s for s in range(n, ctx) if s in stay]
                dst = [s for s in range(n) if s not in stay]
                assert len(src) == len(dst)
                for s, d in zip(src, dst):
                    for x in (k, v):
                        x[(layer, *place(d), h)] = x[(layer, *place(s), h)]
                    weight[layer, b, h, d] = weight[layer, b, h, s]
    return k, v, weight, torch.tensor(new, dtype=torch.int32)
