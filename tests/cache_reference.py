"""Plain 64-bit implementations of the cache operators, in elementary torch operations, and the tolerances their
tests use.

Written from the definitions: token by token, head by head, no shared code with the library.
"""
import math

import torch

# half the spacing of the numbers next to 1: what a rounding to the type is off by at most, relatively
UNIT = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}


def slot_place(table_row, slot, page):
    return int(table_row[slot // page]), slot % page


def sees_matrix(n, mask_row_words, T):
    """[n, n] bool: new token t sees new token u."""
    m = torch.zeros(n, n, dtype=torch.bool)
    for t in range(n):
        for u in range(n):
            m[t, u] = u <= t if mask_row_words is None else bool((int(mask_row_words[t][u // 32]) >> (u % 32)) & 1)
    return m


def attention(q, k, v, table, kv_len, new_len, mask, scale):
    """q [B, T, Hq, D], k, v [pages, page, Hkv, D] (any type). Returns out, lse and the tolerance's two
    magnitudes per row: the weighted sum of |v| and the largest sum of |q_d k_d| * scale, all in 64 bits."""
    B, T, Hq, D = q.shape
    page, Hkv = k.shape[1], k.shape[2]
    G = Hq // Hkv
    dev = q.device
    out = torch.zeros(B, T, Hq, D, dtype=torch.float64, device=dev)
    lse = torch.full((B, T, Hq), -math.inf, dtype=torch.float64, device=dev)
    weight = torch.zeros(B, T, Hq, D, dtype=torch.float64, device=dev)
    reach = torch.zeros(B, T, Hq, dtype=torch.float64, device=dev)
    for b in range(B):
        ctx, n = int(kv_len[b]), int(new_len[b]) if new_len is not None else T
        if n == 0:
            continue
        places = [slot_place(table[b], s, page) for s in range(ctx + n)]
        pid, off = torch.tensor([p for p, _ in places]), torch.tensor([o for _, o in places])
        kk, vv = k[pid, off].double(), v[pid, off].double()  # [ctx + n, Hkv, D]
        tree = sees_matrix(n, None if mask is None else mask[b], T)
        sees = torch.cat([torch.ones(n, ctx, dtype=torch.bool), tree], 1)
        for t in range(n):
            at = sees[t].nonzero().flatten().to(dev)
            if at.numel() == 0:
                continue
            for h in range(Hkv):  # the group's G query heads at once
                x = q[b, t, h * G:(h + 1) * G].double()
                key, val = kk[at, h], vv[at, h]
                z = (x @ key.T) * scale
                w = torch.exp(z - z.max(1, keepdim=True).values)
                w = w / w.sum(1, keepdim=True)
                heads = slice(h * G, (h + 1) * G)
                out[b, t, heads] = w @ val
                lse[b, t, heads] = torch.logsumexp(z, 1)
                weight[b, t, heads] = w @ val.abs()
                reach[b, t, heads] = ((x.abs() @ key.abs().T) * abs(scale)).max(1).values
    return out, lse, weight, reach


def attention_tolerance(dtype, D, slots, weight, reach, out, vmax):
    """Elementwise bound on |out - reference|. Scores are sums of D products in 32 bits (each within D + 2 units of
    the sum of the products' sizes); a softmax weight moves by twice a score's error, by the exponential's few units
    and by its rounding to a 16-bit type; sums of `slots` terms add a unit each; the result is rounded once.
    16-bit weights under the type's normal range (2^-14 of the largest for float16) are off by half its spacing."""
    u = 2.0 ** -24
    rel = 2 * (D + 2) * u * reach[..., None] + 2.0 ** -21 + slots * u
    tol = rel * weight + UNIT[dtype] * out.abs() + 1e-30
    if dtype != torch.float32:
        tol = tol + UNIT[dtype] * weight
    if dtype == torch.float16:
        tol = tol + 2.0 ** -24 + slots * 2.0 ** -25 * vmax
    return tol


def lse_tolerance(D, slots, reach, lse):
    u = 2.0 ** -24
    return (D + 2) * u * reach + 2.0 ** -21 + slots * u + lse.abs().nan_to_num(0, 0, 0) * 2.0 ** -21


def turned(x, w, eps, cos, sin, pos, rot, interleaved):
    """Norm and rotation of one head's row x [D] in 64 bits."""
    x = x.double()
    D = x.numel()
    if w is not None:
        x = x / math.sqrt(float((x * x).sum()) / D + eps) * w.double()
    y = x.clone()
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        c, s = float(cos[pos, i]), float(sin[pos, i])
        y[a], y[b] = x[a] * c - x[b] * s, x[b] * c + x[a] * s
    return y


def append_tolerance(dtype, D, x, w, y):
    """Elementwise bound on |appended - reference| for a row: the norm's sum of D squares, its root and division and
    the rotation's three operations in 32 bits, relative to the largest element that goes into one; one rounding."""
    u = 2.0 ** -24
    big = float(y.abs().max()) * math.sqrt(2.0)
    return UNIT[dtype] * y.abs() + (D + 16) * u * big + (2.0 ** -24 if dtype == torch.float16 else 1e-30)
