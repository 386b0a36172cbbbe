"""Cases of the serving operators around a verified block: appending to a paged cache, attending to it, compacting it.

A decoding round feeds every request's drafted tokens (a chain or a tree, the pending token first) through the target
model. Per layer the keys and values of those tokens go into a paged cache (``asd.kv_append``: norms of queries and
keys per head, position rotation, scatter to pages), and every token attends to its request's context and to its own
ancestors in the tree (``asd.tree_attention``). Once a path has been verified, its keys and values move next to the
context (``asd.kv_compact``).

``run`` takes the plain forms, in elementary torch operations in 32 bits, or with ``own`` the framework's calls.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-6


# ---------------------------------------------------------------- cases

def _attend(name, dtype, B, T, Hq, Hkv, D, ctx, page, chain=False, ragged=False):
    return {"name": name, "op": "attend", "dtype": dtype, "B": B, "T": T, "Hq": Hq, "Hkv": Hkv, "D": D, "ctx": ctx,
            "page": page, "chain": chain, "ragged": ragged}


def _append(name, dtype, B, T, Hq, Hkv, D, rot, ctx, page, norm, interleaved=False, ragged=False):
    return {"name": name, "op": "append", "dtype": dtype, "B": B, "T": T, "Hq": Hq, "Hkv": Hkv, "D": D, "rot": rot,
            "ctx": ctx, "page": page, "norm": norm, "interleaved": interleaved, "ragged": ragged}


def _compact(name, dtype, B, T, P, layers, Hkv, D, ctx, page):
    return {"name": name, "op": "compact", "dtype": dtype, "B": B, "T": T, "P": P, "layers": layers, "Hkv": Hkv,
            "D": D, "ctx": ctx, "page": page}


def listed():
    return [
        # one request decoding one token after a short prompt: latency
        _attend("attend-one-token", "bf16", 1, 1, 40, 8, 128, 700, 64, chain=True),
        # the verify step's batch: 32 requests, a pending token and 8 drafts each, contexts of some thousand tokens
        _attend("attend-chain-b32", "bf16", 32, 9, 40, 8, 128, 8000, 64, chain=True),
        # one long conversation, single tokens: the long axis has to be split
        _attend("attend-long-single", "bf16", 1, 1, 40, 8, 128, 250000, 128, chain=True),
        # wide trees over long documents, small pages: as many operations as bytes
        _attend("attend-tree-long", "bf16", 4, 61, 40, 8, 128, 90000, 16),
        # many short chats with narrow heads, odd pages, requests that drafted less than the others
        _attend("attend-many-short", "f16", 160, 5, 32, 4, 64, 577, 48, ragged=True),
        # a model kept in 32 bits (a small draft model): odd pages, trees
        _attend("attend-f32-tree", "f32", 8, 17, 16, 4, 96, 2900, 24, ragged=True),
        # one decoding step of one request: latency
        _append("append-one-token", "bf16", 1, 1, 40, 8, 128, 128, 700, 64, True),
        # the verify step's batch, requests that drafted less than the others
        _append("append-chain-b32", "bf16", 32, 9, 40, 8, 128, 128, 4000, 64, True, ragged=True),
        # prompts entering the cache
        _append("append-prompts", "bf16", 8, 4093, 40, 8, 128, 128, 100, 64, True),
        # 32-bit model, part of each head rotated, neighbouring pairs, no norms
        _append("append-f32-partial", "f32", 6, 701, 16, 4, 96, 32, 900, 24, False, interleaved=True, ragged=True),
        # one request's accepted path, all layers
        _compact("compact-one", "bf16", 1, 33, 6, 40, 8, 128, 700, 64),
        # the verify step's batch, all layers
        _compact("compact-b32", "bf16", 32, 61, 9, 40, 8, 128, 300, 16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "append", "append", "compact"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    Hkv = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 2, 4, 5, 8])
    D = rng.choice([64, 80, 96, 128, 128])
    page = rng.choice([5, 16, 24, 32, 64, 128, 256])
    token = Hkv * D * BYTES[dtype] * 2  # bytes of a cached token
    if op == "attend":
        B, T = _log(rng, 1, 160), _log(rng, 1, 61)
        most = 0.9e9 / (B * token)                                        # bytes of all contexts
        most = min(most, (2e10 if dtype == "f32" else 2e11) / (4 * B * T * G * Hkv * D))  # operations
        ctx = _log(rng, 1, max(2, min(120000, int(most))))
        return _drop_name(_attend("", dtype, B, T, G * Hkv, Hkv, D, ctx, page, chain=rng.random() < 0.4,
                                  ragged=rng.random() < 0.5))
    if op == "append":
        B = _log(rng, 1, 64)
        T = _log(rng, 1, max(2, min(4000, int(2.5e8 / (B * token * (G + 2))))))
        rot = rng.choice([D, D, D // 2])
        return _drop_name(_append("", dtype, B, T, G * Hkv, Hkv, D, rot, _log(rng, 1, 3000), page, rng.random() < 0.6,
                                  interleaved=rng.random() < 0.4, ragged=rng.random() < 0.5))
    B, P = _log(rng, 1, 64), rng.randint(2, 9)
    return _drop_name(_compact("", dtype, B, rng.randint(2 * P, 64), P, _log(rng, 1, 40), Hkv, D, _log(rng, 1, 300),
                               page))


def _drop_name(case):
    del case["name"]
    return case


def _lens(case):
    """The requests' context lengths: spread from a quarter of the longest to the longest, one of several empty."""
    B, ctx = case["B"], case["ctx"]
    n = [ctx if B == 1 else ctx - (3 * ctx * i) // (4 * (B - 1)) for i in range(B)]
    if case.get("ragged") and B > 2:
        n[B // 2] = 0
    return n


def _news(case):
    """How many of the T tokens each request has; with "ragged", fewer in some and none in one of several."""
    B, T = case["B"], case["T"]
    if not case.get("ragged"):
        return [T] * B
    return [0 if B > 3 and i == 1 else T - (i % 3) * T // 4 for i in range(B)]


def _path_lens(case):
    return [case["P"] if i % 4 != 3 else max(1, case["P"] // 2) for i in range(case["B"])]


def work(case):
    es, D, Hkv, B, T = BYTES[case["dtype"]], case["D"], case["Hkv"], case["B"], case["T"]
    token = 2 * Hkv * D * es
    if case["op"] == "attend":
        pairs = list(zip(_lens(case), _news(case)))
        kv = sum(c + n for c, n in pairs)
        rows = sum(n for _, n in pairs) * case["Hq"]
        byt = kv * token + rows * D * es + B * T * case["Hq"] * (D * es + 4) + -(-kv // case["page"]) * 4
        if not case["chain"]:
            byt += B * T * -(-T // 32) * 4
        return {"bytes": byt, "flops": sum(4 * D * case["Hq"] * n * (c + (n + 1) / 2) for c, n in pairs)}
    if case["op"] == "append":
        n = sum(_news(case))
        heads = case["Hq"] + 2 * Hkv
        # the queries and keys and values in and out, a row of cosines and sines a token, its position
        byt = n * (2 * heads * D * es + case["rot"] * 4 + 4) + (2 * D * es if case["norm"] else 0)
        return {"bytes": byt, "flops": n * (case["Hq"] + Hkv) * (3 * case["rot"] + (4 * D if case["norm"] else 0))}
    moved = sum(n - 1 for n in _path_lens(case)) * case["layers"]
    return {"bytes": 2 * moved * token + B * (case["P"] + 2) * 4, "flops": 0}


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _randn_in(dtype, g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=dtype)


def _shuffled(values, g):
    t = torch.tensor(values, dtype=torch.int32, device="cuda")
    return t[torch.randperm(len(values), generator=g, device="cuda")]


def _pages(B, tokens, page, g):
    """A page table [B, n]: every request's pages, scattered over the cache."""
    n = -(-tokens // page)
    return torch.randperm(B * n, generator=g, device="cuda").to(torch.int32).view(B, n).contiguous()


def _tree(B, T, g):
    """Random trees in topological order: parents [B, T] (the root's is -1), depths, and ancestors-or-self as bits."""
    u = torch.rand(B, T, generator=g, device="cuda")
    t = torch.arange(T, device="cuda")
    back = 1 + (u * u * torch.clamp(t, min=1, max=12)).long()
    parent = torch.where(t > 0, torch.clamp(t - back, min=0), -1).expand(B, T).contiguous()
    sees = torch.eye(T, dtype=torch.bool, device="cuda").expand(B, T, T).clone()
    depth = torch.zeros(B, T, dtype=torch.int32, device="cuda")
    rows = torch.arange(B, device="cuda")
    for i in range(1, T):
        p = parent[:, i]
        sees[:, i] |= sees[rows, p]
        depth[:, i] = depth[rows, p] + 1
    words = -(-T // 32)
    bits = torch.zeros(B, T, words * 32, dtype=torch.int64, device="cuda")
    bits[:, :, :T] = sees.long()
    w = (bits.view(B, T, words, 32) << torch.arange(32, device="cuda")).sum(-1)
    return depth, (w - ((w >> 31) << 32)).to(torch.int32).contiguous()


def prepare(case, seed):
    g = _gen(seed)
    B, T, Hkv, D, page, ctx = (case[k] for k in ("B", "T", "Hkv", "D", "page", "ctx"))
    dt = DTYPES[case["dtype"]]
    table = _pages(B, ctx + T, page, g)
    pages = table.numel()
    s = {"case": case, "table": table}
    layers = case.get("layers")
    shape = (pages, page, Hkv, D) if layers is None else (layers, pages, page, Hkv, D)
    s["k"], s["v"] = _randn_in(dt, g, *shape), _randn_in(dt, g, *shape)
    # the requests of a batch come in no order: contexts and token counts are shuffled together
    order = torch.randperm(B, generator=g, device="cuda")
    s["kv_len"] = torch.tensor(_lens(case), dtype=torch.int32, device="cuda")[order]
    if case["op"] == "compact":
        n = case["P"]
        s["path_len"] = _shuffled(_path_lens(case), g)
        # ascending node numbers: the root, which stays where it is, then nodes that lie further on than they will
        pick = torch.rand(B, T - 2, generator=g, device="cuda").argsort(1)[:, :n - 1].sort(1).values + 2
        s["path"] = torch.cat([torch.zeros(B, 1, dtype=torch.int64, device="cuda"), pick], 1).to(torch.int32)
    else:
        s["new_len"] = torch.tensor(_news(case), dtype=torch.int32, device="cuda")[order] if case["ragged"] else None
        Hq = case["Hq"]
    if case["op"] == "attend":
        # scores of an attention that looks at some tokens more than at others
        s["q"] = (_randn(g, B, T, Hq, D) * 1.5).to(dt)
        s["mask"] = None if case["chain"] else _tree(B, T, g)[1]
        s["scale"] = 1.0 / math.sqrt(D)
        s["out"] = torch.empty(B, T, Hq, D, dtype=dt, device="cuda")
        s["lse"] = torch.empty(B, T, Hq, dtype=torch.float32, device="cuda")
    elif case["op"] == "append":
        qkv = _randn(g, B, T, Hq + 2 * Hkv, D).to(dt)  # the rows that a fused projection writes
        s["q"], s["knew"], s["vnew"] = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
        s["pos"] = (s["kv_len"][:, None] + torch.arange(T, dtype=torch.int32, device="cuda")).contiguous()
        if T <= 61:  # drafted trees; longer inputs are prompts
            s["pos"] = (s["kv_len"][:, None] + _tree(B, T, g)[0]).contiguous()
        inv = 10000.0 ** (-torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / case["rot"])
        angle = torch.arange(ctx + T, device="cuda", dtype=torch.float64)[:, None] * inv
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        s["qw"] = (1 + 0.2 * _randn(g, D)).to(dt) if case["norm"] else None
        s["kw"] = (1 + 0.2 * _randn(g, D)).to(dt) if case["norm"] else None
        s["q_out"] = torch.zeros(B, T, Hq, D, dtype=dt, device="cuda")
    if own:
        from paper_2608_03447_gb300 import asd
        s["cache"] = asd.KVCache(s["k"], s["v"], table)
        if case["op"] == "attend":
            s["ws"] = asd.attention_workspace(s["cache"], T, Hq)
            s["o"] = {"out": s["out"], "lse": s["lse"]}
    return s


# ---------------------------------------------------------------- the operators

def run(s):
    op = s["case"]["op"]
    if own:
        return _run_own(s, op)
    return {"attend": _plain_attend, "append": _plain_append, "compact": _plain_compact}[op](s)


def _run_own(s, op):
    from paper_2608_03447_gb300 import asd
    if op == "attend":
        return asd.tree_attention(s["q"], s["cache"], s["kv_len"], tree_mask=s["mask"], new_len=s["new_len"],
                                  scale=s["scale"], workspace=s["ws"], out=s["o"])
    if op == "append":
        q = asd.kv_append(s["knew"], s["vnew"], s["cache"], s["kv_len"], q=s["q"], q_out=s["q_out"],
                          positions=s["pos"], new_len=s["new_len"], cos=s["cos"], sin=s["sin"],
                          interleaved=s["case"]["interleaved"], q_norm=s["qw"], k_norm=s["kw"], eps=EPS)
        return {"q": q, "k": s["k"], "v": s["v"]}
    asd.kv_compact(s["cache"], s["kv_len"], s["path"], s["path_len"])
    return {"k": s["k"], "v": s["v"]}


def _plain_attend(s):
    c = s["case"]
    B, T, Hq, Hkv, D = c["B"], c["T"], c["Hq"], c["Hkv"], c["D"]
    G, S = Hq // Hkv, s["table"].shape[1] * c["page"]
    at = s["table"].long()
    k = s["k"][at].view(B, S, Hkv, D).permute(0, 2, 3, 1).float()
    v = s["v"][at].view(B, S, Hkv, D).permute(0, 2, 1, 3).float()
    q = s["q"].float().view(B, T, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, D)
    n = s["new_len"].long() if s["new_len"] is not None else torch.full((B,), T, device="cuda")
    t = torch.arange(T, device="cuda")
    # which drafted tokens a token sees, and where they lie
    u = torch.arange(S, device="cuda")[None] - s["kv_len"].long()[:, None]          # [B, S]
    uc = u.clamp(0, T - 1)
    if s["mask"] is None:
        sees = t[None, :, None] >= uc[:, None, :]
    else:
        word = torch.gather(s["mask"].long(), 2, (uc // 32)[:, None, :].expand(B, T, S))
        sees = ((word >> (uc % 32)[:, None, :]) & 1).bool()
    sees = (sees | (u < 0)[:, None, :]) & (u < n[:, None])[:, None, :] & (t[None, :] < n[:, None])[:, :, None]
    z = (q @ k) * s["scale"]
    z = z.view(B, Hkv, T, G, S).masked_fill_(~sees[:, None, :, None, :], -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = (z - top).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.view(B, Hkv, T * G, S) @ v).view(B, Hkv, T, G, D) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + total.log()).squeeze(-1)
    s["out"].copy_(o.permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D))
    s["lse"].copy_(lse.permute(0, 2, 1, 3).reshape(B, T, Hq))
    return {"out": s["out"], "lse": s["lse"]}


def _plain_turn(x, w, s, c):
    """Norm per head and rotation of x [B, T, H, D], in 32 bits."""
    x = x.float()
    if w is not None:
        x = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * w.float()
    rot = c["rot"]
    pos = s["pos"].long()
    cos, sin = s["cos"][pos][:, :, None, :], s["sin"][pos][:, :, None, :]
    r, rest = x[..., :rot], x[..., rot:]
    if c["interleaved"]:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = r[..., :rot // 2], r[..., rot // 2:]
        r = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([r, rest], -1)


def _plain_append(s):
    c = s["case"]
    B, T, page = c["B"], c["T"], c["page"]
    n = s["new_len"].long() if s["new_len"] is not None else torch.full((B,), T, device="cuda")
    t = torch.arange(T, device="cuda")
    has = t[None] < n[:, None]
    dt = s["k"].dtype
    s["q_out"][has] = _plain_turn(s["q"], s["qw"], s, c)[has].to(dt)
    slot = s["kv_len"].long()[:, None] + t
    row = (s["table"].long().gather(1, slot // page) * page + slot % page)[has]
    s["k"].view(-1, c["Hkv"], c["D"])[row] = _plain_turn(s["knew"], s["kw"], s, c)[has].to(dt)
    s["v"].view(-1, c["Hkv"], c["D"])[row] = s["vnew"][has]
    return {"q": s["q_out"], "k": s["k"], "v": s["v"]}


def _plain_compact(s):
    c = s["case"]
    i = torch.arange(c["P"], device="cuda")
    keep = i[None] < s["path_len"].long()[:, None]

    def row(slot):
        return (s["table"].long().gather(1, slot // c["page"]) * c["page"] + slot % c["page"])[keep]
    base = s["kv_len"].long()[:, None]
    src, dst = row(base + s["path"].long()), row(base + i)
    k, v = (x.view(c["layers"], -1, c["Hkv"], c["D"]) for x in (s["k"], s["v"]))
    k[:, dst], v[:, dst] = k[:, src], v[:, src]
    return {"k": s["k"], "v": s["v"]}


# ---------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attend":
        return _exact_attend(s, case)
    if case["op"] == "append":
        return _exact_append(s, case)
    return _exact_compact(s, case)


def _exact_attend(s, c):
    """Request by request, kv head by kv head, over the tokens that exist."""
    B, T, Hq, Hkv, D = c["B"], c["T"], c["Hq"], c["Hkv"], c["D"]
    G = Hq // Hkv
    out = torch.zeros(B, T, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.full((B, T, Hq), -math.inf, dtype=torch.float64, device="cuda")
    lens = s["kv_len"].tolist()
    news = s["new_len"].tolist() if s["new_len"] is not None else [T] * B
    mask = s["mask"].tolist() if s["mask"] is not None else None
    for b in range(B):
        ctx, n = lens[b], news[b]
        if n == 0:
            continue
        last = ctx + n
        ids = s["table"][b, :-(-last // c["page"])].long()
        sees = torch.ones(n, last, dtype=torch.bool)
        for t in range(n):
            for u in range(n):
                sees[t, ctx + u] = u <= t if mask is None else bool((mask[b][t][u // 32] >> (u % 32)) & 1)
        sees = sees.cuda()
        for h in range(Hkv):
            k = s["k"][ids, :, h].reshape(-1, D)[:last].double()
            v = s["v"][ids, :, h].reshape(-1, D)[:last].double()
            q = s["q"][b, :n, h * G:(h + 1) * G].double()
            z = torch.einsum("tgd,sd->tgs", q, k) / math.sqrt(D)
            z = torch.where(sees[:, None, :], z, torch.full_like(z, -math.inf))
            lse[b, :n, h * G:(h + 1) * G] = torch.logsumexp(z, -1)
            out[b, :n, h * G:(h + 1) * G] = torch.einsum("tgs,sd->tgd", torch.softmax(z, -1), v)
    return {"out": out, "lse": lse}


def _exact_append(s, c):
    B, T, D, rot, page = c["B"], c["T"], c["D"], c["rot"], c["page"]
    lens = s["kv_len"].tolist()
    news = s["new_len"].tolist() if s["new_len"] is not None else [T] * B

    def turned(x, w, b, n):
        x = x[b, :n].double()
        if w is not None:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / D + EPS) * w.double()
        y = x.clone()
        at = s["pos"][b, :n].long()
        for i in range(rot // 2):
            lo, hi = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + rot // 2)
            cs, sn = s["cos"][at, i].double()[:, None], s["sin"][at, i].double()[:, None]
            y[..., lo] = x[..., lo] * cs - x[..., hi] * sn
            y[..., hi] = x[..., hi] * cs + x[..., lo] * sn
        return y

    q = torch.zeros(s["q_out"].shape, dtype=torch.float64, device="cuda")
    k, v = s["k"].double(), s["v"].double()
    for b in range(B):
        n = news[b]
        if n == 0:
            continue
        q[b, :n] = turned(s["q"], s["qw"], b, n)
        slots = torch.arange(lens[b], lens[b] + n, device="cuda")
        pages, places = s["table"][b].long()[slots // page], slots % page
        k[pages, places] = turned(s["knew"], s["kw"], b, n)
        v[pages, places] = s["vnew"][b, :n].double()
    return {"q": q, "k": k, "v": v}


def _exact_compact(s, c):
    """Node by node: each goes where its place on the path says."""
    page, after = c["page"], {"k": s["k"].double(), "v": s["v"].double()}
    for b, (start, n) in enumerate(zip(s["kv_len"].tolist(), s["path_len"].tolist())):
        row = s["table"][b].tolist()
        for i, node in enumerate(s["path"][b].tolist()[:n]):
            src, dst = start + node, start + i
            for name, x in after.items():
                x[:, row[dst // page], dst % page] = s[name][:, row[src // page], src % page].double()
    return after
