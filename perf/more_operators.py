"""Cases of the operators that hold a round to a request's rules and its cache to a budget.

Rules: what a request's own text (repetition, frequency and presence penalties), its caller (a bias per token) and its
grammar (tokens that may not come next) do to the logits of a draft block. Row j of a block has seen the drafts before
it. ``asd.rules_verify`` verifies a block under them, ``asd.rules_logits`` writes the changed logits for whoever samples,
``asd.tokens_record`` keeps the token counts that they read.

Eviction: ``asd.kv_weigh`` adds up the attention weight that every cached slot gets, ``asd.kv_evict`` keeps the heaviest
slots of every key/value head, between the first ones and the newest, and moves them into the places of those that go.

``run`` takes the plain forms, in elementary torch operations in 32 bits, or with ``own`` the framework's calls.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
GATE, CAP, BUDGET = 1.0, 2, 8.0
PROMPT = -2 ** 31  # of a record's first word: the token is in the prompt


# ---------------------------------------------------------------- cases

def _verify(name, dtype, B, K, V, said, biased, grammar):
    return {"name": name, "op": "verify", "dtype": dtype, "B": B, "K": K, "V": V, "said": said, "biased": biased,
            "grammar": grammar}


def _logits(name, dtype, B, K, V, said, biased, grammar):
    return {**_verify(name, dtype, B, K, V, said, biased, grammar), "op": "logits"}


def _record(name, B, n, V, said, prompt):
    return {"name": name, "op": "record", "B": B, "n": n, "V": V, "said": said, "prompt": prompt}


def _weigh(name, dtype, B, T, Hq, Hkv, D, ctx, page, decay, path=False):
    return {"name": name, "op": "weigh", "dtype": dtype, "B": B, "T": T, "Hq": Hq, "Hkv": Hkv, "D": D, "ctx": ctx,
            "page": page, "decay": decay, "path": path}


def _evict(name, dtype, layers, B, Hkv, D, ctx, page, keep, first, last):
    return {"name": name, "op": "evict", "dtype": dtype, "layers": layers, "B": B, "Hkv": Hkv, "D": D, "ctx": ctx,
            "page": page, "keep": keep, "first": first, "last": last}


def listed():
    return [
        # one conversation, a block of 8 drafts, under a grammar (a reply in a fixed format): latency
        _verify("verify-one", "bf16", 1, 8, 151936, 900, 0, True),
        # the verify step's batch: 32 requests with some thousand tokens of text each, biases and grammars
        _verify("verify-b32", "bf16", 32, 8, 151936, 4000, 300, True),
        # one request that samples token by token: latency
        _logits("logits-one", "f32", 1, 0, 32000, 300, 0, False),
        # a batch of short blocks in 32 bits whose caller samples: penalties and biases, no grammars
        _logits("logits-b64-f32", "f32", 64, 4, 129280, 2000, 300, False),
        # what a round has emitted, padded with -1: latency
        _record("record-commit", 32, 9, 151936, 1000, False),
        # the prompts of a batch that begins
        _record("record-prompts", 64, 8000, 151936, 0, True),
        # one request, one token: latency
        _weigh("weigh-one-token", "bf16", 1, 1, 40, 8, 128, 4200, 64, 1.0),
        # the verify step's batch: the rows of each tree's accepted path
        _weigh("weigh-chain-b32", "bf16", 32, 9, 40, 8, 128, 8000, 64, 0.97, path=True),
        # the last 64 tokens of long prompts say what of them will be needed: narrow heads, odd pages
        _weigh("weigh-window", "f16", 16, 64, 32, 4, 64, 12000, 48, 0.0),
        # a model kept in 32 bits
        _weigh("weigh-f32", "f32", 8, 17, 16, 4, 96, 2900, 24, 1.0),
        # one conversation over its budget by 128 tokens, all layers
        _evict("evict-one", "bf16", 40, 1, 8, 128, 4224, 64, 4096, 4, 128),
        # prompts cut to a quarter of their length
        _evict("evict-prompts", "bf16", 4, 8, 8, 128, 16000, 16, 4000, 4, 64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["verify", "verify", "logits", "record", "weigh", "weigh", "evict"])
    if op in ("verify", "logits"):
        dtype, B, K = rng.choice(["bf16", "bf16", "f32"]), _log(rng, 1, 128), rng.randint(0, 16)
        most = 80e6 / (B * (K + 1) * BYTES[dtype])
        V = rng.choice([1024, 32000, 32001, 50257, 129280, 151936])
        if V > most:
            V = _log(rng, min(1000, int(most)), int(most))
        said, biased = _log(rng, 1, 5000), rng.choice([0, 0, 20, 300])
        case = (_verify if op == "verify" else _logits)("", dtype, B, K, V, min(said, V), min(biased, V // 4),
                                                        rng.random() < 0.5)
    elif op == "record":
        prompt = rng.random() < 0.5
        n = _log(rng, 1, 8000) if prompt else _log(rng, 1, 32)
        case = _record("", _log(rng, 1, 64), n, rng.choice([32001, 129280, 151936]), rng.randint(0, 500), prompt)
    else:
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        Hkv, G, D = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 80, 96, 128, 128])
        page, es = rng.choice([5, 16, 24, 32, 64, 128, 256]), BYTES[dtype]
        if op == "weigh":
            B, T = _log(rng, 1, 64), _log(rng, 1, 70)
            most = min(4e8 / (B * Hkv * D * es), (5e9 if dtype == "f32" else 4e10) / (2 * B * T * G * Hkv * D),
                       4e8 / (B * T * G * Hkv))
            ctx = _log(rng, 1, max(2, min(60000, int(most))))
            case = _weigh("", dtype, B, T, G * Hkv, Hkv, D, ctx, page, rng.choice([0.0, 1.0, 0.9]), rng.random() < 0.4)
        else:
            layers, B = _log(rng, 1, 40), _log(rng, 1, 32)
            most = 4e8 / (layers * B * Hkv * D * es)
            ctx = _log(rng, min(100, int(most)), max(101, min(30000, int(most))))
            keep = max(1, int(ctx * rng.choice([0.25, 0.5, 0.9, 0.97])))
            case = _evict("", dtype, layers, B, Hkv, D, ctx, page, keep, rng.choice([0, 4]),
                          rng.choice([0, 16, min(64, ctx // 8)]))
    del case["name"]
    return case


def _words(V):
    return -(-V // 32)


def _lens(case):
    """The requests' context lengths: spread from three quarters of the longest to the longest."""
    B, ctx = case["B"], case["ctx"]
    return [ctx if B == 1 else ctx - (ctx * i) // (4 * (B - 1)) for i in range(B)]


def _news(case):
    """How many of a path's T rows each request has."""
    B, T = case["B"], case["T"]
    return [max(1, T - (i % 4) * T // 4) if case["path"] else T for i in range(B)]


def work(case):
    B = case["B"]
    if case["op"] in ("verify", "logits"):
        K, V, es = case["K"], case["V"], BYTES[case["dtype"]]
        logits = B * (K + 1) * V * es
        # a bit a token and the records of those that have one, once a request; the grammar's bits, once a row
        byt = logits + B * (_words(V) * 4 + (case["said"] + case["biased"]) * 8) + B * K * 4
        byt += B * (K + 1) * _words(V) * 4 if case["grammar"] else 0
        byt += logits if case["op"] == "logits" else B * (4 * (K + 1) * 2 + 4 * K + 12 + 16)
        return {"bytes": byt, "flops": B * (K + 1) * V}
    if case["op"] == "record":
        tokens = sum(_counts(case))
        return {"bytes": tokens * (4 + 8 + 8) + B * 4, "flops": 0}
    Hkv, D, es = case["Hkv"], case["D"], BYTES[case["dtype"]]
    if case["op"] == "weigh":
        pairs = list(zip(_lens(case), _news(case)))
        kv, rows = sum(c + n for c, n in pairs), sum(n for _, n in pairs) * case["Hq"]
        byt = kv * Hkv * D * es + kv * Hkv * 4 + rows * (D * es + 4) + -(-kv // case["page"]) * 4
        byt += sum(c for c, _ in pairs) * Hkv * 4 if case["decay"] else 0
        return {"bytes": byt, "flops": sum(2 * D * case["Hq"] * n * (c + (n + 1) / 2) for c, n in pairs)}
    byt = 0
    for c in _lens(case):
        n = min(c, case["keep"])
        last = min(case["last"], n - min(case["first"], n))
        # what cannot be told from the sizes: how many of the heaviest lie past the new end; their share of the places
        moved = min(c - n, last + int((n - last) * max(0, c - n - last) / c))
        byt += case["layers"] * Hkv * (c * 4 + moved * 4 * D * es + n * 4)
    return {"bytes": byt, "flops": 0}


def _counts(case):
    """Tokens of each request: a round's emitted ones, or prompts from half the longest to the longest."""
    B, n = case["B"], case["n"]
    return [max(1, n - (i % 5) * n // 5 if not case["prompt"] else n - (n * i) // (2 * B)) for i in range(B)]


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda", dtype=dtype)


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda")


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _text(g, B, n, V):
    """[B, n] tokens, few of them often and many of them rarely."""
    return (V * _rand(g, B, n) ** 3).long().clamp(max=V - 1) * 7919 % V


def _pack(bits):
    """bool [..., V] -> int32 [..., ceil(V / 32)], bit v % 32 of word v / 32."""
    V = bits.shape[-1]
    full = torch.zeros(*bits.shape[:-1], _words(V) * 32, dtype=torch.bool, device=bits.device)
    full[..., :V] = bits
    full = full.view(*bits.shape[:-1], _words(V), 32)
    w = torch.zeros(full.shape[:-1], dtype=torch.int32, device=bits.device)
    for i in range(32):
        w |= full[..., i].int() << i
    return w


def _state(g, B, V, said, biased):
    """Marks and records of requests that have `said` tokens behind them, a third of them the prompt's."""
    records = torch.zeros(B, V, 2, dtype=torch.int32, device="cuda")
    if said:
        text = _text(g, B, said, V)
        cut = said // 3
        times = torch.zeros(B, V, dtype=torch.int32, device="cuda")
        times.scatter_add_(1, text[:, cut:], torch.ones_like(text[:, cut:], dtype=torch.int32))
        asked = torch.zeros(B, V, dtype=torch.bool, device="cuda").scatter_(1, text[:, :cut], True)
        records[:, :, 0] = torch.where(asked, times | PROMPT, times)
    if biased:
        ids = torch.randint(V, (B, biased), generator=g, device="cuda")
        chosen = torch.zeros(B, V, dtype=torch.bool, device="cuda").scatter_(1, ids, True)
        records[:, :, 1] = torch.where(chosen, 3 * _randn(g, B, V), 0.0).view(torch.int32)
    return _pack((records != 0).any(-1)), records


def _block(s, case, g):
    """Logits, drafts and rules of a verify call. The tokens that lead a row are the text's own half of the time."""
    B, K, V, dt = case["B"], case["K"], case["V"], DTYPES[case["dtype"]]
    s["marks"], s["records"] = _state(g, B, V, case["said"], case["biased"])
    z = _randn(g, B, K + 1, V, dtype=dt).mul_(3.0)
    lead = torch.where(_rand(g, B, K + 1, 4) < 0.5, _text(g, B, (K + 1) * 4, V).view(B, K + 1, 4),
                       torch.randint(V, (B, K + 1, 4), generator=g, device="cuda"))
    top = 14.0 + 4.0 * _rand(g, B, K + 1, 1) - torch.tensor([0.0, 0.4, 1.0, 2.0], device="cuda")
    for i in reversed(range(4)):  # one after the other: a token that leads twice has the larger value
        z.scatter_(2, lead[:, :, i:i + 1], top[:, :, i:i + 1].to(dt))
    pick = torch.multinomial(torch.tensor([0.6, 0.2, 0.1, 0.1], device="cuda"), B * K, True, generator=g) \
        if K else torch.zeros(0, dtype=torch.int64, device="cuda")
    s["logits"] = z
    s["draft"] = lead[:, :K].gather(2, pick.view(B, K, 1)).squeeze(2).int().contiguous()
    s["repetition"] = 1.0 + 0.3 * _rand(g, B)
    s["frequency"] = 0.5 * _rand(g, B)
    s["presence"] = 0.6 * _rand(g, B)
    s["allow"] = None
    if case["grammar"]:  # a third of the vocabulary, and the drafts, which the drafter took from it
        bits = _rand(g, B, K + 1, V) < 0.33
        for i in range(4):
            bits.scatter_(2, lead[:, :, i:i + 1], _rand(g, B, K + 1, 1) < 0.8)
        if K:
            bits[:, :K].scatter_(2, s["draft"].long()[:, :, None], True)
        s["allow"] = _pack(bits)
    if case["op"] == "logits":
        s["changed"] = torch.empty_like(z)
        return
    s["ledger"] = torch.stack([torch.full((B,), BUDGET, device="cuda"), 4.0 * _rand(g, B)], 1).contiguous()
    s["out"] = {"accepted_len": _ints([0] * B), "committed": torch.zeros(B, K + 1, dtype=torch.int32, device="cuda"),
                "recovery": _ints([0] * B), "status": _ints([0] * B),
                "row_argmax": torch.zeros(B, K + 1, dtype=torch.int32, device="cuda"),
                "row_regret": torch.zeros(B, K, device="cuda")}


def _cache(s, case, g, slots, layers):
    B, Hkv, D, page, dt = case["B"], case["Hkv"], case["D"], case["page"], DTYPES[case["dtype"]]
    n = -(-slots // page)
    s["table"] = torch.randperm(B * n, generator=g, device="cuda").to(torch.int32).view(B, n).contiguous()
    order = torch.randperm(B, generator=g, device="cuda")
    s["kv_len"] = _ints(_lens(case))[order]
    for name in "kv" if case["op"] == "evict" else "k":
        s[name] = _randn(g, layers, B * n, page, Hkv, D, dtype=dt)
    return order


def prepare(case, seed):
    g, s, B = _gen(seed), {"case": case}, case["B"]
    if case["op"] in ("verify", "logits"):
        _block(s, case, g)
    elif case["op"] == "record":
        s["marks"], s["records"] = _state(g, B, case["V"], case["said"], 0)
        s["tokens"] = _text(g, B, case["n"], case["V"]).int()
        n = _ints(_counts(case))[torch.randperm(B, generator=g, device="cuda")]
        if case["prompt"]:
            s["token_len"] = n
        else:
            s["token_len"] = None
            s["tokens"][torch.arange(case["n"], device="cuda")[None] >= n[:, None]] = -1
    elif case["op"] == "weigh":
        T, Hq, Hkv, D = case["T"], case["Hq"], case["Hkv"], case["D"]
        order = _cache(s, case, g, case["ctx"] + T, 1)
        slots = case["ctx"] + T
        nodes = T if not case["path"] else 3 * T  # a path's rows lie among a tree's
        rows = _randn(g, B, nodes, Hq + 2 * Hkv, D).mul_(1.5).to(DTYPES[case["dtype"]])  # a fused projection's
        s["q"] = rows[:, :, :Hq]
        s["scale"] = 1.0 / math.sqrt(D)
        # what the attention of these queries over keys of unit variance has on average
        spread = s["q"].float().square().sum(-1) * (0.5 / D)
        s["lse"] = (spread + (s["kv_len"].float() + 1).log()[:, None, None]).contiguous()
        s["new_len"] = _ints(_news(case))[order] if case["path"] else None
        s["path"] = None
        if case["path"]:
            s["path"] = _rand(g, B, nodes).argsort(1)[:, :T].sort(1).values.int().contiguous()
        s["before"] = _rand(g, B, Hkv, slots)
        s["weight"] = torch.zeros(B, Hkv, slots, device="cuda")
    else:
        order = _cache(s, case, g, case["ctx"], case["layers"])
        # a few tokens have most of the weight
        s["before"] = (2.0 * _randn(g, case["layers"], B, case["Hkv"], case["ctx"])).exp_()
        s["weight"] = torch.zeros_like(s["before"])
        s["keep"] = _ints([case["keep"]] * B)
        s["new_len"] = torch.zeros_like(s["kv_len"])
    if own:
        _prepare_own(s, case)
    return s


def _prepare_own(s, case):
    from paper_2608_03447_gb300 import asd
    if case["op"] in ("verify", "logits", "record"):
        s["rules"] = asd.TokenRules(s["marks"], s["records"], repetition=s.get("repetition"),
                                    frequency=s.get("frequency"), presence=s.get("presence"))
        if case["op"] == "verify":
            s["ws"] = asd.Workspace(case["B"], case["K"], case["V"], asd.BF16 if case["dtype"] == "bf16" else asd.F32)
    else:
        # kv_weigh reads keys alone
        s["cache"] = asd.KVCache(s["k"], s.get("v", s["k"]), s["table"])


# ---------------------------------------------------------------- the operators

def run(s):
    op = s["case"]["op"]
    if own:
        return _run_own(s, op)
    return {"verify": _plain_verify, "logits": _plain_logits, "record": _plain_record, "weigh": _plain_weigh,
            "evict": _plain_evict}[op](s)


def _run_own(s, op):
    from paper_2608_03447_gb300 import asd
    if op == "verify":
        asd.rules_verify(s["logits"], s["draft"], s["ledger"], GATE, CAP, s["rules"], allow=s["allow"],
                         workspace=s["ws"], out=s["out"])
        return {**s["out"], "ledger": s["ledger"]}
    if op == "logits":
        return asd.rules_logits(s["logits"], s["draft"], s["rules"], allow=s["allow"], out=s["changed"])
    if op == "record":
        asd.tokens_record(s["tokens"], s["rules"], prompt=s["case"]["prompt"], token_len=s["token_len"])
        return {"marks": s["marks"], "records": s["records"]}
    if op == "weigh":
        return asd.kv_weigh(s["q"], s["lse"], s["cache"], s["kv_len"], s["before"], decay=s["case"]["decay"],
                            new_len=s["new_len"], path=s["path"], scale=s["scale"], out=s["weight"])
    asd.kv_evict(s["cache"], s["kv_len"], s["before"], s["keep"], first=s["case"]["first"], last=s["case"]["last"],
                 out=s["weight"], new_len=s["new_len"])
    return {"k": s["k"], "v": s["v"], "weight": s["weight"], "new_len": s["new_len"]}


def _plain_rules(s):
    """The logits under the rules, float32 [B, K + 1, V]."""
    c = s["case"]
    B, K, V = c["B"], c["K"], c["V"]
    z = s["logits"].float()
    seen = s["records"][:, :, 0]
    times = (seen & 0x7fffffff)[:, None].repeat(1, K + 1, 1)
    for j in range(K):  # a draft counts in the rows behind it
        at = s["draft"][:, j].long()[:, None, None].expand(B, K - j, 1)
        times[:, j + 1:].scatter_add_(2, at, torch.ones_like(at, dtype=torch.int32))
    said = times > 0
    known = said | (seen < 0)[:, None]
    by = s["repetition"][:, None, None]
    z = torch.where(known, torch.where(z > 0, z / by, z * by), z)
    z = torch.where(said, z - times.float() * s["frequency"][:, None, None], z)
    z = torch.where(said, z - s["presence"][:, None, None], z)
    z = z + s["records"][:, :, 1].view(torch.float32)[:, None]
    if s["allow"] is not None:
        bits = (s["allow"][..., None] >> torch.arange(32, dtype=torch.int32, device="cuda")) & 1
        z = torch.where(bits.view(B, K + 1, -1)[..., :V] > 0, z, -math.inf)
    return z


def _plain_logits(s):
    return s["changed"].copy_(_plain_rules(s))


def _plain_verify(s):
    B, K = s["case"]["B"], s["case"]["K"]
    z = _plain_rules(s)
    y = z.argmax(-1)
    top = z.gather(2, y[:, :, None]).squeeze(2)
    r = top[:, :K] - z[:, :K].gather(2, s["draft"].long()[:, :, None]).squeeze(2)
    budget, spent = s["ledger"][:, 0], s["ledger"][:, 1]
    total, misses = torch.zeros_like(spent), torch.zeros(B, dtype=torch.int32, device="cuda")
    going, a = torch.ones(B, dtype=torch.bool, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    for j in range(K):
        miss = y[:, j] != s["draft"][:, j]
        fits = (r[:, j] / torch.full_like(spent, K - j) <= GATE) & (spent + (total + r[:, j]) <= budget) & (misses < CAP)
        going = going & (~miss | fits)
        total = torch.where(going & miss, total + r[:, j], total)
        misses = misses + (going & miss).int()
        a = a + going.int()
    s["ledger"][:, 1] = spent + total
    o = s["out"]
    recovery = y.gather(1, a.long()[:, None]).int()
    at = torch.arange(K + 1, device="cuda")[None]
    drafts = torch.cat([s["draft"], s["draft"].new_zeros(B, 1)], 1)
    o["committed"].copy_(torch.where(at < a[:, None], drafts, torch.where(at == a[:, None], recovery, -1)))
    o["accepted_len"].copy_(a)
    o["recovery"].copy_(recovery.squeeze(1))
    o["row_argmax"].copy_(y)
    o["row_regret"].copy_(r)
    o["status"].zero_()
    return {**o, "ledger": s["ledger"]}


def _plain_record(s):
    c = s["case"]
    B, n, V = c["B"], c["n"], c["V"]
    has = s["tokens"] >= 0
    if s["token_len"] is not None:
        has = torch.arange(n, device="cuda")[None] < s["token_len"][:, None]
    row, col = has.nonzero(as_tuple=True)
    at = row * V + s["tokens"][row, col].long()
    seen = s["records"].view(-1, 2)[:, 0]
    if c["prompt"]:
        seen[at] = seen[at] | PROMPT
    else:
        seen.index_add_(0, at, torch.ones_like(at, dtype=torch.int32))
    new = torch.zeros(B * V, dtype=torch.bool, device="cuda")
    new[at] = True
    s["marks"] |= _pack(new.view(B, V))
    return {"marks": s["marks"], "records": s["records"]}


def _plain_weigh(s):
    c = s["case"]
    B, T, Hq, Hkv, D = c["B"], c["T"], c["Hq"], c["Hkv"], c["D"]
    G, S = Hq // Hkv, c["ctx"] + T
    k = s["k"][0][s["table"].long()].view(B, -1, Hkv, D)[:, :S].permute(0, 2, 3, 1).float()
    q, lse = s["q"], s["lse"]
    if s["path"] is not None:
        rows = torch.arange(B, device="cuda")[:, None]
        q, lse = q[rows, s["path"].long()], lse[rows, s["path"].long()]
    q = q.float().view(B, T, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, D)
    lse = lse.view(B, T, Hkv, G).permute(0, 2, 1, 3).reshape(B, Hkv, T * G, 1)
    n = s["new_len"].long() if s["new_len"] is not None else torch.full((B,), T, device="cuda")
    t, u = torch.arange(T, device="cuda"), torch.arange(S, device="cuda")[None] - s["kv_len"].long()[:, None]
    sees = (u[:, None] <= t[None, :, None]) & (t[None, :] < n[:, None])[:, :, None]
    p = ((q @ k) * s["scale"] - lse).exp_().view(B, Hkv, T, G, S)
    got = torch.where(sees[:, None, :, None], p, 0.0).sum((2, 3))
    if c["decay"]:
        got = torch.where((u < 0)[:, None], s["before"] * c["decay"], 0.0) + got
    s["weight"].copy_(torch.where((u < n[:, None])[:, None], got, s["weight"]))
    return s["weight"]


def _plain_evict(s):
    c = s["case"]
    L, B, H, S, page = c["layers"], c["B"], c["Hkv"], c["ctx"], c["page"]
    at, ctx = torch.arange(S, device="cuda")[None], s["kv_len"].long()[:, None]
    n = torch.minimum(s["keep"].long()[:, None], ctx)
    first = n.clamp(max=c["first"])
    last = (n - first).clamp(max=c["last"])
    always, never = (at < first) | ((at >= ctx - last) & (at < ctx)), at >= ctx
    w = s["before"].masked_fill(always[:, None], math.inf).masked_fill(never[:, None], -math.inf)
    rank = torch.sort(w, dim=-1, descending=True, stable=True).indices.argsort(-1)
    kept, low = rank < n[:, None], (at < n)[:, None].expand(B, H, S)
    src, dst = (kept & ~low).nonzero(), (~kept & low).nonzero()  # as many of each, head by head
    move = torch.where(low.expand(L, B, H, S), s["before"], s["weight"])
    move[dst.unbind(1)] = s["before"][src.unbind(1)]
    s["weight"].copy_(move)

    def place(x):
        layer, b, head, slot = x.unbind(1)
        return layer, s["table"][b, slot // page].long(), slot % page, head
    for name in "kv":
        s[name][place(dst)] = s[name][place(src)]
    s["new_len"].copy_(n.squeeze(1))
    return {"k": s["k"], "v": s["v"], "weight": s["weight"], "new_len": s["new_len"]}


# ---------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("verify", "logits"):
        z = _exact_rules(s, case)
        return z if case["op"] == "logits" else _exact_verify(s, case, z)
    return {"record": _exact_record, "weigh": _exact_weigh, "evict": _exact_evict}[case["op"]](s, case)


def _exact_rules(s, case):
    """Request by request, over the tokens that some rule names."""
    B, K, V = case["B"], case["K"], case["V"]
    z = s["logits"].double()
    for b in range(B):
        drafts = s["draft"][b].tolist()
        named = torch.unique(torch.cat([(s["records"][b] != 0).any(-1).nonzero().flatten(), s["draft"][b].long()]))
        word = s["records"][b, named, 0].long()
        asked, times, bias = word < 0, word & 0x7fffffff, s["records"][b, named, 1].view(torch.float32).double()
        rho, f, pr = (float(s[name][b]) for name in ("repetition", "frequency", "presence"))
        for j in range(K + 1):
            if j:
                times = times + (named == drafts[j - 1])
            x = z[b, j, named]
            x = torch.where((times > 0) | asked, torch.where(x > 0, x / rho, x * rho), x)
            z[b, j, named] = x - (times > 0) * (times * f + pr) + bias
    if s["allow"] is not None:
        for i in range(32):
            part = z[:, :, i::32]
            part[((s["allow"] >> i) & 1)[:, :, :part.shape[2]] == 0] = -math.inf
    return z


def _exact_verify(s, case, z):
    """Request by request, position by position."""
    B, K = case["B"], case["K"]
    top, y = z.max(-1)
    o = {"accepted_len": [], "committed": [], "recovery": [], "status": [0] * B}
    regret, ledger = torch.zeros(B, K, dtype=torch.float64), s["ledger"].double().cpu()
    best, lead, drafts = y.tolist(), top.tolist(), s["draft"].tolist()
    for b in range(B):
        budget, spent = ledger[b].tolist()
        for j in range(K):
            regret[b, j] = lead[b][j] - float(z[b, j, drafts[b][j]])
        a, total, misses = 0, 0.0, 0
        while a < K:
            if drafts[b][a] != best[b][a]:
                r = float(regret[b, a])
                if r / (K - a) > GATE or spent + total + r > budget or misses == CAP:
                    break
                total, misses = total + r, misses + 1
            a += 1
        ledger[b, 1] = spent + total
        o["accepted_len"].append(a)
        o["recovery"].append(best[b][a])
        o["committed"].append(drafts[b][:a] + [best[b][a]] + [-1] * (K - a))
    o = {k: torch.tensor(v, dtype=torch.int32) for k, v in o.items()}
    return {**o, "row_argmax": y.int(), "row_regret": regret, "ledger": ledger}


def _exact_record(s, case):
    """Token by token."""
    V, marks, seen = case["V"], s["marks"].clone().cpu(), s["records"].clone()
    for b in range(case["B"]):
        tokens = s["tokens"][b].tolist()
        tokens = tokens[:int(s["token_len"][b])] if case["prompt"] else [t for t in tokens if t >= 0]
        times = torch.bincount(torch.tensor(tokens), minlength=V).int().cuda()
        seen[b, :, 0] = torch.where(times > 0, seen[b, :, 0] | PROMPT, seen[b, :, 0]) if case["prompt"] \
            else seen[b, :, 0] + times
        bits = [int(w) & 0xffffffff for w in marks[b].tolist()]
        for t in set(tokens):
            bits[t // 32] |= 1 << (t % 32)
        marks[b] = torch.tensor([w - (w >> 31 << 32) for w in bits], dtype=torch.int32)
    return {"marks": marks, "records": seen}


def _exact_weigh(s, case):
    """Request by request, head by head, over the tokens that exist."""
    B, T, Hq, Hkv, page = case["B"], case["T"], case["Hq"], case["Hkv"], case["page"]
    G, out = Hq // Hkv, s["weight"].double()
    lens = s["kv_len"].tolist()
    news = s["new_len"].tolist() if s["new_len"] is not None else [T] * B
    for b in range(B):
        ctx, n = lens[b], news[b]
        rows = s["path"][b, :n].long() if s["path"] is not None else torch.arange(n, device="cuda")
        ids = s["table"][b, :-(-(ctx + n) // page)].long()
        for h in range(Hkv):
            k = s["k"][0][ids, :, h].reshape(-1, case["D"])[:ctx + n].double()
            total = torch.zeros(ctx + n, dtype=torch.float64, device="cuda")
            q, lse = s["q"][b, rows, h * G:(h + 1) * G].double(), s["lse"][b, rows, h * G:(h + 1) * G].double()
            total[:ctx] = torch.exp(q.reshape(n * G, -1) @ k[:ctx].T / math.sqrt(case["D"])
                                    - lse.reshape(n * G, 1)).sum(0)
            for t in range(n):
                z = q[t] @ k[ctx:ctx + t + 1].T / math.sqrt(case["D"])
                total[ctx:ctx + t + 1] += torch.exp(z - lse[t][:, None]).sum(0)
            if case["decay"]:
                total[:ctx] += s["before"][b, h, :ctx].double() * case["decay"]
            out[b, h, :ctx + n] = total
    return out


def _exact_evict(s, case):
    """Head by head: the lightest go, and the ones behind take their places."""
    page, after = case["page"], {"k": s["k"].double(), "v": s["v"].double()}
    weight, lens = s["weight"].double(), s["kv_len"].tolist()
    new = [min(case["keep"], c) for c in lens]
    for b, (ctx, n) in enumerate(zip(lens, new)):
        first = min(case["first"], n)
        last = min(case["last"], n - first)
        row = s["table"][b].long()
        for layer in range(case["layers"]):
            for h in range(case["Hkv"]):
                w = s["before"][layer, b, h, :ctx].double()
                middle = w[first:ctx - last]
                goes = first + torch.sort(-middle, dim=0, stable=True).indices[n - first - last:]
                here = torch.ones(ctx, dtype=torch.bool, device="cuda")
                here[goes] = False
                src, dst = n + here[n:].nonzero().flatten(), (~here[:n]).nonzero().flatten()
                weight[layer, b, h, :n] = w[:n]
                weight[layer, b, h, dst] = w[src]
                for name, x in after.items():
                    x[layer, row[dst // page], dst % page, h] = s[name][layer, row[src // page], src % page, h].double()
    return {**after, "weight": weight, "new_len": torch.tensor(new, dtype=torch.int32)}
