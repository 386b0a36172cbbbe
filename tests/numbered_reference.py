"""A plain form of evictions that know each slot's token, head by head and slot by slot."""
import math


def evicted(k, v, table, kv_len, weight, numbers, tokens, keep, first, last):
    """k, v [layers, pages, page, heads, D], weight and numbers [layers, B, heads, width]: copies after the eviction, and
    the new lengths."""
    k, v, weight, numbers = k.clone(), v.clone(), weight.clone(), numbers.clone()
    layers, page, heads = k.shape[0], k.shape[2], k.shape[3]
    new = []
    for b in range(table.shape[0]):
        ctx, total = int(kv_len[b]), int(tokens[b])
        n = min(int(keep[b]), ctx)
        f = min(first, n)
        r = min(last, n - f)
        new.append(n)
        if n == ctx:
            continue

        def place(slot):
            return int(table[b, slot // page]), slot % page
        for layer in range(layers):
            for h in range(heads):
                w = weight[layer, b, h, :ctx].tolist()
                token = [t if t >= 0 else total - ctx + s for s, t in enumerate(numbers[layer, b, h, :ctx].tolist())]
                stay = {s for s in range(ctx) if s < f or token[s] >= total - r}
                rest = sorted((s for s in range(ctx) if s not in stay),
                              key=lambda s: (-math.inf if math.isnan(w[s]) else w[s], -s), reverse=True)
                stay |= set(rest[:n - len(stay)])
                src = [s for s in range(n, ctx) if s in stay]
                dst = [s for s in range(n) if s not in stay]
                assert len(stay) == n and len(src) == len(dst)
                for s, d in zip(src, dst):
                    for x in (k, v):
                        x[(layer, *place(d), h)] = x[(layer, *place(s), h)]
                    weight[layer, b, h, d] = weight[layer, b, h, s]
                    token[d] = token[s]
                for s in range(ctx):
                    numbers[layer, b, h, s] = token[s] if s < n else -1
    return k, v, weight, numbers, new
