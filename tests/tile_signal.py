"""Long contexts whose every tile of keys and values shows in the result, and a check that sees one of them missing.

With random values the result of a long context is their mean, so small that a tile more or less is within any bound.
Here tile j's values are 1 to 2 in element j % D and 0 elsewhere: an element of the result is the weight of the few
tiles of its class, and its bound is relative to that weight. Tile j's keys add one of five offsets to the scores.
"""
import math

import torch

from cache_reference import UNIT

CTAS = 152  # at least as many as share the work, on the GPU that the tests are for


class Tiles:
    """Inputs on the CPU: B requests with trees, one cache, tiles of `tile` slots that carry a signal."""

    def __init__(self, dtype, T, Hq, Hkv, D, page, ctx, tile=128, seed=0):
        from paper_2608_03447_gb300 import asd
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.T, self.Hq, self.Hkv, self.D, self.page, self.tile = dtype, T, Hq, Hkv, D, page, tile
        self.B, self.ctx, self.scale = len(ctx), list(ctx), 1.0 / math.sqrt(D)
        self.q = torch.randn(self.B, T, Hq, D, generator=g).to(dtype)
        self.q[..., 0] = 1.0
        parents = torch.full((self.B, T), -1, dtype=torch.int64)
        for t in range(1, T):
            parents[:, t] = t - 1 - (torch.rand(self.B, generator=g) ** 2 * min(t, 6)).long()
        self.mask = asd.tree_mask(parents)
        self.keys, self.values = [], []  # of a request, by slot: [slots, Hkv, D]
        for c in self.ctx:
            n = c + T
            j = torch.arange(n) // tile
            k = torch.randn(n, Hkv, D, generator=g) * 0.3
            k[..., 0] = ((((j * 7919) % 5) - 2) * 0.5 * math.sqrt(D))[:, None]
            v = torch.zeros(n, Hkv, D)
            v[torch.arange(n), :, j % D] = 1 + torch.randint(0, 128, (int(j[-1]) + 1, Hkv), generator=g)[j] / 128
            self.keys.append(k.to(dtype))
            self.values.append(v.to(dtype))
        need = [-(-(c + T) // page) for c in self.ctx]
        order = torch.randperm(sum(need), generator=g).to(torch.int32)
        self.table = torch.zeros(self.B, max(need), dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n

    def cache(self, asd):
        k = torch.zeros(int(self.table.max()) + 1, self.page, self.Hkv, self.D, dtype=self.dtype)
        v = torch.zeros_like(k)
        for b in range(self.B):
            slot = torch.arange(self.ctx[b] + self.T)
            page = self.table[b, slot // self.page].long()
            k[page, slot % self.page], v[page, slot % self.page] = self.keys[b], self.values[b]
        return asd.KVCache(k.cuda(), v.cuda(), self.table.cuda())

    def sees(self, b):
        """[T, slots] bool."""
        bits = torch.stack([(self.mask[b, :, u // 32] >> (u % 32)) & 1 for u in range(self.T)], 1).bool()
        return torch.cat([torch.ones(self.T, self.ctx[b], dtype=torch.bool), bits], 1)

    def reference(self, b, device="cpu", plant=None):
        """out [T, Hq, D], lse and the largest sum of |q_d k_d| scale [T, Hq], in 64 bits. plant = (what, j, i): a
        mistake, tile j's keys or values taken from tile i, or (i None) the values zero or the whole tile not seen."""
        G = self.Hq // self.Hkv
        k, v, sees = self.keys[b].double(), self.values[b].double(), self.sees(b)
        if plant:
            what, j, i = plant
            at = slice(j * self.tile, min((j + 1) * self.tile, len(k)))
            n = at.stop - at.start
            if i is None:
                if what == "values":
                    v[at] = 0
                else:
                    sees[:, at] = False
            else:
                x = v if what == "values" else k
                x[at] = x[i * self.tile:i * self.tile + n].clone()
        k, v, sees, q = k.to(device), v.to(device), sees.to(device), self.q[b].double().to(device)
        out = torch.zeros(self.T, self.Hq, self.D, dtype=torch.float64, device=device)
        lse = torch.zeros(self.T, self.Hq, dtype=torch.float64, device=device)
        reach = torch.zeros_like(lse)
        for h in range(self.Hkv):
            heads = slice(h * G, (h + 1) * G)
            z = torch.einsum("tgd,sd->tgs", q[:, heads], k[:, h]) * self.scale
            z = z.masked_fill(~sees[:, None], -math.inf)
            lse[:, heads] = torch.logsumexp(z, -1)
            out[:, heads] = torch.einsum("tgs,sd->tgd", torch.softmax(z, -1), v[:, h])
            reach[:, heads] = (torch.einsum("tgd,d->tg", q[:, heads].abs(), k[:, h].abs().amax(0)) * self.scale)
        return out.cpu(), lse.cpu(), reach.cpu()

    def sums(self):
        """Relative error of a sum over a request's slots. A CTA adds up its share of the tiles, and those of a unit
        are then added: a share is an equal part of all tiles (of all heads and row tiles, of which there are no more
        than one for 100 rows), 16 slots an addition that may cut off (2u) on the tensor cores, one (u) in fp32."""
        units = self.Hkv * (self.T * (self.Hq // self.Hkv) // 100 + 1)
        share = sum(c + self.T for c in self.ctx) * units / CTAS + 4 * self.tile
        return (share / 8 if self.dtype != torch.float32 else share) * 2.0 ** -24 + 2 * CTAS * 2.0 ** -24

    def misses(self, b, out, lse, want):
        """How much further than its bound an element of request b's result is off, at most (<= 0: none)."""
        o, l, reach = want
        u = 2.0 ** -24
        rel = 2 * (self.D + 2) * u * reach[..., None] + 2.0 ** -21 + 2 * self.sums()
        tol = (rel + UNIT[self.dtype] * (1 if self.dtype == torch.float32 else 2)) * o
        if self.dtype == torch.float16:  # weights below 2^-14 where the largest is 2^7, and results below it
            tol = tol + 2 * (self.ctx[b] + self.T) * 2.0 ** -32 + 2.0 ** -24
        may = (self.D + 2) * u * reach + 2.0 ** -20 + self.sums() + l.abs() * 2.0 ** -21
        return max(float(((out.double() - o).abs() - tol).max()), float(((lse.double() - l).abs() - may).max()))
