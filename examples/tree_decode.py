"""Tree-speculative decoding of a small random decoder with libasd around every step that touches the cache.

One round, for every request at once: a tree of drafts grows from the pending token; the target model runs over its
nodes (kv_append norms and rotates queries and keys and writes keys and values into the paged cache, tree_attention
lets every node see the context and its own ancestors); strict verification of all root-to-leaf paths picks one, and
the ledger's verification of that path accepts a prefix; kv_compact moves the accepted nodes' keys and values next to
the context; commit appends the emitted tokens and advances the cache's length.

    python examples/tree_decode.py [--dtype bf16|f32] [--budget 2.0] [--rounds 24]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)
from paper_2608_03447_gb300 import asd  # noqa: E402


def rms(x: torch.Tensor, eps: float = 1e-6) -> torch.Tensor:
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + eps)).to(x.dtype)


class Decoder:
    """Weights of a decoder with grouped heads, norms of queries and keys for each head, rotation of whole heads."""

    def __init__(self, dtype, device="cuda", V=1000, H=256, layers=2, q_heads=8, heads=2, D=64, positions=2048, seed=0):
        g = torch.Generator().manual_seed(seed)

        def weight(*shape, size):
            return (torch.randn(*shape, generator=g) * size).to(dtype).to(device)

        self.V, self.H, self.layers, self.q_heads, self.heads, self.D = V, H, layers, q_heads, heads, D
        self.embed = weight(V, H, size=1.0)
        self.head = weight(V, H, size=0.3)
        self.qkv = [weight((q_heads + 2 * heads) * D, H, size=H ** -0.5) for _ in range(layers)]
        self.out = [weight(H, q_heads * D, size=0.4 * (q_heads * D) ** -0.5) for _ in range(layers)]
        self.up = [weight(2 * H, H, size=H ** -0.5) for _ in range(layers)]
        self.down = [weight(H, 2 * H, size=0.4 * H ** -0.5) for _ in range(layers)]
        self.q_norm = [(1 + 0.1 * torch.randn(D, generator=g)).to(dtype).to(device) for _ in range(layers)]
        self.k_norm = [(1 + 0.1 * torch.randn(D, generator=g)).to(dtype).to(device) for _ in range(layers)]
        angle = torch.arange(positions)[:, None] / 10000.0 ** (torch.arange(D // 2) * 2 / D)
        self.cos, self.sin = angle.cos().float().to(device), angle.sin().float().to(device)

    def cache(self, B: int, slots: int, page: int = 16) -> asd.KVCache:
        width = -(-slots // page)
        shape = (self.layers, B * width, page, self.heads, self.D)
        k = torch.zeros(shape, dtype=self.embed.dtype, device=self.embed.device)
        table = torch.randperm(B * width).to(torch.int32).view(B, width).to(k.device)  # pages lie anywhere
        return asd.KVCache(k, torch.zeros_like(k), table)

    def forward(self, tokens, cache, kv_len, workspace, status, positions=None, mask=None, new_len=None):
        """tokens [B, T] -> final hidden rows [B, T, H]; the tokens' keys and values enter the cache."""
        B, T = tokens.shape
        x = self.embed[tokens.long()]
        for i in range(self.layers):
            q, k, v = (rms(x) @ self.qkv[i].T).view(B, T, -1, self.D).split((self.q_heads, self.heads, self.heads), 2)
            q = asd.kv_append(k, v, cache, kv_len, layer=i, q=q, positions=positions, new_len=new_len, cos=self.cos,
                              sin=self.sin, q_norm=self.q_norm[i], k_norm=self.k_norm[i], status=status)
            a = asd.tree_attention(q, cache, kv_len, layer=i, tree_mask=mask, new_len=new_len, workspace=workspace,
                                   status=status)["out"]
            x = x + a.view(B, T, -1) @ self.out[i].T
            x = x + torch.relu(rms(x) @ self.up[i].T) @ self.down[i].T
        return rms(x)

    def logits(self, hidden):
        """[B, T, H] -> float32 [B, T, V]: libasd's tensor-core product for bf16."""
        rows = hidden.reshape(-1, self.H)
        z = asd.lmhead_logits(rows.contiguous(), self.head) if rows.dtype == torch.bfloat16 else \
            rows.float() @ self.head.float().T
        return z.view(*hidden.shape[:2], self.V)


class Tree:
    """Two drafts under every node of the first `wide` levels, one under each of the rest."""

    def __init__(self, depth: int = 4, wide: int = 2):
        parents, levels, last = [-1], [0], [0]
        for d in range(1, depth + 1):
            now = []
            for node in last:
                for _ in range(2 if d <= wide else 1):
                    now.append(len(parents))
                    parents.append(node)
                    levels.append(d)
            last = now
        self.depth, self.parents, self.levels = depth, parents, levels
        self.paths = []
        for leaf in last:
            path = [leaf]
            while parents[path[0]] >= 0:
                path.insert(0, parents[path[0]])
            self.paths.append(path)


def draft(model: Decoder, tree: Tree, pending: torch.Tensor) -> torch.Tensor:
    """The drafter: the head on a token's embedding alone, its best token (and the second best) under each node."""
    tokens = [pending]
    best = {}
    for node in range(1, len(tree.parents)):
        parent = tree.parents[node]
        if parent not in best:
            best[parent] = (rms(model.embed[tokens[parent].long()]).float() @ model.head.float().T).topk(2).indices
        tokens.append(best[parent][:, 1 if tree.parents[node - 1] == parent else 0].int())
    return torch.stack(tokens, 1)


def decode(model: Decoder, prompts: list, rounds: int, budget: float = 0.0, gate: float = 1.0, cap: int = 2,
           tree: Tree | None = None):
    """-> the emitted tokens of every request (a list of lists), accepted drafts per round (a float)."""
    tree = tree or Tree()
    dev = model.embed.device
    B, T, K = len(prompts), len(tree.parents), tree.depth
    lengths = torch.tensor([len(p) for p in prompts], dtype=torch.int32)
    longest = int(lengths.max())
    cache = model.cache(B, longest + rounds * (K + 1) + T)
    workspace = asd.attention_workspace(cache, max(T, longest), model.q_heads)
    status = torch.zeros(B, dtype=torch.int32, device=dev)
    kv_len = torch.zeros(B, dtype=torch.int32, device=dev)
    ledger = asd.make_ledger(B, budget, device=dev)
    history = torch.zeros(B, rounds * (K + 1), dtype=torch.int32, device=dev)
    emitted = torch.zeros(B, dtype=torch.int32, device=dev)

    # the prompts, all but their last token, which is the first round's pending one
    if longest > 1:
        padded = torch.zeros(B, longest - 1, dtype=torch.int32)
        for b, p in enumerate(prompts):
            padded[b, :len(p) - 1] = torch.tensor(p[:-1], dtype=torch.int32)
        new = (lengths - 1).to(dev)
        model.forward(padded.to(dev), cache, kv_len, workspace, status, new_len=new)
        kv_len += new
    pending = torch.tensor([p[-1] for p in prompts], dtype=torch.int32, device=dev)

    mask = asd.tree_mask(torch.tensor([tree.parents] * B, dtype=torch.int32, device=dev))
    levels = torch.tensor(tree.levels, dtype=torch.int32, device=dev)
    paths = torch.tensor(tree.paths, device=dev)  # [leaves, K + 1]
    drafts = 0
    for _ in range(rounds):
        tokens = draft(model, tree, pending)
        z = model.logits(model.forward(tokens, cache, kv_len, workspace, status, positions=kv_len[:, None] + levels,
                                       mask=mask))
        exact = asd.verify_strict(z[:, paths].flatten(0, 1), tokens[:, paths[:, 1:]].flatten(0, 1).contiguous())
        path = paths[exact["accepted_len"].view(B, -1).argmax(1)]  # [B, K + 1]
        rows = z.gather(1, path[:, :, None].expand(-1, -1, model.V))
        got = asd.verify(rows, tokens.gather(1, path[:, 1:]), ledger, gate, cap)
        asd.kv_compact(cache, kv_len, path.int(), got["accepted_len"] + 1, status=status)
        asd.commit(got["accepted_len"], got["committed"], kv_len=kv_len, tokens=history, token_len=emitted)
        pending = got["recovery"]
        drafts += int(got["accepted_len"].sum())
    if workspace.error() or bool(status.any()):
        raise RuntimeError(f"a call has reported an error: {workspace.error()}, {status.tolist()}")
    out = [history[b, :int(emitted[b])].tolist() for b in range(B)]
    return out, drafts / (rounds * B)


def main() -> None:
    a = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    a.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    a.add_argument("--budget", type=float, default=2.0)
    a.add_argument("--rounds", type=int, default=24)
    a = a.parse_args()
    model = Decoder(torch.bfloat16 if a.dtype == "bf16" else torch.float32)
    prompts = [[1, 2, 3, 4, 5], [7], [11, 13, 17, 19, 23, 29, 31, 37, 41]]
    for budget in (0.0, a.budget):
        out, rate = decode(model, prompts, a.rounds, budget=budget)
        print(f"budget {budget}: {rate:.2f} drafts accepted a round, {sum(map(len, out))} tokens in {a.rounds} rounds")
        for tokens in out:
            print("  ", tokens[:16])


if __name__ == "__main__":
    main()
