"""Rounds of tree speculation for users with adapters of their own: what a server computes between the library's attention and verification.

The target is the toy of cached_tree_rounds.py with a norm and rotary positions, and every sequence has its own low-rank adapter on
the projection that all share.  In a round all nodes of the drafted trees go through that projection; each sequence's adapter is added (adapt), queries and keys are
normed and rotated by their sequence's position and their node's depth (rotate), attend to the cached tokens and their ancestors
(cache_attend), and what is verified (verify_tree) is answered with its log probability, the entropy there and the likeliest tokens
(logprob), for the nodes on the verified path alone, whose keys and values enter the cache (cache_append).  Nothing of that waits for the host.

    python examples/adapted_tree_rounds.py [rounds]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from examples.cached_tree_rounds import D, EXPANSION, HEADS, HEADS_Q, TOP_K, Target, V, layers, verified_path  # noqa: E402
from paper_2512_16273_amd import tslt  # noqa: E402

ADAPTERS, RANK, TOP = 3, 16, 5


class AdaptedTarget(Target):
    def __init__(self, g, device):
        super().__init__(g, device)
        width, out = self.qkv.shape
        self.down = (torch.randn(ADAPTERS, RANK, width, generator=g, device=device) * width ** -0.5).to(torch.bfloat16)
        self.up = (torch.randn(ADAPTERS, out, RANK, generator=g, device=device) * 0.3 * RANK ** -0.5).to(torch.bfloat16)
        self.scale = torch.full((ADAPTERS,), 2.0, device=device)
        self.freq = (10000.0 ** (-torch.arange(D // 2, device=device) * 2.0 / D)).float()
        self.norms = 1 + 0.1 * torch.randn(2, D, generator=g, device=device)

    def project(self, tokens, adapter, base, position=None):
        """Queries, keys and values of tokens [B, n] at base [B] + position [1, n, 1] (None: one after the other)."""
        x = self.embed[tokens.clamp_min(0).long()]
        y = x @ self.qkv
        tslt.adapt(x, y, self.down, self.up, adapter, scale=self.scale, out={"out": y})
        q, k, v = y.unflatten(-1, (HEADS_Q + 2 * HEADS, D)).split((HEADS_Q, HEADS, HEADS), 2)
        tslt.rotate(q, k, position, self.freq, base=base, q_weight=self.norms[0], k_weight=self.norms[1], eps=1e-6, out={"q": q, "k": k})
        return q, k, v


def main(rounds=20, B=4, prompt=100, seed=1, device="cuda:0", report=print):
    g = torch.Generator(device=device).manual_seed(seed)
    target = AdaptedTarget(g, device)
    tree = layers(EXPANSION)
    n_nodes, n_int = sum(w for _, w in tree), sum(w for _, w in tree[:-1])
    adapter = torch.tensor([b % (ADAPTERS + 1) - 1 for b in range(B)], dtype=torch.int32, device=device)      # some sequences have none
    depth = torch.cat([torch.full((w,), d) for d, (_, w) in enumerate(tree)]).to(torch.int32).view(1, n_nodes, 1).to(device)
    width = (prompt + rounds * (len(EXPANSION) + 1) + 63) // 64 + 1
    cache = tslt.cache_create(B * width, HEADS, D, device)
    pages = torch.arange(B * width, dtype=torch.int32, device=device).view(B, width)
    mask = tslt.tree_mask(EXPANSION, device)

    tokens = torch.randint(0, V, (B, prompt), generator=g, device=device)
    length = torch.zeros(B, dtype=torch.int32, device=device)
    _, k, v = target.project(tokens, adapter, length)
    length = tslt.cache_append(cache, pages, length, k, v)["length"]
    root = torch.randint(0, V, (B, 1), generator=g, device=device)
    emitted, logp = torch.zeros(B, dtype=torch.int64, device=device), torch.zeros(B, device=device)
    for step in range(rounds):
        # the device: candidates of every node, layer by layer (its model knows neither adapters nor what came before)
        node_tokens, sets = [root.to(torch.int32)], []
        for (_, w), k_l in zip(tree, EXPANSION):
            draft = target.logits(torch.zeros(B, w, HEADS_Q, D, dtype=torch.bfloat16, device=device), node_tokens[-1]).view(B * w, V)
            made = tslt.truncate(draft, 1.0, TOP_K, 0.0, TOP_K, u=torch.rand(B * w, k_l, generator=g, device=device))
            sets.append({name: made[name].view(B, w, -1) for name in ("idx", "logit", "count")})
            node_tokens.append(made["token"].view(B, w * k_l))
        nodes = torch.cat(node_tokens, 1)
        q_idx, q_logit, q_count = (torch.cat([s[name] for s in sets], 1).contiguous() for name in ("idx", "logit", "count"))
        # the server: all nodes at once, a node at its sequence's position and its depth
        q, k, v = target.project(nodes, adapter, length, depth)
        att = tslt.cache_attend(q, cache, pages, length, k=k, v=v, mask=mask)
        rows = target.logits(att["out"], nodes).contiguous()
        out = tslt.verify_tree(rows, 1.0, EXPANSION, q_idx, q_logit, q_count.view(B, n_int), nodes[:, 1:].contiguous(),
                               torch.rand(B, n_nodes - 1, generator=g, device=device), torch.rand(B, n_nodes, generator=g, device=device))
        path = verified_path(out["node_slot"], out["len"], EXPANSION)
        # what is answered beside the tokens; entries behind a path's end stay 0
        answer = tslt.logprob(rows, 1.0, out["seq"], top=TOP, index=path, count=out["len"],
                              out={"logp": torch.zeros(path.shape, device=device), "entropy": torch.zeros(path.shape, device=device),
                                   "top_idx": torch.zeros(*path.shape, TOP, dtype=torch.int32, device=device),
                                   "top_logp": torch.zeros(*path.shape, TOP, device=device),
                                   "status": torch.zeros(path.shape, dtype=torch.int32, device=device)})
        logp += answer["logp"].sum(1)
        length = tslt.cache_append(cache, pages, length, k, v, count=out["len"], index=path)["length"]
        root = out["seq"].gather(1, (out["len"] - 1).long()[:, None])
        emitted += out["len"]
    torch.cuda.synchronize()
    result = {"emitted": emitted.tolist(), "logp": logp.tolist(), "length": length.tolist(), "rows": rows, "path": path, "verify": out, "answer": answer, "attend": att}
    report(f"{rounds} rounds of {n_nodes} nodes: tokens emitted {result['emitted']}, their mean log probability {[round(l / max(n, 1), 2) for l, n in zip(result['logp'], result['emitted'])]}")
    return result


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 20)
