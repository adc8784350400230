"""Rounds of tree speculation with the target's keys and values in an 8-bit cache: every call of the library that a server makes, in order.

The target is a toy of one attention layer with random weights; the draft is its logits with noise.  A round drafts a tree of tokens
(truncate), runs the target on all of its nodes at once, each seeing the cached tokens and its ancestors (cache_attend), verifies
them (verify_tree), adds the attention weight that each cached token got (cache_weigh) and appends the keys and values of the
verified path alone (cache_append).  Nothing of that waits for the host.  Where a sequence outgrows its budget, its tokens of most weight are
moved to new pages (cache_evict) and the old ones are used again.

    python examples/cached_tree_rounds.py [rounds]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2512_16273_amd import tslt  # noqa: E402

V, HEADS_Q, HEADS, D = 32000, 8, 2, 64
EXPANSION, TOP_K = (2, 2, 2), 16
BUDGET, KEEP, RECENT = 448, 256, 32


class Target:
    """Token and position to queries, keys and values; attention's output to logits."""

    def __init__(self, g, device):
        def matrix(*shape):
            return torch.randn(*shape, generator=g, device=device).to(torch.bfloat16)
        width = HEADS_Q * D
        self.embed, self.head = matrix(V, width), matrix(width, V) * 0.18      # (a few likely tokens behind every one)
        self.qkv = matrix(width, (HEADS_Q + 2 * HEADS) * D) * width ** -0.5

    def project(self, tokens):
        x = (self.embed[tokens.clamp_min(0).long()] @ self.qkv).unflatten(-1, (HEADS_Q + 2 * HEADS, D))
        return x[:, :, :HEADS_Q], x[:, :, HEADS_Q:HEADS_Q + HEADS], x[:, :, HEADS_Q + HEADS:]

    def logits(self, attended, tokens):
        return (attended.flatten(2) + self.embed[tokens.clamp_min(0).long()]) @ self.head


def layers(expansion):
    """First node and width of every layer of the tree."""
    made, first, width = [(0, 1)], 1, 1
    for k in expansion:
        width *= k
        made.append((first, width))
        first += width
    return made


def verified_path(node_slot, length, expansion):
    """Nodes on the verified path of every tree, [B, depth + 1] int32; its first length[b] count."""
    node = torch.zeros_like(length, dtype=torch.int64)
    path = [node]
    for (first, _), (below, _), k in zip(layers(expansion), layers(expansion)[1:], expansion):
        slot = node_slot.gather(1, node[:, None].clamp_max(node_slot.shape[1] - 1))[:, 0].long().clamp_min(0)
        node = below + (node - first).clamp_min(0) * k + slot
        path.append(node)
    return torch.stack(path, 1).to(torch.int32)


def main(rounds=40, B=4, prompt=300, seed=1, device="cuda:0", report=print):
    g = torch.Generator(device=device).manual_seed(seed)
    target = Target(g, device)
    tree = layers(EXPANSION)
    n_nodes, n_int = sum(w for _, w in tree), sum(w for _, w in tree[:-1])
    width = (BUDGET + 63) // 64 + 1
    cache = tslt.cache_create(2 * B * width, HEADS, D, device)
    pages = torch.arange(2 * B * width, dtype=torch.int32, device=device).view(2, B, width)
    now = 0                                                       # which half of the pages the sequences lie in
    mask = tslt.tree_mask(EXPANSION, device)
    weight = torch.zeros(B, HEADS, width * 64, device=device)

    tokens = torch.randint(0, V, (B, prompt), generator=g, device=device)
    _, k, v = target.project(tokens)
    length = tslt.cache_append(cache, pages[now], torch.zeros(B, dtype=torch.int32, device=device), k, v)["length"]
    root = torch.randint(0, V, (B, 1), generator=g, device=device)
    emitted, most = torch.zeros(B, dtype=torch.int64, device=device), prompt
    for step in range(rounds):
        # the device: candidates of every node, layer by layer, from the draft's distribution (here the embedding's logits with noise)
        node_tokens, sets = [root.to(torch.int32)], []
        for (_, w), k_l in zip(tree, EXPANSION):
            draft = target.logits(torch.zeros(B, w, HEADS_Q, D, dtype=torch.bfloat16, device=device), node_tokens[-1]).view(B * w, V)
            made = tslt.truncate(draft, 1.0, TOP_K, 0.0, TOP_K, u=torch.rand(B * w, k_l, generator=g, device=device))
            sets.append({name: made[name].view(B, w, -1) for name in ("idx", "logit", "count")})
            node_tokens.append(made["token"].view(B, w * k_l))
        nodes = torch.cat(node_tokens, 1)
        q_idx, q_logit, q_count = (torch.cat([s[name] for s in sets], 1).contiguous() for name in ("idx", "logit", "count"))
        # the server: all nodes at once
        q, k, v = target.project(nodes)
        att = tslt.cache_attend(q, cache, pages[now], length, k=k, v=v, mask=mask)
        out = tslt.verify_tree(target.logits(att["out"], nodes).contiguous(), 1.0, EXPANSION, q_idx, q_logit, q_count.view(B, n_int),
                               nodes[:, 1:].contiguous(), torch.rand(B, n_nodes - 1, generator=g, device=device),
                               torch.rand(B, n_nodes, generator=g, device=device))
        weight = tslt.cache_weigh(q, att["lse"], cache, pages[now], length, weight, decay=0.95)["weight"]
        # the verified path's keys and values enter the cache; its last output is the next tree's root
        path = verified_path(out["node_slot"], out["len"], EXPANSION)
        length = tslt.cache_append(cache, pages[now], length, k, v, count=out["len"], index=path)["length"]
        root = out["seq"].gather(1, (out["len"] - 1).long()[:, None])
        emitted += out["len"]
        most += len(EXPANSION) + 1                                 # (an upper bound, so that nothing asks the device how long they are)
        if most + len(EXPANSION) + 1 > BUDGET:
            got = tslt.cache_evict(cache, pages[now], length, weight, KEEP, RECENT, pages[1 - now])
            now, length, weight, most = 1 - now, got["length"], got["weight"], KEEP
    torch.cuda.synchronize()
    result = {"emitted": emitted.tolist(), "length": length.tolist(), "attend": att, "verify": out}
    report(f"{rounds} rounds of {n_nodes} nodes: tokens emitted {result['emitted']}, cached {result['length']}")
    return result


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 40)
