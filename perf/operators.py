"""The calls around a key/value cache held in 8 bits that a verification round makes, over the sizes it makes them at.

The server keeps the keys and values of every sequence in pages of 64 tokens, each number in e4m3 with one power-of-two scale
for a page's keys and one for its values, for each head.  A round attends from the draft's tokens (a chain or a tree, whose own
keys and values come beside the cache) to everything before them, verifies, and appends what was accepted; the device, which
has little memory, also accumulates how much attention each cached token gets, and gives up the tokens with the least.

  append  rows of keys and values, chosen by index and count, quantised to the end of the cache
  attend  softmax attention over cached and new tokens
  weigh   each cached token's attention weight, summed over queries and the heads that share its keys, added to what it had
  evict   the `keep` tokens of most weight (the `recent` last ones always) of every head, moved to new pages

A cached page of one head: 64*D bytes of keys, [64 tokens][D], then 64*D bytes of values, [4][D][16 tokens].
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
PAGE = 64
MIN_EXP = -100                 # least exponent of a page's scale
DEV = "cuda"


def listed():
    return [
        # one decoded token of one user goes into the cache: nothing but latency
        dict(name="append_one", op="append", B=1, n=1, heads=8, D=128, lo=1000, hi=1000, dtype="bf16", chosen=False),
        # the accepted tokens of a batch of 256 chains of 8 draft tokens and the one before them, ragged lengths
        dict(name="append_path_256", op="append", B=256, n=9, heads=8, D=128, lo=40, hi=2000, dtype="bf16", chosen=True),
        # whole prompts of eight users
        dict(name="append_prompt", op="append", B=8, n=4001, heads=8, D=128, lo=0, hi=0, dtype="f16", chosen=False),
        # one draft token on the device, heads of the paper's draft model (12 of 64, FP16)
        dict(name="attend_one", op="attend", B=1, n=1, heads_q=12, heads=12, D=64, lo=500, hi=500, dtype="f16", tree=""),
        # a round of 64 chains of 8 draft tokens, grouped heads, ragged lengths
        dict(name="attend_chain_64", op="attend", B=64, n=9, heads_q=32, heads=8, D=128, lo=100, hi=8000, dtype="bf16", tree=""),
        # four users with 128k tokens each, a token at a time: nothing but memory
        dict(name="attend_long", op="attend", B=4, n=1, heads_q=32, heads=8, D=128, lo=120000, hi=131000, dtype="bf16", tree=""),
        # the benchmark's trees (depth 5, four candidates a node) without their last layer, fp32 as its logits are
        dict(name="attend_tree", op="attend", B=8, n=341, heads_q=32, heads=8, D=128, lo=300, hi=2500, dtype="f32", tree="4x4x4x4"),
        # a long prompt's next piece: nothing but matrix products
        dict(name="attend_prompt", op="attend", B=1, n=2048, heads_q=32, heads=8, D=128, lo=16000, hi=16000, dtype="bf16", tree=""),
        # one user's round on the device: weights of a short cache
        dict(name="weigh_one", op="weigh", B=1, n=5, heads_q=12, heads=12, D=64, lo=1500, hi=1500, dtype="f32", decay=1.0),
        # the weights of a batch, once a round
        dict(name="weigh_32", op="weigh", B=32, n=9, heads_q=32, heads=8, D=128, lo=1000, hi=16000, dtype="bf16", decay=0.95),
        # one user's cache brought back to a quarter
        dict(name="evict_one", op="evict", B=1, heads=12, D=64, lo=4096, hi=4096, keep=1024, recent=64),
        # a batch of long caches brought back to half, rounded up to no multiple of a page
        dict(name="evict_16", op="evict", B=16, heads=8, D=128, lo=9000, hi=32768, keep=16001, recent=511),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    op = rng.choice(["append", "attend", "attend", "weigh", "evict"])
    D = rng.choice([64, 128, 128, 256])
    heads = rng.choice([1, 2, 4, 5, 8, 12, 32])
    group = rng.choice([1, 1, 2, 3, 4, 4, 7, 8])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    kind = rng.choice(["few", "few", "many"])
    B = log_int(1, 256)
    if op == "append":
        n = log_int(1, 17) if kind == "few" else log_int(18, 6000)
        n = min(n, 64_000_000 // (2 * heads * D))
        B = max(1, min(B, 64_000_000 // (2 * n * heads * D)))
        lo = rng.choice([0, rng.randrange(0, 4000)])
        return dict(op=op, B=B, n=n, heads=heads, D=D, lo=lo, hi=lo + rng.choice([0, rng.randrange(0, 2000)]), dtype=dtype,
                    chosen=rng.random() < 0.5)
    if op == "evict":
        hi = log_int(70, 60000)
        B = max(1, min(B, 500_000_000 // (hi * heads * D)))
        keep = max(1, int(hi * rng.uniform(0.05, 0.9)))
        return dict(op=op, B=B, heads=heads, D=D, lo=max(1, int(hi * rng.uniform(0.2, 1.0))), hi=hi, keep=keep,
                    recent=rng.randrange(0, max(1, keep // 2)))
    tree = rng.choice(["", "", "2x2x2", "4x4x4", "3x2x1x1", "16"]) if op == "attend" and kind == "few" else ""
    n = _nodes(tree) if tree else log_int(1, 17) if kind == "few" else log_int(18, 1500)
    hi = min(log_int(16, 100_000 if kind == "few" else 12_000), 500_000_000 // (heads * D))
    B = max(1, min(B, 500_000_000 // (hi * heads * D), 300_000_000_000 // (n * heads * group * (hi + n) * D * 4)))
    lo = int(hi * rng.choice([0.0, 1.0, rng.random()]))
    case = dict(op=op, B=B, n=n, heads_q=heads * group, heads=heads, D=D, lo=lo, hi=hi, dtype=dtype)
    case["tree" if op == "attend" else "decay"] = tree if op == "attend" else rng.choice([1.0, 0.9, 0.5])
    return case


# ---- what a case says about its sizes -------------------------------------------------------------------------

def _nodes(tree):
    total = width = 1
    for k in tree.split("x"):
        width *= int(k)
        total += width
    return total


def _lengths(case):
    """Cached tokens of every sequence: from `lo` to `hi`, in no order."""
    B, lo, hi = case["B"], case["lo"], case["hi"]
    return [hi if B == 1 else lo + (hi - lo) * ((b * 37 + 11) % B) // (B - 1) for b in range(B)]


def _counts(case):
    """Tokens that each sequence appends: all of them, or what was accepted of a chain."""
    return [1 + (b * 5 + 3) % case["n"] if case.get("chosen") else case["n"] for b in range(case["B"])]


def _pairs(case):
    """(query, key) pairs of one query head of all sequences: cached tokens, and new ones."""
    n, tree = case["n"], case.get("tree")
    if case["op"] == "weigh":
        new = 0
    elif tree:
        new, width = 1, 1
        for depth, k in enumerate(tree.split("x")):
            width *= int(k)
            new += width * (depth + 2)
    else:
        new = n * (n + 1) // 2
    return n * sum(_lengths(case)), case["B"] * new


def work(case):
    B, H, D, lengths = case["B"], case["heads"], case["D"], _lengths(case)
    row = H * D
    pages = sum(-(-x // PAGE) for x in lengths)
    if case["op"] == "append":
        rows = sum(_counts(case))
        return {"bytes": rows * row * 2 * (BYTES[case["dtype"]] + 1) + 8 * B, "flops": 0}
    if case["op"] == "evict":
        kept = sum(min(x, case["keep"]) for x in lengths)
        return {"bytes": sum(lengths) * H * 4 + kept * (2 * 2 * row + H * 8), "flops": 0}
    cached, new = _pairs(case)
    q = B * case["n"] * case["heads_q"] * D
    if case["op"] == "weigh":
        return {"bytes": sum(lengths) * (row + 8 * H) + pages * (4 * H + 4) + q * BYTES[case["dtype"]] + q // D * 4,
                "flops": 2 * D * case["heads_q"] * cached}
    own_kv = 2 * B * case["n"] * row
    return {"bytes": sum(lengths) * 2 * row + pages * (8 * H + 4) + (2 * q + own_kv) * BYTES[case["dtype"]] + q // D * 4,
            "flops": 4 * D * case["heads_q"] * (cached + new)}


# ---- inputs -----------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(1000003 * int(seed) + 17)


def _channels(g, heads, D):
    """Spread of each channel: a few channels of a head are much larger than the others, as in a model's keys."""
    s = torch.rand(heads, D, generator=g, device=DEV) + 0.5
    return torch.where(torch.rand(heads, D, generator=g, device=DEV) < 0.03, s * 6, s)


def _filled(case, g, spare):
    """A cache that holds the sequences' tokens in pages that lie in no order, and `spare` more pages for each sequence."""
    B, H, D, lengths = case["B"], case["heads"], case["D"], _lengths(case)
    used = [-(-x // PAGE) for x in lengths]
    width = max(used) + spare
    n_pages = max(1, sum(used) + B * spare)
    codes = torch.zeros(n_pages, H, 2, PAGE * D, dtype=torch.uint8, device=DEV)
    scale = torch.ones(n_pages, H, 2, dtype=torch.float32, device=DEV)
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    pages = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    at, last = 0, []
    for b in range(B):
        n = used[b] + spare
        pages[b, :n] = order[at:at + n]
        at += n
        last.append((pages[b, used[b] - 1] if used[b] else order[0], lengths[b] % PAGE if used[b] else PAGE))
    spread = _channels(g, H, D)
    chunk = max(1, (1 << 27) // (H * PAGE * D))
    for p in range(0, n_pages, chunk):
        m = min(chunk, n_pages - p)
        for part in (0, 1):
            x = torch.randn(m, H, PAGE, D, generator=g, device=DEV) * (spread[:, None] if part == 0 else 0.7)
            x = x * torch.exp(0.5 * torch.randn(m, 1, 1, 1, generator=g, device=DEV))
            e = _exponent(x.abs().amax((2, 3)))
            s = _power_of_two(e)
            c = (x / s[:, :, None, None]).to(torch.float8_e4m3fn)
            if part:
                c = c.view(torch.uint8).view(m, H, 4, 16, D).transpose(3, 4)
            codes[p:p + m, :, part] = c.reshape(m, H, PAGE * D).view(torch.uint8)
            scale[p:p + m, :, part] = s
    for b, (page, rest) in enumerate(last):                        # nothing lies behind a sequence's last token
        if rest and rest < PAGE:
            p = int(page)
            codes[p, :, 0].view(H, PAGE, D)[:, rest:] = 0
            v = codes[p, :, 1].view(H, 4, D, 16).transpose(2, 3).reshape(H, PAGE, D).clone()
            v[:, rest:] = 0
            codes[p, :, 1] = v.view(H, 4, 16, D).transpose(2, 3).reshape(H, PAGE * D)
    return dict(codes=codes, scale=scale), pages, torch.tensor(lengths, dtype=torch.int32, device=DEV), spread


def _tree_mask(tree):
    """Bits of the ancestors of every node of a tree stored breadth-first, and its own: [1, nodes, words]."""
    parents, width, first = [-1], 1, 0
    for k in tree.split("x"):
        parents += [first + i for i in range(width) for _ in range(int(k))]
        first, width = first + width, width * int(k)
    n = len(parents)
    words = -(-n // 32)
    rows = []
    for i in range(n):
        bits, j = 0, i
        while j >= 0:
            bits |= 1 << j
            j = parents[j]
        rows.append([(bits >> (32 * w)) & 0xFFFFFFFF for w in range(words)])
    m = torch.tensor(rows, dtype=torch.int64)
    return torch.where(m >= 1 << 31, m - (1 << 32), m).to(torch.int32)[None].to(DEV)


def prepare(case, seed):
    g = _gen(seed)
    B, H, D, op = case["B"], case["heads"], case["D"], case["op"]
    n = case.get("n", 0)
    spare = -(-case["n"] // PAGE) + 1 if op == "append" else 0
    cache, pages, length, spread = _filled(case, g, spare)
    state = dict(case=case, cache=cache, pages=pages, length=length)
    if op == "evict":
        lengths = _lengths(case)
        at = torch.arange(pages.shape[1] * PAGE, device=DEV)
        heavy = torch.rand(B, H, at.numel(), generator=g, device=DEV) < 0.05
        weight = -torch.log(torch.rand(B, H, at.numel(), generator=g, device=DEV).clamp_min(1e-7)) * torch.where(heavy, 20.0, 0.3)
        # (tokens that no query has looked at have exactly nothing: ties)
        weight = torch.where(torch.rand(B, H, at.numel(), generator=g, device=DEV) < 0.1, torch.zeros_like(weight), weight)
        state["weight"] = torch.where(at < length[:, None, None], weight, torch.zeros_like(weight))
        need = [-(-min(x, case["keep"]) // PAGE) for x in lengths]
        first = cache["codes"].shape[0]
        total = first + sum(need)
        for name, x in list(cache.items()):
            cache[name] = torch.cat([x, torch.zeros(total - first, *x.shape[1:], dtype=x.dtype, device=DEV)])
        order = torch.randperm(total - first, generator=g, device=DEV).to(torch.int32) + first
        new_pages = torch.full((B, -(-case["keep"] // PAGE)), -1, dtype=torch.int32, device=DEV)
        at = 0
        for b in range(B):
            new_pages[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
        state["new_pages"] = new_pages
        state["out"] = dict(length=torch.empty(B, dtype=torch.int32, device=DEV),
                            kept=torch.empty(B, H, case["keep"], dtype=torch.int32, device=DEV),
                            weight=torch.empty(B, H, new_pages.shape[1] * PAGE, dtype=torch.float32, device=DEV),
                            status=torch.empty(B, dtype=torch.int32, device=DEV))
        return state
    dt = DTYPES[case["dtype"]]
    Hq = case.get("heads_q", 0)
    # queries, keys and values of the new tokens as one projection leaves them: side by side
    x = torch.randn(B, n, Hq + 2 * H, D, generator=g, device=DEV)
    x[:, :, Hq:Hq + H] *= spread
    x[:, :, :Hq] *= 1.5
    x[:, :, Hq + H:] *= torch.exp(0.5 * torch.randn(B, 1, 1, 1, generator=g, device=DEV))
    x = x.to(dt)
    state.update(q=x[:, :, :Hq], k=x[:, :, Hq:Hq + H], v=x[:, :, Hq + H:])
    if op == "append":
        state["out"] = dict(length=torch.empty(B, dtype=torch.int32, device=DEV), status=torch.empty(B, dtype=torch.int32, device=DEV))
        state["count"] = torch.tensor(_counts(case), dtype=torch.int32, device=DEV)
        state["index"] = None
        if case["chosen"]:                                         # the accepted ones, in order
            pick = torch.rand(B, n, generator=g, device=DEV).argsort(1)
            taken = torch.arange(n, device=DEV) < state["count"][:, None]
            state["index"] = torch.where(taken, pick, torch.full_like(pick, n)).sort(1).values.clamp_max(n - 1).to(torch.int32)
    elif op == "attend":
        state["mask"] = _tree_mask(case["tree"]) if case["tree"] else None
        state["out"] = dict(out=torch.empty(B, n, Hq, D, dtype=dt, device=DEV), lse=torch.empty(B, n, Hq, device=DEV),
                            status=torch.empty(B, dtype=torch.int32, device=DEV))
    else:
        s = _scores(state["q"], _values(cache, pages, D)[0], D)
        s = s.masked_fill(_beyond(pages, length), -math.inf)
        state["lse"] = torch.logsumexp(s, -1).reshape(B, H, n, Hq // H).transpose(1, 2).reshape(B, n, Hq).contiguous()
        state["weight"] = torch.rand(B, H, pages.shape[1] * PAGE, generator=g, device=DEV)
        state["out"] = dict(weight=torch.empty_like(state["weight"]), status=torch.empty(B, dtype=torch.int32, device=DEV))
    state["workspace"] = torch.empty(256 << 20, dtype=torch.uint8, device=DEV) if op == "attend" else None
    return state


# ---- the plain form ---------------------------------------------------------------------------------------------

def _exponent(amax):
    """Least e >= MIN_EXP with amax <= 448 * 2^e."""
    m, e = torch.frexp(amax)                                       # amax = m * 2^e, 1/2 <= m < 1; 448 = 7/8 * 2^9
    return torch.where(amax > 0, (e - 9 + (m > 0.875).to(e.dtype)).clamp_min(MIN_EXP), torch.full_like(e, MIN_EXP))


def _power_of_two(e):
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _values(cache, pages, D):
    """Cached keys and values, [B, heads, tokens, D] in fp32."""
    at = pages.long().clamp_min(0)
    B, W = at.shape
    x = cache["codes"][at].view(torch.float8_e4m3fn).float() * cache["scale"][at][..., None]
    H = x.shape[2]
    k = x[:, :, :, 0].reshape(B, W, H, PAGE, D).transpose(1, 2).reshape(B, H, W * PAGE, D)
    v = x[:, :, :, 1].reshape(B, W, H, 4, D, 16).permute(0, 2, 1, 3, 5, 4).reshape(B, H, W * PAGE, D)
    return k, v


def _stored(x, scale):
    """[..., 2, 64, D] values and their [..., 2] scales as the cache holds them."""
    c = (x / scale[..., None, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    D = c.shape[-1]
    k = c[..., 0, :, :].flatten(-2)
    v = c[..., 1, :, :].unflatten(-2, (4, 16)).transpose(-1, -2).flatten(-3)
    return torch.stack([k, v], -2).view(*c.shape[:-2], PAGE * D)


def _grouped(x, H):
    """[B, n, Hq, D] as [B, heads, n * group, D] in fp32."""
    B, n, Hq, D = x.shape
    return x.float().reshape(B, n, H, Hq // H, D).transpose(1, 2).reshape(B, H, n * (Hq // H), D)


def _scores(q, k, D):
    return torch.matmul(_grouped(q, k.shape[1]), k.transpose(-1, -2)) * (1.0 / math.sqrt(D))


def _beyond(pages, length):
    return (torch.arange(pages.shape[1] * PAGE, device=pages.device) >= length[:, None])[:, None, None]


def _plain_append(s):
    cache, pages, length, count, D = s["cache"], s["pages"], s["length"], s["count"], s["case"]["D"]
    B, n, H, _ = s["k"].shape
    new = torch.stack([s["k"], s["v"]], 3).float()                 # [B, n, heads, 2, D]
    if s["index"] is not None:
        new = new.gather(1, s["index"].long()[:, :, None, None, None].expand(B, n, H, 2, D))
    # the pages that a sequence's new tokens may lie on, whole, with the new tokens in their places
    first = torch.div(length, PAGE, rounding_mode="floor").long()
    W = (n + PAGE - 1) // PAGE + 1
    entry = first[:, None] + torch.arange(W, device=length.device)
    there = entry * PAGE < (length + count)[:, None]
    at = pages.gather(1, entry.clamp_max(pages.shape[1] - 1)).long().clamp_min(0)
    old_scale = cache["scale"][at]                                 # [B, W, heads, 2]
    slot = entry[:, :, None] * PAGE + torch.arange(PAGE, device=length.device)      # [B, W, 64]
    old, fresh = slot < length[:, None, None], slot >= length[:, None, None]
    fresh = fresh & (slot < (length + count)[:, None, None])
    source = (slot - length[:, None, None]).clamp(0, n - 1).reshape(B, W * PAGE).long()
    k, v = _values(cache, at, D)
    held = torch.stack([k, v], 2).reshape(B, H, 2, W, PAGE, D).permute(0, 3, 1, 2, 4, 5)
    came = new.gather(1, source[:, :, None, None, None].expand(B, W * PAGE, H, 2, D)).reshape(B, W, PAGE, H, 2, D).permute(0, 1, 3, 4, 2, 5)
    x = torch.where(fresh[:, :, None, None, :, None], came, torch.where(old[:, :, None, None, :, None], held, torch.zeros_like(held)))
    most = torch.where(fresh[:, :, None, None, :, None], came, torch.zeros_like(came)).abs().amax((4, 5))
    need = _power_of_two(_exponent(most))
    scale = torch.where(old.any(-1)[:, :, None, None], torch.maximum(old_scale, need), need)
    cache["codes"][at[there]] = _stored(x, scale)[there]
    cache["scale"][at[there]] = scale[there]
    torch.add(length, count, out=s["out"]["length"])


def _plain_attend(s):
    cache, D, (B, n, Hq, _), H = s["cache"], s["case"]["D"], s["q"].shape, s["case"]["heads"]
    k, v = _values(cache, s["pages"], D)
    k = torch.cat([k, s["k"].float().transpose(1, 2)], 2)
    v = torch.cat([v, s["v"].float().transpose(1, 2)], 2)
    at = torch.arange(n, device=k.device)
    if s["mask"] is None:
        seen = (at <= at[:, None])[None]
    else:
        seen = ((s["mask"][:, :, at // 32] >> (at % 32)) & 1) != 0
    seen = seen[:, None, :, None].expand(B, 1, n, Hq // H, n).reshape(B, 1, n * (Hq // H), n)
    cached = ~_beyond(s["pages"], s["length"])
    hidden = ~torch.cat([cached.expand(B, 1, seen.shape[2], cached.shape[-1]), seen], -1)
    x = _scores(s["q"], k, D).masked_fill_(hidden, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x.sub_(m))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / total
    lse = (m + torch.log(total))[..., 0]
    s["out"]["out"].copy_(out.reshape(B, H, n, Hq // H, D).transpose(1, 2).reshape(B, n, Hq, D))
    s["out"]["lse"].copy_(lse.reshape(B, H, n, Hq // H).transpose(1, 2).reshape(B, n, Hq))


def _plain_weigh(s):
    case, H = s["case"], s["case"]["heads"]
    B, n, Hq, D = s["q"].shape
    x = _scores(s["q"], _values(s["cache"], s["pages"], D)[0], D)
    lse = s["lse"].reshape(B, n, H, Hq // H).transpose(1, 2).reshape(B, H, n * (Hq // H), 1)
    got = torch.exp(x - lse).sum(2)
    there = ~_beyond(s["pages"], s["length"])[:, 0]
    torch.where(there, s["weight"] * case["decay"] + got, torch.zeros_like(got), out=s["out"]["weight"])


def _plain_evict(s):
    case, cache, pages, D = s["case"], s["cache"], s["pages"], s["case"]["D"]
    B, H, keep = case["B"], case["heads"], case["keep"]
    length = s["length"]
    at = torch.arange(pages.shape[1] * PAGE, device=length.device)
    m = length.clamp_max(keep)
    recent = m.clamp_max(case["recent"])
    key = torch.where(at >= (length - recent)[:, None, None], torch.full_like(s["weight"], math.inf), s["weight"])
    key = torch.where(at < length[:, None, None], key, torch.full_like(key, -math.inf))
    best = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :keep]
    best = torch.nn.functional.pad(best, (0, keep - best.shape[-1]))
    j = torch.arange(keep, device=length.device)
    kept = torch.where(j < m[:, None, None], best, torch.full_like(best, at.numel())).sort(-1).values
    there = j < m[:, None, None]
    s["out"]["kept"].copy_(torch.where(there, kept, torch.full_like(kept, -1)))
    W = s["new_pages"].shape[1]
    kept = torch.nn.functional.pad(torch.where(there, kept, torch.zeros_like(kept)), (0, W * PAGE - keep))
    there = torch.nn.functional.pad(there.expand(B, H, keep), (0, W * PAGE - keep))
    s["out"]["weight"].copy_(torch.where(there, s["weight"].gather(-1, kept), torch.zeros_like(kept, dtype=torch.float32)))
    s["out"]["length"].copy_(m)
    x = torch.stack(_values(cache, pages, D), 2)                   # [B, heads, 2, tokens, D]
    x = x.gather(3, kept[:, :, None, :, None].expand(B, H, 2, W * PAGE, D))
    x = torch.where(there[:, :, None, :, None], x, torch.zeros_like(x))
    source = pages.long().clamp_min(0)[:, None].expand(B, H, -1).gather(2, torch.div(kept, PAGE, rounding_mode="floor"))
    scale = cache["scale"][source, torch.arange(H, device=source.device)[:, None]]              # [B, heads, tokens, 2]
    scale = torch.where(there[..., None], scale, torch.zeros_like(scale)).reshape(B, H, W, PAGE, 2).amax(3)
    x = x.reshape(B, H, 2, W, PAGE, D).permute(0, 3, 1, 2, 4, 5)
    scale = scale.transpose(1, 2)
    used = s["new_pages"] >= 0
    to = s["new_pages"].long()[used]
    cache["codes"][to] = _stored(x, scale)[used]
    cache["scale"][to] = scale[used]


def _outputs(s):
    """What a pass has made.  Codes as the numbers that they stand for, in units of the scales beside them."""
    out, op = s["out"], s["case"]["op"]
    got = {name: x for name, x in out.items() if name != "status"}
    if op in ("append", "evict"):
        got["codes"] = s["cache"]["codes"].view(torch.float8_e4m3fn)
        got["scale"] = s["cache"]["scale"]
    return got


def run(s):
    case, cache = s["case"], s["cache"]
    if own:
        from paper_2512_16273_amd import tslt
        if case["op"] == "append":
            tslt.cache_append(cache, s["pages"], s["length"], s["k"], s["v"], count=s["count"], index=s["index"], out=s["out"])
        elif case["op"] == "attend":
            tslt.cache_attend(s["q"], cache, s["pages"], s["length"], k=s["k"], v=s["v"], mask=s["mask"], out=s["out"],
                              workspace=s["workspace"])
        elif case["op"] == "weigh":
            tslt.cache_weigh(s["q"], s["lse"], cache, s["pages"], s["length"], s["weight"], decay=case["decay"], out=s["out"])
        else:
            tslt.cache_evict(cache, s["pages"], s["length"], s["weight"], keep=case["keep"], recent=case["recent"],
                             new_pages=s["new_pages"], out=s["out"])
    else:
        {"append": _plain_append, "attend": _plain_attend, "weigh": _plain_weigh, "evict": _plain_evict}[case["op"]](s)
    return _outputs(s)


# ---- in 64 bits, from the definitions ---------------------------------------------------------------------------

def _two_to(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)  # (a library's power may be off in its last bit)


def _decoded(codes):
    """e4m3 by its fields: sign, exponent with bias 7 (0: subnormal), three bits of mantissa."""
    b = codes.to(torch.int64)
    e, m = (b >> 3) & 15, (b & 7).double()
    mag = torch.where(e > 0, (1 + m / 8) * _two_to(e - 7), m / 8 * 2.0 ** -6)
    return torch.where(b >= 128, -mag, mag)


def _nearest(x):
    """The nearest e4m3 number, ties to the even one."""
    mag = x.abs().clamp(max=448.0)
    e = torch.floor(torch.log2(mag.clamp(min=2.0 ** -6))).clamp(min=-6)
    e = torch.where(_two_to(e) > mag, (e - 1).clamp(min=-6), e)       # (a logarithm may be rounded up to the next whole number)
    step = _two_to(e - 3)
    return torch.copysign((mag / step).round() * step, x)


def _head(cache, page_ids, h, tokens, D):
    """Keys and values of the first `tokens` tokens of one head of one sequence."""
    ids = page_ids.long()
    s = cache["scale"][ids, h].double()
    k = _decoded(cache["codes"][ids, h, 0]).view(-1, PAGE, D) * s[:, 0, None, None]
    v = _decoded(cache["codes"][ids, h, 1]).view(-1, 4, D, 16).transpose(2, 3).reshape(-1, PAGE, D) * s[:, 1, None, None]
    return k.reshape(-1, D)[:tokens], v.reshape(-1, D)[:tokens]


def _held(x, scale):
    """One head's [tokens <= 64, D] keys or values in units of their scale, with zeros up to a page."""
    c = torch.zeros(PAGE, x.shape[1], dtype=torch.float64, device=x.device)
    c[:x.shape[0]] = _nearest(x / scale)
    return c


def _power(x):
    """The least power of two that brings x to 448 or less, in Python's own numbers."""
    e = MIN_EXP
    if x > 448.0 * 2.0 ** MIN_EXP:
        e = math.frexp(x / 448.0)[1] - 1
        while 448.0 * 2.0 ** e < x:
            e += 1
    return 2.0 ** e


def exact(case, seed):
    op, B, H, D, lengths = case["op"], case["B"], case["heads"], case["D"], _lengths(case)
    steps = {"append": B * H * (-(-case.get("n", 0) // PAGE) + 1), "evict": B * H * (-(-case.get("keep", 0) // PAGE)), "attend": B * H,
             "weigh": B * H}[op]
    if steps > 40000:
        return None
    s = prepare(case, seed)
    cache, pages, n = s["cache"], s["pages"], case.get("n", 0)
    if op in ("append", "evict"):
        values = _decoded(cache["codes"]) if cache["codes"].numel() < 3 << 29 else None
        if values is None:
            return None
        scale = cache["scale"].double()
    if op == "append":
        for b in range(B):
            rows = s["index"][b].long() if s["index"] is not None else torch.arange(n, device=DEV)
            rows = rows[:_counts(case)[b]]
            kv = [x[b][rows].double() for x in (s["k"], s["v"])]
            start, end = lengths[b], lengths[b] + rows.numel()
            page = pages[b].tolist()
            for w in range(start // PAGE, -(-end // PAGE)):
                lo, hi = max(start, w * PAGE), min(end, (w + 1) * PAGE)
                before = lo - w * PAGE
                ks = [x[lo - start:hi - start] for x in kv]
                most = torch.stack([x.abs().amax((0, 2)) for x in ks], 1).tolist()
                for h in range(H):
                    held = _head(cache, pages[b, w:w + 1], h, before, D)
                    for part in (0, 1):
                        to = _power(most[h][part])
                        if before:
                            to = max(to, float(scale[page[w], h, part]))
                        c = _held(torch.cat([held[part], ks[part][:, h]]), to)
                        values[page[w], h, part] = (c if part == 0 else c.view(4, 16, D).transpose(1, 2)).reshape(-1)
                        scale[page[w], h, part] = to
        return dict(length=None, codes=values, scale=scale)
    if op == "evict":
        weights = torch.zeros(B, H, s["new_pages"].shape[1] * PAGE, dtype=torch.float64, device=DEV)
        for b in range(B):
            L, m = lengths[b], min(lengths[b], case["keep"])
            recent = min(case["recent"], m)
            for h in range(H):
                w = s["weight"][b, h, :L - recent].double()
                first = torch.sort(-w, stable=True).indices[:m - recent]
                kept = torch.cat([first.sort().values, torch.arange(L - recent, L, device=DEV)])
                weights[b, h, :m] = s["weight"][b, h, kept].double()
                from_scale = scale[pages[b, kept // PAGE].long(), h]
                k, v = _head(cache, pages[b, :-(-L // PAGE)], h, L, D)
                for w0 in range(0, m, PAGE):
                    p = int(s["new_pages"][b, w0 // PAGE])
                    to = from_scale[w0:w0 + PAGE].amax(0)
                    for part, x in ((0, k), (1, v)):
                        c = _held(x[kept[w0:w0 + PAGE]], to[part])
                        values[p, h, part] = (c if part == 0 else c.view(4, 16, D).transpose(1, 2)).reshape(-1)
                    scale[p, h] = to
        return dict(length=None, kept=None, weight=weights, codes=values, scale=scale)
    Hq, G = case["heads_q"], case["heads_q"] // H
    out = torch.zeros(B, n, Hq, D, dtype=torch.float64, device=DEV)
    lse = torch.zeros(B, n, Hq, dtype=torch.float64, device=DEV)
    weight = torch.zeros(B, H, pages.shape[1] * PAGE, dtype=torch.float64, device=DEV)
    if op == "attend":
        seen = torch.ones(n, n, dtype=torch.bool, device=DEV).tril()
        if s["mask"] is not None:
            at = torch.arange(n, device=DEV)
            seen = (torch.bitwise_right_shift(s["mask"][0][:, torch.div(at, 32, rounding_mode="floor")], at % 32) & 1).bool()
    for b in range(B):
        L = lengths[b]
        for h in range(H):
            k, v = _head(cache, pages[b, :-(-L // PAGE)], h, L, D)
            for i in range(h * G, (h + 1) * G):
                x = s["q"][b, :, i].double() @ k.t() / math.sqrt(D)
                if op == "weigh":
                    weight[b, h, :L] += torch.exp(x - s["lse"][b, :, i].double()[:, None]).sum(0)
                    continue
                y = s["q"][b, :, i].double() @ s["k"][b, :, h].double().t() / math.sqrt(D)
                x = torch.cat([x, torch.where(seen, y, torch.full_like(y, -math.inf))], 1)
                z = torch.logsumexp(x, 1)
                out[b, :, i] = torch.exp(x - z[:, None]) @ torch.cat([v, s["v"][b, :, h].double()])
                lse[b, :, i] = z
            if op == "weigh":
                weight[b, h, :L] += s["weight"][b, h, :L].double() * case["decay"]
    return dict(weight=weight) if op == "weigh" else dict(out=out, lse=lse)
