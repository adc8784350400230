"""The calls beside attention and verification that a round of many requests makes, over the sizes it makes them at.

  adapt            each sequence's own low-rank adapter, added to what a shared projection gave its tokens
  rotate           queries and keys of every head normed, and rotated by their tokens' positions, before they are attended to or cached
  rotate_backward  the gradients of the rows and of the norms' weights
  logprob          of rows of logits the given token's log probability, the entropy and the likeliest tokens: what a server answers with
                   beside the tokens that it has verified
  logprob_backward the gradient of the logits, for a draft model that learns from them
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
DEV = "cuda"
EPS = 1e-6


def listed():
    return [
        # one decoded token of one user: nothing but latency and one adapter
        dict(name="adapt_one", op="adapt", B=1, n=1, K=4096, N=4096, rank=16, adapters=8, ragged=False, dtype="bf16"),
        # a round of 256 chains of 8 draft tokens and the one before them, 48 adapters between them, some sequences without
        dict(name="adapt_chain_256", op="adapt", B=256, n=9, K=4096, N=6144, rank=16, adapters=48, ragged=True, dtype="bf16"),
        # whole prompts of four users, adapters of a higher rank
        dict(name="adapt_prompt", op="adapt", B=4, n=2001, K=4096, N=6144, rank=64, adapters=4, ragged=False, dtype="f16"),
        # one draft token on the device, heads of the paper's draft model (12 of 64, FP16), no norms
        dict(name="rotate_one", op="rotate", B=1, n=1, heads_q=12, heads=12, D=64, rotary=64, axes=1, shared=False, adjacent=False,
             norm=False, far=2000, ragged=False, dtype="f16"),
        # a batch of trees of 21 nodes in long contexts: a node's position is its sequence's and its depth
        dict(name="rotate_tree_64", op="rotate", B=64, n=21, heads_q=32, heads=8, D=128, rotary=128, axes=1, shared=True, adjacent=False,
             norm=True, far=130000, ragged=False, dtype="bf16"),
        # prompts of text, images and video: three axes
        dict(name="rotate_prompt_axes", op="rotate", B=4, n=4001, heads_q=32, heads=8, D=128, rotary=128, axes=3, shared=False, adjacent=False,
             norm=True, far=0, ragged=True, dtype="bf16"),
        # a short sequence of the draft model's, learned from
        dict(name="rotate_backward_short", op="rotate_backward", B=1, n=64, heads_q=12, heads=12, D=64, rotary=32, axes=1, shared=False,
             adjacent=True, norm=True, far=0, ragged=False, dtype="f32"),
        # a training batch
        dict(name="rotate_backward_batch", op="rotate_backward", B=8, n=2048, heads_q=32, heads=8, D=128, rotary=128, axes=1, shared=False,
             adjacent=False, norm=True, far=0, ragged=False, dtype="bf16"),
        # one user's chain of 8 draft tokens, the benchmark's large vocabulary, with alternatives
        dict(name="logprob_round", op="logprob", B=1, n=9, m=9, V=128256, pad=0, T=0.7, top=20, chosen=False, ragged=False, masked=False,
             dtype="bf16"),
        # the benchmark's batch of 256 chains: every row, as all may be accepted
        dict(name="logprob_chain_256", op="logprob", B=256, n=9, m=9, V=128256, pad=0, T=0.7, top=5, chosen=False, ragged=False,
             masked=False, dtype="bf16"),
        # a draft model's logits over one accepted chain
        dict(name="logprob_backward_chain", op="logprob_backward", B=1, n=9, V=32000, pad=0, T=1.0, top=0, ragged=False, masked=False,
             dtype="f16"),
        # a training batch
        dict(name="logprob_backward_batch", op="logprob_backward", B=8, n=256, V=128256, pad=0, T=1.0, top=0, ragged=True, masked=False,
             dtype="bf16"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    op = rng.choice(["adapt", "adapt", "rotate", "rotate_backward", "logprob", "logprob", "logprob_backward"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    B = log_int(1, 256)
    n = log_int(1, 17) if rng.random() < 0.6 else log_int(18, 2500)
    ragged = rng.random() < 0.5
    if op == "adapt":
        K, N, rank = 8 * log_int(16, 1024), 8 * log_int(16, 1400), rng.choice([3, 8, 16, 16, 32, 64, 128])
        most = min(80_000_000 // ((K + 2 * N) * (2 if dtype == "f32" else 1)), 8_000_000_000 // (2 * rank * (K + N)))
        n = max(1, min(n, most))
        B = max(1, min(B, most // n))
        return dict(op=op, B=B, n=n, K=K, N=N, rank=rank, adapters=log_int(1, 64), ragged=ragged, dtype=dtype)
    if op in ("rotate", "rotate_backward"):
        D = rng.choice([64, 128, 128, 256])
        heads, group = rng.choice([1, 2, 4, 5, 8, 12, 32]), rng.choice([1, 1, 2, 3, 4, 4, 7, 8])
        most = (40_000_000 if dtype == "f32" else 80_000_000) // (heads * (group + 2) * D)
        n = max(1, min(n, most))
        axes = rng.choice([1, 1, 1, 2, 3, 4])
        return dict(op=op, B=max(1, min(B, most // n)), n=n, heads_q=heads * group, heads=heads, D=D, rotary=rng.choice([D, D, D // 2, D // 4]),
                    axes=axes, shared=rng.random() < 0.5, adjacent=rng.random() < 0.3, norm=rng.random() < 0.7,
                    far=rng.choice([0, log_int(10, 1_000_000)]), ragged=ragged, dtype=dtype)
    V = log_int(1000, 256000)
    most = 540_000_000 // (V * BYTES[dtype])
    if op == "logprob_backward":
        most //= 2
    n = max(1, min(n, most))
    case = dict(op=op, B=max(1, min(B, most // n)), n=n, V=V, pad=rng.choice([0, 0, rng.randrange(0, 64)]), T=rng.choice([1.0, 1.0, 0.7, 1.3]),
                top=rng.choice([0, 0, 1, 5, 20, 32]), ragged=ragged, masked=rng.random() < 0.3, dtype=dtype)
    if op == "logprob":
        case["chosen"] = rng.random() < 0.4
        case["m"] = rng.randint(1, n) if case["chosen"] else n
    return case


# ---- what a case says about its sizes -------------------------------------------------------------------------

def _counts(case):
    """How many of its tokens (rows) each sequence has: all, or 1 and more in no order."""
    m = case.get("m", case["n"])
    return [1 + m * ((b * 89 + 55) % 144) // 144 if case["ragged"] else m for b in range(case["B"])]


def _adapter_of(case):
    """Each sequence's adapter; where there are several, one of eight sequences has none."""
    return [-1 if case["adapters"] > 1 and b % 8 == 5 else (b * 29 + b // 7) % case["adapters"] for b in range(case["B"])]


def _ranks(case):
    """Each adapter's own rank: most have the largest."""
    return [case["rank"] if a % 4 != 3 else max(1, case["rank"] // 2) for a in range(case["adapters"])]


def work(case):
    op, e, tokens = case["op"], BYTES[case["dtype"]], sum(_counts(case))
    if op == "adapt":
        ranks, ids, each = _ranks(case), _adapter_of(case), case["K"] + case["N"]
        used = sum(ranks[a] for a in set(ids) if a >= 0)
        return {"bytes": e * (sum(c * (2 * case["N"] + (case["K"] if a >= 0 else 0)) for c, a in zip(_counts(case), ids)) + used * each),
                "flops": sum(2 * c * ranks[a] * each for c, a in zip(_counts(case), ids) if a >= 0)}
    if op in ("rotate", "rotate_backward"):
        row = (case["heads_q"] + case["heads"]) * case["D"]
        places = (case["n"] if case["shared"] else case["B"] * case["n"]) * case["axes"] * 4
        return {"bytes": tokens * row * e * (2 if op == "rotate" else 3) + places, "flops": tokens * row * (6 if op == "rotate" else 14)}
    more = tokens * (8 + 8 * case["top"])
    if op == "logprob":
        return {"bytes": tokens * case["V"] * e + more, "flops": 6 * tokens * case["V"]}
    return {"bytes": (tokens + case["B"] * case["n"]) * case["V"] * e + more, "flops": 6 * tokens * case["V"]}


# ---- inputs -----------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(1000003 * int(seed) + 29)


def _logits(case, g):
    """Gaussian rows with a rank bias through no particular order, each in rows of V and `pad` more.  Where a grammar masks them,
    every fourth row has a few tokens left and the others at -inf."""
    B, n, V = case["B"], case["n"], case["V"]
    z = torch.zeros(B * n, V + case["pad"], dtype=DTYPES[case["dtype"]], device=DEV)
    chunk = max(1, (1 << 26) // V)
    for r in range(0, B * n, chunk):
        m = min(chunk, B * n - r)
        x = 2.0 * torch.randn(m, V, generator=g, device=DEV)
        x -= torch.log1p(V * torch.rand(m, V, generator=g, device=DEV))
        if case["masked"]:
            allowed = torch.rand(m, V, generator=g, device=DEV) < 12.0 / V
            allowed[:, :2] = True
            x = torch.where(allowed | (torch.arange(r, r + m, device=DEV) % 4 != 1)[:, None], x, torch.full_like(x, -math.inf))
        z[r:r + m, :V] = x
    return z.view(B, n, V + case["pad"])[:, :, :V]


def _sampled(z, T, g):
    """A token of every row, drawn from its distribution."""
    got = []
    flat = z.reshape(-1, z.shape[-1])
    chunk = max(1, (1 << 26) // z.shape[-1])
    for r in range(0, flat.shape[0], chunk):
        x = flat[r:r + chunk].float() / T
        got.append((x - torch.log(-torch.log(torch.rand(x.shape, generator=g, device=DEV).clamp(1e-7, 1 - 1e-7)))).argmax(-1))
    return torch.cat(got).view(z.shape[:2]).to(torch.int32)


def _positions(case, g):
    """[B or 1, n, axes]: a tree's depths, a chain's places, or a grid's coordinates after some text."""
    B, n, axes = case["B"], case["n"], case["axes"]
    i = torch.arange(n, device=DEV)
    rows = []
    for b in range(1 if case["shared"] else B):
        if axes == 1:
            rows.append(torch.floor(torch.log2(3.0 * i + 1) / 2).long()[:, None] if case["shared"] else i[:, None])
            continue
        text, side = min(n, 16 + 3 * b), max(2, int(round(max(n - 16, 1) ** (1 / 3))) + b % 3)
        j = (i - text).clamp_min(0)
        grid = torch.stack([j // (side * side), j // side % side, j % side, j % (side + 1)][:axes], 1) + text
        rows.append(torch.where((i < text)[:, None], i[:, None].expand(n, axes), grid))
    return torch.stack(rows).to(torch.int32).contiguous()


def prepare(case, seed):
    g = _gen(seed)
    B, n, op, dt = case["B"], case["n"], case["op"], DTYPES[case["dtype"]]
    state = dict(case=case, workspace=torch.empty(256 << 20, dtype=torch.uint8, device=DEV))
    state["count"] = torch.tensor(_counts(case), dtype=torch.int32, device=DEV) if case["ragged"] else None

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)
    if op == "adapt":
        K, N, R, ranks = case["K"], case["N"], case["rank"], _ranks(case)
        held = -(-R // 16) * 16                                    # ranks are laid out in sixteens; what lies behind an adapter's own does not count
        spread = torch.where(torch.rand(K, generator=g, device=DEV) < 0.01, 8.0, 1.0)
        state.update(x=(normal(B, n, K) * spread).to(dt), base=normal(B, n, N).to(dt),
                     a=(normal(case["adapters"], held, K) * K ** -0.5).to(dt), b=(normal(case["adapters"], N, held) * 0.3 * R ** -0.5).to(dt),
                     adapter=torch.tensor(_adapter_of(case), dtype=torch.int32, device=DEV),
                     scale=torch.rand(case["adapters"], generator=g, device=DEV) + 0.5,
                     rank=torch.tensor(ranks, dtype=torch.int32, device=DEV),
                     out=dict(out=torch.zeros(B, n, N, dtype=dt, device=DEV), status=torch.zeros(B, dtype=torch.int32, device=DEV)))
        return state
    if op in ("rotate", "rotate_backward"):
        Hq, H, D, R = case["heads_q"], case["heads"], case["D"], case["rotary"]
        # queries, keys and values as one projection leaves them: side by side
        x = (normal(B, n, Hq + 2 * H, D) * (torch.rand(Hq + 2 * H, D, generator=g, device=DEV) + 0.5)).to(dt)
        state.update(q=x[:, :, :Hq], k=x[:, :, Hq:Hq + H], position=_positions(case, g),
                     freq=(500000.0 if D > 64 else 10000.0) ** (-torch.arange(R // 2, device=DEV, dtype=torch.float64) * 2 / R))
        state["freq"] = state["freq"].to(torch.float32)
        state["axis"] = None if case["axes"] == 1 else (torch.arange(R // 2, device=DEV) * case["axes"] // (R // 2)).to(torch.int32)
        state["base"] = torch.tensor([case["far"] - case["far"] * b // (2 * B) for b in range(B)], dtype=torch.int32, device=DEV) if case["far"] else None
        state["weights"] = (1 + 0.2 * normal(D), 1 + 0.2 * normal(D)) if case["norm"] else (None, None)
        state["out"] = dict(q=torch.zeros(B, n, Hq, D, dtype=dt, device=DEV), k=torch.zeros(B, n, H, D, dtype=dt, device=DEV),
                            status=torch.zeros(B, dtype=torch.int32, device=DEV))
        if op == "rotate_backward":
            state.update(grad_q=normal(B, n, Hq, D).to(dt), grad_k=normal(B, n, H, D).to(dt))
            if case["norm"]:
                state["out"].update(q_weight=torch.zeros(D, device=DEV), k_weight=torch.zeros(D, device=DEV))
        return state
    z, top = _logits(case, g), case["top"]
    state["logits"] = z
    m = case.get("m", n)
    if op == "logprob":
        state["index"] = None
        if case["chosen"]:                                         # a path's rows, in order
            state["index"] = torch.rand(B, n, generator=g, device=DEV).argsort(1)[:, :m].sort(1).values.to(torch.int32).contiguous()
        tokens = _sampled(z, case["T"], g)
        state["tokens"] = (tokens if state["index"] is None else tokens.gather(1, state["index"].long())).contiguous()
        state["out"] = dict(logp=torch.zeros(B, m, device=DEV), entropy=torch.zeros(B, m, device=DEV), lse=torch.zeros(B, m, device=DEV),
                            status=torch.zeros(B, m, dtype=torch.int32, device=DEV))
        if top:
            state["out"].update(top_idx=torch.zeros(B, m, top, dtype=torch.int32, device=DEV), top_logp=torch.zeros(B, m, top, device=DEV))
        return state
    state["tokens"] = _sampled(z, case["T"], g)
    lse, entropy, idx = [], [], []
    flat, chunk = z.reshape(B * n, -1), max(1, (1 << 26) // case["V"])
    for r in range(0, B * n, chunk):                               # what the forward call has left
        s = flat[r:r + chunk].double() * _inverse(case)
        lse.append(torch.logsumexp(s, -1))
        d = s - lse[-1][:, None]
        entropy.append(-torch.where(d > -math.inf, torch.exp(d) * d, torch.zeros_like(d)).sum(-1))
        if top:
            v, i = torch.topk(s, top, dim=-1)
            idx.append(torch.where(v > -math.inf, i, torch.full_like(i, -1)))
    state.update(lse=torch.cat(lse).view(B, n).float(), entropy=torch.cat(entropy).view(B, n).float(),
                 top_idx=torch.cat(idx).view(B, n, top).to(torch.int32) if top else None,
                 grad_top=0.1 * normal(B, n, top) if top else None,
                 grad_logp=-torch.rand(B, n, generator=g, device=DEV) - 0.1, grad_entropy=0.05 * normal(B, n),
                 out=dict(logits=torch.zeros(B, n, case["V"], dtype=dt, device=DEV)))
    return state


def _inverse(case):
    """1 / T as a number of 32 bits, as the library takes it."""
    return float(torch.tensor(1.0) / torch.tensor(case["T"], dtype=torch.float32))


# ---- the plain form ---------------------------------------------------------------------------------------------

def _here(s, m):
    """[B, m]: which tokens (rows) there are."""
    at = torch.arange(m, device=DEV)
    B = s["case"]["B"]
    return torch.ones(B, m, dtype=torch.bool, device=DEV) if s["count"] is None else at < s["count"][:, None]


def _keep(out, there, made):
    """What belongs to no token stays as it was."""
    there = there.view(*there.shape, *[1] * (out.dim() - there.dim()))
    out.copy_(torch.where(there, made.to(out.dtype), out))


def _plain_adapt(s):
    R = s["a"].shape[1]
    at = s["adapter"].long().clamp_min(0)
    h = torch.matmul(s["x"].float(), s["a"][at].float().transpose(1, 2))
    h = torch.where((torch.arange(R, device=DEV) < s["rank"][at][:, None])[:, None], h, torch.zeros_like(h)) * s["scale"][at][:, None, None]
    y = torch.matmul(h, s["b"][at].float().transpose(1, 2))
    y = s["base"].float() + torch.where((s["adapter"] >= 0)[:, None, None], y, torch.zeros_like(y))
    _keep(s["out"]["out"], _here(s, s["case"]["n"]), y)


def _turns(s):
    """cos and sin of every pair's angle, [B, n, 1, pairs]; the angles in 64 bits, as positions may be far."""
    case, at = s["case"], s["position"].long()
    if s["base"] is not None:
        at = at + s["base"].long()[:, None, None]
    at = at.expand(case["B"], case["n"], case["axes"])
    at = at.expand(*at.shape[:2], s["freq"].numel()) if s["axis"] is None else at[:, :, s["axis"].long()]
    angle = at.double() * s["freq"].double()
    return torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]


def _pairs(x, case):
    """The two numbers of every pair, and the channels that are not rotated."""
    R = case["rotary"]
    if case["adjacent"]:
        return x[..., 0:R:2], x[..., 1:R:2], x[..., R:]
    return x[..., :R // 2], x[..., R // 2:R], x[..., R:]


def _joined(a, b, rest, case):
    return torch.cat([torch.stack([a, b], -1).flatten(-2), rest] if case["adjacent"] else [a, b, rest], -1)


def _plain_rotate(s):
    case, (cos, sin) = s["case"], _turns(s)
    for name, w in (("q", s["weights"][0]), ("k", s["weights"][1])):
        x = s[name].float()
        if case["norm"]:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
        a, b, rest = _pairs(x, case)
        _keep(s["out"][name], _here(s, case["n"]), _joined(a * cos - b * sin, b * cos + a * sin, rest, case))


def _plain_rotate_backward(s):
    case, (cos, sin) = s["case"], _turns(s)
    there = _here(s, case["n"])[:, :, None, None]
    for name, w in (("q", s["weights"][0]), ("k", s["weights"][1])):
        x = s[name].float()
        a, b, rest = _pairs(s["grad_" + name].float(), case)
        dy = _joined(a * cos + b * sin, b * cos - a * sin, rest, case)
        if case["norm"]:
            r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
            xr = x * r
            s["out"][name + "_weight"].copy_(torch.where(there, dy * xr, torch.zeros_like(xr)).double().sum((0, 1, 2)))
            dy = dy * w
            dy = r * (dy - xr * (dy * xr).mean(-1, keepdim=True))
        s["out"][name].copy_(torch.where(there, dy, torch.zeros_like(dy)))


def _plain_logprob(s):
    case, out, m = s["case"], s["out"], s["tokens"].shape[1]
    z = s["logits"].float()
    if s["index"] is not None:
        z = z.gather(1, s["index"].long()[:, :, None].expand(-1, -1, z.shape[2]))
    x = z * _inverse(case)
    most = x.amax(-1, keepdim=True)
    d = x - most
    e = torch.exp(d)
    total = e.sum(-1, keepdim=True)
    lse = most + torch.log(total)
    entropy = torch.log(total) - torch.where(d > -math.inf, e * d, torch.zeros_like(d)).sum(-1, keepdim=True) / total
    there = _here(s, m)
    _keep(out["lse"], there, lse[..., 0])
    _keep(out["entropy"], there, entropy[..., 0])
    _keep(out["logp"], there, (x.gather(2, s["tokens"].long()[..., None]) - lse)[..., 0])
    if case["top"]:
        # numbers in their order as whole numbers, the lower index first among equals
        bits = (z + 0.0).view(torch.int32).long()
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
        best = torch.topk(order * 2 ** 32 - torch.arange(z.shape[2], device=DEV), case["top"], dim=-1).values
        idx = torch.remainder(-best, 2 ** 32)
        value = x.gather(2, idx)
        _keep(out["top_idx"], there, torch.where(value > -math.inf, idx, torch.full_like(idx, -1)))
        _keep(out["top_logp"], there, value - lse)


def _plain_logprob_backward(s):
    case, (B, n, V) = s["case"], s["logits"].shape
    d = s["logits"].float() * _inverse(case) - s["lse"][..., None]
    g, gH = s["grad_logp"], s["grad_entropy"]
    all_g = g if s["grad_top"] is None else g + torch.where(s["top_idx"] >= 0, s["grad_top"], torch.zeros_like(s["grad_top"])).sum(-1)
    dz = -torch.exp(d) * (all_g[..., None] + torch.where(d > -math.inf, gH[..., None] * (d + s["entropy"][..., None]), torch.zeros_like(d)))
    dz.scatter_add_(2, s["tokens"].long()[..., None], g[..., None])
    if s["grad_top"] is not None:
        dz.scatter_add_(2, s["top_idx"].long().clamp_min(0), torch.where(s["top_idx"] >= 0, s["grad_top"], torch.zeros_like(s["grad_top"])))
    dz = torch.where(_here(s, n)[..., None], dz * _inverse(case), torch.zeros_like(dz))
    s["out"]["logits"].copy_(dz)


def run(s):
    case, op, out = s["case"], s["case"]["op"], s["out"]
    if own:
        from paper_2512_16273_amd import tslt
        if op == "adapt":
            tslt.adapt(s["x"], s["base"], s["a"], s["b"], s["adapter"], scale=s["scale"], rank=s["rank"], count=s["count"], out=out,
                       workspace=s["workspace"])
        elif op == "rotate":
            tslt.rotate(s["q"], s["k"], s["position"], s["freq"], axis=s["axis"], base=s["base"], q_weight=s["weights"][0],
                        k_weight=s["weights"][1], eps=EPS if case["norm"] else None, adjacent=case["adjacent"], count=s["count"], out=out)
        elif op == "rotate_backward":
            tslt.rotate_backward(s["grad_q"], s["grad_k"], s["q"], s["k"], s["position"], s["freq"], axis=s["axis"], base=s["base"],
                                 q_weight=s["weights"][0], k_weight=s["weights"][1], eps=EPS if case["norm"] else None,
                                 adjacent=case["adjacent"], count=s["count"], out=out, workspace=s["workspace"])
        elif op == "logprob":
            tslt.logprob(s["logits"], case["T"], s["tokens"], top=case["top"], index=s["index"], count=s["count"], out=out,
                         workspace=s["workspace"])
        else:
            tslt.logprob_backward(s["logits"], case["T"], s["tokens"], s["lse"], s["entropy"], grad_logp=s["grad_logp"],
                                  grad_entropy=s["grad_entropy"], top_idx=s["top_idx"], grad_top=s["grad_top"], count=s["count"], out=out)
    else:
        {"adapt": _plain_adapt, "rotate": _plain_rotate, "rotate_backward": _plain_rotate_backward, "logprob": _plain_logprob,
         "logprob_backward": _plain_logprob_backward}[op](s)
    return {name: x for name, x in out.items() if name != "status"}


# ---- in 64 bits, from the definitions ---------------------------------------------------------------------------

def _rotation(case, s, b, transposed):
    """[n, D, D]-products are not needed: cos and sin of every channel, and its partner's channel and sign, of one sequence's tokens."""
    n, D, R = case["n"], case["D"], case["rotary"]
    cos, sin = torch.ones(n, D, dtype=torch.float64, device=DEV), torch.zeros(n, D, dtype=torch.float64, device=DEV)
    partner = torch.arange(D, device=DEV)
    at = s["position"][0 if case["shared"] else b].double()
    far = 0 if s["base"] is None else int(s["base"][b])
    for j in range(R // 2):
        first, second = (2 * j, 2 * j + 1) if case["adjacent"] else (j, j + R // 2)
        axis = 0 if s["axis"] is None else int(s["axis"][j])
        angle = (at[:, axis] + far) * float(s["freq"][j])
        if transposed:
            angle = -angle
        cos[:, first] = cos[:, second] = torch.cos(angle)
        sin[:, first], sin[:, second] = -torch.sin(angle), torch.sin(angle)
        partner[first], partner[second] = second, first
    return cos, sin, partner


def exact(case, seed):
    op, B, n = case["op"], case["B"], case["n"]
    if op in ("rotate", "rotate_backward") and B * case["rotary"] > 24000:
        return None
    s = prepare(case, seed)
    counts = _counts(case)
    if op == "adapt":
        out, ids, ranks = s["out"]["out"].double(), _adapter_of(case), _ranks(case)
        for b in range(B):
            x = s["base"][b, :counts[b]].double()
            if ids[b] >= 0:
                r = ranks[ids[b]]
                x = x + float(s["scale"][ids[b]]) * ((s["x"][b, :counts[b]].double() @ s["a"][ids[b], :r].double().t()) @ s["b"][ids[b], :, :r].double().t())
            out[b, :counts[b]] = x
        return dict(out=out)
    if op in ("rotate", "rotate_backward"):
        got = {}
        for name, w in (("q", s["weights"][0]), ("k", s["weights"][1])):
            y = torch.zeros(s[name].shape, dtype=torch.float64, device=DEV)
            dw = torch.zeros(case["D"], dtype=torch.float64, device=DEV)
            for b in range(B):
                c = counts[b]
                cos, sin, partner = (t if t.dim() == 1 else t[:c, None] for t in _rotation(case, s, b, op == "rotate_backward"))
                x = s[name][b, :c].double()
                root = torch.sqrt((x ** 2).sum(-1, keepdim=True) / case["D"] + EPS) if case["norm"] else 1.0
                if op == "rotate":
                    if case["norm"]:
                        x = x / root * w.double()
                    y[b, :c] = cos * x + sin * x[..., partner]
                    continue
                g = s["grad_" + name][b, :c].double()
                g = cos * g + sin * g[..., partner]
                if case["norm"]:
                    dw += (g * x / root).sum((0, 1))
                    g = g * w.double()
                    g = g / root - x * (g * x).sum(-1, keepdim=True) / (case["D"] * root ** 3)
                y[b, :c] = g
            got[name] = y
            if op == "rotate_backward" and case["norm"]:
                got[name + "_weight"] = dw
        order = ["q", "k", "q_weight", "k_weight"]
        return {name: got[name] for name in order if name in got}
    rT, V = _inverse(case), case["V"]
    if op == "logprob":
        out = {name: s["out"][name].double() for name in s["out"] if name not in ("status", "top_idx")}
        for b in range(B):
            rows = s["logits"][b] if s["index"] is None else s["logits"][b][s["index"][b].long()]
            c = counts[b]
            step = max(1, (1 << 26) // V)
            for r in range(0, c, step):
                to = min(c, r + step)
                x = rows[r:to].double() * rT
                lse = torch.logsumexp(x, -1)
                logp = x - lse[:, None]
                out["lse"][b, r:to] = lse
                out["logp"][b, r:to] = logp.gather(1, s["tokens"][b, r:to].long()[:, None])[:, 0]
                out["entropy"][b, r:to] = torch.special.entr(torch.exp(logp)).sum(-1)
                if case["top"]:
                    out["top_logp"][b, r:to] = torch.topk(logp, case["top"], dim=-1).values
        names = ["logp", "entropy", "lse"] + (["top_idx", "top_logp"] if case["top"] else [])
        return {name: out.get(name) for name in names}
    dz = torch.zeros(B, n, V, dtype=torch.float64, device=DEV)
    for b in range(B):
        c = counts[b]
        x = s["logits"][b, :c].double() * rT - s["lse"][b, :c].double()[:, None]
        p = torch.exp(x)
        g, gH, H = (s[name][b, :c].double()[:, None] for name in ("grad_logp", "grad_entropy", "entropy"))
        y = -g * p - gH * p * torch.where(p > 0, x + H, torch.zeros_like(x))
        if case["top"]:
            gt = torch.where(s["top_idx"][b, :c] >= 0, s["grad_top"][b, :c], torch.zeros_like(s["grad_top"][b, :c])).double()
            y -= p * gt.sum(-1, keepdim=True)
            y.scatter_add_(1, s["top_idx"][b, :c].long().clamp_min(0), gt)
        y.scatter_add_(1, s["tokens"][b, :c].long()[:, None], g)
        dz[b, :c] = y * rT
    return dict(logits=dz)
