"""The calls around attention and verification as they are used: a server's round, and a step of a model that learns."""
import numpy as np
import pytest
import torch

from oracle import round_oracle as O
from paper_2512_16273_amd import tslt

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = float("inf")


def test_rounds_of_users_with_adapters():
    from examples import adapted_tree_rounds as example
    a = example.main(rounds=12, B=5, report=lambda _: None)
    assert all(12 <= n <= 48 for n in a["emitted"]) and a["length"] == [100 + n for n in a["emitted"]]
    assert a["verify"]["status"].tolist() == [0] * 5 and a["attend"]["status"].tolist() == [0] * 5
    for b in range(5):                                            # the last round's answers, from its rows in 64 bits
        n = int(a["verify"]["len"][b])
        for j in range(n):
            z = a["rows"][b, int(a["path"][b, j])].double().cpu().numpy()
            want = O.logprob_row(z, 1.0, int(a["verify"]["seq"][b, j]), example.TOP)
            assert abs(a["answer"]["logp"][b, j].item() - want["logp"]) < 1e-4 and abs(a["answer"]["entropy"][b, j].item() - want["entropy"]) < 1e-4
            assert a["answer"]["top_idx"][b, j].tolist() == want["top_idx"].tolist()
        assert not a["answer"]["logp"][b, n:].any() and not a["answer"]["top_idx"][b, n:].any()
    again = example.main(rounds=12, B=5, report=lambda _: None)
    assert again["emitted"] == a["emitted"] and again["logp"] == a["logp"]


def test_a_round_against_64_bits():
    """Adapter, norms and rotation, attention over cached and new tokens, in one chain."""
    g = torch.Generator(device=DEV).manual_seed(8)
    B, n, K, hq, h, D, R, A = 3, 5, 128, 4, 2, 64, 16, 2
    heads = hq + 2 * h

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)
    x, base = normal(B, n, K), normal(B, n, heads * D)
    a, b = normal(A, R, K) * K ** -0.5, normal(A, heads * D, R) * 0.5
    adapter, scale = torch.tensor([1, -1, 0], dtype=torch.int32, device=DEV), torch.tensor([0.5, 2.0], device=DEV)
    freq, w = torch.rand(D // 2, generator=g, device=DEV), 1 + 0.2 * normal(2, D)
    length = torch.tensor([70, 3, 128], dtype=torch.int32, device=DEV)
    position = torch.tensor([0, 1, 1, 2, 2], dtype=torch.int32, device=DEV).view(1, n, 1)
    cache = tslt.cache_create(B * 3, h, D, DEV)
    pages = torch.randperm(B * 3, generator=g, device=DEV).to(torch.int32).view(B, 3)
    held = [normal(B, 128, h, D) for _ in range(2)]
    tslt.cache_append(cache, pages, torch.zeros_like(length), *held, count=length)
    parents = [-1, 0, 0, 1, 2]
    seen = np.zeros((n, n), dtype=bool)
    for i in range(n):
        j = i
        while j >= 0:
            seen[i, j] = True
            j = parents[j]
    mask = torch.tensor([[sum(1 << j for j in range(n) if seen[i, j])] for i in range(n)], dtype=torch.int32, device=DEV).view(1, n, 1)

    def chain():
        y = tslt.adapt(x, base, a, b, adapter, scale=scale)["out"].view(B, n, heads, D)
        q, k, v = y[:, :, :hq], y[:, :, hq:hq + h], y[:, :, hq + h:]
        turned = tslt.rotate(q, k, position, freq, base=length, q_weight=w[0], k_weight=w[1], eps=1e-6)
        return tslt.cache_attend(turned["q"], cache, pages, length, k=turned["k"], v=v, mask=mask)

    def host(t):
        return t.detach().double().cpu().numpy()
    got = host(chain()["out"])
    y = O.adapt(host(x), host(base), host(a), host(b), adapter.tolist(), host(scale)).reshape(B, n, heads, D)
    cos, sin = O.turns(O.token_positions(B, n, D // 2, position.cpu().numpy(), length.cpu().numpy(), None), host(freq))
    q = O.rotate(y[:, :, :hq], cos, sin, False, host(w[0]), 1e-6)
    k = O.rotate(y[:, :, hq:hq + h], cos, sin, False, host(w[1]), 1e-6)
    from oracle import cache_oracle as C
    codes, scales = cache["codes"].cpu().numpy(), cache["scale"].cpu().numpy()
    for s in range(B):
        L = int(length[s])
        for i in range(hq):
            pk, pv = zip(*[C.page_values(codes, scales, int(p), i // (hq // h)) for p in pages[s]])
            keys = np.concatenate([np.concatenate(pk)[:L], k[s, :, i // (hq // h)]])
            values = np.concatenate([np.concatenate(pv)[:L], y[s, :, hq + h + i // (hq // h)]])
            z = q[s, :, i] @ keys.T / np.sqrt(D)
            z[:, L:][~seen] = -np.inf
            p = np.exp(z - z.max(-1, keepdims=True))
            want = p / p.sum(-1, keepdims=True) @ values
            # scores of some 8 at most are off by a few U of the 64 products' sizes, 2^-18; the weights by as much, the values of some 5 by 2^-20
            assert np.abs(got[s, :, i] - want).max() < 2.0 ** -13


def test_a_step_of_a_model_that_learns():
    """One attention layer: projection, norms and rotation, attention, logits, the loss of given tokens with a bonus for entropy.  The library's gradients of
    the logits and through the rotation, torch's of the products between, against torch's of the whole in 64 bits."""
    g = torch.Generator(device=DEV).manual_seed(3)
    B, n, width, hq, h, D, V = 2, 7, 64, 4, 2, 64, 301

    def normal(*shape, scale=1.0):
        return scale * torch.randn(*shape, generator=g, device=DEV)
    x, head = normal(B, n, width), normal(hq * D, V, scale=0.1)
    W = normal(width, (hq + 2 * h) * D, scale=width ** -0.5).requires_grad_()
    w = (1 + 0.2 * normal(2, D)).requires_grad_()
    freq = (100.0 ** (-torch.arange(D // 2, device=DEV) * 2.0 / D)).float()
    tokens = torch.randint(0, V, (B, n), generator=g, device=DEV, dtype=torch.int32)
    tokens[1, 5:] = -1                                            # no token given there
    causal = torch.ones(n, n, dtype=torch.bool, device=DEV).tril()
    T, bonus = 0.9, 0.05

    def attention(q, k, v):
        k, v = (t.repeat_interleave(hq // h, 2) for t in (k, v))
        s = torch.einsum("bihd,bjhd->bhij", q, k) * D ** -0.5
        return torch.einsum("bhij,bjhd->bihd", torch.softmax(s.masked_fill(~causal.to(s.device), -INF), -1), v).flatten(2)

    y = (x @ W).view(B, n, hq + 2 * h, D)
    q, k, v = y[:, :, :hq], y[:, :, hq:hq + h], y[:, :, hq + h:]
    turned = tslt.rotate(q.detach(), k.detach(), None, freq, q_weight=w[0].detach(), k_weight=w[1].detach(), eps=1e-5)
    leaves = [t.detach().requires_grad_() for t in (turned["q"], turned["k"], v)]
    logits = attention(*leaves) @ head
    z = logits.detach()
    fwd = tslt.logprob(z, T, tokens)
    given = tokens >= 0
    loss = -(torch.where(given, fwd["logp"], 0.0)).sum() - bonus * fwd["entropy"].sum()
    dz = tslt.logprob_backward(z, T, tokens, fwd["lse"], fwd["entropy"], grad_logp=-torch.ones(B, n, device=DEV), grad_entropy=torch.full((B, n), -bonus, device=DEV))["logits"]
    logits.backward(dz)
    dqk = tslt.rotate_backward(leaves[0].grad, leaves[1].grad, q.detach(), k.detach(), None, freq, q_weight=w[0].detach(), k_weight=w[1].detach(), eps=1e-5)
    y.backward(torch.cat([dqk["q"], dqk["k"], leaves[2].grad], 2))

    # the whole in 64 bits on the CPU
    W64, w64 = W.detach().double().cpu().requires_grad_(), w.detach().double().cpu().requires_grad_()
    y = (x.double().cpu() @ W64).view(B, n, hq + 2 * h, D)
    angle = torch.arange(n).double()[:, None] * freq.double().cpu()
    cos, sin = torch.cos(angle)[None, :, None], torch.sin(angle)[None, :, None]

    def rotated(t, weight):
        t = t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-5) * weight
        a, b = t[..., :D // 2], t[..., D // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    logits = attention(rotated(y[:, :, :hq], w64[0]), rotated(y[:, :, hq:hq + h], w64[1]), y[:, :, hq + h:]) @ head.double().cpu()
    p = torch.log_softmax(logits * O.inverse_temperature(T), -1)
    picked = p.gather(2, tokens.long().clamp_min(0).cpu()[..., None])[..., 0]
    want = -(torch.where(given.cpu(), picked, 0.0)).sum() + bonus * (p.exp() * p).sum()
    want.backward()
    # fp32 chains of sums of 64 to 301 numbers, four of them after another: each some 2^-18 of its size
    assert abs(loss.item() - want.item()) < 2.0 ** -16 * abs(want.item())
    for got, grad in ((W.grad, W64.grad), (torch.stack([dqk["q_weight"], dqk["k_weight"]]), w64.grad)):
        assert (got.double().cpu() - grad).norm() < 2.0 ** -15 * grad.norm()


def test_a_captured_round_beside_an_eager_one():
    """adapt, rotate and logprob in one graph, replayed with other inputs, eager calls of the same kind in between with workspaces of their own."""
    g = torch.Generator(device=DEV).manual_seed(5)
    B, n, K, hq, h, D, V = 4, 9, 256, 4, 2, 64, 60000
    heads = hq + 2 * h
    x, base = (torch.randn(B, n, m, generator=g, device=DEV).to(torch.bfloat16) for m in (K, heads * D))
    a, b = (torch.randn(*s, generator=g, device=DEV).to(torch.bfloat16) * 0.1 for s in ((2, 32, K), (2, heads * D, 32)))
    adapter = torch.tensor([0, 1, -1, 1], dtype=torch.int32, device=DEV)
    length = torch.tensor([5, 60, 7, 1000], dtype=torch.int32, device=DEV)
    freq = torch.rand(D // 2, generator=g, device=DEV)
    head = torch.randn(hq * D, V, generator=g, device=DEV).to(torch.bfloat16) * 0.1
    tokens, count = torch.randint(0, V, (B, n), generator=g, device=DEV, dtype=torch.int32), torch.tensor([9, 2, 0, 5], dtype=torch.int32, device=DEV)

    def buffers():
        out = {"y": torch.zeros_like(base), "z": torch.zeros(B, n, V, dtype=torch.bfloat16, device=DEV), "logp": torch.zeros(B, n, device=DEV),
               "top_idx": torch.zeros(B, n, 7, dtype=torch.int32, device=DEV), "top_logp": torch.zeros(B, n, 7, device=DEV), "lse": torch.zeros(B, n, device=DEV)}
        ws = [torch.empty(s, dtype=torch.uint8, device=DEV) for s in (tslt.adapt_workspace_bytes(B, n, K, heads * D, 32), tslt.logprob_workspace_bytes(B, n, V, 7))]
        return out, ws

    def run(out, ws):
        tslt.adapt(x, base, a, b, adapter, out={"out": out["y"]}, workspace=ws[0])
        y = out["y"].view(B, n, heads, D)
        q, k = y[:, :, :hq], y[:, :, hq:hq + h]
        tslt.rotate(q, k, None, freq, base=length, eps=1e-6, out={"q": q, "k": k})
        torch.matmul(q.flatten(2), head, out=out["z"])
        tslt.logprob(out["z"], 0.8, tokens, top=7, count=count, out={k: out[k] for k in ("logp", "top_idx", "top_logp", "lse")}, workspace=ws[1])
        return out
    mine, theirs = buffers(), buffers()
    run(*mine)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(*mine)
    for i in range(4):
        x.mul_(-1.1)
        length.add_(1)
        tokens.copy_((tokens + 17) % V)
        for t in (*mine[0].values(), *theirs[0].values()):
            t.zero_()
        graph.replay()
        run(*theirs)
        torch.cuda.synchronize()
        for name in mine[0]:
            assert torch.equal(mine[0][name], theirs[0][name]), (i, name)


def test_two_streams_at_once():
    """The same calls on two streams, each with its own workspace."""
    g = torch.Generator(device=DEV).manual_seed(6)
    z = torch.randn(2, 3, 5, 120001, generator=g, device=DEV)
    tokens = torch.randint(0, 120001, (2, 3, 5), generator=g, device=DEV, dtype=torch.int32)
    want = [tslt.logprob(z[i], 1.0, tokens[i], top=9) for i in range(2)]
    x, base, a, b = (torch.randn(*s, generator=g, device=DEV) for s in ((2, 3, 40, 512), (2, 3, 40, 600), (2, 48, 512), (2, 600, 48)))
    adapter = torch.tensor([0, 1, 0], dtype=torch.int32, device=DEV)
    added = [tslt.adapt(x[i], base[i], a, b, adapter)["out"] for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append((tslt.logprob(z[i], 1.0, tokens[i], top=9), tslt.adapt(x[i], base[i], a, b, adapter)["out"]))
    torch.cuda.synchronize()
    for i in range(2):
        for out, y in got[i]:
            assert all(torch.equal(out[k], want[i][k]) for k in out) and torch.equal(y, added[i])
