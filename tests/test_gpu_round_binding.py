"""The calls around attention and verification by the native path of the binding and step by step: same outputs, same errors."""
import pytest
import torch

from .test_gpu_binding import both, unwritten

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def normal(*shape, dtype=torch.bfloat16):
    return torch.randn(*shape, device=DEV).to(dtype)


def ints(*shape, high=3):
    return torch.randint(0, high, shape, device=DEV, dtype=torch.int32)


def scratch(n):
    return torch.empty(n, dtype=torch.uint8, device=DEV)


def test_rotate_by_either_path(tslt, monkeypatch):
    B, n, hq, h, D = 3, 5, 4, 2, 64
    x = normal(B, n, hq + 2 * h, D)
    usual = dict(q=x[:, :, :hq], k=x[:, :, hq:hq + h], position=ints(B, n, 2, high=99), freq=torch.rand(16, device=DEV), axis=ints(16, high=2), base=ints(B, high=999),
                 q_weight=torch.rand(D, device=DEV), k_weight=torch.rand(D, device=DEV), eps=1e-5, adjacent=False, count=ints(B, high=n))
    made = {"q": torch.empty_like(usual["q"]), "k": torch.empty_like(usual["k"]), "status": torch.empty(B, dtype=torch.int32, device=DEV)}

    def call(taken=True, drop=(), put={}, **other):
        def run():
            out = {**unwritten(made), **put}
            for name in drop:
                del out[name]
            return tslt.rotate(**{**usual, **other}, out=out)
        return both(tslt, monkeypatch, run, taken)
    plain = call()
    assert torch.equal(plain["q"][0, :1], tslt.rotate(**usual)["q"][0, :1]) or int(usual["count"][0]) == 0
    for other in (dict(adjacent=True), dict(q_weight=None), dict(q_weight=None, k_weight=None, eps=None), dict(position=usual["position"][:1].contiguous()),
                  dict(position=None, axis=None), dict(freq=None, position=None, axis=None), dict(base=None, count=None), dict(eps=0)):
        call(**other)
    call(k=None)
    call(put={"status": None})
    call(drop=("status",))
    bad = [dict(q=x.transpose(2, 3)), dict(q=x[0]), dict(k=usual["k"].float()), dict(k=x[:, 1:, :h]), dict(position=usual["position"].long()), dict(position=ints(B, n + 1, 2)),
           dict(freq=usual["freq"].double()), dict(axis=ints(15)), dict(base=ints(B + 1)), dict(count=usual["count"].cpu()), dict(q_weight=torch.rand(D + 1, device=DEV)),
           dict(eps=None), dict(eps="much"), dict(put={"q": made["k"]}), dict(drop=("q",)), dict(drop=("k",)), dict(put={"status": ints(B + 1)})]
    for other in bad:
        assert call(taken=False, **other)[0] in (tslt.TsltError, ValueError), other
    for other in (dict(freq=torch.rand(12, device=DEV), axis=None), dict(freq=torch.rand(40, device=DEV), axis=None), dict(eps=float("inf"))):
        assert call(**other)[0] is tslt.TsltError
    call(freq=torch.rand(0, device=DEV), axis=None)
    for other in (dict(eps=-1.0, q_weight=None, k_weight=None),):
        call(taken=False, **other)


def test_rotate_backward_by_either_path(tslt, monkeypatch):
    B, n, hq, h, D = 2, 7, 3, 1, 128
    usual = dict(grad_q=normal(B, n, hq, D), grad_k=normal(B, n, h, D), q=normal(B, n, hq, D), k=normal(B, n, h, D), position=None, freq=torch.rand(64, device=DEV),
                 q_weight=torch.rand(D, device=DEV), k_weight=None, eps=1e-5, workspace=scratch(tslt.rotate_backward_workspace_bytes(B, n, hq, h, D)))
    made = {"q": usual["q"], "k": usual["k"], "q_weight": usual["q_weight"], "k_weight": usual["q_weight"], "status": torch.empty(B, dtype=torch.int32, device=DEV)}

    def call(taken=True, put={}, **other):
        return both(tslt, monkeypatch, lambda: tslt.rotate_backward(**{**usual, **other}, out={**unwritten(made), **put}), taken)
    call()
    call(grad_k=None, k=None, put={"k": None, "k_weight": None})
    call(eps=None, q_weight=None, q=None, k=None, put={"q_weight": None, "k_weight": None})
    call(put={"q_weight": None, "k_weight": None, "status": None})
    for other in (dict(workspace=usual["workspace"][:256]), dict(grad_k=None, k=None)):
        assert call(**other)[0] is tslt.TsltError
    for other in (dict(q=None), dict(k=None), dict(q=usual["q"].float()), dict(grad_q=usual["grad_q"][0]), dict(put={"q_weight": torch.zeros(3, device=DEV)}), dict(put={"q": None})):
        assert call(taken=False, **other)[0] is tslt.TsltError


def test_logprob_by_either_path(tslt, monkeypatch):
    B, n, m, V, top = 2, 5, 3, 30011, 6
    wide = normal(B, n, V + 3, dtype=torch.float16)
    usual = dict(logits=wide[:, :, :V], temperature=0.8, tokens=ints(B, m, high=V), top=top, index=ints(B, m, high=n), count=ints(B, high=m + 1),
                 workspace=scratch(tslt.logprob_workspace_bytes(B, m, V, top)))
    made = tslt.logprob(**usual)

    def call(taken=True, drop=(), put={}, **other):
        def run():
            out = {**unwritten(made), **put}
            for name in drop:
                del out[name]
            return tslt.logprob(**{**usual, **other}, out=out)
        return both(tslt, monkeypatch, run, taken)
    call()
    call(top=0)
    call(tokens=None, put={"logp": None})
    call(drop=("lse", "entropy", "status"))
    call(count=None, temperature=1)
    for other in (dict(temperature=0.0), dict(workspace=usual["workspace"][:64])):
        assert call(**other)[0] is tslt.TsltError
    for other in (dict(logits=wide[0]), dict(logits=wide[:, :, ::2]), dict(tokens=usual["tokens"].long()), dict(tokens=usual["tokens"][:, :2]), dict(index=usual["index"][0]),
                  dict(count=ints(B + 1)), dict(top=33), dict(top=-1), dict(top=1 << 40), dict(drop=("top_idx",)), dict(put={"top_logp": None}), dict(put={"logp": ints(B, m)}),
                  dict(top=5), dict(logits=wide.double())):
        assert call(taken=False, **other)[0] is tslt.TsltError, other


def test_logprob_backward_by_either_path(tslt, monkeypatch):
    B, n, V, top = 2, 3, 4001, 4
    z = normal(B, n, V, dtype=torch.float32)
    fwd = tslt.logprob(z, 0.8, ints(B, n, high=V), top=top)
    usual = dict(logits=z, temperature=0.8, tokens=ints(B, n, high=V), lse=fwd["lse"], entropy=fwd["entropy"], grad_logp=torch.rand(B, n, device=DEV),
                 grad_entropy=torch.rand(B, n, device=DEV), grad_lse=torch.rand(B, n, device=DEV), top_idx=fwd["top_idx"], grad_top=torch.rand(B, n, top, device=DEV), count=ints(B, high=n + 1))

    def call(taken=True, out=None, **other):
        return both(tslt, monkeypatch, lambda: tslt.logprob_backward(**{**usual, **other}, out=out or {"logits": torch.full_like(z, 9)}), taken)
    call()
    for none in ({"grad_logp": None, "tokens": None}, {"grad_entropy": None, "entropy": None}, {"grad_lse": None}, {"grad_top": None, "top_idx": None}, {"count": None}):
        call(**none)
    for other in (dict(temperature=-1.0), dict(tokens=None), dict(entropy=None), dict(top_idx=None)):
        assert call(**other)[0] is tslt.TsltError
    for other in (dict(lse=None), dict(lse=fwd["lse"][0]), dict(grad_top=usual["grad_top"][0]), dict(grad_top=torch.rand(B, n, 33, device=DEV)), dict(top_idx=fwd["top_idx"].long()),
                  dict(out={"logits": torch.zeros(B, n, V - 1, device=DEV)}), dict(out={"logits": torch.zeros_like(z, dtype=torch.float16)}), dict(out={"other": z}), dict(logits=z[0])):
        assert call(taken=False, **other)[0] is tslt.TsltError, other


def test_adapt_by_either_path(tslt, monkeypatch):
    B, n, K, N, R, adapters = 3, 4, 72, 50, 16, 2
    wide = normal(B, n, N + 6)
    usual = dict(x=normal(B, n, K), base=wide[:, :, 3:3 + N], a=normal(adapters, R, K), b=normal(adapters, N, R), adapter=ints(B, high=adapters), scale=torch.rand(adapters, device=DEV),
                 rank=ints(adapters, high=R), count=ints(B, high=n + 1), workspace=scratch(tslt.adapt_workspace_bytes(B, n, K, N, R)))
    made = {"out": torch.empty(B, n, N, dtype=torch.bfloat16, device=DEV), "status": torch.empty(B, dtype=torch.int32, device=DEV)}

    def call(taken=True, put={}, **other):
        return both(tslt, monkeypatch, lambda: tslt.adapt(**{**usual, **other}, out={**unwritten(made), **put}), taken)
    call()
    call(scale=None, rank=None, count=None, put={"status": None})
    for other in (dict(workspace=usual["workspace"][:16]), dict(x=normal(B, n, K + 2)[:, :, :K])):
        assert call(**other)[0] is tslt.TsltError
    for other in (dict(x=usual["x"][0]), dict(x=usual["x"].float()), dict(base=wide), dict(a=usual["a"].transpose(1, 2)), dict(a=usual["a"][:, :, :64].contiguous()), dict(b=usual["b"][:1].contiguous()),
                  dict(adapter=ints(B + 1)), dict(scale=torch.rand(3, device=DEV)), dict(rank=usual["rank"].long()), dict(put={"out": wide}), dict(put={"out": None}), dict(a=usual["a"][0])):
        assert call(taken=False, **other)[0] is tslt.TsltError, other
