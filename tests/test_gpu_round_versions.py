"""Results that are written into tensors that torch knows are told to it: a gradient that would need what they held is an error, not a wrong number."""
import pytest
import torch

from paper_2512_16273_amd import tslt

from .test_gpu_binding import Declines

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(params=["native", "step by step"])
def path(request, monkeypatch):
    if request.param != "native":
        tslt.load()
        monkeypatch.setattr(tslt, "_fast", Declines())
    return request.param


def scratch(n):
    return torch.empty(n, dtype=torch.uint8, device=DEV)


def made(**shapes):
    return {k: torch.zeros(*s, dtype=torch.int32 if k in ("status", "top_idx") else torch.float32, device=DEV) for k, s in shapes.items()}


def versions(out):
    return {k: t._version for k, t in out.items()}


def test_every_result_is_told(path):
    B, n, D, V = 2, 3, 64, 50
    q, z, count = torch.randn(B, n, 2, D, device=DEV), torch.randn(B, n, V, device=DEV), torch.full((B,), n, dtype=torch.int32, device=DEV)
    tokens, freq, w = torch.ones(B, n, dtype=torch.int32, device=DEV), torch.rand(32, device=DEV), torch.rand(D, device=DEV)
    a, b, adapter = torch.randn(1, 16, V * 4, device=DEV), torch.randn(1, V, 16, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    for call, out in [
            (lambda out: tslt.rotate(q, q, None, freq, count=count, out=out), made(q=q.shape, k=q.shape, status=(B,))),
            (lambda out: tslt.rotate_backward(q, q, q, q, None, freq, q_weight=w, k_weight=w, eps=1e-5, out=out, workspace=scratch(tslt.rotate_backward_workspace_bytes(B, n, 2, 2, D))),
             made(q=q.shape, k=q.shape, q_weight=(D,), k_weight=(D,), status=(B,))),
            (lambda out: tslt.logprob(z, 1.0, tokens, top=3, out=out, workspace=scratch(1 << 20)),
             made(logp=(B, n), entropy=(B, n), lse=(B, n), status=(B, n), top_idx=(B, n, 3), top_logp=(B, n, 3))),
            (lambda out: tslt.logprob_backward(z, 1.0, tokens, torch.zeros(B, n, device=DEV), grad_logp=torch.ones(B, n, device=DEV), out=out), made(logits=z.shape)),
            (lambda out: tslt.adapt(torch.randn(B, n, V * 4, device=DEV), z, a, b, adapter, out=out, workspace=scratch(tslt.adapt_workspace_bytes(B, n, V * 4, V, 16))),
             made(out=z.shape, status=(B,)))]:
        before = versions(out)
        call(out)
        assert all(t._version > before[k] for k, t in out.items()), sorted(out)


def test_what_autograd_holds_is_not_changed_in_silence(path):
    x = torch.randn(2, 3, 4, 64, device=DEV, requires_grad=True)
    y = x * 2.0
    z = (y * y).sum()                                              # holds y
    held = y.detach()
    tslt.rotate(held, None, None, torch.rand(32, device=DEV), out={"q": held})
    with pytest.raises(RuntimeError, match="inplace"):
        z.backward()
    with torch.inference_mode():                                   # (its tensors have no versions)
        q = torch.randn(2, 3, 4, 64, device=DEV)
        want = tslt.rotate(q, None, None, torch.ones(32, device=DEV))["q"]
        tslt.rotate(q, None, None, torch.ones(32, device=DEV), out={"q": q})
        assert torch.equal(q, want)
