"""Rows that lie further apart than 32 bits reach: the calls around attention and verification give what they give for the same rows side by side."""
import pytest
import torch

from paper_2512_16273_amd import tslt

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FAR = 2 ** 31 + 64                                                # elements: beyond 4 GiB in 16 bits, and beyond a signed count of elements


@pytest.fixture(scope="module")
def memory():
    return torch.zeros(FAR + (1 << 20), dtype=torch.bfloat16, device=DEV)


def apart(memory, x, dim, at=0):
    """x with its second entry along `dim` FAR behind the first."""
    strides = list(x.stride())
    strides[dim] = FAR
    y = memory[at:].as_strided(x.shape, strides)
    y.copy_(x)
    return y


def test_logprob_and_its_gradient(memory):
    z = torch.randn(2, 1, 5001, device=DEV).to(torch.bfloat16)
    tokens = torch.tensor([[4], [5000]], dtype=torch.int32, device=DEV)
    g = torch.randn(2, 1, device=DEV)
    want = tslt.logprob(z, 0.7, tokens, top=4)
    dz = tslt.logprob_backward(z, 0.7, tokens, want["lse"], want["entropy"], grad_logp=g, grad_entropy=g)["logits"]
    for dim, shape in ((0, (2, 1, 5001)), (1, (1, 2, 5001))):
        far = apart(memory, z.view(shape), dim)
        got = tslt.logprob(far, 0.7, tokens.view(shape[:2]), top=4)
        assert torch.equal(got["top_idx"].view(2, 1, 4), want["top_idx"]) and (got["lse"].view(2, 1) - want["lse"]).abs().max() < 1e-5
        at = shape[:2]
        out = {"logits": far}
        tslt.logprob_backward(far, 0.7, tokens.view(at), want["lse"].view(at), want["entropy"].view(at), grad_logp=g.view(at), grad_entropy=g.view(at), out=out)
        assert torch.equal(far.reshape(2, 1, 5001), dz)


def test_rotate_and_its_gradients(memory):
    q, k, g = torch.randn(1, 2, 2, 64, device=DEV).to(torch.bfloat16), torch.randn(1, 2, 2, 64, device=DEV).to(torch.bfloat16), torch.randn(1, 2, 2, 64, device=DEV).to(torch.bfloat16)
    freq = torch.rand(32, device=DEV)
    want = tslt.rotate(q, k, None, freq, eps=1e-5)
    back = tslt.rotate_backward(g, g, q, k, None, freq, eps=1e-5)
    for dim in (1, 2):
        fq, fk = apart(memory, q, dim), apart(memory, k, dim, 1 << 18)
        got = tslt.rotate(fq, fk, None, freq, eps=1e-5, out={"q": fq, "k": fk})
        assert torch.equal(got["q"], want["q"]) and torch.equal(got["k"], want["k"])
        fq, fk, fg, fh = (apart(memory, t, dim, i << 18) for i, t in enumerate((q, k, g, g)))
        got = tslt.rotate_backward(fg, fh, fq, fk, None, freq, eps=1e-5, out={"q": fg, "k": fh})
        assert torch.equal(got["q"], back["q"]) and torch.equal(got["k"], back["k"])


@pytest.mark.parametrize("n", [1, 40])
def test_adapt(memory, n):
    x, base = torch.randn(2, n, 128, device=DEV).to(torch.bfloat16), torch.randn(2, n, 200, device=DEV).to(torch.bfloat16)
    a, b = torch.randn(1, 16, 128, device=DEV).to(torch.bfloat16), torch.randn(1, 200, 16, device=DEV).to(torch.bfloat16)
    adapter = torch.zeros(2, dtype=torch.int32, device=DEV)
    want = tslt.adapt(x, base, a, b, adapter)["out"]
    fx, fb = apart(memory, x, 0), apart(memory, base, 0, 1 << 18)
    assert torch.equal(tslt.adapt(fx, fb, a, b, adapter, out={"out": fb})["out"], want)
    if n == 1:                                                    # one sequence's tokens
        fx, fb = apart(memory, x.view(1, 2, 128), 1), apart(memory, base.view(1, 2, 200), 1, 1 << 18)
        got = tslt.adapt(fx, fb, a, b, adapter[:1], out={"out": fb})["out"]
        assert torch.equal(got.reshape(2, 1, 200), want)
