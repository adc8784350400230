"""tslt_logprob_backward of rows whose logits lie far from 0."""
import numpy as np
import pytest
import torch

from . import test_gpu_logprob as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = L.U


@pytest.mark.parametrize("T,offset", [(0.7, 3.0e6), (1.3, 6.0e6), (1.3, -5.0e6), (37.0, 1.1e8)])
def test_what_a_reference_loses_in_32_bits(T, offset):
    """The gradient by the lse that is given, where lse * T is no number of 32 bits."""
    c = L.make(1, 4, 9001, "f32", T=T, top=6)
    c["logits"].add_(offset)
    fwd, g = L.call(c), L.gradients(c)
    L.check_back(c, fwd, g, L.back(c, fwd, g)["logits"])


def rows_of(kind, n, V, dtype, T, pad=0):
    c = L.make(1, n, V, dtype, T=T, top=5, kind="lowest" if kind == "lowest" else "plain", offset=1, pad=pad)
    g, t = torch.Generator(device=DEV).manual_seed(9), L.TYPES[dtype]
    z = c["logits"]
    if kind.startswith("ties"):                                    # a part of the row at its largest number, the rest one step of the type below
        size = {"ties": 1e10, "ties below": -3e9, "ties at the end": 3.0e38}[kind]
        most = torch.tensor(size, device=DEV).to(t)
        z.copy_(torch.where(torch.rand(z.shape, generator=g, device=DEV) < 0.3, most, most - abs(most) * 2 * torch.finfo(t).eps))
        z[:, 0, 1::2] = -float("inf")
    elif kind != "lowest":
        z.add_(float(kind))
    return c


def check_own(c, fwd, g, dz):
    """Against 64 bits that know the row alone, not the lse that was left of it."""
    z, got, rT = L.host(c["logits"]), L.host(dz), L.O.inverse_temperature(c["T"])
    step, V = torch.finfo(L.TYPES[c["dtype"]]).eps / 2, c["V"]
    f, h = {k: L.host(v) for k, v in fwd.items()}, {k: L.host(v) for k, v in g.items()}
    for i in range(min(c["n"], 5)):
        x = z[0, i] - z[0, i].max()                                # (the gradient does not change with a shift)
        S = np.exp(x * rT).sum()
        lse = z[0, i].max() * rT + np.log(S)
        want = L.O.logprob_backward_row(x, rT, int(c["tokens"][0, i]), np.log(S), f["entropy"][0, i], f["top_idx"][0, i], *(h[k][0, i] for k in ("grad_logp", "grad_entropy", "grad_lse", "grad_top")))
        d = np.maximum(x * rT - np.log(S), -200.0)
        # what is left of lse: half a step of fp32, of p and under the entropy's logarithm; nothing of rows that are summed up again
        given = 0.0 if abs(lse) > 2.0 ** 23 + 1 else U * abs(lse)
        size = sum(np.abs(h[k][0, i]).sum() for k in ("grad_logp", "grad_lse", "grad_top")) + np.abs(h["grad_entropy"][0, i]) * (np.abs(d) + f["entropy"][0, i] + given)
        size = rT * np.exp(d) * size
        put = np.zeros(V)
        for at, v in [(int(c["tokens"][0, i]), h["grad_logp"][0, i]), *zip(f["top_idx"][0, i], h["grad_top"][0, i])]:
            if at >= 0:
                put[at] += rT * abs(v)
        # as in test_gpu_logprob.check_back; of a row's own sum its terms' exponents (weighed by them: ln V at most) and exponentials
        near = size * ((2 * (np.abs(d) + np.log(V)) * 1.4427 + 18) * U + np.expm1(given)) + rT * np.exp(d + given) * np.abs(h["grad_entropy"][0, i]) * given
        near = (near + put * 36 * U + 2.0 ** -125 * (1 + np.abs(size))) * (1 + step) + step * np.abs(want) + L.TINY[c["dtype"]]
        assert np.all(np.abs(got[0, i] - want) <= near), (i, np.max(np.abs(got[0, i] - want) / near))


# (rows that several workgroups share, and that one has)
@pytest.mark.parametrize("n,V", [(3, 40003), (9000, 1501)])
@pytest.mark.parametrize("kind,dtype,T", [("lowest", "f16", 1.0), ("lowest", "f16", 0.8)] + [
    (kind, dtype, T) for kind in ("lowest", "ties", "ties below", "ties at the end") for dtype, T in (("f32", 1.0), ("f32", 0.8), ("bf16", 1.0), ("bf16", 0.8), ("f32", 1.7))])
def test_rows_whose_lse_has_no_room_for_their_sum(kind, dtype, T, n, V):
    c = rows_of(kind, n, V, dtype, T, pad=3)
    fwd, g = L.call(c), L.gradients(c)
    assert not fwd["status"].any()
    dz = L.back(c, fwd, g)["logits"]
    check_own(c, fwd, g, dz)
    L.back(c, fwd, g, out={"logits": c["logits"]})                 # in place
    assert torch.equal(c["logits"], dz)


@pytest.mark.parametrize("offset", ["0", "1e3", "-1e5", "3e6", "2e7"])
def test_what_is_left_of_the_sum_in_lse(offset):
    c = rows_of(offset, 3, 9001, "f32", 1.0)
    fwd, g = L.call(c), L.gradients(c)
    check_own(c, fwd, g, L.back(c, fwd, g)["logits"])


def test_rows_that_cannot_be_used_beside_them():
    """Gradients of rows that hold nothing above -inf, a NaN or +inf are NaN, whatever their lse says; the others are as without them."""
    c = rows_of("lowest", 8, 30001, "f32", 0.8)
    z = c["logits"]
    z[0, 1] = -float("inf")
    z[0, 2, 29999] = float("nan")
    z[0, 3, 0] = float("inf")
    fwd, g = L.call(c), L.gradients(c)
    assert fwd["status"][0].tolist() == [0, 2, 1, 1, 0, 0, 0, 0]
    for lse in (fwd["lse"], fwd["lse"].nan_to_num(nan=-float("inf"))):
        dz = L.back(c, {**fwd, "lse": lse.contiguous()}, g)["logits"]
        assert dz[0, 1:4].isnan().all() and dz[0, 4:].isfinite().all() and dz[0, 0].isfinite().all()
    check_own({**c, "n": 1}, fwd, g, dz)
