"""tslt_logprob of rows whose logits lie far from 0: references that move, on either side of where differences are taken first."""
import numpy as np
import pytest
import torch

from . import test_gpu_logprob as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = L.U


def make(dtype, kind, offset, n, V, T=1.0, top=7):
    c = L.make(1, n, V, dtype, T=T, top=top, kind=kind, offset=1)
    c["logits"].add_(offset)                                       # (rounded to the row's type: what the oracle is given too)
    return c


def check(c, out, rows):
    """The first rows against the oracle."""
    rows = min(rows, c["n"])
    c.update(logits=c["logits"][:, :rows], tokens=c["tokens"][:, :rows].contiguous(), n=rows, m=rows)
    got = {k: L.host(v[:, :rows]) for k, v in out.items()}
    V = c["V"]
    # as in test_gpu_logprob.check: S is off by an exponent's and the scale's rounding, the exponential's, the sums'; and each of a lane's vectors may bring a
    # new reference, whose factor is off by 2 U and whose product by U
    S = (2 * (np.log2(V) + 2) + 2 + V / 1024 + 10 + 3 * (V / 1024 + 2)) * U
    for b, j, z, want in L.oracle(c):
        assert got["status"][b, j] == 0
        assert abs(got["lse"][b, j] - want["lse"]) <= S + U * abs(want["lse"]), (j, got["lse"][b, j] - want["lse"])
        assert abs(got["entropy"][b, j] - want["entropy"]) <= 2 * S * (1 + np.log(V)) + U * want["entropy"], (j, got["entropy"][b, j] - want["entropy"])
        for x, y in [(got["logp"][b, j], want["logp"]), *zip(got["top_logp"][b, j], want["top_logp"])]:
            assert abs(x - y) <= S + U * abs(y) + 1e-15 * abs(want["lse"]), (j, x - y)
        assert np.array_equal(got["top_idx"][b, j], want["top_idx"])


# (n: rows that a workgroup has whole, that several share, and that a wave has)
@pytest.mark.parametrize("shape", [(1100, 40003), (3, 40003), (2100, 1501)], ids=str)
@pytest.mark.parametrize("kind", ["plain", "rising"])
@pytest.mark.parametrize("offset", [1e3, -1e4, 1e5, 1e6, -1e6])
def test_references_that_move(shape, kind, offset):
    for T in (1.0, 0.7):
        c = make("f32", kind, offset, *shape, T=T)
        check(c, L.call(c), 6)


@pytest.mark.parametrize("sign", [1, -1])
def test_references_that_move_past_where_differences_are_taken_first(sign):
    """From fl(k c) below 2^22 to above it, and back: logits in steps of 1/4 around 2^22 / k."""
    for T in (1.0, 0.7):
        c = make("f32", "rising", sign * round(2 ** 22 * np.log(2) * T) - 10, 1100, 40003, T=T)
        check(c, L.call(c), 3)


@pytest.mark.parametrize("dtype,offset", [("f16", 1000), ("bf16", 100), ("bf16", -300)])
def test_references_that_move_in_16_bits(dtype, offset):
    c = make(dtype, "rising", offset, 1100, 40003)
    check(c, L.call(c), 3)
