"""The oracle of the calls around attention and verification against what defines them: differences, small sums, identities."""
import numpy as np
import pytest

from oracle import round_oracle as O


def differences(f, x, h=1e-5):
    """The gradient of the number f(x) by central differences."""
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        up, down = x.copy(), x.copy()
        up[i] += h
        down[i] -= h
        g[i] = (f(up) - f(down)) / (2 * h)
    return g


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("eps", [None, 1e-3])
def test_rotation_keeps_lengths_and_turns_by_differences_of_positions(adjacent, eps):
    r = np.random.default_rng(1)
    freq = r.random(8).astype(np.float32)
    x = r.standard_normal((1, 2, 1, 24))
    at = [O.turns(O.token_positions(1, 2, 8, None, np.array([b]), None), freq) for b in (0, 1000)]
    a, b = (O.rotate(x, *t, adjacent, eps=eps) for t in at)
    n = O.rotate(x, np.ones((1, 2, 0)), np.zeros((1, 2, 0)), adjacent, eps=eps)
    assert np.allclose((a ** 2).sum(-1), (n ** 2).sum(-1)) and np.array_equal(a[..., 16:], n[..., 16:])
    # the product of two tokens' rows depends on how far apart they are
    assert np.allclose((a[:, 0] * a[:, 1]).sum(-1), (b[:, 0] * b[:, 1]).sum(-1))


def test_positions_of_axes():
    position = np.array([[[3, 5, 7], [4, 6, 8]]])
    at = O.token_positions(2, 2, 4, position, np.array([10, -20]), np.array([0, 2, 1, 9]))
    assert at.tolist() == [[[13, 17, 15, 17], [14, 18, 16, 18]], [[-17, -13, -15, -13], [-16, -12, -14, -12]]]


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("eps", [None, 1e-3])
def test_rotation_backward_by_differences(adjacent, eps):
    r = np.random.default_rng(2)
    x, g, w = r.standard_normal((2, 2, 2, 16)), r.standard_normal((2, 2, 2, 16)), r.standard_normal(16)
    cos, sin = O.turns(O.token_positions(2, 2, 4, None, None, None), r.random(4))
    dx, dw = O.rotate_backward(g, x, cos, sin, adjacent, w, eps)
    assert np.allclose(dx, differences(lambda y: (g * O.rotate(y, cos, sin, adjacent, w, eps)).sum(), x), atol=1e-8)
    if eps is not None:
        assert np.allclose(dw, differences(lambda v: (g * O.rotate(x, cos, sin, adjacent, v, eps)).sum(), w), atol=1e-8)


def test_logprob_of_small_rows():
    z = np.log(np.array([0.1, 0.2, 0.4, 0.2, 0.1]))
    got = O.logprob_row(z + 7, 1.0, 3, 4)
    assert np.isclose(got["logp"], np.log(0.2)) and np.isclose(got["lse"], 7) and got["top_idx"].tolist() == [2, 1, 3, 0]
    assert np.isclose(got["entropy"], -(0.2 * np.log(0.1) + 0.4 * np.log(0.2) + 0.4 * np.log(0.4)))
    masked = O.logprob_row([-np.inf, 1.0, -np.inf], 0.5, 0, 2)
    assert masked["logp"] == -np.inf and masked["entropy"] == 0 and masked["top_idx"].tolist() == [1, -1] and masked["lse"] == 0.5
    assert O.logprob_row([np.inf, 0.0], 1.0, 0, 1)["status"] == 1 and O.logprob_row([-np.inf] * 2, 1.0, 0, 1)["status"] == 2


def test_logprob_backward_by_differences():
    r = np.random.default_rng(3)
    z, rT = 2 * r.standard_normal(12), 0.7
    gs = dict(g_logp=0.8, g_entropy=-0.3, g_lse=0.2, g_top=np.array([0.5, -0.4, 0.1]))
    row = O.logprob_row(z, rT, 5, 3)

    def total(y):
        o = O.logprob_row(y, rT, 5, 3)
        return 0.8 * o["logp"] - 0.3 * o["entropy"] + 0.2 * o["lse"] + (gs["g_top"] * o["top_logp"]).sum()
    got = O.logprob_backward_row(z, rT, 5, row["lse"], row["entropy"], row["top_idx"], **gs)
    assert np.allclose(got, differences(total, z), atol=1e-8)


def test_adapters():
    r = np.random.default_rng(4)
    x, base, a, b = r.standard_normal((3, 2, 4)), r.standard_normal((3, 2, 5)), r.standard_normal((2, 3, 4)), r.standard_normal((2, 5, 3))
    got = O.adapt(x, base, a, b, [1, -1, 0], scale=np.array([2.0, 0.5]), rank=np.array([3, 1]))
    assert np.array_equal(got[1], base[1])
    assert np.allclose(got[0], base[0] + 0.5 * x[0] @ a[1, :1].T @ b[1, :, :1].T) and np.allclose(got[2], base[2] + 2 * x[2] @ (b[0] @ a[0]).T)
