"""The cache oracle against what does not come from it: torch's e4m3 casts, a softmax by torch, brute-force selection."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as O


def test_codes_are_torchs_e4m3():
    every = np.arange(256, dtype=np.uint8)
    theirs = torch.from_numpy(every.copy()).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(O.decode(every), theirs, equal_nan=True)
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.normal(size=4000) * 10.0 ** rng.uniform(-5, 2.6, 4000), theirs[np.isfinite(theirs)],
                        (theirs[:126] + theirs[1:127]) / 2]).astype(np.float32).clip(-448, 448)       # ... and every tie
    assert np.array_equal(O.encode(x), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert O.encode(np.array([np.inf, -np.inf, np.nan])).tolist() == [126, 254, 127]


@pytest.mark.parametrize("most,want", [(448.0, 1.0), (448.0001, 2.0), (224.0, 0.5), (0.0, 2.0 ** -100), (1e-40, 2.0 ** -100), (7.0, 2.0 ** -6)])
def test_scale_is_the_least_power_that_fits(most, want):
    assert O.least_scale(most) == want


def test_appended_tokens_come_back_within_half_a_step():
    """Also those that are there before a larger token makes the page's scale grow (two roundings of the smallest ones)."""
    rng = np.random.default_rng(2)
    D = 64
    codes, scale = np.zeros((3, 2, 2, 64 * D), np.uint8), np.ones((3, 2, 2), np.float32)
    tables, length = np.array([[2, 0]]), np.array([0])
    rows = []
    for n, size in ((5, 1.0), (70, 900.0), (3, 0.01)):
        k, v = (rng.normal(size=(1, n, 2, D)).astype(np.float32) * size for _ in range(2))
        codes, scale, length = O.append(codes, scale, tables, length, k, v)
        rows.append((k, v))
    assert length.tolist() == [78]
    for h in range(2):
        got = O.cached(codes, scale, tables[0], 78, h)
        for part in (0, 1):
            want = np.concatenate([r[part][0, :, h] for r in rows])
            unit = np.repeat([scale[2, h, part], scale[0, h, part]], [64, 14])[:, None]
            assert np.all(np.abs(got[part] - want) <= np.abs(want) * 2.0 ** -4 + unit * 2.0 ** -9)


def test_attention_is_a_softmax():
    rng = np.random.default_rng(3)
    B, n, H, G, D = 2, 5, 2, 3, 64
    codes = rng.integers(0, 120, (4, H, 2, 64 * D)).astype(np.uint8)
    scale = np.full((4, H, 2), 2.0 ** -6, np.float32)
    tables, lengths = np.array([[0, 1], [3, 2]]), np.array([70, 0])
    q = rng.normal(size=(B, n, H * G, D))
    k, v = rng.normal(size=(2, B, n, H, D))
    out, lse, _, _ = O.attend(q, codes, scale, tables, lengths, k, v)
    for b in range(B):
        for hq in range(H * G):
            ck, cv, _ = O.cached(codes, scale, tables[b], lengths[b], hq // G)
            for i in range(n):
                kk = torch.from_numpy(np.concatenate([ck, k[b, :i + 1, hq // G]]))
                vv = torch.from_numpy(np.concatenate([cv, v[b, :i + 1, hq // G]]))
                s = kk @ torch.from_numpy(q[b, i, hq]) / D ** 0.5
                assert np.allclose(out[b, i, hq], (torch.softmax(s, 0) @ vv).numpy(), rtol=1e-12, atol=1e-12)
                assert abs(lse[b, i, hq] - float(torch.logsumexp(s, 0))) < 1e-12
    empty = O.attend(q, codes, scale, tables, np.zeros(2, int), None, None)
    assert np.all(empty[0] == 0) and np.all(np.isneginf(empty[1]))
    w, _ = O.weigh(q, lse, codes, scale, tables, lengths, np.zeros((B, H, 128)), 1.0)
    assert np.all(w[1] == 0) and np.all(w[0, :, 70:] == 0) and 0 < w[0, 0].sum() < n * G


def test_eviction_keeps_the_heaviest_and_the_last():
    rng = np.random.default_rng(4)
    weight = rng.integers(0, 4, (1, 1, 128)).astype(np.float32)
    weight[0, 0, 7] = np.nan
    codes = rng.integers(0, 120, (4, 1, 2, 64 * 64)).astype(np.uint8)
    scale = np.array([[[1, 2]], [[4, 1]], [[1, 1]], [[1, 1]]], np.float32)
    _, _, length, kept, w = O.evict(codes, scale, np.array([[1, 0]]), [100], weight, 30, 6, np.array([[3]]))
    assert length.tolist() == [30] and kept[0, 0, -6:].tolist() == list(range(94, 100))
    chosen = set(kept[0, 0, :24].tolist())
    def order(i):
        return (np.isnan(weight[0, 0, i]), -np.nan_to_num(weight[0, 0, i]), i)
    assert chosen == set(sorted(range(94), key=order)[:24]) and list(kept[0, 0]) == sorted(kept[0, 0])
    assert np.array_equal(w[0, 0, :30], weight[0, 0, kept[0, 0]], equal_nan=True)
