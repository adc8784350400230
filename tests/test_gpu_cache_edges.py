"""The calls around the 8-bit cache where numbers are not finite, sequences are long or tables wide: values that the cases of
test_gpu_cache.py do not hold and paths that their sizes do not reach.  Tolerances are that file's."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from tests.test_gpu_cache import DEV, DTYPES, check_attend, check_weigh, make_cache, on_gpu, projection, same_values

pytestmark = pytest.mark.gpu


def weights_with_nan(rng, B, H, tokens, kind):
    weight = rng.random((B, H, tokens)).astype(np.float32) ** 4
    if kind == "all":
        weight[:] = np.nan
    elif kind == "late":
        weight[:, :, 3 * tokens // 4:] = np.nan
    elif kind == "third":
        weight[rng.random(weight.shape) < 0.33] = np.nan
        weight[rng.random(weight.shape) < 0.1] = -np.inf
    else:
        weight[rng.random(weight.shape) < 0.6] = np.nan
    return weight


# (tables of up to 64 and 512 pages: weights' keys in registers, four or 32 to a lane; of more: from memory every time)
@pytest.mark.parametrize("D,H,lengths,keep,recent,width", [(64, 2, [100, 128, 70], 90, 0, 2), (64, 1, [990, 1000, 130], 890, 0, 16),
                                                           (128, 2, [1000, 300], 999, 7, 65), (64, 1, [5000, 700], 4900, 0, 79),
                                                           (64, 2, [1000, 130], 900, 0, 513), (64, 1, [5000, 700], 4900, 11, 700)])
@pytest.mark.parametrize("kind", ["all", "late", "third", "most"])
def test_evict_keeps_the_first_of_the_weights_that_are_nan(tslt, D, H, lengths, keep, recent, width, kind):
    """Weights that are NaN and have to stay, in stretches of more waves than one: the first of them, each once, in order."""
    rng = np.random.default_rng([D, keep, recent, len(kind)])
    B = len(lengths)
    codes, scale, tables, length = make_cache(rng, H, D, lengths)
    tables = np.concatenate([tables, np.full((B, width - tables.shape[1]), -1, np.int32)], 1)
    W, first = -(-keep // 64), codes.shape[0]
    codes = np.concatenate([codes, np.full((B * W,) + codes.shape[1:], 127, np.uint8)])
    scale = np.concatenate([scale, np.full((B * W,) + scale.shape[1:], 1e30, np.float32)])
    new = (first + rng.permutation(B * W)).reshape(B, W).astype(np.int32)
    weight = weights_with_nan(rng, B, H, tables.shape[1] * 64, kind)
    if kind == "late":
        for b, x in enumerate(lengths):
            weight[b, :, 3 * x // 4:] = np.nan
    cache, pages, lens = on_gpu(codes, scale, tables, length)
    got = tslt.cache_evict(cache, pages, lens, torch.from_numpy(weight).to(DEV), keep, recent, torch.from_numpy(new).to(DEV))
    torch.cuda.synchronize()
    want = O.evict(codes, scale, tables, length, weight, keep, recent, new)
    assert got["status"].tolist() == [0] * B
    assert np.array_equal(got["length"].cpu().numpy(), want[2])
    assert np.array_equal(got["kept"].cpu().numpy(), want[3])
    assert np.array_equal(got["weight"].cpu().numpy(), want[4], equal_nan=True)
    same_values((cache["codes"].cpu().numpy(), cache["scale"].cpu().numpy()), want[:2], new, want[2], H)


# (one chunk and several; the kernel for few rows and the one for many)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,G,length", [(3, 2, 70), (3, 2, 6000), (40, 4, 70), (40, 4, 6000)])
def test_a_row_that_is_nan_stays_nan_where_it_sees_an_infinity(tslt, dtype, n, G, length):
    rng = np.random.default_rng([n, length])
    D, H = 64, 2
    codes, scale, tables, lengths = make_cache(rng, H, D, [length])
    codes[tables[0, 0], 1, 1].reshape(4, D, 16)[0, 9, 3] = 127      # a cached value of head 1: its rows are NaN in channel 9
    cache, pages, lens = on_gpu(codes, scale, tables, lengths)
    (q, k, v), _ = projection(rng, 1, n, H * G, H, D, DTYPES[dtype])
    v[0, 0, :, 9], v[0, 0, :, 5] = float("inf"), -float("inf")      # token 0 is seen by all
    q[0, n - 1, 0] = float("nan")
    assert (tslt.cache_attend_workspace_bytes(1, n, H * G, H, D, pages.shape[1]) > 0) == (length > 1000)
    got = tslt.cache_attend(q, cache, pages, lens, k=k, v=v)
    torch.cuda.synchronize()
    out = got["out"].float().cpu()
    assert out[0, n - 1, 0].isnan().all() and got["lse"][0, n - 1, 0].isnan()
    rest = torch.ones(n, H * G, dtype=torch.bool)
    rest[n - 1, 0] = False
    assert (out[0, :, G:, 9]).isnan().all()
    assert (out[0, :, :G, 9][rest[:, :G]] == float("inf")).all() and (out[0][..., 5][rest] == -float("inf")).all()
    fine = [d for d in range(D) if d not in (5, 9)]
    assert out[0][rest][:, fine].isfinite().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,G,length", [(3, 2, 70), (3, 2, 6000), (40, 4, 70), (40, 4, 6000)])
@pytest.mark.parametrize("apart", [0, 200])
def test_infinities_are_the_same_in_one_chunk_and_in_several(tslt, dtype, n, G, length, apart):
    """New tokens with infinite values whose scores lie as high as the cached ones', or, with the whole chunk they are in, so far below them
    (2 * 200 / ln 2 powers of two) that fp32 holds no weight for them: a weight is positive all the same."""
    rng = np.random.default_rng([n, length, apart])
    D, H = 64, 2
    codes, scale, tables, lengths = make_cache(rng, H, D, [length])
    scale[..., 0] = 1.0
    for w, page in enumerate(tables[0]):                            # keys: 1 in the first half of the cache, -1 behind it, in channel 0 alone
        codes[page, :, 0] = 0
        codes[page, :, 0].reshape(H, 64, D)[..., 0] = 0x38 if 2 * w < len(tables[0]) or length < 100 else 0xB8
    cache, pages, lens = on_gpu(codes, scale, tables, lengths)
    (q, k, v), _ = projection(rng, 1, n, H * G, H, D, DTYPES[dtype])
    q[..., 0], q[..., 1:] = apart, 0
    k[..., 0] = -1
    qh, kh, vh = (t.double().cpu().numpy() for t in (q, k, v))
    v[0, 0, :, 5], v[0, 1, 1, 8] = float("inf"), -float("inf")
    v[0, 0, 0, 9], v[0, 1, 0, 9] = float("inf"), -float("inf")      # which add up to NaN
    got = tslt.cache_attend(q, cache, pages, lens, k=k, v=v, scale=1.0)
    torch.cuda.synchronize()
    out = got["out"].float().cpu()
    assert (out[0, :, :, 5] == float("inf")).all()
    assert (out[0, 1:, G:, 8] == -float("inf")).all() and out[0, 0, G:, 8].isfinite().all() and out[0, :, :G, 8].isfinite().all()
    assert (out[0, 0, :G, 9] == float("inf")).all() and out[0, 1:, :G, 9].isnan().all() and out[0, :, G:, 9].isfinite().all()
    want = O.attend(qh, codes, scale, tables, lengths, kh, vh, softmax_scale=1.0)
    for where in (np.s_[0, :, :, 5], np.s_[0, 1:, G:, 8], np.s_[0, :, :G, 9]):
        got["out"][where] = torch.from_numpy(want[0][where]).to(DEV).to(got["out"].dtype)
        want[0][where] = got["out"][where].double().cpu().numpy()
    check_attend(got, want, DTYPES[dtype])


# (few rows; more than there are registers for; many rows on few pages, two sets of rows in registers and one)
WEIGH = [("bf16", 128, 2, 4, 9, [64, 700, 1, 130]), ("f32", 64, 1, 1, 5, [150, 65, 300, 7]), ("f16", 64, 8, 3, 30, [3000, 2000, 4096, 70]),
         ("bf16", 128, 2, 4, 41, [64, 700, 90, 1]), ("f32", 256, 1, 3, 47, [90, 64, 1, 300]), ("f16", 256, 1, 2, 90, [1, 200, 64, 128])]


@pytest.mark.parametrize("dtype,D,H,G,n,lengths", WEIGH)
@pytest.mark.parametrize("odd", [float("nan"), float("inf")])
def test_rows_that_saw_nothing_add_nothing_whatever_they_hold(tslt, dtype, D, H, G, n, lengths, odd):
    """cache_weigh without the count that cache_attend was given: the rows behind it have -inf."""
    rng = np.random.default_rng([D, n, H])
    B = len(lengths)
    codes, scale, tables, length = make_cache(rng, H, D, lengths)
    codes[tables[3, 0], 0, 0, 5] = 127                              # a key of the sequence whose rows all are such
    cache, pages, lens = on_gpu(codes, scale, tables, length)
    (q, k, v), (qh, kh, vh) = projection(rng, B, n, H * G, H, D, DTYPES[dtype])
    counts = np.array([n - 2, 1, n, 0], np.int32)
    count = torch.from_numpy(counts).to(DEV)
    for b, m in enumerate(counts):
        q[b, m:] = odd
    att = tslt.cache_attend(q, cache, pages, lens, k=k, v=v, count=count)
    weight = torch.rand(B, H, pages.shape[1] * 64, device=DEV)
    for given in (None, count):
        got = tslt.cache_weigh(q, att["lse"], cache, pages, lens, weight, decay=0.5, count=given)
        torch.cuda.synchronize()
        assert torch.equal(got["weight"][3, :, :lengths[3]], weight[3, :, :lengths[3]] * 0.5)
        codes[tables[3, 0], 0, 0, 5] = 0                            # (the oracle multiplies NaN by 0)
        lse = att["lse"].double().cpu().numpy()
        check_weigh(got, O.weigh(qh, lse, codes, scale, tables, length, weight.cpu().numpy(), 0.5, counts), weight)


@pytest.mark.parametrize("dtype,D,H,G,n,lengths", WEIGH)
def test_a_row_that_is_nan_makes_nan_of_its_heads_weights(tslt, dtype, D, H, G, n, lengths):
    rng = np.random.default_rng([D, n, H])
    B = len(lengths)
    cache, pages, lens = on_gpu(*make_cache(rng, H, D, lengths))
    (q, k, v), _ = projection(rng, B, n, H * G, H, D, DTYPES[dtype])
    q[2, n - 1, (H - 1) * G] = float("nan")
    att = tslt.cache_attend(q, cache, pages, lens, k=k, v=v)
    weight = torch.rand(B, H, pages.shape[1] * 64, device=DEV)
    got = tslt.cache_weigh(q, att["lse"], cache, pages, lens, weight)["weight"].cpu()
    assert got[2, H - 1, :lengths[2]].isnan().all() and not got[2, H - 1, lengths[2]:].any()
    got[2, H - 1] = 0
    assert got.isfinite().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,G,length", [(2, 4, 1), (2, 4, 129), (2, 4, 6000), (20, 4, 1), (20, 4, 129), (20, 4, 6000)])
def test_scores_beyond_2_to_the_31(tslt, dtype, n, G, length):
    """Equal keys and scores so large that half a step of fp32 is many powers of two: weights are equal all the same, and the output is the mean."""
    rng = np.random.default_rng([n, length])
    D, H = 64, 1
    codes, scale, tables, lengths = make_cache(rng, H, D, [length])
    codes[:, :, 0] = 0
    codes[:, 0, 0].reshape(-1, 64, D)[..., 0] = 0x7E                # 448
    scale[..., 0] = 2.0 ** 12
    host = (codes, scale, tables, lengths)
    cache, pages, lens = on_gpu(*host)
    q = torch.zeros(1, n, G, D, dtype=DTYPES[dtype], device=DEV)
    q[0, :, :, 0] = (1 + torch.arange(n * G, device=DEV) % 8 / 8).view(n, G) * 2.0 ** 11 * (1 + torch.arange(n * G, device=DEV) // 8).view(n, G)
    got = tslt.cache_attend(q, cache, pages, lens, scale=1.0)
    torch.cuda.synchronize()
    _, value, _ = O.cached(*host[:3][:2], tables[0], length, 0)
    half = torch.finfo(DTYPES[dtype]).eps / 2
    mean, size = value.mean(0), np.abs(value).mean(0)
    off = np.abs(got["out"].double().cpu().numpy() - mean)
    assert np.all(off <= half * np.abs(mean) * (1 + 2.0 ** -10) + (2.0 ** -16 if dtype != "f32" else 2.0 ** -22) * size + 2 * (8 * 2.0 ** -24 + 2.0 ** -21) * size + torch.finfo(DTYPES[dtype]).tiny)
    want = q[..., 0].double().cpu().numpy() * 448 * 2.0 ** 12 + np.log(length)
    assert want.min() > 2.0 ** 31
    assert np.all(np.abs(got["lse"].double().cpu().numpy() / want - 1) <= 2.0 ** -21)


@pytest.mark.parametrize("length", [70, 6000])                      # one chunk and several
@pytest.mark.parametrize("n,G", [(3, 2), (40, 4)])
def test_counts_outside_the_call_are_told_and_count_as_the_nearest(tslt, length, n, G):
    rng = np.random.default_rng([n, length])
    D, H = 64, 2
    host = make_cache(rng, H, D, [length, 70, 5, 64])
    cache, pages, lens = on_gpu(*host)
    pages[2, 0] = -1
    (q, k, v), (qh, kh, vh) = projection(rng, 4, n, H * G, H, D, torch.bfloat16)
    count = torch.tensor([n + 1, -1, n + 5, n - 1], dtype=torch.int32, device=DEV)
    fit = count.clamp(0, n)
    got = tslt.cache_attend(q, cache, pages, lens, k=k, v=v, count=count)
    weight = torch.rand(4, H, pages.shape[1] * 64, device=DEV)
    w = tslt.cache_weigh(q, got["lse"], cache, pages, lens, weight, count=count)
    want = tslt.cache_attend(q, cache, pages, lens, k=k, v=v, count=fit)
    want_w = tslt.cache_weigh(q, got["lse"], cache, pages, lens, weight, count=fit)
    torch.cuda.synchronize()
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"]) and torch.equal(w["weight"], want_w["weight"])
    bad = tslt.ROW_BAD_INDEX
    assert got["status"].tolist() == w["status"].tolist() == [bad, bad, bad | tslt.ROW_BAD_PAGE, 0]
    assert want["status"].tolist() == want_w["status"].tolist() == [0, 0, tslt.ROW_BAD_PAGE, 0]


# (new tokens alone; a cache in one chunk, and in several; the kernel for few rows, and the one for many)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,G", [(5, 2), (70, 2)])
@pytest.mark.parametrize("length", [0, 70, 6000])
def test_values_near_the_largest_do_not_overflow(tslt, dtype, n, G, length):
    """Outputs are means of values: finite where these are, though the values times their weights, before the division, would pass fp32's largest."""
    rng = np.random.default_rng([n, length])
    D, H = 64, 2
    codes, scale, tables, lengths = make_cache(rng, H, D, [length])
    codes[:, :, 1][(codes[:, :, 1] & 127) == 127] = 0               # (none of the NaN behind the length)
    codes[:, :, 1].reshape(-1, H, 4, D, 16)[:, :, :, :5] = 0x7E     # of channels 0 .. 4 all 448, the others up to that
    scale[..., 1] = 2.0 ** 118
    host = (codes, scale, tables, lengths)
    cache, pages, lens = on_gpu(*host)
    (q, k, v), _ = projection(rng, 1, n, H * G, H, D, DTYPES[dtype])
    v[:] = torch.sign(v) * 1.5e38
    v[..., :5] = 1.5e38
    qh, kh, vh = (t.double().cpu().numpy() for t in (q, k, v))
    got = tslt.cache_attend(q, cache, pages, lens, k=k, v=v)
    torch.cuda.synchronize()
    check_attend(got, O.attend(qh, *host, kh, vh), DTYPES[dtype])


def reference_rows(cache, pages, length, q, scale, b, h, G):
    """Scores [n * G, length], values and, by torch in fp64 on the GPU, what attention over the cached tokens alone gives the rows of one head."""
    codes, sc = cache["codes"][:, h], cache["scale"][:, h].double()
    D = codes.shape[-1] // 64
    grid = torch.from_numpy(O.decode(np.arange(256, dtype=np.uint8))).to(DEV)
    keys = grid[codes[:, 0].long()].view(-1, 64, D) * sc[:, 0, None, None]
    values = grid[codes[:, 1].long()].view(-1, 4, D, 16).transpose(2, 3).reshape(-1, 64, D) * sc[:, 1, None, None]
    L = int(length[b])
    at = pages[b, :-(-L // 64)].long()
    k, v = keys[at].reshape(-1, D)[:L], values[at].reshape(-1, D)[:L]
    rows = q[b, :, h * G:(h + 1) * G].reshape(-1, D).double()
    s = rows @ k.T.contiguous() * scale
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - lse[:, None])
    return s, lse, p @ v, p @ v.abs(), (rows.abs() @ k.abs().T.contiguous()).amax(1) * scale


@pytest.mark.parametrize("dtype,D,H,G,n,B,long", [("bf16", 64, 8, 2, 2, 66, 70000),      # few rows: more than 64 turns of a wave
                                                  ("f32", 64, 8, 2, 2, 66, 70000),
                                                  ("f16", 128, 8, 4, 10, 66, 45000),     # 40 rows: chunks of more than 64 pages
                                                  ("f32", 64, 4, 4, 20, 130, 15000),     # 80 rows
                                                  ("bf16", 128, 4, 8, 16, 130, 15000)])  # 128 rows
def test_page_lists_of_more_than_64_entries(tslt, dtype, D, H, G, n, B, long):
    """Long sequences, enough of them that their chunks, and shares of a wave, are long too; they lie on the same pages.  More than 64 sequences."""
    rng = np.random.default_rng([D, H, B])
    n_pages, width = 300, -(-long // 64)
    codes = rng.integers(0, 256, (n_pages, H, 2, 64 * D)).astype(np.uint8)
    codes[(codes & 127) >= 120] ^= 64
    scale = np.ldexp(1.0, rng.integers(-9, -4, (n_pages, H, 2))).astype(np.float32)
    tables = rng.integers(0, n_pages, (B, width)).astype(np.int32)
    lengths = rng.integers(long - 3000, long + 1, B).astype(np.int32)
    lengths[:4] = [long, 0, 70, 64 * 64 + 1]
    cache, pages, length = on_gpu(codes, scale, tables, lengths)
    (q, _, _), _ = projection(rng, B, n, H * G, H, D, DTYPES[dtype])
    got = tslt.cache_attend(q, cache, pages, length)
    weight = torch.rand(B, H, width * 64, device=DEV)
    w = tslt.cache_weigh(q, got["lse"], cache, pages, length, weight, decay=0.5)
    torch.cuda.synchronize()
    assert not got["status"].any() and not w["status"].any()
    place = torch.arange(width * 64, device=DEV)
    assert not w["weight"][(place >= length[:, None])[:, None].expand(B, H, -1)].any()
    assert not got["out"][1].any() and torch.isneginf(got["lse"][1]).all()
    half, weight_bits = torch.finfo(DTYPES[dtype]).eps / 2, 2.0 ** -22 if dtype == "f32" else 2.0 ** -16
    for b in (0, 2, 3, 5, 40, 63, 64, 65, B - 1):
        for h in (0, H - 1):
            L = int(lengths[b])
            s, lse, out, size, reach = reference_rows(cache, pages, lengths, q, D ** -0.5, b, h, G)
            rel = 2 * (8 * 2.0 ** -24 * reach + 2.0 ** -21)
            mine = got["out"][b, :, h * G:(h + 1) * G].reshape(-1, D).double()
            tol = half * out.abs() * (1 + 2.0 ** -10) + (weight_bits + rel[:, None]) * size + torch.finfo(DTYPES[dtype]).tiny
            assert ((mine - out).abs() <= tol).all(), (b, h, float(((mine - out).abs() / tol).max()))
            got_lse = got["lse"][b, :, h * G:(h + 1) * G].reshape(-1).double()
            assert ((got_lse - lse).abs() <= rel + 2.0 ** -22 * lse.abs()).all(), (b, h)
            want = 0.5 * weight[b, h, :L].double() + torch.exp(s - got_lse[:, None]).sum(0)
            rel_w = 2 * (8 * 2.0 ** -24 * (reach + got_lse.abs()).max() + 2.0 ** -21)
            assert ((w["weight"][b, h, :L].double() - want).abs() <= (rel_w + 2.0 ** -21) * want + 2.0 ** -30).all(), (b, h)


def test_evict_from_more_than_32768_tokens(tslt):
    """Weights read from memory every time.  All pages of one scale, so that codes are moved as they are."""
    rng = np.random.default_rng(91)
    D, H, lengths, keep, recent = 64, 2, [40001, 300], 25000, 100
    codes, scale, tables, length = make_cache(rng, H, D, lengths)
    scale[:] = 2.0 ** -6
    W, first = -(-keep // 64), codes.shape[0]
    codes = np.concatenate([codes, np.full((2 * W,) + codes.shape[1:], 127, np.uint8)])
    scale = np.concatenate([scale, np.full((2 * W,) + scale.shape[1:], 1e30, np.float32)])
    new = (first + rng.permutation(2 * W)).reshape(2, W).astype(np.int32)
    weight = np.floor(rng.random((2, H, tables.shape[1] * 64)) * 1000).astype(np.float32)       # (many are equal)
    weight[0, 1, rng.random(weight.shape[2]) < 0.6] = np.nan
    cache, pages, lens = on_gpu(codes, scale, tables, length)
    got = tslt.cache_evict(cache, pages, lens, torch.from_numpy(weight).to(DEV), keep, recent, torch.from_numpy(new).to(DEV))
    torch.cuda.synchronize()
    assert got["length"].tolist() == [keep, 300] and got["status"].tolist() == [0, 0]
    after = cache["codes"].cpu().numpy()

    def tokens(table, h, part):
        x = after[table, h, part].reshape(len(table), *((64, D) if part == 0 else (4, D, 16)))
        return (x if part == 0 else x.transpose(0, 1, 3, 2)).reshape(-1, D)
    for b, L in enumerate(lengths):
        m, r = min(L, keep), min(recent, min(L, keep))
        for h in range(H):
            old = weight[b, h, :L - r]
            order = np.lexsort((np.arange(L - r), -np.where(np.isnan(old), -np.inf, old), np.isnan(old)))
            mine = np.sort(np.concatenate([order[:m - r], np.arange(L - r, L)]))
            assert np.array_equal(got["kept"][b, h, :m].cpu().numpy(), mine) and (got["kept"][b, h, m:] == -1).all()
            assert np.array_equal(got["weight"][b, h, :m].cpu().numpy(), weight[b, h, mine], equal_nan=True) and not got["weight"][b, h, m:].any()
            for part in (0, 1):
                assert np.array_equal(tokens(new[b], h, part)[:m], tokens(tables[b, :-(-L // 64)], h, part)[mine]), (b, h, part)
    assert (cache["scale"].cpu().numpy()[new[0]] == 2.0 ** -6).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,G,length", [(3, 4, 70), (3, 4, 6000), (40, 4, 70), (40, 4, 6000)])
def test_scores_beyond_2_to_the_31_of_cached_and_new_tokens_alike(tslt, dtype, n, G, length):
    rng = np.random.default_rng([n, length, 1])
    D, H = 64, 1
    codes, scale, tables, lengths = make_cache(rng, H, D, [length])
    codes[:, :, 0] = 0
    codes[:, 0, 0].reshape(-1, 64, D)[..., 0] = 0x7E                # 448
    scale[..., 0] = 2.0 ** 12
    cache, pages, lens = on_gpu(codes, scale, tables, lengths)
    (q, k, v), (_, _, vh) = projection(rng, 1, n, G, H, D, DTYPES[dtype])
    q[:], k[:] = 0, 0
    q[0, :, :, 0] = (1 + torch.arange(n * G, device=DEV) % 8 / 8).view(n, G) * 2.0 ** 11
    k[..., 0] = 448 * 2.0 ** 12
    got = tslt.cache_attend(q, cache, pages, lens, k=k, v=v, scale=1.0)
    torch.cuda.synchronize()
    _, value, _ = O.cached(codes, scale, tables[0], length, 0)
    half, weight_bits = torch.finfo(DTYPES[dtype]).eps / 2, 2.0 ** -22 if dtype == "f32" else 2.0 ** -16
    for i in range(n):
        seen = np.concatenate([value, vh[0, :i + 1, 0]])
        off = np.abs(got["out"][0, i].double().cpu().numpy() - seen.mean(0))
        tol = half * np.abs(seen.mean(0)) * (1 + 2.0 ** -10) + (weight_bits + 2 * (8 * 2.0 ** -24 + 2.0 ** -21)) * np.abs(seen).mean(0)
        assert np.all(off <= tol), (i, float((off / tol).max()))
