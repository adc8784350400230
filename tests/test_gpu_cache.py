"""The calls around the 8-bit cache against the fp64 oracle.

Tolerances, from the arithmetic.  A score is a sum of D exact products in fp32: with R the largest sum of magnitudes
|q||k| * scale of a row, it is off by at most D * 2^-24 * R and in practice by far less; 8 * 2^-24 * R is allowed, and with it a
factor exp(that) on a weight and as much on the sum of weights.  Beside it exp2 and log2 are good to some 2^-22.  A weight is
two bfloat16 terms (the first cut off, the second rounded: off by 2^-16) for rows of 16 bits, three for fp32 (off by less than fp32 is),
before it meets the values: with A = sum p |v| that is 2^-16 A, or 2^-22 A.  The output's own rounding is half a step of its type.
"""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def rel_of_scores(reach):
    return 2 * (8 * 2.0 ** -24 * reach + 2.0 ** -21)


def check_attend(got, want, dtype):
    out, lse, size, reach = want
    weight_bits = 2.0 ** -22 if dtype == torch.float32 else 2.0 ** -16
    half = torch.finfo(dtype).eps / 2
    tol = half * np.abs(out) * (1 + 2.0 ** -10) + (weight_bits + rel_of_scores(reach)[..., None]) * size + torch.finfo(dtype).tiny
    off = np.abs(got["out"].double().cpu().numpy() - out)
    assert np.all(off <= tol), (float((off / tol).max()), np.argwhere(off > tol)[:3].tolist())
    mine = got["lse"].double().cpu().numpy()
    assert np.array_equal(np.isneginf(mine), np.isneginf(lse))
    fine = ~np.isneginf(lse)
    off = np.abs(mine[fine] - lse[fine])
    assert np.all(off <= rel_of_scores(reach[fine]) + 2.0 ** -22 * np.abs(lse[fine])), float(off.max())


def make_cache(rng, H, D, lengths, spare=0, wide=False):
    """A cache with sequences of these lengths on pages in no order; NaN codes in all places that no token has."""
    used = [-(-x // 64) for x in lengths]
    width = max(max(used) + spare, 1)
    n_pages = max(1, sum(used) + spare * len(lengths)) + 2
    codes = rng.integers(0, 256, (n_pages, H, 2, 64 * D)).astype(np.uint8)
    codes[(codes & 127) >= 120] ^= 64                             # no NaN among them, and few of the largest
    scale = np.ldexp(1.0, rng.integers(-9 if not wide else -40, -4 if not wide else 3, (n_pages, H, 2))).astype(np.float32)
    order = rng.permutation(n_pages)
    tables, at = np.full((len(lengths), width), -1, np.int32), 0
    for b, x in enumerate(lengths):
        m = used[b] + spare
        tables[b, :m] = order[at:at + m]
        at += m
        if x % 64:
            page = tables[b, used[b] - 1]
            codes[page, :, 0].reshape(H, 64, D)[:, x % 64:] = 127
            v = codes[page, :, 1].reshape(H, 4, D, 16).transpose(0, 1, 3, 2).reshape(H, 64, D).copy()
            v[:, x % 64:] = 255
            codes[page, :, 1] = v.reshape(H, 4, 16, D).transpose(0, 1, 3, 2).reshape(H, -1)
        for w in range(used[b], m):
            codes[tables[b, w]] = 127
    return codes, scale, tables, np.array(lengths, np.int32)


def on_gpu(codes, scale, tables, lengths):
    return ({"codes": torch.from_numpy(codes).to(DEV), "scale": torch.from_numpy(scale).to(DEV)}, torch.from_numpy(tables).to(DEV),
            torch.from_numpy(lengths).to(DEV))


def projection(rng, B, n, Hq, H, D, dtype):
    """q, k, v as views of one projection's rows, and the same in fp64."""
    x = torch.from_numpy(rng.normal(size=(B, n, Hq + 2 * H, D)).astype(np.float32)).to(dtype).to(DEV)
    q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:]
    return (q, k, v), tuple(t.double().cpu().numpy() for t in (q, k, v))


ATTEND = [  # dtype, D, heads, group, n, lengths
    ("bf16", 128, 2, 4, 1, [0, 1, 63, 64, 65, 300]),
    ("f16", 64, 3, 1, 1, [500]),
    ("f32", 64, 1, 1, 1, [0]),
    ("f32", 128, 2, 3, 5, [130, 0, 1]),
    ("bf16", 64, 1, 7, 9, [1000, 17]),
    ("f16", 128, 2, 8, 9, [127, 640, 5]),
    ("bf16", 256, 2, 2, 3, [100, 64]),
    ("f32", 256, 1, 4, 6, [90, 0]),
    ("f16", 256, 1, 1, 40, [65]),
    ("bf16", 128, 1, 4, 70, [200, 3]),
    ("f32", 128, 1, 2, 67, [70]),
    ("f16", 64, 2, 5, 65, [0, 129]),
    ("bf16", 128, 2, 1, 17, [5000]),
    ("bf16", 64, 1, 1, 300, [31]),
    ("bf16", 128, 1, 3, 10, [400, 0]),
    ("f32", 64, 2, 12, 4, [66, 700]),
]


@pytest.mark.parametrize("dtype,D,H,G,n,lengths", ATTEND)
def test_chain_over_the_cache(tslt, dtype, D, H, G, n, lengths):
    rng = np.random.default_rng([D, H, G, n, len(lengths), lengths[0]])
    host = make_cache(rng, H, D, lengths, spare=1)
    cache, pages, length = on_gpu(*host)
    (q, k, v), (qh, kh, vh) = projection(rng, len(lengths), n, H * G, H, D, DTYPES[dtype])
    got = tslt.cache_attend(q, cache, pages, length, k=k, v=v)
    torch.cuda.synchronize()
    check_attend(got, O.attend(qh, *host, kh, vh), DTYPES[dtype])
    assert got["status"].tolist() == [0] * len(lengths)
    alone = tslt.cache_attend(q, cache, pages, length, scale=0.3)
    torch.cuda.synchronize()
    check_attend(alone, O.attend(qh, *host, softmax_scale=0.3), DTYPES[dtype])


@pytest.mark.parametrize("dtype,D,expansion,G,lengths", [("f32", 128, (2, 2, 2), 2, [70, 0]), ("bf16", 128, (4, 4, 4), 4, [200, 1]),
                                                         ("f16", 64, (3, 1, 2), 1, [64, 10]), ("bf16", 256, (33,), 1, [100]),
                                                         ("f32", 64, (16, 4), 3, [300])])
def test_tree_sees_its_ancestors(tslt, dtype, D, expansion, G, lengths):
    mask = tslt.tree_mask(expansion, DEV)
    n, H, B = mask.shape[1], 2, len(lengths)
    rng = np.random.default_rng([n, D, G])
    host = make_cache(rng, H, D, lengths)
    cache, pages, length = on_gpu(*host)
    (q, k, v), (qh, kh, vh) = projection(rng, B, n, H * G, H, D, DTYPES[dtype])
    got = tslt.cache_attend(q, cache, pages, length, k=k, v=v, mask=mask)
    torch.cuda.synchronize()
    check_attend(got, O.attend(qh, *host, kh, vh, mask.cpu().numpy()), DTYPES[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n", [9, 70, 130])
def test_masks_of_their_own_counts_and_rows_that_see_nothing(tslt, dtype, n):
    """A mask for each sequence, at random, with empty rows; fewer tokens than rows; tokens that nobody, or not everybody, sees hold
    NaN, infinities and the largest numbers."""
    rng = np.random.default_rng(n)
    D, H, G, lengths = 128, 2, 2, [0, 70, 0, 129]
    B, words = len(lengths), (n + 31) // 32
    host = make_cache(rng, H, D, lengths)
    cache, pages, length = on_gpu(*host)
    seen = rng.random((B, n, n)) < 0.2
    seen[:, ::3] = False
    seen[:, :, 4] = False                                         # token 4 is seen by nobody
    seen[:, :, 6] = False
    seen[:, 2, 6] = True                                          # token 6 by row 2 alone
    bits = np.zeros((B, n, words * 32), bool)
    bits[:, :, :n] = seen
    bits[:, :, n:] = True                                         # (bits of tokens that there are none of mean nothing)
    mask = np.packbits(bits, axis=-1, bitorder="little").view(np.uint32).astype(np.int64)
    mask = np.where(mask >= 1 << 31, mask - (1 << 32), mask).astype(np.int32)
    count = np.array([n, n - 2, 3, 0], np.int32)
    (q, k, v), (qh, kh, vh) = projection(rng, B, n, H * G, H, D, DTYPES[dtype])
    big = torch.finfo(DTYPES[dtype]).max
    k[:, 4], v[:, 4] = float("nan"), float("inf")
    v[:, 6, :, 5] = float("inf")
    v[:, 6, 1, 8] = -float("inf")
    k[1, n - 1], v[1, n - 1] = float("nan"), float("nan")         # behind the count
    k[2, 3:], v[2, 3:] = -float("inf"), big
    got = tslt.cache_attend(q, cache, pages, length, k=k, v=v, mask=torch.from_numpy(mask).to(DEV), count=torch.from_numpy(count).to(DEV))
    torch.cuda.synchronize()
    want = O.attend(qh, *host, kh, vh, mask, count)                # (kh, vh: before the odd numbers went in)
    out = got["out"].double().cpu().numpy()
    row2 = want[1][:, 2] > -np.inf
    there = (count > 6)[:, None] & row2
    assert there.sum() == 8
    for b, hq in zip(*np.nonzero(there)):
        assert out[b, 2, hq, 5] == np.inf
        if hq // G == 1:
            assert out[b, 2, hq, 8] == -np.inf
            got["out"][b, 2, hq, 8] = float(want[0][b, 2, hq, 8])
        got["out"][b, 2, hq, 5] = float(want[0][b, 2, hq, 5])
    assert np.isneginf(want[1]).sum() > 0
    check_attend(got, want, DTYPES[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_few_large_scores_late_in_a_long_cache(tslt, dtype):
    """The maximum grows along the sequence, scales of pages differ by powers up to 2^40, and one token outweighs all others."""
    rng = np.random.default_rng(11)
    D, H, lengths = 64, 1, [3000]
    host = make_cache(rng, H, D, lengths, wide=True)
    host[1][..., 0] = 2.0 ** -7
    cache, pages, length = on_gpu(*host)
    (q, k, v), _ = projection(rng, 1, 3, 4, H, D, DTYPES[dtype])
    q.mul_(torch.linspace(0.01, 6, 12, device=DEV).view(1, 3, 4, 1).to(q.dtype))
    qh, kh, vh = (t.double().cpu().numpy() for t in (q, k, v))
    got = tslt.cache_attend(q, cache, pages, length, k=k, v=v)
    torch.cuda.synchronize()
    check_attend(got, O.attend(qh, *host, kh, vh), DTYPES[dtype])


def test_pages_outside_the_cache_and_lengths_outside_the_table(tslt):
    rng = np.random.default_rng(12)
    D, H, lengths = 64, 2, [200, 130, 64, 100]
    codes, scale, tables, length = make_cache(rng, H, D, lengths)
    tables[0, 1] = codes.shape[0]
    tables[1, 2] = -5
    length[2] = -3
    length[3] = 64 * tables.shape[1] + 1
    want_length = np.array([200, 130, 0, 64 * tables.shape[1]])
    tables[3] = tables[0, 0]
    tables[3, 1:] = [tables[1, 0]] * (tables.shape[1] - 1)
    cache, pages, lens = on_gpu(codes, scale, tables, length)
    (q, k, v), (qh, kh, vh) = projection(rng, 4, 2, 4, H, D, torch.bfloat16)
    got = tslt.cache_attend(q, cache, pages, lens, k=k, v=v)
    torch.cuda.synchronize()
    assert got["status"].tolist() == [16, 16, 16, 16]
    check_attend(got, O.attend(qh, codes, scale, tables, want_length, kh, vh), torch.bfloat16)
    weight = torch.rand(4, H, 64 * tables.shape[1], device=DEV)
    w = tslt.cache_weigh(q, got["lse"], cache, pages, lens, weight)
    torch.cuda.synchronize()
    assert w["status"].tolist() == [16, 16, 16, 16]
    check_weigh(w, O.weigh(qh, got["lse"].double().cpu().numpy(), codes, scale, tables, want_length, weight.cpu().numpy(), 1.0), weight)


def check_weigh(got, want, weight):
    out, reach = want
    mine = got["weight"].double().cpu().numpy()
    tol = (rel_of_scores(reach) + 2.0 ** -21) * out + 2.0 ** -30
    assert np.all(np.abs(mine - out) <= tol), float((np.abs(mine - out) / tol).max())
    assert np.all(mine[out == 0] == 0)


@pytest.mark.parametrize("dtype,D,H,G,n,lengths,decay", [("f32", 64, 3, 1, 5, [150, 0], 1.0), ("bf16", 128, 2, 4, 9, [64, 700, 1], 0.9),
                                                         ("f16", 256, 1, 2, 3, [65], 0.0), ("bf16", 64, 1, 8, 70, [130], 0.5),
                                                         ("f32", 128, 2, 3, 17, [63, 5], -1.0)])
def test_weights_are_those_of_the_attention(tslt, dtype, D, H, G, n, lengths, decay):
    rng = np.random.default_rng([D, n])
    B = len(lengths)
    host = make_cache(rng, H, D, lengths, spare=2)
    cache, pages, length = on_gpu(*host)
    (q, k, v), (qh, kh, vh) = projection(rng, B, n, H * G, H, D, DTYPES[dtype])
    count = torch.tensor([n - b % 3 for b in range(B)], dtype=torch.int32, device=DEV).clamp_min(0)
    att = tslt.cache_attend(q, cache, pages, length, k=k, v=v, count=count)
    weight = torch.rand(B, H, pages.shape[1] * 64, device=DEV)
    if decay < 0:                                                 # in place, on weights that are nothing behind the length
        decay = 0.25
        out = {"weight": weight.clone()}
        got = tslt.cache_weigh(q, att["lse"], cache, pages, length, out["weight"], decay=decay, count=count, out=out)
    else:
        got = tslt.cache_weigh(q, att["lse"], cache, pages, length, weight, decay=decay, count=count)
    torch.cuda.synchronize()
    lse = att["lse"].double().cpu().numpy()
    check_weigh(got, O.weigh(qh, lse, *host, weight.cpu().numpy(), decay, count.cpu().numpy()), weight)
    again = tslt.cache_weigh(q, att["lse"], cache, pages, length, weight, decay=decay, count=count)
    assert torch.equal(again["weight"], got["weight"])
    if decay == 1.0:                                              # cached and new tokens together get one from every row
        total = (got["weight"] - weight * (torch.arange(weight.shape[2], device=DEV) < length[:, None, None])).sum((1, 2))
        assert np.all(total.cpu().numpy() <= count.cpu().numpy() * H * G * (1 + 1e-4))


@pytest.mark.parametrize("dtype,D,H,G,n,lengths", [("bf16", 128, 2, 4, 41, [64, 700, 0, 1]), ("f32", 128, 1, 8, 37, [130, 65, 7, 640]),
                                                   ("f16", 256, 2, 2, 90, [1, 200, 64, 128]), ("f32", 64, 1, 1, 150, [70, 3, 0, 129]),
                                                   ("f32", 256, 1, 3, 47, [90, 64, 1, 300]), ("bf16", 64, 3, 1, 333, [127, 64, 300, 9])])
def test_weights_of_many_rows_on_few_pages(tslt, dtype, D, H, G, n, lengths):
    rng = np.random.default_rng([D, n, 5])
    B = len(lengths)
    host = make_cache(rng, H, D, lengths, spare=1)
    cache, pages, length = on_gpu(*host)
    (q, k, v), (qh, kh, vh) = projection(rng, B, n, H * G, H, D, DTYPES[dtype])
    for counts in ([n, n - 1, 1, n], [0, n, 17, 33]):             # (of few of them some waves have none)
        count = torch.tensor(counts, dtype=torch.int32, device=DEV)
        att = tslt.cache_attend(q, cache, pages, length, k=k, v=v, count=count)
        weight = torch.rand(B, H, pages.shape[1] * 64, device=DEV)
        got = tslt.cache_weigh(q, att["lse"], cache, pages, length, weight, decay=0.7, count=count)
        torch.cuda.synchronize()
        check_weigh(got, O.weigh(qh, att["lse"].double().cpu().numpy(), *host, weight.cpu().numpy(), 0.7, count.cpu().numpy()), weight)
        again = tslt.cache_weigh(q, att["lse"], cache, pages, length, weight, decay=0.7, count=count)
        assert torch.equal(again["weight"], got["weight"]) and not got["status"].any()


def same_values(got, want, table, length, H):
    """Codes as the numbers they stand for, wherever there is a token; scales bit for bit."""
    for b, L in enumerate(length):
        for w in range(-(-int(L) // 64)):
            page = int(table[b][w])
            if not 0 <= page < got[0].shape[0]:
                continue
            assert np.array_equal(got[1][page], want[1][page]), (b, w, got[1][page], want[1][page])
            for h in range(H):
                m = min(64, int(L) - 64 * w)
                for x, y in zip(O.page_values(*got, page, h), O.page_values(*want, page, h)):
                    assert np.array_equal(x[:m], y[:m], equal_nan=True), (b, w, h)


APPEND = [  # dtype, D, heads, n, lengths, chosen
    ("bf16", 128, 2, 1, [0, 1, 15, 16, 63, 64, 100], False),
    ("f32", 64, 3, 9, [0, 60, 55, 130], True),
    ("f16", 256, 1, 5, [62, 10], True),
    ("bf16", 64, 1, 130, [0, 63, 64], False),
    ("f32", 128, 2, 66, [63, 127], True),
    ("f16", 128, 2, 64, [0, 1], False),
    ("f32", 256, 1, 20, [50], False),
]


@pytest.mark.parametrize("dtype,D,H,n,lengths,chosen", APPEND)
def test_append_is_exact(tslt, dtype, D, H, n, lengths, chosen):
    rng = np.random.default_rng([D, n, len(lengths)])
    B = len(lengths)
    host = make_cache(rng, H, D, lengths, spare=-(-n // 64) + 1)
    cache, pages, length = on_gpu(*host)
    _, k, v = projection(rng, B, n, 1, H, D, DTYPES[dtype])[0]
    k.mul_(torch.from_numpy(10.0 ** rng.uniform(-4, 3, (B, 1, H, 1)).astype(np.float32)).to(DEV).to(k.dtype))      # smaller and larger than what is there
    v.mul_(torch.from_numpy(10.0 ** rng.uniform(-4, 3, (B, 1, H, 1)).astype(np.float32)).to(DEV).to(k.dtype))
    index = count = None
    if chosen:
        count = rng.integers(0, n + 1, B).astype(np.int32)
        count[0] = n
        index = np.stack([rng.permutation(n) for _ in range(B)]).astype(np.int32)
    kh, vh = (t.double().cpu().numpy() for t in (k, v))
    want = O.append(*host, kh, vh, index, count)
    dev = [None if x is None else torch.from_numpy(x).to(DEV) for x in (count, index)]
    got = tslt.cache_append(cache, pages, length, k, v, count=dev[0], index=dev[1])
    torch.cuda.synchronize()
    assert got["length"].tolist() == want[2].tolist() and got["status"].tolist() == [0] * B
    same_values((cache["codes"].cpu().numpy(), cache["scale"].cpu().numpy()), want[:2], host[2], want[2], H)
    # once more: what is there already makes no difference
    tslt.cache_append(cache, pages, length, k, v, count=dev[0], index=dev[1])
    torch.cuda.synchronize()
    same_values((cache["codes"].cpu().numpy(), cache["scale"].cpu().numpy()), want[:2], host[2], want[2], H)


def test_append_of_a_few_of_many_tokens(tslt):
    """Index rows of their own width, narrower and wider than the call's tokens."""
    rng = np.random.default_rng(22)
    D, H, B, lengths = 128, 5, 3, [60, 0, 64]
    for n, m, counts in ((40, 4, [4, 0, 2]), (3, 70, [70, 1, 33]), (100, 17, None)):
        host = make_cache(rng, H, D, lengths, spare=3)
        cache, pages, length = on_gpu(*host)
        _, k, v = projection(rng, B, n, 1, H, D, torch.bfloat16)[0]
        index = rng.integers(0, n, (B, m)).astype(np.int32)
        count = None if counts is None else np.array(counts, np.int32)
        want = O.append(*host, *(t.double().cpu().numpy() for t in (k, v)), index, count)
        got = tslt.cache_append(cache, pages, length, k, v, index=torch.from_numpy(index).to(DEV),
                                count=None if count is None else torch.from_numpy(count).to(DEV))
        torch.cuda.synchronize()
        assert got["length"].tolist() == want[2].tolist() and got["status"].tolist() == [0] * B
        same_values((cache["codes"].cpu().numpy(), cache["scale"].cpu().numpy()), want[:2], host[2], want[2], H)


def test_a_page_that_is_begun_is_cleared_behind_its_last_token(tslt):
    for D, n, tokens in ((64, 5, 5), (128, 130, 2), (256, 65, 1)):
        cache = tslt.cache_create(4, 2, D, DEV)
        cache["codes"].fill_(127)
        pages = torch.tensor([[2, 0, 3]], dtype=torch.int32, device=DEV)
        k, v = torch.randn(2, 1, n, 2, D, device=DEV)
        tslt.cache_append(cache, pages, torch.zeros(1, dtype=torch.int32, device=DEV), k, v)
        torch.cuda.synchronize()
        last = pages[0, (n - 1) // 64].item()
        codes = cache["codes"][last].cpu()
        assert not codes[:, 0].view(2, 64, D)[:, tokens:].any()
        assert not codes[:, 1].view(2, 4, D, 16).transpose(2, 3).reshape(2, 64, D)[:, tokens:].any()
        assert (cache["codes"][1] == 127).all()                    # and no other page is touched


def test_append_of_what_is_not_finite_zero_or_out_of_place(tslt):
    rng = np.random.default_rng(21)
    D, H, n, lengths = 64, 2, 6, [10, 61, 120, 126]
    codes, scale, tables, length = make_cache(rng, H, D, lengths, spare=0)
    tables = np.concatenate([tables, np.full((4, 1), -1, np.int32)], 1)
    tables[1, 1] = codes.shape[0] + 7                              # the page that the second sequence goes on to
    tables = np.ascontiguousarray(tables[:, :2])                   # room for 128 tokens
    cache, pages, lens = on_gpu(codes, scale, tables, length)
    _, k, v = projection(rng, 4, n, 1, H, D, torch.float32)[0]
    k[0, 0, 0, 3], k[0, 1, 0, 4], k[0, 2, 1, 5] = float("inf"), -float("inf"), float("nan")
    k[0, :, 0, 6] = 1e-30
    v[0] = 0
    index = np.tile(np.arange(n, dtype=np.int32), (4, 1))
    index[2, 1] = n
    count = np.array([n, n, 5, n + 4], np.int32)
    kh, vh = (t.double().cpu().numpy() for t in (k, v))
    want = O.append(codes, scale, tables, length, kh, vh, index, np.minimum(count, n))
    got = tslt.cache_append(cache, pages, lens, k, v, count=torch.from_numpy(count).to(DEV), index=torch.from_numpy(index).to(DEV))
    torch.cuda.synchronize()
    assert got["length"].tolist() == [16, 67, 125, 128]
    assert got["status"].tolist() == [0, tslt.ROW_BAD_PAGE, tslt.ROW_BAD_INDEX, tslt.ROW_BAD_PAGE | tslt.ROW_BAD_INDEX]
    same_values((cache["codes"].cpu().numpy(), cache["scale"].cpu().numpy()), want[:2], tables, got["length"].tolist(), H)
    held = O.page_values(cache["codes"].cpu().numpy(), cache["scale"].cpu().numpy(), tables[0, 0], 0)[0]
    assert held[10, 3] == 448 * cache["scale"][tables[0, 0], 0, 0].item() == -held[11, 4]


EVICT = [  # D, heads, lengths, keep, recent
    (64, 2, [300, 10, 0], 100, 20),
    (128, 1, [64, 65, 700], 64, 0),
    (256, 2, [130], 129, 200),
    (64, 1, [5000], 37, 5),
    (128, 3, [1000, 999], 900, 1),
]


@pytest.mark.parametrize("D,H,lengths,keep,recent", EVICT)
@pytest.mark.parametrize("ties", [False, True])
def test_evict_is_exact(tslt, D, H, lengths, keep, recent, ties):
    rng = np.random.default_rng([D, keep, recent])
    B = len(lengths)
    codes, scale, tables, length = make_cache(rng, H, D, lengths)
    W = -(-keep // 64) + 1
    first = codes.shape[0]
    codes = np.concatenate([codes, np.full((B * W,) + codes.shape[1:], 127, np.uint8)])
    scale = np.concatenate([scale, np.full((B * W,) + scale.shape[1:], 1e30, np.float32)])
    new = (first + rng.permutation(B * W)).reshape(B, W).astype(np.int32)
    weight = rng.random((B, H, tables.shape[1] * 64)).astype(np.float32) ** 4
    if ties:
        weight = np.floor(weight * 3).astype(np.float32) * np.where(rng.random(weight.shape) < 0.5, -0.0, 1).astype(np.float32)
        weight[:, :, ::17] = np.nan
        weight[:, :, 3::29] = -np.inf
        weight[:, :, 4::31] = np.inf
    cache, pages, lens = on_gpu(codes, scale, tables, length)
    got = tslt.cache_evict(cache, pages, lens, torch.from_numpy(weight).to(DEV), keep, recent, torch.from_numpy(new).to(DEV))
    torch.cuda.synchronize()
    want = O.evict(codes, scale, tables, length, weight, keep, recent, new)
    assert got["status"].tolist() == [0] * B
    assert np.array_equal(got["length"].cpu().numpy(), want[2])
    assert np.array_equal(got["kept"].cpu().numpy(), want[3])
    assert np.array_equal(got["weight"].cpu().numpy(), want[4], equal_nan=True)
    after = (cache["codes"].cpu().numpy(), cache["scale"].cpu().numpy())
    same_values(after, want[:2], new, want[2], H)
    assert np.array_equal(after[0][:first], codes[:first]) and np.array_equal(after[1][:first], scale[:first])      # the old pages are as they were


def test_evict_from_and_to_pages_outside_the_cache(tslt):
    rng = np.random.default_rng(31)
    D, H, lengths, keep = 64, 2, [200, 150], 100
    codes, scale, tables, length = make_cache(rng, H, D, lengths, spare=1)
    new = np.stack([tables[b, [len(tables[b]) - 1, 0]] for b in range(2)]).astype(np.int32)
    used = [-(-x // 64) for x in lengths]
    new = np.array([[tables[0, used[0]], -1], [tables[1, used[1]], codes.shape[0]]], np.int32)
    tables[0, 1] = codes.shape[0] + 1
    weight = rng.random((2, H, tables.shape[1] * 64)).astype(np.float32)
    cache, pages, lens = on_gpu(codes, scale, tables, length)
    got = tslt.cache_evict(cache, pages, lens, torch.from_numpy(weight).to(DEV), keep, 10, torch.from_numpy(new).to(DEV))
    torch.cuda.synchronize()
    want = O.evict(codes, scale, tables, length, weight, keep, 10, new)
    assert got["status"].tolist() == [16, 16]
    assert np.array_equal(got["kept"].cpu().numpy(), want[3])
    same_values((cache["codes"].cpu().numpy(), cache["scale"].cpu().numpy()), want[:2], new, want[2], H)


def test_more_than_two_gigabytes_of_codes(tslt):
    """Offsets that pass 32 bits: the last pages of a cache of 2.3 * 2^31 bytes."""
    D, H = 128, 8
    n_pages = int(2.3 * 2 ** 31) // (H * 2 * 64 * D)
    cache = tslt.cache_create(n_pages, H, D, DEV)
    rng = np.random.default_rng(41)
    pages = torch.tensor([[n_pages - 1, n_pages // 2, n_pages - 2, 0]], dtype=torch.int32, device=DEV)
    length = torch.zeros(1, dtype=torch.int32, device=DEV)
    (q, k, v), (qh, kh, vh) = projection(rng, 1, 150, H, H, D, torch.float16)
    length = tslt.cache_append(cache, pages, length, k, v)["length"]
    few = {name: x[pages[0].long()].cpu().numpy() for name, x in cache.items()}
    got = tslt.cache_attend(q[:, :2], cache, pages, length)
    torch.cuda.synchronize()
    tables = np.arange(4)[None]
    want = O.append(np.zeros_like(few["codes"]), np.ones_like(few["scale"]), tables, np.zeros(1, int), kh, vh)
    same_values((few["codes"], few["scale"]), want[:2], tables, [150], H)
    check_attend(got, O.attend(qh[:, :2], few["codes"], few["scale"], tables, np.array([150])), torch.float16)


def test_on_another_stream_and_with_the_callers_buffers(tslt):
    rng = np.random.default_rng(51)
    D, H, G, n, lengths = 128, 2, 4, 3, [900, 4000]
    host = make_cache(rng, H, D, lengths)
    cache, pages, length = on_gpu(*host)
    (q, k, v), (qh, kh, vh) = projection(rng, 2, n, H * G, H, D, torch.bfloat16)
    out = {"out": torch.empty(2, n, H * G, D, dtype=torch.bfloat16, device=DEV), "lse": torch.empty(2, n, H * G, device=DEV)}
    ws = torch.empty(tslt.cache_attend_workspace_bytes(2, n, H * G, H, D, pages.shape[1]), dtype=torch.uint8, device=DEV).fill_(255)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        tslt.cache_attend(q, cache, pages, length, k=k, v=v, out=out, workspace=ws)
    side.synchronize()
    check_attend(out, O.attend(qh, *host, kh, vh), torch.bfloat16)
    with pytest.raises(tslt.TsltError, match="entries"):
        tslt.cache_attend(q, cache, pages, length, k=k, v=v, out={"out": out["out"], "lse": out["lse"][:1]}, workspace=ws)
    with pytest.raises(tslt.TsltError, match="mask must be"):
        tslt.cache_attend(q, cache, pages, length, k=k, v=v, mask=torch.zeros(2, n, 2, dtype=torch.int32, device=DEV))
    with pytest.raises(tslt.TsltError, match="16 bytes"):
        odd = torch.zeros(2, n, H * G, D + 1, dtype=torch.bfloat16, device=DEV)[..., :D]
        tslt.cache_attend(odd, cache, pages, length)
    with pytest.raises(tslt.TsltError, match="dense"):
        tslt.cache_append(cache, pages, length, k.transpose(2, 3).contiguous().transpose(2, 3), v)


def test_captured_round_replays_like_eager(tslt):
    """Attend, weigh and append of accepted tokens in one graph; lengths and counts are read on the device."""
    rng = np.random.default_rng(61)
    D, H, G, n, lengths = 64, 2, 2, 5, [100, 640, 30]
    host = make_cache(rng, H, D, lengths, spare=1)
    cache, pages, length = on_gpu(*host)
    fresh = {name: x.clone() for name, x in cache.items()}
    weight = torch.rand(3, H, pages.shape[1] * 64, device=DEV)
    sets = [projection(np.random.default_rng(70 + i), 3, n, H * G, H, D, torch.bfloat16)[0] for i in range(3)]
    counts = [torch.tensor(c, dtype=torch.int32, device=DEV) for c in ([5, 1, 3], [2, 4, 5], [1, 1, 1])]
    q, k, v = (x.clone() for x in sets[0])
    count, out_w = counts[0].clone(), torch.empty_like(weight)
    att, app, wgh = {}, {}, {}

    def run(att, wgh, app):
        att = tslt.cache_attend(q, cache, pages, length, k=k, v=v, out=att or None, workspace=ws)
        wgh = tslt.cache_weigh(q, att["lse"], cache, pages, length, weight, out=wgh or None)
        return att, wgh, tslt.cache_append(cache, pages, length, k, v, count=count, out=app or None)

    ws = torch.empty(max(256, tslt.cache_attend_workspace_bytes(3, n, H * G, H, D, pages.shape[1])), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        att, wgh, app = run(att, wgh, app)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(att, wgh, app)
    for rep in range(2):
        for i in range(3):
            results = []
            for captured in (False, True):
                for name, x in cache.items():
                    x.copy_(fresh[name])
                for x, y in zip((q, k, v, count), (*sets[i], counts[i])):
                    x.copy_(y)
                torch.cuda.synchronize()
                graph.replay() if captured else run(att, wgh, app)
                torch.cuda.synchronize()
                results.append([x.clone() for x in (att["out"], att["lse"], wgh["weight"], app["length"], cache["codes"], cache["scale"])])
            assert all(torch.equal(x, y) for x, y in zip(*results)), (rep, i)


@pytest.mark.parametrize("dtype,n,G", [("bf16", 3, 4), ("f16", 9, 4), ("f32", 40, 4)])          # the kernel for few rows, and the one for many
def test_captured_chunks_replay_like_eager(tslt, dtype, n, G):
    """A sequence cut into chunks that its workgroups join: every replay finds the words that the one before left, and none of its own."""
    rng = np.random.default_rng(n)
    D, H, lengths = 128, 1, [6000, 300, 4096]
    host = make_cache(rng, H, D, lengths)
    cache, pages, length = on_gpu(*host)
    need = tslt.cache_attend_workspace_bytes(3, n, H * G, H, D, pages.shape[1])
    assert need > 256                                             # more than one chunk
    ws = torch.empty(need, dtype=torch.uint8, device=DEV).fill_(1)
    sets = [projection(np.random.default_rng(80 + i), 3, n, H * G, H, D, DTYPES[dtype]) for i in range(2)]
    q, k, v = (x.clone() for x in sets[0][0])
    out = {"out": torch.empty_like(q), "lse": torch.empty(3, n, H * G, device=DEV), "status": torch.empty(3, dtype=torch.int32, device=DEV)}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        tslt.cache_attend(q, cache, pages, length, k=k, v=v, out=out, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tslt.cache_attend(q, cache, pages, length, k=k, v=v, out=out, workspace=ws)
    want = [O.attend(qh, *host, kh, vh) for _, (qh, kh, vh) in sets]
    for rep in range(3):
        for i in (0, 1):
            for x, y in zip((q, k, v), sets[i][0]):
                x.copy_(y)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            check_attend(out, want[i], DTYPES[dtype])
            assert out["status"].tolist() == [0, 0, 0]
            replayed = {name: x.clone() for name, x in out.items()}
            tslt.cache_attend(q, cache, pages, length, k=k, v=v, out=out, workspace=ws)
            torch.cuda.synchronize()
            check_attend(out, want[i], DTYPES[dtype])
            assert all(torch.equal(out[name], replayed[name]) for name in out)
