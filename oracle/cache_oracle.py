"""Oracle of the 8-bit key/value cache: NumPy, fp64, from the definitions in include/tslt.h; it shares no code with csrc/.

A cache here is codes [n_pages, heads, 2, 64 * D] uint8 and scale [n_pages, heads, 2] float32, as the library's; `values` and
`store` know their layout and nothing else does.
"""
from __future__ import annotations

import numpy as np

PAGE = 64
MIN_EXP = -100


def decode(codes: np.ndarray) -> np.ndarray:
    """OCP e4m3: sign, four bits of exponent with bias 7 (0: subnormal), three of mantissa; all ones is NaN."""
    b = codes.astype(np.int64)
    e, m = b >> 3 & 15, b & 7
    mag = np.where(e > 0, np.ldexp(1 + m / 8, e - 7), np.ldexp(m / 8, -6))
    mag = np.where((b & 127) == 127, np.nan, mag)
    return np.where(b >= 128, -mag, mag)


_GRID = decode(np.arange(127, dtype=np.uint8))          # magnitudes of the codes 0..126, ascending


def encode(x: np.ndarray) -> np.ndarray:
    """Nearest code, ties to the even one; what lies beyond the largest becomes it; NaN is NaN."""
    x = np.asarray(x, dtype=np.float64)
    mag = np.minimum(np.abs(np.where(np.isnan(x), 0, x)), 448.0)
    hi = np.searchsorted(_GRID, mag).clip(0, 126)
    lo = np.maximum(hi - 1, 0)
    down, up = mag - _GRID[lo], _GRID[hi] - mag
    code = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.isnan(x), 127, code)
    return (code + 128 * np.signbit(x)).astype(np.uint8)


def least_scale(most: float) -> float:
    """The least 2^e, e >= MIN_EXP, that brings `most` to 448 or less."""
    e = MIN_EXP
    while 448.0 * 2.0 ** e < most:
        e += 1
    return 2.0 ** e


def page_values(codes, scale, page, h):
    """Keys and values of one page and head, [64, D] each."""
    D = codes.shape[3] // PAGE
    k = decode(codes[page, h, 0]).reshape(PAGE, D) * float(scale[page, h, 0])
    v = decode(codes[page, h, 1]).reshape(4, D, 16).transpose(0, 2, 1).reshape(PAGE, D) * float(scale[page, h, 1])
    return k, v


def store(codes, page, h, part, slot, row):
    D = codes.shape[3] // PAGE
    if part == 0:
        codes[page, h, 0].reshape(PAGE, D)[slot] = row
    else:
        codes[page, h, 1].reshape(4, D, 16)[slot // 16, :, slot % 16] = row


def cached(codes, scale, table, length, h):
    """Keys and values of a sequence, [length, D] each, and whether each token's page exists."""
    D = codes.shape[3] // PAGE
    k, v, there = np.zeros((length, D)), np.zeros((length, D)), np.ones(length, bool)
    for w in range(-(-length // PAGE)):
        at = slice(w * PAGE, min(length, (w + 1) * PAGE))
        page = int(table[w])
        if not 0 <= page < codes.shape[0]:
            there[at] = False
            continue
        pk, pv = page_values(codes, scale, page, h)
        k[at], v[at] = pk[:at.stop - at.start], pv[:at.stop - at.start]
    return k, v, there


def append(codes, scale, tables, lengths, k, v, index=None, count=None):
    """New codes, scales and lengths.  k, v [B, n, heads, D]."""
    codes, scale = codes.copy(), scale.copy()
    B, n, H, D = k.shape
    out = []
    for b in range(B):
        m = (n if index is None else len(index[b])) if count is None else int(count[b])
        rows = list(range(m)) if index is None else [int(i) for i in index[b][:m]]
        start = int(lengths[b])
        end = min(start + m, len(tables[b]) * PAGE)
        out.append(end)
        for w in range(start // PAGE, -(-end // PAGE)):
            page = int(tables[b][w])
            if not 0 <= page < codes.shape[0]:
                continue
            lo, hi = max(start, w * PAGE), min(end, (w + 1) * PAGE)
            for h in range(H):
                old = page_values(codes, scale, page, h)
                for part, x in ((0, k), (1, v)):
                    new = [x[b, rows[t - start], h].astype(np.float64) if 0 <= rows[t - start] < n else np.zeros(D) for t in range(lo, hi)]
                    fine = [np.abs(r[np.isfinite(r)]).max(initial=0.0) for r in new]
                    to = least_scale(max(fine))
                    before = lo - w * PAGE
                    if before:
                        to = max(to, float(scale[page, h, part]))
                    if to != scale[page, h, part]:
                        for slot in range(before):
                            store(codes, page, h, part, slot, encode(old[part][slot] / to))
                    scale[page, h, part] = to
                    for t, r in zip(range(lo, hi), new):
                        store(codes, page, h, part, t - w * PAGE, encode(r / to))
    return codes, scale, np.array(out)


def sees(mask, n, there, b):
    """[n, n] booleans: token i sees new token j."""
    if mask is None:
        m = np.tril(np.ones((n, n), bool))
    else:
        words = mask[b if mask.shape[0] > 1 else 0].astype(np.uint32)
        m = np.stack([words[:, j // 32] >> np.uint32(j % 32) & np.uint32(1) for j in range(n)], 1) != 0
    m = m.copy()
    m[there:] = False
    m[:, there:] = False
    return m


def attend(q, codes, scale, tables, lengths, k=None, v=None, mask=None, count=None, softmax_scale=None):
    """out, lse, and for each row sum_j p_j |v_j| and max_j scale * sum_d |q_d k_jd|, which bound what rounding can do."""
    B, n, Hq, D = q.shape
    H = codes.shape[1]
    c = D ** -0.5 if softmax_scale is None else softmax_scale
    out, lse = np.zeros(q.shape), np.full((B, n, Hq), -np.inf)
    size, reach = np.zeros(q.shape), np.zeros((B, n, Hq))
    for b in range(B):
        there = n if count is None else int(count[b])
        seen = sees(mask, n, there, b) if k is not None else None
        for hq in range(Hq):
            h = hq // (Hq // H)
            ck, cv, cached_there = cached(codes, scale, tables[b], int(lengths[b]), h)
            ck, cv = ck[cached_there], cv[cached_there]
            for i in range(there):
                kk, vv = ck, cv
                if k is not None:
                    kk = np.concatenate([ck, k[b, :, h][seen[i]].astype(np.float64)])
                    vv = np.concatenate([cv, v[b, :, h][seen[i]].astype(np.float64)])
                if not len(kk):
                    continue
                x = q[b, i, hq].astype(np.float64)
                s = kk @ x * c
                m = s.max()
                p = np.exp(s - m)
                total = p.sum()
                lse[b, i, hq] = m + np.log(total)
                out[b, i, hq] = (p / total) @ vv
                size[b, i, hq] = (p / total) @ np.abs(vv)
                reach[b, i, hq] = (np.abs(kk) @ np.abs(x)).max() * c
    return out, lse, size, reach


def weigh(q, lse, codes, scale, tables, lengths, weight, decay, count=None, softmax_scale=None):
    B, n, Hq, D = q.shape
    H = codes.shape[1]
    c = D ** -0.5 if softmax_scale is None else softmax_scale
    out, reach = np.zeros(weight.shape), np.zeros(weight.shape)
    for b in range(B):
        L, there = int(lengths[b]), n if count is None else int(count[b])
        for h in range(H):
            k, _, ok = cached(codes, scale, tables[b], L, h)
            got = np.zeros(L)
            for hq in range(h * (Hq // H), (h + 1) * (Hq // H)):
                for i in range(there):
                    if np.isneginf(lse[b, i, hq]):
                        continue
                    x = q[b, i, hq].astype(np.float64)
                    got += np.where(ok, np.exp(k @ x * c - lse[b, i, hq]), 0)
                    reach[b, h, :L] = np.maximum(reach[b, h, :L], np.abs(k) @ np.abs(x) * c + abs(lse[b, i, hq]))
            out[b, h, :L] = decay * weight[b, h, :L].astype(np.float64) + got
    return out, reach


def evict(codes, scale, tables, lengths, weight, keep, recent, new_tables):
    codes, scale = codes.copy(), scale.copy()
    B, H = weight.shape[:2]
    W = len(new_tables[0])
    kept, out_weight, out_length = np.full((B, H, keep), -1), np.zeros((B, H, W * PAGE), np.float32), []
    for b in range(B):
        L = int(lengths[b])
        m = min(L, keep)
        r = min(recent, m)
        out_length.append(m)
        for h in range(H):
            w = weight[b, h, :L - r].astype(np.float64)
            w = np.where(np.isnan(w), -np.inf, w)
            # (NaN below -inf: the first key; a stable order leaves ties to the first)
            order = np.lexsort((np.arange(L - r), -w, np.isnan(weight[b, h, :L - r])))
            mine = np.sort(np.concatenate([order[:m - r], np.arange(L - r, L)]))
            kept[b, h, :m] = mine
            out_weight[b, h, :m] = weight[b, h, mine]
            for w0 in range(0, m, PAGE):
                page = int(new_tables[b][w0 // PAGE])
                if not 0 <= page < codes.shape[0]:
                    continue
                tokens = mine[w0:w0 + PAGE]
                source = [int(tables[b][t // PAGE]) for t in tokens]
                real = [s for s in source if 0 <= s < codes.shape[0]]
                for part in (0, 1):
                    to = max([float(scale[s, h, part]) for s in real], default=2.0 ** MIN_EXP)
                    scale[page, h, part] = to
                    for slot, (t, s) in enumerate(zip(tokens, source)):
                        row = np.zeros(codes.shape[3] // PAGE)
                        if 0 <= s < codes.shape[0]:
                            row = page_values(codes, scale, s, h)[part][t % PAGE]
                        store(codes, page, h, part, slot, encode(row / to))
    return codes, scale, np.array(out_length), kept, out_weight
