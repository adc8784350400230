"""What the calls around the 8-bit cache refuse, found on the host before anything is launched."""
import ctypes

import pytest
import torch

from paper_2512_16273_amd import tslt

FAKE = 0x10000


@pytest.fixture(scope="module")
def lib():
    return tslt.load()


def cache(codes=FAKE, scales=FAKE, n_pages=8, heads=2, head_dim=64):
    return tslt._Cache(codes, scales, n_pages, heads, head_dim)


def rows(data=FAKE, seq=1024, token=256, head=64):
    return tslt._Rows(data, seq, token, head)


def message(lib):
    return lib.tslt_last_error().decode()


def common(lib, call, dt_arg=True):
    """Refusals that every call shares; `call` takes the cache, page table and sequences to change."""
    assert call(c=cache(head_dim=80)) == -2 and "head_dim" in message(lib)
    assert call(c=cache(heads=0)) == -1 and call(c=cache(n_pages=0)) == -1
    assert call(c=cache(codes=None)) == -1 and call(c=cache(scales=None)) == -1
    assert call(c=cache(codes=FAKE + 8)) == -1 and "16 bytes" in message(lib)
    assert call(c=None) == -1
    assert call(width=0) == -1 and call(width=1 << 40) == -2
    assert call(pages=None) == -1 and call(length=None) == -1
    assert call(B=-1) == -1
    assert call(B=0) == 0                                        # no sequences: nothing to do


def test_append(lib):
    def call(c=cache(), pages=FAKE, width=4, length=FAKE, B=3, n=2, k=rows(), v=rows(), dt=1, index=None, most=0, out=FAKE + 64):
        return lib.tslt_cache_append(c, pages, width, length, B, n, k, v, dt, index, most, None, out, None, None)
    common(lib, call)
    assert call(n=0) == -1 and call(dt=5) == -1 and call(index=FAKE, most=0) == -1
    assert call(k=None) == -1 and call(v=rows(data=None)) == -1
    assert call(k=rows(data=FAKE + 2)) == -1 and call(v=rows(token=100)) == -1 and "16 bytes" in message(lib)
    assert call(out=None) == -1 and call(out=FAKE) == -1 and "out_length" in message(lib)
    assert call(B=1 << 40) == -2


def test_attend(lib):
    def call(c=cache(), pages=FAKE, width=4, length=FAKE, B=3, n=2, heads_q=4, q=rows(), k=rows(), v=rows(), dt=1, mask=None, mask_seq=0,
             scale=0.125, out=FAKE, lse=FAKE, ws=FAKE, ws_bytes=1 << 40):
        return lib.tslt_cache_attend(c, pages, width, length, B, n, heads_q, q, k, v, dt, mask, mask_seq, None, scale, out, lse, None, ws, ws_bytes, None)
    common(lib, call)
    assert call(n=0) == -1 and call(dt=3) == -1 and call(heads_q=3) == -1 and call(heads_q=1) == -1
    assert call(scale=0.0) == -1 and call(scale=float("nan")) == -1 and call(scale=float("inf")) == -1
    assert call(q=None) == -1 and call(k=None) == -1 and "together" in message(lib)
    assert call(q=rows(head=60)) == -1 and call(v=rows(seq=4)) == -1
    assert call(out=None) == -1 and call(lse=None) == -1 and call(out=FAKE + 8) == -1
    assert call(mask=FAKE, mask_seq=-1) == -1
    need = lib.tslt_cache_attend_workspace_bytes(3, 2, 4, 2, 64, 4000)
    assert need > 0
    assert call(width=4000, ws_bytes=need - 1) == -3 and "workspace" in message(lib)
    assert call(width=4000, ws=None) == -3 and call(width=4000, ws=FAKE + 64) == -3
    assert lib.tslt_cache_attend_workspace_bytes(3, 2, 4, 2, 64, 1) == 0
    assert lib.tslt_cache_attend_workspace_bytes(0, 2, 4, 2, 64, 100) == 0 and lib.tslt_cache_attend_workspace_bytes(3, 2, 5, 2, 64, 100) == 0


def test_weigh(lib):
    def call(c=cache(), pages=FAKE, width=4, length=FAKE, B=3, n=2, heads_q=4, q=rows(), dt=1, lse=FAKE, scale=0.125, weight=FAKE, decay=1.0, out=FAKE):
        return lib.tslt_cache_weigh(c, pages, width, length, B, n, heads_q, q, dt, lse, None, scale, weight, decay, out, None, None)
    common(lib, call)
    assert call(n=0) == -1 and call(dt=-1) == -1 and call(heads_q=5) == -1 and call(scale=-1.0) == -1 and call(decay=float("inf")) == -1
    assert call(q=None) == -1 and call(lse=None) == -1 and call(weight=None) == -1 and call(out=None) == -1


def test_evict(lib):
    def call(c=cache(), pages=FAKE, width=4, length=FAKE, B=3, weight=FAKE, keep=100, recent=5, new_pages=FAKE, new_width=2, out_length=FAKE + 64,
             kept=FAKE, out=FAKE + 64):
        return lib.tslt_cache_evict(c, pages, width, length, B, weight, keep, recent, new_pages, new_width, out_length, kept, out, None, None)
    common(lib, call)
    assert call(keep=0) == -1 and call(recent=-1) == -1 and call(new_width=1) == -1 and "do not hold" in message(lib)
    assert call(weight=None) == -1 and call(new_pages=None) == -1 and call(kept=None) == -1
    assert call(out_length=FAKE) == -1 and call(out=FAKE) == -1


def test_python_binding_refuses_what_is_not_on_a_gpu_or_does_not_fit():
    c = tslt.cache_create(4, 2, 64, device="cpu")
    pages, length = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    x = torch.zeros(1, 1, 2, 64)
    with pytest.raises(tslt.TsltError, match="GPU"):
        tslt.cache_append(c, pages, length, x, x)
    with pytest.raises(tslt.TsltError, match="GPU"):
        tslt.cache_attend(x, c, pages, length)
    with pytest.raises(tslt.TsltError, match="dense"):
        tslt._rows_of(_Fake(torch.zeros(1, 1, 64, 2).transpose(2, 3)), "k", (1, 1, 2, 64), torch.float32)
    with pytest.raises(tslt.TsltError, match="must be"):
        tslt._rows_of(_Fake(x), "k", (1, 2, 2, 64), torch.float32)


@pytest.mark.parametrize("keep,recent", [((1 << 32) + 5, 0), (5, 1 << 32), (1 << 31, 5), (5, -(1 << 32)), (-(1 << 32) + 5, 0)])
def test_numbers_of_an_eviction_that_do_not_fit_are_refused_and_not_cut(keep, recent):
    c = tslt.cache_create(4, 2, 64, device="cpu")
    pages, length = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(tslt.TsltError, match="32 bits"):
        tslt.cache_evict(c, pages, length, torch.zeros(1, 2, 128), keep, recent, pages)


class _Fake:
    """A tensor that says it lies on a GPU, for checks that come before anything is done with it."""
    is_cuda = True

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)


@pytest.mark.parametrize("expansion", [(), (1,), (2, 2, 2), (4, 4, 4, 4), (33,), (3, 1, 2)])
def test_tree_mask_is_ancestors_and_self(expansion):
    parents, layer = [-1], [0]
    for k in expansion:
        layer = [i for i in layer for _ in range(k)]
        parents += layer
        layer = list(range(len(parents) - len(layer), len(parents)))
    m = tslt.tree_mask(expansion, device="cpu")
    n = len(parents)
    assert m.dtype == torch.int32 and tuple(m.shape) == (1, n, (n + 31) // 32)
    for i in range(n):
        want, j = set(), i
        while j >= 0:
            want.add(j)
            j = parents[j]
        assert {j for j in range(32 * m.shape[2]) if int(m[0, i, j // 32]) >> (j % 32) & 1} == want
