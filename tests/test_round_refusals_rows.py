"""Results whose rows lie on each other, wholly or in part, are refused before anything is launched."""
import pytest

from paper_2512_16273_amd import tslt

FAKE = 0x10000


@pytest.fixture(scope="module")
def lib():
    return tslt.load()


def refused(lib, code):
    return code == -1 and "each other" in lib.tslt_last_error().decode()


def rotation():
    return tslt._Rotation(None, 0, None, FAKE, None, 1, 64, 0, -1.0, None, None)


# sequence, token, head; 2 x 4 tokens of 3 heads of 64 in all
OVER = [(800, 200, 56), (800, 184, 64), (760, 192, 64), (-760, 192, 64), (800, -184, 64), (64, 128, 480), (64, 120, 512), (512, 128, 192), (8, 192, 64), (768, 8, 64), (768, 192, 8)]
APART = [(768, 192, 64), (-768, 192, -64), (64, 128, 512), (192, 384, 64), (4096, 64, 1024)]


def rows(at, strides):
    return tslt._Rows(at, *strides)


@pytest.mark.parametrize("which", ["q", "k"])
def test_rotate_and_its_gradients(lib, which):
    fine = rows(FAKE, APART[0])

    def both(strides):
        made = {"q": rows(FAKE * 3, APART[0]), "k": rows(FAKE * 4, APART[0]), which: rows(FAKE * 5, strides)}
        yield lib.tslt_rotate(fine, rows(FAKE * 2, APART[0]), 1, 2, 4, 3, 3, 64, rotation(), None, made["q"], made["k"], None, None)
        yield lib.tslt_rotate_backward(fine, rows(FAKE * 2, APART[0]), None, None, 1, 2, 4, 3, 3, 64, rotation(), None, made["q"], made["k"], None, None, None, None, 0, None)
    for strides in OVER:
        for code in both(strides):
            assert refused(lib, code), strides


def test_adapt(lib):
    def call(seq, token, N=100, B=2, n=3):
        return lib.tslt_adapt(rows(FAKE, (1024, 256, 0)), 64, rows(FAKE * 2, (1024, 256, 0)), rows(FAKE * 3, (seq, token, 0)), N, 1, B, n, FAKE, FAKE, 4, 16, FAKE, None, None, None,
                              None, FAKE * 4, 8, None)
    for seq, token in ((300, 99), (299, 100), (8, 100), (300, 8), (100, 199), (99, 200), (-299, 100), (300, -99)):
        assert refused(lib, call(seq, token)), (seq, token)
    for seq, token in ((300, 100), (100, 200), (-300, 100), (1 << 62, 1 << 60)):
        assert call(seq, token) == -3                              # (the workspace is what is refused then)
    assert call(0, 0, B=1, n=1) == -3 and call(5, 100, B=1) == -3 and call(100, 5, n=1) == -3
    assert refused(lib, call(1 << 62, 1 << 62))


def test_logprob_backward(lib):
    def call(seq, row, B=2, n=3, V=1000):
        return lib.tslt_logprob_backward(FAKE, 1, B, n, V, n * V, V, 1.0, None, None, FAKE, None, None, 0, None, None, None, None, FAKE * 2, seq, row, None)
    for seq, row in ((8, 1000), (2999, 1000), (3000, 999), (1000, 1999), (999, 2000), (0, 1000), (3000, 0), (-2999, 1000)):
        assert refused(lib, call(seq, row)), (seq, row)


def test_rows_apart_are_not_refused():
    """The same rule, by counting."""
    for strides in OVER + APART:
        places = sorted(b * strides[0] + i * strides[1] + h * strides[2] for b in range(2) for i in range(4) for h in range(3))
        assert (min(b - a for a, b in zip(places, places[1:])) >= 64) == (strides in APART), strides
