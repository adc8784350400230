"""Calls of more workgroups than one launch takes, and of sizes next to 2^31: refused on the host."""
import pytest

from paper_2512_16273_amd import tslt

FAKE = 0x10000


@pytest.fixture(scope="module")
def lib():
    return tslt.load()


def adapt(lib, B, n, R=16, K=64, N=64, dt=1):
    rows = tslt._Rows(FAKE, max(n, 1) * 64, 64, 0)
    return lib.tslt_adapt(rows, K, rows, rows, N, dt, B, n, FAKE, FAKE, 4, R, FAKE, None, None, None, None, FAKE, 1 << 62, None)


@pytest.mark.parametrize("n", [(1 << 31) - 1, (1 << 31) - 15, (1 << 31) - 31, (1 << 31) - 62, (1 << 31) - 64, 1 << 30])
@pytest.mark.parametrize("dt", [0, 1])
def test_adapt_of_very_long_sequences(lib, n, dt):
    assert adapt(lib, 1, n, dt=dt) == -2 and "workgroups" in lib.tslt_last_error().decode()
    assert lib.tslt_adapt_workspace_bytes(1, n, 64, 64, 16) == (n * 16 * 4 + 255) // 256 * 256


def test_adapt_of_many_sequences(lib):
    """Workgroups of 64 ranks each: 2^22 sequences of rank 256 are 2^24 of them."""
    for B, R in ((1 << 22, 256), (1 << 23, 128), (1 << 24, 64)):
        assert adapt(lib, B, 1, R=R) == -2 and "workgroups" in lib.tslt_last_error().decode()
