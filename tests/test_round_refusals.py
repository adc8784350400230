"""What the calls around attention and verification refuse, found on the host before anything is launched."""
import pytest
import torch

from paper_2512_16273_amd import tslt

FAKE = 0x10000
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    return tslt.load()


def rows(data=FAKE, seq=1024, token=256, head=64):
    return tslt._Rows(data, seq, token, head)


def how(position=FAKE, seq=8, base=None, freq=FAKE, axis=None, axes=1, rotary=64, adjacent=0, eps=-1.0, qw=None, kw=None):
    return tslt._Rotation(position, seq, base, freq, axis, axes, rotary, adjacent, eps, qw, kw)


def message(lib):
    return lib.tslt_last_error().decode()


def rotation_refusals(lib, call):
    assert call(D=80) == -2 and "head_dim" in message(lib)
    assert call(dt=7) == -1 and call(B=-1) == -1 and call(n=0) == -1 and call(hq=0) == -1 and call(h=0) == -1
    assert call(B=1 << 31) == -2 and call(hq=1 << 22) == -2
    assert call(r=None) == -1
    for rotary in (-16, 8, 72, 80):
        assert call(r=how(rotary=rotary)) == -1 and "rotary" in message(lib)
    assert call(r=how(axes=0)) == -1 and call(r=how(axes=5)) == -1 and "axes" in message(lib)
    assert call(r=how(freq=None)) == -1 and call(r=how(seq=-1)) == -1
    assert call(r=how(eps=NAN)) == -1 and call(r=how(eps=INF)) == -1
    assert call(r=how(qw=FAKE)) == -1 and "norm" in message(lib)
    assert call(q=None) == -1 and call(q=rows(data=FAKE + 2)) == -1 and call(q=rows(token=100)) == -1 and "16 bytes" in message(lib)
    assert call(oq=rows(head=3)) == -1 and call(ok=None) == -1 and "together" in message(lib)
    assert call(oq=rows(seq=2048)) == -1 and "in place" in message(lib)
    for lie in (dict(seq=0), dict(token=0), dict(head=0)):
        assert call(oq=rows(FAKE * 2, **lie)) == -1 and call(ok=rows(FAKE * 3, **lie)) == -1 and "each other" in message(lib)


def test_rotate(lib):
    def call(q=rows(), k=rows(), dt=1, B=2, n=4, hq=4, h=2, D=64, r=how(), oq=rows(FAKE * 2), ok=rows(FAKE * 3)):
        if oq is not None and oq.seq_stride == 2048:
            oq = rows(seq=2048)
        return lib.tslt_rotate(q, k, dt, B, n, hq, h, D, r, None, oq, ok, None, None)
    rotation_refusals(lib, call)
    assert call(k=None) == -1 and "together" in message(lib)
    assert call(B=(1 << 26) + 4, n=1) == -2 and "workgroups" in message(lib)       # four tokens to each, 2^32 threads
    assert call(B=0) == 0


def test_rotate_backward(lib):
    def call(q=rows(), k=rows(), dt=1, B=2, n=4, hq=4, h=2, D=64, r=how(), oq=rows(FAKE * 2), ok=rows(FAKE * 3), x=rows(FAKE * 4), y=rows(FAKE * 5), dq=None, dk=None,
             ws=None, ws_bytes=0):
        return lib.tslt_rotate_backward(q, k, x, y, dt, B, n, hq, h, D, r, None, oq, ok, dq, dk, None, ws, ws_bytes, None)
    rotation_refusals(lib, call)
    normed = how(eps=1e-6)
    assert call(r=normed, x=None) == -1 and call(r=normed, y=rows(data=None)) == -1
    assert call(dq=FAKE) == -1 and "norm" in message(lib)
    assert call(r=normed, dk=FAKE, k=None, ok=None) == -1 and "keys" in message(lib)
    need = lib.tslt_rotate_backward_workspace_bytes(2, 4, 4, 2, 64)
    assert need > 0
    for ws, size in ((None, need), (FAKE + 16, need), (FAKE, need - 1)):
        assert call(r=normed, dq=FAKE, ws=ws, ws_bytes=size) == -3
    assert lib.tslt_rotate_backward_workspace_bytes(2, 4, 4, 2, 80) == 0 and lib.tslt_rotate_backward_workspace_bytes(1 << 31, 4, 4, 2, 64) == 0


def test_rotate_of_tensors():
    cpu = torch.zeros(1, 2, 2, 64)
    with pytest.raises(tslt.TsltError, match="GPU"):
        tslt.rotate(cpu, None, None, None)
    with pytest.raises(tslt.TsltError, match="GPU"):
        tslt.rotate_backward(cpu, None, cpu, None, None, None)


def test_logprob(lib):
    def call(z=FAKE, dt=1, B=2, n=3, V=1000, T=1.0, index=None, m=3, tokens=None, top=0, idx=None, logp=None, ws=FAKE * 2, ws_bytes=1 << 30):
        return lib.tslt_logprob(z, dt, B, n, V, n * V, V, T, index, m, None, tokens, top, None, None, None, idx, logp, None, ws, ws_bytes, None)
    assert call(dt=9) == -1 and call(B=-1) == -1 and call(n=0) == -1 and call(V=0) == -1 and call(z=None) == -1
    assert call(V=1 << 31) == -2 and call(dt=0, V=1 << 30) == -2 and call(B=1 << 31) == -2 and call(index=FAKE, m=1 << 30, B=4) == -2
    for rows_, V in ((1 << 26, 1000), (1 << 24, 17000)):                           # a wave, four waves to each
        assert call(B=rows_, n=1, m=1, V=V) == -2 and "workgroups" in message(lib)
    for T in (0.0, -1.0, NAN, INF, 1e-39, 5e-39, 9e-39):
        assert call(T=T) == -1 and "temperature" in message(lib)
    assert call(m=2) == -1 and call(index=FAKE, m=0) == -1 and "index" in message(lib)
    assert call(top=33) == -2 and call(top=-1) == -2 and call(top=4) == -1 and call(top=4, idx=FAKE) == -1
    assert call(z=FAKE + 1) == -1 and "aligned" in message(lib)
    need = lib.tslt_logprob_workspace_bytes(2, 3, 100000, 0)
    assert need > 0
    for ws, size in ((None, need), (FAKE + 16, need), (FAKE, 64)):
        assert call(V=100000, ws=ws, ws_bytes=size) == -3 and "workspace" in message(lib)
    assert call(B=0) == 0
    assert lib.tslt_logprob_workspace_bytes(0, 3, 1000, 0) == 0 and lib.tslt_logprob_workspace_bytes(1 << 31, 3, 1000, 0) == 0
    assert lib.tslt_logprob_workspace_bytes(2, 3, 1000, 33) == 0


def test_logprob_backward(lib):
    def call(z=FAKE, dt=1, B=2, n=3, V=1000, T=1.0, tokens=FAKE, lse=FAKE, entropy=FAKE, idx=FAKE, top=2, g=FAKE, gh=FAKE, gt=FAKE, out=FAKE * 2, stride=1000):
        return lib.tslt_logprob_backward(z, dt, B, n, V, n * V, V, T, None, tokens, lse, entropy, idx, top, g, gh, None, gt, out, n * stride, stride, None)
    assert call(dt=9) == -1 and call(B=-1) == -1 and call(n=0) == -1 and call(V=0) == -1 and call(z=None) == -1 and call(out=None) == -1 and call(lse=None) == -1
    assert call(V=1 << 31) == -2 and call(B=1 << 31) == -2 and call(T=0.0) == -1 and call(top=33) == -2
    assert call(B=1 << 24, n=1) == -2 and "workgroups" in message(lib)
    assert call(tokens=None) == -1 and "tokens" in message(lib)
    assert call(entropy=None) == -1 and "entropy" in message(lib)
    assert call(idx=None) == -1 and call(top=0) == -1 and "top_idx" in message(lib)
    assert call(z=FAKE + 1) == -1 and call(out=FAKE + 1) == -1
    assert call(out=FAKE, stride=1008) == -1 and "written over" in message(lib)
    assert call(stride=0) == -1 and call(stride=999) == -1 and "each other" in message(lib)
    assert call(B=0) == 0


def test_logprob_of_tensors():
    z = torch.zeros(1, 2, 8)
    with pytest.raises(tslt.TsltError, match="GPU"):
        tslt.logprob(z, 1.0)
    with pytest.raises(tslt.TsltError, match="GPU"):
        tslt.logprob_backward(z, 1.0, None, z[..., 0])


def test_adapt(lib):
    def call(x=rows(), K=64, base=rows(FAKE * 2), out=rows(FAKE * 3), N=100, dt=1, B=2, n=3, a=FAKE, b=FAKE, adapters=4, R=16, adapter=FAKE, ws=FAKE * 4, ws_bytes=1 << 30):
        return lib.tslt_adapt(x, K, base, out, N, dt, B, n, a, b, adapters, R, adapter, None, None, None, None, ws, ws_bytes, None)
    assert call(dt=4) == -1 and call(B=-1) == -1 and call(n=0) == -1 and call(K=0) == -1 and call(N=0) == -1 and call(adapters=0) == -1
    for R in (0, 8, 24, 272, -16):
        assert call(R=R) == -2 and "R must be" in message(lib)
    assert call(K=60) == -2 and call(K=6, dt=0) == -2 and call(K=4) == -2 and "16 bytes" in message(lib)
    assert call(B=1 << 31) == -2 and call(adapters=1 << 31) == -2 and call(N=1 << 29) == -2 and call(K=1 << 29) == -2
    assert call(x=None) == -1 and call(base=rows(data=None)) == -1 and call(out=rows(FAKE * 3 + 1)) == -1 and call(x=rows(token=12)) == -1
    assert call(a=None) == -1 and call(b=None) == -1 and call(adapter=None) == -1 and call(a=FAKE + 8) == -1 and call(b=FAKE + 2) == -1
    assert call(out=rows(FAKE * 2, token=513)) == -1 and "in place" in message(lib)
    assert call(out=rows(FAKE * 3, seq=0)) == -1 and call(out=rows(FAKE * 3, token=0)) == -1 and "each other" in message(lib)
    need = lib.tslt_adapt_workspace_bytes(2, 3, 64, 100, 16)
    assert need > 0
    for ws, size in ((None, need), (FAKE + 16, need), (FAKE, need - 1)):
        assert call(ws=ws, ws_bytes=size) == -3 and "workspace" in message(lib)
    assert call(B=1 << 24, n=1, ws_bytes=1 << 40) == -2 and "workgroups" in message(lib)
    assert call(B=0) == 0
    for bad in ((0, 3, 64, 100, 16), (2, 3, 64, 100, 24), (1 << 31, 3, 64, 100, 16)):
        assert lib.tslt_adapt_workspace_bytes(*bad) == 0


def test_adapt_of_tensors():
    x = torch.zeros(1, 2, 64)
    with pytest.raises(tslt.TsltError, match="GPU"):
        tslt.adapt(x, x, x, x, torch.zeros(1, dtype=torch.int32))
