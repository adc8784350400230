"""The calls around attention and verification at sizes that take the kernels' other ways: many tiles of 64 tokens, workgroups that go on to a second run of channels or to their
next tokens, a wave to each of many rows whose lists are put together on the way.  (Of a GPU of 256 compute units.)"""
import pytest
import torch

from . import test_gpu_adapt as A
from . import test_gpu_logprob as L
from . import test_gpu_rotate as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = ["f32", "bf16", "f16"]

ADAPT = [dict(B=26, n=300, K=264, N=1111, R=48, ranks=[48, 17, 0], ragged=True, strided=True),      # 130 tiles of 64 tokens (fp32: 260 of 32), five runs of 256 channels, one to three workgroups to share them
         dict(B=130, n=40, K=72, N=1030, R=16, ragged=True, adapters=9),
         dict(B=26, n=270, K=520, N=1280, R=16, strided=True, ranks=[16, 3, 11]),
         dict(B=33, n=250, K=136, N=777, R=256, ranks=[256, 199, 70]),
         dict(B=300, n=9, K=264, N=1301, R=16, ragged=True, strided=True, adapters=40),             # 16 tokens: six runs, four workgroups
         dict(B=290, n=16, K=2056, N=1290, R=80, ranks=[80, 41, 16]),
         dict(B=12, n=100, K=128, N=5003, R=32, ragged=True, ranks=[32, 0, 31]),                      # 32 tokens: twenty runs, ten or sixteen workgroups
         dict(B=700, n=1, K=1032, N=1025, R=16, adapters=64)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", ADAPT, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_adapt(case, dtype):
    c = A.make(**case, dtype=dtype)
    B, n, N = case["B"], case["n"], case["N"]
    wide = torch.full((B, n, N + 3), 7.0, dtype=A.TYPES[dtype], device=DEV)
    out = A.call(c, out={"out": wide[:, :, 1:1 + N], "status": torch.ones(B, dtype=torch.int32, device=DEV)})
    assert not out["status"].any()
    A.check(c, out)
    for s, m in enumerate(A.counts(c)):
        assert (wide[s, m:] == 7).all()
    assert (wide[:, :, 0] == 7).all() and (wide[:, :, N + 1:] == 7).all()
    before = c["base"].clone()
    A.call(c, out={"out": c["base"]})
    for s, m in enumerate(A.counts(c)):
        assert torch.equal(c["base"][s, :m], wide[s, :m, 1:1 + N]) and torch.equal(c["base"][s, m:], before[s, m:])


# (more than 4096 tokens: four to a workgroup; backwards more than three workgroups a compute unit have: each goes on to others)
ROTATE = [dict(B=9, n=601, hq=4, h=2, D=64, rotary=32, far=130000, ragged=True, adjacent=True), dict(B=7, n=701, hq=3, h=1, D=128, rotary=128, axes=3, shared=True, ragged=True),
          dict(B=3, n=1503, hq=2, h=2, D=256, rotary=64, eps=None, ragged=True), dict(B=4101, n=1, hq=2, h=1, D=128, rotary=64, far=77, axes=2),
          dict(B=2, n=2050, hq=5, h=1, D=64, rotary=16), dict(B=1501, n=3, hq=1, h=1, D=256, rotary=256, axes=4, adjacent=True, ragged=True)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", ROTATE, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_rotate_and_its_gradients(case, dtype):
    c = R.make(**case, dtype=dtype)
    out = R.call(c, out={"q": torch.full_like(c["q"], 7), "k": torch.full_like(c["k"], 7), "status": torch.ones(c["B"], dtype=torch.int32, device=DEV)})
    assert not out["status"].any()
    R.check(c, out)
    gone = torch.arange(c["n"], device=DEV) >= torch.tensor(R.counts(c), device=DEV)[:, None]
    assert (out["q"][gone] == 7).all() and (out["k"][gone] == 7).all()
    back = R.backward(c)
    assert not back["status"].any()
    R.check_backward(c, back)
    again = R.backward(c, out={**{k: None if v is None else torch.empty_like(v) for k, v in back.items()}, "q": c["grad"][0], "k": c["grad"][1]})
    assert all(torch.equal(again[k], back[k]) for k in back if back[k] is not None)


def first(c, out, B, m):
    """The case and its results, cut down to the first sequences and entries."""
    c.update(logits=c["logits"][:B, :m if c["index"] is None else None], tokens=c["tokens"][:B, :m].contiguous(), B=B, m=m, count=None if c["count"] is None else c["count"][:B].clamp(max=m),
             index=None if c["index"] is None else c["index"][:B, :m])
    c["n"] = c["logits"].shape[1]
    return c, {k: v[:B, :m] for k, v in out.items()}


@pytest.mark.parametrize("kind", ["plain", "equal", "few values", "rising", "falling", "masked", "lowest", "zeros"])
@pytest.mark.parametrize("dtype,V", [("f32", 7001), ("bf16", 15001), ("f16", 16384)])
@pytest.mark.parametrize("top", [11, 32])
def test_logprob_of_many_rows_by_a_wave_each(kind, dtype, V, top):
    c = L.make(1, 2100, V, dtype, top=top, T=1.0 if kind in ("masked", "lowest") else 0.8, kind=kind, offset=0 if V == 16384 else 1)
    out = L.call(c)
    for r in range(0, 2100, 700):                                  # fewer rows, by four waves each
        some = {**c, "logits": c["logits"][:, r:r + 700], "tokens": c["tokens"][:, r:r + 700].contiguous()}
        part = L.call(some)
        assert torch.equal(part["top_idx"], out["top_idx"][:, r:r + 700]) and torch.equal(part["status"], out["status"][:, r:r + 700])
    L.check(*first(c, out, 1, 5))


@pytest.mark.parametrize("dtype,V", [("f32", 8003), ("bf16", 14007), ("f16", 12001)])
def test_logprob_of_chosen_rows_by_a_wave_each(dtype, V):
    c = L.make(300, 9, V, dtype, top=20, m=7, ragged=True, pad=5, T=1.3)
    out = {k: torch.full_like(v, 77) for k, v in L.call(c).items()}
    L.call(c, out=out)
    gone = torch.arange(7, device=DEV) >= c["count"][:, None]
    assert all((v[gone] == 77).all() for v in out.values())
    L.check(*first(c, out, 5, 7))


@pytest.mark.parametrize("dtype,T", [("f32", 1.0), ("bf16", 0.7), ("f16", 1.3)])
def test_the_gradient_of_many_rows_with_likeliest_tokens(dtype, T):
    c = L.make(40, 60, 2503, dtype, top=20, T=T, ragged=True, pad=3)
    fwd = L.call(c)
    g = L.gradients(c)
    dz = L.back(c, fwd, g)["logits"]
    few = {k: v[:4] for k, v in fwd.items()}
    c.update(logits=c["logits"][:4], tokens=c["tokens"][:4], count=c["count"][:4], B=4)
    L.check_back(c, few, {k: None if v is None else v[:4] for k, v in g.items()}, dz[:4])
