"""Norms without a rotation, of one, two and four tokens a workgroup, and backwards of workgroups that go on to their next tokens."""
import pytest
import torch

from . import test_gpu_rotate as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,n,D", [(1, 5, 64), (3, 101, 128), (2, 701, 256), (5, 903, 64)], ids=str)
@pytest.mark.parametrize("eps", [1e-6, None])
def test_without_a_rotation(B, n, D, eps, dtype):
    c = R.make(B=B, n=n, hq=3, h=1, D=D, rotary=0, dtype=dtype, eps=eps, ragged=B > 1)
    out = R.call(c, out={"q": torch.full_like(c["q"], 7), "k": torch.full_like(c["k"], 7), "status": torch.ones(B, dtype=torch.int32, device=DEV)})
    assert not out["status"].any()
    R.check(c, out)
    gone = torch.arange(n, device=DEV) >= torch.tensor(R.counts(c), device=DEV)[:, None]
    assert (out["q"][gone] == 7).all() and (out["k"][gone] == 7).all()
    back = R.backward(c)
    assert not back["status"].any()
    R.check_backward(c, back)
