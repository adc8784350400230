"""Seeded random sizes of the calls around attention and verification against the oracle."""
import random

import pytest
import torch

from . import test_gpu_adapt as A
from . import test_gpu_logprob as L
from . import test_gpu_rotate as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", range(24))
def test_adapt(seed):
    r = random.Random(100 + seed)
    dtype = r.choice(["f32", "bf16", "f16"])
    rank, adapters = 16 * r.choice([1, 1, 2, 3, 4, 5, 8, 16]), r.randint(1, 5)
    c = A.make(B=r.randint(1, 9), n=r.choice([1, 2, r.randint(3, 16), r.randint(17, 150)]), K=8 * r.randint(1, 150), N=r.randint(1, 900), R=rank, dtype=dtype, adapters=adapters,
               ragged=r.random() < 0.5, ranks=[r.randint(0, rank) for _ in range(adapters)] if r.random() < 0.6 else None, seed=seed, strided=r.random() < 0.5)
    A.check(c, A.call(c))


@pytest.mark.parametrize("seed", range(16))
def test_rotate_and_its_gradients(seed):
    r = random.Random(200 + seed)
    D = r.choice([64, 128, 256])
    eps = r.choice([None, 1e-6, 1e-3])
    c = R.make(B=r.randint(1, 6), n=r.choice([1, r.randint(2, 40), r.randint(41, 500)]), hq=r.randint(1, 9), h=r.randint(1, 4), D=D, rotary=16 * r.randint(0, D // 16),
               dtype=r.choice(["f32", "bf16", "f16"]), axes=r.randint(1, 4), adjacent=r.random() < 0.5, eps=eps, shared=r.random() < 0.5, far=r.choice([0, 9, 100000]),
               ragged=r.random() < 0.5, seed=seed)
    if c["freq"] is None:
        c["axis"] = None
    R.check(c, R.call(c))
    R.check_backward(c, R.backward(c))


@pytest.mark.parametrize("seed", range(24))
def test_logprob_and_its_gradient(seed):
    r = random.Random(300 + seed)
    V = r.choice([r.randint(1, 40), r.randint(41, 3000), r.randint(3001, 90000)])
    n = r.choice([1, r.randint(2, 9), r.randint(10, 40) if V < 3000 else 3])
    m = r.randint(1, n) if r.random() < 0.4 else None
    c = L.make(B=r.randint(1, 4), n=n, V=V, dtype=r.choice(["f32", "bf16", "f16"]), T=r.choice([1.0, 0.6, 1.7]), top=r.choice([0, 0, 1, r.randint(2, 32)]), m=m, ragged=r.random() < 0.5,
               pad=r.randint(0, 9), offset=r.randint(0, 9), kind=r.choice(["plain", "plain", "few values", "masked", "rising"]) if V > 2 else "plain", seed=seed)
    fwd = L.call(c)
    L.check(c, fwd)
    if m is None:
        g = L.gradients(c, which=r.sample(["grad_logp", "grad_entropy", "grad_lse", "grad_top"], r.randint(1, 4)))
        L.check_back(c, fwd, g, L.back(c, fwd, g)["logits"])
