"""tslt_logprob_backward of rows whose logits lie far from 0."""
import numpy as np
import pytest
import torch

from . import test_gpu_logprob as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = L.U


@pytest.mark.parametrize("T,offset", [(0.7, 3.0e6), (1.3, 6.0e6), (1.3, -5.0e6), (37.0, 1.1e8)])
def test_what_a_reference_loses_in_32_bits(T, offset):
    """The gradient by the lse that is given, where lse * T is no number of 32 bits."""
    c = L.make(1, 4, 9001, "f32", T=T, top=6)
    c["logits"].add_(offset)
    fwd, g = L.call(c), L.gradients(c)
    L.check_back(c, fwd, g, L.back(c, fwd, g)["logits"])
