"""The calls around attention and verification look at the device of every tensor that they hand over, not of the first one alone."""
import pytest
import torch

from paper_2512_16273_amd import tslt


class Held:
    """What the binding asks of a tensor, of one that lives on a GPU of the given number."""
    is_cuda = True

    def __init__(self, *shape, dtype=torch.float32, on=0):
        self.shape, self.dtype, self.device, self.on = torch.Size(shape), dtype, torch.device("cuda", on), on
        self.meta = torch.empty(shape, dtype=dtype, device="meta")

    def elsewhere(self):
        return Held(*self.shape, dtype=self.dtype, on=1)

    def stride(self, i=None):
        return self.meta.stride() if i is None else self.meta.stride(i)

    def is_contiguous(self):
        return True

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.meta.numel()

    def data_ptr(self):
        return 0x10000


def ints(*shape):
    return Held(*shape, dtype=torch.int32)


def of_bytes(n):
    return Held(n, dtype=torch.uint8)


B, N, HQ, H, D, V, K, W, TOP = 2, 3, 4, 2, 64, 1000, 64, 40, 5
ROTATION = dict(position=ints(B, N, 2), freq=Held(32), axis=ints(32), base=ints(B), q_weight=Held(D), k_weight=Held(D), eps=1e-6, count=ints(B))
LOGITS = dict(logits=Held(B, N, V), temperature=1.0, tokens=ints(B, N), count=ints(B))
CALLS = {
    "rotate": (dict(q=Held(B, N, HQ, D), k=Held(B, N, H, D), **ROTATION), dict(q=Held(B, N, HQ, D), k=Held(B, N, H, D), status=ints(B))),
    "rotate_backward": (dict(grad_q=Held(B, N, HQ, D), grad_k=Held(B, N, H, D), q=Held(B, N, HQ, D), k=Held(B, N, H, D), **ROTATION, workspace=of_bytes(1 << 20)),
                        dict(q=Held(B, N, HQ, D), k=Held(B, N, H, D), q_weight=Held(D), k_weight=Held(D), status=ints(B))),
    "logprob": (dict(**LOGITS, index=ints(B, N), top=TOP, workspace=of_bytes(1 << 20)),
                dict(logp=Held(B, N), entropy=Held(B, N), lse=Held(B, N), status=ints(B, N), top_idx=ints(B, N, TOP), top_logp=Held(B, N, TOP))),
    "logprob_backward": (dict(**LOGITS, lse=Held(B, N), entropy=Held(B, N), grad_logp=Held(B, N), grad_entropy=Held(B, N), grad_lse=Held(B, N), top_idx=ints(B, N, TOP),
                              grad_top=Held(B, N, TOP)), dict(logits=Held(B, N, V))),
    "adapt": (dict(x=Held(B, N, K), base=Held(B, N, W), a=Held(3, 16, K), b=Held(3, W, 16), adapter=ints(B), scale=Held(3), rank=ints(3), count=ints(B), workspace=of_bytes(1 << 20)),
              dict(out=Held(B, N, W), status=ints(B))),
}


class Library:
    """Takes every call and launches nothing."""
    def __init__(self):
        self.calls = 0

    def __getattr__(self, name):
        def call(*a):
            self.calls += 1
            return 0
        return call


@pytest.mark.parametrize("name", CALLS)
def test_every_tensor_lives_on_the_current_device(name, monkeypatch):
    library = Library()
    monkeypatch.setattr(tslt, "load", lambda: library)
    monkeypatch.setattr(tslt, "_fast", None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    monkeypatch.setattr(torch.autograd.graph, "increment_version", lambda tensors: None)
    given, made = CALLS[name]
    call = getattr(tslt, name)
    call(**given, out=dict(made))
    assert library.calls == 1
    for which in [k for k, v in given.items() if isinstance(v, Held)]:
        with pytest.raises(tslt.TsltError, match="cuda:1.*current device is cuda:0"):
            call(**{**given, which: given[which].elsewhere()}, out=dict(made))
    for which in made:
        with pytest.raises(tslt.TsltError, match="out .*cuda:1"):
            call(**given, out={**made, which: made[which].elsewhere()})
    assert library.calls == 1
