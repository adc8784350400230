"""tslt_rotate and tslt_rotate_backward against the oracle, on the GPU."""
import numpy as np
import pytest
import torch

from oracle import round_oracle as O
from paper_2512_16273_amd import tslt

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0 ** -24                                                    # half a step of fp32, relative
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}      # one subnormal step


def make(B, n, hq, h, D, rotary, dtype, axes=1, adjacent=False, eps=1e-6, shared=False, far=0, ragged=False, seed=0, spread=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = (spread * torch.randn(B, n, hq + 2 * h, D, generator=g, device=DEV)).to(TYPES[dtype])
    c = dict(q=x[:, :, :hq], k=x[:, :, hq:hq + h], dtype=dtype, adjacent=adjacent, eps=eps, D=D, B=B, n=n)
    c["position"] = torch.randint(-50, 4000, (1 if shared else B, n, axes), generator=g, device=DEV, dtype=torch.int32)
    c["base"] = far + torch.arange(B, device=DEV, dtype=torch.int32) if far else None
    c["freq"] = (10000.0 ** (-torch.arange(rotary // 2, device=DEV) * 2.0 / max(rotary, 1))).float() if rotary else None
    c["axis"] = torch.randint(0, axes, (rotary // 2,), generator=g, device=DEV, dtype=torch.int32) if axes > 1 else None
    w = 1 + 0.3 * torch.randn(2, D, generator=g, device=DEV)
    c["w"] = (w[0], w[1]) if eps is not None else (None, None)
    c["count"] = torch.tensor([b * 3 % (n + 1) for b in range(B)], device=DEV, dtype=torch.int32) if ragged else None
    c["grad"] = [torch.randn(t.shape, generator=g, device=DEV).to(t.dtype) for t in (c["q"], c["k"])]
    return c


def host(t):
    return None if t is None else t.detach().float().cpu().numpy().astype(np.float64) if t.is_floating_point() else t.cpu().numpy()


def turns(c):
    freq = np.zeros(0) if c["freq"] is None else host(c["freq"])
    at = O.token_positions(c["B"], c["n"], freq.size, host(c["position"]), host(c["base"]), host(c["axis"]))
    cos, sin = O.turns(at, freq)
    # fp64's product with the frequency, by 1 / 2 pi, and its rounding to a turn: 4 * 2^-53 of the angle
    return cos, sin, (np.abs(at).max() * np.abs(freq).max() * 2.0 ** -51 if freq.size else 0.0)


def counts(c):
    return [c["n"]] * c["B"] if c["count"] is None else [min(max(int(x), 0), c["n"]) for x in c["count"]]


def call(c, out=None, **more):
    return tslt.rotate(c["q"], c["k"], c["position"], c["freq"], axis=c["axis"], base=c["base"], q_weight=c["w"][0], k_weight=c["w"][1], eps=c["eps"],
                       adjacent=c["adjacent"], count=c["count"], out=out, **more)


def partner(x, c):
    """|u| + |v| of every channel's pair."""
    u, v = O.pair_channels(0 if c["freq"] is None else 2 * c["freq"].numel(), c["adjacent"])
    a = np.abs(x)
    both = a.copy()
    both[..., u] = both[..., v] = a[..., u] + a[..., v]
    return both


def check(c, out):
    cos, sin, off = turns(c)
    step = torch.finfo(TYPES[c["dtype"]]).eps / 2
    for name, w in zip("qk", c["w"]):
        x = host(c[name])
        want = O.rotate(x, cos, sin, c["adjacent"], host(w), c["eps"])
        normed = O.rotate(x, cos[..., :0], sin[..., :0], c["adjacent"], host(w), c["eps"])
        # x r w: r and two products 3 U; cos and sin: their argument's rounding and the series' last sums 2 U each; the products and sums 2 U
        near = partner(normed, c) * (8 * U + off)
        # the result's own rounding, of what may be off already
        near = near * (1 + step) + step * np.abs(want) + TINY[c["dtype"]]
        got = host(out[name])
        for b, m in enumerate(counts(c)):
            assert np.all(np.abs(got[b, :m] - want[b, :m]) <= near[b, :m]), (name, b, np.max(np.abs(got[b, :m] - want[b, :m]) / near[b, :m]))


CASES = [dict(B=1, n=1, hq=12, h=12, D=64, rotary=64, dtype="f16", eps=None),
         dict(B=1, n=1, hq=1, h=1, D=256, rotary=256, dtype="f32"),
         dict(B=3, n=7, hq=4, h=2, D=64, rotary=32, dtype="bf16", far=130000, ragged=True),
         dict(B=2, n=9, hq=32, h=8, D=128, rotary=128, dtype="bf16", shared=True, far=1000000),
         dict(B=2, n=5, hq=7, h=1, D=128, rotary=64, dtype="f32", axes=3, adjacent=True),
         dict(B=5, n=3, hq=3, h=3, D=256, rotary=64, dtype="f16", axes=4, ragged=True),
         dict(B=2, n=4, hq=2, h=1, D=64, rotary=16, dtype="f32", axes=2, adjacent=True, eps=None, far=2 ** 30),
         dict(B=2, n=3, hq=5, h=5, D=128, rotary=0, dtype="bf16"),
         dict(B=3, n=601, hq=5, h=1, D=64, rotary=64, dtype="bf16", ragged=True),
         dict(B=40, n=33, hq=8, h=2, D=128, rotary=32, dtype="f16", adjacent=True, axes=3, shared=True, far=77),
         dict(B=2, n=700, hq=3, h=2, D=256, rotary=256, dtype="f32", eps=0.0)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_rotate(case):
    c = make(**case)
    out = call(c)
    assert out["status"].tolist() == [0] * c["B"]
    check(c, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_and_what_is_not_counted_stays(dtype):
    c = make(B=4, n=6, hq=4, h=2, D=128, rotary=128, dtype=dtype, ragged=True, seed=3)
    want = call(c, out={"q": torch.full_like(c["q"], 7), "k": torch.full_like(c["k"], 7)})
    before = [c["q"].clone(), c["k"].clone()]
    whole = c["q"]._base.clone() if c["q"]._base is not None else None
    out = call(c, out={"q": c["q"], "k": c["k"], "status": torch.full((4,), 9, dtype=torch.int32, device=DEV)})
    assert out["status"].tolist() == [0] * 4
    for name, was in zip("qk", before):
        for b, m in enumerate(counts(c)):
            assert torch.equal(c[name][b, :m], want[name][b, :m]) and torch.equal(c[name][b, m:], was[b, m:])
            assert torch.equal(want[name][b, m:], torch.full_like(want[name][b, m:], 7))
    if whole is not None:
        assert torch.equal(c["q"]._base[:, :, 6:], whole[:, :, 6:])      # the values beside them


def test_defaults_no_keys_no_positions():
    c = make(B=2, n=70, hq=3, h=1, D=64, rotary=64, dtype="f32", eps=None)
    got = tslt.rotate(c["q"], None, None, c["freq"])
    assert got["k"] is None
    at = torch.arange(70, device=DEV, dtype=torch.int32).view(1, 70, 1)
    assert torch.equal(got["q"], tslt.rotate(c["q"], None, at, c["freq"])["q"])
    axis = torch.arange(32, device=DEV, dtype=torch.int32) % 4
    also = tslt.rotate(c["q"], None, None, c["freq"], axis=axis)   # the same place on every axis
    assert torch.equal(also["q"], got["q"]) and also["status"].tolist() == [0, 0]
    assert torch.equal(tslt.rotate(c["q"], None, None, None)["q"], c["q"])
    normed = tslt.rotate(c["q"], None, None, None, eps=1e-5)["q"]
    want = O.rotate(host(c["q"]), np.ones((2, 70, 0)), np.zeros((2, 70, 0)), False, None, 1e-5)
    assert np.all(np.abs(host(normed) - want) <= 4 * U * np.abs(want))


def test_bad_counts_and_axes_are_told():
    c = make(B=3, n=4, hq=2, h=1, D=64, rotary=32, dtype="bf16", axes=2)
    c["count"] = torch.tensor([-2, 9, 3], dtype=torch.int32, device=DEV)
    out = call(c, out={"q": torch.zeros_like(c["q"]), "k": torch.zeros_like(c["k"]), "status": torch.zeros(3, dtype=torch.int32, device=DEV)})
    assert out["status"].tolist() == [32, 32, 0]
    check(c, out)
    assert not out["q"][0].any()
    c["count"] = None
    c["axis"][3], c["axis"][5] = 2, -1
    out = call(c)
    assert out["status"].tolist() == [32] * 3
    check(c, out)                                                  # (the oracle takes the nearest axis too)


@pytest.mark.parametrize("dtype,size", [("bf16", 1e30), ("f32", 1e25), ("f32", 1e-30), ("f16", 1e4)])
def test_squares_neither_overflow_nor_vanish(dtype, size):
    c = make(B=1, n=3, hq=2, h=2, D=128, rotary=128, dtype=dtype, eps=0.0, spread=size)
    check(c, call(c))


def test_a_row_that_is_not_finite_is_alone():
    c = make(B=1, n=2, hq=8, h=2, D=64, rotary=64, dtype="f32", seed=5)
    want = call(c)
    c["q"][0, 1, 3, 9] = float("nan")
    c["q"][0, 0, 2, 1] = float("inf")
    out = call(c)
    bad = torch.zeros(1, 2, 8, dtype=torch.bool, device=DEV)
    bad[0, 1, 3] = bad[0, 0, 2] = True
    assert torch.equal(out["q"][~bad], want["q"][~bad]) and torch.equal(out["k"], want["k"])
    assert out["q"][0, 1, 3].isnan().all() and not out["q"][0, 0, 2].isfinite().all()


BACK = [dict(B=1, n=1, hq=1, h=1, D=64, rotary=64, dtype="f32"),
        dict(B=1, n=64, hq=12, h=12, D=64, rotary=32, dtype="f32", adjacent=True),
        dict(B=3, n=5, hq=4, h=2, D=128, rotary=128, dtype="bf16", far=130000, ragged=True),
        dict(B=2, n=9, hq=7, h=1, D=256, rotary=64, dtype="f16", axes=3),
        dict(B=2, n=3, hq=2, h=2, D=64, rotary=16, dtype="bf16", eps=None, axes=2, ragged=True),
        dict(B=3, n=801, hq=4, h=2, D=128, rotary=64, dtype="f32", ragged=True, shared=True)]


def backward(c, out=None, **more):
    norm = c["eps"] is not None
    return tslt.rotate_backward(c["grad"][0], c["grad"][1], c["q"] if norm else None, c["k"] if norm else None, c["position"], c["freq"], axis=c["axis"],
                                base=c["base"], q_weight=c["w"][0], k_weight=c["w"][1], eps=c["eps"], adjacent=c["adjacent"], count=c["count"], out=out, **more)


def check_backward(c, out):
    cos, sin, off = turns(c)
    step = torch.finfo(TYPES[c["dtype"]]).eps / 2
    here = np.zeros((c["B"], c["n"], 1, 1))
    for b, m in enumerate(counts(c)):
        here[b, :m] = 1
    for name, g, w in zip("qk", c["grad"], c["w"]):
        g, x, w = host(g) * here, host(c[name]), host(w)
        want, dw = O.rotate_backward(g, x, cos, sin, c["adjacent"], w, c["eps"])
        turned = partner(g, c)
        if c["eps"] is None:
            near = turned * (6 * U + off)
        else:
            # r (h - x r mean(h x r)): h 7 U and `off` of the pair's size (turned back, times the weight), x r 2 U, the mean as far off as its terms and U; three more roundings
            r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + c["eps"])
            h, xr = turned * np.abs(w), np.abs(x) * r
            near = r * (h + xr * (h * xr).mean(-1, keepdims=True)) * (14 * U + off)
            # each term 10 U of |g' x r|; a lane's sum of its rows in fp32 (at most 2 rows of a head for each of its rounds), the rest in fp64, rounded twice
            terms = partner(g, c) * xr
            rounds = 4 + terms.shape[0] * terms.shape[1] * terms.shape[2] / 64
            assert np.all(np.abs(host(out[name + "_weight"]) - dw) <= terms.sum((0, 1, 2)) * ((12 + rounds) * U + off) + 2.0 ** -140), name
        near = near * (1 + step) + step * np.abs(want) + TINY[c["dtype"]]
        assert np.all(np.abs(host(out[name]) - want) <= near), (name, np.max(np.abs(host(out[name]) - want) / near))


@pytest.mark.parametrize("case", BACK, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_rotate_backward(case):
    c = make(**case)
    out = backward(c)
    assert out["status"].tolist() == [0] * c["B"]
    check_backward(c, out)
    again = backward(c)
    assert all(torch.equal(out[k], again[k]) for k in out if out[k] is not None)


def test_gradient_against_differences_of_the_call():
    """fp32, one number moved at a time: (f(x + d) - f(x - d)) / 2d of the call itself.  An output is off by 8 U of its pair (some 2^-21 of numbers around 1), of
    256 outputs with random signs some 2^-17 together, over 2d = 2^-5: 2^-12; the third derivative's part d^2 / 6 is some 2^-14 of a gradient around 1."""
    c = make(B=1, n=2, hq=1, h=1, D=64, rotary=32, dtype="f32", eps=1e-3, seed=11)
    got = backward(c)
    d = 2.0 ** -6
    x0 = c["q"].clone()
    for i, at in [(0, 0), (0, 17), (1, 40), (1, 63), (0, 31)]:
        f = []
        for sign in (1, -1):
            c["q"].copy_(x0)
            c["q"][0, i, 0, at] += sign * d
            f.append((call(c)["q"].double() * c["grad"][0].double()).sum().item())
        c["q"].copy_(x0)
        assert abs((f[0] - f[1]) / (2 * d) - got["q"][0, i, 0, at].item()) < 2.0 ** -10


def test_backward_in_place_without_weights_and_of_nothing():
    c = make(B=3, n=4, hq=3, h=1, D=64, rotary=64, dtype="bf16", ragged=True)
    want = backward(c)
    c["w"] = (None, None)
    plain = backward(c)
    assert plain["q_weight"] is None and plain["k_weight"] is None
    ones = torch.ones(64, device=DEV)
    c["w"] = (ones, ones)
    assert torch.equal(backward(c)["q"], plain["q"])
    c = make(B=3, n=4, hq=3, h=1, D=64, rotary=64, dtype="bf16", ragged=True)
    backward(c, out={"q": c["grad"][0], "k": c["grad"][1]})
    assert torch.equal(c["grad"][0], want["q"]) and torch.equal(c["grad"][1], want["k"])
    c["count"] = torch.zeros(3, dtype=torch.int32, device=DEV)
    none = backward(c, out={"q": torch.full_like(c["q"], 5), "k": torch.full_like(c["k"], 5), "q_weight": torch.full((64,), 5.0, device=DEV),
                            "k_weight": torch.full((64,), 5.0, device=DEV)})
    assert not any(none[k].any() for k in ("q", "k", "q_weight", "k_weight"))
    e = torch.zeros(0, 4, 3, 64, device=DEV)
    got = tslt.rotate_backward(e, None, e, None, None, None, q_weight=ones, eps=1e-6)
    assert not got["q_weight"].any()


def test_on_another_stream_and_replayed():
    c = make(B=4, n=9, hq=8, h=2, D=128, rotary=128, dtype="bf16", far=1000)
    want, back = call(c), backward(c)
    out = {k: torch.zeros_like(v) for k, v in want.items()}
    grads = {k: torch.zeros_like(v) for k, v in back.items()}
    ws = torch.empty(tslt.rotate_backward_workspace_bytes(4, 9, 8, 2, 128), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        call(c, out=out)
        backward(c, out=grads, workspace=ws)
    s.synchronize()
    assert all(torch.equal(out[k], want[k]) for k in want) and all(torch.equal(grads[k], back[k]) for k in back)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(c, out=out)
        backward(c, out=grads, workspace=ws)
    for i in range(3):
        c["base"].add_(17)
        for t in (*out.values(), *grads.values()):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want, back = call(c), backward(c)
        assert all(torch.equal(out[k], want[k]) for k in want) and all(torch.equal(grads[k], back[k]) for k in back)
