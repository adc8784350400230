"""tslt_logprob and tslt_logprob_backward against the oracle, on the GPU."""
import numpy as np
import pytest
import torch

from oracle import round_oracle as O
from paper_2512_16273_amd import tslt

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0 ** -24
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}
INF = float("inf")


def make(B, n, V, dtype, T=1.0, top=0, m=None, ragged=False, pad=0, offset=0, kind="plain", seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    z = torch.full((offset + B * n * (V + pad),), 1000.0, dtype=TYPES[dtype], device=DEV)[offset:].view(B, n, V + pad)
    x = 2.5 * torch.randn(B, n, V, generator=g, device=DEV) - torch.log1p(V * torch.rand(B, n, V, generator=g, device=DEV))
    if kind == "equal":
        x = torch.full_like(x, 1.5)
    elif kind == "few values":
        x = torch.randint(0, 3, x.shape, generator=g, device=DEV).float()
    elif kind == "rising":
        x = torch.arange(V, device=DEV).float().expand_as(x) * (20.0 / V)
    elif kind == "falling":
        x = -torch.arange(V, device=DEV).float().expand_as(x) * (20.0 / V)
    elif kind == "masked":                                         # a few tokens left, or one, or the mask is the type's lowest number
        few = torch.rand(x.shape, generator=g, device=DEV) < 3.0 / V
        few[:, :, V // 2] = True
        low = torch.finfo(TYPES[dtype]).min
        x = torch.where(few, x, torch.where(torch.arange(n, device=DEV)[:, None] % 2 == 0, -INF, low))
    elif kind == "lowest":                                         # nothing but the type's lowest number
        x = torch.full_like(x, torch.finfo(TYPES[dtype]).min)
    elif kind == "far":
        x = x + (30000.0 if dtype == "f16" else 3.0e6)
    elif kind == "zeros":
        x = torch.where(torch.rand(x.shape, generator=g, device=DEV) < 0.5, 0.0, -0.0)
    z[:, :, :V] = x
    m_ = m if m is not None else n
    c = dict(logits=z[:, :, :V], T=T, top=top, dtype=dtype, B=B, n=n, m=m_, V=V)
    c["index"] = torch.randint(0, n, (B, m), generator=g, device=DEV, dtype=torch.int32) if m is not None else None
    c["tokens"] = torch.randint(0, V, (B, m_), generator=g, device=DEV, dtype=torch.int32)
    c["count"] = torch.tensor([(3 * b + 1) % (m_ + 1) for b in range(B)], dtype=torch.int32, device=DEV) if ragged else None
    return c


def call(c, out=None, **more):
    return tslt.logprob(c["logits"], c["T"], c["tokens"], top=c["top"], index=c["index"], count=c["count"], out=out, **more)


def host(t):
    return t.detach().double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def counts(c):
    return [c["m"]] * c["B"] if c["count"] is None else [min(max(int(x), 0), c["m"]) for x in c["count"]]


def oracle(c):
    z, rT = host(c["logits"]), O.inverse_temperature(c["T"])
    for b, m in enumerate(counts(c)):
        for j in range(m):
            i = j if c["index"] is None else int(c["index"][b, j])
            yield b, j, z[b, i] * 1.0, O.logprob_row(z[b, i], rT, int(c["tokens"][b, j]), c["top"])


def check(c, out):
    got = {k: host(v) for k, v in out.items()}
    rT = O.inverse_temperature(c["T"])
    for b, j, z, want in oracle(c):
        where = (b, j)
        assert got["status"][b, j] == want["status"], where
        if want["status"]:
            continue
        # S: an exponent's rounding, U of it and of the scale's (weighed by their terms no more than log2 V + 2 of them count), the exponential's 2 U, a lane's
        # sums of its vectors and within one; rounded once more
        S = (2 * (np.log2(c["V"]) + 2) + 2 + c["V"] / 1024 + 10) * U
        near = S + U * abs(want["lse"]) + 2.0 ** -140
        assert abs(got["lse"][b, j] - want["lse"]) <= near, (where, got["lse"][b, j], want["lse"])
        assert abs(got["entropy"][b, j] - want["entropy"]) <= 2 * S * (1 + np.log(c["V"])) + U * want["entropy"], (where, got["entropy"][b, j], want["entropy"])
        for x, y in [(got["logp"][b, j], want["logp"])] + (list(zip(got["top_logp"][b, j], want["top_logp"])) if c["top"] else []):
            assert x == y if np.isinf(y) else abs(x - y) <= S + U * abs(y) + 1e-15 * abs(want["lse"]), (where, x, y)
        if c["top"]:
            assert np.array_equal(got["top_idx"][b, j], want["top_idx"]), (where, got["top_idx"][b, j], want["top_idx"])


CASES = [dict(B=1, n=1, V=32000, dtype="f16", top=5), dict(B=1, n=1, V=1, dtype="f32", top=3), dict(B=2, n=3, V=7, dtype="bf16", top=8, offset=1),
         dict(B=1, n=9, V=128256, dtype="bf16", top=20, T=0.7), dict(B=3, n=5, V=50257, dtype="bf16", top=32, T=1.3, ragged=True, offset=3),
         dict(B=2, n=21, V=4099, dtype="f32", top=1, m=4, ragged=True, pad=13), dict(B=4, n=9, V=1000, dtype="f16", m=6),
         dict(B=1, n=2, V=256000, dtype="f32", top=32), dict(B=40, n=30, V=2049, dtype="bf16", top=5, offset=5),
         dict(B=1, n=700, V=6001, dtype="f16", top=20, T=0.5), dict(B=1, n=1, V=151936, dtype="f32"), dict(B=1, n=4, V=16384, dtype="bf16", top=31)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_logprob(case):
    c = make(**case)
    check(c, call(c))


@pytest.mark.parametrize("kind", ["equal", "few values", "rising", "falling", "masked", "lowest", "far", "zeros"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", [(1, 2, 40003), (1, 1100, 1501), (1, 600, 70001)], ids=str)
def test_rows_of_every_kind(kind, dtype, shape):
    B, n, V = shape
    c = make(B, n, V, dtype, top=11, T=1.0 if kind in ("masked", "lowest") else 0.8, kind=kind, offset=1)
    out = call(c)
    few = min(n, 75000 // V + 5)                                   # (the oracle sorts every row)
    c.update(logits=c["logits"][:, :few], tokens=c["tokens"][:, :few].contiguous(), n=few, m=few)
    out = {k: v[:, :few].contiguous() for k, v in out.items()}
    check(c, out)


def test_rows_that_cannot_be_used_and_tokens_that_are_none():
    c = make(2, 6, 9001, "bf16", top=4)
    z = c["logits"]
    z[0, 0, 8000] = float("nan")
    z[0, 1, 3] = INF
    z[0, 2] = -INF
    z[0, 3] = float("nan")
    c["tokens"][1, :4] = torch.tensor([-1, 9001, -7, 2 ** 31 - 1])
    out = call(c)
    assert out["status"].tolist() == [[1, 1, 2, 1, 0, 0], [0, 32, 32, 32, 0, 0]]
    assert all(out[k][0, :4].isnan().all() for k in ("logp", "entropy")) and out["lse"][0, 2].item() == -INF and out["lse"][0, [0, 1, 3]].isnan().all()
    assert (out["top_idx"][0, :4] == -1).all() and (out["top_logp"][0, :4] == -INF).all()
    assert out["logp"][1, :4].isnan().all() and out["entropy"][1].isfinite().all() and (out["top_idx"][1] >= 0).all()
    again = tslt.logprob(z, 1.0)
    assert again["logp"].isnan().all() and torch.equal(again["entropy"][1], out["entropy"][1]) and "top_idx" not in again


@pytest.mark.parametrize("V", [900, 30000])
def test_index_count_and_what_stays(V):
    c = make(4, 5, V, "f32", top=3, m=7)
    c["index"][0, 2], c["index"][1, 0], c["index"][2, 1] = 5, -1, 2 ** 31 - 1
    c["index"][3] = 4                                              # one row many times
    c["count"] = torch.tensor([7, 9, 2, -3], dtype=torch.int32, device=DEV)
    names = {"logp": 1, "entropy": 1, "lse": 1, "status": 1, "top_idx": 3, "top_logp": 3}
    out = {k: torch.full((4, 7) if w == 1 else (4, 7, 3), 77, dtype=torch.int32 if k in ("status", "top_idx") else torch.float32, device=DEV) for k, w in names.items()}
    call(c, out=out)
    assert out["status"].tolist() == [[0, 0, 32, 0, 0, 0, 0], [32, 0, 0, 0, 0, 0, 0], [0, 32] + [77] * 5, [32] + [77] * 6]
    assert all((out[k][2, 2:] == 77).all() and (out[k][3] == 77).all() for k in names if k != "status")
    for b, j in ((0, 2), (1, 0), (2, 1)):
        assert out["logp"][b, j].isnan() and out["entropy"][b, j].isnan() and out["lse"][b, j].isnan() and (out["top_idx"][b, j] == -1).all()
    for b, j in ((0, 0), (0, 6), (1, 3), (2, 0)):
        one = tslt.logprob(c["logits"][b:b + 1, int(c["index"][b, j]):int(c["index"][b, j]) + 1], 1.0, c["tokens"][b:b + 1, j:j + 1].contiguous(), top=3)
        assert torch.equal(one["top_idx"][0, 0], out["top_idx"][b, j]) and abs(one["lse"].item() - out["lse"][b, j].item()) < 1e-5
    c["index"], c["count"], c["tokens"] = torch.full((4, 7), 3, dtype=torch.int32, device=DEV), None, c["tokens"][:, :1].expand(4, 7).contiguous()
    same = call(c)
    assert all(torch.equal(same[k], same[k][:, :1].expand_as(same[k])) for k in same)


def test_strides_of_sequences_and_rows():
    c = make(3, 4, 5003, "f16", top=6, pad=5)
    want = call(c)
    wide = torch.zeros(4, 3, 2, 5011, dtype=torch.float16, device=DEV)
    wide[:, :, 1, :5003] = c["logits"].transpose(0, 1)
    c["logits"] = wide[:, :, 1, :5003].transpose(0, 1)
    got = call(c)
    assert torch.equal(got["top_idx"], want["top_idx"]) and (got["lse"] - want["lse"]).abs().max() < 1e-5
    one = c["logits"][1:2, :1].expand(2, 4, 5003)                  # one row for all
    many = tslt.logprob(one, 1.0, top=2)
    assert torch.equal(many["lse"], many["lse"][:1, :1].expand(2, 4))


def test_partial_outputs():
    c = make(1, 3, 20000, "bf16")
    want = call(c)
    for name in ("logp", "entropy", "lse"):
        got = tslt.logprob(c["logits"], 1.0, c["tokens"], out={name: torch.zeros(1, 3, device=DEV)})
        assert torch.equal(got[name], want[name])


# ---- the gradient -----------------------------------------------------------------------------------------------

def gradients(c, seed=1, which=("grad_logp", "grad_entropy", "grad_lse", "grad_top")):
    g = torch.Generator(device=DEV).manual_seed(seed)
    got = {k: torch.randn(c["B"], c["n"], *([c["top"]] if k == "grad_top" else []), generator=g, device=DEV) for k in ("grad_logp", "grad_entropy", "grad_lse", "grad_top")}
    return {k: v if k in which and not (k == "grad_top" and c["top"] == 0) else None for k, v in got.items()}


def back(c, fwd, g, out=None):
    return tslt.logprob_backward(c["logits"], c["T"], c["tokens"], fwd["lse"], fwd["entropy"], top_idx=fwd.get("top_idx"), count=c["count"], out=out, **g)


def check_back(c, fwd, g, dz):
    z, rT, got = host(c["logits"]), O.inverse_temperature(c["T"]), host(dz)
    step = torch.finfo(TYPES[c["dtype"]]).eps / 2
    f = {k: host(v) for k, v in fwd.items()}
    h = {k: None if v is None else host(v) for k, v in g.items()}
    for b, m in enumerate(counts(c)):
        assert not got[b, m:].any()
        for i in range(m):
            of = {k: None if v is None else v[b, i] for k, v in h.items()}
            idx = f["top_idx"][b, i] if c["top"] else None
            want = O.logprob_backward_row(z[b, i], rT, int(c["tokens"][b, i]), f["lse"][b, i], f["entropy"][b, i], idx, of["grad_logp"], of["grad_entropy"], of["grad_lse"], of["grad_top"])
            d = np.maximum(z[b, i] * rT - f["lse"][b, i], -200.0)
            p = np.exp(d)
            size = sum(np.abs(of[k]).sum() for k in ("grad_logp", "grad_lse", "grad_top") if of[k] is not None)
            # (what the kernel has for d + H is fma(c1, d + rho, c0 - c1 rho), rho = k T lse - fl(k T lse), up to U 1.4427 |lse| in powers of two: where d and H
            # vanish, the roundings of both sides are U of |c1 rho|, U^2 |lse| of the gradient, and nothing else is left of them)
            off = U * abs(f["lse"][b, i])
            size = rT * p * (size + (0 if of["grad_entropy"] is None else abs(of["grad_entropy"]) * (np.abs(d) + f["entropy"][b, i] + off)))
            put = np.zeros_like(p)
            for at, v in ([(int(c["tokens"][b, i]), of["grad_logp"])] if of["grad_logp"] is not None else []) + (list(zip(idx, of["grad_top"])) if of["grad_top"] is not None else []):
                if 0 <= at < put.size:
                    put[at] += rT * abs(v)
            # p: its exponent's rounding and the scale's, 2 U of log2 p, the exponential's 2 U; the factors' roundings and the products'
            near = size * (2 * np.abs(d) * 1.4427 + 14) * U + put * 36 * U + 2.0 ** -125 * (1 + np.abs(size))
            near = near * (1 + step) + step * np.abs(want) + TINY[c["dtype"]]
            assert np.all(np.abs(got[b, i] - want) <= near), (b, i, np.max(np.abs(got[b, i] - want) / near))


BACK = [dict(B=1, n=9, V=32000, dtype="f16"), dict(B=1, n=1, V=1, dtype="f32"), dict(B=2, n=3, V=7, dtype="bf16", top=7, offset=1),
        dict(B=2, n=5, V=50257, dtype="bf16", top=20, T=0.7, ragged=True, offset=3), dict(B=3, n=4, V=4099, dtype="f32", top=32, pad=13, T=1.3),
        dict(B=1, n=600, V=3001, dtype="bf16", ragged=True, top=3), dict(B=1, n=3, V=128256, dtype="f32", top=5)]


@pytest.mark.parametrize("case", BACK, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_backward(case):
    c = make(**case)
    fwd, g = call(c), gradients(c)
    check_back(c, fwd, g, back(c, fwd, g)["logits"])


@pytest.mark.parametrize("which", ["grad_logp", "grad_entropy", "grad_lse", "grad_top"])
@pytest.mark.parametrize("kind", ["plain", "masked", "equal", "far"])
def test_each_gradient_alone(which, kind):
    c = make(1, 4, 9001, "f32", top=6, kind=kind)
    fwd, g = call(c), gradients(c, which=(which,))
    check_back(c, fwd, g, back(c, fwd, g)["logits"])


def test_backward_in_place_other_alignments_and_beyond_count():
    for dtype in ("bf16", "f32"):
        c = make(3, 4, 6007, dtype, top=5, ragged=True, pad=3)
        fwd, g = call(c), gradients(c)
        want = back(c, fwd, g)["logits"]
        for shift in (1, 2, 3):                                    # results that lie otherwise than the logits
            held = torch.full((shift + 3 * 4 * 6011,), 9.0, dtype=TYPES[dtype], device=DEV)
            rows = held[shift:].view(3, 4, 6011)
            back(c, fwd, g, out={"logits": rows[:, :, :6007]})
            # (which lanes and how many share a row goes by its alignment, what they compute does not)
            assert torch.equal(rows[:, :, :6007], want) and (rows[:, :, 6007:] == 9).all() and (held[:shift] == 9).all()
        beside = c["logits"]._base.clone()
        back(c, fwd, g, out={"logits": c["logits"]})
        assert torch.equal(c["logits"], want)
        assert torch.equal(c["logits"]._base.reshape(-1)[-3:], beside.reshape(-1)[-3:])


def test_backward_of_rows_and_places_that_are_none():
    c = make(1, 6, 5001, "f32", top=3)
    c["logits"][0, 0, 17] = float("nan")
    c["logits"][0, 1] = -INF
    fwd = call(c)
    c["tokens"][0, 2:5] = torch.tensor([-1, 5001, -9])
    fwd["top_idx"][0, 4] = torch.tensor([7, 7, 9000])              # the same place twice, and none
    g = gradients(c)
    got = back(c, fwd, g)["logits"]
    assert got[0, :2].isnan().all()
    for k in ("logits", "tokens"):
        c[k] = c[k][:, 2:]
    c.update(n=4, m=4)
    check_back(c, {k: v[:, 2:] for k, v in fwd.items()}, {k: v[:, 2:] for k, v in g.items()}, got[:, 2:])


def test_gradient_against_differences_of_the_call():
    """fp32, one logit moved at a time by d = 2^-5: results around 10 are off by some 2^-20 each, 12 of them over 2d: 2^-13; the third derivative's part is d^2 / 6 of
    gradients around 1, 2^-12."""
    c = make(1, 1, 40, "f32", top=4, seed=5)
    g = gradients(c)
    fwd = call(c)
    got = back(c, fwd, g)["logits"]
    z0, d = c["logits"].clone(), 2.0 ** -5
    best = int(fwd["top_idx"][0, 0, 0])
    for at in (best, int(c["tokens"][0, 0]), 3, 39):
        f = []
        for sign in (1, -1):
            c["logits"].copy_(z0)
            c["logits"][0, 0, at] += sign * d
            o = call(c)
            s = c["logits"][0, 0, fwd["top_idx"][0, 0].long()].double() - o["lse"].double()[0, 0]      # (the same tokens, in case their order changed)
            f.append((g["grad_logp"] * o["logp"].double() + g["grad_entropy"] * o["entropy"].double() + g["grad_lse"] * o["lse"].double()).item() + (g["grad_top"][0, 0] * s).sum().item())
        c["logits"].copy_(z0)
        assert abs((f[0] - f[1]) / (2 * d) - got[0, 0, at].item()) < 2.0 ** -9


def test_the_same_bits_on_another_stream_and_replayed():
    c = make(2, 5, 60001, "bf16", top=9, T=0.9)
    fwd, g = call(c), gradients(c)
    grad = back(c, fwd, g)["logits"]
    for _ in range(3):
        again = call(c)
        assert all(torch.equal(again[k], fwd[k]) for k in fwd)
    out = {k: torch.zeros_like(v) for k, v in fwd.items()}
    dz = torch.zeros_like(grad)
    ws = torch.empty(tslt.logprob_workspace_bytes(2, 5, 60001, 9), dtype=torch.uint8, device=DEV)
    assert ws.numel() > 0
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        call(c, out=out, workspace=ws)
        back(c, out, g, out={"logits": dz})
    s.synchronize()
    assert all(torch.equal(out[k], fwd[k]) for k in fwd) and torch.equal(dz, grad)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(c, out=out, workspace=ws)
        back(c, out, g, out={"logits": dz})
    for i in range(4):
        c["logits"].mul_(0.9)
        c["logits"][1, i, 100 * i] = 20.0
        for t in (*out.values(), dz):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        fwd = call(c)
        assert all(torch.equal(out[k], fwd[k]) for k in fwd) and torch.equal(dz, back(c, fwd, g)["logits"])


def test_beside_verification():
    """Of the rows that were verified, the log probability of what was emitted."""
    g = torch.Generator(device=DEV).manual_seed(2)
    B, gamma, V = 3, 4, 5000
    draft = 3 * torch.randn(B * gamma, V, generator=g, device=DEV)
    tr = tslt.truncate(draft, 1.0, 16, 0.0, 16, u=torch.rand(B * gamma, 1, generator=g, device=DEV))
    target = torch.cat([draft.view(B, gamma, V), torch.randn(B, 1, V, generator=g, device=DEV)], 1).contiguous()
    v = tslt.verify(target, 1.0, *(tr[k].view(B, gamma, -1) for k in ("idx", "logit")), tr["count"].view(B, gamma), tr["token"].view(B, gamma),
                    torch.rand(B, gamma, generator=g, device=DEV), torch.rand(B, gamma + 1, generator=g, device=DEV))
    out = {k: torch.full((B, gamma + 1), 7.0, device=DEV) for k in ("logp", "entropy")}
    tslt.logprob(target, 1.0, v["tokens"], count=v["accept_len"] + 1, out=out)
    want = torch.log_softmax(target.double().cpu(), -1)
    for b, a in enumerate(v["accept_len"].tolist()):
        for j in range(gamma + 1):
            x = out["logp"][b, j].item()
            assert x == 7.0 if j > a else abs(x - want[b, j, int(v["tokens"][b, j])].item()) < 1e-5
