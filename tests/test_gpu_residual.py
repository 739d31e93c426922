"""Norms on both sides of a residual sum and their gradients on the GPU against the formulas in 64 bits.

Tolerances.  fp32 sums along rows, in trees of at most 2^10 lanes and chains of at most 130 elements per lane, and the few operations around them err by less than E = 2^-17 of the sum of the terms' sizes;
sums over the rows here, in chains of at most 16 to 90 additions, by less than F = 2^-17.  A value that errs is carried through what it enters.  A bf16 result adds its rounding, at most 2^-8 of its size."""
import ctypes
import itertools
import math

import pytest
import torch

import paper_2511_16041_amd as atb

pytestmark = pytest.mark.gpu
E, F, U = 2.0 ** -17, 2.0 ** -17, 2.0 ** -22
BF16, F32 = torch.bfloat16, torch.float32
ROUNDING = {BF16: 2.0 ** -8, F32: 2.0 ** -24}
EPS = 1e-5


def inputs(M, D, stream=BF16, block=BF16, param=BF16, post="rms", pre="rms", affine="both", groups=1, seed=0, pad=0, scale=0.75, dr=True, device="cuda"):
    """Operands whose rows are `pad` elements further apart than they are long, with NaN between them; groups 0: no gate"""
    g = torch.Generator(device=device).manual_seed(seed)

    def matrix(dtype, s):
        t = (torch.randn((M, D + pad), generator=g, device=device) * s).to(dtype)
        t[:, D:] = float("nan")
        return t[:, :D]

    def vector(at, s, *shape):
        return (at + s * torch.randn(shape or (D,), generator=g, device=device)).to(param)

    def norm(kind):
        return atb.Norm(kind, vector(1, 0.3) if affine in ("both", "weight") else None, vector(0, 0.3) if affine in ("both", "bias") else None, EPS) if kind else None
    rows = torch.exp(torch.randn((M, 1), generator=g, device=device))
    return dict(x=matrix(stream, rows), z=matrix(block, rows), post=norm(post), gate=None if groups == 0 else vector(0.7, 0.3) if groups == 1 else vector(0.7, 0.3, groups, D), scale=scale, pre=norm(pre),
                dr=matrix(stream, 1.0) if dr else None, dh=matrix(block, 1.0) if pre else None)


class _Norm:
    """A norm's row in 64 bits, with what its normed rows may be off where v is off by e"""

    def __init__(self, norm, v, e):
        D, one = v.shape[1], torch.ones(v.shape[1], dtype=torch.float64, device=v.device)
        self.w = norm.weight.double() if norm and norm.weight is not None else one
        self.b = norm.bias.double() if norm and norm.bias is not None else 0 * one
        self.norm, self.centre = norm, norm is not None and norm.kind == "layer"
        if norm is None:
            self.hat, self.e_hat, self.rstd, self.e_rstd = v, e, torch.ones_like(v[:, :1]), 0
        else:
            c = v - v.mean(1, keepdim=True) if self.centre else v
            self.rstd = (c.square().mean(1, keepdim=True) + norm.eps).rsqrt()
            self.hat = c * self.rstd
            top = v.abs().amax(1, keepdim=True) * self.rstd
            spread = self.rstd * e.square().mean(1, keepdim=True).sqrt()
            self.e_rstd = E * (1 + (top if self.centre else 0)) + spread                     # relative
            self.e_hat = self.rstd * (e + (e.mean(1, keepdim=True) if self.centre else 0)) + E * (self.hat.abs() + (top if self.centre else 0)) + self.hat.abs() * self.e_rstd
        self.y = self.hat * self.w + self.b
        self.e_y = self.e_hat * self.w.abs() + U * (self.hat * self.w).abs() + U * self.b.abs() if norm else e

    def back(self, dy, e):
        """The gradient of v, and what it may be off"""
        g, e_g = dy * self.w, e * self.w.abs() + U * (dy * self.w).abs()
        if self.norm is None:
            return g, e_g
        m1 = (g * self.hat).mean(1, keepdim=True)
        e_m1 = E * (g * self.hat).abs().mean(1, keepdim=True) + (g.abs() * self.e_hat + e_g * self.hat.abs()).mean(1, keepdim=True)
        m0 = g.mean(1, keepdim=True) if self.centre else 0 * m1
        e_m0 = E * g.abs().mean(1, keepdim=True) + e_g.mean(1, keepdim=True) if self.centre else 0 * m1
        v = self.rstd * (g - m0 - self.hat * m1)
        return v, self.rstd * (e_g + e_m0 + self.e_hat * m1.abs() + self.hat.abs() * e_m1 + U * (g.abs() + m0.abs() + (self.hat * m1).abs())) + v.abs() * self.e_rstd


def reference(a):
    """{name: (value in 64 bits, tolerance but for the result's own rounding)}"""
    x, z, M, D = a["x"].double(), a["z"].double(), *a["x"].shape
    gate = a["gate"].double().reshape(-1, D) if a["gate"] is not None else torch.ones((1, D), dtype=torch.float64, device=x.device)
    G = gate.shape[0]
    k = gate.repeat_interleave(M // G, 0) if M else gate[:0]
    n1 = _Norm(a["post"], z, 0 * z)
    r = a["scale"] * x + k * n1.y
    e_r = k.abs() * n1.e_y + U * ((a["scale"] * x).abs() + (k * n1.y).abs() + r.abs())
    out = {"r": (r, e_r)}
    d = a["dr"].double() if a["dr"] is not None else 0 * x
    e_d = U * d.abs()
    if a["pre"]:
        n2 = _Norm(a["pre"], r, e_r)
        out["h"] = (n2.y, n2.e_y)
        dh = a["dh"].double()
        back, e = n2.back(dh, 0 * dh)
        d, e_d = d + back, e_d + e + U * (d.abs() + back.abs())
        out["dpre_weight"] = ((dh * n2.hat).sum(0), (dh.abs() * n2.e_hat + F * (dh * n2.hat).abs()).sum(0))
        out["dpre_bias"] = (dh.sum(0), F * dh.abs().sum(0))
    out["dx"] = (a["scale"] * d, abs(a["scale"]) * e_d)

    def over(t):
        return t.reshape(G, -1, D).sum(1)
    out["dgate"] = (over(d * n1.y), over(e_d * n1.y.abs() + d.abs() * n1.e_y + F * d.abs() * ((n1.hat * n1.w).abs() + n1.b.abs())))
    q, e_q = d * k, e_d * k.abs() + U * (d * k).abs()
    if a["post"]:
        out["dpost_weight"] = ((q * n1.hat).sum(0), (e_q * n1.hat.abs() + q.abs() * n1.e_hat + F * (q * n1.hat).abs()).sum(0))
        out["dpost_bias"] = (q.sum(0), (e_q + F * q.abs()).sum(0))
    out["dz"] = n1.back(q, e_q)
    return out


def close(got, want):
    for name, t in got.items():
        if t is None:
            continue
        ref, tol = want[name]
        ref = ref.reshape(t.shape)
        limit = tol.reshape(t.shape) + ROUNDING[t.dtype] * ref.abs() + 1e-30
        off = (t.double() - ref).abs()
        assert bool((off <= limit).all()), f"{name}: worst {float((off / limit).nan_to_num(1e30).max())} of the tolerance"


def run(a, stream=None):
    args = (a["post"], a["gate"], a["scale"], a["pre"])
    r, h, stats = atb.residual_norm(a["x"], a["z"], *args, save=True, stream=stream)
    g = atb.residual_norm_backward(a["dr"], a["dh"], a["x"], a["z"], stats, *args, stream=stream)
    return {"r": r, "h": h, **g._asdict()}


def check(a):
    want, got = reference(a), run(a)
    close(got, want)
    assert (got["h"] is None) == (a["pre"] is None) and (got["dgate"] is None) == (a["gate"] is None)
    for side in ("post", "pre"):
        for name in ("weight", "bias"):
            assert (got[f"d{side}_{name}"] is None) == (a[side] is None or getattr(a[side], name) is None)
    r, h = atb.residual_norm(a["x"], a["z"], a["post"], a["gate"], a["scale"], a["pre"])
    assert torch.equal(r, got["r"]) and (h is None or torch.equal(h, got["h"]))
    return got


SIZES = [(1, 1), (3, 2), (2, 7), (5, 8), (9, 63), (33, 512), (17, 513), (64, 520), (7, 1000), (300, 1024), (9, 1025), (6, 2049), (600, 4096), (40, 4097), (21, 5001), (700, 8192), (6, 8193), (5, 9000),
         (70, 16384), (4, 16385), (3, 70000), (4000, 96)]


@pytest.mark.parametrize("post,pre", [("rms", "rms"), ("layer", "layer"), (None, "rms")])
@pytest.mark.parametrize("stream,block,param", [(BF16, BF16, BF16), (F32, BF16, BF16), (F32, F32, F32)])
@pytest.mark.parametrize("M,D", SIZES)
def test_forward_and_backward(M, D, stream, block, param, post, pre):
    check(inputs(M, D, stream, block, param, post, pre, seed=M * 7 + D))


@pytest.mark.parametrize("M,D", [(37, 333), (130, 5000), (9, 9001)])
@pytest.mark.parametrize("stream,block,param", [(BF16, BF16, F32), (F32, BF16, F32), (F32, F32, BF16)])
@pytest.mark.parametrize("affine", ["both", "weight", "bias", "none"])
@pytest.mark.parametrize("post,pre", [("layer", "rms"), ("rms", "layer"), ("rms", None), (None, None), (None, "layer")])
def test_norms_and_missing_parameters(M, D, stream, block, param, affine, post, pre):
    check(inputs(M, D, stream, block, param, post, pre, affine, seed=3, groups=0 if affine == "none" else 1))


@pytest.mark.parametrize("M,D,groups", [(6, 100, 6), (24, 500, 3), (300, 1000, 300), (600, 4096, 5), (1200, 700, 2), (64, 5000, 4), (30, 9000, 3), (1300, 16, 650)])
@pytest.mark.parametrize("affine", ["both", "weight"])
@pytest.mark.parametrize("stream", [BF16, F32])
def test_a_gate_for_every_group_of_rows(M, D, groups, affine, stream):
    check(inputs(M, D, stream, BF16, BF16, "rms", "layer", affine, groups, seed=4))
    check(inputs(M, D, stream, BF16, BF16, None, "rms", affine, groups, seed=5))


@pytest.mark.parametrize("M,D,pad", [(37, 1000, 3), (5, 8192, 1), (9, 4099, 5), (3, 17000, 5), (130, 77, 51)])
@pytest.mark.parametrize("stream,block", [(BF16, BF16), (F32, BF16), (F32, F32)])
def test_rows_further_apart(M, D, pad, stream, block):
    check(inputs(M, D, stream, block, BF16, "layer", "rms", seed=6, pad=pad))


@pytest.mark.parametrize("D", [300, 5000, 9000])
def test_without_a_gradient_of_the_sum(D):
    check(inputs(50, D, dr=False, seed=7))


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("D", [700, 5000, 20000])
def test_constant_and_empty_rows_and_rows_that_are_not_finite(kind, D):
    a = inputs(8, D, F32, F32, F32, kind, kind, seed=9)
    want = reference(a)
    x, z = a["x"].clone(), a["z"].clone()
    z[1] = 0.0                        # the norm of nothing: its bias
    z[2, 5] = float("nan")
    z[4, D - 1] = float("inf")
    x[6, 3] = float("nan")
    got = run({**a, "x": x, "z": z})
    assert torch.equal(got["r"][1], a["scale"] * x[1] + a["gate"] * a["post"].bias) or bool((got["r"][1] - (a["scale"] * x[1] + a["gate"] * a["post"].bias)).abs().max() <= 2.0 ** -20 * (1 + x[1].abs().max()))
    assert not got["h"][[2, 4, 6]].isfinite().any() and not got["dx"][[2, 4, 6]].isfinite().all(1).any()
    assert got["r"][6].isnan().sum() == 1
    rows = [0, 3, 5, 7]
    close({k: got[k][rows] for k in ("r", "h", "dx", "dz")}, {k: tuple(t[rows] for t in want[k]) for k in ("r", "h", "dx", "dz")})
    assert got["dx"][1].isfinite().all() and got["dz"][1].isfinite().all()


@pytest.mark.parametrize("groups", [0, 1, 4])
def test_no_rows(groups):
    a = inputs(4, 96, groups=groups, seed=8)
    a = {k: t[:0] if k in ("x", "z", "dr", "dh") else t for k, t in a.items()}
    got = run(a)
    assert got["r"].shape == got["h"].shape == got["dx"].shape == (0, 96)
    assert not any(got[k].any() for k in ("dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias"))
    assert groups == 0 or not got["dgate"].any()


def test_same_bits_every_time_and_on_another_stream():
    for D, groups in ((1000, 1), (5000, 3), (9000, 1)):
        a = inputs(300, D, groups=groups, seed=10)
        first = run(a)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        again = run(a, stream=side)
        side.synchronize()
        assert all(torch.equal(first[k], again[k]) for k in first)


def test_captured_and_replayed():
    kinds = dict(stream=F32, groups=4)
    static = inputs(120, 1000, seed=11, **kinds)
    moving = ("x", "z", "dr", "dh")
    static = {k: t.clone() if k in moving else t for k, t in static.items()}
    run(static)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run(static)
    for seed in (11, 12, 13):
        new = inputs(120, 1000, seed=seed, **kinds)
        for k in moving:
            static[k].copy_(new[k])
        graph.replay()
        eager = run({**static, **{k: new[k] for k in moving}})
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], eager[k]) for k in out), seed


def test_in_place_and_only_the_gradients_that_are_asked_for():
    """The C entry points: r in x's and h in z's place; some of the gradients left out."""
    M, D = 70, 1000
    L, stream = atb.lib(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    a = inputs(M, D, groups=2, seed=14)
    all_of = run(a)
    x, z = a["x"].clone(), a["z"].clone()

    def norm(n):
        return atb.NormArgs(n.weight.data_ptr(), n.bias.data_ptr(), n.eps, 1)
    p = atb.ResidualNorm(x.data_ptr(), z.data_ptr(), D, D, norm(a["post"]), norm(a["pre"]), a["gate"].data_ptr(), 2, a["scale"], M, D, 0, 0, 0)
    stats = torch.empty((4, M), device="cuda")
    assert L.atb_residual_norm_forward(ctypes.byref(p), x.data_ptr(), D, z.data_ptr(), D, stats.data_ptr(), stream) == 0
    assert torch.equal(x, all_of["r"]) and torch.equal(z, all_of["h"])
    x.copy_(a["x"])
    z.copy_(a["z"])
    work = torch.empty(L.atb_residual_norm_workspace(M, D, 2), dtype=torch.uint8, device="cuda")
    names = [k for k in all_of if k.startswith("d")]
    out = {k: torch.zeros_like(all_of[k]) for k in names}
    for asked in [("dx",), ("dz",), ("dgate",), ("dpre_weight", "dz"), ("dpost_bias",), ("dx", "dpost_weight", "dpre_bias"), ()]:
        for t in out.values():
            t.zero_()
        ptr = {k: out[k].data_ptr() if k in asked else None for k in names}
        g = atb.ResidualNormGradArgs(ptr["dx"], ptr["dz"], D, D, ptr["dgate"], ptr["dpost_weight"], ptr["dpost_bias"], ptr["dpre_weight"], ptr["dpre_bias"])
        assert L.atb_residual_norm_backward(ctypes.byref(p), stats.data_ptr(), a["dr"].data_ptr(), D, a["dh"].data_ptr(), D, ctypes.byref(g), work.data_ptr(), stream) == 0
        for k in names:
            assert torch.equal(out[k], all_of[k]) if k in asked else not out[k].any(), (asked, k)


@pytest.mark.parametrize("D", [4100, 16400])
def test_more_elements_than_32_bits_count(D):
    M = 2 ** 31 // D + 9
    a = inputs(4, D, seed=15, groups=1)
    rows = [0, M // 2, M - 2, M - 1]
    big = {}
    for k in ("x", "z", "dr", "dh"):
        big[k] = torch.zeros((M, D), dtype=BF16, device="cuda")
        big[k][rows] = a[k]
    got = run({**a, **big})
    want = reference(a)
    # (rows of zeros have gradients of zero: only their 0 dh and dr enter the sums)
    close({k: got[k][rows] for k in ("r", "h", "dx", "dz")}, want)
    close({k: got[k] for k in ("dgate", "dpost_weight", "dpre_weight", "dpre_bias", "dpost_bias")}, want)


def test_gradients_against_differences():
    """The kernels' own forward pass in fp32, moved both ways along each operand's gradient."""
    for post, pre in itertools.product(("rms", "layer"), ("rms", "layer")):
        a = inputs(8, 600, F32, F32, F32, post, pre, groups=2, seed=16)
        got = run(a)

        def loss(b):
            r, h = atb.residual_norm(b["x"], b["z"], b["post"], b["gate"], b["scale"], b["pre"])
            return float((r.double() * a["dr"].double()).sum() + (h.double() * a["dh"].double()).sum())
        size = float((got["r"].double() * a["dr"].double()).abs().sum() + (got["h"].double() * a["dh"].double()).abs().sum())

        def moved(name, t):
            if name in ("dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias"):
                side, which = name[1:].split("_")
                return {**a, side: a[side]._replace(**{which: t})}
            return {**a, name[1:]: t}
        for name in ("dx", "dz", "dgate", "dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias"):
            grad = got[name].double()
            here = getattr(a[name[1:].split("_")[0]], name[1:].split("_")[1]) if "_" in name else a[name[1:]]
            step = grad * (2.0 ** -6 / float(grad.abs().max()))
            ends = [(here.double() + s * step).float() for s in (1, -1)]
            slope = loss(moved(name, ends[0])) - loss(moved(name, ends[1]))
            want = float((grad * (ends[0].double() - ends[1].double())).sum())
            # the results' errors, at most E of each; the third derivative: its share of the slope is the square of the relative move, 2^-12, times a few
            assert abs(slope - want) <= 2 * E * size * 0.1 + 2.0 ** -8 * abs(want), (post, pre, name, slope, want)


# ------------------------------------------------------------------ gradients that are infinite or nearly so

def limits_of(t):
    """A result's infinities and NaNs: 1, -1, 2; of numbers 0"""
    return torch.where(t.isnan(), 2.0, torch.where(t.isinf(), t.double().sign(), 0.0))


@pytest.mark.parametrize("stream,block", [(BF16, BF16), (F32, BF16), (F32, F32)])
@pytest.mark.parametrize("post,pre,of_r", [("rms", "rms", False), ("rms", None, True), ("rms", "layer", True), (None, "rms", False)])
@pytest.mark.parametrize("D", [64, 99, 700, 5000, 9000, 12500, 20000])
def test_gradients_whose_sum_passes_fp32_through_root_mean_square_norms(D, post, pre, of_r, stream, block):
    """These norms' formulas have sum(g xh) in them and not sum(g).  Gradients of 2^129 / D or more, all of one sign: the second is more than a float holds; the first, whose terms have either sign, is about 2^129 / sqrt(D)."""
    a = inputs(6, D, stream, block, BF16, post, pre, seed=D, scale=1.0)
    a["z"], a["x"] = (a["z"].double().sign() * (1 + a["z"].double().abs() % 1)).to(block), (0.5 * a["x"].double().sign()).to(stream)
    large = torch.full((6, D), 2.0 ** (129 - int(math.log2(D))), device="cuda")
    a["dr"] = (large if of_r else 0 * large).to(stream)
    if pre:
        a["dh"], a["pre"] = (0 * large if of_r else large).to(block), a["pre"]._replace(weight=torch.ones_like(a["pre"].weight))
    if post:
        a["post"] = a["post"]._replace(weight=torch.ones_like(a["post"].weight))
    a["gate"] = torch.ones_like(a["gate"])
    got = run(a)
    close({k: got[k] for k in ("dx", "dz")}, reference(a))


def rms_gradient(v, norm, dy):
    """The gradient of a root-mean-square norm's row by its definition, rstd (g - xh mean(g xh)) with g = dy weight, in 64 bits"""
    rstd = (v.square().mean(1, keepdim=True) + norm.eps).rsqrt()
    g, hat = dy * norm.weight.double(), v * rstd
    return rstd * (g - hat * (g * hat).mean(1, keepdim=True))


@pytest.mark.parametrize("stream,block", [(BF16, BF16), (F32, BF16), (F32, F32)])
@pytest.mark.parametrize("D", [7, 64, 99, 700, 5000, 9000, 12500, 20000])
def test_an_infinite_gradient_is_infinite_in_its_row(D, stream, block):
    """dh or dr infinite at one place: through root-mean-square norms dx and dz have the signs that the formulas give, and no other row has any."""
    for post, pre, name in ((None, "rms", "dh"), ("rms", None, "dr")):
        a = inputs(6, D, stream, block, BF16, post, pre, seed=D + 1)
        a[name] = a[name].clone()
        a[name][2, D // 2], a[name][4, D - 1] = float("inf"), float("-inf")
        x, z, gate, t = a["x"].double(), a["z"].double(), a["gate"].double(), a["dr"].double()
        if pre:
            t = t + rms_gradient(a["scale"] * x + gate * z, a["pre"], a["dh"].double())
        want, got = {"dx": a["scale"] * t, "dz": rms_gradient(z, a["post"], t * gate) if post else t * gate}, run(a)
        for k in ("dx", "dz"):
            kinds = limits_of(got[k])
            assert torch.equal(kinds, limits_of(want[k])), (name, k)
            assert kinds[[2, 4]].any() and not kinds[[0, 1, 3, 5]].any(), (name, k)


@pytest.mark.parametrize("groups", [1, 2, 3])
@pytest.mark.parametrize("D", [7, 100, 5000, 9000, 20000])
@pytest.mark.parametrize("post,weight,bias", [(None, None, None), ("rms", 1.0, None), ("rms", 1.0, 0.0), ("layer", None, 0.0), ("layer", 0.0, 0.5), ("rms", 0.0, 0.0)])
def test_an_infinite_gradient_reaches_the_gate_as_it_is(post, weight, bias, D, groups):
    """dr infinite at one place, with a norm `pre` that has a bias: sum t n1 is infinite of the sign of t n1, or NaN where n1 is 0, and nothing else of the gate's gradient is."""
    a = inputs(6, D, F32, F32, F32, post, "layer", groups=groups, seed=D)
    a["dr"], a["dh"] = a["dr"].clone(), 0 * a["dh"]
    at = D // 2
    a["dr"][4, at] = float("inf")
    if post:
        a["post"] = a["post"]._replace(**{k: torch.full_like(a["gate"].reshape(-1, D)[0], v) if v is not None else None for k, v in (("weight", weight), ("bias", bias))})
    want, got = limits_of(reference(a)["dgate"][0]), limits_of(run(a)["dgate"]).reshape(groups, D)
    kind = float(want[4 // (6 // groups), at])
    assert kind == 2 if weight == bias == 0.0 else abs(kind) == 1
    assert torch.equal(got, want)


@pytest.mark.parametrize("stream,block", [(BF16, BF16), (F32, BF16)])
@pytest.mark.parametrize("D", [7, 8, 13, 96, 100, 515, 700, 5001, 8190, 9003, 12501, 20000])
def test_an_infinite_weight_or_gate_gives_what_the_formulas_give(D, stream, block):
    """Weight or gate of a root-mean-square norm infinite at the last elements of the row but one: the signs of dx and dz are the formulas', wherever the last chunks of a row lie."""
    for post, pre, where in ((None, "rms", "pre"), ("rms", None, "post"), ("rms", None, "gate")):
        a = inputs(5, D, stream, block, BF16, post, pre, seed=D + 3)
        t = (a["gate"] if where == "gate" else a[where].weight).clone()
        t[D - 2] = float("inf")
        a = {**a, **({"gate": t} if where == "gate" else {where: a[where]._replace(weight=t)})}
        x, z, gate, d = a["x"].double(), a["z"].double(), a["gate"].double(), a["dr"].double()
        if pre:
            d = d + rms_gradient(a["scale"] * x + gate * z, a["pre"], a["dh"].double())
        want, got = {"dx": a["scale"] * d, "dz": rms_gradient(z, a["post"], d * gate) if post else d * gate}, run(a)
        for k in ("dx", "dz"):
            kinds = limits_of(got[k])
            assert torch.equal(kinds, limits_of(want[k])), (where, k)
            assert kinds.any() == (k == "dz" or where == "pre"), (where, k)
