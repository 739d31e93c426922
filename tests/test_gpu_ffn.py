"""The gated block in bf16 and its gradients on the GPU against the formulas in 64 bits.

Tolerances.  fp32 sums of K products in MFMA accumulators err by less than 2^-15 of the sum of the products' sizes at these K; the activations add 2^-19 of
their size and 2^-21 absolutely (and half a per cent of what is left of a GELU below -5, under 2e-7).  Every rounding to bf16 is at most 2^-8 of a value: of h ahead of the down projection, of
dg and du ahead of theirs, of the results.  An error of an operand goes through a product with the sizes of the other."""
import math

import pytest
import torch

import paper_2511_16041_amd as atb

pytestmark = pytest.mark.gpu
S, R = 2.0 ** -15, 2.0 ** -8


def activation(name, g):
    if name == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p))
    if name == "gelu":
        p = torch.special.ndtr(g)
        return g * p, p + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    c, a = math.sqrt(2 / math.pi), 0.044715
    p = torch.sigmoid(2 * c * (g + a * g ** 3))
    return g * p, p + g * p * (1 - p) * 2 * c * (1 + 3 * a * g * g)


def reference(x, wg, wu, wd, dy, act):
    """{name: (value in 64 bits, tolerance but for the result's own rounding)}"""
    x, wg, wu, wd = (t.double() for t in (x, wg, wu, wd))
    g, u = x @ wg.t(), x @ wu.t()
    e_g, e_u = S * (x.abs() @ wg.abs().t()), S * (x.abs() @ wu.abs().t())
    a, slope = activation(act, g)
    h = a * u
    e_a = 1.2 * e_g + 2.0 ** -19 * a.abs() + 2.0 ** -21                 # |act'| <= 1.13
    e_h = e_a * u.abs() + a.abs() * e_u + e_a * e_u + R * h.abs()
    y = h @ wd.t()
    out = {"y": (y, e_h @ wd.abs().t() + S * (h.abs() @ wd.abs().t()))}
    if dy is None:
        return out
    dy = dy.double()
    dh, e_dh = dy @ wd, S * (dy.abs() @ wd.abs())
    dg, du = dh * u * slope, dh * a
    e_slope = 1.2 * e_g + 2.0 ** -19 + 2.0 ** -16 * g.abs()             # |act''| <= 1.2; g is kept to 2^-16
    e_u = e_u + 2.0 ** -15 * u.abs()
    e_dg = e_dh * (u * slope).abs() + dh.abs() * (e_u * slope.abs() + u.abs() * e_slope) + R * dg.abs()
    e_du = e_dh * a.abs() + dh.abs() * (e_a + 2.0 ** -15 * (g * slope).abs()) + R * du.abs()
    out["dx"] = (dg @ wg + du @ wu, e_dg @ wg.abs() + e_du @ wu.abs() + S * (dg.abs() @ wg.abs() + du.abs() @ wu.abs()))
    out["dwg"] = (dg.t() @ x, (e_dg + S * dg.abs()).t() @ x.abs())
    out["dwu"] = (du.t() @ x, (e_du + S * du.abs()).t() @ x.abs())
    out["dwd"] = (dy.t() @ h, dy.abs().t() @ (e_h + S * h.abs()))
    return out


def close(got, want):
    for name, (ref, tol) in want.items():
        assert got[name].shape == ref.shape and got[name].dtype == torch.bfloat16
        limit = tol + R * ref.abs() + 1e-30
        off = (got[name].double() - ref).abs()
        assert bool((off <= limit).all()), f"{name}: worst {float((off / limit).max())} of the tolerance"
        # and without a few wrong elements in a large tolerance: three roundings to bf16, each at most 2^-8 / sqrt 3, in the 2-norm
        if ref.numel() > 64 and float(ref.norm()) > 0:
            assert float((got[name].double() - ref).norm()) <= 2 * R * float(ref.norm()), name


def make(M, D, F, seed, pad=0, scale=0.05):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def matrix(rows, cols, s):
        t = (s * torch.randn((rows, cols + pad), generator=gen, device="cuda")).bfloat16()
        t[:, cols:] = float("nan")                   # what lies between the rows is never used
        return t[:, :cols]
    return matrix(M, D, 1.0), matrix(F, D, scale), matrix(F, D, scale), matrix(D, F, scale), matrix(M, D, 0.1)


def train(x, wg, wu, wd, dy, act, stream=None):
    y, state = atb.feed_forward(x, wg, wu, wd, act, save=True, stream=stream)
    dx, dwg, dwu, dwd = atb.feed_forward_backward(dy, x, wg, wu, wd, state, stream=stream)
    return {"y": y, "dx": dx, "dwg": dwg, "dwu": dwu, "dwd": dwd}


# one to a few tiles of either size, both sides of a K-step's and a tile's end; then enough tiles for the large ones in each of the products
SIZES = [(1, 8, 8), (2, 64, 64), (3, 72, 136), (16, 128, 256), (17, 200, 328), (32, 64, 1000), (33, 136, 264), (65, 520, 72), (130, 264, 520), (257, 512, 768), (300, 1032, 1000),
         (2100, 136, 3080), (3900, 4104, 72), (70, 4104, 4000), (1000, 8, 8)]


@pytest.mark.parametrize("M,D,F", SIZES)
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_forward_and_backward(M, D, F, act):
    x, wg, wu, wd, dy = make(M, D, F, seed=M + D + F)
    want = reference(x, wg, wu, wd, dy, act)
    close(train(x, wg, wu, wd, dy, act), want)
    close({"y": atb.feed_forward(x, wg, wu, wd, act)}, {"y": want["y"]})


@pytest.mark.parametrize("M,D,F,pad", [(5, 136, 72, 8), (140, 200, 328, 24), (300, 264, 136, 64)])
def test_rows_further_apart(M, D, F, pad):
    x, wg, wu, wd, dy = make(M, D, F, 3, pad)
    want = reference(x, wg, wu, wd, dy, "silu")
    close(train(x, wg, wu, wd, dy, "silu"), want)
    close({"y": atb.feed_forward(x, wg, wu, wd, "silu")}, {"y": want["y"]})


def test_weights_of_one_matrix_with_other_pitches():
    """Gate and up as halves of one matrix, and with a pitch each."""
    x, wg, wu, wd, dy = make(150, 264, 200, 4)
    both = torch.cat((wg, wu))
    first = train(x, wg, wu, wd, dy, "silu")
    wide = torch.full((200, 296), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, :264] = wu
    for a, b in ((both[:200], both[200:]), (wg, wide[:, :264])):
        again = train(x, a, b, wd, dy, "silu")
        assert all(torch.equal(first[k], again[k]) for k in first)
    assert torch.equal(atb.feed_forward(x[:9], wg, wu, wd), atb.feed_forward(x[:9], wg, wide[:, :264], wd))


@pytest.mark.parametrize("M", [7, 200])
def test_rows_that_are_not_finite_stay_alone(M):
    x, wg, wu, wd, dy = make(M, 136, 264, 5)
    want = reference(x, wg, wu, wd, None, "silu")["y"]
    x = x.clone()
    x[3, 135] = float("nan")
    x[5, 0] = float("inf")
    for y in (atb.feed_forward(x, wg, wu, wd), atb.feed_forward(x, wg, wu, wd, save=True)[0]):
        assert not y[[3, 5]].isfinite().any()
        rows = [i for i in range(M) if i not in (3, 5)]
        close({"y": y[rows]}, {"y": (want[0][rows], want[1][rows])})


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_large_gates(act):
    """Far out both ways: the activation is 0 or the identity, its derivative 0 or 1, and nothing is NaN."""
    x, wg, wu, wd, dy = make(40, 64, 72, 6, scale=6.0)
    x = x * 8
    got, want = train(x, wg, wu, wd, dy, act), reference(x, wg, wu, wd, dy, act)
    for name in got:
        assert got[name].isfinite().all()
        assert float((got[name].double() - want[name][0]).norm()) <= 2 * R * float(want[name][0].norm()), name


def test_no_tokens():
    x, wg, wu, wd, dy = make(4, 72, 136, 7)
    got = train(x[:0], wg, wu, wd, dy[:0], "silu")
    assert got["y"].shape == got["dx"].shape == (0, 72)
    assert got["dwg"].shape == (136, 72) and got["dwd"].shape == (72, 136)
    assert not any(got[k].any() for k in ("dwg", "dwu", "dwd"))


def test_same_bits_every_time_and_on_another_stream():
    x, wg, wu, wd, dy = make(700, 520, 1032, 8)
    first = train(x, wg, wu, wd, dy, "silu")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = train(x, wg, wu, wd, dy, "silu", stream=side)
    side.synchronize()
    assert all(torch.equal(first[k], again[k]) for k in first)


def test_only_the_gradients_that_are_asked_for():
    """The C entry point with dx, or the weights' gradients, left out."""
    import ctypes
    x, wg, wu, wd, dy = make(90, 72, 136, 9)
    y, state = atb.feed_forward(x, wg, wu, wd, save=True)
    all_of = train(x, wg, wu, wd, dy, "silu")
    L = atb.lib()
    f = atb.Ffn(x.data_ptr(), wg.data_ptr(), wu.data_ptr(), wd.data_ptr(), 72, 72, 72, 136, 90, 72, 136, 0)
    dg, du = torch.empty_like(state.h), torch.empty_like(state.h)
    out = {"dx": torch.zeros_like(x), "dwg": torch.zeros_like(wg), "dwu": torch.zeros_like(wu), "dwd": torch.zeros_like(wd)}
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    for asked in (("dx",), ("dwg", "dwu"), ("dwd",), ("dx", "dwd")):
        for t in out.values():
            t.zero_()
        ptr = {k: t.data_ptr() if k in asked else None for k, t in out.items()}
        assert L.atb_ffn_backward(ctypes.byref(f), state.h.data_ptr(), state.kept.data_ptr(), dy.data_ptr(), 72, dg.data_ptr(), du.data_ptr(), ptr["dx"], 72, ptr["dwg"], ptr["dwu"],
                                  ptr["dwd"], stream) == 0
        for k, t in out.items():
            assert torch.equal(t, all_of[k]) if k in asked else not t.any(), (asked, k)


# few tiles and a long reduction, in each of the products: shares of it are summed apart and joined; shares of unequal length, one that ends in the other segment of dx, a
# last K-step that is not whole
@pytest.mark.parametrize("M,D,F", [(1, 1024, 2048), (33, 1032, 1544), (64, 2056, 520), (129, 520, 4104), (2000, 136, 72), (1337, 72, 200), (257, 264, 7176), (3500, 200, 264)])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_reductions_in_shares(M, D, F, act):
    assert atb.lib().atb_ffn_backward_workspace(M, D, F) > 0
    x, wg, wu, wd, dy = make(M, D, F, seed=M + D + F, pad=8)
    want = reference(x, wg, wu, wd, dy, act)
    first = train(x, wg, wu, wd, dy, act)
    close(first, want)
    close({"y": atb.feed_forward(x, wg, wu, wd, act)}, {"y": want["y"]})
    again = train(x, wg, wu, wd, dy, act)
    assert all(torch.equal(first[k], again[k]) for k in first)


# the same with enough rows for the large tiles: y and dx; the gradient of the down projection; dh
@pytest.mark.parametrize("M,D,F", [(2600, 2056, 3592), (3600, 2056, 3080), (2600, 3592, 2056)])
def test_reductions_in_shares_of_large_tiles(M, D, F):
    x, wg, wu, wd, dy = make(M, D, F, seed=M + D + F, scale=0.02)
    want = reference(x, wg, wu, wd, dy, "silu")
    first = train(x, wg, wu, wd, dy, "silu")
    close(first, want)
    again = train(x, wg, wu, wd, dy, "silu")
    assert all(torch.equal(first[k], again[k]) for k in first)


def test_without_a_workspace():
    """The C entry points without room for shares: the same products in one run each."""
    import ctypes
    M, D, F = 100, 1032, 1544
    x, wg, wu, wd, dy = make(M, D, F, 10)
    want = reference(x, wg, wu, wd, dy, "silu")
    f = atb.Ffn(x.data_ptr(), wg.data_ptr(), wu.data_ptr(), wd.data_ptr(), D, D, D, F, M, D, F, 0)
    new = lambda rows, cols: torch.full((rows, cols), float("nan"), dtype=torch.bfloat16, device="cuda")
    h, y, kept = new(M, F), new(M, D), torch.empty(6 * M * F, dtype=torch.uint8, device="cuda")
    dg, du, out = new(M, F), new(M, F), {"dx": new(M, D), "dwg": new(F, D), "dwu": new(F, D), "dwd": new(D, F)}
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert atb.lib().atb_ffn_forward(ctypes.byref(f), h.data_ptr(), kept.data_ptr(), y.data_ptr(), D, stream) == 0
    assert atb.lib().atb_ffn_backward(ctypes.byref(f), h.data_ptr(), kept.data_ptr(), dy.data_ptr(), D, dg.data_ptr(), du.data_ptr(), out["dx"].data_ptr(), D,
                                      out["dwg"].data_ptr(), out["dwu"].data_ptr(), out["dwd"].data_ptr(), stream) == 0
    close({"y": y, **out}, want)


def test_shares_of_rows_that_are_not_finite():
    x, wg, wu, wd, dy = make(70, 1032, 1544, 11)
    want = reference(x, wg, wu, wd, None, "silu")["y"]
    x = x.clone()
    x[3, 1031] = float("nan")
    y = atb.feed_forward(x, wg, wu, wd)
    rows = [i for i in range(70) if i != 3]
    assert not y[3].isfinite().any()
    close({"y": y[rows]}, {"y": (want[0][rows], want[1][rows])})


def test_without_a_workspace_where_it_would_hold_shares_of_large_tiles():
    """The C entry points without room for shares, at a size whose y and dx are large tiles in shares with it."""
    import ctypes
    M, D, F = 2600, 2056, 3592
    x, wg, wu, wd, dy = make(M, D, F, 12, scale=0.02)
    want = reference(x, wg, wu, wd, dy, "silu")
    f = atb.Ffn(x.data_ptr(), wg.data_ptr(), wu.data_ptr(), wd.data_ptr(), D, D, D, F, M, D, F, 0)
    new = lambda rows, cols: torch.full((rows, cols), float("nan"), dtype=torch.bfloat16, device="cuda")
    h, y, kept = new(M, F), new(M, D), torch.empty(6 * M * F, dtype=torch.uint8, device="cuda")
    dg, du, out = new(M, F), new(M, F), {"dx": new(M, D), "dwg": new(F, D), "dwu": new(F, D), "dwd": new(D, F)}
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert atb.lib().atb_ffn_forward(ctypes.byref(f), h.data_ptr(), kept.data_ptr(), y.data_ptr(), D, stream) == 0
    assert atb.lib().atb_ffn_backward(ctypes.byref(f), h.data_ptr(), kept.data_ptr(), dy.data_ptr(), D, dg.data_ptr(), du.data_ptr(), out["dx"].data_ptr(), D,
                                      out["dwg"].data_ptr(), out["dwu"].data_ptr(), out["dwd"].data_ptr(), stream) == 0
    close({"y": y, **out}, want)


def test_the_operators_are_not_part_of_autograd():
    """Operands that require gradients give the same results, which require none: the backward passes are calls of their own."""
    x, wg, wu, wd, _ = make(40, 72, 136, 13)
    n = atb.layer_norm(x, wg[0].contiguous())
    y = atb.feed_forward(n, wg, wu, wd)
    asked = [t.clone().requires_grad_() for t in (x, wg, wu, wd)]
    again = atb.layer_norm(asked[0], asked[1][0].contiguous())
    assert torch.equal(again, n) and not again.requires_grad
    z = atb.feed_forward(n, *asked[1:])
    assert torch.equal(y, z) and not z.requires_grad
