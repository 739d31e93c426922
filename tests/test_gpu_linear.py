"""A product with its epilogue and its gradients on the GPU against the formulas in 64 bits.

Tolerances.  fp32 sums of K products in MFMA accumulators err by less than 2^-15 of the sum of the products' sizes at these K; the activations add 2^-19 of their size and 2^-21
absolutely; the kept slope is fp16, 2^-11 of it or 2^-25; roundings to bf16 are at most 2^-8 of a value: of dz ahead of its products, and of the results.  The bias's gradient is a sum in chains of
at most 512 and 80 additions, 2^-14 of the sum of the sizes.  An error of an operand goes through a product with the sizes of the other."""
import ctypes

import pytest
import torch

import paper_2511_16041_amd as atb
from test_gpu_ffn import activation

pytestmark = pytest.mark.gpu
S, R = 2.0 ** -15, 2.0 ** -8
BF16, F32 = torch.bfloat16, torch.float32


def make(M, N, K, seed, pad=0, bias=BF16, residual=True, odd=0):
    """Operands whose rows are `pad` (a multiple of 8) further apart than they are long; the residual and dy by `odd`, any number.  What lies between rows is NaN."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def matrix(rows, cols, s, apart):
        t = (s * torch.randn((rows, cols + apart), generator=gen, device="cuda")).bfloat16()
        t[:, cols:] = float("nan")
        return t[:, :cols]
    x, w = matrix(M, K, 1.0, pad), matrix(N, K, 0.1, pad)
    b = (0.5 * torch.randn(N, generator=gen, device="cuda")).to(bias) if bias else None
    return x, w, b, matrix(M, N, 1.0, odd) if residual else None, matrix(M, N, 0.1, odd)


def reference(x, w, b, res, dy, act):
    """{name: (value in 64 bits, tolerance but for the result's own rounding)}"""
    x, w, dy = x.double(), w.double(), dy.double()
    bias = b.double() if b is not None else torch.zeros(w.shape[0], dtype=torch.float64, device=x.device)
    z = x @ w.t() + bias
    e_z = S * (x.abs() @ w.abs().t()) + 2.0 ** -23 * (z.abs() + bias.abs())
    a, slope = activation(act, z) if act else (z, torch.ones_like(z))
    e_a, e_slope = (1.2 * e_z + 2.0 ** -19 * a.abs() + 2.0 ** -21, 1.2 * e_z + 2.0 ** -19 + 2.0 ** -11 * slope.abs() + 2.0 ** -25) if act else (e_z, 0 * e_z)
    y = a + res.double() if res is not None else a
    dz = dy * slope
    e_dz = dy.abs() * e_slope + 2.0 ** -24 * dz.abs()
    e_op = e_dz + (R * dz.abs() if act else 0)                  # as an operand of the products
    return {"y": (y, e_a + 2.0 ** -23 * (a.abs() + y.abs())), "slope": (slope, e_slope),
            "dx": (dz @ w, e_op @ w.abs() + S * (dz.abs() @ w.abs())), "dw": (dz.t() @ x, e_op.t() @ x.abs() + S * (dz.abs().t() @ x.abs())),
            "db": (dz.sum(0), (e_dz + 2.0 ** -14 * dz.abs()).sum(0))}


ROUNDING = {BF16: R, F32: 2.0 ** -24, torch.float16: 2.0 ** -11}


def close(got, want):
    for name, t in got.items():
        if t is None:
            continue
        ref, tol = want[name]
        assert t.shape == ref.shape, name
        limit = tol + ROUNDING[t.dtype] * ref.abs() + 1e-30
        off = (t.double() - ref).abs()
        assert bool((off <= limit).all()), f"{name}: worst {float((off / limit).max())} of the tolerance"
        # and without a few wrong elements in a large tolerance: two roundings to bf16, each at most 2^-8 / sqrt 3, in the 2-norm
        if ref.numel() > 64 and float(ref.norm()) > 0:
            assert float((t.double() - ref).norm()) <= 1.5 * R * float(ref.norm()), name


def train(x, w, b, res, dy, act, stream=None):
    y, slope = atb.linear(x, w, b, act, res, save=True, stream=stream)
    dx, dw, db = atb.linear_backward(dy, x, w, b, slope, stream=stream)
    return {"y": y, "slope": slope[:, :w.shape[0]] if slope is not None else None, "dx": dx, "dw": dw, "db": db}


# one to a few tiles of either size, ends of tiles and of K-steps on both sides, odd N; long reductions of few tiles (shares); enough tiles for the large ones
SIZES = [(1, 1, 8), (2, 64, 64), (3, 7, 72), (16, 129, 256), (17, 333, 200), (32, 1000, 64), (33, 263, 136), (65, 71, 520), (130, 521, 264), (257, 767, 512), (300, 1001, 1032),
         (70, 4001, 4104), (40, 37, 8200), (1000, 9, 8), (2100, 3081, 136), (3001, 4099, 72), (2600, 2057, 3592),
         (1100, 3841, 520), (2040, 4096, 200),                  # (in tiles of 128 x 256)
         (1000, 1011, 16392), (700, 3001, 1544)]                # (both products of the backward pass in one launch, of tiles of 256 x 256 and of 128 x 128)


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("act", [None, "silu", "gelu", "gelu_tanh"])
def test_forward_and_backward(M, N, K, act):
    x, w, b, res, dy = make(M, N, K, seed=M + N + K)
    want = reference(x, w, b, res, dy, act)
    got = train(x, w, b, res, dy, act)
    assert (got["slope"] is None) == (act is None)
    close(got, want)
    close({"y": atb.linear(x, w, b, act, res)}, want)


@pytest.mark.parametrize("M,N,K", [(5, 40, 64), (5, 41, 64), (200, 264, 136), (200, 259, 136)])
@pytest.mark.parametrize("bias", [None, F32])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("act", [None, "gelu"])
def test_without_bias_or_residual_and_with_a_bias_in_fp32(M, N, K, bias, residual, act):
    x, w, b, res, dy = make(M, N, K, 3, bias=bias, residual=residual)
    want, got = reference(x, w, b, res, dy, act), train(x, w, b, res, dy, act)
    assert got["db"] is None if bias is None else got["db"].dtype == F32
    close(got, want)
    close({"y": atb.linear(x, w, b, act, res)}, want)


@pytest.mark.parametrize("M,N,K,pad,odd", [(5, 136, 72, 8, 3), (140, 203, 328, 24, 1), (300, 264, 136, 64, 8), (33, 131, 520, 8, 5)])
@pytest.mark.parametrize("act", [None, "silu"])
def test_rows_further_apart(M, N, K, pad, odd, act):
    x, w, b, res, dy = make(M, N, K, 4, pad, odd=odd if act or N % 8 else 8)
    want = reference(x, w, b, res, dy, act)
    close(train(x, w, b, res, dy, act), want)
    close({"y": atb.linear(x, w, b, act, res)}, want)


def test_operands_that_begin_at_any_element():
    """The residual and dy from the second element of a buffer on."""
    M, N, K = 150, 131, 264
    x, w, b, res, dy = make(M, N, K, 5)
    want = train(x, w, b, res, dy, "silu")
    moved = [torch.cat((t.new_zeros(1), t.reshape(-1)))[1:].view(M, N) for t in (res, dy)]
    assert moved[0].data_ptr() % 4 == 2
    got = train(x, w, b, *moved, "silu")
    assert all(torch.equal(got[k], want[k]) for k in got)


@pytest.mark.parametrize("M,N,K", [(7, 136, 264), (200, 135, 264), (70, 40, 4104)])
def test_what_is_not_finite_stays_in_its_rows_and_columns(M, N, K):
    x, w, b, res, dy = make(M, N, K, 6)
    want = reference(x, w, b, res, dy, "silu")
    x, res, b, dy = x.clone(), res.clone(), b.clone(), dy.clone()
    x[3, K - 1] = float("nan")
    res[5, 2] = float("inf")
    b[N - 1] = float("nan")
    rows, cols = [i for i in range(M) if i != 3], list(range(N - 1))
    for y in (atb.linear(x, w, b, "silu", res), atb.linear(x, w, b, "silu", res, save=True)[0]):
        assert not y[3].isfinite().any() and y[5, 2] == float("inf") and not y[:, N - 1].isfinite().any()
        y = y.clone()
        y[5, 2] = want["y"][0][5, 2].to(BF16)
        close({"y": y[rows][:, cols]}, {"y": tuple(t[rows][:, cols] for t in want["y"])})
    # a row of dy reaches its own row of dx; a column of it its own row of dw
    x, w, b, res, dy = make(M, N, K, 6)
    slope = atb.linear(x, w, b, "silu", res, save=True)[1]
    dy[4, N - 1] = float("nan")
    dx, dw, db = atb.linear_backward(dy, x, w, b, slope)
    assert dx[4].isnan().all() and dw[N - 1].isnan().all() and db[N - 1].isnan()
    rows = [i for i in range(M) if i != 4]
    close({"dx": dx[rows]}, {"dx": tuple(t[rows] for t in want["dx"])})
    close({"dw": dw[:-1], "db": db[:-1]}, {k: tuple(t[:-1] for t in want[k]) for k in ("dw", "db")})


@pytest.mark.parametrize("N", [72, 71])
def test_no_tokens(N):
    x, w, b, res, dy = make(4, N, 136, 7)
    for act in (None, "silu"):
        got = train(x[:0], w, b, res[:0], dy[:0], act)
        assert got["y"].shape == (0, N) and got["dx"].shape == (0, 136)
        assert got["dw"].shape == (N, 136) and not got["dw"].any() and not got["db"].any()


def test_same_bits_every_time_and_on_another_stream():
    x, w, b, res, dy = make(700, 1031, 520, 8)
    first = train(x, w, b, res, dy, "silu")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = train(x, w, b, res, dy, "silu", stream=side)
    side.synchronize()
    assert all(torch.equal(first[k], again[k]) for k in first)


def test_captured_and_replayed():
    """Forward and backward pass in a graph, replayed with new inputs and work of other calls in between."""
    args = make(100, 1032, 520, 9)
    static = [t.clone() for t in args]
    train(*static, "gelu")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = train(*static, "gelu")
    for seed in (9, 10, 11):
        new = make(100, 1032, 520, seed)
        for a, c in zip(static, new):
            a.copy_(c)
        graph.replay()
        eager = train(*new, "gelu")
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], eager[k]) for k in out), seed


def c_struct(x, w, b, act, work=None):
    return atb.Linear(x.data_ptr(), w.data_ptr(), x.stride(0), w.stride(0), b.data_ptr(), x.shape[0], w.shape[0], w.shape[1], act, 0 if b.dtype == BF16 else 1,
                      work.data_ptr() if work is not None else None)


def test_only_the_gradients_that_are_asked_for():
    """The C entry point with some of the gradients left out, and the residual in y's place."""
    M, N, K = 90, 131, 136
    x, w, b, res, dy = make(M, N, K, 12)
    all_of, slope = train(x, w, b, res, dy, "silu"), atb.linear(x, w, b, "silu", res, save=True)[1]
    L, stream = atb.lib(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    work = torch.empty(L.atb_linear_backward_workspace(M, N, K, 0), dtype=torch.uint8, device="cuda")
    l = c_struct(x, w, b, 0, work)
    out = {"dx": torch.zeros_like(x), "dw": torch.zeros_like(w), "db": torch.zeros_like(b)}
    for asked in (("dx",), ("dw",), ("db",), ("dx", "db"), ()):
        for t in out.values():
            t.zero_()
        ptr = {k: t.data_ptr() if k in asked else None for k, t in out.items()}
        assert L.atb_linear_backward(ctypes.byref(l), slope.data_ptr(), dy.data_ptr(), N, ptr["dx"], K, ptr["dw"], ptr["db"], stream) == 0
        for k, t in out.items():
            assert torch.equal(t, all_of[k]) if k in asked else not t.any(), (asked, k)
    y = res.clone()
    assert L.atb_linear_forward(ctypes.byref(l), y.data_ptr(), N, None, y.data_ptr(), N, stream) == 0
    close({"y": y}, reference(x, w, b, res, dy, "silu"))


def test_without_a_workspace():
    """A forward pass whose reduction would be shared out, without room for the shares."""
    M, N, K = 100, 131, 4104
    x, w, b, res, dy = make(M, N, K, 13)
    L, stream = atb.lib(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert L.atb_linear_workspace(M, N, K) > 0
    l, y = c_struct(x, w, b, 2), torch.empty_like(res)
    assert L.atb_linear_forward(ctypes.byref(l), res.data_ptr(), N, None, y.data_ptr(), N, stream) == 0
    close({"y": y}, reference(x, w, b, res, dy, "gelu_tanh"))


def test_results_beyond_32_bit_offsets():
    """2.2e9 elements of y, residual, slope and dz; rows at the ends against the formulas."""
    M, N, K = 1100003, 2001, 8
    gen = torch.Generator(device="cuda").manual_seed(14)
    x = torch.randn((M, K), generator=gen, device="cuda").bfloat16()
    w = (0.3 * torch.randn((N, K), generator=gen, device="cuda")).bfloat16()
    res = torch.zeros((M, N), dtype=BF16, device="cuda")
    res[-1] = 1.0
    y, slope = atb.linear(x, w, None, "silu", res, save=True)
    rows = [0, 1, 1073000, M - 2, M - 1]                       # (row 1073000 begins behind 2^31 elements)
    dy = res
    dy[rows] = 0.1
    dx, dw, _ = atb.linear_backward(dy, x, w, None, slope)
    r = torch.zeros((5, N), dtype=BF16, device="cuda")
    r[4] = 1.0
    want = reference(x[rows], w, None, r, dy[rows], "silu")
    close({"y": y[rows], "slope": slope[rows][:, :N], "dx": dx[rows], "dw": dw}, want)
    assert not dx[2:1000].any()


def test_gradients_against_differences():
    """The kernel's own forward pass, moved both ways along a direction of x, w and the bias, in the 2-norm's sense: the differences of results that are rounded to bf16."""
    M, N, K, h = 64, 136, 128, 2.0 ** -3
    x, w, b, _, dy = make(M, N, K, 15, bias=F32, residual=False)
    got = train(x, w, b, None, dy, "gelu_tanh")
    gen = torch.Generator(device="cuda").manual_seed(16)
    for grad, at, step in (("dx", 0, 0.25), ("dw", 1, 0.02), ("db", 2, 0.25)):
        args = [x, w, b]
        v = (step * torch.randn(args[at].shape, generator=gen, device="cuda")).to(args[at].dtype)
        ends = [(args[at].double() + s * h * v.double()).to(args[at].dtype) for s in (1, -1)]       # as they are after rounding
        losses, size = [], 0.0
        for t in ends:
            args[at] = t
            y = atb.linear(*args, "gelu_tanh").double()
            losses.append(float((y * dy.double()).sum()))
            size = max(size, float((y * dy.double()).norm()))
        want = float((got[grad].double() * (ends[0].double() - ends[1].double())).sum())
        # roundings of y: independent, at most 2^-8 of each, six deviations of 2^-8 / sqrt 3; the gradient's own two roundings; the third derivative (below 2 for this activation) of a move of z by
        # 0.125 * 0.25 * sqrt(128) * 0.1 .. 0.04 * sqrt(128) < 0.4: 0.4^3 / 3 of |dy| each, in random signs
        limit = 2 * 6 * R / 3 ** 0.5 * size + 2 * R * float((got[grad].double() * (ends[0].double() - ends[1].double())).norm()) * 6 + 6 * 0.03 * float(dy.double().norm())
        assert abs(losses[0] - losses[1] - want) <= limit, (grad, losses[0] - losses[1], want, limit)


def test_gradients_against_differences_along_themselves():
    """The same with the operands moved along their gradients, where the loss moves most: by so much that no z moves by more than an eighth either way."""
    M, N, K = 64, 136, 128
    x, w, b, _, dy = make(M, N, K, 17, bias=F32, residual=False)
    got = train(x, w, b, None, dy, "gelu_tanh")
    dx, dw, db = (got[k].double() for k in ("dx", "dw", "db"))
    moves = {"dx": dx @ w.double().t(), "dw": x.double() @ dw.t(), "db": db.expand(M, N)}          # of z, along each
    for grad, at in (("dx", 0), ("dw", 1), ("db", 2)):
        args, v = [x, w, b], got[grad].double() * (0.125 / float(moves[grad].abs().max()))
        ends = [(args[at].double() + s * v).to(args[at].dtype) for s in (1, -1)]                    # as they are after rounding
        losses, size = [], 0.0
        for t in ends:
            args[at] = t
            y = atb.linear(*args, "gelu_tanh").double()
            losses.append(float((y * dy.double()).sum()))
            size = max(size, float((y * dy.double()).norm()))
        want = float((got[grad].double() * (ends[0].double() - ends[1].double())).sum())
        # six deviations of y's roundings, independent; 2^-7 of the slope itself (its two roundings, in the 2-norm); the third derivative, below 2: 2 / 3 of an eighth cubed of |dy|
        limit = 6 * 2 ** 0.5 * R / 3 ** 0.5 * size + 2 * R * abs(want) + 2 / 3 * 0.125 ** 3 * float(dy.double().abs().sum())
        assert abs(losses[0] - losses[1] - want) <= limit, (grad, losses[0] - losses[1], want, limit)


def difference(args, at, grad, dy, act, h, forward):
    """Loss = sum of y dy: (its difference between the two ends of a move of operand `at` along its gradient, both ways by so much that no z moves by more than h; what the gradient makes of that; what they may be apart)"""
    x, w = args[0].double(), args[1].double()
    g = grad.double()

    def z_of(v):
        return v @ w.t() if at == 0 else x @ v.t() if at == 1 else v.expand(dy.shape)
    v = g * (h / float(z_of(g).abs().max()))
    ends = [(args[at].double() + s * v).to(args[at].dtype) for s in (1, -1)]                       # as they are after rounding
    moved, shift = (z_of(t) for t in ((ends[0].double() - ends[1].double()) / 2, (ends[0].double() + ends[1].double()) / 2 - args[at].double()))
    y = [forward(*args[:at], t, *args[at + 1:], act).double() for t in ends]
    size = max(float((t * dy.double()).norm()) for t in y)
    want, weight = float((g * (ends[0].double() - ends[1].double())).sum()), dy.double().abs()
    # six deviations of y's roundings, independent of each other, of both ends; the gradient's own two roundings in the 2-norm; the third derivative, below 2, and the second, below 1.2, where rounding has moved the middle
    limit = 6 * 2 ** 0.5 * R / 3 ** 0.5 * size + 2 * R * abs(want)
    if act:
        limit += 2 / 3 * float((weight * moved.abs() ** 3).sum()) + 2 * 1.2 * float((weight * moved.abs() * shift.abs()).sum())
    return float((y[0] * dy.double()).sum() - (y[1] * dy.double()).sum()), want, limit


@pytest.mark.parametrize("M,N,K", [(24, 136, 128), (64, 137, 128), (200, 264, 136)])
@pytest.mark.parametrize("act", [None, "silu", "gelu", "gelu_tanh"])
def test_gradients_against_differences_that_tell_them_from_wrong_ones(M, N, K, act):
    """Along each gradient the loss moves by ten times what the difference may be off or more, so one that is zero, half as large or of the other sign is not taken."""
    x, w, b, _, dy = make(M, N, K, 18, bias=F32, residual=False)
    got = train(x, w, b, None, dy, act)
    for name, at in (("dx", 0), ("dw", 1), ("db", 2)):
        moved, want, limit = difference([x, w, b], at, got[name], dy, act, 0.125, atb.linear)
        assert abs(moved - want) <= limit, (name, moved, want, limit)
        assert abs(moved) > 10 * limit and abs(moved - 0.5 * want) > limit and abs(moved + want) > limit, (name, moved, want, limit)


@pytest.mark.parametrize("M", [5, 33, 300])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_the_kept_slope_where_the_activation_is_flat(M, act):
    """z from 5 to 40 on both sides: the slope is off by 2^-11 of itself or by 2^-25, what is more.  Beside it, 2^-15 of it for an exponential whose argument of up to 100 is rounded in fp32 (100 * 2^-24 * log2 e, and as
    much of its result), and 2^-30 for the distribution function's polynomial, 1.6e-3 of 2.9e-7 at -5."""
    N = 72
    z = torch.cat((torch.linspace(-40, -5, M * N // 2 + 1), torch.linspace(5, 40, M * N // 2 + 1)))[:M * N].reshape(M, N).bfloat16().cuda()
    x = torch.zeros((M, 8 * ((M + 7) // 8)), dtype=BF16, device="cuda")
    x[torch.arange(M), torch.arange(M)] = 1.0                  # row m of x picks column m of w: z[m, n] = w[n, m], exactly
    w = torch.zeros((N, x.shape[1]), dtype=BF16, device="cuda")
    w[:, :M] = z.t()
    slope = atb.linear(x, w, None, act, save=True)[1][:, :N].double()
    want = activation(act, z.double())[1]
    limit = torch.maximum(2.0 ** -11 * want.abs(), torch.tensor(2.0 ** -25, dtype=torch.float64, device="cuda")) + 2.0 ** -15 * want.abs() + 2.0 ** -30
    assert bool(((slope - want).abs() <= limit).all()), float(((slope - want).abs() / limit).max())
