"""A mixture of experts for few tokens on the GPU against its definition in 64 bits.

Tolerances.  Which experts a token takes is exact: the router's products are summed in fp64 on both sides, and no two of the random ones here are as near as 2^-40.  The shares come from fp32
exponentials and a sum of at most 256: 2^-19 of each and of the differences of the l's.  The products' fp32 sums err by less than S = 2^-15 of the sum of the terms' sizes; of 4-bit weights, whose
accumulators sum (16 + q) x and take (16 + z) x off again, by 2^-20 of 143 s |x| beside.  The inner activations are rounded to bf16, at most 2^-8 of them, as the result is."""
import ctypes

import pytest
import torch

import paper_2511_16041_amd as atb
from test_gpu_ffn import activation
from test_gpu_q4 import random_weight, steps, values

pytestmark = pytest.mark.gpu
S, E4, R = 2.0 ** -15, 2.0 ** -20, 2.0 ** -8
BF16 = torch.bfloat16


def make(M, E, D, F, seed, group=0, zeros=False, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def matrix(rows, cols, s):
        t = (s * torch.randn((rows, cols + pad), generator=g, device="cuda")).bfloat16()
        t[:, cols:] = float("nan")
        return t[:, :cols]
    x, router = matrix(M, D, 1.0), matrix(E, D, D ** -0.5)
    if group:
        return x, router, random_weight(E * F, D, group, zeros, seed + 1), random_weight(E * F, D, group, zeros, seed + 2), random_weight(E * D, F, group, zeros, seed + 3)
    return (x, router) + tuple((0.05 * torch.randn((E, n, k), generator=g, device="cuda")).bfloat16() for n, k in ((F, D), (F, D), (D, F)))


def routing(x, router, k, renormalize):
    """(experts, shares, what these may be off)"""
    l = x.double() @ router.double().t()
    experts = torch.sort(l.nan_to_num(nan=-float("inf"), posinf=float("inf"), neginf=-float("inf")), dim=1, descending=True, stable=True).indices[:, :k]
    taken = torch.gather(l, 1, experts)
    p = torch.softmax(taken, 1) if renormalize else torch.gather(torch.softmax(l, 1), 1, experts)
    return experts, p, 2.0 ** -19 * p * (1 + (taken - l.amax(1, keepdim=True)).abs())


def of_expert(w, e, n):
    """(values, what a term of a product with each may add to the error of the product beside S of its size)"""
    if isinstance(w, tuple):
        part = atb.Q4Weight(*(t[e * n:(e + 1) * n] if t is not None else None for t in w))
        return values(part), E4 * 143 * steps(part)
    v = w[e].double()
    return v, 0 * v


def reference(x, router, wg, wu, wd, k, act, renormalize):
    """(y, what it may be off but for its own rounding, experts, shares, what they may be off)"""
    M, D = x.shape
    F = (wd[0].shape[1] * 2 if isinstance(wd, tuple) else wd.shape[2])
    experts, p, e_p = routing(x, router, k, renormalize)
    y, tol = torch.zeros((M, D), dtype=torch.float64, device=x.device), torch.zeros((M, D), dtype=torch.float64, device=x.device)
    for e in sorted(set(experts.flatten().tolist())):
        tokens, choice = torch.nonzero(experts == e, as_tuple=True)
        rows = x[tokens].double()
        (g_w, g_e), (u_w, u_e), (d_w, d_e) = of_expert(wg, e, F), of_expert(wu, e, F), of_expert(wd, e, D)
        g, u = rows @ g_w.t(), rows @ u_w.t()
        e_g, e_u = rows.abs() @ (S * g_w.abs() + g_e).t(), rows.abs() @ (S * u_w.abs() + u_e).t()
        a, _ = activation(act, g)
        h = a * u
        e_a = 1.2 * e_g + 2.0 ** -19 * a.abs() + 2.0 ** -21
        e_h = e_a * u.abs() + a.abs() * e_u + e_a * e_u + R * h.abs()
        f, e_f = h @ d_w.t(), e_h @ d_w.abs().t() + h.abs() @ (S * d_w.abs() + d_e).t()
        share, e_share = p[tokens, choice].unsqueeze(1), e_p[tokens, choice].unsqueeze(1)
        y.index_add_(0, tokens, share * f)
        tol.index_add_(0, tokens, share * e_f + e_share * (f.abs() + e_f) + 2.0 ** -20 * (share * f).abs())
    return y, tol, experts, p, e_p


def check(args, k, act="silu", renormalize=True, rows=None, got=None):
    """rows: those that are compared"""
    want_y, tol, experts, p, e_p = reference(*args, k, act, renormalize)
    y, chosen, shares = got if got is not None else atb.moe_feed_forward(*args, k, act, renormalize, routing=True)
    assert y.dtype == BF16 and y.shape == args[0].shape and chosen.dtype == torch.int32 and shares.dtype == torch.float32
    rows = list(range(len(y))) if rows is None else rows
    assert torch.equal(chosen[rows].long(), experts[rows])
    assert bool(((shares.double() - p).abs() <= e_p + 2.0 ** -24 * p)[rows].all())
    limit, off = tol + R * want_y.abs() + 1e-30, (y.double() - want_y).abs()
    assert bool((off <= limit)[rows].all()), f"worst {float((off / limit)[rows].max())} of the tolerance"
    # and without a few wrong elements in a large tolerance: two roundings to bf16, each at most 2^-8 / sqrt 3, in the 2-norm
    if y[rows].numel() > 64 and not isinstance(args[2], tuple):
        assert float((y.double() - want_y)[rows].norm()) <= 1.5 * R * float(want_y[rows].norm())
    return y, chosen, shares


SIZES = [(1, 1, 1, 8, 8), (1, 4, 2, 64, 136), (2, 3, 3, 72, 64), (3, 8, 2, 200, 328), (5, 11, 3, 264, 1000), (8, 64, 8, 136, 72), (9, 7, 2, 520, 264), (16, 5, 1, 1032, 72), (17, 256, 16, 64, 40), (21, 60, 6, 264, 200),
         (33, 4, 4, 136, 520), (40, 3, 1, 328, 264), (64, 2, 2, 72, 136), (64, 64, 8, 200, 72), (64, 255, 2, 40, 64), (1, 8, 2, 4104, 1544), (30, 8, 2, 2056, 1032)]


@pytest.mark.parametrize("M,E,k,D,F", SIZES)
@pytest.mark.parametrize("act,renormalize", [("silu", True), ("gelu", False), ("gelu_tanh", True)])
def test_bf16(M, E, k, D, F, act, renormalize):
    args = make(M, E, D, F, M + E + D + F)
    first = check(args, k, act, renormalize)
    assert torch.equal(first[0], atb.moe_feed_forward(*args, k, act, renormalize))


@pytest.mark.parametrize("group,zeros", [(32, False), (32, True), (64, True), (64, False), (128, False), (128, True)])
@pytest.mark.parametrize("M,E,k,D,F", [(1, 1, 1, 1, 1), (1, 4, 2, 2, 5), (2, 3, 3, 3, 1), (5, 11, 3, 5, 7), (9, 7, 2, 1, 3), (16, 5, 2, 4, 9), (17, 20, 4, 3, 2), (33, 4, 4, 2, 3), (64, 30, 3, 2, 6), (64, 2, 1, 5, 2), (1, 8, 8, 17, 11)])
def test_weights_in_4_bits(M, E, k, D, F, group, zeros):
    args = make(M, E, D * group, F * group, M + E + D + F, group, zeros)
    check(args, k, "silu", k % 2 == 0)


@pytest.mark.parametrize("M", [3, 20, 64])
@pytest.mark.parametrize("group", [0, 32])
def test_all_tokens_choose_the_same_experts(M, group):
    x, router, *w = make(M, 9, 64, 96, 3, group)
    router = torch.zeros_like(router)
    router[7], router[2] = 1.0, 0.5
    x = x.abs()
    got = check((x, router, *w), 2)
    assert bool((got[1] == torch.tensor([7, 2], device="cuda")).all())


def test_of_equal_experts_the_lowest_comes_first():
    x, router, *w = make(6, 12, 64, 72, 4)
    router[3] = router[8] = router[5]
    router[0] = router[11]
    check((x, router, *w), 7)
    check((x, torch.zeros_like(router), *w), 5)               # all equal: experts 0 to 4
    assert bool((atb.moe_feed_forward(x, torch.zeros_like(router), *w, 5, routing=True)[1] == torch.arange(5, device="cuda")).all())


def test_experts_whose_products_lie_close_keep_their_order():
    """2^-9 beside 0.5 is half a step of bf16 and rounds to even, 0.5: experts 0 and 1 are equal; 2^-8 is a step, 2^-19 of the product."""
    D = 4096
    x = torch.ones((1, D), dtype=BF16, device="cuda")
    router = torch.full((3, D), 0.5, dtype=BF16, device="cuda")
    router[1, 17] = 0.5 + 2.0 ** -9
    router[2, 4000] = 0.5 + 2.0 ** -8
    assert float(router[1, 17]) == 0.5 < float(router[2, 4000])
    _, _, *w = make(1, 3, D, 64, 5)
    got = check((x, router, *w), 3)
    assert got[1].tolist() == [[2, 0, 1]]


def test_experts_whose_products_fp32_does_not_tell_apart_keep_their_order():
    """2^24 - 2^24 and 2^-10 of the expert's number: a sum in fp32 that meets the large terms first loses the small one."""
    D = 4096
    x = torch.ones((1, D), dtype=BF16, device="cuda")
    x[0, 0] = x[0, D - 1] = 2.0 ** 24
    router = torch.zeros((5, D), dtype=BF16, device="cuda")
    router[:, 0], router[:, D - 1] = 1.0, -1.0
    router[:, 5] = torch.arange(5, device="cuda") * 2.0 ** -10
    _, _, *w = make(1, 5, D, 64, 5)
    got = check((x * 1.0, router, *(t * 2.0 ** -24 for t in w[:1]), *w[1:]), 3)
    assert got[1].tolist() == [[4, 3, 2]]


@pytest.mark.parametrize("M", [4, 40])
@pytest.mark.parametrize("group", [0, 64])
def test_weights_of_experts_that_no_token_chose_are_not_used(M, group):
    args = make(M, 16, 128, 192, 6, group)
    router = args[1].clone()
    router[::3] = router[::3] * 0 - 0.5 * args[0].float().mean(0).sign().bfloat16()
    chosen = set(routing(args[0], router, 2, True)[0].flatten().tolist())
    assert len(chosen) < 16
    broken = []
    for w, n in ((args[2], 192), (args[3], 192), (args[4], 128)):
        rows = [e * n + i for e in range(16) if e not in chosen for i in range(n)]
        if group:
            scales = w.scales.clone()
            scales[rows] = float("nan")
            broken.append(w._replace(scales=scales))
        else:
            w = w.clone()
            w[[e for e in range(16) if e not in chosen]] = float("nan")
            broken.append(w)
    a = atb.moe_feed_forward(args[0], router, *args[2:], 2)
    assert torch.equal(a, atb.moe_feed_forward(args[0], router, *broken, 2)) and a.isfinite().all()


@pytest.mark.parametrize("M", [5, 20, 64])
@pytest.mark.parametrize("group", [0, 32])
def test_tokens_that_are_not_finite_stay_alone(M, group):
    """Whatever x holds, every token has top_k different experts; a NaN or an infinity makes its own row so."""
    args = make(M, 6, 96, 64, 7, group)
    x = args[0].clone()
    x[1, 95], x[3] = float("nan"), float("inf")
    x[4, 0] = float("-inf")
    y, chosen, shares = atb.moe_feed_forward(x, *args[1:], 3, routing=True)
    assert not y[[1, 3, 4]].isfinite().any()
    assert bool((chosen >= 0).all()) and bool((chosen < 6).all()) and all(len(set(row)) == 3 for row in chosen.tolist())
    assert chosen[1].tolist() == [0, 1, 2] and shares[1].isnan().all()
    check(args, 3, rows=[i for i in range(M) if i not in (1, 3, 4)], got=(y, chosen, shares))


def test_an_expert_that_is_not_finite_reaches_its_own_tokens_alone():
    args = make(30, 8, 136, 72, 8)
    _, chosen, _ = check(args, 2)
    wd, wg = args[4].clone(), args[2].clone()
    wd[3, 5, 71] = float("inf")
    wg[6, 0, 0] = float("nan")
    y = atb.moe_feed_forward(args[0], args[1], wg, args[3], wd, 2)
    struck = (chosen == 3).any(1) | (chosen == 6).any(1)
    assert struck.any() and not struck.all()
    check(args, 2, rows=torch.nonzero(~struck).flatten().tolist(), got=(y,) + atb.moe_feed_forward(*args, 2, routing=True)[1:])
    assert not y[struck].isfinite().all(1).any()


def test_rows_further_apart_and_no_tokens():
    args = make(13, 7, 136, 200, 9, pad=24)
    check(args, 3)
    y, chosen, shares = atb.moe_feed_forward(args[0][:0], *args[1:], 3, routing=True)
    assert y.shape == (0, 136) and chosen.shape == shares.shape == (0, 3)
    one = check((args[0][5:6],) + args[1:], 3)[0]             # a token's bits do not depend on the others in its segments of 8 rows or fewer
    assert torch.equal(one, atb.moe_feed_forward(args[0][5:6].clone(), *args[1:], 3))


def test_same_bits_every_time_on_another_stream_and_at_once():
    args, other = make(30, 12, 520, 264, 10), make(30, 12, 520, 264, 11)
    first, second = atb.moe_feed_forward(*args, 3), atb.moe_feed_forward(*other, 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(5):                                         # two calls at once have a workspace each
        a, b = atb.moe_feed_forward(*args, 3, stream=side), atb.moe_feed_forward(*other, 3)
        side.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(a, first) and torch.equal(b, second)


@pytest.mark.parametrize("group", [0, 64])
def test_captured_and_replayed(group):
    """The plan is made on the device: a replay with other tokens takes other experts."""
    args = make(6, 16, 128, 192, 12, group)
    x = args[0].clone()
    atb.moe_feed_forward(x, *args[1:], 3)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = atb.moe_feed_forward(x, *args[1:], 3, routing=True)
    seen = set()
    for seed in (12, 13, 14, 15):
        x.copy_(make(6, 16, 128, 192, seed, group)[0])
        graph.replay()
        check((x,) + args[1:], 3, got=out)
        eager = atb.moe_feed_forward(x, *args[1:], 3, routing=True)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager))
        seen.add(str(out[1].tolist()))
    assert len(seen) == 4


def test_weights_beyond_32_bit_offsets():
    """Experts that begin behind 2^32 bytes and 2^31 elements of their weight."""
    E, D, F = 70, 8192, 4096
    w = torch.zeros((E, F, D), dtype=BF16, device="cuda")
    assert w[64].data_ptr() - w.data_ptr() >= 1 << 32
    gen = torch.Generator(device="cuda").manual_seed(16)
    for e in (0, 69):
        w[e] = (0.02 * torch.randn((F, D), generator=gen, device="cuda")).bfloat16()
    wd = w.view(E, D, F)
    x = torch.randn((2, D), generator=gen, device="cuda").bfloat16()
    router = torch.zeros((E, D), dtype=BF16, device="cuda")
    router[69], router[0] = 0.01 * x[0], 0.01 * x[1]
    got = check((x, router, w, w, wd), 1)
    assert got[1].flatten().tolist() == [69, 0]


def test_through_the_c_entry_point():
    """Rows of y further apart, without the routing."""
    M, E, D, F, k = 11, 6, 136, 200, 2
    args = make(M, E, D, F, 17)
    want = atb.moe_feed_forward(*args, k)
    L, stream = atb.lib(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    y = torch.full((M, D + 3), 7.0, dtype=BF16, device="cuda")
    work = torch.empty(L.atb_moe_workspace(M, D, F, E, k, 0), dtype=torch.uint8, device="cuda")
    m = atb.Moe(args[0].data_ptr(), args[1].data_ptr(), D, D, *(atb.MoeWeight(w.data_ptr(), None, None) for w in args[2:]), M, D, F, E, k, 0, 0, 1, work.data_ptr())
    assert L.atb_moe_forward(ctypes.byref(m), y.data_ptr(), D + 3, None, None, stream) == 0
    assert torch.equal(y[:, :D], want) and bool((y[:, D:] == 7.0).all())


@pytest.mark.parametrize("M", [1, 2, 8, 30])
@pytest.mark.parametrize("E,group", [(12, 0), (12, 32), (70, 0), (200, 0)])
def test_a_product_that_is_no_number_is_behind_minus_infinity(M, E, group):
    """Experts with l = NaN, -infinity and numbers, by turns, NaN first: a token takes the numbers, then -infinity, whose share is 0, from the lowest index on, then NaN."""
    x, router, *w = make(M, E, 96, 64, E + M, group)
    x, router = x.abs(), router.clone()
    numbers = [E - 1, 5, 2] + ([E // 2] if E > 12 else [])
    for e in range(E):
        if e not in numbers:
            router[e, 7] = float("-inf") if e % 2 else float("nan")
    x[:, 7] = 1.0
    l = x.double() @ router.double().t()
    low = [e for e in range(E) if e not in numbers and e % 2]
    none = [e for e in range(E) if e not in numbers and e % 2 == 0]
    assert l[:, low].isneginf().all() and l[:, none].isnan().all() and l[:, numbers].isfinite().all()
    for k in (len(numbers) + 2, min(16, len(numbers) + len(low)), min(E, 16)):
        y, chosen, shares = atb.moe_feed_forward(x, router, *w, k, routing=True)
        n = len(numbers)
        want = (low + none)[:k - n]
        assert all(sorted(row[:n]) == sorted(numbers) and row[n:] == want for row in chosen.tolist()), (k, chosen[0].tolist())
        if len(low) >= k - n:
            assert not shares[:, n:].any()
            finite = torch.where(router.isfinite(), router, torch.full_like(router, -2.0 ** 20))         # (the others' l far below, for the formula)
            check((x, finite, *w), n, got=(y, chosen[:, :n], shares[:, :n]))
        else:
            assert shares.isnan().all() and y.isnan().all()


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group,D,F", [(32, 67, 33), (32, 33, 67), (64, 33, 41), (64, 41, 33), (128, 17, 19), (128, 33, 17)])
@pytest.mark.parametrize("M,E,k", [(8, 3, 2), (9, 3, 2), (17, 4, 1), (40, 3, 2), (64, 2, 1)])
def test_weights_in_4_bits_over_many_panels(M, E, k, group, D, F, zeros):
    """Reductions of 9 to 17 panels of 256, the last one cut, over four waves of the gate and up products and eight of the down product: a wave's second and third panel, and with more than 8 tokens the wide form.  Beside
    the tolerance of every element, the 2-norm: the inner activations' rounding to bf16 and the result's, each at most 2^-8 / sqrt 3 of their size, are independent of each other and of the weights; all else is
    2^-15 of it."""
    args = make(M, E, D * group, F * group, M + D + F, group, zeros)
    y, _, _ = check(args, k, "gelu_tanh", k == 2)
    want = reference(*args, k, "gelu_tanh", k == 2)[0]
    assert float((y.double() - want).norm()) <= 1.5 * R * float(want.norm())
