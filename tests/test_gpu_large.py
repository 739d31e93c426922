"""The feed-forward operators where operands, results and what is kept pass 2^32 bytes or 2^31 elements, and at the longest rows that are taken.  References in 64 bits, a
part of the rows or of the reduction at a time; tolerances as in test_gpu_ffn.py and test_gpu_q4.py."""
import pytest
import torch

import paper_2511_16041_amd as atb
import test_gpu_ffn as ffn
from test_gpu_q4 import E, check, random_weight, rows, steps, values

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    torch.cuda.empty_cache()


def test_gated_block_of_many_tokens():
    """What is kept: 12.9 GB, h and its like 4.3 GB each."""
    M, D, F = 2 ** 20 + 37, 8, 2056
    x, wg, wu, wd, dy = ffn.make(M, D, F, seed=1)
    x[65536:-65536] = 0                                   # the weights' gradients are sums over the others
    got = ffn.train(x, wg, wu, wd, dy, "silu")
    ends = torch.cat((torch.arange(65536, device="cuda"), torch.arange(M - 65536, M, device="cuda")))
    want = ffn.reference(x[ends], wg, wu, wd, dy[ends], "silu")
    ffn.close({"y": got["y"][ends], "dx": got["dx"][ends], **{k: got[k] for k in ("dwg", "dwu", "dwd")}}, want)
    assert not got["y"][65536:-65536].any() and not got["dx"][65536:-65536].any()


@pytest.mark.parametrize("M", [3, 40])
def test_gated_block_of_large_weights(M):
    """4.3 GB each; 2^21 inner activations are the down projection's reduction."""
    D, F = 1032, 2 ** 21
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((M, D), generator=gen, device="cuda").bfloat16()
    wg, wu, wd = (torch.empty(s, dtype=torch.bfloat16, device="cuda").normal_(0, 0.03, generator=gen) for s in ((F, D), (F, D), (D, F)))
    y = atb.feed_forward(x, wg, wu, wd, "silu")
    ref, tol = torch.zeros((M, D), dtype=torch.float64, device="cuda"), torch.zeros((M, D), dtype=torch.float64, device="cuda")
    for f in range(0, F, 2 ** 17):
        part = slice(f, f + 2 ** 17)
        r, t = ffn.reference(x, wg[part], wu[part], wd[:, part], None, "silu")["y"]
        ref += r
        tol += t
    ffn.close({"y": y}, {"y": (ref, tol)})


@pytest.mark.parametrize("M", [5, 40])
def test_gated_block_of_the_longest_rows(M):
    """D = 2^22 - 8: rows of x and of both weights 8 MiB apart, offsets in a tile up to 2^31."""
    D, F = 2 ** 22 - 8, 264
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, dy = (torch.empty((M, D), dtype=torch.bfloat16, device="cuda").normal_(0, s, generator=gen) for s in (1.0, 0.1))
    wg, wu, wd = (torch.empty(s, dtype=torch.bfloat16, device="cuda").normal_(0, 0.001, generator=gen) for s in ((F, D), (F, D), (D, F)))
    got = ffn.train(x, wg, wu, wd, dy, "silu")
    streamed = atb.feed_forward(x, wg, wu, wd, "silu")
    # g, u and dh are sums over D: in parts; then everything else is, part by part of D, the formulas
    g, u, dh = (torch.zeros((M, F), dtype=torch.float64, device="cuda") for _ in range(3))
    e_g, e_u, e_dh = (torch.zeros((M, F), dtype=torch.float64, device="cuda") for _ in range(3))
    parts = [slice(d, min(D, d + 2 ** 18)) for d in range(0, D, 2 ** 18)]
    for p in parts:
        xd, gd, ud, dd, od = x[:, p].double(), wg[:, p].double(), wu[:, p].double(), wd[p].double(), dy[:, p].double()
        g += xd @ gd.t(); u += xd @ ud.t(); dh += od @ dd
        e_g += ffn.S * (xd.abs() @ gd.abs().t()); e_u += ffn.S * (xd.abs() @ ud.abs().t()); e_dh += ffn.S * (od.abs() @ dd.abs())
    a, slope = ffn.activation("silu", g)
    h = a * u
    e_a = 1.2 * e_g + 2.0 ** -19 * a.abs() + 2.0 ** -21
    e_h = e_a * u.abs() + a.abs() * e_u + e_a * e_u + ffn.R * h.abs()
    dg, du = dh * u * slope, dh * a
    e_slope, e_u = 1.2 * e_g + 2.0 ** -19 + 2.0 ** -16 * g.abs(), e_u + 2.0 ** -15 * u.abs()
    e_dg = e_dh * (u * slope).abs() + dh.abs() * (e_u * slope.abs() + u.abs() * e_slope) + ffn.R * dg.abs() + e_dh * (e_u * slope.abs() + u.abs() * e_slope)
    e_du = e_dh * a.abs() + dh.abs() * (e_a + 2.0 ** -15 * (g * slope).abs()) + ffn.R * du.abs() + e_dh * e_a
    for p in (parts[0], parts[7], parts[-1]):
        xd, gd, ud, dd, od = x[:, p].double(), wg[:, p].double(), wu[:, p].double(), wd[p].double(), dy[:, p].double()
        y = (h @ dd.t(), e_h @ dd.abs().t() + ffn.S * (h.abs() @ dd.abs().t()))
        ffn.close({"y": got["y"][:, p], "dx": got["dx"][:, p], "dwg": got["dwg"][:, p], "dwu": got["dwu"][:, p], "dwd": got["dwd"][p]}, {
            "y": y, "dx": (dg @ gd + du @ ud, e_dg @ gd.abs() + e_du @ ud.abs() + ffn.S * (dg.abs() @ gd.abs() + du.abs() @ ud.abs())),
            "dwg": (dg.t() @ xd, (e_dg + ffn.S * dg.abs()).t() @ xd.abs()), "dwu": (du.t() @ xd, (e_du + ffn.S * du.abs()).t() @ xd.abs()),
            "dwd": (od.t() @ h, od.abs().t() @ (e_h + ffn.S * h.abs()))})
        ffn.close({"y": streamed[:, p]}, {"y": y})


@pytest.mark.parametrize("zeros", [False, True])
def test_4_bit_weights_of_many_outputs(zeros):
    """4.3 GB of codes; results of 2^31 elements and more."""
    N, K, M = 2 ** 22 + 5, 2080, 520
    w, x = random_weight(N, K, 32, zeros, 4), rows(M, K, 5)
    y = atb.q4_matvec(x, w)
    for first in (0, 2 ** 21 - 100, N - 300):
        part = slice(first, first + 300)
        q = atb.Q4Weight(w.packed[part], w.scales[part], w.zeros[part] if zeros else None)
        for m in (slice(0, 20), slice(M - 20, M)):
            check(y[m, part], x[m], q)


def test_4_bit_weights_of_the_longest_rows():
    N, K, M = 40, 2 ** 22, 18
    w, x = random_weight(N, K, 128, True, 6), rows(M, K, 7)
    y = atb.q4_matvec(x, w, torch.float32)
    ref, size = torch.zeros((M, N), dtype=torch.float64, device="cuda"), torch.zeros((M, N), dtype=torch.float64, device="cuda")
    for k in range(0, K, 2 ** 19):
        q = atb.Q4Weight(*(t[:, k // n:(k + 2 ** 19) // n].contiguous() for t, n in ((w.packed, 2), (w.scales, 128), (w.zeros, 128))))
        ref += x[:, k:k + 2 ** 19].double() @ values(q).t()
        size += x[:, k:k + 2 ** 19].double().abs() @ steps(q).t()
    off = (y.double() - ref).abs()
    assert bool((off <= E * 143 * size + E * ref.abs()).all())
