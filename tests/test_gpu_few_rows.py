"""Every kernel for few rows, just past the bounds of the rules that choose it, with several panels for every wave and a last panel that is cut: both buffers of a wave are
filled again.  References and tolerances are test_gpu_q4.py's and test_gpu_ffn.py's."""
import pytest
import torch

import paper_2511_16041_amd as atb
import test_gpu_ffn as ffn
from test_gpu_q4 import E, R, check, random_weight, rows, steps, values

pytestmark = pytest.mark.gpu
# groups along K, an odd number of them: of 16 waves the first have four panels of 256 and the others three; of 8 waves likewise
GROUPS = {16: {32: 405, 64: 203, 128: 101}, 8: {32: 203, 64: 101, 128: 51}}


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,waves", [(4096, 16), (4097, 16), (5001, 16), (8192, 16), (8193, 8)])
def test_products_with_4_bit_weights(N, waves, group, zeros):
    K = group * GROUPS[waves][group]
    w = random_weight(N, K, group, zeros, N + K)
    for M in (1, 5, 17):
        x = rows(M, K, M, pad=8)
        y = atb.q4_matvec(x, w, torch.float32)
        check(y, x, w)
        assert torch.equal(y[:1], atb.q4_matvec(x[:1], w, torch.float32))        # a row's bits do not depend on the others


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M", [1, 16, 33])
def test_gated_block_with_4_bit_weights(M, group, zeros):
    D, F = group * GROUPS[8][group], 256
    wg, wu, wd = random_weight(F, D, group, zeros, 7), random_weight(F, D, group, zeros, 8), random_weight(D, F, group, zeros, 9)
    x = (0.25 * rows(M, D, 10).float()).bfloat16()                               # gates on both sides of 0, not all far out
    g, u = x.double() @ values(wg).t(), x.double() @ values(wu).t()
    a, _ = ffn.activation("silu", g)
    h = a * u
    e_g, e_u = (E * 143 * (x.double().abs() @ steps(w).t()) for w in (wg, wu))
    e_a = 1.2 * e_g + 2.0 ** -19 * a.abs() + 2.0 ** -21
    e_h = e_a * u.abs() + a.abs() * e_u + e_a * e_u + R * h.abs()
    ref = h @ values(wd).t()
    tol = e_h @ values(wd).abs().t() + E * 143 * (h.abs() @ steps(wd).t()) + R * ref.abs()
    y = atb.q4_feed_forward(x, wg, wu, wd, "silu")
    off = (y.double() - ref).abs()
    assert bool((off <= tol).all()), float((off / tol).max())


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("M", [1, 8, 9, 16, 17, 31, 32])
@pytest.mark.parametrize("D,F", [(1032, 1544), (1096, 4104), (8192, 1544), (8200, 1608)])
def test_gated_block(M, D, F, act):
    x, wg, wu, wd, _ = ffn.make(M, D, F, seed=M + D + F, pad=8, scale=0.02)
    ffn.close({"y": atb.feed_forward(x, wg, wu, wd, act)}, ffn.reference(x, wg, wu, wd, None, act))
