"""The gated block's error in the 2-norm is that of the roundings that it is documented to have, and of no others: h, dg and du to bf16 ahead of the products that they are
operands of, and the results.  The same roundings are applied to the formulas in 64 bits.  What a kernel adds is fp32 sums and g and u in 24 bits, below 2^-15 of an element; one
more rounding to bf16 would make the error at least 1.2 times as large (two roundings become three, sqrt(3 / 2)), g and u in bf16 1.29 times that of dx."""
import pytest
import torch

import paper_2511_16041_amd as atb
from test_gpu_ffn import activation, make, train
from test_gpu_q4 import random_weight, rows, values

pytestmark = pytest.mark.gpu
MARGIN = 1.05


def rounded(t):
    return t.bfloat16().double()


def block(x, wg, wu, wd, dy, act, r):
    """The block and its gradients in 64 bits; r: applied to h, dg, du and the results."""
    g, u = x @ wg.t(), x @ wu.t()
    a, slope = activation(act, g)
    h = r(a * u)
    out = {"y": r(h @ wd.t())}
    if dy is not None:
        dh = dy @ wd
        dg, du = r(dh * u * slope), r(dh * a)
        out.update(dx=r(dg @ wg + du @ wu), dwg=r(dg.t() @ x), dwu=r(du.t() @ x), dwd=r(dy.t() @ h))
    return out


def check(got, operands, act):
    operands = [t.double() if t is not None else None for t in operands]
    exact, model = block(*operands, act, lambda t: t), block(*operands, act, rounded)
    for name, y in got.items():
        off, allowed = (float((t.double() - exact[name]).norm() / exact[name].norm()) for t in (y, model[name]))
        assert 1e-3 < off <= MARGIN * allowed, (name, off, allowed)


# for few rows; small tiles; shares of them; large tiles, and shares of those
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("M,D,F", [(20, 1032, 1544), (300, 1032, 1000), (64, 2056, 520), (2100, 520, 3080), (2600, 2056, 3592)])
def test_bf16(M, D, F, act):
    x, wg, wu, wd, dy = make(M, D, F, seed=M + D + F, scale=0.04)
    check(train(x, wg, wu, wd, dy, act), (x, wg, wu, wd, dy), act)
    check({"y": atb.feed_forward(x, wg, wu, wd, act)}, (x, wg, wu, wd, None), act)


@pytest.mark.parametrize("M", [1, 40])
def test_4_bits(M):
    D, F = 4096, 1536
    wg, wu, wd = (random_weight(N, K, 64, True, seed) for N, K, seed in ((F, D, 7), (F, D, 8), (D, F, 9)))
    x = (0.25 * rows(M, D, 10).float()).bfloat16()
    check({"y": atb.q4_feed_forward(x, wg, wu, wd, "silu")}, (x, values(wg), values(wu), values(wd), None), "silu")
