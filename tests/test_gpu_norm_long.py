"""Layer norm of many rows and of long ones, where a call is several launches and sums are long.  The reference and its tolerances are test_gpu_norm.py's."""
import pytest
import torch

import paper_2511_16041_amd as atb
from test_gpu_norm import BF16, F32, close, inputs, reference, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_of_more_than_one_launch(dtype):
    """2^21 rows a launch: the rows on both sides of that, and the statistics' and results' places."""
    M, D = 2 ** 21 + 5, 8
    x, dy, w, b = inputs(M, D, dtype, dtype, 20, pad=3)
    want, got = reference(x, dy, w, b, 1e-5), run(x, dy, w, b, 1e-5)
    for name in ("y", "mean", "rstd", "dx"):
        close(got[name], want[name], name)


@pytest.mark.parametrize("D", [2 ** 17 + 3, 2 ** 24])
def test_sums_along_long_rows(D, monkeypatch):
    """Rows of two values and the gradient of a mean, all of one value: rounding errors of a sum are all of one sign.  A row's sum is taken in chains of at most 128 additions, of their sums at most D / 2^17 more
    and a tree of 10: each errs by at most 2^-24 of the sum of the terms' sizes."""
    monkeypatch.setattr("test_gpu_norm.E", (128 + D / 2 ** 17 + 12) * 2.0 ** -24)
    x, dy = torch.full((2, D), 0.1, device="cuda"), torch.full((2, D), 0.1, device="cuda")
    x[:, 1::2] = 0.101
    x[1, ::4] = -0.2
    want, got = reference(x, dy, None, None, 1e-5), run(x, dy, None, None, 1e-5)
    for name in ("y", "mean", "rstd", "dx"):
        close(got[name], want[name], name)


@pytest.mark.parametrize("M,D", [(2 ** 20 + 3, 8), (2 ** 23, 8), (2 ** 18 + 1, 1030)])
def test_sums_over_many_rows(M, D):
    """The gradients of the parameters where every row adds the same, so that rounding errors have one sign.  A workgroup adds at most 512 rows one after another, then halves of its
    row groups; the partial sums, M / 4096 at most of these rows, are added 64 at a time in 16 runs: each addition errs by at most 2^-24 of the sum of the terms' sizes."""
    value, xh = 0.5079958438873291, 0.75                                 # 4096 of them added in fp32: 6e-5 off
    x, dy = torch.full((M, D), 2.0, device="cuda"), torch.full((M, D), value, device="cuda")
    mean, rstd = torch.full((M,), 1.0, device="cuda"), torch.full((M,), xh, device="cuda")
    _, dw, db = atb.layer_norm_backward(dy, x, mean, rstd, torch.ones(D, device="cuda"))
    chain = 512 + 3 + 64 + M / 4096 / 16 / 64 + 1 + 16 + 1
    for got, want in ((db, M * value), (dw, M * value * xh)):
        assert bool(((got.double() - want).abs() <= (chain + 2) * 2.0 ** -24 * want).all()), float((got.double() / want - 1).abs().max())


def test_sums_over_many_long_rows():
    """The same in rows of more than 8192 elements, whose gradients of the parameters are a pass of their own."""
    M, D, value = 2 ** 17 + 1, 8200, 0.5079958438873291
    x, dy = torch.full((M, D), 2.0, device="cuda"), torch.full((M, D), value, device="cuda")
    mean, rstd = torch.ones((M,), device="cuda"), torch.ones((M,), device="cuda")
    _, dw, db = atb.layer_norm_backward(dy, x, mean, rstd, torch.ones(D, device="cuda"))
    for got in (dw, db):
        assert bool(((got.double() - M * value).abs() <= (512 + 64 + 1 + 16 + 3) * 2.0 ** -24 * M * value).all()), float((got.double() / (M * value) - 1).abs().max())
