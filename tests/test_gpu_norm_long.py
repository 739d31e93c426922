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
