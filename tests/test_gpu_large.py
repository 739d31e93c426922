"""The feed-forward operators at the longest rows that are taken.  References in 64 bits, a part of the reduction at a time; tolerances as in test_gpu_q4.py."""
import pytest
import torch

import paper_2511_16041_amd as atb
from test_gpu_q4 import E, random_weight, rows, steps, values

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    torch.cuda.empty_cache()


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
