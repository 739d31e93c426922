"""A few tokens through a mixture of experts, whose choice the products make themselves: the same experts and weights as among more tokens, bit by bit, and y by the formula."""
import pytest
import torch

import paper_2511_16041_amd as atb
from test_gpu_moe import check, make

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("group", [0, 32])
@pytest.mark.parametrize("E,k", [(1, 1), (2, 1), (16, 16), (63, 5), (64, 16), (65, 2), (100, 7), (128, 16), (129, 3), (200, 16), (255, 1), (256, 16)])
def test_alone_and_among_others(E, k, group):
    args = make(9, E, 96, 64, E + k, group)
    x, router = args[0], args[1].clone()
    if E > 8:
        router[E // 2:E // 2 + 4] = router[3]                  # equal ones
        x = x.clone()
        x[2], x[5, 7] = 0.0, float("nan")                      # all are equal; none is a number
    for renormalize in (True, False):
        _, chosen, weights = atb.moe_feed_forward(x, router, *args[2:], k, renormalize=renormalize, routing=True)
        for m in range(9):
            y1, chosen1, weights1 = atb.moe_feed_forward(x[m:m + 1], router, *args[2:], k, renormalize=renormalize, routing=True)
            assert torch.equal(chosen1[0], chosen[m]), (m, renormalize)
            if E > 8 and m == 5:
                assert weights1.isnan().all() and weights[m].isnan().all() and y1.isnan().all()
                continue
            assert torch.equal(weights1[0], weights[m]), (m, renormalize)
            if m < 3:
                check((x[m:m + 1], router, *args[2:]), k, "silu", renormalize, got=(y1, chosen1, weights1))
            assert torch.equal(y1, atb.moe_feed_forward(x[m:m + 1], router, *args[2:], k, renormalize=renormalize))


@pytest.mark.parametrize("group", [0, 64])
@pytest.mark.parametrize("E,k", [(1, 1), (2, 2), (8, 2), (8, 8), (16, 16), (31, 3), (32, 16), (33, 4), (64, 8), (85, 5), (100, 2), (128, 16)])
def test_a_few_and_among_more(E, k, group):
    """2 to 8 tokens, with up to 256 of the router's products and with more."""
    args = make(12, E, 128, 64, E + k, group)
    x, router = args[0].clone(), args[1].clone()
    x[3] = x[1]
    if E > 8:
        router[E // 2:E // 2 + 3] = router[2]
        x[4], x[6, 5] = 0.0, float("nan")
    _, chosen, weights = atb.moe_feed_forward(x, router, *args[2:], k, "gelu", False, routing=True)
    for M in range(2, 9):
        for first in (0, 12 - M):
            part = x[first:first + M]
            got = atb.moe_feed_forward(part, router, *args[2:], k, "gelu", False, routing=True)
            assert torch.equal(got[1], chosen[first:first + M]), (M, first)
            assert torch.equal(got[2].nan_to_num(-1.0), weights[first:first + M].nan_to_num(-1.0)), (M, first)
            check((part, router, *args[2:]), k, "gelu", False, rows=[m for m in range(M) if E <= 8 or first + m not in (4, 6)], got=got)
            assert torch.equal(got[0].nan_to_num(-1.0), atb.moe_feed_forward(part, router, *args[2:], k, "gelu", False).nan_to_num(-1.0))


def test_one_token_captured_and_replayed():
    """The choice is made anew in every replay."""
    x, *rest = make(6, 40, 128, 192, 3, 64)
    static = x[:1].clone()
    atb.moe_feed_forward(static, *rest, 4)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, chosen, weights = atb.moe_feed_forward(static, *rest, 4, routing=True)
    for m in (1, 2, 3, 4, 5, 0):
        static.copy_(x[m:m + 1])
        graph.replay()
        eager = atb.moe_feed_forward(x[m:m + 1], *rest, 4, routing=True)
        torch.cuda.synchronize()
        assert torch.equal(y, eager[0]) and torch.equal(chosen, eager[1]) and torch.equal(weights, eager[2]), m
