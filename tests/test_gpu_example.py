"""The feed-forward example end to end.

Bounds.  Each of the block's operands and results is rounded to bf16 (2^-9 of its size in the mean square at most, a handful of them in a row), so either way of serving is
within 2^-6 of the formula on its own weights; against the trained weights the 4-bit ones are off by their quantisation, at most s / 2 of a group's max / 7,
in a normal weight a tenth of its size, and the block is a part of the output only."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "feed_forward.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("feed_forward_example", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_trains_and_serves(example):
    lines = []
    got = example.run(128, 256, 512, 40, served=5, report=lines.append)
    assert got["losses"][-1] < 0.7 * got["losses"][0]
    assert got["bf16"] < 2 ** -6 and got["q4"] < 2 ** -6 and got["q4 all"] < 0.25
    assert lines


def test_gradients_are_those_of_the_formula(example):
    """Against differences of the loss in 64 bits along a random direction of every weight and of x."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    w = {k: v.bfloat16() for k, v in example.random_weights(gen, 64, 136).items()}
    x = torch.randn((48, 64), generator=gen, device="cuda").bfloat16()
    dy = torch.randn((48, 64), generator=gen, device="cuda").bfloat16()
    _, saved = example.forward(w, x, save=True)
    grads, dx = example.backward(w, saved, dy)
    for name, grad in {**grads, "x": dx}.items():
        base = x if name == "x" else w[name]
        d = torch.sign(grad.double())                      # along the gradient's signs nothing cancels
        h = 1e-5

        def loss(s):
            moved = {**w, name: base.double() + s * d}
            return float((example.exact({k: v for k, v in moved.items() if k != "x"}, moved.get("x", x)) * dy.double()).sum())
        want, got = (loss(h) - loss(-h)) / (2 * h), float((grad.double() * d).sum())
        assert abs(got - want) <= 2 ** -6 * abs(want), name
