"""The operators around a feed-forward sublayer in a run, as they are used: two norms with their residual sums, an ungated feed-forward block and a head, trained; and the same with a mixture of experts for few tokens.

Tolerances.  Every value on the way is rounded to bf16 once, which moves it by at most 2^-8 / sqrt 3 of itself in the 2-norm, and is the sum or product of a few that were; a loss's way through the run and back passes at
most 12 such roundings, none of which the norms and products here amplify more than twofold."""
import pytest
import torch

import paper_2511_16041_amd as atb
from test_gpu_ffn import activation
from test_gpu_moe import reference as moe_reference

pytestmark = pytest.mark.gpu
LIMIT = 12 * 2 * 2.0 ** -8 / 3 ** 0.5
BF16 = torch.bfloat16


def parameters(D, F, V, seed, groups):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def t(s, *shape, at=0.0):
        return (at + s * torch.randn(shape, generator=g, device="cuda")).to(BF16)
    return {"post1": t(0.1, D, at=1), "gate1": t(0.2, groups, D, at=0.7), "pre1": t(0.1, D, at=1), "pre1b": t(0.1, D), "w1": t(D ** -0.5, F, D), "b1": t(0.1, F), "w2": t(F ** -0.5, D, F), "b2": t(0.1, D),
            "post2": t(0.1, D, at=1), "pre2": t(0.1, D, at=1), "head": t(D ** -0.5, V, D)}


def step(x, z, dlogits, p):
    """Forward and backward pass: (logits, the stream, {name: gradient})"""
    post1, pre1, post2, pre2 = atb.Norm("rms", p["post1"]), atb.Norm("layer", p["pre1"], p["pre1b"]), atb.Norm("rms", p["post2"]), atb.Norm("rms", p["pre2"])
    r1, h1, s1 = atb.residual_norm(x, z, post1, p["gate1"], 1.0, pre1, save=True)
    u, slope = atb.linear(h1, p["w1"], p["b1"], "gelu_tanh", save=True)
    z2 = atb.linear(u, p["w2"], p["b2"])
    r2, h2, s2 = atb.residual_norm(r1, z2, post2, None, 0.9, pre2, save=True)
    logits = atb.linear(h2, p["head"])
    dh2, dhead, _ = atb.linear_backward(dlogits, h2, p["head"])
    g2 = atb.residual_norm_backward(None, dh2, r1, z2, s2, post2, None, 0.9, pre2)
    du, dw2, db2 = atb.linear_backward(g2.dz, u, p["w2"], p["b2"])
    dh1, dw1, db1 = atb.linear_backward(du, h1, p["w1"], p["b1"], slope)
    g1 = atb.residual_norm_backward(g2.dx, dh1, x, z, s1, post1, p["gate1"], 1.0, pre1)
    return logits, r2, {"x": g1.dx, "z": g1.dz, "post1": g1.dpost_weight, "gate1": g1.dgate, "pre1": g1.dpre_weight, "pre1b": g1.dpre_bias, "w1": dw1, "b1": db1, "w2": dw2, "b2": db2,
                        "post2": g2.dpost_weight, "pre2": g2.dpre_weight, "head": dhead}


def rms(v, w):
    return v * (v.square().mean(1, keepdim=True) + 1e-5).rsqrt() * w


def step64(x, z, dlogits, p):
    """The same from the definitions, with autograd"""
    leaf = {k: t.double().requires_grad_() for k, t in {"x": x, "z": z, **p}.items()}
    M, G = x.shape[0], p["gate1"].shape[0]
    r1 = leaf["x"] + leaf["gate1"].repeat_interleave(M // G, 0) * rms(leaf["z"], leaf["post1"])
    var, mean = torch.var_mean(r1, 1, unbiased=False, keepdim=True)
    h1 = (r1 - mean) * (var + 1e-5).rsqrt() * leaf["pre1"] + leaf["pre1b"]
    u = activation("gelu_tanh", h1 @ leaf["w1"].t() + leaf["b1"])[0]
    z2 = u @ leaf["w2"].t() + leaf["b2"]
    r2 = 0.9 * r1 + rms(z2, leaf["post2"])
    logits = rms(r2, leaf["pre2"]) @ leaf["head"].t()
    grads = torch.autograd.grad(logits, list(leaf.values()), dlogits.double())
    return logits.detach(), r2.detach(), dict(zip(leaf, grads))


@pytest.mark.parametrize("M,D,F,V,groups", [(6, 64, 136, 33, 3), (300, 512, 1032, 1001, 2), (64, 1000, 264, 72, 1), (1500, 264, 520, 4099, 5)])
@pytest.mark.parametrize("stream", [BF16, torch.float32])
def test_a_block_in_training(M, D, F, V, groups, stream):
    p = parameters(D, F, V, M + D, groups)
    g = torch.Generator(device="cuda").manual_seed(M)
    x, z = torch.randn((M, D), generator=g, device="cuda").to(stream), torch.randn((M, D), generator=g, device="cuda").to(BF16)
    dlogits = (0.1 * torch.randn((M, V), generator=g, device="cuda")).to(BF16)
    logits, r2, grads = step(x, z, dlogits, p)
    want_logits, want_r2, want = step64(x, z, dlogits, p)
    for name, a, b in [("logits", logits, want_logits), ("stream", r2, want_r2)] + [(k, grads[k], want[k]) for k in want]:
        assert a.shape == b.shape and a.dtype == (stream if name in ("x", "stream") else BF16), name
        assert float((a.double() - b).norm()) <= LIMIT * float(b.norm()), name


def test_a_block_in_training_captured_and_replayed():
    """The whole step as one graph, with the step outside of it in between."""
    p = parameters(512, 1032, 1001, 1, 2)
    x, z, d = (torch.randn(s, device="cuda").to(BF16) for s in ((200, 512), (200, 512), (200, 1001)))
    static = [t.clone() for t in (x, z, d)]
    step(*static, p)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        logits, r2, grads = step(*static, p)
    for n in range(3):
        new = [torch.randn(t.shape, device="cuda").to(BF16) for t in static]
        for a, b in zip(static, new):
            a.copy_(b)
        graph.replay()
        e_logits, e_r2, e_grads = step(*new, p)
        torch.cuda.synchronize()
        assert torch.equal(logits, e_logits) and torch.equal(r2, e_r2) and all(torch.equal(grads[k], e_grads[k]) for k in grads), n


@pytest.mark.parametrize("M,group", [(1, 0), (1, 32), (24, 0), (24, 64)])
def test_tokens_through_a_mixture_of_experts_between_two_norms(M, group):
    """Serving: norm, experts in bf16 and in 4 bits, residual sum and the next norm, head."""
    D, F, E, k, V = 256, 384, 12, 3, 1001
    p = parameters(D, 8, V, 3, 1)
    g = torch.Generator(device="cuda").manual_seed(M)
    x, z, router = (torch.randn(s, generator=g, device="cuda").to(BF16) for s in ((M, D), (M, D), (E, D)))
    router *= D ** -0.5
    weights = [0.06 * torch.randn((E * n, i), generator=g, device="cuda") for n, i in ((F, D), (F, D), (D, F))]
    weights = [atb.q4_quantize(w, group, zeros=True) for w in weights] if group else [w.to(BF16).view(E, -1, w.shape[1]) for w in weights]
    pre1, pre2 = atb.Norm("rms", p["pre1"]), atb.Norm("rms", p["pre2"])
    r1, h1 = atb.residual_norm(x, z, None, p["gate1"][0], 1.0, pre1)
    y = atb.moe_feed_forward(h1, router, *weights, k)
    r2, h2 = atb.residual_norm(r1, y, None, None, 1.0, pre2)
    logits = atb.linear(h2, p["head"])
    want_r1 = x.double() + p["gate1"].double() * z.double()
    want_y = moe_reference(h1, router, *weights, k, "silu", True)[0]            # of the rounded h1: with another, a token may choose other experts
    want_r2 = want_r1 + want_y
    want = rms(want_r2, p["pre2"].double()) @ p["head"].double().t()
    for name, a, b in (("r1", r1, want_r1), ("h1", h1, rms(want_r1, p["pre1"].double())), ("y", y, want_y), ("r2", r2, want_r2), ("logits", logits, want)):
        assert float((a.double() - b).norm()) <= LIMIT * float(b.norm()), name


def test_the_operators_are_not_part_of_autograd():
    p = parameters(64, 136, 40, 4, 1)
    x, z = (torch.randn((20, 64), device="cuda").to(BF16) for _ in range(2))
    asked = {k: t.clone().requires_grad_() for k, t in {"x": x, "z": z, **p}.items()}
    plain = step(x, z, torch.ones((20, 40), dtype=BF16, device="cuda"), p)
    again = step(asked["x"], asked["z"], torch.ones((20, 40), dtype=BF16, device="cuda"), {k: asked[k] for k in p})
    assert torch.equal(plain[0], again[0]) and not again[0].requires_grad and not again[1].requires_grad
    assert all(torch.equal(plain[2][k], again[2][k]) and not again[2][k].requires_grad for k in plain[2])
