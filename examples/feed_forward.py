#!/usr/bin/env python3
"""A transformer's feed-forward sublayer, x + block(layer_norm(x)): trained in bf16, then served token by token with 4-bit weights.

    python examples/feed_forward.py [--width 1024] [--inner 4096] [--tokens 4096] [--steps 60]

The data is synthetic: a sublayer with random weights gives the outputs, and one whose weights are those with noise added learns them (tuning; from scratch such
a function takes thousands of steps).  Training keeps the weights in fp32, multiplies with copies in
bf16 and takes the gradients from layer_norm_backward and feed_forward_backward; serving quantises what was learned in groups of 32 and runs
layer_norm and q4_feed_forward on one token at a time.  Prints the loss on the way and how far both ways of serving are from the learned function.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2511_16041_amd as atb      # noqa: E402


def random_weights(gen, width, inner, device="cuda"):
    """{name: fp32} of a sublayer: normal, of such a size that activations keep their scale."""
    def normal(rows, cols):
        return torch.randn((rows, cols), generator=gen, device=device) / cols ** 0.5
    return {"norm": torch.ones(width, device=device), "shift": torch.zeros(width, device=device),
            "gate": normal(inner, width), "up": normal(inner, width), "down": normal(width, inner)}


def forward(w, x, save=False):
    """x + block(norm(x)) of bf16 tokens; with save what the gradients need as well."""
    n, mean, rstd = atb.layer_norm(x, w["norm"], w["shift"], stats=True)
    if not save:
        return x + atb.feed_forward(n, w["gate"], w["up"], w["down"], "silu")
    y, state = atb.feed_forward(n, w["gate"], w["up"], w["down"], "silu", save=True)
    return x + y, (x, n, mean, rstd, state)


def backward(w, saved, dy):
    """{name: gradient} and the gradient of x."""
    x, n, mean, rstd, state = saved
    dn, gate, up, down = atb.feed_forward_backward(dy, n, w["gate"], w["up"], w["down"], state)
    dx, norm, shift = atb.layer_norm_backward(dn, x, mean, rstd, w["norm"])
    return {"norm": norm, "shift": shift, "gate": gate, "up": up, "down": down}, dx + dy


class Adam:
    """Adam on fp32 weights, plainly."""

    def __init__(self, weights, rate):
        self.weights, self.rate, self.t = weights, rate, 0
        self.m = {k: torch.zeros_like(v) for k, v in weights.items()}
        self.v = {k: torch.zeros_like(v) for k, v in weights.items()}

    def step(self, grads):
        self.t += 1
        for k, w in self.weights.items():
            g = grads[k].float()
            self.m[k].lerp_(g, 0.1)
            self.v[k].lerp_(g * g, 0.01)
            w -= self.rate * (self.m[k] / (1 - 0.9 ** self.t)) / ((self.v[k] / (1 - 0.99 ** self.t)).sqrt() + 1e-8)


def train(width, inner, tokens, steps, seed=0, report=print):
    """The learned weights in bf16, and the loss of every step."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    teacher = {k: v.bfloat16() for k, v in random_weights(gen, width, inner).items()}
    noise = random_weights(gen, width, inner)
    master = {k: 0.8 * v.float() + 0.6 * noise[k] if v.dim() == 2 else v.float() for k, v in teacher.items()}
    optimiser, losses = Adam(master, 0.05 / width ** 0.5), []
    for step in range(steps):
        x = torch.randn((tokens, width), generator=gen, device="cuda").bfloat16()
        target = forward(teacher, x)
        w = {k: v.bfloat16() for k, v in master.items()}
        y, saved = forward(w, x, save=True)
        off = y.float() - target.float()
        losses.append((off * off).mean())
        grads, _ = backward(w, saved, (off * (2 / width)).bfloat16())       # of tokens * loss: a scale that Adam takes out again, and bf16's range keeps
        optimiser.step(grads)
        if step % 10 == 0 or step == steps - 1:
            report(f"step {step:4d}  loss {float(losses[-1]):.4f}")
    return {k: v.bfloat16() for k, v in master.items()}, [float(v) for v in losses]


def quantise(w):
    return {k: atb.q4_quantize(v, group=32) if k in ("gate", "up", "down") else v for k, v in w.items()}


def serve(w, x):
    """One token at a time, weights in 4 bits."""
    out = []
    for i in range(x.shape[0]):
        token = x[i:i + 1]
        out.append(token + atb.q4_feed_forward(atb.layer_norm(token, w["norm"], w["shift"]), w["gate"], w["up"], w["down"], "silu"))
    return torch.cat(out)


def exact(w, x):
    """The sublayer's formula in 64 bits."""
    w, x = {k: v.double() for k, v in w.items()}, x.double()
    c = x - x.mean(1, keepdim=True)
    n = c / ((c * c).mean(1, keepdim=True) + 1e-5).sqrt() * w["norm"] + w["shift"]
    g = n @ w["gate"].t()
    return x + (g * torch.sigmoid(g) * (n @ w["up"].t())) @ w["down"].t()


def run(width, inner, tokens, steps, served=16, report=print):
    """{"losses", "bf16": relative error of the trained sublayer, "q4": of the one in 4 bits against its own values, "q4 all": ... against the trained weights}"""
    w, losses = train(width, inner, tokens, steps, report=report)
    q = quantise(w)
    x = torch.randn((served, width), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()

    def off(y, want):
        return float((y.double() - want).norm() / want.norm())
    held = {k: atb.q4_decode(v, torch.float32) if isinstance(v, tuple) else v for k, v in q.items()}
    y = serve(q, x)
    result = {"losses": losses, "bf16": off(forward(w, x), exact(w, x)), "q4": off(y, exact(held, x)), "q4 all": off(y, exact(w, x))}
    report(f"served in bf16: {result['bf16']:.1e} from the formula; in 4 bits: {result['q4']:.1e} from that of the 4-bit weights, {result['q4 all']:.1e} from the trained ones")
    return result


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--inner", type=int, default=4096)
    ap.add_argument("--tokens", type=int, default=4096, help="of a training step")
    ap.add_argument("--steps", type=int, default=60)
    a = ap.parse_args()
    run(a.width, a.inner, a.tokens, a.steps)


if __name__ == "__main__":
    main()
