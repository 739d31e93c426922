"""Operators around the library's matrix products that it is timed on: a transformer's feed-forward sublayer, trained and served.

Kinds of case
  norm      layer norm of M rows of D; train: the backward pass too, with the gradients of weight and bias
  ffn       gated feed-forward block y = (act(x Wg^T) o (x Wu^T)) Wd^T of M tokens; train: the backward pass too
  q4        y = x W^T of few rows with 4-bit weights, w = s (q - z) in groups of `group` along K
  q4_ffn    the gated block of few tokens with all three weights in 4 bits

Sizes come from the library's own workloads (8192, the MLP-shaped 4096 x 14336 and the ragged 3000 x 5000 x 4104 problem, the
skinny ones) or are the ordinary sizes of a transformer layer.
"""
import math

import torch

own = False                          # True: the library's operators, False: their plain form

FLOP_CAP = 18.0 * 8192 * 4096 * 14336          # the largest listed case; no drawn one costs more


def listed():
    return [
        # the smallest call: the norm of one token's activations while text is generated; launch and latency count
        {"name": "norm_token", "kind": "norm", "M": 1, "D": 4096, "dtype": "bf16", "affine": "both", "train": False},
        # a prompt's activations on the way into a block
        {"name": "norm_prompt", "kind": "norm", "M": 2048, "D": 8192, "dtype": "bf16", "affine": "both", "train": False},
        # a training step over 8192 tokens
        {"name": "norm_train", "kind": "norm", "M": 8192, "D": 4096, "dtype": "bf16", "affine": "both", "train": True},
        # fp32 activations with an odd width, no bias
        {"name": "norm_odd", "kind": "norm", "M": 3000, "D": 5001, "dtype": "f32", "affine": "weight", "train": True},
        # a batch of 16 sequences, one token each, bf16 weights: bound by the weights' bytes
        {"name": "ffn_decode", "kind": "ffn", "M": 16, "D": 4096, "F": 14336, "act": "silu", "train": False},
        # a prompt of 2048 tokens
        {"name": "ffn_prompt", "kind": "ffn", "M": 2048, "D": 4096, "F": 14336, "act": "silu", "train": False},
        # a training step of a small model on a ragged batch
        {"name": "ffn_ragged", "kind": "ffn", "M": 1500, "D": 2056, "F": 5000, "act": "gelu_tanh", "train": True},
        # a training step over 8192 tokens: the largest case
        {"name": "ffn_train", "kind": "ffn", "M": 8192, "D": 4096, "F": 14336, "act": "silu", "train": True},
        # one token through an output projection
        {"name": "q4_token", "kind": "q4", "M": 1, "N": 4096, "K": 4096, "group": 128, "zeros": False, "out": "bf16"},
        # a batch of 16 tokens through a large projection, fine groups with zero points, a result for further sums
        {"name": "q4_batch", "kind": "q4", "M": 16, "N": 8192, "K": 8192, "group": 32, "zeros": True, "out": "f32"},
        # a few drafted tokens, an odd number of outputs
        {"name": "q4_odd", "kind": "q4", "M": 5, "N": 5001, "K": 4128, "group": 32, "zeros": False, "out": "bf16"},
        # one token through the whole gated block
        {"name": "q4_ffn_token", "kind": "q4_ffn", "M": 1, "D": 4096, "F": 14336, "group": 64, "zeros": True, "act": "silu"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["norm", "ffn", "q4", "q4_ffn"], [3, 4, 3, 2])[0]
    act = rng.choice(["silu", "silu", "gelu", "gelu_tanh"])
    if kind == "norm":
        return {"kind": kind, "M": _log_int(rng, 1, 8192), "D": _log_int(rng, 64, 16384), "dtype": rng.choice(["bf16", "bf16", "f32"]),
                "affine": rng.choice(["both", "both", "weight", "none"]), "train": rng.random() < 0.6}
    if kind == "ffn":
        M, D, F = _log_int(rng, 1, 8192), 8 * _log_int(rng, 16, 1024), 8 * _log_int(rng, 16, 2048)
        train = rng.random() < 0.5
        while (18.0 if train else 6.0) * M * D * F > FLOP_CAP:
            M = max(1, M // 2)
        return {"kind": kind, "M": M, "D": D, "F": F, "act": act, "train": train}
    group, zeros, M = rng.choice([32, 64, 128]), rng.random() < 0.5, _log_int(rng, 1, 64)
    if kind == "q4":
        return {"kind": kind, "M": M, "N": _log_int(rng, 64, 16384), "K": group * _log_int(rng, 256 // group, 16384 // group),
                "group": group, "zeros": zeros, "out": rng.choice(["bf16", "bf16", "f32"])}
    return {"kind": kind, "M": M, "D": group * _log_int(rng, 256 // group, 8192 // group), "F": group * _log_int(rng, 256 // group, 16384 // group),
            "group": group, "zeros": zeros, "act": act}


# ------------------------------------------------------------------ inputs, from the seed alone

def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _weight(gen, rows, cols):
    return (_randn(gen, rows, cols) * 0.02).bfloat16()


def _q4_weight(gen, rows, cols, group, zeros):
    """A weight of standard deviation 0.02 as a 4-bit checkpoint holds it: two codes to a byte, the even k in the low half, bf16
    scales and, if asked for, zero points per group."""
    w = (_randn(gen, rows, cols) * 0.02).reshape(rows, cols // group, group)
    if zeros:
        lo, hi = w.amin(2, keepdim=True).clamp(max=0), w.amax(2, keepdim=True).clamp(min=0)
        s = ((hi - lo) / 15).bfloat16().float()
        z = torch.round(-lo / s).clamp(0, 15)
    else:
        s = (w.abs().amax(2, keepdim=True) / 7).bfloat16().float()
        z = torch.full_like(s, 8)
    q = (torch.round(w / s) + z).clamp(0, 15).to(torch.uint8).reshape(rows, cols)
    packed = q[:, 0::2] | (q[:, 1::2] << 4)
    return packed.contiguous(), s.squeeze(2).bfloat16().contiguous(), z.squeeze(2).to(torch.uint8).contiguous() if zeros else None


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, M = case["kind"], case["M"]
    if kind == "norm":
        D = case["D"]
        t = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        # a residual stream: every row off centre and of a scale of its own, a few channels large
        x = _randn(gen, M, D) * torch.exp(_randn(gen, M, 1)) + _randn(gen, M, 1)
        x = x * (1 + 9 * (torch.rand((1, D), generator=gen, device="cuda") < 0.01))
        w = (1 + 0.1 * _randn(gen, D)).to(t) if case["affine"] != "none" else None
        b = (0.1 * _randn(gen, D)).to(t) if case["affine"] == "both" else None
        dy = (0.1 * _randn(gen, M, D)).to(t) if case["train"] else None
        return {"x": x.to(t), "weight": w, "bias": b, "dy": dy}
    if kind == "ffn":
        D, F = case["D"], case["F"]
        # normalised activations in, the gradient of a mean loss back
        s = {"x": _randn(gen, M, D).bfloat16(), "wg": _weight(gen, F, D), "wu": _weight(gen, F, D), "wd": _weight(gen, D, F)}
        if case["train"]:
            s["dy"] = (0.01 * _randn(gen, M, D)).bfloat16()
        return s
    if kind == "q4":
        return {"x": _randn(gen, M, case["K"]).bfloat16(), "w": _q4_weight(gen, case["N"], case["K"], case["group"], case["zeros"])}
    D, F, how = case["D"], case["F"], (case["group"], case["zeros"])
    return {"x": _randn(gen, M, D).bfloat16(), "wg": _q4_weight(gen, F, D, *how), "wu": _q4_weight(gen, F, D, *how), "wd": _q4_weight(gen, D, F, *how)}


EPS = 1e-5


def prepare(case, seed):
    return {"case": case, **_inputs(case, seed)}


# ------------------------------------------------------------------ one pass

def run(state):
    case = state["case"]
    return (_own if own else _plain)[case["kind"]](case, state)


def _own_norm(case, s):
    import paper_2511_16041_amd as atb
    if not case["train"]:
        return {"y": atb.layer_norm(s["x"], s["weight"], s["bias"], EPS)}
    y, mean, rstd = atb.layer_norm(s["x"], s["weight"], s["bias"], EPS, stats=True)
    dx, dw, db = atb.layer_norm_backward(s["dy"], s["x"], mean, rstd, s["weight"], bias=s["bias"] is not None)
    return {"y": y, "mean": mean, "rstd": rstd, "dx": dx, "dw": dw, "db": db}


def _own_ffn(case, s):
    import paper_2511_16041_amd as atb
    if not case["train"]:
        return {"y": atb.feed_forward(s["x"], s["wg"], s["wu"], s["wd"], case["act"])}
    y, saved = atb.feed_forward(s["x"], s["wg"], s["wu"], s["wd"], case["act"], save=True)
    dx, dwg, dwu, dwd = atb.feed_forward_backward(s["dy"], s["x"], s["wg"], s["wu"], s["wd"], saved)
    return {"y": y, "dx": dx, "dwg": dwg, "dwu": dwu, "dwd": dwd}


def _own_q4(case, s):
    import paper_2511_16041_amd as atb
    return {"y": atb.q4_matvec(s["x"], s["w"], torch.float32 if case["out"] == "f32" else torch.bfloat16)}


def _own_q4_ffn(case, s):
    import paper_2511_16041_amd as atb
    return {"y": atb.q4_feed_forward(s["x"], s["wg"], s["wu"], s["wd"], case["act"])}


def _plain_norm(case, s):
    x = s["x"].float()
    t = s["x"].dtype
    w = s["weight"].float() if s["weight"] is not None else None
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + EPS)
    n = c * rstd
    y = n * w if w is not None else n
    if s["bias"] is not None:
        y = y + s["bias"].float()
    if not case["train"]:
        return {"y": y.to(t)}
    dy = s["dy"].float()
    g = dy * w if w is not None else dy
    dx = (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True)) * rstd
    dw = (dy * n).sum(0).to(t) if w is not None else None
    db = dy.sum(0).to(t) if s["bias"] is not None else None
    return {"y": y.to(t), "mean": mean.squeeze(1), "rstd": rstd.squeeze(1), "dx": dx.to(t), "dw": dw, "db": db}


def _act(name, g):
    """act(g) and its derivative"""
    if name == "silu":
        p = 1 / (1 + torch.exp(-g))
        return g * p, p * (1 + g * (1 - p))
    if name == "gelu":
        p = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * p, p + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def _plain_ffn(case, s):
    x, wg, wu, wd = (s[k].float() for k in ("x", "wg", "wu", "wd"))
    g, u = x @ wg.t(), x @ wu.t()
    a, slope = _act(case["act"], g)
    h = a * u
    y = (h @ wd.t()).bfloat16()
    if not case["train"]:
        return {"y": y}
    dy = s["dy"].float()
    dh = dy @ wd
    dg, du = dh * u * slope, dh * a
    return {"y": y, "dx": (dg @ wg + du @ wu).bfloat16(), "dwg": (dg.t() @ x).bfloat16(), "dwu": (du.t() @ x).bfloat16(), "dwd": (dy.t() @ h).bfloat16()}


def _expanded(weight):
    """A 4-bit weight in 32 bits."""
    packed, scales, zeros = weight
    q = torch.stack((packed & 15, packed >> 4), 2).reshape(packed.shape[0], scales.shape[1], -1).float()
    z = zeros.unsqueeze(2).float() if zeros is not None else 8.0
    return ((q - z) * scales.unsqueeze(2).float()).reshape(packed.shape[0], -1)


def _plain_q4(case, s):
    y = s["x"].float() @ _expanded(s["w"]).t()
    return {"y": y if case["out"] == "f32" else y.bfloat16()}


def _plain_q4_ffn(case, s):
    x = s["x"].float()
    a, _ = _act(case["act"], x @ _expanded(s["wg"]).t())
    return {"y": ((a * (x @ _expanded(s["wu"]).t())) @ _expanded(s["wd"]).t()).bfloat16()}


_own = {"norm": _own_norm, "ffn": _own_ffn, "q4": _own_q4, "q4_ffn": _own_q4_ffn}
_plain = {"norm": _plain_norm, "ffn": _plain_ffn, "q4": _plain_q4, "q4_ffn": _plain_q4_ffn}


# ------------------------------------------------------------------ what a pass cannot do without

def _q4_bytes(case, rows, cols):
    return rows * cols * (0.5 + (3.0 if case["zeros"] else 2.0) / case["group"])


def work(case):
    kind, M = case["kind"], case["M"]
    if kind == "norm":
        D, e = case["D"], 4 if case["dtype"] == "f32" else 2
        n = {"both": 2, "weight": 1, "none": 0}[case["affine"]]
        if case["train"]:        # x, dy in; y, dx out; the statistics; weight and bias in, their gradients out
            return {"bytes": e * (4.0 * M * D + 2 * n * D) + 8.0 * M, "flops": 19.0 * M * D}
        return {"bytes": e * (2.0 * M * D + n * D), "flops": 8.0 * M * D}
    if kind == "ffn":
        D, F = case["D"], case["F"]
        if case["train"]:        # x, dy, three weights in; y, dx and three gradients out
            return {"bytes": 2.0 * (4 * M * D + 6 * D * F), "flops": 18.0 * M * D * F}
        return {"bytes": 2.0 * (2 * M * D + 3 * D * F), "flops": 6.0 * M * D * F}
    if kind == "q4":
        N, K = case["N"], case["K"]
        return {"bytes": _q4_bytes(case, N, K) + 2.0 * M * K + (4.0 if case["out"] == "f32" else 2.0) * M * N, "flops": 2.0 * M * N * K}
    D, F = case["D"], case["F"]
    return {"bytes": 3 * _q4_bytes(case, F, D) + 4.0 * M * D, "flops": 6.0 * M * D * F}


# ------------------------------------------------------------------ the definitions in 64 bits

def _activation64(name, g):
    if name == "silu":
        return g * torch.sigmoid(g)
    if name == "gelu":
        return g * torch.special.ndtr(g)
    return g * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3))       # (1 + tanh v) / 2 = sigmoid(2 v)


def _value64(weight, group):
    packed, scales, zeros = weight
    q = torch.empty((packed.shape[0], 2 * packed.shape[1]), dtype=torch.float64, device=packed.device)
    q[:, ::2], q[:, 1::2] = packed % 16, packed // 16
    z = zeros.double().repeat_interleave(group, 1) if zeros is not None else 8
    return scales.double().repeat_interleave(group, 1) * (q - z)


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "norm":
        x = s["x"].double().requires_grad_(case["train"])
        w = s["weight"].double().requires_grad_(case["train"]) if s["weight"] is not None else None
        b = s["bias"].double().requires_grad_(case["train"]) if s["bias"] is not None else None
        var, mean = torch.var_mean(x, 1, unbiased=False)
        rstd = (var + EPS).rsqrt()
        y = (x - mean[:, None]) * rstd[:, None]
        if w is not None:
            y = torch.addcmul(b, y, w) if b is not None else y * w
        if not case["train"]:
            return {"y": y}
        asked = [t for t in (x, w, b) if t is not None]
        grads = list(torch.autograd.grad(y, asked, s["dy"].double())) + [None, None]
        return {"y": y.detach(), "mean": mean.detach(), "rstd": rstd.detach(), "dx": grads[0], "dw": grads[1], "db": grads[2]}
    if kind == "ffn":
        x, wg, wu, wd = (s[k].double() for k in ("x", "wg", "wu", "wd"))
        with torch.enable_grad():
            g, u = (x @ wg.t()).requires_grad_(), (x @ wu.t()).requires_grad_()
            h = _activation64(case["act"], g) * u
        out = {"y": h.detach() @ wd.t()}
        if case["train"]:
            dy = s["dy"].double()
            dg, du = torch.autograd.grad(h, (g, u), dy @ wd)
            out.update(dx=dg @ wg + du @ wu, dwg=dg.t() @ x, dwu=du.t() @ x, dwd=dy.t() @ h.detach())
        return out
    if kind == "q4":
        return {"y": s["x"].double() @ _value64(s["w"], case["group"]).t()}
    x = s["x"].double()
    wg, wu, wd = (_value64(s[k], case["group"]) for k in ("wg", "wu", "wd"))
    return {"y": (_activation64(case["act"], x @ wg.t()) * (x @ wu.t())) @ wd.t()}
