"""Operators beside the library's feed-forward sublayer that it is timed on: what a transformer's block has around and in place of that sublayer.

Kinds of case
  linear    y = act(x W^T + b) + residual, a projection with its epilogue; train: the backward pass too, with the gradients of W and b
  resnorm   r = scale x + gate o N1(z), h = N2(r): a block's result z is normed, gated and added to the residual stream x, and the next block's input
            is normed; N1 and N2 are layer norm, root-mean-square norm or nothing; train: the backward pass too, with the gradients of gate and norms
  moe       a mixture of experts for a few tokens: softmax of the router's products, the top k of E experts, the gated feed-forward block of each
            with weights in bf16 or in 4 bits, and their sum by the router's weights

Sizes are the library's own (4096 x 14336, 8192, the ragged batch's 1500 and 3000 rows) or the ordinary ones of a transformer layer.
"""
import math

import torch

own = False                          # True: the library's operators, False: their plain form

FLOP_CAP = 6.0 * 8192 * 14336 * 4096           # the largest listed case; no drawn one costs more
EXPERT_CAP = 3.0 * 8 * 4096 * 14336            # elements of all experts' weights, likewise


def listed():
    return [
        # one token's attention output through its projection into the residual stream, while text is generated: launch, latency and the weight's bytes
        {"name": "linear_token", "kind": "linear", "M": 1, "N": 4096, "K": 4096, "act": "none", "bias": True, "residual": True, "train": False},
        # a prompt of 2048 tokens through the first product of an ungated feed-forward block
        {"name": "linear_prompt", "kind": "linear", "M": 2048, "N": 14336, "K": 4096, "act": "gelu_tanh", "bias": True, "residual": False, "train": False},
        # a training step of a head with an odd number of outputs on a ragged batch
        {"name": "linear_ragged", "kind": "linear", "M": 1500, "N": 5001, "K": 2056, "act": "gelu", "bias": True, "residual": True, "train": True},
        # a training step over 8192 tokens: the largest case
        {"name": "linear_train", "kind": "linear", "M": 8192, "N": 14336, "K": 4096, "act": "gelu_tanh", "bias": True, "residual": False, "train": True},
        # the smallest call: one token between two blocks, norms on both sides
        {"name": "resnorm_token", "kind": "resnorm", "M": 1, "D": 4096, "stream": "bf16", "block": "bf16", "post": "rms", "pre": "rms", "affine": "weight", "gates": 0, "train": False},
        # a prompt's activations between two blocks that norm their inputs only
        {"name": "resnorm_prompt", "kind": "resnorm", "M": 2048, "D": 8192, "stream": "bf16", "block": "bf16", "post": "none", "pre": "rms", "affine": "weight", "gates": 0, "train": False},
        # a training step over 8192 tokens, norms on both sides and a learned gate per channel
        {"name": "resnorm_train", "kind": "resnorm", "M": 8192, "D": 4096, "stream": "bf16", "block": "bf16", "post": "rms", "pre": "rms", "affine": "weight", "gates": 1, "train": True},
        # six sequences with a gate each from their conditioning, the residual stream in fp32, an odd width
        {"name": "resnorm_gates", "kind": "resnorm", "M": 3000, "D": 5001, "stream": "f32", "block": "bf16", "post": "layer", "pre": "layer", "affine": "both", "gates": 6, "train": True},
        # one token through two of eight large experts: bound by their weights' bytes
        {"name": "moe_token", "kind": "moe", "M": 1, "E": 8, "k": 2, "D": 4096, "F": 14336, "group": 0, "zeros": False, "act": "silu", "renormalize": True},
        # a batch of a few tokens over many small experts, ragged sizes
        {"name": "moe_batch", "kind": "moe", "M": 21, "E": 60, "k": 6, "D": 2056, "F": 1416, "group": 0, "zeros": False, "act": "gelu_tanh", "renormalize": False},
        # one token through eight of 64 small experts in 4 bits: launches and latency
        {"name": "moe_q4_token", "kind": "moe", "M": 1, "E": 64, "k": 8, "D": 2048, "F": 1536, "group": 64, "zeros": True, "act": "silu", "renormalize": True},
        # a batch of 32 sequences, one token each, over eight large experts in 4 bits: all of them are read
        {"name": "moe_q4_batch", "kind": "moe", "M": 32, "E": 8, "k": 2, "D": 4096, "F": 14336, "group": 128, "zeros": False, "act": "silu", "renormalize": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "resnorm", "moe"])
    if kind == "linear":
        M, N, K = _log_int(rng, 1, 8192), _log_int(rng, 64, 16384), 8 * _log_int(rng, 16, 1024)
        train = rng.random() < 0.5
        while (6.0 if train else 2.0) * M * N * K > FLOP_CAP:
            M = max(1, M // 2)
        return {"kind": kind, "M": M, "N": N, "K": K, "act": rng.choice(["none", "silu", "gelu", "gelu_tanh"]), "bias": rng.random() < 0.7,
                "residual": rng.random() < 0.5, "train": train}
    if kind == "resnorm":
        gates = rng.choice([0, 1, 1, _log_int(rng, 2, 64)])
        M = _log_int(rng, 1, 8192) if gates < 2 else gates * max(1, _log_int(rng, 1, 8192) // gates)
        stream = rng.choice(["bf16", "bf16", "f32"])
        return {"kind": kind, "M": M, "D": _log_int(rng, 64, 16384), "stream": stream, "block": "bf16" if stream == "bf16" else rng.choice(["bf16", "f32"]),
                "post": rng.choice(["none", "rms", "layer"]), "pre": rng.choice(["none", "rms", "rms", "layer"]),
                "affine": rng.choice(["weight", "both", "none"]), "gates": gates, "train": rng.random() < 0.6}
    M, E = _log_int(rng, 1, 64), _log_int(rng, 4, 64)
    group = rng.choice([0, 0, 32, 64, 128])
    unit = group or 8
    D, F = unit * _log_int(rng, 512 // unit, 4096 // unit), unit * _log_int(rng, 512 // unit, 14336 // unit)
    while 3.0 * E * D * F > EXPERT_CAP:
        F = max(unit, F // 2 // unit * unit)
    return {"kind": kind, "M": M, "E": E, "k": rng.randint(1, min(8, E)), "D": D, "F": F, "group": group, "zeros": group > 0 and rng.random() < 0.5,
            "act": rng.choice(["silu", "silu", "gelu", "gelu_tanh"]), "renormalize": rng.random() < 0.5}


# ------------------------------------------------------------------ inputs, from the seed alone

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


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


def _experts(gen, case, outputs, inputs):
    """One of the three weights of all experts: E x outputs x inputs in bf16, or the 4-bit weight with the rows of one expert after the other's."""
    if case["group"]:
        return _q4_weight(gen, case["E"] * outputs, inputs, case["group"], case["zeros"])
    return (_randn(gen, case["E"], outputs, inputs) * 0.02).bfloat16()


def _norm(gen, kind, D, affine):
    if kind == "none":
        return None
    return {"kind": kind, "weight": (1 + 0.1 * _randn(gen, D)).bfloat16() if affine != "none" else None, "bias": (0.1 * _randn(gen, D)).bfloat16() if affine == "both" else None}


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, M = case["kind"], case["M"]
    if kind == "linear":
        N, K = case["N"], case["K"]
        return {"x": _randn(gen, M, K).bfloat16(), "w": (_randn(gen, N, K) * 0.02).bfloat16(), "b": (0.1 * _randn(gen, N)).bfloat16() if case["bias"] else None,
                "residual": _randn(gen, M, N).bfloat16() if case["residual"] else None, "dy": (0.01 * _randn(gen, M, N)).bfloat16() if case["train"] else None}
    if kind == "resnorm":
        D, ts, tb = case["D"], TYPES[case["stream"]], TYPES[case["block"]]
        # a residual stream: every row off centre and of a scale of its own, a few channels large; and a block's result
        x = _randn(gen, M, D) * torch.exp(0.5 * _randn(gen, M, 1)) + 0.3 * _randn(gen, M, 1)
        s = {"x": (x * (1 + 9 * (torch.rand((1, D), generator=gen, device="cuda") < 0.01))).to(ts), "z": (_randn(gen, M, D) * torch.exp(_randn(gen, M, 1))).to(tb)}
        gates = case["gates"]
        s["gate"] = (0.5 + 0.2 * _randn(gen, *((D,) if gates == 1 else (gates, D)))).bfloat16() if gates else None
        s["scale"] = 1.0 if case["post"] == "none" else 0.75
        s["post"], s["pre"] = _norm(gen, case["post"], D, case["affine"]), _norm(gen, case["pre"], D, case["affine"])
        if case["train"]:
            s["dr"] = (0.1 * _randn(gen, M, D)).to(ts)
            s["dh"] = (0.1 * _randn(gen, M, D)).to(tb) if s["pre"] else None
        return s
    D, F = case["D"], case["F"]
    return {"x": _randn(gen, M, D).bfloat16(), "router": (_randn(gen, case["E"], D) * 0.02).bfloat16(),
            "wg": _experts(gen, case, F, D), "wu": _experts(gen, case, F, D), "wd": _experts(gen, case, D, F)}


def prepare(case, seed):
    return {"case": case, **_inputs(case, seed)}


# ------------------------------------------------------------------ one pass

def run(state):
    case = state["case"]
    return (_own if own else _plain)[case["kind"]](case, state)


def _own_linear(case, s):
    import paper_2511_16041_amd as atb
    act = None if case["act"] == "none" else case["act"]
    if not case["train"]:
        return {"y": atb.linear(s["x"], s["w"], s["b"], act, s["residual"])}
    y, slope = atb.linear(s["x"], s["w"], s["b"], act, s["residual"], save=True)
    dx, dw, db = atb.linear_backward(s["dy"], s["x"], s["w"], s["b"], slope)
    return {"y": y, "dx": dx, "dw": dw, "db": db}


def _own_resnorm(case, s):
    import paper_2511_16041_amd as atb
    post, pre = (atb.Norm(n["kind"], n["weight"], n["bias"], EPS) if n else None for n in (s["post"], s["pre"]))
    if not case["train"]:
        r, h = atb.residual_norm(s["x"], s["z"], post, s["gate"], s["scale"], pre)
        return {"r": r, "h": h}
    r, h, stats = atb.residual_norm(s["x"], s["z"], post, s["gate"], s["scale"], pre, save=True)
    g = atb.residual_norm_backward(s["dr"], s["dh"], s["x"], s["z"], stats, post, s["gate"], s["scale"], pre)
    return {"r": r, "h": h, "dx": g.dx, "dz": g.dz, "dgate": g.dgate, "dpw": g.dpost_weight, "dpb": g.dpost_bias, "dnw": g.dpre_weight, "dnb": g.dpre_bias}


def _own_moe(case, s):
    import paper_2511_16041_amd as atb
    y, experts, weights = atb.moe_feed_forward(s["x"], s["router"], s["wg"], s["wu"], s["wd"], case["k"], case["act"], case["renormalize"], routing=True)
    return {"y": y, "experts": experts, "weights": weights}


def _act(name, g):
    """act(g) and its derivative"""
    if name == "none":
        return g, torch.ones_like(g)
    if name == "silu":
        p = 1 / (1 + torch.exp(-g))
        return g * p, p * (1 + g * (1 - p))
    if name == "gelu":
        p = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * p, p + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def _plain_linear(case, s):
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.t()
    if s["b"] is not None:
        z = z + s["b"].float()
    a, slope = _act(case["act"], z)
    y = (a + s["residual"].float() if s["residual"] is not None else a).bfloat16()
    if not case["train"]:
        return {"y": y}
    dz = s["dy"].float() * slope
    return {"y": y, "dx": (dz @ w).bfloat16(), "dw": (dz.t() @ x).bfloat16(), "db": dz.sum(0).bfloat16() if s["b"] is not None else None}


def _normed(n, v):
    """The norm of v's rows: its result, the normed rows without weight and bias, and 1 / their size"""
    c = v - v.mean(1, keepdim=True) if n["kind"] == "layer" else v
    rstd = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + EPS)
    hat = c * rstd
    y = hat * n["weight"].float() if n["weight"] is not None else hat
    return y + n["bias"].float() if n["bias"] is not None else y, hat, rstd


def _norm_grad(n, dy, hat, rstd):
    """Gradients of the norm's operand, weight and bias"""
    g = dy * n["weight"].float() if n["weight"] is not None else dy
    d = g - hat * (g * hat).mean(1, keepdim=True)
    if n["kind"] == "layer":
        d = d - g.mean(1, keepdim=True)
    dw = (dy * hat).sum(0).bfloat16() if n["weight"] is not None else None
    return d * rstd, dw, dy.sum(0).bfloat16() if n["bias"] is not None else None


def _plain_resnorm(case, s):
    x, z, post, pre = s["x"].float(), s["z"].float(), s["post"], s["pre"]
    ts, tb = s["x"].dtype, s["z"].dtype
    M, D = x.shape
    n1, hat1, rstd1 = _normed(post, z) if post else (z, None, None)
    gate = s["gate"].float().reshape(-1, 1, D) if s["gate"] is not None else None       # of each run of M / gates rows
    gated = (gate * n1.reshape(gate.shape[0], -1, D)).reshape(M, D) if gate is not None else n1
    r = s["scale"] * x + gated
    h, hat2, rstd2 = _normed(pre, r) if pre else (None, None, None)
    out = {"r": r.to(ts), "h": h.to(tb) if pre else None}
    if not case["train"]:
        return out
    d, dnw, dnb = s["dr"].float(), None, None
    if pre:
        back, dnw, dnb = _norm_grad(pre, s["dh"].float(), hat2, rstd2)
        d = d + back
    dn, dgate = d, None
    if gate is not None:
        dn = (gate * d.reshape(gate.shape[0], -1, D)).reshape(M, D)
        dgate = (d * n1).reshape(gate.shape[0], -1, D).sum(1).reshape(s["gate"].shape).bfloat16()
    dz, dpw, dpb = _norm_grad(post, dn, hat1, rstd1) if post else (dn, None, None)
    return {**out, "dx": (s["scale"] * d).to(ts), "dz": dz.to(tb), "dgate": dgate, "dpw": dpw, "dpb": dpb, "dnw": dnw, "dnb": dnb}


def _of_experts(case, weight, used, outputs):
    """The weights of the experts `used` in 32 bits, experts x outputs x inputs."""
    if not case["group"]:
        return weight[used].float()
    packed, scales, zeros = (t.reshape(case["E"], outputs, -1)[used] if t is not None else None for t in weight)
    q = torch.stack((packed & 15, packed >> 4), 3).reshape(*scales.shape, -1).float()
    z = zeros.unsqueeze(3).float() if zeros is not None else 8.0
    return ((q - z) * scales.unsqueeze(3).float()).reshape(len(used), outputs, -1)


def _plain_moe(case, s):
    x, M = s["x"].float(), case["M"]
    logits = s["x"].double() @ s["router"].double().t()                                 # in 64 bits: which experts are the top k is decided by their order
    p = torch.exp(logits - logits.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    experts = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :case["k"]]       # ties: the lowest index first
    weights = torch.gather(p, 1, experts)
    if case["renormalize"]:
        weights = weights / weights.sum(1, keepdim=True)
    weights = weights.float()
    used, place = torch.unique(experts, return_inverse=True)
    share = torch.zeros((M, len(used)), device=x.device).scatter_(1, place, weights)
    rows = x.expand(len(used), M, -1).contiguous()
    gate, up, down = (_of_experts(case, s[name], used, n).transpose(1, 2).contiguous() for name, n in (("wg", case["F"]), ("wu", case["F"]), ("wd", case["D"])))
    a, _ = _act(case["act"], rows @ gate)
    y = (share.t().unsqueeze(2) * ((a * (rows @ up)) @ down)).sum(0)
    return {"y": y.bfloat16(), "experts": experts.int(), "weights": weights}


_own = {"linear": _own_linear, "resnorm": _own_resnorm, "moe": _own_moe}
_plain = {"linear": _plain_linear, "resnorm": _plain_resnorm, "moe": _plain_moe}


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    kind, M = case["kind"], case["M"]
    if kind == "linear":
        N, K = case["N"], case["K"]
        # x, W, y, the bias and the residual; dy in, and the gradients of x, W and the bias out
        size = 2.0 * (M * K + N * K + M * N + case["bias"] * N + case["residual"] * M * N)
        if case["train"]:
            return {"bytes": size + 2.0 * (M * N + M * K + N * K + case["bias"] * N), "flops": 6.0 * M * N * K}
        return {"bytes": size, "flops": 2.0 * M * N * K}
    if kind == "resnorm":
        D, es, eb = case["D"], 4 if case["stream"] == "f32" else 2, 4 if case["block"] == "f32" else 2
        pre, norms = case["pre"] != "none", (case["post"] != "none") + (case["pre"] != "none")
        vectors = case["gates"] + norms * {"none": 0, "weight": 1, "both": 2}[case["affine"]]
        size = M * D * (2.0 * es + (1 + pre) * eb) + 2.0 * D * vectors               # x, z in; r, h out; gate, weights and biases
        if case["train"]:        # dr, dh in; dx, dz out; the gradients of gate, weights and biases
            return {"bytes": size + M * D * (2.0 * es + (1 + pre) * eb) + 2.0 * D * vectors, "flops": (8.0 + 16.0 * norms) * M * D}
        return {"bytes": size, "flops": (3.0 + 6.0 * norms) * M * D}
    D, F, E, k = case["D"], case["F"], case["E"], case["k"]
    used = E * (1 - (1 - k / E) ** M)                                                  # experts that some token takes, on average
    element = 0.5 + (3.0 if case["zeros"] else 2.0) / case["group"] if case["group"] else 2.0
    return {"bytes": 3.0 * used * D * F * element + 2.0 * E * D + 4.0 * M * D + 8.0 * M * k, "flops": 6.0 * M * k * D * F + 2.0 * M * E * D}


# ------------------------------------------------------------------ the definitions in 64 bits

def _activation64(name, g):
    if name == "none":
        return g
    if name == "silu":
        return g * torch.sigmoid(g)
    if name == "gelu":
        return g * torch.special.ndtr(g)
    return g * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3))       # (1 + tanh v) / 2 = sigmoid(2 v)


def _norm64(n, v, weight, bias):
    square, mean = torch.var_mean(v, 1, unbiased=False, keepdim=True)
    if n["kind"] == "rms":
        square, mean = square + mean ** 2, 0.0
    y = (v - mean) * (square + EPS).rsqrt()
    y = y * weight if weight is not None else y
    return y + bias if bias is not None else y


def _value64(weight, rows, group):
    """Rows of an expert's 4-bit weight"""
    packed, scales, zeros = (t[rows] if t is not None else None for t in weight)
    q = torch.empty((packed.shape[0], 2 * packed.shape[1]), dtype=torch.float64, device=packed.device)
    q[:, ::2], q[:, 1::2] = packed % 16, packed // 16
    z = zeros.double().repeat_interleave(group, 1) if zeros is not None else 8
    return scales.double().repeat_interleave(group, 1) * (q - z)


def _exact_linear(case, s):
    x, w = s["x"].double(), s["w"].double()
    with torch.enable_grad():
        z = torch.addmm(s["b"].double(), x, w.t()) if s["b"] is not None else x @ w.t()
        z.requires_grad_()
        a = _activation64(case["act"], z)
    y = a.detach() + s["residual"].double() if s["residual"] is not None else a.detach()
    if not case["train"]:
        return {"y": y}
    dz = torch.autograd.grad(a, z, s["dy"].double())[0]
    return {"y": y, "dx": dz @ w, "dw": dz.t() @ x, "db": dz.sum(0) if s["b"] is not None else None}


def _exact_resnorm(case, s):
    post, pre, train = s["post"], s["pre"], case["train"]
    named = {"dx": s["x"], "dz": s["z"], "dgate": s["gate"], "dpw": post and post["weight"], "dpb": post and post["bias"], "dnw": pre and pre["weight"], "dnb": pre and pre["bias"]}
    leaf = {name: t.double().requires_grad_(train) if t is not None else None for name, t in named.items()}
    with torch.enable_grad():
        n = _norm64(post, leaf["dz"], leaf["dpw"], leaf["dpb"]) if post else leaf["dz"]
        if leaf["dgate"] is not None:
            n = n * leaf["dgate"].reshape(-1, case["D"]).repeat_interleave(case["M"] // max(1, case["gates"]), 0)
        r = s["scale"] * leaf["dx"] + n
        h = _norm64(pre, r, leaf["dnw"], leaf["dnb"]) if pre else None
    out = {"r": r.detach(), "h": h.detach() if pre else None}
    if not train:
        return out
    asked = [t for t in leaf.values() if t is not None]
    grads = iter(torch.autograd.grad([r, h] if pre else [r], asked, [s["dr"].double(), s["dh"].double()] if pre else [s["dr"].double()]))
    return {**out, **{name: next(grads) if t is not None else None for name, t in leaf.items()}}


def _exact_moe(case, s):
    x, D, F = s["x"].double(), case["D"], case["F"]
    logits = x @ s["router"].double().t()
    ahead = (logits.unsqueeze(1) > logits.unsqueeze(2)).sum(2)                         # experts before each one; of equal ones those of lower index too
    equal = logits.unsqueeze(1) == logits.unsqueeze(2)
    rank = ahead + torch.tril(equal, -1).sum(2)
    experts = torch.argsort(rank, 1)[:, :case["k"]]
    log_p = torch.log_softmax(torch.gather(logits, 1, experts), 1) if case["renormalize"] else torch.gather(torch.log_softmax(logits, 1), 1, experts)
    weights = torch.exp(log_p)
    y = torch.zeros_like(x)
    for e in sorted(set(experts.flatten().tolist())):
        tokens, choice = torch.nonzero(experts == e, as_tuple=True)
        if case["group"]:
            wg, wu, wd = (_value64(s[name], slice(e * n, (e + 1) * n), case["group"]) for name, n in (("wg", F), ("wu", F), ("wd", D)))
        else:
            wg, wu, wd = (s[name][e].double() for name in ("wg", "wu", "wd"))
        rows = x[tokens]
        y[tokens] += weights[tokens, choice].unsqueeze(1) * ((_activation64(case["act"], rows @ wg.t()) * (rows @ wu.t())) @ wd.t())
    return {"y": y, "experts": experts.int(), "weights": weights}


def exact(case, seed):
    return {"linear": _exact_linear, "resnorm": _exact_resnorm, "moe": _exact_moe}[case["kind"]](case, _inputs(case, seed))
