"""The operators of a transformer's feed-forward sublayer around the library's matrix products: layer norm and its gradients, the gated
block in bf16 and its gradients, and the gated block's products with 4-bit weights for few tokens.

Results and workspaces are made on the device of the first tensor; a call is launched asynchronously on `stream`, by default that device's current one, and
memory that it makes belongs to that stream.  The operators are not part of torch's autograd: results never require gradients, whatever the operands do, and a graph ends at
them; a backward pass is the call of that name, with what the forward call returns for it, and the 4-bit products have none.  Tensors that are not what a kernel takes (type, shape, device, rows whose elements
do not lie next to each other) raise AssertionError, sizes that no kernel takes AtbError.  A matrix's rows may lie further apart than they are long."""
from __future__ import annotations

from typing import NamedTuple, Optional, Tuple

from . import AtbError, _address, _launcher, _t

ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2}       # atb_activation


def _call(name: str, where: str, stream, *args):
    """The extension's function `name`; a status in place of a result is raised."""
    call = getattr(_launcher(), name)
    if stream is None:
        out = call(*args)
    else:
        with _t().cuda.stream(stream):
            out = call(*args)
    if type(out) is int:
        raise AtbError(out, where)
    return out


def _activation(name: str) -> int:
    if name not in ACTIVATIONS:
        raise ValueError(f"activation {name!r}: one of {', '.join(ACTIVATIONS)}")
    return ACTIVATIONS[name]


# ------------------------------------------------------------------ layer norm

def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, stats: bool = False, stream=None):
    """(x - mean) / sqrt(variance + eps) * weight + bias over the rows of x (M x D, bf16 or fp32), in x's type.  weight, bias: D elements in bf16 or
    fp32, both of one type, or None.  stats: returns (y, mean, rstd), the statistics in fp32, which the backward pass, layer_norm_backward, takes (autograd does not follow
    this call)."""
    return _call("layer_norm", "atb_layer_norm", stream, _address("atb_layer_norm"), x, weight, bias, eps, stats)


def layer_norm_backward(dy, x, mean, rstd, weight=None, bias: bool = True, stream=None):
    """(dx, dweight, dbias) of layer_norm: dx in x's type, the gradients of the parameters in the weight's (x's without one); dweight is None without a
    weight, dbias with bias=False.  The same inputs give the same bits."""
    return _call("layer_norm_backward", "atb_layer_norm_backward", stream, _address("atb_layer_norm_backward"), _address("atb_layer_norm_workspace"),
                 dy, x, mean, rstd, weight, bias)


# ------------------------------------------------------------------ the gated block in bf16

class FeedForwardState(NamedTuple):
    """What feed_forward keeps for its backward pass, 8 bytes for each of M x F: the inner activations in bf16, and both first products in 24 bits."""
    h: "torch.Tensor"
    kept: "torch.Tensor"
    act: str


def feed_forward(x, w_gate, w_up, w_down, act: str = "silu", save: bool = False, stream=None):
    """(act(x w_gate^T) * (x w_up^T)) w_down^T in bf16: x M x D, w_gate and w_up F x D, w_down D x F (as a linear layer's weight is kept), D and F
    multiples of 8; rows 16-byte aligned and a multiple of 8 elements apart.  act: "silu", "gelu" or "gelu_tanh".  The inner activations are rounded to bf16.  save: returns
    (y, FeedForwardState), which feed_forward_backward takes (autograd does not follow this call)."""
    out = _call("ffn_forward", "atb_ffn_forward", stream, _address("atb_ffn_forward"), _address("atb_ffn_kept_bytes"), _address("atb_ffn_workspace"), x, w_gate, w_up, w_down,
                _activation(act), save)
    return (out[0], FeedForwardState(*out[1:], act)) if save else out


def feed_forward_backward(dy, x, w_gate, w_up, w_down, state: FeedForwardState, stream=None):
    """(dx, dw_gate, dw_up, dw_down) of feed_forward, in bf16, all four; inside, the gradients of both first products are rounded to bf16.  (The C entry point takes NULL for those that are not
    asked for.)"""
    return _call("ffn_backward", "atb_ffn_backward", stream, _address("atb_ffn_backward"), _address("atb_ffn_kept_bytes"), _address("atb_ffn_backward_workspace"), dy, x, w_gate, w_up, w_down,
                 state.h, state.kept, _activation(state.act))


# ------------------------------------------------------------------ 4-bit weights

class Q4Weight(NamedTuple):
    """A weight of N outputs and K inputs in 4 bits, w = scales (codes - zeros) in groups of K / scales.shape[1] (32, 64 or 128) along K."""
    packed: "torch.Tensor"                       # uint8 N x K/2: the code of an even k in the low half of its byte
    scales: "torch.Tensor"                       # bf16 N x K/group
    zeros: Optional["torch.Tensor"] = None       # uint8 N x K/group, or None: 8


def q4_quantize(w, group: int = 128, zeros: bool = False, stream=None) -> Q4Weight:
    """A weight (N x K, bf16 or fp32) in 4 bits: symmetric, or with a zero point per group."""
    return Q4Weight(*_call("q4_quantize", "atb_q4_quantize", stream, _address("atb_q4_quantize"), w, group, zeros))


def q4_decode(weight: Tuple, dtype=None, stream=None):
    """The values of a 4-bit weight (a Q4Weight or a tuple like one): fp32 (exact) or bf16, by default bf16."""
    return _call("q4_decode", "atb_q4_decode", stream, _address("atb_q4_decode"), *Q4Weight(*weight), _is_wide(dtype))


def q4_matvec(x, weight: Tuple, dtype=None, stream=None):
    """x w^T for few rows: x M x K in bf16, the result M x N in bf16 or, with dtype=torch.float32, in fp32."""
    return _call("q4_matvec", "atb_q4_matvec", stream, _address("atb_q4_matvec"), x, *Q4Weight(*weight), _is_wide(dtype))


def q4_feed_forward(x, w_gate: Tuple, w_up: Tuple, w_down: Tuple, act: str = "silu", stream=None):
    """feed_forward of few tokens with all three weights in 4 bits; the inner activations are rounded to bf16.  Any number of tokens is right, but every 16 read the weights again."""
    return _call("q4_ffn", "atb_q4_gated", stream, _address("atb_q4_gated"), _address("atb_q4_matvec"), x, *Q4Weight(*w_gate), *Q4Weight(*w_up),
                 *Q4Weight(*w_down), _activation(act))


def _is_wide(dtype) -> bool:
    torch = _t()
    if dtype not in (None, torch.bfloat16, torch.float32):
        raise ValueError(f"dtype {dtype}: torch.bfloat16 or torch.float32")
    return dtype == torch.float32
