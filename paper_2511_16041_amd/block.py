"""What a transformer's block has around and in place of its feed-forward sublayer: a product with its epilogue, norms on both sides of a residual sum, and their gradients; and for few
tokens a mixture of experts.

As in layers.py: results and workspaces are made on the device of the first tensor, calls are launched asynchronously on `stream`, by default that device's current one, autograd does
not follow them, tensors that are not what a kernel takes raise AssertionError and sizes that no kernel takes AtbError.  A matrix's rows may lie further apart than they are long."""
from __future__ import annotations

from typing import NamedTuple, Optional, Tuple

from . import _address
from .layers import ACTIVATIONS, Q4Weight, _activation, _call

NO_ACTIVATION = len(ACTIVATIONS)       # ATB_ACT_NONE


# ------------------------------------------------------------------ a product with its epilogue

def linear(x, weight, bias=None, act: Optional[str] = None, residual=None, save: bool = False, stream=None):
    """act(x weight^T + bias) + residual in bf16: x M x K, weight N x K (as a linear layer's is kept), residual M x N; bias: N elements in bf16 or fp32.  K a multiple of 8, rows of x and weight
    16-byte aligned and a multiple of 8 elements apart; N any.  act: "silu", "gelu", "gelu_tanh" or None.  save: returns (y, slope), the activation's derivative in fp16 (M rows of
    round_up(N, 8), of which N count; None without an activation; off by 2^-11 of itself or by 2^-25, what is more), which linear_backward takes."""
    return _call("linear", "atb_linear_forward", stream, _address("atb_linear_forward"), _address("atb_linear_workspace"), x, weight, bias,
                 NO_ACTIVATION if act is None else _activation(act), residual, save)


def linear_backward(dy, x, weight, bias=None, slope=None, stream=None):
    """(dx, dweight, dbias) of linear: in bf16, dbias in the bias's type and None without one; the residual's gradient is dy.  All three are
    computed (the C entry point takes NULL for those that are not asked for).  slope: what the forward call returned.  Inside, dy times
    slope is rounded to bf16 for the two products.  Without a slope and with N a multiple of 8 the rows of dy are 16-byte aligned and a multiple of 8 elements apart."""
    return _call("linear_backward", "atb_linear_backward", stream, _address("atb_linear_backward"), _address("atb_linear_backward_workspace"), dy, x, weight, bias, slope)


# ------------------------------------------------------------------ norms on both sides of a residual sum

NORMS = {"rms": 1, "layer": 2}         # atb_norm_kind


class Norm(NamedTuple):
    """A norm of rows v of D elements: "layer", (v - mean) / sqrt(variance + eps) weight + bias, or "rms", v / sqrt(mean of squares + eps) weight + bias.  weight, bias: D elements in bf16 or fp32, or None."""
    kind: str = "rms"
    weight: Optional["torch.Tensor"] = None
    bias: Optional["torch.Tensor"] = None
    eps: float = 1e-5


class ResidualNormGrads(NamedTuple):
    """The gradients of residual_norm's operands; None for those that it does not have."""
    dx: "torch.Tensor"
    dz: "torch.Tensor"
    dgate: Optional["torch.Tensor"]
    dpost_weight: Optional["torch.Tensor"]
    dpost_bias: Optional["torch.Tensor"]
    dpre_weight: Optional["torch.Tensor"]
    dpre_bias: Optional["torch.Tensor"]


def _norm(norm: Optional[Norm]) -> Tuple:
    if norm is None:
        return 0, None, None, 0.0
    kind, weight, bias, eps = norm
    if kind not in NORMS:
        raise ValueError(f"norm {kind!r}: one of {', '.join(NORMS)}, or None in the norm's place")
    return NORMS[kind], weight, bias, eps


def residual_norm(x, z, post: Optional[Norm] = None, gate=None, scale: float = 1.0, pre: Optional[Norm] = None, save: bool = False, stream=None):
    """r = scale x + gate * post(z) and h = pre(r), what lies between a block with the result z, the residual stream x and the next block; returns (r, h), h None without a norm `pre`.  x, z: M x D,
    x in bf16 or fp32, z in x's type or in bf16; r in x's type, h (of the sum before it is rounded) in z's.  gate: D elements, or G x D with M a multiple of G: a row for every M / G rows of
    x.  Gate, weights and biases all in one type, bf16 or fp32.  save: returns (r, h, stats), the norms' statistics (4 x M, fp32), which residual_norm_backward takes."""
    return _call("residual_norm", "atb_residual_norm_forward", stream, _address("atb_residual_norm_forward"), x, z, *_norm(post), gate, scale, *_norm(pre), save)


def residual_norm_backward(dr, dh, x, z, stats, post: Optional[Norm] = None, gate=None, scale: float = 1.0, pre: Optional[Norm] = None, stream=None) -> ResidualNormGrads:
    """The gradients of residual_norm from those of r (by all but h; None: 0) and of h (None without a norm `pre`), each in its operand's type; of everything that is there
    (the C entry point takes NULL for those that are not asked for).  The same inputs give the same bits."""
    return ResidualNormGrads(*_call("residual_norm_backward", "atb_residual_norm_backward", stream, _address("atb_residual_norm_backward"), _address("atb_residual_norm_workspace"),
                                    dr, dh, x, z, stats, *_norm(post), gate, scale, *_norm(pre)))


# ------------------------------------------------------------------ a mixture of experts for few tokens

def _expert_weight(weight) -> Tuple:
    return Q4Weight(*weight) if isinstance(weight, tuple) else (weight, None, None)


def moe_feed_forward(x, router, w_gate, w_up, w_down, top_k: int = 2, act: str = "silu", renormalize: bool = True, routing: bool = False, stream=None):
    """A mixture of E gated blocks for up to 64 tokens: x M x D, router E x D, both in bf16; every token goes through the top_k (16 at most) experts with the largest x router^T (of equal ones the
    lowest), and y, M x D in bf16, is the sum of (act(x w_gate[e]^T) * (x w_up[e]^T)) w_down[e]^T times softmax(x router^T)[e] (renormalize: the softmax of the chosen ones alone).  w_gate and w_up: E x F x D in bf16,
    w_down E x D x F, contiguous, D and F multiples of 8; or all three 4-bit weights (a Q4Weight or a tuple like one, as of q4_quantize) of E F, E F and E D outputs, one expert's after the other's.
    The inner activations are rounded to bf16.  routing: returns (y, experts, weights), M x top_k in int32 and fp32, from the largest on."""
    return _call("moe", "atb_moe_forward", stream, _address("atb_moe_forward"), _address("atb_moe_workspace"), x, router, *_expert_weight(w_gate), *_expert_weight(w_up), *_expert_weight(w_down),
                 top_k, _activation(act), renormalize, routing)
