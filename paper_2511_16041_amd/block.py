"""What a transformer's block has around and in place of its feed-forward sublayer: a product with its epilogue and its gradients.

As in layers.py: results and workspaces are made on the device of the first tensor, calls are launched asynchronously on `stream`, by default that device's current one, autograd does
not follow them, tensors that are not what a kernel takes raise AssertionError and sizes that no kernel takes AtbError.  A matrix's rows may lie further apart than they are long."""
from __future__ import annotations

from typing import Optional

from . import _address
from .layers import ACTIVATIONS, _activation, _call

NO_ACTIVATION = len(ACTIVATIONS)       # ATB_ACT_NONE


# ------------------------------------------------------------------ a product with its epilogue

def linear(x, weight, bias=None, act: Optional[str] = None, residual=None, save: bool = False, stream=None):
    """act(x weight^T + bias) + residual in bf16: x M x K, weight N x K (as a linear layer's is kept), residual M x N; bias: N elements in bf16 or fp32.  K a multiple of 8, rows of x and weight
    16-byte aligned and a multiple of 8 elements apart; N any.  act: "silu", "gelu", "gelu_tanh" or None.  save: returns (y, slope), the activation's derivative in fp16 (None without
    an activation), which linear_backward takes."""
    return _call("linear", "atb_linear_forward", stream, _address("atb_linear_forward"), _address("atb_linear_workspace"), x, weight, bias,
                 NO_ACTIVATION if act is None else _activation(act), residual, save)


def linear_backward(dy, x, weight, bias=None, slope=None, stream=None):
    """(dx, dweight, dbias) of linear: in bf16, dbias in the bias's type and None without one; the residual's gradient is dy.  slope: what the forward call returned.  Inside, dy times
    slope is rounded to bf16 for the two products.  Without a slope and with N a multiple of 8 the rows of dy are 16-byte aligned and a multiple of 8 elements apart."""
    return _call("linear_backward", "atb_linear_backward", stream, _address("atb_linear_backward"), _address("atb_linear_backward_workspace"), dy, x, weight, bias, slope)
