"""The operators of a block around its feed-forward sublayer without a GPU: what their entry points refuse, sizes of workspaces, and the gradients' formulas against differences."""
import ctypes

import pytest

import paper_2511_16041_amd as atb
from test_abi_host import _on_device
from test_layers_host import INVALID, _slope, aligned_address


# ------------------------------------------------------------------ a product with its epilogue

def test_linear_refuses():
    L = atb.lib()
    keep, a = aligned_address()
    good = dict(x=a, w=a, ldx=16, ldw=16, bias=a, M=2, N=7, K=16, act=0, bias_type=0, workspace=a)

    def forward(residual=a, ldr=7, slope=a, y=a, ldy=7, **kw):
        l = atb.Linear(**{**good, **kw})
        return L.atb_linear_forward(ctypes.byref(l), residual, ldr, slope, y, ldy, None)

    def backward(slope=a, dy=a, lddy=7, dx=a, lddx=16, dw=a, db=a, **kw):
        l = atb.Linear(**{**good, **kw})
        return L.atb_linear_backward(ctypes.byref(l), slope, dy, lddy, dx, lddx, dw, db, None)
    shared = [dict(x=None), dict(w=None), dict(x=a + 2), dict(w=a + 8), dict(ldx=15), dict(ldx=20), dict(ldx=8), dict(ldw=8), dict(ldw=2 ** 22), dict(bias=a + 1), dict(bias=a + 2, bias_type=1), dict(M=-1),
              dict(M=2 ** 23 + 1), dict(N=0), dict(N=-1), dict(N=2 ** 22 - 7), dict(K=0), dict(K=12), dict(K=2 ** 22), dict(act=4), dict(act=-1), dict(bias_type=2), dict(workspace=a + 8)]
    for bad in shared + [dict(y=None), dict(y=a + 1), dict(ldy=6), dict(residual=a + 1), dict(ldr=6), dict(slope=a + 1), dict(act=3)]:
        assert forward(**bad) == INVALID, bad
    for bad in shared + [dict(dy=None), dict(dy=a + 1), dict(lddy=6), dict(slope=None), dict(act=3), dict(slope=a + 1), dict(dx=a + 2), dict(lddx=15), dict(lddx=8), dict(dw=a + 8), dict(db=a + 1),
                         dict(db=a + 2, bias_type=1), dict(workspace=None), dict(act=3, slope=None, N=8, lddy=9), dict(act=3, slope=None, N=8, lddy=8, dy=a + 2)]:
        assert backward(**bad) == INVALID, bad
    assert L.atb_linear_forward(None, a, 7, a, a, 7, None) == INVALID and L.atb_linear_backward(None, a, a, 7, a, 16, a, a, None) == INVALID
    assert forward(M=0, x=None, y=None, residual=None, slope=None) == 0
    assert backward(M=0, x=None, dy=None, dx=None, dw=None, db=None) == 0
    # without a device what is right gets as far as the launch
    if not __import__("torch").cuda.is_available():
        assert forward() == forward(residual=None, slope=None, bias=None) == forward(M=40, slope=None, workspace=None) == backward() == backward(act=3, slope=None) == 5
        assert backward(act=3, slope=None, N=8, lddy=8) == backward(M=0, x=None, dy=None) == 5


def test_workspace_of_a_product_with_its_epilogue():
    L = atb.lib()
    for M in (1, 33, 100, 1000, 8192):
        for N in (1, 1031, 14336):
            for K in (8, 1032, 4096):
                assert L.atb_linear_workspace(M, N, K, 0) <= L.atb_linear_workspace(M, N, K, 1) <= 64 << 20
                dz = 2 * M * (N + 7 & -8)
                assert L.atb_linear_backward_workspace(M, N, K, 0) >= dz + 4 * N
                assert L.atb_linear_backward_workspace(M, N, K, 3) >= (dz if N % 8 else 0) + 4 * N
    assert L.atb_linear_backward_workspace(8192, 14336, 4096, 3) < 64 << 20
    for bad in ((-1, 64, 64), (1, 0, 64), (1, 64, 60), (2 ** 23 + 1, 64, 64), (1, 64, 2 ** 22), (1, 2 ** 22, 64)):
        assert L.atb_linear_workspace(*bad, 1) == 0 and L.atb_linear_backward_workspace(*bad, 0) == 0
    assert L.atb_linear_backward_workspace(4, 64, 64, 4) == 0


def test_linear_refuses_tensors_that_a_kernel_would_read_or_store_past():
    import torch
    bf, f32, f16 = torch.bfloat16, torch.float32, torch.float16
    x, w = _on_device((4, 64), bf), _on_device((24, 64), bf)
    r = _on_device((4, 24), bf)
    for args in [(torch.zeros(4, 64, dtype=bf), w), (_on_device((4, 64), f32), w), (x, _on_device((24, 56), bf)), (x, _on_device((64, 24), bf, (1, 64))), (x, w, _on_device((23,), bf)),
                 (x, w, _on_device((24,), f16)), (x, w, _on_device((24,), bf, (2,))), (x, w, torch.zeros(24, dtype=bf)), (x, w, None, None, _on_device((4, 23), bf)), (x, w, None, None, _on_device((4, 24), f32)),
                 (x, w, None, None, _on_device((1, 24), bf)), (x, w, None, None, _on_device((4, 24), bf, (0, 1)))]:
        with pytest.raises(AssertionError):
            atb.linear(*args)
    slope = _on_device((4, 24), f16)
    for args in [(_on_device((4, 23), bf), x, w), (_on_device((4, 24), f32), x, w), (r, x, w, None, _on_device((4, 24), bf)), (r, x, w, None, _on_device((4, 16), f16)),
                 (r, x, w, None, _on_device((4, 24), f16, (32, 1))), (r, x, w, _on_device((25,), bf), slope), (r, x, _on_device((25, 64), bf), None, slope)]:
        with pytest.raises(AssertionError):
            atb.linear_backward(*args)
    with pytest.raises(ValueError, match="silu"):
        atb.linear(x, w, None, "relu")
    with pytest.raises(TypeError):
        atb.linear(x, None)


@pytest.mark.parametrize("act", [None, "silu", "gelu", "gelu_tanh"])
def test_linear_gradients_against_differences(act):
    """The formulas that the GPU tests compare with."""
    import torch
    from test_gpu_linear import reference
    g = torch.Generator().manual_seed(1)
    x, w, b, dy = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((3, 6), (8, 6), (8,), (3, 8)))
    want = reference(x, w, b, None, dy, act)

    def loss(x, w, b):
        return (reference(x, w, b, None, dy, act)["y"][0] * dy).sum()
    for at, name in enumerate(("dx", "dw", "db")):
        v = torch.randn((x, w, b)[at].shape, generator=g, dtype=torch.float64)
        grad = float((want[name][0] * v).sum())
        assert abs(_slope(loss, (x, w, b), at, v) - grad) < 1e-6 * (1 + abs(grad))
