"""The operators of a block around its feed-forward sublayer without a GPU: what their entry points refuse, sizes of workspaces, and the gradients' formulas against differences."""
import ctypes
import os
import shutil
import subprocess

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
    for bad in shared + [dict(y=None), dict(y=a + 1), dict(ldy=6), dict(residual=a + 1), dict(ldr=6), dict(slope=a + 2), dict(act=3)]:
        assert forward(**bad) == INVALID, bad
    for bad in shared + [dict(dy=None), dict(dy=a + 1), dict(lddy=6), dict(slope=None), dict(act=3), dict(slope=a + 8), dict(dx=a + 2), dict(lddx=15), dict(lddx=8), dict(dw=a + 8), dict(db=a + 1),
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
                assert L.atb_linear_workspace(M, N, K) <= 64 << 20
                dz = 2 * M * (N + 7 & -8)
                assert L.atb_linear_backward_workspace(M, N, K, 0) >= dz + 4 * N
                assert L.atb_linear_backward_workspace(M, N, K, 3) >= (dz if N % 8 else 0) + 4 * N
    assert L.atb_linear_backward_workspace(8192, 14336, 4096, 3) < 64 << 20
    for bad in ((-1, 64, 64), (1, 0, 64), (1, 64, 60), (2 ** 23 + 1, 64, 64), (1, 64, 2 ** 22), (1, 2 ** 22, 64)):
        assert L.atb_linear_workspace(*bad) == 0 and L.atb_linear_backward_workspace(*bad, 0) == 0
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


# ------------------------------------------------------------------ norms on both sides of a residual sum

def test_residual_norm_refuses():
    L = atb.lib()
    keep, a = aligned_address()
    rms, nothing = atb.NormArgs(a, a, 1e-5, 1), atb.NormArgs(None, None, 0.0, 0)
    good = dict(x=a, z=a, ldx=8, ldz=8, post=rms, pre=rms, gate=a, groups=2, scale=1.0, M=4, D=8, stream_type=0, block_type=0, param_type=0)

    def forward(r=a, ldr=8, h=a, ldh=8, stats=a, **kw):
        return L.atb_residual_norm_forward(ctypes.byref(atb.ResidualNorm(**{**good, **kw})), r, ldr, h, ldh, stats, None)

    def backward(stats=a, dr=a, lddr=8, dh=a, lddh=8, grads=None, work=a, **kw):
        g = atb.ResidualNormGradArgs(**{**dict(dx=a, dz=a, lddx=8, lddz=8, dgate=a, dpost_weight=a, dpost_bias=a, dpre_weight=a, dpre_bias=a), **(grads or {})})
        return L.atb_residual_norm_backward(ctypes.byref(atb.ResidualNorm(**{**good, **kw})), stats, dr, lddr, dh, lddh, ctypes.byref(g), work, None)
    shared = [dict(x=None), dict(z=None), dict(x=a + 1), dict(z=a + 1), dict(x=a + 2, stream_type=1), dict(ldx=7), dict(ldz=7), dict(gate=a + 1), dict(gate=None), dict(groups=0), dict(groups=3), dict(groups=65536, M=65536),
              dict(M=-2), dict(M=2 ** 23 + 2), dict(D=0), dict(D=2 ** 24 + 1, ldx=2 ** 25, ldz=2 ** 25), dict(stream_type=2), dict(block_type=-1), dict(param_type=2), dict(block_type=1), dict(scale=float("nan")),
              dict(scale=float("inf")), dict(scale=-1e39)]
    for side in ("post", "pre"):
        shared += [{side: atb.NormArgs(a, a, 1e-5, 3)}, {side: atb.NormArgs(a, a, -1.0, 1)}, {side: atb.NormArgs(a, a, float("nan"), 2)}, {side: atb.NormArgs(a + 1, a, 0.0, 1)}, {side: atb.NormArgs(a, a + 1, 0.0, 2)}]
    for bad in shared + [dict(r=None), dict(r=a + 1), dict(ldr=7), dict(h=None), dict(ldh=7), dict(h=a + 1), dict(stats=a + 2), dict(pre=nothing)]:
        assert forward(**bad) == INVALID, bad
    for bad in shared + [dict(stats=None), dict(stats=a + 2), dict(dr=a + 1), dict(lddr=7), dict(dh=None), dict(lddh=7), dict(work=None), dict(work=a + 8), dict(pre=nothing), dict(post=nothing), dict(gate=None, groups=1),
                         dict(grads=dict(dx=a + 1)), dict(grads=dict(lddx=7)), dict(grads=dict(dz=a + 1)), dict(grads=dict(lddz=0)), dict(grads=dict(dgate=a + 1)), dict(grads=dict(dpre_bias=a + 1))]:
        assert backward(**bad) == INVALID, bad
    assert L.atb_residual_norm_forward(None, a, 8, a, 8, a, None) == INVALID
    assert L.atb_residual_norm_backward(ctypes.byref(atb.ResidualNorm(**good)), a, a, 8, a, 8, None, a, None) == INVALID
    assert forward(M=0, x=None, z=None, r=None, h=None) == 0
    assert backward(M=0, x=None, z=None, dh=None, stats=None, grads={k: None for k in ("dgate", "dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias")}) == 0
    if not __import__("torch").cuda.is_available():
        assert forward() == forward(pre=nothing, h=None) == forward(post=nothing, gate=None, groups=1) == forward(D=20000, ldx=20000, ldz=20000, ldr=20000, ldh=20000) == backward() == backward(dr=None) == 5


@pytest.mark.parametrize("eps", [1e-50, 1e-46, 5e-324, 3.5e38, 1e300, float("inf")])
@pytest.mark.parametrize("kind", [1, 2])
def test_residual_norm_refuses_an_eps_that_fp32_does_not_hold(eps, kind):
    """One that fp32 rounds to 0 would make 0 * inf of a row of zeros, one beyond its range 0 of every row."""
    L = atb.lib()
    keep, a = aligned_address()

    def calls(eps, side):
        norms = dict(post=atb.NormArgs(a, a, 1e-5, kind), pre=atb.NormArgs(a, a, 1e-5, kind))
        norms[side].eps = eps
        p = atb.ResidualNorm(a, a, 8, 8, norms["post"], norms["pre"], None, 1, 1.0, 0, 8, 0, 0, 0)
        g = atb.ResidualNormGradArgs()
        return (L.atb_residual_norm_forward(ctypes.byref(p), a, 8, a, 8, a, None), L.atb_residual_norm_backward(ctypes.byref(p), a, a, 8, a, 8, ctypes.byref(g), None, None))
    for side in ("post", "pre"):
        assert calls(eps, side) == (INVALID, INVALID)
        for good in (0.0, 1e-45, 1e-40, 1e-5, 3.4e38):                          # (1e-45: the smallest that fp32 holds)
            assert calls(good, side) == (0, 0), good
        nothing = atb.NormArgs(None, None, eps, 0)                              # not looked at
        assert L.atb_residual_norm_forward(ctypes.byref(atb.ResidualNorm(a, a, 8, 8, nothing, nothing, None, 1, 1.0, 0, 8, 0, 0, 0)), a, 8, None, 8, a, None) == 0


def test_workspace_of_a_residual_norm():
    L = atb.lib()
    for M in (0, 6, 600, 60000, 2 ** 23 - 2 ** 23 % 6):
        for D in (1, 4096, 8193, 2 ** 24):
            for groups in (1, 2, 6):
                assert L.atb_residual_norm_workspace(M, D, groups) >= (16 * D * groups if M else 0) and L.atb_residual_norm_workspace(M, D, groups) % 16 == 0
    assert L.atb_residual_norm_workspace(8192, 4096, 1) <= 32 << 20
    for bad in ((-1, 8, 1), (4, 0, 1), (4, 8, 0), (4, 8, 3), (2 ** 23 + 1, 8, 1), (4, 2 ** 24 + 1, 1), (65536, 8, 65536)):
        assert L.atb_residual_norm_workspace(*bad) == 0


def test_residual_norm_refuses_tensors_that_a_kernel_would_read_or_store_past():
    import torch
    bf, f32 = torch.bfloat16, torch.float32
    x, v = _on_device((4, 64), bf), _on_device((64,), bf)
    wide = _on_device((4, 64), f32)
    for args in [(torch.zeros(4, 64, dtype=bf), x), (x, _on_device((4, 63), bf)), (x, _on_device((3, 64), bf)), (_on_device((4, 64), torch.float16), x), (x, _on_device((4, 64), bf, (1, 4))),
                 (x, x, atb.Norm("rms", _on_device((63,), bf))), (x, x, atb.Norm("rms", v, _on_device((64,), f32))), (x, x, atb.Norm("rms", v), _on_device((64,), f32)), (x, x, atb.Norm("rms", torch.zeros(64, dtype=bf))),
                 (x, x, None, _on_device((2, 64), bf, (128, 1))), (x, x, None, _on_device((2, 63), bf)), (x, x, None, _on_device((1, 1, 64), bf)), (x, x, None, v, 1.0, atb.Norm("rms", _on_device((64,), bf, (2,))))]:
        with pytest.raises(AssertionError):
            atb.residual_norm(*args)
    for args in [(x, x, None, _on_device((3, 64), bf)), (x, x, None, _on_device((0, 64), bf)), (x, wide)]:       # 4 rows in 3 groups, in none, a block wider than the stream
        with pytest.raises(AssertionError):
            atb.residual_norm(*args)
    with pytest.raises(ValueError, match="rms"):
        atb.residual_norm(x, x, atb.Norm("batch"))
    stats = _on_device((4, 4), f32)
    pre = atb.Norm("rms", v)
    for dr, dh, st, norm in [(_on_device((4, 63), bf), x, stats, pre), (wide, x, stats, pre), (x, None, stats, pre), (x, x, stats, None), (x, wide, stats, pre), (x, x, _on_device((4, 3), f32), pre),
                             (x, x, _on_device((4, 4), bf), pre), (x, x, _on_device((4, 4), f32, (1, 4)), pre)]:
        with pytest.raises(AssertionError):
            atb.residual_norm_backward(dr, dh, x, x, st, None, None, 1.0, norm)


@pytest.mark.parametrize("post,pre,groups", [("rms", "rms", 1), ("layer", "layer", 2), (None, "rms", 0), ("layer", None, 4)])
def test_residual_norm_gradients_against_differences(post, pre, groups):
    """The formulas that the GPU tests compare with."""
    import torch
    from test_gpu_residual import inputs, reference
    a = inputs(4, 10, torch.float64, torch.float64, torch.float64, post, pre, groups=groups, seed=2, device="cpu")
    want = reference(a)

    def loss(b):
        out = reference(b)
        return (out["r"][0] * a["dr"]).sum() + ((out["h"][0] * a["dh"]).sum() if pre else 0)
    names = ["dx", "dz"] + ["dgate"] * (groups > 0) + [f"d{s}_{w}" for s, n in (("post", post), ("pre", pre)) if n for w in ("weight", "bias")]
    g = torch.Generator().manual_seed(3)
    for name in names:
        side, _, which = name[1:].partition("_")
        here = getattr(a[side], which) if which else a[side]
        v = torch.randn(here.shape, generator=g, dtype=torch.float64)

        def moved(t):
            return loss({**a, side: a[side]._replace(**{which: t}) if which else t})
        slope = _slope(moved, (here,), 0, v)
        grad = float((want[name][0].reshape(here.shape) * v).sum())
        assert abs(slope - grad) < 1e-6 * (1 + abs(grad)), name


# ------------------------------------------------------------------ a mixture of experts for few tokens

def test_moe_refuses():
    L = atb.lib()
    keep, a = aligned_address()
    bf16, q4, z4 = atb.MoeWeight(a, None, None), atb.MoeWeight(a, a, None), atb.MoeWeight(a, a, a)
    good = dict(x=a, router=a, ldx=64, ld_router=64, w_gate=bf16, w_up=bf16, w_down=bf16, M=2, D=64, F=64, experts=4, top_k=2, group=0, act=0, renormalize=1, workspace=a)

    def forward(y=a, ldy=64, chosen=a, p=a, **kw):
        return L.atb_moe_forward(ctypes.byref(atb.Moe(**{**good, **kw})), y, ldy, chosen, p, None)
    in_4 = dict(w_gate=q4, w_up=q4, w_down=q4)
    for bad in [dict(x=None), dict(router=None), dict(x=a + 2), dict(router=a + 8), dict(ldx=56), dict(ldx=68), dict(ld_router=63), dict(ld_router=2 ** 22), dict(M=-1), dict(M=65), dict(D=0), dict(D=60), dict(F=4),
                dict(D=2 ** 22, ldx=2 ** 22, ld_router=2 ** 22), dict(F=2 ** 22), dict(experts=0), dict(experts=257), dict(top_k=0), dict(top_k=5), dict(experts=40, top_k=17), dict(group=16), dict(group=-32), dict(act=3),
                dict(act=-1), dict(workspace=None), dict(workspace=a + 8), dict(y=None), dict(y=a + 1), dict(ldy=63), dict(chosen=a + 2), dict(p=a + 2), dict(w_gate=atb.MoeWeight(None, None, None)),
                dict(w_up=atb.MoeWeight(a + 8, None, None)), dict(w_down=atb.MoeWeight(None, a, a)), dict(group=32), dict(group=32, w_gate=q4, w_up=q4), dict(group=32, w_gate=z4, w_up=q4, w_down=q4),
                dict(group=32, w_gate=q4, w_up=q4, w_down=z4), dict(group=128, **in_4), dict(group=64, F=96, **in_4), dict(group=32, w_gate=atb.MoeWeight(a, a + 1, None), w_up=q4, w_down=q4)]:
        assert forward(**bad) == INVALID, bad
    assert L.atb_moe_forward(None, a, 64, a, a, None) == INVALID
    assert forward(M=0, x=None, y=None, workspace=None) == 0
    if not __import__("torch").cuda.is_available():
        assert forward() == forward(chosen=None, p=None) == forward(group=32, **in_4) == forward(group=64, w_gate=z4, w_up=z4, w_down=z4) == forward(M=40, experts=2) == 5


def test_workspace_of_a_mixture_of_experts():
    L = atb.lib()
    for M, D, F, E, k in ((0, 8, 8, 1, 1), (1, 8, 8, 1, 1), (1, 4096, 14336, 8, 2), (64, 2048, 14336, 256, 16)):
        size = L.atb_moe_workspace(M, D, F, E, k, 0)
        assert size % 256 == 0 and size >= 8 * M * E + 2 * M * k * F + 8 * 1024
        if D % 128 == 0:
            assert L.atb_moe_workspace(M, D, F, E, k, 128) >= 8 * M * E + 2 * M * k * F + 8 * 1024
    for bad in ((-1, 8, 8, 4, 2, 0), (65, 8, 8, 4, 2, 0), (1, 8, 12, 4, 2, 0), (1, 8, 0, 4, 2, 0), (1, 4, 8, 4, 2, 0), (1, 8, 2 ** 22, 4, 2, 0), (1, 8, 8, 0, 1, 0), (1, 8, 8, 257, 1, 0), (1, 8, 8, 4, 0, 0),
                (1, 8, 8, 4, 5, 0), (1, 8, 8, 40, 17, 0), (1, 64, 64, 4, 2, 16), (1, 64, 96, 4, 2, 64)):
        assert L.atb_moe_workspace(*bad) == 0


def test_moe_refuses_tensors_that_a_kernel_would_read_or_store_past():
    import torch
    bf, f32, u8 = torch.bfloat16, torch.float32, torch.uint8
    x, r = _on_device((3, 64), bf), _on_device((4, 64), bf)
    up, down = _on_device((4, 128, 64), bf), _on_device((4, 64, 128), bf)
    for args in [(torch.zeros(3, 64, dtype=bf), r, up, up, down), (_on_device((3, 64), f32), r, up, up, down), (x, _on_device((4, 56), bf), up, up, down), (x, _on_device((4, 64), f32), up, up, down),
                 (x, _on_device((5, 64), bf), up, up, down), (x, r, up, down, down), (x, r, up, up, up), (x, r, up, _on_device((4, 120, 64), bf), down), (x, r, _on_device((4, 128, 64), f32), up, down),
                 (x, r, _on_device((4, 128, 64), bf, (16384, 128, 1)), up, down), (x, r, up, up, _on_device((4, 64, 128), bf, (8192, 1, 64))), (x, r, up, up, torch.zeros(4, 64, 128, dtype=bf)),
                 (x, r, up, up, down, 0), (x, r, up, up, down, 5), (x, r, _on_device((512, 64), bf), up, down)]:
        with pytest.raises(AssertionError):
            atb.moe_feed_forward(*args)

    def q4(rows, cols, group=32, zeros=False):
        return atb.Q4Weight(_on_device((rows, cols // 2), u8), _on_device((rows, cols // group), bf), _on_device((rows, cols // group), u8) if zeros else None)
    good = (x, r, q4(512, 64), q4(512, 64), q4(256, 128))
    for at, w in [(2, q4(511, 64)), (2, q4(512, 128)), (3, q4(256, 64)), (4, q4(512, 64)), (4, q4(256, 128, 64)), (3, q4(512, 64, 32, True)), (2, up), (4, down), (2, q4(512, 64)._replace(scales=_on_device((512, 2), f32)))]:
        with pytest.raises(AssertionError):
            atb.moe_feed_forward(*good[:at], w, *good[at + 1:])
    with pytest.raises(ValueError, match="silu"):
        atb.moe_feed_forward(x, r, up, up, down, 2, "swish")
    with pytest.raises(TypeError):
        atb.moe_feed_forward(x, r, up, None, down)


# ------------------------------------------------------------------ the host code under sanitizers

def test_the_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    """atb_block_api.cpp and the rules of atb_block.h, which decide the sizes of buffers that kernels write."""
    from test_host_sanitizers import CSRC, NATIVE, ROCM_INC, ROOT
    if shutil.which("g++") is None or not os.path.isdir(ROCM_INC):
        pytest.skip("needs g++ and the HIP headers")
    exe = str(tmp_path / "sanitize_block")
    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-static-libasan", "-static-libubsan", "-fno-omit-frame-pointer", "-g", "-O1"]
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", ROCM_INC, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-Wno-deprecated-declarations",
                    os.path.join(NATIVE, "sanitize_block.cpp"), os.path.join(NATIVE, "stub_device.cpp"), os.path.join(CSRC, "atb_api.cpp"), os.path.join(CSRC, "atb_model.cpp"),
                    os.path.join(CSRC, "atb_block_api.cpp"), "-o", exe, "-lm"] + san, check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], env=env, capture_output=True, text=True, timeout=120)
    out = r.stdout + r.stderr
    assert r.returncode == 0 and "sanitize_block: ok" in r.stdout, out
    assert "AddressSanitizer" not in out and "runtime error" not in out, out
