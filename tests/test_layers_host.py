"""The feed-forward sublayer's operators without a GPU: what their entry points refuse, and the gradients' formulas against differences."""
import ctypes
import math
import os
import subprocess
import sys
import textwrap

import pytest

import paper_2511_16041_amd as atb
from test_abi_host import _on_device

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID = 1


def aligned_address():
    buf = ctypes.create_string_buffer(4096)
    return buf, (ctypes.addressof(buf) + 255) & ~255


def test_layer_norm_refuses():
    L = atb.lib()
    keep, a = aligned_address()

    def norm(x=a, ldx=8, w=a, b=a, eps=1e-5, y=a, ldy=8, mean=a, rstd=a, M=2, D=8, t=0, pt=0):
        return L.atb_layer_norm(x, ldx, w, b, eps, y, ldy, mean, rstd, M, D, t, pt, None)
    for bad in (dict(x=None), dict(y=None), dict(ldx=7), dict(ldy=7), dict(D=0), dict(D=-1), dict(D=2 ** 24 + 1), dict(M=-1), dict(M=2 ** 23 + 1), dict(t=2), dict(pt=-1), dict(eps=-1.0),
                dict(eps=math.nan), dict(x=a + 1), dict(y=a + 1), dict(w=a + 1), dict(x=a + 2, t=1), dict(w=a + 2, pt=1), dict(mean=a + 2)):
        assert norm(**bad) == INVALID, bad
    assert norm(M=0, x=None, y=None) == 0

    def back(dy=a, lddy=8, x=a, ldx=8, mean=a, rstd=a, w=a, dx=a, lddx=8, dw=a, db=a, ws=a, M=2, D=8, t=0, pt=0):
        return L.atb_layer_norm_backward(dy, lddy, x, ldx, mean, rstd, w, dx, lddx, dw, db, ws, M, D, t, pt, None)
    for bad in (dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(ws=None), dict(ws=a + 4), dict(lddx=7), dict(lddy=0), dict(D=0), dict(M=-3), dict(t=9)):
        assert back(**bad) == INVALID, bad
    assert L.atb_layer_norm_workspace(0, 8) == 0 and L.atb_layer_norm_workspace(5, 0) == 0
    for M, D in ((1, 1), (1000, 4096), (5, 40000)):
        assert L.atb_layer_norm_workspace(M, D) >= 8 * D


def test_feed_forward_refuses():
    L = atb.lib()
    keep, a = aligned_address()
    good = dict(x=a, w_gate=a, w_up=a, w_down=a, ldx=8, ld_gate=8, ld_up=8, ld_down=16, M=2, D=8, F=16, act=0)

    def forward(h=a, kept=a, y=a, ldy=8, **kw):
        f = atb.Ffn(**{**good, **kw})
        return L.atb_ffn_forward(ctypes.byref(f), h, kept, y, ldy, None)
    bad_blocks = [dict(x=None), dict(w_gate=None), dict(w_up=None), dict(w_down=None), dict(x=a + 2), dict(w_up=a + 8), dict(ldx=12), dict(ld_gate=7), dict(ld_down=8), dict(ld_up=2 ** 22),
                  dict(M=-1), dict(M=2 ** 23 + 1), dict(D=0), dict(D=12), dict(F=4), dict(F=2 ** 22), dict(act=3), dict(act=-1)]
    for bad in bad_blocks + [dict(h=None), dict(y=None), dict(h=a + 2), dict(kept=a + 2), dict(ldy=7), dict(ldy=12)]:
        assert forward(**bad) == INVALID, bad
    assert L.atb_ffn_forward(None, a, a, a, 8, None) == INVALID
    assert forward(M=0, x=None, h=None, y=None) == 0
    assert L.atb_ffn_kept_bytes(7, 24) == 6 * 7 * 24 and L.atb_ffn_kept_bytes(7, 12) == 0

    def backward(h=a, kept=a, dy=a, lddy=8, dg=a, du=a, dx=a, lddx=8, dwg=a, dwu=a, dwd=a, **kw):
        f = atb.Ffn(**{**good, **kw})
        return L.atb_ffn_backward(ctypes.byref(f), h, kept, dy, lddy, dg, du, dx, lddx, dwg, dwu, dwd, None)
    for bad in bad_blocks + [dict(h=None), dict(kept=None), dict(dy=None), dict(lddy=4), dict(dg=None), dict(du=a + 2), dict(dx=a + 2), dict(lddx=0), dict(dwg=None), dict(dwu=None), dict(dwd=a + 8)]:
        assert backward(**bad) == INVALID, bad
    assert backward(M=0, dwg=None, dwu=None, dwd=None, x=None, dy=None) == 0


def test_q4_refuses():
    L = atb.lib()
    keep, a = aligned_address()
    good = dict(packed=a, scales=a, zeros=None, N=4, K=64, group=32)

    def matvec(x=a, ldx=64, y=a, ldy=4, t=0, M=1, **kw):
        w = atb.Q4(**{**good, **kw})
        return L.atb_q4_matvec(ctypes.byref(w), x, ldx, y, ldy, t, M, None)
    bad_weights = [dict(packed=None), dict(packed=a + 8), dict(scales=None), dict(scales=a + 1), dict(N=0), dict(K=0), dict(K=48), dict(K=2 ** 22 + 32), dict(group=16), dict(group=256), dict(group=0)]
    for bad in bad_weights + [dict(x=None), dict(y=None), dict(ldx=56), dict(ldx=68), dict(x=a + 2), dict(ldy=3), dict(t=5), dict(M=-1), dict(M=2 ** 23 + 1), dict(y=a + 2, t=1)]:
        assert matvec(**bad) == INVALID, bad
    assert L.atb_q4_matvec(None, a, 64, a, 4, 0, 1, None) == INVALID
    assert matvec(M=0, x=None, y=None) == 0

    def gated(up=None, act=0, **kw):
        w, v = atb.Q4(**{**good, **kw}), atb.Q4(**{**good, **(up or {})})
        return L.atb_q4_gated(ctypes.byref(w), ctypes.byref(v), act, a, 64, a, 4, 1, None)
    for bad in [dict(act=7), dict(up=dict(N=5)), dict(up=dict(K=96)), dict(up=dict(group=64)), dict(up=dict(zeros=a)), dict(zeros=a)] + bad_weights:
        assert gated(**bad) == INVALID, bad
    assert L.atb_q4_quantize(None, 64, 1, a, a, None, 4, 64, 32, None) == INVALID
    assert L.atb_q4_quantize(a, 63, 1, a, a, None, 4, 64, 32, None) == INVALID
    w = atb.Q4(**good)
    assert L.atb_q4_decode(ctypes.byref(w), None, 1, None) == INVALID


def test_device_calls_refuse_what_a_kernel_would_read_or_store_past():
    """The binding: host tensors, other types, shapes and layouts, before anything is launched."""
    import torch
    bf, f32, u8 = torch.bfloat16, torch.float32, torch.uint8
    x = _on_device((4, 64), bf)
    v = _on_device((64,), bf)
    bad_norm = [(torch.zeros(4, 64), None, None), (_on_device((4, 64), torch.float16), None, None), (_on_device((64,), bf), None, None), (_on_device((4, 64), bf, (1, 4)), None, None),
                (_on_device((4, 64), bf, (32, 1)), None, None), (x, _on_device((63,), bf), None), (x, v, _on_device((64,), f32)), (x, _on_device((64,), bf, (2,)), None), (x, torch.zeros(64, dtype=bf), None)]
    for args in bad_norm:
        with pytest.raises(AssertionError):
            atb.layer_norm(*args)
    stat = _on_device((4,), f32)
    for args in [(_on_device((4, 63), bf), x, stat, stat), (_on_device((4, 64), f32), x, stat, stat), (x, x, _on_device((3,), f32), stat), (x, x, stat, _on_device((4,), bf)),
                 (x, x, stat, stat, _on_device((65,), bf))]:
        with pytest.raises(AssertionError):
            atb.layer_norm_backward(*args)
    wg, wd = _on_device((128, 64), bf), _on_device((64, 128), bf)
    for args in [(torch.zeros(4, 64, dtype=bf), wg, wg, wd), (_on_device((4, 64), f32), wg, wg, wd), (x, wg, _on_device((120, 64), bf), wd), (x, wg, wg, wg), (x, _on_device((128, 56), bf), wg, wd),
                 (x, _on_device((128, 64), bf, (1, 128)), wg, wd)]:
        with pytest.raises(AssertionError):
            atb.feed_forward(*args)
    state = atb.FeedForwardState(_on_device((4, 128), bf), _on_device((6 * 4 * 128,), u8), "silu")
    for dy, st in [(_on_device((3, 64), bf), state), (x, state._replace(h=_on_device((4, 120), bf))), (x, state._replace(kept=_on_device((6 * 4 * 128 - 1,), u8))), (x, state._replace(h=_on_device((4, 128), bf, (256, 1))))]:
        with pytest.raises(AssertionError):
            atb.feed_forward_backward(dy, x, wg, wg, wd, st)
    w = atb.Q4Weight(_on_device((128, 32), u8), _on_device((128, 2), bf))
    for a, q in [(torch.zeros(4, 64, dtype=bf), w), (_on_device((4, 56), bf), w), (_on_device((4, 64), f32), w), (x, w._replace(packed=_on_device((128, 32), torch.int8))), (x, w._replace(scales=_on_device((127, 2), bf))),
                 (x, w._replace(scales=_on_device((128, 2), f32))), (x, w._replace(zeros=_on_device((128, 1), u8))), (x, w._replace(packed=_on_device((128, 32), u8, (64, 1))))]:
        with pytest.raises(AssertionError):
            atb.q4_matvec(a, q)
    with pytest.raises(AssertionError):
        atb.q4_feed_forward(x, w, w, w)                      # the down projection's inputs are not the gate's outputs
    for bad in (torch.zeros(4, 64), _on_device((4, 64), torch.float16), _on_device((4, 48), f32)):
        with pytest.raises(AssertionError):
            atb.q4_quantize(bad, 32)
    with pytest.raises(AssertionError):
        atb.q4_quantize(x, 16)
    with pytest.raises(ValueError, match="silu"):
        atb.feed_forward(x, wg, wg, wd, "swish")
    with pytest.raises(ValueError, match="float32"):
        atb.q4_matvec(x, w, torch.float16)


def test_launch_without_a_device_returns_hip_error():
    code = textwrap.dedent("""
        import ctypes, sys
        sys.path.insert(0, %r)
        import paper_2511_16041_amd as atb
        L = atb.lib()
        buf = ctypes.create_string_buffer(1 << 16)
        a = (ctypes.addressof(buf) + 255) & ~255
        f = atb.Ffn(a, a, a, a, 8, 8, 8, 16, 2, 8, 16, 0)
        w = atb.Q4(a, a, None, 8, 64, 32)
        assert L.atb_layer_norm(a, 8, a, a, 1e-5, a, 8, a, a, 2, 8, 0, 0, None) == 5
        assert L.atb_layer_norm_backward(a, 8, a, 8, a, a, a, a, 8, a, a, a, 2, 8, 0, 0, None) == 5
        assert L.atb_ffn_forward(ctypes.byref(f), a, None, a, 8, None) == 5 and L.atb_ffn_forward(ctypes.byref(f), a, a, a, 8, None) == 5
        assert L.atb_ffn_backward(ctypes.byref(f), a, a, a, 8, a, a, a, 8, a, a, a, None) == 5
        assert L.atb_q4_matvec(ctypes.byref(w), a, 64, a, 8, 0, 1, None) == 5 and L.atb_q4_gated(ctypes.byref(w), ctypes.byref(w), 0, a, 64, a, 8, 1, None) == 5
        assert L.atb_q4_quantize(a, 64, 1, a, a, None, 8, 64, 32, None) == 5 and L.atb_q4_decode(ctypes.byref(w), a, 1, None) == 5
        assert L.atb_last_hip_error() != 0
        print("no-device ok")
    """ % ROOT)
    env = dict(os.environ, HIP_VISIBLE_DEVICES="", ROCR_VISIBLE_DEVICES="", CUDA_VISIBLE_DEVICES="")
    r = subprocess.run([sys.executable, "-c", code], env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "no-device ok" in r.stdout, r.stdout + r.stderr


# ------------------------------------------------------------------ the formulas that the GPU tests compare with, against differences in 64 bits

def _slope(f, args, at, v, h=1e-5):
    def moved(sign):
        return f(*[a + sign * h * v if i == at else a for i, a in enumerate(args)])
    return float((moved(1) - moved(-1)) / (2 * h))


def test_layer_norm_gradients_against_differences():
    import torch
    g = torch.Generator().manual_seed(0)
    x, w, b, dy = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((5, 12), (12,), (12,), (5, 12)))
    eps = 1e-3

    def loss(x, w, b):
        mean, var = x.mean(1, keepdim=True), x.var(1, keepdim=True, unbiased=False)
        return (((x - mean) / (var + eps).sqrt() * w + b) * dy).sum()
    mean = x.mean(1, keepdim=True)
    r = 1 / (((x - mean) ** 2).mean(1, keepdim=True) + eps).sqrt()
    xh = (x - mean) * r
    gw = dy * w
    grads = [r * (gw - gw.mean(1, keepdim=True) - xh * (gw * xh).mean(1, keepdim=True)), (dy * xh).sum(0), dy.sum(0)]
    for at, (arg, grad) in enumerate(zip((x, w, b), grads)):
        v = torch.randn(arg.shape, generator=g, dtype=torch.float64)
        assert abs(_slope(loss, (x, w, b), at, v) - float((grad * v).sum())) < 1e-7


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_feed_forward_gradients_against_differences(act):
    import torch
    from test_gpu_ffn import activation
    g = torch.Generator().manual_seed(1)
    x, wg, wu, wd, dy = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((3, 6), (8, 6), (8, 6), (6, 8), (3, 6)))

    def loss(x, wg, wu, wd):
        return (((activation(act, x @ wg.t())[0] * (x @ wu.t())) @ wd.t()) * dy).sum()
    gate, up = x @ wg.t(), x @ wu.t()
    a, slope = activation(act, gate)
    dh = dy @ wd
    dg, du = dh * up * slope, dh * a
    grads = [dg @ wg + du @ wu, dg.t() @ x, du.t() @ x, dy.t() @ (a * up)]
    for at, (arg, grad) in enumerate(zip((x, wg, wu, wd), grads)):
        v = torch.randn(arg.shape, generator=g, dtype=torch.float64)
        want = float((grad * v).sum())
        assert abs(_slope(loss, (x, wg, wu, wd), at, v) - want) < 1e-6 * (1 + abs(want))


def test_workspace_of_a_gated_block():
    L = atb.lib()
    for M in (1, 33, 64, 100, 257, 1000, 4096, 8192):
        for D in (64, 1032, 8192):
            for F in (64, 1544, 16384):
                for size in (L.atb_ffn_workspace(M, D, F, 0), L.atb_ffn_workspace(M, D, F, 1), L.atb_ffn_backward_workspace(M, D, F)):
                    assert 0 <= size <= 64 << 20 and size % 16 == 0, (M, D, F)
    assert L.atb_ffn_workspace(1, 4096, 14336, 0) == 0 < L.atb_ffn_workspace(1, 4096, 14336, 1)
    for bad in ((-1, 64, 64), (1, 60, 64), (1, 64, 0), (2 ** 23 + 1, 64, 64), (1, 2 ** 22, 64)):
        assert L.atb_ffn_workspace(*bad, 1) == 0 and L.atb_ffn_backward_workspace(*bad) == 0
    assert L.atb_ffn_backward_workspace(0, 64, 64) == 0


@pytest.mark.parametrize("mistake", ["g and u in bf16", "dh in bf16"])
def test_the_bound_on_the_blocks_error_sees_one_more_rounding(mistake):
    """The bound of test_gpu_ffn_error.py, with the mistake made in the oracle: every gradient that it touches is outside."""
    import torch
    from test_gpu_ffn import activation
    from test_gpu_ffn_error import MARGIN, block, rounded
    gen = torch.Generator().manual_seed(3)
    x, wg, wu, wd, dy = ((s * torch.randn(shape, generator=gen)).bfloat16().double() for s, shape in ((1, (200, 264)), (0.05, (520, 264)), (0.05, (520, 264)), (0.05, (264, 520)), (0.1, (200, 264))))
    exact, model = block(x, wg, wu, wd, dy, "silu", lambda t: t), block(x, wg, wu, wd, dy, "silu", rounded)
    g, u, dh = x @ wg.t(), x @ wu.t(), dy @ wd
    if mistake == "dh in bf16":
        dh = rounded(dh)
    else:
        g, u = rounded(g), rounded(u)
    a, slope = activation("silu", g)
    dg, du = rounded(dh * u * slope), rounded(dh * a)
    for name, y in (("dx", dg @ wg + du @ wu), ("dwg", dg.t() @ x), ("dwu", du.t() @ x)):
        off, allowed = (float((t - exact[name]).norm() / exact[name].norm()) for t in (rounded(y), model[name]))
        assert off > 1.1 * MARGIN * allowed, name
