"""4-bit weights on the GPU: storage against its definition, products against 64 bits.

Tolerances of the products.  The accumulators sum (c + q) x over a group, with c = 16 or at most 128, so at most 143 |x| a term and up to 128 terms, and subtract (c + z) times the sum of
x: 2^-20 of 143 s sum |x| covers the roundings of such a chain (128 of 2^-24, added as a random walk: 11 of them); adding groups costs 2^-20 of the result's terms.  A bf16 result adds 2^-8 of its
size; the block's inner activations are rounded to bf16, 2^-8 of theirs."""
import numpy as np
import pytest
import torch

import paper_2511_16041_amd as atb

pytestmark = pytest.mark.gpu
E, R = 2.0 ** -20, 2.0 ** -8


def codes(packed):
    q = torch.empty((packed.shape[0], 2 * packed.shape[1]), dtype=torch.int64, device=packed.device)
    q[:, ::2], q[:, 1::2] = (packed & 15).long(), (packed >> 4).long()
    return q


def values(w):
    q = codes(w.packed).double()
    group = q.shape[1] // w.scales.shape[1]
    z = w.zeros.double().repeat_interleave(group, 1) if w.zeros is not None else 8.0
    return (q - z) * w.scales.double().repeat_interleave(group, 1)


def steps(w):
    """The scale of every element."""
    return w.scales.double().repeat_interleave(2 * w.packed.shape[1] // w.scales.shape[1], 1)


def random_weight(N, K, group, zeros, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    packed = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = (0.01 * torch.rand((N, K // group), generator=g, device="cuda") + 0.001).bfloat16()
    return atb.Q4Weight(packed, scales, torch.randint(0, 16, (N, K // group), generator=g, device="cuda", dtype=torch.uint8) if zeros else None)


def rows(M, K, seed, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((M, K + pad), generator=g, device="cuda").bfloat16()
    x[:, K:] = float("nan")
    return x[:, :K]


def check(y, x, w):
    ref = x.double() @ values(w).t()
    tol = E * 143 * (x.double().abs() @ steps(w).t()) + E * ref.abs()
    if y.dtype == torch.bfloat16:
        tol = tol + R * ref.abs()
    off = (y.double() - ref).abs()
    assert y.shape == ref.shape and bool((off <= tol).all()), float((off / tol).max())


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("M,N,groups", [(1, 1, 1), (1, 16, 2), (2, 17, 3), (5, 33, 5), (16, 100, 8), (17, 31, 9), (32, 64, 11), (33, 513, 16), (64, 40, 17), (70, 48, 33), (1, 4096, 32), (3, 257, 129)])
def test_matvec(M, N, groups, group, zeros):
    K = group * groups
    w, x = random_weight(N, K, group, zeros, M + N + K), rows(M, K, K)
    check(atb.q4_matvec(x, w), x, w)
    wide = atb.q4_matvec(x, w, torch.float32)
    assert wide.dtype == torch.float32
    check(wide, x, w)
    assert torch.equal(wide, atb.q4_matvec(x, tuple(w), torch.float32))


@pytest.mark.parametrize("M", [1, 20])
def test_rows_further_apart_and_single_rows(M):
    w = random_weight(50, 352, 32, True, 1)
    x = rows(M, 352, 2, pad=40)
    check(atb.q4_matvec(x, w, torch.float32), x, w)


def test_a_row_does_not_depend_on_the_others():
    w, x = random_weight(77, 1056, 32, True, 3), rows(16, 1056, 4)
    y = atb.q4_matvec(x, w, torch.float32)
    for i in (0, 7, 15):
        assert torch.equal(atb.q4_matvec(x[i:i + 1], w, torch.float32), y[i:i + 1])
    bad = x.clone()
    bad[3, 1055] = float("nan")
    z = atb.q4_matvec(bad, w, torch.float32)
    assert z[3].isnan().all()
    keep = [i for i in range(16) if i != 3]
    assert torch.equal(z[keep], y[keep])


def test_parts_of_a_larger_weight():
    """Some rows of a weight: codes, scales and zero points that begin anywhere a row does (an odd number of groups: at 2 bytes)."""
    w, x = random_weight(64, 416, 32, True, 5), rows(4, 416, 6)
    part = atb.Q4Weight(w.packed[5:38], w.scales[5:38], w.zeros[5:38])
    check(atb.q4_matvec(x, part), x, part)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("M,D,F,group,zeros", [(1, 256, 512, 64, True), (3, 416, 96, 32, False), (16, 512, 1024, 128, True), (40, 192, 320, 64, False)])
def test_gated_block(M, D, F, group, zeros, act):
    from test_gpu_ffn import activation
    wg, wu, wd = random_weight(F, D, group, zeros, 7), random_weight(F, D, group, zeros, 8), random_weight(D, F, group, zeros, 9)
    x = rows(M, D, 10)
    g, u = x.double() @ values(wg).t(), x.double() @ values(wu).t()
    a, _ = activation(act, g)
    h = a * u
    e_g, e_u = (E * 143 * (x.double().abs() @ steps(w).t()) for w in (wg, wu))
    e_a = 1.2 * e_g + 2.0 ** -19 * a.abs() + 2.0 ** -21
    e_h = e_a * u.abs() + a.abs() * e_u + e_a * e_u + R * h.abs()
    ref = h @ values(wd).t()
    tol = e_h @ values(wd).abs().t() + E * 143 * (h.abs() @ steps(wd).t()) + R * ref.abs()
    y = atb.q4_feed_forward(x, wg, wu, wd, act)
    off = (y.double() - ref).abs()
    assert bool((off <= tol).all()), float((off / tol).max())


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,groups", [(1, 1), (3, 5), (70, 8), (257, 3)])
def test_quantise_and_decode(N, groups, group, zeros, dtype):
    """Codes, scales and zero points equal the definition, computed with numpy's IEEE fp32; the values equal s (q - z)."""
    K = group * groups
    gen = torch.Generator(device="cuda").manual_seed(N + K)
    wide = (0.02 * torch.randn((N, K + 8), generator=gen, device="cuda")).to(dtype)
    wide[0, :group] = 0                               # a group of zeros
    if groups > 2:
        wide[0, group:2 * group] = wide[0, group:2 * group].abs()
        wide[0, 2 * group:3 * group] = -wide[0, 2 * group:3 * group].abs()
    w = wide[:, :K]
    got = atb.q4_quantize(w, group, zeros)
    f = w.float().cpu().numpy().reshape(N, groups, group)
    hi, lo = np.maximum(f.max(2), 0), np.minimum(f.min(2), 0)
    step = (hi - lo) / np.float32(15) if zeros else np.maximum(hi, -lo) / np.float32(7)
    s = torch.from_numpy(step).bfloat16()
    sf = s.float().numpy()
    safe = np.where(sf > 0, sf, np.float32(1))
    z = np.clip(np.rint(-lo / safe), 0, 15) if zeros else np.full_like(sf, 8)
    z = np.where(sf > 0, z, 0 if zeros else 8).astype(np.float32)
    q = np.where(sf[..., None] > 0, np.clip(np.rint(f / safe[..., None]) + z[..., None], 0, 15), z[..., None]).reshape(N, K)
    assert torch.equal(got.scales.cpu(), s)
    assert np.array_equal(codes(got.packed).cpu().numpy(), q.astype(np.int64))
    assert (got.zeros is None) == (not zeros)
    if zeros:
        assert np.array_equal(got.zeros.cpu().numpy(), z.astype(np.uint8))
    exact = values(got)
    assert torch.equal(atb.q4_decode(got, torch.float32).double(), exact)
    assert torch.equal(atb.q4_decode(got), exact.bfloat16())
    # half a step of the code, 2^-8 of the scale's rounding over 15 codes, the ends cut off by that
    assert bool(((exact - w.double()).abs() <= steps(got) * (0.5 + 15 * R) + 1e-12).all())


def test_no_rows():
    w = random_weight(40, 128, 32, False, 1)
    assert atb.q4_matvec(torch.empty((0, 128), dtype=torch.bfloat16, device="cuda"), w).shape == (0, 40)


def test_another_stream():
    w, x = random_weight(600, 4096, 128, True, 11), rows(2, 4096, 12)
    first = atb.q4_matvec(x, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = atb.q4_matvec(x, w, stream=side)
    side.synchronize()
    assert torch.equal(first, again)


def test_rows_of_more_than_one_launch():
    """65535 blocks of 16 rows a launch: every row, on both sides of that."""
    w, x = random_weight(24, 64, 32, True, 13), rows(65535 * 16 + 5, 64, 14, pad=8)
    check(atb.q4_matvec(x, w, torch.float32), x, w)


@pytest.mark.parametrize("zeros", [False, True])
def test_quantise_the_largest_numbers(zeros):
    """Finite weights whose range, the largest less the smallest, passes fp32's: scale and codes are still the formula's, taken in 64 bits."""
    w = torch.tensor([[3.0e38, -2.6e38] * 16, [1.0e38, -3.3e38] * 16, [3.2e38, -0.0] * 16], device="cuda")
    got = atb.q4_quantize(w, 32, zeros)
    hi, lo = w.double().amax(1, keepdim=True).clamp(min=0), w.double().amin(1, keepdim=True).clamp(max=0)
    s = ((hi - lo) / 15 if zeros else torch.maximum(hi, -lo) / 7).bfloat16()
    z = torch.round(-lo / s.double()).clamp(0, 15) if zeros else torch.full_like(hi, 8)
    assert torch.equal(got.scales, s)
    assert torch.equal(codes(got.packed).double(), (torch.round(w.double() / s.double()) + z).clamp(0, 15))
    assert got.zeros is None or torch.equal(got.zeros.double(), z)
