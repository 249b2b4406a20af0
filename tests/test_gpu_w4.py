"""4-bit weights: the layout against the format's rule (bit-exact) and the matrix-vector products against
the same sums in 64 bits, within bounds that follow from the arithmetic."""
import numpy as np
import pytest
import torch

import paper_2410_18311_b200 as ci
from helpers import require_gpu
from quant4_ref import EPS32, OUT_EPS, values_np, w4_layout

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def lay_out(w, group):
    """Quantises w [N, K] (CUDA, any strides) with the library; (codes, pairs, descriptor)."""
    N, K = w.shape
    codes = torch.full((ci.coreinfer_w4_codes_bytes(N, K),), 0xA5, dtype=torch.uint8, device="cuda")
    pairs = torch.full((ci.coreinfer_w4_pairs_bytes(N, K, group) // 2,), float("nan"), dtype=torch.float16, device="cuda")
    ci.coreinfer_w4_quantize(w, group, codes, pairs)
    return codes, pairs, ci.make_w4_matrix(codes, pairs, N, K, group)


def reference(x, w, bias, act, mul):
    """(y, mass): 64-bit result and the sum of absolute terms of each output."""
    y = x @ w.T
    mass = np.abs(x) @ np.abs(w).T
    if bias is not None:
        y, mass = y + bias, mass + np.abs(bias)
    if act == ci.ACT_RELU:
        y = np.maximum(y, 0)
    elif act == ci.ACT_SILU:
        y = y / (1 + np.exp(-y))
    if mul is not None:
        y, mass = y * mul, mass * np.abs(mul)
    return y, mass


def check(y, ref, mass, spread, K, dtype):
    """|error| <= (rounding steps of a sum of K terms in fp32, halves of 22 bits for fp32 x) * mass + one rounding.
    `spread`: how much larger s c + |o| is than |s c + o|, at most about 4 for values on both sides of 0; SiLU's
    slope is at most 1.1 and its exponential is good to 2^-20 relative."""
    tol = (64 + K / 32) * EPS32 * spread * mass + (OUT_EPS[dtype] + 2.0 ** -19) * np.abs(ref) + 1e-30
    bad = np.abs(y.astype(np.float64) - ref) > tol
    assert not bad.any(), "%d outputs off, worst %.3g of the bound" % (bad.sum(), (np.abs(y - ref) / tol).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N,K,group,transposed", [(1, 1, 32, False), (16, 128, 128, False), (17, 129, 32, True), (40, 333, 64, True),
                                                  (33, 200, 128, False), (96, 64, 64, True)])
def test_layout(N, K, group, transposed, dtype):
    require_gpu()
    g = torch.Generator(device="cuda").manual_seed(N * 1000 + K)
    w = torch.randn(K, N, generator=g, device="cuda").to(DT[dtype]).t() if transposed else torch.randn(N, K, generator=g, device="cuda").to(DT[dtype])
    codes, pairs, _ = lay_out(w, group)
    c, p, _ = w4_layout(values_np(w), group)
    np.testing.assert_array_equal(codes.cpu().numpy(), c.reshape(-1))
    np.testing.assert_array_equal(pairs.cpu().numpy().view(np.uint16), p.reshape(-1).view(np.uint16))


def test_layout_of_unusual_values():
    """Constant groups, zeros, values beyond fp16, infinities and a NaN: the format's rule holds, neighbours are untouched."""
    require_gpu()
    w = torch.randn(16, 256, generator=torch.Generator().manual_seed(1))
    w[0, :32], w[1, 32:64], w[2, 64:96] = 0.0, 3.25, 1e-9
    w[3, 5], w[4, 70], w[5, 130] = 1e30, float("inf"), float("-inf")
    w[6, 200] = float("nan")
    w[7, :] = torch.linspace(-1e-6, 1e-6, 256)
    codes, pairs, _ = lay_out(w.cuda(), 32)
    c, p, _ = w4_layout(w.numpy(), 32)
    np.testing.assert_array_equal(codes.cpu().numpy(), c.reshape(-1))
    got, want = pairs.cpu().numpy(), p.reshape(-1)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    np.testing.assert_array_equal(got[~np.isnan(want)].view(np.uint16), want[~np.isnan(want)].view(np.uint16))


CASES = [
    # N, K, batch, dtype, out, group, act, bias, mul
    (1, 1, 1, "f32", "f32", 32, "none", False, False), (5, 31, 2, "bf16", "bf16", 32, "none", True, False),
    (16, 128, 8, "f16", "f16", 128, "relu", True, True), (100, 127, 3, "f32", "f32", 64, "silu", True, True),
    (257, 1000, 8, "bf16", "f32", 64, "none", True, False), (768, 768, 1, "f32", "f32", 32, "none", True, False),
    (768, 768, 8, "f32", "f32", 128, "none", False, True), (4096, 3277, 5, "f16", "f32", 64, "none", False, False),
    (1000, 4096, 1, "bf16", "bf16", 128, "silu", False, True), (2752, 4096, 7, "bf16", "f32", 32, "relu", False, False),
    (300, 16384, 8, "bf16", "f32", 128, "none", False, False), (130, 20480, 4, "f32", "f32", 32, "none", True, False),
    (9216, 768, 6, "f16", "f16", 32, "none", True, False), (40000, 256, 2, "bf16", "f32", 64, "none", False, False),
    (64, 36864, 8, "bf16", "f32", 64, "none", False, False),
]


@pytest.mark.parametrize("N,K,batch,dtype,out,group,act,bias,mul", CASES)
def test_matvec(N, K, batch, dtype, out, group, act, bias, mul):
    require_gpu()
    dt, odt, act = DT[dtype], DT[out], {"none": ci.ACT_NONE, "relu": ci.ACT_RELU, "silu": ci.ACT_SILU}[act]
    g = torch.Generator(device="cuda").manual_seed(N + 7 * K + batch)
    w = torch.randn(N, K, generator=g, device="cuda") * 0.05
    codes, pairs, w4 = lay_out(w, group)
    _, _, vals = w4_layout(values_np(w), group)
    x = torch.randn(batch, K, generator=g, device="cuda").to(dt)
    b = torch.randn(N, generator=g, device="cuda").to(dt) if bias else None
    m = torch.randn(batch, N, generator=g, device="cuda").to(odt) if mul else None
    y = torch.full((batch, N), float("nan"), dtype=odt, device="cuda")
    ci.coreinfer_w4_matvec(w4, x, act, b, m, y)
    ref, mass = reference(values_np(x).astype(np.float64), vals, None if b is None else values_np(b).astype(np.float64), act,
                          None if m is None else values_np(m).astype(np.float64))
    check(values_np(y), ref, mass, 4.0, K, odt)
    again = torch.empty_like(y)
    ci.coreinfer_w4_matvec(w4, x, act, b, m, again)
    assert torch.equal(y, again)                                   # a fixed order of sums: the same bits


def test_matvec_strides_streams_and_in_place_mul():
    """x a column slice of a wider tensor that starts off any vector boundary, y a slice too, y the same buffer as mul,
    everything on a stream of its own."""
    require_gpu()
    N, K, batch = 70, 500, 4
    g = torch.Generator(device="cuda").manual_seed(3)
    w = torch.randn(N, K, generator=g, device="cuda")
    for dt in DT.values():
        wide = torch.randn(batch, 3 * K + 1, generator=g, device="cuda").to(dt)
        x = wide[:, K + 1:2 * K + 1]
        buf = torch.randn(batch, 2 * N + 1, generator=g, device="cuda").to(dt)
        y = buf[:, 1:N + 1]
        before, m = buf.clone(), values_np(y).astype(np.float64)
        codes, pairs, w4 = lay_out(w, 64)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        ci.coreinfer_w4_matvec(w4, x, ci.ACT_RELU, None, y, y, stream=s)
        s.synchronize()
        ref, mass = reference(values_np(x).astype(np.float64), w4_layout(values_np(w), 64)[2], None, ci.ACT_RELU, m)
        check(values_np(y), ref, mass, 4.0, K, dt)
        assert torch.equal(buf[:, :1], before[:, :1]) and torch.equal(buf[:, N + 1:], before[:, N + 1:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_matvec_wide_range_of_x(dtype):
    """Rows with entries far beyond fp16's range, and far below it, are as exact as any; an infinity or NaN
    stays in its own row."""
    require_gpu()
    N, K, group = 48, 640, 32
    g = torch.Generator(device="cuda").manual_seed(5)
    w = torch.randn(N, K, generator=g, device="cuda")
    codes, pairs, w4 = lay_out(w, group)
    vals = w4_layout(values_np(w), group)[2]
    x = torch.randn(6, K, generator=g, device="cuda")
    x[0] *= 1e30
    x[1] *= 1e-30
    x[2, ::7] *= 1e6
    x[3, 100] = float("inf")
    x[4, 639] = float("nan")
    x = x.to(DT[dtype])
    y = torch.empty(6, N, device="cuda")
    ci.coreinfer_w4_matvec(w4, x, ci.ACT_NONE, None, None, y)
    y = values_np(y)
    rows = [0, 1, 2, 5]
    ref, mass = reference(values_np(x).astype(np.float64)[rows], vals, None, ci.ACT_NONE, None)
    check(y[rows], ref, mass, 4.0, K, torch.float32)
    assert not np.isfinite(y[[3, 4]]).any()


def test_matvec_exact_integers():
    """Weights whose pairs are whole numbers and whole x: every product and sum is exact, so is y."""
    require_gpu()
    N, K, group = 50, 384, 32
    rng = np.random.default_rng(8)
    w = rng.integers(0, 16, size=(N, K)).astype(np.float32)
    w[:, ::32], w[:, 1::32] = 0, 15                                # every group spans 0..15: s = 1, o = 0
    x = rng.integers(-8, 9, size=(8, K)).astype(np.float32)
    codes, pairs, w4 = lay_out(torch.from_numpy(w).cuda(), group)
    for dt in DT.values():
        y = torch.empty(8, N, device="cuda")
        ci.coreinfer_w4_matvec(w4, torch.from_numpy(x).cuda().to(dt), ci.ACT_NONE, None, None, y)
        np.testing.assert_array_equal(y.cpu().numpy(), x @ w.T)


@pytest.mark.parametrize("with_mul", [False, True])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_matvec_nan_and_infinity_pass_every_activation(dtype, act, with_mul):
    """A NaN or infinity in x leaves no finite output in its row, a NaN in the weights or the bias is NaN in its column,
    whatever the activation; everything else is as it was."""
    require_gpu()
    N, K, group = 48, 640, 64
    act = {"none": ci.ACT_NONE, "relu": ci.ACT_RELU, "silu": ci.ACT_SILU}[act]
    g = torch.Generator(device="cuda").manual_seed(17)
    w = torch.randn(N, K, generator=g, device="cuda") * 0.05
    w[7, 130] = float("nan")
    codes, pairs, w4 = lay_out(w, group)
    x = torch.randn(5, K, generator=g, device="cuda")
    x[1, 100], x[2, 639], x[3, 0] = float("inf"), float("nan"), float("-inf")
    bias = torch.randn(N, generator=g, device="cuda")
    bias[20] = float("nan")
    x, bias = x.to(DT[dtype]), bias.to(DT[dtype])
    m = torch.randn(5, N, generator=g, device="cuda").to(DT[dtype]) if with_mul else None
    y = torch.zeros(5, N, dtype=DT[dtype], device="cuda")
    ci.coreinfer_w4_matvec(w4, x, act, bias, m, y)
    y = values_np(y)
    assert not np.isfinite(y[1:4]).any()
    assert np.isnan(y[:, [7, 20]]).all()
    rows, cols = [0, 4], [n for n in range(N) if n not in (7, 20)]
    ref, mass = reference(values_np(x).astype(np.float64)[rows], w4_layout(values_np(w), group)[2][cols], values_np(bias).astype(np.float64)[cols],
                          act, None if m is None else values_np(m).astype(np.float64)[rows][:, cols])
    check(y[rows][:, cols], ref, mass, 4.0, K, DT[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N,K,group", [(1, 1, 32), (17, 129, 64), (70, 300, 128)])
def test_layout_of_a_view_without_a_unit_stride(N, K, group, dtype):
    """Every second row and every third column of a wider matrix, and rows that are all the same one (stride 0)."""
    require_gpu()
    g = torch.Generator(device="cuda").manual_seed(N + K)
    wide = torch.randn(2 * N, 3 * K, generator=g, device="cuda").to(DT[dtype])
    for w in (wide[::2, ::3], wide[:, ::3].t()[:, :N].t(), wide[:1, :K].expand(N, K), wide[:1, ::3].expand(N, K)):
        codes, pairs, _ = lay_out(w, group)
        c, p, _ = w4_layout(values_np(w), group)
        np.testing.assert_array_equal(codes.cpu().numpy(), c.reshape(-1))
        np.testing.assert_array_equal(pairs.cpu().numpy().view(np.uint16), p.reshape(-1).view(np.uint16))
