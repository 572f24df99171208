"""Microscaled 4-bit quantisation against the oracle, byte for byte, and the way back."""

import numpy as np
import pytest
import torch

import paper_2510_19482_b200 as elutq
from oracle import mx4

pytestmark = pytest.mark.gpu
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _values(rng, rows, K, kind):
    """Magnitudes over many powers of two (scales of every kind), small whole multiples (half-way points), plain ones."""
    x = rng.standard_normal((rows, K))
    if kind == "wide":
        x = x * np.exp2(rng.integers(-20, 12, (rows, 1)))
    elif kind == "ties":
        # multiples of 1/4 of a scale of four significant bits: every half-way point, exactly
        x = rng.integers(-24, 25, (rows, K)) * 0.25 * rng.integers(8, 16, (rows, 1)) * np.exp2(rng.integers(-8, 5, (rows, 1)))
        x[:, ::16] = 6.0 * np.abs(x).max(axis=1, keepdims=True) / np.maximum(np.abs(x).max(axis=1, keepdims=True), 1e-30)
    return x


def _check(X, rows, K, fmt, want_y, **kw):
    codes, scales = elutq.elutq_mx4_quantize(X, rows, K, fmt, **kw)
    torch.cuda.synchronize()
    wc, ws = mx4.quantize(want_y, fmt)
    assert np.array_equal(scales.cpu().numpy(), ws)
    got = codes.cpu().numpy()
    bad = got != wc
    assert not bad.any(), f"{int(bad.sum())} bytes differ, first at {np.argwhere(bad)[0]}"
    return codes, scales


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("ty", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,K", [(1, 32), (1, 64), (3, 96), (5, 2880), (8, 4096), (37, 1056), (257, 512), (1000, 4096)])
def test_quantise_byte_for_byte(fmt, ty, rows, K):
    rng = np.random.default_rng(rows * K + fmt)
    for kind in ("plain", "wide", "ties"):
        X = torch.from_numpy(_values(rng, rows, K, kind)).to(TYPES[ty]).cuda()
        _check(X, rows, K, fmt, X.float().cpu().numpy())


@pytest.mark.parametrize("ty", ["f16", "bf16", "f32"])
def test_half_way_points_of_every_scale(ty):
    """NVFP4: for every E4M3 scale, every half-way point and its neighbours on both sides (in the input's type)."""
    mids = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.5])
    s = mx4.E4M3[1:]
    x = torch.from_numpy(np.concatenate([6.0 * s[:, None], mids[None] * s[:, None], np.zeros((126, 7))], axis=1)).to(TYPES[ty])     # amax, then the points
    bits = x.view(torch.int32 if ty == "f32" else torch.int16)
    for step in (-1, 0, 1):
        moved = bits.clone()
        moved[:, 1:9] += step
        v = moved.view(TYPES[ty])
        v[:, 9:16] = -v[:, 2:9]
        X = torch.nan_to_num(torch.cat([v, v], dim=1)).contiguous().cuda()
        _check(X, 126, 32, 1, X.float().cpu().numpy())


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("ty", ["f16", "bf16", "f32"])
def test_infinities_nans_zeros_and_tiny_values(fmt, ty):
    X = torch.randn(12, 128, dtype=torch.float64).to(TYPES[ty])
    X[0, 3], X[1, 40], X[2, 127], X[3] = float("inf"), float("-inf"), float("nan"), 0.0
    X[4] = -0.0
    X[5, ::2] = torch.finfo(TYPES[ty]).max
    X[6] = torch.finfo(TYPES[ty]).tiny / 4          # subnormal
    X[7, 32:64] = torch.finfo(TYPES[ty]).smallest_normal
    X[8, 0] = float("nan")
    X[8, 16:] = float("inf")
    X = X.cuda()
    codes, scales = _check(X, 12, 128, fmt, X.float().cpu().numpy())
    Y = torch.empty((12, 128), device="cuda")
    elutq.elutq_mx4_dequantize(codes, scales, Y, 12, 128, fmt)
    B = mx4.BLOCK[fmt]
    want = (~torch.isfinite(X.float())).reshape(12, -1, B).any(2).repeat_interleave(B, 1)
    assert torch.equal(torch.isnan(Y), want)


@pytest.mark.parametrize("fmt", [0, 1])
def test_prescale_strides_and_bases(fmt):
    rng = np.random.default_rng(5)
    rows, K = 19, 160
    whole = torch.from_numpy(rng.standard_normal((rows, 1000))).half().cuda()
    p = torch.tensor([731.7], device="cuda")
    for first in (0, 8, 16, 24):                    # 16- and 32-byte bases
        X = whole[:, first : first + K]
        _check(X, rows, K, fmt, X.float().cpu().numpy())
        _check(X, rows, K, fmt, X.float().cpu().numpy() * np.float32(731.7), prescale=p)
    f = torch.from_numpy(rng.standard_normal((rows, 204))).float().cuda()[:, 4 : 4 + K]
    _check(f, rows, K, fmt, f.cpu().numpy() * np.float32(731.7), prescale=p)
    with pytest.raises(elutq.ElutqError):
        elutq.elutq_mx4_quantize(whole[:, 4 : 4 + K], rows, K, fmt)
    # prescaled out of range: infinite, so NaN
    codes, scales = elutq.elutq_mx4_quantize(f.contiguous(), rows, K, fmt, prescale=torch.tensor([3e38], device="cuda"))
    assert np.array_equal(scales.cpu().numpy(), mx4.quantize((f.cpu() * 3e38).numpy(), fmt)[1])


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("ty", ["f16", "f32"])
def test_gathered_rows_and_rows_left_alone(fmt, ty):
    rng = np.random.default_rng(6)
    T, K, top, rows = 13, 224, 3, 41
    X = torch.from_numpy(rng.standard_normal((T, K))).to(TYPES[ty]).cuda()
    idx = rng.integers(0, T * top, rows)
    idx[[0, 7, 40]] = [-1, T * top, 2**31 - 1]          # none of these is a row
    idx[1] = idx[2]                                     # the same one twice
    y = np.where(((idx >= 0) & (idx < T * top))[:, None], X.float().cpu().numpy()[np.clip(idx, 0, T * top - 1) // top], 0.0)
    index = torch.from_numpy(idx.astype(np.int32)).cuda()
    _check(X, rows, K, fmt, y.astype(np.float32), index=index, index_div=top)
    wc, ws = mx4.quantize(y.astype(np.float32), fmt)
    for n in (0, 1, 17, 41, 100, -5):
        codes = torch.full((rows, K // 2), 0xA5, dtype=torch.uint8, device="cuda")
        scales = torch.full((rows, K // mx4.BLOCK[fmt]), 0xA5, dtype=torch.uint8, device="cuda")
        elutq.elutq_mx4_quantize(X, rows, K, fmt, codes=codes, scales=scales, index=index, index_div=top, n_rows=torch.tensor([n], dtype=torch.int32, device="cuda"))
        m = min(max(n, 0), rows)
        assert np.array_equal(codes.cpu().numpy()[:m], wc[:m]) and np.array_equal(scales.cpu().numpy()[:m], ws[:m])
        assert (codes[m:] == 0xA5).all() and (scales[m:] == 0xA5).all()


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("ty", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,K", [(1, 32), (33, 1440), (300, 2048)])
def test_swiglu_then_quantise(fmt, ty, rows, K):
    """silu(g) u in fp32 is a few units in the last place off the exact value, which can move a scale or a code that lies within 8 * 2^-24
    of a border: everything else is byte for byte that of the exact value."""
    X = torch.from_numpy(np.random.default_rng(rows + K).standard_normal((rows, 2 * K)) * 2).to(TYPES[ty]).cuda()
    codes, scales = elutq.elutq_mx4_quantize(X, rows, K, fmt, flags=elutq.MX4_FLAG_SWIGLU)
    x = X.double().cpu().numpy()
    y = x[:, :K] / (1 + np.exp(-x[:, :K])) * x[:, K:]
    got = mx4.values(codes.cpu().numpy(), scales.cpu().numpy(), fmt)
    near = [mx4.values(*mx4.quantize((y * (1 + d)).astype(np.float32), fmt), fmt) for d in (-8 * 2.0**-24, 0.0, 8 * 2.0**-24)]
    assert ((got == near[0]) | (got == near[1]) | (got == near[2])).all()
    assert (got != near[1]).mean() < 1e-3


@pytest.mark.parametrize("fmt", [0, 1])
def test_swiglu_far_out(fmt):
    """A gate of minus infinity or far below closes (nothing left of u); infinities and NaN elsewhere make their block NaN."""
    K, inf, nan = 64, float("inf"), float("nan")
    X = torch.ones((12, 2 * K))
    far = [(-inf, 2.0, 0), (-3e38, 2.0, 0), (-1000.0, 2.0, 0), (-88.0, -2.0, 0), (3e38, 0.0, 0), (90.0, 3.0, 270.0), (inf, 1.0, nan), (1.0, inf, nan), (0.0, inf, nan),
           (nan, 1.0, nan), (1.0, nan, nan), (-inf, nan, nan)]
    for r, (g, u, _) in enumerate(far):
        X[r, 7], X[r, K + 7] = g, u
    codes, scales = elutq.elutq_mx4_quantize(X.cuda(), 12, K, fmt, flags=elutq.MX4_FLAG_SWIGLU)
    Y = torch.empty((12, K), device="cuda")
    elutq.elutq_mx4_dequantize(codes, scales, Y, 12, K, fmt)
    B = mx4.BLOCK[fmt]
    y = np.full((12, K), 1 / (1 + np.exp(-1.0)), dtype=np.float32)
    y[:, 7] = [w for _, _, w in far]
    assert np.array_equal(np.nan_to_num(Y.cpu().double().numpy(), nan=-1.0), np.nan_to_num(mx4.values(*mx4.quantize(y, fmt), fmt), nan=-1.0))
    assert torch.isnan(Y[6:, :B]).all() and not torch.isnan(Y[:, B:]).any()


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("out", ["f16", "bf16", "f32"])
def test_dequantise_every_byte(fmt, out):
    """Every code under every scale byte.  One rounding to fp32 (alpha's product) and one to the output's type."""
    rows, K = 256, 32
    codes = torch.arange(256, dtype=torch.uint8).reshape(16, 16).repeat(16, 1).cuda()
    n = K // mx4.BLOCK[fmt]
    scales = torch.arange(256, dtype=torch.uint8).repeat_interleave(n).reshape(rows, n)
    scales = (scales if fmt == 0 else scales & 127).contiguous().cuda()
    v = mx4.values(codes.cpu().numpy(), scales.cpu().numpy(), fmt)
    for alpha in (None, 0.7):
        Y = torch.empty((rows, K), dtype=TYPES[out], device="cuda")
        a = None if alpha is None else torch.tensor([alpha], device="cuda")
        elutq.elutq_mx4_dequantize(codes, scales, Y, rows, K, fmt, alpha=a)
        want = torch.from_numpy(v).float()
        want = (want if alpha is None else want * np.float32(alpha)).to(TYPES[out])
        assert torch.equal(torch.nan_to_num(Y.cpu(), nan=-12345.0), torch.nan_to_num(want, nan=-12345.0))


def test_on_another_stream_captured_and_replayed():
    rows, K = 64, 1024
    X = torch.randn((rows, K), device="cuda", dtype=torch.float16)
    codes = torch.empty((rows, K // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((rows, K // 32), dtype=torch.uint8, device="cuda")
    Y = torch.empty((rows, K), device="cuda", dtype=torch.float16)
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        elutq.elutq_mx4_quantize(X, rows, K, 0, codes=codes, scales=scales)
        elutq.elutq_mx4_dequantize(codes, scales, Y, rows, K, 0)
    for seed in range(3):
        X.copy_(torch.randn((rows, K), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").half())
        graph.replay()
        torch.cuda.synchronize()
        wc, ws = mx4.quantize(X.float().cpu().numpy(), 0)
        assert np.array_equal(codes.cpu().numpy(), wc) and np.array_equal(Y.double().cpu().numpy(), mx4.values(wc, ws, 0))
