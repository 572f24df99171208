"""Pins of the 4-bit oracle, and what the library's 4-bit entries refuse on the host (no GPU needed)."""

import ctypes

import numpy as np
import pytest
import torch

import paper_2510_19482_b200 as elutq
from oracle import mx4


def test_scale_tables_agree_with_torch():
    e4m3 = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(mx4.E4M3, e4m3)
    e8m0 = torch.arange(255, dtype=torch.uint8).view(torch.float8_e8m0fnu).double().numpy()
    assert np.array_equal(mx4.scale_values(np.arange(255), 0), e8m0)
    assert np.isnan(mx4.scale_values(np.array([255]), 0)).all() and np.isnan(mx4.scale_values(np.array([127]), 1)).all()


def test_codes_of_a_known_block():
    # amax 6: scale 1 in both formats, codes by hand (ties: 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5 go to the even code)
    v = np.array([6, 5, 5.01, 3.5, 3.49, 2.5, 2.51, 1.75, 1.74, 1.25, 1.26, 0.75, 0.74, 0.25, 0.26, -0.2], dtype=np.float32)
    want = np.array([7, 6, 7, 6, 5, 4, 5, 4, 3, 2, 3, 2, 1, 0, 1, 8])
    codes, scales = mx4.quantize(np.tile(v, 2)[None], 1)
    assert (scales == 0x38).all()
    assert np.array_equal(codes[0, :8], want[0::2] | want[1::2] << 4)
    codes, scales = mx4.quantize(np.tile(v, 2)[None], 0)
    assert (scales == 127).all() and np.array_equal(codes[0, :8], want[0::2] | want[1::2] << 4)
    # just below 8: the scale stays 1, the value saturates; 8: the scale doubles
    for top, byte, code in ((7.99, 127, 7), (8.0, 128, 6)):
        x = np.zeros((1, 32), dtype=np.float32)
        x[0, 3] = top
        codes, scales = mx4.quantize(x, 0)
        assert scales[0, 0] == byte and codes[0, 1] >> 4 == code


def test_odd_blocks():
    x = np.zeros((4, 32), dtype=np.float32)
    x[1, 5], x[2, 5], x[3, 5] = np.inf, np.nan, 2.0 ** -140
    for fmt, nan in ((0, 255), (1, 127)):
        codes, scales = mx4.quantize(x, fmt)
        assert scales[0, 0] == 0 and scales[1, 0] == nan and scales[2, 0] == nan and scales[3, 0] == 0
        assert not codes.any()


@pytest.mark.parametrize("fmt", [0, 1])
def test_nearest_by_brute_force(fmt):
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((8, 64)) * np.exp2(rng.integers(-6, 7, (8, 1)))).astype(np.float32)
    codes, scales = mx4.quantize(x, fmt)
    v = mx4.values(codes, scales, fmt)
    s = np.repeat(mx4.scale_values(scales, fmt), mx4.BLOCK[fmt], axis=1)
    best = np.abs(x[..., None].astype(np.float64) - np.concatenate([-mx4.E2M1, mx4.E2M1]) * s[..., None]).min(axis=2)
    assert np.array_equal(np.abs(x - v), best)


def test_sizes():
    assert elutq.elutq_mx4_bytes(elutq.MX4_MXFP4, 3, 96) == (3 * 48, 9)
    assert elutq.elutq_mx4_bytes(elutq.MX4_NVFP4, 3, 96) == (3 * 48, 18)
    # a matrix of more than 2^32 values
    assert elutq.elutq_mx4_bytes(elutq.MX4_NVFP4, 1 << 20, 1 << 14) == (1 << 33, 1 << 30)


def test_refusals_of_the_conversions():
    L, a, b = elutq.lib(), ctypes.c_size_t(0), ctypes.c_size_t(0)
    before = elutq.elutq_launch_count()
    for fmt, rows, K, st in ((0, 0, 32, -1), (0, 1, 0, -1), (2, 1, 32, -1), (-1, 1, 32, -1), (0, 1, 48, -2), (1, 1, 16, -2)):
        assert L.elutq_mx4_bytes(fmt, rows, K, ctypes.byref(a), ctypes.byref(b)) == st
        assert L.elutq_mx4_dequantize(16, 16, rows, K, fmt, None, 16, 0, None) == st
        assert L.elutq_mx4_quantize(16, 0, 8, 4096, rows, K, fmt, 0, None, None, 1, None, 16, 16, None) == st
    assert L.elutq_mx4_bytes(0, 1, 32, None, ctypes.byref(b)) == -1

    def quantize(X=16, x_type=0, x_rows=4, ld=64, rows=4, K=64, flags=0, prescale=None, index=None, div=1, n_rows=None, codes=16, scales=16):
        return L.elutq_mx4_quantize(X, x_type, x_rows, ld, rows, K, 0, flags, prescale, index, div, n_rows, codes, scales, None)

    for name in ("X", "codes", "scales"):
        assert quantize(**{name: None}) == -1
    assert quantize(x_type=3) == quantize(x_type=-1) == quantize(flags=2) == quantize(x_rows=0) == quantize(index=16, div=0) == -1
    assert quantize(ld=63) == quantize(ld=127, flags=1) == quantize(x_rows=3) == -2
    assert quantize(X=8) == quantize(codes=8) == quantize(ld=65) == quantize(prescale=2) == quantize(index=6) == quantize(n_rows=2) == -3
    assert quantize(x_type=2, ld=66) == -3
    assert L.elutq_mx4_dequantize(None, 16, 1, 32, 0, None, 16, 0, None) == L.elutq_mx4_dequantize(16, 16, 1, 32, 0, None, 16, 3, None) == -1
    assert L.elutq_mx4_dequantize(8, 16, 1, 32, 0, None, 16, 0, None) == L.elutq_mx4_dequantize(16, 16, 1, 32, 0, 2, 16, 0, None) == -3
    assert L.elutq_mx4_dequantize(16, 16, 1, 32, 0, None, 8, 0, None) == -3
    assert elutq.elutq_launch_count() == before


def test_refusals_of_the_products():
    L = elutq.lib()
    before = elutq.elutq_launch_count()

    def gemm(xc=16, xs=16, wc=16, ws=16, Y=16, y_type=0, M=4, N=4, K=64, fmt=0, alpha=None):
        return L.elutq_mx4_gemm(xc, xs, wc, ws, Y, y_type, M, N, K, fmt, alpha, None)

    def grouped(offsets=16, M=4, N=4, K=64, E=2, fmt=0, alpha=None):
        return L.elutq_mx4_gemm_grouped(16, 16, 16, 16, offsets, 16, 0, M, N, K, E, fmt, alpha, None)

    for name in ("xc", "xs", "wc", "ws", "Y"):
        assert gemm(**{name: None}) == -1
    for name in ("M", "N", "K"):
        assert gemm(**{name: 0}) == gemm(**{name: -1}) == grouped(**{name: 0}) == -1
    assert gemm(y_type=3) == gemm(fmt=2) == grouped(offsets=None) == grouped(E=0) == -1
    assert gemm(K=48) == gemm(M=1 << 30) == gemm(N=1 << 30) == grouped(N=1 << 29, E=2) == grouped(K=40) == -2
    assert gemm(xc=8) == gemm(wc=24) == gemm(Y=8) == gemm(alpha=2) == grouped(offsets=18) == grouped(alpha=6) == -3
    assert grouped(E=1025) == -5
    assert L.elutq_mx4_test_wait_expiry(16, 16, 16, 16, 16, 0, 4, 4, 64, 0, 0, None) == -1
    assert elutq.elutq_launch_count() == before


def test_the_binding_refuses_host_memory():
    """Kernels read addresses as they are: what is not on the current device is turned down before any call."""
    x, c, s = torch.zeros((4, 64), dtype=torch.float16), torch.zeros((4, 32), dtype=torch.uint8), torch.zeros((4, 2), dtype=torch.uint8)
    before = elutq.elutq_launch_count()
    if not torch.cuda.is_available():
        for call in (lambda: elutq.elutq_mx4_quantize(x, 4, 64, 0, stream=0), lambda: elutq.elutq_mx4_dequantize(c, s, x, 4, 64, 0, stream=0),
                     lambda: elutq.elutq_mx4_gemm(c, s, c, s, x, 4, 4, 64, 0, stream=0)):
            with pytest.raises(elutq.ElutqError):
                call()
    assert elutq.elutq_launch_count() == before
