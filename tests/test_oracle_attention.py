"""Pins of the oracle of attention: torch's own softmax, rotations as complex numbers, torch's E4M3 (no GPU needed)."""

import numpy as np
import pytest
import torch

from oracle import attention, mx4


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n,m,Hq,H,D", [(5, 5, 4, 2, 8), (3, 9, 6, 1, 16), (4, 2, 2, 2, 8), (1, 1, 3, 3, 4)])
def test_attention_is_torch_softmax(n, m, Hq, H, D, causal):
    rng = np.random.default_rng(n * m)
    q, k, v = (rng.standard_normal(s) for s in ((n, Hq, D), (m, H, D), (m, H, D)))
    sees = np.clip(np.arange(n) + 1 + m - n, 0, m) if causal else np.full(n, m)
    kk, vv = (torch.from_numpy(x).repeat_interleave(Hq // H, dim=1) for x in (k, v))
    s = torch.einsum("ihd,jhd->hij", torch.from_numpy(q), kk) * 0.3
    s.masked_fill_(torch.arange(m)[None, None] >= torch.from_numpy(sees)[None, :, None], float("-inf"))
    want = torch.einsum("hij,jhd->ihd", torch.softmax(s, dim=2).nan_to_num(0.0), vv).numpy()
    out, mag, span, big = attention.attend(q, k, v, 0.3, sees)
    assert np.abs(out - want).max() < 1e-12
    assert (out[sees == 0] == 0).all() and (np.abs(out) <= mag + 1e-12).all() and (mag.max(2) <= big + 1e-12).all()
    for i, c in enumerate(sees):
        if c:
            assert (span[i] + 1e-12 >= s[:, i, :c].abs().amax(1).numpy()).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_multiplication_by_a_complex_number(interleaved):
    rng = np.random.default_rng(1)
    x, rot, pos = rng.standard_normal((6, 3, 32)).astype(np.float32), 16, np.array([0, 1, 7, 100, 3000, 99999])
    f = attention.frequencies(rot, 10000.0)
    got = attention.rotate(x, attention.angles(100000, f).astype(np.float32), pos, interleaved)
    lo, hi = (x[:, :, 0:rot:2], x[:, :, 1:rot:2]) if interleaved else (x[:, :, : rot // 2], x[:, :, rot // 2 : rot])
    z = (lo + 1j * hi) * np.exp(1j * pos[:, None, None] * f)
    a, b = (got[:, :, 0:rot:2], got[:, :, 1:rot:2]) if interleaved else (got[:, :, : rot // 2], got[:, :, rot // 2 : rot])
    # an entry of the table, two products and a sum, each rounded to fp32
    assert np.abs(a + 1j * b - z).max() < 4 * 2.0 ** -24 * 2 * np.abs(x).max()
    assert np.array_equal(got[:, :, rot:], x[:, :, rot:]) and np.array_equal(got[0], x[0])


def test_frequencies():
    f = attention.frequencies(64, 500000.0)
    assert f[0] == 1 and np.allclose(f[1:] / f[:-1], 500000.0 ** (-1 / 32), rtol=1e-13)
    assert np.allclose(attention.frequencies(64, 500000.0, 1, factor=4.0), f / 4, rtol=1e-15)
    bands = attention.frequencies(64, 500000.0, 2, factor=8.0, low=1.0, high=4.0, original=8192.0)
    turns = 8192 * f / (2 * np.pi)
    assert np.array_equal(bands[turns >= 4], f[turns >= 4]) and np.allclose(bands[turns <= 1], f[turns <= 1] / 8, rtol=1e-15)
    between = (turns > 1) & (turns < 4)
    assert between.any() and ((bands[between] > f[between] / 8) & (bands[between] < f[between])).all() and (np.diff(bands) < 0).all()


def test_e4m3_rows_are_torch_e4m3():
    rng = np.random.default_rng(3)
    y = np.concatenate([rng.standard_normal(2000) * 10.0 ** rng.uniform(-4, 3, 2000), [0.0, -0.0, 448, 464, 465, 1e9, -1e9, 2.0 ** -10, 2.0 ** -9, 1.5 * 2.0 ** -9, 17, 19]]).astype(np.float32)
    codes, scales = attention.stored(y.reshape(1, 1, -1), 1, None)
    want = torch.from_numpy(np.clip(y, -448, 448)).to(torch.float8_e4m3fn)
    assert scales is None and np.array_equal(codes.ravel(), want.view(torch.uint8).numpy())
    assert np.array_equal(attention.held(codes, None, 1, None).ravel(), want.double().numpy())
    assert attention.stored(np.full((1, 1, 4), np.nan, np.float32), 1, None)[0].ravel().tolist() == [127] * 4
    # a factor: the reciprocal is rounded to fp32, and its product
    f = np.array([0.7, 3.0], dtype=np.float32)
    y2 = rng.standard_normal((5, 2, 16)).astype(np.float32)
    codes = attention.stored(y2, 1, f)[0]
    r = np.float32(1) / f
    assert np.array_equal(codes, torch.from_numpy(y2 * r[None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert np.allclose(attention.held(codes, None, 1, f), y2, rtol=2.0 ** -4 * 1.01, atol=2.0 ** -10 * 3)


def test_nvfp4_rows_are_the_quantiser_s():
    rng = np.random.default_rng(4)
    y, f = rng.standard_normal((7, 3, 64)).astype(np.float32), np.array([1.0, 0.25, 2.0], dtype=np.float32)
    codes, scales = attention.stored(y, 2, f)
    for h in range(3):                                   # (powers of two: exact)
        c, s = mx4.quantize(y[:, h] / f[h], 1)
        assert np.array_equal(codes[:, h], c) and np.array_equal(scales[:, h], s)
    assert np.abs(attention.held(codes, scales, 2, f) - y).max() <= np.abs(y).max() / 6 * 1.07
