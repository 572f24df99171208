"""SwiGLU in front of 4-bit quantisation where gates are closed: far below zero, down to minus infinity."""

import numpy as np
import pytest
import torch

import paper_2510_19482_b200 as elutq
from oracle import mx4

pytestmark = pytest.mark.gpu
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
GATES = [-60.0, -63.75, -64.0, -64.25, -66.0, -80.0, -87.0, -87.5, -88.75, -90.0, -91.0, -96.0, -100.0, -104.0, -110.0, -130.0, -160.0, -190.0, -198.0, -199.0, -200.0, -201.0, -240.0,
         -1000.0, -65504.0, -1e30, -3.3e38, -np.inf]


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("ty", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("size", ["ordinary", "large", "largest"])
def test_blocks_of_closed_gates(fmt, ty, size):
    """Whole blocks of one gate, and of two neighbours in the list.  silu(g) u within 8 units of 2^-24 (the exponential's 2^-22, its argument's 2^-24, two
    products' roundings 2^-24 each) and, where that is subnormal, one more unit of 2^-149: what a quantisation of such a value may be."""
    rng = np.random.default_rng(7)
    top = {"ordinary": 1.0, "large": 6e3 if ty == "f16" else 1e30, "largest": 6.5e4 if ty == "f16" else 3.3e38}[size]
    gates = [g for g in GATES if ty != "f16" or g >= -65504.0 or np.isinf(g)]
    rows, K = len(gates), 64
    g = np.repeat(np.array(gates)[:, None], K, axis=1)
    g[1:, 32::2] = g[:-1, 32::2]
    u = rng.uniform(-1.0, 1.0, (rows, K)) * top
    u[:, ::16] = top * np.sign(rng.standard_normal((rows, K // 16)))
    X = torch.from_numpy(np.concatenate([g, u], axis=1)).to(TYPES[ty]).cuda()
    codes, scales = elutq.elutq_mx4_quantize(X, rows, K, fmt, flags=elutq.MX4_FLAG_SWIGLU)
    x = X.double().cpu().numpy()
    closed = np.isneginf(x[:, :K])
    gate = np.where(closed, 0.0, x[:, :K])
    with np.errstate(over="ignore"):
        y = np.where(closed, 0.0, gate / (1 + np.exp(-gate)) * x[:, K:])
    got = mx4.values(codes.cpu().numpy(), scales.cpu().numpy(), fmt)
    near = [mx4.values(*mx4.quantize(np.sign(y).astype(np.float32) * np.maximum(np.abs(y * (1 + d)) + a * 2.0**-149, 0.0).astype(np.float32), fmt), fmt)
            for d in (-8 * 2.0**-24, 0.0, 8 * 2.0**-24) for a in (-1, 0, 1)]
    ok = np.any([got == n for n in near], axis=0)
    assert ok.all(), f"gate {gate[~ok][0]}: got {got[~ok][0]}, exact {y[~ok][0]} ({int((~ok).sum())} of {ok.size} off)"


@pytest.mark.parametrize("fmt", [0, 1])
def test_closed_gates_beside_open_ones(fmt):
    """A single closed gate anywhere in a row, and what it must not do to its neighbours."""
    rng = np.random.default_rng(3)
    rows, K = 64, 128
    x = rng.standard_normal((rows, 2 * K)).astype(np.float32)
    for r in range(rows):
        x[r, 2 * r % K + r % 2] = GATES[r % len(GATES)]
    for ty in TYPES.values():
        X = torch.from_numpy(x).to(ty).cuda()
        X[torch.isinf(X) & (torch.from_numpy(x).cuda() > -1e38)] = -65504.0          # (beyond fp16)
        codes, scales = elutq.elutq_mx4_quantize(X, rows, K, fmt, flags=elutq.MX4_FLAG_SWIGLU)
        v = X.double().cpu().numpy()
        gate = np.where(np.isneginf(v[:, :K]), -1e4, v[:, :K])
        with np.errstate(over="ignore"):
            y = gate / (1 + np.exp(-gate)) * v[:, K:]
        got = mx4.values(codes.cpu().numpy(), scales.cpu().numpy(), fmt)
        near = [mx4.values(*mx4.quantize((y * (1 + d)).astype(np.float32), fmt), fmt) for d in (-8 * 2.0**-24, 0.0, 8 * 2.0**-24)]
        assert ((got == near[0]) | (got == near[1]) | (got == near[2])).all()
