"""4-bit quantisation of half-way points at the sizes of whole matrices: the block's scale is the one that makes them half-way points."""

import numpy as np
import pytest
import torch

import paper_2510_19482_b200 as elutq
from oracle import mx4

pytestmark = pytest.mark.gpu
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
# multiples of a quarter of the scale that lie between two codes: times a scale of four significant bits they have 7 at most, so every type holds them
HALF_WAY = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("ty", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,K", [(1, 32), (3, 96), (37, 1056), (257, 512), (1000, 4096)])
def test_half_way_points(fmt, ty, rows, K):
    rng = np.random.default_rng(rows + K)
    B = mx4.BLOCK[fmt]
    # a scale for each block: powers of two, and 8 to 15 times one where the format has those
    scale = np.exp2(rng.integers(-9, 5, (rows, K // B))) * (rng.integers(8, 16, (rows, K // B)) if fmt == 1 else 8)
    x = HALF_WAY[rng.integers(0, 7, (rows, K))] * rng.choice([-1.0, 1.0], (rows, K))
    x[:, ::B] = 6.0 * rng.choice([-1.0, 1.0], (rows, K // B))
    x = x * np.repeat(scale, B, axis=1)
    X = torch.from_numpy(x).to(TYPES[ty])
    assert np.array_equal(X.double().numpy(), x)
    wc, ws = mx4.quantize(x.astype(np.float32), fmt)
    assert np.array_equal(mx4.scale_values(ws, fmt), scale)
    # the even code of the two: every second one of 0, 0.5, 1, 1.5, 2, 3, 4, 6
    even = np.array([0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0])
    v = mx4.values(wc, ws, fmt) / np.repeat(scale, B, axis=1)
    inner = np.arange(K) % B > 0
    assert np.array_equal(np.abs(v[:, inner]), even[np.searchsorted(HALF_WAY, np.abs(x / np.repeat(scale, B, axis=1))[:, inner])])
    codes, scales = elutq.elutq_mx4_quantize(X.cuda(), rows, K, fmt)
    assert np.array_equal(scales.cpu().numpy(), ws) and np.array_equal(codes.cpu().numpy(), wc)
    # through a factor: the same points from other values
    codes, scales = elutq.elutq_mx4_quantize((X.cuda() * 0.5).contiguous(), rows, K, fmt, prescale=torch.tensor([2.0], device="cuda"))
    assert np.array_equal(scales.cpu().numpy(), ws) and np.array_equal(codes.cpu().numpy(), wc)
