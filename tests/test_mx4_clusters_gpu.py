"""4-bit products whose long K is shared by clusters of CTAs, with more tiles than clusters fit the card: a cluster's memory for parts is used again and again.

A product of this kind has few tokens (96 at most), K of thousands and fewer tiles than SMs; 12 clusters of 8, 30 of 4 and 70 of 2 are fewer than there are tiles."""

import numpy as np
import pytest
import torch

import paper_2510_19482_b200 as elutq
from oracle import mx4
from test_mx4_gemm_gpu import TYPES, _assert_close, _dev, _grouped, _matrix

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K,fmt,out", [(6, 4574, 43904, 1, "f32"), (2, 5000, 45920, 0, "f16"), (20, 9551, 51680, 1, "bf16"), (60, 6100, 63552, 0, "f32"), (6, 19299, 16800, 1, "f16"),
                                           (84, 19181, 30944, 1, "bf16")])
def test_more_tiles_than_clusters(M, N, K, fmt, out):
    rng = np.random.default_rng(M + K)
    xc, xs = _matrix(rng, M, K, fmt)
    gen = torch.Generator(device="cuda").manual_seed(N)
    wc = torch.randint(0, 256, (N, K // 2), generator=gen, dtype=torch.uint8, device="cuda")
    lo, hi, B = (122, 130, 32) if fmt == 0 else (0, 127, 16)
    ws = torch.randint(lo, hi, (N, K // B), generator=gen, dtype=torch.uint8, device="cuda")
    alpha = torch.tensor([2.0**-6], device="cuda")
    Y, again = (torch.full((M, N), float("nan"), dtype=TYPES[out], device="cuda") for _ in range(2))
    x = _dev(xc, xs)
    elutq.elutq_mx4_gemm(*x, wc, ws, Y, M, N, K, fmt, alpha=alpha)
    elutq.elutq_mx4_gemm(*x, wc, ws, again, M, N, K, fmt, alpha=alpha)
    assert elutq.elutq_device_status() == 0
    assert not torch.isnan(Y).any() and torch.equal(Y, again)
    # some columns of every tile of 128
    cols = np.unique(np.concatenate([np.arange(0, N, 128), np.minimum(np.arange(0, N, 128) + rng.integers(0, 128), N - 1), [N - 2, N - 1]]))
    at = torch.from_numpy(cols).cuda()
    part = (xc, xs, wc[at].cpu().numpy(), ws[at].cpu().numpy())
    _assert_close(Y[:, at], mx4.matmul(*part, fmt, 2.0**-6), mx4.magnitude(*part, fmt, 2.0**-6), K, out, f"{M} x {N} x {K}")


@pytest.mark.parametrize("fmt,sizes,N,K", [(1, [12, 13], 2056, 12320), (1, [2] * 8, 243, 25728), (1, [0, 5, 3, 2, 4, 1, 0, 3, 2, 6, 4, 1], 671, 9024), (0, [1, 0, 25], 1128, 39744)])
def test_groups_with_more_tiles_than_clusters(fmt, sizes, N, K):
    rng = np.random.default_rng(N + K)
    borders = [0, *np.cumsum(sizes).tolist()]
    _grouped(rng, borders, N, K, len(sizes), fmt, "bf16", borders[-1], alpha=np.full(len(sizes), 2.0**-7, dtype=np.float32))
