"""4-bit operators at the ends of what they accept: results whose rows are so long that steps of a few rows pass 32 bits."""

import numpy as np
import pytest
import torch

import paper_2510_19482_b200 as elutq
from oracle import mx4
from test_mx4_gemm_gpu import TYPES, _assert_close, _dev, _matrix

pytestmark = pytest.mark.gpu


# 16-bit stores of 16, 8 and 4 bytes and value by value (8, 4, 2 and 4 rows a step), and fp32
@pytest.mark.parametrize("M,N,out", [(16, 1 << 28, "f16"), (13, (1 << 29) + 4, "bf16"), (9, (1 << 29) + 2, "f16"), (6, (1 << 30) - 1, "f16"), (5, (1 << 29) + 8, "f32")])
def test_rows_of_more_than_2_28_results(M, N, out):
    K = 32
    rng = np.random.default_rng(M)
    xc, xs = _matrix(rng, M, K, 0)
    gen = torch.Generator(device="cuda").manual_seed(M)
    wc = torch.randint(0, 256, (N, K // 2), generator=gen, dtype=torch.uint8, device="cuda")
    ws = torch.randint(122, 130, (N, 1), generator=gen, dtype=torch.uint8, device="cuda")
    Y = torch.full((M, N), float("nan"), dtype=TYPES[out], device="cuda")
    elutq.elutq_mx4_gemm(*_dev(xc, xs), wc, ws, Y, M, N, K, 0)
    assert elutq.elutq_device_status() == 0
    for n0 in (0, N // 2 - 200, N - 400):
        part = (xc, xs, wc[n0 : n0 + 400].cpu().numpy(), ws[n0 : n0 + 400].cpu().numpy())
        _assert_close(Y[:, n0 : n0 + 400], mx4.matmul(*part, 0), mx4.magnitude(*part, 0), K, out, f"columns from {n0} on")
    for r in range(M):
        assert not torch.isnan(Y[r]).any(), r
    del wc, ws, Y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("M,N", [(1, 1), (40, 3)])
def test_the_longest_k(fmt, M, N):
    """Codes of 0 but for a few along K, the last among them: sums are exact."""
    K, B = 1 << 28, mx4.BLOCK[fmt]
    one = 127 if fmt == 0 else 56
    xc, wc = (torch.zeros((n, K // 2), dtype=torch.uint8, device="cuda") for n in (M, N))
    xs, ws = (torch.full((n, K // B), one, dtype=torch.uint8, device="cuda") for n in (M, N))
    at = [0, 777, K // 4, K // 2 - 256, K // 2 - 1]                 # bytes of a row; their high halves: 1, 1.5, ...
    for i, k in enumerate(at):
        xc[:, k] = 0x20
        wc[:, k] = 0x10 * (i + 1)
    Y = torch.full((M, N), float("nan"), device="cuda")
    elutq.elutq_mx4_gemm(xc, xs, wc, ws, Y, M, N, K, fmt)
    assert elutq.elutq_device_status() == 0
    assert (Y == float(mx4.E2M1[1 : 1 + len(at)].sum())).all()
