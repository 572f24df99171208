"""4-bit products that are launched early, behind a kernel that takes longer than their own waits may."""

import numpy as np
import pytest
import torch

import paper_2510_19482_b200 as elutq
import workloads
from gpu_util import pack_layer, x_dev
from oracle import mx4
from test_mx4_gemm_gpu import _assert_close, _dev, _matrix
from workloads import synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K,fmt", [(1, 256, 512, 0), (200, 512, 256, 1)])
def test_a_long_kernel_in_front(M, N, K, fmt):
    """The kernel in front lets the next one start at once and then takes 1.5 s (its own waits run out, by their number); a product's clock starts behind it."""
    q, hN, hK, hM = 2, 512, 2048, 64
    assert elutq.elutq_gemm_kernel(hM, hN, hK, q, 128) == elutq.KERNEL_TENSOR_MEMORY
    packed = pack_layer(workloads.hlq_layer(5, "mx4/front", q, 128, hN, hK))
    hx, hY = x_dev(synth.activations(5, "mx4/front/x", hM, hK)), torch.zeros((hM, hN), device="cuda")
    rng = np.random.default_rng(M)
    xc, xs = _matrix(rng, M, K, fmt)
    wc, ws = _matrix(rng, N, K, fmt)
    args, Y = _dev(xc, xs, wc, ws), torch.full((M, N), float("nan"), device="cuda")
    elutq.elutq_mx4_gemm(*args, torch.empty_like(Y), M, N, K, fmt)

    def front(polls, behind=None):
        """ms of the long kernel and, right behind it (with no event in between), of what follows"""
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        elutq.elutq_test_wait_expiry(hx, packed, hY, hM, hN, hK, polls)
        if behind is not None:
            behind()
        end.record()
        end.synchronize()
        return start.elapsed_time(end)

    polls = 4096
    front(polls)                                      # (allocates)
    while (ms := front(polls)) < 100.0:
        polls *= 4
    ms = front(int(polls * 1500.0 / ms), lambda: elutq.elutq_mx4_gemm(*args, Y, M, N, K, fmt))
    elutq.elutq_release_scratch()
    assert 1200.0 < ms < 5000.0
    _assert_close(Y, mx4.matmul(xc, xs, wc, ws, fmt), mx4.magnitude(xc, xs, wc, ws, fmt), K, "f32")
