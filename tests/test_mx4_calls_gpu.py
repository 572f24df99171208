"""4-bit entries called in ways that other tests do not: single rows whose stride means nothing, a process whose first call is captured."""

import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2510_19482_b200 as elutq
from oracle import mx4
from test_mx4_gemm_gpu import _assert_close

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("swiglu", [False, True])
def test_one_row_of_any_stride(fmt, swiglu):
    """A single row is dense whatever its stride says: a column turned over, a row of a matrix of odd width."""
    K, width = 96, 192 if swiglu else 96
    gen = torch.Generator(device="cuda").manual_seed(fmt)
    x = torch.randn(width, generator=gen, device="cuda").half()
    flags = elutq.MX4_FLAG_SWIGLU if swiglu else 0
    want = elutq.elutq_mx4_quantize(x[None].contiguous(), 1, K, fmt, flags=flags)
    column = x[:, None].clone().T
    odd = torch.zeros((1, 1001), device="cuda", dtype=torch.float16)
    odd[0, :width] = x
    for X in (column, odd[:, :width], torch.as_strided(x.clone(), (1, width), (0, 1))):
        for kw in ({}, {"index": torch.zeros(1, dtype=torch.int32, device="cuda")}):
            got = elutq.elutq_mx4_quantize(X, 1, K, fmt, flags=flags, **kw)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # two rows have a stride that counts
    with pytest.raises(elutq.ElutqError):
        elutq.elutq_mx4_quantize(torch.as_strided(x.clone(), (2, width // 2), (1, 1)), 2, K // 2, fmt)


def first_call_captured():
    M, N, K, fmt = 70, 300, 4096, 1
    X, W = torch.empty((M, K), device="cuda"), torch.empty((N, K), device="cuda")
    offsets = torch.tensor([0, 30, 70], dtype=torch.int32, device="cuda")
    Y, G = torch.zeros((M, N), device="cuda"), torch.zeros((M, N // 2), device="cuda")
    V = torch.zeros((M, K), device="cuda", dtype=torch.bfloat16)
    xq, wq = ([torch.zeros((r, K // b), dtype=torch.uint8, device="cuda") for b in (2, 16)] for r in (M, N))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        elutq.elutq_mx4_quantize(X, M, K, fmt, codes=xq[0], scales=xq[1])
        elutq.elutq_mx4_quantize(W, N, K, fmt, codes=wq[0], scales=wq[1])
        elutq.elutq_mx4_gemm(*xq, *wq, Y, M, N, K, fmt)
        elutq.elutq_mx4_gemm_grouped(*xq, *wq, offsets, G, M, N // 2, K, 2, fmt)
        elutq.elutq_mx4_dequantize(*xq, V, M, K, fmt)
    for seed in range(2):
        rng = np.random.default_rng(seed)
        x, w = rng.standard_normal((M, K)).astype(np.float32), rng.standard_normal((N, K)).astype(np.float32)
        X.copy_(torch.from_numpy(x))
        W.copy_(torch.from_numpy(w))
        graph.replay()
        torch.cuda.synchronize()
        assert elutq.elutq_device_status() == 0
        (xc, xs), (wc, ws) = mx4.quantize(x, fmt), mx4.quantize(w, fmt)
        _assert_close(Y, mx4.matmul(xc, xs, wc, ws, fmt), mx4.magnitude(xc, xs, wc, ws, fmt), K, "f32")
        for e, (lo, hi) in enumerate(((0, 30), (30, 70))):
            part = xc[lo:hi], xs[lo:hi], wc[e * 150 : (e + 1) * 150], ws[e * 150 : (e + 1) * 150]
            _assert_close(G[lo:hi], mx4.matmul(*part, fmt), mx4.magnitude(*part, fmt), K, "f32")
        assert np.array_equal(V.double().cpu().numpy(), mx4.values(xc, xs, fmt))


def test_a_process_whose_first_calls_are_captured():
    code = "import sys; sys.path.insert(0, 'tests'); import test_mx4_calls_gpu as t; t.first_call_captured()"
    run = subprocess.run([sys.executable, "-c", code], cwd=ROOT, env=dict(os.environ, PYTHONPATH=ROOT), capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]


def test_products_from_several_threads_and_streams():
    import threading
    M, N, K, fmt = 33, 700, 1024, 0
    rng = np.random.default_rng(1)
    x, w = rng.standard_normal((M, K)).astype(np.float32), rng.standard_normal((N, K)).astype(np.float32)
    X, W = torch.from_numpy(x).cuda(), torch.from_numpy(w).cuda()
    xq, wq = elutq.elutq_mx4_quantize(X, M, K, fmt), elutq.elutq_mx4_quantize(W, N, K, fmt)
    want = torch.empty((M, N), device="cuda")
    elutq.elutq_mx4_gemm(*xq, *wq, want, M, N, K, fmt)
    torch.cuda.synchronize()
    outs, failed = [torch.zeros((20, M, N), device="cuda") for _ in range(4)], []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for k in range(20):
                    q = elutq.elutq_mx4_quantize(X, M, K, fmt)
                    elutq.elutq_mx4_gemm(*q, *wq, outs[i][k], M, N, K, fmt)
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not failed and all(torch.equal(o, want.expand_as(o)) for o in outs)
