"""The status of the 4-bit products: who reads it, when, and what clears it."""

import ctypes
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2510_19482_b200 as elutq
from test_mx4_gemm_gpu import _dev, _matrix

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _status_during_a_capture(stream):
    """elutq_device_status of `stream` while another one is captured (in the mode that lets a thread wait meanwhile), one that the default stream waits for; the
    graph is replayed afterwards."""
    x, y = torch.arange(64, device="cuda", dtype=torch.float32), torch.zeros(64, device="cuda")
    torch.cuda.synchronize()
    raw = ctypes.c_void_p()
    assert ctypes.CDLL("libcudart.so.12").cudaStreamCreate(ctypes.byref(raw)) == 0
    graph, capturing = torch.cuda.CUDAGraph(), torch.cuda.ExternalStream(raw.value)
    with torch.cuda.graph(graph, stream=capturing, capture_error_mode="relaxed"):
        y.copy_(x)
        status = elutq.elutq_device_status(stream)
        y.add_(1.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, x + 1.0)
    return status


def status_where_no_product_ran():
    assert _status_during_a_capture(torch.cuda.Stream()) == 0


def test_reading_the_status_spoils_no_capture_where_no_product_ran():
    """In a process that has launched no 4-bit product."""
    code = "import sys; sys.path.insert(0, 'tests'); import test_mx4_status_gpu as t; t.status_where_no_product_ran()"
    run = subprocess.run([sys.executable, "-c", code], cwd=ROOT, env=dict(os.environ, PYTHONPATH=ROOT), capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]


def test_reading_the_status_spoils_no_capture_behind_a_product():
    rng = np.random.default_rng(0)
    M, N, K = 5, 256, 512
    args, Y = _dev(*_matrix(rng, M, K, 0), *_matrix(rng, N, K, 0)), torch.empty((M, N), device="cuda")
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    elutq.elutq_mx4_gemm(*args, Y, M, N, K, 0, stream=stream)
    assert _status_during_a_capture(stream) == 0
    elutq.elutq_mx4_test_wait_expiry(*args, Y, M, N, K, 0, 1000, stream=stream)
    assert _status_during_a_capture(stream) == 0x7C05
    assert elutq.elutq_device_status() == 0x7C05              # on any stream of the device
    elutq.elutq_release_scratch()
    assert elutq.elutq_device_status(stream) == 0
    assert _status_during_a_capture(stream) == 0
