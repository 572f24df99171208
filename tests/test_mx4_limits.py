"""4-bit operators: sizes at the ends of what they accept, on the host (no GPU needed)."""

import os
import subprocess
import sys

import pytest

import paper_2510_19482_b200 as elutq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("K", [(1 << 28) + 32, (1 << 31) - 512, (1 << 31) - 480, (1 << 31) - 32])
def test_products_turn_down_a_longer_k(K):
    """In front of any arithmetic on K: rounding it up to steps would pass 32 bits."""
    L, before = elutq.lib(), elutq.elutq_launch_count()
    for M in (1, 40, 1000):
        for fmt in (0, 1):
            assert L.elutq_mx4_gemm(16, 16, 16, 16, 16, 0, M, 4, K, fmt, None, None) == -2
            assert L.elutq_mx4_gemm_grouped(16, 16, 16, 16, 16, 16, 0, M, 4, K, 2, fmt, None, None) == -2
    assert elutq.elutq_launch_count() == before


def test_releasing_nothing_needs_no_gpu():
    """Nothing allocated and no 4-bit product launched: no CUDA call.  (A process of its own: others here may have a GPU and use it.)"""
    code = "import paper_2510_19482_b200 as e; raise SystemExit(-e.lib().elutq_release_scratch())"
    env = dict(os.environ, CUDA_VISIBLE_DEVICES="", PYTHONPATH=ROOT + os.pathsep + os.environ.get("PYTHONPATH", ""))
    assert subprocess.run([sys.executable, "-c", code], env=env, cwd=ROOT, timeout=120).returncode == 0
