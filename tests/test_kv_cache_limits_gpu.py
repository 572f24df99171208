"""Reads from a paged cache at the limits of its indices."""

import numpy as np
import pytest
import torch

import paper_2510_19482_b200 as elutq
from kv_util import Paged, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_a_range_that_begins_far_in_front_of_the_rows(fmt):
    """A border far below zero: the tokens of the rows are past 32 bits, have no page, and give zeros."""
    rng = np.random.default_rng(fmt)
    H, D, n, rows = 2, 64, 64, 20
    k, v = ([rng.standard_normal((n, H, D)).astype(np.float32)] for _ in range(2))
    p = Paged(rng, fmt, "f16", [n], H, D, 16, k, v)
    for first, begin in ((2 ** 31 - 1, -2 ** 31), (2 ** 31 - 10, 3 - 2 ** 31), (0, -2 ** 31), (-5, 17 - 2 ** 31)):
        out = torch.full((2, rows, H, D), 5.0, dtype=torch.float16, device="cuda")
        elutq.elutq_kv_read(p.cache, p.table_d, ints([first]), ints([begin, rows]), out[0], out[1])
        assert (out == 0).all(), (first, begin)
