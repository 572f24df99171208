"""The forms of attention over a cache that the sizes choose between: three CTAs to an SM, shares of the whole with several new tokens, the same bits in every call of each."""

import numpy as np
import pytest

import paper_2510_19482_b200 as elutq
from kv_util import Paged, rounded
from test_attn_decode_gpu import call, check, data

pytestmark = pytest.mark.gpu


def made(seed, fmt, dtype, lens, D, Hq, H, new, page):
    rng = np.random.default_rng(seed)
    p = Paged(rng, fmt, dtype, lens, H, D, page, *data(rng, lens, H, D))
    return p, rounded(rng.standard_normal((len(lens) * new, Hq, D)), dtype)


def workspace(p, Hq, new):
    return elutq.elutq_attn_decode_workspace_bytes(p.cache, p.table.shape[1], len(p.lens), new, Hq)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D,Hq,new,longest", [(128, 32, 1, 900), (128, 16, 4, 200), (64, 96, 1, 900), (64, 24, 4, 500), (64, 24, 8, 300)])
def test_three_ctas_to_an_sm(D, Hq, new, longest, dtype):
    """NVFP4, short tables, 400 segments or 800: one round of three CTAs to an SM where two would take two, two where two would take three."""
    H, B = 8, 50
    rng = np.random.default_rng(D + new)
    lens = [longest, 0] + [int(x) for x in rng.integers(1, longest + 1, B - 2)]
    p, q = made(new, 2, dtype, lens, D, Hq, H, new, 64)
    assert workspace(p, Hq, new) == 0
    got = call(p, q, new)
    check(got, p, q, new, D ** -0.5, Hq)
    assert np.array_equal(got, call(p, q, new))


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("dtype,D,Hq,H,new,page", [("f16", 64, 15, 5, 4, 16), ("bf16", 64, 16, 1, 1, 32), ("bf16", 64, 8, 4, 7, 16), ("f16", 128, 8, 4, 5, 64), ("bf16", 128, 8, 2, 2, 16),
                                                   ("f16", 128, 16, 2, 7, 32), ("bf16", 64, 8, 2, 2, 64)])
def test_shares_of_several_new_tokens(fmt, dtype, D, Hq, H, new, page):
    """Long tables: the sequences' tiles are cut into shares.  One or two tiles of columns, several tiles of query rows, sequences shorter than the new tokens."""
    lens = [1, 5000, 0, new + 1, 777, 33, 16, 1501]
    p, q = made(D + new, fmt, dtype, lens, D, Hq, H, new, page)
    p.table = np.concatenate([p.table, np.full((len(lens), 12000 // page), -1, dtype=np.int32)], axis=1)
    p.table_d = p.table_d.new_tensor(p.table)
    assert workspace(p, Hq, new) > 0
    got = call(p, q, new)
    check(got, p, q, new, D ** -0.5, Hq)
    assert np.array_equal(got, call(p, q, new))


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("wide", [448, 9600])
def test_repeated_calls_give_the_same_bits(fmt, wide):
    """Clusters of eight CTAs, which join through their shared memory, and shares, which a second kernel joins."""
    lens, Hq, H, D, page = [448, 1, 300], 8, 2, 128, 64
    p, q = made(fmt, fmt, "bf16", lens, D, Hq, H, 1, page)
    p.table = np.concatenate([p.table, np.full((3, wide // page - p.table.shape[1]), -1, dtype=np.int32)], axis=1)
    p.table_d = p.table_d.new_tensor(p.table)
    assert (workspace(p, Hq, 1) == 0) == (wide == 448)
    first = call(p, q, 1)
    check(first, p, q, 1, D ** -0.5, Hq)
    for _ in range(5):
        assert np.array_equal(first, call(p, q, 1))
