"""Attention of new tokens over a paged cache, against the definition in 64 bits on what the cache holds."""

import numpy as np
import pytest
import torch

import paper_2510_19482_b200 as elutq
from kv_util import HALF_STEP, TYPES, Paged, dev, ints, rounded
from oracle import attention

pytestmark = pytest.mark.gpu


def check(got, p, q, new, scale, Hq, skip=()):
    """Every element of the result against the bound; q fp32 [B * new, Hq, D]."""
    p_step = HALF_STEP["bf16"] if p.fmt == 0 and p.dtype == "bf16" else HALF_STEP["f16"]
    for b, n in enumerate(p.lens):
        if b in skip:
            continue
        rows = slice(b * new, (b + 1) * new)
        sees = n - new + 1 + np.arange(new)
        out, mag, span, big = attention.attend(q[rows], p.held[0][b], p.held[1][b], scale, sees)
        tol = attention.tolerance(out, mag, span, big, p.D, max(n, 1), p_step, HALF_STEP[p.dtype])
        err = np.abs(got[rows] - out)
        assert (err <= tol).all(), (b, n, float((err / tol).max()), float(err.max()))


def call(p, q, new, scale=None, **kw):
    qd = dev(q, p.dtype)
    out = torch.full(qd.shape, float("nan"), dtype=qd.dtype, device="cuda")
    elutq.elutq_attn_decode(p.cache, qd, out, p.table_d, p.lens_d, new, scale=scale, **kw)
    torch.cuda.synchronize()
    return out.double().cpu().numpy()


def data(rng, lens, H, D):
    k = [rng.standard_normal((n, H, D)).astype(np.float32) for n in lens]
    big = rng.random((H, D)) < 0.05
    return [np.where(big, x * 6, x).astype(np.float32) for x in k], [rng.standard_normal((n, H, D)).astype(np.float32) for n in lens]


SHAPES = [  # D, Hq, H, new, page, lens
    (128, 32, 8, 1, 64, [1000]), (128, 8, 8, 1, 16, [1, 15, 16, 17, 0, 63, 64, 65, 129]), (128, 9, 1, 1, 48, [300, 1]), (64, 15, 5, 4, 16, [1, 2, 3, 4, 5, 100, 777]),
    (64, 64, 1, 1, 32, [513]), (128, 16, 1, 5, 128, [7, 0, 2000]), (64, 4, 4, 1, 64, [5000, 3]), (128, 6, 2, 2, 16, [1, 31, 33]), (64, 8, 1, 1, 16, [64] * 70)]


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D,Hq,H,new,page,lens", SHAPES)
def test_decode(fmt, dtype, D, Hq, H, new, page, lens):
    rng = np.random.default_rng(len(lens) + D + Hq)
    p = Paged(rng, fmt, dtype, lens, H, D, page, *data(rng, lens, H, D))
    q = rounded(rng.standard_normal((len(lens) * new, Hq, D)), dtype)
    check(call(p, q, new), p, q, new, D ** -0.5, Hq)


@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_scores_that_climb_and_fall(fmt):
    """Scores over hundreds, rising along the sequence, falling along it, or one key far above all others."""
    rng = np.random.default_rng(fmt)
    H, D, lens = 3, 128, [900, 900, 900]
    k, v = data(rng, lens, H, D)
    q = rounded(rng.standard_normal((3, H, D)), "bf16")
    unit = q / np.linalg.norm(q, axis=2, keepdims=True)
    ramp = np.linspace(-150, 150, 900, dtype=np.float32)[:, None, None]
    k[0] = (k[0] * 0.1 + unit[0] * ramp).astype(np.float32)
    k[1] = (k[1] * 0.1 - unit[1] * ramp).astype(np.float32)
    k[2][777] = unit[2] * 300
    p = Paged(rng, fmt, "bf16", lens, H, D, 64, k, v)
    check(call(p, q, 1, scale=0.5), p, q, 1, 0.5, H)


def test_queries_of_any_size():
    """bf16 queries from 1e-35 to 1e30 beside codes: brought to fp16 by a power of two; the scale makes scores ordinary again."""
    rng = np.random.default_rng(5)
    H, D, lens = 2, 64, [200] * 4
    for fmt in (1, 2):
        p = Paged(rng, fmt, "bf16", lens, H, D, 16, *data(rng, lens, H, D))
        for size in (1e-35, 1e-6, 1e9, 1e30 / 2 ** 8):
            q = rounded(rng.standard_normal((4, 4, D)) * size, "bf16")
            if size == 1e-6:
                q[1] = 0
            scale = float(np.float32(min(0.1 / size, 9e29)))
            check(call(p, q, 1, scale=scale), p, q, 1, scale, 4)


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("new", [1, 3])
def test_masked_places_hold_anything(fmt, new):
    """Behind the sequence: infinities and NaN (the pool is filled with them).  A new token's own K and V that are not finite reach its own row and later ones only."""
    rng = np.random.default_rng(fmt)
    H, Hq, D, lens = 2, 6, 128, [50, 65, 3]
    k, v = data(rng, lens, H, D)
    q = rounded(rng.standard_normal((3 * new, Hq, D)), "f16")
    if new == 3:
        if fmt == 0:
            v[0][-1, 0, 5], v[1][-1, 1, :], k[2][-1, 0, 9] = np.inf, np.nan, np.nan
        else:
            v[0][-1, 0, 5], v[1][-1, 1, :], k[2][-1, 0, 9] = np.nan, np.nan, np.nan
    p = Paged(rng, fmt, "f16", lens, H, D, 16, k, v)
    got = call(p, q, new)
    clean = [np.nan_to_num(x, nan=0.0, posinf=0.0, neginf=0.0) for x in p.held[0]], [np.nan_to_num(x, nan=0.0, posinf=0.0, neginf=0.0) for x in p.held[1]]
    bad = ~np.isfinite(got)
    if new == 3:
        want = np.zeros_like(bad)
        want[2, :3, :] = ~np.isfinite(p.held[1][0][-1, 0])[None, :]
        want[5, 3:, :] = True
        want[8, :3, :] = True
        assert np.array_equal(bad, want)
    else:
        assert not bad.any()
    p.held = clean
    check(np.where(bad, np.concatenate([attention.attend(q[b * new : b * new + new], clean[0][b], clean[1][b], D ** -0.5, lens[b] - new + 1 + np.arange(new))[0]
                                        for b in range(3)]), got), p, q, new, D ** -0.5, Hq)


@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_pages_outside_the_cache_count_as_masked(fmt):
    rng = np.random.default_rng(11)
    H, D, n = 2, 64, 200
    k, v = data(rng, [n], H, D)
    p = Paged(rng, fmt, "f16", [n], H, D, 16, k, v)
    p.table_d[0, 3], p.table_d[0, 11] = -5, p.data[0].shape[0]
    q = rounded(rng.standard_normal((1, 4, D)), "f16")
    got = call(p, q, 1)
    keep = [j for j in range(n) if j // 16 not in (3, 11)]
    p.held = [[p.held[0][0][keep]], [p.held[1][0][keep]]]
    p.lens = [len(keep)]
    check(got, p, q, 1, D ** -0.5, 4)
    p.table_d.fill_(-1)
    assert (call(p, q, 1) == 0).all()


def test_lengths_outside_the_table():
    """Lengths are cut to what the table has room for; below zero is zero."""
    rng = np.random.default_rng(2)
    H, D = 2, 128
    p = Paged(rng, 0, "f16", [64, 64], H, D, 16, *data(rng, [64, 64], H, D))
    q = rounded(rng.standard_normal((2, 2, D)), "f16")
    want = call(p, q, 1)
    p.lens_d = ints([2 ** 31 - 1, -7])
    got = call(p, q, 1)
    assert np.array_equal(got[0], want[0]) and (got[1] == 0).all()


def test_strided_rows_and_results():
    rng = np.random.default_rng(4)
    H, Hq, D, lens = 2, 4, 64, [100, 30, 64]
    p = Paged(rng, 2, "bf16", lens, H, D, 16, *data(rng, lens, H, D))
    wide = torch.full((3, Hq + 3, D), 9.0, dtype=torch.bfloat16, device="cuda")
    q = rounded(rng.standard_normal((3, Hq, D)), "bf16")
    merged = torch.zeros((3, Hq + 2 * H, D), dtype=torch.bfloat16, device="cuda")
    merged[:, :Hq] = dev(q, "bf16")
    table = torch.full((3, p.table.shape[1] + 5), 2 ** 30, dtype=torch.int32, device="cuda")
    table[:, : p.table.shape[1]] = p.table_d
    elutq.elutq_attn_decode(p.cache, merged[:, :Hq], wide[:, 1 : 1 + Hq], table[:, : p.table.shape[1]], p.lens_d)
    got = wide.double().cpu().numpy()
    check(got[:, 1 : 1 + Hq], p, q, 1, D ** -0.5, Hq)
    assert (got[:, 0] == 9).all() and (got[:, 1 + Hq :] == 9).all()


def test_the_same_bits_every_time_in_any_batch_order():
    """Joining goes by place, not by time: twice the same call gives the same bits."""
    rng = np.random.default_rng(9)
    lens = [3000, 1, 777, 4096, 50]
    p = Paged(rng, 1, "f16", lens, 4, 128, 64, *data(rng, lens, 4, 128))
    q = rounded(rng.standard_normal((5, 32, 128)), "f16")
    first = call(p, q, 1)
    for _ in range(3):
        assert np.array_equal(first, call(p, q, 1))


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("scale", [1e3, 3e7, 1e9, 3e12, 1e28])
def test_scores_of_any_size(fmt, scale):
    """One key is nearest to the query by far, or two are equally near: the result is its value, or their mean, however large the scores.  Scores of fp32 are off by
    (D + 8) 2^-23 of 1e3 at most, before the scale; the nearest is ahead by more than 10.  The weights and the result are rounded once each."""
    rng = np.random.default_rng(fmt)
    H, D, lens = 3, 128, [300, 700, 5000, 40]
    k, v = data(rng, lens, H, D)
    u = rng.choice([-1.0, 1.0], (H, D)).astype(np.float32)
    near = [[7], [3, 600], [4000], [39]]
    for b in range(4):
        k[b] = k[b] * 0.01 + u * (2.0 if b % 2 else -4.0)      # (scores below zero, too)
        k[b][near[b]] = u * (4.0 if b % 2 else -2.0)
    p = Paged(rng, fmt, "bf16", lens, H, D, 64, k, v, factors=False)
    q = rounded(np.tile(u, (4, 1, 1)), "bf16")
    got = call(p, q, 1, scale=scale)
    for b in range(4):
        want = p.held[1][b][near[b]]
        tol = (2 * HALF_STEP["bf16"] + 2.0 ** -16) * np.abs(want).mean(0)
        assert (np.abs(got[b] - want.mean(0)) <= tol).all(), (b, float(np.nanmax(np.abs(got[b] - want.mean(0)))))


@pytest.mark.parametrize("fmt,D,Hq,new", [(0, 64, 8, 1), (2, 128, 32, 4), (1, 64, 16, 1)])
@pytest.mark.parametrize("longest", [40, 1700])
def test_more_segments_than_shares(fmt, D, Hq, new, longest):
    """Hundreds of short sequences, some empty, one long or all short: several segments to a share, or a cluster to each."""
    rng = np.random.default_rng(longest)
    H = 8
    lens = [int(x) for x in rng.integers(0, 40, 260)]
    lens[77] = longest
    p = Paged(rng, fmt, "f16", lens, H, D, 16, *data(rng, lens, H, D))
    q = rounded(rng.standard_normal((260 * new, Hq, D)), "f16")
    check(call(p, q, new), p, q, new, D ** -0.5, Hq)


@pytest.mark.parametrize("wide", [1, 400])
def test_all_sequences_empty(wide):
    rng = np.random.default_rng(3)
    p = Paged(rng, 1, "bf16", [0, 0, 0], 2, 64, 16)
    p.table_d = ints(np.zeros((3, wide)))
    assert (call(p, rounded(rng.standard_normal((6, 4, 64)), "bf16"), 2) == 0).all()
