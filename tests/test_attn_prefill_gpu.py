"""Attention over packed prompts, against the definition in 64 bits."""

import numpy as np
import pytest
import torch

import paper_2510_19482_b200 as elutq
from kv_util import HALF_STEP, TYPES, dev, ints, rounded
from oracle import attention

pytestmark = pytest.mark.gpu


def make(rng, lens, keys, Hq, H, D, dtype):
    q = rng.standard_normal((sum(lens), Hq, D)).astype(np.float32)
    k = rng.standard_normal((sum(keys), H, D)).astype(np.float32)
    k = np.where(rng.random((H, D)) < 0.05, k * 6, k)
    v = rng.standard_normal((sum(keys), H, D)).astype(np.float32)
    return [rounded(x, dtype) for x in (q, k, v)]


def run(q, k, v, lens, keys, dtype, causal=True, scale=None, max_q=None):
    qd, kd, vd = (dev(x, dtype) for x in (q, k, v))
    out = torch.full(qd.shape, 77.0, dtype=qd.dtype, device="cuda")
    elutq.elutq_attn_prefill(qd, kd, vd, out, ints(np.cumsum([0] + lens)), ints(np.cumsum([0] + keys)), max_q or max(lens), scale=scale, causal=causal)
    torch.cuda.synchronize()
    assert elutq.elutq_device_status() == 0
    return out.double().cpu().numpy()


def check(got, q, k, v, lens, keys, dtype, causal=True, scale=None, rows=None):
    """Every element of the rows (all, or some of each sequence) against the bound."""
    D, at, ak = q.shape[2], 0, 0
    scale = D ** -0.5 if scale is None else scale
    for n, m in zip(lens, keys):
        pick = np.arange(n) if rows is None else np.unique(np.clip(np.array(rows), 0, max(n - 1, 0)))[: max(n, 0)]
        sees = np.minimum(m, pick + 1 + m - n) if causal else np.full(len(pick), m)
        out, mag, span, big = attention.attend(q[at + pick], k[ak : ak + m], v[ak : ak + m], scale, sees)
        tol = attention.tolerance(out, mag, span, big, D, max(m, 1), HALF_STEP[dtype], HALF_STEP[dtype])
        err = np.abs(got[at + pick] - out)
        assert (err <= tol).all(), (n, m, float((err / tol).max()), float(np.nanmax(err)), np.argwhere(~(err <= tol))[0])
        at, ak = at + n, ak + m


CASES = [  # D, Hq, H, queries, keys
    (128, 1, 1, [128], None), (128, 2, 1, [1], None), (64, 1, 1, [300], None), (128, 4, 2, [127, 129, 1, 0, 256], None), (64, 6, 2, [5, 200, 31], None),
    (128, 3, 1, [260, 128], [400, 128]), (64, 8, 2, [1, 17, 140], [500, 17, 900]), (128, 2, 2, [200, 64], [90, 64]), (64, 5, 1, [130, 3], [1, 0]), (128, 8, 1, [70] * 9, None)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D,Hq,H,lens,keys", CASES)
def test_prefill(D, Hq, H, lens, keys, dtype, causal):
    rng = np.random.default_rng(D + Hq + sum(lens))
    keys = keys or lens
    q, k, v = make(rng, lens, keys, Hq, H, D, dtype)
    check(run(q, k, v, lens, keys, dtype, causal), q, k, v, lens, keys, dtype, causal)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f16", 64)])
def test_long_prompt(dtype, D):
    """Many tiles of keys: every ring slot several times over."""
    rng = np.random.default_rng(D)
    lens = [2500, 1111]
    q, k, v = make(rng, lens, lens, 4, 2, D, dtype)
    check(run(q, k, v, lens, lens, dtype), q, k, v, lens, lens, dtype, rows=[0, 1, 127, 128, 500, 1110, 1111, 2047, 2048, 2303, 2499])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_scores_that_climb_and_fall(dtype):
    rng = np.random.default_rng(3)
    H, D, n = 2, 128, 700
    q, k, v = make(rng, [n, n], [n, n], H, H, D, dtype)
    u = rng.standard_normal((H, D))
    u /= np.linalg.norm(u, axis=1, keepdims=True)
    q = rounded(q * 0.05 + u, dtype)
    ramp = np.linspace(-120, 120, n)[:, None, None]
    k = rounded(np.concatenate([k[:n] * 0.1 + u * ramp, k[n:] * 0.1 - u * ramp]), dtype)
    check(run(q, k, v, [n, n], [n, n], dtype, scale=0.7), q, k, v, [n, n], [n, n], dtype, scale=0.7, rows=[0, 1, 50, 127, 128, 129, 300, 511, 512, 699])


@pytest.mark.parametrize("D", [64, 128])
def test_what_is_not_seen_does_not_matter(D):
    """Infinities and NaN in later tokens, in the next sequence and behind the last one: rows that do not see them are as if they were not there, rows that do are not finite."""
    rng = np.random.default_rng(D)
    lens, H, Hq = [70, 200], 1, 2
    q, k, v = make(rng, lens, lens, Hq, H, D, "f16")
    k2, v2 = k.copy(), v.copy()
    v2[70 + 150, 0, 3], v2[70 + 180, 0, :], k2[70 + 190, 0, 0], k2[60, 0, 1], v2[65, 0, 0] = np.inf, np.nan, np.nan, np.inf, -np.inf
    pad = np.full((100, H, D), np.nan)
    got = run(np.concatenate([q, np.full((100, Hq, D), np.nan)]), np.concatenate([k2, pad]), np.concatenate([v2, pad]), lens, lens, "f16")
    assert (got[270:] == 77).all()
    got = got[:270]
    clean = run(q, k, v, lens, lens, "f16")
    same = [r for r in range(270) if r < 60 or 70 <= r < 70 + 150]
    check(np.where(np.isin(np.arange(270), same)[:, None, None], got, clean), q, k, v, lens, lens, "f16")
    assert np.isfinite(got[same]).all()
    assert not np.isfinite(got[70 + 150 :, :, 3]).any() and not np.isfinite(got[70 + 180 :]).any()
    assert not np.isfinite(got[65:70, :, 0]).any() and np.isnan(got[60:65]).any()
    # between the two, only what the infinity touches
    others = np.delete(np.arange(D), 3)
    assert np.isfinite(got[70 + 150 : 70 + 180][:, :, others]).all()


def test_infinite_scores_are_masked_or_win():
    """A key that makes a score of minus infinity has no weight."""
    rng = np.random.default_rng(8)
    q, k, v = make(rng, [200], [200], 1, 1, 64, "bf16")
    q, k = np.abs(q), k.copy()
    k[100, 0, :] = -np.inf
    got = run(q, k, v, [200], [200], "bf16")
    keep = np.delete(np.arange(200), 100)
    q2, k2, v2 = q[150:], k[keep], v[keep]
    out, mag, span, big = attention.attend(q2, k2, v2, 0.125, np.arange(150, 200))
    assert (np.abs(got[150:] - out) <= attention.tolerance(out, mag, span, big, 64, 200, HALF_STEP["bf16"], HALF_STEP["bf16"])).all()


def test_merged_rows_and_rows_of_no_sequence():
    rng = np.random.default_rng(6)
    Hq, H, D, lens = 6, 2, 128, [33, 150]
    n = sum(lens)
    q, k, v = make(rng, [n], [n], Hq, H, D, "bf16")
    rows = 10 + n + 7
    merged = torch.full((rows, Hq + 2 * H + 1, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    merged[10 : 10 + n, : Hq + 2 * H] = dev(np.concatenate([q, k, v], axis=1), "bf16")
    wide = torch.full((rows, Hq + 2, D), 5.0, dtype=torch.bfloat16, device="cuda")
    cu = ints([10, 43, 10 + n])
    elutq.elutq_attn_prefill(merged[:, :Hq], merged[:, Hq : Hq + H], merged[:, Hq + H : Hq + 2 * H], wide[:, 1 : 1 + Hq], cu, cu, 1000)
    got = wide.double().cpu().numpy()
    check(got[10 : 10 + n, 1 : 1 + Hq], q, k, v, lens, lens, "bf16")
    assert (got[:10] == 5).all() and (got[10 + n :] == 5).all() and (got[:, 0] == 5).all() and (got[:, -1] == 5).all()
    # one head of a wider tensor, a single token of any stride
    one = torch.empty((1, 1, D), dtype=torch.bfloat16, device="cuda")
    x = merged[10:11, 0:1]
    elutq.elutq_attn_prefill(x, merged[10:11, Hq : Hq + 1], merged[10:11, Hq + H : Hq + H + 1], one, ints([0, 1]), ints([0, 1]), 1)
    assert torch.equal(one, merged[10:11, Hq + H : Hq + H + 1])


def test_borders_out_of_range_are_cut():
    rng = np.random.default_rng(1)
    q, k, v = (dev(x, "f16") for x in make(rng, [100], [100], 2, 1, 64, "f16"))
    want = torch.empty_like(q)
    elutq.elutq_attn_prefill(q, k, v, want, ints([0, 100]), ints([0, 100]), 100)
    for cq, ck in (([-5, 2 ** 31 - 1], [-9, 10 ** 9]), ([0, 100, 50], [0, 100, 20])):
        got = torch.empty_like(q)
        elutq.elutq_attn_prefill(q, k, v, got, ints(cq), ints(ck), 100)
        assert torch.equal(got, want)


def test_waits_that_run_out():
    """Nothing is loaded: every role gives up, the status says so, and the next call works."""
    rng = np.random.default_rng(1)
    q, k, v = (dev(x, "bf16") for x in make(rng, [600], [600], 4, 2, 128, "bf16"))
    out, cu = torch.empty_like(q), ints([0, 600])
    want = torch.empty_like(q)
    elutq.elutq_attn_prefill(q, k, v, want, cu, cu, 600)
    elutq.elutq_attn_test_wait_expiry(q, k, v, out, cu, cu, 600, 1000)
    assert elutq.elutq_device_status() == 0x7C05
    elutq.elutq_release_scratch()
    assert elutq.elutq_device_status() == 0
    elutq.elutq_attn_prefill(q, k, v, out, cu, cu, 600)
    assert elutq.elutq_device_status() == 0 and torch.equal(out, want)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("scale", [1e3, 3e7, 1e9, 3e12, 1e28])
def test_scores_of_any_size(dtype, scale):
    """One key is nearest to all queries by far, or two are equally near: the result is its value, or their mean, however large the scores.  Scores of fp32 are off by
    (D + 8) 2^-23 of 1e3 at most, before the scale; the nearest is ahead by more than 10.  The weights and the result are rounded once each."""
    rng = np.random.default_rng(1)
    H, D, lens, near = 2, 128, [200, 150], [[3], [2, 5]]
    q, k, v = make(rng, lens, lens, H, H, D, dtype)
    u = rng.choice([-1.0, 1.0], (H, D)).astype(np.float32)
    q[:] = u
    k[:200] = rounded(k[:200] * 0.01 - u * 4, dtype)           # (scores below zero)
    k[200:] = rounded(k[200:] * 0.01 + u * 2, dtype)
    k[3], k[202], k[205] = u * -2, u * 4, u * 4
    got = run(q, k, v, lens, lens, dtype, scale=scale)
    for at, n, rows in ((0, 200, near[0]), (200, 150, near[1])):
        want = v[at : at + n][rows].astype(np.float64)
        tol = (2 * HALF_STEP[dtype] + 2.0 ** -16) * np.abs(want).mean(0) + 2.0 ** -24
        assert (np.abs(got[at + rows[-1] : at + n] - want.mean(0)) <= tol).all()


@pytest.mark.parametrize("lens,max_q", [([0, 3, 40, 1, 17] * 15 + [300, 2], 400), ([2, 0, 1, 3, 0] * 300, 2 ** 30), ([1] * 33 + [600], 1024)])
def test_many_sequences(lens, max_q):
    """More than the 32 that are looked at together, several pairs of tiles for every CTA, longest lengths far above the true ones."""
    rng = np.random.default_rng(len(lens))
    q, k, v = make(rng, lens, lens, 6, 2, 64, "bf16")
    check(run(q, k, v, lens, lens, "bf16", max_q=max_q), q, k, v, lens, lens, "bf16")


def test_queries_beyond_the_longest_are_left_out():
    rng = np.random.default_rng(2)
    lens = [300, 100]
    q, k, v = make(rng, lens, lens, 2, 1, 64, "f16")
    got = run(q, k, v, lens, lens, "f16", max_q=101)
    assert (got[128:300] == 77).all()
    full = run(q, k, v, lens, lens, "f16")
    assert np.array_equal(got[:128], full[:128]) and np.array_equal(got[300:], full[300:])
    check(full, q, k, v, lens, lens, "f16")
