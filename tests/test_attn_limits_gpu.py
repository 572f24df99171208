"""Attention at the limits of its types: rows whose scores vanish, values next to the largest, a channel far above the others."""

import time

import numpy as np
import pytest
import torch

import paper_2510_19482_b200 as elutq
from kv_util import HALF_STEP, TYPES, Paged, dev, ints, rounded
from oracle import attention
from test_attn_decode_gpu import call, check, data
from test_attn_prefill_gpu import check as check_prefill
from test_attn_prefill_gpu import make, run

pytestmark = pytest.mark.gpu


def with_factors(p, kf, vf=1.0):
    """The cache of p (made without factors), its values times these."""
    f = [torch.full((p.heads,), float(x), device="cuda") for x in (kf, vf)]
    p.held = [[h * float(np.float32(x)) for h in held] for held, x in zip(p.held, (kf, vf))]
    p.cache = elutq.KvCache(p.fmt, TYPES[p.dtype], p.data[0], p.data[1], p.scales[0], p.scales[1], k_factor=f[0], v_factor=f[1])
    return p


@pytest.mark.parametrize("fmt", [1, 2])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new", [1, 3])
@pytest.mark.parametrize("wide", [64, 20000])
@pytest.mark.parametrize("kf,scale", [(1e-8, None), (1.0, 1e-8), (1e-30, 1e-30), (1e-44, 1e-3)])
def test_rows_whose_scores_vanish(fmt, dtype, new, wide, kf, scale):
    """Queries of zeros, of the smallest magnitudes, and ordinary ones, over keys whose factor times the scale is far below what queries of such rows are brought back with: every visible
    value counts the same, and places behind the sequence or on a missing page count nothing."""
    rng = np.random.default_rng(fmt)
    H, Hq, D, lens = 2, 4, 128, [17, 50, 3, 64]
    p = with_factors(Paged(rng, fmt, dtype, lens, H, D, 16, *data(rng, lens, H, D), factors=False), kf)
    table = np.full((4, wide // 16), -1, dtype=np.int32)
    table[:, : p.table.shape[1]] = p.table
    p.table_d = ints(table)
    q = rounded(rng.standard_normal((4 * new, Hq, D)), dtype)
    q[:, 0], q[:, 1, 1:] = 0, 0
    q[:, 3] = rounded(q[:, 3] * 2.0 ** -130 if dtype == "bf16" else q[:, 3] * 2.0 ** -20, dtype)
    check(call(p, q, new, scale=scale), p, q, new, D ** -0.5 if scale is None else scale, Hq)
    p.table_d[1, 1] = -1
    got = call(p, q, new, scale=scale)
    keep = np.r_[0:16, 32:50]
    p.held = [[h if b != 1 else h[keep] for b, h in enumerate(x)] for x in p.held]
    p.lens = [17, 34, 3, 64]
    check(got, p, q, new, D ** -0.5 if scale is None else scale, Hq)


@pytest.mark.parametrize("new", [1, 3])
@pytest.mark.parametrize("wide", [736, 20000])
@pytest.mark.parametrize("size", [2e34, 1e37, 3e38, 1e-30])
def test_values_next_to_the_largest(new, wide, size):
    """bf16 values up to the type's largest: their means are finite, whatever the weights and however many there are, and small ones keep their bits.  In units of `size` the bound is that of
    ordinary values; besides, n products are off by half of the smallest subnormal step, against a largest weight of 2^-(bits of n + 11) at least."""
    rng = np.random.default_rng(1)
    H, Hq, D, lens = 2, 6, 128, [1, 40, 700, 730]
    k, _ = data(rng, lens, H, D)
    v = [rng.uniform(0.3, 1.0, x.shape) * size for x in k]
    p = Paged(rng, 0, "bf16", lens, H, D, 16, k, v)
    table = np.full((4, wide // 16), -1, dtype=np.int32)
    table[:, : p.table.shape[1]] = p.table
    p.table_d = ints(table)
    q = rounded(rng.standard_normal((4 * new, Hq, D)) * rng.choice([0.0, 0.2, 3.0], (4 * new, Hq, 1)), "bf16")
    got = call(p, q, new) / size
    for b, n in enumerate(lens):
        rows = slice(b * new, (b + 1) * new)
        out, mag, span, _ = attention.attend(q[rows], p.held[0][b], p.held[1][b] / size, D ** -0.5, n - new + 1 + np.arange(new))
        tol = attention.tolerance(out, mag, span, np.zeros_like(span), D, n, HALF_STEP["bf16"], HALF_STEP["bf16"]) + n * 2.0 ** (n.bit_length() + 11 - 150) / size
        assert (np.abs(got[rows] - out) <= tol).all(), (b, float((np.abs(got[rows] - out) / tol).max()))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("size", [2e34, 1e37, 3e38])
def test_values_next_to_the_largest_in_prompts(D, causal, size):
    """The same over prompts, in units of `size`."""
    rng = np.random.default_rng(D)
    lens, Hq, H = [1, 40, 333], 3, 1
    q, k, v = make(rng, lens, lens, Hq, H, D, "bf16")
    v = rounded(rng.uniform(0.3, 1.0, v.shape) * size, "bf16")
    got = run(q, k, v, lens, lens, "bf16", causal) / size
    at = 0
    for n in lens:
        s = slice(at, at + n)
        out, mag, span, _ = attention.attend(q[s], k[s], v[s] / size, D ** -0.5, 1 + np.arange(n) if causal else np.full(n, n))
        tol = attention.tolerance(out, mag, span, np.zeros_like(span), D, n, HALF_STEP["bf16"], HALF_STEP["bf16"])
        assert (np.abs(got[s] - out) <= tol).all(), (n, float((np.abs(got[s] - out) / tol).max()))
        at += n


@pytest.mark.parametrize("fmt", [1, 2])
@pytest.mark.parametrize("far", [2.0 ** 16, 2.0 ** 18, 2.0 ** 22, 2.0 ** 30])
def test_a_channel_far_above_the_others_over_keys_that_are_zero_there(fmt, far):
    """A bf16 query's large channel meets keys that hold zeros: its other channels make up the whole score, and keep their bits down to 2^-32 of the large one."""
    rng = np.random.default_rng(fmt)
    H, Hq, D, lens = 2, 6, 64, [100, 33, 7]
    k, v = data(rng, lens, H, D)
    for x in k:
        x[:, 0, 5], x[:, 1, 60] = 0, 0
    q = rounded(rng.standard_normal((3, Hq, D)), "bf16")
    q[:, :3, 5] = far
    q[:, 3:, 60] = -far
    p = Paged(rng, fmt, "bf16", lens, H, D, 16, k, v, factors=False)
    got = call(p, q, 1, scale=0.5)
    for b, n in enumerate(lens):
        out, mag, span, big = attention.attend(q[b : b + 1], p.held[0][b], p.held[1][b], 0.5, [n])
        # a query's largest value comes to 2^15 at least in fp16, the others to multiples of 2^-24 at the coarsest: off by 2^-25, 2^-40 of the largest.  A score is off by that times the sum of
        # a key's magnitudes; in units of the bound's own error of a score, (D + 8) 2^-23 span, it is added to the span
        cut = 2.0 ** -40 * far * np.abs(p.held[0][b]).sum(2).max() * 0.5
        tol = attention.tolerance(out, mag, span + cut / ((D + 8) * 2.0 ** -23), big, D, n, HALF_STEP["f16"], HALF_STEP["bf16"])
        err = np.abs(got[b : b + 1] - out)
        assert (err <= tol).all(), (b, n, float((err / tol).max()), float(err.max()))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens", [[1], [128], [100, 256], [600], [1300] * 5, [2000, 7] * 40])
def test_waits_that_run_out_behind_the_last_load(D, lens):
    """Loads are issued and no product is: the warp that loads may be through with all of its items before another role gives up.  It leaves when they have landed (a wait for a
    load that is not on its way would take a second), and the next call works."""
    rng = np.random.default_rng(1)
    q, k, v = (dev(x, "bf16") for x in make(rng, [sum(lens)], [sum(lens)], 4, 2, D, "bf16"))
    out, want, cu = torch.empty_like(q), torch.empty_like(q), ints(np.cumsum([0] + lens))
    elutq.elutq_attn_prefill(q, k, v, want, cu, cu, max(lens))
    assert elutq.elutq_device_status() == 0
    begin = time.perf_counter()
    for limit in (1, 40):
        elutq.elutq_attn_test_wait_expiry(q, k, v, out, cu, cu, max(lens), limit | elutq.ATTN_TEST_LOADS)
    assert elutq.elutq_device_status() == 0x7C05
    assert time.perf_counter() - begin < 0.9
    elutq.elutq_release_scratch()
    elutq.elutq_attn_prefill(q, k, v, out, cu, cu, max(lens))
    assert elutq.elutq_device_status() == 0 and torch.equal(out, want)


def test_results_beside_their_inputs_in_one_buffer():
    """Columns of the same rows: heads of q, k, v, of the rotated queries and keys, and of results, side by side."""
    rng = np.random.default_rng(0)
    Hq, H, D, n = 4, 2, 64, 70
    p = Paged(rng, 0, "f16", [n], H, D, 16)
    x = rounded(rng.standard_normal((n, Hq + 2 * H, D)), "f16")
    wide = torch.zeros((n, 3 * Hq + 3 * H, D), dtype=torch.float16, device="cuda")
    wide[:, : Hq + 2 * H] = dev(x, "f16")
    q, k, v, q_out, k_out, out = torch.split(wide, [Hq, H, H, Hq, H, Hq], dim=1)
    rope = elutq.elutq_rope_table(n, D)
    elutq.elutq_kv_write(p.cache, k, v, ints(p.slots(0, np.arange(n))), q=q, q_out=q_out, k_out=k_out, positions=ints(np.arange(n)), rope=rope)
    turned = rounded(attention.rotate(x[:, : Hq + H], rope.cpu().numpy(), np.arange(n), False), "f16")
    cu = ints([0, n])
    elutq.elutq_attn_prefill(q_out, k_out, v, out, cu, cu, n)
    got = wide.double().cpu().numpy()
    assert np.array_equal(got[:, : 2 * Hq + 3 * H], np.concatenate([x, turned], axis=1))
    check_prefill(got[:, 2 * Hq + 3 * H :], turned[:, :Hq], turned[:, Hq:], x[:, Hq + H :], [n], [n], "f16")
    # the last token over the cache, its result into columns of the queries' rows
    elutq.elutq_attn_decode(p.cache, q_out[n - 1 :], out[n - 1 :], p.table_d, p.lens_d)
    elutq.elutq_kv_read(p.cache, p.table_d, None, cu, wide[:, :H], wide[:, H : 2 * H])
    p.held = [[turned[:, Hq:].astype(np.float64)], [x[:, Hq + H :].astype(np.float64)]]
    got = wide.double().cpu().numpy()
    check(got[n - 1 :, 2 * Hq + 3 * H :], p, turned[n - 1 :, :Hq], 1, D ** -0.5, Hq)
    assert np.array_equal(got[:, : 2 * H], np.concatenate([turned[:, Hq:], x[:, Hq + H :]], axis=1))
