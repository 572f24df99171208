"""Rotary positions, writes into a paged cache and reads from it, against the oracle: rotation and codes bit for bit."""

import numpy as np
import pytest
import torch

import paper_2510_19482_b200 as elutq
from kv_util import TYPES, Paged, dev, ints, rounded
from oracle import attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scaling,kw", [(0, {}), (1, {"factor": 4.0}), (2, {"factor": 8.0, "low": 1.0, "high": 4.0, "original": 8192.0}),
                                        (2, {"factor": 32.0, "low": 0.0, "high": 2.5, "original": 1000.0, "magnitude": 1.25})])
@pytest.mark.parametrize("n_pos,rot,theta", [(1, 16, 10000.0), (1000, 128, 500000.0), (70001, 48, 1e6)])
def test_rope_table(scaling, kw, n_pos, rot, theta):
    magnitude = kw.get("magnitude", 1.0)
    want = attention.angles(n_pos, attention.frequencies(rot, theta, scaling, **{k: v for k, v in kw.items() if k != "magnitude"}), magnitude)
    got = elutq.elutq_rope_table(n_pos, rot, theta, scaling, **kw).cpu().numpy().astype(np.float64)
    # rounded once to fp32 (half a step: 2^-24 of values below 2); the angle itself has few units of 2^-53 of up to 70001, and the power's exponent as many
    assert np.abs(got - want).max() <= magnitude * (2.0 ** -24 + 70001 * 16 * 2.0 ** -53)


def _inputs(rng, tokens, heads, D):
    x = rng.standard_normal((tokens, heads, D)).astype(np.float32)
    x[:, :, rng.integers(0, D, 3)] *= 20
    if tokens > 4:
        x[1] = 0
        x[2, :, : D // 2] = 0
    return x


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("dtype,D,Hq,H,rot,interleaved,tokens,page", [
    ("f16", 128, 32, 8, 128, False, 1, 64), ("bf16", 128, 32, 8, 128, False, 33, 16), ("f16", 64, 15, 5, 32, True, 7, 48), ("bf16", 64, 3, 3, 64, True, 300, 128),
    ("f16", 128, 1, 1, 16, False, 5, 16), ("bf16", 128, 0, 2, 96, False, 40, 32), ("f16", 64, 9, 1, 48, False, 2000, 16), ("f16", 128, 7, 7, 0, False, 9, 16),
    ("bf16", 128, 64, 8, 128, True, 700, 64)])
def test_write(fmt, dtype, D, Hq, H, rot, interleaved, tokens, page):
    rng = np.random.default_rng(1000 * fmt + tokens + D)
    p = Paged(rng, fmt, dtype, [tokens + 5], H, D, page)
    q, k, v = (rounded(_inputs(rng, tokens, h, D), dtype) for h in (max(Hq, 1), H, H))
    n_pos = 5000
    table = attention.angles(n_pos, attention.frequencies(max(rot, 16), 10000.0)).astype(np.float32)
    positions = rng.integers(0, n_pos, tokens)
    slots = rng.permutation(p.slots(0, np.arange(tokens + 5)))[:tokens]
    before = [[t.clone() for t in (p.data[i], p.scales[i]) if t is not None] for i in range(2)]
    # a merged result, q, k and v side by side with something behind them
    merged = dev(np.concatenate([q, k, v, np.zeros((tokens, 1, D))], axis=1), dtype)
    n = max(Hq, 1)
    qd, kd, vd = merged[:, :n], merged[:, n : n + H], merged[:, n + H : n + 2 * H]
    q_out, k_out = torch.full((tokens, n, D), 7.0, dtype=TYPES[dtype], device="cuda"), torch.full((tokens, H, D), 7.0, dtype=TYPES[dtype], device="cuda")
    kw = {"positions": ints(positions), "rope": torch.from_numpy(table).cuda()} if rot else {}
    if Hq:
        kw |= {"q": qd, "q_out": q_out}
    elutq.elutq_kv_write(p.cache, kd, vd, ints(slots), flags=elutq.ROPE_INTERLEAVED if interleaved else 0, k_out=k_out, **kw)
    torch.cuda.synchronize()
    turned = [attention.rotate(x, table, positions, interleaved) if rot else x for x in (q, k)]
    if Hq:
        assert np.array_equal(q_out.float().cpu().numpy(), rounded(turned[0], dtype))
    assert np.array_equal(k_out.float().cpu().numpy(), rounded(turned[1], dtype))
    for i, x in enumerate((turned[1], v)):
        got = p.bytes_at(i, slots)
        if fmt == 0:
            assert np.array_equal(got[0].float().numpy(), rounded(x, dtype))
        else:
            want = attention.stored(x, fmt, p.factors[i])
            assert np.array_equal(got[0].numpy(), want[0])
            assert fmt != 2 or np.array_equal(got[1].numpy(), want[1])
        # every other slot is as it was
        for pool, old in zip([t for t in (p.data[i], p.scales[i]) if t is not None], before[i]):
            s = torch.from_numpy(slots.astype(np.int64)).cuda()
            old[s // page, :, s % page] = pool[s // page, :, s % page]
            assert torch.equal(pool.view(torch.uint8), old.view(torch.uint8))


@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_write_in_place_and_left_out(fmt):
    """q and k rotated in place; tokens without a slot are rotated and not stored, tokens without a position are left alone."""
    rng = np.random.default_rng(fmt)
    tokens, Hq, H, D, page = 40, 8, 2, 128, 16
    p = Paged(rng, fmt, "f16", [64], H, D, page)
    q, k, v = (rounded(_inputs(rng, tokens, h, D), "f16") for h in (Hq, H, H))
    table = attention.angles(100, attention.frequencies(128, 10000.0)).astype(np.float32)
    positions, slots = np.arange(tokens), p.slots(0, np.arange(tokens))
    slots = slots.copy()
    slots[3], slots[4], slots[5] = -1, p.data[0].shape[0] * page, 2 ** 31 - 1
    positions[7], positions[8] = -1, 100
    before = [[t.clone() for t in (p.data[i], p.scales[i]) if t is not None] for i in range(2)]
    merged = dev(np.concatenate([q, k, v], axis=1), "f16")
    qd, kd, vd = merged[:, :Hq], merged[:, Hq : Hq + H], merged[:, Hq + H :]
    elutq.elutq_kv_write(p.cache, kd, vd, ints(slots), q=qd, q_out=qd, k_out=kd, positions=ints(positions), rope=torch.from_numpy(table).cuda())
    safe = np.clip(positions, 0, 99)
    tq, tk = (rounded(attention.rotate(x, table, safe, False), "f16") for x in (q, k))
    raw_k = attention.rotate(k, table, safe, False)
    for r in (7, 8):
        tq[r], tk[r] = q[r], k[r]
    assert np.array_equal(merged.float().cpu().numpy(), np.concatenate([tq, tk, v], axis=1))
    kept = [r for r in range(tokens) if r not in (3, 4, 5, 7, 8)]
    for i, x in enumerate((raw_k, v)):
        got = p.bytes_at(i, slots[kept])
        if fmt == 0:
            assert np.array_equal(got[0].float().numpy(), rounded(x[kept], "f16"))
        else:
            assert np.array_equal(got[0].numpy(), attention.stored(x[kept], fmt, p.factors[i])[0])
        for pool, old in zip([t for t in (p.data[i], p.scales[i]) if t is not None], before[i]):
            s = torch.from_numpy(slots[kept].astype(np.int64)).cuda()
            old[s // page, :, s % page] = pool[s // page, :, s % page]
            assert torch.equal(pool.view(torch.uint8), old.view(torch.uint8))


@pytest.mark.parametrize("fmt", [1, 2])
def test_write_of_values_that_no_code_holds(fmt):
    rng = np.random.default_rng(3)
    tokens, H, D = 6, 2, 64
    p = Paged(rng, fmt, "bf16", [16], H, D, 16, factors=False)
    k = rounded(rng.standard_normal((tokens, H, D)), "bf16")
    v = k.copy()
    k[0, 0, 3], k[1, 1, 17], k[2, 0, 40], k[3, 1, 5] = np.nan, np.inf, -np.inf, 1e30
    v[0, 0, :], v[1] = 1e-30, -0.0
    elutq.elutq_kv_write(p.cache, dev(k, "bf16"), dev(v, "bf16"), ints(p.slots(0, np.arange(tokens))))
    for i, x in enumerate((k, v)):
        want = attention.stored(x, fmt, None)
        got = p.bytes_at(i, p.slots(0, np.arange(tokens)))
        assert np.array_equal(attention.held(got[0].numpy(), got[1].numpy() if fmt == 2 else None, fmt, None), attention.held(*want, fmt, None), equal_nan=True)


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("dtype,D,H,page,lens", [("f16", 128, 8, 64, [1]), ("bf16", 64, 5, 16, [37, 0, 200, 1]), ("f16", 64, 1, 48, [100] * 3), ("bf16", 128, 2, 32, [0, 700, 31, 33])])
def test_read(fmt, dtype, D, H, page, lens):
    rng = np.random.default_rng(sum(lens) + fmt)
    k, v = ([rng.standard_normal((n, H, D)).astype(np.float32) * 3 for n in lens] for _ in range(2))
    p = Paged(rng, fmt, dtype, lens, H, D, page, k, v)
    first = [min(n, int(rng.integers(0, n // 2 + 1))) for n in lens]
    # two rows in front, three behind
    cu = 2 + np.concatenate([[0], np.cumsum([n - f for n, f in zip(lens, first)])])
    rows = int(cu[-1]) + 3
    wide = torch.full((rows, 2 * H + 1, D), 5.0, dtype=TYPES[dtype], device="cuda")
    ko, vo = wide[:, :H], wide[:, H : 2 * H]
    elutq.elutq_kv_read(p.cache, p.table_d, ints(first), ints(cu), ko, vo)
    for i, o in enumerate((ko, vo)):
        # (code * scale * factor rounded to fp32 first)
        want = np.concatenate([x[f:] for x, f in zip(p.held[i], first)]) if rows > 5 else np.zeros((0, H, D))
        got = o.float().cpu().numpy()
        assert np.array_equal(got[2:-3], rounded(want.astype(np.float32), dtype))
        assert (got[:2] == 5).all() and (got[-3:] == 5).all()
    assert (wide[:, 2 * H :] == 5).all()


@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_read_of_tokens_without_a_page(fmt):
    """Pages outside the cache, positions in front of the table and behind it: zeros."""
    rng = np.random.default_rng(7)
    H, D, page = 2, 64, 16
    k, v = ([rng.standard_normal((64, H, D)).astype(np.float32)] for _ in range(2))
    p = Paged(rng, fmt, "f16", [64], H, D, page, k, v)
    table = p.table_d.clone()
    table[0, 1], table[0, 2] = -1, p.data[0].shape[0]
    rows = 100
    for first in (0, -20, 2 ** 31 - 50):
        ko, vo = (torch.full((rows, H, D), 5.0, dtype=torch.float16, device="cuda") for _ in range(2))
        elutq.elutq_kv_read(p.cache, table, ints([first]), ints([0, rows]), ko, vo)
        for i, o in enumerate((ko, vo)):
            want = np.zeros((rows, H, D), dtype=np.float32)
            for r in range(rows):
                pos = first + r
                if 0 <= pos < 16 or 48 <= pos < 64:
                    want[r] = rounded(p.held[i][0][pos].astype(np.float32), "f16")
            assert np.array_equal(o.float().cpu().numpy(), want)
