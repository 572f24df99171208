"""Entries of the paged cache and of attention: what they refuse, on the host and before any launch (no GPU needed)."""

import ctypes

import pytest

import paper_2510_19482_b200 as elutq


def cache(**kw):
    base = dict(k=1024, v=2048, k_scales=0, v_scales=0, k_factor=0, v_factor=0, format=0, type=0, n_pages=10, heads=2, page_size=16, head_dim=128)
    return elutq.KvCacheDesc(**(base | kw))


BAD_CACHES = [(-1, dict(k=0)), (-1, dict(v=0)), (-1, dict(n_pages=0)), (-1, dict(heads=0)), (-1, dict(page_size=0)), (-1, dict(format=3)), (-1, dict(format=-1)), (-1, dict(type=2)),
              (-1, dict(format=2)), (-1, dict(format=2, k_scales=64)), (-5, dict(head_dim=96)), (-5, dict(head_dim=256)), (-2, dict(page_size=24)),
              (-2, dict(n_pages=1 << 27, page_size=16)), (-3, dict(k=1040)), (-3, dict(v=2056)), (-3, dict(format=2, k_scales=8, v_scales=64)), (-3, dict(format=1, k_factor=2))]


def write(c, q=4096, ldq=512, q_out=8192, ldqo=512, n=4, k=64, ldk=256, k_out=0, ldko=0, v=128, ldv=256, tokens=3, slots=16, positions=32, rope=256, n_pos=100, rot=128, flags=0):
    return elutq.lib().elutq_kv_write(None if c is None else ctypes.byref(c), q, ldq, q_out, ldqo, n, k, ldk, k_out, ldko, v, ldv, tokens, slots, positions, rope, n_pos, rot, flags, None)


def read(c, table=64, ld=5, pages=5, first=0, cu=16, B=2, rows=10, k=64, ldk=256, v=128, ldv=256):
    return elutq.lib().elutq_kv_read(None if c is None else ctypes.byref(c), table, ld, pages, first, cu, B, rows, k, ldk, v, ldv, None)


def decode(c, q=64, ldq=512, out=128, ldo=512, table=16, ld=5, pages=5, lens=8, B=2, new=1, n=4, scale=0.1, ws=1024, size=1 << 30):
    return elutq.lib().elutq_attn_decode(None if c is None else ctypes.byref(c), q, ldq, out, ldo, table, ld, pages, lens, B, new, n, scale, ws, size, None)


@pytest.mark.parametrize("status,kw", BAD_CACHES)
def test_caches_that_are_refused(status, kw):
    before = elutq.elutq_launch_count()
    c = cache(**kw)
    assert write(c) == read(c) == decode(c) == status
    assert elutq.elutq_launch_count() == before


def test_arguments_of_a_write():
    before, c = elutq.elutq_launch_count(), cache()
    assert write(None) == -1
    for kw in (dict(k=0), dict(v=0), dict(slots=0), dict(tokens=0), dict(tokens=-1), dict(n=-1), dict(q=0), dict(q_out=0), dict(flags=2), dict(positions=0), dict(n_pos=0), dict(rot=0)):
        assert write(c, **kw) == -1, kw
    for kw in (dict(rot=144), dict(rot=20), dict(ldq=511), dict(ldk=255), dict(ldv=128), dict(ldqo=256), dict(k_out=64, ldko=128), dict(tokens=2 ** 31 - 1, n=1 << 20, ldq=1 << 30, ldqo=1 << 30)):
        assert write(c, **kw) == -2, kw
    for kw in (dict(q=4104), dict(ldq=516), dict(k=72), dict(v=130), dict(ldv=260), dict(q_out=8200), dict(k_out=72, ldko=256), dict(slots=18), dict(positions=33), dict(rope=264)):
        assert write(c, **kw) == -3, kw
    assert elutq.elutq_launch_count() == before


def test_arguments_of_a_read():
    before, c = elutq.elutq_launch_count(), cache()
    for kw in (dict(table=0), dict(cu=0), dict(k=0), dict(v=0), dict(pages=0), dict(B=0), dict(rows=0)):
        assert read(c, **kw) == -1, kw
    assert read(None) == -1
    assert read(c, ld=4) == read(c, ldk=255) == read(c, ldv=8) == -2
    for kw in (dict(table=66), dict(cu=17), dict(first=2), dict(k=72), dict(ldv=260)):
        assert read(c, **kw) == -3, kw
    assert elutq.elutq_launch_count() == before


def test_arguments_of_a_decoding_step():
    before, c = elutq.elutq_launch_count(), cache()
    for kw in (dict(q=0), dict(out=0), dict(table=0), dict(lens=0), dict(pages=0), dict(B=0), dict(new=0), dict(n=0), dict(scale=0.0), dict(scale=-1.0),
               dict(scale=float("nan")), dict(scale=float("inf"))):
        assert decode(c, **kw) == -1, kw
    assert decode(None) == -1
    for kw in (dict(n=5, ldq=1024, ldo=1024), dict(ld=4), dict(ldq=511), dict(ldo=256), dict(new=1 << 16)):
        assert decode(c, **kw) == -2, kw
    for kw in (dict(q=72), dict(out=136), dict(ldq=516), dict(table=18), dict(lens=9), dict(ws=1032)):
        assert decode(c, **kw) == -3, kw
    out, ask = ctypes.c_size_t(7), elutq.lib().elutq_attn_decode_workspace_bytes
    assert ask(ctypes.byref(c), 5000, 2, 1, 4, ctypes.byref(out)) == 0 and out.value > 0
    assert decode(c, pages=5000, ld=5000, size=out.value - 1) == -4 and decode(c, pages=5000, ld=5000, ws=0) == -1
    assert ask(ctypes.byref(c), 5, 2, 1, 4, ctypes.byref(out)) == 0 and out.value == 0            # a short table: none needed
    assert ask(ctypes.byref(c), 5, 2, 1, 5, ctypes.byref(out)) == -2 and ask(ctypes.byref(c), 5, 2, 1 << 16, 4, ctypes.byref(out)) == -2
    assert ask(None, 5, 2, 1, 4, ctypes.byref(out)) == ask(ctypes.byref(c), 0, 2, 1, 4, ctypes.byref(out)) == ask(ctypes.byref(c), 5, 2, 1, 4, None) == -1
    assert ask(ctypes.byref(cache(head_dim=96)), 5, 2, 1, 4, ctypes.byref(out)) == -5
    assert elutq.elutq_launch_count() == before


def test_sizes_of_a_cache():
    assert elutq.elutq_kv_bytes(0, 3, 2, 16, 128) == (3 * 2 * 16 * 256, 0)
    assert elutq.elutq_kv_bytes(1, 3, 2, 48, 64) == (3 * 2 * 48 * 64, 0)
    assert elutq.elutq_kv_bytes(2, 3, 2, 16, 128) == (3 * 2 * 16 * 64, 3 * 2 * 16 * 8)
    # sizes past 32 bits
    assert elutq.elutq_kv_bytes(0, 1 << 20, 8, 64, 128) == ((1 << 29) * 256, 0)
    L, a, b = elutq.lib(), ctypes.c_size_t(0), ctypes.c_size_t(0)
    assert L.elutq_kv_bytes(3, 3, 2, 16, 128, ctypes.byref(a), ctypes.byref(b)) == L.elutq_kv_bytes(0, 0, 2, 16, 128, ctypes.byref(a), ctypes.byref(b)) == -1
    assert L.elutq_kv_bytes(0, 3, 2, 17, 128, ctypes.byref(a), ctypes.byref(b)) == -2 and L.elutq_kv_bytes(0, 3, 2, 16, 80, ctypes.byref(a), ctypes.byref(b)) == -5


def test_arguments_of_a_table_of_angles():
    L = elutq.lib()
    good = dict(table=64, n=10, rot=64, theta=1e4, scaling=0, factor=1.0, low=1.0, high=4.0, original=8192.0, magnitude=1.0)

    def call(**kw):
        return L.elutq_rope_table(*(good | kw).values(), None)

    before = elutq.elutq_launch_count()
    for kw in (dict(table=0), dict(n=0), dict(rot=0), dict(theta=1.0), dict(theta=float("inf")), dict(scaling=3), dict(scaling=1, factor=0.5), dict(scaling=2, high=1.0),
               dict(scaling=2, original=0.0), dict(magnitude=0.0), dict(magnitude=float("nan"))):
        assert call(**kw) == -1, kw
    assert call(rot=24) == -2 and call(table=72) == -3
    assert elutq.elutq_launch_count() == before


def prefill(entry="elutq_attn_prefill", more=(), **kw):
    good = dict(q=64, ldq=512, k=128, ldk=256, v=256, ldv=256, out=512, ldo=512, type=0, cu_q=8, cu_k=16, B=2, max_q=10, total_q=20, total_k=30, n=4, heads=2, D=128, scale=0.1, flags=0)
    return getattr(elutq.lib(), entry)(*(good | kw).values(), *more, None)


@pytest.mark.parametrize("entry,more", [("elutq_attn_prefill", ()), ("elutq_attn_test_wait_expiry", (5,))])
def test_arguments_of_a_prompt(entry, more):
    before = elutq.elutq_launch_count()
    for kw in (dict(q=0), dict(k=0), dict(v=0), dict(out=0), dict(cu_q=0), dict(cu_k=0), dict(B=0), dict(max_q=0), dict(total_q=0), dict(total_k=0), dict(n=0), dict(heads=0), dict(type=2),
               dict(flags=2), dict(scale=0.0), dict(scale=float("nan"))):
        assert prefill(entry, more, **kw) == -1, kw
    assert prefill(entry, more, D=96) == -5
    for kw in (dict(n=5, ldq=1024, ldo=1024), dict(ldq=504), dict(ldk=248), dict(ldv=128), dict(ldo=504), dict(total_q=1 << 30), dict(ldk=1 << 39), dict(B=1 << 30)):
        assert prefill(entry, more, **kw) == -2, kw
    for kw in (dict(q=72), dict(ldq=516), dict(k=130), dict(ldk=257), dict(v=264), dict(out=520), dict(cu_q=9), dict(cu_k=18)):
        assert prefill(entry, more, **kw) == -3, kw
    assert prefill("elutq_attn_test_wait_expiry", (0,)) == -1
    assert elutq.elutq_launch_count() == before


def test_results_in_place_of_inputs():
    """Queries are read again after the first results are written."""
    before = elutq.elutq_launch_count()
    assert decode(cache(), q=128) == -1
    assert prefill(out=64) == prefill(out=128) == prefill(out=256) == -1
    assert elutq.elutq_launch_count() == before
