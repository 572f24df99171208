"""Entries of the paged cache and of attention: more that they refuse before any launch (no GPU needed)."""

import ctypes

import pytest

import paper_2510_19482_b200 as elutq


def test_a_table_of_angles_on_another_stream():
    """Memory of torch's current stream may still be in use there."""
    before = elutq.elutq_launch_count()
    with pytest.raises(elutq.ElutqError) as e:
        elutq.elutq_rope_table(10, 64, stream=1 << 20)
    assert e.value.status == -1 and "stream" in str(e.value)
    assert elutq.elutq_launch_count() == before


def test_limits_of_the_test_entry():
    before = elutq.elutq_launch_count()
    for limit in (0, elutq.ATTN_TEST_LOADS):
        assert elutq.lib().elutq_attn_test_wait_expiry(64, 512, 65536, 256, 131072, 256, 262144, 512, 0, 8, 16, 2, 10, 20, 30, 4, 2, 128, 0.1, 0, limit, None) == -1
    assert elutq.elutq_launch_count() == before


def refused(status, name, *args):
    """Called with addresses that no kernel may see: refused before any launch."""
    before = elutq.elutq_launch_count()
    assert getattr(elutq.lib(), name)(*args, None) == status, (name, args)
    assert elutq.elutq_launch_count() == before


MB = 1 << 20
CACHE = elutq.KvCacheDesc(k=1 << 30, v=1 << 31, format=0, type=0, n_pages=10, heads=2, page_size=16, head_dim=128)


@pytest.mark.parametrize("kw", [dict(ldqo=520), dict(q_out=MB + 256), dict(q_out=MB + 1024), dict(q_out=MB - 16), dict(q_out=MB + 3 * 1024), dict(q_out=2 * MB), dict(q_out=2 * MB + 512 - 16),
                                dict(q_out=3 * MB - 1024, ldqo=512), dict(k_out=2 * MB, ldko=264), dict(k_out=2 * MB + 256, ldko=256), dict(k_out=3 * MB, ldko=256), dict(k_out=MB + 512, ldko=512),
                                dict(k_out=MB, ldko=512, q_out=MB), dict(q=MB, ldq=1024, q_out=MB + 1024 - 16, ldqo=1024), dict(k_out=4 * MB, ldko=256, q_out=4 * MB)])
def test_a_write_whose_results_meet_its_inputs(kw):
    """In place with another distance between tokens, shifted by a head, by a token, by 16 bytes, over the keys, the values, or one another."""
    a = dict(q=MB, ldq=512, q_out=MB, ldqo=512, n=4, k=2 * MB, ldk=256, k_out=0, ldko=0, v=3 * MB, ldv=256, tokens=4) | kw
    refused(-1, "elutq_kv_write", ctypes.byref(CACHE), a["q"], a["ldq"], a["q_out"], a["ldqo"], a["n"], a["k"], a["ldk"], a["k_out"], a["ldko"], a["v"], a["ldv"], a["tokens"], 16, 0, 0, 0, 0, 0)


@pytest.mark.parametrize("v,ldv", [(MB, 256), (MB + 256, 256), (MB - 16, 256), (MB, 512), (MB + 9 * 512, 512)])
def test_a_read_whose_results_meet(v, ldv):
    refused(-1, "elutq_kv_read", ctypes.byref(CACHE), 64, 5, 5, 0, 16, 2, 10, MB, 256, v, ldv)


@pytest.mark.parametrize("out,ldo", [(MB, 512), (MB, 520), (MB + 256, 512), (MB + 1024, 512), (MB - 1024, 512), (MB + 5 * 1024 + 1024 - 16, 512), (MB - 5 * 1024, 512)])
def test_a_decoding_step_whose_result_meets_its_queries(out, ldo):
    refused(-1, "elutq_attn_decode", ctypes.byref(CACHE), MB, 512, out, ldo, 64, 5, 5, 16, 3, 2, 4, 0.1, 1 << 24, 1 << 30)


@pytest.mark.parametrize("entry,more", [("elutq_attn_prefill", ()), ("elutq_attn_test_wait_expiry", (5,))])
@pytest.mark.parametrize("out,ldo", [(MB, 512), (MB + 256, 512), (MB - 19 * 1024, 512), (2 * MB + 512 * 29, 512), (2 * MB + 256, 512), (3 * MB + 16, 512), (3 * MB - 1024 + 16, 512)])
def test_a_prompt_whose_result_meets_its_inputs(entry, more, out, ldo):
    refused(-1, entry, MB, 512, 2 * MB, 256, 3 * MB, 256, out, ldo, 0, 8, 16, 2, 10, 20, 30, 4, 2, 128, 0.1, 0, *more)
