"""Entries of the paged cache and of attention: more that they refuse before any launch (no GPU needed)."""

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
