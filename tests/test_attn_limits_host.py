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
