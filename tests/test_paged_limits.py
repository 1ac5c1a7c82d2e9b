"""What the host's page table of the paged cache refuses (no GPU)."""
from __future__ import annotations

import pytest

from paper_2607_07046_gb300.paged import PageTable


@pytest.mark.parametrize("max_len,page", [(100, 64), (401, 16), (64, 64), (1, 16)])
def test_no_position_past_the_longest_length(max_len, page):
    """The last page may reach past max_len; the rotation table and so the calls do not."""
    t = PageTable(40, page, 1, -(-max_len // page), max_len)
    slot = t.admit()
    with pytest.raises(RuntimeError):
        t.reserve(slot, max_len + 1)
    assert t.pages[slot] == [] and len(t.free) == 40
    assert t.reserve(slot, max_len)
    t.lens[slot] = max_len
    with pytest.raises(RuntimeError):
        t.reserve(slot, 1)
    assert not t.reserve(slot, 0)
