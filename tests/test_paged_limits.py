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


def test_rows_of_several_slots_are_reserved_together_or_not_at_all():
    t = PageTable(5, 8, 3, 4)
    a, b = t.admit(), t.admit()
    assert t.reserve_all({a: 9, b: 3}) == [a, b]
    t.lens[a], t.lens[b] = 9, 3
    free, pages = list(t.free), [list(p) for p in t.pages]
    for rows, error in (({a: 8, b: 14}, RuntimeError),  # a page and two of the two that are free
                        ({a: 8, b: 30}, RuntimeError),  # more than a slot may have
                        ({a: 8, 2: 1}, ValueError),     # an idle slot
                        ({a: 8, b: -1}, ValueError)):
        with pytest.raises(error):
            t.reserve_all(rows)
        assert (t.free, t.pages) == (free, pages)
    assert t.reserve_all({a: 7, b: 5}) == [] and t.reserve_all({a: 8, b: 5}) == [a]
