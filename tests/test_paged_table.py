"""The host's page table of the paged cache (no GPU): pages are dealt out once, come back, and a refusal
changes nothing."""
from __future__ import annotations

import random

import pytest

from paper_2607_07046_gb300.paged import PageTable


def test_pages_are_dealt_out_once_and_come_back():
    rng = random.Random(3)
    t = PageTable(50, 16, 6, 12)
    held = {}
    for _ in range(2000):
        if held and rng.random() < 0.15:
            slot = rng.choice(list(held))
            t.release(slot)
            del held[slot]
        elif len(held) < 6 and rng.random() < 0.3:
            slot = t.admit()
            assert slot not in held and t.lens[slot] == 0
            held[slot] = 0
        elif held:
            slot, n = rng.choice(list(held)), rng.choice([1, 1, 1, 15, 16, 17, 60])
            free, pages, lens = list(t.free), [list(p) for p in t.pages], list(t.lens)
            try:
                grew = t.reserve(slot, n)
            except RuntimeError:
                assert (t.free, t.pages, t.lens) == (free, pages, lens)
                continue
            assert grew == (len(t.pages[slot]) > len(pages[slot]))
            t.lens[slot] += n
            held[slot] += n
        assert sorted(t.free + [p for s in t.pages for p in s]) == list(range(50))
        for slot, n in held.items():
            assert len(t.pages[slot]) == -(-n // 16) and t.lens[slot] == n


def test_refusals():
    t = PageTable(4, 8, 2, 3)
    with pytest.raises(ValueError):
        t.reserve(0, 1)
    a, b = t.admit(), t.admit()
    with pytest.raises(RuntimeError):
        t.admit()
    with pytest.raises(RuntimeError):
        t.reserve(a, 25)       # four pages of three
    assert t.reserve(a, 24) and not t.reserve(a, 24)
    with pytest.raises(RuntimeError):
        t.reserve(b, 9)        # two pages, one is free
    assert t.reserve(b, 8) and not t.free
