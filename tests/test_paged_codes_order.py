"""Orderings in the tiles' kernel over codes that no run shows (no GPU): read off its source, as in test_paged_order.

Two hand-overs by threads' own stores: the copying warp's words about a block (which rows hold something, whether anything follows), and
the converted values, which the tensor cores read as the copy engine writes."""
from __future__ import annotations

import re

import pytest

from tests.test_paged_order import CODE, KERNEL


def function(name):
    text = CODE[CODE.index(name + "("):]
    return text[:text.index("\n}\n")]


COPIES, CONVERT, QUERIES = function("bool pf_copy_codes"), function("bool pf_convert"), function("bool pf_load_queries")


def test_a_blocks_words_are_stored_before_its_first_arrival():
    """Sixteen lanes store the rows' bits, and one whether this is the last; any lane may be the first to arrive.  So the warp's barrier
    stands between the stores and every arrival of the block."""
    loop = COPIES[COPIES.index("for (int kv = 0"):COPIES.index("at.next(a")]
    stores = [m.end() for m in re.finditer(r"\(m\.rows\)\[|m\.last\[buf\] = 0", loop)]
    arrivals = [m.start() for m in re.finditer(r"mbar_arrive|cp\.async\.mbarrier\.arrive", loop)]
    assert len(stores) == 2 and len(arrivals) == 4
    assert "__syncwarp()" in loop[max(stores):min(arrivals)]
    # the softmax's own words of the block come before both of its halves
    assert COPIES.index("(valid)[") < COPIES.index("for (int kv = 0")


def test_a_buffer_is_written_once_it_has_been_read():
    """All four converting warps free a buffer; the words about it are in it as well."""
    loop = COPIES[COPIES.index("for (int kv = 0"):]
    wait = loop.index("pf_wait(&m.empty[buf], (round - 1) & 1)")
    assert wait < loop.index("(m.rows)[") and "if (!ok) break" in loop[wait:loop.index("(m.rows)[")]
    assert "mbar_init(&rw.empty[s], G::kCopyWarps)" in KERNEL and "mbar_init(&rw.full[s], 33)" in KERNEL


def test_the_end_is_stored_before_its_arrival():
    """The last buffer says that nothing follows, once it is free."""
    end = COPIES[COPIES.index("at.next(a"):]
    store = end.index("m.last[buf] = 1")
    assert "pf_wait(&m.empty[buf], (round - 1) & 1)" in end[:store]
    assert "__syncwarp()" in end[store:end.index("mbar_arrive", store)]


def test_converted_values_are_fenced_before_their_arrival():
    """Stores of threads, read by the MMA through the other proxy: every lane fences its own, the warp's barrier follows, then one lane
    arrives for all."""
    loop = CONVERT[CONVERT.index("for (;;)"):]
    last_store = loop.rindex("sts128_at(")
    fence = loop.index("fence_proxy_async_smem()", last_store)
    barrier = loop.index("__syncwarp()", fence)
    arrive = loop.index("mbar_arrive(&ring.full[slot])")
    assert fence < barrier < arrive
    assert barrier < loop.index("mbar_arrive(&m.empty[buf])")
    between = loop[last_store:fence]
    assert "if" not in between  # every lane comes to the fence


def test_a_slot_is_converted_into_once_its_products_are_done():
    loop = CONVERT[CONVERT.index("for (;;)"):]
    assert loop.index("pf_wait(&m.full[buf], bufs & 1)") < loop.index("m.last[buf]")
    assert loop.index("pf_wait(&ring.empty[slot], (round - 1) & 1)") < loop.index("sts128_at(")


@pytest.mark.parametrize("role,buffers", [(COPIES, "m.full"), (QUERIES, "q_full")])
def test_no_tensor_copy_is_in_flight_when_its_warp_ends(role, buffers):
    """Whether or not the waits before it held."""
    tail = role[role.rindex("at.next(a"):]
    assert f"pf_wait({'&' if '.' in buffers else ''}{buffers}" in tail
