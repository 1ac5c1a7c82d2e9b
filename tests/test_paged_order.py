"""Orderings in the tiles' kernel of the paged prefill that no run shows (no GPU): read off its source.

A missing one is a race whose outcome hardware decides, so the source itself is what can be checked: the fence
or barrier stands between the two accesses that it orders."""
from __future__ import annotations

import re
from pathlib import Path

SOURCE = (Path(__file__).resolve().parents[1] / "paper_2607_07046_gb300" / "csrc" / "paged_prefill.cu").read_text()
CODE = re.sub(r"//[^\n]*", "", SOURCE)
KERNEL = CODE[CODE.index("k_paged_prefill(const __grid_constant__"):CODE.index("struct PfJoin")]


def test_plain_stores_over_the_ring_are_fenced_before_tensor_copies():
    """The blocks of each sequence lie in the memory of Q and the ring: written and read as threads do, then
    written by the copy engine.  Every thread needs a proxy fence before the barrier that lets the copies begin."""
    assert "reinterpret_cast<int64_t*>(smem)" in KERNEL and "uint8_t* Qs = smem" in KERNEL
    between = KERNEL[KERNEL.rindex("tot["):KERNEL.index("const int w = warp - 8")]
    fence = between.rindex("fence_proxy_async_smem()")
    assert "__syncthreads()" in between[fence:]


def test_a_clean_blocks_mask_is_stored_before_its_arrival():
    """Lanes 0 to 3 store the validity words and one elected lane arrives: votes and shuffles order no memory."""
    clean = KERNEL[KERNEL.index("= 0xffffffffu"):KERNEL.index("tma_load_4d")]
    store, arrive = 0, clean.index("mbar_arrive_expect_tx(&full")
    before_branch = clean[store:clean.index("else {")]
    assert "__syncwarp()" in before_branch or "__syncwarp()" in clean[clean.index("if (clean)"):arrive]


def test_a_bounded_wait_of_one_lane_is_passed_on_in_order():
    """One lane acquires the phase; the others read what it announces only behind a barrier of the warp."""
    body = CODE[CODE.index("bool pf_wait(uint64_t* bar"):]
    body = body[:body.index("\n}\n")]
    assert "__syncwarp()" in body[body.index("mbar_wait(bar, parity)"):]
