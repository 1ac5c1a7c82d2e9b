"""Pages for several sequences: which pages of a pool each sequence has, kept on the host, and the tables and
lengths that the paged calls read, kept on the device.

The pools hold one layer's K and V each; tables and lengths are the same for every layer.  A step is

    rows = {slot: new rows, ...}
    batch, starts = cache.step(rows)               # pages for the new rows; slots without rows take no part
    for layer: cache.append(layer, batch, q, k, v, q_out), then cache.attend(layer, batch, q_out, out)
    cache.advance(rows)                            # the new rows are held now

append and attend make the calls that suit the cache (vt_paged_append, _append_qk, _append_mx; vt_paged_decode,
_prefill, _decode_mx, _prefill_mx); a program may make them itself.
"""
from __future__ import annotations

from typing import Dict, List, Optional, Sequence

import torch

from . import vt


class PageTable:
    """The host's side: `slots` sequences of at most `pages_per_seq` pages out of `n_pages`, and of at most `max_len`
    positions (None: as many as the pages have)."""

    def __init__(self, n_pages: int, page_size: int, slots: int, pages_per_seq: int, max_len: Optional[int] = None):
        self.page_size, self.pages_per_seq = page_size, pages_per_seq
        self.max_len = pages_per_seq * page_size if max_len is None else max_len
        self.free: List[int] = list(range(n_pages - 1, -1, -1))
        self.pages: List[List[int]] = [[] for _ in range(slots)]
        self.lens: List[int] = [-1] * slots  # -1: an idle slot

    def admit(self) -> int:
        """A slot for a new sequence, which holds nothing yet."""
        for slot, n in enumerate(self.lens):
            if n < 0:
                self.lens[slot] = 0
                return slot
        raise RuntimeError("every slot of the cache is taken")

    def release(self, slot: int) -> None:
        self.free.extend(reversed(self.pages[slot]))
        self.pages[slot], self.lens[slot] = [], -1

    def reserve(self, slot: int, rows: int) -> bool:
        """Pages for `rows` more positions; True when the slot got new ones.  Nothing changes on an error."""
        return bool(self.reserve_all({slot: rows}))

    def reserve_all(self, rows: Dict[int, int]) -> List[int]:
        """Pages for the new rows of several slots; those that got new ones.  Nothing changes on an error."""
        more = {slot: self._missing(slot, n) for slot, n in rows.items()}
        if sum(more.values()) > len(self.free):
            raise RuntimeError(f"{sum(more.values())} pages are needed and {len(self.free)} are free")
        for slot, n in more.items():
            for _ in range(n):
                self.pages[slot].append(self.free.pop())
        return [slot for slot, n in more.items() if n > 0]

    def _missing(self, slot: int, rows: int) -> int:
        if self.lens[slot] < 0:
            raise ValueError(f"slot {slot} is idle")
        if rows < 0:
            raise ValueError(f"{rows} rows for slot {slot}")
        if self.lens[slot] + rows > self.max_len:
            raise RuntimeError(f"slot {slot} would hold {self.lens[slot] + rows} positions of at most {self.max_len}")
        want = -(-(self.lens[slot] + rows) // self.page_size)
        if want > self.pages_per_seq:
            raise RuntimeError(f"slot {slot} would need {want} pages of at most {self.pages_per_seq}")
        return max(0, want - len(self.pages[slot]))


class PagedCache:
    """`n_layers` pools [pages, KV heads, positions in a page, head dim] and one PageTable.

    code: None for values of `dtype`, or "e4m3" or "int8" for 8-bit codes with a scale for each 32 dimensions (pages of 8
    positions or more), about half the memory.  rotary_dim: the first dimensions of a head that are rotated (None: all)."""

    def __init__(self, n_layers: int, n_kv_heads: int, d_head: int, page_size: int, n_pages: int, slots: int, max_len: int,
                 dtype=torch.float16, theta: float = 1e4, code: Optional[str] = None, rotary_dim: Optional[int] = None):
        if code not in (None, "e4m3", "int8"):
            raise ValueError(f"code {code!r}: expected None, 'e4m3' or 'int8'")
        if code is not None and page_size < 8:
            raise ValueError(f"codes need pages of 8 positions or more, got {page_size}")
        if rotary_dim is not None and (rotary_dim % 16 or not 0 <= rotary_dim <= d_head):
            raise ValueError(f"rotary_dim {rotary_dim}: expected a multiple of 16 in [0, {d_head}]")
        self.code = code
        self.table = PageTable(n_pages, page_size, slots, -(-max_len // page_size), max_len)
        shape = (n_pages, n_kv_heads, page_size, d_head)
        self.pools = [self._pool(shape, dtype) for _ in range(n_layers)]
        self.tables = torch.full((slots, self.table.pages_per_seq), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.full((slots,), -1, dtype=torch.int32, device="cuda")
        self.starts = torch.zeros(slots + 1, dtype=torch.int32, device="cuda")
        rotary_dim = d_head if rotary_dim is None else rotary_dim
        self.rope = torch.empty(max_len, rotary_dim // 2, 2, device="cuda") if rotary_dim else None
        if rotary_dim in (64, 128):
            vt.vt_rope_table(self.rope, theta)
        elif rotary_dim:
            at = torch.arange(max_len, device="cuda", dtype=torch.float64)[:, None] * theta ** (
                torch.arange(rotary_dim // 2, device="cuda", dtype=torch.float64) * (-2.0 / rotary_dim))
            self.rope.copy_(torch.stack((at.cos(), at.sin()), -1))
        # vt_paged_append's own: all of a head, pairs of halves, no norms, values of `dtype`
        self._form = None if code is None and rotary_dim == d_head else vt.make_qk_form(self.rope)
        self.paged = vt.vt_paged_create()
        self._each = vt.make_paged_batch(self.tables, self.lens)
        self._ragged = vt.make_paged_batch(self.tables, self.lens, self.starts)

    def _pool(self, shape, dtype):
        if self.code is None:
            return vt.make_paged_pool(torch.zeros(shape, dtype=dtype, device="cuda"), torch.zeros(shape, dtype=dtype, device="cuda"))
        kind = torch.float8_e4m3fn if self.code == "e4m3" else torch.int8
        k, v = (torch.zeros(shape, dtype=torch.uint8, device="cuda").view(kind) for _ in range(2))
        k_scale, v_scale = (torch.zeros(*shape[:3], shape[3] // 32, dtype=torch.uint8, device="cuda") for _ in range(2))
        return vt.make_paged_mx_pool(k, v, k_scale, v_scale, dtype)

    def append(self, layer: int, batch, q, k, v, q_out, form=None, stream=None) -> None:
        """The new rows' queries rotated into q_out, keys rotated and values stored.  form: vt.make_qk_form(cache.rope, ...) for
        norms of queries and keys or pairs of neighbours."""
        form = self._form if form is None else form
        if self.code is not None:
            vt.vt_paged_append_mx(self.paged, self.pools[layer], batch, q, k, v, form, q_out, stream)
        elif form is not None:
            vt.vt_paged_append_qk(self.paged, self.pools[layer], batch, q, k, v, form, q_out, stream)
        else:
            vt.vt_paged_append(self.paged, self.pools[layer], batch, q, k, v, self.rope, q_out, stream)

    def attend(self, layer: int, batch, q, out, scale: Optional[float] = None, window: int = 0, stream=None) -> None:
        """Attention of the step's rows, which append has stored."""
        if batch.starts is None:
            call = vt.vt_paged_decode if self.code is None else vt.vt_paged_decode_mx
        else:
            call = vt.vt_paged_prefill if self.code is None else vt.vt_paged_prefill_mx
        call(self.paged, self.pools[layer], batch, q, out, scale, window, stream)

    def admit(self) -> int:
        return self.table.admit()

    def release(self, slot: int) -> None:
        self.table.release(slot)
        self.lens[slot] = -1
        self.tables[slot] = -1  # its pages are others' soon

    def step(self, rows: Dict[int, int], one_each: Optional[bool] = None):
        """(batch, first row of every slot) for these new rows.  one_each: one row for every slot, idle or not, as
        vt_paged_decode takes them (row b belongs to slot b); by default where every sequence gets one row.  With it a
        slot that is not in `rows` is idle for this step, and every count has to be 1."""
        if one_each is None:
            one_each = set(rows.values()) == {1} and len(rows) == sum(n >= 0 for n in self.table.lens)
        elif one_each and any(n != 1 for n in rows.values()):
            raise ValueError(f"one_each takes one row of each slot, got {rows}")
        for slot in self.table.reserve_all(rows):
            pages = self.table.pages[slot]
            self.tables[slot, :len(pages)] = torch.tensor(pages, dtype=torch.int32, device="cuda")
        lens = [n if not one_each or slot in rows else -1 for slot, n in enumerate(self.table.lens)]
        self.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        starts = [0]
        for slot in range(len(self.table.lens)):
            starts.append(starts[-1] + (1 if one_each else rows.get(slot, 0)))
        if one_each:
            return self._each, starts
        self.starts.copy_(torch.tensor(starts, dtype=torch.int32))
        return self._ragged, starts

    def advance(self, rows: Dict[int, int]) -> None:
        for slot, n in rows.items():
            self.table.lens[slot] += n

    def close(self) -> None:
        vt.vt_paged_destroy(self.paged)
        self.paged = 0
