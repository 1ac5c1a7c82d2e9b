"""The paged KV cache at the edges of what its calls accept, against plain definitions in 64 bits."""
from __future__ import annotations

import math

import pytest

torch = pytest.importorskip("torch")
from .test_gpu_paged import TINY, TYPE, U, Cache, attention, paged, widened  # noqa: E402,F401

pytestmark = pytest.mark.gpu

FORMS = ["decode", "few", "tiles"]  # vt_paged_decode; vt_paged_prefill by the kernel of single tokens and by the tiles' kernel


def attend(vt, g, c, form, q, scale, window):
    out = torch.full_like(q, 7.0)
    if form == "decode":
        vt.vt_paged_decode(g, c.pool, c.batch(vt, starts=False), q, out, scale, window)
    else:
        vt.vt_paged_prefill(g, c.pool, c.batch(vt), q, out, scale, window)
    return out


@pytest.mark.parametrize("form", FORMS)
def test_a_page_id_of_any_bad_value_is_flagged(vtlib, paged, form):
    """No id outside the pool is taken for a position that is not attended to."""
    vt = vtlib
    c = Cache(vt, [100, 60], [1, 1] if form != "tiles" else [40, 50], "f16", 1, 64, 16)
    if form == "tiles":
        c = widened(c)
    q = c.rows(2)
    want = c.tables[0, 2].item()
    for bad in (-2, -3, -17, c.k.shape[0] + 1, -2 ** 31 + 1):
        c.tables[0, 2] = bad
        attend(vt, paged, c, form, q, 0.125, 0)
        assert vt.vt_paged_status(paged, clear=True) == vt.VT_DEV_BAD_PAGE, bad
    c.tables[0, 2] = want
    attend(vt, paged, c, form, q, 0.125, 0)
    assert vt.vt_paged_status(paged) == 0
