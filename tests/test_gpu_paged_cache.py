"""PagedCache on the GPU: what a step hands to the paged calls."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture()
def make(vtlib):
    from paper_2607_07046_gb300.paged import PagedCache
    made = []

    def new(*args, **kw):
        made.append(PagedCache(1, 1, 64, *args, **kw))
        return made[-1]

    yield new
    for c in made:
        c.close()


def append(vt, cache, batch, n, value):
    """n rows of this value; (their queries as rotated, the status)."""
    x = torch.full((n, 1, 64), float(value), dtype=torch.float16, device="cuda")
    q = torch.full_like(x, 7.0)
    vt.vt_paged_append(cache.paged, cache.pools[0], batch, x, x, x, cache.rope, q)
    return q, vt.vt_paged_status(cache.paged, clear=True)


def held(cache, slot):
    """The values of a slot's positions, one number each."""
    page, n = cache.table.page_size, cache.table.lens[slot]
    v = cache.pools[0].tensors[1]
    return [float(v[cache.table.pages[slot][p // page], 0, p % page, 0]) for p in range(n)]


@pytest.mark.parametrize("max_len,page", [(100, 64), (401, 16)])
def test_every_position_that_a_step_accepts_is_stored(vtlib, make, max_len, page):
    cache = make(page, 40, 2, max_len)
    slot = cache.admit()
    with pytest.raises(RuntimeError):
        cache.step({slot: max_len + 1})
    batch, _ = cache.step({slot: max_len - 1})
    q, status = append(vtlib, cache, batch, max_len - 1, 1.0)
    assert status == 0 and q.any(-1).all()
    cache.advance({slot: max_len - 1})
    batch, _ = cache.step({slot: 1})
    _, status = append(vtlib, cache, batch, 2 if batch.starts is None else 1, 2.0)
    assert status == 0
    cache.advance({slot: 1})
    assert held(cache, slot) == [1.0] * (max_len - 1) + [2.0]
    with pytest.raises(RuntimeError):
        cache.step({slot: 1})
