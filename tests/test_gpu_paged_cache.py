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


def test_one_each_takes_one_row_of_each_slot(make):
    cache = make(16, 40, 3, 100)
    a, b = cache.admit(), cache.admit()
    for rows in ({a: 3}, {a: 1, b: 2}, {a: 0}):
        with pytest.raises(ValueError):
            cache.step(rows, one_each=True)
    assert cache.table.pages == [[], [], []] and len(cache.table.free) == 40


def test_one_each_leaves_the_other_slots_alone(vtlib, make):
    """A live slot that gets no row is idle for the step: nothing is stored for it, not even past its end."""
    vt = vtlib
    cache = make(16, 40, 3, 100)
    a, b = cache.admit(), cache.admit()
    batch, _ = cache.step({a: 16, b: 5})  # a's page is full
    append(vt, cache, batch, 21, 1.0)
    cache.advance({a: 16, b: 5})
    before = cache.pools[0].tensors[1].clone()
    batch, starts = cache.step({b: 1}, one_each=True)
    assert batch.starts is None and starts == [0, 1, 2, 3]
    q, status = append(vt, cache, batch, 3, 2.0)
    assert status == 0 and q[b].any() and not q[a].any() and not q[2].any()
    out = torch.full_like(q, 7.0)
    vt.vt_paged_decode(cache.paged, cache.pools[0], batch, q, out)
    assert vt.vt_paged_status(cache.paged) == 0
    assert out[b].any() and not out[a].any() and not out[2].any()
    cache.advance({b: 1})
    assert held(cache, a) == [1.0] * 16 and held(cache, b) == [1.0] * 5 + [2.0]
    v = cache.pools[0].tensors[1]
    before[cache.table.pages[b][0], 0, 5] = 2.0
    assert torch.equal(v, before)
    batch, _ = cache.step({a: 1, b: 1})  # both take part again
    _, status = append(vt, cache, batch, 3, 3.0)
    cache.advance({a: 1, b: 1})
    assert status == 0 and held(cache, a)[-1] == 3.0 and held(cache, b)[-1] == 3.0


def test_a_step_that_is_refused_changes_nothing(make):
    cache = make(8, 5, 3, 40)
    a, b = cache.admit(), cache.admit()
    cache.step({a: 9, b: 3})
    cache.advance({a: 9, b: 3})
    free, pages, tables = list(cache.table.free), [list(p) for p in cache.table.pages], cache.tables.clone()
    for rows in ({a: 8, b: 14}, {a: 8, b: 60}, {a: 8, 2: 1}):
        with pytest.raises((ValueError, RuntimeError)):
            cache.step(rows)
        assert (cache.table.free, cache.table.pages) == (free, pages) and torch.equal(cache.tables, tables)


def test_a_released_slots_pages_leave_its_table(vtlib, make):
    """Its next sequence has no entry for pages that others hold by now: a position that nothing was reserved for is
    reported, not stored in their pages."""
    vt = vtlib
    cache = make(16, 6, 2, 100)
    a = cache.admit()
    cache.step({a: 80})
    cache.advance({a: 80})
    cache.release(a)
    assert (cache.tables == -1).all()
    a, b = cache.admit(), cache.admit()
    batch, _ = cache.step({a: 16, b: 64})
    append(vt, cache, batch, 80, 1.0)
    cache.advance({a: 16, b: 64})
    cache.lens[a] = 16  # a captured step that is replayed without a step of the cache
    batch = vt.make_paged_batch(cache.tables, cache.lens)
    cache.lens[b] = -1
    _, status = append(vt, cache, batch, 2, 2.0)
    assert status == vt.VT_DEV_BAD_PAGE
    assert held(cache, a) == [1.0] * 16 and held(cache, b) == [1.0] * 64
