"""PagedCache and the serving example over pools in 8 bits, and with norms and other rotations: the calls together, as a
program makes them."""
from __future__ import annotations

import math

import pytest

torch = pytest.importorskip("torch")
from tests import mx_reference as mx  # noqa: E402
from tests.test_gpu_paged import U  # noqa: E402
from tests.test_gpu_paged_qk import formed  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("code,rotary_dim,neighbours,normed", [
    (None, None, False, False), (None, 32, True, True), ("e4m3", None, False, True), ("int8", 16, False, False), ("int8", 0, False, True)])
def test_steps_of_a_cache(vtlib, code, rotary_dim, neighbours, normed):
    """Two layers, prompts, single tokens, a slot released and taken again: what the pools hold afterwards, and every row's
    output over it, from their definitions."""
    from paper_2607_07046_gb300.paged import PagedCache
    vt, K, H, d, dtype = vtlib, 2, 6, 64, "bf16"
    cache = PagedCache(2, K, d, 16, 24, 3, 130, dtype=torch.bfloat16, code=code, rotary_dim=rotary_dim)
    g = torch.Generator(device="cuda").manual_seed(2)
    rotary = d if rotary_dim is None else rotary_dim
    gains = [[(1 + 0.1 * torch.randn(d, generator=g, device="cuda")).bfloat16() if normed else None for _ in range(2)] for _ in range(2)]
    forms = [vt.make_qk_form(cache.rope, neighbours, *w) if normed or neighbours else None for w in gains]
    log = {}  # slot: rows so far, per layer (x, out)

    def step(rows):
        batch, starts = cache.step(rows)
        for l in range(2):
            x = torch.randn(starts[-1], H + 2 * K, d, generator=g, device="cuda").bfloat16()
            q, out = torch.empty_like(x[:, :H]), torch.empty_like(x[:, :H])
            cache.append(l, batch, x[:, :H], x[:, H:H + K], x[:, H + K:], q, forms[l])
            cache.attend(l, batch, q, out)
            for slot, n in rows.items():
                rng = slice(starts[slot], starts[slot] + n)
                log.setdefault(slot, ([], []))[l].append((x[rng], q[rng], out[rng]))
        cache.advance(rows)

    def check(slot):
        n = cache.table.lens[slot]
        pos = torch.arange(n, device="cuda")
        page, off = cache.tables[slot].long()[pos // 16], pos % 16
        for l in range(2):
            x, q, out = (torch.cat(t) for t in zip(*log[slot][l]))
            y, near = formed(x[:, :H], gains[l][0], cache.rope, pos, rotary, neighbours)
            assert ((q.double() - y).abs() <= U[dtype] * y.abs() + 2.0 ** -19 * near + 2.0 ** -134).all()
            if code is None:
                k, v = (t[page, :, off].double() for t in cache.pools[l].tensors)
            else:
                kc, vc, ks, vs = cache.pools[l].tensors
                k, v = (mx.decode(c.view(torch.uint8)[page, :, off].view(c.dtype), s[page, :, off]) for c, s in ((kc, ks), (vc, vs)))
                z, near = formed(x[:, H:H + K], gains[l][1], cache.rope, pos, rotary, neighbours)
                e = ks[page, :, off].double() - 127
                step_ = mx.spacing(torch.maximum((k.unflatten(-1, (-1, 32)) / torch.exp2(e)[..., None]).abs(),
                                                 (z.unflatten(-1, (-1, 32)) / torch.exp2(e)[..., None]).abs()), code) * torch.exp2(e)[..., None]
                assert ((k - z).abs() <= step_.flatten(-2) / 2 + 2.0 ** -19 * near).all()
                want, scales = mx.encode(x[:, H + K:], code, dtype)
                assert torch.equal(v, mx.decode(want, scales))
            hide = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
            for h in range(H):
                w = torch.softmax((q[:, h].double() @ k[:, h // 3].T / 8).masked_fill(hide, -math.inf), -1)
                o, a = w @ v[:, h // 3], w @ v[:, h // 3].abs()
                assert ((out[:, h].double() - o).abs() <= U[dtype] * o.abs() + (U[dtype] + 2.0 ** -16) * a + 2.0 ** -30 * v.abs().max()).all()

    try:
        a, b = cache.admit(), cache.admit()
        step({a: 40, b: 7})
        for _ in range(5):
            step({a: 1, b: 1})
        check(a)
        cache.release(a)
        del log[a]
        a = cache.admit()
        step({a: 90, b: 1})
        step({a: 3, b: 2})
        for _ in range(3):
            step({a: 1, b: 1})
        check(a)
        check(b)
        assert vt.vt_paged_status(cache.paged) == 0
    finally:
        cache.close()


@pytest.mark.parametrize("kw", [dict(code="fp8"), dict(code="int8", page_size=4), dict(rotary_dim=24), dict(rotary_dim=80), dict(rotary_dim=-16)])
def test_what_a_cache_refuses(vtlib, kw):
    from paper_2607_07046_gb300.paged import PagedCache
    with pytest.raises(ValueError):
        PagedCache(1, 1, 64, kw.pop("page_size", 16), 4, 1, 32, **kw)


@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_serving_example_in_8_bits(vtlib, code):
    """It serves its five sequences; codes are off by 2^-4 (e4m3) at most, of values that are averaged: the hidden states stay within
    that of the sequence alone."""
    from examples.paged_serving import serve
    err, n = serve(code)
    assert n == 5 and err <= 2.0 ** -4, err
