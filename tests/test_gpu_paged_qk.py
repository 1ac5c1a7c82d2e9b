"""The appends with norms of queries and keys, both rotations and pools in 8 bits (vt_paged_append_qk,
vt_paged_append_mx) against their definition in 64 bits.

Tolerances, by the arithmetic alone.  The sum of up to 128 squares takes 8 sums in a lane and 4 between lanes, the
root halves their error; the reciprocal root is off by 2 units in the last place, the mean, the sum with eps, the
gain's and the norm's products by half a unit each, and the rotation adds two products and a sum:
((8 + 4) / 2 + 4 + 4 + 3) 2^-24 < 2^-19 of |a| + |b|, the magnitudes that meet in the rotation.  Then a value is rounded
once: to its type (half a unit, and half the smallest step), or to a code (half the distance of the codes around it).
Without norm and rotation there is nothing but the one rounding, and codes and scales are exact."""
from __future__ import annotations

import math

import pytest

torch = pytest.importorskip("torch")
from tests import mx_reference as mx  # noqa: E402
from tests.test_gpu_paged import TINY, TYPE, U, Cache  # noqa: E402

pytestmark = pytest.mark.gpu
EPS = 1e-6
NEAR = 2.0 ** -19


@pytest.fixture()
def paged(vtlib):
    g = vtlib.vt_paged_create()
    yield g
    vtlib.vt_paged_destroy(g)


class MxCache(Cache):
    """A pool in 8 bits whose live entries stand for self.k and self.v; the others hold any codes and NaN scales."""

    def __init__(self, vt, lens, rows, code, dtype="f16", kv_heads=2, d_head=64, page=16, order="head", seed=0, std=1.0, spare=2):
        super().__init__(vt, lens, rows, dtype, kv_heads, d_head, page, order, seed, std, spare)
        self.code, self.plain = code, []
        self.codes, self.scales = [], []
        for name in ("k", "v"):
            x = getattr(self, name)
            dead = ~self.live[:, None, :, None]
            codes, scales = mx.encode(x.masked_fill(dead, 0.0), code, dtype)
            codes = codes.to(mx.CODES[code]) if code == "int8" else codes.float().to(mx.CODES[code])
            junk = torch.randint(0, 256, codes.shape, generator=self.gen, device="cuda", dtype=torch.uint8)
            codes = torch.where(dead, junk, codes.view(torch.uint8)).view(mx.CODES[code])
            scales = scales.masked_fill(dead, 255).contiguous()
            if order == "pos":
                codes = codes.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
            self.codes.append(codes)
            self.scales.append(scales)
            values = mx.decode(codes, scales)
            x.copy_(values.masked_fill(dead, float("nan")))
            assert (x.double() == values).masked_select(~dead.expand_as(x)).all()  # an entry's values are values of the type
        self.plain = self.pool
        self.pool = vt.make_paged_mx_pool(*self.codes, *self.scales, TYPE[dtype])


def formed(x, gain, rope, pos, rotary, neighbours):
    """(values, magnitudes that met) in 64 bits."""
    y = x.double()
    if gain is not None:
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + EPS) * gain.double()
    near = y.abs()
    if rotary:
        i = torch.arange(rotary // 2, device="cuda")
        a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + rotary // 2)
        cos, sin = rope[pos].double()[:, None].unbind(-1)
        y2, near2 = y.clone(), near.clone()
        y2[..., a], y2[..., b] = y[..., a] * cos - y[..., b] * sin, y[..., b] * cos + y[..., a] * sin
        near2[..., a] = near2[..., b] = near[..., a] + near[..., b]
        return y2, near2
    return y, near


def table(n, rotary, theta=1e4):
    at = torch.arange(n, device="cuda").double()[:, None] * theta ** (-2.0 * torch.arange(rotary // 2, device="cuda").double() / max(rotary, 1))
    return torch.stack((at.cos(), at.sin()), -1).float().contiguous() if rotary else None


def run_append(vt, paged, c, code, heads, rotary, neighbours, norm, in_place=False, wide=0):
    d, K, n = c.d_head, c.kv_heads, c.n_rows
    qkv = torch.randn(n, heads + 2 * K + wide, d, generator=c.gen, device="cuda").mul_(1.3).to(TYPE[c.dtype])
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + K], qkv[:, heads + K:heads + 2 * K]
    gains = [(1 + 0.2 * torch.randn(d, generator=c.gen, device="cuda")).to(TYPE[c.dtype]) if g else None for g in norm]
    rope = table(c.tables.shape[1] * c.page, rotary)
    form = vt.make_qk_form(rope, neighbours, *gains, EPS)
    src = qkv.clone()
    q_out = q if in_place else torch.full((n, heads, d), 7.0, dtype=TYPE[c.dtype], device="cuda")
    before = [t.clone() for t in (c.codes + c.scales if code else [c.k, c.v])]
    (vt.vt_paged_append_mx if code else vt.vt_paged_append_qk)(paged, c.pool, c.batch(vt), q, k, v, form, q_out)
    q, k, v = src[:, :heads], src[:, heads:heads + K], src[:, heads + K:heads + 2 * K]
    touched = torch.zeros(c.k.shape[0], c.page, dtype=torch.bool, device="cuda")
    for b, (p, r) in enumerate(zip(c.lens_host, c.rows_host)):
        s0 = c.starts_host[b]
        rows = slice(s0, s0 + r)
        if p < 0 or r == 0:
            assert not q_out[rows].any()
            continue
        pos = torch.arange(p, p + r, device="cuda")
        page, off = c.positions(b, p + r)
        page, off = page[p:], off[p:]
        touched[page, off] = True
        y, near = formed(q[rows], gains[0], rope, pos, rotary, neighbours)
        tol = U[c.dtype] * y.abs() + NEAR * near + (TINY[c.dtype] or 2.0 ** -134)
        far = (q_out[rows].double() - y).abs()
        assert (far <= tol).all(), float((far / tol).max())
        for i, (x, gain, turns) in enumerate(((k, gains[1], rotary), (v, None, 0))):
            y, near = formed(x[rows], gain, rope, pos, turns, neighbours)
            if not code:
                got = (c.k, c.v)[i][page, :, off].double()
                tol = U[c.dtype] * y.abs() + NEAR * near + (TINY[c.dtype] or 2.0 ** -134)
                assert ((got - y).abs() <= (tol if i == 0 else 0 * tol)).all()
                continue
            codes, scales = (t.view(torch.uint8)[page, :, off] for t in (c.codes[i], c.scales[i]))
            z, e = codes.view(mx.CODES[code]).double().unflatten(-1, (-1, 32)), scales.double() - 127
            power = torch.exp2(e)[..., None]
            y, near = y.unflatten(-1, (-1, 32)), near.unflatten(-1, (-1, 32))
            exact = turns == 0 and gain is None
            slack = 0.0 if exact else NEAR
            step = mx.spacing(torch.maximum(z.abs(), y.abs() / power), code) * power
            assert ((z * power - y).abs() <= step / 2 + slack * near).all()
            lo, hi = mx.RANGE[code, c.dtype]
            most, room = y.abs().amax(-1), slack * near.amax(-1)
            top = mx.MOST[code] * torch.exp2(e)
            assert ((most <= top + room) | (e == hi)).all() and ((2 * most >= top - 2 * room) | (e == lo)).all()
            if exact:
                want, bytes_ = mx.encode(x[rows], code, c.dtype)
                assert torch.equal(z.flatten(-2), want) and torch.equal(scales, bytes_)
    # nothing else is touched
    for t, old in zip(c.codes + c.scales if code else [c.k, c.v], before):
        t, old = (x.view(torch.uint8) if code else x.view(torch.int16) for x in (t, old))
        assert torch.equal(t.masked_fill(touched[:, None, :, None], 0), old.masked_fill(touched[:, None, :, None], 0))
    assert vt.vt_paged_status(paged) == 0


LENS, ROWS = [0, 3, -1, 15, 40, 7, 100], [1, 5, 2, 0, 19, 1, 33]


@pytest.mark.parametrize("code", [None, "e4m3", "int8"])
@pytest.mark.parametrize("dtype,d_head,kv_heads,group,page,order,rotary,neighbours,norm", [
    ("f16", 64, 2, 4, 16, "head", 64, False, (True, True)), ("bf16", 128, 2, 4, 8, "pos", 128, False, (True, True)),
    ("f16", 128, 1, 3, 32, "head", 64, True, (True, True)), ("bf16", 64, 3, 1, 8, "pos", 16, False, (False, True)),
    ("f16", 64, 1, 8, 64, "pos", 32, True, (True, False)), ("bf16", 128, 5, 1, 1024, "head", 112, True, (False, False)),
    ("f16", 128, 2, 1, 16, "head", 48, False, (True, True)), ("bf16", 64, 2, 2, 128, "head", 0, False, (True, True)),
    ("f16", 64, 8, 1, 8, "pos", 0, True, (False, False))])
def test_append(vtlib, paged, code, dtype, d_head, kv_heads, group, page, order, rotary, neighbours, norm):
    args = (dtype, kv_heads, d_head, page, order)
    c = MxCache(vtlib, LENS, ROWS, code, *args) if code else Cache(vtlib, LENS, ROWS, *args)
    run_append(vtlib, paged, c, code, kv_heads * group, rotary, neighbours, norm, wide=1)


@pytest.mark.parametrize("code", [None, "e4m3", "int8"])
@pytest.mark.parametrize("dtype,d_head", [("f16", 128), ("bf16", 64)])
def test_many_rows_and_in_place(vtlib, paged, code, dtype, d_head):
    lens, rows = [0, 700, 5, -1, 64], [300, 130, 511, 9, 64]
    args = (dtype, 3, d_head, 16, "pos")
    c = MxCache(vtlib, lens, rows, code, *args) if code else Cache(vtlib, lens, rows, *args)
    run_append(vtlib, paged, c, code, 9, d_head, False, (True, True), in_place=True)


def test_as_the_plain_append_without_norms(vtlib, paged):
    """With the rotation of vt_paged_append and no norm: its pool and queries within a unit in the last place (the same
    products and sum), values bit for bit."""
    vt = vtlib
    a, b = (Cache(vt, LENS, ROWS, "f16", 2, 128, 16, seed=3) for _ in range(2))
    rope = torch.empty(a.tables.shape[1] * 16, 64, 2, device="cuda")
    vt.vt_rope_table(rope, 1e4)
    x = a.rows(8)
    qa, qb = torch.empty_like(x[:, :4]), torch.empty_like(x[:, :4])
    vt.vt_paged_append(paged, a.pool, a.batch(vt), x[:, :4], x[:, 4:6], x[:, 6:], rope, qa)
    vt.vt_paged_append_qk(paged, b.pool, b.batch(vt), x[:, :4], x[:, 4:6], x[:, 6:], vt.make_qk_form(rope), qb)
    assert torch.equal(a.v.view(torch.int16), b.v.view(torch.int16))
    for s, t in ((qa, qb), (a.k[a.live[:, None].expand(-1, 2, -1)], b.k[a.live[:, None].expand(-1, 2, -1)])):
        assert ((s.double() - t.double()).abs() <= 2 * U["f16"] * s.double().abs() + 2.0 ** -19).all()


def patterns(code, dtype):
    """Rows of 64 values where rounding can go wrong, of the type."""
    t, g = TYPE[dtype], torch.Generator().manual_seed(5)
    lo, hi = mx.RANGE[code, dtype]
    rows = [torch.zeros(64), torch.full((64,), -0.0), torch.linspace(-1, 1, 64)]
    ramp = torch.arange(64).double()
    for power in {0, -3, 5, lo, hi - 1}:
        s = 2.0 ** power
        # every code's neighbourhood: ties between codes (the type has the bits for them), the largest code beside them
        grid = torch.tensor(mx.E4M3 if code == "e4m3" else list(range(128)), dtype=torch.float64)
        ties = (grid[1:] + grid[:-1]) / 2
        for part in ties.split(31):
            for sign in (1.0, -1.0):
                row = torch.full((64,), mx.MOST[code] * s, dtype=torch.float64)
                row[1:1 + len(part)] = sign * part * s
                row[33:33 + len(part)] = sign * part * s
                rows.append(row)
        rows.append((ramp - 32) * s / 8)
        # the largest value right at, below and above the border between two scales
        for most in (mx.MOST[code], mx.MOST[code] * (1 - 2.0 ** -7), mx.MOST[code] * (1 + 2.0 ** -6)):
            rows.append(torch.cat((torch.tensor([most * s]), torch.randn(63, generator=g).double() * s)))
    info = torch.finfo(t)
    rows += [torch.full((64,), info.max).double(), torch.full((64,), -info.max).double(), torch.full((64,), info.tiny).double(),
             torch.full((64,), info.smallest_normal / 4).double(), torch.cat((torch.full((32,), info.max).double(), torch.ones(32).double()))]
    # ties that the type can hold exactly; the others are rounded to it, which is fine
    return torch.stack([r.double().clamp(-info.max, info.max) for r in rows]).to(t)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_codes_and_scales_exactly(vtlib, paged, code, dtype):
    vt = vtlib
    x = patterns(code, dtype).cuda()[:, None]
    n = x.shape[0]
    c = MxCache(vt, [0], [n], code, dtype, 1, 64, 8)
    out = torch.empty_like(x)
    vt.vt_paged_append_mx(paged, c.pool, c.batch(vt), x, x, -x, vt.make_qk_form(), out)
    assert torch.equal(out, x)
    page, off = c.positions(0, n)
    for i, y in enumerate((x, -x)):
        want, scales = mx.encode(y, code, dtype)
        got = c.codes[i].view(torch.uint8)[page, :, off].view(mx.CODES[code]).double()
        assert torch.equal(c.scales[i].view(torch.uint8)[page, :, off], scales)
        assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_what_is_not_finite_marks_its_32_dimensions(vtlib, paged, code, dtype):
    vt = vtlib
    c = MxCache(vt, [0], [5], code, dtype, 1, 128, 16)
    x = c.rows(1)
    x[1, 0, 40], x[2, 0, 0], x[3, 0, 127], x[4, 0, 64] = float("nan"), float("inf"), float("-inf"), float("nan")
    bad = {1: 1, 2: 0, 3: 3, 4: 2}
    vt.vt_paged_append_mx(paged, c.pool, c.batch(vt), x, x, x, vt.make_qk_form(), torch.empty_like(x))
    page, off = c.positions(0, 5)
    want, scales = mx.encode(torch.nan_to_num(x, 0.0, 0.0, 0.0), code, dtype)
    for codes, s in zip(c.codes, c.scales):
        codes, s = codes.view(torch.uint8)[page, 0, off].view(mx.CODES[code]).double(), s.view(torch.uint8)[page, 0, off]
        for r in range(5):
            for b in range(4):
                part = codes[r, 32 * b:32 * b + 32]
                if bad.get(r) == b:
                    assert s[r, b] == 255 and not part.any()
                else:
                    assert s[r, b] == scales[r, 0, b] and torch.equal(part, want[r, 0, 32 * b:32 * b + 32])


@pytest.mark.parametrize("code", [None, "e4m3"])
def test_what_does_not_fit_is_skipped_and_flagged(vtlib, paged, code):
    """A position past the table or the rotation, a bad page, an idle slot, rows behind the last sequence."""
    vt = vtlib
    c = MxCache(vt, [30, 5, -1], [4, 4, 2], code, "f16", 1, 64, 16) if code else Cache(vt, [30, 5, -1], [4, 4, 2], "f16", 1, 64, 16)
    call = vt.vt_paged_append_mx if code else vt.vt_paged_append_qk
    x = torch.randn(13, 1, 64, generator=c.gen, device="cuda").half()
    stores = c.codes + c.scales if code else [c.k, c.v]

    def run(rope_len, lens=None):
        if lens is not None:
            c.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        out = torch.full_like(x, 7.0)
        call(paged, c.pool, c.batch(vt), x, x, x, vt.make_qk_form(table(rope_len, 64)), out)
        return out, vt.vt_paged_status(paged, clear=True)

    out, status = run(48)
    assert status == 0 and out[:8].any(-1).all() and not out[8:10].any() and (out[10:] == 7.0).all()
    out, status = run(33)
    assert status == vt.VT_DEV_KV_OVERFLOW and not out[3].any() and out[2].any()
    out, status = run(48, [46, 5, -5])
    assert status == vt.VT_DEV_KV_OVERFLOW and out[1].any() and not out[2:4].any() and out[4:8].any(-1).all()
    for much in (48, 2 ** 31 - 1):
        out, status = run(48, [much, 5, -1])
        assert status == vt.VT_DEV_KV_OVERFLOW and not out[:4].any()
    keep = [t.clone() for t in stores]
    for bad in (-1, c.k.shape[0], 2 ** 31 - 1, -2 ** 31):
        c.tables[0, 1] = bad
        out, status = run(48, [20, 5, -1])
        assert status == vt.VT_DEV_BAD_PAGE and out[:4].any(-1).all()  # queries are formed all the same
        assert all(torch.equal(s.view(torch.uint8), k.view(torch.uint8)) for s, k in zip(stores, keep)) or bad == -1
        keep = [t.clone() for t in stores]


def test_zero_rows_and_eps(vtlib, paged):
    """A head of zeros stays zero with eps > 0; eps 0 gives NaN there, as 0 / 0 does."""
    vt = vtlib
    c = Cache(vt, [0], [2], "bf16", 1, 64, 16)
    x = c.rows(1)
    x[0] = 0.0
    gain = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(x)
    vt.vt_paged_append_qk(paged, c.pool, c.batch(vt), x, x, x, vt.make_qk_form(None, False, gain, gain, 1e-6), out)
    assert not out[0].any() and math.isclose(float(out[1].float().square().mean()), 1.0, rel_tol=2.0 ** -7)
    vt.vt_paged_append_qk(paged, c.pool, c.batch(vt), x, x, x, vt.make_qk_form(None, False, gain, gain, 0.0), out)
    assert out[0].isnan().all() and not out[1].isnan().any()
