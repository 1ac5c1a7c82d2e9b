"""Norms of heads whose squares a 32-bit sum does not hold: bf16 magnitudes from the smallest subnormal number to the largest,
with eps 0 and others, against the definition in 64 bits.  The tolerances are those of test_gpu_paged_qk (a power of two taken out of
a head rounds nothing); 2^-134 is half a bf16's smallest step."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")
from tests import mx_reference as mx  # noqa: E402
from tests.test_gpu_paged import U, Cache  # noqa: E402
from tests.test_gpu_paged_qk import NEAR, MxCache, paged, table  # noqa: E402,F401

pytestmark = pytest.mark.gpu
POWERS = [-132, -120, -100, -90, -80, -75, -70, -66, -63, -50, -40, -21, -20, -19, 0, 7, 19, 20, 21, 40, 55, 59, 60, 61, 63, 64, 90, 110, 124]


def formed(x, gain, eps, rope, neighbours):
    y = x.double()
    y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps) * gain.double()
    near = y.abs()
    half = rope.shape[1]
    i = torch.arange(half, device="cuda")
    a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + half)
    cos, sin = rope[:x.shape[0]].double()[:, None].unbind(-1)
    out, met = y.clone(), near.clone()
    out[..., a], out[..., b] = y[..., a] * cos - y[..., b] * sin, y[..., b] * cos + y[..., a] * sin
    met[..., a] = met[..., b] = near[..., a] + near[..., b]
    return out, met


@pytest.mark.parametrize("eps", [0.0, 2.0 ** -140, 1e-30, 1e-12, 1e-6])
@pytest.mark.parametrize("code", [None, "e4m3", "int8"])
@pytest.mark.parametrize("d_head,neighbours,repeat", [(64, False, 1), (128, True, 1), (128, False, 20)])
def test_heads_of_any_magnitude(vtlib, paged, code, eps, d_head, neighbours, repeat):
    """Every head of a row has another magnitude; some have one large value, or a few, among zeros.  (20 times as many rows: the kernel for
    many.)"""
    vt, K, H = vtlib, 2, 6
    n = len(POWERS) * repeat
    args = ("bf16", K, d_head, 16, "head")
    c = MxCache(vt, [0], [n], code, *args) if code else Cache(vt, [0], [n], *args)
    x = torch.randn(n, H + K, d_head, generator=c.gen, device="cuda").double()
    x[:, 1, 1:] = 0.0
    x[:, H, 5:] = 0.0
    at = (torch.arange(n, device="cuda")[:, None] + 5 * torch.arange(H + K, device="cuda")) % len(POWERS)
    x = (x * torch.exp2(torch.tensor(POWERS, device="cuda").double())[at][..., None]).clamp(-3e38, 3e38).bfloat16()
    if eps == 0.0:  # a head of zeros has no norm there
        x[..., 0] = torch.where((x == 0).all(-1), torch.full_like(x[..., 0], 2.0 ** -133), x[..., 0])
    gains = [(1 + 0.2 * torch.randn(d_head, generator=c.gen, device="cuda")).bfloat16() for _ in range(2)]
    rope = table(n, d_head)
    form = vt.make_qk_form(rope, neighbours, *gains, eps)
    q, k = x[:, :H], x[:, H:]
    out = torch.empty_like(q)
    (vt.vt_paged_append_mx if code else vt.vt_paged_append_qk)(paged, c.pool, c.batch(vt), q, k, k, form, out)
    y, near = formed(q, gains[0], eps, rope, neighbours)
    tol = U["bf16"] * y.abs() + NEAR * near + 2.0 ** -134
    far = (out.double() - y).abs()
    assert (far <= tol).all(), [POWERS[i] for i in at[:, :H][~(far <= tol).all(-1)].unique()]
    y, near = formed(k, gains[1], eps, rope, neighbours)
    page, off = c.positions(0, n)
    if not code:
        far = (c.k[page, :, off].double() - y).abs()
        assert (far <= U["bf16"] * y.abs() + NEAR * near + 2.0 ** -134).all()
    else:
        z, s = (t.view(torch.uint8)[page, :, off] for t in (c.codes[0], c.scales[0]))
        z, power = z.view(mx.CODES[code]).double().unflatten(-1, (-1, 32)), torch.exp2(s.double() - 127)[..., None]
        y, near = y.unflatten(-1, (-1, 32)), near.unflatten(-1, (-1, 32))
        step = mx.spacing(torch.maximum(z.abs(), y.abs() / power), code) * power
        assert (s != 255).all() and ((z * power - y).abs() <= step / 2 + NEAR * near).all()
        most, top = y.abs().amax(-1), mx.MOST[code] * power.squeeze(-1)
        room = NEAR * near.amax(-1)
        assert (most <= top + room).all() and ((2 * most >= top - 2 * room) | (s == 127 + mx.RANGE[code, "bf16"][0])).all()
    assert vt.vt_paged_status(paged) == 0


@pytest.mark.parametrize("small", ["gain", "eps"])
def test_in_place_beside_heads_that_come_out_small(vtlib, paged, small):
    """Queries are formed in place; some have squares that 32 bits do not hold, others come out as small as that (by a gain of 2^-80
    or an eps of 2^80) and must not be taken for them."""
    vt, n, H = vtlib, 600, 6
    eps = 2.0 ** 80 if small == "eps" else 0.0
    c = Cache(vt, [0], [n], "bf16", 1, 128, 16)
    x = torch.randn(n, H + 2, 128, generator=c.gen, device="cuda").double()
    x[:, ::2] *= 2.0 ** -70
    x[::3, 1] *= 2.0 ** 70
    x = x.bfloat16()
    gain = (torch.randn(128, generator=c.gen, device="cuda") * 2.0 ** (-80 if small == "gain" else 0)).bfloat16()
    rope = table(n, 128)
    y, near = formed(x[:, :H], gain, eps, rope, False)
    q = x[:, :H]
    vt.vt_paged_append_qk(paged, c.pool, c.batch(vt), q, x[:, H:H + 1], x[:, H + 1:], vt.make_qk_form(rope, False, gain, gain, eps), q)
    assert ((q.double() - y).abs() <= U["bf16"] * y.abs() + NEAR * near + 2.0 ** -134).all()


@pytest.mark.parametrize("code", [None, "int8"])
def test_what_is_not_finite_stays_so(vtlib, paged, code):
    """An infinity is infinity / infinity, and what stands beside it 0; NaN, and zeros with eps 0, are NaN."""
    vt = vtlib
    c = MxCache(vt, [0], [4], code, "bf16", 1, 64, 16) if code else Cache(vt, [0], [4], "bf16", 1, 64, 16)
    x = c.rows(1)
    x[0, 0, 3], x[1, 0, 3], x[2] = float("inf"), float("nan"), 0.0
    gain = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(x)
    (vt.vt_paged_append_mx if code else vt.vt_paged_append_qk)(paged, c.pool, c.batch(vt), x, x, x, vt.make_qk_form(None, False, gain, gain, 0.0), out)
    assert out[0, 0, 3].isnan() and not out[0, 0, :3].any() and not out[0, 0, 4:].any()
    assert out[1].isnan().all() and out[2].isnan().all() and torch.isfinite(out[3]).all()
