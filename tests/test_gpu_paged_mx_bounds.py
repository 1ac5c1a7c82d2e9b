"""Attention over paged pools in 8 bits by the kernel of few rows, against 64 bits and with the bound that each row has by
itself: what a row does not attend to may not count.

With w_j a row's weights, u half a unit of the type relative to its value and A = sum_j w_j |v_j|,
    |error| <= u |o| + (2^-16 + 2^-22) A + n 2^-36 max_j w_j max_j |v_j| + 2^-25 (fp16 only)
over the n positions that the row attends to: the output is rounded once; fp32 scores, exponentials and sums of these sizes
take 2^-16; two fp16 terms leave 2^-22 of a weight, and 2^-37 of the largest where the second is below the type's smallest step, which
meets at most twice the largest value (a scale is the least power of two that holds its block); an fp16 output has steps of 2^-24."""
from __future__ import annotations

import math

import pytest

torch = pytest.importorskip("torch")
from tests.test_gpu_paged import TINY, TYPE, U  # noqa: E402
from tests.test_gpu_paged_mx import KINDS, attend, paged  # noqa: E402,F401
from tests.test_gpu_paged_qk import MxCache  # noqa: E402

pytestmark = pytest.mark.gpu


def bounded(c, q, scale, window):
    H, G = q.shape[1], q.shape[1] // c.kv_heads
    out, tol = (torch.zeros(q.shape, dtype=torch.float64, device="cuda") for _ in range(2))
    for b, (p, r) in enumerate(zip(c.lens_host, c.rows_host)):
        if p < 0 or r == 0:
            continue
        page, off = c.positions(b, p + r)
        k, v = c.k[page, :, off].double(), c.v[page, :, off].double()
        pos, me = torch.arange(p + r, device="cuda"), torch.arange(p, p + r, device="cuda")[:, None]
        hide = pos > me
        if window:
            hide = hide | (pos <= me - window)
        n, rows = (~hide).sum(-1, keepdim=True), slice(c.starts_host[b], c.starts_host[b] + r)
        for h in range(H):
            vh = v[:, h // G]
            w = torch.softmax((q[rows, h].double() @ k[:, h // G].T * scale).masked_fill(hide, -math.inf), -1)
            o, a = w @ vh, w @ vh.abs()
            most = vh.abs().amax(-1).expand(r, -1).masked_fill(hide, 0.0).amax(-1, keepdim=True)
            out[rows, h] = o
            tol[rows, h] = (U[c.dtype] * o.abs() + (2.0 ** -16 + 2.0 ** -22) * a + n * 2.0 ** -36 * w.amax(-1, keepdim=True) * most
                            + TINY[c.dtype])
    return out, tol


def check(vt, g, c, call, q, window=0, scale=None):
    scale = c.d_head ** -0.5 if scale is None else scale
    out = torch.full_like(q, 7.0)
    attend(vt, g, c, call, q, out, scale, window)
    ref, tol = bounded(c, q, scale, window)
    far = (out.double() - ref).abs()
    assert torch.isfinite(out).all()
    assert (far <= tol).all(), f"{float((far / tol.clamp(min=1e-300)).max())} times the bound"
    assert vt.vt_paged_status(g) == 0
    return out


@pytest.mark.parametrize("d_head,kv_heads,group,page", [(64, 2, 1, 16), (128, 2, 4, 32), (128, 1, 12, 16), (64, 1, 16, 64)])
@pytest.mark.parametrize("call", ["decode", "prefill"])
@pytest.mark.parametrize("dtype,code", KINDS)
def test_weights_carry_two_terms(vtlib, paged, dtype, code, call, d_head, kv_heads, group, page):
    lens = [0, 1, 15, 16, 63, 200, 777, 3000, -1, 5000]
    c = MxCache(vtlib, lens, [1] * len(lens), code, dtype, kv_heads, d_head, page)
    check(vtlib, paged, c, call, c.rows(kv_heads * group))


@pytest.mark.parametrize("d_head,heads", [(64, 4), (128, 4), (128, 12)])
@pytest.mark.parametrize("each", [1, 3])
@pytest.mark.parametrize("dtype,code", KINDS)
def test_many_short_sequences(vtlib, paged, dtype, code, each, d_head, heads):
    """Enough short sequences that each warp has its own, with one row or several and one tile of columns or more."""
    lens = [i % 66 - 1 for i in range(700)]
    c = MxCache(vtlib, lens, [each] * 700, code, dtype, 4, d_head, 16)
    q = c.rows(heads)
    check(vtlib, paged, c, "decode" if each == 1 else "prefill", q)
