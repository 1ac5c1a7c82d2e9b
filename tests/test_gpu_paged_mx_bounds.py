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
from tests import mx_reference as mx  # noqa: E402
from tests.test_gpu_paged import TINY, TYPE, U  # noqa: E402
from tests.test_gpu_paged_mx import KINDS, attend, paged  # noqa: E402,F401
from tests.test_gpu_paged_qk import MxCache  # noqa: E402

pytestmark = pytest.mark.gpu


def set_values(c, side, x):
    """The live entries of one side (0: K, 1: V) anew, from values [pages, KV heads, positions, head dim]."""
    live = c.live[:, None, :, None]
    codes, scales = mx.encode(x.double().masked_fill(~live, 0.0), c.code, c.dtype)
    values = mx.decode(codes, scales)
    codes = (codes if c.code == "int8" else codes.float()).to(mx.CODES[c.code]).view(torch.uint8)
    c.codes[side].view(torch.uint8).copy_(torch.where(live, codes, c.codes[side].view(torch.uint8)))
    c.scales[side].copy_(torch.where(live, scales, c.scales[side]))
    (c.k, c.v)[side].copy_(values.masked_fill(~live, float("nan")))


def entry(c, b, j):
    """Index of position j of sequence b in a side of the pool, all KV heads."""
    page, off = c.positions(b, j + 1)
    return page[j], slice(None), off[j]


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


@pytest.mark.parametrize("window", [0, 3])
@pytest.mark.parametrize("d_head,group,held", [(64, 1, 41), (128, 1, 61), (128, 3, 41), (64, 5, 0), (128, 4, 3000)])
@pytest.mark.parametrize("dtype,code", KINDS)
def test_a_row_is_not_disturbed_by_values_that_it_does_not_attend_to(vtlib, paged, dtype, code, d_head, group, held, window):
    """The values of the last of four new rows, and with a window those of a position that the first row alone attends to, far
    above the others: rows that attend to neither have the bits that they have without."""
    vt = vtlib
    up = 2.0 ** (60 if (dtype, code) == ("bf16", "int8") else 12)
    low = 2.0 ** (-44 if (dtype, code) == ("bf16", "e4m3") else -4 if dtype == "f16" else 0)
    c = MxCache(vt, [held, 9], [4, 1], code, dtype, 2, d_head, 16, spare=0)
    live = c.live[:, None, :, None]
    v = c.v.double().masked_fill(~live, 0.0) * low
    set_values(c, 1, v)
    q = c.rows(2 * group)
    plain = check(vt, paged, c, "prefill", q, window)
    v[entry(c, 0, held + 3)] *= up / low
    first = held - 2
    if window and first >= 0:
        v[entry(c, 0, first)] *= up / low
    set_values(c, 1, v)
    out = check(vt, paged, c, "prefill", q, window)
    quiet = slice(1 if window else 0, 3)
    assert torch.equal(out[quiet].view(torch.int16), plain[quiet].view(torch.int16))


@pytest.mark.parametrize("d_head,kv_heads,group,page", [(64, 2, 1, 16), (128, 2, 4, 32), (128, 1, 12, 16), (64, 1, 16, 64)])
@pytest.mark.parametrize("call", ["decode", "prefill"])
@pytest.mark.parametrize("dtype,code", KINDS)
def test_weights_carry_two_terms(vtlib, paged, dtype, code, call, d_head, kv_heads, group, page):
    lens = [0, 1, 15, 16, 63, 200, 777, 3000, -1, 5000]
    c = MxCache(vtlib, lens, [1] * len(lens), code, dtype, kv_heads, d_head, page)
    check(vtlib, paged, c, call, c.rows(kv_heads * group))


@pytest.mark.parametrize("call,rows", [("decode", [1] * 5), ("prefill", [3, 1, 4, 2, 6])])
@pytest.mark.parametrize("d_head,group", [(64, 1), (128, 4), (128, 12)])
@pytest.mark.parametrize("dtype,code", KINDS)
def test_values_of_many_magnitudes(vtlib, paged, dtype, code, d_head, group, call, rows):
    """Each position's values have a magnitude of their own, over as many powers of two as the type and the code have: in any order,
    and growing all along."""
    lo, hi = {("f16", "e4m3"): (-10, 12), ("bf16", "e4m3"): (-60, 12), ("f16", "int8"): (-14, 12), ("bf16", "int8"): (-60, 60)}[dtype, code]
    c = MxCache(vtlib, [0, 37, 700, -1, 4000], rows, code, dtype, 2, d_head, 16)
    live = c.live[:, None, :, None]
    std = c.v.double().masked_fill(~live, 0.0)
    q = c.rows(2 * group)
    set_values(c, 1, std * torch.exp2(torch.randint(lo, hi, c.live.shape, generator=c.gen, device="cuda").double())[:, None, :, None])
    check(vtlib, paged, c, call, q)
    grown = std.clone()
    for b, (p, r) in enumerate(zip(c.lens_host, c.rows_host)):
        if p >= 0:
            page, off = c.positions(b, p + r)
            grown[page, :, off] *= torch.exp2(torch.linspace(lo, hi, p + r, dtype=torch.float64, device="cuda").floor())[:, None, None]
    set_values(c, 1, grown)
    check(vtlib, paged, c, call, q)


@pytest.mark.parametrize("call,rows", [("decode", [1] * 4), ("prefill", [3, 1, 4, 2])])
@pytest.mark.parametrize("d_head,group", [(64, 1), (128, 4), (128, 12)])
@pytest.mark.parametrize("power", [-110, -60, 60, 100, 115, 122])
def test_keys_and_queries_of_far_magnitudes(vtlib, paged, power, d_head, group, call, rows):
    """bf16 keys in int8 far from 1, and queries as far on the other side: scores are what they are at 1, whatever a part of them is
    on the way.  (Beside them a query of zeros, whose magnitude is the smallest.)"""
    c = MxCache(vtlib, [0, 37, 700, 4000], rows, "int8", "bf16", 2, d_head, 16)
    live = c.live[:, None, :, None]
    set_values(c, 0, (c.k.double().masked_fill(~live, 0.0) * 2.0 ** power).clamp(-(2.0 ** 126), 2.0 ** 126))
    q = c.rows(2 * group).mul_(2.0 ** -power)
    q[-1, -1] = 0.0
    check(vtlib, paged, c, call, q)


@pytest.mark.parametrize("call", ["decode", "prefill"])
@pytest.mark.parametrize("bits", [20.3, 25.6, 27.1])
@pytest.mark.parametrize("dtype,code,value", [(*k, 1.0) for k in KINDS] + [("bf16", "e4m3", 2.0 ** -111), ("bf16", "int8", 2.0 ** -111),
                                                                          ("bf16", "int8", 2.0 ** 100), ("f16", "e4m3", 2.0 ** -9)])
def test_many_small_weights_add_up(vtlib, paged, dtype, code, value, bits, call):
    """One key takes nearly all the weight and its value is 0; 40,000 others have 2^-bits of it each and one value, so that the output
    is their sum alone.  A weight loses 2^-22 of itself or 2^-37 of the largest, and meets the value exactly or, as the bound has
    it, twice.  Scores of up to 40 log2 units carry 2^-24 of that as fp32 values, two roundings each, 2^-17 of a weight; at most 2504
    products are added in a row, 2^-23 of their sum each, and 1400 sums of weights, 2^-24 each: less than 2^-11."""
    n, seqs = 40000, 38
    c = MxCache(vtlib, [n], [1], code, dtype, 8, 64, 64)
    live, at = c.live[:, None, :, None], entry(c, 0, 777)
    k, v = torch.zeros_like(c.k, dtype=torch.float64), torch.zeros_like(c.v, dtype=torch.float64)
    k[at[0], :, at[2], 0] = 1.0
    v.masked_fill_(live, value)
    v[at] = 0.0
    set_values(c, 0, k)
    set_values(c, 1, v)
    assert (c.v.double() == v).masked_select(live.expand_as(v)).all() and (c.k.double() == k).masked_select(live.expand_as(k)).all()
    # as many sequences, on the same pages, as leave each CTA whole histories
    c.tables, c.lens, c.n_rows = c.tables.repeat(seqs, 1), c.lens.repeat(seqs), seqs
    c.starts = torch.arange(seqs + 1, dtype=torch.int32, device="cuda")
    q = torch.zeros(seqs, 16, 64, dtype=TYPE[dtype], device="cuda")
    q[:, :, 0] = 1.0
    out = torch.full_like(q, 7.0)
    attend(vtlib, paged, c, call, q, out, bits * math.log(2.0), 0)
    ref = n * 2.0 ** -bits / (1.0 + n * 2.0 ** -bits) * value
    tol = (U[dtype] + 2.0 ** -11 + 2.0 ** -17 + 2.0 ** -22) * ref + n * 2.0 ** -36 * value + TINY[dtype]
    assert ((out.double() - ref).abs() <= tol).all(), float(((out.double() - ref).abs() / tol).max())


@pytest.mark.parametrize("d_head,heads", [(64, 4), (128, 4), (128, 12)])
@pytest.mark.parametrize("each", [1, 3])
@pytest.mark.parametrize("dtype,code", KINDS)
def test_many_short_sequences(vtlib, paged, dtype, code, each, d_head, heads):
    """Enough short sequences that each warp has its own, with one row or several and one tile of columns or more."""
    lens = [i % 66 - 1 for i in range(700)]
    c = MxCache(vtlib, lens, [each] * 700, code, dtype, 4, d_head, 16)
    q = c.rows(heads)
    check(vtlib, paged, c, "decode" if each == 1 else "prefill", q)
