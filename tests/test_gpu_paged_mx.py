"""Attention over paged pools in 8 bits (vt_paged_decode_mx, vt_paged_prefill_mx) against the definition in 64 bits over the
values that the entries stand for.

An entry's values are values of the rows' type, so the bounds are those of the 16-bit pool (see test_gpu_paged.attention):
half a unit of the type for the output and for a weight, and 2^-16 for the fp32 scores, exponentials and sums.  Where the
tiles' kernel takes the whole batch, its operands are those that it has over a 16-bit pool of the same values, and so
are its outputs' bits.  Two terms come on top: an fp16 output below 2^-14 is rounded to steps of 2^-24, half of one being
2^-25 whatever its size; and a weight below 2^-126 of the row's largest is 0 in 32 bits (2^-126 is their
smallest normal number), which shows where the large ones meet values of exactly 0, as codes are often: (positions)
2^-126 max|v|.
The kernel of few rows takes weights to fp16 (with the scale of their values, over the largest scale), the largest between 2^12 and
2^15: the type's steps of 2^-24 below its normal numbers leave each off by 2^-25, which is 2^-37 of the row's largest weight, times
the largest scale and code, which is less than twice the largest value (the scale is the least power of two that holds it):
(positions) 2^-36 max|v|, which takes the place of the term before."""
from __future__ import annotations

import math

import pytest

torch = pytest.importorskip("torch")
from tests import mx_reference as mx  # noqa: E402
from tests.test_gpu_paged import LENS, TINY, TYPE, U, attention  # noqa: E402
from tests.test_gpu_paged_qk import MxCache, formed, table  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture()
def paged(vtlib):
    g = vtlib.vt_paged_create()
    yield g
    vtlib.vt_paged_destroy(g)


def attend(vt, g, c, call, q, out, scale=None, window=0):
    if call == "decode":
        vt.vt_paged_decode_mx(g, c.pool, c.batch(vt, starts=False), q, out, scale, window)
    else:
        vt.vt_paged_prefill_mx(g, c.pool, c.batch(vt), q, out, scale, window)


def check(vt, g, c, call, heads, window=0, scale=None, q=None, same_bits=False):
    q = c.rows(heads) if q is None else q
    out = torch.full_like(q, 7.0)
    scale = c.d_head ** -0.5 if scale is None else scale
    attend(vt, g, c, call, q, out, scale, window)
    ref, tol = attention(c, q, scale, window)
    tol = tol + 2.0 ** -36 * c.k.shape[0] * c.page * c.v.masked_fill(c.v.isnan(), 0.0).double().abs().max()
    tol = tol + TINY[c.dtype]
    far = (out.double() - ref).abs()
    assert torch.isfinite(out).all()
    assert (far <= tol).all(), f"{float((far / tol.clamp(min=1e-30)).max())} times the bound"
    if same_bits:
        plain = torch.empty_like(out)
        vt.vt_paged_prefill(g, c.plain, c.batch(vt), q, plain, scale, window)
        assert torch.equal(out.view(torch.int16), plain.view(torch.int16))
    assert vt.vt_paged_status(g) == 0


SHAPES = [(64, 8, 1, 16, "head"), (128, 2, 4, 16, "pos"), (128, 1, 1, 8, "head"), (64, 3, 2, 8, "pos"), (128, 2, 8, 64, "head"),
          (128, 1, 12, 32, "pos"), (64, 1, 16, 128, "head"), (128, 2, 3, 256, "head"), (64, 1, 71, 8, "head"), (128, 4, 5, 1024, "pos")]
KINDS = [("f16", "e4m3"), ("bf16", "e4m3"), ("f16", "int8"), ("bf16", "int8")]


@pytest.mark.parametrize("dtype,code", KINDS)
@pytest.mark.parametrize("d_head,kv_heads,group,page,order", SHAPES)
def test_decode(vtlib, paged, dtype, code, d_head, kv_heads, group, page, order):
    c = MxCache(vtlib, LENS, [1] * len(LENS), code, dtype, kv_heads, d_head, page, order)
    check(vtlib, paged, c, "decode", kv_heads * group)


@pytest.mark.parametrize("dtype,code", KINDS)
@pytest.mark.parametrize("window", [1, 16, 37, 200, 100000])
def test_decode_windowed(vtlib, paged, dtype, code, window):
    c = MxCache(vtlib, LENS, [1] * len(LENS), code, dtype, 2, 128, 8, "head")
    check(vtlib, paged, c, "decode", 8, window)


FEW = ([0, 5, 300, -1, 17, 64], [3, 1, 4, 2, 0, 7])
MANY = ([0, 100, -1, 33, 0, 700], [130, 257, 40, 0, 1, 64])


@pytest.mark.parametrize("dtype,code", KINDS)
@pytest.mark.parametrize("window", [0, 50])
@pytest.mark.parametrize("d_head,kv_heads,group,page,order", SHAPES)
def test_prefill(vtlib, paged, dtype, code, d_head, kv_heads, group, page, order, window):
    for lens, rows in (FEW, MANY):
        c = MxCache(vtlib, lens, rows, code, dtype, kv_heads, d_head, page, order)
        check(vtlib, paged, c, "prefill", kv_heads * group, window)


@pytest.mark.parametrize("dtype,code", KINDS)
@pytest.mark.parametrize("d_head,kv_heads,group,page,window", [(128, 16, 4, 16, 0), (64, 20, 1, 64, 0), (128, 12, 2, 8, 333), (64, 9, 8, 256, 0)])
def test_tiles_give_the_bits_of_a_16_bit_pool(vtlib, paged, dtype, code, d_head, kv_heads, group, page, window):
    """Enough work that the tiles' kernel takes it, in both calls."""
    c = MxCache(vtlib, [2000, 0, 700, 3001], [300, 513, 255, 200], code, dtype, kv_heads, d_head, page, "pos")
    check(vtlib, paged, c, "prefill", kv_heads * group, window, same_bits=True)


@pytest.mark.parametrize("dtype,code", KINDS)
def test_long_history_split_over_many(vtlib, paged, dtype, code):
    for d_head, group in ((128, 4), (64, 1)):
        c = MxCache(vtlib, [30000], [1], code, dtype, 2, d_head, 64, "head")
        check(vtlib, paged, c, "decode", 2 * group)
        c = MxCache(vtlib, [20001], [40], code, dtype, 2, d_head, 16, "pos")
        check(vtlib, paged, c, "prefill", 2 * group)


@pytest.mark.parametrize("window", [0, 37])
@pytest.mark.parametrize("dtype,d_head,group,code", [("f16", 128, 4, "e4m3"), ("bf16", 64, 1, "int8"), ("f16", 64, 16, "int8"), ("bf16", 128, 3, "e4m3")])
def test_few_rows_beside_many(vtlib, paged, dtype, d_head, group, code, window):
    """A batch that goes to both kernels."""
    lens = [(i * 7919) % 300 if i % 7 else -1 for i in range(120)]
    rows = [1 + i % 3 if i % 5 else 0 for i in range(120)]
    lens[60], rows[60] = 200, 60
    c = MxCache(vtlib, lens, rows, code, dtype, 2, d_head, 16, "pos")
    check(vtlib, paged, c, "prefill", 2 * group, window)


@pytest.mark.parametrize("dtype,code", KINDS)
def test_many_short_sequences(vtlib, paged, dtype, code):
    c = MxCache(vtlib, [i % 66 - 1 for i in range(700)], [1] * 700, code, dtype, 4, 64, 16)
    check(vtlib, paged, c, "decode", 8)


@pytest.mark.parametrize("call", ["decode", "prefill"])
@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_scale_zero_and_large(vtlib, paged, call, code):
    for seed, dtype, scale in ((0, "f16", 0.0), (1, "bf16", 16.0)):
        c = MxCache(vtlib, [0, 77, 200], [1] * 3 if call == "decode" else [150, 3, 40], code, dtype, 2, 64, 16, seed=seed)
        check(vtlib, paged, c, call, 4, scale=scale)


@pytest.mark.parametrize("std", [2.0 ** -13, 2.0 ** -6, 2.0 ** 10])
@pytest.mark.parametrize("dtype,code", KINDS)
def test_small_and_large_values(vtlib, paged, dtype, code, std):
    """Scales near the ends of what fp16's entries have (codes below its normal numbers among them), and far from 1."""
    for call, rows in (("decode", [1] * 3), ("prefill", [70, 3, 200])):
        c = MxCache(vtlib, [0, 77, 200], rows, code, dtype, 2, 128, 16, std=std)
        check(vtlib, paged, c, call, 8, scale=0.05 / std)


@pytest.mark.parametrize("dtype,code", KINDS)
def test_every_code_and_scale(vtlib, paged, dtype, code):
    """One position attends to itself alone: the output is its entry's values, each code with each scale."""
    vt = vtlib
    lo, hi = mx.RANGE[code, dtype]
    codes = [b for b in range(256) if not (code == "e4m3" and b & 127 == 127) and not (code == "int8" and b == 128)]
    for e in sorted({lo, lo + 1, -14, -10, -1, 0, 3, hi - 1, hi}):
        c = MxCache(vt, [0] * 4, [1] * 4, code, dtype, 1, 64, 8)
        want = torch.zeros(4, 1, 64, dtype=torch.float64, device="cuda")
        for b in range(4):
            row = torch.tensor((codes[64 * b:] + codes)[:64], dtype=torch.uint8, device="cuda")
            page = int(c.tables[b, 0])
            for x, s in zip(c.codes, c.scales):
                x.view(torch.uint8)[page, 0, 0] = row
                s[page, 0, 0] = torch.tensor([e + 127, min(e + 1, hi) + 127], dtype=torch.uint8)
            want[b, 0] = mx.decode(row.view(mx.CODES[code])[None], c.scales[1][page, 0, 0][None])[0]
        q = torch.zeros(4, 1, 64, dtype=TYPE[dtype], device="cuda")
        for call in ("decode", "prefill"):
            out = torch.empty_like(q)
            attend(vt, paged, c, call, q, out)
            assert torch.equal(out.double(), want)


@pytest.mark.parametrize("call", ["decode", "prefill"])
@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_nan_entries_that_nothing_attends_to(vtlib, paged, call, code):
    """A NaN entry reaches the rows that attend to it, through K and through V, and no other sequence; behind the window or the
    length it reaches nothing."""
    vt = vtlib
    c = MxCache(vt, [100, 60], [1, 1] if call == "decode" else [1, 1], code, "f16", 1, 64, 16)
    q = c.rows(2)
    whole, out = torch.empty_like(q), torch.empty_like(q)
    attend(vt, paged, c, call, q, whole, window=50)
    for side in range(2):
        page, off = c.positions(0, 101)
        keep = c.scales[side].clone()
        c.scales[side][page[30], 0, off[30], 0] = 255  # behind the window
        attend(vt, paged, c, call, q, out, window=50)
        assert torch.equal(out, whole)
        attend(vt, paged, c, call, q, out)
        assert out[0, 0, :32].isnan().all() and torch.isfinite(out[1]).all() and (side == 1) == bool(torch.isfinite(out[0, 0, 32:]).all())
        c.scales[side].copy_(keep)


@pytest.mark.parametrize("call", ["decode", "prefill", "tiles"])
@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_bad_pages_and_overflow(vtlib, paged, call, code):
    """A page id that is not one of the pool's: its positions take no part.  A length past the table: the positions that it
    has are attended to."""
    vt = vtlib
    rows = [1, 1] if call != "tiles" else [1300, 1300]
    kv = 1 if call != "tiles" else 16
    c = MxCache(vt, [100, 60], rows, code, "f16", kv, 64, 16)
    q = c.rows(kv)
    out, whole = torch.empty_like(q), torch.empty_like(q)
    attend(vt, paged, c, call, q, whole)
    keep = c.tables.clone()
    for bad in (-1, c.k.shape[0], 2 ** 31 - 1, -2 ** 31):
        c.tables[0, 2] = bad
        attend(vt, paged, c, call, q, out)
        assert vt.vt_paged_status(paged, clear=True) == vt.VT_DEV_BAD_PAGE
        c.tables.copy_(keep)
        page, off = c.positions(0, 101)
        ok = [j for j in range(101) if not 32 <= j < 48]
        kk, vv = (t[page[ok], 0, off[ok]].double() for t in (c.k, c.v))
        ref = torch.softmax(q[0, 0].double() @ kk.T / 8, -1) @ vv
        s1 = c.starts_host[1]
        assert ((out[0, 0].double() - ref).abs() <= 2.0 ** -9 * vv.abs().max()).all() and torch.equal(out[s1:], whole[s1:])
    if call == "tiles":
        return
    for much in (c.tables.shape[1] * 16, 2 ** 31 - 1):
        c.lens[1] = much
        c.tables[1] = c.tables[0]
        attend(vt, paged, c, call, q, out)
        assert vt.vt_paged_status(paged, clear=True) == vt.VT_DEV_KV_OVERFLOW
        assert torch.equal(out[0], whole[0])
        c.tables.copy_(keep)
        c.lens[1] = 60


def test_results_repeat_bit_for_bit(vtlib, paged):
    vt = vtlib
    for call, rows in (("decode", [1] * 5), ("prefill", [4, 130, 9, 1, 300])):
        c = MxCache(vt, [3000, 77, 4097, 0, 900], rows, "e4m3", "f16", 2, 128, 16)
        q = c.rows(8)
        outs = [torch.empty_like(q) for _ in range(4)]
        for out in outs:
            attend(vt, paged, c, call, q, out)
        assert all(torch.equal(outs[0], o) for o in outs[1:])


@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_strided_rows_and_rows_behind_the_last(vtlib, paged, code):
    vt = vtlib
    c = MxCache(vt, [50, 0, 200], [4, 140, 9], code, "bf16", 2, 128, 32)
    n = c.n_rows
    wide = torch.randn(n + 5, 11, 128, generator=c.gen, device="cuda").bfloat16()
    big = torch.full((n + 5, 10, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    vt.vt_paged_prefill_mx(paged, c.pool, c.batch(vt), wide[:, 1:9], big[:, :8])
    ref, tol = attention(c, wide[:n, 1:9], 128 ** -0.5, 0)
    assert ((big[:n, :8].double() - ref).abs() <= tol).all() and (big[:, 8:] == 3.0).all() and (big[n:] == 3.0).all()


def test_offsets_past_32_bits(vtlib, paged):
    """Pages whose codes and scales lie more than 2^31 bytes into the pool."""
    vt, n, stride = vtlib, 6, 2 ** 29 + 16
    small = MxCache(vt, [70, 3], [2, 1], "int8", "f16", 1, 64, 16, spare=0)
    assert small.k.shape[0] == n
    far = []
    for t, entry in zip(small.codes + small.scales, (64, 64, 2, 2)):
        base = torch.full((5 * stride + 16 * 64,), 127, dtype=torch.uint8, device="cuda")
        s = base.as_strided((n, 1, 16, entry), (stride, 16 * entry, entry, 1))
        s.copy_(t.view(torch.uint8))
        far.append(s)
    pool = vt.make_paged_mx_pool(far[0].view(torch.int8), far[1].view(torch.int8), far[2], far[3], torch.float16)
    q = small.rows(2)
    out = torch.empty_like(q)
    vt.vt_paged_prefill_mx(paged, pool, small.batch(vt), q, out)
    ref, tol = attention(small, q, 0.125, 0)
    assert ((out.double() - ref).abs() <= tol).all()
    lens = torch.tensor([71, 3], dtype=torch.int32, device="cuda")
    batch = vt.make_paged_batch(small.tables, lens)
    vt.vt_paged_decode_mx(paged, pool, batch, q[1:], out[1:])
    assert ((out.double() - ref).abs() <= tol).all()
    vt.vt_paged_append_mx(paged, pool, batch, q[1:], q[1:, :1], q[1:, 1:], vt.make_qk_form(), out[1:])
    page, off = small.positions(0, 72)
    for i, x in ((0, q[1, 0]), (1, q[1, 1])):
        codes, scales = mx.encode(x, "int8", "f16")
        assert torch.equal(far[i][page[71], 0, off[71]].view(torch.int8).double(), codes)
        assert torch.equal(far[2 + i][page[71], 0, off[71]], scales)


@pytest.mark.parametrize("dtype,code", KINDS)
def test_a_conversation_in_a_graph_and_out_of_it(vtlib, paged, dtype, code):
    """Prompts appended and attended to in chunks, then tokens one by one, the tokens captured once and replayed: each row as
    the definition has it over what the pool then holds."""
    vt = vtlib
    n = 12
    c = MxCache(vt, [0, 0], [60 + n, 35 + n], code, dtype, 2, 64, 16)
    heads = 4
    rope = table(c.tables.shape[1] * 16, 64)
    gains = [(1 + 0.1 * torch.randn(64, generator=c.gen, device="cuda")).to(TYPE[dtype]) for _ in range(2)]
    form = vt.make_qk_form(rope, True, *gains)
    x = torch.randn(c.n_rows, heads + 4, 64, generator=c.gen, device="cuda").to(TYPE[dtype])
    qr, out = torch.empty_like(x[:, :heads]), torch.empty_like(x[:, :heads])
    chunks = ([40, 35], [20, 0])
    at = [0, 0]
    for rows in chunks:
        idx = torch.cat([torch.arange(c.starts_host[b] + at[b], c.starts_host[b] + at[b] + rows[b]) for b in range(2)]).cuda()
        lens = torch.tensor(at, dtype=torch.int32, device="cuda")
        starts = torch.tensor([0, rows[0], sum(rows)], dtype=torch.int32, device="cuda")
        batch = vt.make_paged_batch(c.tables, lens, starts)
        part, q1, o1 = x[idx], torch.empty_like(x[idx, :heads]), torch.empty_like(x[idx, :heads])
        vt.vt_paged_append_mx(paged, c.pool, batch, part[:, :heads], part[:, heads:heads + 2], part[:, heads + 2:], form, q1)
        vt.vt_paged_prefill_mx(paged, c.pool, batch, q1, o1)
        qr[idx], out[idx] = q1, o1
        at = [a + r for a, r in zip(at, rows)]
    lens = torch.tensor(at, dtype=torch.int32, device="cuda")
    batch = vt.make_paged_batch(c.tables, lens)
    part = torch.empty_like(x[:2])
    q1, o1 = torch.empty_like(part[:, :heads]), torch.empty_like(part[:, :heads])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        vt.vt_paged_append_mx(paged, c.pool, batch, part[:, :heads], part[:, heads:heads + 2], part[:, heads + 2:], form, q1)
        vt.vt_paged_decode_mx(paged, c.pool, batch, q1, o1)
        lens.add_(1)
    with torch.cuda.stream(side):
        for i in range(n):
            idx = torch.tensor([c.starts_host[b] + at[b] + i for b in range(2)], device="cuda")
            part.copy_(x[idx])
            graph.replay()
            qr[idx], out[idx] = q1, o1
    side.synchronize()
    assert vt.vt_paged_status(paged) == 0 and lens.tolist() == [a + n for a in at]
    # what the pool holds now, as values; queries as they were formed
    for i, t in enumerate((c.k, c.v)):
        t.copy_(mx.decode(c.codes[i], c.scales[i]).masked_fill(~c.live[:, None, :, None], float("nan")))
    ref, tol = attention(c, qr, 0.125, 0)
    assert ((out.double() - ref).abs() <= tol).all()
    for b in range(2):
        rows = slice(c.starts_host[b], c.starts_host[b + 1])
        y, near = formed(x[rows, :heads], gains[0], rope, torch.arange(c.rows_host[b], device="cuda"), 64, True)
        assert ((qr[rows].double() - y).abs() <= U[dtype] * y.abs() + 2.0 ** -19 * near + 2.0 ** -25).all()


def test_two_workspaces_on_two_streams(vtlib):
    """Two calls at once, each with its own vt_paged."""
    vt = vtlib
    c = MxCache(vt, [9000, 300, 4000], [1, 1, 1], "e4m3", "bf16", 2, 128, 16)
    d = MxCache(vt, [3000, 0], [100, 260], "int8", "bf16", 4, 128, 16)
    qc, qd = c.rows(8), d.rows(8)
    gs, streams = [vt.vt_paged_create() for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(qc), torch.empty_like(qd)]
    torch.cuda.synchronize()
    for _ in range(20):
        vt.vt_paged_decode_mx(gs[0], c.pool, c.batch(vt, False), qc, outs[0], stream=streams[0])
        vt.vt_paged_prefill_mx(gs[1], d.pool, d.batch(vt), qd, outs[1], stream=streams[1])
    torch.cuda.synchronize()
    for cache, q, out in ((c, qc, outs[0]), (d, qd, outs[1])):
        ref, tol = attention(cache, q, 1 / math.sqrt(128), 0)
        assert ((out.double() - ref).abs() <= tol).all()
    for g in gs:
        assert vt.vt_paged_status(g) == 0
        vt.vt_paged_destroy(g)


def spread(vt, c, pos=16, head=48, page=112, scale_head=16, scale_page=64):
    """The cache's pool again, its entries, heads and pages further apart; what lies between is 0x7f and 255."""
    out = []
    n, K, P, d = c.codes[0].shape
    for t in c.codes:
        ps, hs = d + pos, P * (d + pos) + head
        base = torch.full((n * (K * hs + page),), 0x7f, dtype=torch.uint8, device="cuda")
        s = base.as_strided((n, K, P, d), (K * hs + page, hs, ps, 1))
        s.copy_(t.view(torch.uint8))
        out.append(s.view(t.dtype))
    for t in c.scales:
        nb = t.shape[3]
        hs = P * nb + scale_head
        base = torch.full((n * (K * hs + scale_page),), 255, dtype=torch.uint8, device="cuda")
        s = base.as_strided(t.shape, (K * hs + scale_page, hs, nb, 1))
        s.copy_(t)
        out.append(s)
    return vt.make_paged_mx_pool(*out, TYPE[c.dtype])


@pytest.mark.parametrize("dtype,code", KINDS)
@pytest.mark.parametrize("d_head,page", [(128, 16), (64, 64), (128, 8), (64, 256)])
def test_pools_with_gaps(vtlib, paged, dtype, code, d_head, page):
    vt = vtlib
    for call, lens, rows, heads in (("decode", LENS, [1] * len(LENS), 6), ("prefill", [2000, 0, 700], [300, 513, 40], 48)):
        c = MxCache(vt, lens, rows, code, dtype, 3 if call == "decode" else 12, d_head, page)
        q = c.rows(heads)
        want, out = torch.empty_like(q), torch.empty_like(q)
        attend(vt, paged, c, call, q, want)
        c.pool = spread(vt, c)
        attend(vt, paged, c, call, q, out)
        assert torch.equal(out.view(torch.int16), want.view(torch.int16))
        ref, tol = attention(c, q, d_head ** -0.5, 0)
        tol = tol + TINY[dtype] + 2.0 ** -36 * c.k.shape[0] * page * c.v.masked_fill(c.v.isnan(), 0.0).double().abs().max()
        assert ((out.double() - ref).abs() <= tol).all()
        assert vt.vt_paged_status(paged) == 0


def test_tiles_with_offsets_past_32_bits(vtlib, paged):
    """Pages far apart, and enough rows for the tiles' kernel: the same bits as from pages side by side."""
    vt, stride = vtlib, 2 ** 27 + 16
    c = MxCache(vt, [70, 3], [300, 40], "e4m3", "f16", 1, 128, 16, spare=0)
    n = c.k.shape[0]
    assert (n - 1) * stride > 2 ** 31
    far = []
    for t, entry in zip(c.codes + c.scales, (128, 128, 4, 4)):
        base = torch.full(((n - 1) * stride + 16 * 128,), 127, dtype=torch.uint8, device="cuda")
        s = base.as_strided((n, 1, 16, entry), (stride, 16 * entry, entry, 1))
        s.copy_(t.view(torch.uint8))
        far.append(s)
    q = c.rows(16)
    want, out = torch.empty_like(q), torch.empty_like(q)
    attend(vt, paged, c, "prefill", q, want)
    plain = torch.empty_like(q)
    vt.vt_paged_prefill(paged, c.plain, c.batch(vt), q, plain)
    assert torch.equal(want.view(torch.int16), plain.view(torch.int16))  # the tiles' kernel took it
    c.pool = vt.make_paged_mx_pool(far[0].view(torch.float8_e4m3fn), far[1].view(torch.float8_e4m3fn), far[2], far[3], torch.float16)
    attend(vt, paged, c, "prefill", q, out)
    assert torch.equal(out.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("d_head", [64, 128])
def test_as_many_sequences_as_a_batch_takes(vtlib, paged, d_head):
    """16384 slots of one position and more, most of them idle or without rows: one batch through all three calls."""
    vt, n = vtlib, 16384
    lens = [(i * 37) % 20 if i % 61 == 0 else -1 for i in range(n)]
    for rows in ([1] * n, [3 if i % 61 == 0 else 0 for i in range(n)]):
        c = MxCache(vt, lens, rows, "int8", "bf16", 1, d_head, 8)
        q = c.rows(2)
        out = torch.full_like(q, 7.0)
        one = rows[1] == 1
        attend(vt, paged, c, "decode" if one else "prefill", q, out)
        live = [b for b in range(n) if lens[b] >= 0]
        for b in live[::20] + live[-1:]:
            s0, r, p = c.starts_host[b], rows[b], lens[b]
            page, off = c.positions(b, p + r)
            k, v = (t[page, 0, off].double() for t in (c.k, c.v))
            hide = torch.arange(p + r, device="cuda") > torch.arange(p, p + r, device="cuda")[:, None]
            for h in range(2):
                w = torch.softmax((q[s0:s0 + r, h].double() @ k.T * d_head ** -0.5).masked_fill(hide, -math.inf), -1)
                o, a = w @ v, w @ v.abs()
                assert ((out[s0:s0 + r, h].double() - o).abs() <= U["bf16"] * o.abs() + (U["bf16"] + 2.0 ** -16) * a + 2.0 ** -30).all()
        idle = torch.tensor([c.starts_host[b] for b in range(n) if lens[b] < 0 and rows[b]][::50], dtype=torch.long, device="cuda")
        assert not out[idle].any() and vt.vt_paged_status(paged) == 0


@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_captured_prefill_at_other_lengths(vtlib, paged, code):
    """One capture of append and prefill, replayed with other lengths, tables and row starts than it was captured with."""
    vt, H, K, d = vtlib, 8, 2, 128
    caches = [MxCache(vt, lens, rows, code, "bf16", K, d, 16, seed=i) for i, (lens, rows) in enumerate((
        ([200, 0, 33], [100, 300, 7]), ([0, 900, -1], [7, 250, 150]), ([31, 64, 500], [1, 405, 1])))]
    most = max(c.codes[0].shape[0] for c in caches)
    per = max(c.tables.shape[1] for c in caches)
    codes = [torch.zeros(most, K, 16, d, dtype=torch.uint8, device="cuda").view(mx.CODES[code]) for _ in range(2)]
    scales = [torch.full((most, K, 16, d // 32), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    pool = vt.make_paged_mx_pool(*codes, *scales, torch.bfloat16)
    tables = torch.full((3, per), -1, dtype=torch.int32, device="cuda")
    lens, starts = torch.full((3,), -1, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    x = torch.zeros(407, H + 2 * K, d, dtype=torch.bfloat16, device="cuda")
    q, out = torch.zeros_like(x[:, :H]), torch.zeros_like(x[:, :H])
    form = vt.make_qk_form(table(per * 16, 128))
    batch = vt.make_paged_batch(tables, lens, starts)

    def calls():
        vt.vt_paged_append_mx(paged, pool, batch, x[:, :H], x[:, H:H + K], x[:, H + K:], form, q)
        vt.vt_paged_prefill_mx(paged, pool, batch, q, out)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls()
    for c in caches:
        with torch.cuda.stream(side):
            n = c.codes[0].shape[0]
            for dst, src in zip(codes + scales, c.codes + c.scales):
                dst.view(torch.uint8)[:n] = src.view(torch.uint8)
            tables.fill_(-1)
            tables[:, :c.tables.shape[1]] = c.tables
            lens.copy_(c.lens)
            starts.copy_(c.starts)
            x.normal_(generator=c.gen)
            out.fill_(7.0)
            graph.replay()
        side.synchronize()
        got, gq, pools = out.clone(), q.clone(), [t.clone() for t in codes + scales]
        calls()  # the same, not captured
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.equal(gq, q)
        assert all(torch.equal(s.view(torch.uint8), t.view(torch.uint8)) for s, t in zip(pools, codes + scales))
        for i, t in enumerate((c.k, c.v)):
            t.copy_(mx.decode(codes[i][:n], scales[i][:n]).masked_fill(~c.live[:, None, :, None], float("nan")))
        ref, tol = attention(c, q[:c.n_rows], d ** -0.5, 0)
        assert ((out[:c.n_rows].double() - ref).abs() <= tol + 2.0 ** -30).all() and (out[c.n_rows:] == 7.0).all()
        assert vt.vt_paged_status(paged) == 0


@pytest.mark.parametrize("call", ["decode", "prefill"])
@pytest.mark.parametrize("dtype,code", KINDS)
def test_largest_scale_and_scores_of_zero(vtlib, paged, call, dtype, code):
    """Keys of zeros, and large queries: every score is 0 whatever the scale, and the output the mean of the values."""
    vt = vtlib
    c = MxCache(vt, [40, 3], [1, 1] if call == "decode" else [5, 90], code, dtype, 1, 64, 16)
    live = c.live[:, None, :, None]
    c.codes[0].view(torch.uint8).masked_fill_(live, 0)
    c.k.masked_fill_(live, 0.0)
    q = c.rows(4).mul_(2.0 ** 13 if dtype == "f16" else 2.0 ** 40)
    for scale in (0.0, 1.0, 3.4028234663852886e38):
        out = torch.empty_like(q)
        attend(vt, paged, c, call, q, out, scale)
        ref, tol = attention(c, torch.zeros_like(q), 1.0, 0)
        assert ((out.double() - ref).abs() <= tol + TINY[dtype]).all()
