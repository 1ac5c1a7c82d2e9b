"""The paged KV cache (vt_paged_append, vt_paged_decode, vt_paged_prefill) against plain definitions in
64 bits, one sequence after another.

Tolerances, by the arithmetic alone.  u is half a unit in the last place of the type relative to its
value: 2^-11 (fp16) or 2^-8 (bf16).  An attention weight p may be rounded to the type before it meets
v, and the output is rounded once, so with A = sum_j softmax_j |v_j|
    |error| <= u |o| + u A + 2^-16 A + n 2^-25 max|v| (fp16 only: weights below 2^-14 of the row's
    largest are subnormal, each up to 2^-25 off),
where 2^-16 A covers the fp32 scores, exponentials and sums of these sizes.  The rotation computes each
value with two fp32 products and one sum and rounds once: u |x'| + 2^-22 (|a| + |b|), plus half the
type's smallest step.
"""
from __future__ import annotations

import ctypes
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TYPE = {"f16": torch.float16, "bf16": torch.bfloat16}
TINY = {"f16": 2.0 ** -25, "bf16": 0.0}


@pytest.fixture()
def paged(vtlib):
    g = vtlib.vt_paged_create()
    yield g
    vtlib.vt_paged_destroy(g)


class Cache:
    """A pool whose pages are dealt out in random order; entries that no sequence holds are NaN, table
    entries past a sequence's last page are -1."""

    def __init__(self, vt, lens, rows, dtype="f16", kv_heads=2, d_head=64, page=16, order="head", seed=0, std=1.0, spare=2):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.lens_host, self.rows_host, self.page, self.dtype = list(lens), list(rows), page, dtype
        held = [p + r if p >= 0 else 0 for p, r in zip(lens, rows)]
        pages = [-(-h // page) for h in held]
        n_pages, per = sum(pages) + spare, max(1, max(pages, default=1))
        perm = torch.randperm(n_pages, generator=gen, device="cuda").tolist()
        tables, at = torch.full((len(lens), per), -1, dtype=torch.int32), 0
        shape = (n_pages, kv_heads, page, d_head) if order == "head" else (n_pages, page, kv_heads, d_head)
        self.k = torch.randn(shape, generator=gen, device="cuda").mul_(std).to(TYPE[dtype])
        self.v = torch.randn(shape, generator=gen, device="cuda").mul_(std).to(TYPE[dtype])
        if order == "pos":
            self.k, self.v = self.k.permute(0, 2, 1, 3), self.v.permute(0, 2, 1, 3)
        live = torch.zeros(n_pages, page, dtype=torch.bool)
        for b, n in enumerate(pages):
            tables[b, :n] = torch.tensor(perm[at:at + n], dtype=torch.int32)
            for j in range(n):
                live[perm[at + j], :max(0, min(page, held[b] - j * page))] = True
            at += n
        self.live = live.cuda()
        for t in (self.k, self.v):
            t.masked_fill_(~self.live[:, None, :, None], float("nan"))
        self.tables = tables.cuda()
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.starts_host = [0]
        for r in rows:
            self.starts_host.append(self.starts_host[-1] + r)
        self.starts = torch.tensor(self.starts_host, dtype=torch.int32, device="cuda")
        self.n_rows, self.gen = self.starts_host[-1], gen
        self.pool = vt.make_paged_pool(self.k, self.v)
        self.kv_heads, self.d_head = kv_heads, d_head

    def batch(self, vt, starts=True):
        return vt.make_paged_batch(self.tables, self.lens, self.starts if starts else None)

    def rows(self, heads, std=1.0):
        return torch.randn(self.n_rows, heads, self.d_head, generator=self.gen, device="cuda").mul_(std).to(TYPE[self.dtype])

    def positions(self, b, n):
        pos = torch.arange(n, device="cuda")
        return self.tables[b].long()[pos // self.page], pos % self.page


def attention(c, q, scale, window):
    """(output, bound of its error) in 64 bits."""
    H, G = q.shape[1], q.shape[1] // c.kv_heads
    out, tol = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    for b, (p, r) in enumerate(zip(c.lens_host, c.rows_host)):
        if p < 0 or r == 0:
            continue
        page, off = c.positions(b, p + r)
        k, v = c.k[page, :, off].double(), c.v[page, :, off].double()  # [n, K, d]
        pos, me = torch.arange(p + r, device="cuda"), torch.arange(p, p + r, device="cuda")[:, None]
        hide = pos > me
        if window:
            hide = hide | (pos <= me - window)
        s0 = c.starts_host[b]
        for h in range(H):
            w = torch.softmax((q[s0:s0 + r, h].double() @ k[:, h // G].T * scale).masked_fill(hide, -math.inf), -1)
            o, a = w @ v[:, h // G], w @ v[:, h // G].abs()
            u = U[c.dtype]
            out[s0:s0 + r, h] = o
            tol[s0:s0 + r, h] = u * o.abs() + (u + 2.0 ** -16) * a + TINY[c.dtype] * (p + r) * v.abs().max()
    return out, tol


def check_attention(vt, g, c, call, heads, window=0, scale=None, q=None):
    q = c.rows(heads) if q is None else q
    out = torch.full_like(q, 7.0)
    scale = c.d_head ** -0.5 if scale is None else scale
    if call == "decode":
        vt.vt_paged_decode(g, c.pool, c.batch(vt, starts=False), q, out, scale, window)
    else:
        vt.vt_paged_prefill(g, c.pool, c.batch(vt), q, out, scale, window)
    ref, tol = attention(c, q, scale, window)
    far = (out.double() - ref).abs()
    assert torch.isfinite(out).all()
    assert (far <= tol).all(), f"{float((far / tol.clamp(min=1e-30)).max())} times the bound"
    assert vt.vt_paged_status(g) == 0


LENS = [0, 1, 14, 15, 16, 17, -1, 62, 63, 64, 65, 127, 128, 300, -1, 1000]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d_head,kv_heads,group,page,order", [
    (64, 8, 1, 16, "head"), (128, 2, 4, 16, "pos"), (128, 1, 1, 8, "head"), (64, 3, 2, 1, "pos"),
    (128, 2, 8, 64, "head"), (128, 1, 12, 32, "pos"), (64, 1, 16, 128, "head"), (128, 2, 3, 256, "head"),
    (64, 1, 71, 2, "head"), (128, 4, 5, 1024, "pos")])
def test_decode(vtlib, paged, dtype, d_head, kv_heads, group, page, order):
    c = Cache(vtlib, LENS, [1] * len(LENS), dtype, kv_heads, d_head, page, order)
    check_attention(vtlib, paged, c, "decode", kv_heads * group)


@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 100, 5000])
@pytest.mark.parametrize("call", ["decode", "prefill"])
def test_window(vtlib, paged, call, window):
    rows = [1] * len(LENS) if call == "decode" else [1 + 19 * (i % 4) for i in range(len(LENS))]
    c = Cache(vtlib, LENS, rows, "f16", 2, 128, 32, "pos", seed=window)
    check_attention(vtlib, paged, c, call, 4, window)


@pytest.mark.parametrize("n", [1, 2, 40, 333, 1100])
def test_decode_batch_sizes(vtlib, paged, n):
    """Few and many sequences, most of them short."""
    lens = [(i * 7919) % 97 if i % 11 else -1 for i in range(n)]
    lens[-1] = 700
    check_attention(vtlib, paged, Cache(vtlib, lens, [1] * n, "f16", 1, 64, 16), "decode", 2)


@pytest.mark.parametrize("dtype,d_head,kv_heads,group,length", [
    ("f16", 128, 1, 8, 40000), ("bf16", 128, 2, 4, 33333), ("f16", 64, 3, 1, 50001), ("bf16", 64, 1, 20, 20000)])
def test_decode_long(vtlib, paged, dtype, d_head, kv_heads, group, length):
    """One sequence over the whole GPU, beside a short and an idle one."""
    c = Cache(vtlib, [length, 3, -1], [1, 1, 1], dtype, kv_heads, d_head, 64)
    check_attention(vtlib, paged, c, "decode", kv_heads * group)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d_head,kv_heads,group,page,order", [
    (64, 8, 1, 16, "head"), (128, 2, 4, 16, "pos"), (128, 1, 1, 8, "head"), (64, 3, 2, 1, "pos"),
    (128, 2, 8, 64, "head"), (128, 1, 12, 32, "pos"), (128, 2, 3, 256, "head"), (64, 1, 71, 2, "head"),
    (128, 1, 128, 128, "pos")])
def test_prefill(vtlib, paged, dtype, d_head, kv_heads, group, page, order):
    """Rows from none to more than two tiles, behind nothing and behind a history; an idle slot with rows."""
    lens = [0, 0, 0, 5, 127, 128, 129, -1, 300, 0, 1000, 63]
    rows = [1, 0, 130, 1, 64, 128, 7, 33, 65, 300, 2, 129]
    c = Cache(vtlib, lens, rows, dtype, kv_heads, d_head, page, order)
    check_attention(vtlib, paged, c, "prefill", kv_heads * group)


@pytest.mark.parametrize("length,rows", [(20000, 1), (20000, 4), (9000, 130), (0, 1500)])
def test_prefill_long(vtlib, paged, length, rows):
    """Few rows behind a long history (the history is split over the GPU), and a long prompt."""
    c = Cache(vtlib, [length, 0], [rows, 3], "bf16", 2, 128, 64)
    check_attention(vtlib, paged, c, "prefill", 8)


@pytest.mark.parametrize("call", ["decode", "prefill"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("std", [0.0, 0.05, 4.0])
def test_score_ranges(vtlib, paged, call, dtype, std):
    """Equal scores, nearly equal ones, and scores where one key takes all the weight."""
    lens = [0, 100, 513]
    c = Cache(vtlib, lens, [1] * 3 if call == "decode" else [140, 3, 70], dtype, 2, 128, 16, std=1.0)
    q = c.rows(8, std)
    check_attention(vtlib, paged, c, call, 8, scale=1.0, q=q)


@pytest.mark.parametrize("call", ["decode", "prefill"])
def test_rising_scores(vtlib, paged, call):
    """Every key scores higher than the one before it: the running maximum moves at each."""
    c = Cache(vtlib, [700], [1 if call == "decode" else 150], "f16", 1, 64, 16)
    page, off = c.positions(0, 700 + c.rows_host[0])
    c.k[page, 0, off] = (torch.arange(len(page), device="cuda")[:, None] / 64).half().expand(-1, 64)
    q = torch.ones(c.n_rows, 2, 64, dtype=torch.float16, device="cuda")
    check_attention(vtlib, paged, c, call, 2, scale=0.25, q=q)


@pytest.mark.parametrize("call", ["decode", "prefill"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_infinities_and_nan_stay_in_their_row(vtlib, paged, call, dtype):
    """A key that scores -inf takes no weight; a NaN key or value reaches the rows that attend to it and
    no other sequence."""
    c = Cache(vtlib, [40, 40, 40], [1] * 3 if call == "decode" else [5, 5, 5], dtype, 1, 64, 16)
    q = c.rows(1).abs()
    page, off = c.positions(0, 45 if call == "prefill" else 41)
    c.k[page[3], 0, off[3]] = float("-inf")
    page2, off2 = c.positions(2, 41)
    c.v[page2[7], 0, off2[7]] = float("nan")
    out = torch.empty_like(q)
    if call == "decode":
        vtlib.vt_paged_decode(paged, c.pool, c.batch(vtlib, False), q, out)
    else:
        vtlib.vt_paged_prefill(paged, c.pool, c.batch(vtlib), q, out)
    n = c.rows_host[0]
    assert torch.isfinite(out[:2 * n]).all() and torch.isnan(out[2 * n:]).all()
    c.v[page2[7], 0, off2[7]] = 0.0
    ref, tol = attention(c, q, 0.125, 0)
    assert ((out.double() - ref).abs() <= tol)[:2 * n].all()


def rotated(x, rope, pos):
    d = x.shape[-1]
    a, b = x.double()[..., :d // 2], x.double()[..., d // 2:]
    c, s = rope[pos].double()[:, None, :, 0], rope[pos].double()[:, None, :, 1]
    return torch.cat((a * c - b * s, b * c + a * s), -1), torch.cat((a.abs() + b.abs(),) * 2, -1)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d_head,heads,kv_heads,page,order,fused,one_each", [
    (64, 8, 8, 16, "head", True, False), (128, 32, 8, 32, "pos", True, False), (128, 3, 1, 1, "head", False, False),
    (64, 71, 1, 256, "pos", True, False), (128, 8, 2, 64, "head", False, True), (64, 1, 1, 8, "pos", True, True)])
def test_append(vtlib, paged, dtype, d_head, heads, kv_heads, page, order, fused, one_each):
    vt = vtlib
    lens = [0, 1, 15, 16, 100, -1, 255, 0, 31, 7]
    rows = [1] * 10 if one_each else [3, 0, 1, 17, 40, 2, 1, 260, 33, 0]
    c = Cache(vt, lens, rows, dtype, kv_heads, d_head, page, order, std=2.0)
    if fused:
        qkv = c.rows(heads + 2 * kv_heads, 2.0)
        q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
    else:
        q, k, v = c.rows(heads, 2.0), c.rows(kv_heads, 2.0), c.rows(kv_heads, 2.0)
    rope = torch.empty(400, d_head // 2, 2, device="cuda")
    vt.vt_rope_table(rope, 1e4)
    ang = torch.arange(400, device="cuda").double()[:, None] * 1e4 ** (-2.0 * torch.arange(d_head // 2, device="cuda").double() / d_head)
    assert (rope.double() - torch.stack((ang.cos(), ang.sin()), -1)).abs().max() <= 2.0 ** -24
    kw, vw = c.k.clone(), c.v.clone()
    q_out = torch.full((c.n_rows, heads, d_head), 7.0, dtype=TYPE[dtype], device="cuda")
    vt.vt_paged_append(paged, c.pool, c.batch(vt, not one_each), q, k, v, rope, q_out)
    assert vt.vt_paged_status(paged) == 0
    u, tiny = U[dtype], 2.0 ** -25
    for b, (p, r) in enumerate(zip(lens, rows)):
        at = slice(c.starts_host[b], c.starts_host[b] + r)
        if p < 0:
            assert not q_out[at].any()
            continue
        pos = torch.arange(p, p + r, device="cuda")
        ref, mag = rotated(q[at], rope, pos)
        assert ((q_out[at].double() - ref).abs() <= u * ref.abs() + 2.0 ** -22 * mag + tiny).all()
        ref, mag = rotated(k[at], rope, pos)
        pg, off = c.tables[b].long()[pos // page], pos % page
        assert ((c.k[pg, :, off].double() - ref).abs() <= u * ref.abs() + 2.0 ** -22 * mag + tiny).all()
        assert torch.equal(c.v[pg, :, off], v[at])
        kw[pg, :, off], vw[pg, :, off] = c.k[pg, :, off], v[at]
    # nothing else of the pool has changed
    assert torch.equal(torch.nan_to_num(c.k, 9.0), torch.nan_to_num(kw, 9.0))
    assert torch.equal(torch.nan_to_num(c.v, 9.0), torch.nan_to_num(vw, 9.0))


def test_append_in_place(vtlib, paged):
    vt = vtlib
    c = Cache(vt, [9], [50], "bf16", 2, 128, 16)
    q, k, v = c.rows(8), c.rows(2), c.rows(2)
    rope = torch.empty(64, 64, 2, device="cuda")
    vt.vt_rope_table(rope, 5e5)
    out = torch.empty_like(q)
    vt.vt_paged_append(paged, c.pool, c.batch(vt), q, k, v, rope, out)
    vt.vt_paged_append(paged, c.pool, c.batch(vt), q, k, v, rope, q)
    assert torch.equal(q, out)


def test_append_then_attend_on_a_side_stream_and_in_a_graph(vtlib, paged):
    """Tokens one after another through append and decode, replayed from one graph, equal a prefill of
    the same rows; lengths are advanced on the device."""
    vt, n = vtlib, 37
    c = Cache(vt, [20, 5], [n, n], "f16", 2, 64, 16)
    q, k, v = c.rows(4), c.rows(2), c.rows(2)
    rope = torch.empty(64, 32, 2, device="cuda")
    vt.vt_rope_table(rope, 1e4)
    qr, want = torch.empty_like(q), torch.empty_like(q)
    vt.vt_paged_append(paged, c.pool, c.batch(vt), q, k, v, rope, qr)
    vt.vt_paged_prefill(paged, c.pool, c.batch(vt), qr, want)
    torch.cuda.synchronize()
    for t in (c.k, c.v):  # forget the appended rows again
        for b, p in enumerate(c.lens_host):
            page, off = c.positions(b, p + n)
            t[page[p:], :, off[p:]] = float("nan")
    side = torch.cuda.Stream()
    x = torch.empty(2, 8, 64, dtype=torch.float16, device="cuda")
    qo, out = torch.empty(2, 4, 64, dtype=torch.float16, device="cuda"), torch.empty(2, 4, 64, dtype=torch.float16, device="cuda")
    got = torch.empty_like(want)
    batch = c.batch(vt, starts=False)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        vt.vt_paged_append(paged, c.pool, batch, x[:, :4], x[:, 4:6], x[:, 6:], rope, qo)
        vt.vt_paged_decode(paged, c.pool, batch, qo, out)
        c.lens.add_(1)
    with torch.cuda.stream(side):
        for i in range(n):
            at = torch.tensor([i, n + i], device="cuda")
            x.copy_(torch.cat((q[at], k[at], v[at]), 1))
            graph.replay()
            got[at] = out
    side.synchronize()
    assert vt.vt_paged_status(paged) == 0 and c.lens.tolist() == [20 + n, 5 + n]
    ref, tol = attention(c, qr, 0.125, 0)
    assert ((got.double() - ref).abs() <= tol).all() and ((want.double() - ref).abs() <= tol).all()


def test_results_repeat_bit_for_bit(vtlib, paged):
    vt = vtlib
    for call, rows in (("decode", [1] * 5), ("prefill", [4, 130, 9, 1, 300])):
        c = Cache(vt, [3000, 77, 4097, 0, 900], rows, "f16", 2, 128, 16)
        q = c.rows(8)
        outs = []
        for _ in range(4):
            out = torch.empty_like(q)
            if call == "decode":
                vt.vt_paged_decode(paged, c.pool, c.batch(vt, False), q, out)
            else:
                vt.vt_paged_prefill(paged, c.pool, c.batch(vt), q, out)
            outs.append(out)
        assert all(torch.equal(outs[0], o) for o in outs[1:])


def test_shared_pages(vtlib, paged):
    """Two sequences whose tables begin with the same pages."""
    vt = vtlib
    c = Cache(vt, [95, 111, 100], [1, 1, 1], "f16", 2, 64, 16)
    c.tables[1, :4] = c.tables[0, :4]
    check_attention(vt, paged, c, "decode", 4)


def test_strided_rows_and_outputs(vtlib, paged):
    vt = vtlib
    c = Cache(vt, [50, 0, 200], [4, 140, 9], "bf16", 2, 128, 32)
    wide = c.rows(11)
    q, big = wide[:, 1:9], torch.full((c.n_rows, 10, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    vt.vt_paged_prefill(paged, c.pool, c.batch(vt), q, big[:, :8])
    ref, tol = attention(c, q, 128 ** -0.5, 0)
    assert ((big[:, :8].double() - ref).abs() <= tol).all() and (big[:, 8:] == 3.0).all()


def test_offsets_past_32_bits(vtlib, paged):
    """Pages whose entries lie more than 2^31 elements into the pool."""
    vt, n, stride = vtlib, 6, 2 ** 29 + 8
    base = [torch.full((5 * stride + 16 * 64,), float("nan"), dtype=torch.float16, device="cuda") for _ in range(2)]
    k, v = (t.as_strided((n, 1, 16, 64), (stride, 64, 64, 1)) for t in base)
    small = Cache(vt, [70, 3], [2, 1], "f16", 1, 64, 16, spare=0)
    assert small.k.shape[0] == n
    k.copy_(small.k)
    v.copy_(small.v)
    q = small.rows(2)
    out = torch.empty_like(q)
    vt.vt_paged_prefill(paged, vt.make_paged_pool(k, v), small.batch(vt), q, out)
    ref, tol = attention(small, q, 0.125, 0)
    assert ((out.double() - ref).abs() <= tol).all()
    small.rows_host, small.lens_host = [1, 1], [71, 3]
    lens = torch.tensor([71, 3], dtype=torch.int32, device="cuda")
    vt.vt_paged_decode(paged, vt.make_paged_pool(k, v), vt.make_paged_batch(small.tables, lens), q[1:], out[1:])
    assert ((out.double() - ref).abs() <= tol).all()
    rope = torch.empty(128, 32, 2, device="cuda")
    vt.vt_rope_table(rope, 1e4)
    vt.vt_paged_append(paged, vt.make_paged_pool(k, v), vt.make_paged_batch(small.tables, lens), q[1:], q[1:, :1], q[1:, 1:],
                       rope, out[1:])
    page, off = small.positions(0, 72)
    assert torch.equal(v[page[71], 0, off[71]], q[1, 1])


def test_bad_pages_and_overflow_are_flagged_and_skipped(vtlib, paged):
    """A page id that is not one of the pool's: its positions take no part.  A length past the table: the
    positions that it has are attended to."""
    vt = vtlib
    for call in ("decode", "prefill"):
        c = Cache(vt, [100, 60], [1, 1], "f16", 1, 64, 16)
        q = c.rows(2)
        out, whole = torch.empty_like(q), torch.empty_like(q)

        def run(dst):
            if call == "decode":
                vt.vt_paged_decode(paged, c.pool, c.batch(vt, False), q, dst)
            else:
                vt.vt_paged_prefill(paged, c.pool, c.batch(vt), q, dst)

        run(whole)
        keep = c.tables.clone()
        for bad in (-1, c.k.shape[0], 2 ** 31 - 1, -2 ** 31):
            c.tables[0, 2] = bad
            run(out)
            assert vt.vt_paged_status(paged, clear=True) == vt.VT_DEV_BAD_PAGE
            page, off = c.positions(0, 101)
            ok = [j for j in range(101) if not 32 <= j < 48]
            kk, vv = (t[page[ok], 0, off[ok]].double() for t in (c.k, c.v))
            ref = torch.softmax(q[0].double() @ kk.T / 8, -1) @ vv
            assert ((out[0].double() - ref).abs() <= 2.0 ** -9 * vv.abs().max()).all() and torch.equal(out[1], whole[1])
        c.tables.copy_(keep)
        for much in (c.tables.shape[1] * 16, 2 ** 31 - 1):
            c.lens[1] = much
            c.tables[1] = c.tables[0]
            page, off = c.positions(0, 101)
            run(out)
            assert vt.vt_paged_status(paged, clear=True) == vt.VT_DEV_KV_OVERFLOW
            assert torch.equal(out[0], whole[0])
            c.tables.copy_(keep)
            c.lens[1] = 60


def test_append_skips_what_does_not_fit(vtlib, paged):
    vt = vtlib
    c = Cache(vt, [30, 5, 3], [4, 4, 4], "f16", 1, 64, 16)  # tables of three pages
    q, k, v = c.rows(2), c.rows(1), c.rows(1)
    rope = torch.empty(33, 32, 2, device="cuda")
    vt.vt_rope_table(rope, 1e4)
    out = torch.full_like(q, 7.0)
    before = c.v.clone()
    c.tables[1, 0] = 99
    vt.vt_paged_append(paged, c.pool, c.batch(vt), q, k, v, rope, out)  # position 33 is past the rotation table
    assert vt.vt_paged_status(paged, clear=True) == vt.VT_DEV_KV_OVERFLOW | vt.VT_DEV_BAD_PAGE
    assert out[:3].any() and not out[3].any()
    page, off = c.positions(0, 34)
    assert torch.equal(c.v[page[30:33], 0, off[30:33]], v[:3, 0]) and torch.equal(c.v[page[33], 0, off[33]], before[page[33], 0, off[33]])
    c.lens.fill_(2 ** 31 - 1)
    before = c.v.clone()
    vt.vt_paged_append(paged, c.pool, c.batch(vt), q, k, v, rope, out)
    assert vt.vt_paged_status(paged, clear=True) == vt.VT_DEV_KV_OVERFLOW
    assert torch.equal(torch.nan_to_num(c.v, 9.0), torch.nan_to_num(before, 9.0)) and not out.any()


def test_rows_outside_every_sequence_are_left_alone(vtlib, paged):
    """starts that end before the last row, begin after the first, run past the end, or fall."""
    vt = vtlib
    c = Cache(vt, [20, 9], [3, 4], "f16", 1, 64, 16)
    q = torch.randn(9, 2, 64, device="cuda").half()
    for starts in ([1, 4, 8], [-5, 2, 100], [5, 3, 7], [9, 9, 9], [-3, -2, -1]):
        s = torch.tensor(starts, dtype=torch.int32, device="cuda")
        out = torch.full_like(q, 7.0)
        vt.vt_paged_prefill(paged, c.pool, vt.make_paged_batch(c.tables, torch.tensor([1, 1], dtype=torch.int32, device="cuda"), s), q, out)
        a = [max(0, min(9, x)) for x in starts]
        inside = torch.zeros(9, dtype=torch.bool, device="cuda")
        for b in range(2):
            inside[a[b]:a[b + 1]] = True
        assert (out[~inside] == 7.0).all()
        assert torch.isfinite(out[inside]).all()
        assert vt.vt_paged_status(paged, clear=True) == 0


def test_nothing_to_do(vtlib, paged):
    vt = vtlib
    c = Cache(vt, [3], [1], "f16", 1, 64, 16)
    none = torch.empty(0, 2, 64, dtype=torch.float16, device="cuda")
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    batch = vt.make_paged_batch(torch.empty(0, 3, dtype=torch.int32, device="cuda"), e)
    rope = torch.zeros(8, 32, 2, device="cuda")
    vt.vt_paged_decode(paged, c.pool, batch, none, none)
    vt.vt_paged_prefill(paged, c.pool, batch, none, none)
    vt.vt_paged_append(paged, c.pool, batch, none, none[:, :1], none[:, :1], rope, none)
    vt.vt_paged_prefill(paged, c.pool, c.batch(vt), none, none)


def test_refusals(vtlib, paged):
    """Every refusal comes before anything is enqueued, with a status and a message."""
    vt = vtlib
    L = vt.lib()
    c = Cache(vt, [20, 9], [1, 1], "f16", 2, 64, 16)
    q = c.rows(4)
    out = torch.full_like(q, 7.0)
    rope = torch.zeros(64, 32, 2, device="cuda")

    def change(x, **kw):
        y = type(x)()
        ctypes.memmove(ctypes.addressof(y), ctypes.addressof(x), ctypes.sizeof(x))
        for name, value in kw.items():
            setattr(y, name, value)
        return y

    batch, pool = c.batch(vt, False), c.pool

    def decode(g=paged, p=pool, b=batch, heads=4, qp=q.data_ptr(), ql=256, scale=0.1, window=0, o=out.data_ptr(), ol=256):
        return L.vt_paged_decode(g, p, b, heads, qp, ql, scale, window, o, ol, 0)

    inv, shape = vt.VT_ERR_INVALID_ARG, vt.VT_ERR_SHAPE
    cases = [
        (dict(g=None), inv), (dict(p=None), inv), (dict(b=None), inv), (dict(qp=None), inv), (dict(o=None), inv),
        (dict(qp=q.data_ptr() + 2), inv), (dict(ol=252), inv), (dict(ql=128), inv), (dict(ql=260), inv),
        (dict(scale=float("nan")), inv), (dict(scale=float("inf")), inv), (dict(scale=-0.1), inv), (dict(window=-1), inv),
        (dict(heads=3), shape), (dict(heads=0), shape), (dict(heads=2 * 129), shape),
        (dict(b=c.batch(vt)), inv),
    ]
    for kw, want in (({"dtype": 2}, shape), ({"d_head": 96}, shape), ({"page_size": 12}, shape), ({"page_size": 0}, shape),
                     ({"page_size": 2048}, shape), ({"n_kv_heads": 0}, shape), ({"n_pages": 0}, inv), ({"k": None}, inv),
                     ({"v": pool.v + 8}, inv), ({"page_stride": 100}, inv), ({"head_stride": 32}, inv), ({"pos_stride": 0}, inv),
                     ({"page_stride": -2048}, inv)):
        cases.append((dict(p=change(pool, **kw)), want))
    for kw in ({"tables": None}, {"lens": None}, {"n_seqs": -1}, {"n_seqs": 16385}, {"pages_per_seq": 0}, {"pages_per_seq": 1 << 27}):
        cases.append((dict(b=change(batch, **kw)), inv))
    for kw, want in cases:
        assert decode(**kw) == want, kw
        assert vt.vt_last_error()
    a = [paged, pool, batch, 2, 4, q.data_ptr(), 256, q.data_ptr(), 256, q.data_ptr(), 256, rope.data_ptr(), 64, out.data_ptr(), 256, 0]
    for at, value, want in ((0, None, inv), (3, 3, inv), (3, -1, inv), (4, 5, shape), (5, None, inv), (7, None, inv), (8, 64, inv),
                            (9, q.data_ptr() + 4, inv), (10, 129, inv), (11, None, inv), (11, rope.data_ptr() + 8, inv), (12, 0, inv),
                            (13, None, inv), (14, 100, inv)):
        assert L.vt_paged_append(*(a[:at] + [value] + a[at + 1:])) == want, (at, value)
    assert L.vt_paged_prefill(paged, pool, batch, 3, 4, q.data_ptr(), 256, 0.1, 0, out.data_ptr(), 256, 0) == inv
    assert L.vt_paged_prefill(paged, pool, c.batch(vt), 1 << 25, 4, q.data_ptr(), 256, 0.1, 0, out.data_ptr(), 256, 0) == inv
    assert L.vt_rope_table(rope.data_ptr(), 64, 96, 1e4, 0) == shape
    assert L.vt_rope_table(rope.data_ptr(), 0, 64, 1e4, 0) == inv and L.vt_rope_table(rope.data_ptr(), 64, 64, -1.0, 0) == inv
    for bad in (dict(q=q.cpu()), dict(q=q[:1]), dict(out=out[:, :3]), dict(q=q.transpose(1, 2)), dict(out=out.float())):
        with pytest.raises((ValueError, TypeError)):
            vt.vt_paged_decode(paged, pool, batch, bad.get("q", q), bad.get("out", out))
    with pytest.raises((ValueError, TypeError)):
        vt.make_paged_pool(c.k, c.v.float())
    with pytest.raises((ValueError, TypeError)):
        vt.make_paged_pool(c.k, c.v[:1])
    with pytest.raises((ValueError, TypeError)):
        vt.make_paged_batch(c.tables.long(), c.lens)
    with pytest.raises((ValueError, TypeError)):
        vt.make_paged_batch(c.tables, c.lens, c.starts[:2])
    torch.cuda.synchronize()
    assert (out == 7.0).all() and vt.vt_paged_status(paged) == 0


def test_serving_example(vtlib):
    """The example serves five sequences; two layers of fp16 projections and activations leave each sequence's
    hidden states within 2^-8 of the sequence alone in 64 bits (about ten roundings of 2^-11 a layer)."""
    from examples.paged_serving import serve
    err, n = serve()
    assert n == 5 and err <= 2.0 ** -8, err


@pytest.mark.parametrize("window", [0, 37])
@pytest.mark.parametrize("dtype,d_head,group", [("f16", 128, 4), ("bf16", 64, 1), ("f16", 64, 16), ("bf16", 128, 3)])
def test_few_rows_beside_many(vtlib, paged, dtype, d_head, group, window):
    """Sequences of one to a few rows, and one whose rows fill many tiles of the kernel for few."""
    lens = [(i * 7919) % 300 if i % 7 else -1 for i in range(120)]
    rows = [1 + i % 3 if i % 5 else 0 for i in range(120)]
    lens[60], rows[60] = 200, 60
    c = Cache(vtlib, lens, rows, dtype, 2, d_head, 16, "pos")
    check_attention(vtlib, paged, c, "prefill", 2 * group, window)


@pytest.mark.parametrize("call", ["decode", "prefill"])
def test_scale_zero_and_large(vtlib, paged, call):
    """scale 0: every attended value weighs the same; a large scale: the highest score takes everything."""
    c = Cache(vtlib, [0, 77, 200], [1] * 3 if call == "decode" else [150, 3, 40], "f16", 2, 64, 16)
    check_attention(vtlib, paged, c, call, 4, scale=0.0)
    c = Cache(vtlib, [0, 77, 200], [1] * 3 if call == "decode" else [150, 3, 40], "bf16", 2, 64, 16, seed=1)
    check_attention(vtlib, paged, c, call, 4, scale=16.0)


def test_many_sequences_of_one_block(vtlib, paged):
    """More units than CTAs, most of a single block: the ends of units dominate."""
    n = 400
    lens = [(i * 613) % 90 for i in range(n)]
    rows = [20 + i % 23 for i in range(n)]
    check_attention(vtlib, paged, Cache(vtlib, lens, rows, "f16", 1, 64, 32), "prefill", 1)


@pytest.mark.parametrize("window", [0, 20])
@pytest.mark.parametrize("call", ["decode", "prefill"])
@pytest.mark.parametrize("dtype,d_head,group,longest", [("f16", 64, 1, 3), ("bf16", 128, 2, 40), ("f16", 128, 7, 126), ("bf16", 64, 12, 70),
                                                       ("f16", 128, 1, 200)])
def test_many_short_sequences(vtlib, paged, call, dtype, d_head, group, longest, window):
    """Many times more units than the GPU holds, of a few positions each, idle slots among them."""
    n = 230
    lens = [(i * 7919) % longest if i % 9 else -1 for i in range(n)]
    rows = [1 if call == "decode" else (0 if i % 13 == 5 else 1 + (i % 17 == 0) * 2) for i in range(n)]
    check_attention(vtlib, paged, Cache(vtlib, lens, rows, dtype, 8, d_head, 16, "pos"), call, 8 * group, window)


@pytest.mark.parametrize("dtype,d_head,kv_heads,group,window,rows", [
    ("f16", 64, 1, 5, 0, 77), ("bf16", 128, 2, 1, 3000, 129), ("f16", 128, 1, 128, 0, 9), ("bf16", 64, 3, 8, 6100, 33)])
def test_prefill_of_many_parts(vtlib, paged, dtype, d_head, kv_heads, group, window, rows):
    """A few long units, each shared by many SMs; a sequence with nothing to join and an idle one beside them."""
    c = Cache(vtlib, [9999, 0, -1, 12345], [rows, 2, 5, 40], dtype, kv_heads, d_head, 32)
    check_attention(vtlib, paged, c, "prefill", kv_heads * group, window)


def widened(c, positions=60000):
    """Tables as wide as a server's, nearly all of it unused: the widths alone keep the tiles' kernel."""
    c.tables = torch.nn.functional.pad(c.tables, (0, positions // c.page), value=-1).contiguous()
    return c


@pytest.mark.parametrize("window", [0, 1, 2, 15, 127, 128, 129, 300, 5000])
@pytest.mark.parametrize("dtype,d_head,kv_heads,group,page,order", [
    ("f16", 128, 2, 2, 32, "pos"), ("bf16", 64, 1, 7, 16, "head"), ("f16", 64, 2, 1, 4, "head"), ("bf16", 128, 1, 20, 128, "pos")])
def test_prefill_window_wide_tables(vtlib, paged, window, dtype, d_head, kv_heads, group, page, order):
    rows = [30 + 57 * (i % 4) for i in range(len(LENS))]
    c = widened(Cache(vtlib, LENS, rows, dtype, kv_heads, d_head, page, order, seed=window))
    check_attention(vtlib, paged, c, "prefill", kv_heads * group, window)


@pytest.mark.parametrize("std,scale", [(0.0, 1.0), (0.05, 1.0), (4.0, 1.0), (1.0, 0.0), (1.0, 16.0)])
@pytest.mark.parametrize("dtype,d_head", [("f16", 128), ("bf16", 64)])
def test_prefill_score_ranges_wide_tables(vtlib, paged, dtype, d_head, std, scale):
    c = widened(Cache(vtlib, [0, 100, 513], [140, 30, 70], dtype, 2, d_head, 16))
    check_attention(vtlib, paged, c, "prefill", 8, scale=scale, q=c.rows(8, std))


def test_prefill_rising_scores_wide_tables(vtlib, paged):
    c = widened(Cache(vtlib, [700], [150], "f16", 1, 64, 16))
    page, off = c.positions(0, 850)
    c.k[page, 0, off] = (torch.arange(850, device="cuda")[:, None] / 64).half().expand(-1, 64)
    q = torch.ones(c.n_rows, 2, 64, dtype=torch.float16, device="cuda")
    check_attention(vtlib, paged, c, "prefill", 2, scale=0.25, q=q)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_prefill_infinities_and_nan_wide_tables(vtlib, paged, dtype):
    """A key that scores -inf takes no weight; NaN reaches the rows that attend to it and no other sequence."""
    c = widened(Cache(vtlib, [40, 40, 40], [50, 60, 70], dtype, 1, 64, 16))
    q = c.rows(1).abs()
    page, off = c.positions(0, 90)
    c.k[page[3], 0, off[3]] = float("-inf")
    page2, off2 = c.positions(2, 110)
    c.v[page2[7], 0, off2[7]] = float("nan")
    out = torch.empty_like(q)
    vtlib.vt_paged_prefill(paged, c.pool, c.batch(vtlib), q, out)
    assert torch.isfinite(out[:110]).all() and torch.isnan(out[110:]).all()
    c.v[page2[7], 0, off2[7]] = 0.0
    ref, tol = attention(c, q, 0.125, 0)
    assert ((out.double() - ref).abs() <= tol)[:110].all()


@pytest.mark.parametrize("page", [4, 16, 64])
def test_prefill_bad_pages_and_overflow_wide_tables(vtlib, paged, page):
    """A page id that is not one of the pool's: its positions take no part, the call says so."""
    vt = vtlib
    c = widened(Cache(vt, [400, 60], [40, 50], "f16", 1, 64, page))
    q = c.rows(2)
    out, whole = torch.empty_like(q), torch.empty_like(q)
    vt.vt_paged_prefill(paged, c.pool, c.batch(vt), q, whole)
    keep = c.tables.clone()
    page_id, off = c.positions(0, 440)
    for bad in (-1, c.k.shape[0], 2 ** 31 - 1, -2 ** 31):
        c.tables[0, 2] = bad
        vt.vt_paged_prefill(paged, c.pool, c.batch(vt), q, out)
        assert vt.vt_paged_status(paged, clear=True) == vt.VT_DEV_BAD_PAGE
        c.tables.copy_(keep)
        hide = torch.arange(440, device="cuda") > torch.arange(400, 440, device="cuda")[:, None]
        hide[:, 2 * page:3 * page] = True
        kk, vv = c.k[page_id, 0, off].double(), c.v[page_id, 0, off].double()
        for h in range(2):
            ref = torch.softmax((q[:40, h].double() @ kk.T / 8).masked_fill(hide, -math.inf), -1) @ vv
            assert ((out[:40, h].double() - ref).abs() <= 2.0 ** -9 * vv.abs().max()).all()
        assert torch.equal(out[40:], whole[40:])
    ref, tol = attention(c, q, 0.125, 0)
    c.tables[1, -(-110 // page):] = c.tables[0, 0]
    c.lens[1] = 2 ** 31 - 1
    vt.vt_paged_prefill(paged, c.pool, c.batch(vt), q, out)
    assert vt.vt_paged_status(paged, clear=True) == vt.VT_DEV_KV_OVERFLOW
    assert ((out.double() - ref).abs() <= tol)[:40].all()  # (the longer batch is cut elsewhere: not the same bits)


def test_prefill_rows_outside_every_sequence_wide_tables(vtlib, paged):
    """starts that end before the last row, begin after the first, run past the end, or fall."""
    vt = vtlib
    c = widened(Cache(vt, [20, 9], [80, 70], "f16", 1, 64, 16))
    q = torch.randn(90, 2, 64, device="cuda").half()
    lens = torch.tensor([1, 1], dtype=torch.int32, device="cuda")
    for starts in ([10, 40, 80], [-5, 20, 1000], [50, 30, 70], [90, 90, 90], [-30, -20, -10]):
        s = torch.tensor(starts, dtype=torch.int32, device="cuda")
        out = torch.full_like(q, 7.0)
        vt.vt_paged_prefill(paged, c.pool, vt.make_paged_batch(c.tables, lens, s), q, out)
        a = [max(0, min(90, x)) for x in starts]
        inside = torch.zeros(90, dtype=torch.bool, device="cuda")
        for b in range(2):
            inside[a[b]:a[b + 1]] = True
        assert (out[~inside] == 7.0).all() and torch.isfinite(out[inside]).all()
        assert vt.vt_paged_status(paged, clear=True) == 0


def test_prefill_strides_and_offsets_past_32_bits_wide_tables(vtlib, paged):
    """Pages whose entries lie more than 2^31 elements into the pool; rows and outputs with gaps."""
    vt, stride = vtlib, 2 ** 29 + 8
    small = widened(Cache(vt, [50, 3], [30, 40], "f16", 1, 64, 16, spare=0))
    n = small.k.shape[0]
    base = [torch.full(((n - 1) * stride + 16 * 64,), float("nan"), dtype=torch.float16, device="cuda") for _ in range(2)]
    k, v = (t.as_strided((n, 1, 16, 64), (stride, 64, 64, 1)) for t in base)
    k.copy_(small.k)
    v.copy_(small.v)
    q, big = small.rows(7)[:, 1:4], torch.full((small.n_rows, 5, 64), 3.0, dtype=torch.float16, device="cuda")
    vt.vt_paged_prefill(paged, vt.make_paged_pool(k, v), small.batch(vt), q, big[:, :3])
    ref, tol = attention(small, q, 0.125, 0)
    assert ((big[:, :3].double() - ref).abs() <= tol).all() and (big[:, 3:] == 3.0).all()


def test_prefill_repeats_bit_for_bit_wide_tables(vtlib, paged):
    vt = vtlib
    for rows, heads in (([40, 130, 30, 77], 2), ([60], 2), ([300, 200, 250, 280], 16)):
        c = widened(Cache(vt, [3000, 77, 4097, 9000][:len(rows)], rows, "f16", 2, 128, 16))
        q, outs = c.rows(heads), []
        for _ in range(4):
            outs.append(torch.empty_like(q))
            vt.vt_paged_prefill(paged, c.pool, c.batch(vt), q, outs[-1])
        assert all(torch.equal(outs[0], o) for o in outs[1:])


def test_prefill_of_many_parts_in_a_graph(vtlib, paged):
    """A captured call serves other lengths: parts of few long units, then no parts at all, then idle slots."""
    vt = vtlib
    c = Cache(vt, [9000, 5000], [60, 70], "f16", 2, 128, 64)
    q = c.rows(4)
    out = torch.empty_like(q)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        vt.vt_paged_prefill(paged, c.pool, c.batch(vt), q, out)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        batch = c.batch(vt)
        with torch.cuda.graph(graph, stream=stream):
            vt.vt_paged_prefill(paged, c.pool, batch, q, out)
        for lens in ([9000, 5000], [40, 3], [-1, 5000], [8999, -1], [-1, -1], [9000, 5000]):
            c.lens.copy_(torch.tensor(lens, dtype=torch.int32))
            c.lens_host = lens
            out.fill_(7.0)
            graph.replay()
            stream.synchronize()
            ref, tol = attention(c, q, 128 ** -0.5, 0)
            assert ((out.double() - ref).abs() <= tol).all(), lens
    assert vt.vt_paged_status(paged) == 0
