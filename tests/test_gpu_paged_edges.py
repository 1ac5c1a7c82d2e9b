"""The paged KV cache at the edges of what its calls accept, against plain definitions in 64 bits."""
from __future__ import annotations

import math

import pytest

torch = pytest.importorskip("torch")
from .test_gpu_paged import TINY, TYPE, U, Cache, attention, check_attention, paged, widened  # noqa: E402,F401

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


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("window", [1, 16, 50])
@pytest.mark.parametrize("past", [0, 5, 30, 1000, 2 ** 30])
def test_window_of_a_length_past_the_table(vtlib, paged, form, window, past):
    """Row i of a sequence whose length is `past` positions over its table attends to [p - window + 1, p] at its true
    position p: to what of it the table has, and to nothing when it has none of it."""
    vt = vtlib
    rows, kv = {"decode": ([1, 1], 1), "few": ([40, 30], 1), "tiles": ([600, 30], 8)}[form]
    c = Cache(vt, [704 - rows[0], 20], rows, "f16", kv, 64, 16)
    cap = c.tables.shape[1] * 16
    c.lens[0] = cap + past
    q = c.rows(2 * kv)
    out = attend(vt, paged, c, form, q, 0.125, window)
    assert vt.vt_paged_status(paged, clear=True) == vt.VT_DEV_KV_OVERFLOW
    for i in range(rows[0]):
        seen = torch.arange(min(cap, max(0, cap + past + i - window + 1)), cap, device="cuda")
        if len(seen) == 0:
            assert not out[i:rows[0]].any(), i
            break
        page, off = c.tables[0].long()[seen // 16], seen % 16
        k, v = (t[page, :, off].double().transpose(0, 1) for t in (c.k, c.v))
        w = torch.softmax(q[i].double().reshape(kv, 2, 64) @ k.transpose(1, 2) / 8, -1)
        o, a = (w @ v).reshape(2 * kv, 64), (w @ v.abs()).reshape(2 * kv, 64)
        tol = U["f16"] * o.abs() + (U["f16"] + 2.0 ** -16) * a + TINY["f16"] * window * v.abs().max()
        assert ((out[i].double() - o).abs() <= tol).all(), i
    ref, tol = attention(c, q, 0.125, window)
    assert ((out.double() - ref).abs() <= tol)[rows[0]:].all()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("bits", [20.3, 25.6, 27.1])
def test_many_small_weights_add_up(vtlib, paged, form, dtype, bits):
    """One key takes nearly all the weight and its value is 0; 40,000 others have 2^-bits of it each and a value of 1, so
    that the output is their sum alone.  Weights may be rounded to the type, u each, and lose what lies below the type's
    smallest step: fp16 weights that are scaled to 2^15 (decode, two terms) or to at least 2^7 (prefill) at the largest
    lose at most 2^-40 and 2^-32 of it each.  Scores of up to 40 log2 units carry 2^-24 of that as fp32 values, two
    roundings each, 2^-17 of a weight; at most 2504 products are added in a row, 2^-23 of their sum each, and 700 sums of
    weights, 2^-24 each: less than 2^-11."""
    n, seqs, each = 40000, 38, 130 if form == "tiles" else 1
    c = Cache(vtlib, [n], [each], dtype, 8, 64, 64)
    c.k.masked_fill_(c.live[:, None, :, None], 0.0)
    c.v.masked_fill_(c.live[:, None, :, None], 1.0)
    page, off = c.positions(0, n)
    c.k[page[777], :, off[777], 0] = 1.0
    c.v[page[777], :, off[777]] = 0.0
    # as many sequences, on the same pages, as leave each CTA whole histories
    c.tables, c.lens, c.n_rows = c.tables.repeat(seqs, 1), c.lens.repeat(seqs), seqs * each
    c.starts = torch.arange(0, c.n_rows + 1, each, dtype=torch.int32, device="cuda")
    q = torch.zeros(c.n_rows, 16, 64, dtype=TYPE[dtype], device="cuda")
    q[:, :, 0] = 1.0
    out = attend(vtlib, paged, c, form, q, bits * math.log(2.0), 0).double()
    u, floor = U[dtype], 0.0 if dtype == "bf16" else 2.0 ** (-32 if form == "tiles" else -40)
    m = (n + torch.arange(c.n_rows, device="cuda") % each).double()[:, None, None]
    ref = m * 2.0 ** -bits / (1.0 + m * 2.0 ** -bits)
    tol = (2 * u + 2.0 ** -11 + 2.0 ** -17) * ref + m * floor + (2.0 ** -25 if dtype == "f16" else 0.0)
    assert ((out - ref).abs() <= tol).all(), float(((out - ref).abs() / ref).max())


@pytest.mark.parametrize("window", [0, 16])
@pytest.mark.parametrize("form", ["few", "tiles"])
def test_a_slot_without_rows_overflows_nothing(vtlib, paged, form, window):
    """A length past the table is reported where a new row is at or past it, and only there, by every call alike."""
    vt = vtlib
    c = Cache(vt, [30, 40], [0, 600 if form == "tiles" else 5], "f16", 8, 64, 16)
    c.lens[0] = c.tables.shape[1] * 16 + 3
    q = c.rows(16)
    out = attend(vt, paged, c, form, q, 0.125, window)
    assert vt.vt_paged_status(paged, clear=True) == 0
    ref, tol = attention(c, q, 0.125, window)
    assert ((out.double() - ref).abs() <= tol).all()
    c.lens[0] = 30
    c.lens[1] += c.tables.shape[1] * 16 - 600 - 40 + 1 if form == "tiles" else c.tables.shape[1] * 16 - 5 - 40 + 1
    attend(vt, paged, c, form, q, 0.125, window)  # the last row is one position past the table
    assert vt.vt_paged_status(paged, clear=True) == vt.VT_DEV_KV_OVERFLOW


def test_an_idle_slot_overflows_nothing(vtlib, paged):
    """An idle slot with more rows than the table has positions: zeros, and no status bit."""
    vt = vtlib
    c = Cache(vt, [-1, 30], [60, 5], "f16", 2, 64, 16)
    assert c.tables.shape[1] * 16 < 59
    q = c.rows(4)
    out = attend(vt, paged, c, "few", q, 0.125, 0)
    assert vt.vt_paged_status(paged, clear=True) == 0 and not out[:60].any()
    ref, tol = attention(c, q, 0.125, 0)
    assert ((out.double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("window", [0, 200])
@pytest.mark.parametrize("dtype,d_head,kv_heads,group", [("f16", 128, 2, 4), ("bf16", 64, 8, 1), ("f16", 64, 1, 30)])
def test_a_prompt_among_tokens_and_empty_slots(vtlib, paged, dtype, d_head, kv_heads, group, window):
    """Single tokens, a few drafted ones, prompts, idle slots (one of them with rows) and slots without rows in one
    batch, by trimmed tables and by a server's."""
    lens = [(i * 7919) % 3000 if i % 6 else -1 for i in range(150)]
    rows = [(0, 1, 1, 0, 3, 0)[i % 6] for i in range(150)]
    lens[40], rows[40] = 1500, 400
    lens[41], rows[41] = 0, 130
    lens[42], rows[42] = -1, 50
    lens[149], rows[149] = 77, 24 // group + 1
    c = Cache(vtlib, lens, rows, dtype, kv_heads, d_head, 16, "pos")
    check_attention(vtlib, paged, c, "prefill", kv_heads * group, window)
    check_attention(vtlib, paged, widened(c), "prefill", kv_heads * group, window)


@pytest.mark.parametrize("heads,kv_heads,length,rows,slots", [(32, 8, 4000, 380, 64), (32, 32, 0, 3000, 128)])
def test_empty_slots_cost_a_prompt_little(vtlib, paged, heads, kv_heads, length, rows, slots):
    """A prompt takes about as long among slots without rows as by itself.  (The kernel of single tokens would take five
    to eleven times as long; three times leaves room for another user of the machine.)"""
    vt = vtlib
    best = []
    for n in (1, slots):
        c = Cache(vt, [length] + [-1] * (n - 1), [rows] + [0] * (n - 1), "bf16", kv_heads, 128, 16)
        q, batch = c.rows(heads), c.batch(vt)
        out = torch.empty_like(q)
        times = []
        for _ in range(8):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(10):
                vt.vt_paged_prefill(paged, c.pool, batch, q, out)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        best.append(min(times))
    assert best[1] <= 3 * best[0], best


def test_rows_that_move_between_slots_in_a_graph(vtlib, paged):
    """A captured call serves other rows per slot: which kernel takes a slot goes by its rows at replay."""
    vt = vtlib
    n, total = 60, 300
    c = Cache(vt, [2000 + i for i in range(n)], [5] * n, "f16", 2, 64, 64)
    c.tables = torch.cat((c.tables, c.tables.roll(1, 0)[:, :8]), 1).contiguous()  # room for more rows in every slot
    c.tables.clamp_(min=0)
    c.k.nan_to_num_(0.25)
    c.v.nan_to_num_(0.25)
    q = torch.randn(total, 8, 64, generator=c.gen, device="cuda").half()
    out, batch, stream = torch.empty_like(q), c.batch(vt), torch.cuda.Stream()
    with torch.cuda.stream(stream):
        vt.vt_paged_prefill(paged, c.pool, batch, q, out)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            vt.vt_paged_prefill(paged, c.pool, batch, q, out)
        for kind in range(4):
            rows = [[5] * n, [1] * (n - 1) + [total - n + 1], [0] * 10 + [total] + [0] * (n - 11), [7 * (i % 2) + 1 for i in range(n)]][kind]
            starts = [0]
            for r in rows:
                starts.append(starts[-1] + r)
            c.starts.copy_(torch.tensor(starts, dtype=torch.int32))
            c.rows_host, c.starts_host = rows, starts
            out.fill_(7.0)
            graph.replay()
            stream.synchronize()
            ref, tol = attention(c, q, 0.125, 0)
            assert ((out.double() - ref).abs() <= tol)[:starts[-1]].all(), kind
    assert vt.vt_paged_status(paged) == 0


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("form,d_head,kv_heads,group,page", [
    ("decode", 64, 2, 1, 16), ("decode", 128, 2, 4, 32), ("decode", 128, 1, 12, 16), ("decode", 64, 1, 40, 64),
    ("few", 64, 2, 1, 16), ("few", 128, 2, 4, 32), ("few", 128, 1, 12, 16)])  # (a group of 40 is the tiles')
def test_weights_of_single_tokens_carry_two_terms(vtlib, paged, form, dtype, d_head, kv_heads, group, page):
    """The kernel of single tokens keeps a weight in two 16-bit terms: p - hi - lo is at most u^2 p, so beside the
    output's own rounding, u |o|, only 2^-16 A (fp32 scores, exponentials and sums) and 2^-16 A (two bf16 terms) remain,
    A = sum_j softmax_j |v_j|; fp16 outputs below 2^-14 are 2^-25 off at most.  (One term alone would be u A off.)"""
    lens = [0, 1, 15, 16, 63, 200, 777, 3000, -1, 5000]
    c = Cache(vtlib, lens, [1] * len(lens), dtype, kv_heads, d_head, page)
    q = c.rows(kv_heads * group)
    out = attend(vtlib, paged, c, form, q, d_head ** -0.5, 0).double()
    ref, loose = attention(c, q, d_head ** -0.5, 0)
    u = U[dtype]
    a = (loose - u * ref.abs()) / (u + 2.0 ** -16)  # (with a little more in fp16: its bound for small weights)
    tol = u * ref.abs() + (2.0 ** -15) * a + TINY[dtype]
    assert ((out - ref).abs() <= tol).all(), float(((out - ref).abs() / tol.clamp(min=1e-30)).max())


@pytest.mark.parametrize("form", ["decode", "few", "tiles"])
def test_as_many_sequences_as_a_batch_takes(vtlib, paged, form):
    """16384 sequences, short and idle ones; for the tiles' kernel some with rows enough for it."""
    vt, n = vtlib, 16384
    gen = torch.Generator(device="cuda").manual_seed(5)
    lens = (torch.arange(n, device="cuda") * 7919 % 40 - 3).int()  # below 0: idle
    rows = torch.ones(n, dtype=torch.int32, device="cuda") if form != "tiles" else torch.arange(n, device="cuda").int() % 3 * 20
    page, per = 16, 6
    k, v = (torch.randn(500, 1, page, 64, generator=gen, device="cuda").half() for _ in range(2))
    tables = torch.randint(500, (n, per), generator=gen, device="cuda").int()
    starts = torch.cat((torch.zeros(1, dtype=torch.int32, device="cuda"), rows.cumsum(0).int()))
    total = int(starts[-1])
    q = torch.randn(total, 2, 64, generator=gen, device="cuda").half()
    out, pool = torch.full_like(q, 7.0), vt.make_paged_pool(k, v)
    batch = vt.make_paged_batch(tables, lens, None if form == "decode" else starts)
    (vt.vt_paged_decode if form == "decode" else vt.vt_paged_prefill)(paged, pool, batch, q, out)
    assert vt.vt_paged_status(paged) == 0
    # every row padded to the table, in 64 bits, some thousands at a time
    row = torch.arange(total, device="cuda")
    seq = torch.searchsorted(starts.long(), row, right=True) - 1
    at = lens.long()[seq] + row - starts.long()[seq]
    pos = torch.arange(per * page, device="cuda")
    u = U["f16"]
    for part in torch.split(row, 8192):
        b = seq[part]
        sees = (pos <= at[part][:, None]) & (lens[b] >= 0)[:, None]
        kk, vv = (t[tables[b].long()].squeeze(2).reshape(len(b), per * page, 64).double() for t in (k, v))
        s = torch.einsum("rhd,rpd->rhp", q[part].double(), kk) / 8
        w = torch.softmax(s.masked_fill(~sees[:, None], -math.inf), -1).nan_to_num(0.0)
        o, a = w @ vv, w @ vv.abs()
        far = (out[part].double() - o).abs()
        assert (far <= u * o.abs() + (u + 2.0 ** -16) * a + 100 * 2.0 ** -25 * 6).all()


def test_append_as_many_sequences_as_a_batch_takes(vtlib, paged):
    vt, n = vtlib, 16384
    lens = (torch.arange(n, device="cuda") * 7919 % 16 - 1).int()
    rows = (torch.arange(n, device="cuda") % 2).int()
    starts = torch.cat((torch.zeros(1, dtype=torch.int32, device="cuda"), rows.cumsum(0).int()))
    total = int(starts[-1])
    k, v = (torch.zeros(n, 1, 16, 64, dtype=torch.float16, device="cuda") for _ in range(2))
    tables = torch.randperm(n, device="cuda").int()[:, None].contiguous()
    x = torch.randn(total, 3, 64, device="cuda").half()
    rope = torch.empty(16, 32, 2, device="cuda")
    vt.vt_rope_table(rope, 1e4)
    q_out = torch.full((total, 1, 64), 7.0, dtype=torch.float16, device="cuda")
    vt.vt_paged_append(paged, vt.make_paged_pool(k, v), vt.make_paged_batch(tables, lens, starts), x[:, :1], x[:, 1:2],
                       x[:, 2:], rope, q_out)
    assert vt.vt_paged_status(paged) == 0
    b = torch.arange(1, n, 2, device="cuda")
    live = b[lens[b] >= 0]
    want = torch.zeros_like(v)
    want[tables[live, 0].long(), 0, lens[live].long()] = x[(live - 1) // 2, 2]
    assert torch.equal(v, want)
    assert not q_out[(lens[b] < 0)].any() and q_out[lens[b] >= 0].any(-1).all()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("scale", [2.0 ** 127, 3.4e38, 1e-45, 1e-39])
def test_the_largest_and_smallest_scales(vtlib, paged, form, scale):
    """Scores of 0 weigh the same at every scale that the call takes; any scores do at the smallest."""
    rows = [600, 3] if form == "tiles" else [1, 1]
    c = Cache(vtlib, [50, 300], rows, "f16", 8, 64, 16)
    q = c.rows(16)
    if scale > 1:
        q.zero_()
    out = attend(vtlib, paged, c, form, q, scale, 0)
    ref, tol = attention(c, q, 0.0, 0)
    assert ((out.double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("wide", [False, True])
def test_an_idle_slot_of_many_rows_among_tokens(vtlib, paged, wide):
    """Idle slots get zeros whichever kernels the batch goes to, also when no sequence has rows enough for the tiles'."""
    n = 60
    lens, rows = [1500 + 7 * i for i in range(n)], [1 + i % 2 for i in range(n)]
    lens[3], rows[3] = -1, 194
    lens[50], rows[50] = -1, 25
    c = Cache(vtlib, lens, rows, "bf16", 8, 64, 128, "pos")
    check_attention(vtlib, paged, widened(c) if wide else c, "prefill", 16)
