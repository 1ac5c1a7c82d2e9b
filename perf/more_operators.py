"""The operators around a paged key-value cache in 8 bits, as measurable cases: what a program does that serves
several sequences at once and wants twice as many positions in the same memory, or models whose queries and keys
are normalised for each head.

  append_qk  vt_paged_append_qk: a row's queries and keys are normalised for each head (root mean square and a
             gain), rotated to their position (pairs of halves or of neighbours, all of the head or its first
             dimensions), and keys and values are written to the pages of their sequences
  append_mx  vt_paged_append_mx: the same, and keys and values are written in 8 bits
  decode     vt_paged_decode_mx: one new token of every sequence attends to that sequence's pages
  prefill    vt_paged_prefill_mx: several new rows of every sequence attend causally to them

An entry in 8 bits (one position's key or value of one KV head) is a code for each dimension and a scale for each
32 of them, a power of two: the smallest 2^E with which the largest code holds the largest value.  Codes are e4m3
(largest 448) or whole numbers up to 127 (int8), rounded to nearest, ties to even; scales are stored as E + 127.
E is kept where every code times its scale is a value of the rows' type (_RANGE).

A pool is seen as [pages, KV heads, positions in a page, head dim]; in memory the KV heads lie outside the
positions (order "head") or inside them (order "pos"); scales are [pages, KV heads, positions, head dim / 32].
Sequence b holds lens[b] positions before the call, and its new rows come after them; lens[b] < 0 marks an idle
slot of the batch.  How long each sequence is goes by the case alone; the values, and which pages a sequence has,
go by the seed.

Head shapes are the repository's: the 512-wide test layer (8 heads of 64), 7B (32 heads of 128), 13B (40 heads, in
shards of 20, 12 and 8) and 8B (32 query heads on 8 KV heads), whole or the part of one device.
"""
import math

import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
MOST = {"e4m3": 448.0, "int8": 127.0}
_RANGE = {("e4m3", "f16"): (-15, 7), ("e4m3", "bf16"): (-117, 7), ("int8", "f16"): (-24, 9), ("int8", "bf16"): (-117, 119)}
BLOCK = 32  # dimensions that share a scale
SPARE = 3   # pages of a pool that no sequence of the batch holds
EPS = 1e-6


def _case(name, kind, dtype, heads, kv_heads, d_head, n, len_lo, len_hi, page, order="head", rows_lo=1, rows_hi=1,
          window=0, idle=0, theta=1e4, code="", norm=False, rotary=0, pairs="halves"):
    """n sequences that hold len_lo .. len_hi positions and get rows_lo .. rows_hi new rows; idle: every so many-th slot of the
    batch is idle (0: none); rotary: the dimensions of a head that are rotated."""
    c = dict(kind=kind, dtype=dtype, heads=heads, kv_heads=kv_heads, d_head=d_head, n=n, len_lo=len_lo, len_hi=len_hi,
             page=page, order=order, rows_lo=rows_lo, rows_hi=rows_hi, window=window, idle=idle, theta=theta, code=code,
             norm=norm, rotary=rotary, pairs=pairs)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one user, one new token of the smallest model: only the call's latency counts
        _case("append qk one token", "append_qk", "f16", 8, 8, 64, 1, 128, 128, 16, norm=True, rotary=64),
        # prompts that come in together, odd lengths, some behind an earlier turn: bandwidth counts
        _case("append qk prompts", "append_qk", "bf16", 32, 8, 128, 7, 0, 2000, 16, rows_lo=300, rows_hi=2500, theta=5e5,
              norm=True, rotary=128),
        # the ordinary step of a server: one new token for each of 64 sequences, half of each head rotated by neighbours
        _case("append mx 64 tokens", "append_mx", "bf16", 32, 8, 128, 64, 100, 8000, 32, order="pos", theta=5e5, code="e4m3",
              norm=True, rotary=64, pairs="neighbours"),
        # the prompts again, into 8 bits
        _case("append mx prompts", "append_mx", "f16", 32, 8, 128, 7, 0, 2000, 16, rows_lo=300, rows_hi=2500, theta=5e5,
              code="e4m3", norm=True, rotary=128),
        # one user, the smallest model at the length that its test has: latency
        _case("decode one short", "decode", "f16", 8, 8, 64, 1, 128, 128, 16, code="int8"),
        # one user at the end of a very long document: a few KV heads have to keep the whole GPU busy
        _case("decode one long", "decode", "bf16", 32, 8, 128, 1, 130999, 130999, 64, code="e4m3"),
        # a server's step: 64 slots from fresh to long, some of them idle
        _case("decode 64 ragged", "decode", "f16", 32, 8, 128, 64, 1, 8191, 16, idle=9, code="e4m3"),
        # no grouped heads, sliding window, the pool in the other order
        _case("decode 16 windowed", "decode", "bf16", 32, 32, 128, 16, 500, 4096, 32, order="pos", window=1024, code="int8"),
        # the next short turn of a chat, behind a cached history
        _case("prefill turn", "prefill", "f16", 32, 8, 128, 1, 300, 300, 16, rows_lo=77, rows_hi=77, code="e4m3"),
        # four drafted tokens of each of 16 sequences are checked at once, one device's 12 heads
        _case("prefill drafts", "prefill", "bf16", 12, 12, 128, 16, 50, 4000, 16, rows_lo=4, rows_hi=4, code="int8"),
        # a chunk of a long document behind what came before it
        _case("prefill chunk", "prefill", "f16", 32, 8, 128, 1, 16000, 16000, 64, rows_lo=512, rows_hi=512, code="e4m3"),
        # one long prompt without grouped heads: the matrix products count
        _case("prefill long", "prefill", "bf16", 32, 32, 128, 1, 0, 0, 128, rows_lo=4096, rows_hi=4096, code="int8"),
    ]


def _log(rng, lo, hi):
    """Even over the logarithm; large drawn sizes fill no whole tile, the listed cases have those that do."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n + 1 if n >= 64 and n % 64 == 0 else n


def draw(rng):
    kind = rng.choice(["append_qk", "append_mx", "decode", "decode", "prefill", "prefill"])
    heads, kv_heads, d_head, theta = rng.choice([(8, 8, 64, 1e4), (32, 32, 128, 1e4), (8, 8, 128, 1e4), (12, 12, 128, 1e4),
                                                 (20, 20, 128, 1e4), (32, 8, 128, 5e5), (8, 2, 128, 5e5), (16, 8, 64, 5e5)])
    dtype, order = rng.choice(["f16", "bf16"]), rng.choice(["head", "pos"])
    page = rng.choice([8, 16, 32, 64, 128, 256])
    code = "" if kind == "append_qk" else "e4m3" if kind == "append_mx" else rng.choice(["e4m3", "int8"])
    window = _log(rng, 16, 2048) if kind in ("decode", "prefill") and rng.random() < 0.25 else 0
    if kind in ("append_qk", "append_mx"):
        rows = _log(rng, 1, 8000)
        n = min(_log(rng, 1, 200), rows)
        each = max(1, rows // n)
        lo, hi = rng.choice([(each, each), (each // 3 | 1, each)])
        return _case(None, kind, dtype, heads, kv_heads, d_head, n, 0, _log(rng, 1, 8000), page, order, lo, hi, theta=theta, code=code,
                     norm=rng.random() < 0.75, rotary=rng.choice([d_head, d_head, d_head // 2, d_head // 4, 0]),
                     pairs=rng.choice(["halves", "neighbours"]))
    if kind == "decode":
        # at most the positions of the listed cases, as pages and padded to the longest sequence
        longest = _log(rng, 1, 130000 if kv_heads <= 8 else 30000)
        n = _log(rng, 1, max(1, min(200, 500000 // longest * 8 // max(8, kv_heads))))
        lo = rng.choice([longest, 0, longest // 4 | 1])
        return _case(None, kind, dtype, heads, kv_heads, d_head, n, lo, longest, page, order, window=window,
                     idle=rng.choice([0, 0, 5]), code=code)
    rows = _log(rng, 2, 2500)
    before = _log(rng, 1, 12000) if rng.random() < 0.6 else 0
    # padded to the longest of each, the scores and the positions are no more than those of the listed cases
    if heads * rows * (rows + before) > 2.5e8:
        before = 0
    n = _log(rng, 1, max(1, min(32, int(2.5e8 / (heads * rows * (rows + before + page))), int(4e6 / (kv_heads * (rows + before))))))
    return _case(None, kind, dtype, heads, kv_heads, d_head, n, rng.choice([before, 0]), before, page, order,
                 rng.choice([rows, rows // 5 | 1]), rows, window=window, code=code)


# ------------------------------------------------------------------ sizes, by the case alone

def _spread(n, lo, hi, turn):
    """n whole numbers between lo and hi, evenly over their logarithm and in no order."""
    return [int(round((lo + 1) * ((hi + 1) / (lo + 1)) ** ((turn + (i + 1) * 0.6180339887498949) % 1.0))) - 1 for i in range(n)]


def _sizes(c):
    """(positions held, new rows) of every sequence; -1 positions: an idle slot."""
    lens = _spread(c["n"], c["len_lo"], c["len_hi"], 0.25)
    rows = _spread(c["n"], c["rows_lo"], c["rows_hi"], 0.6)
    if c["idle"]:
        lens = [-1 if i % c["idle"] == c["idle"] - 2 else v for i, v in enumerate(lens)]
    return lens, rows


def work(case):
    """An append reads q, k, v, the rotation of each position and the gains, and writes q, k, v.  Attention reads the codes and
    scales that any row of a sequence attends to, reads q and writes as much."""
    lens, rows = _sizes(case)
    H, K, d, W = case["heads"], case["kv_heads"], case["d_head"], case["window"]
    total = sum(rows)
    entry = 2 * d if not case["code"] else d + d // BLOCK  # bytes
    if case["kind"].startswith("append"):
        return {"bytes": total * ((2 * H + 2 * K) * d * 2 + 2 * K * entry + case["rotary"] * 4) + (4 * d if case["norm"] else 0),
                "flops": total * (H + K) * ((4 * d if case["norm"] else 0) + 3 * case["rotary"])}
    read = pairs = 0
    for p, r in zip(lens, rows):
        first = 0 if p < 0 or not W else max(0, p + 1 - W)
        read += max(0, p + r - first) if p >= 0 else 0
        if p >= 0:
            full = r * p + r * (r + 1) // 2  # positions 0 .. p + i for row i
            cut = sum(max(0, p + i + 1 - W) for i in range(r)) if W else 0
            pairs += full - cut
    return {"bytes": read * K * 2 * entry + total * H * d * 4, "flops": 4 * H * d * pairs}


# ------------------------------------------------------------------ 8 bits

def _to_codes(x, code, dtype):
    """(codes, E + 127) of values [..., d] in 32 bits."""
    lo, hi = _RANGE[code, dtype]
    y = x.unflatten(-1, (-1, BLOCK))
    part, power = torch.frexp(y.abs().amax(-1))             # part in [0.5, 1)
    top, top_power = math.frexp(MOST[code])
    e = (power - top_power + (part > top)).clamp(lo, hi)
    e = torch.where(part == 0, lo, e)
    y = torch.ldexp(y, -e[..., None]).clamp(-MOST[code], MOST[code])
    y = (torch.round(y) if code == "int8" else y).to(CODES[code])
    return y.flatten(-2), (e + 127).to(torch.uint8)


def _values(codes, scales):
    """What they stand for, in 32 bits."""
    power = torch.exp2(scales.view(torch.uint8).float() - 127.0)
    return (codes.float().unflatten(-1, (-1, BLOCK)) * power[..., None]).flatten(-2)


# ------------------------------------------------------------------ inputs, from the seed alone

def _normal(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _pool(c, g, pages, std):
    """(codes or values, scales or None) of one side of the pool."""
    d, P, K = c["d_head"], c["page"], c["kv_heads"]
    x = _normal(g, (pages, K, P, d) if c["order"] == "head" else (pages, P, K, d), std, TYPES[c["dtype"]])
    if not c["code"]:
        return (x if c["order"] == "head" else x.permute(0, 2, 1, 3)), None
    codes, scales = _to_codes(x.float(), c["code"], c["dtype"])
    if c["order"] == "pos":
        codes, scales = codes.permute(0, 2, 1, 3), scales.permute(0, 2, 1, 3).contiguous()
    return codes, scales.view(torch.float8_e8m0fnu)


def _inputs(c, seed):
    """Everything that lies on the GPU before the call."""
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 29)
    lens, rows = _sizes(c)
    H, K, d, P, dt = c["heads"], c["kv_heads"], c["d_head"], c["page"], TYPES[c["dtype"]]
    held = [max(0, p + r) if p >= 0 else 0 for p, r in zip(lens, rows)]
    pages = [-(-h // P) for h in held]
    per, total = max(1, max(pages)), sum(pages)
    starts = [0] + torch.tensor(rows).cumsum(0).tolist()
    # the pages lie anywhere in the pool; entries of a table past a sequence's last page hold no page
    order = torch.randperm(total + SPARE, generator=g, device="cuda").to(torch.int32)
    ends = torch.tensor(pages, device="cuda").cumsum(0)
    at = torch.arange(per, device="cuda")[None, :]
    count = torch.tensor(pages, device="cuda")[:, None]
    tables = torch.where(at < count, order[((ends[:, None] - count) + at).clamp(0, total + SPARE - 1)], -1).to(torch.int32)
    x = {"lens": torch.tensor(lens, dtype=torch.int32, device="cuda"),
         "starts": torch.tensor(starts, dtype=torch.int32, device="cuda"), "tables": tables.contiguous()}
    # projections of a unit-RMS input by weights of N(0, 0.02^2) have this spread at d_model 4096
    std = 1.28
    x["kp"], x["ks"] = _pool(c, g, total + SPARE, std)
    x["vp"], x["vs"] = _pool(c, g, total + SPARE, std)
    x["rope"] = x["q_gain"] = x["k_gain"] = None
    if c["kind"].startswith("append"):
        # q, k and v of a row lie side by side, as one projection leaves them
        qkv = _normal(g, (starts[-1], H + 2 * K, d), std, dt)
        x["q"], x["k"], x["v"] = qkv[:, :H], qkv[:, H:H + K], qkv[:, H + K:]
        if c["rotary"]:
            angle = torch.arange(max(held) + 1, device="cuda", dtype=torch.float64)[:, None] * c["theta"] ** (
                torch.arange(c["rotary"] // 2, device="cuda", dtype=torch.float64) * (-2.0 / c["rotary"]))
            x["rope"] = torch.stack((angle.cos(), angle.sin()), -1).float().contiguous()
        if c["norm"]:
            x["q_gain"], x["k_gain"] = ((1.0 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(dt) for _ in range(2))
    else:
        x["q"] = _normal(g, (starts[-1], H, d), std, dt)
        # what no sequence holds (whole pages, and the ends of last pages) may be anything: here its scales are NaN, so that
        # a use of it shows
        live = torch.zeros(total + SPARE, P, dtype=torch.bool, device="cuda")
        pos = at[..., None] * P + torch.arange(P, device="cuda")
        here = (pos < torch.tensor(held, device="cuda")[:, None, None]) & (tables[..., None] >= 0)
        live[tables.clamp(min=0).long()[..., None].expand_as(here)[here], (pos % P).expand_as(here)[here]] = True
        x["ks"].view(torch.uint8).masked_fill_(~live[:, None, :, None], 255)
        x["vs"].view(torch.uint8).masked_fill_(~live[:, None, :, None], 255)
    return x


class State:
    def __init__(self, case, seed):
        lens, rows = _sizes(case)
        self.case, self.max_rows = case, max(rows)
        self.x = x = _inputs(case, seed)
        self.scale = 1.0 / math.sqrt(case["d_head"])
        self.out = torch.empty(sum(rows), case["heads"], case["d_head"], dtype=TYPES[case["dtype"]], device="cuda")
        self.paged = 0
        if own:
            from paper_2607_07046_gb300 import vt
            self.vt = vt
            self.paged = vt.vt_paged_create()
            self.pool = (vt.make_paged_mx_pool(x["kp"], x["vp"], x["ks"], x["vs"], TYPES[case["dtype"]]) if case["code"]
                         else vt.make_paged_pool(x["kp"], x["vp"]))
            self.batch = vt.make_paged_batch(x["tables"], x["lens"], None if case["kind"] == "decode" else x["starts"])
            if case["kind"].startswith("append"):
                self.form = vt.make_qk_form(x["rope"], case["pairs"] == "neighbours", x["q_gain"], x["k_gain"], EPS)

    def __del__(self):
        if self.paged:
            self.vt.vt_paged_destroy(self.paged)


def prepare(case, seed):
    return State(case, seed)


# ------------------------------------------------------------------ the operators

def run(state):
    s, x, kind = state, state.x, state.case["kind"]
    if own:
        vt = s.vt
        if kind.startswith("append"):
            append = vt.vt_paged_append_mx if kind == "append_mx" else vt.vt_paged_append_qk
            append(s.paged, s.pool, s.batch, x["q"], x["k"], x["v"], s.form, s.out)
            return _stored(s)
        attend = vt.vt_paged_decode_mx if kind == "decode" else vt.vt_paged_prefill_mx
        attend(s.paged, s.pool, s.batch, x["q"], s.out, s.scale, s.case["window"])
        return {"out": s.out}
    if kind.startswith("append"):
        return _append(s)
    return _attend(s)


def _stored(s):
    """Codes are the 8-bit floats that they are held as, and so are the scales."""
    x = s.x
    if s.case["kind"] == "append_qk":
        return {"q": s.out, "k_pool": x["kp"], "v_pool": x["vp"]}
    return {"q": s.out, "k_codes": x["kp"], "k_scales": x["ks"], "v_codes": x["vp"], "v_scales": x["vs"]}


def _formed(x, gain, cos, sin, rotary, pairs):
    """Every head of x over its root mean square, times the gain, its first `rotary` dimensions turned; in 32 bits."""
    x = x.float()
    if gain is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain.float()
    if not rotary:
        return x
    y, rest = x[..., :rotary], x[..., rotary:]
    a, b = y.chunk(2, -1) if pairs == "halves" else (y[..., 0::2], y[..., 1::2])
    a, b = a * cos - b * sin, b * cos + a * sin
    y = torch.cat((a, b), -1) if pairs == "halves" else torch.stack((a, b), -1).flatten(-2)
    return torch.cat((y, rest), -1)


def _append(s):
    x, c, P = s.x, s.case, s.case["page"]
    row = torch.arange(s.out.shape[0], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(x["starts"], row, right=True) - 1
    pos = (x["lens"][seq] + row - x["starts"][seq]).long()
    cos, sin = x["rope"][pos][:, None].unbind(-1) if c["rotary"] else (None, None)
    page, at = x["tables"][seq, pos // P].long(), pos % P
    s.out.copy_(_formed(x["q"], x["q_gain"], cos, sin, c["rotary"], c["pairs"]))
    k = _formed(x["k"], x["k_gain"], cos, sin, c["rotary"], c["pairs"])
    if c["kind"] == "append_qk":
        x["kp"][page, :, at] = k.to(x["kp"].dtype)
        x["vp"][page, :, at] = x["v"]
        return _stored(s)
    k, ks = _to_codes(k, c["code"], c["dtype"])
    v, vs = _to_codes(x["v"].float(), c["code"], c["dtype"])
    x["kp"].view(torch.uint8)[page, :, at] = k.view(torch.uint8)
    x["vp"].view(torch.uint8)[page, :, at] = v.view(torch.uint8)
    x["ks"].view(torch.uint8)[page, :, at] = ks
    x["vs"].view(torch.uint8)[page, :, at] = vs
    return _stored(s)


def _attend(s):
    """Every sequence padded to the most rows and positions of the batch."""
    x, W = s.x, s.case["window"]
    lens, starts, tables = x["lens"], x["starts"], x["tables"].clamp(min=0).long()
    B, K, d = lens.shape[0], s.case["kv_heads"], s.case["d_head"]
    G, R, L = s.case["heads"] // K, s.max_rows, tables.shape[1] * s.case["page"]
    code = s.case["code"]
    k = _values(x["kp"].view(torch.uint8)[tables].view(CODES[code]), x["ks"].view(torch.uint8)[tables])
    v = _values(x["vp"].view(torch.uint8)[tables].view(CODES[code]), x["vs"].view(torch.uint8)[tables])
    k, v = k.permute(0, 2, 1, 3, 4).reshape(B, K, L, d), v.permute(0, 2, 1, 3, 4).reshape(B, K, L, d)
    j = torch.arange(R, device="cuda")
    q = x["q"][(starts[:-1, None] + j).clamp(max=x["q"].shape[0] - 1).long()]
    q = q.reshape(B, R, K, G, d).permute(0, 2, 3, 1, 4).reshape(B, K, G * R, d).float()
    pos, at = torch.arange(L, device="cuda"), lens[:, None] + j
    new = (starts[1:] - starts[:-1])[:, None]
    sees = (pos <= at[..., None]) & (lens >= 0)[:, None, None] & (j < new)[..., None]
    if W:
        sees &= pos > at[..., None] - W
    held = (pos < lens[:, None] + new) & (lens >= 0)[:, None]
    score = (q @ k.transpose(-1, -2) * s.scale).reshape(B, K, G, R, L)
    score = score.masked_fill(~sees[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - top.masked_fill(top == -math.inf, 0.0))
    p = (p / p.sum(-1, keepdim=True).clamp(min=1e-30)).reshape(B, K, G * R, L)
    o = p @ v.masked_fill(~held[:, None, :, None], 0.0)
    o = o.reshape(B, K, G, R, d).permute(0, 3, 1, 2, 4).reshape(B, R, K * G, d)
    row = torch.arange(s.out.shape[0], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(starts, row, right=True) - 1
    s.out.copy_(o[seq, (row - starts[seq]).long()])
    return {"out": s.out}


# ------------------------------------------------------------------ the definition, in 64 bits

def _grid(y, code, lo, hi):
    """The nearest code and scale of values [..., 32], from the definition of the formats: an e4m3 number has a step of an eighth
    of its power of two, and of 2^-9 below 2^-6."""
    most = y.abs().amax(-1)
    e = torch.ceil(torch.log2(most / MOST[code])).clamp(-200, 200)
    e = torch.where(torch.exp2(e) * MOST[code] < most, e + 1, e)
    e = torch.where(torch.exp2(e - 1) * MOST[code] >= most, e - 1, e)  # (a logarithm next to a whole number)
    e = torch.where(most == 0, float(lo), e.clamp(lo, hi))
    z = (y / torch.exp2(e)[..., None]).clamp(-MOST[code], MOST[code])
    if code == "int8":
        return torch.round(z), torch.exp2(e)
    step = torch.exp2(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(z / step) * step, torch.exp2(e)


def exact(case, seed):
    """One sequence after another, every head of it from the definition."""
    c, x = case, _inputs(case, seed)
    lens, rows = _sizes(c)
    H, K, d, P, W, n_rot = c["heads"], c["kv_heads"], c["d_head"], c["page"], c["window"], c["rotary"]
    f64 = dict(dtype=torch.float64, device="cuda")
    if c["kind"].startswith("append"):
        out, first = torch.zeros(sum(rows), H, d, **f64), 0
        pools = {"k": x["kp"].double(), "v": x["vp"].double()}
        if c["code"]:
            scales = {"k": x["ks"].float().double(), "v": x["vs"].float().double()}
        # pair i of a head, as dimensions
        i = torch.arange(n_rot // 2, device="cuda")
        re, im = (i, i + n_rot // 2) if c["pairs"] == "halves" else (2 * i, 2 * i + 1)
        for b, (p, r) in enumerate(zip(lens, rows)):
            pos = torch.arange(p, p + r, device="cuda")
            page, at = x["tables"][b].long()[pos // P], pos % P
            for which, gain in (("q", x["q_gain"]), ("k", x["k_gain"]), ("v", None)):
                y = x[which][first:first + r].double()
                if gain is not None:
                    y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / d + EPS) * gain.double()
                if which != "v" and n_rot:
                    turn = torch.complex(x["rope"][pos, :, 0].double(), x["rope"][pos, :, 1].double())[:, None]
                    z = torch.complex(y[..., re], y[..., im]) * turn
                    y = y.clone()
                    y[..., re], y[..., im] = z.real, z.imag
                if which == "q":
                    out[first:first + r] = y
                elif not c["code"]:
                    pools[which][page, :, at] = y
                else:
                    codes, scale = _grid(y.reshape(r, K, d // BLOCK, BLOCK), c["code"], *_RANGE[c["code"], c["dtype"]])
                    pools[which][page, :, at] = codes.reshape(r, K, d)
                    scales[which][page, :, at] = scale
            first += r
        if not c["code"]:
            return {"q": out, "k_pool": pools["k"], "v_pool": pools["v"]}
        return {"q": out, "k_codes": pools["k"], "k_scales": scales["k"], "v_codes": pools["v"], "v_scales": scales["v"]}
    out, first = torch.zeros(sum(rows), H, d, **f64), 0
    for b, (p, r) in enumerate(zip(lens, rows)):
        if p >= 0:
            pos = torch.arange(p + r, device="cuda")
            page = x["tables"][b].long()[pos // P]
            i = torch.arange(p, p + r, device="cuda")[:, None]
            hidden = pos[None, :] > i
            if W:
                hidden |= pos[None, :] <= i - W
            for kvh in range(K):
                key, val = ((x[n].view(torch.uint8)[page, kvh, pos % P].view(CODES[c["code"]]).double().reshape(-1, d // BLOCK, BLOCK)
                             * 2.0 ** (x[m].view(torch.uint8)[page, kvh, pos % P].double() - 127)[..., None]).reshape(-1, d)
                            for n, m in (("kp", "ks"), ("vp", "vs")))
                for h in range(kvh * (H // K), (kvh + 1) * (H // K)):
                    z = x["q"][first:first + r, h].double() @ key.T / math.sqrt(d)
                    out[first:first + r, h] = torch.softmax(z.masked_fill(hidden, -math.inf), -1) @ val
        first += r
    return {"out": out}
