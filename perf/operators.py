"""The operators of a paged key-value cache, as measurable cases: what a program does that serves several
sequences at once from one pool of pages.

  append   vt_paged_append: the new rows' queries and keys are rotated to their positions, the keys and
           values are written to the pages of their sequences
  decode   vt_paged_decode: one new token of every sequence attends to that sequence's pages
  prefill  vt_paged_prefill: several new rows of every sequence (a prompt, the next turn of a chat, the
           drafted tokens of a speculation) attend causally to that sequence's pages

A pool is seen as [pages, KV heads, positions in a page, head dim]; in memory the KV heads lie outside
the positions (order "head") or inside them (order "pos").  Sequence b holds lens[b] positions before
the call, and its new rows come after them; lens[b] < 0 marks an idle slot of the batch, which has no
position to attend to and gets zeros.  How long each sequence is goes by the case alone; the values,
and which pages a sequence has, go by the seed.

Head shapes are the repository's: the 512-wide test layer (8 heads of 64), 7B (32 heads of 128), 13B (40
heads, in shards of 20, 12 and 8) and 8B (32 query heads on 8 KV heads), whole or the part of one device.
"""
import math

import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
SPARE = 3  # pages of a pool that no sequence of the batch holds


def _case(name, kind, dtype, heads, kv_heads, d_head, n, len_lo, len_hi, page, order="head", rows_lo=1, rows_hi=1,
          window=0, idle=0, theta=1e4):
    """n sequences that hold len_lo .. len_hi positions and get rows_lo .. rows_hi new rows; idle: every so many-th
    slot of the batch is idle (0: none)."""
    c = dict(kind=kind, dtype=dtype, heads=heads, kv_heads=kv_heads, d_head=d_head, n=n, len_lo=len_lo, len_hi=len_hi,
             page=page, order=order, rows_lo=rows_lo, rows_hi=rows_hi, window=window, idle=idle, theta=theta)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one user, one new token of the smallest model: only the call's latency counts
        _case("append one token", "append", "f16", 8, 8, 64, 1, 128, 128, 16),
        # the ordinary step of a server: one new token for each of 64 sequences, half-filled pages
        _case("append 64 tokens", "append", "bf16", 32, 8, 128, 64, 100, 8000, 32, order="pos", theta=5e5),
        # prompts that come in together, odd lengths, some behind an earlier turn: bandwidth counts
        _case("append prompts", "append", "f16", 32, 8, 128, 7, 0, 2000, 16, rows_lo=300, rows_hi=2500, theta=5e5),
        # one user, the smallest model at the length that its test has: latency
        _case("decode one short", "decode", "f16", 8, 8, 64, 1, 128, 128, 16),
        # one user at the end of a very long document: a few KV heads have to keep the whole GPU busy
        _case("decode one long", "decode", "bf16", 32, 8, 128, 1, 130999, 130999, 64, theta=5e5),
        # a server's step: 64 slots from fresh to long, some of them idle
        _case("decode 64 ragged", "decode", "f16", 32, 8, 128, 64, 1, 8191, 16, idle=9, theta=5e5),
        # no grouped heads, sliding window, the pool in the other order
        _case("decode 16 windowed", "decode", "bf16", 32, 32, 128, 16, 500, 4096, 32, order="pos", window=1024),
        # the next short turn of a chat, behind a cached history
        _case("prefill turn", "prefill", "f16", 32, 8, 128, 1, 300, 300, 16, rows_lo=77, rows_hi=77, theta=5e5),
        # four drafted tokens of each of 16 sequences are checked at once, one device's 12 heads
        _case("prefill drafts", "prefill", "bf16", 12, 12, 128, 16, 50, 4000, 16, rows_lo=4, rows_hi=4),
        # prompts of several users together, from nothing, odd lengths
        _case("prefill prompts", "prefill", "bf16", 32, 8, 128, 5, 0, 0, 32, order="pos", rows_lo=150, rows_hi=900, theta=5e5),
        # a chunk of a long document behind what came before it
        _case("prefill chunk", "prefill", "f16", 32, 8, 128, 1, 16000, 16000, 64, rows_lo=512, rows_hi=512, theta=5e5),
        # one long prompt without grouped heads: the matrix products count
        _case("prefill long", "prefill", "f16", 32, 32, 128, 1, 0, 0, 128, rows_lo=4096, rows_hi=4096),
    ]


def _log(rng, lo, hi):
    """Even over the logarithm; large drawn sizes fill no whole tile, the listed cases have those that do."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n + 1 if n >= 64 and n % 64 == 0 else n


def draw(rng):
    kind = rng.choice(["append", "decode", "decode", "prefill", "prefill"])
    heads, kv_heads, d_head, theta = rng.choice([(8, 8, 64, 1e4), (32, 32, 128, 1e4), (8, 8, 128, 1e4), (12, 12, 128, 1e4),
                                                 (20, 20, 128, 1e4), (32, 8, 128, 5e5), (8, 2, 128, 5e5), (16, 8, 64, 5e5)])
    dtype, order = rng.choice(["f16", "bf16"]), rng.choice(["head", "pos"])
    page = rng.choice([8, 16, 32, 64, 128, 256])
    window = _log(rng, 16, 2048) if kind != "append" and rng.random() < 0.25 else 0
    if kind == "append":
        rows = _log(rng, 1, 8000)
        n = min(_log(rng, 1, 200), rows)
        each = max(1, rows // n)
        lo, hi = rng.choice([(each, each), (each // 3 | 1, each)])
        return _case(None, kind, dtype, heads, kv_heads, d_head, n, 0, _log(rng, 1, 8000), page, order, lo, hi, theta=theta)
    if kind == "decode":
        # at most the positions of the listed cases, as pages and padded to the longest sequence
        longest = _log(rng, 1, 130000 if kv_heads <= 8 else 30000)
        n = _log(rng, 1, max(1, min(200, 500000 // longest * 8 // max(8, kv_heads))))
        lo = rng.choice([longest, 0, longest // 4 | 1])
        return _case(None, kind, dtype, heads, kv_heads, d_head, n, lo, longest, page, order, window=window,
                     idle=rng.choice([0, 0, 5]), theta=theta)
    rows = _log(rng, 2, 2500)
    before = _log(rng, 1, 12000) if rng.random() < 0.6 else 0
    # padded to the longest of each, the scores and the positions are no more than those of the listed cases
    if heads * rows * (rows + before) > 2.5e8:
        before = 0
    n = _log(rng, 1, max(1, min(32, int(2.5e8 / (heads * rows * (rows + before + page))), int(4e6 / (kv_heads * (rows + before))))))
    return _case(None, kind, dtype, heads, kv_heads, d_head, n, rng.choice([before, 0]), before, page, order,
                 rng.choice([rows, rows // 5 | 1]), rows, window=window, theta=theta)


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
    """An append reads q, k, v and the rotation of each position and writes q, k, v.  Attention reads the keys and
    values that any row of a sequence attends to, reads q and writes as much."""
    lens, rows = _sizes(case)
    H, K, d, W = case["heads"], case["kv_heads"], case["d_head"], case["window"]
    total = sum(rows)
    if case["kind"] == "append":
        return {"bytes": total * ((2 * H + 4 * K) * d * 2 + d * 4), "flops": 3 * total * (H + K) * d}
    read = pairs = 0
    for p, r in zip(lens, rows):
        first = 0 if p < 0 or not W else max(0, p + 1 - W)
        read += max(0, p + r - first) if p >= 0 else 0
        if p >= 0:
            full = r * p + r * (r + 1) // 2  # positions 0 .. p + i for row i
            cut = sum(max(0, p + i + 1 - W) for i in range(r)) if W else 0
            pairs += full - cut
    return {"bytes": read * K * d * 4 + total * H * d * 4, "flops": 4 * H * d * pairs}


# ------------------------------------------------------------------ inputs, from the seed alone

def _normal(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _inputs(c, seed):
    """Everything that lies on the GPU before the call."""
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)
    lens, rows = _sizes(c)
    H, K, d, P, dt = c["heads"], c["kv_heads"], c["d_head"], c["page"], TYPES[c["dtype"]]
    held = [max(0, p + r) if p >= 0 else 0 for p, r in zip(lens, rows)]
    pages = [-(-h // P) for h in held]
    per, total = max(1, max(pages)), sum(pages)
    starts = [0]
    for r in rows:
        starts.append(starts[-1] + r)
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
    shape = (total + SPARE, K, P, d) if c["order"] == "head" else (total + SPARE, P, K, d)
    for name in ("kp", "vp"):
        pool = _normal(g, shape, std, dt)
        x[name] = pool if c["order"] == "head" else pool.permute(0, 2, 1, 3)
    if c["kind"] == "append":
        # q, k and v of a row lie side by side, as one projection leaves them
        qkv = _normal(g, (starts[-1], H + 2 * K, d), std, dt)
        x["q"], x["k"], x["v"] = qkv[:, :H], qkv[:, H:H + K], qkv[:, H + K:]
        angle = torch.arange(max(held) + 1, device="cuda", dtype=torch.float64)[:, None] * torch.tensor(
            [c["theta"] ** (-2.0 * i / d) for i in range(d // 2)], device="cuda", dtype=torch.float64)
        x["rope"] = torch.stack((angle.cos(), angle.sin()), -1).float().contiguous()
    else:
        x["q"] = _normal(g, (starts[-1], H, d), std, dt)
        # what no sequence holds (whole pages, and the ends of last pages) may be anything: here it is NaN,
        # so that a read of it shows
        live = torch.zeros(total + SPARE, P, dtype=torch.bool, device="cuda")
        pos = at[..., None] * P + torch.arange(P, device="cuda")
        here = (pos < torch.tensor(held, device="cuda")[:, None, None]) & (tables[..., None] >= 0)
        live[tables.clamp(min=0).long()[..., None].expand_as(here)[here], (pos % P).expand_as(here)[here]] = True
        for name in ("kp", "vp"):
            x[name].masked_fill_(~live[:, None, :, None], float("nan"))
    return x


class State:
    def __init__(self, case, seed):
        lens, rows = _sizes(case)
        self.case, self.max_rows = case, max(rows)
        self.x = _inputs(case, seed)
        self.scale = 1.0 / math.sqrt(case["d_head"])
        self.out = torch.empty(sum(rows), case["heads"], case["d_head"], dtype=TYPES[case["dtype"]], device="cuda")
        self.paged = 0
        if own:
            from paper_2607_07046_gb300 import vt
            self.vt = vt
            self.paged = vt.vt_paged_create()
            self.pool = vt.make_paged_pool(self.x["kp"], self.x["vp"])
            self.batch = vt.make_paged_batch(self.x["tables"], self.x["lens"],
                                             None if case["kind"] == "decode" else self.x["starts"])

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
        if kind == "append":
            vt.vt_paged_append(s.paged, s.pool, s.batch, x["q"], x["k"], x["v"], x["rope"], s.out)
            return {"q": s.out, "k_pool": x["kp"], "v_pool": x["vp"]}
        if kind == "decode":
            vt.vt_paged_decode(s.paged, s.pool, s.batch, x["q"], s.out, s.scale, s.case["window"])
        else:
            vt.vt_paged_prefill(s.paged, s.pool, s.batch, x["q"], s.out, s.scale, s.case["window"])
        return {"out": s.out}
    if kind == "append":
        return _append(s)
    return _attend(s)


def _rotated(x, cos, sin):
    """Dimensions i and i + d/2 of every head turned by the angle of the row's position."""
    a, b = x.float().chunk(2, -1)
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1).to(x.dtype)


def _append(s):
    x, P = s.x, s.case["page"]
    row = torch.arange(s.out.shape[0], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(x["starts"], row, right=True) - 1
    pos = (x["lens"][seq] + row - x["starts"][seq]).long()
    cos, sin = x["rope"][pos][:, None].unbind(-1)
    page, at = x["tables"][seq, pos // P].long(), pos % P
    s.out.copy_(_rotated(x["q"], cos, sin))
    x["kp"][page, :, at] = _rotated(x["k"], cos, sin)
    x["vp"][page, :, at] = x["v"]
    return {"q": s.out, "k_pool": x["kp"], "v_pool": x["vp"]}


def _attend(s):
    """Every sequence padded to the most rows and positions of the batch."""
    x, W = s.x, s.case["window"]
    lens, starts, tables = x["lens"], x["starts"], x["tables"].clamp(min=0).long()
    B, K, d = lens.shape[0], s.case["kv_heads"], s.case["d_head"]
    G, R, L = s.case["heads"] // K, s.max_rows, tables.shape[1] * s.case["page"]
    k = x["kp"][tables].permute(0, 2, 1, 3, 4).reshape(B, K, L, d).float()
    v = x["vp"][tables].permute(0, 2, 1, 3, 4).reshape(B, K, L, d).float()
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

def exact(case, seed):
    """One sequence after another, every head of it from the definition."""
    x = _inputs(case, seed)
    lens, rows = _sizes(case)
    H, K, d, P, W = case["heads"], case["kv_heads"], case["d_head"], case["page"], case["window"]
    f64 = dict(dtype=torch.float64, device="cuda")
    if case["kind"] == "append":
        q, kp, vp = x["q"].double(), x["kp"].double().clone(), x["vp"].double().clone()
        rope, out, first = x["rope"].double(), torch.zeros(sum(rows), H, d, **f64), 0
        for b, (p, r) in enumerate(zip(lens, rows)):
            pos = torch.arange(p, p + r, device="cuda")
            turn = torch.complex(rope[pos, :, 0], rope[pos, :, 1])[:, None]  # pair i of a head, as one number
            for src, h in ((q, H), (x["k"].double(), K)):
                y = src[first:first + r]
                z = torch.complex(y[..., :d // 2], y[..., d // 2:]) * turn
                y = torch.cat((z.real, z.imag), -1)
                if h == H and src is q:
                    out[first:first + r] = y
                else:
                    kp[x["tables"][b].long()[pos // P], :, pos % P] = y
            vp[x["tables"][b].long()[pos // P], :, pos % P] = x["v"][first:first + r].double()
            first += r
        return {"q": out, "k_pool": kp, "v_pool": vp}
    out, first = torch.zeros(sum(rows), H, d, **f64), 0
    for b, (p, r) in enumerate(zip(lens, rows)):
        if p >= 0:
            pos = torch.arange(p + r, device="cuda")
            page = x["tables"][b].long()[pos // P]
            i = torch.arange(p, p + r, device="cuda")[:, None]
            hidden = pos[None, :] > i
            if W:
                hidden |= pos[None, :] <= i - W
            for h in range(H):
                key = x["kp"][page, h // (H // K), pos % P].double()
                val = x["vp"][page, h // (H // K), pos % P].double()
                z = x["q"][first:first + r, h].double() @ key.T / math.sqrt(d)
                out[first:first + r, h] = torch.softmax(z.masked_fill(hidden, -math.inf), -1) @ val
        first += r
    return {"out": out}
