"""Several users of one small model: prompts come in together and one at a time, tokens are decoded for all of
them at once, a sequence that ends gives its pages to the next.

The attention of every step runs through the paged cache (PagedCache.append, then PagedCache.attend); the
projections around it are torch products.  Every sequence's hidden states are checked against the same model run
for that sequence alone, without a cache, in 64 bits.

    python examples/paged_serving.py [e4m3 | int8]

With a code the cache holds 8-bit codes, and the model's queries and keys are normalised for each head and rotated
by neighbours in the first half of their dimensions.
"""
from __future__ import annotations

import math
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parents[1]))
from paper_2607_07046_gb300 import vt  # noqa: E402
from paper_2607_07046_gb300.paged import PagedCache  # noqa: E402

LAYERS, D, HEADS, KV_HEADS, DH, F = 2, 512, 8, 2, 64, 1408
EPS, THETA = 1e-5, 1e4


def weights(seed=0):
    """Of each layer; the gains of queries and keys, and half of a head rotated, are for models that have them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    shapes = {"qkv": ((HEADS + 2 * KV_HEADS) * DH, D), "o": (D, HEADS * DH), "gate": (F, D), "up": (F, D), "down": (D, F)}
    layers = [{n: (torch.randn(s, generator=g, device="cuda") / math.sqrt(s[1])).half() for n, s in shapes.items()} for _ in range(LAYERS)]
    for w in layers:
        w["q_gain"], w["k_gain"] = ((1 + 0.1 * torch.randn(DH, generator=g, device="cuda")).half() for _ in range(2))
    return layers


def norm(x):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)


def forward(layers, x, attend):
    """Hidden states of the rows x; attend(layer, qkv rows) -> attention output rows."""
    for l, w in enumerate(layers):
        h = x + attend(l, norm(x) @ w["qkv"].to(x.dtype).T) @ w["o"].to(x.dtype).T
        n = norm(h)
        x = h + (torch.nn.functional.silu(n @ w["gate"].to(x.dtype).T) * (n @ w["up"].to(x.dtype).T)) @ w["down"].to(x.dtype).T
    return x


def alone(layers, x, norms=False):
    """One sequence by itself, in 64 bits."""
    n, rotary = x.shape[0], DH // 2 if norms else DH
    ang = torch.arange(n, device="cuda").double()[:, None] * THETA ** (-2.0 * torch.arange(rotary // 2, device="cuda").double() / rotary)
    c, s = ang.cos()[:, None], ang.sin()[:, None]

    def turn(y, gain):
        if not norms:
            a, b = y[..., :DH // 2], y[..., DH // 2:]
            return torch.cat((a * c - b * s, b * c + a * s), -1)
        y = norm(y) * gain.double()
        a, b = y[..., 0:rotary:2], y[..., 1:rotary:2]
        return torch.cat((torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2), y[..., rotary:]), -1)

    def attend(l, qkv):
        y, w = qkv.reshape(n, -1, DH), layers[l]
        q, k, v = turn(y[:, :HEADS], w["q_gain"]), turn(y[:, HEADS:HEADS + KV_HEADS], w["k_gain"]), y[:, HEADS + KV_HEADS:]
        k, v = (t.repeat_interleave(HEADS // KV_HEADS, 1).transpose(0, 1) for t in (k, v))
        s = q.transpose(0, 1) @ k.transpose(1, 2) / math.sqrt(DH)
        hide = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
        return (torch.softmax(s.masked_fill(hide, -math.inf), -1) @ v).transpose(0, 1).reshape(n, -1)

    return forward(layers, x.double(), attend)


class Server:
    def __init__(self, layers, slots=4, pages=40, page_size=16, max_len=400, code=None):
        self.layers = layers
        self.cache = PagedCache(LAYERS, KV_HEADS, DH, page_size, pages, slots, max_len, theta=THETA, code=code,
                                rotary_dim=DH if code is None else DH // 2)
        self.forms = [None if code is None else vt.make_qk_form(self.cache.rope, True, w["q_gain"], w["k_gain"], EPS) for w in layers]

    def step(self, new):
        """new: {slot: rows of inputs}; the hidden states of those rows."""
        c, rows = self.cache, {slot: x.shape[0] for slot, x in new.items()}
        batch, starts = c.step(rows)
        x = torch.zeros(starts[-1], D, dtype=torch.float16, device="cuda")
        for slot, part in new.items():
            x[starts[slot]:starts[slot] + part.shape[0]] = part
        q_rot, out = (torch.empty(starts[-1], HEADS, DH, dtype=torch.float16, device="cuda") for _ in range(2))

        def attend(l, qkv):
            y = qkv.reshape(starts[-1], HEADS + 2 * KV_HEADS, DH)
            c.append(l, batch, y[:, :HEADS], y[:, HEADS:HEADS + KV_HEADS], y[:, HEADS + KV_HEADS:], q_rot, self.forms[l])
            c.attend(l, batch, q_rot, out)
            return out.reshape(starts[-1], HEADS * DH)

        y = forward(self.layers, x, attend)
        c.advance(rows)
        return {slot: y[starts[slot]:starts[slot] + n] for slot, n in rows.items()}


def serve(code=None):
    """The largest relative error of any sequence's hidden states against the sequence alone, and how many there were."""
    layers = weights()
    g = torch.Generator(device="cuda").manual_seed(1)
    server = Server(layers, code=code)
    inputs, outputs, finished = {}, {}, []

    def feed(new):
        for slot, y in server.step(new).items():
            inputs[slot].append(new[slot])
            outputs[slot].append(y)

    def rows(n):
        return torch.randn(n, D, generator=g, device="cuda").half()

    def admit():
        slot = server.cache.admit()
        inputs[slot], outputs[slot] = [], []
        return slot

    def leave(slot):
        finished.append((torch.cat(inputs.pop(slot)), torch.cat(outputs.pop(slot))))
        server.cache.release(slot)

    a, b, c = admit(), admit(), admit()
    feed({a: rows(130), b: rows(7), c: rows(61)})        # three prompts at once
    for _ in range(20):
        feed({s: rows(1) for s in (a, b, c)})            # a token each (an idle fourth slot rides along)
    leave(a)
    d = admit()                                          # in the pages that have come free
    feed({d: rows(200), b: rows(1), c: rows(5)})         # a prompt beside a token and five drafted ones
    e = admit()
    feed({e: rows(90)})
    for _ in range(10):
        feed({s: rows(1) for s in (b, c, d, e)})
    for s in (b, c, d, e):
        leave(s)
    torch.cuda.synchronize()
    status = vt.vt_paged_status(server.cache.paged)
    server.cache.close()
    assert status == 0, f"status {status}"
    worst = 0.0
    for x, y in finished:
        ref = alone(layers, x, norms=code is not None)
        worst = max(worst, float((y.double() - ref).norm() / ref.norm()))
    return worst, len(finished)


if __name__ == "__main__":
    err, n = serve(*sys.argv[1:2])
    print(f"{n} sequences served; largest relative error of a sequence's hidden states against 64 bits: {err:.2e}")
