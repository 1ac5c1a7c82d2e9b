"""What the paged calls with norms, other rotations and pools in 8 bits refuse (no GPU: nothing here launches a
kernel; pointers are only looked at)."""
from __future__ import annotations

import ctypes
import types

import pytest

torch = pytest.importorskip("torch")
from paper_2607_07046_gb300 import vt  # noqa: E402
from tests.test_paged_devices import Stand  # noqa: E402

PTR = 1 << 20  # aligned, never read


def copied(struct, **kw):
    new = type(struct)()
    ctypes.memmove(ctypes.addressof(new), ctypes.addressof(struct), ctypes.sizeof(new))
    for name, value in kw.items():
        setattr(new, name, value)
    return new


@pytest.fixture()
def parts(vtlib):
    handle = ctypes.create_string_buffer(512)  # what a refused call does not get to use
    pool = vt.vt_paged_pool(PTR, PTR, vt.VT_F16, 4, 16, 2, 64, 2048, 1024, 64)
    mx = vt.vt_paged_mx_pool(PTR, PTR, PTR, PTR, vt.VT_F16, vt.VT_MX_E4M3, 4, 16, 2, 64, 2048, 1024, 64, 64, 32)
    batch = vt.vt_paged_batch(PTR, PTR, None, 2, 3)
    form = vt.vt_qk_form(PTR, PTR, PTR, 48, 32, vt.VT_ROPE_HALVES, 1e-6)
    return types.SimpleNamespace(g=ctypes.addressof(handle), handle=handle, pool=pool, mx=mx, batch=batch, form=form)


def append(s, call, **kw):
    a = dict(g=s.g, pool=s.mx if call == "mx" else s.pool, batch=s.batch, rows=2, heads=4, q=PTR, ql=256, k=PTR, kl=256, v=PTR, vl=256,
             form=s.form, out=PTR, ol=256)
    a.update(kw)
    f = getattr(vt.lib(), "vt_paged_append_" + call)
    return f(a["g"], a["pool"], a["batch"], a["rows"], a["heads"], a["q"], a["ql"], a["k"], a["kl"], a["v"], a["vl"], a["form"], a["out"],
             a["ol"], None)


@pytest.mark.parametrize("call", ["qk", "mx"])
def test_append(parts, call):
    s, inv, shape = parts, vt.VT_ERR_INVALID_ARG, vt.VT_ERR_SHAPE
    cases = [({"g": None}, inv), ({"pool": None}, inv), ({"batch": None}, inv), ({"form": None}, inv), ({"rows": 3}, inv),
             ({"rows": -1}, inv), ({"heads": 5}, shape), ({"heads": 0}, shape), ({"heads": 2 * 129}, shape), ({"q": None}, inv),
             ({"k": None}, inv), ({"v": PTR + 8}, inv), ({"out": PTR + 2}, inv), ({"ql": 255}, inv), ({"kl": 64}, inv), ({"vl": 132}, inv),
             ({"ol": 250}, inv)]
    for kw, want in (({"rotary_dim": 8}, shape), ({"rotary_dim": 40}, shape), ({"rotary_dim": 80}, shape), ({"rotary_dim": -16}, shape),
                     ({"rope": None}, inv), ({"rope": PTR + 8}, inv), ({"rope_len": 0}, inv), ({"pairs": 2}, inv), ({"pairs": -1}, inv),
                     ({"eps": -1e-6}, inv), ({"eps": float("nan")}, inv), ({"eps": float("inf")}, inv), ({"q_gain": PTR + 8}, inv),
                     ({"k_gain": PTR + 2}, inv)):
        cases.append(({"form": copied(s.form, **kw)}, want))
    for kw, want in cases:
        assert append(s, call, **kw) == want, kw
        assert vt.vt_last_error()


def test_no_rows_is_nothing(parts):
    s = parts
    none = copied(s.batch, n_seqs=0)
    for call in ("qk", "mx"):
        assert append(s, call, batch=none, rows=0, q=None, k=None, v=None, out=None) == vt.VT_OK
        # without a rotation its table is not looked at
        assert append(s, call, batch=none, rows=0, form=copied(s.form, rotary_dim=0, rope=None, rope_len=0, q_gain=None, k_gain=None)) == vt.VT_OK
    L = vt.lib()
    assert L.vt_paged_decode_mx(s.g, s.mx, none, 4, None, 0, 0.1, 0, None, 0, None) == vt.VT_OK
    assert L.vt_paged_prefill_mx(s.g, s.mx, none, 0, 4, None, 0, 0.1, 0, None, 0, None) == vt.VT_OK


def test_pools_in_8_bits(parts):
    s, L, inv, shape = parts, vt.lib(), vt.VT_ERR_INVALID_ARG, vt.VT_ERR_SHAPE
    cases = [({"format": 2}, shape), ({"format": -1}, shape), ({"dtype": 2}, shape), ({"page_size": 4}, shape), ({"page_size": 1}, shape),
             ({"page_size": 24}, shape), ({"page_size": 2048}, shape), ({"d_head": 96}, shape), ({"d_head": 32}, shape),
             ({"n_kv_heads": 0}, shape), ({"n_pages": 0}, inv), ({"k": None}, inv), ({"v": PTR + 8}, inv), ({"k_scale": None}, inv),
             ({"v_scale": None}, inv), ({"k_scale": PTR + 4}, inv), ({"page_stride": 2040}, inv), ({"head_stride": 1032}, inv),
             ({"pos_stride": 72}, inv), ({"pos_stride": 48}, inv), ({"pos_stride": 0}, inv), ({"page_stride": -2048}, inv),
             ({"page_stride": 1 << 41}, inv), ({"scale_page_stride": 16}, inv), ({"scale_head_stride": 24}, inv),
             ({"scale_head_stride": 40}, inv), ({"scale_page_stride": -64}, inv), ({"scale_page_stride": 1 << 41}, inv)]
    for kw, want in cases:
        bad = copied(s.mx, **kw)
        assert append(s, "mx", pool=bad) == want, kw
        assert L.vt_paged_decode_mx(s.g, bad, s.batch, 4, PTR, 256, 0.1, 0, PTR, 256, None) == want, kw
        assert L.vt_paged_prefill_mx(s.g, bad, s.batch, 2, 4, PTR, 256, 0.1, 0, PTR, 256, None) == want, kw
        assert vt.vt_last_error()


def test_attention(parts):
    s, L, inv, shape = parts, vt.lib(), vt.VT_ERR_INVALID_ARG, vt.VT_ERR_SHAPE
    good = dict(g=s.g, pool=s.mx, batch=s.batch, rows=2, heads=4, q=PTR, ql=256, scale=0.1, window=0, out=PTR, ol=256)
    cases = [({"g": None}, inv), ({"pool": None}, inv), ({"batch": None}, inv), ({"heads": 3}, shape), ({"q": None}, inv), ({"q": PTR + 8}, inv),
             ({"out": None}, inv), ({"ql": 8}, inv), ({"ol": 260}, inv), ({"scale": float("nan")}, inv), ({"scale": -1.0}, inv),
             ({"scale": float("inf")}, inv), ({"window": -1}, inv)]
    for kw in ({"tables": None}, {"lens": None}, {"n_seqs": -1}, {"n_seqs": 16385}, {"pages_per_seq": 0}, {"pages_per_seq": 1 << 27}):
        cases.append(({"batch": copied(s.batch, **kw)}, inv))
    for kw, want in cases:
        a = dict(good, **kw)
        tail = (a["heads"], a["q"], a["ql"], a["scale"], a["window"], a["out"], a["ol"], None)
        assert L.vt_paged_decode_mx(a["g"], a["pool"], a["batch"], *tail) == want, kw
        rows = a["batch"].n_seqs if a["batch"] is not None else 2
        assert L.vt_paged_prefill_mx(a["g"], a["pool"], a["batch"], rows, *tail) == want, kw
        assert vt.vt_last_error()
    started = copied(s.batch, starts=PTR)
    assert L.vt_paged_decode_mx(s.g, s.mx, started, 4, PTR, 256, 0.1, 0, PTR, 256, None) == inv
    assert L.vt_paged_prefill_mx(s.g, s.mx, s.batch, 3, 4, PTR, 256, 0.1, 0, PTR, 256, None) == inv
    assert L.vt_paged_prefill_mx(s.g, s.mx, started, 1 << 25, 4, PTR, 256, 0.1, 0, PTR, 256, None) == inv


# ------------------------------------------------------------------ the binding

@pytest.fixture()
def reached(monkeypatch):
    """The names of the library's functions that were called."""
    names = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: names.append(name) or 0

    monkeypatch.setattr(vt, "lib", lambda: Lib())
    monkeypatch.setattr(vt, "_ptr", lambda t, dtype=None: 0 if t is None else t.data_ptr())
    return names


def calls(gain=None, rope_device=0):
    pool = types.SimpleNamespace(device=0, d_head=64, n_kv_heads=1, torch_dtype=torch.float16)
    q = Stand((2, 1, 64), 0)
    form = vt.make_qk_form(Stand((8, 32, 2), rope_device, torch.float32), False, gain)
    return {"append_qk": lambda b: vt.vt_paged_append_qk(1, pool, b, q, q, q, form, q, stream=0),
            "append_mx": lambda b: vt.vt_paged_append_mx(1, pool, b, q, q, q, form, q, stream=0),
            "decode_mx": lambda b: vt.vt_paged_decode_mx(1, pool, b, q, q, stream=0),
            "prefill_mx": lambda b: vt.vt_paged_prefill_mx(1, pool, b, q, q, stream=0)}


def batch(device):
    return vt.make_paged_batch(Stand((2, 4), device, torch.int32), Stand((2,), device, torch.int32))


@pytest.mark.parametrize("call", ["append_qk", "append_mx", "decode_mx", "prefill_mx"])
def test_batch_of_another_device(reached, call):
    calls()[call](batch(0))
    assert reached == ["vt_paged_" + call]
    with pytest.raises(ValueError):
        calls()[call](batch(1))
    assert len(reached) == 1


@pytest.mark.parametrize("call", ["append_qk", "append_mx"])
def test_forms_that_do_not_fit(reached, call):
    with pytest.raises(ValueError):
        calls(rope_device=1)[call](batch(0))
    with pytest.raises(ValueError):  # rope and gain on two devices
        calls(gain=Stand((64,), 1))
    for gain in (Stand((128,), 0), Stand((64,), 0, torch.bfloat16)):
        with pytest.raises(ValueError):
            calls(gain=gain)[call](batch(0))
    for gain in (Stand((64, 1), 0), Stand((64,), 0, torch.float32)):
        with pytest.raises(ValueError):
            calls(gain=gain)
    for rope in (Stand((8, 32), 0, torch.float32), Stand((8, 32, 3), 0, torch.float32)):
        with pytest.raises(ValueError):
            vt.make_qk_form(rope)
    assert reached == []


def test_pools_that_do_not_fit():
    with pytest.raises(ValueError):
        t = torch.zeros(2, 1, 16, 64, dtype=torch.int8)
        vt.make_paged_mx_pool(t, t, t[..., :2], t[..., :2], torch.float16)  # not on a GPU
