"""The paged calls refuse tensors of another device than the pool's before the library sees them (no GPU: the
tensors are stand-ins)."""
from __future__ import annotations

import types

import pytest

torch = pytest.importorskip("torch")
from paper_2607_07046_gb300 import vt  # noqa: E402


class Stand:
    """What the checks ask of a contiguous CUDA tensor."""
    is_cuda = True

    def __init__(self, shape, device, dtype=torch.float16):
        self.shape, self.device, self.dtype = tuple(shape), torch.device("cuda", device), dtype

    def get_device(self):
        return self.device.index

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        s = [1]
        for n in self.shape[:0:-1]:
            s.insert(0, s[0] * n)
        return tuple(s) if i is None else s[i]

    def numel(self):
        n = 1
        for x in self.shape:
            n *= x
        return n

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 256


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


def calls(rope_device=0):
    pool = types.SimpleNamespace(device=0, d_head=64, n_kv_heads=1, torch_dtype=torch.float16)
    q, rope = Stand((2, 1, 64), 0), Stand((8, 32, 2), rope_device, torch.float32)
    return {"append": lambda b: vt.vt_paged_append(1, pool, b, q, q, q, rope, q, stream=0),
            "decode": lambda b: vt.vt_paged_decode(1, pool, b, q, q, stream=0),
            "prefill": lambda b: vt.vt_paged_prefill(1, pool, b, q, q, stream=0)}


def batch(device):
    return vt.make_paged_batch(Stand((2, 4), device, torch.int32), Stand((2,), device, torch.int32))


@pytest.mark.parametrize("call", ["append", "decode", "prefill"])
def test_batch_of_another_device(reached, call):
    calls()[call](batch(0))
    assert reached == ["vt_paged_" + call]
    with pytest.raises(ValueError):
        calls()[call](batch(1))
    assert len(reached) == 1


def test_rotation_table_of_another_device(reached):
    with pytest.raises(ValueError):
        calls(rope_device=1)["append"](batch(0))
    assert reached == []
