"""What the binding of the few-token layer refuses before the library sees a
pointer, and what it passes on, with tensors that only say what they are."""
import ctypes
import types

import pytest
import torch

from paper_2606_22541_gb300 import api

H = 512


class T:
    def __init__(self, *shape, dtype=torch.bfloat16, ptr=0x1000, strides=None, is_cuda=True):
        self.shape, self.dtype, self.is_cuda, self._ptr, self.device = shape, dtype, is_cuda, ptr, "fake"
        dense = []
        for s in reversed(shape):
            dense.insert(0, dense[0] * last if dense else 1)
            last = s
        self._dense, self._strides = tuple(dense), tuple(strides or dense)

    def stride(self):
        return self._strides

    def is_contiguous(self):
        return all(a == b or s == 1 for a, b, s in zip(self._strides, self._dense, self.shape))

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def element_size(self):
        return self.dtype.itemsize

    def is_floating_point(self):
        return self.dtype.is_floating_point

    def data_ptr(self):
        return self._ptr


@pytest.fixture
def calls(monkeypatch):
    seen = []

    def few(*a):
        seen.append([v.value if isinstance(v, (ctypes.c_void_p, ctypes.c_size_t)) else v for v in a])
        return 0

    monkeypatch.setattr(api, "lib", lambda: types.SimpleNamespace(asap_moe_layer_few=few))
    return seen


def arguments(**change):
    a = dict(h=types.SimpleNamespace(ptr=0x77, cfg=types.SimpleNamespace(hidden=H)), x=T(9, H, ptr=0x2000),
             out=T(9, H, ptr=0x3000), ws=T(4096, dtype=torch.uint8, ptr=0x4000),
             stream=types.SimpleNamespace(cuda_stream=0x55), layer_id=None)
    return a | change


def test_what_is_passed_on(calls):
    api.asap_moe_layer_few(**arguments())
    api.asap_moe_layer_few(**arguments(out=T(64, H, ptr=0x3000), ws=T(100, dtype=torch.float32, ptr=0x4000),
                                       layer_id=T(1, dtype=torch.int32, ptr=0x5000)))
    api.asap_moe_layer_few(**arguments(x=T(1, H, ptr=0x2000, strides=(9 * H, 1)), out=T(1, H, strides=(7, 1), ptr=0x3000)))
    api.asap_moe_layer_few(**arguments(x=T(0, H, ptr=0), out=T(0, H, ptr=0), ws=None))
    # the library says what is wrong with these
    api.asap_moe_layer_few(**arguments(layer_id=T(14, dtype=torch.uint8, ptr=0x5002)))
    api.asap_moe_layer_few(**arguments(x=T(65, H), out=T(65, H)))
    assert calls[0] == [0x77, None, 0x2000, 9, 0x3000, 0x4000, 4096, 0x55]
    assert calls[1] == [0x77, 0x5000, 0x2000, 9, 0x3000, 0x4000, 400, 0x55]
    assert [c[3] for c in calls] == [9, 9, 1, 0, 9, 65]


@pytest.mark.parametrize("change", [
    dict(x=T(9, H, dtype=torch.float32)), dict(x=T(9, H, dtype=torch.float16)), dict(x=T(9, H, is_cuda=False)),
    dict(x=T(9, H, strides=(2 * H, 1))), dict(x=T(9, H, strides=(1, 9))), dict(x=T(9, H - 256)), dict(x=T(9, 2 * H)),
    dict(x=T(9 * H)), dict(out=T(8, H)), dict(out=T(9, H, dtype=torch.float32)), dict(out=T(9, H, is_cuda=False)),
    dict(out=T(9, H, strides=(H + 8, 1))), dict(out=T(9, H - 256)), dict(out=T(9, H, strides=(0, 1))),
    dict(ws=T(4096, dtype=torch.uint8, is_cuda=False)), dict(ws=T(4096, dtype=torch.uint8, strides=(2,))),
    dict(ws=T(64, 64, dtype=torch.uint8, strides=(0, 1))),
    dict(layer_id=T(1, dtype=torch.int32, is_cuda=False)), dict(layer_id=T(0, dtype=torch.int32)),
    dict(layer_id=T(1, dtype=torch.float32)), dict(layer_id=T(3, dtype=torch.uint8))],
    ids=lambda c: next(iter(c)))
def test_what_is_refused(calls, change):
    with pytest.raises(ValueError):
        api.asap_moe_layer_few(**arguments(**change))
    assert not calls
