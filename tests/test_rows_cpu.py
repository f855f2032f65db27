"""Pure-host behaviour of the operators around a training step's expert products:
workspace sizes, constants and refusals that need no GPU."""
import os
import re

import pytest
import torch

from paper_2606_22541_gb300 import _native, api, build as build_mod

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "asap_moe.h")
INVALID, OK, WORKSPACE = _native.ASAP_ERR_INVALID, _native.ASAP_OK, _native.ASAP_ERR_WORKSPACE
P = 1 << 20   # an address that nothing reads


@pytest.fixture(scope="module")
def L():
    build_mod.build()
    return _native.lib()


def test_constants_of_the_header():
    text = open(HEADER).read()
    assert int(re.search(r"#define ASAP_MOE_SORT_MAX_EXPERTS (\d+)", text).group(1)) == api.SORT_MAX_EXPERTS
    for name, t in (("BF16", torch.bfloat16), ("F16", torch.float16), ("F32", torch.float32)):
        assert int(re.search(rf"ASAP_ELEM_{name} = (\d+)", text).group(1)) == api._ELEM[t]
    assert int(re.search(r"ASAP_ELEM_E4M3 = (\d+)", text).group(1)) == api._BYTES[torch.float8_e4m3fn]


@pytest.mark.parametrize("k,experts", [(1, 1), (2, 8), (8, 256), (17, 1024)])
def test_workspace_of_more_entries_serves_fewer(L, k, experts):
    sizes = [api.asap_moe_sort_workspace_size(n, k, experts) for n in range(0, 40000, 577)]
    assert sizes[0] == 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))
    assert api.asap_moe_sort_workspace_size((1 << 31) // k - 1, k, experts) >= sizes[-1] if k > 1 else True


@pytest.mark.parametrize("n,k,experts", [(-1, 1, 8), (1, 0, 8), (1, 1, 0), (1, 1, 1025), (1 << 29, 4, 8),
                                         ((1 << 30) + 1, 1, 8)])
def test_sort_sizes_refused(L, n, k, experts):
    with pytest.raises(_native.AsapError):
        api.asap_moe_sort_workspace_size(n, k, experts)
    assert L.asap_moe_sort(P, n, k, experts, P, P, None, P, 1 << 40, None) == INVALID


def test_sort_refused(L):
    assert L.asap_moe_sort(None, 1, 1, 8, P, P, None, None, 0, None) == INVALID
    assert L.asap_moe_sort(P, 1, 1, 8, None, P, None, None, 0, None) == INVALID
    assert L.asap_moe_sort(P, 1, 1, 8, P, None, None, None, 0, None) == INVALID
    assert L.asap_moe_sort(P + 2, 1, 1, 8, P, P, None, None, 0, None) == INVALID
    need = api.asap_moe_sort_workspace_size(60000, 8, 256)
    assert need > 0
    assert L.asap_moe_sort(P, 60000, 8, 256, P, P, None, P, need - 1, None) == WORKSPACE
    assert L.asap_moe_sort(P, 60000, 8, 256, P, P, None, None, need, None) == WORKSPACE
    assert L.asap_moe_sort(P, 60000, 8, 256, P, P, None, P + 2, need, None) == WORKSPACE


# argument lists that would launch; a change of one of them is refused before anything is enqueued
CALLS = {
    "permute": dict(type=0, x=P, ldx=64, n=4, cols=64, perm=P, k=2, y=P, ldy=64, rows=8, status=None, stream=None),
    "unpermute": dict(type=0, y=P, ldy=64, rows=8, cols=64, w=P, perm=P, n=4, k=2, out=P, ldo=64, status=None, stream=None),
    "unpermute_backward": dict(type=0, d=P, ldo=64, y=P, ldy=64, w=P, perm=P, n=4, k=2, cols=64, dy=P, ldd=64, rows=8,
                               dw=P, status=None, stream=None),
    "fp8_dequantize": dict(type=0, q=P, ldq=64, s=P, lds=1, n=4, cols=64, perm=P, k=2, x=P, ldx=64, rows=8, status=None,
                           stream=None),
    "swiglu_save": dict(type=0, gate=P, up=P, ld=64, rows=8, cols=64, n_rows=None, h=P, ldh=64, gq=P, uq=P, ldq=64, gs=P,
                        us=P, lds=1, stream=None),
    "swiglu_backward": dict(type=0, d=P, ldd=64, gq=P, uq=P, ldq=64, gs=P, us=P, lds=1, rows=8, cols=64, n_rows=None,
                            dg=P, du=P, ldg=64, h=P, ldh=64, stream=None),
}
BIG = (1 << 30) + 1
CHANGES = [("permute", c) for c in (
    dict(type=4), dict(type=-1), dict(n=-1), dict(n=BIG), dict(cols=-1), dict(cols=BIG), dict(rows=-1), dict(rows=BIG),
    dict(k=0), dict(k=1 << 30), dict(x=None), dict(perm=None), dict(y=None), dict(x=P + 1), dict(y=P + 1), dict(perm=P + 2),
    dict(ldx=63), dict(ldy=63), dict(ldx=-64), dict(status=P + 1))]
CHANGES += [("unpermute", c) for c in (
    dict(type=3), dict(n=-1), dict(k=0), dict(k=1 << 30), dict(y=None), dict(out=None), dict(perm=None), dict(w=P + 2),
    dict(y=P + 1), dict(out=P + 1), dict(ldy=63), dict(ldo=0), dict(rows=BIG), dict(cols=-5), dict(status=P + 3))]
CHANGES += [("unpermute_backward", c) for c in (
    dict(type=3), dict(n=BIG), dict(k=-1), dict(d=None), dict(y=None), dict(perm=None), dict(dw=P + 2), dict(dy=P + 1),
    dict(type=2, y=P + 2), dict(ldo=63), dict(ldy=63), dict(ldd=63), dict(rows=-1))]
CHANGES += [("fp8_dequantize", c) for c in (
    dict(type=3), dict(perm=None), dict(perm=None, k=1), dict(q=None), dict(s=None), dict(s=P + 2), dict(x=None),
    dict(lds=0), dict(ldq=63), dict(ldx=63), dict(x=P + 1), dict(n=-2), dict(k=0))]
CHANGES += [("swiglu_save", c) for c in (
    dict(type=3), dict(rows=-1), dict(cols=BIG), dict(gate=None), dict(up=None), dict(h=None), dict(gq=None), dict(uq=None),
    dict(gs=None), dict(us=P + 2), dict(gate=P + 1), dict(ld=63), dict(ldh=63), dict(ldq=63), dict(lds=0),
    dict(n_rows=P + 2))]
CHANGES += [("swiglu_backward", c) for c in (
    dict(type=3), dict(rows=BIG), dict(d=None), dict(dg=None), dict(du=None), dict(gq=None), dict(us=None), dict(ldd=63),
    dict(ldg=63), dict(ldh=63), dict(h=P + 1), dict(lds=0), dict(n_rows=P + 1))]


@pytest.mark.parametrize("call,change", CHANGES, ids=lambda v: v if isinstance(v, str) else "-".join(v))
def test_refused_by_the_library(L, call, change):
    assert getattr(L, "asap_moe_" + call)(*(CALLS[call] | change).values()) == INVALID
    assert api.asap_moe_last_error()


@pytest.mark.parametrize("call,empty", [
    ("permute", dict(n=0)), ("permute", dict(cols=0)), ("unpermute", dict(n=0)), ("unpermute", dict(cols=0)),
    ("unpermute_backward", dict(n=0)), ("unpermute_backward", dict(dw=None, dy=None)),
    ("unpermute_backward", dict(dw=None, cols=0)), ("fp8_dequantize", dict(n=0)), ("fp8_dequantize", dict(cols=0)),
    ("swiglu_save", dict(rows=0)), ("swiglu_save", dict(cols=0)), ("swiglu_backward", dict(rows=0)),
    ("swiglu_backward", dict(cols=0))], ids=lambda v: v if isinstance(v, str) else "-".join(v))
def test_nothing_to_do_is_no_error(L, call, empty):
    assert getattr(L, "asap_moe_" + call)(*(CALLS[call] | empty).values()) == OK


def test_the_binding_refuses_host_tensors_and_misfits():
    i32 = dict(dtype=torch.int32)
    idx, off, perm = torch.zeros(4, 2, **i32), torch.zeros(9, **i32), torch.zeros(4, 2, **i32)
    x, y, w = torch.zeros(4, 64), torch.zeros(8, 64), torch.zeros(4, 2)
    q, s = torch.zeros(8, 64, dtype=torch.float8_e4m3fn), torch.zeros(8, 1)
    for call in (lambda: api.asap_moe_sort(idx, 8, off, perm),                       # not on a GPU
                 lambda: api.asap_moe_sort(idx.long(), 8, off, perm), lambda: api.asap_moe_sort(idx, 9, off, perm),
                 lambda: api.asap_moe_permute(x, perm, y), lambda: api.asap_moe_permute(x.long(), perm, y.long()),
                 lambda: api.asap_moe_permute(x, perm[:3], y), lambda: api.asap_moe_permute(x, perm, y.half()),
                 lambda: api.asap_moe_unpermute(y, w, perm, x), lambda: api.asap_moe_unpermute(y, w.double(), perm, x),
                 lambda: api.asap_moe_unpermute(y[:, :32], w, perm, x),
                 lambda: api.asap_moe_unpermute_backward(x, y, w, perm, y, w),
                 lambda: api.asap_moe_unpermute_backward(x, None, w, perm, y, w),
                 lambda: api.asap_moe_unpermute_backward(x, y, w, perm, y[:7], w),
                 lambda: api.asap_moe_fp8_dequantize(q, s, y), lambda: api.asap_moe_fp8_dequantize(q, s, y[:4]),
                 lambda: api.asap_moe_fp8_dequantize(q, s[:4], y, perm),
                 lambda: api.asap_moe_swiglu_save(y, y, y, q, s, q, s),
                 lambda: api.asap_moe_swiglu_save(y, y.half(), y, q, s, q, s),
                 lambda: api.asap_moe_swiglu_save(y, y, y, q, s, q[:, :32], s),
                 lambda: api.asap_moe_swiglu_backward(y, q, s, q, s, y, y, y),
                 lambda: api.asap_moe_permute(x, perm, y, status=torch.zeros(1, **i32))):
        with pytest.raises(ValueError):
            call()


# ------------------------------------------------------------------ the compiled marshalling

class T:
    """What the compiled marshalling looks at of a tensor."""

    def __init__(self, shape, dtype, ptr, strides=None, device=3):
        self.shape, self.dtype, self._ptr, self._device = tuple(shape), dtype, ptr, device
        self._strides = strides or tuple([shape[1], 1] if len(shape) == 2 else [1])

    def get_device(self):
        return self._device

    def stride(self):
        return self._strides

    def data_ptr(self):
        return self._ptr


BF16, F16, F32, F8, U8, I32 = (object() for _ in range(6))
NAMES = ["sort", "permute", "unpermute", "unpermute_backward", "swiglu_save", "swiglu_backward", "dequantize"]


@pytest.fixture
def calls():
    import ctypes
    build_mod.build()
    marshal = pytest.importorskip("paper_2606_22541_gb300._marshal")
    seen = []
    none = [ctypes.CFUNCTYPE(ctypes.c_int32)(lambda: 0) for _ in range(3)]
    entry = ["asap_moe_fp8_dequantize" if n == "dequantize" else "asap_moe_" + n for n in NAMES]
    fns = [ctypes.CFUNCTYPE(ctypes.c_int32, *_native.SIGNATURES[e])(lambda *a, n=n: seen.append((n,) + a) or 7)
           for n, e in zip(NAMES, entry)]
    address = lambda f: ctypes.cast(f, ctypes.c_void_p).value
    marshal.bind(*map(address, none), BF16, F32, F8, U8, lambda: 3, lambda d: 0x90 + d)
    marshal.bind_rows(*map(address, fns), F16, I32)
    yield marshal, seen
    _native._fast = None  # bound to the library again by its next user


def arguments():
    perm, w = T((6, 2), I32, 0x10), T((6, 2), F32, 0x20)
    x, y = T((6, 100), F16, 0x30, (104, 1)), T((12, 100), F16, 0x40, (112, 1))
    q, s = T((12, 300), F8, 0x50, (304, 1)), T((12, 3), F32, 0x60, (4, 1))
    q2, s2 = T((12, 300), U8, 0x51, (304, 1)), T((12, 3), F32, 0x61, (4, 1))
    g, u, h = T((12, 300), BF16, 0x70, (600, 1)), T((12, 300), BF16, 0x71, (600, 1)), T((12, 300), BF16, 0x72)
    count = T((1,), I32, 0x80)
    return dict(
        sort=[perm, 8, T((9,), I32, 0xA0), T((6, 2), I32, 0xB0), T((512,), U8, 0xC0), T((12,), I32, 0xD0), None],
        permute=[x, perm, y, None, None], unpermute=[y, w, perm, x, None, None],
        unpermute_backward=[x, y, w, perm, T((12, 100), F16, 0x41), T((6, 2), F32, 0x21), None, None],
        swiglu_save=[g, u, h, q, s, q2, s2, None, count], swiglu_backward=[h, q, s, q2, s2, g, u, None, None, None],
        dequantize=[T((6, 300), F8, 0x52), T((6, 3), F32, 0x62), T((12, 300), F32, 0x73), perm, None, None])


def test_marshalled(calls):
    marshal, seen = calls
    want = dict(
        sort=(0x10, 6, 2, 8, 0xA0, 0xB0, 0xD0, 0xC0, 512, 0x93),
        permute=(1, 0x30, 104, 6, 100, 0x10, 2, 0x40, 112, 12, None, 0x93),
        unpermute=(1, 0x40, 112, 12, 100, 0x20, 0x10, 6, 2, 0x30, 104, None, 0x93),
        unpermute_backward=(1, 0x30, 104, 0x40, 112, 0x20, 0x10, 6, 2, 100, 0x41, 100, 12, 0x21, None, 0x93),
        swiglu_save=(0, 0x70, 0x71, 600, 12, 300, 0x80, 0x72, 300, 0x50, 0x51, 304, 0x60, 0x61, 4, 0x93),
        swiglu_backward=(0, 0x72, 300, 0x50, 0x51, 304, 0x60, 0x61, 4, 12, 300, None, 0x70, 0x71, 600, None, 0, 0x93),
        dequantize=(2, 0x52, 300, 0x62, 3, 6, 300, 0x10, 2, 0x73, 300, 12, None, 0x93))
    for name in NAMES:
        assert getattr(marshal, name)(*arguments()[name]) == 7
        assert seen.pop() == (name,) + want[name]
    a = arguments()
    a["sort"][4] = a["sort"][5] = None
    assert marshal.sort(*a["sort"]) == 7 and seen.pop()[7:10] == (None, None, 0)
    a["unpermute"][1] = None
    assert marshal.unpermute(*a["unpermute"]) == 7 and seen.pop()[6] is None
    a["dequantize"][3], a["dequantize"][2] = None, T((6, 300), BF16, 1)
    assert marshal.dequantize(*a["dequantize"]) == 7 and seen.pop()[8:10] == (None, 1)
    a["permute"][0], a["permute"][2] = T((6, 100), U8, 1), T((12, 100), U8, 1)
    assert marshal.permute(*a["permute"]) == 7 and seen.pop()[1] == 3


@pytest.mark.parametrize("name", NAMES)
def test_what_does_not_fit_is_left_to_the_checks(calls, name):
    """Every tensor in turn on another device, of another type, shape or stride, or no tensor at all."""
    marshal, seen = calls
    good = arguments()[name]
    for i, t in enumerate(good):
        if not isinstance(t, T):
            continue
        two = len(t.shape) == 2
        others = [T(t.shape, t.dtype, 1, t._strides, device=2), T(t.shape, t.dtype, 1, t._strides, device=-1),
                  T(t.shape, object(), 1, t._strides), T(t.shape + (1,), t.dtype, 1, t._strides + (1,)), 5]
        if two:
            if not (t.dtype is I32 and name in ("permute", "dequantize")):   # (any number of places a token)
                others.append(T((t.shape[0], t.shape[1] + 129), t.dtype, 1))
            others += [T((0, t.shape[1]), t.dtype, 1), T(t.shape, t.dtype, 1, (t._strides[0], 2))]
        if not (name == "sort" and i == 4):   # (a workspace of any length)
            others += [T((t.shape[0] + 1,) + t.shape[1:], t.dtype, 1)] if not two or t.dtype is I32 else []
        for o in others:
            assert getattr(marshal, name)(*good[:i], o, *good[i + 1:]) is None, (i, vars(o) if isinstance(o, T) else o)
    assert getattr(marshal, name)(*good[:-1]) is None and getattr(marshal, name)() is None
    assert not seen
