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
