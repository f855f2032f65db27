"""The compiled marshalling of the short calls against recorded calls: what it
passes on for tensors that fit, and that it leaves everything else alone."""
import ctypes

import pytest

from paper_2606_22541_gb300 import _native, build as build_mod

build_mod.build()
marshal = pytest.importorskip("paper_2606_22541_gb300._marshal")

BF16, F32, F8, U8 = object(), object(), object(), object()
P, L, I = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32


class T:
    """What the marshalling looks at of a tensor."""

    def __init__(self, rows, cols, dtype, ptr, strides=None, is_cuda=True):
        self.shape, self.dtype, self.is_cuda = (rows, cols), dtype, is_cuda
        self._strides, self._ptr = strides or (cols, 1), ptr

    def stride(self):
        return self._strides

    def data_ptr(self):
        return self._ptr


class Stream:
    cuda_stream = 0x55


@pytest.fixture
def calls():
    seen = []

    def recorder(*types):
        return ctypes.CFUNCTYPE(I, *types)(lambda *a: seen.append(a) or 7)

    q = recorder(P, L, I, I, P, L, P, L, P)
    s = recorder(P, P, L, I, I, P, L, P, L, P)
    m = recorder(P, L, P, L, P, L, P, L, P, L, I, I, I, P, P)
    marshal.bind(*(ctypes.cast(f, P).value for f in (q, s, m)), BF16, F32, F8, U8, lambda: 3, lambda d: 0x90 + d)
    yield seen
    _native._fast = None  # bound to the library again by its next user


def test_quantize(calls):
    x, q, s = T(5, 300, BF16, 0x1000, (640, 1)), T(5, 300, F8, 0x2000, (304, 1)), T(5, 3, F32, 0x3000)
    assert marshal.quantize(x, q, s, None) == 7
    assert marshal.quantize(T(1, 300, BF16, 1 << 40, (1, 1)), T(1, 300, U8, 0x20), T(1, 3, F32, 0x30), Stream()) == 7
    assert calls == [(0x1000, 640, 5, 300, 0x2000, 304, 0x3000, 3, 0x93),
                     (1 << 40, 304, 1, 300, 0x20, 304, 0x30, 16, 0x55)]


def test_swiglu(calls):
    g, u = T(4, 200, BF16, 0x10, (400, 1)), T(4, 200, BF16, 0x1A0, (400, 1))
    q, s = T(4, 200, F8, 0x5000, (208, 1)), T(4, 2, F32, 0x6000, (9, 1))
    assert marshal.swiglu_quantize(g, u, q, s, None) == 7
    assert calls == [(0x10, 0x1A0, 400, 4, 200, 0x5000, 208, 0x6000, 9, 0x93)]
    assert marshal.swiglu_quantize(g, T(4, 200, BF16, 0x1A0, (401, 1)), q, s, None) is None  # another row stride
    assert len(calls) == 1


def operands(m=6, n=260, k=500):
    return dict(a=T(m, k, F8, 0x100, (512, 1)), sa=T(m, 4, F32, 0x200), b=T(n, k, U8, 0x300, (1024, 1)),
                sb=T(3, 4, F32, 0x400, (4, 1)), out=T(m, n, BF16, 0x500, (264, 1)), stream=None, status=None)


def test_matmul(calls):
    assert marshal.matmul(*operands().values()) == 7
    assert calls == [(0x100, 512, 0x200, 4, 0x300, 1024, 0x400, 4, 0x500, 264, 6, 260, 500, None, 0x93)]
    marshal.matmul(*(operands() | dict(status=T(1, 1, F32, 0x700))).values())
    assert calls[1][13] == 0x700


@pytest.mark.parametrize("change", [
    dict(a=T(6, 500, BF16, 1)), dict(a=T(6, 499, F8, 1)), dict(a=T(6, 500, F8, 1, (500, 2))), dict(a=T(0, 500, F8, 1)),
    dict(a=T(6, 500, F8, 1, is_cuda=False)), dict(a=T(6, 500, F8, 1, (0, 1))), dict(sa=T(6, 3, F32, 1)),
    dict(sa=T(5, 4, F32, 1)), dict(sb=T(2, 4, F32, 1)), dict(sb=T(3, 4, BF16, 1)), dict(b=T(260, 500, F32, 1)),
    dict(out=T(6, 261, BF16, 1)), dict(out=T(7, 260, BF16, 1)), dict(out=None), dict(a=3), dict(status=4),
    dict(stream=4), dict(a=T((1 << 30) + 1, 500, F8, 1))], ids=lambda c: next(iter(c)))
def test_what_does_not_fit_is_left_alone(calls, change):
    assert marshal.matmul(*(operands() | change).values()) is None and not calls


def test_wrong_counts_and_attributes(calls):
    class Odd(T):
        def stride(self):
            raise RuntimeError("sparse")

    class Three(T):
        def __init__(self):
            super().__init__(1, 1, BF16, 1)
            self.shape = (1, 1, 1)

    q, s = T(5, 300, F8, 1), T(5, 3, F32, 1)
    assert marshal.quantize() is None and marshal.quantize(1, 2) is None
    assert marshal.quantize(Odd(5, 300, BF16, 1), q, s, None) is None
    assert marshal.quantize(Three(), q, s, None) is None
    assert marshal.quantize(T(5, 300, BF16, 1), T(5, 299, F8, 1), s, None) is None
    assert not calls
