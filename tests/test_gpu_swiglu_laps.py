"""SwiGLU with kept activations on more groups of 128 columns than a grid has teams:
each team then takes a group, the one a lap further on, and so on, backward with the
next one's loads out before this one's results are written.  Rows all differ, and every
row is compared bit by bit with the same rows in calls of less than one lap, those
with float64."""
import math

import pytest
import torch

from paper_2606_22541_gb300 import api

pytestmark = pytest.mark.gpu
DEV, F8 = "cuda", torch.float8_e4m3fn
U = 2.0 ** -24
SMS, THREADS = 152, 256
# (rows, columns): columns an access 8 (4 in fp32), 8, 4, 2, 1, and many short rows; the groups of a row divide the teams
# of a lap only in the first
SHAPES = [(16384, 2048), (9000, 2184), (9000, 2180), (9000, 2186), (9000, 2187), (70000, 264)]


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def access(c, dtype):
    return next(v for v in ((8, 4, 2, 1) if dtype.itemsize == 2 else (4, 2, 1)) if c % v == 0)


def lap(c, dtype, forward):
    """Groups that the largest grid takes at once."""
    v = access(c, dtype)
    team = (8 if v >= 4 else 16) if forward else (16 if v == 8 else 32)
    return SMS * (16 if forward else 40) * (THREADS // team)


def randn(shape, seed, std=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV) * std


def both(y, d, dtype, n_rows=None):
    """Everything that the two calls write: 3 (scales 7, codes NaN) where they write nothing."""
    n, c = d.shape
    b = -(-c // 128)
    q = torch.full((n, 2 * c), 0x7F, dtype=torch.uint8, device=DEV).view(F8)
    s = torch.full((n, 2 * b), 7.0, device=DEV)
    h, h2 = torch.full((n, c), 3.0, dtype=dtype, device=DEV), torch.full((n, c), 3.0, dtype=dtype, device=DEV)
    d_y = torch.full((n, 2 * c), 3.0, dtype=dtype, device=DEV)
    parts = (q[:, :c], s[:, :b], q[:, c:], s[:, b:])
    api.asap_moe_swiglu_save(y[:, :c], y[:, c:], h, *parts, n_rows=n_rows)
    api.asap_moe_swiglu_backward(d, *parts, d_y[:, :c], d_y[:, c:], h2, n_rows=n_rows)
    return q.view(torch.uint8), s, h, d_y, h2


@pytest.mark.parametrize("n,c", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_every_lap(n, c, dtype):
    groups = -(-c // 128)
    assert n * groups > lap(c, dtype, True) and n * groups > lap(c, dtype, False)
    y, d = randn((n, 2 * c), n + c).to(dtype), randn((n, c), c, 0.1).to(dtype)
    got = both(y, d, dtype)
    part = 8 * (min(lap(c, dtype, True), lap(c, dtype, False)) // (8 * groups))
    assert part * groups <= min(lap(c, dtype, True), lap(c, dtype, False)) and part < n
    for r in range(0, n, part):
        for a, b in zip(got, both(y[r:r + part], d[r:r + part], dtype)):
            assert torch.equal(a[r:r + part], b), r
    # float64: S within D of itself (the fast functions' bounds, or expf's and a division's), two more products, one rounding
    e = torch.finfo(dtype).eps / 2
    sub = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}[dtype]
    for r in range(0, n, part):
        g, u = y[r:r + part, :c].double(), y[r:r + part, c:].double()
        D = torch.full_like(g, 2.0 ** -22) if dtype is torch.float32 else (5 + 1.2 * g.abs()) * 2.0 ** -23
        ref = g * torch.sigmoid(g) * u
        tol = (e + (D + 2 * U) * (1 + e)) * ref.abs() + 2.0 ** -126 * (g * u).abs() + sub
        assert ((got[2][r:r + part].double() - ref).abs() <= tol).all(), r

    # rows filled up to the middle of each call's last lap (one of them at a time) and into the first
    last = [lap(c, dtype, f) * (n * groups // lap(c, dtype, f)) for f in (True, False)]
    for filled in sorted([(x + n * groups) // 2 // groups for x in last] + [part // 2 + 3], reverse=True):
        count = torch.tensor([filled], dtype=torch.int32, device=DEV)
        y[filled:], d[filled:] = math.nan, math.nan
        some = both(y, d, dtype, count)
        for a, b in zip(some, got):
            assert torch.equal(a[:filled], b[:filled])
        q, s, h, d_y, h2 = some
        assert (q[filled:] == 0x7F).all() and (s[filled:] == 7).all()
        assert (h[filled:] == 3).all() and (d_y[filled:] == 3).all() and (h2[filled:] == 3).all()
