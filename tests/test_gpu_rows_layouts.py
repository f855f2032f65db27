"""The row operators on tensors that are laid out differently from each other, with
more rows than a grid has CTAs, more places than a warp has lanes and rows shorter
than an access; both ways of marshalling.  Values that 32-bit sums give exactly
(small whole numbers), so outputs are compared bit by bit."""
import itertools
import math

import pytest
import torch

from paper_2606_22541_gb300 import _native, api

pytestmark = pytest.mark.gpu
DEV, F8 = "cuda", torch.float8_e4m3fn
TYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def whole(shape, seed, dtype, most=7):
    return torch.randint(-most, most + 1, shape, generator=gen(seed), device=DEV).to(dtype)


def strided(rows, cols, pad, offset, dtype, fill):
    ld = cols + pad
    flat = torch.full((rows * ld + offset + 40,), fill, device=DEV).to(dtype)
    return flat, flat[offset:offset + rows * ld].view(rows, ld)[:, :cols]


def places(n, k, E, seed, drop=0.2):
    g = gen(seed)
    idx = torch.randint(0, E, (n, k), generator=g, device=DEV).to(torch.int32)
    idx[torch.rand((n, k), generator=g, device=DEV) < drop] = -1
    off = torch.empty(E + 1, dtype=torch.int32, device=DEV)
    perm = torch.empty((n, k), dtype=torch.int32, device=DEV)
    api.asap_moe_sort(idx, E, off, perm, api.sort_workspace(n, k, E))
    return perm


def check_all(n, k, c, dtype, layouts, seed=1):
    """Every row operator; layouts: (padding, offset) of x, x_perm, out, d_out, y, d_y and the e4m3 rows."""
    lx, lp, lo, lg, ly, ld, lq = layouts
    perm = places(n, k, 16, seed)
    rows = n * k + 1
    t, j = torch.nonzero(perm >= 0, as_tuple=True)
    p = perm[t, j].long()
    bits = torch.int32 if dtype is torch.float32 else torch.int16

    def same(flat, view, want, fill):
        """view holds want, and what lies around it in flat is untouched."""
        assert torch.equal(view, want)
        view.fill_(fill)
        assert torch.equal(flat.view(bits), torch.full_like(flat, fill).view(bits))

    _, x = strided(n, c, *lx, dtype, math.nan)
    x.copy_(whole((n, c), 2, dtype))
    flat, xp = strided(rows, c, *lp, dtype, 3.0)
    api.asap_moe_permute(x, perm, xp)
    want = torch.full((rows, c), 3.0, device=DEV, dtype=dtype)
    want[p] = x[t]
    same(flat, xp, want, 3.0)

    _, y = strided(rows, c, *ly, dtype, math.nan)   # (NaNs beside the rows, and in the rows that nothing names)
    y[p] = whole((p.numel(), c), 3, dtype)
    w = whole((n, k), 4, torch.float32, 2)
    full = torch.zeros((n, k, c), device=DEV)
    full[t, j] = y[p].float()
    flat, out = strided(n, c, *lo, dtype, 3.0)
    api.asap_moe_unpermute(y, w, perm, out)
    same(flat, out, (full * w[:, :, None]).sum(1).to(dtype), 3.0)

    _, g = strided(n, c, *lg, dtype, math.nan)
    g.copy_(whole((n, c), 5, dtype, 1))
    flat, dy = strided(rows, c, *ld, dtype, 3.0)
    dw = torch.empty((n, k), device=DEV)
    api.asap_moe_unpermute_backward(g, y, w, perm, dy, dw)
    want = torch.full((rows, c), 3.0, device=DEV, dtype=dtype)
    want[p] = (w[t, j, None] * g[t].float()).to(dtype)
    assert torch.equal(dw, (full * g.float()[:, None, :]).sum(2))
    same(flat, dy, want, 3.0)
    alone = torch.empty_like(dw)
    api.asap_moe_unpermute_backward(g, y, w, perm, None, alone)
    assert torch.equal(dw, alone)

    qflat, q = strided(n, c, *lq, F8, 1.0)
    qflat.view(torch.uint8).fill_(0x7F)    # (NaN)
    q.copy_(whole((n, c), 6, torch.float32).to(F8))
    s = 2.0 ** torch.randint(-3, 4, (n, -(-c // 128)), generator=gen(7), device=DEV)
    flat, xr = strided(rows, c, *lp, dtype, 3.0)
    api.asap_moe_fp8_dequantize(q, s, xr, perm)
    v = (q.float() * s.repeat_interleave(128, 1)[:, :c]).to(dtype)
    want = torch.full((rows, c), 3.0, device=DEV, dtype=dtype)
    want[p] = v[t]
    same(flat, xr, want, 3.0)
    flat, xr = strided(n, c, *lp, dtype, 3.0)
    api.asap_moe_fp8_dequantize(q, s, xr)
    same(flat, xr, v, 3.0)


# paddings and offsets in elements: rows on 16 bytes, on 8, on 4 and elsewhere, alike in all rows or not
ODD = [(0, 0), (8, 0), (3, 0), (0, 1), (1, 2), (5, 3), (2, 4), (7, 5), (4, 8), (6, 7), (1, 15)]


@pytest.mark.parametrize("c", [1, 2, 3, 5, 8, 15, 16, 17, 33, 120, 127, 129, 258])
@pytest.mark.parametrize("turn", range(5))
@pytest.mark.parametrize("dtype", TYPES)
def test_mixed_layouts(c, turn, dtype):
    pick = itertools.cycle(ODD[turn * 2:] + ODD[:turn * 2])
    skip = lambda n: [next(pick) for _ in range(n)][-1]
    check_all(7, 3, c, dtype, [skip(turn + 1) for _ in range(7)], seed=c)


@pytest.mark.parametrize("k", [5, 8, 9, 16, 31, 40, 70])
@pytest.mark.parametrize("c", [24, 77, 1040])
@pytest.mark.parametrize("odd", [False, True])
def test_many_places(k, c, odd):
    check_all(9, k, c, torch.bfloat16, [(c % 8 and 8 - c % 8, 0)] * 7 if not odd else [(1, 1)] * 7)


@pytest.mark.parametrize("n,k,c,dtype", [(30000, 2, 64, torch.bfloat16), (30000, 1, 65, torch.float16),
                                         (9000, 3, 520, torch.bfloat16), (9000, 3, 521, torch.bfloat16),
                                         (12000, 4, 300, torch.float32), (12000, 5, 301, torch.float32),
                                         (5000, 8, 1090, torch.float16), (153, 8, 4097, torch.bfloat16),
                                         (152, 8, 8200, torch.bfloat16), (700, 2, 6000, torch.float32)])
def test_more_rows_than_a_grid_takes_at_once(n, k, c, dtype):
    pad = c % 8 and 8 - c % 8
    check_all(n, k, c, dtype, [(0, 0)] * 7)
    if pad:
        check_all(n, k, c, dtype, [(pad, 0)] * 7)


@pytest.mark.parametrize("way", ["compiled", "python"])
def test_both_ways_of_marshalling(way, monkeypatch):
    """The compiled one takes what a program usually passes, the other one everything; their launches are the same."""
    if way == "python":
        monkeypatch.setattr(api, "fast", lambda: False)
    else:
        assert _native.fast()
    check_all(50, 4, 264, torch.bfloat16, [(0, 0)] * 7)
    check_all(1, 4, 264, torch.float32, [(5, 3)] * 7)
    n, c = 30, 384
    y = torch.randn((n, 2 * c), generator=gen(1), device=DEV).bfloat16()
    q, s = torch.empty((n, 2 * c), dtype=F8, device=DEV), torch.empty((n, 6), device=DEV)
    h, dy = torch.empty((n, c), dtype=torch.bfloat16, device=DEV), torch.empty_like(y)
    parts = (q[:, :c], s[:, :3], q[:, c:], s[:, 3:])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    api.asap_moe_swiglu_save(y[:, :c], y[:, c:], h, *parts, stream=side)
    api.asap_moe_swiglu_backward(h, *parts, dy[:, :c], dy[:, c:], stream=side)
    side.synchronize()
    monkeypatch.setattr(api, "fast", lambda: False)
    q2, s2, h2, dy2 = (torch.empty_like(t) for t in (q, s, h, dy))
    parts = (q2[:, :c], s2[:, :3], q2[:, c:], s2[:, 3:])
    api.asap_moe_swiglu_save(y[:, :c], y[:, c:], h2, *parts)
    api.asap_moe_swiglu_backward(h2, *parts, dy2[:, :c], dy2[:, c:])
    for a, b in ((q.view(torch.uint8), q2.view(torch.uint8)), (s, s2), (h, h2), (dy, dy2)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("n,c", [(40000, 72), (3000, 5001)])
@pytest.mark.parametrize("dtype", TYPES)
def test_swiglu_of_more_groups_than_a_grid_takes_at_once(n, c, dtype):
    """Every row the same: every row's results are the first one's, which other tests compare with float64."""
    y = torch.randn((1, 2 * c), generator=gen(1), device=DEV).to(dtype).expand(n, 2 * c).contiguous()
    q, s = torch.zeros((n, 2 * c), dtype=F8, device=DEV), torch.zeros((n, 2 * -(-c // 128)), device=DEV)
    h, dy, h2 = torch.zeros((n, c), dtype=dtype, device=DEV), torch.zeros_like(y), torch.zeros((n, c), dtype=dtype, device=DEV)
    b = s.shape[1] // 2
    parts = (q[:, :c], s[:, :b], q[:, c:], s[:, b:])
    api.asap_moe_swiglu_save(y[:, :c], y[:, c:], h, *parts)
    api.asap_moe_swiglu_backward(h, *parts, dy[:, :c], dy[:, c:], h2)
    for t in (q.view(torch.uint8), s, h, dy, h2):
        assert torch.equal(t, t[:1].expand_as(t)) and t[0].float().abs().sum() > 0
