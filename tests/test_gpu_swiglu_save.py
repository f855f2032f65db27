"""SwiGLU with activations kept in e4m3, its gradients, and a training step of an
expert layer through all operators: against float64.

Tolerances (u = 2^-24; e = finfo(type).eps / 2).  16-bit results take the fast
exponential and reciprocal: within 2 + 1.16 |g| and 2 units of 2^-23 by CUDA's
documentation, so the sigmoid S is within D = (5 + 1.2 |g|) 2^-23 of its value
(relative); fp32 results take expf (1 unit) and a division (half): D = 2^-22.
Where e^-g passes 2^126 S may be 0."""
import math

import pytest
import torch

from paper_2606_22541_gb300 import api, inputs
from paper_2606_22541_gb300.configs import TINY

pytestmark = pytest.mark.gpu
DEV, F8 = "cuda", torch.float8_e4m3fn
U = 2.0 ** -24
TYPES = [torch.bfloat16, torch.float16, torch.float32]
SUBNORMAL = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}
SHAPES = [(1, 1), (1, 128), (3, 127), (2, 129), (5, 256), (7, 1000), (64, 2048), (33, 2052), (1, 14336), (300, 8),
          (1000, 640), (2, 65536)]
LAYOUTS = [(0, 0), (8, 8), (4, 4), (5, 3)]   # padding of a row, offset of the first


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def randn(shape, seed, std=1.0):
    return torch.randn(shape, generator=gen(seed), device=DEV) * std


def strided(rows, cols, pad, offset, dtype, fill):
    ld = cols + pad
    flat = torch.full((rows * ld + offset + 32,), fill, device=DEV).to(dtype)
    return flat, flat[offset:offset + rows * ld].view(rows, ld)[:, :cols]


def blocks(c):
    return (c + 127) // 128


def encode(v):
    """The definition in fp32: scale amax * fl(1 / 448) per 128 columns, quotient by division."""
    n, c = v.shape
    p = torch.nn.functional.pad(v, (0, -c % 128)).view(n, -1, 128)
    s = p.nan_to_num(0.0, math.inf, -math.inf).abs().amax(2) * torch.tensor(1.0 / 448.0, device=DEV)
    s = torch.where(s > 0, s, torch.ones_like(s))
    return (p / s[:, :, None]).clamp(-448, 448).to(F8).view(n, -1)[:, :c], s


def decode(q, s):
    return q.float().double() * s.double().repeat_interleave(128, 1)[:, :q.shape[1]]


def sigma_error(g, dtype):
    return torch.full_like(g, 2.0 ** -22) if dtype is torch.float32 else (5 + 1.2 * g.abs()) * 2.0 ** -23


def check_h(h, g, u, dtype):
    """h against g, u in float64: three factors, rounded once."""
    ref = g * torch.sigmoid(g) * u
    e = torch.finfo(dtype).eps / 2
    tol = (e + (sigma_error(g, dtype) + 2 * U) * (1 + e)) * ref.abs() + 2.0 ** -126 * (g * u).abs() + SUBNORMAL[dtype]
    assert ((h.double() - ref).abs() <= tol).all()


def kept(n, c, pad=0, offset=0):
    """gate_q, gate_s, up_q, up_s as halves of one tensor each, and those tensors."""
    b = blocks(c)
    qflat, q = strided(n, 2 * c, pad, offset, F8, 1.0)
    sflat, s = strided(n, 2 * b, pad, offset, torch.float32, 7.0)
    return (q[:, :c], s[:, :b], q[:, c:], s[:, b:]), (qflat, q, sflat, s)


@pytest.mark.parametrize("n,c", SHAPES)
@pytest.mark.parametrize("pad,offset", LAYOUTS)
@pytest.mark.parametrize("dtype", TYPES)
def test_forward(n, c, pad, offset, dtype):
    _, y = strided(n, 2 * c, pad, offset, dtype, math.nan)
    y.copy_(randn((n, 2 * c), n + c) * torch.exp(randn((1, 2 * c), c)))
    gate, up = y[:, :c], y[:, c:]
    parts, (qflat, q, sflat, s) = kept(n, c, pad, offset)
    before = qflat.view(torch.uint8).clone()
    hflat, h = strided(n, c, pad, offset, dtype, 3.0)
    keep = hflat.clone()
    api.asap_moe_swiglu_save(gate, up, h, *parts)
    check_h(h, gate.double(), up.double(), dtype)
    for half, (vq, vs) in ((gate, parts[:2]), (up, parts[2:])):
        rq, rs = encode(half.float())
        assert torch.equal(vs, rs)
        assert torch.equal(vq.contiguous().view(torch.uint8), rq.contiguous().view(torch.uint8))
        if dtype is torch.bfloat16:
            oq, os_ = torch.empty((n, c), dtype=F8, device=DEV), torch.empty((n, blocks(c)), device=DEV)
            api.asap_moe_fp8_quantize(half, oq, os_)
            assert torch.equal(oq.view(torch.uint8), vq.contiguous().view(torch.uint8)) and torch.equal(os_, vs)
    # nothing beside the rows is written
    ld = 2 * c + pad
    q.view(torch.uint8).copy_(before[offset:offset + n * ld].view(n, ld)[:, :2 * c])
    assert torch.equal(qflat.view(torch.uint8), before)
    s.fill_(7.0)
    assert (sflat == 7.0).all()
    keep[offset:offset + n * (c + pad)].view(n, c + pad)[:, :c] = h
    assert torch.equal(hflat, keep)


@pytest.mark.parametrize("n,c", SHAPES)
@pytest.mark.parametrize("pad,offset", LAYOUTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("wants_h", [True, False])
def test_backward(n, c, pad, offset, dtype, wants_h):
    parts, (_, q, _, s) = kept(n, c, pad, offset)
    v = randn((n, 2 * c), n + c, 2.0) * torch.exp(randn((1, 2 * c), c))
    for half in (0, 1):
        eq, es = encode(v[:, half * c:(half + 1) * c])
        parts[2 * half].copy_(eq)
        parts[2 * half + 1].copy_(es)
    _, d_h = strided(n, c, pad, offset, dtype, math.nan)
    d_h.copy_(randn((n, c), 9, 0.1))
    dflat, d_y = strided(n, 2 * c, pad, offset, dtype, 3.0)
    hflat, h = strided(n, c, pad, offset, dtype, 3.0)
    keep, hkeep = dflat.clone(), hflat.clone()
    api.asap_moe_swiglu_backward(d_h, *parts, d_y[:, :c], d_y[:, c:], h if wants_h else None)
    g, u, d = decode(*parts[:2]), decode(*parts[2:]), d_h.double()
    p = torch.sigmoid(g)
    D, e = sigma_error(g, dtype) + 2 * U, torch.finfo(dtype).eps / 2   # (g and u are rounded to fp32 themselves)
    slope = p + g * p * (1 - p)
    # S + t (1 - S), t = g S: S off by D S, 1 - S by D S + u, t by (D + u) t; two roundings
    off = p * D + (g * p).abs() * ((D + 2 * U) * (1 - p) + D * p + U) + 2 * U * (p + (g * p * (1 - p)).abs())
    # g itself is off by u g, which moves S by S (1 - S) u |g| and the slope by at most (2 + |g|) S u |g|
    off = off + (2 + g.abs()) * p * U * g.abs()
    far = (1 + g.abs()) * 2.0 ** -125
    ref = d * u * slope
    tol = (d * u).abs() * (off + far) * (1 + e) + (e + 4 * U) * ref.abs() + SUBNORMAL[dtype]
    assert ((d_y[:, :c].double() - ref).abs() <= tol).all()
    ref = d * g * p
    tol = (e + (D + 4 * U + U * g.abs()) * (1 + e)) * ref.abs() + d.abs() * far + SUBNORMAL[dtype]
    assert ((d_y[:, c:].double() - ref).abs() <= tol).all()
    if wants_h:
        ref = g * p * u
        tol = (e + (D + 5 * U + U * g.abs()) * (1 + e)) * ref.abs() + u.abs() * far + SUBNORMAL[dtype]
        assert ((h.double() - ref).abs() <= tol).all()
        hkeep[offset:offset + n * (c + pad)].view(n, c + pad)[:, :c] = h
    assert torch.equal(hflat, hkeep)
    keep[offset:offset + n * (2 * c + pad)].view(n, 2 * c + pad)[:, :2 * c] = d_y
    assert torch.equal(dflat, keep)


def test_backward_against_differences():
    """Central differences of silu(g) u in float64 at the kept values; fp32 results: within 2^-20 of the sum of the
    terms, the differences within step^2 / 6 of the third derivative (below 1 in size, times |g| + 3)."""
    n, c, step = 9, 300, 1e-4
    parts, _ = kept(n, c)
    y, h = randn((n, 2 * c), 1, 2.0), torch.empty((n, c), device=DEV)
    api.asap_moe_swiglu_save(y[:, :c], y[:, c:], h, *parts)
    d, d_y = randn((n, c), 2), torch.empty((n, 2 * c), device=DEV)
    api.asap_moe_swiglu_backward(d, *parts, d_y[:, :c], d_y[:, c:])
    g, u, d = decode(*parts[:2]), decode(*parts[2:]), d.double()
    f = lambda g, u: g * torch.sigmoid(g) * u
    dg = d * (f(g + step, u) - f(g - step, u)) / (2 * step)
    du = d * (f(g, u + step) - f(g, u - step)) / (2 * step)
    size = d.abs() * (u.abs() * (1 + g.abs()) + g.abs())
    tol = 2.0 ** -20 * size + step ** 2 * d.abs() * u.abs() * (g.abs() + 3) + 1e-10 * size
    assert ((d_y[:, :c].double() - dg).abs() <= tol).all() and ((d_y[:, c:].double() - du).abs() <= tol).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_extremes(dtype):
    big = torch.finfo(dtype).max
    vals = torch.tensor([0.0, -0.0, 1e-30, -20.0, 20.0, 87.0, -87.0, 88.5, -88.5, 100.0, -100.0, 1e4, -1e4, big, -big],
                        device=DEV).to(dtype)
    n = vals.numel()
    g = vals[:, None].expand(n, 128).contiguous()
    u = torch.full((n, 128), 0.5, device=DEV).to(dtype)
    h = torch.empty_like(g)
    parts, _ = kept(n, 128)
    parts = tuple(t.contiguous() for t in parts)
    api.asap_moe_swiglu_save(g, u, h, *parts)
    check_h(h, g.double(), u.double(), dtype)
    d = torch.ones_like(g)
    dg, du = torch.empty_like(g), torch.empty_like(g)
    api.asap_moe_swiglu_backward(d, *parts, dg, du, h)
    assert dg.isfinite().all() and du.float().isfinite().all()
    assert (dg[vals.float() >= 20] == u[0, 0]).all() and (dg[vals.float() <= -1e4] == 0).all()
    check_h(h, decode(*parts[:2]), decode(*parts[2:]), dtype)


def test_nan_and_infinities_stay_in_their_group():
    g, u = randn((4, 384), 1).bfloat16(), randn((4, 384), 2).bfloat16()
    g[1, 5], g[2, 130] = math.nan, -math.inf
    h = torch.empty_like(g)
    parts = tuple(t.contiguous() for t in kept(4, 384)[0])
    api.asap_moe_swiglu_save(g, u, h, *parts)
    bad = torch.zeros((4, 384), dtype=torch.bool, device=DEV)
    bad[1, 5] = bad[2, 130] = True
    assert torch.equal(h.isnan(), bad)
    dg, du = torch.empty_like(g), torch.empty_like(g)
    api.asap_moe_swiglu_backward(torch.ones_like(g), *parts, dg, du)
    bad[2, 128:256] = True       # an infinity gives its group an infinite scale
    assert torch.equal(dg.isnan(), bad) and torch.equal(du.isnan(), bad)


@pytest.mark.parametrize("filled", [0, 1, 7, 40, 41, -3])
def test_rows_behind_the_last_are_left_alone(filled):
    n, c = 40, 520
    y = randn((n, 2 * c), 1).bfloat16()
    r = max(0, min(filled, n))
    y[r:] = math.nan
    count = torch.tensor([filled], dtype=torch.int32, device=DEV)
    parts, (qflat, q, _, s) = kept(n, c)
    h = torch.full((n, c), 3.0, device=DEV).bfloat16()
    api.asap_moe_swiglu_save(y[:, :c], y[:, c:], h, *parts, n_rows=count)
    assert (h[r:] == 3).all() and (s[r:] == 7).all() and (q[r:].float() == 1).all()
    check_h(h[:r], y[:r, :c].double(), y[:r, c:].double(), torch.bfloat16)
    d_y, h2 = torch.full((n, 2 * c), 3.0, device=DEV).bfloat16(), torch.full((n, c), 3.0, device=DEV).bfloat16()
    d = torch.where(torch.arange(n, device=DEV)[:, None] < r, 1.0, math.nan).expand(n, c).contiguous().bfloat16()
    api.asap_moe_swiglu_backward(d, *parts, d_y[:, :c], d_y[:, c:], h2, n_rows=count)
    assert (d_y[r:] == 3).all() and (h2[r:] == 3).all() and d_y.isfinite().all()
    check_h(h2[:r], decode(*parts[:2])[:r], decode(*parts[2:])[:r], torch.bfloat16)


def test_offsets_past_32_bits():
    ld, c, n = (1 << 30) + 64, 200, 3
    flat = torch.zeros(2 * ld + 2 * c, dtype=torch.bfloat16, device=DEV)
    y = flat.as_strided((n, 2 * c), (ld, 1))
    y.copy_(randn((n, 2 * c), 1))
    q = torch.zeros(2 * ld + 2 * c, dtype=torch.uint8, device=DEV).as_strided((n, 2 * c), (ld, 1))
    s = torch.zeros((n, 4), device=DEV)
    h = torch.zeros(2 * ld + c, dtype=torch.bfloat16, device=DEV).as_strided((n, c), (ld, 1))
    parts = (q[:, :c], s[:, :2], q[:, c:], s[:, 2:])
    api.asap_moe_swiglu_save(y[:, :c], y[:, c:], h, *parts)
    check_h(h, y[:, :c].double(), y[:, c:].double(), torch.bfloat16)
    assert torch.equal(q[2:, :c], encode(y[2:, :c].float())[0].view(torch.uint8))
    hc, near = h.contiguous(), torch.empty((n, 2 * c), dtype=torch.bfloat16, device=DEV)
    api.asap_moe_swiglu_backward(hc, *(t.contiguous() for t in parts), near[:, :c], near[:, c:])
    api.asap_moe_swiglu_backward(hc, *parts, y[:, :c], y[:, c:], h)
    assert torch.equal(y, near)


def test_graph_capture():
    n, c = 500, 1024
    y, y2 = randn((n, 2 * c), 1).bfloat16(), randn((n, 2 * c), 2).bfloat16()
    count = torch.tensor([n], dtype=torch.int32, device=DEV)
    d, h, d_y = randn((n, c), 3).bfloat16(), torch.empty((n, c), dtype=torch.bfloat16, device=DEV), torch.empty_like(y)
    parts, _ = kept(n, c)

    def both():
        api.asap_moe_swiglu_save(y[:, :c], y[:, c:], h, *parts, n_rows=count)
        api.asap_moe_swiglu_backward(d, *parts, d_y[:, :c], d_y[:, c:], h, n_rows=count)

    first = y.clone()
    both()
    torch.cuda.synchronize()
    want = (h.clone(), d_y.clone())
    y.copy_(y2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    graph.replay()
    torch.cuda.synchronize()
    other = (h.clone(), d_y.clone())
    y.copy_(first)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(h, want[0]) and torch.equal(d_y, want[1]) and not torch.equal(other[1], want[1])
    count.fill_(100)        # read when the kernels run
    h.fill_(3.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(h[:100], want[0][:100]) and (h[100:] == 3).all()


def test_refusals():
    n, c = 4, 256
    y, h = randn((n, 2 * c), 1), randn((n, c), 2)
    parts, _ = kept(n, c)
    gq, gs, uq, us = parts
    for call in (lambda: api.asap_moe_swiglu_save(y[:, :c], h, h.clone(), *parts),                     # two row strides
                 lambda: api.asap_moe_swiglu_save(y[:, :c], y[:, c:], h.half(), *parts),
                 lambda: api.asap_moe_swiglu_save(y[:, :c], y[:, c:], h, gq, gs[:, :1], uq, us[:, :1]),
                 lambda: api.asap_moe_swiglu_save(y[:, :c], y[:, c:], h, gq, gs, uq.contiguous(), us),
                 lambda: api.asap_moe_swiglu_save(y[:, :c], y[:, c:], h, *parts, n_rows=torch.tensor([1], device=DEV)),
                 lambda: api.asap_moe_swiglu_save(y[:, :c].int(), y[:, c:].int(), h.int(), *parts),
                 lambda: api.asap_moe_swiglu_backward(h, *parts, y[:, :c], h.clone()),
                 lambda: api.asap_moe_swiglu_backward(h, *parts, y[:, :c], y[:, c:], h[:, :5])):
        with pytest.raises(ValueError):
            call()


# ------------------------------------------------------------------ a training step

def test_training_step_of_an_expert_layer():
    """Forward and backward of routed experts as a program would run them: the router of a handle, the sort, rows to their
    experts, the products, SwiGLU kept in e4m3, rows back, and every gradient down to x, the routing weights and the
    experts' matrices; the tokens themselves are kept in e4m3 for the first product's weight gradient.  The reference is
    the same computation in float64 at the values that were kept; its tolerance is that of six bf16 roundings on the way, each
    within 2^-8 of a value and so below 2^-9 in the norm (a third of the square, over values spread within a power of two)."""
    cfg = TINY
    E, H, I, k, n = cfg.n_experts, cfg.hidden, cfg.inter, cfg.top_k, 100
    w = inputs.make_weights(cfg, DEV)
    handle = api.asap_moe_create(cfg, w, n)
    x = inputs.make_tokens(cfg, n, 0, DEV)
    i32, b16 = dict(dtype=torch.int32, device=DEV), dict(dtype=torch.bfloat16, device=DEV)
    idx, p = torch.empty((n, k), **i32), torch.empty((n, k), device=DEV)
    api.asap_moe_route(handle, x, idx, p, torch.empty(E, **i32), torch.empty(E + 1, **i32), api.workspace(handle, n))
    idx[90:] = -1            # padding tokens
    idx[5, 1] = -1           # an entry over its expert's capacity
    off, perm = torch.empty(E + 1, **i32), torch.empty((n, k), **i32)
    api.asap_moe_sort(idx, E, off, perm, api.sort_workspace(n, k, E))
    xq, xs = torch.empty((n, H), dtype=F8, device=DEV), torch.empty((n, blocks(H)), device=DEV)
    api.asap_moe_fp8_quantize(x, xq, xs)
    rows = n * k
    junk = lambda c: torch.full((rows, c), math.nan, **b16)
    xp, gu, h, y, out = junk(H), junk(2 * I), junk(I), junk(H), torch.empty((n, H), **b16)
    api.asap_moe_permute(x, perm, xp)
    o = off.tolist()
    seg = [slice(a, b) for a, b in zip(o, o[1:])]
    wgu = torch.cat([w["w_gate"], w["w_up"]], 1)     # [E, 2 I, H]
    for e, s in enumerate(seg):
        gu[s] = xp[s] @ wgu[e].t()
    parts, _ = kept(rows, I)
    taken = off[E:]
    api.asap_moe_swiglu_save(gu[:, :I], gu[:, I:], h, *parts, n_rows=taken)
    for e, s in enumerate(seg):
        y[s] = h[s] @ w["w_down"][e].t()
    api.asap_moe_unpermute(y, p, perm, out)

    d_out = randn((n, H), 5).bfloat16()
    d_y, d_h, d_gu, h2, d_xp, xr = junk(H), junk(I), junk(2 * I), junk(I), junk(H), junk(H)
    d_p, d_x = torch.empty((n, k), device=DEV), torch.empty((n, H), **b16)
    api.asap_moe_unpermute_backward(d_out, y, p, perm, d_y, d_p)
    for e, s in enumerate(seg):
        d_h[s] = d_y[s] @ w["w_down"][e]
    api.asap_moe_swiglu_backward(d_h, *parts, d_gu[:, :I], d_gu[:, I:], h2, n_rows=taken)
    api.asap_moe_fp8_dequantize(xq, xs, xr, perm)
    d_wgu, d_wd = torch.zeros((E, 2 * I, H), device=DEV), torch.zeros((E, H, I), device=DEV)
    for e, s in enumerate(seg):
        d_xp[s] = d_gu[s] @ wgu[e]
        d_wgu[e] = (d_gu[s].t() @ xr[s]).float()
        d_wd[e] = (d_y[s].t() @ h2[s]).float()
    api.asap_moe_unpermute(d_xp, None, perm, d_x)

    # float64, token by token and slot by slot
    dbl = lambda t: t.double()
    live = idx >= 0
    t, j = torch.nonzero(live, as_tuple=True)
    e, r = idx[t, j].long(), perm[t, j].long()
    X, W1, W2 = dbl(x)[t], dbl(wgu)[e], dbl(w["w_down"])[e]
    GU = torch.bmm(W1, X[:, :, None])[:, :, 0]
    silu = lambda g: g * torch.sigmoid(g)
    Y = torch.bmm(W2, (silu(GU[:, :I]) * GU[:, I:])[:, :, None])[:, :, 0]
    OUT = torch.zeros((n, H), dtype=torch.float64, device=DEV).index_add_(0, t, Y * dbl(p)[t, j, None])
    G, V = decode(*parts[:2])[r], decode(*parts[2:])[r]
    S = torch.sigmoid(G)
    D = dbl(d_out)[t]
    DY = D * dbl(p)[t, j, None]
    DH = torch.bmm(W2.transpose(1, 2), DY[:, :, None])[:, :, 0]
    DGU = torch.cat([DH * V * (S + G * S * (1 - S)), DH * G * S], 1)
    DX = torch.zeros((n, H), dtype=torch.float64, device=DEV).index_add_(
        0, t, torch.bmm(W1.transpose(1, 2), DGU[:, :, None])[:, :, 0])
    XR = decode(xq, xs)[t]
    DW1, DW2 = torch.zeros((E, 2 * I, H)).double().to(DEV), torch.zeros((E, H, I)).double().to(DEV)
    DW1.index_add_(0, e, DGU[:, :, None] * XR[:, None, :])
    DW2.index_add_(0, e, DY[:, :, None] * (G * S * V)[:, None, :I])
    DP = torch.zeros((n, k), dtype=torch.float64, device=DEV)
    DP[t, j] = (D * Y).sum(1)
    for name, got, ref in (("out", out, OUT), ("d_p", d_p, DP), ("d_x", d_x, DX), ("d_gate_up", d_wgu, DW1),
                           ("d_down", d_wd, DW2)):
        err = ((got.double() - ref).norm() / ref.norm()).item()
        assert err < 6 * 2.0 ** -9, (name, err)
    assert (out[90:] == 0).all() and (d_x[90:] == 0).all() and (d_p[90:] == 0).all()
    handle.close()
