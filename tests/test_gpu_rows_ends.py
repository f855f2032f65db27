"""The ends of the ranges of the operators around a training step's expert products: the widest rows, the first call of a
process inside a graph capture, and the places next to those of asap_moe_dispatch."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2606_22541_gb300 import api, inputs
from paper_2606_22541_gb300.configs import MIXTRAL

pytestmark = pytest.mark.gpu
DEV, F8 = "cuda", torch.float8_e4m3fn
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


@pytest.mark.parametrize("c", [1 << 30, (1 << 30) - 5])
def test_widest_rows(c):
    """2^30 columns, the most that is allowed, and an odd number of them (rows of two that start on odd addresses)."""
    small = torch.randint(-7, 8, (1, 1 << 20), generator=gen(1), device=DEV).to(torch.bfloat16)
    x = small.repeat(1, 1024)[:, :c].contiguous()
    perm = torch.tensor([[1, 0]], dtype=torch.int32, device=DEV)
    y = torch.zeros((2, c), dtype=torch.bfloat16, device=DEV)
    api.asap_moe_permute(x, perm, y)
    assert torch.equal(y[0], x[0]) and torch.equal(y[1], x[0])
    out = torch.zeros_like(x)
    w = torch.tensor([[2.0, -1.0]], device=DEV)
    api.asap_moe_unpermute(y, w, perm, out)
    assert torch.equal(out, x)
    d_y, d_w = torch.zeros_like(y), torch.zeros((1, 2), device=DEV)
    api.asap_moe_unpermute_backward(torch.ones_like(x), y, w, perm, d_y, d_w)
    assert (d_y[1] == 2).all() and (d_y[0] == -1).all()
    n, total = 0, 0
    for a in range(0, c, 1 << 26):
        total += int(x[0, a:a + (1 << 26)].double().sum())
        n += int(x[0, a:a + (1 << 26)].double().abs().sum())
    # at most c / 1024 + 32 additions of whole numbers one after the other
    assert (d_w.double() - total).abs().max() <= (c / 1024 + 32) * 2.0 ** -24 * n and d_w[0, 0] == d_w[0, 1]
    del d_y
    q = x.to(F8)
    s = torch.full((1, -(-c // 128)), 0.5, device=DEV)
    y.zero_()
    api.asap_moe_fp8_dequantize(q, s, y, perm)
    assert torch.equal(y[0], x[0] / 2) and torch.equal(y[1], x[0] / 2)
    del y
    h, uq, us = torch.zeros_like(x), torch.zeros_like(q), torch.zeros_like(s)
    gq, gs = torch.zeros_like(q), torch.zeros_like(s)
    api.asap_moe_swiglu_save(x, out, h, gq, gs, uq, us)
    tail = torch.empty_like(x[:, -(c % 128 + 1280):])   # the last groups, alone
    t = (x[:, -tail.shape[1]:].contiguous(), out[:, -tail.shape[1]:].contiguous())
    tq, ts = torch.empty(tail.shape, dtype=F8, device=DEV), torch.empty((1, -(-tail.shape[1] // 128)), device=DEV)
    api.asap_moe_swiglu_save(*t, tail, tq, ts, tq.clone(), ts.clone())
    assert torch.equal(tail, h[:, -tail.shape[1]:]) and torch.equal(gs[:, -ts.shape[1]:], ts)
    assert torch.equal(gq[:, -tq.shape[1]:].view(torch.uint8), tq.view(torch.uint8))
    d_up = torch.zeros_like(x)
    api.asap_moe_swiglu_backward(x, gq, gs, uq, us, out, d_up)
    near = [torch.empty_like(tail) for _ in range(2)]
    api.asap_moe_swiglu_backward(t[0], tq, ts, tq, ts, *near)
    assert torch.equal(near[0], out[:, -tail.shape[1]:]) and torch.equal(near[1], d_up[:, -tail.shape[1]:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_closed_gates_under_the_largest_values(dtype):
    """A gate far below zero closes whatever stands beside it: results and gradients of 0, not of infinity times 0."""
    n, c = 3, 300
    big = torch.finfo(dtype).max / 4
    g = torch.full((n, c), -1e5, device=DEV).to(dtype)
    u = torch.full((n, c), big, device=DEV).to(dtype)
    d = torch.full((n, c), 100.0, device=DEV).to(dtype)
    q, s = [torch.empty((n, c), dtype=F8, device=DEV) for _ in range(2)], [torch.empty((n, 3), device=DEV) for _ in range(2)]
    h, dg, du, h2 = (torch.full((n, c), 5.0, device=DEV).to(dtype) for _ in range(4))
    api.asap_moe_swiglu_save(g, u, h, q[0], s[0], q[1], s[1])
    api.asap_moe_swiglu_backward(d, q[0], s[0], q[1], s[1], dg, du, h2)
    for t in (h, dg, du, h2):
        assert (t == 0).all()


FIRST = """
import torch
from paper_2606_22541_gb300 import api
n, k, E, c = 700, 8, 1000, 520
g = torch.Generator(device="cuda")
g.manual_seed(1)
idx = torch.randint(0, E, (n, k), generator=g, device="cuda").int()
many = torch.randint(0, E, (9000, k), generator=g, device="cuda").int()
x = torch.randn((n, c), generator=g, device="cuda").bfloat16()
w = torch.rand((n, k), generator=g, device="cuda")
def buffers():
    z = lambda *s, **kw: torch.zeros(s, device="cuda", **kw)
    i, b, f = dict(dtype=torch.int32), dict(dtype=torch.bfloat16), dict(dtype=torch.float8_e4m3fn)
    return [z(E + 1, **i), z(n, k, **i), z(n * k, c, **b), z(n, c, **b), z(n * k, c, **b), z(n, k), z(n * k, c, **f),
            z(n * k, 5), z(n * k, c, **b), z(n * k, c, **b), z(n * k, c, **b), z(n, c, **f), z(n, 5), z(E + 1, **i),
            z(9000, k, **i)]
def chain(o):
    off, perm, xp, out, dy, dw, q, s, h, dg, du, xq, xs, off2, perm2 = o
    api.asap_moe_sort(idx, E, off, perm, None)
    api.asap_moe_sort(many, E, off2, perm2, ws)
    api.asap_moe_permute(x, perm, xp)
    api.asap_moe_unpermute(xp, w, perm, out)
    api.asap_moe_unpermute_backward(x, xp, w, perm, dy, dw)
    api.asap_moe_swiglu_save(xp, dy, h, q, s, q2, s2)
    api.asap_moe_swiglu_backward(dy, q, s, q2, s2, dg, du)
    api.asap_moe_fp8_quantize(x, xq, xs)
    api.asap_moe_fp8_dequantize(xq, xs, xp, perm)
ws = api.sort_workspace(9000, k, E)
a, b = buffers(), buffers()
q2, s2 = torch.zeros_like(a[6]), torch.zeros_like(a[7])
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):      # nothing of the library has run before
    chain(a)
graph.replay()
torch.cuda.synchronize()
chain(b)
torch.cuda.synchronize()
for u, v in zip(a, b):
    bits = torch.uint8 if u.element_size() == 1 else torch.int16 if u.element_size() == 2 else torch.int32
    assert torch.equal(u.view(bits), v.view(bits)) and v.view(bits).any()
print("same")
"""


def test_first_calls_of_a_process_captured():
    r = subprocess.run([sys.executable, "-c", FIRST], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stdout + r.stderr


@pytest.mark.parametrize("n", [1, 97, 3000, 16384])
def test_places_of_dispatch(n):
    """The places of routed tokens are those that a handle's dispatch gives them."""
    cfg = inputs.small_variant(MIXTRAL, name="e8", hidden=256, inter=128, microbatches=[n])
    h = api.asap_moe_create(cfg, inputs.make_weights(cfg, DEV), n)
    x = inputs.make_tokens(cfg, n, 0, DEV)
    k, E = cfg.top_k, cfg.n_experts
    i32 = dict(dtype=torch.int32, device=DEV)
    idx, w = torch.empty((n, k), **i32), torch.empty((n, k), device=DEV)
    counts, off, ws = torch.empty(E, **i32), torch.empty(E + 1, **i32), api.workspace(h, n)
    api.asap_moe_route(h, x, idx, w, counts, off, ws)
    xp, src, dst = torch.empty((n * k, 256), dtype=torch.bfloat16, device=DEV), torch.empty(n * k, **i32), torch.empty((n, k), **i32)
    api.asap_moe_dispatch(h, x, idx, xp, src, dst, ws)
    off2, perm, src2 = torch.empty_like(off), torch.empty_like(dst), torch.empty_like(src)
    api.asap_moe_sort(idx, E, off2, perm, api.sort_workspace(n, k, E), src2)
    xp2 = torch.empty_like(xp)
    api.asap_moe_permute(x, perm, xp2)
    for a, b in ((off, off2), (dst, perm), (src, src2), (xp, xp2)):
        assert torch.equal(a, b)
    out, out2 = torch.empty_like(x), torch.empty_like(x)
    api.asap_moe_combine(h, xp, None, w, dst, out)
    api.asap_moe_unpermute(xp, w, perm, out2)
    assert torch.equal(out, out2)
    h.close()
