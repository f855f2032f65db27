"""The gate's gradient d_h U slope where its factors are far apart: whichever two of
them pass the ends of fp32 when multiplied, the product of all three is right.

Tolerance (u = 2^-24, e = finfo(type).eps / 2, against float64 at the kept values,
which are exact here): the sigmoid S is within D (relative) as in the SwiGLU tests, t =
G S within D + u of itself, 1 - S within S D + u, and the slope S + t (1 - S) is rounded
once more; the two products round once each, the result to its type.  The sizes keep S
above 2^-120 and the gradient a normal number."""
import math

import pytest
import torch

from paper_2606_22541_gb300 import api

pytestmark = pytest.mark.gpu
DEV, F8 = "cuda", torch.float8_e4m3fn
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def gradients(d, g, u, dtype, pad, offset):
    """d_gate at kept values of sign * scale: g, u, d [rows, groups], each over the 128 columns of its group (the last group is
    short by pad columns)."""
    n, c = g.shape[0], g.shape[1] * 128 - pad
    ld = 2 * c + pad
    wide = lambda v: v.repeat_interleave(128, 1)[:, :c]
    q = torch.cat([wide(g.sign()), wide(u.sign())], 1).to(F8)
    flat = torch.empty(n * ld + offset, dtype=dtype, device=DEV)
    d_y = flat[offset:].view(n, ld)[:, :2 * c]
    d_h = torch.empty(n * c + offset, dtype=dtype, device=DEV)[offset:].view(n, c)
    d_h.copy_(wide(d))
    s = torch.cat([g.abs(), u.abs()], 1)
    b = g.shape[1]
    api.asap_moe_swiglu_backward(d_h, q[:, :c], s[:, :b], q[:, c:], s[:, b:], d_y[:, :c], d_y[:, c:])
    return d_y[:, :c], d_h.double(), wide(g).double(), wide(u).double()


# log2 of d_h and of U, and G: d slope below 2^-149; below 2^-126; d U above 2^128, U or d_h the larger one; d U below 2^-126
# beside a slope of one (a gradient that is subnormal is none of these); and ordinary ones
FAR = [(-120, 100, -30.0), (-100, 100, -30.0), (-60, 70, -75.0), (-126, 110, -5.0), (70, 70, -60.0), (100, 60, -55.0),
       (20, 120, -50.0), (110, 40, -45.0), (-3, 2, 1.5), (0, 0, -1.0), (-10, 20, 40.0), (30, 90, -80.0)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pad,offset", [(0, 0), (4, 4), (2, 2), (1, 1)])
def test_factors_far_apart(dtype, pad, offset):
    rows = torch.tensor(FAR, dtype=torch.float64, device=DEV)
    # groups of one row differ, and so do the rows, so that both orders meet in one warp
    pick = (torch.arange(len(FAR), device=DEV)[:, None] + torch.arange(7, device=DEV)[None, :]) % len(FAR)
    v = rows[pick]
    d, u, g = (2.0 ** v[:, :, 0]).float(), (1.375 * 2.0 ** v[:, :, 1]).float(), v[:, :, 2].float()
    got, d, g, u = gradients(d, g, u, dtype, pad, offset)
    s = torch.sigmoid(g)
    # (1 - s cancels in float64 as well; s of the negated value does not)
    slope = s + g * s * torch.sigmoid(-g)
    D = torch.full_like(g, 2.0 ** -22) if dtype is torch.float32 else (5 + 1.2 * g.abs()) * 2.0 ** -23
    e = torch.finfo(dtype).eps / 2
    off = s * D + (g * s).abs() * ((D + 2 * U) * (1 - s) + D * s + U) + U * slope.abs()
    ref = d * u * slope
    assert (ref.abs() > 2.0 ** -126).all() and (ref.abs() < 2.0 ** 127).all()
    tol = ((d * u).abs() * off * (1 + 4 * U) + 2 * U * ref.abs()) * (1 + e) + e * ref.abs()
    assert ((got.double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_closed_gates_meet_no_infinity(dtype):
    """S is 0 far below: the gradient is 0 whatever d U is, and an infinite or NaN d_h still shows."""
    big = 2.0 ** 120
    g = torch.tensor([[-1e4, -300.0, -1e30, -1e4, -1e4]], device=DEV).expand(3, 5).contiguous()
    u = torch.full((3, 5), big, device=DEV)
    d = torch.tensor([[big], [1.0], [-big]], device=DEV).expand(3, 5).contiguous()
    d[:, 3], d[:, 4] = math.inf, math.nan
    got, _, _, _ = gradients(d, g, u, dtype, 0, 0)
    assert (got[:, :3 * 128] == 0).all() and got[:, 3 * 128:].isnan().all()
    ones = torch.full_like(g, 30.0)      # an open gate: the slope is one
    got, _, _, _ = gradients(d, ones, u, dtype, 0, 0)
    assert (got[0, :384] == math.inf).all() and (got[2, :384] == -math.inf).all()
    assert (got[:, 384:512] == math.inf).all() and got[:, 512:].isnan().all()
