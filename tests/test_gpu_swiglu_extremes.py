"""SwiGLU with quantise where the sigmoid is far out: every value in a group of
its own, so that nothing else decides the group's scale, and groups that mix
values whose quotient is divided with values whose quotient is corrected."""
import math

import pytest
import torch

from paper_2606_22541_gb300 import api
from test_gpu_fp8_ops import DEV, F8, encode

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def swiglu(g, u):
    q = torch.empty(g.shape, dtype=F8, device=DEV)
    s = torch.empty((g.shape[0], -(-g.shape[1] // 128)), device=DEV)
    api.asap_moe_fp8_swiglu_quantize(g, u, q, s)
    return q, s


# bf16 values on both sides of 80, where the division takes over, and up to what e^-g leaves finite
GATES = [0.0, 1e-30, -1e-30, 1.0, -1.0, 20.0, -20.0, 60.0, -60.0, 79.0, -79.0, 79.5, -79.5, 80.0, -80.0, 80.5, -80.5, 84.0,
         -84.0, 88.0, -88.0, 88.5, -88.5, 100.0, 1e4, 3e38]


@pytest.mark.parametrize("columns", [[0], [37], [127], list(range(128))], ids=["first", "inside", "last", "all"])
def test_one_value_per_group(columns):
    """The largest value of a group is 448 times its scale: q s gives v itself, which fp32 computes within a few 2^-23
    (exponential, sum, quotient, product, scale; 16 in all)."""
    g = torch.zeros((len(GATES), 128), dtype=torch.bfloat16, device=DEV)
    u = torch.zeros_like(g)
    for i, v in enumerate(GATES):
        g[i, columns] = v
        # (an up that brings the product to a few thousandths at least and overflows nothing)
        u[i, columns] = 1e-30 if v > 1e30 else 2.0 ** max(0, round(-1.4427 * v) - 10) if v < 0 else -3.0
    q, s = swiglu(g, u)
    g64 = g.double()
    want = g64 / (1 + (-g64).exp()) * u.double()
    got = q.double() * s.double()
    assert torch.equal(q.double().abs()[want != 0], torch.full_like(want, 448.0)[want != 0])
    err = (got - want).abs()[want != 0] / want.abs()[want != 0]
    assert float(err.max()) <= 16 * 2.0 ** -23
    assert (got[want == 0] == 0).all()


def test_beyond_the_exponential():
    """e^-g is infinite in fp32 from -89 on: the value is 0, of the sign that the definition gives it."""
    g = torch.tensor([[-89.0] * 128, [-100.0] * 128, [-1e5] * 128, [-3e38] * 128], device=DEV).bfloat16()
    q, s = swiglu(g, torch.full_like(g, 2.0))
    assert (q.float() == 0).all() and (s == 1).all()
    assert q.float().signbit().all()


def test_infinities_and_nans_stay_in_their_group():
    g = torch.ones((5, 384), device=DEV).bfloat16()
    u = torch.ones_like(g)
    clean, sc = swiglu(g, u)
    g[0, 130], g[1, 130], u[2, 130], u[3, 130] = math.inf, math.nan, math.inf, math.nan
    g[4, 130], u[4, 130] = -90.0, math.inf   # 0 times infinity
    q, s = swiglu(g, u)
    assert torch.equal(q[:, :128].float(), clean[:, :128].float()) and torch.equal(q[:, 256:].float(), clean[:, 256:].float())
    assert torch.equal(s[:, ::2], sc[:, ::2])
    assert (s[[0, 2], 1] == math.inf).all() and q[0, 128:256].float().isnan().all() and q[2, 128:256].float().isnan().all()
    for r in (1, 3, 4):  # a NaN leaves the group's scale and its other values alone
        row = q[r, 128:256].float()
        assert s[r, 1] == sc[r, 1] and row[2].isnan() and int(row.isnan().sum()) == 1


@pytest.mark.parametrize("offset", [0, 1, 4])
def test_groups_of_near_and_far_values(offset):
    """Gates on both sides of 80 in one group and in the sixteen columns of one thread, with ups that bring all values
    to one size.  As for any v: within half a step of e4m3 (2^-4 of the value, 2^-10 of the scale)."""
    n, c = 64, 300
    gen = torch.Generator(device=DEV)
    gen.manual_seed(5)
    flat = torch.empty(n * (2 * c + offset) + offset, dtype=torch.bfloat16, device=DEV)
    y = flat[offset:offset + n * (2 * c + offset)].view(n, 2 * c + offset)[:, :2 * c]
    g, u = y[:, :c], y[:, c:]
    g.copy_((torch.rand((n, c), generator=gen, device=DEV) - 0.5) * 176)   # -88 .. 88
    g[:, ::7] = 79.5
    g[:, 3::16] = -84.0
    v64 = g.double() / (1 + (-g.double()).exp())
    u.copy_((torch.randn((n, c), generator=gen, device=DEV).double() / v64).float().clamp(-3e38, 3e38))
    q, s = swiglu(g, u)
    v = v64 * u.double()
    _, rs = encode(v.float())
    assert float(((s - rs).abs() / rs).max()) <= 16 * 2.0 ** -23
    spread = s.double().repeat_interleave(128, 1)[:, :c]
    step = torch.maximum(v.abs() * 2.0 ** -4, spread * 2.0 ** -10)
    assert ((q.double() * spread - v).abs() <= step * (1 + 1e-4)).all()


@pytest.mark.parametrize("columns", [1, 127, 128, 300])
def test_zeros_keep_their_sign(columns):
    """-0 / s is -0: alone in its group, beside values, and where a gate of either sign makes the zero."""
    x = torch.zeros((4, columns), dtype=torch.bfloat16, device=DEV)
    x[1] = -0.0
    x[2, ::2] = -0.0
    x[3] = torch.linspace(-2, 2, columns, device=DEV).bfloat16()
    x[3, ::3] = -0.0
    q = torch.empty(x.shape, dtype=F8, device=DEV)
    s = torch.empty((4, -(-columns // 128)), device=DEV)
    api.asap_moe_fp8_quantize(x, q, s)
    rq, rs = encode(x.float())
    assert torch.equal(s, rs) and torch.equal(q.view(torch.uint8), rq.view(torch.uint8))
    for up in (1.0, -1.0):
        q, _ = swiglu(x, torch.full_like(x, up))
        v = x.float() / (1 + (-x.float()).exp()) * up
        assert torch.equal(q.float()[v == 0], torch.zeros_like(v)[v == 0])
        assert torch.equal(q.float().signbit()[v == 0], v.signbit()[v == 0])
