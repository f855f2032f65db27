"""h at the end of fp32's range in the few-token layer's BF16 form, which keeps
it as two bf16: a value that bf16 would round to infinity is still finite, and
one that is infinite gives infinities of the sign that its weights have."""
from dataclasses import replace

import pytest
import torch

from paper_2606_22541_gb300 import api
from paper_2606_22541_gb300.configs import TINY

from test_gpu_few import DEV, TOL, few, make, tokens

pytestmark = pytest.mark.gpu
CHANNEL = 5
CFG = replace(TINY, name="few_overflow", n_experts=1, top_k=1, hidden=768)


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def weights():
    """One expert whose channel 5 is x0 * x1 (silu(x0) = x0 for large x0), met by weights of +-1/2."""
    w = make(CFG)
    w["router_w"][:, :2] = 0
    for name in ("w_gate", "w_up"):
        w[name][:, :, :2] = 0
        w[name][:, CHANNEL] = 0
    w["w_gate"][0, CHANNEL, 0] = 1
    w["w_up"][0, CHANNEL, 1] = 1
    sign = torch.ones(CFG.hidden, device=DEV)
    sign[1::3] = -1
    w["w_down"][0, :, CHANNEL] = 0.5 * sign
    return w, sign


def factors(lo, hi):
    """Two bf16 values whose product lies between lo and hi times 2^127."""
    m = torch.arange(128, 256, dtype=torch.float64) / 128
    at = ((m[:, None] * m[None] > lo) & (m[:, None] * m[None] < hi)).nonzero()[0]
    return float(m[at[0]] * 2.0 ** 64), float(m[at[1]] * 2.0 ** 63)


@pytest.mark.parametrize("n", [1, 5, 17])
def test_h_at_the_end_of_the_range(n):
    w, sign = weights()
    h = api.asap_moe_create(CFG, w, 64)
    x = tokens(CFG, n)
    x[:, :2] = 0
    clean = few(h, x)
    last = n - 1
    # fp32 holds the product, bf16 rounds it to infinity: the output is half of it
    x[last, 0], x[last, 1] = factors(2 - 2.0 ** -8, 2)
    got = few(h, x)
    want = 0.5 * sign.double() * float(x[last, 0].double() * x[last, 1].double())
    assert float(((got[last].double() - want).norm() / want.norm())) <= TOL["bf16"]
    assert torch.equal(got[:last], clean[:last])
    # the largest value that bf16 holds
    x[last, 0], x[last, 1] = factors(2 - 2.0 ** -6, 2 - 2.0 ** -8)
    got = few(h, x)
    want = 0.5 * sign.double() * float(x[last, 0].double() * x[last, 1].double())
    assert float(((got[last].double() - want).norm() / want.norm())) <= TOL["bf16"]
    # fp32 does not hold it, of either sign; and no number
    x[last, 0], x[last, 1] = factors(2, 4)
    for s in (1, -1):
        x[last, 1] = s * x[last, 1].abs()
        got = few(h, x)
        assert torch.equal(got[last].float(), s * sign * float("inf"))
        assert torch.equal(got[:last], clean[:last])
    x[last, 1] = float("nan")
    got = few(h, x)
    assert got[last].isnan().all() and torch.equal(got[:last], clean[:last])
    assert api.asap_moe_status(h) == (0, 0)
    h.close()
