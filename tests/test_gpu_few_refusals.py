"""The binding of the few-token layer on real tensors: what would be read or
written out of range is refused, and what fits still runs."""
import pytest
import torch

from paper_2606_22541_gb300 import api
from paper_2606_22541_gb300.configs import TINY

from test_gpu_few import few, make, tokens

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def test_refusals_leave_the_output_alone():
    h = api.asap_moe_create(TINY, make(TINY), 64)
    x = tokens(TINY, 9)
    want = few(h, x)
    out, ws = torch.full_like(x, 7.0), api.workspace(h, 9)
    wide = torch.zeros((9, 2 * TINY.hidden), dtype=torch.bfloat16, device=DEV)
    layer = torch.zeros(1, dtype=torch.int32, device=DEV)
    for bad in (dict(x=x.float()), dict(x=x.cpu()), dict(x=wide[:, :TINY.hidden]), dict(x=wide), dict(out=out[:8]),
                dict(out=wide[:, TINY.hidden:]), dict(out=out.float()), dict(ws=ws.cpu()), dict(ws=ws[::2]),
                dict(layer_id=layer.cpu()), dict(layer_id=layer[:0]), dict(layer_id=layer.float())):
        with pytest.raises(ValueError):
            api.asap_moe_layer_few(**(dict(h=h, x=x, out=out, ws=ws) | bad))
    torch.cuda.synchronize()
    assert (out == 7.0).all() and (wide == 0).all()
    # more rows than tokens: those behind stay as they are
    rows = torch.full((20, TINY.hidden), 7.0, dtype=torch.bfloat16, device=DEV)
    api.asap_moe_layer_few(h, x, rows, ws, layer_id=layer)
    assert torch.equal(rows[:9], want) and (rows[9:] == 7.0).all()
    assert api.asap_moe_status(h) == (0, 0)
    h.close()
