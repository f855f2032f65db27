"""The decode step (dense e4m3 layers and MoE layers in turn) against the same
step in float64 of plain operations."""
import pytest
import torch

from paper_2606_22541_gb300 import api, decode_step, inputs
from paper_2606_22541_gb300.configs import DSV3_FP8

from test_gpu_few import gate64, layer64, make, quantised

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def dense64(layer, x):
    def w(v, s):
        return v.double() * s.double().repeat_interleave(128, 0).repeat_interleave(128, 1)

    # the product's output is bf16, as the layer keeps it
    y = (quantised(x) @ w(layer.gate_up, layer.s_gate_up).t()).bfloat16().double()
    g, u = y[:, :layer.inter], y[:, layer.inter:]
    return quantised(g * g.sigmoid() * u) @ w(layer.down, layer.s_down).t()


@pytest.mark.parametrize("n", [1, 5, 33])
def test_step_against_float64(n):
    """Layer by layer: each layer's output is taken for the input that the step gave it, so that an e4m3 value that
    falls the other way does not decide the rest.  Tolerances of the layers: bf16 outputs 2^-9, and in the dense layer
    another 2^-9 on its inner values, of which e4m3 makes up to sqrt(2^-9 / 16) / 16 * 4 = 2.8e-3 (values that fall
    the other way); 6e-3 and 4e-3 in all."""
    cfg = inputs.small_variant(DSV3_FP8, name="step", hidden=512, inter=256, shared_inter=256, zipf_s=None)
    weights = [make(cfg, seed=s) for s in range(2)]
    handle = api.asap_moe_create_layers(cfg, weights, 64)
    dense = [decode_step._dense_layer(cfg.hidden, 640, 64, s, DEV) for s in range(2)]
    x0 = inputs.make_tokens(cfg, n, 0, DEV)
    x = x0.clone()
    step = decode_step.DecodeStep(dense, handle, n)
    step(x)
    # the same, one layer at a time
    z, y = x0.clone(), torch.empty_like(x0)
    for layer in dense:
        layer(z, y)
        ref = dense64(layer, z)
        assert float((y.double() - ref).norm() / ref.norm()) <= 6e-3
        z += y
    for l, w in enumerate(weights):
        api.asap_moe_layer_few(handle, z, y, step.ws, layer_id=step.ids[l:l + 1])
        ref, _ = layer64(cfg, w, z)
        decided = gate64(cfg, z.double() @ w["router_w"].double().t(), w["router_bias"])[2]
        assert float((y.double() - ref)[decided].norm() / ref[decided].norm()) <= 4e-3
        z += y
    assert torch.equal(x, z)
    # and from a graph
    graph = torch.cuda.CUDAGraph()
    g = x0.clone()
    with torch.cuda.graph(graph):
        g.copy_(x0)
        step(g)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(g, x)
    assert api.asap_moe_status(handle) == (0, 0)
    handle.close()
