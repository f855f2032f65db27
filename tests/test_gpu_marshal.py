"""The binding's two ways of marshalling the short calls: the same launches,
the same refusals."""
import pytest
import torch

from paper_2606_22541_gb300 import _native, api

pytestmark = pytest.mark.gpu
DEV, F8 = "cuda", torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


@pytest.fixture(params=["compiled", "python"])
def way(request, monkeypatch):
    if request.param == "python":
        monkeypatch.setattr(api, "fast", lambda: False)
    else:
        assert _native.fast()
    return request.param


def tensors():
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    x = torch.randn((9, 1040), generator=g, device=DEV).bfloat16()
    w = torch.randn((260, 512), generator=g, device=DEV).to(F8)
    return dict(x=x, w=w, q=torch.empty((9, 512), dtype=F8, device=DEV), s=torch.empty((9, 4), device=DEV),
                ws=torch.rand((3, 4), generator=g, device=DEV), y=torch.empty((9, 260), dtype=torch.bfloat16, device=DEV))


def run(t, stream=None):
    api.asap_moe_fp8_swiglu_quantize(t["x"][:, 8:508], t["x"][:, 520:1020], t["q"][:, :500], t["s"], stream)
    sw = t["q"].view(torch.uint8).clone()
    api.asap_moe_fp8_quantize(t["x"][:, :512], t["q"], t["s"], stream)
    api.asap_moe_fp8_matmul(t["q"], t["s"], t["w"], t["ws"], t["y"], stream)
    return sw[:, :500], t["q"].view(torch.uint8).clone(), t["s"].clone(), t["y"].clone()


def test_both_ways_launch_the_same(way, monkeypatch):
    t = tensors()
    got = run(t)
    monkeypatch.setattr(api, "fast", lambda: False)
    for a, b in zip(got, run(t)):
        assert torch.equal(a, b)


def test_streams(way):
    t = tensors()
    want = run(t)
    side = torch.cuda.Stream()
    t["y"].zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):   # the current stream
        got = run(t)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    t["y"].zero_()
    torch.cuda.synchronize()
    api.asap_moe_fp8_matmul(t["q"], t["s"], t["w"], t["ws"], t["y"], stream=side)
    side.synchronize()
    assert torch.equal(t["y"], want[3])


def test_refusals(way):
    t = tensors()
    with pytest.raises(ValueError, match="e4m3"):
        api.asap_moe_fp8_quantize(t["x"][:, :512].float(), t["q"], t["s"])
    with pytest.raises(ValueError):
        api.asap_moe_fp8_quantize(t["x"][:, :512], t["q"], t["s"].t().contiguous().t())  # columns not contiguous
    with pytest.raises(ValueError):
        api.asap_moe_fp8_matmul(t["q"], t["s"], t["w"][:, :256], t["ws"], t["y"])
    with pytest.raises(ValueError):
        api.asap_moe_fp8_matmul(t["q"].cpu(), t["s"], t["w"], t["ws"], t["y"])
    with pytest.raises(_native.AsapError, match="16-byte"):
        api.asap_moe_fp8_matmul(t["q"][:, 8:], t["s"], t["w"][:, 8:], t["ws"], t["y"])
    api.asap_moe_fp8_matmul(t["q"][:0], t["s"][:0], t["w"], t["ws"], t["y"][:0])  # nothing to do
