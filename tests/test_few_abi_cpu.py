"""Pure-host behaviour of the few-token layer and the e4m3 operators: workspace
sizes, the binding's constants and the refusals that need no GPU."""
import os
import re

import pytest
import torch

from paper_2606_22541_gb300 import _native, api, build as build_mod, inputs
from paper_2606_22541_gb300.configs import CONFIGS, DSV3, DSV3_FP8

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "asap_moe.h")


@pytest.fixture(scope="module")
def L():
    build_mod.build()
    return _native.lib()


def test_token_limit_of_the_header():
    assert int(re.search(r"#define ASAP_MOE_FEW_MAX_TOKENS (\d+)", open(HEADER).read()).group(1)) == api.FEW_MAX_TOKENS


@pytest.mark.parametrize("cfg", list(CONFIGS.values()) + [
    inputs.small_variant(c, name="small", hidden=512, inter=256, shared_inter=256) for c in (DSV3, DSV3_FP8)],
    ids=lambda c: f"{c.name}-{c.hidden}")
def test_workspace_of_more_tokens_serves_fewer(L, cfg):
    """A program sizes its workspace once, for its largest call; a call of fewer tokens can be split more often."""
    sizes = [api.asap_moe_workspace_size(cfg, n, 4096) for n in range(0, 130)]
    assert sizes[0] == 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))


def test_refusals_without_a_gpu(L):
    one = torch.empty(1, 128)
    q, s = torch.empty(1, 128, dtype=torch.float8_e4m3fn), torch.empty(1, 1)
    x = one.bfloat16()
    with pytest.raises(ValueError):
        api.asap_moe_fp8_quantize(one, q, s)             # fp32 rows
    with pytest.raises(ValueError):
        api.asap_moe_fp8_quantize(x, q, torch.empty(1, 2))
    with pytest.raises(ValueError):
        api.asap_moe_fp8_quantize(x, q, s)               # not on a GPU
    with pytest.raises(ValueError):
        api.asap_moe_fp8_swiglu_quantize(x, x[:, :64], q, s)
    with pytest.raises(ValueError):
        api.asap_moe_fp8_matmul(q, s, q, torch.empty(2, 1), torch.empty(1, 1, dtype=torch.bfloat16))
    invalid = _native.ASAP_ERR_INVALID
    assert L.asap_moe_layer_few(None, None, None, 1, None, None, 0, None) == invalid
    assert L.asap_moe_fp8_quantize(None, 128, 1, 128, None, 128, None, 1, None) == invalid
    assert L.asap_moe_fp8_quantize(None, 128, 0, 128, None, 128, None, 1, None) == _native.ASAP_OK
    assert L.asap_moe_fp8_quantize(16, 64, 1, 128, 16, 128, 16, 1, None) == invalid     # rows overlap
    assert L.asap_moe_fp8_matmul(16, 100, 16, 1, 16, 112, 16, 1, 16, 4, 1, 4, 100, None, None) == invalid
    assert "16-byte" in str(api.asap_moe_last_error())
