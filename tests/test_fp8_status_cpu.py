"""The product's status word is checked before either way of marshalling sees
it: a kernel whose wait has run out adds error bits there."""
import types

import pytest
import torch

from paper_2606_22541_gb300 import api


@pytest.fixture(params=["compiled", "python"])
def seen(request, monkeypatch):
    """The status that the chosen way of marshalling is given."""
    got = []
    way = lambda *a: got.append(a[6]) or 0
    monkeypatch.setattr(api, "fast", lambda: types.SimpleNamespace(matmul=way) if request.param == "compiled" else False)
    monkeypatch.setattr(api, "_matmul", way)
    return got


def word(dtype=torch.int32, n=1, is_cuda=True):
    t = types.SimpleNamespace(dtype=dtype, is_cuda=is_cuda, shape=(n,), device="fake", numel=lambda: n,
                              stride=lambda: (1,), data_ptr=lambda: 0x700)
    return t


@pytest.mark.parametrize("status", [None, word(), word(n=5), word(torch.uint32)], ids=["none", "one", "more", "unsigned"])
def test_passed_on(seen, status):
    api.asap_moe_fp8_matmul(1, 2, 3, 4, 5, status=status)
    assert len(seen) == 1 and seen[0] is status


@pytest.mark.parametrize("status", [word(is_cuda=False), word(n=0), word(torch.float32), word(torch.int64),
                                    word(torch.uint8, n=4), torch.zeros(1, dtype=torch.int32)],
                         ids=["host", "empty", "fp32", "int64", "bytes", "host tensor"])
def test_refused(seen, status):
    with pytest.raises(ValueError, match="status"):
        api.asap_moe_fp8_matmul(1, 2, 3, 4, 5, status=status)
    assert not seen
