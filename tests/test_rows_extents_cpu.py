"""The ends of the extents that the operators on rows of tokens take: no GPU is
needed, what is refused enqueues nothing."""
import pytest

from paper_2606_22541_gb300 import _native, api, build as build_mod

P = 1 << 20   # an address that nothing reads
MOST = 1 << 30


@pytest.fixture(scope="module")
def L():
    build_mod.build()
    return _native.lib()


# (one token: n * k alone would let k up to 2^31 - 1 pass, and the loops over a token's places count in 32 bits)
@pytest.mark.parametrize("n", [0, 1])
@pytest.mark.parametrize("k", [MOST + 1, (1 << 31) - 9, (1 << 31) - 1])
def test_more_slots_than_an_extent_may_have(L, n, k):
    calls = {
        "asap_moe_sort": (P, n, k, 8, P, P, None, P, 1 << 40, None),
        "asap_moe_permute": (0, P, 64, n, 64, P, k, P, 64, 8, None, None),
        "asap_moe_unpermute": (0, P, 64, 8, 64, P, P, n, k, P, 64, None, None),
        "asap_moe_unpermute_backward": (0, P, 64, P, 64, P, P, n, k, 64, P, 64, 8, P, None, None),
        "asap_moe_fp8_dequantize": (0, P, 64, P, 1, n, 64, P, k, P, 64, 8, None, None),
    }
    for call, args in calls.items():
        assert getattr(L, call)(*args) == _native.ASAP_ERR_INVALID, call
    with pytest.raises(_native.AsapError):
        api.asap_moe_sort_workspace_size(n, k, 8)


def test_as_many_slots_as_an_extent_may_have(L):
    """The largest k is no error where nothing is to be done, and has a workspace."""
    assert L.asap_moe_permute(0, P, 64, 0, 64, P, MOST, P, 64, 8, None, None) == _native.ASAP_OK
    assert L.asap_moe_unpermute(0, P, 64, 8, 64, P, P, 0, MOST, P, 64, None, None) == _native.ASAP_OK
    assert api.asap_moe_sort_workspace_size(1, MOST, 8) == ((MOST >> 11) + 1) * 8 * 4
