"""The e4m3 product where its tiles are cut along k and where one kind of tile
takes over from another: every number of slices, uneven ones among them, rows
of several tiles, and outputs of every alignment."""
import pytest
import torch

from paper_2606_22541_gb300 import api
from test_gpu_fp8_ops import F8, DEV, gen, magnitude64, operands, product64, store

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def check(m, n, k, seed, ldc=None, offset=0):
    """bf16 rounding 2^-9 of the value (2^-8 leaves room for the sum's own error); sums of a block 2^-21 of its
    magnitudes, and fp32 additions of the blocks and slices 2^-23 each."""
    a, sa, b, sb = operands(m, n, k, seed)
    flat, out = store(m, n, ldc or n, offset, torch.bfloat16, 7.0)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    api.asap_moe_fp8_matmul(a, sa, b, sb, out, status=status)
    ref = product64(a, sa, b, sb)
    bound = ref.abs() * 2.0 ** -8 + magnitude64(a, sa, b, sb) * (2.0 ** -20 + sa.shape[1] * 2.0 ** -22)
    assert ((out.double() - ref).abs() <= bound).all() and int(status) == 0
    again = torch.empty_like(out)
    api.asap_moe_fp8_matmul(a, sa, b, sb, again)
    assert torch.equal(out.contiguous(), again)
    out.fill_(7.0)
    assert (flat == 7.0).all()


# tiles of 128 rows of b: few of them are cut into as many slices as there are pairs of blocks, many into what one wave
# of CTAs leaves
@pytest.mark.parametrize("m", [1, 17, 33, 64])
@pytest.mark.parametrize("n,k", [(128, 128 * b) for b in range(2, 20, 2)] + [(300, 1200), (5000, 900), (7000, 1600),
                                 (13000, 1300), (20001, 700)])
def test_slices_of_few_rows(m, n, k):
    check(m, n, k, m + n + k)


@pytest.mark.parametrize("m", [65, 100, 128, 129, 200, 256, 257, 511, 1000])
@pytest.mark.parametrize("n,k", [(100, 1900), (512, 2048), (700, 1920), (1000, 3200), (2048, 4000), (260, 6500)])
def test_rows_of_several_tiles(m, n, k):
    check(m, n, k, m + n + k)


@pytest.mark.parametrize("m", [70, 130, 500])
@pytest.mark.parametrize("n,pad,offset", [(520, 0, 0), (520, 8, 8), (520, 4, 4), (520, 2, 2), (520, 1, 1), (515, 13, 0),
                                          (520, 24, 3), (1, 0, 0), (7, 1, 0), (1024, 0, 1)])
@pytest.mark.parametrize("k", [400, 5000])
def test_output_alignment(m, n, pad, offset, k):
    check(m, n, k, m + n, n + pad, offset)


def test_slices_keep_infinities_and_nans_in_their_rows():
    m, n, k = 100, 300, 4000
    a, sa, b, sb = operands(m, n, k, 3)
    out = torch.empty((m, n), dtype=torch.bfloat16, device=DEV)
    api.asap_moe_fp8_matmul(a, sa, b, sb, out)
    clean = out.clone()
    a.view(torch.uint8)[70, 3999] = 0x7F
    b.view(torch.uint8)[299, 0] = 0xFF
    sa[3, 9] = float("nan")
    api.asap_moe_fp8_matmul(a, sa, b, sb, out)
    rows = [i for i in range(m) if i not in (3, 70)]
    assert out[3].isnan().all() and out[70].isnan().all() and out[:, 299].isnan().all()
    assert torch.equal(out[rows][:, :299], clean[rows][:, :299])


def test_whole_numbers_are_exact_in_every_slice():
    for m, n, k in ((64, 128, 2048), (45, 7000, 1600), (128, 512, 2100), (300, 1000, 6400), (500, 4100, 3300)):
        g = gen(m + n)
        ld = -(-k // 16) * 16
        a = torch.randint(-1, 2, (m, ld), generator=g, device=DEV).float()
        b = torch.randint(-1, 2, (n, ld), generator=g, device=DEV).float()
        nb = -(-k // 128)
        sa = 2.0 ** torch.randint(0, 2, (m, nb), generator=g, device=DEV).float()
        sb = 2.0 ** torch.randint(0, 2, (-(-n // 128), nb), generator=g, device=DEV).float()
        out = torch.empty((m, n), dtype=torch.bfloat16, device=DEV)
        api.asap_moe_fp8_matmul(a.to(F8)[:, :k], sa, b.to(F8)[:, :k], sb, out)
        assert torch.equal(out, product64(a[:, :k], sa, b[:, :k], sb).bfloat16())
