"""The e4m3 product's outputs whose rows start on 16 bytes and end inside a
32-column box: tiles of which some columns leave by bulk stores and some
directly."""
import pytest

from test_gpu_fp8_slices import check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


# n % 128 in 33 .. 63 (one box, then a cut one), 65 .. 95 (two) and 97 .. 127 (three), in either half of a 256-column
# tile; k too short for tiles to be cut; from 3000 rows on a CTA takes several tiles
@pytest.mark.parametrize("n", [36, 60, 68, 90, 170, 213, 291, 345, 357, 383, 556, 603])
@pytest.mark.parametrize("m,k", [(70, 130), (500, 400), (3000, 256)])
def test_cut_and_whole_boxes(m, n, k):
    for _ in range(3):
        check(m, n, k, m + n + k, ldc=-(-n // 8) * 8 + 8)


@pytest.mark.parametrize("m,n,k", [(3000, 4140, 512), (3000, 4139, 128), (8045, 2148, 300), (2000, 20010, 128),
                                   (5000, 4189, 200)])
def test_many_tiles(m, n, k):
    for _ in range(3):
        check(m, n, k, m + n + k, ldc=-(-n // 8) * 8)
