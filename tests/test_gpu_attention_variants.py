"""Every kernel that a call of fdy_tree_attention or fdy_paged_attention may take, by type, cache, head size, page size, query rows of a
cache head and the table's width, at rows in one part and in several."""
import pytest

from tests import test_gpu_paged_attention as paged
from tests import test_gpu_tree_attention as trees

pytestmark = pytest.mark.gpu
KINDS = [("bf16", "bf16"), ("f16", "f16"), ("bf16", "f8"), ("f16", "f8")]


@pytest.mark.parametrize("kind,cache", KINDS)
@pytest.mark.parametrize("D", [64, 128, 256, 48, 112, 240])
@pytest.mark.parametrize("pt", [8, 16])
@pytest.mark.parametrize("drafts", [4, 8, 16, 40])
def test_trees(drafts, pt, D, kind, cache):
    """16, 32, 64 and 160 query rows of a cache head."""
    trees.check([1500, drafts + 60], [drafts, drafts - 1], 4, 1, D, kind=kind, cache=cache, pt=pt)
    trees.check([drafts + 30, drafts], [drafts, drafts], 4, 1, D, kind=kind, cache=cache, pt=pt, order="head", shape="chain")


@pytest.mark.parametrize("kind,cache", KINDS)
@pytest.mark.parametrize("D", [64, 128, 256, 112])
@pytest.mark.parametrize("pt,row_pages", [(8, None), (16, None), (16, 512)])
@pytest.mark.parametrize("Hq", [4, 20, 33, 64])
def test_one_token(Hq, pt, row_pages, D, kind, cache):
    """Query heads of one cache head: a tile of 16, one of 32, several of 16, several of 32."""
    paged.check([2500, 17, 300], Hq, 1, D, kind=kind, cache=cache, pt=pt, row_pages=row_pages)
