"""Every kernel that a call of fdy_tree_attention or fdy_paged_attention may take, by type, cache, head size, page size, query rows of a
cache head and the table's width, at rows in one part and in several."""
import pytest
import torch

from paper_2604_06664_amd import decode as fdd
from tests import test_gpu_paged_attention as paged
from tests import test_gpu_tree_attention as trees
from tests.support.paged import DEV, near

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


@pytest.mark.parametrize("kind,cache", [("bf16", "bf16"), ("f16", "f8")])
@pytest.mark.parametrize("pt,drafts", [(16, 20), (16, 40), (8, 20), (8, 40)])
def test_trees_of_many_rows_behind_32_bits(pt, drafts, kind, cache):
    """40 and 80 query rows of a cache head; pages a GiB apart, so that the row's last lies 2 to 7 GiB into the pool."""
    small = trees.Drafts([drafts + 20], [drafts], 2, 1, 64, kind=kind, cache=cache, spare=0, pt=pt)
    c, of_page = small.cache, pt * 64
    n_pages, es = c.n_pages, 1 if cache == "f8" else 2
    apart = (1 << 30) // es
    pools = [torch.empty((n_pages - 1) * apart + of_page, dtype=torch.uint8 if es == 1 else torch.int16, device=DEV) for _ in "kv"]
    for src, dst in zip(c.d_pools, pools):
        for j, x in enumerate(src.view(-1, of_page)):
            dst[j * apart:j * apart + of_page] = x
    kv = fdd.make_kv(*pools, type=fdd.TYPES[cache], n_pages=n_pages, page_tokens=pt, n_heads=1, head_dim=64, page_stride=apart,
                     token_stride=64, head_stride=64, k_scale=c.d_scales[0], v_scale=c.d_scales[1])
    got = small.run(kv=kv)
    assert got[2] == 0
    near(got, small.want(), kind)
