"""fdy_tree_attention over the longest rows there may be: some tokens less than 2^31, in pages that the row holds again and again."""
import math

import pytest
import torch

from paper_2604_06664_amd import decode as fdd
from tests.support.paged import DEV, int32

pytestmark = pytest.mark.gpu
D, DRAFTS = 64, 8


@pytest.mark.parametrize("Hq", [2, 8, 16])  # 16, 64 and 128 query rows
@pytest.mark.parametrize("pt", [8, 16])
def test_the_last_drafted_token_is_seen_by_itself_alone(pt, Hq):
    """All keys but the last are 0 and all values 1: sums of values and of weights are the same, the result is 1 and the logarithm that of
    the number of tokens.  The last token outweighs all others by far and has the value 100: only its own query may give that."""
    pages = (1 << 31) // pt - 1
    n = pages * pt
    table = torch.zeros(1, pages, dtype=torch.int32, device=DEV)
    table[0, -1] = 1
    k, v = torch.zeros(2, pt, 1, D, dtype=torch.bfloat16, device=DEV), torch.ones(2, pt, 1, D, dtype=torch.bfloat16, device=DEV)
    k[1, -1, 0, 0], v[1, -1] = 40.0, 100.0
    kv = fdd.make_kv(k, v, type=fdd.FDY_BF16, n_pages=2, page_tokens=pt, n_heads=1, head_dim=D, page_stride=pt * D, token_stride=D,
                     head_stride=D)
    q = torch.zeros(DRAFTS, Hq, D, dtype=torch.bfloat16, device=DEV)
    q[:, :, 0] = 1
    out, lse = torch.empty_like(q), torch.empty(DRAFTS, Hq, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    desc = fdd.make_draft_desc(q=q, out=out, lse=lse, table=table, lens=int32([n]), kv=kv, scale=1.0, max_draft=DRAFTS)
    ws = torch.empty(fdd.fdy_tree_attention_workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    fdd.fdy_tree_attention(desc, ws, ws.numel(), status)
    torch.cuda.synchronize()
    assert int(status) == 0
    assert bool(((out[:-1].float() - 1).abs() <= 2.0 ** -8).all()), out[:, 0, 0].tolist()
    assert bool(((out[-1].float() - 100).abs() <= 100 * 2.0 ** -8).all())
    for j in range(DRAFTS - 1):
        assert bool(((lse[j] - math.log(n - DRAFTS + 1 + j)).abs() <= 3e-4).all()), lse[:, 0].tolist()
    assert bool(((lse[-1] - 40).abs() <= 3e-4).all())
