"""Bounds of pages kept beside the pages: after drafted tokens came and some of them stayed, and after pages moved, they are what they would
be if they were made anew."""
import numpy as np
import pytest
import torch

import oracle.decode as od
from paper_2604_06664_amd import decode as fdd
from tests.support.paged import DEV, DTYPES, int32
from tests.test_gpu_draft_rounds import D, H, HQ, PAGES, PT, ROWS, Pool

pytestmark = pytest.mark.gpu
DRAFTS = 25


def bring_up(pool, bounds, fresh):
    fdd.fdy_page_bounds(fdd.make_bounds_desc(bounds=bounds, table=pool.table, lens=pool.lens, kv=pool.kv, fresh=int32(fresh), max_fresh=512),
                        pool.status)


def as_made_anew(pool, bounds, cache):
    torch.cuda.synchronize()
    assert int(pool.status) == 0
    lens, table = pool.lens.tolist(), pool.table.cpu().numpy()
    want = torch.zeros(PAGES, H, 2, D, dtype=torch.float64)
    od.page_bounds(want, pool.planes[0].view(DTYPES[cache]).cpu(), table, lens, lens)
    pages = [int(p) for r, n in enumerate(lens) for p in table[r, :-(-n // PT)]]
    assert torch.equal(bounds.cpu().double()[pages], want[pages])


@pytest.mark.parametrize("cache", ["bf16", "f8"])
@pytest.mark.parametrize("drafts_too", [False, True])
def test_after_drafted_tokens_and_moved_pages(drafts_too, cache):
    rng = np.random.default_rng(3)
    new = lambda n, heads: torch.from_numpy(rng.standard_normal((n, heads, D)).astype(np.float32)).to(torch.bfloat16).to(DEV)  # noqa: E731
    angles = torch.empty(512, 2, D // 2, device=DEV)
    fdd.fdy_rope_table(fdd.make_rope(D), 0, 512, angles)
    pool = Pool(cache)
    bounds = torch.zeros(PAGES, H, 2, D, dtype=DTYPES[cache], device=DEV)
    prompts = [50, 16, 31]
    pool.append(prompts, new(97, HQ), new(97, H), new(97, H), [0] * 97, angles)
    bring_up(pool, bounds, prompts)
    as_made_anew(pool, bounds, cache)
    for turn in range(6):
        drafts = [int(x) for x in rng.integers(1, DRAFTS + 1, ROWS)]
        n = sum(drafts)
        pool.append(drafts, new(n, HQ), new(n, H), new(n, H), [0] * n, angles)
        if drafts_too:
            bring_up(pool, bounds, drafts)
            as_made_anew(pool, bounds, cache)
        kept = [int(rng.integers(0, c // 2 + 1)) for c in drafts]
        kept[turn % ROWS] = 0
        keep = torch.full((ROWS, DRAFTS), -1, dtype=torch.int32, device=DEV)
        for r in range(ROWS):
            keep[r, :kept[r]] = int32(sorted(rng.permutation(drafts[r])[:kept[r]].tolist()))
        fdd.fdy_pages_keep(pool.desc, pool.token, int32(list(range(ROWS))), int32(drafts), keep, int32(kept), ROWS, DRAFTS, pool.ws,
                           pool.ws.numel(), pool.status)
        bring_up(pool, bounds, [k + 1 for k in kept])
        as_made_anew(pool, bounds, cache)
    fdd.fdy_pages_free(pool.desc, int32([1]), 1, pool.status)
    to, n_live = torch.empty(PAGES, dtype=torch.int32, device=DEV), int32([0])
    fdd.fdy_pages_compact(pool.desc, to, n_live, pool.ws, pool.ws.numel(), pool.status)
    live = torch.nonzero(to >= 0)[:, 0]
    assert bool((to[live] != live).any())
    moved = torch.zeros_like(bounds)
    moved[to[live].long()] = bounds[live]
    as_made_anew(pool, moved, cache)
