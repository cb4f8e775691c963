"""fdy_page_select over wide tables: choices equal to the oracle's, whatever the table's width has each thread hold of a row's keys, and
nothing written outside the lists."""
import math

import numpy as np
import pytest
import torch

import oracle.decode as od
from paper_2604_06664_amd import decode as fdd
from tests.support.paged import DEV, int32

pytestmark = pytest.mark.gpu
H, D, GUARD = 2, 8, 4096
WIDTHS = [2047, 2049, 8191, 8193, 16384, 16385, 20000]  # entries of a table: keys in registers up to 16,384, read again behind
MIXED, POSITIVE, NEGATIVE, EQUAL, KINDS = "mixed", "positive", "negative", "equal", "three kinds"


def bounds_of(scores):
    """A page's bounds such that its score for a query of (1, 0, ..) is the given one."""
    b = torch.zeros(len(scores), H, 2, D, dtype=torch.float32)
    b[:, :, :, 0] = torch.from_numpy(np.asarray(scores, np.float32))[:, None, None]
    return b.to(torch.bfloat16)


def choose(scores, width, budget, sinks=0, recent=1, pt=1):
    """The rows' scores, one page each of `pt` tokens, over a table of `width`; lists lie between guards."""
    rng = np.random.default_rng(7)
    lens = [len(x) * pt for x in scores]
    n_pages = sum(len(x) for x in scores)
    table, order, at = np.full((len(scores), width), -1, np.int32), rng.permutation(n_pages), 0
    flat = np.empty(n_pages, np.float32)
    for r, x in enumerate(scores):
        table[r, :len(x)] = order[at:at + len(x)]
        flat[order[at:at + len(x)]] = x
        at += len(x)
    bounds = bounds_of(flat)
    q = torch.zeros(len(scores), H, D, dtype=torch.bfloat16)
    q[:, :, 0] = 1.0
    n = len(scores) * H * budget
    held = torch.full((n + 2 * GUARD,), -9, dtype=torch.int32, device=DEV)
    pages, seen = held[GUARD:GUARD + n].view(len(scores), H, budget), torch.full((len(scores),), -9, dtype=torch.int32, device=DEV)
    d_q, d_bounds, d_table, d_lens = q.to(DEV), bounds.to(DEV), torch.from_numpy(table).to(DEV), int32(lens)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    kv = fdd.make_kv(None, None, type=fdd.FDY_BF16, n_pages=n_pages, page_tokens=pt, n_heads=H, head_dim=D, page_stride=0, token_stride=0,
                     head_stride=0)
    desc = fdd.make_select_desc(q=d_q, bounds=d_bounds, table=d_table, lens=d_lens, kv=kv, pages=pages, seen=seen, sinks=sinks, recent=recent)
    size = fdd.fdy_page_select_workspace_bytes(desc)
    fdd.fdy_page_select(desc, torch.randint(0, 256, (size,), dtype=torch.uint8, device=DEV), size, status)
    torch.cuda.synchronize()
    want, want_seen = od.page_select(q, bounds, table, lens, pt, budget, sinks, recent)
    assert int(status) == 0 and seen.cpu().tolist() == want_seen.tolist()
    assert bool((held[:GUARD] == -9).all()) and bool((held[GUARD + n:] == -9).all())
    assert np.array_equal(pages.cpu().numpy(), want), np.argwhere(pages.cpu().numpy() != want)[:5]


def scores_of(kind, n, seed=1):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(n).astype(np.float32) + 0.0
    if kind == POSITIVE:
        return np.abs(x) + 1
    if kind == NEGATIVE:
        return -np.abs(x) - 1
    if kind == EQUAL:
        return np.full(n, 0.5, np.float32)
    if kind == KINDS:
        return rng.integers(-1, 2, n).astype(np.float32)
    return x


@pytest.mark.parametrize("kind", [MIXED, POSITIVE, NEGATIVE, EQUAL, KINDS])
@pytest.mark.parametrize("width", WIDTHS)
def test_long_and_short_rows(width, kind):
    long = min(width, 16400) if kind in (MIXED, EQUAL) else width // 3
    choose([scores_of(kind, long), scores_of(kind, 40, 2), scores_of(kind, 1), scores_of(kind, 0)], width, 13)


@pytest.mark.parametrize("width", [8193, 16385])
@pytest.mark.parametrize("sinks,recent,budget", [(0, 1, 1), (0, 1, 2), (5, 7, 12), (5, 7, 13), (0, 600, 1200), (700, 1, 1300), (0, 1, 1999)])
def test_shares_of_the_list(sinks, recent, budget, width):
    choose([scores_of(MIXED, 2000), scores_of(KINDS, 1500)], width, budget, sinks, recent, pt=4)


@pytest.mark.parametrize("odd", [1, 12, 13, 14, 40])
@pytest.mark.parametrize("special", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("kind", [POSITIVE, NEGATIVE])
@pytest.mark.parametrize("width", [2049, 8193, 16385])
def test_pages_of_the_largest_and_smallest_keys(width, kind, special, odd):
    """13 places beside the last page's, and fewer, as many and more pages whose score is no number or infinite: the key of a score that
    is no number is the last of all 64-bit integers."""
    x = scores_of(kind, 900, odd)
    x[np.random.default_rng(odd).permutation(899)[:odd]] = special
    choose([x, x[:100].copy()], width, 14)
    choose([x, x[:100].copy()], width, odd + 1 + (special == -math.inf), 1, 1)


@pytest.mark.parametrize("width,budget", [(40, 40), (40, 41), (40, 500), (41, 40), (2049, 2048), (2049, 2049), (16385, 16384), (16385, 16400)])
def test_lists_as_long_as_tables(width, budget):
    choose([scores_of(MIXED, width), scores_of(MIXED, 40, 2), scores_of(MIXED, 0), scores_of(EQUAL, width - 1)], width, budget)
