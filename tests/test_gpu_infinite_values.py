"""Infinite values under attention over pages: an element of a result is infinite, with the value's sign, exactly where the definition in 64
bits has it so, and no number where it has none, as long as the value's weight is not less of the largest than the header says."""
import math

import pytest
import torch

from tests.support.paged import ROUND
from tests.test_gpu_paged_attention import Problem
from tests.test_gpu_tree_attention import Drafts, bits_of

pytestmark = pytest.mark.gpu
KINDS = ["bf16", "f16"]
LEAST = dict(bf16=-96.0, f16=-37.0)  # powers of two


def alike(got, want, kind, spread=4.0):
    out, o = got[0].double(), want[0]
    assert got[2] == 0
    for special in (torch.isnan, torch.isposinf, torch.isneginf):
        assert torch.equal(special(out), special(o)), special.__name__
    fine = torch.isfinite(o)
    assert bool(((out - o).abs()[fine] <= spread * (2.0 ** -11 + 2.0 ** -15) + ROUND[kind] * o.abs()[fine]).all())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("pt", [8, 16])
@pytest.mark.parametrize("D", [64, 128, 48])
@pytest.mark.parametrize("drafts", [[6, 9, 20], [30, 40, 20]])
def test_of_drafted_tokens(drafts, D, pt, kind):
    """In values of drafted tokens: those that see them, and nobody else."""
    p = Drafts([40, 170, 33], drafts, 4, 2, D, kind=kind, pt=pt)
    c = p.cache
    for r, j, d, bad in ((0, 3, 5, math.inf), (1, 2, 0, math.inf), (1, 4, D - 1, -math.inf), (1, 1, 7, math.inf), (1, 6, 7, -math.inf), (2, 0, 1, -math.inf)):
        t = c.lens[r] - p.drafts[r] + j
        c.views[1][c.table[r, t // pt], t % pt, :, d] = bad
    first = p.drafts[0]
    p.sees[first + 8] = {1, 6, 8}  # one of each sign in one element: no number
    p.d_sees = bits_of(p.sees, 1)
    c.upload()
    want = p.want()
    assert bool(torch.isnan(want[0]).any()) and bool(torch.isposinf(want[0]).any()) and bool(torch.isneginf(want[0]).any())
    alike(p.run(), want, kind)


def scores(views, table, lens, pt, power, at, bad):
    """Scores of 0, `power` where the infinite value lies, and for every third row a larger one behind it, of half the power's size."""
    for r, n in enumerate(lens):
        for t in range(n):
            views[0][table[r, t // pt], t % pt] = 0
        for t in at[r]:
            views[0][table[r, t // pt], t % pt, :, 0] = power if r % 3 else power + 20
            views[1][table[r, t // pt], t % pt, :, 3] = bad
        if r % 3 == 0:
            views[0][table[r, (n - 1) // pt], (n - 1) % pt, :, 0] = 20.0


@pytest.mark.parametrize("bad", [math.inf, -math.inf])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("pt", [8, 16])
@pytest.mark.parametrize("Hq", [4, 64])
def test_of_small_weights_under_trees(Hq, pt, kind, bad):
    """8 and 128 query rows of a cache head, in tiles that all see in full, in the last ones, and in rows in parts."""
    lens = [90, 300, 2500, 70]
    p = Drafts(lens, [2, 2, 2, 2], Hq, 1, 64, kind=kind, pt=pt, scale=math.log(2.0), shape="chain")
    p.q[:] = 0
    p.q[:, :, 0] = 1
    p.d_q.copy_(p.q)
    c = p.cache
    scores(c.views, c.table, lens, pt, LEAST[kind], [[2], [40, 297], [700, 2100], [66]], bad)
    c.upload()
    want = p.want()
    assert bool(torch.isinf(want[0][:, :, 3]).all())
    alike(p.run(), want, kind)


@pytest.mark.parametrize("bad", [math.inf, -math.inf])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("pt", [8, 16])
@pytest.mark.parametrize("Hq", [4, 64])
def test_of_small_weights_under_one_token(Hq, pt, kind, bad):
    lens = [90, 300, 2500, 70]
    p = Problem(lens, Hq, 1, 64, kind=kind, cache=kind, pt=pt, scale=math.log(2.0))
    p.q[:] = 0
    p.q[:, :, 0] = 1
    p.d["q"].copy_(p.q)
    views = [v.clone() for v in p.views]
    scores(views, p.table, lens, pt, LEAST[kind], [[2], [40, 297], [700, 2100], [66]], bad)
    p.views = views
    for pool, v in zip(p.pools, views):
        torch.as_strided(pool.view(v.dtype), v.shape, (*p.strides, 1)).copy_(v)
    want = p.want()
    assert bool(torch.isinf(want[0][:, :, 3]).all())
    alike(p.run(), want, kind)
