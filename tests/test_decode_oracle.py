"""The oracle of the pages against what has to hold after any call, whatever the pool has left."""
import numpy as np
import pytest

import oracle.decode as od


def shares(rng, n_groups, beams, pt, free):
    """Groups of rows that hold the same pages, a partly filled last one among them, and `free` pages that nobody holds."""
    lens = np.repeat(rng.integers(1, 3 * pt, n_groups), beams)
    pages = -(-lens[::beams] // pt)
    table, refs = np.full((n_groups * beams, 6), -1, int), np.zeros(int(pages.sum()) + free, int)
    order, at = rng.permutation(len(refs)), 0
    for g, k in enumerate(pages):
        table[g * beams:(g + 1) * beams, :k] = order[at:at + k]
        refs[order[at:at + k]] = beams
        at += k
    return refs, table, lens


@pytest.mark.parametrize("seed", range(20))
def test_a_new_token_goes_to_a_page_of_its_row_alone(seed):
    rng = np.random.default_rng(seed)
    pt, beams = 8, int(rng.integers(2, 5))
    refs, table, lens = shares(rng, 6, beams, pt, int(rng.integers(0, 12)))
    b = od.Books(refs, table, lens, pt, np.arange(len(refs))[None, :, None])
    for _ in range(6):
        rows = [int(r) for r in rng.permutation(len(lens))[:int(rng.integers(1, len(lens) + 1))]]
        slots, _ = b.extend(rows, None, len(rows))
        for s in slots:
            if s >= 0:
                assert b.refs[s // pt] == 1, "a token is written to a page that another row holds"
        counts = np.bincount([p for r in range(len(lens)) for p in b.held(r)], minlength=len(refs))
        assert counts.tolist() == b.refs


def test_rows_that_keep_a_page_wait_for_the_other_holders():
    """Two rows of one partly filled page and no page left: the first gets no copy, so the second must not go on in the page."""
    b = od.Books([2], [[0], [0]], [5, 5], 16)
    slots, _ = b.extend([0, 1], None, 2)
    assert slots.tolist() == [-1, -1] and b.lens == [5, 5] and b.status == od.ST_CAPACITY
