"""fdy_pages_extend where lists are long, pools large and books wrong: the kernel of more than 1,024 entries in every case that the one
of few has, more pages taken than a workgroup keeps at hand (4,096), free pages behind the first 65,536; and books with numbers out
of range between guard words, the good rows' results compared after every call."""
import numpy as np
import pytest
import torch

import oracle.decode as od
from paper_2604_06664_amd import decode as fdd
from test_gpu_pages import DEV, Pool

pytestmark = pytest.mark.gpu


def pool_of(rng, n_rows, row_pages, pt, spare, beams=1, n_planes=1):
    """Rows of random lengths in groups that hold the same pages, and `spare` pages that nobody holds."""
    lens = np.repeat(rng.integers(0, (row_pages - 1) * pt + 1, -(-n_rows // beams)), beams)[:n_rows]
    pages = -(-lens // pt)
    first = np.arange(n_rows) // beams * beams
    need = int(pages[first == np.arange(n_rows)].sum())
    table, refs = np.full((n_rows, row_pages), -3, int), np.zeros(need + spare, int)
    order, at = rng.permutation(len(refs)), 0
    for r in range(n_rows):
        if first[r] == r:
            mine = order[at:at + pages[r]]
            at += pages[r]
        table[r, :pages[r]] = mine
        refs[mine] += 1
    return Pool(refs, table, lens, pt, n_planes=n_planes, page_bytes=16, stride=16)


LENGTHS = [1025, 3000]


@pytest.mark.parametrize("n", LENGTHS)
@pytest.mark.parametrize("beams", [1, 3])
def test_rows_named_twice_or_none(n, beams):
    rng = np.random.default_rng(n + beams)
    p = pool_of(rng, 800, 5, 8, 6000, beams)
    for _ in range(2):
        rows = rng.integers(0, 800, n)
        rows[rng.integers(0, n, 60)] = -1
        rows[rng.integers(0, n, 60)] = 800
        rows[rng.integers(0, n, 9)] = [1 << 30, -(1 << 31), (1 << 31) - 1] * 3
        rows = [int(r) for r in rows]
        p.extend(rows, None)
        p.extend(rows, [int(c) for c in rng.integers(-2, 12, n)])
    assert p.want.status == od.ST_BAD_INDEX | od.ST_CAPACITY  # (rows that are full are among them)


@pytest.mark.parametrize("n", LENGTHS)
@pytest.mark.parametrize("beams", [1, 2, 4])
def test_too_few_pages(n, beams):
    rng = np.random.default_rng(7 * n + beams)
    for spare in (0, 1, n // 8, n // 3):
        p = pool_of(rng, n, 5, 8, spare, beams)
        p.extend([int(r) for r in rng.permutation(n)], [int(c) for c in rng.integers(0, 9, n)])
        assert p.want.status == od.ST_CAPACITY
        p.free([int(r) for r in rng.permutation(n)[:n // 10]])
        p.extend(None, None)


@pytest.mark.parametrize("n", LENGTHS)
def test_too_few_slots(n):
    rng = np.random.default_rng(11 * n)
    p = pool_of(rng, n, 9, 8, 4 * n, 2)
    p.extend(None, [int(c) for c in rng.integers(0, 9, n)], n_slots=3 * n)
    assert p.want.status == od.ST_CAPACITY
    p.extend([int(r) for r in rng.permutation(n)], None, n_slots=n - 100)
    p.extend([int(r) for r in rng.permutation(n)], None, n_slots=0)


@pytest.mark.parametrize("n", [12, 1000, 1025, 3000])
def test_rows_whose_books_are_wrong(n):
    """They get nothing and are left as they are; the others get what they would get without them."""
    rng = np.random.default_rng(13 * n)
    pt, row_pages = 8, 5
    p = pool_of(rng, n, row_pages, pt, 2 * n)
    bad = {}
    for r in rng.permutation(n)[:max(3, n // 10)]:
        r = int(r)
        kind = len(bad) % 4
        bad[r] = True
        if kind == 0:
            p.want.lens[r] = -1 - r
        elif kind == 1:
            p.want.lens[r] = row_pages * pt + 1 + r
        else:  # the partly filled last page is none
            p.want.lens[r] = 2 * pt + 3
            p.want.table[r, 2] = [len(p.want.refs), -1][kind - 2]
    p.table.copy_(torch.from_numpy(p.want.table))
    p.lens.copy_(torch.tensor(p.want.lens, dtype=torch.int32))
    rows = [int(r) for r in rng.permutation(n)]
    for counts in (None, [int(c) for c in rng.integers(0, 9, n)]):
        lists = [None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV) for x in (rows, counts)]
        total = n if counts is None else sum(counts)
        slots = torch.full((total,), -9, dtype=torch.int64, device=DEV)
        pos = torch.full((total,), -9, dtype=torch.int32, device=DEV)
        ws, size = p.ws(n)
        fdd.fdy_pages_extend(p.desc, *lists, n, slots, pos, total, ws, size, p.status)
        s, q = p.want.extend([-1 if r in bad else r for r in rows], counts, total)
        p.same()
        assert slots.cpu().tolist() == s.tolist() and pos.cpu().tolist() == q.tolist()
        assert p.want.status & od.ST_BAD_INDEX


@pytest.mark.parametrize("n", [600, 1024, 1025])
def test_more_pages_than_are_kept_at_hand_behind_the_first_65536(n):
    """Each row takes nine or ten pages of a pool of 80,000 of whose first 65,600 all but a few hundred are held."""
    rng = np.random.default_rng(n)
    pt, n_pages, row_pages = 2, 80_000, 200
    refs = np.zeros(n_pages, int)
    refs[:65_600] = 1
    refs[rng.integers(0, 65_600, 700)] = 0
    refs[rng.integers(65_600, n_pages, 1500)] = 1
    held = np.flatnonzero(refs)
    rng.shuffle(held)
    keepers = -(-len(held) // row_pages)  # rows behind the first n hold them
    table = np.full((n + keepers, row_pages), -1, int)
    table[n:].reshape(-1)[:len(held)] = held
    lens = [0] * n + [row_pages * pt] * keepers
    lens[-1] = (len(held) - (keepers - 1) * row_pages) * pt
    p = Pool(refs, table, lens, pt, n_planes=1, page_bytes=16, stride=16)
    p.extend(list(range(n)), [int(c) for c in rng.integers(17, 21, n)])
    assert p.want.status == 0 and sum(p.want.lens[:n]) // pt > 4096 and p.want.table[n - 1, 0] > 65_600
    p.extend([int(r) for r in rng.permutation(n)], [int(c) for c in rng.integers(0, 10, n)])
    p.extend([int(r) for r in rng.permutation(n)], [30] * n)  # more than are left
    assert p.want.status == od.ST_CAPACITY


class Guarded:
    """The books of six rows, three of them wrong, between guard words."""

    GUARD = 0x5A5A5A5A

    def __init__(self):
        pt, self.n_pages = 8, 16
        table = np.array([[0, 1, -1], [99, -4, -1], [2, 3, -1], [4, 5, -1], [12, 6, -1], [-1, -1, -1]], np.int32)
        lens = np.array([9, 12, 1000, -8, 16, 0], np.int32)
        refs = np.zeros(16, np.int32)
        refs[[0, 1, 2, 3, 4, 5, 12, 6]] = 1
        free = sum(1 << p for p in range(16) if refs[p] == 0)
        parts = dict(refs=refs, bits=np.array([free], np.int64).view(np.int32), table=table.reshape(-1), lens=lens,
                     plane=np.arange(16 * 4, dtype=np.int32))
        self.at, words = {}, 0
        for name, x in parts.items():
            words += 16
            self.at[name] = slice(words, words + len(x))
            words += -(-len(x) // 16) * 16
        self.host = np.full(words + 16, self.GUARD, np.int32)
        for name, x in parts.items():
            self.host[self.at[name]] = x
        self.all = torch.from_numpy(self.host.copy()).to(DEV)
        dev = {name: self.all[s] for name, s in self.at.items()}
        self.addr = torch.tensor([dev["plane"].data_ptr()], dtype=torch.int64, device=DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.desc = fdd.make_pages(refs=dev["refs"], free_bits=dev["bits"].view(torch.int64), table=dev["table"].view(6, 3),
                                   lens=dev["lens"], page_tokens=pt, planes=self.addr, page_bytes=16, page_stride=16)
        self.bytes = fdd.fdy_pages_workspace_bytes(self.desc, 8)
        self.ws = torch.full((self.bytes + 256,), 0x77, dtype=torch.uint8, device=DEV)

    def after(self):
        torch.cuda.synchronize()
        assert int(self.status) == od.ST_BAD_INDEX
        assert bool((self.ws[self.bytes:] == 0x77).all())
        got = self.all.cpu().numpy()
        inside = np.zeros(len(got), bool)
        for s in self.at.values():
            inside[s] = True
        assert (got[~inside] == self.GUARD).all()
        x = {name: got[s] for name, s in self.at.items()}
        return x["refs"], x["table"].reshape(6, 3), x["lens"], x["plane"].reshape(16, 4), int(x["bits"].view(np.int64)[0])


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def test_extend_between_guards():
    g = Guarded()
    slots = torch.full((7,), -9, dtype=torch.int64, device=DEV)
    pos = torch.full((7,), -9, dtype=torch.int32, device=DEV)
    fdd.fdy_pages_extend(g.desc, None, None, 6, slots, pos, 6, g.ws, g.bytes, g.status)
    refs, table, lens, plane, bits = g.after()
    assert slots.cpu().tolist() == [1 * 8 + 1, -1, -1, -1, 7 * 8, 8 * 8, -9] and int(pos[6]) == -9
    assert lens.tolist() == [10, 12, 1000, -8, 17, 1] and table[4].tolist() == [12, 6, 7] and table[5, 0] == 8
    assert refs.tolist() == [1] * 9 + [0] * 3 + [1] + [0] * 3 and bits == sum(1 << p for p in range(16) if refs[p] == 0)


def test_fork_between_guards():
    g = Guarded()
    fdd.fdy_pages_fork(g.desc, ints(4, 2, 1, 77, 0), ints(5, 3, 2, 0, 6), 5, g.ws, g.bytes, g.status)
    refs, table, lens, plane, bits = g.after()
    assert table[5, :2].tolist() == [12, 6] and lens[5] == 16 and refs[12] == 2 and refs[6] == 2
    assert table[0].tolist() == [0, 1, -1] and lens[0] == 9 and refs[0] == 1 and refs[1] == 1 and table[4].tolist() == [12, 6, -1]


def test_free_between_guards():
    g = Guarded()
    fdd.fdy_pages_free(g.desc, ints(0, 1, 3, 4, 9, -1), 6, g.status)
    refs, table, lens, plane, bits = g.after()
    assert lens[[0, 4]].tolist() == [0, 0] and refs[[0, 1, 6, 12]].tolist() == [0] * 4 and refs[[2, 3]].tolist() == [1, 1]
    freed = 1 << 12 | 1 << 6 | 3
    assert bits & freed == freed and not bits >> 16


def test_compact_between_guards():
    g = Guarded()
    to = torch.full((17,), -9, dtype=torch.int32, device=DEV)
    live = torch.zeros(1, dtype=torch.int32, device=DEV)
    fdd.fdy_pages_compact(g.desc, to, live, g.ws, g.bytes, g.status)
    refs, table, lens, plane, bits = g.after()
    assert int(live) == 8 and to.cpu().tolist() == list(range(7)) + [-1] * 5 + [7] + [-1] * 3 + [-9]
    assert table[4].tolist() == [7, 6, -1] and table[0].tolist() == [0, 1, -1] and lens.tolist() == [9, 12, 1000, -8, 16, 0]
    assert refs.tolist() == [1] * 8 + [0] * 8 and bits == 0xFF00 and plane[7].tolist() == [48, 49, 50, 51]


def test_copy_between_guards():
    g = Guarded()
    fdd.fdy_pages_copy(g.desc, ints(1, 77, 2, -5), ints(13, 3, -1, 16), 4, g.status)
    refs, table, lens, plane, bits = g.after()
    want = np.arange(64).reshape(16, 4)
    want[13] = want[1]
    assert np.array_equal(plane, want) and refs.sum() == 8
