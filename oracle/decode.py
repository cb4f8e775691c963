"""Oracle of the decode operators (include/fdy_decode.h): the definitions, in 64 bits, one token, row and page after the
other, on the CPU.  TEST INFRASTRUCTURE ONLY, like the rest of this package; shares nothing with the product's code."""
from __future__ import annotations

import math

import numpy as np
import torch

F8_MOST = 448.0
ST_CAPACITY, ST_BAD_INDEX = 1, 2


# ---- rotary positions ---------------------------------------------------------------------------
def rope_frequencies(rot, base=10000.0, scaling="plain", factor=1.0, low=1.0, high=32.0, trained=4096.0):
    """The rot / 2 frequencies of the header's five schemes, as mathematics says them."""
    out = []
    b = base * factor ** (rot / (rot - 2)) if scaling == "ntk" else base

    def pair_at(turns):  # the pair that makes `turns` turns over the trained length: trained * base^(-2i/rot) = 2 pi turns
        return rot / 2 * math.log(trained / (2 * math.pi * turns)) / math.log(base)

    for i in range(rot // 2):
        f = b ** (-2 * i / rot)
        if scaling == "linear":
            f = f / factor
        elif scaling == "yarn":
            lo = min(max(math.floor(pair_at(high)), 0), rot - 1)
            hi = min(max(math.ceil(pair_at(low)), 0), rot - 1)
            hi = hi if hi > lo else lo + 0.001
            kept = 1 - min(max((i - lo) / (hi - lo), 0), 1)
            f = f * kept + f / factor * (1 - kept)
        elif scaling == "bands":
            turns = trained * f / (2 * math.pi)
            if turns < low:
                f = f / factor
            elif turns <= high:
                s = (turns - low) / (high - low)
                f = (1 - s) * f / factor + s * f
        out.append(f)
    return np.array(out)


def rope_table(freqs, first, n, magnitude=1.0):
    """[n, 2, rot / 2] in 64 bits; angles by exact reduction in extended precision where the platform has it."""
    p = np.arange(first, first + n, dtype=np.longdouble)[:, None] * np.asarray(freqs, np.longdouble)
    return np.stack([np.cos(p), np.sin(p)], 1).astype(np.float64) * magnitude


def turned(x, table_row, rot, layout):
    """x [heads, dim] (64 bits) turned by one table row [2, rot / 2]; also the size of the terms that were added."""
    y, size = x.clone(), x.abs()
    for i in range(rot // 2):
        a, b = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
        c, s = float(table_row[0, i]), float(table_row[1, i])
        y[:, a] = x[:, a] * c - x[:, b] * s
        y[:, b] = x[:, b] * c + x[:, a] * s
        size[:, a] = (x[:, a] * c).abs() + (x[:, b] * s).abs()
        size[:, b] = (x[:, b] * c).abs() + (x[:, a] * s).abs()
    return y, size


# ---- attention ----------------------------------------------------------------------------------
def attend(q, k_view, v_view, table, lens, scale, window=0, rows=None, k_scale=None, v_scale=None):
    """q [seqs, heads, dim]; k_view, v_view [page, token, head, dim] of stored elements; all CPU.
    -> out, lse (64 bits), spread: the largest |v| among what a row sees."""
    B, Hq, D = q.shape
    n_pages, pt, H, _ = k_view.shape
    group = Hq // H
    out = torch.zeros(B, Hq, D, dtype=torch.float64)
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64)
    spread = torch.zeros(B, Hq, dtype=torch.float64)
    for s in range(B):
        r = s if rows is None else int(rows[s])
        if not 0 <= r < table.shape[0]:
            continue
        n = min(max(int(lens[r]), 0), table.shape[1] * pt)
        at = [t for t in range(max(0, n - window) if window else 0, n) if 0 <= int(table[r, t // pt]) < n_pages]
        if not at:
            continue
        page = torch.tensor([int(table[r, t // pt]) for t in at])
        place = torch.tensor([t % pt for t in at])
        k, v = k_view[page, place].double(), v_view[page, place].double()
        if k_scale is not None:
            k = k * k_scale.double()[:, None]
        if v_scale is not None:
            v = v * v_scale.double()[:, None]
        for h in range(Hq):
            x = scale * (k[:, h // group] @ q[s, h].double())
            m = x.max()
            if m == -math.inf:
                continue
            e = torch.exp(x - m)
            out[s, h] = (e[:, None] * v[:, h // group]).sum(0) / e.sum()
            lse[s, h] = m + torch.log(e.sum())
            spread[s, h] = v[:, h // group].abs().max()
    return out, lse, spread


# ---- pages --------------------------------------------------------------------------------------
class Books:
    """A pool's books and contents as plain lists; every call as the header says it, one entry after the other."""

    def __init__(self, refs, table, lens, page_tokens, planes=None):
        self.refs = [int(x) for x in refs]
        self.table = np.array(table, np.int32)
        self.lens = [int(x) for x in lens]
        self.pt = page_tokens
        self.planes = None if planes is None else np.array(planes)  # [plane, page, ...]
        self.status = 0

    def copy(self):
        b = Books(self.refs, self.table, self.lens, self.pt, self.planes)
        b.status = self.status
        return b

    def pages_of(self, n):
        return -(-n // self.pt)

    def free_bits(self):
        bits = np.zeros(-(-len(self.refs) // 64) * 64, np.uint8)
        bits[:len(self.refs)] = [r == 0 for r in self.refs]
        return np.packbits(bits, bitorder="little").view(np.uint64)

    def held(self, r):
        return [int(p) for p in self.table[r, :self.pages_of(self.lens[r])]]

    def extend(self, rows, counts, n_slots):
        """-> (slots, positions), packed."""
        n = len(counts) if rows is None else len(rows)
        rows = list(range(n)) if rows is None else [int(r) for r in rows]
        counts = [1] * n if counts is None else [int(c) for c in counts]
        for i, c in enumerate(counts):
            if c < 0:
                self.status |= ST_BAD_INDEX
                counts[i] = 0
        seen, good = set(), []
        for r in rows:
            ok = 0 <= r < len(self.lens) and r not in seen
            if not ok:
                self.status |= ST_BAD_INDEX
            seen.add(r)
            good.append(ok)
        begin = np.concatenate([[0], np.cumsum(counts)]).astype(int)
        # who asks for a shared, partly filled last page
        fits, last, asks = [], [], {}
        for i, r in enumerate(rows):
            ok = good[i] and counts[i] > 0
            if ok and (self.lens[r] + counts[i] > self.table.shape[1] * self.pt or begin[i + 1] > n_slots):
                self.status |= ST_CAPACITY
                ok = False
            fits.append(ok)
            p = int(self.table[r, self.lens[r] // self.pt]) if ok and self.lens[r] % self.pt else -1
            last.append(p)
            if p >= 0 and self.refs[p] > 1:
                asks.setdefault(p, []).append(i)
        copies, others = [False] * n, [[] for _ in rows]
        for p, who in asks.items():
            keeps = len(who) == self.refs[p]
            for i in who[:-1] if keeps else who:
                copies[i] = True
            if keeps:
                others[who[-1]] = who[:-1]
        need = [(self.pages_of(self.lens[r] + counts[i]) - self.pages_of(self.lens[r]) + copies[i]) if fits[i] else 0
                for i, r in enumerate(rows)]
        free = [p for p, c in enumerate(self.refs) if c == 0]
        slots, positions = [], []
        taken, moved, got = 0, [], []
        for i, r in enumerate(rows):
            served = fits[i]
            if served and need[i] and taken + need[i] > len(free):
                self.status |= ST_CAPACITY
                served = False
            if served and not all(got[j] for j in others[i]):  # the page that it would keep is still another's as well
                self.status |= ST_CAPACITY
                served = False
            got.append(served)
            mine = free[taken:taken + need[i]]
            taken += need[i]
            old = self.lens[r] if good[i] else 0
            if served:
                before = self.pages_of(old)
                if copies[i]:
                    moved.append((last[i], mine[0]))
                    self.table[r, before - 1] = mine[0]
                    mine = mine[1:]
                self.table[r, before:before + len(mine)] = mine
                self.lens[r] = old + counts[i]
                for j in range(counts[i]):
                    t = old + j
                    slots.append(int(self.table[r, t // self.pt]) * self.pt + t % self.pt)
            else:
                slots += [-1] * counts[i]
            positions += [old + j for j in range(counts[i])]
            for p in ([moved[-1][1]] if served and copies[i] else []) + (mine if served else []):
                self.refs[p] = 1
        before = None if self.planes is None else self.planes.copy()
        for src, dst in moved:
            self.refs[src] -= 1
            if before is not None:
                self.planes[:, dst] = before[:, src]
        return np.array(slots[:n_slots], np.int64), np.array(positions[:n_slots], np.int32)

    def fork(self, src, dst):
        old_table, old_lens = self.table.copy(), list(self.lens)
        seen, change = set(), []
        for s, d in zip(src, dst):
            s, d = int(s), int(d)
            ok = 0 <= s < len(self.lens) and 0 <= d < len(self.lens) and d not in seen
            if 0 <= d < len(self.lens):
                seen.add(d)
            if not ok:
                self.status |= ST_BAD_INDEX
            else:
                change.append((s, d))
        for s, d in change:
            for p in old_table[d, :self.pages_of(old_lens[d])]:
                self.refs[p] -= 1
            for j, p in enumerate(old_table[s, :self.pages_of(old_lens[s])]):
                self.refs[p] += 1
                self.table[d, j] = p
            self.lens[d] = old_lens[s]

    def free(self, rows):
        seen = set()
        for r in rows:
            r = int(r)
            if not 0 <= r < len(self.lens) or r in seen:
                self.status |= ST_BAD_INDEX
                continue
            seen.add(r)
            for p in self.held(r):
                self.refs[p] -= 1
            self.lens[r] = 0

    def compact(self):
        """-> (map, n_live)"""
        n_live = sum(c > 0 for c in self.refs)
        holes = [p for p in range(n_live) if self.refs[p] == 0]
        movers = [p for p in range(n_live, len(self.refs)) if self.refs[p] > 0]
        to = [p if c > 0 else -1 for p, c in enumerate(self.refs)]
        for src, dst in zip(movers, holes):
            to[src] = dst
            self.refs[dst], self.refs[src] = self.refs[src], 0
            if self.planes is not None:
                self.planes[:, dst] = self.planes[:, src]
        for r in range(len(self.lens)):
            for j in range(self.pages_of(self.lens[r])):
                self.table[r, j] = to[self.table[r, j]]
        return np.array(to, np.int32), n_live
