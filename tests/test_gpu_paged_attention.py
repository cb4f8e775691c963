"""fdy_paged_attention through the C ABI against its definition in 64 bits.

Tolerances.  Each weight e^(x - max) is rounded to the queries' type for its product with v (2^-8 of it for bf16, 2^-11 for
f16), so the output moves by at most that share of the largest |v| that the row sees; scores are sums of up to 256 products
in 32 bits, |x| stays below 64 here, which with the exponential is allowed 2^-13 more; the result is rounded once.  lse: up to
256 roundings of 2^-24 of terms that add up to less than 16 in size (3e-4)."""
import math

import numpy as np
import pytest
import torch

import oracle.decode as od
from paper_2604_06664_amd import decode as fdd

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = dict(bf16=torch.bfloat16, f16=torch.float16, f8=torch.float8_e4m3fn)
ROUND = dict(bf16=2.0 ** -8, f16=2.0 ** -11)
NAN_F8 = 0x7F


class Problem:
    """Rows of the given lengths over scattered pages; everything that no row holds is NaN."""

    def __init__(self, lens, Hq, H, D, pt=16, order="token", kind="bf16", cache="bf16", window=0, seed=1, row_pages=None,
                 pad=0, scale=None, spare=3, sharp=1.0, first_tokens_gone=False):
        rng = np.random.default_rng(seed)
        self.lens, self.window, self.kind, self.cache, self.H, self.D = list(lens), window, kind, cache, H, D
        B, pages = len(lens), [-(-n // pt) for n in lens]
        P = row_pages or max(pages + [1]) + 2
        n_pages = sum(pages) + spare
        order_of = rng.permutation(n_pages)
        table = np.full((B, P), -1, np.int32)
        at = 0
        for r, n in enumerate(pages):
            table[r, :n] = order_of[at:at + n]
            at += n
        ts = (H * (D + pad)) if order == "token" else D + pad
        hs = (D + pad) if order == "token" else pt * (D + pad)
        ps = pt * H * (D + pad) + pad
        self.strides = (ps, ts, hs)
        bits = torch.uint8 if cache == "f8" else torch.int16
        nan = torch.tensor([NAN_F8], dtype=torch.uint8) if cache == "f8" else torch.tensor([math.nan]).to(DTYPES[cache]).view(bits)
        self.pools, self.views = [], []
        for _ in "kv":
            pool = nan.repeat(n_pages * ps)
            view = torch.as_strided(pool, (n_pages, pt, H, D), (ps, ts, hs, 1))
            for r, n in enumerate(lens):
                lo = max(0, n - window) if window and first_tokens_gone else 0
                for j in range(pages[r]):
                    a, b = max(lo, j * pt), min(n, (j + 1) * pt)
                    if a < b:
                        x = torch.from_numpy(rng.standard_normal((b - a, H, D)).astype(np.float32)).to(DTYPES[cache]).view(bits)
                        view[table[r, j], a - j * pt:b - j * pt] = x
                    elif first_tokens_gone:
                        table[r, j] = -7  # given away
            dev = pool.to(DEV)
            self.pools.append(dev)
            self.views.append(view.view(DTYPES[cache]))
        self.scales = [torch.from_numpy(rng.uniform(0.5, 1.5, H).astype(np.float32)) if cache == "f8" else None for _ in "kv"]
        self.q = torch.from_numpy(rng.standard_normal((B, Hq, D)).astype(np.float32) * sharp).to(DTYPES[kind])
        self.scale = D ** -0.5 if scale is None else scale
        self.table, self.n_pages, self.pt = table, n_pages, pt
        self.d = dict(q=self.q.to(DEV), out=torch.full((B, Hq, D), 5.0, dtype=DTYPES[kind], device=DEV),
                      lse=torch.full((B, Hq), 5.0, device=DEV), table=torch.from_numpy(table).to(DEV),
                      lens=torch.tensor(self.lens, dtype=torch.int32, device=DEV), status=torch.zeros(1, dtype=torch.int32, device=DEV),
                      scales=[None if s is None else s.to(DEV) for s in self.scales])
        self.ws = None

    def desc(self, **kw):
        d = self.d
        kv = fdd.make_kv(*self.pools, type=fdd.TYPES[self.cache], n_pages=self.n_pages, page_tokens=self.pt, n_heads=self.H,
                         head_dim=self.D, page_stride=self.strides[0], token_stride=self.strides[1],
                         head_stride=self.strides[2], k_scale=d["scales"][0], v_scale=d["scales"][1])
        args = dict(q=d["q"], out=d["out"], lse=d["lse"], table=d["table"], lens=d["lens"], kv=kv, scale=self.scale,
                    window=self.window)
        args.update(kw)
        return fdd.make_attend_desc(**args)

    def run(self, **kw):
        desc = self.desc(**kw)
        n = fdd.fdy_paged_attention_workspace_bytes(desc)
        if self.ws is None or self.ws.numel() < n:
            self.ws = torch.zeros(n, dtype=torch.uint8, device=DEV)
        fdd.fdy_paged_attention(desc, self.ws, n, self.d["status"])
        torch.cuda.synchronize()
        return self.d["out"].cpu(), self.d["lse"].cpu(), int(self.d["status"])

    def want(self, rows=None, lens=None, table=None, q=None):
        return od.attend(self.q if q is None else q, *self.views, self.table if table is None else table,
                         self.lens if lens is None else lens, self.scale, self.window, rows, *self.scales)


def near(got, want, kind):
    (out, lse), (o, l, spread) = got[:2], want
    u = ROUND[kind]
    bound = spread[..., None] * (u + 2.0 ** -13) + u * o.abs() + 2.0 ** -24
    err = (out.double() - o).abs()
    assert bool((err <= bound).all()), (float((err - bound).max()), int((~(err <= bound)).sum()))
    none = l == -math.inf
    assert torch.equal(lse == -math.inf, none)
    assert bool(((lse.double() - l).abs()[~none] <= 3e-4).all())
    assert bool((out[none] == 0).all())


def check(*args, **kw):
    p = Problem(*args, **kw)
    got = p.run()
    assert got[2] == 0
    near(got, p.want(), p.kind)
    assert bool((p.ws[: len(p.lens) * p.H * 4] == 0).all())  # the counters, one a row and cache head at least, are left at zero
    return p, got


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 300]


@pytest.mark.parametrize("kind,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "f8"), ("f16", "f8")])
@pytest.mark.parametrize("D", [64, 128, 256, 16, 48, 80, 96, 160, 192])
def test_lengths_around_tiles(D, kind, cache):
    check(EDGES, 4, 2, D, kind=kind, cache=cache)


@pytest.mark.parametrize("D", [8, 24, 40, 72, 136, 248])
def test_head_sizes_that_are_odd_multiples_of_8(D):
    check([1, 33, 130], 3, 3, D, kind="f16", cache="f16")


@pytest.mark.parametrize("Hq,H", [(1, 1), (3, 3), (7, 1), (15, 1), (16, 1), (17, 1), (32, 1), (40, 2), (64, 4), (70, 2), (100, 1)])
def test_groups(Hq, H):
    check([5, 100, 0, 333], Hq, H, 64)
    check([290], Hq, H, 128, cache="f8", order="head")


@pytest.mark.parametrize("Hq,H,D,cache", [(20, 1, 256, "bf16"), (20, 1, 256, "f8"), (33, 1, 128, "bf16"), (64, 2, 96, "f8"), (24, 1, 80, "bf16")])
def test_groups_over_long_and_small_pages(Hq, H, D, cache):
    check([2500, 17, 0, 700], Hq, H, D, cache=cache)
    check([600, 17], Hq, H, D, cache=cache, pt=8)


@pytest.mark.parametrize("order", ["token", "head"])
@pytest.mark.parametrize("pt", [1, 2, 4, 8, 16, 32, 128, 1024])
def test_page_sizes(pt, order):
    check([1, 17, 40, 129, 200], 4, 2, 64, pt=pt, order=order)
    check([3, 70], 4, 2, 128, pt=pt, order=order, kind="f16", cache="f8")


@pytest.mark.parametrize("window", [1, 2, 16, 31, 33, 64, 100, 1000])
@pytest.mark.parametrize("pt", [4, 16, 64])
def test_windows_and_what_lies_before_them(window, pt):
    check([0, 1, 30, 64, 65, 100, 333, 520], 4, 2, 64, pt=pt, window=window, first_tokens_gone=True)


@pytest.mark.parametrize("lens", [[4000], [3001, 5], [1, 700, 2300, 31], [2049] * 3])
@pytest.mark.parametrize("D,cache", [(64, "bf16"), (128, "f8"), (256, "bf16")])
def test_rows_in_pieces(lens, D, cache):
    p, got = check(lens, 8, 2, D, cache=cache, sharp=2.0)
    for _ in range(2):  # the same every time, over the same workspace
        again = p.run()
        assert torch.equal(again[0].view(torch.int16), got[0].view(torch.int16)) and torch.equal(again[1], got[1])


def test_many_rows():
    rng = np.random.default_rng(4)
    lens = [int(x) for x in rng.integers(0, 60, 700)]
    lens[123] = 3000
    check(lens, 2, 1, 64)


@pytest.mark.parametrize("Hq,H,D,cache", [(8, 2, 64, "bf16"), (16, 4, 128, "f8"), (5, 1, 256, "bf16")])
def test_batches_of_many_sizes_in_turn_over_one_workspace(Hq, H, D, cache):
    rng = np.random.default_rng(5)
    batches = [[int(x) for x in rng.integers(0, 500, 96)] + [2800, 1900], [2500, 17], [3000], [600, 0, 900, 1500, 40], [9] * 40]
    problems = [Problem(lens, Hq, H, D, cache=cache, row_pages=200) for lens in batches]
    ws = torch.zeros(fdd.fdy_paged_attention_workspace_bytes(problems[0].desc()), dtype=torch.uint8, device=DEV)
    wants = [p.want() for p in problems]
    for i in [0, 1, 0, 2, 3, 0, 4, 1, 3, 0]:
        p = problems[i]
        p.ws = ws
        near(p.run(), wants[i], p.kind)
        assert p.ws is ws  # it was wide enough


@pytest.mark.parametrize("lens", [[40, 0, 0], [0, 0, 0, 0], [0, 0], [300, 9, 0, 0, 0, 0, 0]])
@pytest.mark.parametrize("n", [1, 2])
def test_nothing_behind_the_last_sequence_is_written(lens, n):
    p = Problem(lens, 4, 2, 64)  # only the first n are asked for; rows behind them are empty, as the last asked for may be
    out, lse = p.d["out"], p.d["lse"]
    p.run(q=p.d["q"][:n], out=out[:n], lse=lse[:n])
    o, l = p.want()[:2]
    assert torch.equal(lse.cpu()[:n] == -math.inf, l[:n] == -math.inf)
    assert bool((out[n:] == 5).all()) and bool((lse[n:] == 5).all())


WIDE = 8192 // 16  # pages of a table that allows long rows, whatever their lengths are


@pytest.mark.parametrize("lens", [EDGES, [2500, 17, 0, 700], [5, 0, 9, 0], [3000], [1, 2, 3] * 90 + [0]])
@pytest.mark.parametrize("D,kind,cache", [(128, "bf16", "bf16"), (128, "f16", "f8"), (64, "f16", "f16"), (80, "bf16", "bf16"), (48, "bf16", "f8")])
def test_tables_that_allow_long_rows(lens, D, kind, cache):
    check(lens, 8, 4, D, kind=kind, cache=cache, row_pages=WIDE)
    check(lens[:6], 3, 1, D, kind=kind, cache=cache, row_pages=WIDE, order="head")


@pytest.mark.parametrize("Hq,H", [(1, 1), (16, 1), (32, 1), (40, 1), (64, 2), (33, 3), (100, 1), (24, 8)])
@pytest.mark.parametrize("D,cache", [(64, "bf16"), (128, "f8"), (128, "bf16")])
def test_groups_in_tables_that_allow_long_rows(Hq, H, D, cache):
    p, got = check([1900, 0, 333, 64, 2100], Hq, H, D, cache=cache, row_pages=WIDE, sharp=2.0)
    again = p.run()  # the same every time, over the same workspace
    assert torch.equal(again[0].view(torch.int16), got[0].view(torch.int16)) and torch.equal(again[1], got[1])


@pytest.mark.parametrize("Hq,H", [(8, 4), (16, 1), (20, 1), (3, 1)])
def test_wide_heads_of_8_bits_in_tables_that_allow_long_rows(Hq, H):
    for D in (192, 256):
        check([1900, 0, 333, 64, 2100, 31], Hq, H, D, cache="f8", row_pages=WIDE)
        check([9, 0, 100, 0], Hq, H, D, cache="f8", row_pages=WIDE)


def test_windows_in_tables_that_allow_long_rows():
    for window in (1, 33, 500):
        check([0, 1, 64, 333, 1520, 2000], 4, 2, 128, row_pages=WIDE, window=window, first_tokens_gone=True)


def test_wide_and_narrow_tables_in_turn_over_one_workspace():
    wide = Problem([900, 5, 2400, 31], 8, 4, 128, row_pages=WIDE)
    narrow = Problem([900, 5, 2400, 31], 8, 4, 128)
    few = Problem([4], 8, 4, 128)
    ws = torch.zeros(fdd.fdy_paged_attention_workspace_bytes(wide.desc()), dtype=torch.uint8, device=DEV)
    for p in (wide, narrow, wide, few, narrow, few, wide):
        p.ws = ws
        near(p.run(), p.want(), "bf16")
        assert p.ws is ws


def test_table_far_wider_than_the_rows():
    check([40, 700], 4, 2, 64, row_pages=5000)


def test_padded_strides():
    check([5, 100, 290], 4, 2, 64, pad=8)
    check([5, 100, 290], 4, 2, 80, pad=16, cache="f8", order="head")


def test_strided_queries_and_outputs():
    p = Problem([9, 77], 4, 2, 64)
    wide = torch.zeros(2, 4, 3, 64, dtype=torch.bfloat16, device=DEV)
    q = wide[:, :, 1]
    q.copy_(p.d["q"])
    out = torch.full((4, 2, 72), 5.0, dtype=torch.bfloat16, device=DEV)
    p.run(q=q, out=out[:, :, :64].transpose(0, 1), lse=None)
    o, _, spread = p.want()
    got = out.cpu()
    near((got[:, :, :64].transpose(0, 1).contiguous(), p.want()[1].float()), p.want(), "bf16")
    assert bool((got[:, :, 64:] == 5).all())


def test_rows_of_a_larger_pool():
    p = Problem([9, 77, 150, 0, 40], 4, 2, 64)
    rows = [4, 0, 2, 2]
    d_rows = torch.tensor(rows, dtype=torch.int32, device=DEV)
    out, lse = torch.empty(4, 4, 64, dtype=torch.bfloat16, device=DEV), torch.empty(4, 4, device=DEV)
    desc = p.desc(q=p.d["q"][:4], out=out, lse=lse, rows=d_rows)
    n = fdd.fdy_paged_attention_workspace_bytes(desc)
    ws = torch.zeros(n, dtype=torch.uint8, device=DEV)
    fdd.fdy_paged_attention(desc, ws, n, p.d["status"])
    near((out.cpu(), lse.cpu()), p.want(rows=rows, q=p.q[:4]), "bf16")
    assert int(p.d["status"]) == 0


@pytest.mark.parametrize("pt", [8, 32])
def test_numbers_out_of_range_are_left_out(pt):
    p = Problem([100, 50, 64, 90, 130], 4, 2, 64, pt=pt)
    table, lens = p.table.copy(), list(p.lens)
    table[0, 1] = p.n_pages  # a page that is none
    table[3, 0] = -1
    lens[1] = -3
    lens[4] = 1 << 30  # held to the table's width: entries behind the row's own pages are -1
    p.d["table"].copy_(torch.from_numpy(table))
    p.d["lens"].copy_(torch.tensor(lens, dtype=torch.int32))
    for v in p.views:  # its last page's tail is seen now
        v.view(torch.int16)[table[4, 130 // pt], 130 % pt:] = 0x3F80
    for i in range(2):
        p.pools[i].copy_(p.views[i].view(torch.int16).as_strided((p.pools[i].numel(),), (1,)))
    got = p.run()
    assert got[2] == od.ST_BAD_INDEX
    near(got, p.want(lens=lens, table=table), "bf16")
    rows = torch.tensor([2, 7, -1, 2, 2], dtype=torch.int32, device=DEV)
    p.d["status"].zero_()
    got = p.run(rows=rows)
    assert got[2] == od.ST_BAD_INDEX
    near(got, p.want(lens=lens, table=table, rows=rows.tolist()), "bf16")


def test_infinite_and_nan_scores():
    """Values of the row itself: as the formula has them."""
    for pt in (8, 16):
        p = Problem([40, 40, 40, 40], 2, 1, 64, pt=pt)
        kb, vb = (v.clone() for v in p.views)
        p.q[:] = 1.0
        p.d["q"].copy_(p.q)
        kb[p.table[0, 0], 3] = -math.inf  # weight 0
        for j in range(-(-40 // pt)):  # all weights 0
            n = min(pt, 40 - j * pt)
            kb[p.table[1, j], :n] = -math.inf
        kb[p.table[2, 1], 1, :, 7] = math.nan
        vb[p.table[3, 0], 2, :, 5] = math.inf
        for i, v in enumerate((kb, vb)):
            p.views[i] = v
            p.pools[i].copy_(v.contiguous().view(torch.int16).flatten())
        out, lse, status = p.run()
        assert status == 0
        want = p.want()
        near((out[:2], lse[:2]), [w[:2] for w in want], "bf16")
        assert bool(torch.isnan(out[2]).all()) and bool(torch.isnan(lse[2]).all())
        assert bool(torch.isinf(out[3, :, 5]).all()) and bool(torch.isfinite(out[3, :, :5]).all())


def test_large_scores_do_not_overflow():
    p, (out, lse, _) = None, (None, None, None)
    p = Problem([70, 300], 4, 2, 64, sharp=1.0, scale=4.0)  # scores up to about 150, weights mostly 0
    got = p.run()
    o, l, spread = p.want()
    u = ROUND["bf16"]
    # scores of this size carry 2^-24 * 64 * 150 of error into the exponent
    bound = spread[..., None] * (u + 2.0 ** -10) + u * o.abs()
    assert bool(((got[0].double() - o).abs() <= bound).all())
    assert bool(((got[1].double() - l).abs() <= 1e-3).all())


def test_offsets_behind_32_bits():
    """Pages a GiB apart: the pool's last page starts 6 GiB in."""
    D, pt, n_pages, ps = 64, 16, 7, 1 << 29
    pools = [torch.empty(n_pages * ps // 2, dtype=torch.int32, device=DEV) for _ in "kv"]
    small = Problem([60], 2, 1, D, spare=0)
    for src, dst in zip(small.pools, pools):
        x = src.view(4, pt * D)
        flat = dst.view(torch.int16)
        for j in range(4):
            flat[(n_pages - 1 - j) * ps:(n_pages - 1 - j) * ps + pt * D] = x[j]
    table = torch.from_numpy(np.where(small.table >= 0, n_pages - 1 - small.table, -1).astype(np.int32)).to(DEV)
    kv = fdd.make_kv(*pools, type=fdd.FDY_BF16, n_pages=n_pages, page_tokens=pt, n_heads=1, head_dim=D, page_stride=ps,
                     token_stride=D, head_stride=D)
    got = small.run(kv=kv, table=table)
    near(got, small.want(), "bf16")
    small_pages = Problem([56], 2, 1, D, pt=8, spare=0)  # and where every lane finds its own page
    for src, dst in zip(small_pages.pools, pools):
        x = src.view(n_pages, 8 * D)
        flat = dst.view(torch.int16)
        for j in range(n_pages):
            flat[j * ps:j * ps + 8 * D] = x[j]
    kv.page_tokens = 8
    got = small_pages.run(kv=kv)
    near(got, small_pages.want(), "bf16")


def test_replays_while_rows_grow():
    """One captured launch on a stream of its own; lengths, tables and queries change between the replays."""
    p = Problem([900, 1500, 64], 4, 2, 64)
    p.ws = torch.zeros(fdd.fdy_paged_attention_workspace_bytes(p.desc()), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        p.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fdd.fdy_paged_attention(p.desc(), p.ws, p.ws.numel(), p.d["status"])
    for lens in ([1, 0, 3], [300, 1500, 64], [900, 33, 1], [899, 1499, 63], [900, 1500, 64]):
        p.lens = lens
        p.d["lens"].copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        near((p.d["out"].cpu(), p.d["lse"].cpu()), p.want(), "bf16")
    assert int(p.d["status"]) == 0


def test_no_sequences():
    p = Problem([5], 2, 1, 64)
    d = p.desc()
    d.n_seqs = 0
    fdd.fdy_paged_attention(d, None, 0)
    torch.cuda.synchronize()
    assert bool((p.d["out"] == 5).all())


def put(p, which, values):
    """values [row][token, head, dim] in the place of the rows' keys (0) or values (1), on both sides."""
    view = p.views[which].clone().contiguous()
    for r, x in enumerate(values):
        for t in range(x.shape[0]):
            view[p.table[r, t // p.pt], t % p.pt] = x[t].to(view.dtype)
    p.views[which] = view
    p.pools[which].copy_(view.view(torch.uint8 if p.cache == "f8" else torch.int16).flatten())


@pytest.mark.parametrize("kind,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "f8"), ("f16", "f8")])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scores_of_any_size(kind, cache, sign):
    """Scores of 2^20 to 2^30 (2^60 with bf16), which are not more than a few bits of 32: the largest, of one token or of three,
    take all the weight, and the weight is theirs in full.  Each score is one exact product, so nothing but the rounding of
    weights and result is allowed: 1 or 1/3 of at most 4."""
    lens, most = [40, 300, 3000, 1], 30 if kind == "f16" else 60
    p = Problem(lens, 8, 2, 64, kind=kind, cache=cache, scale=sign * 1.75, seed=21)
    rng = np.random.default_rng(22)
    wide = 8 if cache == "f8" else 15 if kind == "f16" else 30  # bits of the largest key
    sizes = np.linspace(20, most, 8) - wide
    # keys of a few bits, three of them or one the largest; queries with some bits of their own
    q = torch.zeros_like(p.q)
    q[:, :, 0] = torch.from_numpy(2.0 ** np.minimum(sizes, 15 if kind == "f16" else 100) * rng.uniform(1, 1.9, (4, 8))).to(q.dtype)
    p.q = q
    p.d["q"].copy_(q)
    keys = []
    for n in lens:
        k = torch.zeros(n, 2, 64)
        k[:, :, 0] = torch.from_numpy(rng.integers(-6, 6, (n, 2)).astype(np.float32)) * 2.0 ** (wide - 4)
        for h in range(2):
            k[rng.permutation(n)[:3 if h else 1], h, 0] = 7.0 * 2.0 ** (wide - 4)
        keys.append(k * sign)
    put(p, 0, keys)
    if p.scales[0] is not None:
        for s, d in zip(p.scales, p.d["scales"]):
            s.copy_(torch.tensor([0.5, 2.0]))  # products stay exact
            d.copy_(s)
    out, lse, status = p.run()
    assert status == 0
    o, l, spread = p.want()
    u = ROUND[kind]
    assert bool(((out.double() - o).abs() <= 2 * u * spread[..., None]).all()), float((out.double() - o).abs().max())
    assert bool(((lse.double() - l).abs() <= l.abs() * 2.0 ** -21 + 1e-6).all())


@pytest.mark.parametrize("kind,cache", [("bf16", "bf16"), ("f16", "f16"), ("f16", "f8")])
@pytest.mark.parametrize("pt", [4, 16])
def test_many_small_weights_beside_large_ones(kind, cache, pt):
    """In every 32 tokens one takes nearly all the weight and has the value 0; what comes out is of the others, whose scores are
    up to 20 below.  Relative to the result: one rounding of a weight to the type and one of the result (in f16 half the smallest
    step, 2^-25, where that is more), and 2^-13 for scores of this size and the exponential.  (Heads differ in how far below.)"""
    lens = [33, 300, 2111, 64]
    p = Problem(lens, 8, 2, 64, kind=kind, cache=cache, pt=pt, scale=1.0, seed=31)
    rng = np.random.default_rng(32)
    q = torch.zeros_like(p.q)
    q[:, :, 0] = torch.tensor([10.0, 14.0, 15.5, 16.5, 17.0, 17.5, 18.0, 20.0]).to(q.dtype)
    p.q = q
    p.d["q"].copy_(q)
    keys, values = [], []
    for n in lens:
        k, v = torch.zeros(n, 2, 64), torch.from_numpy(rng.uniform(100, 400, (n, 2, 64)).astype(np.float32)) * (1 if cache == "f8" else 16)
        k[:, :, 0] = -1.0
        for t in range(0, n, 32):
            at = t + int(rng.integers(0, min(32, n - t)))
            k[at], v[at] = 0.0, 0.0
        keys.append(k)
        values.append(v)
    put(p, 0, keys)
    put(p, 1, values)
    for s, d in zip(p.scales, p.d["scales"]):
        if s is not None:
            s.copy_(torch.tensor([1.0, 1.0]))
            d.copy_(s)
    out, lse, status = p.run()
    assert status == 0
    o, l, _ = p.want()
    u = ROUND[kind]
    seen = o != 0
    err = ((out.double() - o).abs() - (2.0 ** -25 if kind == "f16" else 0))[seen] / o[seen]
    assert float(err.max()) <= 2 * u + 2.0 ** -13, float(err.max())
    assert bool(((lse.double() - l).abs() <= 3e-5).all())


@pytest.mark.parametrize("kind,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "f8")])
@pytest.mark.parametrize("group", [4, 32])
def test_weights_are_held_in_more_bits_than_the_type_has(kind, cache, group):
    """One token of 32 takes most of the weight and has the value 0, all others have one and the same score and the value 1, so
    a rounding of the weights would not average out.  Products are exact; 2^-15 is left to the weights, 2^-16 to factor,
    exponential and sums, and the result is rounded once."""
    lens = [33, 64, 300, 2111]
    p = Problem(lens, 2 * group, 2, 128, kind=kind, cache=cache, scale=1.0, seed=41)
    q = torch.zeros_like(p.q)
    q[:, :, 0] = torch.linspace(1.5, 7.5, 4 * 2 * group).view(4, -1).to(q.dtype)
    p.q = q
    p.d["q"].copy_(q)
    keys, values = [], []
    for n in lens:
        k, v = torch.zeros(n, 2, 128), torch.ones(n, 2, 128)
        k[:, :, 0] = -1.0
        k[5::32], v[5::32] = 0.0, 0.0
        keys.append(k)
        values.append(v)
    put(p, 0, keys)
    put(p, 1, values)
    for s, d in zip(p.scales, p.d["scales"]):
        if s is not None:
            s.copy_(torch.tensor([1.0, 1.0]))
            d.copy_(s)
    out, lse, status = p.run()
    assert status == 0
    o, l, _ = p.want()
    err = float(((out.double() - o).abs() / o).max())
    assert err <= ROUND[kind] + 2.0 ** -15 + 2.0 ** -16, err
    assert bool(((lse.double() - l).abs() <= 3e-5).all())


def counters(p):
    """Bytes of the workspace's counters: for each share and column, as many as there can be whatever the rows are (a column is 16 or
    32 query heads of a cache head, a workgroup may take two or four of them).  Parts lie behind them."""
    group = p.q.shape[1] // p.H
    two = p.pt >= 16 and (p.D <= 128 or p.cache == "f8") and -(-group // 32) * 2 == -(-group // 16)
    columns = p.H * -(-group // (32 if two else 16))
    together = 4 if columns % 4 == 0 else 2 if columns % 2 == 0 else 1
    return -(-max(columns, 512) * together * 4 // 256) * 256


@pytest.mark.parametrize("Hq,H,D,cache", [(8, 2, 64, "bf16"), (16, 4, 128, "f8"), (5, 1, 256, "bf16"), (32, 1, 128, "bf16"), (100, 2, 64, "f8"),
                                          (12, 12, 64, "bf16")])
def test_all_counters_are_left_at_zero(Hq, H, D, cache):
    """After every call over a shared workspace, whatever rows were in parts; parts were written where they are expected."""
    rng = np.random.default_rng(51)
    ragged = [int(x) for x in rng.integers(0, 700, 60)] + [2800, 1900]
    problems = [Problem(lens, Hq, H, D, cache=cache, row_pages=pages) for lens in ([4000], [1, 700, 2300, 31], ragged, [9] * 40)
                for pages in (256, WIDE)]
    ws = torch.zeros(max(fdd.fdy_paged_attention_workspace_bytes(p.desc()) for p in problems), dtype=torch.uint8, device=DEV)
    n = counters(problems[0])
    for i in [0, 1, 2, 3, 4, 5, 6, 7, 4, 0, 6, 5, 1, 2]:
        p = problems[i]
        p.ws = ws
        ws[n:] = 0
        out, lse, _ = p.run()
        assert p.ws is ws and bool((ws[:n] == 0).all()), i
        if i < 2:
            assert bool((ws[n:] != 0).any()), i
        near((out, lse), p.want(), p.kind)
