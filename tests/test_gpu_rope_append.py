"""fdy_rope_append and fdy_rope_table through the C ABI against their definitions in 64 bits.

Tolerances.  A result is worked out in 32 bits (at most three roundings of terms as large as |x cos| + |y sin|, one more
for the scale of an 8-bit cache and its reciprocal: 2^-22 of them is allowed) and rounded once to the type it is stored in:
half a unit in the last place, 2^-8 of the value for bf16, 2^-11 for f16, 2^-4 for e4m3, or half the smallest step."""
import numpy as np
import pytest
import torch

import oracle.decode as od
from paper_2604_06664_amd import decode as fdd

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = dict(bf16=torch.bfloat16, f16=torch.float16, f8=torch.float8_e4m3fn)
ROUND = dict(bf16=(2.0 ** -8, 2.0 ** -134), f16=(2.0 ** -11, 2.0 ** -25), f8=(2.0 ** -4, 2.0 ** -10))


def close(got, want, size, kind):
    rel, least = ROUND[kind]
    err = (got.double() - want).abs()
    bound = rel * want.abs() + least + 2.0 ** -22 * size
    bad = ~(err <= bound)
    assert not bool(bad.any()), (kind, int(bad.sum()), float((err - bound).max()))


def pool(rng, order, n_pages, pt, H, D, kind):
    shape = (n_pages, pt, H, D) if order == "token" else (n_pages, H, pt, D)
    p = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(DTYPES[kind]).to(DEV)
    return p, (p if order == "token" else p.transpose(1, 2))


def table_of(rot, n):
    return torch.from_numpy(od.rope_table(od.rope_frequencies(rot), 0, n).astype(np.float32)).to(DEV)


def one(T, Hq, H, D, rot, layout, kind, cache, pt=16, order="token", pad=0, at=0, seed=1, inplace=False, k_out=False,
        scaled=True, bad=True):
    rng = np.random.default_rng(seed)
    n_pos, n_pages = 50, -(-(T + 3) // pt) + 2
    ts = (Hq + 2 * H) * (D + pad) + at  # strides: heads and tokens apart, first element off by `at`
    flat = torch.from_numpy(rng.standard_normal(T * ts + at + 8).astype(np.float32) * 2).to(DTYPES[kind]).to(DEV)
    whole = torch.as_strided(flat, (T, Hq + 2 * H, D), (ts, D + pad, 1), at)
    q, k, v = whole[:, :Hq], whole[:, Hq:Hq + H], whole[:, Hq + H:]
    before = [x.clone().cpu().double() for x in (q, k, v)]
    qo = q if inplace else torch.full((T, Hq, D), 7.0, dtype=q.dtype, device=DEV)
    ko = (k if inplace else torch.full((T, H, D), 7.0, dtype=q.dtype, device=DEV)) if k_out else None
    pos = rng.integers(0, n_pos, T).astype(np.int32)
    slots = rng.permutation(n_pages * pt)[:T].astype(np.int64)
    want_status = 0
    if bad and T > 4:
        slots[1] = -1
        slots[2] = n_pages * pt + 5
        pos[3] = n_pos
        want_status = od.ST_BAD_INDEX
    (kp, kv_), (vp, vv) = (pool(rng, order, n_pages, pt, H, D, cache) for _ in "kv")
    kept = [x.clone() for x in (kp, vp)]
    scales = [torch.from_numpy(rng.uniform(0.01, 0.5, H).astype(np.float32)).to(DEV) if cache == "f8" and scaled else None
              for _ in "kv"]
    st = kv_.stride()
    kv = fdd.make_kv(kp, vp, type=fdd.TYPES[cache], n_pages=n_pages, page_tokens=pt, n_heads=H, head_dim=D,
                     page_stride=st[0], token_stride=st[1], head_stride=st[2], k_scale=scales[0], v_scale=scales[1])
    table = table_of(rot, n_pos)
    d_pos, d_slots = torch.from_numpy(pos).to(DEV), torch.from_numpy(slots).to(DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    desc = fdd.make_append_desc(q=q, k=k, v=v, q_out=qo, k_out=ko, positions=d_pos, table=table, slots=d_slots, kv=kv,
                                rot_dim=rot, layout=fdd.LAYOUTS[layout])
    fdd.fdy_rope_append(desc, status)
    torch.cuda.synchronize()
    assert int(status) == want_status
    host = table.cpu()
    got_q, got_k = qo.cpu(), None if ko is None else ko.cpu()
    got = [kv_.cpu(), vv.cpu()]
    want = [x.cpu().clone() if order == "token" else x.cpu().transpose(1, 2).clone() for x in kept]
    bits = torch.uint8 if cache == "f8" else torch.int16
    for t in range(T):
        if not 0 <= pos[t] < n_pos:
            if not inplace:
                assert bool((got_q[t] == 7).all())
            continue
        y, size = od.turned(before[0][t], host[pos[t]], rot, layout)
        close(got_q[t], y, size, kind)
        y, size = od.turned(before[1][t], host[pos[t]], rot, layout)
        if got_k is not None:
            close(got_k[t], y, size, kind)
        s = int(slots[t])
        if not 0 <= s < n_pages * pt:
            continue
        for side, (val, sz) in enumerate(((y, size), (before[2][t], before[2][t].abs()))):
            if scales[side] is not None:
                f = scales[side].cpu().double()[:, None]
                val, sz = val / f, sz / f
            if cache == "f8":
                val = val.clamp(-od.F8_MOST, od.F8_MOST)
            close(got[side][s // pt, s % pt], val, sz, cache)
            want[side].view(bits)[s // pt, s % pt] = got[side].view(bits)[s // pt, s % pt]  # looked at; the rest is as it was
    for a, b in zip(got, want):
        assert torch.equal(a.contiguous().view(bits), b.contiguous().view(bits))


@pytest.mark.parametrize("kind,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "f8"), ("f16", "f8")])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,Hq,H,D,rot", [
    (1, 32, 8, 128, 128), (7, 8, 2, 64, 64), (5, 3, 3, 96, 32), (9, 28, 4, 80, 80), (6, 2, 1, 256, 64), (5, 5, 1, 192, 192),
    (8, 4, 4, 24, 16), (6, 1, 1, 16, 16), (300, 4, 2, 128, 64), (5, 70, 1, 8, 8), (5, 2, 2, 40, 16),
    (5, 3, 1, 80, 40), (5, 2, 2, 7, 6), (5, 2, 1, 33, 2), (5, 2, 2, 255, 254), (6, 3, 2, 100, 50)])
def test_sizes(T, Hq, H, D, rot, layout, kind, cache):
    one(T, Hq, H, D, rot, layout, kind, cache)


@pytest.mark.parametrize("order", ["token", "head"])
@pytest.mark.parametrize("pt", [1, 2, 8, 64, 4096])
def test_page_sizes_and_orders(pt, order):
    one(37, 4, 2, 64, 64, "half", "bf16", "bf16", pt=pt, order=order)
    one(37, 4, 2, 64, 32, "interleaved", "f16", "f8", pt=pt, order=order, scaled=False)


@pytest.mark.parametrize("pad,at", [(8, 0), (8, 16), (1, 0), (0, 1), (4, 4)])
def test_strides_and_alignment(pad, at):
    for layout in ("half", "interleaved"):
        one(11, 5, 3, 64, 32, layout, "bf16", "bf16", pad=pad, at=at, k_out=True)


@pytest.mark.parametrize("D,rot", [(128, 128), (64, 32), (33, 8)])
def test_in_place_and_dense_keys(D, rot):
    for layout in ("half", "interleaved"):
        one(9, 4, 2, D, rot, layout, "f16", "f16", inplace=True, k_out=True)
        one(9, 4, 2, D, rot, layout, "bf16", "f8", k_out=True)


def test_many_tokens_take_one_wave_each():
    one(5000, 2, 1, 64, 64, "half", "bf16", "bf16", pt=32)


def test_queries_or_cache_left_out():
    rng = np.random.default_rng(3)
    T, H, D = 5, 2, 64
    k = torch.from_numpy(rng.standard_normal((T, H, D)).astype(np.float32)).to(torch.bfloat16).to(DEV)
    ko = torch.empty_like(k)
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    table = table_of(D, 8)
    kv = fdd.make_kv(None, None, type=fdd.FDY_BF16, n_pages=1, page_tokens=16, n_heads=H, head_dim=D, page_stride=0,
                     token_stride=0, head_stride=0)
    desc = fdd.make_append_desc(q=None, k=k, v=None, q_out=None, k_out=ko, positions=pos, table=table, kv=kv, rot_dim=D)
    fdd.fdy_rope_append(desc)
    for t in range(T):
        y, size = od.turned(k[t].cpu().double(), table[t].cpu(), D, "half")
        close(ko[t].cpu(), y, size, "bf16")
    desc.n_tokens = 0
    fdd.fdy_rope_append(desc)  # nothing to do


def test_eight_bit_cache_saturates_and_keeps_nan():
    T, H, D = 1, 1, 64
    v = torch.zeros(T, H, D)
    v[0, 0, :6] = torch.tensor([1e4, -1e4, float("inf"), float("-inf"), float("nan"), 500.0])
    v = v.to(torch.bfloat16).to(DEV)
    for D_, rot in ((64, 16), (64, 2)):  # wide accesses, single elements
        kp, vp = (torch.zeros(1, 16, H, D_, device=DEV).to(torch.float8_e4m3fn) for _ in "kv")
        kv = fdd.make_kv(kp, vp, type=fdd.FDY_F8, n_pages=1, page_tokens=16, n_heads=H, head_dim=D_, page_stride=16 * D_,
                         token_stride=D_, head_stride=D_)
        desc = fdd.make_append_desc(q=None, k=v, v=v, q_out=None, positions=torch.zeros(1, dtype=torch.int32, device=DEV),
                                    table=table_of(rot, 4), kv=kv, rot_dim=rot, slots=torch.zeros(1, dtype=torch.int64, device=DEV))
        fdd.fdy_rope_append(desc)
        got = vp.float().cpu()[0, 0, 0, :6]
        assert got[:4].tolist() == [448.0, -448.0, 448.0, -448.0] and bool(torch.isnan(got[4])) and got[5] == 448.0


@pytest.mark.parametrize("scaling", ["plain", "linear", "ntk", "yarn", "bands"])
@pytest.mark.parametrize("rot,base,first,n", [(64, 10000.0, 0, 700), (128, 500000.0, 130000, 300), (10, 1e6, 0, 33), (4, 10000.0, 2**31 - 7, 7)])
def test_table(scaling, rot, base, first, n):
    """Angles in 64 bits: at position p an error of p f 2^-52 and of sine and cosine themselves, then one rounding to 32."""
    kw = dict(plain={}, linear=dict(factor=4.0), ntk=dict(factor=8.0), yarn=dict(factor=16.0, low=1.0, high=32.0, trained=8192.0),
              bands=dict(factor=8.0, low=1.0, high=4.0, trained=8192.0))[scaling]
    rope = fdd.make_rope(rot, base, getattr(fdd, "FDY_ROPE_" + scaling.upper()), factor=kw.get("factor", 1.0), low=kw.get("low", 1.0),
                         high=kw.get("high", 32.0), trained_len=kw.get("trained", 4096.0), magnitude=1.25)
    freqs = od.rope_frequencies(rot, base, scaling, **kw)
    _, got_f = fdd.fdy_rope_frequencies(rope)
    assert np.allclose(got_f, freqs, rtol=1e-13, atol=0)
    out = torch.full((n + 1, 2, rot // 2), 9.0, device=DEV)
    fdd.fdy_rope_table(rope, first, n, out)
    got = out.cpu().numpy()
    want = od.rope_table(got_f, first, n, 1.25)
    assert np.abs(got[:n] - want).max() <= 1.25 * (2.0 ** -24 + (first + n) * 2.0 ** -51 + 2.0 ** -50)
    assert (got[n] == 9.0).all()


def test_another_stream_and_replays():
    """A captured call on a stream of its own, replayed with new positions and slots in the same arrays."""
    rng = np.random.default_rng(5)
    T, Hq, H, D, pt, n_pages = 3, 4, 2, 64, 16, 4
    q, k, v = (torch.from_numpy(rng.standard_normal((T, h, D)).astype(np.float32)).to(torch.bfloat16).to(DEV) for h in (Hq, H, H))
    qo = torch.empty_like(q)
    kp, vp = (torch.zeros(n_pages, pt, H, D, dtype=torch.bfloat16, device=DEV) for _ in "kv")
    kv = fdd.make_kv(kp, vp, type=fdd.FDY_BF16, n_pages=n_pages, page_tokens=pt, n_heads=H, head_dim=D, page_stride=pt * H * D,
                     token_stride=H * D, head_stride=D)
    pos, slots = torch.zeros(T, dtype=torch.int32, device=DEV), torch.arange(T, dtype=torch.int64, device=DEV)
    table = table_of(D, 64)
    desc = fdd.make_append_desc(q=q, k=k, v=v, q_out=qo, positions=pos, table=table, kv=kv, rot_dim=D, slots=slots)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fdd.fdy_rope_append(desc)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fdd.fdy_rope_append(desc)
    for step in range(4):
        pos.copy_(torch.from_numpy(rng.integers(0, 64, T).astype(np.int32)))
        slots.copy_(torch.from_numpy(rng.permutation(n_pages * pt)[:T]))
        q.copy_(torch.from_numpy(rng.standard_normal((T, Hq, D)).astype(np.float32)))
        graph.replay()
        torch.cuda.synchronize()
        for t in range(T):
            y, size = od.turned(q[t].cpu().double(), table[int(pos[t])].cpu(), D, "half")
            close(qo[t].cpu(), y, size, "bf16")
            s = int(slots[t])
            assert torch.equal(vp[s // pt, s % pt], v[t])


@pytest.mark.parametrize("cache", ["bf16", "f8"])
def test_cache_offsets_behind_32_bits(cache):
    T, H, D, pt, stride = 3, 2, 64, 16, (1 << 32) + 4096  # elements from page 0 to page 1
    rng = np.random.default_rng(7)
    k, v = (torch.from_numpy(rng.standard_normal((T, H, D)).astype(np.float32)).to(torch.bfloat16).to(DEV) for _ in "kv")
    pools = [torch.empty(stride + pt * H * D, dtype=DTYPES[cache], device=DEV) for _ in "kv"]
    kv = fdd.make_kv(*pools, type=fdd.TYPES[cache], n_pages=2, page_tokens=pt, n_heads=H, head_dim=D, page_stride=stride,
                     token_stride=H * D, head_stride=D)
    place = [0, pt - 1, 5]
    slots = torch.tensor([pt + p for p in place], dtype=torch.int64, device=DEV)
    pos = torch.tensor([2, 7, 0], dtype=torch.int32, device=DEV)
    table = table_of(D, 8)
    fdd.fdy_rope_append(fdd.make_append_desc(q=None, k=k, v=v, q_out=None, positions=pos, table=table, kv=kv, rot_dim=D, slots=slots))
    got_k, got_v = (p[stride:].view(pt, H, D)[place].cpu() for p in pools)
    for t in range(T):
        y, size = od.turned(k[t].cpu().double(), table[int(pos[t])].cpu(), D, "half")
        close(got_k[t], y, size, cache)
        close(got_v[t], v[t].cpu().double(), v[t].cpu().double().abs(), cache)


def quotients_next_to_ties():
    """Scales, and elements for which x / scale and x * (1 / scale), in 32 bits, lie on two sides of a tie of e4m3 or on it."""
    out = []
    for m in range(1, 256):
        for t in (17, 19, 21, 23, 25, 27, 29, 31):
            s = np.float32(m) / np.float32(t)
            for f in (np.nextafter(s, np.float32(0)), s, np.nextafter(s, np.float32(1e9))):
                a, b = torch.tensor([m / f, np.float32(m) * (np.float32(1) / f)]).to(torch.float8_e4m3fn).float().tolist()
                if a != b:
                    out.append((m, float(f)))
    return out


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("rot", [16, 8, 2])
def test_eight_bit_elements_are_divided_by_their_scale(kind, rot):
    """What is stored is the quotient in 32 bits, rounded: to the bit, as it is worked out on the CPU.  At position 0 keys are not
    turned either.  Scales of the ends of the range, too."""
    pairs = quotients_next_to_ties()
    assert len(pairs) > 100
    scales = sorted({f for _, f in pairs})[:200] + [2.0 ** -130, 2.0 ** -140, 2.0 ** -61, 2.0 ** 61, 1e30, -0.3, 1e-20]
    H, D, T = len(scales), 64, 4
    x = torch.randint(-255, 256, (T, H, D), generator=torch.Generator().manual_seed(3)).float()
    x[..., :16] = torch.tensor([0.0, -0.0, 448.0, -448.0, 1e4, -1e4, 1e-6, 6e-5, float("inf"), float("-inf"), float("nan"), 1, 2, 3, 4, 5])
    for h, s in enumerate(scales):
        for j, (m, f) in enumerate([p for p in pairs if p[1] == s][:40]):
            x[0, h, 20 + j] = m
    x = x.to(DTYPES[kind])
    f = torch.tensor(scales)
    want = (x.float() / f[:, None]).clamp(-od.F8_MOST, od.F8_MOST).to(torch.float8_e4m3fn)
    d_f, pools = f.to(DEV), [torch.zeros(1, 16, H, D, dtype=torch.uint8, device=DEV) for _ in "kv"]
    kv = fdd.make_kv(*pools, type=fdd.FDY_F8, n_pages=1, page_tokens=16, n_heads=H, head_dim=D, page_stride=16 * H * D,
                     token_stride=H * D, head_stride=D, k_scale=d_f, v_scale=d_f)
    d = x.to(DEV)
    table = table_of(rot, 1)
    pos, slots = torch.zeros(T, dtype=torch.int32, device=DEV), torch.arange(T, device=DEV)
    fdd.fdy_rope_append(fdd.make_append_desc(q=None, k=d, v=d, q_out=None, positions=pos, table=table, kv=kv, rot_dim=rot, slots=slots))
    nan = torch.isnan(want.float())
    for name, pool, first in (("v", pools[1], 0), ("k", pools[0], 16)):  # (an infinite key times a sine of 0 is no number)
        got = pool[0, :T].cpu().view(torch.float8_e4m3fn)
        assert torch.equal(torch.isnan(got.float())[..., first:], nan[..., first:]), name
        a, b = (y.view(torch.uint8)[..., first:].clone() for y in (got, want))
        assert torch.equal(a[~nan[..., first:]], b[~nan[..., first:]]), (name, int((a != b).sum()))
