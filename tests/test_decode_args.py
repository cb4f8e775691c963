"""What the decode operators refuse, and their host-side sizes (no GPU call is made before these return)."""
import ctypes as C

import pytest

from paper_2604_06664_amd import FDY_ERR_INVALID_ARG, FDY_ERR_WORKSPACE, FDY_OK
from paper_2604_06664_amd import decode as fdd

A = 0x10000  # an address that is aligned and never touched


def kv(**kw):
    f = dict(type=fdd.FDY_BF16, n_pages=4, page_tokens=16, n_heads=2, head_dim=64, page_stride=16 * 128, token_stride=128,
             head_stride=64)
    f.update(kw)
    return fdd.make_kv(f.pop("k", A), f.pop("v", A), **f)


def changed(desc, **kw):
    d = type(desc).from_buffer_copy(desc)
    for name, value in kw.items():
        setattr(d, name, value)
    return d


def append(**kw):
    d = fdd.fdy_append(q=A, k=A, v=A, q_out=A + 0x1000, k_out=None, positions=A, table=A, slots=A, q_token=256, q_head=64,
                       k_token=128, k_head=64, v_token=128, v_head=64, q_out_token=256, q_out_head=64, kv=kv(), n_tokens=3,
                       n_q_heads=4, n_positions=10, rot_dim=64, type=fdd.FDY_BF16, layout=fdd.FDY_ROPE_HALF)
    return changed(d, **kw)


BAD_KV = [dict(type=3), dict(page_tokens=0), dict(page_tokens=24), dict(page_tokens=1 << 17), dict(n_heads=0),
          dict(head_dim=0), dict(head_dim=264), dict(n_pages=0), dict(n_pages=1 << 31), dict(token_stride=1 << 31),
          dict(head_stride=1 << 40), dict(token_stride=(1 << 31) - 1), dict(page_stride=1 << 41)]


def attend(**kw):
    d = fdd.fdy_attend(q=A, out=A, lse=A, table=A, lens=A, rows=None, q_seq=256, q_head=64, out_seq=256, out_head=64, kv=kv(),
                       scale=0.125, window=0, n_seqs=3, n_q_heads=4, n_rows=3, row_pages=5, type=fdd.FDY_BF16)
    return changed(d, **kw)


def pages(**kw):
    d = fdd.fdy_pages(refs=A, free_bits=A, table=A, lens=A, planes=A, page_bytes=4096, page_stride=4096, n_pages=100,
                      page_tokens=16, n_rows=8, row_pages=10, n_planes=4)
    return changed(d, **kw)


def test_sizes_of_the_structs():
    assert [C.sizeof(s) for s in (fdd.fdy_kv, fdd.fdy_rope, fdd.fdy_append, fdd.fdy_attend, fdd.fdy_pages)] == [80, 56, 248, 192, 80]


@pytest.mark.parametrize("kw", BAD_KV + [dict(type=fdd.FDY_F16), dict(k=None), dict(v=None), dict(k=A + 1)])
def test_append_refuses_caches(kw):
    assert fdd.fdy_rope_append(append(kv=kv(**kw)), stream=0, check=False) == FDY_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [
    dict(type=fdd.FDY_F8), dict(type=7), dict(layout=2), dict(rot_dim=0), dict(rot_dim=63), dict(rot_dim=66), dict(k=None),
    dict(positions=None), dict(table=None), dict(table=A + 4), dict(positions=A + 2), dict(slots=A + 4), dict(v=None),
    dict(q_out=None), dict(n_q_heads=0), dict(n_q_heads=65537), dict(q=A + 1), dict(k_out=A + 1), dict(n_tokens=(1 << 23) + 1),
    dict(q_out=A, q_out_head=128), dict(k_out=A, k_out_token=64)])
def test_append_refuses(kw):
    assert fdd.fdy_rope_append(append(**kw), stream=0, check=False) == FDY_ERR_INVALID_ARG
    assert fdd.fdy_rope_append(None, stream=0, check=False) == FDY_ERR_INVALID_ARG


def test_append_of_nothing_is_fine():
    assert fdd.fdy_rope_append(append(n_tokens=0, k=None, positions=None), stream=0) == FDY_OK


def test_rope_refuses():
    ok = dict(rot_dim=64, base=1e4, scaling=fdd.FDY_ROPE_YARN, factor=4.0, low=1.0, high=32.0, trained_len=4096.0, magnitude=1.0)
    assert fdd.fdy_rope_frequencies(fdd.make_rope(**ok))[0] == FDY_OK
    nan, inf = float("nan"), float("inf")
    for kw in (dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=258), dict(scaling=5), dict(base=1.0), dict(base=nan), dict(base=inf),
               dict(factor=0.0), dict(factor=nan), dict(low=0.0), dict(high=1.0), dict(high=nan), dict(trained_len=0.0),
               dict(trained_len=inf), dict(magnitude=nan), dict(scaling=fdd.FDY_ROPE_NTK, rot_dim=2)):
        assert fdd.fdy_rope_frequencies(fdd.make_rope(**{**ok, **kw}), check=False)[0] == FDY_ERR_INVALID_ARG, kw
        assert fdd.fdy_rope_table(fdd.make_rope(**{**ok, **kw}), 0, 4, A, stream=0, check=False) == FDY_ERR_INVALID_ARG, kw
    rope = fdd.make_rope(64)
    assert fdd.fdy_rope_table(rope, 0, 4, None, stream=0, check=False) == FDY_ERR_INVALID_ARG
    assert fdd.fdy_rope_table(rope, 0, 4, A + 4, stream=0, check=False) == FDY_ERR_INVALID_ARG
    assert fdd.fdy_rope_table(rope, 1 << 31, 1, A, stream=0, check=False) == FDY_ERR_INVALID_ARG
    assert fdd.fdy_rope_table(rope, 1 << 31, 0, None, stream=0, check=False) == FDY_OK


@pytest.mark.parametrize("kw", [dict(kv=kv(**k)) for k in BAD_KV + [dict(type=fdd.FDY_F16), dict(head_dim=60)]] + [
    dict(kv=kv(type=fdd.FDY_F8, head_dim=72)), dict(type=2), dict(reserved=1), dict(n_seqs=65537), dict(n_q_heads=0),
    dict(n_q_heads=5), dict(n_q_heads=65538), dict(n_seqs=65536, n_q_heads=66), dict(row_pages=1 << 27)])
def test_attention_refuses_sizes(kw):
    d = attend(**kw)
    assert fdd.fdy_paged_attention_workspace_bytes(d) == 0
    assert fdd.fdy_paged_attention(d, A, 1 << 40, stream=0, check=False) == FDY_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(q=None), dict(q=A + 8), dict(out=None), dict(out=A + 2), dict(lse=A + 1), dict(table=None),
                                dict(lens=None), dict(lens=A + 2), dict(rows=A + 1), dict(kv=kv(k=None)), dict(kv=kv(v=A + 8)),
                                dict(q_head=60), dict(out_seq=4), dict(kv=kv(token_stride=132)), dict(kv=kv(k_scale=A + 2)),
                                dict(kv=kv(type=fdd.FDY_F8, token_stride=136))])
def test_attention_refuses_pointers_and_strides(kw):
    assert fdd.fdy_paged_attention(attend(**kw), A, 1 << 40, stream=0, check=False) == FDY_ERR_INVALID_ARG


def test_attention_workspace():
    d = attend()
    n = fdd.fdy_paged_attention_workspace_bytes(d)
    assert 0 < n < 32 << 20 and n % 256 == 0
    for ws, size in ((None, n), (A + 128, n), (A, n - 1)):
        assert fdd.fdy_paged_attention(d, ws, size, stream=0, check=False) == FDY_ERR_WORKSPACE
    last = n
    for seqs in (4, 100, 200, 1000, 65536 // 2):  # one made for more sequences serves fewer
        m = fdd.fdy_paged_attention_workspace_bytes(attend(n_seqs=seqs))
        assert m >= last
        last = m
    assert fdd.fdy_paged_attention(attend(n_seqs=0, q=None), None, 0, stream=0) == FDY_OK
    assert fdd.fdy_paged_attention(None, A, n, stream=0, check=False) == FDY_ERR_INVALID_ARG
    assert fdd.fdy_paged_attention_workspace_bytes(None) == 0


CONTENTS, WORKSPACE = ("extend", "copy", "compact"), ("extend", "fork", "compact")
ALL = ("reset", "extend", "fork", "free", "copy", "compact")


def page_calls(d, names, ws=A, size=1 << 50):
    """Return codes of the named calls.  Only calls that have to be refused are made: the addresses are none."""
    kw = dict(stream=0, check=False)
    calls = dict(reset=lambda: fdd.fdy_pages_reset(d, **kw),
                 extend=lambda: fdd.fdy_pages_extend(d, A, A, 3, A, A, 9, ws, size, A, **kw),
                 fork=lambda: fdd.fdy_pages_fork(d, A, A, 3, ws, size, A, **kw),
                 free=lambda: fdd.fdy_pages_free(d, A, 3, A, **kw),
                 copy=lambda: fdd.fdy_pages_copy(d, A, A, 3, A, **kw),
                 compact=lambda: fdd.fdy_pages_compact(d, A, A, ws, size, A, **kw))
    return {name: calls[name]() for name in names}


@pytest.mark.parametrize("kw", [dict(reserved=1), dict(n_pages=0), dict(n_pages=(1 << 28) + 1), dict(n_rows=(1 << 28) + 1),
                                dict(page_tokens=0), dict(page_tokens=48), dict(page_tokens=1 << 17), dict(row_pages=(1 << 25) + 1),
                                dict(row_pages=1 << 24, page_tokens=128), dict(page_bytes=24), dict(page_stride=8),
                                dict(page_bytes=1 << 30), dict(n_planes=32769)])
def test_pages_refuse_sizes(kw):
    d = pages(**kw)
    assert fdd.fdy_pages_workspace_bytes(d, 3) == 0
    assert set(page_calls(d, ALL).values()) == {FDY_ERR_INVALID_ARG}


def test_pages_refuse_pointers():
    for kw in (dict(refs=None), dict(refs=A + 2), dict(free_bits=None), dict(free_bits=A + 4), dict(lens=None), dict(lens=A + 1),
               dict(table=None), dict(table=A + 2)):
        assert set(page_calls(pages(**kw), [n for n in ALL if n != "copy"]).values()) == {FDY_ERR_INVALID_ARG}, kw
    for kw in (dict(planes=None), dict(planes=A + 4)):
        assert set(page_calls(pages(**kw), CONTENTS).values()) == {FDY_ERR_INVALID_ARG}, kw
    assert set(page_calls(None, ALL).values()) == {FDY_ERR_INVALID_ARG}
    d, k = pages(), dict(stream=0, check=False)
    for lists in ((A + 2, A, A, A), (A, A + 1, A, A), (A, A, A + 4, A), (A, A, A, A + 2)):
        assert fdd.fdy_pages_extend(d, lists[0], lists[1], 3, lists[2], lists[3], 9, A, 1 << 50, A, **k) == FDY_ERR_INVALID_ARG
    assert fdd.fdy_pages_extend(d, None, A, 9, A, A, 9, A, 1 << 50, A, **k) == FDY_ERR_INVALID_ARG  # more than there are rows
    assert fdd.fdy_pages_extend(d, A, A, 65537, A, A, 9, A, 1 << 50, A, **k) == FDY_ERR_INVALID_ARG
    assert fdd.fdy_pages_extend(d, A, A, 3, A, A, 1 << 31, A, 1 << 50, A, **k) == FDY_ERR_INVALID_ARG
    for a, b in ((None, A), (A, None), (A + 2, A), (A, A + 2)):
        assert fdd.fdy_pages_fork(d, a, b, 3, A, 1 << 50, A, **k) == FDY_ERR_INVALID_ARG
        assert fdd.fdy_pages_copy(d, a, b, 3, A, **k) == FDY_ERR_INVALID_ARG
    assert fdd.fdy_pages_free(d, None, 3, A, **k) == FDY_ERR_INVALID_ARG
    assert fdd.fdy_pages_free(d, A + 2, 3, A, **k) == FDY_ERR_INVALID_ARG
    assert fdd.fdy_pages_compact(d, A + 2, A, A, 1 << 50, A, **k) == FDY_ERR_INVALID_ARG
    assert fdd.fdy_pages_compact(d, A, A + 2, A, 1 << 50, A, **k) == FDY_ERR_INVALID_ARG


def test_pages_workspace():
    d = pages()
    n = fdd.fdy_pages_workspace_bytes(d, 3)
    assert n > 0 and n % 256 == 0 and fdd.fdy_pages_workspace_bytes(d, 65537) == 0 and fdd.fdy_pages_workspace_bytes(None, 1) == 0
    for ws, size in ((None, 1 << 40), (A + 128, 1 << 40), (A, 0)):
        assert set(page_calls(d, WORKSPACE, ws, size).values()) == {FDY_ERR_WORKSPACE}


def test_lists_of_nothing_are_fine():
    d, k = pages(), dict(stream=0, check=False)
    assert fdd.fdy_pages_extend(d, None, None, 0, None, None, 0, None, 0, None, **k) == FDY_OK
    assert fdd.fdy_pages_fork(d, None, None, 0, None, 0, None, **k) == FDY_OK
    assert fdd.fdy_pages_free(d, None, 0, None, **k) == FDY_OK
    assert fdd.fdy_pages_copy(d, None, None, 0, None, **k) == FDY_OK
    assert fdd.fdy_pages_copy(pages(n_planes=0), A, A, 3, None, **k) == FDY_OK


class Meta:
    """Tensors that own nothing, of a kind that each helper takes; a wrong one is refused."""

    @staticmethod
    def of(shape, dtype="float32"):
        torch = pytest.importorskip("torch")
        return torch.empty(shape, dtype=getattr(torch, dtype), device="meta")

    def append(self, **kw):
        x = lambda h: self.of((3, h, 64), "bfloat16")  # noqa: E731
        args = dict(q=x(4), k=x(2), v=x(2), q_out=x(4), k_out=x(2), positions=self.of(3, "int32"), table=self.of((9, 2, 16)),
                    slots=self.of(3, "int64"), kv=kv(n_heads=2, head_dim=64), rot_dim=32)
        return fdd.make_append_desc(**{**args, **kw})

    def attend(self, **kw):
        x = self.of((3, 4, 64), "bfloat16")
        args = dict(q=x, out=x, lse=self.of((3, 4)), table=self.of((5, 7), "int32"), lens=self.of(5, "int32"),
                    rows=self.of(3, "int32"), kv=kv(n_heads=2, head_dim=64), scale=1.0)
        return fdd.make_attend_desc(**{**args, **kw})

    def pages(self, **kw):
        args = dict(refs=self.of(70, "int32"), free_bits=self.of(2, "int64"), table=self.of((5, 7), "int32"),
                    lens=self.of(5, "int32"), page_tokens=16, planes=self.of(3, "int64"))
        return fdd.make_pages(**{**args, **kw})


@pytest.mark.parametrize("helper,wrong", [
    ("append", dict(q=((3, 4, 64), "float16"))), ("append", dict(q=((2, 4, 64), "bfloat16"))), ("append", dict(k=((3, 1, 64), "bfloat16"))),
    ("append", dict(v=((3, 2, 32), "bfloat16"))), ("append", dict(q_out=((3, 2, 64), "bfloat16"))), ("append", dict(k_out=((3, 128), "bfloat16"))),
    ("append", dict(positions=((3,), "int64"))), ("append", dict(positions=((4,), "int32"))), ("append", dict(slots=((3,), "int32"))),
    ("append", dict(table=((9, 2, 32), "float32"))), ("append", dict(table=((9, 2, 16), "float64"))),
    ("attend", dict(q=((3, 4, 32), "bfloat16"))), ("attend", dict(out=((3, 2, 64), "bfloat16"))), ("attend", dict(out=((3, 4, 64), "float32"))),
    ("attend", dict(table=((5, 7), "int64"))), ("attend", dict(lens=((5,), "int64"))), ("attend", dict(lens=((4,), "int32"))),
    ("attend", dict(rows=((5,), "int32"))), ("attend", dict(lse=((3, 4), "bfloat16"))), ("attend", dict(lse=((4, 3), "float32"))),
    ("pages", dict(refs=((70,), "int64"))), ("pages", dict(free_bits=((1,), "int64"))), ("pages", dict(free_bits=((2,), "int32"))),
    ("pages", dict(table=((5, 7), "int64"))), ("pages", dict(lens=((7,), "int32"))), ("pages", dict(planes=((3,), "int32")))])
def test_helpers_refuse_other_types_and_shapes(helper, wrong):
    make = getattr(Meta(), helper)
    make()
    with pytest.raises(ValueError):
        make(**{name: Meta.of(*x) for name, x in wrong.items()})


def test_helpers_refuse_other_orders():
    m = Meta()
    with pytest.raises(ValueError):
        m.attend(table=m.of((7, 5), "int32").t())
    with pytest.raises(ValueError):
        m.attend(q=m.of((3, 64, 4), "bfloat16").transpose(1, 2))
    with pytest.raises(ValueError):
        m.append(k=m.of((3, 64, 2), "bfloat16").transpose(1, 2))


def test_pages_refuse_more_pieces_than_32_bits_count():
    """32,768 planes of pages of 2^30 - 16 bytes are 2^32 pieces of 8 KiB: a count in 32 bits would be 0, and nothing copied."""
    d = pages(n_planes=32768, page_bytes=(1 << 30) - 16, page_stride=1 << 30)
    assert fdd.fdy_pages_workspace_bytes(d, 3) == 0
    assert set(page_calls(d, ALL).values()) == {FDY_ERR_INVALID_ARG}
    assert fdd.fdy_pages_workspace_bytes(pages(n_planes=32767, page_bytes=(1 << 30) - 16, page_stride=1 << 30), 3) > 0


CACHE = dict(type=fdd.FDY_BF16, n_pages=4, page_tokens=16, n_heads=2, head_dim=64, page_stride=2048, token_stride=128, head_stride=64)


@pytest.mark.parametrize("type_,dtype", [(fdd.FDY_BF16, "bfloat16"), (fdd.FDY_F16, "float16"), (fdd.FDY_F8, "float8_e4m3fn")])
def test_caches_of_tensors(type_, dtype):
    of, args = Meta.of, {**CACHE, "type": type_}
    scale = of(2) if type_ == fdd.FDY_F8 else None
    fdd.make_kv(of((4, 16, 2, 64), dtype), of((4, 16, 2, 64), dtype), k_scale=scale, v_scale=scale, **args)
    raw = of(4 * 2048 * (1 if type_ == fdd.FDY_F8 else 2), "uint8")  # storage without a type
    fdd.make_kv(raw, raw, **args)
    both = of((4, 2, 16, 2, 64), dtype)  # keys and values of a page side by side: the values' last page ends with the tensor
    fdd.make_kv(both[:, 0], both[:, 1], **{**args, "page_stride": 4096})
    with pytest.raises(ValueError):
        fdd.make_kv(both[:, 1], both[:, 1], **{**args, "page_stride": 4096 + 8})
    for other in {"bfloat16", "float16", "float8_e4m3fn", "float32"} - {dtype}:
        for pools in ((of((4, 16, 2, 64), other), of((4, 16, 2, 64), dtype)), (of((4, 16, 2, 64), dtype), of((4, 16, 2, 64), other))):
            with pytest.raises(ValueError):
                fdd.make_kv(*pools, **args)


@pytest.mark.parametrize("kw", [dict(n_pages=5), dict(n_pages=9999), dict(page_stride=2056), dict(token_stride=136), dict(head_dim=128),
                                dict(n_heads=3), dict(page_tokens=32)])
def test_caches_behind_the_end_of_their_tensors_are_refused(kw):
    good, short = Meta.of((5, 32, 3, 128), "bfloat16"), Meta.of((4, 16, 2, 64), "bfloat16")
    args = {**CACHE, **kw}
    for pools in ((good, short), (short, good)):
        with pytest.raises(ValueError):
            fdd.make_kv(*[p if p is short else None for p in pools], **args)
    fdd.make_kv(A, A, **args)  # addresses are the caller's word


@pytest.mark.parametrize("shape,dtype", [((1,), "float32"), ((), "float32"), ((3,), "float32"), ((2,), "float64"), ((2,), "bfloat16"),
                                         ((2, 1), "float32")])
def test_scales_of_other_types_and_shapes_are_refused(shape, dtype):
    pool, scale = Meta.of((4, 16, 2, 64), "float8_e4m3fn"), Meta.of(2)
    args = {**CACHE, "type": fdd.FDY_F8}
    fdd.make_kv(pool, pool, k_scale=scale, v_scale=scale, **args)
    for kw in (dict(k_scale=Meta.of(shape, dtype), v_scale=scale), dict(k_scale=scale, v_scale=Meta.of(shape, dtype)),
               dict(k_scale=Meta.of((2, 2))[:, 0], v_scale=scale)):
        with pytest.raises(ValueError):
            fdd.make_kv(pool, pool, **kw, **args)


BAD_LISTS = [((3,), "int64"), ((3,), "float32"), ((2,), "int32"), ((0,), "int32"), ((3, 2), "int32")]  # the last: every second element


@pytest.mark.parametrize("shape,dtype", BAD_LISTS)
def test_lists_of_other_types_and_lengths_are_refused(shape, dtype):
    """Three entries are asked for; nothing is launched."""
    of, d, k = Meta.of, pages(), dict(stream=0, check=False)
    bad = of(shape, dtype)[:, 0] if len(shape) == 2 else of(shape, dtype)
    for args in ((bad, A, A, A), (A, bad, A, A), (A, A, A, bad)):
        with pytest.raises(ValueError):
            fdd.fdy_pages_extend(d, args[0], args[1], 3, args[2], args[3], 3, A, 1 << 50, A, **k)
    for args in ((bad, A), (A, bad)):
        with pytest.raises(ValueError):
            fdd.fdy_pages_fork(d, *args, 3, A, 1 << 50, A, **k)
        with pytest.raises(ValueError):
            fdd.fdy_pages_copy(d, *args, 3, A, **k)
    with pytest.raises(ValueError):
        fdd.fdy_pages_free(d, bad, 3, A, **k)
    with pytest.raises(ValueError):
        fdd.fdy_pages_compact(pages(n_pages=3), bad, A, A, 1 << 50, A, **k)


def test_other_arrays_of_calls_are_refused():
    of, d, k = Meta.of, pages(), dict(stream=0, check=False)
    for slots in (of(9, "int32"), of(8, "int64"), of((9, 2), "int64")[:, 0]):
        with pytest.raises(ValueError):
            fdd.fdy_pages_extend(d, A, A, 3, slots, A, 9, A, 1 << 50, A, **k)
    for n_live in (of(1, "int64"), of(0, "int32")):
        with pytest.raises(ValueError):
            fdd.fdy_pages_compact(d, A, n_live, A, 1 << 50, A, **k)
    for table in (of((4, 2, 32), "float64"), of((4, 2, 32), "bfloat16"), of((3, 2, 32)), of((4, 2, 64))[:, :, :32]):
        with pytest.raises(ValueError):
            fdd.fdy_rope_table(fdd.make_rope(64), 0, 4, table, **k)
