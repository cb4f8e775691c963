"""What the operators of drafted tokens and chosen pages refuse, and their host-side sizes (no GPU call is made before these return)."""
import ctypes as C

import pytest

from paper_2604_06664_amd import FDY_ERR_INVALID_ARG, FDY_ERR_WORKSPACE, FDY_OK
from paper_2604_06664_amd import decode as fdd

A = 0x10000  # an address that is aligned and never touched


def changed(desc, **kw):
    d = type(desc).from_buffer_copy(desc)
    for name, value in kw.items():
        setattr(d, name, value)
    return d


def kv(**kw):
    f = dict(type=fdd.FDY_BF16, n_pages=4, page_tokens=16, n_heads=2, head_dim=64, page_stride=16 * 128, token_stride=128,
             head_stride=64)
    f.update(kw)
    return fdd.make_kv(f.pop("k", A), f.pop("v", A), **f)


def draft(**kw):
    d = fdd.fdy_draft(q=A, out=A, lse=A, table=A, lens=A, rows=None, first=A, sees=A, q_token=256, q_head=64, out_token=256, out_head=64,
                      kv=kv(), scale=0.125, window=0, n_seqs=3, n_q_heads=4, n_rows=3, row_pages=5, n_tokens=20, max_draft=8,
                      sees_words=1, type=fdd.FDY_BF16)
    return changed(d, **kw)


def bounds(**kw):
    return changed(fdd.fdy_bounds(bounds=A, table=A, lens=A, rows=None, fresh=A, kv=kv(), n_seqs=3, n_rows=3, row_pages=5, max_fresh=4), **kw)


def select(**kw):
    d = fdd.fdy_select(q=A, bounds=A, table=A, lens=A, rows=None, pages=A, seen=A, q_seq=256, q_head=64, kv=kv(), n_seqs=3, n_q_heads=4,
                       n_rows=3, row_pages=50, budget=6, sinks=1, recent=2, type=fdd.FDY_BF16)
    return changed(d, **kw)


def attend(**kw):
    d = fdd.fdy_attend(q=A, out=A, lse=A, table=A, lens=A, rows=None, q_seq=256, q_head=64, out_seq=256, out_head=64, kv=kv(),
                       scale=0.125, window=0, n_seqs=3, n_q_heads=4, n_rows=3, row_pages=5, type=fdd.FDY_BF16)
    return changed(d, **kw)


BAD_KV = [dict(type=3), dict(page_tokens=0), dict(page_tokens=24), dict(page_tokens=1 << 17), dict(n_heads=0), dict(head_dim=0),
          dict(head_dim=264), dict(n_pages=0), dict(n_pages=1 << 31)]
BAD_STRIDES = [dict(token_stride=1 << 31), dict(head_stride=1 << 40), dict(token_stride=(1 << 31) - 1), dict(page_stride=1 << 41)]
BIG = 1 << 50


def test_sizes_of_the_structs():
    assert [C.sizeof(s) for s in (fdd.fdy_draft, fdd.fdy_bounds, fdd.fdy_select, fdd.fdy_token)] == [216, 136, 184, 24]


def refused(call, d, *more):
    return call(d, *more, stream=0, check=False)


@pytest.mark.parametrize("kw", [dict(kv=kv(**k)) for k in BAD_KV + BAD_STRIDES + [dict(type=fdd.FDY_F16), dict(head_dim=60)]] + [
    dict(kv=kv(type=fdd.FDY_F8, head_dim=72)), dict(type=2), dict(n_seqs=65537), dict(n_q_heads=0), dict(n_q_heads=5),
    dict(n_q_heads=65538), dict(n_tokens=(1 << 23) + 1), dict(n_tokens=1 << 23, n_q_heads=16), dict(max_draft=0), dict(max_draft=1025),
    dict(sees_words=0), dict(max_draft=65), dict(sees_words=65), dict(sees=None), dict(first=None), dict(row_pages=1 << 27),
    dict(row_pages=1 << 20, n_seqs=65536)])
def test_tree_refuses_sizes(kw):
    d = draft(**kw)
    assert fdd.fdy_tree_attention_workspace_bytes(d) == 0
    assert refused(fdd.fdy_tree_attention, d, A, BIG) == FDY_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(q=None), dict(q=A + 8), dict(out=None), dict(out=A + 2), dict(lse=A + 1), dict(table=None),
                                dict(lens=None), dict(lens=A + 2), dict(rows=A + 1), dict(first=A + 2), dict(sees=A + 4), dict(kv=kv(k=None)),
                                dict(kv=kv(v=A + 8)), dict(q_head=60), dict(out_token=4), dict(kv=kv(token_stride=132)),
                                dict(kv=kv(k_scale=A + 2)), dict(kv=kv(type=fdd.FDY_F8, token_stride=136))])
def test_tree_refuses_pointers_and_strides(kw):
    assert refused(fdd.fdy_tree_attention, draft(**kw), A, BIG) == FDY_ERR_INVALID_ARG


def test_tree_workspace():
    d = draft()
    n = fdd.fdy_tree_attention_workspace_bytes(d)
    assert 0 < n < 256 << 20 and n % 256 == 0
    for ws, size in ((None, n), (A + 128, n), (A, n - 1)):
        assert refused(fdd.fdy_tree_attention, d, ws, size) == FDY_ERR_WORKSPACE
    for other in (draft(n_seqs=300, n_rows=300, n_tokens=4000), draft(max_draft=512, sees_words=8, n_tokens=1500), draft(row_pages=4000)):
        assert fdd.fdy_tree_attention_workspace_bytes(other) <= n  # one for all with these heads
    assert fdd.fdy_tree_attention(draft(n_seqs=0, q=None), None, 0, stream=0) == FDY_OK
    assert fdd.fdy_tree_attention(draft(n_tokens=0, q=None), None, 0, stream=0) == FDY_OK
    assert refused(fdd.fdy_tree_attention, None, A, n) == FDY_ERR_INVALID_ARG
    assert fdd.fdy_tree_attention_workspace_bytes(None) == 0


@pytest.mark.parametrize("kw", [dict(kv=kv(**k)) for k in BAD_KV + BAD_STRIDES + [
    dict(head_dim=60), dict(k=None), dict(k=A + 8), dict(token_stride=132), dict(type=fdd.FDY_F8, head_dim=72)]] + [
    dict(n_seqs=65537), dict(row_pages=1 << 27), dict(bounds=None), dict(bounds=A + 8), dict(table=None), dict(table=A + 2), dict(lens=None),
    dict(lens=A + 2), dict(rows=A + 2), dict(fresh=A + 1)])
def test_bounds_refuse(kw):
    assert refused(fdd.fdy_page_bounds, bounds(**kw)) == FDY_ERR_INVALID_ARG
    assert refused(fdd.fdy_page_bounds, None) == FDY_ERR_INVALID_ARG
    assert fdd.fdy_page_bounds(bounds(n_seqs=0, bounds=None), stream=0) == FDY_OK


@pytest.mark.parametrize("kw", [dict(kv=kv(**k)) for k in BAD_KV + [dict(type=fdd.FDY_F16), dict(head_dim=60)]] + [
    dict(kv=kv(type=fdd.FDY_F8, head_dim=72)), dict(type=2), dict(n_seqs=65537), dict(n_q_heads=0), dict(n_q_heads=5), dict(n_q_heads=65538),
    dict(n_seqs=65536, n_q_heads=66), dict(row_pages=1 << 27), dict(recent=0), dict(sinks=5), dict(budget=(1 << 25) + 1),
    dict(sinks=0xFFFFFFFF), dict(n_seqs=65536, row_pages=40000, n_q_heads=2)])
def test_choice_refuses_sizes(kw):
    d = select(**kw)
    assert fdd.fdy_page_select_workspace_bytes(d) == 0
    assert refused(fdd.fdy_page_select, d, A, BIG) == FDY_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(q=None), dict(q=A + 8), dict(bounds=None), dict(bounds=A + 8), dict(table=None), dict(lens=None),
                                dict(lens=A + 2), dict(rows=A + 1), dict(pages=None), dict(pages=A + 2), dict(seen=None), dict(seen=A + 1),
                                dict(q_head=60), dict(kv=kv(k_scale=A + 2))])
def test_choice_refuses_pointers(kw):
    assert refused(fdd.fdy_page_select, select(**kw), A, BIG) == FDY_ERR_INVALID_ARG


def test_choice_workspace():
    d = select(kv=kv(k=None, v=None, token_stride=1 << 40))  # pools and strides are not looked at
    n = fdd.fdy_page_select_workspace_bytes(d)
    assert n >= 3 * 2 * 50 * 8 and n % 256 == 0
    for ws, size in ((None, n), (A + 128, n), (A, n - 1)):
        assert refused(fdd.fdy_page_select, d, ws, size) == FDY_ERR_WORKSPACE
    assert fdd.fdy_page_select(select(n_seqs=0, q=None), None, 0, stream=0) == FDY_OK
    assert fdd.fdy_page_select_workspace_bytes(None) == 0


@pytest.mark.parametrize("kw", [dict(kv=kv(**k)) for k in BAD_KV + BAD_STRIDES] + [dict(type=2), dict(reserved=1), dict(n_q_heads=5),
                                                                                  dict(n_rows=1 << 30), dict(row_pages=1 << 27)])
def test_attention_over_lists_refuses_sizes(kw):
    d = attend(**kw)
    assert fdd.fdy_selected_attention_workspace_bytes(d) == 0
    assert refused(fdd.fdy_selected_attention, d, A, BIG) == FDY_ERR_INVALID_ARG


def test_attention_over_lists_refuses_pointers_and_workspaces():
    for kw in (dict(q=None), dict(out=A + 2), dict(table=None), dict(lens=None), dict(kv=kv(k=None)), dict(q_head=60)):
        assert refused(fdd.fdy_selected_attention, attend(**kw), A, BIG) == FDY_ERR_INVALID_ARG
    n = fdd.fdy_selected_attention_workspace_bytes(attend())
    for ws, size in ((None, n), (A + 128, n), (A, n - 1)):
        assert refused(fdd.fdy_selected_attention, attend(), ws, size) == FDY_ERR_WORKSPACE
    assert fdd.fdy_selected_attention(attend(n_seqs=0, q=None), A, n, stream=0) == FDY_OK


def pages(**kw):
    d = fdd.fdy_pages(refs=A, free_bits=A, table=A, lens=A, planes=A, page_bytes=4096, page_stride=4096, n_pages=100,
                      page_tokens=16, n_rows=8, row_pages=10, n_planes=4)
    return changed(d, **kw)


def keep(d, t, rows=A, drafts=A, lists=A, kept=A, n=3, most=4, ws=A, size=BIG):
    return fdd.fdy_pages_keep(d, t, rows, drafts, lists, kept, n, most, ws, size, A, stream=0, check=False)


def test_keep_refuses():
    ok = fdd.make_token(token_stride=256, piece_bytes=128, pieces=2, piece_stride=128)
    for kw in (dict(reserved=1), dict(n_pages=0), dict(page_tokens=48), dict(refs=None), dict(lens=A + 1), dict(planes=None), dict(page_bytes=24)):
        assert keep(pages(**kw), ok) == FDY_ERR_INVALID_ARG
    for kw in (dict(token_stride=24), dict(piece_stride=8), dict(piece_bytes=8), dict(piece_bytes=0), dict(pieces=0), dict(pieces=3),
               dict(token_stride=272), dict(token_stride=1 << 62), dict(piece_stride=1 << 40), dict(piece_stride=0, pieces=1 << 31),
               dict(piece_bytes=0xFFFFFFF0)):
        assert keep(pages(), changed(ok, **kw)) == FDY_ERR_INVALID_ARG, kw
    for kw in (dict(rows=None), dict(drafts=None), dict(lists=None), dict(kept=None), dict(rows=A + 2), dict(drafts=A + 1), dict(lists=A + 2),
               dict(kept=A + 3), dict(n=65537), dict(most=(1 << 20) + 1), dict(n=65536, most=1 << 16)):
        assert keep(pages(), ok, **kw) == FDY_ERR_INVALID_ARG, kw
    assert keep(None, ok) == FDY_ERR_INVALID_ARG and keep(pages(), None) == FDY_ERR_INVALID_ARG
    n = fdd.fdy_pages_workspace_bytes(pages(), 3)
    for ws, size in ((None, n), (A + 128, n), (A, n - 1)):
        assert keep(pages(), ok, ws=ws, size=size) == FDY_ERR_WORKSPACE
    assert keep(pages(), ok, n=0, rows=None, drafts=None, ws=None) == FDY_OK


def test_helpers_refuse_tensors():
    import torch

    c = kv(k=None, v=None)
    q, table, lens = torch.zeros(20, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 5, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    args = dict(q=q, out=q, table=table, lens=lens, kv=c, scale=1.0, max_draft=8, first=torch.zeros(4, dtype=torch.int32),
                sees=torch.zeros(20, 1, dtype=torch.int64))
    d = fdd.make_draft_desc(**args)
    assert (d.n_seqs, d.n_tokens, d.sees_words, d.row_pages) == (3, 20, 1, 5)
    assert fdd.make_draft_desc(**{**args, "first": None, "sees": None, "max_draft": 6}).n_seqs == 3
    for bad in (dict(lens=lens.long()), dict(first=lens.long()), dict(sees=torch.zeros(19, 1, dtype=torch.int64)), dict(q=q[:, :, :60]),
                dict(sees=torch.zeros(20, 1, dtype=torch.int32)), dict(out=q.half()), dict(rows=torch.zeros(2, dtype=torch.int32)),
                dict(lse=torch.zeros(20, 3)), dict(table=table.t())):
        with pytest.raises(ValueError):
            fdd.make_draft_desc(**{**args, **bad})
    b = torch.zeros(4, 2, 2, 64, dtype=torch.bfloat16)
    assert fdd.make_bounds_desc(bounds=b, table=table, lens=lens, kv=c, rows=lens[:2]).n_seqs == 2
    for bad in (dict(bounds=b.half()), dict(bounds=b[:3]), dict(fresh=lens[:2]), dict(lens=lens.long())):
        with pytest.raises(ValueError):
            fdd.make_bounds_desc(**{**dict(bounds=b, table=table, lens=lens, kv=c), **bad})
    args = dict(q=q[:3], bounds=b, table=table, lens=lens, kv=c, pages=torch.zeros(3, 2, 7, dtype=torch.int32), seen=lens)
    assert fdd.make_select_desc(**args).budget == 7
    for bad in (dict(pages=torch.zeros(3, 1, 7, dtype=torch.int32)), dict(pages=torch.zeros(3, 2, 7)), dict(seen=lens[:2]), dict(bounds=b.float())):
        with pytest.raises(ValueError):
            fdd.make_select_desc(**{**args, **bad})
    args = dict(q=q[:3], out=q[:3], table=torch.zeros(3, 2, 7, dtype=torch.int32), lens=lens, kv=c, scale=1.0)
    assert fdd.make_selected_desc(**args).row_pages == 7
    for bad in (dict(table=torch.zeros(3, 1, 7, dtype=torch.int32)), dict(out=q), dict(lens=lens[:2])):
        with pytest.raises(ValueError):
            fdd.make_selected_desc(**{**args, **bad})
