"""Binding of include/fdy_decode.h (operators of a decode step over a paged cache): same names, marshalling only.

The descriptors are made once by the make_* helpers from the tensors that they describe (shapes and strides are
taken from them; the caller keeps the tensors alive) and handed to every call."""
from __future__ import annotations

import ctypes as C

from . import FDY_ERR_INVALID_ARG, FDY_ERR_WORKSPACE, FDY_OK, FdyError, _check, _ptr, _stream, lib  # noqa: F401

FDY_BF16, FDY_F16, FDY_F8 = 0, 1, 2
FDY_ROPE_PLAIN, FDY_ROPE_LINEAR, FDY_ROPE_NTK, FDY_ROPE_YARN, FDY_ROPE_BANDS = range(5)
FDY_ROPE_HALF, FDY_ROPE_INTERLEAVED = 0, 1
FDY_DECODE_ARG_BYTES = 512

TYPES = dict(bf16=FDY_BF16, f16=FDY_F16, f8=FDY_F8)
LAYOUTS = dict(half=FDY_ROPE_HALF, interleaved=FDY_ROPE_INTERLEAVED)


def _struct(name, pointers=(), u64=(), middle=(), u32=()):
    fields = [(n, C.c_void_p) for n in pointers] + [(n, C.c_uint64) for n in u64] + list(middle)
    return type(name, (C.Structure,), dict(_fields_=fields + [(n, C.c_uint32) for n in u32]))


fdy_kv = _struct("fdy_kv", ("k", "v", "k_scale", "v_scale"), ("page_stride", "token_stride", "head_stride"), (),
                 ("type", "n_pages", "page_tokens", "n_heads", "head_dim", "reserved"))
fdy_append = _struct("fdy_append", ("q", "k", "v", "q_out", "k_out", "positions", "table", "slots"),
                     ("q_token", "q_head", "k_token", "k_head", "v_token", "v_head", "q_out_token", "q_out_head",
                      "k_out_token", "k_out_head"), [("kv", fdy_kv)],
                     ("n_tokens", "n_q_heads", "n_positions", "rot_dim", "type", "layout"))
fdy_attend = _struct("fdy_attend", ("q", "out", "lse", "table", "lens", "rows"), ("q_seq", "q_head", "out_seq", "out_head"),
                     [("kv", fdy_kv), ("scale", C.c_float)],
                     ("window", "n_seqs", "n_q_heads", "n_rows", "row_pages", "type", "reserved"))
fdy_draft = _struct("fdy_draft", ("q", "out", "lse", "table", "lens", "rows", "first", "sees"),
                    ("q_token", "q_head", "out_token", "out_head"), [("kv", fdy_kv), ("scale", C.c_float)],
                    ("window", "n_seqs", "n_q_heads", "n_rows", "row_pages", "n_tokens", "max_draft", "sees_words", "type"))
fdy_bounds = _struct("fdy_bounds", ("bounds", "table", "lens", "rows", "fresh"), (), [("kv", fdy_kv)],
                     ("n_seqs", "n_rows", "row_pages", "max_fresh"))
fdy_select = _struct("fdy_select", ("q", "bounds", "table", "lens", "rows", "pages", "seen"), ("q_seq", "q_head"), [("kv", fdy_kv)],
                     ("n_seqs", "n_q_heads", "n_rows", "row_pages", "budget", "sinks", "recent", "type"))
fdy_token = _struct("fdy_token", (), ("token_stride", "piece_stride"), (), ("piece_bytes", "pieces"))
fdy_pages = _struct("fdy_pages", ("refs", "free_bits", "table", "lens", "planes"), ("page_bytes", "page_stride"), (),
                    ("n_pages", "page_tokens", "n_rows", "row_pages", "n_planes", "reserved"))


class fdy_rope(C.Structure):
    _fields_ = [("scaling", C.c_uint32), ("rot_dim", C.c_uint32)] + [
        (n, C.c_double) for n in ("base", "factor", "low", "high", "trained_len", "magnitude")]


_lib = None


def _L():
    global _lib
    if _lib is None:
        L = lib()
        p, u, z, i = C.c_void_p, C.c_uint32, C.c_size_t, C.c_int
        for name, result, args in (
                ("fdy_rope_frequencies", i, [p, p]),
                ("fdy_rope_table", i, [p, C.c_uint64, u, p, p]),
                ("fdy_rope_append", i, [p, p, p]),
                ("fdy_paged_attention_workspace_bytes", z, [p]),
                ("fdy_paged_attention", i, [p, p, z, p, p]),
                ("fdy_tree_attention_workspace_bytes", z, [p]),
                ("fdy_tree_attention", i, [p, p, z, p, p]),
                ("fdy_page_bounds", i, [p, p, p]),
                ("fdy_page_select_workspace_bytes", z, [p]),
                ("fdy_page_select", i, [p, p, z, p, p]),
                ("fdy_selected_attention_workspace_bytes", z, [p]),
                ("fdy_selected_attention", i, [p, p, z, p, p]),
                ("fdy_pages_keep", i, [p, p, p, p, p, p, u, u, p, z, p, p]),
                ("fdy_pages_reset", i, [p, p]),
                ("fdy_pages_workspace_bytes", z, [p, u]),
                ("fdy_pages_extend", i, [p, p, p, u, p, p, u, p, z, p, p]),
                ("fdy_pages_fork", i, [p, p, p, u, p, z, p, p]),
                ("fdy_pages_free", i, [p, p, u, p, p]),
                ("fdy_pages_copy", i, [p, p, p, u, p, p]),
                ("fdy_pages_compact", i, [p, p, p, p, z, p, p])):
            f = getattr(L, name)
            f.restype, f.argtypes = result, args
        _lib = L
    return _lib


def _d(desc):
    return None if desc is None else C.addressof(desc)


# ---- descriptors ------------------------------------------------------------------------------
def type_of(tensor):
    """FDY_BF16 / FDY_F16 / FDY_F8 of a torch tensor."""
    return {"torch.bfloat16": FDY_BF16, "torch.float16": FDY_F16, "torch.float8_e4m3fn": FDY_F8}[str(tensor.dtype)]


def _want(name, x, types, shape):
    """The kernels know of an array only its address: a tensor of another type, shape or order is refused here."""
    if x is None or not hasattr(x, "is_contiguous"):  # a plain address is the caller's word
        return
    if str(x.dtype) not in [f"torch.{t}" for t in types] or tuple(x.shape) != tuple(shape) or not x.is_contiguous():
        raise ValueError(f"{name}: {types[0]} {list(shape)}, contiguous, is wanted, not {x.dtype} {list(x.shape)}")


_names = {}  # of dtypes, as "int32"


def _list(name, x, types, n):
    """Address of a tensor that a call reads or writes `n` elements of.  Made for every call: a captured step's books are enqueued in
    8 us, and each look at a tensor costs a tenth of one."""
    if x is None or x.__class__ is int or not hasattr(x, "is_contiguous"):
        return _ptr(x)
    kind = x.dtype
    if (_names.get(kind) or _names.setdefault(kind, str(kind).split(".")[-1])) not in types or x.numel() < n or not x.is_contiguous():
        raise ValueError(f"{name}: {types[0]}, contiguous, of {n} elements at least, is wanted, not {kind} {list(x.shape)}")
    return x.data_ptr()


def _heads(name, x, like, shape):
    if x.dtype != like.dtype or tuple(x.shape) != tuple(shape) or (x.shape[2] > 1 and x.stride(2) != 1):
        raise ValueError(f"{name}: {like.dtype} {list(shape)} with contiguous last dimension is wanted, not {x.dtype} {list(x.shape)}")


_KV_TYPES = {FDY_BF16: "torch.bfloat16", FDY_F16: "torch.float16", FDY_F8: "torch.float8_e4m3fn"}


def _pool(name, x, type, n_pages, page_tokens, n_heads, head_dim, page_stride, token_stride, head_stride):
    """A pool's elements are of the cache's type (or integers, as raw storage), and its last page ends within its storage."""
    if x is None or not hasattr(x, "untyped_storage"):
        return
    if (x.is_floating_point() or x.is_complex()) and str(x.dtype) != _KV_TYPES.get(type):
        raise ValueError(f"{name}: a pool of {_KV_TYPES.get(type, 'a known type')} is wanted, not {x.dtype}")
    last = ((n_pages - 1) * page_stride + (page_tokens - 1) * token_stride + (n_heads - 1) * head_stride + head_dim)
    there = x.untyped_storage().nbytes() - x.storage_offset() * x.element_size()
    if last * (1 if type == FDY_F8 else 2) > there:
        raise ValueError(f"{name}: {n_pages} pages with these strides end behind the tensor's {there} bytes")


def make_rope(rot_dim, base=10000.0, scaling=FDY_ROPE_PLAIN, factor=1.0, low=1.0, high=32.0, trained_len=4096.0,
              magnitude=1.0):
    return fdy_rope(scaling, rot_dim, base, factor, low, high, trained_len, magnitude)


def make_kv(k, v, *, type, n_pages, page_tokens, n_heads, head_dim, page_stride, token_stride, head_stride,
            k_scale=None, v_scale=None):
    """k, v: device pools (tensors or addresses) or None; strides in elements; scales float32 [n_heads]."""
    for name, x in (("k", k), ("v", v)):
        _pool(name, x, type, n_pages, page_tokens, n_heads, head_dim, page_stride, token_stride, head_stride)
    if type == FDY_F8:  # others have none that is read
        _want("k_scale", k_scale, ["float32"], (n_heads,))
        _want("v_scale", v_scale, ["float32"], (n_heads,))
    return fdy_kv(_ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale), page_stride, token_stride, head_stride, type, n_pages,
                  page_tokens, n_heads, head_dim, 0)


def make_append_desc(*, q, k, v, q_out, positions, table, kv, rot_dim, slots=None, k_out=None, layout=FDY_ROPE_HALF):
    """q, k, v, q_out, k_out: tensors [tokens, heads, dim] with contiguous last dimension; table [positions, 2, rot_dim / 2]."""
    d = fdy_append()
    n, keys = k.shape[0], (k.shape[0], kv.n_heads, kv.head_dim)
    queries = None if q is None else (n, q.shape[1], kv.head_dim)
    for name, x, shape in (("q", q, queries), ("k", k, keys), ("v", v, keys), ("q_out", q_out, queries), ("k_out", k_out, keys)):
        setattr(d, name, _ptr(x))
        if x is not None:
            _heads(name, x, k, shape or keys)
            setattr(d, name + "_token", x.stride(0))
            setattr(d, name + "_head", x.stride(1))
    _want("positions", positions, ["int32"], (n,))
    _want("table", table, ["float32"], (table.shape[0], 2, rot_dim // 2))
    _want("slots", slots, ["int64"], (n,))
    d.positions, d.table, d.slots = _ptr(positions), _ptr(table), _ptr(slots)
    d.kv, d.n_tokens, d.n_q_heads = kv, n, 0 if q is None else q.shape[1]
    d.n_positions, d.rot_dim, d.type, d.layout = table.shape[0], rot_dim, type_of(k), layout
    return d


def make_attend_desc(*, q, out, table, lens, kv, scale, lse=None, rows=None, window=0):
    """q, out: tensors [sequences, heads, dim] with contiguous last dimension; table [rows, pages] and lens, 32-bit."""
    for name, x in (("q", q), ("out", out)):
        _heads(name, x, q, (q.shape[0], q.shape[1], kv.head_dim))
    _want("table", table, ["int32"], table.shape[:2])
    _want("lens", lens, ["int32"], table.shape[:1])
    _want("rows", rows, ["int32"], q.shape[:1])
    _want("lse", lse, ["float32"], q.shape[:2])
    d = fdy_attend(_ptr(q), _ptr(out), _ptr(lse), _ptr(table), _ptr(lens), _ptr(rows), q.stride(0), q.stride(1),
                   out.stride(0), out.stride(1), kv, scale, window, q.shape[0], q.shape[1], table.shape[0],
                   table.shape[1], type_of(q), 0)
    return d


def make_draft_desc(*, q, out, table, lens, kv, scale, max_draft, first=None, sees=None, lse=None, rows=None, window=0):
    """q, out: tensors [tokens, heads, dim] with contiguous last dimension, the sequences' drafted tokens one after the other;
    first [sequences + 1] 32-bit (None: max_draft tokens each); sees [tokens, words] of 64 bits (None: chains)."""
    for name, x in (("q", q), ("out", out)):
        _heads(name, x, q, (q.shape[0], q.shape[1], kv.head_dim))
    n_seqs = first.shape[0] - 1 if first is not None else q.shape[0] // max(1, max_draft)
    _want("table", table, ["int32"], table.shape[:2])
    _want("lens", lens, ["int32"], table.shape[:1])
    _want("rows", rows, ["int32"], (n_seqs,))
    _want("first", first, ["int32"], (n_seqs + 1,))
    _want("sees", sees, ["int64", "uint64"], q.shape[:1] + (0 if sees is None else sees.shape[1],))
    _want("lse", lse, ["float32"], q.shape[:2])
    return fdy_draft(_ptr(q), _ptr(out), _ptr(lse), _ptr(table), _ptr(lens), _ptr(rows), _ptr(first), _ptr(sees), q.stride(0),
                     q.stride(1), out.stride(0), out.stride(1), kv, scale, window, n_seqs, q.shape[1], table.shape[0],
                     table.shape[1], q.shape[0], max_draft, 0 if sees is None else sees.shape[1], type_of(q))


def make_bounds_desc(*, bounds, table, lens, kv, fresh=None, rows=None, max_fresh=1):
    """bounds [pages, heads, 2, dim] of the cache's type; one sequence for each of rows, or for each row of the table."""
    n_seqs = (table if rows is None else rows).shape[0]
    _want("bounds", bounds, [_KV_TYPES[kv.type].split(".")[1], "uint8" if kv.type == FDY_F8 else "int16"],
          (kv.n_pages, kv.n_heads, 2, kv.head_dim))
    _want("table", table, ["int32"], table.shape[:2])
    _want("lens", lens, ["int32"], table.shape[:1])
    _want("rows", rows, ["int32"], (n_seqs,))
    _want("fresh", fresh, ["int32"], (n_seqs,))
    return fdy_bounds(_ptr(bounds), _ptr(table), _ptr(lens), _ptr(rows), _ptr(fresh), kv, n_seqs, table.shape[0], table.shape[1],
                      max_fresh)


def make_select_desc(*, q, bounds, table, lens, kv, pages, seen, sinks=1, recent=1, rows=None):
    """q [sequences, heads, dim] with contiguous last dimension; pages [sequences, cache heads, budget] and seen receive the choice.
    kv: of make_kv; its pools may be None here."""
    _heads("q", q, q, (q.shape[0], q.shape[1], kv.head_dim))
    _want("bounds", bounds, [_KV_TYPES[kv.type].split(".")[1], "uint8" if kv.type == FDY_F8 else "int16"],
          (kv.n_pages, kv.n_heads, 2, kv.head_dim))
    _want("table", table, ["int32"], table.shape[:2])
    _want("lens", lens, ["int32"], table.shape[:1])
    _want("rows", rows, ["int32"], q.shape[:1])
    _want("pages", pages, ["int32"], (q.shape[0], kv.n_heads, pages.shape[2]))
    _want("seen", seen, ["int32"], q.shape[:1])
    return fdy_select(_ptr(q), _ptr(bounds), _ptr(table), _ptr(lens), _ptr(rows), _ptr(pages), _ptr(seen), q.stride(0), q.stride(1),
                      kv, q.shape[0], q.shape[1], table.shape[0], table.shape[1], pages.shape[2], sinks, recent, type_of(q))


def make_selected_desc(*, q, out, table, lens, kv, scale, lse=None, rows=None, window=0):
    """As make_attend_desc, with table [rows, cache heads, pages]: a list of pages for every cache head."""
    for name, x in (("q", q), ("out", out)):
        _heads(name, x, q, (q.shape[0], q.shape[1], kv.head_dim))
    _want("table", table, ["int32"], (table.shape[0], kv.n_heads, table.shape[2]))
    _want("lens", lens, ["int32"], table.shape[:1])
    _want("rows", rows, ["int32"], q.shape[:1])
    _want("lse", lse, ["float32"], q.shape[:2])
    return fdy_attend(_ptr(q), _ptr(out), _ptr(lse), _ptr(table), _ptr(lens), _ptr(rows), q.stride(0), q.stride(1), out.stride(0),
                      out.stride(1), kv, scale, window, q.shape[0], q.shape[1], table.shape[0], table.shape[2], type_of(q), 0)


def make_token(*, token_stride, piece_bytes, pieces=1, piece_stride=0):
    """Where a token's bytes lie in a page of a plane; strides and sizes in bytes."""
    return fdy_token(token_stride, piece_stride, piece_bytes, pieces)


def make_pages(*, refs, free_bits, table, lens, page_tokens, planes=None, page_bytes=0, page_stride=0):
    """refs [pages], table [rows, pages of a row], lens [rows], 32-bit; free_bits, planes (device addresses) 64-bit."""
    _want("refs", refs, ["int32", "uint32"], refs.shape[:1])
    _want("free_bits", free_bits, ["int64", "uint64"], ((refs.shape[0] + 63) // 64,))
    _want("table", table, ["int32"], table.shape[:2])
    _want("lens", lens, ["int32"], table.shape[:1])
    _want("planes", planes, ["int64", "uint64"], () if planes is None else planes.shape[:1])
    return fdy_pages(_ptr(refs), _ptr(free_bits), _ptr(table), _ptr(lens), _ptr(planes), page_bytes, page_stride,
                     refs.shape[0], page_tokens, table.shape[0], table.shape[1], 0 if planes is None else planes.shape[0], 0)


_I32, _U32, _I64 = ("int32",), ("int32", "uint32"), ("int64",)


# ---- entry points (names as in include/fdy_decode.h) --------------------------------------------
def fdy_rope_frequencies(h_rope, check=True):
    """-> (rc, host array of rot_dim / 2 frequencies)."""
    import numpy as np

    f = np.zeros(max(1, h_rope.rot_dim // 2), np.float64)
    rc = _L().fdy_rope_frequencies(_d(h_rope), _ptr(f))
    if check:
        _check(rc, "fdy_rope_frequencies")
    return rc, f


def fdy_rope_table(h_rope, first, n_positions, d_table, stream=None, check=True):
    table = _list("d_table", d_table, ("float32",), 0 if h_rope is None else int(n_positions) * h_rope.rot_dim)
    rc = _L().fdy_rope_table(_d(h_rope), int(first), int(n_positions), table, _stream(stream))
    return _check(rc, "fdy_rope_table") if check else rc


def fdy_rope_append(h_desc, d_status=None, stream=None, check=True):
    rc = _L().fdy_rope_append(_d(h_desc), _ptr(d_status), _stream(stream))
    return _check(rc, "fdy_rope_append") if check else rc


def fdy_paged_attention_workspace_bytes(h_desc):
    return _L().fdy_paged_attention_workspace_bytes(_d(h_desc))


def fdy_paged_attention(h_desc, d_workspace, workspace_bytes, d_status=None, stream=None, check=True):
    rc = _L().fdy_paged_attention(_d(h_desc), _ptr(d_workspace), int(workspace_bytes), _ptr(d_status), _stream(stream))
    return _check(rc, "fdy_paged_attention") if check else rc


def fdy_tree_attention_workspace_bytes(h_desc):
    return _L().fdy_tree_attention_workspace_bytes(_d(h_desc))


def fdy_tree_attention(h_desc, d_workspace, workspace_bytes, d_status=None, stream=None, check=True):
    rc = _L().fdy_tree_attention(_d(h_desc), _ptr(d_workspace), int(workspace_bytes), _ptr(d_status), _stream(stream))
    return _check(rc, "fdy_tree_attention") if check else rc


def fdy_page_bounds(h_desc, d_status=None, stream=None, check=True):
    rc = _L().fdy_page_bounds(_d(h_desc), _ptr(d_status), _stream(stream))
    return _check(rc, "fdy_page_bounds") if check else rc


def fdy_page_select_workspace_bytes(h_desc):
    return _L().fdy_page_select_workspace_bytes(_d(h_desc))


def fdy_page_select(h_desc, d_workspace, workspace_bytes, d_status=None, stream=None, check=True):
    rc = _L().fdy_page_select(_d(h_desc), _ptr(d_workspace), int(workspace_bytes), _ptr(d_status), _stream(stream))
    return _check(rc, "fdy_page_select") if check else rc


def fdy_selected_attention_workspace_bytes(h_desc):
    return _L().fdy_selected_attention_workspace_bytes(_d(h_desc))


def fdy_selected_attention(h_desc, d_workspace, workspace_bytes, d_status=None, stream=None, check=True):
    rc = _L().fdy_selected_attention(_d(h_desc), _ptr(d_workspace), int(workspace_bytes), _ptr(d_status), _stream(stream))
    return _check(rc, "fdy_selected_attention") if check else rc


def fdy_pages_reset(h_pages, stream=None, check=True):
    rc = _L().fdy_pages_reset(_d(h_pages), _stream(stream))
    return _check(rc, "fdy_pages_reset") if check else rc


def fdy_pages_workspace_bytes(h_pages, n):
    return _L().fdy_pages_workspace_bytes(_d(h_pages), int(n))


def fdy_pages_extend(h_pages, d_rows, d_counts, n, d_slots, d_positions, n_slots, d_workspace, workspace_bytes,
                     d_status=None, stream=None, check=True):
    rows, counts = _list("d_rows", d_rows, _I32, n), _list("d_counts", d_counts, _I32, n)
    slots, positions = _list("d_slots", d_slots, _I64, n_slots), _list("d_positions", d_positions, _I32, n_slots)
    rc = _L().fdy_pages_extend(_d(h_pages), rows, counts, int(n), slots, positions, int(n_slots), _ptr(d_workspace),
                               int(workspace_bytes), _ptr(d_status), _stream(stream))
    return _check(rc, "fdy_pages_extend") if check else rc


def fdy_pages_fork(h_pages, d_src, d_dst, n, d_workspace, workspace_bytes, d_status=None, stream=None, check=True):
    src, dst = _list("d_src", d_src, _I32, n), _list("d_dst", d_dst, _I32, n)
    rc = _L().fdy_pages_fork(_d(h_pages), src, dst, int(n), _ptr(d_workspace), int(workspace_bytes),
                             _ptr(d_status), _stream(stream))
    return _check(rc, "fdy_pages_fork") if check else rc


def fdy_pages_free(h_pages, d_rows, n, d_status=None, stream=None, check=True):
    rc = _L().fdy_pages_free(_d(h_pages), _list("d_rows", d_rows, _I32, n), int(n), _ptr(d_status), _stream(stream))
    return _check(rc, "fdy_pages_free") if check else rc


def fdy_pages_keep(h_pages, h_token, d_rows, d_drafts, d_keep, d_kept, n, most, d_workspace, workspace_bytes, d_status=None,
                   stream=None, check=True):
    rows, drafts, kept = _list("d_rows", d_rows, _I32, n), _list("d_drafts", d_drafts, _I32, n), _list("d_kept", d_kept, _I32, n)
    rc = _L().fdy_pages_keep(_d(h_pages), _d(h_token), rows, drafts, _list("d_keep", d_keep, _I32, int(n) * int(most)), kept, int(n),
                             int(most), _ptr(d_workspace), int(workspace_bytes), _ptr(d_status), _stream(stream))
    return _check(rc, "fdy_pages_keep") if check else rc


def fdy_pages_copy(h_pages, d_src, d_dst, n, d_status=None, stream=None, check=True):
    src, dst = _list("d_src", d_src, _I32, n), _list("d_dst", d_dst, _I32, n)
    rc = _L().fdy_pages_copy(_d(h_pages), src, dst, int(n), _ptr(d_status), _stream(stream))
    return _check(rc, "fdy_pages_copy") if check else rc


def fdy_pages_compact(h_pages, d_map, d_n_live, d_workspace, workspace_bytes, d_status=None, stream=None, check=True):
    to, n_live = _list("d_map", d_map, _I32, 0 if h_pages is None else h_pages.n_pages), _list("d_n_live", d_n_live, _U32, 1)
    rc = _L().fdy_pages_compact(_d(h_pages), to, n_live, _ptr(d_workspace), int(workspace_bytes), _ptr(d_status),
                                _stream(stream))
    return _check(rc, "fdy_pages_compact") if check else rc
