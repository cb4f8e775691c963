/*
 * fdy_decode.h - operators of a decode step over a paged key-value cache, for MI355X (gfx950), C ABI.
 *
 * What the captured decode graphs of a serving engine hold at every layer (Section 2.1: one graph per batch size;
 * Section 4.1.1: the KV cache is one of the allocations that the deterministic layout places): rotary positions with the
 * append of keys and values to their pages, attention of one new token of every sequence over its pages, and, once a
 * step, the keeping of the pages themselves.  They are made to be captured and restored by the calls of fdy.h:
 *   - every kernel of a step takes ONE argument, a plain struct of FDY_DECODE_ARG_BYTES bytes whose pointers lie at
 *     multiples of 8 bytes, so that fdy_scan_pointers finds them in its argument buffer and fdy_materialize /
 *     fdy_scan_rebase move them to a new layout (fdy_rope_table, which is called once, is not meant);
 *   - grids follow from host sizes alone (rows, heads, capacity), lengths are read on the device: a captured launch
 *     stays right while the sequences grow;
 *   - nothing is read back to the host, nothing is allocated, no memory is cleared by a memset.
 *
 * The conventions of fdy.h on memory, streams and errors hold (its integers do not: these work on floats): d_* / device
 * pointers inside the descriptors are the caller's, descriptors are HOST
 * structs that are read during the call only, calls only enqueue, return codes and status bits are those of fdy.h.  What
 * only the device can see (a length, a page number, a row number out of range) raises FDY_ST_BAD_INDEX and is skipped as
 * stated at each call.  Unless stated otherwise arrays that a call writes do not overlap arrays that it reads.
 */
#ifndef FDY_DECODE_H
#define FDY_DECODE_H

#include <stddef.h>
#include <stdint.h>

#include "fdy.h"

#ifdef __cplusplus
extern "C" {
#endif

#define FDY_DECODE_ARG_BYTES 512u /* bytes of every kernel's argument */

/* ---- element types -------------------------------------------------------------------- */
#define FDY_BF16 0u /* bfloat16                                                               */
#define FDY_F16 1u  /* IEEE half                                                              */
#define FDY_F8 2u   /* 8-bit e4m3 (OCP: no infinities, largest 448); caches only              */

/* One layer's keys and values in pages.  Token `i` of page `p`, head `h`, starts at element
 *   p * page_stride + i * token_stride + h * head_stride
 * of k and of v, and its head_dim elements are contiguous; so both [page][token][head][dim] and
 * [page][head][token][dim] are served.  An F8 element x stands for x * scale[h].
 *   page_tokens  a power of two, at most 65,536
 *   head_dim     1 to 256 (see the calls for what they take)
 *   a page's elements span less than 2^31 bytes; n_pages < 2^31 */
typedef struct {
  void* k;
  void* v;
  const float* k_scale; /* [n_heads] device, F8 only; NULL: 1 */
  const float* v_scale;
  uint64_t page_stride, token_stride, head_stride; /* elements */
  uint32_t type;                                   /* FDY_BF16, FDY_F16 or FDY_F8 */
  uint32_t n_pages, page_tokens, n_heads, head_dim;
  uint32_t reserved; /* 0 */
} fdy_kv;            /* 80 B */

/* ---- rotary positions -------------------------------------------------------------------
 * The angle of pair i of rot_dim / 2 at position p is p * f_i, f_i = base^(-2 i / rot_dim), rescaled for contexts longer
 * than the trained ones by one of
 *   FDY_ROPE_PLAIN   f_i
 *   FDY_ROPE_LINEAR  f_i / factor (positions interpolated)
 *   FDY_ROPE_NTK     f_i with base * factor^(rot_dim / (rot_dim - 2)); rot_dim >= 4
 *   FDY_ROPE_YARN    f_i ((1 - g) / factor + g), g = 1 - clamp((i - lo) / (hi - lo), 0, 1), where lo and hi are the (real)
 *                    pair numbers at which a pair makes `high` and `low` turns over trained_len positions:
 *                    rot_dim ln(trained_len / (2 pi turns)) / (2 ln base), lo rounded down and hi up, both held
 *                    within [0, rot_dim - 1], hi = lo + 0.001 where they meet
 *   FDY_ROPE_BANDS   f_i where trained_len f_i / (2 pi) > high (short waves), f_i / factor where it is < low, and between
 *                    them f_i ((1 - s) / factor + s) with s = (trained_len f_i / (2 pi) - low) / (high - low)
 * and cos and sin are multiplied by `magnitude` (1 unless a scheme wants another). */
#define FDY_ROPE_PLAIN 0u
#define FDY_ROPE_LINEAR 1u
#define FDY_ROPE_NTK 2u
#define FDY_ROPE_YARN 3u
#define FDY_ROPE_BANDS 4u
typedef struct {
  uint32_t scaling;   /* FDY_ROPE_PLAIN ... FDY_ROPE_BANDS */
  uint32_t rot_dim;   /* even, 2 to 256 */
  double base;        /* > 1 */
  double factor;      /* > 0; not read by FDY_ROPE_PLAIN */
  double low, high;   /* turns, 0 < low < high: FDY_ROPE_YARN, FDY_ROPE_BANDS */
  double trained_len; /* > 0: FDY_ROPE_YARN, FDY_ROPE_BANDS */
  double magnitude;   /* finite */
} fdy_rope;           /* 56 B */

/* Writes d_table[p][0][i] = magnitude cos((first + p) f_i), d_table[p][1][i] = magnitude sin(...) for 0 <= p < n_positions,
 * i < rot_dim / 2: what fdy_rope_append reads, made once.  Angles are worked out in 64 bits (in 32 a position of a million
 * would be 0.06 radians off), the table holds 32.  d_table 16-byte aligned; first + n_positions <= 2^31.
 * FDY_ERR_INVALID_ARG: a field out of the ranges above, a null or misaligned pointer. */
int fdy_rope_table(const fdy_rope* h_rope, uint64_t first, uint32_t n_positions, float* d_table, void* hip_stream);

/* The frequencies f_i that the table is made of (host; h_freq[rot_dim / 2]). */
int fdy_rope_frequencies(const fdy_rope* h_rope, double* h_freq);

/* ---- rotary positions + append to the pages ---------------------------------------------
 * For token t: the first rot_dim elements of every query and key head are turned by the table's row positions[t],
 *   FDY_ROPE_HALF         pairs (x_i, x_{i + rot_dim/2})
 *   FDY_ROPE_INTERLEAVED  pairs (x_{2i}, x_{2i+1})
 *   (x, y) -> (x cos - y sin, y cos + x sin),
 * the others are copied; queries go to q_out, keys to k_out (if not NULL) and, with the values, to the cache at
 * slots[t] = page * page_tokens + place.  Worked out in 32 bits, each result rounded once to the type it is stored in (to
 * nearest, ties to even; F8 saturates at +-448, NaN stays NaN).
 *   n_tokens at most 2^23.
 *   A position outside [0, n_positions) leaves the whole token out and raises FDY_ST_BAD_INDEX.
 *   slots[t] = -1: no cache is written for t (rows that pad a captured batch); any other slot outside the cache: the same,
 *   and FDY_ST_BAD_INDEX.  Two tokens with one slot: the cache holds either's element by element.
 *   q NULL: no queries.  slots NULL: no cache is written (kv.k, kv.v may be NULL, v is not read).
 *   q_out may be q and k_out may be k with the same strides (in place).
 * Token strides, head strides: in elements; a head's head_dim elements are contiguous.  kv.head_dim, kv.n_heads give the
 * heads' size and the number of key heads also where no cache is written; kv.type is `type` or FDY_F8.  Any head_dim up to
 * 256 and any even rot_dim up to it are served; rot_dim a multiple of 16, head_dim of 8, and pointers and strides at
 * multiples of 16 bytes (8 elements) take the widest accesses, half of each the next, anything else single elements. */
#define FDY_ROPE_HALF 0u
#define FDY_ROPE_INTERLEAVED 1u
typedef struct {
  const void* q; /* [n_tokens][n_q_heads][head_dim] or NULL */
  const void* k; /* [n_tokens][kv.n_heads][head_dim]        */
  const void* v;
  void* q_out;
  void* k_out;              /* or NULL */
  const int32_t* positions; /* [n_tokens] */
  const float* table;       /* fdy_rope_table's, [n_positions][2][rot_dim / 2], 16-byte aligned */
  const int64_t* slots;     /* [n_tokens] or NULL */
  uint64_t q_token, q_head, k_token, k_head, v_token, v_head;     /* strides */
  uint64_t q_out_token, q_out_head, k_out_token, k_out_head;
  fdy_kv kv;
  uint32_t n_tokens, n_q_heads, n_positions, rot_dim;
  uint32_t type;   /* FDY_BF16 or FDY_F16 */
  uint32_t layout; /* FDY_ROPE_HALF or FDY_ROPE_INTERLEAVED */
} fdy_append;      /* 248 B */
int fdy_rope_append(const fdy_append* h_desc, uint32_t* d_status, void* hip_stream);

/* ---- attention of one new token over the pages -------------------------------------------
 * For sequence s with row r = rows[s] (s where rows is NULL), n = lens[r] tokens of which token t lies in page
 * table[r][t / page_tokens], and query head h (of cache head h / (n_q_heads / kv.n_heads)):
 *   x_t = scale * q_h . k_t            over t in [max(0, n - window), n)     (window 0: all)
 *   out_h = sum_t e^(x_t) v_t / sum_t e^(x_t),   lse_h = ln sum_t e^(x_t)
 * No tokens (or all x_t minus infinity): out 0, lse minus infinity.  Products are of the stored types (F8 widened
 * exactly), sums, maxima and the joining of parts are held in 32 bits; e^(x_t - max) goes as two elements of `type`
 * into its product with v (2^-15 of it is lost with bf16, 2^-21 with f16; of one below 2^-18 with f16 2^-40), out is rounded
 * once at the end.  What lies in pages behind the row's length is not read.
 *   lens outside [0, row_pages * page_tokens]: held within, FDY_ST_BAD_INDEX; rows outside [0, n_rows): as no tokens, and
 *   FDY_ST_BAD_INDEX; a page number outside [0, kv.n_pages): its tokens are left out, FDY_ST_BAD_INDEX.
 * The results do not depend on what else is in the batch except in the rounding of joined parts, and are the same every
 * time for the same call.
 *   q, out, kv.k, kv.v 16-byte aligned, strides multiples of 8 elements (kv's of 16 bytes); head_dim a multiple of 8
 *   (of 16 with F8) up to 256; n_q_heads a multiple of kv.n_heads; kv.type is `type` or FDY_F8; n_seqs <= 65,536,
 *   n_q_heads <= 65,536, n_seqs * n_q_heads <= 2^22, row_pages * page_tokens < 2^31, n_seqs times that <= 2^36.
 *   workspace  device, 256-byte aligned, fdy_paged_attention_workspace_bytes() (0: a field out of range).  The caller
 *              clears it once, before its first use; every call leaves what it needs cleared cleared.  Calls that share one
 *              must not overlap in time, and after FDY_ERR_HIP it is cleared again.  One sized for a descriptor serves
 *              every one with no more sequences, no wider tables and the same heads, head_dim, page_tokens and kv.type, in
 *              any order. */
typedef struct {
  const void* q;        /* [n_seqs][n_q_heads][head_dim] */
  void* out;            /* [n_seqs][n_q_heads][head_dim] */
  float* lse;           /* [n_seqs][n_q_heads] or NULL   */
  const int32_t* table; /* [n_rows][row_pages]           */
  const int32_t* lens;  /* [n_rows]                      */
  const int32_t* rows;  /* [n_seqs] or NULL              */
  uint64_t q_seq, q_head, out_seq, out_head; /* strides  */
  fdy_kv kv;
  float scale;
  uint32_t window; /* 0: none */
  uint32_t n_seqs, n_q_heads, n_rows, row_pages;
  uint32_t type; /* FDY_BF16 or FDY_F16 */
  uint32_t reserved;
} fdy_attend; /* 192 B */
size_t fdy_paged_attention_workspace_bytes(const fdy_attend* h_desc);
int fdy_paged_attention(const fdy_attend* h_desc, void* d_workspace, size_t workspace_bytes, uint32_t* d_status,
                        void* hip_stream);

/* ---- keeping the pages --------------------------------------------------------------------
 * A pool of n_pages pages that rows of pages share.  Its books are device arrays of the caller's:
 *   refs[p]       rows that hold page p (a row that holds it twice counts twice)
 *   free_bits     bit p of the array is set iff refs[p] == 0 (bits from n_pages on are clear)
 *   table[r][j]   page that holds tokens [j * page_tokens, (j+1) * page_tokens) of row r, for j < ceil(lens[r] / page_tokens);
 *                 what lies behind is not read
 *   lens[r]       tokens of row r
 * and its contents are n_planes areas (keys and values of every layer): page p of plane i is page_bytes bytes at
 * planes[i] + p * page_stride.  planes[i] are device addresses, in a device array; n_planes 0: books only.
 * Everything below is deterministic: pages are taken lowest number first, in the order of the list of rows.
 * Books that contradict each other (or lists with a row twice) give unspecified books, with no access out of bounds:
 * page and row numbers and lengths out of range are skipped and raise FDY_ST_BAD_INDEX; of entries with the same row to
 * be written the first counts, the others are skipped with FDY_ST_BAD_INDEX.
 *   refs, table, lens, rows 4-byte, free_bits, planes, slots 8-byte aligned; planes' addresses, page_bytes, page_stride
 *   multiples of 16, page_bytes < 2^30; page_tokens a power of two up to 65,536; n_pages, n_rows <= 2^28, row_pages <= 2^25,
 *   row_pages * page_tokens < 2^31, n_planes <= 32,768, n_planes * ceil(page_bytes / 8,192) < 2^32 */
typedef struct {
  uint32_t* refs;      /* [n_pages]              */
  uint64_t* free_bits; /* [ceil(n_pages / 64)]   */
  int32_t* table;      /* [n_rows][row_pages]    */
  int32_t* lens;       /* [n_rows]               */
  const uint64_t* planes; /* [n_planes] addresses, or NULL */
  uint64_t page_bytes, page_stride;
  uint32_t n_pages, page_tokens, n_rows, row_pages, n_planes;
  uint32_t reserved;
} fdy_pages; /* 80 B */

/* All pages free, all rows empty. */
int fdy_pages_reset(const fdy_pages* h_pages, void* hip_stream);

/* Workspace (device, 256-byte aligned, contents irrelevant) of the calls below for lists of up to n entries; 0: a field
 * out of range.  Calls that share one must not overlap in time. */
size_t fdy_pages_workspace_bytes(const fdy_pages* h_pages, uint32_t n);

/* Room for counts[i] (1 each where counts is NULL) more tokens of row rows[i] (i where rows is NULL), i < n: new pages are
 * taken, lens grows, and slots / positions (either may be NULL) receive, packed in the order of the list, where each new
 * token goes and its number in its row: what fdy_rope_append takes.  A partly filled last page that other rows hold too is
 * copied first, in all planes, to a page of the row's own; of rows that hold such a page among themselves alone the last in
 * the list keeps it.
 *   A row gets all or nothing: one that does not fit its table, or whose pages the pool has not left after all rows before
 *   it (those that get nothing for want of pages count as well), or that would keep a page of which one of these still holds
 *   the other share, or whose tokens end behind n_slots, stays as it is, its slots are -1 (positions as if), and
 *   FDY_ST_CAPACITY is raised.
 *   counts[i] < 0 counts as 0 and raises FDY_ST_BAD_INDEX.  n <= 65,536; the sum of counts < 2^31. */
int fdy_pages_extend(const fdy_pages* h_pages, const int32_t* d_rows, const int32_t* d_counts, uint32_t n,
                     int64_t* d_slots, int32_t* d_positions, uint32_t n_slots, void* d_workspace, size_t workspace_bytes,
                     uint32_t* d_status, void* hip_stream);

/* Row dst[i] becomes a holder of what row src[i] held before the call, for all i < n at once (a permutation of rows, beams
 * that go on from other beams); what dst[i] held is given up, pages that nobody holds any more become free.  Entries of
 * dst[i]'s table behind its new length stay what they were.  No page is copied: fdy_pages_extend does it when a shared
 * page is to be written.  n <= 65,536 */
int fdy_pages_fork(const fdy_pages* h_pages, const int32_t* d_src, const int32_t* d_dst, uint32_t n, void* d_workspace,
                   size_t workspace_bytes, uint32_t* d_status, void* hip_stream);

/* Rows rows[i] give up their pages and become empty.  n <= 65,536 */
int fdy_pages_free(const fdy_pages* h_pages, const int32_t* d_rows, uint32_t n, uint32_t* d_status, void* hip_stream);

/* The contents of page src[i] to page dst[i] in all planes, i < n; no page may be both, or twice in dst.  The books stay
 * as they are. */
int fdy_pages_copy(const fdy_pages* h_pages, const int32_t* d_src, const int32_t* d_dst, uint32_t n, uint32_t* d_status,
                   void* hip_stream);

/* Moves pages so that the live ones are [0, *d_n_live): the k-th live page from there on goes to the k-th free page below,
 * with its contents in all planes, and the rows' tables follow.  d_map[n_pages] (may be NULL) receives the new number of
 * every live page, -1 for the free ones (for page numbers kept elsewhere). */
int fdy_pages_compact(const fdy_pages* h_pages, int32_t* d_map, uint32_t* d_n_live, void* d_workspace,
                      size_t workspace_bytes, uint32_t* d_status, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* FDY_DECODE_H */
