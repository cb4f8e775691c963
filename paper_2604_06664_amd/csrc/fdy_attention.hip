// fdy_attention.hip - attention of one new token of every sequence over its pages, split over the length and joined.
//
// out = sum_t e^(x_t) v_t / sum_t e^(x_t), x_t = scale k_t.q, in one pass over the keys and values with a running maximum
// and sum.  All query heads of a cache head read the same keys and values, 2 * group flops a byte: the bound is memory, and
// the matrix cores only keep the arithmetic out of its way (a 16-row tile holds up to 16 query heads of a cache head).
//
// A wave takes 32 tokens at a time, straight from the pages into the operands, no LDS in the loop:
//   S^T = K Q^T   lane l holds key row l % 16 (of 16 tokens) and the elements of group l / 16; the sums come out with a
//                 query head a lane column and tokens 4 (l / 16) + i in the lane's four registers,
//   O^T = V^T P^T whose second operand wants, for the lane's query head, eight tokens: these same registers of the two
//                 16-token halves, once the products' inner index runs over tokens in that order.  Its first operand wants
//                 the same eight tokens of one element of v in a lane: the lane loads eight tokens by eight elements and
//                 transposes them in registers (v_perm).
// A query head's maximum, sum and output all lie in one lane column, so rescaling needs no exchange but the maximum over the
// four groups.  Four waves take the tiles of a piece in turn and join in LDS; the pieces of a row are joined by whichever
// workgroup finishes last.
#include "fdy_types.hpp"

using namespace fdy;

namespace {

constexpr u32 kWaves = 4, kTile = 32, kCus = 256;
constexpr u32 kLeast = 8;  // tiles of a piece, at least: two for each wave
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct AttendArg {
  fdy_attend d;
  u32* status;
  u32* counters;  // [n_seqs][columns], zero between calls
  float* parts;   // [pieces][columns] of: [rows][head_dim] sums, [rows] maxima, [rows] sums of e; each 16-byte aligned
  u32 page_shift, group, q_tiles, columns, extra, rows;  // columns: cache heads x q_tiles; rows: query heads of a tile
};
typedef Arg<AttendArg> Attend;

template <typename T>
__device__ __forceinline__ f32x4 mfma(typename T::x8 a, typename T::x8 b, f32x4 c);
template <>
__device__ __forceinline__ f32x4 mfma<Bf16>(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
template <>
__device__ __forceinline__ f32x4 mfma<F16>(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Two e4m3 of a word as two elements (exact: 4 bits of significand, exponents within both types).
template <typename T, bool kHigh>
__device__ __forceinline__ u32 widen_f8x2(u32 w);
template <>
__device__ __forceinline__ u32 widen_f8x2<Bf16, false>(u32 w) {
  return __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false));
}
template <>
__device__ __forceinline__ u32 widen_f8x2<Bf16, true>(u32 w) {
  return __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true));
}
template <>
__device__ __forceinline__ u32 widen_f8x2<F16, false>(u32 w) {
  return __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false));
}
template <>
__device__ __forceinline__ u32 widen_f8x2<F16, true>(u32 w) {
  return __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true));
}

// Largest / sum over the four lanes that differ in l / 16: a swap of halves, then of rows, of a value with itself.  (The
// results are taken out of their vector first: hipcc 7.2 casts element 0 whichever element of a vector it is handed.)
__device__ __forceinline__ float over_groups(float x, float (*op)(float, float)) {
  const u32 v = __builtin_bit_cast(u32, x);
  const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  const u32 a0 = a[0], a1 = a[1];
  const u32 w = __builtin_bit_cast(u32, op(__builtin_bit_cast(float, a0), __builtin_bit_cast(float, a1)));
  const auto b = __builtin_amdgcn_permlane16_swap(w, w, false, false);
  const u32 b0 = b[0], b1 = b[1];
  return op(__builtin_bit_cast(float, b0), __builtin_bit_cast(float, b1));
}
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float plus(float a, float b) { return a + b; }

__host__ __device__ inline u32 part_floats(u32 rows, u32 head_dim) { return rows * head_dim + (2 * rows + 3) / 4 * 4; }

// ---- which tokens a workgroup takes -----------------------------------------------------------------
// A row's tokens, in tiles of 32 that begin at multiples of 32.
struct Span {
  u32 first, end;  // tokens seen
  u32 row;
  bool bad;
  __device__ u32 tiles() const { return end > first ? (end + kTile - 1) / kTile - first / kTile : 0; }
};

__device__ __forceinline__ Span span_of(const Attend& a, u32 s) {
  Span r;
  const int row = a.d.rows ? a.d.rows[s] : (int)s;
  r.row = (u32)row;
  r.bad = r.row >= a.d.n_rows;
  if (r.bad) r.row = 0;
  int n = r.bad ? 0 : a.d.lens[r.row];
  const u32 most = a.d.row_pages << a.page_shift;
  if (n < 0 || (u32)n > most) r.bad = true, n = n < 0 ? 0 : (int)most;
  r.end = (u32)n;
  r.first = a.d.window && r.end > a.d.window ? r.end - a.d.window : 0;
  return r;
}

struct Piece {
  u32 seq, split, n_splits, at;  // `at`: number of the piece
  bool none;
};

// The pieces of all rows, as equal as whole rows allow: every piece has at most `per` tiles, where
// sum(ceil(tiles / per)) <= sum(tiles) / per + n_seqs is at most the grid.  Every wave works this out for itself.
__device__ __forceinline__ Piece piece_of(const Attend& a, u32 at) {
  const u32 lane = lane_id(), n = a.d.n_seqs;
  u64 total = 0;
  for (u32 s0 = 0; s0 < n; s0 += 64) {
    const u32 s = s0 + lane;
    const u32 t = s < n ? span_of(a, s).tiles() : 0;
    const u64 inc = wave_incl_scan((u64)t);
    total += (u64)__shfl((long long)inc, 63);
  }
  u32 per = (u32)((total + a.extra - 1) / a.extra);
  if (per < kLeast) per = kLeast;
  Piece p;
  p.at = at;
  p.none = true;
  u32 base = 0;
  for (u32 s0 = 0; s0 < n; s0 += 64) {
    const u32 s = s0 + lane;
    u32 t = s < n ? span_of(a, s).tiles() : 0;
    u32 k = s < n ? (t > per ? (t + per - 1) / per : 1u) : 0u;
    const u32 inc = wave_incl_scan(k), sum = (u32)__shfl((int)inc, 63);
    if (at < base + sum) {
      const u32 l = (u32)__popcll(ballot(base + inc <= at));
      p.seq = s0 + l;
      p.n_splits = (u32)__shfl((int)k, (int)l);
      p.split = at - (base + (u32)__shfl((int)inc, (int)l) - p.n_splits);
      p.none = false;
      return p;
    }
    base += sum;
  }
  return p;
}

// ---- loads ------------------------------------------------------------------------------------------
template <int kBytes>
struct Word;
template <>
struct Word<16> {
  typedef v4u32 type;
  static __device__ type load(__amdgpu_buffer_rsrc_t r, u32 at, u32 plus) {
    return __builtin_amdgcn_raw_buffer_load_b128(r, at, plus, 0);
  }
};
template <>
struct Word<8> {
  typedef v2u32 type;
  static __device__ type load(__amdgpu_buffer_rsrc_t r, u32 at, u32 plus) {
    return __builtin_amdgcn_raw_buffer_load_b64(r, at, plus, 0);
  }
};
template <>
struct Word<4> {
  typedef u32 type;
  static __device__ type load(__amdgpu_buffer_rsrc_t r, u32 at, u32 plus) {
    return __builtin_amdgcn_raw_buffer_load_b32(r, at, plus, 0);
  }
};

template <typename W>
__device__ __forceinline__ u32 word(const W& w, int i) {
  return w[i];
}
template <>
__device__ __forceinline__ u32 word<u32>(const u32& w, int) {
  return w;
}

// kDim: head_dim rounded up to 64, 128 or 256.  kSmall: pages of less than 16 tokens, where 16 tokens lie in several pages
// and every lane looks its own up; otherwise 16 tokens have one page, whose address is the wave's.
template <typename T, bool kF8, int kDim, bool kSmall>
struct Tile {
  typedef typename T::x8 x8;
  static constexpr int kEs = kF8 ? 1 : 2;
  static constexpr int kLoads = kDim * kEs / 64;          // of 16 bytes a lane and 16 tokens of k
  static constexpr int kSteps = kDim / 32;                // products over 32 elements
  static constexpr int kWide = kDim >= 128 ? 8 : kDim / 16;  // elements of v a lane and token
  static constexpr int kParts = kDim / (16 * kWide);      // of v's row
  typedef typename Word<kWide * kEs>::type vword;
  v4u32 k[2][kLoads];
  vword v[8][kParts];

  // The wave's constant offsets
  struct Lanes {
    u32 col, grp;
    u32 k_at[kLoads];  // byte offsets of the lane's pieces of a key row, kNowhere behind head_dim
    u32 v_at[kParts];
    u64 k_head, v_head;
  };

  static __device__ void lanes(const Attend& a, u32 head, Lanes& z) {
    const u32 l = lane_id(), D = a.d.kv.head_dim;
    z.col = l & 15, z.grp = l >> 4;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const u32 e = (j * 4 + z.grp) * (16 / kEs);
      z.k_at[j] = e < D ? e * kEs : kNowhere;
    }
#pragma unroll
    for (int j = 0; j < kParts; ++j) {
      const u32 e = j * 16 * kWide + z.col * kWide;
      z.v_at[j] = e < D ? e * kEs : kNowhere;
    }
  }

  // Tokens [t, t + 32) of the row; those outside [first, end) read as zero.  Returns which of the two halves have a page.
  __device__ void load(const Attend& a, const Lanes& z, const Span& span, u32 head, u32 t, bool& bad) {
    const fdy_kv& c = a.d.kv;
    const u32 token_bytes = (u32)c.token_stride * kEs;
    const u64 head_bytes = head * c.head_stride * kEs;
    const int* table = a.d.table + (u64)span.row * a.d.row_pages;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const u32 t0 = t + u * 16;
      if (!kSmall) {
        const bool seen = t0 < span.end && t0 + 16 > span.first;
        const u32 page = seen ? uniform((u32)table[t0 >> a.page_shift]) : ~0u;
        const bool in = page < c.n_pages;
        bad |= seen && !in;
        const u64 at = in ? page * c.page_stride * kEs + (t0 & (c.page_tokens - 1)) * (u64)token_bytes + head_bytes : 0;
        const auto rk = buffer((const uint8_t*)c.k + at, kNowhere - 1), rv = buffer((const uint8_t*)c.v + at, kNowhere - 1);
        const u32 tk = t0 + z.col;
        const bool ok = in && tk >= span.first && tk < span.end;
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
          k[u][j] = Word<16>::load(rk, ok && z.k_at[j] != kNowhere ? z.k_at[j] + z.col * token_bytes : kNowhere, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const u32 tv = t0 + z.grp * 4 + i;
          const bool okv = in && tv >= span.first && tv < span.end;
#pragma unroll
          for (int j = 0; j < kParts; ++j)
            v[u * 4 + i][j] = Word<kWide * kEs>::load(
                rv, okv && z.v_at[j] != kNowhere ? z.v_at[j] + z.grp * 4 * token_bytes : kNowhere, i * token_bytes);
        }
      } else {
        const u32 tk = t0 + z.col;
        const bool seen = tk >= span.first && tk < span.end;
        const u32 page = seen ? (u32)table[tk >> a.page_shift] : ~0u;
        const bool ok = page < c.n_pages;
        bad |= seen && !ok;
        const uint8_t* p =
            (const uint8_t*)c.k + (ok ? page * c.page_stride * kEs + (tk & (c.page_tokens - 1)) * (u64)token_bytes + head_bytes : 0);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          k[u][j] = 0;
          if (ok && z.k_at[j] != kNowhere) k[u][j] = *(const v4u32*)(p + z.k_at[j]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const u32 tv = t0 + z.grp * 4 + i;
          const bool sv = tv >= span.first && tv < span.end;
          const u32 pv = sv ? (u32)table[tv >> a.page_shift] : ~0u;
          const bool okv = pv < c.n_pages;
          const uint8_t* q =
              (const uint8_t*)c.v + (okv ? pv * c.page_stride * kEs + (tv & (c.page_tokens - 1)) * (u64)token_bytes + head_bytes : 0);
#pragma unroll
          for (int j = 0; j < kParts; ++j) {
            v[u * 4 + i][j] = 0;
            if (okv && z.v_at[j] != kNowhere) v[u * 4 + i][j] = *(const vword*)(q + z.v_at[j]);
          }
        }
      }
    }
  }

  // Which of the lane's eight scores (tokens t + 16 u + 4 grp + i) have a key.
  __device__ u32 seen(const Attend& a, const Lanes& z, const Span& span, u32 t) const {
    u32 bits = 0;
    const int* table = a.d.table + (u64)span.row * a.d.row_pages;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32 tok = t + u * 16 + z.grp * 4 + i;
        bool ok = tok >= span.first && tok < span.end;
        if (ok) ok = (u32)table[tok >> a.page_shift] < a.d.kv.n_pages;
        bits |= (ok ? 1u : 0u) << (u * 4 + i);
      }
    return bits;
  }

  __device__ x8 key(int u, int step) const {
    if (!kF8) return __builtin_bit_cast(x8, k[u][step]);
    const u32 lo = k[u][step / 2][(step & 1) * 2], hi = k[u][step / 2][(step & 1) * 2 + 1];
    const v4u32 w = {widen_f8x2<T, false>(lo), widen_f8x2<T, true>(lo), widen_f8x2<T, false>(hi), widen_f8x2<T, true>(hi)};
    return __builtin_bit_cast(x8, w);
  }

  // Elements 2 e, 2 e + 1 of the lane's piece of a token's v.
  __device__ u32 value2(int token, int part, int e) const {
    if (!kF8) return word(v[token][part], e);
    const u32 w = word(v[token][part], e / 2);
    return e & 1 ? widen_f8x2<T, true>(w) : widen_f8x2<T, false>(w);
  }
};

// ---- the kernel -----------------------------------------------------------------------------------------
template <typename T, bool kF8, int kDim, bool kSmall>
__global__ void __launch_bounds__(256) attend_kernel(Attend a) {
  typedef Tile<T, kF8, kDim, kSmall> Tl;
  typedef typename T::x8 x8;
  typedef typename T::elem elem;
  constexpr int kWide = Tl::kWide, kParts = Tl::kParts, kSteps = Tl::kSteps, kPad = kDim + 4;
  __shared__ alignas(16) float s_o[kWaves][16][kPad];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  __shared__ u32 s_last;

  const u32 column = blockIdx.x % a.columns, at = blockIdx.x / a.columns;
  const Piece piece = piece_of(a, uniform(at));
  if (piece.none) return;
  const u32 wave = threadIdx.x >> 6, seq = uniform(piece.seq), head = column / a.q_tiles, tile = column % a.q_tiles;
  Span span = span_of(a, seq);
  span.first = uniform(span.first), span.end = uniform(span.end), span.row = uniform(span.row);
  bool bad = span.bad && piece.split == 0;
  const u32 D = a.d.kv.head_dim, q0 = tile * 16;
  const u32 rows = a.group - q0 < 16 ? a.group - q0 : 16;  // query heads of this tile

  typename Tl::Lanes z;
  Tl::lanes(a, head, z);

  // the tile's queries as the products' second operand: the same elements a lane as its keys
  x8 q[kSteps];
  {
    const elem* src = (const elem*)a.d.q + seq * a.d.q_seq + (head * a.group + q0 + z.col) * a.d.q_head;
#pragma unroll
    for (int st = 0; st < kSteps; ++st) {
      const u32 e = kF8 ? (st / 2) * 64 + z.grp * 16 + (st & 1) * 8 : st * 32 + z.grp * 8;
      const v4u32 none = 0;
      q[st] = __builtin_bit_cast(x8, none);
      if (z.col < rows && e < D) q[st] = *(const x8*)(src + e);
    }
  }
  const float scale = a.d.scale * (kF8 && a.d.kv.k_scale ? a.d.kv.k_scale[head] : 1.f) * kLog2e;

  f32x4 o[kParts * kWide];
#pragma unroll
  for (int i = 0; i < kParts * kWide; ++i) o[i] = 0;
  float m = -INFINITY, sum = 0.f;

  const u32 all = span.tiles(), tile0 = span.first / kTile;
  const u32 begin = tile0 + (u32)((u64)all * piece.split / piece.n_splits);
  const u32 end = tile0 + (u32)((u64)all * (piece.split + 1) / piece.n_splits);
  for (u32 i = begin + wave; i < end; i += kWaves) {
    const u32 t = uniform(i * kTile);
    Tl x;
    x.load(a, z, span, head, t, bad);
    f32x4 s[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      s[u] = 0;
#pragma unroll
      for (int st = 0; st < kSteps; ++st) s[u] = mfma<T>(x.key(u, st), q[st], s[u]);
    }
    const u32 seen = x.seen(a, z, span, t);
    float mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i2 = 0; i2 < 4; ++i2) {
        s[u][i2] = seen >> (u * 4 + i2) & 1 ? s[u][i2] * scale : -INFINITY;
        mx = fmaxf(mx, s[u][i2]);
      }
    mx = over_groups(mx, larger);
    const float m_new = fmaxf(m, mx), ref = m_new == -INFINITY ? 0.f : m_new;
    const float keep = __builtin_amdgcn_exp2f(m - ref);
    m = m_new;
    x8 p;
    float part = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float e = __builtin_amdgcn_exp2f(s[j / 4][j % 4] - ref);
      part += e;
      p[j] = (elem)e;
    }
    sum = sum * keep + part;
#pragma unroll
    for (int part_ = 0; part_ < kParts; ++part_)
#pragma unroll
      for (int e2 = 0; e2 < kWide / 2; ++e2) {
        v4u32 lo, hi;  // eight tokens of elements 2 e2 and 2 e2 + 1
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const u32 x0 = x.value2(2 * j, part_, e2), x1 = x.value2(2 * j + 1, part_, e2);
          lo[j] = __builtin_amdgcn_perm(x1, x0, 0x05040100u);
          hi[j] = __builtin_amdgcn_perm(x1, x0, 0x07060302u);
        }
        f32x4& c0 = o[part_ * kWide + 2 * e2];
        f32x4& c1 = o[part_ * kWide + 2 * e2 + 1];
        c0 = mfma<T>(__builtin_bit_cast(x8, lo), p, c0 * keep);
        c1 = mfma<T>(__builtin_bit_cast(x8, hi), p, c1 * keep);
      }
  }
  sum = over_groups(sum, plus);
  if (ballot(bad) && lane_id() == 0) raise_status(a.status, FDY_ST_BAD_INDEX);

  // the four waves' sums, joined
#pragma unroll
  for (int part_ = 0; part_ < kParts; ++part_)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < kWide; ++e) s_o[wave][z.col][part_ * 16 * kWide + (z.grp * 4 + i) * kWide + e] = o[part_ * kWide + e][i];
  if (z.grp == 0) s_m[wave][z.col] = m, s_l[wave][z.col] = sum;
  __syncthreads();
  const u32 quads = D / 4;
  const float v_scale = kF8 && a.d.kv.v_scale ? a.d.kv.v_scale[head] : 1.f;
  const u64 slot_floats = part_floats(a.rows, D);
  float* mine = a.parts + ((u64)piece.at * a.columns + column) * slot_floats;
  auto finish = [&](u32 r, u32 qd, float M, float L, f32x4 x) {
    const u32 h = head * a.group + q0 + r;
    x = x * (L == 0.f ? 0.f : v_scale / L);
    elem* out = (elem*)a.d.out + seq * a.d.out_seq + h * a.d.out_head + qd * 4;
    typedef elem x4 __attribute__((ext_vector_type(4)));
    *(x4*)out = __builtin_convertvector(x, x4);
    if (qd == 0 && a.d.lse) a.d.lse[(u64)seq * a.d.n_q_heads + h] = L == 0.f ? -INFINITY : (M + __builtin_log2f(L)) * kLn2;
  };
  for (u32 i = threadIdx.x; i < rows * quads; i += 256) {
    const u32 r = i / quads, qd = i - r * quads;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < (int)kWaves; ++w) M = fmaxf(M, s_m[w][r]);
    const float ref = M == -INFINITY ? 0.f : M;
    float L = 0.f;
    f32x4 x = 0;
#pragma unroll
    for (int w = 0; w < (int)kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(s_m[w][r] - ref);
      L += f * s_l[w][r];
      x += f * *(const f32x4*)&s_o[w][r][qd * 4];
    }
    if (piece.n_splits == 1) {
      finish(r, qd, ref, L, x);
    } else {
      *(f32x4*)(mine + r * D + qd * 4) = x;
      if (qd == 0) mine[a.rows * D + r] = M, mine[a.rows * (D + 1) + r] = L;
    }
  }
  if (piece.n_splits == 1) return;

  // the row's pieces, joined by the workgroup that finishes last; its counter is left at zero
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    u32* counter = a.counters + seq * a.columns + column;
    const u32 before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
    s_last = before == piece.n_splits - 1;
    if (s_last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  const float* parts = a.parts + ((u64)(piece.at - piece.split) * a.columns + column) * slot_floats;
  const u64 apart = (u64)a.columns * slot_floats;
  for (u32 i = threadIdx.x; i < rows * quads; i += 256) {
    const u32 r = i / quads, qd = i - r * quads;
    float M = -INFINITY;
    for (u32 k = 0; k < piece.n_splits; ++k) M = fmaxf(M, parts[k * apart + a.rows * D + r]);
    const float ref = M == -INFINITY ? 0.f : M;
    float L = 0.f;
    f32x4 x = 0;
#pragma unroll 4
    for (u32 k = 0; k < piece.n_splits; ++k) {
      const float* p = parts + k * apart;
      const float f = __builtin_amdgcn_exp2f(p[a.rows * D + r] - ref);
      L += f * p[a.rows * (D + 1) + r];
      x += f * *(const f32x4*)(p + r * D + qd * 4);
    }
    finish(r, qd, ref, L, x);
  }
}

template <typename T, bool kF8, int kDim>
int launch_attend(const Attend& a, hipStream_t stream) {
  const u32 blocks = (a.d.n_seqs + a.extra) * a.columns;
  (void)hipGetLastError();  // drop any stale error left by earlier, unrelated runtime calls
  if (a.d.kv.page_tokens < 16)
    hipLaunchKernelGGL((attend_kernel<T, kF8, kDim, true>), dim3(blocks), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((attend_kernel<T, kF8, kDim, false>), dim3(blocks), dim3(256), 0, stream, a);
  FDY_HIP_TRY(hipGetLastError());
  return FDY_OK;
}

template <typename T, bool kF8>
int launch_attend(const Attend& a, hipStream_t stream) {
  if (a.d.kv.head_dim <= 64) return launch_attend<T, kF8, 64>(a, stream);
  if (a.d.kv.head_dim <= 128) return launch_attend<T, kF8, 128>(a, stream);
  return launch_attend<T, kF8, 256>(a, stream);
}

bool sizes_valid(const fdy_attend& d) {
  if (!kv_valid(d.kv) || d.reserved || d.type > FDY_F16 || (d.kv.type != d.type && d.kv.type != FDY_F8)) return false;
  if (d.kv.head_dim % (d.kv.type == FDY_F8 ? 16 : 8)) return false;
  if (d.n_seqs > 65536u || !d.n_q_heads || d.n_q_heads > 65536u || d.n_q_heads % d.kv.n_heads) return false;
  if ((u64)d.n_seqs * d.n_q_heads > 1u << 22) return false;
  return (u64)d.row_pages * d.kv.page_tokens < 1ull << 31;
}

// How the call is laid out; the same for the workspace's size and the launch.
void lay_out(const fdy_attend& d, Attend& a) {
  a.d = d;
  a.page_shift = log2_of(d.kv.page_tokens);
  a.group = d.n_q_heads / d.kv.n_heads;
  a.q_tiles = (a.group + 15) / 16;
  a.columns = d.kv.n_heads * a.q_tiles;
  a.rows = a.group < 16 ? a.group : 16;
  // pieces beyond one a row: enough to fill the chip with four workgroups a compute unit, and to halve rows longer than
  // the mean where there are more rows than that
  a.extra = (kCus * 4 + a.columns - 1) / a.columns;
  if (a.extra < d.n_seqs) a.extra = d.n_seqs;
}
size_t counter_bytes(const Attend& a) { return ((size_t)a.d.n_seqs * a.columns * 4 + 255) / 256 * 256; }

}  // namespace

extern "C" size_t fdy_paged_attention_workspace_bytes(const fdy_attend* h) {
  if (!h || !sizes_valid(*h)) return 0;
  Attend a{};
  lay_out(*h, a);
  const size_t parts = (size_t)(h->n_seqs + a.extra) * a.columns * part_floats(a.rows, h->kv.head_dim) * 4;
  return counter_bytes(a) + (parts + 255) / 256 * 256;
}

extern "C" int fdy_paged_attention(const fdy_attend* h, void* d_workspace, size_t workspace_bytes, uint32_t* d_status,
                                   void* stream) {
  if (!h || !sizes_valid(*h)) return FDY_ERR_INVALID_ARG;
  const fdy_attend& d = *h;
  if (d.n_seqs == 0) return FDY_OK;
  if (!d.q || !d.out || !d.table || !d.lens || !d.kv.k || !d.kv.v) return FDY_ERR_INVALID_ARG;
  if (!aligned(d.q, 16) || !aligned(d.out, 16) || !aligned(d.kv.k, 16) || !aligned(d.kv.v, 16) || !aligned(d.lse, 4) ||
      !aligned(d.table, 4) || !aligned(d.lens, 4) || !aligned(d.rows, 4) || !aligned(d.kv.k_scale, 4) || !aligned(d.kv.v_scale, 4))
    return FDY_ERR_INVALID_ARG;
  if ((d.q_seq | d.q_head | d.out_seq | d.out_head) % 8) return FDY_ERR_INVALID_ARG;
  if ((d.kv.page_stride | d.kv.token_stride | d.kv.head_stride) % (d.kv.type == FDY_F8 ? 16 : 8)) return FDY_ERR_INVALID_ARG;
  if (!d_workspace || !aligned(d_workspace, 256) || workspace_bytes < fdy_paged_attention_workspace_bytes(h))
    return FDY_ERR_WORKSPACE;
  Attend a{};
  lay_out(d, a);
  a.status = d_status;
  a.counters = (u32*)d_workspace;
  a.parts = (float*)((uint8_t*)d_workspace + counter_bytes(a));
  const bool f8 = d.kv.type == FDY_F8;
  if (d.type == FDY_BF16)
    return f8 ? launch_attend<Bf16, true>(a, (hipStream_t)stream) : launch_attend<Bf16, false>(a, (hipStream_t)stream);
  return f8 ? launch_attend<F16, true>(a, (hipStream_t)stream) : launch_attend<F16, false>(a, (hipStream_t)stream);
}
