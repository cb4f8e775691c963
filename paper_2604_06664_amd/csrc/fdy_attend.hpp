// What the kernels of attention over a paged cache share (gfx950): the products, the weights in two parts, a row's tokens, and a
// tile of 32 of them from the pages to the operands.  Not installed.
#pragma once
#include "fdy_types.hpp"

namespace fdy {

constexpr u32 kTile = 32;
constexpr u32 kCus = 256;  // of the card: the workspace's size is asked for without a device
constexpr u32 kEach = 3;  // what a row costs beside its tiles (queries, join, output), in tiles
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Weights e^(x - max) are at most 1.  In f16 they would be held in steps of 2^-24 below 2^-14, and at 2^-25 be gone, which many
// small ones beside a large one together are not: there they are held 2^15 times as large (as are their sum and the output until
// the division), with all 11 bits down to 2^-29.
template <typename T>
inline constexpr float kLift = 0.f;
template <>
inline constexpr float kLift<F16> = 15.f;

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

// A product with v takes weights of its own type only, 8 bits of bf16 and 11 of f16, which is all that the outputs have: so each
// goes as two, the first rounded down to one step below, the rest (of one to two steps) as the second: 2^-15 of a weight is lost, or 2^-21.
// The rest is not 0 where the weight is not, for an infinite value times 0 would be no number.  The second product costs nothing
// where memory bounds the call (64 rows of 4,096 tokens 171 us with and without), 1 or 2 % in 8 bits (64 of 4,096 tokens, 40 heads of
// one: 60 for 59).
template <typename T>
__device__ __forceinline__ void split(float x, float y, u32& first, u32& rest);
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u32 step_below(u32 pair) {
  return __builtin_bit_cast(u32, __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, pair), (u16x2)(1)));
}
template <>
__device__ __forceinline__ void split<Bf16>(float x, float y, u32& first, u32& rest) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  first = step_below(__builtin_amdgcn_perm(__builtin_bit_cast(u32, y), __builtin_bit_cast(u32, x), 0x07060302u));
  const bf16x2 r = {(__bf16)(x - __builtin_bit_cast(float, first << 16)), (__bf16)(y - __builtin_bit_cast(float, first & 0xffff0000u))};
  rest = __builtin_bit_cast(u32, r);
}
template <>
__device__ __forceinline__ void split<F16>(float x, float y, u32& first, u32& rest) {
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  first = step_below(__builtin_bit_cast(u32, __builtin_amdgcn_cvt_pkrtz(x, y)));
  const f16x2 f = __builtin_bit_cast(f16x2, first), r = {(_Float16)(x - (float)f[0]), (_Float16)(y - (float)f[1])};
  rest = __builtin_bit_cast(u32, r);
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

// Parts go from one workgroup to another, on another die as it may be: they are written through to memory and read from
// there (device scope on each access), for a fence would write back and drop all that the dies' caches hold, once a wave.
constexpr int kDeviceScope = 0x10;  // sc1
__device__ __forceinline__ float as_float(u32 v) { return __builtin_bit_cast(float, v); }
__device__ __forceinline__ void put_part(__amdgpu_buffer_rsrc_t part, u32 at, f32x4 x) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u32, x), part, at * 4, 0, kDeviceScope);
}
__device__ __forceinline__ void put_part(__amdgpu_buffer_rsrc_t part, u32 at, float x, float y) {
  const v2u32 w = {__builtin_bit_cast(u32, x), __builtin_bit_cast(u32, y)};
  __builtin_amdgcn_raw_buffer_store_b64(w, part, at * 4, 0, kDeviceScope);
}
__device__ __forceinline__ f32x4 get_part4(__amdgpu_buffer_rsrc_t part, u32 at) {
  return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(part, at * 4, 0, kDeviceScope));
}
__device__ __forceinline__ v2u32 get_part2(__amdgpu_buffer_rsrc_t part, u32 at) {
  return __builtin_amdgcn_raw_buffer_load_b64(part, at * 4, 0, kDeviceScope);
}
__host__ __device__ inline u32 part_floats(u32 rows, u32 head_dim) { return rows * head_dim + (2 * rows + 3) / 4 * 4; }

// ---- which tokens a workgroup takes -----------------------------------------------------------------
// A row's tokens, in tiles of 32 that begin at multiples of 32.
struct Span {
  u32 first, end;  // tokens seen
  u32 row;
  bool bad;
  __device__ u32 tiles() const { return end > first ? (end + kTile - 1) / kTile - first / kTile : 0; }
};

template <typename A>
__device__ __forceinline__ Span span_of(const A& a, u32 s) {
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

// ---- loads ------------------------------------------------------------------------------------------
// Keys and values that are read once are marked so (two rows of 10^5 tokens: 171 us, marked 154); those of query heads that
// take several workgroups are read by each, and not.
template <int kBytes, int kPolicy>
struct Word;
template <int kPolicy>
struct Word<16, kPolicy> {
  typedef v4u32 type;
  static __device__ type load(__amdgpu_buffer_rsrc_t r, u32 at, u32 plus) {
    return __builtin_amdgcn_raw_buffer_load_b128(r, at, plus, kPolicy);
  }
};
template <int kPolicy>
struct Word<8, kPolicy> {
  typedef v2u32 type;
  static __device__ type load(__amdgpu_buffer_rsrc_t r, u32 at, u32 plus) {
    return __builtin_amdgcn_raw_buffer_load_b64(r, at, plus, kPolicy);
  }
};
template <int kPolicy>
struct Word<4, kPolicy> {
  typedef u32 type;
  static __device__ type load(__amdgpu_buffer_rsrc_t r, u32 at, u32 plus) {
    return __builtin_amdgcn_raw_buffer_load_b32(r, at, plus, kPolicy);
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
template <typename T, bool kF8, int kDim, bool kSmall, int kPolicy>
struct Tile {
  typedef typename T::x8 x8;
  static constexpr int kEs = kF8 ? 1 : 2;
  static constexpr int kLoads = kDim * kEs / 64;          // of 16 bytes a lane and 16 tokens of k
  static constexpr int kSteps = kDim / 32;                // products over 32 elements
  static constexpr int kWide = kDim >= 128 ? 8 : kDim / 16;  // elements of v a lane and token
  static constexpr int kParts = kDim / (16 * kWide);      // of v's row
  typedef typename Word<kWide * kEs, kPolicy>::type vword;
  v4u32 k[2][kLoads];
  vword v[8][kParts];

  // The lane's constant offsets in a page: kNowhere behind head_dim
  struct Lanes {
    u32 col, grp, token_bytes;
    u32 k_at[kLoads], v_at[kParts];
    u64 head;  // bytes
  };

  template <typename A>
  static __device__ __forceinline__ void lanes(const A& a, u32 head, Lanes& z) {
    const u32 l = lane_id(), D = a.d.kv.head_dim;
    z.col = l & 15, z.grp = l >> 4;
    z.token_bytes = (u32)a.d.kv.token_stride * kEs;
    z.head = head * a.d.kv.head_stride * kEs;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const u32 e = (j * 4 + z.grp) * (16 / kEs);
      z.k_at[j] = e < D ? e * kEs + (kSmall ? 0 : z.col * z.token_bytes) : kNowhere;
    }
#pragma unroll
    for (int j = 0; j < kParts; ++j) {
      const u32 e = j * 16 * kWide + z.col * kWide;
      z.v_at[j] = e < D ? e * kEs + (kSmall ? 0 : z.grp * 4 * z.token_bytes) : kNowhere;
    }
  }

  // The pages of tokens [t, t + 32): the wave's two, looked up by scalar loads a tile ahead.  ~0: none to be seen.  Small pages: bits
  // of the half's tokens that are there, once its keys have been asked for
  struct Ids {
    u32 page[2];
  };
  // All 32 tokens' pages (not the tokens) are there
  static __device__ __forceinline__ bool whole(const Ids& ids) {
    return kSmall ? (ids.page[0] & ids.page[1]) == 0xffffu : ids.page[0] != ~0u && ids.page[1] != ~0u;
  }
  template <typename A>
  static __device__ __forceinline__ Ids ids(const A& a, const Span& span, u32 t, bool& bad) {
    Ids r;
    if (kSmall) return r;
    typedef const __attribute__((address_space(4))) u32* table_t;  // no one writes it while the kernel runs
    const table_t table = (table_t)(uintptr_t)(a.d.table + (u64)span.row * a.d.row_pages);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const u32 t0 = t + u * 16;
      r.page[u] = ~0u;
      if (t0 < span.end && t0 + 16 > span.first) {
        const u32 p = table[t0 >> a.page_shift];
        if (p < a.d.kv.n_pages)
          r.page[u] = p;
        else
          bad = true;
      }
    }
    return r;
  }

  template <typename A>
  static __device__ __forceinline__ u64 place(const A& a, const Lanes& z, u32 page, u32 t) {
    return page * a.d.kv.page_stride * kEs + (t & (a.d.kv.page_tokens - 1)) * (u64)z.token_bytes + z.head;
  }
  template <typename A>
  static __device__ __forceinline__ __amdgpu_buffer_rsrc_t half(const A& a, const Lanes& z, const Ids& ids, int u, u32 t,
                                                                const void* pool) {
    return buffer((const uint8_t*)pool + (ids.page[u] != ~0u ? place(a, z, ids.page[u], t + u * 16) : 0), kNowhere - 1);
  }
  // Where a lane finds a token of a small page, or null
  template <typename A>
  static __device__ __forceinline__ const uint8_t* small(const A& a, const Lanes& z, const Span& span, u32 t, const void* pool,
                                                         bool& bad) {
    if (t - span.first >= span.end - span.first) return nullptr;
    const u32 page = (u32)a.d.table[(u64)span.row * a.d.row_pages + (t >> a.page_shift)];
    if (page >= a.d.kv.n_pages) {
      bad = true;
      return nullptr;
    }
    return (const uint8_t*)pool + place(a, z, page, t);
  }

  // Keys, then values of tokens [t, t + 32); those outside the span read as zero (so do all, at a `t` behind it).
  template <typename A>
  __device__ __forceinline__ void load_k(const A& a, const Lanes& z, const Span& span, Ids& ids, u32 t, bool& bad) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const u32 tk = t + u * 16 + z.col;
      if (kSmall) {
        const uint8_t* p = small(a, z, span, tk, a.d.kv.k, bad);
        ids.page[u] = (u32)ballot(p != nullptr) & 0xffffu;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          k[u][j] = 0;
          if (p && z.k_at[j] != kNowhere) k[u][j] = *(const v4u32*)(p + z.k_at[j]);
        }
      } else {
        const auto r = half(a, z, ids, u, t, a.d.kv.k);
        const bool ok = ids.page[u] != ~0u && tk - span.first < span.end - span.first;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) k[u][j] = Word<16, kPolicy>::load(r, ok ? z.k_at[j] : kNowhere, 0);
      }
    }
  }
  template <typename A>
  __device__ __forceinline__ void load_v(const A& a, const Lanes& z, const Span& span, const Ids& ids, u32 t, bool& bad) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const auto r = kSmall ? buffer(nullptr, 0) : half(a, z, ids, u, t, a.d.kv.v);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32 tv = t + u * 16 + z.grp * 4 + i;
        const uint8_t* p = kSmall ? small(a, z, span, tv, a.d.kv.v, bad) : nullptr;
        const bool ok = !kSmall && ids.page[u] != ~0u && tv - span.first < span.end - span.first;
#pragma unroll
        for (int j = 0; j < kParts; ++j) {
          if (kSmall) {
            v[u * 4 + i][j] = 0;
            if (p && z.v_at[j] != kNowhere) v[u * 4 + i][j] = *(const vword*)(p + z.v_at[j]);
          } else {
            v[u * 4 + i][j] = Word<kWide * kEs, kPolicy>::load(r, ok ? z.v_at[j] : kNowhere, i * z.token_bytes);
          }
        }
      }
    }
  }

  // Whether the lane's score i of half u (token t + 16 u + 4 grp + i) has a key.
  template <typename A>
  __device__ __forceinline__ bool seen(const A& a, const Lanes& z, const Span& span, const Ids& ids, u32 t, int u, int i) const {
    if (kSmall) return ids.page[u] >> (z.grp * 4 + i) & 1;
    return t + u * 16 + z.grp * 4 + i - span.first < span.end - span.first && ids.page[u] != ~0u;
  }

  __device__ x8 key(int u, int step) const {
    if (!kF8) return __builtin_bit_cast(x8, k[u][step]);
    const u32 lo = k[u][step / 2][(step & 1) * 2], hi = k[u][step / 2][(step & 1) * 2 + 1];
    const v4u32 w = {widen_f8x2<T, false>(lo), widen_f8x2<T, true>(lo), widen_f8x2<T, false>(hi), widen_f8x2<T, true>(hi)};
    return __builtin_bit_cast(x8, w);
  }

  // Elements 2 e and 2 e + 1 of the lane's piece of v, of its eight tokens: the products' first operand.
  __device__ __forceinline__ void values(int part, int e, x8& even, x8& odd) const {
    v4u32 lo, hi;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (kF8) {  // bytes {x, y, x', y'} of tokens 2 j and 2 j + 1, widened two at a time
        const u32 x = word(v[2 * j][part], e / 2), y = word(v[2 * j + 1][part], e / 2);
        const u32 xy = __builtin_amdgcn_perm(y, x, e & 1 ? 0x07030602u : 0x05010400u);
        lo[j] = widen_f8x2<T, false>(xy), hi[j] = widen_f8x2<T, true>(xy);
      } else {
        const u32 x = word(v[2 * j][part], e), y = word(v[2 * j + 1][part], e);
        lo[j] = __builtin_amdgcn_perm(y, x, 0x05040100u), hi[j] = __builtin_amdgcn_perm(y, x, 0x07060302u);
      }
    }
    even = __builtin_bit_cast(x8, lo), odd = __builtin_bit_cast(x8, hi);
  }
};

}  // namespace fdy
