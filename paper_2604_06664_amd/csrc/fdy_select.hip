// fdy_select.hip - which pages of a long context matter to a step: bounds of every page's keys, scores of the pages from
// them, and the choice of the best.
//
// Between its smallest and largest element low_d and high_d a key's product with q is at most sum_d max(q_d low_d, q_d high_d);
// summed over the query heads of a cache head that is sum_d high_d up_d + low_d down_d with the sums of the positive and of the
// negative elements: one product of 2 head_dim elements for each page, however many query heads there are.  Bounds are read
// once, two operations an element: memory bounds it.
#include <type_traits>

#include "fdy_types.hpp"

using namespace fdy;

namespace {

// Two elements of a word in 32 bits (exact).
template <int kType>
__device__ __forceinline__ void widen2(u32 w, float& a, float& b);
template <>
__device__ __forceinline__ void widen2<FDY_BF16>(u32 w, float& a, float& b) {
  a = __builtin_bit_cast(float, w << 16), b = __builtin_bit_cast(float, w & 0xffff0000u);
}
template <>
__device__ __forceinline__ void widen2<FDY_F16>(u32 w, float& a, float& b) {
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  const f16x2 x = __builtin_bit_cast(f16x2, w);
  a = (float)x[0], b = (float)x[1];
}

// The elements of 16 bytes.
template <int kType>
constexpr int kElems = kType == FDY_F8 ? 16 : 8;
template <int kType>
__device__ __forceinline__ void widen(v4u32 w, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (kType == FDY_F8) {
      typedef float f32x2 __attribute__((ext_vector_type(2)));
      const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], true);
      x[4 * i] = lo[0], x[4 * i + 1] = lo[1], x[4 * i + 2] = hi[0], x[4 * i + 3] = hi[1];
    } else {
      widen2<kType>(w[i], x[2 * i], x[2 * i + 1]);
    }
  }
}
// Back again, of values that came from such elements.
template <int kType>
__device__ __forceinline__ v4u32 narrow(const float* x) {
  v4u32 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (kType == FDY_F8) {
      w[i] = to_f8x4_in_range(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    } else if constexpr (kType == FDY_BF16) {
      const u32 a = __builtin_bit_cast(u32, x[2 * i]), b = __builtin_bit_cast(u32, x[2 * i + 1]);
      w[i] = a >> 16 | (b & 0xffff0000u);
    } else {
      typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
      const f16x2 y = {(_Float16)x[2 * i], (_Float16)x[2 * i + 1]};
      w[i] = __builtin_bit_cast(u32, y);
    }
  }
  return w;
}
inline u32 up_to_power(u32 v) { return v <= 1 ? 1 : 2u << log2_of(v - 1); }

// Row and length of a sequence, held within what there is.
template <typename D>
__device__ __forceinline__ u32 tokens_of(const D& d, u32 s, u32 shift, u32& row, bool& bad) {
  row = d.rows ? (u32)d.rows[s] : s;
  if (row >= d.n_rows) {
    bad = true, row = 0;
    return 0;
  }
  const int n = d.lens[row];
  const u32 most = d.row_pages << shift;
  if (n >= 0 && (u32)n <= most) return (u32)n;
  bad = true;
  return n < 0 ? 0 : most;
}

// ---- bounds -----------------------------------------------------------------------------------------
struct BoundsArg {
  fdy_bounds d;
  u32* status;
  u32 shift, lanes, slots, fill;  // lanes: of 16 bytes a token's head, up to a power of two; slots: pages of a sequence at most
};
typedef Arg<BoundsArg> Bounds;

// A wave takes one head of one page: 64 / lanes tokens at a time, kAhead loads of a lane under way, then the lanes that hold the same
// elements of different tokens are joined.  Tokens behind the last are the last once more.  Memory bounds it: prompts of 131,000 tokens, 8
// heads of 128, 53 us, 5.0 TB/s (again over the same 267 MB, part of which the card's cache then holds, 43); a step of 256 rows 4.4, a
// launch and two dependent loads.
template <int kType>
__global__ void __launch_bounds__(256) bounds_kernel(Bounds a) {
  constexpr int kE = kElems<kType>, kAhead = 4;
  constexpr u32 kEs = kType == FDY_F8 ? 1 : 2;
  const u32 s = blockIdx.x, H = a.d.kv.n_heads, D = a.d.kv.head_dim, pt = a.d.kv.page_tokens;
  bool bad = false;
  u32 row;
  const u32 n = uniform(tokens_of(a.d, s, a.shift, row, bad));
  int fresh = a.d.fresh ? a.d.fresh[s] : 1;
  if (a.d.fresh && (fresh < 0 || (u32)fresh > a.d.max_fresh)) bad = true, fresh = fresh < 0 ? 0 : (int)a.d.max_fresh;
  const u32 begin = n - min((u32)fresh, n), first = begin >> a.shift;
  const u32 pages = uniform(begin < n ? ((n - 1) >> a.shift) - first + 1 : 0);
  const u32 lane = lane_id() & (a.lanes - 1), at = lane_id() / a.lanes, step = 64 / a.lanes;
  const u32 e = lane * kE < D ? lane * kE : 0;
  for (u32 u = blockIdx.y * 4 + (threadIdx.x >> 6); u < pages * H; u += gridDim.y * 4) {
    const u32 j = uniform(first + u / H), h = uniform(u % H), page = (u32)a.d.table[(u64)row * a.d.row_pages + j];
    if (page >= a.d.kv.n_pages) {
      bad = true;
      continue;
    }
    const u32 held = min(pt, n - (j << a.shift));
    const uint8_t* k = (const uint8_t*)a.d.kv.k + (page * a.d.kv.page_stride + h * a.d.kv.head_stride + e) * kEs;
    const u64 token = a.d.kv.token_stride * kEs;
    float low[kE], high[kE];
#pragma unroll
    for (int i = 0; i < kE; ++i) low[i] = INFINITY, high[i] = -INFINITY;
    for (u32 t0 = 0; t0 < held; t0 += step * kAhead) {
      v4u32 w[kAhead];
#pragma unroll
      for (u32 g = 0; g < kAhead; ++g) w[g] = *(const v4u32*)(k + min(t0 + g * step + at, held - 1) * token);
#pragma unroll
      for (u32 g = 0; g < kAhead; ++g) {
        float x[kE];
        widen<kType>(w[g], x);
#pragma unroll
        for (int i = 0; i < kE; ++i)
          low[i] = __builtin_elementwise_minimum(low[i], x[i]), high[i] = __builtin_elementwise_maximum(high[i], x[i]);
      }
    }
    for (u32 m = a.lanes; m < 64; m *= 2) {
#pragma unroll
      for (int i = 0; i < kE; ++i) {
        low[i] = __builtin_elementwise_minimum(low[i], __shfl_xor(low[i], m));
        high[i] = __builtin_elementwise_maximum(high[i], __shfl_xor(high[i], m));
      }
    }
    uint8_t* out = (uint8_t*)a.d.bounds + (((u64)page * H + h) * 2 * D + e) * kEs;
    if (at == 0 && lane * kE < D) {
      *(v4u32*)out = narrow<kType>(low);
      *(v4u32*)(out + D * kEs) = narrow<kType>(high);
    }
  }
  if (bad && lane_id() == 0) raise_status(a.status, FDY_ST_BAD_INDEX);
}

// ---- scores -----------------------------------------------------------------------------------------
struct SelectArg {
  fdy_select d;
  u32* status;
  u64* keys;  // [n_seqs][heads][row_pages]: the scores, as integers in their order
  u32 shift, group, lanes, head_blocks;  // lanes: of 16 bytes a page's bounds of a head, up to a power of two
};
typedef Arg<SelectArg> Select;

__device__ __forceinline__ u64 key_of(double x) {
  const u64 v = __builtin_bit_cast(u64, x);
  if (x != x) return ~0ull;
  return v >> 63 ? ~v : v | 1ull << 63;
}
constexpr u64 kNoKey = 0x000fffffffffffffull;  // of a page that is none: minus infinity's

template <int kCtrl, int kRows = 0xf>
__device__ __forceinline__ double plus_dpp(double x) {
  const u64 v = __builtin_bit_cast(u64, x);
  return x + __builtin_bit_cast(double, dpp<kCtrl, kRows>(v, (u64)0));
}

// A row's pages in chunks, for each block of heads one after the other: a line through all rows that have more pages than are
// chosen, of which every workgroup takes an equal share, whatever the rows' lengths are.
constexpr u32 kPages = 8;           // of a wave, under way together
constexpr u32 kChunk = 4 * kPages;  // of a workgroup
template <int kType>
constexpr u32 kResident = kType == FDY_F8 ? 2 : 4;  // workgroups of a compute unit
struct Place {
  u32 s, row, pages, chunks, block, chunk;
};

// The row of a sequence, in units of the line.
__device__ __forceinline__ u32 units_of(const Select& a, u32 s, u32& row, u32& pages, bool& bad) {
  pages = (tokens_of(a.d, s, a.shift, row, bad) + a.d.kv.page_tokens - 1) >> a.shift;
  return pages > a.d.budget ? (pages + kChunk - 1) / kChunk * a.head_blocks : 0;
}
__device__ __forceinline__ void go_to(const Select& a, u32 s, u32 unit, Place& p) {
  bool bad = false;
  p.s = s;
  units_of(a, s, p.row, p.pages, bad);
  p.row = uniform(p.row), p.pages = uniform(p.pages);
  p.chunks = (p.pages + kChunk - 1) / kChunk, p.block = unit / p.chunks, p.chunk = unit - p.block * p.chunks;
}

// All threads of a workgroup of four waves: its first unit, and how many.
__device__ __forceinline__ u32 find_units(const Select& a, Place& p) {
  __shared__ u64 s_sum[4];
  __shared__ u32 s_seq, s_unit;
  const u32 n = a.d.n_seqs, tid = threadIdx.x, slice = (n + 255) / 256, s0 = min(tid * slice, n), s1 = min(s0 + slice, n);
  u64 mine = 0;
  bool bad = false;
  u32 row, pages;
  for (u32 s = s0; s < s1; ++s) mine += units_of(a, s, row, pages, bad);
  if (bad && blockIdx.x == 0) raise_status(a.status, FDY_ST_BAD_INDEX);
  const u64 inc = wave_incl_scan(mine);
  if (lane_id() == 63) s_sum[tid >> 6] = inc;
  __syncthreads();
  u64 before = inc - mine, total = 0;
#pragma unroll
  for (u32 w = 0; w < 4; ++w) {
    if (w < tid >> 6) before += s_sum[w];
    total += s_sum[w];
  }
  const u64 per = (total + gridDim.x - 1) / gridDim.x, begin = blockIdx.x * per;
  if (begin >= total) return 0;
  if (begin >= before && begin < before + mine) {
    u32 s = s0;
    u64 at = begin - before;
    for (;; ++s) {
      const u32 units = units_of(a, s, row, pages, bad);
      if (at < units) break;
      at -= units;
    }
    s_seq = s, s_unit = (u32)at;
  }
  __syncthreads();
  go_to(a, uniform(s_seq), uniform(s_unit), p);
  return (u32)min(per, total - begin);
}

// A wave's pages of a chunk: their numbers, looked up by scalar loads, and their bounds.
struct Pages {
  u32 page[kPages];
  __device__ __forceinline__ void load(const Select& a, const Place& p, u32 wave) {
    typedef const __attribute__((address_space(4))) u32* table_t;  // no one writes it while the kernel runs
    const table_t table = (table_t)(uintptr_t)(a.d.table + (u64)p.row * a.d.row_pages);
#pragma unroll
    for (u32 i = 0; i < kPages; ++i) page[i] = table[min(p.chunk * kChunk + wave * kPages + i, p.pages - 1)];
  }
};
template <int kType>
struct Chunk {
  v4u32 w[kPages];
  u32 none;  // bits of pages that are none
  __device__ __forceinline__ void load(const Select& a, const Pages& p, u32 head, u32 at) {
    const u32 H = a.d.kv.n_heads, of_head = 2 * a.d.kv.head_dim * (kType == FDY_F8 ? 1 : 2);
    none = 0;
#pragma unroll
    for (u32 i = 0; i < kPages; ++i) {
      if (p.page[i] >= a.d.kv.n_pages) none |= 1u << i;
      w[i] = 0;
      if (head < H && at < of_head && p.page[i] < a.d.kv.n_pages)
        w[i] = *(const v4u32*)((const uint8_t*)a.d.bounds + ((u64)p.page[i] * H + head) * of_head + at);
    }
  }
};

// Sums over a group of lanes.  From 16 lanes on of four pages at once: neighbours exchange what they do not go on with, so that lane
// l has page l % 4 of its four, then the fours are added; the sum that counts, of lanes 12 to 15 of each 16, is formed in the same
// order for every page.  Smaller groups: of one page, the last lane's counts.
__device__ __forceinline__ double choose(bool c, double x, double y) { return c ? x : y; }
__device__ __forceinline__ double sum4(double x0, double x1, double x2, double x3, u32 lanes) {
  const u32 l = lane_id();
  const bool odd = l & 1, two = l & 2;
  constexpr int kXor1 = 0xb1, kXor2 = 0x4e, kRor4 = 0x124, kRor8 = 0x128;
  auto from = [](auto ctrl, double x) {
    return __builtin_bit_cast(double, dpp<decltype(ctrl)::value>(__builtin_bit_cast(u64, x), (u64)0));
  };
  const double p = choose(odd, x1, x0) + from(std::integral_constant<int, kXor1>(), choose(odd, x0, x1));
  const double q = choose(odd, x3, x2) + from(std::integral_constant<int, kXor1>(), choose(odd, x2, x3));
  double r = choose(two, q, p) + from(std::integral_constant<int, kXor2>(), choose(two, p, q));
  r += from(std::integral_constant<int, kRor4>(), r);
  r += from(std::integral_constant<int, kRor8>(), r);
  auto halves = [](auto swap, double x) {
    const u64 v = __builtin_bit_cast(u64, x);
    const auto lo = swap((u32)v), hi = swap((u32)(v >> 32));
    const u32 lo0 = lo[0], lo1 = lo[1], hi0 = hi[0], hi1 = hi[1];
    return __builtin_bit_cast(double, pair64(lo0, hi0)) + __builtin_bit_cast(double, pair64(lo1, hi1));
  };
  if (lanes > 16) r = halves([](u32 v) { return __builtin_amdgcn_permlane16_swap(v, v, false, false); }, r);
  if (lanes > 32) r = halves([](u32 v) { return __builtin_amdgcn_permlane32_swap(v, v, false, false); }, r);
  return r;
}
__device__ __forceinline__ double sum1(double x, u32 lanes) {
  x = plus_dpp<kShr1>(x);
  if (lanes > 2) x = plus_dpp<kShr2>(x);
  if (lanes > 4) x = plus_dpp<kShr4>(x);
  return x;
}

// A wave takes 64 / lanes heads and kPages pages at a time, the next ones asked for ahead.  A lane's 8 (16) factors stay in
// registers, in 64 bits; where one is 0 the element is made 0, whatever it is.  8,192 pages of 8 heads 12 us (34 MB, half of it start and
// end); 96 rows of up to 4,096 pages in 8 bits 56 us, 3.7 TB/s, where widening twice and adding up in 64 bits weigh as much as the loads.
template <typename T, int kType>
__global__ void __launch_bounds__(256, kResident<kType>) scores_kernel(Select a) {
  constexpr int kE = kElems<kType>, kQ = T::kType;
  __shared__ double s_f[4][kE][64];
  const u32 H = a.d.kv.n_heads, D = a.d.kv.head_dim, wave = uniform(threadIdx.x >> 6), l = lane_id();
  const u32 piece = l & (a.lanes - 1), of_block = 64 / a.lanes, in_block = l / a.lanes;
  const bool high = piece * kE >= D;
  Place p;
  u32 units = find_units(a, p);
  if (!units) return;
  // the bounds of the next unit are asked for ahead of this one's sums, and the page numbers of the one behind it
  auto follow = [&](Place& p) {
    if (++p.chunk < p.chunks) return;
    p.chunk = 0;
    if (++p.block < a.head_blocks) return;
    u32 s = p.s, row, pages;
    bool bad = false;
    do ++s;
    while (s < a.d.n_seqs && !uniform(units_of(a, s, row, pages, bad)));
    if (s < a.d.n_seqs) go_to(a, s, 0, p);
  };
  Pages pages;
  pages.load(a, p, wave);
  Chunk<kType> now;
  now.load(a, pages, p.block * of_block + in_block, piece * 16);
  Place then = p;
  if (units > 1) follow(then), pages.load(a, then, wave);
  u32 last_s = ~0u, last_block = 0;
  double f[kE];
  v4u32 keep = 0;
  for (;;) {
    const u32 head = p.block * of_block + in_block;
    if (p.s != last_s || p.block != last_block) {
      last_s = p.s, last_block = p.block;
      keep = 0;
#pragma unroll
      for (int i = 0; i < kE; ++i) f[i] = 0;
      if (head < H && piece * kE < 2 * D) {  // a wave every fourth query head, two of them asked for at once
        const double k_scale = kType == FDY_F8 && a.d.kv.k_scale ? (double)a.d.kv.k_scale[head] : 1.0;
        const char* q = (const char*)a.d.q + (p.s * a.d.q_seq + head * a.group * a.d.q_head + piece * kE - (high ? D : 0)) * 2;
        for (u32 g = wave; g < a.group; g += 8) {
          v4u32 y[2][kE / 8];
#pragma unroll
          for (u32 k = 0; k < 2; ++k)
#pragma unroll
            for (int h = 0; h < kE / 8; ++h) {
              y[k][h] = 0;
              if (g + 4 * k < a.group) y[k][h] = *(const v4u32*)(q + ((g + 4 * k) * a.d.q_head + h * 8) * 2);
            }
#pragma unroll
          for (u32 k = 0; k < 2; ++k)
#pragma unroll
            for (int h = 0; h < kE / 8; ++h) {
              float z[8];
              widen<kQ>(y[k][h], z);
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const double x = (double)z[i] * k_scale;
                f[h * 8 + i] += (high ? x > 0 : x < 0) ? x : 0.0;
              }
            }
        }
      }
      __syncthreads();  // the sums before have been read
#pragma unroll
      for (int i = 0; i < kE; ++i) s_f[wave][i][l] = f[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kE; ++i) {
        f[i] = s_f[0][i][l] + s_f[1][i][l] + (s_f[2][i][l] + s_f[3][i][l]);
        if (f[i] != 0) keep[i / (kE / 4)] |= (kType == FDY_F8 ? 0xffu : 0xffffu) << i % (kE / 4) * (32 / (kE / 4));
      }
    }
    const Place at = p;
    Chunk<kType> next;
    if (--units) {
      next.load(a, pages, then.block * of_block + in_block, piece * 16);
      p = then;
      if (units > 1) follow(then), pages.load(a, then, wave);
    }
    const u32 p0 = at.chunk * kChunk + wave * kPages;
    double sum[kPages];
#pragma unroll
    for (u32 i = 0; i < kPages; ++i) {
      float x[kE];
      widen<kType>(now.w[i] & keep, x);
      sum[i] = 0;
#pragma unroll
      for (int k = 0; k < kE; ++k) sum[i] = __builtin_fma(f[k], (double)x[k], sum[i]);
    }
    u64* keys = a.keys + ((u64)at.s * H + head) * a.d.row_pages + p0;
    if (a.lanes >= 16) {
#pragma unroll
      for (u32 i = 0; i < kPages; i += 4) {
        const u64 key = key_of(sum4(sum[i], sum[i + 1], sum[i + 2], sum[i + 3], a.lanes));
        const u32 mine = i + (l & 3);
        if (head < H && piece >= 12 && piece < 16 && p0 + mine < at.pages) keys[mine] = now.none >> mine & 1 ? kNoKey : key;
      }
    } else {
#pragma unroll
      for (u32 i = 0; i < kPages; ++i) {
        const u64 key = key_of(sum1(sum[i], a.lanes));
        if (head < H && piece == a.lanes - 1 && p0 + i < at.pages) keys[i] = now.none >> i & 1 ? kNoKey : key;
      }
    }
    if (now.none && l == 0) raise_status(a.status, FDY_ST_BAD_INDEX);
    if (!units) return;
    now = next;
  }
}

// ---- choice -----------------------------------------------------------------------------------------
// One workgroup for a cache head of a sequence: the key that the last one taken has, ten bits at a time from the highest in which
// the keys differ, then those above it and as many of those equal to it as there is room for, in the order of the row.
// kMine: keys that a thread holds in registers, every kThreads-th of the row; 0: keys are read again from the workspace, for tables
// of more pages (rows' lengths are not known at the launch).  8,192 pages of 8 heads 13 us: a chain of two or three turns, three barriers each;
// 768 lists of 4,096 pages 13.  Scores and choice of 8,192 pages under a table of 16,384 23 us, of 16,385 39.
constexpr u32 kThreads = 512, kWaves = kThreads / 64, kBits = 10, kBins = 1u << kBits;
template <u32 kMine>
__global__ void __launch_bounds__(kThreads) choice_kernel(Select a) {
  __shared__ u64 s_low, s_high, s_scan[17];
  __shared__ alignas(16) u32 s_bins[2][kBins];
  constexpr u32 kRanks = (kMine * kWaves + 63) / 64 * 64;  // a whole number of every lane's, of which those behind the last count nothing
  __shared__ u32 s_bin, s_above, s_here, s_ranks[kRanks + 1];
  __shared__ u64 s_words[kMine * kWaves + 1];
  const u32 H = a.d.kv.n_heads, s = blockIdx.x / H, g = blockIdx.x % H, tid = threadIdx.x, budget = a.d.budget;
  const u32 wave = tid >> 6, l = lane_id();
  bool bad = false;
  u32 row;
  const u32 n = uniform(tokens_of(a.d, s, a.shift, row, bad)), pages = (n + a.d.kv.page_tokens - 1) >> a.shift;
  const u32 taken = min(pages, budget);
  const int32_t* table = a.d.table + (u64)row * a.d.row_pages;
  int32_t* out = a.d.pages + (u64)blockIdx.x * budget;
  if (g == 0 && tid == 0) a.d.seen[s] = (int32_t)(n - ((pages - taken) << a.shift));
  for (u32 i = taken + tid; i < budget; i += kThreads) out[i] = -1;
  if (pages <= budget) {
    for (u32 j = tid; j < pages; j += kThreads) {
      out[j] = table[j];
      if ((u32)table[j] >= a.d.kv.n_pages) bad = true;
    }
    if (bad) raise_status(a.status, FDY_ST_BAD_INDEX);
    return;
  }
  const u32 sinks = a.d.sinks, recent = a.d.recent, end = pages - recent;
  u32 left = budget - sinks - recent;  // to be taken of [sinks, end), which are more
  const u64* keys = a.keys + (u64)blockIdx.x * a.d.row_pages;
  u64 mine[kMine ? kMine : 1];
#pragma unroll
  for (u32 i = 0; i < kMine; ++i) {
    const u32 j = sinks + i * kThreads + tid;
    mine[i] = j < end ? keys[j] : 0;
  }
  for (u32 i = tid; i < sinks; i += kThreads) out[i] = table[i];
  for (u32 i = tid; i < recent; i += kThreads) out[budget - recent + i] = table[end + i];
  if (left == 0) return;
  auto each = [&](auto f) {  // f(key), of the thread's
    if constexpr (kMine > 0) {
#pragma unroll
      for (u32 i = 0; i < kMine; ++i)
        if (sinks + i * kThreads < end && sinks + i * kThreads + tid < end) f(mine[i]);
    } else {
      for (u32 j = sinks + tid; j < end; j += kThreads) f(keys[j]);
    }
  };
  auto ranks_ahead = [&] {  // s_ranks, each the sum of those ahead of it
    __syncthreads();
    constexpr u32 kOf = kRanks / 64;
    if (wave == 0) {
      u32 c[kOf + 1], sum = 0;
#pragma unroll
      for (u32 i = 0; i < kOf; ++i) c[i] = s_ranks[l * kOf + i], sum += c[i];
      u32 before = wave_incl_scan(sum) - sum;
#pragma unroll
      for (u32 i = 0; i < kOf; ++i) s_ranks[l * kOf + i] = before, before += c[i];
    }
    __syncthreads();
  };
  if (tid == 0) s_low = ~0ull, s_high = 0, s_here = end - sinks;
  for (u32 i = tid; i < 2 * kBins; i += kThreads) s_bins[0][i] = 0;
  __syncthreads();
  u64 low = ~0ull, high = 0;
  each([&](u64 key) { low = min(low, key), high = max(high, key); });
  low = ~wave_incl_most(~low), high = wave_incl_most(high);
  if (l == 63) atomicMin((unsigned long long*)&s_low, low), atomicMax((unsigned long long*)&s_high, high);
  __syncthreads();
  // All of the search is the workgroup's own and stays in scalar registers.  (Not only for speed: with its amounts of shifts in vector
  // registers the variant that reads keys again had one in the last of 64, and there v_lshlrev_b64 took another register's value.)
  low = uniform(s_low), high = uniform(s_high) - low;
  // of the keys less `low` those from `bound` + 2^shift on are taken, and of those from `bound` on `left`
  u32 shift = high ? 64 - (u32)__builtin_clzll(high) : 0;
  u64 bound = 0;
  for (u32 turn = 0; shift; turn ^= 1) {
    const u32 bits = min(shift, kBits), below = shift - bits;
    each([&](u64 key) {
      const u64 x = key - low - bound;  // (those below the bound wrap round)
      if (shift == 64 || !(x >> shift)) atomicAdd(&s_bins[turn][(u32)(x >> below)], 1u);
    });
    __syncthreads();
    if (wave == 0) {  // kBins / 64 neighbouring bins a lane, the highest in the first
      constexpr u32 kOf = kBins / 64;
      u32 c[kOf], sum = 0;
#pragma unroll
      for (u32 i = 0; i < kOf; ++i) c[i] = s_bins[turn][(63 - l) * kOf + i], sum += c[i];
      u32 above = wave_incl_scan(sum) - sum;
#pragma unroll
      for (u32 i = kOf; i-- > 0;) {
        if (above < left && above + c[i] >= left) s_bin = (63 - l) * kOf + i, s_above = above, s_here = c[i];
        above += c[i];
      }
    } else {
      for (u32 i = tid - 64; i < kBins; i += kThreads - 64) s_bins[turn ^ 1][i] = 0;
    }
    __syncthreads();
    left -= uniform(s_above);
    bound += (u64)uniform(s_bin) << below;
    shift = below;
    if (uniform(s_here) == left) break;  // all that have these bits are taken
  }
  // (what the next turn writes to s_bin it writes behind a barrier that all have come to)
  const bool some = uniform(s_here) != left;  // of those equal
  bound += low;
  // (a difference, for bound + 2^shift may lie behind the last of all keys)
  auto above = [&](u64 key) { return key >= bound && (key - bound) >> shift; };
  auto equal = [&](u64 key) { return key >= bound && !((key - bound) >> shift); };
  if constexpr (kMine > 0) {
    // a bit for each page that is taken, with the sums ahead of each word; then every place of the list looks for its page
    u32 rank = 0;
    if (some) {
#pragma unroll
      for (u32 i = 0; i < kMine; ++i) {
        const u32 c = (u32)__popcll(ballot(sinks + i * kThreads + tid < end && equal(mine[i])));
        if (l == i) rank = c;
      }
      if (l < kMine) s_ranks[l * kWaves + wave] = rank;
      ranks_ahead();
    }
    u64 word = 0;
#pragma unroll
    for (u32 i = 0; i < kMine; ++i) {
      bool take = sinks + i * kThreads + tid < end && mine[i] >= bound;
      if (some) {
        const bool e = take && equal(mine[i]);
        const u32 at = s_ranks[i * kWaves + wave] + (u32)__popcll(ballot(e) & lanemask_lt());
        take = take && (!e || at < left);
      }
      const u64 taken_here = ballot(take);
      if (l == i) word = taken_here;
    }
    __syncthreads();
    if (l < kMine) s_words[l * kWaves + wave] = word, s_ranks[l * kWaves + wave] = (u32)__popcll(word);
    ranks_ahead();
    for (u32 k = tid; k < budget - sinks - recent; k += kThreads) {
      u32 at = 0;  // the last word with no more than k ahead of it
#pragma unroll
      for (u32 m = kMine * kWaves / 2; m; m /= 2)
        if (s_ranks[at + m] <= k) at += m;
      u64 bits = s_words[at];
      u32 r = k - s_ranks[at], bit = 0;  // its bit number r
#pragma unroll
      for (u32 m = 32; m; m /= 2) {
        const u32 c = (u32)__popcll(bits & ((1ull << m) - 1));
        if (r >= c) r -= c, bits >>= m, bit += m;
      }
      out[sinks + k] = table[sinks + at * 64 + bit];
    }
  } else {
    u64 before = 0;  // those above in the low half, those equal in the high
    for (u32 j0 = sinks; j0 < end; j0 += kThreads) {
      const u32 j = j0 + tid;
      const u64 key = j < end ? keys[j] : 0, x = j < end ? (above(key) ? 1ull : equal(key) ? 1ull << 32 : 0) : 0;
      u64 sum;
      const u64 rank = before + block_excl_scan(x, s_scan, sum);
      before += sum;
      const u32 equals = (u32)(rank >> 32);
      const u32 at = (u32)rank + min(equals, left);
      // (keys are read twice here: whatever became of them meanwhile, nothing is written behind the list)
      if ((x == 1 || (x && equals < left)) && at < budget - sinks - recent) out[sinks + at] = table[j];
    }
  }
}

template <typename F, typename A>
int go(F kernel, dim3 grid, u32 threads, void* stream, const A& a) {
  (void)hipGetLastError();  // drop any stale error left by earlier, unrelated runtime calls
  hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, (hipStream_t)stream, a);
  FDY_HIP_TRY(hipGetLastError());
  return FDY_OK;
}

// Pages of a sequence that have new tokens, at most.
u32 slots_of(const fdy_bounds& d) {
  const u32 fresh = d.fresh && d.max_fresh ? d.max_fresh : 1, slots = (fresh - 1) / d.kv.page_tokens + 2;
  return slots < d.row_pages ? slots : d.row_pages ? d.row_pages : 1;
}

bool bounds_valid(const fdy_bounds& d) {
  if (!kv_valid(d.kv) || d.n_seqs > 65536u || (u64)d.row_pages * d.kv.page_tokens >> 31) return false;
  if ((u64)slots_of(d) * d.kv.n_heads >> 31) return false;
  const u32 per = d.kv.type == FDY_F8 ? 16 : 8;
  return d.kv.head_dim % per == 0 && (d.kv.page_stride | d.kv.token_stride | d.kv.head_stride) % per == 0;
}

bool select_valid(const fdy_select& d) {
  fdy_kv kv = d.kv;
  kv.page_stride = kv.token_stride = kv.head_stride = 0;  // not read
  if (!kv_valid(kv) || d.type > FDY_F16 || d.n_seqs > 65536u || (u64)d.row_pages * kv.page_tokens >> 31) return false;
  if (kv.head_dim % (kv.type == FDY_F8 ? 16 : 8)) return false;
  if (!d.n_q_heads || d.n_q_heads > 65536u || d.n_q_heads % kv.n_heads || (u64)d.n_seqs * d.n_q_heads > 1u << 22) return false;
  if (!d.recent || (u64)d.sinks + d.recent > d.budget || d.budget > 1u << 25) return false;
  return (u64)d.n_seqs * kv.n_heads * d.row_pages <= 1ull << 32 && (kv.type == d.type || kv.type == FDY_F8);
}

}  // namespace

extern "C" int fdy_page_bounds(const fdy_bounds* h, uint32_t* d_status, void* stream) {
  if (!h || !bounds_valid(*h)) return FDY_ERR_INVALID_ARG;
  const fdy_bounds& d = *h;
  if (d.n_seqs == 0) return FDY_OK;
  if (!d.bounds || !d.table || !d.lens || !d.kv.k) return FDY_ERR_INVALID_ARG;
  if (!aligned(d.bounds, 16) || !aligned(d.kv.k, 16) || !aligned(d.table, 4) || !aligned(d.lens, 4) || !aligned(d.rows, 4) ||
      !aligned(d.fresh, 4))
    return FDY_ERR_INVALID_ARG;
  Bounds a{};
  a.d = d;
  a.status = d_status;
  a.shift = log2_of(d.kv.page_tokens);
  a.lanes = up_to_power(d.kv.head_dim / (d.kv.type == FDY_F8 ? 16 : 8));
  a.slots = slots_of(d);
  const u64 blocks = ((u64)a.slots * d.kv.n_heads + 3) / 4;
  const dim3 grid(d.n_seqs, (u32)(blocks < 32768 ? blocks : 32768));
  if (d.kv.type == FDY_BF16) return go(bounds_kernel<FDY_BF16>, grid, 256, stream, a);
  if (d.kv.type == FDY_F16) return go(bounds_kernel<FDY_F16>, grid, 256, stream, a);
  return go(bounds_kernel<FDY_F8>, grid, 256, stream, a);
}

extern "C" size_t fdy_page_select_workspace_bytes(const fdy_select* h) {
  if (!h || !select_valid(*h)) return 0;
  const size_t bytes = (size_t)h->n_seqs * h->kv.n_heads * h->row_pages * 8;
  return (bytes + 255) / 256 * 256 + 256;
}

extern "C" int fdy_page_select(const fdy_select* h, void* d_workspace, size_t workspace_bytes, uint32_t* d_status, void* stream) {
  if (!h || !select_valid(*h)) return FDY_ERR_INVALID_ARG;
  const fdy_select& d = *h;
  if (d.n_seqs == 0) return FDY_OK;
  if (!d.q || !d.bounds || !d.table || !d.lens || !d.pages || !d.seen) return FDY_ERR_INVALID_ARG;
  if (!aligned(d.q, 16) || !aligned(d.bounds, 16) || !aligned(d.table, 4) || !aligned(d.lens, 4) || !aligned(d.rows, 4) ||
      !aligned(d.pages, 4) || !aligned(d.seen, 4) || !aligned(d.kv.k_scale, 4) || (d.q_seq | d.q_head) % 8)
    return FDY_ERR_INVALID_ARG;
  if (!d_workspace || !aligned(d_workspace, 256) || workspace_bytes < fdy_page_select_workspace_bytes(h)) return FDY_ERR_WORKSPACE;
  Select a{};
  a.d = d;
  a.status = d_status;
  a.keys = (u64*)d_workspace;
  a.shift = log2_of(d.kv.page_tokens);
  a.group = d.n_q_heads / d.kv.n_heads;
  a.lanes = up_to_power(2 * d.kv.head_dim / (d.kv.type == FDY_F8 ? 16 : 8));
  a.head_blocks = (d.kv.n_heads + 64 / a.lanes - 1) / (64 / a.lanes);
  if (d.row_pages > d.budget) {
    // as many workgroups as the card holds (or as there can be units)
    const u64 units = (u64)d.n_seqs * ((d.row_pages + kChunk - 1) / kChunk) * a.head_blocks;
    const u64 most = 256 * (d.kv.type == FDY_F8 ? kResident<FDY_F8> : kResident<FDY_BF16>);
    const dim3 grid((u32)(units < most ? units : most));
    int rc;
    if (d.type == FDY_BF16)
      rc = d.kv.type == FDY_F8 ? go(scores_kernel<Bf16, FDY_F8>, grid, 256, stream, a) : go(scores_kernel<Bf16, FDY_BF16>, grid, 256, stream, a);
    else
      rc = d.kv.type == FDY_F8 ? go(scores_kernel<F16, FDY_F8>, grid, 256, stream, a) : go(scores_kernel<F16, FDY_F16>, grid, 256, stream, a);
    if (rc != FDY_OK) return rc;
  }
  const dim3 grid(d.n_seqs * d.kv.n_heads);
  if (d.row_pages <= kThreads * 4) return go(choice_kernel<4>, grid, kThreads, stream, a);
  if (d.row_pages <= kThreads * 16) return go(choice_kernel<16>, grid, kThreads, stream, a);
  if (d.row_pages <= kThreads * 32) return go(choice_kernel<32>, grid, kThreads, stream, a);
  return go(choice_kernel<0>, grid, kThreads, stream, a);
}
