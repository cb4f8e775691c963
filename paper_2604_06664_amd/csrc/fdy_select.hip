// fdy_select.hip - which pages of a long context matter to a step: bounds of every page's keys, scores of the pages from
// them, and the choice of the best.
//
// Between its smallest and largest element low_d and high_d a key's product with q is at most sum_d max(q_d low_d, q_d high_d);
// summed over the query heads of a cache head that is sum_d high_d up_d + low_d down_d with the sums of the positive and of the
// negative elements: one product of 2 head_dim elements for each page, however many query heads there are.  Bounds are read
// once, two operations an element: memory bounds it.
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
// elements of different tokens are joined.  Tokens behind the last are the last once more.
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

// The element of q (type of the queries) as 64 bits.
template <typename T>
__device__ __forceinline__ double element(const void* q, u64 at) {
  return (double)(float)((const typename T::elem*)q)[at];
}

// A wave takes 64 / lanes heads and every fourth page of the workgroup's.  A lane's 8 (16) factors stay in registers.
constexpr u32 kPages = 8;           // of a wave, loads under way together
constexpr u32 kChunk = 4 * kPages * 2;  // pages of a workgroup
template <typename T, int kType>
__global__ void __launch_bounds__(256) scores_kernel(Select a) {
  constexpr int kE = kElems<kType>;
  constexpr u32 kEs = kType == FDY_F8 ? 1 : 2;
  const u32 s = blockIdx.x, H = a.d.kv.n_heads, D = a.d.kv.head_dim, wave = threadIdx.x >> 6, l = lane_id();
  bool bad = false;
  u32 row;
  const u32 n = uniform(tokens_of(a.d, s, a.shift, row, bad)), pages = (n + a.d.kv.page_tokens - 1) >> a.shift;
  if (bad && blockIdx.y == 0 && threadIdx.x == 0) raise_status(a.status, FDY_ST_BAD_INDEX);
  if (pages <= a.d.budget) return;
  bad = false;
  const u32 chunks = (pages + kChunk - 1) / kChunk;
  u32 last_block = ~0u;
  double f[kE];
  for (u32 b = blockIdx.y; b < chunks * a.head_blocks; b += gridDim.y) {
    const u32 block = b % a.head_blocks, chunk = b / a.head_blocks;
    const u32 head = block * (64 / a.lanes) + l / a.lanes, piece = l & (a.lanes - 1);
    const bool works = head < H && piece * kE < 2 * D;
    const bool high = piece * kE >= D;
    if (block != last_block) {
      last_block = block;
#pragma unroll
      for (int i = 0; i < kE; ++i) f[i] = 0;
      if (works) {
        const double k_scale = kType == FDY_F8 && a.d.kv.k_scale ? (double)a.d.kv.k_scale[head] : 1.0;
        for (u32 g = 0; g < a.group; ++g) {
          const u64 at = s * a.d.q_seq + (head * a.group + g) * a.d.q_head + piece * kE - (high ? D : 0);
#pragma unroll
          for (int i = 0; i < kE; ++i) {
            const double x = element<T>(a.d.q, at + i) * k_scale;
            if (high ? x > 0 : x < 0) f[i] += x;
          }
        }
      }
    }
    for (u32 p0 = chunk * kChunk + wave * kPages; p0 < min(pages, (chunk + 1) * kChunk); p0 += 4 * kPages) {
      v4u32 w[kPages];
      bool none[kPages];
#pragma unroll
      for (u32 i = 0; i < kPages; ++i) {
        const u32 j = min(p0 + i, pages - 1), page = (u32)a.d.table[(u64)row * a.d.row_pages + j];
        none[i] = page >= a.d.kv.n_pages;
        w[i] = 0;
        if (works && !none[i]) w[i] = *(const v4u32*)((const uint8_t*)a.d.bounds + ((u64)page * H + head) * 2 * D * kEs + piece * 16);
      }
#pragma unroll
      for (u32 i = 0; i < kPages; ++i) {
        float x[kE];
        widen<kType>(w[i], x);
        double sum = 0;
#pragma unroll
        for (int k = 0; k < kE; ++k) sum += f[k] != 0 ? f[k] * (double)x[k] : 0.0;
        sum = plus_dpp<kShr1>(sum);
        if (a.lanes > 2) sum = plus_dpp<kShr2>(sum);
        if (a.lanes > 4) sum = plus_dpp<kShr4>(sum);
        if (a.lanes > 8) sum = plus_dpp<kShr8>(sum);
        if (a.lanes > 16) sum = plus_dpp<kOfRow, 0xa>(sum);
        if (a.lanes > 32) sum = plus_dpp<kOfHalf, 0xc>(sum);
        if (none[i] && p0 + i < pages) bad = true;
        if (head < H && piece == a.lanes - 1 && p0 + i < pages)
          a.keys[((u64)s * H + head) * a.d.row_pages + p0 + i] = none[i] ? kNoKey : key_of(sum);
      }
    }
  }
  if (bad) raise_status(a.status, FDY_ST_BAD_INDEX);
}

// ---- choice -----------------------------------------------------------------------------------------
// One workgroup for a cache head of a sequence: the key that the last one taken has, eight bits at a time from the highest in which
// the keys differ, then those above it and as many of those equal to it as there is room for, in the order of the row.
constexpr u32 kThreads = 1024;
__global__ void __launch_bounds__(kThreads) choice_kernel(Select a) {
  __shared__ u64 s_scan[17];
  __shared__ u64 s_low[16], s_high[16];
  __shared__ u32 s_bins[256], s_bin, s_above, s_here;
  const u32 H = a.d.kv.n_heads, s = blockIdx.x / H, g = blockIdx.x % H, tid = threadIdx.x, budget = a.d.budget;
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
  for (u32 i = tid; i < sinks; i += kThreads) out[i] = table[i];
  for (u32 i = tid; i < recent; i += kThreads) out[budget - recent + i] = table[end + i];
  u32 left = budget - sinks - recent;  // to be taken of [sinks, end), which are more
  if (left == 0) return;
  const u64* keys = a.keys + (u64)blockIdx.x * a.d.row_pages;
  u64 low = ~0ull, high = 0;
  for (u32 j = sinks + tid; j < end; j += kThreads) low = min(low, keys[j]), high = max(high, keys[j]);
  for (u32 m = 1; m < 64; m *= 2) low = min(low, (u64)__shfl_xor((unsigned long long)low, m)), high = max(high, (u64)__shfl_xor((unsigned long long)high, m));
  if (lane_id() == 0) s_low[tid >> 6] = low, s_high[tid >> 6] = high;
  __syncthreads();
  for (u32 w = 0; w < kThreads / 64; ++w) low = min(low, s_low[w]), high = max(high, s_high[w]);
  // keys from `bound` on, whose bits below `shift` are 0, are `left` and those of its own 2^shift more
  u32 shift = low == high ? 0 : 64 - (u32)__builtin_clzll(low ^ high);
  u64 bound = shift == 64 ? 0 : high >> shift << shift;
  while (shift) {
    const u32 bits = min(shift, 8u), below = shift - bits;
    if (tid < 256) s_bins[tid] = 0;
    __syncthreads();
    for (u32 j = sinks + tid; j < end; j += kThreads) {
      const u64 key = keys[j];
      if (shift == 64 || key >> shift == bound >> shift) atomicAdd(&s_bins[(u32)(key >> below) & ((1u << bits) - 1)], 1u);
    }
    __syncthreads();
    if (tid < 64) {  // four bins a lane, from the highest down
      u32 c[4], sum = 0;
#pragma unroll
      for (u32 i = 0; i < 4; ++i) c[i] = s_bins[255 - tid * 4 - i], sum += c[i];
      u32 above = wave_incl_scan(sum) - sum;
#pragma unroll
      for (u32 i = 0; i < 4; ++i) {
        if (above < left && above + c[i] >= left) s_bin = 255 - tid * 4 - i, s_above = above, s_here = c[i];
        above += c[i];
      }
    }
    __syncthreads();
    left -= s_above;
    bound |= (u64)s_bin << below;
    shift = below;
    const bool all = s_here == left;
    __syncthreads();
    if (all) break;  // all that have these bits are taken
  }
  u64 before = 0;  // those above in the low half, those equal in the high
  for (u32 j0 = sinks; j0 < end; j0 += kThreads) {
    const u32 j = j0 + tid;
    const u64 key = j < end ? keys[j] >> shift : 0, at = bound >> shift;
    const u64 mine = j < end ? (key > at ? 1ull : key == at ? 1ull << 32 : 0) : 0;
    u64 sum;
    const u64 rank = before + block_excl_scan(mine, s_scan, sum);
    before += sum;
    const u32 equal = (u32)(rank >> 32);
    if (mine == 1 || (mine && equal < left)) out[sinks + (u32)rank + min(equal, left)] = table[j];
  }
}

template <typename F, typename A>
int go(F kernel, dim3 grid, u32 threads, void* stream, const A& a) {
  (void)hipGetLastError();  // drop any stale error left by earlier, unrelated runtime calls
  hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, (hipStream_t)stream, a);
  FDY_HIP_TRY(hipGetLastError());
  return FDY_OK;
}

bool bounds_valid(const fdy_bounds& d) {
  if (!kv_valid(d.kv) || d.n_seqs > 65536u || (u64)d.row_pages * d.kv.page_tokens >> 31) return false;
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
  const u32 fresh = d.max_fresh ? d.max_fresh : 1;
  a.slots = (fresh - 1) / d.kv.page_tokens + 2;
  if (a.slots > d.row_pages) a.slots = d.row_pages ? d.row_pages : 1;
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
    const u64 blocks = (u64)((d.row_pages + kChunk - 1) / kChunk) * a.head_blocks;
    const dim3 grid(d.n_seqs, (u32)(blocks < 32768 ? blocks : 32768));
    int rc;
    if (d.type == FDY_BF16)
      rc = d.kv.type == FDY_F8 ? go(scores_kernel<Bf16, FDY_F8>, grid, 256, stream, a) : go(scores_kernel<Bf16, FDY_BF16>, grid, 256, stream, a);
    else
      rc = d.kv.type == FDY_F8 ? go(scores_kernel<F16, FDY_F8>, grid, 256, stream, a) : go(scores_kernel<F16, FDY_F16>, grid, 256, stream, a);
    if (rc != FDY_OK) return rc;
  }
  return go(choice_kernel, dim3(d.n_seqs * d.kv.n_heads), kThreads, stream, a);
}
