// fdy_rope.hip - rotary positions: the table of angles, and their application with the append of keys and values to the
// pages of a cache.
#include <math.h>

#include "fdy_types.hpp"

using namespace fdy;

namespace {

constexpr double kTwoPi = 6.283185307179586476925286766559;

struct Freqs {
  double f[128];
};

// One thread a pair and position; p * f and its reduction to a turn in 64 bits.
__global__ void __launch_bounds__(256) rope_table_kernel(Freqs freqs, u64 first, u64 n, u32 half, double magnitude,
                                                         float* out) {
  for (u64 at = (u64)blockIdx.x * 256 + threadIdx.x; at < n * half; at += (u64)gridDim.x * 256) {
    const u64 p = at / half;
    const u32 i = (u32)(at - p * half);
    double s, c;
    sincos((double)(first + p) * freqs.f[i], &s, &c);
    out[p * 2 * half + i] = (float)(c * magnitude);
    out[(p * 2 + 1) * half + i] = (float)(s * magnitude);
  }
}

// ---- append ---------------------------------------------------------------------------------------
// y0 = x0 cos - x1 sin, y1 = x1 cos + x0 sin on pairs of a head's elements: three operations an element and no reuse, so
// the bound is memory (each element of q, k, v read once, written once) or, for the few tokens of a decode step, the
// latency of two dependent loads (position, then its angles).
struct AppendArg {
  fdy_append d;
  u32* status;
  u32 page_shift, unit_shift, n_heads, slices;  // n_heads: of queries, keys and values together
};
typedef Arg<AppendArg> Append;

template <typename T, int kN>
struct Chunk {
  typedef typename T::elem raw __attribute__((ext_vector_type(kN)));
  typedef float wide __attribute__((ext_vector_type(kN)));
};

// The scale of an 8-bit cache's head, by which elements are divided.  A product with the reciprocal is up to one and a half units
// off; with its remainder, which a fused operation gives exactly, it becomes the quotient as rounded once (the reciprocal being
// so itself, and nothing going out of range: elements are held within those that saturate, and other scales take the
// division).  The bare product, this and the division throughout: 16,411 tokens of 40 heads 165, 165 and 176 us, 4,096 tokens of 8
// cache heads 17.3, 18.0 and 19.9.
struct Scale {
  float by, inv, most;
  bool tame;
  __device__ explicit Scale(float s)
      : by(s), inv(1.f / s), most(kF8Most * s), tame(s >= 0x1p-60f && s <= 0x1p60f) {}
  __device__ __forceinline__ float quotient(float x) const {
    const float y = __builtin_amdgcn_fmed3f(x, -most, most), q = y * inv;
    return x != x ? x : __builtin_fmaf(-__builtin_fmaf(q, by, -y), inv, q);  // (this way round a zero keeps its sign)
  }
};

// A chunk of elements to a cache: rounded once, to the cache's type.
template <typename T, int kN, bool kF8>
__device__ __forceinline__ void put(void* base, u64 at, typename Chunk<T, kN>::wide x, const Scale& scale) {
  if (kF8) {
    typedef u32 words __attribute__((ext_vector_type(kN / 4)));
    words w;
    if (scale.tame) {
#pragma unroll
      for (int i = 0; i < kN; ++i) x[i] = scale.quotient(x[i]);
#pragma unroll
      for (int i = 0; i < kN / 4; ++i) w[i] = to_f8x4_in_range(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    } else {
#pragma unroll
      for (int i = 0; i < kN; ++i) x[i] /= scale.by;
#pragma unroll
      for (int i = 0; i < kN / 4; ++i) w[i] = to_f8x4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    }
    *(words*)((uint8_t*)base + at) = w;
  } else {
    typedef typename Chunk<T, kN>::raw raw;
    *(raw*)((typename T::elem*)base + at) = __builtin_convertvector(x, raw);
  }
}

template <typename V, int kN>
__device__ __forceinline__ void turn(V& a, V& b, V cs, V sn, bool half) {
  const V x = a, y = b;
  if (half) {
    a = x * cs - y * sn;
    b = y * cs + x * sn;
  } else {
#pragma unroll
    for (int i = 0; i < kN / 2; ++i) {
      a[2 * i] = x[2 * i] * cs[i] - x[2 * i + 1] * sn[i];
      a[2 * i + 1] = x[2 * i + 1] * cs[i] + x[2 * i] * sn[i];
      b[2 * i] = y[2 * i] * cs[kN / 2 + i] - y[2 * i + 1] * sn[kN / 2 + i];
      b[2 * i + 1] = y[2 * i + 1] * cs[kN / 2 + i] + y[2 * i] * sn[kN / 2 + i];
    }
  }
}

// Where a head's elements come from and go to.
struct Route {
  const void* src;
  u64 from;       // element
  void* out;      // rotated copy, or null
  u64 to;
  void* cache;    // or null
  u64 in_cache;
  float scale;    // of an 8-bit cache
  bool turned;
};

template <bool kF8>
__device__ __forceinline__ Route route_of(const Append& a, u32 t, u32 h, bool stored, u64 page, u32 place) {
  const fdy_append& d = a.d;
  const u32 nq = d.q ? d.n_q_heads : 0, nk = d.kv.n_heads;
  Route r;
  r.cache = nullptr;
  r.scale = 1.f;
  r.in_cache = 0;
  r.turned = h < nq + nk;
  if (h < nq) {
    r.src = d.q, r.from = t * d.q_token + h * d.q_head;
    r.out = d.q_out, r.to = t * d.q_out_token + h * d.q_out_head;
    return r;
  }
  const bool key = h < nq + nk;
  const u32 g = key ? h - nq : h - nq - nk;
  r.src = key ? d.k : d.v, r.from = key ? t * d.k_token + g * d.k_head : t * d.v_token + g * d.v_head;
  r.out = key ? d.k_out : nullptr, r.to = t * d.k_out_token + g * d.k_out_head;
  if (stored) {
    r.cache = key ? d.kv.k : d.kv.v;
    r.in_cache = page * d.kv.page_stride + place * d.kv.token_stride + g * d.kv.head_stride;
    const float* scale = key ? d.kv.k_scale : d.kv.v_scale;
    if (kF8 && scale) r.scale = scale[g];
  }
  return r;
}

// The token's page and place, whether it is stored, and what is wrong with it.
__device__ __forceinline__ bool slot_of(const Append& a, u32 t, u64& page, u32& place, u32* status) {
  if (!a.d.slots) return false;
  const int64_t s = a.d.slots[t];
  page = (u64)s >> a.page_shift;
  place = (u32)s & (a.d.kv.page_tokens - 1);
  const bool in = s >= 0 && page < a.d.kv.n_pages;
  if (!in && s != -1) raise_status(status, FDY_ST_BAD_INDEX);
  return in;
}

// A wave takes a token; a lane takes 2 kN elements of a head at a time (two loads of kN: the two halves of kN pairs) and keeps
// their kN cosines and sines in registers over all heads that it visits.  kN is 8, or 4 where heads, halves or addresses are
// multiples of 8 bytes only (4,096 tokens of 32 + 8 heads of 80, of which 40 turned: 161 us one element a thread).
template <typename T, int kN, bool kF8>
__global__ void __launch_bounds__(256) append_kernel(Append a) {
  typedef typename Chunk<T, kN>::raw raw;
  typedef typename Chunk<T, kN>::wide wide;
  typedef typename T::elem elem;
  const u32 t = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= a.d.n_tokens) return;
  const u32 lane = lane_id(), D = a.d.kv.head_dim, rot = a.d.rot_dim;
  const u32 u = lane & ((1u << a.unit_shift) - 1), hs = lane >> a.unit_shift, step = 64u >> a.unit_shift;
  const bool half = a.d.layout == FDY_ROPE_HALF;
  const int p = a.d.positions[t];
  if ((u32)p >= a.d.n_positions) {
    if (lane == 0) raise_status(a.status, FDY_ST_BAD_INDEX);
    return;
  }
  u64 page = 0;
  u32 place = 0;
  const bool stored = slot_of(a, t, page, place, lane == 0 ? a.status : nullptr);
  if (u * 2 * kN >= D) return;
  const bool turns = u < rot / (2 * kN);
  wide cs = 0, sn = 0;
  if (turns) {
    const float* row = a.d.table + (u64)p * rot + u * kN;
    cs = *(const wide*)row;
    sn = *(const wide*)(row + rot / 2);
  }
  // offsets of the two chunks in a turned head, and in one that is copied
  const u32 va = u * 2 * kN, vb = va + kN, ta = turns && half ? u * kN : va, tb = turns && half ? rot / 2 + u * kN : vb;
  const u32 n = a.n_heads, stride = step * a.slices;
  constexpr int kDeep = 2;  // heads under way at once (four: into 8 bits 182 us for 177)
  for (u32 h0 = hs + blockIdx.y * step; h0 < n; h0 += stride * kDeep) {
    raw xa[kDeep], xb[kDeep];
    Route r[kDeep];
#pragma unroll
    for (int i = 0; i < kDeep; ++i) {
      const u32 h = h0 + i * stride;
      if (h >= n) continue;
      r[i] = route_of<kF8>(a, t, h, stored, page, place);
      const elem* src = (const elem*)r[i].src + r[i].from;
      xa[i] = *(const raw*)(src + (r[i].turned ? ta : va));
      const u32 b = r[i].turned ? tb : vb;
      if (b < D) xb[i] = *(const raw*)(src + b);
    }
#pragma unroll
    for (int i = 0; i < kDeep; ++i) {
      const u32 h = h0 + i * stride;
      if (h >= n) continue;
      wide fa = __builtin_convertvector(xa[i], wide), fb = __builtin_convertvector(xb[i], wide);
      if (r[i].turned && turns) turn<wide, kN>(fa, fb, cs, sn, half);
      const u32 at = r[i].turned ? ta : va, bt = r[i].turned ? tb : vb;
      if (r[i].out) {
        put<T, kN, false>(r[i].out, r[i].to + at, fa, Scale(1.f));
        if (bt < D) put<T, kN, false>(r[i].out, r[i].to + bt, fb, Scale(1.f));
      }
      if (r[i].cache) {
        const Scale scale(r[i].scale);
        put<T, kN, kF8>(r[i].cache, r[i].in_cache + at, fa, scale);
        if (bt < D) put<T, kN, kF8>(r[i].cache, r[i].in_cache + bt, fb, scale);
      }
    }
  }
}

// Any even rot_dim, any head size, any strides and alignment: a thread takes one pair, or one element that is not turned.
template <typename T, bool kF8>
__device__ __forceinline__ void put1(const Route& r, u32 e, float x) {
  typedef typename T::elem elem;
  if (r.out) ((elem*)r.out)[r.to + e] = (elem)x;
  if (r.cache) {
    if (kF8)
      ((uint8_t*)r.cache)[r.in_cache + e] = (uint8_t)to_f8x4(x / r.scale, 0.f, 0.f, 0.f);
    else
      ((elem*)r.cache)[r.in_cache + e] = (elem)x;
  }
}

template <typename T, bool kF8>
__global__ void __launch_bounds__(256) append_any_kernel(Append a) {
  typedef typename T::elem elem;
  const u32 D = a.d.kv.head_dim, rot = a.d.rot_dim, pairs = rot / 2, t = blockIdx.x;
  const bool half = a.d.layout == FDY_ROPE_HALF;
  const int p = a.d.positions[t];
  const bool speaks = threadIdx.x == 0 && blockIdx.y == 0;
  if ((u32)p >= a.d.n_positions) {
    if (speaks) raise_status(a.status, FDY_ST_BAD_INDEX);
    return;
  }
  u64 page = 0;
  u32 place = 0;
  const bool stored = slot_of(a, t, page, place, speaks ? a.status : nullptr);
  const float* row = a.d.table + (u64)p * rot;
  for (u32 h = blockIdx.y; h < a.n_heads; h += gridDim.y) {
    const Route r = route_of<kF8>(a, t, h, stored, page, place);
    const elem* src = (const elem*)r.src + r.from;
    const u32 n = r.turned ? D - pairs : D;
    for (u32 i = threadIdx.x; i < n; i += 256) {
      if (r.turned && i < pairs) {
        const u32 ea = half ? i : 2 * i, eb = half ? i + pairs : 2 * i + 1;
        const float x = (float)src[ea], y = (float)src[eb], c = row[i], s = row[pairs + i];
        put1<T, kF8>(r, ea, x * c - y * s);
        put1<T, kF8>(r, eb, y * c + x * s);
      } else {
        const u32 e = r.turned ? i + pairs : i;
        put1<T, kF8>(r, e, (float)src[e]);
      }
    }
  }
}

// `wide`: elements of an access, 8, 4 or 1
template <typename T, bool kF8>
int launch_append(const Append& a, u32 wide, u32 n_cu, hipStream_t stream) {
  (void)hipGetLastError();  // drop any stale error left by earlier, unrelated runtime calls
  const u32 n = a.d.n_tokens;
  if (wide > 1) {
    Append b = a;
    b.unit_shift = 0;
    while ((2 * wide << b.unit_shift) < a.d.kv.head_dim) ++b.unit_shift;
    // heads that a wave visits one after another are spread over more waves where these would be less than four a SIMD
    const u32 step = 64u >> b.unit_shift, rounds = (a.n_heads + step - 1) / step, slices = n_cu * 16 / n;
    b.slices = slices < 1 ? 1 : slices > rounds ? rounds : slices;
    const dim3 grid((n + 3) / 4, b.slices);
    if (wide == 8)
      hipLaunchKernelGGL((append_kernel<T, 8, kF8>), grid, dim3(256), 0, stream, b);
    else
      hipLaunchKernelGGL((append_kernel<T, 4, kF8>), grid, dim3(256), 0, stream, b);
  } else {
    const u32 y = a.n_heads < 1024 ? a.n_heads : 1024;
    hipLaunchKernelGGL((append_any_kernel<T, kF8>), dim3(n, y), dim3(256), 0, stream, a);
  }
  FDY_HIP_TRY(hipGetLastError());
  return FDY_OK;
}

}  // namespace

extern "C" int fdy_rope_frequencies(const fdy_rope* h, double* h_freq) {
  if (!h || !h_freq) return FDY_ERR_INVALID_ARG;
  const u32 rot = h->rot_dim;
  if (h->scaling > FDY_ROPE_BANDS || rot < 2 || rot > 256 || rot % 2) return FDY_ERR_INVALID_ARG;
  if (!(h->base > 1) || !isfinite(h->base) || !isfinite(h->magnitude)) return FDY_ERR_INVALID_ARG;
  if (h->scaling != FDY_ROPE_PLAIN && (!(h->factor > 0) || !isfinite(h->factor))) return FDY_ERR_INVALID_ARG;
  if (h->scaling == FDY_ROPE_NTK && rot < 4) return FDY_ERR_INVALID_ARG;
  const bool turns = h->scaling == FDY_ROPE_YARN || h->scaling == FDY_ROPE_BANDS;
  if (turns && (!(h->low > 0) || !(h->high > h->low) || !isfinite(h->high) || !(h->trained_len > 0) ||
                !isfinite(h->trained_len)))
    return FDY_ERR_INVALID_ARG;
  const double base = h->scaling == FDY_ROPE_NTK ? h->base * pow(h->factor, rot / (rot - 2.0)) : h->base;
  double lo = 0, hi = 0;
  if (h->scaling == FDY_ROPE_YARN) {
    auto pair_of = [&](double t) { return rot * log(h->trained_len / (t * kTwoPi)) / (2 * log(h->base)); };
    auto held = [&](double x) { return x < 0 ? 0 : x > rot - 1.0 ? rot - 1.0 : x; };
    lo = held(floor(pair_of(h->high)));
    hi = held(ceil(pair_of(h->low)));
    if (hi <= lo) hi = lo + 0.001;
  }
  for (u32 i = 0; i < rot / 2; ++i) {
    double f = pow(base, -2.0 * i / rot);
    if (h->scaling == FDY_ROPE_LINEAR) f /= h->factor;
    if (h->scaling == FDY_ROPE_YARN) {
      double r = (i - lo) / (hi - lo);
      const double g = 1 - (r < 0 ? 0 : r > 1 ? 1 : r);
      f = f * ((1 - g) / h->factor + g);
    }
    if (h->scaling == FDY_ROPE_BANDS) {
      const double t = h->trained_len * f / kTwoPi, s = (t - h->low) / (h->high - h->low);
      f = t > h->high ? f : t < h->low ? f / h->factor : f * ((1 - s) / h->factor + s);
    }
    h_freq[i] = f;
  }
  return FDY_OK;
}

extern "C" int fdy_rope_table(const fdy_rope* h, uint64_t first, uint32_t n_positions, float* d_table, void* stream) {
  Freqs freqs;
  const int rc = fdy_rope_frequencies(h, freqs.f);
  if (rc != FDY_OK) return rc;
  if (first > 1ull << 31 || first + n_positions > 1ull << 31) return FDY_ERR_INVALID_ARG;
  if (n_positions == 0) return FDY_OK;
  if (!d_table || !aligned(d_table, 16)) return FDY_ERR_INVALID_ARG;
  const u32 half = h->rot_dim / 2;
  const u64 n = (u64)n_positions * half, blocks = (n + 255) / 256;
  (void)hipGetLastError();
  hipLaunchKernelGGL(rope_table_kernel, dim3((u32)(blocks < kMostBlocks ? blocks : kMostBlocks)), dim3(256), 0, (hipStream_t)stream, freqs, first,
                     (u64)n_positions, half, h->magnitude, d_table);
  FDY_HIP_TRY(hipGetLastError());
  return FDY_OK;
}

extern "C" int fdy_rope_append(const fdy_append* h, uint32_t* d_status, void* stream) {
  if (!h) return FDY_ERR_INVALID_ARG;
  const fdy_append& d = *h;
  if (!kv_valid(d.kv) || d.type > FDY_F16 || (d.kv.type != d.type && d.kv.type != FDY_F8)) return FDY_ERR_INVALID_ARG;
  if (d.layout > FDY_ROPE_INTERLEAVED || d.rot_dim < 2 || d.rot_dim % 2 || d.rot_dim > d.kv.head_dim) return FDY_ERR_INVALID_ARG;
  if (d.q && (!d.q_out || !d.n_q_heads || d.n_q_heads > 65536u)) return FDY_ERR_INVALID_ARG;
  if (d.n_tokens > kMostBlocks || d.n_positions > 1u << 31) return FDY_ERR_INVALID_ARG;
  if (d.n_tokens == 0) return FDY_OK;
  if (!d.k || !d.positions || !d.table || !aligned(d.positions, 4) || !aligned(d.table, 16)) return FDY_ERR_INVALID_ARG;
  if (d.slots && (!aligned(d.slots, 8) || !d.v || !d.kv.k || !d.kv.v)) return FDY_ERR_INVALID_ARG;
  const void* elems[] = {d.q, d.q_out, d.k, d.k_out, d.slots ? d.v : nullptr};
  for (const void* p : elems)
    if (!aligned(p, 2)) return FDY_ERR_INVALID_ARG;
  const u32 cache_bytes = elem_bytes(d.kv.type);
  if (d.slots && (!aligned(d.kv.k, cache_bytes) || !aligned(d.kv.v, cache_bytes) || !aligned(d.kv.k_scale, 4) ||
                  !aligned(d.kv.v_scale, 4)))
    return FDY_ERR_INVALID_ARG;
  // in place is element by element: only with the same strides
  if (d.q && d.q == d.q_out && (d.q_token != d.q_out_token || d.q_head != d.q_out_head)) return FDY_ERR_INVALID_ARG;
  if (d.k == d.k_out && (d.k_token != d.k_out_token || d.k_head != d.k_out_head)) return FDY_ERR_INVALID_ARG;

  Append a{};
  a.d = d;
  a.status = d_status;
  a.page_shift = log2_of(d.kv.page_tokens);
  a.unit_shift = 0;
  a.slices = 1;
  a.n_heads = (d.q ? d.n_q_heads : 0) + d.kv.n_heads * (d.slots ? 2 : 1);
  u64 strides = d.k_token | d.k_head;
  if (d.q) strides |= d.q_token | d.q_head | d.q_out_token | d.q_out_head;
  if (d.k_out) strides |= d.k_out_token | d.k_out_head;
  if (d.slots) strides |= d.v_token | d.v_head | d.kv.page_stride | d.kv.token_stride | d.kv.head_stride;
  u32 wide = 8;  // elements of an access that sizes, strides and addresses allow
  for (; wide > 1; wide = wide == 8 ? 4 : 1) {
    bool fits = d.rot_dim % (2 * wide) == 0 && d.kv.head_dim % wide == 0 && strides % wide == 0;
    for (const void* p : elems) fits = fits && aligned(p, 2 * wide);
    if (d.slots) fits = fits && aligned(d.kv.k, wide * cache_bytes) && aligned(d.kv.v, wide * cache_bytes);
    if (fits) break;
  }
  int dev, n_cu;
  const int rc = current_device(&dev, &n_cu);
  if (rc != FDY_OK) return rc;
  const bool f8 = d.kv.type == FDY_F8;
  if (d.type == FDY_BF16)
    return f8 ? launch_append<Bf16, true>(a, wide, (u32)n_cu, (hipStream_t)stream)
              : launch_append<Bf16, false>(a, wide, (u32)n_cu, (hipStream_t)stream);
  return f8 ? launch_append<F16, true>(a, wide, (u32)n_cu, (hipStream_t)stream)
            : launch_append<F16, false>(a, wide, (u32)n_cu, (hipStream_t)stream);
}
