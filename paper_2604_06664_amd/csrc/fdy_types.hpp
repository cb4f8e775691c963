// Element types of the decode operators (gfx950): vectors of 8 elements as registers hold them, and their way to and from
// 32 bits.  Not installed.
#pragma once
#include "fdy_decode.h"
#include "fdy_device.hpp"

namespace fdy {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

struct Bf16 {
  typedef __bf16 elem;
  typedef bf16x8 x8;
};
struct F16 {
  typedef _Float16 elem;
  typedef f16x8 x8;
};

constexpr float kF8Most = 448.f;  // largest finite e4m3

// Four values to e4m3, to nearest even, saturating; NaN stays NaN (med3 would drop it).
__device__ __forceinline__ float f8_range(float x) {
  const float y = __builtin_amdgcn_fmed3f(x, -kF8Most, kF8Most);
  return x != x ? x : y;
}
__device__ __forceinline__ u32 to_f8x4_in_range(float a, float b, float c, float d) {
  const int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (u32)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}
__device__ __forceinline__ u32 to_f8x4(float a, float b, float c, float d) {
  return to_f8x4_in_range(f8_range(a), f8_range(b), f8_range(c), f8_range(d));
}

inline u32 log2_of(u32 v) { return 31u - (u32)__builtin_clz(v); }
inline bool power_of_two(u32 v) { return v && !(v & (v - 1)); }
inline u32 elem_bytes(u32 type) { return type == FDY_F8 ? 1u : 2u; }

// What every call asks of a cache, whatever it does with it: known type, sizes in range, a page's elements within
// 2^31 bytes (offsets in a page are 32 bits wide, a page's own place in the pool is 64).
inline bool kv_valid(const fdy_kv& c) {
  if (c.type > FDY_F8 || c.reserved || !power_of_two(c.page_tokens) || c.page_tokens > 65536u) return false;
  if (!c.n_heads || c.n_heads > 65536u || !c.head_dim || c.head_dim > 256u || !c.n_pages || c.n_pages >= 1u << 31) return false;
  if (c.token_stride >> 31 || c.head_stride >> 31 || c.page_stride >> 40) return false;
  const u64 last = (c.page_tokens - 1) * c.token_stride + (c.n_heads - 1) * c.head_stride + c.head_dim;
  return last * elem_bytes(c.type) < 1ull << 31;
}

// The one argument of every kernel of a decode step: its struct, filled up with zeros to FDY_DECODE_ARG_BYTES.
template <typename T>
struct Arg : T {
  static_assert(sizeof(T) % 8 == 0 && sizeof(T) < FDY_DECODE_ARG_BYTES, "pointers lie at multiples of 8 bytes");
  uint8_t fill[FDY_DECODE_ARG_BYTES - sizeof(T)];
};
constexpr u32 kMostBlocks = 1u << 23;  // of one launch in x: 2^32 threads are the limit of a dimension

inline bool aligned(const void* p, u32 to) { return ((uintptr_t)p & (to - 1)) == 0; }

}  // namespace fdy
