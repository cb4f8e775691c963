// fdy_tree.hip - attention of several drafted tokens of every sequence over its pages, each with its own view of the others.
//
// The same sum as for one new token (fdy_attention.hip), with drafted tokens x query heads as the query rows of a cache head: a
// tile's 16 (32) rows are any of them, its keys and values are read once for all.  A few drafted tokens are still bounded by
// memory; from about 200 rows on by the matrix cores and by the vector unit, which has the weights to work out.
//
// What a row sees differs only in the row's last c tokens (and where a window begins): tiles elsewhere need no masks.  Where
// rows see different tokens, a value that is no number would come out of the product with weight 0 as NaN in rows that do not see it;
// such values are taken out of the product and added to the rows that see them one by one.
#include <type_traits>

#include "fdy_attend.hpp"

using namespace fdy;

namespace {

// A unit of work (below) in parts: where it is, and its parts.  0 of them: none.
struct Split {
  u32 parts, seq, unit, second;  // second: the first part lies in the second place of its share
};

struct TreeArg {
  fdy_draft d;
  u32* status;
  struct Split* splits;  // [shares]: of the unit that goes on from the share to the next
  float* parts;          // [shares][2] of: [rows][head_dim] sums, [rows] pairs of a maximum and a sum of e; 16-byte aligned
  u32 page_shift, group;
  u32 solid, least;  // solid 1: no unit of work is divided; least: places of a share
};
typedef Arg<TreeArg> Tree;

// ---- which work a workgroup takes -------------------------------------------------------------------
// The query rows of a cache head (drafted tokens x query heads) are tiles of kRows; all heads' tiles one after the other are the
// columns of a sequence.  `together` waves take as many columns of a head side by side, which read the same (kLeast of them at least; with
// kLeast 1, where every wave reads for itself, a head has one column), and the workgroup's other waves other tokens: `apart` tiles of 32 a
// round.  A unit is one such group of columns of one sequence; units lie one after the other on a line, kEach places and then a place for
// every round, and equal shares of the line go to the workgroups.  Where there is a workgroup for every round, each takes one.
struct Seq {
  Span span;        // tokens that any of its queries sees
  u32 query, count;  // its first drafted token in q, and how many
  int base;         // tokens ahead of them
  u32 rows, tiles, columns, together, rounds;  // tiles: of a head's rows
  __device__ u32 units() const { return (columns + together - 1) / together; }
  __device__ u32 unit(u32 each) const { return rounds + each ? rounds + each : 1; }
};
__device__ __forceinline__ Seq uniform(const Seq& v) {
  Seq q;
  q.span.first = fdy::uniform(v.span.first), q.span.end = fdy::uniform(v.span.end), q.span.row = fdy::uniform(v.span.row);
  q.span.bad = v.span.bad;
  q.query = fdy::uniform(v.query), q.count = fdy::uniform(v.count), q.base = (int)fdy::uniform((u32)v.base);
  q.rows = fdy::uniform(v.rows), q.together = fdy::uniform(v.together), q.tiles = fdy::uniform(v.tiles);
  q.columns = fdy::uniform(v.columns);
  q.rounds = fdy::uniform(v.rounds);
  return q;
}

template <u32 kRows, u32 kWaves, u32 kLeast>
__device__ __forceinline__ Seq seq_of(const Tree& a, u32 s) {
  Seq q;
  q.span.row = a.d.rows ? (u32)a.d.rows[s] : s;
  q.span.bad = q.span.row >= a.d.n_rows;
  if (q.span.bad) q.span.row = 0;
  int n = q.span.bad ? 0 : a.d.lens[q.span.row];
  const u32 room = a.d.row_pages << a.page_shift;
  if (n < 0 || (u32)n > room) q.span.bad = true, n = n < 0 ? 0 : (int)room;
  u32 from = s * a.d.max_draft, to = from + a.d.max_draft;
  if (a.d.first) from = (u32)a.d.first[s], to = (u32)a.d.first[s + 1];
  q.query = from, q.count = to - from;
  if (to < from || to > a.d.n_tokens || q.count > a.d.max_draft) q.span.bad = true, q.count = 0;
  if (q.count > (u32)n && n >= 0) q.span.bad = true;
  q.base = n - (int)q.count;
  q.span.end = q.count ? (u32)n : 0;
  q.span.first = a.d.window && q.base > 0 && (u32)q.base > a.d.window ? (u32)q.base - a.d.window : 0;
  q.rows = q.count * a.group;
  q.tiles = (q.rows + kRows - 1) / kRows;
  q.together = kLeast;
  if (kLeast > 1) {
    while (q.together < kWaves && q.together < q.tiles) q.together *= 2;
    q.tiles = (q.tiles + q.together - 1) / q.together * q.together;  // a group's are of one head
  }
  q.columns = q.tiles * a.d.kv.n_heads;
  const u32 apart = kWaves / q.together;
  q.rounds = (q.span.tiles() + apart - 1) / apart;
  if (a.solid && q.rounds) q.rounds = 1;  // all of them as one
  return q;
}

struct TreeShare {
  u32 begin, end, per;  // places
  u32 seq, start;       // the sequence at `begin`, and its own place
  u32 at, each;         // each: places ahead of a unit's rounds
};
template <u32 kWaves>
struct TreeLds {
  u32 sum[kWaves], units[kWaves], seq, start;
};

// All threads of the workgroup.
template <u32 kRows, u32 kWaves, u32 kLeast>
__device__ __forceinline__ bool find_tree_share(const Tree& a, TreeShare& out, TreeLds<kWaves>& lds) {
  constexpr u32 kThreads = 64 * kWaves;
  const u32 n = a.d.n_seqs, tid = threadIdx.x, slice = (n + kThreads - 1) / kThreads;
  const u32 s0 = min(tid * slice, n), s1 = min(s0 + slice, n);
  u32 mine = 0, units = 0;  // places, without any ahead of rounds
  for (u32 s = s0; s < s1; ++s) {
    const Seq q = seq_of<kRows, kWaves, kLeast>(a, s);
    if (q.span.bad && q.count == 0 && blockIdx.x == 0) raise_status(a.status, FDY_ST_BAD_INDEX);  // no one else looks at it
    mine += q.units() * q.unit(0), units += q.units();
  }
  const u32 inc = wave_incl_scan(mine);
  if (kLeast > 1) units = wave_incl_scan(units);
  if (lane_id() == 63) lds.sum[tid >> 6] = inc, lds.units[tid >> 6] = units;
  __syncthreads();
  u32 before = inc - mine, total = 0;
  units = 0;
#pragma unroll
  for (u32 w = 0; w < kWaves; ++w) {
    if (w < tid >> 6) before += lds.sum[w];
    total += lds.sum[w], units += lds.units[w];
  }
  out.each = fdy::uniform(total <= gridDim.x || a.solid ? 0 : kEach);
  if (out.each) {
    mine = 0, before = 0, total = 0;
    for (u32 s = s0; s < s1; ++s) {
      const Seq q = seq_of<kRows, kWaves, kLeast>(a, s);
      mine += q.units() * q.unit(kEach);
    }
    const u32 inc = wave_incl_scan(mine);
    __syncthreads();
    if (lane_id() == 63) lds.sum[tid >> 6] = inc;
    __syncthreads();
    before = inc - mine;
#pragma unroll
    for (u32 w = 0; w < kWaves; ++w) {
      if (w < tid >> 6) before += lds.sum[w];
      total += lds.sum[w];
    }
  }
  total = fdy::uniform(total);
  // dies take workgroups in turn: neighbours on the line, which read the same keys and values, go to one
  const u32 g = gridDim.x;
  out.at = g % 8 ? blockIdx.x : blockIdx.x % 8 * (g / 8) + blockIdx.x / 8;
  if (tid == 0) a.splits[out.at].parts = 0;
  if (total == 0) return false;
  out.per = max((total - 1) / g + 1, out.each + 1);
  if (kLeast > 1 && out.per < a.least) out.per = max(out.per, min(a.least, total / fdy::uniform(units)));  // (no more than units have, on average)
  if ((u64)out.at * out.per >= total) return false;
  out.begin = out.at * out.per;
  out.end = total - out.begin > out.per ? out.begin + out.per : total;
  if (out.begin >= before && out.begin < before + mine) {
    u32 s = s0;
    for (;; ++s) {
      const Seq q = seq_of<kRows, kWaves, kLeast>(a, s);
      const u32 c = q.units() * q.unit(out.each);
      if (out.begin < before + c) break;
      before += c;
    }
    lds.seq = s, lds.start = before;
  }
  __syncthreads();
  out.seq = fdy::uniform(lds.seq), out.start = fdy::uniform(lds.start);
  return true;
}

// ---- what a query row sees --------------------------------------------------------------------------
struct View {
  int from;   // its first token
  int upto;   // chains: its last
  u32 words;  // trees: where its bits begin, in words of 32
};

__device__ __forceinline__ View view_of(const Tree& a, const Seq& q, u32 j) {
  View v;
  v.from = 0, v.upto = q.base + (int)j, v.words = 0;
  const u32 w = a.d.window;
  if (!a.d.sees) {
    if (w && v.upto >= (int)w) v.from = v.upto + 1 - (int)w;
    return v;
  }
  const u64* bits = a.d.sees + (u64)(q.query + j) * a.d.sees_words;
  v.words = (q.query + j) * a.d.sees_words * 2;
  if (!w) return v;
  u32 seen = 0;
  const u32 words = (q.count + 63) / 64;
  auto word = [&](u32 i) { return q.count - i * 64 < 64 ? bits[i] & ((1ull << (q.count - i * 64)) - 1) : bits[i]; };
  for (u32 i = 0; i < words; ++i) seen += (u32)__popcll(word(i));
  if (seen < w) {
    v.from = q.base > (int)(w - seen) ? q.base - (int)(w - seen) : 0;
    return v;
  }
  u32 skip = seen - w;  // of the drafted ones that it sees the first are out of the window
  for (u32 i = 0; i < words; ++i) {
    u64 x = word(i);
    const u32 c = (u32)__popcll(x);
    if (skip >= c) {
      skip -= c;
      continue;
    }
    for (; skip; --skip) x &= x - 1;
    v.from = q.base + (int)(i * 64 + (u32)__builtin_ctzll(x));
    break;
  }
  return v;
}

// Bit i: whether the row sees token t + i, i < 4.
__device__ __forceinline__ u32 sees4(const Tree& a, const Seq& q, const View& v, int t) {
  u32 r = 0xf;
  const int b = t - q.base;  // number of the first among the drafted ones
  if (b > -4) {
    if (a.d.sees) {
      const u32 at = b > 0 ? (u32)b : 0, words = (q.count + 31) / 32, i = at >> 5;
      const u32* bits = (const u32*)a.d.sees + v.words;
      const u32 lo = i < words ? bits[i] : 0, hi = i + 1 < words ? bits[i + 1] : 0;
      r = (u32)(pair64(lo, hi) >> (at & 31));
      if (b < 0) r = r << -b | ((1u << -b) - 1);
    } else {
      r = t + 3 <= v.upto ? 0xf : t > v.upto ? 0 : (2u << (v.upto - t)) - 1;
    }
  }
  if (t < v.from) r = v.from - t >= 4 ? 0 : r & (0xfu << (v.from - t));
  return r & 0xf;
}

// ---- values that are no finite numbers --------------------------------------------------------------
template <typename T>
constexpr u32 kExponent = 0x7c00u;
template <>
inline constexpr u32 kExponent<Bf16> = 0x7f80u;

template <typename T, bool kF8>
__device__ __forceinline__ u32 odd_mask(u32 w) {  // all bits of each element of the word that is infinite or no number
  if (kF8) {
    u32 m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if ((w >> 8 * i & 0x7f) == 0x7f) m |= 0xffu << 8 * i;
    return m;
  }
  return ((w & kExponent<T>) == kExponent<T> ? 0xffffu : 0) | ((w >> 16 & kExponent<T>) == kExponent<T> ? 0xffff0000u : 0);
}

// ---- a wave's sums ----------------------------------------------------------------------------------
// Weights are at most 1 with bf16, of whatever size the slack leaves them; f16, which holds them lifted, has no room for any.
template <typename T>
inline constexpr float kSlack = kLift<T> == 0.f ? 4.f : 0.f;
template <typename T>
inline constexpr float kRaise = kLift<T> - kSlack<T>;

// Weights in two parts, as split(), for those that are worked on beside the matrix cores: bf16 with one operation an element less.  What
// makes the second part more than nothing is 2^-20 of the weight here.
template <typename T>
__device__ __forceinline__ void split_near(float x, float y, u32& first, u32& rest) {
  split<T>(x, y, first, rest);
}
template <>
__device__ __forceinline__ void split_near<Bf16>(float x, float y, u32& first, u32& rest) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const u32 a = __builtin_bit_cast(u32, x), b = __builtin_bit_cast(u32, y);
  constexpr float kMore = 1.f + 0x1p-20f;
  first = __builtin_amdgcn_perm(b, a, 0x07060302u);
  const bf16x2 r = {(__bf16)__builtin_fmaf(x, kMore, -__builtin_bit_cast(float, a & 0xffff0000u)),
                    (__bf16)__builtin_fmaf(y, kMore, -__builtin_bit_cast(float, b & 0xffff0000u))};
  rest = __builtin_bit_cast(u32, r);
}

template <typename T, int kDim, int kTiles>
struct Sums {
  typedef typename T::x8 x8;
  f32x4 o[kTiles][kDim / 16];
  float m[kTiles], sum[kTiles];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int qt = 0; qt < kTiles; ++qt) {
      m[qt] = -INFINITY, sum[qt] = 0.f;
#pragma unroll
      for (int i = 0; i < kDim / 16; ++i) o[qt][i] = 0;
    }
  }

  // The weights of a tile's scores, in two parts: 2^kRaise e^(x - m).  m follows the maximum once that is more than 2^kSlack ahead of it:
  // in the first few tiles and then hardly ever, where the maximum of one of 32 rows moves in three tiles of five.
  __device__ __forceinline__ void follow(const f32x4 (*s)[2], float scale) {
    float top[kTiles];
    bool moved = false;
#pragma unroll
    for (int qt = 0; qt < kTiles; ++qt) {
      float mx = s[qt][0][0];
#pragma unroll
      for (int j = 1; j < 8; ++j) mx = fmaxf(mx, s[qt][j / 4][j % 4]);
      top[qt] = over_groups(mx, larger);
      moved |= (top[qt] - m[qt]) * scale > kSlack<T>;
    }
    if (ballot(moved))
#pragma unroll
      for (int qt = 0; qt < kTiles; ++qt) {
        const float m_new = (top[qt] - m[qt]) * scale > kSlack<T> ? top[qt] : m[qt], ref = m_new == -INFINITY ? 0.f : m_new;
        const float keep = __builtin_amdgcn_exp2f((m[qt] - ref) * scale);
        m[qt] = m_new, sum[qt] *= keep;
#pragma unroll
        for (int i = 0; i < kDim / 16; ++i) o[qt][i] *= keep;
      }
  }
  // Two of a row's weights, and all of them.
  __device__ __forceinline__ void weigh2(const f32x4 (*s)[2], float scale, int qt, int j, v4u32* first_of, v4u32* rest_of) {
    const float ref = m[qt] == -INFINITY ? 0.f : m[qt];
    const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[qt][j / 2][2 * j % 4] - ref, scale, kRaise<T>));
    const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[qt][j / 2][2 * j % 4 + 1] - ref, scale, kRaise<T>));
    sum[qt] += e0 + e1;
    u32 hi_of, lo_of;
    split_near<T>(e0, e1, hi_of, lo_of);
    first_of[qt][j] = hi_of, rest_of[qt][j] = lo_of;
  }
  __device__ __forceinline__ void weigh(const f32x4 (*s)[2], float scale, v4u32* first_of, v4u32* rest_of) {
#pragma unroll
    for (int qt = 0; qt < kTiles; ++qt)
#pragma unroll
      for (int j = 0; j < 4; ++j) weigh2(s, scale, qt, j, first_of, rest_of);
  }
};

// Which of the lane's eight scores of a tile each of its rows sees; those that it does not at minus infinity.
template <int kTiles>
__device__ __forceinline__ void show(const Tree& a, const Seq& q, const u32* draft, u32 there, int tok, f32x4 (*s)[2]) {
#pragma unroll
  for (int qt = 0; qt < kTiles; ++qt) {
    u32 j0 = draft[qt];
    asm volatile("" : "+v"(j0));  // (nothing of this is worked out ahead of the loop over tiles, where registers are short)
    const View view = view_of(a, q, j0);
    const u32 shown = there & (sees4(a, q, view, tok) | sees4(a, q, view, tok + 16) << 4);
#pragma unroll
    for (int j = 0; j < 8; ++j) s[qt][j / 4][j % 4] = shown >> j & 1 ? s[qt][j / 4][j % 4] : -INFINITY;
  }
}

// The tokens of a tile that a lane's row sees (bit i: token i), from the four lanes that have eight of them each.
__device__ __forceinline__ u32 tokens_seen(const Tree& a, const Seq& q, const View& v, u32 there, int tok) {
  const u32 mine = there & (sees4(a, q, v, tok) | sees4(a, q, v, tok + 16) << 4), col = lane_id() & 15;
  u32 all = 0;
#pragma unroll
  for (u32 g = 0; g < 4; ++g) {
    const u32 of = (u32)__shfl((int)mine, (int)(col + 16 * g));
    all |= (of & 0xf) << 4 * g | (of >> 4) << (16 + 4 * g);
  }
  return all;
}

// ---- tiles from the pages to registers --------------------------------------------------------------
// Every wave for itself; the next tile's keys are asked for as soon as this one's are used up, its values likewise.  As in Tile,
// o[.][part * kWide + e][i] is of element part * 16 * kWide + (4 grp + i) * kWide + e.
template <typename T, bool kF8, int kDim, bool kSmall, int kPolicy, int kTiles>
struct Alone {
  typedef Tile<T, kF8, kDim, kSmall, kPolicy> Tl;
  typedef typename T::x8 x8;
  static constexpr int kWide = Tl::kWide, kParts = Tl::kParts, kSteps = Tl::kSteps;
  static __device__ __forceinline__ u32 element(u32 i, u32 k, u32 grp) {  // of o[.][i][k]
    return i / kWide * 16 * kWide + (grp * 4 + k) * kWide + i % kWide;
  }

  static __device__ __forceinline__ void walk(const Tree& a, const Seq& q, const typename Tl::Lanes& z, const x8 (*qs)[kSteps],
                                              const u32* draft, float scale, u32 t, u32 t_end, u32 t_step,
                                              Sums<T, kDim, kTiles>& sums, bool& bad) {
    if (t >= t_end) return;
    // tiles in which rows see different tokens, or tokens are not there
    const int past = q.base, opens = a.d.window ? (int)(q.span.end - a.d.window) : 0;
    Tl x;
    typename Tl::Ids ids = Tl::ids(a, q.span, t, bad);
    x.load_k(a, z, q.span, ids, t, bad);
    x.load_v(a, z, q.span, ids, t, bad);
    for (; t < t_end; t += t_step) {
      const u32 t_next = t + t_step < t_end ? t + t_step : 0x7fffffc0u;  // behind every row
      typename Tl::Ids ids_next = Tl::ids(a, q.span, t_next, bad);
      f32x4 s[kTiles][2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int qt = 0; qt < kTiles; ++qt) s[qt][u] = 0;
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
          const x8 key = x.key(u, st);
#pragma unroll
          for (int qt = 0; qt < kTiles; ++qt) s[qt][u] = mfma<T>(key, qs[qt][st], s[qt][u]);
        }
      }
      x.load_k(a, z, q.span, ids_next, t_next, bad);
      bool odd = false;
      u32 there = 0;
      if (!(Tl::whole(ids) && (int)(t + kTile - 1) < past && (int)t >= opens)) {  // (t + kTile may be 2^31)
        u32 any = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) there |= x.seen(a, z, q.span, ids, t, j / 4, j % 4) ? 1u << j : 0;
        show<kTiles>(a, q, draft, there, (int)(t + z.grp * 4), s);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int pt = 0; pt < kParts; ++pt)
#pragma unroll
            for (int k = 0; k < (int)sizeof(typename Tl::vword) / 4; ++k) {
              const u32 m = odd_mask<T, kF8>(word(x.v[i][pt], k));
              any |= m;
              if constexpr (sizeof(typename Tl::vword) == 4)
                x.v[i][pt] &= ~m;
              else
                x.v[i][pt][k] &= ~m;
            }
        odd = ballot(any != 0) != 0;
      }
      v4u32 p[kTiles], rest[kTiles];
      sums.follow(s, scale);
      sums.weigh(s, scale, p, rest);
#pragma unroll
      for (int pt = 0; pt < kParts; ++pt)
#pragma unroll
        for (int e2 = 0; e2 < kWide / 2; ++e2) {
          x8 even, odd_e;
          x.values(pt, e2, even, odd_e);
#pragma unroll
          for (int qt = 0; qt < kTiles; ++qt) {
            f32x4& c0 = sums.o[qt][pt * kWide + 2 * e2];
            f32x4& c1 = sums.o[qt][pt * kWide + 2 * e2 + 1];
            c0 = mfma<T>(even, __builtin_bit_cast(x8, p[qt]), c0);
            c1 = mfma<T>(odd_e, __builtin_bit_cast(x8, p[qt]), c1);
            c0 = mfma<T>(even, __builtin_bit_cast(x8, rest[qt]), c0);
            c1 = mfma<T>(odd_e, __builtin_bit_cast(x8, rest[qt]), c1);
          }
        }
      if (odd) {  // the elements that were taken out, to the rows that see them: whatever the weight is, it is not 0
        u32 seen[kTiles];
#pragma unroll
        for (int qt = 0; qt < kTiles; ++qt) seen[qt] = tokens_seen(a, q, view_of(a, q, draft[qt]), there, (int)(t + z.grp * 4));
        for (u32 i = 0; i < kTile; ++i) {
          const u32 tok = t + i;
          if (tok - q.span.first >= q.span.end - q.span.first) continue;
          const u32 page = (u32)a.d.table[(u64)q.span.row * a.d.row_pages + (tok >> a.page_shift)];
          if (page >= a.d.kv.n_pages) continue;
          const uint8_t* from = (const uint8_t*)a.d.kv.v + Tl::place(a, z, page, tok);
#pragma unroll
          for (int d = 0; d < kDim / 16; ++d)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const u32 e = element(d, k, z.grp);
              if (e >= a.d.kv.head_dim) continue;
              float y;
              if (kF8)
                y = (from[e] & 0x7f) == 0x7f ? NAN : 0.f;
              else
                y = (float)((const typename T::elem*)from)[e];
              if (__builtin_isfinite(y)) continue;
#pragma unroll
              for (int qt = 0; qt < kTiles; ++qt)
                if (seen[qt] >> i & 1) sums.o[qt][d][k] += y;
            }
        }
      }
      x.load_v(a, z, q.span, ids_next, t_next, bad);
      ids = ids_next;
    }
  }
};

// ---- tiles through shared memory --------------------------------------------------------------------
// Where several waves take the same tokens, a workgroup reads a tile once: its eight waves bring pieces of 1 KiB of several tiles from
// the pages to registers, a stage ahead, and from there to LDS (8-bit elements widened on the way), in two slots that take turns.
// A token's row of kDim elements lies in chunks of 32 bytes, chunk c at c ^ turn(token), so that neither the keys' rows (16 bytes of
// 16 tokens) nor the values' columns (16 elements of 4 tokens, which the transposing read hands out token by token) meet in a bank.
// o[.][i][k] is of element 16 i + 4 grp + k.
//
// kDirect: straight from the pages to LDS, which 16-bit elements and heads of exactly kDim allow.  kSmall: pages of less than 16 tokens;
// a wave looks up the page of every token of a stage, a lane each, and hands them to the lanes that read (248 rows a head over pages of 8
// tokens, 16 rows of 5,319: 433 us where every 16 rows read for themselves, 144 so).
template <typename T, bool kF8, int kDim, int kTiles, bool kDirect, u32 kWaves, bool kSmall>
struct Together {
  typedef typename T::x8 x8;
  typedef typename T::elem elem;
  static constexpr u32 kEs = kF8 ? 1 : 2, kRow = kDim * 2, kTileBytes = 2 * kTile * kRow;  // of keys, then values
  static constexpr u32 kMost = kDirect && kTiles == 2 ? 4 : kWaves / 4;  // tiles of a stage
  static constexpr u32 kSlot = kMost * kTileBytes;
  static constexpr int kSteps = kDim / 32;
  static constexpr u32 kPieces = 2 * kTile * kDim * kEs / 1024, kMine = (kPieces + kWaves - 1) / kWaves;  // of a tile; of a wave
  static constexpr u32 kLanes = kDim * kEs / 16, kTokens = 64 / kLanes;  // lanes of a token, tokens of a piece
  static __device__ __forceinline__ u32 element(u32 i, u32 k, u32 grp) { return i * 16 + grp * 4 + k; }
  static __device__ __forceinline__ u32 turn(u32 token) { return kDim == 64 ? token >> 1 & 3 : token & 7; }

  // Pages of a stage's tiles (0 where a number is none: what comes of it is not looked at).  Tiles that reach over the row's ends take
  // its first or last page there.
  typedef typename std::conditional<kSmall, u64, u32>::type Bits;  // of halves of tiles that have a page, or of tokens
  static_assert(!kSmall || (!kDirect && kMost <= 2), "a lane for every token of a stage");
  struct Ids {
    u32 page[kMost][2];
    Bits there;
  };
  static __device__ __forceinline__ Bits of_tile(Bits pages, u32 i) { return kSmall ? pages >> 32 * i & 0xffffffffu : pages >> 2 * i & 3; }
  static __device__ __forceinline__ bool has_page(Bits of, u32 token) { return of >> (kSmall ? token : token / 16) & 1; }
  static __device__ __forceinline__ bool all_there(Bits pages, u32 n) { return !(~pages & (((Bits)1 << (kSmall ? 16 : 1) * n << (kSmall ? 16 : 1) * n) - 1)); }
  static __device__ __forceinline__ void look_up(const Tree& a, const Seq& q, u32 tile, Ids& ids, bool& bad) {
    typedef const __attribute__((address_space(4))) u32* table_t;  // no one writes it while the kernel runs
    const table_t table = (table_t)(uintptr_t)(a.d.table + (u64)q.span.row * a.d.row_pages);
    const u32 low = q.span.first >> a.page_shift, high = (q.span.end - 1) >> a.page_shift;
    ids.there = 0;
    if constexpr (kSmall) {
      const u32 l = lane_id(), j = (tile * kTile + (kMost > 1 ? l : l % kTile)) >> a.page_shift;
      const u32 page = (u32)a.d.table[(u64)q.span.row * a.d.row_pages + max(low, min(j, high))];
      const bool ok = page < a.d.kv.n_pages;
      ids.there = ballot(ok);
      ids.page[0][0] = ok ? page : 0;
      bad |= !ok;
      return;
    }
#pragma unroll
    for (u32 i = 0; i < kMost; ++i)
#pragma unroll
      for (u32 u = 0; u < 2; ++u) {
        const u32 j = ((tile + i) * kTile + u * 16) >> a.page_shift;
        ids.page[i][u] = table[max(low, min(j, high))];
      }
#pragma unroll
    for (u32 i = 0; i < kMost; ++i)
#pragma unroll
      for (u32 u = 0; u < 2; ++u) {
        const bool ok = ids.page[i][u] < a.d.kv.n_pages;
        ids.there |= ok ? (Bits)1 << (2 * i + u) : 0;
        ids.page[i][u] = ok ? ids.page[i][u] : 0;
        bad |= !ok;
      }
  }

  v4u32 w[kMost][kMine];
  u32 lane_at[kMine];  // the lane's place in its piece's 16 tokens; kNowhere behind head_dim
  __device__ __forceinline__ void lanes(const Tree& a, u32 wave) {
    const u32 l = lane_id(), in = l / kLanes, c = l % kLanes, token_bytes = (u32)a.d.kv.token_stride * kEs;
#pragma unroll
    for (u32 m = 0; m < kMine; ++m) {
      const u32 token = token_of(wave + m * kWaves) + in;
      // 16-bit: the lane's 16 bytes go to half c % 2 of chunk c / 2; 8-bit: they are a chunk
      const u32 chunk = (kF8 ? c : c / 2) ^ turn(token), at = kF8 ? chunk * 16 : chunk * 32 + c % 2 * 16;
      lane_at[m] = at < a.d.kv.head_dim * kEs ? (kSmall ? 0 : (token & 15) * token_bytes) + at : kNowhere;
    }
  }
  static __device__ __forceinline__ u32 token_of(u32 piece) { return piece % (kPieces / 2) * kTokens; }
  __device__ __forceinline__ void load(const Tree& a, u32 of_head, u32 wave, u32 tile, u32 n, const Ids& ids) {
    const u64 page_bytes = a.d.kv.page_stride * kEs;
    const u32 token_bytes = (u32)a.d.kv.token_stride * kEs;
    if constexpr (kSmall) {
#pragma unroll
      for (u32 i = 0; i < kMost; ++i)
#pragma unroll
        for (u32 m = 0; m < kMine; ++m) {
          const u32 piece = wave + m * kWaves, token = i * kTile + token_of(piece) + lane_id() / kLanes;
          const u32 page = (u32)__shfl((int)ids.page[0][0], (int)token);
          w[i][m] = 0;
          if (i < n && piece < kPieces && lane_at[m] != kNowhere)
            w[i][m] = *(const v4u32*)((const uint8_t*)(piece >= kPieces / 2 ? a.d.kv.v : a.d.kv.k) + page * page_bytes +
                                      ((tile * kTile + token) & (a.d.kv.page_tokens - 1)) * (u64)token_bytes + of_head + lane_at[m]);
        }
      return;
    }
#pragma unroll
    for (u32 i = 0; i < kMost; ++i)
#pragma unroll
      for (u32 m = 0; m < kMine; ++m) {
        const u32 piece = wave + m * kWaves, u = token_of(piece) / 16;
        const u32 page = ids.page[i][0] ^ ((ids.page[i][0] ^ ids.page[i][1]) & (0u - u));
        const u32 in_page = (((tile + i) * kTile + u * 16) & (a.d.kv.page_tokens - 1)) * token_bytes + of_head;
        const auto from = buffer((const uint8_t*)(piece >= kPieces / 2 ? a.d.kv.v : a.d.kv.k) + page * page_bytes, kNowhere - 1);
        w[i][m] = 0;
        if (i < n && piece < kPieces) w[i][m] = __builtin_amdgcn_raw_buffer_load_b128(from, lane_at[m], in_page, 0);
      }
  }
  // The same to LDS, 1 KiB of it from `slot` on for each piece.  (Written as it stands since the compiler has every later read of LDS wait
  // for such loads, whichever slot it is of; the workgroup's barrier behind arrived() is what orders them.  m0 is the compiler's own and
  // is not taken as one of a statement's clobbers: no other instruction of these kernels may use it, which a test of the compiled code holds.)
  __device__ __forceinline__ void bring(const Tree& a, u32 of_head, u32 wave, u32 tile, u32 n, const Ids& ids, u32 slot) const {
    const u64 page_bytes = a.d.kv.page_stride * kEs;
    const u32 token_bytes = (u32)a.d.kv.token_stride * kEs;
#pragma unroll
    for (u32 i = 0; i < kMost; ++i)
#pragma unroll
      for (u32 m = 0; m < kMine; ++m) {
        const u32 piece = wave + m * kWaves, u = token_of(piece) / 16;
        const u32 page = ids.page[i][0] ^ ((ids.page[i][0] ^ ids.page[i][1]) & (0u - u));
        const u32 in_page = (((tile + i) * kTile + u * 16) & (a.d.kv.page_tokens - 1)) * token_bytes + of_head;
        const u64 from = fdy::uniform((u64)(uintptr_t)(piece >= kPieces / 2 ? a.d.kv.v : a.d.kv.k) + page * page_bytes);
        const v4u32 rsrc = {(u32)from, (u32)(from >> 32) & 0xffffu, kNowhere - 1, 0x00020000u};
        const u32 to = fdy::uniform(slot + i * kTileBytes + piece * 1024);
        if (i < n && piece < kPieces)
          asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                       :
                       : "s"(to), "v"(lane_at[m]), "s"(rsrc), "s"(fdy::uniform(in_page))
                       : "memory");
      }
  }
  static __device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
  __device__ __forceinline__ void store(uint8_t* slot, u32 wave, u32 n) const {
    const u32 l = lane_id();
#pragma unroll
    for (u32 i = 0; i < kMost; ++i)
#pragma unroll
      for (u32 m = 0; m < kMine; ++m) {
        const u32 piece = wave + m * kWaves;
        if (i >= n || piece >= kPieces) continue;
        uint8_t* to = slot + i * kTileBytes + (piece * 64 + l) * (kF8 ? 32 : 16);
        if constexpr (kF8) {
          v4u32 lo, hi;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            lo[2 * k] = widen_f8x2<T, false>(w[i][m][k]), lo[2 * k + 1] = widen_f8x2<T, true>(w[i][m][k]);
            hi[2 * k] = widen_f8x2<T, false>(w[i][m][2 + k]), hi[2 * k + 1] = widen_f8x2<T, true>(w[i][m][2 + k]);
          }
          *(v4u32*)to = lo, *(v4u32*)(to + 16) = hi;
        } else {
          *(v4u32*)to = w[i][m];
        }
      }
  }

  // Eight tokens of the lane's element of 16 i + ..., as the products take them.
  static __device__ __forceinline__ x8 value(const uint8_t* v, u32 at, u32 i) {
    typedef short i16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) i16x4* lds_t;
    const uint8_t* from = v + (at ^ i * 32);
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)from);
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(from + 16 * kRow));
    return __builtin_bit_cast(x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }

  // The scores of a tile whose keys lie at `k`; c of 2 kSteps is a step and a half of the tile.
  static __device__ __forceinline__ u32 key_at() {
    const u32 l = lane_id(), col = l & 15, grp = l >> 4;
    u32 at = col * kRow + ((grp >> 1 ^ turn(col)) * 32 + (grp & 1) * 16);
    asm volatile("" : "+v"(at));  // worked out again for each tile: what follows from it would take half a dozen registers
    return at;
  }
  static __device__ __forceinline__ x8 key(const uint8_t* k, u32 at, int c) {
    return __builtin_bit_cast(x8, *(const v4u32*)(k + (at ^ c / 2 * 64) + c % 2 * 16 * kRow));
  }
  static __device__ __forceinline__ void score(const uint8_t* k, const x8 (*qs)[kSteps], f32x4 (*s)[2]) {
    const u32 at = key_at();
#pragma unroll
    for (int c = 0; c < 2 * kSteps; ++c) {
      const x8 x = key(k, at, c);
#pragma unroll
      for (int qt = 0; qt < kTiles; ++qt) s[qt][c % 2] = mfma<T>(x, qs[qt][c / 2], c < 2 ? (f32x4)(0.f) : s[qt][c % 2]);
    }
  }

  // A tile whose values lie at `v`, with the scores s.  kPlain: all its rows see all of its tokens.  kOn: the scores of the tile at
  // k_next replace s; the matrix cores work on them while the vector unit does on this tile's weights.  With two waves a SIMD
  // little else hides how long LDS takes to answer, so the order of reads is the one written here: the first values ahead of the weights.
  template <bool kPlain, bool kOn>
  static __device__ __forceinline__ void take(const Tree& a, const Seq& q, const uint8_t* v, const uint8_t* k_next, u32 t, Bits pages,
                                              const x8 (*qs)[kSteps], const u32* draft, float scale, f32x4 (*s)[2],
                                              Sums<T, kDim, kTiles>& sums) {
    constexpr int kValues = kDim / 16, kAhead = 4;
    u32 l = lane_id();
    if (!kPlain) asm volatile("" : "+v"(l));  // as in show()
    const u32 col = l & 15, grp = l >> 4;
    const u32 v_token = grp * 4 + (col >> 2);
    u32 v_at = v_token * kRow + (turn(v_token) * 32 + (col & 3) * 8);
    asm volatile("" : "+v"(v_at));
    x8 values[kValues];
    constexpr int kTurns = 2 * kSteps, kPairs = 4 * kTiles;
    x8 x0, x1;
    u32 at = 0;
    if constexpr (kOn) at = key_at(), x0 = key(k_next, at, 0), x1 = key(k_next, at, 1);
    u32 there = 0, any = 0;
    if (!kPlain) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const u32 tok = t + (j / 4) * 16 + grp * 4 + j % 4;
        if (tok - q.span.first < q.span.end - q.span.first && has_page(pages, tok - t)) there |= 1u << j;
      }
      show<kTiles>(a, q, draft, there, (int)(t + grp * 4), s);
    }
    v4u32 p[kTiles], rest[kTiles];
    sums.follow(s, scale);
    f32x4 s_next[kTiles][2];
    if constexpr (kOn) {
#pragma unroll
      for (int c = 0; c < kTurns; ++c) {
        const x8 x2 = c + 2 < kTurns ? key(k_next, at, c + 2) : x0;
        if (c + kAhead >= kTurns) values[c + kAhead - kTurns] = value(v, v_at, c + kAhead - kTurns);
#pragma unroll
        for (int qt = 0; qt < kTiles; ++qt) s_next[qt][c % 2] = mfma<T>(x0, qs[qt][c / 2], c < 2 ? (f32x4)(0.f) : s_next[qt][c % 2]);
#pragma unroll
        for (int i = c * kPairs / kTurns; i < (c + 1) * kPairs / kTurns; ++i) sums.weigh2(s, scale, i / 4, i % 4, p, rest);
        __builtin_amdgcn_sched_barrier(0);
        x0 = x1, x1 = x2;
      }
#pragma unroll
      for (int qt = 0; qt < kTiles; ++qt) s[qt][0] = s_next[qt][0], s[qt][1] = s_next[qt][1];
    } else {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) values[i] = value(v, v_at, i);
      sums.weigh(s, scale, p, rest);
    }
    __builtin_amdgcn_s_setprio(1);  // products ahead of another wave's weights: 275 us -> 271 (eight wide trees)
#pragma unroll
    for (int i = 0; i < kValues; ++i) {
      if (i + kAhead < kValues) values[i + kAhead] = value(v, v_at, i + kAhead);
      x8 x = values[i];
      if (!kPlain) {  // nothing of tokens that are not there, and no infinities
        v4u32 y = __builtin_bit_cast(v4u32, x);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          y[j] &= (there >> (2 * j) & 1 ? 0xffffu : 0) | (there >> (2 * j + 1) & 1 ? 0xffff0000u : 0);
          const u32 m = odd_mask<T, false>(y[j]);
          any |= m;
          y[j] &= ~m;
        }
        x = __builtin_bit_cast(x8, y);
      }
#pragma unroll
      for (int qt = 0; qt < kTiles; ++qt) sums.o[qt][i] = mfma<T>(x, __builtin_bit_cast(x8, p[qt]), sums.o[qt][i]);
#pragma unroll
      for (int qt = 0; qt < kTiles; ++qt) sums.o[qt][i] = mfma<T>(x, __builtin_bit_cast(x8, rest[qt]), sums.o[qt][i]);
      if (kOn) __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    if (!kPlain && ballot(any != 0)) {  // what was taken out, to the rows that see it: whatever the weight is, it is not 0
      u32 seen[kTiles];
#pragma unroll
      for (int qt = 0; qt < kTiles; ++qt) {
        u32 j0 = draft[qt];
        asm volatile("" : "+v"(j0));
        seen[qt] = tokens_seen(a, q, view_of(a, q, j0), there, (int)(t + grp * 4));
      }
      for (u32 token = 0; token < kTile; ++token) {
        if (t + token - q.span.first >= q.span.end - q.span.first || !has_page(pages, token)) continue;
#pragma unroll
        for (int i = 0; i < kDim / 16; ++i) {
          asm volatile("" ::: "memory");  // a few at a time: this is seldom
#pragma unroll
          for (u32 e = 0; e < 4; ++e) {
            const float y = (float)*(const elem*)(v + token * kRow + ((i ^ turn(token)) * 32 + (grp * 4 + e) * 2));
            if (__builtin_isfinite(y)) continue;
#pragma unroll
            for (int qt = 0; qt < kTiles; ++qt)
              if (seen[qt] >> token & 1) sums.o[qt][i][e] += y;
          }
        }
      }
    }
  }

  // Tiles [tile, end): of each stage's the wave takes those that are its `turn` of `apart`.  All waves of the workgroup.
  static __device__ __forceinline__ void walk(const Tree& a, const Seq& q, u32 head, const x8 (*qs)[kSteps], const u32* draft, float scale,
                                              u32 tile, u32 end, u32 apart, u32 mine, bool works, uint8_t* lds, Sums<T, kDim, kTiles>& sums,
                                              bool& bad) {
    const u32 wave = fdy::uniform(threadIdx.x >> 6);
    constexpr u32 step = kMost;
    const int opens = a.d.window ? (int)(q.span.end - a.d.window) : 0;  // from there on all rows' windows are open
    auto count = [&](u32 from) { return from >= end ? 0 : end - from < step ? end - from : step; };
    // page numbers two stages ahead, loads one, so that both are under way while a stage is worked on
    const u32 of_head = head * (u32)a.d.kv.head_stride * kEs, at = (u32)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    Together x;
    x.lanes(a, wave);
    Ids ids;
    look_up(a, q, tile, ids, bad);
    if (kDirect)
      x.bring(a, of_head, wave, tile, count(tile), ids, at);
    else
      x.load(a, of_head, wave, tile, count(tile), ids);
    u32 slot = 0;
    Bits pages = ids.there, pages_next = 0;
    look_up(a, q, tile + step, ids, bad);
    if (!kDirect) {
      x.store(lds, wave, count(tile));
      x.load(a, of_head, wave, tile + step, count(tile + step), ids);
      pages_next = ids.there;
      look_up(a, q, tile + 2 * step, ids, bad);
    }
    // while a stage is worked on the next one is brought to LDS; or that to LDS, the one behind it to registers
    for (; tile < end; tile += step, slot ^= 1) {
      if (kDirect) arrived();
      __syncthreads();  // the slot is filled, the other one read
      Bits pages_then = 0;
      if (kDirect) {
        x.bring(a, of_head, wave, tile + step, count(tile + step), ids, at + (slot ^ 1) * kSlot);
        pages_next = ids.there;
        look_up(a, q, tile + 2 * step, ids, bad);
      } else {
        x.store(lds + (slot ^ 1) * kSlot, wave, count(tile + step));
        x.load(a, of_head, wave, tile + 2 * step, count(tile + 2 * step), ids);
        pages_then = ids.there;
        look_up(a, q, tile + 3 * step, ids, bad);
      }
      const u32 n = count(tile);
      if (works && mine < n) {
        const uint8_t* k = lds + slot * kSlot + mine * kTileBytes;
        f32x4 s[kTiles][2];
        const u32 first = tile * kTile;
        if (all_there(pages, n) && (int)(first + n * kTile - 1) < q.base && (int)first >= opens) {  // (the sum may be 2^31)
          score(k, qs, s);
          u32 i = mine;
          for (; i + apart < n; i += apart, k += apart * kTileBytes)
            take<true, true>(a, q, k + kTile * kRow, k + apart * kTileBytes, 0, 3, qs, draft, scale, s, sums);
          take<true, false>(a, q, k + kTile * kRow, k, 0, 3, qs, draft, scale, s, sums);
        } else {
          for (u32 i = mine; i < n; i += apart, k += apart * kTileBytes) {
            score(k, qs, s);
            take<false, false>(a, q, k + kTile * kRow, k, (tile + i) * kTile, of_tile(pages, i), qs, draft, scale, s, sums);
          }
        }
      }
      pages = pages_next, pages_next = pages_then;
    }
    __syncthreads();  // what follows goes where the slots lie
  }
};

// Elements [d, d + 4) of a head's row, from the sums over all of its tokens.
template <typename E>
__device__ __forceinline__ void finish_row(const Tree& a, const Seq& q, u32 kv_head, u32 row, u32 d, float M, float L, f32x4 y) {
  const u32 j = row / a.group, h = kv_head * a.group + row - j * a.group;
  const float v_scale = a.d.kv.type == FDY_F8 && a.d.kv.v_scale ? a.d.kv.v_scale[kv_head] : 1.f;
  y = y * (L == 0.f ? 0.f : v_scale / L);
  typedef E x4 __attribute__((ext_vector_type(4)));
  *(x4*)((E*)a.d.out + (u64)(q.query + j) * a.d.out_token + (u64)h * a.d.out_head + d) = __builtin_convertvector(y, x4);
  if (d == 0 && a.d.lse) a.d.lse[(u64)(q.query + j) * a.d.n_q_heads + h] = L == 0.f ? -INFINITY : (M + __builtin_log2f(L)) * kLn2;
}

// ---- the kernel -------------------------------------------------------------------------------------
constexpr u32 resident(int dim, u32 waves) { return dim <= 128 ? 8 / waves : 1; }  // workgroups of a compute unit
constexpr u32 resident(int dim, u32 waves, bool shared) { return shared ? (waves == 4 ? 3 : 1) : resident(dim, waves); }

// kShared: four waves at least take the same tokens, through LDS, four or eight waves a workgroup; otherwise every wave reads for itself.
// us with both launches: 8 rows of 6,000 to 8,192 tokens, 512 query rows a head 270 (445 TFLOP/s of scores and sums, half as much again
// done, for weights go in two parts); 33 of up to 8,192, 64 query rows 83 (3.1 TB/s); 64 windows of 2,048 in 8 bits, 5 rows 180 (4.4 TB/s);
// one of 517 tokens 16.5, a chain.  What the first spends: without loads 227, those alone 110, without both 43; without
// the second part of the weights 42 less, without following the maximum 26 less, without the exponentials 8; products with values beside
// the next tile's weights in one wave gained nothing (275 for 275), keys a tile ahead in registers neither (283).
// Its loads are not hidden: variants of 32 rows a wave keep 8 registers in scratch memory (20 to 38 with 8-bit caches, small pages or heads
// that are not exactly kDim; heads of more than 128 8 to 25), and a wait for one of them back is a wait for all loads, the next stage's too.
template <typename T, bool kF8, int kDim, bool kSmall, int kPolicy, int kTiles, u32 kWaves, bool kShared, bool kDirect>
__global__ void __launch_bounds__(64 * kWaves, resident(kDim, kWaves, kShared) * kWaves / 4) tree_kernel(Tree a) {
  typedef Tile<T, kF8, kDim, kSmall, kPolicy> Tl;
  typedef Together<T, kF8, kDim, kTiles, kDirect, kWaves, kSmall && kShared> Both;
  typedef typename std::conditional<kShared, Both, Alone<T, kF8, kDim, kSmall, kPolicy, kTiles>>::type Way;
  typedef typename T::x8 x8;
  typedef typename T::elem elem;
  constexpr int kSteps = kDim / 32, kPad = kDim + 4;
  constexpr u32 kLeast = kShared ? 4 : 1;  // so that a stage of two tiles has work for all waves
  constexpr u32 kRows = 16 * kTiles, kThreads = 64 * kWaves;
  constexpr u32 kSumBytes = kWaves * kRows * kPad * 4, kSlotBytes = kShared ? 2 * Both::kSlot : 0;
  __shared__ alignas(16) uint8_t s_mem[kSumBytes > kSlotBytes ? kSumBytes : kSlotBytes];
  float(*s_o)[kRows][kPad] = (float(*)[kRows][kPad])s_mem;
  __shared__ float s_m[kWaves][kRows], s_l[kWaves][kRows];
  __shared__ TreeLds<kWaves> s_share;

  TreeShare share;
  if (!find_tree_share<kRows, kWaves, kLeast>(a, share, s_share)) return;
  const u32 wave = fdy::uniform(threadIdx.x >> 6), D = a.d.kv.head_dim, quads = D / 4;
  const u32 part_size = part_floats(kRows * kWaves, D);
  // parts are written through to memory as they come: what the caches held of them would be written at the kernel's end, by itself
  const auto parts = buffer(a.parts, gridDim.x * 2 * part_size * 4);  // within 2^30 bytes

  u32 seq = share.seq, seq_start = share.start;
  Seq q = uniform(seq_of<kRows, kWaves, kLeast>(a, seq));
  for (u32 place = share.begin; place < share.end;) {
    while (place - seq_start >= q.units() * q.unit(share.each)) {
      seq_start += q.units() * q.unit(share.each);
      q = uniform(seq_of<kRows, kWaves, kLeast>(a, ++seq));
    }
    const u32 of_unit = q.unit(share.each), unit = fdy::uniform((place - seq_start) / of_unit);
    const u32 u_start = seq_start + unit * of_unit, start = u_start + share.each, next = u_start + of_unit;
    place = next;
    const u32 lo = start > share.begin ? start : share.begin, hi = next < share.end ? next : share.end;
    if (q.rounds ? lo >= hi : u_start < share.begin) continue;
    const bool whole = !q.rounds || (lo == start && hi == next);
    const u32 together = q.together, apart = kWaves / together, turn = wave / together;
    const u32 column0 = unit * together, column = column0 + wave % together;  // the workgroup's first, the wave's
    const u32 head = column < q.columns ? fdy::uniform(column / q.tiles) : 0, q0 = column < q.columns ? column % q.tiles * kRows : q.rows;
    const bool works = q0 < q.rows;
    bool bad = q.span.bad;

    // the factor of the scores, made positive (its sign goes to the queries)
    const float factor = a.d.scale * (kF8 && a.d.kv.k_scale ? a.d.kv.k_scale[head] : 1.f) * kLog2e;
    const float scale = factor == 0.f ? 1.f : fabsf(factor);
    const u32 q_keep = factor == 0.f ? 0u : ~0u, q_flip = factor < 0.f ? 0x80008000u : 0u;
    typename Tl::Lanes z;
    Tl::lanes(a, head, z);

    x8 qs[kTiles][kSteps];
    u32 draft[kTiles];  // of the lane's rows
#pragma unroll
    for (int qt = 0; qt < kTiles; ++qt) {
      const u32 r = q0 + qt * 16 + z.col, j = r / a.group, h = r - j * a.group;
      const bool there = works && r < q.rows;
      const elem* src = (const elem*)a.d.q + (u64)(q.query + j) * a.d.q_token + (u64)(head * a.group + h) * a.d.q_head;
#pragma unroll
      for (int st = 0; st < kSteps; ++st) {
        const u32 e = kF8 && !kShared ? (st / 2) * 64 + z.grp * 16 + (st & 1) * 8 : st * 32 + z.grp * 8;
        v4u32 w = 0;
        if (there && e < D) w = *(const v4u32*)(src + e);
        qs[qt][st] = __builtin_bit_cast(x8, (w & q_keep) ^ q_flip);
      }
      draft[qt] = there ? j : 0;
    }

    Sums<T, kDim, kTiles> sums;
    sums.clear();
    const u32 tile0 = q.span.first / kTile, tiles = q.span.tiles();
    u32 begin = (lo - start) * apart, end = (hi - start) * apart < tiles ? (hi - start) * apart : tiles;
    if (a.solid) begin = 0, end = tiles;
    if constexpr (kShared) {
      if (q.rounds)
        Way::walk(a, q, head, qs, draft, scale, fdy::uniform(tile0 + begin), fdy::uniform(tile0 + end), apart, turn, works, s_mem, sums, bad);
    } else {
      if (q.rounds && works)
        Way::walk(a, q, z, qs, draft, scale, fdy::uniform((tile0 + begin + turn) * kTile), fdy::uniform((tile0 + end) * kTile),
                  apart * kTile, sums, bad);
    }
    if (ballot(bad) && lane_id() == 0) raise_status(a.status, FDY_ST_BAD_INDEX);

    u32 tid = threadIdx.x;
    asm volatile("" : "+v"(z.col), "+v"(z.grp), "+v"(tid));  // nothing of what follows is worked out ahead of the tiles
    const u32 items = together * kRows * quads;  // item i: four elements of a row
    // row r of the workgroup's: its head and its number among the head's rows (~0: none)
    auto row_of = [&](u32 r, u32& kv_head) {
      const u32 c = column0 + r / kRows;
      kv_head = c / q.tiles;
      const u32 row = (c - kv_head * q.tiles) * kRows + r % kRows;
      return c < q.columns && row < q.rows ? row : ~0u;
    };
    const u32 mine = (share.at * 2 + (start > share.begin)) * part_size;
    if (kShared && apart == 1) {  // no other wave has sums of these rows
#pragma unroll
      for (int qt = 0; qt < kTiles; ++qt) {
        const u32 in = qt * 16 + z.col, r = wave * kRows + in, row = q0 + in;
        const float L = over_groups(sums.sum[qt], plus), M = sums.m[qt] * scale - kRaise<T>;
        if (!works || row >= q.rows) continue;
#pragma unroll
        for (int i = 0; i < kDim / 16; ++i) {
          const u32 d = Way::element(i, 0, z.grp);
          if (d >= D) continue;
          if (whole)
            finish_row<elem>(a, q, head, row, d, M == -INFINITY ? 0.f : M, L, sums.o[qt][i]);
          else
            put_part(parts, mine + r * D + d, sums.o[qt][i]);
        }
        if (!whole && z.grp == 0) put_part(parts, mine + kRows * kWaves * D + 2 * r, M, L);
      }
    } else {  // the waves' sums, joined
#pragma unroll
      for (int qt = 0; qt < kTiles; ++qt) {
        const float sum = over_groups(sums.sum[qt], plus);
#pragma unroll
        for (int i = 0; i < kDim / 16; ++i)
#pragma unroll
          for (int k = 0; k < 4; ++k) s_o[wave][qt * 16 + z.col][Way::element(i, k, z.grp)] = sums.o[qt][i][k];
        if (z.grp == 0) s_m[wave][qt * 16 + z.col] = sums.m[qt] * scale - kRaise<T>, s_l[wave][qt * 16 + z.col] = sum;
      }
      __syncthreads();
      for (u32 i = tid; i < items; i += kThreads) {
        const u32 r = i / quads, qd = i - r * quads, c = r / kRows, in = r % kRows;
        u32 kv_head;
        const u32 row = row_of(r, kv_head);
        if (row == ~0u) continue;
        constexpr u32 kApart = kWaves / kLeast;  // the most waves that have sums of a row; those behind the last count nothing
        float m[kApart], l[kApart], M = -INFINITY, L = 0.f;
        f32x4 o[kApart], y = 0;
#pragma unroll
        for (u32 k = 0; k < kApart; ++k) {
          const u32 w = k < apart ? c + k * together : c;
          m[k] = k < apart ? s_m[w][in] : -INFINITY, l[k] = s_l[w][in], o[k] = *(const f32x4*)&s_o[w][in][qd * 4];
        }
#pragma unroll
        for (u32 k = 0; k < kApart; ++k) M = fmaxf(M, m[k]);
        const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (u32 k = 0; k < kApart; ++k) {
          const float f = __builtin_amdgcn_exp2f(m[k] - ref);
          if (k < apart) L += f * l[k], y += f * o[k];
        }
        if (whole) {
          finish_row<elem>(a, q, kv_head, row, qd * 4, ref, L, y);
        } else {
          put_part(parts, mine + r * D + qd * 4, y);
          if (qd == 0) put_part(parts, mine + kRows * kWaves * D + 2 * r, M, L);
        }
      }
    }
    if (whole) {
      __syncthreads();  // the next unit's sums go where these lay
      continue;
    }

    // where the unit's parts are, written by the workgroup that has the first of them
    const u32 first = start / share.per;
    if (first == share.at && threadIdx.x == 0) {
      Split* split = a.splits + first;
      split->seq = seq, split->unit = unit, split->second = start > first * share.per;
      split->parts = (next - 1) / share.per - first + 1;
    }
    __syncthreads();  // the next unit's sums go where these lay
  }
}

// Units in parts, joined: a workgroup for every share that a unit goes on from, and a slice of its rows.  In a launch of its own, which
// all of the card takes part in (by the workgroup that finished last, through memory: 18 to 30 us for 0.4 MB of parts; so 6 to 9).
template <typename T, u32 kRows, u32 kWaves, u32 kLeast>
__global__ void __launch_bounds__(256) tree_join_kernel(Tree a) {
  typedef typename T::elem elem;
  const Split* split = a.splits + blockIdx.x;
  const u32 n_parts = fdy::uniform(split->parts), seq = fdy::uniform(split->seq), unit = fdy::uniform(split->unit);
  if (n_parts == 0) return;
  const u32 second = fdy::uniform(split->second), first = blockIdx.x, D = a.d.kv.head_dim, quads = D / 4;
  const Seq q = uniform(seq_of<kRows, kWaves, kLeast>(a, seq));
  const u32 part_size = part_floats(kRows * kWaves, D), items = q.together * kRows * quads, column0 = unit * q.together;
  // kItems items of a thread at once, kAtOnce parts of each
  auto join = [&](auto n_items, auto at_once) {
    constexpr u32 kItems = decltype(n_items)::value, kAtOnce = decltype(at_once)::value;
    const u32 step = gridDim.y * 256;
    for (u32 i0 = blockIdx.y * 256 + threadIdx.x; i0 < items; i0 += kItems * step) {
      float M[kItems], L[kItems];
      f32x4 y[kItems];
      u32 at[kItems], at_ml[kItems];
#pragma unroll
      for (u32 g = 0; g < kItems; ++g) {
        const u32 i = min(i0 + g * step, items - 1), r = i / quads;
        at[g] = r * D + (i - r * quads) * 4, at_ml[g] = kRows * kWaves * D + 2 * r;
        M[g] = -INFINITY, L[g] = 0.f, y[g] = 0;
      }
      for (u32 k0 = 0; k0 < n_parts; k0 += kAtOnce) {
        f32x4 part[kItems][kAtOnce];
        float m[kItems][kAtOnce], l[kItems][kAtOnce];
#pragma unroll
        for (u32 j = 0; j < kAtOnce; ++j) {
          const u32 k = k0 + j < n_parts ? k0 + j : k0;
          const float* from = a.parts + (u64)((first + k) * 2 + (k == 0 && second)) * part_size;
#pragma unroll
          for (u32 g = 0; g < kItems; ++g) {
            part[g][j] = *(const f32x4*)(from + at[g]);
            m[g][j] = from[at_ml[g]], l[g][j] = from[at_ml[g] + 1];
          }
        }
#pragma unroll
        for (u32 g = 0; g < kItems; ++g) {
          float top = M[g];
#pragma unroll
          for (u32 j = 0; j < kAtOnce; ++j) top = fmaxf(top, m[g][j]);
          const float ref = top == -INFINITY ? 0.f : top, keep = __builtin_amdgcn_exp2f(M[g] - ref);
          y[g] *= keep, L[g] *= keep, M[g] = top;
#pragma unroll
          for (u32 j = 0; j < kAtOnce; ++j)
            if (k0 + j < n_parts) {
              const float f = __builtin_amdgcn_exp2f(m[g][j] - ref);
              L[g] += f * l[g][j];
              y[g] += f * part[g][j];
            }
        }
      }
#pragma unroll
      for (u32 g = 0; g < kItems; ++g) {
        const u32 i = i0 + g * step, r = i / quads, d = (i - r * quads) * 4, c = column0 + r / kRows, head = c / q.tiles;
        const u32 row = (c - head * q.tiles) * kRows + r % kRows;
        if (i < items && c < q.columns && row < q.rows) finish_row<elem>(a, q, head, row, d, M[g] == -INFINITY ? 0.f : M[g], L[g], y[g]);
      }
    }
  };
  if (n_parts <= 4)
    join(std::integral_constant<u32, 2>(), std::integral_constant<u32, 4>());
  else
    join(std::integral_constant<u32, 1>(), std::integral_constant<u32, 8>());
}

// Workgroups: as many as are resident together, fewer where there are not the rounds.
u64 row_tiles(const fdy_draft& d) { return ((u64)d.row_pages * d.kv.page_tokens + kTile - 1) / kTile; }
u64 most_places(const fdy_draft& d, u32 rows) {
  const u64 tiles = ((u64)d.max_draft * (d.n_q_heads / d.kv.n_heads) + rows - 1) / rows;
  return d.n_seqs * d.kv.n_heads * tiles * (row_tiles(d) + 2 + kEach);
}
constexpr u32 kMostShares = kCus * 4;
constexpr size_t kSplitBytes = kMostShares * sizeof(Split);
constexpr u32 kSolid = 3, kSolidShared = 4;  // tiles of a wave, and of a workgroup that shares them

template <typename T, bool kF8, int kDim>
int launch_tree(const Tree& a, hipStream_t stream) {
  (void)hipGetLastError();  // drop any stale error left by earlier, unrelated runtime calls
  auto go = [&](auto kernel, auto join, u32 rows, u32 waves, u32 of_unit, u32 solid, bool shared = false) {
    u64 shares = kCus * of_unit;
    const u64 most = most_places(a.d, 16);
    if (shares > most) shares = most;
    // Few units, and none of more rounds than a launch that joins parts is worth: each goes to one workgroup (8 drafted tokens over 517,
    // three rounds: 16.4 us, in parts 18.4; over 1,000, four rounds: 21.4 and 20.0).
    Tree b = a;
    const u64 tiles_of = a.d.window && a.d.window < 1u << 30 ? (a.d.window + a.d.max_draft) / kTile + 2 : ~0ull, tiles = row_tiles(a.d);
    const u64 units = a.d.n_seqs * (u64)a.d.kv.n_heads * ((a.d.max_draft * a.group + rows - 1) / rows);
    b.solid = units <= shares && (tiles < tiles_of ? tiles : tiles_of) <= solid;
    if (b.solid) shares = units;
    // Shares of one or two tiles have more to write and to join than to work on where many rows share a tile: at least four, eight of
    // long rows (64 drafted tokens over 1,000: one 85 us, four 38, eight 44; over 4,000: four 91, eight 56).
    b.least = !shared || b.solid ? 1 : tiles > 64 ? 8 : 4;
    hipLaunchKernelGGL(kernel, dim3((u32)shares), dim3(64 * waves), 0, stream, b);
    if (b.solid) return;
    // slices of at least 256 items of four elements (64 drafted tokens over 2,000: 16 of them 52 us, 32 42; 12 such rows 88 and 90)
    const u32 slices = (rows * waves * (a.d.kv.head_dim / 4) + 255) / 256, most_slices = units <= 256 ? 32 : 16;
    if (shares > 1) hipLaunchKernelGGL(join, dim3((u32)shares, slices < most_slices ? slices : most_slices), dim3(256), 0, stream, b);
  };
  // 32 rows a wave, 16 where their sums would not fit the registers or where there are no more
  constexpr int kTwo = kDim <= 128 ? 2 : 1, kOnce = kNonTemporal;
  constexpr u32 kMost = kDim <= 128 ? 8 : 4, kFew = kDim <= 128 ? 4 : 8;
  const u32 rows = a.d.max_draft * a.group;
  const bool direct = !kF8 && a.d.kv.head_dim == kDim;
  const bool small = a.d.kv.page_tokens < 16;
  if (small && rows <= 16)
    go(tree_kernel<T, kF8, kDim, true, 0, 1, 4, false, false>, tree_join_kernel<T, 16, 4, 1>, 16, 4, resident(kDim, 4), kSolid * 4);
  else if (small && rows <= 64 && kDim <= 128)
    go(tree_kernel<T, kF8, kDim, true, 0, 1, kFew, true, false>, tree_join_kernel<T, 16, kFew, 4>, 16, kFew, resident(kDim, kFew, true), kSolidShared, true);
  else if (small)
    go(tree_kernel<T, kF8, kDim, true, 0, kTwo, 8, true, false>, tree_join_kernel<T, 16 * kTwo, 8, 4>, 16 * kTwo, 8, resident(kDim, 8, true), kSolidShared, true);
  else if (rows <= 16)
    go(tree_kernel<T, kF8, kDim, false, kOnce, 1, kMost, false, false>, tree_join_kernel<T, 16, kMost, 1>, 16, kMost, resident(kDim, kMost), kSolid * kMost);
  else if (rows <= 16 * kTwo)
    go(tree_kernel<T, kF8, kDim, false, kOnce, kTwo, kMost, false, false>, tree_join_kernel<T, 16 * kTwo, kMost, 1>, 16 * kTwo, kMost,
       resident(kDim, kMost), kSolid * kMost);
  else if (rows <= 64 && kDim <= 128)
    go(direct ? tree_kernel<T, kF8, kDim, false, 0, 1, kFew, true, !kF8> : tree_kernel<T, kF8, kDim, false, 0, 1, kFew, true, false>,
       tree_join_kernel<T, 16, kFew, 4>, 16, kFew, resident(kDim, kFew, true), kSolidShared, true);
  else
    go(direct ? tree_kernel<T, kF8, kDim, false, 0, kTwo, 8, true, !kF8> : tree_kernel<T, kF8, kDim, false, 0, kTwo, 8, true, false>,
       tree_join_kernel<T, 16 * kTwo, 8, 4>, 16 * kTwo, 8, resident(kDim, 8, true), kSolidShared, true);
  FDY_HIP_TRY(hipGetLastError());
  return FDY_OK;
}

template <typename T, bool kF8>
int launch_tree(const Tree& a, hipStream_t stream) {
  if (a.d.kv.head_dim <= 64) return launch_tree<T, kF8, 64>(a, stream);
  if (a.d.kv.head_dim <= 128) return launch_tree<T, kF8, 128>(a, stream);
  return launch_tree<T, kF8, 256>(a, stream);
}

bool sizes_valid(const fdy_draft& d) {
  if (!kv_valid(d.kv) || d.type > FDY_F16 || (d.kv.type != d.type && d.kv.type != FDY_F8)) return false;
  if (d.kv.head_dim % (d.kv.type == FDY_F8 ? 16 : 8)) return false;
  if (d.n_seqs > 65536u || !d.n_q_heads || d.n_q_heads > 65536u || d.n_q_heads % d.kv.n_heads) return false;
  if (!d.max_draft || d.max_draft > 1024u || d.n_tokens > 1u << 23 || (u64)d.n_tokens * d.n_q_heads > 1u << 26) return false;
  if (d.sees ? d.sees_words < (d.max_draft + 63) / 64 || d.sees_words > 64u : d.sees_words != 0) return false;
  if (!d.first && (u64)d.n_seqs * d.max_draft > d.n_tokens) return false;
  if ((u64)d.row_pages * d.kv.page_tokens >> 31) return false;
  return most_places(d, 16) >> 31 == 0;
}

}  // namespace

extern "C" size_t fdy_tree_attention_workspace_bytes(const fdy_draft* h) {
  if (!h || !sizes_valid(*h)) return 0;
  // for as many shares and rows as any call has
  const u32 rows = h->kv.head_dim <= 128 ? 8 * 32 : 8 * 16, shares = kCus;  // (twice the shares have half the rows)
  return kSplitBytes + ((size_t)shares * 2 * part_floats(rows, h->kv.head_dim) * 4 + 255) / 256 * 256;
}

extern "C" int fdy_tree_attention(const fdy_draft* h, void* d_workspace, size_t workspace_bytes, uint32_t* d_status, void* stream) {
  if (!h || !sizes_valid(*h)) return FDY_ERR_INVALID_ARG;
  const fdy_draft& d = *h;
  if (d.n_seqs == 0 || d.n_tokens == 0) return FDY_OK;
  if (!d.q || !d.out || !d.table || !d.lens || !d.kv.k || !d.kv.v) return FDY_ERR_INVALID_ARG;
  if (!aligned(d.q, 16) || !aligned(d.out, 16) || !aligned(d.kv.k, 16) || !aligned(d.kv.v, 16) || !aligned(d.lse, 4) ||
      !aligned(d.table, 4) || !aligned(d.lens, 4) || !aligned(d.rows, 4) || !aligned(d.first, 4) || !aligned(d.sees, 8) ||
      !aligned(d.kv.k_scale, 4) || !aligned(d.kv.v_scale, 4))
    return FDY_ERR_INVALID_ARG;
  if ((d.q_token | d.q_head | d.out_token | d.out_head) % 8) return FDY_ERR_INVALID_ARG;
  if ((d.kv.page_stride | d.kv.token_stride | d.kv.head_stride) % (d.kv.type == FDY_F8 ? 16 : 8)) return FDY_ERR_INVALID_ARG;
  if (!d_workspace || !aligned(d_workspace, 256) || workspace_bytes < fdy_tree_attention_workspace_bytes(h)) return FDY_ERR_WORKSPACE;
  Tree a{};
  a.d = d;
  if (d.window >> 31) a.d.window = 0;  // rows have fewer tokens
  a.status = d_status;
  a.splits = (Split*)d_workspace;
  a.parts = (float*)((uint8_t*)d_workspace + kSplitBytes);
  a.page_shift = log2_of(d.kv.page_tokens);
  a.group = d.n_q_heads / d.kv.n_heads;
  const bool f8 = d.kv.type == FDY_F8;
  if (d.type == FDY_BF16)
    return f8 ? launch_tree<Bf16, true>(a, (hipStream_t)stream) : launch_tree<Bf16, false>(a, (hipStream_t)stream);
  return f8 ? launch_tree<F16, true>(a, (hipStream_t)stream) : launch_tree<F16, false>(a, (hipStream_t)stream);
}
