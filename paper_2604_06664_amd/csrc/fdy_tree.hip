// fdy_tree.hip - attention of several drafted tokens of every sequence over its pages, each with its own view of the others.
//
// The same sum as for one new token (fdy_attention.hip), with drafted tokens x query heads as the query rows of a cache head: a
// tile's 16 (32) rows are any of them, its keys and values are read once for all.  A few drafted tokens are still bounded by
// memory; from about 200 rows on by the matrix cores and by the vector unit, which has the weights to work out.
//
// What a row sees differs only in the row's last c tokens (and where a window begins): tiles elsewhere need no masks.  Where
// rows see different tokens, a value that is no number would come out of the product with weight 0 as NaN in rows that do not see it;
// such values are taken out of the product and added to the rows that see them one by one.
#include "fdy_attend.hpp"

using namespace fdy;

namespace {

struct TreeArg {
  fdy_draft d;
  u32* status;
  u32* counters;  // [shares], zero between calls; a unit in parts has its first share's
  float* parts;   // [shares][2] of: [rows][head_dim] sums, [rows] pairs of a maximum and a sum of e; 16-byte aligned
  u32 page_shift, group;
};
typedef Arg<TreeArg> Tree;

// ---- which work a workgroup takes -------------------------------------------------------------------
// The query rows of a cache head (drafted tokens x query heads, kRows of them a tile) go to `together` waves side by side, as many
// times as they need (`groups`); the waves that are left over take other tokens: `apart` tiles of 32 tokens a round.
// A unit is one such group of one cache head of one sequence; units lie one after the other on a line, kEach places and then a place
// for every round, and equal shares of the line go to the workgroups.  Groups of one cache head, which read the same, are next to
// each other.
struct Seq {
  Span span;        // tokens that any of its queries sees
  u32 query, count;  // its first drafted token in q, and how many
  int base;         // tokens ahead of them
  u32 rows, together, groups, rounds;
  __device__ u32 unit() const { return rounds + kEach; }
};
__device__ __forceinline__ Seq uniform(const Seq& v) {
  Seq q;
  q.span.first = fdy::uniform(v.span.first), q.span.end = fdy::uniform(v.span.end), q.span.row = fdy::uniform(v.span.row);
  q.span.bad = v.span.bad;
  q.query = fdy::uniform(v.query), q.count = fdy::uniform(v.count), q.base = (int)fdy::uniform((u32)v.base);
  q.rows = fdy::uniform(v.rows), q.together = fdy::uniform(v.together), q.groups = fdy::uniform(v.groups);
  q.rounds = fdy::uniform(v.rounds);
  return q;
}

template <u32 kRows, u32 kWaves>
__device__ __forceinline__ Seq seq_of(const Tree& a, u32 s) {
  Seq q;
  q.span.row = a.d.rows ? (u32)a.d.rows[s] : s;
  q.span.bad = q.span.row >= a.d.n_rows;
  if (q.span.bad) q.span.row = 0;
  int n = q.span.bad ? 0 : a.d.lens[q.span.row];
  const u32 most = a.d.row_pages << a.page_shift;
  if (n < 0 || (u32)n > most) q.span.bad = true, n = n < 0 ? 0 : (int)most;
  u32 from = s * a.d.max_draft, to = from + a.d.max_draft;
  if (a.d.first) from = (u32)a.d.first[s], to = (u32)a.d.first[s + 1];
  q.query = from, q.count = to - from;
  if (to < from || to > a.d.n_tokens || q.count > a.d.max_draft) q.span.bad = true, q.count = 0;
  if (q.count > (u32)n && n >= 0) q.span.bad = true;
  q.base = n - (int)q.count;
  q.span.end = q.count ? (u32)n : 0;
  q.span.first = a.d.window && q.base > 0 && (u32)q.base > a.d.window ? (u32)q.base - a.d.window : 0;
  q.rows = q.count * a.group;
  const u32 tiles = (q.rows + kRows - 1) / kRows;
  q.together = 1;
  while (q.together < kWaves && q.together < tiles) q.together *= 2;
  q.groups = (tiles + q.together - 1) / q.together;
  const u32 apart = kWaves / q.together;
  q.rounds = (q.span.tiles() + apart - 1) / apart;
  return q;
}

struct TreeShare {
  u32 begin, end, per;  // places
  u32 seq, start;       // the sequence at `begin`, and its own place
  u32 at;
};
template <u32 kWaves>
struct TreeLds {
  u32 sum[kWaves], seq, start;
};

// All threads of the workgroup.
template <u32 kRows, u32 kWaves>
__device__ __forceinline__ bool find_tree_share(const Tree& a, TreeShare& out, TreeLds<kWaves>& lds) {
  constexpr u32 kThreads = 64 * kWaves;
  const u32 n = a.d.n_seqs, tid = threadIdx.x, slice = (n + kThreads - 1) / kThreads;
  const u32 s0 = min(tid * slice, n), s1 = min(s0 + slice, n);
  auto cost = [&](u32 s) {
    const Seq q = seq_of<kRows, kWaves>(a, s);
    if (q.span.bad && q.count == 0 && blockIdx.x == 0) raise_status(a.status, FDY_ST_BAD_INDEX);  // no one else looks at it
    return a.d.kv.n_heads * q.groups * q.unit();
  };
  u32 mine = 0;
  for (u32 s = s0; s < s1; ++s) mine += cost(s);
  const u32 inc = wave_incl_scan(mine);
  if (lane_id() == 63) lds.sum[tid >> 6] = inc;
  __syncthreads();
  u32 before = inc - mine, total = 0;
#pragma unroll
  for (u32 w = 0; w < kWaves; ++w) {
    if (w < tid >> 6) before += lds.sum[w];
    total += lds.sum[w];
  }
  total = fdy::uniform(total);
  if (total == 0) return false;
  // dies take workgroups in turn: neighbours on the line, which read the same keys and values, go to one
  const u32 g = gridDim.x;
  out.at = g % 8 ? blockIdx.x : blockIdx.x % 8 * (g / 8) + blockIdx.x / 8;
  out.per = max((total - 1) / g + 1, kEach + 1);
  if ((u64)out.at * out.per >= total) return false;
  out.begin = out.at * out.per;
  out.end = total - out.begin > out.per ? out.begin + out.per : total;
  if (out.begin >= before && out.begin < before + mine) {
    u32 s = s0;
    for (;; ++s) {
      const u32 c = cost(s);
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
template <typename T, bool kF8>
__device__ __forceinline__ u32 odd_mask(u32 w) {  // all bits of each element of the word that is infinite or no number
  if (kF8) {
    u32 m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if ((w >> 8 * i & 0x7f) == 0x7f) m |= 0xffu << 8 * i;
    return m;
  }
  constexpr u32 kExp = sizeof(typename T::elem) == 2 && __is_same(T, Bf16) ? 0x7f80u : 0x7c00u;
  return ((w & kExp) == kExp ? 0xffffu : 0) | ((w >> 16 & kExp) == kExp ? 0xffff0000u : 0);
}

// ---- the kernel -------------------------------------------------------------------------------------
constexpr u32 resident(int dim, u32 waves) { return dim <= 128 ? 8 / waves : 1; }

template <typename T, bool kF8, int kDim, bool kSmall, int kPolicy, int kTiles, u32 kWaves>
__global__ void __launch_bounds__(64 * kWaves, resident(kDim, kWaves)) tree_kernel(Tree a) {
  typedef Tile<T, kF8, kDim, kSmall, kPolicy> Tl;
  typedef typename T::x8 x8;
  typedef typename T::elem elem;
  constexpr int kWide = Tl::kWide, kParts = Tl::kParts, kSteps = Tl::kSteps, kPad = kDim + 4;
  constexpr u32 kRows = 16 * kTiles, kThreads = 64 * kWaves;
  __shared__ alignas(16) float s_o[kWaves][kRows][kPad];
  __shared__ float s_m[kWaves][kRows], s_l[kWaves][kRows];
  __shared__ TreeLds<kWaves> s_share;
  __shared__ u32 s_last;

  TreeShare share;
  if (!find_tree_share<kRows, kWaves>(a, share, s_share)) return;
  const u32 wave = fdy::uniform(threadIdx.x >> 6), D = a.d.kv.head_dim, quads = D / 4, H = a.d.kv.n_heads;
  const u32 part_size = part_floats(kRows * kWaves, D);
  const auto parts = buffer(a.parts, gridDim.x * 2 * part_size * 4);  // within 2^30 bytes

  u32 seq = share.seq, seq_start = share.start;
  Seq q = uniform(seq_of<kRows, kWaves>(a, seq));
  for (u32 place = share.begin; place < share.end;) {
    while (place - seq_start >= H * q.groups * q.unit()) {
      seq_start += H * q.groups * q.unit();
      q = uniform(seq_of<kRows, kWaves>(a, ++seq));
    }
    const u32 unit = fdy::uniform((place - seq_start) / q.unit()), u_start = seq_start + unit * q.unit(), start = u_start + kEach;
    const u32 next = u_start + q.unit();
    place = next;
    const u32 lo = start > share.begin ? start : share.begin, hi = next < share.end ? next : share.end;
    if (q.rounds ? lo >= hi : u_start < share.begin) continue;
    const bool whole = !q.rounds || (lo == start && hi == next);
    const u32 together = q.together, apart = kWaves / together, turn = wave / together;
    const u32 head = fdy::uniform(unit / q.groups), row0 = unit % q.groups * together * kRows;  // of the workgroup's rows
    const u32 q0 = row0 + wave % together * kRows;                                         // of the wave's
    bool bad = q.span.bad;

    // the factor of the scores, made positive (its sign goes to the queries)
    const float factor = a.d.scale * (kF8 && a.d.kv.k_scale ? a.d.kv.k_scale[head] : 1.f) * kLog2e;
    const float scale = factor == 0.f ? 1.f : fabsf(factor);
    const u32 q_keep = factor == 0.f ? 0u : ~0u, q_flip = factor < 0.f ? 0x80008000u : 0u;
    typename Tl::Lanes z;
    Tl::lanes(a, head, z);

    x8 qs[kTiles][kSteps];
    View view[kTiles];
#pragma unroll
    for (int qt = 0; qt < kTiles; ++qt) {
      const u32 r = q0 + qt * 16 + z.col, j = r / a.group, h = r - j * a.group;
      const bool there = r < q.rows;
      const elem* src = (const elem*)a.d.q + (u64)(q.query + j) * a.d.q_token + (u64)(head * a.group + h) * a.d.q_head;
#pragma unroll
      for (int st = 0; st < kSteps; ++st) {
        const u32 e = kF8 ? (st / 2) * 64 + z.grp * 16 + (st & 1) * 8 : st * 32 + z.grp * 8;
        v4u32 w = 0;
        if (there && e < D) w = *(const v4u32*)(src + e);
        qs[qt][st] = __builtin_bit_cast(x8, (w & q_keep) ^ q_flip);
      }
      view[qt] = view_of(a, q, there ? j : 0);
    }

    f32x4 o[kTiles][kParts * kWide];
    float m[kTiles], sum[kTiles];
#pragma unroll
    for (int qt = 0; qt < kTiles; ++qt) {
      m[qt] = -INFINITY, sum[qt] = 0.f;
#pragma unroll
      for (int i = 0; i < kParts * kWide; ++i) o[qt][i] = 0;
    }

    const u32 tile0 = q.span.first / kTile, tiles = q.span.tiles();
    const u32 begin = (lo - start) * apart, end = (hi - start) * apart < tiles ? (hi - start) * apart : tiles;
    const u32 t_end = fdy::uniform((tile0 + end) * kTile), t_step = apart * kTile;
    u32 t = fdy::uniform((tile0 + begin + turn) * kTile);
    // tiles in which rows see different tokens, or tokens are not there
    const int past = q.base, opens = a.d.window ? (int)(q.span.end - a.d.window) : 0;
    if (q.rounds && t < t_end && q0 < q.rows) {
      Tl x;
      typename Tl::Ids ids = Tl::ids(a, q.span, t, bad);
      x.load_k(a, z, q.span, ids, t, bad);
      x.load_v(a, z, q.span, ids, t, bad);
      for (; t < t_end; t += t_step) {
        const u32 t_next = t + t_step < t_end ? t + t_step : 0x7fffffc0u;  // behind every row
        const typename Tl::Ids ids_next = Tl::ids(a, q.span, t_next, bad);
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
        const bool mixed = kSmall || (int)(t + kTile) > past || (int)t < opens || (ids.page[0] | ids.page[1]) == ~0u;
        bool odd = false;
        u32 shown[kTiles];
        if (mixed) {
          u32 there = 0;
#pragma unroll
          for (int j = 0; j < 8; ++j) there |= x.seen(a, z, q.span, ids, t, j / 4, j % 4) ? 1u << j : 0;
#pragma unroll
          for (int qt = 0; qt < kTiles; ++qt) {
            const int tok = (int)(t + z.grp * 4);
            shown[qt] = there & (sees4(a, q, view[qt], tok) | sees4(a, q, view[qt], tok + 16) << 4);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[qt][j / 4][j % 4] = shown[qt] >> j & 1 ? s[qt][j / 4][j % 4] : -INFINITY;
          }
          u32 any = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int pt = 0; pt < kParts; ++pt)
#pragma unroll
              for (int k = 0; k < (int)sizeof(typename Tl::vword) / 4; ++k) any |= odd_mask<T, kF8>(word(x.v[i][pt], k));
          odd = ballot(any != 0) != 0;
        }
        x8 p[kTiles], rest[kTiles];
        float keep[kTiles], weight[kTiles][8];
#pragma unroll
        for (int qt = 0; qt < kTiles; ++qt) {
          float mx = s[qt][0][0];
#pragma unroll
          for (int j = 1; j < 8; ++j) mx = fmaxf(mx, s[qt][j / 4][j % 4]);
          const float m_new = fmaxf(m[qt], over_groups(mx, larger)), ref = m_new == -INFINITY ? 0.f : m_new;
          keep[qt] = __builtin_amdgcn_exp2f((m[qt] - ref) * scale);
          m[qt] = m_new;
          float part = 0.f;
          v4u32 first_of, rest_of;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[qt][j / 2][2 * j % 4] - ref, scale, kLift<T>));
            const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[qt][j / 2][2 * j % 4 + 1] - ref, scale, kLift<T>));
            part += e0 + e1;
            weight[qt][2 * j] = e0, weight[qt][2 * j + 1] = e1;
            u32 hi_of, lo_of;
            split<T>(e0, e1, hi_of, lo_of);
            first_of[j] = hi_of, rest_of[j] = lo_of;
          }
          p[qt] = __builtin_bit_cast(x8, first_of), rest[qt] = __builtin_bit_cast(x8, rest_of);
          sum[qt] = sum[qt] * keep[qt] + part;
        }
        if (odd) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int pt = 0; pt < kParts; ++pt) {
              if constexpr (sizeof(typename Tl::vword) == 4) {
                x.v[i][pt] &= ~odd_mask<T, kF8>(x.v[i][pt]);
              } else {
#pragma unroll
                for (int k = 0; k < (int)sizeof(typename Tl::vword) / 4; ++k) x.v[i][pt][k] &= ~odd_mask<T, kF8>(x.v[i][pt][k]);
              }
            }
        }
#pragma unroll
        for (int pt = 0; pt < kParts; ++pt)
#pragma unroll
          for (int e2 = 0; e2 < kWide / 2; ++e2) {
            x8 even, odd_e;
            x.values(pt, e2, even, odd_e);
#pragma unroll
            for (int qt = 0; qt < kTiles; ++qt) {
              f32x4& c0 = o[qt][pt * kWide + 2 * e2];
              f32x4& c1 = o[qt][pt * kWide + 2 * e2 + 1];
              c0 = mfma<T>(even, p[qt], c0 * keep[qt]);
              c1 = mfma<T>(odd_e, p[qt], c1 * keep[qt]);
              c0 = mfma<T>(even, rest[qt], c0);
              c1 = mfma<T>(odd_e, rest[qt], c1);
            }
          }
        if (odd) {  // the elements that were taken out, to the rows that see them
          for (u32 i = 0; i < kTile; ++i) {
            const u32 tok = t + i, in_half = i & 15, slot = (i >> 4) * 4 + (in_half & 3), owner = in_half >> 2;
            if (tok - q.span.first >= q.span.end - q.span.first) continue;
            const u32 page = (u32)a.d.table[(u64)q.span.row * a.d.row_pages + (tok >> a.page_shift)];
            if (page >= a.d.kv.n_pages) continue;
            const uint8_t* from = (const uint8_t*)a.d.kv.v + Tl::place(a, z, page, tok);
            float w[kTiles];
#pragma unroll
            for (int qt = 0; qt < kTiles; ++qt) {
              float mine = -1.f;  // not seen
#pragma unroll
              for (u32 j = 0; j < 8; ++j)
                if (j == slot && (shown[qt] >> j & 1)) mine = weight[qt][j];
              w[qt] = __shfl(mine, (int)(z.col + 16 * owner));
            }
#pragma unroll
            for (int pt = 0; pt < kParts; ++pt)
#pragma unroll
              for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int e = 0; e < kWide; ++e) {
                  const u32 d = pt * 16 * kWide + (z.grp * 4 + k) * kWide + e;
                  if (d >= D) continue;
                  float y;
                  if (kF8) {
                    y = (from[d] & 0x7f) == 0x7f ? NAN : 0.f;
                  } else {
                    y = (float)((const elem*)from)[d];
                  }
                  if (__builtin_isfinite(y)) continue;
#pragma unroll
                  for (int qt = 0; qt < kTiles; ++qt)
                    if (!(w[qt] < 0.f)) o[qt][pt * kWide + e][k] += w[qt] * y;
                }
          }
        }
        x.load_v(a, z, q.span, ids_next, t_next, bad);
        ids = ids_next;
      }
    }
    if (ballot(bad) && lane_id() == 0) raise_status(a.status, FDY_ST_BAD_INDEX);

    // the waves' sums, joined
#pragma unroll
    for (int qt = 0; qt < kTiles; ++qt) {
      sum[qt] = over_groups(sum[qt], plus);
#pragma unroll
      for (int pt = 0; pt < kParts; ++pt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < kWide; ++e)
            s_o[wave][qt * 16 + z.col][pt * 16 * kWide + (z.grp * 4 + i) * kWide + e] = o[qt][pt * kWide + e][i];
      if (z.grp == 0) s_m[wave][qt * 16 + z.col] = m[qt] * scale - kLift<T>, s_l[wave][qt * 16 + z.col] = sum[qt];
    }
    __syncthreads();
    const u32 items = together * kRows * quads;  // item i: four elements of a row
    auto finish = [&](u32 r, u32 qd, float M, float L, f32x4 y) {
      const u32 j = (row0 + r) / a.group, h = head * a.group + (row0 + r) - j * a.group;
      const float v_scale = kF8 && a.d.kv.v_scale ? a.d.kv.v_scale[head] : 1.f;
      y = y * (L == 0.f ? 0.f : v_scale / L);
      typedef elem x4 __attribute__((ext_vector_type(4)));
      *(x4*)((elem*)a.d.out + (u64)(q.query + j) * a.d.out_token + (u64)h * a.d.out_head + qd * 4) = __builtin_convertvector(y, x4);
      if (qd == 0 && a.d.lse)
        a.d.lse[(u64)(q.query + j) * a.d.n_q_heads + h] = L == 0.f ? -INFINITY : (M + __builtin_log2f(L)) * kLn2;
    };
    for (u32 i = threadIdx.x; i < items; i += kThreads) {
      const u32 r = i / quads, qd = i - r * quads, c = r / kRows, in = r % kRows;
      if (row0 + r >= q.rows) continue;
      float M = -INFINITY;
      for (u32 w = c; w < kWaves; w += together) M = fmaxf(M, s_m[w][in]);
      const float ref = M == -INFINITY ? 0.f : M;
      float L = 0.f;
      f32x4 y = 0;
      for (u32 w = c; w < kWaves; w += together) {
        const float f = __builtin_amdgcn_exp2f(s_m[w][in] - ref);
        L += f * s_l[w][in];
        y += f * *(const f32x4*)&s_o[w][in][qd * 4];
      }
      if (whole) {
        finish(r, qd, ref, L, y);
      } else {
        const u32 mine = (share.at * 2 + (start > share.begin)) * part_size;
        put_part(parts, mine + r * D + qd * 4, y);
        if (qd == 0) put_part(parts, mine + kRows * kWaves * D + 2 * r, M, L);
      }
    }
    if (whole) {
      __syncthreads();  // the next unit's sums go where these lay
      continue;
    }

    // the unit's parts, joined by the workgroup that finishes last; its counter is left at zero
    const u32 first = start / share.per, n_parts = (next - 1) / share.per - first + 1;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's part has arrived where all workgroups see it
    __syncthreads();
    if (threadIdx.x == 0) {
      const u32 before = __hip_atomic_fetch_add(a.counters + first, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      s_last = before == n_parts - 1;
      if (s_last) __hip_atomic_store(a.counters + first, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!s_last) continue;  // (s_last is written again only behind the next unit's barriers)
    const bool second = start > first * share.per;
    for (u32 i = threadIdx.x; i < items; i += kThreads) {
      const u32 r = i / quads, qd = i - r * quads;
      if (row0 + r >= q.rows) continue;
      float M = -INFINITY, L = 0.f;
      f32x4 y = 0;
      for (u32 k0 = 0; k0 < n_parts; k0 += 4) {
        f32x4 part[4];
        v2u32 ml[4];
#pragma unroll
        for (u32 j = 0; j < 4; ++j) {
          const u32 k = k0 + j < n_parts ? k0 + j : k0, from = ((first + k) * 2 + (k == 0 && second)) * part_size;
          part[j] = get_part4(parts, from + r * D + qd * 4);
          ml[j] = get_part2(parts, from + kRows * kWaves * D + 2 * r);
        }
        float top = M;
#pragma unroll
        for (u32 j = 0; j < 4; ++j) top = fmaxf(top, as_float(ml[j].x));
        const float ref = top == -INFINITY ? 0.f : top, keep = __builtin_amdgcn_exp2f(M - ref);
        y *= keep, L *= keep, M = top;
#pragma unroll
        for (u32 j = 0; j < 4; ++j)
          if (k0 + j < n_parts) {
            const float f = __builtin_amdgcn_exp2f(as_float(ml[j].x) - ref);
            L += f * as_float(ml[j].y);
            y += f * part[j];
          }
      }
      finish(r, qd, M == -INFINITY ? 0.f : M, L, y);
    }
  }
}

// Workgroups: as many as are resident together, fewer where there are not the rounds.
u64 row_tiles(const fdy_draft& d) { return ((u64)d.row_pages * d.kv.page_tokens + kTile - 1) / kTile; }
u64 most_places(const fdy_draft& d, u32 rows) {
  const u64 tiles = ((u64)d.max_draft * (d.n_q_heads / d.kv.n_heads) + rows - 1) / rows;
  return d.n_seqs * d.kv.n_heads * tiles * (row_tiles(d) + 2 + kEach);
}
constexpr u32 kMostShares = kCus * 2;
constexpr size_t kCounterBytes = kMostShares * 4;

template <typename T, bool kF8, int kDim>
int launch_tree(const Tree& a, hipStream_t stream) {
  (void)hipGetLastError();  // drop any stale error left by earlier, unrelated runtime calls
  auto go = [&](auto kernel, u32 waves) {
    u64 shares = kCus * resident(kDim, waves);
    const u64 most = most_places(a.d, 16) / (kEach + 1) + 1;
    if (shares > most) shares = most;
    hipLaunchKernelGGL(kernel, dim3((u32)shares), dim3(64 * waves), 0, stream, a);
  };
  // 32 rows a wave, 16 where their sums would not fit the registers, where pages are small or where there are no more
  constexpr int kTwo = kDim <= 128 || kF8 ? 2 : 1, kOnce = kNonTemporal;
  constexpr u32 kMost = kDim <= 128 ? 8 : 4;
  const u32 rows = a.d.max_draft * a.group;
  if (a.d.kv.page_tokens < 16)
    go(tree_kernel<T, kF8, kDim, true, 0, 1, 4>, 4);
  else if (rows <= 16)
    go(tree_kernel<T, kF8, kDim, false, kOnce, 1, kMost>, kMost);
  else if (rows <= 16 * kTwo)
    go(tree_kernel<T, kF8, kDim, false, kOnce, kTwo, kMost>, kMost);
  else
    go(tree_kernel<T, kF8, kDim, false, 0, kTwo, kMost>, kMost);
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
  const u32 rows = h->kv.head_dim <= 128 ? 8 * 32 : 4 * 32, shares = kCus;
  return kCounterBytes + ((size_t)shares * 2 * part_floats(rows, h->kv.head_dim) * 4 + 255) / 256 * 256;
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
  a.counters = (u32*)d_workspace;
  a.parts = (float*)((uint8_t*)d_workspace + kCounterBytes);
  a.page_shift = log2_of(d.kv.page_tokens);
  a.group = d.n_q_heads / d.kv.n_heads;
  const bool f8 = d.kv.type == FDY_F8;
  if (d.type == FDY_BF16)
    return f8 ? launch_tree<Bf16, true>(a, (hipStream_t)stream) : launch_tree<Bf16, false>(a, (hipStream_t)stream);
  return f8 ? launch_tree<F16, true>(a, (hipStream_t)stream) : launch_tree<F16, false>(a, (hipStream_t)stream);
}
