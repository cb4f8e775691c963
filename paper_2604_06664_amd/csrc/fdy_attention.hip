// fdy_attention.hip - attention of one new token of every sequence over its pages, split over the length and joined.
//
// out = sum_t e^(x_t) v_t / sum_t e^(x_t), x_t = scale k_t.q, in one pass over the keys and values with a running maximum
// and sum.  All query heads of a cache head read the same keys and values, a flop a byte each (two in 8 bits): the bound is memory, and
// the matrix cores only keep the arithmetic out of its way (a tile holds 16 query heads of a cache head, a wave one or two of them).
//
// A wave takes 32 tokens at a time, straight from the pages into the operands, no LDS in the loop:
//   S^T = K Q^T   lane l holds key row l % 16 (of 16 tokens) and the elements of group l / 16; the sums come out with a
//                 query head a lane column and tokens 4 (l / 16) + i in the lane's four registers,
//   O^T = V^T P^T whose second operand wants, for the lane's query head, eight tokens: these same registers of the two
//                 16-token halves, once the products' inner index runs over tokens in that order.  Its first operand wants
//                 the same eight tokens of one element of v in a lane: the lane loads eight tokens by eight elements and
//                 transposes them in registers (v_perm).
// A query head's maximum, sum and output all lie in one lane column, so rescaling needs no exchange but the maximum over the
// four groups.  Four or eight waves take the tiles of a piece in turn and join in LDS; the pieces of a row are joined by whichever
// workgroup finishes last.
#include "fdy_attend.hpp"

using namespace fdy;

namespace {

struct AttendArg {
  fdy_attend d;
  u32* status;
  u32* counters;  // [shares][columns], zero between calls; a row in parts has its first share's
  float* parts;   // [shares][columns][2] of: [rows][head_dim] sums, [rows] pairs of a maximum and a sum of e; 16-byte aligned
  // columns: cache heads x q_tiles; rows: query heads of a tile; together, may_together: columns that a workgroup takes at once
  // where there is much to do, and at most
  u32 page_shift, group, q_tiles, columns, rows, together, may_together;
  u32 eight;  // waves of a workgroup are eight, not four
  u32 lists;  // of pages a row: 1, or one for each cache head
  u32 fill;
};
typedef Arg<AttendArg> Attend;

// The rows' tiles lie one after the other on a line, kEach places ahead of each row's; equal shares of the line go to the
// workgroups of a column.  So all of them have the same to do whatever the lengths are, and a row is in as many parts as
// shares reach into it.
//
// A workgroup takes one column, its waves every fourth or eighth tile, or two or four columns, as many waves as that leaves to
// each.  Where there is much to do it takes four (with less of it two) if the heads of a token lie side by side: one head's
// keys are 128 or 256 bytes at every n_heads-th place, and memory gives less of them than of four heads' as one piece (8 heads,
// 4,096 tokens a row: 128 rows in 8 bits 231 us alone, 193 in twos, 177 in fours; 64 rows in 16 bits 191, 173 and 171; 16 rows
// 58 alone and 53 in twos; 33 rows of 1,024 and 256 elements 49, 46 and, in fours, where a share is short and a row in many parts, 51).
//
// Where there is little, time goes by what happens one after the other: rows of few tiles are in one part, and every row has a
// workgroup of its own if they are enough with four columns each at most (64 rows of up to 200 tokens 17 us without, 11 with;
// 512 rows of up to 90, which are more than workgroups, 43 and 29).
struct Share {
  u32 begin, end, per;  // places
  u32 seq, start;       // the row at `begin`, and its own place
  u32 seq_end;          // rows that there are for the share, for a row of no tiles does not reach a share's end
  u32 at, column, together;
  u32 whole;            // tiles up to which a row is one part, its who has its first tile
};
constexpr u32 kMuch = 16, kSome = 2, kLittle = 5;  // tiles of a wave
constexpr u32 kWhole = 8;                         // tiles of a row

template <u32 kWaves>
struct ShareLds {
  u32 sum[kWaves], most[kWaves], seq, start;
};

// All threads of the workgroup.
template <u32 kWaves>
__device__ __forceinline__ bool find_share(const Attend& a, Share& out, ShareLds<kWaves>& lds) {
  constexpr u32 kThreads = 64 * kWaves;
  const u32 n = a.d.n_seqs, tid = threadIdx.x, slice = (n + kThreads - 1) / kThreads;
  const u32 s0 = tid * slice, s1 = s0 + slice < n ? s0 + slice : n;
  u32 mine = 0, most = 0, before = 0, total = 0;
  if (n == 1) {
    most = span_of(a, 0).tiles();
    total = most + kEach;
  } else {
    for (u32 s = s0; s < s1; ++s) {
      const u32 t = span_of(a, s).tiles();
      mine += t + kEach, most = max(most, t);
    }
    const u32 inc = wave_incl_scan(mine);
    most = wave_incl_most(most);
    if (lane_id() == 63) lds.sum[tid >> 6] = inc, lds.most[tid >> 6] = most;
    __syncthreads();
    before = inc - mine;
    most = 0;
#pragma unroll
    for (u32 w = 0; w < kWaves; ++w) {
      if (w < tid >> 6) before += lds.sum[w];
      total += lds.sum[w], most = max(most, lds.most[w]);
    }
  }
  total = uniform(total), most = uniform(most);
  const u64 waves = (u64)gridDim.x * kWaves, tiles = (u64)(total - n * kEach) * a.columns;
  const bool much = tiles >= waves * kMuch, little = tiles < waves * kLittle;
  out.together = much ? a.together : tiles >= waves * kSome && a.together > 1 ? 2 : 1;
  u32 columns = a.columns / out.together, shares = gridDim.x / columns;
  if (little)
    while (n > shares && out.together < a.may_together) out.together *= 2, columns /= 2, shares *= 2;
  out.at = blockIdx.x / columns, out.column = blockIdx.x % columns * out.together;
  out.whole = little ? kWhole : 0;
  out.seq = 0, out.start = 0, out.seq_end = n;
  if (little && n <= shares && most <= kWhole) {  // a row each
    out.seq = out.at, out.seq_end = out.at + 1, out.per = 1;
    out.begin = 0, out.end = kEach + 1;
    return out.at < n;
  }
  const u32 least = kWaves / out.together + kEach;
  out.per = max((total - 1) / shares + 1, least);
  if (out.at >= shares || (u64)out.at * out.per >= total) return false;
  out.begin = out.at * out.per;
  out.end = total - out.begin > out.per ? out.begin + out.per : total;
  if (n == 1) return true;
  if (out.begin >= before && out.begin < before + mine) {
    u32 s = s0;
    for (;; ++s) {
      const u32 cost = span_of(a, s).tiles() + kEach;
      if (out.begin < before + cost) break;
      before += cost;
    }
    lds.seq = s, lds.start = before;
  }
  __syncthreads();
  out.seq = uniform(lds.seq), out.start = uniform(lds.start);
  return true;
}

// ---- the kernel -----------------------------------------------------------------------------------------
// Workgroups of a compute unit that are launched, and that the registers leave room for.  More do not help: of rows of 4,096
// tokens in 8 bits, three of four waves give 4.6 TB/s where two give 5.1; and one more of 128 elements in 16 bits leaves 168 registers and
// a few spills, whose reloads wait behind all keys and values under way (2.1 TB/s).
//
// Eight waves of one workgroup do the work of two workgroups of four in half as many parts and with less of a tail, as all waves
// of a compute unit end together (see `lay_out`).  Of 256 elements in 16 bits four waves have all the registers, and are alone.
constexpr u32 resident(int dim, u32 waves) { return dim <= 128 ? 8 / waves : 1; }

// kTiles: tiles of 16 query heads a workgroup, for one read of their keys and values (64 rows of 8,192 tokens, 32 heads of one
// cache head, workgroups of four waves: of 128 elements 77 us with one for each 16, 73 so; of 64 elements, two cache heads, 81 and 66;
// with eight waves 62 and 58.  What is left above the read is the parts' 16 KiB a workgroup, written through to memory by all at once).
template <typename T, bool kF8, int kDim, bool kSmall, int kPolicy, int kTiles, u32 kWaves>
__global__ void __launch_bounds__(64 * kWaves, resident(kDim, kWaves)) attend_kernel(Attend a) {
  typedef Tile<T, kF8, kDim, kSmall, kPolicy> Tl;
  typedef typename T::x8 x8;
  typedef typename T::elem elem;
  constexpr int kWide = Tl::kWide, kParts = Tl::kParts, kSteps = Tl::kSteps, kPad = kDim + 4;
  constexpr u32 kRows = 16 * kTiles, kThreads = 64 * kWaves;
  constexpr int kPair = kTiles == 2 && (kF8 || kDim <= 64) ? 2 : 1;  // (128 elements in 16 bits would spill)
  __shared__ alignas(16) float s_o[kWaves][kRows][kPad];
  __shared__ float s_m[kWaves][kRows], s_l[kWaves][kRows];
  __shared__ ShareLds<kWaves> s_share;
  __shared__ u32 s_last;

  Share share;
  if (!find_share(a, share, s_share)) return;
  const u32 together = share.together, apart = kWaves / together;  // `apart`: waves of a column
  const u32 wave = threadIdx.x >> 6, turn = uniform(wave / together), column = uniform(share.column + wave % together);
  const u32 head = column / a.q_tiles, q0 = column % a.q_tiles * a.rows;
  const u32 D = a.d.kv.head_dim, quads = D / 4, part_size = part_floats(a.rows, D);
  const auto parts = buffer(a.parts, gridDim.x * a.may_together * 2 * part_size * 4);  // within 2^30 bytes
  // the factor of the scores, made positive (its sign goes to the queries; where it is 0 they are 0, too), so that the largest
  // score is the one of the largest product and masked ones stay minus infinity
  const float factor = a.d.scale * (kF8 && a.d.kv.k_scale ? a.d.kv.k_scale[head] : 1.f) * kLog2e;
  const float scale = factor == 0.f ? 1.f : fabsf(factor);
  const u32 q_keep = factor == 0.f ? 0u : ~0u, q_flip = factor < 0.f ? 0x80008000u : 0u;
  typename Tl::Lanes z;
  Tl::lanes(a, head, z);

  u32 next = share.start;
  for (u32 seq = share.seq; seq < share.seq_end && next < share.end; ++seq) {
    const u32 first_place = next, start = next + kEach;  // places of the row, and of its first tile
    Span span = span_of(a, seq);
    span.first = uniform(span.first), span.end = uniform(span.end), span.row = uniform(span.row);
    const u32 all = span.tiles();
    bool bad = span.bad;
    if (a.lists > 1) span.row = span.row * a.lists + head;
    next = start + all;
    // the tiles of the row that lie in the share; a row of none is its who has the row's first place
    u32 lo = start > share.begin ? start : share.begin, hi = next < share.end ? next : share.end;
    if (all && all <= share.whole) {
      if (start < share.begin || start >= share.end) continue;
      lo = start, hi = next;
    }
    if (all ? lo >= hi : first_place < share.begin) continue;
    const u32 tile0 = span.first / kTile, begin = tile0 + lo - start, end = all ? tile0 + hi - start : begin;
    const bool whole = !all || (lo == start && hi == next);

    // the tiles' queries as the products' second operand: the same elements a lane as its keys
    x8 q[kTiles][kSteps];
#pragma unroll
    for (int qt = 0; qt < kTiles; ++qt) {
      const u32 h = q0 + qt * 16 + z.col;
      const elem* src = (const elem*)a.d.q + seq * a.d.q_seq + (head * a.group + h) * a.d.q_head;
#pragma unroll
      for (int st = 0; st < kSteps; ++st) {
        const u32 e = kF8 ? (st / 2) * 64 + z.grp * 16 + (st & 1) * 8 : st * 32 + z.grp * 8;
        v4u32 w = 0;
        if (h < a.group && qt * 16 + z.col < a.rows && e < D) w = *(const v4u32*)(src + e);
        q[qt][st] = __builtin_bit_cast(x8, (w & q_keep) ^ q_flip);
      }
    }

    f32x4 o[kTiles][kParts * kWide];
    float m[kTiles], sum[kTiles];
#pragma unroll
    for (int qt = 0; qt < kTiles; ++qt) {
      m[qt] = -INFINITY, sum[qt] = 0.f;
#pragma unroll
      for (int i = 0; i < kParts * kWide; ++i) o[qt][i] = 0;
    }

    // keys of the next tile are asked for as soon as this one's are used up, values likewise: there is always as much under
    // way as the registers hold
    const u32 t_end = end * kTile, t_step = apart * kTile;
    u32 t = uniform((begin + turn) * kTile);
    if (t < t_end) {
      Tl x;
      typename Tl::Ids ids = Tl::ids(a, span, t, bad);
      x.load_k(a, z, span, ids, t, bad);
      x.load_v(a, z, span, ids, t, bad);
      for (; t < t_end; t += t_step) {
        const u32 t_next = t + t_step < t_end ? t + t_step : 0x7fffffc0u;  // behind every row
        typename Tl::Ids ids_next = Tl::ids(a, span, t_next, bad);
        f32x4 s[kTiles][2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
          for (int qt = 0; qt < kTiles; ++qt) s[qt][u] = 0;
#pragma unroll
          for (int st = 0; st < kSteps; ++st) {
            const x8 key = x.key(u, st);
#pragma unroll
            for (int qt = 0; qt < kTiles; ++qt) s[qt][u] = mfma<T>(key, q[qt][st], s[qt][u]);
          }
        }
        x.load_k(a, z, span, ids_next, t_next, bad);
        bool seen[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) seen[j] = x.seen(a, z, span, ids, t, j / 4, j % 4);
        x8 p[kTiles], rest[kTiles];
        float keep[kTiles];
#pragma unroll
        for (int qt = 0; qt < kTiles; ++qt) {
          float y[8];  // the lane's products, those without a key at minus infinity
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = seen[j] ? s[qt][j / 4][j % 4] : -INFINITY;
          float mx = y[0];
#pragma unroll
          for (int j = 1; j < 8; ++j) mx = fmaxf(mx, y[j]);
          // The maximum is kept of the products, and the factor is applied to differences from it: the largest weight is
          // 1 (2^15 in f16) whatever the size of the scores.  (Of scores of 2^30 and more the rounding of `product * factor` is worth e^64.)
          const float m_new = fmaxf(m[qt], over_groups(mx, larger)), ref = m_new == -INFINITY ? 0.f : m_new;
          keep[qt] = __builtin_amdgcn_exp2f((m[qt] - ref) * scale);
          m[qt] = m_new;
          float part = 0.f;
          v4u32 first_of, rest_of;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(y[2 * j] - ref, scale, kLift<T>));
            const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(y[2 * j + 1] - ref, scale, kLift<T>));
            part += e0 + e1;
            u32 a, b;
            split<T>(e0, e1, a, b);
            first_of[j] = a, rest_of[j] = b;
          }
          p[qt] = __builtin_bit_cast(x8, first_of), rest[qt] = __builtin_bit_cast(x8, rest_of);
          sum[qt] = sum[qt] * keep[qt] + part;
        }
#pragma unroll
        for (int pt = 0; pt < kParts; ++pt)
#pragma unroll
          for (int e2 = 0; e2 < kWide / 2; ++e2) {
            x8 even, odd;
            x.values(pt, e2, even, odd);
#pragma unroll
            for (int qt = 0; qt < kTiles; ++qt) {
              f32x4& c0 = o[qt][pt * kWide + 2 * e2];
              f32x4& c1 = o[qt][pt * kWide + 2 * e2 + 1];
              c0 = mfma<T>(even, p[qt], c0 * keep[qt]);
              c1 = mfma<T>(odd, p[qt], c1 * keep[qt]);
              c0 = mfma<T>(even, rest[qt], c0);
              c1 = mfma<T>(odd, rest[qt], c1);
            }
          }
        x.load_v(a, z, span, ids_next, t_next, bad);
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
    // item i: four elements (from 4 qd on) of query head r of column c of the workgroup's
    struct Item {
      u32 c, r, qd;
      bool there;
    };
    const u32 items = together * a.rows * quads;
    auto item = [&](u32 i) {
      Item it;
      const u32 row = i / quads;
      it.qd = i - row * quads, it.c = row / a.rows, it.r = row - it.c * a.rows;
      it.there = i < items && (share.column + it.c) % a.q_tiles * a.rows + it.r < a.group;
      return it;
    };
    auto finish = [&](const Item& it, float M, float L, f32x4 x) {
      const u32 col = share.column + it.c, kv_head = col / a.q_tiles;
      const u32 h = kv_head * a.group + col % a.q_tiles * a.rows + it.r;
      const float v_scale = kF8 && a.d.kv.v_scale ? a.d.kv.v_scale[kv_head] : 1.f;
      x = x * (L == 0.f ? 0.f : v_scale / L);
      elem* out = (elem*)a.d.out + seq * a.d.out_seq + h * a.d.out_head + it.qd * 4;
      typedef elem x4 __attribute__((ext_vector_type(4)));
      *(x4*)out = __builtin_convertvector(x, x4);
      if (it.qd == 0 && a.d.lse) a.d.lse[(u64)seq * a.d.n_q_heads + h] = L == 0.f ? -INFINITY : (M + __builtin_log2f(L)) * kLn2;
    };
    // where a share's part of a column lies: its second where the row begins within the share
    auto part_at = [&](u32 share_no, u32 c, bool second) {
      return ((share_no * a.columns + share.column + c) * 2 + second) * part_size;
    };
    for (u32 i = threadIdx.x; i < items; i += kThreads) {
      const Item it = item(i);
      if (!it.there) continue;
      float M = -INFINITY;
      for (u32 w = it.c; w < kWaves; w += together) M = fmaxf(M, s_m[w][it.r]);
      const float ref = M == -INFINITY ? 0.f : M;
      float L = 0.f;
      f32x4 x = 0;
      for (u32 w = it.c; w < kWaves; w += together) {
        const float f = __builtin_amdgcn_exp2f(s_m[w][it.r] - ref);
        L += f * s_l[w][it.r];
        x += f * *(const f32x4*)&s_o[w][it.r][it.qd * 4];
      }
      if (whole) {
        finish(it, ref, L, x);
      } else {
        const u32 mine = part_at(share.at, it.c, start > share.begin);
        put_part(parts, mine + it.r * D + it.qd * 4, x);
        if (it.qd == 0) put_part(parts, mine + a.rows * D + 2 * it.r, M, L);
      }
    }
    if (whole) {
      __syncthreads();  // the next row's sums go where these lay
      continue;
    }

    // the row's parts, joined by the workgroup that finishes last; its counter is left at zero
    const u32 first = start / share.per, n_parts = (next - 1) / share.per - first + 1;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's part has arrived where all workgroups see it
    __syncthreads();
    if (threadIdx.x == 0) {
      u32* counter = a.counters + first * a.columns + share.column;  // no other row goes on from that share to the next
      const u32 before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      s_last = before == n_parts - 1;
      if (s_last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!s_last) continue;  // (s_last is written again only behind the next row's barriers)
    const bool second = start > first * share.per;
    // `crews` of threads take every crews-th part each, or kPair items at once where there are more than threads, eight parts'
    // loads of each under way: what comes from another die takes microseconds
    const u32 crews = items >= kThreads ? 1 : kThreads / items;
    for (u32 i0 = 0; i0 < items; i0 += kThreads * kPair) {
      const u32 crew = crews > 1 ? threadIdx.x / items : 0, i = i0 + threadIdx.x - crew * items;
      Item it[kPair];
      bool works[kPair];
      float M[kPair], L[kPair];
      f32x4 x[kPair];
#pragma unroll
      for (int g = 0; g < kPair; ++g) {
        it[g] = item(i + kThreads * g);
        works[g] = it[g].there && (g ? crews == 1 : crew < crews);
        M[g] = -INFINITY, L[g] = 0.f, x[g] = 0;
      }
      if (works[0]) {
        for (u32 k0 = crew; k0 < n_parts; k0 += crews * 8) {
          f32x4 y[kPair][8];
          v2u32 ml[kPair][8];
#pragma unroll
          for (int g = 0; g < kPair; ++g)
            if (g == 0 || works[g])
#pragma unroll
              for (u32 j = 0; j < 8; ++j) {
                const u32 k = k0 + j * crews < n_parts ? k0 + j * crews : k0, from = part_at(first + k, it[g].c, k == 0 && second);
                y[g][j] = get_part4(parts, from + it[g].r * D + it[g].qd * 4);
                ml[g][j] = get_part2(parts, from + a.rows * D + 2 * it[g].r);
              }
#pragma unroll
          for (int g = 0; g < kPair; ++g)
            if (g == 0 || works[g]) {
              float top = M[g];
#pragma unroll
              for (u32 j = 0; j < 8; ++j) top = fmaxf(top, as_float(ml[g][j].x));
              const float ref = top == -INFINITY ? 0.f : top, keep = __builtin_amdgcn_exp2f(M[g] - ref);
              x[g] *= keep, L[g] *= keep, M[g] = top;
#pragma unroll
              for (u32 j = 0; j < 8; ++j)
                if (k0 + j * crews < n_parts) {
                  const float f = __builtin_amdgcn_exp2f(as_float(ml[g][j].x) - ref);
                  L[g] += f * as_float(ml[g][j].y);
                  x[g] += f * y[g][j];
                }
            }
        }
      }
      if (crews > 1) {  // the crews' sums, in their order
        float(*c_x)[4] = (float(*)[4])s_o;
        float(*c_ml)[2] = (float(*)[2])(c_x + kThreads);
        if (works[0]) *(f32x4*)c_x[threadIdx.x] = x[0], c_ml[threadIdx.x][0] = M[0], c_ml[threadIdx.x][1] = L[0];
        __syncthreads();
        if (works[0] && crew == 0) {
          float top = M[0];
          for (u32 c = 1; c < crews; ++c) top = fmaxf(top, c_ml[c * items + i][0]);
          const float ref = top == -INFINITY ? 0.f : top;
          float f = __builtin_amdgcn_exp2f(M[0] - ref);
          x[0] *= f, L[0] *= f, M[0] = top;
          for (u32 c = 1; c < crews; ++c) {
            f = __builtin_amdgcn_exp2f(c_ml[c * items + i][0] - ref);
            L[0] += f * c_ml[c * items + i][1];
            x[0] += f * *(const f32x4*)c_x[c * items + i];
          }
        }
      }
#pragma unroll
      for (int g = 0; g < kPair; ++g)
        if (works[g] && crew == 0) finish(it[g], M[g] == -INFINITY ? 0.f : M[g], L[g], x[g]);
    }
    __syncthreads();  // the next row's sums go where the crews' lay
  }
}

// As many workgroups as are resident together, fewer where the longest rows that the table allows have not the tiles; a
// multiple of the columns.
u64 row_tiles(const fdy_attend& d) { return ((u64)d.row_pages * d.kv.page_tokens + kTile - 1) / kTile; }
u32 blocks_of(const Attend& a, u32 waves) {
  u64 shares = kCus * resident((int)a.d.kv.head_dim, waves) / a.columns;
  const u64 places = a.d.n_seqs * (row_tiles(a.d) + 1 + kEach);
  const u64 most = places / (waves + kEach) + 1 + a.d.n_seqs;
  if (shares > most) shares = most;
  return (u32)(shares < 1 ? 1 : shares) * a.columns;
}

template <typename T, bool kF8, int kDim>
int launch_attend(const Attend& a, hipStream_t stream) {
  (void)hipGetLastError();  // drop any stale error left by earlier, unrelated runtime calls
  auto go = [&](auto kernel, u32 waves) {
    hipLaunchKernelGGL(kernel, dim3(blocks_of(a, waves)), dim3(64 * waves), 0, stream, a);
  };
  constexpr int kTwo = kDim <= 128 || kF8 ? 2 : 1, kOnce = kNonTemporal;
  constexpr u32 kMost = kDim <= 128 || kF8 ? 8 : 4, kMostTwo = kDim <= 128 ? 8 : 4;
  if (a.d.kv.page_tokens < 16)
    go(attend_kernel<T, kF8, kDim, true, 0, 1, 4>, 4);
  else if (a.eight && a.q_tiles == 1)
    a.rows > 16 ? go(attend_kernel<T, kF8, kDim, false, kOnce, kTwo, kMostTwo>, kMostTwo) : go(attend_kernel<T, kF8, kDim, false, kOnce, 1, kMost>, kMost);
  else if (a.eight)
    a.rows > 16 ? go(attend_kernel<T, kF8, kDim, false, 0, kTwo, kMostTwo>, kMostTwo) : go(attend_kernel<T, kF8, kDim, false, 0, 1, kMost>, kMost);
  else if (a.q_tiles == 1)
    a.rows > 16 ? go(attend_kernel<T, kF8, kDim, false, kOnce, kTwo, 4>, 4) : go(attend_kernel<T, kF8, kDim, false, kOnce, 1, 4>, 4);
  else
    a.rows > 16 ? go(attend_kernel<T, kF8, kDim, false, 0, kTwo, 4>, 4) : go(attend_kernel<T, kF8, kDim, false, 0, 1, 4>, 4);
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
  const u64 most = (u64)d.row_pages * d.kv.page_tokens;
  return most < 1ull << 31 && d.n_seqs * most <= 1ull << 36;
}

// How the call is laid out; the same for the workspace's size and the launch.
void lay_out(const fdy_attend& d, bool lists, Attend& a) {
  a.d = d;
  a.lists = lists ? d.kv.n_heads : 1;
  a.page_shift = log2_of(d.kv.page_tokens);
  a.group = d.n_q_heads / d.kv.n_heads;
  // 32 query heads of a cache head go together; 16 where their sums would not fit the registers, where pages are small, or where
  // tiles of 16 are fewer (40 heads of one, 64 rows of 4,096 tokens in 8 bits, four waves: 61 us, and 74 as two times 20)
  const bool two = d.kv.page_tokens >= 16 && (d.kv.head_dim <= 128 || d.kv.type == FDY_F8) && (a.group + 31) / 32 * 2 == (a.group + 15) / 16;
  const u32 rows = two ? 32 : 16;
  a.q_tiles = (a.group + rows - 1) / rows;
  a.columns = d.kv.n_heads * a.q_tiles;
  a.rows = (a.group + a.q_tiles - 1) / a.q_tiles;
  a.may_together = a.columns % 4 == 0 ? 4 : a.columns % 2 == 0 ? 2 : 1;
  // heads that lie side by side in a token, and query heads of one cache head, go together
  const bool beside = (d.kv.head_stride < d.kv.token_stride && a.lists == 1) || a.q_tiles > 1;
  a.together = beside ? a.may_together : 1;
  // Eight waves a workgroup where the tables allow much (the lengths are not known here) and a token's heads lie together: 64 rows
  // of 1,024 tokens 48 us, with four 58; 128 of 4,096 in 8 bits 176 and 206; 32 of 512 18 and 23; 8 of 8,192 with one cache head
  // 35 and 57.  Four where it is little (8 rows of 300 to 900 tokens 15, with eight 19; 64 of 20 to 200 11 and 13) or the heads
  // lie apart (64 of 4,096 160 and 165); of 256 elements eight are too many for the registers in 16 bits, for LDS with 32 query heads
  const u64 tiles = row_tiles(d), all = tiles * d.n_seqs * a.columns, waves = kCus * 8;
  a.eight = (d.kv.head_dim <= 128 || (d.kv.type == FDY_F8 && a.rows <= 16)) && d.kv.page_tokens >= 16 &&
            (d.kv.head_stride <= d.kv.token_stride || a.q_tiles > 1) && (tiles >= 256 || (tiles >= 16 && all >= waves * 2));
}
// For as many shares as there can be, so that it does not depend on the rows: calls for more and for fewer find their counters at
// the same place, and neither's parts there.
size_t counter_bytes(const Attend& a) {
  const size_t blocks = a.columns > kCus * 2 ? a.columns : kCus * 2;
  return (blocks * a.may_together * 4 + 255) / 256 * 256;
}

size_t workspace_bytes_of(const fdy_attend* h, bool lists) {
  if (!h || !sizes_valid(*h) || (lists && (u64)h->n_rows * h->kv.n_heads >> 31)) return 0;
  Attend a{};
  lay_out(*h, lists, a);
  // (four waves' workgroups, which are more: a call for fewer rows or narrower tables may take these)
  const size_t parts = (size_t)blocks_of(a, 4) * a.may_together * 2 * part_floats(a.rows, h->kv.head_dim) * 4;
  return counter_bytes(a) + (parts + 255) / 256 * 256;
}

int attention(const fdy_attend* h, bool lists, void* d_workspace, size_t workspace_bytes, uint32_t* d_status, void* stream) {
  const size_t need = workspace_bytes_of(h, lists);
  if (!need) return FDY_ERR_INVALID_ARG;
  const fdy_attend& d = *h;
  if (d.n_seqs == 0) return FDY_OK;
  if (!d.q || !d.out || !d.table || !d.lens || !d.kv.k || !d.kv.v) return FDY_ERR_INVALID_ARG;
  if (!aligned(d.q, 16) || !aligned(d.out, 16) || !aligned(d.kv.k, 16) || !aligned(d.kv.v, 16) || !aligned(d.lse, 4) ||
      !aligned(d.table, 4) || !aligned(d.lens, 4) || !aligned(d.rows, 4) || !aligned(d.kv.k_scale, 4) || !aligned(d.kv.v_scale, 4))
    return FDY_ERR_INVALID_ARG;
  if ((d.q_seq | d.q_head | d.out_seq | d.out_head) % 8) return FDY_ERR_INVALID_ARG;
  if ((d.kv.page_stride | d.kv.token_stride | d.kv.head_stride) % (d.kv.type == FDY_F8 ? 16 : 8)) return FDY_ERR_INVALID_ARG;
  if (!d_workspace || !aligned(d_workspace, 256) || workspace_bytes < need)
    return FDY_ERR_WORKSPACE;
  Attend a{};
  lay_out(d, lists, a);
  a.status = d_status;
  a.counters = (u32*)d_workspace;
  a.parts = (float*)((uint8_t*)d_workspace + counter_bytes(a));
  const bool f8 = d.kv.type == FDY_F8;
  if (d.type == FDY_BF16)
    return f8 ? launch_attend<Bf16, true>(a, (hipStream_t)stream) : launch_attend<Bf16, false>(a, (hipStream_t)stream);
  return f8 ? launch_attend<F16, true>(a, (hipStream_t)stream) : launch_attend<F16, false>(a, (hipStream_t)stream);
}

}  // namespace

extern "C" size_t fdy_paged_attention_workspace_bytes(const fdy_attend* h) { return workspace_bytes_of(h, false); }

extern "C" int fdy_paged_attention(const fdy_attend* h, void* d_workspace, size_t workspace_bytes, uint32_t* d_status,
                                   void* stream) {
  return attention(h, false, d_workspace, workspace_bytes, d_status, stream);
}

extern "C" size_t fdy_selected_attention_workspace_bytes(const fdy_attend* h) { return workspace_bytes_of(h, true); }

extern "C" int fdy_selected_attention(const fdy_attend* h, void* d_workspace, size_t workspace_bytes, uint32_t* d_status,
                                      void* stream) {
  return attention(h, true, d_workspace, workspace_bytes, d_status, stream);
}
