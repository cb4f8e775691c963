// fdy_pages.hip - keeping the pages of a cache: taking, sharing, giving up, copying and compacting them.
//
// The books (holders of each page, a bitmap of the free ones, the rows' tables and lengths) are small against the contents:
// what the calls wait for is a few dependent reads of the books, and the bytes of the pages that they copy.  Results do not
// depend on the order in which atomics arrive: free pages are a set (bits), counts of holders are sums, and where order
// matters (who takes which page) it follows from prefix sums over the list.
#include "fdy_types.hpp"

using namespace fdy;

namespace {

constexpr u32 kMostEntries = 65536, kBooksThreads = 1024;

struct PagesArg {
  fdy_pages d;
  u32* status;
  const int32_t* from;  // lists of the call: rows or pages
  const int32_t* to;
  int64_t* slots;
  int32_t* positions;
  int32_t* map;
  u32* n_live;
  u32* ws;  // words of the workspace, laid out by each call
  u32 n, n_slots, shift, slices, pieces;  // pieces: of a page in a plane
  u32 fill;
};
typedef Arg<PagesArg> Pages;

__device__ __forceinline__ u32 fresh(const u32* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ u32 pages_of(const Pages& a, u32 tokens) { return (tokens + a.d.page_tokens - 1) >> a.shift; }

// A row's length, held within its table; `bad` where it is not.
__device__ __forceinline__ u32 length_of(const Pages& a, u32 row, bool& bad) {
  const int n = a.d.lens[row];
  const u32 most = a.d.row_pages << a.shift;
  if (n >= 0 && (u32)n <= most) return (u32)n;
  bad = true;
  return n < 0 ? 0 : most;
}

template <typename A>
__device__ __forceinline__ void set_free(const A& a, u32 page) {
  atomicOr((u32*)a.d.free_bits + (page >> 5), 1u << (page & 31));
}

// One holder less; nobody left: the page is free.  False: nobody held it.
template <typename A>
__device__ __forceinline__ bool drop(const A& a, u32 page) {
  const u32 before = atomicSub(a.d.refs + page, 1u);
  if (before == 1) set_free(a, page);
  if (before == 0) atomicAdd(a.d.refs + page, 1u);
  return before != 0;
}

// Whether an earlier entry of the list names the same row (all threads of a workgroup take part).
__device__ __forceinline__ bool named_before(const int32_t* list, u32 i) {
  const int row = list[i];
  bool found = false;
  for (u32 j = threadIdx.x; j < i; j += blockDim.x) found |= list[j] == row;
  return __syncthreads_or(found);
}

// One piece of a page's contents in one plane, by the threads of a workgroup: two 16-byte loads each under way.  The bound is
// memory.  Stores are marked as not to be kept, which what is copied (read a step later at the earliest) does not need: 25,920
// pages for an extend 180 us without, 168 with; loads are marked where no page is a source twice (184 us where three beams
// copy one page).
constexpr u32 kPiece = 256 * 2 * 16;
template <bool kOnce>
__device__ __forceinline__ void copy_piece(const Pages& a, u32 plane, u32 src, u32 dst, u32 piece) {
  const u64 base = a.d.planes[plane], at = (u64)piece * kPiece, left = a.d.page_bytes - at;
  const u32 n = (u32)(left < kPiece ? left : kPiece), i = threadIdx.x * 16;
  const auto s = buffer((const void*)(base + src * a.d.page_stride + at), n), d = buffer((const void*)(base + dst * a.d.page_stride + at), n);
  v4u32 x[2];
#pragma unroll
  for (u32 j = 0; j < 2; ++j) x[j] = __builtin_amdgcn_raw_buffer_load_b128(s, i + j * 4096, 0, kOnce ? kNonTemporal : 0);
#pragma unroll
  for (u32 j = 0; j < 2; ++j) __builtin_amdgcn_raw_buffer_store_b128(x[j], d, i + j * 4096, 0, kNonTemporal);
}

// ---- reset ------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(256) pages_reset_kernel(Pages a) {
  const u32 words = (a.d.n_pages + 63) / 64, most = a.d.n_pages > a.d.n_rows ? a.d.n_pages : a.d.n_rows;
  for (u32 i = blockIdx.x * 256 + threadIdx.x; i < most; i += gridDim.x * 256) {
    if (i < a.d.n_pages) a.d.refs[i] = 0;
    if (i < a.d.n_rows) a.d.lens[i] = 0;
    if (i < words) a.d.free_bits[i] = i + 1 < words || a.d.n_pages % 64 == 0 ? ~0ull : (1ull << a.d.n_pages % 64) - 1;
  }
}

// ---- extend -----------------------------------------------------------------------------------------
// Words of the workspace: per row who names it first, per page how many ask for it and who last, the pages taken, and per
// entry its first token, its row's length, its last page, its pages and their first number.
struct ExtendWords {
  u32 *claim, *asked, *latest, *taken, *begin, *length, *last, *need, *rank, *copy;
};
constexpr u32 kUnserved = 0x80000000u;  // of `length`
constexpr u32 kNoPage = ~0u;
constexpr u32 kCopies = 0x80000000u;  // of `need`
__host__ __device__ inline u64 extend_words(const fdy_pages& d, u32 n) { return (u64)d.n_rows + 3ull * d.n_pages + 6ull * n; }
__device__ __forceinline__ ExtendWords extend_layout(const Pages& a) {
  ExtendWords w;
  w.claim = a.ws;
  w.asked = w.claim + a.d.n_rows;
  w.latest = w.asked + a.d.n_pages;
  w.taken = w.latest + a.d.n_pages;
  w.begin = w.taken + a.d.n_pages;
  w.length = w.begin + a.n;
  w.last = w.length + a.n;
  w.need = w.last + a.n;
  w.rank = w.need + a.n;
  w.copy = w.rank + a.n;
  return w;
}

// What an entry of the list wants, and its pages' first number among those found.
struct Entry {
  u32 row, count, length, last, need, rank;
  u32 others;  // of one that keeps a shared page: up to which number of found pages the others' copies of it go, where pages are short
  bool copies, fits;
};

// Gives entry i its pages, if they were found, and writes its slot and position where it has one token.
template <typename Taken>
__device__ __forceinline__ void serve(const Pages& a, const ExtendWords& w, u32 i, const Entry& e, u32 found, Taken taken,
                                      u32* s_served, u32& wrong) {
  bool served = e.fits;
  // (one that keeps a page takes none, but the page is not its own as long as another has not got its copy)
  if (served && ((e.need && (u64)e.rank + e.need > found) || e.others > found)) wrong |= FDY_ST_CAPACITY, served = false;
  u32 copy = kNoPage;
  int32_t* table = a.d.table + (u64)(served ? e.row : 0) * a.d.row_pages;
  u32 at_end = kNoPage;  // page of the first new token
  if (served) {
    const u32 before = pages_of(a, e.length), end = e.rank + e.need;
    u32 at = e.rank;
    if (e.copies) {
      copy = taken(at);
      table[before - 1] = (int32_t)copy;
      atomicSub(a.d.refs + e.last, 1u);
      ++at;
    }
    for (u32 j = before; at < end; ++at, ++j) table[j] = (int32_t)taken(at);
    for (at = e.rank; at < end; ++at) a.d.refs[taken(at)] = 1;
    a.d.lens[e.row] = (int32_t)(e.length + e.count);
    if (e.need) {
      atomicMax(s_served, end);
      at_end = taken(e.rank);
    }
  }
  if (a.d.n_planes || a.to) {  // for the launch that follows
    w.copy[i] = copy;
    w.last[i] = e.last;
    w.length[i] = e.length | (served ? 0 : kUnserved);
  }
  if (!a.to && i < a.n_slots) {
    if (a.slots) {
      if (served && at_end == kNoPage) at_end = (u32)table[e.length >> a.shift];
      a.slots[i] = served ? (int64_t)at_end * a.d.page_tokens + e.length % a.d.page_tokens : -1;
    }
    if (a.positions) a.positions[i] = (int32_t)e.length;
  }
}

// One workgroup keeps the books.
__global__ void __launch_bounds__(kBooksThreads) extend_books_kernel(Pages a) {
  __shared__ u64 s_scan[17];
  __shared__ u32 s_served;
  const ExtendWords w = extend_layout(a);
  const u32 tid = threadIdx.x, pt = a.d.page_tokens, most = a.d.row_pages << a.shift;
  u32 wrong = 0;
  auto row_of = [&](u32 i) { return a.from ? (u32)a.from[i] : i; };
  if (tid == 0) s_served = 0;
  // who names a row first
  if (a.from) {
    for (u32 i = tid; i < a.n; i += kBooksThreads)
      if (row_of(i) < a.d.n_rows) w.claim[row_of(i)] = ~0u;
    __syncthreads();
    for (u32 i = tid; i < a.n; i += kBooksThreads)
      if (row_of(i) < a.d.n_rows) atomicMin(w.claim + row_of(i), i);
    __syncthreads();
  }
  // where the entries' tokens begin, whether they fit, and shared last pages
  u64 base = 0;
  for (u32 i0 = 0; i0 < a.n; i0 += kBooksThreads) {
    const u32 i = i0 + tid;
    int count = i < a.n ? (a.to ? a.to[i] : 1) : 0;
    if (count < 0) wrong |= FDY_ST_BAD_INDEX, count = 0;
    u64 sum;
    const u64 begin = base + block_excl_scan((u64)count, s_scan, sum);
    base += sum;
    if (i >= a.n) continue;
    const u32 row = row_of(i);
    bool good = row < a.d.n_rows && (!a.from || fresh(w.claim + row) == i);
    u32 length = 0, last = kNoPage;
    if (good) {
      bool bad = false;
      length = length_of(a, row, bad);
      if (length % pt) {
        last = (u32)a.d.table[(u64)row * a.d.row_pages + (length >> a.shift)];
        bad |= last >= a.d.n_pages;
      }
      if (bad) good = false, length = 0;
    }
    if (!good) wrong |= FDY_ST_BAD_INDEX;
    bool fits = good && count > 0;
    if (fits && ((u64)length + (u32)count > most || begin + (u32)count > a.n_slots)) wrong |= FDY_ST_CAPACITY, fits = false;
    if (!fits || (last != kNoPage && a.d.refs[last] <= 1)) last = kNoPage;
    if (last != kNoPage) w.asked[last] = 0, w.latest[last] = 0;
    w.begin[i] = begin < a.n_slots ? (u32)begin : a.n_slots;
    w.length[i] = length | (fits ? 0 : kUnserved);
    w.last[i] = last;
  }
  __syncthreads();
  for (u32 i = tid; i < a.n; i += kBooksThreads)
    if (w.last[i] != kNoPage) atomicAdd(w.asked + w.last[i], 1u), atomicMax(w.latest + w.last[i], i + 1);
  __syncthreads();
  // how many pages each wants; of those that hold a page among themselves alone the last keeps it
  u64 total = 0;
  for (u32 i0 = 0; i0 < a.n; i0 += kBooksThreads) {
    const u32 i = i0 + tid;
    u32 need = 0, copies = 0;
    if (i < a.n && !(w.length[i] & kUnserved)) {
      const u32 length = w.length[i], count = a.to ? (u32)a.to[i] : 1u, last = w.last[i];
      copies = last != kNoPage && !(fresh(w.asked + last) == a.d.refs[last] && fresh(w.latest + last) == i + 1);
      need = pages_of(a, length + count) - pages_of(a, length) + copies;
    }
    u64 sum;
    const u64 rank = total + block_excl_scan(need, s_scan, sum);
    total += sum;
    if (i < a.n) {
      w.need[i] = need | (copies ? kCopies : 0);
      w.rank[i] = rank < a.d.n_pages ? (u32)rank : a.d.n_pages;
    }
  }
  // that many free pages, lowest first
  u64 found = 0;
  const u32 words = (a.d.n_pages + 63) / 64;
  for (u32 w0 = 0; w0 < words && found < total; w0 += kBooksThreads) {
    u64 bits = w0 + tid < words ? a.d.free_bits[w0 + tid] : 0;
    if (w0 + tid == words - 1 && a.d.n_pages % 64) bits &= (1ull << a.d.n_pages % 64) - 1;
    u64 sum;
    u64 rank = found + block_excl_scan((u64)__popcll(bits), s_scan, sum);
    found += sum;
    for (; bits && rank < total; bits &= bits - 1) w.taken[rank++] = (w0 + tid) * 64 + (u32)__builtin_ctzll(bits);
  }
  if (found > total) found = total;
  auto keeps = [&](u32 i) { return w.last[i] != kNoPage && !(w.need[i] & kCopies); };
  if (found < total) {
    for (u32 i = tid; i < a.n; i += kBooksThreads)
      if (keeps(i)) w.asked[w.last[i]] = 0;
    __syncthreads();
    for (u32 i = tid; i < a.n; i += kBooksThreads)
      if (w.need[i] & kCopies) atomicMax(w.asked + w.last[i], w.rank[i] + (w.need[i] & ~kCopies));
  }
  __syncthreads();
  // the rows that get theirs
  for (u32 i = tid; i < a.n; i += kBooksThreads) {
    Entry e;
    e.others = found < total && keeps(i) ? fresh(w.asked + w.last[i]) : 0;
    e.row = row_of(i), e.count = a.to ? (u32)a.to[i] : 1u, e.length = w.length[i] & ~kUnserved, e.last = w.last[i];
    e.need = w.need[i] & ~kCopies, e.rank = w.rank[i], e.copies = w.need[i] & kCopies, e.fits = !(w.length[i] & kUnserved);
    serve(a, w, i, e, (u32)found, [&](u32 r) { return w.taken[r]; }, &s_served, wrong);
  }
  __syncthreads();
  for (u32 r = tid; r < s_served; r += kBooksThreads) {
    const u32 page = w.taken[r];
    atomicAnd((u32*)a.d.free_bits + (page >> 5), ~(1u << (page & 31)));
  }
  if (wrong) raise_status(a.status, wrong);
}

// The same for up to 1,024 entries, one a thread, which keeps what it knows in registers; who names a row first and who asks
// for a page are counted in LDS, by hashing (512 rows: 20 us through the workspace, 14 so).
constexpr u32 kHash = 2048, kTakenHere = 4096;
struct Counts {
  u32 key[kHash], sum[kHash], top[kHash];
};
__device__ __forceinline__ void clear(Counts& c) {
  for (u32 i = threadIdx.x; i < kHash; i += kBooksThreads) c.key[i] = ~0u, c.sum[i] = 0, c.top[i] = 0;
}
__device__ __forceinline__ u32 place_of(Counts& c, u32 key) {  // at most half full: ends
  u32 at = key * 0x9e3779b1u >> 21;
  for (;; at = (at + 1) % kHash) {
    const u32 there = atomicCAS(&c.key[at], ~0u, key);
    if (there == ~0u || there == key) return at;
  }
}

__global__ void __launch_bounds__(kBooksThreads) extend_few_kernel(Pages a) {
  __shared__ u64 s_scan[17];
  __shared__ Counts s_rows, s_pages;
  __shared__ u32 s_taken[kTakenHere];
  __shared__ u32 s_served;
  const ExtendWords w = extend_layout(a);
  const u32 i = threadIdx.x, pt = a.d.page_tokens, words = (a.d.n_pages + 63) / 64;
  u32 wrong = 0;
  u64 bits = i < words ? a.d.free_bits[i] : 0;  // the first pages' are asked for ahead of all else
  const bool there = i < a.n;
  Entry e{};
  e.last = kNoPage;
  e.row = there ? (a.from ? (u32)a.from[i] : i) : ~0u;
  int count = there ? (a.to ? a.to[i] : 1) : 0;
  if (count < 0) wrong |= FDY_ST_BAD_INDEX, count = 0;
  e.count = (u32)count;
  bool good = there && e.row < a.d.n_rows;
  if (good) {
    bool bad = false;
    e.length = length_of(a, e.row, bad);
    if (e.length % pt) {
      e.last = (u32)a.d.table[(u64)e.row * a.d.row_pages + (e.length >> a.shift)];
      bad |= e.last >= a.d.n_pages;
    }
    if (bad) good = false;
  }
  u32 holders = good && e.last != kNoPage ? a.d.refs[e.last] : 0;
  clear(s_pages);
  if (a.from) clear(s_rows);
  if (i == 0) s_served = 0;
  u64 sum, begin = i;
  if (a.to)
    begin = block_excl_scan(e.count, s_scan, sum);
  else
    __syncthreads();
  u32 row_at = 0;
  if (a.from) {
    if (there && e.row < a.d.n_rows) row_at = place_of(s_rows, e.row), atomicMax(&s_rows.top[row_at], a.n - i);
    __syncthreads();
    good = good && s_rows.top[row_at] == a.n - i;
  }
  if (!good) e.length = 0;
  if (there && !good) wrong |= FDY_ST_BAD_INDEX;
  e.fits = good && count > 0;
  if (e.fits && ((u64)e.length + e.count > a.d.row_pages << a.shift || begin + e.count > a.n_slots)) wrong |= FDY_ST_CAPACITY, e.fits = false;
  const bool shared = e.fits && e.last != kNoPage && holders > 1;
  if (!shared) e.last = kNoPage;
  u32 page_at = 0;
  if (shared) page_at = place_of(s_pages, e.last), atomicAdd(&s_pages.sum[page_at], 1u), atomicMax(&s_pages.top[page_at], i + 1);
  __syncthreads();
  e.copies = shared && !(s_pages.sum[page_at] == holders && s_pages.top[page_at] == i + 1);
  if (e.fits) e.need = pages_of(a, e.length + e.count) - pages_of(a, e.length) + e.copies;
  u64 total;
  const u64 rank = block_excl_scan(e.need, s_scan, total);
  e.rank = rank < a.d.n_pages ? (u32)rank : a.d.n_pages;
  u64 found = 0;
  for (u32 w0 = 0; w0 < words && found < total; w0 += kBooksThreads) {
    if (w0) bits = w0 + i < words ? a.d.free_bits[w0 + i] : 0;
    if (w0 + i == words - 1 && a.d.n_pages % 64) bits &= (1ull << a.d.n_pages % 64) - 1;
    u64 r = found + block_excl_scan((u64)__popcll(bits), s_scan, sum);
    found += sum;
    for (; bits && r < total; bits &= bits - 1, ++r) {
      const u32 page = (w0 + i) * 64 + (u32)__builtin_ctzll(bits);
      if (r < kTakenHere)
        s_taken[r] = page;
      else
        w.taken[r] = page;
    }
  }
  if (found > total) found = total;
  if (found < total) {
    const bool keeps = shared && !e.copies;
    if (keeps) s_pages.sum[page_at] = 0;
    __syncthreads();
    if (e.copies) atomicMax(&s_pages.sum[page_at], e.rank + e.need);
    __syncthreads();
    if (keeps) e.others = s_pages.sum[page_at];
  }
  __syncthreads();
  const auto taken = [&](u32 r) { return r < kTakenHere ? s_taken[r] : w.taken[r]; };
  if (there) {
    if (a.to) w.begin[i] = begin < a.n_slots ? (u32)begin : a.n_slots;
    serve(a, w, i, e, (u32)found, taken, &s_served, wrong);
  }
  __syncthreads();
  for (u32 r = i; r < s_served; r += kBooksThreads) {
    const u32 page = taken(r);
    atomicAnd((u32*)a.d.free_bits + (page >> 5), ~(1u << (page & 31)));
  }
  if (wrong) raise_status(a.status, wrong);
}

// The copies of shared pages, and the slots of entries of several tokens.
__global__ void __launch_bounds__(256) extend_copy_kernel(Pages a) {
  const ExtendWords w = extend_layout(a);
  const u32 i = blockIdx.x, copy = w.copy[i];
  if (copy != kNoPage) {
    const u32 src = w.last[i];
    for (u32 t = blockIdx.y; t < a.d.n_planes * a.pieces; t += gridDim.y) copy_piece<false>(a, t / a.pieces, src, copy, t % a.pieces);
  }
  if (!a.to || blockIdx.y) return;
  const u32 row = a.from ? (u32)a.from[i] : i;
  const int count = a.to[i];
  const bool served = !(w.length[i] & kUnserved);
  const u32 length = w.length[i] & ~kUnserved, begin = w.begin[i], pt = a.d.page_tokens;
  for (u32 j = threadIdx.x; (int)j < count && begin + j < a.n_slots; j += 256) {
    const u32 t = length + j;
    if (a.slots)
      a.slots[begin + j] = served ? (int64_t)a.d.table[(u64)row * a.d.row_pages + (t >> a.shift)] * pt + t % pt : -1;
    if (a.positions) a.positions[begin + j] = (int32_t)t;
  }
}

// ---- fork -------------------------------------------------------------------------------------------
// First all rows' pages are noted (and their holders counted up), then the rows are written (and holders counted down): a row
// may be both.  Pages that a row has at the same place before and after are left alone.
__host__ __device__ inline u64 fork_words(const fdy_pages& d, u32 n) { return (u64)n * d.row_pages + 2ull * n; }
constexpr u32 kForkPages = 1024;  // pages of a row a workgroup takes

__global__ void __launch_bounds__(256) fork_note_kernel(Pages a) {
  constexpr u32 kMine = kForkPages / 256;
  const u32 i = blockIdx.x, s = (u32)a.from[i], d = (u32)a.to[i], j0 = blockIdx.y * kForkPages + threadIdx.x;
  const bool in = s < a.d.n_rows && d < a.d.n_rows;
  u32* lens = a.ws + (u64)a.n * a.d.row_pages + 2 * i;
  // what the row holds and held is asked for before the list is searched
  bool bad = false;
  const u32 now = in ? length_of(a, s, bad) : 0, old = in ? length_of(a, d, bad) : 0, n = pages_of(a, now), n_old = pages_of(a, old);
  const int32_t *src = a.d.table + (u64)s * a.d.row_pages, *dst = a.d.table + (u64)d * a.d.row_pages;
  u32 p[kMine], q[kMine];
#pragma unroll
  for (u32 k = 0; k < kMine; ++k) {
    const u32 j = j0 + k * 256;
    p[k] = j < n ? (u32)src[j] : kNoPage;
    q[k] = j < n && j < n_old ? (u32)dst[j] : kNoPage;
  }
  if (!in || named_before(a.to, i)) {
    if (threadIdx.x == 0 && blockIdx.y == 0) lens[0] = kUnserved, raise_status(a.status, FDY_ST_BAD_INDEX);
    return;
  }
  if (threadIdx.x == 0 && blockIdx.y == 0) lens[0] = now, lens[1] = old;
  u32* noted = a.ws + (u64)i * a.d.row_pages;
#pragma unroll
  for (u32 k = 0; k < kMine; ++k) {
    const u32 j = j0 + k * 256;
    if (j >= n) break;
    noted[j] = p[k];
    if (p[k] == q[k] && j < n_old) continue;
    if (p[k] < a.d.n_pages)
      atomicAdd(a.d.refs + p[k], 1u);
    else
      bad = true;
  }
  if (bad) raise_status(a.status, FDY_ST_BAD_INDEX);
}

__global__ void __launch_bounds__(256) fork_write_kernel(Pages a) {
  const u32 i = blockIdx.x, d = (u32)a.to[i];
  const u32* lens = a.ws + (u64)a.n * a.d.row_pages + 2 * i;
  if (lens[0] == kUnserved) return;
  const u32 n = pages_of(a, lens[0]), n_old = pages_of(a, lens[1]), most = n > n_old ? n : n_old;
  int32_t* dst = a.d.table + (u64)d * a.d.row_pages;
  const u32* noted = a.ws + (u64)i * a.d.row_pages;
  bool bad = false;
  const u32 end = most < (blockIdx.y + 1) * kForkPages ? most : (blockIdx.y + 1) * kForkPages;
  for (u32 j = blockIdx.y * kForkPages + threadIdx.x; j < end; j += 256) {
    const u32 old = (u32)dst[j], p = j < n ? noted[j] : kNoPage;
    if (j < n && j < n_old && old == p) continue;
    if (j < n_old && (old >= a.d.n_pages || !drop(a, old))) bad = true;
    if (j < n) dst[j] = (int32_t)p;
  }
  if (threadIdx.x == 0 && blockIdx.y == 0) a.d.lens[d] = (int32_t)lens[0];
  if (bad) raise_status(a.status, FDY_ST_BAD_INDEX);
}

// ---- free -------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(256) free_kernel(Pages a) {
  const u32 i = blockIdx.x, r = (u32)a.from[i];
  if (r >= a.d.n_rows || named_before(a.from, i)) {
    if (threadIdx.x == 0) raise_status(a.status, FDY_ST_BAD_INDEX);
    return;
  }
  bool bad = false;
  const u32 n = pages_of(a, length_of(a, r, bad));
  const int32_t* table = a.d.table + (u64)r * a.d.row_pages;
  for (u32 j = threadIdx.x; j < n; j += 256) {
    const u32 p = (u32)table[j];
    if (p >= a.d.n_pages || !drop(a, p)) bad = true;
  }
  __syncthreads();  // the length has been read by all
  if (threadIdx.x == 0) a.d.lens[r] = 0;
  if (bad) raise_status(a.status, FDY_ST_BAD_INDEX);
}

// ---- keep -------------------------------------------------------------------------------------------
// First all rows are looked at (a row is served or not by what was there before the call), then tokens move and books change.
// Words of the workspace, an entry: first token that moves (kUnserved: the row stays as it is), tokens ahead of the drafted
// ones, tokens that stay, and the row's length.
struct KeepArg {
  fdy_pages d;
  fdy_token t;
  u32* status;
  const int32_t *rows, *drafts, *keep, *kept;
  u32* ws;
  u32 n, most, shift, columns;  // columns: 16-byte words of a token in a plane
};
typedef Arg<KeepArg> Keep;

__global__ void __launch_bounds__(1024) keep_plan_kernel(Keep a) {
  __shared__ u32 s_moves;
  const u32 i = blockIdx.x, r = (u32)a.rows[i], tid = threadIdx.x;
  const int drafts = a.drafts[i], kept = a.kept[i];
  u32* plan = a.ws + 4 * i;
  u32 wrong = 0;
  if (tid == 0) s_moves = kept > 0 ? (u32)kept : 0;
  __syncthreads();
  bool bad = r >= a.d.n_rows || named_before(a.rows, i);
  u32 n = 0;
  if (!bad) n = (u32)a.d.lens[r], bad = n > a.d.row_pages << a.shift;
  bad = bad || drafts < 0 || (u32)drafts > n || kept < 0 || kept > drafts || (u32)kept > a.most;
  if (!bad) {
    const u32 base = n - (u32)drafts;
    const int32_t *keep = a.keep + (u64)i * a.most, *table = a.d.table + (u64)r * a.d.row_pages;
    for (u32 j = tid; j < (u32)kept; j += blockDim.x) {
      const int k = keep[j], before = j ? keep[j - 1] : -1;
      if (k <= before || k >= drafts) {
        wrong |= FDY_ST_BAD_INDEX;
      } else if ((u32)k != j) {  // it moves (from the first such on all do)
        atomicMin(&s_moves, j);
        const u32 from = (u32)table[(base + (u32)k) >> a.shift], to = (u32)table[(base + j) >> a.shift];
        if (from >= a.d.n_pages || to >= a.d.n_pages)
          wrong |= FDY_ST_BAD_INDEX;
        else if (a.d.refs[to] > 1)
          wrong |= FDY_ST_CAPACITY;
      }
    }
    const u32 in_page = a.d.page_tokens - 1;
    for (u32 j = ((base + (u32)kept + in_page) >> a.shift) + tid; j < (n + in_page) >> a.shift; j += blockDim.x)  // those given up
      if ((u32)table[j] >= a.d.n_pages) wrong |= FDY_ST_BAD_INDEX;
  }
  if (bad) wrong = FDY_ST_BAD_INDEX;
  const bool refused = __syncthreads_or((int)(wrong & FDY_ST_BAD_INDEX)), shared = __syncthreads_or((int)(wrong & FDY_ST_CAPACITY));
  if (tid) return;
  if (refused || shared) raise_status(a.status, refused ? FDY_ST_BAD_INDEX : FDY_ST_CAPACITY);
  plan[0] = refused || shared ? kUnserved : s_moves;
  plan[1] = n - (u32)drafts, plan[2] = (u32)kept, plan[3] = n;
}

// Where all sources lie behind all places that are written to, every 16-byte word of every token goes by itself, a workgroup
// kMoved * 256 of a plane's.  Otherwise a lane takes one word of the row's tokens in one plane and moves it for one token after
// the other, so that a place is read before it is written to: tokens only move to the front.  kSerial of them are under way together.
// Memory bounds it where many move (1.05 GB read + written 236 us, 4.4 TB/s); few are a chain of the plan, page numbers, words and stores
// (64 paths of 4 tokens of 2 KiB in 72 planes: 22 us; several planes a workgroup 24, one division of 64 bits less no change).
constexpr u32 kMoved = 4, kSerial = 16;
__global__ void __launch_bounds__(256) keep_move_kernel(Keep a) {
  const u32 i = blockIdx.x;
  const u32* plan = a.ws + 4 * i;
  const u32 begin = uniform(plan[0]), base = uniform(plan[1]), kept = uniform(plan[2]), n = uniform(plan[3]);
  if (begin == kUnserved) return;
  const u32 r = (u32)a.rows[i], in_page = a.d.page_tokens - 1;
  const int32_t *table = a.d.table + (u64)r * a.d.row_pages, *keep = a.keep + (u64)i * a.most;
  const u32 words = a.t.piece_bytes / 16;
  auto place = [&](u64 plane, u32 token, u32 piece, u32 word) {
    return (v4u32*)((uint8_t*)plane + (u32)table[token >> a.shift] * a.d.page_stride + (token & in_page) * a.t.token_stride +
                    piece * a.t.piece_stride + word * 16);
  };
  const u32 moves = kept - begin;
  if (begin < kept && a.d.n_planes && (u32)keep[begin] >= kept && !((u64)moves * words >> 32)) {
    const u64 of_plane = (u64)moves * a.columns;
    const u32 chunks = (u32)((of_plane + kMoved * 256 - 1) / (kMoved * 256));
    for (u64 c = blockIdx.y; c < (u64)chunks * a.d.n_planes; c += gridDim.y) {
      const u32 plane_no = (u32)(c / chunks);
      const u64 plane = a.d.planes[plane_no], at0 = (c - (u64)plane_no * chunks) * (kMoved * 256) + threadIdx.x;
      v4u32 x[kMoved];
      v4u32* to[kMoved];
#pragma unroll
      for (u32 k = 0; k < kMoved; ++k) {
        const u64 at = at0 + k * 256;
        to[k] = nullptr;
        if (at >= of_plane) continue;
        // neighbouring lanes take what lies side by side: a token's pieces, or a piece's tokens
        u32 token, piece, word;
        if (a.t.pieces == 1 || a.t.piece_stride < a.t.token_stride) {
          token = (u32)(at / a.columns);
          const u32 rest = (u32)(at - (u64)token * a.columns);
          piece = rest / words, word = rest - piece * words;
        } else {
          const u32 of_piece = moves * words;
          piece = (u32)(at / of_piece);
          const u32 rest = (u32)(at - (u64)piece * of_piece);
          token = rest / words, word = rest - token * words;
        }
        x[k] = __builtin_nontemporal_load(place(plane, base + (u32)keep[begin + token], piece, word));
        to[k] = place(plane, base + begin + token, piece, word);
      }
#pragma unroll
      for (u32 k = 0; k < kMoved; ++k)
        if (to[k]) __builtin_nontemporal_store(x[k], to[k]);
    }
  } else {
    const u64 all = (u64)a.columns * a.d.n_planes;
    for (u64 c = blockIdx.y * 256 + threadIdx.x; begin < kept && c < all; c += gridDim.y * 256) {
      const u32 plane = (u32)(c / a.columns), at = (u32)(c - (u64)plane * a.columns), piece = at / words, word = at - piece * words;
      for (u32 j0 = begin; j0 < kept; j0 += kSerial) {
        v4u32 x[kSerial];
#pragma unroll
        for (u32 j = 0; j < kSerial; ++j)
          if (j0 + j < kept) x[j] = *place(a.d.planes[plane], base + (u32)keep[j0 + j], piece, word);
#pragma unroll
        for (u32 j = 0; j < kSerial; ++j)
          if (j0 + j < kept) *place(a.d.planes[plane], base + j0 + j, piece, word) = x[j];
      }
    }
  }
  if (blockIdx.y) return;
  bool bad = false;
  for (u32 j = ((base + kept + in_page) >> a.shift) + threadIdx.x; j < (n + in_page) >> a.shift; j += 256)
    if (!drop(a, (u32)table[j])) bad = true;
  if (threadIdx.x == 0) a.d.lens[r] = (int32_t)(base + kept);
  if (bad) raise_status(a.status, FDY_ST_BAD_INDEX);
}

// ---- copy -------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(256) copy_kernel(Pages a) {
  const u32 i = blockIdx.x, s = (u32)a.from[i], d = (u32)a.to[i];
  if (s >= a.d.n_pages || d >= a.d.n_pages) {
    if (threadIdx.x == 0 && blockIdx.y == 0) raise_status(a.status, FDY_ST_BAD_INDEX);
    return;
  }
  for (u32 t = blockIdx.y; t < a.d.n_planes * a.pieces; t += gridDim.y) copy_piece<false>(a, t / a.pieces, s, d, t % a.pieces);
}

// ---- compact ----------------------------------------------------------------------------------------
// Words of the workspace: {moves, live pages}, the free pages below, the live ones behind, each page's new number (where
// it moves), and the free bits as they were.
struct CompactWords {
  u32 *counts, *holes, *movers, *to;
  u64* was_free;
};
__host__ __device__ inline u64 compact_words(const fdy_pages& d) { return 64 + (d.n_pages + 63) / 64 * 2 + 3ull * d.n_pages; }
__device__ __forceinline__ CompactWords compact_layout(const Pages& a) {
  CompactWords w;
  w.counts = a.ws;
  w.was_free = (u64*)(a.ws + 64);
  w.holes = a.ws + 64 + (a.d.n_pages + 63) / 64 * 2;
  w.movers = w.holes + a.d.n_pages;
  w.to = w.movers + a.d.n_pages;
  return w;
}

__global__ void __launch_bounds__(kBooksThreads) compact_plan_kernel(Pages a) {
  __shared__ u64 s_scan[17];
  const CompactWords w = compact_layout(a);
  const u32 tid = threadIdx.x, words = (a.d.n_pages + 63) / 64;
  auto pages_in = [&](u32 i) { return i + 1 < words || a.d.n_pages % 64 == 0 ? ~0ull : (1ull << a.d.n_pages % 64) - 1; };
  u64 n_free = 0;
  for (u32 i0 = 0; i0 < words; i0 += kBooksThreads) {
    const u32 i = i0 + tid;
    const u64 bits = i < words ? a.d.free_bits[i] & pages_in(i) : 0;
    if (i < words) w.was_free[i] = bits;
    u64 sum;
    block_excl_scan((u64)__popcll(bits), s_scan, sum);
    n_free += sum;
  }
  const u32 n_live = a.d.n_pages - (u32)n_free;
  u64 base = 0;  // free pages below n_live, and live ones from there on in the high half
  for (u32 i0 = 0; i0 < words; i0 += kBooksThreads) {
    const u32 i = i0 + tid;
    u64 holes = 0, movers = 0;
    if (i < words) {
      const u64 bits = w.was_free[i], first = (u64)i * 64;
      const u64 below = first + 64 <= n_live ? ~0ull : first >= n_live ? 0 : (1ull << (n_live - first)) - 1;
      holes = bits & below;
      movers = ~bits & ~below & pages_in(i);
    }
    u64 sum;
    const u64 rank = base + block_excl_scan((u64)__popcll(holes) | (u64)__popcll(movers) << 32, s_scan, sum);
    base += sum;
    for (u32 r = (u32)rank; holes; holes &= holes - 1) w.holes[r++] = i * 64 + (u32)__builtin_ctzll(holes);
    for (u32 r = (u32)(rank >> 32); movers; movers &= movers - 1) w.movers[r++] = i * 64 + (u32)__builtin_ctzll(movers);
  }
  __syncthreads();
  const u32 moves = (u32)base;
  for (u32 k = tid; k < moves; k += kBooksThreads) w.to[w.movers[k]] = w.holes[k];
  if (tid == 0) {
    w.counts[0] = moves, w.counts[1] = n_live;
    if (a.n_live) *a.n_live = n_live;
  }
}

// The first `slices` workgroups keep the books, the others copy pieces of pages, plane after plane.
__global__ void __launch_bounds__(256) compact_move_kernel(Pages a) {
  const CompactWords w = compact_layout(a);
  const u32 moves = w.counts[0], n_live = w.counts[1];
  if (blockIdx.x >= a.slices) {
    const u64 of_plane = (u64)moves * a.pieces, tasks = of_plane * a.d.n_planes;
    for (u64 t = blockIdx.x - a.slices; t < tasks; t += gridDim.x - a.slices) {
      const u32 plane = tasks >> 32 ? (u32)(t / of_plane) : (u32)t / (u32)of_plane;
      const u64 rest = t - plane * of_plane;
      const u32 k = rest >> 32 ? (u32)(rest / a.pieces) : (u32)rest / a.pieces;
      copy_piece<true>(a, plane, w.movers[k], w.holes[k], (u32)(rest - (u64)k * a.pieces));
    }
    return;
  }
  const u32 at = blockIdx.x * 256 + threadIdx.x, step = a.slices * 256, words = (a.d.n_pages + 63) / 64;
  bool bad = false;
  for (u32 k = at; k < moves; k += step) {
    a.d.refs[w.holes[k]] = a.d.refs[w.movers[k]];
    a.d.refs[w.movers[k]] = 0;
  }
  for (u32 i = at; i < words; i += step) {
    const u64 first = (u64)i * 64;
    u64 bits = first >= n_live ? ~0ull : first + 64 <= n_live ? 0 : ~0ull << (n_live - first);
    if (i + 1 == words && a.d.n_pages % 64) bits &= (1ull << a.d.n_pages % 64) - 1;
    a.d.free_bits[i] = bits;
  }
  if (a.map)
    for (u32 p = at; p < a.d.n_pages; p += step)
      a.map[p] = w.was_free[p >> 6] >> (p & 63) & 1 ? -1 : (int32_t)(p < n_live ? p : w.to[p]);
  for (u32 r = blockIdx.x; r < a.d.n_rows; r += a.slices) {
    const u32 n = pages_of(a, length_of(a, r, bad));
    int32_t* table = a.d.table + (u64)r * a.d.row_pages;
    for (u32 j = threadIdx.x; j < n; j += 256) {
      const u32 p = (u32)table[j];
      if (p >= a.d.n_pages || w.was_free[p >> 6] >> (p & 63) & 1)
        bad = true;  // no page, or one that nobody holds
      else if (p >= n_live)
        table[j] = (int32_t)w.to[p];
    }
  }
  if (bad) raise_status(a.status, FDY_ST_BAD_INDEX);
}

// ---- the calls --------------------------------------------------------------------------------------
bool pages_valid(const fdy_pages& d) {
  if (d.reserved || !d.n_pages || d.n_pages > 1u << 28 || d.n_rows > 1u << 28 || d.row_pages > 1u << 25) return false;
  if (!power_of_two(d.page_tokens) || d.page_tokens > 65536u || (u64)d.row_pages * d.page_tokens >= 1ull << 31) return false;
  if (d.n_planes && (d.page_bytes % 16 || d.page_stride % 16 || d.page_bytes >> 30 || d.page_stride >> 40)) return false;
  if (d.n_planes * ((d.page_bytes + kPiece - 1) / kPiece) >> 32) return false;  // kernels count a page's pieces in 32 bits
  return d.n_planes <= 32768u;
}

// `books`: the call reads or writes the books; `planes`: it moves contents
int check(const fdy_pages* h, bool books, bool planes) {
  if (!h || !pages_valid(*h)) return FDY_ERR_INVALID_ARG;
  if (books && (!h->refs || !h->free_bits || !aligned(h->refs, 4) || !aligned(h->free_bits, 8))) return FDY_ERR_INVALID_ARG;
  if (books && h->n_rows && (!h->lens || !aligned(h->lens, 4) || (h->row_pages && !h->table) || !aligned(h->table, 4)))
    return FDY_ERR_INVALID_ARG;
  if (planes && h->n_planes && (!h->planes || !aligned(h->planes, 8))) return FDY_ERR_INVALID_ARG;
  return FDY_OK;
}

Pages args(const fdy_pages* h, u32 n, void* ws, u32* status) {
  Pages a{};
  a.d = *h;
  a.n = n;
  a.ws = (u32*)ws;
  a.status = status;
  a.shift = log2_of(h->page_tokens);
  a.pieces = (u32)((h->page_bytes + kPiece - 1) / kPiece);
  return a;
}

template <typename K, typename A>
int go(K kernel, dim3 grid, u32 threads, void* stream, const A& a) {
  (void)hipGetLastError();  // drop any stale error left by earlier, unrelated runtime calls
  hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, (hipStream_t)stream, a);
  FDY_HIP_TRY(hipGetLastError());
  return FDY_OK;
}

u32 at_most(u64 n, u32 most) { return n < most ? (u32)n : most; }
bool workspace_bad(const fdy_pages* h, u32 n, const void* ws, size_t bytes) {
  return !ws || !aligned(ws, 256) || bytes < fdy_pages_workspace_bytes(h, n);
}

}  // namespace

extern "C" size_t fdy_pages_workspace_bytes(const fdy_pages* h, uint32_t n) {
  if (!h || !pages_valid(*h) || n > kMostEntries) return 0;
  u64 words = extend_words(*h, n);
  if (fork_words(*h, n) > words) words = fork_words(*h, n);
  if (compact_words(*h) > words) words = compact_words(*h);
  return (size_t)((words * 4 + 255) / 256 * 256);
}

extern "C" int fdy_pages_reset(const fdy_pages* h, void* stream) {
  const int rc = check(h, true, false);
  if (rc != FDY_OK) return rc;
  const u32 most = h->n_pages > h->n_rows ? h->n_pages : h->n_rows;
  return go(pages_reset_kernel, dim3(at_most((most + 255) / 256, 4096)), 256, stream, args(h, 0, nullptr, nullptr));
}

extern "C" int fdy_pages_extend(const fdy_pages* h, const int32_t* d_rows, const int32_t* d_counts, uint32_t n,
                                int64_t* d_slots, int32_t* d_positions, uint32_t n_slots, void* ws, size_t ws_bytes,
                                uint32_t* d_status, void* stream) {
  int rc = check(h, true, true);
  if (rc != FDY_OK) return rc;
  if (n > kMostEntries || n_slots >> 31 || (!d_rows && n > h->n_rows)) return FDY_ERR_INVALID_ARG;
  if (!aligned(d_rows, 4) || !aligned(d_counts, 4) || !aligned(d_slots, 8) || !aligned(d_positions, 4)) return FDY_ERR_INVALID_ARG;
  if (n == 0) return FDY_OK;
  if (workspace_bad(h, n, ws, ws_bytes)) return FDY_ERR_WORKSPACE;
  Pages a = args(h, n, ws, d_status);
  a.from = d_rows, a.to = d_counts, a.slots = d_slots, a.positions = d_positions, a.n_slots = n_slots;
  rc = n <= kBooksThreads ? go(extend_few_kernel, dim3(1), kBooksThreads, stream, a)
                          : go(extend_books_kernel, dim3(1), kBooksThreads, stream, a);
  if (rc != FDY_OK || (!h->n_planes && !d_counts)) return rc;
  return go(extend_copy_kernel, dim3(n, at_most((u64)h->n_planes * a.pieces + (h->n_planes * a.pieces == 0), 1024)), 256, stream, a);
}

extern "C" int fdy_pages_fork(const fdy_pages* h, const int32_t* d_src, const int32_t* d_dst, uint32_t n, void* ws,
                              size_t ws_bytes, uint32_t* d_status, void* stream) {
  int rc = check(h, true, false);
  if (rc != FDY_OK) return rc;
  if (n > kMostEntries || !aligned(d_src, 4) || !aligned(d_dst, 4)) return FDY_ERR_INVALID_ARG;
  if (n == 0) return FDY_OK;
  if (!d_src || !d_dst) return FDY_ERR_INVALID_ARG;
  if (workspace_bad(h, n, ws, ws_bytes)) return FDY_ERR_WORKSPACE;
  Pages a = args(h, n, ws, d_status);
  a.from = d_src, a.to = d_dst;
  const dim3 grid(n, (h->row_pages + kForkPages - 1) / kForkPages + (h->row_pages == 0));
  rc = go(fork_note_kernel, grid, 256, stream, a);
  return rc == FDY_OK ? go(fork_write_kernel, grid, 256, stream, a) : rc;
}

extern "C" int fdy_pages_free(const fdy_pages* h, const int32_t* d_rows, uint32_t n, uint32_t* d_status, void* stream) {
  const int rc = check(h, true, false);
  if (rc != FDY_OK) return rc;
  if (n > kMostEntries || !aligned(d_rows, 4)) return FDY_ERR_INVALID_ARG;
  if (n == 0) return FDY_OK;
  if (!d_rows) return FDY_ERR_INVALID_ARG;
  Pages a = args(h, n, nullptr, d_status);
  a.from = d_rows;
  return go(free_kernel, dim3(n), 256, stream, a);
}

extern "C" int fdy_pages_keep(const fdy_pages* h, const fdy_token* h_token, const int32_t* d_rows, const int32_t* d_drafts,
                              const int32_t* d_keep, const int32_t* d_kept, uint32_t n, uint32_t most, void* ws, size_t ws_bytes,
                              uint32_t* d_status, void* stream) {
  int rc = check(h, true, true);
  if (rc != FDY_OK) return rc;
  if (!h_token || n > kMostEntries || most > 1u << 20 || (u64)n * most >> 31) return FDY_ERR_INVALID_ARG;
  const fdy_token& t = *h_token;
  if (h->n_planes) {
    if (!t.pieces || !t.piece_bytes || (t.token_stride | t.piece_stride | t.piece_bytes) % 16) return FDY_ERR_INVALID_ARG;
    if (t.token_stride >> 30 || t.piece_stride >> 30 ||
        (h->page_tokens - 1) * t.token_stride + (t.pieces - 1) * t.piece_stride + t.piece_bytes > h->page_bytes ||
        (u64)t.pieces * t.piece_bytes > h->page_bytes)
      return FDY_ERR_INVALID_ARG;
  }
  if (!aligned(d_rows, 4) || !aligned(d_drafts, 4) || !aligned(d_keep, 4) || !aligned(d_kept, 4)) return FDY_ERR_INVALID_ARG;
  if (n == 0) return FDY_OK;
  if (!d_rows || !d_drafts || !d_kept || (!d_keep && most)) return FDY_ERR_INVALID_ARG;
  if (workspace_bad(h, n, ws, ws_bytes)) return FDY_ERR_WORKSPACE;
  Keep a{};
  a.d = *h;
  a.t = t;
  a.status = d_status;
  a.rows = d_rows, a.drafts = d_drafts, a.keep = d_keep, a.kept = d_kept;
  a.ws = (u32*)ws;
  a.n = n, a.most = most;
  a.shift = log2_of(h->page_tokens);
  a.columns = h->n_planes ? t.pieces * (t.piece_bytes / 16) : 0;
  rc = go(keep_plan_kernel, dim3(n), most > 256 ? 1024 : 256, stream, a);
  if (rc != FDY_OK) return rc;
  // (how many tokens move is not known here)
  const u64 blocks = (((u64)most * a.columns + kMoved * 256 - 1) / (kMoved * 256)) * h->n_planes;
  const u32 y = at_most(blocks + (blocks == 0), 32768 / n < 512 ? 512 : 32768 / n);
  return go(keep_move_kernel, dim3(n, y), 256, stream, a);
}

extern "C" int fdy_pages_copy(const fdy_pages* h, const int32_t* d_src, const int32_t* d_dst, uint32_t n,
                              uint32_t* d_status, void* stream) {
  const int rc = check(h, false, true);
  if (rc != FDY_OK) return rc;
  if (n > kMostBlocks || !aligned(d_src, 4) || !aligned(d_dst, 4)) return FDY_ERR_INVALID_ARG;
  if (n == 0 || h->n_planes == 0) return FDY_OK;
  if (!d_src || !d_dst) return FDY_ERR_INVALID_ARG;
  Pages a = args(h, n, nullptr, d_status);
  a.from = d_src, a.to = d_dst;
  return go(copy_kernel, dim3(n, at_most((u64)h->n_planes * a.pieces + (a.pieces == 0), 1024)), 256, stream, a);
}

extern "C" int fdy_pages_compact(const fdy_pages* h, int32_t* d_map, uint32_t* d_n_live, void* ws, size_t ws_bytes,
                                 uint32_t* d_status, void* stream) {
  int rc = check(h, true, true);
  if (rc != FDY_OK) return rc;
  if (!aligned(d_map, 4) || !aligned(d_n_live, 4)) return FDY_ERR_INVALID_ARG;
  if (workspace_bad(h, 0, ws, ws_bytes)) return FDY_ERR_WORKSPACE;
  Pages a = args(h, 0, ws, d_status);
  a.map = d_map, a.n_live = d_n_live;
  rc = go(compact_plan_kernel, dim3(1), kBooksThreads, stream, a);
  if (rc != FDY_OK) return rc;
  // books: a workgroup a row or 1,024 pages.  Contents: up to 65,536 workgroups, the next piece to the next (158,400 pieces of
  // 16 KiB: 605 us, and 645 with 4,096 workgroups, 690 with 2,048 that go round); more would cost where little is to be moved
  a.slices = at_most(h->n_rows > h->n_pages / 1024 ? h->n_rows : h->n_pages / 1024 + 1, 1024);
  const u32 copiers = at_most((u64)(h->n_pages / 2 + 1) * (h->n_planes ? a.pieces : 0) * h->n_planes, 65536);
  return go(compact_move_kernel, dim3(a.slices + copiers), 256, stream, a);
}
