// decode_graph.hip - a decode step's own kernels captured, rebased and replayed (test program, not part of the library).
//
// What the library restores are graphs of a serving engine's decode steps.  Here is one made of the operators of
// fdy_decode.h: rows change parents (fork), every row gets room for a token (extend, shared last pages copied), and in each
// of two layers queries and keys are turned, keys and values appended to the pages, and the token attends over its row.
//   1. prompts of six rows are brought into a cache that lies in arena A (reset, extend, append), by plain calls;
//   2. the step is captured from a stream; the argument buffer of every node is its one struct of FDY_DECODE_ARG_BYTES;
//   3. all argument buffers, and the device array of the planes' addresses, are rebased for arena B in one pass
//      (fdy_scan_rebase), the arguments installed in a second executable graph, the contents copied over;
//   4. both graphs are replayed with the same new tokens and parents, B's first: after every step all that lies in B's
//      allocations equals what lies in A's, and A has not been touched by B's replay;
//   5. the outputs of A's replays equal those of the same calls made on a third arena without a graph.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <vector>

#include "fdy_arena.h"
#include "fdy_decode.h"

namespace {

constexpr uint32_t kRows = 6, kHeads = 4, kKvHeads = 2, kDim = 64, kPt = 16, kPages = 80, kRowPages = 12, kLayers = 2;
constexpr uint32_t kQkv = (kHeads + 2 * kKvHeads) * kDim, kPromptMost = 240, kPositions = kRowPages * kPt;
constexpr size_t kPageBytes = (size_t)kPt * kKvHeads * kDim * 2;
constexpr int kSteps = 20;

#define CK(expr)                                                              \
  do {                                                                        \
    hipError_t e__ = (expr);                                                  \
    if (e__ != hipSuccess) {                                                  \
      snprintf(msg, msg_len, "%s failed: %s", #expr, hipGetErrorString(e__)); \
      return 1;                                                               \
    }                                                                         \
  } while (0)
#define FD(expr)                                                                                          \
  do {                                                                                                    \
    int r__ = (expr);                                                                                     \
    if (r__ != FDY_OK) {                                                                                  \
      snprintf(msg, msg_len, "%s failed: %s [%s]", #expr, fdy_strerror(r__), fdy_arena_last_failure());  \
      return 1;                                                                                           \
    }                                                                                                     \
  } while (0)

// What an instance allocates, in this order: the same offsets in every arena.
struct Buffers {
  void *status, *refs, *bits, *table, *lens, *planes, *slots, *positions, *src, *dst, *rope, *prompt, *counts, *pages_ws, *attend_ws;
  void *cache[kLayers][2], *qkv[kLayers], *q[kLayers], *out[kLayers];
};

uint16_t bf16(float x) {
  uint32_t u;
  memcpy(&u, &x, 4);
  return (uint16_t)((u + 0x7fff + (u >> 16 & 1)) >> 16);
}

struct Random {
  uint64_t s;
  uint32_t next() {
    s += 0x9e3779b97f4a7c15ull;
    uint64_t z = s;
    z = (z ^ z >> 30) * 0xbf58476d1ce4e5b9ull;
    z = (z ^ z >> 27) * 0x94d049bb133111ebull;
    return (uint32_t)(z >> 32);
  }
  float value() { return (float)(int32_t)next() * (1.f / 1073741824.f); }  // in [-2, 2)
  std::vector<uint16_t> values(size_t n) {
    std::vector<uint16_t> v(n);
    for (auto& x : v) x = bf16(value());
    return v;
  }
};

struct Instance {
  fdy_arena* arena = nullptr;
  Buffers b{};
  fdy_pages pages{};
  fdy_append append[kLayers]{};
  fdy_attend attend[kLayers]{};
  size_t pages_bytes = 0, attend_bytes = 0;

  fdy_kv cache(int layer) const {
    fdy_kv c{};
    c.k = b.cache[layer][0], c.v = b.cache[layer][1];
    c.page_stride = kPageBytes / 2, c.token_stride = kKvHeads * kDim, c.head_stride = kDim;
    c.type = FDY_BF16, c.n_pages = kPages, c.page_tokens = kPt, c.n_heads = kKvHeads, c.head_dim = kDim;
    return c;
  }

  // tokens of `from` ([n][kQkv]) at the slots and positions that the last extend gave out
  fdy_append append_of(int layer, void* from, uint32_t n) const {
    fdy_append d{};
    uint16_t* x = (uint16_t*)from;
    d.q = x, d.k = x + kHeads * kDim, d.v = x + (kHeads + kKvHeads) * kDim, d.q_out = b.q[layer];
    d.positions = (const int32_t*)b.positions, d.table = (const float*)b.rope, d.slots = (const int64_t*)b.slots;
    d.q_token = d.k_token = d.v_token = kQkv, d.q_head = d.k_head = d.v_head = kDim;
    d.q_out_token = kHeads * kDim, d.q_out_head = kDim;
    d.kv = cache(layer);
    d.n_tokens = n, d.n_q_heads = kHeads, d.n_positions = kPositions, d.rot_dim = kDim / 2;
    d.type = FDY_BF16, d.layout = FDY_ROPE_HALF;
    return d;
  }

  int allocate(uint64_t hint, char* msg, int msg_len) {
    FD(fdy_arena_create(&arena, hint, 16u << 20));
    pages.page_bytes = pages.page_stride = kPageBytes;
    pages.n_pages = kPages, pages.page_tokens = kPt, pages.n_rows = kRows, pages.row_pages = kRowPages, pages.n_planes = 2 * kLayers;
    pages_bytes = fdy_pages_workspace_bytes(&pages, kRows);
    fdy_attend shape{};
    shape.kv = cache(0);
    shape.n_seqs = shape.n_rows = kRows, shape.n_q_heads = kHeads, shape.row_pages = kRowPages;
    attend_bytes = fdy_paged_attention_workspace_bytes(&shape);
    struct {
      void** p;
      size_t bytes;
    } list[] = {{&b.status, 4}, {&b.refs, kPages * 4}, {&b.bits, (kPages + 63) / 64 * 8}, {&b.table, kRows * kRowPages * 4},
                {&b.lens, kRows * 4}, {&b.planes, 2 * kLayers * 8}, {&b.slots, kPromptMost * 8}, {&b.positions, kPromptMost * 4},
                {&b.src, kRows * 4}, {&b.dst, kRows * 4}, {&b.rope, kPositions * kDim / 2 * 4}, {&b.prompt, kPromptMost * kQkv * 2},
                {&b.counts, kRows * 4}, {&b.pages_ws, pages_bytes}, {&b.attend_ws, attend_bytes}};
    for (auto& l : list) {
      FD(fdy_arena_alloc(arena, l.bytes, 256, l.p));
      CK(hipMemset(*l.p, 0, l.bytes));
    }
    for (uint32_t i = 0; i < kLayers; ++i) {
      for (int s = 0; s < 2; ++s) {
        FD(fdy_arena_alloc(arena, kPages * kPageBytes, 4096, &b.cache[i][s]));
        CK(hipMemset(b.cache[i][s], 0x7f, kPages * kPageBytes));  // NaN wherever nothing has been written
      }
      FD(fdy_arena_alloc(arena, kRows * kQkv * 2, 256, &b.qkv[i]));
      FD(fdy_arena_alloc(arena, kPromptMost * kHeads * kDim * 2, 256, &b.q[i]));
      FD(fdy_arena_alloc(arena, kRows * kHeads * kDim * 2, 256, &b.out[i]));
      CK(hipMemset(b.qkv[i], 0, kRows * kQkv * 2));
      CK(hipMemset(b.q[i], 0, kPromptMost * kHeads * kDim * 2));
      CK(hipMemset(b.out[i], 0, kRows * kHeads * kDim * 2));
    }
    pages.refs = (uint32_t*)b.refs, pages.free_bits = (uint64_t*)b.bits, pages.table = (int32_t*)b.table;
    pages.lens = (int32_t*)b.lens, pages.planes = (const uint64_t*)b.planes;
    uint64_t planes[2 * kLayers];
    for (uint32_t i = 0; i < 2 * kLayers; ++i) planes[i] = (uint64_t)(uintptr_t)b.cache[i / 2][i % 2];
    CK(hipMemcpy(b.planes, planes, sizeof planes, hipMemcpyHostToDevice));
    for (uint32_t i = 0; i < kLayers; ++i) {
      append[i] = append_of((int)i, b.qkv[i], kRows);
      fdy_attend& d = attend[i];
      d.q = b.q[i], d.out = b.out[i], d.table = pages.table, d.lens = pages.lens;
      d.q_seq = d.out_seq = kHeads * kDim, d.q_head = d.out_head = kDim;
      d.kv = cache((int)i);
      d.scale = 0.125f;
      d.n_seqs = d.n_rows = kRows, d.n_q_heads = kHeads, d.row_pages = kRowPages, d.type = FDY_BF16;
    }
    return 0;
  }

  // Six prompts by plain calls.
  int prompts(hipStream_t stream, char* msg, int msg_len) {
    const int32_t counts[kRows] = {5, 40, 16, 1, 33, 64};
    Random r{7};
    const auto x = r.values((size_t)kPromptMost * kQkv);
    fdy_rope rope{};
    rope.scaling = FDY_ROPE_LINEAR, rope.rot_dim = kDim / 2, rope.base = 10000., rope.factor = 2., rope.magnitude = 1.;
    CK(hipMemcpy(b.counts, counts, sizeof counts, hipMemcpyHostToDevice));
    CK(hipMemcpy(b.prompt, x.data(), x.size() * 2, hipMemcpyHostToDevice));
    FD(fdy_rope_table(&rope, 0, kPositions, (float*)b.rope, stream));
    FD(fdy_pages_reset(&pages, stream));
    FD(fdy_pages_extend(&pages, nullptr, (const int32_t*)b.counts, kRows, (int64_t*)b.slots, (int32_t*)b.positions, kPromptMost,
                        b.pages_ws, pages_bytes, (uint32_t*)b.status, stream));
    for (uint32_t i = 0; i < kLayers; ++i) {
      const fdy_append d = append_of((int)i, b.prompt, 5 + 40 + 16 + 1 + 33 + 64);
      FD(fdy_rope_append(&d, (uint32_t*)b.status, stream));
    }
    CK(hipStreamSynchronize(stream));
    return 0;
  }

  int step(hipStream_t stream, char* msg, int msg_len) {
    uint32_t* status = (uint32_t*)b.status;
    FD(fdy_pages_fork(&pages, (const int32_t*)b.src, (const int32_t*)b.dst, kRows, b.pages_ws, pages_bytes, status, stream));
    FD(fdy_pages_extend(&pages, nullptr, nullptr, kRows, (int64_t*)b.slots, (int32_t*)b.positions, kRows, b.pages_ws, pages_bytes,
                        status, stream));
    for (uint32_t i = 0; i < kLayers; ++i) {
      FD(fdy_rope_append(&append[i], status, stream));
      FD(fdy_paged_attention(&attend[i], b.attend_ws, attend_bytes, status, stream));
    }
    return 0;
  }

  // The tokens of a step and who goes on from whom.
  int inputs(int number, char* msg, int msg_len) {
    Random r{100u + (uint32_t)number};
    int32_t src[kRows], dst[kRows];
    for (uint32_t i = 0; i < kRows; ++i) dst[i] = (int32_t)i, src[i] = (int32_t)(number % 3 ? i : i / 3 * 3 + r.next() % 3);
    CK(hipMemcpy(b.src, src, sizeof src, hipMemcpyHostToDevice));
    CK(hipMemcpy(b.dst, dst, sizeof dst, hipMemcpyHostToDevice));
    for (uint32_t i = 0; i < kLayers; ++i) {
      const auto x = r.values((size_t)kRows * kQkv);
      CK(hipMemcpy(b.qkv[i], x.data(), x.size() * 2, hipMemcpyHostToDevice));
    }
    return 0;
  }
};

// Everything in an arena's allocations.
int contents(const Instance& x, std::vector<std::vector<uint8_t>>* all, char* msg, int msg_len) {
  const uint32_t n = fdy_arena_count(x.arena);
  std::vector<fdy_alloc> t(n);
  FD(fdy_arena_table(x.arena, t.data(), n));
  all->assign(n, {});
  for (uint32_t i = 0; i < n; ++i) {
    (*all)[i].resize(t[i].size);
    CK(hipMemcpy((*all)[i].data(), (void*)(uintptr_t)t[i].base, t[i].size, hipMemcpyDeviceToHost));
  }
  return 0;
}
constexpr uint32_t kPlanesAt = 5, kWorkspaceAt = 13;  // allocations whose contents differ by nature: addresses, scratch

}  // namespace

extern "C" int decode_graph_check(char* msg, int msg_len) {
  hipStream_t stream;
  CK(hipStreamCreate(&stream));
  Instance A, B, C;
  if (A.allocate(0x210000000000ull, msg, msg_len) || B.allocate(0x310000000000ull, msg, msg_len) ||
      C.allocate(0x410000000000ull, msg, msg_len))
    return 1;
  if (A.prompts(stream, msg, msg_len) || C.prompts(stream, msg, msg_len)) return 1;

  // the step, captured on A
  CK(hipStreamBeginCapture(stream, hipStreamCaptureModeThreadLocal));
  const int rc = A.step(stream, msg, msg_len);
  hipGraph_t graph = nullptr;
  const hipError_t ended = hipStreamEndCapture(stream, &graph);
  if (rc) return rc;
  CK(ended);
  size_t n_nodes = 0;
  CK(hipGraphGetNodes(graph, nullptr, &n_nodes));
  std::vector<hipGraphNode_t> nodes(n_nodes);
  CK(hipGraphGetNodes(graph, nodes.data(), &n_nodes));
  constexpr size_t kWords = FDY_DECODE_ARG_BYTES / 8;
  std::vector<uint64_t> words(n_nodes * kWords + 2 * kLayers);
  std::vector<hipKernelNodeParams> params(n_nodes);
  for (size_t i = 0; i < n_nodes; ++i) {
    hipGraphNodeType type;
    CK(hipGraphNodeGetType(nodes[i], &type));
    if (type != hipGraphNodeTypeKernel) {
      snprintf(msg, msg_len, "node %zu of the step is no kernel", i);
      return 1;
    }
    CK(hipGraphKernelNodeGetParams(nodes[i], &params[i]));
    memcpy(&words[i * kWords], params[i].kernelParams[0], FDY_DECODE_ARG_BYTES);
  }
  CK(hipMemcpy(&words[n_nodes * kWords], A.b.planes, 2 * kLayers * 8, hipMemcpyDeviceToHost));
  hipGraphExec_t exec_a, exec_b;
  CK(hipGraphInstantiate(&exec_a, graph, nullptr, nullptr, 0));
  CK(hipGraphInstantiate(&exec_b, graph, nullptr, nullptr, 0));

  // rebased for B: its bases in the place of A's, found by value alone
  const uint32_t n_alloc = fdy_arena_count(A.arena);
  std::vector<fdy_alloc> ta(n_alloc), tb(n_alloc);
  FD(fdy_arena_table(A.arena, ta.data(), n_alloc));
  FD(fdy_arena_table(B.arena, tb.data(), n_alloc));
  std::vector<uint64_t> new_base(n_alloc);
  for (uint32_t i = 0; i < n_alloc; ++i) {
    new_base[i] = tb[i].base;
    if (i != kWorkspaceAt) CK(hipMemcpy((void*)(uintptr_t)tb[i].base, (void*)(uintptr_t)ta[i].base, ta[i].size, hipMemcpyDeviceToDevice));
  }
  void *d_words, *d_table, *d_nb, *d_out, *d_count, *d_ws;
  const size_t ws_bytes = fdy_scan_workspace_bytes(words.size(), n_alloc);
  CK(hipMalloc(&d_words, words.size() * 8));
  CK(hipMalloc(&d_out, words.size() * 8));
  CK(hipMalloc(&d_table, n_alloc * sizeof(fdy_alloc)));
  CK(hipMalloc(&d_nb, n_alloc * 8));
  CK(hipMalloc(&d_count, 8));
  CK(hipMalloc(&d_ws, ws_bytes));
  CK(hipMemcpy(d_words, words.data(), words.size() * 8, hipMemcpyHostToDevice));
  CK(hipMemcpy(d_table, ta.data(), n_alloc * sizeof(fdy_alloc), hipMemcpyHostToDevice));
  CK(hipMemcpy(d_nb, new_base.data(), n_alloc * 8, hipMemcpyHostToDevice));
  FD(fdy_scan_rebase((const uint64_t*)d_words, words.size(), (const fdy_alloc*)d_table, n_alloc, (const uint64_t*)d_nb,
                     (uint64_t*)d_out, (uint64_t*)d_count, nullptr, d_ws, ws_bytes, nullptr, stream));
  CK(hipStreamSynchronize(stream));
  uint64_t count = 0;
  CK(hipMemcpy(&count, d_count, 8, hipMemcpyDeviceToHost));
  CK(hipMemcpy(words.data(), d_out, words.size() * 8, hipMemcpyDeviceToHost));
  CK(hipMemcpy(B.b.planes, &words[n_nodes * kWords], 2 * kLayers * 8, hipMemcpyHostToDevice));
  for (size_t i = 0; i < n_nodes; ++i) {
    void* arg[1] = {&words[i * kWords]};
    hipKernelNodeParams np = params[i];
    np.kernelParams = arg;
    np.extra = nullptr;
    CK(hipGraphExecKernelNodeSetParams(exec_b, nodes[i], &np));
  }

  std::vector<std::vector<uint8_t>> a0, a1, b1, c1;
  std::vector<uint16_t> last;
  for (int s = 0; s < kSteps; ++s) {
    if (A.inputs(s, msg, msg_len) || B.inputs(s, msg, msg_len) || C.inputs(s, msg, msg_len)) return 1;
    if (contents(A, &a0, msg, msg_len)) return 1;
    CK(hipGraphLaunch(exec_b, stream));
    CK(hipStreamSynchronize(stream));
    if (contents(A, &a1, msg, msg_len)) return 1;
    if (a0 != a1) {
      snprintf(msg, msg_len, "step %d: the replay on arena B wrote to arena A", s);
      return 1;
    }
    CK(hipGraphLaunch(exec_a, stream));
    if (C.step(stream, msg, msg_len)) return 1;
    CK(hipStreamSynchronize(stream));
    if (contents(A, &a1, msg, msg_len) || contents(B, &b1, msg, msg_len) || contents(C, &c1, msg, msg_len)) return 1;
    for (uint32_t i = 0; i < n_alloc; ++i) {
      if (i == kPlanesAt || i == kWorkspaceAt || i == kWorkspaceAt + 1) continue;
      if (a1[i] != b1[i] || a1[i] != c1[i]) {
        snprintf(msg, msg_len, "step %d: allocation %u differs (%s)", s, i, a1[i] != b1[i] ? "rebased graph" : "plain calls");
        return 1;
      }
    }
    uint32_t status = 0;
    int32_t lens[kRows];
    std::vector<uint16_t> out(kRows * kHeads * kDim);
    CK(hipMemcpy(&status, B.b.status, 4, hipMemcpyDeviceToHost));
    CK(hipMemcpy(lens, B.b.lens, sizeof lens, hipMemcpyDeviceToHost));
    CK(hipMemcpy(out.data(), B.b.out[kLayers - 1], out.size() * 2, hipMemcpyDeviceToHost));
    bool finite = true;
    for (uint16_t x : out) finite = finite && (x & 0x7f80) != 0x7f80;
    if (status || !finite || out == last) {
      snprintf(msg, msg_len, "step %d: status %u, outputs %s", s, status, finite ? "unchanged" : "not finite");
      return 1;
    }
    last = out;
  }
  CK(hipGraphExecDestroy(exec_a));
  CK(hipGraphExecDestroy(exec_b));
  CK(hipGraphDestroy(graph));
  for (void* p : {d_words, d_out, d_table, d_nb, d_count, d_ws}) CK(hipFree(p));
  FD(fdy_arena_destroy(A.arena));
  FD(fdy_arena_destroy(B.arena));
  FD(fdy_arena_destroy(C.arena));
  CK(hipStreamDestroy(stream));
  snprintf(msg, msg_len, "ok: %zu nodes, %llu pointers rebased, %d steps alike on two arenas and without a graph", n_nodes,
           (unsigned long long)count, kSteps);
  return 0;
}
