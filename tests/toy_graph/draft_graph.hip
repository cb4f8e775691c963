// draft_graph.hip - a round of drafted tokens and of chosen pages captured, rebased and replayed (test program, not part of the library).
//
// The step: every row gets room for five drafted tokens, in each of two layers keys and values are appended and the trees attend
// over their rows; the accepted paths move together; then the pages' bounds are brought up to date, and in each layer one token of every
// row attends over the pages that are chosen for it.  As for a step of single tokens (decode_graph.hip) it is captured on arena A, the
// argument buffers and the planes' addresses are rebased for arena B in one pass, and both are replayed with the same inputs, B's
// first: all of B's allocations equal A's, A's those of the same calls made on a third arena without a graph, and B's replay leaves A alone.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <vector>

#include "fdy_arena.h"
#include "fdy_decode.h"

namespace {

constexpr uint32_t kRows = 6, kHeads = 8, kKvHeads = 2, kDim = 64, kPt = 16, kPages = 100, kRowPages = 16, kLayers = 2, kDrafts = 5;
constexpr uint32_t kTokens = kRows * kDrafts, kQkv = (kHeads + 2 * kKvHeads) * kDim, kPromptMost = 200, kBudget = 4;
constexpr size_t kTokenBytes = kKvHeads * kDim * 2, kPageBytes = kPt * kTokenBytes;
constexpr int kSteps = 16;

#define CK(expr)                                                              \
  do {                                                                        \
    hipError_t e__ = (expr);                                                  \
    if (e__ != hipSuccess) {                                                  \
      snprintf(msg, msg_len, "%s failed: %s", #expr, hipGetErrorString(e__)); \
      return 1;                                                               \
    }                                                                         \
  } while (0)
#define FD(expr)                                                                                         \
  do {                                                                                                   \
    int r__ = (expr);                                                                                    \
    if (r__ != FDY_OK) {                                                                                 \
      snprintf(msg, msg_len, "%s failed: %s [%s]", #expr, fdy_strerror(r__), fdy_arena_last_failure()); \
      return 1;                                                                                          \
    }                                                                                                    \
  } while (0)

struct Random {
  uint64_t s;
  uint32_t next() {
    s = s * 6364136223846793005ull + 1442695040888963407ull;
    return (uint32_t)(s >> 33) ^ (uint32_t)(s >> 17);
  }
  std::vector<uint16_t> values(size_t n) {  // bf16, of either sign, from 2^-3 to 2
    std::vector<uint16_t> v(n);
    for (auto& x : v) x = (uint16_t)((next() & 0x807f) | (124 + next() % 4) << 7);
    return v;
  }
};

struct Instance {
  fdy_arena* arena = nullptr;
  // the same allocations, in this order, in every arena; those from `scratch` on differ by nature
  void *status, *refs, *bits, *table, *lens, *slots, *positions, *counts, *rows, *first, *sees, *keep, *kept, *rope, *prompt;
  void *cache[kLayers][2], *qkv[kLayers], *q[kLayers], *out[kLayers], *lse[kLayers], *bounds[kLayers], *pages[kLayers], *seen[kLayers],
      *near_out[kLayers];
  void *planes, *pages_ws, *tree_ws, *select_ws, *near_ws;
  uint32_t scratch = 0;
  fdy_pages books{};
  fdy_token token{kTokenBytes, 0, (uint32_t)kTokenBytes, 1};
  fdy_append append[kLayers]{};
  fdy_draft draft[kLayers]{};
  fdy_bounds bound[kLayers]{};
  fdy_select select[kLayers]{};
  fdy_attend near[kLayers]{};
  size_t pages_bytes = 0, tree_bytes = 0, select_bytes = 0, near_bytes = 0;

  fdy_kv cache_of(uint32_t layer) const {
    fdy_kv c{};
    c.k = cache[layer][0], c.v = cache[layer][1];
    c.page_stride = kPageBytes / 2, c.token_stride = kKvHeads * kDim, c.head_stride = kDim;
    c.type = FDY_BF16, c.n_pages = kPages, c.page_tokens = kPt, c.n_heads = kKvHeads, c.head_dim = kDim;
    return c;
  }
  fdy_append append_of(uint32_t layer, void* from, uint32_t n) const {
    fdy_append d{};
    uint16_t* x = (uint16_t*)from;
    d.q = x, d.k = x + kHeads * kDim, d.v = x + (kHeads + kKvHeads) * kDim, d.q_out = q[layer];
    d.positions = (const int32_t*)positions, d.table = (const float*)rope, d.slots = (const int64_t*)slots;
    d.q_token = d.k_token = d.v_token = kQkv, d.q_head = d.k_head = d.v_head = kDim;
    d.q_out_token = kHeads * kDim, d.q_out_head = kDim;
    d.kv = cache_of(layer);
    d.n_tokens = n, d.n_q_heads = kHeads, d.n_positions = kRowPages * kPt, d.rot_dim = kDim;
    d.type = FDY_BF16, d.layout = FDY_ROPE_HALF;
    return d;
  }

  int place(void** p, size_t bytes, int fill, char* msg, int msg_len) {
    FD(fdy_arena_alloc(arena, bytes, 256, p));
    CK(hipMemset(*p, fill, bytes));
    return 0;
  }

  int allocate(uint64_t hint, char* msg, int msg_len) {
    FD(fdy_arena_create(&arena, hint, 64u << 20));
    struct {
      void** p;
      size_t bytes;
    } list[] = {{&status, 4}, {&refs, kPages * 4}, {&bits, (kPages + 63) / 64 * 8}, {&table, kRows * kRowPages * 4}, {&lens, kRows * 4},
                {&slots, kPromptMost * 8}, {&positions, kPromptMost * 4}, {&counts, kRows * 4}, {&rows, kRows * 4},
                {&first, (kRows + 1) * 4}, {&sees, kTokens * 8}, {&keep, kTokens * 4}, {&kept, kRows * 4},
                {&rope, kRowPages * kPt * kDim * 4}, {&prompt, kPromptMost * kQkv * 2}};
    for (auto& l : list)
      if (place(l.p, l.bytes, 0, msg, msg_len)) return 1;
    for (uint32_t i = 0; i < kLayers; ++i) {
      for (void*& c : cache[i])
        if (place(&c, kPages * kPageBytes, 0xff, msg, msg_len)) return 1;  // no numbers wherever nothing has been written
      if (place(&qkv[i], kTokens * kQkv * 2, 0, msg, msg_len) || place(&q[i], kPromptMost * kHeads * kDim * 2, 0, msg, msg_len) ||
          place(&out[i], kTokens * kHeads * kDim * 2, 0, msg, msg_len) || place(&lse[i], kTokens * kHeads * 4, 0, msg, msg_len) ||
          place(&bounds[i], kPages * kKvHeads * 2 * kDim * 2, 0, msg, msg_len) ||
          place(&pages[i], kRows * kKvHeads * kBudget * 4, 0, msg, msg_len) || place(&seen[i], kRows * 4, 0, msg, msg_len) ||
          place(&near_out[i], kRows * kHeads * kDim * 2, 0, msg, msg_len))
        return 1;
    }
    scratch = fdy_arena_count(arena);
    books.refs = (uint32_t*)refs, books.free_bits = (uint64_t*)bits, books.table = (int32_t*)table, books.lens = (int32_t*)lens;
    books.page_bytes = books.page_stride = kPageBytes;
    books.n_pages = kPages, books.page_tokens = kPt, books.n_rows = kRows, books.row_pages = kRowPages, books.n_planes = 2 * kLayers;
    for (uint32_t i = 0; i < kLayers; ++i) {
      append[i] = append_of(i, qkv[i], kTokens);
      fdy_draft& d = draft[i];
      d.q = q[i], d.out = out[i], d.lse = (float*)lse[i], d.table = books.table, d.lens = books.lens;
      d.first = (const int32_t*)first, d.sees = (const uint64_t*)sees;
      d.q_token = d.out_token = kHeads * kDim, d.q_head = d.out_head = kDim;
      d.kv = cache_of(i), d.scale = 0.125f;
      d.n_seqs = d.n_rows = kRows, d.n_q_heads = kHeads, d.row_pages = kRowPages, d.n_tokens = kTokens, d.max_draft = kDrafts;
      d.sees_words = 1, d.type = FDY_BF16;
      fdy_bounds& b = bound[i];
      b.bounds = bounds[i], b.table = books.table, b.lens = books.lens, b.fresh = (const int32_t*)kept, b.kv = cache_of(i);
      b.n_seqs = b.n_rows = kRows, b.row_pages = kRowPages, b.max_fresh = kDrafts;
      fdy_select& s = select[i];
      s.q = q[i], s.bounds = bounds[i], s.table = books.table, s.lens = books.lens, s.pages = (int32_t*)pages[i], s.seen = (int32_t*)seen[i];
      s.q_seq = kDrafts * kHeads * kDim, s.q_head = kDim;
      s.kv = cache_of(i);
      s.n_seqs = s.n_rows = kRows, s.n_q_heads = kHeads, s.row_pages = kRowPages, s.budget = kBudget, s.sinks = s.recent = 1, s.type = FDY_BF16;
      fdy_attend& a = near[i];
      a.q = q[i], a.out = near_out[i], a.table = (const int32_t*)pages[i], a.lens = (const int32_t*)seen[i];
      a.q_seq = kDrafts * kHeads * kDim, a.out_seq = kHeads * kDim, a.q_head = a.out_head = kDim;
      a.kv = cache_of(i), a.scale = 0.125f;
      a.n_seqs = a.n_rows = kRows, a.n_q_heads = kHeads, a.row_pages = kBudget, a.type = FDY_BF16;
    }
    pages_bytes = fdy_pages_workspace_bytes(&books, kRows);
    tree_bytes = fdy_tree_attention_workspace_bytes(&draft[0]);
    select_bytes = fdy_page_select_workspace_bytes(&select[0]);
    near_bytes = fdy_selected_attention_workspace_bytes(&near[0]);
    if (place(&planes, 2 * kLayers * 8, 0, msg, msg_len) || place(&pages_ws, pages_bytes, 0, msg, msg_len) ||
        place(&tree_ws, tree_bytes, 0, msg, msg_len) || place(&select_ws, select_bytes, 0, msg, msg_len) ||
        place(&near_ws, near_bytes, 0, msg, msg_len))
      return 1;
    books.planes = (const uint64_t*)planes;
    uint64_t at[2 * kLayers];
    for (uint32_t i = 0; i < 2 * kLayers; ++i) at[i] = (uint64_t)(uintptr_t)cache[i / 2][i % 2];
    CK(hipMemcpy(planes, at, sizeof at, hipMemcpyHostToDevice));
    return 0;
  }

  // Six prompts and the bounds of their pages, by plain calls.
  int prompts(hipStream_t stream, char* msg, int msg_len) {
    const int32_t n[kRows] = {5, 40, 16, 1, 33, 64}, drafts[kRows] = {kDrafts, kDrafts, kDrafts, kDrafts, kDrafts, kDrafts};
    int32_t each[kRows], from[kRows + 1];
    for (uint32_t i = 0; i <= kRows; ++i) from[i] = (int32_t)(i * kDrafts);
    for (uint32_t i = 0; i < kRows; ++i) each[i] = (int32_t)i;
    Random r{7};
    const auto x = r.values((size_t)kPromptMost * kQkv);
    fdy_rope plain{};
    plain.rot_dim = kDim, plain.base = 10000., plain.magnitude = 1.;
    CK(hipMemcpy(counts, n, sizeof n, hipMemcpyHostToDevice));
    CK(hipMemcpy(rows, each, sizeof each, hipMemcpyHostToDevice));
    CK(hipMemcpy(first, from, sizeof from, hipMemcpyHostToDevice));
    CK(hipMemcpy(prompt, x.data(), x.size() * 2, hipMemcpyHostToDevice));
    FD(fdy_rope_table(&plain, 0, kRowPages * kPt, (float*)rope, stream));
    FD(fdy_pages_reset(&books, stream));
    FD(fdy_pages_extend(&books, nullptr, (const int32_t*)counts, kRows, (int64_t*)slots, (int32_t*)positions, kPromptMost, pages_ws,
                        pages_bytes, (uint32_t*)status, stream));
    for (uint32_t i = 0; i < kLayers; ++i) {
      const fdy_append d = append_of(i, prompt, 5 + 40 + 16 + 1 + 33 + 64);
      FD(fdy_rope_append(&d, (uint32_t*)status, stream));
      fdy_bounds b = bound[i];
      b.fresh = (const int32_t*)counts, b.max_fresh = 64;
      FD(fdy_page_bounds(&b, (uint32_t*)status, stream));
    }
    CK(hipStreamSynchronize(stream));
    CK(hipMemcpy(counts, drafts, sizeof drafts, hipMemcpyHostToDevice));
    return 0;
  }

  int step(hipStream_t stream, char* msg, int msg_len) {
    uint32_t* st = (uint32_t*)status;
    FD(fdy_pages_extend(&books, nullptr, (const int32_t*)counts, kRows, (int64_t*)slots, (int32_t*)positions, kTokens, pages_ws, pages_bytes,
                        st, stream));
    for (uint32_t i = 0; i < kLayers; ++i) {
      FD(fdy_rope_append(&append[i], st, stream));
      FD(fdy_tree_attention(&draft[i], tree_ws, tree_bytes, st, stream));
    }
    FD(fdy_pages_keep(&books, &token, (const int32_t*)rows, (const int32_t*)counts, (const int32_t*)keep, (const int32_t*)kept, kRows, kDrafts,
                      pages_ws, pages_bytes, st, stream));
    for (uint32_t i = 0; i < kLayers; ++i) {
      FD(fdy_page_bounds(&bound[i], st, stream));
      FD(fdy_page_select(&select[i], select_ws, select_bytes, st, stream));
      FD(fdy_selected_attention(&near[i], near_ws, near_bytes, st, stream));
    }
    return 0;
  }

  // The drafted tokens of a step, who goes on from whom, and the paths that are accepted.
  int inputs(int number, char* msg, int msg_len) {
    Random r{100u + (uint32_t)number};
    uint64_t who[kTokens];
    int32_t stay[kTokens] = {}, n[kRows];
    for (uint32_t i = 0; i < kRows; ++i) {
      for (uint32_t j = 0; j < kDrafts; ++j) {
        const uint32_t from = r.next() % (j + 1);  // 0: from the cached ones
        who[i * kDrafts + j] = 1ull << j | (from ? who[i * kDrafts + from - 1] : 0);
      }
      uint64_t path = who[i * kDrafts + r.next() % kDrafts];
      if (r.next() % 5 == 0) path = 0;
      n[i] = 0;
      for (uint32_t j = 0; j < kDrafts; ++j)
        if (path >> j & 1) stay[i * kDrafts + n[i]++] = (int32_t)j;
    }
    CK(hipMemcpy(sees, who, sizeof who, hipMemcpyHostToDevice));
    CK(hipMemcpy(keep, stay, sizeof stay, hipMemcpyHostToDevice));
    CK(hipMemcpy(kept, n, sizeof n, hipMemcpyHostToDevice));
    for (uint32_t i = 0; i < kLayers; ++i) {
      const auto x = r.values((size_t)kTokens * kQkv);
      CK(hipMemcpy(qkv[i], x.data(), x.size() * 2, hipMemcpyHostToDevice));
    }
    return 0;
  }
};

int contents(const Instance& x, std::vector<std::vector<uint8_t>>* all, char* msg, int msg_len) {
  std::vector<fdy_alloc> t(fdy_arena_count(x.arena));
  FD(fdy_arena_table(x.arena, t.data(), (uint32_t)t.size()));
  all->assign(t.size(), {});
  for (size_t i = 0; i < t.size(); ++i) {
    (*all)[i].resize(t[i].size);
    CK(hipMemcpy((*all)[i].data(), (void*)(uintptr_t)t[i].base, t[i].size, hipMemcpyDeviceToHost));
  }
  return 0;
}

}  // namespace

extern "C" int draft_graph_check(char* msg, int msg_len) {
  hipStream_t stream;
  CK(hipStreamCreate(&stream));
  Instance A, B, C;
  if (A.allocate(0x220000000000ull, msg, msg_len) || B.allocate(0x320000000000ull, msg, msg_len) ||
      C.allocate(0x420000000000ull, msg, msg_len))
    return 1;
  if (A.prompts(stream, msg, msg_len) || C.prompts(stream, msg, msg_len)) return 1;

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
  CK(hipMemcpy(&words[n_nodes * kWords], A.planes, 2 * kLayers * 8, hipMemcpyDeviceToHost));
  hipGraphExec_t exec_a, exec_b;
  CK(hipGraphInstantiate(&exec_a, graph, nullptr, nullptr, 0));
  CK(hipGraphInstantiate(&exec_b, graph, nullptr, nullptr, 0));

  // all of A's addresses, wherever they lie in the arguments, become B's
  const uint32_t n_alloc = fdy_arena_count(A.arena);
  std::vector<fdy_alloc> ta(n_alloc), tb(n_alloc);
  FD(fdy_arena_table(A.arena, ta.data(), n_alloc));
  FD(fdy_arena_table(B.arena, tb.data(), n_alloc));
  std::vector<uint64_t> new_base(n_alloc);
  for (uint32_t i = 0; i < n_alloc; ++i) {
    new_base[i] = tb[i].base;
    if (i < A.scratch) CK(hipMemcpy((void*)(uintptr_t)tb[i].base, (void*)(uintptr_t)ta[i].base, ta[i].size, hipMemcpyDeviceToDevice));
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
  CK(hipMemcpy(B.planes, &words[n_nodes * kWords], 2 * kLayers * 8, hipMemcpyHostToDevice));
  for (size_t i = 0; i < n_nodes; ++i) {
    void* arg[1] = {&words[i * kWords]};
    hipKernelNodeParams np = params[i];
    np.kernelParams = arg;
    np.extra = nullptr;
    CK(hipGraphExecKernelNodeSetParams(exec_b, nodes[i], &np));
  }

  std::vector<std::vector<uint8_t>> a0, a1, b1, c1;
  std::vector<uint16_t> last(2 * kLayers);
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
    for (uint32_t i = 0; i < A.scratch; ++i)
      if (a1[i] != b1[i] || a1[i] != c1[i]) {
        snprintf(msg, msg_len, "step %d: allocation %u differs (%s)", s, i, a1[i] != b1[i] ? "rebased graph" : "plain calls");
        return 1;
      }
    uint32_t status = 0;
    CK(hipMemcpy(&status, B.status, 4, hipMemcpyDeviceToHost));
    bool finite = true, changed = true;
    for (uint32_t i = 0; i < 2 * kLayers; ++i) {
      std::vector<uint16_t> out((i % 2 ? kRows : kTokens) * kHeads * kDim);
      CK(hipMemcpy(out.data(), i % 2 ? B.near_out[i / 2] : B.out[i / 2], out.size() * 2, hipMemcpyDeviceToHost));
      for (uint16_t x : out) finite = finite && (x & 0x7f80) != 0x7f80;
      uint16_t sum = 0;
      for (uint16_t x : out) sum = (uint16_t)(sum * 31 + x);
      changed = changed && sum != last[i];
      last[i] = sum;
    }
    if (status || !finite || !changed) {
      snprintf(msg, msg_len, "step %d: status %u, outputs %s", s, status, finite ? "unchanged" : "not finite");
      return 1;
    }
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
