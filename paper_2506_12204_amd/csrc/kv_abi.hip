// C ABI of the paged 8-bit KV cache: argument checks, workspace layout and
// launches. The operations are defined in semsched.h; every step of them runs
// in kv_pages.hip, kv_append.hip and kv_attend.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "abi_common.h"
#include "kv.h"
#include "semsched.h"

using namespace semsched;

namespace {

// What callers zero: the status word's 256 bytes and the counters.
constexpr size_t kZeroed = kHeaderBytes + 4 * (size_t)kKvCounts;
static_assert(kZeroed == SEM_KV_ZEROED_BYTES, "the header's size is the layouts'");

constexpr int32_t kMaxLayers = 4096, kMaxHeads = 1024, kMaxPageTokens = 1024;

// The sizes alone (no pointer is looked at).
int check_sizes(const sem_kv_cache* c) {
  if (!c || c->num_pages < 0 || c->num_pages > INT32_MAX || c->slots < 0 || c->max_blocks < 0 ||
      c->layers < 1 || c->layers > kMaxLayers || c->kv_heads < 1 || c->kv_heads > kMaxHeads ||
      (c->format != SEM_KV_INT8 && c->format != SEM_KV_FP8))
    return SEM_EINVAL;
  if (c->page_tokens < kKvTile || c->page_tokens > kMaxPageTokens ||
      (c->page_tokens & (c->page_tokens - 1)) != 0 ||
      (int64_t)c->max_blocks * c->page_tokens > INT32_MAX)
    return SEM_EINVAL;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return SEM_ENOTIMPL;
  return SEM_OK;
}

int64_t page_bytes(const sem_kv_cache* c) {
  return (int64_t)c->layers * 2 * c->kv_heads * c->page_tokens * c->head_dim;
}

int check_cache(const sem_kv_cache* c) {
  const int rc = check_sizes(c);
  if (rc != SEM_OK) return rc;
  if (c->num_pages > 0 && (!c->data || !c->scale || !c->live || !c->refs)) return SEM_EINVAL;
  if (c->slots > 0 && (!c->lens || (c->max_blocks > 0 && !c->tables))) return SEM_EINVAL;
  if (reinterpret_cast<uintptr_t>(c->data) % 16 != 0) return SEM_EINVAL;
  return SEM_OK;
}

KvView view_of(const sem_kv_cache* c, void* ws) {
  KvView v = {};
  v.data = static_cast<uint8_t*>(c->data);
  v.scale = c->scale;
  v.live = c->live;
  v.refs = c->refs;
  v.lens = c->lens;
  v.tables = c->tables;
  v.num_pages = c->num_pages;
  v.page_bytes = page_bytes(c);
  v.slots = c->slots;
  v.max_blocks = c->max_blocks;
  v.layers = c->layers;
  v.kv_heads = c->kv_heads;
  v.head_dim = c->head_dim;
  v.page_tokens = c->page_tokens;
  v.page_shift = __builtin_ctz((unsigned)c->page_tokens);
  v.format = c->format;
  v.page_scales = c->layers * 2 * c->kv_heads;
  v.flags = static_cast<uint32_t*>(ws);
  return v;
}

// Reserve's lists and compact's lists share the space after the header.
struct PagesLayout {
  size_t ncopies = 64, counts = 64;  // in the header, after the status word
  size_t begin = 0, copies = 0, fresh = 0, moves = 0, remap = 0, total = kZeroed;
};

PagesLayout pages_layout(const sem_kv_cache* c) {
  PagesLayout L;
  size_t off = kZeroed;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = align_up(off + bytes);
    return at;
  };
  const size_t slots = (size_t)c->slots, pages = (size_t)c->num_pages;
  L.begin = take(4 * slots);
  L.copies = take(8 * slots);
  L.fresh = take(4 * pages);
  const size_t reserve = off;
  off = kZeroed;
  L.moves = take(8 * (pages / 2 + 1));
  L.remap = take(4 * pages);
  L.total = std::max(off, reserve);
  return L;
}

bool workspace_ok(const void* ws, size_t have, size_t need) {
  return ws && have >= need && reinterpret_cast<uintptr_t>(ws) % kAlign == 0;
}

int status_of(hipError_t e) {
  // (a grid that is too large: the call has launched nothing)
  if (e == hipErrorInvalidConfiguration) return SEM_ENOTIMPL;
  return e == hipSuccess ? SEM_OK : SEM_EDEVICE;
}

// A blocking call: the library's workspace with its first bytes zeroed, the
// asynchronous form on the blocking calls' stream, the status.
template <typename F>
int blocking(size_t bytes, F enqueue) {
  std::lock_guard<std::mutex> g(blocking_mutex());
  void* ws = nullptr;
  int rc = blocking_workspace(bytes, &ws);
  if (rc != SEM_OK) return rc;
  const hipStream_t st = blocking_stream();
  if (launch_fill_zero(static_cast<uint32_t*>(ws), kZeroed / 4, st) != hipSuccess)
    return SEM_EDEVICE;
  rc = enqueue(ws, bytes, st);
  return rc != SEM_OK ? rc : blocking_finish(ws, st);
}

int check_list(const sem_kv_cache* c, const void* list, int64_t n) {
  if (n < 0 || n > c->slots) return SEM_EINVAL;  // a sequence is listed once at most
  return n > 0 && !list ? SEM_EINVAL : SEM_OK;
}

int check_rows(const sem_kv_cache* c, int32_t layer, const int32_t* seqs, const int32_t* cu,
               int64_t n, int64_t tokens) {
  const int rc = check_list(c, seqs, n);
  if (rc != SEM_OK) return rc;
  if (layer < 0 || layer >= c->layers || tokens < 0 || tokens > INT32_MAX) return SEM_EINVAL;
  if (!cu && tokens != n) return SEM_EINVAL;  // without offsets one token each
  if (n == 0 && tokens > 0) return SEM_EINVAL;  // rows of no sequence
  return SEM_OK;
}

bool aligned16(const void* p, int64_t a, int64_t b) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && a % 8 == 0 && b % 8 == 0;
}

int check_lists(const sem_kv_cache* c, const int32_t* x, const int32_t* y, int64_t n) {
  int rc = check_cache(c);
  if (rc == SEM_OK) rc = check_list(c, x, n);
  return rc == SEM_OK ? check_list(c, y, n) : rc;
}

int check_free(const sem_kv_cache* c, const int32_t* seqs, int64_t n) {
  const int rc = check_cache(c);
  return rc == SEM_OK ? check_list(c, seqs, n) : rc;
}

int check_append(const sem_kv_cache* c, int32_t layer, const void* k, const void* v, int32_t dtype,
                 int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head,
                 const int32_t* seqs, const int32_t* cu, int64_t n, int64_t tokens) {
  int rc = check_cache(c);
  if (rc == SEM_OK) rc = check_rows(c, layer, seqs, cu, n, tokens);
  if (rc != SEM_OK) return rc;
  if ((dtype != SEM_KV_BF16 && dtype != SEM_KV_F16) || (tokens > 0 && (!k || !v)) ||
      k_token < 0 || k_head < 0 || v_token < 0 || v_head < 0 ||
      reinterpret_cast<uintptr_t>(k) % 2 != 0 || reinterpret_cast<uintptr_t>(v) % 2 != 0)
    return SEM_EINVAL;
  return SEM_OK;
}

struct AttendPlan {
  KvSplit split = {};
  size_t part_o = 0, part_ml = 0, cuts = 0, total = kZeroed;
};

AttendPlan attend_plan(const sem_kv_cache* c, int32_t heads, int64_t n, int64_t tokens,
                       int64_t max_new, int64_t max_len) {
  AttendPlan p;
  max_len = std::min<int64_t>(max_len > 0 ? max_len : INT32_MAX,
                              (int64_t)c->max_blocks * c->page_tokens);
  max_new = std::min<int64_t>(max_new > 0 ? max_new : tokens, std::max<int64_t>(tokens, 1));
  p.split = kv_attend_split(c->head_dim, n, tokens, heads, c->kv_heads, max_new, max_len);
  if (p.split.part_rows > 0) {
    const size_t rows = (size_t)p.split.part_rows;
    p.part_o = kZeroed;
    p.part_ml = align_up(p.part_o + 4 * rows * (size_t)c->head_dim);
    p.cuts = align_up(p.part_ml + 8 * rows);
    p.total = align_up(p.cuts + (p.split.tiled ? kKvPieces * sizeof(KvCut) : 0));
  }
  return p;
}

int check_attend(const sem_kv_cache* c, int32_t layer, const sem_kv_query* q, const int32_t* seqs,
                 const int32_t* cu, int64_t n) {
  int rc = check_cache(c);
  if (rc != SEM_OK) return rc;
  if (!q) return SEM_EINVAL;
  rc = check_rows(c, layer, seqs, cu, n, q->tokens);
  if (rc != SEM_OK) return rc;
  if (q->heads < 1 || q->heads % c->kv_heads != 0 || q->window < 0 || !std::isfinite(q->scale) ||
      (q->dtype != SEM_KV_BF16 && q->dtype != SEM_KV_F16) || q->max_new < 0 || q->max_len < 0)
    return SEM_EINVAL;
  if (q->q_token_stride < 0 || q->q_head_stride < 0 || q->out_token_stride < 0 ||
      q->out_head_stride < 0)
    return SEM_EINVAL;
  if (q->tokens > 0 && (!q->q || !q->out)) return SEM_EINVAL;
  if (reinterpret_cast<uintptr_t>(q->q) % 2 != 0 || reinterpret_cast<uintptr_t>(q->out) % 2 != 0)
    return SEM_EINVAL;
  // (rows are counted in 32 bits)
  if (q->heads > 65536 || (q->tokens + n) * (int64_t)q->heads > INT32_MAX) return SEM_ENOTIMPL;
  return SEM_OK;
}

}  // namespace

extern "C" {

size_t sem_kv_page_bytes(const sem_kv_cache* cache) {
  return check_sizes(cache) == SEM_OK ? (size_t)page_bytes(cache) : 0;
}

size_t sem_kv_workspace_bytes(const sem_kv_cache* cache) {
  return check_sizes(cache) == SEM_OK ? pages_layout(cache).total : 0;
}

size_t sem_kv_attend_workspace_bytes(const sem_kv_cache* cache, int32_t heads, int64_t n,
                                     int64_t tokens, int64_t max_new, int64_t max_len) {
  if (check_sizes(cache) != SEM_OK || heads < 1 || heads % cache->kv_heads != 0 || n < 0 ||
      tokens < 0 || tokens > INT32_MAX || max_new < 0 || max_len < 0)
    return 0;
  return attend_plan(cache, heads, n, tokens, max_new, max_len).total;
}

int sem_kv_fork_async(const sem_kv_cache* cache, const int32_t* src, const int32_t* dst,
                      const int32_t* tokens, int64_t n, void* workspace, size_t ws_bytes,
                      void* stream) {
  const int rc = check_lists(cache, src, dst, n);
  if (rc != SEM_OK) return rc;
  if (!workspace_ok(workspace, ws_bytes, kZeroed)) return SEM_EINVAL;
  const KvForkArgs a = {view_of(cache, workspace), src, dst, tokens, n};
  return status_of(launch_kv_fork(a, static_cast<hipStream_t>(stream)));
}

int sem_kv_fork(const sem_kv_cache* cache, const int32_t* src, const int32_t* dst,
                const int32_t* tokens, int64_t n) {
  const int rc = check_lists(cache, src, dst, n);
  if (rc != SEM_OK) return rc;
  return blocking(kZeroed, [&](void* ws, size_t bytes, hipStream_t st) {
    return sem_kv_fork_async(cache, src, dst, tokens, n, ws, bytes, st);
  });
}

int sem_kv_free_async(const sem_kv_cache* cache, const int32_t* seqs, const int32_t* keep,
                      int64_t n, void* workspace, size_t ws_bytes, void* stream) {
  const int rc = check_free(cache, seqs, n);
  if (rc != SEM_OK) return rc;
  if (!workspace_ok(workspace, ws_bytes, kZeroed)) return SEM_EINVAL;
  const KvFreeArgs a = {view_of(cache, workspace), seqs, keep, n};
  return status_of(launch_kv_free(a, static_cast<hipStream_t>(stream)));
}

int sem_kv_free(const sem_kv_cache* cache, const int32_t* seqs, const int32_t* keep, int64_t n) {
  const int rc = check_free(cache, seqs, n);
  if (rc != SEM_OK) return rc;
  return blocking(kZeroed, [&](void* ws, size_t bytes, hipStream_t st) {
    return sem_kv_free_async(cache, seqs, keep, n, ws, bytes, st);
  });
}

int sem_kv_reserve_async(const sem_kv_cache* cache, const int32_t* seqs, const int32_t* tokens,
                         int64_t n, void* workspace, size_t ws_bytes, void* stream) {
  const int rc = check_lists(cache, seqs, tokens, n);
  if (rc != SEM_OK) return rc;
  const PagesLayout L = pages_layout(cache);
  if (!workspace_ok(workspace, ws_bytes, L.total)) return SEM_EINVAL;
  char* base = static_cast<char*>(workspace);
  KvReserveArgs a = {};
  a.c = view_of(cache, workspace);
  a.seqs = seqs;
  a.grow = tokens;
  a.n = n;
  a.begin = reinterpret_cast<uint32_t*>(base + L.begin);
  a.fresh = reinterpret_cast<uint32_t*>(base + L.fresh);
  a.copies = reinterpret_cast<uint64_t*>(base + L.copies);
  a.ncopies = reinterpret_cast<uint32_t*>(base + L.ncopies);
  a.room = cache->num_pages;
  return status_of(launch_kv_reserve(a, static_cast<hipStream_t>(stream)));
}

int sem_kv_reserve(const sem_kv_cache* cache, const int32_t* seqs, const int32_t* tokens,
                   int64_t n) {
  const int rc = check_lists(cache, seqs, tokens, n);
  if (rc != SEM_OK) return rc;
  return blocking(pages_layout(cache).total, [&](void* ws, size_t bytes, hipStream_t st) {
    return sem_kv_reserve_async(cache, seqs, tokens, n, ws, bytes, st);
  });
}

int sem_kv_compact_async(const sem_kv_cache* cache, void* workspace, size_t ws_bytes,
                         void* stream) {
  const int rc = check_cache(cache);
  if (rc != SEM_OK) return rc;
  const PagesLayout L = pages_layout(cache);
  if (!workspace_ok(workspace, ws_bytes, L.total)) return SEM_EINVAL;
  char* base = static_cast<char*>(workspace);
  KvCompactArgs a = {};
  a.c = view_of(cache, workspace);
  a.moves = reinterpret_cast<uint64_t*>(base + L.moves);
  a.remap = reinterpret_cast<uint32_t*>(base + L.remap);
  a.counts = reinterpret_cast<uint32_t*>(base + L.counts);
  return status_of(launch_kv_compact(a, static_cast<hipStream_t>(stream)));
}

int sem_kv_compact(const sem_kv_cache* cache) {
  const int rc = check_cache(cache);
  if (rc != SEM_OK) return rc;
  return blocking(pages_layout(cache).total, [&](void* ws, size_t bytes, hipStream_t st) {
    return sem_kv_compact_async(cache, ws, bytes, st);
  });
}

int sem_kv_append_async(const sem_kv_cache* cache, int32_t layer, const void* k, const void* v,
                        int32_t dtype, int64_t k_token_stride, int64_t k_head_stride,
                        int64_t v_token_stride, int64_t v_head_stride, const int32_t* seqs,
                        const int32_t* cu, int64_t n, int64_t tokens, void* workspace,
                        size_t ws_bytes, void* stream) {
  const int rc = check_append(cache, layer, k, v, dtype, k_token_stride, k_head_stride,
                              v_token_stride, v_head_stride, seqs, cu, n, tokens);
  if (rc != SEM_OK) return rc;
  if (!workspace_ok(workspace, ws_bytes, kZeroed)) return SEM_EINVAL;
  KvAppendArgs a = {};
  a.c = view_of(cache, workspace);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.k_token = k_token_stride;
  a.k_head = k_head_stride;
  a.v_token = v_token_stride;
  a.v_head = v_head_stride;
  a.seqs = seqs;
  a.cu = cu;
  a.n = n;
  a.tokens = tokens;
  a.layer = layer;
  a.bf16 = dtype == SEM_KV_BF16;
  a.wide = aligned16(k, k_token_stride, k_head_stride) && aligned16(v, v_token_stride, v_head_stride);
  return status_of(launch_kv_append(a, static_cast<hipStream_t>(stream)));
}

int sem_kv_append(const sem_kv_cache* cache, int32_t layer, const void* k, const void* v,
                  int32_t dtype, int64_t k_token_stride, int64_t k_head_stride,
                  int64_t v_token_stride, int64_t v_head_stride, const int32_t* seqs,
                  const int32_t* cu, int64_t n, int64_t tokens) {
  const int rc = check_append(cache, layer, k, v, dtype, k_token_stride, k_head_stride,
                              v_token_stride, v_head_stride, seqs, cu, n, tokens);
  if (rc != SEM_OK) return rc;
  return blocking(kZeroed, [&](void* ws, size_t bytes, hipStream_t st) {
    return sem_kv_append_async(cache, layer, k, v, dtype, k_token_stride, k_head_stride,
                               v_token_stride, v_head_stride, seqs, cu, n, tokens, ws, bytes, st);
  });
}

int sem_kv_attend_async(const sem_kv_cache* cache, int32_t layer, const sem_kv_query* query,
                        const int32_t* seqs, const int32_t* cu, int64_t n, void* workspace,
                        size_t ws_bytes, void* stream) {
  const int rc = check_attend(cache, layer, query, seqs, cu, n);
  if (rc != SEM_OK) return rc;
  const AttendPlan p = attend_plan(cache, query->heads, n, query->tokens, query->max_new,
                                   query->max_len);
  if (!workspace_ok(workspace, ws_bytes, p.total)) return SEM_EINVAL;
  char* base = static_cast<char*>(workspace);
  KvAttendArgs a = {};
  a.c = view_of(cache, workspace);
  a.q = static_cast<const uint16_t*>(query->q);
  a.out = static_cast<uint16_t*>(query->out);
  a.lse = query->lse;
  a.q_token = query->q_token_stride;
  a.q_head = query->q_head_stride;
  a.out_token = query->out_token_stride;
  a.out_head = query->out_head_stride;
  a.seqs = seqs;
  a.cu = cu;
  a.n = n;
  a.tokens = query->tokens;
  a.layer = layer;
  a.heads = query->heads;
  a.group = query->heads / cache->kv_heads;
  a.bf16 = query->dtype == SEM_KV_BF16;
  a.wide = aligned16(query->q, query->q_token_stride, query->q_head_stride);
  a.wide_out = aligned16(query->out, query->out_token_stride, query->out_head_stride);
  a.causal = query->causal != 0;
  a.window = query->window;
  a.scale_log2 = query->scale * 1.4426950408889634f;
  a.tiled = p.split.tiled;
  a.whole = p.split.whole;
  a.waves = p.split.waves;
  a.parts = p.split.parts;
  a.part_chunks = p.split.part_chunks;
  a.counts = reinterpret_cast<uint32_t*>(base + kHeaderBytes);
  a.part_o = reinterpret_cast<float*>(base + p.part_o);
  a.part_ml = reinterpret_cast<float*>(base + p.part_ml);
  a.cuts = reinterpret_cast<KvCut*>(base + p.cuts);
  return status_of(launch_kv_attend(a, static_cast<hipStream_t>(stream)));
}

int sem_kv_attend(const sem_kv_cache* cache, int32_t layer, const sem_kv_query* query,
                  const int32_t* seqs, const int32_t* cu, int64_t n) {
  const int rc = check_attend(cache, layer, query, seqs, cu, n);
  if (rc != SEM_OK) return rc;
  const size_t need = attend_plan(cache, query->heads, n, query->tokens, query->max_new,
                                  query->max_len).total;
  return blocking(need, [&](void* ws, size_t bytes, hipStream_t st) {
    return sem_kv_attend_async(cache, layer, query, seqs, cu, n, ws, bytes, st);
  });
}

}  // extern "C"
