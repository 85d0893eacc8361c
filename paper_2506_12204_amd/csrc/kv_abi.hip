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

// The arguments of an attention call whose own were checked.
int attend_args(const sem_kv_cache* cache, int32_t layer, const sem_kv_query* query,
                const int32_t* seqs, const int32_t* cu, int64_t n, void* workspace,
                size_t ws_bytes, KvAttendArgs& a) {
  const AttendPlan p = attend_plan(cache, query->heads, n, query->tokens, query->max_new,
                                   query->max_len);
  if (!workspace_ok(workspace, ws_bytes, p.total)) return SEM_EINVAL;
  char* base = static_cast<char*>(workspace);
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
  return SEM_OK;
}

// The plan, sources and scales of sequences that keep `total` tokens among their
// listed ones.
struct KeepLayout {
  size_t kept = kZeroed, source = 0, pages = 0, scales = 0, total = 0;
};

KeepLayout keep_layout(const sem_kv_cache* c, int64_t n, int64_t sources, int64_t blocks) {
  KeepLayout L;
  L.source = align_up(L.kept + sizeof(KvKept) * (size_t)n);
  L.pages = align_up(L.source + 8 * (size_t)sources);
  L.scales = align_up(L.pages + 4 * (size_t)sources);
  L.total = align_up(L.scales + 4 * (size_t)blocks * (size_t)(c->layers * 2 * c->kv_heads));
  return L;
}

KeepLayout keep_layout(const sem_kv_cache* c, int64_t n, int64_t total) {
  // (a sequence's first block may begin a page before its first listed token, and
  // its last one ends a page after it)
  return keep_layout(c, n, total + n * c->page_tokens, total / c->page_tokens + 2 * n);
}

KvKeepArgs keep_args(const sem_kv_cache* c, const KeepLayout& L, const int32_t* seqs, int64_t n,
                     void* workspace) {
  char* base = static_cast<char*>(workspace);
  KvKeepArgs a = {};
  a.c = view_of(c, workspace);
  a.seqs = seqs;
  a.n = n;
  a.kept = reinterpret_cast<KvKept*>(base + L.kept);
  a.source = reinterpret_cast<int64_t*>(base + L.source);
  a.pages = reinterpret_cast<int32_t*>(base + L.pages);
  a.scales = reinterpret_cast<float*>(base + L.scales);
  return a;
}

int check_keep(const sem_kv_cache* c, const int32_t* seqs, const int32_t* last,
               const int32_t* index, const int32_t* cu, int64_t n, int64_t total) {
  int rc = check_cache(c);
  if (rc == SEM_OK) rc = check_list(c, seqs, n);
  if (rc != SEM_OK) return rc;
  if (total < 0 || total > INT32_MAX || (n == 0 && total > 0) || (n > 0 && (!last || !cu)) ||
      (total > 0 && !index))
    return SEM_EINVAL;
  return SEM_OK;
}

int64_t most_tokens(const sem_kv_cache* c) { return (int64_t)c->max_blocks * c->page_tokens; }

int check_mass(const sem_kv_cache* c, const float* mass, int64_t mass_stride) {
  if (mass_stride < most_tokens(c) || reinterpret_cast<uintptr_t>(mass) % 4 != 0)
    return SEM_EINVAL;
  return !mass && c->slots > 0 && most_tokens(c) > 0 ? SEM_EINVAL : SEM_OK;
}

int check_weigh(const sem_kv_cache* c, int32_t layer, const sem_kv_query* q, const int32_t* seqs,
                const int32_t* cu, int64_t n, const float* mass, int64_t mass_stride) {
  if (!q) return check_cache(c) == SEM_OK ? SEM_EINVAL : check_cache(c);
  sem_kv_query asked = *q;  // (its output is not looked at)
  asked.out = const_cast<void*>(q->q);
  asked.out_token_stride = asked.out_head_stride = 0;
  int rc = check_attend(c, layer, &asked, seqs, cu, n);
  if (rc == SEM_OK) rc = check_mass(c, mass, mass_stride);
  if (rc != SEM_OK) return rc;
  return q->tokens > 0 && !q->lse ? SEM_EINVAL : SEM_OK;
}

// A sequence keeps no more than it can hold.
KeepLayout prune_layout(const sem_kv_cache* c, int64_t n, int64_t budget) {
  budget = std::min(budget, most_tokens(c));
  return keep_layout(c, n, n * budget, n * ((budget + c->page_tokens - 1) / c->page_tokens));
}

int check_prune(const sem_kv_cache* c, const float* mass, int64_t mass_stride, const int32_t* seqs,
                int64_t n, int64_t budget, int64_t sinks, int64_t recent) {
  int rc = check_cache(c);
  if (rc == SEM_OK) rc = check_list(c, seqs, n);
  if (rc == SEM_OK) rc = check_mass(c, mass, mass_stride);
  if (rc != SEM_OK) return rc;
  return budget < 0 || sinks < 0 || recent < 0 ? SEM_EINVAL : SEM_OK;
}

int check_words(int32_t mask_words) {
  return mask_words < 1 || mask_words > kKvMaskWords ? SEM_EINVAL : SEM_OK;
}

int check_tree(const sem_kv_cache* c, const int32_t* parents, const int32_t* seqs,
               const int32_t* cu, int64_t n, int64_t tokens, int32_t mask_words,
               const uint32_t* mask, const int32_t* positions) {
  int rc = check_cache(c);
  if (rc == SEM_OK) rc = check_rows(c, 0, seqs, cu, n, tokens);
  if (rc == SEM_OK) rc = check_words(mask_words);
  if (rc != SEM_OK) return rc;
  return tokens > 0 && (!parents || !mask || !positions) ? SEM_EINVAL : SEM_OK;
}

int check_attend_tree(const sem_kv_cache* c, int32_t layer, const sem_kv_query* q,
                      const uint32_t* mask, int32_t mask_words, const int32_t* seqs,
                      const int32_t* cu, int64_t n) {
  int rc = check_attend(c, layer, q, seqs, cu, n);
  if (rc == SEM_OK) rc = check_words(mask_words);
  if (rc != SEM_OK) return rc;
  // (what a row sees is in its mask)
  return !q->causal || q->window != 0 || (q->tokens > 0 && !mask) ? SEM_EINVAL : SEM_OK;
}

int check_rotate(const sem_qk_rotary* r) {
  if (!r || r->tokens < 0 || r->tokens > INT32_MAX || r->heads < 0 || r->kv_heads < 0 ||
      (r->dtype != SEM_KV_BF16 && r->dtype != SEM_KV_F16) || !std::isfinite(r->eps) || r->eps < 0)
    return SEM_EINVAL;
  if (r->rot_dim < 0 || r->rot_dim > r->head_dim || r->rot_dim % 16 != 0) return SEM_EINVAL;
  for (const int64_t stride : {r->q_token_stride, r->q_head_stride, r->k_token_stride,
                               r->k_head_stride, r->q_out_token_stride, r->q_out_head_stride,
                               r->k_out_token_stride, r->k_out_head_stride})
    if (stride < 0) return SEM_EINVAL;
  if (r->tokens > 0 && ((r->heads > 0 && (!r->q || !r->q_out)) ||
                        (r->kv_heads > 0 && (!r->k || !r->k_out)) ||
                        (r->rot_dim > 0 && (!r->positions || !r->inv_freq))))
    return SEM_EINVAL;
  for (const void* p : {r->q, r->k, (const void*)r->q_out, (const void*)r->k_out})
    if (reinterpret_cast<uintptr_t>(p) % 2 != 0) return SEM_EINVAL;
  for (const void* p : {(const void*)r->positions, (const void*)r->inv_freq,
                        (const void*)r->q_weight, (const void*)r->k_weight})
    if (reinterpret_cast<uintptr_t>(p) % 4 != 0) return SEM_EINVAL;
  if (r->head_dim != 64 && r->head_dim != 128 && r->head_dim != 256) return SEM_ENOTIMPL;
  if (r->heads > 65536 || r->kv_heads > 65536) return SEM_ENOTIMPL;
  return SEM_OK;
}

}  // namespace

extern "C" {

int sem_qk_rotate_async(const sem_qk_rotary* rotary, void* stream) {
  const int rc = check_rotate(rotary);
  if (rc != SEM_OK) return rc;
  const sem_qk_rotary& r = *rotary;
  QkRotateArgs a = {};
  a.q = static_cast<const uint16_t*>(r.q);
  a.k = static_cast<const uint16_t*>(r.k);
  a.q_out = static_cast<uint16_t*>(r.q_out);
  a.k_out = static_cast<uint16_t*>(r.k_out);
  a.q_token = r.q_token_stride;
  a.q_head = r.q_head_stride;
  a.k_token = r.k_token_stride;
  a.k_head = r.k_head_stride;
  a.qo_token = r.q_out_token_stride;
  a.qo_head = r.q_out_head_stride;
  a.ko_token = r.k_out_token_stride;
  a.ko_head = r.k_out_head_stride;
  a.positions = r.positions;
  a.inv_freq = r.inv_freq;
  a.q_weight = r.q_weight;
  a.k_weight = r.k_weight;
  a.tokens = r.heads + r.kv_heads > 0 ? r.tokens : 0;
  a.heads = r.heads;
  a.kv_heads = r.kv_heads;
  a.rot_dim = r.rot_dim;
  a.bf16 = r.dtype == SEM_KV_BF16;
  a.pairs = r.interleaved != 0;
  a.wide = (r.heads == 0 || (aligned16(r.q, a.q_token, a.q_head) &&
                             aligned16(r.q_out, a.qo_token, a.qo_head))) &&
           (r.kv_heads == 0 || (aligned16(r.k, a.k_token, a.k_head) &&
                                aligned16(r.k_out, a.ko_token, a.ko_head)));
  a.eps = r.eps;
  return status_of(launch_qk_rotate(a, r.head_dim, static_cast<hipStream_t>(stream)));
}

int sem_qk_rotate(const sem_qk_rotary* rotary) {
  const int rc = check_rotate(rotary);
  if (rc != SEM_OK) return rc;
  return blocking(kZeroed, [&](void*, size_t, hipStream_t st) {
    return sem_qk_rotate_async(rotary, st);
  });
}

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
  int rc = check_attend(cache, layer, query, seqs, cu, n);
  if (rc != SEM_OK) return rc;
  KvAttendArgs a = {};
  rc = attend_args(cache, layer, query, seqs, cu, n, workspace, ws_bytes, a);
  return rc == SEM_OK ? status_of(launch_kv_attend(a, static_cast<hipStream_t>(stream))) : rc;
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

int sem_kv_attend_tree_async(const sem_kv_cache* cache, int32_t layer, const sem_kv_query* query,
                             const uint32_t* mask, int32_t mask_words, const int32_t* seqs,
                             const int32_t* cu, int64_t n, void* workspace, size_t ws_bytes,
                             void* stream) {
  int rc = check_attend_tree(cache, layer, query, mask, mask_words, seqs, cu, n);
  if (rc != SEM_OK) return rc;
  KvAttendArgs a = {};
  rc = attend_args(cache, layer, query, seqs, cu, n, workspace, ws_bytes, a);
  if (rc != SEM_OK) return rc;
  a.causal = 0;
  a.mask = mask;
  a.mask_words = mask_words;
  return status_of(launch_kv_attend_tree(a, static_cast<hipStream_t>(stream)));
}

int sem_kv_attend_tree(const sem_kv_cache* cache, int32_t layer, const sem_kv_query* query,
                       const uint32_t* mask, int32_t mask_words, const int32_t* seqs,
                       const int32_t* cu, int64_t n) {
  const int rc = check_attend_tree(cache, layer, query, mask, mask_words, seqs, cu, n);
  if (rc != SEM_OK) return rc;
  const size_t need = attend_plan(cache, query->heads, n, query->tokens, query->max_new,
                                  query->max_len).total;
  return blocking(need, [&](void* ws, size_t bytes, hipStream_t st) {
    return sem_kv_attend_tree_async(cache, layer, query, mask, mask_words, seqs, cu, n, ws, bytes,
                                    st);
  });
}

int sem_kv_tree_async(const sem_kv_cache* cache, const int32_t* parents, const int32_t* starts,
                      const int32_t* seqs, const int32_t* cu, int64_t n, int64_t tokens,
                      int32_t mask_words, uint32_t* mask_out, int32_t* positions_out,
                      void* workspace, size_t ws_bytes, void* stream) {
  const int rc = check_tree(cache, parents, seqs, cu, n, tokens, mask_words, mask_out,
                            positions_out);
  if (rc != SEM_OK) return rc;
  if (!workspace_ok(workspace, ws_bytes, kZeroed)) return SEM_EINVAL;
  KvTreeArgs a = {};
  a.c = view_of(cache, workspace);
  a.parents = parents;
  a.starts = starts;
  a.seqs = seqs;
  a.cu = cu;
  a.n = n;
  a.tokens = tokens;
  a.words = mask_words;
  a.mask = mask_out;
  a.positions = positions_out;
  return status_of(launch_kv_tree(a, static_cast<hipStream_t>(stream)));
}

int sem_kv_tree(const sem_kv_cache* cache, const int32_t* parents, const int32_t* starts,
                const int32_t* seqs, const int32_t* cu, int64_t n, int64_t tokens,
                int32_t mask_words, uint32_t* mask_out, int32_t* positions_out) {
  const int rc = check_tree(cache, parents, seqs, cu, n, tokens, mask_words, mask_out,
                            positions_out);
  if (rc != SEM_OK) return rc;
  return blocking(kZeroed, [&](void* ws, size_t bytes, hipStream_t st) {
    return sem_kv_tree_async(cache, parents, starts, seqs, cu, n, tokens, mask_words, mask_out,
                             positions_out, ws, bytes, st);
  });
}

size_t sem_kv_keep_workspace_bytes(const sem_kv_cache* cache, int64_t n, int64_t total) {
  if (check_sizes(cache) != SEM_OK || n < 0 || n > cache->slots || total < 0 || total > INT32_MAX)
    return 0;
  return keep_layout(cache, n, total).total;
}

int sem_kv_keep_async(const sem_kv_cache* cache, const int32_t* seqs, const int32_t* last,
                      const int32_t* index, const int32_t* cu, int64_t n, int64_t total,
                      void* workspace, size_t ws_bytes, void* stream) {
  const int rc = check_keep(cache, seqs, last, index, cu, n, total);
  if (rc != SEM_OK) return rc;
  const KeepLayout L = keep_layout(cache, n, total);
  if (!workspace_ok(workspace, ws_bytes, L.total)) return SEM_EINVAL;
  KvKeepArgs a = keep_args(cache, L, seqs, n, workspace);
  a.last = last;
  a.index = index;
  a.cu = cu;
  a.total = total;
  return status_of(launch_kv_keep(a, static_cast<hipStream_t>(stream)));
}

int sem_kv_keep(const sem_kv_cache* cache, const int32_t* seqs, const int32_t* last,
                const int32_t* index, const int32_t* cu, int64_t n, int64_t total) {
  const int rc = check_keep(cache, seqs, last, index, cu, n, total);
  if (rc != SEM_OK) return rc;
  return blocking(keep_layout(cache, n, total).total, [&](void* ws, size_t bytes, hipStream_t st) {
    return sem_kv_keep_async(cache, seqs, last, index, cu, n, total, ws, bytes, st);
  });
}

int sem_kv_weigh_async(const sem_kv_cache* cache, int32_t layer, const sem_kv_query* query,
                       const int32_t* seqs, const int32_t* cu, int64_t n, float* mass,
                       int64_t mass_stride, void* workspace, size_t ws_bytes, void* stream) {
  const int rc = check_weigh(cache, layer, query, seqs, cu, n, mass, mass_stride);
  if (rc != SEM_OK) return rc;
  if (!workspace_ok(workspace, ws_bytes, kZeroed)) return SEM_EINVAL;
  KvWeighArgs a = {};
  a.c = view_of(cache, workspace);
  a.q = static_cast<const uint16_t*>(query->q);
  a.lse = query->lse;
  a.mass = mass;
  a.q_token = query->q_token_stride;
  a.q_head = query->q_head_stride;
  a.mass_stride = mass_stride;
  a.seqs = seqs;
  a.cu = cu;
  a.n = n;
  a.tokens = query->tokens;
  a.layer = layer;
  a.heads = query->heads;
  a.group = query->heads / cache->kv_heads;
  a.bf16 = query->dtype == SEM_KV_BF16;
  a.causal = query->causal != 0;
  a.window = query->window;
  a.scale_log2 = query->scale * 1.4426950408889634f;
  const int64_t most = most_tokens(cache);
  const int64_t max_len = query->max_len > 0 ? std::min(query->max_len, most) : most;
  const int64_t max_new = !cu ? 1 : query->max_new > 0 ? query->max_new : query->tokens;
  return status_of(launch_kv_weigh(a, std::min(max_new, query->tokens), max_len,
                                   static_cast<hipStream_t>(stream)));
}

int sem_kv_weigh(const sem_kv_cache* cache, int32_t layer, const sem_kv_query* query,
                 const int32_t* seqs, const int32_t* cu, int64_t n, float* mass,
                 int64_t mass_stride) {
  const int rc = check_weigh(cache, layer, query, seqs, cu, n, mass, mass_stride);
  if (rc != SEM_OK) return rc;
  return blocking(kZeroed, [&](void* ws, size_t bytes, hipStream_t st) {
    return sem_kv_weigh_async(cache, layer, query, seqs, cu, n, mass, mass_stride, ws, bytes, st);
  });
}

size_t sem_kv_prune_workspace_bytes(const sem_kv_cache* cache, int64_t n, int64_t budget) {
  if (check_sizes(cache) != SEM_OK || n < 0 || n > cache->slots || budget < 0) return 0;
  return prune_layout(cache, n, budget).total;
}

int sem_kv_prune_async(const sem_kv_cache* cache, float* mass, int64_t mass_stride,
                       const int32_t* seqs, int64_t n, int64_t budget, int64_t sinks,
                       int64_t recent, void* workspace, size_t ws_bytes, void* stream) {
  const int rc = check_prune(cache, mass, mass_stride, seqs, n, budget, sinks, recent);
  if (rc != SEM_OK) return rc;
  const KeepLayout L = prune_layout(cache, n, budget);
  if (!workspace_ok(workspace, ws_bytes, L.total)) return SEM_EINVAL;
  KvPruneArgs a = {};
  a.k = keep_args(cache, L, seqs, n, workspace);
  a.mass = mass;
  a.mass_stride = mass_stride;
  a.budget = std::min(budget, most_tokens(cache));
  a.sinks = sinks;
  a.recent = recent;
  return status_of(launch_kv_prune(a, static_cast<hipStream_t>(stream)));
}

int sem_kv_prune(const sem_kv_cache* cache, float* mass, int64_t mass_stride, const int32_t* seqs,
                 int64_t n, int64_t budget, int64_t sinks, int64_t recent) {
  const int rc = check_prune(cache, mass, mass_stride, seqs, n, budget, sinks, recent);
  if (rc != SEM_OK) return rc;
  return blocking(prune_layout(cache, n, budget).total,
                  [&](void* ws, size_t bytes, hipStream_t st) {
                    return sem_kv_prune_async(cache, mass, mass_stride, seqs, n, budget, sinks,
                                              recent, ws, bytes, st);
                  });
}

}  // extern "C"
