// Host/device interface of the paged 8-bit KV cache (internal to the library;
// the operations are defined in semsched.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"

namespace semsched {

constexpr int kKvCounts = 1024;      // counters of attention's tiles with several parts
constexpr int kKvPieces = 256;       // of attention's work, where it is cut into equal ones
constexpr int kKvTile = 16;          // tokens per tile of a page's block
constexpr int kKvMaskWords = 128;    // most words of a drafted token's mask

// The cache as the kernels see it: the caller's arrays and the derived sizes.
struct KvView {
  uint8_t* data;    // [num_pages][layers][2][kv_heads][page_tokens * head_dim]
  float* scale;     // [num_pages][layers][2][kv_heads]
  uint32_t* live;   // one bit per page
  int32_t* refs;    // [num_pages]
  int32_t* lens;    // [slots]
  int32_t* tables;  // [slots][max_blocks], -1 beyond a sequence's blocks
  int64_t num_pages, page_bytes;
  int32_t slots, max_blocks, layers, kv_heads, head_dim, page_tokens, page_shift, format;
  int32_t page_scales;  // layers * 2 * kv_heads
  uint32_t* flags;
};

struct KvForkArgs {
  KvView c;
  const int32_t *src, *dst, *tokens;  // tokens may be null: the whole source
  int64_t n;
};

struct KvFreeArgs {
  KvView c;
  const int32_t *seqs, *keep;  // keep may be null: all 0
  int64_t n;
};

struct KvReserveArgs {
  KvView c;
  const int32_t *seqs, *grow;
  int64_t n;
  uint32_t* begin;    // [n] first entry of each sequence in `fresh`
  uint32_t* fresh;    // [room] the free pages taken, ascending
  uint64_t* copies;   // [n] pages to copy: from | to << 32
  uint32_t* ncopies;  // [1]
  int64_t room;       // entries of `fresh`
};

struct KvCompactArgs {
  KvView c;
  uint64_t* moves;   // [num_pages / 2] from | to << 32
  uint32_t* remap;   // [num_pages] where a moved page goes
  uint32_t* counts;  // [2] moves, live pages
};

struct KvAppendArgs {
  KvView c;
  const uint16_t *k, *v;  // 16-bit elements
  int64_t k_token, k_head, v_token, v_head;  // strides in elements
  const int32_t *seqs, *cu;                  // cu may be null: one token each
  int64_t n, tokens;
  int32_t layer;
  int32_t bf16;  // else IEEE half
  int32_t wide;  // 16-byte loads are aligned
  uint32_t units;  // of work (set by the launch); workgroups behind them check offsets
};

// A row tile whose keys went to several of attention's pieces.
struct KvCut {
  int32_t parts, piece;  // how many (0: none), the first of them
  int32_t row0, rows;    // the sequence's first query token, rows of a KV head
  int32_t tile, head;    // its number in the sequence, the KV head
};

struct KvAttendArgs {
  KvView c;
  const uint16_t* q;
  uint16_t* out;
  float* lse;  // [tokens][heads], may be null
  int64_t q_token, q_head, out_token, out_head;  // strides in elements
  const int32_t *seqs, *cu;
  int64_t n, tokens;
  int32_t layer, heads, group;
  int32_t bf16, wide, wide_out;  // 16-byte accesses to q, to out, are aligned
  int32_t causal, window;
  float scale_log2;  // softmax scale * log2(e)
  int32_t tiled;       // the kernel for many rows per sequence
  int32_t whole;       // a tile per workgroup of it, else a piece of all tiles' keys
  int32_t waves;       // of the other kernel's workgroups, 4 or 8
  int32_t parts;       // most parts that the keys of a row tile are split into,
  int32_t part_chunks; // of so many chunks of 64 keys each
  uint32_t tiles;      // its row tiles (set by the launch); workgroups behind them check offsets
  uint32_t* counts;    // [kKvCounts] parts finished, zero between calls
  // partial outputs, [parts][tokens * heads] rows or, tiled, two tiles per piece
  float* part_o;   // [rows][head_dim]
  float* part_ml;  // [rows][2]: maximum (log2), sum
  KvCut* cuts;     // [kKvPieces], of the tile that a piece ends with
  // of drafted trees: [tokens][mask_words]
  const uint32_t* mask;
  int32_t mask_words;
};

struct KvTreeArgs {
  KvView c;
  const int32_t *parents, *starts;  // starts may be null: the lengths less the tokens
  const int32_t *seqs, *cu;
  int64_t n, tokens;
  int32_t words;
  uint32_t* mask;      // [tokens][words]
  int32_t* positions;  // [tokens]
};

// A sequence that keeps some of its tokens.
struct KvKept {
  int32_t seq;             // -1: nothing changes
  int32_t now;             // its new length
  int32_t begin, end;      // the blocks whose tokens change
  int64_t source, scales;  // where its tokens' sources and its blocks' scales start
};

struct KvKeepArgs {
  KvView c;
  const int32_t *seqs, *last, *index, *cu;
  int64_t n, total;
  KvKept* kept;     // [n]
  // of each token from block `begin` on: where it comes from, the byte of its tile in a
  // block of its page plus its place among the tile's 16 tokens, and that page
  int64_t* source;
  int32_t* pages;
  float* scales;    // [blocks][page_scales]
};

__device__ __forceinline__ void write_source(const KvKeepArgs& a, int64_t at, int32_t page,
                                             int in_page) {
  a.source[at] = page * a.c.page_bytes +
                 (int64_t)(in_page / kKvTile) * (kKvTile * a.c.head_dim) + in_page % kKvTile;
  a.pages[at] = page;
}

struct KvPruneArgs {
  KvKeepArgs k;  // (its lists are not there)
  float* mass;
  int64_t mass_stride, budget, sinks, recent;
};

struct KvWeighArgs {
  KvView c;
  const uint16_t* q;
  const float* lse;  // [tokens][heads]
  float* mass;       // [slots][mass_stride]
  int64_t q_token, q_head, mass_stride;
  const int32_t *seqs, *cu;
  int64_t n, tokens;
  int32_t layer, heads, group;
  int32_t bf16, causal, window;
  float scale_log2;
};

struct QkRotateArgs {
  const uint16_t *q, *k;  // 16-bit elements
  uint16_t *q_out, *k_out;
  int64_t q_token, q_head, k_token, k_head, qo_token, qo_head, ko_token, ko_head;  // strides
  const int32_t* positions;
  const float *inv_freq, *q_weight, *k_weight;  // weights may be null: no norm
  int64_t tokens;
  int32_t heads, kv_heads, rot_dim;
  int32_t bf16, pairs, wide;  // neighbours are paired; 16-byte accesses are aligned
  float eps;
  int32_t steps, parts;  // of rows per wave, of a token (set by the launch)
};

// Whether a grid can be launched: its threads are counted in 32 bits. The launches
// below return hipErrorInvalidConfiguration where it cannot.
inline bool grid_fits(int64_t workgroups, int threads) {
  return workgroups <= (int64_t)(UINT32_MAX / (uint32_t)threads);
}

hipError_t launch_kv_fork(const KvForkArgs& a, hipStream_t st);
hipError_t launch_kv_free(const KvFreeArgs& a, hipStream_t st);
hipError_t launch_kv_reserve(const KvReserveArgs& a, hipStream_t st);
hipError_t launch_kv_compact(const KvCompactArgs& a, hipStream_t st);
hipError_t launch_kv_append(const KvAppendArgs& a, hipStream_t st);
hipError_t launch_qk_rotate(const QkRotateArgs& a, int head_dim, hipStream_t st);
hipError_t launch_kv_attend(const KvAttendArgs& a, hipStream_t st);
hipError_t launch_kv_attend_tree(const KvAttendArgs& a, hipStream_t st);
hipError_t launch_kv_weigh(const KvWeighArgs& a, int64_t max_new, int64_t max_len, hipStream_t st);
bool kv_kept_fits(const KvKeepArgs& a);
hipError_t launch_kv_kept(const KvKeepArgs& a, int64_t tokens, hipStream_t st);
hipError_t launch_kv_prune(const KvPruneArgs& a, hipStream_t st);
hipError_t launch_kv_keep(const KvKeepArgs& a, hipStream_t st);
hipError_t launch_kv_tree(const KvTreeArgs& a, hipStream_t st);

// How an attention call of these sizes is split (its workspace holds the
// parts' partial outputs).
struct KvSplit {
  int tiled, whole, waves, parts, part_chunks;
  int64_t part_rows;  // of partial outputs
};
KvSplit kv_attend_split(int dim, int64_t n, int64_t tokens, int heads, int kv_heads,
                        int64_t max_new, int64_t max_len);

}  // namespace semsched
