// Attention over the KV cache by rows at the last positions of their sequences:
// the kernels' launch, and the rule which of them.
#include "kv_attend_kernels.h"

#include <algorithm>
#include <cstdlib>

namespace semsched {

// Which kernel, and how many parts of the key axis. Rules measured on MI355X:
//   * The kernel of few rows takes cost_few ns of the whole device per tile of 16
//     rows and chunk of 64 keys, the tile kernel cost_tile ns per tile and 32 keys
//     (256 rows, 128 for 256 channels), and 20 us more for its longer start and
//     end: 16 sequences of 128 rows over 4096 keys (8 KV heads, 128 channels) take
//     78 us with the one and 105 us with the other, of 256 rows 139 and 97 us.
//   * Few rows: parts only where there are fewer workgroups than compute units,
//     then as many as those; each is eight waves with long runs of keys (four
//     contexts of 131072 tokens take 175 us with 256 workgroups, 187 us with 768),
//     and not for fewer than 24 chunks (a single token over 1024 keys takes 10 us
//     in one part; two add 3 us of joining). With more workgroups than compute
//     units four waves each, without parts (256 ragged requests: 87 us, 95 us with
//     parts of 2048 keys). Equal contexts of 32768 keys, 8 KV heads, are read at
//     5.3 to 5.7 TB/s (8 to 17 sequences), 6.0 (24 to 32, 64) and 5.0 (40, a second
//     round that does not fill the device). Unequal ones are not balanced: 31
//     sequences of 1024 keys and one of 131072 take 942 us, as long as eight
//     workgroups need for the long one, where the bytes take 60.
//   * Tiles: see kPieces.
KvSplit kv_attend_split(int dim, int64_t n, int64_t tokens, int heads, int kv_heads,
                        int64_t max_new, int64_t max_len) {
  KvSplit s = {};
  const int group = heads / kv_heads;
  const int64_t chunks = std::max<int64_t>((max_len + kChunk - 1) / kChunk, 1);
  // row tiles of the grid, and what there are of them if max_new holds
  auto grid_of = [&](int64_t rows) { return tokens * group / rows + n; };
  auto tiles_of = [&](int64_t rows) {
    return std::min(grid_of(rows), n * ((max_new * group + rows - 1) / rows));
  };
  const int tile = dim == 256 ? tile_rows<256>() : tile_rows<128>();
  const double cost_few = dim == 64 ? 0.7 : dim == 128 ? 1.0 : 2.8;
  const double cost_tile = dim == 64 ? 3.7 : dim == 128 ? 4.6 : 5.4;
  const double each = (double)kv_heads * (double)chunks;
  s.tiled = cost_tile * 2 * each * (double)tiles_of(tile) + 20e3 <
            cost_few * each * (double)tiles_of(kRows);
  // SEMSCHED_KV_TILES=0 or 1 takes one kernel for all sizes, so that both stay
  // testable on small ones.
  const char* forced = std::getenv("SEMSCHED_KV_TILES");
  if (forced && (forced[0] == '0' || forced[0] == '1')) s.tiled = forced[0] == '1';
  if (s.tiled) {
    s.whole = tokens * group / tile * kv_heads >= kWholeRounds * kPieces;
    if (!s.whole) s.part_rows = 2 * kPieces * tile;
    return s;
  }
  const int64_t groups = std::max<int64_t>(tiles_of(kRows) * kv_heads, 1);
  s.waves = groups < 256 && dim <= 128 ? 8 : 4;
  const int64_t least = 2 * s.waves;  // chunks of a part
  // (a tile with parts needs a counter)
  const int64_t want = chunks <= 3 * s.waves || grid_of(kRows) * kv_heads > kKvCounts ? 1 : 256;
  const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(want / groups, kMostParts));
  s.part_chunks = (int)std::max<int64_t>(least, (chunks + parts - 1) / parts);
  s.parts = (int)((chunks + s.part_chunks - 1) / s.part_chunks);
  if (s.parts > 1) s.part_rows = s.parts * tokens * heads;
  return s;
}

hipError_t launch_kv_attend(const KvAttendArgs& a, hipStream_t st) {
  if (a.n == 0) return hipSuccess;  // (without tokens the offsets are looked at)
  switch (a.c.head_dim) {
    case 64: return launch_dim<64, false>(a, st);
    case 128: return launch_dim<128, false>(a, st);
    default: return launch_dim<256, false>(a, st);
  }
}

}  // namespace semsched
