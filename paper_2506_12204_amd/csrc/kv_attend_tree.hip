// Attention over the KV cache by the tokens of drafted trees: the launch of the
// kernels that look at masks. The split is that of attention without masks, and so is
// what bounds it: 64 trees of 5 to 24 tokens over 64 to 8192 keys, 32 heads on 8 of 128
// channels, 107 us, the same rows causal 105; 8 trees of 57 to 64 over 8192 to 32768 keys
// 158 us by tiles and 17 for the join of their parts (179 and 18 in the first calls, before
// the clock is up).
#include "kv_attend_kernels.h"

namespace semsched {

hipError_t launch_kv_attend_tree(const KvAttendArgs& a, hipStream_t st) {
  if (a.n == 0) return hipSuccess;  // (without tokens the offsets are looked at)
  switch (a.c.head_dim) {
    case 64: return launch_dim<64, true>(a, st);
    case 128: return launch_dim<128, true>(a, st);
    default: return launch_dim<256, true>(a, st);
  }
}

}  // namespace semsched
