// Attention over the KV cache by the tokens of drafted trees: the launch of the
// kernels that look at masks.
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
