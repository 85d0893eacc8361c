// Trees of drafted tokens, from their parents: for every token the mask of the
// tokens that it continues (itself among them) and its position.
//
//   mask[t] = mask[parent[t]] | bit t,  position[t] = start + depth of t
//
// One workgroup per sequence, a thread per token, which walks to the root: parents
// come before their children, so the words of a mask are written once each, from the
// last to the first. The parents lie in LDS, so a step of the walk is one LDS read.
// Bound by the launch and the chain from the sequence to its parents: 2.6 us for one tree
// of 13 tokens, 5 us for 64 of up to 24 or 8 of up to 64.
#include "device_common.h"
#include "kv.h"

namespace semsched {

namespace {

constexpr int TT = 256;

__global__ __launch_bounds__(TT) void kv_tree(KvTreeArgs a) {
  __shared__ int32_t parent[32 * kKvMaskWords];
  const KvView& c = a.c;
  const int64_t i = blockIdx.x;
  auto wrong = [&] { atomicOr(c.flags, kFlagInval); };
  if (a.cu && i == 0 && threadIdx.x == 0 && (a.cu[0] != 0 || a.cu[a.n] != a.tokens)) wrong();
  const int64_t row0 = a.cu ? a.cu[i] : i;
  const int64_t fresh = a.cu ? (int64_t)a.cu[i + 1] - row0 : 1;
  if (fresh < 0 || row0 < 0 || row0 + fresh > a.tokens) {
    if (threadIdx.x == 0) wrong();
    return;
  }
  const int32_t s = a.seqs[i];
  const bool known = (uint32_t)s < (uint32_t)c.slots;
  const int64_t len = known ? c.lens[s] : -1;
  if (threadIdx.x == 0 && (len < 0 || len > ((int64_t)c.max_blocks << c.page_shift))) wrong();
  const uint32_t start = a.starts ? (uint32_t)a.starts[i] : (uint32_t)(len - fresh);
  const int words = a.words;
  const int n = (int)min(fresh, (int64_t)32 * words);
  if (fresh > n) {  // tokens without a bit of their own: they see the context alone
    if (threadIdx.x == 0) wrong();
    for (int64_t t = n + threadIdx.x; t < fresh; t += TT) {
      for (int w = 0; w < words; ++w) a.mask[(row0 + t) * words + w] = 0;
      a.positions[row0 + t] = (int32_t)start;
    }
  }
  for (int t = threadIdx.x; t < n; t += TT) {
    int32_t p = a.parents[row0 + t];
    if (p < -1 || p >= t) {  // parents come first
      wrong();
      p = -1;
    }
    parent[t] = p;
  }
  block_sync();
  for (int t = threadIdx.x; t < n; t += TT) {
    uint32_t* row = a.mask + (row0 + t) * words;
    int depth = 0, w = words - 1;
    uint32_t bits = 0;
    for (int p = t; p >= 0; p = parent[p], ++depth) {
      for (; w > p >> 5; --w) {
        row[w] = bits;
        bits = 0;
      }
      bits |= 1u << (p & 31);
    }
    for (; w >= 0; --w) {
      row[w] = bits;
      bits = 0;
    }
    a.positions[row0 + t] = (int32_t)(start + (uint32_t)depth - 1u);
  }
}

}  // namespace

hipError_t launch_kv_tree(const KvTreeArgs& a, hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  if (!grid_fits(a.n, TT)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(kv_tree, dim3((unsigned)a.n), dim3(TT), 0, st, a);
  return hipGetLastError();
}

}  // namespace semsched
