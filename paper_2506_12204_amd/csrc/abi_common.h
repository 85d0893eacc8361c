// What the C ABI's translation units share: the state of the blocking calls
// (abi.hip owns it) and the workspace conventions.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>

#include <mutex>

namespace semsched {

constexpr size_t kAlign = 256;
constexpr size_t kHeaderBytes = 256;  // flags, counters, ranges, plan

inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

// Held by a blocking call from taking the workspace to reading its status.
std::mutex& blocking_mutex();
hipStream_t blocking_stream();
// The library's workspace of the current device, of at least `bytes`.
int blocking_workspace(size_t bytes, void** out);
// Waits for the stream and maps the error bits of the workspace's first word.
int blocking_finish(void* ws, hipStream_t st);

}  // namespace semsched
