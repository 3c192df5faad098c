// Host helpers shared by libasv's translation units.
#pragma once

#include <hip/hip_runtime.h>

#include <stddef.h>
#include <stdint.h>

namespace asv {

// Keep the text of a failure for asv_last_error.
void set_error(const char* what, hipError_t e);

// ASV_OK when the launches enqueued so far succeeded, else ASV_EHIP with the error recorded.
int launch_status(const char* what);

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// A launch along x holds fewer than 2^32 threads; beyond, workgroups are dropped without an error.
inline bool launch_fits(int64_t workgroups, int threads) {
  return workgroups >= 0 && workgroups * threads < (int64_t)1 << 32;
}

// Compute units of the current device, queried once per device.
int cu_count();

}  // namespace asv
