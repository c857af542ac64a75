// Host-side helpers of the C ABI entry points: alignment, overlap and
// workspace checks.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/trevs.h"

namespace trevs {

constexpr size_t kWsAlign = 256;

inline size_t align_up(size_t x) { return (x + kWsAlign - 1) / kWsAlign * kWsAlign; }
inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline bool finite(float x) { return isfinite(x) != 0; }
inline int elem_bytes(int dtype) { return dtype == TREVS_BF16 ? 2 : 4; }

struct Span {
  const void* p;
  size_t n;
};
inline bool overlap(Span a, Span b) {
  if (!a.p || !b.p || a.n == 0 || b.n == 0) return false;
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
  return a0 < b0 + b.n && b0 < a0 + a.n;
}
// Every output span must be disjoint from every input span and from the
// other outputs.
inline bool any_overlap(const Span* out, int n_out, const Span* in, int n_in) {
  for (int i = 0; i < n_out; ++i) {
    for (int j = 0; j < n_in; ++j)
      if (overlap(out[i], in[j])) return true;
    for (int j = i + 1; j < n_out; ++j)
      if (overlap(out[i], out[j])) return true;
  }
  return false;
}

// Workgroups in x of a launch with blocks of up to 256 threads: its threads are counted in 32 bits.
constexpr int64_t kMaxGroups = UINT32_MAX / 256;

inline trevs_status check_ws(void* ws, size_t ws_bytes, size_t need) {
  if (need == 0) return TREVS_OK;
  if (!ws || ws_bytes < need || !aligned(ws, kWsAlign)) return TREVS_ERR_WORKSPACE;
  return TREVS_OK;
}

}  // namespace trevs

#define TREVS_TRY(x)                            \
  do {                                          \
    const trevs_status st_ = (x);               \
    if (st_ != TREVS_OK) return st_;            \
  } while (0)
#define TREVS_HIP(x)                                   \
  do {                                                 \
    if ((x) != hipSuccess) return TREVS_ERR_HIP;       \
  } while (0)
