// api_common.hpp -- host helpers shared by the entry points: error returns,
// address ranges and the device scope of a call.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <vector>

#include "tlc.h"
#include "tlc_internal.h"

#define TLC_API extern "C" __attribute__((visibility("default")))

namespace tlc {

// Also takes the error off the calling thread, where hipGetLastError() after
// the next launch, of any context or library, would find it again.
inline int hip_fail(hipError_t e, const char* what) {
  (void)hipGetLastError();
  return fail(TLC_E_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

inline size_t ceil_div(size_t a, size_t b) { return (a + b - 1) / b; }

inline bool overlap(const void* a, size_t an, const void* b, size_t bn) {
  const uintptr_t pa = (uintptr_t)a, pb = (uintptr_t)b;
  return an && bn && pa < pb + bn && pb < pa + an;
}

// A device address range of one call's arguments; `written` ranges must
// not overlap any other range of the call.
struct Span {
  uintptr_t lo, hi;
  bool written;
};

// Sorts the spans by start address and reports whether a written span
// overlaps another span (read-only spans may overlap each other: one stream
// decoded into several outputs, one tensor read twice).  In start order a
// span overlaps an earlier one exactly when it starts below that one's end,
// so it suffices to keep the largest end of all earlier spans and of the
// earlier written ones.  std::sort works in place: nothing is allocated.
inline bool spans_conflict(std::vector<Span>& v) {
  std::sort(v.begin(), v.end(), [](const Span& a, const Span& b) { return a.lo < b.lo; });
  uintptr_t end_all = 0, end_written = 0;
  for (const Span& sp : v) {
    if (sp.lo < (sp.written ? end_all : end_written)) return true;
    end_all = std::max(end_all, sp.hi);
    if (sp.written) end_written = std::max(end_written, sp.hi);
  }
  return false;
}

// spans_conflict for a call whose spans may repeat the previous call's
// (`last`: the spans of the last call that passed, in call order).  A
// training loop passes the same buffers every step: the list then equals
// `last`, which was checked already, and the sort is skipped.  `last`
// has the capacity of `v`, so nothing is allocated.
inline bool spans_conflict_cached(std::vector<Span>& v, std::vector<Span>& last) {
  if (v.size() == last.size() &&
      std::equal(v.begin(), v.end(), last.begin(), [](const Span& a, const Span& b) {
        return a.lo == b.lo && a.hi == b.hi && a.written == b.written;
      }))
    return false;
  last = v;
  if (!spans_conflict(v)) return false;
  last.clear();
  return true;
}

inline void add_span(std::vector<Span>& v, const void* p, size_t bytes, bool written) {
  if (bytes) v.push_back(Span{(uintptr_t)p, (uintptr_t)p + bytes, written});
}

// Makes the context's device current for one entry point and restores the
// caller's device when the entry point returns.
class DeviceScope {
 public:
  explicit DeviceScope(int dev) {
    err_ = hipGetDevice(&prev_);
    if (err_ == hipSuccess && prev_ != dev) {
      err_ = hipSetDevice(dev);
      switched_ = err_ == hipSuccess;
    }
  }
  ~DeviceScope() {
    if (switched_) (void)hipSetDevice(prev_);
  }
  DeviceScope(const DeviceScope&) = delete;
  DeviceScope& operator=(const DeviceScope&) = delete;
  int status() const { return err_ == hipSuccess ? TLC_OK : hip_fail(err_, "hipSetDevice"); }

 private:
  int prev_ = -1;
  bool switched_ = false;
  hipError_t err_ = hipSuccess;
};

}  // namespace tlc
