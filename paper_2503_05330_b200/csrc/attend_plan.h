// Attention: which CTAs left parts of an item, as the launch that joins them reads it.  Plain arithmetic, host and device.
#pragma once

#ifndef SDMS_HD
#ifdef __CUDACC__
#define SDMS_HD __host__ __device__ __forceinline__
#else
#define SDMS_HD inline
#endif
#endif

namespace sdms {

constexpr int kCtas = 148;               // of attend_kernel: one per SM

// An item's parts come from CTAs first .. first + count - 1.  What the workspace says is not taken on trust: where a wait ran out, the item's CTAs may have left
// nothing there, and it holds what it held before the call.  Then there are no parts.
struct PartRun { int first, count; };
SDMS_HD PartRun part_run(int first, int last) {
  const bool good = first >= 0 && first <= last && last < kCtas;
  return PartRun{good ? first : 0, good ? last - first + 1 : 0};
}

}  // namespace sdms
