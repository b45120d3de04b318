// What the training operators' files share (gfx950): the element types, and the host's checks of device
// arrays.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <type_traits>
#include <utility>
#include <vector>

#include "wn_train.h"
#include "wn.h"
#include "wn_internal.h"

namespace wnt {

typedef unsigned short u16;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf16_val(u16 b) { return __uint_as_float((unsigned)b << 16); }
// Nearest even.
__device__ __forceinline__ u16 bf16_bits(float v) { return __builtin_bit_cast(u16, (__bf16)v); }
__device__ __forceinline__ unsigned bf16_pair(float a, float b) { return (unsigned)bf16_bits(a) | (unsigned)bf16_bits(b) << 16; }

// Elements as the arrays hold them: float, or u16 (bf16 bits).
__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(u16 v) { return bf16_val(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(u16* p, float v) { *p = bf16_bits(v); }

inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }
inline size_t ceil_div(size_t a, size_t b) { return (a + b - 1) / b; }

// A launch takes fewer than 2^32 threads in a dimension: more than 2^20 blocks go on in grid.y (the last ones behind the end).
inline dim3 many_blocks(size_t blocks) {
  const size_t x = std::min<size_t>(blocks, (size_t)1 << 20);
  return dim3((unsigned)x, (unsigned)ceil_div(blocks, x));
}
__device__ __forceinline__ long long block_of_many() { return (long long)blockIdx.y * gridDim.x + blockIdx.x; }

// Makes the device that the call's arrays live on current until the end of the scope.  check() an array before the
// scope is entered: WN_EINVAL for memory that is not on a device (or on another one than the others).
class ArrayScope {
 public:
  ~ArrayScope() {
    if (prev_ >= 0) (void)hipSetDevice(prev_);
  }
  int check(const void* p, const char* name) {
    hipPointerAttribute_t at{};
    const hipError_t e = hipPointerGetAttributes(&at, p);
    if (e != hipSuccess || (at.type != hipMemoryTypeDevice && at.type != hipMemoryTypeManaged)) {
      if (e != hipSuccess) (void)hipGetLastError();
      return fail(name, " is not device memory");
    }
    if (dev_ >= 0 && at.device != dev_) return fail(name, " is on another device");
    dev_ = at.device;
    return WN_OK;
  }
  int enter() {
    int cur = 0;
    if (hipGetDevice(&cur) != hipSuccess) return wn_set_last_error(WN_EHIP, "hipGetDevice failed");
    if (cur != dev_) {
      if (hipSetDevice(dev_) != hipSuccess) return wn_set_last_error(WN_EHIP, "cannot select the arrays' device");
      prev_ = cur;
    }
    return WN_OK;
  }

 private:
  static int fail(const char* name, const char* what) {
    char msg[96];
    std::snprintf(msg, sizeof msg, "%s%s", name, what);
    return wn_set_last_error(WN_EINVAL, msg);
  }
  int dev_ = -1, prev_ = -1;
};

// Whether an output (`out`) of a list of arrays overlaps another one, or an input (`g`) that it is not the whole of: blocks
// would read what others have written.  bytes(array): its size, 0 of one that is not looked at.  Throws std::bad_alloc.
template <class A, class Bytes>
bool overlap(int n, const A* arrays, Bytes bytes) {
  typedef std::pair<uintptr_t, uintptr_t> Span;
  auto span = [&](const A& a, const void* p) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    return Span(at, at + bytes(a));
  };
  std::vector<Span> outs;
  outs.reserve(n);
  for (int k = 0; k < n; ++k)
    if (bytes(arrays[k])) outs.push_back(span(arrays[k], arrays[k].out));
  if (!std::is_sorted(outs.begin(), outs.end())) std::sort(outs.begin(), outs.end());
  for (size_t i = 1; i < outs.size(); ++i)
    if (outs[i].first < outs[i - 1].second) return true;
  for (int k = 0; k < n; ++k) {
    if (!bytes(arrays[k]) || arrays[k].g == arrays[k].out) continue;
    const Span g = span(arrays[k], arrays[k].g);
    const auto after = std::lower_bound(outs.begin(), outs.end(), Span(g.second, 0));
    if (after != outs.begin() && (after - 1)->second > g.first) return true;
  }
  return false;
}

inline int bad_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return WN_OK;
  if (!ws) return wn_set_last_error(WN_EINVAL, "null workspace");
  if (reinterpret_cast<uintptr_t>(ws) % 256 != 0) return wn_set_last_error(WN_EINVAL, "workspace must be 256-byte aligned");
  if (have < need) return wn_set_last_error(WN_EINVAL, "workspace too small");
  return WN_OK;
}

inline int bad_dtype(int dtype) {
  if (dtype == WN_F32 || dtype == WN_BF16) return WN_OK;
  if (dtype == WN_I8) return wn_set_last_error(WN_EUNSUPPORTED, "int8 arrays are not supported here");
  return wn_set_last_error(WN_EINVAL, "unknown dtype");
}

}  // namespace wnt
