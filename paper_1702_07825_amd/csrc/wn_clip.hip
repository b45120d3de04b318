// The norm over many gradient arrays and their clip (gfx950).  Declarations and contracts are in
// include/wn_train.h.
//
// Two passes over the arrays: sums of squares per block, then every block joins the blocks' sums in the same
// order and scales its share.  The arrays go to the kernels as arguments (kArrays of them a launch), cut
// into chunks of equal length that the blocks take in turn, so that one launch serves arrays of any
// sizes.  Squares are summed in fp64: a chunk's sum of fp32 squares would overflow from gradients of 1e19 on
// and vanish below 1e-23.
//
// Bound: two reads and a write of the arrays (a second read of what does not stay in the caches).  Measured: 0.91 GB in
// 295 arrays, squares 167 us (5.4 TB/s), scaling 349 us (5.2 TB/s); 3.6 MB in 127 arrays 6.5 us each.
#include "wn_arrays.h"

#include "wn_wave.h"

#include <cmath>
#include <new>
#include <utility>
#include <vector>

namespace {

using namespace wnt;

constexpr int kArrays = 168;   // arrays of a launch: the arguments stay under 4 KB
constexpr int kThreads = 256;
// Elements of a chunk: long ones keep more loads in flight, short ones spread small models over the chip.  Both passes in us,
// short and long, 127 arrays of 2^20 fp32 elements in all 10.2 and 10.4 (bf16 9.4, 10.7), of 2^22 21.6 and 14.4 (18.7, 12.4),
// of 2^26 138 and 132 (81, 70); 16 arrays 9.4 and 11.2 (8.6, 10.4), 12.7 and 13.6 (11.6, 10.7), 125 and 125 (74, 67).
constexpr int kLong = 16384, kShort = 4096;
constexpr long long kShortUpTo = 1LL << 21;
constexpr int kSlots = 1024;   // blocks of a launch, partial sums

struct Arrays {
  const void* g[kArrays];
  void* out[kArrays];
  unsigned first[kArrays + 1];         // chunks before the array
  unsigned short last[kArrays];        // elements of its last chunk; | kBf16
  int count, elems;
};
constexpr unsigned short kBf16 = 0x8000;
static_assert(sizeof(Arrays) < 3900 && kLong < kBf16, "kernel arguments");

// Four words at any element's alignment.
typedef unsigned u32x4u __attribute__((ext_vector_type(4), aligned(2)));

// The array that a chunk lies in: the last one whose first chunk is at most the chunk.
__device__ __forceinline__ int array_of(const Arrays& a, unsigned chunk) {
  int lo = 0, hi = a.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.first[mid] <= chunk) lo = mid;
    else hi = mid;
  }
  return lo;
}

// The chunks of block b: b, b + grid, .., the same in both passes, so that the blocks in flight read one moving window of
// memory; f(array, first element, elements) for each, in order or (`back`) from the last.
template <class F>
__device__ __forceinline__ void for_share(const Arrays& a, bool back, F f) {
  const long long all = a.first[a.count], grid = gridDim.x, last = all - 1 - blockIdx.x;
  if (last < 0) return;
  int k = array_of(a, (unsigned)(blockIdx.x + (back ? last / grid * grid : 0)));
  for (long long i = 0; i <= last / grid; ++i) {
    const unsigned c = (unsigned)(blockIdx.x + (back ? last / grid - i : i) * grid);
    // (an array has a chunk at least, and a block's chunks come in order: at most a step for each array in all)
    if (back)
      while (a.first[k] > c) --k;
    else
      while (a.first[k + 1] <= c) ++k;
    f(k, (long long)(c - a.first[k]) * a.elems, c + 1 == a.first[k + 1] ? a.last[k] & (kBf16 - 1) : a.elems);
  }
}

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double s[kThreads / 64];
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, 64);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s[0];
  for (int w = 1; w < kThreads / 64; ++w) v += s[w];
  __syncthreads();
  return v;
}

__device__ __forceinline__ double squares(u32x4 w, bool bf16) {
  double v = 0.0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (bf16) {
      const double a = __uint_as_float(w[e] << 16), b = __uint_as_float(w[e] & 0xffff0000u);
      v += a * a + b * b;
    } else {
      const double a = __uint_as_float(w[e]);
      v += a * a;
    }
  }
  return v;
}

constexpr int kUnroll = 8;  // 16-byte loads in flight per thread

// slot[b] (+)= the squares of block b's share
__global__ __launch_bounds__(kThreads) void clip_squares(const Arrays a, double* slot, int add) {
  double sum[4] = {0.0, 0.0, 0.0, 0.0};
  for_share(a, false, [&](int k, long long at, int n) {
    const bool bf = a.last[k] & kBf16;
    const int per = bf ? 8 : 4;
    const char* p = static_cast<const char*>(a.g[k]) + at * (bf ? 2 : 4);
    const int whole = n / per;
    int i = threadIdx.x;
    for (; i + (kUnroll - 1) * kThreads < whole; i += kUnroll * kThreads) {
      u32x4u w[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) w[u] = *reinterpret_cast<const u32x4u*>(p + 16 * (i + u * kThreads));
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) sum[u & 3] += squares(u32x4{w[u][0], w[u][1], w[u][2], w[u][3]}, bf);
    }
    for (; i < whole; i += kThreads) {
      const u32x4u w = *reinterpret_cast<const u32x4u*>(p + 16 * i);
      sum[0] += squares(u32x4{w[0], w[1], w[2], w[3]}, bf);
    }
    const int rest = whole * per + threadIdx.x;
    if (rest < n) {
      const double v = bf ? bf16_val(reinterpret_cast<const u16*>(p)[rest]) : reinterpret_cast<const float*>(p)[rest];
      sum[0] += v * v;
    }
  });
  const double v = block_sum((sum[0] + sum[1]) + (sum[2] + sum[3]));
  if (threadIdx.x == 0) slot[blockIdx.x] = add ? slot[blockIdx.x] + v : v;
}

// The factor max_norm / norm as f 2^k: k is 0 unless fp32 would hold the factor in fewer bits (below its smallest normal value,
// for norms near its largest) or not at all.
struct Factor {
  float f;
  int k;
  __device__ __forceinline__ float operator()(float v) const { return k ? ldexpf(v * f, k) : v * f; }
};
__device__ __forceinline__ Factor factor_of(double r) {
  const int k = r > 0.0 && r < 0x1p-126 ? ilogb(r) + 1 : 0;  // f in [1/2, 1): no product overflows
  return {(float)ldexp(r, -k), k};
}

__device__ __forceinline__ u32x4u times(u32x4u w, Factor f, bool bf) {
  u32x4u r;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    r[e] = bf ? bf16_pair(f(__uint_as_float(w[e] << 16)), f(__uint_as_float(w[e] & 0xffff0000u)))
              : __float_as_uint(f(__uint_as_float(w[e])));
  return r;
}

// The chunks from the last: what the first pass read last is still in the caches, and the stores go past them.
__global__ __launch_bounds__(kThreads) void clip_scale(const Arrays a, const double* slot, int slots, float max_norm, float* norm_out,
                                                       int first) {
  double sum = 0.0;
  for (int i = threadIdx.x; i < slots; i += kThreads) sum += slot[i];
  const double wide = sqrt(block_sum(sum));
  const float norm = (float)wide;
  if (first && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
  // (max_norm = 0: 0 times each element)
  const bool scaled = norm > max_norm && norm < INFINITY;
  const Factor f = factor_of(scaled ? max_norm / wide : 1.0);
  for_share(a, true, [&](int k, long long at, int n) {
    if (!scaled && a.out[k] == a.g[k]) return;
    const bool bf = a.last[k] & kBf16;
    const int per = bf ? 8 : 4;
    const char* p = static_cast<const char*>(a.g[k]) + at * (bf ? 2 : 4);
    char* o = static_cast<char*>(a.out[k]) + at * (bf ? 2 : 4);
    const int whole = n / per, steps = whole / (kUnroll * kThreads);
    for (int i = whole - 1 - (int)threadIdx.x; i >= steps * kUnroll * kThreads; i -= kThreads) {
      const u32x4u w = *reinterpret_cast<const u32x4u*>(p + 16 * i);
      __builtin_nontemporal_store(scaled ? times(w, f, bf) : w, reinterpret_cast<u32x4u*>(o + 16 * i));
    }
    for (int s = steps - 1; s >= 0; --s) {
      const int i = s * kUnroll * kThreads + threadIdx.x;
      u32x4u w[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) w[u] = *reinterpret_cast<const u32x4u*>(p + 16 * (i + u * kThreads));
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) 
        __builtin_nontemporal_store(scaled ? times(w[u], f, bf) : w[u], reinterpret_cast<u32x4u*>(o + 16 * (i + u * kThreads)));
    }
    const int rest = whole * per + threadIdx.x;
    if (rest < n) {
      if (bf) {
        const u16 v = reinterpret_cast<const u16*>(p)[rest];
        reinterpret_cast<u16*>(o)[rest] = scaled ? bf16_bits(f(bf16_val(v))) : v;
      } else {
        const float v = reinterpret_cast<const float*>(p)[rest];
        reinterpret_cast<float*>(o)[rest] = scaled ? f(v) : v;
      }
    }
  });
}

// Whether an output overlaps another one, or an input that it is not the whole of: blocks would read what others have
// scaled.  Throws std::bad_alloc.
bool overlap(int n, const wn_clip_array* arrays) {
  typedef std::pair<uintptr_t, uintptr_t> Span;
  auto span = [](const wn_clip_array& a, const void* p) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    return Span(at, at + (uintptr_t)a.n * (a.dtype == WN_BF16 ? 2 : 4));
  };
  std::vector<Span> outs;
  outs.reserve(n);
  for (int k = 0; k < n; ++k)
    if (arrays[k].n) outs.push_back(span(arrays[k], arrays[k].out));
  if (!std::is_sorted(outs.begin(), outs.end())) std::sort(outs.begin(), outs.end());
  for (size_t i = 1; i < outs.size(); ++i)
    if (outs[i].first < outs[i - 1].second) return true;
  for (int k = 0; k < n; ++k) {
    if (!arrays[k].n || arrays[k].g == arrays[k].out) continue;
    const Span g = span(arrays[k], arrays[k].g);
    const auto after = std::lower_bound(outs.begin(), outs.end(), Span(g.second, 0));
    if (after != outs.begin() && (after - 1)->second > g.first) return true;
  }
  return false;
}

}  // namespace

extern "C" {

size_t wn_clip_workspace_bytes(void) { return kSlots * sizeof(double); }

int wn_clip(int32_t n_arrays, const wn_clip_array* arrays, float max_norm, float* norm, void* workspace, size_t ws_bytes,
            void* stream) {
  wn_clear_last_error();
  if (n_arrays < 0 || n_arrays > 1 << 20) return wn_set_last_error(WN_EINVAL, "n_arrays must be 0..2^20");
  if ((n_arrays && !arrays) || !norm) return wn_set_last_error(WN_EINVAL, "null pointer");
  if (!(max_norm >= 0.f)) return wn_set_last_error(WN_EINVAL, "max_norm must be >= 0");
  long long all = 0;
  for (int k = 0; k < n_arrays; ++k) {
    const wn_clip_array& a = arrays[k];
    const int rc = bad_dtype(a.dtype);
    if (rc != WN_OK) return rc;
    if (a.n < 0 || a.n > 1LL << 40) return wn_set_last_error(WN_EINVAL, "an array's n must be 0..2^40");
    if (a.n && (!a.g || !a.out)) return wn_set_last_error(WN_EINVAL, "null pointer");
    const uintptr_t size = a.dtype == WN_BF16 ? 2 : 4;
    if (a.n && (reinterpret_cast<uintptr_t>(a.g) % size || reinterpret_cast<uintptr_t>(a.out) % size))
      return wn_set_last_error(WN_EINVAL, "an array is not aligned to its elements");
    all += a.n;
    if (all > 1LL << 44) return wn_set_last_error(WN_EINVAL, "too many elements");
  }
  try {
    if (overlap(n_arrays, arrays)) return wn_set_last_error(WN_EINVAL, "arrays overlap");
  } catch (const std::bad_alloc&) {
    return wn_set_last_error(WN_ENOMEM, "out of host memory");
  }
  const int elems = all <= kShortUpTo ? kShort : kLong;
  int rc = bad_workspace(workspace, ws_bytes, wn_clip_workspace_bytes());
  if (rc != WN_OK) return rc;
  ArrayScope scope;
  if ((rc = scope.check(norm, "norm")) != WN_OK || (rc = scope.check(workspace, "workspace")) != WN_OK) return rc;
  // (the first array stands for all: asking for each took longer than the clip of a model's hundred gradients)
  for (int k = 0; k < n_arrays; ++k)
    if (arrays[k].n) {
      if ((rc = scope.check(arrays[k].g, "g")) != WN_OK || (rc = scope.check(arrays[k].out, "out")) != WN_OK) return rc;
      break;
    }
  if ((rc = scope.enter()) != WN_OK) return rc;
  double* const slot = static_cast<double*>(workspace);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const unsigned grid = (unsigned)std::max<size_t>(1, std::min<size_t>(kSlots, ceil_div((size_t)all, elems) + n_arrays));
  for (int pass = 0; pass < 2; ++pass) {
    int k = 0;
    bool first = true;
    do {
      Arrays a{};
      a.elems = elems;
      for (; k < n_arrays && a.count < kArrays; ++k) {
        if (!arrays[k].n) continue;
        const int i = a.count++;
        a.g[i] = arrays[k].g;
        a.out[i] = arrays[k].out;
        a.last[i] = (unsigned short)((arrays[k].n - 1) % elems + 1) | (arrays[k].dtype == WN_BF16 ? kBf16 : 0);
        a.first[i + 1] = a.first[i] + (unsigned)ceil_div((size_t)arrays[k].n, elems);
      }
      if (pass == 0) hipLaunchKernelGGL(clip_squares, dim3(grid), dim3(kThreads), 0, st, a, slot, !first);
      else hipLaunchKernelGGL(clip_scale, dim3(grid), dim3(kThreads), 0, st, a, slot, (int)grid, max_norm, norm, (int)first);
      first = false;
    } while (k < n_arrays);
  }
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? WN_OK : wn_set_last_error(WN_EHIP, hipGetErrorString(e));
}

}  // extern "C"
