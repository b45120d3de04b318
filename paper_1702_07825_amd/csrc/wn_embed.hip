// An embedding and its gradient by sorted tokens (gfx950).  Declarations and contracts are in
// include/wn_train.h.
//
// The gradient's rows are sums over the rows of dout that share a token.  Atomic adds would make the sums
// depend on their order and serialise where a token is common (silence is a fifth of a voice's samples), so
// the tokens are sorted first, stably, and the sorted rows cut into chunks of equal length: a
// chunk sums each run of equal tokens in it; runs that lie within a chunk are done, the others leave a
// partial sum per chunk, which the last kernel joins in order.
//
// Bound: reading dout and writing the table.  Measured: 512000 rows of 64 fp32 into 256 (131 MB, runs of up to 100,000
// rows): sort 28 us, sums 26, join 21 (one block a run: 78 where all rows have one token); 8191 bf16 rows of 2048 into 65536 (302 MB): the sort beside the table's zeros 44 us
// (6.1 TB/s), sums 23, join 8.  The lookups 25 us (5.2 TB/s) and 16 us.
#include "wn_arrays.h"

#include "wn_wave.h"

#include <cmath>

namespace {

using namespace wnt;

constexpr int kMaxN = 1 << 27, kMaxD = 1 << 16, kMaxV = 1 << 24;

// W elements in one access, at any element's alignment.
template <class E, int W>
struct Vec {
  typedef E type __attribute__((ext_vector_type(W), aligned(sizeof(E))));
};
template <class E, int W>
__device__ __forceinline__ void load(const E* p, float (&v)[W]) {
  if constexpr (W == 1) {
    v[0] = value(*p);
  } else {
    const typename Vec<E, W>::type x = *reinterpret_cast<const typename Vec<E, W>::type*>(p);
#pragma unroll
    for (int e = 0; e < W; ++e) v[e] = value((E)x[e]);
  }
}
template <class E, int W>
__device__ __forceinline__ void store(E* p, const float (&v)[W]) {
  if constexpr (W == 1) {
    put(p, v[0]);
  } else {
    typename Vec<E, W>::type x;
#pragma unroll
    for (int e = 0; e < W; ++e) {
      E t;
      put(&t, v[e]);
      x[e] = t;
    }
    *reinterpret_cast<typename Vec<E, W>::type*>(p) = x;
  }
}

// W elements of which `left` exist (the rest read as 0, and are not stored).
template <class E, int W>
__device__ __forceinline__ void piece(const E* p, int left, float (&v)[W]) {
  if (left >= W) {
    load<E, W>(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < W; ++e) v[e] = e < left ? value(p[e]) : 0.f;
  }
}
template <class E, int W>
__device__ __forceinline__ void put_piece(E* p, int left, const float (&v)[W]) {
  if (left >= W) {
    store<E, W>(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < W; ++e)
      if (e < left) put(p + e, v[e]);
  }
}

// G lanes take a row, W elements each in turn; 256 / G rows a block.
template <class E, int W>
__global__ __launch_bounds__(256) void embed_rows(const E* table, const int32_t* t, int N, int D, int V, float scale, E* out, int G) {
  const int lane = threadIdx.x & (G - 1);
  const long long n = block_of_many() * (256 / G) + threadIdx.x / G;
  if (n >= N) return;
  const int v = t[n];
  const bool ok = v >= 0 && v < V;
  const E* src = table + (size_t)(ok ? v : 0) * D;
  E* dst = out + (size_t)n * D;
  const int whole = D / W * W;
  for (int k = lane * W; k < whole; k += G * W) {
    float x[W];
    load<E, W>(src + k, x);
#pragma unroll
    for (int e = 0; e < W; ++e) x[e] = ok ? x[e] * scale : 0.f;
    store<E, W>(dst + k, x);
  }
  for (int k = whole + lane; k < D; k += G) put(dst + k, ok ? value(src[k]) * scale : 0.f);
}

// ------------------------------------------------------------------------------------------------
// The sort: by digits of up to 9 bits, from the lowest, each pass stable.  Tokens outside the table sort
// last, as V.
// ------------------------------------------------------------------------------------------------
constexpr int kDigits = 512;

__device__ __forceinline__ unsigned key_of(int t, int V) { return t >= 0 && t < V ? (unsigned)t : (unsigned)V; }

// The lanes below this one whose digit is the same, and whether none above has it; `on`: this lane has an element.
__device__ __forceinline__ void match(unsigned digit, int bits, bool on, int lane, int& below, bool& last, int& all) {
  unsigned long long m = __ballot(on);
  for (int b = 0; b < bits; ++b) {
    const bool bit = digit >> b & 1;
    const unsigned long long k = __ballot(bit);
    m &= bit ? k : ~k;
  }
  below = __popcll(m & ((1ull << lane) - 1));
  all = __popcll(m);
  last = below == all - 1;
}

struct Digit {
  int shift, bits;
};

// count[digit][unit]: a unit is a wave with its run of `per` elements (a multiple of 64).
// Zeros to the gradient's table, by the sort's first launch beside it: most rows of a large table have no token, and
// finding them first would put this write behind the sort.
__device__ __forceinline__ void zero_table(char* out, size_t bytes, int block, int blocks) {
  // (bytes is a multiple of 2 and so is the address: whole 16-byte pieces, then 2-byte ones)
  typedef unsigned u32x4u __attribute__((ext_vector_type(4), aligned(2)));
  const size_t whole = bytes / 16, step = (size_t)blocks * blockDim.x;
  for (size_t i = (size_t)block * blockDim.x + threadIdx.x; i < whole; i += step)
    *reinterpret_cast<u32x4u*>(out + 16 * i) = u32x4u{0u, 0u, 0u, 0u};
  if (block == 0 && threadIdx.x < (bytes & 15) / 2) reinterpret_cast<u16*>(out + 16 * whole)[threadIdx.x] = 0;
}
__global__ __launch_bounds__(256) void sort_count(const int32_t* t, const unsigned* key, int N, int V, Digit d, int per, int units,
                                                  unsigned* count, int blocks, char* table, size_t bytes) {
  if ((int)blockIdx.x >= blocks) {
    zero_table(table, bytes, blockIdx.x - blocks, gridDim.x - blocks);
    return;
  }
  __shared__ unsigned s[4][kDigits];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, unit = blockIdx.x * 4 + w;
  for (int i = lane; i < kDigits; i += 64) s[w][i] = 0;
  __syncthreads();
  const long long at = (long long)unit * per;
  for (int i = 0; i < per; i += 64) {
    const long long k = at + i + lane;
    const bool on = k < N;
    const unsigned x = on ? (key ? key[k] : key_of(t[k], V)) : 0;
    if (on) atomicAdd(&s[w][x >> d.shift & ((1 << d.bits) - 1)], 1u);  // (counts: the order does not matter)
  }
  __syncthreads();
  if (unit < units)
    for (int i = lane; i < 1 << d.bits; i += 64) count[(size_t)i * units + unit] = s[w][i];
}

// A digit's counts to the counts before each unit, and their total; a block per digit.
__global__ __launch_bounds__(256) void sort_scan(unsigned* count, int units, unsigned* total) {
  __shared__ unsigned s[256];
  unsigned* c = count + (size_t)blockIdx.x * units;
  const int per = (units + 255) / 256, b = threadIdx.x * per, e = min(units, b + per);
  unsigned sum = 0;
  for (int i = b; i < e; ++i) sum += c[i];
  s[threadIdx.x] = sum;
  __syncthreads();
  for (int d = 1; d < 256; d <<= 1) {
    const unsigned v = threadIdx.x >= d ? s[threadIdx.x - d] : 0;
    __syncthreads();
    s[threadIdx.x] += v;
    __syncthreads();
  }
  unsigned before = s[threadIdx.x] - sum;
  for (int i = b; i < e; ++i) {
    const unsigned v = c[i];
    c[i] = before;
    before += v;
  }
  if (threadIdx.x == 255) total[blockIdx.x] = s[255];
}

__global__ __launch_bounds__(256) void sort_scatter(const int32_t* t, const unsigned* key, const unsigned* row, int N, int V, Digit d,
                                                    int per, int units, const unsigned* count, const unsigned* total,
                                                    unsigned* key_out, unsigned* row_out) {
  __shared__ unsigned s[4][kDigits];
  __shared__ unsigned base[kDigits], part[256];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, unit = blockIdx.x * 4 + w;
  // the digits' first places: two digits a thread
  const unsigned t0 = 2 * threadIdx.x < 1 << d.bits ? total[2 * threadIdx.x] : 0;
  const unsigned t1 = 2 * threadIdx.x + 1 < 1 << d.bits ? total[2 * threadIdx.x + 1] : 0;
  part[threadIdx.x] = t0 + t1;
  __syncthreads();
  for (int k = 1; k < 256; k <<= 1) {
    const unsigned v = threadIdx.x >= k ? part[threadIdx.x - k] : 0;
    __syncthreads();
    part[threadIdx.x] += v;
    __syncthreads();
  }
  base[2 * threadIdx.x] = part[threadIdx.x] - t0 - t1;
  base[2 * threadIdx.x + 1] = part[threadIdx.x] - t1;
  __syncthreads();
  if (unit >= units) return;
  for (int i = lane; i < 1 << d.bits; i += 64) s[w][i] = base[i] + count[(size_t)i * units + unit];
  __builtin_amdgcn_wave_barrier();
  const long long at = (long long)unit * per;
  for (int i = 0; i < per; i += 64) {
    const long long k = at + i + lane;
    const bool on = k < N;
    const unsigned x = on ? (key ? key[k] : key_of(t[k], V)) : 0, digit = x >> d.shift & ((1 << d.bits) - 1);
    int below, all;
    bool last;
    match(digit, d.bits, on, lane, below, last, all);
    if (on) {
      const unsigned to = s[w][digit] + below;
      key_out[to] = x;
      row_out[to] = row ? row[k] : (unsigned)k;
      if (last) s[w][digit] = to + 1;  // (read above by every lane of the wave before)
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// The whole sort of up to kOne elements by one block: 16 waves, each with a run of kOne / 16 elements in
// registers, counts and ranks as above.  The blocks behind it clear the table.
constexpr int kOneThreads = 1024, kOne = 16384, kOnePer = kOne / kOneThreads;
__global__ __launch_bounds__(kOneThreads) void sort_one(const int32_t* t, int N, int V, int passes, int bits, unsigned* key_out,
                                                        unsigned* row_out, char* table, size_t bytes) {
  if (blockIdx.x) {
    zero_table(table, bytes, blockIdx.x - 1, gridDim.x - 1);
    return;
  }
  extern __shared__ __align__(16) char dyn[];
  unsigned* const keys = reinterpret_cast<unsigned*>(dyn);                  // [N]
  u16* const rows = reinterpret_cast<u16*>(keys + (N + 1) / 2 * 2);         // [N]
  u16* const count = rows + (N + 1) / 2 * 2;                                // [16][1 << bits]
  __shared__ unsigned part[kDigits];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, waves = blockDim.x >> 6, digits = 1 << bits;
  const int per = ((N + waves - 1) / waves + 63) / 64;  // runs of 64 of a wave
  unsigned x[kOnePer];
  u16 r[kOnePer];
  int to[kOnePer];
#pragma unroll
  for (int i = 0; i < kOnePer; ++i) {
    const int k = (w * per + i) * 64 + lane;
    x[i] = i < per && k < N ? key_of(t[k], V) : 0;
    r[i] = (u16)k;
  }
  for (int p = 0; p < passes; ++p) {
    for (int i = threadIdx.x; i < waves * digits; i += blockDim.x) count[i] = 0;
    __syncthreads();
    // ranks within the wave's run
#pragma unroll
    for (int i = 0; i < kOnePer; ++i) {
      const int k = (w * per + i) * 64 + lane;
      const bool on = i < per && k < N;
      if (i >= per) break;
      const unsigned digit = x[i] >> (p * bits) & (digits - 1);
      int below, all;
      bool last;
      match(digit, bits, on, lane, below, last, all);
      const int before = on ? count[w * digits + digit] : 0;
      to[i] = before + below;
      __builtin_amdgcn_wave_barrier();
      if (on && last) count[w * digits + digit] = (u16)(before + all);
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    // a digit's counts to those before each wave, then the digits' first places
    for (int i = threadIdx.x; i < digits; i += blockDim.x) {
      unsigned sum = 0;
      for (int k = 0; k < waves; ++k) {
        const u16 v = count[k * digits + i];
        count[k * digits + i] = (u16)sum;
        sum += v;
      }
      part[i] = sum;
    }
    __syncthreads();
    if (w == 0) {
      unsigned before = 0;
      for (int i0 = 0; i0 < digits; i0 += 64) {
        const unsigned own = i0 + lane < digits ? part[i0 + lane] : 0;
        unsigned v = own;
        for (int d = 1; d < 64; d <<= 1) {
          const unsigned u = __shfl_up(v, d, 64);
          if (lane >= d) v += u;
        }
        if (i0 + lane < digits) part[i0 + lane] = before + v - own;
        before += __shfl(v, 63, 64);
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kOnePer; ++i) {
      const int k = (w * per + i) * 64 + lane;
      if (i < per && k < N) {
        const unsigned digit = x[i] >> (p * bits) & (digits - 1);
        const unsigned at = to[i] + count[w * digits + digit] + part[digit];
        keys[at] = x[i];
        rows[at] = r[i];
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kOnePer; ++i) {
      const int k = (w * per + i) * 64 + lane;
      if (i < per && k < N) {
        x[i] = keys[k];
        r[i] = rows[k];
      }
    }
    __syncthreads();
  }
  for (int k = threadIdx.x; k < N; k += blockDim.x) {
    key_out[k] = keys[k];
    row_out[k] = rows[k];
  }
}

// ------------------------------------------------------------------------------------------------
// The sums
// ------------------------------------------------------------------------------------------------
struct Sums {
  const unsigned *key, *row;
  int N, D, V;
  int per, chunks;  // sorted rows of a chunk
  float scale;
  float* part;  // [chunks][2][D]: of the run that comes in from the chunk before, and of the one that goes on
  int* end;     // [V]: where a token's run ends, for runs over several chunks
};

// G lanes take a chunk's rows, W elements of D each; grid.y covers D.
template <class E, int W>
__global__ __launch_bounds__(256) void sum_runs(const Sums s, const E* dout, E* out, int G) {
  const int lane = threadIdx.x & (G - 1);
  const int c = blockIdx.x * (256 / G) + threadIdx.x / G;
  const int k = (blockIdx.y * G + lane) * W;
  if (c >= s.chunks || k >= s.D) return;
  const int b = c * s.per, e = min(s.N, b + s.per);
  unsigned cur = s.key[b];
  bool in = b > 0 && s.key[b - 1] == cur;  // the run began in a chunk before
  float sum[W];
#pragma unroll
  for (int i = 0; i < W; ++i) sum[i] = 0.f;
  auto take = [&](float* part) { put_piece<float, W>(part, s.D - k, sum); };
  auto finish = [&](bool on, int at) {  // the run of `cur` ends before `at`, or goes on
    if (cur >= (unsigned)s.V) return;
    float* p = s.part + (size_t)c * 2 * s.D + k;
    if (in) take(p);
    else if (on) take(p + s.D);
    else {
      float v[W];
#pragma unroll
      for (int i = 0; i < W; ++i) v[i] = sum[i] * s.scale;
      put_piece<E, W>(out + (size_t)cur * s.D + k, s.D - k, v);
    }
    if (in && !on && k == 0) s.end[cur] = at;
  };
  // kBatch rows at a time, all of their loads in flight before the first is added (row by row, the places of the rows,
  // then the rows: 512000 rows of 64 took 85 us, not 38)
  constexpr int kBatch = 8;
  bool done = false;
  for (int i0 = b; i0 < e && !done; i0 += kBatch) {
    unsigned key[kBatch], row[kBatch];
    float v[kBatch][W];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int at = min(i0 + i, e - 1);
      key[i] = s.key[at];
      row[i] = s.row[at];
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) piece<E, W>(dout + (size_t)row[i] * s.D + k, s.D - k, v[i]);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (i0 + i >= e || done) continue;
      if (key[i] != cur) {
        finish(false, i0 + i);
        cur = key[i];
        in = false;
#pragma unroll
        for (int q = 0; q < W; ++q) sum[q] = 0.f;
      }
      if (cur >= (unsigned)s.V) {  // the rest is padding
        done = true;
        continue;
      }
#pragma unroll
      for (int q = 0; q < W; ++q) sum[q] += v[i][q];
    }
  }
  const bool on = e < s.N && s.key[e] == cur;
  finish(on, e);
}

// Runs over several chunks: the block of the chunk that a run begins in adds the chunks' partial sums, over
// kJoin / G runs of chunks, then those.
constexpr int kJoin = 512;
template <class E, int W>
__global__ __launch_bounds__(kJoin) void join_runs(const Sums s, E* out, int G) {
  __shared__ float part[kJoin * W];
  const int c = blockIdx.x, last = min(s.N, (c + 1) * s.per) - 1;
  if (last + 1 >= s.N) return;
  const unsigned key = s.key[last];
  if (key >= (unsigned)s.V || s.key[last + 1] != key) return;
  const int b = c * s.per;
  if (b > 0 && s.key[b - 1] == key) return;  // it began before
  const int lane = threadIdx.x & (G - 1), g = threadIdx.x / G, groups = kJoin / G;
  const int n = (s.end[key] - 1) / s.per - c + 1;  // chunks
  const int each = (n + groups - 1) / groups;
  const int k = (blockIdx.y * G + lane) * W;
  float sum[W];
#pragma unroll
  for (int i = 0; i < W; ++i) sum[i] = 0.f;
  if (k < s.D)
#pragma unroll 8
    for (int i = g * each; i < min(n, (g + 1) * each); ++i) {
      float v[W];
      piece<float, W>(s.part + ((size_t)(c + i) * 2 + (i == 0 ? 1 : 0)) * s.D + k, s.D - k, v);
#pragma unroll
      for (int q = 0; q < W; ++q) sum[q] += v[q];
    }
#pragma unroll
  for (int q = 0; q < W; ++q) part[threadIdx.x * W + q] = sum[q];
  __syncthreads();
  if (g == 0 && k < s.D) {
    for (int i = 1; i < groups; ++i)
#pragma unroll
      for (int q = 0; q < W; ++q) sum[q] += part[(i * G + lane) * W + q];
#pragma unroll
    for (int q = 0; q < W; ++q) sum[q] *= s.scale;
    put_piece<E, W>(out + (size_t)key * s.D + k, s.D - k, sum);
  }
}

template <class E>
__global__ __launch_bounds__(256) void fill_zero(E* out, size_t n) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) out[i] = (E)0;
}

// ------------------------------------------------------------------------------------------------
// Host
// ------------------------------------------------------------------------------------------------
bool sizes_ok(int N, int D, int V) { return N >= 0 && N <= kMaxN && D >= 1 && D <= kMaxD && V >= 1 && V <= kMaxV; }

int check(int dtype, int N, int D, int V, float scale) {
  const int rc = bad_dtype(dtype);
  if (rc != WN_OK) return rc;
  if (!sizes_ok(N, D, V)) return wn_set_last_error(WN_EINVAL, "N must be 0..2^27, D 1..2^16, V 1..2^24");
  if (!std::isfinite(scale)) return wn_set_last_error(WN_EINVAL, "scale must be finite");
  return WN_OK;
}

// Lanes of a row of D elements, W each: a power of two up to 256.
int lanes_of(int D, int W) {
  int g = 1;
  while (g < 256 && g * W < D) g *= 2;
  return g;
}

int bits_of(int V) {
  int b = 1;
  while (b < 31 && V >> b) ++b;
  return b;
}

struct Plan {
  int passes, bits;
  int unit, units;   // sort of many blocks: elements of a unit
  int per, chunks;   // sums
  size_t key[2], row[2], count, total_off, part, end, total;
  Plan(int N, int D, int V) {
    passes = (bits_of(V) + 8) / 9;
    bits = (bits_of(V) + passes - 1) / passes;
    unit = (int)std::min<size_t>(4096, std::max<size_t>(256, ceil_div(ceil_div(N, 1024), 64) * 64));
    units = (int)ceil_div(N, unit);
    // chunks of 16 to 256 rows, about 8192 of them
    per = (int)std::min<size_t>(256, std::max<size_t>(16, ceil_div(ceil_div(N, 8192), 8) * 8));
    chunks = (int)ceil_div(N, per);
    size_t at = 0;
    auto take = [&](size_t bytes) {
      const size_t off = at;
      at += up256(bytes);
      return off;
    };
    for (int i = 0; i < 2; ++i) {
      key[i] = take((size_t)N * 4);
      row[i] = take((size_t)N * 4);
    }
    count = take((size_t)units * kDigits * 4);
    total_off = take(kDigits * 4);
    part = take((size_t)chunks * 2 * D * 4);
    end = take((size_t)V * 4);
    total = at;
  }
};

template <class E>
int run_backward(int N, int D, int V, const E* dout, const int32_t* t, float scale, E* out, char* ws, hipStream_t st) {
  const Plan p(N, D, V);
  auto words = [&](size_t off) { return reinterpret_cast<unsigned*>(ws + off); };
  int* const end = reinterpret_cast<int*>(ws + p.end);
  const size_t bytes = (size_t)V * D * sizeof(E);
  const unsigned clear = (unsigned)std::min<size_t>(2048, ceil_div(bytes, 32768));
  int at = 0;  // the sorted keys' buffer
  if (N <= kOne) {
    const int threads = (int)std::min<size_t>(kOneThreads, ceil_div(N, 64) * 64);
    const size_t lds = (size_t)(N + 1) / 2 * 2 * 6 + (size_t)(threads / 64) * 2 * ((size_t)1 << p.bits);
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(sort_one), hipFuncAttributeMaxDynamicSharedMemorySize,
                                             kOne * 6 + 16 * 2 * kDigits);
    if (e != hipSuccess) return wn_set_last_error(WN_EHIP, hipGetErrorString(e));
    hipLaunchKernelGGL(sort_one, dim3(1 + clear), dim3(threads), lds, st, t, N, V, p.passes, p.bits, words(p.key[0]),
                       words(p.row[0]), reinterpret_cast<char*>(out), bytes);
  } else {
    const unsigned *key = nullptr, *row = nullptr;
    for (int i = 0; i < p.passes; ++i) {
      const Digit d{i * p.bits, p.bits};
      at = i & 1;
      const dim3 grid((unsigned)ceil_div(p.units, 4));
      hipLaunchKernelGGL(sort_count, dim3(grid.x + (i == 0 ? clear : 0)), dim3(256), 0, st, t, key, N, V, d, p.unit, p.units,
                         words(p.count), (int)grid.x, reinterpret_cast<char*>(out), bytes);
      hipLaunchKernelGGL(sort_scan, dim3(1 << p.bits), dim3(256), 0, st, words(p.count), p.units, words(p.total_off));
      hipLaunchKernelGGL(sort_scatter, grid, dim3(256), 0, st, t, key, row, N, V, d, p.unit, p.units, words(p.count),
                         words(p.total_off), words(p.key[at]), words(p.row[at]));
      key = words(p.key[at]);
      row = words(p.row[at]);
    }
  }
  Sums s{words(p.key[at]), words(p.row[at]), N, D, V, p.per, p.chunks, scale, reinterpret_cast<float*>(ws + p.part),
         end};
  constexpr int W = 16 / sizeof(E);
  const int G = lanes_of(D, W);
  const unsigned y = (unsigned)ceil_div(D, (size_t)G * W);
  hipLaunchKernelGGL((sum_runs<E, W>), dim3((unsigned)ceil_div(p.chunks, 256 / G), y), dim3(256), 0, st, s, dout, out, G);
  if (p.chunks > 1) hipLaunchKernelGGL((join_runs<E, W>), dim3(p.chunks, y), dim3(kJoin), 0, st, s, out, G);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? WN_OK : wn_set_last_error(WN_EHIP, hipGetErrorString(e));
}

template <class E>
int run_forward(int N, int D, int V, const E* table, const int32_t* t, float scale, E* out, hipStream_t st) {
  constexpr int W = 16 / sizeof(E);
  const int G = lanes_of(D, W);
  hipLaunchKernelGGL((embed_rows<E, W>), many_blocks(ceil_div(N, 256 / G)), dim3(256), 0, st, table, t, N, D, V, scale, out, G);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? WN_OK : wn_set_last_error(WN_EHIP, hipGetErrorString(e));
}

}  // namespace

extern "C" {

size_t wn_embed_backward_workspace_bytes(int32_t N, int32_t D, int32_t V) {
  if (!sizes_ok(N, D, V) || N == 0) return 0;
  return Plan(N, D, V).total;
}

int wn_embed(int32_t dtype, int32_t N, int32_t D, int32_t V, const void* table, const int32_t* t, float scale, void* out,
             void* stream) {
  wn_clear_last_error();
  int rc = check(dtype, N, D, V, scale);
  if (rc != WN_OK || N == 0) return rc;
  if (!table || !t || !out) return wn_set_last_error(WN_EINVAL, "null pointer");
  ArrayScope scope;
  if ((rc = scope.check(table, "table")) != WN_OK || (rc = scope.check(t, "t")) != WN_OK || (rc = scope.check(out, "out")) != WN_OK ||
      (rc = scope.enter()) != WN_OK)
    return rc;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == WN_F32) return run_forward(N, D, V, static_cast<const float*>(table), t, scale, static_cast<float*>(out), st);
  return run_forward(N, D, V, static_cast<const u16*>(table), t, scale, static_cast<u16*>(out), st);
}

int wn_embed_backward(int32_t dtype, int32_t N, int32_t D, int32_t V, const void* dout, const int32_t* t, float scale, void* dtable,
                      void* workspace, size_t ws_bytes, void* stream) {
  wn_clear_last_error();
  int rc = check(dtype, N, D, V, scale);
  if (rc != WN_OK) return rc;
  if (!dtable || (N > 0 && (!dout || !t))) return wn_set_last_error(WN_EINVAL, "null pointer");
  rc = bad_workspace(workspace, ws_bytes, wn_embed_backward_workspace_bytes(N, D, V));
  if (rc != WN_OK) return rc;
  ArrayScope scope;
  if ((rc = scope.check(dtable, "dtable")) != WN_OK) return rc;
  if (N > 0 && ((rc = scope.check(dout, "dout")) != WN_OK || (rc = scope.check(t, "t")) != WN_OK ||
                (rc = scope.check(workspace, "workspace")) != WN_OK))
    return rc;
  if ((rc = scope.enter()) != WN_OK) return rc;
  char* const ws = static_cast<char*>(workspace);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (N == 0) {
    if (dtype == WN_F32) hipLaunchKernelGGL(fill_zero<float>, dim3(1024), dim3(256), 0, st, static_cast<float*>(dtable), (size_t)V * D);
    else hipLaunchKernelGGL(fill_zero<u16>, dim3(1024), dim3(256), 0, st, static_cast<u16*>(dtable), (size_t)V * D);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? WN_OK : wn_set_last_error(WN_EHIP, hipGetErrorString(e));
  }
  if (dtype == WN_F32)
    return run_backward(N, D, V, static_cast<const float*>(dout), t, scale, static_cast<float*>(dtable), ws, st);
  return run_backward(N, D, V, static_cast<const u16*>(dout), t, scale, static_cast<u16*>(dtable), ws, st);
}

}  // extern "C"
