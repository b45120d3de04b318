// Tiled products of 16-bit operands (gfx950): what the files that use them share.  C[b][a] = sum_k A[a][k] B[b][k]
// with different ends (product).
//
// Operands are 16-bit: bf16 arrays as they are, fp32 ones in two fp16 parts each (pack_rows): a
// row is scaled by a power of two so that its largest value lies in [2^14, 2^15), hi = fp16(v),
// lo = fp16(v - hi), which holds v to 2^-22 of itself or 2^-39 of the row's largest, and a product takes
// hi hi + hi lo + lo hi (lo lo is below 2^-22 of it), summed in fp32.
#pragma once
#include "wn_few.h"

namespace {

using namespace wnt;

// A row of an operand is a run of chunks of 64 16-bit units (128 bytes): 64 bf16 values, or the hi parts of
// 32 values and then their lo parts.
constexpr int kChunk = 64;
__host__ __device__ constexpr int chunk_values(bool sp) { return sp ? 32 : 64; }
inline int padded_units(int k, bool sp) { return (int)ceil_div(k, chunk_values(sp)) * kChunk; }

struct Operand {
  const u16* p;
  long long rows;
  int ld;  // units from row to row (a multiple of 8; 16-byte aligned)
  int k;   // units of a row that hold values; those behind read as 0
};

struct Product {
  Operand a, b;
  int ta, tb;    // tiles
  int splits, cps;  // parts of the sum over k, chunks of each
};

typedef __amdgpu_buffer_rsrc_t rsrc;
typedef __attribute__((address_space(3))) void lds_void;

// Tiles of TA x TB outputs by WA x WB waves, with room in LDS for kStages chunks of both operands (a power of two).
template <int TA_, int TB_, int WA_, int WB_, int kStages_ = 2>
struct Tile {
  static constexpr int TA = TA_, TB = TB_, WA = WA_, WB = WB_, kStages = kStages_;
  static constexpr int kWaves = WA * WB, kThreads = 64 * kWaves;
  static constexpr int NA = TA / WA / 16, NB = TB / WB / 16;  // 16 x 16 outputs of a wave
  static constexpr int kStage = (TA + TB) * kChunk * 2;        // bytes of a chunk of both operands
  static constexpr int kLds = kStages * kStage;
  static constexpr int IA = TA * 8 / kThreads, IB = TB * 8 / kThreads;  // 16-byte pieces of a chunk per thread
  static constexpr int kOccupancy = 2;  // waves of a SIMD
  static_assert(NB <= NA, "the order of the reads in product");
};
constexpr int kBand = 8;
using Big = Tile<256, 256, 2, 4>;
using Small = Tile<128, 128, 2, 2>;

// A wave's place in the tile's outputs: lane (n, quad) ends with outputs a = a0 + 16 i + 4 quad + 0..3 of
// row b = b0 + 16 j + n.
struct Place {
  int ta, tb, split;  // tile
  int last;           // the last chunk of the sum
  int a0, b0;         // this wave's first output
  int wa, wb, n, quad;
  // This thread's place in tile (ta, tb).
  template <class T>
  __device__ __forceinline__ void in_tile() {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    wa = wave / T::WB;
    wb = wave % T::WB;
    n = lane & 15;
    quad = lane >> 4;
    a0 = ta * T::TA + wa * (T::TA / T::WA);
    b0 = tb * T::TB + wb * (T::TB / T::WB);
  }
};

// Four 16-bit values at any element's alignment.
typedef u16 u16x4u __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// The sums of chunks c0 .. c1 - 1 of a tile, in V8's type of 16-bit values (SP: hi and lo parts).  Operands go from memory
// straight to LDS (kStages chunks of each), from there to registers half a chunk ahead of their products.
template <class T, bool SP, class V8, class End>
__device__ __forceinline__ void tile_sums(f32x4 (&acc)[T::NA][T::NB], const Operand& a, const Operand& b, const Place& pl, int c0, int c1,
                                          char* lds, const End& end) {
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  auto resource = [&](const Operand& o, long long row0, int rows) {
    const long long left = o.rows - row0 < rows ? o.rows - row0 : rows;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<u16*>(o.p) + row0 * o.ld, (short)0,
                                             (int)(((left - 1) * o.ld + o.k) * 2), 0x00020000);
  };
  const rsrc ares = resource(a, (long long)pl.ta * T::TA, T::TA), bres = resource(b, (long long)pl.tb * T::TB, T::TB);
  // 16-byte piece `pos` of row r in LDS is piece pos ^ (r >> 1 & 7) of the row's chunk: the 16 rows that 16 lanes
  // read at one piece then fall on different banks.  A thread's pieces are all at the same place of their rows
  // (kThreads / 8 rows is a multiple of 16).
  const int piece = (tid & 7) ^ (tid >> 4 & 7);
  const int va = (tid >> 3) * a.ld * 2 + piece * 16, vb = (tid >> 3) * b.ld * 2 + piece * 16;
  auto stage_piece = [&](int c, char* to, int i) {
    const bool isa = i < T::IA;
    const int k = isa ? i : i - T::IA;
    const int at = (k * T::kThreads + wave * 64) * 16 + (isa ? 0 : T::TA * kChunk * 2);
    // (a piece behind the row's values reads past the buffer's end, which gives 0)
    const int v = piece * 8 < (isa ? a.k : b.k) - c * kChunk ? (isa ? va : vb) + k * (T::kThreads / 8) * (isa ? a.ld : b.ld) * 2 : (int)0x80000000;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(isa ? ares : bres, (lds_void*)(to + at), 16, v, c * kChunk * 2, 0, 0);
  };
  constexpr int kPieces = T::IA + T::IB;
  auto stage = [&](int c, char* to) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) stage_piece(c, to, i);
  };
  // the pieces that step i of T::NA issues
  auto stage_part = [&](int c, char* to, int i) {
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
      if (k * T::NA / kPieces == i) stage_piece(c, to, k);
  };
#pragma unroll
  for (int i = 0; i < T::NA; ++i)
#pragma unroll
    for (int j = 0; j < T::NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  constexpr int S = T::kStages;
  const int ra = pl.wa * (T::TA / T::WA), rb = pl.wb * (T::TB / T::WB);
  const int sw = pl.n >> 1;
  const int fa = (ra + pl.n) * kChunk * 2, fb = (T::TA + rb + pl.n) * kChunk * 2;
  const int s0 = (pl.quad ^ sw) * 16, s1 = ((4 + pl.quad) ^ sw) * 16;
  auto buffer = [&](int c) { return lds + ((c - c0) & (S - 1)) * T::kStage; };
  auto get = [&](const char* at, int row, int s) { return *reinterpret_cast<const V8*>(at + row + s); };
  constexpr int kRow = 16 * kChunk * 2;
  // a chunk's first and second half of each operand's values (SP: hi and lo parts)
  V8 a0[T::NA], a1[T::NA], b0[T::NB], b1[T::NB];
  if (c0 < c1) {
#pragma unroll
    for (int k = 0; k < S; ++k)
      if (c0 + k < c1) stage(c0 + k, lds + k * T::kStage);
    if (c0 + S - 1 < c1) {
      asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"i"((S - 1) * kPieces) : "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    }
    const char* at = buffer(c0);
#pragma unroll
    for (int j = 0; j < T::NB; ++j) b0[j] = get(at, fb + j * kRow, s0);
#pragma unroll
    for (int i = 0; i < T::NA; ++i) a0[i] = get(at, fa + i * kRow, s0);
  }
  // A chunk in two halves, each half's operands read from LDS during the products of the half before.  The one
  // barrier stands where a chunk's last reads are done: it lets the chunk after next into its buffer, whose loads are
  // spread over the second half's products, and says that the next one has arrived.
  for (int c = c0; c < c1; ++c) {
    const char* at = buffer(c);
    char* const to = buffer(c);
    if constexpr (End::kScaledByTile)
      if (c > c0) end.template to_chunk<T>(acc, pl, c);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int i = 0; i < T::NA; ++i) {
      a1[i] = get(at, fa + i * kRow, s1);
      if (i < T::NB) b1[i] = get(at, fb + i * kRow, s1);
#pragma unroll
      for (int j = 0; j < T::NB; ++j) acc[i][j] = mma(a0[i], b0[j], acc[i][j]);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    // (of what is under way only the next chunk is waited for, while all buffers are in use)
    if (S == 2 || c + S - 1 >= c1) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"i"((S - 2) * kPieces) : "memory");
    const bool more = c + S < c1;
    at = buffer(c + 1);
    __builtin_amdgcn_s_setprio(1);
    if constexpr (SP) {
      if (more) stage(c + S, to);  // (spread over the products they spill)
#pragma unroll
      for (int i = 0; i < T::NA; ++i) {
#pragma unroll
        for (int j = 0; j < T::NB; ++j) acc[i][j] = mma(a1[i], b0[j], acc[i][j]);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < T::NA; ++i) {
        if (i < T::NB) b0[i] = get(at, fb + i * kRow, s0);
#pragma unroll
        for (int j = 0; j < T::NB; ++j) acc[i][j] = mma(a0[i], b1[j], acc[i][j]);
        a0[i] = get(at, fa + i * kRow, s0);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < T::NA; ++i) {
        if (more) stage_part(c + S, to, i);
        a0[i] = get(at, fa + i * kRow, s0);
        if (i < T::NB) b0[i] = get(at, fb + i * kRow, s0);
#pragma unroll
        for (int j = 0; j < T::NB; ++j) acc[i][j] = mma(a1[i], b1[j], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __builtin_amdgcn_s_setprio(0);
  }
  __syncthreads();
}

// C[b][a] = sum_k A[a][k] B[b][k] on v_mfma_f32_16x16x32_bf16 or _f16; `end` takes the tile's sums.  Bound: the
// matrix units at the clock that the card holds under them.  Measured, bf16: 8192 x 65536 outputs over 2048 with the
// forward end 1.69 ms, 1.30 PFLOP/s (a plain library product of this shape 1.58 ms), dw of 65536 x 2048 over 8192 and
// dx over pieces of 22016 classes 1.27 PFLOP/s (library 1.24); the matrix units are busy 55 % of the cycles at 2.1 GHz,
// on another card 66 % at 1.8, no LDS bank conflicts.  256 x 128 tiles with two blocks a CU, so that one's ends run
// beside the other's products, reached 1.18 PFLOP/s where these reach 1.5 (their operands come from L2 half as often
// again).
template <class T, bool SP, class End>
__global__ __launch_bounds__(T::kThreads, T::kOccupancy) void product(const Product g, const End end) {
  extern __shared__ __align__(16) char lds[];
  Place pl;
  {
    // Block b runs on XCD b mod 8.  Each XCD takes a run of tiles, in the order of bands of kBand tiles of b:
    // the tiles it works on at a time share the operands' rows in its L2.
    const int blocks = gridDim.x, xcd = blockIdx.x & 7, per = blocks >> 3, rem = blocks & 7;
    int t = xcd * per + min(xcd, rem) + (blockIdx.x >> 3);
    const int tiles = g.ta * g.tb;
    pl.split = t / tiles;
    t -= pl.split * tiles;
    const int band = t / (kBand * g.ta), in = t - band * kBand * g.ta, wide = min(kBand, g.tb - band * kBand);
    pl.ta = in / wide;
    pl.tb = band * kBand + in - pl.ta * wide;
  }
  pl.in_tile<T>();
  const int kc = (max(g.a.k, g.b.k) + kChunk - 1) / kChunk;
  const int c0 = pl.split * g.cps, c1 = min(kc, c0 + g.cps);
  pl.last = c1 - 1;
  f32x4 acc[T::NA][T::NB];
  tile_sums<T, SP, typename std::conditional<SP, f16x8, bf16x8>::type>(acc, g.a, g.b, pl, c0, c1, lds, end);
  end.template operator()<T>(acc, pl, lds);
}

// What both ends of the logits product need: l[n][v] = acc 2^-(ex[n] + ew[v]) + b[v].
struct Logits {
  const int *ex, *ew;  // the operands' scales (fp32 arrays), or null
  const float* bias;   // of the piece, or null
  const int32_t* y;
  int N, V, v0, V_all;  // rows; classes of the piece, the first of them, and of the layer
  template <class T>
  __device__ __forceinline__ void take(f32x4 (&acc)[T::NA][T::NB], const Place& pl) const {
    if (ew) {
      int sn[T::NB];
#pragma unroll
      for (int j = 0; j < T::NB; ++j) sn[j] = ex[min(pl.b0 + 16 * j + pl.n, N - 1)];
#pragma unroll
      for (int i = 0; i < T::NA; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int sv = ew[min(pl.a0 + 16 * i + 4 * pl.quad + e, V - 1)];
#pragma unroll
          for (int j = 0; j < T::NB; ++j) acc[i][j][e] = ldexpf(acc[i][j][e], -(sv + sn[j]));
        }
    }
    if (bias) {
#pragma unroll
      for (int i = 0; i < T::NA; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float bv = bias[min(pl.a0 + 16 * i + 4 * pl.quad + e, V - 1)];
#pragma unroll
          for (int j = 0; j < T::NB; ++j) acc[i][j][e] += bv;
        }
    }
    if (pl.a0 + 16 * T::NA > V) {  // the last tile: no classes behind V
#pragma unroll
      for (int i = 0; i < T::NA; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool in = pl.a0 + 16 * i + 4 * pl.quad + e < V;
#pragma unroll
          for (int j = 0; j < T::NB; ++j) acc[i][j][e] = in ? acc[i][j][e] : -INFINITY;
        }
    }
  }
  // Calls f(i, e) where this lane holds class t (of the piece) as its output i, e of a row; few waves hold any
  // row's target, so the search is skipped where none does.
  template <class T, class F>
  __device__ __forceinline__ static void at_target(const Place& pl, int t, F f) {
    const int r = t - pl.a0 - 4 * pl.quad;
    if (!__any(t >= pl.a0 && t < pl.a0 + 16 * T::NA)) return;
#pragma unroll
    for (int i = 0; i < T::NA; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (r == 16 * i + e) f(i, e);
  }
};

__device__ __forceinline__ void split(float v, u16& hi, u16& lo) {
  const _Float16 h = (_Float16)v;
  const float r = v - (float)h;
  hi = __builtin_bit_cast(u16, h);
  lo = __builtin_bit_cast(u16, (_Float16)(r == r ? r : 0.f));  // (an infinity has no rest)
}

// ------------------------------------------------------------------------------------------------
// The operands
// ------------------------------------------------------------------------------------------------
// The scale of a row whose largest magnitude is m: m 2^e in [2^14, 2^15).
__device__ __forceinline__ int scale_of(float m) { return m > 0.f && m < INFINITY ? 14 - ilogbf(m) : 0; }

// Values k .. k + 3 of a row of K, zeros behind it.
__device__ __forceinline__ f32x4 four(const float* s, int k, int K) {
  if (k + 3 < K) {
    const f32x4u x = *reinterpret_cast<const f32x4u*>(s + k);
    return f32x4{x[0], x[1], x[2], x[3]};
  }
  return f32x4{k < K ? s[k] : 0.f, k + 1 < K ? s[k + 1] : 0.f, k + 2 < K ? s[k + 2] : 0.f, 0.f};
}
// Four values' hi and lo parts to a row's place for value k (a multiple of 4).
__device__ __forceinline__ void put_split(u16* row, int k, f32x4 v) {
  u16 hi[4], lo[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) split(v[e], hi[e], lo[e]);
  u16* p = row + k / 32 * kChunk + k % 32;
  *reinterpret_cast<u32x2*>(p) = u32x2{(unsigned)hi[0] | (unsigned)hi[1] << 16, (unsigned)hi[2] | (unsigned)hi[3] << 16};
  *reinterpret_cast<u32x2*>(p + 32) = u32x2{(unsigned)lo[0] | (unsigned)lo[1] << 16, (unsigned)lo[2] | (unsigned)lo[3] << 16};
}
__device__ __forceinline__ f32x4 scaled(f32x4 v, int e) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = ldexpf(v[i], e);
  return v;
}

// Bound, all of these: reading the array and writing as much.  Measured: [16000][256] fp32 rows 12 us, columns 11 and
// their maxima 12; [22016][2048] bf16 columns 53 us (3.4 TB/s).
// Rows [R][K] as they are; a wave per row.  fp32 rows of up to 1024 values stay in registers between the search
// for their scale and the split.
// One launch takes up to two arrays.
template <class E>
struct Rows {
  const E* src;
  int R, K;
  u16* dst;
  int units;
  int* scale;
};
template <class E>
__global__ __launch_bounds__(256) void pack_rows(const Rows<E> first, const Rows<E> second, int blocks) {
  const bool two = (int)blockIdx.x >= blocks;  // (blocks: the first array's)
  const Rows<E>& a = two ? second : first;
  const int r = ((int)blockIdx.x - (two ? blocks : 0)) * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= a.R) return;
  const int K = a.K, units = a.units;
  const E* s = a.src + (size_t)r * K;
  u16* d = a.dst + (size_t)r * units;
  if constexpr (sizeof(E) == 2) {
    typedef u16 u16x8u __attribute__((ext_vector_type(8), aligned(2)));
    typedef u16 u16x8 __attribute__((ext_vector_type(8)));
    for (int k = 8 * lane; k < units; k += 512) {
      u16x8 x;
      if (k + 7 < K) {
        const u16x8u v = *reinterpret_cast<const u16x8u*>(s + k);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = v[e];
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = k + e < K ? s[k + e] : (u16)0;
      }
      *reinterpret_cast<u16x8*>(d + k) = x;
    }
  } else {
    constexpr int H = 4;
    f32x4 v[H];
    float m = 0.f;
#pragma unroll
    for (int h = 0; h < H; ++h) v[h] = 256 * h < K ? four(s, 256 * h + 4 * lane, K) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int h = 0; h < H; ++h) m = fmaxf(fmaxf(fmaxf(m, fabsf(v[h][0])), fabsf(v[h][1])), fmaxf(fabsf(v[h][2]), fabsf(v[h][3])));
    for (int k = 256 * H + 4 * lane; k < K; k += 256) {
      const f32x4 x = four(s, k, K);
      m = fmaxf(fmaxf(fmaxf(m, fabsf(x[0])), fabsf(x[1])), fmaxf(fabsf(x[2]), fabsf(x[3])));
    }
    const int e = scale_of(wnk::wave_max(m));
    if (lane == 0) a.scale[r] = e;
#pragma unroll
    for (int h = 0; h < H; ++h)
      if (256 * h + 4 * lane < units / 2) put_split(d, 256 * h + 4 * lane, scaled(v[h], e));
    for (int k = 256 * H + 4 * lane; k < units / 2; k += 256) put_split(d, k, scaled(four(s, k, K), e));
  }
}

// ------------------------------------------------------------------------------------------------
// Host
// ------------------------------------------------------------------------------------------------
constexpr size_t kForwardPiece = (size_t)64 << 20;    // bytes of packed w in the forward pass
constexpr int kMaxN = 1 << 20, kMaxD = 1 << 16, kMaxV = 1 << 24;
constexpr size_t kSplitFloats = (size_t)64 << 20;     // values of a product's parts, at most

inline bool sizes_ok(int dtype, int N, int D, int V) {
  return (dtype == WN_F32 || dtype == WN_BF16) && N >= 0 && N <= kMaxN && D >= 1 && D <= kMaxD && V >= 1 && V <= kMaxV;
}

// How a product of a x b outputs over `chunks` chunks is tiled, and in how many parts its sum is taken: the shortest
// time by a model of the two tiles.  A chunk of 256 x 256 outputs takes a CU 1.4 us (three products of fp16 parts:
// 2.1), of 128 x 128 two blocks on a CU 1.2 us; a tile's start and end 6 and 4 us; parts are written and joined
// at 4.5 TB/s.
struct Shape {
  bool big;
  int splits;
  double us;
};
inline Shape shape_for(size_t a, size_t b, int units, bool sp, bool may_split) {
  static const int kSplits[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 64, 96, 128};
  const size_t chunks = ceil_div(units, kChunk);
  Shape best{false, 1, 1e30};
  for (int big = 0; big < 2; ++big) {
    const size_t t = big ? 256 : 128, tiles = ceil_div(a, t) * ceil_div(b, t), room = big ? 256 : 512;
    const double chunk = (big ? 1.4 : 1.2) * (sp ? 1.5 : 1.0), ends = big ? 6.0 : 4.0;
    for (int s : kSplits) {
      if (s > 1 && (!may_split || chunks / s < 4 || (size_t)s * a * b > kSplitFloats)) break;
      const double us = (double)ceil_div(tiles * s, room) * ((double)ceil_div(chunks, s) * chunk + ends) +
                        (s > 1 ? 5.0 + (s + 1.0) * a * b * 4 / 4.5e6 : 0.0);
      if (us < best.us) best = {big != 0, s, us};
    }
  }
  return best;
}

// Classes of a forward piece: a multiple of 256, pieces alike.  `each`: bytes of a packed class, 0 where w stays as it is.  A
// launch takes fewer than 2^32 threads: 256 for 128 x 128 outputs, half as many for 256 x 256.
inline int forward_piece(int N, int V, size_t each) {
  const size_t launch = (((size_t)1 << 24) - 1) / ceil_div(N, 128) * 128;
  const size_t most = std::max<size_t>(256, (each ? std::min(launch, kForwardPiece / each) : launch) / 256 * 256);
  const size_t pieces = ceil_div(V, most);
  return (int)std::min<size_t>(V, ceil_div(ceil_div(V, pieces), 256) * 256);
}

struct Carve {
  size_t at = 0;
  size_t take(size_t bytes) {
    const size_t off = at;
    at += up256(bytes);
    return off;
  }
};

template <class T, bool SP, class End>
hipError_t launch_product(Product g, const End& end, hipStream_t st) {
  g.ta = (int)ceil_div(g.a.rows, T::TA);
  g.tb = (int)ceil_div(g.b.rows, T::TB);
  const int kc = (int)ceil_div(std::max(g.a.k, g.b.k), kChunk);
  g.cps = (int)ceil_div(kc, g.splits);
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(product<T, SP, End>),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, T::kLds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((product<T, SP, End>), dim3((unsigned)g.ta * g.tb * g.splits), dim3(T::kThreads), T::kLds, st, g, end);
  return hipGetLastError();
}

// Rows of the tile are a tile's rows in `part` and `db`: big says which.
template <bool SP, class End>
hipError_t run_product(const Product& g, bool big, const End& end, hipStream_t st) {
  return big ? launch_product<Big, SP>(g, end, st) : launch_product<Small, SP>(g, end, st);
}

// [R][K] as operands: as they lie, or packed into `dst` by launch(), up to two of them.
template <class E>
struct RowPacker {
  Rows<E> todo[2];
  int n = 0;
  Operand add(const E* src, int R, int K, u16* dst, int* scale) {
    constexpr bool sp = sizeof(E) == 4;
    if (!sp && K % 8 == 0 && reinterpret_cast<uintptr_t>(src) % 16 == 0) return {reinterpret_cast<const u16*>(src), R, K, K};
    const int units = padded_units(K, sp);
    todo[n++] = {src, R, K, dst, units, scale};
    return {dst, R, units, units};
  }
  void launch(hipStream_t st) {
    if (!n) return;
    const unsigned one = (unsigned)ceil_div(todo[0].R, 4), both = one + (n > 1 ? (unsigned)ceil_div(todo[1].R, 4) : 0);
    hipLaunchKernelGGL(pack_rows<E>, dim3(both), dim3(256), 0, st, todo[0], todo[n - 1], (int)one);
    n = 0;
  }
};

inline int check_sizes(int dtype, int N, int D, int V) {
  const int rc = bad_dtype(dtype);
  if (rc != WN_OK) return rc;
  return sizes_ok(dtype, N, D, V) ? WN_OK : wn_set_last_error(WN_EINVAL, "N must be 0..2^20, D 1..2^16, V 1..2^24");
}

}  // namespace
