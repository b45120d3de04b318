// The loss of an output layer and its gradients without keeping the logits (gfx950).  Declarations and
// contracts are in include/wn_train.h.
//
// Everything heavy is one product C[b][a] = sum_k A[a][k] B[b][k] with different ends (product):
//   logits   A = w, B = x           the tile's largest logit and sum of exponentials of each row (forward), or
//                                   q = exp(l - lse) - [v = y] as the next products' operand (backward)
//   dx       A = w transposed, B = q
//   dw       A = x transposed, B = q transposed
// Both operands lie along k in memory, so the transposed ones are copies (pack_cols); the backward pass takes
// the vocabulary in pieces, so that they and q stay within a fixed size.
//
// Operands are 16-bit: bf16 arrays as they are, fp32 ones in two fp16 parts each (pack_rows, pack_cols): a
// row is scaled by a power of two so that its largest value lies in [2^14, 2^15), hi = fp16(v),
// lo = fp16(v - hi), which holds v to 2^-22 of itself or 2^-39 of the row's largest, and a product takes
// hi hi + hi lo + lo hi (lo lo is below 2^-22 of it), summed in fp32.
//
// Up to kFewRows rows go to wn_few.hip, which is bound by reading w once (64 and 65 rows x 50021 classes x 777: forward 42
// and 70 us in bf16, 79 and 134 in fp32).
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

// Tiles of TA x TB outputs by WA x WB waves.
template <int TA_, int TB_, int WA_, int WB_>
struct Tile {
  static constexpr int TA = TA_, TB = TB_, WA = WA_, WB = WB_;
  static constexpr int kWaves = WA * WB, kThreads = 64 * kWaves;
  static constexpr int NA = TA / WA / 16, NB = TB / WB / 16;  // 16 x 16 outputs of a wave
  static constexpr int kStage = (TA + TB) * kChunk * 2;        // bytes of a chunk of both operands
  static constexpr int kLds = 2 * kStage;
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
};

// Four 16-bit or fp32 values at any element's alignment.
typedef u16 u16x4u __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// C[b][a] = sum_k A[a][k] B[b][k] on v_mfma_f32_16x16x32_bf16 or _f16; `end` takes the tile's sums.  Operands go from
// memory straight to LDS (two chunks of each), from there to registers half a chunk ahead of their products.  Bound: the
// matrix units at the clock that the card holds under them.  Measured, bf16: 8192 x 65536 outputs over 2048 with the
// forward end 1.69 ms, 1.30 PFLOP/s (a plain library product of this shape 1.58 ms), dw of 65536 x 2048 over 8192 and
// dx over pieces of 22016 classes 1.27 PFLOP/s (library 1.24); the matrix units are busy 55 % of the cycles at 2.1 GHz,
// on another card 66 % at 1.8, no LDS bank conflicts.  256 x 128 tiles with two blocks a CU, so that one's ends run beside the other's products,
// reached 1.18 PFLOP/s where these reach 1.5 (their operands come from L2 half as often again).
template <class T, bool SP, class End>
__global__ __launch_bounds__(T::kThreads, T::kOccupancy) void product(const Product g, const End end) {
  extern __shared__ __align__(16) char lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
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
  pl.wa = wave / T::WB;
  pl.wb = wave % T::WB;
  pl.n = lane & 15;
  pl.quad = lane >> 4;
  const int ra = pl.wa * (T::TA / T::WA), rb = pl.wb * (T::TB / T::WB);
  pl.a0 = pl.ta * T::TA + ra;
  pl.b0 = pl.tb * T::TB + rb;

  auto resource = [&](const Operand& o, long long row0, int rows) {
    const long long left = o.rows - row0 < rows ? o.rows - row0 : rows;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<u16*>(o.p) + row0 * o.ld, (short)0,
                                             (int)(((left - 1) * o.ld + o.k) * 2), 0x00020000);
  };
  const rsrc ares = resource(g.a, (long long)pl.ta * T::TA, T::TA), bres = resource(g.b, (long long)pl.tb * T::TB, T::TB);
  // 16-byte piece `pos` of row r in LDS is piece pos ^ (r >> 1 & 7) of the row's chunk: the 16 rows that 16 lanes
  // read at one piece then fall on different banks.  A thread's pieces are all at the same place of their rows
  // (kThreads / 8 rows is a multiple of 16).
  const int piece = (tid & 7) ^ (tid >> 4 & 7);
  const int va = (tid >> 3) * g.a.ld * 2 + piece * 16, vb = (tid >> 3) * g.b.ld * 2 + piece * 16;
  const int kc = (max(g.a.k, g.b.k) + kChunk - 1) / kChunk;
  const int c0 = pl.split * g.cps, c1 = min(kc, c0 + g.cps);
  pl.last = c1 - 1;
  auto stage_piece = [&](int c, char* to, int i) {
    const bool isa = i < T::IA;
    const int k = isa ? i : i - T::IA;
    const int at = (k * T::kThreads + wave * 64) * 16 + (isa ? 0 : T::TA * kChunk * 2);
    // (a piece behind the row's values reads past the buffer's end, which gives 0)
    const int v = piece * 8 < (isa ? g.a.k : g.b.k) - c * kChunk ? (isa ? va : vb) + k * (T::kThreads / 8) * (isa ? g.a.ld : g.b.ld) * 2 : (int)0x80000000;
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
  f32x4 acc[T::NA][T::NB];
#pragma unroll
  for (int i = 0; i < T::NA; ++i)
#pragma unroll
    for (int j = 0; j < T::NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  typedef typename std::conditional<SP, f16x8, bf16x8>::type V8;
  const int sw = pl.n >> 1;
  const int fa = (ra + pl.n) * kChunk * 2, fb = (T::TA + rb + pl.n) * kChunk * 2;
  const int s0 = (pl.quad ^ sw) * 16, s1 = ((4 + pl.quad) ^ sw) * 16;
  auto buffer = [&](int c) { return lds + ((c - c0) & 1) * T::kStage; };
  auto get = [&](const char* at, int row, int s) { return *reinterpret_cast<const V8*>(at + row + s); };
  constexpr int kRow = 16 * kChunk * 2;
  // a chunk's first and second half of each operand's values (SP: hi and lo parts)
  V8 a0[T::NA], a1[T::NA], b0[T::NB], b1[T::NB];
  if (c0 < c1) {
    stage(c0, buffer(c0));
    if (c0 + 1 < c1) {
      stage(c0 + 1, buffer(c0 + 1));
      asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"i"(T::IA + T::IB) : "memory");
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
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const bool more = c + 2 < c1;
    at = buffer(c + 1);
    __builtin_amdgcn_s_setprio(1);
    if constexpr (SP) {
      if (more) stage(c + 2, to);  // (spread over the products they spill)
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
        if (more) stage_part(c + 2, to, i);
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

// Forward: (largest logit, sum of exp(l - largest)) of each row in the tile's classes, and the target's logit.  The largest
// is taken off a logit before the product with log2 e: l - largest is exact near it, so the largest class counts 1 wherever the
// logits lie and no loss is negative.  (fma(l, log2 e, -largest log2 e) is one operation shorter, but the rounding of
// its last term moves every exponential of the row: by 1e-6 at logits of 20, a factor of 3e5 at -1e9.)
struct StatsEnd {
  static constexpr bool kScaledByTile = false;
  Logits l;
  float2* part;   // [tiles of all pieces][N]
  int tile0;      // the piece's first
  float* target;  // [N]
  template <class T>
  __device__ void operator()(f32x4 (&acc)[T::NA][T::NB], const Place& pl, char* lds) const {
    l.take<T>(acc, pl);
    float2* const s = reinterpret_cast<float2*>(lds);  // [WA][TB]
#pragma unroll
    for (int j = 0; j < T::NB; ++j) {
      const int n = pl.b0 + 16 * j + pl.n;
      const int yn = n < l.N ? l.y[n] : -1, t = yn >= 0 ? yn - l.v0 : -1;
      float m = -INFINITY, sum = 0.f;
#pragma unroll
      for (int i = 0; i < T::NA; ++i) m = fmaxf(fmaxf(fmaxf(m, acc[i][j][0]), acc[i][j][1]), fmaxf(acc[i][j][2], acc[i][j][3]));
      m = quads_max(m);
      Logits::at_target<T>(pl, t < l.V ? t : -1, [&](int i, int e) { target[n] = acc[i][j][e]; });
      // (a row without a class yet: every exponential is 0, not exp(-inf + inf))
      const float at = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int i = 0; i < T::NA; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += wnk::expf_fast(acc[i][j][e] - at);
      sum = quads_sum(sum);
      if (pl.quad == 0) s[pl.wa * T::TB + pl.wb * (T::TB / T::WB) + 16 * j + pl.n] = make_float2(m, sum);
    }
    __syncthreads();
    for (int k = threadIdx.x; k < T::TB; k += T::kThreads) {
      const int n = pl.tb * T::TB + k;
      float2 r = s[k];
#pragma unroll
      for (int w = 1; w < T::WA; ++w) {
        const float2 o = s[w * T::TB + k];
        const float m = fmaxf(r.x, o.x), at = m == -INFINITY ? 0.f : m;
        r = make_float2(m, r.y * wnk::expf_fast(r.x - at) + o.y * wnk::expf_fast(o.x - at));
      }
      if (n < l.N) part[(size_t)(tile0 + pl.ta) * l.N + n] = r;
    }
  }
};

// Largest |g| of the rows with a target: parts[blockIdx.x] of each block's, joined by whoever needs it.
constexpr int kGParts = 64;
__global__ __launch_bounds__(256) void largest_g(const float* g, const int32_t* y, int N, int V, float* parts) {
  __shared__ float s[4];
  float m = 0.f;
  for (int n = blockIdx.x * 256 + threadIdx.x; n < N; n += gridDim.x * 256) {
    const int t = y[n];
    if (t >= 0 && t < V) m = fmaxf(m, fabsf(g[n]));
  }
  m = wnk::wave_max(m);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x == 0) parts[blockIdx.x] = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
}
__device__ __forceinline__ float join_largest(const float* parts, int n) {
  const int lane = threadIdx.x & 63;
  return wnk::wave_max(lane < n ? parts[lane] : 0.f);
}

// 16-bit operand units of q: bf16, or fp16 parts of q 2^e.  As dx's operand e is 14: a row's largest q is off by 2^-24 as
// 1 - p, so what 2^-39 cuts off is not seen.  As dw's operand a row is a class, which no row may target and whose
// probabilities may all be small: there e is the class's own within a tile of rows, so that the tile's
// largest p (1 if a row targets the class) lies in [2^14, 2^15), up to kQMost (a tile all below 2^-66 is held to 2^-105).  dw's sums change from one tile's
// scale to the next by at most 2^66: below 2^116 with 2^20 rows of products below 2^30.
constexpr int kQScale = 14, kQMost = 80;
__device__ __forceinline__ void split(float v, u16& hi, u16& lo) {
  const _Float16 h = (_Float16)v;
  const float r = v - (float)h;
  hi = __builtin_bit_cast(u16, h);
  lo = __builtin_bit_cast(u16, (_Float16)(r == r ? r : 0.f));  // (an infinity has no rest)
}

// Backward: q of the tile's rows and classes as the operands of dx ([n][v]) and dw ([v][n]), and the sums of g q
// over the tile's rows.  q enters the products without g (|q| <= 1): dx's rows take their g afterwards, and so does dw:
// fp32 arrays with x's rows, bf16 ones as g / max |g| here and max |g| afterwards.  So the target's entry, -1 and a
// probability, is hardly touched by q's rounding to bf16: with g in q all rows of a mean shared the rounding
// error of -1 / N, which was off by 0.38 % in both gradients (4096 rows of text; now 0.17 %, what the
// gradients' own rounding costs).  A lane holds four classes of a row, so [n][v] is
// stored from the registers (32-byte runs); [v][n] goes through LDS, a wave's classes by 64 rows (fp32: 32 rows,
// hi and lo parts) at a time, so that its stores are runs of 128 bytes.
template <bool SP>
struct GradEnd {
  static constexpr bool kScaledByTile = false;
  Logits l;
  const float *lse, *g;
  const float* gmax;  // bf16: parts of max |g| (largest_g); null without qt
  int gparts;
  u16 *q, *qt;     // or null
  int ldq, ldqt;
  int* eq;         // fp32: qt's scales, [tiles of rows][V]
  float* db;       // [tiles of rows][V], or null
  // 2^e of this lane's classes over the tile's rows, whose log p are in acc: a class's rows lie in 16 lanes of each of WB
  // waves.  A class that a row of the tile targets may have a q near -1.
  template <class T>
  __device__ __forceinline__ void class_scales(const f32x4 (&acc)[T::NA][T::NB], const Place& pl, char* lds, f32x4 (&by)[T::NA]) const {
    float* const s = reinterpret_cast<float*>(lds);  // [WB][TA], and [TA]: 0 for a target, -inf
    for (int k = threadIdx.x; k < T::TA; k += T::kThreads) s[T::WB * T::TA + k] = -INFINITY;
    __syncthreads();
    for (int k = threadIdx.x; k < T::TB; k += T::kThreads) {
      const int n = pl.tb * T::TB + k, yn = n < l.N ? l.y[n] : -1, a = yn < 0 ? -1 : yn - l.v0 - pl.ta * T::TA;
      if (a >= 0 && a < T::TA) s[T::WB * T::TA + a] = 0.f;
    }
    const int at = pl.wa * 16 * T::NA + 4 * pl.quad;
#pragma unroll
    for (int i = 0; i < T::NA; ++i) {
      f32x4 m;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        m[e] = acc[i][0][e];
#pragma unroll
        for (int j = 1; j < T::NB; ++j) m[e] = fmaxf(m[e], acc[i][j][e]);
        m[e] = row16_max(m[e]);
      }
      if (pl.n == 0) *reinterpret_cast<f32x4*>(s + pl.wb * T::TA + at + 16 * i) = m;
    }
    __syncthreads();
    for (int k = threadIdx.x; k < T::TA; k += T::kThreads) {
      float m = s[k];
#pragma unroll
      for (int w = 1; w <= T::WB; ++w) m = fmaxf(m, s[w * T::TA + k]);
      const int e = kQScale - (int)fminf(fmaxf(floorf(m * 1.4426950408889634f), kQScale - kQMost), 0.f), v = pl.ta * T::TA + k;
      s[k] = __uint_as_float((unsigned)(127 + e) << 23);
      if (v < l.V) eq[(size_t)pl.tb * l.V + v] = e;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < T::NA; ++i) by[i] = *reinterpret_cast<const f32x4*>(s + at + 16 * i);
    __syncthreads();  // (what follows writes where s lies)
  }
  template <class T>
  __device__ void operator()(f32x4 (&acc)[T::NA][T::NB], const Place& pl, char* lds) const {
    l.take<T>(acc, pl);
    const float most = !SP && qt ? join_largest(gmax, gparts) : 1.f;
    constexpr int RA = 16 * T::NA, RB = 16 * T::NB;  // the wave's classes and rows
    static_assert(RB == 64, "a row of the transposed tile is 128 bytes");
    char* const tr = lds + (pl.wa * T::WB + pl.wb) * RA * 128;
    const int lane = threadIdx.x & 63;
    // Two lanes that hold neighbouring rows (n even, n + 1) swap two of their four classes: the even lane then holds
    // classes 0 and 1 of both rows, the odd one classes 2 and 3, and each writes pairs.
    const bool odd = lane & 1;
    auto swap = [&](u16 (&v)[4], unsigned& p0, unsigned& p1) {
      const unsigned lo = (unsigned)v[0] | (unsigned)v[1] << 16, hi = (unsigned)v[2] | (unsigned)v[3] << 16;
      const unsigned give = odd ? lo : hi, keep = odd ? hi : lo;
      const unsigned got = (unsigned)__builtin_amdgcn_update_dpp(0, (int)give, 0xB1, 0xf, 0xf, false);
      const unsigned e = odd ? got : keep, o = odd ? keep : got;  // of the even and the odd row
      p0 = (e & 0xffffu) | o << 16;
      p1 = e >> 16 | (o & 0xffff0000u);
    };
    // piece (16 bytes) of row v of the transposed tile, as it lies
    auto place = [](int v, int piece) { return v * 128 + ((piece ^ (v >> 1 & 7)) << 4); };
    auto put_pair = [&](int i, int col, u16 (&v)[4]) {  // col: unit of the row's first of the two
      unsigned p0, p1;
      swap(v, p0, p1);
      const int r = 16 * i + 4 * pl.quad + (odd ? 2 : 0);
      *reinterpret_cast<unsigned*>(tr + place(r, col >> 3) + (col & 7) * 2) = p0;
      *reinterpret_cast<unsigned*>(tr + place(r + 1, col >> 3) + (col & 7) * 2) = p1;
    };
    auto store_rows = [&](int units) {  // the transposed tile's rows to qt, from unit `units` of them
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the wave's own part of LDS)
#pragma unroll 4
      for (int k = 0; k < RA / 8; ++k) {
        const int r = 8 * k + (lane >> 3), v = pl.a0 + r, piece = lane & 7;
        const u32x4 x = *reinterpret_cast<const u32x4*>(tr + place(r, piece));
        if (v < l.V && units + 8 * piece < ldqt) *reinterpret_cast<u32x4*>(qt + (size_t)v * ldqt + units + 8 * piece) = x;
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    float gn[T::NB];
    int t[T::NB];
    auto less_lse = [&](int j) {  // acc: log p (p is 0 in a row without a target, whatever it holds)
      const int n = pl.b0 + 16 * j + pl.n;
      const int yn = n < l.N ? l.y[n] : -1;
      const bool ok = yn >= 0 && yn < l.V_all;
      const float ln = ok ? lse[n] : 0.f;
      gn[j] = ok ? g[n] : 0.f;
      t[j] = ok && yn - l.v0 < l.V ? yn - l.v0 : -1;
#pragma unroll
      for (int i = 0; i < T::NA; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = ok ? acc[i][j][e] - ln : -INFINITY;
    };
    f32x4 by[SP ? T::NA : 1];
    if constexpr (SP) {
#pragma unroll
      for (int j = 0; j < T::NB; ++j) less_lse(j);
      if (qt) class_scales<T>(acc, pl, lds, by);
    }
#pragma unroll
    for (int j = 0; j < T::NB; ++j) {
      if constexpr (!SP) less_lse(j);
#pragma unroll
      for (int i = 0; i < T::NA; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = wnk::expf_fast(acc[i][j][e]);
      Logits::at_target<T>(pl, t[j], [&](int i, int e) { acc[i][j][e] -= 1.f; });
      const int n = pl.b0 + 16 * j + pl.n;
      const float gh = most != 0.f ? gn[j] / most : gn[j];  // (1 where all rows weigh alike; a NaN, which max |g| passes over, stays)
#pragma unroll
      for (int i = 0; i < T::NA; ++i) {
        const int v = pl.a0 + 16 * i + 4 * pl.quad;
        const f32x4 p = acc[i][j];
        acc[i][j] = p * gn[j];
        if constexpr (SP) {
          u16 hi[4], lo[4];
          if (q && n < l.N && v < ldq / 2) {
#pragma unroll
            for (int e = 0; e < 4; ++e) split(p[e] * (1 << kQScale), hi[e], lo[e]);
            u16* d = q + (size_t)n * ldq + v / 32 * kChunk + v % 32;
            *reinterpret_cast<u32x2*>(d) = u32x2{(unsigned)hi[0] | (unsigned)hi[1] << 16, (unsigned)hi[2] | (unsigned)hi[3] << 16};
            *reinterpret_cast<u32x2*>(d + 32) = u32x2{(unsigned)lo[0] | (unsigned)lo[1] << 16, (unsigned)lo[2] | (unsigned)lo[3] << 16};
          }
          if (qt) {
#pragma unroll
            for (int e = 0; e < 4; ++e) split(p[e] * by[i][e], hi[e], lo[e]);
            put_pair(i, 16 * (j & 1) + (pl.n & ~1), hi);
            put_pair(i, 32 + 16 * (j & 1) + (pl.n & ~1), lo);
          }
        } else {
          if (q && n < l.N && v < ldq)
            *reinterpret_cast<u32x2*>(q + (size_t)n * ldq + v) = u32x2{bf16_pair(p[0], p[1]), bf16_pair(p[2], p[3])};
          if (qt) {
            u16 h[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = bf16_bits(p[e] * gh);
            put_pair(i, 16 * j + (pl.n & ~1), h);
          }
        }
      }
      if (SP && qt && j & 1) store_rows((pl.b0 + 16 * (j - 1)) * 2);
    }
    if (!SP && qt) store_rows(pl.b0);
    if (!db) return;
    __syncthreads();
    float* const s = reinterpret_cast<float*>(lds);  // [WB][TA]
#pragma unroll
    for (int i = 0; i < T::NA; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < T::NB; ++j) sum += acc[i][j][e];
        sum = wnk::gsum16(sum);
        if (pl.n == 0) s[pl.wb * T::TA + pl.wa * (T::TA / T::WA) + 16 * i + 4 * pl.quad + e] = sum;
      }
    __syncthreads();
    for (int k = threadIdx.x; k < T::TA; k += T::kThreads) {
      const int v = pl.ta * T::TA + k;
      float sum = s[k];
#pragma unroll
      for (int w = 1; w < T::WB; ++w) sum += s[w * T::TA + k];
      if (v < l.V) db[(size_t)pl.tb * l.V + v] = sum;
    }
  }
};

// dx and dw: out[b][a] (rows of D).  DW in fp32: operand B's scales change from tile to tile of k.
template <class E, bool DW>
struct OutEnd {
  static constexpr bool kScaledByTile = sizeof(E) == 4 && DW;
  int A, B;           // D, rows
  const int* ea;      // fp32: scales of operand A's rows; the product is acc 2^-(ea[a] + eb)
  const int* eq;      // fp32 dw: eb of each tile of k, [tiles][B] (dx: kQScale)
  int tile;           // log2 of its chunks
  const int32_t* y;   // dx: rows whose y is outside 0 .. V-1 are 0; or null
  const float* g;     // dx: the row's factor; or null
  const float* gmax;  // bf16 dw: parts of the factor of all (largest_g); or null
  int gparts;
  int V;
  float* sum;         // [splits][B][A], set (add = 0) or added to; or null
  int add;
  E* out;             // where sum is null
  // The sums before chunk c in the units of its tile, where it is the first of one.
  template <class T>
  __device__ __forceinline__ void to_chunk(f32x4 (&acc)[T::NA][T::NB], const Place& pl, int c) const {
    if (c & ((1 << tile) - 1)) return;
    const int* now = eq + (size_t)(c >> tile) * B;
#pragma unroll
    for (int j = 0; j < T::NB; ++j) {
      const int b = min(pl.b0 + 16 * j + pl.n, B - 1);
      const float f = __uint_as_float((unsigned)(127 + now[b] - (now - B)[b]) << 23);  // (at most 2^66 either way)
#pragma unroll
      for (int i = 0; i < T::NA; ++i) acc[i][j] *= f;
    }
  }
  template <class T>
  __device__ void operator()(f32x4 (&acc)[T::NA][T::NB], const Place& pl, char*) const {
    if constexpr (sizeof(E) == 4) {
      int eb[T::NB];
#pragma unroll
      for (int j = 0; j < T::NB; ++j) eb[j] = kScaledByTile ? eq[(size_t)(pl.last >> tile) * B + min(pl.b0 + 16 * j + pl.n, B - 1)] : kQScale;
#pragma unroll
      for (int i = 0; i < T::NA; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int s = ea[min(pl.a0 + 16 * i + 4 * pl.quad + e, A - 1)];
#pragma unroll
          for (int j = 0; j < T::NB; ++j) acc[i][j][e] = ldexpf(acc[i][j][e], -(s + eb[j]));
        }
    }
    const float all = gmax ? join_largest(gmax, gparts) : 1.f;
#pragma unroll
    for (int j = 0; j < T::NB; ++j) {
      const int b = pl.b0 + 16 * j + pl.n;
      const bool in = b < B;
      float f = all;
      bool ok = true;
      if (y) {
        const int yb = in ? y[b] : -1;
        ok = yb >= 0 && yb < V;
        if (g && ok) f = g[b];
      }
#pragma unroll
      for (int i = 0; i < T::NA; ++i) {
        const int a = pl.a0 + 16 * i + 4 * pl.quad;
        f32x4 v = acc[i][j] * f;
        if (!ok) v = f32x4{0.f, 0.f, 0.f, 0.f};
        if (!in) continue;
        if (sum) {
          float* d = sum + ((size_t)pl.split * B + b) * A + a;
          if (a + 3 < A) {
            if (add) {
              const f32x4u o = *reinterpret_cast<const f32x4u*>(d);
              v += f32x4{o[0], o[1], o[2], o[3]};
            }
            *reinterpret_cast<f32x4u*>(d) = f32x4u{v[0], v[1], v[2], v[3]};
          } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
              if (a + e < A) d[e] = add ? d[e] + v[e] : v[e];
          }
        } else {
          E* d = out + (size_t)b * A + a;
          if (a + 3 < A) {
            if constexpr (sizeof(E) == 4) *reinterpret_cast<f32x4u*>(d) = f32x4u{v[0], v[1], v[2], v[3]};
            else *reinterpret_cast<u16x4u*>(d) = u16x4u{bf16_bits(v[0]), bf16_bits(v[1]), bf16_bits(v[2]), bf16_bits(v[3])};
          } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
              if (a + e < A) put(d + e, v[e]);
          }
        }
      }
    }
  }
};

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

// A row of x counts in the sums over rows by its factor: g (fp32 arrays) or 1; not at all without a target.
struct RowFactor {
  const int32_t* y;  // null: every row counts
  const float* g;    // null: factor 1
  int V;
  __device__ bool ok(int r) const { return !y || (y[r] >= 0 && y[r] < V); }
  __device__ float factor(int r) const { return g ? g[r] : 1.f; }
};

// Largest magnitudes of the columns of [R][K], over the rows of blockIdx.y's run: part[blockIdx.y][K].
__global__ __launch_bounds__(256) void column_max(const float* src, int R, int K, int run, RowFactor f, float* part) {
  __shared__ f32x4 s[16][16];
  const int c = threadIdx.x & 15, w = threadIdx.x >> 4, k = blockIdx.x * 64 + 4 * c;
  const int r0 = blockIdx.y * run, r1 = min(R, r0 + run);
  f32x4 m{0.f, 0.f, 0.f, 0.f};
  if (k < K)
#pragma unroll 4
    for (int r = r0 + w; r < r1; r += 16) {
      const f32x4 v = four(src + (size_t)r * K, k, K);
      const float g = f.ok(r) ? f.factor(r) : 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) m[e] = fmaxf(m[e], g == 0.f ? 0.f : fabsf(v[e] * g));
    }
  s[w][c] = m;
  __syncthreads();
  if (threadIdx.x < 64 && blockIdx.x * 64 + threadIdx.x < K) {
    float v = 0.f;
    for (int i = 0; i < 16; ++i) v = fmaxf(v, s[i][threadIdx.x >> 2][threadIdx.x & 3]);
    part[(size_t)blockIdx.y * K + blockIdx.x * 64 + threadIdx.x] = v;
  }
}

// The columns of [R][K] as rows: dst[k][r], 64 x 64 values per block.
__global__ __launch_bounds__(256) void pack_cols(const float* src, int R, int K, RowFactor f, u16* dst, int units, const float* part,
                                                 int parts, int* scale) {
  __shared__ float s[64][65];
  __shared__ int se[64];
  const int tid = threadIdx.x, k0 = blockIdx.x * 64, r0 = blockIdx.y * 64;
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    const int i = 16 * h + (tid >> 4), c = 4 * (tid & 15), r = r0 + i;
    f32x4 v{0.f, 0.f, 0.f, 0.f};
    if (r < R && f.ok(r)) {
      v = four(src + (size_t)r * K, k0 + c, K) * f.factor(r);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) s[i][c + e] = v[e];
  }
  {
    const int k = k0 + (tid >> 2);
    float m = 0.f;
    if (k < K)
      for (int i = tid & 3; i < parts; i += 4) m = fmaxf(m, part[(size_t)i * K + k]);
    m = fmaxf(m, wnk::dpp<0xB1>(m));
    m = fmaxf(m, wnk::dpp<0x4E>(m));
    if ((tid & 3) == 0) {
      se[tid >> 2] = scale_of(m);
      if (blockIdx.y == 0 && k < K) scale[k] = se[tid >> 2];
    }
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    const int i = 16 * h + (tid >> 4), c = 4 * (tid & 15);
    if (k0 + i >= K || r0 + c >= units / 2) continue;
    put_split(dst + (size_t)(k0 + i) * units, r0 + c, scaled(f32x4{s[c][i], s[c + 1][i], s[c + 2][i], s[c + 3][i]}, se[i]));
  }
}
__global__ __launch_bounds__(256) void pack_cols(const u16* src, int R, int K, RowFactor f, u16* dst, int units) {
  __shared__ __align__(16) u16 s[64][72];  // [k][r]
  typedef u16 u16x8u __attribute__((ext_vector_type(8), aligned(2)));
  const int tid = threadIdx.x, k0 = blockIdx.x * 64, r0 = blockIdx.y * 64;
  // a thread reads 8 columns of two neighbouring rows and writes pairs
  {
    const int c = 8 * (tid & 7), i = 2 * (tid >> 3), k = k0 + c;
    u16 v[2][8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = r0 + i + h;
      const bool on = r < R && f.ok(r);
      const u16* p = src + (size_t)r * K + k;
      if (on && k + 7 < K) {
        const u16x8u x = *reinterpret_cast<const u16x8u*>(p);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[h][e] = x[e];
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[h][e] = on && k + e < K ? p[e] : (u16)0;
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) *reinterpret_cast<unsigned*>(&s[c + e][i]) = (unsigned)v[0][e] | (unsigned)v[1][e] << 16;
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = 32 * h + (tid >> 3), c = 8 * (tid & 7);
    if (k0 + i < K && r0 + c < units)
      *reinterpret_cast<u32x4*>(dst + (size_t)(k0 + i) * units + r0 + c) = *reinterpret_cast<const u32x4*>(&s[i][c]);
  }
}

// ------------------------------------------------------------------------------------------------
// Joins
// ------------------------------------------------------------------------------------------------
// lse and loss of a row from its tiles' (largest, sum): 16 rows by 16 runs of tiles per block.
__global__ __launch_bounds__(256) void join_loss(const float2* part, int tiles, const float* target, const int32_t* y,
                                                 int N, int V, float* loss, float* lse) {
  __shared__ float2 s[16][16];
  const int c = threadIdx.x & 15, w = threadIdx.x >> 4, n = blockIdx.x * 16 + c;
  float m = -INFINITY, sum = 0.f;
  if (n < N)
    for (int t = w; t < tiles; t += 16) {
      const float2 p = part[(size_t)t * N + n];
      const float top = fmaxf(m, p.x), at = top == -INFINITY ? 0.f : top;
      sum = sum * wnk::expf_fast(m - at) + p.y * wnk::expf_fast(p.x - at);
      m = top;
    }
  s[w][c] = make_float2(m, sum);
  __syncthreads();
  if (w || n >= N) return;
  for (int k = 1; k < 16; ++k) {
    const float2 p = s[k][c];
    const float top = fmaxf(m, p.x), at = top == -INFINITY ? 0.f : top;
    sum = sum * wnk::expf_fast(m - at) + p.y * wnk::expf_fast(p.x - at);
    m = top;
  }
  const float z = logf(sum);
  lse[n] = m + z;  // (no class at all: -inf)
  const int t = y[n];
  loss[n] = t >= 0 && t < V ? m - target[n] + z : 0.f;  // (in this order log(sum) is not lost beside a large m)
}

// The same for few rows: a block per row.
__global__ __launch_bounds__(256) void join_loss_few(const float2* part, int tiles, const float* target, const int32_t* y, int N,
                                                     int V, float* loss, float* lse) {
  __shared__ float2 s[4];
  const int n = blockIdx.x;
  float2 a{-INFINITY, 0.f};
  auto add = [&](float2 p) {
    const float top = fmaxf(a.x, p.x), at = top == -INFINITY ? 0.f : top;
    a = make_float2(top, a.y * wnk::expf_fast(a.x - at) + p.y * wnk::expf_fast(p.x - at));
  };
#pragma unroll 4
  for (int t = threadIdx.x; t < tiles; t += 256) add(part[(size_t)t * N + n]);
  for (int d = 32; d; d >>= 1) add(make_float2(__shfl_xor(a.x, d, 64), __shfl_xor(a.y, d, 64)));
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = a;
  __syncthreads();
  if (threadIdx.x) return;
  for (int w = 1; w < 4; ++w) add(s[w]);
  const float z = logf(a.y);
  lse[n] = a.x + z;
  const int t = y[n];
  loss[n] = t >= 0 && t < V ? a.x - target[n] + z : 0.f;
}

// out[i] = sum over the parts: 64 places of four values by 4 runs of parts per block, then the runs in order.
// With y the values are rows of D that take the factors g, and those without a target are 0 whatever the parts hold.
template <class E>
__global__ __launch_bounds__(256) void join_parts(const float* part, int parts, size_t n, E* out, const int32_t* y, int V, unsigned D, const float* g) {
  __shared__ f32x4 s[3][64];
  const int c = threadIdx.x & 63, w = threadIdx.x >> 6, each = (parts + 3) / 4;
  const size_t i = ((size_t)block_of_many() * 64 + c) * 4;
  f32x4 v{0.f, 0.f, 0.f, 0.f};
  if (i + 3 < n) {
#pragma unroll 8
    for (int k = w * each; k < min(parts, (w + 1) * each); ++k) {
      const f32x4u x = *reinterpret_cast<const f32x4u*>(part + k * n + i);
      v += f32x4{x[0], x[1], x[2], x[3]};
    }
  } else if (i < n) {
    for (int k = w * each; k < min(parts, (w + 1) * each); ++k)
      for (int e = 0; e < 3; ++e)
        if (i + e < n) v[e] += part[k * n + i + e];
  }
  if (w) s[w - 1][c] = v;
  __syncthreads();
  if (w || i >= n) return;
  v = ((v + s[0][c]) + s[1][c]) + s[2][c];
  if (y) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const unsigned r = (unsigned)(i + e) / D;
      const int t = i + e < n ? y[r] : -1;
      v[e] = t < 0 || t >= V ? 0.f : v[e] * g[r];
    }
  }
  if (i + 3 < n) {
    if constexpr (sizeof(E) == 4) *reinterpret_cast<f32x4u*>(out + i) = f32x4u{v[0], v[1], v[2], v[3]};
    else *reinterpret_cast<u16x4u*>(out + i) = u16x4u{bf16_bits(v[0]), bf16_bits(v[1]), bf16_bits(v[2]), bf16_bits(v[3])};
  } else {
    for (int e = 0; e < 3; ++e)
      if (i + e < n) put(out + i + e, v[e]);
  }
}

template <class E>
__global__ __launch_bounds__(256) void fill_zero(E* out, size_t n) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) out[i] = (E)0;
}

// ------------------------------------------------------------------------------------------------
// Host
// ------------------------------------------------------------------------------------------------
constexpr size_t kForwardPiece = (size_t)64 << 20;    // bytes of packed w in the forward pass
constexpr size_t kBackwardPiece = (size_t)1 << 30;   // bytes of w's forms and q in the backward pass
constexpr int kMaxN = 1 << 20, kMaxD = 1 << 16, kMaxV = 1 << 24;
constexpr size_t kSplitFloats = (size_t)64 << 20;     // values of a product's parts, at most
constexpr int kColumnParts = 64;  // of column_max

bool sizes_ok(int dtype, int N, int D, int V) {
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
Shape shape_for(size_t a, size_t b, int units, bool sp, bool may_split) {
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
int forward_piece(int N, int V, size_t each) {
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

// The workspace's parts, with room for every form that a call with these sizes may take.
struct Forward {
  int piece;  // classes
  size_t part, target, x, ex, w, ew, total;
  Forward(bool sp, int N, int D, int V) {
    const size_t units = padded_units(D, sp);
    Carve c;
    if (N <= kFewRows) {
      part = c.take(ceil_div(V, wn_few_classes(sp, N, D, V)) * N * sizeof(float2));
      target = c.take((size_t)N * 4);
      total = c.at;
      return;
    }
    piece = forward_piece(N, V, units * 2 + 4);
    part = c.take(ceil_div(V, 128) * N * sizeof(float2));
    target = c.take((size_t)N * 4);
    x = c.take((size_t)N * units * 2);
    ex = c.take((size_t)N * 4);
    w = c.take(piece * units * 2);
    ew = c.take((size_t)piece * 4);
    total = c.at;
  }
};

struct Backward {
  int piece;
  Shape logits, dxs, dws;  // of a whole piece
  size_t x, ex, xt, ext, w, ew, wt, ewt, q, qt, eq, db, cmax, gmax, dx, dw, total;
  WnFewPlan few;
  void plan(bool sp, int N, int D, int p) {
    piece = p;
    logits = shape_for(p, N, padded_units(D, sp), sp, false);
    dxs = shape_for(D, N, padded_units(p, sp), sp, true);
    dws = shape_for(D, p, padded_units(N, sp), sp, true);
  }
  Backward(bool sp, int N, int D, int V) {
    if (N <= kFewRows) {
      few = wn_few_plan(sp, N, D, V);
      Carve c;
      q = c.take(few.q_bytes);
      qt = c.take(few.qt_bytes);
      dx = c.take(few.sum_bytes);
      total = c.at;
      return;
    }
    const size_t ud = padded_units(D, sp), un = padded_units(N, sp), e = sp ? 4 : 2;
    const size_t each = ud * 2 + D * e + 2 * un * 2;
    // pieces alike, the fewest that fit and a few more, or of whole rounds of the products' tiles: the fastest by the model
    const size_t most = std::min<size_t>(V, std::max<size_t>(256, kBackwardPiece / each / 256 * 256)), fewest = ceil_div(V, most);
    const size_t round = 256 * std::max<size_t>(1, 256 / ceil_div(D, 256));
    double best = 1e30;
    int at = (int)most;
    for (int c = 0; c < 5; ++c) {
      size_t p = c < 4 ? std::min<size_t>(V, ceil_div(ceil_div(V, fewest + c), 256) * 256) : most / round * round;
      if (p == 0 || p > most) continue;
      plan(sp, N, D, (int)p);
      const double us = (logits.us + dxs.us + dws.us + 10) * (double)V / (double)p;
      if (us < best * 0.999) {
        best = us;
        at = (int)p;
      }
      if (fewest == 1) break;
    }
    plan(sp, N, D, at);
    const size_t uv = padded_units(piece, sp);
    Carve c;
    x = c.take((size_t)N * ud * 2);
    ex = c.take((size_t)N * 4);
    xt = c.take((size_t)D * un * 2);
    ext = c.take((size_t)D * 4);
    w = c.take((size_t)piece * ud * 2);
    ew = c.take((size_t)piece * 4);
    wt = c.take((size_t)D * uv * 2);
    ewt = c.take((size_t)D * 4);
    q = c.take((size_t)N * uv * 2);
    qt = c.take((size_t)piece * un * 2);
    eq = c.take(sp ? ceil_div(N, 128) * piece * 4 : 0);
    db = c.take(ceil_div(N, 128) * piece * 4);
    cmax = c.take((size_t)kColumnParts * D * 4);
    gmax = c.take(kGParts * 4);
    dx = c.take(piece == V && dxs.splits == 1 ? 0 : (size_t)dxs.splits * N * D * 4);
    dw = c.take(dws.splits == 1 ? 0 : (size_t)dws.splits * piece * D * 4);
    total = c.at;
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

template <class E>
Operand cols_operand(const E* src, int R, int K, const RowFactor& f, u16* dst, float* part, int* scale, hipStream_t st) {
  constexpr bool sp = sizeof(E) == 4;
  const int units = padded_units(R, sp);
  const dim3 grid((unsigned)ceil_div(K, 64), (unsigned)ceil_div(R, 64));
  if constexpr (sp) {
    const int run = (int)ceil_div(R, std::min<size_t>(kColumnParts, ceil_div(R, 64))), parts = (int)ceil_div(R, run);
    hipLaunchKernelGGL(column_max, dim3(grid.x, parts), dim3(256), 0, st, src, R, K, run, f, part);
    hipLaunchKernelGGL(static_cast<void (*)(const float*, int, int, RowFactor, u16*, int, const float*, int, int*)>(pack_cols), grid,
                       dim3(256), 0, st, src, R, K, f, dst, units, part, parts, scale);
  } else {
    hipLaunchKernelGGL(static_cast<void (*)(const u16*, int, int, RowFactor, u16*, int)>(pack_cols), grid, dim3(256), 0, st, src, R, K,
                       f, dst, units);
  }
  return {dst, K, units, units};
}

template <class E>
int run_forward(int N, int D, int V, const E* x, const E* w, const float* b, const int32_t* y, float* loss, float* lse,
                char* ws, hipStream_t st) {
  constexpr bool sp = sizeof(E) == 4;
  const Forward f(sp, N, D, V);
  if (N <= kFewRows) {
    float2* const part = reinterpret_cast<float2*>(ws + f.part);
    float* const target = reinterpret_cast<float*>(ws + f.target);
    hipError_t e = wn_few_loss<E>({N, D, V, x, w, b, y}, part, target, st);
    if (e == hipSuccess) {
      hipLaunchKernelGGL(join_loss_few, dim3(N), dim3(256), 0, st, part, (int)ceil_div(V, wn_few_classes(sp, N, D, V)), target, y, N, V, loss, lse);
      e = hipGetLastError();
    }
    return e == hipSuccess ? WN_OK : wn_set_last_error(WN_EHIP, hipGetErrorString(e));
  }
  int* const ex = reinterpret_cast<int*>(ws + f.ex);
  int* const ew = reinterpret_cast<int*>(ws + f.ew);
  u16* const wp = reinterpret_cast<u16*>(ws + f.w);
  RowPacker<E> pack;
  const Operand ox = pack.add(x, N, D, reinterpret_cast<u16*>(ws + f.x), ex);
  const bool direct = !sp && D % 8 == 0 && reinterpret_cast<uintptr_t>(w) % 16 == 0;
  const int piece = direct ? forward_piece(N, V, 0) : f.piece;
  int tiles = 0;
  for (int v0 = 0; v0 < V; v0 += piece) {
    const int n = std::min(piece, V - v0);
    const Operand ow = pack.add(w + (size_t)v0 * D, n, D, wp, ew);
    pack.launch(st);
    const bool big = shape_for(n, N, ox.k, sp, false).big;
    StatsEnd end{{sp ? ex : nullptr, sp ? ew : nullptr, b ? b + v0 : nullptr, y, N, n, v0, V},
                 reinterpret_cast<float2*>(ws + f.part), tiles, reinterpret_cast<float*>(ws + f.target)};
    const hipError_t e = run_product<sp>({ow, ox, 0, 0, 1, 0}, big, end, st);
    if (e != hipSuccess) return wn_set_last_error(WN_EHIP, hipGetErrorString(e));
    tiles += (int)ceil_div(n, big ? 256 : 128);
  }
  hipLaunchKernelGGL(join_loss, dim3((unsigned)ceil_div(N, 16)), dim3(256), 0, st, reinterpret_cast<const float2*>(ws + f.part),
                     tiles, reinterpret_cast<const float*>(ws + f.target), y, N, V, loss, lse);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? WN_OK : wn_set_last_error(WN_EHIP, hipGetErrorString(e));
}

template <class E>
hipError_t join(const float* part, int parts, size_t n, E* out, hipStream_t st, const int32_t* y = nullptr, int V = 0, int D = 1,
                const float* g = nullptr) {
  hipLaunchKernelGGL(join_parts<E>, many_blocks(ceil_div(n, 256)), dim3(256), 0, st, part, parts, n, out, y, V, (unsigned)D, g);
  return hipGetLastError();
}

template <class E>
int run_backward(int N, int D, int V, const E* x, const E* w, const float* b, const int32_t* y, const float* lse,
                 const float* g, E* dx, E* dw, float* db, char* ws, hipStream_t st) {
  constexpr bool sp = sizeof(E) == 4;
  const Backward f(sp, N, D, V);
  auto ints = [&](size_t off) { return reinterpret_cast<int*>(ws + off); };
  auto units = [&](size_t off) { return reinterpret_cast<u16*>(ws + off); };
  auto floats = [&](size_t off) { return reinterpret_cast<float*>(ws + off); };
  if (N <= kFewRows) {
    hipError_t e = wn_few_grads<E>({N, D, V, x, w, b, y}, f.few, lse, g, dx != nullptr, dw, db, ws + f.q, ws + f.qt, floats(f.dx), st);
    if (e == hipSuccess && dx) e = join(floats(f.dx), f.few.parts, (size_t)N * D, dx, st, y, V, D, g);
    return e == hipSuccess ? WN_OK : wn_set_last_error(WN_EHIP, hipGetErrorString(e));
  }
  RowPacker<E> pack;
  const Operand ox = pack.add(x, N, D, units(f.x), ints(f.ex));
  Operand oxt{};
  const float* gmax = nullptr;
  const int gparts = (int)std::min<size_t>(kGParts, ceil_div(N, 1024));
  if (dw && !sp) {
    hipLaunchKernelGGL(largest_g, dim3(gparts), dim3(256), 0, st, g, y, N, V, floats(f.gmax));
    gmax = floats(f.gmax);
  }
  if (dw) oxt = cols_operand(x, N, D, RowFactor{y, sp ? g : nullptr, V}, units(f.xt), floats(f.cmax), ints(f.ext), st);
  hipError_t e = hipGetLastError();
  for (int v0 = 0; v0 < V && e == hipSuccess; v0 += f.piece) {
    const int n = std::min(f.piece, V - v0);
    const E* wv = w + (size_t)v0 * D;
    const int ldq = padded_units(n, sp), ldqt = padded_units(N, sp);
    const Operand ow = pack.add(wv, n, D, units(f.w), ints(f.ew));
    pack.launch(st);
    const bool big = f.logits.big;
    GradEnd<sp> end{{sp ? ints(f.ex) : nullptr, sp ? ints(f.ew) : nullptr, b ? b + v0 : nullptr, y, N, n, v0, V},
                    lse, g, gmax, gparts, dx ? units(f.q) : nullptr, dw ? units(f.qt) : nullptr, ldq, ldqt,
                    ints(f.eq), db ? floats(f.db) : nullptr};
    e = run_product<sp>({ow, ox, 0, 0, 1, 0}, big, end, st);
    if (e == hipSuccess && db) e = join(floats(f.db), (int)ceil_div(N, big ? 256 : 128), n, db + v0, st);
    if (e == hipSuccess && dx) {
      const Operand owt = cols_operand(wv, n, D, RowFactor{nullptr, nullptr, 0}, units(f.wt), floats(f.cmax), ints(f.ewt), st);
      const bool whole = f.piece == V && f.dxs.splits == 1;
      const OutEnd<E, false> o{D, N, ints(f.ewt), nullptr, 0, y, g, nullptr, 0, V, whole ? nullptr : floats(f.dx), v0 > 0, dx};
      e = run_product<sp>({owt, {units(f.q), N, ldq, ldq}, 0, 0, f.dxs.splits, 0}, f.dxs.big, o, st);
      if (e == hipSuccess && !whole && v0 + n == V) e = join(floats(f.dx), f.dxs.splits, (size_t)N * D, dx, st);
    }
    if (e == hipSuccess && dw) {
      E* const out = dw + (size_t)v0 * D;
      const OutEnd<E, true> o{D, n, ints(f.ext), sp ? ints(f.eq) : nullptr, big ? 3 : 2, nullptr, nullptr, gmax, gparts, 1, f.dws.splits == 1 ? nullptr : floats(f.dw), 0, out};
      e = run_product<sp>({oxt, {units(f.qt), n, ldqt, ldqt}, 0, 0, f.dws.splits, 0}, f.dws.big, o, st);
      if (e == hipSuccess && f.dws.splits > 1) e = join(floats(f.dw), f.dws.splits, (size_t)n * D, out, st);
    }
  }
  return e == hipSuccess ? WN_OK : wn_set_last_error(WN_EHIP, hipGetErrorString(e));
}

int check_sizes(int dtype, int N, int D, int V) {
  const int rc = bad_dtype(dtype);
  if (rc != WN_OK) return rc;
  return sizes_ok(dtype, N, D, V) ? WN_OK : wn_set_last_error(WN_EINVAL, "N must be 0..2^20, D 1..2^16, V 1..2^24");
}

}  // namespace

extern "C" {

size_t wn_loss_workspace_bytes(int32_t dtype, int32_t N, int32_t D, int32_t V) {
  if (!sizes_ok(dtype, N, D, V) || N == 0) return 0;
  return Forward(dtype == WN_F32, N, D, V).total;
}

size_t wn_loss_backward_workspace_bytes(int32_t dtype, int32_t N, int32_t D, int32_t V) {
  if (!sizes_ok(dtype, N, D, V) || N == 0) return 0;
  return Backward(dtype == WN_F32, N, D, V).total;
}

int wn_loss(int32_t dtype, int32_t N, int32_t D, int32_t V, const void* x, const void* w, const float* b, const int32_t* y,
            float* loss, float* lse, void* workspace, size_t ws_bytes, void* stream) {
  wn_clear_last_error();
  int rc = check_sizes(dtype, N, D, V);
  if (rc != WN_OK || N == 0) return rc;
  if (!x || !w || !y || !loss || !lse) return wn_set_last_error(WN_EINVAL, "null pointer");
  rc = bad_workspace(workspace, ws_bytes, wn_loss_workspace_bytes(dtype, N, D, V));
  if (rc != WN_OK) return rc;
  ArrayScope scope;
  const struct { const void* p; const char* name; } arrays[] = {{x, "x"}, {w, "w"}, {b, "b"}, {y, "y"}, {loss, "loss"},
                                                                {lse, "lse"}, {workspace, "workspace"}};
  for (const auto& a : arrays)
    if (a.p && (rc = scope.check(a.p, a.name)) != WN_OK) return rc;
  if ((rc = scope.enter()) != WN_OK) return rc;
  char* const ws = static_cast<char*>(workspace);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == WN_F32)
    return run_forward(N, D, V, static_cast<const float*>(x), static_cast<const float*>(w), b, y, loss, lse, ws, st);
  return run_forward(N, D, V, static_cast<const u16*>(x), static_cast<const u16*>(w), b, y, loss, lse, ws, st);
}

int wn_loss_backward(int32_t dtype, int32_t N, int32_t D, int32_t V, const void* x, const void* w, const float* b,
                     const int32_t* y, const float* lse, const float* g, void* dx, void* dw, float* db, void* workspace,
                     size_t ws_bytes, void* stream) {
  wn_clear_last_error();
  int rc = check_sizes(dtype, N, D, V);
  if (rc != WN_OK) return rc;
  if (!dx && !dw && !db) return wn_set_last_error(WN_EINVAL, "no gradient is wanted");
  if (N > 0 && (!x || !w || !y || !lse || !g)) return wn_set_last_error(WN_EINVAL, "null pointer");
  if (N == 0 && !dw && !db) return WN_OK;
  rc = bad_workspace(workspace, ws_bytes, wn_loss_backward_workspace_bytes(dtype, N, D, V));
  if (rc != WN_OK) return rc;
  ArrayScope scope;
  const struct { const void* p; const char* name; } arrays[] = {
      {N ? x : nullptr, "x"}, {N ? w : nullptr, "w"}, {N ? b : nullptr, "b"}, {N ? y : nullptr, "y"}, {N ? lse : nullptr, "lse"},
      {N ? g : nullptr, "g"}, {N ? dx : nullptr, "dx"}, {dw, "dw"}, {db, "db"}, {N ? workspace : nullptr, "workspace"}};
  for (const auto& a : arrays)
    if (a.p && (rc = scope.check(a.p, a.name)) != WN_OK) return rc;
  if ((rc = scope.enter()) != WN_OK) return rc;
  char* const ws = static_cast<char*>(workspace);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (N == 0) {
    if (dw && dtype == WN_F32) hipLaunchKernelGGL(fill_zero<float>, dim3(1024), dim3(256), 0, st, static_cast<float*>(dw), (size_t)V * D);
    if (dw && dtype == WN_BF16) hipLaunchKernelGGL(fill_zero<u16>, dim3(1024), dim3(256), 0, st, static_cast<u16*>(dw), (size_t)V * D);
    if (db) hipLaunchKernelGGL(fill_zero<float>, dim3(1024), dim3(256), 0, st, db, (size_t)V);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? WN_OK : wn_set_last_error(WN_EHIP, hipGetErrorString(e));
  }
  if (dtype == WN_F32)
    return run_backward(N, D, V, static_cast<const float*>(x), static_cast<const float*>(w), b, y, lse, g,
                        static_cast<float*>(dx), static_cast<float*>(dw), db, ws, st);
  return run_backward(N, D, V, static_cast<const u16*>(x), static_cast<const u16*>(w), b, y, lse, g, static_cast<u16*>(dx),
                      static_cast<u16*>(dw), db, ws, st);
}

}  // extern "C"
