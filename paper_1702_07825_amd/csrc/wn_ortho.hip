// Updates orthogonalised by Newton-Schulz products (gfx950).  Declarations and contracts are in include/wn_train.h.
//
// Each matrix is X [m][n] with m <= n (a taller one transposed), its Frobenius norm at most 1.  A step is
//   A = X X',  B = a I + b A + c A A,  X <- B X
// three products of 16-bit operands on wn_product.h's tiles, all matrices of a call in one launch each.  A and B are symmetric:
// their tiles on one side of the diagonal are computed and stored twice.  Both operands of a product lie along its sum, so
// X is kept in both orders (the end of a step writes both).
//
// Values are held as fp16 of a power of two times themselves (kX, kA, kB): no entry exceeds its matrix's largest singular
// value, which starts at 1 or below and stays near 1.2 with the usual coefficients, so one scale serves all entries, and what
// fp16 cuts off (2^-37 of 1) is nothing beside the products' own rounding.  Matrices of bf16 take one fp16 value (2^-11 of
// itself, where their results are rounded to 2^-8), those of fp32 hi and lo parts and three products (2^-22).
#include "wn_product.h"

#include <cmath>
#include <new>
#include <vector>

namespace {

constexpr int kX = 12, kA = 12, kB = 10;  // X 2^kX and so on are held: up to 16, 16 and 64
constexpr int kMostSteps = 64, kMostSide = 1 << 18;
constexpr long long kMostElements = 1LL << 32;
constexpr size_t kGroupBytes = (size_t)4 << 30;  // of the matrices that go through the steps together

// (small products are a chain of a few chunks' loads: room for four)
using Tiny = Tile<64, 64, 2, 2, 4>;

// Addresses that kernels read from memory, as pointers that are known to lie in memory and not in LDS: through a pointer that
// could be either, accesses are slower and the waits for LDS wait for them too.
typedef unsigned long long Address;
template <class T>
__device__ __forceinline__ T* in_memory(Address p) {
  return (T*)(__attribute__((address_space(1))) T*)p;
}

struct Matrix {
  Address g, out;
  Address x, xt[2], a, b;  // X [m][ldn], its transpose [n][ldm] of this step and the next, A and B [m][ldm]
  int m, n, ldm, ldn;      // m <= n; units from row to row
  int tall;                // g is X transposed
  float scale;
  int chunk0, chunks;      // of the array's elements, for its norm
  long long chunk;         // elements of one
  int pack0, sym0, step0;  // first blocks of the packing, of the products that give A and B, and of the one that gives X
  int packs, syms, steps;
};
// Matrices of a group, in the workspace.  of[block] says which matrix a block works on; each tile of a product has its matrix by
// itself, as one load less stands before the operands' then (six small matrices 102.8 us and 101.9, 14 of width 333 156.3 and 155.0).
struct Group {
  Matrix* matrices;
  double* squares;
  int *of_chunk, *of_pack;
  Matrix *of_sym, *of_step;
};

// What a matrix is put together from: as many of a list as a launch's arguments hold (82 small ones take two launches of 4 us;
// as whole descriptors five, and a call 14 us longer).
struct Given {
  Address g, out, buffers;
  int rows, cols;
  float scale;
  int chunk0, pack0, sym0, step0;
};
constexpr int kBatch = 68;
struct Batch {
  Given given[kBatch];
  int first, sym_side, step_side;  // sides of the products' tiles
};
static_assert(sizeof(Batch) < 3900, "kernel arguments");

__host__ __device__ constexpr int tiles_of(int v, int side) { return (v + side - 1) / side; }
__host__ __device__ constexpr size_t bytes_of(int rows, int ld) { return ((size_t)rows * ld * 2 + 255) / 256 * 256; }
__host__ __device__ constexpr long long chunk_of(long long n) {
  const long long c = (n + 1024 * 8 - 1) / (1024 * 8) * 8;
  return c < 16384 ? 16384 : c;
}

__host__ __device__ inline Matrix matrix_of(const Given& v, bool sp, int sym_side, int step_side) {
  Matrix m;
  m.g = v.g, m.out = v.out, m.scale = v.scale;
  m.tall = v.rows > v.cols;
  m.m = m.tall ? v.cols : v.rows;
  m.n = m.tall ? v.rows : v.cols;
  const int values = chunk_values(sp);
  m.ldm = tiles_of(m.m, values) * kChunk;
  m.ldn = tiles_of(m.n, values) * kChunk;
  m.x = v.buffers;
  m.xt[0] = m.x + bytes_of(m.m, m.ldn);
  m.xt[1] = m.xt[0] + bytes_of(m.n, m.ldm);
  m.a = m.xt[1] + bytes_of(m.n, m.ldm);
  m.b = m.a + bytes_of(m.m, m.ldm);
  const long long all = (long long)m.m * m.n;
  m.chunk = chunk_of(all);
  m.chunk0 = v.chunk0, m.pack0 = v.pack0, m.sym0 = v.sym0, m.step0 = v.step0;
  m.chunks = (int)((all + m.chunk - 1) / m.chunk);
  m.packs = tiles_of(m.m, 64) * tiles_of(m.n, 64);
  const int t = tiles_of(m.m, sym_side);
  m.syms = t * (t + 1) / 2;
  m.steps = tiles_of(m.m, step_side) * tiles_of(m.n, step_side);
  return m;
}

// A block for each matrix of a batch.
template <class E>
__global__ __launch_bounds__(256) void put_matrices(const Batch batch, const Group g) {
  constexpr int kWords = sizeof(Matrix) / 8;
  static_assert(sizeof(Matrix) % 8 == 0, "words");
  __shared__ union { Matrix m; Address words[kWords]; } s;
  const int at = batch.first + blockIdx.x;
  if (threadIdx.x == 0) s.m = matrix_of(batch.given[blockIdx.x], sizeof(E) == 4, batch.sym_side, batch.step_side);
  __syncthreads();
  auto copies = [&](Matrix* to, int n) {
    for (int k = threadIdx.x; k < n * kWords; k += 256) reinterpret_cast<Address*>(to)[k] = s.words[k % kWords];
  };
  copies(g.matrices + at, 1);
  copies(g.of_sym + s.m.sym0, s.m.syms);
  copies(g.of_step + s.m.step0, s.m.steps);
  for (int k = threadIdx.x; k < s.m.chunks; k += 256) g.of_chunk[s.m.chunk0 + k] = at;
  for (int k = threadIdx.x; k < s.m.packs; k += 256) g.of_pack[s.m.pack0 + k] = at;
}

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double s[4];
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, 64);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// Squares in 64 bits: fp32 values neither overflow nor vanish.  A block for each chunk of a matrix.  Bound: reading them
// (26 bf16 matrices, 457 MB: 89 us, 5.1 TB/s).
template <class E>
__global__ __launch_bounds__(256) void squares(const Group g) {
  const Matrix& m = g.matrices[g.of_chunk[blockIdx.x]];
  const long long all = (long long)m.m * m.n, at = (blockIdx.x - m.chunk0) * m.chunk, end = at + m.chunk < all ? at + m.chunk : all;
  constexpr int W = Piece<E>::n;
  const E* p = in_memory<const E>(m.g);
  double sum[2] = {0.0, 0.0};
  auto add = [&](const P<E>& v) {
#pragma unroll
    for (int e = 0; e < W; ++e) {
      const double d = value(v[e]);
      sum[e & 1] += d * d;
    }
  };
  constexpr int kAhead = 8;
  long long i = at + threadIdx.x * W;
  for (; i + 256 * W * (kAhead - 1) + W <= end; i += 256 * W * kAhead) {
    P<E> v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) v[k] = whole_piece(p + i + 256 * W * k);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) add(v[k]);
  }
  for (; i < end; i += 256 * W) add(piece_at(p + i, (int)(end - i < W ? end - i : W)));
  const double s = block_sum(sum[0] + sum[1]);
  if (threadIdx.x == 0) g.squares[blockIdx.x] = s;
}

// (Value by value: the compiler makes one wide load of a factor and what lies beside it where it is multiplied with a vector,
// and then keeps the structure that both are members of in private memory.)
__device__ __forceinline__ f32x4 times(f32x4 v, float f) {
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] *= f;
  return v;
}

// Four values to place k of a row (a multiple of 4), times 2^kX where they are of X.
template <bool SP>
__device__ __forceinline__ void put4(u16* row, int k, f32x4 v) {
  if constexpr (SP) {
    put_split(row, k, v);
  } else {
    u16 h[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = __builtin_bit_cast(u16, (_Float16)v[e]);
    *reinterpret_cast<u32x2*>(row + k) = u32x2{(unsigned)h[0] | (unsigned)h[1] << 16, (unsigned)h[2] | (unsigned)h[3] << 16};
  }
}
template <bool SP>
__device__ __forceinline__ f32x4 get4(const u16* row, int k) {
  const u16* p = SP ? row + k / 32 * kChunk + k % 32 : row + k;
  typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
  const f16x4 hi = *reinterpret_cast<const f16x4*>(p);
  f32x4 v{(float)hi[0], (float)hi[1], (float)hi[2], (float)hi[3]};
  if constexpr (SP) {
    const f16x4 lo = *reinterpret_cast<const f16x4*>(p + 32);
    v += f32x4{(float)lo[0], (float)lo[1], (float)lo[2], (float)lo[3]};
  }
  return v;
}
template <bool SP>
__device__ __forceinline__ int values_of(int units) { return SP ? units / 2 : units; }

// X = G / (|G| + eps) in both orders, 64 x 64 values per block; zeros behind a row's values.  Bound: reading G and writing
// twice as much (26 bf16 matrices, 1.37 GB in all: 356 us, 3.9 TB/s).
template <class E>
__global__ __launch_bounds__(256) void pack(const Group g, double eps) {
  constexpr bool SP = sizeof(E) == 4;
  __shared__ float s[64][65];
  const Matrix& m = g.matrices[g.of_pack[blockIdx.x]];
  double sum = 0.0;
  for (int k = threadIdx.x; k < m.chunks; k += 256) sum += g.squares[m.chunk0 + k];
  const double norm = sqrt(block_sum(sum)) + eps, f = norm != 0.0 ? (1 << kX) / norm : 0.0;
  const int rows = m.tall ? m.n : m.m, cols = m.tall ? m.m : m.n, wide = (cols + 63) / 64, t = blockIdx.x - m.pack0;
  const int r0 = t / wide * 64, c0 = t % wide * 64, tid = threadIdx.x;
  const E* p = in_memory<const E>(m.g);
  u16* const as = in_memory<u16>(m.tall ? m.xt[0] : m.x);
  u16* const across = in_memory<u16>(m.tall ? m.x : m.xt[0]);
  const int lda = m.tall ? m.ldm : m.ldn, ldc = m.tall ? m.ldn : m.ldm;
  // a thread has 16 values of a row, then of a column
  const int i = tid >> 2, c = 16 * (tid & 3), r = r0 + i;
  constexpr int W = Piece<E>::n;
  f32x4 v[4];
#pragma unroll
  for (int h = 0; h < 16 / W; ++h) {
    P<E> x{};
    if (r < rows && c0 + c + W * h < cols) x = piece_at(p + (size_t)r * cols + c0 + c + W * h, cols - (c0 + c + W * h));
#pragma unroll
    for (int e = 0; e < W; ++e) v[(W * h + e) / 4][e % 4] = (float)((double)value(x[e]) * f);  // (behind a row's values: zeros)
  }
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    if (r < rows && c0 + c + 4 * h < values_of<SP>(lda)) put4<SP>(as + (size_t)r * lda, c0 + c + 4 * h, v[h]);
#pragma unroll
    for (int e = 0; e < 4; ++e) s[i][c + 4 * h + e] = v[h][e];
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    const int k = c + 4 * h;
    if (c0 + i < cols && r0 + k < values_of<SP>(ldc))
      put4<SP>(across + (size_t)(c0 + i) * ldc, r0 + k, f32x4{s[k][i], s[k + 1][i], s[k + 2][i], s[k + 3][i]});
  }
}

// ------------------------------------------------------------------------------------------------
// Products
// ------------------------------------------------------------------------------------------------
enum Phase { kGram, kPoly, kStep, kLast };

// rows[b][a] and cols[a][b] = alpha (sum), and of kPoly + beta with[b][a] + unit [a = b], in the units of their operands.  (Phases are
// parameters of the templates: an end that is put together at run time would be kept in private memory.)
template <bool SP, int kPhase>
struct Keep {
  static constexpr bool kScaledByTile = false;
  float alpha, beta, unit;
  const u16* with;   // [B][ldr]
  u16 *rows, *cols;
  int A, B, ldr, ldc;
  template <class T>
  __device__ __forceinline__ void operator()(f32x4 (&acc)[T::NA][T::NB], const Place& pl, char* lds) const {
    constexpr int RA = 16 * T::NA, kPer = SP ? 2 : T::NB;  // the wave's a; tiles of b that go through LDS together
    constexpr int kBytes = SP ? 128 : 32 * T::NB, kPieces = kBytes / 16;
    static_assert(T::NB % kPer == 0 && T::kWaves * RA * kBytes <= T::kLds, "the transposed tile");
    char* const tr = lds + (pl.wa * T::WB + pl.wb) * RA * kBytes;
    const int lane = threadIdx.x & 63;
    const bool odd = lane & 1;
    const bool across = kPhase == kStep || pl.ta != pl.tb;  // (a tile on the diagonal of a symmetric product holds both)
    auto place = [](int v, int piece) { return v * kBytes + ((piece ^ (v >> 1 & (kPieces - 1))) << 4); };
    // Two lanes that hold neighbouring rows of b (n even, n + 1) swap two of their four values: the even lane then holds
    // values 0 and 1 of both, the odd one 2 and 3, and each writes pairs.
    auto put_pair = [&](int i, int col, const u16 (&v)[4]) {
      const unsigned lo = (unsigned)v[0] | (unsigned)v[1] << 16, hi = (unsigned)v[2] | (unsigned)v[3] << 16;
      const unsigned give = odd ? lo : hi, keep = odd ? hi : lo;
      const unsigned got = (unsigned)__builtin_amdgcn_update_dpp(0, (int)give, 0xB1, 0xf, 0xf, false);
      const unsigned e = odd ? got : keep, o = odd ? keep : got;
      const int r = 16 * i + 4 * pl.quad + (odd ? 2 : 0);
      *reinterpret_cast<unsigned*>(tr + place(r, col >> 3) + (col & 7) * 2) = (e & 0xffffu) | o << 16;
      *reinterpret_cast<unsigned*>(tr + place(r + 1, col >> 3) + (col & 7) * 2) = e >> 16 | (o & 0xffff0000u);
    };
#pragma unroll
    for (int j = 0; j < T::NB; ++j) {
      const int b = pl.b0 + 16 * j + pl.n;
      if constexpr (kPhase == kPoly) {  // (all of a row's reads before its stores, which could be to the same place for all that is known)
        f32x4 more[T::NA];
#pragma unroll
        for (int i = 0; i < T::NA; ++i) {
          const int a = pl.a0 + 16 * i + 4 * pl.quad;
          more[i] = b < B && a < values_of<SP>(ldr) ? get4<SP>(with + (size_t)b * ldr, a) : f32x4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int i = 0; i < T::NA; ++i) {
          const int a = pl.a0 + 16 * i + 4 * pl.quad;
          acc[i][j] = times(acc[i][j], alpha) + times(more[i], beta);
          if (pl.ta == pl.tb)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] += a + e == b ? unit : 0.f;
        }
      }
#pragma unroll
      for (int i = 0; i < T::NA; ++i) {
        const int a = pl.a0 + 16 * i + 4 * pl.quad;
        const bool in = b < B && a < values_of<SP>(ldr);
        const f32x4 v = kPhase == kPoly ? acc[i][j] : times(acc[i][j], alpha);
        u16 hi[4], lo[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (SP) split(v[e], hi[e], lo[e]);
          else hi[e] = __builtin_bit_cast(u16, (_Float16)v[e]);
        }
        if (in) {
          u16* d = rows + (size_t)b * ldr + (SP ? a / 32 * kChunk + a % 32 : a);
          *reinterpret_cast<u32x2*>(d) = u32x2{(unsigned)hi[0] | (unsigned)hi[1] << 16, (unsigned)hi[2] | (unsigned)hi[3] << 16};
          if constexpr (SP)
            *reinterpret_cast<u32x2*>(d + 32) = u32x2{(unsigned)lo[0] | (unsigned)lo[1] << 16, (unsigned)lo[2] | (unsigned)lo[3] << 16};
        }
        if (across) {
          put_pair(i, 16 * (j % kPer) + (pl.n & ~1), hi);
          if constexpr (SP) put_pair(i, 32 + 16 * (j % kPer) + (pl.n & ~1), lo);
        }
      }
      if (j % kPer != kPer - 1 || !across) continue;
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the wave's own part of LDS)
      const int unit0 = SP ? (pl.b0 + 16 * (j - 1)) * 2 : pl.b0;
      constexpr int kRows = 64 / kPieces;
#pragma unroll 4
      for (int k = 0; k < RA / kRows; ++k) {
        const int r = kRows * k + lane / kPieces, a = pl.a0 + r, piece = lane % kPieces;
        const u32x4 x = *reinterpret_cast<const u32x4*>(tr + place(r, piece));
        if (a < A && unit0 + 8 * piece < ldc) *reinterpret_cast<u32x4*>(cols + (size_t)a * ldc + unit0 + 8 * piece) = x;
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
  }
};

// out[b][a] = scale (alpha sum), alpha a power of two (alpha scale may lie below fp32's smallest normal value).
template <class E>
struct Result {
  static constexpr bool kScaledByTile = false;
  float alpha, scale;
  E* out;  // [B][A]
  int A, B;
  template <class T>
  __device__ __forceinline__ void operator()(f32x4 (&acc)[T::NA][T::NB], const Place& pl, char*) const {
#pragma unroll
    for (int j = 0; j < T::NB; ++j) {
      const int b = pl.b0 + 16 * j + pl.n;
      if (b >= B) continue;
#pragma unroll
      for (int i = 0; i < T::NA; ++i) {
        const int a = pl.a0 + 16 * i + 4 * pl.quad;
        if (a >= A) continue;
        const f32x4 v = times(times(acc[i][j], alpha), scale);
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
};

struct Step {
  float a, b, c;
  int now;  // which of xt is this step's
};

// The order of a launch's tiles: classes of matrices alike, those with the longest tiles first.  Each XCD (block b runs on XCD b
// mod 8) takes an eighth of every class, one run of it: so the tiles it works on at a time share their operands' rows in its
// L2, all XCDs have as much to do, and the last tiles are short.
constexpr int kClasses = 16;
struct Order {
  int n;
  int start[kClasses + 1];
  __host__ __device__ static int share(int all, int xcd) { return (all >> 3) * xcd + ((all & 7) * xcd >> 3); }  // all * xcd / 8
  // The tile of a block, or -1.
  __device__ __forceinline__ int tile() const {
    const int xcd = blockIdx.x & 7;
    int k = blockIdx.x >> 3;
    for (int c = 0; c < n; ++c) {
      const int all = start[c + 1] - start[c], lo = share(all, xcd), many = share(all, xcd + 1) - lo;
      if (k < many) return start[c] + lo + k;
      k -= many;
    }
    return -1;
  }
  unsigned blocks() const {
    int most = 0;
    for (int x = 0; x < 8; ++x) {
      int many = 0;
      for (int c = 0; c < n; ++c) many += share(start[c + 1] - start[c], x + 1) - share(start[c + 1] - start[c], x);
      most = std::max(most, many);
    }
    return 8u * most;
  }
};

// A phase of all matrices.  Bound: large matrices by the matrix units (busy 51 % of the cycles), small ones by the chain of a
// launch's loads and stores.  Measured: 26 matrices of widths 2048 and 8192 in bf16, a step: X X' 451 us and B X 948, 1.0
// PFLOP/s (of the triangle with its diagonal tiles; a plain library product of 16384^3 1.6), the polynomial 280; the smallest lists
// 6 to 7 us a phase.
template <class T, class E, int kPhase>
__global__ __launch_bounds__(T::kThreads, T::kOccupancy) void newton(const Group g, const Step s, const Order order) {
  constexpr bool SP = sizeof(E) == 4, kSym = kPhase <= kPoly;
  extern __shared__ __align__(16) char lds[];
  const int block = order.tile();
  if (block < 0) return;
  const Matrix& m = (kSym ? g.of_sym : g.of_step)[block];
  Place pl;
  Operand oa, ob;
  if constexpr (kSym) {
    const int t = block - m.sym0;
    int i = (int)((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
    while (i * (i + 1) / 2 > t) --i;
    while ((i + 1) * (i + 2) / 2 <= t) ++i;
    pl.tb = i;
    pl.ta = t - i * (i + 1) / 2;
    const int ld = kPhase == kGram ? m.ldn : m.ldm;
    oa = {in_memory<u16>(kPhase == kGram ? m.x : m.a), m.m, ld, ld};
    ob = oa;
  } else {
    const bool turned = kPhase == kLast && m.tall;
    const Address xt = s.now ? m.xt[1] : m.xt[0];
    oa = {in_memory<u16>(turned ? m.b : xt), turned ? m.m : m.n, m.ldm, m.ldm};
    ob = {in_memory<u16>(turned ? xt : m.b), turned ? m.n : m.m, m.ldm, m.ldm};
    const int ta = (int)((oa.rows + T::TA - 1) / T::TA), tb = (int)((ob.rows + T::TB - 1) / T::TB), t = block - m.step0;
    const int band = t / (kBand * ta), in = t - band * kBand * ta, wide = min(kBand, tb - band * kBand);
    pl.ta = in / wide;
    pl.tb = band * kBand + in - pl.ta * wide;
  }
  pl.in_tile<T>();
  f32x4 acc[T::NA][T::NB];
  auto exp2i = [](int e) { return __uint_as_float((unsigned)(127 + e) << 23); };
  if constexpr (kPhase == kLast) {
    const Result<E> end{exp2i(-kB - kX), m.scale, in_memory<E>(m.out), (int)oa.rows, (int)ob.rows};
    tile_sums<T, SP, f16x8>(acc, oa, ob, pl, 0, oa.k / kChunk, lds, end);
    end.template operator()<T>(acc, pl, lds);
  } else {
    u16* const rows = in_memory<u16>(kPhase == kGram ? m.a : kPhase == kPoly ? m.b : m.x);
    const Keep<SP, kPhase> end{kPhase == kGram ? exp2i(kA - 2 * kX) : kPhase == kPoly ? s.c * exp2i(kB - 2 * kA) : exp2i(-kB),
                               s.b * exp2i(kB - kA),
                               s.a * exp2i(kB),
                               in_memory<const u16>(m.a),
                               rows,
                               kSym ? rows : in_memory<u16>(s.now ? m.xt[0] : m.xt[1]),
                               (int)oa.rows,
                               (int)ob.rows,
                               kPhase == kStep ? m.ldn : m.ldm,
                               m.ldm};
    tile_sums<T, SP, f16x8>(acc, oa, ob, pl, 0, oa.k / kChunk, lds, end);
    end.template operator()<T>(acc, pl, lds);
  }
}

// ------------------------------------------------------------------------------------------------
// Host
// ------------------------------------------------------------------------------------------------
struct Sides {
  int m, n, ldm, ldn;
  bool tall;
  Sides(const wn_ortho_array& a) : m(std::min(a.rows, a.cols)), n(std::max(a.rows, a.cols)), tall(a.rows > a.cols) {
    ldm = padded_units(m, a.dtype == WN_F32);
    ldn = padded_units(n, a.dtype == WN_F32);
  }
  size_t bytes() const { return bytes_of(m, ldn) + 2 * bytes_of(n, ldm) + 2 * bytes_of(m, ldm); }  // (as matrix_of lays them out)
};
inline bool empty(const wn_ortho_array& a) { return a.rows == 0 || a.cols == 0; }

// The tiles of a launch: by a model of its time.  A chunk of 256 x 256 outputs takes a CU 1.4 us (three products of fp16
// parts: 2.1), of 128 x 128 two blocks on a CU 1.2 us, of 64 x 64 two 0.45 us; a tile's start and end 8, 6 and 2.5 us.
// Both sides of 64 and 128 (us a call of five steps, bf16 and fp32): B X of 576 tiles of 64 145 and 147, 227 and 228 (9 matrices of
// 512 x 512), 768 193 and 200, 346 and 352 (3 of 1024 x 1024), 982 160 and 167, 248 and 264 (14 of width 333), 896 155 and 152, 263 and
// 254 (14 of 512 x 512), 1024 241 and 237, 450 and 429 (1024 x 4096), 1536 324 and 300, 622 and 587 (6 of 1024 x 1024); X X' and the
// polynomial of 816 193 and 253, 346 and 460 (3 of 1024 x 1024), 1056 423 and 432, 817 and 806 (2048 x 2048), 1200 153 and 157, 239 and 260
// (60 of 256 x 256, where the model takes 128), 1632 324 and 314, 622 and 595 (6 of 1024 x 1024).
constexpr int kTileSides[3] = {256, 128, 64};
// What the LDS of 256 CUs holds.
template <class T>
constexpr int blocks_at_once() { return 256 * (160 * 1024 / T::kLds); }
static_assert(blocks_at_once<Big>() == 256 && blocks_at_once<Small>() == 512 && blocks_at_once<Tiny>() == 512, "the model's figures");
struct Plan {
  double sum[3] = {0, 0, 0}, longest[3] = {0, 0, 0}, blocks[3] = {0, 0, 0};
  void add(int k, double tiles, int units, bool sp) {
    static const double kChunkUs[3] = {1.4, 1.2, 0.45}, kEnds[3] = {8.0, 6.0, 2.5};
    const double us = units / kChunk * kChunkUs[k] * (sp ? 1.5 : 1.0) + kEnds[k];
    sum[k] += tiles * us;
    blocks[k] += tiles;
    longest[k] = std::max(longest[k], us);
  }
  int best() const {
    static const double kRoom[3] = {blocks_at_once<Big>(), blocks_at_once<Small>(), blocks_at_once<Tiny>()};
    int at = 0;
    double least = 1e300;
    for (int k = 0; k < 3; ++k) {
      const double us = blocks[k] <= kRoom[k] ? longest[k] : sum[k] / kRoom[k] + longest[k] / 2;
      if (us < least) least = us, at = k;
    }
    return at;
  }
};
inline double side_tiles(int v, int k) { return (double)ceil_div(v, kTileSides[k]); }

// The arrays of one dtype that go together: from `at` on, until their buffers fill kGroupBytes.
struct GroupPlan {
  std::vector<int> arrays;  // those with the longest tiles first
  int sym = 0, step = 0;  // tiles
  long long chunks = 0, packs = 0, syms = 0, steps = 0;
  Order sym_order{}, step_order{};
  size_t buffers = 0;
  // Bytes of all: descriptors, indexes, sums and buffers.
  size_t total() const {
    return up256(arrays.size() * sizeof(Matrix)) + up256(chunks * 8) + up256(chunks * 4) + up256(packs * 4) +
           up256(syms * sizeof(Matrix)) + up256(steps * sizeof(Matrix)) + buffers;
  }
};

GroupPlan next_group(int n_arrays, const wn_ortho_array* arrays, int dtype, int& at) {
  GroupPlan p;
  Plan sym, step;
  const bool sp = dtype == WN_F32;
  for (; at < n_arrays; ++at) {
    const wn_ortho_array& a = arrays[at];
    if (a.dtype != dtype || empty(a)) continue;
    const Sides s(a);
    if (!p.arrays.empty() && p.buffers + s.bytes() > kGroupBytes) break;
    p.arrays.push_back(at);
    p.buffers += s.bytes();
    for (int k = 0; k < 3; ++k) {
      const double tm = side_tiles(s.m, k);
      sym.add(k, tm * (tm + 1) / 2, s.ldn, sp);
      sym.add(k, tm * (tm + 1) / 2, s.ldm, sp);
      step.add(k, tm * side_tiles(s.n, k), s.ldm, sp);
    }
  }
  p.sym = sym.best();
  p.step = step.best();
  std::sort(p.arrays.begin(), p.arrays.end(), [&](int i, int k) {
    const Sides a(arrays[i]), b(arrays[k]);
    return a.ldn + a.ldm != b.ldn + b.ldm ? a.ldn + a.ldm > b.ldn + b.ldm : a.ldn != b.ldn ? a.ldn > b.ldn : i < k;
  });
  int ldn = -1, ldm = -1;
  for (int i : p.arrays) {
    const Sides s(arrays[i]);
    if ((s.ldn != ldn || s.ldm != ldm) && p.sym_order.n < kClasses) {
      p.sym_order.start[p.sym_order.n++] = (int)p.syms;
      p.step_order.start[p.step_order.n++] = (int)p.steps;
      ldn = s.ldn;
      ldm = s.ldm;
    }
    const long long tm = (long long)side_tiles(s.m, p.sym);
    p.chunks += (long long)ceil_div((size_t)s.m * s.n, (size_t)chunk_of((long long)s.m * s.n));
    p.packs += (long long)(ceil_div(s.m, 64) * ceil_div(s.n, 64));
    p.syms += tm * (tm + 1) / 2;
    p.steps += (long long)(side_tiles(s.m, p.step) * side_tiles(s.n, p.step));
  }
  p.sym_order.start[p.sym_order.n] = (int)p.syms;
  p.step_order.start[p.step_order.n] = (int)p.steps;
  return p;
}

template <class T, class E, int kPhase>
hipError_t launch_newton(const Group& g, const Step& s, const Order& order, hipStream_t st) {
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(newton<T, E, kPhase>), hipFuncAttributeMaxDynamicSharedMemorySize, T::kLds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((newton<T, E, kPhase>), dim3(order.blocks()), dim3(T::kThreads), T::kLds, st, g, s, order);
  return hipGetLastError();
}
template <class E, int kPhase>
hipError_t launch_tiles(int tile, const Group& g, const Step& s, const Order& order, hipStream_t st) {
  return tile == 0 ? launch_newton<Big, E, kPhase>(g, s, order, st)
                   : tile == 1 ? launch_newton<Small, E, kPhase>(g, s, order, st) : launch_newton<Tiny, E, kPhase>(g, s, order, st);
}

template <class E>
hipError_t run_group(const GroupPlan& p, const wn_ortho_array* arrays, int steps, const float* coefficients, float eps, char* ws,
                     hipStream_t st) {
  Carve c;
  Group g;
  g.matrices = reinterpret_cast<Matrix*>(ws + c.take(p.arrays.size() * sizeof(Matrix)));
  g.squares = reinterpret_cast<double*>(ws + c.take(p.chunks * 8));
  g.of_chunk = reinterpret_cast<int*>(ws + c.take(p.chunks * 4));
  g.of_pack = reinterpret_cast<int*>(ws + c.take(p.packs * 4));
  g.of_sym = reinterpret_cast<Matrix*>(ws + c.take(p.syms * sizeof(Matrix)));
  g.of_step = reinterpret_cast<Matrix*>(ws + c.take(p.steps * sizeof(Matrix)));
  int chunks = 0, packs = 0, syms = 0, products = 0;
  Batch batch;
  batch.sym_side = kTileSides[p.sym];
  batch.step_side = kTileSides[p.step];
  for (size_t at = 0; at < p.arrays.size();) {
    batch.first = (int)at;
    int n = 0;
    for (; n < kBatch && at < p.arrays.size(); ++n, ++at) {
      const wn_ortho_array& a = arrays[p.arrays[at]];
      const Address buffers = reinterpret_cast<Address>(ws + c.take(Sides(a).bytes()));
      batch.given[n] = {reinterpret_cast<Address>(a.g), reinterpret_cast<Address>(a.out), buffers, a.rows, a.cols, a.scale, chunks, packs, syms, products};
      const Matrix m = matrix_of(batch.given[n], sizeof(E) == 4, batch.sym_side, batch.step_side);
      chunks += m.chunks, packs += m.packs, syms += m.syms, products += m.steps;
    }
    hipLaunchKernelGGL(put_matrices<E>, dim3(n), dim3(256), 0, st, batch, g);
  }
  hipLaunchKernelGGL(squares<E>, dim3(chunks), dim3(256), 0, st, g);
  hipLaunchKernelGGL(pack<E>, dim3(packs), dim3(256), 0, st, g, (double)eps);
  hipError_t e = hipGetLastError();
  for (int k = 0; k < steps && e == hipSuccess; ++k) {
    const Step s{coefficients[3 * k], coefficients[3 * k + 1], coefficients[3 * k + 2], k & 1};
    e = launch_tiles<E, kGram>(p.sym, g, s, p.sym_order, st);
    if (e == hipSuccess) e = launch_tiles<E, kPoly>(p.sym, g, s, p.sym_order, st);
    if (e == hipSuccess) e = k + 1 < steps ? launch_tiles<E, kStep>(p.step, g, s, p.step_order, st) : launch_tiles<E, kLast>(p.step, g, s, p.step_order, st);
  }
  return e;
}

int check_arrays(int n_arrays, const wn_ortho_array* arrays) {
  if (n_arrays < 0 || n_arrays > 1 << 16) return wn_set_last_error(WN_EINVAL, "n_arrays must be 0..2^16");
  if (n_arrays && !arrays) return wn_set_last_error(WN_EINVAL, "null pointer");
  for (int k = 0; k < n_arrays; ++k) {
    const wn_ortho_array& a = arrays[k];
    const int rc = bad_dtype(a.dtype);
    if (rc != WN_OK) return rc;
    if (a.rows < 0 || a.rows > kMostSide || a.cols < 0 || a.cols > kMostSide || (long long)a.rows * a.cols > kMostElements)
      return wn_set_last_error(WN_EINVAL, "an array's rows and cols must be 0..2^18, their product at most 2^32");
  }
  return WN_OK;
}

// Of all groups, which share it one after the other.  Throws std::bad_alloc.
size_t workspace_bytes(int n_arrays, const wn_ortho_array* arrays) {
  size_t most = 0;
  for (int dtype : {WN_F32, WN_BF16})
    for (int at = 0; at < n_arrays;) {
      const GroupPlan p = next_group(n_arrays, arrays, dtype, at);
      if (!p.arrays.empty()) most = std::max(most, p.total());
    }
  return most;
}

}  // namespace

extern "C" {

size_t wn_orthogonalize_workspace_bytes(int32_t n_arrays, const wn_ortho_array* arrays) {
  if (check_arrays(n_arrays, arrays) != WN_OK) return 0;
  try {
    return workspace_bytes(n_arrays, arrays);
  } catch (const std::bad_alloc&) {
    return 0;
  }
}

int wn_orthogonalize(int32_t n_arrays, const wn_ortho_array* arrays, int32_t steps, const float* coefficients, float eps,
                     void* workspace, size_t ws_bytes, void* stream) {
  wn_clear_last_error();
  int rc = check_arrays(n_arrays, arrays);
  if (rc != WN_OK) return rc;
  if (steps < 1 || steps > kMostSteps) return wn_set_last_error(WN_EINVAL, "steps must be 1..64");
  if (!coefficients) return wn_set_last_error(WN_EINVAL, "null pointer");
  for (int k = 0; k < 3 * steps; ++k)
    if (!std::isfinite(coefficients[k])) return wn_set_last_error(WN_EINVAL, "coefficients must be finite");
  if (!(eps >= 0.f) || std::isinf(eps)) return wn_set_last_error(WN_EINVAL, "eps must be finite and >= 0");
  const wn_ortho_array* first = nullptr;
  for (int k = 0; k < n_arrays; ++k) {
    const wn_ortho_array& a = arrays[k];
    if (empty(a)) continue;
    if (!first) first = &a;
    if (!a.g || !a.out) return wn_set_last_error(WN_EINVAL, "null pointer");
    const uintptr_t size = a.dtype == WN_BF16 ? 2 : 4;
    if (reinterpret_cast<uintptr_t>(a.g) % size || reinterpret_cast<uintptr_t>(a.out) % size)
      return wn_set_last_error(WN_EINVAL, "an array is not aligned to its elements");
    if (!std::isfinite(a.scale)) return wn_set_last_error(WN_EINVAL, "scales must be finite");
  }
  if (!first) return WN_OK;
  try {
    if (overlap(n_arrays, arrays, [](const wn_ortho_array& a) { return (uintptr_t)a.rows * a.cols * (a.dtype == WN_BF16 ? 2 : 4); }))
      return wn_set_last_error(WN_EINVAL, "arrays overlap");
    rc = bad_workspace(workspace, ws_bytes, workspace_bytes(n_arrays, arrays));
    if (rc != WN_OK) return rc;
    ArrayScope scope;
    // (the first array stands for all, as in wn_clip)
    if ((rc = scope.check(workspace, "workspace")) != WN_OK || (rc = scope.check(first->g, "g")) != WN_OK ||
        (rc = scope.check(first->out, "out")) != WN_OK || (rc = scope.enter()) != WN_OK)
      return rc;
    char* const ws = static_cast<char*>(workspace);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    for (int dtype : {WN_F32, WN_BF16})
      for (int at = 0; at < n_arrays;) {
        const GroupPlan p = next_group(n_arrays, arrays, dtype, at);
        if (p.arrays.empty()) continue;
        const hipError_t e = dtype == WN_F32 ? run_group<float>(p, arrays, steps, coefficients, eps, ws, st)
                                             : run_group<u16>(p, arrays, steps, coefficients, eps, ws, st);
        if (e != hipSuccess) return wn_set_last_error(WN_EHIP, hipGetErrorString(e));
      }
  } catch (const std::bad_alloc&) {
    return wn_set_last_error(WN_ENOMEM, "out of host memory");
  }
  return WN_OK;
}

}  // extern "C"
