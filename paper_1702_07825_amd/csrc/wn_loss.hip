// The loss of an output layer and its gradients without keeping the logits (gfx950).  Declarations and
// contracts are in include/wn_train.h.
//
// Everything heavy is one product C[b][a] = sum_k A[a][k] B[b][k] with different ends (product):
//   logits   A = w, B = x           the tile's largest logit and sum of exponentials of each row (forward), or
//                                   q = exp(l - lse) - [v = y] as the next products' operand (backward; for log
//                                   probabilities and entropies another q, see row_terms)
//   dx       A = w transposed, B = q
//   dw       A = x transposed, B = q transposed
// Both operands lie along k in memory, so the transposed ones are copies (pack_cols); the backward pass takes
// the vocabulary in pieces, so that they and q stay within a fixed size.
//
// Operands are 16-bit: bf16 arrays as they are, fp32 ones in two fp16 parts each (wn_product.h).
//
// Up to kFewRows rows go to wn_few.hip, which is bound by reading w once (64 and 65 rows x 50021 classes x 777: forward 42
// and 70 us in bf16, 79 and 134 in fp32).
#include "wn_product.h"

namespace {

using namespace wnt;

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
// scale to the next by at most 2^66, those of log probabilities and entropies (whose |q| is below 8, e from 12) by 2^68: below 2^118
// with 2^20 rows of products below 2^30.  (A tile whose q is not finite takes e = 0; the class's sums are not finite then.)
constexpr int kQScale = 14, kQMost = 80;
// With upstream gradients g of a row's log probability and h of its entropy the logits' gradient is
//   g ([v = y] - p) - h p (log p + H) = c q,   q = a [v = y] - p (a + e (log p + H)),   c = max(|g|, |h|), a = g / c, e = h / c:
// the row's factor c takes the part of the loss's g, so that the target's entry is near +-1 where the log probability weighs
// most.  |q| is below 1 + p |log p + H|, at most 5.3 for 2^24 classes (half of the probability on one class, the other
// half even), so its fp16 parts as dx's operand are those of q 2^13.
__global__ __launch_bounds__(256) void row_terms(const float* g, const float* h, const int32_t* y, int N, int V, float* c, float* a, float* e) {
  const int n = blockIdx.x * 256 + threadIdx.x;
  if (n >= N) return;
  const int t = y[n];
  const bool ok = t >= 0 && t < V;
  const float gn = ok && g ? g[n] : 0.f, hn = ok && h ? h[n] : 0.f;
  const float most = gn != gn || hn != hn ? gn + hn : fmaxf(fabsf(gn), fabsf(hn));  // (a NaN stays)
  c[n] = most;
  a[n] = most != 0.f ? gn / most : 0.f;
  e[n] = most != 0.f ? hn / most : 0.f;
}

// Backward: q of the tile's rows and classes as the operands of dx ([n][v]) and dw ([v][n]), and the sums of g q
// over the tile's rows.  q enters the products without g (|q| <= 1): dx's rows take their g afterwards, and so does dw:
// fp32 arrays with x's rows, bf16 ones as g / max |g| here and max |g| afterwards.  So the target's entry, -1 and a
// probability, is hardly touched by q's rounding to bf16: with g in q all rows of a mean shared the rounding
// error of -1 / N, which was off by 0.38 % in both gradients (4096 rows of text; now 0.17 %, what the
// gradients' own rounding costs).  A lane holds four classes of a row, so [n][v] is
// stored from the registers (32-byte runs); [v][n] goes through LDS, a wave's classes by 64 rows (fp32: 32 rows,
// hi and lo parts) at a time, so that its stores are runs of 128 bytes.
template <bool SP, bool ENT>
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
  WnTerms terms;   // ENT
  static constexpr int kScale = ENT ? kQScale - 1 : kQScale;  // of q as dx's operand
  // 2^e of this lane's classes over the tile's rows, whose log p (ENT: whose q) are in acc: a class's rows lie in 16 lanes
  // of each of WB waves.  A class that a row of the tile targets may have a q near -1.
  template <class T>
  __device__ __forceinline__ void class_scales(const f32x4 (&acc)[T::NA][T::NB], const Place& pl, char* lds, f32x4 (&by)[T::NA]) const {
    float* const s = reinterpret_cast<float*>(lds);  // [WB][TA], and [TA]: 0 for a target, -inf
    for (int k = threadIdx.x; k < T::TA; k += T::kThreads) s[T::WB * T::TA + k] = -INFINITY;
    __syncthreads();
    for (int k = threadIdx.x; !ENT && k < T::TB; k += T::kThreads) {
      const int n = pl.tb * T::TB + k, yn = n < l.N ? l.y[n] : -1, a = yn < 0 ? -1 : yn - l.v0 - pl.ta * T::TA;
      if (a >= 0 && a < T::TA) s[T::WB * T::TA + a] = 0.f;
    }
    const int at = pl.wa * 16 * T::NA + 4 * pl.quad;
#pragma unroll
    for (int i = 0; i < T::NA; ++i) {
      f32x4 m;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        m[e] = ENT ? fabsf(acc[i][0][e]) : acc[i][0][e];
#pragma unroll
        for (int j = 1; j < T::NB; ++j) m[e] = fmaxf(m[e], ENT ? fabsf(acc[i][j][e]) : acc[i][j][e]);
        m[e] = row16_max(m[e]);
      }
      if (pl.n == 0) *reinterpret_cast<f32x4*>(s + pl.wb * T::TA + at + 16 * i) = m;
    }
    __syncthreads();
    for (int k = threadIdx.x; k < T::TA; k += T::kThreads) {
      float m = s[k];
#pragma unroll
      for (int w = 1; w <= T::WB; ++w) m = fmaxf(m, s[w * T::TA + k]);
      int e;
      if constexpr (ENT) e = m < 0x1p-66f ? kQMost : m < 0x1p13f ? kQScale - ilogbf(m) : 0;  // (|q| is below 8 unless it is not finite)
      else e = kQScale - (int)fminf(fmaxf(floorf(m * 1.4426950408889634f), kQScale - kQMost), 0.f);
      const int v = pl.ta * T::TA + k;
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
    auto to_q = [&](int j) {  // log p to q
      float an = 0.f, en = 0.f, hn = 0.f;
      if constexpr (ENT) {
        const int n = pl.b0 + 16 * j + pl.n, yn = n < l.N ? l.y[n] : -1;
        if (yn >= 0 && yn < l.V_all) an = terms.target[n], en = terms.spread[n], hn = terms.entropy[n];
      }
#pragma unroll
      for (int i = 0; i < T::NA; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = ENT ? wn_spread(acc[i][j][e], an, en, hn) : wnk::expf_fast(acc[i][j][e]);
      Logits::at_target<T>(pl, t[j], [&](int i, int e) { acc[i][j][e] += ENT ? an : -1.f; });
    };
    f32x4 by[SP ? T::NA : 1];
    if constexpr (SP) {
#pragma unroll
      for (int j = 0; j < T::NB; ++j) {
        less_lse(j);
        if constexpr (ENT) to_q(j);
      }
      if (qt) class_scales<T>(acc, pl, lds, by);
    }
#pragma unroll
    for (int j = 0; j < T::NB; ++j) {
      if constexpr (!SP) less_lse(j);
      if constexpr (!SP || !ENT) to_q(j);
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
            for (int e = 0; e < 4; ++e) split(p[e] * (1 << kScale), hi[e], lo[e]);
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
  const int* eq;      // fp32 dw: eb of each tile of k, [tiles][B]
  int eb_all;         // fp32 dx: eb
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
      const float f = __uint_as_float((unsigned)(127 + now[b] - (now - B)[b]) << 23);  // (at most 2^68 either way where q is finite)
#pragma unroll
      for (int i = 0; i < T::NA; ++i) acc[i][j] *= f;
    }
  }
  template <class T>
  __device__ void operator()(f32x4 (&acc)[T::NA][T::NB], const Place& pl, char*) const {
    if constexpr (sizeof(E) == 4) {
      int eb[T::NB];
#pragma unroll
      for (int j = 0; j < T::NB; ++j) eb[j] = kScaledByTile ? eq[(size_t)(pl.last >> tile) * B + min(pl.b0 + 16 * j + pl.n, B - 1)] : eb_all;
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
constexpr size_t kBackwardPiece = (size_t)1 << 30;   // bytes of w's forms and q in the backward pass
constexpr int kColumnParts = 64;  // of column_max

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

// ENT: for log probabilities and entropies, g the rows' factors (row_terms).
template <bool ENT, class E>
int run_backward(int N, int D, int V, const E* x, const E* w, const float* b, const int32_t* y, const float* lse,
                 const float* g, const WnTerms& terms, E* dx, E* dw, float* db, char* ws, hipStream_t st) {
  constexpr bool sp = sizeof(E) == 4;
  const Backward f(sp, N, D, V);
  auto ints = [&](size_t off) { return reinterpret_cast<int*>(ws + off); };
  auto units = [&](size_t off) { return reinterpret_cast<u16*>(ws + off); };
  auto floats = [&](size_t off) { return reinterpret_cast<float*>(ws + off); };
  if (N <= kFewRows) {
    hipError_t e = wn_few_grads<E>({N, D, V, x, w, b, y}, f.few, lse, g, ENT ? &terms : nullptr, dx != nullptr, dw, db, ws + f.q, ws + f.qt, floats(f.dx), st);
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
    GradEnd<sp, ENT> end{{sp ? ints(f.ex) : nullptr, sp ? ints(f.ew) : nullptr, b ? b + v0 : nullptr, y, N, n, v0, V},
                    lse, g, gmax, gparts, dx ? units(f.q) : nullptr, dw ? units(f.qt) : nullptr, ldq, ldqt,
                    ints(f.eq), db ? floats(f.db) : nullptr, terms};
    e = run_product<sp>({ow, ox, 0, 0, 1, 0}, big, end, st);
    if (e == hipSuccess && db) e = join(floats(f.db), (int)ceil_div(N, big ? 256 : 128), n, db + v0, st);
    if (e == hipSuccess && dx) {
      const Operand owt = cols_operand(wv, n, D, RowFactor{nullptr, nullptr, 0}, units(f.wt), floats(f.cmax), ints(f.ewt), st);
      const bool whole = f.piece == V && f.dxs.splits == 1;
      const OutEnd<E, false> o{D, N, ints(f.ewt), nullptr, GradEnd<sp, ENT>::kScale, 0, y, g, nullptr, 0, V, whole ? nullptr : floats(f.dx), v0 > 0, dx};
      e = run_product<sp>({owt, {units(f.q), N, ldq, ldq}, 0, 0, f.dxs.splits, 0}, f.dxs.big, o, st);
      if (e == hipSuccess && !whole && v0 + n == V) e = join(floats(f.dx), f.dxs.splits, (size_t)N * D, dx, st);
    }
    if (e == hipSuccess && dw) {
      E* const out = dw + (size_t)v0 * D;
      const OutEnd<E, true> o{D, n, ints(f.ext), sp ? ints(f.eq) : nullptr, 0, big ? 3 : 2, nullptr, nullptr, gmax, gparts, 1, f.dws.splits == 1 ? nullptr : floats(f.dw), 0, out};
      e = run_product<sp>({oxt, {units(f.qt), n, ldqt, ldqt}, 0, 0, f.dws.splits, 0}, f.dws.big, o, st);
      if (e == hipSuccess && f.dws.splits > 1) e = join(floats(f.dw), f.dws.splits, (size_t)n * D, out, st);
    }
  }
  return e == hipSuccess ? WN_OK : wn_set_last_error(WN_EHIP, hipGetErrorString(e));
}

// The terms of the rows lie behind the rest of the workspace.
size_t backward_bytes(int dtype, int N, int D, int V, bool ent) {
  if (!sizes_ok(dtype, N, D, V) || N == 0) return 0;
  return Backward(dtype == WN_F32, N, D, V).total + (ent ? 3 * up256((size_t)N * 4) : 0);
}

// Both entry points' checks and call (ENT: wn_logprobs_backward).
template <bool ENT>
int backward(int32_t dtype, int32_t N, int32_t D, int32_t V, const void* x, const void* w, const float* b, const int32_t* y,
             const float* lse, const float* entropy, const float* g, const float* h, void* dx, void* dw, float* db,
             void* workspace, size_t ws_bytes, void* stream) {
  wn_clear_last_error();
  int rc = check_sizes(dtype, N, D, V);
  if (rc != WN_OK) return rc;
  if (!dx && !dw && !db) return wn_set_last_error(WN_EINVAL, "no gradient is wanted");
  if (N > 0 && (!x || !w || !y || !lse || (ENT ? !entropy || (!g && !h) : !g))) return wn_set_last_error(WN_EINVAL, "null pointer");
  if (N == 0 && !dw && !db) return WN_OK;
  rc = bad_workspace(workspace, ws_bytes, backward_bytes(dtype, N, D, V, ENT));
  if (rc != WN_OK) return rc;
  ArrayScope scope;
  const struct { const void* p; const char* name; } arrays[] = {
      {N ? x : nullptr, "x"}, {N ? w : nullptr, "w"}, {N ? b : nullptr, "b"}, {N ? y : nullptr, "y"}, {N ? lse : nullptr, "lse"},
      {N ? entropy : nullptr, "entropy"}, {N ? g : nullptr, "g"}, {N ? h : nullptr, "h"},
      {N ? dx : nullptr, "dx"}, {dw, "dw"}, {db, "db"}, {N ? workspace : nullptr, "workspace"}};
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
  WnTerms terms{};
  if constexpr (ENT) {
    const size_t each = up256((size_t)N * 4);
    float* const c = reinterpret_cast<float*>(ws + backward_bytes(dtype, N, D, V, false));
    float* const a = c + each / 4;
    float* const e = a + each / 4;
    hipLaunchKernelGGL(row_terms, dim3((unsigned)ceil_div(N, 256)), dim3(256), 0, st, g, h, y, N, V, c, a, e);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return wn_set_last_error(WN_EHIP, hipGetErrorString(err));
    terms = {entropy, a, e};
    g = c;
  }
  if (dtype == WN_F32)
    return run_backward<ENT>(N, D, V, static_cast<const float*>(x), static_cast<const float*>(w), b, y, lse, g, terms,
                             static_cast<float*>(dx), static_cast<float*>(dw), db, ws, st);
  return run_backward<ENT>(N, D, V, static_cast<const u16*>(x), static_cast<const u16*>(w), b, y, lse, g, terms, static_cast<u16*>(dx),
                           static_cast<u16*>(dw), db, ws, st);
}

}  // namespace

extern "C" {

size_t wn_loss_workspace_bytes(int32_t dtype, int32_t N, int32_t D, int32_t V) {
  if (!sizes_ok(dtype, N, D, V) || N == 0) return 0;
  return Forward(dtype == WN_F32, N, D, V).total;
}

size_t wn_loss_backward_workspace_bytes(int32_t dtype, int32_t N, int32_t D, int32_t V) {
  return backward_bytes(dtype, N, D, V, false);
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
  return backward<false>(dtype, N, D, V, x, w, b, y, lse, nullptr, g, nullptr, dx, dw, db, workspace, ws_bytes, stream);
}

size_t wn_logprobs_backward_workspace_bytes(int32_t dtype, int32_t N, int32_t D, int32_t V) {
  return backward_bytes(dtype, N, D, V, true);
}

int wn_logprobs_backward(int32_t dtype, int32_t N, int32_t D, int32_t V, const void* x, const void* w, const float* b,
                         const int32_t* y, const float* lse, const float* entropy, const float* g, const float* h, void* dx,
                         void* dw, float* db, void* workspace, size_t ws_bytes, void* stream) {
  return backward<true>(dtype, N, D, V, x, w, b, y, lse, entropy, g, h, dx, dw, db, workspace, ws_bytes, stream);
}

}  // extern "C"
