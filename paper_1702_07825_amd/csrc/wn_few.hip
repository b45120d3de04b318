// The loss of an output layer and its gradients for up to 64 rows (gfx950): scoring single tokens, or the last rows
// of short sequences.
//
// So few rows leave the products bound by the reads of w (and dw by its writes), so w goes from memory straight to the
// operands' registers, once in each pass, at whatever alignment it has and without a packed copy: bf16 on
// v_mfma_f32_16x16x32_bf16, fp32 on v_mfma_f32_16x16x4f32, whose rate just covers 64 rows at the memory's.  x is read
// the same way and stays in the caches.  Operand A's index is the classes (logits) or the columns (dx, dw),
// operand B's the rows, NB tiles of 16.
#include "wn_few.h"

namespace {

using namespace wnt;

template <class E>
__device__ __forceinline__ P<E> no_piece() {
  P<E> v;
#pragma unroll
  for (int e = 0; e < Piece<E>::n; ++e) v[e] = (E)0;
  return v;
}

// c += A B over 32 (bf16) or 16 (fp32) values of k: lane (n, quad) holds row n's pieces at 8 quad or 4 quad; product e
// of fp32 takes the values at 4 quad + e.
__device__ __forceinline__ f32x4 mma(u16x8 a, u16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  return c;
}

// ------------------------------------------------------------------------------------------------
// Logits: a wave takes T tiles of 16 classes.  The next U pieces of w are in flight during the current ones'
// products.  One tile of x's rows comes from the caches as an operand; more go through LDS, once for the block's four
// waves (straight from the caches, 37 rows x 50021 classes x 777, the reads of x took the pass from 40 to 92 us).
// ------------------------------------------------------------------------------------------------
template <int NB>
constexpr int kTilesOf = NB == 1 ? 1 : 2;  // T (wn_few_classes: 64 T a block)
constexpr int kRowBytes = 256, kPitch = kRowBytes + 16;  // of a chunk of x in LDS: 16 rows' pieces on different banks

//
// Few classes of long rows (wn_few_shared) leave most CUs idle so: there the block's four waves share their classes,
// a quarter of each row each, and the first adds the others' sums (16 rows x 3906 classes x 3398, fp32: 46 us a pass
// without, 19 so).
template <class E, int NB, bool kShared, class End>
__global__ __launch_bounds__(256, 2) void few_logits(const WnFew f, const End end) {
  constexpr int W = Piece<E>::n, K = 4 * W, T = kTilesOf<NB>, U = NB == 1 ? 8 : kRowBytes / 64;
  constexpr bool kStaged = NB > 1 && !kShared;
  __shared__ __align__(16) char xs[kStaged ? 2 * 16 * NB * kPitch : kShared ? 3 * T * NB * 64 * 16 : 16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, quad = lane >> 4;
  int v0 = (kShared ? blockIdx.x : blockIdx.x * 4 + wave) * 16 * T;
  // rows behind the last one repeat it: what they give is not used
  const E* w[T];
#pragma unroll
  for (int t = 0; t < T; ++t) w[t] = static_cast<const E*>(f.w) + (size_t)min(v0 + 16 * t + n, f.V - 1) * f.D + quad * W;
  f32x4 acc[T][NB];
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  P<E> a[T][U], next[T][U];
  const int whole = f.D / (U * K), chunks = (f.D + U * K - 1) / (U * K);
  auto fetch = [&](P<E> (&to)[T][U], int c) {
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = (c * U + u) * K;
        to[t][u] = c < whole ? whole_piece(w[t] + k) : piece_at(w[t] + k, f.D - k - quad * W);
      }
  };
  const int c0 = kShared ? chunks * wave / 4 : 0, c1 = kShared ? chunks * (wave + 1) / 4 : chunks;
  if (!kShared || c0 < c1) fetch(a, c0);
  if constexpr (kStaged) {
    constexpr int kPieces = 16 * NB * (kRowBytes / 16) / 256;  // of a chunk of x per thread
    P<E> xv[kPieces];
    const int xr = threadIdx.x >> 4, xc = threadIdx.x & 15;
    auto fetch_x = [&](int c) {
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const int k = c * U * K + xc * W;
        xv[i] = piece_at(static_cast<const E*>(f.x) + (size_t)min(xr + 16 * i, f.N - 1) * f.D + k, f.D - k);
      }
    };
    auto keep_x = [&](int c) {
#pragma unroll
      for (int i = 0; i < kPieces; ++i)
        *reinterpret_cast<P<E>*>(xs + (c & 1) * 16 * NB * kPitch + (xr + 16 * i) * kPitch + xc * 16) = xv[i];
    };
    fetch_x(0);
    keep_x(0);
    for (int c = 0; c < chunks; ++c) {
      const bool more = c + 1 < chunks;
      if (more) {
        fetch_x(c + 1);
        fetch(next, c + 1);
      }
      wnk::lds_barrier();  // (its waits leave the loads in flight)
      const char* at = xs + (c & 1) * 16 * NB * kPitch + n * kPitch + quad * 16;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        P<E> b[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) b[j] = *reinterpret_cast<const P<E>*>(at + j * 16 * kPitch + u * 64);
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
          for (int j = 0; j < NB; ++j) acc[t][j] = mma(a[t][u], b[j], acc[t][j]);
      }
      if (more) {
        keep_x(c + 1);  // (the other buffer: its readers passed the barrier above)
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
          for (int u = 0; u < U; ++u) a[t][u] = next[t][u];
      }
    }
  } else {
    const E* x[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) x[j] = static_cast<const E*>(f.x) + (size_t)min(16 * j + n, f.N - 1) * f.D + quad * W;
    for (int c = c0; c < c1; ++c) {
      P<E> b[U][NB];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = (c * U + u) * K;
#pragma unroll
        for (int j = 0; j < NB; ++j) b[u][j] = c < whole ? whole_piece(x[j] + k) : piece_at(x[j] + k, f.D - k - quad * W);
      }
      if (c + 1 < c1) fetch(next, c + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
          for (int j = 0; j < NB; ++j) acc[t][j] = mma(a[t][u], b[u][j], acc[t][j]);
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int u = 0; u < U; ++u) a[t][u] = next[t][u];
    }
  }
  if constexpr (kShared) {
    f32x4* const s = reinterpret_cast<f32x4*>(xs);
    if (wave)
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int j = 0; j < NB; ++j) s[((wave - 1) * T * NB + t * NB + j) * 64 + lane] = acc[t][j];
    __syncthreads();
    if (wave == 0) {
      for (int w4 = 0; w4 < 3; ++w4)
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
          for (int j = 0; j < NB; ++j) acc[t][j] += s[(w4 * T * NB + t * NB + j) * 64 + lane];
    } else {
      v0 = 1 << 29;  // no classes: the first wave has them
    }
  }
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int v = v0 + 16 * t + 4 * quad + e;
      const float bv = f.b ? f.b[min(v, f.V - 1)] : 0.f;
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[t][j][e] = v < f.V ? acc[t][j][e] + bv : -INFINITY;
    }
  end(f, acc, v0 + 4 * quad, n, quad, wave);
}

struct FewStats {
  float2* part;
  float* target;
  template <int T, int NB>
  __device__ void operator()(const WnFew& f, f32x4 (&acc)[T][NB], int v, int n, int quad, int wave) const {
    __shared__ float2 s[4][16 * NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int r = 16 * j + n;
      const int y = r < f.N ? f.y[r] : -1;
      float m = -INFINITY;
#pragma unroll
      for (int t = 0; t < T; ++t) m = fmaxf(m, fmaxf(fmaxf(acc[t][j][0], acc[t][j][1]), fmaxf(acc[t][j][2], acc[t][j][3])));
      m = quads_max(m);
      const float at = m == -INFINITY ? 0.f : m;
      float sum = 0.f;
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sum += wnk::expf_fast(acc[t][j][e] - at);
          if (y == v + 16 * t + e && y < f.V) target[r] = acc[t][j][e];
        }
      sum = quads_sum(sum);
      if (quad == 0) s[wave][r] = make_float2(m, sum);
    }
    __syncthreads();
    const int r = threadIdx.x;
    if (r >= f.N) return;
    float2 o = s[0][r];
#pragma unroll
    for (int w = 1; w < 4; ++w) {
      const float2 p = s[w][r];
      const float m = fmaxf(o.x, p.x), at = m == -INFINITY ? 0.f : m;
      o = make_float2(m, o.y * wnk::expf_fast(o.x - at) + p.y * wnk::expf_fast(p.x - at));
    }
    part[(size_t)blockIdx.x * f.N + r] = o;
  }
};

// The same with the sum that the entropy takes, and the largest logit of every 8 classes: those of an even quad and the odd
// one behind it.
struct FewProbe {
  float2* part;
  float *spread, *target;
  float* groups;  // [N][ceil(V / 8)], or null
  template <int T, int NB>
  __device__ void operator()(const WnFew& f, f32x4 (&acc)[T][NB], int v, int n, int quad, int wave) const {
    __shared__ WnStat s[4][16 * NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int r = 16 * j + n;
      const int y = r < f.N ? f.y[r] : -1;
      float g[T];
      WnStat o{-INFINITY, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < T; ++t) {
        g[t] = fmaxf(fmaxf(acc[t][j][0], acc[t][j][1]), fmaxf(acc[t][j][2], acc[t][j][3]));
        o.m = fmaxf(o.m, g[t]);
      }
      o.m = quads_max(o.m);
      const float at = o.m == -INFINITY ? 0.f : o.m;
#pragma unroll
      for (int t = 0; t < T; ++t) {
        if (groups) {
          const float m8 = fmaxf(g[t], __shfl_xor(g[t], 16, 64));
          const int v8 = v + 16 * t;  // (an even quad's is a multiple of 8)
          if (!(quad & 1) && r < f.N && v8 < f.V) groups[(size_t)r * ((f.V + 7) / 8) + v8 / 8] = m8;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          o.count(acc[t][j][e], at);
          if (y == v + 16 * t + e && y < f.V) target[r] = acc[t][j][e];
        }
      }
      o.s = quads_sum(o.s);
      o.t = quads_sum(o.t);
      if (quad == 0) s[wave][r] = o;
    }
    __syncthreads();
    const int r = threadIdx.x;
    if (r >= f.N) return;
    WnStat o = s[0][r];
#pragma unroll
    for (int w = 1; w < 4; ++w) o.add(s[w][r]);
    part[(size_t)blockIdx.x * f.N + r] = make_float2(o.m, o.s);
    spread[(size_t)blockIdx.x * f.N + r] = o.t;
  }
};

// q as the operand of dx ([n][v]; its rows take g where their parts are joined), q g / max |g| as that of dw ([v][n]), so
// that rounding to bf16 leaves the targets' entries near -1 alone; and db, all of whose rows are here.
template <class E, bool ENT>
struct FewGrad {
  const float *lse, *g;
  E *q, *qt;  // or null
  int vpad, npad;
  float* db;  // or null
  WnTerms terms;  // ENT: of log probabilities and entropies
  template <int T, int NB>
  __device__ void operator()(const WnFew& f, f32x4 (&acc)[T][NB], int first, int n, int quad, int) const {
    float ln[NB], gn[NB], most = 0.f;
    float an[NB], en[NB], hn[NB];
    int y[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int r = 16 * j + n;
      y[j] = r < f.N ? f.y[r] : -1;
      if (y[j] >= f.V) y[j] = -1;
      ln[j] = y[j] >= 0 ? lse[r] : 0.f;
      gn[j] = y[j] >= 0 ? g[r] : 0.f;
      if constexpr (ENT) {
        an[j] = y[j] >= 0 ? terms.target[r] : 0.f;
        en[j] = y[j] >= 0 ? terms.spread[r] : 0.f;
        hn[j] = y[j] >= 0 ? terms.entropy[r] : 0.f;
      }
      most = fmaxf(most, fabsf(gn[j]));
    }
    most = row16_max(most);
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const int v = first + 16 * t;
      f32x4 sum{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const int r = 16 * j + n;
        f32x4 p;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (ENT) p[e] = wn_spread(acc[t][j][e] - ln[j], an[j], en[j], hn[j]) + (v + e == y[j] ? an[j] : 0.f);
          else p[e] = wnk::expf_fast(acc[t][j][e] - ln[j]) - (v + e == y[j] ? 1.f : 0.f);
          p[e] = y[j] >= 0 && v + e < f.V ? p[e] : 0.f;
        }
        sum += p * gn[j];
        if (q && r < f.N && v < vpad) {
          E* d = q + (size_t)r * vpad + v;
          if constexpr (sizeof(E) == 4) *reinterpret_cast<f32x4*>(d) = p;
          else *reinterpret_cast<u32x2*>(d) = u32x2{bf16_pair(p[0], p[1]), bf16_pair(p[2], p[3])};
        }
        if (qt) {
          const float gh = most != 0.f ? gn[j] / most : gn[j];  // (a NaN, which max |g| passes over, stays)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (v + e < f.V) put(qt + (size_t)(v + e) * npad + r, p[e] * gh);
        }
      }
      if (NB == 1 && qt) {  // (bf16 takes 32 rows at a time)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (v + e < f.V) put(qt + (size_t)(v + e) * npad + 16 + n, 0.f);
      }
      if (!db) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float s = wnk::gsum16(sum[e]);
        if (n == 0 && v + e < f.V) db[v + e] = s;
      }
    }
  }
};

// ------------------------------------------------------------------------------------------------
// dx and dw: operand A is a row-major array's columns, kSlab of them, its k the array's rows.  A lane reads a piece of
// a row at column W n, for the rows at W quad .. + W - 1 of a step: piece t, element u is then column W n + u of row
// W quad + t, so fragment u (columns W n + u, n = 0 .. 15) takes element u of every piece.  (bf16: pairs
// of rows by one v_perm each.)
// ------------------------------------------------------------------------------------------------
template <class E>
constexpr int kSlab = 16 * Piece<E>::n;
template <class E>
constexpr int kStep = 4 * Piece<E>::n;  // rows of a step

template <class E>
struct Columns {
  P<E> f[Piece<E>::n];
  // rows r0 + W quad + t of [R][D] (rows behind the last: the last again), columns c0 + W n ..
  __device__ __forceinline__ void load(const E* p, int R, int D, int r0, int c, int quad) {
    constexpr int W = Piece<E>::n;
#pragma unroll
    for (int t = 0; t < W; ++t) f[t] = piece_at(p + (size_t)min(r0 + W * quad + t, R - 1) * D + c, D - c);
  }
  __device__ __forceinline__ P<E> fragment(int u) const {
    constexpr int W = Piece<E>::n;
    P<E> r;
    if constexpr (W == 4) {
#pragma unroll
      for (int t = 0; t < W; ++t) r[t] = f[t][u];
    } else {
      u32x4 o;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const unsigned a = __builtin_bit_cast(u32x4, f[2 * t])[u >> 1], b = __builtin_bit_cast(u32x4, f[2 * t + 1])[u >> 1];
        o[t] = __builtin_amdgcn_perm(b, a, u & 1 ? 0x07060302u : 0x05040100u);
      }
      r = __builtin_bit_cast(P<E>, o);
    }
    return r;
  }
};

// Bound: reading w (dx) and writing as much (dw).  Measured, 37 rows x 50021 classes x 777 (odd rows of 78 MB), bf16: dx
// 43 us, dw 36, the logits 38; 1 row x 32000 x 2048 (131 MB): logits 24 us, 5.4 TB/s, where w stays in the caches between
// passes; with 12 such w in turn 33 us a call, not 26.
// dx's parts: a block takes a slab of columns and a run of classes, its waves a quarter of the run each, and adds the
// quarters up.
template <class E, int NB>
__global__ __launch_bounds__(256, 2) void few_dx(const WnFew f, const E* q, int vpad, int each, float* sum) {
  constexpr int W = Piece<E>::n, S = kStep<E>;
  extern __shared__ __align__(16) char dyn[];
  f32x4* const s = reinterpret_cast<f32x4*>(dyn);  // [W NB][64]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, quad = lane >> 4;
  const int c = blockIdx.x * kSlab<E> + W * n;
  const int quarter = each / 4, v0 = blockIdx.y * each + wave * quarter, v1 = min(f.V, v0 + quarter);
  const E* w = static_cast<const E*>(f.w);
  f32x4 acc[W][NB];
#pragma unroll
  for (int u = 0; u < W; ++u)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[u][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int cc = min(c, f.D - 1);  // (columns behind the last are not stored)
  if (v0 < v1) {
    Columns<E> a, next;
    a.load(w, f.V, f.D, v0, cc, quad);
    for (int v = v0; v < v1; v += S) {
      P<E> b[NB];
#pragma unroll
      for (int j = 0; j < NB; ++j)
        b[j] = 16 * j + n < f.N ? whole_piece(q + (size_t)(16 * j + n) * vpad + v + W * quad) : no_piece<E>();
      next.load(w, f.V, f.D, v + S < v1 ? v + S : v, cc, quad);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = 0; u < W; ++u) {
        const P<E> x = a.fragment(u);
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[u][j] = mma(x, b[j], acc[u][j]);
      }
      a = next;
    }
  }
  for (int w4 = 1; w4 < 4; ++w4) {
    __syncthreads();
    if (wave == w4)
#pragma unroll
      for (int u = 0; u < W; ++u)
#pragma unroll
        for (int j = 0; j < NB; ++j) s[(u * NB + j) * 64 + lane] = acc[u][j];
    __syncthreads();
    if (wave == 0)
#pragma unroll
      for (int u = 0; u < W; ++u)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[u][j] += s[(u * NB + j) * 64 + lane];
  }
  if (wave) return;
  // lane (n, quad): columns W (4 quad + i) + u of row 16 j + n
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int r = 16 * j + n;
    if (r >= f.N) continue;
    float* d = sum + ((size_t)blockIdx.y * f.N + r) * f.D + blockIdx.x * kSlab<E>;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int u = 0; u < W; ++u) {
        const int k = W * (4 * quad + i) + u;
        if (blockIdx.x * kSlab<E> + k < f.D) d[k] = acc[u][j][i];
      }
  }
}

// dw: a wave keeps its slab of x's columns in registers and goes over its classes, 16 at a time.
template <class E, int NB>
__global__ __launch_bounds__(256, 2) void few_dw(const WnFew f, const E* qt, int npad, const float* g, E* dw) {
  constexpr int W = Piece<E>::n, S = kStep<E>, K = (16 * NB + S - 1) / S, kTiles = 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, quad = lane >> 4;
  const int c0 = blockIdx.y * kSlab<E>, c = min(c0 + W * n, f.D - 1);
  float most = 0.f;  // max |g|, which q was divided by
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int r = 16 * j + n, t = r < f.N ? f.y[r] : -1;
    if (t >= 0 && t < f.V) most = fmaxf(most, fabsf(g[r]));
  }
  most = row16_max(most);
  __shared__ __align__(16) char stage[4][16 * 256];
  char* const mine = stage[wave];
  P<E> a[K][W];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    Columns<E> t;
    // (rows behind N and rows without a target meet zeros in q: anything but a NaN would do, so they are zeroed)
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const int r = k * S + W * quad + i, yr = r < f.N ? f.y[r] : -1;
      t.f[i] = yr >= 0 && yr < f.V ? piece_at(static_cast<const E*>(f.x) + (size_t)r * f.D + c, f.D - c) : no_piece<E>();
    }
#pragma unroll
    for (int u = 0; u < W; ++u) a[k][u] = t.fragment(u);
  }
  for (int t = 0; t < kTiles; ++t) {
    const int v0 = ((blockIdx.x * 4 + wave) * kTiles + t) * 16;
    if (v0 >= f.V) return;
    const int v = v0 + n;
    f32x4 acc[W];
#pragma unroll
    for (int u = 0; u < W; ++u) acc[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const P<E> b = whole_piece(qt + (size_t)min(v, f.V - 1) * npad + k * S + W * quad);
#pragma unroll
      for (int u = 0; u < W; ++u) acc[u] = mma(a[k][u], b, acc[u]);
    }
    // lane (n, quad) holds columns W (4 quad + i) .. + W - 1 of class n; through LDS, so that 16 lanes store a class's
    // 256 bytes (each lane storing its own pieces, 64 places an instruction, 37 rows x 50021 classes x 777 took 44 us)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      P<E> o;
#pragma unroll
      for (int u = 0; u < W; ++u) {
        E e;
        put(&e, acc[u][i] * most);
        o[u] = e;
      }
      const int p = 4 * quad + i;
      *reinterpret_cast<P<E>*>(mine + n * 256 + ((p ^ n) << 4)) = o;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the wave's own part)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 4 * i + quad, k = c0 + W * n;
      const P<E> o = *reinterpret_cast<const P<E>*>(mine + r * 256 + ((n ^ r) << 4));
      if (v0 + r >= f.V) continue;
      E* d = dw + (size_t)(v0 + r) * f.D + k;
      if (k + W <= f.D) {
        typename Piece<E>::any x;
#pragma unroll
        for (int u = 0; u < W; ++u) x[u] = o[u];
        *reinterpret_cast<typename Piece<E>::any*>(d) = x;
      } else {
#pragma unroll
        for (int u = 0; u < W; ++u)
          if (k + u < f.D) d[u] = o[u];
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
}

template <class F>
void by_tiles(int tiles, F f) {
  if (tiles == 1) f(std::integral_constant<int, 1>{});
  else if (tiles == 2) f(std::integral_constant<int, 2>{});
  else f(std::integral_constant<int, 4>{});
}

template <class E, int NB, class End>
void launch_logits(const WnFew& f, int classes, const End& end, hipStream_t st) {
  const dim3 grid((unsigned)ceil_div(classes, wn_few_classes(sizeof(E) == 4, f.N, f.D, f.V)));
  if (wn_few_shared(sizeof(E) == 4, f.N, f.D, f.V)) hipLaunchKernelGGL((few_logits<E, NB, true, End>), grid, dim3(256), 0, st, f, end);
  else hipLaunchKernelGGL((few_logits<E, NB, false, End>), grid, dim3(256), 0, st, f, end);
}

}  // namespace

template <class E>
hipError_t wn_few_loss(const WnFew& f, float2* part, float* target, hipStream_t st) {
  by_tiles(wn_few_tiles(sizeof(E) == 4, f.N, f.D, f.V), [&](auto nb) {
    const FewStats end{part, target};
    launch_logits<E, decltype(nb)::value>(f, f.V, end, st);
  });
  return hipGetLastError();
}

template <class E>
hipError_t wn_few_probe(const WnFew& f, float2* part, float* spread, float* target, float* groups, hipStream_t st) {
  by_tiles(wn_few_tiles(sizeof(E) == 4, f.N, f.D, f.V), [&](auto nb) {
    const FewProbe end{part, spread, target, groups};
    launch_logits<E, decltype(nb)::value>(f, f.V, end, st);
  });
  return hipGetLastError();
}

WnFewPlan wn_few_plan(bool f32, int N, int D, int V) {
  WnFewPlan p;
  const int step = f32 ? 16 : 32, e = f32 ? 4 : 2, slab = f32 ? 64 : 128;
  // q's rows hold zeros from V to vpad, past which no step reads; each block of dx takes 4 quarters of whole steps, some 512 blocks
  p.vpad = (int)ceil_div(V, 64) * 64;
  p.npad = N <= 32 ? 32 : 64;
  p.slabs = (int)ceil_div(D, slab);
  const size_t want = std::max<size_t>(1, 512 / p.slabs);
  p.each = (int)(std::max<size_t>(1, ceil_div(V, want * 4 * step)) * 4 * step);
  p.parts = (int)ceil_div(V, p.each);
  p.q_bytes = (size_t)N * p.vpad * e;
  p.qt_bytes = (size_t)V * p.npad * e;
  p.sum_bytes = (size_t)p.parts * N * D * 4;
  return p;
}

template <class E>
hipError_t wn_few_grads(const WnFew& f, const WnFewPlan& p, const float* lse, const float* g, const WnTerms* terms, bool dx, void* dw,
                        float* db, void* q, void* qt, float* sum, hipStream_t st) {
  by_tiles(wn_few_tiles(sizeof(E) == 4, f.N, f.D, f.V), [&](auto nb) {
    auto grads = [&](auto ent) {
      const FewGrad<E, decltype(ent)::value> end{lse, g, dx ? static_cast<E*>(q) : nullptr, dw ? static_cast<E*>(qt) : nullptr, p.vpad,
                                                 p.npad, db, terms ? *terms : WnTerms{}};
      launch_logits<E, decltype(nb)::value>(f, p.vpad, end, st);  // (q holds zeros behind V)
    };
    if (terms) grads(std::true_type{});
    else grads(std::false_type{});
  });
  by_tiles(f.N <= 16 ? 1 : f.N <= 32 ? 2 : 4, [&](auto nb) {
    constexpr int NB = decltype(nb)::value, W = Piece<E>::n;
    if (dx)
      hipLaunchKernelGGL((few_dx<E, NB>), dim3(p.slabs, p.parts), dim3(256), W * NB * 64 * 16, st, f, static_cast<const E*>(q), p.vpad,
                         p.each, sum);
    if (dw)
      hipLaunchKernelGGL((few_dw<E, NB>), dim3((unsigned)ceil_div(f.V, 256), p.slabs), dim3(256), 0, st, f, static_cast<const E*>(qt),
                         p.npad, g, static_cast<E*>(dw));
  });
  return hipGetLastError();
}

template hipError_t wn_few_loss<float>(const WnFew&, float2*, float*, hipStream_t);
template hipError_t wn_few_loss<u16>(const WnFew&, float2*, float*, hipStream_t);
template hipError_t wn_few_probe<float>(const WnFew&, float2*, float*, float*, float*, hipStream_t);
template hipError_t wn_few_probe<u16>(const WnFew&, float2*, float*, float*, float*, hipStream_t);
template hipError_t wn_few_grads<float>(const WnFew&, const WnFewPlan&, const float*, const float*, const WnTerms*, bool, void*, float*,
                                        void*, void*, float*, hipStream_t);
template hipError_t wn_few_grads<u16>(const WnFew&, const WnFewPlan&, const float*, const float*, const WnTerms*, bool, void*, float*,
                                      void*, void*, float*, hipStream_t);
