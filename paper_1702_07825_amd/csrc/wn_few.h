// Interface of the loss's kernels for few rows (gfx950).
#pragma once
#include "wn_arrays.h"

#include "wn_wave.h"

namespace wnt {

typedef u16 u16x8u __attribute__((ext_vector_type(8), aligned(2)));
typedef u16 u16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

// A 16-byte piece of a row: 8 bf16 or 4 fp32 values.
template <class E>
struct Piece;
template <>
struct Piece<u16> {
  typedef u16x8 type;
  typedef u16x8u any;
  static constexpr int n = 8;
};
template <>
struct Piece<float> {
  typedef f32x4 type;
  typedef f32x4u any;
  static constexpr int n = 4;
};
template <class E>
using P = typename Piece<E>::type;

// Elements k .. of p, of which `left` exist (any number); the rest are 0.
template <class E>
__device__ __forceinline__ P<E> piece_at(const E* p, int left) {
  constexpr int n = Piece<E>::n;
  P<E> v;
  if (left >= n) {
    const typename Piece<E>::any x = *reinterpret_cast<const typename Piece<E>::any*>(p);
#pragma unroll
    for (int e = 0; e < n; ++e) v[e] = x[e];
  } else {
#pragma unroll
    for (int e = 0; e < n; ++e) v[e] = e < left ? p[e] : (E)0;
  }
  return v;
}
template <class E>
__device__ __forceinline__ P<E> whole_piece(const E* p) {
  const typename Piece<E>::any x = *reinterpret_cast<const typename Piece<E>::any*>(p);
  P<E> v;
#pragma unroll
  for (int e = 0; e < Piece<E>::n; ++e) v[e] = x[e];
  return v;
}

// Over a lane's place in the four rows of 16 lanes.
__device__ __forceinline__ float quads_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float quads_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// Over the 16 lanes of a row of lanes.
__device__ __forceinline__ float row16_max(float v) {
  v = fmaxf(v, wnk::dpp<0xB1>(v));
  v = fmaxf(v, wnk::dpp<0x4E>(v));
  v = fmaxf(v, wnk::dpp<0x141>(v));
  return fmaxf(v, wnk::dpp<0x140>(v));
}

}  // namespace wnt

// A row's largest logit m in some classes, the sum s of exp(l - m) there, and t, that of exp(l - m) (l - m).
struct WnStat {
  float m, s, t;  // (-INFINITY, 0, 0 of no classes)
  // (differences of infinities are cut to -1e30: their exponentials are 0, and a product with 0 then is too)
  __device__ __forceinline__ void add(const WnStat& o) {
    const float top = fmaxf(m, o.m), at = top == -INFINITY ? 0.f : top;
    const float da = fmaxf(m - at, -1e30f), db = fmaxf(o.m - at, -1e30f), ea = wnk::expf_fast(m - at), eb = wnk::expf_fast(o.m - at);
    t = ea * (t + da * s) + eb * (o.t + db * o.s);
    s = s * ea + o.s * eb;
    m = top;
  }
  // One logit, where m is known to be the largest.
  __device__ __forceinline__ void count(float l, float at) {
    const float d = l - at, e = wnk::expf_fast(d);
    s += e;
    t += e * fmaxf(d, -1e30f);
  }
};

// q of a class before its target's entry, from its log p: the gradient of log probabilities and entropies is
// c (a [v = y] - p (a + e (log p + H))).  (log 0 is -infinity: its product with p is 0)
__device__ __forceinline__ float wn_spread(float lp, float a, float e, float H) {
  return -wnk::expf_fast(lp) * (a + e * (fmaxf(lp, -3e38f) + H));
}

// Calls of up to this many rows read w from memory straight into registers, once each pass, instead of through tiles
// in LDS.
constexpr int kFewRows = 64;
// Whether a block's four waves share its classes: where a run of classes each would leave too few blocks, and the rows
// are long enough to cut in four.  A forward pass with classes of its own for each wave and with shared ones (us), rows of 1000
// values: 64 rows, fp32 51 and 24 at 8000 classes, 51 and 42 at 16384, 51 and 55 at 20000; 17 rows 32 and 16, 32 and 26,
// 33 and 35; 16 rows 32 and 13, 32 and 21, 33 and 24, 33 and 31 at 26000; bf16, 32 rows 13 and 10, 14 and 13, 15 and 17;
// 64 rows 16 and 13, 17 and 17 at 12000 (of 2048 values 27 and 30), 18 and 18 at 16384.  Of 200 values at 8000 classes: 64
// rows, fp32 18 and 13, bf16 11 and 11.
inline bool wn_few_shared(bool f32, int N, int D, int V) {
  return V <= (f32 || N <= 32 ? 1 << 14 : 1 << 13) && D * (f32 ? 4 : 2) >= 800;
}
// Tiles of 16 rows in the logits: 1, 2 or 4.  One tile takes x from the caches and two or more through LDS, which is faster
// from a few rows on (50021 classes x 777, bf16: 4 rows 48 and 35 us, 16 rows 60 and 36); shared classes take it from
// the caches anyway.
inline int wn_few_tiles(bool f32, int N, int D, int V) {
  if (N <= 16 && (N == 1 || wn_few_shared(f32, N, D, V))) return 1;
  return N <= 32 ? 2 : 4;
}
// Classes of a block: a place in `part`.
inline int wn_few_classes(bool f32, int N, int D, int V) {
  return (wn_few_tiles(f32, N, D, V) == 1 ? 16 : 32) * (wn_few_shared(f32, N, D, V) ? 1 : 4);
}

struct WnFew {
  int N, D, V;
  const void *x, *w;  // float or bf16
  const float* b;     // or null
  const int32_t* y;
};

// Forward: (largest logit, sum of exponentials) of each row in each run of wn_few_classes() classes, part[run][N], and the
// targets' logits.
template <class E>
hipError_t wn_few_loss(const WnFew& f, float2* part, float* target, hipStream_t st);

// Log probabilities, entropies and alternatives: beside the above spread[run][N], each run's sum of exp(l - largest)
// (l - largest), and the largest logit of every 8 classes, groups[N][ceil(V / 8)] (null: not wanted).
template <class E>
hipError_t wn_few_probe(const WnFew& f, float2* part, float* spread, float* target, float* groups, hipStream_t st);

// Backward.  Workspace of the q's ([N][V] and [V][N], padded) and of dx's parts; `parts` of them, [parts][N][D] fp32,
// are left in `sum` for the caller to join (rows without a target hold anything there).
struct WnFewPlan {
  int vpad;                 // row of q
  int npad;                 // row of the transposed one
  int slabs, parts, each;   // dx: runs of columns, of classes; classes of a run
  size_t q_bytes, qt_bytes, sum_bytes;
};
WnFewPlan wn_few_plan(bool f32, int N, int D, int V);
// Of log probabilities and entropies, whose rows' factors then stand for g: entropies, and what the target's entry and the
// spread of the others take, [N] each.
struct WnTerms {
  const float *entropy, *target, *spread;
};
// (terms null: the loss's)
template <class E>
hipError_t wn_few_grads(const WnFew& f, const WnFewPlan& p, const float* lse, const float* g, const WnTerms* terms, bool dx, void* dw,
                        float* db, void* q, void* qt, float* sum, hipStream_t st);
