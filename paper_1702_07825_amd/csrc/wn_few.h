// Interface of the loss's kernels for few rows (gfx950).
#pragma once
#include "wn_arrays.h"

#include "wn_wave.h"

namespace wnt {

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

// Backward.  Workspace of the q's ([N][V] and [V][N], padded) and of dx's parts; `parts` of them, [parts][N][D] fp32,
// are left in `sum` for the caller to join (rows without a target hold anything there).
struct WnFewPlan {
  int vpad;                 // row of q
  int npad;                 // row of the transposed one
  int slabs, parts, each;   // dx: runs of columns, of classes; classes of a run
  size_t q_bytes, qt_bytes, sum_bytes;
};
WnFewPlan wn_few_plan(bool f32, int N, int D, int V);
template <class E>
hipError_t wn_few_grads(const WnFew& f, const WnFewPlan& p, const float* lse, const float* g, bool dx, void* dw, float* db, void* q,
                        void* qt, float* sum, hipStream_t st);
