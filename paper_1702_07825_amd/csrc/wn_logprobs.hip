// Log probabilities of given tokens under an output layer, entropies and the likeliest classes, without keeping the
// logits (gfx950).  Declarations and contracts are in include/wn_train.h; the gradients are in wn_loss.hip.
//
// The logits are one product (wn_product.h; up to kFewRows rows: wn_few.hip) whose end leaves, per row and tile, the
// largest logit m, s = sum exp(l - m) and t = sum exp(l - m) (l - m).  With these joined, lse = m + log s and
//   H = lse - sum p l = log s - t / s:
// both terms are at least 0, so no entropy is negative and none is the difference of large numbers.
//
// Alternatives: the end also leaves the largest logit of every 8 classes.  The K likeliest classes lie in the K groups of
// 8 whose largest logits are largest (any K classes from K other groups would be less likely), so a row's groups are
// searched for a few more than K (kept()), and their classes' logits are computed anew, in 64 bits.  So the logits
// are neither kept nor sorted, classes next to each other are in order although the product's sums are of 32 bits, and
// equal ones (copies of a row of w) are equal: the lowest index comes first.
#include "wn_product.h"

namespace {

constexpr int kMostTop = 32;
constexpr size_t kGroupsBytes = (size_t)256 << 20;  // of the groups' largest logits of a piece: they stay in the last-level cache

// Groups of 8 classes kept for `top` alternatives: more than `top`, since a group's largest logit is off by the product's
// rounding.  Classes are missed only if more groups than the surplus lie within that rounding of the last one wanted.
__host__ __device__ constexpr int kept(int top) { return top + 2 + top / 8; }
static_assert(kept(kMostTop) <= 64, "a lane for each");

struct ProbeEnd {
  static constexpr bool kScaledByTile = false;
  Logits l;
  float2* part;    // [tiles of all pieces][N]: m and s
  float* spread;   // t
  int tile0;       // the piece's first
  float* target;   // [N]
  float* groups;   // [N][ceil(l.V / 8)], or null
  template <class T>
  __device__ void operator()(f32x4 (&acc)[T::NA][T::NB], const Place& pl, char* lds) const {
    l.take<T>(acc, pl);
    WnStat* const s = reinterpret_cast<WnStat*>(lds);  // [WA][TB]
    const int ng = (l.V + 7) / 8;
#pragma unroll
    for (int j = 0; j < T::NB; ++j) {
      const int n = pl.b0 + 16 * j + pl.n;
      const int yn = n < l.N ? l.y[n] : -1, t = yn >= 0 ? yn - l.v0 : -1;
      float g[T::NA];
      WnStat o{-INFINITY, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < T::NA; ++i) {
        g[i] = fmaxf(fmaxf(acc[i][j][0], acc[i][j][1]), fmaxf(acc[i][j][2], acc[i][j][3]));
        o.m = fmaxf(o.m, g[i]);
      }
      o.m = quads_max(o.m);
      Logits::at_target<T>(pl, t < l.V ? t : -1, [&](int i, int e) { target[n] = acc[i][j][e]; });
      if (groups) {
        // an even quad and the odd one behind it hold 8 classes of a row: the even one stores those of even i
#pragma unroll
        for (int i = 0; i < T::NA; i += 2) {
          const bool odd = pl.quad & 1;
          const float a = fmaxf(g[i], __shfl_xor(g[i], 16, 64)), b = fmaxf(g[i + 1], __shfl_xor(g[i + 1], 16, 64));
          const int at = (pl.a0 + 16 * i) / 8 + (pl.quad >> 1) + (odd ? 2 : 0);
          if (n < l.N && at < ng) groups[(size_t)n * ng + at] = odd ? b : a;
        }
      }
      // (rows without a class yet: every exponential is 0, not exp(-inf + inf))
      const float at = o.m == -INFINITY ? 0.f : o.m;
#pragma unroll
      for (int i = 0; i < T::NA; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o.count(acc[i][j][e], at);
      o.s = quads_sum(o.s);
      o.t = quads_sum(o.t);
      if (pl.quad == 0) s[pl.wa * T::TB + pl.wb * (T::TB / T::WB) + 16 * j + pl.n] = o;
    }
    __syncthreads();
    for (int k = threadIdx.x; k < T::TB; k += T::kThreads) {
      const int n = pl.tb * T::TB + k;
      WnStat r = s[k];
#pragma unroll
      for (int w = 1; w < T::WA; ++w) r.add(s[w * T::TB + k]);
      if (n >= l.N) continue;
      part[(size_t)(tile0 + pl.ta) * l.N + n] = make_float2(r.m, r.s);
      spread[(size_t)(tile0 + pl.ta) * l.N + n] = r.t;
    }
  }
};

// What a row's joined parts give.
struct RowOut {
  const float* target;
  const int32_t* y;
  int N, V;
  float *logprob, *entropy, *lse;
  float* log_s;  // [N]
  __device__ __forceinline__ void put(int n, const WnStat& o) const {
    const float z = logf(o.s);
    const int t = y[n];
    lse[n] = o.m + z;
    logprob[n] = t >= 0 && t < V ? (target[n] - o.m) - z : 0.f;  // (in this order log s is not lost beside a large m)
    entropy[n] = z - o.t / o.s;
    log_s[n] = z;
  }
};

// 16 rows by 16 runs of tiles per block.
__global__ __launch_bounds__(256) void join_probe(const float2* part, const float* spread, int tiles, const RowOut r) {
  __shared__ WnStat s[16][16];
  const int c = threadIdx.x & 15, w = threadIdx.x >> 4, n = blockIdx.x * 16 + c;
  WnStat o{-INFINITY, 0.f, 0.f};
  if (n < r.N)
    for (int t = w; t < tiles; t += 16) {
      const float2 p = part[(size_t)t * r.N + n];
      o.add({p.x, p.y, spread[(size_t)t * r.N + n]});
    }
  s[w][c] = o;
  __syncthreads();
  if (w || n >= r.N) return;
  for (int k = 1; k < 16; ++k) o.add(s[k][c]);
  r.put(n, o);
}

// The same for few rows: a block per row.
__global__ __launch_bounds__(256) void join_probe_few(const float2* part, const float* spread, int tiles, const RowOut r) {
  __shared__ WnStat s[4];
  const int n = blockIdx.x;
  WnStat o{-INFINITY, 0.f, 0.f};
#pragma unroll 4
  for (int t = threadIdx.x; t < tiles; t += 256) {
    const float2 p = part[(size_t)t * r.N + n];
    o.add({p.x, p.y, spread[(size_t)t * r.N + n]});
  }
  for (int d = 32; d; d >>= 1) o.add({__shfl_xor(o.m, d, 64), __shfl_xor(o.s, d, 64), __shfl_xor(o.t, d, 64)});
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = o;
  __syncthreads();
  if (threadIdx.x) return;
  for (int w = 1; w < 4; ++w) o.add(s[w]);
  r.put(n, o);
}

// ------------------------------------------------------------------------------------------------
// Alternatives
// ------------------------------------------------------------------------------------------------
struct Group {
  float v;  // largest logit
  int g;    // classes 8 g ..; kNone: no group
};
constexpr int kNone = (1 << 24) - 1;  // (numbers of groups are compared as floats)
static_assert(kMaxV / 8 < kNone, "groups");

// The `want` largest of a wave's R entries a lane, by value and then by the lower number: lane r ends with the r-th.
template <int R>
__device__ __forceinline__ Group largest_of(Group (&e)[R], int want) {
  const int lane = threadIdx.x & 63;
  Group mine{-INFINITY, kNone};
  for (int r = 0; r < want; ++r) {
    Group b = e[0];
#pragma unroll
    for (int k = 1; k < R; ++k)
      if (e[k].v > b.v || (e[k].v == b.v && e[k].g < b.g)) b = e[k];
    const float top = wnk::wave_max(b.v);
    const int g = (int)-wnk::wave_max(b.v == top ? -(float)b.g : -(float)kNone);
    if (lane == r) mine = {top, g};
#pragma unroll
    for (int k = 0; k < R; ++k)
      if (e[k].g == g) e[k] = {-INFINITY, kNone};
  }
  return mine;
}

struct Alternatives {
  const float* groups;  // [N][count] of this piece
  int count, first;     // its groups, the number of the first
  int N, D, V, top;
  const void *x, *w;
  const float* b;       // or null
  const float* log_s;   // [N]
  Group* list;          // [N][kept(top)] from piece to piece
  int seen, last;       // 0: list is empty; the last piece
  int32_t* ids;         // [N][top]
  float* logprobs;
};
constexpr int kSegment = 16;  // groups a lane looks at together

// The classes of the kept groups: their logits in 64 bits, a wave for each group; lane 8 c of a wave ends with class c's.
template <class E>
__device__ __forceinline__ double class_logit(const Alternatives& a, int n, int g) {
  constexpr int W = Piece<E>::n;
  const int lane = threadIdx.x & 63;
  const E* x = static_cast<const E*>(a.x) + (size_t)n * a.D;
  const E* w = static_cast<const E*>(a.w) + (size_t)g * 8 * a.D;
  double sum[8];
  size_t row[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    sum[c] = 0.0;
    row[c] = (size_t)min(c, a.V - 1 - g * 8) * a.D;  // (classes behind the last: the last again)
  }
  auto add = [&](const P<E>& xv, const P<E> (&wv)[8]) {
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const double xd = value(xv[k]);
#pragma unroll
      for (int c = 0; c < 8; ++c) sum[c] += xd * (double)value(wv[c][k]);
    }
  };
  const int whole = a.D / (64 * W) * (64 * W);
  for (int k = lane * W; k < whole; k += 64 * W) {
    P<E> wv[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) wv[c] = whole_piece(w + row[c] + k);
    add(whole_piece(x + k), wv);
  }
  if (const int k = whole + lane * W; k < a.D) {
    P<E> wv[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) wv[c] = piece_at(w + row[c] + k, a.D - k);
    add(piece_at(x + k, a.D - k), wv);
  }
  // halves of the lanes take halves of the classes, three times; then 8 lanes add up
#pragma unroll
  for (int h = 4; h; h >>= 1) {
    const bool up = lane & (h * 8);
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (c < h) {
        const double give = up ? sum[c] : sum[c + h], keep = up ? sum[c + h] : sum[c];
        sum[c] = keep + __shfl_xor(give, h * 8, 64);
      }
  }
  double s = sum[0];
  for (int d = 4; d; d >>= 1) s += __shfl_xor(s, d, 64);
  const int v = g * 8 + (lane >> 3);
  if (a.b && v < a.V) s += (double)a.b[v];
  return s;
}

// A block per row: each wave finds the largest groups of its segments, the first joins them; in the last piece the
// waves compute their classes' logits, which are then ranked.
template <class E, int kWaves>
__global__ __launch_bounds__(64 * kWaves) void alternatives(const Alternatives a) {
  __shared__ Group found[kWaves + 1][64];
  __shared__ double logit[64 * 8];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = blockIdx.x, want = kept(a.top);
  const float* groups = a.groups + (size_t)n * a.count;
  Group mine{-INFINITY, kNone};
  for (int s = wave * 64 * kSegment; s < a.count; s += kWaves * 64 * kSegment) {
    Group e[kSegment + 1];
    float most = -INFINITY;
#pragma unroll
    for (int k = 0; k < kSegment; ++k) {
      const int i = s + k * 64 + lane;
      const float v = i < a.count ? groups[i] : -INFINITY;
      e[k] = {v == v ? v : -INFINITY, i < a.count ? a.first + i : kNone};  // (a NaN would be neither before nor behind another)
      most = fmaxf(most, e[k].v);
    }
    // (numbers rise from segment to segment, so an equal value comes behind those kept)
    const Group least{__shfl(mine.v, want - 1, 64), __shfl(mine.g, want - 1, 64)};
    if (least.g != kNone && !__any(most > least.v)) continue;
    e[kSegment] = mine;
    mine = largest_of(e, want);
  }
  found[wave][lane] = mine;
  if (wave == 0) found[kWaves][lane] = a.seen && lane < want ? a.list[(size_t)n * want + lane] : Group{-INFINITY, kNone};
  __syncthreads();
  if (wave == 0) {
    Group e[kWaves + 1];
#pragma unroll
    for (int k = 0; k <= kWaves; ++k) e[k] = found[k][lane];
    mine = largest_of(e, want);
    found[0][lane] = mine;
    if (!a.last && lane < want) a.list[(size_t)n * want + lane] = mine;
  }
  if (!a.last) return;
  __syncthreads();
  for (int k = wave; k < want; k += kWaves) {
    const int g = found[0][k].g;
    if (g == kNone) continue;
    const double s = class_logit<E>(a, n, g);
    if ((lane & 7) == 0) logit[k * 8 + (lane >> 3)] = s;
  }
  __syncthreads();
  const float z = a.log_s[n];
  auto class_of = [&](int i) {  // or -1
    const int g = found[0][i >> 3].g, v = g * 8 + (i & 7);
    return g != kNone && v < a.V ? v : -1;
  };
  for (int i = threadIdx.x; i < want * 8; i += 64 * kWaves) {
    const int v = class_of(i);
    if (v < 0) continue;
    const double l = logit[i], key = l == l ? l : -INFINITY;
    int rank = 0;
    double most = -INFINITY;
    for (int k = 0; k < want * 8; ++k) {
      const int o = class_of(k);
      const double ol = logit[k], okey = ol == ol ? ol : -INFINITY;
      rank += o >= 0 && (okey > key || (okey == key && o < v));
      if (o >= 0) most = fmax(most, okey);
    }
    if (rank < a.top) {
      a.ids[(size_t)n * a.top + rank] = v;
      // (the row's largest logit is taken off as it is here, not as the product rounded it: no log probability is above 0)
      a.logprobs[(size_t)n * a.top + rank] = (float)((l - most) - (double)z);
    }
  }
}

// ------------------------------------------------------------------------------------------------
// Host
// ------------------------------------------------------------------------------------------------
// Classes of a piece; `each` as for forward_piece.
int probe_piece(int N, int V, size_t each, int top) {
  const int most = forward_piece(N, V, each);
  if (!top) return most;
  const size_t fit = std::max<size_t>(256, kGroupsBytes / 4 * 8 / N / 256 * 256);
  return (int)std::min<size_t>(most, fit);
}

struct Probe {
  int piece;
  size_t part, spread, target, log_s, groups, list, x, ex, w, ew, total;
  Probe(bool sp, int N, int D, int V, int top) {
    Carve c;
    const bool few = N <= kFewRows;
    const size_t units = padded_units(D, sp), tiles = few ? ceil_div(V, wn_few_classes(sp, N, D, V)) : ceil_div(V, 128);
    piece = few ? V : probe_piece(N, V, units * 2 + 4, top);
    part = c.take(tiles * N * sizeof(float2));
    spread = c.take(tiles * N * 4);
    target = c.take((size_t)N * 4);
    log_s = c.take((size_t)N * 4);
    groups = c.take(top ? (size_t)N * ceil_div(few ? V : probe_piece(N, V, 0, top), 8) * 4 : 0);
    list = c.take(top ? (size_t)N * kept(top) * sizeof(Group) : 0);
    if (!few) {
      x = c.take((size_t)N * units * 2);
      ex = c.take((size_t)N * 4);
      w = c.take(piece * units * 2);
      ew = c.take((size_t)piece * 4);
    }
    total = c.at;
  }
};

template <class E>
hipError_t launch_alternatives(const Alternatives& a, hipStream_t st) {
  // one wave for each segment, or each kept group
  const int waves = (int)std::max<size_t>(ceil_div(a.count, 64 * kSegment), a.last ? kept(a.top) : 1);
  if (waves > 4) hipLaunchKernelGGL((alternatives<E, 8>), dim3(a.N), dim3(512), 0, st, a);
  else hipLaunchKernelGGL((alternatives<E, 4>), dim3(a.N), dim3(256), 0, st, a);
  return hipGetLastError();
}

struct ProbeCall {
  int N, D, V, top;
  const float* b;
  const int32_t* y;
  float *logprob, *entropy, *lse;
  int32_t* ids;
  float* top_logprobs;
};

template <class E>
int run_probe(const ProbeCall& c, const E* x, const E* w, char* ws, hipStream_t st) {
  constexpr bool sp = sizeof(E) == 4;
  const int N = c.N, D = c.D, V = c.V;
  const Probe f(sp, N, D, V, c.top);
  float2* const part = reinterpret_cast<float2*>(ws + f.part);
  float* const spread = reinterpret_cast<float*>(ws + f.spread);
  float* const target = reinterpret_cast<float*>(ws + f.target);
  float* const log_s = reinterpret_cast<float*>(ws + f.log_s);
  float* const groups = c.top ? reinterpret_cast<float*>(ws + f.groups) : nullptr;
  const RowOut rows{target, c.y, N, V, c.logprob, c.entropy, c.lse, log_s};
  Alternatives alt{groups, 0, 0, N, D, V, c.top, x, w, c.b, log_s, reinterpret_cast<Group*>(ws + f.list), 0, 0, c.ids, c.top_logprobs};
  if (N <= kFewRows) {
    hipError_t e = wn_few_probe<E>({N, D, V, x, w, c.b, c.y}, part, spread, target, groups, st);
    if (e == hipSuccess) {
      hipLaunchKernelGGL(join_probe_few, dim3(N), dim3(256), 0, st, part, spread, (int)ceil_div(V, wn_few_classes(sp, N, D, V)), rows);
      e = hipGetLastError();
    }
    if (e == hipSuccess && c.top) {
      alt.count = (int)ceil_div(V, 8);
      alt.last = 1;
      e = launch_alternatives<E>(alt, st);
    }
    return e == hipSuccess ? WN_OK : wn_set_last_error(WN_EHIP, hipGetErrorString(e));
  }
  int* const ex = reinterpret_cast<int*>(ws + f.ex);
  int* const ew = reinterpret_cast<int*>(ws + f.ew);
  RowPacker<E> pack;
  const Operand ox = pack.add(x, N, D, reinterpret_cast<u16*>(ws + f.x), ex);
  const bool direct = !sp && D % 8 == 0 && reinterpret_cast<uintptr_t>(w) % 16 == 0;
  const int piece = direct ? probe_piece(N, V, 0, c.top) : f.piece;
  int tiles = 0;
  hipError_t e = hipSuccess;
  for (int v0 = 0; v0 < V && e == hipSuccess; v0 += piece) {
    const int n = std::min(piece, V - v0);
    const Operand ow = pack.add(w + (size_t)v0 * D, n, D, reinterpret_cast<u16*>(ws + f.w), ew);
    pack.launch(st);
    const bool big = shape_for(n, N, ox.k, sp, false).big;
    const ProbeEnd end{{sp ? ex : nullptr, sp ? ew : nullptr, c.b ? c.b + v0 : nullptr, c.y, N, n, v0, V}, part, spread, tiles, target, groups};
    e = run_product<sp>({ow, ox, 0, 0, 1, 0}, big, end, st);
    tiles += (int)ceil_div(n, big ? 256 : 128);
    alt.count = (int)ceil_div(n, 8);
    alt.first = v0 / 8;
    alt.last = v0 + n == V;
    if (e == hipSuccess && alt.last) {
      hipLaunchKernelGGL(join_probe, dim3((unsigned)ceil_div(N, 16)), dim3(256), 0, st, part, spread, tiles, rows);
      e = hipGetLastError();
    }
    if (e == hipSuccess && c.top) e = launch_alternatives<E>(alt, st);
    alt.seen = 1;
  }
  return e == hipSuccess ? WN_OK : wn_set_last_error(WN_EHIP, hipGetErrorString(e));
}

}  // namespace

extern "C" {

size_t wn_logprobs_workspace_bytes(int32_t dtype, int32_t N, int32_t D, int32_t V, int32_t top) {
  if (!sizes_ok(dtype, N, D, V) || N == 0 || top < 0 || top > std::min(kMostTop, V)) return 0;
  return Probe(dtype == WN_F32, N, D, V, top).total;
}

int wn_logprobs(int32_t dtype, int32_t N, int32_t D, int32_t V, int32_t top, const void* x, const void* w, const float* b,
                const int32_t* y, float* logprob, float* entropy, float* lse, int32_t* top_ids, float* top_logprobs,
                void* workspace, size_t ws_bytes, void* stream) {
  wn_clear_last_error();
  int rc = check_sizes(dtype, N, D, V);
  if (rc != WN_OK) return rc;
  if (top < 0 || top > std::min(kMostTop, V)) return wn_set_last_error(WN_EINVAL, "top must be 0..32 and at most V");
  if (N == 0) return WN_OK;
  if (!x || !w || !y || !logprob || !entropy || !lse || (top && (!top_ids || !top_logprobs)))
    return wn_set_last_error(WN_EINVAL, "null pointer");
  rc = bad_workspace(workspace, ws_bytes, wn_logprobs_workspace_bytes(dtype, N, D, V, top));
  if (rc != WN_OK) return rc;
  ArrayScope scope;
  const struct { const void* p; const char* name; } arrays[] = {
      {x, "x"}, {w, "w"}, {b, "b"}, {y, "y"}, {logprob, "logprob"}, {entropy, "entropy"}, {lse, "lse"},
      {top ? top_ids : nullptr, "top_ids"}, {top ? top_logprobs : nullptr, "top_logprobs"}, {workspace, "workspace"}};
  for (const auto& a : arrays)
    if (a.p && (rc = scope.check(a.p, a.name)) != WN_OK) return rc;
  if ((rc = scope.enter()) != WN_OK) return rc;
  char* const ws = static_cast<char*>(workspace);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const ProbeCall c{N, D, V, top, b, y, logprob, entropy, lse, top_ids, top_logprobs};
  if (dtype == WN_F32) return run_probe(c, static_cast<const float*>(x), static_cast<const float*>(w), ws, st);
  return run_probe(c, static_cast<const u16*>(x), static_cast<const u16*>(w), ws, st);
}

}  // extern "C"
