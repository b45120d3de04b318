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
// searched for a few more than K (kept()), and their classes' logits are computed anew: in 32 bits with a bound of their
// rounding, and those in 64 that may be among the K by it.  (Of up to 1024 classes each is a group by itself, see group_of.)
// So the logits of many classes are neither kept nor sorted, classes next to each other are in order although the product's
// sums are of 32 bits, and equal ones (copies of a row of w) are equal: the lowest index comes first.
#include "wn_product.h"

namespace {

constexpr int kMostTop = 32;
constexpr size_t kGroupsBytes = (size_t)256 << 20;  // of the groups' largest logits of a piece: they stay in the last-level cache

// Groups of 8 classes kept for `top` alternatives: more than `top`, since a group's largest logit is off by the product's
// rounding.  Classes are missed only if more groups than the surplus lie within that rounding of the last one wanted.  (Of a
// group that is kept every class may be an alternative.)
__host__ __device__ constexpr int kept(int top) { return top + 2 + top / 8; }
static_assert(kept(kMostTop) <= 64, "a lane for each");

// Bound: the product, as in the loss.  Measured: 8192 rows x 65536 classes x 2048 in bf16 1.72 to 1.78 ms (the loss's end 1.69
// to 1.78), 4096 x 65536 x 1024 with alternatives 546 to 595 us, 16000 x 256 x 256 in fp32 17 (without 14.5).
struct ProbeEnd {
  static constexpr bool kScaledByTile = false;
  Logits l;
  float2* part;    // [tiles of all pieces][N]: m and s
  float* spread;   // t
  int tile0;       // the piece's first
  float* target;   // [N]
  float* groups;   // [N][ceil(l.V / 8)] or [N][l.V], or null
  int per;         // classes of a group: 8 or 1
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
      if (groups && per == 1) {
#pragma unroll
        for (int i = 0; i < T::NA; ++i) {
          const int v = pl.a0 + 16 * i + 4 * pl.quad;
          float* const at = groups + (size_t)n * l.V + v;
          if (n < l.N && v + 3 < l.V) {
            *reinterpret_cast<f32x4u*>(at) = f32x4u{acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
          } else if (n < l.N) {
#pragma unroll
            for (int e = 0; e < 3; ++e)
              if (v + e < l.V) at[e] = acc[i][j][e];
          }
        }
      } else if (groups) {
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
  // (a block's first thread writes; the others get log s too)
  __device__ __forceinline__ float put(int n, const WnStat& o, bool write = threadIdx.x == 0) const {
    const float z = logf(o.s);
    if (!write) return z;
    const int t = y[n];
    lse[n] = o.m + z;
    logprob[n] = t >= 0 && t < V ? (target[n] - o.m) - z : 0.f;  // (in this order log s is not lost beside a large m)
    entropy[n] = z - o.t / o.s;
    log_s[n] = z;
    return z;
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
  r.put(n, o, true);
}

// A row's parts joined by a block; every thread gets them.
template <int kThreads>
__device__ __forceinline__ WnStat join_tiles(const float2* part, const float* spread, int tiles, int N, int n) {
  __shared__ WnStat s[kThreads / 64];
  WnStat o{-INFINITY, 0.f, 0.f};
#pragma unroll 4
  for (int t = threadIdx.x; t < tiles; t += kThreads) {
    const float2 p = part[(size_t)t * N + n];
    o.add({p.x, p.y, spread[(size_t)t * N + n]});
  }
  for (int d = 32; d; d >>= 1) o.add({__shfl_xor(o.m, d, 64), __shfl_xor(o.s, d, 64), __shfl_xor(o.t, d, 64)});
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = o;
  __syncthreads();
  o = s[0];
  for (int w = 1; w < kThreads / 64; ++w) o.add(s[w]);
  return o;
}

// For few rows, without alternatives: a block per row.
__global__ __launch_bounds__(256) void join_probe_few(const float2* part, const float* spread, int tiles, const RowOut r) {
  r.put(blockIdx.x, join_tiles<256>(part, spread, tiles, r.N, blockIdx.x));
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

__device__ __forceinline__ bool before(const Group& a, const Group& b) { return a.v > b.v || (a.v == b.v && a.g < b.g); }

// The `want` largest of a wave's R entries a lane, by value and then by the lower number: lane r ends with the r-th.
template <int R>
__device__ __forceinline__ Group largest_of(Group (&e)[R], int want) {
  const int lane = threadIdx.x & 63;
  Group mine{-INFINITY, kNone};
  for (int r = 0; r < want; ++r) {
    Group b = e[0];
#pragma unroll
    for (int k = 1; k < R; ++k)
      if (before(e[k], b)) b = e[k];
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
  int per;              // classes of a group: 8 or 1
  int count, first;     // its groups, the number of the first
  int N, D, V, top;
  const void *x, *w;
  const float* b;       // or null
  const float* log_s;   // [N]
  Group* list;          // [N][kept(top)] from piece to piece
  int seen, last;       // 0: list is empty; the last piece
  const float2* part;   // few rows: a row's statistics are joined here; or null
  const float* spread;
  int tiles;
  RowOut rows;
  int32_t* ids;         // [N][top]
  float* logprobs;
};
constexpr int kSegment = 16;  // groups a lane looks at together
constexpr int kMostKept = kept(kMostTop);

// A wave's segment of up to 64 kSegment groups (v[k] of group first + 64 k + lane, `left` of them) joined with the list `mine`,
// of which lane r holds the r-th largest.  The want-th largest of the lanes' largest values is one that at least want groups
// reach, so only groups that reach it are looked at again: a few more than want, unless many are equal.
__device__ __forceinline__ Group join_segment(const float (&v)[kSegment], int first, int left, Group mine, int want, Group* room) {
  const int lane = threadIdx.x & 63;
  float most = v[0];
#pragma unroll
  for (int k = 1; k < kSegment; ++k) most = fmaxf(most, v[k]);
  // (numbers rise from segment to segment, so an equal value comes behind those kept)
  const Group least{__shfl(mine.v, want - 1, 64), __shfl(mine.g, want - 1, 64)};
  if (least.g != kNone && !__any(most > least.v)) return mine;
  const int had = __popcll(__ballot(mine.g != kNone));
  // the list, then the groups that reach t (with a full list: its least, while few do)
  float t = least.v;
  auto reach = [&]() {
    int n = had;
#pragma unroll
    for (int k = 0; k < kSegment; ++k) n += __popcll(__ballot(v[k] >= t && k * 64 + lane < left));
    return n;
  };
  int n = 65;
  if (least.g != kNone) n = reach();
  if (n > 64) {
    for (int r = 0; r < want; ++r) {
      t = wnk::wave_max(most);
      if (lane == __ffsll(__ballot(most == t)) - 1) most = -INFINITY;
    }
    t = fmaxf(t, least.v);  // (-infinity without a full list)
    n = reach();
  }
  if (n > 64) {  // (many equal ones, or many of one lane)
    Group e[kSegment + 1];
#pragma unroll
    for (int k = 0; k < kSegment; ++k) e[k] = k * 64 + lane < left ? Group{v[k], first + k * 64 + lane} : Group{-INFINITY, kNone};
    e[kSegment] = mine;
    return largest_of(e, want);
  }
  if (mine.g != kNone) room[lane] = mine;
  n = had;
#pragma unroll
  for (int k = 0; k < kSegment; ++k) {
    const bool in = v[k] >= t && k * 64 + lane < left;
    const unsigned long long all = __ballot(in);
    if (in) room[n + __popcll(all & ((1ull << lane) - 1))] = {v[k], first + k * 64 + lane};
    n += __popcll(all);
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the wave's own part of LDS)
  const Group e = lane < n ? room[lane] : Group{-INFINITY, kNone};
  int rank = 0;
  for (int k = 0; k < n; ++k) {
    const Group o{__builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, e.v), k)), __builtin_amdgcn_readlane(e.g, k)};
    rank += before(o, e);
  }
  asm volatile("" ::: "memory");  // (every entry has been read)
  if (lane < n && rank < want) room[rank] = e;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  return lane < want && lane < n ? room[lane] : Group{-INFINITY, kNone};
}

// C classes' logits, summed in S by a wave: lanes 64 / C c .. of it end with class v[c]'s.  `size`, in 32 bits: sum |x w| over all
// C, of which each class's is a part.
template <class E, class S, int C, int kAhead>
__device__ __forceinline__ S class_logits(const Alternatives& a, int n, const int (&v)[C], float* size = nullptr) {
  constexpr int W = Piece<E>::n;
  const int lane = threadIdx.x & 63;
  const E* x = static_cast<const E*>(a.x) + (size_t)n * a.D;
  const E* w[C];
  S sum[C];
  float all[2] = {0.f, 0.f};
#pragma unroll
  for (int c = 0; c < C; ++c) {
    sum[c] = 0;
    w[c] = static_cast<const E*>(a.w) + (size_t)v[c] * a.D;
  }
  auto add = [&](const P<E>& xv, const P<E> (&wv)[C]) {
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const S xs = value(xv[k]);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        sum[c] += xs * (S)value(wv[c][k]);
        if (size) all[c & 1] = fmaf(fabsf(value(xv[k])), fabsf(value(wv[c][k])), all[c & 1]);
      }
    }
  };
  const int whole = a.D / (64 * W) * (64 * W);
#pragma unroll kAhead
  for (int k = lane * W; k < whole; k += 64 * W) {
    P<E> wv[C];
#pragma unroll
    for (int c = 0; c < C; ++c) wv[c] = whole_piece(w[c] + k);
    add(whole_piece(x + k), wv);
  }
  if (const int k = whole + lane * W; k < a.D) {
    P<E> wv[C];
#pragma unroll
    for (int c = 0; c < C; ++c) wv[c] = piece_at(w[c] + k, a.D - k);
    add(piece_at(x + k, a.D - k), wv);
  }
  // halves of the lanes take halves of the classes until each has one; then the lanes of a class add up
#pragma unroll
  for (int h = C / 2; h; h >>= 1) {
    const int d = h * 64 / C;
    const bool up = lane & d;
#pragma unroll
    for (int c = 0; c < C / 2; ++c)
      if (c < h) {
        const S give = up ? sum[c] : sum[c + h], keep = up ? sum[c + h] : sum[c];
        sum[c] = keep + __shfl_xor(give, d, 64);
      }
  }
  S s = sum[0];
#pragma unroll
  for (int d = 32 / C; d; d >>= 1) s += __shfl_xor(s, d, 64);
  int mine = v[0];
#pragma unroll
  for (int c = 1; c < C; ++c) mine = lane / (64 / C) == c ? v[c] : mine;
  if (a.b) s += (S)a.b[mine];
  if (size) *size = wnk::wave_sum(all[0] + all[1]);
  return s;
}
// A class's logit of 32 bits is off by `off`, in its sum, and by the roundings of the bias's addition and of what is computed
// here, 2^-22 of itself: it lies between these two.  (An infinity stays one.)
__device__ __forceinline__ float at_least(float l, float off) { return fminf(l * (1.f - 0x1p-22f), l * (1.f + 0x1p-22f)) - off; }
__device__ __forceinline__ float at_most(float l, float off) { return fmaxf(l * (1.f - 0x1p-22f), l * (1.f + 0x1p-22f)) + off; }

// A block per row.  The waves find the largest groups of their segments, which are then joined; in the last piece, unless
// the groups are single classes, they compute the logits of these groups' classes in 32 bits.  At least `top` of them are at
// least at_least() of the top-th largest, so a class that is less at most is none of the alternatives; the others, hardly more than
// `top` unless classes are nearly alike, are computed in 64 and ranked by counting.  For few rows the block joins its row's
// statistics first.
// Bound: many rows by reading the groups and the classes' rows of w (4096 rows x 65536 classes x 1024, bf16, 8 alternatives: 134 MB
// and 0.74 GB, most of it from the caches, 177 us; 16000 x 256 x 256 in fp32, 3: 38); few rows by a chain of some ten reads and
// reductions (1 x 32000 x 2048, bf16, 5: 23 us).
template <class E, int kWaves>
__global__ __launch_bounds__(64 * kWaves, kWaves == 1 ? 5 : kWaves <= 4 ? 6 : 2) void alternatives(const Alternatives a) {
  constexpr int kThreads = 64 * kWaves, kAhead = kWaves <= 4 ? 1 : 2;
  __shared__ Group found[(kWaves + 1) * kMostKept], best[kMostKept], room[kWaves][64];
  __shared__ union { Group near[kMostKept * 8]; double logit[kMostKept * 8]; } s;  // (near is done with before the first logit)
  __shared__ Group pick[kMostKept * 8];  // classes by their logits in 32 bits, the largest first
  __shared__ float top_of[kMostKept], size_of[kMostKept];
  __shared__ int many;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = blockIdx.x, want = kept(a.top);
  float z = 0.f;
  if (a.part) z = a.rows.put(n, join_tiles<kThreads>(a.part, a.spread, a.tiles, a.N, n));
  const float* groups = a.groups + (size_t)n * a.count;
  Group mine{-INFINITY, kNone};
  for (int at = wave * 64 * kSegment; at < a.count; at += kThreads * kSegment) {
    float v[kSegment];
#pragma unroll
    for (int k = 0; k < kSegment; ++k) {
      const int i = at + k * 64 + lane;
      v[k] = fmaxf(i < a.count ? groups[i] : -INFINITY, -INFINITY);  // (a NaN would be neither before nor behind another)
    }
    mine = join_segment(v, a.first + at, a.count - at, mine, want, room[wave]);
  }
  if (a.count <= 64 * kSegment && !a.seen) {
    if (tid < want) best[tid] = mine;
  } else {
    if (lane < want) found[wave * want + lane] = mine;
    if (tid < want) {
      found[kWaves * want + tid] = a.seen ? a.list[(size_t)n * want + tid] : Group{-INFINITY, kNone};
      best[tid] = {-INFINITY, kNone};
    }
    __syncthreads();
    // An entry's rank: how many of each list, all sorted, are before it.  (Compared with every entry, one after the other in
    // LDS, 1 row x 32000 classes x 2048 with 20 alternatives took 19 us longer, 37 x 50021 x 777 with 20 18.)
    const int all = (kWaves + 1) * want;
    for (int i = tid; i < all; i += kThreads) {
      const Group e = found[i];
      int ahead[kWaves + 1];
#pragma unroll
      for (int l = 0; l <= kWaves; ++l) ahead[l] = 0;
#pragma unroll 1
      for (int h = 32; h; h >>= 1)
#pragma unroll
        for (int l = 0; l <= kWaves; ++l) {
          // (Without a branch: given `if (k <= want && before(o, e)) ahead[l] = k` with nine lists, hipcc 7.2 keeps `ahead` in one run
          // of registers and copies the old run on the path where the values are equal and o's number is lower, so equal entries
          // got the same rank.  A kernel of this loop alone does so at -O1 to -O3, not at -O0, and not with two lists.)
          const int k = ahead[l] + h;
          const Group o = found[l * want + min(k, want) - 1];
          const int in = (int)(k <= want) & ((int)(o.v > e.v) | ((int)(o.v == e.v) & (int)(o.g < e.g)));
          ahead[l] += in * h;
        }
      int rank = 0;
#pragma unroll
      for (int l = 0; l <= kWaves; ++l) rank += ahead[l];
      if (e.g != kNone && rank < want) best[rank] = e;
    }
  }
  __syncthreads();
  if (!a.last) {
    if (tid < want) a.list[(size_t)n * want + tid] = best[tid];
    return;
  }
  const bool single = a.per == 1;  // (then the groups are the classes themselves)
  const Group* const chosen = single ? best : pick;
  int picked = min(a.V, want);
  if (!single) {
    for (int k = wave; k < want; k += kWaves) {
      const int g = best[k].g, c = lane >> 3;
      Group e{-INFINITY, kNone};
      float size = 0.f;
      if (g != kNone) {
        int v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = min(g * 8 + i, a.V - 1);
        const float l = class_logits<E, float, 8, kAhead>(a, n, v, &size);
        if (g * 8 + c < a.V) e = {fmaxf(l, -INFINITY), g * 8 + c};
      }
      if ((lane & 7) == 0) s.near[k * 8 + c] = e;
      const float m = wnk::wave_max(e.v);
      if (lane == 0) top_of[k] = m, size_of[k] = size;
    }
    __syncthreads();
    if (wave == 0) {
      // A lane adds up D / 64 terms and a piece at most, then come 6 sums of lanes.  (Where it overflows every class stays in.)
      const float size = wnk::wave_max(lane < want ? size_of[lane] : 0.f), off = (float)(a.D / 64 + 16) * 0x1.04p-24f * size;
      // as many classes as groups reach the least of the groups' largest
      const float t = -wnk::wave_max(lane < want ? -top_of[lane] : -INFINITY), low = at_least(t, off);
      int m = 0;
      for (int i = 0; i < want * 8; i += 64) {
        const Group e = i + lane < want * 8 ? s.near[i + lane] : Group{-INFINITY, kNone};
        const bool in = e.g != kNone && !(at_most(e.v, off) < low);
        const unsigned long long all = __ballot(in);
        asm volatile("" ::: "memory");
        if (in) s.near[m + __popcll(all & ((1ull << lane) - 1))] = e;  // (never behind what is still to be read)
        m += __popcll(all);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      for (int i = lane; i < m; i += 64) {
        const Group e = s.near[i];
        int rank = 0;
#pragma unroll 8
        for (int k = 0; k < m; ++k) rank += before(s.near[k], e);
        pick[rank] = e;
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      // (Where fewer than top are left of a mask, the last one is the mask's value: if the products are nothing beside it in 64 bits
      // either, 32 have the masked classes in order already.)
      const float last = pick[a.top - 1].v, low_last = at_least(last, off);
      int c = 0;
      if (fabsf(last) >= size * 0x1p55f) c = a.top;
      else
        for (int i = 0; i < m; i += 64) c += __popcll(__ballot(i + lane < m && !(at_most(pick[min(i + lane, m - 1)].v, off) < low_last)));
      if (lane == 0) many = c;
    }
    __syncthreads();
    picked = many;
  }
  for (int k = wave * 4; k < picked; k += kWaves * 4) {
    int v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = chosen[min(k + i, picked - 1)].g;
    const double l = class_logits<E, double, 4, kAhead>(a, n, v);
    if ((lane & 15) == 0 && k + (lane >> 4) < picked)
      s.logit[k + (lane >> 4)] = l == l ? l : -INFINITY;  // (where a logit is a NaN, log s is, and so is what comes out)
  }
  __syncthreads();
  if (!a.part) z = a.log_s[n];
  for (int i = tid; i < picked; i += kThreads) {
    const int v = chosen[i].g;
    const double l = s.logit[i];
    int rank = 0;
    double most = -INFINITY;
#pragma unroll 4
    for (int k = 0; k < picked; ++k) {
      const int o = chosen[k].g;
      const double ol = s.logit[k];
      rank += ol > l || (ol == l && o < v);
      most = fmax(most, ol);
    }
    if (rank >= a.top) continue;
    a.ids[(size_t)n * a.top + rank] = v;
    // (the row's largest logit is taken off as it is here, not as the product rounded it: no log probability is above 0)
    a.logprobs[(size_t)n * a.top + rank] = (float)((l - most) - (double)z);
  }
}

// ------------------------------------------------------------------------------------------------
// Host
// ------------------------------------------------------------------------------------------------
// Classes of a group.  Where one segment holds a row's logits, they are kept and searched themselves, which costs less than
// the logits of eight classes for each one wanted.  Groups of 8 and of 1 (us a call): 16000 rows x 256 classes x 256 in fp32, 3
// alternatives 84 and 59, in bf16 20 of them 294 and 107; 16000 x 1024 x 256, 5: 121 and 78; 300 x 1000 x 1024, 20: 48 and 36;
// 2000 x 1024 x 64, 5: 34 and 28; but 16000 x 1030 x 256, 5: 139 and 229, and few rows gain nothing (64 x 1000 x 1024, 5: 25
// and 25; 1 x 2048 x 2048: 20 and 27).
int group_of(int N, int V) { return N > kFewRows && V <= 64 * kSegment && (size_t)N * V * 4 <= kGroupsBytes ? 1 : 8; }

// Classes of a piece; `each` as for forward_piece.
int probe_piece(int N, int V, size_t each, int top) {
  const int most = forward_piece(N, V, each);
  if (!top) return most;
  const size_t fit = std::max<size_t>(256, kGroupsBytes / 4 * group_of(N, V) / N / 256 * 256);
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
    groups = c.take(top ? (size_t)N * ceil_div(few ? V : probe_piece(N, V, 0, top), group_of(N, V)) * 4 : 0);
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

// Waves of a row.  Few rows leave the chip empty, so a row takes many; many rows of few groups take one each, which has no
// other to wait for.  Measured with 1, 4 and 8 waves (us beside the call without alternatives): 1 row x 32000 classes x
// 2048, 5 alternatives 58, 22, 19 and 20 of them 133, 44, 35; 37 x 50021 x 777 in fp32, 20: 144, 54, 37; 128 x 32000 x 1024 in
// fp32, 5: 61, 34, 35; 300 x 32000 x 1024, 5: 51, 24, 39; 1000 x 32000 x 1024, 20: 118, 83, 135; 4096 x 65536 x 1024, 8: 220,
// 191, 394; 16000 x 256 x 256 in fp32, 3: 31, 74, 364.  The chip holds 1536 blocks of 4 waves at a time, and rows of one segment
// beyond that take one wave (1 and 4): 1536 x 1000 x 1024, 20 31 and 28, 1537 of them 31 and 36; 1536 x 8000 x 1024, 5 38 and 37,
// 1537 39 and 45.
template <class E>
hipError_t launch_alternatives(const Alternatives& a, hipStream_t st) {
  if (a.N <= 128) hipLaunchKernelGGL((alternatives<E, 8>), dim3(a.N), dim3(512), 0, st, a);
  else if (a.N <= 1536 || a.count > 64 * kSegment) hipLaunchKernelGGL((alternatives<E, 4>), dim3(a.N), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((alternatives<E, 1>), dim3(a.N), dim3(64), 0, st, a);
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
  const int per = group_of(N, V);
  Alternatives alt{groups, per, 0, 0, N, D, V, c.top, x, w, c.b, log_s, reinterpret_cast<Group*>(ws + f.list), 0, 0, nullptr, nullptr, 0, rows,
                   c.ids, c.top_logprobs};
  if (N <= kFewRows) {
    hipError_t e = wn_few_probe<E>({N, D, V, x, w, c.b, c.y}, part, spread, target, groups, st);
    const int tiles = (int)ceil_div(V, wn_few_classes(sp, N, D, V));
    if (e == hipSuccess && !c.top) {
      hipLaunchKernelGGL(join_probe_few, dim3(N), dim3(256), 0, st, part, spread, tiles, rows);
      e = hipGetLastError();
    }
    if (e == hipSuccess && c.top) {
      alt.count = (int)ceil_div(V, per);
      alt.last = 1;
      alt.part = part;
      alt.spread = spread;
      alt.tiles = tiles;
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
    const ProbeEnd end{{sp ? ex : nullptr, sp ? ew : nullptr, c.b ? c.b + v0 : nullptr, c.y, N, n, v0, V}, part, spread, tiles, target, groups, per};
    e = run_product<sp>({ow, ox, 0, 0, 1, 0}, big, end, st);
    tiles += (int)ceil_div(n, big ? 256 : 128);
    alt.count = (int)ceil_div(n, per);
    alt.first = v0 / per;
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
