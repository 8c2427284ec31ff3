// swiftkv_verify_drafts: which drafted tokens stand against the target's probabilities, and the token behind them.
//
// With w_v = 2^((z_v - m) c), c = log2(e) / T, m the row's largest logit and S = sum w, a drafted token stands if u (S - R) < w (R: brothers that
// fell before it) or, with the drafter's probabilities, u q S < w; the next token is the first v whose prefix sum of r (w without the
// fallen, or max(w - S q, 0)) exceeds u sum r.
//
// A cluster of blocks walks one sequence: every block has its part of the vocabulary, and only rows on the walk are read -- of a
// tree of 32 tokens some four -- and what the ring holds ahead of it along the first children.  Where a block's part of a row is small one exchange
// over distributed shared memory decides up to four rows.
//
// What bounds it: a sequence's chain of steps, not HBM.  Per group of rows an exchange and its verdicts (3 us), at the end one pass over the last row's
// weights in 64 bits, two with the drafter's probabilities (3 elements per clock and SM of the 4.9 that the 64-bit units give; 10 us each for 128256 logits in four
// blocks), and the search of the token (2.5 us).  Measured at 128256 bf16 logits (device time, graph): 1 sequence x 5 tokens 18 us, 8 x 8 27 us, 16 trees of
// up to 32 tokens 27 us, 64 x 8 with the drafter's probabilities 69 us (104 MB read), without 52 us, greedy 34 us; 256 x 6 fp32 of 100003 125 us (246 MB).  Tried and slower: a second
// kernel for the draw (64 x 8 76 - 94 us), a ninth warp that fills the ring (76 us, registers spill), blocks of 512 threads (68 - 88 us), two steps of a
// tile at once (74 us), the search over the pass's own code (75 us), three blocks per SM (89 us).
//
// Decisions are those of 64-bit arithmetic.  S, formed in 32 bits, is off by at most `unsure` relative to itself:
//   the difference z - r, its product with c and c itself are rounded (3 x 2^-24 |t| ln 2 relative, t the exponent; over a row the mean of |t| weighted
//   with w is at most log2(vocab) <= 30: 4e-6), the approximate exponential has 2^-22, a thread's sums have (32 + chunks) 2^-24, and its reference moves
//   at most once a chunk, and three times when parts are joined, by a factor that is off by 2^-22: 2^-16 + (chunks + 4) 2^-21 covers them.
//   A token's own w is off by 1.3e-7 |t|, at most 1.6e-5 where it is not zero; where it is, it is below 2^-126.
// A decision whose two sides are nearer to each other than twice that (and than 2^-126) is taken again with the row's sum in 64 bits (a few in 10^4).
// A token is drawn from sums in 64 bits: the borders between tokens lie 1 / vocab apart, nearer than 32 bits resolve.  The power of
// two is there 2^(n / 16), of a table of 16, times a polynomial of the 5th degree (1e-14): 13 operations of the 64-bit units for
// a token instead of 18 without the table.
#include <cooperative_groups.h>

#include <atomic>
#include <type_traits>

#include "logits_common.cuh"

namespace skv {
namespace {
namespace cg = cooperative_groups;
using tc::F2;
using tc::add2;
using tc::mul2;

constexpr int VD_THREADS = 256, VD_WARPS = VD_THREADS / 32;
constexpr int VD_UNROLL = 4;                 // 16-byte vectors of a chunk per thread
constexpr int VD_CHUNK = VD_THREADS * VD_UNROLL;
constexpr int VD_STAGES = 4;                 // chunks of the ring
constexpr int VD_MAX_NEW = 1024;
constexpr int VD_MAX_CLUSTER = 16;
constexpr int VD_GROUP = 4;                  // rows that one exchange may decide
constexpr int VD_TILES = 1024;               // parts of a block's part of a row whose sums are kept for the draw
constexpr int NO_CHILD = 0x7fffffff;
// Temperatures: a denormal logit, which counts as 0, must not matter; and a difference of two logits that is not must have no probability
constexpr float VD_COLDEST = 0x1p-64f, VD_HOTTEST = 0x1p100f;

struct VdArgs {
  const void *logits;
  long long stride, draft_stride;
  const int32_t *tokens, *cu, *parents;
  const float *draft, *uniforms, *temperatures;
  float temperature;
  int total, max_new, vocab, log_splits, group;
  float unsure;
  int32_t *n_accepted, *tokens_out, *path;
  unsigned int *status;
};

// a part of a row: its largest logit, sum of w relative to it, and (T = 0) the lowest index of the largest
struct VdPart { float m, l; int idx; };
enum : int { VD_MOVE, VD_DRAW, VD_EXACT, VD_GREEDY, VD_DONE };
// what a row says of the drafted tokens behind it: the place of the first that stands, or one of these
enum : int { VD_NONE = -1, VD_UNSURE = -2, VD_UNCLEAR = -3 };      // none; 32 bits do not decide; a row without probabilities
struct VdVerdict { int to, best; float m; };                       // best (T = 0): the largest logit's token

struct VdWeights {      // what a token's weight in the draw is made of
  double m, c, s;       // the row's largest logit, log2(e) / T, and with q the row's sum
  const float *q;       // the fallen token's distribution, or null
  int n_tried;          // tokens of `tried` that have none
  float low;            // the logit whose weight is 2^-1000: below it there is none
};

struct VdShared {
  double sum[2][VD_MAX_CLUSTER];
  double root[16];                             // 2^(i / 16)
  double tile[VD_TILES];
  double step_sum[VD_WARPS];
  VdWeights k;
  VdPart part[2][VD_GROUP][VD_MAX_CLUSTER];
  float2 thread_part[VD_GROUP][VD_THREADS];    // the threads' parts of the rows of a group: largest, and sum or (as a whole number) the chunk that has it
  VdVerdict verdict[VD_GROUP];
  uint64_t full[VD_STAGES], empty[VD_STAGES];
  double before;
  int to, fetched, last;
};
// a sequence's drafted tokens: arrays of max_new entries behind the ring
struct VdDrafts {
  int *token, *first, *next, *path, *tried;    // first: a token's first child; next: its next brother
  float *u, *z, *q;                            // its random number, its logit in its parent's row, and what the drafter gave it
};
constexpr int VD_ARRAYS = 8;

// 2^t for -1000 <= t <= 0.  2^0 is 1, so that equal logits have equal whole weights.
constexpr int VD_ROOTS = 16;                   // (16 numbers of 64 bits lie in banks of their own)
__device__ __forceinline__ double exp2_64(const double *root, double t) {
  // e^x = 1 + x + ... + x^5 / 120 for |x| <= A, with x^5 / 720 of the next term replaced by what its Chebyshev polynomial leaves
  constexpr double L = 0.693147180559945309417, A = L / (2 * VD_ROOTS);
  constexpr double C1 = L, C2 = (1.0 / 2 - A * A * A * A * 5 / 16 / 720) * L * L, C3 = L * L * L / 6, C4 = (1.0 / 24 + A * A * 20 / 16 / 720) * L * L * L * L, C5 = L * L * L * L * L / 120;
  constexpr double ROUND = 6755399441055744.0 / VD_ROOTS;      // 1.5 2^52 / 16: adding it leaves the nearest multiple of 1/16, in 16ths in the low word
  const double r = t + ROUND, f = t - (r - ROUND);
  double p = fma(f, C5, C4);
  p = fma(f, p, C3);
  p = fma(f, p, C2);
  p = fma(f, p, C1);
  p = fma(f, p, 1.0);
  const int n = __double2loint(r);
  p *= root[n & (VD_ROOTS - 1)];
  return __hiloint2double(__double2hiint(p) + ((n >> 4) << 20), __double2loint(p));
}
// the weight of logit e, in 64 bits; low: the logit whose weight is 2^-1000, below which there is none
__device__ __forceinline__ double weight_64(const double *root, float e, double m, double c, float low) {
  const double w = exp2_64(root, ((double)e - m) * c);
  return e < low ? 0.0 : w;
}
__device__ __forceinline__ float lowest_64(double m, double c) { return __double2float_ru(m - 1000.0 / c); }

// A block's part of a row as the sums in 32 bits see it: elements before the row's first 16-byte boundary (head, the first block's), whole
// vectors [begin, end), elements behind them (the last block's)
template <typename T>
struct VdSpan {
  static constexpr int N = LpVec<T>::N;
  const T *x;
  int head, tail0, begin, end;
  __device__ __forceinline__ VdSpan(const VdArgs &a, long long row, int part) {
    x = reinterpret_cast<const T *>(a.logits) + row * a.stride;
    const int mis = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));
    head = min(a.vocab, mis ? N - mis : 0);
    const unsigned n = (unsigned)(a.vocab - head) / N;
    tail0 = head + (int)n * N;
    begin = (int)(((unsigned long long)n * part) >> a.log_splits);
    end = (int)(((unsigned long long)n * (part + 1)) >> a.log_splits);
  }
};
// ... and as the draw sees it, in the order of the tokens: units of 8 elements counted from the 16-byte boundary before the row (so that mis elements of the first
// are not the row's, nor are the last one's behind the vocabulary), in tiles of 32 `steps` units: four steps where every warp has a tile then (a tile's sum
// over the lanes costs as much as half a step), more where there would be over VD_TILES
template <typename T>
struct VdRow {
  static constexpr int N = 8, WORDS = N * sizeof(T) / 16;
  struct Unit { uint4 x[WORDS]; };
  const T *x;
  int vocab, mis, begin, end, steps, tiles;
  __device__ __forceinline__ VdRow(const VdArgs &a, long long row, int part) {
    x = reinterpret_cast<const T *>(a.logits) + row * a.stride;
    vocab = a.vocab;
    mis = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));
    const unsigned n = ((unsigned)vocab + mis + N - 1) / N;
    begin = (int)(((unsigned long long)n * part) >> a.log_splits);
    end = (int)(((unsigned long long)n * (part + 1)) >> a.log_splits);
    const int lines = (end - begin + 31) / 32;
    steps = max(min(4, (lines + VD_WARPS - 1) / VD_WARPS), (lines + VD_TILES - 1) / VD_TILES);
    tiles = steps ? (lines + steps - 1) / steps : 0;
  }
  __device__ __forceinline__ int element(int v, int i) const { return v * N - mis + i; }
  __device__ __forceinline__ bool inside(int v) const { return (v > 0 || mis == 0) && element(v, N) <= vocab; }
  // unit v; elements that are not the row's, and units that are not the part's, are -inf
  __device__ __forceinline__ Unit load(int v) const {
    Unit r;
    const T *at = x + element(v, 0);
    if (v < end && inside(v)) {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) r.x[i] = __ldg(reinterpret_cast<const uint4 *>(at) + i);
      return r;
    }
    const uint32_t none = no_logits<T>();
#pragma unroll
    for (int i = 0; i < WORDS; ++i) r.x[i] = make_uint4(none, none, none, none);
    T *e = reinterpret_cast<T *>(&r);
    if (v < end) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (element(v, i) >= 0 && element(v, i) < vocab) e[i] = at[i];
    }
    return r;
  }
  static __device__ __forceinline__ void unpack(const Unit &u, float (&e)[N]) {
    constexpr int M = LpVec<T>::N;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      float x[M];
      LpVec<T>::unpack(u.x[i], x);
#pragma unroll
      for (int j = 0; j < M; ++j) e[i * M + j] = x[j];
    }
  }
};

__device__ __forceinline__ double warp_sum64(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ double warp_prefix64(double v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double w = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += w;
  }
  return v;
}

// One warp: the weights of a lane's unit v; k says what they are made of.  LESS: w - s q.
template <typename T, bool LESS>
__device__ __forceinline__ void vd_weights(double (&w)[8], const double *root, const int *tried, const VdRow<T> &r, const typename VdRow<T>::Unit &raw, const float (&q)[8], int v,
                                           const VdWeights &k) {
  constexpr int N = 8;
  float e[N];
  VdRow<T>::unpack(raw, e);
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = exp2_64(root, ((double)e[i] - k.m) * k.c);
  const float least = fminf(fminf(fminf(e[0], e[1]), fminf(e[2], e[3])), fminf(fminf(e[4], e[5]), fminf(e[6], e[7])));
  if (least < k.low) {                           // (masked ones; what was formed of them is no number)
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (e[i] < k.low) w[i] = 0.0;
  }
  if (LESS) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      w[i] = fma(-k.s, (double)fmaxf(q[i], 0.f), w[i]);
      if (__double2hiint(w[i]) < 0) w[i] = 0.0;
    }
  } else {
    const int lane = threadIdx.x & 31, lo = r.element(v - lane, 0), hi = lo + 32 * N;      // (a warp's units lie side by side)
    for (int t0 = 0; t0 < k.n_tried; t0 += 32) {
      const int x = t0 + lane < k.n_tried ? tried[t0 + lane] : -1;
      for (unsigned hit = __ballot_sync(0xffffffffu, x >= 0 && x >= lo && x < hi); hit; hit &= hit - 1) {
        const int token = __shfl_sync(0xffffffffu, x, __ffs(hit) - 1);
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (r.element(v, i) == token) w[i] = 0.0;
      }
    }
  }
}
// the drafter's probabilities of unit v's tokens; whole: 16-byte loads are aligned
template <typename T>
__device__ __forceinline__ void vd_probs(float (&q)[8], const VdRow<T> &r, const float *from, int v, bool whole) {
  const float *at = from + r.element(v, 0);
  if (whole && v < r.end && r.inside(v)) {
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const float4 x = __ldg(reinterpret_cast<const float4 *>(at + i));
      q[i] = x.x; q[i + 1] = x.y; q[i + 2] = x.z; q[i + 3] = x.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = v < r.end && r.element(v, i) >= 0 && r.element(v, i) < r.vocab ? __ldg(at + i) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ bool vd_whole(const VdRow<T> &r, const float *q) { return ((reinterpret_cast<uintptr_t>(q) - 4 * r.mis) & 15) == 0; }

// all warps: the tiles' sums into sh.tile
template <typename T, bool LESS>
__device__ __forceinline__ void vd_tiles(VdShared &sh, const int *tried, const VdRow<T> &r) {
  using Unit = typename VdRow<T>::Unit;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const VdWeights k = sh.k;
  const bool whole = LESS && vd_whole(r, k.q);
  int t = warp, s = 0, tl = warp, sl = 0;       // the step that is looked at, and the one that is loaded
  auto unit_of = [&](int tile, int step) { return tile < r.tiles ? r.begin + (tile * r.steps + step) * 32 + lane : r.end; };
  auto load = [&]() {
    const Unit x = r.load(unit_of(tl, sl));
    if (++sl == r.steps) { sl = 0; tl += VD_WARPS; }
    return x;
  };
  Unit raw = load(), next = load(), third = load();
  float q[8], q_next[8];
  if (LESS) vd_probs(q_next, r, k.q, unit_of(t, 0), whole);
  double sum = 0.0;
#pragma unroll 1
  while (t < r.tiles) {
    const Unit later = load();
    const int v = unit_of(t, s);
    const bool ends = s + 1 == r.steps;
    if (LESS) {
#pragma unroll
      for (int i = 0; i < 8; ++i) q[i] = q_next[i];
      vd_probs(q_next, r, k.q, ends ? unit_of(t + VD_WARPS, 0) : unit_of(t, s + 1), whole);
    }
    double w[8];
    vd_weights<T, LESS>(w, sh.root, tried, r, raw, q, v, k);
#pragma unroll
    for (int n = 4; n > 0; n >>= 1)
#pragma unroll
      for (int i = 0; i < n; ++i) w[i] += w[i + n];
    sum += w[0];
    ++s;
    if (ends) {
      sum = warp_sum64(sum);
      if (lane == 0) sh.tile[t] = sum;
      sum = 0.0;
      s = 0;
      t += VD_WARPS;
    }
    raw = next;
    next = third;
    third = later;
  }
}
// one warp: every lane's stretch of n numbers (an odd number of them: no bank conflicts), its sum and the sum up to its end
struct VdStretch { int i0, i1; double sum, until; };
__device__ __forceinline__ VdStretch vd_stretch(const double *x, int n) {
  const int lane = threadIdx.x & 31, each = ((n + 31) / 32) | 1;
  VdStretch s{min(n, lane * each), min(n, (lane + 1) * each), 0.0, 0.0};
  for (int i = s.i0; i < s.i1; ++i) s.sum += x[i];
  s.until = warp_prefix64(s.sum);
  return s;
}
// all warps of the block that has it: the first token of the block's part at which the sum of the weights exceeds target (the last that has a weight where
// rounding leaves none); true in the one thread that found it.  Sums of the same numbers differ by how they are taken together, so each choice -- tile, step, lane,
// element -- is made among candidates that have a weight and does not lean on the choice before it: what lies before a tile counts as at most target, and the step
// is the one whose own two ends, each formed once, enclose it.
template <typename T>
__device__ __forceinline__ bool vd_find(VdShared &sh, const int *tried, const VdRow<T> &r, double target, int &token) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (warp == 0) {                               // the tile
    const VdStretch s = vd_stretch(sh.tile, r.tiles);
    const unsigned over = __ballot_sync(0xffffffffu, s.sum > 0.0 && s.until > target), some = __ballot_sync(0xffffffffu, s.sum > 0.0);
    const int who = over ? __ffs(over) - 1 : 31 - __clz(some | 1u);
    if (lane == who) {
      double sum = fmin(s.until - s.sum, target), before = sum;
      int tile = 0;
      for (int i = s.i0; i < s.i1; ++i) {
        const double w = sh.tile[i];
        if (!(w > 0.0)) continue;
        tile = i;
        before = sum;
        sum += w;
        if (sum > target) break;
      }
      sh.to = tile;
      sh.before = before;
      sh.last = -1;
    }
  }
  __syncthreads();
  const int tile = sh.to;
  double before = sh.before;
  const VdWeights k = sh.k;
  bool found = false;
  for (int s0 = 0; s0 < r.steps; s0 += VD_WARPS) {       // its steps, a warp each
    const int s = s0 + warp, v = s < r.steps ? r.begin + (tile * r.steps + s) * 32 + lane : r.end;
    const typename VdRow<T>::Unit raw = r.load(v);
    float q[8];
    double w[8], sum = 0.0;
    if (k.q) {
      vd_probs(q, r, k.q, v, vd_whole(r, k.q));
      vd_weights<T, true>(w, sh.root, tried, r, raw, q, v, k);
    } else {
      vd_weights<T, false>(w, sh.root, tried, r, raw, q, v, k);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += w[i];
    const double until = warp_prefix64(sum);
    if (lane == 31) sh.step_sum[warp] = until;
    __syncthreads();
    double base = before;
    for (int i = 0; i < warp; ++i) base += sh.step_sum[i];
    const bool here = !(base > target) && base + sh.step_sum[warp] > target;
    const unsigned over = __ballot_sync(0xffffffffu, sum > 0.0 && base + until > target), some = __ballot_sync(0xffffffffu, sum > 0.0);
    const int who = over ? __ffs(over) - 1 : 31 - __clz(some | 1u);
    if (some && lane == who) {
      double at = base + until - sum;
      int e = -1;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (e >= 0 && at > target) continue;
        at += w[i];
        if (w[i] > 0.0) e = r.element(v, i);
      }
      if (here) {
        token = e;
        found = true;
      } else {
        atomicMax(&sh.last, e);
      }
    }
    for (int i = 0; i < VD_WARPS; ++i) before += sh.step_sum[i];
    __syncthreads();
    if (before > target) return found;
  }
  if (threadIdx.x == 0) token = max(0, sh.last);
  return threadIdx.x == 0;
}

__device__ __forceinline__ float unit(float u) { return fminf(fmaxf(u, 0.f), 0.999999940395355f); }      // [0, 1), NaN counts as 0

// One warp: the drafted tokens behind node y one after the other; the first that stands, or what else there is to say.  total, m: the row's sum and
// largest logit.
template <bool EXACT, typename Sum>
__device__ __forceinline__ int vd_children(const VdDrafts &d, const double *root, const VdArgs &a, int n, int y, float m, Sum total, float c, double c64) {
  const int lane = threadIdx.x & 31;
  const bool certain = !a.draft;                               // the drafter gives its tokens all of the probability
  double gone = 0.0;
  for (int child = d.first[y]; child < n;) {
    const int from = child;
    int mine = NO_CHILD;
    for (int i = 0; i < 32 && child < n; ++i) {
      if (lane == i) mine = child;
      child = d.next[child];
    }
    const int token = mine < n ? d.token[mine] : -1 - lane;
    const bool is = mine < n && token >= 0 && token < a.vocab, several = from != d.first[y] || d.next[from] < n;
    bool again = false;                                        // of the same token twice the second has no weight left
    if (certain && several) {
      again = (__match_any_sync(0xffffffffu, token) & ((1u << lane) - 1u)) != 0;
      for (int t = d.first[y]; t != from; t = d.next[t]) again = again || d.token[t] == token;
    }
    Sum w = 0, u = 0;
    double q = 1.0;
    if (is) {
      const float z = d.z[mine];
      if (!again) w = EXACT ? (Sum)weight_64(root, z, (double)m, c64, lowest_64((double)m, c64)) : (Sum)exp2_approx((z - m) * c);
      u = (Sum)unit(d.u[mine]);
      q = (double)d.q[mine];
    }
    double sofar = 0.0;                                        // what fell before this one, in this turn of 32
    if (certain && several) sofar = warp_prefix64((double)w) - (double)w;
    const double left = certain ? (double)total - (gone + sofar) : (double)total * q;
    const double diff = (double)w - (double)u * left;
    const double near = EXACT ? 0.0 : 2.0 * a.unsure * ((double)w + (double)u * (certain ? (double)total : left)) + 0x1p-126;
    const unsigned stands = __ballot_sync(0xffffffffu, is && diff > near);
    const unsigned open = __ballot_sync(0xffffffffu, is && !EXACT && !(diff > near) && !(diff < -near) && !again);
    if (stands | open) {
      const int who = __ffs(stands | open) - 1;
      if (open >> who & 1) return VD_UNSURE;
      return __shfl_sync(0xffffffffu, mine, who);
    }
    if (child < n) gone += __shfl_sync(0xffffffffu, sofar + (double)w, 31);
  }
  return VD_NONE;
}

// one warp: parts of a row as one, the same bits in every block of the cluster
template <bool GREEDY>
__device__ __forceinline__ VdPart vd_join(VdPart p, float c) {
  VdPart r{p.m, p.l, p.idx};
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) r.m = max_nan(r.m, __shfl_xor_sync(0xffffffffu, r.m, o));
  if (GREEDY) {
    r.idx = (int)__reduce_min_sync(0xffffffffu, p.m == r.m || (p.m != p.m && r.m != r.m) ? p.idx : NO_CHILD);
  } else {
    if (p.m != r.m && p.l > 0.f) r.l *= exp2_approx((p.m - r.m) * c);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) r.l += __shfl_xor_sync(0xffffffffu, r.l, o);
  }
  return r;
}

template <typename T>
__global__ void __launch_bounds__(VD_THREADS, 2) verify_drafts_kernel(const __grid_constant__ VdArgs a) {
  constexpr int N = LpVec<T>::N;
  __shared__ VdShared sh;
  extern __shared__ __align__(128) uint8_t vd_ring[];      // [VD_STAGES][VD_CHUNK] vectors, then a sequence's drafted tokens
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int splits = 1 << a.log_splits, part = blockIdx.x & (splits - 1), b = blockIdx.x >> a.log_splits;
  const int begin = min(max(a.cu[b], 0), a.total), stop = min(max(a.cu[b + 1], begin), a.total), n = min(stop - begin, a.max_new);
  float temperature = a.temperatures ? a.temperatures[b] : a.temperature;
  const bool usable = temperature >= VD_COLDEST && temperature <= VD_HOTTEST;
  if (part == 0 && tid == 0 && (begin != a.cu[b] || stop != a.cu[b + 1] || n != stop - begin || (!usable && (__float_as_uint(temperature) << 1) != 0u))) atomicOr(a.status, STATUS_BAD_TOKEN);
  const bool greedy = !usable;
  const double c64 = greedy ? 0.0 : 1.4426950408889634074 / (double)temperature;
  const float c = (float)c64;
  int32_t *const out = a.tokens_out + (size_t)b * a.max_new, *const path = a.path + (size_t)b * a.max_new;
  if (n == 0) {                                        // (the same in every block of the cluster)
    if (part == 0) {
      for (int j = tid; j < a.max_new; j += VD_THREADS) out[j] = path[j] = -1;
      if (tid == 0) a.n_accepted[b] = 0;
    }
    return;
  }
  VdDrafts d;
  {
    int *at = reinterpret_cast<int *>(vd_ring + (size_t)VD_STAGES * VD_CHUNK * 16);
    d.token = at; d.first = at + a.max_new; d.next = at + 2 * a.max_new; d.path = at + 3 * a.max_new; d.tried = at + 4 * a.max_new;
    float *f = reinterpret_cast<float *>(at + 5 * a.max_new);
    d.u = f; d.z = f + a.max_new; d.q = f + 2 * a.max_new;
  }
  const bool producer = tid == VD_THREADS - 32;        // keeps the ring full (the first warps look up the drafted tokens meanwhile)
  if (producer) {
    for (int i = 0; i < VD_STAGES; ++i) {
      tc::mbar_init(tc::smem_u32(&sh.full[i]), 1);
      tc::mbar_init(tc::smem_u32(&sh.empty[i]), VD_WARPS);
    }
    tc::fence_barrier_init();
    tc::fence_proxy_async_smem();                      // (its copies are asked for before the block meets)
  }
  cluster.barrier_arrive();                            // (waited for before the first exchange: its blocks are there)
  bool alive = true;            // a wait that ran out (never, unless something is broken): no further waits or copies
  auto wait = [&](uint64_t *bar, uint32_t parity) {
    if (alive && !tc::mbar_wait(tc::smem_u32(bar), parity)) {
      alive = false;
      atomicOr(a.status, STATUS_TIMEOUT);
    }
  };
  const long long row0 = begin;
  // ---- the ring, filled along the first children: as many rows ahead as it holds
  int p_node = 0, p_v = 0, p_end = 0, p_stage = 0, p_use = 0, p_count = 0;
  const uint4 *p_src = nullptr;
  auto p_open = [&](int node) {
    for (p_node = node; p_node < n; p_node = d.first[p_node]) {
      const VdSpan<T> r(a, row0 + p_node, part);
      p_src = reinterpret_cast<const uint4 *>(r.x + r.head);
      p_v = r.begin;
      p_end = r.end;
      if (p_v < p_end) return;
    }
  };
  auto fetch = [&](bool known) {          // the next chunk, if there is one; known: what the tokens hang on has been read
    if (p_node >= n || p_v >= p_end || !alive) return;
    const uint32_t bar = tc::smem_u32(&sh.full[p_stage]);
    if (p_use > 0) wait(&sh.empty[p_stage], (p_use - 1) & 1);
    if (!alive) return;
    const uint32_t bytes = (uint32_t)min(VD_CHUNK, p_end - p_v) * 16;
    tc::mbar_expect_tx(bar, bytes);
    bulk_load(tc::smem_u32(vd_ring) + p_stage * VD_CHUNK * 16, p_src + p_v, bytes, bar);
    ++p_count;
    if (++p_stage == VD_STAGES) { p_stage = 0; ++p_use; }
    p_v += VD_CHUNK;
    if (p_v >= p_end && known) p_open(d.first[p_node]);
  };
  if (producer) {
    const VdSpan<T> r(a, row0, part);
    p_src = reinterpret_cast<const uint4 *>(r.x + r.head);
    p_v = r.begin;
    p_end = r.end;
    for (int i = 0; i < VD_STAGES - 1; ++i) fetch(false);
  }
  // ---- the sequence's drafted tokens
  const T *const rows0 = reinterpret_cast<const T *>(a.logits) + row0 * a.stride;
  for (int j = tid; j < n; j += VD_THREADS) {
    const int token = a.tokens[begin + j];
    int p = j - 1;
    if (a.parents && j > 0) {
      p = a.parents[begin + j];
      if (p < 0 || p >= j) {
        p = -1;
        if (part == 0) atomicOr(a.status, STATUS_BAD_TOKEN);
      }
    }
    d.token[j] = token;
    d.tried[j] = p;                                    // (the parents, until the walk begins)
    // a chain ends in front of an id that is none: it cannot stand, and nothing was drawn from its row of probabilities, which therefore does not go off the target
    if (a.parents || j == n - 1) d.first[j] = NO_CHILD;
    if (!a.parents && j > 0) d.first[j - 1] = token >= 0 && token < a.vocab ? j : NO_CHILD;
    d.next[j] = NO_CHILD;
    if (part == 0 && j > 0 && token >= a.vocab) atomicOr(a.status, STATUS_BAD_TOKEN);
    if (!greedy) {
      const bool is = p >= 0 && token >= 0 && token < a.vocab;
      d.u[j] = a.uniforms[begin + j];
      d.z[j] = is ? lp_load(rows0 + p * a.stride + token) : -INFINITY;
      d.q[j] = is && a.draft ? fmaxf(__ldg(a.draft + (row0 + j) * a.draft_stride + token), 0.f) : 1.f;
    }
  }
  if (warp == 1 && lane < VD_ROOTS) sh.root[lane] = exp2((double)lane / VD_ROOTS);
  if (tid == 0) d.path[0] = 0;
  __syncthreads();
  if (a.parents) {
    for (int j = tid; j < n; j += VD_THREADS)
      if (d.tried[j] >= 0) atomicMin(&d.first[d.tried[j]], j);
    __syncthreads();
  }
  if (producer) {
    if (p_v >= p_end) p_open(d.first[0]);
    while (p_count < VD_STAGES - 1 && p_node < n && alive) fetch(true);
  }
  if (a.parents) {
    for (int j = tid; j < n; j += VD_THREADS) {
      if (d.tried[j] < 0) continue;
      for (int i = j + 1; i < n; ++i)
        if (d.tried[i] == d.tried[j]) { d.next[j] = i; break; }
    }
    __syncthreads();
  }
  cluster.barrier_wait();

  int stage = 0, use = 0, count = 0;                   // of the ring: the chunk that is consumed next
  auto consumed = [&]() {
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(tc::smem_u32(&sh.empty[stage]));
    ++count;
    if (++stage == VD_STAGES) { stage = 0; ++use; }
  };
  // what was fetched ahead is dropped, and (node < n) the ring filled along another branch
  auto redirect = [&](int node) {
    if (producer) sh.fetched = p_count;
    __syncthreads();
    for (int upto = sh.fetched; count < upto;) {
      wait(&sh.full[stage], use & 1);
      consumed();
    }
    if (producer && node < n) {
      p_open(node);
      for (int i = 0; i < VD_STAGES - 1; ++i) fetch(true);
    }
  };
  int turn = 0;                                        // exchanges so far: their buffers alternate, so that one barrier each is enough
  // Every warp's part of the rows of `rows` nodes from x along the first children, and, of all warps and blocks, to every block.  GREEDY: the largest logit
  // and where it is (NaN counts as the largest); else the largest and the sum.
  auto scan = [&](int x, int rows, auto is_greedy) {
    constexpr bool GREEDY = decltype(is_greedy)::value;
    int node = x;
    for (int g = 0; g < rows; ++g) {
      const VdSpan<T> r(a, row0 + node, part);
      const int edge = part == 0 && warp == 0 && lane < r.head ? lane : part == splits - 1 && warp == VD_WARPS - 1 && lane < a.vocab - r.tail0 ? r.tail0 + lane : -1;
      const float edge_v = edge >= 0 ? lp_load(r.x + edge) : -INFINITY;
      float m = -INFINITY;
      F2 l{{0.f, 0.f}};
      int from = r.begin;
      for (int v0 = r.begin; v0 < r.end; v0 += VD_CHUNK) {
        if (producer) fetch(true);                         // (into the stage that the chunk before this one left)
        wait(&sh.full[stage], use & 1);
        const uint4 *chunk = reinterpret_cast<const uint4 *>(vd_ring) + stage * VD_CHUNK + tid;
        uint4 raw[VD_UNROLL];
#pragma unroll
        for (int u = 0; u < VD_UNROLL; ++u) raw[u] = chunk[u * VD_THREADS];
        consumed();
        if (v0 + VD_CHUNK > r.end) {
          const uint32_t none = no_logits<T>();
#pragma unroll
          for (int u = 0; u < VD_UNROLL; ++u)
            if (v0 + u * VD_THREADS + tid >= r.end) raw[u] = make_uint4(none, none, none, none);
        }
        const float vmax = chunk_max(raw, (const T *)nullptr);
        if (!(vmax <= m) && m == m) {
          if (!GREEDY) {
            const float f = m != -INFINITY ? exp2_approx((m - vmax) * c) : 0.f;
            l = mul2(l, F2{{f, f}});
          }
          m = vmax;
          from = v0;
        }
        if (!GREEDY && m != -INFINITY) {
          F2 s{{0.f, 0.f}};
#pragma unroll
          for (int u = 0; u < VD_UNROLL; ++u) {
            float e[N];
            LpVec<T>::unpack(raw[u], e);
#pragma unroll
            for (int i = 0; i < N; i += 2) {
              F2 t = mul2(add2(F2{{e[i], e[i + 1]}}, F2{{-m, -m}}), F2{{c, c}});
              t.f[0] = exp2_approx(t.f[0]);
              t.f[1] = exp2_approx(t.f[1]);
              s = add2(s, t);
            }
          }
          l = add2(l, s);
        }
      }
      float2 mine = make_float2(max_nan(m, edge_v), l.f[0] + l.f[1]);
      if (GREEDY) {
        // an odd end that is larger than what the thread's vectors have, or as large and before them, or all that it has
        const bool nan = m != m, same = edge_v == m || (nan && edge_v != edge_v);
        if (edge >= 0 && (same ? edge < r.head || r.begin + tid >= r.end : !nan && !(edge_v <= m))) from = -1 - edge;
        mine.y = __int_as_float(from);
      } else if (edge >= 0 && edge_v != -INFINITY) {
        mine.y = (m != -INFINITY ? mine.y * exp2_approx((m - mine.x) * c) : 0.f) + exp2_approx((edge_v - mine.x) * c);
      }
      sh.thread_part[g][tid] = mine;
      node = d.first[node];
    }
    __syncthreads();
    if (warp < rows) {                                 // a row's threads as one: a warp each
      VdPart p{-INFINITY, 0.f, NO_CHILD};
      float2 x8[VD_THREADS / 32];
#pragma unroll
      for (int i = 0; i < VD_THREADS / 32; ++i) {
        x8[i] = sh.thread_part[warp][i * 32 + lane];
        p.m = max_nan(p.m, x8[i].x);
      }
      if (GREEDY) {
        float top = p.m;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
        auto is_top = [&](float v) { return v == top || (v != v && top != top); };
        int y = x;
        for (int g = 0; g < warp; ++g) y = d.first[y];
        const VdSpan<T> r(a, row0 + y, part);
#pragma unroll 1
        for (int i = 0; i < VD_THREADS / 32; ++i) {
          const float2 t = sh.thread_part[warp][i * 32 + lane];
          const int from = __float_as_int(t.y);
          if (!is_top(t.x)) continue;
          if (from < 0) { p.idx = min(p.idx, -1 - from); continue; }
          for (int u = 0; u < VD_UNROLL; ++u) {        // the first element that is the largest, in the thread's first chunk that has it
            const int v = from + u * VD_THREADS + i * 32 + lane;
            if (v >= r.end) break;
            const T *at = r.x + r.head + (size_t)v * N;
            int k = 0;
            while (k < N && !is_top(lp_load(at + k))) ++k;
            if (k < N) { p.idx = min(p.idx, r.head + v * N + k); break; }
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < VD_THREADS / 32; ++i)
          if (x8[i].y > 0.f || x8[i].y != x8[i].y) p.l += x8[i].x == p.m ? x8[i].y : x8[i].y * exp2_approx((x8[i].x - p.m) * c);
      }
      p = vd_join<GREEDY>(p, c);
      if (lane < splits) cluster.map_shared_rank(&sh, lane)->part[turn & 1][warp][part] = p;
    }
    cluster.sync();
    // every row's own verdict, a warp each
    if (warp < rows) {
      int y = x;
      for (int g = 0; g < warp; ++g) y = d.first[y];
      const VdPart p = vd_join<GREEDY>(lane < splits ? sh.part[turn & 1][warp][lane] : VdPart{-INFINITY, 0.f, NO_CHILD}, c);
      VdVerdict v{VD_NONE, p.idx, p.m};
      if (GREEDY) {
        for (int j = d.first[y]; j < n && v.to < 0; j = d.next[j])
          if (d.token[j] == p.idx) v.to = j;
      } else {
        v.to = p.l > 0.f && p.l < INFINITY ? vd_children<false>(d, sh.root, a, n, y, p.m, p.l, c, c64) : VD_UNCLEAR;
      }
      if (lane == 0) sh.verdict[warp] = v;
    }
    ++turn;
    __syncthreads();
  };
  int x = 0, depth = 0, ahead = 0;                     // ahead: the node whose row is next in the ring
  bool by_largest = greedy;                            // T = 0, or a row without probabilities
  while (true) {
    // ---- rows from x along the first children, and what they decide
    if (x != ahead) redirect(x);
    int rows = 1;
    for (int y = x; rows < a.group && !(by_largest && !greedy) && d.first[y] < n; ++rows) y = d.first[y];
    if (by_largest) scan(x, rows, std::true_type());
    else scan(x, rows, std::false_type());
    int at = x, action = VD_MOVE;
    ahead = x;
    for (int g = 0; g < rows; ++g) ahead = d.first[ahead];
    float m = 0.f;
    for (int g = 0; g < rows; ++g) {
      const VdVerdict v = sh.verdict[g];
      m = v.m;
      if (v.to < 0) {
        action = by_largest ? VD_DONE : v.to == VD_NONE ? VD_DRAW : v.to == VD_UNSURE ? VD_EXACT : VD_GREEDY;
        if (by_largest) at = v.best;
        break;
      }
      const int along = d.first[at];
      at = v.to;
      ++depth;
      if (tid == 0) d.path[depth] = at;
      if (at != along) break;
    }
    if (by_largest != greedy) by_largest = greedy;     // (that row is decided)
    else if (action == VD_GREEDY) by_largest = true;
    if (action == VD_MOVE || action == VD_GREEDY) {
      x = at;
      if (action == VD_GREEDY) ahead = -1;             // (its row is read again)
      __syncthreads();                                 // (the verdicts have been read)
      continue;
    }
    if (action == VD_DONE) {
      if (part == 0 && tid == 0) out[depth] = at;
      break;
    }
    // ---- the row's weights in 64 bits: 0 all of them, where their sum is wanted; 1 without what fell; 2 all of them, where that leaves nothing
    const bool fell = d.first[at] < n;
    const VdRow<T> r(a, row0 + at, part);
    int pass = action == VD_EXACT || (a.draft && fell) ? 0 : 1, to = VD_NONE;
    double total = 0.0, before = 0.0;
    while (true) {
      if (tid == 0) {
        VdWeights k{(double)m, c64, total, nullptr, 0, lowest_64((double)m, c64)};
        if (pass == 1 && fell) {
          if (a.draft) k.q = a.draft + (row0 + d.first[at]) * a.draft_stride;
          else
            for (int j = d.first[at]; j < n; j = d.next[j]) d.tried[k.n_tried++] = d.token[j];
        }
        sh.k = k;
        if (pass == 0 && fell && a.draft) {            // the drafter's row on its way into L2 while this one's sum is formed
          const float *q = a.draft + (row0 + d.first[at]) * a.draft_stride;
          const uintptr_t q0 = reinterpret_cast<uintptr_t>(q + max(0, r.element(r.begin, 0))) & ~(uintptr_t)15, q1 = reinterpret_cast<uintptr_t>(q + min(a.vocab, r.element(r.end, 0))) & ~(uintptr_t)15;
          const uintptr_t inside = q0 < reinterpret_cast<uintptr_t>(q) ? q0 + 16 : q0;
          if (inside < q1) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(inside), "r"((uint32_t)(q1 - inside)) : "memory");
        }
      }
      __syncthreads();
      if (pass == 1 && fell && a.draft) vd_tiles<T, true>(sh, d.tried, r);
      else vd_tiles<T, false>(sh, d.tried, r);
      __syncthreads();
      if (warp == 0) {
        const VdStretch s = vd_stretch(sh.tile, r.tiles);
        const double mine = __shfl_sync(0xffffffffu, s.until, 31);
        if (lane < splits) cluster.map_shared_rank(&sh, lane)->sum[turn & 1][part] = mine;
      }
      cluster.sync();
      total = 0.0;
      for (int i = 0; i < splits; ++i) {
        if (i == part) before = total;
        total += sh.sum[turn & 1][i];
      }
      ++turn;
      if (pass == 0) {
        if (action == VD_EXACT) {
          if (warp == 0) {
            to = vd_children<true>(d, sh.root, a, n, at, m, total, c, c64);
            if (lane == 0) sh.to = to;
          }
          __syncthreads();
          to = sh.to;
          if (to >= 0) break;
        }
        pass = 1;
      } else if (pass == 2 || !fell || total > 0.0) {
        break;
      } else {
        pass = 2;
      }
    }
    if (to >= 0) {
      x = to;
      ++depth;
      if (tid == 0) d.path[depth] = to;
      ahead = -1;                                      // (rows of the same group may have been consumed)
      __syncthreads();
      continue;
    }
    // ---- the next token
    {
      // the block with the token: the first whose end lies beyond the target, or the last with any weight
      const double target = (double)unit(d.u[0]) * total;
      double until = 0.0;
      int owner = -1;
      for (int i = 0; i < splits; ++i) {
        const double w = sh.sum[(turn - 1) & 1][i];
        until += w;
        if (w > 0.0) owner = i;
        if (w > 0.0 && until > target) break;
      }
      int token;
      if (owner == part && vd_find<T>(sh, d.tried, r, target - before, token)) out[depth] = token;
    }
    break;
  }
  redirect(n);                                         // (copies under way land before the ring is given back; the barrier inside orders the path's entries)
  if (producer && !alive)
    for (int i = max(0, p_count - VD_STAGES); i < p_count; ++i) tc::mbar_wait(tc::smem_u32(&sh.full[i % VD_STAGES]), (i / VD_STAGES) & 1);
  if (part == 0) {
    for (int j = tid; j < a.max_new; j += VD_THREADS) {
      path[j] = j <= depth ? d.path[j] : -1;
      if (j != depth) out[j] = j < depth ? d.token[d.path[j + 1]] : -1;
    }
    if (tid == 0) a.n_accepted[b] = depth;
  }
}

size_t verify_smem(int max_new) { return (size_t)VD_STAGES * VD_CHUNK * 16 + (size_t)VD_ARRAYS * max_new * 4; }
template <typename T>
cudaError_t verify_config(cudaLaunchConfig_t &cfg, cudaLaunchAttribute &at, int n_seqs, int log_splits, int max_new, cudaStream_t st) {
  cfg = cudaLaunchConfig_t{};
  cfg.gridDim = dim3((unsigned)((long long)n_seqs << log_splits));
  cfg.blockDim = dim3(VD_THREADS);
  cfg.dynamicSmemBytes = verify_smem(max_new);
  cfg.stream = st;
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = 1u << log_splits;
  at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  if (ensure_dynamic_smem(reinterpret_cast<const void *>(verify_drafts_kernel<T>), (int)verify_smem(VD_MAX_NEW))) return cudaErrorInvalidValue;
  return cudaSuccess;
}
// How many clusters of 2^log_splits blocks run at once on the current device (a cluster lies within a GPC: of 16 blocks, two per SM, 14 do, not
// 18); asked for once, 0 on an error
template <typename T>
int verify_clusters(int log_splits) {
  constexpr int MAX_DEVICES = 64;
  static std::atomic<int> known[MAX_DEVICES][5];
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return 0;
  std::atomic<int> &slot = known[dev][log_splits];
  if (const int n = slot.load()) return n - 1;
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute at[1];
  int n = 0;
  if (verify_config<T>(cfg, at[0], 1, log_splits, 64, nullptr) != cudaSuccess) return 0;
  if (cudaFuncSetAttribute(verify_drafts_kernel<T>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return 0;      // (clusters of 16)
  if (cudaOccupancyMaxActiveClusters(&n, verify_drafts_kernel<T>, &cfg) != cudaSuccess) {
    cudaGetLastError();                                // (not kept: the next call asks again)
    return 0;
  }
  slot.store(n + 1);
  return n;
}
template <typename T>
cudaError_t launch_verify(VdArgs a, int n_seqs, cudaStream_t st) {
  static_assert(sizeof(VdShared) <= 32 * 1024, "shared memory");
  // a sequence gets a cluster of as many blocks as run at once with all the others' (16 at most), each with thousands of logits of a row, and of at least so
  // many that none has more than 256 KB of it.  Both sides of that border, chains of 4 tokens, us with one block a sequence / with two: below it 200 x 131000 bf16 112 / 102,
  // 256 sequences 113 / 114, 400 sequences 184 / 159; above it 200 x 133000 117 / 110, 256 117 / 121, 400 187 / 171; fp32 200 x 67000 81 / 82, 256 83 / 97, 400 138 / 133,
  // 200 x 100003 118 / 108, 256 113 / 126, 400 179 / 171, but 256 of 1 - 6 tokens 137 / 126.  It gains up to a tenth where two turns of blocks are needed anyway, and loses
  // up to a sixth of fp32 rows just above it where one block each fits in one turn; a border at half of that loses a sixth at 128 sequences (133000 bf16: 69 with
  // two blocks, 82 with four).
  static_assert(1 << 4 == VD_MAX_CLUSTER, "from the largest cluster down");
  for (a.log_splits = 4; a.log_splits > 0; --a.log_splits)
    if (a.vocab >> a.log_splits >= 2048 && (n_seqs <= verify_clusters<T>(a.log_splits) || ((long long)a.vocab * (long long)sizeof(T)) >> (a.log_splits - 1) > 262144)) break;
  // one exchange decides several rows where a block's part of a row takes less time than the exchange
  const long long bytes = ((long long)a.vocab * sizeof(T)) >> a.log_splits;
  a.group = bytes <= 32768 ? VD_GROUP : bytes <= 65536 ? 2 : 1;
  const long long chunks = bytes / 16 / VD_CHUNK + 1;
  a.unsure = (float)(0x1p-16 + (double)(chunks + 4) * 0x1p-21);
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute at[1];
  const cudaError_t e = verify_config<T>(cfg, at[0], n_seqs, a.log_splits, a.max_new, st);
  return e != cudaSuccess ? e : cudaLaunchKernelEx(&cfg, verify_drafts_kernel<T>, a);
}

}  // namespace
}  // namespace skv

using namespace skv;

extern "C" int32_t swiftkv_verify_drafts(const void *logits, int64_t row_stride, int32_t dtype, const int32_t *tokens, const int32_t *cu_new,
                                         const int32_t *parents, const float *draft_probs, int64_t draft_stride, const float *uniforms,
                                         const float *temperatures, float temperature, int32_t n_seqs, int32_t total_new, int32_t max_new,
                                         int32_t vocab, int32_t *n_accepted, int32_t *tokens_out, int32_t *path, void *cuda_stream) {
  if (!logits || !tokens || !cu_new || !n_accepted || !tokens_out || !path) return report_error(SWIFTKV_ERR_INVALID_ARG, "null argument");
  if (dtype != SWIFTKV_DTYPE_F32 && dtype != SWIFTKV_DTYPE_BF16 && dtype != SWIFTKV_DTYPE_F16) return report_error(SWIFTKV_ERR_INVALID_ARG, "unknown dtype");
  if (n_seqs < 1 || n_seqs > (1 << 24) || total_new < 1 || max_new < 1 || max_new > VD_MAX_NEW || vocab < 1 || vocab > (1 << 30) || row_stride < vocab)
    return report_error(SWIFTKV_ERR_INVALID_ARG, "bad shape (n_seqs in [1, 2^24], max_new in [1, 1024], vocab in [1, 2^30], row_stride >= vocab)");
  if (draft_probs && parents) return report_error(SWIFTKV_ERR_INVALID_ARG, "draft_probs go with chains, not with parents");
  if (draft_probs && draft_stride < vocab) return report_error(SWIFTKV_ERR_INVALID_ARG, "bad shape (draft_stride >= vocab)");
  if (!temperatures && !(temperature == 0.f || (temperature >= VD_COLDEST && temperature <= VD_HOTTEST)))
    return report_error(SWIFTKV_ERR_INVALID_ARG, "temperature must be 0 or in [2^-64, 2^100]");
  if (!uniforms && (temperatures || temperature != 0.f)) return report_error(SWIFTKV_ERR_INVALID_ARG, "null argument (uniforms may be null at temperature 0 alone)");
  const size_t es = dtype == SWIFTKV_DTYPE_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(logits) % es || reinterpret_cast<uintptr_t>(draft_probs) % 4) return report_error(SWIFTKV_ERR_INVALID_ARG, "misaligned logits or draft_probs");
  const size_t total = (size_t)total_new, seqs = (size_t)n_seqs, out = seqs * max_new * 4;
  const ByteRows in[] = {{logits, total, (size_t)row_stride * es, (size_t)vocab * es}, {tokens, 1, total * 4, total * 4}, {cu_new, 1, (seqs + 1) * 4, (seqs + 1) * 4},
                         {parents, 1, total * 4, total * 4}, {draft_probs, total, (size_t)draft_stride * 4, (size_t)vocab * 4}, {uniforms, 1, total * 4, total * 4},
                         {temperatures, 1, seqs * 4, seqs * 4}};
  const ByteRows outs[] = {{n_accepted, 1, seqs * 4, seqs * 4}, {tokens_out, 1, out, out}, {path, 1, out, out}};
  for (int i = 0; i < 3; ++i) {
    for (const ByteRows &r : in)
      if (r.p && overlap(outs[i], r)) return report_error(SWIFTKV_ERR_INVALID_ARG, "an output overlaps an input");
    for (int j = 0; j < i; ++j)
      if (overlap(outs[i], outs[j])) return report_error(SWIFTKV_ERR_INVALID_ARG, "two outputs overlap");
  }
  unsigned int *status = op_status_word();
  if (!status) return report_error(SWIFTKV_ERR_CUDA, "no status word");
  VdArgs a{logits, row_stride, draft_stride, tokens, cu_new, parents, draft_probs, uniforms, temperatures, temperature, total_new, max_new, vocab, 0, 0, 0.f,
           n_accepted, tokens_out, path, status};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = dtype == SWIFTKV_DTYPE_F32 ? launch_verify<float>(a, n_seqs, st) : dtype == SWIFTKV_DTYPE_BF16 ? launch_verify<bf16>(a, n_seqs, st) : launch_verify<__half>(a, n_seqs, st);
  if (e != cudaSuccess) return report_error(SWIFTKV_ERR_CUDA, cudaGetErrorString(e));
  return SWIFTKV_OK;
}
