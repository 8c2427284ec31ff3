// swiftkv_token_logprobs: log probability of a given token per row of logits, with the row's log-sum-exp, entropy and its
// top_k alternatives, in ONE pass over the logits; swiftkv_token_logprobs_bwd: the gradient with respect to the logits.
//
// With c = log2(e) / T a thread keeps, relative to a reference r,
//   l = sum 2^(x c - r)      and      s = sum 2^(x c - r) (x c - r)
// and at the end r = m c with m the largest logit, so that  lse = m / T + ln l,  entropy = (log2 l - s / l) ln 2  (every term of s
// has one sign: nothing cancels), and  logprob(t) = (x_t - m) / T - ln l.  x c - r is one fused multiply-add, rounded once at its own
// size; sums are fp32.  r moves only when the sums could grow by more than 2^16, and stays within 2^30.
//
// Top-k: a bound that at least k logits reach -- after a row's first chunk the k-th largest of the
// warps' four best thread maxima, later the k-th largest of 32 groups of all threads' maxima so far, which one warp keeps
// forming anew (an old maximum is only a lower one, so nobody waits).  Logits that reach the
// bound -- a few dozen per row -- are noted, and in the end those that reach the last bound are ranked by counting.  A row that
// floods the notes (rising, or with thousands of equal logits) is read again with a sorted list, which holds for any order.
//
// What bounds it: HBM (the logits are read once), with about five instructions and one exponential per logit close behind for
// 16-bit types.  Blocks are persistent and stream rows through a ring of 32 KB bulk copies; a warp of its own joins up a
// finished row while the others go on with the next.  Few rows: a row is shared by a cluster of up to 8 blocks whose partial
// results meet in distributed shared memory, so one launch needs no workspace at any size.  Measured at 128256 logits: 4096 rows
// bf16 with top 5 226 us (4.7 TB/s), 2048 rows fp32 without top k 157 us (6.7 TB/s), 33 rows fp32 with top 8 12 us; the gradient of 2048
// rows bf16 169 us (6.2 TB/s).
#include <cooperative_groups.h>

#include "common.cuh"
#include "tc_common.cuh"

namespace skv {
namespace {
namespace cg = cooperative_groups;
using tc::F2;
using tc::add2;
using tc::fma2;
using tc::max_nan;

constexpr int LP_THREADS = 256, LP_WARPS = LP_THREADS / 32;     // threads that read logits; one more warp joins up
constexpr int LP_MAX_TOP = 32;
constexpr int LP_MAX_CLUSTER = 8;
constexpr int LP_UNROLL = 8;                 // 16-byte vectors of a chunk per thread
constexpr int LP_CHUNK = LP_THREADS * LP_UNROLL;          // vectors of a chunk
constexpr int LP_STAGES = 3;
constexpr int LP_SMEM = LP_STAGES * LP_CHUNK * 16;
constexpr float LP_RESCALE = 16.f;           // the reference moves when the sums could grow by more than 2^16
constexpr float LOWEST = -3.0e38f;
// Largest |x c| whose exponents are formed as x c - r: the product's rounding, which r has and the fused multiply-add has not, is up to
// half a step, 64 here, and sums of 2^64 are still far from infinite.
constexpr float LP_FAR = 1073741824.f;

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 16 bytes of logits as fp32; adding zero turns -0 into +0, so that equal values have equal order keys
template <typename T> struct LpVec;
template <> struct LpVec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4 &v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};
template <> struct LpVec<bf16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4 &v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    return make_uint4(tc::pack_bf16x2(x[0], x[1]), tc::pack_bf16x2(x[2], x[3]), tc::pack_bf16x2(x[4], x[5]), tc::pack_bf16x2(x[6], x[7]));
  }
};
__device__ __forceinline__ uint32_t pack_half2_ieee(float lo, float hi) {      // beyond the range: infinity, as a cast gives
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&h);
}
template <> struct LpVec<__half> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4 &v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
      x[2 * i] = f.x; x[2 * i + 1] = f.y;
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    return make_uint4(pack_half2_ieee(x[0], x[1]), pack_half2_ieee(x[2], x[3]), pack_half2_ieee(x[4], x[5]), pack_half2_ieee(x[6], x[7]));
  }
};
__device__ __forceinline__ float lp_load(const float *p) { return *p; }
__device__ __forceinline__ float lp_load(const bf16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ float lp_load(const __half *p) { return __half2float(*p); }
__device__ __forceinline__ void lp_store(float *p, float v) { *p = v; }
__device__ __forceinline__ void lp_store(bf16 *p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void lp_store(__half *p, float v) { *p = __float2half_rn(v); }

// whole-number keys in the order of the values (NaN above all); 0 stands for "no element"
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  if (x != x) return 0xffffffffu;
  return b ^ ((b & 0x80000000u) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  if (k == 0xffffffffu) return __uint_as_float(0x7fffffffu);
  return __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k);
}

// a set of logits: its maximum m, and l, s relative to it (exponents in units of log 2); m = -inf: no finite logit, l and s are 0 or NaN
struct LpSums { float m, l, s; };
// l, s relative to a reference that lies d above: a factor f, and s moves by l d.  A factor of zero drops them: d may then be as large
// as the type's lowest value (a masked logit met first), whose multiple by l is not finite.
__device__ __forceinline__ void lp_move(float &l, float &s, float d) {
  const float f = exp2_approx(d), l2 = l * f;               // (a NaN stays one)
  s = f == 0.f ? l2 : (s + l * d) * f;
  l = l2;
}
// joins the lanes' sets: the same bits in every lane (the maximum first; sums of pairs do not depend on their order)
__device__ __forceinline__ LpSums lp_warp_join(LpSums t, float c) {
  float m = t.m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (t.m != -INFINITY) lp_move(t.l, t.s, (t.m - m) * c);
  t.m = m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    t.l += __shfl_xor_sync(0xffffffffu, t.l, o);
    t.s += __shfl_xor_sync(0xffffffffu, t.s, o);
  }
  return t;
}

// one warp's k best, sorted across its lanes: lane i holds the i-th best
struct WarpTop {
  uint32_t key = 0;
  int idx = 0x7fffffff;
  uint32_t kth = 0;            // the k-th best key (0 while the list is not full)
  __device__ __forceinline__ void insert(uint32_t ck, int ci, int k) {       // arguments are the same in every lane
    const int lane = threadIdx.x & 31;
    const unsigned before = __ballot_sync(0xffffffffu, key > ck || (key == ck && idx < ci));
    const int pos = __popc(before);
    const uint32_t pk = __shfl_up_sync(0xffffffffu, key, 1);
    const int pi = __shfl_up_sync(0xffffffffu, idx, 1);
    if (lane > pos) { key = pk; idx = pi; }
    else if (lane == pos) { key = ck; idx = ci; }
    kth = __shfl_sync(0xffffffffu, key, k - 1);
  }
};

struct LpArgs {
  const void *logits;
  long long stride;
  const int32_t *targets;
  float *logprob, *entropy, *lse, *top_lp;
  int32_t *top_ids;
  int rows, vocab, top_k, splits;
  float c, inv_t, low;     // low: what -inf is lifted to
  unsigned int *status;
};

constexpr int LP_NOTES = 768;
struct LpShared {
  // two rows: the one that is read, and the one that is joined up
  LpSums warp_sums[2][LP_WARPS];
  uint32_t warp_top[2][32];          // every warp's four best thread maxima after the first chunk
  uint32_t best[2][LP_THREADS];      // every thread's largest so far (0: none)
  uint32_t bound[2];                 // what at least k of the logits so far reach (0: none yet)
  uint32_t n_notes[2];
  uint2 note[2][LP_NOTES];           // (index, order key) of logits of the block's part that may be among its k best
  // the row that is joined up
  LpSums sums;
  uint2 top[LP_MAX_TOP];             // the block's k best, in order (key 0: none)
  uint64_t full[LP_STAGES], empty[LP_STAGES], row_done[2], row_free[2];
};

// the lanes' keys, largest first
__device__ __forceinline__ uint32_t sort_lanes(uint32_t v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
    for (int j = size >> 1; j > 0; j >>= 1) {
      const uint32_t other = __shfl_xor_sync(0xffffffffu, v, j);
      v = (((lane & j) == 0) == ((lane & size) == 0 || size == 32)) ? max(v, other) : min(v, other);
    }
  return v;
}
__device__ __forceinline__ uint32_t kth_of_lanes(uint32_t v, int k) { return __shfl_sync(0xffffffffu, sort_lanes(v), k - 1); }

// the better of two notes is the larger number: the key, then the lower index
__device__ __forceinline__ unsigned long long note_order(uint2 n) { return (unsigned long long)n.y << 32 | (0xffffffffu - n.x); }

// one warp: the best k of n notes in shared memory, in order; a note's rank is the number of better ones, and those with key 0 are none
__device__ __forceinline__ void rank_notes(uint2 (&top)[LP_MAX_TOP], const uint2 *note, int n, int k) {
  const int lane = threadIdx.x & 31;
  top[lane] = make_uint2(0x7fffffffu, 0u);
  __syncwarp();
  for (int i = lane; i < n; i += 32) {
    const uint2 mine = note[i];
    if (mine.y == 0) continue;
    const unsigned long long order = note_order(mine);
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) rank += note_order(note[j]) > order;
    if (rank < k) top[rank] = mine;
  }
  __syncwarp();
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// a block's part of a row: elements before the row's first 16-byte boundary (head), whole vectors [v_begin, v_end), elements behind
struct LpRow {
  int head, tail0, v_begin, v_end;
};
template <typename T>
__device__ __forceinline__ LpRow lp_row(const LpArgs &a, int row, int part) {
  constexpr int N = LpVec<T>::N;
  const uintptr_t at = reinterpret_cast<uintptr_t>(reinterpret_cast<const T *>(a.logits) + (size_t)row * a.stride);
  const int mis = (int)((at & 15) / sizeof(T));
  LpRow r;
  r.head = min(a.vocab, mis ? N - mis : 0);
  const int n_vec = (a.vocab - r.head) / N;
  r.tail0 = r.head + n_vec * N;
  r.v_begin = (int)((long long)n_vec * part / a.splits);
  r.v_end = (int)((long long)n_vec * (part + 1) / a.splits);
  return r;
}

// A thread's vectors of a chunk: their maximum (NaN if they hold one), and what stands for logits that are not there.  clamp: lifts -inf to a finite value
// far below anything that counts, two 16-bit logits per instruction (fp32: in the accumulation).
__device__ __forceinline__ float chunk_max(const uint4 (&v)[LP_UNROLL], const float *) {
  float m = -INFINITY;
#pragma unroll
  for (int u = 0; u < LP_UNROLL; ++u)
    m = max_nan(m, max_nan(max_nan(__uint_as_float(v[u].x), __uint_as_float(v[u].y)), max_nan(__uint_as_float(v[u].z), __uint_as_float(v[u].w))));
  return m;
}
template <typename H2>
__device__ __forceinline__ H2 chunk_max2(const uint4 (&v)[LP_UNROLL]) {
  H2 m[LP_UNROLL];
#pragma unroll
  for (int u = 0; u < LP_UNROLL; ++u) {
    const H2 *h = reinterpret_cast<const H2 *>(&v[u]);
    m[u] = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
  }
#pragma unroll
  for (int n = LP_UNROLL / 2; n > 0; n >>= 1)
#pragma unroll
    for (int u = 0; u < n; ++u) m[u] = __hmax2_nan(m[u], m[u + n]);
  return m[0];
}
__device__ __forceinline__ float chunk_max(const uint4 (&v)[LP_UNROLL], const bf16 *) {
  const __nv_bfloat162 m = chunk_max2<__nv_bfloat162>(v);
  return max_nan(__low2float(m), __high2float(m));
}
__device__ __forceinline__ float chunk_max(const uint4 (&v)[LP_UNROLL], const __half *) {
  const __half2 m = chunk_max2<__half2>(v);
  return max_nan(__low2float(m), __high2float(m));
}
template <typename T> __device__ __forceinline__ uint32_t no_logits();
template <> __device__ __forceinline__ uint32_t no_logits<float>() { return 0xff800000u; }
template <> __device__ __forceinline__ uint32_t no_logits<bf16>() { return 0xff80ff80u; }
template <> __device__ __forceinline__ uint32_t no_logits<__half>() { return 0xfc00fc00u; }
__device__ __forceinline__ void clamp_vec(uint4 &, float, const float *) {}
__device__ __forceinline__ void clamp_vec(uint4 &v, float low, const bf16 *) {
  const __nv_bfloat162 lo = __float2bfloat162_rn(low);
  __nv_bfloat162 *h = reinterpret_cast<__nv_bfloat162 *>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __hmax2_nan(h[i], lo);
}
__device__ __forceinline__ void clamp_vec(uint4 &v, float low, const __half *) {
  const __half2 lo = __float2half2_rn(low);
  __half2 *h = reinterpret_cast<__half2 *>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __hmax2_nan(h[i], lo);
}

// one warp: the bound that the threads' maxima so far give
__device__ __forceinline__ uint32_t lp_bound(const LpShared &sh, int par, int k) {
  const volatile uint32_t *b = sh.best[par];
  const int lane = threadIdx.x & 31;
  uint32_t v = 0;
#pragma unroll
  for (int i = 0; i < LP_THREADS / 32; ++i) v = max(v, b[i * 32 + lane]);
  return kth_of_lanes(v, k);
}

// one warp: a finished row's sums and, TOP, the block's k best, into sh.sums / top_key / top_idx
template <typename T, bool TOP>
__device__ __forceinline__ void lp_finish(LpShared &sh, int par, const LpArgs &a, const T *x, const LpRow &rw, int part) {
  constexpr int N = LpVec<T>::N;
  const int lane = threadIdx.x & 31, k = a.top_k;
  const LpSums b = lp_warp_join(lane < LP_WARPS ? sh.warp_sums[par][lane] : LpSums{-INFINITY, 0.f, 0.f}, a.c);
  if (lane == 0) sh.sums = b;
  if (TOP) {
    const uint32_t bound = lp_bound(sh, par, k);
    const int notes = (int)sh.n_notes[par];
    uint2 *note = sh.note[par];
    if (notes <= LP_NOTES) {
      int n = 0;                                             // those that reach the last bound move to the front
      for (int i0 = 0; i0 < notes; i0 += 32) {
        const uint2 mine = i0 + lane < notes ? note[i0 + lane] : make_uint2(0u, 0u);
        const bool in = mine.y >= bound && mine.y != 0;
        const unsigned all = __ballot_sync(0xffffffffu, in);
        if (in) note[n + __popc(all & ((1u << lane) - 1u))] = mine;
        n += __popc(all);
        __syncwarp();
      }
      rank_notes(sh.top, note, n, k);
    } else {
      // flooded: a sorted list.  Elements come in ascending order, so that of equal ones the first stays.
      WarpTop top;
      const int e_begin = part == 0 ? 0 : rw.head + rw.v_begin * N, e_end = part == a.splits - 1 ? a.vocab : rw.head + rw.v_end * N;
      for (int i0 = e_begin; i0 < e_end; i0 += 256) {
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = i0 + q * 32 + lane < e_end ? lp_load(x + i0 + q * 32 + lane) : 0.f;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int i = i0 + q * 32 + lane;
          const uint32_t key = i < e_end ? order_key(v[q]) : 0;
          unsigned pass = __ballot_sync(0xffffffffu, key > top.kth);
          while (pass) {
            const int src = __ffs(pass) - 1;
            pass &= pass - 1;
            const uint32_t ck = __shfl_sync(0xffffffffu, key, src);
            if (ck > top.kth) top.insert(ck, i - lane + src, k);
          }
        }
      }
      sh.top[lane] = make_uint2((uint32_t)top.idx, lane < k ? top.key : 0u);
      __syncwarp();
    }
#pragma unroll
    for (int i = 0; i < LP_THREADS / 32; ++i) sh.best[par][i * 32 + lane] = 0;      // for the next row but one
    if (lane == 0) sh.n_notes[par] = sh.bound[par] = 0;
  }
  __syncwarp();
}
// ... and the row's results from them
template <typename T, bool TOP>
__device__ __forceinline__ void lp_write(const LpShared &sh, const LpArgs &a, const LpSums &all, int row, int tgt, float tgt_v) {
  constexpr float LN2 = 0.6931471805599453f;
  const int lane = threadIdx.x & 31, k = a.top_k;
  // no finite logit, or none beside a NaN of its vector: l is 0 or NaN, and only lse may still be a value (-inf)
  const bool none = all.m == -INFINITY;
  const float log_l = none ? __uint_as_float(0x7fffffffu) : __log2f(all.l);
  if (lane == 0) {
    a.lse[row] = none ? -INFINITY + all.l : fmaf(all.m, a.inv_t, log_l * LN2);
    a.entropy[row] = (log_l - all.s / all.l) * LN2;
    if (tgt >= a.vocab) atomicOr(a.status, STATUS_BAD_TOKEN);
    a.logprob[row] = tgt >= 0 && tgt < a.vocab ? (tgt_v - all.m) * a.inv_t - log_l * LN2 : 0.f;
  }
  if (TOP && lane < k) {
    a.top_ids[(size_t)row * k + lane] = (int)sh.top[lane].x;
    a.top_lp[(size_t)row * k + lane] = (key_value(sh.top[lane].y) - all.m) * a.inv_t - log_l * LN2;
  }
}

template <typename T, bool TOP>
__global__ void __launch_bounds__(LP_THREADS + 32, 2) token_logprobs_kernel(LpArgs a) {
  constexpr int N = LpVec<T>::N;
  __shared__ LpShared sh;
  extern __shared__ __align__(128) uint8_t lp_ring[];      // [LP_STAGES][LP_CHUNK] vectors
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int part = blockIdx.x % a.splits, row0 = blockIdx.x / a.splits, row_step = gridDim.x / a.splits;
  const float c = a.c;
  const int k = a.top_k;
  if (tid == 0) {
    for (int i = 0; i < LP_STAGES; ++i) {
      tc::mbar_init(tc::smem_u32(&sh.full[i]), 1);
      tc::mbar_init(tc::smem_u32(&sh.empty[i]), LP_WARPS);
    }
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(tc::smem_u32(&sh.row_done[i]), LP_WARPS);
      tc::mbar_init(tc::smem_u32(&sh.row_free[i]), 1);
      sh.n_notes[i] = sh.bound[i] = 0;
    }
  }
  if (tid == 0) tc::fence_barrier_init();
  if (tid < LP_THREADS) sh.best[0][tid] = sh.best[1][tid] = 0;
  __syncthreads();
  if (warp == LP_WARPS) {
    // ---- the warp that joins rows up
    int turn = 0;
    bool alive = true;
    for (int row = row0; row < a.rows; row += row_step, ++turn) {
      const int par = turn & 1;
      const T *x = reinterpret_cast<const T *>(a.logits) + (size_t)row * a.stride;
      const LpRow rw = lp_row<T>(a, row, part);
      const int tgt = a.targets ? a.targets[row] : -1;
      const float tgt_v = tgt >= 0 && tgt < a.vocab ? lp_load(x + tgt) : 0.f;
      const uint32_t done = tc::smem_u32(&sh.row_done[par]);
      const long long t0 = clock64();
      // (the lanes leave together: what is between the looks has the whole warp's shuffles)
      while (alive && !__any_sync(0xffffffffu, tc::mbar_try_wait(done, (turn >> 1) & 1))) {
        if (__any_sync(0xffffffffu, clock64() - t0 > tc::WAIT_LIMIT_CLOCKS)) {
          if (lane == 0) atomicOr(a.status, STATUS_TIMEOUT);
          alive = false;
        }
        if (TOP) {
          const uint32_t bound = lp_bound(sh, par, k);
          if (lane == 0) *reinterpret_cast<volatile uint32_t *>(&sh.bound[par]) = bound;
          __nanosleep(300);                // (leaves the issue slots to the others)
        }
      }
      __syncwarp();
      lp_finish<T, TOP>(sh, par, a, x, rw, part);
      if (a.splits == 1) {
        lp_write<T, TOP>(sh, a, sh.sums, row, tgt, tgt_v);
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(tc::smem_u32(&sh.row_free[par]));
      } else {
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        if (part == 0) {
          const LpSums all = lp_warp_join(lane < a.splits ? cluster.map_shared_rank(&sh, lane)->sums : LpSums{-INFINITY, 0.f, 0.f}, c);
          if (TOP) {
            const int n = a.splits * k;
            for (int i = lane; i < n; i += 32) sh.note[par][i] = cluster.map_shared_rank(&sh, i / k)->top[i % k];
            __syncwarp();          // (the ranking clears this block's own list)
            rank_notes(sh.top, sh.note[par], n, k);
          }
          lp_write<T, TOP>(sh, a, all, row, tgt, tgt_v);
        }
        cluster.sync();            // no block leaves while its shared memory is read
      }
    }
    return;
  }
  bool alive = true;            // a wait that ran out (never, unless something is broken): no further waits or copies
  auto wait = [&](uint64_t *bar, uint32_t parity) {
    if (alive && !tc::mbar_wait(tc::smem_u32(bar), parity)) {
      alive = false;
      atomicOr(a.status, STATUS_TIMEOUT);
    }
  };
  // thread 0 keeps the ring full: chunk p_count of this block's rows, one after the other
  int p_row = row0, p_v = 0, p_end = 0, p_count = 0;
  const uint4 *p_src = nullptr;
  auto p_open = [&]() {
    while (p_row < a.rows) {
      const LpRow r = lp_row<T>(a, p_row, part);
      p_src = reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(a.logits) + (size_t)p_row * a.stride + r.head);
      p_v = r.v_begin;
      p_end = r.v_end;
      if (p_v < p_end) return;
      p_row += row_step;
    }
  };
  auto fetch = [&]() {          // the next chunk, if there is one; its stage must have been emptied
    if (p_row >= a.rows || !alive) return;
    const int st = p_count % LP_STAGES;
    const uint32_t bar = tc::smem_u32(&sh.full[st]);
    if (p_count >= LP_STAGES) wait(&sh.empty[st], (p_count / LP_STAGES - 1) & 1);
    if (!alive) return;
    const uint32_t bytes = (uint32_t)min(LP_CHUNK, p_end - p_v) * 16;
    tc::mbar_expect_tx(bar, bytes);
    bulk_load(tc::smem_u32(lp_ring) + st * LP_CHUNK * 16, p_src + p_v, bytes, bar);
    ++p_count;
    p_v += LP_CHUNK;
    if (p_v >= p_end) { p_row += row_step; p_open(); }
  };
  if (tid == 0) {
    p_open();
    for (int i = 0; i < LP_STAGES - 1; ++i) fetch();
  }
  int count = 0, turn = 0;      // chunks and rows consumed
  for (int row = row0; row < a.rows; row += row_step, ++turn) {
    const int par = turn & 1;
    if (turn > 1) wait(&sh.row_free[par], ((turn >> 1) - 1) & 1);
    const T *x = reinterpret_cast<const T *>(a.logits) + (size_t)row * a.stride;
    const LpRow rw = lp_row<T>(a, row, part);
    const uint4 *xv = reinterpret_cast<const uint4 *>(x + rw.head);
    // a row's odd ends: a warp of the first / last part takes them
    const int edge = part == 0 && warp == 0 && lane < rw.head ? lane
                     : part == a.splits - 1 && warp == LP_WARPS - 1 && lane < a.vocab - rw.tail0 ? rw.tail0 + lane : -1;
    const float edge_v = edge >= 0 ? lp_load(x + edge) : -INFINITY;
    float r = -INFINITY, m = -INFINITY;
    F2 l2{{0.f, 0.f}}, s2{{0.f, 0.f}};                       // sums over even and odd elements
    float best = edge_v, bound = -INFINITY;                 // top-k: this thread's largest (NaN counts), what a candidate has to reach
    bool any = edge >= 0;
    auto note = [&](float v, int i) {
      if (v < bound) return;
      const uint32_t n = atomicAdd(&sh.n_notes[par], 1u);
      if (n < LP_NOTES) sh.note[par][n] = make_uint2((uint32_t)i, order_key(v));
    };
    // Makes room for logits up to vmax; false: they are not to be added.  Those far below zero (masked ones) have no probability beside any
    // other, and a thread whose largest is far from zero forms its sums anew in the end.
    auto refer = [&](float vmax) -> bool {
      m = fmaxf(m, vmax);
      const float y = vmax * c;
      if (!(fabsf(y) <= LP_FAR)) {
        if (vmax != vmax) l2.f[0] = vmax;
        return false;
      }
      if (y - r > LP_RESCALE) {
        if (r != -INFINITY) {
          lp_move(l2.f[0], s2.f[0], r - y);
          lp_move(l2.f[1], s2.f[1], r - y);
        }
        r = y;
      }
      return true;
    };
    auto add = [&](float d) {
      d = max_nan(d, LOWEST);                               // (-inf would make the product below NaN)
      const float e = exp2_approx(d);
      l2.f[0] += e;
      s2.f[0] = fmaf(e, d, s2.f[0]);
    };
    // (thread 0's p_... state runs ahead; sums and notes go to this row's half of `sh`)
    for (int v0 = rw.v_begin; v0 < rw.v_end; v0 += LP_CHUNK, ++count) {
      const int st = count % LP_STAGES;
      if (tid == 0) fetch();
      wait(&sh.full[st], (count / LP_STAGES) & 1);
      const uint4 *chunk = reinterpret_cast<const uint4 *>(lp_ring) + st * LP_CHUNK + tid;
      uint4 raw[LP_UNROLL];
#pragma unroll
      for (int u = 0; u < LP_UNROLL; ++u) raw[u] = chunk[u * LP_THREADS];
      if (v0 + LP_CHUNK > rw.v_end) {
        const uint32_t none = no_logits<T>();
#pragma unroll
        for (int u = 0; u < LP_UNROLL; ++u)
          if (v0 + u * LP_THREADS + tid >= rw.v_end) raw[u] = make_uint4(none, none, none, none);
      }
      const float vmax = chunk_max(raw, (const T *)nullptr);
      if (refer(vmax)) {
#pragma unroll
        for (int u = 0; u < LP_UNROLL; ++u) {
          float e[N];
          clamp_vec(raw[u], a.low, (const T *)nullptr);
          LpVec<T>::unpack(raw[u], e);
#pragma unroll
          for (int i = 0; i < N; i += 2) {
            F2 d = fma2(F2{{e[i], e[i + 1]}}, F2{{c, c}}, F2{{-r, -r}}), p;
            if (sizeof(T) == 4) { d.f[0] = max_nan(d.f[0], LOWEST); d.f[1] = max_nan(d.f[1], LOWEST); }
            p.f[0] = exp2_approx(d.f[0]);
            p.f[1] = exp2_approx(d.f[1]);
            l2 = add2(l2, p);
            s2 = fma2(p, d, s2);
          }
        }
      }
      if (TOP) {
        best = max_nan(best, vmax);
        any = any || v0 + tid < rw.v_end;
        const uint32_t mine = any ? order_key(best) : 0;
        *reinterpret_cast<volatile uint32_t *>(&sh.best[par][tid]) = mine;
        uint32_t key = *reinterpret_cast<volatile uint32_t *>(&sh.bound[par]);
        if (v0 == rw.v_begin) {                              // the first bound
          static_assert(LP_WARPS * 4 == 32, "four of each warp fill the lanes");
          const uint32_t sorted = sort_lanes(mine);
          if (lane < 4) sh.warp_top[par][warp * 4 + lane] = sorted;
          asm volatile("bar.sync 1, %0;" ::"n"(LP_THREADS) : "memory");
          key = kth_of_lanes(sh.warp_top[par][lane], k);
        }
        if (key) bound = max_nan(bound, key_value(key));
        // the vectors of a thread whose maximum reaches the bound are looked through by its whole warp
        for (unsigned hit = __ballot_sync(0xffffffffu, !(vmax < bound)); hit; hit &= hit - 1) {
          const int src = __ffs(hit) - 1, at0 = v0 + warp * 32 + src;
          const T *from = reinterpret_cast<const T *>(chunk + (src - lane));
          const float b = __shfl_sync(0xffffffffu, bound, src);
#pragma unroll
          for (int q = 0; q < LP_UNROLL * N / 32; ++q) {
            const int i = q * 32 + lane, at = at0 + i / N * LP_THREADS;
            const float v = lp_load(from + (size_t)(i / N) * LP_THREADS * N + i % N);
            if (at < rw.v_end && !(v < b)) note(v, rw.head + at * N + i % N);
          }
        }
      }
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(tc::smem_u32(&sh.empty[st]));
    }
    if (edge >= 0 && refer(edge_v)) add(fmaf(edge_v, c, -r));
    float l = l2.f[0] + l2.f[1], s = s2.f[0] + s2.f[1];
    if (m != -INFINITY) {
      if (fabsf(m * c) <= LP_FAR && m * c > a.low * c + 1024.f) {
        lp_move(l, s, r - m * c);
        lp_move(l, s, fmaf(-m, c, m * c));                  // (m c is a rounded product: what it lacks)
      } else {
        // logits whose products with c are too large, or which a lifted -inf would reach: this thread's once more, differences first
        l2.f[0] = s2.f[0] = 0.f;
        for (int at = rw.v_begin + tid; at < rw.v_end; at += LP_THREADS) {
          float e[N];
          LpVec<T>::unpack(xv[at], e);
#pragma unroll
          for (int i = 0; i < N; ++i) add((e[i] - m) * c);
        }
        if (edge >= 0) add((edge_v - m) * c);
        l = l2.f[0];
        s = s2.f[0];
      }
    }

    // ---- the row's sums and notes are complete.  Relative to the maximum l is at least 1, and log2 l is exact where one logit has
    // nearly all the mass.
    const LpSums t = lp_warp_join(LpSums{m, l, s}, c);
    if (lane == 0) sh.warp_sums[par][warp] = t;
    if (TOP) {
      sh.best[par][tid] = any ? order_key(best) : 0;
      if (edge >= 0) note(edge_v, edge);
    }
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(tc::smem_u32(&sh.row_done[par]));
    if (a.splits > 1) {
      cg::cluster_group cluster = cg::this_cluster();
      cluster.sync();
      cluster.sync();
    }
  }
  // giving up: copies under way land before the ring is given back (these waits are bounded too)
  if (tid == 0 && !alive)
    for (int i = max(0, p_count - LP_STAGES); i < p_count; ++i) tc::mbar_wait(tc::smem_u32(&sh.full[i % LP_STAGES]), (i / LP_STAGES) & 1);
}

// d logits = ( g_lp (1[v = t] - p_v) - g_H p_v (log p_v + H) ) / T  with p = exp(z - lse): elementwise, one read and one
// write of the logits' size.  LB: bytes of one load (16, or what the two rows' alignments have in common; stores are 16 wide)
struct LpBwdArgs {
  const void *logits;
  void *out;
  long long stride, out_stride;
  const int32_t *targets;
  const float *lse, *entropy, *g_lp, *g_h;
  int rows, vocab, blocks_per_row;
  float inv_t;
  unsigned int *status;
};
constexpr int LB_THREADS = 256, LB_UNROLL = 4;
template <typename T, int LB>
__global__ void __launch_bounds__(LB_THREADS) token_logprobs_bwd_kernel(LpBwdArgs a) {
  constexpr int N = LpVec<T>::N;
  const int row = blockIdx.x / a.blocks_per_row, part = blockIdx.x % a.blocks_per_row;
  const T *x = reinterpret_cast<const T *>(a.logits) + (size_t)row * a.stride;
  T *y = reinterpret_cast<T *>(a.out) + (size_t)row * a.out_stride;
  const int tgt = a.targets[row];
  if (tgt >= a.vocab && part == 0 && threadIdx.x == 0) atomicOr(a.status, STATUS_BAD_TOKEN);
  const bool known = tgt >= 0 && tgt < a.vocab;
  const float lse = a.lse[row], h = a.g_h ? a.entropy[row] : 0.f;
  const float gl = known ? a.g_lp[row] * a.inv_t : 0.f, gh = a.g_h ? a.g_h[row] * a.inv_t : 0.f;
  const float c = 1.4426950408889634f;
  auto grad = [&](float v, int i) {
    const float lp = fmaf(v, a.inv_t, -lse);
    const float p = exp2_approx(lp * c);
    const float d = p == 0.f ? 0.f : -p * fmaf(gh, lp + h, gl);      // (what has no probability has log p = -inf and no gradient)
    return i == tgt ? d + gl : d;
  };
  const int mis = (int)((reinterpret_cast<uintptr_t>(y) & 15) / sizeof(T));
  const int head = min(a.vocab, mis ? N - mis : 0);
  const int n_vec = (a.vocab - head) / N, tail0 = head + n_vec * N;
  if (part == 0) {
    if ((int)threadIdx.x < head) lp_store(y + threadIdx.x, grad(lp_load(x + threadIdx.x), threadIdx.x));
    const int i = tail0 + threadIdx.x;
    if (i < a.vocab) lp_store(y + i, grad(lp_load(x + i), i));
  }
  const int stride = a.blocks_per_row * LB_THREADS;
  for (int v0 = part * LB_THREADS + threadIdx.x; v0 < n_vec; v0 += stride * LB_UNROLL) {
    uint4 raw[LB_UNROLL];
#pragma unroll
    for (int u = 0; u < LB_UNROLL; ++u) {
      const int i = v0 + u * stride;
      if (i >= n_vec) continue;
      const T *src = x + head + (size_t)i * N;
      if constexpr (LB == 16) raw[u] = __ldcs(reinterpret_cast<const uint4 *>(src));
      else if constexpr (LB == 8) {
        const uint2 p0 = __ldg(reinterpret_cast<const uint2 *>(src)), p1 = __ldg(reinterpret_cast<const uint2 *>(src) + 1);
        raw[u] = make_uint4(p0.x, p0.y, p1.x, p1.y);
      } else if constexpr (LB == 4) {
        const uint32_t *p = reinterpret_cast<const uint32_t *>(src);
        raw[u] = make_uint4(__ldg(p), __ldg(p + 1), __ldg(p + 2), __ldg(p + 3));
      } else {
        const uint16_t *p = reinterpret_cast<const uint16_t *>(src);
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = (uint32_t)__ldg(p + 2 * j) | ((uint32_t)__ldg(p + 2 * j + 1) << 16);
        raw[u] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
#pragma unroll
    for (int u = 0; u < LB_UNROLL; ++u) {
      const int i = v0 + u * stride;
      if (i >= n_vec) continue;
      float e[N];
      LpVec<T>::unpack(raw[u], e);
#pragma unroll
      for (int j = 0; j < N; ++j) e[j] = grad(e[j], head + i * N + j);
      __stcs(reinterpret_cast<uint4 *>(y + head) + i, LpVec<T>::pack(e));
    }
  }
}

template <typename T>
cudaError_t launch_logprobs(const LpArgs &a, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  // persistent where rows are not split: two blocks fit an SM
  const int blocks = a.splits > 1 ? a.rows * a.splits : a.rows < 2 * num_sms() ? a.rows : 2 * num_sms();
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.dynamicSmemBytes = LP_SMEM;
  const void *kernel = a.top_k ? reinterpret_cast<const void *>(token_logprobs_kernel<T, true>) : reinterpret_cast<const void *>(token_logprobs_kernel<T, false>);
  if (ensure_dynamic_smem(kernel, LP_SMEM)) return cudaErrorInvalidValue;
  cfg.blockDim = dim3(LP_THREADS + 32);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)a.splits;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return a.top_k ? cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, true>, a) : cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, false>, a);
}
template <typename T>
cudaError_t launch_logprobs_bwd(const LpBwdArgs &a, cudaStream_t st) {
  const unsigned grid = (unsigned)((long long)a.rows * a.blocks_per_row);
  // what the input row is aligned to where the output row is aligned to 16 bytes, the same for every row
  const long long off = (long long)(reinterpret_cast<uintptr_t>(a.logits) & 15) - (long long)(reinterpret_cast<uintptr_t>(a.out) & 15);
  const long long step = (a.stride - a.out_stride) * (long long)sizeof(T);
  const unsigned long long both = (unsigned long long)off | (a.rows > 1 ? (unsigned long long)step : 0ull) | 16ull;
  const int common = (int)(both & (~both + 1));
  if (common >= 16) token_logprobs_bwd_kernel<T, 16><<<grid, LB_THREADS, 0, st>>>(a);
  else if (common == 8) token_logprobs_bwd_kernel<T, 8><<<grid, LB_THREADS, 0, st>>>(a);
  else if (common == 4) token_logprobs_bwd_kernel<T, 4><<<grid, LB_THREADS, 0, st>>>(a);
  else if constexpr (sizeof(T) == 2) token_logprobs_bwd_kernel<T, 2><<<grid, LB_THREADS, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace
}  // namespace skv

using namespace skv;

static int32_t check_logits(const void *logits, int64_t row_stride, int32_t rows, int32_t vocab, int32_t dtype, float temperature) {
  if (!logits) return report_error(SWIFTKV_ERR_INVALID_ARG, "null argument");
  // (the kernels count a row's elements in 32 bits, in steps of a block's work)
  if (rows < 1 || rows > (1 << 26) || vocab < 1 || vocab > (1 << 30) || row_stride < vocab)
    return report_error(SWIFTKV_ERR_INVALID_ARG, "bad shape (rows in [1, 2^26], vocab in [1, 2^30], row_stride >= vocab)");
  // (below 2^-125 the factor log2(e) / temperature would be infinite, and a row's largest logit 0 times it)
  if (!(temperature >= 0x1p-125f) || !(temperature < INFINITY)) return report_error(SWIFTKV_ERR_INVALID_ARG, "temperature must be in [2^-125, infinity)");
  if (dtype != SWIFTKV_DTYPE_F32 && dtype != SWIFTKV_DTYPE_BF16 && dtype != SWIFTKV_DTYPE_F16)
    return report_error(SWIFTKV_ERR_INVALID_ARG, "unknown dtype");
  if (reinterpret_cast<uintptr_t>(logits) % (dtype == SWIFTKV_DTYPE_F32 ? 4 : 2)) return report_error(SWIFTKV_ERR_INVALID_ARG, "misaligned logits");
  return SWIFTKV_OK;
}

extern "C" int32_t swiftkv_token_logprobs(const void *logits, int64_t row_stride, int32_t dtype, const int32_t *targets, int32_t rows,
                                          int32_t vocab, float temperature, int32_t top_k, float *logprob, float *entropy, float *lse,
                                          int32_t *top_ids, float *top_logprobs, void *cuda_stream) {
  if (const int32_t rc = check_logits(logits, row_stride, rows, vocab, dtype, temperature)) return rc;
  if (!logprob || !entropy || !lse || (top_k > 0 && (!top_ids || !top_logprobs))) return report_error(SWIFTKV_ERR_INVALID_ARG, "null argument");
  if (top_k < 0 || top_k > LP_MAX_TOP || top_k > vocab) return report_error(SWIFTKV_ERR_INVALID_ARG, "top_k outside [0, min(32, vocab)]");
  unsigned int *status = op_status_word();
  if (!status) return report_error(SWIFTKV_ERR_CUDA, "no status word");
  // a row is split as far as all blocks run at once (two fit an SM; 64 x 128256 fp32: 13 us with 4 parts, 22 us with 8) and every
  // part keeps thousands of logits
  int splits = 1;
  while (splits < LP_MAX_CLUSTER && (long long)rows * splits * 2 <= 2 * num_sms() && vocab / (2 * splits) >= 4096) splits *= 2;
  LpArgs a{logits, row_stride, targets, logprob, entropy, lse, top_logprobs, top_ids, rows, vocab, top_k, splits, (float)(1.4426950408889634 / temperature), 1.0f / temperature, 0.f, status};
  a.low = dtype == SWIFTKV_DTYPE_F16 ? -65504.f : (float)(-2e38 / (a.c > 1.f ? a.c : 1.f));
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = dtype == SWIFTKV_DTYPE_F32 ? launch_logprobs<float>(a, st) : dtype == SWIFTKV_DTYPE_BF16 ? launch_logprobs<bf16>(a, st) : launch_logprobs<__half>(a, st);
  if (e != cudaSuccess) return report_error(SWIFTKV_ERR_CUDA, cudaGetErrorString(e));
  return SWIFTKV_OK;
}

extern "C" int32_t swiftkv_token_logprobs_bwd(const void *logits, int64_t row_stride, int32_t dtype, const int32_t *targets, int32_t rows,
                                              int32_t vocab, float temperature, const float *lse, const float *entropy,
                                              const float *grad_logprob, const float *grad_entropy, void *grad_logits,
                                              int64_t grad_stride, void *cuda_stream) {
  if (const int32_t rc = check_logits(logits, row_stride, rows, vocab, dtype, temperature)) return rc;
  if (!targets || !lse || !grad_logprob || !grad_logits || (grad_entropy && !entropy)) return report_error(SWIFTKV_ERR_INVALID_ARG, "null argument");
  if (grad_stride < vocab) return report_error(SWIFTKV_ERR_INVALID_ARG, "bad shape (grad_stride >= vocab)");
  const size_t es = dtype == SWIFTKV_DTYPE_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(grad_logits) % es) return report_error(SWIFTKV_ERR_INVALID_ARG, "misaligned gradient");
  // in place (same pointer, same stride) every element is read before the thread that read it writes it; any other overlap is not
  const uintptr_t i0 = reinterpret_cast<uintptr_t>(logits), o0 = reinterpret_cast<uintptr_t>(grad_logits);
  const size_t i_n = ((size_t)(rows - 1) * row_stride + vocab) * es, o_n = ((size_t)(rows - 1) * grad_stride + vocab) * es;
  if (i0 < o0 + o_n && o0 < i0 + i_n && !(i0 == o0 && row_stride == grad_stride))
    return report_error(SWIFTKV_ERR_INVALID_ARG, "the gradient overlaps the logits other than in place");
  unsigned int *status = op_status_word();
  if (!status) return report_error(SWIFTKV_ERR_CUDA, "no status word");
  const int n_vec = (int)(((size_t)vocab * es + 15) / 16);
  int per_row = (n_vec + LB_THREADS * LB_UNROLL - 1) / (LB_THREADS * LB_UNROLL);
  if ((long long)rows * per_row > 0x7fffffffLL) per_row = 1;
  LpBwdArgs a{logits, grad_logits, row_stride, grad_stride, targets, lse, entropy, grad_logprob, grad_entropy, rows, vocab, per_row, 1.0f / temperature, status};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = dtype == SWIFTKV_DTYPE_F32 ? launch_logprobs_bwd<float>(a, st) : dtype == SWIFTKV_DTYPE_BF16 ? launch_logprobs_bwd<bf16>(a, st) : launch_logprobs_bwd<__half>(a, st);
  if (e != cudaSuccess) return report_error(SWIFTKV_ERR_CUDA, cudaGetErrorString(e));
  return SWIFTKV_OK;
}
