// swiftkv_token_logprobs: log probability of a given token per row of logits, with the row's log-sum-exp, entropy and its
// top_k alternatives, in ONE pass over the logits; swiftkv_token_logprobs_bwd: the gradient with respect to the logits.
//
// With z = x / T and m the running maximum of x, a thread keeps
//   l = sum exp(z - m/T)      and      s = sum exp(z - m/T) (x - m)
// so that  lse = m/T + log l,  entropy = log l - (s / T) / l  (every term of s has one sign: nothing cancels), and
// logprob(t) = (x_t - m)/T - log l.  All sums are fp32; x - m is formed before the multiplication by log2(e)/T, so an
// exponent's error is relative to the exponent and not to the logit.
//
// Top-k: every warp keeps its k best (value, index) pairs sorted across its lanes.  A vector of logits is looked at only if
// its maximum -- needed for m anyway -- passes the warp's k-th best and the best k-th value of all the block's warps, which
// after the first few thousand logits hardly happens (about k ln(n / 1024) times per warp).  Elements are met in ascending
// index order, so that of equal values the lowest index stays.
//
// What bounds it: HBM (the logits are read once).  Few rows: a row is shared by a cluster of up to 8 blocks whose partial
// results meet in distributed shared memory, so one launch needs no workspace at any size.
#include <cooperative_groups.h>

#include "common.cuh"
#include "tc_common.cuh"

namespace skv {
namespace {
namespace cg = cooperative_groups;

constexpr int LP_THREADS = 512, LP_WARPS = LP_THREADS / 32;
constexpr int LP_MAX_TOP = 32;
constexpr int LP_MAX_CLUSTER = 8;
constexpr int LP_UNROLL = 4;                 // 16-byte loads in flight per thread
constexpr float LP_RESCALE = 16.f;           // the reference maximum moves when the sums could grow by more than 2^16
constexpr float LOWEST = -3.0e38f;

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
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

struct LpSums { float m, l, s; };
// sums relative to a.m -> relative to m: factor f, and s moves by l (a.m - m).  A factor of zero drops them: the distance may then
// be as large as the type's lowest value (a masked logit met first), whose multiple by l is not finite.
__device__ __forceinline__ void lp_move(LpSums a, float m, float c, float &l, float &s) {
  const float d = a.m - m, f = exp2_approx(d * c);
  l = a.l * f;                                            // (a NaN stays one)
  s = f == 0.f ? l : (a.s + a.l * d) * f;
}
__device__ __forceinline__ void lp_rescale(LpSums &a, float m_new, float c) {
  // (before the first finite logit the sums are 0, or NaN)
  if (a.m != -INFINITY) lp_move(a, m_new, c, a.l, a.s);
  a.m = m_new;
}
__device__ __forceinline__ LpSums lp_join(LpSums a, LpSums b, float c) {
  const float m = max_nan(a.m, b.m);
  lp_rescale(a, m, c);
  lp_rescale(b, m, c);
  return LpSums{m, a.l + b.l, a.s + b.s};
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
  float inv_t;
  unsigned int *status;
};

struct LpShared {
  LpSums warp_sums[LP_WARPS];
  LpSums sums;
  uint32_t key[LP_WARPS][LP_MAX_TOP];
  int idx[LP_WARPS][LP_MAX_TOP];
  uint32_t best_kth;
};

template <typename T, bool TOP>
__global__ void __launch_bounds__(LP_THREADS, 2) token_logprobs_kernel(LpArgs a) {
  constexpr int N = LpVec<T>::N;
  __shared__ LpShared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row = blockIdx.x / a.splits, part = blockIdx.x % a.splits;
  const T *x = reinterpret_cast<const T *>(a.logits) + (size_t)row * a.stride;
  const float c = a.inv_t * 1.4426950408889634f;
  const int k = a.top_k;
  if (TOP) {
    if (tid == 0) sh.best_kth = 0;
    __syncthreads();
  }
  LpSums t{-INFINITY, 0.f, 0.f};
  float m_true = -INFINITY;      // (t.m may lag behind it by LP_RESCALE)
  WarpTop top;
  auto add = [&](float v) {
    const float d = max_nan(v - (t.m == -INFINITY ? 0.f : t.m), LOWEST);
    const float e = exp2_approx(d * c);
    t.l += e;
    t.s = fmaf(e, d, t.s);
  };
  auto refer = [&](float vmax) {
    m_true = fmaxf(m_true, vmax);
    if ((vmax - t.m) * c > LP_RESCALE || (t.m == -INFINITY && vmax > t.m)) lp_rescale(t, vmax, c);
  };
  // offers the warp's elements v (one per lane, index i, `ok` where there is one) to its list, lowest lane first
  auto offer = [&](float v, int i, bool ok) {
    const uint32_t key = ok ? order_key(v) : 0;
    unsigned pass = __ballot_sync(0xffffffffu, key > top.kth);
    while (pass) {
      const int src = __ffs(pass) - 1;
      pass &= pass - 1;
      const uint32_t ck = __shfl_sync(0xffffffffu, key, src);
      if (ck > top.kth) top.insert(ck, __shfl_sync(0xffffffffu, i, src), k);
    }
  };

  // elements before the first 16-byte boundary of the row, whole vectors, elements behind the last one
  const int mis = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));
  const int head = min(a.vocab, mis ? N - mis : 0);
  const int n_vec = (a.vocab - head) / N;
  const int tail0 = head + n_vec * N;
  if (part == 0 && warp == 0 && head) {
    const bool ok = lane < head;
    const float v = ok ? lp_load(x + lane) : -INFINITY;
    if (ok) { refer(v); add(v); }
    if (TOP) offer(v, lane, ok);
  }
  const uint4 *xv = reinterpret_cast<const uint4 *>(x + head);
  const int v_begin = (int)((long long)n_vec * part / a.splits), v_end = (int)((long long)n_vec * (part + 1) / a.splits);
  for (int v0 = v_begin; v0 < v_end; v0 += LP_THREADS * LP_UNROLL) {
    uint4 raw[LP_UNROLL];
#pragma unroll
    for (int u = 0; u < LP_UNROLL; ++u) {
      const int i = v0 + u * LP_THREADS + tid;
      if (i < v_end) raw[u] = __ldcs(xv + i);
    }
    float vm[LP_UNROLL];
#pragma unroll
    for (int u = 0; u < LP_UNROLL; ++u) {
      const bool ok = v0 + u * LP_THREADS + tid < v_end;
      vm[u] = -INFINITY;
      if (ok) {
        float e[N];
        LpVec<T>::unpack(raw[u], e);
        float mx = e[0];
#pragma unroll
        for (int i = 1; i < N; ++i) mx = max_nan(mx, e[i]);
        vm[u] = mx;
        refer(mx);
        const float mr = t.m == -INFINITY ? 0.f : t.m;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float d = max_nan(e[i] - mr, LOWEST);
          const float p = exp2_approx(d * c);
          t.l += p;
          t.s = fmaf(p, d, t.s);
        }
      }
    }
    if (TOP) {
      uint32_t floor_key = max(top.kth, *reinterpret_cast<volatile uint32_t *>(&sh.best_kth));
      if (v0 == v_begin) {
        // nothing is known yet: at least k elements reach the k-th largest of the lanes' maxima, so only those are sorted in
        float best = vm[0];
#pragma unroll
        for (int u = 1; u < LP_UNROLL; ++u) best = max_nan(best, vm[u]);
        const bool any = v0 + tid < v_end;
        uint32_t mine = any ? order_key(best) : 0;
        // rank of this lane's maximum among the warp's (ties by lane): the lane of rank k - 1 holds the bound
        int rank = 0;
#pragma unroll
        for (int o = 0; o < 32; ++o) {
          const uint32_t other = __shfl_sync(0xffffffffu, mine, o);
          rank += other > mine || (other == mine && o < lane);
        }
        const unsigned at = __ballot_sync(0xffffffffu, rank == k - 1);
        floor_key = max(floor_key, __shfl_sync(0xffffffffu, mine, __ffs(at) - 1));
      }
      const uint32_t had = top.kth;
#pragma unroll
      for (int u = 0; u < LP_UNROLL; ++u) {
        const bool ok = v0 + u * LP_THREADS + tid < v_end;
        // (>= the floor: a value equal to another warp's k-th may still win by its index)
        const uint32_t mk = ok ? order_key(vm[u]) : 0;
        unsigned hit = __ballot_sync(0xffffffffu, ok && mk >= floor_key && mk > top.kth);
        while (hit) {
          const int src = __ffs(hit) - 1;
          hit &= hit - 1;
          float e[N];
          LpVec<T>::unpack(raw[u], e);
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const uint32_t ck = __shfl_sync(0xffffffffu, order_key(e[i]), src);
            if (ck >= floor_key && ck > top.kth) top.insert(ck, head + (v0 + u * LP_THREADS + warp * 32 + src) * N + i, k);
          }
        }
      }
      if (top.kth > had && lane == 0) atomicMax(&sh.best_kth, top.kth);
    }
  }
  if (part == a.splits - 1 && warp == 0 && tail0 < a.vocab) {
    const bool ok = lane < a.vocab - tail0;
    const float v = ok ? lp_load(x + tail0 + lane) : -INFINITY;
    if (ok) { refer(v); add(v); }
    if (TOP) offer(v, tail0 + lane, ok);
  }

  // ---- the block's sums and list, then the cluster's.  Relative to the true maximum l is at least 1 and log l is exact where
  // one logit has nearly all the mass.
  if (m_true > t.m) lp_rescale(t, m_true, c);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const LpSums b{__shfl_xor_sync(0xffffffffu, t.m, o), __shfl_xor_sync(0xffffffffu, t.l, o), __shfl_xor_sync(0xffffffffu, t.s, o)};
    // both lanes of a pair join in the same order, so that every lane ends with the same bits
    t = (lane & o) ? lp_join(b, t, c) : lp_join(t, b, c);
  }
  if (lane == 0) sh.warp_sums[warp] = t;
  if (TOP) { sh.key[warp][lane] = lane < k ? top.key : 0; sh.idx[warp][lane] = top.idx; }
  __syncthreads();
  if (warp == 0) {
    LpSums b = lane < LP_WARPS ? sh.warp_sums[lane] : LpSums{-INFINITY, 0.f, 0.f};
#pragma unroll
    for (int o = LP_WARPS / 2; o > 0; o >>= 1) {
      const LpSums d{__shfl_xor_sync(0xffffffffu, b.m, o), __shfl_xor_sync(0xffffffffu, b.l, o), __shfl_xor_sync(0xffffffffu, b.s, o)};
      b = (lane & o) ? lp_join(d, b, c) : lp_join(b, d, c);
    }
    if (lane == 0) sh.sums = b;
    if (TOP) {
      for (int w = 1; w < LP_WARPS; ++w) {
        const uint32_t wk = sh.key[w][lane];
        const int wi = sh.idx[w][lane];
        for (int i = 0; i < k; ++i) {              // lists are sorted: the first that does not enter ends one
          const uint32_t ck = __shfl_sync(0xffffffffu, wk, i);
          const int ci = __shfl_sync(0xffffffffu, wi, i);
          const int li = __shfl_sync(0xffffffffu, top.idx, k - 1);
          if (ck == 0 || ck < top.kth || (ck == top.kth && ci > li)) break;
          top.insert(ck, ci, k);
        }
      }
      __syncwarp();
      sh.key[0][lane] = lane < k ? top.key : 0;
      sh.idx[0][lane] = top.idx;
    }
  }
  LpSums all;
  if (a.splits > 1) {
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    if (part == 0 && warp == 0) {
      all = sh.sums;
      for (int r = 1; r < a.splits; ++r) {
        const LpShared *o = cluster.map_shared_rank(&sh, r);
        all = lp_join(all, o->sums, c);
        if (TOP) {
          const uint32_t wk = o->key[0][lane];
          const int wi = o->idx[0][lane];
          for (int i = 0; i < k; ++i) {
            const uint32_t ck = __shfl_sync(0xffffffffu, wk, i);
            const int ci = __shfl_sync(0xffffffffu, wi, i);
            const int li = __shfl_sync(0xffffffffu, top.idx, k - 1);
            if (ck == 0 || ck < top.kth || (ck == top.kth && ci > li)) break;
            top.insert(ck, ci, k);
          }
        }
      }
    }
    cluster.sync();                                 // no block leaves while its shared memory is read
  } else {
    __syncwarp();
    all = sh.sums;
  }
  if (part == 0 && warp == 0) {
    const float log_l = all.m == -INFINITY ? -INFINITY : logf(all.l);
    const float mz = all.m * a.inv_t;
    if (lane == 0) {
      a.lse[row] = all.m == -INFINITY ? -INFINITY + all.l : mz + log_l;
      a.entropy[row] = all.m == -INFINITY ? __uint_as_float(0x7fffffffu) : log_l - all.s * a.inv_t / all.l;
      const int tgt = a.targets ? a.targets[row] : -1;
      float lp = 0.f;
      if (tgt >= a.vocab) atomicOr(a.status, STATUS_BAD_TOKEN);
      else if (tgt >= 0) lp = (lp_load(x + tgt) - all.m) * a.inv_t - log_l;
      a.logprob[row] = lp;
    }
    if (TOP && lane < k) {
      a.top_ids[(size_t)row * k + lane] = top.idx;
      a.top_lp[(size_t)row * k + lane] = (key_value(top.key) - all.m) * a.inv_t - log_l;
    }
  }
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
  cfg.gridDim = dim3((unsigned)((long long)a.rows * a.splits));
  cfg.blockDim = dim3(LP_THREADS);
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
  if (rows < 1 || rows > (1 << 26) || vocab < 1 || row_stride < vocab)
    return report_error(SWIFTKV_ERR_INVALID_ARG, "bad shape (rows in [1, 2^26], vocab >= 1, row_stride >= vocab)");
  if (!(temperature > 0.f) || !(temperature < INFINITY)) return report_error(SWIFTKV_ERR_INVALID_ARG, "temperature must be positive and finite");
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
  // two blocks fit an SM: a row is split while that leaves half of them idle and every part keeps a few thousand logits
  int splits = 1;
  while (splits < LP_MAX_CLUSTER && (long long)rows * splits < num_sms() && vocab / (2 * splits) >= 4096) splits *= 2;
  LpArgs a{logits, row_stride, targets, logprob, entropy, lse, top_logprobs, top_ids, rows, vocab, top_k, splits, 1.0f / temperature, status};
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
