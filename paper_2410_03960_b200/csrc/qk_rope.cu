// swiftkv_qk_norm_rope: per-head RMSNorm of queries and keys, rotary embedding, and the store of the keys and values into
// cache rows, in one pass; swiftkv_qk_norm_rope_bwd: its gradient.
//
// Per head x of hd elements, with pairs (i, i + hd/2), c = cos, s = sin of position * theta^(-2i/hd):
//   h = x * rsqrt(mean(x^2) + eps) * g        (g null: h = x)
//   y_i = h_i c_i - h_{i+hd/2} s_i,   y_{i+hd/2} = h_{i+hd/2} c_i + h_i s_i
// backward, dz = the inverse rotation of dy, xh = x r, r = rsqrt(mean(x^2) + eps):
//   dg = sum over tokens and heads of dz xh;     dx = r (dz g - xh mean(dz g xh)).
// Everything is fp32 between the load and the one rounding of the store.  An FP8 cache row is quantized from that fp32 row
// (scale = max(max|y|, 2^-64) / 448, code = e4m3(y / scale), as swiftkv_quantize_rows_fp8), not from a 16-bit copy of it.
//
// What bounds it: HBM, every row read once and written once.  Vector form: hd/16 lanes hold one head, 16 bytes of its lower
// and 16 bytes of its upper half each, so a rotation pair sits in one thread, a head's mean needs log2(hd/16) shuffles, and
// a thread's cos / sin / gain values serve every head that it walks over.  Other shapes, fp32 and unaligned tensors take the
// general form (one warp per head, a pair per lane and step).
#include "common.cuh"
#include "tc_common.cuh"

namespace skv {
namespace {

enum : int { ROLE_ALL = 0, ROLE_Q = 1, ROLE_K = 2, ROLE_V = 3 };

struct RopeArgs {
  const void *q, *k, *v;                     // [T][n][hd], token strides in elements
  long long q_stride, k_stride, v_stride;
  const void *q_gain, *k_gain;               // [hd] or null
  const int32_t *positions;
  const float *cos_tab, *sin_tab;            // [max_pos][hd / 2]
  const int32_t *slot_map;                   // null: row t
  void *q_out, *k_out, *v_out;               // q_out: token stride qo_stride; k_out, v_out: [cache_rows][n_kv][hd]
  long long qo_stride;
  float *k_scale, *v_scale;                  // FP8 rows
  int tokens, n_q, n_kv, hd, max_pos, cache_rows;
  float eps;
  unsigned int *status;
};

// ---- 16 bytes of a 16-bit type as 8 floats ---------------------------------------------------------------
__device__ __forceinline__ void unpack8(const uint4 &v, float (&x)[8], const bf16 *) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void unpack8(const uint4 &v, float (&x)[8], const __half *) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
    x[2 * i] = f.x; x[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8], const bf16 *) {
  return make_uint4(tc::pack_bf16x2(x[0], x[1]), tc::pack_bf16x2(x[2], x[3]), tc::pack_bf16x2(x[4], x[5]), tc::pack_bf16x2(x[6], x[7]));
}
// half stores round like a cast (beyond the range: infinity)
__device__ __forceinline__ uint4 pack8(const float (&x)[8], const __half *) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t *>(&h);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T> __device__ __forceinline__ T round_to(float v);
template <> __device__ __forceinline__ float round_to<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 round_to<bf16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half round_to<__half>(float v) { return __float2half_rn(v); }

__device__ __forceinline__ uint8_t code_of(float x, float scale) {
  return (uint8_t)__nv_cvt_float_to_fp8(__fdiv_rn(x, scale), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float row_scale(float amax) { return __fdiv_rn(fmaxf(amax, FP8_AMAX_FLOOR), FP8_MAX); }

__device__ __forceinline__ int checked_position(const RopeArgs &a, int t) {
  const int p = a.positions[t];
  if (p >= 0 && p < a.max_pos) return p;
  if (threadIdx.x == 0) atomicOr(a.status, STATUS_BAD_TOKEN);
  return p < 0 ? 0 : a.max_pos - 1;
}
// cache row of token t, -1: not stored
__device__ __forceinline__ int checked_slot(const RopeArgs &a, int t) {
  const int s = a.slot_map ? a.slot_map[t] : t;
  if (s < a.cache_rows) return s < 0 ? -1 : s;
  if (threadIdx.x == 0) atomicOr(a.status, STATUS_BAD_TOKEN);
  return -1;
}

__device__ __forceinline__ float block_max_all(float v, float *red, int warps) {
  v = warp_max(v);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  float m = red[0];
  for (int w = 1; w < warps; ++w) m = fmaxf(m, red[w]);
  return m;
}

__device__ __forceinline__ void load8f(const float *p, float (&x)[8]) {
  const float4 a = __ldg(reinterpret_cast<const float4 *>(p)), b = __ldg(reinterpret_cast<const float4 *>(p) + 1);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}

// ---- forward, vector form: block (token) or, FP8, (token, Q / K / V) --------------------------------------
// UNITS heads are loaded together per thread, so that their loads are in flight at once
template <typename T, int L, int UNITS>
__global__ void qk_norm_rope_vec_kernel(RopeArgs a) {
  const int t = blockIdx.x, half = 8 * L;
  const int sub = threadIdx.x % L, unit0 = threadIdx.x / L, step = blockDim.x / L;
  const int n_units = a.n_q + 2 * a.n_kv;
  const int slot = checked_slot(a, t), pos = checked_position(a, t);
  uint4 lo[UNITS], hi[UNITS];
  auto source = [&](int u) -> const T * {
    if (u < a.n_q) return reinterpret_cast<const T *>(a.q) + (size_t)t * a.q_stride + (size_t)u * (2 * half);
    u -= a.n_q;
    if (u < a.n_kv) return reinterpret_cast<const T *>(a.k) + (size_t)t * a.k_stride + (size_t)u * (2 * half);
    return reinterpret_cast<const T *>(a.v) + (size_t)t * a.v_stride + (size_t)(u - a.n_kv) * (2 * half);
  };
  float c[8], s[8];
  for (int base = 0; base < n_units; base += step * UNITS) {
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int u = base + unit0 + i * step;
      if (u < n_units) {
        const uint4 *p = reinterpret_cast<const uint4 *>(source(u) + 8 * sub);
        lo[i] = __ldcs(p);
        hi[i] = __ldcs(p + L);
      }
    }
    if (base == 0) {
      load8f(a.cos_tab + (size_t)pos * half + 8 * sub, c);
      load8f(a.sin_tab + (size_t)pos * half + 8 * sub, s);
    }
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int u = base + unit0 + i * step;
      const bool ok = u < n_units, is_q = u < a.n_q, is_v = u >= a.n_q + a.n_kv;
      // every lane of a warp walks the shuffles of the norm (heads of one warp may belong to q, K and V)
      float x0[8], x1[8];
      if (!ok) { lo[i] = hi[i] = make_uint4(0u, 0u, 0u, 0u); }
      unpack8(lo[i], x0, (const T *)nullptr);
      unpack8(hi[i], x1, (const T *)nullptr);
      const T *gain = reinterpret_cast<const T *>(is_q ? a.q_gain : a.k_gain);
      float r = 1.f;
      if (a.q_gain || a.k_gain) {
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) ss = fmaf(x0[j], x0[j], fmaf(x1[j], x1[j], ss));
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        r = rsqrtf(ss * (1.f / (16 * L)) + a.eps);
      }
      if (!ok) continue;
      if (is_v) {
        if (slot >= 0) {
          uint4 *d = reinterpret_cast<uint4 *>(reinterpret_cast<T *>(a.v_out) + ((size_t)slot * a.n_kv + (u - a.n_q - a.n_kv)) * (2 * half) + 8 * sub);
          d[0] = lo[i];
          d[L] = hi[i];
        }
        continue;
      }
      if (gain) {
        float g[8];
        unpack8(__ldg(reinterpret_cast<const uint4 *>(gain + 8 * sub)), g, (const T *)nullptr);
#pragma unroll
        for (int j = 0; j < 8; ++j) x0[j] *= r * g[j];
        unpack8(__ldg(reinterpret_cast<const uint4 *>(gain + half + 8 * sub)), g, (const T *)nullptr);
#pragma unroll
        for (int j = 0; j < 8; ++j) x1[j] *= r * g[j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float y0 = x0[j] * c[j] - x1[j] * s[j], y1 = x1[j] * c[j] + x0[j] * s[j];
        x0[j] = y0;
        x1[j] = y1;
      }
      uint4 *d;
      if (is_q) d = reinterpret_cast<uint4 *>(reinterpret_cast<T *>(a.q_out) + (size_t)t * a.qo_stride + (size_t)u * (2 * half) + 8 * sub);
      else if (slot >= 0) d = reinterpret_cast<uint4 *>(reinterpret_cast<T *>(a.k_out) + ((size_t)slot * a.n_kv + (u - a.n_q)) * (2 * half) + 8 * sub);
      else continue;
      d[0] = pack8(x0, (const T *)nullptr);
      d[L] = pack8(x1, (const T *)nullptr);
    }
  }
}

// ---- forward, general form: block (token, role); one warp per head, lane and step one rotation pair ---------
// A row of an FP8 cache waits in shared memory as fp32 between its maximum and its codes.
constexpr int RG_THREADS = 256;
template <typename T>
__global__ void __launch_bounds__(RG_THREADS) qk_norm_rope_kernel(RopeArgs a, int first_role) {
  extern __shared__ float rg_row[];                // [n_kv * hd], FP8 rows only
  __shared__ float red[RG_THREADS / 32];
  const int t = blockIdx.x, role = first_role + blockIdx.y, half = a.hd >> 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool fp8 = role != ROLE_Q && a.k_scale != nullptr;
  const int pos = checked_position(a, t);
  const int slot = role == ROLE_Q ? 0 : checked_slot(a, t);
  const int heads = role == ROLE_Q ? a.n_q : a.n_kv;
  const T *src = role == ROLE_Q ? reinterpret_cast<const T *>(a.q) + (size_t)t * a.q_stride
                : role == ROLE_K ? reinterpret_cast<const T *>(a.k) + (size_t)t * a.k_stride : reinterpret_cast<const T *>(a.v) + (size_t)t * a.v_stride;
  const T *gain = reinterpret_cast<const T *>(role == ROLE_Q ? a.q_gain : role == ROLE_K ? a.k_gain : nullptr);
  if (slot < 0) return;
  T *dst = role == ROLE_Q ? reinterpret_cast<T *>(a.q_out) + (size_t)t * a.qo_stride
                          : reinterpret_cast<T *>(role == ROLE_K ? a.k_out : a.v_out) + (size_t)slot * a.n_kv * a.hd;
  float amax = 0.f;
  for (int h = warp; h < heads; h += RG_THREADS / 32) {
    float x0[4], x1[4], ss = 0.f;                  // hd <= 256: at most 4 pairs per lane
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = lane + 32 * j;
      x0[j] = x1[j] = 0.f;
      if (i < half) { x0[j] = to_f(src[h * a.hd + i]); x1[j] = to_f(src[h * a.hd + i + half]); }
      ss = fmaf(x0[j], x0[j], fmaf(x1[j], x1[j], ss));
    }
    float r = 1.f;
    if (gain) r = rsqrtf(warp_sum(ss) / a.hd + a.eps);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = lane + 32 * j;
      if (i >= half) continue;
      float y0 = x0[j], y1 = x1[j];
      if (gain) { y0 *= r * to_f(gain[i]); y1 *= r * to_f(gain[i + half]); }
      if (role != ROLE_V) {
        const float c = a.cos_tab[(size_t)pos * half + i], s = a.sin_tab[(size_t)pos * half + i];
        const float z0 = y0 * c - y1 * s;
        y1 = y1 * c + y0 * s;
        y0 = z0;
      }
      if (fp8) {
        rg_row[h * a.hd + i] = y0;
        rg_row[h * a.hd + i + half] = y1;
        amax = fmaxf(amax, fmaxf(fabsf(y0), fabsf(y1)));
      } else {
        dst[h * a.hd + i] = round_to<T>(y0);
        dst[h * a.hd + i + half] = round_to<T>(y1);
      }
    }
  }
  if (fp8) {
    amax = block_max_all(amax, red, RG_THREADS / 32);       // (its barrier also publishes the row)
    const float scale = row_scale(amax);
    if (threadIdx.x == 0) (role == ROLE_K ? a.k_scale : a.v_scale)[slot] = scale;
    uint8_t *codes = reinterpret_cast<uint8_t *>(role == ROLE_K ? a.k_out : a.v_out) + (size_t)slot * a.n_kv * a.hd;
    for (int i = threadIdx.x; i < a.n_kv * a.hd; i += RG_THREADS) codes[i] = code_of(rg_row[i], scale);
  }
}

// ---- backward ------------------------------------------------------------------------------------------------
struct RopeBwdArgs {
  const void *dq, *dk;                       // [T][n][hd] contiguous
  const void *q, *k;
  long long q_stride, k_stride;
  const void *q_gain, *k_gain;
  const int32_t *positions;
  const float *cos_tab, *sin_tab;
  void *dq_in, *dk_in;                       // [T][n][hd] contiguous; dq_in == dq, dk_in == dk allowed
  float *partial;                            // [blocks][2][hd] gain gradients of each block
  int tokens, n_q, n_kv, hd, max_pos;
  float eps;
  unsigned int *status;
};
constexpr int RB_THREADS = 256;
constexpr int RB_BLOCKS_PER_SM = 4;

// vector form: L lanes per head; a block walks over tokens, a thread over heads of a token; gain gradients stay in registers
template <typename T, int L>
__global__ void __launch_bounds__(RB_THREADS) qk_norm_rope_bwd_vec_kernel(RopeBwdArgs a) {
  constexpr int half = 8 * L, HD = 16 * L, GROUPS = RB_THREADS / L;
  __shared__ float red[RB_THREADS / 32][HD];
  const int sub = threadIdx.x % L, unit0 = threadIdx.x / L;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll 1
  for (int which = 0; which < 2; ++which) {
    const int heads = which ? a.n_kv : a.n_q;
    const T *gain = reinterpret_cast<const T *>(which ? a.k_gain : a.q_gain);
    const T *x = reinterpret_cast<const T *>(which ? a.k : a.q);
    const long long x_stride = which ? a.k_stride : a.q_stride;
    const T *dy = reinterpret_cast<const T *>(which ? a.dk : a.dq);
    T *dx = reinterpret_cast<T *>(which ? a.dk_in : a.dq_in);
    float gl[8], gh[8], al[8], ah[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) al[j] = ah[j] = 0.f;
    if (gain) {
      unpack8(__ldg(reinterpret_cast<const uint4 *>(gain + 8 * sub)), gl, (const T *)nullptr);
      unpack8(__ldg(reinterpret_cast<const uint4 *>(gain + half + 8 * sub)), gh, (const T *)nullptr);
    }
    // (token, head) pairs in order, GROUPS of them per step of the block; whole warps stay together for the shuffles
    const long long n_units = (long long)a.tokens * heads, grid_step = (long long)gridDim.x * GROUPS;
    for (long long base = (long long)blockIdx.x * GROUPS; base < n_units; base += grid_step) {
      const long long u = base + unit0;
      const bool ok = u < n_units;
      const int t = ok ? (int)(u / heads) : 0, h = ok ? (int)(u - (long long)t * heads) : 0;
      uint4 d0 = make_uint4(0u, 0u, 0u, 0u), d1 = d0, v0 = d0, v1 = d0;
      float c[8], s[8];
      if (ok) {
        const uint4 *p = reinterpret_cast<const uint4 *>(dy + ((size_t)t * heads + h) * HD + 8 * sub);
        d0 = p[0];
        d1 = p[L];
        if (gain) {
          const uint4 *xp = reinterpret_cast<const uint4 *>(x + (size_t)t * x_stride + (size_t)h * HD + 8 * sub);
          v0 = xp[0];
          v1 = xp[L];
        }
      }
      int pos = a.positions[t];
      if (pos < 0 || pos >= a.max_pos) {
        if (sub == 0) atomicOr(a.status, STATUS_BAD_TOKEN);
        pos = pos < 0 ? 0 : a.max_pos - 1;
      }
      load8f(a.cos_tab + (size_t)pos * half + 8 * sub, c);
      load8f(a.sin_tab + (size_t)pos * half + 8 * sub, s);
      float z0[8], z1[8], x0[8], x1[8];
      unpack8(d0, z0, (const T *)nullptr);
      unpack8(d1, z1, (const T *)nullptr);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float w0 = z0[j] * c[j] + z1[j] * s[j], w1 = z1[j] * c[j] - z0[j] * s[j];
        z0[j] = w0;
        z1[j] = w1;
      }
      if (gain) {
        unpack8(v0, x0, (const T *)nullptr);
        unpack8(v1, x1, (const T *)nullptr);
        float ss = 0.f, dot = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          ss = fmaf(x0[j], x0[j], fmaf(x1[j], x1[j], ss));
          dot = fmaf(z0[j] * gl[j], x0[j], fmaf(z1[j] * gh[j], x1[j], dot));
        }
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) {
          ss += __shfl_xor_sync(0xffffffffu, ss, o);
          dot += __shfl_xor_sync(0xffffffffu, dot, o);
        }
        const float r = rsqrtf(ss * (1.f / HD) + a.eps);
        const float m = dot * r * r * (1.f / HD);          // mean(dz g xh) r, to be multiplied by x
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (ok) { al[j] = fmaf(z0[j], x0[j] * r, al[j]); ah[j] = fmaf(z1[j], x1[j] * r, ah[j]); }
          z0[j] = r * fmaf(-x0[j], m, z0[j] * gl[j]);
          z1[j] = r * fmaf(-x1[j], m, z1[j] * gh[j]);
        }
      }
      if (ok) {
        uint4 *o = reinterpret_cast<uint4 *>(dx + ((size_t)t * heads + h) * HD + 8 * sub);
        o[0] = pack8(z0, (const T *)nullptr);
        o[L] = pack8(z1, (const T *)nullptr);
      }
    }
    if (!gain) continue;
    // lanes sub, sub + L, ... of a warp, then the warps, in a fixed order
#pragma unroll
    for (int o = L; o < 32; o <<= 1)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        al[j] += __shfl_xor_sync(0xffffffffu, al[j], o);
        ah[j] += __shfl_xor_sync(0xffffffffu, ah[j], o);
      }
    __syncthreads();                 // (the previous tensor's sums have been read)
    if (lane < L) {
#pragma unroll
      for (int j = 0; j < 8; ++j) { red[warp][8 * sub + j] = al[j]; red[warp][half + 8 * sub + j] = ah[j]; }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < HD; i += RB_THREADS) {
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < RB_THREADS / 32; ++w) v += red[w][i];
      a.partial[((size_t)blockIdx.x * 2 + which) * HD + i] = v;
    }
  }
}

// general form: one warp per head
template <typename T>
__global__ void __launch_bounds__(RB_THREADS) qk_norm_rope_bwd_kernel(RopeBwdArgs a) {
  extern __shared__ float rb_red[];            // [warps][hd]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, half = a.hd >> 1;
  constexpr int WARPS = RB_THREADS / 32;
  for (int which = 0; which < 2; ++which) {
    const int heads = which ? a.n_kv : a.n_q;
    const T *gain = reinterpret_cast<const T *>(which ? a.k_gain : a.q_gain);
    const T *x = reinterpret_cast<const T *>(which ? a.k : a.q);
    const long long x_stride = which ? a.k_stride : a.q_stride;
    const T *dy = reinterpret_cast<const T *>(which ? a.dk : a.dq);
    T *dx = reinterpret_cast<T *>(which ? a.dk_in : a.dq_in);
    float a0[4] = {0.f, 0.f, 0.f, 0.f}, a1[4] = {0.f, 0.f, 0.f, 0.f};
    const long long n_units = (long long)a.tokens * heads;
    for (long long u = (long long)blockIdx.x * WARPS + warp; u < n_units; u += (long long)gridDim.x * WARPS) {
      const int t = (int)(u / heads), h = (int)(u - (long long)t * heads);
      int pos = a.positions[t];
      if (pos < 0 || pos >= a.max_pos) {
        if (lane == 0) atomicOr(a.status, STATUS_BAD_TOKEN);
        pos = pos < 0 ? 0 : a.max_pos - 1;
      }
      const T *xr = x + (size_t)t * x_stride + (size_t)h * a.hd, *dr = dy + ((size_t)t * heads + h) * a.hd;
      T *o = dx + ((size_t)t * heads + h) * a.hd;
      float z0[4], z1[4], x0[4], x1[4], ss = 0.f, dot = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = lane + 32 * j;
        z0[j] = z1[j] = x0[j] = x1[j] = 0.f;
        if (i < half) {
          const float c = a.cos_tab[(size_t)pos * half + i], s = a.sin_tab[(size_t)pos * half + i];
          const float d0 = to_f(dr[i]), d1 = to_f(dr[i + half]);
          z0[j] = d0 * c + d1 * s;
          z1[j] = d1 * c - d0 * s;
          if (gain) {
            x0[j] = to_f(xr[i]);
            x1[j] = to_f(xr[i + half]);
            ss = fmaf(x0[j], x0[j], fmaf(x1[j], x1[j], ss));
            dot = fmaf(z0[j] * to_f(gain[i]), x0[j], fmaf(z1[j] * to_f(gain[i + half]), x1[j], dot));
          }
        }
      }
      float r = 1.f, m = 0.f;
      if (gain) {
        r = rsqrtf(warp_sum(ss) / a.hd + a.eps);
        m = warp_sum(dot) * r * r / a.hd;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = lane + 32 * j;
        if (i >= half) continue;
        float y0 = z0[j], y1 = z1[j];
        if (gain) {
          a0[j] = fmaf(z0[j], x0[j] * r, a0[j]);
          a1[j] = fmaf(z1[j], x1[j] * r, a1[j]);
          y0 = r * fmaf(-x0[j], m, z0[j] * to_f(gain[i]));
          y1 = r * fmaf(-x1[j], m, z1[j] * to_f(gain[i + half]));
        }
        o[i] = round_to<T>(y0);
        o[i + half] = round_to<T>(y1);
      }
    }
    if (!gain) continue;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = lane + 32 * j;
      if (i < half) { rb_red[warp * a.hd + i] = a0[j]; rb_red[warp * a.hd + i + half] = a1[j]; }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.hd; i += RB_THREADS) {
      float v = 0.f;
      for (int w = 0; w < WARPS; ++w) v += rb_red[w * a.hd + i];
      a.partial[((size_t)blockIdx.x * 2 + which) * a.hd + i] = v;
    }
  }
}

// gain gradients: block (32 elements, q or k) adds the blocks' partial sums, eight rows of warps side by side, in a fixed order
__global__ void __launch_bounds__(256) gain_grad_kernel(const float *__restrict__ partial, int blocks, int hd, float *__restrict__ dq_gain,
                                                        float *__restrict__ dk_gain) {
  __shared__ float red[8][33];
  const int which = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
  float *dst = which ? dk_gain : dq_gain;
  if (!dst) return;
  float v = 0.f;
  if (i < hd)
#pragma unroll 8
    for (int b = warp; b < blocks; b += 8) v += partial[((size_t)b * 2 + which) * hd + i];
  red[warp][lane] = v;
  __syncthreads();
  if (warp == 0 && i < hd) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += red[w][lane];
    dst[i] = s;
  }
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <typename T>
cudaError_t launch_qk_rope(const RopeArgs &a, cudaStream_t st) {
  const bool fp8 = a.k_scale != nullptr;
  if constexpr (sizeof(T) == 2) {
    const bool vec = !fp8 && (a.hd == 64 || a.hd == 128 || a.hd == 256) && aligned16(a.q) && aligned16(a.k) && aligned16(a.v) && aligned16(a.q_out) &&
                     aligned16(a.k_out) && aligned16(a.v_out) && aligned16(a.q_gain) && aligned16(a.k_gain) && aligned16(a.cos_tab) &&
                     aligned16(a.sin_tab) && ((a.q_stride | a.k_stride | a.v_stride | a.qo_stride) & 7) == 0;
    if (vec) {
      const int lanes = a.hd / 16, units = a.n_q + 2 * a.n_kv;
      int threads = (units + 2) / 3 * lanes;               // three heads per thread
      threads = (threads + 31) / 32 * 32;
      if (threads > 512) threads = 512;
      if (a.hd == 64) qk_norm_rope_vec_kernel<T, 4, 3><<<a.tokens, threads, 0, st>>>(a);
      else if (a.hd == 128) qk_norm_rope_vec_kernel<T, 8, 3><<<a.tokens, threads, 0, st>>>(a);
      else qk_norm_rope_vec_kernel<T, 16, 3><<<a.tokens, threads, 0, st>>>(a);
      return cudaGetLastError();
    }
  }
  const size_t smem = fp8 ? (size_t)a.n_kv * a.hd * sizeof(float) : 0;
  qk_norm_rope_kernel<T><<<dim3(a.tokens, 3), RG_THREADS, smem, st>>>(a, ROLE_Q);
  return cudaGetLastError();
}

int bwd_blocks() { return num_sms() * RB_BLOCKS_PER_SM; }

template <typename T>
cudaError_t launch_qk_rope_bwd(const RopeBwdArgs &a, float *dq_gain, float *dk_gain, cudaStream_t st) {
  bool vec = false;
  const int lanes = a.hd / 16;
  if constexpr (sizeof(T) == 2) {
    vec = (a.hd == 64 || a.hd == 128 || a.hd == 256) && aligned16(a.q) && aligned16(a.k) && aligned16(a.dq) && aligned16(a.dk) && aligned16(a.dq_in) &&
          aligned16(a.dk_in) && aligned16(a.q_gain) && aligned16(a.k_gain) && aligned16(a.cos_tab) && aligned16(a.sin_tab) &&
          ((a.q_stride | a.k_stride) & 7) == 0;
  }
  const long long per_block = vec ? RB_THREADS / lanes : RB_THREADS / 32;
  const long long want = ((long long)a.tokens * a.n_q + per_block - 1) / per_block;
  const int blocks = (int)(want < bwd_blocks() ? want : bwd_blocks());
  if constexpr (sizeof(T) == 2) {
    if (vec) {
      if (a.hd == 64) qk_norm_rope_bwd_vec_kernel<T, 4><<<blocks, RB_THREADS, 0, st>>>(a);
      else if (a.hd == 128) qk_norm_rope_bwd_vec_kernel<T, 8><<<blocks, RB_THREADS, 0, st>>>(a);
      else qk_norm_rope_bwd_vec_kernel<T, 16><<<blocks, RB_THREADS, 0, st>>>(a);
    }
  }
  if (!vec) qk_norm_rope_bwd_kernel<T><<<blocks, RB_THREADS, (size_t)(RB_THREADS / 32) * a.hd * sizeof(float), st>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || (!dq_gain && !dk_gain)) return e;
  gain_grad_kernel<<<dim3((a.hd + 31) / 32, 2), 256, 0, st>>>(a.partial, blocks, a.hd, dq_gain, dk_gain);
  return cudaGetLastError();
}

bool dtype_ok(int32_t d) { return d == SWIFTKV_DTYPE_F32 || d == SWIFTKV_DTYPE_BF16 || d == SWIFTKV_DTYPE_F16; }
bool misaligned(const void *p, int32_t dtype) { return reinterpret_cast<uintptr_t>(p) % (dtype == SWIFTKV_DTYPE_F32 ? 4 : 2) != 0; }

}  // namespace
}  // namespace skv

using namespace skv;

extern "C" int32_t swiftkv_rope_table(float *cos_tab, float *sin_tab, int32_t max_pos, int32_t head_dim, double theta, void *cuda_stream) {
  if (!cos_tab || !sin_tab) return report_error(SWIFTKV_ERR_INVALID_ARG, "null argument");
  if (max_pos < 1 || head_dim < 2 || head_dim > 256 || head_dim % 2 || !(theta > 0.0))
    return report_error(SWIFTKV_ERR_INVALID_ARG, "bad shape (max_pos >= 1, even head_dim in [2, 256], theta > 0)");
  launch_rope_table(cos_tab, sin_tab, max_pos, head_dim, theta, reinterpret_cast<cudaStream_t>(cuda_stream));
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return report_error(SWIFTKV_ERR_CUDA, cudaGetErrorString(e));
  return SWIFTKV_OK;
}

extern "C" int32_t swiftkv_qk_norm_rope(const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                                        int32_t dtype, int32_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                        const void *q_gain, const void *k_gain, float eps, const int32_t *positions, const float *cos_tab,
                                        const float *sin_tab, int32_t max_pos, void *q_out, int64_t q_out_stride, void *k_cache,
                                        void *v_cache, float *k_scale, float *v_scale, int32_t cache_rows, const int32_t *slot_map,
                                        void *cuda_stream) {
  if (!q || !k || !v || !positions || !cos_tab || !sin_tab || !q_out || !k_cache || !v_cache) return report_error(SWIFTKV_ERR_INVALID_ARG, "null argument");
  if (n_tokens < 1 || n_q_heads < 1 || n_kv_heads < 1 || n_kv_heads > 1024 || n_q_heads > 1024 || head_dim < 2 || head_dim > 256 || head_dim % 2 ||
      max_pos < 1 || cache_rows < 1)
    return report_error(SWIFTKV_ERR_INVALID_ARG, "bad shape (even head_dim in [2, 256], at most 1024 heads)");
  const int64_t nq = (int64_t)n_q_heads * head_dim, nkv = (int64_t)n_kv_heads * head_dim;
  if (q_stride < nq || k_stride < nkv || v_stride < nkv || q_out_stride < nq) return report_error(SWIFTKV_ERR_INVALID_ARG, "a token stride is shorter than a token's heads");
  if (!dtype_ok(dtype)) return report_error(SWIFTKV_ERR_INVALID_ARG, "unknown dtype");
  if (!k_scale != !v_scale) return report_error(SWIFTKV_ERR_INVALID_ARG, "k_scale and v_scale must both be given (FP8 cache) or both be null");
  if (k_scale && nkv > 8192) return report_error(SWIFTKV_ERR_UNSUPPORTED, "an FP8 row holds at most 8192 values");
  if (!slot_map && cache_rows < n_tokens) return report_error(SWIFTKV_ERR_INVALID_ARG, "without a slot map the cache needs a row per token");
  if (!(eps >= 0.f)) return report_error(SWIFTKV_ERR_INVALID_ARG, "eps must not be negative");
  if (misaligned(q, dtype) || misaligned(k, dtype) || misaligned(v, dtype) || misaligned(q_out, dtype) || (!k_scale && (misaligned(k_cache, dtype) || misaligned(v_cache, dtype))))
    return report_error(SWIFTKV_ERR_INVALID_ARG, "misaligned pointer");
  unsigned int *status = op_status_word();
  if (!status) return report_error(SWIFTKV_ERR_CUDA, "no status word");
  RopeArgs a{q, k, v, q_stride, k_stride, v_stride, q_gain, k_gain, positions, cos_tab, sin_tab, slot_map, q_out, k_cache, v_cache, q_out_stride,
             k_scale, v_scale, n_tokens, n_q_heads, n_kv_heads, head_dim, max_pos, cache_rows, eps, status};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = dtype == SWIFTKV_DTYPE_F32 ? launch_qk_rope<float>(a, st) : dtype == SWIFTKV_DTYPE_BF16 ? launch_qk_rope<bf16>(a, st) : launch_qk_rope<__half>(a, st);
  if (e != cudaSuccess) return report_error(SWIFTKV_ERR_CUDA, cudaGetErrorString(e));
  return SWIFTKV_OK;
}

extern "C" size_t swiftkv_qk_norm_rope_bwd_scratch_bytes(int32_t head_dim) {
  if (head_dim < 2 || head_dim > 256) return 0;
  return (size_t)bwd_blocks() * 2 * head_dim * sizeof(float);
}

extern "C" int32_t swiftkv_qk_norm_rope_bwd(const void *dq, const void *dk, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                                            int32_t dtype, int32_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                            const void *q_gain, const void *k_gain, float eps, const int32_t *positions, const float *cos_tab,
                                            const float *sin_tab, int32_t max_pos, void *dq_in, void *dk_in, float *dq_gain, float *dk_gain,
                                            void *scratch, size_t scratch_bytes, void *cuda_stream) {
  if (!dq || !dk || !q || !k || !positions || !cos_tab || !sin_tab || !dq_in || !dk_in || (q_gain && !dq_gain) || (k_gain && !dk_gain) || !scratch)
    return report_error(SWIFTKV_ERR_INVALID_ARG, "null argument");
  if ((!q_gain && dq_gain) || (!k_gain && dk_gain)) return report_error(SWIFTKV_ERR_INVALID_ARG, "a gain gradient without its gain");
  if (n_tokens < 1 || n_q_heads < 1 || n_kv_heads < 1 || n_kv_heads > 1024 || n_q_heads > 1024 || head_dim < 2 || head_dim > 256 || head_dim % 2 || max_pos < 1)
    return report_error(SWIFTKV_ERR_INVALID_ARG, "bad shape (even head_dim in [2, 256], at most 1024 heads)");
  if (q_stride < (int64_t)n_q_heads * head_dim || k_stride < (int64_t)n_kv_heads * head_dim) return report_error(SWIFTKV_ERR_INVALID_ARG, "a token stride is shorter than a token's heads");
  if (!dtype_ok(dtype)) return report_error(SWIFTKV_ERR_INVALID_ARG, "unknown dtype");
  if (!(eps >= 0.f)) return report_error(SWIFTKV_ERR_INVALID_ARG, "eps must not be negative");
  if (misaligned(q, dtype) || misaligned(k, dtype) || misaligned(dq, dtype) || misaligned(dk, dtype) || misaligned(dq_in, dtype) || misaligned(dk_in, dtype) ||
      (reinterpret_cast<uintptr_t>(scratch) & 15))
    return report_error(SWIFTKV_ERR_INVALID_ARG, "misaligned pointer");
  if (scratch_bytes < swiftkv_qk_norm_rope_bwd_scratch_bytes(head_dim)) return report_error(SWIFTKV_ERR_WORKSPACE_SMALL, "scratch too small");
  unsigned int *status = op_status_word();
  if (!status) return report_error(SWIFTKV_ERR_CUDA, "no status word");
  RopeBwdArgs a{dq, dk, q, k, q_stride, k_stride, q_gain, k_gain, positions, cos_tab, sin_tab, dq_in, dk_in, reinterpret_cast<float *>(scratch),
                n_tokens, n_q_heads, n_kv_heads, head_dim, max_pos, eps, status};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = dtype == SWIFTKV_DTYPE_F32 ? launch_qk_rope_bwd<float>(a, dq_gain, dk_gain, st)
                        : dtype == SWIFTKV_DTYPE_BF16 ? launch_qk_rope_bwd<bf16>(a, dq_gain, dk_gain, st) : launch_qk_rope_bwd<__half>(a, dq_gain, dk_gain, st);
  if (e != cudaSuccess) return report_error(SWIFTKV_ERR_CUDA, cudaGetErrorString(e));
  return SWIFTKV_OK;
}
