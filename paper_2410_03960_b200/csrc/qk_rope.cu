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
// and 16 bytes of its upper half each, so a rotation pair sits in one thread and a head's mean needs log2(hd/16) shuffles; as
// many blocks as run at once walk over the (token, head) pairs, and what limits them is how many warps' registers fit beside
// the loads under way.  Other shapes, fp32 and unaligned tensors take the general form (one warp per head, a pair per lane
// and step).  Measured, 32 + 8 heads of 128, bf16: 16411 tokens 73 us (5.5 TB/s; torch's copy of as many bytes 64 us), 4096
// tokens into an FP8 cache 27 - 29 us; gradient of 8195 tokens 53 us (4.8 TB/s).
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

__device__ __forceinline__ int checked_position(int p, int max_pos, unsigned int *status, bool reports) {
  if (p >= 0 && p < max_pos) return p;
  if (reports) atomicOr(status, STATUS_BAD_TOKEN);
  return p < 0 ? 0 : max_pos - 1;
}
// cache row of a token whose slot is s, -1: not stored
__device__ __forceinline__ int checked_slot(const RopeArgs &a, int s, bool reports) {
  if (s < a.cache_rows) return s < 0 ? -1 : s;
  if (reports) atomicOr(a.status, STATUS_BAD_TOKEN);
  return -1;
}
__device__ __forceinline__ int slot_of(const RopeArgs &a, int t) { return a.slot_map ? a.slot_map[t] : t; }

__device__ __forceinline__ float block_max_all(float v, float *red, int warps) {
  v = warp_max(v);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  float m = red[0];
  for (int w = 1; w < warps; ++w) m = fmaxf(m, red[w]);
  return m;
}

// ---- two fp32 values per operation; eight of them from 16 bytes of a 16-bit type ---------------------------------------
using tc::F2;
using tc::add2;
using tc::fma2;
using tc::mul2;
__device__ __forceinline__ F2 both(float v) { return F2{{v, v}}; }
template <typename T>
__device__ __forceinline__ void unpack(const uint4 &v, F2 (&x)[4]) {
  float f[8];
  unpack8(v, f, (const T *)nullptr);
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = F2{{f[2 * i], f[2 * i + 1]}};
}
template <typename T>
__device__ __forceinline__ uint4 pack(const F2 (&x)[4]) {
  const float f[8] = {x[0].f[0], x[0].f[1], x[1].f[0], x[1].f[1], x[2].f[0], x[2].f[1], x[3].f[0], x[3].f[1]};
  return pack8(f, (const T *)nullptr);
}
__device__ __forceinline__ void load8(const float *p, F2 (&x)[4]) {
  const float4 a = __ldg(reinterpret_cast<const float4 *>(p)), b = __ldg(reinterpret_cast<const float4 *>(p) + 1);
  x[0] = F2{{a.x, a.y}}; x[1] = F2{{a.z, a.w}}; x[2] = F2{{b.x, b.y}}; x[3] = F2{{b.z, b.w}};
}
template <int L>
__device__ __forceinline__ float sum_lanes(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ uint2 codes8(const F2 (&x)[4], float scale) {
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i / 4] |= (uint32_t)code_of(x[i / 2].f[i & 1], scale) << (8 * (i & 3));
  return make_uint2(w[0], w[1]);
}
// (token, head) pairs in order, `groups` of them per step of a block and `blocks` blocks side by side
struct Walk {
  int steps, groups, heads, t_step, h_step;                 // steps of this block: the same for all its threads
  long long first;
  __device__ __forceinline__ Walk(long long pairs, int block, int blocks, int groups_, int heads_) : groups(groups_), heads(heads_) {
    const long long step = (long long)blocks * groups;
    first = (long long)block * groups;
    steps = first < pairs ? (int)((pairs - first + step - 1) / step) : 0;
    t_step = (int)(step / heads);
    h_step = (int)(step % heads);
  }
  __device__ __forceinline__ void start(int group, int &t, int &h) const {
    t = (int)((first + group) / heads);
    h = (int)((first + group) % heads);
  }
  __device__ __forceinline__ void advance(int &t, int &h) const {
    t += t_step;
    h += h_step;
    if (h >= heads) { h -= heads; ++t; }
  }
};

// a head's 16 values of this thread -> normed (norm; g: gains of the lower / upper half) and rotated (plain: left as they are)
template <int L>
__device__ __forceinline__ void norm_rotate(F2 (&lo)[4], F2 (&hi)[4], bool norm, bool plain, const F2 (&gl)[4], const F2 (&gh)[4], const F2 (&c)[4],
                                            const F2 (&s)[4], float eps) {
  float r = 1.f;
  if (norm) {
    F2 ss = mul2(lo[0], lo[0]);
#pragma unroll
    for (int i = 1; i < 4; ++i) ss = fma2(lo[i], lo[i], ss);
#pragma unroll
    for (int i = 0; i < 4; ++i) ss = fma2(hi[i], hi[i], ss);
    r = rsqrtf(sum_lanes<L>(ss.f[0] + ss.f[1]) * (1.f / (16 * L)) + eps);
  }
  if (plain) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    F2 a = lo[i], b = hi[i];
    if (norm) { a = mul2(mul2(a, gl[i]), both(r)); b = mul2(mul2(b, gh[i]), both(r)); }
    const F2 bs = mul2(b, s[i]), as = mul2(a, s[i]);
    lo[i] = fma2(a, c[i], F2{{-bs.f[0], -bs.f[1]}});
    hi[i] = fma2(b, c[i], as);
  }
}

// ---- forward, vector form: L lanes per head -----------------------------------------------------------------------------
// Threads of a block and blocks per SM: registers for one step of loads under way beside one at work, 8 bytes of them spilled (16411 tokens
// of the 8B shape: 73 us; 3 x 256 threads 76, 2 x 256 89, 4 x 256 with a few spilled 79, gains read again from L1 82).  FP8 rows
// take larger blocks: a row's maximum is taken over one block.
__host__ __device__ constexpr int rv_threads(bool fp8) { return fp8 ? 256 : 128; }
__host__ __device__ constexpr int rv_blocks_per_sm(bool fp8) { return fp8 ? 3 : 7; }
// The first q_blocks blocks walk over the (token, query head) pairs, the next k_blocks over the key heads, the rest over the value
// heads, as many blocks as run at once and the next pair's loads under way while one is computed.
// FP8: the rest are rows of keys and values, RV_THREADS / row_lanes of them a block, a row's heads side by side in registers.
template <typename T, int L, bool FP8>
__global__ void __launch_bounds__(rv_threads(FP8), rv_blocks_per_sm(FP8)) qk_norm_rope_vec_kernel(RopeArgs a, int q_blocks, int k_blocks, int row_lanes) {
  constexpr int RV_THREADS = rv_threads(FP8);
  constexpr int half = 8 * L, HD = 16 * L, GROUPS = RV_THREADS / L;
  const int sub = threadIdx.x % L, unit0 = threadIdx.x / L;
  if (FP8 && (int)blockIdx.x >= q_blocks) {
    __shared__ float red[RV_THREADS / 32];
    const int lane = threadIdx.x % row_lanes, h = lane / L;
    const long long row = (long long)(blockIdx.x - q_blocks) * (RV_THREADS / row_lanes) + threadIdx.x / row_lanes;
    const int t = (int)(row >> 1);
    const bool is_v = row & 1, have = t < a.tokens && h < a.n_kv;
    F2 x[4], y[4];
    int slot = -1;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = y[i] = both(0.f);
    F2 c[4], s[4], gl[4], gh[4];
    const T *gain = reinterpret_cast<const T *>(is_v ? nullptr : a.k_gain);
#pragma unroll
    for (int i = 0; i < 4; ++i) { c[i] = gl[i] = gh[i] = both(1.f); s[i] = both(0.f); }
    if (have) {
      const T *src = is_v ? reinterpret_cast<const T *>(a.v) + (size_t)t * a.v_stride : reinterpret_cast<const T *>(a.k) + (size_t)t * a.k_stride;
      const uint4 *p = reinterpret_cast<const uint4 *>(src + (size_t)h * HD + 8 * sub);
      const uint4 lo = __ldcs(p), hi = __ldcs(p + L);
      const int pos = checked_position(a.positions[t], a.max_pos, a.status, lane == 0);
      slot = checked_slot(a, slot_of(a, t), lane == 0);
      if (!is_v) {
        load8(a.cos_tab + (size_t)pos * half + 8 * sub, c);
        load8(a.sin_tab + (size_t)pos * half + 8 * sub, s);
        if (gain) {
          unpack<T>(__ldg(reinterpret_cast<const uint4 *>(gain + 8 * sub)), gl);
          unpack<T>(__ldg(reinterpret_cast<const uint4 *>(gain + half + 8 * sub)), gh);
        }
      }
      unpack<T>(lo, x);
      unpack<T>(hi, y);
    }
    norm_rotate<L>(x, y, gain != nullptr, is_v, gl, gh, c, s, a.eps);       // (every lane walks its shuffles)
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) amax = fmaxf(fmaxf(fmaxf(fabsf(x[i].f[0]), fabsf(x[i].f[1])), fmaxf(fabsf(y[i].f[0]), fabsf(y[i].f[1]))), amax);
    for (int o = (row_lanes < 32 ? row_lanes : 32) / 2; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    if (row_lanes > 32) {
      if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = amax;
      __syncthreads();
      for (int w = 0; w < row_lanes / 32; ++w) amax = fmaxf(amax, red[threadIdx.x / row_lanes * (row_lanes / 32) + w]);
    }
    if (slot < 0) return;
    const float scale = row_scale(amax);
    if (lane == 0) (is_v ? a.v_scale : a.k_scale)[slot] = scale;
    uint8_t *d = reinterpret_cast<uint8_t *>(is_v ? a.v_out : a.k_out) + ((size_t)slot * a.n_kv + h) * HD + 8 * sub;
    *reinterpret_cast<uint2 *>(d) = codes8(x, scale);
    *reinterpret_cast<uint2 *>(d + half) = codes8(y, scale);
    return;
  }
  const int role = (int)blockIdx.x < q_blocks ? ROLE_Q : (int)blockIdx.x < q_blocks + k_blocks ? ROLE_K : ROLE_V;
  const int first = role == ROLE_Q ? 0 : role == ROLE_K ? q_blocks : q_blocks + k_blocks;
  const int blocks = role == ROLE_Q ? q_blocks : role == ROLE_K ? k_blocks : (int)gridDim.x - first;
  const int heads = role == ROLE_Q ? a.n_q : a.n_kv;
  const T *src = reinterpret_cast<const T *>(role == ROLE_Q ? a.q : role == ROLE_K ? a.k : a.v);
  const long long stride = role == ROLE_Q ? a.q_stride : role == ROLE_K ? a.k_stride : a.v_stride;
  const long long out_stride = role == ROLE_Q ? a.qo_stride : (long long)a.n_kv * HD;
  T *dst = reinterpret_cast<T *>(role == ROLE_Q ? a.q_out : role == ROLE_K ? a.k_out : a.v_out);
  const T *gain = reinterpret_cast<const T *>(role == ROLE_Q ? a.q_gain : role == ROLE_K ? a.k_gain : nullptr);
  uint4 gain_lo = make_uint4(0u, 0u, 0u, 0u), gain_hi = gain_lo;
  if (gain) {
    gain_lo = __ldg(reinterpret_cast<const uint4 *>(gain + 8 * sub));
    gain_hi = __ldg(reinterpret_cast<const uint4 *>(gain + half + 8 * sub));
  }
  const Walk walk((long long)a.tokens * heads, blockIdx.x - first, blocks, GROUPS, heads);
  int t, h;
  walk.start(unit0, t, h);
  struct Unit { uint4 lo, hi; int pos, row; };               // row: of the output, -1 none
  auto fetch = [&](Unit &n) {
    n.lo = n.hi = make_uint4(0u, 0u, 0u, 0u);
    n.pos = 0;
    n.row = -1;
    if (t >= a.tokens) return;
    const uint4 *p = reinterpret_cast<const uint4 *>(src + (size_t)t * stride + h * HD + 8 * sub);
    n.lo = __ldcs(p);
    n.hi = __ldcs(p + L);
    n.row = role == ROLE_Q ? t : slot_of(a, t);
    if (role != ROLE_V) n.pos = a.positions[t];
  };
  Unit next;
  fetch(next);
  for (int left = walk.steps; left > 0; --left) {
    const Unit now = next;
    const int at = h * HD + 8 * sub;
    walk.advance(t, h);
    fetch(next);
    const int row = role == ROLE_Q ? now.row : checked_slot(a, now.row, sub == 0);
    uint4 lo = now.lo, hi = now.hi;
    if (role != ROLE_V) {
      const int pos = checked_position(now.pos, a.max_pos, a.status, sub == 0);
      F2 c[4], s[4], x[4], y[4], gl[4], gh[4];
      load8(a.cos_tab + (size_t)pos * half + 8 * sub, c);
      load8(a.sin_tab + (size_t)pos * half + 8 * sub, s);
      unpack<T>(lo, x);
      unpack<T>(hi, y);
      unpack<T>(gain_lo, gl);
      unpack<T>(gain_hi, gh);
      norm_rotate<L>(x, y, gain != nullptr, false, gl, gh, c, s, a.eps);
      lo = pack<T>(x);
      hi = pack<T>(y);
    }
    if (row < 0) continue;
    uint4 *d = reinterpret_cast<uint4 *>(dst + (size_t)row * out_stride + at);
    __stcs(d, lo);
    __stcs(d + L, hi);
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
  const int pos = checked_position(a.positions[t], a.max_pos, a.status, threadIdx.x == 0);
  const int slot = role == ROLE_Q ? 0 : checked_slot(a, slot_of(a, t), threadIdx.x == 0);
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
  float *partial;                            // [blocks][hd] gain gradients of each block
  int tokens, n_q, n_kv, hd, max_pos;
  float eps;
  unsigned int *status;
};
constexpr int RB_THREADS = 256;
constexpr int RB_BLOCKS_PER_SM = 2;      // as many of the vector form as run at once
// vector form: L lanes per head; the first q_blocks blocks walk over the (token, query head) pairs, the rest over the key heads, the next
// pair's loads under way while one is computed; gain gradients stay in registers.  These hold it to 16 warps per SM, of 285 instructions
// a pair and step: 53 us for 8195 tokens of the 8B shape (half as many elements per thread and 24 warps 59, loads by asynchronous
// copies and two to four steps ahead 59, four times as many blocks 69).
template <typename T, int L>
__global__ void __launch_bounds__(RB_THREADS, RB_BLOCKS_PER_SM) qk_norm_rope_bwd_vec_kernel(RopeBwdArgs a, int q_blocks) {
  constexpr int half = 8 * L, HD = 16 * L, GROUPS = RB_THREADS / L;
  __shared__ float red[RB_THREADS / 32][HD];
  const int sub = threadIdx.x % L, unit0 = threadIdx.x / L;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int which = (int)blockIdx.x >= q_blocks, first = which ? q_blocks : 0;
  const int heads = which ? a.n_kv : a.n_q;
  const T *gain = reinterpret_cast<const T *>(which ? a.k_gain : a.q_gain);
  const T *x = reinterpret_cast<const T *>(which ? a.k : a.q);
  const long long x_stride = which ? a.k_stride : a.q_stride;
  const T *dy = reinterpret_cast<const T *>(which ? a.dk : a.dq);
  T *dx = reinterpret_cast<T *>(which ? a.dk_in : a.dq_in);
  F2 al[4], ah[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) al[j] = ah[j] = both(0.f);
  uint4 gain_lo = make_uint4(0u, 0u, 0u, 0u), gain_hi = gain_lo;
  if (gain) {
    gain_lo = __ldg(reinterpret_cast<const uint4 *>(gain + 8 * sub));
    gain_hi = __ldg(reinterpret_cast<const uint4 *>(gain + half + 8 * sub));
  }
  const Walk walk((long long)a.tokens * heads, blockIdx.x - first, which ? gridDim.x - q_blocks : q_blocks, GROUPS, heads);
  int t, h;                               // (whole warps stay together for the shuffles)
  walk.start(unit0, t, h);
  struct Unit { uint4 d0, d1, v0, v1; int pos; };
  auto fetch = [&](Unit &n) {
    n.d0 = n.d1 = n.v0 = n.v1 = make_uint4(0u, 0u, 0u, 0u);
    n.pos = 0;
    if (t >= a.tokens) return;
    const uint4 *p = reinterpret_cast<const uint4 *>(dy + ((size_t)t * heads + h) * HD + 8 * sub);
    n.d0 = __ldcs(p);
    n.d1 = __ldcs(p + L);
    if (gain) {
      const uint4 *xp = reinterpret_cast<const uint4 *>(x + (size_t)t * x_stride + h * HD + 8 * sub);
      n.v0 = __ldcs(xp);
      n.v1 = __ldcs(xp + L);
    }
    n.pos = a.positions[t];
  };
  Unit next;
  fetch(next);
  for (int left = walk.steps; left > 0; --left) {
    const Unit now = next;
    const bool ok = t < a.tokens;
    uint4 *o = reinterpret_cast<uint4 *>(dx + ((size_t)t * heads + h) * HD + 8 * sub);
    walk.advance(t, h);
    fetch(next);
    const int pos = checked_position(now.pos, a.max_pos, a.status, sub == 0);
    F2 c[4], s[4], z0[4], z1[4];
    load8(a.cos_tab + (size_t)pos * half + 8 * sub, c);
    load8(a.sin_tab + (size_t)pos * half + 8 * sub, s);
    unpack<T>(now.d0, z0);
    unpack<T>(now.d1, z1);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const F2 s1 = mul2(z1[j], s[j]), s0 = mul2(z0[j], s[j]);
      z0[j] = fma2(z0[j], c[j], s1);
      z1[j] = fma2(z1[j], c[j], F2{{-s0.f[0], -s0.f[1]}});
    }
    if (gain) {
      F2 x0[4], x1[4], gl[4], gh[4], ss = both(0.f), dot = both(0.f);
      unpack<T>(gain_lo, gl);
      unpack<T>(gain_hi, gh);
      unpack<T>(now.v0, x0);
      unpack<T>(now.v1, x1);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        ss = fma2(x0[j], x0[j], ss);
        ss = fma2(x1[j], x1[j], ss);
        dot = fma2(mul2(z0[j], gl[j]), x0[j], dot);
        dot = fma2(mul2(z1[j], gh[j]), x1[j], dot);
      }
      const float r = rsqrtf(sum_lanes<L>(ss.f[0] + ss.f[1]) * (1.f / HD) + a.eps);
      const float m = -sum_lanes<L>(dot.f[0] + dot.f[1]) * r * r * (1.f / HD);          // -mean(dz g xh) r, to be multiplied by x
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        al[j] = fma2(z0[j], mul2(x0[j], both(r)), al[j]);              // (a pair that is not there adds zeros)
        ah[j] = fma2(z1[j], mul2(x1[j], both(r)), ah[j]);
        z0[j] = mul2(both(r), fma2(x0[j], both(m), mul2(z0[j], gl[j])));
        z1[j] = mul2(both(r), fma2(x1[j], both(m), mul2(z1[j], gh[j])));
      }
    }
    if (ok) {
      __stcs(o, pack<T>(z0));
      __stcs(o + L, pack<T>(z1));
    }
  }
  if (!gain) return;
  // lanes sub, sub + L, ... of a warp, then the warps, in a fixed order
#pragma unroll
  for (int o = L; o < 32; o <<= 1)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        al[j].f[q] += __shfl_xor_sync(0xffffffffu, al[j].f[q], o);
        ah[j].f[q] += __shfl_xor_sync(0xffffffffu, ah[j].f[q], o);
      }
  if (lane < L) {
#pragma unroll
    for (int j = 0; j < 8; ++j) { red[warp][8 * sub + j] = al[j / 2].f[j & 1]; red[warp][half + 8 * sub + j] = ah[j / 2].f[j & 1]; }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < HD; i += RB_THREADS) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < RB_THREADS / 32; ++w) v += red[w][i];
    a.partial[(size_t)blockIdx.x * HD + i] = v;
  }
}

// general form: one warp per head
template <typename T>
__global__ void __launch_bounds__(RB_THREADS) qk_norm_rope_bwd_kernel(RopeBwdArgs a, int q_blocks) {
  extern __shared__ float rb_red[];            // [warps][hd]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, half = a.hd >> 1;
  constexpr int WARPS = RB_THREADS / 32;
  const int which = (int)blockIdx.x >= q_blocks, first = which ? q_blocks : 0, blocks = which ? gridDim.x - q_blocks : q_blocks;
  const int heads = which ? a.n_kv : a.n_q;
  const T *gain = reinterpret_cast<const T *>(which ? a.k_gain : a.q_gain);
  const T *x = reinterpret_cast<const T *>(which ? a.k : a.q);
  const long long x_stride = which ? a.k_stride : a.q_stride;
  const T *dy = reinterpret_cast<const T *>(which ? a.dk : a.dq);
  T *dx = reinterpret_cast<T *>(which ? a.dk_in : a.dq_in);
  float a0[4] = {0.f, 0.f, 0.f, 0.f}, a1[4] = {0.f, 0.f, 0.f, 0.f};
  const long long n_units = (long long)a.tokens * heads;
  for (long long u = (long long)(blockIdx.x - first) * WARPS + warp; u < n_units; u += (long long)blocks * WARPS) {
    const int t = (int)(u / heads), h = (int)(u - (long long)t * heads);
    const int pos = checked_position(a.positions[t], a.max_pos, a.status, lane == 0);
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
  if (!gain) return;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i = lane + 32 * j;
    if (i < half) { rb_red[warp * a.hd + i] = a0[j]; rb_red[warp * a.hd + i + half] = a1[j]; }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.hd; i += RB_THREADS) {
    float v = 0.f;
    for (int w = 0; w < WARPS; ++w) v += rb_red[w * a.hd + i];
    a.partial[(size_t)blockIdx.x * a.hd + i] = v;
  }
}

// gain gradients: block (32 elements, q or k) adds the blocks' partial sums, 32 rows of warps side by side, in a fixed order (one row of
// eight warps took 7 us for 296 blocks, most of it waiting)
constexpr int GG_WARPS = 32;
__global__ void __launch_bounds__(32 * GG_WARPS) gain_grad_kernel(const float *partial, int q_blocks, int blocks, int hd,
                                                                 float *__restrict__ dq_gain, float *__restrict__ dk_gain) {
  __shared__ float red[GG_WARPS][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
  float *dst = blockIdx.y ? dk_gain : dq_gain;
  wait_for_previous();
  if (!dst) return;
  const int end = blockIdx.y ? blocks : q_blocks;
  float v = 0.f;
  if (i < hd)
#pragma unroll 8
    for (int b = (blockIdx.y ? q_blocks : 0) + warp; b < end; b += GG_WARPS) v += partial[(size_t)b * hd + i];
  red[warp][lane] = v;
  __syncthreads();
  if (warp == 0 && i < hd) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < GG_WARPS; ++w) s += red[w][lane];
    dst[i] = s;
  }
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <typename T>
cudaError_t launch_qk_rope(const RopeArgs &a, cudaStream_t st) {
  const bool fp8 = a.k_scale != nullptr;
  if constexpr (sizeof(T) == 2) {
    const int lanes = a.hd / 16;
    bool vec = (a.hd == 64 || a.hd == 128 || a.hd == 256) && aligned16(a.q) && aligned16(a.k) && aligned16(a.v) && aligned16(a.q_out) &&
               aligned16(a.k_out) && aligned16(a.v_out) && aligned16(a.q_gain) && aligned16(a.k_gain) && aligned16(a.cos_tab) &&
               aligned16(a.sin_tab) && ((a.q_stride | a.k_stride | a.v_stride | a.qo_stride) & 7) == 0;
    int row_lanes = lanes;
    while (row_lanes < a.n_kv * lanes) row_lanes *= 2;
    const int threads = rv_threads(fp8);
    vec = vec && !(fp8 && row_lanes > threads);                // (an FP8 row's maximum is taken over one block's registers)
    if (vec) {
      const int groups = threads / lanes, all = num_sms() * rv_blocks_per_sm(fp8), heads = a.n_q + 2 * a.n_kv;
      auto share = [&](int n) {                                // blocks for n heads a token
        const long long want = ((long long)a.tokens * n + groups - 1) / groups, most = (long long)all * n / heads;
        return (int)(want < most ? want : most > 0 ? most : 1);
      };
      const int qb = share(a.n_q), kb = fp8 ? 0 : share(a.n_kv), per = threads / row_lanes;
      const long long rest = fp8 ? (2ll * a.tokens + per - 1) / per : share(a.n_kv);
      const unsigned grid = (unsigned)(qb + kb + rest);
#define SKV_ROPE_VEC(LANES)                                                                                \
  (fp8 ? qk_norm_rope_vec_kernel<T, LANES, true><<<grid, threads, 0, st>>>(a, qb, kb, row_lanes)        \
       : qk_norm_rope_vec_kernel<T, LANES, false><<<grid, threads, 0, st>>>(a, qb, kb, row_lanes))
      if (a.hd == 64) SKV_ROPE_VEC(4);
      else if (a.hd == 128) SKV_ROPE_VEC(8);
      else SKV_ROPE_VEC(16);
#undef SKV_ROPE_VEC
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
  if constexpr (sizeof(T) == 2) {
    vec = (a.hd == 64 || a.hd == 128 || a.hd == 256) && aligned16(a.q) && aligned16(a.k) && aligned16(a.dq) && aligned16(a.dk) && aligned16(a.dq_in) &&
          aligned16(a.dk_in) && aligned16(a.q_gain) && aligned16(a.k_gain) && aligned16(a.cos_tab) && aligned16(a.sin_tab) &&
          ((a.q_stride | a.k_stride) & 7) == 0;
  }
  const int per_block = vec ? RB_THREADS / (a.hd / 16) : RB_THREADS / 32;
  auto share = [&](int n) {                                  // blocks for n heads a token
    const long long want = ((long long)a.tokens * n + per_block - 1) / per_block, most = (long long)bwd_blocks() * n / (a.n_q + a.n_kv);
    return (int)(want < most ? want : most > 0 ? most : 1);
  };
  const int qb = share(a.n_q), blocks = qb + share(a.n_kv);
  if constexpr (sizeof(T) == 2) {
    if (vec) {
      if (a.hd == 64) qk_norm_rope_bwd_vec_kernel<T, 4><<<blocks, RB_THREADS, 0, st>>>(a, qb);
      else if (a.hd == 128) qk_norm_rope_bwd_vec_kernel<T, 8><<<blocks, RB_THREADS, 0, st>>>(a, qb);
      else qk_norm_rope_bwd_vec_kernel<T, 16><<<blocks, RB_THREADS, 0, st>>>(a, qb);
    }
  }
  if (!vec) qk_norm_rope_bwd_kernel<T><<<blocks, RB_THREADS, (size_t)(RB_THREADS / 32) * a.hd * sizeof(float), st>>>(a, qb);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || (!dq_gain && !dk_gain)) return e;
  return launch_early(gain_grad_kernel, dim3((a.hd + 31) / 32, 2), 32 * GG_WARPS, st, a.partial, qb, blocks, a.hd, dq_gain, dk_gain);
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
  // in place a head is read by the threads that write it; any other overlap is not
  const size_t es = dtype == SWIFTKV_DTYPE_F32 ? 4 : 2, T = (size_t)n_tokens;
  const ByteRows rq{q, T, q_stride * es, nq * es}, rk{k, T, k_stride * es, nkv * es}, rv{v, T, v_stride * es, nkv * es}, ro{q_out, T, q_out_stride * es, nq * es};
  const size_t plane = (size_t)cache_rows * nkv * (k_scale ? 1 : es);
  const ByteRows ck{k_cache, 1, plane, plane}, cv{v_cache, 1, plane, plane};
  auto rows_in_place = [&](const void *cache, const void *x, int64_t stride) { return cache == x && !slot_map && !k_scale && (stride == nkv || n_tokens == 1); };
  if ((overlap(ro, rq) && !(q_out == q && (q_out_stride == q_stride || n_tokens == 1))) || overlap(ro, rk) || overlap(ro, rv) || overlap(ro, ck) || overlap(ro, cv) ||
      overlap(ck, cv) || overlap(ck, rq) || overlap(cv, rq) || overlap(ck, rv) || overlap(cv, rk) || (overlap(ck, rk) && !rows_in_place(k_cache, k, k_stride)) ||
      (overlap(cv, rv) && !rows_in_place(v_cache, v, v_stride)))
    return report_error(SWIFTKV_ERR_INVALID_ARG, "an output overlaps an input other than in place, or another output");
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
  return (size_t)(bwd_blocks() + 1) * head_dim * sizeof(float);      // (at least one block each for queries and keys)
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
  // in place a head is read by the threads that write it; any other overlap is not
  const size_t es = dtype == SWIFTKV_DTYPE_F32 ? 4 : 2, T = (size_t)n_tokens;
  const int64_t nq = (int64_t)n_q_heads * head_dim, nkv = (int64_t)n_kv_heads * head_dim;
  const ByteRows rq{q, T, q_stride * es, nq * es}, rk{k, T, k_stride * es, nkv * es}, dyq{dq, T, nq * es, nq * es}, dyk{dk, T, nkv * es, nkv * es},
      oq{dq_in, T, nq * es, nq * es}, ok{dk_in, T, nkv * es, nkv * es};
  if ((overlap(oq, dyq) && dq_in != dq) || (overlap(oq, rq) && !(dq_in == q && (q_stride == nq || n_tokens == 1))) || overlap(oq, dyk) || overlap(oq, rk) ||
      (overlap(ok, dyk) && dk_in != dk) || (overlap(ok, rk) && !(dk_in == k && (k_stride == nkv || n_tokens == 1))) || overlap(ok, dyq) || overlap(ok, rq) || overlap(oq, ok))
    return report_error(SWIFTKV_ERR_INVALID_ARG, "an output overlaps an input other than in place, or another output");
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
