// swiftkv_tree_attention: several new tokens per sequence (drafted tokens, a prompt chunk, or one decode token) against the
// sequence's cache rows, contiguous or paged, in the model's type or FP8.
//
// Sequence b has past_b committed tokens (positions 0 .. past_b - 1) and new_b new ones, whose K / V rows already sit in the
// cache at positions past_b .. past_b + new_b - 1.  New token i sees every committed token and the new tokens j that its
// mask row names (bit j; null: j <= i):
//   o_i = sum_j p_ij v_j,  p = softmax_j(scale q_i k_j),  lse_i = log sum_j exp(scale q_i k_j);  a token that sees nothing: o = 0, lse = -inf.
#include <math.h>

#include "common.cuh"
#include "tc_common.cuh"

namespace skv {
namespace {

struct TreeArgs {
  const void *q;
  long long q_stride;            // elements between tokens
  const void *k, *v;             // [cache_rows][n_kv][hd]
  const float *k_scale, *v_scale;
  const int32_t *blk;
  int max_blocks;
  const int32_t *row0, *past, *cu, *mask;
  int mask_words;
  void *out;                     // [T][n_q][hd]
  float *lse;                    // [T][n_q] or null
  float *scratch;
  int cache_rows, n_seqs, total_new, max_new, max_kv, n_q, n_kv, hd;
  float scale;
  unsigned int *status;
};

// lengths beyond what the host promised (max_new, max_kv, total_new) are cut, so that no loop outgrows them, and reported
__device__ __forceinline__ void tree_lengths(const TreeArgs &a, int b, int &tok0, int &n, int &past) {
  const int c0 = a.cu[b], c1 = a.cu[b + 1], p = a.past[b];
  tok0 = min(max(0, c0), a.total_new);
  n = min(min(min(max(0, c1 - c0), a.max_new), a.total_new - tok0), a.max_kv);
  past = min(max(0, p), a.max_kv - n);
  if ((n != c1 - c0 || past != p) && threadIdx.x == 0) atomicOr(a.status, STATUS_BAD_TOKEN);
}
// cache row of key p, -1 where the tables lead outside the cache (such a row reads as zeros)
__device__ __forceinline__ int tree_row(const TreeArgs &a, int b, int p) {
  long long row;
  if (a.blk) {
    const int j = p >> 7;
    if (j >= a.max_blocks) return -1;
    row = (long long)a.blk[(size_t)b * a.max_blocks + j] * PAGE_ROWS + (p & (PAGE_ROWS - 1));
  } else {
    row = (long long)a.row0[b] + p;
  }
  return row >= 0 && row < a.cache_rows ? (int)row : -1;
}
// whether new token i (index t among all) sees key p
__device__ __forceinline__ bool tree_sees(const TreeArgs &a, int t, int i, int past, int n, int p) {
  if (p < past) return true;
  const int j = p - past;
  if (j >= n) return false;
  if (!a.mask) return j <= i;
  const int w = j >> 5;
  return w < a.mask_words && ((a.mask[(size_t)t * a.mask_words + w] >> (j & 31)) & 1);
}
template <typename T> __device__ __forceinline__ T tree_round(float v);
template <> __device__ __forceinline__ float tree_round<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 tree_round<bf16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half tree_round<__half>(float v) { return __float2half_rn(v); }

// ---------------------------------------------------------------------------------------------------------
// General form (any head_dim up to 256, fp32 too) on the CUDA cores: block (sequence, KV head, 8 query rows, key split).
// A query row is a (new token, query head of the group) pair; the rows of a block share its K and V tiles of 32 keys, kept
// as fp32 in shared memory.  Scores: a lane per key, a warp per row; output: a thread per element, all rows.
// ---------------------------------------------------------------------------------------------------------
constexpr int TS_THREADS = 128, TS_ROWS = 8, TS_KEYS = 32, TS_SPLIT_KEYS = 1024, TS_MAX_SPLITS = 32;

int simt_splits(int max_kv) {
  const int s = (max_kv + TS_SPLIT_KEYS - 1) / TS_SPLIT_KEYS;
  return s < 1 ? 1 : s > TS_MAX_SPLITS ? TS_MAX_SPLITS : s;
}

template <typename TQ, typename TKV>
__global__ void __launch_bounds__(TS_THREADS) tree_attention_simt_kernel(TreeArgs a, int row_chunks, int splits) {
  extern __shared__ float ts_smem[];
  const int hd = a.hd, rep = a.n_q / a.n_kv;
  float *qs = ts_smem;                                   // [TS_ROWS][hd]
  float *ks = qs + TS_ROWS * hd;                         // [TS_KEYS][hd + 1]
  float *vs = ks + TS_KEYS * (hd + 1);                   // [TS_KEYS][hd]
  __shared__ float ps[TS_ROWS][TS_KEYS];                 // probabilities; -1: not seen
  __shared__ float corr[TS_ROWS], row_m[TS_ROWS], row_l[TS_ROWS];
  int u = blockIdx.x;
  const int split = u % splits; u /= splits;
  const int chunk = u % row_chunks; u /= row_chunks;
  const int kvh = u % a.n_kv, b = u / a.n_kv;
  int tok0, n, past;
  tree_lengths(a, b, tok0, n, past);
  const int rows = n * rep, r0 = chunk * TS_ROWS, kv = past + n;
  if (r0 >= rows) return;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // keys of this split: whole tiles, the same number for every split
  const int tiles = (kv + TS_KEYS - 1) / TS_KEYS, per = (tiles + splits - 1) / splits;
  const int k_begin = split * per * TS_KEYS, k_end = min(kv, k_begin + per * TS_KEYS);
  for (int i = tid; i < TS_ROWS * hd; i += TS_THREADS) {
    const int r = r0 + i / hd;
    float x = 0.f;
    if (r < rows) x = to_f(reinterpret_cast<const TQ *>(a.q)[(size_t)(tok0 + r / rep) * a.q_stride + (size_t)(kvh * rep + r % rep) * hd + i % hd]) * a.scale;
    qs[i] = x;
  }
  if (tid < TS_ROWS) { row_m[tid] = -INFINITY; row_l[tid] = 0.f; }
  float acc[TS_ROWS][2];
#pragma unroll
  for (int r = 0; r < TS_ROWS; ++r) acc[r][0] = acc[r][1] = 0.f;
  for (int c0 = k_begin; c0 < k_end; c0 += TS_KEYS) {
    __syncthreads();
    for (int i = warp; i < TS_KEYS; i += TS_THREADS / 32) {
      const int p = c0 + i, row = p < k_end ? tree_row(a, b, p) : -1;
      const size_t at = ((size_t)(row < 0 ? 0 : row) * a.n_kv + kvh) * hd;
      const float sk = a.k_scale && row >= 0 ? a.k_scale[row] : 1.f, sv = a.v_scale && row >= 0 ? a.v_scale[row] : 1.f;
      for (int d = lane; d < hd; d += 32) {
        ks[i * (hd + 1) + d] = row < 0 ? 0.f : to_f(reinterpret_cast<const TKV *>(a.k)[at + d]) * sk;
        vs[i * hd + d] = row < 0 ? 0.f : to_f(reinterpret_cast<const TKV *>(a.v)[at + d]) * sv;
      }
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < TS_ROWS / 4; ++h) {
      const int r = warp + 4 * h, row = r0 + r, p = c0 + lane;
      const bool sees = row < rows && p < k_end && tree_sees(a, tok0 + row / rep, row / rep, past, n, p);
      float s = 0.f;
      for (int d = 0; d < hd; ++d) s = fmaf(qs[r * hd + d], ks[lane * (hd + 1) + d], s);
      const float m_old = row_m[r], mx = warp_max(sees ? s : -INFINITY);
      const float m = fmaxf(m_old, mx), m_ref = m == -INFINITY ? 0.f : m;
      const float pr = sees ? __expf(s - m_ref) : 0.f;
      const float sum = warp_sum(pr);
      ps[r][lane] = sees ? pr : -1.f;
      __syncwarp();
      if (lane == 0) {
        const float f = m_old == -INFINITY ? 0.f : __expf(m_old - m_ref);
        corr[r] = f;
        row_m[r] = m;
        row_l[r] = row_l[r] * f + sum;
      }
      __syncwarp();
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int d = tid + j * TS_THREADS;
      if (d >= hd) break;
#pragma unroll
      for (int r = 0; r < TS_ROWS; ++r) acc[r][j] *= corr[r];
      const int keys = min(TS_KEYS, k_end - c0);
      for (int i = 0; i < keys; ++i) {
        const float v = vs[i * hd + d];
#pragma unroll
        for (int r = 0; r < TS_ROWS; ++r) {
          const float pr = ps[r][i];
          if (pr >= 0.f || pr != pr) acc[r][j] = fmaf(pr, v, acc[r][j]);      // (an unseen key's V may hold anything)
        }
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < TS_ROWS; ++r) {
    const int row = r0 + r;
    if (row >= rows) break;
    const size_t head = (size_t)(tok0 + row / rep) * a.n_q + kvh * rep + row % rep;
    const float l = row_l[r];
    if (splits == 1) {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      for (int j = 0, d = tid; d < hd; d += TS_THREADS, ++j) reinterpret_cast<TQ *>(a.out)[head * hd + d] = tree_round<TQ>(l == 0.f ? 0.f : acc[r][j] * inv);
      if (a.lse && tid == 0) a.lse[head] = l == 0.f ? -INFINITY : row_m[r] + logf(l);
    } else {
      float *dst = a.scratch + (head * splits + split) * (hd + 2);
      if (tid == 0) { dst[0] = row_m[r]; dst[1] = l; }
      for (int j = 0, d = tid; d < hd; d += TS_THREADS, ++j) dst[2 + d] = acc[r][j];
    }
  }
}

// joins the splits of one (token, query head): block per pair
template <typename TQ>
__global__ void __launch_bounds__(TS_THREADS) tree_attention_join_kernel(TreeArgs a, int splits) {
  const int t = blockIdx.x / a.n_q;
  if (t < a.cu[0] || t >= a.cu[a.n_seqs]) return;              // rows behind the last sequence stay as they were
  const size_t head = blockIdx.x;
  const float *src = a.scratch + head * splits * (a.hd + 2);
  float M = -INFINITY, L = 0.f;
  for (int s = 0; s < splits; ++s) M = fmaxf(M, src[(size_t)s * (a.hd + 2)]);
  float acc[2] = {0.f, 0.f};
  for (int s = 0; s < splits; ++s) {
    const float *p = src + (size_t)s * (a.hd + 2);
    const float l = p[1];
    if (l == 0.f) continue;
    const float f = __expf(p[0] - M);
    L = fmaf(l, f, L);
    for (int j = 0, d = threadIdx.x; d < a.hd; d += TS_THREADS, ++j) acc[j] = fmaf(p[2 + d], f, acc[j]);
  }
  for (int j = 0, d = threadIdx.x; d < a.hd; d += TS_THREADS, ++j) reinterpret_cast<TQ *>(a.out)[head * a.hd + d] = tree_round<TQ>(L == 0.f ? 0.f : acc[j] / L);
  if (a.lse && threadIdx.x == 0) a.lse[head] = L == 0.f ? -INFINITY : M + logf(L);
}

template <typename TQ, typename TKV>
int32_t launch_simt(const TreeArgs &a, int max_kv, cudaStream_t st) {
  const int splits = simt_splits(max_kv), rep = a.n_q / a.n_kv;
  const int row_chunks = (a.max_new * rep + TS_ROWS - 1) / TS_ROWS;
  const long long grid = (long long)a.n_seqs * a.n_kv * row_chunks * splits;
  if (grid > 0x7fffffffLL || (long long)a.total_new * a.n_q > 0x7fffffffLL) return report_error(SWIFTKV_ERR_UNSUPPORTED, "too many query rows for one launch");
  const size_t smem = ((size_t)TS_ROWS * a.hd + (size_t)TS_KEYS * (2 * a.hd + 1)) * sizeof(float);
  if (smem > 40 * 1024 && ensure_dynamic_smem(reinterpret_cast<const void *>(tree_attention_simt_kernel<TQ, TKV>), 80 * 1024))
    return report_error(SWIFTKV_ERR_CUDA, "shared memory");
  tree_attention_simt_kernel<TQ, TKV><<<(unsigned)grid, TS_THREADS, smem, st>>>(a, row_chunks, splits);
  cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess && splits > 1) {
    tree_attention_join_kernel<TQ><<<(unsigned)(a.total_new * a.n_q), TS_THREADS, 0, st>>>(a, splits);
    e = cudaGetLastError();
  }
  return e == cudaSuccess ? SWIFTKV_OK : report_error(SWIFTKV_ERR_CUDA, cudaGetErrorString(e));
}

size_t simt_scratch(int total_new, int max_kv, int n_q, int hd) {
  const int splits = simt_splits(max_kv);
  return splits > 1 ? (size_t)total_new * n_q * splits * (hd + 2) * sizeof(float) : 0;
}

}  // namespace
}  // namespace skv

using namespace skv;

extern "C" size_t swiftkv_tree_attention_scratch_bytes(int32_t total_new, int32_t max_kv, int32_t n_q_heads, int32_t head_dim) {
  if (total_new < 1 || max_kv < 1 || n_q_heads < 1 || head_dim < 1 || head_dim > 256) return 0;
  return simt_scratch(total_new, max_kv, n_q_heads, head_dim);
}

extern "C" int32_t swiftkv_tree_attention(const void *q, int64_t q_stride, int32_t q_dtype, const void *k_cache, const void *v_cache,
                                          int32_t kv_dtype, const float *k_scale, const float *v_scale, int32_t cache_rows,
                                          const int32_t *block_table, int32_t max_blocks, const int32_t *row0, const int32_t *n_past,
                                          const int32_t *cu_new, const int32_t *tree_mask, int32_t mask_words, void *out, float *lse,
                                          int32_t n_seqs, int32_t total_new, int32_t max_new, int32_t max_kv, int32_t n_q_heads,
                                          int32_t n_kv_heads, int32_t head_dim, float softmax_scale, void *scratch, size_t scratch_bytes,
                                          void *cuda_stream) {
  if (!q || !k_cache || !v_cache || !n_past || !cu_new || !out) return report_error(SWIFTKV_ERR_INVALID_ARG, "null argument");
  if (!block_table == !row0) return report_error(SWIFTKV_ERR_INVALID_ARG, "exactly one of block_table and row0 must be given");
  if (n_seqs < 1 || total_new < 1 || max_new < 1 || max_kv < 1 || n_q_heads < 1 || n_kv_heads < 1 || n_q_heads % n_kv_heads || head_dim < 2 ||
      head_dim > 256 || cache_rows < 1 || (block_table && max_blocks < 1) || (tree_mask && mask_words < 1))
    return report_error(SWIFTKV_ERR_INVALID_ARG, "bad shape (head_dim in [2, 256], n_q_heads a multiple of n_kv_heads)");
  if (q_stride < (int64_t)n_q_heads * head_dim) return report_error(SWIFTKV_ERR_INVALID_ARG, "q_stride is shorter than a token's heads");
  const bool fp8 = kv_dtype == SWIFTKV_DTYPE_FP8_E4M3;
  const bool q_ok = q_dtype == SWIFTKV_DTYPE_F32 || q_dtype == SWIFTKV_DTYPE_BF16 || q_dtype == SWIFTKV_DTYPE_F16;
  if (!q_ok || (!fp8 && kv_dtype != q_dtype)) return report_error(SWIFTKV_ERR_INVALID_ARG, "q must be fp32, bf16 or f16 and the cache of the same type or FP8");
  if (fp8 ? (!k_scale || !v_scale) : (k_scale || v_scale)) return report_error(SWIFTKV_ERR_INVALID_ARG, "row scales go with an FP8 cache, and with it alone");
  if (!(softmax_scale >= 0.f) || !(softmax_scale < INFINITY)) return report_error(SWIFTKV_ERR_INVALID_ARG, "softmax_scale must be finite and not negative");
  const uintptr_t es = q_dtype == SWIFTKV_DTYPE_F32 ? 4 : 2, kes = fp8 ? 1 : es;
  if ((uintptr_t)q % es || (uintptr_t)out % es || (uintptr_t)k_cache % kes || (uintptr_t)v_cache % kes || ((uintptr_t)scratch & 15))
    return report_error(SWIFTKV_ERR_INVALID_ARG, "misaligned pointer");
  const size_t need = swiftkv_tree_attention_scratch_bytes(total_new, max_kv, n_q_heads, head_dim);
  if (need && (!scratch || scratch_bytes < need)) return report_error(SWIFTKV_ERR_WORKSPACE_SMALL, "scratch too small (see swiftkv_tree_attention_scratch_bytes)");
  unsigned int *status = op_status_word();
  if (!status) return report_error(SWIFTKV_ERR_CUDA, "no status word");
  TreeArgs a{};
  a.q = q; a.q_stride = q_stride; a.k = k_cache; a.v = v_cache; a.k_scale = k_scale; a.v_scale = v_scale;
  a.blk = block_table; a.max_blocks = max_blocks; a.row0 = row0; a.past = n_past; a.cu = cu_new; a.mask = tree_mask; a.mask_words = mask_words;
  a.out = out; a.lse = lse; a.scratch = reinterpret_cast<float *>(scratch);
  a.cache_rows = cache_rows; a.n_seqs = n_seqs; a.total_new = total_new; a.max_new = max_new; a.max_kv = max_kv; a.n_q = n_q_heads; a.n_kv = n_kv_heads; a.hd = head_dim;
  a.scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)head_dim);
  a.status = status;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (fp8) {
    if (q_dtype == SWIFTKV_DTYPE_F32) return launch_simt<float, fp8e4>(a, max_kv, st);
    if (q_dtype == SWIFTKV_DTYPE_BF16) return launch_simt<bf16, fp8e4>(a, max_kv, st);
    return launch_simt<__half, fp8e4>(a, max_kv, st);
  }
  if (q_dtype == SWIFTKV_DTYPE_F32) return launch_simt<float, float>(a, max_kv, st);
  if (q_dtype == SWIFTKV_DTYPE_BF16) return launch_simt<bf16, bf16>(a, max_kv, st);
  return launch_simt<__half, __half>(a, max_kv, st);
}
