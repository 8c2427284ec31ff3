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

constexpr int TREE_MAX_KV = 1 << 30;      // a longer sequence is cut there

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
__device__ __forceinline__ void tree_lengths(const TreeArgs &a, int b, int &tok0, int &n, int &past, bool report) {
  const int c0 = a.cu[b], c1 = a.cu[b + 1], p = a.past[b];
  tok0 = min(max(0, c0), a.total_new);
  n = min(min(min(max(0, c1 - c0), a.max_new), a.total_new - tok0), a.max_kv);
  past = min(max(0, p), a.max_kv - n);
  if (report && (n != c1 - c0 || past != p)) atomicOr(a.status, STATUS_BAD_TOKEN);
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
// At most so many partial rows: 16384 blocks, 110 for each SM, and 68 MB of scratch at head_dim 128.  More query rows than that fill the GPU
// without splitting the keys.
constexpr long long TS_PARTS = 131072;

long long simt_splits_by_keys(int max_kv) {
  const long long s = ((long long)max_kv + TS_SPLIT_KEYS - 1) / TS_SPLIT_KEYS;
  return s < TS_MAX_SPLITS ? s : TS_MAX_SPLITS;
}
int simt_splits(int total_new, int max_kv, int n_q) {
  const long long by_keys = simt_splits_by_keys(max_kv), by_rows = TS_PARTS / ((long long)total_new * n_q);
  return (int)(by_rows < 1 ? 1 : by_keys < by_rows ? by_keys : by_rows);
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
  tree_lengths(a, b, tok0, n, past, threadIdx.x == 0);
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
  int inside = 0;
  for (int b = threadIdx.x; b < a.n_seqs; b += TS_THREADS) {
    int tok0, n, past;
    tree_lengths(a, b, tok0, n, past, false);
    inside |= t >= tok0 && t < tok0 + n;
  }
  if (!__syncthreads_or(inside)) return;                       // rows of no sequence, and those cut off one, stay as they were
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
int32_t launch_simt(const TreeArgs &a, cudaStream_t st) {
  const int splits = simt_splits(a.total_new, a.max_kv, a.n_q), rep = a.n_q / a.n_kv;
  const long long chunks = ((long long)a.max_new * rep + TS_ROWS - 1) / TS_ROWS;
  const double blocks = (double)a.n_seqs * a.n_kv * chunks * splits;        // (the products pass 64 bits for the largest arguments)
  if (blocks > 0x7fffffff || (double)a.total_new * a.n_q > 0x7fffffff) return report_error(SWIFTKV_ERR_UNSUPPORTED, "too many query rows for one launch");
  const int row_chunks = (int)chunks;
  const size_t smem = ((size_t)TS_ROWS * a.hd + (size_t)TS_KEYS * (2 * a.hd + 1)) * sizeof(float);
  if (smem > 40 * 1024 && ensure_dynamic_smem(reinterpret_cast<const void *>(tree_attention_simt_kernel<TQ, TKV>), 80 * 1024))
    return report_error(SWIFTKV_ERR_CUDA, "shared memory");
  tree_attention_simt_kernel<TQ, TKV><<<(unsigned)blocks, TS_THREADS, smem, st>>>(a, row_chunks, splits);
  cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess && splits > 1) {
    tree_attention_join_kernel<TQ><<<(unsigned)(a.total_new * a.n_q), TS_THREADS, 0, st>>>(a, splits);
    e = cudaGetLastError();
  }
  return e == cudaSuccess ? SWIFTKV_OK : report_error(SWIFTKV_ERR_CUDA, cudaGetErrorString(e));
}

// (enough for fewer rows and keys as well: these have at most as many partial rows)
size_t simt_scratch(int total_new, int max_kv, int n_q, int hd) {
  const long long by_keys = simt_splits_by_keys(max_kv), parts = (long long)total_new * n_q * by_keys;
  return by_keys > 1 ? (size_t)(parts < TS_PARTS ? parts : TS_PARTS) * (hd + 2) * sizeof(float) : 0;
}

// ---------------------------------------------------------------------------------------------------------
// Tensor-core form (head_dim 64 / 128, 16-bit queries, cache of their type or FP8).
//
// A query tile is 128 rows = (128 / rep new tokens) x (the rep query heads of one KV head), so that a K / V tile of 128 keys
// -- exactly one page -- is read once for all of them.  tcgen05: S = Q K^T into tensor memory, a row per softmax thread,
// P back over S in 16 bits, O += P V with P read from tensor memory (P bf16; f16 with f16 caches).  Two streams of softmax
// warps keep the tensor pipe and the loads busy while the other one exponentiates:
//   W = 2: stream w owns query tile w of a pair, both use every K / V tile (up to 256 rows a pass over the cache);
//   W = 1: stream w owns the key tiles of parity w of ONE query tile, and the two accumulators are joined at the end.
// Sums and maxima are fp32; the reference maximum moves only when a row outgrows it by 2^8 (O is then rescaled).
//
// Work split: the (sequence, tile group, KV head, key tile) units of a call, in this order, are cut into equal contiguous
// ranges, one per CTA (one CTA per SM).  The lengths live on the device, so every CTA sums them up for itself.  A range that
// starts or ends inside a (sequence, group, head) leaves an unnormalised partial result in `scratch` (at most two per CTA),
// and a second kernel joins those in the order of the keys: deterministic, and balanced for any mix of lengths.  Where the
// longest sequence has two groups, the CTAs form two classes, one per group, that walk over the same keys in step, so that
// the second one finds them in L2 (of a sequence with one group each class takes every other head).
//
// FP8 rows: TMA brings the codes and four warps widen them to IEEE half, exactly (every e4m3 number is one).  Queries in bf16
// become halves too, each row times a power of two that brings its maximum to 2^14 .. 2^15: what that loses (elements below 2^-38 of the
// maximum) is below the accumulation's own rounding.  K scales multiply the scores; V scales enter P, whose reference
// exponent follows the largest scale-weighted probability of the row, so that P keeps the full half precision.  The two scales make
// the softmax the longest step of a tile, and its time is a thread's: one row of 128 columns.  So a tile of at most 64 (32) rows is laid
// out 2 (4) times along M, which the MMA does for nothing; each copy's softmax warps do their share of the tile's columns and
// leave zeros for the others, and the copies are joined like the pieces of a split key range (in the CTA, through shared memory: 222 us instead of
// 151 for 24 sequences of 10000 keys).
//
// What bounds it: HBM for 16-bit caches and up to about 64 query rows per KV head (24 sequences of one token over 10000 keys 159 us,
// 0.96 of the copy bandwidth; 16 of 9 to 32 tokens over 2048 to 8192 keys 70 us, 4.3 TB/s); each stream's chain of softmax, P V and next
// Q K^T for two full tiles (2 x 64 tokens, 8 heads per KV head, over 131072 keys 450 - 520 us, 1.0 - 1.2 PFLOP/s); shared memory for FP8
// caches (24 sequences of up to 8 tokens over up to 10000 keys 130 us, 2.8 TB/s); latency for few keys (1 token over 700 keys 11.7 us).
// These repeat a call; with the L2 cache emptied between calls: 77, 545, 143 and 12.3 us for the last four.
// The layouts go by max_new, not by the lengths, which the host does not know: the FP8 case takes 160 us with max_new 16 and 217 with 64.
//
// What is not seen must not matter: keys behind the sequence and unseen drafts get S = -inf, and the V rows of the last
// tiles are cleaned in shared memory first (0 * NaN is NaN): rows behind the sequence become zeros, and so do infinities and NaN in a
// drafted token's V row, which the epilogue hands to the rows that do see them.
// ---------------------------------------------------------------------------------------------------------
constexpr int TT_KEYS = 128;
constexpr float TT_RESCALE = 8.0f;       // in log2 units
// FP8: how far a small V scale (0 for a row outside the cache) draws the reference below the scores.  A key adds at most 2^(80 + TT_RESCALE) to the
// sum, so 2^30 of them stay below 2^127; rows quantized from zeros (2^-64 / 448) lie above.  (Below 2^-94, where the format has no scale, P
// falls under the half's normal range; and beside a row of scale 0 what has less than about 2^-100 of its probability adds nothing.)
constexpr float TT_LEAST_LOG2 = -80.f;

template <int HD, int W, bool FP8>
struct TreeLayout {
  static constexpr int TILE = 128 * HD * 2, CHUNK = 128 * 128, CHUNKS = HD / 64;
  static constexpr int CODE_TILE = 128 * HD;
  static constexpr int KS = FP8 ? 1 : (HD == 64 ? 4 : 2), VS = FP8 ? 2 : (HD == 64 ? 4 : (W == 2 ? 2 : 3)), CS = FP8 ? 5 : 1;
  static constexpr int Q = 0, K = W * TILE, V = K + KS * TILE, C = V + VS * TILE, SC = C + (FP8 ? CS * CODE_TILE : 0);
  static constexpr int ML = SC + (FP8 ? (4 * 3 + 2) * 128 * 4 : 0); // scales: 4 tiles x (K, V, log2 V) x 128; query rows' powers of two x 2
  static constexpr int BAR = ML + 2 * 2 * 128 * 8;                  // (m, l) of both streams, two items
  static constexpr int BYTES = BAR + 512 + 1024;
  // copies, MMA, [FP8: row scales, none,] softmax of two streams, [widening]; FP8: whole warpgroups, for their register shares
  static constexpr int SOFT = FP8 ? 4 : 2, WARPS = FP8 ? 16 : 10;
  static constexpr int THREADS = WARPS * 32;
};

struct TreeTcArgs {
  TreeArgs a;
  int npt;               // new tokens per query tile
  int copies;            // FP8: how often a query tile of few rows is laid out, see below
  int slot_rows;         // rows of a partial result in scratch
  int classes;           // 1 or 2 classes of CTAs
  float *part_o;         // [slot][slot_rows][HD] unnormalised outputs; (m, l) pairs [slot][slot_rows] at a.scratch
  float scale_log2;
  int store32;
};

__device__ __forceinline__ bool tt_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag, unsigned int *status) {
  if (tc::mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  for (unsigned spins = 1;; ++spins) {
    if (tc::mbar_try_wait(bar, parity)) return true;
    if ((spins & 31u) == 0u) {
      if (*abort_flag) return false;
      if (clock64() - t0 > tc::WAIT_LIMIT_CLOCKS) {
        *abort_flag = 1;
        atomicOr(status, STATUS_TIMEOUT);
        return false;
      }
    }
  }
}
// natural logarithm of l 2^m: with an FP8 cache m and the logarithm of l may be large and cancel
__device__ __forceinline__ float tt_lse(float m, float l, bool fp8) {
  if (!fp8 || !(l >= 1.1754944e-38f && l < INFINITY)) return m * 0.6931471805599453f + logf(l);
  const int bits = __float_as_int(l), e = (bits >> 23) - 127;
  return (m + (float)e + log2f(__int_as_float((bits & 0x7fffff) | 0x3f800000))) * 0.6931471805599453f;
}
__device__ __forceinline__ float tt_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// What a class of CTAs does of a sequence: all key tiles x `heads` KV heads, every h_step-th from h0 on, x `groups` groups of W query tiles
// from group g0 on.  Of two classes each takes one of two groups; of a sequence with one group, every other head.
struct SeqShape { int tok0, n, past, tiles, g0, groups, h0, h_step, heads; };
struct Split { int group_tokens, classes, cls; };
__device__ __forceinline__ SeqShape seq_shape(const TreeArgs &a, int b, const Split &sp) {
  SeqShape s;
  tree_lengths(a, b, s.tok0, s.n, s.past, false);
  s.tiles = (s.past + s.n + TT_KEYS - 1) / TT_KEYS;
  s.groups = (s.n + sp.group_tokens - 1) / sp.group_tokens;
  s.g0 = s.h0 = 0;
  s.h_step = 1;
  s.heads = a.n_kv;
  if (sp.classes == 2 && s.groups == 2) {
    s.g0 = sp.cls;
    s.groups = 1;
  } else if (sp.classes == 2) {
    s.h0 = (sp.cls + b) & 1;
    s.h_step = 2;
    s.heads = (a.n_kv + 1 - s.h0) / 2;
  }
  return s;
}
__device__ __forceinline__ int units_of(const SeqShape &s) { return s.tiles * s.groups * s.heads; }
// a CTA's walk over its units, one (sequence, group, head) piece after the other; every role keeps its own
struct Pieces {
  int b, gi, g, h, kt0, kt1, left;
  Split sp;
  SeqShape s;
  __device__ __forceinline__ void begin(const TreeArgs &a, int b0, int within, int units, const Split &split) {
    sp = split;
    b = b0;
    s = seq_shape(a, b, sp);
    left = units;
    const int item = within / s.tiles;
    kt0 = within % s.tiles;
    h = s.h0 + item % s.heads * s.h_step;
    gi = item / s.heads;
    g = s.g0 + gi;
    kt1 = min(s.tiles, kt0 + left);
  }
  __device__ __forceinline__ bool next(const TreeArgs &a) {
    left -= kt1 - kt0;
    if (left <= 0) return false;
    if ((h += s.h_step) >= a.n_kv) {
      if (++gi >= s.groups) {
        gi = 0;
        do { s = seq_shape(a, ++b, sp); } while (units_of(s) == 0);
      }
      h = s.h0;
      g = s.g0 + gi;
    }
    kt0 = 0;
    kt1 = min(s.tiles, kt0 + left);
    return true;
  }
  __device__ __forceinline__ bool whole() const { return kt0 == 0 && kt1 == s.tiles; }
};

// 32 visibility bits of keys j0 .. j0 + 31, counted from the first new token (negative: committed), for new token i
__device__ __forceinline__ uint32_t mask_word(const TreeArgs &a, int t, int i, int n, int w) {
  const int first = 32 * w;
  if (first >= n) return 0u;
  uint32_t m;
  if (a.mask) m = w < a.mask_words ? (uint32_t)a.mask[(size_t)t * a.mask_words + w] : 0u;
  else m = i >= first + 31 ? 0xffffffffu : i < first ? 0u : (2u << (i - first)) - 1u;
  return n - first >= 32 ? m : m & ((1u << (n - first)) - 1u);
}
__device__ __forceinline__ uint32_t sees_word(const TreeArgs &a, int t, int i, int n, int j0) {
  if (j0 <= -32) return 0xffffffffu;
  if (j0 < 0) return (mask_word(a, t, i, n, 0) << -j0) | ((1u << -j0) - 1u);
  const uint32_t lo = mask_word(a, t, i, n, j0 >> 5);
  return (j0 & 31) ? __funnelshift_r(lo, mask_word(a, t, i, n, (j0 >> 5) + 1), j0 & 31) : lo;
}

// four e4m3 codes as IEEE halves, exactly
__device__ __forceinline__ void widen4(uint32_t codes, uint32_t &lo, uint32_t &hi) {
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"((uint16_t)codes));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"((uint16_t)(codes >> 16)));
}

// Where key tile j starts, in two steps, so that nothing waits for the block table before it must: what the table (or row0) says ...
__device__ __forceinline__ int tile_entry(const TreeArgs &a, int b, int j) {
  return !a.blk ? a.row0[b] : j < a.max_blocks ? a.blk[(size_t)b * a.max_blocks + j] : -1;
}
// ... and the first cache row (outside the cache: it reads as zeros)
__device__ __forceinline__ int tile_row(const TreeArgs &a, int entry, int j) {
  if (a.blk) return entry < 0 || entry > a.cache_rows / PAGE_ROWS ? a.cache_rows : entry * PAGE_ROWS;
  const long long r = (long long)entry + (long long)j * TT_KEYS;
  return r < -TT_KEYS || r > a.cache_rows ? a.cache_rows : (int)r;
}

template <int HD, int W, bool F16, bool FP8>
__global__ void __launch_bounds__(TreeLayout<HD, W, FP8>::THREADS, 1)
tree_attention_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                         const __grid_constant__ TreeTcArgs p) {
  using L = TreeLayout<HD, W, FP8>;
  constexpr bool MMA_F16 = F16 || FP8;          // type of the operands: FP8 rows are widened to halves, bf16 queries converted
  const TreeArgs &a = p.a;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = smem_raw + (-tc::smem_u32(smem_raw) & 1023u);        // (an offset, so that accesses stay known as shared-memory ones)
  uint64_t *bars = reinterpret_cast<uint64_t *>(smem + L::BAR);
  uint64_t *q_full = bars, *o_full = bars + 2, *o_empty = bars + 3, *x_full = bars + 4;
  uint64_t *s_full = bars + 5, *s_half = bars + 7;                               // [2] each: all of S, its first 64 keys
  uint64_t *k_full = bars + 9, *k_empty = k_full + 4, *v_full = k_empty + 4, *v_empty = v_full + 4;      // rings of up to 4
  uint64_t *c_full = v_empty + 4, *c_empty = c_full + 5;                         // rings of up to 5 (FP8 codes)
  uint64_t *q_ready = c_empty + 5, *p_part = q_ready + 1;                        // queries as halves (FP8); [half of the keys][stream] P
  uint64_t *g_full = p_part + 4, *g_empty = g_full + 4, *q_scaled = g_empty + 4; // [4] row scales of a tile, [2] powers of two of the query rows (FP8)
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(q_scaled + 2);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
  volatile int *bad_item = reinterpret_cast<volatile int *>(tmem_slot + 2);      // [2]
  int *start = reinterpret_cast<int *>(tmem_slot + 4);                           // first sequence, units before the range in it
  int *issued = start + 2;                                                       // giving up: K, V (FP8: codes), query tiles that were requested
  uint64_t *drained = reinterpret_cast<uint64_t *>(tmem_slot + 10);
  float2 *ml = reinterpret_cast<float2 *>(smem + L::ML);                         // [item & 1][stream][128]
  float *scales = reinterpret_cast<float *>(smem + L::SC);                       // [tile & 3][K, V, log2 V][128], then [item & 1][128]

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rep = a.n_q / a.n_kv;
  const Split split{W * p.npt, p.classes, p.classes == 2 ? (int)blockIdx.x & 1 : 0};
  const int cta = (int)blockIdx.x / p.classes, ctas = ((int)gridDim.x - split.cls + p.classes - 1) / p.classes;      // within the class

  // ---- this CTA's range of units: prefix sums over the sequences (in the ring's memory, not yet in use)
  int *warp_sum_s = reinterpret_cast<int *>(smem);
  const int per_thread = (a.n_seqs + L::THREADS - 1) / L::THREADS;
  const int b_lo = min(a.n_seqs, (int)threadIdx.x * per_thread), b_hi = min(a.n_seqs, b_lo + per_thread);
  int mine = 0;
  for (int b = b_lo; b < b_hi; ++b) {
    if (blockIdx.x == 0) { int x, y, z; tree_lengths(a, b, x, y, z, true); }
    mine += units_of(seq_shape(a, b, split));
  }
  int inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += x;
  }
  if (lane == 31) warp_sum_s[warp] = inc;
  __syncthreads();
  int before = inc - mine, total = 0;
  for (int w = 0; w < L::WARPS; ++w) {
    if (w < warp) before += warp_sum_s[w];
    total += warp_sum_s[w];
  }
  launch_dependents();
  const int per = (total + ctas - 1) / ctas;
  const int u0 = (int)min((long long)total, (long long)cta * per), units = min(total - u0, per);
  if (units <= 0) return;
  if (u0 >= before && u0 < before + mine) {
    int at = before;
    for (int b = b_lo; b < b_hi; ++b) {
      const int n = units_of(seq_shape(a, b, split));
      if (u0 < at + n) { start[0] = b; start[1] = u0 - at; break; }
      at += n;
    }
  }

  if (threadIdx.x == 0) {
    tc::mbar_init(tc::smem_u32(q_full), 1);
    tc::mbar_init(tc::smem_u32(o_full), 1);
    tc::mbar_init(tc::smem_u32(o_empty), 8);
    tc::mbar_init(tc::smem_u32(x_full), 8);
    for (int s = 0; s < 2; ++s) {
      tc::mbar_init(tc::smem_u32(&s_full[s]), 1);
      tc::mbar_init(tc::smem_u32(&p_part[s]), 4);
      tc::mbar_init(tc::smem_u32(&p_part[2 + s]), 4);
      tc::mbar_init(tc::smem_u32(&s_half[s]), 1);
    }
    tc::mbar_init(tc::smem_u32(q_ready), 4);
    tc::mbar_init(tc::smem_u32(drained), 1);
    tc::mbar_init(tc::smem_u32(&q_scaled[0]), 4);
    tc::mbar_init(tc::smem_u32(&q_scaled[1]), 4);
    for (int s = 0; s < 4; ++s) {
      tc::mbar_init(tc::smem_u32(&k_full[s]), FP8 ? 4 : 1);
      tc::mbar_init(tc::smem_u32(&k_empty[s]), 1);
      tc::mbar_init(tc::smem_u32(&v_full[s]), FP8 ? 4 : 1);
      tc::mbar_init(tc::smem_u32(&v_empty[s]), 1);
      tc::mbar_init(tc::smem_u32(&g_full[s]), 1);
      tc::mbar_init(tc::smem_u32(&g_empty[s]), 4);
    }
    for (int s = 0; s < 5; ++s) {
      tc::mbar_init(tc::smem_u32(&c_full[s]), 1);
      tc::mbar_init(tc::smem_u32(&c_empty[s]), 4);
    }
    *abort_flag = 0;
    bad_item[0] = bad_item[1] = 0;
    tc::fence_barrier_init();
    tc::tma_prefetch_desc(&tmQ);
    tc::tma_prefetch_desc(&tmK);
    tc::tma_prefetch_desc(&tmV);
  }
  if (warp == 1) tc::tmem_alloc(tc::smem_u32(tmem_slot), 512);
  tc::tc_fence_before_sync();
  __syncthreads();
  tc::tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  // tensor-memory columns: S0 [0, 128) S1 [128, 256) O0 [256, 256 + HD) O1 [384, 384 + HD); P_w over the first 64 of S_w
  Pieces it;
  it.begin(a, start[0], start[1], units, split);
  auto wait = [&](uint64_t *bar, uint32_t parity) { return tt_wait(tc::smem_u32(bar), parity, abort_flag, a.status); };

  // FP8: 16 warps at 128 registers; what the copying and widening warps leave goes to the softmax warps (72 + 88 + 2 x 176 = 4 x 128)
  if (warp < L::SOFT) {
    if constexpr (FP8) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 0) {
      if (lane == 0) {
        // ------------------------------------------------------------------ K / V tiles (FP8: their codes, K and V in turn)
        int kc = 0, vc = 0, cc = 0;
        bool ok = true;
        int entry = tile_entry(a, it.b, it.kt0);
        do {
          for (int j = it.kt0; j < it.kt1 && ok; ++j) {
            const int now = tile_row(a, entry, j);
            if (j + 1 < it.kt1) entry = tile_entry(a, it.b, j + 1);      // (the table's answer travels while this tile waits)
            if constexpr (FP8) {
              for (int kv = 0; kv < 2 && ok; ++kv, ++cc) {
                const int s = cc % L::CS;
                ok = wait(&c_empty[s], ((cc / L::CS) & 1) ^ 1);
                if (!ok) break;
                const uint32_t bar = tc::smem_u32(&c_full[s]);
                tc::mbar_expect_tx(bar, L::CODE_TILE);
                tc::tma_load_2d(tc::smem_u32(smem + L::C + s * L::CODE_TILE), kv ? &tmV : &tmK, bar, it.h * (HD / 2), now);
              }
            } else {
              int s = kc % L::KS;
              ok = wait(&k_empty[s], ((kc / L::KS) & 1) ^ 1);
              if (!ok) break;
              uint32_t bar = tc::smem_u32(&k_full[s]);
              tc::mbar_expect_tx(bar, L::TILE);
              for (int c = 0; c < L::CHUNKS; ++c)
                tc::tma_load_2d(tc::smem_u32(smem + L::K + s * L::TILE + c * L::CHUNK), &tmK, bar, it.h * HD + c * 64, now);
              ++kc;
              s = vc % L::VS;
              ok = wait(&v_empty[s], ((vc / L::VS) & 1) ^ 1);
              if (!ok) break;
              bar = tc::smem_u32(&v_full[s]);
              tc::mbar_expect_tx(bar, L::TILE);
              for (int c = 0; c < L::CHUNKS; ++c)
                tc::tma_load_2d(tc::smem_u32(smem + L::V + s * L::TILE + c * L::CHUNK), &tmV, bar, it.h * HD + c * 64, now);
              ++vc;
            }
          }
          if (!ok || !it.next(a)) break;
          entry = tile_entry(a, it.b, it.kt0);
        } while (true);
        issued[0] = FP8 ? cc : kc;
        issued[1] = vc;
      }
    } else if (warp == 1) {
      // -------------------------------------------------------------------- MMA issuer (one elected lane), query tiles
      const bool leader = tc::elect_one();
      constexpr int QK_PARTS = FP8 ? 1 : 2;       // (FP8: shared-memory bandwidth counts, and each part reads Q again)
      constexpr uint32_t idesc_qk = tc::umma_idesc(128, TT_KEYS / QK_PARTS, 0, 0, MMA_F16, MMA_F16);
      constexpr uint32_t idesc_pv = tc::umma_idesc(128, HD, 0, 1, MMA_F16, MMA_F16);
      const uint64_t q_desc = tc::umma_desc_sw128(tc::smem_u32(smem + L::Q), 16, 1024);
      const uint64_t k_desc = tc::umma_desc_sw128(tc::smem_u32(smem + L::K), 16, 1024);
      const uint64_t v_desc = tc::umma_desc_sw128(tc::smem_u32(smem + L::V), L::CHUNK, 1024);
      int kc = 0, vc = 0, item = 0, sc0 = 0, sc1 = 0;
      bool ok = true, more;
      auto load_q = [&]() {
        const uint32_t bar = tc::smem_u32(q_full);
        const int copies = FP8 ? p.copies : 1;
        tc::mbar_expect_tx(bar, W * copies * L::CHUNKS * p.npt * rep * 128);
        for (int w = 0; w < W; ++w)
          for (int q = 0; q < copies; ++q)
            for (int c = 0; c < L::CHUNKS; ++c)
              tc::tma_load_3d(tc::smem_u32(smem + L::Q + w * L::TILE + c * L::CHUNK + q * (128 / copies) * 128), &tmQ, bar, c * 64, it.h * rep,
                              it.s.tok0 + (it.g * W + w) * p.npt);
      };
      if (leader) load_q();
      do {
        const int nt = it.kt1 - it.kt0, steps = W == 2 ? 2 * nt : nt;
        // S of a step; steps alternate between the streams.  The stream's last P V was issued before, and runs before.
        auto issue_qk = [&](int step) -> bool {
          const int w = step & 1, s = kc % L::KS;
          if (W == 1 || w == 0) {
            if (!wait(&k_full[s], (kc / L::KS) & 1)) return false;
            tc::tc_fence_after_sync();
          }
          if (leader) {
            // the scores of 64 keys after the other 64: the softmax warps start on the first half
            const uint64_t qd = q_desc + (uint64_t)((W == 2 ? w : 0) * (L::TILE >> 4)), kd = k_desc + (uint64_t)(s * (L::TILE >> 4));
#pragma unroll
            for (int hf = 0; hf < QK_PARTS; ++hf) {
#pragma unroll
              for (int kk = 0; kk < HD / 16; ++kk) {
                const uint32_t off = ((kk >> 2) * L::CHUNK + (kk & 3) * 32) >> 4;
                tc::umma_ss(tmem_base + w * 128 + hf * 64, qd + off, kd + off + hf * (64 * 128 >> 4), idesc_qk, kk != 0);
              }
              tc::umma_commit(tc::smem_u32(hf == QK_PARTS - 1 ? &s_full[w] : &s_half[w]));
            }
            if (W == 1 || w == 1) tc::umma_commit(tc::smem_u32(&k_empty[s]));
          }
          if (W == 1 || w == 1) ++kc;
          return true;
        };
        ok = wait(FP8 ? q_ready : q_full, item & 1);
        tc::tc_fence_after_sync();
        ok = ok && issue_qk(0);
        for (int step = 0; step < steps && ok; ++step) {
          if (step + 1 < steps && !(ok = issue_qk(step + 1))) break;
          const int w = step & 1, s = vc % L::VS;
          if (W == 1 || w == 0)
            if (!(ok = wait(&v_full[s], (vc / L::VS) & 1))) break;
          if (step == 0 && !(ok = wait(o_empty, (item & 1) ^ 1))) break;
          // O += P V in two halves of 64 keys, in the order in which the softmax warps finish them
          constexpr int FIRST = FP8 ? 0 : 1;
          int &sc = w ? sc1 : sc0;
          const uint64_t vd = v_desc + (uint64_t)(s * (L::TILE >> 4));
          auto issue_pv = [&](int hf, bool accumulate) {
#pragma unroll
            for (int k4 = 0; k4 < TT_KEYS / 32; ++k4)
              tc::umma_ts(tmem_base + 256 + w * 128, tmem_base + w * 128 + hf * 64 + k4 * 8, vd + (uint64_t)(((hf * 4 + k4) * 16 * 128) >> 4), idesc_pv,
                          (accumulate || k4 != 0) ? 1u : 0u);
          };
          if (!(ok = wait(&p_part[FIRST * 2 + w], sc & 1))) break;
          tc::tc_fence_after_sync();
          if (leader) issue_pv(FIRST, step > 1);
          if (!(ok = wait(&p_part[(1 - FIRST) * 2 + w], sc & 1))) break;
          ++sc;
          tc::tc_fence_after_sync();
          if (leader) {
            issue_pv(1 - FIRST, true);
            if (W == 1 || w == 1) tc::umma_commit(tc::smem_u32(&v_empty[s]));
            if (step == steps - 1) tc::umma_commit(tc::smem_u32(o_full));
          }
          if (W == 1 || w == 1) ++vc;
        }
        ++item;
        __syncwarp();
        // the next piece's queries: every Q K^T of this one has retired (its last P came from it), so their place is free
        more = ok && it.next(a);
        if (more && leader) load_q();
      } while (more);
      issued[2] = item;
    } else if (FP8 && warp == 2) {
      // -------------------------------------------------------------------- row scales, four keys per lane, a tile ahead of their use
      int tile = 0;
      bool ok = true;
      do {
        const int kv_len = it.s.past + it.s.n;
        float k1[4], v1[4], k0[4], v0[4];
        auto request = [&](int entry, int j, float (&k)[4], float (&v)[4]) {
          const int base = tile_row(a, entry, j);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = i * 32 + lane, row = base + key;
            const bool there = j < it.kt1 && j * TT_KEYS + key < kv_len && row >= 0 && row < a.cache_rows;
            k[i] = there ? a.k_scale[row] : 0.f;
            v[i] = there ? a.v_scale[row] : 0.f;
          }
        };
        int entry1 = tile_entry(a, it.b, min(it.kt0 + 1, it.kt1 - 1));
        request(tile_entry(a, it.b, it.kt0), it.kt0, k1, v1);
        for (int j = it.kt0; j < it.kt1 && ok; ++j, ++tile) {
#pragma unroll
          for (int i = 0; i < 4; ++i) { k0[i] = k1[i]; v0[i] = v1[i]; }
          request(entry1, j + 1, k1, v1);
          entry1 = tile_entry(a, it.b, min(j + 2, it.kt1 - 1));
          if (!(ok = wait(&g_empty[tile & 3], ((tile >> 2) & 1) ^ 1))) break;
          float *to = scales + (tile & 3) * 384;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            to[i * 32 + lane] = k0[i];
            to[128 + i * 32 + lane] = v0[i];
            to[256 + i * 32 + lane] = fminf(fmaxf(__log2f(v0[i]), TT_LEAST_LOG2), 60.f);      // (beyond 2^60 P itself overflows)
          }
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(tc::smem_u32(&g_full[tile & 3]));
        }
      } while (ok && it.next(a));
    }
  } else if (warp < L::SOFT + 8) {
    if constexpr (FP8) asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");
    // -------------------------------------------------------------------- softmax: stream w, a query row per thread
    const int w = (warp - L::SOFT) >> 2, quarter = warp & 3, r = quarter * 32 + lane;
    const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
    const uint32_t t_s = tmem_base + lane_base + w * 128, t_o = tmem_base + lane_base + 256;
    // m_ref in units of the scores (FP8: already in log2 units, c being the row's own)
    float c = p.scale_log2;
    const float cm = FP8 ? 1.f : c;
    int item = 0, sc = 0, tc_count = 0;          // tc_count: tiles of earlier pieces (ring positions)
    bool ok = true;
    do {
      const int nt = it.kt1 - it.kt0;
      const int node0 = (it.g * W + (W == 2 ? w : 0)) * p.npt;
      const int rows = min(p.npt, it.s.n - node0) * rep;              // may be <= 0: the pair's second tile
      // FP8: this row's copy, its row in the copy, and the copy's share of the columns
      const int per_copy = FP8 ? 128 / p.copies : 128, copy = FP8 ? r / per_copy : 0, rl = FP8 ? r % per_copy : r;
      const int ch_lo = FP8 ? copy * (4 / p.copies) : 0, ch_hi = FP8 ? ch_lo + 4 / p.copies : 4;
      const bool warp_active = (FP8 ? quarter * 32 % per_copy : quarter * 32) < rows, valid = rl < rows;
      const int node = valid ? node0 + rl / rep : 0, tok = it.s.tok0 + node;
      float m_ref = -INFINITY, l = 0.f;
      bool first = true;
      for (int j = W == 2 ? 0 : w; j < nt; j += W == 2 ? 1 : 2) {
        const int tile = tc_count + j;
        const int j0 = (it.kt0 + j) * TT_KEYS - it.s.past;            // the tile's first key, counted from the first new token
        const bool edge = j0 > -TT_KEYS;                              // holds new tokens (and perhaps rows behind them)
        if (!(ok = wait(FP8 ? &s_full[w] : &s_half[w], sc & 1))) break;
        tc::tc_fence_after_sync();
        if (edge && (W == 1 || w == 0)) {
          // V rows that must not meet a zero probability as NaN or infinity (comment at the top).  Behind the wait for S: it was issued
          // after the P V of two tiles before, so the V ring's place is in this tile's phase or the one before, never two before,
          // which the parity could not tell from this one.
          const int s = tile % L::VS, key = j0 + r;
          if (!(ok = wait(&v_full[s], (tile / L::VS) & 1))) break;
          if (key >= 0) {
            uint8_t *vrow = smem + L::V + s * L::TILE + r * 128;
            const bool behind = key >= it.s.n;
            bool handed = false;
            constexpr uint32_t e = MMA_F16 ? 0x7c007c00u : 0x7f807f80u;
#pragma unroll 1
            for (int i = 0; i < L::CHUNKS * 8; ++i) {
              uint4 *at = reinterpret_cast<uint4 *>(vrow + (i >> 3) * L::CHUNK + ((i ^ r) & 7) * 16);      // (eight rows, eight bank groups)
              const uint4 x = *at;
              uint32_t xs[4] = {x.x, x.y, x.z, x.w}, worst = 0;
#pragma unroll
              for (int q4 = 0; q4 < 4; ++q4) {
                const uint32_t gone = ((xs[q4] & e & 0xffff0000u) == (e & 0xffff0000u) ? 0xffff0000u : 0u) | ((xs[q4] & e & 0xffffu) == (e & 0xffffu) ? 0xffffu : 0u);
                worst |= gone;
                xs[q4] &= ~gone;
              }
              if (behind) *at = make_uint4(0u, 0u, 0u, 0u);
              else if (worst) { *at = make_uint4(xs[0], xs[1], xs[2], xs[3]); handed = true; }
            }
            if (handed) bad_item[item & 1] = item + 1;
            if (behind || handed) tc::fence_proxy_async_smem();
          }
        }
        const float4 *ksc = reinterpret_cast<const float4 *>(scales + (tile & 3) * 384), *vsc = ksc + 32, *lvs = ksc + 64;
        if constexpr (FP8) {
          if (!(ok = wait(&g_full[tile & 3], (tile >> 2) & 1))) break;
          if (j == w) {
            if (!(ok = wait(&q_scaled[item & 1], (item >> 1) & 1))) break;
            c = p.scale_log2 * scales[4 * 384 + (item & 1) * 128 + r];
          }
        }
        if (warp_active) {
          // moves the reference to mx where the row outgrew it; S of this step is complete, so every earlier P V of the stream has
          // retired and O may be rescaled
          auto refer = [&](float mx) {
            const bool need = first || (mx - m_ref) * cm > TT_RESCALE;
            const float m_new = need ? mx : m_ref;
            if (!first && __any_sync(0xffffffffu, need && valid)) {
              const float f = need ? tt_exp2((m_ref - m_new) * cm) : 1.f;
              l *= f;
#pragma unroll 1
              for (int ch = 0; ch < HD / 16; ++ch) {
                uint32_t o[16];
                tc::tmem_ld_32x32b_x16(t_o + w * 128 + ch * 16, o);
                tc::tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                tc::tmem_st_32x32b_x16(t_o + w * 128 + ch * 16, o);
              }
            }
            m_ref = m_new;
            first = false;
          };
          auto announce = [&](int hf) {                                       // 64 keys of P (half hf) are in tensor memory
            tc::tmem_st_wait();
            tc::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(tc::smem_u32(&p_part[hf * 2 + w]));
          };
          if constexpr (!FP8) {
            // Scores in four chunks of 32 columns.  All four give the maximum; chunks 2 and 3 stay in registers and are exponentiated
            // first, chunks 0 and 1 are read again (128 scores in registers would spill, and spilled registers live in L2: shared
            // memory leaves L1 next to nothing).  P of keys 64 .. 127 goes over chunk 2, that of 0 .. 63 over chunk 0.
            auto mask = [&](uint32_t (&d)[32], int ch) {
              if (!edge) return;
              const uint32_t seen = valid ? sees_word(a, tok, node, it.s.n, j0 + ch * 32) : 0u;
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (!((seen >> i) & 1u)) d[i] = 0xff800000u;      // -inf
            };
            float m0 = -INFINITY, m1 = -INFINITY;
            auto maximum = [&](const uint32_t (&d)[32]) {
#pragma unroll
              for (int i = 0; i < 32; i += 4) {
                m0 = tc::max3(m0, __uint_as_float(d[i]), __uint_as_float(d[i + 1]));
                m1 = tc::max3(m1, __uint_as_float(d[i + 2]), __uint_as_float(d[i + 3]));
              }
            };
            uint32_t u[32], v[32];
            tc::tmem_ld_32x32b_x32(t_s, u);
            tc::tmem_ld_32x32b_x32(t_s + 32, v);
            tc::tmem_ld_wait();
            mask(u, 0);
            mask(v, 1);
            maximum(u);
            maximum(v);
            if (!(ok = wait(&s_full[w], sc & 1))) break;
            tc::tc_fence_after_sync();
            tc::tmem_ld_32x32b_x32(t_s + 64, u);
            tc::tmem_ld_32x32b_x32(t_s + 96, v);
            tc::tmem_ld_wait();
            mask(u, 2);
            mask(v, 3);
            maximum(u);
            maximum(v);
            refer(fmaxf(m0, m1));
            const float neg_mc = m_ref == -INFINITY ? 0.f : -m_ref * cm;      // (a row that sees nothing yet: every exponential is 0)
            tc::F2 la{{0.f, 0.f}}, lb{{0.f, 0.f}};
            const tc::F2 c2{{c, c}}, n2{{neg_mc, neg_mc}};
            auto exponentials = [&](const uint32_t (&d)[32], int ch) {
              uint32_t packed[16];
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                tc::F2 x = tc::fma2(tc::F2{{__uint_as_float(d[2 * i]), __uint_as_float(d[2 * i + 1])}}, c2, n2);
                x = tc::F2{{tt_exp2(x.f[0]), tt_exp2(x.f[1])}};
                if (i & 1) lb = tc::add2(lb, x); else la = tc::add2(la, x);
                packed[i] = F16 ? tc::pack_f16x2(x.f[0], x.f[1]) : tc::pack_bf16x2(x.f[0], x.f[1]);
              }
              tc::tmem_st_32x32b_x16(t_s + (ch >> 1) * 64 + (ch & 1) * 16, packed);
            };
            exponentials(u, 2);
            tc::tmem_ld_32x32b_x32(t_s, u);
            exponentials(v, 3);
            announce(1);
            tc::tmem_ld_32x32b_x32(t_s + 32, v);
            tc::tmem_ld_wait();
            mask(u, 0);
            mask(v, 1);
            exponentials(u, 0);
            exponentials(v, 1);
            announce(0);
            l += (la.f[0] + la.f[1]) + (lb.f[0] + lb.f[1]);
          } else {
            // 32 columns at a time, once for the maximum and once for the exponentials: scores times the row scales of K
            auto load = [&](int ch, tc::F2 (&d)[16], uint32_t &seen) {
              uint32_t raw[32];
              tc::tmem_ld_32x32b_x32(t_s + ch * 32, raw);
              seen = !edge ? 0xffffffffu : valid ? sees_word(a, tok, node, it.s.n, j0 + ch * 32) : 0u;
              float4 k4[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) k4[i] = ksc[ch * 8 + i];
              tc::tmem_ld_wait();
              if (seen != 0xffffffffu) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {                                   // (the scale of an unseen row may be anything)
                  k4[i].x = (seen >> (4 * i)) & 1u ? k4[i].x : 1.f; k4[i].y = (seen >> (4 * i)) & 2u ? k4[i].y : 1.f;
                  k4[i].z = (seen >> (4 * i)) & 4u ? k4[i].z : 1.f; k4[i].w = (seen >> (4 * i)) & 8u ? k4[i].w : 1.f;
                }
#pragma unroll
                for (int i = 0; i < 32; ++i)
                  if (!((seen >> i) & 1u)) raw[i] = 0xff800000u;                // -inf
              }
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                d[2 * i] = tc::mul2(tc::F2{{__uint_as_float(raw[4 * i]), __uint_as_float(raw[4 * i + 1])}}, tc::F2{{k4[i].x, k4[i].y}});
                d[2 * i + 1] = tc::mul2(tc::F2{{__uint_as_float(raw[4 * i + 2]), __uint_as_float(raw[4 * i + 3])}}, tc::F2{{k4[i].z, k4[i].w}});
              }
            };
            tc::F2 d[16];
            uint32_t seen;
            const tc::F2 c2{{c, c}};
            float m0 = -INFINITY, m1 = -INFINITY;
#pragma unroll 1
            for (int ch = ch_lo; ch < ch_hi; ++ch) {
              load(ch, d, seen);
              // the reference follows the scale-weighted probabilities: s c + log2(V scale)
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const float4 l4 = lvs[ch * 8 + i];
                const tc::F2 x = tc::fma2(d[2 * i], c2, tc::F2{{l4.x, l4.y}}), y = tc::fma2(d[2 * i + 1], c2, tc::F2{{l4.z, l4.w}});
                m0 = tc::max3(m0, x.f[0], x.f[1]);
                m1 = tc::max3(m1, y.f[0], y.f[1]);
              }
            }
            refer(fmaxf(m0, m1));
            const float neg_mc = m_ref == -INFINITY ? 0.f : -m_ref;
            const tc::F2 n2{{neg_mc, neg_mc}};
            tc::F2 la{{0.f, 0.f}}, lb{{0.f, 0.f}};
#pragma unroll 1
            for (int ch = 0; ch < 4; ++ch) {
              uint32_t packed[16];
              if (ch < ch_lo || ch >= ch_hi) {                                  // another copy's columns
#pragma unroll
                for (int i = 0; i < 16; ++i) packed[i] = 0u;
              } else {
                if (ch_hi - ch_lo > 1) load(ch, d, seen);                       // (a single chunk is still there)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                  tc::F2 x = tc::fma2(d[2 * i], c2, n2), y = tc::fma2(d[2 * i + 1], c2, n2);
                  x = tc::F2{{tt_exp2(x.f[0]), tt_exp2(x.f[1])}};
                  y = tc::F2{{tt_exp2(y.f[0]), tt_exp2(y.f[1])}};
                  la = tc::add2(la, x);
                  lb = tc::add2(lb, y);
                  const float4 v4 = vsc[ch * 8 + i];
                  x = tc::mul2(x, tc::F2{{v4.x, v4.y}});
                  y = tc::mul2(y, tc::F2{{v4.z, v4.w}});
                  if (seen != 0xffffffffu) {
                    x.f[0] = (seen >> (4 * i)) & 1u ? x.f[0] : 0.f; x.f[1] = (seen >> (4 * i)) & 2u ? x.f[1] : 0.f;
                    y.f[0] = (seen >> (4 * i)) & 4u ? y.f[0] : 0.f; y.f[1] = (seen >> (4 * i)) & 8u ? y.f[1] : 0.f;
                  }
                  const __half2 h0 = __floats2half2_rn(x.f[0], x.f[1]), h1 = __floats2half2_rn(y.f[0], y.f[1]);      // (an infinite scale stays infinite)
                  packed[2 * i] = *reinterpret_cast<const uint32_t *>(&h0);
                  packed[2 * i + 1] = *reinterpret_cast<const uint32_t *>(&h1);
                }
              }
              tc::tmem_st_32x32b_x16(t_s + (ch >> 1) * 64 + (ch & 1) * 16, packed);      // (chunk 3 is still to be read when chunk 2 is overwritten)
              if (ch & 1) announce(ch >> 1);
            }
            l += (la.f[0] + la.f[1]) + (lb.f[0] + lb.f[1]);
          }
        } else {
          if (!FP8 && !(ok = wait(&s_full[w], sc & 1))) break;
          tc::tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) {
            tc::mbar_arrive(tc::smem_u32(&p_part[w]));
            tc::mbar_arrive(tc::smem_u32(&p_part[2 + w]));
          }
        }
        ++sc;
        if constexpr (FP8) {
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(tc::smem_u32(&g_empty[tile & 3]));
        }
      }
      if (!ok) break;
      // ---- the piece's result.  Both streams meet here once (W = 1: to join their halves of the keys).
      ml[((item & 1) * 2 + w) * 128 + r] = make_float2(m_ref, l);
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(tc::smem_u32(x_full));
      if (!(ok = wait(x_full, item & 1)) || !(ok = wait(o_full, item & 1))) break;
      tc::tc_fence_after_sync();
      if (warp_active) {
        float m = m_ref, f0 = 1.f, f1 = 0.f;
        if constexpr (W == 1) {
          const float2 x0 = ml[((item & 1) * 2) * 128 + r], x1 = ml[((item & 1) * 2 + 1) * 128 + r];
          m = fmaxf(x0.x, x1.x);
          f0 = x0.x == -INFINITY ? 0.f : tt_exp2((x0.x - m) * cm);
          f1 = x1.x == -INFINITY ? 0.f : tt_exp2((x1.x - m) * cm);
          l = x0.y * f0 + (nt > 1 ? x1.y * f1 : 0.f);
        }
        // (copies of a query tile leave partial results of their own, complete pieces by token and head)
        const bool complete = it.whole(), whole = complete && (!FP8 || p.copies == 1), bad = bad_item[item & 1] == item + 1;
        const float inv = (whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f);
        const size_t head = (size_t)tok * a.n_q + it.h * rep + (valid ? rl % rep : 0);
        const int slot = (int)blockIdx.x * 2 + (it.kt0 == 0 ? 1 : 0);
        const size_t srow = FP8 && complete ? (size_t)gridDim.x * 2 * p.slot_rows + (size_t)copy * a.total_new * a.n_q + head
                                            : (size_t)slot * p.slot_rows + (W == 2 ? w : 0) * p.npt * rep + r;
        constexpr int COLS = W == 1 ? HD / 2 : HD;
        const int col0 = W == 1 ? w * COLS : 0;
        if (valid && col0 == 0 && (W == 2 || w == 0)) {
          if (!whole) reinterpret_cast<float2 *>(a.scratch)[srow] = make_float2(m * cm, l);
          else if (a.lse) a.lse[head] = l == 0.f ? -INFINITY : FP8 ? tt_lse(m, l, true) : m * (cm * 0.6931471805599453f) + logf(l);
        }
#pragma unroll 1
        for (int ch = 0; ch < COLS / 32; ++ch) {
          const int d0 = col0 + ch * 32;
          uint32_t x[32];
          float o[32];
          tc::tmem_ld_32x32b_x32(t_o + (W == 2 ? w * 128 : 0) + d0, x);
          tc::tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = W == 1 ? __uint_as_float(x[i]) * f0 : __uint_as_float(x[i]);
          if (W == 1 && nt > 1) {
            tc::tmem_ld_32x32b_x32(t_o + 128 + d0, x);
            tc::tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = fmaf(__uint_as_float(x[i]), f1, o[i]);
          }
          if (valid) {
            if (bad && (!FP8 || copy == 0)) {
              // drafted tokens of this piece whose V row was not finite: what the rows that see them get from it
#pragma unroll 1
              for (int q2 = max(0, it.kt0 * TT_KEYS - it.s.past); q2 < min(it.s.n, it.kt1 * TT_KEYS - it.s.past); ++q2) {
                const int row = tree_row(a, it.b, it.s.past + q2);
                if (row < 0 || !tree_sees(a, tok, node, it.s.past, it.s.n, it.s.past + q2)) continue;
                if constexpr (FP8) {
                  const uint8_t *v = reinterpret_cast<const uint8_t *>(a.v) + ((size_t)row * a.n_kv + it.h) * HD + d0;
#pragma unroll
                  for (int i = 0; i < 32; ++i)
                    if ((v[i] & 0x7f) == 0x7f) o[i] = NAN;
                  continue;
                }
                const uint16_t *v = reinterpret_cast<const uint16_t *>(a.v) + ((size_t)row * a.n_kv + it.h) * HD + d0;
                const uint16_t e = F16 ? 0x7c00 : 0x7f80;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                  const uint16_t bits = v[i];
                  if ((bits & e) == e) o[i] += F16 ? __half2float(__ushort_as_half(bits)) : __uint_as_float((uint32_t)bits << 16);
                }
              }
            }
            if (whole) {
              uint32_t y[16];
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const float e0 = l == 0.f ? 0.f : o[2 * i] * inv, e1 = l == 0.f ? 0.f : o[2 * i + 1] * inv;
                if constexpr (F16) {
                  const __half2 h2 = __floats2half2_rn(e0, e1);
                  y[i] = *reinterpret_cast<const uint32_t *>(&h2);
                } else {
                  y[i] = tc::pack_bf16x2(e0, e1);
                }
              }
              uint16_t *dst = reinterpret_cast<uint16_t *>(a.out) + head * HD + d0;
              if (p.store32) {
                tc::st_global_v8(dst, y);
                tc::st_global_v8(dst + 16, y + 8);
              } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) dst[i] = (uint16_t)(y[i >> 1] >> ((i & 1) * 16));
              }
            } else {
              float *dst = p.part_o + srow * HD + d0;
#pragma unroll
              for (int i = 0; i < 32; i += 8) {
                uint32_t y[8];
#pragma unroll
                for (int q4 = 0; q4 < 8; ++q4) y[q4] = __float_as_uint(o[i + q4]);
                tc::st_global_v8(dst + i, y);
              }
            }
          }
        }
      }
      tc::tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(tc::smem_u32(o_empty));
      tc_count += nt;
      ++item;
    } while (it.next(a));
  } else if constexpr (FP8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    // -------------------------------------------------------------------- widening warps: codes -> swizzled halves, scales; queries
    const int t = threadIdx.x - 12 * 32;
    int cc = 0, tile = 0, item = 0;
    bool ok = true;
    do {
      const int kv_len = it.s.past + it.s.n;
      // the query rows, one per thread: times a power of two, bf16 -> half
      if (!(ok = wait(q_full, item & 1))) break;
      float back = 1.f;
      if constexpr (!F16) {
        uint8_t *qrow = smem + L::Q + t * 128;               // (its pieces in an order that has eight lanes in eight bank groups)
        uint32_t top = 0;
#pragma unroll 1
        for (int i = 0; i < L::CHUNKS * 8; ++i) {
          const uint4 x = *reinterpret_cast<const uint4 *>(qrow + (i >> 3) * L::CHUNK + ((i ^ t) & 7) * 16);
          const uint32_t xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) top = max(top, max(xs[q4] & 0x7f80u, (xs[q4] >> 16) & 0x7f80u));
        }
        // exponent of the row's maximum -> 14 (a row without finite maximum, and one of zeros: as it is)
        const int e = (int)(top >> 7);
        const int shift = e == 0 || e == 255 ? 0 : min(max(14 - (e - 127), -120), 120);
        const float up = __uint_as_float((uint32_t)(127 + shift) << 23);
        back = __uint_as_float((uint32_t)(127 - shift) << 23);
#pragma unroll 1
        for (int i = 0; i < L::CHUNKS * 8; ++i) {
          uint4 *at = reinterpret_cast<uint4 *>(qrow + (i >> 3) * L::CHUNK + ((i ^ t) & 7) * 16);
          const uint4 x = *at;
          uint32_t xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const __half2 h2 = __floats2half2_rn(__uint_as_float(xs[q4] << 16) * up, __uint_as_float(xs[q4] & 0xffff0000u) * up);
            xs[q4] = *reinterpret_cast<const uint32_t *>(&h2);
          }
          *at = make_uint4(xs[0], xs[1], xs[2], xs[3]);
        }
        tc::fence_proxy_async_smem();
      }
      scales[4 * 384 + (item & 1) * 128 + t] = back;
      __syncwarp();
      if (lane == 0) {
        tc::mbar_arrive(tc::smem_u32(q_ready));
        tc::mbar_arrive(tc::smem_u32(&q_scaled[item & 1]));
      }
      ++item;
      for (int j = it.kt0; j < it.kt1 && ok; ++j, ++tile) {
        const int live = kv_len - j * TT_KEYS;                 // rows from here on are behind the sequence: zeros
#pragma unroll
        for (int kv = 0; kv < 2; ++kv, ++cc) {
          const int cs = cc % L::CS, ds = kv ? tile % L::VS : 0;
          const uint8_t *src = smem + L::C + cs * L::CODE_TILE + t * HD;
          uint8_t *dst = smem + (kv ? L::V : L::K) + ds * L::TILE + t * 128;
          ok = ok && wait(&c_full[cs], (cc / L::CS) & 1) && (kv ? wait(&v_empty[ds], ((tile / L::VS) & 1) ^ 1) : wait(&k_empty[0], (tile & 1) ^ 1));
          if (!ok) break;
          // A thread widens its key's row: eight lanes, eight rows, one 16-byte column -- with the swizzles of the codes (TMA's) and of the
          // MMA's operand no two of them share a bank.
          constexpr int PIECES = HD / 16;
          const uint32_t from = HD == 128 ? (t & 7) << 4 : ((t >> 1) & 3) << 4, to = (t & 7) << 4;
          uint4 c4[PIECES];
#pragma unroll
          for (int i = 0; i < PIECES; ++i) c4[i] = t < live ? *reinterpret_cast<const uint4 *>(src + ((i << 4) ^ from)) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
          for (int i = 0; i < PIECES; ++i) {
            uint4 h0, h1;
            widen4(c4[i].x, h0.x, h0.y);
            widen4(c4[i].y, h0.z, h0.w);
            widen4(c4[i].z, h1.x, h1.y);
            widen4(c4[i].w, h1.z, h1.w);
            uint8_t *line = dst + (i >> 2) * L::CHUNK;
            *reinterpret_cast<uint4 *>(line + (((i & 3) << 5) ^ to)) = h0;
            *reinterpret_cast<uint4 *>(line + ((((i & 3) << 5) | 16) ^ to)) = h1;
          }
          tc::fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            tc::mbar_arrive(tc::smem_u32(&c_empty[cs]));
            tc::mbar_arrive(tc::smem_u32(kv ? &v_full[ds] : &k_full[0]));
          }
        }
      }
    } while (ok && it.next(a));
  }
  tc::tc_fence_before_sync();
  __syncthreads();
  if (*abort_flag) {
    // a wait ran out: copies and products under way end before shared and tensor memory are given back (these waits are bounded too)
    if (warp == 0 && lane == 0) {
      auto landed = [&](uint64_t *full, int places, int n) {
        for (int i = max(0, n - places); i < n; ++i) tc::mbar_wait(tc::smem_u32(&full[i % places]), (i / places) & 1);
      };
      if constexpr (FP8) {
        landed(c_full, L::CS, issued[0]);
      } else {
        landed(k_full, L::KS, issued[0]);
        landed(v_full, L::VS, issued[1]);
      }
      landed(q_full, 1, issued[2]);
    }
    if (warp == 1) {
      if (tc::elect_one()) tc::umma_commit(tc::smem_u32(drained));
      __syncwarp();
      tc::mbar_wait(tc::smem_u32(drained), 0);
    }
    __syncthreads();
  }
  if (warp == 1) {
    __syncwarp();
    tc::tc_fence_after_sync();
    tc::tmem_dealloc(tmem_base, 512);
  }
}

// joins the partial results of the pieces that a (sequence, group, head) was cut into: gridDim.y blocks per new token, TJ_THREADS / (HD / 4) heads
// at a time
constexpr int TJ_THREADS = 256;
template <int HD, bool F16>
__global__ void __launch_bounds__(TJ_THREADS) tree_attention_tc_join_kernel(TreeTcArgs p, int grid, int tiles_per_group) {
  const TreeArgs &a = p.a;
  const int t = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int group_tokens = tiles_per_group * p.npt, rep = a.n_q / a.n_kv;
  // (the lengths are the call's inputs: the sums over them run beside the pieces' kernel)
  __shared__ int s_sum[2][2][TJ_THREADS / 32], s_b;        // [class][before, total]
  if (tid == 0) s_b = -1;
  __syncthreads();
  int sum[2][2] = {{0, 0}, {0, 0}};
  for (int b = tid; b < a.n_seqs; b += TJ_THREADS) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (k >= p.classes) break;
      const SeqShape s = seq_shape(a, b, Split{group_tokens, p.classes, k});
      const int u = units_of(s);
      sum[k][1] += u;
      if (s.tok0 + s.n <= t) sum[k][0] += u;
      else if (s.tok0 <= t) s_b = b;
    }
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (k >= p.classes) break;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      int v = sum[k][q];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      if (lane == 0) s_sum[k][q][warp] = v;
    }
  }
  __syncthreads();
  wait_for_previous();
  const int b = s_b;
  if (b < 0) return;                                       // a row behind the last sequence
  // what the classes do of this token's sequence
  SeqShape of[2];
  int before[2] = {0, 0}, per[2] = {1, 1};
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (k >= p.classes) break;
    of[k] = seq_shape(a, b, Split{group_tokens, p.classes, k});
    int total = 0;
#pragma unroll
    for (int w = 0; w < TJ_THREADS / 32; ++w) { before[k] += s_sum[k][0][w]; total += s_sum[k][1][w]; }
    const int ctas = (grid - k + p.classes - 1) / p.classes;
    per[k] = max(1, (total + ctas - 1) / ctas);
  }
  const int node = t - of[0].tok0, g = node / group_tokens;
  constexpr int LANES = HD / 4, PER_PASS = TJ_THREADS / LANES;
  const int d = (tid % LANES) * 4, shift = p.copies == 4 ? 2 : p.copies == 2 ? 1 : 0;
#pragma unroll 1
  for (int hq = blockIdx.y * PER_PASS + tid / LANES; hq < a.n_q; hq += gridDim.y * PER_PASS) {
    // the CTAs that worked on this row's item, of one class, in the order of the keys
    const int h = hq / rep, row = (node - g * group_tokens) * rep + hq % rep;
    int cls = 0, c0 = 0, n = 0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (k >= p.classes) break;
      const SeqShape &s = of[k];
      if (g < s.g0 || g >= s.g0 + s.groups || (h - s.h0) % s.h_step) continue;
      const int first = before[k] + ((g - s.g0) * s.heads + (h - s.h0) / s.h_step) * s.tiles;
      cls = k;
      c0 = first / per[k];
      n = (first + s.tiles - 1) / per[k] - c0 + 1;
    }
    const int pieces = n;
    n *= p.copies;
    if (n <= 1) continue;                                    // whole: already in `out`
    // the first piece starts at the first key: its CTA's slot 1; the others are the first piece of theirs: slot 0.  Copies of a complete
    // piece (a CTA may have many of these): by token and head.
    auto piece = [&](int ic) -> size_t {
      const int i = ic >> shift, copy = ic & (p.copies - 1);
      if (pieces == 1) return (size_t)grid * 2 * p.slot_rows + ((size_t)copy * a.total_new + t) * a.n_q + hq;
      return (size_t)(((c0 + i) * p.classes + cls) * 2 + (i == 0 ? 1 : 0)) * p.slot_rows + copy * (128 >> shift) + row;
    };
    const float2 *ml = reinterpret_cast<const float2 *>(a.scratch);
    float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f, o2 = 0.f, o3 = 0.f;
    for (int i0 = 0; i0 < n; i0 += 4) {                      // four pieces in flight
      float2 x[4];
      float4 u[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        x[q] = make_float2(-INFINITY, 0.f);
        if (i0 + q < n) {
          const size_t at = piece(i0 + q);
          x[q] = ml[at];
          u[q] = *reinterpret_cast<const float4 *>(p.part_o + at * HD + d);
        }
      }
      float m_new = m;
#pragma unroll
      for (int q = 0; q < 4; ++q) m_new = fmaxf(m_new, x[q].x);
      const float back = m == -INFINITY ? 0.f : tt_exp2(m - m_new);
      l *= back; o0 *= back; o1 *= back; o2 *= back; o3 *= back;
      m = m_new;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float f = x[q].x == -INFINITY ? 0.f : tt_exp2(x[q].x - m);
        if (f == 0.f && x[q].y == 0.f) continue;             // saw nothing
        l = fmaf(x[q].y, f, l);
        o0 = fmaf(u[q].x, f, o0); o1 = fmaf(u[q].y, f, o1); o2 = fmaf(u[q].z, f, o2); o3 = fmaf(u[q].w, f, o3);
      }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (l == 0.f) o0 = o1 = o2 = o3 = 0.f;
    const size_t head = (size_t)t * a.n_q + hq;
    uint16_t y[4];
    if constexpr (F16) {
      y[0] = __half_as_ushort(__float2half_rn(o0 * inv)); y[1] = __half_as_ushort(__float2half_rn(o1 * inv));
      y[2] = __half_as_ushort(__float2half_rn(o2 * inv)); y[3] = __half_as_ushort(__float2half_rn(o3 * inv));
    } else {
      y[0] = __bfloat16_as_ushort(__float2bfloat16_rn(o0 * inv)); y[1] = __bfloat16_as_ushort(__float2bfloat16_rn(o1 * inv));
      y[2] = __bfloat16_as_ushort(__float2bfloat16_rn(o2 * inv)); y[3] = __bfloat16_as_ushort(__float2bfloat16_rn(o3 * inv));
    }
    uint16_t *dst = reinterpret_cast<uint16_t *>(a.out) + head * HD + d;
    if (p.store32) *reinterpret_cast<uint2 *>(dst) = make_uint2((uint32_t)y[0] | (uint32_t)y[1] << 16, (uint32_t)y[2] | (uint32_t)y[3] << 16);
    else { dst[0] = y[0]; dst[1] = y[1]; dst[2] = y[2]; dst[3] = y[3]; }
    if (a.lse && d == 0) a.lse[head] = l == 0.f ? -INFINITY : tt_lse(m, l, a.k_scale != nullptr);
  }
}

// rows of a partial result: those of a group of query tiles, or all that a call has for one KV head
int tc_slot_rows(int total_new, int n_q, int n_kv) {
  const long long all = (long long)total_new * (n_q / n_kv);
  return all < 256 ? (int)all : 256;
}
// copies of query tiles: at most so many (copy, token) pairs leave results of their own (34 MB of scratch for 32 heads of 128); calls of
// more tokens lay their tiles out less often, for they have rows enough elsewhere
constexpr int TC_COPY_TOKENS = 2048;
size_t tc_scratch(int total_new, int n_q, int hd) {
  // (independent of the group size: a call's rows of one KV head are at most all its rows)
  const int rows = tc_slot_rows(total_new, n_q, 1);
  const long long copied = 4ll * total_new < TC_COPY_TOKENS ? 4ll * total_new : TC_COPY_TOKENS;
  return ((size_t)num_sms() * 2 * (rows < 128 ? 128 : rows) + (size_t)copied * n_q) * (hd + 2) * sizeof(float) + 256;
}

// shapes and addresses that the tensor-core form takes (TMA: 16-byte boundaries and strides)
bool tc_supported(const TreeArgs &a, bool q16, bool fp8) {
  if (!q16 || (a.hd != 64 && a.hd != 128) || a.n_q / a.n_kv > 128) return false;
  const uintptr_t at = (uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v | (uintptr_t)(a.q_stride * 2);
  return (at & 15) == 0 && a.cache_rows < (1 << 30) && (!fp8 || (a.n_kv * a.hd) % 16 == 0);
}

template <int HD, int W, bool F16, bool FP8>
int32_t launch_tc(TreeTcArgs p, cudaStream_t st) {
  using L = TreeLayout<HD, W, FP8>;
  static_assert(L::BYTES <= 232448, "shared memory of one CTA");
  const TreeArgs &a = p.a;
  const int rep = a.n_q / a.n_kv;
  CUtensorMap tq, tk, tv;
  const uint64_t cols = (uint64_t)a.n_kv * HD / (FP8 ? 2 : 1);             // codes travel as pairs of bytes
  if (make_tmap_3d_bf16(&tq, a.q, HD, a.n_q, a.total_new, HD, a.q_stride, 64, rep, p.npt) ||
      make_tmap_2d_bf16(&tk, a.k, a.cache_rows, cols, cols, TT_KEYS, FP8 ? HD / 2 : 64, FP8 && HD == 64 ? TMAP_SWIZZLE_64B : TMAP_SWIZZLE_128B) ||
      make_tmap_2d_bf16(&tv, a.v, a.cache_rows, cols, cols, TT_KEYS, FP8 ? HD / 2 : 64, FP8 && HD == 64 ? TMAP_SWIZZLE_64B : TMAP_SWIZZLE_128B))
    return report_error(SWIFTKV_ERR_CUDA, "tensor map");
  auto kernel = tree_attention_tc_kernel<HD, W, F16, FP8>;
  if (ensure_dynamic_smem(reinterpret_cast<const void *>(kernel), L::BYTES)) return report_error(SWIFTKV_ERR_CUDA, "shared memory");
  const long long groups = ((long long)a.max_new + W * p.npt - 1) / (W * p.npt), tiles = ((long long)a.max_kv + TT_KEYS - 1) / TT_KEYS;
  const double most = (double)groups * tiles * a.n_kv * a.n_seqs;
  if (most > 0x7fffffff) return report_error(SWIFTKV_ERR_UNSUPPORTED, "too many key tiles for one launch");
  const int grid = most < num_sms() ? (int)most : num_sms();
  p.classes = groups == 2 && grid > 1 ? 2 : 1;
  const size_t rows = (size_t)grid * 2 * p.slot_rows + (p.copies > 1 ? (size_t)p.copies * a.total_new * a.n_q : 0);
  const size_t ml_bytes = (rows * sizeof(float2) + 255) & ~(size_t)255;
  p.part_o = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(a.scratch) + ml_bytes);
  kernel<<<grid, L::THREADS, L::BYTES, st>>>(tq, tk, tv, p);
  cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess && (grid > 1 || p.copies > 1)) {
    constexpr int PER_PASS = TJ_THREADS / (HD / 4);
    // few tokens: their heads side by side; many: one block walks over a token's heads, for finding its pieces costs more than joining them
    // (64 sequences of 32 tokens over 1024 keys: 97 us -> 86; 16 of up to 32 tokens, with one block a token: 69.5 -> 70.8)
    const int passes = (a.n_q + PER_PASS - 1) / PER_PASS, wide = 8 * num_sms() / a.total_new + 1;
    e = launch_early(tree_attention_tc_join_kernel<HD, F16>, dim3(a.total_new, passes < wide ? passes : wide), TJ_THREADS, st, p, grid, W);
  }
  return e == cudaSuccess ? SWIFTKV_OK : report_error(SWIFTKV_ERR_CUDA, cudaGetErrorString(e));
}

template <int HD, bool F16>
int32_t launch_tc_for(const TreeArgs &a, bool fp8, cudaStream_t st) {
  TreeTcArgs p{};
  p.a = a;
  const int rep = a.n_q / a.n_kv;
  // (24 sequences of 10000 keys, 32 rows: 170 us in four copies, 214 us in two, 294 us in one; 64 rows: 222 us in two, 300 us in one)
  const long long rows = (long long)a.max_new * rep;
  p.copies = !fp8 ? 1 : rows <= 32 ? 4 : rows <= 64 ? 2 : 1;
  while (p.copies > 1 && (long long)p.copies * a.total_new > TC_COPY_TOKENS) p.copies /= 2;
  p.npt = 128 / p.copies / rep;
  p.slot_rows = p.copies > 1 ? 128 : tc_slot_rows(a.total_new, a.n_q, a.n_kv);
  p.scale_log2 = a.scale * 1.4426950408889634f;
  p.store32 = ((uintptr_t)a.out & 31) == 0;
  if (fp8) return launch_tc<HD, 1, F16, true>(p, st);
  // more rows than one query tile holds: two tiles share the key tiles of a pass
  return a.max_new > p.npt ? launch_tc<HD, 2, F16, false>(p, st) : launch_tc<HD, 1, F16, false>(p, st);
}

}  // namespace
}  // namespace skv

using namespace skv;

extern "C" size_t swiftkv_tree_attention_scratch_bytes(int32_t total_new, int32_t max_kv, int32_t n_q_heads, int32_t head_dim) {
  if (total_new < 1 || max_kv < 1 || n_q_heads < 1 || head_dim < 1 || head_dim > 256) return 0;
  const size_t simt = simt_scratch(total_new, max_kv, n_q_heads, head_dim);
  if (head_dim != 64 && head_dim != 128) return simt;
  const size_t tcs = tc_scratch(total_new, n_q_heads, head_dim);
  return simt > tcs ? simt : tcs;
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
  if ((uintptr_t)q % es || (uintptr_t)out % es || (uintptr_t)k_cache % kes || (uintptr_t)v_cache % kes || ((uintptr_t)scratch & 255))
    return report_error(SWIFTKV_ERR_INVALID_ARG, "misaligned pointer");
  const size_t need = swiftkv_tree_attention_scratch_bytes(total_new, max_kv, n_q_heads, head_dim);
  if (need && (!scratch || scratch_bytes < need)) return report_error(SWIFTKV_ERR_WORKSPACE_SMALL, "scratch too small (see swiftkv_tree_attention_scratch_bytes)");
  // a query tile is read by every block that has keys for it, also after another has written its rows
  const size_t row = (size_t)n_q_heads * head_dim * es, plane = (size_t)cache_rows * n_kv_heads * head_dim * kes;
  auto part = [](const void *p, size_t bytes) { return ByteRows{p, 1, bytes, bytes}; };
  const ByteRows in[] = {{q, (size_t)total_new, (size_t)q_stride * es, row}, part(k_cache, plane), part(v_cache, plane)};
  const ByteRows outs[] = {part(out, total_new * row), part(lse, lse ? (size_t)total_new * n_q_heads * sizeof(float) : 0), part(scratch, need)};
  for (int i = 0; i < 3; ++i) {
    if (!outs[i].width) continue;
    for (int j = 0; j < 3; ++j)
      if (overlap(outs[i], in[j]) || (j < i && outs[j].width && overlap(outs[i], outs[j])))
        return report_error(SWIFTKV_ERR_INVALID_ARG, "out, lse or scratch overlaps q, the cache or another of them");
  }
  unsigned int *status = op_status_word();
  if (!status) return report_error(SWIFTKV_ERR_CUDA, "no status word");
  // max_kv: lengths rounded up to whole tiles stay inside 32 bits.  max_new: no sequence has more new tokens than there are, so that a limit
  // far above them neither picks the kernel's form nor sizes its grid.
  TreeArgs a{};
  a.q = q; a.q_stride = q_stride; a.k = k_cache; a.v = v_cache; a.k_scale = k_scale; a.v_scale = v_scale;
  a.blk = block_table; a.max_blocks = max_blocks; a.row0 = row0; a.past = n_past; a.cu = cu_new; a.mask = tree_mask; a.mask_words = mask_words;
  a.out = out; a.lse = lse; a.scratch = reinterpret_cast<float *>(scratch);
  a.max_new = max_new < total_new ? max_new : total_new; a.max_kv = max_kv < TREE_MAX_KV ? max_kv : TREE_MAX_KV;
  a.cache_rows = cache_rows; a.n_seqs = n_seqs; a.total_new = total_new; a.n_q = n_q_heads; a.n_kv = n_kv_heads; a.hd = head_dim;
  a.scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)head_dim);
  a.status = status;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (tc_supported(a, q_dtype != SWIFTKV_DTYPE_F32, fp8)) {
    if (q_dtype == SWIFTKV_DTYPE_BF16) return head_dim == 64 ? launch_tc_for<64, false>(a, fp8, st) : launch_tc_for<128, false>(a, fp8, st);
    return head_dim == 64 ? launch_tc_for<64, true>(a, fp8, st) : launch_tc_for<128, true>(a, fp8, st);
  }
  if (fp8) {
    if (q_dtype == SWIFTKV_DTYPE_F32) return launch_simt<float, fp8e4>(a, st);
    if (q_dtype == SWIFTKV_DTYPE_BF16) return launch_simt<bf16, fp8e4>(a, st);
    return launch_simt<__half, fp8e4>(a, st);
  }
  if (q_dtype == SWIFTKV_DTYPE_F32) return launch_simt<float, float>(a, st);
  if (q_dtype == SWIFTKV_DTYPE_BF16) return launch_simt<bf16, bf16>(a, st);
  return launch_simt<__half, __half>(a, st);
}
