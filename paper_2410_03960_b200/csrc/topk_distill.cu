// swiftkv_topk_distill: the divergence of a student's distribution from a teacher's largest log probabilities, and its gradient with respect
// to the student's logits; swiftkv_topk_distill_bwd: the gradient alone.
//
// With the K given tokens and all others as one outcome, q_k = e^(z_k - lse), q_r = e^(lse_r - lse) (lse_r over the others) and the mass P = sum p_k + p_r,
// the gradient is g (P q_k - p_k) / T at the given tokens and g (P q_r - p_r) / T times the others' own softmax e^(z - lse_r) elsewhere -- a
// factor of at most P and a softmax, so nothing overflows where the others have hardly any probability.  P is 1 but where p_r is cut off at 0 or counts as 0, or
// nothing has any probability.  For the same reason the others
// are summed apart: taking the given tokens' exponentials off a sum over everything would leave rounding.  Given tokens are
// blanked in shared memory before a chunk is summed.  What is formed of the K + 1 outcomes is 64-bit: the loss is a small difference of
// logarithms, and p_r = 1 - sum p loses its bits where the teacher is sure.  An error of the others' sum itself enters the loss by
// q_r - p_r only.
//
// Blocks are persistent and stream rows through a ring of 32 KB bulk copies.  One warp feeds the ring and blanks, so that the reading warps need no barrier
// among themselves (4096 rows bf16: 210 us with one per chunk, 178 without); another reads the entries of up to four rows ahead, and a third joins up finished
// rows (where rows are short these two are what a block waits for: 4096 x 1252 bf16 of 100 entries 75 us, 80 with one warp for both; with the gradient 76 and 93).  With the gradient a row is looked at twice: its last three chunks are still in the ring, and the lines of the others are kept in L2
// (evict_last; all else evict_first), so that HBM sees hardly more than one read and one write (581 + 466 MB for 2 x 525; without the hints
// 881 MB are read).  Few rows: a cluster of up to 8 blocks shares a row.
//
// What bounds it: HBM for the loss alone, the exponential units (71 %) close behind for 16-bit logits: 4096 x 128256 bf16 178 - 181 us (5.9 TB/s), 1024 x 128256 fp32
// 81 us (6.5 TB/s).  With the gradient the join between a row's two looks, behind which two blocks per SM hide one another only in part: 2048 x 128256
// bf16 211 - 216 us (5.0 TB/s); the gradient alone 170 us (6.2 TB/s), 1024 x 128256 fp32 174 us.  33 rows fp32 7.7 us.  Tried and slower: rows split over two blocks
// (248 us), one block per SM with twice the ring (239 us), chunks of half the size (233 against 221 us).
#include <cooperative_groups.h>

#include "logits_common.cuh"

namespace skv {
namespace {
namespace cg = cooperative_groups;
using tc::F2;
using tc::add2;
using tc::mul2;

constexpr int TD_MAX_TOP = 128, TD_LANE_TOP = TD_MAX_TOP / 32;
constexpr int TD_MAX_CLUSTER = 8;
constexpr int TD_THREADS = 256, TD_WARPS = TD_THREADS / 32;     // threads that read logits; three more warps feed the ring, read entries, and join rows up
constexpr int TD_ROWS = 4;                   // rows of a block whose entries are known before they are joined up
constexpr int TD_UNROLL = 8;                 // 16-byte vectors of a chunk per thread
constexpr int TD_CHUNK = TD_THREADS * TD_UNROLL;
constexpr int TD_STAGES = 3;                 // chunks of the ring: 96 KB, two blocks share an SM
constexpr int TD_SMEM = TD_STAGES * TD_CHUNK * 16;
// Temperatures: a denormal logit, which counts as 0, must not matter; and a difference of two logits that is not must have no probability
constexpr float TD_COLDEST = 0x1p-64f, TD_HOTTEST = 0x1p100f;
// Others whose sum is below 2^-1000 of the whole are masked ones, by whatever constant: -inf, -1e9, the type's lowest value (whose log sum in fp32 would have
// lost the sum altogether).  They get no probability from the teacher and no gradient.
constexpr double TD_MASKED = 0x1p-1000, TD_MASKED_LOG = 693.14718055994531;

struct TdArgs {
  const void *logits;
  void *out;
  long long stride, out_stride;
  const int32_t *ids;
  const float *logprobs, *g;
  float *loss, *lse, *rest_lse;
  int rows, vocab, k, splits;
  float c;
  double inv_t;
  int rest;
  unsigned int *status;
};

// The gradient is formed of what a program in 32 bits has: of logits / T, a product with 1 / T in fp32, and of the log sums as they are returned.  So the
// operator at T is the operator at 1 on such logits, and the gradient that comes with the loss is that of the gradient's own call, which has no other log
// sums; where q and p nearly cancel at an entry, 64-bit logits in one of them would show.  (From 64 on not: there the rounding would take more than 2^-18.)
__device__ __forceinline__ double td_rounding(float z, double inv_t) {
  const double exact = (double)z * inv_t;
  return fabs(exact) < 64.0 ? (double)(z * (float)inv_t) - exact : 0.0;
}
__device__ __forceinline__ double td_rounding(double x) { return fabs(x) < 64.0 ? (double)(float)x - x : 0.0; }

// The mass P = sum p_k + p_r of entries with the sum p: p_r makes it 1 where there are others for it and p leaves it something, dividing by p where that is not 0
// (a NaN stays).  Log probabilities in fp32 of logits up to 64 are off by 2 x 2^-18, and so is their sum where the teacher is sure: that near to 1 it is 1.  (Of 7500
// drawn fp32 batches two, of one and two rows, had gradients 6e-5 and 3e-4 off without this, in the 2-norm; the others are the same.)
__device__ __forceinline__ double td_mass(double p, int rest, bool some) { return (rest ? (some && p <= 1.0) || fabs(p - 1.0) <= 0x1p-17 : p > 0.0) ? 1.0 : p; }

struct TdPart { float m, l; };               // a set of logits: its maximum, and the sum of 2^((x - m) c)
// One warp's sums over a row's entries: their largest logit (-inf: none), weights relative to it, the teacher's probabilities, sum p (log p - z / T)
struct TdEntries {
  float top;
  double w, p, loss;
  bool any;
};
struct alignas(16) TdRow {                               // what the two kinds of warps tell each other about a row
  int id[TD_MAX_TOP];                        // given tokens, -1: none
  float grad[TD_MAX_TOP];                    // the gradient there
  double w[TD_MAX_TOP], p[TD_MAX_TOP];       // their weights 2^((z - their largest) c), as the gradient takes them, and the teacher's probabilities
  unsigned head, tail;                       // which elements of the row's odd ends are given
  float m, scale;                            // gradient elsewhere: scale 2^((x - m) c)
  TdEntries e;
  int any;                                   // 0: a row whose others have no gradient (no entries, or the others masked)
  TdPart warp[TD_WARPS];
};
struct TdShared {
  TdRow row[TD_ROWS];
  TdPart part[TD_MAX_CLUSTER];               // of the row that a cluster's blocks share (it has one)
  uint64_t full[TD_STAGES], ready[TD_STAGES], empty[TD_STAGES], given[TD_ROWS], weighed[TD_ROWS], summed[TD_ROWS], joined[TD_ROWS], left[TD_ROWS], met;
  int known;                                 // the last row (of the block's, counted) whose tokens are known
};

// bulk_load with what L2 is to do with the lines: keep them for a second look, or let them go first
__device__ __forceinline__ uint64_t keep_policy() {
  uint64_t p;
  asm("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ __forceinline__ uint64_t pass_policy() {
  uint64_t p;
  asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar, uint64_t policy) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar), "l"(policy)
               : "memory");
}

// whether a barrier's phase is over, without waiting
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}

// arrives at block `rank`'s copy of a barrier; what the thread wrote to that block before is seen by who waits there
__device__ __forceinline__ void cluster_arrive(uint32_t bar, uint32_t rank) {
  asm volatile(
      "{\n\t.reg .b32 at;\n\t"
      "mapa.shared::cluster.u32 at, %0, %1;\n\t"
      "mbarrier.arrive.release.cluster.shared::cluster.b64 _, [at];\n\t}"
      ::"r"(bar), "r"(rank)
      : "memory");
}
__device__ __forceinline__ bool cluster_wait(uint32_t bar, uint32_t parity) {
  const long long t0 = clock64();
  while (true) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    if (ok) return true;
    if (clock64() - t0 > tc::WAIT_LIMIT_CLOCKS) return false;
  }
}

// the 16 bytes that begin `bytes` (0 to 15) behind lo's first, hi following lo
__device__ __forceinline__ uint4 shift_16(const uint4 &lo, const uint4 &hi, int bytes) {
  uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
  for (int i = 0; i < 6; ++i) w[i] = bytes & 8 ? w[i + 2] : w[i];
#pragma unroll
  for (int i = 0; i < 5; ++i) w[i] = bytes & 4 ? w[i + 1] : w[i];
  const int s = (bytes & 3) * 8;
  return make_uint4(__funnelshift_r(w[0], w[1], s), __funnelshift_r(w[1], w[2], s), __funnelshift_r(w[2], w[3], s), __funnelshift_r(w[3], w[4], s));
}

// a block's part of a row: elements before the row's first 16-byte boundary (head), whole vectors [v_begin, v_end), elements behind
struct TdSpan { int head, tail0, v_begin, v_end; };
template <typename T>
__device__ __forceinline__ TdSpan td_span(const TdArgs &a, int row, int part) {
  constexpr int N = LpVec<T>::N;
  const uintptr_t at = reinterpret_cast<uintptr_t>(reinterpret_cast<const T *>(a.logits) + (size_t)row * a.stride);
  const int mis = (int)((at & 15) / sizeof(T));
  TdSpan r;
  // (a vocabulary of one warp's size is all head: rows either all have whole vectors or none has)
  r.head = a.vocab <= 32 ? a.vocab : mis ? N - mis : 0;
  const int n_vec = (a.vocab - r.head) / N;
  r.tail0 = r.head + n_vec * N;
  r.v_begin = (int)((long long)n_vec * part / a.splits);
  r.v_end = (int)((long long)n_vec * (part + 1) / a.splits);
  return r;
}

__device__ __forceinline__ TdPart td_warp_join(TdPart t, float c) {
  float m = t.m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (t.m != m && t.l > 0.f) t.l *= exp2_approx((t.m - m) * c);
  t.m = m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t.l += __shfl_xor_sync(0xffffffffu, t.l, o);
  return t;
}
__device__ __forceinline__ double td_warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// A row's entries on their way: a lane's tokens and log probabilities are asked for a row ahead, their logits before the row before is joined up
struct TdLane {
  int id[TD_LANE_TOP];
  float lp[TD_LANE_TOP], z[TD_LANE_TOP];
};
__device__ __forceinline__ void td_ask(TdLane &e, const TdArgs &a, int row) {
#pragma unroll
  for (int i = 0; i < TD_LANE_TOP; ++i) {
    const int k = i * 32 + (threadIdx.x & 31);
    e.id[i] = k < a.k ? a.ids[(size_t)row * a.k + k] : -1;
    e.lp[i] = k < a.k ? a.logprobs[(size_t)row * a.k + k] : 0.f;
  }
}
// The tokens into r, their logits asked for.  Ids that are none, and later ones of the same token, become -1.
template <typename T>
__device__ __forceinline__ void td_tokens(TdLane &l, TdRow &r, const TdArgs &a, int row, bool reports) {
  const int lane = threadIdx.x & 31;
  const T *x = reinterpret_cast<const T *>(a.logits) + (size_t)row * a.stride;
  auto &id = l.id;
  auto &z = l.z;
#pragma unroll
  for (int i = 0; i < TD_LANE_TOP; ++i) {
    z[i] = -INFINITY;
    if (id[i] >= a.vocab && reports) atomicOr(a.status, STATUS_BAD_TOKEN);
    if (id[i] < 0 || id[i] >= a.vocab) id[i] = -1;
    if (id[i] >= 0) z[i] = lp_load(x + id[i]);
    r.id[i * 32 + lane] = id[i];
  }
  __syncwarp();
  // every entry against those before it: of its own 32, and of the earlier ones four at a time from shared memory, where no comparison waits for another
  bool again[TD_LANE_TOP];
#pragma unroll
  for (int i = 0; i < TD_LANE_TOP; ++i) {
    again[i] = false;
    if (i * 32 >= a.k) continue;
    again[i] = (__match_any_sync(0xffffffffu, id[i] >= 0 ? id[i] : -1 - lane) & ((1u << lane) - 1u)) != 0;
    unsigned least[4] = {~0u, ~0u, ~0u, ~0u};              // of what two tokens differ in: 0 if any are the same
#pragma unroll
    for (int s = 0; s < 8 * i; ++s) {
      const int4 other = reinterpret_cast<const int4 *>(r.id)[s];
      least[0] = min(least[0], (unsigned)(other.x ^ id[i]));
      least[1] = min(least[1], (unsigned)(other.y ^ id[i]));
      least[2] = min(least[2], (unsigned)(other.z ^ id[i]));
      least[3] = min(least[3], (unsigned)(other.w ^ id[i]));
    }
    again[i] = again[i] || min(min(least[0], least[1]), min(least[2], least[3])) == 0u;
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < TD_LANE_TOP; ++i) {
    if (!again[i]) continue;
    id[i] = -1;
    r.id[i * 32 + lane] = -1;
  }
}
// The entries' weights and probabilities into r, and their sums
__device__ __forceinline__ TdEntries td_entries(const TdLane &l, TdRow &r, const TdArgs &a) {
  const int lane = threadIdx.x & 31;
  auto &id = l.id;
  auto &lp = l.lp;
  auto &z = l.z;
  TdEntries e{-INFINITY, 0.0, 0.0, 0.0, false};
#pragma unroll
  for (int i = 0; i < TD_LANE_TOP; ++i)
    if (id[i] >= 0) e.top = max_nan(e.top, z[i]);
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) e.top = max_nan(e.top, __shfl_xor_sync(0xffffffffu, e.top, s));
#pragma unroll
  for (int i = 0; i < TD_LANE_TOP; ++i) {
    if (i * 32 >= a.k) continue;
    const bool is = id[i] >= 0, none = !is || z[i] == -INFINITY;
    const double x = exp(none ? 0.0 : ((double)z[i] - (double)e.top) * a.inv_t), p = exp(is ? (double)lp[i] : -(double)INFINITY), w = none ? 0.0 : x;
    r.w[i * 32 + lane] = w * (1.0 + td_rounding(z[i], a.inv_t));
    r.p[i * 32 + lane] = p;
    e.any = e.any || is;
    e.w += w;
    e.p += p;
    if (is && !(p == 0.0)) e.loss += p * ((double)lp[i] - (double)z[i] * a.inv_t);
  }
  e.any = __any_sync(0xffffffffu, e.any);
  e.w = td_warp_sum(e.w);
  e.p = td_warp_sum(e.p);
  e.loss = td_warp_sum(e.loss);
  return e;
}

// one warp: what the others' sum adds to the entries
struct TdOutcome {
  float top;               // the row's largest logit
  double total, rest;      // sum of weights relative to it, and the others'
  double p_r, norm;        // the others' probability, and what the entries' are divided by
  double mass;             // what all outcomes have together
  double f;                // the entries' weights are relative to their own largest: times this
  bool some;               // there are others that are not masked
};
__device__ __forceinline__ TdOutcome td_outcome(const TdEntries &e, const TdPart &others, const TdArgs &a) {
  TdOutcome o;
  o.top = max_nan(e.top, others.m);
  const bool none = others.m == -INFINITY;           // (a NaN counts)
  // (one exponential for both: even lanes the entries', odd lanes the others')
  const bool odd = threadIdx.x & 1;
  const float m = odd ? others.m : e.top;
  const double f = m == -INFINITY && o.top != -INFINITY ? 0.0 : exp(((double)m - (double)o.top) * a.inv_t);
  const double fe = __shfl_sync(0xffffffffu, f, 0), fr = __shfl_sync(0xffffffffu, f, 1);
  o.rest = none ? 0.0 : (double)others.l * fr;
  o.f = fe;
  o.total = e.w * fe + o.rest;
  o.some = !none && !(o.rest < o.total * TD_MASKED);
  o.p_r = a.rest && o.some ? fmax(1.0 - e.p, 0.0) : 0.0;
  o.norm = a.rest || !(e.p > 0.0) ? 1.0 : e.p;
  o.mass = td_mass(e.p, a.rest, o.some);
  return o;
}

// A walk over the chunks that a block's ring holds one after the other: of every row its vectors [begin, end) in chunks and, GRAD, once more those that the ring
// no longer holds when the last has come (the first n - STAGES)
template <typename T, bool GRAD>
struct TdWalk {
  const TdArgs &a;
  int row, step, part, begin, end, v, upto, turn, stage = 0, use = 0;
  bool again;                                              // the second look
  __device__ __forceinline__ TdWalk(const TdArgs &args, int row0, int row_step, int p) : a(args), row(row0 - row_step), step(row_step), part(p), turn(-1) { open(); }
  __device__ __forceinline__ void open() {                 // the next row that has whole vectors
    do {
      row += step;
      ++turn;
      if (row >= a.rows) return;
      const TdSpan s = td_span<T>(a, row, part);
      begin = s.v_begin;
      end = s.v_end;
    } while (begin >= end);
    v = begin;
    upto = end;
    again = false;
  }
  __device__ __forceinline__ bool more() const { return row < a.rows; }
  __device__ __forceinline__ static int kept(int begin, int end) {      // the first vector that the ring still holds when the row's last chunk is there
    return begin + max(0, (end - begin + TD_CHUNK - 1) / TD_CHUNK - TD_STAGES) * TD_CHUNK;
  }
  __device__ __forceinline__ void advance() {
    if (++stage == TD_STAGES) { stage = 0; ++use; }
    v += TD_CHUNK;
    if (v < upto) return;
    if (GRAD && !again && kept(begin, end) > begin) {
      again = true;
      v = begin;
      upto = kept(begin, end);
    } else {
      open();
    }
  }
};

template <typename T, bool GRAD>
__global__ void __launch_bounds__(TD_THREADS + 96, 2) topk_distill_kernel(const __grid_constant__ TdArgs a) {
  constexpr int N = LpVec<T>::N;
  using Walk = TdWalk<T, GRAD>;
  __shared__ TdShared sh;
  extern __shared__ __align__(128) uint8_t td_ring[];      // [TD_STAGES][TD_CHUNK] vectors
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int part = blockIdx.x % a.splits, row0 = blockIdx.x / a.splits, row_step = gridDim.x / a.splits;
  const float c = a.c;
  if (tid == 0) {
    for (int i = 0; i < TD_STAGES; ++i) {
      tc::mbar_init(tc::smem_u32(&sh.full[i]), 1);
      tc::mbar_init(tc::smem_u32(&sh.ready[i]), 1);
      tc::mbar_init(tc::smem_u32(&sh.empty[i]), TD_WARPS);
    }
    sh.known = -1;
    tc::mbar_init(tc::smem_u32(&sh.met), a.splits);
    for (int i = 0; i < TD_ROWS; ++i) {
      tc::mbar_init(tc::smem_u32(&sh.given[i]), 1);
      tc::mbar_init(tc::smem_u32(&sh.weighed[i]), 1);
      tc::mbar_init(tc::smem_u32(&sh.summed[i]), TD_WARPS);
      tc::mbar_init(tc::smem_u32(&sh.joined[i]), 1);
      tc::mbar_init(tc::smem_u32(&sh.left[i]), TD_WARPS);
    }
    tc::fence_barrier_init();
  }
  __syncthreads();
  bool alive = true;            // a wait that ran out (never, unless something is broken): no further waits or copies
  auto wait = [&](uint64_t *bar, uint32_t parity) {
    if (alive && !tc::mbar_wait(tc::smem_u32(bar), parity)) {
      alive = false;
      atomicOr(a.status, STATUS_TIMEOUT);
    }
  };
  if (a.splits > 1) cg::this_cluster().sync();             // the cluster's blocks are there
  if (warp == TD_WARPS) {
    // ---- the warp that feeds the ring: copies into stages that are empty, given tokens blanked in chunks that have come
    Walk in(a, row0, row_step, part), out(a, row0, row_step, part);
    int copied = 0, blanked = 0, turn = -1;
    int id[TD_LANE_TOP];
    TdSpan span{};
    const uint64_t keep = keep_policy(), pass = pass_policy();
    long long since = clock64();
    while (out.more() && alive) {
      bool moved = false;
      if (in.more() && copied < blanked + TD_STAGES && (in.use == 0 || __shfl_sync(0xffffffffu, (int)mbar_test(tc::smem_u32(&sh.empty[in.stage]), (in.use - 1) & 1), 0))) {
        if (lane == 0) {
          const uint32_t bar = tc::smem_u32(&sh.full[in.stage]), bytes = (uint32_t)min(TD_CHUNK, in.upto - in.v) * 16;
          const T *x = reinterpret_cast<const T *>(a.logits) + (size_t)in.row * a.stride + td_span<T>(a, in.row, part).head;
          tc::mbar_expect_tx(bar, bytes);
          bulk_load(tc::smem_u32(td_ring) + in.stage * TD_CHUNK * 16, reinterpret_cast<const uint4 *>(x) + in.v, bytes, bar,
                    GRAD && !in.again && in.v < Walk::kept(in.begin, in.end) ? keep : pass);
        }
        ++copied;
        in.advance();
        moved = true;
      }
      // (rows without whole vectors are passed over here, so that it takes a count to know that a row's tokens are there, not a barrier's parity)
      if (blanked < copied && (turn == out.turn || __shfl_sync(0xffffffffu, *const_cast<volatile int *>(&sh.known), 0) >= out.turn) &&
          __shfl_sync(0xffffffffu, (int)mbar_test(tc::smem_u32(&sh.full[out.stage]), out.use & 1), 0)) {
        if (!out.again) {
          if (turn != out.turn) {                          // the row's entries
            turn = out.turn;
            __threadfence_block();
            span = td_span<T>(a, out.row, part);
#pragma unroll
            for (int i = 0; i < TD_LANE_TOP; ++i) id[i] = sh.row[turn % TD_ROWS].id[i * 32 + lane];
          }
          uint8_t *const stage = td_ring + (size_t)out.stage * TD_CHUNK * 16;
          const int e0 = span.head + out.v * N, n = min(TD_CHUNK, out.upto - out.v) * N;
          bool blank = false;
#pragma unroll
          for (int i = 0; i < TD_LANE_TOP; ++i) {
            const int at = id[i] - e0;
            if (id[i] < 0 || at < 0 || at >= n) continue;
            if (sizeof(T) == 4) reinterpret_cast<uint32_t *>(stage)[at] = no_logits<T>();
            else reinterpret_cast<uint16_t *>(stage)[at] = (uint16_t)no_logits<T>();
            blank = true;
          }
          if (blank) tc::fence_proxy_async_smem();         // (the stage is written by a bulk copy next; once: it costs more than all else here)
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(tc::smem_u32(&sh.ready[out.stage]));
        ++blanked;
        out.advance();
        moved = true;
      }
      if (moved) {
        since = clock64();
      } else if (__any_sync(0xffffffffu, clock64() - since > tc::WAIT_LIMIT_CLOCKS)) {
        alive = false;
        if (lane == 0) atomicOr(a.status, STATUS_TIMEOUT);
      } else {
        __nanosleep(40);                                   // (leaves the issue slots to the others)
      }
    }
    // giving up: copies under way land before the ring is given back (these waits are bounded too)
    if (!alive)
      for (int i = max(0, copied - TD_STAGES); i < copied; ++i) tc::mbar_wait(tc::smem_u32(&sh.full[i % TD_STAGES]), (i / TD_STAGES) & 1);
    return;
  }
  if (warp == TD_WARPS + 1) {
    // ---- the warp of the entries
    TdLane now, next{};
    if (row0 < a.rows) td_ask(next, a, row0);
    for (int row = row0, turn = 0; row < a.rows; row += row_step, ++turn) {
      const int par = turn % TD_ROWS;
      TdRow &r = sh.row[par];
      now = next;
      if (row + row_step < a.rows) td_ask(next, a, row + row_step);
      if (turn >= TD_ROWS) wait(GRAD ? &sh.left[par] : &sh.joined[par], (turn / TD_ROWS - 1) & 1);
      alive = __all_sync(0xffffffffu, alive);
      td_tokens<T>(now, r, a, row, part == 0);
      const TdSpan s = td_span<T>(a, row, part);
      unsigned head = 0, tail = 0;
#pragma unroll
      for (int i = 0; i < TD_LANE_TOP; ++i) {
        const int id = now.id[i];
        if (id >= 0 && id < s.head) head |= 1u << id;
        if (id >= s.tail0) tail |= 1u << (id - s.tail0);
      }
      head = __reduce_or_sync(0xffffffffu, head);
      tail = __reduce_or_sync(0xffffffffu, tail);
      if (lane == 0) {
        r.head = head;
        r.tail = tail;
      }
      __syncwarp();
      if (lane == 0) {
        __threadfence_block();
        *const_cast<volatile int *>(&sh.known) = turn;
        tc::mbar_arrive(tc::smem_u32(&sh.given[par]));
      }
      const TdEntries e = td_entries(now, r, a);
      if (lane == 0) r.e = e;
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(tc::smem_u32(&sh.weighed[par]));
    }
    return;
  }
  if (warp == TD_WARPS + 2) {
    // ---- the warp that joins rows up
    for (int row = row0, turn = 0; row < a.rows; row += row_step, ++turn) {
      const int par = turn % TD_ROWS;
      TdRow &r = sh.row[par];
      const float g = GRAD ? a.g[row] : 0.f;
      wait(&sh.weighed[par], (turn / TD_ROWS) & 1);
      wait(&sh.summed[par], (turn / TD_ROWS) & 1);
      alive = __all_sync(0xffffffffu, alive);
      const TdEntries now = r.e;
      TdPart all = td_warp_join(lane < TD_WARPS ? r.warp[lane] : TdPart{-INFINITY, 0.f}, c);
      if (a.splits > 1) {
        // to every block of the cluster; each waits for all
        if (lane < a.splits) {
          TdShared *const peer = cg::this_cluster().map_shared_rank(&sh, lane);
          peer->part[part] = all;
          cluster_arrive(tc::smem_u32(&sh.met), lane);
        }
        __syncwarp();
        if (alive && !cluster_wait(tc::smem_u32(&sh.met), 0)) {
          alive = false;
          atomicOr(a.status, STATUS_TIMEOUT);
        }
        alive = __all_sync(0xffffffffu, alive);
        all = td_warp_join(lane < a.splits ? sh.part[lane] : TdPart{-INFINITY, 0.f}, c);
      }
      const TdOutcome o = td_outcome(now, all, a);
      // (one logarithm for all)
      const double x = lane == 0 ? o.total : lane == 1 ? (double)all.l : lane == 2 ? o.p_r : o.norm, log_x = log(x);
      const double lse = (double)o.top * a.inv_t + __shfl_sync(0xffffffffu, log_x, 0), log_r = __shfl_sync(0xffffffffu, log_x, 2), log_norm = __shfl_sync(0xffffffffu, log_x, 3);
      const double rest_lse = all.m == -INFINITY ? -INFINITY : (double)all.m * a.inv_t + __shfl_sync(0xffffffffu, log_x, 1);
      if (GRAD) {
        const double off = -td_rounding(lse), off_r = -td_rounding(rest_lse);      // (so small that 1 + off is e^off)
        const double of_w = o.mass * o.f / o.total * (1.0 + off), of_p = 1.0 / o.norm;
#pragma unroll
        for (int i = 0; i < TD_LANE_TOP; ++i) {
          const int k = i * 32 + lane;
          if (r.id[k] >= 0) r.grad[k] = (float)((double)g * (r.w[k] * of_w - r.p[k] * of_p) * a.inv_t);
        }
        if (lane == 0) {
          r.m = all.m;
          r.scale = (float)((double)g * (o.mass * o.rest / o.total * (1.0 + off - off_r) - o.p_r) * a.inv_t / (double)all.l * (1.0 + off_r));
          r.any = now.any && o.some;                       // (others that are masked may be finite and large: an exponential of theirs is not formed)
        }
      }
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(tc::smem_u32(&sh.joined[par]));
      if (part == 0) {
        double loss = now.loss / o.norm + now.p / o.norm * (lse - log_norm);
        if (o.p_r > 0.0) loss += o.p_r * (log_r - (rest_lse - lse));
        if (!(o.total == o.total)) loss = o.total;           // (a NaN or +inf among the logits)
        if (lane == 0) {
          a.loss[row] = now.any ? (float)loss : 0.f;
          a.lse[row] = now.any ? (float)lse : 0.f;
          a.rest_lse[row] = now.any ? (float)rest_lse : 0.f;
        }
      }
    }
    return;
  }
  // ---- the others.  The ring's chunk `count` is the next one to come.
  int stage = 0, use = 0, turn = 0;
  auto come = [&]() {
    wait(&sh.full[stage], use & 1);
    wait(&sh.ready[stage], use & 1);
  };
  auto release = [&](int st) {
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(tc::smem_u32(&sh.empty[st]));
  };
  auto step = [&]() {
    if (++stage == TD_STAGES) { stage = 0; ++use; }
  };
  for (int row = row0; row < a.rows; row += row_step, ++turn) {
    const int par = turn % TD_ROWS;
    TdRow &r = sh.row[par];
    const T *x = reinterpret_cast<const T *>(a.logits) + (size_t)row * a.stride;
    const TdSpan s = td_span<T>(a, row, part);
    const int kept = GRAD ? Walk::kept(s.v_begin, s.v_end) : s.v_end;      // chunks from here on stay in the ring for the second look
    // a row's odd ends: a warp of the first / last part takes them
    const int edge = part == 0 && warp == 0 && lane < s.head ? lane
                     : part == a.splits - 1 && warp == TD_WARPS - 1 && lane < a.vocab - s.tail0 ? s.tail0 + lane : -1;
    const float edge_v = edge >= 0 ? lp_load(x + edge) : -INFINITY;
    float m = -INFINITY;
    F2 l{{0.f, 0.f}};
    for (int v0 = s.v_begin; v0 < s.v_end; v0 += TD_CHUNK) {
      come();
      const uint4 *chunk = reinterpret_cast<const uint4 *>(td_ring) + stage * TD_CHUNK + tid;
      uint4 raw[TD_UNROLL];
#pragma unroll
      for (int u = 0; u < TD_UNROLL; ++u) raw[u] = chunk[u * TD_THREADS];
      if (v0 < kept) release(stage);
      step();
      if (v0 + TD_CHUNK > s.v_end) {
        const uint32_t none = no_logits<T>();
#pragma unroll
        for (int u = 0; u < TD_UNROLL; ++u)
          if (v0 + u * TD_THREADS + tid >= s.v_end) raw[u] = make_uint4(none, none, none, none);
      }
      const float vmax = chunk_max(raw, (const T *)nullptr);
      if (!(vmax <= m) && m == m) {
        const float f = m != -INFINITY ? exp2_approx((m - vmax) * c) : 0.f;
        l = mul2(l, F2{{f, f}});
        m = vmax;
      }
      if (m != -INFINITY) {
        F2 sum{{0.f, 0.f}};
#pragma unroll
        for (int u = 0; u < TD_UNROLL; ++u) {
          float e[N];
          LpVec<T>::unpack(raw[u], e);
#pragma unroll
          for (int i = 0; i < N; i += 2) {
            F2 d = mul2(add2(F2{{e[i], e[i + 1]}}, F2{{-m, -m}}), F2{{c, c}});
            d.f[0] = exp2_approx(d.f[0]);
            d.f[1] = exp2_approx(d.f[1]);
            sum = add2(sum, d);
          }
        }
        l = add2(l, sum);
      }
    }
    wait(&sh.given[par], (turn / TD_ROWS) & 1);
    const bool edge_given = edge >= 0 && ((edge < s.head ? r.head >> edge : r.tail >> (edge - s.tail0)) & 1u);
    TdPart mine_l{m, l.f[0] + l.f[1]};
    if (edge >= 0 && !edge_given && edge_v != -INFINITY) {
      const float top = max_nan(m, edge_v);
      mine_l.l = (m != -INFINITY ? mine_l.l * exp2_approx((m - top) * c) : 0.f) + exp2_approx((edge_v - top) * c);
      mine_l.m = top;
    }
    const TdPart t = td_warp_join(mine_l, c);
    if (lane == 0) r.warp[warp] = t;
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(tc::smem_u32(&sh.summed[par]));
    if (GRAD) {
      // ---- the row once more: first the chunks that are still there
      T *y = reinterpret_cast<T *>(a.out) + (size_t)row * a.out_stride;
      const int given = tid < a.k ? r.id[tid] : -1;
      wait(&sh.joined[par], (turn / TD_ROWS) & 1);
      // (nothing for the others: as if their logits were 0, whatever they are, times 0)
      const bool any = r.any != 0;
      const float top = any ? r.m : 0.f, scale = any ? r.scale : 0.f;
      const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
      // elements of the row's vectors before the output's first 16-byte boundary
      const int over = (int)((reinterpret_cast<uintptr_t>(y + s.head) & 15) / sizeof(T)), ahead = over ? N - over : 0;
      auto slope = [&](float v) { return any ? scale * exp2_approx((v - top) * c) : 0.f; };
      if (edge >= 0) lp_store(y + edge, slope(edge_v));
      auto slopes = [&](const uint4 &raw) {
        float e[N];
        LpVec<T>::unpack(any ? raw : zero, e);
#pragma unroll
        for (int i = 0; i < N; i += 2) {
          F2 d = mul2(add2(F2{{e[i], e[i + 1]}}, F2{{-top, -top}}), F2{{c, c}});
          d.f[0] = exp2_approx(d.f[0]);
          d.f[1] = exp2_approx(d.f[1]);
          d = mul2(d, F2{{scale, scale}});
          e[i] = d.f[0];
          e[i + 1] = d.f[1];
        }
        return LpVec<T>::pack(e);
      };
      auto write = [&](int v0, int st) {
        const uint4 *chunk = reinterpret_cast<const uint4 *>(td_ring) + st * TD_CHUNK;
        const int vectors = min(TD_CHUNK, s.v_end - v0);
        T *to = y + s.head + (size_t)v0 * N;
        if (ahead == 0) {
#pragma unroll
          for (int u = 0; u < TD_UNROLL; ++u) {
            const int v = u * TD_THREADS + tid;
            if (v < vectors) __stcs(reinterpret_cast<uint4 *>(to) + v, slopes(chunk[v]));
          }
        } else {                                           // vectors of the output lie across two of the input's
          const int left = vectors * N - ahead, whole = left / N, behind = left % N;
          if (tid < ahead) lp_store(to + tid, slope(lp_load(reinterpret_cast<const T *>(chunk) + tid)));
          if (tid < behind) lp_store(to + ahead + whole * N + tid, slope(lp_load(reinterpret_cast<const T *>(chunk) + ahead + whole * N + tid)));
          for (int v = tid; v < whole; v += TD_THREADS) __stcs(reinterpret_cast<uint4 *>(to + ahead) + v, slopes(shift_16(chunk[v], chunk[v + 1], ahead * (int)sizeof(T))));
        }
        release(st);
      };
      {
        int st = stage - (s.v_end - kept + TD_CHUNK - 1) / TD_CHUNK;
        if (st < 0) st += TD_STAGES;
        for (int v0 = kept; v0 < s.v_end; v0 += TD_CHUNK) {
          write(v0, st);
          if (++st == TD_STAGES) st = 0;
        }
      }
      for (int v0 = s.v_begin; v0 < kept; v0 += TD_CHUNK) {
        come();
        write(v0, stage);
        step();
      }
      asm volatile("bar.sync 1, %0;" ::"n"(TD_THREADS) : "memory");
      const int e0 = part == 0 ? 0 : s.head + s.v_begin * N, e1 = part == a.splits - 1 ? a.vocab : s.head + s.v_end * N;
      if (given >= e0 && given < e1) lp_store(y + given, r.grad[tid]);
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(tc::smem_u32(&sh.left[par]));
    }
  }
}

// The gradient alone: elementwise, one read and one write, vectors on the output's 16-byte boundaries.  EVEN: these are the input's too.  2048 x 128256 bf16 170 us
// (6.2 TB/s; 212 us with the loads behind the entries and half the work per block); 1000 x 100001 with other strides 80 us, 69 us where rows are even
constexpr int TB_THREADS = 256, TB_UNROLL = 8;
struct TdBwdArgs {
  TdArgs a;
  const float *lse, *rest_lse;
  int blocks_per_row;
};
template <typename T, bool EVEN>
__global__ void __launch_bounds__(TB_THREADS) topk_distill_bwd_kernel(TdBwdArgs b) {
  constexpr int N = LpVec<T>::N, UNROLL = EVEN ? TB_UNROLL : TB_UNROLL / 2;
  __shared__ int s_id[TD_MAX_TOP];
  __shared__ double s_p[TD_MAX_TOP / 32];
  __shared__ double s_mass;                                // (a register that the vectors need)
  const TdArgs &a = b.a;
  const int tid = threadIdx.x, lane = tid & 31;
  const int row = blockIdx.x / b.blocks_per_row, part = blockIdx.x % b.blocks_per_row;
  const T *x = reinterpret_cast<const T *>(a.logits) + (size_t)row * a.stride;
  T *y = reinterpret_cast<T *>(a.out) + (size_t)row * a.out_stride;
  const int mis = (int)((reinterpret_cast<uintptr_t>(y) & 15) / sizeof(T));
  int head = min(a.vocab, mis ? N - mis : 0), n_vec = (a.vocab - head) / N;
  const int off = EVEN ? 0 : (int)(reinterpret_cast<uintptr_t>(x + head) & 15);      // bytes
  if (!EVEN) {           // a vector is read as two aligned ones; the first and the last, where those would reach beyond the row, go to its odd ends
    if (n_vec > 0 && head * (int)sizeof(T) < off) { head += N; --n_vec; }
    if (n_vec > 0 && (a.vocab - head - n_vec * N) * (int)sizeof(T) < 16 - off) --n_vec;
  }
  const int tail0 = head + n_vec * N;
  const int v_begin = (int)((long long)n_vec * part / b.blocks_per_row), v_end = (int)((long long)n_vec * (part + 1) / b.blocks_per_row);
  const int e0 = part == 0 ? 0 : head + v_begin * N, e1 = part == b.blocks_per_row - 1 ? a.vocab : head + v_end * N;
  // the first vectors are on their way while the entries are looked at.  Not EVEN: a vector's bytes lie in the aligned one of its lane and in that of the next
  // lane (for which the lane behind the last one reads, too); the last lane of a warp reads both.
  const uint4 *const from = reinterpret_cast<const uint4 *>(reinterpret_cast<const uint8_t *>(x + head) - off);
  uint4 raw[UNROLL], last[UNROLL];
  auto load = [&](int v0) {
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int v = v0 + u * TB_THREADS;
      if (EVEN ? v < v_end : v <= v_end && v_begin < v_end) raw[u] = __ldcs(from + v);
      if (!EVEN && lane == 31 && v < v_end) last[u] = __ldcs(from + v + 1);
    }
  };
  load(v_begin + tid);
  // ---- the entries: every block of a row needs the sum of their probabilities, and sets the gradients that lie in its part
  int id = tid < a.k ? a.ids[(size_t)row * a.k + tid] : -1;
  const float lse = b.lse[row], rest_lse = b.rest_lse[row], g = a.g[row];
  double p = 0.0;
  float z = 0.f;
  if (tid < TD_MAX_TOP) {
    if (id >= a.vocab) {
      if (part == 0) atomicOr(a.status, STATUS_BAD_TOKEN);
      id = -1;
    }
    if (id >= 0) p = exp((double)a.logprobs[(size_t)row * a.k + tid]);
    if (id >= e0 && id < e1) z = lp_load(x + id);
    const unsigned same = __match_any_sync(0xffffffffu, id >= 0 ? id : -1 - lane);
    if (same & ((1u << lane) - 1u)) id = -1;               // of two entries with one token the first counts
    s_id[tid] = id;
  }
  __syncthreads();
  if (tid < TD_MAX_TOP) {
    for (int k = 0; id >= 0 && k < (tid & ~31); ++k)
      if (s_id[k] == id) id = -1;
    if (id < 0) p = 0.0;
    const double sum = td_warp_sum(p);
    if (lane == 0) s_p[tid >> 5] = sum;
  }
  const bool any = __syncthreads_or(id >= 0);              // (and every entry's logit has been read before any gradient is written)
  double all_p = 0.0;
#pragma unroll
  for (int w = 0; w < TD_MAX_TOP / 32; ++w) all_p += s_p[w];
  const bool some = rest_lse != -INFINITY && !((double)rest_lse < (double)lse - TD_MASKED_LOG);      // (a NaN counts)
  const double p_r = a.rest && some ? fmax(1.0 - all_p, 0.0) : 0.0, norm = a.rest || !(all_p > 0.0) ? 1.0 : all_p, mass = td_mass(all_p, a.rest, some);
  if (tid == 0) s_mass = mass;
  const float scale = some ? (float)((double)g * (mass * exp((double)rest_lse - (double)lse) - p_r) * a.inv_t) : 0.f;
  const float c = (float)(1.4426950408889634 * a.inv_t);
  // No term of a softmax is above 1: a reference that does not resolve that (from 2^18 on: exponents off by 3 x 2^-6) is raised by what rest_lse, it and c may be rounded by
  const float near_ref = (float)(1.4426950408889634 * (double)rest_lse), ref = fabsf(near_ref) > 0x1p18f ? near_ref + fabsf(near_ref) * 0x1p-22f : near_ref;
  const bool sloped = any && some;                         // (no entries, or others that are masked, be they finite and large: 0)
  auto slope = [&](float v) { return sloped ? scale * exp2_approx(fmaf(v, c, -ref)) : 0.f; };
  if (part == 0 && tid < head) lp_store(y + tid, slope(lp_load(x + tid)));
  if (part == b.blocks_per_row - 1 && tail0 + tid < a.vocab) lp_store(y + tail0 + tid, slope(lp_load(x + tail0 + tid)));
  for (int v0 = v_begin + tid; v0 - lane < v_end; v0 += TB_THREADS * UNROLL) {      // (the warp's lanes stay together)
    if (v0 >= v_begin + TB_THREADS) load(v0);
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int v = v0 + u * TB_THREADS;
      if (!EVEN) {
        uint4 hi = make_uint4(__shfl_down_sync(0xffffffffu, raw[u].x, 1), __shfl_down_sync(0xffffffffu, raw[u].y, 1), __shfl_down_sync(0xffffffffu, raw[u].z, 1),
                              __shfl_down_sync(0xffffffffu, raw[u].w, 1));
        if (lane == 31) hi = last[u];
        raw[u] = shift_16(raw[u], hi, off);
      }
      if (v >= v_end) continue;
      float e[N];
      LpVec<T>::unpack(raw[u], e);
#pragma unroll
      for (int i = 0; i < N; ++i) e[i] = slope(e[i]);
      __stcs(reinterpret_cast<uint4 *>(y + head) + v, LpVec<T>::pack(e));
    }
  }
  __syncthreads();
  if (id >= e0 && id < e1) {
    const double t = (double)z * a.inv_t + td_rounding(z, a.inv_t) - (double)lse;
    const bool above = __double2hiint(t) >= 0x3f900000 && __double2hiint(t) <= 0x7ff00000;      // (2^-6 to infinity: an entry's likewise; what is less is the rounding of an ordinary lse)
    lp_store(y + id, (float)((double)g * (s_mass * exp(above ? 0.0 : t) - p / norm) * a.inv_t));
  }
}

template <typename T, bool GRAD>
cudaError_t launch_distill(const TdArgs &a, cudaStream_t st) {
  // persistent where rows are not split: two blocks fit an SM
  const int blocks = a.splits > 1 ? a.rows * a.splits : a.rows < 2 * num_sms() ? a.rows : 2 * num_sms();
  if (ensure_dynamic_smem(reinterpret_cast<const void *>(topk_distill_kernel<T, GRAD>), TD_SMEM)) return cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.dynamicSmemBytes = TD_SMEM;
  cfg.blockDim = dim3(TD_THREADS + 96);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)a.splits;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, topk_distill_kernel<T, GRAD>, a);
}
template <typename T>
cudaError_t launch_distill(const TdArgs &a, cudaStream_t st) { return a.out ? launch_distill<T, true>(a, st) : launch_distill<T, false>(a, st); }
template <typename T>
cudaError_t launch_distill_bwd(const TdBwdArgs &b, cudaStream_t st) {
  const unsigned grid = (unsigned)((long long)b.a.rows * b.blocks_per_row);
  const int common = common_alignment(b.a.logits, b.a.stride, b.a.out, b.a.out_stride, b.a.rows, sizeof(T));
  if (common >= 16) topk_distill_bwd_kernel<T, true><<<grid, TB_THREADS, 0, st>>>(b);
  else topk_distill_bwd_kernel<T, false><<<grid, TB_THREADS, 0, st>>>(b);
  return cudaGetLastError();
}

size_t element_bytes(int32_t dtype) { return dtype == SWIFTKV_DTYPE_F32 ? 4 : 2; }

// arguments that both calls have; the gradient may lie on the logits themselves
int32_t check_distill(const void *logits, int64_t row_stride, int32_t dtype, const int32_t *top_ids, const float *top_logprobs, int32_t rows, int32_t vocab, int32_t top_k,
                      double temperature, const float *grad_loss, const void *grad_logits, int64_t grad_stride) {
  if (!logits || !top_ids || !top_logprobs) return report_error(SWIFTKV_ERR_INVALID_ARG, "null argument");
  if (dtype != SWIFTKV_DTYPE_F32 && dtype != SWIFTKV_DTYPE_BF16 && dtype != SWIFTKV_DTYPE_F16) return report_error(SWIFTKV_ERR_INVALID_ARG, "unknown dtype");
  // (the kernels count a row's elements in 32 bits, in steps of a block's work)
  if (rows < 1 || rows > (1 << 26) || vocab < 1 || vocab > (1 << 30) || row_stride < vocab)
    return report_error(SWIFTKV_ERR_INVALID_ARG, "bad shape (rows in [1, 2^26], vocab in [1, 2^30], row_stride >= vocab)");
  if (top_k < 1 || top_k > TD_MAX_TOP) return report_error(SWIFTKV_ERR_INVALID_ARG, "top_k outside [1, 128]");
  if (!(temperature >= TD_COLDEST && temperature <= TD_HOTTEST)) return report_error(SWIFTKV_ERR_INVALID_ARG, "temperature must be in [2^-64, 2^100]");
  const size_t es = element_bytes(dtype);
  if (reinterpret_cast<uintptr_t>(logits) % es) return report_error(SWIFTKV_ERR_INVALID_ARG, "misaligned logits");
  if (!grad_logits != !grad_loss) return report_error(SWIFTKV_ERR_INVALID_ARG, "grad_loss and grad_logits go together");
  if (!grad_logits) return SWIFTKV_OK;
  if (grad_stride < vocab) return report_error(SWIFTKV_ERR_INVALID_ARG, "bad shape (grad_stride >= vocab)");
  if (reinterpret_cast<uintptr_t>(grad_logits) % es) return report_error(SWIFTKV_ERR_INVALID_ARG, "misaligned gradient");
  return SWIFTKV_OK;
}
ByteRows words(const void *p, size_t n) { return ByteRows{p, 1, n * 4, n * 4}; }

}  // namespace
}  // namespace skv

using namespace skv;

extern "C" int32_t swiftkv_topk_distill(const void *logits, int64_t row_stride, int32_t dtype, const int32_t *top_ids, const float *top_logprobs,
                                        int32_t rows, int32_t vocab, int32_t top_k, double temperature, int32_t rest, float *loss, float *lse,
                                        float *rest_lse, const float *grad_loss, void *grad_logits, int64_t grad_stride, void *cuda_stream) {
  if (const int32_t rc = check_distill(logits, row_stride, dtype, top_ids, top_logprobs, rows, vocab, top_k, temperature, grad_loss, grad_logits, grad_stride)) return rc;
  if (!loss || !lse || !rest_lse) return report_error(SWIFTKV_ERR_INVALID_ARG, "null argument");
  const size_t es = element_bytes(dtype), n = (size_t)rows;
  const ByteRows x{logits, n, (size_t)row_stride * es, (size_t)vocab * es}, y{grad_logits, n, (size_t)grad_stride * es, (size_t)vocab * es};
  const ByteRows in[] = {words(top_ids, n * top_k), words(top_logprobs, n * top_k), words(grad_loss, n), x};
  const ByteRows out[] = {words(loss, n), words(lse, n), words(rest_lse, n), y};
  for (int i = 0; i < 4; ++i) {
    if (!out[i].p) continue;
    for (int j = 0; j < 4; ++j)
      if (in[j].p && overlap(out[i], in[j]) && !(i == 3 && j == 3 && logits == grad_logits && row_stride == grad_stride))
        return report_error(SWIFTKV_ERR_INVALID_ARG, "an output overlaps an input (other than the gradient in place)");
    for (int j = 0; j < i; ++j)
      if (overlap(out[i], out[j])) return report_error(SWIFTKV_ERR_INVALID_ARG, "two outputs overlap");
  }
  unsigned int *status = op_status_word();
  if (!status) return report_error(SWIFTKV_ERR_CUDA, "no status word");
  // a row is split as far as all blocks run at once (two fit an SM) and every part keeps thousands of logits
  int splits = 1;
  while (splits < TD_MAX_CLUSTER && (long long)rows * splits * 2 <= 2 * num_sms() && vocab / (2 * splits) >= 4096) splits *= 2;
  TdArgs a{logits, grad_logits, row_stride, grad_stride, top_ids, top_logprobs, grad_loss, loss, lse, rest_lse, rows, vocab, top_k, splits,
           (float)(1.4426950408889634 / temperature), 1.0 / temperature, rest, status};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = dtype == SWIFTKV_DTYPE_F32 ? launch_distill<float>(a, st) : dtype == SWIFTKV_DTYPE_BF16 ? launch_distill<bf16>(a, st) : launch_distill<__half>(a, st);
  if (e != cudaSuccess) return report_error(SWIFTKV_ERR_CUDA, cudaGetErrorString(e));
  return SWIFTKV_OK;
}

extern "C" int32_t swiftkv_topk_distill_bwd(const void *logits, int64_t row_stride, int32_t dtype, const int32_t *top_ids, const float *top_logprobs,
                                            int32_t rows, int32_t vocab, int32_t top_k, double temperature, int32_t rest, const float *lse,
                                            const float *rest_lse, const float *grad_loss, void *grad_logits, int64_t grad_stride,
                                            void *cuda_stream) {
  if (!lse || !rest_lse || !grad_loss || !grad_logits) return report_error(SWIFTKV_ERR_INVALID_ARG, "null argument");
  if (const int32_t rc = check_distill(logits, row_stride, dtype, top_ids, top_logprobs, rows, vocab, top_k, temperature, grad_loss, grad_logits, grad_stride)) return rc;
  const size_t es = element_bytes(dtype), n = (size_t)rows;
  const ByteRows x{logits, n, (size_t)row_stride * es, (size_t)vocab * es}, y{grad_logits, n, (size_t)grad_stride * es, (size_t)vocab * es};
  for (const ByteRows &r : {words(top_ids, n * top_k), words(top_logprobs, n * top_k), words(grad_loss, n), words(lse, n), words(rest_lse, n), x})
    if (overlap(y, r) && !(r.p == logits && logits == grad_logits && row_stride == grad_stride))
      return report_error(SWIFTKV_ERR_INVALID_ARG, "the gradient overlaps an input other than the logits in place");
  unsigned int *status = op_status_word();
  if (!status) return report_error(SWIFTKV_ERR_CUDA, "no status word");
  const int n_vec = (int)(((size_t)vocab * es + 15) / 16);
  // two turns a block where that leaves enough of them: a block's entries cost as much as half a turn
  int per_row = (n_vec + TB_THREADS * TB_UNROLL - 1) / (TB_THREADS * TB_UNROLL);
  if ((long long)rows * per_row > 32LL * num_sms()) per_row = (per_row + 1) / 2;
  if ((long long)rows * per_row > 0x7fffffffLL) per_row = 1;
  TdBwdArgs b{{logits, grad_logits, row_stride, grad_stride, top_ids, top_logprobs, grad_loss, nullptr, nullptr, nullptr, rows, vocab, top_k, 1,
               0.f, 1.0 / temperature, rest, status}, lse, rest_lse, per_row};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = dtype == SWIFTKV_DTYPE_F32 ? launch_distill_bwd<float>(b, st) : dtype == SWIFTKV_DTYPE_BF16 ? launch_distill_bwd<bf16>(b, st) : launch_distill_bwd<__half>(b, st);
  if (e != cudaSuccess) return report_error(SWIFTKV_ERR_CUDA, cudaGetErrorString(e));
  return SWIFTKV_OK;
}
