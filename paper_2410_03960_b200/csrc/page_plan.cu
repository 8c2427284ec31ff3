// swiftkv_plan_pages: cache rows of a step's new tokens, planned on the device from the sequences' lengths.
//
// With page size P = 128, sequence b (past_b cached tokens, new_b new ones, owned_b table entries in use) needs
//   need_b = max(0, ceil((past_b + new_b) / P) - owned_b)
// further pages; taken in sequence order from the end of the free list, so entry owned_b + i becomes
//   free[n_free - 1 - (sum_{a < b} need_a + i)],
// and new token t of sequence b (position p = past_b + t - cu_b) lands in cache row table[b][p / P] * P + p % P.
//
// Everything after the two prefix sums is independent per table entry and per token: some blocks write the tokens' rows, the others
// the tables.  The sums run over a few thousand integers at most, so EVERY block computes them for itself (about 1 us for 1024
// sequences, served by L2) instead of waiting for one that does: a single launch without any communication between blocks.
// What bounds it: latencies, one after the other (the launch, the lengths, a token's search and page): 3.4 - 3.8 us for 8 sequences,
// 8.0 us for 1024 sequences with 6.5 MB of tables (their copy alone would take 1 us).
#include "common.cuh"
#include "tc_common.cuh"

namespace skv {
namespace {

constexpr int PP_THREADS = 256;
constexpr int PP_AHEAD = 8;
constexpr int PP_MAX_SEQS = 8192;

struct PlanArgs {
  const int32_t *past, *n_new, *owned, *table, *free_pages, *n_free;
  int32_t *table_out, *owned_out, *n_free_out, *cu_new, *slot_map, *positions, *info;
  int n_seqs, max_blocks, free_cap, max_tokens;
};

// lengths as the device finds them: counts below zero read as zero, entries in use are at most what a table row holds
__device__ __forceinline__ void plan_lengths(const PlanArgs &a, int &past, int &fresh, int &owned, int &need, int &lacking) {
  past = max(0, past);
  fresh = min(max(0, fresh), 0x7fffffff - past);
  owned = min(max(0, owned), a.max_blocks);
  const int wanted = (int)(((unsigned)past + (unsigned)fresh + PAGE_ROWS - 1) / PAGE_ROWS);
  need = max(0, min(wanted, a.max_blocks) - owned);
  lacking = max(0, wanted - a.max_blocks);
}

__global__ void __launch_bounds__(PP_THREADS) plan_pages_kernel(PlanArgs a, int token_blocks) {
  extern __shared__ int32_t pp_smem[];
  int32_t *s_cu = pp_smem;                    // [n_seqs + 1]
  int32_t *s_first = pp_smem + a.n_seqs + 1;  // [n_seqs + 1] pages taken before sequence b
  __shared__ int2 s_warp[PP_THREADS / 32];
  __shared__ int s_over[PP_THREADS / 32], s_long[PP_THREADS / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (a.n_seqs + PP_THREADS - 1) / PP_THREADS;
  const int b0 = min(a.n_seqs, tid * per), b1 = min(a.n_seqs, b0 + per);
  int2 sum = make_int2(0, 0);
  int over = 0, longest = 0;
  for (int c0 = b0; c0 < b1; c0 += 4) {              // four sequences' loads under way at a time
    int past[4], fresh[4], owned[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const bool there = c0 + q < b1;
      past[q] = there ? a.past[c0 + q] : 0;
      fresh[q] = there ? a.n_new[c0 + q] : 0;
      owned[q] = there ? a.owned[c0 + q] : 0;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (c0 + q >= b1) break;
      int need, lacking;
      plan_lengths(a, past[q], fresh[q], owned[q], need, lacking);
      s_cu[c0 + q] = sum.x;
      s_first[c0 + q] = sum.y;
      sum.x += fresh[q];
      sum.y += need;
      over += lacking;
      longest = max(longest, past[q] + fresh[q]);
    }
  }
  int2 inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, inc.x, o), y = __shfl_up_sync(0xffffffffu, inc.y, o);
    if (lane >= o) { inc.x += x; inc.y += y; }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    over += __shfl_xor_sync(0xffffffffu, over, o);
    longest = max(longest, __shfl_xor_sync(0xffffffffu, longest, o));
  }
  if (lane == 31) s_warp[warp] = inc;
  if (lane == 0) { s_over[warp] = over; s_long[warp] = longest; }
  __syncthreads();
  int2 base = make_int2(0, 0), all = make_int2(0, 0);
#pragma unroll
  for (int w = 0; w < PP_THREADS / 32; ++w) {
    if (w < warp) { base.x += s_warp[w].x; base.y += s_warp[w].y; }
    all.x += s_warp[w].x;
    all.y += s_warp[w].y;
  }
  base.x += inc.x - sum.x;
  base.y += inc.y - sum.y;
  for (int b = b0; b < b1; ++b) { s_cu[b] += base.x; s_first[b] += base.y; }
  if (tid == 0) { s_cu[a.n_seqs] = all.x; s_first[a.n_seqs] = all.y; }
  __syncthreads();

  const int n_free = min(max(0, *a.n_free), a.free_cap);
  const int taken = min(all.y, n_free);
  const int total = min(all.x, a.max_tokens);
  // the page of table entry j of sequence b, -1 where it has none (j and the rank are negative where the sums of what was given wrap)
  auto page_of = [&](int b, int owned, int j) -> int {
    if (j >= 0 && j < owned) return a.table[(size_t)b * a.max_blocks + j];
    const int rank = s_first[b] + j - owned;
    return (j >= owned && j < a.max_blocks && rank >= 0 && rank < s_first[b + 1] && rank < n_free) ? a.free_pages[n_free - 1 - rank] : -1;
  };
  // new tokens, one per thread: the sequence by a binary search in the offsets
  if ((int)blockIdx.x < token_blocks) {
    for (int t = blockIdx.x * PP_THREADS + tid; t < total; t += token_blocks * PP_THREADS) {
      int lo = 0, hi = a.n_seqs;          // s_cu[lo] <= t < s_cu[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s_cu[mid] <= t) lo = mid; else hi = mid;
      }
      const int pos = max(0, a.past[lo]) + t - s_cu[lo];
      const int page = page_of(lo, min(max(0, a.owned[lo]), a.max_blocks), pos / PAGE_ROWS);
      a.slot_map[t] = page >= 0 && page < 0x7fffffff / PAGE_ROWS ? page * PAGE_ROWS + pos % PAGE_ROWS : -1;
      a.positions[t] = pos;
    }
    return;
  }
  // block tables, one warp per row; in place only the entries behind the used ones are written
  const bool in_place = a.table_out == a.table;
  for (int b = ((int)blockIdx.x - token_blocks) * (PP_THREADS / 32) + warp; b < a.n_seqs; b += ((int)gridDim.x - token_blocks) * (PP_THREADS / 32)) {
    const int owned = min(max(0, a.owned[b]), a.max_blocks);
    int32_t *row = a.table_out + (size_t)b * a.max_blocks;
    const int32_t *old = a.table + (size_t)b * a.max_blocks;
    if (!in_place) {
      int j = lane;
      for (; j < owned; j += 32 * PP_AHEAD) {       // PP_AHEAD loads in flight per lane
        int x[PP_AHEAD];
#pragma unroll
        for (int q = 0; q < PP_AHEAD; ++q) x[q] = j + 32 * q < owned ? old[j + 32 * q] : 0;
#pragma unroll
        for (int q = 0; q < PP_AHEAD; ++q)
          if (j + 32 * q < owned) row[j + 32 * q] = x[q];
      }
    }
    for (int j = owned + lane; j < a.max_blocks; j += 32) row[j] = page_of(b, owned, j);
    if (lane == 0) a.owned_out[b] = owned + max(0, min(s_first[b + 1], n_free) - s_first[b]);
  }
  if ((int)blockIdx.x == token_blocks) {
    for (int b = tid; b <= a.n_seqs; b += PP_THREADS) a.cu_new[b] = s_cu[b];
    if (tid == 0) {
      int o = 0, l = 0;
      for (int w = 0; w < PP_THREADS / 32; ++w) { o += s_over[w]; l = max(l, s_long[w]); }
      *a.n_free_out = n_free - taken;
      a.info[0] = all.x;
      a.info[1] = taken;
      a.info[2] = all.y - taken + o;
      a.info[3] = l;
    }
  }
}

}  // namespace
}  // namespace skv

using namespace skv;

extern "C" int32_t swiftkv_plan_pages(const int32_t *n_past, const int32_t *n_new, const int32_t *n_owned, int32_t n_seqs,
                                      const int32_t *block_table, int32_t max_blocks, const int32_t *free_pages,
                                      int32_t free_capacity, const int32_t *n_free, int32_t *block_table_out, int32_t *n_owned_out,
                                      int32_t *n_free_out, int32_t *cu_new, int32_t *slot_map, int32_t *positions,
                                      int32_t max_tokens, int32_t *info, void *cuda_stream) {
  if (!n_past || !n_new || !n_owned || !block_table || !n_free || !block_table_out || !n_owned_out || !n_free_out || !cu_new || !info)
    return report_error(SWIFTKV_ERR_INVALID_ARG, "null argument");
  if (n_seqs < 1 || n_seqs > PP_MAX_SEQS || max_blocks < 1 || max_blocks > (1 << 24) || free_capacity < 0 || max_tokens < 0)
    return report_error(SWIFTKV_ERR_INVALID_ARG, "bad shape (n_seqs must be in [1, 8192], max_blocks in [1, 2^24])");
  if ((free_capacity > 0 && !free_pages) || (max_tokens > 0 && (!slot_map || !positions)))
    return report_error(SWIFTKV_ERR_INVALID_ARG, "null argument");
  // every block reads the lengths for itself, so none may be overwritten by another: only the table can be updated in place
  struct Range { const void *p; size_t n; };
  const size_t w = sizeof(int32_t), table_n = (size_t)n_seqs * max_blocks;
  const Range in[] = {{n_past, (size_t)n_seqs}, {n_new, (size_t)n_seqs}, {n_owned, (size_t)n_seqs}, {n_free, 1},
                      {free_pages, (size_t)free_capacity}, {block_table, table_n}};
  const Range out[] = {{n_owned_out, (size_t)n_seqs}, {n_free_out, 1}, {cu_new, (size_t)n_seqs + 1}, {slot_map, (size_t)max_tokens},
                       {positions, (size_t)max_tokens}, {info, 4}, {block_table_out, table_n}};
  auto overlap = [&](const Range &x, const Range &y) {
    const uintptr_t a = (uintptr_t)x.p, b = (uintptr_t)y.p;
    return x.n && y.n && a < b + y.n * w && b < a + x.n * w;
  };
  for (size_t i = 0; i < sizeof out / sizeof out[0]; ++i) {
    for (const Range &r : in)
      if (overlap(out[i], r) && !(out[i].p == block_table_out && r.p == block_table && block_table_out == block_table))
        return report_error(SWIFTKV_ERR_INVALID_ARG, "an output overlaps an input (only the block table may be updated in place)");
    for (size_t j = 0; j < i; ++j)
      if (overlap(out[i], out[j])) return report_error(SWIFTKV_ERR_INVALID_ARG, "two outputs overlap");
  }
  PlanArgs a{n_past, n_new, n_owned, block_table, free_pages, n_free, block_table_out, n_owned_out, n_free_out, cu_new, slot_map, positions,
             info, n_seqs, max_blocks, free_capacity, max_tokens};
  const size_t smem = 2 * ((size_t)n_seqs + 1) * sizeof(int32_t);
  if (smem > 48 * 1024 && ensure_dynamic_smem(reinterpret_cast<const void *>(plan_pages_kernel), (int)(2 * (PP_MAX_SEQS + 1) * sizeof(int32_t))))
    return report_error(SWIFTKV_ERR_CUDA, "shared memory");
  // blocks of 256 tokens, then blocks of 8 table rows, at most one of each per SM: each repeats the prefix sums
  const long long by_tokens = ((long long)max_tokens + PP_THREADS - 1) / PP_THREADS, by_rows = (n_seqs + 7) / 8, most = num_sms();
  const int token_blocks = (int)(by_tokens < most ? by_tokens : most), row_blocks = (int)(by_rows < most ? by_rows : most);
  plan_pages_kernel<<<token_blocks + row_blocks, PP_THREADS, smem, reinterpret_cast<cudaStream_t>(cuda_stream)>>>(a, token_blocks);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return report_error(SWIFTKV_ERR_CUDA, cudaGetErrorString(e));
  return SWIFTKV_OK;
}
