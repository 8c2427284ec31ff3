// swiftkv_commit_drafts: the cache rows of the drafted tokens that stand move together, in every plane of the cache, and lengths grow.
//
// Row path[j] of a sequence's new tokens goes to row j.  Entries ascend, so path[j] >= j: whoever moves a column's rows in ascending order never
// overwrites one that is still to be read.  One thread therefore moves a column (16 bytes, or what a plane's alignment allows) of all of a
// sequence's rows, CD_AHEAD of them read before the first of these is written, and threads need nothing from one another.
//
// What bounds it: a chain of reads (the count, the path, the table's pages, the rows) and then HBM; moved rows alone are touched.  A block looks
// the rows of one sequence up and moves them in one plane: thousands of small blocks for a batch, which hide each other's chains.  64 sequences of
// up to 8 moved rows of 2 KB in 32 planes (29 MB) 6.6 us, 7.2 us with eight rows ahead (two waves of blocks instead of one); a small batch 4.3 us.
#include "common.cuh"

#include <algorithm>
#include <vector>

namespace skv {
namespace {

constexpr int CD_THREADS = 128;
constexpr int CD_AHEAD = 4;                  // (32 registers: 16 blocks per SM)
constexpr int CD_MAX_NEW = 1024;
constexpr int CD_PLANES = 224;               // of one launch: what its parameters hold

struct CommitArgs {
  const int32_t *table, *row0, *past, *accepted, *path;
  int32_t *past_out;
  int max_blocks, max_new, cache_rows, last;
  unsigned int *status;
};
struct CommitPlanes {
  uint8_t *p[CD_PLANES];
  int32_t bytes[CD_PLANES];
};

template <typename V>
__device__ __forceinline__ void move_rows(uint8_t *plane, int bytes, const int *from, const int *to, int count) {
  const int columns = bytes / (int)sizeof(V);
  for (int col = threadIdx.x; col < columns; col += CD_THREADS) {
    for (int j0 = 0; j0 < count; j0 += CD_AHEAD) {
      V x[CD_AHEAD];
#pragma unroll
      for (int j = 0; j < CD_AHEAD; ++j)
        if (j0 + j < count) x[j] = *reinterpret_cast<const V *>(plane + (size_t)from[j0 + j] * bytes + (size_t)col * sizeof(V));
#pragma unroll
      for (int j = 0; j < CD_AHEAD; ++j)
        if (j0 + j < count) *reinterpret_cast<V *>(plane + (size_t)to[j0 + j] * bytes + (size_t)col * sizeof(V)) = x[j];
    }
  }
}

__global__ void __launch_bounds__(CD_THREADS, 16) commit_drafts_kernel(const __grid_constant__ CommitPlanes planes, CommitArgs a, int n_planes) {
  __shared__ int s_from[CD_MAX_NEW], s_to[CD_MAX_NEW];
  __shared__ int s_warp[CD_THREADS / 32];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int32_t *path = a.path + (size_t)b * a.max_new;
  const int past = max(0, a.past[b]), wanted = min(max(a.accepted[b], 0), a.max_new - 1) + 1;
  // how far the path ascends from an entry of at least 0
  int kept = wanted;
  for (int j = tid; j < wanted; j += CD_THREADS)
    if (path[j] < 0 || (j > 0 && path[j] <= path[j - 1])) { kept = j; break; }
  kept = __reduce_min_sync(0xffffffffu, kept);
  if (lane == 0) s_warp[warp] = kept;
  __syncthreads();
  for (int w = 0; w < CD_THREADS / 32; ++w) kept = min(kept, s_warp[w]);
  auto row_of = [&](long long p) -> long long {          // -1: no row of the cache
    long long row = -1;
    if (a.table) {
      if (p / PAGE_ROWS < a.max_blocks) {
        const long long page = a.table[(size_t)b * a.max_blocks + p / PAGE_ROWS];
        if (page >= 0) row = page * PAGE_ROWS + p % PAGE_ROWS;
      }
    } else {
      row = a.row0[b] + p;
    }
    return row >= 0 && row < a.cache_rows ? row : -1;
  };
  // the moves in order, without those that stay where they are or have no row
  int count = 0;
  for (int j0 = 0; j0 < kept; j0 += CD_THREADS) {
    const int j = j0 + tid;
    long long from = -1, to = -1;
    if (j < kept && path[j] != j) {
      from = row_of((long long)past + path[j]);
      to = row_of((long long)past + j);
    }
    const bool is = from >= 0 && to >= 0;
    const unsigned all = __ballot_sync(0xffffffffu, is);
    __syncthreads();
    if (lane == 0) s_warp[warp] = __popc(all);
    __syncthreads();
    int at = count;
    for (int w = 0; w < CD_THREADS / 32; ++w) {
      if (w < warp) at += s_warp[w];
      count += s_warp[w];
    }
    if (is) {
      at += __popc(all & ((1u << lane) - 1u));
      s_from[at] = (int)from;
      s_to[at] = (int)to;
    }
  }
  __syncthreads();
  if (count) {
    for (int p = blockIdx.y; p < n_planes; p += gridDim.y) {
      uint8_t *plane = planes.p[p];
      const int bytes = planes.bytes[p];
      const unsigned common = (unsigned)reinterpret_cast<uintptr_t>(plane) | (unsigned)bytes;
      if (common % 16 == 0) move_rows<uint4>(plane, bytes, s_from, s_to, count);
      else if (common % 4 == 0) move_rows<uint32_t>(plane, bytes, s_from, s_to, count);
      else move_rows<uint8_t>(plane, bytes, s_from, s_to, count);
    }
  }
  if (a.last && blockIdx.y == 0 && tid == 0) {
    const long long grown = (long long)past + kept;
    a.past_out[b] = grown > 0x7fffffff ? 0x7fffffff : (int)grown;
    if (kept < wanted && !(kept == 0 && wanted == 1)) atomicOr(a.status, STATUS_BAD_TOKEN);
  }
}

}  // namespace
}  // namespace skv

using namespace skv;

extern "C" int32_t swiftkv_commit_drafts(void *const *planes, const int64_t *row_bytes, int32_t n_planes, int32_t cache_rows,
                                         const int32_t *block_table, int32_t max_blocks, const int32_t *row0, const int32_t *n_past,
                                         const int32_t *n_accepted, const int32_t *path, int32_t max_new, int32_t n_seqs, int32_t *n_past_out,
                                         void *cuda_stream) {
  if (!n_past || !n_accepted || !path || !n_past_out || (!block_table && !row0) || (n_planes > 0 && (!planes || !row_bytes)))
    return report_error(SWIFTKV_ERR_INVALID_ARG, "null argument");
  if (block_table && row0) return report_error(SWIFTKV_ERR_INVALID_ARG, "block_table or row0, not both");
  if (n_planes < 0 || n_planes > (1 << 16) || cache_rows < 1 || max_new < 1 || max_new > CD_MAX_NEW || n_seqs < 1 || n_seqs > 65535 || (block_table && max_blocks < 1))
    return report_error(SWIFTKV_ERR_INVALID_ARG, "bad shape (n_planes in [0, 65536], cache_rows >= 1, max_new in [1, 1024], n_seqs in [1, 65535], max_blocks >= 1)");
  auto flat = [](const void *p, size_t n) { return ByteRows{p, 1, n, n}; };
  const size_t seqs = (size_t)n_seqs, table_n = block_table ? seqs * max_blocks * 4 : 0;
  const ByteRows out = flat(n_past_out, seqs * 4);
  const ByteRows in[] = {flat(n_past, seqs * 4), flat(n_accepted, seqs * 4), flat(path, seqs * max_new * 4), flat(block_table, table_n), flat(row0, seqs * 4)};
  for (const ByteRows &r : in)
    if (r.p && overlap(out, r)) return report_error(SWIFTKV_ERR_INVALID_ARG, "n_past_out overlaps an input");
  // planes in the order of their addresses: each must end before the next begins
  try {
    std::vector<std::pair<uintptr_t, uintptr_t>> spans((size_t)n_planes);
    for (int i = 0; i < n_planes; ++i) {
      if (!planes[i]) return report_error(SWIFTKV_ERR_INVALID_ARG, "null argument");
      if (row_bytes[i] < 1 || row_bytes[i] > (1 << 20)) return report_error(SWIFTKV_ERR_INVALID_ARG, "bad shape (row_bytes in [1, 2^20])");
      const uintptr_t p = reinterpret_cast<uintptr_t>(planes[i]);
      const size_t size = (size_t)cache_rows * (size_t)row_bytes[i];
      spans[i] = {p, p + size};
      const ByteRows plane = flat(planes[i], size);
      if (overlap(out, plane)) return report_error(SWIFTKV_ERR_INVALID_ARG, "n_past_out overlaps a plane");
      for (const ByteRows &r : in)
        if (r.p && overlap(plane, r)) return report_error(SWIFTKV_ERR_INVALID_ARG, "a plane overlaps an input");
    }
    if (!std::is_sorted(spans.begin(), spans.end())) std::sort(spans.begin(), spans.end());
    for (int i = 1; i < n_planes; ++i)
      if (spans[i].first < spans[i - 1].second) return report_error(SWIFTKV_ERR_INVALID_ARG, "two planes overlap (one that layers share is given once)");
  } catch (...) {
    return report_error(SWIFTKV_ERR_INVALID_ARG, "out of host memory");
  }
  unsigned int *status = op_status_word();
  if (!status) return report_error(SWIFTKV_ERR_CUDA, "no status word");
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  CommitArgs a{block_table, row0, n_past, n_accepted, path, n_past_out, max_blocks, max_new, cache_rows, 0, status};
  int done = 0;
  do {
    CommitPlanes part;
    const int n = std::min(CD_PLANES, n_planes - done);
    for (int i = 0; i < n; ++i) {
      part.p[i] = static_cast<uint8_t *>(planes[done + i]);
      part.bytes[i] = (int32_t)row_bytes[done + i];
    }
    for (int i = n; i < CD_PLANES; ++i) { part.p[i] = nullptr; part.bytes[i] = 0; }
    done += n;
    a.last = done >= n_planes;
    commit_drafts_kernel<<<dim3((unsigned)n_seqs, (unsigned)std::max(n, 1)), CD_THREADS, 0, st>>>(part, a, n);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return report_error(SWIFTKV_ERR_CUDA, cudaGetErrorString(e));
  } while (done < n_planes);
  return SWIFTKV_OK;
}
