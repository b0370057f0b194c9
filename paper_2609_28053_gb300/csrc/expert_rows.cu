// expert_rows.cu -- the experts' rows from the tokens' lists: a stable counting
// sort of the list entries by expert.
//
// The entries are cut into chunks, one a block.  One kernel counts every chunk's
// entries of each expert, and one gives every entry its row: the rows of the experts
// before, of the chunks before, of the block's warps before, and of the entries
// before it in the warp's 32, which __match_any_sync counts.  Every step counts in
// a fixed order, so rows are in ascending order of entry.  Few entries are one
// chunk, whose block needs no other kernel; of many chunks a third kernel forms
// each expert's running sums (a warp an expert), of up to kAddedCounts counts every
// block adds those before its own itself.
//
// It is latency that counts: launches, and loads that wait for one another.  A lane
// asks for eight entries together (T = 65,536, K = 8, E = 128: 14.1 us with one at a
// time and three launches, 10.8 us).
#include "eqb_device.cuh"

namespace eqb {

namespace {

constexpr int kRowsWarps = 16;
constexpr int kRowsThreads = kRowsWarps * 32;
constexpr int kRowsChunk = 4096;  // least entries of a chunk
constexpr int kRowsChunks = 608;  // most chunks, about
constexpr int kRowsAhead = 8;     // entries that a lane asks for together
constexpr int kAddedCounts = 1 << 15;
constexpr int kRowsFree = 47 * 1024;  // what every launch may have, less room for the kernel's static part

struct RowsPlan {
  int chunks, per;  // per: entries of a chunk, a multiple of kRowsThreads
};
RowsPlan plan_rows(int64_t n) {
  RowsPlan p;
  const int64_t even = (n + kRowsChunks - 1) / kRowsChunks;
  const int64_t per = even > kRowsChunk ? even : n < kRowsChunk ? (n > 0 ? n : 1) : kRowsChunk;
  p.per = static_cast<int>((per + kRowsThreads - 1) / kRowsThreads * kRowsThreads);
  p.chunks = static_cast<int>((n + p.per - 1) / p.per);
  if (p.chunks < 1) p.chunks = 1;
  return p;
}

__host__ __device__ constexpr bool added_counts(int chunks, int E) { return static_cast<int64_t>(chunks) * E <= kAddedCounts; }

__device__ __forceinline__ int expert_of(const ExpertRowsArgs& a, int64_t i, int64_t end) {
  if (i >= end) return -1;
  const int e = __ldg(a.idx + i);
  return e >= 0 && e < a.E ? e : -1;
}

__global__ void __launch_bounds__(kRowsThreads) rows_count_kernel(const ExpertRowsArgs a, int per, int chunks) {
  __shared__ int cnt[kMaxExperts];
  for (int e = threadIdx.x; e < a.E; e += kRowsThreads) cnt[e] = 0;
  __syncthreads();
  griddep_wait();
  const int64_t i0 = static_cast<int64_t>(blockIdx.x) * per, end = min(a.n, i0 + per);
  for (int64_t i = i0 + threadIdx.x; i < end; i += kRowsThreads * kRowsAhead) {
    int e[kRowsAhead];
#pragma unroll
    for (int k = 0; k < kRowsAhead; ++k) e[k] = expert_of(a, i + k * kRowsThreads, end);
#pragma unroll
    for (int k = 0; k < kRowsAhead; ++k)
      if (e[k] >= 0) atomicAdd(cnt + e[k], 1);
  }
  __syncthreads();
  // a row of counts a chunk, or, to be scanned, a row of chunks an expert
  const bool added = added_counts(chunks, a.E);
  for (int e = threadIdx.x; e < a.E; e += kRowsThreads)
    a.ws[added ? static_cast<int64_t>(blockIdx.x) * a.E + e : static_cast<int64_t>(e) * chunks + blockIdx.x] = cnt[e];
}

// Running sums over the chunks, exclusive, and each expert's total behind them.
__global__ void __launch_bounds__(256) rows_scan_kernel(const ExpertRowsArgs a, int chunks) {
  const int e = static_cast<int>(blockIdx.x) * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  griddep_wait();
  if (e >= a.E) return;
  int* row = a.ws + static_cast<int64_t>(e) * chunks;
  int run = 0;
  for (int c0 = 0; c0 < chunks; c0 += 32) {
    const int v = c0 + lane < chunks ? row[c0 + lane] : 0;
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(kFull, x, o);
      if (lane >= o) x += y;
    }
    if (c0 + lane < chunks) row[c0 + lane] = run + x - v;
    run += __shfl_sync(kFull, x, 31);
  }
  if (lane == 0) a.ws[static_cast<int64_t>(a.E) * chunks + e] = run;
}

__global__ void __launch_bounds__(kRowsThreads) rows_place_kernel(const ExpertRowsArgs a, int per, int chunks) {
  extern __shared__ int cnt[];  // [warps][E], then the experts' totals, first rows and rows of the chunks before [E] each
  __shared__ int part[2][kRowsWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, E = a.E;
  int* total = cnt + kRowsWarps * E;
  int* first = total + E;
  int* before = first + E;
  for (int i = threadIdx.x; i < (kRowsWarps + 3) * E; i += kRowsThreads) cnt[i] = 0;
  __syncthreads();
  griddep_wait();
  // a warp's entries: a contiguous part of the chunk
  const int64_t w0 = static_cast<int64_t>(blockIdx.x) * per + warp * (per / kRowsWarps);
  const int64_t end = min(a.n, w0 + per / kRowsWarps);
  int* mine = cnt + warp * E;
  const bool again = per / kRowsWarps > 32 * kRowsAhead;  // the warp's entries do not stay in e
  int e[kRowsAhead];
  auto load = [&](int64_t i) {
#pragma unroll
    for (int k = 0; k < kRowsAhead; ++k) e[k] = expert_of(a, i + k * 32 + lane, end);
  };
  load(w0);
  if (chunks > 1) {
    if (added_counts(chunks, E)) {
      // kRowsThreads / E threads an expert, each some of the chunks, 32 asked for together
      const int threads = max(kRowsThreads / E, 1);
      for (int u = threadIdx.x; u < E * threads; u += kRowsThreads) {
        const int x = u % E;
        int all = 0, ahead = 0;
        for (int c0 = u / E; c0 < chunks; c0 += 32 * threads) {
          int v[32];
#pragma unroll
          for (int k = 0; k < 32; ++k) {
            const int c = c0 + k * threads;
            v[k] = c < chunks ? __ldcg(a.ws + static_cast<int64_t>(c) * E + x) : 0;
          }
#pragma unroll
          for (int k = 0; k < 32; ++k) {
            all += v[k];
            ahead += c0 + k * threads < static_cast<int>(blockIdx.x) ? v[k] : 0;
          }
        }
        atomicAdd(total + x, all);
        atomicAdd(before + x, ahead);
      }
    } else {
      for (int x = threadIdx.x; x < E; x += kRowsThreads) {
        total[x] = __ldcg(a.ws + static_cast<int64_t>(E) * chunks + x);
        before[x] = __ldcg(a.ws + static_cast<int64_t>(x) * chunks + blockIdx.x);
      }
    }
  }
  for (int64_t i = w0; i < end; i += 32 * kRowsAhead) {
    if (i > w0) load(i);
#pragma unroll
    for (int k = 0; k < kRowsAhead; ++k)
      if (e[k] >= 0) atomicAdd(mine + e[k], 1);
  }
  __syncthreads();
  // what the chunk's warps before have
  for (int x = threadIdx.x; x < E; x += kRowsThreads) {
    int run = 0, v[kRowsWarps];
#pragma unroll
    for (int w = 0; w < kRowsWarps; ++w) v[w] = cnt[w * E + x];
#pragma unroll
    for (int w = 0; w < kRowsWarps; ++w) {
      cnt[w * E + x] = run;
      run += v[w];
    }
    if (chunks == 1) total[x] = run;
  }
  __syncthreads();
  // first rows and blocks of the experts: two neighbours a thread
  {
    const int e0 = 2 * threadIdx.x;
    const int n0 = e0 < E ? total[e0] : 0, n1 = e0 + 1 < E ? total[e0 + 1] : 0;
    const int b0 = (n0 + kExpertBlock - 1) / kExpertBlock, b1 = (n1 + kExpertBlock - 1) / kExpertBlock;
    int x = n0 + n1, y = b0 + b1;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int p = __shfl_up_sync(kFull, x, o), q = __shfl_up_sync(kFull, y, o);
      if (lane >= o) {
        x += p;
        y += q;
      }
    }
    if (lane == 31) {
      part[0][warp] = x;
      part[1][warp] = y;
    }
    __syncthreads();
    int rows = x - n0 - n1, blks = y - b0 - b1;
    for (int w = 0; w < warp; ++w) {
      rows += part[0][w];
      blks += part[1][w];
    }
    if (e0 < E) first[e0] = rows;
    if (e0 + 1 < E) first[e0 + 1] = rows + n0;
    if (blockIdx.x == 0) {
      if (e0 < E) {
        a.offsets[e0 + 1] = rows + n0;
        a.blocks[e0 + 1] = blks + b0;
      }
      if (e0 + 1 < E) {
        a.offsets[e0 + 2] = rows + n0 + n1;
        a.blocks[e0 + 2] = blks + b0 + b1;
      }
      if (threadIdx.x == 0) a.offsets[0] = a.blocks[0] = 0;
    }
  }
  __syncthreads();
  const int all = first[E - 1] + total[E - 1];
  for (int x = threadIdx.x; x < E; x += kRowsThreads) {
    const int base = first[x] + before[x];
#pragma unroll
    for (int w = 0; w < kRowsWarps; ++w) cnt[w * E + x] += base;
  }
  __syncthreads();
  for (int64_t i = w0; i < end; i += 32 * kRowsAhead) {
    if (again) load(i);
#pragma unroll
    for (int k = 0; k < kRowsAhead; ++k) {
      const uint32_t same = __match_any_sync(kFull, e[k]);
      const int row = e[k] >= 0 ? mine[e[k]] + __popc(same & ((1u << lane) - 1u)) : -1;
      __syncwarp();
      if (e[k] >= 0 && lane == __ffs(same) - 1) mine[e[k]] += __popc(same);
      __syncwarp();
      const int64_t at = i + k * 32 + lane;
      if (at < end) {
        a.slot[at] = row;
        if (row >= 0) a.entry[row] = static_cast<int32_t>(at);
      }
    }
  }
  // the rows of this chunk's numbers that no entry has
  const int64_t r0 = static_cast<int64_t>(blockIdx.x) * per, r1 = min(a.n, r0 + per);
  for (int64_t r = max(r0, static_cast<int64_t>(all)) + threadIdx.x; r < r1; r += kRowsThreads) a.entry[r] = -1;
}

}  // namespace

size_t expert_rows_workspace(int64_t n, int E) {
  const RowsPlan p = plan_rows(n);
  return p.chunks == 1 ? 0 : carve_round((static_cast<size_t>(p.chunks) + 1) * static_cast<size_t>(E) * 4);
}

int launch_expert_rows(const ExpertRowsArgs& a, cudaStream_t s) {
  const RowsPlan p = plan_rows(a.n);
  const int smem = (kRowsWarps + 3) * a.E * 4;
  if (smem > kRowsFree && !allow_smem(rows_place_kernel, (kRowsWarps + 3) * kMaxExperts * 4)) return kErrCuda;
  if (p.chunks > 1) {
    if (launch_dependent(rows_count_kernel, dim3(p.chunks), dim3(kRowsThreads), 0, s, a, p.per, p.chunks) != cudaSuccess)
      return kErrCuda;
    if (!added_counts(p.chunks, a.E) &&
        launch_dependent(rows_scan_kernel, dim3((a.E + 7) / 8), dim3(256), 0, s, a, p.chunks) != cudaSuccess)
      return kErrCuda;
  }
  return launch_dependent(rows_place_kernel, dim3(p.chunks), dim3(kRowsThreads), smem, s, a, p.per, p.chunks) == cudaSuccess
             ? kOk
             : kErrCuda;
}

}  // namespace eqb
