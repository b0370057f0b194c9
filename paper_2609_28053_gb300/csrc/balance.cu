// balance.cu -- the balance loss: per-expert counts from the routing lists,
// the launch of the pass over z (balance.cuh), and the sums of its blocks.
#include "eqb_device.cuh"

namespace eqb {

namespace {

constexpr int kCountThreads = 256;
constexpr int kCountWarps = kCountThreads / 32;

__global__ void balance_clear_kernel(int32_t* counts, int64_t n, int32_t* valid, int M) {
  griddep_wait();
  griddep_launch();
  const int64_t i0 = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  const int64_t step = static_cast<int64_t>(gridDim.x) * blockDim.x;
  for (int64_t i = i0; i < n; i += step) counts[i] = 0;
  if (valid)
    for (int64_t i = i0; i < M; i += step) valid[i] = 0;
}

// counts[l, e] += the entries of the lists of microbatch l's valid tokens that
// name expert e (others, as -1, name none); valid[l] += its valid tokens.  A
// block takes a contiguous range of tokens; each warp counts into a histogram
// of its own in shared memory, so that only lanes of a warp meet on a hot expert.
__global__ void __launch_bounds__(kCountThreads) balance_count_kernel(BalanceArgs a, int64_t tokens_per_cta, int copies) {
  extern __shared__ int32_t hist[];
  const int E = a.E, K = a.K;
  int32_t* mine = hist + static_cast<int>((threadIdx.x >> 5) % copies) * E;
  for (int i = threadIdx.x; i < copies * E; i += kCountThreads) hist[i] = 0;
  griddep_wait();
  const int64_t tb = static_cast<int64_t>(blockIdx.x) * tokens_per_cta;
  const int64_t te = min(tb + tokens_per_cta, a.T);
  if (tb >= te) return;
  int l = microbatch_of_warp(a.off, a.M, tb, threadIdx.x & 31);
  int64_t t = tb;
  while (t < te) {
    while (__ldg(a.off + l + 1) <= t && l + 1 < a.M) ++l;  // the next one that is not empty
    const int64_t hi = __ldg(a.off + l + 1);
    const int64_t seg_end = hi > t ? min(te, hi) : te;
    __syncthreads();
    // below 2^31: a block has at most T / grid tokens of at most 31 entries, or 64
    const int m = static_cast<int>((seg_end - t) * K);
    const int32_t* idx = a.idx + t * K;
    auto count = [&](int e) {
      if (static_cast<unsigned>(e) < static_cast<unsigned>(E)) atomicAdd(mine + e, 1);
    };
    if (a.mask) {
      for (int i = threadIdx.x; i < m; i += kCountThreads) {
        const int e = __ldcs(idx + i);
        if (a.mask[t + i / K]) count(e);
      }
    } else {
      // four entries a load, two loads in flight; single ones up to the first
      // 16-byte boundary and at the end
      const int head = min(m, static_cast<int>((16u - (reinterpret_cast<uintptr_t>(idx) & 15u)) & 15u) / 4);
      const int quads = (m - head) / 4;
      const int4* q4 = reinterpret_cast<const int4*>(idx + head);
      for (int i = threadIdx.x; i < quads; i += 2 * kCountThreads) {
        const bool two = i + kCountThreads < quads;
        const int4 w0 = __ldcs(q4 + i);
        const int4 w1 = two ? __ldcs(q4 + i + kCountThreads) : make_int4(-1, -1, -1, -1);
        count(w0.x); count(w0.y); count(w0.z); count(w0.w);
        count(w1.x); count(w1.y); count(w1.z); count(w1.w);
      }
      if (static_cast<int>(threadIdx.x) < head) count(idx[threadIdx.x]);
      const int end = head + 4 * quads + static_cast<int>(threadIdx.x);
      if (end < m) count(idx[end]);
    }
    if (a.mask) {
      int v = 0;
      for (int64_t i = t + threadIdx.x; i < seg_end; i += kCountThreads) v += a.mask[i] != 0;
      v = __reduce_add_sync(kFull, v);
      if ((threadIdx.x & 31) == 0 && v) atomicAdd(a.valid + l, v);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += kCountThreads) {
      int c = 0;
      for (int q = 0; q < copies; ++q) {
        c += hist[q * E + e];
        hist[q * E + e] = 0;
      }
      if (c) atomicAdd(a.counts + static_cast<int64_t>(l) * E + e, c);
    }
    t = seg_end;
  }
}

// prob and loss of microbatch blockIdx.y from its rows of a.part, which the
// blocks of its tokens wrote: 32 experts a block, its warps every W-th row.
template <int W>
__global__ void __launch_bounds__(32 * W) balance_finish_kernel(BalanceArgs a, uint32_t tokens_per_cta) {
  __shared__ float col[W][32];
  __shared__ double tot[W][3];
  griddep_wait();
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  for (int l = blockIdx.y; l < a.M; l += gridDim.y) {
    const int64_t lo = __ldg(a.off + l), hi = min(__ldg(a.off + l + 1), a.T);
    const int64_t n = a.mask ? a.valid[l] : hi - lo;
    // tokens are fewer than 2^31
    const uint32_t first = static_cast<uint32_t>(lo) / tokens_per_cta;
    const int rows = hi > lo ? static_cast<int>(static_cast<uint32_t>(hi - 1) / tokens_per_cta - first) + 1 : 0;
    const float* p = a.part + (static_cast<int64_t>(first) + l) * a.row;
    const int e = blockIdx.x * 32 + lane;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (e < a.E && a.prob)
      for (int q = wid; q < rows; q += 4 * W) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (q + W * u < rows) v[u] += __ldcg(p + static_cast<int64_t>(q + W * u) * a.row + 4 + e);
      }
    if (W > 1) col[wid][lane] = (v[0] + v[1]) + (v[2] + v[3]);
    const bool sums = blockIdx.x == 0 && a.loss;
    if (sums && lane < 3) {
      double s = 0.0;
      for (int q = wid; q < rows; q += W) s += static_cast<double>(__ldcg(p + static_cast<int64_t>(q) * a.row + lane));
      tot[wid][lane] = s;
    }
    __syncthreads();
    if (wid == 0 && e < a.E && a.prob) {
      float x = (v[0] + v[1]) + (v[2] + v[3]);
#pragma unroll
      for (int q = 1; q < W; ++q) x += col[q][lane];
      a.prob[static_cast<int64_t>(l) * a.E + e] = n > 0 ? x / static_cast<float>(n) : 0.f;
    }
    if (sums && threadIdx.x == 0) {
      double h = 0.0, zz = 0.0, alive = 0.0;
#pragma unroll
      for (int q = 0; q < W; ++q) {
        h += tot[q][0];
        zz += tot[q][1];
        alive += tot[q][2];
      }
      const double r = n > 0 ? 1.0 / static_cast<double>(n) : 0.0;
      a.loss[2 * l] = static_cast<float>(a.alpha * (h + alive / a.E) * r);
      a.loss[2 * l + 1] = static_cast<float>(a.zeta * zz * r);
    }
    __syncthreads();
  }
}

}  // namespace

// counts (and valid, with a mask) of the whole batch.
int launch_balance_counts(const BalanceArgs& a, cudaStream_t s) {
  DeviceInfo di;
  if (int rc = device_info(&di)) return rc;
  const int64_t cells = static_cast<int64_t>(a.M) * a.E;
  const int64_t cgrid = (cells + 1023) / 1024;
  if (launch_dependent(balance_clear_kernel, dim3(static_cast<unsigned>(cgrid < 1024 ? cgrid : 1024)), dim3(256), 0, s, a.counts,
                       cells, a.mask ? a.valid : nullptr, a.M) != cudaSuccess)
    return kErrCuda;
  if (a.T == 0) return kOk;
  int64_t grid = (a.T + 63) / 64;
  if (grid > di.sm_count * 8) grid = di.sm_count * 8;
  const int64_t tpc = (a.T + grid - 1) / grid;
  const int copies = a.E <= 512 ? kCountWarps : kCountWarps / 2;
  return launch_dependent(balance_count_kernel, dim3(static_cast<unsigned>((a.T + tpc - 1) / tpc)), dim3(kCountThreads),
                          static_cast<size_t>(copies) * a.E * 4, s, a, tpc, copies) == cudaSuccess
             ? kOk
             : kErrCuda;
}

int launch_balance(BalanceArgs a, cudaStream_t s) {
  const bool sums = a.prob || a.loss;
  if (!sums) a.part = nullptr;
  BalanceRun run{1, 1, 0};
  if (a.T > 0 && (sums || a.grad_out)) {
    const int rc = a.sigmoid ? (a.grad_out ? launch_balance_sigmoid_grad(a, &run, s) : launch_balance_sigmoid_value(a, &run, s))
                             : (a.grad_out ? launch_balance_softmax_grad(a, &run, s) : launch_balance_softmax_value(a, &run, s));
    if (rc) return rc;
  } else if (int rc = launch_balance_counts(a, s)) {
    return rc;
  }
  if (!sums || run.done) return kOk;
  const dim3 fin(static_cast<unsigned>((a.E + 31) / 32), static_cast<unsigned>(a.M < 4096 ? a.M : 4096));
  // a warp a block where a microbatch has a few rows
  const bool few = a.T / run.tokens_per_cta <= 16 * static_cast<int64_t>(a.M);
  const auto kern = few ? balance_finish_kernel<1> : balance_finish_kernel<8>;
  return launch_dependent(kern, fin, dim3(few ? 32 : 256), 0, s, a, static_cast<uint32_t>(run.tokens_per_cta)) == cudaSuccess
             ? kOk
             : kErrCuda;
}

}  // namespace eqb
