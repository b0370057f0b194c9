// balance.cu -- the balance loss: per-expert counts from the routing lists,
// the launch of the pass over z (balance.cuh), and the sums of its blocks.
#include "eqb_device.cuh"

namespace eqb {

namespace {

constexpr int kCountThreads = 256;

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
  const int E = a.E, K = a.K, threads = static_cast<int>(blockDim.x);
  int32_t* mine = hist + static_cast<int>((threadIdx.x >> 5) % copies) * E;
  for (int i = threadIdx.x; i < copies * E; i += threads) hist[i] = 0;
  griddep_wait();
  griddep_launch();  // the pass over z may start its loads: what came before the call is complete
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
      // an entry's token, which goes on by threads / K
      const int whole = threads / K, part = threads - whole * K;
      int token = static_cast<int>(threadIdx.x) / K, in = static_cast<int>(threadIdx.x) - token * K;
      for (int i = threadIdx.x; i < m; i += 4 * threads) {  // four entries in flight
        int e[4];
        uint8_t ok[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int j = i + u * threads;
          e[u] = j < m ? __ldcs(idx + j) : -1;
          ok[u] = j < m ? a.mask[t + token] : 0;
          token += whole;
          in += part;
          if (in >= K) {
            in -= K;
            ++token;
          }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (ok[u]) count(e[u]);
      }
    } else {
      // four entries a load, two loads in flight; single ones up to the first
      // 16-byte boundary and at the end
      const int head = min(m, static_cast<int>((16u - (reinterpret_cast<uintptr_t>(idx) & 15u)) & 15u) / 4);
      const int quads = (m - head) / 4;
      const int4* q4 = reinterpret_cast<const int4*>(idx + head);
      for (int i = threadIdx.x; i < quads; i += 2 * threads) {
        const bool two = i + threads < quads;
        const int4 w0 = __ldcs(q4 + i);
        const int4 w1 = two ? __ldcs(q4 + i + threads) : make_int4(-1, -1, -1, -1);
        count(w0.x); count(w0.y); count(w0.z); count(w0.w);
        count(w1.x); count(w1.y); count(w1.z); count(w1.w);
      }
      if (static_cast<int>(threadIdx.x) < head) count(idx[threadIdx.x]);
      const int end = head + 4 * quads + static_cast<int>(threadIdx.x);
      if (end < m) count(idx[end]);
    }
    if (a.mask) {
      int v = 0;
      for (int64_t i = t + threadIdx.x; i < seg_end; i += threads) v += a.mask[i] != 0;
      v = __reduce_add_sync(kFull, v);
      if ((threadIdx.x & 31) == 0 && v) atomicAdd(a.valid + l, v);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += threads) {
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
  __shared__ double tot[W][2];
  griddep_wait();
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  for (int l = blockIdx.y; l < a.M; l += gridDim.y) {
    const int64_t lo = min(max(__ldg(a.off + l), int64_t(0)), a.T), hi = min(max(__ldg(a.off + l + 1), lo), a.T);
    const int64_t n = a.mask ? a.valid[l] : hi - lo;
    // tokens are fewer than 2^31
    const uint32_t first = static_cast<uint32_t>(lo) / tokens_per_cta;
    const int rows = hi > lo ? static_cast<int>(static_cast<uint32_t>(hi - 1) / tokens_per_cta - first) + 1 : 0;
    const float* p = a.part + (static_cast<int64_t>(first) + l) * a.row;
    const int e = blockIdx.x * 32 + lane;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (e < a.E && a.prob)
      for (int q = wid; q < rows; q += 8 * W) {  // eight loads in flight
        float w[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) w[u] = q + W * u < rows ? __ldcg(p + static_cast<int64_t>(q + W * u) * a.row + 4 + e) : 0.f;
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u & 3] += w[u];
      }
    if (W > 1) col[wid][lane] = (v[0] + v[1]) + (v[2] + v[3]);
    const bool sums = blockIdx.x == 0 && a.loss;
    double t2[2] = {0.0, 0.0};
    if (sums) {
      for (int q = threadIdx.x; q < rows; q += 32 * W) {
        const float2 w = __ldcg(reinterpret_cast<const float2*>(p + static_cast<int64_t>(q) * a.row));
        t2[0] += w.x; t2[1] += w.y;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int m = 1; m < 32; m <<= 1) t2[i] += __shfl_xor_sync(kFull, t2[i], m);
        if (lane == 0) tot[wid][i] = t2[i];
      }
    }
    __syncthreads();
    if (wid == 0 && e < a.E && a.prob) {
      float x = (v[0] + v[1]) + (v[2] + v[3]);
#pragma unroll
      for (int q = 1; q < W; ++q) x += col[q][lane];
      a.prob[static_cast<int64_t>(l) * a.E + e] = n > 0 ? x / static_cast<float>(n) : 0.f;
    }
    if (sums && threadIdx.x == 0) {
      double h = 0.0, zz = 0.0;
#pragma unroll
      for (int q = 0; q < W; ++q) {
        h += tot[q][0];
        zz += tot[q][1];
      }
      const float n1 = static_cast<float>(n);
      a.loss[2 * l] = n > 0 ? static_cast<float>(a.alpha) * (static_cast<float>(h) / n1) : 0.f;
      a.loss[2 * l + 1] = n > 0 ? static_cast<float>(a.zeta) * (static_cast<float>(zz) / n1) : 0.f;
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
  // fewer threads a block where a microbatch's lists are shorter than four
  // entries for each of 256, and more blocks
  const int64_t mean = a.T / a.M * a.K;
  int threads = kCountThreads;
  while (threads > 32 && threads * 4 > mean) threads /= 2;
  // a block a microbatch of mean length, or 4,096 entries of a longer one where
  // that leaves every SM a block: its counts then go to global memory once
  int64_t least = a.K * (a.T / a.M) < 4096 ? a.T / a.M : 4096 / a.K;
  if (least > a.T / di.sm_count) least = a.T / di.sm_count;
  if (least < threads / 4) least = threads / 4;
  const int64_t most = di.sm_count * 8 * (kCountThreads / threads);
  int64_t grid = (a.T + least - 1) / least;
  if (grid > most) grid = most;
  const int64_t tpc = (a.T + grid - 1) / grid;
  int copies = threads / 32;
  if (a.E > 512 && copies > 4) copies = 4;
  return launch_dependent(balance_count_kernel, dim3(static_cast<unsigned>((a.T + tpc - 1) / tpc)), dim3(threads),
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
