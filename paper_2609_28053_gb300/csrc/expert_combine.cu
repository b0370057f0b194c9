// expert_combine.cu -- the weighted sum of a token's rows, and its gradients.
//
// Both stream: 2 n bytes of every row that a slot names, and of every token.  What
// bounds them is how many loads are on their way: a lane has eight neighbouring
// columns and asks for eight rows at a time (a row after the other: T = 16,411, n = 2,048, K = 8
// 118 us, its gradient at T = 16,384, n = 4,096 480 us; so 103 and 337).
#include "eqb_device.cuh"

namespace eqb {

namespace {

constexpr int kCombineWarps = 8;
constexpr int kRowsAhead = 8;  // rows, or parts of rows, of a token that are asked for together

__device__ __forceinline__ void unpack8(const uint4& x, float* v) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = bf16_lo(w[i]);
    v[2 * i + 1] = bf16_hi(w[i]);
  }
}
__device__ __forceinline__ uint4 pack8(const float* v) {
  return make_uint4(pack_bf16x2_rn(v[0], v[1]), pack_bf16x2_rn(v[2], v[3]), pack_bf16x2_rn(v[4], v[5]), pack_bf16x2_rn(v[6], v[7]));
}

// Slots k0 .. k0 + 7 of token t in lanes 0 .. 7 (-1 where one names no row), and the weights.
__device__ __forceinline__ int slots_of(const CombineArgs& a, int64_t t, int k0, int lane, float* w) {
  int r = -1;
  *w = 1.f;
  if (lane < kRowsAhead && k0 + lane < a.K) {
    r = __ldg(a.slot + t * a.K + k0 + lane);
    if (r < 0 || r >= a.R) r = -1;
    if (a.weight) *w = __ldg(a.weight + t * a.K + k0 + lane);
  }
  return r;
}

// A warp takes 256 columns of a token; the sums stay in registers, in ascending k.
__global__ void __launch_bounds__(kCombineWarps * 32) combine_kernel(const CombineArgs a, int strips) {
  const int lane = threadIdx.x & 31;
  const int64_t items = a.T * strips;
  griddep_wait();
  for (int64_t it = static_cast<int64_t>(blockIdx.x) * kCombineWarps + (threadIdx.x >> 5); it < items;
       it += static_cast<int64_t>(gridDim.x) * kCombineWarps) {
    const int64_t t = it / strips;
    const int j = static_cast<int>(it - t * strips) * 256 + lane * 8;
    float acc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = 0.f;
    for (int k0 = 0; k0 < a.K; k0 += kRowsAhead) {
      float w;
      const int r = slots_of(a, t, k0, lane, &w);
      uint4 x[kRowsAhead];
#pragma unroll
      for (int k = 0; k < kRowsAhead; ++k) {
        const int rk = __shfl_sync(kFull, r, k);
        x[k] = rk >= 0 && j < a.n ? __ldg(reinterpret_cast<const uint4*>(a.rows + static_cast<int64_t>(rk) * a.n + j))
                                  : make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
      for (int k = 0; k < kRowsAhead; ++k) {
        const float wk = __shfl_sync(kFull, r >= 0 ? w : 0.f, k);
        float v[8];
        unpack8(x[k], v);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = __fmaf_rn(wk, v[i], acc[i]);
      }
    }
    if (j < a.n) *reinterpret_cast<uint4*>(a.out + t * a.n + j) = pack8(acc);
  }
}

// A warp a token, N of its rows and M parts of 256 columns at a time (N M = 8): the rows' dot
// products stay in the lanes' registers over all columns.
template <int N>
__global__ void __launch_bounds__(kCombineWarps * 32, 2) combine_grad_kernel(const CombineArgs a) {
  constexpr int M = kRowsAhead / N;
  const int lane = threadIdx.x & 31;
  griddep_wait();
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * kCombineWarps + (threadIdx.x >> 5); t < a.T;
       t += static_cast<int64_t>(gridDim.x) * kCombineWarps) {
    for (int k0 = 0; k0 < a.K; k0 += N) {
      float w;
      const int r = slots_of(a, t, k0, lane, &w);
      int rk[N];
      float wk[N], dot[N];
#pragma unroll
      for (int k = 0; k < N; ++k) {
        rk[k] = __shfl_sync(kFull, r, k);
        wk[k] = __shfl_sync(kFull, w, k);
        dot[k] = 0.f;
      }
#pragma unroll 1
      for (int j0 = lane * 8; j0 < a.n; j0 += 256 * M) {
        uint4 x[N][M], gr[M];
#pragma unroll
        for (int m = 0; m < M; ++m) {
          const int j = j0 + 256 * m;
          const bool in = M == 1 || j < a.n;
          gr[m] = in ? __ldg(reinterpret_cast<const uint4*>(a.grad + t * a.n + j)) : make_uint4(0u, 0u, 0u, 0u);
          if (a.gw) {
#pragma unroll
            for (int k = 0; k < N; ++k)
              x[k][m] = in && rk[k] >= 0 ? *reinterpret_cast<const uint4*>(a.rows + static_cast<int64_t>(rk[k]) * a.n + j)
                                         : make_uint4(0u, 0u, 0u, 0u);
          }
        }
#pragma unroll
        for (int m = 0; m < M; ++m) {
          const int j = j0 + 256 * m;
          float g[8];
          unpack8(gr[m], g);
#pragma unroll
          for (int k = 0; k < N; ++k) {
            if (a.gw) {
              float v[8];
              unpack8(x[k][m], v);
#pragma unroll
              for (int i = 0; i < 8; ++i) dot[k] = __fmaf_rn(g[i], v[i], dot[k]);
            }
            if (a.out && rk[k] >= 0 && (M == 1 || j < a.n)) {
              float v[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) v[i] = g[i] * wk[k];
              *reinterpret_cast<uint4*>(a.out + static_cast<int64_t>(rk[k]) * a.n + j) = pack8(v);
            }
          }
        }
      }
      if (a.gw) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) dot[k] = __fadd_rn(dot[k], __shfl_xor_sync(kFull, dot[k], o));
          if (lane == 0 && k0 + k < a.K) a.gw[t * a.K + k0 + k] = rk[k] >= 0 ? dot[k] : 0.f;
        }
      }
    }
  }
}

int grid_of(int64_t items, const DeviceInfo& di) {
  const int64_t blocks = (items + kCombineWarps - 1) / kCombineWarps, most = static_cast<int64_t>(di.sm_count) * 64;
  return static_cast<int>(blocks < most ? blocks : most);
}

}  // namespace

int launch_combine(const CombineArgs& a, cudaStream_t s) {
  DeviceInfo di;
  if (int rc = device_info(&di)) return rc;
  const int strips = (a.n + 255) / 256;
  return launch_dependent(combine_kernel, dim3(grid_of(a.T * strips, di)), dim3(kCombineWarps * 32), 0, s, a, strips) == cudaSuccess
             ? kOk
             : kErrCuda;
}

int launch_combine_grad(const CombineArgs& a, cudaStream_t s) {
  DeviceInfo di;
  if (int rc = device_info(&di)) return rc;
  const dim3 grid(grid_of(a.T, di)), block(kCombineWarps * 32);
  const cudaError_t e = a.K <= 2   ? launch_dependent(combine_grad_kernel<2>, grid, block, 0, s, a)
                        : a.K <= 4 ? launch_dependent(combine_grad_kernel<4>, grid, block, 0, s, a)
                                   : launch_dependent(combine_grad_kernel<8>, grid, block, 0, s, a);
  return e == cudaSuccess ? kOk : kErrCuda;
}

}  // namespace eqb
