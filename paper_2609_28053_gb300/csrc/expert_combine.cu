// expert_combine.cu -- the weighted sum of a token's rows, and its gradients.
//
// Both stream: 2 n bytes of every row that a slot names, and of every token.  A
// warp takes a part of 512 columns of a token, 16 a lane, and its K rows one after
// the other, so that the sums stay in registers and their order is fixed.
#include "eqb_device.cuh"

namespace eqb {

namespace {

constexpr int kCombineWarps = 8;

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

// The k-th slot of token t, -1 where it names no row.
__device__ __forceinline__ int64_t row_of(const CombineArgs& a, int64_t t, int k) {
  const int r = __ldg(a.slot + t * a.K + k);
  return r >= 0 && r < a.R ? r : -1;
}

__global__ void __launch_bounds__(kCombineWarps * 32) combine_kernel(const CombineArgs a, int strips) {
  const int lane = threadIdx.x & 31;
  const int64_t items = a.T * strips;
  griddep_wait();
  for (int64_t it = static_cast<int64_t>(blockIdx.x) * kCombineWarps + (threadIdx.x >> 5); it < items;
       it += static_cast<int64_t>(gridDim.x) * kCombineWarps) {
    const int64_t t = it / strips;
    const int j = static_cast<int>(it % strips) * 256 + lane * 8;
    if (j >= a.n) continue;
    float acc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = 0.f;
    for (int k = 0; k < a.K; ++k) {
      const int64_t r = row_of(a, t, k);
      if (r < 0) continue;
      const float w = a.weight ? __ldg(a.weight + t * a.K + k) : 1.f;
      float v[8];
      unpack8(__ldg(reinterpret_cast<const uint4*>(a.rows + r * a.n + j)), v);
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] = __fmaf_rn(w, v[i], acc[i]);
    }
    *reinterpret_cast<uint4*>(a.out + t * a.n + j) = pack8(acc);
  }
}

// A warp a token: its columns 256 at a time, the dot products of up to eight rows
// in the lanes' registers.
__global__ void __launch_bounds__(kCombineWarps * 32) combine_grad_kernel(const CombineArgs a) {
  const int lane = threadIdx.x & 31;
  griddep_wait();
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * kCombineWarps + (threadIdx.x >> 5); t < a.T;
       t += static_cast<int64_t>(gridDim.x) * kCombineWarps) {
    for (int k = 0; k < a.K; ++k) {
      const int64_t r = row_of(a, t, k);
      float dot = 0.f;
      if (r >= 0) {
        const float w = a.weight ? __ldg(a.weight + t * a.K + k) : 1.f;
        for (int j = lane * 8; j < a.n; j += 256) {
          float g[8], v[8];
          unpack8(__ldg(reinterpret_cast<const uint4*>(a.grad + t * a.n + j)), g);
          if (a.gw) {
            unpack8(*reinterpret_cast<const uint4*>(a.rows + r * a.n + j), v);
#pragma unroll
            for (int i = 0; i < 8; ++i) dot = __fmaf_rn(g[i], v[i], dot);
          }
          if (a.out) {
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] *= w;
            *reinterpret_cast<uint4*>(a.out + r * a.n + j) = pack8(g);
          }
        }
      }
      if (a.gw) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) dot = __fadd_rn(dot, __shfl_xor_sync(kFull, dot, o));
        if (lane == 0) a.gw[t * a.K + k] = dot;
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
  return launch_dependent(combine_grad_kernel, dim3(grid_of(a.T, di)), dim3(kCombineWarps * 32), 0, s, a) == cudaSuccess ? kOk
                                                                                                                          : kErrCuda;
}

}  // namespace eqb
