// gate.cu -- the gate: experts and weights of every token from its logits, with
// experts in groups, and the gradient of the weights.
//
//   c_e = z_e + b_e decides (fp32, one rounding: the same bits as routing's
//   scores), groups are ranked by their largest or two largest c, and the weights
//   come from the unbiased z (sigmoid or softmax).
//
// A warp takes a token, eight neighbouring experts a lane and pass of 256.  c is
// kept as an unsigned key that orders as the value does, so that a round of the
// selection is one maximum over the warp and one minimum over the experts that
// have it.
#include "eqb_device.cuh"

namespace eqb {

namespace {

constexpr int kGateWarps = 4;
constexpr uint32_t kClosed = 0x007fffffu;  // the key of -inf: an open expert's is larger

// Order-preserving key of a float; -0 as +0.
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t u = __float_as_uint(__fadd_rn(v, 0.0f));
  return u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}

template <class F>
__device__ __forceinline__ float warp_all(float v, F f) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = f(v, __shfl_xor_sync(kFull, v, o));
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
  return warp_all(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float warp_sum(float v) {
  return warp_all(v, [](float a, float b) { return __fadd_rn(a, b); });
}

// Eight logits from expert e0 of a row on.
template <bool F32>
__device__ __forceinline__ void load8(const void* z, int64_t at, float (&v)[8]) {
  if (F32) {
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(z) + at);
    const float4 x = __ldg(p), y = __ldg(p + 1);
    v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
    v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
  } else {
    const uint4 x = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(z) + at));
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = bf16_lo(w[i]);
      v[2 * i + 1] = bf16_hi(w[i]);
    }
  }
}
template <bool F32>
__device__ __forceinline__ float load1(const void* z, int64_t at) {
  return F32 ? __ldg(static_cast<const float*>(z) + at) : bf16_bits_to_f32(__ldg(static_cast<const uint16_t*>(z) + at));
}

// sigmoid(z) of the entries that are there (z = -inf: not), each divided by their
// sum.  The sigmoids are taken relative to exp(m), m = min(0, largest z), so that
// however low the logits are the largest one does not underflow.
__device__ __forceinline__ float sigmoid_share(float z) {
  const float m = fminf(warp_max(z), 0.f);
  if (m == -INFINITY) return 0.f;
  const float u = z > 0.f ? 1.f / (1.f + expf(-z)) : expf(z - m) / (1.f + expf(z));
  return u / warp_sum(u);
}
__device__ __forceinline__ float softmax_share(float z) {
  const float m = warp_max(z);
  if (m == -INFINITY) return 0.f;
  const float u = expf(z - m);
  return u / warp_sum(u);
}

template <int NC, bool F32>
__global__ void __launch_bounds__(kGateWarps * 32) gate_warp_kernel(const GateArgs a) {
  __shared__ float rows[kGateWarps][NC * 256];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, E = a.E, K = a.K;
  const bool grouped = a.top_groups < a.groups;
  const int gs = E / a.groups;
  // lanes of a group in the ranking of groups
  int per = 32;
  while (per * a.groups > 32) per >>= 1;
  const bool softmax_all = !a.sigmoid && !a.renorm;
  griddep_wait();
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * kGateWarps + warp; t < a.T; t += static_cast<int64_t>(gridDim.x) * kGateWarps) {
    int mine = -1;  // lane k: the k-th expert
    float zmax = -INFINITY, zsum = 0.f;
    if (!a.mask || a.mask[t]) {
      uint32_t key[NC][8];
      bool bad = false;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int e0 = c * 256 + lane * 8;
        float z[8], b[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          z[j] = -INFINITY;
          b[j] = 0.f;
        }
        if (e0 < E) {
          load8<F32>(a.z, t * E + e0, z);
          if (a.b) {
#pragma unroll
            for (int j = 0; j < 8; ++j) b[j] = __ldg(a.b + e0 + j);
          }
        }
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float v = __fadd_rn(z[j], b[j]);
          bad |= !(v < INFINITY);
          key[c][j] = key_of(v);
          top = fmaxf(top, z[j]);
          if (grouped) rows[warp][e0 + j] = v;
        }
        if (softmax_all) {  // the running maximum and sum
          const float m = fmaxf(zmax, top);
          if (m > -INFINITY) {
            zsum = zsum * expf(zmax - m);
#pragma unroll
            for (int j = 0; j < 8; ++j) zsum = zsum + expf(z[j] - m);
            zmax = m;
          }
        }
      }
      if (__any_sync(kFull, bad) && lane == 0) raise_flag(a.err, kErrNonfinite);
      if (softmax_all) {
        const float m = warp_max(zmax);
        zsum = warp_sum(zmax > -INFINITY ? zsum * expf(zmax - m) : 0.f);
        zmax = m;
      }
      if (grouped) {
        __syncwarp();
        const int g = lane / per;
        float m1 = -INFINITY, m2 = -INFINITY;
        if (g < a.groups)
          for (int i = lane % per; i < gs; i += per) {
            const float v = rows[warp][g * gs + i];
            m2 = fmaxf(m2, fminf(m1, v));
            m1 = fmaxf(m1, v);
          }
        for (int o = per >> 1; o > 0; o >>= 1) {
          const float n1 = __shfl_xor_sync(kFull, m1, o), n2 = __shfl_xor_sync(kFull, m2, o);
          m2 = fmaxf(fmaxf(m2, n2), fminf(m1, n1));
          m1 = fmaxf(m1, n1);
        }
        const float score = a.top2 && m2 > -INFINITY ? __fadd_rn(m1, m2) : m1;
        int ahead = 0;
        for (int j = 0; j < a.groups; ++j) {
          const float s = __shfl_sync(kFull, score, j * per);
          ahead += s > score || (s == score && j < g);
        }
        const uint32_t open = __ballot_sync(kFull, g < a.groups && ahead < a.top_groups);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int e = c * 256 + lane * 8 + j;
            if (e < E && !(open >> (e / gs * per) & 1u)) key[c][j] = 0u;
          }
        __syncwarp();  // the row is read
      }
      for (int k = 0; k < K; ++k) {
        uint32_t best = 0u;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int j = 0; j < 8; ++j) best = max(best, key[c][j]);
        best = __reduce_max_sync(kFull, best);
        if (best <= kClosed) break;
        uint32_t e = 0xffffffffu;
#pragma unroll
        for (int c = NC - 1; c >= 0; --c)
#pragma unroll
          for (int j = 7; j >= 0; --j)
            if (key[c][j] == best) e = static_cast<uint32_t>(c * 256 + lane * 8 + j);
        e = __reduce_min_sync(kFull, e);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (static_cast<uint32_t>(c * 256 + lane * 8 + j) == e) key[c][j] = 0u;
        if (lane == k) mine = min(static_cast<int>(e), E - 1);
      }
    }
    if (lane < K) a.idx[t * K + lane] = mine;
    if (a.weight) {
      const float z = mine >= 0 ? load1<F32>(a.z, t * E + mine) : -INFINITY;
      float w;
      if (a.renorm) w = a.sigmoid ? sigmoid_share(z) : softmax_share(z);
      else if (a.sigmoid) w = 1.f / (1.f + expf(-z));
      else w = mine >= 0 ? expf(z - zmax) / zsum : 0.f;
      if (lane < K) a.weight[t * K + lane] = w * a.scale;
    }
  }
}

// A warp a token.  The row is written from eight neighbouring experts a lane, then
// the list's entries once more by the lanes that hold them (the barrier of the warp
// between the two orders the stores).
template <bool F32, bool BF16>
__global__ void __launch_bounds__(kGateWarps * 32) gate_grad_kernel(const GateGradArgs a) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, E = a.E, K = a.K;
  const bool dense = !a.sigmoid && !a.renorm;
  const bool in_place = a.grad_in && a.grad_out == static_cast<const void*>(a.grad_in);
  griddep_wait();
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * kGateWarps + warp; t < a.T; t += static_cast<int64_t>(gridDim.x) * kGateWarps) {
    int e = -1;
    float g = 0.f, z = -INFINITY, old = 0.f;
    if (lane < K) {
      e = a.idx[t * K + lane];
      if (e < 0 || e >= E) e = -1;
    }
    if (e >= 0) {
      g = a.gw[t * K + lane];
      z = load1<F32>(a.z, t * E + e);
      if (a.grad_in) old = a.grad_in[t * E + e];
    }
    const bool any = __any_sync(kFull, e >= 0);
    float d = 0.f, zmax = -INFINITY, rest = 0.f;  // rest: -scale gb / sum, the factor of exp(z_j - zmax) for every j
    if (any) {
      if (dense) {
        float sum = 0.f;
        for (int e0 = lane * 8; e0 < E; e0 += 256) {
          float v[8];
          load8<F32>(a.z, t * E + e0, v);
          float top = v[0];
#pragma unroll
          for (int j = 1; j < 8; ++j) top = fmaxf(top, v[j]);
          const float m = fmaxf(zmax, top);
          if (m > -INFINITY) {
            sum = sum * expf(zmax - m);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = sum + expf(v[j] - m);
            zmax = m;
          }
        }
        const float m = warp_max(zmax);
        sum = warp_sum(zmax > -INFINITY ? sum * expf(zmax - m) : 0.f);
        zmax = m;
        const float p = e >= 0 && m > -INFINITY ? expf(z - m) / sum : 0.f;
        const float gb = warp_sum(p * g);
        rest = m > -INFINITY ? -(gb * a.scale) / sum : 0.f;
        // an expert named twice: its g's added, gb taken off once
        float both = g;
        bool first = true;
        for (int k = 0; k < K; ++k) {
          const int ek = __shfl_sync(kFull, e, k);
          const float gk = __shfl_sync(kFull, g, k);
          if (k != lane && ek == e && e >= 0) {
            both = both + gk;
            first &= k > lane;
          }
        }
        d = p * (both - gb) * a.scale;
        if (!first) e = -1;
      } else {
        if (!a.renorm) {
          const float s = 1.f / (1.f + expf(-z));
          d = e >= 0 ? g * s * (1.f / (1.f + expf(z))) * a.scale : 0.f;
        } else {
          const float w = a.sigmoid ? sigmoid_share(z) : softmax_share(z);
          const float gb = warp_sum(w * g);
          d = e >= 0 ? w * (g - gb) * a.scale : 0.f;
          if (a.sigmoid) d = d * (1.f / (1.f + expf(z)));
        }
        float both = d;
        bool first = true;
        for (int k = 0; k < K; ++k) {
          const int ek = __shfl_sync(kFull, e, k);
          const float dk = __shfl_sync(kFull, d, k);
          if (k != lane && ek == e && e >= 0) {
            both = both + dk;
            first &= k > lane;
          }
        }
        d = both;
        if (!first) e = -1;
      }
    }
    if (!(in_place && (!dense || !any))) {
      for (int e0 = lane * 8; e0 < E; e0 += 256) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.f;
        if (dense && any) {
          load8<F32>(a.z, t * E + e0, v);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = v[j] > -INFINITY ? expf(v[j] - zmax) * rest : 0.f;
        }
        if (a.grad_in) {
          const float4* p = reinterpret_cast<const float4*>(a.grad_in + t * E + e0);
          const float4 x = p[0], y = p[1];
          v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
          v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
        }
        if (BF16) {
          *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.grad_out) + t * E + e0) =
              make_uint4(pack_bf16x2_rn(v[0], v[1]), pack_bf16x2_rn(v[2], v[3]), pack_bf16x2_rn(v[4], v[5]), pack_bf16x2_rn(v[6], v[7]));
        } else {
          float4* p = reinterpret_cast<float4*>(static_cast<float*>(a.grad_out) + t * E + e0);
          p[0] = make_float4(v[0], v[1], v[2], v[3]);
          p[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
      }
      __syncwarp();
    }
    if (e >= 0) {
      const float v = old + d;
      if (BF16) static_cast<uint16_t*>(a.grad_out)[t * E + e] = static_cast<uint16_t>(pack_bf16x2_rn(v, 0.f));
      else static_cast<float*>(a.grad_out)[t * E + e] = v;
    }
  }
}

template <int NC>
int launch_gate_warp(const GateArgs& a, int grid, cudaStream_t s) {
  const cudaError_t e = a.z_fp32 ? launch_dependent(gate_warp_kernel<NC, true>, dim3(grid), dim3(kGateWarps * 32), 0, s, a)
                                 : launch_dependent(gate_warp_kernel<NC, false>, dim3(grid), dim3(kGateWarps * 32), 0, s, a);
  return e == cudaSuccess ? kOk : kErrCuda;
}

int warp_grid(int64_t T, const DeviceInfo& di) {
  const int64_t blocks = (T + kGateWarps - 1) / kGateWarps, most = static_cast<int64_t>(di.sm_count) * 32;
  return static_cast<int>(blocks < most ? blocks : most);
}

}  // namespace

int launch_gate(const GateArgs& a, cudaStream_t s) {
  DeviceInfo di;
  if (int rc = device_info(&di)) return rc;
  const int grid = warp_grid(a.T, di);
  if (a.E <= 256) return launch_gate_warp<1>(a, grid, s);
  if (a.E <= 512) return launch_gate_warp<2>(a, grid, s);
  return launch_gate_warp<4>(a, grid, s);
}

int launch_gate_grad(const GateGradArgs& a, cudaStream_t s) {
  DeviceInfo di;
  if (int rc = device_info(&di)) return rc;
  const dim3 grid(warp_grid(a.T, di)), block(kGateWarps * 32);
  cudaError_t e;
  if (a.z_fp32)
    e = a.grad_bf16 ? launch_dependent(gate_grad_kernel<true, true>, grid, block, 0, s, a)
                    : launch_dependent(gate_grad_kernel<true, false>, grid, block, 0, s, a);
  else
    e = a.grad_bf16 ? launch_dependent(gate_grad_kernel<false, true>, grid, block, 0, s, a)
                    : launch_dependent(gate_grad_kernel<false, false>, grid, block, 0, s, a);
  return e == cudaSuccess ? kOk : kErrCuda;
}

}  // namespace eqb
