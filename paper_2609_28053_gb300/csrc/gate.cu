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
#include "f32x2.cuh"

namespace eqb {

namespace {

constexpr int kGateWarps = 4;
// Up to here a warp a token.  us of a warp / of a thread a token (bf16, K = 8, sigmoids
// renormalised, launches in a graph) at T = 2,048, 4,096 and 8,192: E = 40 4.0 / 7.1, 5.6 /
// 7.2, 9.2 / 7.3; E = 128 4.2 / 5.9, 5.8 / 6.0, 9.5 / 6.2; E = 256 4.3 / 7.8, 6.3 / 8.1, 10.0 /
// 7.9, in 8 groups 6.6 / 8.2, 9.7 / 8.7, 15.4 / 8.4; E = 512 6.3 / 10.7, 9.3 / 11.2, 15.2 / 11.3,
// in 8 groups 9.6 / 11.0, 15.2 / 12.0, 24.3 / 11.8.  fp32 and softmax over all are alike: the
// two meet between 2,048 and about 8,192 tokens at every width from 8 to 512.
constexpr int64_t kFewGateTokens = 4096;
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

// Eight logits as they lie in memory.
template <bool F32>
struct Raw8 {
  uint4 q[F32 ? 2 : 1];
  __device__ __forceinline__ void load(const void* z, int64_t at) {
    const uint4* p = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(z) + at * (F32 ? 4 : 2));
    q[0] = __ldg(p);
    if (F32) q[F32 ? 1 : 0] = __ldg(p + 1);
  }
  __device__ __forceinline__ void fill(uint32_t w) {
#pragma unroll
    for (int i = 0; i < (F32 ? 2 : 1); ++i) q[i] = make_uint4(w, w, w, w);
  }
  __device__ __forceinline__ void unpack(float (&v)[8]) const {
    const uint32_t w[4] = {q[0].x, q[0].y, q[0].z, q[0].w};
    if (F32) {
      const uint4 y = q[F32 ? 1 : 0];
      v[0] = __uint_as_float(w[0]); v[1] = __uint_as_float(w[1]); v[2] = __uint_as_float(w[2]); v[3] = __uint_as_float(w[3]);
      v[4] = __uint_as_float(y.x); v[5] = __uint_as_float(y.y); v[6] = __uint_as_float(y.z); v[7] = __uint_as_float(y.w);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = bf16_lo(w[i]);
        v[2 * i + 1] = bf16_hi(w[i]);
      }
    }
  }
};
// Eight logits from element `at` on.
template <bool F32>
__device__ __forceinline__ void load8(const void* z, int64_t at, float (&v)[8]) {
  Raw8<F32> r;
  r.load(z, at);
  r.unpack(v);
}
template <bool F32>
__device__ __forceinline__ float load1(const void* z, int64_t at) {
  return F32 ? __ldg(static_cast<const float*>(z) + at) : bf16_bits_to_f32(__ldg(static_cast<const uint16_t*>(z) + at));
}

// 1 / (1 + exp(-z)).  From -88.7 down exp(-z) is infinite, where exp(z) is still a number
// (from -17 down the two are equal in fp32).
__device__ __forceinline__ float sigmoid_of(float z) {
  const bool low = z < -80.f;
  const float n = expf(low ? z : -z);
  return low ? n : 1.f / (1.f + n);
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
      else if (a.sigmoid) w = sigmoid_of(z);
      else w = mine >= 0 ? expf(z - zmax) / zsum : 0.f;
      if (lane < K) a.weight[t * K + lane] = w * a.scale;
    }
  }
}

// Sums and maxima over the LPT lanes of a token.
template <int LPT, class F>
__device__ __forceinline__ float lanes_all(float v, F f) {
#pragma unroll
  for (int o = LPT >> 1; o > 0; o >>= 1) v = f(v, __shfl_xor_sync(kFull, v, o));
  return v;
}
template <int LPT>
__device__ __forceinline__ float lanes_max(float v) {
  return lanes_all<LPT>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int LPT>
__device__ __forceinline__ float lanes_sum(float v) {
  return lanes_all<LPT>(v, [](float a, float b) { return __fadd_rn(a, b); });
}

// The gradient.  LPT lanes take a token, eight neighbouring experts each and pass
// (NC of them), and one entry of its list each.  The row is written from the
// lanes' experts, then the list's entries once more by the lanes that hold them; the
// barrier of the warp between the two orders the stores, and one before them what
// the entries' lanes have read of a row that is added to in place.
template <int LPT, int NC, bool dense, bool F32, bool BF16>
__global__ void __launch_bounds__(kGateWarps * 32) gate_grad_kernel(const GateGradArgs a) {
  constexpr int kTokens = 32 / LPT;  // of a warp
  constexpr float kLog2e = 1.4426950408889634f;
  const int lane = threadIdx.x & 31, sub = lane % LPT, E = a.E, K = a.K;
  const bool in_place = a.grad_in && a.grad_out == static_cast<const void*>(a.grad_in);
  const int64_t step = static_cast<int64_t>(gridDim.x) * kGateWarps * kTokens;
  griddep_wait();
  // what the next token needs is on its way while this one's gradient is formed
  Raw8<F32> row[NC];
  int next_e = -1;
  float next_g = 0.f;
  auto fetch = [&](int64_t t) {
    const bool live = t < a.T;
    if (dense) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int e0 = (c * LPT + sub) * 8;
        if (live && e0 < E) row[c].load(a.z, t * E + e0);
        else row[c].fill(F32 ? 0xff800000u : 0xff80ff80u);  // -inf
      }
    }
    next_e = -1;
    if (live && sub < K) {
      next_e = __ldg(a.idx + t * K + sub);
      next_g = __ldg(a.gw + t * K + sub);
    }
  };
  const int64_t first = (static_cast<int64_t>(blockIdx.x) * kGateWarps + (threadIdx.x >> 5)) * kTokens;
  fetch(first + lane / LPT);
  // a warp's tokens leave the loop together
  for (int64_t w0 = first; w0 < a.T; w0 += step) {
    const int64_t t = w0 + lane / LPT;
    const bool live = t < a.T;
    float v[NC][8];
    if constexpr (dense) {
#pragma unroll
      for (int c = 0; c < NC; ++c) row[c].unpack(v[c]);
    }
    int e = next_e >= 0 && next_e < E ? next_e : -1;
    float g = 0.f, z = -INFINITY, old = 0.f;
    if (e >= 0) {
      g = next_g;
      z = load1<F32>(a.z, t * E + e);
      if (a.grad_in) old = a.grad_in[t * E + e];
    }
    fetch(t + step);
    const uint32_t mine = LPT == 32 ? kFull : ((1u << (LPT & 31)) - 1u) << (lane / LPT * LPT);
    const bool any = (__ballot_sync(kFull, e >= 0) & mine) != 0u;
    // lanes of the token with the same expert: its terms are added, in the list's order, by the first
    const uint32_t same = __match_any_sync(kFull, e >= 0 ? e * kTokens + lane / LPT : -1 - lane);
    float d = 0.f;
    if (dense) {
      float top = -INFINITY;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, v[c][j]);
      top = lanes_max<LPT>(top);
      const float ref = top > -INFINITY ? top : 0.f;
      float sum = 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[c][j] = ex2_approx((v[c][j] - ref) * kLog2e);
          sum = sum + v[c][j];
        }
      sum = lanes_sum<LPT>(sum);
      const float f = sum > 0.f ? __fdiv_rn(1.f, sum) : 0.f;
      const float p = e >= 0 ? ex2_approx((z - ref) * kLog2e) * f : 0.f;
      const float gb = lanes_sum<LPT>(e >= 0 ? p * g : 0.f);
      const float rest = any ? -(gb * a.scale) * f : 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[c][j] = any ? v[c][j] * rest : 0.f;
      d = g;
      if (__any_sync(kFull, same & (same - 1u))) {
        d = 0.f;
        for (int k = 0; k < 32; ++k) {
          const float gk = __shfl_sync(kFull, g, k);
          if (same >> k & 1u) d = d + gk;
        }
      }
      d = p * (d - gb) * a.scale;
    } else {
      const float s1 = sigmoid_of(-z);  // 1 - s
      if (!a.renorm) {
        d = e >= 0 ? g * sigmoid_of(z) * s1 * a.scale : 0.f;
      } else {
        const float m = lanes_max<LPT>(z), ref = a.sigmoid ? fminf(m, 0.f) : m;
        float u = 0.f;
        if (e >= 0 && m > -INFINITY) u = !a.sigmoid ? expf(z - ref) : z > 0.f ? 1.f / (1.f + expf(-z)) : expf(z - ref) * s1;
        const float sum = lanes_sum<LPT>(u);
        const float w = sum > 0.f ? u / sum : 0.f;
        const float gb = lanes_sum<LPT>(e >= 0 ? w * g : 0.f);
        d = e >= 0 ? w * (g - gb) * a.scale : 0.f;
        if (a.sigmoid) d = d * s1;
      }
      if (__any_sync(kFull, same & (same - 1u))) {
        float both = 0.f;
        for (int k = 0; k < 32; ++k) {
          const float dk = __shfl_sync(kFull, d, k);
          if (same >> k & 1u) both = both + dk;
        }
        d = both;
      }
    }
    if (!in_place || dense) {
      if (dense) __syncwarp();
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int e0 = (c * LPT + sub) * 8;
        if (!live || e0 >= E) continue;
        if (!dense) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[c][j] = 0.f;
        }
        if (a.grad_in) {
          const float4* p = reinterpret_cast<const float4*>(a.grad_in + t * E + e0);
          const float4 x = p[0], y = p[1];
          v[c][0] += x.x; v[c][1] += x.y; v[c][2] += x.z; v[c][3] += x.w;
          v[c][4] += y.x; v[c][5] += y.y; v[c][6] += y.z; v[c][7] += y.w;
        }
        if (BF16) {
          *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.grad_out) + t * E + e0) =
              make_uint4(pack_bf16x2_rn(v[c][0], v[c][1]), pack_bf16x2_rn(v[c][2], v[c][3]), pack_bf16x2_rn(v[c][4], v[c][5]),
                         pack_bf16x2_rn(v[c][6], v[c][7]));
        } else {
          float4* p = reinterpret_cast<float4*>(static_cast<float*>(a.grad_out) + t * E + e0);
          p[0] = make_float4(v[c][0], v[c][1], v[c][2], v[c][3]);
          p[1] = make_float4(v[c][4], v[c][5], v[c][6], v[c][7]);
        }
      }
      __syncwarp();
    }
    if (e >= 0 && lane == __ffs(same) - 1) {
      const float x = old + d;
      if (BF16) static_cast<uint16_t*>(a.grad_out)[t * E + e] = static_cast<uint16_t>(pack_bf16x2_rn(x, 0.f));
      else static_cast<float*>(a.grad_out)[t * E + e] = x;
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

template <int LPT, int NC, bool dense>
int launch_gate_grad_t(const GateGradArgs& a, const DeviceInfo& di, cudaStream_t s) {
  const dim3 grid(warp_grid((a.T + 32 / LPT - 1) / (32 / LPT), di)), block(kGateWarps * 32);
  cudaError_t e;
  if (a.z_fp32)
    e = a.grad_bf16 ? launch_dependent(gate_grad_kernel<LPT, NC, dense, true, true>, grid, block, 0, s, a)
                    : launch_dependent(gate_grad_kernel<LPT, NC, dense, true, false>, grid, block, 0, s, a);
  else
    e = a.grad_bf16 ? launch_dependent(gate_grad_kernel<LPT, NC, dense, false, true>, grid, block, 0, s, a)
                    : launch_dependent(gate_grad_kernel<LPT, NC, dense, false, false>, grid, block, 0, s, a);
  return e == cudaSuccess ? kOk : kErrCuda;
}

template <bool dense>
int launch_gate_grad_d(const GateGradArgs& a, const DeviceInfo& di, cudaStream_t s) {
  int lanes = 8;  // of a token: as many as its list has entries, and a pass for its experts
  while (lanes < 32 && (lanes * 8 < a.E || lanes < a.K)) lanes *= 2;
  if (lanes == 8) return launch_gate_grad_t<8, 1, dense>(a, di, s);
  if (lanes == 16) return launch_gate_grad_t<16, 1, dense>(a, di, s);
  if (a.E <= 256) return launch_gate_grad_t<32, 1, dense>(a, di, s);
  if (a.E <= 512) return launch_gate_grad_t<32, 2, dense>(a, di, s);
  return launch_gate_grad_t<32, 4, dense>(a, di, s);
}

}  // namespace

int launch_gate(const GateArgs& a, cudaStream_t s) {
  DeviceInfo di;
  if (int rc = device_info(&di)) return rc;
  const int G = a.top_groups < a.groups ? a.groups : 1;
  if (a.T > kFewGateTokens && a.K <= 8 && a.E <= 512 && (G == 1 || G == 2 || G == 4 || G == 8) && a.E / 8 % G == 0)
    return a.z_fp32 ? launch_gate_tile_fp32(a, s) : launch_gate_tile_bf16(a, s);
  const int grid = warp_grid(a.T, di);
  if (a.E <= 256) return launch_gate_warp<1>(a, grid, s);
  if (a.E <= 512) return launch_gate_warp<2>(a, grid, s);
  return launch_gate_warp<4>(a, grid, s);
}

int launch_gate_grad(const GateGradArgs& a, cudaStream_t s) {
  DeviceInfo di;
  if (int rc = device_info(&di)) return rc;
  return !a.sigmoid && !a.renorm ? launch_gate_grad_d<true>(a, di, s) : launch_gate_grad_d<false>(a, di, s);
}

}  // namespace eqb
