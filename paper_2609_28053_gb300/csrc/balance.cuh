// balance.cuh -- the balance loss with its gradient: what its kernels share.
//
// For the n valid tokens of a microbatch (a token may be masked out) and the
// counts f_e of its experts' lists, F_e = f_e / (K n):
//   p_t  = softmax(z_t), or sigmoid(z_t) over its sum,
//   loss = alpha sum_e F_e P_e (P = mean of p_t) + zeta mean(lse_t^2),
//   d loss / d z_{t,j} = p_j (alpha / n (F_j - p.F) + 2 zeta / n lse)       (softmax)
//                      = p_j (1 - s_j) alpha / n (F_j - p.F)                (sigmoid),
// F a constant.  The counts come from the lists alone (4 K bytes a token), so
// once they are there a single pass over z gives the loss and the gradient.
// R_e = F_e - 1/E takes the place of F_e: p.F = p.R + 1/E, and R is formed from
// an exact whole number, so that balanced counts give exactly 0.
#pragma once

#include "eqb_device.cuh"

namespace eqb {

namespace {

constexpr int kBalThreads = 256;
constexpr int kBalWarps = kBalThreads / 32;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float ex2_approx(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Sum over the lanes that share `lane & (step - 1)` (step a power of two).
__device__ __forceinline__ float sum_slots(float x, int step) {
  for (int m = step; m < 32; m <<= 1) x += __shfl_xor_sync(kFull, x, m);
  return x;
}

// One block takes a contiguous range of tokens and walks the microbatches in
// it.  LPT lanes share a token, eight experts a lane and chunk (CPL chunks a
// lane where E > 256); U tokens a lane are in flight.  The sums of a
// microbatch's tokens go to the row blockIdx + microbatch of a.part, which no
// other pair of the two has, and are added up in ascending order by
// balance_finish: no atomics, so the same call gives the same bits.
template <bool SIG, bool GRAD, bool F32, int LPT, int CPL>
__global__ void __launch_bounds__(kBalThreads) balance_kernel(BalanceArgs a, int64_t tokens_per_cta) {
  constexpr int TPW = 32 / LPT;  // tokens a warp takes at a time
  constexpr int U = CPL > 1 ? 1 : 2;
  constexpr int EM = LPT * CPL * 8;  // experts the lanes hold
  __shared__ __align__(16) float Rs[EM];
  __shared__ __align__(16) float colsum[kBalWarps][EM];
  __shared__ float sums[kBalWarps][3];
  __shared__ double inv;  // 1 / (K n E)
  __shared__ float cs[2];
  const int E = a.E, nch = E >> 3;
  griddep_wait();
  const int64_t tb = static_cast<int64_t>(blockIdx.x) * tokens_per_cta;
  const int64_t te = min(tb + tokens_per_cta, a.T);
  if (tb >= te) return;
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const int sub = lane & (LPT - 1), slot = lane / LPT;
  const float gs = GRAD && a.grad_scale ? *a.grad_scale : 1.0f;

  int64_t t = tb;
  while (t < te) {
    const int l = microbatch_of(a.off, a.M, t);
    const int64_t lo = __ldg(a.off + l), hi = __ldg(a.off + l + 1);
    // malformed offsets must not stall the loop
    const int64_t seg_end = hi > t ? min(te, hi) : te;
    const int64_t n = a.mask ? a.valid[l] : hi - lo;
    __syncthreads();  // the previous microbatch is done with the shared values
    if (threadIdx.x == 0) {
      inv = n > 0 ? 1.0 / (static_cast<double>(a.K) * static_cast<double>(n) * static_cast<double>(E)) : 0.0;
      cs[0] = n > 0 ? gs * __double2float_rn(a.alpha / static_cast<double>(n)) : 0.f;
      cs[1] = n > 0 ? gs * __double2float_rn(2.0 * a.zeta / static_cast<double>(n)) : 0.f;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < EM; e += kBalThreads) {
      float r = 0.f;
      if (e < E) {
        const int64_t f = a.counts[static_cast<int64_t>(l) * E + e];
        r = __double2float_rn(static_cast<double>(f * E - static_cast<int64_t>(a.K) * n) * inv);
      }
      Rs[e] = r;
    }
    __syncthreads();
    float r[CPL][8], acc[CPL][8];
#pragma unroll
    for (int k = 0; k < CPL; ++k) {
      const float4 r0 = reinterpret_cast<const float4*>(Rs)[2 * (sub + k * LPT)];
      const float4 r1 = reinterpret_cast<const float4*>(Rs)[2 * (sub + k * LPT) + 1];
      r[k][0] = r0.x; r[k][1] = r0.y; r[k][2] = r0.z; r[k][3] = r0.w;
      r[k][4] = r1.x; r[k][5] = r1.y; r[k][6] = r1.z; r[k][7] = r1.w;
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[k][i] = 0.f;
    }
    const float ca = cs[0], cz = cs[1];
    float hsum = 0.f, zsum = 0.f, alive_n = 0.f;

    const int64_t stride = kBalWarps * TPW;
    for (int64_t base = t + static_cast<int64_t>(wid) * TPW; base < seg_end; base += U * stride) {
      float z[U][CPL][8];
      bool ok[U];  // a token of the range that counts
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t tok = base + u * stride + slot;
        ok[u] = tok < seg_end && (!a.mask || a.mask[tok]);
#pragma unroll
        for (int k = 0; k < CPL; ++k) {
          const int c = sub + k * LPT;
          const bool have = ok[u] && c < nch;
          if constexpr (F32) {
            const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(a.z) + tok * E) + 2 * c;
            const float4 none = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            const float4 w0 = have ? __ldcs(p) : none, w1 = have ? __ldcs(p + 1) : none;
            z[u][k][0] = w0.x; z[u][k][1] = w0.y; z[u][k][2] = w0.z; z[u][k][3] = w0.w;
            z[u][k][4] = w1.x; z[u][k][5] = w1.y; z[u][k][6] = w1.z; z[u][k][7] = w1.w;
          } else {
            const uint32_t none = 0xff80ff80u;  // -inf
            const uint4 w = have ? __ldcs(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.z) + tok * E) + c)
                                 : make_uint4(none, none, none, none);
            z[u][k][0] = bf16_lo(w.x); z[u][k][1] = bf16_hi(w.x);
            z[u][k][2] = bf16_lo(w.y); z[u][k][3] = bf16_hi(w.y);
            z[u][k][4] = bf16_lo(w.z); z[u][k][5] = bf16_hi(w.z);
            z[u][k][6] = bf16_lo(w.w); z[u][k][7] = bf16_hi(w.w);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t tok = base + u * stride + slot;
        float top = -INFINITY;
#pragma unroll
        for (int k = 0; k < CPL; ++k)
#pragma unroll
          for (int i = 0; i < 8; ++i) top = fmaxf(top, z[u][k][i]);
#pragma unroll
        for (int m = 1; m < LPT; m <<= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, m));
        // a row without a finite logit has no probabilities (nor has a masked one)
        const bool alive = ok[u] && top > -INFINITY;
        // sigmoids are taken relative to e^top where all are far below 0.5:
        // s e^-top = 1 / (e^top + e^(top - z))
        const float ref = !alive ? 0.f : SIG ? fminf(top, 0.f) : top;
        const float m2 = ref * kLog2e;
        const float em = SIG ? ex2_approx(m2) : 0.f;
        float w[CPL][8];  // 1 - s (sigmoid with gradient)
        float d = 0.f, h = 0.f;
#pragma unroll
        for (int k = 0; k < CPL; ++k)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if constexpr (SIG) {
              const float x = ex2_approx(__fmaf_rn(z[u][k][i], -kLog2e, m2));
              const float s = rcp_approx(em + x);
              if constexpr (GRAD) w[k][i] = fminf(x, 0x1p120f) * s;
              z[u][k][i] = s;
            } else {
              z[u][k][i] = ex2_approx(__fmaf_rn(z[u][k][i], kLog2e, -m2));
            }
            d += z[u][k][i];
            h = __fmaf_rn(z[u][k][i], r[k][i], h);
          }
#pragma unroll
        for (int m = 1; m < LPT; m <<= 1) {
          d += __shfl_xor_sync(kFull, d, m);
          h += __shfl_xor_sync(kFull, h, m);
        }
        if (alive && !(d < INFINITY)) raise_flag(a.err, kErrNonfinite);
        const float id = alive ? __frcp_rn(d) : 0.f;
        h *= id;
        float lse = 0.f;
        if (!SIG && a.zeta != 0.0) lse = alive ? top + logf(d) : 0.f;
        if (sub == 0) {
          hsum += h;
          zsum = __fmaf_rn(lse, lse, zsum);
          alive_n += alive ? 1.f : 0.f;
        }
        const float cl = cz * lse;
#pragma unroll
        for (int k = 0; k < CPL; ++k) {
          const int c = sub + k * LPT;
          float gr[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float p = z[u][k][i] * id;
            acc[k][i] += p;
            if constexpr (GRAD) {
              float q = __fmaf_rn(ca, r[k][i] - h, cl);
              if constexpr (SIG) q *= w[k][i];
              gr[i] = p * q;
            }
          }
          if constexpr (GRAD) {
            if (tok >= seg_end || c >= nch) continue;
            if (a.grad_in) {
              const float4* gp = reinterpret_cast<const float4*>(a.grad_in + tok * E) + 2 * c;
              const float4 g0 = __ldcs(gp), g1 = __ldcs(gp + 1);
              gr[0] += g0.x; gr[1] += g0.y; gr[2] += g0.z; gr[3] += g0.w;
              gr[4] += g1.x; gr[5] += g1.y; gr[6] += g1.z; gr[7] += g1.w;
            }
            if (a.grad_bf16) {
              __stcs(reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.grad_out) + tok * E) + c,
                     make_uint4(pack_bf16x2_rn(gr[0], gr[1]), pack_bf16x2_rn(gr[2], gr[3]), pack_bf16x2_rn(gr[4], gr[5]),
                                pack_bf16x2_rn(gr[6], gr[7])));
            } else {
              float4* op = reinterpret_cast<float4*>(static_cast<float*>(a.grad_out) + tok * E) + 2 * c;
              __stcs(op, make_float4(gr[0], gr[1], gr[2], gr[3]));
              __stcs(op + 1, make_float4(gr[4], gr[5], gr[6], gr[7]));
            }
          }
        }
      }
    }

    // the block's sums of this microbatch
    if (a.part) {
      float* row = a.part + (static_cast<int64_t>(blockIdx.x) + l) * a.row;
#pragma unroll
      for (int k = 0; k < CPL; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float v = sum_slots(acc[k][i], LPT);
          if (slot == 0) colsum[wid][(sub + k * LPT) * 8 + i] = v;
        }
      hsum = sum_slots(hsum, 1);
      zsum = sum_slots(zsum, 1);
      alive_n = sum_slots(alive_n, 1);
      if (lane == 0) {
        sums[wid][0] = hsum;
        sums[wid][1] = zsum;
        sums[wid][2] = alive_n;
      }
      __syncthreads();
      for (int e = threadIdx.x; e < E; e += kBalThreads) {
        float v = 0.f;
#pragma unroll
        for (int q = 0; q < kBalWarps; ++q) v += colsum[q][e];
        row[4 + e] = v;
      }
      if (threadIdx.x < 3) {
        float v = 0.f;
#pragma unroll
        for (int q = 0; q < kBalWarps; ++q) v += sums[q][threadIdx.x];
        row[threadIdx.x] = v;
      }
    }
    t = seg_end;
  }
}

template <bool SIG, bool GRAD, bool F32, int LPT, int CPL>
int launch_bal(const BalanceArgs& a, int64_t tokens_per_cta, cudaStream_t s) {
  const int64_t grid = (a.T + tokens_per_cta - 1) / tokens_per_cta;
  return launch_dependent(balance_kernel<SIG, GRAD, F32, LPT, CPL>, dim3(static_cast<unsigned>(grid)), dim3(kBalThreads), 0,
                          s, a, tokens_per_cta) == cudaSuccess
             ? kOk
             : kErrCuda;
}

template <bool SIG, bool GRAD, bool F32>
int launch_bal_width(const BalanceArgs& a, int64_t tpc, cudaStream_t s) {
  const int nch = a.E >> 3;
  if (nch <= 1) return launch_bal<SIG, GRAD, F32, 1, 1>(a, tpc, s);
  if (nch <= 2) return launch_bal<SIG, GRAD, F32, 2, 1>(a, tpc, s);
  if (nch <= 4) return launch_bal<SIG, GRAD, F32, 4, 1>(a, tpc, s);
  if (nch <= 8) return launch_bal<SIG, GRAD, F32, 8, 1>(a, tpc, s);
  if (nch <= 16) return launch_bal<SIG, GRAD, F32, 16, 1>(a, tpc, s);
  if (nch <= 32) return launch_bal<SIG, GRAD, F32, 32, 1>(a, tpc, s);
  if (nch <= 48) return launch_bal<SIG, GRAD, F32, 16, 3>(a, tpc, s);
  if (nch <= 64) return launch_bal<SIG, GRAD, F32, 32, 2>(a, tpc, s);
  if (nch <= 96) return launch_bal<SIG, GRAD, F32, 32, 3>(a, tpc, s);
  if (nch <= 128) return launch_bal<SIG, GRAD, F32, 32, 4>(a, tpc, s);
  return kErrUnsupported;
}

template <bool SIG, bool GRAD>
int launch_bal_type(const BalanceArgs& a, int64_t tpc, cudaStream_t s) {
  return a.z_fp32 ? launch_bal_width<SIG, GRAD, true>(a, tpc, s) : launch_bal_width<SIG, GRAD, false>(a, tpc, s);
}

}  // namespace

}  // namespace eqb
