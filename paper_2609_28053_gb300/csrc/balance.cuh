// balance.cuh -- the balance loss with its gradient: the pass over z.
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
// an exact whole number, so that balanced counts give exactly 0.  The loss is the
// sum of p by F itself, from the sums of p: p.R + 1/E would cancel where the lists
// name experts of little probability.  Without a gradient nothing else needs the
// counts, and the pass runs beside the kernel that forms them (T = 524,288, E = 128,
// sigmoid: 50.5 us the call, 7 more with a product token by token behind the counts).
//
// The pass is a stream.  Rows lie one after the other, so each warp fetches its
// groups of up to 32 tokens (z and grad_in) by bulk copies into a ring of its
// own in shared memory: what is in flight does not depend on registers.  LPT
// lanes share a token, C chunks of four experts a lane, chunk k at LPT k + sub,
// so that fp32 and bf16 rows are both written in whole sectors.  Few lanes with
// many experts each (32 at E = 256), because what a token costs beside its
// experts -- three reductions over its lanes, a reciprocal, a logarithm -- is
// paid once for the tokens of a warp: with 32 lanes a token and 8 experts a
// lane E = 256 took 480 instructions a token, and issue slots bounded the pass.
#pragma once

#include "eqb_device.cuh"
#include "f32x2.cuh"
#include "mbarrier.cuh"

namespace eqb {

namespace {

constexpr int kBalThreads = 256;
constexpr int kBalWarps = kBalThreads / 32;
constexpr int kBalMaxStages = 4;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Sum over the lanes that share `lane & (step - 1)` (step a power of two).
__device__ __forceinline__ float sum_slots(float x, int step) {
  for (int m = step; m < 32; m <<= 1) x += __shfl_xor_sync(kFull, x, m);
  return x;
}

// A choice made once for a step, as a constant of the code below it.
struct Yes {
  __device__ constexpr operator bool() const { return true; }
};
struct No {
  __device__ constexpr operator bool() const { return false; }
};

// A launch's cut: tokens a block (0: a cluster of blocks a microbatch), blocks a
// cluster, tokens a group, stages of a warp's ring.
struct BalanceCut {
  int64_t tokens_per_cta;
  int cluster, group, stages;
};

// Blocks an SM holds, by their registers.
constexpr int bal_blocks(bool grad, int C) { return C <= 3 || (C == 4 && !grad) ? 3 : 2; }

// Rows of the block's column sums in shared memory: the warps add theirs in
// rounds where a row each would take much of it.
__host__ __device__ constexpr int bal_rows(int EM, int warps) { return EM <= 256 || warps < 2 ? warps : 2; }

// Shared memory: F [EM], a cluster's counts [EM], with a gradient R [EM], the
// warps' column sums [bal_rows, EM], the rings.
__host__ __device__ constexpr int bal_fixed_bytes(int EM, int warps, bool grad) {
  return 4 * EM * (2 + grad + bal_rows(EM, warps));
}
__host__ __device__ constexpr int bal_stage_bytes(int E, int group, bool f32, bool gin) {
  return group * E * ((f32 ? 4 : 2) + (gin ? 4 : 0));
}

// A word of the same place in another block's shared memory.
__device__ __forceinline__ uint32_t peer_word(const void* p, uint32_t rank) {
  uint32_t at, v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ float peer_float(const void* p, uint32_t rank) { return __uint_as_float(peer_word(p, rank)); }

// One block takes a contiguous range of tokens and walks the microbatches in
// it.  The sums of a microbatch's tokens go to the row blockIdx + microbatch of
// a.part, which no other pair of the two has, and balance_finish adds them up
// in ascending order: no atomics, so the same call gives the same bits.
// Of few tokens a cluster takes each microbatch, a slice a block, and does all
// of the call: the blocks count their lists, add up the cluster's counts, pass
// over z, and add up the cluster's sums, so that one launch takes the place of
// four.  The first CMIN chunks of every lane lie within E for all widths of an
// instance.
template <bool SIG, bool GRAD, bool F32, int LPT, int C, int CMIN>
__global__ void __launch_bounds__(kBalThreads, bal_blocks(GRAD, C)) balance_kernel(BalanceArgs a, BalanceCut cut) {
  constexpr int TPW = 32 / LPT;    // tokens a warp takes at a time
  constexpr int EM = LPT * C * 4;  // experts the lanes hold
  // chunks that need no test.  Not with a gradient and many chunks: without the
  // branches between them the loads and stores of a row crowd together, and
  // E = 256 takes 1,037 us where it took 665 (E = 128's value 69 with, 74 without)
  constexpr int SURE = GRAD && C > 4 ? 0 : CMIN;
  extern __shared__ __align__(128) uint8_t sm[];
  __shared__ float sums[kBalWarps][2];
  __shared__ __align__(8) uint64_t bars[kBalWarps * kBalMaxStages];
  __shared__ float tot[2];
  __shared__ int valid_n, aborted;
  float* Fs = reinterpret_cast<float*>(sm);
  int* hist = reinterpret_cast<int*>(Fs + EM);
  float* Rs = Fs + 2 * EM;  // with a gradient
  float* colsum = Fs + (GRAD ? 3 : 2) * EM;
  const int E = a.E, nch = E >> 2, G = cut.group, D = cut.stages;
  const int threads = static_cast<int>(blockDim.x), warps = threads >> 5;  // 8, or fewer for short microbatches
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const int sub = lane & (LPT - 1), slot = lane / LPT;
  const bool gin = GRAD && a.grad_in;
  const uint32_t zrow = static_cast<uint32_t>(E) * (F32 ? 4u : 2u), grow = gin ? static_cast<uint32_t>(E) * 4u : 0u;
  const uint32_t stage_bytes = static_cast<uint32_t>(G) * (zrow + grow);
  uint8_t* ring = sm + bal_fixed_bytes(EM, warps, GRAD) + static_cast<size_t>(wid) * D * stage_bytes;
  const uint32_t ring_s = smem_u32(ring), bar0 = smem_u32(bars + wid * kBalMaxStages);
  if (lane == 0) {
    for (int s = 0; s < D; ++s) mbar_init(bar0 + 8u * s, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (threadIdx.x == 0) valid_n = aborted = 0;
  if (cut.cluster)
    for (int e = threadIdx.x; e < EM; e += threads) hist[e] = 0;
  // The counts' kernel lets this one start once what came before the call is
  // complete, so that z, grad_in, the mask and the offsets may be read; what it
  // writes is waited for below, before F is formed.
  if (cut.cluster) griddep_wait();
  int l = 0;
  uint32_t rank = 0;
  int64_t tb, te, len = 0;
  if (cut.cluster) {
    l = static_cast<int>(blockIdx.x) / cut.cluster;
    rank = blockIdx.x % static_cast<unsigned>(cut.cluster);
    // within the batch whatever the offsets say
    const int64_t lo = min(max(__ldg(a.off + l), int64_t(0)), a.T);
    len = min(max(__ldg(a.off + l + 1), lo), a.T) - lo;
    tb = lo + len * rank / cut.cluster;
    te = lo + len * (rank + 1) / cut.cluster;
  } else {
    tb = static_cast<int64_t>(blockIdx.x) * cut.tokens_per_cta;
    te = min(tb + cut.tokens_per_cta, a.T);  // beyond tb: the grid is cut to the tokens
    l = microbatch_of_warp(a.off, a.M, tb, lane);
  }
  // tokens are counted from tb on from here
  const int nt = static_cast<int>(te - tb);
  const uint8_t* zb = static_cast<const uint8_t*>(a.z) + tb * zrow;
  const float* gb = gin ? a.grad_in + tb * E : nullptr;
  const uint8_t* mb = a.mask ? a.mask + tb : nullptr;
  __syncthreads();
  // this warp's groups start at wid G, (wid + warps) G, ...
  const int gstep = warps * G;
  int g0 = wid * G;
  auto issue = [&](int at, int stage) {
    if (lane == 0 && at < nt) {
      const uint32_t cnt = static_cast<uint32_t>(min(G, nt - at));
      const uint32_t dst = ring_s + static_cast<uint32_t>(stage) * stage_bytes, bar = bar0 + 8u * stage;
      mbar_expect_tx(bar, cnt * (zrow + grow));
      bulk_load(dst, zb + static_cast<int64_t>(at) * zrow, cnt * zrow, bar);
      if (gin) bulk_load(dst + static_cast<uint32_t>(G) * zrow, gb + static_cast<int64_t>(at) * E, cnt * grow, bar);
    }
  };
  for (int s = 0; s < D; ++s) issue(g0 + s * gstep, s);
  const float gs = GRAD && a.grad_scale ? *a.grad_scale : 1.0f;
  auto mask_of = [&](int at) -> uint32_t {  // of a group's tokens, one bit each
    if (!mb || at >= nt) return kFull;
    return __ballot_sync(kFull, lane < G && at + lane < nt && mb[at + lane]);
  };
  uint32_t mbits = mask_of(g0), mnext = mask_of(g0 + gstep);

  if (cut.cluster) {  // the lists' counts, this block's and then the cluster's
    const int32_t* idx = a.idx + tb * a.K;
    for (int i = threadIdx.x; i < nt * a.K; i += threads) {
      const int e = idx[i];
      if (static_cast<unsigned>(e) < static_cast<unsigned>(E) && (!mb || mb[i / a.K])) atomicAdd(hist + e, 1);
    }
    if (mb) {
      int v = 0;
      for (int i = threadIdx.x; i < nt; i += threads) v += mb[i] != 0;
      v = __reduce_add_sync(kFull, v);
      if (lane == 0 && v) atomicAdd(&valid_n, v);
    }
    cluster_sync();
  }

  if (GRAD && !cut.cluster) griddep_wait();
  int stage = 0, waited = -1;
  uint32_t phase = 0;
  bool dead = false;  // a wait of this warp ran out
  int t = 0, ahead = -1, ahead_valid = 0;  // the microbatch whose counts are on their way to hist
  do {
    int64_t n = len;
    int seg_end = nt;
    if (!cut.cluster) {
      // malformed offsets must not stall the loop
      int64_t lo = __ldg(a.off + l), hi = __ldg(a.off + l + 1);
      while (hi <= tb + t && l + 1 < a.M) {  // the next one that is not empty
        ++l;
        lo = hi;
        hi = __ldg(a.off + l + 1);
      }
      if (hi > tb + t && hi < te) seg_end = static_cast<int>(hi - tb);
      n = hi - lo;
      // the previous microbatch is done with F and R: its sums' barrier says so, if it has sums
      if (GRAD && !a.part) __syncthreads();
    }
    // n, F and R of this microbatch, R from an exact whole number, so that balanced counts give 0
    float rn;
    auto put_f = [&]() {
      if (mb) {
        if (cut.cluster) {
          n = 0;
          for (int q = 0; q < cut.cluster; ++q) n += peer_word(&valid_n, q);
        } else {
          n = l == ahead ? ahead_valid : __ldcg(a.valid + l);
        }
      }
      rn = n > 0 ? __frcp_rn(static_cast<float>(n)) : 0.f;
      const float rkn = rn / static_cast<float>(a.K), rkne = rn / static_cast<float>(a.K * E);
      if (ahead >= 0) asm volatile("cp.async.wait_all;" ::: "memory");
      for (int e = threadIdx.x; e < EM; e += threads) {
        int64_t f = 0;
        if (e < E) {
          if (cut.cluster) {
            for (int q = 0; q < cut.cluster; ++q) f += peer_word(hist + e, q);
            if (rank == 0) a.counts[static_cast<int64_t>(l) * E + e] = static_cast<int32_t>(f);
          } else {
            f = l == ahead ? hist[e] : __ldcg(a.counts + static_cast<int64_t>(l) * E + e);
          }
        }
        Fs[e] = __ll2float_rn(f) * rkn;
        if constexpr (GRAD) Rs[e] = e < E ? __ll2float_rn(f * E - a.K * n) * rkne : 0.f;
      }
      __syncthreads();
    };
    if constexpr (GRAD) {
      put_f();
      if (seg_end < nt && l + 1 < a.M) {
        // The next one's counts, while this one's tokens are at work (700 sequences
        // of 286 tokens: 71.5 us for 72.8; 470 of 9, E = 256: 47.6 for 50.3).  Each
        // thread fetches the words that it reads itself: no barrier is needed.
        ahead = l + 1;
        if (mb) ahead_valid = __ldcg(a.valid + ahead);
        for (int e = threadIdx.x; e < E; e += threads)
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4;"
                       :: "r"(smem_u32(hist + e)), "l"(a.counts + static_cast<int64_t>(ahead) * E + e) : "memory");
      }
    }
    F2 acc[C][2];
#pragma unroll
    for (int k = 0; k < C; ++k) acc[k][0] = acc[k][1] = f2(0.f, 0.f);
    const float ca = GRAD ? gs * (static_cast<float>(a.alpha) * rn) : 0.f;
    const float cz = GRAD ? gs * (2.0f * static_cast<float>(a.zeta) * rn) : 0.f;
    float zsum = 0.f;

    while (g0 < seg_end && !dead) {
      if (waited != g0) {
        waited = g0;
        dead = !__all_sync(kFull, mbar_wait(bar0 + 8u * stage, phase, &aborted));
        if (dead) break;
      }
      const uint8_t* zs = ring + static_cast<uint32_t>(stage) * stage_bytes;
      const uint8_t* gsrc = zs + static_cast<uint32_t>(G) * zrow;
      // the group's tokens of this microbatch, counted from g0
      const int from = max(t - g0, 0), to = min(seg_end - g0, G);
      for (int i0 = from / TPW * TPW; i0 < to; i0 += TPW) {
        const int i = i0 + slot;
        const bool in = i >= from && i < to;
        const bool ok = in && (mbits >> i & 1u);
        // a row that does not count is taken as zeros: finite, and its p becomes 0
        const bool whole = __all_sync(kFull, ok);
        F2 e[C][2];
        float top, low;
        if constexpr (F32) {
          const float4* zr = reinterpret_cast<const float4*>(zs + static_cast<uint32_t>(i) * zrow) + sub;
          top = -INFINITY;
          low = INFINITY;
#pragma unroll
          for (int k = 0; k < C; ++k) {
            float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
            if (k < SURE || sub + k * LPT < nch) {
              w = zr[k * LPT];
              if (!whole && !ok) w = make_float4(0.f, 0.f, 0.f, 0.f);
              top = fmaxf(fmaxf(top, fmaxf(w.x, w.y)), fmaxf(w.z, w.w));
              if constexpr (SIG) low = fminf(fminf(low, fminf(w.x, w.y)), fminf(w.z, w.w));
            }
            e[k][0] = f2(w.x, w.y);
            e[k][1] = f2(w.z, w.w);
          }
#pragma unroll
          for (int m = 1; m < LPT; m <<= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, m));
        } else {
          const uint2* zr = reinterpret_cast<const uint2*>(zs + static_cast<uint32_t>(i) * zrow) + sub;
          uint32_t top2 = 0xff80ff80u, low2 = 0x7f807f80u;  // -inf, inf
#pragma unroll
          for (int k = 0; k < C; ++k) {
            uint2 w = make_uint2(0u, 0u);
            if (k < SURE || sub + k * LPT < nch) {
              w = zr[k * LPT];
              if (!whole && !ok) w = make_uint2(0u, 0u);
              top2 = hmax2_bf16(top2, hmax2_bf16(w.x, w.y));
              if constexpr (SIG) low2 = hmin2_bf16(low2, hmin2_bf16(w.x, w.y));
            }
            e[k][0] = f2(bf16_lo(w.x), bf16_hi(w.x));
            e[k][1] = f2(bf16_lo(w.y), bf16_hi(w.y));
          }
#pragma unroll
          for (int m = 1; m < LPT; m <<= 1) top2 = hmax2_bf16(top2, __shfl_xor_sync(kFull, top2, m));
          top = fmaxf(bf16_lo(top2), bf16_hi(top2));
          low = fminf(bf16_lo(low2), bf16_hi(low2));
        }
        // a row without a finite logit has no probabilities (nor has a masked one)
        const bool alive = ok && top > -INFINITY;
        // sigmoids are taken relative to e^top where all are far below 0.5:
        // s e^-top = 1 / (e^top + e^(top - z))
        const float ref = !(top > -INFINITY) ? 0.f : SIG ? fminf(top, 0.f) : top;
        const F2 mul = splat2(SIG ? -kLog2e : kLog2e);
        float m2 = ref * kLog2e;
        const float em = SIG ? ex2_approx(m2) : 0.f;
        const F2 em2 = splat2(em);
        // The power's argument is z log2(e) less m2, and m2's rounding scales all of a
        // row alike.  Far from zero (rows closed by the type's lowest value, say) it
        // would be off by whole powers of two, or infinite: there the reference is
        // taken off z itself.
        const bool wide = fabsf(ref) > 0x1p20f;
        // one reciprocal serves two sigmoids as long as the product of the two
        // denominators is finite; beyond 2^60 of the row's reference (-inf
        // among them) a sigmoid counts as zero.  Most rows are nearer than that.
        constexpr float kFar = 0x1p60f;
        const bool rare = __any_sync(kFull, wide || (SIG && low < ref - 40.f)), far = SIG && rare;
        if (rare && __any_sync(kFull, wide)) {
          const F2 off = splat2(wide ? ref : 0.f);
#pragma unroll
          for (int k = 0; k < C; ++k) {
            e[k][0] = sub2(e[k][0], off);
            e[k][1] = sub2(e[k][1], off);
          }
          if (wide) m2 = 0.f;
        }
        const F2 shift = splat2(SIG ? m2 : -m2);
        auto sigmoids = [&](auto FAR, F2 x) {
          const F2 xc = FAR ? f2(fmin_nan(lo2(x), kFar), fmin_nan(hi2(x), kFar)) : x;
          const F2 y = add2(em2, xc);
          const float rr = rcp_approx(lo2(y) * hi2(y));
          const F2 sg = f2(rr * hi2(y), rr * lo2(y));  // two products: a pair would have to be turned and spread
          return FAR ? f2(lo2(x) > kFar ? 0.f : lo2(sg), hi2(x) > kFar ? 0.f : hi2(sg)) : sg;
        };
        F2 d2 = f2(0.f, 0.f), h2 = f2(0.f, 0.f);
        auto sums_of = [&](auto FAR) {
#pragma unroll
          for (int k = 0; k < C; ++k) {
            if (k < SURE || sub + k * LPT < nch) {
              float4 rw = make_float4(0.f, 0.f, 0.f, 0.f);
              if constexpr (GRAD) rw = reinterpret_cast<const float4*>(Rs)[sub + k * LPT];
              const F2 rk[2] = {f2(rw.x, rw.y), f2(rw.z, rw.w)};
#pragma unroll
              for (int q = 0; q < 2; ++q) {
                F2 x = fma2(e[k][q], mul, shift);
                x = f2(ex2_approx(lo2(x)), ex2_approx(hi2(x)));
                const F2 sg = SIG ? sigmoids(FAR, x) : x;
                // with a gradient the sigmoid is formed again from x, which 1 - s needs too
                e[k][q] = SIG && GRAD ? x : sg;
                d2 = add2(d2, sg);
                if constexpr (GRAD) h2 = fma2(sg, rk[q], h2);
              }
            } else {
              e[k][0] = e[k][1] = f2(0.f, 0.f);
            }
          }
        };
        if (far) sums_of(Yes{});
        else sums_of(No{});
        float d = lo2(d2) + hi2(d2), h = lo2(h2) + hi2(h2);
#pragma unroll
        for (int m = 1; m < LPT; m <<= 1) {
          d += __shfl_xor_sync(kFull, d, m);
          if constexpr (GRAD) h += __shfl_xor_sync(kFull, h, m);
        }
        // of a row without a finite logit too: the maxima drop NaN, and a row that
        // is NaN throughout looks closed, but only a closed one has a sum of 0
        if (ok && !(d < INFINITY)) raise_flag(a.err, kErrNonfinite);
        float id = rcp_approx(d);
        id = alive ? __fmaf_rn(id, __fmaf_rn(-d, id, 1.0f), id) : 0.f;
        h *= id;
        float lse = 0.f;
        if (!SIG && a.zeta != 0.0) lse = alive ? __fmaf_rn(lg2_approx(d), kLn2, top) : 0.f;
        if (sub == 0) zsum = __fmaf_rn(lse, lse, zsum);
        const F2 id2 = splat2(id);
        if constexpr (!GRAD) {
#pragma unroll
          for (int k = 0; k < C; ++k)
#pragma unroll
            for (int q = 0; q < 2; ++q) acc[k][q] = fma2(e[k][q], id2, acc[k][q]);
        } else {
          const F2 ca2 = splat2(ca), k2 = splat2(__fmaf_rn(-ca, h, cz * lse));
          const float4* gr = reinterpret_cast<const float4*>(gsrc + static_cast<uint32_t>(i) * grow) + sub;
          const int64_t at = (tb + g0 + i) * nch + sub;  // chunk of the output
          auto gradients = [&](auto FAR) {
#pragma unroll
          for (int k = 0; k < C; ++k) {
            if (k >= SURE && sub + k * LPT >= nch) continue;
            const float4 rw = reinterpret_cast<const float4*>(Rs)[sub + k * LPT];
            const F2 rk[2] = {f2(rw.x, rw.y), f2(rw.z, rw.w)};
            float4 old = make_float4(0.f, 0.f, 0.f, 0.f);
            if (gin) old = gr[k * LPT];
            F2 g[2] = {f2(old.x, old.y), f2(old.z, old.w)};
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              const F2 sg = SIG ? sigmoids(FAR, e[k][q]) : e[k][q];
              acc[k][q] = fma2(sg, id2, acc[k][q]);
              F2 v = fma2(ca2, rk[q], k2);
              if constexpr (SIG) {
                const F2 xc = FAR ? f2(fmin_nan(lo2(e[k][q]), kFar), fmin_nan(hi2(e[k][q]), kFar)) : e[k][q];
                v = mul2(v, mul2(xc, sg));
              }
              g[q] = fma2(mul2(sg, id2), v, g[q]);
            }
            if (!in) continue;
            if (a.grad_bf16)
              __stcs(static_cast<uint2*>(a.grad_out) + at + k * LPT,
                     make_uint2(pack_bf16x2_rn(lo2(g[0]), hi2(g[0])), pack_bf16x2_rn(lo2(g[1]), hi2(g[1]))));
            else
              __stcs(static_cast<float4*>(a.grad_out) + at + k * LPT, make_float4(lo2(g[0]), hi2(g[0]), lo2(g[1]), hi2(g[1])));
          }
          };
          if (far) gradients(Yes{});
          else gradients(No{});
        }
      }
      if (g0 + G > seg_end && seg_end < nt) break;  // the rest is the next microbatch's
      __syncwarp();
      issue(g0 + D * gstep, stage);
      g0 += gstep;
      mbits = mnext;
      mnext = mask_of(g0 + gstep);
      if (++stage == D) { stage = 0; phase ^= 1u; }
    }

    // Without a gradient F, for which the counts have to be there, is wanted only now.
    if constexpr (!GRAD) {
      if (!cut.cluster) griddep_wait();
      put_f();
    }
    // the block's sums of this microbatch
    if (a.part || cut.cluster) {
      float* row = a.part + (static_cast<int64_t>(blockIdx.x) + l) * a.row;  // not used by a cluster
      const int ROWS = bal_rows(EM, warps);
      float hsum = 0.f;  // of p.F: the warp's sums of p by F
      for (int round = 0; round < warps / ROWS; ++round) {
        if (round) __syncthreads();
        if (wid / ROWS != round) continue;
#pragma unroll
        for (int k = 0; k < C; ++k) {
          float4 v = make_float4(sum_slots(lo2(acc[k][0]), LPT), sum_slots(hi2(acc[k][0]), LPT),
                                 sum_slots(lo2(acc[k][1]), LPT), sum_slots(hi2(acc[k][1]), LPT));
          const float4 fw = reinterpret_cast<const float4*>(Fs)[sub + k * LPT];
          hsum += __fmaf_rn(v.x, fw.x, v.y * fw.y) + __fmaf_rn(v.z, fw.z, v.w * fw.w);
          float4* col = reinterpret_cast<float4*>(colsum + wid % ROWS * EM) + sub + k * LPT;
          if (round) {
            const float4 w = *col;
            v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
          }
          __syncwarp();
          if (slot == 0) *col = v;
        }
      }
#pragma unroll
      for (int m = 1; m < LPT; m <<= 1) hsum += __shfl_xor_sync(kFull, hsum, m);
      zsum = sum_slots(zsum, 1);
      if (lane == 0) {
        sums[wid][0] = hsum;
        sums[wid][1] = zsum;
      }
      __syncthreads();
      for (int e = threadIdx.x; e < E; e += threads) {
        float v = 0.f;
        for (int q = 0; q < ROWS; ++q) v += colsum[q * EM + e];
        if (cut.cluster) colsum[e] = v;
        else row[4 + e] = v;
      }
      if (threadIdx.x < 2) {
        float v = 0.f;
        for (int q = 0; q < warps; ++q) v += sums[q][threadIdx.x];
        if (cut.cluster) tot[threadIdx.x] = v;
        else row[threadIdx.x] = v;
      }
    }
    if (cut.cluster) {
      cluster_sync();
      const float n1 = static_cast<float>(n);
      if (a.prob)
        for (int e = rank * threads + threadIdx.x; e < E; e += cut.cluster * threads) {
          float v = 0.f;
          for (int q = 0; q < cut.cluster; ++q) v += peer_float(colsum + e, q);
          a.prob[static_cast<int64_t>(l) * E + e] = n > 0 ? v / n1 : 0.f;
        }
      if (a.loss && rank == 0 && threadIdx.x == 0) {
        float v[2] = {0.f, 0.f};
        for (int q = 0; q < cut.cluster; ++q)
#pragma unroll
          for (int i = 0; i < 2; ++i) v[i] += peer_float(tot + i, q);
        a.loss[2 * l] = n > 0 ? static_cast<float>(a.alpha) * (v[0] / n1) : 0.f;
        a.loss[2 * l + 1] = n > 0 ? static_cast<float>(a.zeta) * (v[1] / n1) : 0.f;
      }
      cluster_sync();  // no block leaves while another reads its sums
    }
    t = seg_end;
  } while (t < nt);
  if (dead && lane == 0) {  // the copies in flight must land before the block leaves
    const int j = g0 / gstep;
    const int sent = min((nt - wid * G + gstep - 1) / gstep, j + D);
    drain_loads(sent, D, [&](int s) { return bar0 + 8u * s; });
    raise_flag(a.err, kErrCuda);
  }
}

template <bool SIG, bool GRAD, bool F32, int LPT, int C, int CMIN>
int launch_bal(const BalanceArgs& a, BalanceRun* run, cudaStream_t s) {
  constexpr int TPW = 32 / LPT, EM = LPT * C * 4;
  DeviceInfo di;
  if (int rc = device_info(&di)) return rc;
  const bool gin = GRAD && a.grad_in;
  // Few tokens: a cluster a microbatch.  A block passes over 3,000 elements a
  // microsecond, the four launches take 17 us (M = 1, T = 8,000, E = 128 by one
  // cluster 44 us, by four launches 16).  The host does not know how long the
  // microbatches are: the limit is 2^15 elements a block if the longest has twice
  // the mean, and eight times that if one has all the tokens.
  BalanceCut cut;
  cut.cluster = 0;
  if (run->may_cluster) {
    const int cl = a.M >= di.sm_count ? 1 : a.M >= 64 ? 2 : a.M >= 32 ? 4 : 8;
    const int even = a.M >= 8 ? 4 : a.M >= 2 ? (a.M + 1) / 2 : 1;
    if (a.T * a.E <= (int64_t(1) << 15) * cl * even) cut.cluster = cl;
  }
  // Warps of a block: no more than a microbatch of mean length keeps busy
  // for a round (50,000 tokens in 1,900 microbatches, E = 64: this pass 16 us with
  // one warp a block, 22 with four, 21 with eight; 4,370 in 470, E = 256 with a
  // sigmoid's gradient: 53 with one, 31 with four).
  const int64_t mean = a.T / a.M / (cut.cluster ? cut.cluster : 1);
  int warps = kBalWarps;
  while (warps > 1 && warps * TPW > mean && !(cut.cluster && warps * 64 <= EM)) warps /= 2;
  const int stage1 = bal_stage_bytes(a.E, TPW, F32, gin);
  // one SM's memory over its blocks, 1 KB of each reserved and about 0.5 KB static
  int blocks = bal_blocks(GRAD, C) * kBalWarps / warps;
  const int fixed = bal_fixed_bytes(EM, warps, GRAD), two = fixed + 2 * warps * stage1 + 2048;
  if (warps < kBalWarps && blocks > di.max_smem_optin / two) blocks = di.max_smem_optin / two;
  const int room = di.max_smem_optin / blocks - 2048 - fixed;
  int64_t grid;
  if (cut.cluster) {
    grid = static_cast<int64_t>(a.M) * cut.cluster;
    cut.tokens_per_cta = (a.T + grid - 1) / grid;
  } else {
    // at least a round of the block's warps, and of short microbatches a whole one
    int64_t least = warps * TPW;
    if (warps < kBalWarps && least < mean) least = mean;
    grid = (a.T + least - 1) / least;
    const int64_t most = di.sm_count * blocks < kBalMaxGrid ? di.sm_count * blocks : kBalMaxGrid;
    if (grid > most) grid = most;
    cut.tokens_per_cta = (a.T + grid - 1) / grid;
    grid = (a.T + cut.tokens_per_cta - 1) / cut.tokens_per_cta;
  }
  // groups of up to 4 KB, two of them for every warp where there are as many
  // tokens, and a ring as deep as the blocks of an SM leave room for
  cut.group = TPW;
  while (cut.group * 2 <= 32 && bal_stage_bytes(a.E, cut.group * 2, F32, gin) <= 4096 &&
         cut.group * 4 * warps <= cut.tokens_per_cta && 4 * warps * bal_stage_bytes(a.E, cut.group, F32, gin) <= room)
    cut.group *= 2;
  cut.stages = room / (warps * bal_stage_bytes(a.E, cut.group, F32, gin));
  if (cut.stages > kBalMaxStages) cut.stages = kBalMaxStages;
  if (cut.stages < 1) return kErrUnsupported;
  run->tokens_per_cta = cut.tokens_per_cta;
  run->done = cut.cluster != 0;
  const int smem = fixed + warps * cut.stages * bal_stage_bytes(a.E, cut.group, F32, gin);
  const auto kern = balance_kernel<SIG, GRAD, F32, LPT, C, CMIN>;
  if (!allow_smem(kern, di.max_smem_optin - 2048)) return kErrCuda;
  if (cut.cluster == 0) {
    if (int rc = launch_balance_counts(a, s)) return rc;
  }
  return launch_clusters(kern, dim3(static_cast<unsigned>(grid)), dim3(32 * warps), smem, s, cut.cluster, a, cut) == cudaSuccess
             ? kOk
             : kErrCuda;
}

template <bool SIG, bool GRAD, bool F32>
int launch_bal_width(const BalanceArgs& a, BalanceRun* run, cudaStream_t s) {
  if (a.E <= 8) return launch_bal<SIG, GRAD, F32, 1, 2, 2>(a, run, s);
  if (a.E <= 16) return launch_bal<SIG, GRAD, F32, 2, 2, 2>(a, run, s);
  if (a.E <= 32) return launch_bal<SIG, GRAD, F32, 4, 2, 1>(a, run, s);
  if (a.E <= 48) return launch_bal<SIG, GRAD, F32, 4, 3, 2>(a, run, s);
  if (a.E <= 64) return launch_bal<SIG, GRAD, F32, 4, 4, 3>(a, run, s);
  if (a.E <= 96) return launch_bal<SIG, GRAD, F32, 8, 3, 2>(a, run, s);
  if (a.E <= 128) return launch_bal<SIG, GRAD, F32, 8, 4, 3>(a, run, s);
  if (a.E <= 192) return launch_bal<SIG, GRAD, F32, 8, 6, 4>(a, run, s);
  if (a.E <= 256) return launch_bal<SIG, GRAD, F32, 8, 8, 6>(a, run, s);
  if (a.E <= 384) return launch_bal<SIG, GRAD, F32, 16, 6, 4>(a, run, s);
  if (a.E <= 512) return launch_bal<SIG, GRAD, F32, 16, 8, 6>(a, run, s);
  if (a.E <= 768) return launch_bal<SIG, GRAD, F32, 32, 6, 4>(a, run, s);
  if (a.E <= 1024) return launch_bal<SIG, GRAD, F32, 32, 8, 6>(a, run, s);
  return kErrUnsupported;
}

template <bool SIG, bool GRAD>
int launch_bal_type(const BalanceArgs& a, BalanceRun* run, cudaStream_t s) {
  return a.z_fp32 ? launch_bal_width<SIG, GRAD, true>(a, run, s) : launch_bal_width<SIG, GRAD, false>(a, run, s);
}

}  // namespace

}  // namespace eqb
