// gate_tile.cuh -- the gate of many tokens (see gate.cu): a thread takes a token
// whose row of z lies in shared memory, a warp a tile of 32 tokens.
//
// The row is cut into 16, 12 or 8 equal parts (8 of different size where its chunks of
// 8 experts do not make equal ones), each within a group:
//   1. the two largest c = z + b of every part, in pairs: exact (fp32), so the
//      groups' scores and their ranking are too;
//   2. of the parts that stay open, the K-th largest of their two largest is a lower
//      bound of the K-th largest c (K <= 8): from the eight largest of either, sorted, the
//      smallest over i of the larger of one's i-th and the other's (K + 1 - i)-th;
//   3. a bit for every open expert at or above the bound;
//   4. those are inserted in ascending order into a sorted list: with 4 of 8 groups of
//      32 open and K = 8 there are 8.1 a token and 9.0 in the lane of a warp that has
//      most, which is how often the warp inserts (with eight parts 11.0 and 18.6).
// Phases 1 and 3 take four to five instructions a value, phase 4 about seventy a
// candidate of the lane that has most.  A thread a token needs about a tenth of
// the instructions of a warp a token (gate.cu), which waits for every maximum of
// the warp.
//
// Lanes bring their rows with bulk copies (a barrier a warp), at a stride of 4
// (mod 8) words so that the lanes' 16-byte reads of one column hit distinct banks.
#pragma once

#include <float.h>

#include "f32x2.cuh"
#include "route_wide.cuh"

namespace eqb {

namespace {

constexpr int kMaxGateWarps = 16;

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// The eight largest of 8 to 16 values, descending, in a[0..7].
__device__ __forceinline__ void top8(float (&a)[8]) { sort_desc<8>(a); }
template <int N>
__device__ __forceinline__ void top8(float (&a)[N]) {
  float x[8], y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[i] = a[i];
    y[i] = 8 + i < N ? a[8 + i] : -INFINITY;
  }
  sort_desc<8>(x);
  sort_desc<8>(y);
  // the larger of the i-th of one and the i-th from behind of the other: the eight
  // largest, first falling, then rising
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = fmaxf(x[i], y[7 - i]);
#pragma unroll
  for (int j = 4; j > 0; j >>= 1)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (!(i & j)) {
        const float h = fmaxf(a[i], a[i | j]), l = fminf(a[i], a[i | j]);
        a[i] = h;
        a[i | j] = l;
      }
}

// The two largest of two pairs of the two largest.  NaN stays in the first.
__device__ __forceinline__ void merge2(float& m1, float& m2, float h, float l) {
  const float lo = fminf(m1, h);
  m2 = max3(lo, m2, l);
  m1 = fmax_nan(m1, h);
}

template <bool F32>
__device__ __forceinline__ void row8(const uint8_t* row, int chunk, F2 (&v)[4]) {
  if (F32) {
    const float4 x = *reinterpret_cast<const float4*>(row + 32 * chunk), y = *reinterpret_cast<const float4*>(row + 32 * chunk + 16);
    v[0] = f2(x.x, x.y);
    v[1] = f2(x.z, x.w);
    v[2] = f2(y.x, y.y);
    v[3] = f2(y.z, y.w);
  } else {
    const uint4 x = lds128(row + 16 * chunk);
    v[0] = f2(bf16_lo(x.x), bf16_hi(x.x));
    v[1] = f2(bf16_lo(x.y), bf16_hi(x.y));
    v[2] = f2(bf16_lo(x.z), bf16_hi(x.z));
    v[3] = f2(bf16_lo(x.w), bf16_hi(x.w));
  }
}
template <bool F32>
__device__ __forceinline__ float row1(const uint8_t* row, int e) {
  return F32 ? *reinterpret_cast<const float*>(row + 4 * e) : bf16_bits_to_f32(lds_u16(row + 2 * e));
}
// fp32(z) + b of the two bf16 values of a word, one rounding each: the sum takes the
// bf16 value as it is, so that nothing is unpacked (the shifts and masks of that
// run where the minima and maxima do, and those bound this kernel).
__device__ __forceinline__ F2 add_wide(uint32_t w, float b0, float b1) {
  float x, y;
  asm("{\n\t.reg .b16 l, h;\n\t"
      "mov.b32 {l, h}, %2;\n\t"
      "add.rn.f32.bf16 %0, l, %3;\n\t"
      "add.rn.f32.bf16 %1, h, %4;\n\t}"
      : "=f"(x), "=f"(y)
      : "r"(w), "f"(b0), "f"(b1));
  return f2(x, y);
}
// c of eight experts.
template <bool F32>
__device__ __forceinline__ void scores8(const uint8_t* row, const float* bs, int chunk, F2 (&v)[4]) {
  const float4 x = *reinterpret_cast<const float4*>(bs + 8 * chunk), y = *reinterpret_cast<const float4*>(bs + 8 * chunk + 4);
  if (F32) {
    row8<F32>(row, chunk, v);
    v[0] = add2(v[0], f2(x.x, x.y));
    v[1] = add2(v[1], f2(x.z, x.w));
    v[2] = add2(v[2], f2(y.x, y.y));
    v[3] = add2(v[3], f2(y.z, y.w));
  } else {
    const uint4 w = lds128(row + 16 * chunk);
    v[0] = add_wide(w.x, x.x, x.y);
    v[1] = add_wide(w.y, x.z, x.w);
    v[2] = add_wide(w.z, y.x, y.y);
    v[3] = add_wide(w.w, y.z, y.w);
  }
}

struct GateTile {
  int stride;  // bytes of a staged row
  int warp_bytes;
  int64_t tiles_per_warp;
};

// First chunk (of eight experts) of part s: C chunks a part, or (C = 0) groups of gc
// chunks in SP parts.
template <int SP, int C>
__device__ __forceinline__ int part_chunk(int s, int gc) {
  return C ? s * C : s / SP * gc + s % SP * gc / SP;
}

// P parts of C chunks each; C = 0: eight parts of any size.
template <bool F32, int G, int KP, int P, int C>
__global__ void __launch_bounds__(32 * kMaxGateWarps, 1) gate_tile_kernel(const GateArgs a, const GateTile g) {
  constexpr int kParts = P, SP = kParts / G;  // SP: parts of a group
  extern __shared__ __align__(16) uint8_t smem[];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, nw = blockDim.x >> 5;
  const int E = C ? 8 * P * C : a.E, K = a.K, gc = E / 8 / G, words = (E + 31) / 32;
  float* bs = reinterpret_cast<float*>(smem);
  uint8_t* mine = smem + 4 * E + wid * g.warp_bytes;
  uint32_t* mw = reinterpret_cast<uint32_t*>(mine + 32 * g.stride) + lane;  // [words][32 lanes]
  const uint32_t bar = saddr(mine + 32 * g.stride + words * 128);
  const uint8_t* row = mine + lane * g.stride;
  const int row_bytes = E * (F32 ? 4 : 2);
  if (lane == 0) {
    bar_init(bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  griddep_wait();
  for (int e = threadIdx.x; e < E; e += blockDim.x) bs[e] = a.b ? a.b[e] : 0.f;
  __syncthreads();
  const int64_t ntiles = (a.T + 31) >> 5;
  const int64_t tb = (static_cast<int64_t>(blockIdx.x) * nw + wid) * g.tiles_per_warp, te = min(tb + g.tiles_per_warp, ntiles);
  if (tb >= te) return;
  const uint8_t* z = static_cast<const uint8_t*>(a.z);
  auto load_tile = [&](int64_t tl) {
    const int64_t t0 = tl << 5;
    const int rows = static_cast<int>(min(static_cast<int64_t>(32), a.T - t0));
    if (lane == 0) bar_expect_tx(bar, static_cast<uint32_t>(rows * row_bytes));
    __syncwarp();
    if (lane < rows) {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      bulk_copy(saddr(mine + lane * g.stride), z + (t0 + lane) * row_bytes, row_bytes, bar);
    }
  };
  auto prefetch = [&](int64_t tl) {
    if (lane == 0 && tl < te) {
      const int64_t t0 = tl << 5;
      const uint32_t bytes = static_cast<uint32_t>(min(static_cast<int64_t>(32), a.T - t0) * row_bytes);
      asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(z + t0 * row_bytes), "r"(bytes) : "memory");
    }
  };
  uint32_t phase = 0;
  load_tile(tb);
  prefetch(tb + 1);
  for (int64_t tl = tb; tl < te; ++tl) {
    if (!__all_sync(kFull, bar_wait_bounded(bar, phase, kRouteWaitLimit))) {
      raise_flag(a.err, kErrCuda);
      bar_wait_bounded(bar, phase, kRouteWaitLimit);
      return;
    }
    phase ^= 1u;
    const int64_t t = (tl << 5) + lane;
    const bool valid = t < a.T && (!a.mask || a.mask[t]);

    // ---- 1: the parts' two largest
    float m1[kParts], m2[kParts];
    bool bad = false;
#pragma unroll
    for (int s = 0; s < kParts; ++s) {
      m1[s] = m2[s] = -INFINITY;
      const int c1 = part_chunk<SP, C>(s + 1, gc);
#pragma unroll
      for (int c = part_chunk<SP, C>(s, gc); c < c1; ++c) {
        F2 v[4];
        scores8<F32>(row, bs, c, v);
        float h[4], l[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          h[i] = fmax_nan(lo2(v[i]), hi2(v[i]));
          l[i] = fminf(lo2(v[i]), hi2(v[i]));
        }
        merge2(h[0], l[0], h[1], l[1]);
        merge2(h[2], l[2], h[3], l[3]);
        merge2(h[0], l[0], h[2], l[2]);
        merge2(m1[s], m2[s], h[0], l[0]);
      }
      bad |= !(m1[s] < INFINITY);
      if (C == 4) asm volatile("" ::: "memory");  // all parts' loads at once do not fit in registers
    }
    if (valid && bad) raise_flag(a.err, kErrNonfinite);

    // ---- the groups' ranking: bits of the open groups
    uint32_t open = (1u << G) - 1u;
    if (G > 1 && a.top_groups < G) {
      float score[G];
      int ahead[G];
#pragma unroll
      for (int i = 0; i < G; ++i) {
        float h = m1[i * SP], l = m2[i * SP];
#pragma unroll
        for (int j = 1; j < SP; ++j) merge2(h, l, m1[i * SP + j], m2[i * SP + j]);
        score[i] = a.top2 && l > -INFINITY ? __fadd_rn(h, l) : h;
        ahead[i] = 0;
      }
#pragma unroll
      for (int i = 0; i < G; ++i)
#pragma unroll
        for (int j = i + 1; j < G; ++j) {
          const bool later = score[j] > score[i];
          ahead[i] += later;
          ahead[j] += !later;
        }
      open = 0u;
#pragma unroll
      for (int i = 0; i < G; ++i) open |= ahead[i] < a.top_groups ? 1u << i : 0u;
    }

    // ---- 2: a lower bound of the K-th largest
    float bound = INFINITY;
    {
#pragma unroll
      for (int s = 0; s < kParts; ++s)
        if (!(open >> (s / SP) & 1u)) m1[s] = m2[s] = -INFINITY;
      top8(m1);
      top8(m2);
#pragma unroll
      for (int k = 1; k <= KP; ++k)
        if (k == K) {
#pragma unroll
          for (int i = 0; i < k; ++i) bound = fminf(bound, fmaxf(m1[i], m2[k - 1 - i]));
        }
      bound = fmaxf(bound, -FLT_MAX);  // a closed expert is never chosen
    }

    // ---- 3: who is at or above it: the sign of c - bound, 32 experts a word.  All
    // chunks alike: of the open groups alone, each lane would read other places, in
    // banks that meet, and wait for them (362 us at T = 2,097,152, E = 256, 4 of 8
    // groups, where this takes 337)
    uint32_t hits = 0u;
    if (!valid) open = 0u;
    {
      // +0 from a bound of either zero: -0 + -0 would be below, though the two are equal
      const F2 less = splat2(__fsub_rn(0.f, bound));
      uint32_t word = 0u;
      int group = 0, left = gc;  // chunks of the group from here on
#pragma unroll
      for (int c = 0; c < E / 8; ++c) {
        F2 v[4];
        scores8<F32>(row, bs, c, v);
        uint32_t bits = 0u;  // signs: set where it is below
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const F2 d = add2(v[i], less);
          bits = __funnelshift_l(__float_as_uint(lo2(d)), bits, 1);
          bits = __funnelshift_l(__float_as_uint(hi2(d)), bits, 1);
        }
        word = word << 8 | (open >> group & 1u ? ~bits & 0xffu : 0u);
        if ((c & 3) == 3 || c == E / 8 - 1) {
          word <<= 8 * (3 - (c & 3));
          mw[(c >> 2) << 5] = word;
          hits |= word != 0u ? 0x80000000u >> (c >> 2) : 0u;
          word = 0u;
          if (C == 4) asm volatile("" ::: "memory");
        }
        if (--left == 0) {
          ++group;
          left = gc;
        }
      }
    }
    // ---- 4: the candidates in ascending order
    float v[KP];
    int id[KP];
#pragma unroll
    for (int j = 0; j < KP; ++j) {
      v[j] = -INFINITY;
      id[j] = -1;
    }
    uint32_t m = 0u;
    int wb = 0;
    auto fetch = [&]() -> int {
      if (m == 0u && hits != 0u) {
        const int k = __clz(hits);
        hits ^= 0x80000000u >> k;
        m = mw[k << 5];
        wb = k << 5;
      }
      const int p = __clz(m);
      const int e = m != 0u ? wb + p : -1;
      m &= shr_clamp(0x7fffffffu, p);
      return e;
    };
    // the next candidate's c is formed while this one is inserted
    auto score_of = [&](int e) { return e >= 0 ? __fadd_rn(row1<F32>(row, e), bs[e]) : -INFINITY; };
    int e0 = fetch();
    float s0 = score_of(e0);
    while (__any_sync(kFull, e0 >= 0)) {
      const int e1 = fetch();
      const float s1 = score_of(e1);
      insert_sorted<KP>(v, id, s0, e0);
      e0 = e1;
      s0 = s1;
    }
    // after a NaN (flagged) a finished lane's entry can stand before others; it is -1

    // ---- the weights
    float w[KP];
    if (a.weight) {
      float top = -INFINITY;
#pragma unroll
      for (int j = 0; j < KP; ++j) {
        w[j] = id[j] >= 0 && j < K ? row1<F32>(row, id[j]) : -INFINITY;
        top = fmaxf(top, w[j]);
      }
      float sum = 0.f;
      if (a.sigmoid) {
        // relative to exp(min(0, top)) where they are renormalised: see gate.cu
        const float ref = a.renorm && top > -INFINITY ? fminf(top, 0.f) : 0.f;
#pragma unroll
        for (int j = 0; j < KP; ++j) {
          const float n = expf(-fabsf(w[j])), r = __fdividef(1.f, 1.f + n);
          w[j] = w[j] > 0.f ? r : (a.renorm ? expf(w[j] - ref) : n) * r;
          sum = sum + w[j];
        }
      } else if (a.renorm) {
#pragma unroll
        for (int j = 0; j < KP; ++j) {
          w[j] = w[j] > -INFINITY ? expf(w[j] - top) : 0.f;
          sum = sum + w[j];
        }
      } else {
        // the sum over the whole row, relative to its largest logit
        float zm = -INFINITY;
        for (int c = 0; c < E / 8; ++c) {
          F2 x[4];
          row8<F32>(row, c, x);
#pragma unroll
          for (int i = 0; i < 4; ++i) zm = max3(zm, lo2(x[i]), hi2(x[i]));
        }
        constexpr float kLog2e = 1.4426950408889634f;
        const float ref = zm > -INFINITY ? zm : 0.f;
        F2 acc[4] = {splat2(0.f), splat2(0.f), splat2(0.f), splat2(0.f)};
        for (int c = 0; c < E / 8; ++c) {
          F2 x[4];
          row8<F32>(row, c, x);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const F2 d = mul2(sub2(x[i], splat2(ref)), splat2(kLog2e));
            acc[i] = add2(acc[i], f2(ex2_approx(lo2(d)), ex2_approx(hi2(d))));
          }
        }
        const F2 all = add2(add2(acc[0], acc[1]), add2(acc[2], acc[3]));
        sum = lo2(all) + hi2(all);
#pragma unroll
        for (int j = 0; j < KP; ++j) w[j] = w[j] > -INFINITY ? expf(w[j] - ref) : 0.f;
      }
      // a sum of sigmoids is half at least: over twice the sum the factor becomes no larger
      const bool plain = a.sigmoid && !a.renorm;
      const float f = plain ? a.scale : sum > 0.f ? __fdiv_rn(a.scale, sum + sum) : 0.f;
#pragma unroll
      for (int j = 0; j < KP; ++j) w[j] = (plain ? w[j] : w[j] + w[j]) * f;
    }
    __syncwarp();  // every lane is done with the tile
    if (tl + 1 < te) {
      load_tile(tl + 1);
      prefetch(tl + 2);
    }
    if (t < a.T) {
      int32_t* idx = a.idx + t * K;
      float* out = a.weight ? a.weight + t * K : nullptr;
      if (K == 8 && KP == 8 && (reinterpret_cast<uintptr_t>(a.idx) & 15u) == 0 && (reinterpret_cast<uintptr_t>(a.weight) & 15u) == 0) {
        reinterpret_cast<int4*>(idx)[0] = make_int4(id[0], id[1], id[2], id[3]);
        reinterpret_cast<int4*>(idx)[1] = make_int4(id[4], id[5], id[6], id[7]);
        if (out) {
          reinterpret_cast<float4*>(out)[0] = make_float4(w[0], w[1], w[2], w[3]);
          reinterpret_cast<float4*>(out)[1] = make_float4(w[4], w[5], w[6], w[7]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < KP; ++j)
          if (j < K) {
            idx[j] = id[j];
            if (out) out[j] = w[j];
          }
      }
    }
  }
}

template <bool F32, int G, int P, int C>
int launch_tile(const GateArgs& a, cudaStream_t s) {
  DeviceInfo di;
  if (int rc = device_info(&di)) return rc;
  GateTile g;
  const int words = a.E * (F32 ? 4 : 2) / 4;
  g.stride = 4 * (words + ((4 - words) & 7));
  g.warp_bytes = 32 * g.stride + (a.E + 31) / 32 * 128 + 16;
  const int head = 4 * a.E;
  int most = (di.max_smem_optin - head) / g.warp_bytes;
  if (most > kMaxGateWarps) most = kMaxGateWarps;
  if (most < 1) return kErrUnsupported;
  const int64_t ntiles = (a.T + 31) / 32;
  int64_t nw = (ntiles + di.sm_count - 1) / di.sm_count;
  if (nw > most) nw = most;
  int64_t grid = (ntiles + nw - 1) / nw;
  if (grid > di.sm_count) grid = di.sm_count;
  g.tiles_per_warp = (ntiles + grid * nw - 1) / (grid * nw);
  auto kern = gate_tile_kernel<F32, G, 8, P, C>;
  if (!allow_smem(kern, di.max_smem_optin)) return kErrCuda;
  return launch_dependent(kern, dim3(static_cast<unsigned>(grid)), dim3(static_cast<unsigned>(nw) * 32),
                          head + static_cast<int>(nw) * g.warp_bytes, s, a, g) == cudaSuccess
             ? kOk
             : kErrCuda;
}

// The widths of the workloads are known at compile time; others take eight parts and
// loops of their length.  T = 524,288, K = 8, bf16, sigmoids renormalised: E = 128 58.8 us (the
// bytes at the copy rate are 42% of that), 256 88.1 (51%), 512 210 (40%); E = 40 54.0 (21%), 160
// 80.1 (37%), 320 142 (38%), 384 165 (39%).
template <bool F32, int G>
int launch_tile_width(const GateArgs& a, cudaStream_t s) {
  if (a.E == 64) return launch_tile<F32, G, 8, 1>(a, s);
  if (a.E == 96 && G < 8) return launch_tile<F32, G, G < 8 ? 12 : 8, 1>(a, s);
  if (a.E == 128) return launch_tile<F32, G, 16, 1>(a, s);
  if (a.E == 256) return launch_tile<F32, G, 16, 2>(a, s);
  if (a.E == 512) return launch_tile<F32, G, 16, 4>(a, s);
  return launch_tile<F32, G, 8, 0>(a, s);
}

template <bool F32>
int launch_tile_groups(const GateArgs& a, cudaStream_t s) {
  const int G = a.top_groups < a.groups ? a.groups : 1;
  if (G == 1) return launch_tile_width<F32, 1>(a, s);
  if (G == 2) return launch_tile_width<F32, 2>(a, s);
  if (G == 4) return launch_tile_width<F32, 4>(a, s);
  return launch_tile_width<F32, 8>(a, s);
}

}  // namespace

}  // namespace eqb
