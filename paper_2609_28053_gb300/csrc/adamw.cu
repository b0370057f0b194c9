// adamw.cu -- one AdamW step over many tensors in one launch, with the two
// moments in 32 bits or in 8 (e4m3 with an fp32 scale per 256 elements).
//
//   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2,
//   p = (1 - lr wd) p - (lr / bc1) m / (sqrt(v) / sqrt(bc2) + eps)
//
// (decoupled weight decay, bc_i = 1 - beta_i^step).  A stream: every element
// is read once and written once, so memory bounds it.  The tensors' pointers
// and lengths travel in the launch's parameters (no table in device memory, so
// nothing to copy, to own or to keep), a block finds its tensor by bisection,
// and a warp takes 256 consecutive elements at a time, eight a lane: the elements
// of one 8-bit scale, whose largest magnitude is then one reduction within the
// warp.  Every operation up to the moments and their scales is rounded to
// nearest by itself, so that the 8-bit codes do not depend on how the compiler
// fuses them.
#include "eqb_device.cuh"

namespace eqb {

namespace {

constexpr int kAdamThreads = 256;
constexpr int kAdamWarps = kAdamThreads / 32;
constexpr int kUnit = 256;       // elements a warp takes at a time: the block of an 8-bit scale
constexpr float kTop = 448.0f;   // largest e4m3 value
constexpr float kLeast = 0.001953125f;       // 2^-9, the least positive one
constexpr float kMinNormal = 1.17549435e-38f;

template <int CAP>
struct AdamwTable {
  AdamwTensor t[CAP];
  int32_t first[CAP];  // the first block of each tensor
  int32_t count;
  int32_t units;       // units a block takes
  AdamwScalars s;
};

// Root and quotient of the update, within 2 ulps: the rounded-to-nearest ones
// take about twenty instructions of the sixty an element has time for.
__device__ __forceinline__ float sqrt_approx(float x) {
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// two e4m3 codes -> fp32, and back (nearest even, NaN stays NaN)
__device__ __forceinline__ void e4m3x2_to_f32(uint32_t c, float& lo, float& hi) {
  uint32_t h;
  asm("{\n\t.reg .b16 t;\n\tcvt.u16.u32 t, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, t;\n\t}" : "=r"(h) : "r"(c));
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}"
      : "=f"(lo), "=f"(hi)
      : "r"(h));
}
__device__ __forceinline__ uint32_t f32_to_e4m3x2(float lo, float hi) {
  uint32_t r;
  asm("{\n\t.reg .b16 t;\n\tcvt.rn.satfinite.e4m3x2.f32 t, %2, %1;\n\tcvt.u32.u16 %0, t;\n\t}"
      : "=r"(r)
      : "f"(lo), "f"(hi));
  return r;
}

// Element j (0..7) of a lane: two groups of four neighbours where the unit is
// whole and aligned, else one of every 32.
template <bool VEC>
__device__ __forceinline__ int place(int j, int lane) {
  return VEC ? (j >> 2) * 128 + lane * 4 + (j & 3) : j * 32 + lane;
}

template <bool BF16, bool VEC>
__device__ __forceinline__ void load8(const void* src, int64_t base, int left, int lane, float (&x)[8]) {
  if constexpr (VEC && BF16) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint2 w = __ldcs(reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(src) + base + h * 128) + lane);
      x[4 * h] = bf16_lo(w.x); x[4 * h + 1] = bf16_hi(w.x);
      x[4 * h + 2] = bf16_lo(w.y); x[4 * h + 3] = bf16_hi(w.y);
    }
  } else if constexpr (VEC) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float4 w = __ldcs(reinterpret_cast<const float4*>(static_cast<const float*>(src) + base + h * 128) + lane);
      x[4 * h] = w.x; x[4 * h + 1] = w.y; x[4 * h + 2] = w.z; x[4 * h + 3] = w.w;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = place<false>(j, lane);
      x[j] = i >= left ? 0.f
             : BF16    ? bf16_bits_to_f32(static_cast<const uint16_t*>(src)[base + i])
                       : static_cast<const float*>(src)[base + i];
    }
  }
}

template <bool BF16, bool VEC>
__device__ __forceinline__ void store8(void* dst, int64_t base, int left, int lane, const float (&x)[8]) {
  if constexpr (VEC && BF16) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      __stcs(reinterpret_cast<uint2*>(static_cast<uint16_t*>(dst) + base + h * 128) + lane,
             make_uint2(pack_bf16x2_rn(x[4 * h], x[4 * h + 1]), pack_bf16x2_rn(x[4 * h + 2], x[4 * h + 3])));
  } else if constexpr (VEC) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      __stcs(reinterpret_cast<float4*>(static_cast<float*>(dst) + base + h * 128) + lane,
             make_float4(x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = place<false>(j, lane);
      if (i >= left) continue;
      if (BF16) static_cast<uint16_t*>(dst)[base + i] = static_cast<uint16_t>(pack_bf16x2_rn(x[j], 0.f));
      else static_cast<float*>(dst)[base + i] = x[j];
    }
  }
}

template <bool VEC>
__device__ __forceinline__ void load8_e4m3(const void* src, int64_t base, int left, int lane, float scale,
                                           float (&x)[8]) {
  const uint8_t* c = static_cast<const uint8_t*>(src) + base;
  if constexpr (VEC) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t w = __ldcs(reinterpret_cast<const uint32_t*>(c + h * 128) + lane);
      e4m3x2_to_f32(w & 0xffffu, x[4 * h], x[4 * h + 1]);
      e4m3x2_to_f32(w >> 16, x[4 * h + 2], x[4 * h + 3]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = place<false>(j, lane);
      float none;
      e4m3x2_to_f32(i < left ? c[i] : 0u, x[j], none);
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = __fmul_rn(x[j], scale);
}

template <bool VEC>
__device__ __forceinline__ void store8_e4m3(void* dst, int64_t base, int left, int lane, const float (&x)[8]) {
  uint8_t* c = static_cast<uint8_t*>(dst) + base;
  if constexpr (VEC) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      __stcs(reinterpret_cast<uint32_t*>(c + h * 128) + lane,
             f32_to_e4m3x2(x[4 * h], x[4 * h + 1]) | f32_to_e4m3x2(x[4 * h + 2], x[4 * h + 3]) << 16);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = place<false>(j, lane);
      if (i < left) c[i] = static_cast<uint8_t>(f32_to_e4m3x2(x[j], 0.f));
    }
  }
}

// The scale of a unit and its reciprocal, from the largest magnitude of the
// warp's elements (a NaN is larger than all, so it stays visible).  A unit
// below the normal numbers is stored as zeros.
__device__ __forceinline__ void unit_scale(const float (&x)[8], float& scale, float& inv) {
  uint32_t a = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) a = max(a, __float_as_uint(x[j]) & 0x7fffffffu);
  scale = __fmul_rn(__uint_as_float(__reduce_max_sync(kFull, a)), 1.0f / kTop);
  if (scale < kMinNormal) scale = 0.f;
  inv = scale > 0.f ? __frcp_rn(scale) : 0.f;
}

// One unit of a tensor: `left` elements from `base` on (256 where VEC).
template <int BITS, bool PB, bool GB, bool VEC>
__device__ __forceinline__ bool adamw_unit(const AdamwTensor& t, const AdamwScalars& s, float gs, int64_t base, int left,
                                           int lane) {
  float p[8], g[8], m[8], v[8];
  load8<PB, VEC>(t.p, base, left, lane, p);
  load8<GB, VEC>(t.g, base, left, lane, g);
  const int64_t unit = base / kUnit;
  if constexpr (BITS == 32) {
    load8<false, VEC>(t.m, base, left, lane, m);
    load8<false, VEC>(t.v, base, left, lane, v);
  } else {
    load8_e4m3<VEC>(t.m, base, left, lane, t.ms[unit], m);
    load8_e4m3<VEC>(t.v, base, left, lane, t.vs[unit], v);
  }
  bool bad = false;
  float root[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float gj = __fmul_rn(g[j], gs);
    if constexpr (BITS == 8) v[j] = __fmul_rn(v[j], v[j]);  // the root is what 8 bits hold
    m[j] = __fadd_rn(__fmul_rn(m[j], s.b1), __fmul_rn(gj, s.c1));
    v[j] = __fadd_rn(__fmul_rn(v[j], s.b2), __fmul_rn(__fmul_rn(gj, s.c2), gj));
    root[j] = sqrt_approx(v[j]);
    const float den = __fadd_rn(__fmul_rn(root[j], s.rbc2), s.eps);
    p[j] = __fsub_rn(__fmul_rn(p[j], s.decay), __fmul_rn(__fdividef(m[j], den), s.step));
    bad |= !(fabsf(p[j]) < INFINITY) || !(v[j] < INFINITY);
  }
  store8<PB, VEC>(t.p, base, left, lane, p);
  if (!PB && t.copy) store8<true, VEC>(t.copy, base, left, lane, p);
  if constexpr (BITS == 32) {
    store8<false, VEC>(t.m, base, left, lane, m);
    store8<false, VEC>(t.v, base, left, lane, v);
  } else {
    float ms, mi, vs, vi;
    unit_scale(m, ms, mi);
    unit_scale(root, vs, vi);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      m[j] = __fmul_rn(m[j], mi);
      const float u = __fmul_rn(root[j], vi);
      // a root that is not zero stays so: eps alone in the denominator would
      // make a step out of what is left in m
      root[j] = vi > 0.f && root[j] > 0.f ? fmaxf(u, kLeast) : u;
    }
    store8_e4m3<VEC>(t.m, base, left, lane, m);
    store8_e4m3<VEC>(t.v, base, left, lane, root);
    if (lane == 0) {
      t.ms[unit] = ms;
      t.vs[unit] = vs;
    }
  }
  return bad;
}

template <int CAP, int BITS>
__global__ void __launch_bounds__(kAdamThreads) adamw_kernel(const __grid_constant__ AdamwTable<CAP> tab) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int lo = 0, hi = tab.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (tab.first[mid] <= static_cast<int32_t>(blockIdx.x)) lo = mid; else hi = mid - 1;
  }
  const AdamwTensor& t = tab.t[lo];
  const int64_t chunk = static_cast<int64_t>(blockIdx.x) - tab.first[lo];
  griddep_wait();
  const float gs = tab.s.grad_scale ? *tab.s.grad_scale : 1.0f;
  bool bad = false;
  for (int k = warp; k < tab.units; k += kAdamWarps) {
    const int64_t base = (chunk * tab.units + k) * kUnit;
    if (base >= t.n) break;
    const int left = t.n - base < kUnit ? static_cast<int>(t.n - base) : kUnit;
    const int kind = t.flags & 3;  // uniform in the block
    if ((t.flags & 4) && left == kUnit) {
      if (kind == 0) bad |= adamw_unit<BITS, false, false, true>(t, tab.s, gs, base, left, lane);
      else if (kind == 1) bad |= adamw_unit<BITS, true, false, true>(t, tab.s, gs, base, left, lane);
      else if (kind == 2) bad |= adamw_unit<BITS, false, true, true>(t, tab.s, gs, base, left, lane);
      else bad |= adamw_unit<BITS, true, true, true>(t, tab.s, gs, base, left, lane);
    } else {
      if (kind == 0) bad |= adamw_unit<BITS, false, false, false>(t, tab.s, gs, base, left, lane);
      else if (kind == 1) bad |= adamw_unit<BITS, true, false, false>(t, tab.s, gs, base, left, lane);
      else if (kind == 2) bad |= adamw_unit<BITS, false, true, false>(t, tab.s, gs, base, left, lane);
      else bad |= adamw_unit<BITS, true, true, false>(t, tab.s, gs, base, left, lane);
    }
  }
  if (bad) raise_flag(tab.s.err, kErrNonfinite);
}

template <int CAP>
int launch_adamw_cap(const AdamwTensor* t, int count, int bits, const AdamwScalars& sc, cudaStream_t s) {
  DeviceInfo di;
  if (int rc = device_info(&di)) return rc;
  AdamwTable<CAP> tab;
  tab.s = sc;
  tab.count = 0;
  tab.units = 4 * kAdamWarps;
  int64_t blocks = 0;
  for (int i = 0; i < count; ++i) {
    tab.t[tab.count] = t[i];
    tab.first[tab.count++] = static_cast<int32_t>(blocks);
    const int64_t per = static_cast<int64_t>(tab.units) * kUnit;
    blocks += (t[i].n + per - 1) / per;
    if (blocks > INT32_MAX) return kErrUnsupported;
  }
  const auto kern = bits == 8 ? adamw_kernel<CAP, 8> : adamw_kernel<CAP, 32>;
  return launch_dependent(kern, dim3(static_cast<unsigned>(blocks)), dim3(kAdamThreads), 0, s, tab) == cudaSuccess
             ? kOk
             : kErrCuda;
}

}  // namespace

// At most kAdamwBatch tensors, none of them empty.
int launch_adamw(const AdamwTensor* t, int count, int bits, const AdamwScalars& sc, cudaStream_t s) {
  return count <= 16 ? launch_adamw_cap<16>(t, count, bits, sc, s) : launch_adamw_cap<kAdamwBatch>(t, count, bits, sc, s);
}

}  // namespace eqb
