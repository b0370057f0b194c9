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
#include "f32x2.cuh"

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

// Two e4m3 codes -> fp32, and back (nearest even, NaN stays NaN).
__device__ __forceinline__ F2 e4m3x2_to_f32(uint32_t c) {
  float lo, hi;
  asm("{\n\t.reg .b16 t, a, b;\n\t.reg .b32 h;\n\tcvt.u16.u32 t, %2;\n\tcvt.rn.f16x2.e4m3x2 h, t;\n\t"
      "mov.b32 {a, b}, h;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}"
      : "=f"(lo), "=f"(hi)
      : "r"(c));
  return f2(lo, hi);
}
__device__ __forceinline__ uint32_t f32_to_e4m3x2(F2 x) {
  uint32_t r;
  asm("{\n\t.reg .b16 t;\n\tcvt.rn.satfinite.e4m3x2.f32 t, %2, %1;\n\tcvt.u32.u16 %0, t;\n\t}"
      : "=r"(r)
      : "f"(lo2(x)), "f"(hi2(x)));
  return r;
}

// Where a lane's eight elements lie in its unit, in pairs: neighbours
// (Run, for rows of 2- and 1-byte elements), two groups of four neighbours
// (Quads, where 4-byte elements are among them), or one of every 32 (Single:
// arrays that are not aligned, and a tensor's last unit).
enum Layout { Run, Quads, Single };

template <bool BF16, Layout L>
__device__ __forceinline__ void load8(const void* src, int64_t base, int left, int lane, F2 (&x)[4]) {
  if constexpr (L == Single) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = j * 32 + lane;
      v[j] = i >= left ? 0.f
             : BF16    ? bf16_bits_to_f32(static_cast<const uint16_t*>(src)[base + i])
                       : static_cast<const float*>(src)[base + i];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = f2(v[2 * j], v[2 * j + 1]);
  } else if constexpr (BF16 && L == Run) {
    const uint4 w = __ldcs(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(src) + base) + lane);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = f2(bf16_lo(u[j]), bf16_hi(u[j]));
  } else if constexpr (BF16) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint2 w = __ldcs(reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(src) + base + h * 128) + lane);
      x[2 * h] = f2(bf16_lo(w.x), bf16_hi(w.x));
      x[2 * h + 1] = f2(bf16_lo(w.y), bf16_hi(w.y));
    }
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(src) + base);
      const float4 w = __ldcs(p + (L == Run ? 2 * lane + h : 32 * h + lane));
      x[2 * h] = f2(w.x, w.y);
      x[2 * h + 1] = f2(w.z, w.w);
    }
  }
}

template <bool BF16, Layout L>
__device__ __forceinline__ void store8(void* dst, int64_t base, int left, int lane, const F2 (&x)[4]) {
  if constexpr (L == Single) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = j * 32 + lane;
      const float v = j & 1 ? hi2(x[j >> 1]) : lo2(x[j >> 1]);
      if (i >= left) continue;
      if (BF16) static_cast<uint16_t*>(dst)[base + i] = static_cast<uint16_t>(pack_bf16x2_rn(v, 0.f));
      else static_cast<float*>(dst)[base + i] = v;
    }
  } else if constexpr (BF16) {
    uint32_t u[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) u[j] = pack_bf16x2_rn(lo2(x[j]), hi2(x[j]));
    if constexpr (L == Run) {
      __stcs(reinterpret_cast<uint4*>(static_cast<uint16_t*>(dst) + base) + lane, make_uint4(u[0], u[1], u[2], u[3]));
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        __stcs(reinterpret_cast<uint2*>(static_cast<uint16_t*>(dst) + base + h * 128) + lane, make_uint2(u[2 * h], u[2 * h + 1]));
    }
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float4* p = reinterpret_cast<float4*>(static_cast<float*>(dst) + base);
      __stcs(p + (L == Run ? 2 * lane + h : 32 * h + lane),
             make_float4(lo2(x[2 * h]), hi2(x[2 * h]), lo2(x[2 * h + 1]), hi2(x[2 * h + 1])));
    }
  }
}

template <Layout L>
__device__ __forceinline__ void load8_e4m3(const void* src, int64_t base, int left, int lane, float scale, F2 (&x)[4]) {
  const uint8_t* c = static_cast<const uint8_t*>(src) + base;
  if constexpr (L == Single) {
    uint32_t v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j * 32 + lane < left ? c[j * 32 + lane] : 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = e4m3x2_to_f32(v[2 * j] | v[2 * j + 1] << 8);
  } else {
    uint32_t w[2];
    if constexpr (L == Run) {
      const uint2 u = __ldcs(reinterpret_cast<const uint2*>(c) + lane);
      w[0] = u.x;
      w[1] = u.y;
    } else {
      w[0] = __ldcs(reinterpret_cast<const uint32_t*>(c) + lane);
      w[1] = __ldcs(reinterpret_cast<const uint32_t*>(c + 128) + lane);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      x[2 * h] = e4m3x2_to_f32(w[h] & 0xffffu);
      x[2 * h + 1] = e4m3x2_to_f32(w[h] >> 16);
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = mul2(x[j], splat2(scale));
}

template <Layout L>
__device__ __forceinline__ void store8_e4m3(void* dst, int64_t base, int left, int lane, const F2 (&x)[4]) {
  uint8_t* c = static_cast<uint8_t*>(dst) + base;
  uint32_t p[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) p[j] = f32_to_e4m3x2(x[j]);
  if constexpr (L == Single) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j * 32 + lane < left) c[j * 32 + lane] = static_cast<uint8_t>(j & 1 ? p[j >> 1] >> 8 : p[j >> 1]);
  } else if constexpr (L == Run) {
    __stcs(reinterpret_cast<uint2*>(c) + lane, make_uint2(p[0] | p[1] << 16, p[2] | p[3] << 16));
  } else {
    __stcs(reinterpret_cast<uint32_t*>(c) + lane, p[0] | p[1] << 16);
    __stcs(reinterpret_cast<uint32_t*>(c + 128) + lane, p[2] | p[3] << 16);
  }
}

// The scale of a unit and its reciprocal, from the largest magnitude of the
// warp's elements (a NaN is larger than all, so it stays visible).  A unit
// below the normal numbers is stored as zeros.  False if it is not finite.
__device__ __forceinline__ bool unit_scale(const F2 (&x)[4], float& scale, float& inv) {
  uint32_t a = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    a = max(a, max(__float_as_uint(lo2(x[j])) & 0x7fffffffu, __float_as_uint(hi2(x[j])) & 0x7fffffffu));
  a = __reduce_max_sync(kFull, a);
  scale = __fmul_rn(__uint_as_float(a), 1.0f / kTop);
  if (scale < kMinNormal) scale = 0.f;
  inv = scale > 0.f ? __frcp_rn(scale) : 0.f;
  return a < 0x7f800000u;
}

// One unit of a tensor: `left` elements from `base` on (256 unless Single).
// The update's root and quotient are within 2 ulps: rounded to nearest they take
// about twenty instructions of the fifty-five that an 8-bit element has time for.
template <int BITS, bool PB, bool GB, Layout L>
__device__ __forceinline__ bool adamw_unit(const AdamwTensor& t, const AdamwScalars& s, float gs, int64_t base, int left,
                                           int lane) {
  F2 p[4], g[4], m[4], v[4];
  const int64_t unit = base / kUnit;
  float ms = 0.f, vs = 0.f;
  if constexpr (BITS == 8) {
    ms = t.ms[unit];
    vs = t.vs[unit];
  }
  load8<PB, L>(t.p, base, left, lane, p);
  load8<GB, L>(t.g, base, left, lane, g);
  if constexpr (BITS == 32) {
    load8<false, L>(t.m, base, left, lane, m);
    load8<false, L>(t.v, base, left, lane, v);
  } else {
    load8_e4m3<L>(t.m, base, left, lane, ms, m);
    load8_e4m3<L>(t.v, base, left, lane, vs, v);
  }
  bool bad = false;
  F2 root[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const F2 gj = mul2(g[j], splat2(gs));
    if constexpr (BITS == 8) v[j] = mul2(v[j], v[j]);  // the root is what 8 bits hold
    m[j] = add2(mul2(m[j], splat2(s.b1)), mul2(gj, splat2(s.c1)));
    v[j] = add2(mul2(v[j], splat2(s.b2)), mul2(mul2(gj, splat2(s.c2)), gj));
    root[j] = f2(sqrt_approx(lo2(v[j])), sqrt_approx(hi2(v[j])));
    const F2 den = add2(mul2(root[j], splat2(s.rbc2)), splat2(s.eps));
    const F2 q = mul2(m[j], f2(rcp_approx(lo2(den)), rcp_approx(hi2(den))));
    p[j] = sub2(mul2(p[j], splat2(s.decay)), mul2(q, splat2(s.step)));
    if constexpr (BITS == 32)
      bad |= !(fabsf(lo2(m[j])) < INFINITY) || !(fabsf(hi2(m[j])) < INFINITY) || !(lo2(v[j]) < INFINITY) ||
             !(hi2(v[j]) < INFINITY);
  }
  store8<PB, L>(t.p, base, left, lane, p);
  if (!PB && t.copy) store8<true, L>(t.copy, base, left, lane, p);
  if constexpr (BITS == 32) {
    store8<false, L>(t.m, base, left, lane, m);
    store8<false, L>(t.v, base, left, lane, v);
  } else {
    float mi, vi;
    bad = !unit_scale(m, ms, mi);
    bad |= !unit_scale(root, vs, vi);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m[j] = mul2(m[j], splat2(mi));
      const F2 u = mul2(root[j], splat2(vi));
      // a root that is not zero stays so: eps alone in the denominator would
      // make a step out of what is left in m.  (fmaxf would drop a NaN.)
      root[j] = f2(lo2(root[j]) > 0.f && lo2(u) < kLeast && vi > 0.f ? kLeast : lo2(u),
                   hi2(root[j]) > 0.f && hi2(u) < kLeast && vi > 0.f ? kLeast : hi2(u));
    }
    store8_e4m3<L>(t.m, base, left, lane, m);
    store8_e4m3<L>(t.v, base, left, lane, root);
    if (lane == 0) {
      t.ms[unit] = ms;
      t.vs[unit] = vs;
    }
  }
  return bad;
}

template <int BITS, bool PB, bool GB>
__device__ __forceinline__ bool adamw_any(const AdamwTensor& t, const AdamwScalars& s, float gs, int64_t base, int left,
                                          int lane) {
  constexpr Layout wide = BITS == 8 && PB ? Run : Quads;
  if ((t.flags & 4) && left == kUnit) return adamw_unit<BITS, PB, GB, wide>(t, s, gs, base, left, lane);
  return adamw_unit<BITS, PB, GB, Single>(t, s, gs, base, left, lane);
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
    if (kind == 0) bad |= adamw_any<BITS, false, false>(t, tab.s, gs, base, left, lane);
    else if (kind == 1) bad |= adamw_any<BITS, true, false>(t, tab.s, gs, base, left, lane);
    else if (kind == 2) bad |= adamw_any<BITS, false, true>(t, tab.s, gs, base, left, lane);
    else bad |= adamw_any<BITS, true, true>(t, tab.s, gs, base, left, lane);
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
  // a block takes 32 units, or as few as 8 where the blocks would be too few to
  // fill the SMs four times (each with four blocks)
  int64_t units = 0;
  for (int i = 0; i < count; ++i) units += (t[i].n + kUnit - 1) / kUnit;
  int64_t per_warp = units / (static_cast<int64_t>(kAdamWarps) * di.sm_count * 16);
  tab.units = kAdamWarps * static_cast<int>(per_warp < 1 ? 1 : per_warp > 4 ? 4 : per_warp);
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
