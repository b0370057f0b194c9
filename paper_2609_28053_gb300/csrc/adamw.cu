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
// warp.  With 8-bit states a lane reads 48 bytes a unit, too few to hide a
// load's latency behind the warps of an SM, so there each warp fetches its units
// by bulk copies into a ring of its own in shared memory (192 matrices of 2^21 bf16
// parameters: 625 us, 6.5 TB/s; 1,148 by loads into registers).  With 32-bit states
// and bf16 gradients and copies the same take 1,630 us, 6.9 TB/s.  Of 8-bit states
// every operation up to the moments, their scales and codes is rounded to nearest
// by itself, so that a code does not depend on how operations are fused.
#include "eqb_device.cuh"
#include "f32x2.cuh"
#include "mbarrier.cuh"

namespace eqb {

namespace {

constexpr int kAdamThreads = 256;
constexpr int kAdamWarps = kAdamThreads / 32;
constexpr int kUnit = 256;       // elements a warp takes at a time: the block of an 8-bit scale
constexpr float kTop = 448.0f;   // largest e4m3 value
constexpr float kLeast = 0.001953125f;  // 2^-9, the least positive one
constexpr float kFull8 = 0.015625f;     // 2^-6, from which on all have three places
constexpr float kMinNormal = 1.17549435e-38f;

template <int CAP>
struct AdamwTable {
  AdamwTensor t[CAP];
  int32_t first[CAP];  // the first block of each tensor
  int32_t count;
  int32_t units;       // units a block takes
  int32_t stage;       // bytes of a stage of a warp's ring (8 bits)
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

// Eight elements of a lane as they lie in memory: W words for elements of
// 4 W / 8 bytes (single ones of 1 and 2 bytes are packed as the wide loads
// have them).
template <int W, Layout L>
__device__ __forceinline__ void load_words(const void* src, int64_t base, int left, int lane, uint32_t (&w)[W]) {
  constexpr int B = W / 2;  // bytes an element
  const uint8_t* p = static_cast<const uint8_t*>(src) + base * B;
  if constexpr (L == Single) {
    uint32_t v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = j * 32 + lane;
      v[j] = 0;
      if (i < left)
        v[j] = B == 4 ? reinterpret_cast<const uint32_t*>(p)[i] : B == 2 ? reinterpret_cast<const uint16_t*>(p)[i] : p[i];
    }
#pragma unroll
    for (int k = 0; k < W; ++k) {
      if constexpr (B == 4) w[k] = v[k];
      else if constexpr (B == 2) w[k] = v[2 * k] | v[2 * k + 1] << 16;
      else w[k] = v[4 * k] | v[4 * k + 1] << 8 | v[4 * k + 2] << 16 | v[4 * k + 3] << 24;
    }
  } else if constexpr (L == Run && W == 2) {
    const uint2 u = __ldcs(reinterpret_cast<const uint2*>(p) + lane);
    w[0] = u.x; w[1] = u.y;
  } else if constexpr (L == Run) {
#pragma unroll
    for (int h = 0; h < W / 4; ++h) {
      const uint4 u = __ldcs(reinterpret_cast<const uint4*>(p) + W / 4 * lane + h);
      w[4 * h] = u.x; w[4 * h + 1] = u.y; w[4 * h + 2] = u.z; w[4 * h + 3] = u.w;
    }
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (W == 8) {
        const uint4 u = __ldcs(reinterpret_cast<const uint4*>(p) + 32 * h + lane);
        w[4 * h] = u.x; w[4 * h + 1] = u.y; w[4 * h + 2] = u.z; w[4 * h + 3] = u.w;
      } else if constexpr (W == 4) {
        const uint2 u = __ldcs(reinterpret_cast<const uint2*>(p) + 32 * h + lane);
        w[2 * h] = u.x; w[2 * h + 1] = u.y;
      } else {
        w[h] = __ldcs(reinterpret_cast<const uint32_t*>(p) + 32 * h + lane);
      }
    }
  }
}

// The words' values, in pairs.
__device__ __forceinline__ void values_of(const uint32_t (&w)[8], F2 (&x)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = f2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
}
__device__ __forceinline__ void values_of(const uint32_t (&w)[4], F2 (&x)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = f2(bf16_lo(w[j]), bf16_hi(w[j]));
}
__device__ __forceinline__ void values_of(const uint32_t (&w)[2], F2 (&x)[4]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    x[2 * h] = e4m3x2_to_f32(w[h] & 0xffffu);
    x[2 * h + 1] = e4m3x2_to_f32(w[h] >> 16);
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

// a b + c d, each operation rounded.
__device__ __forceinline__ float ema(float a, float b, float c, float d) {
  return __fadd_rn(__fmul_rn(a, b), __fmul_rn(c, d));
}

// fp32 max of a and |b| that propagates NaN.
__device__ __forceinline__ float max_abs(float a, float b) { return fmax_nan(a, fabsf(b)); }

// The largest magnitude of the warp's elements.
__device__ __forceinline__ float largest(const F2 (&x)[4]) {
  float a = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) a = max_abs(max_abs(a, lo2(x[j])), hi2(x[j]));
  // bit patterns of magnitudes are in their order, NaN above all
  return __uint_as_float(__reduce_max_sync(kFull, __float_as_uint(a)));
}

// The scale of a unit and its reciprocal, from its largest magnitude.  A unit
// below the normal numbers is stored as zeros.  False if it is not finite.
__device__ __forceinline__ bool unit_scale(float top, float& scale, float& inv) {
  scale = __fmul_rn(top, 1.0f / kTop);
  if (scale < kMinNormal) scale = 0.f;
  inv = scale > 0.f ? __frcp_rn(scale) : 0.f;
  return top < INFINITY;
}

// Whether x, of e4m3's full range, lies within 16 last places of the middle of
// two of its values.
__device__ __forceinline__ bool near_middle(float x) { return ((__float_as_uint(x) + 0x80010u) & 0xfffffu) <= 32u; }

// What a lane reads of one unit of a tensor: `left` elements from `base` on
// (256 unless Single).
template <int BITS, bool PB, bool GB>
struct UnitWords {
  uint32_t p[PB ? 4 : 8], g[GB ? 4 : 8], m[BITS / 4], v[BITS / 4];
  float ms, vs;
};
template <int BITS, bool PB, bool GB, Layout L>
__device__ __forceinline__ void load_unit(const AdamwTensor& t, int64_t base, int left, int lane, UnitWords<BITS, PB, GB>& w) {
  load_words<PB ? 4 : 8, L>(t.p, base, left, lane, w.p);
  load_words<GB ? 4 : 8, L>(t.g, base, left, lane, w.g);
  load_words<BITS / 4, L>(t.m, base, left, lane, w.m);
  load_words<BITS / 4, L>(t.v, base, left, lane, w.v);
  if constexpr (BITS == 8) {
    w.ms = t.ms[base / kUnit];
    w.vs = t.vs[base / kUnit];
  }
}

// The update's quotient is within 2 ulps (and with 32-bit states its root):
// rounded to nearest it takes about ten of the fifty-five instructions that an
// 8-bit element has time for.
template <int BITS, bool PB, bool GB, Layout L>
__device__ __forceinline__ bool adamw_unit(const AdamwTensor& t, const AdamwScalars& s, float gs, int64_t base, int left,
                                           int lane, const UnitWords<BITS, PB, GB>& w) {
  F2 p[4], g[4], m[4], v[4];
  const int64_t unit = base / kUnit;
  values_of(w.p, p);
  values_of(w.g, g);
  values_of(w.m, m);
  values_of(w.v, v);
  bool bad = false;
  F2 root[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const F2 gj = mul2(g[j], splat2(gs));
    if constexpr (BITS == 8) {
      m[j] = mul2(m[j], splat2(w.ms));
      v[j] = mul2(v[j], splat2(w.vs));
      v[j] = mul2(v[j], v[j]);  // the root is what 8 bits hold
    }
    if constexpr (BITS == 8) {
      // not in pairs: the assembler fuses those
      m[j] = f2(ema(lo2(m[j]), s.b1, lo2(gj), s.c1), ema(hi2(m[j]), s.b1, hi2(gj), s.c1));
      v[j] = f2(ema(lo2(v[j]), s.b2, __fmul_rn(lo2(gj), s.c2), lo2(gj)), ema(hi2(v[j]), s.b2, __fmul_rn(hi2(gj), s.c2), hi2(gj)));
    } else {
      m[j] = fma2(m[j], splat2(s.b1), mul2(gj, splat2(s.c1)));
      v[j] = fma2(v[j], splat2(s.b2), mul2(mul2(gj, splat2(s.c2)), gj));
    }
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
    // What 8 bits hold is rounded to nearest at every step up to its codes: a
    // code that falls the other way moves its value by a sixteenth, and the block's
    // scale with it once that value is the largest.
    float ms, vs, mi, vi;
    bad = !unit_scale(largest(m), ms, mi);
    const float v1 = largest(v);
    bad |= !(v1 < INFINITY);
    unit_scale(__fsqrt_rn(v1), vs, vi);
    float low = INFINITY;
    bool near = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m[j] = mul2(m[j], splat2(mi));
      root[j] = mul2(root[j], splat2(vi));
      low = fminf(low, fminf(lo2(root[j]), hi2(root[j])));
      near |= near_middle(lo2(root[j])) || near_middle(hi2(root[j]));
    }
    // Rounding the roots themselves takes ten instructions and a slow path each
    // (403M parameters 727 us, 625 with this test): only where one is so near the
    // middle of two codes that its last places decide, or below their full range.
    // There a root that is not zero does not become zero: eps alone in the
    // denominator would make a step out of what is left in m.
    if (near || (low < kFull8 && vi > 0.f)) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float r0 = __fsqrt_rn(lo2(v[j])), r1 = __fsqrt_rn(hi2(v[j]));
        const float u0 = __fmul_rn(r0, vi), u1 = __fmul_rn(r1, vi);
        root[j] = f2(r0 > 0.f && u0 < kLeast && vi > 0.f ? kLeast : u0, r1 > 0.f && u1 < kLeast && vi > 0.f ? kLeast : u1);
      }
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

// A warp's units of a block's chunk, numbers warp, warp + 8, ... of `units`;
// with 32-bit states the next one's loads are issued before the current one's
// arithmetic (403M fp32 parameters with bf16 gradients and copies 1,640 -> 1,618 us).
template <int BITS, bool PB, bool GB, Layout L>
__device__ __forceinline__ bool adamw_units(const AdamwTensor& t, const AdamwScalars& s, float gs, int64_t first, int units,
                                            int warp, int lane) {
  UnitWords<BITS, PB, GB> w, next;
  constexpr bool AHEAD = BITS == 32 && L != Single;
  bool bad = false;
  auto left_of = [&](int k) {
    const int64_t n = t.n - (first + k) * kUnit;
    return n < kUnit ? static_cast<int>(n) : kUnit;
  };
  if (AHEAD && warp < units) load_unit<BITS, PB, GB, L>(t, (first + warp) * kUnit, left_of(warp), lane, w);
  for (int k = warp; k < units; k += kAdamWarps) {
    if (!AHEAD)
      load_unit<BITS, PB, GB, L>(t, (first + k) * kUnit, left_of(k), lane, w);
    else if (k + kAdamWarps < units)
      load_unit<BITS, PB, GB, L>(t, (first + k + kAdamWarps) * kUnit, left_of(k + kAdamWarps), lane, next);
    bad |= adamw_unit<BITS, PB, GB, L>(t, s, gs, (first + k) * kUnit, left_of(k), lane, w);
    if (AHEAD) w = next;
  }
  return bad;
}

// A warp's ring: stages of two units (p, g, m and v one after the other, as far
// as the chunk goes), and where it stands.
struct AdamwRing {
  uint8_t* at;
  uint32_t bar;  // kRing barriers
  uint32_t bytes;
};
constexpr int kRing = 2;

// The whole units of a chunk with 8-bit states, through the ring: numbers
// 16 j + 2 warp and the one after it.  `stalled`: a wait ran out.
template <bool PB, bool GB>
__device__ __forceinline__ bool adamw_stream(const AdamwTensor& t, const AdamwScalars& s, float gs, int64_t first, int units,
                                             int warp, int lane, const AdamwRing& ring, volatile int* stalled) {
  constexpr uint32_t PE = PB ? 2 : 4, GE = GB ? 2 : 4, U = kUnit;
  const int nj = (units - 2 * warp + 2 * kAdamWarps - 1) / (2 * kAdamWarps);  // may be 0 or less
  auto unit_of = [&](int j) { return first + 2 * (j * kAdamWarps + warp); };
  auto count_of = [&](int j) { return min(2, units - 2 * (j * kAdamWarps + warp)); };
  auto issue = [&](int j) {
    if (lane == 0) {
      const int64_t u = unit_of(j);
      const uint32_t n = static_cast<uint32_t>(count_of(j)) * U, dst = smem_u32(ring.at) + (j & (kRing - 1)) * ring.bytes;
      const uint32_t bar = ring.bar + 8u * (j & (kRing - 1));
      mbar_expect_tx(bar, n * (PE + GE + 2));
      bulk_load(dst, static_cast<const uint8_t*>(t.p) + u * U * PE, n * PE, bar);
      bulk_load(dst + 2 * U * PE, static_cast<const uint8_t*>(t.g) + u * U * GE, n * GE, bar);
      bulk_load(dst + 2 * U * (PE + GE), static_cast<const uint8_t*>(t.m) + u * U, n, bar);
      bulk_load(dst + 2 * U * (PE + GE + 1), static_cast<const uint8_t*>(t.v) + u * U, n, bar);
    }
  };
  // lanes 0, 1: the scales of m of the two units, lanes 2, 3: of v
  auto scale_of = [&](int j) {
    const int64_t u = unit_of(j) + (lane & 1);
    return lane < 4 && (lane & 1) < count_of(j) ? (lane < 2 ? t.ms : t.vs)[u] : 0.f;
  };
  for (int j = 0; j < kRing && j < nj; ++j) issue(j);
  float scale = nj > 0 ? scale_of(0) : 0.f;
  bool bad = false;
  for (int j = 0; j < nj; ++j) {
    const float next = j + 1 < nj ? scale_of(j + 1) : 0.f;
    if (!__all_sync(kFull, mbar_wait(ring.bar + 8u * (j & (kRing - 1)), (j / kRing) & 1u, stalled))) {
      if (lane == 0) drain_loads(min(nj, j + kRing), kRing, [&](int k) { return ring.bar + 8u * k; });
      return bad;
    }
    const uint8_t* src = ring.at + (j & (kRing - 1)) * ring.bytes;
    const int n = count_of(j);
    for (int i = 0; i < n; ++i) {
      UnitWords<8, PB, GB> w;
      auto take = [&](uint32_t off, auto& x) {
        constexpr int W = sizeof(x) / 4;
        if constexpr (W == 2) {
          const uint2 v = reinterpret_cast<const uint2*>(src + off)[lane + 32 * i];
          x[0] = v.x; x[1] = v.y;
        } else {
#pragma unroll
          for (int h = 0; h < W / 4; ++h) {
            // Run: a lane's eight elements are neighbours; Quads: two groups of four
            const int c = PB ? W / 4 * lane + h : 32 * h + lane;
            const uint4 v = reinterpret_cast<const uint4*>(src + off)[c + 32 * (W / 4) * i];
            x[4 * h] = v.x; x[4 * h + 1] = v.y; x[4 * h + 2] = v.z; x[4 * h + 3] = v.w;
          }
        }
      };
      auto take_quads = [&](uint32_t off, auto& x) {  // the same of 2- and 1-byte elements in the layout Quads
        constexpr int W = sizeof(x) / 4;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if constexpr (W == 4) {
            const uint2 v = reinterpret_cast<const uint2*>(src + off)[64 * i + 32 * h + lane];
            x[2 * h] = v.x; x[2 * h + 1] = v.y;
          } else {
            x[h] = reinterpret_cast<const uint32_t*>(src + off)[64 * i + 32 * h + lane];
          }
        }
      };
      take(0, w.p);
      if constexpr (!PB && GB) take_quads(2 * U * PE, w.g);
      else take(2 * U * PE, w.g);
      if constexpr (PB) {
        take(2 * U * (PE + GE), w.m);
        take(2 * U * (PE + GE + 1), w.v);
      } else {
        take_quads(2 * U * (PE + GE), w.m);
        take_quads(2 * U * (PE + GE + 1), w.v);
      }
      w.ms = __shfl_sync(kFull, scale, i);
      w.vs = __shfl_sync(kFull, scale, 2 + i);
      bad |= adamw_unit<8, PB, GB, PB ? Run : Quads>(t, s, gs, (unit_of(j) + i) * U, kUnit, lane, w);
    }
    scale = next;
    __syncwarp();
    if (j + kRing < nj) issue(j + kRing);
  }
  return bad;
}

// The chunk of `units` units from number `first` of a tensor on, as far as the
// tensor goes.
template <int BITS, bool PB, bool GB>
__device__ __forceinline__ bool adamw_chunk(const AdamwTensor& t, const AdamwScalars& s, float gs, int64_t first, int units,
                                            int warp, int lane, const AdamwRing& ring, volatile int* stalled) {
  const int64_t whole = t.n / kUnit - first;  // whole units left
  const int all = static_cast<int>(min(static_cast<int64_t>(units), (t.n + kUnit - 1) / kUnit - first));
  if (!(t.flags & 4)) return adamw_units<BITS, PB, GB, Single>(t, s, gs, first, all, warp, lane);
  bool bad;
  const int n = whole < units ? static_cast<int>(whole) : units;
  if constexpr (BITS == 8) bad = adamw_stream<PB, GB>(t, s, gs, first, n, warp, lane, ring, stalled);
  else bad = adamw_units<BITS, PB, GB, Quads>(t, s, gs, first, n, warp, lane);
  if (whole < all && warp == 0) bad |= adamw_units<BITS, PB, GB, Single>(t, s, gs, first + whole, 1, 0, lane);
  return bad;
}

template <int CAP, int BITS>
__global__ void __launch_bounds__(kAdamThreads, BITS == 8 ? 4 : 2) adamw_kernel(const __grid_constant__ AdamwTable<CAP> tab) {
  extern __shared__ __align__(128) uint8_t sm[];
  __shared__ __align__(8) uint64_t bars[kAdamWarps * kRing];
  __shared__ int stalled;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int lo = 0, hi = tab.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (tab.first[mid] <= static_cast<int32_t>(blockIdx.x)) lo = mid; else hi = mid - 1;
  }
  const AdamwTensor& t = tab.t[lo];
  const int64_t chunk = static_cast<int64_t>(blockIdx.x) - tab.first[lo];
  AdamwRing ring{sm + static_cast<size_t>(warp) * kRing * tab.stage, smem_u32(bars + warp * kRing),
                 static_cast<uint32_t>(tab.stage)};
  if constexpr (BITS == 8) {
    if (lane == 0) {
      for (int k = 0; k < kRing; ++k) mbar_init(ring.bar + 8u * k, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (threadIdx.x == 0) stalled = 0;
    __syncthreads();
  }
  griddep_wait();
  const float gs = tab.s.grad_scale ? *tab.s.grad_scale : 1.0f;
  const int kind = t.flags & 3;  // uniform in the block
  const int64_t first = chunk * tab.units;
  bool bad;
  if (kind == 0) bad = adamw_chunk<BITS, false, false>(t, tab.s, gs, first, tab.units, warp, lane, ring, &stalled);
  else if (kind == 1) bad = adamw_chunk<BITS, true, false>(t, tab.s, gs, first, tab.units, warp, lane, ring, &stalled);
  else if (kind == 2) bad = adamw_chunk<BITS, false, true>(t, tab.s, gs, first, tab.units, warp, lane, ring, &stalled);
  else bad = adamw_chunk<BITS, true, true>(t, tab.s, gs, first, tab.units, warp, lane, ring, &stalled);
  if (bad) raise_flag(tab.s.err, kErrNonfinite);
  if (BITS == 8 && lane == 0 && *static_cast<volatile int*>(&stalled)) raise_flag(tab.s.err, kErrCuda);
}

template <int CAP>
int launch_adamw_cap(const AdamwTensor* t, int count, int bits, const AdamwScalars& sc, cudaStream_t s) {
  DeviceInfo di;
  if (int rc = device_info(&di)) return rc;
  AdamwTable<CAP> tab;
  tab.s = sc;
  tab.count = 0;
  // units a warp of a block takes: up to 4, with the rings of 8 bits up to 16 (two
  // rounds of a ring of two stages leave its start and end uncovered), or as few
  // as leave every SM four blocks four times over
  int64_t units = 0;
  for (int i = 0; i < count; ++i) units += (t[i].n + kUnit - 1) / kUnit;
  const int64_t most = bits == 8 ? 16 : 4;
  int64_t per_warp = units / (static_cast<int64_t>(kAdamWarps) * di.sm_count * 16);
  tab.units = kAdamWarps * static_cast<int>(per_warp < 1 ? 1 : per_warp > most ? most : per_warp);
  int64_t blocks = 0;
  for (int i = 0; i < count; ++i) {
    tab.t[tab.count] = t[i];
    tab.first[tab.count++] = static_cast<int32_t>(blocks);
    const int64_t per = static_cast<int64_t>(tab.units) * kUnit;
    blocks += (t[i].n + per - 1) / per;
    if (blocks > INT32_MAX) return kErrUnsupported;
  }
  // the widest element of p and g among the tensors sets the ring's stage
  int wide = 4;
  for (int i = 0; i < count; ++i) {
    const int w = (t[i].flags & 1 ? 2 : 4) + (t[i].flags & 2 ? 2 : 4);
    if (w > wide) wide = w;
  }
  tab.stage = bits == 8 ? 2 * kUnit * (wide + 2) : 0;
  const int smem = kAdamWarps * kRing * tab.stage;
  const auto kern = bits == 8 ? adamw_kernel<CAP, 8> : adamw_kernel<CAP, 32>;
  if (smem && !allow_smem(kern, kAdamWarps * kRing * 2 * kUnit * 10)) return kErrCuda;
  return launch_dependent(kern, dim3(static_cast<unsigned>(blocks)), dim3(kAdamThreads), smem, s, tab) == cudaSuccess ? kOk
                                                                                                                   : kErrCuda;
}

}  // namespace

// At most kAdamwBatch tensors, none of them empty.
int launch_adamw(const AdamwTensor* t, int count, int bits, const AdamwScalars& sc, cudaStream_t s) {
  return count <= 16 ? launch_adamw_cap<16>(t, count, bits, sc, s) : launch_adamw_cap<kAdamwBatch>(t, count, bits, sc, s);
}

}  // namespace eqb
