// quant.cu -- values in 8 bits (e4m3) with an fp32 scale for each block of 128:
//   scale = max |x| * fp32(1 / 448),   code = e4m3(x * fp32(1 / scale)),
// along a row (rows), along 128 rows (cols, turned), and over 128 x 128 (blocks).
//
// All three stream: two or four bytes a value in, one a copy out.  A block's values
// stay in registers between its maximum and its codes, so x is read once.  The
// maximum is one of magnitudes that NaN stays in, so that one comparison a block
// finds infinities and NaN.
#include "eqb_device.cuh"

namespace eqb {

namespace {

constexpr uint32_t kAbs2 = 0x7fff7fffu;

struct Scale {
  float scale, inv;
};
// From the largest magnitude of a block.
__device__ __forceinline__ Scale scale_of(float top) {
  Scale s;
  s.scale = __fmul_rn(top, 1.0f / 448.0f);
  if (s.scale < 0x1p-126f) s.scale = 0.f;
  s.inv = s.scale > 0.f ? __frcp_rn(s.scale) : 0.f;
  return s;
}
// Four codes, a's in the lowest byte.  The conversion rounds to nearest even and keeps
// what is above 448 there, so that the clamp is its own.
__device__ __forceinline__ uint32_t code4(float a, float b, float c, float d) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\t"
      "mov.b32 %0, {l, h};\n\t}"
      : "=r"(r)
      : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}
// The larger magnitudes of two bf16 pairs (their signs are anything; NaN stays).
__device__ __forceinline__ uint32_t larger2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// ---- rows.  A lane has 16 neighbours, eight lanes a block.
constexpr int kRowWarps = 8;

template <bool SLOT>
__global__ void __launch_bounds__(kRowWarps * 32)
    quant_rows_kernel(const uint16_t* __restrict__ x, int64_t T, int d, int strips, const int32_t* __restrict__ slot, int K,
                      uint8_t* __restrict__ q, float* __restrict__ scale, int32_t* err) {
  const int lane = threadIdx.x & 31, nb = (d + 127) / 128;
  const int64_t items = T * strips, R = T * K;
  griddep_wait();
  for (int64_t it = static_cast<int64_t>(blockIdx.x) * kRowWarps + (threadIdx.x >> 5); it < items;
       it += static_cast<int64_t>(gridDim.x) * kRowWarps) {
    const int64_t t = it / strips;
    const int j = static_cast<int>(it % strips) * 512 + lane * 16;
    if (SLOT) {  // a token that no expert has is not looked at
      bool any = false;
      for (int k = lane; k < K; k += 32) {
        const int r = __ldg(slot + t * K + k);
        any |= r >= 0 && r < R;
      }
      if (!__any_sync(kFull, any)) continue;
    }
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 0u;
    if (j < d) {
      const uint4* p = reinterpret_cast<const uint4*>(x + t * d + j);
      const uint4 a = __ldg(p), b = __ldg(p + 1);
      w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
      w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
    }
    uint32_t m = w[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) m = larger2(m, w[i]);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) m = larger2(m, __shfl_xor_sync(kFull, m, o));
    m &= kAbs2;
    const uint32_t top = max(m & 0xffffu, m >> 16);
    if (top >= 0x7f80u) raise_flag(err, kErrNonfinite);
    const Scale sc = scale_of(bf16_bits_to_f32(top));
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      c[i] = code4(bf16_lo(w[2 * i]) * sc.inv, bf16_hi(w[2 * i]) * sc.inv, bf16_lo(w[2 * i + 1]) * sc.inv,
                   bf16_hi(w[2 * i + 1]) * sc.inv);
    if (j >= d) continue;
    const uint4 out = make_uint4(c[0], c[1], c[2], c[3]);
    if (!SLOT) {
      *reinterpret_cast<uint4*>(q + t * d + j) = out;
      if ((lane & 7) == 0) scale[t * nb + j / 128] = sc.scale;
    } else {
      for (int k = 0; k < K; ++k) {
        const int64_t r = __ldg(slot + t * K + k);
        if (r < 0 || r >= R) continue;
        *reinterpret_cast<uint4*>(q + r * d + j) = out;
        if ((lane & 7) == 0) scale[r * nb + j / 128] = sc.scale;
      }
    }
  }
}

// The expert whose blocks contain block b (E if none): blocks[e] <= b < blocks[e + 1].
// A warp looks at 32 experts at a time.
__device__ __forceinline__ int expert_of_block(const int32_t* __restrict__ blocks, int E, int64_t b, int lane) {
  for (int e0 = 0; e0 < E; e0 += 32) {
    const int e = e0 + lane;
    const uint32_t hit = __ballot_sync(kFull, e < E && b < __ldg(blocks + min(e, E - 1) + 1));
    if (hit) return e0 + __ffs(hit) - 1;
  }
  return E;
}

// ---- cols.  A warp takes 128 rows x 32 columns, a lane 16 neighbouring rows x eight
// columns: 16 codes of a column are 16 bytes of the output's line, so that nothing
// is turned in shared memory and no warp waits for another; and of the 32 scales
// every lane forms one.  The next step's values are copied into the warp's own part of
// shared memory meanwhile (the lanes' registers have no room for them, nor for the
// numbers of their rows: 208 us where they were kept and others spilled).  Blocks go over
// all rows of a group of columns first: a gathered row is wanted by K experts at
// different times, and the group's columns of every token stay in L2 in between.
// T = 16,384, c = 4,096, K = 8, 128 experts: 194 us; 235 where 24 warps an SM read their
// values twice instead of keeping them, 218 with 128 x 64 a block, turned in shared memory,
// 444 with all of a row of blocks at a time and a scale formed by every thread that needs
// it.  What bounds it is waiting: neither the memory (39% of the copy rate under ncu, c = 2,048)
// nor the issue slots (43%) are full; a warp has one step, 64 bytes of every row, on its
// way.  Rows that are read once (K = 1) come at 94% of the copy rate.
constexpr int kColWarps = 8;
constexpr int kColSteps = 4;  // of kColWarps * 32 columns a block, at most
// 64 bytes of every row; 16 rows and 64 bytes apart, so that two lanes' rows lie in different banks
constexpr int kColGroup = 16 * 64 + 64, kColWarpBytes = 8 * kColGroup;

__global__ void __launch_bounds__(kColWarps * 32, 2) quant_cols_kernel(const QuantColsArgs a, int steps) {
  extern __shared__ __align__(16) uint8_t ahead[];
  __shared__ __align__(16) int tokens[128];  // rows of x (-1: zeros)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, q = lane & 3, rg = lane >> 2;
  uint8_t* mine = ahead + warp * kColWarpBytes + rg * kColGroup + q * 16;
  const int64_t b = blockIdx.x % a.P;
  const int c0 = static_cast<int>(blockIdx.x / a.P) * (steps * kColWarps * 32), c1 = min(c0 + steps * kColWarps * 32, a.c);
  griddep_wait();
  const int e = expert_of_block(a.blocks, a.E, b, lane);
  if (e >= a.E) return;
  const int64_t r0 = static_cast<int64_t>(__ldg(a.offsets + e)) + (b - __ldg(a.blocks + e)) * kExpertBlock;
  const int64_t r1 = min(static_cast<int64_t>(__ldg(a.offsets + e + 1)), a.R);
  if (threadIdx.x < 128) {
    const int64_t r = r0 + threadIdx.x;
    int n = -1;
    if (r >= 0 && r < r1) {
      n = static_cast<int>(r);
      if (a.entry) {
        n = __ldg(a.entry + r);
        if (n >= 0) n = static_cast<int>(static_cast<uint32_t>(n) / static_cast<uint32_t>(a.K));
      }
    }
    tokens[threadIdx.x] = n < a.T ? n : -1;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i)  // where there is no row, zeros stay in its place
    if (tokens[rg * 16 + i] < 0) *reinterpret_cast<uint4*>(mine + i * 64) = make_uint4(0u, 0u, 0u, 0u);
  const int64_t pitch = a.P * kExpertBlock;
  auto fetch = [&](int j) {  // a lane copies what it reads itself
    const uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(mine));
    if (j < c1) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int4 t = *reinterpret_cast<const int4*>(tokens + rg * 16 + 4 * g);
        const int from[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (from[i] >= 0)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + (4 * g + i) * 64),
                         "l"(a.x + static_cast<int64_t>(from[i]) * a.c + j)
                         : "memory");
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  fetch(c0 + warp * 32 + q * 8);
  for (int j0 = c0 + warp * 32; j0 < c1; j0 += kColWarps * 32) {
    const int j = j0 + q * 8;
    uint32_t w[16][4];  // [row][pair of columns]
    asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint4 v = *reinterpret_cast<const uint4*>(mine + i * 64);
      w[i][0] = v.x; w[i][1] = v.y; w[i][2] = v.z; w[i][3] = v.w;
    }
    if (j0 + kColWarps * 32 < c1) fetch(j + kColWarps * 32);
    uint32_t m[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      m[p] = w[0][p];
#pragma unroll
      for (int i = 1; i < 16; ++i) m[p] = larger2(m[p], w[i][p]);
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) m[p] = larger2(m[p], __shfl_xor_sync(kFull, m[p], o));
      m[p] &= kAbs2;
    }
    // this lane's column of the 32: the rg-th of its eight
    uint32_t t = rg & 4 ? (rg & 2 ? m[3] : m[2]) : (rg & 2 ? m[1] : m[0]);
    t = rg & 1 ? t >> 16 : t & 0xffffu;
    if (t >= 0x7f80u && j < c1) raise_flag(a.err, kErrNonfinite);
    const Scale sc = scale_of(bf16_bits_to_f32(t));
    if (j < c1) a.scale[b * a.c + j + rg] = sc.scale;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const float f0 = __shfl_sync(kFull, sc.inv, (2 * p) * 4 + q), f1 = __shfl_sync(kFull, sc.inv, (2 * p + 1) * 4 + q);
      uint32_t lo[4], hi[4];
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        lo[g] = code4(bf16_lo(w[4 * g][p]) * f0, bf16_lo(w[4 * g + 1][p]) * f0, bf16_lo(w[4 * g + 2][p]) * f0, bf16_lo(w[4 * g + 3][p]) * f0);
        hi[g] = code4(bf16_hi(w[4 * g][p]) * f1, bf16_hi(w[4 * g + 1][p]) * f1, bf16_hi(w[4 * g + 2][p]) * f1, bf16_hi(w[4 * g + 3][p]) * f1);
      }
      if (j < c1) {
        uint8_t* out = a.q + (j + 2 * p) * pitch + b * kExpertBlock + rg * 16;
        *reinterpret_cast<uint4*>(out) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        *reinterpret_cast<uint4*>(out + pitch) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      }
    }
  }
}

// ---- blocks of 128 x 128.  A block of 256 threads takes one, a thread eight
// rows x eight columns.  128 matrices of 2,048 x 4,096 with their transposes: 887 us from fp32,
// 630 from bf16, 727 and 458 without, none longer than the bytes take at the copy rate.
template <bool F32>
__global__ void __launch_bounds__(256)
    quant_blocks_kernel(const void* __restrict__ w, int n, int d, uint8_t* __restrict__ q, float* __restrict__ scale,
                        uint8_t* __restrict__ q_t, float* __restrict__ scale_t, int32_t* err) {
  __shared__ uint32_t tops[8];
  __shared__ uint32_t tile[128][33];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cg = threadIdx.x & 15, rg = threadIdx.x >> 4;
  const int jb = blockIdx.x, ib = blockIdx.y, e = blockIdx.z, nb = (n + 127) / 128, db = (d + 127) / 128;
  const int j = jb * 128 + cg * 8, i0 = ib * 128 + rg * 8;
  const int64_t base = static_cast<int64_t>(e) * n * d;
  griddep_wait();
  float v[8][8];
  uint32_t m = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const bool there = i0 + i < n && j < d;
    const int64_t at = base + static_cast<int64_t>(i0 + i) * d + j;
    if (F32) {
      uint4 x = make_uint4(0u, 0u, 0u, 0u), y = x;
      if (there) {
        const uint4* p = reinterpret_cast<const uint4*>(static_cast<const float*>(w) + at);
        x = __ldg(p);
        y = __ldg(p + 1);
      }
      const uint32_t u[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        m = max(m, u[k] & 0x7fffffffu);
        v[i][k] = __uint_as_float(u[k]);
      }
    } else {
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (there) x = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(w) + at));
      const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        m = max(m, max((u[k] << 16) & 0x7fffffffu, u[k] & 0x7fff0000u));
        v[i][2 * k] = bf16_lo(u[k]);
        v[i][2 * k + 1] = bf16_hi(u[k]);
      }
    }
  }
  m = __reduce_max_sync(kFull, m);
  if (lane == 0) tops[warp] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, tops[i]);
  if (m >= 0x7f800000u && threadIdx.x == 0) raise_flag(err, kErrNonfinite);
  const Scale sc = scale_of(__uint_as_float(m));
  if (threadIdx.x == 0) {
    scale[(static_cast<int64_t>(e) * nb + ib) * db + jb] = sc.scale;
    if (scale_t) scale_t[(static_cast<int64_t>(e) * db + jb) * nb + ib] = sc.scale;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[i][k] = __fmul_rn(v[i][k], sc.inv);
    if (i0 + i < n && j < d)
      *reinterpret_cast<uint2*>(q + base + static_cast<int64_t>(i0 + i) * d + j) =
          make_uint2(code4(v[i][0], v[i][1], v[i][2], v[i][3]), code4(v[i][4], v[i][5], v[i][6], v[i][7]));
  }
  if (!q_t) return;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    tile[cg * 8 + k][rg * 2] = code4(v[0][k], v[1][k], v[2][k], v[3][k]);
    tile[cg * 8 + k][rg * 2 + 1] = code4(v[4][k], v[5][k], v[6][k], v[7][k]);
  }
  __syncthreads();
  // a column of the block: 128 codes, 16 of them at least are there
  for (int col = warp; col < 128; col += 8)
    if (jb * 128 + col < d && ib * 128 + lane * 4 < n)
      reinterpret_cast<uint32_t*>(q_t + base + static_cast<int64_t>(jb * 128 + col) * n + ib * 128)[lane] = tile[col][lane];
}

int status_of(cudaError_t e) { return e == cudaSuccess ? kOk : kErrCuda; }

}  // namespace

int launch_quant_rows(const uint16_t* x, int64_t T, int d, const int32_t* slot, int K, uint8_t* q, float* scale, int32_t* err,
                      cudaStream_t s) {
  DeviceInfo di;
  if (int rc = device_info(&di)) return rc;
  const int strips = (d + 511) / 512;
  const int64_t blocks = (T * strips + kRowWarps - 1) / kRowWarps, most = static_cast<int64_t>(di.sm_count) * 64;
  const dim3 grid(static_cast<unsigned>(blocks < most ? blocks : most)), block(kRowWarps * 32);
  return status_of(slot ? launch_dependent(quant_rows_kernel<true>, grid, block, 0, s, x, T, d, strips, slot, K, q, scale, err)
                        : launch_dependent(quant_rows_kernel<false>, grid, block, 0, s, x, T, d, strips, slot, K, q, scale, err));
}

int launch_quant_cols(const QuantColsArgs& a, cudaStream_t s) {
  DeviceInfo di;
  if (int rc = device_info(&di)) return rc;
  // as many steps a block as leave every SM some blocks
  constexpr int kStep = kColWarps * 32;
  int steps = kColSteps;
  while (steps > 1 && a.P * ((a.c + steps * kStep - 1) / (steps * kStep)) < 16 * di.sm_count) steps /= 2;
  const int64_t grid = a.P * ((a.c + steps * kStep - 1) / (steps * kStep));
  if (grid > 0x7fffffff) return kErrUnsupported;
  if (!allow_smem(quant_cols_kernel, kColWarps * kColWarpBytes)) return kErrCuda;
  return status_of(launch_dependent(quant_cols_kernel, dim3(static_cast<unsigned>(grid)), dim3(kColWarps * 32),
                                    kColWarps * kColWarpBytes, s, a, steps));
}

int launch_quant_blocks(const void* w, int w_fp32, int E, int n, int d, uint8_t* q, float* scale, uint8_t* q_t, float* scale_t,
                        int32_t* err, cudaStream_t s) {
  const dim3 grid((d + 127) / 128, (n + 127) / 128, E);
  return status_of(w_fp32 ? launch_dependent(quant_blocks_kernel<true>, grid, dim3(256), 0, s, w, n, d, q, scale, q_t, scale_t, err)
                          : launch_dependent(quant_blocks_kernel<false>, grid, dim3(256), 0, s, w, n, d, q, scale, q_t, scale_t, err));
}

}  // namespace eqb
