// quant.cu -- values in 8 bits (e4m3) with an fp32 scale for each block of 128:
//   scale = max |x| * fp32(1 / 448),   code = e4m3(x * fp32(1 / scale)),
// along a row (rows), along 128 rows (cols, turned), and over 128 x 128 (blocks).
//
// All three stream: two or four bytes a value in, one a copy out.  A block's values
// stay in registers between its maximum and its codes, so x is read once.  The
// maximum is taken of the patterns without their signs, as whole numbers: they
// order as the magnitudes do, and infinities and NaN come out on top, so that one
// comparison a block finds them.
#include "eqb_device.cuh"
#include "f32x2.cuh"

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
// Two codes, lo in the low byte.  The conversion rounds to nearest even and keeps
// what is above 448 there, so that the clamp is its own.
__device__ __forceinline__ uint32_t code2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t code4(float a, float b, float c, float d) { return code2(a, b) | code2(c, d) << 16; }

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
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = __vmaxu2(m, w[i] & kAbs2);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) m = __vmaxu2(m, __shfl_xor_sync(kFull, m, o));
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

// ---- cols.  A block of 256 threads takes 128 rows x kColStrips strips of 64
// columns, a thread four neighbouring rows x eight columns of each: four codes of a
// column are a word of the output's line, which is turned in shared memory.  The
// next strip's values are on their way while this one's are turned.  The grid goes
// over all rows of a group of strips first: a gathered row is wanted by K experts at
// different times, and kColStrips * 128 bytes of every token stay in L2 in between
// (T = 16,384, c = 4,096, K = 8 339 us, 444 with a row of blocks at a time).
constexpr int kColThreads = 256;
constexpr int kColStrips = 16;  // at most

__global__ void __launch_bounds__(kColThreads, 4) quant_cols_kernel(const QuantColsArgs a, int strips) {
  __shared__ uint32_t tops[8][32];  // of every warp: the largest patterns of 64 columns, two a word
  __shared__ __align__(16) float inv[64];
  __shared__ __align__(16) uint32_t tile[64 * 32];  // [column][word]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t b = blockIdx.x % a.P;
  const int cg = threadIdx.x & 7, rg = threadIdx.x >> 3;
  int j0 = static_cast<int>(blockIdx.x / a.P) * (strips * 64);
  const int j1 = min(j0 + strips * 64, a.c);
  griddep_wait();
  const int e = expert_of_block(a.blocks, a.E, b, lane);
  if (e >= a.E) return;
  const int64_t r0 = static_cast<int64_t>(__ldg(a.offsets + e)) + (b - __ldg(a.blocks + e)) * kExpertBlock;
  const int64_t r1 = min(static_cast<int64_t>(__ldg(a.offsets + e + 1)), a.R);
  const uint16_t* from[4];  // the thread's rows (null: zeros)
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    int64_t r = r0 + rg * 4 + i;
    bool there = r >= 0 && r < r1;
    if (there && a.entry) {
      const int n = __ldg(a.entry + r);
      there = n >= 0;
      r = static_cast<uint32_t>(n) / static_cast<uint32_t>(a.K);
    }
    from[i] = there && r < a.T ? a.x + r * a.c + cg * 8 : nullptr;
  }
  auto load = [&](int j, uint4 (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[i] = from[i] && j + cg * 8 < j1 ? __ldg(reinterpret_cast<const uint4*>(from[i] + j)) : make_uint4(0u, 0u, 0u, 0u);
  };
  const int64_t pitch = a.P * kExpertBlock;
  uint8_t* out = a.q + b * kExpertBlock + (lane & 7) * 16;
  uint4 next[4];
  load(j0, next);
  for (; j0 < j1; j0 += 64) {
    uint32_t w[4][4];  // [row][pair of columns]
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i][0] = next[i].x; w[i][1] = next[i].y; w[i][2] = next[i].z; w[i][3] = next[i].w;
    }
    load(j0 + 64, next);
    const int j = j0 + cg * 8;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      uint32_t m = __vmaxu2(__vmaxu2(w[0][p] & kAbs2, w[1][p] & kAbs2), __vmaxu2(w[2][p] & kAbs2, w[3][p] & kAbs2));
      m = __vmaxu2(m, __shfl_xor_sync(kFull, m, 8));
      m = __vmaxu2(m, __shfl_xor_sync(kFull, m, 16));
      if (lane < 8) tops[warp][cg * 4 + p] = m;
    }
    __syncthreads();
    if (threadIdx.x < 64) {  // a column's scale, once
      const int col = threadIdx.x;
      uint32_t t = tops[0][col >> 1];
#pragma unroll
      for (int v = 1; v < 8; ++v) t = __vmaxu2(t, tops[v][col >> 1]);
      t = col & 1 ? t >> 16 : t & 0xffffu;
      if (t >= 0x7f80u) raise_flag(a.err, kErrNonfinite);
      const Scale sc = scale_of(bf16_bits_to_f32(t));
      inv[col] = sc.inv;
      if (j0 + col < a.c) a.scale[b * a.c + j0 + col] = sc.scale;
    }
    __syncthreads();
    {
      // a word is four rows of a column; groups of four words are turned by the
      // column's eight, so that neither these stores nor the loads below meet in a bank
      const float4 x = *reinterpret_cast<const float4*>(inv + cg * 8), y = *reinterpret_cast<const float4*>(inv + cg * 8 + 4);
      const float f[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
      uint32_t* to = tile + cg * 256 + ((warp ^ cg) << 2) + (lane >> 3);
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const F2 f0 = splat2(f[2 * p]), f1 = splat2(f[2 * p + 1]);
        const F2 a0 = mul2(f2(bf16_lo(w[0][p]), bf16_lo(w[1][p])), f0), a1 = mul2(f2(bf16_lo(w[2][p]), bf16_lo(w[3][p])), f0);
        const F2 b0 = mul2(f2(bf16_hi(w[0][p]), bf16_hi(w[1][p])), f1), b1 = mul2(f2(bf16_hi(w[2][p]), bf16_hi(w[3][p])), f1);
        to[(2 * p) * 32] = code4(lo2(a0), hi2(a0), lo2(a1), hi2(a1));
        to[(2 * p + 1) * 32] = code4(lo2(b0), hi2(b0), lo2(b1), hi2(b1));
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int col = i * 32 + warp * 4 + (lane >> 3);
      if (j0 + col < a.c)
        *reinterpret_cast<uint4*>(out + (j0 + col) * pitch) = *reinterpret_cast<const uint4*>(tile + col * 32 + (((lane & 7) ^ (col >> 3)) << 2));
    }
  }
}

// ---- blocks of 128 x 128.  A block of 256 threads takes one, a thread eight
// rows x eight columns.
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
  // as many strips a block as leave every SM some blocks
  int strips = kColStrips;
  while (strips > 1 && a.P * ((a.c + strips * 64 - 1) / (strips * 64)) < 16 * di.sm_count) strips /= 2;
  const int64_t grid = a.P * ((a.c + strips * 64 - 1) / (strips * 64));
  if (grid > 0x7fffffff) return kErrUnsupported;
  return status_of(launch_dependent(quant_cols_kernel, dim3(static_cast<unsigned>(grid)), dim3(kColThreads), 0, s, a, strips));
}

int launch_quant_blocks(const void* w, int w_fp32, int E, int n, int d, uint8_t* q, float* scale, uint8_t* q_t, float* scale_t,
                        int32_t* err, cudaStream_t s) {
  const dim3 grid((d + 127) / 128, (n + 127) / 128, E);
  return status_of(w_fp32 ? launch_dependent(quant_blocks_kernel<true>, grid, dim3(256), 0, s, w, n, d, q, scale, q_t, scale_t, err)
                          : launch_dependent(quant_blocks_kernel<false>, grid, dim3(256), 0, s, w, n, d, q, scale, q_t, scale_t, err));
}

}  // namespace eqb
