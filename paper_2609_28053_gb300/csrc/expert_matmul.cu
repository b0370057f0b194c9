// expert_matmul.cu -- the experts' products in 8 bits (e4m3 with an fp32 scale for
// each block of 128), on the tensor cores (tcgen05, kind::f8f6f4):
//   forward   out[r, j] = sum_B scale[r, B] w_scale[e, j / 128, B] (q_r . w_ej over block B)
//   weights   dW[e, i, j] = sum_B a_scale[B, i] b_scale[B, j] (a_i . b_j over block B of e's rows)
// Both operands lie K-major, so both are one kernel: tiles of 128 x BN of the
// output, 128 of K (one 128-byte swizzle atom) a stage.
//
// A scale belongs to 128 values of K, so the tensor cores' sums end with each
// stage: the accumulators of a stage (two of BN columns of tensor memory
// alternate) are read by eight warps, multiplied by the stage's scales and added to
// fp32 sums in registers.  That also keeps the tensor cores' own sums, which cut
// off instead of rounding, 128 products long.
//
// Roles, bounded waits and the way out of a stall are those of the router's
// projection: warp 0 loads, warp 1 issues the MMAs, the others take the
// accumulators out.  A block goes over tiles blockIdx.x, blockIdx.x + gridDim.x, ...;
// which expert and rows a tile has follows from `first`, read on the device.
#include "f32x2.cuh"
#include "tcgen05.cuh"

namespace eqb {

namespace {

// Warps 0 and 1 load and issue the MMAs (2 and 3 fill their warpgroup), 4 to 11
// take accumulators out.
constexpr int kMmThreads = 384;
// Registers a thread at the launch, and of both kinds of warpgroups after the
// split of the widest tiles (which keep 128 sums a thread): what the launch has.
constexpr int kMmRegs = 168, kMmFew = 72, kMmMany = 216;
static_assert(128 * kMmFew + 256 * kMmMany <= kMmThreads * kMmRegs, "more registers than the launch has");
constexpr uint32_t kATile = 128 * 128;  // bytes of A's part of a stage
constexpr int kMmWarps = 8;             // that take accumulators out

// Instruction descriptor, kind::f8f6f4: fp32 accumulator, A and B e4m3 (0), both K-major.
__host__ __device__ constexpr uint32_t umma_idesc_e4m3(int M, int N) {
  return (1u << 4) | ((static_cast<uint32_t>(N) >> 3) << 17) | ((static_cast<uint32_t>(M) >> 4) << 24);
}
__device__ __forceinline__ void umma_e4m3(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}
__device__ __forceinline__ void store_sector8(void* p, const uint32_t (&w)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
               "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

struct MmArgs {
  const float* a_scale;
  const float* b_scale;
  const int32_t* first;  // [E+1]: rows (forward) or blocks (weights)
  int64_t limit;         // rows of A, or blocks
  int E, n, k;           // columns of the output; forward: of K
  int rows;              // weights: rows of a tile's matrix
  int nt, mt;            // tiles along the columns; weights: along the rows
  int S;
  void* out;
  int out_fp32, add;
  int32_t* err;
};

// A tile: expert, first row, rows, first block of K and blocks of it.
struct Tile {
  int e, m, rows, n0, b0, kb;
};

__device__ __forceinline__ int64_t clamp64(int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; }

// Tile t; *e moves on to the tile's expert (tiles come in ascending order).
template <int BN, bool WG>
__device__ __forceinline__ Tile tile_of(const MmArgs& a, const int64_t* table, int64_t t, int* e) {
  Tile x;
  if (WG) {
    const int per = a.nt * a.mt;
    x.e = static_cast<int>(t / per);
    const int rest = static_cast<int>(t % per);
    x.m = rest / a.nt * kBM;
    x.n0 = rest % a.nt * BN;
    x.rows = min(kBM, a.rows - x.m);
    const int64_t lo = clamp64(__ldg(a.first + x.e), 0, a.limit), hi = clamp64(__ldg(a.first + x.e + 1), lo, a.limit);
    x.b0 = static_cast<int>(lo);
    x.kb = static_cast<int>(hi - lo);
  } else {
    const int64_t mt = t / a.nt;
    while (table[*e + 1] <= mt) ++*e;
    x.e = *e;
    x.n0 = static_cast<int>(t - mt * a.nt) * BN;
    const int64_t lo = clamp64(__ldg(a.first + x.e), 0, a.limit), hi = clamp64(__ldg(a.first + x.e + 1), lo, a.limit);
    const int64_t m = lo + (mt - table[x.e]) * kBM;
    x.m = static_cast<int>(m);
    x.rows = static_cast<int>(min(static_cast<int64_t>(kBM), hi - m));
    x.b0 = 0;
    x.kb = (a.k + 127) / 128;
  }
  return x;
}

template <int BN, bool WG>
__global__ void __launch_bounds__(kMmThreads, 1)
    expert_matmul_kernel(const __grid_constant__ CUtensorMap tma128, const __grid_constant__ CUtensorMap tma32,
                         const __grid_constant__ CUtensorMap tmb, const MmArgs a) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * 8 + 5];  // full, empty, accumulators full and empty, drain
  __shared__ uint32_t tmem_holder;
  __shared__ int abort_word, issued;
  __shared__ int64_t table[WG ? 1 : kMaxExperts + 1];  // tiles of 128 rows of the experts before
  __shared__ __align__(16) float bscale[WG ? kMmWarps : 1][2][WG ? BN / 2 : 1];
  constexpr uint32_t kStage = kATile + BN * 128u;
  constexpr int kCols = BN / 2;  // columns of a warp that takes accumulators out
  volatile int* abort_flag = &abort_word;
  const int S = a.S;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t bar0 = smem_u32(bars);
  auto full = [&](int s) { return bar0 + 8u * s; };
  auto empty = [&](int s) { return bar0 + 8u * (8 + s); };
  auto accf = [&](int b) { return bar0 + 8u * (16 + b); };
  auto acce = [&](int b) { return bar0 + 8u * (18 + b); };
  const uint32_t drain = bar0 + 8u * 20;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(accf(b), 1);
      mbar_init(acce(b), kMmWarps);
    }
    mbar_init(drain, 1);
    abort_word = 0;
    issued = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_holder)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  griddep_wait();
  int64_t total;
  if (WG) {
    total = static_cast<int64_t>(a.E) * a.nt * a.mt;
  } else {
    for (int e = threadIdx.x; e < a.E; e += kMmThreads) {
      const int64_t lo = clamp64(__ldg(a.first + e), 0, a.limit), hi = clamp64(__ldg(a.first + e + 1), lo, a.limit);
      table[e + 1] = (hi - lo + kBM - 1) / kBM;
    }
    __syncthreads();
    if (warp == 0) {
      int64_t run = 0;
      if (lane == 0) table[0] = 0;
      for (int e0 = 0; e0 < a.E; e0 += 32) {
        int64_t v = e0 + lane < a.E ? table[e0 + lane + 1] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int64_t y = __shfl_up_sync(kFull, v, o);
          if (lane >= o) v += y;
        }
        if (e0 + lane < a.E) table[e0 + lane + 1] = run + v;
        run += __shfl_sync(kFull, v, 31);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (!WG) total = table[a.E] * a.nt;
  const uint32_t tmem = tmem_holder;

  if (warp < 4) {
    if constexpr (BN == 256) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kMmFew));
    if (warp == 0 && lane == 0) {
      int stage = 0, n = 0, e = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int64_t t = blockIdx.x; t < total && ok; t += gridDim.x) {
        const Tile x = tile_of<BN, WG>(a, table, t, &e);
        // of a short tile only the groups of 32 rows that there are; what the others
        // of the stage hold goes into rows of the accumulator that nobody takes out
        const int parts = WG || x.rows > 96 ? 0 : (x.rows + 31) / 32;
        const uint32_t bytes = (parts ? static_cast<uint32_t>(parts) * (kATile / 4) : kATile) + BN * 128u;
        for (int i = 0; i < x.kb; ++i, ++n) {
          if (!mbar_wait(empty(stage), phase ^ 1u, abort_flag)) { ok = false; break; }
          const uint32_t dst = base + static_cast<uint32_t>(stage) * kStage;
          const int c = (x.b0 + i) * 128;
          mbar_expect_tx(full(stage), bytes);
          if (parts) {
            for (int p = 0; p < parts; ++p)
              tma_load_2d(dst + static_cast<uint32_t>(p) * (kATile / 4), &tma32, full(stage), c, x.m + p * 32);
          } else {
            tma_load_2d(dst, &tma128, full(stage), c, x.m);
          }
          tma_load_3d(dst + kATile, &tmb, full(stage), c, x.n0, WG ? 0 : x.e);
          if (++stage == S) { stage = 0; phase ^= 1u; }
        }
      }
      issued = n;
    } else if (warp == 1 && lane == 0) {
      constexpr uint32_t idesc = umma_idesc_e4m3(kBM, BN);
      int stage = 0, chunk = 0, e = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int64_t t = blockIdx.x; t < total && ok; t += gridDim.x) {
        const Tile x = tile_of<BN, WG>(a, table, t, &e);
        for (int i = 0; i < x.kb; ++i, ++chunk) {
          const int buf = chunk & 1;
          if (!mbar_wait(acce(buf), (static_cast<uint32_t>(chunk >> 1) & 1u) ^ 1u, abort_flag) ||
              !mbar_wait(full(stage), phase, abort_flag)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t sa = base + static_cast<uint32_t>(stage) * kStage;
          const uint64_t ad = sw128_desc(sa), bd = sw128_desc(sa + kATile);
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)  // 32 of K an MMA: 32 bytes
            umma_e4m3(tmem + static_cast<uint32_t>(buf * 256), ad + 2u * kk, bd + 2u * kk, idesc, kk > 0 ? 1u : 0u);
          umma_commit(empty(stage));
          umma_commit(accf(buf));
          if (++stage == S) { stage = 0; phase ^= 1u; }
        }
      }
      umma_commit(drain);
      for (uint32_t i = 0; i < kSpinLimit; ++i)
        if (mbar_try_wait(drain, 0u)) break;
    }
  } else {
    if constexpr (BN == 256) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kMmMany));
    // warps 4..7 and 8..11 take the two halves of an accumulator's columns
    const int q = warp & 3, h = (warp - 4) >> 2, w = warp - 4, c0 = h * kCols;
    const uint32_t mine = tmem + (static_cast<uint32_t>(q * 32) << 16) + static_cast<uint32_t>(c0);
    const int row = q * 32 + lane;
    int chunk = 0, e = 0;
    bool ok = true;
    for (int64_t t = blockIdx.x; t < total && ok; t += gridDim.x) {
      const Tile x = tile_of<BN, WG>(a, table, t, &e);
      const bool live = row < x.rows;
      const int col = x.n0 + c0;
      F2 acc[kCols / 2];
#pragma unroll
      for (int i = 0; i < kCols / 2; ++i) acc[i] = splat2(0.f);
      const float* sa = nullptr;
      const float* sb = nullptr;
      int64_t sa_step = 1;
      if (WG) {
        sa = a.a_scale + static_cast<int64_t>(x.b0) * a.rows + x.m + row;
        sa_step = a.rows;
        sb = a.b_scale + static_cast<int64_t>(x.b0) * a.n + col + lane * 4;
      } else {
        const int nb = (a.n + 127) / 128;
        sa = a.a_scale + static_cast<int64_t>(x.m + row) * x.kb;
        sb = a.b_scale + (static_cast<int64_t>(x.e) * nb + min(col / 128, nb - 1)) * x.kb;
      }
      const bool quad = WG && lane * 4 < kCols && col + lane * 4 < a.n;  // this lane has four of b's scales
      float na = live && x.kb > 0 ? __ldg(sa) : 0.f, nb1 = !WG && x.kb > 0 ? __ldg(sb) : 0.f;
      float4 nb4 = make_float4(0.f, 0.f, 0.f, 0.f);
      if (quad && x.kb > 0) nb4 = __ldg(reinterpret_cast<const float4*>(sb));
      for (int i = 0; i < x.kb; ++i, ++chunk) {
        const int buf = chunk & 1;
        const float f = WG ? na : na * nb1;
        if (WG) {
          if (lane * 4 < kCols) *reinterpret_cast<float4*>(&bscale[w][i & 1][lane * 4]) = nb4;
          __syncwarp();
        }
        if (i + 1 < x.kb) {  // the next stage's scales, on their way meanwhile
          if (live) na = __ldg(sa + (i + 1) * sa_step);
          if (WG) {
            if (quad) nb4 = __ldg(reinterpret_cast<const float4*>(sb + static_cast<int64_t>(i + 1) * a.n));
          } else {
            nb1 = __ldg(sb + i + 1);
          }
        }
        ok = __all_sync(kFull, mbar_wait(accf(buf), static_cast<uint32_t>(chunk >> 1) & 1u, abort_flag));
        if (!ok) break;
        tc_fence_after();
        if (q * 32 < x.rows) {
          const F2 ff = splat2(f);
#pragma unroll
          for (int g = 0; g < kCols / 32; ++g) {
            uint32_t r[32];
            tmem_ld32(mine + static_cast<uint32_t>(buf * 256 + g * 32), r);
#pragma unroll
            for (int v = 0; v < 16; ++v) {
              F2 d = f2(__uint_as_float(r[2 * v]), __uint_as_float(r[2 * v + 1]));
              if (WG) {
                const float2 s = *reinterpret_cast<const float2*>(&bscale[w][i & 1][g * 32 + 2 * v]);
                d = mul2(d, f2(s.x, s.y));
              }
              acc[g * 16 + v] = fma2(d, ff, acc[g * 16 + v]);
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(acce(buf));
      }
      if (!ok) break;
      if (!live) continue;
      const int64_t at = (WG ? static_cast<int64_t>(x.e) * a.rows + x.m + row : static_cast<int64_t>(x.m) + row) * a.n + col;
      if (!WG && !a.out_fp32) {
        uint16_t* o = static_cast<uint16_t*>(a.out) + at;
#pragma unroll
        for (int i = 0; i < kCols / 16; ++i)
          if (col + i * 16 < a.n) {
            uint32_t p[8];
#pragma unroll
            for (int v = 0; v < 8; ++v) p[v] = pack_bf16x2_rn(lo2(acc[i * 8 + v]), hi2(acc[i * 8 + v]));
            store_sector8(o + i * 16, p);
          }
      } else {
        float* o = static_cast<float*>(a.out) + at;
#pragma unroll
        for (int i = 0; i < kCols / 8; ++i)
          if (col + i * 8 < a.n) {
            uint32_t p[8];
            if (WG && a.add) {
              const float4 u = *reinterpret_cast<const float4*>(o + i * 8), v = *reinterpret_cast<const float4*>(o + i * 8 + 4);
              acc[i * 4] = add2(acc[i * 4], f2(u.x, u.y));
              acc[i * 4 + 1] = add2(acc[i * 4 + 1], f2(u.z, u.w));
              acc[i * 4 + 2] = add2(acc[i * 4 + 2], f2(v.x, v.y));
              acc[i * 4 + 3] = add2(acc[i * 4 + 3], f2(v.z, v.w));
            }
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              p[2 * v] = __float_as_uint(lo2(acc[i * 4 + v]));
              p[2 * v + 1] = __float_as_uint(hi2(acc[i * 4 + v]));
            }
            store_sector8(o + i * 8, p);
          }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
  if (threadIdx.x == 0 && *abort_flag) {
    drain_loads(issued, S, full);
    raise_flag(a.err, kErrCuda);
  }
}

__global__ void __launch_bounds__(256) zero_weights_kernel(float4* p, int64_t n) {
  griddep_wait();
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256)
    p[i] = make_float4(0.f, 0.f, 0.f, 0.f);
}

// Tensor map of [depth, rows, cols] bytes, box [1, box_rows, 128].
bool make_map8(CUtensorMap* m, const void* ptr, uint64_t depth, uint64_t rows, uint64_t cols, uint32_t box_rows, int dims) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t size[3] = {cols, rows, depth};
  const cuuint64_t strides[2] = {cols, cols * rows};
  const cuuint32_t box[3] = {128, box_rows, 1};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, static_cast<cuuint32_t>(dims), const_cast<void*>(ptr), size, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int BN, bool WG>
int launch_mm(const ExpertMatmulArgs& g, const DeviceInfo& di, cudaStream_t s) {
  constexpr int kStage = static_cast<int>(kATile) + BN * 128;
  constexpr int kStatic = 24 * 8 + 64 + (WG ? kMmWarps * BN * 4 : (kMaxExperts + 1) * 8) + 512;  // shared memory beside the stages
  MmArgs a;
  a.a_scale = g.a_scale;
  a.b_scale = g.b_scale;
  a.first = g.first;
  a.limit = g.R;
  a.E = g.E;
  a.rows = g.n;
  a.n = WG ? g.d : g.n;
  a.k = g.d;
  a.nt = (a.n + BN - 1) / BN;
  a.mt = (g.n + kBM - 1) / kBM;
  a.out = g.out;
  a.out_fp32 = g.out_fp32;
  a.add = g.add;
  a.err = g.err;
  const int room = di.max_smem_optin - kStatic - 1024;
  a.S = room / kStage < 8 ? room / kStage : 8;
  if (a.S < 2) return kErrUnsupported;
  // before the maps: encoding them needs a context, which a thread's first runtime call makes current
  if (BN == 256) {
    // the split of the registers waits for ever where the launch has fewer
    static std::atomic<int> checked{0};
    if (!checked.load(std::memory_order_relaxed)) {
      cudaFuncAttributes at;
      if (cudaFuncGetAttributes(&at, expert_matmul_kernel<BN, WG>) != cudaSuccess) return kErrCuda;
      if (at.numRegs < kMmRegs) return kErrUnsupported;
      checked.store(1, std::memory_order_relaxed);
    }
  }
  if (!allow_smem(expert_matmul_kernel<BN, WG>, 8 * kStage + 1024 < room + 1024 ? 8 * kStage + 1024 : room + 1024)) return kErrCuda;
  CUtensorMap t128, t32, tb;
  const uint64_t pitch = static_cast<uint64_t>(WG ? g.R * 128 : g.d);
  const uint64_t arows = static_cast<uint64_t>(WG ? g.n : g.R);
  if (!make_map8(&t128, g.a, 1, arows, pitch, 128, 2) || !make_map8(&t32, g.a, 1, arows, pitch, 32, 2) ||
      !make_map8(&tb, g.b, static_cast<uint64_t>(WG ? 1 : g.E), static_cast<uint64_t>(a.n), pitch, BN, 3))
    return kErrCuda;
  const int64_t most = WG ? static_cast<int64_t>(g.E) * a.nt * a.mt : (g.R / kBM + (g.R < g.E ? g.R : g.E)) * a.nt;
  const int grid = static_cast<int>(most < di.sm_count ? most : di.sm_count);
  return launch_dependent(expert_matmul_kernel<BN, WG>, dim3(grid), dim3(kMmThreads), a.S * kStage + 1024, s, t128, t32, tb, a) ==
                 cudaSuccess
             ? kOk
             : kErrCuda;
}

}  // namespace

int launch_expert_matmul(const ExpertMatmulArgs& g, cudaStream_t s) {
  DeviceInfo di;
  if (int rc = device_info(&di)) return rc;
  const int64_t mt = g.R / kBM + (g.R < g.E ? g.R : g.E);
  if (mt * ((g.n + 255) / 256) >= di.sm_count) return launch_mm<256, false>(g, di, s);
  return launch_mm<64, false>(g, di, s);
}

int launch_expert_wgrad(const ExpertMatmulArgs& g, cudaStream_t s) {
  DeviceInfo di;
  if (int rc = device_info(&di)) return rc;
  if (g.R == 0) {
    const int64_t n = static_cast<int64_t>(g.E) * g.n * g.d / 4;
    const int64_t blocks = (n + 255) / 256 < 4096 ? (n + 255) / 256 : 4096;
    return launch_dependent(zero_weights_kernel, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, s, static_cast<float4*>(g.out),
                            n) == cudaSuccess
               ? kOk
               : kErrCuda;
  }
  return launch_mm<256, true>(g, di, s);
}

}  // namespace eqb
