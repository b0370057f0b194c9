// expert_matmul.cu -- the experts' products in 8 bits (e4m3 with an fp32 scale for
// each block of 128), on the tensor cores (tcgen05, kind::f8f6f4):
//   forward   out[r, j] = sum_B scale[r, B] w_scale[e, j / 128, B] (q_r . w_ej over block B)
//   weights   dW[e, i, j] = sum_B a_scale[B, i] b_scale[B, j] (a_i . b_j over block B of e's rows)
// Both operands lie K-major, so both are one kernel: tiles of the output, 128 of K
// (one 128-byte swizzle atom) a stage.
//
// A scale belongs to 128 values of K, so the tensor cores' sums end with each
// stage: the accumulators of a stage (BN columns of tensor memory, two to four of
// them in turn) are read by eight warps, multiplied by the stage's scales and added to
// fp32 sums in registers.  That also keeps the tensor cores' own sums, which cut
// off instead of rounding, 128 products long.
//
// What bounds it with many rows an expert is that way out.  R = 131,072, n = 2,048, d =
// 4,096, 128 experts: 897 us and 2.45 PFLOP/s where all have the same number of rows, 943
// where some have a multiple of others' (ten calls in a row; over seconds the power limit
// lowers the clock, and the second takes 1,040 to 1,090).  A stage takes an SM about 970
// clocks, of which its MMAs are 512: an accumulator goes round in 1,900, of which there
// are two.  By clock stamps: 330 from the last warp's release to the first MMA, 800 until
// the last is done and its barrier says so, 245 until the takers see it, 530 until
// their loads are done: a warp waits three times for tensor memory (about 130 clocks
// whatever it asked for), and beside 128 sums there are registers for 48 columns on
// their way (64 with 24 bytes spilled: 1,120 us).  Tiles 192 wide, whose 96 columns a warp
// come with one wait, took 1,140: a stage costs what it costs, and does less.  Polls
// that do not suspend, 975.  The scales count too: every scale fetched once, four
// stages at a time, took 947 us where each stage's own loads took 1,030.  Pairs of SMs
// (cta_group::2) take in less a stage and were slower: tiles of 256 x 256 with two
// accumulators 1,025 us, of 256 x 160 with three 1,195.
// Few rows an expert: the weights are what is read (256 rows in 109 of the 128 experts
// 138 us, 99% of the copy rate), and a tile of 128 rows needs no more of A than the
// groups of 32 rows that there are.  Where the tiles of 256 columns leave SMs without
// one, they are 64 wide (8 rows in 8 experts of 2,048 x 4,096: 16.8 us).
// Weights' gradient: a stage has a factor for each column beside the row's, one more
// multiplication a sum, and takes about 1,400 clocks; an expert's rows are few stages (R =
// 65,536 over 64 experts, n = 1,024, d = 2,048: eight and a half), so the sums' way to
// memory, 128 KB a tile, counts as well: 245 us where the output alone takes 79.  Whole lines
// instead of sectors a store (248 where sectors took 253) and the two halves of a
// tile as blocks of their own on one SM (282) did not change that.  Added to what is there
// it takes 776 us (190 by the bytes; where they go is not measured).  A tile's stages are one
// block's, so few tiles leave SMs idle: 131,072 rows, n = d = 64, 8 experts 88 us on 8 of them
// (2.5 by the bytes).
//
// Roles: warp 0 loads, warp 1 issues the MMAs, warps 2 and 3 bring the scales'
// products to shared memory (in the warps that need them they took the registers of
// their sums), the others take the accumulators out.  Every wait is bounded; after one
// that ran out the block waits for its loads in flight, frees its tensor memory and
// returns.  A block goes over tiles blockIdx.x, blockIdx.x + gridDim.x, ...; which
// expert and rows a tile has follows from `first`, read on the device.
#include "expert_mm.cuh"

namespace eqb {

namespace {

// Accumulators of BN columns: what tensor memory holds, at most four.  Few rows are a
// chain of stages, each of which waits for its MMAs, its way out and the next's
// barriers: with more stages in between they overlap.
constexpr int kMaxBufs = 4;
constexpr int mm_buffers(int BN) { return 512 / BN < kMaxBufs ? 512 / BN : kMaxBufs; }

template <int BN, bool WG>
__global__ void __launch_bounds__(kMmThreads, 1)
    expert_matmul_kernel(const __grid_constant__ CUtensorMap tma128, const __grid_constant__ CUtensorMap tma32,
                         const __grid_constant__ CUtensorMap tmb, const MmArgs a) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * 8 + 3 * kMaxBufs + 1];  // full, empty, accumulators full, empty and factors read, drain
  __shared__ uint32_t tmem_holder;
  __shared__ int abort_word, issued;
  __shared__ Table table;
  constexpr int kBufs = mm_buffers(BN);
  __shared__ __align__(16) Factors<BN, WG> ring[kBufs];
  constexpr uint32_t kStage = kATile + BN * 128u;
  constexpr int kCols = BN / 2;  // columns of a warp that takes accumulators out
  volatile int* abort_flag = &abort_word;
  const int S = a.S;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t bar0 = smem_u32(bars);
  auto full = [&](int s) { return bar0 + 8u * s; };
  auto empty = [&](int s) { return bar0 + 8u * (8 + s); };
  auto accf = [&](uint32_t b) { return bar0 + 8u * (16 + b); };
  auto acce = [&](uint32_t b) { return bar0 + 8u * (16 + kMaxBufs + b); };
  auto read = [&](uint32_t b) { return bar0 + 8u * (16 + 2 * kMaxBufs + b); };
  const uint32_t drain = bar0 + 8u * (16 + 3 * kMaxBufs);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), 1);
    }
    for (int b = 0; b < kBufs; ++b) {
      mbar_init(accf(b), 3);  // the MMAs, and both warps that bring factors
      mbar_init(read(b), kMmWarps);
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
  fill_table<kBM, WG>(a, table);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const int total = WG ? a.most : tiles_of(a, table);
  const int first = static_cast<int>(blockIdx.x), step = static_cast<int>(gridDim.x);
  const uint32_t tmem = tmem_holder;

  if (warp < 4) {
    if constexpr (BN == 256) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kMmFew));
    if (warp == 0 && lane == 0) {
      int stage = 0, n = 0, e = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int t = first; t < total && ok; t += step) {
        const Tile x = tile_of<kBM, BN, WG>(a, table, t, &e);
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
    } else if (warp == 1) {
      // The whole warp goes through the loop, so that addresses and descriptors are the
      // same for all lanes, and one lane issues.  The operands' barrier comes first: it
      // is there already when the accumulator's, which the chain hangs on, completes (the
      // other way round 1,073 us where this took 1,031)
      constexpr uint32_t idesc = umma_idesc_e4m3(kBM, BN);
      const uint32_t gone = smem_u32(&abort_word);
      const uint64_t ad0 = sw128_desc(base), bd0 = sw128_desc(base + kATile);
      int stage = 0, chunk = 0, e = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int t = first; t < total && ok; t += step) {
        const int kb = tile_of<kBM, BN, WG>(a, table, t, &e).kb;
        for (int i = 0; i < kb; ++i, ++chunk) {
          const uint32_t buf = static_cast<uint32_t>(chunk % kBufs), phase_acc = static_cast<uint32_t>(chunk / kBufs) & 1u;
          ok = mbar_wait_warp(full(stage), phase, gone) && mbar_wait_warp(acce(buf), phase_acc ^ 1u, gone);
          if (!ok) break;
          tc_fence_after();
          const uint64_t at = static_cast<uint64_t>(stage) * (kStage >> 4);
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)  // 32 of K an MMA: 32 bytes
              umma_e4m3(tmem + buf * BN, ad0 + at + 2u * kk, bd0 + at + 2u * kk, idesc, kk > 0 ? 1u : 0u);
            umma_commit(accf(buf));  // first: it is waited for (the other way round no slower than runs differ)
            umma_commit(empty(stage));
          }
          __syncwarp();
          if (++stage == S) { stage = 0; phase ^= 1u; }
        }
      }
      if (elect_one()) {
        umma_commit(drain);
        for (uint32_t i = 0; i < kSpinLimit; ++i)
          if (mbar_try_wait(drain, 0u)) break;
      }
      __syncwarp();
    } else if (warp >= 2) {
      int chunk = 0, e = 0;
      for (int t = first; t < total; t += step) {
        const Tile x = tile_of<kBM, BN, WG>(a, table, t, &e);
        if (!bring_factors<BN, WG, kBufs>(a, x, 0, warp - 2, lane, ring, &chunk, read, accf, smem_u32(&abort_word))) break;
      }
    }
  } else {
    if constexpr (BN == 256) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kMmMany));
    // warps 4..7 and 8..11 take the two halves of an accumulator's columns.  What a
    // tile is, is asked for again once its sums are complete: the sums and two loads take
    // 192 registers, and what is not kept meanwhile does not have to be spilled
    const int q = warp & 3, h = (warp - 4) >> 2;
    const uint32_t mine = tmem + (static_cast<uint32_t>(q * 32) << 16) + static_cast<uint32_t>(h * kCols);
    const int line = q * 32 + (WG ? lane >> 2 : lane), quad = WG ? 2 * (lane & 3) : 0;  // the thread's first row and column
    const uint32_t factor = smem_u32(&ring[0].row[WG || mm_blocks(BN) == 1 ? 0 : h][line]), gone = smem_u32(&abort_word);
    const uint32_t factor_col = smem_u32(&ring[0].col[WG ? h * kCols + quad : 0]);
    int chunk = 0, e = 0;
    bool ok = true;
    for (int t = first; t < total && ok; t += step) {
      F2 acc[kCols / 2];
#pragma unroll
      for (int i = 0; i < kCols / 2; ++i) acc[i] = splat2(0.f);
      int kb;
      bool some;  // of the warp's rows are there
      {
        const Tile x = tile_of<kBM, BN, WG>(a, table, t, &e);
        kb = x.kb;
        some = q * 32 < x.rows;
      }
      for (; kb > 0; --kb, ++chunk) {
        const uint32_t buf = static_cast<uint32_t>(chunk % kBufs), phase_acc = static_cast<uint32_t>(chunk / kBufs) & 1u;
        ok = mbar_wait_warp(accf(buf), phase_acc, gone);
        if (!ok) break;
        tc_fence_after();
        const uint32_t there = buf * static_cast<uint32_t>(sizeof(Factors<BN, WG>));
        float f[WG ? 4 : 1];
#pragma unroll
        for (int k = 0; k < (WG ? 4 : 1); ++k) f[k] = lds_f32(factor + there + 32u * k);
        auto release = [&]() {
          tc_fence_before();
          __syncwarp();
          mbar_arrive_one(acce(buf), read(buf), lane);
        };
        if (!some) release();
        else if constexpr (WG) add_stage_columns<kCols>(mine + buf * BN, f, factor_col + there, acc, release);
        else add_stage<kCols>(mine + buf * BN, f[0], acc, release);
      }
      if (!ok) break;
      const Tile x = tile_of<kBM, BN, WG>(a, table, t, &e);
      const int col = x.n0 + h * kCols + quad;
      if constexpr (WG) {  // nothing is added to an expert without blocks
        if (x.kb > 0 || !a.add) store_quads<kCols>(a, static_cast<int64_t>(x.e) * a.rows + x.m + line, x.rows - line, col, acc);
      } else if (line < x.rows) store_row<kCols>(a, static_cast<int64_t>(x.m) + line, col, acc);
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

template <int BN, bool WG>
int launch_mm(const ExpertMatmulArgs& g, const DeviceInfo& di, cudaStream_t s) {
  constexpr int kStage = static_cast<int>(kATile) + BN * 128;
  constexpr int kStatic = (17 + 3 * kMaxBufs) * 8 + 64 + sizeof(Table) + mm_buffers(BN) * sizeof(Factors<BN, WG>) + 512;  // shared memory beside the stages
  MmArgs a;
  if (!mm_args<kBM, BN, WG>(g, &a)) return kErrUnsupported;
  const int room = di.max_smem_optin - kStatic - 1024;
  a.S = room / kStage < 8 ? room / kStage : 8;
  if (a.S < 2) return kErrUnsupported;
  if (BN == 256) {
    static std::atomic<int> checked{0};
    if (int rc = check_registers(expert_matmul_kernel<BN, WG>, &checked)) return rc;
  }
  // before the maps: encoding them needs a context, which a thread's first runtime call makes current
  if (!allow_smem(expert_matmul_kernel<BN, WG>, 8 * kStage < room ? 8 * kStage + 1024 : room + 1024)) return kErrCuda;
  CUtensorMap t128, t32, tb;
  const uint64_t pitch = static_cast<uint64_t>(WG ? g.R * 128 : g.d), rows = static_cast<uint64_t>(WG ? g.n : g.R);
  if (!make_map8(&t128, g.a, 1, rows, pitch, 128, 2) || !make_map8(&t32, g.a, 1, rows, pitch, 32, 2) ||
      !make_map8(&tb, g.b, static_cast<uint64_t>(WG ? 1 : g.E), static_cast<uint64_t>(a.n), pitch, BN, 3))
    return kErrCuda;
  const int grid = a.most < di.sm_count ? a.most : di.sm_count;
  return launch_dependent(expert_matmul_kernel<BN, WG>, dim3(grid), dim3(kMmThreads), a.S * kStage + 1024, s, t128, t32, tb, a) ==
                 cudaSuccess
             ? kOk
             : kErrCuda;
}

}  // namespace

int launch_expert_matmul(const ExpertMatmulArgs& g, cudaStream_t s) {
  DeviceInfo di;
  if (int rc = device_info(&di)) return rc;
  const int64_t used = g.R < g.E ? g.R : g.E;  // experts that can have rows
  if ((g.R / kBM + used) * ((g.n + 255) / 256) >= di.sm_count) return launch_mm<256, false>(g, di, s);
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
