// router_grad.cu -- the gradients of the router projection z = x W_r^T:
//   dx = dz W_r   [T,d] bf16,      dW = dz^T x   [E,d] fp32,
// on the tensor cores (tcgen05, fp32 accumulators in tensor memory).
//
// Both products are as large as the forward one (2 T d E flops beside T d
// bf16 values read or written): at E = 256 the tensor cores and the memory need
// about the same time, below that memory bounds them.  W_r, x and, for dW, dz
// are stored with the dimension that is summed over as the slow one, so they
// enter the MMAs as MN-major operands: a tile of 64 columns (one 128-byte
// swizzle atom) x R rows as TMA writes it, its 8-row groups 1 KiB apart, the
// next 64 columns one tile further.
//
// dx: a block keeps a slab of W_r (all E rows, N columns) in shared memory and
// runs over tiles of 128 tokens; dz streams through a ring of [128 x 64]
// stages, two accumulators alternate, and four warps round the accumulators to
// bf16 and turn them in shared memory, so that a store takes whole 128-byte lines
// (T = 32,768, d = 4,096, E = 128: 50 us; 62 with a row a lane, 32 bytes of 32
// rows a store; 63 by TMA from the same tiles).  Where dx is added to, a further
// warp loads the old values into a ring ahead, and they are turned in its stages.
// dW: a block has 128 experts x N columns of d and some of the tokens; dz and x
// stream through one ring, 64 tokens a stage, and x is read from memory once
// (above 128 experts two neighbouring blocks share it through L2).  The blocks'
// sums are added in order by a second kernel.
//
// Roles, bounded waits and the way out of a stall are those of the forward
// projection: warp 0 loads, warp 1 issues the MMAs, the others take the
// accumulators out.
#include "tcgen05.cuh"

namespace eqb {

namespace {

constexpr int kDxThreads = 224;    // two warps, four that take accumulators out, one that loads old values
constexpr int kGradThreads = 320;  // dW: two warps, eight that take accumulators out
// Blocks of a dW grid: one an SM of a GB300.  Fixed, so that the workspace's size can
// be asked for without a device; no block waits for another, so other counts only
// take longer.
constexpr int kGradCtas = 152;
constexpr uint32_t kTile64 = 64 * 128;    // bytes of 64 rows of 64 bf16
constexpr uint32_t kDxStage = 128 * 128;  // dx: 128 tokens x 64 experts of dz or columns of dx

// Shared-memory descriptor of an MN-major operand in 128-byte swizzled rows:
// `lead` bytes between tiles of 64 columns, 1 KiB between groups of 8 rows.
__device__ __forceinline__ uint64_t mn128_desc(uint32_t saddr, uint32_t lead) {
  uint64_t d = static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>(lead >> 4) << 16;
  d |= static_cast<uint64_t>(1024u >> 4) << 32;
  d |= static_cast<uint64_t>(1u) << 46;
  d |= static_cast<uint64_t>(2u) << 61;
  return d;
}
constexpr uint32_t kMnA = 1u << 15, kMnB = 1u << 16;  // instruction descriptor: A, B are MN-major

// 32 bytes a lane: one whole sector.
__device__ __forceinline__ void store_sector(void* p, const uint32_t (&w)[2][4]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0][0]), "r"(w[0][1]), "r"(w[0][2]),
               "r"(w[0][3]), "r"(w[1][0]), "r"(w[1][1]), "r"(w[1][2]), "r"(w[1][3])
               : "memory");
}
__device__ __forceinline__ void lds128(uint32_t at, uint32_t (&w)[4]) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
}

struct DxArgs {
  int T, d, E, N, slabs, ntiles;
  int S, SO;  // stages of dz, and of the output's old values (add)
  uint16_t* dx;
  int add;
  int32_t* err;
};

// dx of the items of block `block` of `blocks`.
__device__ __forceinline__ void dx_block(uint8_t* smem_raw, const CUtensorMap& tmz, const CUtensorMap& tmw,
                                         const CUtensorMap& tmi, const DxArgs& a, int block, int blocks) {
  const int S = a.S, SO = a.SO, E = a.E, KC = (E + 63) / 64;
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* sm = smem_raw + (base - raw);
  const uint32_t wtile = static_cast<uint32_t>(E) * 128u;  // bytes of W's E rows x 64 columns
  const uint32_t ring = base + wtile * static_cast<uint32_t>(a.N / 64);
  const uint32_t stag = ring + static_cast<uint32_t>(S) * kDxStage;
  const uint32_t bars = stag + static_cast<uint32_t>(SO) * kDxStage;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (S + s); };
  auto ofull = [&](int s) { return bars + 8u * (2 * S + s); };
  auto oempty = [&](int s) { return bars + 8u * (2 * S + SO + s); };
  const uint32_t rest = bars + 8u * (2 * S + 2 * SO);
  auto accf = [&](int b) { return rest + 8u * b; };
  auto acce = [&](int b) { return rest + 8u * (2 + b); };
  const uint32_t wfull = rest + 32u, wempty = rest + 40u, drain = rest + 48u;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(sm + (rest - base) + 56u);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  int* issued = reinterpret_cast<int*>(tmem_holder + 2);  // loads of dz, of W, of the output's old values
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), 1);
    }
    for (int s = 0; s < SO; ++s) {
      mbar_init(ofull(s), 1);
      mbar_init(oempty(s), 4);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(accf(b), 1);
      mbar_init(acce(b), 128);
    }
    mbar_init(wfull, 1);
    mbar_init(wempty, 1);
    mbar_init(drain, 1);
    *abort_flag = 0;
    issued[0] = issued[1] = issued[2] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  griddep_wait();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_holder;
  // items (slab, tile), slab-major; a block has a contiguous range of them.  (Blocks
  // that keep a slab and write the slabs of a row at the same time are as fast an
  // item, but leave SMs over: 63 us for 60 at d = 4,096 with the stores of that time.)
  const int64_t items = static_cast<int64_t>(a.slabs) * a.ntiles, i0 = items * block / blocks;
  const int64_t mine = items * (block + 1) / blocks - i0;
  const int sl0 = static_cast<int>(i0 / a.ntiles), tile0 = static_cast<int>(i0 % a.ntiles);
  // the item after (sl, tile); a division an item and role would take as long as its MMAs
  auto advance = [&](int& sl, int& tile) {
    if (++tile == a.ntiles) {
      tile = 0;
      ++sl;
    }
  };

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0, n = 0, nw = 0, slab = -1, sl = sl0, tile = tile0;
      uint32_t phase = 0;
      bool ok = true;
      for (int64_t i = 0; i < mine && ok; ++i, advance(sl, tile)) {
        if (sl != slab) {
          slab = sl;
          if (!mbar_wait(wempty, (static_cast<uint32_t>(nw) & 1u) ^ 1u, abort_flag)) break;
          const int chunks = min(a.N, a.d - sl * a.N) / 64;
          mbar_expect_tx(wfull, wtile * static_cast<uint32_t>(chunks));
          for (int c = 0; c < chunks; ++c)
            tma_load_2d(base + wtile * static_cast<uint32_t>(c), &tmw, wfull, sl * a.N + c * 64, 0);
          ++nw;
        }
        for (int kc = 0; kc < KC; ++kc, ++n) {
          if (!mbar_wait(empty(stage), phase ^ 1u, abort_flag)) { ok = false; break; }
          mbar_expect_tx(full(stage), kDxStage);
          tma_load_2d(ring + static_cast<uint32_t>(stage) * kDxStage, &tmz, full(stage), kc * 64, tile * kBM);
          if (++stage == S) { stage = 0; phase ^= 1u; }
        }
      }
      issued[0] = n;
      issued[1] = nw;
    }
  } else if (warp == 6) {
    if (lane == 0 && a.add) {  // the output's old values, as far ahead as its ring goes
      int stage = 0, n = 0, sl = sl0, tile = tile0;
      uint32_t phase = 0;
      bool ok = true;
      for (int64_t i = 0; i < mine && ok; ++i, advance(sl, tile)) {
        const int chunks = min(a.N, a.d - sl * a.N) / 64;
        for (int c = 0; c < chunks; ++c, ++n) {
          if (!mbar_wait(oempty(stage), phase ^ 1u, abort_flag)) { ok = false; break; }
          mbar_expect_tx(ofull(stage), kDxStage);
          tma_load_2d(stag + static_cast<uint32_t>(stage) * kDxStage, &tmi, ofull(stage), sl * a.N + c * 64, tile * kBM);
          if (++stage == SO) { stage = 0; phase ^= 1u; }
        }
      }
      issued[2] = n;
    }
  } else if (warp == 1) {
    if (lane == 0) {
      int stage = 0, nw = 0, slab = -1, it = 0, sl = sl0, tile = tile0;
      uint32_t phase = 0, idesc = 0;
      bool ok = true;
      for (int64_t i = 0; i < mine && ok; ++i, ++it, advance(sl, tile)) {
        if (sl != slab) {
          if (slab >= 0) umma_commit(wempty);  // the slab may be replaced once its MMAs are done
          slab = sl;
          if (!mbar_wait(wfull, static_cast<uint32_t>(nw) & 1u, abort_flag)) break;
          tc_fence_after();
          ++nw;
          idesc = umma_idesc_bf16(kBM, min(a.N, a.d - sl * a.N)) | kMnB;
        }
        const int buf = it & 1;
        if (!mbar_wait(acce(buf), (static_cast<uint32_t>(it >> 1) & 1u) ^ 1u, abort_flag)) break;
        tc_fence_after();
        const uint32_t dt = tmem + static_cast<uint32_t>(buf * 256);
        for (int kc = 0; kc < KC; ++kc) {
          if (!mbar_wait(full(stage), phase, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint64_t ad = sw128_desc(ring + static_cast<uint32_t>(stage) * kDxStage);
          const int steps = min(4, (E - kc * 64) / 16);
          for (int kk = 0; kk < steps; ++kk)
            umma_bf16(dt, ad + 2u * kk, mn128_desc(base + static_cast<uint32_t>(kc * 64 + kk * 16) * 128u, wtile), idesc,
                      (kc | kk) != 0 ? 1u : 0u);
          umma_commit(empty(stage));
          if (++stage == S) { stage = 0; phase ^= 1u; }
        }
        if (!ok) break;
        umma_commit(accf(buf));
      }
      umma_commit(drain);
      for (uint32_t i = 0; i < kSpinLimit; ++i)
        if (mbar_try_wait(drain, 0u)) break;
    }
  } else if (warp < 6) {
    const int q = warp & 3;
    const uint32_t lane_base = static_cast<uint32_t>(q * 32) << 16;
    const uint32_t swz = static_cast<uint32_t>(lane & 7);
    int it = 0, stage = 0;
    int sl = sl0, tile = tile0;
    uint32_t phase = 0;
    bool ok = true;
    for (int64_t i = 0; i < mine && ok; ++i, ++it, advance(sl, tile)) {
      const int chunks = min(a.N, a.d - sl * a.N) / 64;
      // a store takes 128-byte lines of eight rows, four lanes a line
      const int row = tile * kBM + q * 32 + (lane >> 2);
      uint16_t* out = a.dx + static_cast<int64_t>(row) * a.d + sl * a.N + (lane & 3) * 16;
      const int buf = it & 1;
      ok = __all_sync(0xffffffffu, mbar_wait(accf(buf), static_cast<uint32_t>(it >> 1) & 1u, abort_flag));
      if (!ok) break;
      tc_fence_after();
      for (int c = 0; c < chunks; ++c) {
        if (a.add) {
          ok = __all_sync(0xffffffffu, mbar_wait(ofull(stage), phase, abort_flag));
          if (!ok) break;
        }
        // the warp's 32 rows x 64 columns, swizzled: the old values' stage, or the one stage without them
        const uint32_t tile64 = stag + static_cast<uint32_t>(stage) * kDxStage + static_cast<uint32_t>(q * 32) * 128u;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t r[32];
          tmem_ld32(tmem + lane_base + static_cast<uint32_t>(buf * 256 + c * 64 + half * 32), r);
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const uint32_t at = tile64 + static_cast<uint32_t>(lane) * 128u + ((static_cast<uint32_t>(4 * half + v) ^ swz) << 4);
            if (a.add) {
              uint32_t w[4];
              lds128(at, w);
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                r[8 * v + 2 * k] = __float_as_uint(__uint_as_float(r[8 * v + 2 * k]) + bf16_lo(w[k]));
                r[8 * v + 2 * k + 1] = __float_as_uint(__uint_as_float(r[8 * v + 2 * k + 1]) + bf16_hi(w[k]));
              }
            }
            uint32_t p[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
              p[k] = pack_bf16x2_rn(__uint_as_float(r[8 * v + 2 * k]), __uint_as_float(r[8 * v + 2 * k + 1]));
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(p[0]), "r"(p[1]), "r"(p[2]), "r"(p[3])
                         : "memory");
          }
        }
        if (c == chunks - 1) {  // the accumulator is read
          tc_fence_before();
          mbar_arrive(acce(buf));
        }
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t rr = static_cast<uint32_t>(8 * k + (lane >> 2)), c2 = static_cast<uint32_t>(2 * (lane & 3));
          uint32_t w[2][4];
          lds128(tile64 + rr * 128u + ((c2 ^ (rr & 7u)) << 4), w[0]);
          lds128(tile64 + rr * 128u + (((c2 + 1u) ^ (rr & 7u)) << 4), w[1]);
          if (row + 8 * k < a.T) store_sector(out + static_cast<int64_t>(8 * k) * a.d + c * 64, w);
        }
        // the stage was written here by ordinary stores and is refilled by TMA:
        // every lane orders its own before the arrival that frees the stage
        if (a.add) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();  // the stage is read
        if (a.add) {
          if (lane == 0) mbar_arrive(oempty(stage));
          if (++stage == SO) { stage = 0; phase ^= 1u; }
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
    drain_loads(issued[0], S, full);
    drain_loads(issued[1], 1, [&](int) { return wfull; });
    drain_loads(issued[2], SO, ofull);
    raise_flag(a.err, kErrCuda);
  }
}

// dW's accumulators.  The tensor cores cut their fp32 sums off instead of
// rounding them, which draws every sum toward zero: 1.0e-9 of it a token (d =
// 38,912, E = 128, one sum over 512, 4,096 and 16,384 tokens: off by 4.7e-7,
// 4.4e-6 and 1.9e-5; the same sums rounded to nearest by 1.6e-7 to 1.5e-6).  So
// 512 tokens are summed in tensor memory at a time, in two accumulators that
// alternate, and eight warps add each to the sums that they hold in registers
// (128 a thread, which bounds a block to 128 experts x 256 columns).
constexpr int kDwStages = 8;      // stages of 64 tokens between two of these additions

// dW is cut into cols tiles of N columns (and two groups of experts above 128),
// each over `stages` stages of 64 tokens.  The blocks of a group take equal,
// contiguous shares of the cols x stages, so that any number of blocks is as
// good; block c of a group adds what it has of tile t to row c + t of `part`,
// which no other pair of the two has, and a second kernel adds up the rows of a
// tile in order.  With a block for every tile (direct) it is dW that they write.
struct DwArgs {
  int T, d, E, N, cols, groups, share, S;  // share: blocks of a group
  int64_t stages;  // of 64 tokens, in all
  float* out;      // dW, or part: rows of groups x [N / 4, 128] x 4 sums
  int direct, add;
  int32_t* err;
};

// The sums of block `block`: its share of a group's tiles and stages.
__device__ __forceinline__ void dw_block(uint8_t* smem_raw, const CUtensorMap& tmz, const CUtensorMap& tmx, const DwArgs& a,
                                         int block) {
  const int S = a.S;
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* sm = smem_raw + (base - raw);
  constexpr uint32_t a_bytes = 2u * kTile64;
  const uint32_t stage_bytes = a_bytes + static_cast<uint32_t>(a.N / 64) * kTile64;
  const uint32_t bars = base + static_cast<uint32_t>(S) * stage_bytes;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (S + s); };
  auto accf = [&](int b) { return bars + 8u * (2 * S + b); };
  auto acce = [&](int b) { return bars + 8u * (2 * S + 2 + b); };
  const uint32_t drain = bars + 8u * (2 * S + 4);
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(sm + (bars - base) + 8u * (2 * S + 5));
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  int* issued = reinterpret_cast<int*>(tmem_holder + 2);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(accf(b), 1);
      mbar_init(acce(b), 256);
    }
    mbar_init(drain, 1);
    *abort_flag = 0;
    *issued = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  griddep_wait();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_holder;
  // neighbours share x where there are two groups of experts
  const int eg = a.groups == 2 ? block & 1 : 0, b = a.groups == 2 ? block >> 1 : block, e0 = eg * 128;
  // with whole parts of every tile, neighbours take the same tokens of different tiles
  const int parts = a.share / a.cols, c = parts * a.cols == a.share ? b % a.cols * parts + b / a.cols : b;
  const int64_t total = a.stages * a.cols, u0 = total * c / a.share, u1 = total * (c + 1) / a.share;
  const int col0 = static_cast<int>(u0 / a.stages);
  const int64_t first0 = u0 - col0 * a.stages;
  // tile `col` from its stage `first` on: `ns` stages, as far as the tile and the share go
  auto stages_of = [&](int col, int64_t first) {
    return static_cast<int>(min(a.stages, u1 - static_cast<int64_t>(col) * a.stages) - first);
  };

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0, n = 0, col = col0;
      int64_t first = first0;
      uint32_t phase = 0;
      bool ok = true;
      for (int ns; ok && (ns = stages_of(col, first)) > 0; ++col, first = 0) {
        const int j0 = col * a.N, nn = min(a.N, a.d - j0);
        const uint32_t bytes = a_bytes + static_cast<uint32_t>(nn / 64) * kTile64;
        for (int k = 0; k < ns; ++k, ++n) {
          if (!mbar_wait(empty(stage), phase ^ 1u, abort_flag)) { ok = false; break; }
          const uint32_t dst = base + static_cast<uint32_t>(stage) * stage_bytes;
          const int t = static_cast<int>((first + k) * 64);
          mbar_expect_tx(full(stage), bytes);
          // experts past E (and tokens past T) are filled with zeros
          for (int i = 0; i < 2; ++i) tma_load_2d(dst + static_cast<uint32_t>(i) * kTile64, &tmz, full(stage), e0 + i * 64, t);
          for (int i = 0; i < nn / 64; ++i)
            tma_load_2d(dst + a_bytes + static_cast<uint32_t>(i) * kTile64, &tmx, full(stage), j0 + i * 64, t);
          if (++stage == S) { stage = 0; phase ^= 1u; }
        }
      }
      *issued = n;
    }
  } else if (warp == 1) {
    if (lane == 0) {
      int stage = 0, col = col0, chunk = 0;
      int64_t first = first0;
      uint32_t phase = 0;
      bool ok = true;
      for (int ns; ok && (ns = stages_of(col, first)) > 0; ++col, first = 0) {
        const uint32_t idesc = umma_idesc_bf16(kBM, min(a.N, a.d - col * a.N)) | kMnA | kMnB;
        for (int k = 0; k < ns; ++k) {
          const int buf = chunk & 1;
          if (k % kDwStages == 0) {
            if (!mbar_wait(acce(buf), (static_cast<uint32_t>(chunk >> 1) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
            tc_fence_after();
          }
          if (!mbar_wait(full(stage), phase, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint32_t sa = base + static_cast<uint32_t>(stage) * stage_bytes;
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)  // 16 tokens per MMA
            umma_bf16(tmem + static_cast<uint32_t>(buf * 256), mn128_desc(sa + kk * 2048u, kTile64),
                      mn128_desc(sa + a_bytes + kk * 2048u, kTile64), idesc, k % kDwStages != 0 || kk > 0 ? 1u : 0u);
          umma_commit(empty(stage));
          if (k % kDwStages == kDwStages - 1 || k == ns - 1) {
            umma_commit(accf(buf));
            ++chunk;
          }
          if (++stage == S) { stage = 0; phase ^= 1u; }
        }
      }
      umma_commit(drain);
      for (uint32_t i = 0; i < kSpinLimit; ++i)
        if (mbar_try_wait(drain, 0u)) break;
    }
  } else {
    // warps 2..5 and 6..9 take the two halves of an accumulator's columns
    const int q = warp & 3, h = (warp - 2) >> 2, cw = a.N / 2, c0 = h * cw;
    const uint32_t mine = tmem + (static_cast<uint32_t>(q * 32) << 16) + static_cast<uint32_t>(c0);
    const int row = q * 32 + lane, e = e0 + row;
    int col = col0, chunk = 0;
    int64_t first = first0;
    bool ok = true;
    for (int ns; ok && (ns = stages_of(col, first)) > 0; ++col, first = 0) {
      float acc[4][32];
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int i = 0; i < 32; ++i) acc[g][i] = 0.f;
      for (int k = 0; k < ns; k += kDwStages, ++chunk) {
        const int buf = chunk & 1;
        ok = __all_sync(0xffffffffu, mbar_wait(accf(buf), static_cast<uint32_t>(chunk >> 1) & 1u, abort_flag));
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int g = 0; g < 4; ++g)
          if (g * 32 < cw) {
            uint32_t r[32];
            tmem_ld32(mine + static_cast<uint32_t>(buf * 256 + g * 32), r);
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[g][i] = __fadd_rn(acc[g][i], __uint_as_float(r[i]));
          }
        tc_fence_before();
        mbar_arrive(acce(buf));
      }
      if (!ok || e >= a.E) continue;
      const int nn = min(a.N, a.d - col * a.N);
      // in part the rows of four columns lie one after the other, so that a
      // warp's stores are whole lines
      float4* out = a.direct ? reinterpret_cast<float4*>(a.out + static_cast<size_t>(e) * a.d + col * a.N + c0)
                             : reinterpret_cast<float4*>(a.out) +
                                   ((static_cast<size_t>(c) + col) * a.groups + eg) * (a.N / 4) * 128 + (c0 / 4) * 128 + row;
      const int next = a.direct ? 1 : 128;
#pragma unroll
      for (int g = 0; g < 4; ++g)
        if (g * 32 < cw && c0 + g * 32 < nn) {
#pragma unroll
          for (int v = 0; v < 8; ++v) {
            float4 o = make_float4(acc[g][4 * v], acc[g][4 * v + 1], acc[g][4 * v + 2], acc[g][4 * v + 3]);
            float4* dst = out + (8 * g + v) * next;
            if (a.add) {
              const float4 w = *dst;
              o.x += w.x; o.y += w.y; o.z += w.z; o.w += w.w;
            }
            *dst = o;
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
    drain_loads(*issued, S, full);
    raise_flag(a.err, kErrCuda);
  }
}

__global__ void __launch_bounds__(kDxThreads, 1)
    router_dx_kernel(const __grid_constant__ CUtensorMap tmz, const __grid_constant__ CUtensorMap tmw,
                     const __grid_constant__ CUtensorMap tmi, DxArgs a) {
  extern __shared__ uint8_t smem_raw[];
  dx_block(smem_raw, tmz, tmw, tmi, a, static_cast<int>(blockIdx.x), static_cast<int>(gridDim.x));
}

__global__ void __launch_bounds__(kGradThreads, 1)
    router_dw_kernel(const __grid_constant__ CUtensorMap tmz, const __grid_constant__ CUtensorMap tmx, DwArgs a) {
  extern __shared__ uint8_t smem_raw[];
  dw_block(smem_raw, tmz, tmx, a, static_cast<int>(blockIdx.x));
}

// Both gradients in one launch, the first blocks dW's, the others dx's.
__global__ void __launch_bounds__(kGradThreads, 1)
    router_dxdw_kernel(const __grid_constant__ CUtensorMap tmz, const __grid_constant__ CUtensorMap tmw,
                       const __grid_constant__ CUtensorMap tmi, const __grid_constant__ CUtensorMap tmz64, const __grid_constant__ CUtensorMap tmx, DxArgs a,
                       DwArgs w) {
  extern __shared__ uint8_t smem_raw[];
  const int block = static_cast<int>(blockIdx.x);
  const int nw = w.share * w.groups;
  if (block < nw) dw_block(smem_raw, tmz64, tmx, w, block);
  else dx_block(smem_raw, tmz, tmw, tmi, a, block - nw, static_cast<int>(gridDim.x) - nw);
}

// dW (+)= the rows of part that belong to each tile, in ascending order: four
// columns of an expert a thread.
__global__ void __launch_bounds__(256) router_dw_sum_kernel(const float4* part, DwArgs a, float* dW) {
  const int quads = a.N / 4 * 128;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int tile = static_cast<int>(i / quads), at = static_cast<int>(i % quads);  // at = column / 4 * 128 + row
  const int col = tile / a.groups, eg = tile % a.groups, e = eg * 128 + (at & 127), j = col * a.N + (at >> 7) * 4;
  const int64_t total = a.stages * a.cols, x0 = a.stages * col, x1 = x0 + a.stages - 1;
  // the blocks that hold the tile's first and last stages
  const int first = static_cast<int>(((x0 + 1) * a.share - 1) / total), last = static_cast<int>(((x1 + 1) * a.share - 1) / total);
  griddep_wait();
  if (col >= a.cols || e >= a.E || j >= a.d) return;
  const float4* p = part + (static_cast<size_t>(first + col) * a.groups + eg) * quads + at;
  const size_t row = static_cast<size_t>(a.groups) * quads;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int c = first; c <= last; ++c, p += row) {
    const float4 w = __ldcg(p);
    s.x += w.x; s.y += w.y; s.z += w.z; s.w += w.w;
  }
  float4* o = reinterpret_cast<float4*>(dW + static_cast<size_t>(e) * a.d + j);
  if (a.add) {
    const float4 w = *o;
    s.x += w.x; s.y += w.y; s.z += w.z; s.w += w.w;
  }
  *o = s;
}

__global__ void __launch_bounds__(256) zero_kernel(float* p, int64_t n) {
  griddep_wait();
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256)
    p[i] = 0.f;
}

struct DwPlan {
  int N, cols, groups, share;
  int64_t stages;
  bool direct;
};

// Up to this many tokens dW's tiles are narrow and take all tokens: a sum of
// parts would cost a launch.
constexpr int64_t kFewTokens = 1024;

// Both gradients share a launch, each on a part of the SMs, where dx is added to,
// and up to this many elements of x where it is written: of two launches each
// has its start and its end, and only the shared one reads and writes all along
// (T = 300, d = 1,024, E = 64 8.3 us for 11.5; 7,520, 1,792, 96 19 for 31; 60,000,
// 256, 64 26 for 50; 65,536, 4,096, 128 added to 255 for 280, without it 212 for 198).
constexpr int64_t kSharedElements = int64_t(1) << 27;

// The blocks of a group, of `most`: as many for every tile if that leaves no more
// than a tenth of them out.  Blocks that take the same tokens at the same time
// share dz on its way (T = 65,536, d = 4,096, E = 128 by two launches: 274 us with
// 144 of 152 for dW, 285 with all of them); an uneven share fills the SMs (T =
// 30,000, d = 1,024, E = 128, each on a part of them: 31 us for 38).
int even_share(int most, int cols) {
  const int even = most / cols * cols;
  return 10 * even >= 9 * most ? even : most;
}

// Columns of a dW tile and blocks of a group, at most one an SM: the widest tile
// that leaves most of the SMs a block with at least four stages; of few tokens
// the narrowest one that needs no more than a wave of blocks.
DwPlan plan_dw(int64_t T, int d, int E) {
  DwPlan p;
  p.groups = E > 128 ? 2 : 1;
  p.stages = (T + 63) / 64;
  p.direct = T <= kFewTokens;
  if (p.direct) {
    p.N = 64;
    while (p.N < 256 && (d + p.N - 1) / p.N * p.groups > kGradCtas) p.N *= 2;
    p.cols = p.share = (d + p.N - 1) / p.N;
    return p;
  }
  for (p.N = 256;; p.N /= 2) {
    p.cols = (d + p.N - 1) / p.N;
    const int64_t most = p.stages * p.cols / 4, sms = kGradCtas / p.groups;
    p.share = even_share(static_cast<int>(most < sms ? most : sms), p.cols);
    if (p.N == 64 || p.share * p.groups >= 120) break;
  }
  return p;
}
size_t part_bytes(const DwPlan& p) {
  return p.direct ? 0 : (static_cast<size_t>(p.share) + p.cols) * p.groups * p.N * 128 * 4;
}

struct DxLaunch {
  DxArgs a;
  CUtensorMap tmz, tmw, tmi;
  int smem;
  int64_t items;
};
// dx on up to `sms` blocks.
int plan_dx(const RouterGradArgs& g, const DeviceInfo& di, int sms, DxLaunch* l) {
  DxArgs& a = l->a;
  a = DxArgs{static_cast<int>(g.T), g.d, g.E, 256, 0, static_cast<int>((g.T + kBM - 1) / kBM), 0, 0, g.dx, g.add_dx, g.err};
  // narrower slabs while the tiles leave SMs without work
  for (;; a.N /= 2) {
    a.slabs = (g.d + a.N - 1) / a.N;
    if (a.N == 64 || static_cast<int64_t>(a.slabs) * a.ntiles >= sms) break;
  }
  // what W_r's slab leaves: a stage for the way out, with add_dx half of them for
  // the old values, the others for dz
  const int extra = 1024 + 8 * (4 * 8 + 7) + 20;
  const int wbytes = a.E * 128 * (a.N / 64);
  const int stages = (di.max_smem_optin - extra - wbytes) / static_cast<int>(kDxStage);
  a.SO = !g.add_dx ? 1 : stages / 2 < 8 ? stages / 2 : 8;
  a.S = stages - a.SO < 8 ? stages - a.SO : 8;
  if (a.S < 2) return kErrUnsupported;
  if (!make_map(&l->tmz, g.dz, static_cast<uint64_t>(g.T), static_cast<uint64_t>(g.E), kBM) ||
      !make_map(&l->tmw, g.W, static_cast<uint64_t>(g.E), static_cast<uint64_t>(g.d), static_cast<uint32_t>(g.E)) ||
      (g.add_dx && !make_map(&l->tmi, g.dx, static_cast<uint64_t>(g.T), static_cast<uint64_t>(g.d), kBM)))
    return kErrCuda;
  if (!g.add_dx) l->tmi = l->tmz;  // not used
  l->items = static_cast<int64_t>(a.slabs) * a.ntiles;
  l->smem = wbytes + (a.S + a.SO) * static_cast<int>(kDxStage) + extra;
  return kOk;
}

struct DwLaunch {
  DwArgs a;
  CUtensorMap tmz, tmx;
  int smem;
};
int plan_dw_launch(const RouterGradArgs& g, const DeviceInfo& di, const DwPlan& p, DwLaunch* l) {
  l->a = DwArgs{static_cast<int>(g.T), g.d, g.E, p.N, p.cols, p.groups, p.share, 0, p.stages, p.direct ? g.dW : g.part, p.direct,
                p.direct ? g.add_dW : 0, g.err};
  const int extra = 1024 + 8 * (2 * 8 + 5) + 16;
  const int stage_bytes = static_cast<int>(kTile64) * (2 + p.N / 64);
  l->a.S = (di.max_smem_optin - extra) / stage_bytes;
  if (l->a.S > 8) l->a.S = 8;
  if (l->a.S < 2) return kErrUnsupported;
  if (!make_map(&l->tmz, g.dz, static_cast<uint64_t>(g.T), static_cast<uint64_t>(g.E), 64) ||
      !make_map(&l->tmx, g.x, static_cast<uint64_t>(g.T), static_cast<uint64_t>(g.d), 64))
    return kErrCuda;
  l->smem = l->a.S * stage_bytes + extra;
  return kOk;
}

int status_of(cudaError_t e) { return e == cudaSuccess ? kOk : kErrCuda; }

}  // namespace

size_t router_grad_workspace(int64_t T, int d, int E) {
  return part_bytes(plan_dw(T, d, E));
}

int launch_router_grad(const RouterGradArgs& g, cudaStream_t s) {
  DeviceInfo di;
  if (int rc = device_info(&di)) return rc;
  const int64_t n = static_cast<int64_t>(g.E) * g.d;
  if (g.T == 0) {
    if (!g.dW || g.add_dW) return kOk;
    return status_of(launch_dependent(zero_kernel, dim3(static_cast<unsigned>((n + 1023) / 1024)), dim3(256), 0, s, g.dW, n));
  }
  DxLaunch x;
  DwLaunch w;
  DwPlan p = plan_dw(g.T, g.d, g.E);
  // SMs of dx where both share a launch.  What a tile of 128 tokens x 256 columns
  // takes an SM of either side beside the other one, from the split that is
  // fastest: 64 SMs of 152 for dW (E = 32 to 128, d = 512 to 4,096; some GPUs like 56
  // and others 72 a little better), 48 where dx is added to, 80 and 62 above 128
  // experts (T = 32,768, d = 4,096, E = 128 added to: 136 us with 48, 149 with 57,
  // 158 with 64; T = 65,536, d = 2,048, E = 64: 98 to 108 with 64, 100 to 120 with 80).
  int sms = di.sm_count;
  const bool one = g.dx && g.dW && (g.add_dx || g.T * g.d <= kSharedElements) &&
                   (!p.direct || 4 * p.cols * p.groups <= 3 * di.sm_count);
  if (one) {
    if (!p.direct) {
      const double dx = g.add_dx ? 4.33 : 2.75, dw = p.groups == 2 ? 3.0 : 2.0;
      const int want = static_cast<int>(di.sm_count * dw / (dx + dw) / p.groups + 0.5);
      if (p.share > want) p.share = even_share(want, p.cols);
    }
    sms = di.sm_count - p.share * p.groups;
  }
  // before the maps: encoding them needs a context, which a thread's first runtime call makes current
  if (one ? !allow_smem(router_dxdw_kernel, di.max_smem_optin)
          : (g.dx && !allow_smem(router_dx_kernel, di.max_smem_optin)) ||
                (g.dW && !allow_smem(router_dw_kernel, di.max_smem_optin)))
    return kErrCuda;
  if (g.dW)
    if (int rc = plan_dw_launch(g, di, p, &w)) return rc;
  if (g.dx)
    if (int rc = plan_dx(g, di, sms, &x)) return rc;
  const int nx = g.dx ? static_cast<int>(x.items < sms ? x.items : sms) : 0;
  if (one) {
    if (int rc = status_of(launch_dependent(router_dxdw_kernel, dim3(nx + p.share * p.groups), dim3(kGradThreads),
                                            x.smem > w.smem ? x.smem : w.smem, s, x.tmz, x.tmw, x.tmi, w.tmz, w.tmx, x.a,
                                            w.a)))
      return rc;
  } else if (g.dx) {
    if (int rc = status_of(launch_dependent(router_dx_kernel, dim3(nx), dim3(kDxThreads), x.smem, s, x.tmz, x.tmw, x.tmi,
                                            x.a)))
      return rc;
  }
  if (!g.dW) return kOk;
  if (!one)
    if (int rc = status_of(launch_dependent(router_dw_kernel, dim3(p.share * p.groups), dim3(kGradThreads), w.smem, s, w.tmz, w.tmx,
                                            w.a)))
      return rc;
  if (p.direct) return kOk;
  w.a.add = g.add_dW;
  const int64_t threads = static_cast<int64_t>(p.cols) * p.groups * (p.N / 4) * 128;
  return status_of(launch_dependent(router_dw_sum_kernel, dim3(static_cast<unsigned>((threads + 255) / 256)), dim3(256), 0, s,
                                    reinterpret_cast<const float4*>(g.part), w.a, g.dW));
}

}  // namespace eqb
