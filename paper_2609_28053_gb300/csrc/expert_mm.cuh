// expert_mm.cuh -- parts of the experts' products (expert_matmul.cu): tiles and whose
// they are, the instruction of 8-bit operands, the scales' way in, the way from
// tensor memory into the sums, and the tensor maps.
#pragma once

#include "f32x2.cuh"
#include "tcgen05.cuh"

namespace eqb {

namespace {

// Warps 0 and 1 load and issue the MMAs, 2 and 3 bring the scales, 4 to 11 take
// accumulators out.
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
  int most;              // tiles that there can be
  void* out;
  int out_fp32, add;
  int32_t* err;
};

// A tile: expert, first row, rows, first block of K and blocks of it.
struct Tile {
  int e, m, rows, n0, b0, kb;
};

// What the tiles of a call are, in shared memory: read from `first` once, so that a
// tile's start waits for no memory.
struct Table {
  int tiles[kMaxExperts + 1];  // forward: tiles of the experts before
  int lo[kMaxExperts], n[kMaxExperts];  // first row and rows, or blocks
  uint32_t order[kMaxExperts];  // weights: the tiles' experts, min(blocks, 2^22 - 1) and 1023 - expert
  int group[kMaxExperts / 32];
};

// Tile t; *e moves on to the tile's expert (tiles come in ascending order).
template <int BM, int BN, bool WG>
__device__ __forceinline__ Tile tile_of(const MmArgs& a, const Table& table, int t, int* e) {
  Tile x;
  if (WG) {
    const int per = a.nt * a.mt;
    const int i = t / per, rest = t - i * per, mt = rest / a.nt;
    x.e = kMaxExperts - 1 - static_cast<int>(table.order[i] % kMaxExperts);
    x.m = mt * BM;
    x.n0 = (rest - mt * a.nt) * BN;
    x.rows = min(BM, a.rows - x.m);
    x.b0 = table.lo[x.e];
    x.kb = table.n[x.e];
  } else {
    const int mt = t / a.nt;
    if (table.tiles[*e + 1] <= mt) {  // the first expert behind it whose tiles end after mt
      int lo = *e + 1, hi = a.E - 1;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (table.tiles[mid + 1] <= mt) lo = mid + 1;
        else hi = mid;
      }
      *e = lo;
    }
    x.e = *e;
    x.n0 = (t - mt * a.nt) * BN;
    const int first = (mt - table.tiles[x.e]) * BM;
    x.m = table.lo[x.e] + first;
    x.rows = min(BM, table.n[x.e] - first);
    x.b0 = 0;
    x.kb = (a.k + 127) / 128;
  }
  return x;
}

// Fills the table by the block's threads: `first` is kept within [0, limit] and in order
// whatever it says; tiles add up to at most 2^30.  Weights: the experts by falling
// number of blocks (then by number; a bitonic sort), so that what every SM gets, each 152nd
// tile, differs by no more than one tile's blocks.  R = 65,536 over 64 experts, n = 1,024, d =
// 2,048: 245 us, in the experts' order 253, with rows an expert whose logarithm deviates
// by 0.5 from its mean; by 1.5, 262 and 295.  Experts of few tiles keep their order:
// sorting takes 2 us of 128 experts and 8 of 1,024.  us sorted / in order, by 0.5 and by 1.5:
// 128 experts, 512 rows each on the mean, of 1 tile 18.5 / 16.2 and 51 / 49, of 4 38 / 35 and 67 /
// 60, of 8 54 / 54 and 82 / 84, of 16 95 / 93 and 118 / 129; 1,024 experts, 128 rows, of 1 tile 48 /
// 40 and 63 / 54, of 8 239 / 219 and 247 / 242; 64 experts, 2,048 rows, of 8 79 / 74 and 177 / 172.
constexpr int kOrderTiles = 8;
template <int BM, bool WG>
__device__ __forceinline__ void fill_table(const MmArgs& a, Table& table) {
  constexpr int kMost = 1 << 30;
  const int lane = threadIdx.x & 31, limit = static_cast<int>(a.limit);
  // running sums within 32 experts, then over the sums of the 32 groups
  for (int e0 = static_cast<int>(threadIdx.x) & ~31; e0 < a.E; e0 += blockDim.x) {
    const int e = e0 + lane;
    int v = 0;
    if (e < a.E) {
      const int lo = min(max(__ldg(a.first + e), 0), limit), n = min(max(__ldg(a.first + e + 1), lo), limit) - lo;
      table.lo[e] = lo;
      table.n[e] = n;
      v = (n + BM - 1) / BM;
    }
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(kFull, v, o);
      if (lane >= o) v = min(v + y, kMost);
    }
    if (e < a.E) table.tiles[e + 1] = v;
    if (lane == 31) table.group[e0 >> 5] = v;
  }
  if (WG) {
    int size = 1;
    while (size < a.E) size *= 2;
    for (int e = threadIdx.x; e < size; e += blockDim.x)
      table.order[e] = e < a.E ? static_cast<uint32_t>(min(table.n[e], (1 << 22) - 1)) * kMaxExperts + (kMaxExperts - 1 - e) : 0u;
    for (int run = 2; run <= size && a.nt * a.mt >= kOrderTiles; run *= 2)
      for (int apart = run / 2; apart; apart /= 2) {
        __syncthreads();
        for (int i = threadIdx.x; i < size / 2; i += blockDim.x) {
          const int lo = 2 * i - (i & (apart - 1)), hi = lo + apart;
          const uint32_t x = table.order[lo], y = table.order[hi];
          if (((lo & run) == 0) == (x < y)) {
            table.order[lo] = y;
            table.order[hi] = x;
          }
        }
      }
    return;
  }
  __syncthreads();
  if (threadIdx.x < 32) {
    if (lane == 0) table.tiles[0] = 0;
    const int own = lane * 32 < a.E ? table.group[lane] : 0;
    int v = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(kFull, v, o);
      if (lane >= o) v = min(v + y, kMost);
    }
    const int before = __shfl_up_sync(kFull, v, 1);
    __syncwarp();
    table.group[lane] = lane ? before : 0;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += blockDim.x) table.tiles[e + 1] = min(table.tiles[e + 1] + table.group[e >> 5], kMost);
}
// The tiles of a table.
__device__ __forceinline__ int tiles_of(const MmArgs& a, const Table& table) {
  const int64_t n = static_cast<int64_t>(table.tiles[a.E]) * a.nt;
  return n < a.most ? static_cast<int>(n) : a.most;
}

__device__ __forceinline__ float lds_f32(uint32_t at) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ F2 lds_f2(uint32_t at) {
  float x, y;
  asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(x), "=f"(y) : "r"(at) : "memory");
  return f2(x, y);
}

// 32 or 16 columns of the warp's lanes, on their way until tmem_wait has returned.
// The registers pass through it, or through tmem_here after it, so that no use of them
// moves before it; and the loads that come again into the same registers take
// their old values along, so that no use of those moves behind.
__device__ __forceinline__ void tmem_start(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_again(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
        "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),
        "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
        "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_start(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_again(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
        "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_wait(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                 "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]),
                 "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]),
                 "+r"(r[30]), "+r"(r[31])
               :
               : "memory");
}
__device__ __forceinline__ void tmem_here(uint32_t (&r)[16]) {
  asm volatile(""
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]));
}

// N columns of a stage, times f, added to the sums.
template <int N>
__device__ __forceinline__ void add_columns(const uint32_t (&r)[N], const F2& ff, F2* acc) {
#pragma unroll
  for (int v = 0; v < N / 2; ++v) acc[v] = fma2(f2(__uint_as_float(r[2 * v]), __uint_as_float(r[2 * v + 1])), ff, acc[v]);
}

// Takes kCols columns of the warp's lanes out of tensor memory and adds them to the
// sums; `release` runs as soon as the last of them are in registers.  A wait is for
// all loads on their way and takes about 130 cycles however much was asked for, so 48
// columns share one (64 do not fit in registers beside 128 sums).
template <int kCols, class Release>
__device__ __forceinline__ void add_stage(uint32_t taddr, float f, F2 (&acc)[kCols / 2], Release release) {
  static_assert(kCols == 32 || kCols == 128, "columns of a warp");
  const F2 ff = splat2(f);
  uint32_t r[32];
  tmem_start(taddr, r);
  if constexpr (kCols == 32) {
    tmem_wait(r);
    release();
    add_columns(r, ff, acc);
  } else {
    uint32_t s[16];
    tmem_start(taddr + 32u, s);
    tmem_wait(r);
    tmem_here(s);
    add_columns(r, ff, acc);
    tmem_again(taddr + 48u, r);
    add_columns(s, ff, acc + 16);
    tmem_again(taddr + 80u, s);
    tmem_wait(r);
    tmem_here(s);
    add_columns(r, ff, acc + 24);
    tmem_again(taddr + 96u, r);
    add_columns(s, ff, acc + 40);
    tmem_wait(r);
    release();
    add_columns(r, ff, acc + 48);
  }
}
// 32 columns of 16 lanes: of every 8 columns, a thread gets columns 2 (lane % 4) and the
// next of lanes lane / 4 and 8 further.
__device__ __forceinline__ void tmem_quads(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
        "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_wait(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
}
// The same where each column has a factor of its own.  A row a lane, every lane would
// need every column's factor, and 128 of them to each lane of eight warps are 1,024
// clocks of shared memory a stage; in quads of lanes a thread has four rows and a
// quarter of the columns.  acc[c / 8 * 4 + r]: columns c + 2 (lane % 4) and the next of
// row lane / 4 + 8 r; f: the rows' factors, cs: those of columns 2 (lane % 4) and on.
template <int kCols, class Release>
__device__ __forceinline__ void add_stage_columns(uint32_t taddr, const float (&f)[4], uint32_t cs, F2 (&acc)[kCols / 2], Release release) {
  uint32_t r[2][16];
#pragma unroll
  for (int i = 0; i < 16; ++i) r[0][i] = r[1][i] = 0u;
  tmem_quads(taddr, r[0]);
  tmem_quads(taddr + (16u << 16), r[1]);
#pragma unroll
  for (int c = 0; c < kCols; c += 32) {
    F2 p[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) p[g] = lds_f2(cs + static_cast<uint32_t>(c + 8 * g) * 4u);
    tmem_wait(r[0]);
    tmem_here(r[1]);
    if (c + 32 == kCols) release();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          F2& sum = acc[(c / 8 + g) * 4 + 2 * h + k];
          const F2 d = f2(__uint_as_float(r[h][4 * g + 2 * k]), __uint_as_float(r[h][4 * g + 2 * k + 1]));
          sum = fma2(mul2(d, p[g]), splat2(f[2 * h + k]), sum);
        }
      if (c + 32 < kCols) tmem_quads(taddr + (static_cast<uint32_t>(16 * h) << 16) + c + 32u, r[h]);
    }
  }
}

// Up to 64 polls of at most ~1 us for the phase of parity `parity`, in one loop of
// three instructions: where a step of the pipeline hangs on a phase that is there
// already, what follows the poll counts (with the poll, its limit and the abort word in
// one loop: 1,202 us for the product that takes 1,073 so; one lane polling for its
// warp: 2,150).
__device__ __forceinline__ uint32_t mbar_try64(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p, more;\n\t.reg .u32 left;\n\t"
      "mov.u32 left, 64;\n"
      "again_%=:\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
      "@p bra there_%=;\n\t"
      "sub.u32 left, left, 1;\n\t"
      "setp.ne.u32 more, left, 0;\n\t"
      "@more bra again_%=;\n"
      "there_%=:\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity), "r"(1000u)
      : "memory");
  return ok;
}
// Bounded wait of a whole warp, false when it ran out or another role aborted.  The
// abort word by its address in shared memory: it takes fewer registers.
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, uint32_t parity, uint32_t abort_word) {
  if (__all_sync(kFull, mbar_try64(bar, parity))) return true;
  for (uint32_t i = 0; i < kSpinLimit / 64; ++i) {
    int gone;
    asm volatile("ld.volatile.shared.s32 %0, [%1];" : "=r"(gone) : "r"(abort_word) : "memory");
    if (__any_sync(kFull, gone)) return false;
    if (__all_sync(kFull, mbar_try64(bar, parity))) return true;
  }
  asm volatile("st.volatile.shared.s32 [%0], %1;" ::"r"(abort_word), "r"(1) : "memory");
  return false;
}
// One lane of a whole warp, the same one every time.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(p));
  return p != 0;
}
// Lane 0 arrives at both: by predicate, so that the warp does not part and meet again
// in between.
__device__ __forceinline__ void mbar_arrive_one(uint32_t first, uint32_t second, int lane) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.eq.s32 p, %2, 0;\n\t"
      "@p mbarrier.arrive.shared::cta.b64 _, [%0];\n\t"
      "@p mbarrier.arrive.shared::cta.b64 _, [%1];\n\t}" ::"r"(first),
      "r"(second), "r"(lane)
      : "memory");
}
// The warp's lanes' sums, a row a lane, to its kCols columns of the output from
// `col` on, a whole sector a store.
template <int kCols>
__device__ __forceinline__ void store_row(const MmArgs& a, int64_t row, int col, F2 (&acc)[kCols / 2]) {
  const int64_t at = row * a.n + col;
  if (!a.out_fp32) {
    uint16_t* o = static_cast<uint16_t*>(a.out) + at;
#pragma unroll
    for (int i = 0; i < kCols / 16; ++i)
      if (col + i * 16 < a.n) {
        uint32_t p[8];
#pragma unroll
        for (int v = 0; v < 8; ++v) p[v] = pack_bf16x2_rn(lo2(acc[i * 8 + v]), hi2(acc[i * 8 + v]));
        store_sector8(o + i * 16, p);
      }
    return;
  }
  float* o = static_cast<float*>(a.out) + at;
#pragma unroll
  for (int i = 0; i < kCols / 8; ++i)
    if (col + i * 8 < a.n) {
      uint32_t p[8];
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        p[2 * v] = __float_as_uint(lo2(acc[i * 4 + v]));
        p[2 * v + 1] = __float_as_uint(hi2(acc[i * 4 + v]));
      }
      store_sector8(o + i * 8, p);
    }
}
// The same of sums in quads of lanes, `row` and `col` being the lane's first: a quad
// writes a sector.  `rows`: how many there are behind row.
template <int kCols>
__device__ __forceinline__ void store_quads(const MmArgs& a, int64_t row, int rows, int col, F2 (&acc)[kCols / 2]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (8 * k >= rows) break;
    float* o = static_cast<float*>(a.out) + (row + 8 * k) * a.n + col;
#pragma unroll
    for (int g = 0; g < kCols / 8; ++g)
      if (col + g * 8 < a.n) {
        F2 v = acc[g * 4 + k];
        float2* to = reinterpret_cast<float2*>(o + g * 8);
        if (a.add) {
          const float2 u = *to;
          v = add2(v, f2(u.x, u.y));
        }
        *to = make_float2(lo2(v), hi2(v));
      }
  }
}

// The factors of a stage, in shared memory.  Forward: of every row, both scales'
// product, for each of the blocks of 128 columns that a tile of BN touches.  Weights:
// of the rows, and of the columns.
constexpr int mm_blocks(int BN) { return BN > 128 ? BN / 128 : 1; }
template <int BN, bool WG>
struct Factors {
  float row[WG ? 1 : mm_blocks(BN)][kBM];
  float col[WG ? BN : 4];
};

// Warps 2 (h = 0) and 3 (h = 1): the factors of one tile's stages into `ring`, kBufs
// stages deep.  ring[buf] may be written once `freed(buf)` has a phase for it, and adds
// its arrival to what `ready(buf)` waits for.  False when a wait ran out.
template <int BN, bool WG, int kBufs, class Freed, class Ready>
__device__ __forceinline__ bool bring_factors(const MmArgs& a, const Tile& x, int row0, int h, int lane, Factors<BN, WG>* ring,
                                              int* chunk, Freed freed, Ready ready, uint32_t gone) {
  auto begin = [&](int* buf) {
    *buf = *chunk % kBufs;
    return mbar_wait_warp(freed(*buf), (static_cast<uint32_t>(*chunk / kBufs) & 1u) ^ 1u, gone);
  };
  auto end = [&](int buf) {
    __syncwarp();
    if (lane == 0) mbar_arrive(ready(buf));
    ++*chunk;
  };
  if constexpr (!WG) {
    // rows h * 64 + lane and 32 further, four stages of their scales at a time, the
    // next four on their way meanwhile; b's scales of four stages in lanes 4 j + i
    constexpr int kBlocks = mm_blocks(BN);
    const int nb = (a.n + 127) / 128, i4 = lane & 3;
    const float* pa[2];
    bool la[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int row = row0 + h * 64 + r * 32 + lane;
      la[r] = row < x.rows;
      pa[r] = a.a_scale + (static_cast<int64_t>(x.m) + row) * x.kb;
    }
    const float* pb = a.b_scale + (static_cast<int64_t>(x.e) * nb + min(x.n0 / 128 + (lane >> 2), nb - 1)) * x.kb + i4;
    const bool lb = lane < 4 * kBlocks, wide = (x.kb & 3) == 0 && (reinterpret_cast<uintptr_t>(a.a_scale) & 15u) == 0;
    float next[2][4] = {}, next_b = 0.f;
    auto fetch = [&](int k0) {
      if (k0 >= x.kb) return;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        if (!la[r]) continue;
        if (wide) {
          const float4 v = __ldg(reinterpret_cast<const float4*>(pa[r] + k0));
          next[r][0] = v.x; next[r][1] = v.y; next[r][2] = v.z; next[r][3] = v.w;
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (k0 + i < x.kb) next[r][i] = __ldg(pa[r] + k0 + i);
        }
      }
      if (lb && k0 + i4 < x.kb) next_b = __ldg(pb + k0);
    };
    fetch(0);
    for (int k0 = 0; k0 < x.kb; k0 += 4) {
      float va[2][4];
      const float vb = next_b;
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) va[r][i] = next[r][i];
      fetch(k0 + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (k0 + i >= x.kb) break;
        int buf;
        if (!begin(&buf)) return false;
#pragma unroll
        for (int j = 0; j < kBlocks; ++j) {
          const float b = __shfl_sync(kFull, vb, 4 * j + i);
#pragma unroll
          for (int r = 0; r < 2; ++r) ring[buf].row[j][h * 64 + r * 32 + lane] = va[r][i] * b;
        }
        end(buf);
      }
    }
  } else if (h == 0) {
    // rows lane, lane + 32, ... of a, two stages ahead
    const float* pa = a.a_scale + static_cast<int64_t>(x.b0) * a.rows + x.m + row0 + lane;
    float v[2][4] = {};
    auto fetch = [&](int i, int s) {
      if (i >= x.kb) return;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (row0 + k * 32 + lane < x.rows) v[s][k] = __ldg(pa + static_cast<int64_t>(i) * a.rows + k * 32);
    };
    fetch(0, 0);
    fetch(1, 1);
    for (int i0 = 0; i0 < x.kb; i0 += 2) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (i0 + s >= x.kb) break;
        int buf;
        if (!begin(&buf)) return false;
#pragma unroll
        for (int k = 0; k < 4; ++k) ring[buf].row[0][k * 32 + lane] = v[s][k];
        end(buf);
        fetch(i0 + s + 2, s);
      }
    }
  } else {
    // columns 4 lane .. 4 lane + 3 of b, and those 128 further, two stages ahead
    const float* pb = a.b_scale + static_cast<int64_t>(x.b0) * a.n + x.n0 + lane * 4;
    const bool l0 = x.n0 + lane * 4 < a.n && lane * 4 < BN, l1 = x.n0 + 128 + lane * 4 < a.n && 128 + lane * 4 < BN;
    float4 q0[2], q1[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) q0[s] = q1[s] = make_float4(0.f, 0.f, 0.f, 0.f);
    auto fetch = [&](int i, int s) {
      if (i >= x.kb) return;
      if (l0) q0[s] = __ldg(reinterpret_cast<const float4*>(pb + static_cast<int64_t>(i) * a.n));
      if (l1) q1[s] = __ldg(reinterpret_cast<const float4*>(pb + static_cast<int64_t>(i) * a.n + 128));
    };
    fetch(0, 0);
    fetch(1, 1);
    for (int i0 = 0; i0 < x.kb; i0 += 2) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (i0 + s >= x.kb) break;
        int buf;
        if (!begin(&buf)) return false;
        if (lane * 4 < BN) *reinterpret_cast<float4*>(ring[buf].col + lane * 4) = q0[s];
        if (128 + lane * 4 < BN) *reinterpret_cast<float4*>(ring[buf].col + 128 + lane * 4) = q1[s];
        end(buf);
        fetch(i0 + s + 2, s);
      }
    }
  }
  return true;
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

// false: more tiles than the kernels count (no output of that size fits a GPU).
template <int BM, int BN, bool WG>
bool mm_args(const ExpertMatmulArgs& g, MmArgs* out) {
  MmArgs& a = *out;
  a.a_scale = g.a_scale;
  a.b_scale = g.b_scale;
  a.first = g.first;
  a.limit = g.R;
  a.E = g.E;
  a.rows = g.n;
  a.n = WG ? g.d : g.n;
  a.k = g.d;
  a.nt = (a.n + BN - 1) / BN;
  a.mt = (g.n + BM - 1) / BM;
  a.S = 0;
  const int64_t most = WG ? static_cast<int64_t>(g.E) * a.nt * a.mt : (g.R / BM + (g.R < g.E ? g.R : g.E)) * a.nt;
  a.most = static_cast<int>(most);
  a.out = g.out;
  a.out_fp32 = g.out_fp32;
  a.add = g.add;
  a.err = g.err;
  return most <= 1 << 30;
}

// The split of the registers would wait for ever where the launch has fewer.
template <typename... KArgs>
int check_registers(void (*kern)(KArgs...), std::atomic<int>* checked) {
  if (checked->load(std::memory_order_relaxed)) return kOk;
  cudaFuncAttributes at;
  if (cudaFuncGetAttributes(&at, kern) != cudaSuccess) return kErrCuda;
  if (at.numRegs < kMmRegs) return kErrUnsupported;
  checked->store(1, std::memory_order_relaxed);
  return kOk;
}

}  // namespace

}  // namespace eqb
