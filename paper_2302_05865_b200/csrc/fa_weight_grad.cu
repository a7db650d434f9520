// Weight gradient of a linear layer from the 8-bit checkpoint of its input:
//   dW[o][i] = sum over tokens t of dY[t][o] * X[t][i],   X read back from the checkpoint.
//
// A product of two matrices that are both stored with the summed index (t) as their rows, so both are
// operands with the kept index contiguous ("MN-major").  The transposed product is formed,
// D[i][o] = X^T dY, in tiles of 128 inputs x N outputs, on the 5th-generation tensor cores:
//   * the codes are the operand that needs work before it can be multiplied, so they take the short
//     side of the tile: 64 tokens x 128 codes come in by TMA, their scales by 4-byte asynchronous
//     copies, and converter warps form code * 2^e in bf16 (exact) and write the 128-byte-swizzled layout
//     the MMA reads.  (Loads from global memory in these warps, three or four stages ahead in
//     registers, were waited for all the same: twice the time of the products);
//   * dY is loaded by TMA straight into that layout;
//   * a row of the accumulator is one input, so the 32 lanes of a read-out warp hold 32 neighbouring
//     inputs of one output: stores to dW are coalesced for any alignment of dW.
// fp32 dY is split into three bf16 terms (8 + 8 + 8 bits, exact down to 2^-133) by a pass in front, and the tile is
// multiplied with each; the same pass lays out a bf16 dY whose rows TMA cannot address.
// Few tiles and many tokens: the tokens are split over the blocks, partial products go to scratch in
// fp32 and a second kernel adds them in a fixed order.
// Shared memory bounds it (see Cfg), the read-outs between runs (see kRunF32), and the power limit in a long run.
// Measured with the bias gradient, bf16: 4096 x 4096 from 16384 tokens 479 us, 1147 TFLOP/s, 4096 x 1024 from 32768
// tokens 255 us, 1078 TFLOP/s (294 us in a long run), 768 x 768 from 16384 into fp32 33 us (590 TFLOP/s: 32 steps a pair
// of blocks, and joining 8 splits); an fp32 dY, three products: 4096 x 1024 from 16384 488 us (519 into fp32).
#include <cuda.h>

#include <atomic>
#include <type_traits>

#include "../../include/fa.h"
#include "fa_columns.cuh"
#include "fa_common.cuh"
#include "fa_tensor_map.cuh"
#include "fa_train.h"

namespace fa {
namespace wgrad {

constexpr int kTokens = 64;                          // tokens per stage
constexpr int kIns = 128;                            // inputs per tile: rows of the accumulator
constexpr int kBoxBytes = 64 * kTokens * 2;          // 64 columns x 64 tokens of bf16
constexpr int kBytesA = 2 * kBoxBytes;
constexpr int kCodeBytes = kIns * kTokens;           // codes of a stage as they are stored
constexpr int kRawBytes = kCodeBytes + 4 * kTokens;  // and the scales of the tile's four groups, a word per token
// Most stages of a run.  The tensor cores cut their sums off rather than rounding them, an error that grows with the
// number of additions: 3.1e-7 of a result (inputs of random sign) after 24 stages and in proportion beyond.  So sums are
// read out in runs, whatever the type of the result, and the runs added in fp32.  A bf16 result takes longer ones, off by
// 8e-7, about as a plain fp32 product is: 4096 x 1024 from 32768 tokens 368 us in runs of 24, 270 in runs of 64, 255 in
// one; 4096 x 4096 from 16384 700, 508 and 390.  In one run the error would have no bound: after 131072 tokens 1.7 % of
// the results are rounded to another value, in runs of 64 0.07 %.
constexpr int kRunF32 = 24, kRunBf16 = 64;
constexpr int kConvGroups = 3;                       // a group of four warps converts every third step
// A wait tells two neighbouring phases of a barrier apart and no more, so a role must not be able to arrive at a
// barrier two phases early.  For the converter groups, which skip steps:
//   * a stage of codes belongs to one group (kStagesRaw is a multiple of kConvGroups), which has itself used the
//     stage's previous phase up;
//   * `empty` of step n: the group has done step n - kConvGroups, for which products n - kConvGroups - kStages
//     had ended; with kConvGroups <= kStages that is at most one phase before the one waited for.
constexpr long long kLandCycles = 1LL << 24;         // ~9 ms: far more than any copy takes
constexpr int kScaleWarp = 6 + 4 * kConvGroups;
constexpr int kColumnWarp = kScaleWarp + 1;
// warp 0 dY, 1 MMA, 2-5 read-out, 6.. converters, codes, and (SIDE) four for column sums
template <bool SIDE> constexpr int kThreads = 32 * (kColumnWarp + (SIDE ? 4 : 0));

// A tile of kIns * PAIR inputs x N outputs, by one block or by a pair of blocks on neighbouring SMs.  In a pair each
// block holds its own 128 inputs and half of every 256 of dY's columns, and the tensor cores read the other half from
// the neighbour.  Shared memory moves 128 bytes a cycle for the copies, the converters and the products together: a
// step of 256 outputs, whose products take 512 cycles, costs 898 of its cycles with one block, 642 with a pair and 513
// with a pair whose tile has 512 outputs, where converted codes are used twice.  Such a tile fills tensor memory, so
// that it cannot be read out while the next one is summed.
template <int N, int PAIR> struct Cfg {
  static constexpr int kMma = N < 256 ? N : 256;     // outputs of one instruction
  static constexpr int kAccs = N == 512 ? 1 : 2;     // accumulators; one takes N of the 512 columns of tensor memory
  static constexpr int kBytesB = N / PAIR / 64 * kBoxBytes;
  static constexpr int kStage = kBytesA + kBytesB;   // a stage: codes as bf16, then dY
  static constexpr int kStages = N / PAIR == 256 ? 4 : 5;
  static constexpr int kStagesRaw = N / PAIR == 256 ? kConvGroups : 2 * kConvGroups;
  static_assert(kConvGroups <= kStages && kStagesRaw % kConvGroups == 0, "see the note on phases");
  static constexpr size_t kSmem = 1024 + (size_t)kStages * kStage + (size_t)kStagesRaw * kRawBytes + 256;
  // kind::f16: D fp32, A and B bf16, both MN-major, M = 128 or 256
  static constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) |
                                     ((uint32_t)(kMma >> 3) << 17) | ((uint32_t)(kIns * PAIR >> 4) << 24);
};

struct Params {
  const uint8_t* scales;
  long long rows;
  int scale_pitch;
  int outs, ins;
  int planes;                    // terms of dY; every term is a step of its own, with the codes converted anew
  int tiles_i, tiles;            // tiles along the inputs, in all
  int splits;
  int ksteps;                    // stages of tokens in all
  int run;                       // stages summed in an accumulator, with every term, before they are added in fp32
  int joint;                     // a unit is at most two runs, and no block has two units: both are read out at once
  void* dw;
  int gbf16;
  float* partials;               // fp32 sums [splits][split_stride] for the finishing kernel; null: formed in dw
  size_t split_stride;
  const bf16* dy;                // what map_dy reads: rows `ld`, terms `plane` elements apart
  long long ld, plane;
  float* columns;                // column sums of dY: [splits * tiles_i * 4][width], or null
  int width;                     // outs rounded up to 8
  long long wait_cycles;         // limit of a wait (kWaitCycles unless a test shortened it)
};

template <int N, int PAIR>
struct Bars {
  uint64_t full[Cfg<N, PAIR>::kStages], empty[Cfg<N, PAIR>::kStages];      // full: of the pair's first block
  uint64_t raw_full[Cfg<N, PAIR>::kStagesRaw], raw_empty[Cfg<N, PAIR>::kStagesRaw];
  uint64_t acc_full[2], acc_empty[2];                                      // acc_empty: of the pair's first block
  uint64_t drained;
  uint32_t tmem_base;
};

// MN-major, 128-byte swizzle: 64 elements x 8 tokens are 1024 bytes; the next 8 tokens follow at once,
// the next 64 elements a box later.  Descriptor version 1, layout type 2.
__device__ __forceinline__ uint64_t mn_desc(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(kBoxBytes >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
         ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}

template <int PAIR>
__device__ __forceinline__ void umma(uint32_t tmem_d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if constexpr (PAIR == 1)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem_d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem_d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
// The barrier (in a pair: both blocks') is arrived at when the products issued so far have ended.
template <int PAIR>
__device__ __forceinline__ void umma_commit(uint64_t* bar) {
  if constexpr (PAIR == 1)
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar))
                 : "memory");
  else
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
            smem_u32(bar)),
        "h"((uint16_t)3)
        : "memory");
}
// Address of the same place in the pair's first block.
__device__ __forceinline__ uint32_t in_first(uint32_t saddr) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(saddr));
  return a;
}
// Hands something of this SM (an operand that fence.proxy.async has shown to its tensor core, or accumulators
// read out) over to the thread that issues the products.  No data of this SM is read by that thread, so the
// arrival needs no order of other SMs' memory: as a release for the whole cluster it took half as long again
// as the step it hands over (711 against 484 us for 16384 x 4096 x 4096).
template <int PAIR>
__device__ __forceinline__ void arrive_first(uint64_t* bar) {
  if constexpr (PAIR == 1) mbar_arrive(bar);
  else asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(in_first(smem_u32(bar))) : "memory");
}
template <int PAIR>
__device__ __forceinline__ void sync_all() {
  if constexpr (PAIR == 1) {
    __syncthreads();
  } else {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]),
        "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]),
        "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// A box of dY into this block's memory; its bytes are counted on the barrier of the pair's first block.
template <int PAIR>
__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
  if constexpr (PAIR == 1)
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
            smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, "
        "%4}], [%5];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(in_first(smem_u32(bar)))
        : "memory");
}

__device__ __forceinline__ bool elect_one() {
  uint32_t leader;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(leader));
  return leader != 0;
}

// A unit of work of a block or pair: one tile and one share of the tokens.  Units of one share are neighbours, so the
// blocks that run at the same time read the same tokens.
struct Unit {
  int i0, o0, split, k0, k1;
};
template <int N, int PAIR>
__device__ __forceinline__ Unit unit_of(const Params& p, int u, int rank) {
  Unit w;
  w.split = u / p.tiles;
  const int tile = u - w.split * p.tiles;
  const int oi = tile / p.tiles_i;
  w.i0 = ((tile - oi * p.tiles_i) * PAIR + rank) * kIns;
  w.o0 = oi * N;
  w.k0 = (int)((long long)p.ksteps * w.split / p.splits);
  w.k1 = (int)((long long)p.ksteps * (w.split + 1) / p.splits);
  return w;
}

// Two codes (bytes 0 and 1 of each half of `x`, spread to 16 bits) times the scale, in bf16: with the
// code's low 7 bits l and its sign s, (128 + l) - (128 + 128 s) = code; both operands are bf16 by their bits.
__device__ __forceinline__ uint32_t codes_to_bf16(uint32_t x, __nv_bfloat162 scale) {
  uint32_t a = (x & 0x007F007Fu) | 0x43004300u, b = (x & 0x00800080u) | 0x43004300u;
  __nv_bfloat162 v = __hmul2(__hsub2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b)), scale);
  return *reinterpret_cast<uint32_t*>(&v);
}
// The scale, twice.  The byte is a bf16's exponent, except that 2^-127 has the bits 0x0040; 255 gives Inf, and
// the codes of such a group are 0, so that the products are NaN.
__device__ __forceinline__ __nv_bfloat162 scale_bf16(uint32_t byte) {
  uint32_t s = byte * 0x00800080u;
  if (byte == 0) s = 0x00400040u;
  return *reinterpret_cast<__nv_bfloat162*>(&s);
}

// The steps of a unit in their order: run by run, and within one the smallest terms first, so that the accumulator is
// as small as they are while they are added (what it loses by each addition goes by its own size).
struct Steps {
  int k, pl;             // stage of tokens, term
  int r0, r1, run, k1, planes;
  __device__ __forceinline__ Steps(const Params& p, const Unit& w)
      : k(w.k0), pl(p.planes - 1), r0(w.k0), r1(min(w.k0 + p.run, w.k1)), run(p.run), k1(w.k1), planes(p.planes) {}
  __device__ __forceinline__ bool more() const { return r0 < k1; }
  __device__ __forceinline__ void advance() {
    if (++k < r1) return;
    if (--pl < 0) {
      pl = planes - 1;
      r0 = r1;
      r1 = min(r0 + run, k1);
    }
    k = r0;
  }
};

// Column sums of dY while the products run: the tiles that read the same columns share the steps out among themselves,
// so that every value of dY is read once more, when it is in L2.  (For 4096 x 1024 outputs and inputs of 32768 tokens
// this takes 27 us of 263, 20 of 297 with an fp32 result; a pass of its own over dY took 46.)  Four warps: each takes every fourth pair of
// rows, half a warp (16 chunks of 8 columns) a row, and has sums of its own.
// They are the read-out warps, which have nothing to do until a unit's products end.  Where a unit is read out in
// several runs they do have, and four more warps form the sums (SIDE): 270 against 385 us for the shape above.
// Elsewhere these would only take registers from the others: 35 against 31 us for 768 x 768 from 16384.
template <int N, int PAIR>
struct ColumnSums {
  static constexpr int kCols = N / PAIR;             // this block's
  static constexpr int kHalf = kTokens / 16;         // rows of a thread per half step
  // The unit's steps that are this tile's; half a step's loads are always under way.
  __device__ __forceinline__ static void run(const Params& p, const Unit& w, int tile_i, int rank, int warp, int lane) {
    const int steps = (w.k1 - w.k0) * p.planes;
    const int halves = tile_i < steps ? 2 * ((steps - tile_i + p.tiles_i - 1) / p.tiles_i) : 0;
    float* out = p.columns + ((size_t)(w.split * p.tiles_i + tile_i) * 4 + warp) * p.width;
    for (int c = 0; c < kCols; c += 128) {
      const int col = w.o0 + (c >> 7) * (128 * PAIR) + rank * 128 + (lane & 15) * 8;
      F2 acc[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = two(0.f);
      Raw8<bf16> raw[2][kHalf];
      auto load = [&](int h, Raw8<bf16> (&r)[kHalf]) {
        const int j = tile_i + (h >> 1) * p.tiles_i, k = w.k0 + j / p.planes;
        const bf16* src = p.dy + (long long)(j % p.planes) * p.plane;
        const long long row0 = (long long)k * kTokens + (h & 1) * (kTokens / 2) + 2 * warp + (lane >> 4);
#pragma unroll
        for (int q = 0; q < kHalf; ++q) {
          r[q].zero();
          const long long row = row0 + q * 8;
          if (h < halves && row < p.rows) {
            if (col + 8 <= p.outs) r[q].load(src + row * p.ld + col);
            else if (col < p.outs) r[q] = load_some(src + row * p.ld + col, p.outs - col);
          }
        }
      };
      auto take = [&](const Raw8<bf16> (&r)[kHalf]) {
#pragma unroll
        for (int q = 0; q < kHalf; ++q) {
          F2 v[4];
          r[q].get(v);
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[i] = add2(acc[i], v[i]);
        }
      };
      load(0, raw[0]);
      load(1, raw[1]);
      for (int h = 0; h < halves; h += 2) {
        take(raw[0]);
        load(h + 2, raw[0]);
        take(raw[1]);
        load(h + 3, raw[1]);
      }
      float v[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) apart(acc[i], &v[2 * i], &v[2 * i + 1]);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], 16);
      if (lane < 16 && col < p.width) {
        Raw8<float> r;
        r.put(v);
        r.store(out + col);
      }
    }
  }
};

template <int N, int PAIR, bool SIDE>
__global__ void __launch_bounds__(kThreads<SIDE>, 1) weight_grad_kernel(const __grid_constant__ CUtensorMap map_dy,
                                                                  const __grid_constant__ CUtensorMap map_codes, Params prm) {
  using C = Cfg<N, PAIR>;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* stages =
      reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  unsigned char* raws = stages + (size_t)C::kStages * C::kStage;
  Bars<N, PAIR>* bars = reinterpret_cast<Bars<N, PAIR>*>(raws + (size_t)C::kStagesRaw * kRawBytes);
  static_assert(sizeof(Bars<N, PAIR>) <= 256, "barrier block");
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int units = prm.tiles * prm.splits;
  const int rank = PAIR == 1 ? 0 : blockIdx.x & 1, first_unit = blockIdx.x / PAIR, unit_step = gridDim.x / PAIR;

  if (tid == 0) {
    for (int s = 0; s < C::kStages; ++s) { mbar_init(&bars->full[s], 1 + 4 * PAIR); mbar_init(&bars->empty[s], 1); }
    for (int s = 0; s < C::kStagesRaw; ++s) { mbar_init(&bars->raw_full[s], 1 + 32); mbar_init(&bars->raw_empty[s], 4); }
    for (int s = 0; s < 2; ++s) { mbar_init(&bars->acc_full[s], 1); mbar_init(&bars->acc_empty[s], 4 * PAIR); }
    mbar_init(&bars->drained, 1);
    if (PAIR > 1) asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async();
  }
  if (warp == 1) {
    if constexpr (PAIR == 1) {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem_base)),
                   "r"(C::kAccs * N)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem_base)),
                   "r"(C::kAccs * N)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  __syncthreads();
  sync_all<PAIR>();
  tc_fence_after();
  const uint32_t tmem_base = *reinterpret_cast<volatile uint32_t*>(&bars->tmem_base);
  // Every wait is bounded.  A role whose wait ran out arrives nowhere any more, the others' waits then run out as
  // well, and the read-out writes NaN.  (A shared flag looked at after every wait cost 8 % of the run time.)
  auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait(bar, parity, prm.wait_cycles); };
  if (warp == 0) {
    // ---------------- dY by TMA
    if (elect_one()) {
      uint32_t n = 0;                                   // steps asked for so far
      bool ok = true;
      for (int u = first_unit; u < units && ok; u += unit_step) {
        const Unit w = unit_of<N, PAIR>(prm, u, rank);
        Steps at(prm, w);
        for (; at.more(); at.advance(), ++n) {
          const int s = n % C::kStages;
          ok = wait(&bars->empty[s], ((n / C::kStages) & 1) ^ 1);
          if (!ok) break;
          if (rank == 0) mbar_arrive_expect_tx(&bars->full[s], PAIR * C::kBytesB);
          unsigned char* b = stages + (size_t)s * C::kStage + kBytesA;
#pragma unroll
          for (int q = 0; q < N / PAIR / 64; ++q)
            tma_load_3d<PAIR>(b + q * kBoxBytes, &map_dy, w.o0 + (q >> 1) * (128 * PAIR) + rank * 128 + (q & 1) * 64, at.k * kTokens,
                              at.pl, &bars->full[s]);
        }
      }
      // copies still in flight must land before the block may exit: used up, or, after a wait that ran out, by the time
      // that is given to them here
      for (uint32_t m = n > (uint32_t)C::kStages ? n - C::kStages : 0; m < n; ++m)
        (void)mbar_wait(&bars->empty[m % C::kStages], (m / C::kStages) & 1, kLandCycles);
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---------------- MMA: one elected thread.  (Chosen by `lane == 0` instead, the products alone took a fifth
    // longer: 579 against 484 us for 16384 x 4096 x 4096.)
    if (rank == 0 && elect_one()) {
      uint32_t n = 0, nu = 0;
      bool ok = true;
      for (int u = first_unit; u < units && ok; u += unit_step) {
        const Unit w = unit_of<N, PAIR>(prm, u, rank);
        for (int j0 = w.k0; j0 < w.k1 && ok; j0 += prm.run, ++nu) {
          const int steps = (min(j0 + prm.run, w.k1) - j0) * prm.planes;
          const uint32_t acc = nu % C::kAccs, d = tmem_base + acc * N;
          ok = wait(&bars->acc_empty[acc], ((nu / C::kAccs) & 1) ^ 1);
          for (int j = 0; j < steps && ok; ++j, ++n) {
            const int s = n % C::kStages;
            ok = wait(&bars->full[s], (n / C::kStages) & 1);
            if (!ok) break;
            tc_fence_after();
            const uint32_t a = smem_u32(stages + (size_t)s * C::kStage), b = a + kBytesA;
#pragma unroll
            for (int q = 0; q < kTokens / 16; ++q)      // 16 tokens are two groups of 8: 2048 bytes
#pragma unroll
              for (int h = 0; h < N / C::kMma; ++h)
                umma<PAIR>(d + h * C::kMma, mn_desc(a + q * 2048), mn_desc(b + h * (C::kMma / PAIR / 64) * kBoxBytes + q * 2048),
                           C::kIdesc, (j == 0 && q == 0) ? 0u : 1u);
            umma_commit<PAIR>(&bars->empty[s]);
          }
          if (ok) umma_commit<PAIR>(&bars->acc_full[acc]);
        }
      }
      if (!ok) {                                        // products under way must end before the block may exit
        umma_commit<PAIR>(&bars->drained);
        (void)mbar_wait(&bars->drained, 0);
      }
    }
    __syncwarp();
  } else if (warp < 6) {
    // ---------------- read-out: warp w reads the 32 accumulator rows of its quarter, run by run (see kRunF32).  Two runs
    // and no more: one in each accumulator, added here.  Otherwise the first is stored in fp32, the others are added to
    // it in L2: only this thread ever touches the element, one run after the other, so the order is fixed; an atomic
    // addition is used because nothing has to wait for it (a load, add and store took 100 us of 590 for
    // 16384 x 4096 x 4096).
    const int quarter = warp & 3;
    uint32_t nu = 0;
    bool ok = true;
    for (int u = first_unit; u < units; u += unit_step) {
      const Unit w = unit_of<N, PAIR>(prm, u, rank);
      const int i = w.i0 + quarter * 32 + lane;
      float* sums = prm.partials ? prm.partials + (size_t)w.split * prm.split_stride : static_cast<float*>(prm.dw);
      const bool to_bf16 = prm.gbf16 && !prm.partials;
      if (!SIDE && prm.columns)
        ColumnSums<N, PAIR>::run(prm, w, (u - w.split * prm.tiles) % prm.tiles_i, rank, warp & 3, lane);
      for (int j0 = w.k0; j0 < w.k1;) {
        const bool two_runs = prm.joint && j0 + prm.run < w.k1;
        const uint32_t acc = nu % C::kAccs;
        ok = __all_sync(0xffffffffu, ok && wait(&bars->acc_full[acc], (nu / C::kAccs) & 1));
        if (C::kAccs == 2 && two_runs) ok = __all_sync(0xffffffffu, ok && wait(&bars->acc_full[acc ^ 1], ((nu + 1) >> 1) & 1));
        tc_fence_after();
        for (int c = 0; c < N; c += 32) {
          const uint32_t at_lane = tmem_base + (static_cast<uint32_t>(32 * quarter) << 16) + c;
          uint32_t v[32];
          if (ok) {
            tmem_ld32(at_lane + acc * N, v);
            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
            if (C::kAccs == 2 && two_runs) {
              uint32_t u[32];
              tmem_ld32(at_lane + (acc ^ 1) * N, u);
              asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
              for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) + __uint_as_float(u[j]));
            }
          } else {                                     // a wait ran out: the result shows it
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = 0x7FC00000u;
          }
          const int left = prm.outs - (w.o0 + c);      // outputs from here on
          if (i >= prm.ins || left <= 0) continue;
          const size_t at = (size_t)(w.o0 + c) * prm.ins + i;
          if (j0 > w.k0) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (j < left) atomicAdd(sums + at + (size_t)j * prm.ins, __uint_as_float(v[j]));
          } else if (to_bf16) {
            bf16* out = static_cast<bf16*>(prm.dw) + at;
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (j < left) out[(size_t)j * prm.ins] = __float2bfloat16_rn(__uint_as_float(v[j]));
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (j < left) sums[at + (size_t)j * prm.ins] = __uint_as_float(v[j]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (ok && lane == 0) {
          arrive_first<PAIR>(&bars->acc_empty[acc]);
          if (C::kAccs == 2 && two_runs) arrive_first<PAIR>(&bars->acc_empty[acc ^ 1]);
        }
        nu += two_runs ? 2 : 1;
        j0 += two_runs ? 2 * prm.run : prm.run;
      }
    }
  } else if (warp < kScaleWarp) {
    // ---------------- converters: thread -> 8 codes of tokens t, t + 8, ..., t + 56 of the stage.  All eight
    // lie at fixed distances, in the codes as in the swizzled operand (the swizzle goes by t mod 8).
    const int ct = (tid - 192) & 127, c = ct & 15, t = ct >> 4;
    const uint32_t from = t * kIns + c * 8, scale_from = kCodeBytes + t * 4 + (c >> 2);
    const uint32_t to = (c >> 3) * kBoxBytes + t * 128 + (((c & 7) ^ t) << 4);
    int total = 0;
    for (int u = first_unit; u < units; u += unit_step) {
      const Unit w = unit_of<N, PAIR>(prm, u, rank);
      total += (w.k1 - w.k0) * prm.planes;
    }
    for (int n = (warp - 6) >> 2; n < total; n += kConvGroups) {
      const int s = n % C::kStages, r = n % C::kStagesRaw;
      if (!__all_sync(0xffffffffu, wait(&bars->raw_full[r], (n / C::kStagesRaw) & 1))) break;
      const unsigned char* raw = raws + (size_t)r * kRawBytes;
      uint2 q[8];
      uint32_t e[8];
      uint4 v[8];
#pragma unroll
      for (int h = 0; h < 8; ++h) {
        q[h] = *reinterpret_cast<const uint2*>(raw + from + h * 8 * kIns);
        e[h] = raw[scale_from + h * 32];
      }
#pragma unroll
      for (int h = 0; h < 8; ++h) {
        const __nv_bfloat162 sc = scale_bf16(e[h]);
        v[h].x = codes_to_bf16(__byte_perm(q[h].x, 0, 0x4140), sc);
        v[h].y = codes_to_bf16(__byte_perm(q[h].x, 0, 0x4342), sc);
        v[h].z = codes_to_bf16(__byte_perm(q[h].y, 0, 0x4140), sc);
        v[h].w = codes_to_bf16(__byte_perm(q[h].y, 0, 0x4342), sc);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars->raw_empty[r]);     // every lane has its codes
      if (!__all_sync(0xffffffffu, wait(&bars->empty[s], ((n / C::kStages) & 1) ^ 1))) break;
      unsigned char* dst = stages + (size_t)s * C::kStage + to;
#pragma unroll
      for (int h = 0; h < 8; ++h) *reinterpret_cast<uint4*>(dst + h * 1024) = v[h];
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) arrive_first<PAIR>(&bars->full[s]);
    }
  } else if (SIDE && warp >= kColumnWarp) {
    // ---------------- column sums of dY
    for (int u = first_unit; u < units; u += unit_step) {
      const Unit w = unit_of<N, PAIR>(prm, u, rank);
      ColumnSums<N, PAIR>::run(prm, w, (u - w.split * prm.tiles) % prm.tiles_i, rank, warp - kColumnWarp, lane);
    }
  } else {
    // ---------------- codes by TMA, and their scales: a lane copies the words of two tokens; words past the last
    // token are zero (their codes are zero as well), the copies' arrival is counted on the stage's barrier.
    // A warp of its own, so that codes are asked for as soon as the converters have room, whatever dY waits for.
    uint32_t n = 0;
    bool ok = true;
    const bool leader = elect_one();
    for (int u = first_unit; u < units && ok; u += unit_step) {
      const Unit w = unit_of<N, PAIR>(prm, u, rank);
      // (the second block of a pair may have no inputs at all: its results are not stored)
      const uint8_t* column = prm.scales + ((w.i0 >> 5) < prm.scale_pitch ? w.i0 >> 5 : 0);
      for (Steps at(prm, w); at.more(); at.advance(), ++n) {
        const int r = n % C::kStagesRaw;
        ok = __all_sync(0xffffffffu, wait(&bars->raw_empty[r], ((n / C::kStagesRaw) & 1) ^ 1));
        if (!ok) break;
        if (leader) {
          mbar_arrive_expect_tx(&bars->raw_full[r], kCodeBytes);
          tma_load_2d(raws + (size_t)r * kRawBytes, &map_codes, w.i0, at.k * kTokens, &bars->raw_full[r]);
        }
        __syncwarp();
        const uint32_t dst = smem_u32(raws + (size_t)r * kRawBytes + kCodeBytes);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int t = lane + h * 32;
          const long long row = (long long)at.k * kTokens + t;
          const bool inside = row < prm.rows;
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst + t * 4),
                       "l"(column + (size_t)(inside ? row : 0) * prm.scale_pitch), "r"(inside ? 4 : 0)
                       : "memory");
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&bars->raw_full[r])) : "memory");
      }
    }
    // nothing may be in flight when the block exits: the codes of every step have to have landed
    asm volatile("cp.async.wait_all;" ::: "memory");
    for (uint32_t m = n > (uint32_t)C::kStagesRaw ? n - C::kStagesRaw : 0; m < n; ++m)
      (void)mbar_wait(&bars->raw_full[m % C::kStagesRaw], (m / C::kStagesRaw) & 1);
    __syncwarp();
  }

  tc_fence_before();
  __syncthreads();
  sync_all<PAIR>();                          // neither block of a pair leaves while the other may still reach into it
  if (warp == 1) {
    tc_fence_after();
    if constexpr (PAIR == 1)
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(C::kAccs * N) : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(C::kAccs * N) : "memory");
  }
}

// Adds partial results in a fixed order: blocks below `product_blocks` the partial products, the others the column sums
// (32 columns a block, a warp taking every eighth part).  Launched while the products still run.
struct Finish {
  const float* partials;
  size_t split_stride, n;
  int splits;
  void* dw;
  const float* columns;
  int parts, width, outs;
  void* db;
  int gbf16;
  unsigned product_blocks;
};
__global__ void __launch_bounds__(256) finish_kernel(Finish f) {
  __shared__ float s[8][32];
  cudaGridDependencySynchronize();
  if (blockIdx.x < f.product_blocks) {
    const size_t j = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= f.n) return;
    float v = 0.f;
#pragma unroll 8
    for (int k = 0; k < f.splits; ++k) v += f.partials[k * f.split_stride + j];
    if (f.gbf16) static_cast<bf16*>(f.dw)[j] = __float2bfloat16_rn(v);
    else static_cast<float*>(f.dw)[j] = v;
    return;
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int col = (blockIdx.x - f.product_blocks) * 32 + lane;
  float v = 0.f;
  if (col < f.outs) {
#pragma unroll 8
    for (int k = warp; k < f.parts; k += 8) v += f.columns[(size_t)k * f.width + col];
  }
  s[warp][lane] = v;
  __syncthreads();
  if (warp == 0 && col < f.outs) {
    v = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) v += s[k][lane];
    if (f.gbf16) static_cast<bf16*>(f.db)[col] = __float2bfloat16_rn(v);
    else static_cast<float*>(f.db)[col] = v;
  }
}

// dY as bf16 terms that add up to it exactly (down to 2^-133, bf16's smallest), rows of `pitch` elements:
// [planes][rows][pitch].  Terms are cut off rather than rounded, so that no finite value becomes infinite; what is not
// finite is one term.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) pack_kernel(Source<T> dy, long long rows, int outs,
                                                   int pitch, int planes, bf16* __restrict__ out) {
  const int per_row = pitch / 8;
  const long long n = rows * per_row, plane = rows * pitch;
  for (long long j = (long long)blockIdx.x * 256 + threadIdx.x; j < n; j += (long long)gridDim.x * 256) {
    const long long r = j / per_row;
    const int first = static_cast<int>(j - r * per_row) * 8;
    float v[8];
    Chunk<T, VEC> in;
    in.fetch(dy, dy.p + r * dy.ld, first, outs);
    in.raw(first < outs).get(v);
    for (int q = 0; q < planes; ++q) {
      float term[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        term[k] = sizeof(T) == 2 ? v[k] : __uint_as_float(__float_as_uint(v[k]) & 0xffff0000u);
        if (isnan(v[k])) term[k] = v[k];
        v[k] = isfinite(v[k]) ? v[k] - term[k] : 0.f;
      }
      Raw8<bf16> o;
      o.put(term);
      o.store(out + q * plane + r * pitch + first);
    }
  }
}

constexpr double kWideStep = 1.55;       // time of a step with 512 outputs, in steps with 256 (0.74 and 0.48 us)

// How a product is cut up.  Per block and stage the MMA takes N / 256 * 512 cycles or so; a split costs
// a write and a read of the whole result.
struct Plan {
  int n, pair, tiles_i, tiles_o, tiles, splits, ksteps, planes;
  int run;
  bool joint;
  bool several;        // units are read out more than once: of a bf16 result through fp32 sums and the finishing kernel
  bool pack;
  int pitch;
  size_t pack_bytes, split_stride, partial_bytes, column_bytes;
};

// `gdtype` of the result: one in fp32 is read out in short runs, for which a tile of 512 outputs would have to wait.
Plan plan_of(long long rows, long long outs, long long ins, int dtype, int gdtype, bool pack) {
  Plan p{};
  p.planes = dtype == FA_F32 ? 3 : 1;
  p.pack = pack;
  p.pitch = static_cast<int>((outs + 7) / 8 * 8);
  p.pack_bytes = pack ? ((size_t)p.planes * rows * p.pitch * 2 + 255) / 256 * 256 : 0;
  p.ksteps = static_cast<int>((rows + kTokens - 1) / kTokens);
  auto cut = [&](int n, int pair, double step) {
    p.n = n;
    p.pair = pair;
    p.tiles_i = static_cast<int>((ins + kIns * pair - 1) / (kIns * pair));
    p.tiles_o = static_cast<int>((outs + n - 1) / n);
    const long long tiles = (long long)p.tiles_i * p.tiles_o, blocks = sm_count() / pair;
    p.tiles = static_cast<int>(tiles);
    // splits that fill the blocks once; each keeps at least 4 stages
    long long s = tiles >= blocks ? 1 : blocks / tiles;
    const long long least = (p.ksteps * p.planes + 3) / 4;
    if (s > least) s = least;
    if (s > p.ksteps) s = p.ksteps;
    if (s > 32) s = 32;
    p.splits = static_cast<int>(s < 1 ? 1 : s);
    // time of the busiest block in steps with 256 outputs (0.47 us), and what writing, reading and adding the splits
    // costs in these (2 TB/s: little of it is hidden)
    const long long turns = (tiles * p.splits + blocks - 1) / blocks;
    return (double)turns * ((p.ksteps + p.splits - 1) / p.splits) * p.planes * step +
           (p.splits > 1 ? (double)p.splits * outs * ins * 8.0 / 2e6 / 0.47 : 0.0);
  };
  // Tiles of 128 x 128 by single blocks where there is little to do: more blocks share the read-out, and no pair has to
  // be set up (256 x 256 from 512 tokens 8.8 against 12.5 us, 768 x 768 from 2048 14.8 against 15.8); pairs for more
  // (1024 x 1024 from 8192 29.9 against 41.3).
  const bool little = (double)rows * (double)outs * (double)ins * p.planes <= 2147483648.0;
  const int n = little || outs <= 128 ? 128 : 256, pair = !little && ins > kIns && outs > 128 ? 2 : 1;
  const double cost = cut(n, pair, 1.0);
  if (pair == 2 && outs > 256 && gdtype == FA_BF16 && cut(512, 2, kWideStep) >= cost) cut(n, pair, 1.0);
  const int steps = (p.ksteps + p.splits - 1) / p.splits, most = gdtype == FA_BF16 ? kRunBf16 : kRunF32;
  p.joint = p.n <= 256 && steps <= 2 * most && p.tiles * (long long)p.splits <= sm_count() / p.pair;
  p.run = p.joint ? (steps + 1) / 2 : most;
  p.several = !p.joint && steps > most;
  p.split_stride = ((size_t)outs * ins + 63) / 64 * 64;
  p.partial_bytes = p.splits > 1 || (p.several && gdtype == FA_BF16) ? p.splits * p.split_stride * sizeof(float) : 0;
  p.column_bytes = (size_t)p.splits * p.tiles_i * 4 * p.pitch * sizeof(float);
  return p;
}

}  // namespace wgrad

bool linear_weight_grad_direct(Mat dy, int dtype, long long outs) {
  return dtype == FA_BF16 && aligned16(dy.p) && dy.ld % 8 == 0 && dy.ld >= outs && dy.ld < (1LL << 38);
}

size_t linear_weight_grad_scratch_bytes(long long rows, long long outs, long long ins, int dtype, bool direct) {
  // the type of the result is known at the call
  const wgrad::Plan p = wgrad::plan_of(rows, outs, ins, dtype, FA_F32, !direct);
  const wgrad::Plan q = wgrad::plan_of(rows, outs, ins, dtype, FA_BF16, !direct);
  const size_t a = p.partial_bytes + p.column_bytes, b = q.partial_bytes + q.column_bytes;
  return p.pack_bytes + (a > b ? a : b);
}

namespace {
std::atomic<long long> g_wait_cycles{kWaitCycles};
}  // namespace

}  // namespace fa

// Test hook (exported, but deliberately not declared in include/fa.h): shortens the waits of the weight gradient's kernel
// so that a test can watch them run out on a launch that is otherwise correct.  cycles <= 0 restores the default.
extern "C" void fa_test_set_weight_grad_wait_cycles(long long cycles) {
  fa::g_wait_cycles.store(cycles > 0 ? cycles : fa::kWaitCycles);
}

namespace fa {

template <int N, int PAIR, bool SIDE>
static cudaError_t launch_product(const CUtensorMap& map, const CUtensorMap& map_codes, const wgrad::Params& prm,
                                  cudaStream_t st) {
  using C = wgrad::Cfg<N, PAIR>;
  auto kernel = wgrad::weight_grad_kernel<N, PAIR, SIDE>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(C::kSmem));
  if (e != cudaSuccess) return e;
  const int units = prm.tiles * prm.splits, most = sm_count() / PAIR;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(PAIR * (units < most ? units : most));
  cfg.blockDim = dim3(wgrad::kThreads<SIDE>);
  cfg.dynamicSmemBytes = C::kSmem;
  cfg.stream = st;
  cudaLaunchAttribute cluster{};
  cluster.id = cudaLaunchAttributeClusterDimension;
  cluster.val.clusterDim.x = PAIR;
  cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
  cfg.attrs = &cluster;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, map, map_codes, prm);
}

cudaError_t launch_linear_weight_grad(Mat dy, int dtype, long long rows, long long outs, long long ins, const void* ck,
                                      void* dweight, void* dbias, int gdtype, void* scratch, cudaStream_t st) {
  const size_t n = (size_t)outs * ins;
  if (rows == 0) {
    const size_t g = gdtype == FA_BF16 ? 2 : 4;
    const cudaError_t e = cudaMemsetAsync(dweight, 0, n * g, st);
    return e != cudaSuccess || !dbias ? e : cudaMemsetAsync(dbias, 0, outs * g, st);
  }
  const bool direct = linear_weight_grad_direct(dy, dtype, outs);
  const wgrad::Plan p = wgrad::plan_of(rows, outs, ins, dtype, gdtype, !direct);
  const void* base = dy.p;
  long long ld = dy.ld;
  if (!direct) {
    bf16* packed = static_cast<bf16*>(scratch);
    const bool vec = dtype == FA_F32 && mat_vec<float>(dy, outs);
    const long long want = (rows * (p.pitch / 8) + 255) / 256, most = 16LL * sm_count();
    const unsigned grid = static_cast<unsigned>(want < most ? want : most);
    auto go = [&](auto kernel, auto src) {
      kernel<<<grid, 256, 0, st>>>(src, rows, (int)outs, p.pitch, p.planes, packed);
    };
    if (dtype == FA_BF16) go(wgrad::pack_kernel<bf16, false>, source_of<bf16>(dy, 0, rows, outs));
    else if (vec) go(wgrad::pack_kernel<float, true>, source_of<float>(dy, 0, rows, outs));
    else go(wgrad::pack_kernel<float, false>, source_of<float>(dy, 0, rows, outs));
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    base = packed;
    ld = p.pitch;
  }
  EncodeTiledFn enc = encode_tiled();
  if (!enc) return cudaErrorNotSupported;
  CUtensorMap map;
  const cuuint64_t dims[3] = {(cuuint64_t)outs, (cuuint64_t)rows, (cuuint64_t)p.planes};
  const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)ld * 2 * (p.planes > 1 ? rows : 1)};
  const cuuint32_t box[3] = {64, wgrad::kTokens, 1};
  const cuuint32_t estr[3] = {1, 1, 1};
  if (enc(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr,
          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  const Act8 a = act8_at(ck, rows, ins, 0);
  CUtensorMap map_codes;
  const cuuint64_t code_dims[2] = {(cuuint64_t)act8_groups(ins) * 32, (cuuint64_t)rows};
  const cuuint64_t code_strides[1] = {(cuuint64_t)act8_groups(ins) * 32};
  const cuuint32_t code_box[2] = {wgrad::kIns, wgrad::kTokens};
  if (enc(&map_codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, a.codes, code_dims, code_strides, code_box, estr,
          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  wgrad::Params prm{};
  prm.scales = a.scales;
  prm.rows = rows;
  prm.scale_pitch = static_cast<int>(act8_scale_pitch(ins));
  prm.outs = static_cast<int>(outs); prm.ins = static_cast<int>(ins);
  prm.planes = p.planes;
  prm.tiles_i = p.tiles_i; prm.tiles = p.tiles; prm.splits = p.splits; prm.ksteps = p.ksteps;
  prm.dw = dweight; prm.gbf16 = gdtype == FA_BF16;
  prm.run = p.run; prm.joint = p.joint;
  char* room = static_cast<char*>(scratch) + p.pack_bytes;
  prm.partials = p.partial_bytes ? reinterpret_cast<float*>(room) : nullptr;
  prm.split_stride = p.split_stride;
  prm.dy = static_cast<const bf16*>(base);
  prm.ld = ld;
  prm.plane = ld * rows;
  prm.columns = dbias ? reinterpret_cast<float*>(room + p.partial_bytes) : nullptr;
  prm.width = p.pitch;
  prm.wait_cycles = g_wait_cycles.load();
  const bool side = dbias && p.several;
  auto go = [&](auto with_side) {
    constexpr bool SIDE = decltype(with_side)::value;
    return p.n == 512   ? launch_product<512, 2, SIDE>(map, map_codes, prm, st)
           : p.pair == 2 ? launch_product<256, 2, SIDE>(map, map_codes, prm, st)
           : p.n == 256 ? launch_product<256, 1, SIDE>(map, map_codes, prm, st)
                        : launch_product<128, 1, SIDE>(map, map_codes, prm, st);
  };
  const cudaError_t e = side ? go(std::true_type{}) : go(std::false_type{});
  if (e != cudaSuccess || (!prm.partials && !dbias)) return e;
  wgrad::Finish f{};
  f.partials = prm.partials; f.split_stride = p.split_stride; f.n = n; f.splits = p.splits;
  f.dw = dweight;
  f.columns = prm.columns; f.parts = p.splits * p.tiles_i * 4; f.width = p.pitch; f.outs = (int)outs;
  f.db = dbias;
  f.gbf16 = prm.gbf16;
  f.product_blocks = prm.partials ? (unsigned)((n + 255) / 256) : 0;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(f.product_blocks + (dbias ? (unsigned)((outs + 31) / 32) : 0));
  cfg.blockDim = dim3(256);
  cfg.stream = st;
  cudaLaunchAttribute early{};
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &early;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, wgrad::finish_kernel, f);
}

}  // namespace fa
