// Weight gradient of a linear layer from an 8-bit checkpoint of its input: dW[n, k] = sum_t dY[t, n] x^[t, k].
// Part of the translation unit adagc_ops.cu (included there; not compiled on its own).
//
// A contraction over tokens on the 5th-generation tensor cores: tcgen05.mma, bf16 x bf16 into fp32 accumulators in tensor
// memory.  Both operands lie with the token as the slow axis, i.e. "MN-major": 64 consecutive features of one token are one
// 128-byte row of a swizzled tile, as they lie in memory, so no transposition is needed anywhere.
//   D rows (256)    = input features k, 128 per block of a pair (operand A: the checkpoint, decoded on its way)
//   D columns (256) = output features n (operand B: dY, copied by TMA, 128 per block)
// With k along the lanes of the accumulator the epilogue's stores are consecutive in memory.
// The codes of a step of 64 tokens are copied by TMA (a quarter of the bytes that a decoded copy in HBM would cost to write
// and read), decoded to bf16 by eight warps and written to shared memory in the layout the tensor core reads.  Decoding is
// exact: |code| < 2^7 and the scale is a power of two.
//
// What bounds it is shared memory: per step a block's copies and its decoding write 40 KB and read 8 KB there besides the
// operands that the tensor core reads.  Hence two SMs work on one tile (cta_group::2): each keeps one half of both operands.
// Large products then run into the power limit: 8192 x 4096 x 11008 takes 540 us in short runs (1368 TFLOP/s, tensor pipe 81 %
// active) and 630 to 640 us back to back, at an SM clock of 1.28 GHz.
//
// Roles of a block's 16 warps: 0 copies the codes, 1 (of the pair's first block) issues the MMAs, 2 fetches the exponents,
// 3 copies dY and owns the tensor memory, 4-7 epilogue, 8-15 decode.  The codes have a ring of their own, so that they are
// there before a slot of the operands' ring is.  Two accumulators, so the epilogue of one tile runs behind the MMAs of the
// next.  Every wait is bounded; a block that gives up writes NaN over what it still owes.
//
// The tensor core cuts, not rounds, when it adds to an accumulator: measured against 64 bits, the relative error of a
// gradient grows from 2e-7 (1024 tokens) over 1.1e-6 (4096) to 7e-6 (16384), and twice that where the tokens' scales differ.  Where all
// products have one sign it is 5e-5 at 16384 tokens, 3e-4 at 65536 and 1.6e-3 at 262144.
// An fp32 result therefore leaves the accumulator every 1536 tokens at most and is added up in fp32 with rounding (8192 x 4096 x
// 11008: 567 us with 2816, 664 with 1536, 728 with 1024), a bf16 result every 16384.  fp32 is added up in dW itself; bf16, and fp32 if
// dW holds something to be added to, in a block of the workspace: the old values may be far above the sum, and are rounded onto
// once (755 to 800 us; adding to dW at each exit took 760 to 810).
#pragma once

#include <cuda.h>

namespace {

constexpr int kWgTileK = 128, kWgTileN = 256, kWgStep = 64;  // kWgTileK: of one block; a pair has twice that
constexpr int kWgPairK = 2 * kWgTileK, kWgHalfN = kWgTileN / 2;
constexpr int kWgThreads = 512;
constexpr int kWgDecodeWarps = 8, kWgDecodeTeamWarps = 2, kWgEpilogueWarps = 4;
constexpr int kWgDecodeTeams = kWgDecodeWarps / kWgDecodeTeamWarps;
constexpr int kWgSlots = 5, kWgSlotsCodes = 7;  // steps of both operands; steps of codes
static_assert(kWgDecodeTeams <= kWgSlots && kWgDecodeTeams <= kWgSlotsCodes, "a team may be one turn of a ring ahead at most: its waits go by parity");
constexpr int kWgBytesA = kWgTileK * kWgStep * 2, kWgBytesB = kWgHalfN * kWgStep * 2;
constexpr int kWgBytesCodes = kWgTileK * kWgStep, kWgBytesExps = kWgStep * (kWgTileK / 32);
constexpr int kWgSmem = 1024 + kWgSlots * (kWgBytesA + kWgBytesB) + kWgSlotsCodes * (kWgBytesCodes + kWgBytesExps);
constexpr int kWgAtom = 64 * kWgStep * 2;  // 64 features x 64 tokens of bf16: one swizzled column of a tile
constexpr uint32_t kWgTmemCols = 512;
constexpr int kWgExactSteps = 1536 / kWgStep;  // steps after which an fp32 result leaves the accumulator, at most
constexpr int kWgLongSteps = 16384 / kWgStep;  // the same of a bf16 result

// Instruction descriptor of tcgen05.mma kind::f16: fp32 accumulator, bf16 operands, both MN-major, M = 256, N = 256.
constexpr uint32_t kWgInstr = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((kWgTileN / 8) << 17) | ((kWgPairK / 16) << 24);

struct WgradArgs {
  const uint8_t* exps;
  void* out;        // dW
  float* partials;  // 256 x 256 blocks (n, k): of the split tiles, one per split and tile; then, with `apart`, one per pair
  int64_t ld_out, exps_pitch;
  int tokens, n, k;
  int tiles_n;
  int whole, tail, splits;     // tiles taken whole; tiles whose steps are shared out among `splits` pairs of blocks
  int steps, steps_per_split;  // of kWgStep tokens
  int steps_per_flush;
  int out_bf16, accumulate;
  int apart;  // tiles taken whole are summed up in their pair's block and added to dW at their end
};

constexpr uint64_t kDrainNs = 100000000ull;  // for what is still in flight when a block gives up

__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// Arrives at the barrier of the same name in the pair's first block.  What the arrival stands for is either already in the
// async proxy (a landed copy) or has been put there by the arriving warp's fence.proxy.async, so the arrival itself orders
// nothing beyond this block; with .release.cluster each one cost about 1900 cycles.
__device__ __forceinline__ void mbar_arrive_first(uint64_t* bar) {
  asm volatile("{\n .reg .b32 first;\n mapa.shared::cluster.u32 first, %0, 0;\n mbarrier.arrive.shared::cluster.b64 _, [first];\n}\n" ::"r"(smem_u32(bar))
               : "memory");
}
// A bounded wait that also ends when another role of the block has given up.
__device__ __forceinline__ bool wg_wait(uint64_t* bar, uint32_t parity, volatile int* gave_up) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = global_timer_ns();
  for (uint32_t spins = 1;; ++spins) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((spins & 63u) == 0 && (*gave_up || global_timer_ns() - t0 > kWaitLimitNs)) {
      *gave_up = 1;
      return false;
    }
  }
}
__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {  // without waiting
  uint32_t done;
  asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
               : "=r"(done)
               : "r"(smem_u32(bar)), "r"(parity)
               : "memory");
  return done != 0;
}
__device__ __forceinline__ void tma_load_2d(void* dst, const CUtensorMap* map, int x, int y, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(smem_u32(dst)),
               "l"(map), "r"(x), "r"(y), "r"(smem_u32(bar))
               : "memory");
}
// Shared-memory matrix descriptor: MN-major, 128-byte swizzle; `leading` = bytes from one column of 64 features to the next,
// 1024 bytes from 8 tokens to the next 8.
__device__ __forceinline__ uint64_t wg_smem_desc(uint32_t addr, uint32_t leading) {
  return static_cast<uint64_t>((addr & 0x3ffffu) >> 4) | (static_cast<uint64_t>(leading >> 4) << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) |
         (1ull << 46) | (2ull << 61);
}
// The whole warp calls these with the same operands (which then stay in uniform registers); lane 0 issues.
__device__ __forceinline__ void wg_mma(uint32_t lane, uint32_t d, uint64_t a, uint64_t b, uint32_t instr, uint32_t add) {
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.b32 p, %4, 0;\n setp.eq.u32 q, %5, 0;\n @q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(instr), "r"(add), "r"(lane)
      : "memory");
}
// The barriers of the same name in both blocks are told when the MMAs issued so far are done.
__device__ __forceinline__ void wg_commit(uint32_t lane, uint64_t* bar) {
  asm volatile(
      "{\n .reg .pred q;\n setp.eq.u32 q, %2, 0;\n @q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n}\n" ::"r"(
          smem_u32(bar)),
      "h"(static_cast<uint16_t>(3)), "r"(lane)
      : "memory");
}
__device__ __forceinline__ void wg_tmem_load16(uint32_t addr, uint32_t (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                 "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(addr));
}
// The registers of outstanding loads are valid after this (they pass through it, so that nothing uses them before).
__device__ __forceinline__ void wg_tmem_wait(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                 "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
}

// Four codes of one group as two pairs of bf16.  A code's low 7 bits under the exponent byte 0x43 are 128 + those bits; its
// sign bit under 0xc3 is -128 or -256; their sum is the code, times a power of two: every step is exact.
__device__ __forceinline__ uint2 wg_decode4(uint32_t w, __nv_bfloat162 scale) {
  const uint32_t low = w & 0x7f7f7f7fu, sign = w & 0x80808080u;
  uint32_t v0 = __byte_perm(low, 0x43434343u, 0x4140), v1 = __byte_perm(low, 0x43434343u, 0x4342);
  uint32_t b0 = __byte_perm(sign, 0xc3c3c3c3u, 0x4140), b1 = __byte_perm(sign, 0xc3c3c3c3u, 0x4342);
  __nv_bfloat162 x0 = __hmul2(__hadd2(*reinterpret_cast<__nv_bfloat162*>(&v0), *reinterpret_cast<__nv_bfloat162*>(&b0)), scale);
  __nv_bfloat162 x1 = __hmul2(__hadd2(*reinterpret_cast<__nv_bfloat162*>(&v1), *reinterpret_cast<__nv_bfloat162*>(&b1)), scale);
  return make_uint2(*reinterpret_cast<uint32_t*>(&x0), *reinterpret_cast<uint32_t*>(&x1));
}

struct WgTile {
  int n0, k0;
  __host__ __device__ WgTile(int tiles_n, int tile) : n0(tile % tiles_n * kWgTileN), k0(tile / tiles_n * kWgPairK) {}
};
struct WgUnit {  // one tile of dW over one range of steps
  int n0, k0, step0, steps;
  int block;  // of the partials, -1: into dW
  bool whole;
  __device__ __forceinline__ WgUnit(const WgradArgs& a, int u, int rank) {
    const int split = u < a.whole ? 0 : (u - a.whole) / a.tail, tile = u < a.whole ? u : a.whole + (u - a.whole) % a.tail;
    const WgTile t(a.tiles_n, tile);
    n0 = t.n0;
    k0 = t.k0 + rank * kWgTileK;
    whole = u < a.whole;
    block = !whole ? u - a.whole : a.apart ? a.tail * a.splits + static_cast<int>(blockIdx.x / 2) : -1;
    step0 = split * a.steps_per_split;
    steps = u < a.whole ? a.steps : min(a.steps_per_split, a.steps - step0);
  }
};

__device__ __forceinline__ float wg_load(const float* p) { return *p; }
__device__ __forceinline__ float wg_load(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void wg_put(float* p, float x) { *p = x; }
__device__ __forceinline__ void wg_put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
__device__ __forceinline__ void wg_add(float* p, float x) { asm volatile("red.relaxed.gpu.global.add.f32 [%0], %1;" ::"l"(p), "f"(x) : "memory"); }

// One lane's row of an accumulator (one k, 256 n) into `out`, n by n `ld` apart; with kAdd, onto what is there, whose loads
// run 32 ahead (the first ones while the MMAs still run).  The accumulator is read 16 columns ahead of the stores.  !ok: NaN.
template <bool kAdd, typename T, typename Arrived>
__device__ __forceinline__ void wg_store(T* out, int64_t ld, int n, bool mine, uint32_t acc, const bool& ok, Arrived arrived) {
  constexpr int kCols = 16;
  int left = mine ? min(n, kWgTileN) : 0;  // columns from `out` on
  float old[2][kCols];
  const auto fetch = [&](const T* p, int there, float (&o)[kCols]) {
    if (there >= kCols) {  // (loads under a condition each can end up waiting for one another)
#pragma unroll
      for (int c = 0; c < kCols; ++c, p += ld) o[c] = wg_load(p);
    } else {
#pragma unroll
      for (int c = 0; c < kCols; ++c, p += ld)
        if (c < there) o[c] = wg_load(p);
    }
  };
  if constexpr (kAdd) {
    fetch(out, left, old[0]);
    fetch(out + kCols * ld, left - kCols, old[1]);
  }
  arrived();
  uint32_t v[2][kCols];
  __syncwarp();
  wg_tmem_load16(acc, v[0]);
  wg_tmem_wait(v[0]);
#pragma unroll 1
  for (int c0 = 0; c0 < kWgTileN; c0 += 2 * kCols) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      __syncwarp();
      // (the last turn reads the first columns again)
      wg_tmem_load16(acc + (c0 + kCols * (h + 1)) % kWgTileN, v[h ^ 1]);
      T* p = out;
      if (left >= kCols) {
#pragma unroll
        for (int c = 0; c < kCols; ++c, p += ld) {
          const float x = ok ? __uint_as_float(v[h][c]) : quiet_nan();
          wg_put(p, kAdd ? x + old[h][c] : x);
        }
      } else {
#pragma unroll
        for (int c = 0; c < kCols; ++c, p += ld) {
          const float x = ok ? __uint_as_float(v[h][c]) : quiet_nan();
          if (c < left) wg_put(p, kAdd ? x + old[h][c] : x);
        }
      }
      out = p;
      left -= kCols;
      if constexpr (kAdd) fetch(out + kCols * ld, left - kCols, old[h]);
      __syncwarp();
      wg_tmem_wait(v[h ^ 1]);
    }
  }
}

// The end of a tile that is summed up apart from dW: the accumulator and `sums`, added, into `out`; onto what it holds for fp32, and
// with `onto` for bf16; in one rounding.  fp32: a reduction (one addition per element: nothing depends on an order) in place of a load
// and a store, because the usual paths leave no registers for both: with loads here 8192 x 4096 x 11008 took 950 us instead of 770.
template <typename T, typename Arrived>
__device__ __forceinline__ void wg_finish(T* out, int64_t ld, bool onto, const float* sums, int n, uint32_t acc, const bool& ok, Arrived arrived) {
  constexpr int kCols = 16;
  arrived();
#pragma unroll 1
  for (int c0 = 0; c0 < kWgTileN; c0 += kCols, sums += kCols * kWgPairK) {
    float sum[kCols];
#pragma unroll
    for (int c = 0; c < kCols; ++c) sum[c] = sums[c * kWgPairK];
    uint32_t v[kCols];
    __syncwarp();
    wg_tmem_load16(acc + c0, v);
    wg_tmem_wait(v);
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int c = 0; c < kCols; ++c, out += ld)
        if (c0 + c < n) wg_add(out, ok ? __uint_as_float(v[c]) + sum[c] : quiet_nan());
    } else {
#pragma unroll
      for (int c = 0; c < kCols; ++c) sum[c] = ok ? __uint_as_float(v[c]) + sum[c] : quiet_nan();
      if (onto && c0 < n) {
        const T* p = out;
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
          v[c] = *reinterpret_cast<const uint16_t*>(p);
          if (c0 + c + 1 < n) p += ld;  // (beyond the last column that one again)
        }
#pragma unroll
        for (int c = 0; c < kCols; ++c) sum[c] += __uint_as_float(v[c] << 16);
      }
#pragma unroll
      for (int c = 0; c < kCols; ++c, out += ld)
        if (c0 + c < n) wg_put(out, sum[c]);
    }
  }
}

// Calls flush(unit, first step, steps, first flush of the unit, last one) for everything this pair of blocks has to do, in order;
// every role goes through the same list.
template <typename F>
__device__ __forceinline__ void wg_each(const WgradArgs& a, int rank, F flush) {
  const int units = a.whole + a.tail * a.splits;
  for (int u = blockIdx.x / 2; u < units; u += gridDim.x / 2) {
    const WgUnit w(a, u, rank);
    for (int i = 0; i < w.steps; i += a.steps_per_flush)
      if (!flush(w, w.step0 + i, min(a.steps_per_flush, w.steps - i), i == 0, i + a.steps_per_flush >= w.steps)) return;
  }
}

__global__ void __launch_bounds__(kWgThreads, 1) __cluster_dims__(2, 1, 1)
adagc_act8_wgrad_kernel(const __grid_constant__ CUtensorMap map_codes, const __grid_constant__ CUtensorMap map_dy, const WgradArgs a) {
  extern __shared__ unsigned char wg_raw[];
  __shared__ __align__(8) uint64_t full_codes[kWgSlotsCodes], free_codes[kWgSlotsCodes];
  __shared__ __align__(8) uint64_t full_b[kWgSlots], ready[kWgSlots], free_ab[kWgSlots], acc_full[2], acc_empty[2], drain;
  __shared__ uint32_t tmem_base;
  __shared__ int gave_up_flag;
  volatile int* gave_up = &gave_up_flag;
  // swizzled tiles want 1024-byte boundaries; the two blocks' tiles lie at the same addresses
  unsigned char* const tile_a = wg_raw + ((1024u - (smem_u32(wg_raw) & 1023u)) & 1023u);
  unsigned char* const tile_b = tile_a + kWgSlots * kWgBytesA;
  unsigned char* const codes = tile_b + kWgSlots * kWgBytesB;
  unsigned char* const exps = codes + kWgSlotsCodes * kWgBytesCodes;
  // (through a shuffle, so that branches on the warp are known to be uniform)
  const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, rank = blockIdx.x & 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kWgSlotsCodes; ++s) {
      mbar_init(&full_codes[s], 1 + 32);  // the copy's expected bytes, and a lane each of the exponents' warp
      mbar_init(&free_codes[s], kWgDecodeTeamWarps);
    }
    for (int s = 0; s < kWgSlots; ++s) {
      mbar_init(&full_b[s], 1);
      mbar_init(&ready[s], 2 * kWgDecodeTeamWarps);  // both blocks' decoders (in the first block)
      mbar_init(&free_ab[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&acc_full[b], 1);
      mbar_init(&acc_empty[b], 2 * kWgEpilogueWarps);
    }
    mbar_init(&drain, 1);
    gave_up_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 3) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "r"(kWgTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  cg::this_cluster().sync();  // both blocks' barriers exist
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_base;
  // What follows in the stream may start its own set-up (the join of this call, the product of the next one); every block of
  // this kernel is resident.  And this kernel may have been started while the one before it still runs: nothing outside the
  // block is touched before that one is complete.
  griddep_launch_dependents();
  griddep_wait();

  if (warp == 0) {
    if (lane == 0) {
      int it = 0;
      bool ok = true;
      wg_each(a, rank, [&](const WgUnit& w, int step0, int steps, bool, bool) {
        for (int i = 0; i < steps; ++i, ++it) {
          const int s = it % kWgSlotsCodes;
          if (it >= kWgSlotsCodes && !(ok = wg_wait(&free_codes[s], (it / kWgSlotsCodes - 1) & 1, gave_up))) return false;
          mbar_arrive_expect_tx(&full_codes[s], kWgBytesCodes);
          tma_load_2d(codes + s * kWgBytesCodes, &map_codes, w.k0, (step0 + i) * kWgStep, &full_codes[s]);
        }
        return true;
      });
      if (!ok)  // copies still in flight must land before the block ends
        for (int j = max(0, it - kWgSlotsCodes); j < it; ++j)
          (void)mbar_wait_bounded(&full_codes[j % kWgSlotsCodes], (j / kWgSlotsCodes) & 1, kDrainNs);
    }
  } else if (warp == 1) {
    if (rank == 0) {  // the whole warp, in step
      int tile = 0, s = 0, parity = 0;
      bool ok = true, there = false;
      const uint64_t desc_a = wg_smem_desc(smem_u32(tile_a), kWgAtom), desc_b = wg_smem_desc(smem_u32(tile_b), kWgAtom);
      wg_each(a, rank, [&](const WgUnit&, int, int steps, bool, bool) {
        const int buf = tile & 1;
        if (tile >= 2 && !(ok = __all_sync(0xffffffffu, wg_wait(&acc_empty[buf], (tile / 2 - 1) & 1, gave_up)))) return false;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t d = tmem + buf * kWgTileN;
        for (int i = 0; i < steps; ++i) {
          if (!there && !(ok = __all_sync(0xffffffffu, wg_wait(&ready[s], parity, gave_up)))) return false;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint64_t da = desc_a + s * (kWgBytesA >> 4), db = desc_b + s * (kWgBytesB >> 4);
          const int next = s + 1 == kWgSlots ? 0 : s + 1, next_parity = parity ^ (next == 0);
#pragma unroll
          for (int q = 0; q < kWgStep / 16; ++q) {  // 16 tokens are 2048 bytes further in both tiles
            wg_mma(lane, d, da + q * (2048 >> 4), db + q * (2048 >> 4), kWgInstr, (i | q) != 0);
            if (q == 1) there = __all_sync(0xffffffffu, mbar_test(&ready[next], next_parity));  // asked for while the tensor core has work
          }
          wg_commit(lane, &free_ab[s]);
          s = next;
          parity = next_parity;
        }
        wg_commit(lane, &acc_full[buf]);
        ++tile;
        return true;
      });
      if (!ok) {
        wg_commit(lane, &drain);
        (void)mbar_wait_bounded(&drain, 0, kDrainNs);
      }
    }
  } else if (warp == 2) {  // exponents: four bytes per token and step, two tokens per lane
    int it = 0;
    wg_each(a, rank, [&](const WgUnit& w, int step0, int steps, bool, bool) {
      for (int i = 0; i < steps; ++i, ++it) {
        const int s = it % kWgSlotsCodes;
        if (it >= kWgSlotsCodes && !wg_wait(&free_codes[s], (it / kWgSlotsCodes - 1) & 1, gave_up)) return false;
        const int64_t col = w.k0 / 32;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = lane + 32 * h, token = (step0 + i) * kWgStep + r;
          const bool there = token < a.tokens && col < a.exps_pitch;  // the second block of a pair may lie beyond the last column
          const uint8_t* src = there ? a.exps + token * a.exps_pitch + col : a.exps;
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(exps + s * kWgBytesExps + r * 4)), "l"(src), "r"(there ? 4 : 0)
                       : "memory");
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&full_codes[s])) : "memory");
      }
      return true;
    });
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp == 3) {
    if (lane == 0) {
      int it = 0;
      bool ok = true;
      wg_each(a, rank, [&](const WgUnit& w, int step0, int steps, bool, bool) {
        for (int i = 0; i < steps; ++i, ++it) {
          const int s = it % kWgSlots;
          if (it >= kWgSlots && !(ok = wg_wait(&free_ab[s], (it / kWgSlots - 1) & 1, gave_up))) return false;
          mbar_arrive_expect_tx(&full_b[s], kWgBytesB);
#pragma unroll
          for (int j = 0; j < kWgHalfN / 64; ++j)
            tma_load_2d(tile_b + s * kWgBytesB + j * kWgAtom, &map_dy, w.n0 + rank * kWgHalfN + j * 64, (step0 + i) * kWgStep, &full_b[s]);
        }
        return true;
      });
      if (!ok)
        for (int j = max(0, it - kWgSlots); j < it; ++j) (void)mbar_wait_bounded(&full_b[j % kWgSlots], (j / kWgSlots) & 1, kDrainNs);
    }
  } else if (warp >= 8) {
    // Teams of two warps take every fourth step each, so four steps' chains of waits, loads, stores and fences overlap.
    constexpr int kRows = 8 * kWgDecodeTeamWarps;
    const int team = (warp - 8) / kWgDecodeTeamWarps, t = threadIdx.x - 256 - team * 32 * kWgDecodeTeamWarps;
    const int r0 = t >> 2, q = t & 3;  // first token of the step (then every kRows-th), group of 32 features
    const int flip = q >> 1;  // the two upper groups go through their halves in the other order: no bank conflicts
    int it = 0;
    wg_each(a, rank, [&](const WgUnit&, int, int steps, bool, bool) {
      for (int i = (team - it % kWgDecodeTeams + kWgDecodeTeams) % kWgDecodeTeams; i < steps; i += kWgDecodeTeams) {
        const int x = it + i, sc = x % kWgSlotsCodes, sa = x % kWgSlots;
        bool ok = wg_wait(&full_codes[sc], (x / kWgSlotsCodes) & 1, gave_up);
        if (x >= kWgSlots) ok = ok && wg_wait(&free_ab[sa], (x / kWgSlots - 1) & 1, gave_up);
        if (!__all_sync(0xffffffffu, ok)) return false;
        const unsigned char* src = codes + sc * kWgBytesCodes + r0 * 128;
        unsigned char* dst = tile_a + sa * kWgBytesA + (q >> 1) * kWgAtom + r0 * 128;
#pragma unroll
        for (int j = 0; j < kWgStep / kRows; ++j, src += kRows * 128, dst += kRows * 128) {
          const uint32_t e = exps[sc * kWgBytesExps + (r0 + j * kRows) * 4 + q];
          const uint32_t sb = (e == 255u ? 0x7fc0u : e << 7) * 0x10001u;
          const __nv_bfloat162 scale = *reinterpret_cast<const __nv_bfloat162*>(&sb);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int half = h ^ flip;
            const uint4 c = *reinterpret_cast<const uint4*>(src + ((2 * q + half) ^ (r0 & 7)) * 16);
            const uint2 x0 = wg_decode4(c.x, scale), x1 = wg_decode4(c.y, scale), x2 = wg_decode4(c.z, scale), x3 = wg_decode4(c.w, scale);
            const int chunk = 4 * (q & 1) + 2 * half;
            *reinterpret_cast<uint4*>(dst + (chunk ^ (r0 & 7)) * 16) = make_uint4(x0.x, x0.y, x1.x, x1.y);
            *reinterpret_cast<uint4*>(dst + ((chunk + 1) ^ (r0 & 7)) * 16) = make_uint4(x2.x, x2.y, x3.x, x3.y);
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the tensor core reads through the async proxy
        __syncwarp();
        if (lane == 0) mbar_arrive(&free_codes[sc]);
        if (!__all_sync(0xffffffffu, wg_wait(&full_b[sa], (x / kWgSlots) & 1, gave_up))) return false;  // this block's half of dY has landed, too
        if (lane == 0) mbar_arrive_first(&ready[sa]);
      }
      it += steps;
      return true;
    });
  } else if (warp >= 4) {
    const int quad = warp & 3;
    int tile = 0;
    bool ok = true;
    wg_each(a, rank, [&](const WgUnit& w, int, int, bool first, bool last) {
      const int buf = tile & 1, k = w.k0 + quad * 32 + lane;
      const uint32_t acc = tmem + (static_cast<uint32_t>(quad * 32) << 16) + buf * kWgTileN;
      const auto arrived = [&] {
        ok = __all_sync(0xffffffffu, ok && wg_wait(&acc_full[buf], (tile / 2) & 1, gave_up));
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      };
      const bool part = w.block >= 0, add = !first || (a.accumulate && !part);
      if (part && w.whole && last) {
        const float* sums = a.partials + static_cast<int64_t>(w.block) * kWgTileN * kWgPairK + (rank * kWgTileK + quad * 32 + lane);
        const int n = k < a.k ? a.n - w.n0 : 0;
        if (a.out_bf16) wg_finish(static_cast<__nv_bfloat16*>(a.out) + w.n0 * a.ld_out + k, a.ld_out, a.accumulate, sums, n, acc, ok, arrived);
        else wg_finish(static_cast<float*>(a.out) + w.n0 * a.ld_out + k, a.ld_out, true, sums, n, acc, ok, arrived);
      } else if (part || !a.out_bf16) {
        float* out = part ? a.partials + static_cast<int64_t>(w.block) * kWgTileN * kWgPairK + (rank * kWgTileK + quad * 32 + lane)
                          : static_cast<float*>(a.out) + w.n0 * a.ld_out + k;
        const int64_t ld = part ? kWgPairK : a.ld_out;
        const int n = part ? kWgTileN : a.n - w.n0;
        if (add) wg_store<true>(out, ld, n, part || k < a.k, acc, ok, arrived);
        else wg_store<false>(out, ld, n, part || k < a.k, acc, ok, arrived);
      } else {
        __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) + w.n0 * a.ld_out + k;
        if (add) wg_store<true>(out, a.ld_out, a.n - w.n0, k < a.k, acc, ok, arrived);
        else wg_store<false>(out, a.ld_out, a.n - w.n0, k < a.k, acc, ok, arrived);
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive_first(&acc_empty[buf]);
      ++tile;
      return true;
    });
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  cg::this_cluster().sync();  // neither block leaves while the other may still reach its memory
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 3) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kWgTmemCols));
}

// The split tiles of dW from their partial sums, added in the splits' order.  A block takes one n of one tile.
template <bool kBF16>
__global__ void __launch_bounds__(kWgPairK)
adagc_act8_wgrad_join_kernel(const WgradArgs a) {
  using E = Elem<kBF16>;
  griddep_wait();  // (what follows is not let in early: the next product's blocks between the join's cost 10 us of 630)
  const int t = blockIdx.x / kWgTileN, row = blockIdx.x % kWgTileN;
  const WgTile tile(a.tiles_n, a.whole + t);
  const int n = tile.n0 + row, k = tile.k0 + static_cast<int>(threadIdx.x);
  if (n >= a.n || k >= a.k) return;
  const float* p = a.partials + (static_cast<int64_t>(t) * kWgTileN + row) * kWgPairK + threadIdx.x;
  const int64_t step = static_cast<int64_t>(a.tail) * kWgTileN * kWgPairK, at = n * a.ld_out + k;
  float sum = p[0];
#pragma unroll 4
  for (int s = 1; s < a.splits; ++s) sum += p[s * step];
  E::store(a.out, at, a.accumulate ? sum + E::load(a.out, at) : sum);
}

// dY into rows that TMA can address (16-byte boundaries), for bases or leading dimensions that are not.  A thread takes 8
// columns; the columns up to the pitch are filled with zeros.
__global__ void __launch_bounds__(kActThreads)
adagc_act8_wgrad_pack_kernel(MatrixIn src, MatrixOut dst, UnitGrid g) {
  griddep_wait();
  griddep_launch_dependents();
  const UnitPlace<kAnywhere> p(g, unit_of<1>(0));
  float v[kUnit];
  load_unit<true, kAnywhere>(src, p, g.cols, v);
  if (p.valid) __stcs(reinterpret_cast<uint4*>(dst.p) + p.at, Elem<true>::collect(v));
}

// dW = 0 (no tokens).
template <bool kBF16>
__global__ void __launch_bounds__(256)
adagc_act8_wgrad_zero_kernel(void* out, int64_t n, int64_t k, int64_t ld) {
  griddep_wait();
  griddep_launch_dependents();
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n * k; i += gridDim.x * 256ll) Elem<kBF16>::store(out, i / k * ld + i % k, 0.0f);
}

}  // namespace
