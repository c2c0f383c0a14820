// Products of microscaled 4-bit operands (mx_format.cuh), plain and grouped by expert, on 5th-generation tensor cores:
//
//   y[t, o] = sum over blocks b of 32 channels of 2^(bx + bw - 254) sum_{i in b} c_x[t, i] c_w[o, i]
//
// The tensor cores multiply the format as it is stored (tcgen05.mma.kind::mxf4.block_scale, K = 64): codes go from
// memory to 128B-swizzled shared memory by TMA and are read there, scales go by TMA to shared memory and from there,
// through registers, to tensor memory, where the MMA reads 2 bytes a row and K = 64.  Sums are float32 in tensor memory.
//
// Weights are the M operand and tokens the N operand: M is 128 whatever the call, N any multiple of 8, so a tile fits
// the tokens there are -- one token of a decode step, an expert's ragged rows -- and the padding is at most 7 of them.
// An accumulator's lane is a channel, so a warp of the epilogue turns 32 channels of a few tokens at a time (`Kept`).
//
// Two forms of one kernel:
//   * CG = 2, CTA pairs: a tile is 256 channels by up to 256 tokens, each CTA with its 128 channels and half of the
//     tokens' codes in shared memory (and all of the tokens' scales in its tensor memory); persistent, one pair a tile;
//   * CG = 1: 128 channels by up to 128 tokens; K may be cut over the CTAs of a cluster (`split`), whose parts are
//     exchanged through distributed shared memory and summed in the order of their K, so results do not depend on timing.
//
// Warps (512 threads):
//   0       TMA of codes              1  issues the MMAs (CG = 2, odd CTA: forwards stages to the even one)
//   2       TMA of scales             3  TMEM (CG = 2, odd CTA: forwards scale slots)
//   4..7    scales from shared to tensor memory, each to its own 32 lanes (the MMA reads a copy in each)
//   8..15   epilogue, two warps a lane quadrant, taking 32-token chunks in turn
// TMEM: accumulators (two where they fit) from column 0, then the scale slots of 512 channels each.  Every wait is
// bounded; a wait that gives up raises the device status word and all roles drain and exit.
#include <cstring>

#include "gemm_pair.cuh"
#include "mx_format.cuh"
#include "per_device.h"
#include "tensor_map.h"

namespace cat {
namespace {

constexpr int kThreads = 512;
constexpr int BM = 128;                     // channels per CTA
constexpr int BK = 256;                     // values per K step (128 bytes a row)
constexpr int kChunk = 512;                 // values per scale slot (16 bytes a row)
constexpr int kMaxStages = 8, kMaxSlots = 4;
// Scales come from memory two slots at a time: a copy's cost goes by its rows, not their bytes, and 384 rows of 16 bytes a
// slot beside 512 of 128 for its codes kept the copy engine from feeding the MMAs.
constexpr int kRing = 2, kGroup = 2, kScaleRow = 16 * kGroup;
constexpr int kScaleWarp0 = 4, kScaleWarps = 4, kEpiWarp0 = 8, kEpiWarps = 8;
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kStageW = BM * 128;      // 16 KiB of weight codes a stage
constexpr uint32_t kStageOut = 1024;        // an epilogue warp's outputs on their way: 16 bf16 or 8 float32 tokens
constexpr uint32_t kScalesW = BM * kScaleRow;   // 4 KiB of weight scales a ring slot
// Shared memory: at least half an SM's, as two CTAs would wait for each other's tensor memory.  Clusters take all but
// 12 KB, whatever they need: a CTA that holds its SM's tensor memory while its cluster waits for another SM's must not
// share the SM with a CTA of some other kernel of which the same holds (all that use tensor memory need more than 12 KB);
// those 12 KB let the next call's CTAs come early.  Pairs take those too, for a sixth stage of 256-token tiles
// (8192 x 8192 -> 28672 561 -> 545 us, 4096 x 14336 -> 4096 86 -> 79).
constexpr size_t kPairSmem = 227 * 1024, kMaxSmem = 215 * 1024, kMinSmem = 120 * 1024;

__device__ uint64_t g_mx_wait_limit = kWaitLimitNs;   // bound of the pipeline waits (cat_set_wait_limit_ns)

struct MxArgs {
  const int32_t* offsets;                   // grouped: [experts + 1], else null
  void* y;
  uint32_t* status;
  int experts, m, d, d_out;
  int nt;                                   // most tokens of a tile
  int channel_tiles, token_tiles;           // tiles along each side (token_tiles: not grouped)
  int bx, bxs;                              // token rows per TMA box: codes, scales
  int stages, acc_bufs, slots, xcols;       // xcols: TMEM columns of the tokens' scales per 128 channels
  int split, split_log;                     // CTAs that share a tile's K (CG = 1), a power of two up to 8, and its logarithm
  uint32_t stage_bytes, ring_bytes;
  uint32_t off_ring, off_out, off_red, off_table, off_bars;
};

struct Bars {
  uint64_t full[kMaxStages], ready[kMaxStages], empty[kMaxStages];
  uint64_t sfull[kRing], sempty[kRing];                       // scales in shared memory
  uint64_t tfull[kMaxSlots], tready[kMaxSlots], tempty[kMaxSlots];   // scales in tensor memory
  uint64_t acc_full[2], acc_empty[2], mma_done;
  uint32_t fwd_stage[kMaxStages], fwd_slot[kMaxSlots], fwd_acc[kEpiWarps];   // even CTA: targets of the odd CTA's st.async
  uint32_t tmem_addr;
  int abort;
};

// A place in a ring of buffers and the parity of its round: next() in step with the ring's other side.
struct Place {
  uint32_t at = 0, round = 0;
  __device__ __forceinline__ void next(uint32_t of) {
    if (++at == of) {
      at = 0;
      ++round;
    }
  }
  // waits that follow the ring's fillings (full) or the buffer's release in the round before (free)
  __device__ __forceinline__ bool first() const { return round == 0; }
  __device__ __forceinline__ uint32_t full() const { return round & 1; }
  __device__ __forceinline__ uint32_t free() const { return (round - 1) & 1; }
};

// Whether a barrier's phase is over, without waiting.
__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {
  uint32_t over;
  asm volatile("{ .reg .pred p; mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
               : "=r"(over)
               : "r"(smem_u32(bar)), "r"(parity)
               : "memory");
  return over != 0;
}

// A whole warp waits (and knows the outcome to be the same in all lanes).
__device__ __forceinline__ bool all_wait(uint64_t* bar, uint32_t parity, volatile int* abort, int line, uint64_t limit) {
  return (bool)__all_sync(0xFFFFFFFFu, mbar_wait_bounded(bar, parity, abort, line, limit));
}
// Waits for the last fillings of a ring's buffers, `at` its next place: at most kWaitLimitNs in all (after a wait that gave
// up, a buffer's other signal may never come).
__device__ __forceinline__ void drain(uint64_t* full, Place at, uint32_t of) {
  volatile int no_abort = 0;
  const uint64_t t0 = globaltimer_ns();
  for (uint32_t b = 0; b < of; ++b) {
    const uint32_t fills = at.round + (b < at.at ? 1u : 0u);
    const uint64_t spent = globaltimer_ns() - t0;
    if (fills > 0) mbar_wait_bounded(&full[b], (fills - 1) & 1, &no_abort, 1, spent < kWaitLimitNs ? kWaitLimitNs - spent : 1);
  }
}

struct Tile {
  int w_row;                                // the expert's first row of the weights
  int o0;                                   // first channel (of the pair)
  int t0, valid, n;                         // tokens: first row, how many, padded to a multiple of 8 CG
};

// ---- tensor memory and MMA ---------------------------------------------------------------------
// N consecutive columns of this warp's 32 lanes
template <int N>
__device__ __forceinline__ void tmem_st(uint32_t taddr, const uint32_t* v);
template <>
__device__ __forceinline__ void tmem_st<8>(uint32_t taddr, const uint32_t* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
template <>
__device__ __forceinline__ void tmem_st<16>(uint32_t taddr, const uint32_t* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}
template <>
__device__ __forceinline__ void tmem_st<32>(uint32_t taddr, const uint32_t* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Instruction descriptor of kind::mxf4: A and B E2M1, K-major, scales E8M0, D fp32, shape M x N.
__device__ __forceinline__ uint32_t idesc_mxf4(int M, int N) {
  return (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | (1u << 23) | ((uint32_t)(M >> 7) << 27);
}
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{ .reg .pred q; elect.sync _|q, 0xFFFFFFFF; selp.u32 %0, 1, 0, q; }" : "=r"(p));
  return p != 0;
}
// which byte of a scale column's word an MMA's first scale is in (0 or 2), of A and of B
__device__ __forceinline__ uint32_t idesc_scale_byte(uint32_t id) { return (id << 4) | (id << 29); }

template <int CG>
__device__ __forceinline__ void mma_mxf4(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t a_scale,
                                         uint32_t b_scale, uint32_t accumulate) {
  if constexpr (CG == 2)
    asm volatile(
        "{ .reg .pred p; setp.ne.b32 p, %6, 0; "
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p; }" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(a_scale), "r"(b_scale), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{ .reg .pred p; setp.ne.b32 p, %6, 0; "
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p; }" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(a_scale), "r"(b_scale), "r"(accumulate)
        : "memory");
}
template <int CG>
__device__ __forceinline__ void commit(uint64_t* bar) {
  if constexpr (CG == 2)
    mma_commit_pair(bar);
  else
    mma_commit(bar);
}

// Scales of 32 R rows, 16 bytes of row 32 j + lane (half g of its 32), to w[R i + j] = the word of blocks 4 i .. 4 i + 3;
// bytes from `have` on are zero.  The rows lie with the copy engine's 32-byte swizzle (halves change places in every
// second four rows), which eight lanes' reads of a half take without bank conflicts.
template <int R>
__device__ __forceinline__ void load_scales(const uint8_t* src, int lane, int g, int have, uint32_t* w) {
  const uint8_t* at = src + lane * kScaleRow + ((g ^ (lane >> 2 & 1)) << 4);
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const uint4 v = *reinterpret_cast<const uint4*>(at + 32 * kScaleRow * j);
    w[j] = v.x;
    w[R + j] = v.y;
    w[2 * R + j] = v.z;
    w[3 * R + j] = v.w;
  }
  if (have < 16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int left = have - 4 * i;
      const uint32_t mask = left >= 4 ? 0xFFFFFFFFu : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
#pragma unroll
      for (int j = 0; j < R; ++j) w[R * i + j] &= mask;
    }
  }
}
template <int R>
__device__ __forceinline__ void store_scales(const uint8_t* src, int lane, int g, int have, uint32_t taddr) {
  uint32_t w[4 * R];
  load_scales<R>(src, lane, g, have, w);
  if constexpr (R == 6) {
    tmem_st<16>(taddr, w);
    tmem_st<8>(taddr + 16, w + 16);
  } else {
    tmem_st<4 * R>(taddr, w);
  }
}

// A cluster barrier in two parts, which orders no memory.
__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// a float32 into CTA `rank`'s shared memory at this address's offset
__device__ __forceinline__ void st_cluster(float* p, uint32_t rank, float v) {
  uint32_t remote;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(remote), "f"(v) : "memory");
}

template <typename T>
__device__ __forceinline__ T to_out(float v);
template <>
__device__ __forceinline__ float to_out<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 to_out<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Named barrier 4: warp 2 has asked for the first scales, warp 0 goes on behind it.
__device__ __forceinline__ void first_scales_arrive() { asm volatile("bar.arrive 4, 64;" ::: "memory"); }
__device__ __forceinline__ void first_scales_sync() { asm volatile("bar.sync 4, 64;" ::: "memory"); }

// Named barrier 5: all but the copies' warps, 0 and 2.
__device__ __forceinline__ void tmem_there_sync() { asm volatile("bar.sync 5, %0;" ::"n"(kThreads - 64) : "memory"); }

// Two float32 bit patterns to bf16, the first in the low half.
__device__ __forceinline__ uint32_t pack_bf16(uint32_t lo, uint32_t hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(lo), __uint_as_float(hi));
  return *reinterpret_cast<const uint32_t*>(&h);
}

// 16 lanes of tensor memory by 32 columns: of each 8 columns g, thread l has lanes l / 4 (v[4 g], v[4 g + 1]) and l / 4 + 8
// (v[4 g + 2], v[4 g + 3]) at columns 8 g + 2 (l % 4) and the next -- as the rows of stmatrix's 8 x 8 matrices lie.
__device__ __forceinline__ void tmem_ld_16x256b_x4(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr));
}
__device__ __forceinline__ void stmatrix_x4_trans(uint32_t row, const uint32_t* r) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(row), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3])
               : "memory");
}

// An accumulator chunk (32 tokens of a warp's 32 channels) as a warp keeps it until it is stored, and its way to rows of y
// (`left` tokens and `channels` channels of it are there).  Rows of 16-byte multiples (WHOLE) go through the warp's part of
// shared memory, a few tokens at a time as [token][32 channels], and leave 16 bytes a lane; others straight from the
// registers, a channel a lane, 64 or 128 bytes of a token an instruction (3843 x 2560 -> 3709, bf16: 27.1 us; through shared
// memory in 2-byte pieces 31.4, in words that straddle them 37.3).  (One part for the four warps of a half, whole
// 256-byte rows, took two barriers every 16 tokens and 790 cycles; bf16 put in shared memory a value at a time, 500: 521 x
// 1024 -> 23104 18.0 us, 15.3 here.)
template <typename T, bool WHOLE>
struct Kept;

template <bool WHOLE>
struct Kept<float, WHOLE> {
  static constexpr int kAtOnce = 2;                // chunks kept at once
  uint32_t r[32];                                  // lane = channel, a token a word
  __device__ __forceinline__ void load(uint32_t taddr) {
    CAT_TMEM_LD32(taddr, r);
    tmem_ld_wait();
  }
  __device__ __forceinline__ void store(float* p, int d_out, uint8_t* stage_, int channels, int left) const {
    const int lane = threadIdx.x & 31;
    if constexpr (WHOLE) {
      constexpr int kStaged = kStageOut / 128;     // 8 tokens, four an instruction
      float* stage = reinterpret_cast<float*>(stage_);
      const int c = lane % 8 * 4;
      left = c < channels ? left - lane / 8 : 0;   // (16 bytes are wholly in or out of a row)
      float* to = p + (size_t)(lane / 8) * d_out + c;
      const size_t step = 4 * (size_t)d_out;
#pragma unroll
      for (int i0 = 0; i0 < 32; i0 += kStaged) {
        __syncwarp();                              // the tokens before have been read
#pragma unroll
        for (int i = 0; i < kStaged; ++i) stage[i * 32 + lane] = __uint_as_float(r[i0 + i]);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kStaged; i += 4, to += step)
          if (i0 + i < left) *reinterpret_cast<float4*>(to) = *reinterpret_cast<const float4*>(stage + i * 32 + lane * 4);
      }
    } else if (lane < channels) {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (i < left) p[(size_t)i * d_out + lane] = __uint_as_float(r[i]);
    }
  }
};

template <>
struct Kept<__nv_bfloat16, true> {
  static constexpr int kAtOnce = 4;
  uint32_t r[16];                                  // word 4 g + m: 8 x 8 values, tokens 8 g .. by channels 8 m ..; a lane has
                                                   // tokens 2 (lane % 4), + 1 of channel lane / 4
  __device__ __forceinline__ void load(uint32_t taddr) {
    uint32_t v[16], u[16];                         // channels 0 .. 15 and 16 .. 31
    tmem_ld_16x256b_x4(taddr, v);
    tmem_ld_16x256b_x4(taddr + (16u << 16), u);
    tmem_ld_wait();
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      r[4 * g] = pack_bf16(v[4 * g], v[4 * g + 1]);
      r[4 * g + 1] = pack_bf16(v[4 * g + 2], v[4 * g + 3]);
      r[4 * g + 2] = pack_bf16(u[4 * g], u[4 * g + 1]);
      r[4 * g + 3] = pack_bf16(u[4 * g + 2], u[4 * g + 3]);
    }
  }
  // A token's four 16-byte pieces lie as piece q at q ^ (token / 2 mod 4): the eight rows of a matrix, and eight lanes'
  // pieces of two tokens, are in different banks.
  __device__ __forceinline__ void store(__nv_bfloat16* p, int d_out, uint8_t* stage, int channels, int left) const {
    static_assert(kStageOut == 16 * 64, "two groups of eight tokens are staged at once");
    int lane = threadIdx.x & 31;
    asm volatile("" : "+r"(lane));                 // (addresses made per chunk, not kept across them: registers are short)
    const int c = lane % 4 * 8;
    left = c < channels ? left - lane / 4 : 0;
    __nv_bfloat16* to = p + (size_t)(lane / 4) * d_out + c;
    const size_t step = 8 * (size_t)d_out;
    // lane l gives the row of token l % 8 of the matrix of channels 8 (l / 8) .., and takes piece l % 4 of token l / 4
    const uint32_t row = smem_u32(stage) + (uint32_t)(lane & 7) * 64u + (uint32_t)(((lane >> 3) ^ (lane >> 1 & 3)) << 4);
    const uint8_t* from = stage + (lane >> 2) * 64 + (((lane & 3) ^ (lane >> 3 & 3)) << 4);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      __syncwarp();                                // the tokens before have been read
#pragma unroll
      for (int g = 0; g < 2; ++g) stmatrix_x4_trans(row + (uint32_t)g * 512u, r + 8 * h + 4 * g);
      __syncwarp();
#pragma unroll
      for (int g = 0; g < 2; ++g, to += step)
        if (16 * h + 8 * g < left) *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(from + g * 512);
    }
  }
};

template <>
struct Kept<__nv_bfloat16, false> {
  static constexpr int kAtOnce = 4;
  uint32_t r[16];                                  // lane = channel, two tokens a word
  __device__ __forceinline__ void load(uint32_t taddr) {
    uint32_t v[32];
    CAT_TMEM_LD32(taddr, v);
    tmem_ld_wait();
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
  }
  __device__ __forceinline__ void store(__nv_bfloat16* p, int d_out, uint8_t*, int channels, int left) const {
    const int lane = threadIdx.x & 31;
    if (lane < channels) {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (i < left) p[(size_t)i * d_out + lane] = __ushort_as_bfloat16((unsigned short)(r[i / 2] >> (16 * (i & 1))));
    }
  }
};

// Grouped: all threads fill the table: rows[e], the first row of expert e (rows[experts]: one past the last), and
// tiles[e], the tiles of the experts before it (tiles[experts]: all).  Offsets are taken in order and within [0, m],
// whatever they are.  Scans by warps of 32 entries each, then the 32s' totals: one round trip to memory.
constexpr int kMaxChunks = (int)kMxMaxExperts / 32 + 1;
__device__ __forceinline__ void make_table(const MxArgs& a, int* rows, int* tiles, int channel_tiles, int* totals) {
  const int lane = threadIdx.x & 31, first = threadIdx.x & ~31;
  const int entries = a.experts + 1;
  for (int e0 = first; e0 < entries; e0 += kThreads) {
    const int e = e0 + lane;
    int o = e < entries ? min(max(a.offsets[e], 0), a.m) : 0;
#pragma unroll
    for (int k = 1; k < 32; k <<= 1) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, o, k);
      if (lane >= k) o = max(o, v);
    }
    if (e < entries) rows[e] = o;
    if (lane == 31) totals[e0 / 32] = o;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < entries; e += kThreads) {
    int o = rows[e];
    for (int c = 0; c < e / 32; ++c) o = max(o, totals[c]);
    rows[e] = o;
  }
  __syncthreads();
  for (int e0 = first; e0 < entries; e0 += kThreads) {
    const int e = e0 + lane;
    const int mine = e < a.experts ? (rows[e + 1] - rows[e] + a.nt - 1) / a.nt * channel_tiles : 0;
    int s = mine;
#pragma unroll
    for (int k = 1; k < 32; k <<= 1) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, s, k);
      if (lane >= k) s += v;
    }
    if (e < entries) tiles[e] = s - mine;
    if (lane == 31) totals[kMaxChunks + e0 / 32] = s;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < entries; e += kThreads) {
    int s = tiles[e];
    for (int c = 0; c < e / 32; ++c) s += totals[kMaxChunks + c];
    tiles[e] = s;
  }
}

// WHOLE: rows of y are multiples of 16 bytes.
template <int CG, typename T, bool WHOLE>
__global__ void __launch_bounds__(kThreads, 1)
    mx_gemm_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX,
                   const __grid_constant__ CUtensorMap tmWs, const __grid_constant__ CUtensorMap tmXs,
                   const __grid_constant__ MxArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* ring = smem + a.off_ring;            // kRing x [weights' scales 128 x 32 B | tokens' scales]
  float* red = reinterpret_cast<float*>(smem + a.off_red);   // split: [part][token of this CTA's][128 channels]
  int* rows = reinterpret_cast<int*>(smem + a.off_table);    // grouped: see make_table
  int* tiles = rows + a.experts + 1;
  Bars* bars = reinterpret_cast<Bars*>(smem + a.off_bars);
  volatile int* abort_flag = &bars->abort;
  T* y = static_cast<T*>(a.y);

  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);   // (known to be the same in all lanes)
  const uint32_t rank = cluster_rank();
  const int csize_log = CG == 2 ? 1 : a.split_log;   // CTAs of a cluster
  const int cluster = blockIdx.x >> csize_log, clusters = gridDim.x >> csize_log;
  const int channel_tiles = a.channel_tiles, token_tiles = a.token_tiles;
  const int chunks = (a.d + kChunk - 1) / kChunk, steps = (a.d + BK - 1) / BK;
  // this CTA's share of K, in whole chunks
  const int c0 = CG == 2 ? 0 : (int)rank * chunks >> a.split_log, c1 = CG == 2 ? chunks : ((int)rank + 1) * chunks >> a.split_log;
  const int k0 = 2 * c0, k1 = min(2 * c1, steps);

  if (warp == 2 && lane == 0) {                  // (parameters: no need to wait for the kernel before)
    prefetch_tensormap(&tmW);
    prefetch_tensormap(&tmX);
    prefetch_tensormap(&tmWs);
    prefetch_tensormap(&tmXs);
  }
  if (tid == 0) {
    for (int s = 0; s < a.stages; ++s) {
      mbar_init(&bars->full[s], 1);
      mbar_init(&bars->ready[s], 1);
      mbar_init(&bars->empty[s], 1);
    }
    for (int s = 0; s < kRing; ++s) {
      mbar_init(&bars->sfull[s], 1);
      mbar_init(&bars->sempty[s], kScaleWarps);
    }
    for (int s = 0; s < a.slots; ++s) {
      mbar_init(&bars->tfull[s], kScaleWarps);
      mbar_init(&bars->tready[s], kScaleWarps);
      mbar_init(&bars->tempty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&bars->acc_full[b], 1);
      mbar_init(&bars->acc_empty[b], kEpiWarps);   // (CG = 2, even CTA: + 4 bytes from each of the odd CTA's warps)
    }
    mbar_init(&bars->mma_done, 1);
    bars->abort = 0;
    fence_mbar_init();
  }
  if constexpr (CG == 2) {
    cluster_sync();                              // barriers are there, in the whole cluster
  } else {
    __syncthreads();
    cluster_arrive_relaxed();                    // (a split's other CTAs have to be there only when parts are sent)
  }
  pdl_wait_then_release();                       // nothing global or in tensor memory before this
  const uint64_t lim = g_mx_wait_limit;
  if (a.offsets) {
    make_table(a, rows, tiles, channel_tiles, tiles + a.experts + 1);
    __syncthreads();
  }
  // The copies start here; the others wait for tensor memory.  (The even CTA's MMAs write the odd one's too: they wait for its
  // scales, which come after its allocation.)
  uint32_t tmem = 0;
  if (warp == 3) {
    if constexpr (CG == 2)
      tmem_alloc_pair(&bars->tmem_addr, kTmemCols);
    else
      tmem_alloc(&bars->tmem_addr, kTmemCols);
  }
  if (warp != 0 && warp != 2) {
    tc_fence_before();
    tmem_there_sync();
    tc_fence_after();
    tmem = __shfl_sync(0xFFFFFFFFu, bars->tmem_addr, 0);
  }
  const int total = a.offsets ? tiles[a.experts] : token_tiles * channel_tiles;

  if (a.offsets) {                               // rows of no group
    const int64_t head = (int64_t)rows[0] * a.d_out, from = (int64_t)rows[a.experts] * a.d_out,
                  all = (int64_t)a.m * a.d_out;
    const int64_t stride = (int64_t)gridDim.x * kThreads, first = (int64_t)blockIdx.x * kThreads + tid;
    for (int64_t i = first; i < head; i += stride) y[i] = to_out<T>(0.f);
    for (int64_t i = from + first; i < all; i += stride) y[i] = to_out<T>(0.f);
  }

  // tile u of the launch, for a whole warp; e: the caller's place in the table (tiles are asked for in order)
  auto tile_at = [&](int u, int& e) {
    Tile t;
    int begin = 0, end = a.m, tt, ct, n_tiles = token_tiles;
    if (a.offsets) {
      // the last expert that begins at u or before (the others there are empty), 32 entries a look (a binary search:
      // 6000 rows of 64 experts, 1024 -> 768, 14.7 us, 14.2 here)
      for (int n = 32; n == 32; e += n) {
        const int next = e + 1 + lane;
        n = __popc(__ballot_sync(0xFFFFFFFFu, next < a.experts && tiles[next] <= u));
      }
      begin = rows[e];
      end = rows[e + 1];
      u -= tiles[e];
      if (end - begin > a.nt) n_tiles = (end - begin + a.nt - 1) / a.nt;
      else n_tiles = 1;
    }
    // tiles of equal size, as few as there must be
    constexpr int kUnit = 8 * CG;
    int size = end - begin;
    tt = 0;
    ct = u;
    if (n_tiles > 1) {
      size = (size + n_tiles - 1) / n_tiles;
      if (a.offsets) {
        ct = u / n_tiles;
        tt = u - ct * n_tiles;
      } else {
        tile_coords(u, token_tiles, channel_tiles, &tt, &ct);
      }
    }
    size = (size + kUnit - 1) / kUnit * kUnit;
    t.w_row = e * a.d_out;
    t.o0 = ct * CG * BM;
    t.t0 = begin + tt * size;
    t.valid = min(size, end - t.t0);             // (may be none, in the last tile)
    t.n = size;
    return t;
  };

  if (warp == 0) {
    // ---------------------------------------------------------------- TMA of codes
    // (Here too all lanes go through the loop and one is elected: a copy issued in a branch of lane 0's took ~300 cycles.  In
    // neither loop do the others wait for it but where they next vote or elect, 3 to 6 % of a K step of up to 128 tokens.)
    first_scales_sync();                           // copies are made in the order they are asked for, and MMAs need both
    Place st;
    bool ok = true;
    int e = 0;
    for (int u = cluster; u < total && ok; u += clusters) {
      const Tile t = tile_at(u, e);
      const int wrow = t.w_row + t.o0 + (int)(CG == 2 ? rank : 0) * BM;
      const int mine = t.n / CG, xrow = t.t0 + (CG == 2 ? (int)rank : 0) * mine;
      const int boxes = mine > a.bx ? (mine + a.bx - 1) / a.bx : 1;
      const uint32_t bytes = kStageW + (uint32_t)(boxes * a.bx) * 128u;
      for (int ks = k0; ks < k1; ++ks, st.next(a.stages)) {
        if (!st.first() && !(ok = all_wait(&bars->empty[st.at], st.free(), abort_flag, __LINE__, lim))) break;
        uint8_t* dst = smem + st.at * a.stage_bytes;
        uint64_t* fb = CG == 2 && rank == 1 ? &bars->ready[st.at] : &bars->full[st.at];
        if (elect_one()) {
          mbar_arrive_expect_tx(fb, bytes + (CG == 2 && rank == 0 ? 4u : 0u));   // (+ the odd CTA's signal)
          tma_load_2d(dst, &tmW, ks * (BK / 2), wrow, fb);
          tma_load_2d(dst + kStageW, &tmX, ks * (BK / 2), xrow, fb);
          if (boxes > 1)                           // (a loop for the first box too: 6 % of a pair's K step)
            for (int b = 1; b < boxes; ++b)
              tma_load_2d(dst + kStageW + (uint32_t)(b * a.bx) * 128u, &tmX, ks * (BK / 2), xrow + b * a.bx, fb);
        }
      }
    }
    // the copies in flight land before the CTA exits (they have, unless a wait gave up)
    if (lane == 0) drain(CG == 2 && rank == 1 ? bars->ready : bars->full, st, a.stages);
  } else if (warp == 2) {
    // ---------------------------------------------------------------- TMA of scales
    bool told = false;                             // the codes' warp, that the first are asked for
    Place rg;
    bool ok = true;
    int e = 0;
    for (int u = cluster; u < total && ok; u += clusters) {
      const Tile t = tile_at(u, e);
      const int wrow = t.w_row + t.o0 + (int)(CG == 2 ? rank : 0) * BM;
      const int boxes = t.n > a.bxs ? (t.n + a.bxs - 1) / a.bxs : 1;
      const uint32_t bytes = kScalesW + (uint32_t)(boxes * a.bxs * kScaleRow);
      for (int c = c0; c < c1; c += kGroup, rg.next(kRing)) {
        if (!rg.first() && !(ok = all_wait(&bars->sempty[rg.at], rg.free(), abort_flag, __LINE__, lim))) break;
        uint8_t* dst = ring + rg.at * a.ring_bytes;
        uint64_t* fb = &bars->sfull[rg.at];
        if (elect_one()) {
          mbar_arrive_expect_tx(fb, bytes);
          tma_load_2d(dst, &tmWs, c * 16, wrow, fb);
          for (int b = 0; b < boxes; ++b)
            tma_load_2d(dst + kScalesW + (uint32_t)(b * a.bxs * kScaleRow), &tmXs, c * 16, t.t0 + b * a.bxs, fb);
        }
        __syncwarp();
        if (!told) first_scales_arrive();
        told = true;
      }
    }
    if (!told) first_scales_arrive();
    if (lane == 0) drain(bars->sfull, rg, kRing);
  } else if (CG == 2 && rank == 1 && (warp == 1 || warp == 3)) {
    // ---------------------------------------------------------------- odd CTA: forward stages (1) and scale slots (3)
    // (an arrive on the even CTA's barrier from the warps that wrote the data would stall them; a thread that waits for
    // them here carries the signal over with an asynchronous 4-byte store)
    if (lane == 0) {
      Place st;
      bool ok = true;
      for (int u = cluster; u < total && ok; u += clusters)
        for (int j = warp == 1 ? k0 : c0; j < (warp == 1 ? k1 : c1); ++j, st.next(warp == 1 ? a.stages : a.slots)) {
          const uint32_t s = st.at;
          uint64_t* here = warp == 1 ? &bars->ready[s] : &bars->tready[s];
          if (!(ok = mbar_wait_bounded(here, st.full(), abort_flag, __LINE__, lim))) break;
          tc_fence_after();
          if (warp == 1)
            st_async_signal(&bars->fwd_stage[s], &bars->full[s], 0);
          else
            st_async_signal(&bars->fwd_slot[s], &bars->tfull[s], 0);
        }
      if (warp == 1) {                           // the pair's last commits have arrived here too
        volatile int no_abort = 0;
        mbar_wait_bounded(&bars->mma_done, 0, &no_abort);
      }
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issuer
    // The tensor cores wait for this warp wherever its instructions between two MMAs take longer than one.  So all lanes
    // go through the loop (what the MMAs need stays in uniform registers) and one is elected to issue, places are counted,
    // not divided, and a K step always has its four MMAs: behind the row's end the codes are zeros and the scales finite.
    const uint32_t npad = (uint32_t)(a.nt + 31) / 32 * 32, scale0 = tmem + a.acc_bufs * npad;
    const uint32_t slot_cols = 16u + 4u * a.xcols, xcols = a.xcols;
    const uint64_t wdesc0 = sdesc_kmajor_sw128(smem_u32(smem)), xdesc0 = sdesc_kmajor_sw128(smem_u32(smem) + kStageW);
    const uint32_t stage16 = a.stage_bytes >> 4;
    auto wait = [&](uint64_t* bar, uint32_t parity, int line) { return all_wait(bar, parity, abort_flag, line, lim); };
    Place st, sl, ac;
    bool ok = true, st_in = false, sl_in = false;   // st_in, sl_in: the next stage, slot has been seen full
    int e = 0;
    for (int u = cluster; u < total && ok; u += clusters, ac.next(a.acc_bufs)) {
      const Tile t = tile_at(u, e);
      const uint32_t acc = tmem + ac.at * npad, idesc = idesc_mxf4(CG * BM, t.n);
      if (!ac.first() && !(ok = wait(&bars->acc_empty[ac.at], ac.free(), __LINE__))) break;
      uint32_t more = 0;                           // accumulate (0: the tile's first MMA)
      for (int ks = k0; ks < k1 && ok; sl.next(a.slots)) {
        if (!__all_sync(0xFFFFFFFFu, sl_in) && !(ok = wait(&bars->tfull[sl.at], sl.full(), __LINE__))) break;
        sl_in = false;
        const uint32_t sw = scale0 + sl.at * slot_cols, sx = sw + 16;
#pragma unroll
        for (int h = 0; h < 2; ++h) {              // the slot's two K steps
          if (h == 1 && ks == k1) break;
          if (!__all_sync(0xFFFFFFFFu, st_in) && !(ok = wait(&bars->full[st.at], st.full(), __LINE__))) break;
          tc_fence_after();
          Place next = st;                         // (the next waits are looked at while these MMAs are issued)
          next.next(a.stages);
          st_in = mbar_test(&bars->full[next.at], next.full());
          if (h == 1) {
            Place next_sl = sl;
            next_sl.next(a.slots);
            sl_in = mbar_test(&bars->tfull[next_sl.at], next_sl.full());
          }
          if (elect_one()) {
            const uint64_t wd = wdesc0 + st.at * stage16, xd = xdesc0 + st.at * stage16;
#pragma unroll
            for (int kk = 0; kk < BK / 64; ++kk) {
              const uint32_t word = h * 2 + (kk >> 1);               // 128 channels' scales a word
              mma_mxf4<CG>(acc, wd + 2 * kk, xd + 2 * kk, idesc | idesc_scale_byte(2u * (kk & 1)), sw + 4 * word,
                           sx + xcols * word, kk ? 1u : more);
            }
            commit<CG>(&bars->empty[st.at]);
          }
          more = 1;
          st.next(a.stages);
          ++ks;
        }
        if (ok && elect_one()) commit<CG>(&bars->tempty[sl.at]);
      }
      if (ok && elect_one()) commit<CG>(&bars->acc_full[ac.at]);
      __syncwarp();
    }
    if (elect_one()) commit<CG>(&bars->mma_done);  // all MMAs complete before TMEM is released
    __syncwarp();
    if (lane == 0) {
      volatile int no_abort = 0;
      mbar_wait_bounded(&bars->mma_done, 0, &no_abort);
      if (CG == 2) drain(bars->acc_empty, ac, a.acc_bufs);   // the odd CTA's last signals have landed
    }
  } else if (warp >= kScaleWarp0 && warp < kScaleWarp0 + kScaleWarps) {
    // ---------------------------------------------------------------- scales to tensor memory
    // Column j of 128 channels' scales holds rows 32 j .. 32 j + 31, a row a lane, its word the scales of 4 blocks; each
    // quadrant of 32 lanes has a copy.  Rows behind the tile's tokens are whatever shared memory holds: nothing uses them.
    const uint32_t quad = (uint32_t)(warp & 3) * 32u << 16;
    const uint32_t npad = (uint32_t)(a.nt + 31) / 32 * 32, scale0 = tmem + a.acc_bufs * npad + quad;
    const uint32_t slot_cols = 16u + 4u * a.xcols;
    Place rg, sl;
    bool ok = true;
    for (int u = cluster; u < total && ok; u += clusters)
      for (int c = c0; c < c1; ++c, sl.next(a.slots)) {
        const int g = (c - c0) % kGroup;           // which slot of its group's copy
        const uint32_t r = rg.at, slot = sl.at;
        if (g == 0 && !(ok = mbar_wait_bounded(&bars->sfull[r], rg.full(), abort_flag, __LINE__, lim))) break;
        if (!sl.first() && !(ok = mbar_wait_bounded(&bars->tempty[slot], sl.free(), abort_flag, __LINE__, lim))) break;
        __syncwarp();
        tc_fence_after();
        const uint8_t* src = ring + r * a.ring_bytes;
        const uint32_t dst = scale0 + slot * slot_cols;
        // the last chunk's bytes behind the row's scales: the MMAs that cover them multiply zero codes, so any finite
        // scale will do
        const int have = a.d / 32 - c * 16;
        uint32_t w[16];
        load_scales<4>(src, lane, g, have, w);
        switch (a.xcols) {                         // 64 tokens a step
          case 2: store_scales<2>(src + kScalesW, lane, g, have, dst + 16); break;
          case 4: store_scales<4>(src + kScalesW, lane, g, have, dst + 16); break;
          case 6: store_scales<6>(src + kScalesW, lane, g, have, dst + 16); break;
          default: store_scales<8>(src + kScalesW, lane, g, have, dst + 16); break;
        }
        tmem_st<16>(dst, w);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        const bool last = g == kGroup - 1 || c == c1 - 1;
        if (last) rg.next(kRing);
        if (lane == 0) {
          if (CG == 2 && rank == 1)
            mbar_arrive(&bars->tready[slot]);
          else if (CG == 2 && warp == kScaleWarp0)
            mbar_arrive_expect_tx(&bars->tfull[slot], 4u);   // the odd CTA's signal completes the slot
          else
            mbar_arrive(&bars->tfull[slot]);
          if (last) mbar_arrive(&bars->sempty[r]);
        }
      }
  } else if (warp >= kEpiWarp0) {
    // ---------------------------------------------------------------- epilogue
    const int quad = warp & 3, half = (warp - kEpiWarp0) >> 2;
    const uint32_t npad = (uint32_t)(a.nt + 31) / 32 * 32;
    uint8_t* stage = smem + a.off_out + (warp - kEpiWarp0) * kStageOut;
    if (CG == 1) cluster_wait();                   // a split's CTAs have all started
    Place ac;
    int e = 0;
    for (int u = cluster; u < total; u += clusters, ac.next(a.acc_bufs)) {
      const Tile t = tile_at(u, e);
      if (!mbar_wait_bounded(&bars->acc_full[ac.at], ac.full(), abort_flag, __LINE__, lim)) break;
      __syncwarp();
      tc_fence_after();
      const int row = quad * 32 + lane, o_first = t.o0 + (CG == 2 ? (int)rank * BM : 0);
      const uint32_t acc = tmem + ((uint32_t)(quad * 32) << 16) + ac.at * npad;
      if (CG == 1 && a.split > 1) {
        // this CTA's part of K: token k of the tile is summed by CTA k mod split, its k / split-th
        const int each = (a.nt + a.split - 1) >> a.split_log;
        for (int c = half; c * 32 < t.valid; c += 2) {
          uint32_t r[32];
          __syncwarp();
          CAT_TMEM_LD32(acc + c * 32, r);
          tmem_ld_wait();
          float* part = red + ((size_t)rank * each + ((c * 32) >> a.split_log)) * BM + row;   // (split divides 32)
#pragma unroll
          for (int i0 = 0; i0 < 32; i0 += 8) {     // (1 x 4096 -> 6144: all 32 passed 7.2 us, out early 6.9)
            if (c * 32 + i0 >= t.valid) break;
#pragma unroll
            for (int i = i0; i < i0 + 8; ++i)
              if (c * 32 + i < t.valid)
                st_cluster(part + (i >> a.split_log) * BM, (uint32_t)i & (a.split - 1), __uint_as_float(r[i]));
          }
        }
        break;                                     // (a split tile is its cluster's only one)
      }
      // The accumulator is read to registers and given back before anything is stored (bf16: all of this warp's part
      // at once; float32: half of it), so the next tile's MMAs wait for the reads alone.
      constexpr int kAtOnce = Kept<T, WHOLE>::kAtOnce;
      bool held = true;
#pragma unroll 1
      for (int c0_ = half; held; c0_ += 2 * kAtOnce) {
        Kept<T, WHOLE> kept[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
          const int c = c0_ + 2 * k;
          if (c * 32 < t.valid) {
            __syncwarp();
            kept[k].load(acc + c * 32);
          }
        }
        held = (c0_ + 2 * kAtOnce) * 32 < t.valid;
        if (!held) {
          tc_fence_before();
          __syncwarp();
          // (an arrive on the even CTA's barrier would wait for this warp's stores of the tile before, ~2000 cycles)
          if (lane == 0) {
            if (CG == 2 && rank == 1)
              st_async_signal(&bars->fwd_acc[warp - kEpiWarp0], &bars->acc_empty[ac.at], 0);
            else if (CG == 2 && warp == kEpiWarp0)
              mbar_arrive_expect_tx(&bars->acc_empty[ac.at], 4u * kEpiWarps);
            else
              mbar_arrive(&bars->acc_empty[ac.at]);
          }
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
          const int c = c0_ + 2 * k, left = t.valid - c * 32;     // tokens of this chunk on
          if (left <= 0) break;
          T* p = y + (size_t)(t.t0 + c * 32) * a.d_out + o_first + quad * 32;
          const int channels = a.d_out - o_first - quad * 32;     // of this warp's 32 that there are
          kept[k].store(p, a.d_out, stage, channels, left);
        }
      }
    }
  }

  __syncwarp();
  tc_fence_before();
  if (CG == 1 && warp < kEpiWarp0) cluster_wait();   // (the epilogue has)
  // MMAs and epilogues are done with TMEM; a split's parts have arrived
  if (CG == 1 && a.split > 1) {
    cluster_sync();
  } else if (CG == 2) {
    cluster_arrive_relaxed();                    // (a releasing one would wait for all stores)
    cluster_wait();
  } else {
    __syncthreads();
  }
  if (CG == 1 && a.split > 1 && cluster < total && !bars->abort) {
    int e = 0;
    const Tile t = tile_at(cluster, e);
    const int each = (a.nt + a.split - 1) >> a.split_log, o = t.o0 + (tid & (BM - 1));
    for (int j = tid / BM; (j << a.split_log) + (int)rank < t.valid; j += kThreads / BM) {
      float sum = 0.f;
      for (int p = 0; p < a.split; ++p) sum += red[((size_t)p * each + j) * BM + (tid & (BM - 1))];
      if (o < a.d_out) y[(size_t)(t.t0 + (j << a.split_log) + (int)rank) * a.d_out + o] = to_out<T>(sum);
    }
  }
  if (bars->abort && tid == 0) report(a.status, timeout_bits(kWhereMxGemm, bars->abort));
  if (warp == 3) {
    tc_fence_after();
    if constexpr (CG == 2)
      tmem_dealloc_pair(tmem, kTmemCols);
    else
      tmem_dealloc(tmem, kTmemCols);
  }
}

// Bytes [rows][row_bytes], box [box_rows][box_bytes] with a swizzle of its row, out-of-range reads zero.
bool make_map(CUtensorMap* map, const uint8_t* base, int64_t rows, int64_t row_bytes, int box_rows, int box_bytes) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)row_bytes, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)row_bytes};
  cuuint32_t box[2] = {(cuuint32_t)box_bytes, (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, box_bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_32B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int sm_count() {
  static PerDevice<int> asked;
  return asked.get([] {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 148;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms <= 0) return 148;
    return sms;
  });
}

struct Call {
  const uint8_t *xq, *xs, *wq, *ws;
  const int32_t* offsets;
  int64_t experts, m, d, d_out;
  void* y;
  uint32_t* status;
  cudaStream_t stream;
};

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// Tensor memory of tiles of up to nt tokens: accumulators, two where two slots of scales fit beside them (to 192 tokens).
struct Columns {
  int xcols, acc_bufs, slots;
  explicit Columns(int nt) {
    xcols = 2 * ((nt + 63) / 64);
    const int npad = (nt + 31) / 32 * 32, slot_cols = 16 + 4 * xcols;
    acc_bufs = 2 * npad + 2 * slot_cols <= (int)kTmemCols ? 2 : 1;
    slots = ((int)kTmemCols - acc_bufs * npad) / slot_cols;
    if (slots > kMaxSlots) slots = kMaxSlots;
  }
};

template <int CG, typename T, bool WHOLE>
cudaError_t launch_form(const Call& c, int nt, int split) {
  MxArgs a;
  memset(&a, 0, sizeof(a));
  a.offsets = c.offsets;
  a.y = c.y;
  a.status = c.status;
  a.experts = c.offsets ? (int)c.experts : 0;
  a.m = (int)c.m;
  a.d = (int)c.d;
  a.d_out = (int)c.d_out;
  a.nt = nt;
  a.channel_tiles = (int)((c.d_out + CG * BM - 1) / (CG * BM));
  a.token_tiles = (int)((c.m + nt - 1) / nt);
  a.split = split;
  a.split_log = split == 8 ? 3 : split / 2;
  // boxes of a whole tile's tokens, or with groups, whose tiles differ, of up to 32 a CTA (64 for pairs: many rows)
  constexpr int kGroupBox = 32 * CG;
  a.bx = c.offsets && nt / CG > kGroupBox ? kGroupBox : nt / CG;
  a.bxs = c.offsets && nt > kGroupBox ? kGroupBox : nt;
  const Columns columns(nt);
  a.xcols = columns.xcols;
  a.acc_bufs = columns.acc_bufs;
  a.slots = columns.slots;
  a.stage_bytes = kStageW + (uint32_t)up(nt / CG, a.bx) * 128u;
  a.ring_bytes = kScalesW + (uint32_t)up(up(nt, a.bxs), 64) * kScaleRow;
  const size_t red = split > 1 ? (size_t)split * ((nt + split - 1) / split) * BM * 4 : 0;
  const size_t table = c.offsets ? up((2 * (c.experts + 1) + 2 * kMaxChunks) * 4, 128) : 0;
  const size_t rest = (size_t)kRing * a.ring_bytes + kEpiWarps * kStageOut + red + table + sizeof(Bars) + 1024;
  const size_t most = CG == 2 ? kPairSmem : kMaxSmem;
  const int stages = (int)((most - rest) / a.stage_bytes);
  a.stages = stages < kMaxStages ? stages : kMaxStages;
  if (a.slots < 2 || a.stages < 2 || nt % (8 * CG) != 0 || a.bx > 256 || a.bxs > 256) return cudaErrorInvalidConfiguration;
  a.off_ring = a.stages * a.stage_bytes;
  a.off_out = a.off_ring + kRing * a.ring_bytes;
  a.off_red = a.off_out + kEpiWarps * kStageOut;
  a.off_table = a.off_red + (uint32_t)red;
  a.off_bars = a.off_table + (uint32_t)table;
  size_t smem = a.off_bars + sizeof(Bars) + 1024;
  if (smem < kMinSmem) smem = kMinSmem;
  if (CG == 2 || split > 1) smem = most;

  CUtensorMap tw, tx, tws, txs;
  const int64_t pitch = mx_pitch(c.d), wrows = (c.offsets ? c.experts : 1) * c.d_out;
  if (!make_map(&tw, c.wq, wrows, c.d / 2, BM, 128) || !make_map(&tx, c.xq, c.m, c.d / 2, a.bx, 128) ||
      !make_map(&tws, c.ws, wrows, pitch, BM, kScaleRow) || !make_map(&txs, c.xs, c.m, pitch, a.bxs, kScaleRow))
    return cudaErrorInvalidValue;
  static PerDevice<cudaError_t> allowed;
  const cudaError_t attr_err = allowed.get([] { return allow_smem(mx_gemm_kernel<CG, T, WHOLE>, CG == 2 ? kPairSmem : kMaxSmem); });
  if (attr_err != cudaSuccess) return attr_err;

  // at most this many tiles (with groups the device knows how many)
  const int64_t token_tiles = (c.m + nt - 1) / nt + (c.offsets ? (c.experts < c.m ? c.experts : c.m) : 0);
  const int64_t tiles = token_tiles * ((c.d_out + CG * BM - 1) / (CG * BM));
  const int csize = CG == 2 ? 2 : split;
  const int64_t resident = sm_count() / csize;
  const int64_t clusters = split > 1 ? tiles : (tiles < resident ? tiles : resident);   // a split tile has a cluster of its own
  if (clusters * csize > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
  note_launch();
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3((unsigned)(clusters * csize), 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = c.stream;
  cudaLaunchAttribute attrs[2];
  attrs[0] = pdl_attr();
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = csize;
  attrs[1].val.clusterDim.y = 1;
  attrs[1].val.clusterDim.z = 1;
  cfg.attrs = attrs;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, mx_gemm_kernel<CG, T, WHOLE>, tw, tx, tws, txs, a);
}

// What a call runs on: pairs or single CTAs, the most tokens of a tile, the CTAs that share a tile's K.
struct Form {
  int cg, nt, split;
};

// The form of least estimated time.  A round of tiles costs its K steps and a little for its tokens, whatever is between 8 and 256
// of them; so as few rounds as can be, and in them the narrowest tiles.  A step is 0.28 us where the issuing warps' instructions
// bound it (as fitted; since they look ahead, pairs take 0.24 and single CTAs 0.245: alike, so the constants stand); with
// many CTAs it takes what its bytes do: the weights from memory (6 TB/s), all operands from L2 (16 TB/s: 201 x 4096 -> 6144, whose
// weights three token tiles read, 0.23 us); and a round never takes less than its outputs' way out.  The constants (us) are fitted to bf16 outputs of 1 to 512 tokens on
// 4096 -> 6144, 4096 -> 14336, 14336 -> 4096, 4096 -> 4096, 1024 -> 1024 and 2048 -> 640, and of 521 to 8192 on K of 256 to
// 7040.  Of 90 other calls of 1 to 8192 tokens, 256 to 14336 -> 64 to 28672, the form taken is on average 1 % slower than the
// best of 3 to 25 tried, at most 12 %.  One token, 4096 -> 6144: K in two 7.0 us, whole 7.9; 128 tokens, 14336 -> 4096: K in
// four 13.6, in two (64-wide) 14.7, pairs 18.7; 200, 4096 -> 14336: pairs (one round) 11.8, single CTAs (two) 14.4; 512,
// 4096 -> 4096: 128-wide 9.7, 256-wide 11.4; 3843, 2560 -> 3712: pairs 22.7, single CTAs 24.0; 4674, 1440 -> 2176: pairs of 192
// tokens (two accumulators) 16.9, single CTAs 20.1.
Form pick_form(int64_t groups, int64_t rows, int64_t d, int64_t d_out) {
  const int64_t sms = sm_count(), chunks = (d + kChunk - 1) / kChunk;
  const double steps = (double)((d + BK - 1) / BK);
  Form best = {2, 256, 1};
  double least = 1e30;
  // `at_once` clusters are resident (a cluster stays within a group of 14 to 22 SMs)
  auto consider = [&](int cg, int split, int64_t widest, int64_t at_once) {
    const int64_t unit = 8 * cg, channel_tiles = groups * ((d_out + cg * BM - 1) / (cg * BM));
    const int64_t fewest = (rows + widest - 1) / widest;
    const int64_t rounds = (fewest * channel_tiles + at_once - 1) / at_once;
    if (split > 1 && rounds > 1) return;          // (a split tile has a cluster of its own, launched with the others)
    const int64_t narrow = split > 1 ? 32 : 64, most = (rows + narrow - 1) / narrow;
    int64_t tiles = rounds * at_once / channel_tiles;
    tiles = tiles < fewest ? fewest : tiles > most ? (most < fewest ? fewest : most) : tiles;
    const int64_t nt = up((rows + tiles - 1) / tiles, unit);
    const double active = (double)(cg * split * (tiles * channel_tiles < at_once ? tiles * channel_tiles : at_once));
    const double streams = (double)(cg * split * (channel_tiles < at_once ? channel_tiles : at_once));   // of weights
    const double from_memory = 0.0029 * streams, from_l2 = active * (18.4 + 0.144 * nt / cg) / 16000.0;
    double step = cg == 1 ? 0.28 + 0.0003 * nt : 0.29 + 0.0002 * nt;
    step = step < from_memory ? from_memory : step;
    step = step < from_l2 ? from_l2 : step;
    double round = steps / split * step, us = cg == 1 ? 3.6 + 0.004 * nt : 4.6, out = 0.6 + (nt > 160 ? 0.009 : 0.011) * nt;
    if (cg == 2 && Columns((int)nt).acc_bufs == 1) {   // a tile's MMAs wait for the one before to be read
      round += 0.8 + 0.002 * nt;
      us += round < out ? out : round;
    } else {
      us += round + (cg == 1 ? 0.0 : nt > 160 ? 0.8 + 0.002 * nt : 1.0 + 0.003 * nt);
    }
    us += (rounds - 1) * (round < out ? out : round) + (split > 1 ? 1.2 + 0.02 * nt : 0.0);
    if (us < least) {
      least = us;
      best = {cg, (int)nt, split};
    }
  };
  consider(1, 1, 128, sms);
  const int64_t resident[4] = {0, sms / 2, sms * 36 / 152, sms * 15 / 152};
  for (int k = 1; k < 4; ++k)
    if ((1 << k) <= chunks) consider(1, 1 << k, 128, resident[k]);
  consider(2, 1, 256, sms / 2);
  consider(2, 1, 160, sms / 2);
  return best;
}

template <typename T>
cudaError_t launch_typed(const Call& c) {
  const int64_t groups = c.offsets ? (c.experts < c.m ? c.experts : c.m) : 1;   // with rows, at most
  const int64_t rows = (c.m + groups - 1) / groups;                             // of each, on average
  Form f = pick_form(groups, rows, c.d, c.d_out);
  if (c.offsets) {
    // the host knows no group's rows: tiles have room for four times the average (each takes what its group needs).  Of twelve
    // calls of 4 to 64 experts, twice the average took 2.6 % longer (128 tokens to 4 of 64, a group of 122, 17.5 us against 15.3),
    // eight times as long (1258 rows of 53, 28.5 against 30.3; 8192 of 8, 175 against 172)
    const int64_t room = up(c.m < 4 * rows ? c.m : 4 * rows, 8 * f.cg), widest = 128 * f.cg;
    f.nt = (int)(room < widest ? room : widest);
  }
  if (c.d_out * (int64_t)sizeof(T) % 16 == 0)
    return f.cg == 2 ? launch_form<2, T, true>(c, f.nt, 1) : launch_form<1, T, true>(c, f.nt, f.split);
  return f.cg == 2 ? launch_form<2, T, false>(c, f.nt, 1) : launch_form<1, T, false>(c, f.nt, f.split);
}

}  // namespace

cudaError_t set_mx_wait_limit(uint64_t ns) { return cudaMemcpyToSymbol(g_mx_wait_limit, &ns, sizeof(ns)); }

// offsets == nullptr: one group of all m rows.  Rows that belong to no group are zero.
cudaError_t launch_mx_gemm(const uint8_t* xq, const uint8_t* xs, const uint8_t* wq, const uint8_t* ws,
                           const int32_t* offsets, int64_t experts, int64_t m, int64_t d, int64_t d_out, int out_dtype,
                           void* y, uint32_t* status, cudaStream_t stream) {
  const Call c = {xq, xs, wq, ws, offsets, experts, m, d, d_out, y, status, stream};
  return out_dtype == 0 ? launch_typed<float>(c) : launch_typed<__nv_bfloat16>(c);
}

}  // namespace cat
