// Attention of few query rows over pages of the 4-bit cache (mx_cache.cuh): a decode step, drafted tokens.
//
//   out = sum_t softmax_t(scale q k_t) v_t,   k_t[c] = 2^(bk - 127) e(c),   v_t[c] = 2^(bv - 127) e(c),   e(c) of the E2M1 codes
//
// The scales stay out of the products: a score is the sum over blocks of 2^(bk - 127) times the product of the block's codes with
// the query, and a weight times 2^(bv - 127) multiplies the codes of a block of values.  So the matrix instructions' operands are
// codes as they are (float16, exact) and never scaled numbers, and what is rounded is the query (scaled by a power of two so that
// its largest channel is in [2^13, 2^14): bf16's 8 bits are exact down to 2^-27 of the largest) and the weights.
//
// A token's keys and values are 17/16 of a byte a channel for both, read once for all the query heads that share them: 152 SMs have
// ~2.9 lane instructions a code in the time its bytes take from memory, and the unpacking is most of what there is to do: ~400 warp
// instructions for 16 tokens of a head of 128 channels and 8 rows, 172 of them on the pipe that issues one every other cycle a scheduler.
// 64 sequences of up to 8192 tokens, 8 key heads: 292 MB in 85 us (3.4 TB/s); one of 131000 tokens 46.5 us, 41 of them here; 2.3
// instructions a cycle, from 16 warps an SM (128 registers; 12 and 20 warps were no faster).
// Codes go from memory to registers in the layout of the matrix instructions' operands (which is what the cache's pieces are for) and
// are unpacked in pairs there.  tcgen05 would want them unpacked into shared memory first, for 128 rows where there are 1 to 32.
//
//   S^T [16 tokens x 8 rows] = K Q^T:  a lane (g, t) = (lane / 4, lane % 4) has channels 8 t .. 8 t + 7 of every block of tokens g, g + 8
//   O^T [16 channels x 8 rows] = V^T P^T: channels 4 g .. 4 g + 3 of every block of tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9
// Scores leave with lane (g, t) having tokens g, g + 8 of rows 2 t, 2 t + 1; times the values' scales of its tokens they are
// turned to the second product's operand by movmatrix.
//
// Work is cut evenly, whatever the lengths: units (sequence, row tile, head) lie one behind the other on a line of 32-token steps, and
// each CTA has an equal piece of it, found from the lengths on the device.  A unit in one piece is written at once; the others'
// parts go through the workspace, and a second kernel joins them in the order of their tokens.
#include <cuda_fp16.h>

#include <algorithm>

#include "mx_attention.cuh"
#include "per_device.h"

namespace cat {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kStep = 32;                   // tokens a warp takes at once (two of the products' 16)
constexpr int kUnitCost = 10;               // a unit's beginning and end, in steps (measured: 2 and 24 were up to 11 and 8 % slower)
constexpr int kAhead = kStep * kWarps;      // tokens between a warp's steps
constexpr int kLeastPiece = 4;              // steps a CTA is worth
// The values' reference, a scale byte, as the weights have it: 2^(136 - ref) is what they are times, and within these float32 holds both their
// sums and those that count little.
constexpr int kLowR = 80, kHighR = 200;
constexpr int kBeyond = 2;                  // what a row's reference may be above the largest that the row sees
__device__ __forceinline__ int within(int ref) { return min(max(ref, kLowR), kHighR); }

struct Seq : Rows {
  int steps, tiles;                         // steps and row tiles; no steps: none, or the other kernel's
  __device__ __forceinline__ int64_t cost(int hkv) const { return steps ? (int64_t)tiles * hkv * (steps + kUnitCost) : 0; }
};
template <int ROWS>
__device__ __forceinline__ Seq seq_at(const AttnArgs& a, int s) {
  Seq q;
  static_cast<Rows&>(q) = rows_of(a, s);
  const int64_t rows = (int64_t)q.ql * a.group;
  q.steps = q.any() && rows <= a.few ? (int)((q.end + kStep - 1) / kStep - q.first / kStep) : 0;
  q.tiles = (int)((rows + ROWS - 1) / ROWS);
  return q;
}

// 16 x 8 += 16 x 16 times 16 x 8, float16 operands
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transpose(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// The float16 values of the two codes in byte I of w, the first in the low half.
template <int I>
__device__ __forceinline__ uint32_t code_pair(uint32_t w) {
  uint32_t r;
  if constexpr (I == 0)
    asm("{ .reg .b8 a, b, c, d; mov.b32 {a, b, c, d}, %1; cvt.rn.f16x2.e2m1x2 %0, a; }" : "=r"(r) : "r"(w));
  else if constexpr (I == 1)
    asm("{ .reg .b8 a, b, c, d; mov.b32 {a, b, c, d}, %1; cvt.rn.f16x2.e2m1x2 %0, b; }" : "=r"(r) : "r"(w));
  else if constexpr (I == 2)
    asm("{ .reg .b8 a, b, c, d; mov.b32 {a, b, c, d}, %1; cvt.rn.f16x2.e2m1x2 %0, c; }" : "=r"(r) : "r"(w));
  else
    asm("{ .reg .b8 a, b, c, d; mov.b32 {a, b, c, d}, %1; cvt.rn.f16x2.e2m1x2 %0, d; }" : "=r"(r) : "r"(w));
  return r;
}
__device__ __forceinline__ uint32_t f16_pair(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Four scale bytes as the powers of two (and NaN) that they stand for.
__device__ __forceinline__ void scales4(uint32_t w, float* s) {
  uint32_t lo, hi;
  asm("{ .reg .b16 a, b; mov.b32 {a, b}, %2; cvt.rn.bf16x2.ue8m0x2 %0, a; cvt.rn.bf16x2.ue8m0x2 %1, b; }" : "=r"(lo), "=r"(hi) : "r"(w));
  s[0] = __uint_as_float(lo << 16);
  s[1] = __uint_as_float(lo & 0xFFFF0000u);
  s[2] = __uint_as_float(hi << 16);
  s[3] = __uint_as_float(hi & 0xFFFF0000u);
}
template <int NB>
__device__ __forceinline__ void scales_of(const uint32_t* w, float (&s)[NB]) {
  if constexpr (NB == 2) {
    uint32_t lo;
    asm("{ .reg .b16 a, b; mov.b32 {a, b}, %1; cvt.rn.bf16x2.ue8m0x2 %0, a; }" : "=r"(lo) : "r"(w[0]));
    s[0] = __uint_as_float(lo << 16);
    s[1] = __uint_as_float(lo & 0xFFFF0000u);
  } else {
#pragma unroll
    for (int i = 0; i < NB; i += 4) scales4(w[i / 4], s + i);
  }
}
__device__ __forceinline__ uint32_t byte_at(const uint32_t* w, int b) { return w[b / 4] >> (8 * (b & 3)) & 0xFFu; }

// The largest byte of a word.
__device__ __forceinline__ uint32_t most_byte(uint32_t w) {
  const uint32_t m = __vmaxu2(w & 0x00FF00FFu, (w >> 8) & 0x00FF00FFu);
  return max(m & 0xFFFFu, m >> 16);
}

template <int WORDS>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t* w) {
  if constexpr (WORDS == 1) {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if constexpr (WORDS == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    w[0] = v.x, w[1] = v.y;
  } else {
#pragma unroll
    for (int i = 0; i < WORDS; i += 4) {
      const uint4 v = reinterpret_cast<const uint4*>(p)[i / 4];
      w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
    }
  }
}
// a token's NB scale bytes
template <int NB>
__device__ __forceinline__ void load_scales(const uint8_t* p, uint32_t* w) {
  if constexpr (NB == 2)
    w[0] = *reinterpret_cast<const uint16_t*>(p);
  else
    load_words<NB / 4>(p, w);
}

template <bool B>
struct Bool {
  static constexpr bool value = B;
};
// What a CTA keeps.  A warp's region is its ring of steps (the codes of 32 tokens' keys, of their values, their scales), and then what it
// hands on of its rows.
template <int NB, int NT, int RESIDENT>
struct Layout {
  static constexpr int D = 32 * NB, ROWS = 8 * NT, kPitch = D + 4;
  static constexpr int kCodes = kStep * 16 * NB, kScales = kStep * NB, kStage = 2 * (kCodes + kScales);
  static constexpr int kStages = NB == 2 ? 4 : NB == 4 ? (RESIDENT == 2 ? 4 : 3) : (RESIDENT == 3 ? 2 : 3);
  static constexpr int kHanded = ROWS * kPitch * 4;
  static constexpr int kRegion = kStages * kStage > kHanded ? kStages * kStage : kHanded;
  static constexpr int kQ = kWarps * kRegion, kMl = kQ + ROWS * D * 2, kRows = kMl + kWarps * ROWS * 8, kBytes = kRows + (kWarps + 4) * ROWS * 4;
  static_assert(kRegion % 16 == 0 && kQ % 16 == 0 && kMl % 16 == 0, "");
};

// A CTA's piece.
template <int NB, int NT, int RESIDENT>
__device__ __forceinline__ void attend(const AttnArgs& a, uint8_t* smem) {
  using L = Layout<NB, NT, RESIDENT>;
  constexpr int D = L::D, ROWS = L::ROWS, kPitch = L::kPitch, kStages = L::kStages;
  constexpr bool kKeepQ = NT * NB <= 8;                  // queries in registers
  uint2* qs = reinterpret_cast<uint2*>(smem + L::kQ);                           // [NT][NB][2][32 lanes] of four float16
  float2* mls = reinterpret_cast<float2*>(smem + L::kMl);                       // [warps][ROWS]
  float* fac = reinterpret_cast<float*>(smem + L::kRows);                       // rows: what a product of codes is times,
  int* lim = reinterpret_cast<int*>(fac + ROWS);                                // the last token seen (-1: none),
  int* low = lim + ROWS;                                                        // and the first,
  int* power = low + ROWS;                                                      // fac over the scale, as a power of two
  __shared__ int64_t scan[kWarps];
  __shared__ int found_s;
  __shared__ int64_t found_at;
  __shared__ uint64_t full_bars[kWarps][kStages];
  __shared__ int has[kWarps][kStages];                   // which halves of a step are there
  __shared__ Waits waits;

  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), g = lane >> 2, t = lane & 3;
  float* fac_step = reinterpret_cast<float*>(power + ROWS) + warp * ROWS;       // fac where a step's scales are relative to their largest
  const int hkv = a.c.hkv, cta = blockIdx.x;
  if (tid == 0) {
    for (int i = 0; i < kWarps * kStages; ++i) mbar_init(&full_bars[0][0] + i, 1);
    waits.init();
    fence_mbar_init();
  }
  if (!a.beside) pdl_wait_then_release();

  // ---- this CTA's piece of the line
  const int per = (a.seqs + kThreads - 1) / kThreads, s_from = min(tid * per, a.seqs), s_to = min(s_from + per, a.seqs);
  int64_t mine = 0;
  for (int s = s_from; s < s_to; ++s) mine += seq_at<ROWS>(a, s).cost(hkv);
  int64_t before = mine;
#pragma unroll
  for (int k = 1; k < 32; k <<= 1) {
    const int64_t v = __shfl_up_sync(0xFFFFFFFFu, before, k);
    if (lane >= k) before += v;
  }
  if (lane == 31) scan[warp] = before;
  __syncthreads();
  int64_t total = 0;
  before -= mine;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += scan[w];
    total += scan[w];
  }
  int64_t ctas = (total + kLeastPiece - 1) / kLeastPiece;
  if (ctas > gridDim.x) ctas = gridDim.x;
  // cut k of the line; the quotient first, as total * k could pass 64 bits
  const int64_t each = ctas ? total / ctas : 0, rest = ctas ? total - each * ctas : 0;
  auto cut = [&](int64_t k) { return each * k + (k < rest ? k : rest); };
  const int64_t from = cut(cta), to = cut(cta + 1);
  if (cta < ctas && mine > 0 && before <= from && from < before + mine) {
    int64_t at = before;
    for (int s = s_from; s < s_to; ++s) {
      const int64_t c = seq_at<ROWS>(a, s).cost(hkv);
      if (from < at + c) {
        found_s = s;
        found_at = from - at;
        break;
      }
      at += c;
    }
  }

  if (a.clears) clear_rows<D>(a);
  __syncthreads();
  if (tid < 2) a.plan[2 * cta + tid].last = -1;
  __syncwarp();
  if (cta >= ctas) return;

  int s = found_s;
  int64_t at = found_at;                                 // place in the sequence's part of the line
  int64_t left = to - from;
  Seq sq = seq_at<ROWS>(a, s);
  uint8_t* const ring = smem + warp * L::kRegion;
  uint64_t* const full = full_bars[warp];
  int put = 0, get = 0, flying = 0;                      // ring places, steps on their way
  uint32_t get_round = 0;
  while (left > 0) {
    while (at >= sq.cost(hkv)) {                         // the next sequence with work
      at -= sq.cost(hkv);
      sq = seq_at<ROWS>(a, ++s);
    }
    const int unit_cost = sq.steps + kUnitCost;
    const int unit = (int)(at / unit_cost), place = (int)(at - (int64_t)unit * unit_cost);
    const int rt = unit / hkv, h = unit - rt * hkv;
    const int64_t end_place = place + left < unit_cost ? place + left : unit_cost;
    const int step0 = max(place - kUnitCost, 0), step1 = max((int)end_place - kUnitCost, 0);
    const bool whole = step0 == 0 && step1 == sq.steps, starts = step0 == 0;
    if (tid == 0 && step1 > 0 && !whole) {
      // (`to` is where this piece ends on the line; a unit's parts begin with its first step)
      const int64_t end = to - left + (unit_cost - place);
      const int cta_first = starts ? cta : cta_of(end - sq.steps, each, rest), cta_last = cta_of(end - 1, each, rest);
      const int row0 = rt * ROWS, n_rows = (int)min((int64_t)ROWS, (int64_t)sq.ql * a.group - row0);
      a.plan[2 * cta + starts] = {cta_first, cta_last, sq.begin, h, row0, n_rows};
    }
    left -= end_place - place;
    at += end_place - place;
    if (starts && step1 == 0) continue;                  // (only the unit's beginning: the next CTA has its first step)
    const int slot = 2 * cta + (starts ? 1 : 0);

    const int t_base = (int)(sq.first / kStep) * kStep, t_end = (int)sq.end;
    const int32_t* pages = a.table + (int64_t)s * a.width;
    const uint8_t* head = a.c.base + (int64_t)h * a.c.part;
    const int64_t page_bytes = 2 * a.c.hkv * a.c.part, to_v = a.c.hkv * a.c.part;
    const int page = a.c.page;
    auto page_of = [&](int tk, bool in) {                // -1: none
      if (!in || tk >= t_end) return -1;
      const int pg = __ldg(pages + (tk >> a.c.page_log));
      return pg < 0 || pg >= a.pages ? -1 : pg;
    };
    // The step at token tk into the ring, if it is one of this piece's; the pages of the one after are looked up.
    int pg0 = page_of(t_base + kStep * (step0 + warp), step0 + warp < step1);
    int pg1 = page_of(t_base + kStep * (step0 + warp) + 16, step0 + warp < step1);
    auto issue = [&](int st, int tk) {
      if (st < step1) {
        if (elect_one()) {
          uint8_t* to = ring + put * L::kStage;
          has[warp][put] = (pg0 >= 0 ? 1 : 0) | (pg1 >= 0 ? 2 : 0);
          const bool together = page >= kStep && pg0 >= 0 && pg1 >= 0;
          mbar_arrive_expect_tx(&full[put], (uint32_t)((pg0 >= 0) + (pg1 >= 0)) * (L::kStage / 2));
#pragma unroll 1
          for (int half = 0; half < (together ? 1 : 2); ++half) {
            const int pg = half ? pg1 : pg0, n = together ? kStep : kStep / 2, o = half * (kStep / 2);
            if (pg < 0) continue;
            const uint8_t* k = head + pg * page_bytes;
            const int r = (tk + o) & (page - 1);
            const uint8_t* sc = k + (page * 16 + r) * NB;
            k += r * (16 * NB);
            bulk_load(to + o * (16 * NB), k, n * 16 * NB, &full[put]);
            bulk_load(to + 2 * L::kCodes + o * NB, sc, n * NB, &full[put]);
            bulk_load(to + L::kCodes + o * (16 * NB), k + to_v, n * 16 * NB, &full[put]);
            bulk_load(to + 2 * L::kCodes + L::kScales + o * NB, sc + to_v, n * NB, &full[put]);
          }
        }
        if (++put == kStages) put = 0;
        ++flying;
        pg0 = page_of(tk + kAhead, st + kWarps < step1);
        pg1 = page_of(tk + kAhead + 16, st + kWarps < step1);
      }
    };
    int step = step0 + warp, tok = t_base + kStep * step;
    fence_proxy_async_smem();                            // (the region was written and read otherwise)
    __syncthreads();                                     // the unit before has been handed on
#pragma unroll 1
    for (int i = 0; i < kStages - 1; ++i) issue(step + i * kWarps, tok + i * kAhead);

    // ---- queries to float16, in the order of the operand
    const int rows = min(ROWS, sq.ql * a.group - rt * ROWS);
    constexpr int kPer = NB, kMine = ROWS / kWarps;      // channels a lane: D / 32; rows a warp, all on their way at once
    uint32_t q_raw[kMine][kPer / 2];
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
      const int r = warp + k * kWarps, rr = rt * ROWS + r, j = rr / a.group;
      const __nv_bfloat16* p = a.q + ((int64_t)(sq.begin + j) * a.hq + h * a.group + (rr - j * a.group)) * D + lane * kPer;
#pragma unroll
      for (int i = 0; i < kPer / 2; ++i) q_raw[k][i] = r < rows ? reinterpret_cast<const uint32_t*>(p)[i] : 0u;
    }
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
      const int r = warp + k * kWarps, j = (rt * ROWS + r) / a.group;
      float x[kPer];
      float amax = 0.f;
#pragma unroll
      for (int i = 0; i < kPer; i += 2) {
        x[i] = __uint_as_float(q_raw[k][i / 2] << 16);
        x[i + 1] = __uint_as_float(q_raw[k][i / 2] & 0xFFFF0000u);
      }
#pragma unroll
      for (int i = 0; i < kPer; ++i) amax = fmaxf(amax, __uint_as_float(min(__float_as_uint(x[i]) & 0x7FFFFFFFu, 0x7F800000u)));
      const uint32_t largest = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(amax));
      const int e = largest ? max((int)(largest >> 23), 1) : 127;
      const float up = e >= 254 ? 0x1p-127f : __uint_as_float((uint32_t)(254 - e) << 23);      // 2^(127 - e)
      uint32_t w[kPer / 2];
#pragma unroll
      for (int i = 0; i < kPer; i += 2) w[i / 2] = e == 255 ? 0x7FFF7FFFu : f16_pair(x[i] * up * 0x1p13f, x[i + 1] * up * 0x1p13f);
      // channel c: block c / 32, lane's t = c % 32 / 8, then two halves u of four
#pragma unroll
      for (int i = 0; i < kPer; i += 2) {
        const int c = lane * kPer + i, b = c / 32, tt = c % 32 / 8, u = c % 8 / 4, two = c % 4 / 2;
        reinterpret_cast<uint32_t*>(qs + (((r / 8) * NB + b) * 2 + u) * 32 + (r & 7) * 4 + tt)[two] = w[i / 2];
      }
      if (lane == 0) {
        const int64_t p = sq.len - sq.ql + j;
        fac[r] = ldexpf(a.scale, e - 140);
        power[r] = e - 140;
        lim[r] = r < rows ? (int)(p < sq.end - 1 ? p : sq.end - 1) : -1;
        low[r] = a.window && p - a.window + 1 > 0 ? (int)(p - a.window + 1) : 0;
      }
    }
    __syncthreads();

    uint2 qf[kKeepQ ? NT : 1][NB][2];
    if constexpr (kKeepQ) {
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int u = 0; u < 2; ++u) qf[j][b][u] = qs[((j * NB + b) * 2 + u) * 32 + lane];
    }
    // A score, codes' product times fac, less its row's `base` is what the exponential takes: base = m - (136 - ref), the weights times 2^(136 - ref), so
    // that with a value's scale, 2^(byte - 127) of a byte up to ref, they are at most 2^(9 + kSlack).  (A reference outside kLowR .. kHighR: the
    // nearest one that is within, and `adjust` for the rest.)
    float f[NT][2], m[NT][2], base[NT][2], l[NT][2], acc[NB][2][NT][4];
    bool odd_unit = false;                               // (uniform) what `steps` below goes on with in its other form
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f[j][i] = fac[8 * j + 2 * t + i];
        odd_unit |= !(fabsf(f[j][i]) < 0x1p100f);
        base[j][i] = m[j][i] = kNone;
        l[j][i] = 0.f;
      }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int k = 0; k < 4; ++k) acc[b][i][j][k] = 0.f;
    odd_unit = __any_sync(0xFFFFFFFFu, odd_unit);
    int ref = -1;                                        // largest scale byte of values so far,
    int sure = -1;                                       // and one that all rows have seen
    float most = kSlack + (float)(136 - within(-1));     // what a score may exceed its base by
    // tokens that all rows see
    const int64_t p_first = sq.len - sq.ql + (rt * ROWS) / a.group, p_last = sq.len - sq.ql + (rt * ROWS + rows - 1) / a.group;
    const int all_to = (int)(p_first < sq.end - 1 ? p_first : sq.end - 1);
    const int all_from = a.window && p_last - a.window + 1 > 0 ? (int)(p_last - a.window + 1) : 0;
    const int sure_to = max(all_to, 0);                  // (rows before a sequence's beginning see nothing)
    odd_unit |= all_from > sure_to;
    // and that some row sees
    const int some_to = (int)(p_last < sq.end - 1 ? p_last : sq.end - 1);
    const int some_from = a.window && p_first - a.window + 1 > 0 ? (int)(p_first - a.window + 1) : 0;

    // The steps that are left.  What is out of the ordinary has a copy of the code of its own, in which a warp does the rest of a unit (true:
    // it is to go on there), and costs the other next to nothing (2 to 12 % where one code looked out for all of it):
    // keys' scales of 2^65 and more, factors far from one, scores of more than 2^16 (a sum of codes times scales is at most 2^27 times
    // the largest scale, and its row's factor comes after it: scales are taken relative to the largest of those that some row sees, and a
    // score is rounded to float32 before its maximum is taken off); values of NaN scales, of references that are not within kLowR ..
    // kHighR, and of tokens that some rows see and others do not and that are larger than all that these see: a reference a row.
    bool issued = false, large = false;
    int refs[NT][2];                                     // a reference a row, in that form
    auto adjust = [](int r) { return r < 0 ? 1.f : __uint_as_float((uint32_t)(127 + within(r) - r) << 23); };
    // A row's sums, relative to another reference.
    auto follow = [&](int j, int i, float by, float by_l) {
      l[j][i] *= by_l;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          acc[b][c][j][i] *= by;
          acc[b][c][j][2 + i] *= by;
        }
    };
    auto steps = [&](auto odd_form) -> bool {
      constexpr bool kOdd = decltype(odd_form)::value;
      for (; step < step1; step += kWarps, tok += kAhead) {
        if (!issued) issue(step + (kStages - 1) * kWarps, tok + (kStages - 1) * kAhead);
        issued = false;
        if (!__all_sync(0xFFFFFFFFu, short_wait<false, true>(&full[get], get_round & 1, &waits, __LINE__))) return false;
        const uint8_t* st = ring + get * L::kStage;
        const int here = has[warp][get];
        uint32_t own[(NB + 3) / 4], own_k[(NB + 3) / 4], high = 0u;      // a token's values' and keys' scales; keys' of 2^65 and more
        load_scales<NB>(st + 2 * L::kCodes + L::kScales + lane * NB, own);
        load_scales<NB>(st + 2 * L::kCodes + lane * NB, own_k);
        if (!(here >> (lane >> 4) & 1))
#pragma unroll
          for (int i = 0; i < (NB + 3) / 4; ++i) own[i] = own_k[i] = 0u;
#pragma unroll
        for (int i = 0; i < (NB + 3) / 4; ++i) high |= own_k[i] & (own_k[i] << 1) & 0x80808080u;

        float down = 1.f;                                  // (kOdd) the power of two that the keys' scales are multiplied by
        if constexpr (kOdd) {
          uint32_t real = 0;                               // (NaN's 255 is none, nor is what no row sees)
          if (tok + lane >= some_from && tok + lane <= some_to)
#pragma unroll
            for (int b = 0; b < NB; ++b)
              if (byte_at(own_k, b) != 255u) real = max(real, byte_at(own_k, b));
          const int kr = (int)__reduce_max_sync(0xFFFFFFFFu, real);
          down = kr == 254 ? 0x1p-127f : __uint_as_float((uint32_t)(254 - kr) << 23);
          __syncwarp();
          if (lane < ROWS) fac_step[lane] = fminf(fmaxf(ldexpf(a.scale, power[lane] + kr - 127), -kMost), kMost);
          __syncwarp();
        }

        // ---- the values' reference
        bool nan = false;
        uint32_t big = most_byte(own[0]);
        if constexpr (NB == 8) big = max(big, most_byte(own[NB / 4 - 1]));
        if (__any_sync(0xFFFFFFFFu, (int)big > (sure < 0 ? -1 : ref) || (!kOdd && high))) {
          int real = -1;                                   // NaN's 255 is none, nor is what no row sees, which may be anything
          if (tok + lane >= some_from && tok + lane <= some_to && (here >> (lane >> 4) & 1))
#pragma unroll
            for (int b = 0; b < NB; ++b)
              if (byte_at(own, b) != 255u) real = max(real, (int)byte_at(own, b));
          const int now = __reduce_max_sync(0xFFFFFFFFu, real), top = max(now, ref);
          if constexpr (!kOdd) {
            int all = now;
            if (tok < all_from || tok + kStep - 1 > all_to)
              all = __reduce_max_sync(0xFFFFFFFFu, tok + lane >= all_from && tok + lane <= sure_to ? real : -1);
            sure = max(sure, all);
            if (__any_sync(0xFFFFFFFFu, high || big == 255u) || (sure >= 0 && top > sure + kBeyond) || (top >= 0 && top != within(top))) {
              issued = true;
              return true;
            }
            const float by = ex2((float)(ref - top));
            ref = top;
            most = kSlack + (float)(136 - within(ref));
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                base[j][i] = m[j][i] - (float)(136 - within(ref));
                follow(j, i, by, by);
              }
          } else {
            nan = __any_sync(0xFFFFFFFFu, big == 255u);
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const int r = 8 * j + k, own_top = __reduce_max_sync(0xFFFFFFFFu, tok + lane >= low[r] && tok + lane <= lim[r] ? real : -1);
                if (k / 2 == t) {
                  const int was = refs[j][k & 1], need = max(was, own_top), to = now <= need + kBeyond ? max(now, was) : need;
                  refs[j][k & 1] = to;
                  follow(j, k & 1, ex2((float)(was - to)), ex2((float)(within(was) - within(to))));
                }
              }
          }
        }

#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (!(here >> half & 1)) continue;
          const int t0 = tok + 16 * half;
          const uint8_t* kc = st + (16 * half + g) * (16 * NB) + t * (4 * NB);
          const uint8_t* ks = st + 2 * L::kCodes + (16 * half + g) * NB;
          const uint8_t* vc = st + L::kCodes + (16 * half + 2 * t) * (16 * NB) + g * (2 * NB);

          // ---- scores
          float x[NT][4];
          {
            float s0[NB], s1[NB];
            uint32_t w0[(NB + 3) / 4], w1[(NB + 3) / 4], k0[NB], k1[NB];
            load_scales<NB>(ks, w0);
            load_scales<NB>(ks + 8 * NB, w1);
            load_words<NB>(kc, k0);
            load_words<NB>(kc + 8 * 16 * NB, k1);
            scales_of<NB>(w0, s0);
            scales_of<NB>(w1, s1);
            if constexpr (kOdd)
#pragma unroll
              for (int b = 0; b < NB; ++b) s0[b] *= down, s1[b] *= down;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
              const uint32_t lo[4] = {code_pair<0>(k0[b]), code_pair<0>(k1[b]), code_pair<1>(k0[b]), code_pair<1>(k1[b])};
              const uint32_t hi[4] = {code_pair<2>(k0[b]), code_pair<2>(k1[b]), code_pair<3>(k0[b]), code_pair<3>(k1[b])};
#pragma unroll
              for (int j = 0; j < NT; ++j) {
                const uint2 q0 = kKeepQ ? qf[kKeepQ ? j : 0][b][0] : qs[((j * NB + b) * 2) * 32 + lane];
                const uint2 q1 = kKeepQ ? qf[kKeepQ ? j : 0][b][1] : qs[((j * NB + b) * 2 + 1) * 32 + lane];
                float part[4];
                mma_first(part, lo, q0.x, q0.y);
                mma(part, hi, q1.x, q1.y);
                if (b == 0) {
                  x[j][0] = part[0] * s0[0], x[j][1] = part[1] * s0[0], x[j][2] = part[2] * s1[0], x[j][3] = part[3] * s1[0];
                } else {
                  x[j][0] = fmaf(part[0], s0[b], x[j][0]), x[j][1] = fmaf(part[1], s0[b], x[j][1]);
                  x[j][2] = fmaf(part[2], s1[b], x[j][2]), x[j][3] = fmaf(part[3], s1[b], x[j][3]);
                }
              }
            }
          }
          const bool partial = t0 + 15 > all_to || t0 < all_from;
          auto hidden = [&](int j, int k) {
            const int at_tok = t0 + g + 8 * (k >> 1), r = 8 * j + 2 * t + (k & 1);
            return at_tok > lim[r] || at_tok < low[r];
          };
          float e[NT][4], top = kNone;
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              if constexpr (kOdd) {                        // (rounded before the maximum is taken off, and that before what the base has beside it)
                x[j][k] *= fac_step[8 * j + 2 * t + (k & 1)];
                e[j][k] = x[j][k] - m[j][k & 1];
              } else {
                e[j][k] = fmaf(x[j][k], f[j][k & 1], -base[j][k & 1]);
              }
              if (partial && hidden(j, k)) e[j][k] = __int_as_float(0xFF800000);
              top = fmaxf(top, e[j][k]);
            }

          // ---- running maxima
          if (__any_sync(0xFFFFFFFFu, top > (kOdd ? kSlack : most) || (!kOdd && large))) {
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                // (rounded here: what a product keeps beyond float32 would be a large difference of large scores)
                if constexpr (!kOdd) x[j][i] *= f[j][i], x[j][2 + i] *= f[j][i];
                const float lo = partial && hidden(j, i) ? kNone : x[j][i];
                const float hi = partial && hidden(j, 2 + i) ? kNone : x[j][2 + i];
                float up = fmaxf(lo, hi);
#pragma unroll
                for (int k = 4; k < 32; k <<= 1) up = fmaxf(up, __shfl_xor_sync(0xFFFFFFFFu, up, k));
                up = fmaxf(up, m[j][i]);
                const float by = ex2(m[j][i] - up);
                if constexpr (!kOdd) large |= __any_sync(0xFFFFFFFFu, fabsf(up) > 0x1p16f && up != kNone);
                m[j][i] = up;
                if constexpr (!kOdd) base[j][i] = up - (float)(136 - within(ref));
                l[j][i] *= by;
#pragma unroll
                for (int k = i; k < 4; k += 2)
                  if (!(partial && hidden(j, k))) e[j][k] = (x[j][k] - up) + (kOdd ? 0.f : (float)(136 - within(ref)));
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                  for (int c = 0; c < 2; ++c) {
                    acc[b][c][j][i] *= by;
                    acc[b][c][j][2 + i] *= by;
                  }
              }
          }
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              if constexpr (kOdd) e[j][k] += (float)(136 - within(refs[j][k & 1]));
              x[j][k] = ex2(e[j][k]);
              if constexpr (kOdd)
                if (e[j][k] == __int_as_float(0xFF800000)) x[j][k] = -0.f;       // (not seen: told from weights below float32)
              l[j][k & 1] += x[j][k];
            }

          // ---- values
          float s0[NB], s1[NB];
          uint32_t w0[(NB + 3) / 4], w1[(NB + 3) / 4], v[4][NB / 2];
          load_scales<NB>(ks + L::kScales, w0);
          load_scales<NB>(ks + L::kScales + 8 * NB, w1);
#pragma unroll
          for (int i = 0; i < 4; ++i) load_words<NB / 2>(vc + ((i & 1) + 8 * (i >> 1)) * (16 * NB), v[i]);
          scales_of<NB>(w0, s0);
          scales_of<NB>(w1, s1);
#pragma unroll
          for (int i = 0; i < NB / 2; ++i) {
            // even and odd channels of pairs of tokens: nibbles side by side
            uint32_t ev[2], ov[2];
#pragma unroll
            for (int h2 = 0; h2 < 2; ++h2) {
              const uint32_t A = v[2 * h2][i], B = v[2 * h2 + 1][i];
              ev[h2] = (A & 0x0F0F0F0Fu) | ((B << 4) & 0xF0F0F0F0u);
              ov[h2] = ((A >> 4) & 0x0F0F0F0Fu) | (B & 0xF0F0F0F0u);
            }
            const uint32_t va[4][4] = {{code_pair<0>(ev[0]), code_pair<0>(ov[0]), code_pair<0>(ev[1]), code_pair<0>(ov[1])},
                                       {code_pair<1>(ev[0]), code_pair<1>(ov[0]), code_pair<1>(ev[1]), code_pair<1>(ov[1])},
                                       {code_pair<2>(ev[0]), code_pair<2>(ov[0]), code_pair<2>(ev[1]), code_pair<2>(ov[1])},
                                       {code_pair<3>(ev[0]), code_pair<3>(ov[0]), code_pair<3>(ev[1]), code_pair<3>(ov[1])}};
#pragma unroll
            for (int o = 0; o < 2; ++o) {
              const int b = 2 * i + o;
#pragma unroll
              for (int j = 0; j < NT; ++j) {
                float w[4] = {x[j][0] * s0[b], x[j][1] * s0[b], x[j][2] * s1[b], x[j][3] * s1[b]};
                if constexpr (kOdd)
#pragma unroll
                  for (int k = 0; k < 4; ++k) w[k] *= adjust(refs[j][k & 1]);
                if (kOdd && nan) {                         // a NaN scale counts for rows that see its token only
#pragma unroll
                  for (int k = 0; k < 4; ++k)
                    if (__float_as_uint(x[j][k]) == 0x80000000u) w[k] = 0.f;
                }
                const uint32_t p0 = transpose(f16_pair(w[0], w[1])), p1 = transpose(f16_pair(w[2], w[3]));
                mma(acc[b][0][j], va[2 * o], p0, p1);
                mma(acc[b][1][j], va[2 * o + 1], p0, p1);
              }
            }
          }
        }
        __syncwarp();                                      // all lanes have read the step
        --flying;
        if (++get == kStages) {
          get = 0;
          ++get_round;
        }
        if (!kOdd && large) {
          step += kWarps, tok += kAhead;
          return true;
        }
      }
      return false;
    };
    if (!odd_unit) odd_unit = steps(Bool<false>());
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) refs[j][i] = odd_unit && low[8 * j + 2 * t + i] >= tok ? -1 : ref;      // (none yet: nothing seen)
    if (odd_unit) steps(Bool<true>());
    if (waits.abort) {                                   // a wait gave up: the copies still on their way, then out
      volatile int none = 0;
      for (; flying > 0; --flying) {
        mbar_wait_bounded(&full[get], get_round & 1, &none);
        if (++get == kStages) {
          get = 0;
          ++get_round;
        }
      }
    }
    __syncthreads();                                     // (the warps' last reads of their rings, too)
    if (waits.abort) {
      if (tid == 0) report(a.status, timeout_bits(kWhereMxAttention, waits.abort));
      return;
    }

    if (odd_unit) {
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) follow(j, i, 1.f / adjust(refs[j][i]), 1.f);
    }
    // ---- the warps' parts together: means of values each, as everywhere from here on (sums of many large values could leave float32)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int k = 4; k < 32; k <<= 1) l[j][i] += __shfl_xor_sync(0xFFFFFFFFu, l[j][i], k);
        const float by = l[j][i] == 0.f ? 0.f : __fdividef(1.f, l[j][i]);
        if (g == 0) mls[warp * ROWS + 8 * j + 2 * t + i] = make_float2(m[j][i], l[j][i] * ex2((float)(within(refs[j][i]) - 136)));
        float* o = reinterpret_cast<float*>(smem + warp * L::kRegion) + (8 * j + 2 * t + i) * kPitch;
#pragma unroll
        for (int b = 0; b < NB; ++b)
          *reinterpret_cast<float4*>(o + 32 * b + 4 * g) = make_float4(acc[b][0][j][i] * by, acc[b][0][j][2 + i] * by,
                                                                       acc[b][1][j][i] * by, acc[b][1][j][2 + i] * by);
      }
    __syncthreads();
    for (int i = tid; i < rows * (D / 4); i += kThreads) {
      const int r = i / (D / 4), c = i - r * (D / 4);
      float top = mls[r].x, sum = 0.f, share[kWarps];
#pragma unroll
      for (int w = 1; w < kWarps; ++w) top = fmaxf(top, mls[w * ROWS + r].x);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float2 ml = mls[w * ROWS + r];
        share[w] = ml.y * ex2(ml.x - top);
        sum += share[w];
      }
      const float inv = sum == 0.f ? 0.f : __fdividef(1.f, sum);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float by = share[w] * inv;
        const float4 v = *reinterpret_cast<const float4*>(smem + w * L::kRegion + (r * kPitch + 4 * c) * 4);
        o.x = fmaf(v.x, by, o.x), o.y = fmaf(v.y, by, o.y), o.z = fmaf(v.z, by, o.z), o.w = fmaf(v.w, by, o.w);
      }
      if (whole) {
        const int rr = rt * ROWS + r, j = rr / a.group;
        const int64_t to_row = ((int64_t)(sq.begin + j) * a.hq + h * a.group + (rr - j * a.group)) * D + 4 * c;
        store4(a, to_row, o);
      } else {
        *reinterpret_cast<float4*>(a.parts + ((int64_t)slot * ROWS + r) * D + 4 * c) = o;
        if (c == 0) *reinterpret_cast<float2*>(a.ml + ((int64_t)slot * ROWS + r) * 2) = make_float2(top, sum);
      }
    }
  }
}

// Beside the tiles of the same call (which have waited for what was before them, and share nothing with this) it waits for them at its
// end, so that what comes after it comes after both: 16 sequences of 5 drafted tokens, where the tiles have nothing to do, 54 us
// instead of 57.  Where the tiles have work, their shared memory leaves no room for this kernel's CTAs, which start on an SM when its
// tiles' CTA leaves: 64 sequences of 4000 tokens beside 2048 rows over 8192, 430 us, apart 79 and 284.
template <int NB, int NT, int RESIDENT>
__global__ void __launch_bounds__(kThreads, RESIDENT) mx_attention_kernel(const __grid_constant__ AttnArgs a) {
  extern __shared__ __align__(128) uint8_t smem[];
  attend<NB, NT, RESIDENT>(a, smem);
  if (a.beside) asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Tiles of 8 rows that the units of sequences of few rows have, and CTAs an SM: by what a warp keeps in registers.
struct Form {
  int nt, resident;
};
Form form_of(int64_t n, int64_t seqs, int64_t group, int64_t d) {
  // Of a sequence, on average, the tiles' among them, as the host does not know which those are: beside a long chunk, sequences of one row
  // go by the form for 24 (63 of them and 2048 rows, 64 / 8 heads: 673 us, apart 79 and 532).
  const int64_t rows = (n + seqs - 1) / seqs * group;
  const int nt = rows <= 8 ? 1 : rows <= 16 || d == 256 ? 2 : 3;
  return {nt, nt * d <= 128 ? 4 : nt * d <= 256 ? 3 : 2};
}

// Which kernels a call takes.  Both can do any number of rows.  With no more rows than sequences (a decode step, whatever its offsets),
// and where rows and the tokens that a table's width has room for are few, the first does all (tiles have a longer way from a unit's
// beginning to its end: 48 rows a key head over 100 tokens 19 us against 24, 192 over 2000 30 against 41; 384 over 2000 42 against 35);
// with one sequence or many heads on a key head it is known which is the better one for all, and else either leaves the other's sequences out.
constexpr int64_t kFewWork = int64_t(1) << 22;           // rows of all heads times tokens
struct Needs {
  int most;                                 // rows of a sequence and key head up to which the first kernel is the faster
  bool few, tiles;
  Needs(int64_t n, int64_t seqs, int64_t hq, int64_t hkv, int64_t d, int64_t room) : most(d == 256 ? 16 : 24) {
    const int64_t group = hq / hkv;
    tiles = (group > most || (n > seqs && n * group > most)) && (double)(n * hq) * (double)room > (double)kFewWork;
    few = !tiles || (group <= most && seqs > 1);
  }
  int most_few() const { return few ? tiles ? most : 0x7FFFFFFF : 0; }
};

// With the tiles' launch before it, where there is one, and the joining of both's parts.
template <int NB, int NT, int RESIDENT, int TILE_ROWS = NB == 8 ? 128 : 256>
cudaError_t run(const AttnArgs& a, int grid, const AttnArgs& tiles, int tile_grid, cudaStream_t stream) {
  static PerDevice<cudaError_t> allowed;
  constexpr int kSmem = Layout<NB, NT, RESIDENT>::kBytes;
  cudaError_t e = allowed.get([] { return allow_smem(mx_attention_kernel<NB, NT, RESIDENT>, kSmem); });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr = pdl_attr();
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  note_launch();
  if ((e = cudaLaunchKernelEx(&cfg, mx_attention_kernel<NB, NT, RESIDENT>, a)) != cudaSuccess) return e;
  // Launched when all is done: CTAs that wait beside this kernel's, 2 to 4 an SM, are in the way of the next call's, which then come
  // to lie unevenly (64 sequences of up to 8192 tokens in a row of calls: 98 us each, against 83 as it was then).
  note_launch();
  const int entries = 2 * grid;
  if (!tile_grid) {
    cfg = join_config(entries, stream);
    return cudaLaunchKernelEx(&cfg, mx_attention_join_kernel<32 * NB, 8 * NT>, a);
  }
  cfg = join_config(entries + 2 * tile_grid * join_split(TILE_ROWS), stream);
  return cudaLaunchKernelEx(&cfg, mx_attention_join_both_kernel<32 * NB, 8 * NT, TILE_ROWS>, a, entries, tiles);
}

int sm_count() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return -1;
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms <= 0) return -1;
  return sms;
}

}  // namespace

cudaError_t set_attention_wait_limit(uint64_t ns) { return cudaMemcpyToSymbol(g_wait_limit, &ns, sizeof(ns)); }

int64_t mx_attention_workspace(int64_t n, int64_t seqs, int64_t hq, int64_t hkv, int64_t d) {
  if (seqs == 0) return 0;
  const int sms = sm_count();
  if (sms < 0) return -1;
  const int64_t group = hq / hkv;
  const Form f = form_of(n, seqs, group, d);
  const Needs needs(n, seqs, hq, hkv, d, INT64_MAX);       // (a table with little room may need the first's alone)
  const size_t few = Parts((size_t)sms * f.resident, 8 * f.nt, d).bytes, tiles = needs.tiles ? Parts(sms, attention_tile_rows(d), d).bytes : 0;
  return (int64_t)(needs.few ? few + tiles : std::max(few, tiles));
}

cudaError_t launch_mx_attention(const void* q, int64_t n, int64_t hq, const uint8_t* cache, int64_t pages, int64_t page, int64_t hkv,
                                int64_t d, const int32_t* table, int64_t width, const int32_t* lens, int64_t seqs,
                                const int32_t* offsets, float scale, int64_t window, int out_dtype, void* out, void* workspace,
                                uint32_t* status, cudaStream_t stream) {
  if (seqs == 0) return cudaMemsetAsync(out, 0, (size_t)n * hq * d * (out_dtype == 0 ? 4 : 2), stream);
  const int sms = sm_count();
  if (sms < 0) return cudaErrorInvalidDevice;
  AttnArgs a = {};
  int log = 0;
  while ((int64_t(1) << log) < page) ++log;
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.c = {const_cast<uint8_t*>(cache), pages * page, (int)page, log, (int)hkv, mx_page_bytes(page, d)};
  a.pages = pages, a.table = table, a.lens = lens, a.offsets = offsets, a.width = width;
  a.n = (int)n, a.hq = (int)hq, a.group = (int)(hq / hkv), a.seqs = (int)seqs;
  a.scale = std::min(std::max(scale * 1.44269504f, -kMost), kMost);
  a.status = status, a.window = window, a.out = out, a.out_f32 = out_dtype == 0;
  const Form f = form_of(n, seqs, a.group, d);
  const Needs needs(n, seqs, hq, hkv, d, width * page);
  a.few = needs.most_few();
  const Parts parts((size_t)sms * f.resident, 8 * f.nt, d), tiles(sms, attention_tile_rows(d), d);
  a.clears = 1;
  AttnArgs t = a;
  tiles.place(&t, workspace);
  if (needs.tiles) {
    const cudaError_t e = launch_attention_tiles(t, d, sms, !needs.few, stream);
    if (e != cudaSuccess || !needs.few) return e;
    workspace = static_cast<uint8_t*>(workspace) + tiles.bytes;
    a.clears = 0, a.beside = 1;
  }
  parts.place(&a, workspace);
  const int grid = sms * f.resident, tg = needs.tiles ? sms : 0;
  if (d == 64) return f.nt == 1 ? run<2, 1, 4>(a, grid, t, tg, stream) : f.nt == 2 ? run<2, 2, 4>(a, grid, t, tg, stream) : run<2, 3, 3>(a, grid, t, tg, stream);
  if (d == 128) return f.nt == 1 ? run<4, 1, 4>(a, grid, t, tg, stream) : f.nt == 2 ? run<4, 2, 3>(a, grid, t, tg, stream) : run<4, 3, 2>(a, grid, t, tg, stream);
  return f.nt == 1 ? run<8, 1, 3>(a, grid, t, tg, stream) : run<8, 2, 2>(a, grid, t, tg, stream);
}

}  // namespace cat
