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
// ~2.9 lane instructions a code in the time its bytes take from memory, and the unpacking is most of what there is to do.
// Codes go from memory to registers in the layout of the matrix instructions' operands (which is what the cache's pieces are for) and
// are unpacked in pairs there.  tcgen05 would want them unpacked into shared memory first, for 128 rows where there are 1 to 32.
//
//   S^T [16 tokens x 8 rows] = K Q^T:  a lane (g, t) = (lane / 4, lane % 4) has channels 8 t .. 8 t + 7 of every block of tokens g, g + 8
//   O^T [16 channels x 8 rows] = V^T P^T: channels 4 g .. 4 g + 3 of every block of tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9
// Scores leave with lane (g, t) having tokens g, g + 8 of rows 2 t, 2 t + 1; times the values' scales of its tokens they are
// turned to the second product's operand by movmatrix.
//
// Work is cut evenly, whatever the lengths: units (sequence, row tile, head) lie one behind the other on a line of 16-token steps, and
// each CTA has an equal piece of it, found from the lengths on the device.  A unit in one piece is written at once; the others'
// parts go through the workspace, and a second kernel joins them in the order of their tokens.
#include <cuda_fp16.h>

#include "mx_cache.cuh"
#include "per_device.h"

namespace cat {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kUnitCost = 4;                // a unit's beginning and end, in steps
constexpr int kLeastPiece = 8;              // steps a CTA is worth
constexpr float kSlack = 6.f;               // a row's scores may exceed its running maximum by this (binary orders) before it follows
constexpr int kLowR = 40;                   // least reference exponent of the values (below it they count less bits)

// A CTA's piece that begins a unit which others go on with.
struct Plan {
  int s, h, rt, last;                       // last: the last CTA with a part of it; -1: none
};

struct AttnArgs {
  const __nv_bfloat16* q;
  MxCache c;
  int64_t pages;
  const int32_t *table, *lens, *offsets;
  int64_t width;
  int n, hq, group, seqs;
  float scale;                              // scale log2 e
  int64_t window;
  void* out;
  int out_f32;
  float *parts, *ml;                        // [2 grid][rows][D], [2 grid][rows][2]
  Plan* plan;
};

struct Seq {
  int begin, ql, steps, tiles;              // first row, rows, 16-token steps and row tiles
  int64_t len, first, end;                  // tokens; the first a row sees; one past the last in the cache
  __device__ __forceinline__ int64_t cost(int hkv) const { return steps ? (int64_t)tiles * hkv * (steps + kUnitCost) : 0; }
};

template <int ROWS>
__device__ __forceinline__ Seq seq_at(const AttnArgs& a, int s) {
  Seq q;
  int end;
  if (a.offsets) {
    q.begin = min(max(a.offsets[s], 0), a.n);
    end = min(max(a.offsets[s + 1], q.begin), a.n);
  } else {
    q.begin = s;
    end = s + 1;
  }
  q.ql = end - q.begin;
  q.len = a.lens[s];
  const int64_t cap = a.width << a.c.page_log, p = q.len - q.ql;
  q.end = q.len < cap ? q.len : cap;
  q.first = a.window && p - a.window + 1 > 0 ? p - a.window + 1 : 0;
  q.steps = q.ql > 0 && q.end > q.first ? (int)((q.end + 15) / 16 - q.first / 16) : 0;
  q.tiles = (int)(((int64_t)q.ql * a.group + ROWS - 1) / ROWS);
  return q;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 16 x 8 += 16 x 16 times 16 x 8, float16 operands
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// The float16 values of a byte's two codes, the first in the low half (byte i of w).
template <int I>
__device__ __forceinline__ uint32_t code_pair(uint32_t w) {
  uint32_t r;
  asm("{ .reg .b8 a, b, c, d; mov.b32 {a, b, c, d}, %1; cvt.rn.f16x2.e2m1x2 %0, a; }" : "=r"(r) : "r"(I ? w >> (8 * I) : w));
  return r;
}
__device__ __forceinline__ uint32_t f16_pair(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// 2^(byte - 127) of byte i of w; 0 for a byte of 0 and infinity for 255.
template <int I>
__device__ __forceinline__ float byte_scale(uint32_t w) {
  return __uint_as_float((I < 3 ? w << (23 - 8 * I) : w >> 1) & 0x7F800000u);
}
__device__ __forceinline__ float byte_scale_at(const uint32_t* w, int b) {
  switch (b & 3) {
    case 0: return byte_scale<0>(w[b / 4]);
    case 1: return byte_scale<1>(w[b / 4]);
    case 2: return byte_scale<2>(w[b / 4]);
    default: return byte_scale<3>(w[b / 4]);
  }
}
__device__ __forceinline__ uint32_t byte_at(const uint32_t* w, int b) { return w[b / 4] >> (8 * (b & 3)) & 0xFFu; }

// The largest byte of two words.
__device__ __forceinline__ uint32_t most_byte(uint32_t a, uint32_t b) {
  const uint32_t m = __vmaxu2(__vmaxu2(a & 0x00FF00FFu, (a >> 8) & 0x00FF00FFu), __vmaxu2(b & 0x00FF00FFu, (b >> 8) & 0x00FF00FFu));
  return max(m & 0xFFFFu, m >> 16);
}

template <int WORDS>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t* w) {
  if constexpr (WORDS == 1) {
    asm("ld.global.nc.L1::no_allocate.b32 %0, [%1];" : "=r"(w[0]) : "l"(p));
  } else if constexpr (WORDS == 2) {
    asm("ld.global.nc.L1::no_allocate.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
  } else {
#pragma unroll
    for (int i = 0; i < WORDS; i += 4)
      asm("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];"
          : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3])
          : "l"(p + 4 * i));
  }
}

// A lane's part of 16 tokens, as it is in the cache.
template <int NB>
struct Step {
  static constexpr int kScaleWords = (NB + 3) / 4;
  uint32_t k[2][NB], v[4][NB / 2], ks[2][kScaleWords], vs[2][kScaleWords];
  // r: the first token's place in its page
  __device__ __forceinline__ void load(const uint8_t* kp, const uint8_t* vp, int page, int r, int g, int t) {
    constexpr int kRow = 16 * NB;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      load_words<NB>(kp + (r + g + 8 * i) * kRow + t * (4 * NB), k[i]);
      const int sc = page * kRow + (r + g + 8 * i) * NB;
      if constexpr (NB == 2) {
        uint16_t a, b;
        asm("ld.global.nc.b16 %0, [%1];" : "=h"(a) : "l"(kp + sc));
        asm("ld.global.nc.b16 %0, [%1];" : "=h"(b) : "l"(vp + sc));
        ks[i][0] = a;
        vs[i][0] = b;
      } else {
        load_words<kScaleWords>(kp + sc, ks[i]);
        load_words<kScaleWords>(vp + sc, vs[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) load_words<NB / 2>(vp + (r + 2 * t + (i & 1) + 8 * (i >> 1)) * kRow + g * (2 * NB), v[i]);
  }
  __device__ __forceinline__ uint32_t most_scale() const {
    if constexpr (NB == 8) return max(most_byte(vs[0][0], vs[1][0]), most_byte(vs[0][1], vs[1][1]));
    else return most_byte(vs[0][0], vs[1][0]);
  }
  // (all 255s left out)
  __device__ __forceinline__ uint32_t most_real_scale() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const uint32_t s = byte_at(vs[i], b);
        if (s != 255u) m = max(m, s);
      }
    return m;
  }
  __device__ __forceinline__ bool nan_key(int i) const {
    bool any = false;
#pragma unroll
    for (int b = 0; b < NB; ++b) any |= byte_at(ks[i], b) == 255u;
    return any;
  }
};

template <int NB, int NT>
constexpr int smem_bytes() {
  return 8 * NT * 32 * NB * 2 + kWarps * 8 * NT * (32 * NB + 4) * 4 + kWarps * 8 * NT * 8 + 8 * NT * 16;
}

template <int NB, int NT, int RESIDENT>
__global__ void __launch_bounds__(kThreads, RESIDENT) mx_attention_kernel(const __grid_constant__ AttnArgs a) {
  constexpr int D = 32 * NB, ROWS = 8 * NT, kPitch = D + 4;
  constexpr bool kKeepQ = NT * NB <= 8;                  // queries in registers
  extern __shared__ __align__(16) uint8_t smem[];
  uint2* qs = reinterpret_cast<uint2*>(smem);                                   // [NT][NB][2][32 lanes] of four float16
  float* os = reinterpret_cast<float*>(smem + ROWS * D * 2);                    // [warps][ROWS][kPitch]
  float2* mls = reinterpret_cast<float2*>(os + kWarps * ROWS * kPitch);         // [warps][ROWS]
  float* fac = reinterpret_cast<float*>(mls + kWarps * ROWS);                   // rows: what a product of codes is times,
  int* lim = reinterpret_cast<int*>(fac + ROWS);                                // the last token seen (-1: none),
  int* low = lim + ROWS;                                                        // and the first
  __shared__ int64_t scan[kWarps];
  __shared__ int found_s;
  __shared__ int64_t found_at;

  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), g = lane >> 2, t = lane & 3;
  const int hkv = a.c.hkv, cta = blockIdx.x;
  pdl_wait_then_release();

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

  // ---- rows that see nothing because their sequence has no tokens, and rows of no sequence
  {
    const int64_t row_words = (int64_t)a.hq * D / (a.out_f32 ? 4 : 8);
    uint4* out = static_cast<uint4*>(a.out);
    auto clear = [&](int64_t r0, int64_t r1, int64_t first, int64_t stride) {
      for (int64_t i = r0 * row_words + first; i < r1 * row_words; i += stride) out[i] = make_uint4(0u, 0u, 0u, 0u);
    };
    for (int s = cta; s < a.seqs; s += gridDim.x) {
      const Seq q = seq_at<ROWS>(a, s);
      if (!q.steps && q.ql > 0) clear(q.begin, q.begin + q.ql, tid, kThreads);
    }
    if (a.offsets) {
      const int64_t first = (int64_t)cta * kThreads + tid, stride = (int64_t)gridDim.x * kThreads;
      const int head = min(max(a.offsets[0], 0), a.n), tail = min(max(a.offsets[a.seqs], 0), a.n);
      clear(0, head, first, stride);
      clear(max(tail, head), a.n, first, stride);
    }
  }
  __syncthreads();
  if (tid == 0 && a.plan) a.plan[cta].last = -1;
  if (cta >= ctas) return;

  int s = found_s;
  int64_t at = found_at;                                 // place in the sequence's part of the line
  int64_t left = to - from;
  Seq sq = seq_at<ROWS>(a, s);
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
    if (tid == 0 && starts && step1 > 0 && !whole) {
      // the last CTA with a part: that of the unit's last step
      const int64_t last_place = to - end_place + unit_cost - 1;         // on the line (`to` is where this piece ends)
      Plan p = {s, h, rt, 0};
      int64_t k = last_place < rest * (each + 1) ? last_place / (each + 1) : rest + (last_place - rest * (each + 1)) / each;
      p.last = (int)k;
      a.plan[cta] = p;
    }
    left -= end_place - place;
    at += end_place - place;
    if (starts && step1 == 0) continue;                  // (only the unit's beginning: the next CTA has its first step)
    const int slot = 2 * cta + (starts ? 1 : 0);

    // ---- queries to float16, in the order of the operand
    const int rows = min(ROWS, sq.ql * a.group - rt * ROWS);
    __syncthreads();                                     // (the unit before has been written)
    for (int r = warp; r < ROWS; r += kWarps) {
      constexpr int kPer = NB;                           // channels a lane: D / 32
      float x[kPer];
      float amax = 0.f;
      const int rr = rt * ROWS + r, j = rr / a.group;
#pragma unroll
      for (int i = 0; i < kPer; ++i) x[i] = 0.f;
      if (r < rows) {
        const __nv_bfloat16* p = a.q + ((int64_t)(sq.begin + j) * a.hq + h * a.group + (rr - j * a.group)) * D + lane * kPer;
#pragma unroll
        for (int i = 0; i < kPer; i += 2) {
          const uint32_t w = *reinterpret_cast<const uint32_t*>(p + i);
          x[i] = __uint_as_float(w << 16);
          x[i + 1] = __uint_as_float(w & 0xFFFF0000u);
        }
      }
#pragma unroll
      for (int i = 0; i < kPer; ++i) amax = fmaxf(amax, __uint_as_float(min(__float_as_uint(x[i]) & 0x7FFFFFFFu, 0x7F800000u)));
      const int e = max((int)(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(amax)) >> 23), 1);
      const float up = e >= 254 ? 0x1p-127f : __uint_as_float((uint32_t)(254 - e) << 23);      // 2^(127 - e)
      uint32_t w[kPer / 2];
#pragma unroll
      for (int i = 0; i < kPer; i += 2) w[i / 2] = e == 255 ? 0x7FFF7FFFu : f16_pair(x[i] * up * 0x1p13f, x[i + 1] * up * 0x1p13f);
      // channel c: block c / 32, lane's t = c % 32 / 8, then two halves u of four
#pragma unroll
      for (int i = 0; i < kPer; i += 2) {
        const int c = lane * kPer + i, b = c / 32, tt = c % 32 / 8, u = c % 8 / 4, k = c % 4 / 2;
        reinterpret_cast<uint32_t*>(qs + (((r / 8) * NB + b) * 2 + u) * 32 + (r & 7) * 4 + tt)[k] = w[i / 2];
      }
      if (lane == 0) {
        const int64_t p = sq.len - sq.ql + j;
        fac[r] = ldexpf(a.scale, e - 140);
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
    float f[NT][2], m[NT][2], l[NT][2], acc[NB][2][NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f[j][i] = fac[8 * j + 2 * t + i];
        m[j][i] = -1e30f;
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
    int ref = kLowR;                                     // largest scale byte of values so far
    // tokens that all rows see
    const int64_t p_first = sq.len - sq.ql + (rt * ROWS) / a.group, p_last = sq.len - sq.ql + (rt * ROWS + rows - 1) / a.group;
    const int64_t all_to = p_first < sq.end - 1 ? p_first : sq.end - 1, all_from = a.window ? p_last - a.window + 1 : 0;

    const int64_t t_base = sq.first / 16 * 16;
    const int32_t* pages = a.table + (int64_t)s * a.width;
    auto page_of = [&](int step) { return step < step1 ? (int64_t)pages[(t_base + 16 * (int64_t)step) >> a.c.page_log] : -1; };
    auto load = [&](Step<NB>& st, int64_t pg, int step) {
      if (pg < 0 || pg >= a.pages) return;
      const uint8_t* kp = a.c.at(pg, 0, h);
      st.load(kp, kp + a.c.hkv * a.c.part, a.c.page, (int)((t_base + 16 * (int64_t)step) & (a.c.page - 1)), g, t);
    };
    int step = step0 + warp;
    Step<NB> next;
    int64_t pg = page_of(step), pg_next = page_of(step + kWarps);
    load(next, pg, step);
    for (; step < step1; step += kWarps) {
      const Step<NB> cur = next;
      const int64_t here = pg;
      pg = pg_next;
      pg_next = page_of(step + 2 * kWarps);
      load(next, pg, step + kWarps);
      if (here < 0 || here >= a.pages) continue;

      // ---- scores
      float x[NT][4];
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) x[j][k] = 0.f;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        float part[NT][4];
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int k = 0; k < 4; ++k) part[j][k] = 0.f;
        const uint32_t lo[4] = {code_pair<0>(cur.k[0][b]), code_pair<0>(cur.k[1][b]), code_pair<1>(cur.k[0][b]), code_pair<1>(cur.k[1][b])};
        const uint32_t hi[4] = {code_pair<2>(cur.k[0][b]), code_pair<2>(cur.k[1][b]), code_pair<3>(cur.k[0][b]), code_pair<3>(cur.k[1][b])};
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const uint2 q0 = kKeepQ ? qf[kKeepQ ? j : 0][b][0] : qs[((j * NB + b) * 2) * 32 + lane];
          const uint2 q1 = kKeepQ ? qf[kKeepQ ? j : 0][b][1] : qs[((j * NB + b) * 2 + 1) * 32 + lane];
          mma(part[j], lo, q0.x, q0.y);
          mma(part[j], hi, q1.x, q1.y);
        }
        const float s0 = byte_scale_at(cur.ks[0], b), s1 = byte_scale_at(cur.ks[1], b);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          x[j][0] = fmaf(part[j][0], s0, x[j][0]);
          x[j][1] = fmaf(part[j][1], s0, x[j][1]);
          x[j][2] = fmaf(part[j][2], s1, x[j][2]);
          x[j][3] = fmaf(part[j][3], s1, x[j][3]);
        }
      }
      const bool nan0 = cur.nan_key(0), nan1 = cur.nan_key(1);
      const int64_t t0 = t_base + 16 * (int64_t)step;
      bool over = false;
      const bool partial = t0 + 15 > all_to || t0 < all_from;
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          x[j][k] *= f[j][k & 1];
          if (k < 2 ? nan0 : nan1) x[j][k] = __int_as_float(0x7FFFFFFF);
          if (partial) {
            const int tok = (int)t0 + g + 8 * (k >> 1), r = 8 * j + 2 * t + (k & 1);
            if (tok > lim[r] || tok < low[r]) x[j][k] = __int_as_float(0xFF800000);
          }
          over |= x[j][k] > m[j][k & 1] + kSlack;
        }

      // ---- running maxima and the values' reference
      if (__any_sync(0xFFFFFFFFu, over)) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float top = fmaxf(x[j][i], x[j][2 + i]);
#pragma unroll
            for (int k = 4; k < 32; k <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, k));
            top = fmaxf(top, m[j][i]);
            const float by = ex2(m[j][i] - top);
            m[j][i] = top;
            l[j][i] *= by;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                acc[b][c][j][i] *= by;
                acc[b][c][j][2 + i] *= by;
              }
          }
      }
      bool odd = false;
      if (__any_sync(0xFFFFFFFFu, cur.most_scale() > (uint32_t)ref)) {
        const int top = max((int)__reduce_max_sync(0xFFFFFFFFu, cur.most_real_scale()), ref);
        odd = __any_sync(0xFFFFFFFFu, cur.most_scale() == 255u);
        const float by = ex2((float)(ref - top));
        ref = top;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          l[j][0] *= by;
          l[j][1] *= by;
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
              for (int k = 0; k < 4; ++k) acc[b][c][j][k] *= by;
        }
      }

      // ---- weights times 2^(136 - ref): with a value's scale, 2^(byte - 127), at most 2^15
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          x[j][k] = ex2(x[j][k] - (m[j][k & 1] - (float)(136 - ref)));
          l[j][k & 1] += x[j][k];
        }

      // ---- values
#pragma unroll
      for (int i = 0; i < NB / 2; ++i) {
        // even and odd channels of pairs of tokens: nibbles side by side
        uint32_t ev[2], ov[2];
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2) {
          const uint32_t A = cur.v[2 * h2][i], B = cur.v[2 * h2 + 1][i];
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
          const float s0 = byte_scale_at(cur.vs[0], b), s1 = byte_scale_at(cur.vs[1], b);
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            float w[4] = {x[j][0] * s0, x[j][1] * s0, x[j][2] * s1, x[j][3] * s1};
            if (odd) {                                   // a NaN scale counts for rows that see its token only
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                if (byte_at(cur.vs[k >> 1], b) == 255u) w[k] = __int_as_float(0x7FFFFFFF);
                if (x[j][k] == 0.f) w[k] = 0.f;
              }
            }
            const uint32_t p0 = transpose(f16_pair(w[0], w[1])), p1 = transpose(f16_pair(w[2], w[3]));
            mma(acc[b][0][j], va[2 * o], p0, p1);
            mma(acc[b][1][j], va[2 * o + 1], p0, p1);
          }
        }
      }
    }

    // ---- the warps' parts together
    const float unref = ex2((float)(ref - 136));
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int k = 4; k < 32; k <<= 1) l[j][i] += __shfl_xor_sync(0xFFFFFFFFu, l[j][i], k);
        if (g == 0) mls[warp * ROWS + 8 * j + 2 * t + i] = make_float2(m[j][i], l[j][i] * unref);
        float* o = os + (warp * ROWS + 8 * j + 2 * t + i) * kPitch;
#pragma unroll
        for (int b = 0; b < NB; ++b)
          *reinterpret_cast<float4*>(o + 32 * b + 4 * g) = make_float4(acc[b][0][j][i] * unref, acc[b][0][j][2 + i] * unref,
                                                                       acc[b][1][j][i] * unref, acc[b][1][j][2 + i] * unref);
      }
    __syncthreads();
    for (int i = tid; i < rows * (D / 4); i += kThreads) {
      const int r = i / (D / 4), c = i - r * (D / 4);
      float top = mls[r].x, sum = 0.f;
#pragma unroll
      for (int w = 1; w < kWarps; ++w) top = fmaxf(top, mls[w * ROWS + r].x);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float2 ml = mls[w * ROWS + r];
        const float by = ex2(ml.x - top);
        const float4 v = *reinterpret_cast<const float4*>(os + (w * ROWS + r) * kPitch + 4 * c);
        sum = fmaf(ml.y, by, sum);
        o.x = fmaf(v.x, by, o.x), o.y = fmaf(v.y, by, o.y), o.z = fmaf(v.z, by, o.z), o.w = fmaf(v.w, by, o.w);
      }
      if (whole) {
        const int rr = rt * ROWS + r, j = rr / a.group;
        const int64_t to_row = ((int64_t)(sq.begin + j) * a.hq + h * a.group + (rr - j * a.group)) * D + 4 * c;
        const float inv = sum == 0.f ? 0.f : __fdividef(1.f, sum);
        o.x *= inv, o.y *= inv, o.z *= inv, o.w *= inv;
        if (a.out_f32) {
          *reinterpret_cast<float4*>(static_cast<float*>(a.out) + to_row) = o;
        } else {
          const __nv_bfloat162 lo = __floats2bfloat162_rn(o.x, o.y), hi = __floats2bfloat162_rn(o.z, o.w);
          *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + to_row) =
              make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
        }
      } else {
        *reinterpret_cast<float4*>(a.parts + ((int64_t)slot * ROWS + r) * D + 4 * c) = o;
        if (c == 0) *reinterpret_cast<float2*>(a.ml + ((int64_t)slot * ROWS + r) * 2) = make_float2(top, sum);
      }
    }
  }
}

// The parts of a unit, one row a CTA: blockIdx.x the CTA that began it.
template <int NB, int NT>
__global__ void __launch_bounds__(kThreads) mx_attention_join_kernel(const __grid_constant__ AttnArgs a) {
  constexpr int D = 32 * NB, ROWS = 8 * NT, kLanes = D / 4, kGroups = kThreads / kLanes;   // lanes a row of four channels; parts at once
  __shared__ float4 os[kThreads];
  __shared__ float2 mls[kGroups];
  pdl_wait_then_release();
  const int cta = blockIdx.x, r = blockIdx.y;
  const Plan p = a.plan[cta];
  if (p.last < 0) return;
  const Seq sq = seq_at<ROWS>(a, p.s);
  if (r >= min(ROWS, sq.ql * a.group - p.rt * ROWS)) return;
  const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  float top = -1e30f, sum = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k = cta + group; k <= p.last; k += kGroups) {
    const int64_t slot = ((int64_t)2 * k + (k == cta ? 1 : 0)) * ROWS + r;
    const float2 ml = *reinterpret_cast<const float2*>(a.ml + slot * 2);
    const float4 v = *reinterpret_cast<const float4*>(a.parts + slot * D + 4 * lane);
    const float now = fmaxf(top, ml.x), was = ex2(top - now), by = ex2(ml.x - now);
    top = now;
    sum = sum * was + ml.y * by;
    o.x = o.x * was + v.x * by, o.y = o.y * was + v.y * by, o.z = o.z * was + v.z * by, o.w = o.w * was + v.w * by;
  }
  os[threadIdx.x] = o;
  if (lane == 0) mls[group] = make_float2(top, sum);
  __syncthreads();
  if (group != 0) return;
  for (int w = 1; w < kGroups; ++w) {
    const float2 ml = mls[w];
    const float4 v = os[w * kLanes + lane];
    const float now = fmaxf(top, ml.x), was = ex2(top - now), by = ex2(ml.x - now);
    top = now;
    sum = sum * was + ml.y * by;
    o.x = o.x * was + v.x * by, o.y = o.y * was + v.y * by, o.z = o.z * was + v.z * by, o.w = o.w * was + v.w * by;
  }
  const int rr = p.rt * ROWS + r, j = rr / a.group;
  const int64_t to_row = ((int64_t)(sq.begin + j) * a.hq + p.h * a.group + (rr - j * a.group)) * D + 4 * lane;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  o.x *= inv, o.y *= inv, o.z *= inv, o.w *= inv;
  if (a.out_f32) {
    *reinterpret_cast<float4*>(static_cast<float*>(a.out) + to_row) = o;
  } else {
    const __nv_bfloat162 lo = __floats2bfloat162_rn(o.x, o.y), hi = __floats2bfloat162_rn(o.z, o.w);
    *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + to_row) =
        make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
  }
}

int sm_count() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return -1;
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms <= 0) return -1;
  return sms;
}

// Tiles of 8 rows that a call's units have, and CTAs an SM: by what a warp keeps in registers (NT 16-channel accumulators a block of
// 32 channels, and two steps' codes).
struct Form {
  int nt, resident;
};
Form form_of(int64_t n, int64_t seqs, int64_t hq, int64_t hkv, int64_t d) {
  const int64_t rows = (n + seqs - 1) / seqs * (hq / hkv);     // of a sequence, on average
  const int most = d == 256 ? 2 : 4;
  int nt = rows <= 8 ? 1 : rows <= 16 ? 2 : 4;
  if (nt > most) nt = most;
  return {nt, (int)(nt * d <= 128 ? 4 : nt * d <= 256 ? 3 : 2)};
}

size_t round_up(size_t v) { return (v + 255) / 256 * 256; }

template <int NB, int NT, int RESIDENT>
cudaError_t run(AttnArgs a, int grid, cudaStream_t stream) {
  static PerDevice<cudaError_t> allowed;
  constexpr int kSmem = smem_bytes<NB, NT>();
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
  cfg.gridDim = dim3((unsigned)grid, 8 * NT);
  cfg.dynamicSmemBytes = 0;
  note_launch();
  return cudaLaunchKernelEx(&cfg, mx_attention_join_kernel<NB, NT>, a);
}

}  // namespace

int64_t mx_attention_workspace(int64_t n, int64_t seqs, int64_t hq, int64_t hkv, int64_t d) {
  if (seqs == 0) return 0;
  const int sms = sm_count();
  if (sms < 0) return -1;
  const Form f = form_of(n, seqs, hq, hkv, d);
  const size_t grid = (size_t)sms * f.resident, rows = 2 * grid * 8 * f.nt;
  return (int64_t)(round_up(rows * d * 4) + round_up(rows * 8) + round_up(grid * sizeof(Plan)));
}

cudaError_t launch_mx_attention(const void* q, int64_t n, int64_t hq, const uint8_t* cache, int64_t pages, int64_t page, int64_t hkv,
                                int64_t d, const int32_t* table, int64_t width, const int32_t* lens, int64_t seqs,
                                const int32_t* offsets, float scale, int64_t window, int out_dtype, void* out, void* workspace,
                                cudaStream_t stream) {
  if (seqs == 0) return cudaMemsetAsync(out, 0, (size_t)n * hq * d * (out_dtype == 0 ? 4 : 2), stream);
  const int sms = sm_count();
  if (sms < 0) return cudaErrorInvalidDevice;
  const Form f = form_of(n, seqs, hq, hkv, d);
  const int grid = sms * f.resident;
  const size_t rows = (size_t)2 * grid * 8 * f.nt;
  AttnArgs a = {};
  int log = 0;
  while ((int64_t(1) << log) < page) ++log;
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.c = {const_cast<uint8_t*>(cache), pages * page, (int)page, log, (int)hkv, mx_page_bytes(page, d)};
  a.pages = pages, a.table = table, a.lens = lens, a.offsets = offsets, a.width = width;
  a.n = (int)n, a.hq = (int)hq, a.group = (int)(hq / hkv), a.seqs = (int)seqs;
  a.scale = scale * 1.44269504f;
  a.window = window, a.out = out, a.out_f32 = out_dtype == 0;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  a.parts = reinterpret_cast<float*>(ws);
  a.ml = reinterpret_cast<float*>(ws + round_up(rows * d * 4));
  a.plan = reinterpret_cast<Plan*>(ws + round_up(rows * d * 4) + round_up(rows * 8));
  if (d == 64) return f.nt == 1 ? run<2, 1, 4>(a, grid, stream) : f.nt == 2 ? run<2, 2, 4>(a, grid, stream) : run<2, 4, 3>(a, grid, stream);
  if (d == 128) return f.nt == 1 ? run<4, 1, 4>(a, grid, stream) : f.nt == 2 ? run<4, 2, 3>(a, grid, stream) : run<4, 4, 2>(a, grid, stream);
  return f.nt == 1 ? run<8, 1, 3>(a, grid, stream) : run<8, 2, 2>(a, grid, stream);
}

}  // namespace cat
