// Attention of tiles of query rows over pages of the 4-bit cache: prompts, and more rows than mx_attention.cu is for.
//
//   S = Q K^T (128 rows x KT tokens, float32 in tensor memory),  P = 2^(s - m),  O = O 2^(m' - m) + P V
//
// on 5th-generation tensor cores, float16 operands.  The tensor cores take the codes as numbers only after they are unpacked: each of
// a step's keys and values to float16, code times 2^(byte - ref + 12) with ref the largest scale byte of a warp's tokens (keys;
// the products of 32 tokens are times its power again) or of all values so far (O is scaled when it grows).  That is exact down to 2^-35
// of the largest block.  A row may see other tokens than its neighbours, and its result does not depend on the size of the others: where
// tokens lie apart (keys by more than 2^8; values by more than 2^2 at an edge of what rows see, or below the reference) each has a reference of its own,
// which its scores get back where they are, and its weights carry.  A step's unpacking is shared by 256 rows (two tiles of 128; d = 256:
// one): queries of a key head's group lie together, row r is head r % group of token r / group.
//
// Per step of 128 tokens at d = 128 the MMAs take 2080 cycles of an SM (32 of them, 65 each), the exponentials of 2 x 16384 scores 1024, the
// unpacking ~400 issue slots a scheduler.  A step takes ~4800: a tile's weights (~2900: two passes over its scores, their way from and to
// tensor memory), its two products and the waits between them follow one another, and two tiles in turn fill the tensor cores to 42 %.
// 2048 tokens of 32 heads over 32768: 1099 us, 0.97 PFLOP/s; a prompt of 4096: 217, a unit's beginning and end 12000 cycles of ~150000
// (1082 and 211 before scores and values of any size were looked out for).  What was slower: steps of 64 tokens with two buffers of scores a tile, whose
// products of 64 columns take as long as those of 128 (1350 to 1530 us); the maximum found along with the weights, and these again where
// it grew, whose code does not stay in the instruction cache beside the other roles' (1360 with steps of 64); one ring for the copies
// of keys and of values, where values that wait for room keep keys back (1430).
//
// Warps (576 threads, one CTA an SM):
//   0..3, 4..7   a tile's rows each, one a thread: scores from tensor memory, weights back to it (over the scores; the A operand of P V
//                is read there), the running maximum and sum, O's correction where the maximum grows by more than 2^6, output
//   8..11        keys to float16, 12..15 values: a token's row a thread (d = 256: half of one)
//   16           issues the MMAs: P V of a tile, behind it the tile's next scores (d = 256: of the step after the next), in the weights' place
//   17           bulk copies of the codes as they are, a ring each of keys and values
// MMAs of one thread are carried out in the order of their issue, so next scores may follow the product that reads the weights
// in their place.  Every wait is bounded; one that gives up raises the device status word and all roles drain and leave.  (One copy of the
// wait out of line, for all places: in line at each, a prompt of 4096 took 226 us, of heads of 64 203 instead of 180.)
//
// A CTA has an equal piece of a line of all units as mx_attention.cu's; a unit's length there is a straight line in its number (the
// tokens that its last row sees, or the window), so that its place can be found without a list.
#include <cuda_fp16.h>

#include "mx_attention.cuh"
#include "per_device.h"

namespace cat {
namespace {

constexpr int kThreads = 576;
constexpr int kKeyWarp0 = 8, kValueWarp0 = 12, kMmaWarp = 16, kLoadWarp = 17;
constexpr int kUnitCost = 448;              // a unit's beginning and end, in tokens (measured: 768 and 1024 were up to 4 and 7 % slower)
constexpr int kLeastPiece = 256;            // tokens (with units' costs) that a CTA is worth
constexpr int kLowR = 16;                   // least reference scale byte
constexpr int kKeysApart = 8;               // what 32 tokens' keys may lie apart before each has its own reference
constexpr int kBeyond = 2;                  // what a step's tokens may lie apart, or below the reference, before each has its own
constexpr uint32_t kTmemCols = 512;
constexpr int kBarRoom = 8192;

template <int NB>
struct Tc {
  static constexpr int D = 32 * NB, QT = NB == 8 ? 1 : 2, ROWS = 128 * QT;
  static constexpr int KT = NB == 8 ? 64 : 128;          // tokens a step
  static constexpr int SB = NB == 8 ? 2 : 1;             // buffers of a tile's scores
  static constexpr int kBufs = 2, kBufLog = 1;           // of unpacked keys, and of values
  static constexpr int kQ = 128 * D * 2, kTile = KT * D * 2, kCodes = KT * 16 * NB, kRaw = kCodes + KT * NB;
  static constexpr int kRingK = 2, kRingV = NB == 2 ? 2 : 1, kRing = kRingK + kRingV;      // codes as they are: of keys, of values
  static constexpr int kOffK = QT * kQ, kOffV = kOffK + kBufs * kTile, kOffRaw = kOffV + kBufs * kTile, kOffBars = kOffRaw + kRing * kRaw;
  static constexpr int kSmem = 1024 + kOffBars + kBarRoom;
  static constexpr uint32_t kO = QT * SB * KT;           // tensor memory: the scores, then O's
  static_assert(kSmem <= 227 * 1024 && QT * (SB * KT + D) <= (int)kTmemCols, "");
};

struct Seq : Rows {
  int tiles;
  int64_t a, b;                             // a unit of row tile i has a + b i of the line
  __device__ __forceinline__ int64_t before(int64_t i) const { return a * i + b * (i * (i - 1) / 2); }     // tiles 0 .. i - 1
};
template <int ROWS>
__device__ __forceinline__ Seq seq_at(const AttnArgs& a, int s) {
  Seq q;
  static_cast<Rows&>(q) = rows_of(a, s);
  const int64_t rows = (int64_t)q.ql * a.group;
  q.tiles = q.any() && rows > a.few ? (int)((rows + ROWS - 1) / ROWS) : 0;
  const int64_t tokens = (ROWS + a.group - 1) / a.group, past = q.len > q.ql ? q.len - q.ql : 0;
  q.a = kUnitCost + past + tokens;
  q.b = tokens;
  if (a.window && a.window + tokens < past + tokens * q.tiles) {
    q.a = kUnitCost + a.window + tokens;
    q.b = 0;
  }
  return q;
}

// A CTA's way along its piece, the same in all warps; each keeps its own in shared memory (registers are short).
struct Unit {
  int s, h, rt, rows, j0, j1;               // the steps of KT tokens, from the sequence's beginning
  bool starts, whole, nothing;              // nothing: no row sees a token
  int64_t p0;                               // the token of the sequence's first row
  int64_t t0, t1;                           // the tokens that some row sees,
  int64_t a0, a1;                           // and that all rows see (but those before the sequence's beginning, which see nothing)
  int64_t from, end;                        // where the unit's first step ends on the line (of a later piece), and its end
  int begin;                                // the sequence's first row,
  int64_t tokens;                           // and one past its last token in the cache
};
struct Walk {
  int s, rt, h;                             // the next unit,
  int64_t place, left, to;                  // where in it; what is left of the piece, and its end
  Seq q;
  Unit u;
  template <int NB>
  __device__ __forceinline__ void begin(const AttnArgs& a, int s_, int64_t at, int64_t from, int64_t to_) {
    s = s_, left = to_ - from, to = to_;
    q = seq_at<Tc<NB>::ROWS>(a, s_);
    int lo = 0, hi = q.tiles - 1;                        // the last tile that begins at `at` or before
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (a.c.hkv * q.before(mid) <= at)
        lo = mid;
      else
        hi = mid - 1;
    }
    const int64_t in = at - a.c.hkv * q.before(lo), length = q.a + q.b * lo;
    rt = lo, h = (int)(in / length), place = in - h * length;
  }
  // A whole warp: the next unit with something to do.
  template <int NB>
  __device__ __forceinline__ bool next(const AttnArgs& a) {
    __syncwarp();                                        // (all lanes are done with the unit before)
    bool more = false;
    if ((threadIdx.x & 31) == 0) more = advance<NB>(a);
    more = __shfl_sync(0xFFFFFFFFu, more, 0);
    __syncwarp();
    return more;
  }
  template <int NB>
  __device__ __noinline__ bool advance(const AttnArgs& a) {
    using C = Tc<NB>;
    constexpr int KT = C::KT;
    while (left > 0) {
      const int64_t length = q.a + q.b * rt, end = place + left < length ? place + left : length;
      const uint32_t group = (uint32_t)a.group, row0 = (uint32_t)rt * C::ROWS;
      u.s = s, u.h = h, u.rt = rt;
      u.rows = (int)min((int64_t)C::ROWS, (int64_t)q.ql * a.group - (int64_t)row0);
      u.p0 = q.len - q.ql;
      const int64_t p_first = u.p0 + row0 / group, p_last = u.p0 + (row0 + (uint32_t)u.rows - 1) / group;
      const int64_t t1 = p_last + 1 < q.end ? p_last + 1 : q.end, t0 = a.window && p_first - a.window + 1 > 0 ? p_first - a.window + 1 : 0;
      u.a0 = a.window && p_last - a.window + 1 > 0 ? p_last - a.window + 1 : 0;
      u.a1 = (p_first > 0 ? p_first : 0) + 1;
      u.t0 = t0, u.t1 = t1, u.begin = q.begin, u.tokens = q.end;
      const int first = (int)(t0 / KT), steps = t1 > t0 ? (int)((t1 + KT - 1) / KT) - first : 0;
      // (any growing map of the line to steps will do that is the same for all: in float32)
      auto step_of = [&](int64_t x) { return x == length ? steps : min((int)((float)x / (float)length * (float)steps), steps); };
      const int x0 = step_of(place), x1 = step_of(end);
      u.j0 = first + x0, u.j1 = first + x1;
      u.starts = x0 == 0;
      u.whole = u.starts && x1 == steps;
      u.nothing = steps == 0;
      const bool cleared = u.nothing && place == 0;
      // a unit's later piece may have no step: its part is marked empty
      const bool empty_part = x0 == x1 && x0 > 0;
      left -= end - place;
      u.end = to - left + (length - end);
      if (x0 > 0) {                                      // (the first end with a step; beside the quotient for rounding's sake)
        int64_t x = length / steps;
        while (step_of(x - 1) > 0) --x;
        while (step_of(x) == 0) ++x;
        u.from = u.end - length + x - 1;                 // (a piece's end counts for its steps)
      }
      place = end;
      if (end == length) {                               // the next unit
        place = 0;
        if (++h == a.c.hkv) {
          h = 0;
          if (++rt == q.tiles && left > 0) {
            rt = 0;
            do q = seq_at<C::ROWS>(a, ++s);
            while (q.tiles == 0);
          }
        }
      }
      if (x1 > x0 || cleared || empty_part) return true;
    }
    return false;
  }
};

struct Bars {
  uint64_t raw_full[6], raw_empty[6], k_full[4], k_empty[4], v_full[4], v_empty[4], q_full, s_full[2][2], p_full[2][2], pv_done[2][2], most_full,
      mma_done;
  // (of eight steps: keys are unpacked up to five steps ahead of scores that are still read)
  int k_power[8][4];                        // 2^(ref - 139) of 32 tokens' keys, as a float32's exponent field
  uint32_t k_apart[8];                      // a byte for 32 tokens: whether their products are times 2^(k_own - ref) each
  uint8_t k_own[8][128];
  uint32_t there[8];                        // which 16-token groups of a step are on pages
  uint32_t raw_there[6];
  uint32_t v_ref[2];                        // the values' reference, + 256 where a scale of the step's is NaN, + 512 where each token has its own
  uint32_t v_most[2][4];                    // the largest of a warp's tokens, + 256 the same, + 65536 times the least of its tokens' largest
  uint8_t v_own[2][128];                    // a token's own reference
  uint8_t v_nan[2][2][128];                  // a token's blocks of NaN scales (d = 256: those of half of them)
  int64_t scan[20];
  int64_t found_at;
  int found_s;
  Waits waits;
  uint32_t tmem_addr;
  Walk walks[20];
};
static_assert(sizeof(Bars) <= kBarRoom, "barrier room");

// ---- tensor memory
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Instruction descriptor of kind::f16: float16 operands, D float32, M = 128; A K-major, B K-major or (bit 16) MN-major.
__host__ __device__ constexpr uint32_t idesc_f16(int n, bool b_mn) { return (1u << 4) | (b_mn ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24); }
// MN-major operand, 128-byte swizzle: a token a 128-byte row of 64 channels, 8 tokens 1 KiB apart, 64 channels `lbo` bytes.
__device__ __forceinline__ uint64_t sdesc_mnmajor_sw128(uint32_t saddr, uint32_t lbo) {
  return (uint64_t)((saddr >> 4) & 0x3FFFu) | ((uint64_t)((lbo >> 4) & 0x3FFFu) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }" ::"r"(d), "l"(a), "l"(b),
               "r"(idesc), "r"(accumulate)
               : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }" ::"r"(d), "r"(a), "l"(b),
               "r"(idesc), "r"(accumulate)
               : "memory");
}

__device__ __forceinline__ uint32_t f16_pair(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// The four pairs of a word's codes, times a scale.
__device__ __forceinline__ void unpack8(uint32_t w, __half2 s, uint32_t (&r)[4]) {
  asm("{ .reg .b8 a, b, c, d; mov.b32 {a, b, c, d}, %4; cvt.rn.f16x2.e2m1x2 %0, a; cvt.rn.f16x2.e2m1x2 %1, b; "
      "cvt.rn.f16x2.e2m1x2 %2, c; cvt.rn.f16x2.e2m1x2 %3, d; }"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
      : "r"(w));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 v = __hmul2_rn(*reinterpret_cast<const __half2*>(&r[i]), s);
    r[i] = *reinterpret_cast<const uint32_t*>(&v);
  }
}
// 2^(byte - ref + 12) twice (byte <= ref), subnormal below 2^-14 and 0 below 2^-24.
__device__ __forceinline__ __half2 half_scale(int byte, int ref) {
  const int e = byte - ref + 27;
  const uint32_t h = e > 0 ? (uint32_t)e << 10 : e > -10 ? 512u >> -e : 0u, two = h | h << 16;
  return *reinterpret_cast<const __half2*>(&two);
}

// Two float32 operations at once.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  uint64_t r;
  asm("{ .reg .b64 x, y, z; mov.b64 x, {%1, %2}; mov.b64 y, {%3, %4}; mov.b64 z, {%5, %6}; fma.rn.f32x2 %0, x, y, z; }"
      : "=l"(r)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  float2 o;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(o.x), "=f"(o.y) : "l"(r));
  return o;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  uint64_t r;
  asm("{ .reg .b64 x, y; mov.b64 x, {%1, %2}; mov.b64 y, {%3, %4}; mul.rn.f32x2 %0, x, y; }"
      : "=l"(r)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  float2 o;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(o.x), "=f"(o.y) : "l"(r));
  return o;
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  uint64_t r;
  asm("{ .reg .b64 x, y; mov.b64 x, {%1, %2}; mov.b64 y, {%3, %4}; add.rn.f32x2 %0, x, y; }"
      : "=l"(r)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  float2 o;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(o.x), "=f"(o.y) : "l"(r));
  return o;
}

// A token's row of keys or values (d = 256: half of its blocks) to float16 operands.  Operands are rows of
// 64 channels, 128 bytes each, 16-byte pieces at piece ^ (row mod 8).  Quarters are taken in an order that differs from lane to lane, so that
// neither reads nor writes meet in a bank (reads of d = 256 do in pairs).
template <int NB>
__device__ __forceinline__ void unpack_row(const uint8_t* raw, uint8_t* tile, int row, int half, bool values,
                                            const __half2 (&scale)[NB < 4 ? NB : 4]) {
  constexpr int KT = Tc<NB>::KT, kHere = NB < 4 ? NB : 4;
  const int block0 = NB == 8 ? 4 * half : 0, turn = (NB == 2 ? row >> 2 : row >> 1) & 3;
#pragma unroll 1
  for (int i = 0; i < 4; ++i) {
    const int p = i ^ turn;                              // the quarter: channels 8 p .. 8 p + 7 of every block
    const uint8_t* at = raw + row * (16 * NB) + p * (4 * NB);
    uint32_t w[kHere];
    if constexpr (NB == 2) {
      const uint2 v = *reinterpret_cast<const uint2*>(at);
      w[0] = v.x, w[1] = v.y;
    } else if constexpr (NB == 4) {
      const uint4 v = *reinterpret_cast<const uint4*>(at);
      w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    } else {                                             // (half of a quarter's words; of values, half of either row of halfwords)
      const uint2 v = *reinterpret_cast<const uint2*>(at + (values ? 8 : 16) * half), n = *reinterpret_cast<const uint2*>(at + (values ? 8 * half + 16 : 16 * half + 8));
      w[0] = v.x, w[1] = v.y, w[2] = n.x, w[3] = n.y;
    }
    if (values) {                                        // halfwords [2][blocks]
      uint32_t t[kHere];
#pragma unroll
      for (int b = 0; b < kHere; b += 2) {
        t[b] = __byte_perm(w[b / 2], w[kHere / 2 + b / 2], 0x5410);
        t[b + 1] = __byte_perm(w[b / 2], w[kHere / 2 + b / 2], 0x7632);
      }
#pragma unroll
      for (int b = 0; b < kHere; ++b) w[b] = t[b];
    }
#pragma unroll
    for (int b = 0; b < kHere; ++b) {
      uint32_t r[4];
      unpack8(w[b], scale[b], r);
      const int block = block0 + b, piece = (block & 1) * 4 + p;
      *reinterpret_cast<uint4*>(tile + (block >> 1) * (KT * 128) + row * 128 + ((piece ^ (row & 7)) << 4)) = make_uint4(r[0], r[1], r[2], r[3]);
    }
  }
}

// 16 columns of this warp's 32 lanes
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
                 "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
               : "r"(taddr));
}

// The same, there: what is done with them is behind this.
__device__ __forceinline__ void tmem_have32(uint32_t (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]),
                 "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]), "+r"(v[17]), "+r"(v[18]),
                 "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23])
               :
               : "memory");
  asm volatile("" : "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31]));
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float m;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
  return m;
}
__device__ __forceinline__ void tmem_have16(uint32_t (&v)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]),
                 "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])::"memory");
}

// What a product of a row's query and keys is times: significand * 2^power of the row, times the keys' power of two.  Never 0, which would
// make NaN of the infinity that stands for what is not seen, nor infinite, which would of a product that is 0.
struct Factor {
  uint32_t significand;                     // of [1, 2), its 23 bits
  int power;
  __device__ __forceinline__ float of(int k_power) const {
    return __uint_as_float((uint32_t)min(max(power + k_power, 1), 254) << 23 | significand);
  }
};

// The largest score of a row's KT, times its factors.
template <int KT>
__device__ __forceinline__ float largest(uint32_t s_col, const int* k_power, Factor fac) {
  float most = -INFINITY;
  uint32_t a[16], b[16];
  auto of = [](const uint32_t (&v)[16]) {
    float m[2] = {fmaxf(__uint_as_float(v[0]), __uint_as_float(v[1])), fmaxf(__uint_as_float(v[2]), __uint_as_float(v[3]))};
#pragma unroll
    for (int i = 4; i < 16; i += 4) {
      m[0] = max3(m[0], __uint_as_float(v[i]), __uint_as_float(v[i + 1]));
      m[1] = max3(m[1], __uint_as_float(v[i + 2]), __uint_as_float(v[i + 3]));
    }
    return fmaxf(m[0], m[1]);
  };
  tmem_ld16(s_col, a);
  tmem_have16(a);
#pragma unroll 1
  for (int c = 0; c < KT / 32; ++c) {
    tmem_ld16(s_col + 32 * c + 16, b);
    const float f = fac.of(k_power[c]), m = of(a);
    tmem_have16(b);
    tmem_ld16(s_col + 32 * min(c + 1, KT / 32 - 1), a);
    most = fmaxf(most, fmaxf(m, of(b)) * f);
    tmem_have16(a);
  }
  return most;
}
// A row's weights 2^(score + base), as float16 pairs in the scores' place; their sum is added to `sum`.
template <int KT>
__device__ __forceinline__ void weights(uint32_t s_col, const int* k_power, Factor fac, float base, float2& sum) {
  float2 part = make_float2(0.f, 0.f);
#pragma unroll 1
  for (int c = 0; c < KT / 32; ++c) {
    uint32_t v[32], w[16];
    CAT_TMEM_LD32(s_col + 32 * c, v);
    const float f = fac.of(k_power[c]);
    tmem_have32(v);
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
      float2 x = fma2(make_float2(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), make_float2(f, f), make_float2(base, base));
      x.x = ex2(x.x), x.y = ex2(x.y);
      if (i & 2)
        part = add2(part, x);
      else
        sum = add2(sum, x);
      w[i / 2] = f16_pair(x.x, x.y);
    }
    tmem_st16(s_col + 16 * c, w);
  }
  sum = add2(sum, part);
}
// The same of scores that are rounded before m is taken off (what a product keeps beyond float32 would be a large difference of large
// scores), times 2^(own - ref) of each token's own reference where there are such.
template <int KT>
__device__ __forceinline__ float weights_apart(uint32_t s_col, const int* k_power, Factor fac, float m, const uint8_t* own, int ref) {
  float sum = 0.f;
#pragma unroll 1
  for (int c = 0; c < KT / 16; ++c) {
    uint32_t v[16], w[8];
    tmem_ld16(s_col + 16 * c, v);
    const float f = fac.of(k_power[c / 2]);
    tmem_have16(v);
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const float x = ex2(__fadd_rn(__fmul_rn(__uint_as_float(v[i]), f), -m) + 8.f), y = ex2(__fadd_rn(__fmul_rn(__uint_as_float(v[i + 1]), f), -m) + 8.f);
      sum += x + y;
      // (what is not seen, 0, may be of any size)
      const float up = own ? ex2((float)min((int)own[16 * c + i] - ref, 0)) : 1.f, up2 = own ? ex2((float)min((int)own[16 * c + i + 1] - ref, 0)) : 1.f;
      w[i / 2] = f16_pair(x * up, y * up2);
    }
    tmem_st8(s_col + 8 * c, w);
  }
  return sum;
}
// Scores of tokens that a row does not see become -infinity where they are, and products of keys with references of their own get them
// (steps at an end of what the rows see, and such, alone come here).
template <int KT>
__device__ __forceinline__ void hide(uint32_t s_col, int t0, int lim, int low, uint32_t there, uint32_t apart, const uint8_t* own, const int* k_power) {
#pragma unroll 1
  for (int c = 0; c < KT / 16; ++c) {
    uint32_t v[16];
    tmem_ld16(s_col + 16 * c, v);
    tmem_have16(v);
    if (apart >> (8 * (c / 2)) & 1u) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        v[i] = __float_as_uint(__uint_as_float(v[i]) * ex2((float)((int)own[16 * c + i] - (k_power[c / 2] + 12))));
    }
    const bool on = there >> c & 1;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int at = t0 + 16 * c + i;
      if (!on || at > lim || at < low) v[i] = 0xFF800000u;
    }
    tmem_st16(s_col + 16 * c, v);
  }
  tmem_st_wait();
}

template <int NB>
__global__ void __launch_bounds__(kThreads, 1) mx_attention_tiles_kernel(const __grid_constant__ AttnArgs a) {
  using C = Tc<NB>;
  constexpr int D = C::D, KT = C::KT, SB = C::SB, QT = C::QT, kBufs = C::kBufs, kBufLog = C::kBufLog, ROWS = C::ROWS, kHere = NB < 4 ? NB : 4;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  Bars* bars = reinterpret_cast<Bars*>(smem + C::kOffBars);
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), cta = blockIdx.x, hkv = a.c.hkv;

  if (tid == 0) {
    for (int i = 0; i < 6; ++i) mbar_init(&bars->raw_full[i], 1), mbar_init(&bars->raw_empty[i], 4);
    for (int i = 0; i < 8; ++i) bars->k_apart[i] = 0u;
    for (int i = 0; i < 4; ++i) {
      mbar_init(&bars->k_full[i], 4), mbar_init(&bars->v_full[i], 4);
      mbar_init(&bars->k_empty[i], 1), mbar_init(&bars->v_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars->s_full[i][0], 1), mbar_init(&bars->s_full[i][1], 1);
      mbar_init(&bars->p_full[i][0], 4), mbar_init(&bars->p_full[i][1], 4);
      mbar_init(&bars->pv_done[i][0], 1), mbar_init(&bars->pv_done[i][1], 1);
    }
    mbar_init(&bars->q_full, 4 * QT);
    mbar_init(&bars->most_full, 4);
    mbar_init(&bars->mma_done, 1);
    bars->waits.init();
    fence_mbar_init();
  }
  pdl_wait_then_release();

  // ---- this CTA's piece of the line
  const int per = (a.seqs + kThreads - 1) / kThreads, s_from = min(tid * per, a.seqs), s_to = min(s_from + per, a.seqs);
  auto cost = [&](int s) {
    const Seq q = seq_at<ROWS>(a, s);
    return hkv * q.before(q.tiles);
  };
  int64_t mine = 0;
  for (int s = s_from; s < s_to; ++s) mine += cost(s);
  int64_t before = mine, total = 0;
#pragma unroll
  for (int k = 1; k < 32; k <<= 1) {
    const int64_t v = __shfl_up_sync(0xFFFFFFFFu, before, k);
    if (lane >= k) before += v;
  }
  if (lane == 31) bars->scan[warp] = before;
  __syncthreads();
  before -= mine;
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) before += bars->scan[w];
    total += bars->scan[w];
  }
  int64_t ctas = (total + kLeastPiece - 1) / kLeastPiece;
  if (ctas > gridDim.x) ctas = gridDim.x;
  const int64_t each = ctas ? total / ctas : 0, rest = ctas ? total - each * ctas : 0;
  auto cut = [&](int64_t k) { return each * k + (k < rest ? k : rest); };
  const int64_t from = cut(cta), to = cut(cta + 1);
  if (cta < ctas && mine > 0 && before <= from && from < before + mine) {
    int64_t at = before;
    for (int s = s_from; s < s_to; ++s) {
      const int64_t c = cost(s);
      if (from < at + c) {
        bars->found_s = s;
        bars->found_at = from - at;
        break;
      }
      at += c;
    }
  }
  if (a.clears) clear_rows<D>(a);
  if (tid < 2) a.plan[2 * cta + tid].last = -1;
  __syncwarp();
  const bool works = cta < ctas;
  if (warp == kMmaWarp && works) tmem_alloc(&bars->tmem_addr, kTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (!works) return;
  const uint32_t tmem = bars->tmem_addr;
  Walk& walk = bars->walks[warp];
  const Unit& u = walk.u;
  if (lane == 0) walk.begin<NB>(a, bars->found_s, bars->found_at, from, to);
  bool ok = true;
  uint32_t jj = 0;                                       // steps so far
// (The roles' loops have to stay in the instruction cache together: with the timed wait in line at every place, and copies of the weights' code, 77 %
// of the cache's rate behind it went into fetching them again.  Polls are for the MMAs' warp, behind which all others are.)
#define CAT_WAIT(bar, parity) (ok = ok && (bool)__all_sync(0xFFFFFFFFu, short_wait<false>(bar, parity, &bars->waits, __LINE__)))
#define CAT_POLL(bar, parity) (ok = ok && (bool)__all_sync(0xFFFFFFFFu, short_wait<true>(bar, parity, &bars->waits, __LINE__)))

  if (warp < 4 * QT) {
    // ---------------------------------------------------------------- rows
    const int tile = warp >> 2, r = tile * 128 + (warp & 3) * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21), s_cols = lanes + tile * (SB * KT), o_col = lanes + C::kO + tile * D;
    uint32_t units = 0, tj = 0;                          // units and this tile's steps so far
    while (ok && walk.next<NB>(a)) {
      if (tid == 0 && !u.whole)
        a.plan[2 * cta + u.starts] = {u.starts ? cta : cta_of(u.from, each, rest), cta_of(u.end - 1, each, rest), u.begin, u.h, u.rt * ROWS, u.rows};
      const uint32_t rr = (uint32_t)u.rt * ROWS + r;     // (a sequence has less than 2^31 rows)
      const int j = (int)(rr / (uint32_t)a.group);
      const int64_t row = ((int64_t)(u.begin + j) * a.hq + u.h * a.group + (int)(rr - (uint32_t)j * (uint32_t)a.group)) * D;
      const bool real = r < u.rows;
      const int slot = 2 * cta + (u.starts ? 1 : 0);
      if (u.j0 == u.j1) {                                // no tokens: rows of zeros, or an empty part
        if (real && u.nothing) {
          for (int c = 0; c < D; c += 4) store4(a, row + c, make_float4(0.f, 0.f, 0.f, 0.f));
        } else if (real) {
          *reinterpret_cast<float2*>(a.ml + ((int64_t)slot * ROWS + r) * 2) = make_float2(kNone, 0.f);
        }
        continue;
      }
      // The warp's rows to float16, a row's largest channel in [2^13, 2^14); a negative scale goes into its sign.  All of them on their
      // way at once (D / 8 lanes a row), to where each thread then rewrites its own.
      Factor fac;
      {
        constexpr int kLanes = D / 8, kAtOnce = 32 / kLanes;
        const int warp_row = tile * 128 + (warp & 3) * 32;
        uint8_t* const to_q = smem + tile * C::kQ + (warp & 3) * (32 * 128);
        auto place = [&](int at, int piece) { return to_q + (piece >> 3) * (128 * 128) + at * 128 + (((piece & 7) ^ (at & 7)) << 4); };
        __syncwarp();                                    // (what was there has been read)
#pragma unroll 4
        for (int i = 0; i < 32; i += kAtOnce) {
          const int at = i + lane / kLanes, piece = lane % kLanes;
          const int64_t from_q = __shfl_sync(0xFFFFFFFFu, row, at);
          const bool in = warp_row + at < u.rows;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(place(at, piece))),
                       "l"(a.q + (in ? from_q + piece * 8 : 0)), "r"(in ? 16 : 0)
                       : "memory");
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncwarp();
        uint32_t m2[2] = {0u, 0u};
#pragma unroll 4
        for (int i = 0; i < D / 8; ++i) {
          const uint4 v = *reinterpret_cast<const uint4*>(place(lane, i));
          m2[0] = __vmaxu2(m2[0], __vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu));
          m2[1] = __vmaxu2(m2[1], __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
        }
        const uint32_t both = __vmaxu2(m2[0], m2[1]);
        const int e = max((int)(max(both & 0xFFFFu, both >> 16) >> 7), 1);           // this thread's row's exponent
        // (a row with an infinity or a NaN is NaN; the two factors together could leave float32's range)
        const float up = (e == 255 ? __int_as_float(0x7FFFFFFF) : e == 254 ? 0x1p-127f : __uint_as_float((uint32_t)(254 - e) << 23)) *
                         (a.scale < 0.f ? -1.f : 1.f);
        auto half2_of = [&](uint32_t w) {
          const float2 x = mul2(mul2(make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)), make_float2(up, up)),
                                make_float2(0x1p13f, 0x1p13f));
          return f16_pair(x.x, x.y);
        };
#pragma unroll 2
        for (int i = 0; i < D / 8; ++i) {
          uint4* const p = reinterpret_cast<uint4*>(place(lane, i));
          const uint4 v = *p;
          *p = make_uint4(half2_of(v.x), half2_of(v.y), half2_of(v.z), half2_of(v.w));
        }
        int power;
        const float scale = 2.f * frexpf(fabsf(a.scale), &power);      // (of [1, 2), or 0)
        fac = {__float_as_uint(scale) & 0x7FFFFFu, a.scale == 0.f ? -1000 : power - 1 + e - 140};
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (elect_one()) mbar_arrive(&bars->q_full);
      if (!CAT_WAIT(&bars->q_full, units & 1)) break;    // (nobody is at the next unit's queries before all are at this one's)
      ++units;
      const int64_t p = u.p0 + j;
      const int lim = real ? (int)(p < u.tokens - 1 ? p : u.tokens - 1) : 0x7FFFFFFF;
      const int low = real && a.window && p - a.window + 1 > 0 ? (int)(p - a.window + 1) : 0;
      const bool tile_real = tile * 128 < u.rows, any_real = __any_sync(0xFFFFFFFFu, real);
      float m = 0.f;
      bool seen = false, apart = false;                  // the maximum is one of scores; some row's is more than 2^16
      float2 l2 = make_float2(0.f, 0.f);
      int ref = 0;
      uint32_t nan_blocks = 0;
      for (int step = u.j0; step < u.j1; ++step, ++jj) {
        if (!tile_real) continue;
        const uint32_t b = jj & (kBufs - 1), s_col = s_cols + tj % SB * KT;
        const int* k_power = bars->k_power[jj & 7];
        if (!CAT_WAIT(&bars->s_full[tile][tj % SB], tj / SB & 1)) break;
        tc_fence_after();
        if (!any_real) {
          if (!CAT_WAIT(&bars->v_full[b], (jj >> kBufLog) & 1)) break;       // (so that no step is left behind by two rounds)
        } else {
          const int t0 = step * KT;
          const uint32_t there = bars->there[jj & 7];
          constexpr uint32_t kAll = (1u << (KT / 16)) - 1u;
          const uint32_t keys_apart = bars->k_apart[jj & 7];
          const bool full = __all_sync(0xFFFFFFFFu, t0 + KT - 1 <= lim && t0 >= low) && there == kAll && keys_apart == 0u;
          if (!full) hide<KT>(s_col, t0, lim, low, there, keys_apart, bars->k_own[jj & 7], k_power);
          const float most = largest<KT>(s_col, k_power, fac);
          if (!CAT_WAIT(&bars->v_full[b], (jj >> kBufLog) & 1)) break;       // (the values' reference)
          // The row's reference: at least that of the values that it sees, and no more above them than 2^(2 kBeyond), so that what it does not
          // see, which may be anything, costs it no bits.
          const uint32_t v_ref = bars->v_ref[b];
          const bool own = v_ref & 512u;
          int now = t0 <= lim && t0 + KT > low ? max(ref, (int)(v_ref & 255u)) : ref;
          if (own) {
            now = ref;
#pragma unroll 1
            for (int i = 0; i < KT; ++i)
              if (t0 + i <= lim && t0 + i >= low) now = max(now, (int)bars->v_own[b][i]);
          }
          const bool grows = seen ? most > m + kSlack : most > -INFINITY;
          if (__any_sync(0xFFFFFFFFu, grows || now != ref)) {
            const float up = grows ? most : m, by = seen ? ex2(m - up) : 1.f;       // (nothing seen: all is 0)
            m = up;
            seen |= grows;
            apart = __any_sync(0xFFFFFFFFu, fabsf(m) > 0x1p16f);
            l2.x *= by, l2.y *= by;
            if (step != u.j0) {
              if (!CAT_WAIT(&bars->pv_done[tile][(tj - 1) % SB], (tj - 1) / SB & 1)) break;
              tc_fence_after();
              const float scale_o = by * ex2((float)(ref - now));
#pragma unroll 1
              for (int c = 0; c < D; c += 16) {
                uint32_t v[16];
                tmem_ld16(o_col + c, v);
                tmem_have16(v);
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * scale_o);
                tmem_st16(o_col + c, v);
              }
            }
            ref = now;
          }
          if (__builtin_expect(apart || own, 0))
            l2.x += weights_apart<KT>(s_col, k_power, fac, m, own ? bars->v_own[b] : nullptr, ref);
          else
            weights<KT>(s_col, k_power, fac, 8.f - m, l2);   // (times 2^8)
          if (v_ref & 256u)
            for (int i = 0; i < KT; ++i) {
              const int at = t0 + i;
              if (at <= lim && at >= low) nan_blocks |= (uint32_t)bars->v_nan[b][0][i] | (NB == 8 ? bars->v_nan[b][1][i] : 0u);
            }
          tmem_st_wait();
        }
        tc_fence_before();
        __syncwarp();
        if (elect_one()) mbar_arrive(&bars->p_full[tile][tj % SB]);    // (a warp may be a step ahead of another: a barrier for each buffer)
        ++tj;
      }
      if (!ok) break;
      if (!tile_real) continue;
      // ---- out
      if (!CAT_WAIT(&bars->pv_done[tile][(tj - 1) % SB], (tj - 1) / SB & 1)) break;
      tc_fence_after();
      if (any_real) {
        const float l = l2.x + l2.y;
        const float unref = l == 0.f ? 0.f : ldexpf(1.f / l, ref - 139);           // (parts are means, too)
        // 128 bytes of each of the warp's rows at a time (32 channels in float32, 64 in bf16) through the place of its queries, whose
        // products are done: eight lanes a row
        const bool narrow = u.whole && !a.out_f32;
        uint8_t* const mine = !real     ? nullptr
                              : narrow  ? static_cast<uint8_t*>(a.out) + row * 2
                              : u.whole ? static_cast<uint8_t*>(a.out) + row * 4
                                        : reinterpret_cast<uint8_t*>(a.parts + ((int64_t)slot * ROWS + r) * D);
        uint8_t* to[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint64_t base = __shfl_sync(0xFFFFFFFFu, reinterpret_cast<uint64_t>(mine), 4 * k + (lane >> 3));
          to[k] = base ? reinterpret_cast<uint8_t*>(base) + 16 * (lane & 7) : nullptr;
        }
        uint8_t* const stage = smem + tile * C::kQ + (warp & 3) * (32 * 128);
        auto staged = [&](int j) { return reinterpret_cast<uint4*>(stage + lane * 128 + ((j ^ (lane & 7)) << 4)); };
#pragma unroll 1
        for (int c = 0; c < D;) {
#pragma unroll 1
          for (int half = 0; half < (narrow ? 2 : 1); ++half, c += 32) {
            uint32_t v[32];
            CAT_TMEM_LD32(o_col + c, v);
            tmem_have32(v);
            const float by = nan_blocks >> (c / 32) & 1 ? __int_as_float(0x7FFFFFFF) : unref;
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * by);
            if (narrow) {
#pragma unroll
              for (int i = 0; i < 32; i += 2) v[i / 2] = bf16_pair(__uint_as_float(v[i]), __uint_as_float(v[i + 1]));
#pragma unroll
              for (int j = 0; j < 4; ++j) *staged(4 * half + j) = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
            } else {
#pragma unroll
              for (int j = 0; j < 8; ++j) *staged(j) = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
            }
          }
          __syncwarp();
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const int at = 4 * k + (lane >> 3);
            const uint4 o = *reinterpret_cast<const uint4*>(stage + at * 128 + (((lane & 7) ^ (at & 7)) << 4));
            if (to[k]) {
              *reinterpret_cast<uint4*>(to[k]) = o;
              to[k] += 128;
            }
          }
          __syncwarp();
        }
        if (real && !u.whole) *reinterpret_cast<float2*>(a.ml + ((int64_t)slot * ROWS + r) * 2) = make_float2(m, l);
      }
      tc_fence_before();
    }
  } else if (warp >= kKeyWarp0 && warp < kMmaWarp) {
    // ---------------------------------------------------------------- keys and values to float16
    const bool values = warp >= kValueWarp0;
    const int w = (warp - kKeyWarp0) & 3, row = NB == 8 ? (w & 1) * 32 + lane : w * 32 + lane, half = NB == 8 ? w >> 1 : 0, first_block = NB == 8 ? half * 4 : 0;
    int ref = kLowR;
    while (ok && walk.next<NB>(a)) {
      if (values) ref = kLowR;                           // (O begins anew)
      for (int step = u.j0; step < u.j1; ++step, ++jj) {
        const uint32_t ring = values ? C::kRingV : C::kRingK, st = (values ? C::kRingK : 0) + jj % ring, b = jj & (kBufs - 1);
        if (!CAT_WAIT(&bars->raw_full[st], (jj / ring) & 1)) break;
        const uint8_t* raw = smem + C::kOffRaw + st * C::kRaw;
        const uint32_t there = bars->raw_there[st];
        const int64_t token = (int64_t)step * KT + row;
        const bool on = (there >> (row / 16) & 1) && token >= u.t0 && token < u.t1;      // (what no row sees is zeros, and no reference)
        int bytes[kHere];
        uint32_t most = 0, nan = 0;
#pragma unroll
        for (int i = 0; i < kHere; ++i) {
          bytes[i] = on ? raw[C::kCodes + row * NB + first_block + i] : 0;
          if (bytes[i] == 255)
            nan |= 1u << (first_block + i);
          else
            most = max(most, (uint32_t)bytes[i]);
        }
        most = __reduce_max_sync(0xFFFFFFFFu, most);
        __half2 scale[kHere];
        if (values) {
          // The reference is the largest scale so far; tokens have their own instead where some rows see others than others do and those
          // differ, or where what was larger is seen no more, perhaps.
          const bool odd = __any_sync(0xFFFFFFFFu, nan != 0);
          const int64_t t = (int64_t)step * KT;
          const bool partial = max(t, u.t0) < u.a0 || min(t + KT, u.t1) > u.a1;
          auto token_most = [&] {
            int m = 0;
#pragma unroll
            for (int i = 0; i < NB; ++i) {
              const int o = on ? raw[C::kCodes + row * NB + i] : 0;
              if (o != 255) m = max(m, o);
            }
            return m;
          };
          uint32_t least = 255u;
          if (partial) {
            const uint32_t m = (uint32_t)token_most();
            least = __reduce_min_sync(0xFFFFFFFFu, m ? m : 255u);
          }
          if (lane == 0) {
            bars->v_most[jj & 1][w] = most | (odd ? 256u : 0u) | least << 16;
            mbar_arrive(&bars->most_full);
          }
          if (!CAT_WAIT(&bars->most_full, jj & 1)) break;
          uint32_t all = 0;
          int now = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t v = bars->v_most[jj & 1][i];
            all |= v & 256u;
            now = max(now, (int)(v & 255u));
            least = min(least, v >> 16);
          }
          ref = max(ref, now);
          const bool own = now < ref - kBeyond || (int)least < now - kBeyond;
          const int to = own ? token_most() : ref;
#pragma unroll
          for (int i = 0; i < kHere; ++i) scale[i] = on && bytes[i] != 255 ? half_scale(bytes[i], to) : half_scale(-1000, 0);
          if (jj >= kBufs && !CAT_WAIT(&bars->v_empty[b], ((jj >> kBufLog) - 1) & 1)) break;
          bars->v_nan[b][half][row] = (uint8_t)nan;
          if (own && half == 0) bars->v_own[b][row] = (uint8_t)to;
          if (w == 0 && lane == 0) bars->v_ref[b] = (uint32_t)ref | all | (own ? 512u : 0u);
        } else {
          // (d = 256: the two halves' largest differ; the keys' reference is of all their blocks)
          uint32_t mine = 0;
#pragma unroll
          for (int i = 0; i < kHere; ++i)
            if (bytes[i] != 255) mine = max(mine, (uint32_t)bytes[i]);
          if constexpr (NB == 8) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t o = on ? raw[C::kCodes + row * NB + (first_block ^ 4) + i] : 0u;
              if (o != 255u) mine = max(mine, o);
            }
            most = __reduce_max_sync(0xFFFFFFFFu, mine);
          }
          const int kref = max((int)most, kLowR);
          // (a row may see none of the largest, or nothing of what it is large in)
          const bool apart = __any_sync(0xFFFFFFFFu, mine && (int)mine < kref - kKeysApart);
          const int to = apart ? (int)mine : kref;
#pragma unroll
          for (int i = 0; i < kHere; ++i) {
            scale[i] = on ? half_scale(bytes[i], to) : half_scale(-1000, 0);
            if (bytes[i] == 255) scale[i] = __half2half2(__ushort_as_half(0x7FFF));
          }
          if (jj >= kBufs && !CAT_WAIT(&bars->k_empty[b], ((jj >> kBufLog) - 1) & 1)) break;
          if (half == 0) {
            if (apart) bars->k_own[jj & 7][row] = (uint8_t)to;
            if (lane == 0) {
              bars->k_power[jj & 7][row / 32] = kref - 12;
              reinterpret_cast<uint8_t*>(&bars->k_apart[jj & 7])[row / 32] = apart;
            }
          }
          if (w == 0 && lane == 0) bars->there[jj & 7] = there;
        }
        unpack_row<NB>(raw, smem + (values ? C::kOffV : C::kOffK) + b * C::kTile, row, half, values, scale);
        fence_proxy_async_smem();
        __syncwarp();
        if (elect_one()) {
          mbar_arrive(&bars->raw_empty[st]);
          mbar_arrive(values ? &bars->v_full[b] : &bars->k_full[b]);
        }
      }
    }
  } else if (warp == kMmaWarp) {
    // ---------------------------------------------------------------- MMAs
    constexpr uint32_t kScores = idesc_f16(KT, false), kOut = idesc_f16(D, true);
    uint32_t units = 0, tj[2] = {0, 0};
    // (in loops, not in line: this warp's code is not in the instruction cache when its turn comes)
    auto scores = [&](int tile, uint32_t j, uint32_t buffer) {
      uint64_t qd = sdesc_kmajor_sw128(smem_u32(smem + tile * C::kQ)), kd = sdesc_kmajor_sw128(smem_u32(smem + C::kOffK + (j & (kBufs - 1)) * C::kTile));
      const uint32_t to = tmem + (tile * SB + buffer) * KT;
#pragma unroll 1
      for (int kk = 0; kk < D / 16; ++kk) {              // (16 channels are 32 bytes of a row)
        mma_ss(to, qd, kd, kScores, kk);
        qd += (kk & 3) == 3 ? 128 * 128 / 16 - 6 : 2;
        kd += (kk & 3) == 3 ? KT * 128 / 16 - 6 : 2;
      }
      mma_commit(&bars->s_full[tile][buffer]);
    };
    while (ok && walk.next<NB>(a)) {
      if (u.j0 == u.j1) continue;
      const int tiles = u.rows > 128 ? 2 : 1;
      if (!CAT_POLL(&bars->q_full, units & 1)) break;
      ++units;
#pragma unroll 1
      for (int i = 0; i < SB && u.j0 + i < u.j1; ++i) {  // the first scores
        const uint32_t j = jj + i;
        if (!CAT_POLL(&bars->k_full[j & (kBufs - 1)], (j >> kBufLog) & 1)) break;
        tc_fence_after();
        if (elect_one()) {
#pragma unroll 1
          for (int tile = 0; tile < tiles; ++tile) scores(tile, j, (tj[tile] + i) % SB);
          mma_commit(&bars->k_empty[j & (kBufs - 1)]);
        }
        __syncwarp();
      }
      for (int step = u.j0; step < u.j1 && ok; ++step, ++jj) {
        const bool more = step + SB < u.j1;
        const uint32_t vb = jj & (kBufs - 1), ahead = jj + SB;
#pragma unroll 1
        for (int tile = 0; tile < tiles; ++tile) {
          if (tile == 0 && !CAT_POLL(&bars->v_full[vb], (jj >> kBufLog) & 1)) break;
          const uint32_t buffer = tj[tile] % SB;
          if (!CAT_POLL(&bars->p_full[tile][buffer], tj[tile] / SB & 1)) break;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t vd = sdesc_mnmajor_sw128(smem_u32(smem + C::kOffV + vb * C::kTile), KT * 128);
            const uint32_t to = tmem + C::kO + tile * D, p = tmem + (tile * SB + buffer) * KT;
#pragma unroll
            for (int kk = 0; kk < KT / 16; ++kk) mma_ts(to, p + kk * 8, vd + kk * (2048 / 16), kOut, step > u.j0 || kk != 0);
            mma_commit(&bars->pv_done[tile][buffer]);
            if (tile == tiles - 1) mma_commit(&bars->v_empty[vb]);
          }
          __syncwarp();
          if (more) {
            if (tile == 0 && !CAT_POLL(&bars->k_full[ahead & (kBufs - 1)], (ahead >> kBufLog) & 1)) break;
            tc_fence_after();
            if (elect_one()) {
              scores(tile, ahead, buffer);
              if (tile == tiles - 1) mma_commit(&bars->k_empty[ahead & (kBufs - 1)]);
            }
            __syncwarp();
          }
          ++tj[tile];
        }
      }
    }
    if (elect_one()) mma_commit(&bars->mma_done);
    __syncwarp();
    volatile int none = 0;
    mbar_wait_bounded(&bars->mma_done, 0, &none);        // (nothing is on its way to tensor memory any more)
  } else if (warp == kLoadWarp) {
    // ---------------------------------------------------------------- copies
    const int most = a.c.page < KT ? a.c.page : KT, copies = KT / most;      // tokens a copy; copies a step, a lane each
    uint32_t sent[2] = {0, 0};
    while (ok && walk.next<NB>(a)) {
      const int32_t* pages = a.table + (int64_t)u.s * a.width;
      const uint8_t* head = a.c.base + (int64_t)u.h * a.c.part;
      const int64_t page_bytes = 2 * a.c.hkv * a.c.part;
      auto page_of = [&](int step) {                     // of this lane's tokens, -1: none
        const int t0 = step * KT + lane * most;
        if (lane >= copies || step >= u.j1 || t0 >= u.tokens) return -1;
        const int pg = __ldg(pages + (t0 >> a.c.page_log));
        return pg < 0 || pg >= a.pages ? -1 : pg;
      };
      int pg_next = page_of(u.j0);
      for (int step = u.j0; step < u.j1 && ok; ++step, ++jj) {
        const int pg = pg_next, r = (step * KT + lane * most) & (a.c.page - 1), o = lane * most;
        pg_next = page_of(step + 1);
        const uint32_t have = __ballot_sync(0xFFFFFFFFu, pg >= 0);
        uint32_t groups = 0;                             // of 16 tokens
        for (int i = 0; i < copies; ++i)
          if (have >> i & 1) groups |= ((1u << (most / 16)) - 1u) << (i * (most / 16));
#pragma unroll 1
        for (int kind = 0; kind < 2; ++kind) {
          const uint32_t ring = kind ? C::kRingV : C::kRingK, st = (kind ? C::kRingK : 0) + jj % ring;
          if (jj >= ring && !CAT_WAIT(&bars->raw_empty[st], (jj / ring - 1) & 1)) break;
          uint8_t* raw = smem + C::kOffRaw + st * C::kRaw;
          if (lane == 0) {
            bars->raw_there[st] = groups;
            mbar_arrive_expect_tx(&bars->raw_full[st], (uint32_t)(__popc(have) * most * 17 * NB));
          }
          __syncwarp();
          if (pg >= 0) {
            const uint8_t* part = head + pg * page_bytes + kind * a.c.hkv * a.c.part;
            bulk_load(raw + o * (16 * NB), part + r * (16 * NB), most * 16 * NB, &bars->raw_full[st]);
            bulk_load(raw + C::kCodes + o * NB, part + (a.c.page * 16 + r) * NB, most * NB, &bars->raw_full[st]);
          }
          __syncwarp();
          ++sent[kind];
        }
      }
    }
    volatile int none = 0;                               // the last copies have come, whatever became of the others' waits
    for (int kind = 0; kind < 2; ++kind) {
      const uint32_t ring = kind ? C::kRingV : C::kRingK;
      for (uint32_t i = sent[kind] > ring ? sent[kind] - ring : 0; i < sent[kind]; ++i)
        mbar_wait_bounded(&bars->raw_full[(kind ? C::kRingK : 0) + i % ring], (i / ring) & 1, &none);
    }
  }
#undef CAT_WAIT
#undef CAT_POLL
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) tmem_dealloc(tmem, kTmemCols);
  if (tid == 0 && bars->waits.abort) report(a.status, timeout_bits(kWhereMxAttention, bars->waits.abort));
}

template <int NB>
cudaError_t run(const AttnArgs& a, int grid, bool join, cudaStream_t stream) {
  static PerDevice<cudaError_t> allowed;
  // No other kernel's CTA with tensor memory beside this one, which takes all of it.
  constexpr int kSmem = Tc<NB>::kSmem < 216 * 1024 ? 216 * 1024 : Tc<NB>::kSmem;
  cudaError_t e = allowed.get([] { return allow_smem(mx_attention_tiles_kernel<NB>, kSmem); });
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
  e = cudaLaunchKernelEx(&cfg, mx_attention_tiles_kernel<NB>, a);
  if (e != cudaSuccess || !join) return e;
  cfg = join_config(2 * grid * join_split(Tc<NB>::ROWS), stream);      // (its CTAs may wait while the tiles' still work)
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  note_launch();
  return cudaLaunchKernelEx(&cfg, mx_attention_join_kernel<32 * NB, Tc<NB>::ROWS>, a);
}

}  // namespace

cudaError_t set_attention_tiles_wait_limit(uint64_t ns) { return cudaMemcpyToSymbol(g_wait_limit, &ns, sizeof(ns)); }

int attention_tile_rows(int64_t d) { return d == 256 ? Tc<8>::ROWS : Tc<4>::ROWS; }

cudaError_t launch_attention_tiles(const AttnArgs& a, int64_t d, int grid, bool join, cudaStream_t stream) {
  return d == 64 ? run<2>(a, grid, join, stream) : d == 128 ? run<4>(a, grid, join, stream) : run<8>(a, grid, join, stream);
}

}  // namespace cat
