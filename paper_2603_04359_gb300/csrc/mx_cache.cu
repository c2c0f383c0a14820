// Rows of the paged 4-bit key/value cache (mx_cache.cuh): keys and values in, values out, and a fused projection's output
// through its heads' norms and rotation into the cache.
//
// All have little more to do than move bytes: a value costs its input and 17/32 of a byte of the form.  A lane has quarter p of a head's row
// (channels 8 p .. 8 p + 7 of each block of 32), so four neighbouring lanes have a row: they read it in 16-byte pieces, 64 or 128
// bytes side by side, find a block's largest magnitude in two shuffles, and write their quarter of the codes at once.
#include "mx_cache.cuh"

namespace cat {
namespace {

constexpr int kThreads = 128;
constexpr int kFlatBlocks = 16;             // most blocks an SM of a grid-stride loop

__device__ __forceinline__ float lo_f32(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f32(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ void unpack8(const uint4& a, float (&v)[8]) {
  v[0] = lo_f32(a.x), v[1] = hi_f32(a.x), v[2] = lo_f32(a.y), v[3] = hi_f32(a.y);
  v[4] = lo_f32(a.z), v[5] = hi_f32(a.z), v[6] = lo_f32(a.w), v[7] = hi_f32(a.w);
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = __ldcs(reinterpret_cast<const float4*>(p)), b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&v)[8]) {
  unpack8(__ldcs(reinterpret_cast<const uint4*>(p)), v);
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
}

// The larger magnitude; a NaN is larger than all.
__device__ __forceinline__ float max_magnitude(float a, float b) {
  float m;
  asm("{ .reg .f32 x, y; abs.f32 x, %1; abs.f32 y, %2; max.NaN.f32 %0, x, y; }" : "=f"(m) : "f"(a), "f"(b));
  return m;
}
// over the four lanes of a row
__device__ __forceinline__ float row_max(float m) {
  m = max_magnitude(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
  return max_magnitude(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
}
__device__ __forceinline__ float row_sum(float s) {
  s += __shfl_xor_sync(0xFFFFFFFFu, s, 1);
  return s + __shfl_xor_sync(0xFFFFFFFFu, s, 2);
}

// Two float32 operations at once.
__device__ __forceinline__ uint64_t two(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void apart(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// A row's quarter in the 4-bit form: NB words, and the row's NB scale bytes (each lane has all).
template <int NB>
struct Codes {
  uint32_t w[NB], s[(NB + 3) / 4];
  __device__ __forceinline__ void set_scale(int b, uint32_t byte) {
    if (b % 4 == 0) s[b / 4] = 0u;
    s[b / 4] |= byte << (8 * (b & 3));
  }
  // (any b)
  __device__ __forceinline__ void replace(int b, uint32_t codes, uint32_t byte) {
#pragma unroll
    for (int i = 0; i < NB; ++i)
      if (i == b) {
        w[i] = codes;
        s[i / 4] = (s[i / 4] & ~(0xFFu << (8 * (i & 3)))) | byte << (8 * (i & 3));
      }
  }
  __device__ __forceinline__ uint32_t scale(int b) const { return s[b / 4] >> (8 * (b & 3)) & 0xFFu; }
  // Values' pieces are halfwords: a quarter is the low halves of all words, then the high ones.
  __device__ __forceinline__ void to_pieces() {
    uint32_t t[NB];
#pragma unroll
    for (int i = 0; i < NB / 2; ++i) {
      t[i] = __byte_perm(w[2 * i], w[2 * i + 1], 0x5410);
      t[NB / 2 + i] = __byte_perm(w[2 * i], w[2 * i + 1], 0x7632);
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) w[i] = t[i];
  }
  __device__ __forceinline__ void from_pieces() {
    uint32_t t[NB];
#pragma unroll
    for (int i = 0; i < NB / 2; ++i) {
      t[2 * i] = __byte_perm(w[i], w[NB / 2 + i], 0x5410);
      t[2 * i + 1] = __byte_perm(w[i], w[NB / 2 + i], 0x7632);
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) w[i] = t[i];
  }
  // to and from place `r` of a head's part of a page
  __device__ __forceinline__ void store(uint8_t* part, int page, int r, int p, int kind) {
    if (kind) to_pieces();
    uint8_t* at = part + (int64_t)r * (16 * NB) + p * (4 * NB);
    if constexpr (NB == 2) {
      *reinterpret_cast<uint2*>(at) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
      for (int i = 0; i < NB; i += 4) reinterpret_cast<uint4*>(at)[i / 4] = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
    }
    if (p == 0) {
      uint8_t* sc = part + (int64_t)page * (16 * NB) + r * NB;
      if constexpr (NB == 2)
        *reinterpret_cast<uint16_t*>(sc) = (uint16_t)s[0];
      else if constexpr (NB == 4)
        *reinterpret_cast<uint32_t*>(sc) = s[0];
      else
        *reinterpret_cast<uint2*>(sc) = make_uint2(s[0], s[1]);
    }
  }
  __device__ __forceinline__ void load(const uint8_t* part, int page, int r, int p, int kind) {
    const uint8_t* at = part + (int64_t)r * (16 * NB) + p * (4 * NB);
    const uint8_t* sc = part + (int64_t)page * (16 * NB) + r * NB;
    if constexpr (NB == 2) {
      const uint2 a = *reinterpret_cast<const uint2*>(at);
      w[0] = a.x, w[1] = a.y;
      s[0] = *reinterpret_cast<const uint16_t*>(sc);
    } else {
#pragma unroll
      for (int i = 0; i < NB; i += 4) {
        const uint4 a = reinterpret_cast<const uint4*>(at)[i / 4];
        w[i] = a.x, w[i + 1] = a.y, w[i + 2] = a.z, w[i + 3] = a.w;
        s[i / 4] = reinterpret_cast<const uint32_t*>(sc)[i / 4];
      }
    }
    if (kind) from_pieces();
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < NB; ++i) w[i] = 0u;
#pragma unroll
    for (int i = 0; i < (NB + 3) / 4; ++i) s[i] = 0u;
  }
};

// The 4-bit form of a block (whole warps); whether it is not finite.
template <int NB>
__device__ __forceinline__ bool quantize_block(const float (&v)[8], int b, Codes<NB>& out) {
  float a = max_magnitude(max_magnitude(max_magnitude(v[0], v[1]), max_magnitude(v[2], v[3])),
                          max_magnitude(max_magnitude(v[4], v[5]), max_magnitude(v[6], v[7])));
  a = row_max(a);
  const uint32_t byte = mx_scale_byte(__float_as_uint(a));
  const float inv = byte == 255u ? 0.f : mx_inverse_scale(byte);
  float u[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) u[i] = v[i] * inv;
  out.w[b] = byte == 255u ? 0u : mx_pack8(u);
  out.set_scale(b, byte);
  return byte == 255u;
}

// Rows of (token, head) in a grid-stride loop of quarters: token and head counted on, not divided.
struct Rows {
  int64_t token;
  int head;
  __device__ __forceinline__ Rows(int64_t i, int heads) : token(i / heads), head((int)(i - token * heads)) {}
  __device__ __forceinline__ void next(int64_t step_tokens, int step_heads, int heads) {
    token += step_tokens;
    head += step_heads;
    if (head >= heads) {
      head -= heads;
      ++token;
    }
  }
};

// blockIdx.y: 0 keys, 1 values.  Bound by memory: 8000 float32 tokens of 16 heads of 64 channels, 74 MB, 12.3 us (6.0 TB/s).
template <typename T, int NB>
__global__ void __launch_bounds__(kThreads) mx_cache_write_kernel(const T* __restrict__ k, const T* __restrict__ v, int64_t n,
                                                                  const int32_t* __restrict__ slots, MxCache c,
                                                                  int64_t step_tokens, int step_heads, uint32_t* __restrict__ status) {
  const int kind = blockIdx.y, lane = threadIdx.x & 31, p = lane & 3;
  const T* x = kind ? v : k;
  const int64_t total = n * c.hkv, stride = (int64_t)gridDim.x * (kThreads / 4);
  int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / 4;
  Rows row(i, c.hkv);
  pdl_wait_then_release();
  bool bad = false;
  for (; i - lane / 4 < total; i += stride, row.next(step_tokens, step_heads, c.hkv)) {      // (whole warps: the shuffles)
    int64_t slot = -1;
    if (i < total) slot = slots[row.token];
    const bool in = slot >= 0 && slot < c.rows;
    Codes<NB> out;
    float f[NB][8];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      if (in) {
        load8(x + i * (32 * NB) + 32 * b + 8 * p, f[b]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[b][j] = 0.f;
      }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) bad |= quantize_block<NB>(f[b], b, out);
    if (in) out.store(c.at(slot >> c.page_log, kind, row.head), c.page, (int)(slot & (c.page - 1)), p, kind);
  }
  if (__any_sync(0xFFFFFFFFu, bad) && lane == 0) report(status, kStatusNonFinite);
}

// Two E2M1 codes (nibbles 0 and 1 of c) as bf16 values 2^126 too small, the first in the low half: the code's magnitude
// bits are a bf16's last exponent bits and first mantissa bit (a subnormal for 0.5).
__device__ __forceinline__ uint32_t code_pair(uint32_t c) {
  return ((c & 7u) << 6) | ((c & 0x70u) << 18) | ((c & 8u) << 12) | ((c & 0x80u) << 24);
}
// times 2^126, then the scale: each exact (one factor for both could be out of range)
__device__ __forceinline__ void values8(uint32_t w, uint32_t byte, float (&v)[8]) {
  const float s = mx_scale(byte);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t p = code_pair(w >> (8 * i));
    v[2 * i] = lo_f32(p) * 0x1p126f * s;
    v[2 * i + 1] = hi_f32(p) * 0x1p126f * s;
  }
}

// Bound by memory: 32768 tokens of 8 heads of 128 channels to bf16, 170 MB, 27.7 us (6.1 TB/s).
template <typename T, int NB>
__global__ void __launch_bounds__(kThreads) mx_cache_read_kernel(MxCache c, const int32_t* __restrict__ slots, int64_t m,
                                                                 int64_t step_tokens, int step_heads, T* __restrict__ k,
                                                                 T* __restrict__ v) {
  const int kind = blockIdx.y, p = threadIdx.x & 3;
  T* out = kind ? v : k;
  const int64_t total = m * c.hkv, stride = (int64_t)gridDim.x * (kThreads / 4);
  int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / 4;
  Rows row(i, c.hkv);
  pdl_wait_then_release();
  for (; i < total; i += stride, row.next(step_tokens, step_heads, c.hkv)) {
    const int64_t slot = slots[row.token];
    Codes<NB> in;
    if (slot >= 0 && slot < c.rows)
      in.load(c.at(slot >> c.page_log, kind, row.head), c.page, (int)(slot & (c.page - 1)), p, kind);
    else
      in.zero();
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      float f[8];
      values8(in.w[b], in.scale(b), f);
      store8(out + i * (32 * NB) + 32 * b + 8 * p, f);
    }
  }
}

// ---- head norms, rotation, and the cache

struct RopeArgs {
  const void* qkv;
  int64_t n;
  int hq, heads, groups;                    // heads: hq + 2 hkv; groups: warps a token, eight heads each
  const void *q_weight, *k_weight;
  int weight_f32;
  double eps;
  const int32_t* positions;
  const float *cos, *sin;
  int64_t table_rows;
  int rot;
  const int32_t* slots;
  MxCache c;
  __nv_bfloat16* q_out;
  uint32_t* status;
};

// How a pair's channels lie: neighbours; D / 2 apart (a whole head turned) or D / 4 (half of it), in one lane; any other distance
// (a multiple of 8: the partner is read again, from the cache).
enum { kNeighbours = 0, kHalves = 1, kQuarters = 2, kAnyHalves = 3 };

__device__ __forceinline__ void load4(const float* p, float (&v)[8], int at) {
  const float4 f = __ldg(reinterpret_cast<const float4*>(p));
  v[at] = f.x, v[at + 1] = f.y, v[at + 2] = f.z, v[at + 3] = f.w;
}
__device__ __forceinline__ void load_weight8(const RopeArgs& a, const void* w, int c, float (&v)[8]) {
  if (a.weight_f32) {
    load4(static_cast<const float*>(w) + c, v, 0);
    load4(static_cast<const float*>(w) + c + 4, v, 4);
  } else {
    const uint4 u = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(w) + c));
    unpack8(u, v);
  }
}

// The factors of channels c .. c + 7: y_i = x_i co[i] + x_partner(i) si[i].
template <bool NEIGHBOURS>
__device__ __forceinline__ void turn_factors(const RopeArgs& a, int64_t pos, int c, float (&co)[8], float (&si)[8]) {
  const int half = a.rot / 2;
  const float *cs = a.cos + pos * half, *sn = a.sin + pos * half;
  if constexpr (NEIGHBOURS) {
    float u[8], w[8];
    load4(cs + c / 2, u, 0);
    load4(sn + c / 2, w, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      co[2 * i] = co[2 * i + 1] = u[i];
      si[2 * i] = -w[i];
      si[2 * i + 1] = w[i];
    }
  } else {
    const int at = c < half ? c : c - half;
    load4(cs + at, co, 0);
    load4(cs + at + 4, co, 4);
    load4(sn + at, si, 0);
    load4(sn + at + 4, si, 4);
    if (c < half)
#pragma unroll
      for (int i = 0; i < 8; ++i) si[i] = -si[i];
  }
}

__device__ __forceinline__ double row_sum(double s) {
  s += __shfl_xor_sync(0xFFFFFFFFu, s, 1);
  return s + __shfl_xor_sync(0xFFFFFFFFu, s, 2);
}

// A double as a float whose last bit says whether anything was cut off: it compares with the middles between E2M1 values, and
// rounds to them, as the double does.
__device__ __forceinline__ float sticky(double v) {
  const float f = __double2float_rz(v);
  return (double)f == v || !isfinite(v) ? f : __uint_as_float(__float_as_uint(f) | 1u);
}

// a + b as a sum and its error
__device__ __forceinline__ void two_sum(float a, float b, float& s, float& e) {
  s = __fadd_rn(a, b);
  const float t = __fsub_rn(s, a);
  e = __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t));
}

// A key's quarter of the blocks in `blocks` (the same in all lanes) from its exact values, read again and computed in float64: some
// hundred operations of it, whose rate is 1/64 of float32's, so that the squares are summed in pairs of float32 (to some 2^-45) and no
// more blocks are done than have to be.  Whole warps; lanes without a key (on = false) take part in the shuffles only.
template <typename T, int NB>
__device__ __noinline__ void exact_key(const RopeArgs& a, const T* x, const void* weight, bool neighbours, int64_t pos, bool valid,
                                       bool on, int p, uint32_t blocks, Codes<NB>* out) {
  float f[8], w[8], g[8];
  double r = 1.0;
  if (__any_sync(0xFFFFFFFFu, on && weight)) {
    double sum = 0.0;
    if (on && weight) {
      float hi = 0.f, lo = 0.f;
      bool odd = false;                                  // squares that leave the range where the errors are exact
#pragma unroll 1
      for (int b = 0; b < NB; ++b) {
        load8(x + 32 * b + 8 * p, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float sq = __fmul_rn(f[i], f[i]), low = __fmaf_rn(f[i], f[i], -sq);
          float e;
          odd |= f[i] != 0.f && !(sq > 0x1p-100f && sq < 0x1p100f);
          two_sum(hi, sq, hi, e);
          lo = __fadd_rn(lo, __fadd_rn(e, low));
        }
      }
      sum = (double)hi + (double)lo;
      if (odd) {
        sum = 0.0;
#pragma unroll 1
        for (int b = 0; b < NB; ++b) {
          load8(x + 32 * b + 8 * p, f);
#pragma unroll 1
          for (int i = 0; i < 8; ++i) sum += (double)f[i] * (double)f[i];
        }
      }
    }
    sum = row_sum(sum);
    if (weight) r = 1.0 / sqrt(sum / (32 * NB) + a.eps);
  }
#pragma unroll 1
  for (int b = 0; b < NB; ++b) {
    if (!(blocks >> b & 1u)) continue;
    const int c = 32 * b + 8 * p;
    double y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = 0.0;
    if (on) {
      load8(x + c, f);
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = 1.f;
      if (weight) load_weight8(a, weight, c, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = weight ? (double)f[i] * (double)w[i] : (double)f[i];
      if (c < a.rot && valid) {
        float co[8], si[8];
        double z[8];
        if (neighbours) {
          turn_factors<true>(a, pos, c, co, si);
#pragma unroll
          for (int i = 0; i < 8; ++i) z[i] = y[i ^ 1];
        } else {
          turn_factors<false>(a, pos, c, co, si);
          const int o = c < a.rot / 2 ? c + a.rot / 2 : c - a.rot / 2;
          load8(x + o, g);
          if (weight) load_weight8(a, weight, o, w);
#pragma unroll
          for (int i = 0; i < 8; ++i) z[i] = weight ? (double)g[i] * (double)w[i] : (double)g[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = y[i] * (double)co[i] + z[i] * (double)si[i];
      }
      if (weight)
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] *= r;
      if (!valid)
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __longlong_as_double(0x7FF8000000000000ll);
    }
    // magnitudes as integers compare like the numbers
    int64_t big = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t m = __double_as_longlong(y[i]) & 0x7FFFFFFFFFFFFFFFll;
      big = m > big ? m : big;
    }
    const int64_t o1 = __shfl_xor_sync(0xFFFFFFFFu, big, 1);
    big = o1 > big ? o1 : big;
    const int64_t o2 = __shfl_xor_sync(0xFFFFFFFFu, big, 2);
    big = o2 > big ? o2 : big;
    // floor(log2 most) + 125: of a double's exponent field 1023 + e (2047: not finite)
    const int e = (int)(big >> 52) - 1023 + 125;
    const uint32_t byte = e > 254 ? 255u : e > 0 ? (uint32_t)e : 0u;
    float u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = byte == 255u ? 0.f : sticky(y[i] * __longlong_as_double((int64_t)(1150 - (int)byte) << 52));
    const uint32_t codes = byte == 255u ? 0u : mx_pack8(u);
    if (on) out->replace(b, codes, byte);
  }
}

// A number as the sum of two float32, the second some units of the first at most.
struct Pair {
  float h, l;
};
__device__ __forceinline__ Pair product(float a, float b) {
  const float h = __fmul_rn(a, b);
  return {h, __fmaf_rn(a, b, -h)};
}
__device__ __forceinline__ Pair times(Pair a, float b) {
  const float h = __fmul_rn(a.h, b);
  return {h, __fmaf_rn(a.l, b, __fmaf_rn(a.h, b, -h))};
}
__device__ __forceinline__ Pair times(Pair a, Pair b) {
  const float h = __fmul_rn(a.h, b.h);
  return {h, __fmaf_rn(a.h, b.l, __fmaf_rn(a.l, b.h, __fmaf_rn(a.h, b.h, -h)))};
}
__device__ __forceinline__ Pair plus(Pair a, Pair b) {
  Pair s;
  float e;
  two_sum(a.h, b.h, s.h, e);
  e = __fadd_rn(e, __fadd_rn(a.l, b.l));
  const float h = __fadd_rn(s.h, e);
  return {h, __fsub_rn(e, __fsub_rn(h, s.h))};
}
// The float32 that rounds, and compares with powers of two, as the pair does: the nearest, moved by a unit toward the rest's side where
// that could be a border (few bits of the significand are set).
__device__ __forceinline__ float nudged(Pair v) {
  const float h = __fadd_rn(v.h, v.l), l = __fsub_rn(v.l, __fsub_rn(h, v.h));
  const uint32_t u = __float_as_uint(h);
  if ((u & 0xFFFFu) != 0u || l == 0.f || h == 0.f) return h;
  return __uint_as_float((l > 0.f) == (h > 0.f) ? u + 1u : u - 1u);
}

// exact_key for values of ordinary sizes, in pairs of float32: to some 2^-43 of |y co| + |y' si|, where float64's few and slow units
// took 6 us for a key (999 tokens of 48 heads without a norm: 12 us with them, 6 without any such key).
template <typename T, int NB>
__device__ __noinline__ void near_key(const RopeArgs& a, const T* x, const void* weight, bool neighbours, int64_t pos, bool on, int p,
                                      uint32_t blocks, Codes<NB>* out) {
  float f[8], w[8];
  Pair r = {1.f, 0.f};
  if (__any_sync(0xFFFFFFFFu, on && weight)) {
    Pair sum = {0.f, 0.f};
    if (on && weight)
#pragma unroll 1
      for (int b = 0; b < NB; ++b) {
        load8(x + 32 * b + 8 * p, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const Pair q = product(f[i], f[i]);
          float e;
          two_sum(sum.h, q.h, sum.h, e);
          sum.l = __fadd_rn(sum.l, __fadd_rn(e, q.l));
        }
      }
#pragma unroll
    for (int k = 1; k < 4; k <<= 1) {
      const Pair other = {__shfl_xor_sync(0xFFFFFFFFu, sum.h, k), __shfl_xor_sync(0xFFFFFFFFu, sum.l, k)};
      sum = plus(sum, other);
    }
    if (weight) {
      // m to the power -1/2: the rounded root, and a step of Newton's from it
      const float eps = (float)a.eps;
      const Pair m = plus({sum.h * (1.f / (32 * NB)), sum.l * (1.f / (32 * NB))}, {eps, (float)(a.eps - (double)eps)});
      const float r0 = __frsqrt_rn(m.h);
      const Pair t = times(product(r0, r0), m);
      r = {r0, 0.5f * r0 * __fsub_rn(__fsub_rn(1.f, t.h), t.l)};
    }
  }
#pragma unroll 1
  for (int b = 0; b < NB; ++b) {
    if (!(blocks >> b & 1u)) continue;
    const int c = 32 * b + 8 * p;
    Pair y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = {0.f, 0.f};
    if (on) {
      load8(x + c, f);
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = 1.f;
      if (weight) load_weight8(a, weight, c, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = product(f[i], weight ? w[i] : 1.f);
      if (c < a.rot) {
        float co[8], si[8];
        if (neighbours) {
          turn_factors<true>(a, pos, c, co, si);
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            const Pair u = y[i], v = y[i + 1];
            y[i] = plus(times(u, co[i]), times(v, si[i]));
            y[i + 1] = plus(times(v, co[i + 1]), times(u, si[i + 1]));
          }
        } else {
          turn_factors<false>(a, pos, c, co, si);
          const int o = c < a.rot / 2 ? c + a.rot / 2 : c - a.rot / 2;
          load8(x + o, f);
          if (weight) load_weight8(a, weight, o, w);
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = plus(times(y[i], co[i]), times(product(f[i], weight ? w[i] : 1.f), si[i]));
        }
      }
      if (weight)
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = times(y[i], r);
    }
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(nudged(y[i])));
    m = row_max(m);
    const uint32_t byte = mx_scale_byte(__float_as_uint(m));
    const float inv = mx_inverse_scale(byte);            // (finite: of ordinary sizes)
    float u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = nudged(y[i]) * inv;
    const uint32_t codes = mx_pack8(u);
    if (on) out->replace(b, codes, byte);
  }
}

// float32's error in a key's channel y = r w x co + r w' x' si, relative to m = |r w x co| + |r w' x' si|: r's is at most 12 units
// of 2^-24 (a row's squares summed in four chains and two levels, at most 20 roundings, half of which the root passes on; its
// own and eps's), the two products with r and w 2, those with co and si and the sum 2, and the margin's own arithmetic 1: 17.  20
// units are allowed here.  Where y minus and plus that have the same code, and the block's largest magnitude the same exponent,
// the key's code is that of the exact value.
constexpr float kMargin = 20.f * 0x1p-24f;

// A warp has eight heads of a token, four lanes a head, its values in registers from the norm to the codes.  8192 tokens of 80 heads of 128 channels
// in bf16, 311 MB, 78 us (4.0 TB/s): a warp's loads come at its beginning, and the 28 warps of an SM (72 registers) are too few to hide them
// behind one another's arithmetic (2.2 instructions a cycle); with 24 warps, and a channel at a time instead of two, 118.
template <typename T, int NB, int PAIRS>
__global__ void __launch_bounds__(kThreads, NB == 8 ? 4 : 7) mx_rope_kernel(const __grid_constant__ RopeArgs a) {
  constexpr int D = 32 * NB;
  const int lane = threadIdx.x & 31, p = lane & 3;
  const int64_t item = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 5;
  const int64_t t = item / a.groups;
  pdl_wait_then_release();
  if (t >= a.n) return;                                  // (a warp's lanes have one token)
  const int head = (int)(item - t * a.groups) * 8 + lane / 4;
  const bool in = head < a.heads, is_q = head < a.hq, is_v = head >= a.hq + a.c.hkv, is_k = in && !is_q && !is_v;
  const void* weight = is_q ? a.q_weight : is_v ? nullptr : a.k_weight;
  const int64_t pos = a.positions[t];
  const bool valid = is_v || (pos >= 0 && pos < a.table_rows);
  int64_t slot = -1;
  if (in && !is_q) slot = a.slots[t];
  const T* x = static_cast<const T*>(a.qkv) + (t * a.heads + head) * D;

  float y[NB][8], sq[4];
  uint64_t sq2[2] = {0ull, 0ull};
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    if (in) {
      load8(x + 32 * b + 8 * p, y[b]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[b][i] = 0.f;
    }
  }
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const uint64_t v = two(y[b][i], y[b][i + 1]);
      sq2[i / 2 & 1] = fma2(v, v, sq2[i / 2 & 1]);
    }
  apart(sq2[0], sq[0], sq[1]);
  apart(sq2[1], sq[2], sq[3]);
  const float mean = row_sum((sq[0] + sq[1]) + (sq[2] + sq[3])) * (1.f / D) + (float)a.eps;
  float r = __frsqrt_rn(mean);
  // Squares that leave float32's range, though the norm does not: summed again in float64.
  const bool odd = in && weight && !(mean >= 0x1p-80f && mean < __int_as_float(0x7F800000));
  if (__any_sync(0xFFFFFFFFu, odd)) {
    double s = 0.0;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 8; ++i) s += (double)y[b][i] * (double)y[b][i];
    s = row_sum(s);
    if (odd) r = (float)(1.0 / sqrt(s / D + a.eps));
  }
  if (in && weight) {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      float w[8];
      load_weight8(a, weight, 32 * b + 8 * p, w);
      const uint64_t rr = two(r, r);
#pragma unroll
      for (int i = 0; i < 8; i += 2) apart(mul2(mul2(two(y[b][i], y[b][i + 1]), rr), two(w[i], w[i + 1])), y[b][i], y[b][i + 1]);
    }
  }
  float most[NB];                                        // keys: of |y co| + |y' si|
#pragma unroll
  for (int b = 0; b < NB; ++b) most[b] = 0.f;
  const bool keys = __any_sync(0xFFFFFFFFu, is_k);
  if (in && !is_v && valid) {
    if constexpr (PAIRS == kHalves || PAIRS == kQuarters) {
      constexpr int kApart = PAIRS == kHalves ? NB / 2 : NB / 4;
#pragma unroll
      for (int b = 0; b < kApart; ++b) {
        float co[8], si[8];
        turn_factors<false>(a, pos, 32 * b + 8 * p, co, si);     // (si is -sin here)
        if (keys) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float u = y[b][i], v = y[b + kApart][i];
            most[b] = fmaxf(most[b], fabsf(u * co[i]) + fabsf(v * si[i]));
            most[b + kApart] = fmaxf(most[b + kApart], fabsf(v * co[i]) + fabsf(u * si[i]));
          }
        }
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const uint64_t u = two(y[b][i], y[b][i + 1]), v = two(y[b + kApart][i], y[b + kApart][i + 1]);
          const uint64_t c2 = two(co[i], co[i + 1]), s2 = two(si[i], si[i + 1]), n2 = two(-si[i], -si[i + 1]);
          apart(fma2(v, s2, mul2(u, c2)), y[b][i], y[b][i + 1]);
          apart(fma2(u, n2, mul2(v, c2)), y[b + kApart][i], y[b + kApart][i + 1]);
        }
      }
    } else {
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int c = 32 * b + 8 * p;
        if (c < a.rot) {
          float co[8], si[8], z[8];
          turn_factors<PAIRS == kNeighbours>(a, pos, c, co, si);
          if constexpr (PAIRS == kNeighbours) {
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = y[b][i ^ 1];
          } else {
            const int o = c < a.rot / 2 ? c + a.rot / 2 : c - a.rot / 2;
            load8(x + o, z);
            if (weight) {
              float w[8];
              load_weight8(a, weight, o, w);
#pragma unroll
              for (int i = 0; i < 8; ++i) z[i] = z[i] * r * w[i];
            }
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float yc = y[b][i] * co[i];
            if (keys) most[b] = fmaxf(most[b], fabsf(yc) + fabsf(z[i] * si[i]));
            y[b][i] = fmaf(z[i], si[i], yc);
          }
        }
      }
    }
  }
  if (!valid) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 8; ++i) y[b][i] = __int_as_float(0x7FFFFFFF);
  }
  if (in && is_q) {
#pragma unroll
    for (int b = 0; b < NB; ++b) store8(a.q_out + (t * a.hq + head) * D + 32 * b + 8 * p, y[b]);
    if (!valid && p == 0) report(a.status, kStatusNonFinite);
  }
  const bool writes = slot >= 0 && slot < a.c.rows;
  if (!__any_sync(0xFFFFFFFFu, writes)) return;

  Codes<NB> out;
  uint32_t near = odd && is_k ? (1u << NB) - 1u : 0u;    // blocks whose codes float32's error could change
  bool far = odd || !valid || (weight && !(mean < 0x1p100f));
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max_magnitude(m, y[b][i]);
    m = row_max(m);
    float e = 0.f, all = 0.f;
    if (keys) {                                          // (all lanes shuffle, whatever their heads are; channels that are not turned)
      all = fmaxf(row_max(most[b]), m);
      if (is_k) e = all * kMargin;
    }
    const uint32_t byte = mx_scale_byte(__float_as_uint(m));
    const float inv = byte == 255u ? 0.f : mx_inverse_scale(byte);
    float u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = y[b][i] * inv;
    out.w[b] = byte == 255u ? 0u : mx_pack8(u);
    out.set_scale(b, byte);
    if (keys) {
      float below[8], above[8];
      const float margin = e * inv;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        below[i] = u[i] - margin;
        above[i] = u[i] + margin;
      }
      // (codes that differ in their signs alone are 0 and -0)
      if (is_k && (byte == 255u || ((mx_pack8(below) ^ mx_pack8(above)) & 0x77777777u) != 0u ||
                   mx_scale_byte(__float_as_uint(fmaxf(m - e, 0.f))) != byte || mx_scale_byte(__float_as_uint(m + e)) != byte))
        near |= 1u << b;
      // sizes at which pairs of float32 would lose bits (nothing tells what a NaN or an infinity is made of)
      far |= is_k && !((m > 0x1p-40f || all == 0.f) && e < 0x1p40f && byte != 255u);
    }
  }
  const uint32_t blocks = __reduce_or_sync(0xFFFFFFFFu, near);
  if (blocks) {
    if (__any_sync(0xFFFFFFFFu, is_k && far))            // (all of the warp's keys get these blocks anew)
      exact_key<T, NB>(a, x, weight, PAIRS == kNeighbours, pos, valid, is_k, p, blocks, &out);
    else
      near_key<T, NB>(a, x, weight, PAIRS == kNeighbours, pos, is_k, p, blocks, &out);
  }
  bool bad = false;
#pragma unroll
  for (int b = 0; b < NB; ++b) bad |= out.scale(b) == 255u;
  if (writes) {
    const int kind = is_v, h = head - a.hq - (is_v ? a.c.hkv : 0);
    out.store(a.c.at(slot >> a.c.page_log, kind, h), a.c.page, (int)(slot & (a.c.page - 1)), p, kind);
    if (bad && p == 0) report(a.status, kStatusNonFinite);
  }
}

int sm_count() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 148;
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms <= 0) return 148;
  return sms;
}

template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, cudaStream_t stream, A... args) {
  note_launch();
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.stream = stream;
  cudaLaunchAttribute attr = pdl_attr();
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

// Blocks of a grid-stride loop over the rows' quarters, and its stride in tokens and heads.
struct Flat {
  int64_t blocks, step_tokens;
  int step_heads;
  Flat(int64_t n, int heads) {
    const int64_t want = (n * heads * 4 + kThreads - 1) / kThreads, cap = (int64_t)sm_count() * kFlatBlocks;
    blocks = want < cap ? want : cap;
    step_tokens = blocks * (kThreads / 4) / heads;
    step_heads = (int)(blocks * (kThreads / 4) % heads);
  }
};

MxCache cache_of(const uint8_t* base, int64_t pages, int64_t page, int64_t hkv, int64_t d) {
  int log = 0;
  while ((int64_t(1) << log) < page) ++log;
  return {const_cast<uint8_t*>(base), pages * page, (int)page, log, (int)hkv, mx_page_bytes(page, d)};
}

template <typename T, int NB>
cudaError_t write(const void* k, const void* v, int64_t n, const int32_t* slots, const MxCache& c, uint32_t* status,
                  cudaStream_t stream) {
  const Flat f(n, c.hkv);
  return launch(mx_cache_write_kernel<T, NB>, dim3((unsigned)f.blocks, 2), stream, static_cast<const T*>(k), static_cast<const T*>(v),
                n, slots, c, f.step_tokens, f.step_heads, status);
}
template <typename T>
cudaError_t write_d(const void* k, const void* v, int64_t n, const int32_t* slots, const MxCache& c, int64_t d, uint32_t* status,
                    cudaStream_t s) {
  return d == 64    ? write<T, 2>(k, v, n, slots, c, status, s)
         : d == 128 ? write<T, 4>(k, v, n, slots, c, status, s)
                    : write<T, 8>(k, v, n, slots, c, status, s);
}

template <typename T, int NB>
cudaError_t read(const MxCache& c, const int32_t* slots, int64_t m, void* k, void* v, cudaStream_t stream) {
  const Flat f(m, c.hkv);
  return launch(mx_cache_read_kernel<T, NB>, dim3((unsigned)f.blocks, 2), stream, c, slots, m, f.step_tokens, f.step_heads,
                static_cast<T*>(k), static_cast<T*>(v));
}
template <typename T>
cudaError_t read_d(const MxCache& c, const int32_t* slots, int64_t m, int64_t d, void* k, void* v, cudaStream_t s) {
  return d == 64 ? read<T, 2>(c, slots, m, k, v, s) : d == 128 ? read<T, 4>(c, slots, m, k, v, s) : read<T, 8>(c, slots, m, k, v, s);
}

template <typename T, int NB>
cudaError_t rope(const RopeArgs& a, int interleaved, cudaStream_t stream) {
  const int64_t blocks = (a.n * a.groups + kThreads / 32 - 1) / (kThreads / 32);
  if (blocks > 0x7FFFFFFF) return cudaErrorInvalidValue;
  const dim3 grid((unsigned)blocks);
  if (interleaved) return launch(mx_rope_kernel<T, NB, kNeighbours>, grid, stream, a);
  if (a.rot == 32 * NB) return launch(mx_rope_kernel<T, NB, kHalves>, grid, stream, a);
  if constexpr (NB > 2)
    if (a.rot == 16 * NB) return launch(mx_rope_kernel<T, NB, kQuarters>, grid, stream, a);
  return launch(mx_rope_kernel<T, NB, kAnyHalves>, grid, stream, a);
}
template <typename T>
cudaError_t rope_d(const RopeArgs& a, int64_t d, int interleaved, cudaStream_t s) {
  return d == 64 ? rope<T, 2>(a, interleaved, s) : d == 128 ? rope<T, 4>(a, interleaved, s) : rope<T, 8>(a, interleaved, s);
}

}  // namespace

cudaError_t launch_mx_cache_write(const void* k, const void* v, int dtype, int64_t n, const int32_t* slots, uint8_t* cache,
                                  int64_t pages, int64_t page, int64_t hkv, int64_t d, uint32_t* status, cudaStream_t stream) {
  const MxCache c = cache_of(cache, pages, page, hkv, d);
  return dtype == 0 ? write_d<float>(k, v, n, slots, c, d, status, stream) : write_d<__nv_bfloat16>(k, v, n, slots, c, d, status, stream);
}

cudaError_t launch_mx_cache_read(const uint8_t* cache, int64_t pages, int64_t page, int64_t hkv, int64_t d, const int32_t* slots,
                                 int64_t m, int dtype, void* k, void* v, cudaStream_t stream) {
  const MxCache c = cache_of(cache, pages, page, hkv, d);
  return dtype == 0 ? read_d<float>(c, slots, m, d, k, v, stream) : read_d<__nv_bfloat16>(c, slots, m, d, k, v, stream);
}

cudaError_t launch_mx_rope(const void* qkv, int dtype, int64_t n, int64_t hq, const void* q_weight, const void* k_weight,
                           int weight_dtype, double eps, const int32_t* positions, const float* cos, const float* sin,
                           int64_t table_rows, int64_t rot, int interleaved, const int32_t* slots, uint8_t* cache, int64_t pages,
                           int64_t page, int64_t hkv, int64_t d, void* q_out, uint32_t* status, cudaStream_t stream) {
  RopeArgs a = {};
  a.qkv = qkv, a.n = n, a.hq = (int)hq, a.heads = (int)(hq + 2 * hkv), a.groups = (a.heads + 7) / 8;
  a.q_weight = q_weight, a.k_weight = k_weight, a.weight_f32 = weight_dtype == 0, a.eps = eps;
  a.positions = positions, a.cos = cos, a.sin = sin, a.table_rows = table_rows, a.rot = (int)rot;
  a.slots = slots, a.c = cache_of(cache, pages, page, hkv, d), a.q_out = static_cast<__nv_bfloat16*>(q_out), a.status = status;
  return dtype == 0 ? rope_d<float>(a, d, interleaved, stream) : rope_d<__nv_bfloat16>(a, d, interleaved, stream);
}

}  // namespace cat
