// Row kernels of the microscaled 4-bit format: quantization of activations and weights (with a gather of rows for
// experts' tokens), of SwiGLU's product, and of a root-mean-square norm with the residual's addition; dequantization.
//
// All are bound by the bytes that they move: every input is read once and the 4-bit form (17/32 of a byte a value) is
// all that is written beside the norm's sum, so the norm's or SwiGLU's 16-bit output never goes through memory.
//
// Memory gives an SM 22 bytes a cycle, 256 bf16 values in 23 cycles: what bounds these kernels in practice are the
// instructions a value takes.  So a thread of the flat kernels takes 16 consecutive values in one 32-byte load, two lanes a
// block of 32, bf16 values are compared and scaled two at a time, places are counted on instead of divided, and the row
// numbers of a gather have a kernel of their own.  Codes leave 8 bytes a lane, a warp's scales are 16 neighbouring bytes.
#include "mx_format.cuh"

namespace cat {
namespace {

constexpr int kThreads = 256;
constexpr int kWarpOcts = 64;     // rows of a norm up to this have a warp each (8192 x 256 bf16 4.5 us, a CTA each 8.7; x 768 13.5, 12.3)
constexpr int kFlatBlocks = 32;  // most blocks an SM of a grid-stride loop

struct Oct {
  float v[8];
};

__device__ __forceinline__ float lo_f32(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f32(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

__device__ __forceinline__ __nv_bfloat162 bf16_pair(uint32_t bits) {
  const uint32_t two = bits | (bits << 16);
  return *reinterpret_cast<const __nv_bfloat162*>(&two);
}

__device__ __forceinline__ Oct load_oct(const float* p) {
  const float4 a = __ldcs(reinterpret_cast<const float4*>(p)), b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
  return {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
__device__ __forceinline__ Oct load_oct(const __nv_bfloat16* p) {
  const uint4 w = __ldcs(reinterpret_cast<const uint4*>(p));
  return {{lo_f32(w.x), hi_f32(w.x), lo_f32(w.y), hi_f32(w.y), lo_f32(w.z), hi_f32(w.z), lo_f32(w.w), hi_f32(w.w)}};
}
__device__ __forceinline__ void store_oct(float* p, const Oct& o) {
  reinterpret_cast<float4*>(p)[0] = make_float4(o.v[0], o.v[1], o.v[2], o.v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(o.v[4], o.v[5], o.v[6], o.v[7]);
}
__device__ __forceinline__ void store_oct(__nv_bfloat16* p, const Oct& o) {
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(o.v[2 * i], o.v[2 * i + 1]);
    r[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(r[0], r[1], r[2], r[3]);
}

// The larger magnitude; a NaN is larger than all.
__device__ __forceinline__ float max_magnitude(float a, float b) {
  float m;
  asm("{ .reg .f32 x, y; abs.f32 x, %1; abs.f32 y, %2; max.NaN.f32 %0, x, y; }" : "=f"(m) : "f"(a), "f"(b));
  return m;
}

// The 4-bit form of a lane's 8 values of a block of 32 (four neighbouring lanes, all of which call this): the codes
// and the block's scale byte.
__device__ __forceinline__ uint32_t quantize_oct(const Oct& o, uint32_t* scale_byte) {
  const float m0 = max_magnitude(max_magnitude(o.v[0], o.v[1]), max_magnitude(o.v[2], o.v[3]));
  const float m1 = max_magnitude(max_magnitude(o.v[4], o.v[5]), max_magnitude(o.v[6], o.v[7]));
  float a = max_magnitude(m0, m1);
  a = max_magnitude(a, __shfl_xor_sync(0xFFFFFFFFu, a, 1));
  a = max_magnitude(a, __shfl_xor_sync(0xFFFFFFFFu, a, 2));
  const uint32_t b = mx_scale_byte(__float_as_uint(a) & 0x7FFFFFFFu);
  *scale_byte = b;
  if (b == 255u) return 0u;
  const float inv = mx_inverse_scale(b);
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = o.v[i] * inv;
  return mx_pack8(v);
}
// silu(g) u: g / (1 + exp(-g)) u.  The reciprocal is within a unit of the last place, 0 of infinity.
__device__ __forceinline__ float swiglu(float g, float u) {
  float r;
  asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(1.f + __expf(-g)));
  return g * r * u;
}

// Writes a lane's codes, and for the block's first lane its scale byte (and the row's pad bytes behind the last).
__device__ __forceinline__ void store_codes(uint32_t w, uint32_t b, int64_t row, int oct, int octs, uint32_t* xq,
                                            uint8_t* xs, int pitch) {
  *xq = w;
  if ((oct & 3) == 0) {
    uint8_t* s = xs + row * pitch + (oct >> 2);
    *s = (uint8_t)b;
    if (oct == octs - 4)
      for (int i = 1; i < pitch - (oct >> 2); ++i) s[i] = 0;
  }
}

// ---- the flat kernels: a thread takes half a block, 16 values -------------------------------------------------

// 32 bytes from or to memory, at once where they lie on a 32-byte boundary (`wide`).
__device__ __forceinline__ void load32(const void* p, bool wide, uint32_t* r) {
  if (wide) {
    asm volatile("ld.global.cs.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "l"(p)
                 : "memory");
  } else {
    const uint4 a = __ldcs(static_cast<const uint4*>(p)), b = __ldcs(static_cast<const uint4*>(p) + 1);
    r[0] = a.x, r[1] = a.y, r[2] = a.z, r[3] = a.w, r[4] = b.x, r[5] = b.y, r[6] = b.z, r[7] = b.w;
  }
}
__device__ __forceinline__ void store32(void* p, bool wide, const uint32_t* r) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]),
                 "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
  } else {
    static_cast<uint4*>(p)[0] = make_uint4(r[0], r[1], r[2], r[3]);
    static_cast<uint4*>(p)[1] = make_uint4(r[4], r[5], r[6], r[7]);
  }
}

// Half a block as it is in memory: 8 words of bf16 pairs, or 16 of float32.
template <typename T>
struct Half {
  static constexpr int kWords = 4 * sizeof(T);
  uint32_t r[kWords];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) r[i] = 0u;
  }
  __device__ __forceinline__ void load(const T* p, bool wide) {
#pragma unroll
    for (int i = 0; i < kWords; i += 8) load32(reinterpret_cast<const uint32_t*>(p) + i, wide, r + i);
  }
  __device__ __forceinline__ float value(int i) const {
    return sizeof(T) == 4 ? __uint_as_float(r[i]) : i & 1 ? hi_f32(r[i / 2]) : lo_f32(r[i / 2]);
  }
};

// The 4-bit form of half a block (two neighbouring lanes, both of which call this): the codes and the block's scale byte.
__device__ __forceinline__ uint2 quantize_half(const Half<float>& h, uint32_t* scale_byte) {
  float m[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) m[i] = max_magnitude(h.value(i), h.value(i + 8));
#pragma unroll
  for (int k = 4; k; k >>= 1)
#pragma unroll
    for (int i = 0; i < k; ++i) m[i] = max_magnitude(m[i], m[i + k]);
  const float a = max_magnitude(m[0], __shfl_xor_sync(0xFFFFFFFFu, m[0], 1));
  const uint32_t b = mx_scale_byte(__float_as_uint(a) & 0x7FFFFFFFu);
  *scale_byte = b;
  if (b == 255u) return make_uint2(0u, 0u);
  const float inv = mx_inverse_scale(b);
  float lo[8], hi[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo[i] = h.value(i) * inv;
    hi[i] = h.value(i + 8) * inv;
  }
  return make_uint2(mx_pack8(lo), mx_pack8(hi));
}
// bf16 magnitudes are compared as 16-bit integers, two at a time (a NaN is the largest), and scaled two at a time: exact in
// bf16 too (what underflows has the code 0 either way).
__device__ __forceinline__ uint2 quantize_half(const Half<__nv_bfloat16>& h, uint32_t* scale_byte) {
  constexpr uint32_t kMag = 0x7FFF7FFFu;
  uint32_t m[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) m[i] = __vmaxu2(h.r[i] & kMag, h.r[i + 4] & kMag);
  uint32_t a = __vmaxu2(__vmaxu2(m[0], m[1]), __vmaxu2(m[2], m[3]));
  a = __vmaxu2(a, __shfl_xor_sync(0xFFFFFFFFu, a, 1));
  const uint32_t b = mx_scale_byte(max(a & 0xFFFF0000u, a << 16));
  *scale_byte = b;
  if (b == 255u) return make_uint2(0u, 0u);
  const __nv_bfloat162 inv = bf16_pair((254u - b) << 7);
  float v[2][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const __nv_bfloat162 p = __hmul2_rn(*reinterpret_cast<const __nv_bfloat162*>(&h.r[i]), inv);
    const uint32_t q = *reinterpret_cast<const uint32_t*>(&p);
    v[i / 4][2 * (i & 3)] = lo_f32(q);
    v[i / 4][2 * (i & 3) + 1] = hi_f32(q);
  }
  return make_uint2(mx_pack8(v[0]), mx_pack8(v[1]));
}

// A thread's halves in a grid-stride loop: row and place in it counted on, not divided.
struct Walk {
  int row, half;
  __device__ __forceinline__ Walk(int64_t first, int halves)
      : row((int)(first / halves)), half((int)(first - (int64_t)row * halves)) {}
  __device__ __forceinline__ void next(int step_rows, int step_halves, int halves) {
    row += step_rows;
    half += step_halves;
    if (half >= halves) {
      half -= halves;
      ++row;
    }
  }
};

// What a row's values are made of: x itself, x's row rows[row], or silu(g) u of x [n][2 d] = [g | u].
enum { kPlain = 0, kRows = 1, kGated = 2 };

template <typename T, int FROM>
__global__ void __launch_bounds__(kThreads) mx_quantize_kernel(const T* __restrict__ x, int64_t n,
                                                               const int32_t* __restrict__ rows, int64_t m, int halves,
                                                               int step_rows, int step_halves, int wide,
                                                               uint8_t* __restrict__ xq, uint8_t* __restrict__ xs,
                                                               int pitch, uint32_t* __restrict__ status) {
  const int64_t total = m * halves, stride = (int64_t)gridDim.x * kThreads;
  int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int lane = threadIdx.x & 31;
  Walk w(i, halves);
  pdl_wait_then_release();
  bool bad = false;
  // a whole warp goes on together (the shuffles): the bound is its first half
  for (; i - lane < total; i += stride, w.next(step_rows, step_halves, halves)) {
    const bool in = i < total;
    uint32_t b;
    uint2 c;
    if constexpr (FROM == kGated) {
      Half<float> o;
      o.zero();
      if (in) {
        const T* p = x + ((int64_t)w.row * halves + i) * 16;       // 2 halves a row
        Half<T> g, u;
        g.load(p, wide);
        u.load(p + (int64_t)halves * 16, wide);
#pragma unroll
        for (int k = 0; k < 16; ++k) o.r[k] = __float_as_uint(swiglu(g.value(k), u.value(k)));
      }
      c = quantize_half(o, &b);
    } else {
      int64_t src = i;
      bool have = in;
      if constexpr (FROM == kRows) {
        const int64_t row = in ? rows[w.row] : -1;
        have = row >= 0 && row < n;
        src = row * halves + w.half;
      }
      Half<T> v;
      v.zero();
      if (have) v.load(x + src * 16, wide);
      c = quantize_half(v, &b);
    }
    if (in) {
      reinterpret_cast<uint2*>(xq)[i] = c;
      if ((w.half & 1) == 0) {                     // the block's scale, and the row's pad bytes behind the last
        uint8_t* s = xs + (int64_t)w.row * pitch + (w.half >> 1);
        *s = (uint8_t)b;
        if (w.half == halves - 2)
          for (int k = 1; k < pitch - (w.half >> 1); ++k) s[k] = 0;
      }
      bad |= b == 255u;
    }
  }
  if (__any_sync(0xFFFFFFFFu, bad) && lane == 0) report(status, kStatusNonFinite);
}

// Two E2M1 codes (nibbles 0 and 1 of c) as bf16 values 2^126 too small, the first in the low half: the code's magnitude
// bits are a bf16's last exponent bits and first mantissa bit (a subnormal for 0.5).
__device__ __forceinline__ uint32_t code_pair(uint32_t c) {
  return ((c & 7u) << 6) | ((c & 0x70u) << 18) | ((c & 8u) << 12) | ((c & 0x80u) << 24);
}
// times 2^126, then the scale: each exact, in bf16 too (one factor for both could be out of range)
__device__ __forceinline__ void dequantize_half(const uint2& c, uint32_t b, Half<float>& out) {
  const float s = mx_scale(b);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const uint32_t p = code_pair((k < 4 ? c.x : c.y) >> (8 * (k & 3)));
    out.r[2 * k] = __float_as_uint(lo_f32(p) * 0x1p126f * s);
    out.r[2 * k + 1] = __float_as_uint(hi_f32(p) * 0x1p126f * s);
  }
}
__device__ __forceinline__ void dequantize_half(const uint2& c, uint32_t b, Half<__nv_bfloat16>& out) {
  const __nv_bfloat162 up = bf16_pair((126u + 127u) << 7), s = bf16_pair(b == 255u ? 0x7FFFu : b == 0u ? 0x0040u : b << 7);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const uint32_t p = code_pair((k < 4 ? c.x : c.y) >> (8 * (k & 3)));
    const __nv_bfloat162 v = __hmul2_rn(__hmul2_rn(*reinterpret_cast<const __nv_bfloat162*>(&p), up), s);
    out.r[k] = *reinterpret_cast<const uint32_t*>(&v);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) mx_dequantize_kernel(const uint8_t* __restrict__ xq,
                                                                 const uint8_t* __restrict__ xs, int64_t n, int halves,
                                                                 int step_rows, int step_halves, int wide, int pitch,
                                                                 T* __restrict__ out) {
  const int64_t total = n * halves, stride = (int64_t)gridDim.x * kThreads;
  int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  Walk w(i, halves);
  pdl_wait_then_release();
  for (; i < total; i += stride, w.next(step_rows, step_halves, halves)) {
    const uint2 c = __ldcs(reinterpret_cast<const uint2*>(xq) + i);
    const uint32_t b = xs[(int64_t)w.row * pitch + (w.half >> 1)];
    Half<T> v;
    dequantize_half(c, b, v);
#pragma unroll
    for (int k = 0; k < Half<T>::kWords; k += 8) store32(reinterpret_cast<uint32_t*>(out + i * 16) + k, wide, v.r + k);
  }
}

// ---- h = x + residual in 32 bits, stored in x's type; v = h / sqrt(mean(h^2) + eps) * weight, of the unrounded h; then
// the 4-bit form of v.  Rows of up to 512 values have a warp each, up to 16384 a CTA each, whose threads hold them in
// registers (an octet each to 8192, two beyond); with persistent CTAs that load the next row while this one's sum is
// formed, 8192 x 8192 bf16 takes 82 us (5.3 TB/s), without 93, and 106 with four octets a thread.  Copying rows ahead into
// shared memory was no faster for 8192 rows of 8192 (83) and slower for all smaller (2048 x 4096 19 us, 13 here).
// h may be x or residual: a row's values are read by the CTA (warp) that writes them, before it writes.

__device__ __forceinline__ Oct load_weights(const float* p) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  return {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
__device__ __forceinline__ Oct load_weights(const __nv_bfloat16* p) {
  const uint4 w = __ldg(reinterpret_cast<const uint4*>(p));
  return {{lo_f32(w.x), hi_f32(w.x), lo_f32(w.y), hi_f32(w.y), lo_f32(w.z), hi_f32(w.z), lo_f32(w.w), hi_f32(w.w)}};
}

__device__ __forceinline__ void add(Oct& a, const Oct& b) {
#pragma unroll
  for (int k = 0; k < 8; ++k) a.v[k] += b.v[k];
}
__device__ __forceinline__ float squares(const Oct& a, float sum) {
#pragma unroll
  for (int k = 0; k < 8; ++k) sum = fmaf(a.v[k], a.v[k], sum);
  return sum;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}

struct NormOut {
  void* h;
  uint8_t *xq, *xs;
  int octs, pitch;
};

// The second half for one octet of a row (whole warps; lanes past the row's end hold nothing): h and the 4-bit form.
template <typename T, typename W>
__device__ __forceinline__ bool finish_oct(const NormOut& out, const W* weight, int64_t row, int oct, const Oct& a, float r) {
  const bool in = oct < out.octs;
  Oct v = {{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
  const int64_t at = row * out.octs + oct;
  if (in) {
    if (out.h) store_oct(static_cast<T*>(out.h) + at * 8, a);
    const Oct w = load_weights(weight + (int64_t)oct * 8);
#pragma unroll
    for (int k = 0; k < 8; ++k) v.v[k] = a.v[k] * w.v[k] * r;   // (bf16 times bf16 is mostly exact: one rounding, of the last product)
  }
  uint32_t b;
  const uint32_t c = quantize_oct(v, &b);
  if (in) store_codes(c, b, row, oct, out.octs, reinterpret_cast<uint32_t*>(out.xq) + at, out.xs, out.pitch);
  return in && b == 255u;
}

// A warp a row of up to 32 ITEMS octets.
template <typename T, typename W, int ITEMS>
__global__ void __launch_bounds__(kThreads) mx_rmsnorm_warp_kernel(const T* x, const T* residual,
                                                                   const W* __restrict__ weight, int64_t n, float eps,
                                                                   const NormOut out, uint32_t* __restrict__ status) {
  pdl_wait_then_release();
  const int lane = threadIdx.x & 31, octs = out.octs;
  const int64_t stride = (int64_t)gridDim.x * (kThreads / 32);
  bool bad = false;
  for (int64_t row = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); row < n; row += stride) {
    Oct a[ITEMS];
    float sq = 0.f;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      const int oct = 32 * j + lane;
      if (oct < octs) {
        a[j] = load_oct(x + (row * octs + oct) * 8);
        if (residual) add(a[j], load_oct(residual + (row * octs + oct) * 8));
        sq = squares(a[j], sq);
      }
    }
    const float r = __frsqrt_rn(warp_sum(sq) / (float)(octs * 8) + eps);
#pragma unroll
    for (int j = 0; j < ITEMS; ++j)
      if (32 * j < octs) bad |= finish_oct<T>(out, weight, row, 32 * j + lane, a[j], r);
  }
  if (__any_sync(0xFFFFFFFFu, bad) && lane == 0) report(status, kStatusNonFinite);
}

// An octet as it is in memory.
template <typename T>
struct Raw;
template <>
struct Raw<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = __ldcs(reinterpret_cast<const float4*>(p));
    b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
  }
  __device__ __forceinline__ Oct oct() const { return {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}}; }
};
template <>
struct Raw<__nv_bfloat16> {
  uint4 w;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { w = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ Oct oct() const {
    return {{lo_f32(w.x), hi_f32(w.x), lo_f32(w.y), hi_f32(w.y), lo_f32(w.z), hi_f32(w.z), lo_f32(w.w), hi_f32(w.w)}};
  }
};

// A CTA a row, ITEMS octets a thread in registers; the next row's are on their way while this one's sum is formed.
template <typename T, typename W, int ITEMS>
__global__ void __launch_bounds__(1024) mx_rmsnorm_row_kernel(const T* x, const T* residual, const W* __restrict__ weight,
                                                              int64_t n, float eps, const NormOut out,
                                                              uint32_t* __restrict__ status) {
  __shared__ float part[2][32];
  pdl_wait_then_release();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, octs = out.octs;
  Raw<T> nx[ITEMS], nr[ITEMS];
  auto load = [&](int64_t row) {
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      const int oct = j * blockDim.x + threadIdx.x;
      if (row < n && oct < octs) {
        nx[j].load(x + (row * octs + oct) * 8);
        if (residual) nr[j].load(residual + (row * octs + oct) * 8);
      }
    }
  };
  bool bad = false;
  int turn = 0;
  load(blockIdx.x);
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x, turn ^= 1) {
    Oct a[ITEMS];
    float sq = 0.f;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      if (j * (int)blockDim.x + (int)threadIdx.x < octs) {
        a[j] = nx[j].oct();
        if (residual) add(a[j], nr[j].oct());
        sq = squares(a[j], sq);
      }
    }
    load(row + gridDim.x);
    sq = warp_sum(sq);
    if (lane == 0) part[turn][warp] = sq;
    __syncthreads();                                     // (part[] has two turns, so one barrier a row will do)
    const float r = __frsqrt_rn(warp_sum(lane < warps ? part[turn][lane] : 0.f) / (float)(octs * 8) + eps);
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      const int oct = j * blockDim.x + threadIdx.x;
      if (oct - lane < octs) bad |= finish_oct<T>(out, weight, row, oct, a[j], r);
    }
  }
  if (__any_sync(0xFFFFFFFFu, bad) && lane == 0) report(status, kStatusNonFinite);
}

// Longer rows are read twice (before h is written).
template <typename T, typename W>
__global__ void __launch_bounds__(1024) mx_rmsnorm_long_kernel(const T* x, const T* residual, const W* __restrict__ weight,
                                                               int64_t n, float eps, const NormOut out,
                                                               uint32_t* __restrict__ status) {
  __shared__ float part[32];
  pdl_wait_then_release();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, octs = out.octs;
  bool bad = false;
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
    const int64_t base = row * octs;
    auto sum_of = [&](int oct) {
      Oct a = load_oct(x + (base + oct) * 8);
      if (residual) add(a, load_oct(residual + (base + oct) * 8));
      return a;
    };
    float sq = 0.f;
    for (int oct = threadIdx.x; oct < octs; oct += blockDim.x) sq = squares(sum_of(oct), sq);
    sq = warp_sum(sq);
    if (lane == 0) part[warp] = sq;
    __syncthreads();
    const float r = __frsqrt_rn(warp_sum(lane < warps ? part[lane] : 0.f) / (float)(octs * 8) + eps);
    for (int oct = threadIdx.x; oct - lane < octs; oct += blockDim.x)
      bad |= finish_oct<T>(out, weight, row, oct, oct < octs ? sum_of(oct) : Oct{}, r);
    __syncthreads();                                     // part[] is read before the next row's sums
  }
  if (__any_sync(0xFFFFFFFFu, bad) && lane == 0) report(status, kStatusNonFinite);
}

int sm_count() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 148;
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms <= 0) return 148;
  return sms;
}

template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), int64_t blocks, int threads, cudaStream_t stream, A... args) {
  note_launch();
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks, 1, 1);
  cfg.blockDim = dim3((unsigned)threads, 1, 1);
  cfg.stream = stream;
  cudaLaunchAttribute attr = pdl_attr();
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

// Blocks of a grid-stride loop over `rows` rows of halves, and its stride in rows and halves.
struct Flat {
  int halves, step_rows, step_halves;
  int64_t blocks;
  Flat(int64_t rows, int64_t d) : halves((int)(d / 16)) {
    const int64_t want = (rows * halves + kThreads - 1) / kThreads, cap = (int64_t)sm_count() * kFlatBlocks;
    blocks = want < cap ? want : cap;
    step_rows = (int)(blocks * kThreads / halves);
    step_halves = (int)(blocks * kThreads % halves);
  }
};
int aligned32(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 31u) == 0; }

template <typename T, int FROM>
cudaError_t quantize(const void* x, int64_t n, int64_t d, const int32_t* rows, int64_t m, uint8_t* xq, uint8_t* xs,
                     uint32_t* status, cudaStream_t stream) {
  const Flat f(m, d);
  return launch(mx_quantize_kernel<T, FROM>, f.blocks, kThreads, stream, static_cast<const T*>(x), n, rows, m, f.halves,
                f.step_rows, f.step_halves, aligned32(x), xq, xs, (int)mx_pitch(d), status);
}

template <typename T, typename W>
cudaError_t rmsnorm(const void* x_, const void* residual_, const void* weight_, int64_t n, int64_t d, float eps, void* h,
                    uint8_t* xq, uint8_t* xs, uint32_t* status, cudaStream_t stream) {
  const int octs = (int)(d / 8);
  const NormOut out = {h, xq, xs, octs, (int)mx_pitch(d)};
  const T *x = static_cast<const T*>(x_), *residual = static_cast<const T*>(residual_);
  const W* weight = static_cast<const W*>(weight_);
  const int64_t sms = sm_count();
  if (octs <= kWarpOcts) {
    const int64_t want = (n + kThreads / 32 - 1) / (kThreads / 32), blocks = want < sms * 16 ? want : sms * 16;
    auto go = [&](auto kernel) { return launch(kernel, blocks, kThreads, stream, x, residual, weight, n, eps, out, status); };
    return octs <= 32 ? go(mx_rmsnorm_warp_kernel<T, W, 1>) : go(mx_rmsnorm_warp_kernel<T, W, 2>);
  }
  const int threads = octs < 1024 ? (octs + 31) / 32 * 32 : 1024;
  const int64_t most = sms * (2048 / threads), blocks = n < most ? n : most;
  auto go = [&](auto kernel) { return launch(kernel, blocks, threads, stream, x, residual, weight, n, eps, out, status); };
  if (octs <= 1024) return go(mx_rmsnorm_row_kernel<T, W, 1>);
  if (octs <= 2048) return go(mx_rmsnorm_row_kernel<T, W, 2>);
  return go(mx_rmsnorm_long_kernel<T, W>);
}

}  // namespace

template <typename T>
static cudaError_t quantize_from(const void* x, int64_t n, int64_t d, const int32_t* rows, int64_t m, int gated, uint8_t* xq,
                                 uint8_t* xs, uint32_t* status, cudaStream_t stream) {
  if (gated) return quantize<T, kGated>(x, n, d, rows, m, xq, xs, status, stream);
  return rows ? quantize<T, kRows>(x, n, d, rows, m, xq, xs, status, stream)
              : quantize<T, kPlain>(x, n, d, rows, m, xq, xs, status, stream);
}

cudaError_t launch_mx_quantize(const void* x, int dtype, int64_t n, int64_t d, const int32_t* rows, int64_t m, int gated,
                               uint8_t* xq, uint8_t* xs, uint32_t* status, cudaStream_t stream) {
  return dtype == 0 ? quantize_from<float>(x, n, d, rows, m, gated, xq, xs, status, stream)
                    : quantize_from<__nv_bfloat16>(x, n, d, rows, m, gated, xq, xs, status, stream);
}

cudaError_t launch_mx_dequantize(const uint8_t* xq, const uint8_t* xs, int64_t n, int64_t d, int dtype, void* out,
                                 cudaStream_t stream) {
  const int pitch = (int)mx_pitch(d);
  const Flat f(n, d);
  if (dtype == 0)
    return launch(mx_dequantize_kernel<float>, f.blocks, kThreads, stream, xq, xs, n, f.halves, f.step_rows, f.step_halves,
                  aligned32(out), pitch, static_cast<float*>(out));
  return launch(mx_dequantize_kernel<__nv_bfloat16>, f.blocks, kThreads, stream, xq, xs, n, f.halves, f.step_rows,
                f.step_halves, aligned32(out), pitch, static_cast<__nv_bfloat16*>(out));
}

cudaError_t launch_mx_rmsnorm_quantize(const void* x, const void* residual, const void* weight, int dtype,
                                       int weight_dtype, int64_t n, int64_t d, float eps, void* h, uint8_t* xq, uint8_t* xs,
                                       uint32_t* status, cudaStream_t stream) {
  using B = __nv_bfloat16;
  if (dtype == 0)
    return weight_dtype == 0 ? rmsnorm<float, float>(x, residual, weight, n, d, eps, h, xq, xs, status, stream)
                             : rmsnorm<float, B>(x, residual, weight, n, d, eps, h, xq, xs, status, stream);
  return weight_dtype == 0 ? rmsnorm<B, float>(x, residual, weight, n, d, eps, h, xq, xs, status, stream)
                           : rmsnorm<B, B>(x, residual, weight, n, d, eps, h, xq, xs, status, stream);
}

}  // namespace cat
