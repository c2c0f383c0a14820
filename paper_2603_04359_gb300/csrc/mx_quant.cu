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
constexpr int kRowThreads = 512;  // most threads of a norm's CTA
constexpr int kFlatBlocks = 32;  // most blocks an SM of a grid-stride loop

__device__ __forceinline__ float lo_f32(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f32(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

__device__ __forceinline__ __nv_bfloat162 bf16_pair(uint32_t bits) {
  const uint32_t two = bits | (bits << 16);
  return *reinterpret_cast<const __nv_bfloat162*>(&two);
}

// The larger magnitude; a NaN is larger than all.
__device__ __forceinline__ float max_magnitude(float a, float b) {
  float m;
  asm("{ .reg .f32 x, y; abs.f32 x, %1; abs.f32 y, %2; max.NaN.f32 %0, x, y; }" : "=f"(m) : "f"(a), "f"(b));
  return m;
}

// silu(g) u: g / (1 + exp(-g)) u, by 2^x and the reciprocal, each within two units of the last place (and the rounding of
// g log2 e, |g| 2^-24), without the steps that subnormal numbers take: 2^x below 2^-126 adds nothing to 1, and the reciprocal
// of (1 + exp(-g)) / 16 is 2^-124 or more, or 0 of infinity (4096 x 14336 bf16: 40 us, 46 with those steps).  The sixteenth goes
// back into the reciprocal, not into g: of that it would take a subnormal gate's last bits, which a large u brings back.  (Below
// g = -87.3 the factor is subnormal itself and rounded by up to 2^-22 of it.)
__device__ __forceinline__ float swiglu(float g, float u) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(g * -1.44269504f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(fmaf(e, 0.0625f, 0.0625f)));
  return g * (0.0625f * r) * u;
}

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

// Writes half `half` of row `row`: its codes, and for the block's first lane the scale byte (behind the row's last, its pad
// bytes).
__device__ __forceinline__ void store_half(const uint2& c, uint32_t b, int row, int half, int halves, uint8_t* xq, uint8_t* xs,
                                           int pitch) {
  reinterpret_cast<uint2*>(xq)[(int64_t)row * halves + half] = c;
  if ((half & 1) == 0) {
    uint8_t* s = xs + (int64_t)row * pitch + (half >> 1);
    *s = (uint8_t)b;
    if (half == halves - 2)
      for (int k = 1; k < pitch - (half >> 1); ++k) s[k] = 0;
  }
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
      store_half(c, b, w.row, w.half, halves, xq, xs, pitch);
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

// ---- h = x + residual in 32 bits, stored in x's type; v = h weight / sqrt(mean(h^2) + eps), of the unrounded h; then
// the 4-bit form of v.  Rows of up to 512 values have a warp each, up to 16384 a CTA each, whose threads hold them in
// registers (half a block each to 8192, two beyond) and load the next row's while this one's sum is formed.  Moves 436 MB
// in 66 us at 8192 x 8192 bf16 (6.6 TB/s); with 8 values a thread 79, without the loads ahead 93, through shared memory
// (bulk copies of the next rows) 83.  The grid is what 64 registers a thread let be resident, 1024 threads an SM: a grid of more
// CTAs than that took up to 14 % longer.  Only bf16 rows to 8192 keep to 64; of float32 rows and longer ones (94 to 128) half
// of the CTAs run in a second wave (float32 8192 x 8192 136 us for 124 of bytes, bf16 1000 x 14336 21.7 for 13.8).
// h may be x or residual: a row's values are read by the CTA (warp) that writes them, before it writes.

struct NormArgs {
  const void *x, *residual, *weight;
  void* h;
  uint8_t *xq, *xs;
  int64_t n;
  int halves, pitch, wide;                  // wide: x, residual and h lie on 32-byte boundaries
  float eps;
  uint32_t* status;
};

// x and residual of half a block, as they are in memory.
template <typename T>
struct Pair {
  Half<T> x, r;
  __device__ __forceinline__ void load(const NormArgs& a, int64_t at) {
    x.load(static_cast<const T*>(a.x) + at * 16, a.wide);
    if (a.residual) r.load(static_cast<const T*>(a.residual) + at * 16, a.wide);
  }
  // the sum, and its squares added to `sq`
  __device__ __forceinline__ float sum(const NormArgs& a, float (&h)[16], float sq) const {
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      h[k] = x.value(k);
      if (a.residual) h[k] += r.value(k);
      sq = fmaf(h[k], h[k], sq);
    }
    return sq;
  }
};

__device__ __forceinline__ void load_weights(const float* p, float (&w)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 v = __ldg(reinterpret_cast<const float4*>(p) + i);
    w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
  }
}
__device__ __forceinline__ void load_weights(const __nv_bfloat16* p, float (&w)[16]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint4 v = __ldg(reinterpret_cast<const uint4*>(p) + i);
    const uint32_t r[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      w[8 * i + 2 * k] = lo_f32(r[k]);
      w[8 * i + 2 * k + 1] = hi_f32(r[k]);
    }
  }
}
__device__ __forceinline__ void round_half(const float (&h)[16], Half<float>& out) {
#pragma unroll
  for (int k = 0; k < 16; ++k) out.r[k] = __float_as_uint(h[k]);
}
__device__ __forceinline__ void round_half(const float (&h)[16], Half<__nv_bfloat16>& out) {
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(h[2 * k], h[2 * k + 1]);
    out.r[k] = *reinterpret_cast<const uint32_t*>(&v);
  }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}
__device__ __forceinline__ float mean_square(const NormArgs& a, float sum) { return sum / (float)(a.halves * 16) + a.eps; }
__device__ __forceinline__ float row_factor(float mean) { return __frsqrt_rn(mean); }

// Rows whose squares leave float32's range, though the norm does not (|h| from about 1e19 on, or below 1e-19 with an eps of
// nothing): their sum is infinite, or has lost what was below 2^-126.  Such a row is summed again times a power of two that
// brings it back: a mean of 2^110 or more (d is at most 2^18) to at most 2^106 and at least 2^-40, one below 2^-80 to at
// most 2^100.  The factor of the scaled row times the power is the row's own.  (eps of 2^-80 or more keeps a mean from being small.)
__device__ __forceinline__ bool out_of_range(float mean) { return mean < 0x1p-80f || mean == __int_as_float(0x7F800000); }
__device__ __forceinline__ float back_in_range(float mean) { return mean < 1.f ? 0x1p90f : 0x1p-75f; }
__device__ __forceinline__ float scaled_factor(const NormArgs& a, float sum, float by) {
  return __frsqrt_rn(sum / (float)(a.halves * 16) + a.eps * by * by) * by;
}
__device__ __forceinline__ float scaled_squares(const float (&h)[16], float by, float sq) {
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const float v = h[k] * by;
    sq = fmaf(v, v, sq);
  }
  return sq;
}

// The second half of a row's work for half a block (whole warps; lanes past the row's end hold nothing): h and the 4-bit
// form.  Whether the block is not finite.
template <typename T, typename W>
__device__ __forceinline__ bool finish_half(const NormArgs& a, int64_t row, int half, const float (&h)[16], float r) {
  const bool in = half < a.halves;
  Half<float> v;
  v.zero();
  if (in) {
    if (a.h) {
      Half<T> out;
      round_half(h, out);
      uint32_t* p = reinterpret_cast<uint32_t*>(static_cast<T*>(a.h) + (row * a.halves + half) * 16);
#pragma unroll
      for (int k = 0; k < Half<T>::kWords; k += 8) store32(p + k, a.wide, out.r + k);
    }
    float w[16];
    load_weights(static_cast<const W*>(a.weight) + (int64_t)half * 16, w);
    // (h times the factor is at most sqrt(d); h times the weight could leave float32's range on the way to a value within it)
#pragma unroll
    for (int k = 0; k < 16; ++k) v.r[k] = __float_as_uint(h[k] * r * w[k]);
  }
  uint32_t b;
  const uint2 c = quantize_half(v, &b);
  if (in) store_half(c, b, (int)row, half, a.halves, a.xq, a.xs, a.pitch);
  return in && b == 255u;
}

// A warp a row of up to 32 halves.
template <typename T, typename W>
__global__ void __launch_bounds__(kThreads) mx_rmsnorm_warp_kernel(const __grid_constant__ NormArgs a) {
  pdl_wait_then_release();
  const int lane = threadIdx.x & 31;
  const int64_t stride = (int64_t)gridDim.x * (kThreads / 32);
  bool bad = false;
  for (int64_t row = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); row < a.n; row += stride) {
    float h[16], sq = 0.f;
    if (lane < a.halves) {
      Pair<T> p;
      p.load(a, row * a.halves + lane);
      sq = p.sum(a, h, 0.f);
    }
    const float mean = mean_square(a, warp_sum(sq));
    float r = row_factor(mean);
    if (out_of_range(mean)) {                            // (the same in all lanes)
      const float by = back_in_range(mean);
      r = scaled_factor(a, warp_sum(lane < a.halves ? scaled_squares(h, by, 0.f) : 0.f), by);
    }
    bad |= finish_half<T, W>(a, row, lane, h, r);
  }
  if (__any_sync(0xFFFFFFFFu, bad) && lane == 0) report(a.status, kStatusNonFinite);
}

// A CTA a row, ITEMS halves a thread in registers; the next row's are on their way while this one's sum is formed.
template <typename T, typename W, int ITEMS>
__global__ void __launch_bounds__(kRowThreads, sizeof(T) * ITEMS == 2 ? 2 : 1)
    mx_rmsnorm_row_kernel(const __grid_constant__ NormArgs a) {
  __shared__ float part[2][32];
  pdl_wait_then_release();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  Pair<T> next[ITEMS];
  auto load = [&](int64_t row) {
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      const int half = j * blockDim.x + threadIdx.x;
      if (row < a.n && half < a.halves) next[j].load(a, row * a.halves + half);
    }
  };
  bool bad = false;
  int turn = 0;
  load(blockIdx.x);
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x, turn ^= 1) {
    float h[ITEMS][16], sq = 0.f;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j)
      if (j * (int)blockDim.x + (int)threadIdx.x < a.halves) sq = next[j].sum(a, h[j], sq);
    load(row + gridDim.x);
    sq = warp_sum(sq);
    if (lane == 0) part[turn][warp] = sq;
    __syncthreads();                                     // (part[] has two turns, so one barrier a row will do)
    const float mean = mean_square(a, warp_sum(lane < warps ? part[turn][lane] : 0.f));
    float r = row_factor(mean);
    if (out_of_range(mean)) {                            // (the same in all threads)
      const float by = back_in_range(mean);
      sq = 0.f;
#pragma unroll
      for (int j = 0; j < ITEMS; ++j)
        if (j * (int)blockDim.x + (int)threadIdx.x < a.halves) sq = scaled_squares(h[j], by, sq);
      sq = warp_sum(sq);
      __syncthreads();                                   // the first sums have been read
      if (lane == 0) part[turn][warp] = sq;
      __syncthreads();
      r = scaled_factor(a, warp_sum(lane < warps ? part[turn][lane] : 0.f), by);
    }
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      const int half = j * blockDim.x + threadIdx.x;
      if (half - lane < a.halves) bad |= finish_half<T, W>(a, row, half, h[j], r);
    }
  }
  if (__any_sync(0xFFFFFFFFu, bad) && lane == 0) report(a.status, kStatusNonFinite);
}

// Longer rows are read twice (before h is written), rows that leave the range three times.
template <typename T, typename W>
__global__ void __launch_bounds__(kRowThreads) mx_rmsnorm_long_kernel(const __grid_constant__ NormArgs a) {
  __shared__ float part[32];
  pdl_wait_then_release();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  bool bad = false;
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    float h[16], sq = 0.f;
    Pair<T> p;
    for (int half = threadIdx.x; half < a.halves; half += blockDim.x) {
      p.load(a, row * a.halves + half);
      sq = p.sum(a, h, sq);
    }
    sq = warp_sum(sq);
    if (lane == 0) part[warp] = sq;
    __syncthreads();
    const float mean = mean_square(a, warp_sum(lane < warps ? part[lane] : 0.f));
    float r = row_factor(mean);
    if (out_of_range(mean)) {                            // (the same in all threads)
      const float by = back_in_range(mean);
      sq = 0.f;
      for (int half = threadIdx.x; half < a.halves; half += blockDim.x) {
        p.load(a, row * a.halves + half);
        p.sum(a, h, 0.f);
        sq = scaled_squares(h, by, sq);
      }
      sq = warp_sum(sq);
      __syncthreads();                                   // the first sums have been read
      if (lane == 0) part[warp] = sq;
      __syncthreads();
      r = scaled_factor(a, warp_sum(lane < warps ? part[lane] : 0.f), by);
    }
    for (int half = threadIdx.x; half - lane < a.halves; half += blockDim.x) {
      if (half < a.halves) {
        p.load(a, row * a.halves + half);
        p.sum(a, h, 0.f);
      }
      bad |= finish_half<T, W>(a, row, half, h, r);
    }
    __syncthreads();                                     // part[] is read before the next row's sums
  }
  if (__any_sync(0xFFFFFFFFu, bad) && lane == 0) report(a.status, kStatusNonFinite);
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
cudaError_t rmsnorm(const NormArgs& a, cudaStream_t stream) {
  const int64_t sms = sm_count();
  if (a.halves <= 32) {
    const int64_t want = (a.n + kThreads / 32 - 1) / (kThreads / 32), blocks = want < sms * 16 ? want : sms * 16;
    return launch(mx_rmsnorm_warp_kernel<T, W>, blocks, kThreads, stream, a);
  }
  const int threads = a.halves < kRowThreads ? (a.halves + 31) / 32 * 32 : kRowThreads;
  const int64_t most = sms * (1024 / threads), blocks = a.n < most ? a.n : most;
  if (a.halves <= kRowThreads) return launch(mx_rmsnorm_row_kernel<T, W, 1>, blocks, threads, stream, a);
  if (a.halves <= 2 * kRowThreads) return launch(mx_rmsnorm_row_kernel<T, W, 2>, blocks, threads, stream, a);
  return launch(mx_rmsnorm_long_kernel<T, W>, blocks, threads, stream, a);
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
  const NormArgs a = {x, residual, weight, h, xq, xs, n, (int)(d / 16), (int)mx_pitch(d),
                      aligned32(x) & aligned32(residual) & aligned32(h), eps, status};
  if (dtype == 0) return weight_dtype == 0 ? rmsnorm<float, float>(a, stream) : rmsnorm<float, B>(a, stream);
  return weight_dtype == 0 ? rmsnorm<B, float>(a, stream) : rmsnorm<B, B>(a, stream);
}

}  // namespace cat
