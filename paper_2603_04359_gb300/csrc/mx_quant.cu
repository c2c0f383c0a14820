// Row kernels of the microscaled 4-bit format: quantization of activations and weights (with a gather of rows for
// experts' tokens), of SwiGLU's product, and of a root-mean-square norm with the residual's addition; dequantization.
//
// All are bound by the bytes that they move: every input is read once and the 4-bit form (17/32 of a byte a value) is
// all that is written beside the norm's sum, so the norm's or SwiGLU's 16-bit output never goes through memory.
//
// A thread takes 8 consecutive values (16 bytes of bf16), four lanes a block of 32: the block's largest magnitude takes
// two shuffles, a warp's codes are 128 consecutive bytes and its scales 8.  Magnitudes are compared as integers, their
// bits without the sign, so a NaN or an infinity is the largest of all and needs no test of its own.
#include "mx_format.cuh"

namespace cat {
namespace {

constexpr int kThreads = 256;

struct Oct {
  float v[8];
};

__device__ __forceinline__ Oct load_oct(const float* p) {
  const float4 a = __ldcs(reinterpret_cast<const float4*>(p)), b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
  return {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
__device__ __forceinline__ Oct load_oct(const __nv_bfloat16* p) {
  const uint4 w = __ldcs(reinterpret_cast<const uint4*>(p));
  Oct o;
  const uint32_t r[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o.v[2 * i] = __uint_as_float(r[i] << 16);
    o.v[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
  }
  return o;
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

// The 4-bit form of a lane's 8 values of a block of 32 (four neighbouring lanes, all of which call this): the codes
// and the block's scale byte.
__device__ __forceinline__ uint32_t quantize_oct(const Oct& o, uint32_t* scale_byte) {
  uint32_t a = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) a = max(a, __float_as_uint(o.v[i]) & 0x7FFFFFFFu);
  a = max(a, __shfl_xor_sync(0xFFFFFFFFu, a, 1));
  a = max(a, __shfl_xor_sync(0xFFFFFFFFu, a, 2));
  const uint32_t b = mx_scale_byte(a);
  *scale_byte = b;
  if (b == 255u) return 0u;
  const float inv = mx_inverse_scale(b);
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = o.v[i] * inv;
  return mx_pack8(v);
}

// Writes a lane's codes, and for the block's first lane its scale byte (and the row's pad bytes behind the last).
__device__ __forceinline__ void store_codes(uint32_t w, uint32_t b, int64_t row, int oct, int octs, uint8_t* xq,
                                            uint8_t* xs, int pitch) {
  reinterpret_cast<uint32_t*>(xq)[row * octs + oct] = w;
  if ((oct & 3) == 0) {
    uint8_t* s = xs + row * pitch + (oct >> 2);
    *s = (uint8_t)b;
    if (oct == octs - 4)
      for (int i = 1; i < pitch - (oct >> 2); ++i) s[i] = 0;
  }
}

// x [n][d] (or its rows `rows`) -> 4-bit form; GATED: x is [n][2 d] = [g | u] and the values are silu(g) u.
template <typename T, bool GATED>
__global__ void __launch_bounds__(kThreads) mx_quantize_kernel(const T* __restrict__ x, int64_t n,
                                                               const int32_t* __restrict__ rows, int64_t m, int octs,
                                                               uint8_t* __restrict__ xq, uint8_t* __restrict__ xs,
                                                               int pitch, uint32_t* __restrict__ status) {
  pdl_wait_then_release();
  const int64_t total = m * octs, stride = (int64_t)gridDim.x * kThreads;
  // a whole warp goes on together (the shuffles): the bound is the warp's first octet
  for (int64_t i0 = (int64_t)blockIdx.x * kThreads + (threadIdx.x & ~31); i0 < total; i0 += stride) {
    const int64_t i = i0 + (threadIdx.x & 31);
    const bool in = i < total;
    const int64_t row = in ? i / octs : 0;
    const int oct = in ? (int)(i - row * octs) : 0;
    const int64_t src = rows && in ? rows[row] : row;
    Oct o = {{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
    if (in && src >= 0 && src < n) {
      if (GATED) {
        const T* p = x + (src * 2 * octs + oct) * 8;
        const Oct g = load_oct(p), u = load_oct(p + (int64_t)octs * 8);
#pragma unroll
        for (int k = 0; k < 8; ++k) o.v[k] = g.v[k] / (1.f + __expf(-g.v[k])) * u.v[k];
      } else {
        o = load_oct(x + (src * octs + oct) * 8);
      }
    }
    uint32_t b;
    const uint32_t w = quantize_oct(o, &b);
    if (in) store_codes(w, b, row, oct, octs, xq, xs, pitch);
    if (in && b == 255u) report(status, kStatusNonFinite);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) mx_dequantize_kernel(const uint8_t* __restrict__ xq,
                                                                 const uint8_t* __restrict__ xs, int64_t n, int octs,
                                                                 int pitch, T* __restrict__ out) {
  pdl_wait_then_release();
  const int64_t total = n * octs, stride = (int64_t)gridDim.x * kThreads;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += stride) {
    const int64_t row = i / octs;
    const int oct = (int)(i - row * octs);
    const uint32_t w = reinterpret_cast<const uint32_t*>(xq)[i];
    const float s = mx_scale(xs[row * pitch + (oct >> 2)]);
    Oct o;
#pragma unroll
    for (int k = 0; k < 8; ++k) o.v[k] = mx_code_value((w >> (4 * k)) & 15u) * s;
    store_oct(out + i * 8, o);
  }
}

// One row a CTA.  h = x + residual in 32 bits, stored in x's type; v = h / sqrt(mean(h^2) + eps) * weight, of the
// unrounded h; then the 4-bit form of v.  A thread keeps ITEMS octets of h in registers, so the row is read once; with
// ITEMS = 0 (rows too long for that) it is read again for the second pass, before h is written, so h may be x or residual.
template <typename T, typename W, int ITEMS>
__global__ void __launch_bounds__(1024) mx_rmsnorm_quantize_kernel(const T* x, const T* residual,
                                                                   const W* __restrict__ weight, int64_t n, int octs,
                                                                   float eps, T* h, uint8_t* __restrict__ xq,
                                                                   uint8_t* __restrict__ xs, int pitch,
                                                                   uint32_t* __restrict__ status) {
  __shared__ float part[32];
  pdl_wait_then_release();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
    const int64_t base = row * octs;
    auto sum_of = [&](int oct) {
      Oct a = load_oct(x + (base + oct) * 8);
      if (residual) {
        const Oct r = load_oct(residual + (base + oct) * 8);
#pragma unroll
        for (int k = 0; k < 8; ++k) a.v[k] += r.v[k];
      }
      return a;
    };
    constexpr int kKept = ITEMS ? ITEMS : 1;
    const int steps = ITEMS ? ITEMS : (octs + (int)blockDim.x - 1) / (int)blockDim.x;
    Oct kept[kKept];
    float sq = 0.f;
    if (ITEMS) {
#pragma unroll
      for (int j = 0; j < kKept; ++j) {
        const int oct = j * blockDim.x + threadIdx.x;
        if (oct < octs) {
          kept[j] = sum_of(oct);
#pragma unroll
          for (int k = 0; k < 8; ++k) sq = fmaf(kept[j].v[k], kept[j].v[k], sq);
        }
      }
    } else {
      for (int oct = threadIdx.x; oct < octs; oct += blockDim.x) {
        const Oct a = sum_of(oct);
#pragma unroll
        for (int k = 0; k < 8; ++k) sq = fmaf(a.v[k], a.v[k], sq);
      }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) sq += __shfl_xor_sync(0xFFFFFFFFu, sq, d);
    if (lane == 0) part[warp] = sq;
    __syncthreads();
    float all = lane < warps ? part[lane] : 0.f;
#pragma unroll
    for (int d = 16; d; d >>= 1) all += __shfl_xor_sync(0xFFFFFFFFu, all, d);
    const float r = 1.f / sqrtf(all / (float)(octs * 8) + eps);
#pragma unroll
    for (int j = 0; j < (ITEMS ? kKept : steps); ++j) {
      const int oct = j * blockDim.x + threadIdx.x;
      if (oct - lane >= octs) break;                     // whole warps (the shuffles)
      Oct v = {{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
      if (oct < octs) {
        const Oct a = ITEMS ? kept[ITEMS ? j : 0] : sum_of(oct);
        if (h) store_oct(h + (base + oct) * 8, a);
        const Oct w = load_oct(weight + (int64_t)oct * 8);
#pragma unroll
        for (int k = 0; k < 8; ++k) v.v[k] = a.v[k] * r * w.v[k];
      }
      uint32_t b;
      const uint32_t c = quantize_oct(v, &b);
      if (oct < octs) {
        store_codes(c, b, row, oct, octs, xq, xs, pitch);
        if (b == 255u) report(status, kStatusNonFinite);
      }
    }
    __syncthreads();                                     // part[] is read before the next row's sums
  }
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

int64_t flat_blocks(int64_t octets) {
  const int64_t blocks = (octets + kThreads - 1) / kThreads, cap = (int64_t)sm_count() * 32;
  return blocks < cap ? blocks : cap;
}

template <typename T, bool GATED>
cudaError_t quantize(const void* x, int64_t n, int64_t d, const int32_t* rows, int64_t m, uint8_t* xq, uint8_t* xs,
                     uint32_t* status, cudaStream_t stream) {
  const int octs = (int)(d / 8);
  return launch(mx_quantize_kernel<T, GATED>, flat_blocks(m * octs), kThreads, stream, static_cast<const T*>(x), n, rows, m,
                octs, xq, xs, (int)mx_pitch(d), status);
}

template <typename T, typename W>
cudaError_t rmsnorm(const void* x, const void* residual, const void* weight, int64_t n, int64_t d, float eps, void* h,
                    uint8_t* xq, uint8_t* xs, uint32_t* status, cudaStream_t stream) {
  const int octs = (int)(d / 8);
  int threads = 32;
  while (threads < 1024 && threads * (threads < 256 ? 1 : 4) < octs) threads *= 2;
  const int items = (octs + threads - 1) / threads;
  auto go = [&](auto kernel) {
    const int64_t cap = (int64_t)sm_count() * 64;
    return launch(kernel, n < cap ? n : cap, threads, stream, static_cast<const T*>(x), static_cast<const T*>(residual),
                  static_cast<const W*>(weight), n, octs, eps, static_cast<T*>(h), xq, xs, (int)mx_pitch(d), status);
  };
  if (items == 1) return go(mx_rmsnorm_quantize_kernel<T, W, 1>);
  if (items == 2) return go(mx_rmsnorm_quantize_kernel<T, W, 2>);
  if (items <= 4) return go(mx_rmsnorm_quantize_kernel<T, W, 4>);
  return go(mx_rmsnorm_quantize_kernel<T, W, 0>);
}

}  // namespace

cudaError_t launch_mx_quantize(const void* x, int dtype, int64_t n, int64_t d, const int32_t* rows, int64_t m, int gated,
                               uint8_t* xq, uint8_t* xs, uint32_t* status, cudaStream_t stream) {
  if (dtype == 0)
    return gated ? quantize<float, true>(x, n, d, rows, m, xq, xs, status, stream)
                 : quantize<float, false>(x, n, d, rows, m, xq, xs, status, stream);
  return gated ? quantize<__nv_bfloat16, true>(x, n, d, rows, m, xq, xs, status, stream)
               : quantize<__nv_bfloat16, false>(x, n, d, rows, m, xq, xs, status, stream);
}

cudaError_t launch_mx_dequantize(const uint8_t* xq, const uint8_t* xs, int64_t n, int64_t d, int dtype, void* out,
                                 cudaStream_t stream) {
  const int octs = (int)(d / 8), pitch = (int)mx_pitch(d);
  if (dtype == 0)
    return launch(mx_dequantize_kernel<float>, flat_blocks(n * octs), kThreads, stream, xq, xs, n, octs, pitch,
                  static_cast<float*>(out));
  return launch(mx_dequantize_kernel<__nv_bfloat16>, flat_blocks(n * octs), kThreads, stream, xq, xs, n, octs, pitch,
                static_cast<__nv_bfloat16*>(out));
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
