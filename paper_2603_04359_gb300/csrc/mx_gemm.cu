// Products of microscaled 4-bit operands (mx_format.cuh), plain and grouped by expert:
//
//   y[t, o] = sum over blocks b of 32 channels of 2^(bx + bw - 254) sum_{i in b} c_x[t, i] c_w[o, i]
//
// A simple kernel: 64 tokens by 64 channels a CTA, operands widened to float32 in shared memory, four by four outputs
// a thread, sums in 32 bits.
#include "mx_format.cuh"

namespace cat {
namespace {

constexpr int kTile = 64, kStep = 32;

template <typename T>
__device__ __forceinline__ T to_out(float v);
template <>
__device__ __forceinline__ float to_out<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 to_out<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// A group's first row and the one past its last: offsets in order within [0, m], whatever the caller's are.
__device__ __forceinline__ int edge(const int32_t* offsets, int e, int m, int before) {
  return min(max(offsets[e], before), m);
}

template <typename T>
__global__ void __launch_bounds__(256) mx_gemm_kernel(const uint8_t* __restrict__ xq, const uint8_t* __restrict__ xs,
                                                      const uint8_t* __restrict__ wq, const uint8_t* __restrict__ ws,
                                                      const int32_t* __restrict__ offsets, int experts, int m, int d,
                                                      int d_out, T* __restrict__ y) {
  pdl_wait_then_release();
  // token tile blockIdx.y of the groups' tiles, in order
  int expert = 0, row0 = 0, row1 = m, tile = blockIdx.y;
  if (offsets) {
    int lo = edge(offsets, 0, m, 0), hi = lo;
    for (expert = 0; expert < experts; ++expert, lo = hi) {
      hi = edge(offsets, expert + 1, m, lo);
      const int tiles = (hi - lo + kTile - 1) / kTile;
      if (tile < tiles) break;
      tile -= tiles;
    }
    if (expert == experts) return;
    row0 = lo;
    row1 = hi;
  }
  row0 += tile * kTile;
  if (row0 >= row1) return;
  const int o0 = blockIdx.x * kTile, pitch = (int)mx_pitch(d);
  wq += (size_t)expert * d_out * (d / 2);
  ws += (size_t)expert * d_out * pitch;
  __shared__ float sx[kStep][kTile + 1], sw[kStep][kTile + 1];
  const int tid = threadIdx.x, tr = tid / 16, tc = tid % 16;
  float acc[4][4] = {};
  for (int k = 0; k < d; k += kStep) {
    // 64 rows x 4 octets an operand, one a thread
    const int r = tid / 4, oct = tid % 4;
    uint32_t wx = 0, ww = 0;
    float fx = 0.f, fw = 0.f;
    if (row0 + r < row1) {
      wx = *reinterpret_cast<const uint32_t*>(xq + (size_t)(row0 + r) * (d / 2) + k / 2 + 4 * oct);
      fx = mx_scale(xs[(size_t)(row0 + r) * pitch + k / 32]);
    }
    if (o0 + r < d_out) {
      ww = *reinterpret_cast<const uint32_t*>(wq + (size_t)(o0 + r) * (d / 2) + k / 2 + 4 * oct);
      fw = mx_scale(ws[(size_t)(o0 + r) * pitch + k / 32]);
    }
    for (int i = 0; i < 8; ++i) {
      sx[8 * oct + i][r] = mx_code_value((wx >> (4 * i)) & 15u) * fx;
      sw[8 * oct + i][r] = mx_code_value((ww >> (4 * i)) & 15u) * fw;
    }
    __syncthreads();
#pragma unroll 8
    for (int i = 0; i < kStep; ++i) {
      float a[4], b[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        a[j] = sx[i][tr * 4 + j];
        b[j] = sw[i][tc + 16 * j];
      }
#pragma unroll
      for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[p][q] = fmaf(a[p], b[q], acc[p][q]);
    }
    __syncthreads();
  }
  for (int p = 0; p < 4; ++p)
    for (int q = 0; q < 4; ++q) {
      const int t = row0 + tr * 4 + p, o = o0 + tc + 16 * q;
      if (t < row1 && o < d_out) y[(size_t)t * d_out + o] = to_out<T>(acc[p][q]);
    }
}

}  // namespace

// offsets == nullptr: one group of all m rows.  Rows that belong to no group are zero.
cudaError_t launch_mx_gemm(const uint8_t* xq, const uint8_t* xs, const uint8_t* wq, const uint8_t* ws,
                           const int32_t* offsets, int64_t experts, int64_t m, int64_t d, int64_t d_out, int out_dtype,
                           void* y, uint32_t*, cudaStream_t stream) {
  if (offsets) {
    const cudaError_t e = cudaMemsetAsync(y, 0, (size_t)m * d_out * (out_dtype == 0 ? 4 : 2), stream);
    if (e != cudaSuccess) return e;
  }
  const int64_t tiles = (m + kTile - 1) / kTile + (offsets ? (experts < m ? experts : m) : 0);
  const dim3 grid((unsigned)((d_out + kTile - 1) / kTile), (unsigned)tiles, 1);
  note_launch();
  if (out_dtype == 0)
    mx_gemm_kernel<float><<<grid, 256, 0, stream>>>(xq, xs, wq, ws, offsets, (int)experts, (int)m, (int)d, (int)d_out,
                                                    static_cast<float*>(y));
  else
    mx_gemm_kernel<__nv_bfloat16><<<grid, 256, 0, stream>>>(xq, xs, wq, ws, offsets, (int)experts, (int)m, (int)d,
                                                            (int)d_out, static_cast<__nv_bfloat16*>(y));
  return cudaGetLastError();
}

}  // namespace cat
