// What the two kernels of attention over the 4-bit cache share: few query rows a sequence (mx_attention.cu) and tiles of them
// (mx_attention_tiles.cu).
#pragma once
#include "mx_cache.cuh"

namespace cat {

constexpr float kSlack = 6.f;               // a row's scores may exceed its running maximum by this (binary orders) before it follows

// A CTA's piece that begins a unit (sequence, row tile, head) which others go on with.
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
  int few;                                  // sequences of at most this many rows are the first kernel's, others the second's
  int clears;                               // this launch clears the rows that see nothing
  float scale;                              // scale log2 e
  int64_t window;
  void* out;
  int out_f32;
  float *parts, *ml;                        // [2 grid][rows][D], [2 grid][rows][2]: maximum and sum
  Plan* plan;
  uint32_t* status;
};

// Where the parts of a launch lie in its workspace.
struct Parts {
  size_t ml, plan, bytes;
  Parts(size_t grid, size_t rows, size_t d) {
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    ml = up(2 * grid * rows * d * 4);
    plan = ml + up(2 * grid * rows * 8);
    bytes = plan + up(grid * sizeof(Plan));
  }
  void place(AttnArgs* a, void* workspace) const {
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    a->parts = reinterpret_cast<float*>(ws);
    a->ml = reinterpret_cast<float*>(ws + ml);
    a->plan = reinterpret_cast<Plan*>(ws + plan);
  }
};

// Tiles of more rows: the grid, rows a tile, and the launch (with the joining of parts).
int attention_tile_rows(int64_t d);
cudaError_t launch_attention_tiles(const AttnArgs& a, int64_t d, int grid, cudaStream_t stream);

namespace {

// A sequence's rows of q and the tokens that they see.
struct Rows {
  int begin, ql;                            // first row, rows
  int64_t len, first, end;                  // tokens; the first that a row sees; one past the last in the cache
  __device__ __forceinline__ bool any() const { return ql > 0 && end > first; }
};
__device__ __forceinline__ Rows rows_of(const AttnArgs& a, int s) {
  Rows q;
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
  return q;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{ .reg .pred q; elect.sync _|q, 0xFFFFFFFF; selp.u32 %0, 1, 0, q; }" : "=r"(p));
  return p != 0;
}
// `bytes` (a multiple of 16) from memory to shared memory, counted on `bar`
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)), "l"(src),
               "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

// Four channels of a row of the output.
__device__ __forceinline__ void store4(const AttnArgs& a, int64_t at, const float4& o) {
  if (a.out_f32) {
    *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = o;
  } else {
    const __nv_bfloat162 lo = __floats2bfloat162_rn(o.x, o.y), hi = __floats2bfloat162_rn(o.z, o.w);
    *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + at) =
        make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
  }
}

// Zeros to rows whose sequence has no tokens that they could see, and to rows of no sequence.
template <int D>
__device__ __forceinline__ void clear_rows(const AttnArgs& a) {
  const int64_t row_words = (int64_t)a.hq * D / (a.out_f32 ? 4 : 8);
  uint4* out = static_cast<uint4*>(a.out);
  auto clear = [&](int64_t r0, int64_t r1, int64_t first, int64_t stride) {
    for (int64_t i = r0 * row_words + first; i < r1 * row_words; i += stride) out[i] = make_uint4(0u, 0u, 0u, 0u);
  };
  for (int s = blockIdx.x; s < a.seqs; s += gridDim.x) {
    const Rows q = rows_of(a, s);
    if (!q.any() && q.ql > 0) clear(q.begin, q.begin + q.ql, threadIdx.x, blockDim.x);
  }
  if (a.offsets) {
    const int64_t first = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, stride = (int64_t)gridDim.x * blockDim.x;
    const int head = min(max(a.offsets[0], 0), a.n), tail = min(max(a.offsets[a.seqs], 0), a.n);
    clear(0, head, first, stride);
    clear(max(tail, head), a.n, first, stride);
  }
}

constexpr int kJoinThreads = 128;

// The parts of a unit, some of its rows a CTA: blockIdx.x the CTA that began it.
template <int D, int ROWS>
__global__ void __launch_bounds__(kJoinThreads) mx_attention_join_kernel(const __grid_constant__ AttnArgs a) {
  constexpr int kLanes = D / 4, kGroups = kJoinThreads / kLanes;       // lanes a row of four channels; parts at once
  __shared__ float4 os[kJoinThreads];
  __shared__ float2 mls[kGroups];
  pdl_wait_then_release();
  const int cta = blockIdx.x;
  const Plan p = a.plan[cta];
  if (p.last < 0) return;
  const Rows sq = rows_of(a, p.s);
  const int rows = (int)min((int64_t)ROWS, (int64_t)sq.ql * a.group - (int64_t)p.rt * ROWS);
  const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  for (int r = blockIdx.y; r < rows; r += gridDim.y) {
    float top = -1e30f, sum = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](const float2& ml, const float4& v) {
      const float now = fmaxf(top, ml.x), was = ex2(top - now), by = ex2(ml.x - now);
      top = now;
      sum = sum * was + ml.y * by;
      o.x = o.x * was + v.x * by, o.y = o.y * was + v.y * by, o.z = o.z * was + v.z * by, o.w = o.w * was + v.w * by;
    };
    for (int k = cta + group; k <= p.last; k += kGroups) {
      const int64_t slot = ((int64_t)2 * k + (k == cta ? 1 : 0)) * ROWS + r;
      const float2 ml = *reinterpret_cast<const float2*>(a.ml + slot * 2);
      if (ml.y != 0.f) add(ml, *reinterpret_cast<const float4*>(a.parts + slot * D + 4 * lane));       // (a part of no tokens has no values)
    }
    __syncthreads();                                     // (the row before has been joined)
    os[threadIdx.x] = o;
    if (lane == 0) mls[group] = make_float2(top, sum);
    __syncthreads();
    if (group == 0) {
      for (int w = 1; w < kGroups; ++w) add(mls[w], os[w * kLanes + lane]);
      const int rr = p.rt * ROWS + r, j = rr / a.group;
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      o.x *= inv, o.y *= inv, o.z *= inv, o.w *= inv;
      store4(a, ((int64_t)(sq.begin + j) * a.hq + p.h * a.group + (rr - j * a.group)) * D + 4 * lane, o);
    }
  }
}

template <int D, int ROWS>
cudaError_t launch_join(const AttnArgs& a, int grid, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid, ROWS < 32 ? ROWS : 32);
  cfg.blockDim = dim3(kJoinThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr = pdl_attr();
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  note_launch();
  return cudaLaunchKernelEx(&cfg, mx_attention_join_kernel<D, ROWS>, a);
}

}  // namespace
}  // namespace cat
