// What the two kernels of attention over the 4-bit cache share: few query rows a sequence (mx_attention.cu) and tiles of them
// (mx_attention_tiles.cu).
#pragma once
#include "mx_cache.cuh"

namespace cat {

constexpr float kMost = 3.402823466e38f;    // the largest float32
constexpr float kNone = -kMost;             // the maximum of no scores: none is less, but one that float32 does not hold
constexpr float kSlack = 6.f;               // a row's scores may exceed its running maximum by this (binary orders) before it follows

// A unit (sequence, row tile, head) of which a CTA has a part and not the whole: it has two at most, that which it goes on with and
// that which it begins.
struct alignas(16) Plan {
  int first, last;                          // the CTAs with a part of it; last = -1: no such unit
  int begin, h, row0, rows;                 // its sequence's first row; its head, first row of the head's group, and rows
};
// The CTA that a place of the line is a piece of: `each` places a CTA, one more for the first `rest` of them.
__device__ __forceinline__ int cta_of(int64_t place, int64_t each, int64_t rest) {
  return (int)(place < rest * (each + 1) ? place / (each + 1) : rest + (place - rest * (each + 1)) / each);
}

struct AttnArgs {
  const __nv_bfloat16* q;
  MxCache c;
  int64_t pages;
  const int32_t *table, *lens, *offsets;
  int64_t width;
  int n, hq, group, seqs;
  int few;                                  // sequences of at most this many rows are the first kernel's, others the second's
  int clears;                               // this launch clears the rows that see nothing
  int beside;                               // this launch does not wait for the one before it until its end
  float scale;                              // scale log2 e
  int64_t window;
  void* out;
  int out_f32;
  float *parts, *ml;                        // [2 grid][rows][D], [2 grid][rows][2]: maximum and sum
  Plan* plan;                               // [grid][2]
  uint32_t* status;
};

// Where the parts of a launch lie in its workspace.
struct Parts {
  size_t ml, plan, bytes;
  Parts(size_t grid, size_t rows, size_t d) {
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    ml = up(2 * grid * rows * d * 4);
    plan = ml + up(2 * grid * rows * 8);
    bytes = plan + up(2 * grid * sizeof(Plan));
  }
  void place(AttnArgs* a, void* workspace) const {
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    a->parts = reinterpret_cast<float*>(ws);
    a->ml = reinterpret_cast<float*>(ws + ml);
    a->plan = reinterpret_cast<Plan*>(ws + plan);
  }
};

// Tiles of more rows: rows a tile, and the launch (and that of its joining of parts).
int attention_tile_rows(int64_t d);
cudaError_t launch_attention_tiles(const AttnArgs& a, int64_t d, int grid, bool join, cudaStream_t stream);

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

// Bound of the pipeline waits (ns; of each kernel's own): kWaitLimitNs unless a test shortens it (cat_set_wait_limit_ns).
__device__ uint64_t g_wait_limit = kWaitLimitNs;

// What a CTA's waits have in common, in shared memory.
struct Waits {
  int abort;                                // the line of the first wait that gave up
  int patience;                             // tries before a wait looks at the clock: 0 with a short limit, and once a wait has given up
  uint32_t limit;                           // (1 s at most, of a clock's low word)
  __device__ __forceinline__ void init() {
    limit = (uint32_t)g_wait_limit;
    patience = limit < kWaitLimitNs ? 0 : 64;
    abort = 0;
  }
};
__device__ __forceinline__ bool mbar_test_wait(uint64_t* bar, uint32_t parity) {
  uint32_t p;
  asm volatile("{ .reg .pred p; mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
               : "=r"(p)
               : "r"(smem_u32(bar)), "r"(parity)
               : "memory");
  return p != 0;
}
// A wait whose first try has failed.  The clock is looked at every `patience` tries only (of up to some microseconds; polls of some 50 ns: 64
// times as many).  Out of line: one copy of it for all waits stays in the instruction cache.
template <bool POLL>
__device__ __noinline__ bool long_wait(uint64_t* bar, uint32_t parity, volatile Waits* w, int site) {
  uint32_t since = 0;
#pragma unroll 1
  for (int n = 0;; ++n) {
    if (n >= (POLL ? w->patience << 6 : w->patience)) {
      if (w->abort) return false;
      n = 0;
      const uint32_t now = (uint32_t)globaltimer_ns();
      if (since == 0) since = now ? now : 1u;            // (0: not looked at yet)
      if ((int32_t)(now - since) + 1 >= (int32_t)w->limit) {
        w->abort = site;
        w->patience = 0;
        return false;
      }
    }
    if (POLL ? mbar_test_wait(bar, parity) : mbar_try_wait(bar, parity)) return true;
  }
}
// A bounded wait.  POLL: without letting the hardware suspend the thread, whose waking takes longer.  TEST: the first try alone (what
// is there at once needs no more, and with a short limit what is not gives up there).
template <bool POLL, bool TEST = POLL>
__device__ __forceinline__ bool short_wait(uint64_t* bar, uint32_t parity, volatile Waits* w, int site) {
  if (TEST ? mbar_test_wait(bar, parity) : mbar_try_wait(bar, parity)) return true;
  return long_wait<POLL>(bar, parity, w, site);
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

constexpr int kJoinWarps = 4, kJoinThreads = 32 * kJoinWarps;

// A row of a unit's output, or 4 kLanes kWide channels of it, from some of its parts: a lane has kWide times four channels.  Parts are means
// of values with the sums of their weights, and so is what is made of them: a sum of many large values could leave float32.
template <int D, int kLanes, int kWide>
struct JoinRow {
  static constexpr int lanes = kLanes, wide = kWide;
  float top, sum;
  float4 o[kWide];
  __device__ __forceinline__ void clear() {
    top = kNone, sum = 0.f;
#pragma unroll
    for (int i = 0; i < kWide; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  // Weights that add up to `more`, relative to 2^now, are to be added: what they are times is returned.
  __device__ __forceinline__ float follow(float now, float more) {
    const float had = sum * ex2(top - now);
    top = now, sum = had + more;
    const float inv = sum == 0.f ? 0.f : 1.f / sum, was = had * inv;
#pragma unroll
    for (int i = 0; i < kWide; ++i) o[i].x *= was, o[i].y *= was, o[i].z *= was, o[i].w *= was;
    return inv;
  }
  __device__ __forceinline__ void add(const float4 (&v)[kWide], float by) {
#pragma unroll
    for (int i = 0; i < kWide; ++i)
      o[i].x = fmaf(v[i].x, by, o[i].x), o[i].y = fmaf(v[i].y, by, o[i].y), o[i].z = fmaf(v[i].z, by, o[i].z), o[i].w = fmaf(v[i].w, by, o[i].w);
  }
  // A warp: row r of the parts of CTAs from, from + stride, ..., last; `first` is the one that began the unit.
  template <int ROWS>
  __device__ __forceinline__ void parts(const AttnArgs& a, int r, int first, int from, int last, int stride, int channel = 0) {
    const int lane = threadIdx.x & 31;
    for (int base = from; base <= last; base += 32 * stride) {
      const int k = base + lane * stride;
      auto slot_of = [&](int c) { return ((int64_t)2 * c + (c == first ? 1 : 0)) * ROWS + r; };
      float2 ml = make_float2(kNone, 0.f);
      if (k <= last) ml = *reinterpret_cast<const float2*>(a.ml + slot_of(k) * 2);
      const bool some = ml.y != 0.f;                     // (a part of no tokens has no values)
      float now = some ? fmaxf(top, ml.x) : top;
#pragma unroll
      for (int i = 1; i < 32; i <<= 1) now = fmaxf(now, __shfl_xor_sync(0xFFFFFFFFu, now, i));
      float mine = some ? ml.y * ex2(ml.x - now) : 0.f, more = mine;
#pragma unroll
      for (int i = 1; i < 32; i <<= 1) more += __shfl_xor_sync(0xFFFFFFFFu, more, i);
      mine *= follow(now, more);
      const uint32_t which = __ballot_sync(0xFFFFFFFFu, some);
      const int count = min(32, (last - base) / stride + 1);
#pragma unroll 8
      for (int i = 0; i < count; i += 32 / kLanes) {
        const int j = i + lane / kLanes;                 // (< 32: `count` is even there or followed by one that is not `some`)
        const float by = __shfl_sync(0xFFFFFFFFu, mine, j);
        if (which >> j & 1) {
          const float* at = a.parts + slot_of(base + j * stride) * D + channel + 4 * (lane % kLanes);
          float4 v[kWide];
#pragma unroll
          for (int w = 0; w < kWide; ++w) v[w] = *reinterpret_cast<const float4*>(at + 128 * w);
          add(v, by);
        }
      }
    }
#pragma unroll
    for (int i = kLanes; i < 32; i <<= 1)
#pragma unroll
      for (int w = 0; w < kWide; ++w) {
        o[w].x += __shfl_xor_sync(0xFFFFFFFFu, o[w].x, i), o[w].y += __shfl_xor_sync(0xFFFFFFFFu, o[w].y, i);
        o[w].z += __shfl_xor_sync(0xFFFFFFFFu, o[w].z, i), o[w].w += __shfl_xor_sync(0xFFFFFFFFu, o[w].w, i);
      }
  }
};

// The parts of units, in the order of their tokens.  The CTAs with a part of a unit share its rows out among them (tiles': eight times):
// one launch of as many CTAs as the SMs hold at once, however many parts a unit has.  A row of few parts is a warp's; of many the
// warps of a CTA take every fourth part each, of all its channels or, where there are CTAs enough, of 32, all loads independent.  (One unit and row a CTA, its parts one behind the other,
// and CTAs for all that could begin one: a step of 64 heads over 131000 tokens spent 10 us here, one of 27 short sequences 5.)
__host__ __device__ constexpr int join_split(int rows) { return rows < 128 ? 1 : 8; }
template <int D, int ROWS>
__device__ __forceinline__ void join(const AttnArgs& a, int index) {
  constexpr int kLanes = D == 64 ? 16 : 32, kWide = D == 256 ? 2 : 1;
  constexpr int split = join_split(ROWS);
  __shared__ float4 os[kJoinWarps][D / 4];
  __shared__ float2 mls[kJoinWarps];
  const int entry = index / split, cta = entry / 2, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Plan p = a.plan[entry];
  if (p.last < 0) return;
  const int stride = (p.last - p.first + 1) * split, r0 = (cta - p.first) * split + index % split;
  auto store = [&](int r, int at, float4 o) {
    const int rr = p.row0 + r, j = rr / a.group;
    store4(a, ((int64_t)(p.begin + j) * a.hq + p.h * a.group + (rr - j * a.group)) * D + at, o);
  };
  if (p.last - p.first < 2 * kJoinWarps) {
    JoinRow<D, kLanes, kWide> row;
    for (int r = r0 + warp * stride; r < p.rows; r += kJoinWarps * stride) {
      row.clear();
      row.template parts<ROWS>(a, r, p.first, p.first, p.last, 1);
#pragma unroll
      for (int w = 0; w < kWide; ++w)
        if (lane < kLanes) store(r, 4 * lane + 128 * w, row.o[w]);
    }
    return;
  }
  auto shared = [&](auto row, int width) {               // all of a row's channels, or 32 of them
    const int pieces = D / width;
    for (int i = r0; i < p.rows * pieces; i += stride) {
      const int r = i / pieces, channel = width * (i - r * pieces);
      row.clear();
      row.template parts<ROWS>(a, r, p.first, p.first + warp, p.last, kJoinWarps, channel);
      __syncthreads();                                   // (the channels before have been joined)
#pragma unroll
      for (int w = 0; w < row.wide; ++w)
        if (lane < row.lanes) os[warp][lane + 32 * w] = row.o[w];
      if (lane == 0) mls[warp] = make_float2(row.top, row.sum);
      __syncthreads();
      if (threadIdx.x < width / 4) {
        float top = mls[0].x, sum = 0.f, share[kJoinWarps];
#pragma unroll
        for (int w = 1; w < kJoinWarps; ++w) top = fmaxf(top, mls[w].x);
#pragma unroll
        for (int w = 0; w < kJoinWarps; ++w) {
          share[w] = mls[w].y * ex2(mls[w].x - top);
          sum += share[w];
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kJoinWarps; ++w) {
          const float by = share[w] * inv;
          const float4 v = os[w][threadIdx.x];
          o.x = fmaf(v.x, by, o.x), o.y = fmaf(v.y, by, o.y), o.z = fmaf(v.z, by, o.z), o.w = fmaf(v.w, by, o.w);
        }
        store(r, channel + 4 * threadIdx.x, o);
      }
    }
  };
  if (p.rows * (D / 32) <= stride)
    shared(JoinRow<D, 8, 1>(), 32);
  else
    shared(JoinRow<D, kLanes, kWide>(), D);
}

template <int D, int ROWS>
__global__ void __launch_bounds__(kJoinThreads) mx_attention_join_kernel(const __grid_constant__ AttnArgs a) {
  pdl_wait_then_release();
  join<D, ROWS>(a, blockIdx.x);
}
// Those of both kernels.
template <int D, int ROWS, int TILE_ROWS>
__global__ void __launch_bounds__(kJoinThreads) mx_attention_join_both_kernel(const __grid_constant__ AttnArgs few, int few_grid,
                                                                              const __grid_constant__ AttnArgs tiles) {
  pdl_wait_then_release();
  if ((int)blockIdx.x < few_grid)
    join<D, ROWS>(few, blockIdx.x);
  else
    join<D, TILE_ROWS>(tiles, blockIdx.x - few_grid);
}

inline cudaLaunchConfig_t join_config(int grid, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(kJoinThreads);
  cfg.stream = stream;
  return cfg;
}

}  // namespace
}  // namespace cat
