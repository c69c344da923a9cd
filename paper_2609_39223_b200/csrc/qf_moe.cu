// Mixture-of-experts routing around the grouped linear layer: the routing table (a stable counting sort of the
// (token, expert) pairs), tokens into expert order, and the weighted sum back, with both gradients.
#include "qf_common.cuh"

namespace qf {
namespace {

// ---- routing table ----------------------------------------------------------------------------------------------

constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;

template <typename Id>
__device__ __forceinline__ int expert_of(const Id* __restrict__ ids, int64_t p, int G) {
  const Id e = ids[p];
  return e >= 0 && e < static_cast<Id>(G) ? static_cast<int>(e) : -1;
}

// row_of[p] = offs[e] + #{q < p : id_q = e}. Every warp owns a contiguous run of pairs. First every warp counts its run;
// the counts, summed over the warps before it, give each warp its first row in every segment; then every warp walks its
// run again, 32 pairs at a time, and numbers equal ids inside a group of 32 by lane: the order of p is kept.
template <typename Id>
__global__ void __launch_bounds__(kSortThreads) moe_sort_kernel(const Id* __restrict__ ids, int64_t pairs, int G, int64_t rows,
                                                                int32_t* __restrict__ row_of, int32_t* __restrict__ offs,
                                                                int32_t* __restrict__ counts) {
  extern __shared__ uint32_t hist[];                 // [kSortWarps][G]
  __shared__ uint32_t warp_sum[kSortWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int i = tid; i < kSortWarps * G; i += kSortThreads) hist[i] = 0u;
  __syncthreads();
  const int64_t run = (pairs + kSortWarps * 32 - 1) / (kSortWarps * 32) * 32;
  const int64_t first = warp * run, last = min(first + run, pairs);
  uint32_t* mine = hist + warp * G;
  for (int64_t p = first + lane; p < last; p += 32) {
    const int e = expert_of(ids, p, G);
    if (e >= 0) atomicAdd(mine + e, 1u);
  }
  __syncthreads();
  uint32_t count = 0;                                // of expert tid
  if (tid < G) {
    for (int w = 0; w < kSortWarps; ++w) {
      const uint32_t c = hist[w * G + tid];
      hist[w * G + tid] = count;
      count += c;
    }
  }
  // exclusive scan of the padded counts
  const uint32_t padded = (count + 127u) & ~127u;
  uint32_t incl = padded;
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, incl, d);
    if (lane >= d) incl += v;
  }
  if (lane == 31) warp_sum[warp] = incl;
  __syncthreads();
  uint32_t start = incl - padded;
  for (int w = 0; w < warp; ++w) start += warp_sum[w];
  if (tid < G) {
    for (int w = 0; w < kSortWarps; ++w) hist[w * G + tid] += start;
    const uint32_t top = static_cast<uint32_t>(rows), from = min(start, top);
    offs[tid] = static_cast<int32_t>(from);
    counts[tid] = static_cast<int32_t>(min(count, top - from));
    if (tid == G - 1) offs[G] = static_cast<int32_t>(min(start + padded, top));
  }
  __syncthreads();
  for (int64_t p0 = first; p0 < last; p0 += 32) {
    const int64_t p = p0 + lane;
    const int e = p < last ? expert_of(ids, p, G) : -1;
    const uint32_t same = __match_any_sync(0xFFFFFFFFu, e);
    const uint32_t rank = __popc(same & ((1u << lane) - 1u));
    uint32_t base = 0;
    if (e >= 0) base = mine[e];
    __syncwarp();
    if (e >= 0 && rank == 0) mine[e] = base + __popc(same);
    __syncwarp();
    if (p < last) row_of[p] = e >= 0 && base + rank < static_cast<uint32_t>(rows) ? static_cast<int32_t>(base + rank) : -1;
  }
}

// ---- eight consecutive elements of a row ------------------------------------------------------------------------

struct Vec8 { float v[8]; };

template <typename T> struct Io8;
template <> struct Io8<__nv_bfloat16> {
  using Raw = uint4;
  static __device__ __forceinline__ Raw load(const void* base, int64_t chunk) { return __ldg(static_cast<const uint4*>(base) + chunk); }
  static __device__ __forceinline__ Vec8 widen(const Raw& r) {
    return {{bf16_lo(r.x), bf16_hi(r.x), bf16_lo(r.y), bf16_hi(r.y), bf16_lo(r.z), bf16_hi(r.z), bf16_lo(r.w), bf16_hi(r.w)}};
  }
  static __device__ __forceinline__ void store(void* base, int64_t chunk, const Vec8& a) {
    static_cast<uint4*>(base)[chunk] = make_uint4(pack_bf16x2(a.v[0], a.v[1]), pack_bf16x2(a.v[2], a.v[3]),
                                                  pack_bf16x2(a.v[4], a.v[5]), pack_bf16x2(a.v[6], a.v[7]));
  }
};
struct Float8 { float4 a, b; };
template <> struct Io8<float> {
  using Raw = Float8;
  static __device__ __forceinline__ Raw load(const void* base, int64_t chunk) {
    const float4* p = static_cast<const float4*>(base) + 2 * chunk;
    return {__ldg(p), __ldg(p + 1)};
  }
  static __device__ __forceinline__ Vec8 widen(const Raw& r) { return {{r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w}}; }
  static __device__ __forceinline__ void store(void* base, int64_t chunk, const Vec8& a) {
    float4* p = static_cast<float4*>(base) + 2 * chunk;
    p[0] = make_float4(a.v[0], a.v[1], a.v[2], a.v[3]);
    p[1] = make_float4(a.v[4], a.v[5], a.v[6], a.v[7]);
  }
};

constexpr int kThreads = 256;

inline unsigned blocks_for(int64_t n) { return static_cast<unsigned>((n + kThreads - 1) / kThreads); }

// Row of pair p in the sorted buffer; -1 for a dropped pair and for any entry outside the buffer.
__device__ __forceinline__ int row_of_pair(const MoeTable& t, int64_t p) {
  const int r = t.row_of ? __ldg(t.row_of + p) : static_cast<int>(p);
  return r >= 0 && r < t.rows ? r : -1;
}

// ---- tokens into expert order: one thread per 8 elements of a token, read once and written top_k times ---------------

__global__ void __launch_bounds__(kThreads) moe_dispatch_kernel(const MoeTable t, const uint4* __restrict__ x, uint4* __restrict__ xs) {
  const int64_t nv = t.hidden / 8, i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (i >= t.tokens * nv) return;
  const int64_t token = i / nv, chunk = i - token * nv;
  const uint4 v = __ldg(x + i);
  for (int j = 0; j < t.top_k; ++j) {
    const int r = row_of_pair(t, token * t.top_k + j);
    if (r >= 0) xs[r * nv + chunk] = v;
  }
}

// ---- weighted sum back: one thread per 8 elements of a token ---------------------------------------------------------

template <typename In, typename Out, bool WEIGHTED>
__global__ void __launch_bounds__(kThreads) moe_combine_kernel(const MoeTable t, const void* __restrict__ ys,
                                                               const float* __restrict__ weights, void* __restrict__ out) {
  const int64_t nv = t.hidden / 8, i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (i >= t.tokens * nv) return;
  const int64_t token = i / nv, chunk = i - token * nv;
  Vec8 acc = {};
  for (int j = 0; j < t.top_k; ++j) {
    const int64_t p = token * t.top_k + j;
    const int r = row_of_pair(t, p);
    if (r < 0) continue;
    const Vec8 y = Io8<In>::widen(Io8<In>::load(ys, r * nv + chunk));
    const float w = WEIGHTED ? __ldg(weights + p) : 1.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc.v[e] = WEIGHTED ? fmaf(w, y.v[e], acc.v[e]) : acc.v[e] + y.v[e];
  }
  Io8<Out>::store(out, i, acc);
}

// ---- gradient of the weighted sum: one block per token -----------------------------------------------------------------

template <typename DOut, typename In>
__global__ void __launch_bounds__(kThreads) moe_combine_bwd_kernel(const MoeTable t, const void* __restrict__ dout,
                                                                   const void* __restrict__ ys, const float* __restrict__ weights,
                                                                   void* __restrict__ dys, float* __restrict__ dweights) {
  __shared__ float part[kThreads / 32];
  const int64_t nv = t.hidden / 8, token = blockIdx.x;
  for (int j = 0; j < t.top_k; ++j) {
    const int64_t p = token * t.top_k + j;
    const int r = row_of_pair(t, p);
    float dot = 0.0f;
    if (r >= 0) {
      const float w = __ldg(weights + p);
      for (int64_t c = threadIdx.x; c < nv; c += kThreads) {
        const Vec8 d = Io8<DOut>::widen(Io8<DOut>::load(dout, token * nv + c));
        Vec8 g;
#pragma unroll
        for (int e = 0; e < 8; ++e) g.v[e] = w * d.v[e];
        Io8<__nv_bfloat16>::store(dys, r * nv + c, g);
        if (dweights) {
          const Vec8 y = Io8<In>::widen(Io8<In>::load(ys, r * nv + c));
#pragma unroll
          for (int e = 0; e < 8; ++e) dot = fmaf(d.v[e], y.v[e], dot);
        }
      }
    }
    if (dweights) {
      for (int d = 16; d > 0; d >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, d);
      __syncthreads();
      if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = dot;
      __syncthreads();
      if (threadIdx.x == 0) {
        float sum = 0.0f;
        for (int w = 0; w < kThreads / 32; ++w) sum += part[w];
        dweights[p] = sum;
      }
    }
  }
}

}  // namespace

cudaError_t launch_moe_sort(const void* ids, bool ids64, int64_t pairs, int G, int64_t rows, int32_t* row_of, int32_t* offs,
                            int32_t* counts, cudaStream_t st) {
  const size_t smem = static_cast<size_t>(kSortWarps) * G * 4;
  auto go = [&](auto kernel, auto* p) -> cudaError_t {
    if (smem > 48 * 1024)
    if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSortWarps * QF_MOE_MAX_EXPERTS * 4)) return e;
    kernel<<<1, kSortThreads, smem, st>>>(p, pairs, G, rows, row_of, offs, counts);
    return cudaGetLastError();
  };
  return ids64 ? go(moe_sort_kernel<int64_t>, static_cast<const int64_t*>(ids)) : go(moe_sort_kernel<int32_t>, static_cast<const int32_t*>(ids));
}

cudaError_t launch_moe_dispatch(const MoeTable& t, const void* x, void* xs, cudaStream_t st) {
  if (cudaError_t e = cudaMemsetAsync(xs, 0, static_cast<size_t>(t.rows) * t.hidden * 2, st)) return e;
  if (t.tokens == 0) return cudaSuccess;
  moe_dispatch_kernel<<<blocks_for(t.tokens * (t.hidden / 8)), kThreads, 0, st>>>(t, static_cast<const uint4*>(x), static_cast<uint4*>(xs));
  return cudaGetLastError();
}

cudaError_t launch_moe_combine(const MoeTable& t, const void* ys, int ys_dtype, const float* weights, void* out, int out_dtype,
                               cudaStream_t st) {
  auto go = [&](auto kernel) {
    kernel<<<blocks_for(t.tokens * (t.hidden / 8)), kThreads, 0, st>>>(t, ys, weights, out);
    return cudaGetLastError();
  };
  using B = __nv_bfloat16;
  if (weights) {
    if (ys_dtype == QF_DT_F32) return out_dtype == QF_DT_F32 ? go(moe_combine_kernel<float, float, true>) : go(moe_combine_kernel<float, B, true>);
    return out_dtype == QF_DT_F32 ? go(moe_combine_kernel<B, float, true>) : go(moe_combine_kernel<B, B, true>);
  }
  if (ys_dtype == QF_DT_F32) return out_dtype == QF_DT_F32 ? go(moe_combine_kernel<float, float, false>) : go(moe_combine_kernel<float, B, false>);
  return out_dtype == QF_DT_F32 ? go(moe_combine_kernel<B, float, false>) : go(moe_combine_kernel<B, B, false>);
}

cudaError_t launch_moe_combine_bwd(const MoeTable& t, const void* dout, int dout_dtype, const void* ys, int ys_dtype,
                                   const float* weights, void* dys, float* dweights, cudaStream_t st) {
  if (cudaError_t e = cudaMemsetAsync(dys, 0, static_cast<size_t>(t.rows) * t.hidden * 2, st)) return e;
  if (t.tokens == 0) return cudaSuccess;
  auto go = [&](auto kernel) {
    kernel<<<static_cast<unsigned>(t.tokens), kThreads, 0, st>>>(t, dout, ys, weights, dys, dweights);
    return cudaGetLastError();
  };
  using B = __nv_bfloat16;
  if (dout_dtype == QF_DT_F32) return ys_dtype == QF_DT_F32 ? go(moe_combine_bwd_kernel<float, float>) : go(moe_combine_bwd_kernel<float, B>);
  return ys_dtype == QF_DT_F32 ? go(moe_combine_bwd_kernel<B, float>) : go(moe_combine_bwd_kernel<B, B>);
}

}  // namespace qf
