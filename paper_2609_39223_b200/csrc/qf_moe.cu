// Mixture-of-experts routing around the grouped linear layer: the routing table (a stable counting sort of the
// (token, expert) pairs), tokens into expert order, and the weighted sum back, with both gradients.
#include <cooperative_groups.h>

#include "qf_common.cuh"

namespace cg = cooperative_groups;

namespace qf {
namespace {

// ---- routing table ----------------------------------------------------------------------------------------------

constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortBatch = 8;                        // loads of ids in flight per lane

template <typename Id>
__device__ __forceinline__ int expert_of(const Id* __restrict__ ids, int64_t p, int64_t last, int G) {
  if (p >= last) return -1;
  const Id e = __ldg(ids + p);
  return e >= 0 && e < static_cast<Id>(G) ? static_cast<int>(e) : -1;
}

// row_of[p] = offs[e] + #{q < p : id_q = e}. Every warp of the cluster owns a contiguous run of pairs. First every warp counts its
// run; the counts, summed over the warps and CTAs before it, give each warp its first row in every segment; then every warp walks
// its run again, 32 pairs at a time, and numbers equal ids inside a group of 32 by lane: the order of p is kept. One launch,
// no global scratch: the CTAs of a cluster read one another's counts in shared memory.
// Bound by instructions and latency, not by the 8 bytes a pair: 131072 pairs to 128 experts 11.1 us, with 56% of the issue slots of its 16
// SMs busy (142 us with one CTA and a walk by single pairs); 56 pairs 4.0 us, the launch and six barriers.
template <typename Id>
__global__ void __launch_bounds__(kSortThreads) moe_sort_kernel(const Id* __restrict__ ids, int64_t pairs, int G, int64_t rows,
                                                                int32_t* __restrict__ row_of, int32_t* __restrict__ offs,
                                                                int32_t* __restrict__ counts) {
  extern __shared__ uint32_t hist[];                 // [kSortWarps][G], then the CTA's counts [G]
  __shared__ uint32_t warp_sum[kSortWarps];
  const cg::cluster_group cluster = cg::this_cluster();
  const int ctas = gridDim.x, rank_cta = blockIdx.x;
  uint32_t* total = hist + kSortWarps * G;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int i = tid; i < kSortWarps * G; i += kSortThreads) hist[i] = 0u;
  __syncthreads();
  const int64_t runs = static_cast<int64_t>(ctas) * kSortWarps, run = (pairs + runs * 32 - 1) / (runs * 32) * 32;
  const int64_t first = (static_cast<int64_t>(rank_cta) * kSortWarps + warp) * run, last = min(first + run, pairs);
  uint32_t* mine = hist + warp * G;
  const uint32_t bits = 32 - __clz(G);               // of id + 1
  for (int64_t p0 = first + lane; p0 < last; p0 += 32 * kSortBatch) {
    int e[kSortBatch];
#pragma unroll
    for (int i = 0; i < kSortBatch; ++i) e[i] = expert_of(ids, p0 + 32 * i, last, G);
#pragma unroll
    for (int i = 0; i < kSortBatch; ++i)
      if (e[i] >= 0) atomicAdd(mine + e[i], 1u);
  }
  __syncthreads();
  uint32_t count = 0;                                // of expert tid
  if (tid < G) {
#pragma unroll 8
    for (int w = 0; w < kSortWarps; ++w) {
      const uint32_t c = hist[w * G + tid];
      hist[w * G + tid] = count;
      count += c;
    }
    total[tid] = count;
  }
  uint32_t before = 0;                               // of the CTAs before this one
  if (ctas > 1) {
    cluster.sync();
    if (tid < G) {
      count = 0;
#pragma unroll 4
      for (int c = 0; c < ctas; ++c) {
        const uint32_t v = *cluster.map_shared_rank(total + tid, c);
        before += c < rank_cta ? v : 0u;
        count += v;
      }
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
#pragma unroll 8
    for (int w = 0; w < kSortWarps; ++w) hist[w * G + tid] += start + before;
    if (rank_cta == 0) {
      const uint32_t top = static_cast<uint32_t>(rows), from = min(start, top);
      offs[tid] = static_cast<int32_t>(from);
      counts[tid] = static_cast<int32_t>(min(count, top - from));
      if (tid == G - 1) offs[G] = static_cast<int32_t>(min(start + padded, top));
    }
  }
  if (ctas > 1) cluster.barrier_arrive();            // this CTA needs no other's counts any more
  __syncthreads();
  for (int64_t p0 = first; p0 < last; p0 += 32 * kSortBatch) {
    int e[kSortBatch];
#pragma unroll
    for (int i = 0; i < kSortBatch; ++i) e[i] = expert_of(ids, p0 + 32 * i + lane, last, G);
#pragma unroll
    for (int i = 0; i < kSortBatch; ++i) {
      const int64_t p = p0 + 32 * i + lane;
      if (p - lane >= last) break;
      // the lanes with the same id, bit by bit of id + 1 (0: none)
      uint32_t same = 0xFFFFFFFFu;
      for (uint32_t b = 0; b < bits; ++b) {
        const bool one = (static_cast<uint32_t>(e[i] + 1) >> b) & 1u;
        const uint32_t vote = __ballot_sync(0xFFFFFFFFu, one);
        same &= one ? vote : ~vote;
      }
      const uint32_t rank = __popc(same & ((1u << lane) - 1u));
      uint32_t base = 0;
      if (e[i] >= 0) base = mine[e[i]];
      __syncwarp();
      if (e[i] >= 0 && rank == 0) mine[e[i]] = base + __popc(same);
      __syncwarp();
      if (p < last) row_of[p] = e[i] >= 0 && base + rank < static_cast<uint32_t>(rows) ? static_cast<int32_t>(base + rank) : -1;
    }
  }
  if (ctas > 1) cluster.barrier_wait();              // and no other needs this one's
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

// ---- rows that no pair owns -------------------------------------------------------------------------------------------
// Zeros for the padding at the end of every segment and for the rows past the last one. kZeroParts CTAs take turns at the rows of
// a segment's padding (at most 127), kTailCtas at the rest. Only these rows are zeroed: setting the whole buffer first would write
// the other ones twice.

constexpr int kZeroParts = 4;
constexpr int kTailCtas = 296;
inline unsigned zero_blocks(const MoeTable& t) { return static_cast<unsigned>(t.G) * kZeroParts + kTailCtas; }

__device__ __forceinline__ void zero_rows(const MoeTable& t, unsigned block, uint4* __restrict__ buf) {
  const int64_t nv = t.hidden / 8;
  const unsigned segments = static_cast<unsigned>(t.G) * kZeroParts;
  int64_t r, end, step;
  if (block < segments) {
    const unsigned e = block / kZeroParts;
    const int64_t from = min(max(__ldg(t.offs + e), 0), static_cast<int>(t.rows));
    end = min(max(__ldg(t.offs + e + 1), 0), static_cast<int>(t.rows));
    r = from + max(__ldg(t.counts + e), 0) + block % kZeroParts;
    step = kZeroParts;
  } else {
    r = min(max(__ldg(t.offs + t.G), 0), static_cast<int>(t.rows)) + static_cast<int64_t>(block - segments);
    end = t.rows;
    step = kTailCtas;
  }
  for (; r < end; r += step)
    for (int64_t c = threadIdx.x; c < nv; c += blockDim.x) buf[r * nv + c] = make_uint4(0u, 0u, 0u, 0u);
}

// ---- tokens into expert order: one thread per 8 elements of a token, read once and written top_k times ---------------
// Bound by the writes. 16384 tokens of 2048, 8 experts each, into 147328 rows: 110 us, 6.1 TB/s (180 us when the
// whole buffer was set to zero first; 4096 tokens of 4096: 76 us, 79 when the row numbers were loaded one by one).

__global__ void __launch_bounds__(kThreads) moe_dispatch_kernel(const MoeTable t, unsigned token_blocks, const uint4* __restrict__ x, uint4* __restrict__ xs) {
  if (blockIdx.x >= token_blocks) {
    zero_rows(t, blockIdx.x - token_blocks, xs);
    return;
  }
  const int64_t nv = t.hidden / 8, i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (i >= t.tokens * nv) return;
  const int64_t token = i / nv, chunk = i - token * nv;
  const uint4 v = __ldg(x + i);
  constexpr int kTogether = 8;                       // row numbers loaded at a time
  for (int j0 = 0; j0 < t.top_k; j0 += kTogether) {
    int row[kTogether];
#pragma unroll
    for (int j = 0; j < kTogether; ++j) row[j] = j0 + j < t.top_k ? row_of_pair(t, token * t.top_k + j0 + j) : -1;
#pragma unroll
    for (int j = 0; j < kTogether; ++j)
      if (row[j] >= 0) xs[row[j] * nv + chunk] = v;
  }
}

// ---- weighted sum back: one thread per 8 elements of a token ---------------------------------------------------------
// out = sum over j of w_j * row_j, in FP32 and in the order of j. Bound by the reads. The numbers, weights and rows of four pairs are
// loaded together (a row's address waits for its number). 16384 tokens of 2048, 8 pairs each, BF16: 97 us, 6.2 TB/s (106 us pair by
// pair, 97 with eight together); without weights, as the gradient of dispatch, 91 us (105, 96); 33 tokens 2.9 us (3.6, 2.8).

constexpr int kTogether = 4;

template <typename In, typename Out, bool WEIGHTED>
__global__ void __launch_bounds__(kThreads) moe_combine_kernel(const MoeTable t, const void* __restrict__ ys,
                                                               const float* __restrict__ weights, void* __restrict__ out) {
  const int64_t nv = t.hidden / 8, i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (i >= t.tokens * nv) return;
  const int64_t token = i / nv, chunk = i - token * nv;
  Vec8 acc = {};
  for (int j0 = 0; j0 < t.top_k; j0 += kTogether) {
    const int64_t p = token * t.top_k + j0;
    int row[kTogether];
    float w[kTogether];
    typename Io8<In>::Raw y[kTogether] = {};
#pragma unroll
    for (int j = 0; j < kTogether; ++j) {
      row[j] = j0 + j < t.top_k ? row_of_pair(t, p + j) : -1;
      w[j] = WEIGHTED && j0 + j < t.top_k ? __ldg(weights + p + j) : 1.0f;
    }
#pragma unroll
    for (int j = 0; j < kTogether; ++j)
      if (row[j] >= 0) y[j] = Io8<In>::load(ys, row[j] * nv + chunk);
#pragma unroll
    for (int j = 0; j < kTogether; ++j) {
      if (row[j] < 0) continue;
      const Vec8 v = Io8<In>::widen(y[j]);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc.v[e] = WEIGHTED ? fmaf(w[j], v.v[e], acc.v[e]) : acc.v[e] + v.v[e];
    }
  }
  Io8<Out>::store(out, i, acc);
}

// ---- gradient of the weighted sum: one CTA per token --------------------------------------------------------------------
// dout is read once for kPairs pairs, whose rows of ys are loaded together; the pairs' inner products stay in registers and are
// reduced at the end: over the lanes by halving (lane bits 4..2 choose the pair, so that a step moves half of what the last one
// did), then over the warps in their order. Bound by the traffic of ys and dys: 16384 tokens of 2048, 8 pairs each, in BF16: 207 us,
// 5.84 TB/s. (Three CTAs an SM are asked for: 80 registers; 247 us with the 117 it would take, 226 us with 64.) That was found for BF16 ys; with
// FP32 ys, whose eight rows alone are 64 registers, 256 bytes a thread are spilled in the loop: 373 us (dout BF16) and 443 us (FP32) for
// 1746 and 1813 MB, 4.7 and 4.1 TB/s. Without dweights, BF16 dout: 153 us for 671 MB, 4.4 TB/s.

constexpr int kPairs = 8;

template <typename DOut, typename In>
__global__ void __launch_bounds__(kThreads, 3) moe_combine_bwd_kernel(const MoeTable t, unsigned token_blocks, const void* __restrict__ dout,
                                                                   const void* __restrict__ ys, const float* __restrict__ weights,
                                                                   void* __restrict__ dys, float* __restrict__ dweights) {
  if (blockIdx.x >= token_blocks) {
    zero_rows(t, blockIdx.x - token_blocks, static_cast<uint4*>(dys));
    return;
  }
  __shared__ float part[kThreads / 32][kPairs];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t nv = t.hidden / 8, token = blockIdx.x;
  for (int j0 = 0; j0 < t.top_k; j0 += kPairs) {
    const int64_t p0 = token * t.top_k + j0;
    int row[kPairs];
    float w[kPairs], dot[kPairs];
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
      row[j] = j0 + j < t.top_k ? row_of_pair(t, p0 + j) : -1;
      w[j] = row[j] >= 0 ? __ldg(weights + p0 + j) : 0.0f;
      dot[j] = 0.0f;
    }
    for (int64_t c = threadIdx.x; c < nv; c += blockDim.x) {
      typename Io8<In>::Raw y[kPairs] = {};
      if (dweights) {
#pragma unroll
        for (int j = 0; j < kPairs; ++j)
          if (row[j] >= 0) y[j] = Io8<In>::load(ys, row[j] * nv + c);
      }
      const Vec8 d = Io8<DOut>::widen(Io8<DOut>::load(dout, token * nv + c));
#pragma unroll
      for (int j = 0; j < kPairs; ++j) {
        if (row[j] < 0) continue;
        Vec8 g;
#pragma unroll
        for (int e = 0; e < 8; ++e) g.v[e] = w[j] * d.v[e];
        Io8<__nv_bfloat16>::store(dys, row[j] * nv + c, g);
        const Vec8 v = Io8<In>::widen(y[j]);
#pragma unroll
        for (int e = 0; e < 8; ++e) dot[j] = fmaf(d.v[e], v.v[e], dot[j]);
      }
    }
    if (!dweights) continue;
#pragma unroll
    for (int half = kPairs / 2; half > 0; half >>= 1) {                 // lane bits 16, 8, 4
      const int bit = 32 * half / kPairs;
      const bool upper = (lane & bit) != 0;
#pragma unroll
      for (int j = 0; j < half; ++j) {
        const float send = upper ? dot[j] : dot[j + half], keep = upper ? dot[j + half] : dot[j];
        dot[j] = keep + __shfl_xor_sync(0xFFFFFFFFu, send, bit);
      }
    }
    dot[0] += __shfl_xor_sync(0xFFFFFFFFu, dot[0], 2);
    dot[0] += __shfl_xor_sync(0xFFFFFFFFu, dot[0], 1);
    if ((lane & 3) == 0) part[warp][lane >> 2] = dot[0];
    __syncthreads();
    if (threadIdx.x < kPairs && j0 + static_cast<int>(threadIdx.x) < t.top_k) {
      float sum = 0.0f;
      for (unsigned v = 0; v < blockDim.x / 32; ++v) sum += part[v][threadIdx.x];
      dweights[p0 + threadIdx.x] = sum;
    }
    __syncthreads();
  }
}

}  // namespace

// Readies the sort kernels on the current device, once: room for the largest table that a call may ask for (never lowered for a smaller
// one: another host thread may be about to launch with a larger one) and clusters of 16. *ctas: the largest cluster that the device can hold.
static cudaError_t sort_cluster(int* ctas) {
  static int known[64] = {};
  int dev = 0;
  if (cudaError_t e = cudaGetDevice(&dev)) return e;
  if (dev < 64 && (*ctas = __atomic_load_n(&known[dev], __ATOMIC_ACQUIRE))) return cudaSuccess;
  constexpr int kMostSmem = (kSortWarps + 1) * QF_MOE_MAX_EXPERTS * 4;
  bool room = true;
  auto ask = [&](auto kernel) -> cudaError_t {
    if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem)) return e;
    if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1)) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(16);
    cfg.blockDim = dim3(kSortThreads);
    cfg.dynamicSmemBytes = kMostSmem;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 16;
    attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    if (cudaError_t e = cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg)) return e;
    room = room && clusters > 0;
    return cudaSuccess;
  };
  if (cudaError_t e = ask(moe_sort_kernel<int32_t>)) return e;
  if (cudaError_t e = ask(moe_sort_kernel<int64_t>)) return e;
  *ctas = room ? 16 : 8;
  if (dev < 64) __atomic_store_n(&known[dev], *ctas, __ATOMIC_RELEASE);
  return cudaSuccess;
}

cudaError_t launch_moe_sort(const void* ids, bool ids64, int64_t pairs, int G, int64_t rows, int32_t* row_of, int32_t* offs,
                            int32_t* counts, cudaStream_t st) {
  // one CTA of a cluster for every kSortPairs pairs: up to 16 (10.9 us for 131072 pairs to 128 experts, 17.0 with 8 CTAs), or
  // the portable 8 where the device has no room for 16
  constexpr int64_t kSortPairs = 4096;
  int most = 1, ctas = 1;
  if (cudaError_t e = sort_cluster(&most)) return e;
  while (ctas < most && pairs > ctas * kSortPairs) ctas *= 2;
  auto go = [&](auto kernel, auto* p) -> cudaError_t {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kSortThreads);
    cfg.dynamicSmemBytes = static_cast<size_t>(kSortWarps + 1) * G * 4;
    cfg.stream = st;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = ctas;
    attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, p, pairs, G, rows, row_of, offs, counts);
  };
  return ids64 ? go(moe_sort_kernel<int64_t>, static_cast<const int64_t*>(ids)) : go(moe_sort_kernel<int32_t>, static_cast<const int32_t*>(ids));
}

cudaError_t launch_moe_dispatch(const MoeTable& t, const void* x, void* xs, cudaStream_t st) {
  const unsigned tokens = blocks_for(t.tokens * (t.hidden / 8));
  moe_dispatch_kernel<<<tokens + zero_blocks(t), kThreads, 0, st>>>(t, tokens, static_cast<const uint4*>(x), static_cast<uint4*>(xs));
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
  const unsigned tokens = static_cast<unsigned>(t.tokens);
  // a thread for every 8 elements of a token, up to kThreads
  const int64_t lanes = (t.hidden / 8 + 31) / 32 * 32;
  const unsigned threads = lanes < kThreads ? static_cast<unsigned>(lanes) : kThreads;
  auto go = [&](auto kernel) {
    kernel<<<tokens + zero_blocks(t), threads, 0, st>>>(t, tokens, dout, ys, weights, dys, dweights);
    return cudaGetLastError();
  };
  using B = __nv_bfloat16;
  if (dout_dtype == QF_DT_F32) return ys_dtype == QF_DT_F32 ? go(moe_combine_bwd_kernel<float, float>) : go(moe_combine_bwd_kernel<float, B>);
  return ys_dtype == QF_DT_F32 ? go(moe_combine_bwd_kernel<B, float>) : go(moe_combine_bwd_kernel<B, B>);
}

}  // namespace qf
