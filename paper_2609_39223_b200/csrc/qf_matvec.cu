// Products with a few tokens straight from 4-bit codes and block scales: Y = X . deq(W)^T, plain and per expert.
#include "qf_common.cuh"

namespace qf {
namespace {

constexpr int kThreads = 256;

template <typename Id>
__device__ __forceinline__ int expert_id(const void* ids, int64_t p, int G) {
  const Id e = static_cast<const Id*>(ids)[p];
  return e >= 0 && e < static_cast<Id>(G) ? static_cast<int>(e) : -1;
}

// Scale and offset of sub-block b from the 16 metadata bytes of a Q4_K super-block (Eq. q4k-dequant): es = d * s6, em = dmin * m6.
__device__ __forceinline__ float2 q4k_scale(const uint4& r, int b) {
  const float d = __half2float(__ushort_as_half(static_cast<unsigned short>(r.x & 0xFFFFu)));
  const float dmin = __half2float(__ushort_as_half(static_cast<unsigned short>(r.x >> 16)));
  const int sh = 8 * (b & 3);
  const uint32_t lo = r.y >> sh, mid = r.z >> sh, hi = r.w >> sh;      // bytes b&3 of the three groups of four
  const uint32_t s6 = b < 4 ? lo & 63u : (hi & 15u) | ((lo >> 2) & 48u);
  const uint32_t m6 = b < 4 ? mid & 63u : ((hi >> 4) & 15u) | ((mid >> 2) & 48u);
  return make_float2(d * static_cast<float>(s6), dmin * static_cast<float>(m6));
}

// One warp per output element: lanes take units of 16 weights (8 bytes).
template <int FMT>
__global__ void __launch_bounds__(kThreads) matvec_kernel(const MatvecArgs a) {
  const int lane = threadIdx.x & 31;
  const int64_t n = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) >> 5;
  if (n >= a.N) return;
  const int64_t units = a.K / 16;
  for (int64_t m = blockIdx.y; m < a.M; m += gridDim.y) {
    int g = 0;
    if (a.ids) g = a.ids64 ? expert_id<int64_t>(a.ids, m, a.G) : expert_id<int32_t>(a.ids, m, a.G);
    float acc = 0.0f;
    if (g >= 0) {
      const int64_t row = static_cast<int64_t>(g) * a.N + n;
      const uint2* codes = reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(a.codes) + row * (a.K / 2));
      const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(a.X) + (m / a.x_div) * a.K;
      for (int64_t u = lane; u < units; u += 32) {
        const uint2 q = codes[u];
        const uint32_t w[2] = {q.x, q.y};
        if constexpr (FMT == QF_FMT_Q4_K) {
          // byte l of a 32-byte chunk: element l in the low nibble, element l + 32 in the high one
          const int64_t sb = u / 16, chunk = (u / 4) % 4, l0 = (u % 4) * 8;
          const uint4 meta = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(a.scales) + (row * (a.K / 256) + sb) * 16);
          for (int half = 0; half < 2; ++half) {
            const float2 sc = q4k_scale(meta, static_cast<int>(2 * chunk + half));
            const __nv_bfloat16* xp = x + sb * 256 + chunk * 64 + half * 32 + l0;
            float dot = 0.0f, sum = 0.0f;
            for (int l = 0; l < 8; ++l) {
              const float v = __bfloat162float(xp[l]);
              dot = fmaf(static_cast<float>((w[l / 4] >> (8 * (l % 4) + 4 * half)) & 15u), v, dot);
              sum += v;
            }
            acc = fmaf(sc.x, dot, fmaf(-sc.y, sum, acc));
          }
        } else {
          const uint8_t* sc = static_cast<const uint8_t*>(a.scales) + row * (a.K / (FMT == QF_FMT_NVFP4 ? 16 : 32));
          const float s = FMT == QF_FMT_NVFP4 ? e4m3_decode(sc[u]) : e8m0_scale(sc[u / 2]);
          float dot = 0.0f;
          for (int l = 0; l < 8; ++l) {
            const float2 v = e2m1x2_decode((w[l / 4] >> (8 * (l % 4))) & 0xFFu);
            dot = fmaf(v.x, __bfloat162float(x[u * 16 + 2 * l]), dot);
            dot = fmaf(v.y, __bfloat162float(x[u * 16 + 2 * l + 1]), dot);
          }
          acc = fmaf(s, dot, acc);
        }
      }
      for (int d = 16; d > 0; d >>= 1) acc += __shfl_xor_sync(0xFFFFFFFFu, acc, d);
      if (FMT == QF_FMT_NVFP4) acc *= a.tscale[g];
    }
    if (lane == 0) {
      if (a.y_dtype == QF_DT_F32) static_cast<float*>(a.Y)[m * a.N + n] = acc;
      else static_cast<__nv_bfloat16*>(a.Y)[m * a.N + n] = __float2bfloat16_rn(acc);
    }
  }
}

}  // namespace

cudaError_t launch_matvec(const MatvecArgs& a, cudaStream_t st) {
  const dim3 grid(static_cast<unsigned>((a.N + kThreads / 32 - 1) / (kThreads / 32)), static_cast<unsigned>(a.M < 65535 ? a.M : 65535));
  switch (a.fmt) {
    case QF_FMT_NVFP4: matvec_kernel<QF_FMT_NVFP4><<<grid, kThreads, 0, st>>>(a); break;
    case QF_FMT_MXFP4: matvec_kernel<QF_FMT_MXFP4><<<grid, kThreads, 0, st>>>(a); break;
    default: matvec_kernel<QF_FMT_Q4_K><<<grid, kThreads, 0, st>>>(a); break;
  }
  return cudaGetLastError();
}

}  // namespace qf
