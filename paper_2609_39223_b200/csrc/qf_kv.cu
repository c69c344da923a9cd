// The 4-bit key/value cache: keys and values quantized as they are written, rows read back, and attention of a few tokens over it.
#include <math.h>

#include "qf_qdq_body.cuh"

namespace qf {
namespace {

// ---- writing and reading rows --------------------------------------------------------------------------------------------
// A thread owns 16 consecutive elements of one head's row, of the keys or of the values: an NVFP4 block, or half an MXFP4 block (one
// shuffle with its neighbour). Neighbouring threads own neighbouring parts, then heads, then values after keys, then tokens.

struct KvRows {
  const __nv_bfloat16* k;
  const __nv_bfloat16* v;
  int64_t k_stride, v_stride;
  __nv_bfloat16* k_out;
  __nv_bfloat16* v_out;
  const void* slots;
  uint8_t* k_codes;
  uint8_t* k_scales;
  uint8_t* v_codes;
  uint8_t* v_scales;
  const float* k_tscale;
  const float* v_tscale;
  int64_t slots_most;                // of the cache
  int64_t units;                     // parts of 16 elements in all
  int page_size, heads, parts;       // parts: of a row
  bool slots64, noclip;
};

__device__ __forceinline__ int64_t slot_of(const KvRows& p, int64_t t) {
  const int64_t s = p.slots64 ? static_cast<const int64_t*>(p.slots)[t] : static_cast<const int32_t*>(p.slots)[t];
  return s >= 0 && s < p.slots_most ? s : -1;
}

// Part `part` of head h at a slot, in units of 16 elements.
__device__ __forceinline__ int64_t cache_unit(const KvRows& p, int64_t slot, int h, int part) {
  const int64_t page = slot / p.page_size;
  return ((page * p.heads + h) * p.page_size + (slot - page * p.page_size)) * p.parts + part;
}

template <int FMT>
__global__ void __launch_bounds__(kQdqThreads) kv_append_kernel(const KvRows p) {
  const int64_t u = static_cast<int64_t>(blockIdx.x) * kQdqThreads + threadIdx.x;
  const bool any = u < p.units;
  const int64_t i = any ? u : p.units - 1;
  const int part = static_cast<int>(i % p.parts);
  const int64_t row = i / p.parts;
  const int64_t t = row / (2 * p.heads);
  const int hv = static_cast<int>(row - t * 2 * p.heads);
  const bool value = hv >= p.heads;
  const int h = value ? hv - p.heads : hv;
  const uint4* in = reinterpret_cast<const uint4*>((value ? p.v + t * p.v_stride : p.k + t * p.k_stride) + (h * p.parts + part) * 16);
  const uint4 a = in[0], b = in[1];
  const int64_t slot = slot_of(p, t);
  const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  uint32_t m = unit_amax_bits(w), scale_code;
  UnitOut r;
  if (FMT == QF_FMT_MXFP4) {
    m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
    r = mxfp4_unit(w, m, p.noclip, scale_code);
  } else {
    const Nvfp4Tensor nt = nvfp4_tensor(*(value ? p.v_tscale : p.k_tscale));
    const float amax_b = __uint_as_float(m << 16);
    if (__all_sync(0xFFFFFFFFu, nt.denom_safe && (amax_b == 0.0f || amax_b >= 0x1p-60f)))
      r = nvfp4_unit<true>(w, amax_b, nt.s_t, nt.denom, nt.rc_denom, scale_code);
    else r = nvfp4_unit<false>(w, amax_b, nt.s_t, nt.denom, nt.rc_denom, scale_code);
  }
  if (!any || slot < 0) return;
  const int64_t at = cache_unit(p, slot, h, part);
  reinterpret_cast<uint2*>(value ? p.v_codes : p.k_codes)[at] = r.codes;
  uint8_t* scales = value ? p.v_scales : p.k_scales;
  if (FMT == QF_FMT_NVFP4) scales[at] = static_cast<uint8_t>(scale_code);
  else if ((part & 1) == 0) scales[at >> 1] = static_cast<uint8_t>(scale_code);
}

template <int FMT>
__global__ void __launch_bounds__(kQdqThreads) kv_read_kernel(const KvRows p) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kQdqThreads + threadIdx.x;
  if (i >= p.units) return;
  const bool both = p.k_out && p.v_out;
  const int part = static_cast<int>(i % p.parts);
  const int64_t row = i / p.parts;
  const int rows = both ? 2 * p.heads : p.heads;
  const int64_t t = row / rows;
  const int hv = static_cast<int>(row - t * rows);
  const bool value = both ? hv >= p.heads : !p.k_out;
  const int h = both && value ? hv - p.heads : hv;
  const int64_t slot = slot_of(p, t);
  uint32_t w[8] = {};
  if (slot >= 0) {
    const int64_t at = cache_unit(p, slot, h, part);
    const uint2 c = reinterpret_cast<const uint2*>(value ? p.v_codes : p.k_codes)[at];
    const uint8_t* scales = value ? p.v_scales : p.k_scales;
    const float2 st = splat(FMT == QF_FMT_NVFP4 ? *(value ? p.v_tscale : p.k_tscale) : 1.0f);
    const float2 sb = splat(FMT == QF_FMT_NVFP4 ? e4m3_decode(scales[at] & 0x7Fu) : e8m0_scale(scales[at >> 1]));
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float2 o = __fmul2_rn(sb, e2m1x2_decode(((j < 4 ? c.x : c.y) >> (8 * (j & 3))) & 0xFFu));
      if (FMT == QF_FMT_NVFP4) o = __fmul2_rn(o, st);
      w[j] = pack_bf16x2(o.x, o.y);
    }
  }
  uint4* out = reinterpret_cast<uint4*>((value ? p.v_out : p.k_out) + ((t * p.heads + h) * p.parts + part) * 16);
  out[0] = make_uint4(w[0], w[1], w[2], w[3]);
  out[1] = make_uint4(w[4], w[5], w[6], w[7]);
}

KvRows kv_rows(const qf_kv_cache_t& c, const void* slots, bool slots64) {
  KvRows p{};
  p.k_codes = static_cast<uint8_t*>(c.k_codes);
  p.k_scales = static_cast<uint8_t*>(c.k_scales);
  p.v_codes = static_cast<uint8_t*>(c.v_codes);
  p.v_scales = static_cast<uint8_t*>(c.v_scales);
  p.k_tscale = c.k_tscale;
  p.v_tscale = c.v_tscale;
  p.slots = slots;
  p.slots64 = slots64;
  p.slots_most = c.pages * c.page_size;
  p.page_size = c.page_size;
  p.heads = c.kv_heads;
  p.parts = c.head_dim / 16;
  return p;
}

// ---- attention -----------------------------------------------------------------------------------------------------------
// One CTA per (sequence, token, query head): its four warps take every fourth key, a lane D / 32 of the dimensions.

struct KvAttn {
  const __nv_bfloat16* q;
  int64_t q_stride;
  const uint8_t* k_codes;
  const uint8_t* k_scales;
  const uint8_t* v_codes;
  const uint8_t* v_scales;
  const float* k_tscale;
  const float* v_tscale;
  const int32_t* table;
  const int32_t* lens;
  __nv_bfloat16* out;
  float* lse;
  int64_t pages;
  int max_pages, page_size, q_len, q_heads, kv_heads;
  float scale;
};

template <int FMT, int D>
__device__ __forceinline__ void row_values(const uint8_t* codes, const uint8_t* scales, int64_t row, int lane, float (&x)[D / 32]) {
  constexpr int E = D / 32, BLOCK = FMT == QF_FMT_NVFP4 ? 16 : 32;
  const uint32_t s = scales[row * (D / BLOCK) + lane * E / BLOCK];
  const float sb = FMT == QF_FMT_NVFP4 ? e4m3_decode(s & 0x7Fu) : e8m0_scale(s);
#pragma unroll
  for (int i = 0; i < E / 2; ++i) {
    const float2 v = e2m1x2_decode(codes[row * (D / 2) + lane * (E / 2) + i]);
    x[2 * i] = v.x * sb;
    x[2 * i + 1] = v.y * sb;
  }
}

template <int FMT, int D>
__global__ void __launch_bounds__(128) kv_attention_kernel(const KvAttn p) {
  constexpr int E = D / 32;
  const int head = blockIdx.x % p.q_heads;
  const int64_t token = blockIdx.x / p.q_heads;
  const int64_t b = token / p.q_len;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t len = min(static_cast<int64_t>(max(p.lens[b], 0)), static_cast<int64_t>(p.max_pages) * p.page_size);
  const int64_t keys = len - p.q_len + (token - b * p.q_len) + 1;
  const int h = head / (p.q_heads / p.kv_heads);
  float q[E], o[E] = {}, m = -INFINITY, l = 0.0f;
#pragma unroll
  for (int i = 0; i < E; ++i) q[i] = __bfloat162float(p.q[token * p.q_stride + head * D + lane * E + i]);
  const float sk = p.scale * (FMT == QF_FMT_NVFP4 ? *p.k_tscale : 1.0f);
  for (int64_t j = warp; j < keys; j += 4) {
    const int64_t page = min(max(static_cast<int64_t>(p.table[b * p.max_pages + j / p.page_size]), static_cast<int64_t>(0)), p.pages - 1);
    const int64_t row = (page * p.kv_heads + h) * p.page_size + j % p.page_size;
    float x[E], s = 0.0f;
    row_values<FMT, D>(p.k_codes, p.k_scales, row, lane, x);
#pragma unroll
    for (int i = 0; i < E; ++i) s = fmaf(q[i], x[i], s);
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    s *= sk;
    const float top = fmaxf(m, s), keep = expf(m - top), e = expf(s - top);
    row_values<FMT, D>(p.v_codes, p.v_scales, row, lane, x);
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] = fmaf(o[i], keep, e * x[i]);
    l = fmaf(l, keep, e);
    m = top;
  }
  __shared__ float so[4][D], sm[4], sl[4];
#pragma unroll
  for (int i = 0; i < E; ++i) so[warp][lane * E + i] = o[i];
  if (lane == 0) { sm[warp] = m; sl[warp] = l; }
  __syncthreads();
  float top = -INFINITY, total = 0.0f, w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) top = fmaxf(top, sm[i]);
#pragma unroll
  for (int i = 0; i < 4; ++i) { w[i] = top == -INFINITY ? 0.0f : expf(sm[i] - top); total = fmaf(w[i], sl[i], total); }
  const float by = total > 0.0f ? (FMT == QF_FMT_NVFP4 ? *p.v_tscale : 1.0f) / total : 0.0f;
  for (int d = threadIdx.x; d < D; d += 128)
    p.out[(token * p.q_heads + head) * D + d] = __float2bfloat16_rn((w[0] * so[0][d] + w[1] * so[1][d] + w[2] * so[2][d] + w[3] * so[3][d]) * by);
  if (p.lse && threadIdx.x == 0) p.lse[token * p.q_heads + head] = total > 0.0f ? top + logf(total) : -INFINITY;
}

template <int FMT>
cudaError_t attend(const KvAttn& p, int head_dim, int64_t ctas, cudaStream_t st) {
  const unsigned grid = static_cast<unsigned>(ctas);
  if (head_dim == 64) kv_attention_kernel<FMT, 64><<<grid, 128, 0, st>>>(p);
  else if (head_dim == 128) kv_attention_kernel<FMT, 128><<<grid, 128, 0, st>>>(p);
  else kv_attention_kernel<FMT, 256><<<grid, 128, 0, st>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv_append(const qf_kv_cache_t& c, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int64_t tokens,
                             const void* slots, bool slots64, bool noclip, cudaStream_t st) {
  KvRows p = kv_rows(c, slots, slots64);
  p.k = static_cast<const __nv_bfloat16*>(k);
  p.v = static_cast<const __nv_bfloat16*>(v);
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.noclip = noclip;
  p.units = tokens * 2 * p.heads * p.parts;
  const unsigned grid = static_cast<unsigned>((p.units + kQdqThreads - 1) / kQdqThreads);
  if (c.fmt == QF_FMT_NVFP4) kv_append_kernel<QF_FMT_NVFP4><<<grid, kQdqThreads, 0, st>>>(p);
  else kv_append_kernel<QF_FMT_MXFP4><<<grid, kQdqThreads, 0, st>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_kv_read(const qf_kv_cache_t& c, const void* slots, bool slots64, int64_t rows, void* k, void* v, cudaStream_t st) {
  KvRows p = kv_rows(c, slots, slots64);
  p.k_out = static_cast<__nv_bfloat16*>(k);
  p.v_out = static_cast<__nv_bfloat16*>(v);
  p.units = rows * (k && v ? 2 : 1) * p.heads * p.parts;
  const unsigned grid = static_cast<unsigned>((p.units + kQdqThreads - 1) / kQdqThreads);
  if (c.fmt == QF_FMT_NVFP4) kv_read_kernel<QF_FMT_NVFP4><<<grid, kQdqThreads, 0, st>>>(p);
  else kv_read_kernel<QF_FMT_MXFP4><<<grid, kQdqThreads, 0, st>>>(p);
  return cudaGetLastError();
}

size_t kv_attention_ws_bytes(int64_t, int, int, int) { return 0; }

cudaError_t launch_kv_attention(const KvAttentionArgs& a, cudaStream_t st) {
  KvAttn p{};
  p.q = static_cast<const __nv_bfloat16*>(a.q);
  p.q_stride = a.q_stride;
  p.k_codes = static_cast<const uint8_t*>(a.cache.k_codes);
  p.k_scales = static_cast<const uint8_t*>(a.cache.k_scales);
  p.v_codes = static_cast<const uint8_t*>(a.cache.v_codes);
  p.v_scales = static_cast<const uint8_t*>(a.cache.v_scales);
  p.k_tscale = a.cache.k_tscale;
  p.v_tscale = a.cache.v_tscale;
  p.table = a.table;
  p.lens = a.lens;
  p.out = static_cast<__nv_bfloat16*>(a.out);
  p.lse = a.lse;
  p.pages = a.cache.pages;
  p.max_pages = static_cast<int>(a.max_pages);
  p.page_size = a.cache.page_size;
  p.q_len = a.q_len;
  p.q_heads = a.q_heads;
  p.kv_heads = a.cache.kv_heads;
  p.scale = a.scale;
  const int64_t ctas = a.batch * a.q_len * a.q_heads;
  return a.cache.fmt == QF_FMT_NVFP4 ? attend<QF_FMT_NVFP4>(p, a.cache.head_dim, ctas, st) : attend<QF_FMT_MXFP4>(p, a.cache.head_dim, ctas, st);
}

}  // namespace qf
