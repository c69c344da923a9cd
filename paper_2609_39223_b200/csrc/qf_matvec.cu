// Products with a few tokens straight from 4-bit codes and block scales: Y = X . deq(W)^T, plain and per expert.
//
// The weights are the only large operand, so the bound is the read of codes and scales (0.53-0.56 bytes per weight). One
// FP32 multiply-add per weight and token would cost more issue slots than that read leaves (about 2.8 instructions per weight
// at the copy rate), and the decode alone takes two. So the multiply-adds go to mma.sync m16n8k16 (16 weight rows x 8
// tokens): a tcgen05 tile needs 128 rows of an operand in shared memory, which would mean writing every decoded weight there
// first; here the decoded weights never leave registers.
//
//  * A fragments: a lane loads 32 (or 8) consecutive bytes of codes of one weight row and decodes them in place. Which k a
//    lane's elements stand for is free as long as both operands agree, so no code is ever moved between lanes.
//  * B fragments: the CTA stages its slice of X in shared memory once, already in the order the lanes read it.
//  * FP4 codes become BF16 by one multiplication: a nibble times 0x1040 puts its sign at bit 15 and its three other bits
//    at bits 8..6, which is the value as a BF16 number scaled by 2^-126 (subnormals included); one packed BF16 product
//    with the block scale times a power of two gives value * scale, exactly (two and four significant bits).
//  * Q4_K codes are whole numbers below 16; a sub-block's sum of C*x is finished in FP32 with its scale and offset.
//  * Rows are cut into tiles of 16 for a warp; the contraction is split over the warps of a CTA and over the CTAs of a cluster
//    where there are too few tiles to keep every SM loading; the parts meet in (distributed) shared memory in a fixed order.
#include <cooperative_groups.h>

#include "qf_common.cuh"

namespace cg = cooperative_groups;

namespace qf {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kListCap = 1024;                       // pairs looked at in one go by a CTA of the grouped product
constexpr int kXBytes = 64 * 1024;                   // shared memory for the staged slice of X

struct MvParams {
  const __nv_bfloat16* X;
  const uint8_t* codes;
  const uint8_t* scales;
  const float* tscale;
  const void* ids;
  void* Y;
  int64_t x_div;
  int M, N, K, G;
  int kw;                                            // warps of a CTA that share a row tile (1, 2, 4 or 8)
  int kz;                                            // contraction length of a CTA (a multiple of 256)
  int kc;                                            // contraction length staged at a time (a multiple of 256)
  int x_words;                                       // 32-bit words of shared memory for X
  bool ids64, by_pair, y_f32;
};

__device__ __forceinline__ int expert_id(const MvParams& p, int i) {
  if (p.ids64) {
    const int64_t e = static_cast<const int64_t*>(p.ids)[i];
    return e >= 0 && e < p.G ? static_cast<int>(e) : -1;
  }
  const int32_t e = static_cast<const int32_t*>(p.ids)[i];
  return e >= 0 && e < p.G ? e : -1;
}

// D += A . B, A 16x16 and B 16x8 in BF16, FP32 accumulators
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) { return bf2_bits(__hmul2(bits_bf2(a), bits_bf2(b))); }

// Eight E2M1 codes -> four BF16 pairs (elements i and i + 4), each the code's value times 2^-126.
__device__ __forceinline__ void e2m1_words(uint32_t q, uint32_t (&w)[4]) {
  const uint32_t h = q >> 8;
  w[0] = ((q & 0x000F000Fu) * 0x1040u) & 0x81C081C0u;
  w[1] = ((q & 0x00F000F0u) * 0x0104u) & 0x81C081C0u;
  w[2] = ((h & 0x000F000Fu) * 0x1040u) & 0x81C081C0u;
  w[3] = ((h & 0x00F000F0u) * 0x0104u) & 0x81C081C0u;
}

// 16 elements of X in the order the A words have: FP4 pairs (i, i + 4), Q4_K pairs (i, i + 2)
template <int FMT>
__device__ __forceinline__ uint4 x_unit(uint4 v) {
  if constexpr (FMT == QF_FMT_Q4_K)
    return make_uint4(__byte_perm(v.x, v.y, 0x5410), __byte_perm(v.x, v.y, 0x7632), __byte_perm(v.z, v.w, 0x5410), __byte_perm(v.z, v.w, 0x7632));
  else
    return make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
}

__device__ __forceinline__ void load32(const uint8_t* p, uint32_t (&q)[8]) {
  asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(q[0]), "=r"(q[1]), "=r"(q[2]), "=r"(q[3]), "=r"(q[4]), "=r"(q[5]), "=r"(q[6]), "=r"(q[7])
               : "l"(p));
}

// What a lane holds of one weight row for one step of the contraction: FP4 wide 64 weights (a step is 256), FP4 narrow 16
// weights (a step is 64), Q4_K 64 weights of a super-block (8 bytes of each of its four chunks).
template <int FMT, bool WIDE>
struct RowPart {
  static constexpr int kWords = FMT == QF_FMT_Q4_K || WIDE ? 8 : 2;
  uint32_t q[kWords];
  uint32_t s[FMT == QF_FMT_Q4_K ? 4 : 1];            // block scales as stored
};

template <int FMT, bool WIDE>
__device__ __forceinline__ void load_part(RowPart<FMT, WIDE>& r, const uint8_t* codes, const uint8_t* scales, int k_step, int K, int t) {
  if constexpr (FMT == QF_FMT_Q4_K) {
    const uint8_t* c = codes + k_step / 2 + t * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint2 v = __ldg(reinterpret_cast<const uint2*>(c + 32 * i));
      r.q[2 * i] = v.x;
      r.q[2 * i + 1] = v.y;
    }
    const uint4 m = __ldg(reinterpret_cast<const uint4*>(scales + k_step / 16));
    r.s[0] = m.x; r.s[1] = m.y; r.s[2] = m.z; r.s[3] = m.w;
  } else {
    const int k = k_step + t * (WIDE ? 64 : 16);
    if (k < K) {
      if constexpr (WIDE) {
        load32(codes + k / 2, r.q);
        if constexpr (FMT == QF_FMT_NVFP4) r.s[0] = __ldg(reinterpret_cast<const uint32_t*>(scales + k / 16));
        else r.s[0] = __ldg(reinterpret_cast<const uint16_t*>(scales + k / 32));
      } else {
        const uint2 v = __ldg(reinterpret_cast<const uint2*>(codes + k / 2));
        r.q[0] = v.x;
        r.q[1] = v.y;
        r.s[0] = __ldg(scales + k / (FMT == QF_FMT_NVFP4 ? 16 : 32));
      }
    } else {
#pragma unroll
      for (int i = 0; i < RowPart<FMT, WIDE>::kWords; ++i) r.q[i] = 0u;
      r.s[0] = 0u;
    }
  }
}

// The packed BF16 factor that turns value * 2^-126 into value * scale (NVFP4: times 2^-7, put right at the end).
template <int FMT>
__device__ __forceinline__ uint32_t fp4_factor(uint32_t code) {
  if constexpr (FMT == QF_FMT_NVFP4) {
    // code << 20 is the scale times 2^-120 as FP32
    const uint32_t f = __float_as_uint(__fmul_rn(__fmul_rn(__uint_as_float(code << 20), 0x1p127f), 0x1p112f));
    return __byte_perm(f, f, 0x3232);
  } else {
    return min(code + 126u, 254u) * 0x00800080u;       // 2^(p + 126), p = code - 127; above p = 1 the rest follows separately
  }
}

template <int FMT, int NT, bool WIDE>
__global__ void __launch_bounds__(kThreads, 2) matvec_kernel(const __grid_constant__ MvParams p) {
  constexpr int MT = 8 * NT;                           // tokens of a pass
  constexpr bool Q4K = FMT == QF_FMT_Q4_K;
  constexpr int STEP = Q4K || WIDE ? 256 : 64;
  constexpr int LW = Q4K || WIDE ? 8 : 2;              // 16-byte units of X per lane and step
  extern __shared__ uint4 smem[];                      // X slice | Q4_K: sums of X per sub-block | partial sums
  uint4* xs = smem;
  float* sx = reinterpret_cast<float*>(smem) + p.x_words;                          // [kc / 32][MT]
  float* red = sx + (Q4K ? p.kc / 32 * MT : 0);                                    // [kw][rows of the CTA][MT]
  __shared__ int list[kListCap];
  __shared__ int warp_count[kWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int rows_cta = kWarps / p.kw * 16;
  const int rw = warp / p.kw, kw = warp - rw * p.kw;
  const int n_cta = blockIdx.x * rows_cta, n_warp = n_cta + rw * 16;
  const int z = blockIdx.z, nz = gridDim.z;
  const int k_begin = z * p.kz, k_end = min(p.K, k_begin + p.kz);

  int e = 0;
  if (p.ids) {
    if (p.by_pair) {
      // slot = pair: the first pair that names an expert takes all pairs that do
      e = expert_id(p, blockIdx.y);
      bool seen = false;
      for (int i = tid; i < static_cast<int>(blockIdx.y); i += kThreads) seen |= expert_id(p, i) == e;
      if (__syncthreads_or(seen) && e >= 0) return;
      if (e < 0) {
        if (z == 0)
          for (int i = tid; i < min(rows_cta, p.N - n_cta); i += kThreads) {
            const int64_t at = static_cast<int64_t>(blockIdx.y) * p.N + n_cta + i;
            if (p.y_f32) static_cast<float*>(p.Y)[at] = 0.0f;
            else static_cast<__nv_bfloat16*>(p.Y)[at] = __float2bfloat16_rn(0.0f);
          }
        return;
      }
    } else {
      e = blockIdx.y;
    }
  }
  const float tscale = FMT == QF_FMT_NVFP4 ? p.tscale[e] * 0x1p7f : 1.0f;
  const int64_t row0 = static_cast<int64_t>(e) * p.N;
  const int64_t ra = row0 + min(n_warp + g, p.N - 1), rb = row0 + min(n_warp + g + 8, p.N - 1);
  const int64_t scale_pitch = Q4K ? p.K / 16 : p.K / (FMT == QF_FMT_NVFP4 ? 16 : 32);
  const uint8_t* ca = p.codes + ra * (p.K / 2);
  const uint8_t* cb = p.codes + rb * (p.K / 2);
  const uint8_t* sa = p.scales + ra * scale_pitch;
  const uint8_t* sb = p.scales + rb * scale_pitch;

  for (int w0 = 0; w0 < p.M; w0 += kListCap) {
    // the rows of Y that this CTA's weights serve
    const int w1 = min(p.M, w0 + kListCap);
    int count = w1 - w0;
    if (p.ids) {
      count = 0;
      for (int i0 = w0; i0 < w1; i0 += kThreads) {
        const int i = i0 + tid;
        const int id = i < w1 ? expert_id(p, i) : -2;
        const bool mine = id == e;
        if (!p.by_pair && e == 0 && id == -1 && z == 0)
          for (int n = n_cta; n < min(n_cta + rows_cta, p.N); ++n) {
            const int64_t at = static_cast<int64_t>(i) * p.N + n;
            if (p.y_f32) static_cast<float*>(p.Y)[at] = 0.0f;
            else static_cast<__nv_bfloat16*>(p.Y)[at] = __float2bfloat16_rn(0.0f);
          }
        const uint32_t vote = __ballot_sync(0xFFFFFFFFu, mine);
        __syncthreads();
        if (lane == 0) warp_count[warp] = __popc(vote);
        __syncthreads();
        int at = count + __popc(vote & ((1u << lane) - 1u));
        for (int w = 0; w < kWarps; ++w) {
          if (w < warp) at += warp_count[w];
          count += warp_count[w];
        }
        if (mine) list[at] = i;
      }
      __syncthreads();
    }
    for (int c0 = 0; c0 < count; c0 += MT) {
      const int mt = min(MT, count - c0);
      float acc[NT][4] = {};
      for (int kc0 = k_begin; kc0 < k_end; kc0 += p.kc) {
        const int kc1 = min(kc0 + p.kc, k_end), steps = (kc1 - kc0 + STEP - 1) / STEP;
        RowPart<FMT, WIDE> a[2], b[2];
        if (kw < steps) {
          load_part(a[0], ca, sa, kc0 + kw * STEP, p.K, t);
          load_part(b[0], cb, sb, kc0 + kw * STEP, p.K, t);
        }
        __syncthreads();
        // X slice: unit u of 8 elements of token m; zeros past the end of the contraction
        const int units = steps * (STEP / 8);
        for (int i = tid; i < mt * units; i += kThreads) {
          const int m = i / units, u = i - m * units, k = kc0 + u * 8;
          const int64_t row = p.ids ? list[c0 + m] : w0 + c0 + m;
          uint4 v = make_uint4(0u, 0u, 0u, 0u);
          if (k < p.K) v = __ldg(reinterpret_cast<const uint4*>(p.X + row / p.x_div * p.K + k));
          if constexpr (Q4K) {
            xs[((u >> 2) * mt + m) * 4 + (u & 3)] = x_unit<FMT>(v);
            const float s = bf16_lo(v.x) + bf16_hi(v.x) + bf16_lo(v.y) + bf16_hi(v.y) + (bf16_lo(v.z) + bf16_hi(v.z) + bf16_lo(v.w) + bf16_hi(v.w));
            // units is a multiple of 32, so the four lanes of a sub-block are here together
            const float s2 = s + __shfl_xor_sync(0xFFFFFFFFu, s, 1);
            const float s4 = s2 + __shfl_xor_sync(0xFFFFFFFFu, s2, 2);
            if ((u & 3) == 0) sx[(u >> 2) * MT + m] = s4;
          } else {
            xs[((u / (4 * LW) * LW + u % LW) * mt + m) * 4 + u / LW % 4] = x_unit<FMT>(v);
          }
        }
        __syncthreads();
        for (int s0 = kw, i = 0; s0 < steps; s0 += 2 * p.kw, i += 2) {
#pragma unroll
          for (int d = 0; d < 2; ++d) {
            const int s = s0 + d * p.kw;
            if (s < steps) {
              if (s + p.kw < steps) {
                load_part(a[1 - d], ca, sa, kc0 + (s + p.kw) * STEP, p.K, t);
                load_part(b[1 - d], cb, sb, kc0 + (s + p.kw) * STEP, p.K, t);
              }
              if constexpr (Q4K) {
                const uint4 ma = make_uint4(a[d].s[0], a[d].s[1], a[d].s[2], a[d].s[3]), mb = make_uint4(b[d].s[0], b[d].s[1], b[d].s[2], b[d].s[3]);
                const uint32_t s6a[2] = {ma.y & 0x3F3F3F3Fu, (ma.w & 0x0F0F0F0Fu) | ((ma.y >> 2) & 0x30303030u)};
                const uint32_t m6a[2] = {ma.z & 0x3F3F3F3Fu, ((ma.w >> 4) & 0x0F0F0F0Fu) | ((ma.z >> 2) & 0x30303030u)};
                const uint32_t s6b[2] = {mb.y & 0x3F3F3F3Fu, (mb.w & 0x0F0F0F0Fu) | ((mb.y >> 2) & 0x30303030u)};
                const uint32_t m6b[2] = {mb.z & 0x3F3F3F3Fu, ((mb.w >> 4) & 0x0F0F0F0Fu) | ((mb.z >> 2) & 0x30303030u)};
                const float2 fa = __half22float2(*reinterpret_cast<const __half2*>(&ma.x)), fb = __half22float2(*reinterpret_cast<const __half2*>(&mb.x));
#pragma unroll
                for (int blk = 0; blk < 8; ++blk) {
                  const uint32_t qa[2] = {a[d].q[blk / 2 * 2] >> (4 * (blk & 1)), a[d].q[blk / 2 * 2 + 1] >> (4 * (blk & 1))};
                  const uint32_t qb[2] = {b[d].q[blk / 2 * 2] >> (4 * (blk & 1)), b[d].q[blk / 2 * 2 + 1] >> (4 * (blk & 1))};
                  uint32_t wa[4], wb[4];
#pragma unroll
                  for (int h = 0; h < 4; ++h) {       // 128 + C as BF16, minus 128
                    const __nv_bfloat162 off = bits_bf2(0x43004300u);
                    wa[h] = bf2_bits(__hsub2(bits_bf2(((qa[h / 2] >> (8 * (h & 1))) & 0x000F000Fu) | 0x43004300u), off));
                    wb[h] = bf2_bits(__hsub2(bits_bf2(((qb[h / 2] >> (8 * (h & 1))) & 0x000F000Fu) | 0x43004300u), off));
                  }
                  const float esa = fa.x * static_cast<float>((s6a[blk / 4] >> (8 * (blk & 3))) & 63u);
                  const float ema = fa.y * static_cast<float>((m6a[blk / 4] >> (8 * (blk & 3))) & 63u);
                  const float esb = fb.x * static_cast<float>((s6b[blk / 4] >> (8 * (blk & 3))) & 63u);
                  const float emb = fb.y * static_cast<float>((m6b[blk / 4] >> (8 * (blk & 3))) & 63u);
                  const uint32_t f0[4] = {wa[0], wb[0], wa[1], wb[1]}, f1[4] = {wa[2], wb[2], wa[3], wb[3]};
                  const int sub = s * 8 + blk;
#pragma unroll
                  for (int nt = 0; nt < NT; ++nt) {
                    uint4 x = make_uint4(0u, 0u, 0u, 0u);
                    if (nt * 8 + g < mt) x = xs[(sub * mt + nt * 8 + g) * 4 + t];
                    float c[4] = {};
                    mma16816(c, f0, x.x, x.y);
                    mma16816(c, f1, x.z, x.w);
                    const float2 sum = *reinterpret_cast<const float2*>(sx + sub * MT + nt * 8 + 2 * t);
                    acc[nt][0] = fmaf(esa, c[0], fmaf(-ema, sum.x, acc[nt][0]));
                    acc[nt][1] = fmaf(esa, c[1], fmaf(-ema, sum.y, acc[nt][1]));
                    acc[nt][2] = fmaf(esb, c[2], fmaf(-emb, sum.x, acc[nt][2]));
                    acc[nt][3] = fmaf(esb, c[3], fmaf(-emb, sum.y, acc[nt][3]));
                  }
                }
              } else {
                constexpr int PER = FMT == QF_FMT_NVFP4 ? 2 : 4;         // words of codes per scale
                float c[NT][4] = {};
#pragma unroll
                for (int w = 0; w < LW; ++w) {
                  const uint32_t ea = (a[d].s[0] >> (8 * (w / PER))) & 0xFFu, eb = (b[d].s[0] >> (8 * (w / PER))) & 0xFFu;
                  const uint32_t fa = fp4_factor<FMT>(ea), fb = fp4_factor<FMT>(eb);
                  uint32_t wa[4], wb[4];
                  e2m1_words(a[d].q[w], wa);
                  e2m1_words(b[d].q[w], wb);
#pragma unroll
                  for (int h = 0; h < 4; ++h) {
                    wa[h] = mul_bf16x2(wa[h], fa);
                    wb[h] = mul_bf16x2(wb[h], fb);
                  }
                  if constexpr (FMT == QF_FMT_MXFP4) {
                    // scales above 2^1 (weights of 8 and more): the rest of the power
                    if (__any_sync(0xFFFFFFFFu, max(ea, eb) > 128u)) {
                      const uint32_t ga = (max(ea, 128u) - 1u) * 0x00800080u, gb = (max(eb, 128u) - 1u) * 0x00800080u;
#pragma unroll
                      for (int h = 0; h < 4; ++h) {
                        wa[h] = mul_bf16x2(wa[h], ga);
                        wb[h] = mul_bf16x2(wb[h], gb);
                      }
                    }
                  }
                  const uint32_t f0[4] = {wa[0], wb[0], wa[1], wb[1]}, f1[4] = {wa[2], wb[2], wa[3], wb[3]};
#pragma unroll
                  for (int nt = 0; nt < NT; ++nt) {
                    uint4 x = make_uint4(0u, 0u, 0u, 0u);
                    if (nt * 8 + g < mt) x = xs[((s * LW + w) * mt + nt * 8 + g) * 4 + t];
                    mma16816(c[nt], f0, x.x, x.y);
                    mma16816(c[nt], f1, x.z, x.w);
                  }
                }
                // the tensor core truncates as it accumulates: a step at a time, the steps in FP32 adds
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                  for (int j = 0; j < 4; ++j) acc[nt][j] += c[nt][j];
              }
            }
          }
        }
      }
      // partial sums: [kw][row][token]
      float* mine = red + (kw * rows_cta + rw * 16) * MT;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 4; ++j) mine[(g + (j >> 1) * 8) * MT + nt * 8 + 2 * t + (j & 1)] = acc[nt][j];
      if (nz > 1) cg::this_cluster().sync();
      else __syncthreads();
      // CTA z of the cluster finishes every nz-th part of the outputs
      for (int i = tid + z * kThreads; i < rows_cta * mt; i += kThreads * nz) {
        const int m = i / rows_cta, r = i - m * rows_cta, n = n_cta + r;
        if (n >= p.N) continue;
        float sum = 0.0f;
        for (int zz = 0; zz < nz; ++zz) {
          const float* part = nz > 1 ? cg::this_cluster().map_shared_rank(red, zz) : red;
          for (int k = 0; k < p.kw; ++k) sum += part[(k * rows_cta + r) * MT + m];
        }
        const int64_t row = p.ids ? list[c0 + m] : w0 + c0 + m;
        if (FMT == QF_FMT_NVFP4) sum *= tscale;
        if (p.y_f32) static_cast<float*>(p.Y)[row * p.N + n] = sum;
        else static_cast<__nv_bfloat16*>(p.Y)[row * p.N + n] = __float2bfloat16_rn(sum);
      }
      if (nz > 1) cg::this_cluster().sync();
      else __syncthreads();
    }
  }
}

template <int FMT, int NT, bool WIDE>
cudaError_t launch(const MvParams& p, dim3 grid, size_t smem, cudaStream_t st) {
  auto kernel = matvec_kernel<FMT, NT, WIDE>;
  if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 128 * 1024)) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = 1;
  attr.val.clusterDim.y = 1;
  attr.val.clusterDim.z = grid.z;
  cfg.attrs = &attr;
  cfg.numAttrs = grid.z > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <int FMT, bool WIDE>
cudaError_t launch_nt(int nt, const MvParams& p, dim3 grid, size_t smem, cudaStream_t st) {
  if (nt == 1) return launch<FMT, 1, WIDE>(p, grid, smem, st);
  if (nt == 2) return launch<FMT, 2, WIDE>(p, grid, smem, st);
  return launch<FMT, 4, WIDE>(p, grid, smem, st);
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

cudaError_t launch_matvec(const MatvecArgs& a, cudaStream_t st) {
  MvParams p{};
  p.X = static_cast<const __nv_bfloat16*>(a.X);
  p.codes = static_cast<const uint8_t*>(a.codes);
  p.scales = static_cast<const uint8_t*>(a.scales);
  p.tscale = a.tscale;
  p.ids = a.ids;
  p.ids64 = a.ids64;
  p.Y = a.Y;
  p.x_div = a.x_div;
  p.M = static_cast<int>(a.M); p.N = static_cast<int>(a.N); p.K = static_cast<int>(a.K); p.G = a.G;
  p.y_f32 = a.y_dtype == QF_DT_F32;
  p.by_pair = a.ids && a.M <= a.G;
  const int slots = !a.ids ? 1 : p.by_pair ? p.M : a.G;
  // tokens of a pass: few pairs per expert are the rule in the grouped product
  const int nt = a.ids ? (a.M <= 4ll * a.G || a.M <= 8 ? 1 : 4) : a.M <= 8 ? 1 : a.M <= 16 ? 2 : 4;
  const int mt = static_cast<int>(a.M < 8 * nt ? a.M : 8 * nt);
  // Split of the contraction: enough warps for 16 on each SM, no warp with less than one step of 256. Within a CTA the warps
  // that share a row tile multiply the traffic for X (every CTA stages its slice), so with many tokens the cluster splits.
  const int64_t tiles = ceil_div(a.N, 16) * slots;
  int split = 1;
  while (split < 64 && tiles * split < 16 * kNumSMs && a.K > 256 * split) split *= 2;
  const int kw_most = mt <= 2 ? 8 : mt <= 4 ? 4 : 2;
  p.kw = split < kw_most ? split : kw_most;
  int nz = split / p.kw;
  if (nz > 8) nz = 8;
  p.kz = static_cast<int>(ceil_div(ceil_div(a.K, nz), 256) * 256);
  nz = static_cast<int>(ceil_div(a.K, p.kz));
  const int kc_most = kXBytes / (2 * mt) / 256 * 256;
  p.kc = p.kz < kc_most ? p.kz : kc_most;
  p.x_words = mt * p.kc / 2;
  const int rows_cta = kWarps / p.kw * 16;
  const size_t smem = 4 * (static_cast<size_t>(p.x_words) + (a.fmt == QF_FMT_Q4_K ? p.kc / 32 * 8 * nt : 0) + kWarps * 16 * 8 * nt);
  const dim3 grid(static_cast<unsigned>(ceil_div(a.N, rows_cta)), static_cast<unsigned>(slots), static_cast<unsigned>(nz));
  // 32-byte loads of codes need rows that start on 32 bytes
  const bool wide = a.K % 64 == 0 && (reinterpret_cast<uintptr_t>(a.codes) & 31u) == 0;
  switch (a.fmt) {
    case QF_FMT_NVFP4: return wide ? launch_nt<QF_FMT_NVFP4, true>(nt, p, grid, smem, st) : launch_nt<QF_FMT_NVFP4, false>(nt, p, grid, smem, st);
    case QF_FMT_MXFP4: return wide ? launch_nt<QF_FMT_MXFP4, true>(nt, p, grid, smem, st) : launch_nt<QF_FMT_MXFP4, false>(nt, p, grid, smem, st);
    default: return launch_nt<QF_FMT_Q4_K, true>(nt, p, grid, smem, st);
  }
}

}  // namespace qf
