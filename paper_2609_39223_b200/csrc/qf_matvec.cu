// Products with a few tokens straight from 4-bit codes and block scales: Y = X . deq(W)^T, plain and per expert.
//
// The weights are the only large operand, so the floor is the read of codes and scales (0.53-0.56 bytes per weight). At the
// copy rate that leaves about 2.8 instructions per weight, decode included: too few for one FP32 multiply-add per weight and
// token. So the multiply-adds go to mma.sync m16n8k16 (16 weight rows x 8 tokens): a tcgen05 tile needs 128 rows of an operand
// in shared memory, which would mean writing every decoded weight there first; here decoded weights never leave registers.
//
//  * A fragments: a lane decodes 32 consecutive bytes of codes of one weight row in place. Which k a lane's elements stand
//    for is free as long as both operands agree, so no code is ever moved between lanes.
//  * Every decoded weight is exact in FP16 up to a factor that a row or a step shares: E2M1 value times E4M3 scale has six
//    significant bits; E2M1 value times 2^p is exact while p lies in [-21, 5]; a Q4_K code C times its 6-bit scale s6 is a whole
//    number below 1024, kept as that multiple of 2^-24 (an FP16 subnormal is its own bit pattern, so C needs no conversion).
//    One conversion and one packed product decode two FP4 weights, one mask and one product two Q4_K weights.
//  * B fragments: the CTA stages its slice of X in shared memory once, in the order the lanes read it, as FP16 of 2^6 x. That is
//    exact for zeros and 2^-23 <= |x| < 1023. A token that has another x in a step of the contraction (or a tile with another p)
//    takes that step with BF16 fragments, weights and X read again: a sum of exact products either way, so the choice
//    costs time only. It goes by token: rows of X do not influence one another. One of ten million N(0, 1) values falls below,
//    but 2.5e-6 of silu(g) u with g, u ~ N(0, 1), 5e-5 with N(0, 0.2), 6e-4 with N(0, 0.05); and an all-zero MXFP4 block has scale code
//    0. A warp that meets one reads all its steps of every tile again: NVFP4 4096 x 14336 with one token takes 13.1 us for N(0, 1) and
//    for silu(g) u of N(0, 1), 17.5 and 29.0 for N(0, 0.2) and N(0, 0.05); MXFP4 31.4 instead of 12.6 with one row of 64 zero.
//  * BF16 fragments from FP4 codes: a nibble times 0x1040 puts its sign at bit 15 and its three other bits at bits 8..6, which is
//    the value as a BF16 number scaled by 2^-126 (subnormals included); a packed product with the scale gives value * scale.
//    This takes 15 instructions for eight weights where the FP16 route takes 8, which is why it is not the only route.
//  * Q4_K offsets: sum over sub-blocks of m6 * sum(x) is a product of its own, 8 sub-blocks deep, with the sums of x split into
//    three BF16 parts (24 bits); one FP32 multiply-add per super-block applies d and dmin.
//  * The tensor core truncates as it accumulates: it adds up one step of 256 elements at a time, the steps are added in FP32.
//  * Codes arrive through a ring of kStages steps per warp in shared memory (cp.async), so that loads in flight cost no registers.
//  * Rows are cut into tiles of 16 for a warp; the contraction is split over the warps of a CTA and over the CTAs of a
//    cluster where there are too few tiles to keep every SM loading; the parts meet in (distributed) shared memory in a fixed order.
//
// What bounds it. 128256 x 4096, NVFP4: 59 us with one token (5.0 TB/s, 0.76 of the copy rate), 64 with 8, 80 with 16; MXFP4 81 with 16;
// Q4_K 70 with one (4.2 TB/s). A warp's step of 16 x 256 weights takes about 250 instructions: 165 to decode and multiply (Q4_K
// 205), 45 for the ring, the rest for tile ends and X. Decode and products alone, from registers, take an SM's schedulers 286
// cycles a step (440 with two token tiles, whose X also takes 0.6 of the shared memory bandwidth) where the copy rate allows 394: both
// have to overlap with four warps a scheduler, which is all that 128 registers leave (at 96 registers the spills cost 1.7 times). Sums
// kept in two chains of products, Q4_K scales applied after the products instead of before: no gain, 1.03 times as long.
// Small weights are bound by the launch, one staging of X and one trip to memory: 1024 x 4096 takes 5.1 us.
#include <cooperative_groups.h>
#include <math.h>

#include <type_traits>

#include "qf_common.cuh"

namespace cg = cooperative_groups;

namespace qf {
namespace {

constexpr int kWarpsMost = 16;                       // of a CTA; 128 registers a thread, so 16 warps fill an SM
// Steps of codes that a warp has in shared memory or on the way: four (9 KB a warp), or two where the X of two token tiles takes the
// room (five tokens, 4096 x 14336: 17.9 us with two, 15.3 with four and the contraction split at any step)
template <int NT>
constexpr int kStages = NT == 1 ? 4 : 2;
constexpr int kSmemMost = 232448 - 128;              // dynamic shared memory of a CTA
constexpr float kXScale = 64.0f;                     // X is staged as FP16 of this times x
constexpr int kListCap = 1024;                       // pairs looked at in one go by a CTA of the grouped product

struct MvParams {
  const __nv_bfloat16* X;
  const uint8_t* codes;
  const uint8_t* scales;
  const uint8_t* scales_end;
  const float* tscale;
  const void* ids;
  void* Y;
  int x_div;
  int M, N, K, G;
  int blocks;                                        // row blocks of a weight; CTA x takes blocks x, x + gridDim.x, ...
  int kw;                                            // warps of a CTA that share a row tile
  int kz;                                            // contraction length of a CTA (a multiple of 256)
  int kc;                                            // contraction length staged at a time (a multiple of 256)
  int sx_at, flags_at, list_at, red_at, ring_at;     // bytes from the start of dynamic shared memory (X comes first)
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

__device__ __forceinline__ void store_y(const MvParams& p, int64_t row, int n, float v) {
  if (p.y_f32) static_cast<float*>(p.Y)[row * p.N + n] = v;
  else static_cast<__nv_bfloat16*>(p.Y)[row * p.N + n] = __float2bfloat16_rn(v);
}

// D = A . B (+ D), A 16x16 and B 16x8, FP32 accumulators; a0/a1: rows g / g + 8, first k pair, a2/a3: second k pair
template <bool F16>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (F16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) { return bf2_bits(__hmul2(bits_bf2(a), bits_bf2(b))); }
__device__ __forceinline__ __half2 bits_h2(uint32_t v) { return *reinterpret_cast<__half2*>(&v); }
__device__ __forceinline__ uint32_t h2_bits(__half2 v) { return *reinterpret_cast<uint32_t*>(&v); }
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) { return h2_bits(__hmul2(bits_h2(a), bits_h2(b))); }

// Eight E2M1 codes -> four FP16 pairs (2i, 2i + 1)
__device__ __forceinline__ void e2m1_f16(uint32_t q, uint32_t (&w)[4]) {
  asm("{\n.reg .b8 a, b, c, d;\nmov.b32 {a, b, c, d}, %4;\n"
      "cvt.rn.f16x2.e2m1x2 %0, a;\ncvt.rn.f16x2.e2m1x2 %1, b;\ncvt.rn.f16x2.e2m1x2 %2, c;\ncvt.rn.f16x2.e2m1x2 %3, d;\n}"
      : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
      : "r"(q));
}
// Two E4M3 codes -> FP16 pair
__device__ __forceinline__ uint32_t e4m3_f16(uint32_t two) {
  uint32_t r;
  asm("{\n.reg .b16 h;\ncvt.u16.u32 h, %1;\ncvt.rn.f16x2.e4m3x2 %0, h;\n}" : "=r"(r) : "r"(two));
  return r;
}

// Eight E2M1 codes -> four BF16 pairs (i, i + 4), each the code's value times 2^-126.
__device__ __forceinline__ void e2m1_bf16(uint32_t q, uint32_t (&w)[4]) {
  const uint32_t h = q >> 8;
  w[0] = ((q & 0x000F000Fu) * 0x1040u) & 0x81C081C0u;
  w[1] = ((q & 0x00F000F0u) * 0x0104u) & 0x81C081C0u;
  w[2] = ((h & 0x000F000Fu) * 0x1040u) & 0x81C081C0u;
  w[3] = ((h & 0x00F000F0u) * 0x0104u) & 0x81C081C0u;
}

// Packed 6-bit scales (first two words) and offsets (last two) of a Q4_K super-block, a byte per sub-block.
__device__ __forceinline__ void q4k_unpack(const uint32_t (&m)[4], uint32_t (&v)[4]) {
  v[0] = m[1] & 0x3F3F3F3Fu;
  v[1] = (m[3] & 0x0F0F0F0Fu) | ((m[1] >> 2) & 0x30303030u);
  v[2] = m[2] & 0x3F3F3F3Fu;
  v[3] = ((m[3] >> 4) & 0x0F0F0F0Fu) | ((m[2] >> 2) & 0x30303030u);
}

// Eight elements of X, by an ordinary load. This grid may be placed while the product that writes X still runs (launch_after_previous), and
// the read-only path (__ldg) asks for memory that nobody writes as long as the grid lives.
__device__ __forceinline__ uint4 load_x(const uint4* x) {
  uint4 v;
  asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(x));
  return v;
}

constexpr int kStep = 256;                            // weights of a row that a warp takes at a time
constexpr int kWords = 8;                             // words of codes (FP4) or sub-blocks (Q4_K) that a lane holds of a row

// What a lane holds of one weight row for one step of the contraction: 32 bytes of codes. FP4: 64 consecutive weights. Q4_K: 8
// bytes of each of the four chunks of a super-block.
template <int FMT>
struct RowPart {
  uint32_t q[8];
  uint32_t s[FMT == QF_FMT_Q4_K ? 4 : 1];            // block scales as stored
};

template <int FMT>
constexpr int kBlock = FMT == QF_FMT_MXFP4 ? 32 : 16;                   // weights per block scale (Q4_K: per byte of metadata)

// The same straight from global memory, piece by piece; zeros (with a scale in range) past the end of the contraction.
template <int FMT>
__device__ __forceinline__ void load_part(RowPart<FMT>& r, const uint8_t* codes, const uint8_t* scales, int k_step, int K, int t) {
  const int k = FMT == QF_FMT_Q4_K ? k_step + t * 16 : k_step + t * 64;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint2 v = make_uint2(0u, 0u);
    if (FMT == QF_FMT_Q4_K || k + 16 * i < K) v = __ldg(reinterpret_cast<const uint2*>(codes + k / 2 + i * (FMT == QF_FMT_Q4_K ? 32 : 8)));
    r.q[2 * i] = v.x;
    r.q[2 * i + 1] = v.y;
  }
  if constexpr (FMT == QF_FMT_Q4_K) {
    const uint4 m = __ldg(reinterpret_cast<const uint4*>(scales + k_step / 16));
    r.s[0] = m.x; r.s[1] = m.y; r.s[2] = m.z; r.s[3] = m.w;
  } else {
    r.s[0] = 0u;
#pragma unroll
    for (int i = 0; i < 64 / kBlock<FMT>; ++i)
      r.s[0] |= (k + i * kBlock<FMT> < K ? static_cast<uint32_t>(__ldg(scales + k / kBlock<FMT> + i)) : FMT == QF_FMT_MXFP4 ? 127u : 0u) << (8 * i);
  }
}

// ---- a warp's ring of steps in shared memory, filled by asynchronous copies -----------------------------------------------
// The codes of 16 rows, 128 bytes each, in pieces of 16 bytes that eight lanes copy for a row at a time. (Four lanes a row, 64 bytes
// of eight rows at a time, took 81 us for the copies of a 128256 x 4096 weight where this takes 49.) Pieces are permuted
// inside a row so that the lanes that read together meet different banks. Then the scales of every row.
// LOOSE: rows that do not start on 16 bytes, or scales that do not start on words (K not a multiple of 128): pieces of 8 bytes,
// 16 lanes a row, and for the scales the aligned words around them (NVFP4, one token, 32768 x 4112: 31 us, where 4096 takes 21; with lanes that copied their own 8 bytes of two rows it was 49).

template <int FMT, bool LOOSE>
constexpr int kStepScales = LOOSE ? (FMT == QF_FMT_MXFP4 ? 16 : 24) : FMT == QF_FMT_MXFP4 ? 8 : 16;       // bytes a row
template <int FMT, bool LOOSE>
constexpr int kStepBytes = 16 * (128 + kStepScales<FMT, LOOSE>);

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src) {
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
// four bytes, of which the first `bytes` exist; zeros for the others
__device__ __forceinline__ void copy_word(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// place of 16-byte piece `piece` of row r: FP4 lanes read pieces 2t (then 2t + 1) of two rows together, Q4_K lanes halves of
// pieces 2c and 2c + 1 of four rows
template <int FMT>
__device__ __forceinline__ uint32_t piece_at(int r, int piece) {
  return r * 128 + ((piece ^ (FMT == QF_FMT_Q4_K ? (r & 3) * 2 : r & 1)) * 16);
}

// Where a warp's next step of codes and scales lies. The addresses advance from turn to turn; they are set up anew for every tile.
// A lane whose piece lies past the end of the contraction copies an earlier one of its row: any finite weight will do, X is
// zero there.
template <int FMT, bool LOOSE>
struct Source {
  static constexpr int SHIFT = FMT == QF_FMT_MXFP4 ? 4 : 3;            // bytes of codes to bytes of scales
  const uint8_t* codes;                              // this lane's piece in the first row it copies
  const uint8_t* scales;
  int k;                                             // of the step
  int more;                                          // LOOSE: rows of the weight after that first one
  uint32_t row[3];                                   // otherwise: bytes of codes to the other rows

  __device__ __forceinline__ void tile(const MvParams& p, int64_t row0, int n0, int k_step, int lane) {
    const int first = n0 + (LOOSE ? lane >> 4 : lane >> 3), n = min(first, p.N - 1);
    const uint32_t pitch = static_cast<uint32_t>(p.K) / 2;
    k = k_step;
    more = p.N - 1 - n;
    if constexpr (!LOOSE) {
#pragma unroll
      for (int h = 1; h < 4; ++h) row[h - 1] = static_cast<uint32_t>(min(4 * h, more)) * pitch;
    }
    codes = p.codes + (row0 + n) * pitch + k / 2 + (LOOSE ? (lane & 15) * 8 : (lane & 7) * 16);
    const int row = FMT == QF_FMT_Q4_K ? lane & 15 : lane >> 1;         // Q4_K: one lane for a row's scales, otherwise two
    const int64_t at = ((row0 + min(n0 + row, p.N - 1)) * pitch + k / 2) >> SHIFT;
    if constexpr (LOOSE) scales = p.scales + (at & ~static_cast<int64_t>(3)) + (lane & 1) * (kStepScales<FMT, LOOSE> / 2);
    else scales = p.scales + at + (FMT == QF_FMT_Q4_K ? 0 : (lane & 1) * (kStepScales<FMT, LOOSE> / 2));
  }
  __device__ __forceinline__ void advance(int dk) {
    k += dk;
    codes += dk / 2;
    scales += dk / kBlock<FMT>;
  }
  // Starts the copies of the step.
  __device__ __forceinline__ void start(const MvParams& p, uint32_t stage, int lane) const {
    constexpr int ROWS = LOOSE ? 8 : 4, GAP = 16 / ROWS, PIECE = LOOSE ? 8 : 16, HALF = kStepScales<FMT, LOOSE> / 2;
    const int piece = LOOSE ? lane & 15 : lane & 7;
    const uint32_t to = stage + (LOOSE ? piece_at<FMT>(lane >> 4, piece >> 1) + (piece & 1) * 8 : piece_at<FMT>(lane >> 3, piece));
    const uint8_t *c = codes, *sc = scales;
    if (FMT != QF_FMT_Q4_K && p.K % kStep) {             // the same for all: rows of whole steps skip the comparisons
      if (k + piece * (2 * PIECE) >= p.K) c -= piece * PIECE;
      if (!LOOSE && k + 128 >= p.K && (lane & 1)) sc -= HALF;
    }
#pragma unroll
    for (int h = 0; h < ROWS; ++h) {                   // a gap keeps the bits of the row that permute pieces
      const uint32_t off = h == 0 ? 0u : LOOSE ? static_cast<uint32_t>(min(h * GAP, more)) * (static_cast<uint32_t>(p.K) / 2) : row[(h - 1) & 3];
      copy_async<PIECE>(to + h * GAP * 128, c + off);
    }
    const uint32_t to_sc = stage + 16 * 128;
    if constexpr (FMT == QF_FMT_Q4_K) {
      if (lane < 16) copy_async<16>(to_sc + lane * 16, scales);
    } else if constexpr (!LOOSE) {
      copy_async<HALF>(to_sc + lane * HALF, sc);
    } else {
      const int64_t room = p.scales_end - scales;      // the last words may lie past the end of the tensor
#pragma unroll
      for (int i = 0; i < HALF / 4; ++i) {
        const int64_t rest = room - 4 * i;
        copy_word(to_sc + lane * HALF + 4 * i, rest > 0 ? scales + 4 * i : p.scales, rest >= 4 ? 4 : rest > 0 ? static_cast<int>(rest) : 0);
      }
    }
  }
};

// A step back from the ring; skew: LOOSE, where in its first word each row's scales begin.
template <int FMT, bool LOOSE>
__device__ __forceinline__ void read_step(RowPart<FMT> (&r)[2], const uint8_t* stage, int lane, const uint32_t (&skew)[2]) {
  const int g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = g + 8 * i;
    const uint8_t* sc = stage + 16 * 128 + row * kStepScales<FMT, LOOSE>;
    if constexpr (FMT == QF_FMT_Q4_K) {
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const uint2 v = *reinterpret_cast<const uint2*>(stage + piece_at<FMT>(row, 2 * c) + t * 8);
        r[i].q[2 * c] = v.x;
        r[i].q[2 * c + 1] = v.y;
      }
      const uint4 m = *reinterpret_cast<const uint4*>(sc);
      r[i].s[0] = m.x; r[i].s[1] = m.y; r[i].s[2] = m.z; r[i].s[3] = m.w;
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint4 v = *reinterpret_cast<const uint4*>(stage + piece_at<FMT>(row, 2 * t + h));
        r[i].q[4 * h] = v.x; r[i].q[4 * h + 1] = v.y; r[i].q[4 * h + 2] = v.z; r[i].q[4 * h + 3] = v.w;
      }
      if constexpr (!LOOSE) {
        r[i].s[0] = FMT == QF_FMT_NVFP4 ? reinterpret_cast<const uint32_t*>(sc)[t] : reinterpret_cast<const uint16_t*>(sc)[t];
      } else if constexpr (FMT == QF_FMT_NVFP4) {
        const uint8_t* b = sc + skew[i] + t * 4;
        r[i].s[0] = b[0] | b[1] << 8 | b[2] << 16 | static_cast<uint32_t>(b[3]) << 24;
      } else {
        const uint8_t* b = sc + skew[i] + t * 2;
        r[i].s[0] = b[0] | b[1] << 8;
      }
    }
  }
}

// The packed BF16 factor that turns value * 2^-126 into value * scale (NVFP4: times 2^-7, put right at the end).
template <int FMT>
__device__ __forceinline__ uint32_t bf16_factor(uint32_t code) {
  if constexpr (FMT == QF_FMT_NVFP4) {
    // code << 20 is the scale times 2^-120 as FP32
    const uint32_t f = __float_as_uint(__fmul_rn(__fmul_rn(__uint_as_float(code << 20), 0x1p127f), 0x1p112f));
    return __byte_perm(f, f, 0x3232);
  } else {
    return min(code + 126u, 254u) * 0x00800080u;       // 2^(p + 126), p = code - 127; above p = 1 the rest follows separately
  }
}

// MXFP4 scale codes for which value * 2^p, kept as value * 2^(p + 7), is exact in FP16: p in [-21, 5]
constexpr uint32_t kMxLow = 106, kMxHigh = 132;

// whether that holds for all scales of the warp's step
__device__ __forceinline__ bool mx_exact(const RowPart<QF_FMT_MXFP4> (&r)[2]) {
  constexpr int NS = 2;
  bool in = true;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < NS; ++j) in = in && ((r[i].s[0] >> (8 * j)) & 0xFFu) - kMxLow <= kMxHigh - kMxLow;
  return __all_sync(0xFFFFFFFFu, in);
}

// ---- one step of the contraction, FP16 fragments from shared memory: c[nt] += A . B ------------------------------------
// x: the step's X in shared memory, `at` this lane's place in each token tile. Returns false if a scale is out of range (c is then
// worthless). c is the sum times 2^6 (from X) and times 1 (NVFP4), 2^7 (MXFP4) or 2^-24 / d (Q4_K).

// Bytes between consecutive words of X where several token tiles stand word by word (16 of padding, so that the threads that
// stage consecutive words meet different banks).
template <int NT>
constexpr int kXPitch = 8 * NT * 64 + 16;

// This lane's 16 bytes of X for one word of codes (Q4_K: one sub-block). A single token tile stands lane by lane, 16 bytes of
// padding after each lane's words, so that a lane's words have fixed distances; lanes without a token read nothing (columns of
// the product do not meet, whatever is in their registers). Several tiles stand word by word.
template <int NT>
__device__ __forceinline__ uint4 x_word(uint32_t x, int w, uint32_t at, bool live) {
  uint4 v;
  if constexpr (NT == 1)
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %5, 0;\n@p ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n}"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "r"(x + at + w * 16), "r"(static_cast<int>(live)));
  else
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(x + at + w * kXPitch<NT>));
  return v;
}

template <int FMT, int NT>
__device__ __forceinline__ bool step_f16(const RowPart<FMT> (&r)[2], uint32_t x, const uint32_t (&at)[NT], bool live, float (&c)[NT][4]) {
  bool in = true;
  if constexpr (FMT == QF_FMT_Q4_K) {
    uint32_t v[2][4];
#pragma unroll
    for (int i = 0; i < 2; ++i) q4k_unpack(r[i].s, v[i]);
#pragma unroll
    for (int chunk = 0; chunk < 4; ++chunk) {
      __half2 f[2];                               // s6 of the chunk's two sub-blocks; the odd one's codes come out 16 times as large
#pragma unroll
      for (int i = 0; i < 2; ++i)
        f[i] = __hfma2(bits_h2(__byte_perm(v[i][chunk >> 1], 0x64646464u, chunk & 1 ? 0x4342 : 0x4140)), bits_h2(0x2C003C00u), bits_h2(0xD400E400u));
#pragma unroll
      for (int odd = 0; odd < 2; ++odd) {
        uint4 xv[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) xv[nt] = x_word<NT>(x, 2 * chunk + odd, at[nt], live);
        uint32_t w[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t mask = odd ? 0x00F000F0u : 0x000F000Fu;
          const __half2 fac = odd ? __high2half2(f[i]) : __low2half2(f[i]);
          const uint32_t q0 = r[i].q[2 * chunk], q1 = r[i].q[2 * chunk + 1];
          w[i][0] = h2_bits(__hmul2(bits_h2(q0 & mask), fac));
          w[i][1] = h2_bits(__hmul2(bits_h2((q0 >> 8) & mask), fac));
          w[i][2] = h2_bits(__hmul2(bits_h2(q1 & mask), fac));
          w[i][3] = h2_bits(__hmul2(bits_h2((q1 >> 8) & mask), fac));
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          mma16816<true>(c[nt], w[0][0], w[1][0], w[0][1], w[1][1], xv[nt].x, xv[nt].y);
          mma16816<true>(c[nt], w[0][2], w[1][2], w[0][3], w[1][3], xv[nt].z, xv[nt].w);
        }
      }
    }
  } else {
    constexpr int PER = FMT == QF_FMT_NVFP4 ? 2 : 4;   // words of codes per scale
    uint32_t f[2];
    __half2 pair[2];                              // NVFP4: two scales as FP16
#pragma unroll
    for (int w = 0; w < kWords; ++w) {
      if (w % PER == 0) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if constexpr (FMT == QF_FMT_NVFP4) {
            if (w % 4 == 0) pair[i] = bits_h2(e4m3_f16((w ? r[i].s[0] >> 16 : r[i].s[0]) & 0xFFFFu));
            f[i] = h2_bits(w % 4 ? __high2half2(pair[i]) : __low2half2(pair[i]));
          } else {
            const uint32_t u = ((r[i].s[0] >> (8 * (w / PER))) & 0xFFu) - kMxLow;
            in = in && u <= kMxHigh - kMxLow;
            f[i] = u * 0x04000400u + 0x04000400u;      // 2^(p + 7): exponent field p + 22 = code - 105
          }
        }
      }
      uint4 xv[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) xv[nt] = x_word<NT>(x, w, at[nt], live);
      uint32_t wa[4], wb[4];
      e2m1_f16(r[0].q[w], wa);
      e2m1_f16(r[1].q[w], wb);
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        wa[h] = mul_f16x2(wa[h], f[0]);
        wb[h] = mul_f16x2(wb[h], f[1]);
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        mma16816<true>(c[nt], wa[0], wb[0], wa[1], wb[1], xv[nt].x, xv[nt].y);
        mma16816<true>(c[nt], wa[2], wb[2], wa[3], wb[3], xv[nt].z, xv[nt].w);
      }
    }
  }
  return in;
}

// ---- the same step with BF16 fragments for the tokens in `bad` (all of them if a scale of the tile is out of the FP16 range),
// weights and X read again from global memory: their sums in the final units (NVFP4: without the tensor scale), zero for the
// other tokens. Out of line, so that it costs the fast path no registers.

template <int NT>
struct Sums { float c[NT][4]; };

template <int FMT, int NT>
__device__ __noinline__ Sums<NT> step_bf16(const MvParams& p, const uint16_t* list, int w0, int c0, int mt, int64_t row0, int n0, int k_step, uint32_t bad) {
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int64_t scale_pitch = FMT == QF_FMT_Q4_K ? p.K / 16 : p.K / (FMT == QF_FMT_NVFP4 ? 16 : 32);
  Sums<NT> sum = {};
  RowPart<FMT> r[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int64_t row = row0 + min(n0 + g + 8 * i, p.N - 1);
    load_part<FMT>(r[i], p.codes + row * (p.K / 2), p.scales + row * scale_pitch, k_step, p.K, t);
  }
  if constexpr (FMT == QF_FMT_MXFP4)
    if (!mx_exact(r)) bad = 0xFFFFFFFFu;
  if (bad == 0u) return sum;
  const __nv_bfloat16* xrow[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int m = c0 + min(nt * 8 + g, mt - 1);
    xrow[nt] = p.X + static_cast<int64_t>((w0 + (p.ids ? list[m] : m)) / p.x_div) * p.K;
  }
  if constexpr (FMT == QF_FMT_Q4_K) {
#pragma unroll
    for (int blk = 0; blk < 8; ++blk) {
      const int k = k_step + blk * 32 + t * 8;
      uint32_t w[2][4];
      float es[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const RowPart<FMT>& part = r[i];
        uint32_t v[4];
        q4k_unpack(part.s, v);
#pragma unroll
        for (int h = 0; h < 4; ++h) {                // 128 + C as BF16, minus 128: elements (0, 2), (1, 3), (4, 6), (5, 7)
          const uint32_t n = (part.q[blk / 2 * 2 + h / 2] >> (4 * (blk & 1) + 8 * (h & 1))) & 0x000F000Fu;
          w[i][h] = bf2_bits(__hsub2(bits_bf2(n | 0x43004300u), bits_bf2(0x43004300u)));
        }
        const float d = __half2float(__ushort_as_half(static_cast<unsigned short>(part.s[0] & 0xFFFFu)));
        es[i] = d * static_cast<float>((v[blk / 4] >> (8 * (blk & 3))) & 63u);
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const uint4 x = load_x(reinterpret_cast<const uint4*>(xrow[nt] + k));
        float c[4] = {};
        mma16816<false>(c, w[0][0], w[1][0], w[0][1], w[1][1], __byte_perm(x.x, x.y, 0x5410), __byte_perm(x.x, x.y, 0x7632));
        mma16816<false>(c, w[0][2], w[1][2], w[0][3], w[1][3], __byte_perm(x.z, x.w, 0x5410), __byte_perm(x.z, x.w, 0x7632));
#pragma unroll
        for (int j = 0; j < 4; ++j) sum.c[nt][j] = fmaf(es[j >> 1], c[j], sum.c[nt][j]);
      }
    }
  } else {
    constexpr int PER = FMT == QF_FMT_NVFP4 ? 2 : 4;
#pragma unroll
    for (int word = 0; word < kWords; ++word) {
      const int k = k_step + t * 64 + word * 8;
      uint32_t w[2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t code = (r[i].s[0] >> (8 * (word / PER))) & 0xFFu, f = bf16_factor<FMT>(code);
        e2m1_bf16(r[i].q[word], w[i]);
        const uint32_t rest = FMT == QF_FMT_MXFP4 ? (max(code, 128u) - 1u) * 0x00800080u : 0x3F803F80u;
#pragma unroll
        for (int h = 0; h < 4; ++h) w[i][h] = mul_bf16x2(mul_bf16x2(w[i][h], f), rest);
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        uint4 x = make_uint4(0u, 0u, 0u, 0u);
        if (k < p.K) x = load_x(reinterpret_cast<const uint4*>(xrow[nt] + k));
        mma16816<false>(sum.c[nt], w[0][0], w[1][0], w[0][1], w[1][1], __byte_perm(x.x, x.z, 0x5410), __byte_perm(x.x, x.z, 0x7632));
        mma16816<false>(sum.c[nt], w[0][2], w[1][2], w[0][3], w[1][3], __byte_perm(x.y, x.w, 0x5410), __byte_perm(x.y, x.w, 0x7632));
      }
    }
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      sum.c[nt][j] = (bad >> (nt * 8 + 2 * t + (j & 1))) & 1u ? sum.c[nt][j] * (FMT == QF_FMT_NVFP4 ? 0x1p7f : 1.0f) : 0.0f;
  return sum;
}

// Stages 8 elements: FP16 of 2^6 x. False if that is not exact for one of them (or it is a NaN).
__device__ __forceinline__ bool stage_f16(const uint4& v, uint32_t (&h)[4]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  bool exact = true;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float lo = bf16_lo(w[i]) * kXScale, hi = bf16_hi(w[i]) * kXScale;
    const __half2 r = __floats2half2_rn(lo, hi);
    const float2 back = __half22float2(r);
    exact = exact && back.x == lo && back.y == hi;
    h[i] = h2_bits(r);
  }
  return exact;
}

// One step with FP16 fragments into acc; the tokens in `bad` are left out. Returns bad, or all ones if a scale of the tile is out of
// the FP16 range.
template <int FMT, int NT>
__device__ __forceinline__ uint32_t add_step(const RowPart<FMT> (&r)[2], uint32_t x, uint32_t sx, const uint32_t (&at)[NT], const uint32_t (&sx_at)[NT],
                                             bool live, int t, uint32_t bad, float (&acc)[NT][4]) {
  float c[NT][4] = {};
  const bool in = step_f16<FMT, NT>(r, x, at, live, c);
  if constexpr (FMT == QF_FMT_MXFP4)
    if (!__all_sync(0xFFFFFFFFu, in)) bad = 0xFFFFFFFFu;
  if (__builtin_expect(bad != 0u, 0)) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 4; ++j) c[nt][j] = (bad >> (nt * 8 + 2 * t + (j & 1))) & 1u ? 0.0f : c[nt][j];
  }
  float f[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    f[i] = FMT == QF_FMT_NVFP4 ? 1.0f / kXScale : 1.0f / (kXScale * 128.0f);
    if constexpr (FMT == QF_FMT_Q4_K) f[i] = __half2float(__ushort_as_half(static_cast<unsigned short>(r[i].s[0] & 0xFFFFu))) * (0x1p24f / kXScale);
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[nt][j] = fmaf(f[j >> 1], c[nt][j], acc[nt][j]);
  if constexpr (FMT == QF_FMT_Q4_K) {
    // offsets: m6 [16 rows x 8 sub-blocks] times the three parts of the sums of X
    uint32_t m6[2];
    float dmin[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t v[4];
      q4k_unpack(r[i].s, v);
      m6[i] = bf2_bits(__hsub2(bits_bf2(__byte_perm(t & 2 ? v[3] : v[2], 0x43434343u, 0x4140u + (t & 1) * 0x0202u)), bits_bf2(0x43004300u)));
      dmin[i] = __half2float(__ushort_as_half(static_cast<unsigned short>(r[i].s[0] >> 16)));
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      uint4 b;
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "r"(sx + sx_at[nt]));
      float m[4] = {};
      mma16816<false>(m, m6[0], m6[1], m6[0], m6[1], b.x, b.y);
      mma16816<false>(m, m6[0], m6[1], 0u, 0u, b.z, 0u);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[nt][j] = fmaf(-dmin[j >> 1], m[j], acc[nt][j]);
    }
  }
  return bad;
}

template <int FMT, int NT, bool LOOSE>
__global__ void __launch_bounds__(32 * kWarpsMost, 1) matvec_kernel(const __grid_constant__ MvParams p) {
  constexpr int MT = 8 * NT;                           // tokens of a pass
  constexpr bool Q4K = FMT == QF_FMT_Q4_K;
  // The next copies into a step's place start as soon as it is in registers for FP4 and one token tile (128256 x 4096, 8 tokens: 65 us,
  // 74 when they start after the products), after the products otherwise (two tiles 82 us against 96, Q4_K with one token 70 against 72)
  constexpr bool EARLY = NT == 1 && !Q4K;
  constexpr int XL = kWords * 16 + 16;                     // a lane's bytes of X for a step (a single token tile)
  extern __shared__ __align__(16) uint8_t smem[];                                  // X: [kc / kStep][tokens][4 lanes][XL], or [kc / kStep][kWords][MT][4 lanes][16] and padding
  uint4* sx = reinterpret_cast<uint4*>(smem + p.sx_at);                            // Q4_K: [kc / 256][MT][4]: sums over two sub-blocks in three BF16 parts
  uint32_t* inexact = reinterpret_cast<uint32_t*>(smem + p.flags_at);              // [kc / kStep]: tokens whose X is not exact as staged
  uint16_t* list = reinterpret_cast<uint16_t*>(smem + p.list_at);                  // grouped: rows of Y served, from w0
  float* red = reinterpret_cast<float*>(smem + p.red_at);                          // split contraction: [kw][MT][rows of the CTA + 4]
  __shared__ int warp_count[kWarpsMost];
  const int tid = threadIdx.x, threads = blockDim.x, lane = tid & 31, warp = tid >> 5, warps = threads >> 5, g = lane >> 2, t = lane & 3;
  constexpr int SB = kStepBytes<FMT, LOOSE>;
  const int ring = p.ring_at + warp * kStages<NT> * SB, ring_end = ring + kStages<NT> * SB;     // in bytes from the start
  const uint32_t smem0 = smem_addr(smem);
  const int rows_cta = warps / p.kw * 16, red_pitch = rows_cta + 4;
  const int rw = warp / p.kw, kw = warp - rw * p.kw;
  const int z = blockIdx.z, nz = gridDim.z;
  const int k_begin = z * p.kz, k_end = min(p.K, k_begin + p.kz);
  const bool whole = p.kc >= p.kz;                     // the slice of X is staged once for all row blocks
  const bool split = p.kw > 1 || nz > 1;
  // split contraction: the row of a tile and the tokens out_m, out_m + out_step, ... that this thread finishes (rows_cta is a power of
  // two and at most the number of threads)
  const int out_n = (tid + z * threads) & (rows_cta - 1), out_m = (tid + z * threads) >> (31 - __clz(rows_cta)), out_step = threads * nz >> (31 - __clz(rows_cta));

  launch_after_previous();
  int e = 0;
  if (p.ids) {
    if (p.by_pair) {
      // slot = pair: the first pair that names an expert takes all pairs that do
      e = expert_id(p, blockIdx.y);
      bool seen = false;
      for (int i = tid; i < static_cast<int>(blockIdx.y); i += threads) seen |= expert_id(p, i) == e;
      if (__syncthreads_or(seen) && e >= 0) return;
      if (e < 0) {
        if (z == 0)
          for (int n = blockIdx.x * threads + tid; n < p.N; n += gridDim.x * threads) store_y(p, blockIdx.y, n, 0.0f);
        return;
      }
    } else {
      e = blockIdx.y;
    }
  }
  const float unit = FMT == QF_FMT_NVFP4 ? p.tscale[e] : 1.0f;
  const int64_t row0 = static_cast<int64_t>(e) * p.N;

  for (int w0 = 0; w0 < p.M; w0 += kListCap) {
    // the rows of Y that this CTA's weight serves
    const int w1 = min(p.M, w0 + kListCap);
    int count = w1 - w0;
    if (p.ids) {
      count = 0;
      for (int i0 = w0; i0 < w1; i0 += threads) {
        const int i = i0 + tid;
        const int id = i < w1 ? expert_id(p, i) : -2;
        const bool mine = id == e;
        if (!p.by_pair && e == 0 && id == -1 && z == 0)
          for (int n = blockIdx.x; n < p.N; n += gridDim.x) store_y(p, i, n, 0.0f);
        const uint32_t vote = __ballot_sync(0xFFFFFFFFu, mine);
        __syncthreads();
        if (lane == 0) warp_count[warp] = __popc(vote);
        __syncthreads();
        int to = count + __popc(vote & ((1u << lane) - 1u));
        for (int w = 0; w < warps; ++w) {
          if (w < warp) to += warp_count[w];
          count += warp_count[w];
        }
        if (mine) list[to] = static_cast<uint16_t>(i - w0);
      }
      __syncthreads();
    }
    for (int c0 = 0; c0 < count; c0 += MT) {
      const int mt = min(MT, count - c0);
      // columns of the product do not meet: a lane whose token does not exist reads the last one's X instead
      const bool live = g < mt;
      uint32_t at[NT], sx_at[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int m = min(nt * 8 + g, mt - 1);
        at[nt] = NT == 1 ? (m * 4 + t) * XL : (m * 4 + t) * 16;
        sx_at[nt] = (m * 4 + t) * 16;
      }
      const uint32_t x_step = NT == 1 ? mt * 4 * XL : kWords * kXPitch<NT>;      // bytes of X of a step
      float acc[NT][4] = {};

      for (int b0 = blockIdx.x; b0 < p.blocks; b0 += whole ? p.blocks : gridDim.x) {
        for (int kc0 = k_begin; kc0 < k_end; kc0 += p.kc) {
          const int kc1 = min(kc0 + p.kc, k_end), steps = (kc1 - kc0 + kStep - 1) / kStep;
          const int per_tile = kw < steps ? (steps - kw + p.kw - 1) / p.kw : 0;      // steps of this warp in a tile
          const int tiles = whole ? (p.blocks - b0 + gridDim.x - 1) / gridDim.x : 1;
          // the first codes are under way while X is staged
          int next_n = b0 * rows_cta + rw * 16, next = 0, tiles_left = per_tile ? tiles : 0;
          Source<FMT, LOOSE> src;
          if (tiles_left) src.tile(p, row0, next_n, kc0 + kw * kStep, lane);
          auto start = [&](int stage) {
            if (tiles_left > 0) {
              src.start(p, smem0 + stage, lane);
              if (++next < per_tile) {
                src.advance(p.kw * kStep);
              } else if (--tiles_left > 0) {
                next = 0;
                next_n += gridDim.x * rows_cta;
                src.tile(p, row0, next_n, kc0 + kw * kStep, lane);
              }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
          };
#pragma unroll 1
          for (int d = 0; d < kStages<NT>; ++d) start(ring + d * SB);
          for (int i = tid; i < steps; i += threads) inexact[i] = 0u;
          __syncthreads();
          bool exact = true;
          // X slice: as many warps for a token as there are to spare; a warp loads 32 units of 8 elements, kBatch times over before
          // it waits
          constexpr int kBatch = 8;
          const int units = steps * (kStep / 8), groups = (units + 31) / 32;
          int share = warps;                             // warps of a token
          while (share > 1 && share * mt > warps) share >>= 1;
          for (int m = warp / share; m < mt; m += warps / share) {
            const int row = w0 + (p.ids ? list[c0 + m] : c0 + m);
            const uint4* x = reinterpret_cast<const uint4*>(p.X + static_cast<int64_t>(row / p.x_div) * p.K + kc0);
            for (int g0 = warp & (share - 1); g0 < groups; g0 += share * kBatch) {
              uint4 q[kBatch];
#pragma unroll
              for (int i = 0; i < kBatch; ++i) {
                const int v = (g0 + i * share) * 32 + lane, s = v / (kStep / 8), w = v / 4 % kWords;       // step, word of codes, and lane v % 4
                const int unit = Q4K ? v : s * (kStep / 8) + (v & 3) * kWords + w;
                q[i] = make_uint4(0u, 0u, 0u, 0u);
                if (v < units && kc0 + 8 * unit < p.K) q[i] = load_x(x + unit);
              }
#pragma unroll
              for (int i = 0; i < kBatch; ++i) {
                const int v = (g0 + i * share) * 32 + lane, s = v / (kStep / 8), w = v / 4 % kWords;
                if (v >= units) continue;                // for Q4_K a whole warp or none of it
                uint32_t h[4];
                if (!stage_f16(q[i], h)) {
                  exact = false;
                  atomicOr(inexact + s, 1u << m);
                }
                uint4* to = reinterpret_cast<uint4*>(smem + s * x_step + (NT == 1 ? (m * 4 + (v & 3)) * XL + w * 16 : w * kXPitch<NT> + m * 64 + (v & 3) * 16));
                if constexpr (Q4K) {                     // elements (0, 2), (1, 3), (4, 6), (5, 7): the order of the decoded words
                  *to = make_uint4(__byte_perm(h[0], h[1], 0x5410), __byte_perm(h[0], h[1], 0x7632), __byte_perm(h[2], h[3], 0x5410), __byte_perm(h[2], h[3], 0x7632));
                  float sum = bf16_lo(q[i].x) + bf16_hi(q[i].x) + bf16_lo(q[i].y) + bf16_hi(q[i].y) +
                              (bf16_lo(q[i].z) + bf16_hi(q[i].z) + bf16_lo(q[i].w) + bf16_hi(q[i].w));
                  sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 1);
                  sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 2);
                  if ((v & 3) < 3) {
                    const __nv_bfloat16 p1 = __float2bfloat16_rn(sum), p2 = __float2bfloat16_rn(sum - __bfloat162float(p1));
                    const __nv_bfloat16 p3 = __float2bfloat16_rn(sum - __bfloat162float(p1) - __bfloat162float(p2));
                    reinterpret_cast<__nv_bfloat16*>(sx + (s * MT + m) * 4 + w / 2)[2 * (v & 3) + (w & 1)] = (v & 3) == 0 ? p1 : (v & 3) == 1 ? p2 : p3;
                  }
                } else {
                  *to = make_uint4(h[0], h[1], h[2], h[3]);
                }
              }
            }
          }
          const bool any_inexact = __syncthreads_or(!exact);

          int stage = ring;
#pragma unroll 1
          for (int tile = 0; tile < tiles; ++tile) {
            const int block = b0 + tile * gridDim.x;
            uint32_t any_bad = 0u;
            uint32_t skew[2] = {0u, 0u};
            if constexpr (LOOSE) {
#pragma unroll
              for (int i = 0; i < 2; ++i)
                skew[i] = (static_cast<uint32_t>(row0) + min(block * rows_cta + rw * 16 + g + 8 * i, p.N - 1)) * static_cast<uint32_t>(p.K / kBlock<FMT>) & 3u;
            }
            int s = kw;
#pragma unroll 1
            for (int j = 0; j < per_tile; ++j) {
              // the oldest step's copies are complete
              asm volatile("cp.async.wait_group %0;" ::"n"(kStages<NT> - 1) : "memory");
              __syncwarp();
              RowPart<FMT> r[2];
              read_step<FMT, LOOSE>(r, smem + stage, lane, skew);
              if constexpr (FMT == QF_FMT_MXFP4 && LOOSE) {
                // what stands past the end of the row is no scale of it: one in range instead
                const int left = p.K - (kc0 + s * kStep + t * 64);
                if (left < 64) {
#pragma unroll
                  for (int i = 0; i < 2; ++i) r[i].s[0] = left <= 0 ? 0x7F7Fu : (r[i].s[0] & 0xFFu) | (left <= 32 ? 0x7F00u : r[i].s[0] & 0xFF00u);
                }
              }
              if constexpr (EARLY) {
                __syncwarp();
                start(stage);
                stage = stage + SB == ring_end ? ring : stage + SB;
              }
              uint32_t bad = 0u;
              if (any_inexact) bad = inexact[s];
              any_bad |= add_step<FMT, NT>(r, smem0 + s * x_step, smem0 + p.sx_at + s * MT * 64, at, sx_at, live, t, bad, acc);
              if constexpr (!EARLY) {
                __syncwarp();
                start(stage);
                stage = stage + SB == ring_end ? ring : stage + SB;
              }
              s += p.kw;
            }
            // end of the tile; a warp without a step in a split contraction meets the others here all the same
            const int n_cta = block * rows_cta, n_warp = n_cta + rw * 16;
            if (any_bad) {
              for (int s = 0; s < steps; ++s) {
                if (s % p.kw != kw) continue;
                const Sums<NT> sum = step_bf16<FMT, NT>(p, list, w0, c0, mt, row0, n_warp, kc0 + s * kStep, inexact[s]);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                  for (int j = 0; j < 4; ++j) acc[nt][j] += sum.c[nt][j];
              }
            }
            if (kc1 == k_end) {
              if (!split) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                  for (int j = 0; j < 4; ++j) {
                    const int n = n_warp + g + (j >> 1) * 8, m = nt * 8 + 2 * t + (j & 1);
                    if (n < p.N && m < mt) store_y(p, w0 + (p.ids ? list[c0 + m] : c0 + m), n, acc[nt][j] * unit);
                  }
              } else {
                float* mine = red + kw * MT * red_pitch + rw * 16 + g;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                  for (int j = 0; j < 4; ++j) mine[(nt * 8 + 2 * t + (j & 1)) * red_pitch + (j >> 1) * 8] = acc[nt][j];
                if (nz > 1) cg::this_cluster().sync();
                else __syncthreads();
                // the CTAs of the cluster share the outputs
                if (n_cta + out_n < p.N) {
                  for (int m = out_m; m < mt; m += out_step) {
                    const int at_m = m * red_pitch + out_n;
                    float sum = 0.0f;
                    if (nz == 1) {
#pragma unroll 2
                      for (int k = 0; k < p.kw; ++k) sum += red[at_m + k * MT * red_pitch];
                    } else {
                      for (int zz = 0; zz < nz; ++zz) {
                        const float* part = cg::this_cluster().map_shared_rank(red, zz) + at_m;
#pragma unroll 2
                        for (int k = 0; k < p.kw; ++k) sum += part[k * MT * red_pitch];
                      }
                    }
                    store_y(p, w0 + (p.ids ? list[c0 + m] : c0 + m), n_cta + out_n, sum * unit);
                  }
                }
                if (nz > 1) cg::this_cluster().sync();
                else __syncthreads();
              }
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[nt][j] = 0.0f;
            }
          }
          __syncthreads();                               // the slice is read; its memory is free
        }
      }
    }
  }
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// How a product is cut: warps of a CTA, warps that share a tile, CTAs of a cluster that share the contraction, row blocks.
struct Cut {
  int warps, kw, nz;
  int64_t kz, kc, blocks, grid_x;
  size_t smem;
};

// Picks the cut with the least estimated time. The constants are microseconds measured on this part: a step takes step_fixed and
// step_each per warp that the SM holds, 0.5 at least; meeting costs 0.5 in a CTA and 2 in a cluster (3.5 if there are tiles to
// come, since it empties the rings); a slice of X takes 0.7 and 1 per 30 KB that the SM stages. Over 58 products from
// 1024 x 4096 to 128256 x 4096 with 1 to 24 tokens the choice took 1.02 times as long as the best cut in the mean, 1.22 at most (128
// experts of 2048 x 768, one token: 8.3 us, 6.8 with twice the CTAs of two warps a tile). Outside them it can be far off: 128 experts of
// 1536 x 2048 with one token take 15.3 us (NVFP4) and 16.5 (Q4_K) with 16 warps, 8 a tile, where MXFP4 takes 8.3 with 4 and 2.
Cut choose_cut(int64_t N, int64_t K, double slots, double tokens, int mt, int nt, int ring_bytes, int x_bytes, bool q4k, bool loose, bool grouped, MvParams& p) {
  Cut best{};
  double best_time = 1e30;
  const double step_fixed = q4k ? 0.28 : 0.13, step_each = nt == 1 ? 0.055 + 0.0008 * tokens : 0.075;
  const int64_t steps = ceil_div(K, kStep);
  // the small copies of loose rows go through L1, which has to be left some room (32768 x 4128, 8 tokens: 52 us at 230 KB, 34 at 160)
  const size_t smem_most = loose ? 200 * 1024 : kSmemMost;
  for (int warps = 4; warps <= kWarpsMost; warps *= 2)
    for (int kw = 1; kw <= warps; kw *= 2)
      for (int nz = 1; nz <= 4; nz *= 2) {
        if ((kw > 1 || nz > 1) && kw * nz > steps) continue;
        Cut c{};
        c.warps = warps; c.kw = kw;
        c.kz = ceil_div(steps, nz) * kStep;
        c.nz = static_cast<int>(ceil_div(K, c.kz));
        if (c.nz != nz) continue;
        const int rows_cta = warps / kw * 16;
        c.blocks = ceil_div(N, rows_cta);
        const size_t ring = static_cast<size_t>(warps) * ring_bytes;
        const size_t red = kw > 1 || nz > 1 ? static_cast<size_t>(kw) * 8 * nt * (rows_cta + 4) * 4 : 0;
        const size_t fixed = ring + red + (grouped ? kListCap * 2 : 0) + 64;
        const int64_t per_k = x_bytes + 4 + (q4k ? 8 * nt * 64 : 0);                            // bytes per step of the contraction
        if (fixed + per_k > smem_most) continue;
        const int64_t most = (smem_most - fixed) / per_k * kStep;
        c.kc = c.kz < most ? c.kz : most;
        c.smem = fixed + c.kc / kStep * per_k;
        int per_sm = kWarpsMost / warps;
        if (per_sm > static_cast<int>(kSmemMost / (c.smem + 1024))) per_sm = static_cast<int>(kSmemMost / (c.smem + 1024));
        if (per_sm < 1) per_sm = 1;
        const int64_t room = static_cast<int64_t>(nz == 4 ? 33 : kNumSMs / nz) * per_sm;        // clusters that run at a time
        int64_t gx = static_cast<int64_t>(room / slots);
        if (gx < 1) gx = 1;
        if (gx > c.blocks) gx = c.blocks;
        c.grid_x = gx;
        const int64_t grid = static_cast<int64_t>(gx * slots + 0.5), waves = ceil_div(grid, room);
        const int64_t sm_ctas = ceil_div(grid * nz, kNumSMs), resident = sm_ctas < per_sm ? sm_ctas : per_sm;
        // CTAs that share an SM even out some of what they have more or less of
        const double most_tiles = static_cast<double>(ceil_div(c.blocks, gx)), tiles = resident > 1 && nz == 1 ? 0.75 * most_tiles + 0.25 * c.blocks / gx : most_tiles;
        const double stage_x = 0.7 + resident * tokens * c.kz * 2 / 3e4;
        const double step = fmax(0.5, step_fixed + step_each * resident * warps);
        const double tile = ceil_div(c.kz / kStep, kw) * step + (nz > 1 ? (most_tiles > 1 ? 3.5 : 2.0) : kw > 1 ? 0.5 : 0.05) +
                            (warps == 4 ? 0.0 : (warps == 8 && resident > 1 ? 0.09 : 0.025) * ceil_div(c.kz / kStep, kw));
        const double time = waves * ((c.kc >= c.kz ? stage_x : tiles * (stage_x + 1.5 * ceil_div(c.kz, c.kc))) + tiles * tile);
        if (time < best_time) { best_time = time; best = c; }
      }
  p.blocks = static_cast<int>(best.blocks);
  p.kw = best.kw;
  p.kz = static_cast<int>(best.kz);
  p.kc = static_cast<int>(best.kc);
  p.sx_at = static_cast<int>(best.kc / kStep * x_bytes);
  p.flags_at = p.sx_at + (q4k ? static_cast<int>(best.kc / kStep * 8 * nt * 64) : 0);
  p.list_at = static_cast<int>(ceil_div(p.flags_at + best.kc / kStep * 4, 16) * 16);
  p.red_at = p.list_at + (grouped ? kListCap * 2 : 0);
  const int rows_cta = best.warps / best.kw * 16;
  p.ring_at = static_cast<int>(ceil_div(p.red_at + (best.kw > 1 || best.nz > 1 ? best.kw * 8 * nt * (rows_cta + 4) * 4 : 0), 16) * 16);
  return best;
}

template <int FMT, int NT, bool LOOSE>
Cut cut_of(MvParams& p, int mt) {
  // experts that even routing is expected to meet; the others' CTAs leave at once
  const double busy = p.ids ? p.G * (1.0 - pow(1.0 - 1.0 / p.G, p.M)) : 1.0;
  return choose_cut(p.N, p.K, busy, p.ids ? fmin(mt, fmax(1.0, p.M / busy)) : mt, mt, NT, kStages<NT> * kStepBytes<FMT, LOOSE>, NT == 1 ? mt * 4 * 144 : 8 * kXPitch<NT>, FMT == QF_FMT_Q4_K, LOOSE, p.ids != nullptr, p);
}

template <int FMT, int NT, bool LOOSE>
cudaError_t launch(MvParams& p, int slots, int mt, cudaStream_t st) {
  const Cut c = cut_of<FMT, NT, LOOSE>(p, mt);
  auto kernel = matvec_kernel<FMT, NT, LOOSE>;
  static bool ready[64] = {};                          // per device
  int dev = 0;
  if (cudaError_t e = cudaGetDevice(&dev)) return e;
  if (dev >= 64 || !ready[dev]) {
    if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMost)) return e;
    if (dev < 64) ready[dev] = true;
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(c.grid_x), static_cast<unsigned>(slots), static_cast<unsigned>(c.nz));
  cfg.blockDim = dim3(32 * c.warps);
  cfg.dynamicSmemBytes = c.smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 1;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = c.nz;
  cfg.attrs = attr;
  cfg.numAttrs = c.nz > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

MvParams params_of(const MatvecArgs& a) {
  MvParams p{};
  p.X = static_cast<const __nv_bfloat16*>(a.X);
  p.codes = static_cast<const uint8_t*>(a.codes);
  p.scales = static_cast<const uint8_t*>(a.scales);
  p.scales_end = p.scales + (a.ids ? a.G : 1) * a.N * (a.K / (a.fmt == QF_FMT_MXFP4 ? 32 : 16));
  p.tscale = a.tscale;
  p.ids = a.ids;
  p.ids64 = a.ids64;
  p.Y = a.Y;
  p.x_div = static_cast<int>(a.x_div);
  p.M = static_cast<int>(a.M); p.N = static_cast<int>(a.N); p.K = static_cast<int>(a.K); p.G = a.G;
  p.y_f32 = a.y_dtype == QF_DT_F32;
  p.by_pair = a.ids && a.M <= a.G;
  return p;
}

// Calls go(format, token tiles, loose, p, tokens of a pass), the first three as constants, for the kernel that serves a product.
template <typename Go>
auto with_kernel(const MatvecArgs& a, Go go) {
  MvParams p = params_of(a);
  // tokens of a pass: few pairs per expert are the rule in the grouped product
  const int nt = (a.ids ? a.M <= 4ll * a.G || a.M <= 8 : a.M <= 8) ? 1 : 2;
  const int mt = static_cast<int>(a.M < 8 * nt ? a.M : 8 * nt);
  const bool loose = a.K % 128 != 0;
  using One = std::integral_constant<int, 1>;
  using Two = std::integral_constant<int, 2>;
  auto tiles = [&](auto fmt) {
    if constexpr (fmt.value != QF_FMT_Q4_K)            // rows of Q4_K are whole super-blocks
      if (loose) return nt == 1 ? go(fmt, One{}, std::true_type{}, p, mt) : go(fmt, Two{}, std::true_type{}, p, mt);
    return nt == 1 ? go(fmt, One{}, std::false_type{}, p, mt) : go(fmt, Two{}, std::false_type{}, p, mt);
  };
  if (a.fmt == QF_FMT_Q4_K) return tiles(std::integral_constant<int, QF_FMT_Q4_K>{});
  if (a.fmt == QF_FMT_NVFP4) return tiles(std::integral_constant<int, QF_FMT_NVFP4>{});
  return tiles(std::integral_constant<int, QF_FMT_MXFP4>{});
}

}  // namespace

cudaError_t launch_matvec(const MatvecArgs& a, cudaStream_t st) {
  return with_kernel(a, [&](auto fmt, auto nt, auto loose, MvParams& p, int mt) {
    const int slots = !p.ids ? 1 : p.by_pair ? p.M : p.G;
    return launch<fmt.value, nt.value, loose.value>(p, slots, mt, st);
  });
}

void matvec_cut(const MatvecArgs& a, int* cut) {
  with_kernel(a, [&](auto fmt, auto nt, auto loose, MvParams& p, int mt) {
    const Cut c = cut_of<fmt.value, nt.value, loose.value>(p, mt);
    const int all[9] = {nt.value, loose.value, c.warps, c.kw, c.nz, p.kz, p.kc, p.blocks, static_cast<int>(c.grid_x)};
    for (int i = 0; i < 9; ++i) cut[i] = all[i];
  });
}

}  // namespace qf
