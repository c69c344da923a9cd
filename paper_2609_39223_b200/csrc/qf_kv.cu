// The 4-bit key/value cache: keys and values quantized as they are written, rows read back, and attention of a few tokens over it.
#include <cooperative_groups.h>
#include <math.h>

#include "qf_qdq_body.cuh"

namespace cg = cooperative_groups;

namespace qf {
namespace {

// ---- writing and reading rows --------------------------------------------------------------------------------------------
// Bound by memory: 2 bytes an element on one side, 0.53 or 0.56 on the other.
// Writing, a thread owns 16 consecutive elements of one head's row, of the keys or of the values: an NVFP4 block, or half an MXFP4 block
// (one shuffle with its neighbour). Reading, it owns 8, so that a warp's store is 512 bytes on end (with 16 elements and two stores of
// 32-byte steps the L1's write path was 75% busy: 78 us for 16 contexts of up to 8192 tokens, 62 now, 0.91 of the copy rate). A CTA takes
// a few tokens (slots): where their rows lie is found once per token, and a thread keeps its head and part while it goes through them, so
// that little is left to do per row but the row itself (divisions for every part: 94 us). Writing 16384 tokens of 8 heads of 128 takes
// 16.2 us in MXFP4 and 20.5 in NVFP4 (0.81 and 0.65 of the copy rate), whose quantizer has 1.3 times the instructions: half of the issue slots
// are used, warps wait for their CTA's slots (the barrier is the largest stall in MXFP4) and for the arithmetic's own results (in NVFP4). One
// row of a thread on the way instead of two: 16.9 and 20.1; four: 20.6 and 26.1 (registers).

constexpr int kRowsTokens = 64;      // tokens of a CTA at most
constexpr int kAppendTurns = 4, kReadTurns = 16;              // rows of a thread, where there are enough

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
  int64_t tokens;
  int each;                          // tokens of a CTA
  int page_size, heads;
  int units;                         // parts of a token
  int span, side;                    // threads for a token (CTAs beside one another have the next), tokens side by side: span * side <= kQdqThreads
  int shift;                         // parts of a head's row: 1 << shift
  bool slots64, noclip;
};

// Rows of the CTA's tokens in the cache: head h of token t lies in row at[t] + h * page_size; -1 outside the cache.
__device__ __forceinline__ int tokens_here(const KvRows& p) {
  return static_cast<int>(min(static_cast<int64_t>(p.each), p.tokens - static_cast<int64_t>(blockIdx.x) * p.each));
}
__device__ __forceinline__ void find_rows(const KvRows& p, int64_t (&at)[kRowsTokens]) {
  if (threadIdx.x < tokens_here(p)) {
    const int64_t t = static_cast<int64_t>(blockIdx.x) * p.each + threadIdx.x;
    const int64_t s = p.slots64 ? static_cast<const int64_t*>(p.slots)[t] : static_cast<const int32_t*>(p.slots)[t];
    const bool in = s >= 0 && s < p.slots_most;
    const int64_t page = !in ? 0 : s <= UINT32_MAX ? static_cast<uint32_t>(s) / static_cast<uint32_t>(p.page_size) : s / p.page_size;
    at[threadIdx.x] = in ? page * p.heads * p.page_size + (s - page * p.page_size) : -1;
  }
  __syncthreads();
}

template <int FMT>
__global__ void __launch_bounds__(kQdqThreads) kv_append_kernel(const __grid_constant__ KvRows p) {
  constexpr int TURNS = 2;           // rows of a thread that are loaded together, the next ones before these are quantized
  launch_after_previous();
  __shared__ int64_t at[kRowsTokens];
  const int here = tokens_here(p);
  const int column = static_cast<int>(threadIdx.x) % p.span, beside = static_cast<int>(threadIdx.x) / p.span;
  const int r = static_cast<int>(blockIdx.y) * p.span + column;
  const bool mine = r < p.units && beside < p.side, value = (r >> p.shift) >= p.heads;
  const int part = r & ((1 << p.shift) - 1), h = mine ? (r >> p.shift) - (value ? p.heads : 0) : 0;
  const int64_t stride = value ? p.v_stride : p.k_stride;
  const __nv_bfloat16* in = (value ? p.v : p.k) + static_cast<int64_t>(blockIdx.x) * p.each * stride + ((h << p.shift) + part) * 16;
  const int64_t row0 = static_cast<int64_t>(h) * p.page_size;
  uint8_t* codes = (value ? p.v_codes : p.k_codes) + ((row0 << p.shift) + part) * 8;
  uint8_t* scales = (value ? p.v_scales : p.k_scales) + (FMT == QF_FMT_NVFP4 ? (row0 << p.shift) + part : ((row0 << p.shift) + part) >> 1);
  // tokens that go nowhere are loaded as well: their slots need not be known yet
  uint4 x[TURNS][2];
  const auto load = [&](int t0) {
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
      const int t = t0 + i * p.side + beside;
      x[i][0] = x[i][1] = make_uint4(0, 0, 0, 0);
      if (mine && t < here) {
        const uint4* from = reinterpret_cast<const uint4*>(in + t * stride);
        x[i][0] = from[0];
        x[i][1] = from[1];
      }
    }
  };
  load(0);
  const Nvfp4Tensor nt = nvfp4_tensor(FMT == QF_FMT_NVFP4 ? *(value ? p.v_tscale : p.k_tscale) : 1.0f);
  find_rows(p, at);
  for (int t0 = 0; t0 < here; t0 += TURNS * p.side) {
    uint32_t w[TURNS][8];
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
      w[i][0] = x[i][0].x; w[i][1] = x[i][0].y; w[i][2] = x[i][0].z; w[i][3] = x[i][0].w;
      w[i][4] = x[i][1].x; w[i][5] = x[i][1].y; w[i][6] = x[i][1].z; w[i][7] = x[i][1].w;
    }
    load(t0 + TURNS * p.side);
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
      const int t = t0 + i * p.side + beside;
      const int64_t row = mine && t < here ? at[t] : -1;
      uint32_t m = unit_amax_bits(w[i]), scale_code;
      UnitOut o;
      if (FMT == QF_FMT_MXFP4) {
        m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
        o = mxfp4_unit(w[i], m, p.noclip, scale_code);
      } else {
        const float amax_b = __uint_as_float(m << 16);
        if (__all_sync(0xFFFFFFFFu, nt.denom_safe && (amax_b == 0.0f || amax_b >= 0x1p-60f)))
          o = nvfp4_unit<true>(w[i], amax_b, nt.s_t, nt.denom, nt.rc_denom, scale_code);
        else o = nvfp4_unit<false>(w[i], amax_b, nt.s_t, nt.denom, nt.rc_denom, scale_code);
      }
      if (row < 0) continue;
      *reinterpret_cast<uint2*>(codes + (row << (p.shift + 3))) = o.codes;
      if (FMT == QF_FMT_NVFP4) scales[row << p.shift] = static_cast<uint8_t>(scale_code);
      else if ((part & 1) == 0) scales[row << (p.shift - 1)] = static_cast<uint8_t>(scale_code);
    }
  }
}

template <int FMT>
__global__ void __launch_bounds__(kQdqThreads) kv_read_kernel(const __grid_constant__ KvRows p) {
  constexpr int TURNS = 4;
  launch_after_previous();
  __shared__ int64_t at[kRowsTokens];
  find_rows(p, at);
  const int here = tokens_here(p);
  const int column = static_cast<int>(threadIdx.x) % p.span, beside = static_cast<int>(threadIdx.x) / p.span;
  const int r = static_cast<int>(blockIdx.y) * p.span + column;
  if (beside >= p.side || r >= p.units) return;
  const bool value = !p.k_out || (r >> p.shift) >= p.heads;
  const int part = r & ((1 << p.shift) - 1), h = (r >> p.shift) - ((r >> p.shift) >= p.heads ? p.heads : 0);
  const int64_t first = ((static_cast<int64_t>(h) * p.page_size) << p.shift) + part, pitch = static_cast<int64_t>(p.heads) << p.shift;
  const uint32_t* codes = reinterpret_cast<const uint32_t*>(value ? p.v_codes : p.k_codes) + first;
  const uint8_t* scales = (value ? p.v_scales : p.k_scales) + (first >> (FMT == QF_FMT_NVFP4 ? 1 : 2));
  uint4* out = reinterpret_cast<uint4*>(value ? p.v_out : p.k_out) + static_cast<int64_t>(blockIdx.x) * p.each * pitch + (h << p.shift) + part;
  const float2 st = splat(FMT == QF_FMT_NVFP4 ? *(value ? p.v_tscale : p.k_tscale) : 1.0f);
  for (int t0 = beside; t0 < here; t0 += TURNS * p.side) {
    uint32_t c[TURNS], sc[TURNS];
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
      const int t = t0 + i * p.side;
      const int64_t row = t < here ? at[t] : -1;
      c[i] = sc[i] = 0u;
      if (row >= 0) {
        c[i] = codes[row << p.shift];
        sc[i] = scales[row << (p.shift - (FMT == QF_FMT_NVFP4 ? 1 : 2))];
      }
    }
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
      const int t = t0 + i * p.side;
      if (t >= here) break;
      const float2 sb = splat(FMT == QF_FMT_NVFP4 ? e4m3_decode(sc[i] & 0x7Fu) : e8m0_scale(sc[i]));
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float2 o = __fmul2_rn(sb, e2m1x2_decode((c[i] >> (8 * j)) & 0xFFu));
        if (FMT == QF_FMT_NVFP4) o = __fmul2_rn(o, st);
        w[j] = pack_bf16x2(o.x, o.y);
      }
      out[t * pitch] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

KvRows kv_rows(const qf_kv_cache_t& c, const void* slots, bool slots64, int64_t tokens) {
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
  p.tokens = tokens;
  p.page_size = c.page_size;
  p.heads = c.kv_heads;
  return p;
}

template <typename... Params, typename... Args>
cudaError_t launch_overlapping(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, cudaStream_t st, int cluster, Args... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// parts: of a head's row (a power of two from 4 on); kinds: keys, values or both. A CTA gets tokens for a few turns of its threads, fewer
// where that would leave SMs without a CTA.
cudaError_t launch_rows(void (*kernel)(KvRows), KvRows& p, int parts, int kinds, int turns, cudaStream_t st) {
  for (p.shift = 2; 1 << p.shift < parts; ++p.shift) {}
  p.units = kinds * p.heads << p.shift;
  p.span = p.units < kQdqThreads ? p.units : kQdqThreads;
  p.side = kQdqThreads / p.span;
  const int columns = (p.units + p.span - 1) / p.span;         // CTAs side by side for a token's row
  const int64_t step = 4 * p.side, work = p.tokens * columns, even = work / (12 * kNumSMs * step) * step;
  const int64_t each = even >= turns * p.side ? turns * p.side : even > 0 ? even : work >= 2 * kNumSMs * step ? step : p.side;
  p.each = static_cast<int>(each < kRowsTokens ? each : kRowsTokens);
  return launch_overlapping(kernel, dim3(static_cast<unsigned>((p.tokens + p.each - 1) / p.each), columns), kQdqThreads, 0, st, 1, p);
}

// ---- attention -----------------------------------------------------------------------------------------------------------
// The floor is one read of the sequences' codes and scales. Both products run on mma.sync m16n8k16 with FP16 operands and FP32 sums, keys
// (values) as the 16-row operand and up to 8 NT rows of queries as columns. A tcgen05 tile would need the decoded keys and values in shared
// memory, 4 bytes of traffic for each element that takes 0.56 bytes of HBM; here a decoded element never leaves its lane's registers.
//
//  * Decoding. One conversion for two codes, one packed product for two scales. Keys: a lane's codes of a row are pairs of dimensions, and
//    which dimensions is free as long as the queries agree. Values: the contraction runs over keys, so the pairs are of two keys: the
//    nibbles of two rows' words are interleaved first (two logic operations for eight values).
//  * Exactness. An E2M1 value times its E4M3 scale has six significant bits and is exact in FP16. MXFP4 keys: the E2M1 values alone are
//    multiplied, and a block's sum gets its power of two in FP32. MXFP4 values: FP16 powers of two relative to a scale code that moves
//    with the data (28 binades without a move). A unit whose values' scales lie further apart takes them relative to each key's largest
//    (exact over 36 binades, below counts as zero) and that one's power into the key's weight, with a maximum of score plus power for the
//    FP16 range. Where the reference moves up, a row's base (below) moves down with it as far as its products so far allow. A query row is
//    scaled by a power of two to a maximum in [2^14, 2^15): exact in FP16 down to 2^-31 of its largest element. So scores are FP32 sums of
//    exact products.
//  * One pass over the keys. A row's weights are 2^(score - base); they enter the value product as FP16 numbers (off by 2^-11 of
//    themselves at most, or, below 2^-20 of the largest, by 2^-31 of that), the sum of weights takes them unrounded. The base is 2^6 below
//    the largest score of the unit that set it and moves when a score passes it by 2^14: rarely, so that most units need no exchange
//    between lanes but one vote (as against a maximum over the lanes and a product with all sums for every unit: 32 instructions of
//    600). A unit's value product starts from zero and is added in FP32: the tensor core truncates as it accumulates, and a chain of
//    thousands would drift.
//  * Copies: cp.async, two units a warp, with the pieces of a row in an order that keeps all reads free of bank conflicts.
//  * Work. Units of 32 keys of one (sequence, key head, tile of query rows) are numbered in that order, with 8 places for the start of each:
//    the CTAs take equal runs of them, whatever the lengths (sequences of up to 384 keys are not cut). A CTA's warps
//    share what it has of a sequence and meet in shared memory. Only a CTA's first and last pieces can be parts of longer sequences:
//    those go to the workspace, and a second kernel joins them in order. Where the page table holds short sequences only, each gets a
//    cluster of up to 8 CTAs instead, which meets in distributed shared memory: nothing to count, no second kernel (1 x 1000 keys: 8.8 us
//    without, 5.5 with); or, where there are many, a warp: no meeting either.
//
// What bounds it: latency. A unit's products are one chain from shared memory through conversion, scale, product, exponential and transpose to
// the second product, and an SM has 8 to 16 warps to run beside one another. 8 heads of 128, up to 8 rows: 613 instructions a unit in
// NVFP4 (257 on the ALU, which takes one every other cycle, 238 on the FMA pipes), 633 in MXFP4; a copy at the full rate leaves an SM's scheduler
// 806 cycles for a unit, and 56% of the issue slots are used. 128 x 8192: 230 us NVFP4, 234 MXFP4 (0.81 and 0.76 of the copy
// rate), heads of 256 212 and 227, of 64 (16 of them) 288 and 307. Three CTAs an SM with 168 registers: four with 128 took 1.01 times as long, two
// with 64 keys a unit 0.98 (and 1.03 to 1.2 times at ragged and short ones). Around the keys a call spends 3.7 us until the first data, up to
// 4 us on shares that the memory serves unevenly, 2 us where warps meet and 3.5 us in the second kernel: 1 x 131072 keys take 38 us where
// 23.4 is the floor.

constexpr int kUnitKeys = 32;
constexpr int kAttnWarpBits = 2, kAttnWarps = 1 << kAttnWarpBits;       // of a CTA
constexpr int kStages = 2;                    // units a warp has in shared memory or on the way
constexpr int kPieceCost = 8;                 // what a sequence's queries, meeting and result cost, in units
constexpr int kWhole = 12;                    // sequences of up to so many units are not cut
constexpr int kDirectUnits = 24;              // of a CTA, where every sequence gets CTAs of its own
constexpr int kAloneUnits = 4, kAloneMost = 64;              // of a warp, where every sequence gets a warp: per round of CTAs otherwise, at most
constexpr float kWeightTop = 6.0f, kWeightRoom = 8.0f;       // weights start at up to 2^6 and may reach 2^14 before their base is moved

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
  uint8_t* ws;
  int batch, pages, max_pages, page_size, max_keys;
  int q_len, q_heads, kv_heads, group;
  int rows, tiles, segs;                      // query rows of a key head; tiles of them; (key head, tile) pairs of a sequence
  int split;                                  // CTAs of a segment, a cluster, where each has its own; 0: a warp each
  bool by_segment;                            // JoinTasks are numbered by segment, not by CTA
  int64_t page_codes;                         // bytes of codes in a page
  float scale;                                // times log2 e
};

// Sizes of the kernel for a format, a head size and query rows in units of 8.
template <int FMT, int D, int NT>
struct Shape {
  static constexpr int BLOCK = FMT == QF_FMT_NVFP4 ? 16 : 32, NB = D / BLOCK;              // blocks of a row
  static constexpr int HALVES = D == 256 ? 2 : 1;                                          // 128-element halves of a row
  static constexpr int CODES = kUnitKeys * D / 2, SCALES = kUnitKeys * NB, STAGE = 2 * (CODES + SCALES);
  static constexpr int VMUL = FMT == QF_FMT_MXFP4 ? kUnitKeys * NB * 2 : 0;                // values' multipliers, where they need a pass of their own
  static constexpr int WARP = kStages * STAGE + VMUL;
  static constexpr int MT = D / 16;                                                        // 16-row tiles of the value product
  static constexpr int PART = (MT * NT * 4 + 4 * NT) * 32 * 4;                             // a warp's sums and maxima, bytes
  static constexpr int SMEM = kAttnWarps * WARP + kAttnWarps / 2 * PART;
  static constexpr int FIT = 232448 / (SMEM + 1024), WANT = D == 256 ? 2 : D == 128 ? (NT == 1 ? 3 : 2) : NT < 3 ? 4 : 6 - NT;
  static constexpr int CTAS = FIT < WANT ? FIT : WANT;                                     // of an SM
};

// Workspace: a task per CTA (or per segment, where there are fewer), then two parts per CTA (the piece it continues, the piece it begins).
struct JoinTask { int cta, more, b, seg; };   // parts are those of CTAs cta, cta + 1, ..., cta + more (more = 0: nothing to join)

__device__ __forceinline__ uint32_t f16x2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b) {
  const __half2 h = __hmul2(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Eight E2M1 codes -> four FP16 pairs (2i, 2i + 1)
__device__ __forceinline__ void e2m1_f16(uint32_t q, uint32_t (&w)[4]) {
  asm("{\n.reg .b8 a, b, c, d;\nmov.b32 {a, b, c, d}, %4;\n"
      "cvt.rn.f16x2.e2m1x2 %0, a;\ncvt.rn.f16x2.e2m1x2 %1, b;\ncvt.rn.f16x2.e2m1x2 %2, c;\ncvt.rn.f16x2.e2m1x2 %3, d;\n}"
      : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
      : "r"(q));
}
// An E4M3 code's seven bits under FP16's exponent are its value times 2^-8, exactly, subnormals included, and code 0x7F, the scale of a
// block of NaNs, is the number 480 that reading it back takes it for. (As the NaN of the conversion instruction it would reach the sums of
// tokens that do not see its key.)
constexpr int kE4m3Down = 8;
__device__ __forceinline__ uint32_t e4m3_twice(uint32_t code) { return code * 0x00800080u; }
__device__ __forceinline__ uint32_t e4m3_pair(uint32_t low, uint32_t high) { return low * 0x80u + high * 0x00800000u; }
// E8M0 code `i` of four -> its power of two; code 0 -> 0 (zeros, or elements below 2^-124)
__device__ __forceinline__ float e8m0_of(uint32_t codes, int i) {
  const uint32_t at = i == 3 ? codes >> 1 : codes << (23 - 8 * i);
  return __uint_as_float(at & 0x7F800000u);
}
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// Places in dynamic shared memory are bytes from its start: plain accesses, which the compiler may order between the barriers.
template <typename T>
__device__ __forceinline__ T smem_load(uint32_t at) {
  extern __shared__ __align__(128) uint8_t smem[];
  return *reinterpret_cast<const T*>(smem + at);
}
template <typename T>
__device__ __forceinline__ void smem_store(uint32_t at, const T& v) {
  extern __shared__ __align__(128) uint8_t smem[];
  *reinterpret_cast<T*>(smem + at) = v;
}

__device__ __forceinline__ int keys_of(const KvAttn& p, int b) { return min(max(p.lens[b], 0), p.max_keys); }
__device__ __forceinline__ int units_of(int keys) { return (keys + kUnitKeys - 1) / kUnitKeys; }
// what a segment of a sequence counts for in the shares: a sequence without keys nothing (its zeros are written beforehand)
__device__ __forceinline__ int cost_of(int keys) { return keys == 0 ? 0 : units_of(keys) + kPieceCost; }

// end of part i - 1 of 1 << bits parts of n units, start of part i
__device__ __forceinline__ int part_of(int n, int i, int bits) { return static_cast<int>(static_cast<int64_t>(n) * i >> bits); }
// token of a query row of a key head, key head of a segment
__device__ __forceinline__ int token_of(const KvAttn& p, int row) { return p.q_len == 1 ? 0 : row / p.group; }
__device__ __forceinline__ int head_of(const KvAttn& p, int segment) { return p.tiles == 1 ? segment : segment / p.tiles; }

// The pieces of a CTA's share, one (sequence, segment) after the other: units [j, j + n) of segment s of sequence b; n = 0 at the end.
// In a segment's part of the shares kPieceCost places come first, then a place per unit.
struct Walk {
  int b, s, keys, units, j, n, left, pos;     // left: places of the share behind this piece; pos: place in the segment where the share starts
  __device__ __forceinline__ void settle(const KvAttn& p) {
    for (n = 0; left > 0;) {
      const int here = min(left, units + kPieceCost - pos);
      j = max(pos - kPieceCost, 0);
      n = max(pos + here - kPieceCost, 0) - j;
      left -= here;
      if (n > 0 || left <= 0) return;
      segment(p);
    }
  }
  __device__ __forceinline__ void segment(const KvAttn& p) {
    pos = 0;
    if (++s < p.segs) return;
    s = 0;
    do keys = keys_of(p, ++b);                // places are left, so there is a sequence with keys
    while (keys == 0);
    units = units_of(keys);
  }
  __device__ __forceinline__ void next(const KvAttn& p) {
    n = 0;
    if (left <= 0) return;
    segment(p);
    settle(p);
  }
};

// 16-byte piece c of a row's codes lies in place c ^ turn(row), so that lanes that read together meet different banks: of keys a row's
// pieces for two rows (NVFP4) or a piece of each of eight rows (MXFP4), of values half a row's for four rows from either end of eight.
template <int D>
__device__ __forceinline__ int turn(int row) {
  return ((row >> 2) & 1) + (D >= 128 ? ((row >> 1) & 1) * 2 : 0) + (D == 256 ? (row & 1) * 4 : 0);
}

// A warp's copies into its ring: its quarter of every piece, unit by unit, ahead of the products. Keys come in groups of 16 that lie in
// one page; the first group of a unit always holds a key, the second may not.
template <int FMT, int D>
struct Copier {
  using S = Shape<FMT, D, 1>;
  static constexpr int ROW = D / 2, PIECES = ROW / 16, SROW = S::NB, CHUNKS = SROW, SHIFT = FMT == QF_FMT_NVFP4 ? 3 : 4;   // ROW = SROW << SHIFT
  static constexpr bool ONCE = 4 * CHUNKS <= 32;               // one instruction copies the unit's scales
  Walk w;
  int cur, end, page, off;                    // unit, end of this warp's part of the piece, page and place of its first key
  int id0, id1;                               // pages of its two groups
  const int32_t* pages;                       // of the sequence
  const uint8_t* kp;                          // this lane's first piece of a group, in page 0 from the head's first key on
  const uint8_t* vp;
  const uint8_t* sp;                          // and its scales, keys' or values'
  uint32_t to, to_scales;                     // their places in a stage

  __device__ __forceinline__ void ids(const KvAttn& p) {
    const uint32_t most = static_cast<uint32_t>(p.pages - 1);
    id1 = id0 = static_cast<int>(min(static_cast<uint32_t>(pages[page]), most));
    if (off + 16 >= p.page_size && cur * kUnitKeys + 16 < w.keys) id1 = static_cast<int>(min(static_cast<uint32_t>(pages[page + 1]), most));
  }
  __device__ __forceinline__ void piece(const KvAttn& p, int warp, int bits, int lane) {
    for (; w.n > 0; w.next(p)) {
      cur = w.j + part_of(w.n, warp, bits);
      end = w.j + part_of(w.n, warp + 1, bits);
      if (cur < end) break;
    }
    if (w.n == 0) return;
    page = cur * kUnitKeys / p.page_size;
    off = cur * kUnitKeys - page * p.page_size;
    pages = p.table + static_cast<int64_t>(w.b) * p.max_pages;
    const int64_t row = static_cast<int64_t>(head_of(p, w.s)) * p.page_size;
    kp = p.k_codes + row * ROW + lane * 16;
    vp = p.v_codes + row * ROW + lane * 16;
    const int c = lane % (2 * CHUNKS);
    sp = (c >= CHUNKS ? p.v_scales : p.k_scales) + row * SROW + c % CHUNKS * 16;
    ids(p);
  }
  __device__ __forceinline__ void start(const KvAttn& p, int warp, int bits, int lane) {
    const int r = lane / PIECES, c = lane % (2 * CHUNKS);
    to = r * ROW + ((lane % PIECES) ^ turn<D>(r)) * 16;
    to_scales = 2 * S::CODES + (c >= CHUNKS ? S::SCALES : 0) + c % CHUNKS * 16 + (ONCE ? lane / (2 * CHUNKS) * 16 * SROW : 0);
    piece(p, warp, bits, lane);
  }
  __device__ __forceinline__ void codes(uint32_t stage, int64_t at) const {
#pragma unroll
    for (int i = 0; i < PIECES / 2; ++i) {
      const uint32_t here = D == 256 && (i & 1) ? to ^ 16 : to;          // rows 4 i and on: the lowest bit of their turn
      copy16(stage + here + i * 512, kp + at + i * 512);
      copy16(stage + here + S::CODES + i * 512, vp + at + i * 512);
    }
  }
  __device__ __forceinline__ void issue(const KvAttn& p, uint32_t stage, int warp, int bits, int lane) {
    if (w.n > 0) {
      const bool two = cur * kUnitKeys + 16 < w.keys;
      const int64_t a0 = id0 * p.page_codes + off * ROW;
      const int64_t a1 = id1 * p.page_codes + (off + 16 < p.page_size ? off + 16 : 0) * ROW;
      codes(stage, a0);
      if (two) codes(stage + 16 * ROW, a1);
      if constexpr (ONCE) {
        const bool second = lane >= 2 * CHUNKS;
        if (lane < (two ? 4 : 2) * CHUNKS) copy16(stage + to_scales, sp + ((second ? a1 : a0) >> SHIFT));
      } else {
        copy16(stage + to_scales, sp + (a0 >> SHIFT));
        if (two) copy16(stage + to_scales + 16 * SROW, sp + (a1 >> SHIFT));
      }
      if (++cur < end) {
        off += kUnitKeys;
        while (off >= p.page_size) { off -= p.page_size; ++page; }
        ids(p);
      } else {
        w.next(p);
        piece(p, warp, bits, lane);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
};

// What a lane has of a piece: of the value product row 16 i + g (dimension 2i of the lane's, i counting) and row 16 i + g + 8 (dimension
// 2i + 1), columns (query rows) 8 n + 2t and 8 n + 2t + 1; and of these columns the maximum and the sum.
template <int MT, int NT>
struct Sums {
  float o[MT][NT][4];
  float m[NT][2], l[NT][2];
};

// Element of the head that row r (0 or 1) of value tile i holds for lane row g.
template <int D>
__device__ __forceinline__ int dim_of(int i, int g) {
  return D == 64 ? g * 8 + 2 * i : (i >> 3) * 128 + g * 16 + 2 * (i & 7);
}

constexpr float kNoWeights = -3.4028234663852886e38f;        // base of a column without weights: no finite score is below it
// Power of two that brings a sum of weights into [1/4, 1/2) (zero stays zero) and its base along with it; what the base moved by is
// returned in `by`. MXFP4's values may fill FP32's range: sums of them stay in it as long as their weights add up to less than one. (A
// base so large that its steps are whole powers moves as far as it can, and the sum with it.)
__device__ __forceinline__ float even_out(float& m, float l, float& by) {
  const float to = m + static_cast<float>(static_cast<int>(__float_as_uint(l) >> 23) - 125);
  by = to - m;
  m = to;
  return exp2_approx(-by);
}
// Two columns of weights into one: factors of the sums that belong to them, base and sum.
template <bool EVEN>
__device__ __forceinline__ void join_weights(float& m, float& l, float mb, float lb, float& fa, float& fb) {
  const float most = fmaxf(m, mb);
  fa = exp2_approx(m - most);
  fb = exp2_approx(mb - most);
  l = l * fa + lb * fb;
  m = most;
  if constexpr (EVEN) {
    float by;
    const float f = even_out(m, l, by);
    fa *= f;
    fb *= f;
    l *= f;
  }
}

// A value tile's sums over several parts, with the bases and sums of the lane's two columns.
template <bool EVEN>
struct Joint {
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f), ml = make_float4(kNoWeights, 0.0f, kNoWeights, 0.0f);
  __device__ __forceinline__ void add(const float4& v, const float4& w) {
    float fa[2], fb[2];
    join_weights<EVEN>(ml.x, ml.y, w.x, w.y, fa[0], fb[0]);
    join_weights<EVEN>(ml.z, ml.w, w.z, w.w, fa[1], fb[1]);
    o.x = o.x * fa[0] + v.x * fb[0];
    o.y = o.y * fa[1] + v.y * fb[1];
    o.z = o.z * fa[0] + v.z * fb[0];
    o.w = o.w * fa[1] + v.w * fb[1];
  }
};

// What sums of products have to be multiplied with, for a sum of weights
template <bool MX>
__device__ __forceinline__ float part_factor(float vt, float l) { return l == 0.0f ? 0.0f : vt / (MX ? l : l * (1.0f / (1 << kE4m3Down))); }
// Of no weight at all: -infinity; of a sum that is NaN: NaN, like the row's outputs.
__device__ __forceinline__ float log_sum(float m, float l) { return l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f; }

__device__ __forceinline__ float4* parts_of(const KvAttn& p, int grid) {
  return reinterpret_cast<float4*>(p.ws + ((grid * sizeof(JoinTask) + 255) & ~static_cast<size_t>(255)));
}

template <int D, int NT, bool EVEN>
__device__ __forceinline__ void write_tile(const KvAttn& p, const Joint<EVEN>& sum, int b, int segment, int tile, int lane, float vt) {
  const int h = head_of(p, segment), i = tile / NT, n = tile % NT, g = lane >> 2, t = lane & 3;
  const int row0 = (segment - h * p.tiles) * (8 * NT) + 8 * n + 2 * t;
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const int row = row0 + c;
    if (row >= p.rows) continue;
    const int token = token_of(p, row), head = h * p.group + (row - token * p.group);
    const int64_t at = (static_cast<int64_t>(b) * p.q_len + token) * p.q_heads + head;
    const float l = c ? sum.ml.w : sum.ml.y, f = part_factor<EVEN>(vt, l);
    *reinterpret_cast<uint32_t*>(p.out + at * D + dim_of<D>(i, g)) = pack_bf16x2((c ? sum.o.y : sum.o.x) * f, (c ? sum.o.w : sum.o.z) * f);
    if (p.lse && i == 0 && g == 0) p.lse[at] = log_sum(c ? sum.ml.z : sum.ml.x, l);
  }
}

// DIRECT: a cluster of p.split CTAs (or one CTA) to every segment, in place of equal shares of all of them.
template <int FMT, int D, int NT, bool DIRECT>
__global__ void __launch_bounds__(kAttnWarps * 32, (Shape<FMT, D, NT>::CTAS)) kv_attention_kernel(const __grid_constant__ KvAttn p) {
  using S = Shape<FMT, D, NT>;
  constexpr int MT = S::MT, NB = S::NB, HALVES = S::HALVES;
  constexpr bool MX = FMT == QF_FMT_MXFP4;
  constexpr int NW = D / 32;                                   // words of codes of a key that a lane holds
  constexpr int VWORDS = D == 64 ? 1 : 2;                      // and of a value, per half
  constexpr bool QS = D == 256 && NT == 2;                     // queries in shared memory (where the parts meet later) instead of 64 registers
  constexpr uint32_t QUERIES = NT * NW * 512;                  // of a warp
  static_assert(!QS || kAttnWarps * QUERIES <= kAttnWarps / 2 * S::PART, "a warp's queries for each");
  extern __shared__ __align__(128) uint8_t smem[];
  launch_after_previous();
  const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t base = static_cast<uint32_t>(__cvta_generic_to_shared(smem));
  const uint32_t ring = warp * S::WARP, vmul = ring + kStages * S::STAGE, parts = kAttnWarps * S::WARP;
  JoinTask* tasks = reinterpret_cast<JoinTask*>(p.ws);
  const int cta = blockIdx.x;
  const bool alone = DIRECT && p.split == 0;                   // this warp has a segment for itself: no meeting anywhere below
  const int part = alone ? 0 : warp, bits = alone ? 0 : kAttnWarpBits;
  if (!DIRECT && !p.by_segment && threadIdx.x == 0) tasks[cta].more = 0;

  const float vt = MX ? 1.0f : *p.v_tscale;
  const float kt = p.scale * (MX ? 1.0f : *p.k_tscale);
  const float sign = kt < 0.0f ? -1.0f : 1.0f;                 // of the scale: goes to the queries, so that a column's factor is positive

  // A sequence without keys: zeros. (With keys: nothing.)
  const auto write_zeros = [&](int b) {
    if (keys_of(p, b) > 0) return;
    const int64_t first = static_cast<int64_t>(b) * p.q_len * p.q_heads, rows = static_cast<int64_t>(p.q_len) * p.q_heads;
    const int thread = alone ? lane : threadIdx.x, threads = alone ? 32 : kAttnWarps * 32;
    uint4* out = reinterpret_cast<uint4*>(p.out + first * D);
    for (int64_t i = thread; i < rows * (D / 8); i += threads) out[i] = make_uint4(0, 0, 0, 0);
    if (p.lse)
      for (int64_t i = thread; i < rows; i += threads) p.lse[first + i] = -INFINITY;
    if (p.by_segment)
      for (int i = threadIdx.x; i < p.segs; i += kAttnWarps * 32) tasks[b * p.segs + i].more = 0;
  };

  Walk w;
  int ctas = 0;                                                // shares
  int64_t total = 0, share = 0, u1 = 0;                        // places of all, places of a share, end of this one
  if constexpr (DIRECT) {
    const int split = alone ? 1 : p.split;
    const int segment = alone ? cta * kAttnWarps + warp : cta / split, rank = alone ? 0 : cta - segment * split;
    w.b = segment / p.segs;
    if (w.b >= p.batch) return;                                // (warps of their own only)
    w.s = segment - w.b * p.segs;
    w.keys = keys_of(p, w.b);
    if (w.keys == 0) {
      if (w.s == 0 && rank == 0) write_zeros(w.b);
      return;
    }
    w.units = units_of(w.keys);
    w.j = static_cast<int>(static_cast<int64_t>(w.units) * rank / split);
    w.n = static_cast<int>(static_cast<int64_t>(w.units) * (rank + 1) / split) - w.j;
    w.left = w.pos = 0;
  } else {
    // This CTA's share. All places are counted by all CTAs, each thread a run of the sequences. A border between two shares that falls into
    // a short sequence moves to the nearer end of it, for both of them.
    __shared__ int64_t warp_places[kAttnWarps], border[2];
    __shared__ int first_b, first_s, first_pos, first_keys;
    const int per = (p.batch + kAttnWarps * 32 - 1) / (kAttnWarps * 32);
    const int b0 = min(static_cast<int>(threadIdx.x) * per, p.batch), b1 = min(b0 + per, p.batch);
    const int keys0 = b0 < b1 ? keys_of(p, b0) : 0;            // of the run's first
    int64_t mine = cost_of(keys0);
    for (int b = b0 + 1; b < b1; ++b) mine += cost_of(keys_of(p, b));
    mine *= p.segs;
    int64_t before = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int64_t o = __shfl_up_sync(0xFFFFFFFFu, before, d);
      if (lane >= d) before += o;
    }
    if (lane == 31) warp_places[warp] = before;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kAttnWarps; ++i) {
      if (i < warp) before += warp_places[i];
      total += warp_places[i];
    }
    before -= mine;
    ctas = static_cast<int>(min(static_cast<int64_t>(gridDim.x), (total + kAttnWarps - 1) / kAttnWarps));
    bool idle = cta >= ctas;
    if (!idle) {
      // the first CTAs take a place more each, as many as are left over
      share = total <= UINT32_MAX ? static_cast<uint32_t>(total) / static_cast<uint32_t>(ctas) : total / ctas;
      const int rest = static_cast<int>(total - share * ctas);
      u1 = (cta + 1) * share + min(cta + 1, rest);
#pragma unroll 1
      for (int i = 0; i < 2; ++i) {
        const int64_t u = i ? u1 : cta * share + min(cta, rest);
        if (u == total && threadIdx.x == 0) border[i] = total;
        if (u < before || u >= before + mine) continue;
        int64_t r = u - before;
        int b = b0, keys = keys0;
        for (; r >= static_cast<int64_t>(cost_of(keys)) * p.segs; keys = keys_of(p, ++b)) r -= static_cast<int64_t>(cost_of(keys)) * p.segs;
        const int cost = cost_of(keys), s = static_cast<int>(r <= UINT32_MAX ? static_cast<uint32_t>(r) / static_cast<uint32_t>(cost) : r / cost);
        const int pos = static_cast<int>(r - static_cast<int64_t>(s) * cost);
        const int moved = cost > kWhole + kPieceCost ? pos : 2 * pos < cost ? 0 : cost;
        border[i] = u + (moved - pos);
        if (i == 0) {
          first_b = b;
          first_s = s;
          first_pos = moved;
          first_keys = keys;
        }
      }
      __syncthreads();
      idle = border[1] <= border[0];
    }
    if (idle) {
      for (int b = cta; b < p.batch; b += gridDim.x) write_zeros(b);
      return;
    }
    w.b = first_b;
    w.s = first_s;
    w.pos = first_pos;
    w.keys = first_keys;
    w.units = units_of(w.keys);
    w.left = static_cast<int>(border[1] - border[0]);
    w.settle(p);
  }

  // Queries of a piece: 8 rows to a tile, row g of which is this lane's
  uint4 raw[NT][NW];
  const auto fetch = [&](const Walk& x) {
    const int h = head_of(p, x.s), row0 = (x.s - h * p.tiles) * (8 * NT);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int row = row0 + 8 * n + g;
      const bool any = x.n > 0 && row < p.rows;
      const int token = any ? token_of(p, row) : 0, head = h * p.group + (any ? row - token * p.group : 0);
      const __nv_bfloat16* src = p.q + (static_cast<int64_t>(x.b) * p.q_len + token) * p.q_stride + static_cast<int64_t>(head) * D;
#pragma unroll
      for (int i = 0; i < NW; ++i) {
        const int at = MX ? i * 32 + t * 8 : D == 64 ? t * 16 + 8 * i : (i >> 2) * 128 + t * 32 + 8 * (i & 3);
        raw[n][i] = any ? *reinterpret_cast<const uint4*>(src + at) : make_uint4(0, 0, 0, 0);
      }
    }
  };
  fetch(w);
  Copier<FMT, D> copy;
  copy.w = w;
  copy.start(p, part, bits, lane);
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) copy.issue(p, base + ring + i * S::STAGE, part, bits, lane);
  int stage = 0;
  if constexpr (!DIRECT)
    for (int b = cta; b < p.batch; b += gridDim.x) write_zeros(b);       // while the first keys are on their way

  // Row g of a 16-key tile is key own0 of its first eight, row g + 8 the same of the second; the keys of a lane's columns of the value product
  // then are t and 7 - t of both eights.
  const int own0 = (g & 1) ? 7 - (g >> 1) : g >> 1;
  // This lane's places in a stage: its words of keys, their scales; its words of values for keys t and 7 - t, and their scales. (Kept as they
  // are: the compiler would work them out for every unit.)
  uint32_t k_at = own0 * (D / 2) + (MX ? turn<D>(own0) * 16 + t * 4 : D == 64 ? ((t >> 1) ^ turn<D>(own0)) * 16 + (t & 1) * 8 : (t ^ turn<D>(own0)) * 16);
  uint32_t ks_at = 2 * S::CODES + own0 * NB + (MX ? 0 : D == 64 ? t : 2 * t);
  uint32_t v_at[2], vs_at[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int own = i ? 7 - t : t, block = MX ? (D == 64 ? g >> 2 : g >> 1) : D == 64 ? g >> 1 : g;
    v_at[i] = S::CODES + own * (D / 2) + (D == 64 ? ((g >> 2) ^ turn<D>(own)) * 16 + (g & 3) * 4 : ((g >> 1) ^ turn<D>(own)) * 16 + (g & 1) * 8);
    vs_at[i] = 2 * S::CODES + S::SCALES + own * NB + block;
    asm volatile("" : "+r"(v_at[i]), "+r"(vs_at[i]));
  }
  asm volatile("" : "+r"(k_at), "+r"(ks_at));
  // (a CTA of a cluster may have no unit of its segment, and meets the others all the same)
  for (Walk next; DIRECT || w.n > 0; w = next) {
    const int h = head_of(p, w.s), row0 = (w.s - h * p.tiles) * (8 * NT);
    // queries of this tile as FP16 fragments, and what a score has to be multiplied with
    uint32_t qf[NT][D / 16][2];
    float by[NT][2];
    int seen[NT][2], least = w.keys;                           // keys that a column sees
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < NW; ++i) top = max(top, chunk_amax_bits(raw[n][i]));
      top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
      top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
      const int e = max(static_cast<int>(top >> 7), 14);       // exponent of the row's largest element
      const float up = sign * __uint_as_float(static_cast<uint32_t>(268 - e) << 23);
      const int undo = e - 14 + (MX ? 0 : kE4m3Down);
      const float down = undo == 0 ? 0x1p-127f : __uint_as_float(static_cast<uint32_t>(undo) << 23);
#pragma unroll
      for (int i = 0; i < NW; ++i) {
        const uint32_t v[4] = {raw[n][i].x, raw[n][i].y, raw[n][i].z, raw[n][i].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) qf[n][2 * i + (k >> 1)][k & 1] = f16x2(bf16_lo(v[k]) * up, bf16_hi(v[k]) * up);
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        // not zero, so that a score of -infinity stays one
        by[n][c] = fmaxf(__shfl_sync(0xFFFFFFFFu, down, (2 * t + c) * 4) * fabsf(kt), 0x1p-149f);
        const int tok = token_of(p, min(row0 + 8 * n + 2 * t + c, p.rows - 1));
        seen[n][c] = min(max(w.keys - p.q_len + tok + 1, 0), w.keys);
      }
      if (n == 0) least = min(max(w.keys - p.q_len + token_of(p, row0) + 1, 0), w.keys);
    }

    const uint32_t queries = parts + (alone ? warp * QUERIES : 0);
    if constexpr (QS) {
      if (warp == 0 || alone) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < NW; ++i)
            smem_store(queries + ((n * NW + i) * 32 + lane) * 16, make_uint4(qf[n][2 * i][0], qf[n][2 * i][1], qf[n][2 * i + 1][0], qf[n][2 * i + 1][1]));
      }
      if (alone) __syncwarp();
      else __syncthreads();
    }
    // fragments of word i of the rows of tile n
    const auto query = [&](int n, int i) {
      if constexpr (QS) return smem_load<uint4>(queries + ((n * NW + i) * 32 + lane) * 16);
      else return make_uint4(qf[n][2 * i][0], qf[n][2 * i][1], qf[n][2 * i + 1][0], qf[n][2 * i + 1][1]);
    };

    // m: base of a column's weights, which are 2^(score - m); l: the lane's share of their sum; ve (MXFP4): o is in units of 2^ve; vref: the
    // scale code that the values' multipliers refer to (none yet: far below all)
    Sums<MT, NT> a;
    float ve[NT][2];
    int vref = -100, vhigh = 0;                                // vhigh: largest scale code so far
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int c = 0; c < 2; ++c) { a.m[n][c] = kNoWeights; a.l[n][c] = 0.0f; ve[n][c] = -1000.0f; }
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) a.o[i][n][c] = 0.0f;
    }

    const int from = w.j + part_of(w.n, part, bits), to = w.j + part_of(w.n, part + 1, bits);
    for (int u = from; u < to; ++u) {
      copy.issue(p, base + ring + (stage == 0 ? kStages - 1 : stage - 1) * S::STAGE, part, bits, lane);
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
      __syncwarp();
      const uint32_t here = ring + stage * S::STAGE;
      stage = stage + 1 == kStages ? 0 : stage + 1;
      const int key0 = u * kUnitKeys;

      // Scores. NVFP4: a lane's words are one or two whole blocks, whose scale goes to the key's elements. MXFP4: word x of the four lanes of a
      // row is block x, whose power of two goes to the block's sum.
      float s[2][NT][4];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) s[half][n][c] = 0.0f;
        const uint32_t keys = here + k_at + half * 16 * (D / 2), kscales = here + ks_at + half * 16 * NB;      // row g; row g + 8 is 8 rows on
        if constexpr (MX) {
          uint32_t f0[(NB + 3) / 4], f1[(NB + 3) / 4];
#pragma unroll
          for (int i = 0; i < (NB + 3) / 4; ++i) {
            if constexpr (NB == 2) {
              f0[i] = smem_load<uint16_t>(kscales);
              f1[i] = smem_load<uint16_t>(kscales + 8 * NB);
            } else {
              f0[i] = smem_load<uint32_t>(kscales + 4 * i);
              f1[i] = smem_load<uint32_t>(kscales + 8 * NB + 4 * i);
            }
          }
#pragma unroll
          for (int x = 0; x < NW; ++x) {
            const uint32_t word = here + (k_at ^ (x * 16)) + half * 16 * (D / 2);
            uint32_t d0[4], d1[4];
            e2m1_f16(smem_load<uint32_t>(word), d0);
            e2m1_f16(smem_load<uint32_t>(word + 8 * (D / 2)), d1);
            const float y0 = e8m0_of(f0[x / 4], x & 3), y1 = e8m0_of(f1[x / 4], x & 3);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
              const uint4 q = query(n, x);
              mma(z, d0[0], d1[0], d0[1], d1[1], q.x, q.y);
              mma(z, d0[2], d1[2], d0[3], d1[3], q.z, q.w);
              s[half][n][0] = fmaf(z[0], y0, s[half][n][0]);
              s[half][n][1] = fmaf(z[1], y0, s[half][n][1]);
              s[half][n][2] = fmaf(z[2], y1, s[half][n][2]);
              s[half][n][3] = fmaf(z[3], y1, s[half][n][3]);
            }
          }
        } else {
#pragma unroll
          for (int hh = 0; hh < HALVES; ++hh) {
            constexpr int WORDS = D == 64 ? 2 : 4;
            uint32_t c0[WORDS], c1[WORDS], x0[2], x1[2];
            if constexpr (D == 64) {
              const uint2 v0 = smem_load<uint2>(keys), v1 = smem_load<uint2>(keys + 8 * 32);
              c0[0] = v0.x; c0[1] = v0.y; c1[0] = v1.x; c1[1] = v1.y;
              x0[0] = e4m3_twice(smem_load<uint8_t>(kscales));
              x1[0] = e4m3_twice(smem_load<uint8_t>(kscales + 8 * NB));
            } else {
              const uint32_t words = hh == 0 ? keys : here + (k_at ^ 64) + half * 16 * (D / 2);
              const uint4 v0 = smem_load<uint4>(words), v1 = smem_load<uint4>(words + 8 * (D / 2));
              c0[0] = v0.x; c0[1] = v0.y; c0[2] = v0.z; c0[3] = v0.w;
              c1[0] = v1.x; c1[1] = v1.y; c1[2] = v1.z; c1[3] = v1.w;
              const uint32_t y0 = smem_load<uint16_t>(kscales + hh * 8), y1 = smem_load<uint16_t>(kscales + 8 * NB + hh * 8);
              x0[0] = e4m3_twice(y0 & 0xFFu); x0[1] = e4m3_twice(y0 >> 8);
              x1[0] = e4m3_twice(y1 & 0xFFu); x1[1] = e4m3_twice(y1 >> 8);
            }
#pragma unroll
            for (int x = 0; x < WORDS; ++x) {
              uint32_t d0[4], d1[4];
              e2m1_f16(c0[x], d0);
              e2m1_f16(c1[x], d1);
#pragma unroll
              for (int i = 0; i < 4; ++i) { d0[i] = hmul2(d0[i], x0[x >> 1]); d1[i] = hmul2(d1[i], x1[x >> 1]); }
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                const uint4 q = query(n, hh * 4 + x);
                mma(s[half][n], d0[0], d1[0], d0[1], d1[1], q.x, q.y);
                mma(s[half][n], d0[2], d1[2], d0[3], d1[3], q.z, q.w);
              }
            }
          }
        }
      }
      if (key0 + kUnitKeys > least) {
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 4; ++c)
              if (key0 + half * 16 + (c >> 1) * 8 + own0 >= seen[n][c & 1]) s[half][n][c] = -INFINITY;
      }

      // Scores, rounded for themselves: of the unrounded product less its base something would be left over, and be more than the room
      // there is where scores are large. Bases move only when a score passes one by more than that.
      float top[NT][2];
      bool move = false;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float2 by2 = make_float2(by[n][0], by[n][1]);
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const float2 x = __fmul2_rn(make_float2(s[half][n][2 * r], s[half][n][2 * r + 1]), by2);
            s[half][n][2 * r] = x.x;
            s[half][n][2 * r + 1] = x.y;
          }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          top[n][c] = fmaxf(fmaxf(s[0][n][c], s[0][n][c + 2]), fmaxf(s[1][n][c], s[1][n][c + 2]));
          move |= top[n][c] - a.m[n][c] > kWeightTop + kWeightRoom;
        }
      }
      // MXFP4: a scale code c of the values is taken as the FP16 number 2^(c - vref + 5), which is exact and in range for c in
      // [vref - 19, vref + 8]; a code of 0 comes with zeros, whatever it is taken for. A lane looks at its key's codes: largest, and
      // smallest but 0, less 1.
      int key_top = 0, key_low = 0xFFFF;
      bool wide = false;
      uint32_t vword[(NB + 3) / 4];
      if constexpr (MX) {
        uint32_t top2 = 0, low2 = 0xFFFFFFFFu;
#pragma unroll
        for (int i = 0; i < (NB + 3) / 4; ++i) {
          if constexpr (NB == 2) vword[i] = __byte_perm(smem_load<uint16_t>(here + 2 * S::CODES + S::SCALES + lane * NB), 0, 0x4140);
          else vword[i] = smem_load<uint32_t>(here + 2 * S::CODES + S::SCALES + lane * NB + 4 * i);
          const uint32_t even = NB == 2 ? vword[i] : vword[i] & 0x00FF00FFu, odd = NB == 2 ? even : __byte_perm(vword[i], 0, 0x4341);
          top2 = __vmaxu2(top2, __vmaxu2(even, odd));
          low2 = __viaddmin_u16x2(even, 0xFFFFFFFFu, __viaddmin_u16x2(odd, 0xFFFFFFFFu, low2));
        }
        if (key0 + lane < w.keys) {
          key_top = max(top2 & 0xFFFFu, top2 >> 16);
          key_low = min(low2 & 0xFFFFu, low2 >> 16);
        }
        move |= key_top > vref + 8 || key_low < vref - 20;
      }
      if (__any_sync(0xFFFFFFFFu, move)) {
        float was[NT][2];                                      // logarithm of what the weights so far have to be multiplied with
        const int vtop = MX ? __reduce_max_sync(0xFFFFFFFFu, key_top) : 0, vlow = MX ? __reduce_min_sync(0xFFFFFFFFu, key_low) + 1 : 0;
        // (scores of keys without values, vtop 0, do not bind the values' weights either)
        const bool refer = MX && (vtop > vref + 8 || vlow < vref - 19 || vtop == 0), first = vref < 0 && vhigh == 0;
        vhigh = max(vhigh, vtop);
        wide = MX && (vtop - vlow > 19 || (refer && vhigh - vtop > 60));         // sums in units of so much less than their values could overflow
        if (__builtin_expect(MX && refer && !wide && !first, false)) {
          // Far larger values may matter with weights that are lost as FP16 numbers under a base that follows the scores alone. It goes down,
          // to where theirs start at 2^6, as long as the sums of products so far stay below 2^21 in the new unit (what they hold is
          // not outweighed then) and the sum of weights below 2^101.
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              float sums = 0.0f, weights = a.l[n][c];
#pragma unroll
              for (int i = 0; i < MT; ++i) sums = fmaxf(sums, fmaxf(fabsf(a.o[i][n][c]), fabsf(a.o[i][n][c + 2])));
#pragma unroll
              for (int d = 4; d < 32; d *= 2) {
                sums = fmaxf(sums, __shfl_xor_sync(0xFFFFFFFFu, sums, d));
                weights += __shfl_xor_sync(0xFFFFFFFFu, weights, d);
              }
              const int sums_log = max(static_cast<int>(__float_as_uint(sums) >> 23) - 127, -80), weights_log = max(static_cast<int>(__float_as_uint(weights) >> 23) - 127, 0);
              float down = fminf(fmaxf(ve[n][c] - static_cast<float>(vtop - 132 + 20 - sums_log), static_cast<float>(weights_log - 100)), 0.0f);
              down = a.m[n][c] + down - a.m[n][c];             // as far as the base can follow
              a.m[n][c] += down;
              a.l[n][c] *= exp2_approx(-down);
              ve[n][c] -= down;                                // (the sums follow with their new unit)
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float most = top[n][c];
#pragma unroll
            for (int d = 4; d < 32; d *= 2) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
            const float now = fmaxf(a.m[n][c], most - kWeightTop);
            was[n][c] = a.m[n][c] - now;
            a.m[n][c] = now;
            a.l[n][c] *= exp2_approx(was[n][c]);
          }
        if constexpr (MX) {
          if (wide) {
            // A key's value codes relative to its own largest one, exact over 36 binades, with that one's power of two in the weight: the
            // weights of the value product are kept in FP16's range by a maximum of their own.
            const float key_up = static_cast<float>(key_top - 140);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                float most = -INFINITY;
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                  for (int r = 0; r < 2; ++r)
                    most = fmaxf(most, s[half][n][2 * r + c] - a.m[n][c] + __shfl_sync(0xFFFFFFFFu, key_up, half * 16 + r * 8 + own0));
#pragma unroll
                for (int d = 4; d < 32; d *= 2) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
                const float so_far = ve[n][c] + was[n][c];
                ve[n][c] = fmaxf(so_far, most - kWeightTop);
                was[n][c] = so_far - ve[n][c];
              }
            vref = -100;
          } else if (refer) {
            vref = vtop;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                was[n][c] += ve[n][c] - static_cast<float>(vtop - 132);
                ve[n][c] = static_cast<float>(vtop - 132);
              }
          }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const float f = exp2_approx(was[n][c]);
#pragma unroll
            for (int i = 0; i < MT; ++i) { a.o[i][n][c] *= f; a.o[i][n][c + 2] *= f; }
          }
      }

      // weights, as fragments of the value product
      uint32_t pf[2][NT][2];
      if (MX && wide) {
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const float up = __shfl_sync(0xFFFFFFFFu, static_cast<float>(key_top - 140), half * 16 + r * 8 + own0);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const float x0 = s[half][n][2 * r] - a.m[n][0], x1 = s[half][n][2 * r + 1] - a.m[n][1];
              a.l[n][0] += exp2_approx(x0);
              a.l[n][1] += exp2_approx(x1);
              pf[half][n][r] = transpose8x8(f16x2(exp2_approx(x0 + up - ve[n][0]), exp2_approx(x1 + up - ve[n][1])));
            }
          }
        // multipliers, a key per lane, in pairs of a key and the last, second last, ... of its group of eight
        const bool low = (lane & 4) == 0;
        const uint32_t vto = vmul + ((lane >> 3) * 4 + (low ? lane & 3 : 3 - (lane & 3))) * NB * 4;
#pragma unroll
        for (int i = 0; i < NB / 2; ++i) {
          const uint32_t two = NB == 2 ? __byte_perm(vword[0], 0, 0x4420) : vword[i / 2] >> (16 * (i & 1));
          const int c0 = two & 0xFF, c1 = (two >> 8) & 0xFF;
          const uint32_t own = f16x2(__uint_as_float(static_cast<uint32_t>(max(c0 - key_top + 140, 0)) << 23), __uint_as_float(static_cast<uint32_t>(max(c1 - key_top + 140, 0)) << 23));
          const uint32_t got = __shfl_xor_sync(0xFFFFFFFFu, own, 7);
          if (low) smem_store(vto + 8 * i, make_uint2(__byte_perm(own, got, 0x5410), __byte_perm(own, got, 0x7632)));
        }
        __syncwarp();
      } else {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const float2 m2 = make_float2(-a.m[n][0], -a.m[n][1]);
          float2 l2 = make_float2(a.l[n][0], a.l[n][1]);
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const float2 x = __fadd2_rn(make_float2(s[half][n][2 * r], s[half][n][2 * r + 1]), m2);
              const float2 e = make_float2(exp2_approx(x.x), exp2_approx(x.y));
              l2 = __fadd2_rn(l2, e);
              pf[half][n][r] = transpose8x8(f16x2(e.x, e.y));
            }
          a.l[n][0] = l2.x;
          a.l[n][1] = l2.y;
        }
      }

      // values
#pragma unroll
      for (int hh = 0; hh < HALVES; ++hh) {
        uint32_t y[2][2];                                      // multipliers of the lane's block, for the pairs of keys t and 7 - t
        const int block = FMT == QF_FMT_NVFP4 ? (D == 64 ? g >> 1 : hh * 8 + g) : (D == 64 ? g >> 2 : hh * 4 + (g >> 1));
        if (MX && wide) {
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int r = 0; r < 2; ++r) y[half][r] = smem_load<uint32_t>(vmul + (((half * 2 + r) * 4 + t) * NB + block) * 4);
        } else {
          const uint32_t up = (static_cast<uint32_t>(20 - vref) & 0xFFFFu) * 0x10001u;
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const uint32_t first = smem_load<uint8_t>(here + vs_at[0] + (half * 16 + r * 8) * NB + hh * (128 / S::BLOCK));
              const uint32_t second = smem_load<uint8_t>(here + vs_at[1] + (half * 16 + r * 8) * NB + hh * (128 / S::BLOCK));
              if constexpr (MX) y[half][r] = __viaddmax_s16x2_relu(__byte_perm(first, second, 0x5410), up, 0) << 10;
              else y[half][r] = e4m3_pair(first, second);
            }
        }
        if (key0 + kUnitKeys > w.keys) {                       // what stands behind the last key
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const int key = key0 + half * 16 + r * 8;
              y[half][r] &= (key + t < w.keys ? 0xFFFFu : 0u) | (key + 7 - t < w.keys ? 0xFFFF0000u : 0u);
            }
        }
        uint32_t c[2][4][VWORDS];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t words = here + (hh == 0 ? v_at[k & 1] : v_at[k & 1] ^ 64) + (half * 16 + (k >> 1) * 8) * (D / 2);
            if constexpr (D == 64) {
              c[half][k][0] = smem_load<uint32_t>(words);
            } else {
              const uint2 v = smem_load<uint2>(words);
              c[half][k][0] = v.x;
              c[half][k][1] = v.y;
            }
          }
#pragma unroll
        for (int x = 0; x < VWORDS; ++x) {
          uint32_t d[2][4][4];                                 // [half][even / odd dimensions of the two pairs][tile]
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const uint32_t p0 = c[half][2 * r][x], p1 = c[half][2 * r + 1][x];
              e2m1_f16((p0 & 0x0F0F0F0Fu) | ((p1 << 4) & 0xF0F0F0F0u), d[half][2 * r]);
              e2m1_f16(((p0 >> 4) & 0x0F0F0F0Fu) | (p1 & 0xF0F0F0F0u), d[half][2 * r + 1]);
#pragma unroll
              for (int i = 0; i < 4; ++i) { d[half][2 * r][i] = hmul2(d[half][2 * r][i], y[half][r]); d[half][2 * r + 1][i] = hmul2(d[half][2 * r + 1][i], y[half][r]); }
            }
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
              mma(z, d[0][0][i], d[0][1][i], d[0][2][i], d[0][3][i], pf[0][n][0], pf[0][n][1]);
              mma(z, d[1][0][i], d[1][1][i], d[1][2][i], d[1][3][i], pf[1][n][0], pf[1][n][1]);
              float (&o)[4] = a.o[hh * 8 + x * 4 + i][n];
              const float2 lo = __fadd2_rn(make_float2(o[0], o[1]), make_float2(z[0], z[1])), hi = __fadd2_rn(make_float2(o[2], o[3]), make_float2(z[2], z[3]));
              o[0] = lo.x; o[1] = lo.y; o[2] = hi.x; o[3] = hi.y;
            }
        }
      }
      __syncwarp();
    }

    next = w;
    if constexpr (!DIRECT) next.next(p);
    if constexpr (!DIRECT) fetch(next);                                               // on the way while this piece's parts meet
    if (QS && !alone) __syncthreads();                         // the queries have been read
    // One result of the piece: sums of a column's weights over the lanes, then warps 2 and 3 to 0 and 1, then 1 to 0.
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int d = 4; d < 32; d *= 2) a.l[n][c] += __shfl_xor_sync(0xFFFFFFFFu, a.l[n][c], d);
        if constexpr (MX) {
          float moved;
          const float even = even_out(a.m[n][c], a.l[n][c], moved);
          a.l[n][c] *= even;
          const float f = exp2_approx(0.5f * (ve[n][c] - moved));        // twice: the power itself may be out of FP32's range where the product is not
#pragma unroll
          for (int i = 0; i < MT; ++i) { a.o[i][n][c] = a.o[i][n][c] * f * f; a.o[i][n][c + 2] = a.o[i][n][c + 2] * f * f; }
        }
      }
#pragma unroll
    for (int d = kAttnWarps / 2; d > 0; d /= 2) {
      if (alone) break;
      if (warp >= d && warp < 2 * d) {
        const uint32_t at = parts + (warp - d) * S::PART + lane * 16;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int n = 0; n < NT; ++n)
            smem_store(at + (i * NT + n) * 512, make_float4(a.o[i][n][0], a.o[i][n][1], a.o[i][n][2], a.o[i][n][3]));
#pragma unroll
        for (int n = 0; n < NT; ++n)
          smem_store(at + (MT * NT + n) * 512, make_float4(a.m[n][0], a.l[n][0], a.m[n][1], a.l[n][1]));
      }
      __syncthreads();
      if (warp < d) {
        const uint32_t at = parts + warp * S::PART + lane * 16;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const float4 v = smem_load<float4>(at + (MT * NT + n) * 512);
          float fa[2], fb[2];
          join_weights<MX>(a.m[n][0], a.l[n][0], v.x, v.y, fa[0], fb[0]);
          join_weights<MX>(a.m[n][1], a.l[n][1], v.z, v.w, fa[1], fb[1]);
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            const float4 o = smem_load<float4>(at + (i * NT + n) * 512);
            a.o[i][n][0] = a.o[i][n][0] * fa[0] + o.x * fb[0];
            a.o[i][n][1] = a.o[i][n][1] * fa[1] + o.y * fb[1];
            a.o[i][n][2] = a.o[i][n][2] * fa[0] + o.z * fb[0];
            a.o[i][n][3] = a.o[i][n][3] * fa[1] + o.w * fb[1];
          }
        }
      }
      __syncthreads();
    }
    if (DIRECT && p.split > 1) {
      // the cluster's CTAs put their sums into shared memory, and take turns at the value tiles
      constexpr int TILES = MT * NT;
      if (warp == 0) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int n = 0; n < NT; ++n) smem_store(parts + lane * 16 + (i * NT + n) * 512, make_float4(a.o[i][n][0], a.o[i][n][1], a.o[i][n][2], a.o[i][n][3]));
#pragma unroll
        for (int n = 0; n < NT; ++n) smem_store(parts + lane * 16 + (TILES + n) * 512, make_float4(a.m[n][0], a.l[n][0], a.m[n][1], a.l[n][1]));
      }
      const cg::cluster_group cluster = cg::this_cluster();
      cluster.sync();
      for (int tile = static_cast<int>(cluster.block_rank()) * kAttnWarps + warp; tile < TILES; tile += p.split * kAttnWarps) {
        Joint<MX> sum;
        for (int k = 0; k < p.split; ++k) {
          const float4* part = cluster.map_shared_rank(reinterpret_cast<const float4*>(smem + parts), k) + lane;
          sum.add(part[tile * 32], part[(TILES + tile % NT) * 32]);
        }
        write_tile<D, NT>(p, sum, w.b, w.s, tile, lane, vt);
      }
      cluster.sync();
    } else if (warp == 0 || alone) {
      const bool begins = w.j == 0;
      if (DIRECT || w.n == w.units) {                          // the whole sequence: the result itself
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int row = row0 + 8 * n + 2 * t + c;
            if (row < p.rows) {
              const int token = token_of(p, row), head = h * p.group + (row - token * p.group);
              const int64_t at = (static_cast<int64_t>(w.b) * p.q_len + token) * p.q_heads + head;
              const float f = part_factor<MX>(vt, a.l[n][c]);
              uint32_t* out = reinterpret_cast<uint32_t*>(p.out + at * D);
#pragma unroll
              for (int i = 0; i < MT; i += 4)
                *reinterpret_cast<uint4*>(out + dim_of<D>(i, g) / 2) =
                    make_uint4(pack_bf16x2(a.o[i][n][c] * f, a.o[i][n][c + 2] * f), pack_bf16x2(a.o[i + 1][n][c] * f, a.o[i + 1][n][c + 2] * f),
                               pack_bf16x2(a.o[i + 2][n][c] * f, a.o[i + 2][n][c + 2] * f), pack_bf16x2(a.o[i + 3][n][c] * f, a.o[i + 3][n][c + 2] * f));
              if (p.lse && g == 0) p.lse[at] = log_sum(a.m[n][c], a.l[n][c]);
            }
          }
      } else {
        float4* to_part = parts_of(p, gridDim.x) + static_cast<int64_t>(cta * 2 + (begins ? 1 : 0)) * (S::PART / 16) + lane;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int n = 0; n < NT; ++n) to_part[(i * NT + n) * 32] = make_float4(a.o[i][n][0], a.o[i][n][1], a.o[i][n][2], a.o[i][n][3]);
#pragma unroll
        for (int n = 0; n < NT; ++n) to_part[(MT * NT + n) * 32] = make_float4(a.m[n][0], a.l[n][0], a.m[n][1], a.l[n][1]);
      }
      if (!DIRECT && begins && lane == 0 && (p.by_segment || w.n < w.units)) {
        const int64_t last = u1 + (w.units - w.n) - 1;         // place of the sequence's last unit, if others go on with it
        const int64_t wider = (total - share * ctas) * (share + 1);            // end of the shares with a place more
        const int more = w.n < w.units ? static_cast<int>(last < wider ? last / (share + 1) : (last - wider) / share + (total - share * ctas)) - cta : 0;
        tasks[p.by_segment ? w.b * p.segs + w.s : cta] = JoinTask{cta, more, w.b, w.s};
      }
    }
    if constexpr (DIRECT) return;
  }
}

// Joins the parts of sequences that several CTAs shared. A task's value tiles go to the warps of gridDim.y CTAs, one after the
// other; or, where there are many parts, a tile at a time to a CTA whose warps share them. In a fixed order either way.
template <int FMT, int D, int NT>
__global__ void __launch_bounds__(1024) kv_join_kernel(const __grid_constant__ KvAttn p, int ctas) {
  using S = Shape<FMT, D, NT>;
  constexpr int PART4 = S::PART / 16, TILES = S::MT * NT;
  launch_after_previous();
  const float vt = FMT == QF_FMT_NVFP4 ? *p.v_tscale : 1.0f;
  const JoinTask task = reinterpret_cast<const JoinTask*>(p.ws)[blockIdx.x];
  if (task.more == 0) return;
  const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5, lane = threadIdx.x & 31;
  const float4* parts = parts_of(p, ctas) + static_cast<int64_t>(task.cta) * 2 * PART4 + lane;
  extern __shared__ __align__(128) uint8_t smem[];
  float4* met = reinterpret_cast<float4*>(smem);               // sums and weights of a warp, from the second half of the warps
  const bool many = task.more >= 8;
  const int first = many ? warp : 0, step = many ? warps : 1;
  for (int tile = many ? blockIdx.y : blockIdx.y * warps + warp; tile < TILES; tile += gridDim.y * (many ? 1 : warps)) {
    Joint<FMT == QF_FMT_MXFP4> sum;
    for (int k0 = first; k0 <= task.more; k0 += 4 * step) {    // four parts on the way together
      float4 v[4], w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = min(k0 + j * step, task.more);
        const float4* part = parts + static_cast<int64_t>(2 * k + (k == 0 ? 1 : 0)) * PART4;
        v[j] = part[tile * 32];
        w[j] = part[(TILES + tile % NT) * 32];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (k0 + j * step <= task.more) sum.add(v[j], w[j]);
    }
    if (many) {
      for (int d = warps / 2; d > 0; d /= 2) {
        if (warp >= d && warp < 2 * d) {
          met[(warp - d) * 64 + lane] = sum.o;
          met[(warp - d) * 64 + 32 + lane] = sum.ml;
        }
        __syncthreads();
        if (warp < d) sum.add(met[warp * 64 + lane], met[warp * 64 + 32 + lane]);
        __syncthreads();
      }
      if (warp != 0) continue;
    }
    write_tile<D, NT>(p, sum, task.b, task.seg, tile, lane, vt);
  }
}

template <int FMT, int D, int NT, bool DIRECT>
cudaError_t launch_attention(const KvAttn& p, int64_t ctas, int cluster, cudaStream_t st) {
  using S = Shape<FMT, D, NT>;
  static bool ready[64] = {};                                  // the attribute stays set for the process
  int dev = 0;
  if (cudaError_t e = cudaGetDevice(&dev)) return e;
  if (dev >= 64 || !ready[dev]) {
    if (cudaError_t e = cudaFuncSetAttribute(kv_attention_kernel<FMT, D, NT, DIRECT>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM)) return e;
    if (dev < 64) ready[dev] = true;
  }
  return launch_overlapping(kv_attention_kernel<FMT, D, NT, DIRECT>, dim3(static_cast<unsigned>(ctas)), kAttnWarps * 32, S::SMEM, st, cluster, p);
}

// How the work is cut: CTAs of the attention kernel; tasks of the second one, 0 without it. Sets p.split and p.by_segment.
struct AttnCut {
  bool direct;
  int64_t ctas;
  int tasks;
};
template <int FMT, int D, int NT>
AttnCut cut_attention(KvAttn& p) {
  using S = Shape<FMT, D, NT>;
  constexpr int64_t ROOM = kNumSMs * S::CTAS;
  const int64_t segments = static_cast<int64_t>(p.batch) * p.segs;
  const int units = (p.max_keys + kUnitKeys - 1) / kUnitKeys;
  // Many short sequences, by what the page table holds: a warp each. A CTA each would be several rounds of CTAs, each with a start and
  // a meeting for a few units a warp, and equal shares have those to count and to pay for too (heads of 128, ragged: 3200 segments of up to 8
  // keys 27.3 us with CTAs, 8.4 with warps; of up to 380 43.2 and 32.1; 8000 of up to 1500 218 with shares, 198 with warps; but 720 of up to 240
  // 11.3 with CTAs, 12.9 with warps, whose units then take longer than a second round). At most 64, for the one long sequence among short ones.
  if (segments > ROOM && units <= kAloneMost && units * ROOM <= kAloneUnits * segments && segments <= INT32_MAX) {
    p.split = 0;
    return {true, (segments + kAttnWarps - 1) / kAttnWarps, 0};
  }
  // Short sequences: CTAs of their own for each, so that nothing has to be counted, nor joined by a second
  // kernel. As many as there is room for and as have a unit for every warp.
  p.split = 1;
  while (p.split < 8 && p.split * kAttnWarps < units && 2 * p.split * segments <= ROOM) p.split *= 2;
  if (p.split * kDirectUnits >= units && segments <= INT32_MAX) return {true, segments * p.split, 0};
  // no more CTAs than there can be work for
  const int64_t most = segments * (units + kPieceCost) / kAttnWarps + 1;
  const int grid = static_cast<int>(most < ROOM ? most : ROOM);
  p.by_segment = segments <= grid;
  return {false, grid, p.by_segment ? static_cast<int>(segments) : grid};
}

template <int FMT, int D, int NT>
cudaError_t attend(KvAttn& p, cudaStream_t st, int* told) {
  using S = Shape<FMT, D, NT>;
  const AttnCut cut = cut_attention<FMT, D, NT>(p);
  if (told) {
    const int all[5] = {NT, cut.direct ? p.split : -1, static_cast<int>(cut.ctas), cut.tasks, p.by_segment};
    for (int i = 0; i < 5; ++i) told[i] = all[i];
    return cudaSuccess;
  }
  if (cut.direct) return launch_attention<FMT, D, NT, true>(p, cut.ctas, p.split > 1 ? p.split : 1, st);
  if (cudaError_t e = launch_attention<FMT, D, NT, false>(p, cut.ctas, 1, st)) return e;
  // the fewer sequences, the more parts each may have: up to a CTA per value tile
  const int grid = static_cast<int>(cut.ctas), share = 4 * kNumSMs / cut.tasks, parts = grid / cut.tasks, threads = parts < 32 ? 256 : parts < 128 ? 512 : 1024;
  return launch_overlapping(kv_join_kernel<FMT, D, NT>, dim3(cut.tasks, share < 1 ? 1 : share < S::MT * NT ? share : S::MT * NT), threads, threads * 16, st, 1, p, grid);
}

// Query rows of a tile, in units of 8, at most: what registers hold next to the decoded words. (Heads of 256 with 16 rows: only with the
// queries in shared memory, 50 us for 12 rows of 4 heads over 32 sequences of 4096 keys where two tiles of 8 rows take 62.)
constexpr int tile_most(int head_dim) { return head_dim == 64 ? 4 : head_dim == 128 ? 3 : 2; }

// The cache is decoded once per tile, which costs as much as the products of 14 rows (32 sequences of 4096 keys, heads of 128: 38, 52 and
// 66 us for 8, 16 and 24 rows): as few tiles as can be, evenly filled. But where a table holds few keys, smaller tiles give more CTAs a
// part and each less to do after its last key: as long as all tiles' units are no more than about three a warp (4 heads of 128, 40 rows
// each: one sequence of 300 keys 6.1 us instead of 9.1, 7 of them 8.0 instead of 10.4; 7 of 2500 keys 17.4, with tiles of 8 rows 20.0).
constexpr int64_t kTileUnits = 3 * 2 * kNumSMs * kAttnWarps;
template <int FMT>
cudaError_t attend_format(KvAttn& p, int head_dim, cudaStream_t st, int* told) {
  const int eights = (p.rows + 7) / 8, most = tile_most(head_dim);
  const int64_t units = static_cast<int64_t>(p.batch) * p.kv_heads * ((p.max_keys + kUnitKeys - 1) / kUnitKeys);
  int nt = 1;
  while (nt < most && (eights + nt - 1) / nt * units > kTileUnits) ++nt;
  p.tiles = (eights + nt - 1) / nt;
  nt = (eights + p.tiles - 1) / p.tiles;
  p.segs = p.tiles * p.kv_heads;
  if (head_dim == 64) return nt == 1 ? attend<FMT, 64, 1>(p, st, told) : nt == 2 ? attend<FMT, 64, 2>(p, st, told) : nt == 3 ? attend<FMT, 64, 3>(p, st, told) : attend<FMT, 64, 4>(p, st, told);
  if (head_dim == 128) return nt == 1 ? attend<FMT, 128, 1>(p, st, told) : nt == 2 ? attend<FMT, 128, 2>(p, st, told) : attend<FMT, 128, 3>(p, st, told);
  return nt == 1 ? attend<FMT, 256, 1>(p, st, told) : attend<FMT, 256, 2>(p, st, told);
}

// Workspace: for the largest kernel of a head size, whatever the format and the tile, since how the rows are split over sequences is
// not known when it is asked for.
template <int FMT, int D, int NT>
constexpr size_t part_bytes() {
  using S = Shape<FMT, D, NT>;
  return static_cast<size_t>(kNumSMs) * S::CTAS * (sizeof(JoinTask) + 2 * S::PART) + 256;
}
constexpr size_t larger(size_t a, size_t b) { return a > b ? a : b; }
template <int D, int NT>
constexpr size_t ws_bytes() {
  const size_t here = larger(part_bytes<QF_FMT_NVFP4, D, NT>(), part_bytes<QF_FMT_MXFP4, D, NT>());
  if constexpr (NT > 1) return larger(here, ws_bytes<D, NT - 1>());
  else return here;
}

}  // namespace

cudaError_t launch_kv_append(const qf_kv_cache_t& c, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int64_t tokens,
                             const void* slots, bool slots64, bool noclip, cudaStream_t st) {
  KvRows p = kv_rows(c, slots, slots64, tokens);
  p.k = static_cast<const __nv_bfloat16*>(k);
  p.v = static_cast<const __nv_bfloat16*>(v);
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.noclip = noclip;
  return launch_rows(c.fmt == QF_FMT_NVFP4 ? kv_append_kernel<QF_FMT_NVFP4> : kv_append_kernel<QF_FMT_MXFP4>, p, c.head_dim / 16, 2, kAppendTurns, st);
}

cudaError_t launch_kv_read(const qf_kv_cache_t& c, const void* slots, bool slots64, int64_t rows, void* k, void* v, cudaStream_t st) {
  KvRows p = kv_rows(c, slots, slots64, rows);
  p.k_out = static_cast<__nv_bfloat16*>(k);
  p.v_out = static_cast<__nv_bfloat16*>(v);
  return launch_rows(c.fmt == QF_FMT_NVFP4 ? kv_read_kernel<QF_FMT_NVFP4> : kv_read_kernel<QF_FMT_MXFP4>, p, c.head_dim / 8, k && v ? 2 : 1, kReadTurns, st);
}

size_t kv_attention_ws_bytes(int64_t, int, int head_dim, int) {
  return head_dim <= 64 ? ws_bytes<64, tile_most(64)>() : head_dim <= 128 ? ws_bytes<128, tile_most(128)>() : ws_bytes<256, tile_most(256)>();
}

static cudaError_t kv_attention(const KvAttentionArgs& a, cudaStream_t st, int* told) {
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
  p.ws = static_cast<uint8_t*>(a.workspace);
  p.batch = static_cast<int>(a.batch);
  p.pages = static_cast<int>(a.cache.pages);
  p.max_pages = static_cast<int>(a.max_pages);
  p.page_size = a.cache.page_size;
  p.max_keys = static_cast<int>(a.max_pages * a.cache.page_size);
  p.q_len = a.q_len;
  p.q_heads = a.q_heads;
  p.kv_heads = a.cache.kv_heads;
  p.group = a.q_heads / a.cache.kv_heads;
  p.rows = a.q_len * p.group;
  p.scale = a.scale * 1.4426950408889634f;
  p.page_codes = static_cast<int64_t>(p.kv_heads) * p.page_size * (a.cache.head_dim / 2);
  return a.cache.fmt == QF_FMT_NVFP4 ? attend_format<QF_FMT_NVFP4>(p, a.cache.head_dim, st, told) : attend_format<QF_FMT_MXFP4>(p, a.cache.head_dim, st, told);
}

cudaError_t launch_kv_attention(const KvAttentionArgs& a, cudaStream_t st) { return kv_attention(a, st, nullptr); }

void kv_attention_cut(const KvAttentionArgs& a, int* cut) { kv_attention(a, nullptr, cut); }

}  // namespace qf
