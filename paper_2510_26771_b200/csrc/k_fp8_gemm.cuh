// Product of block-scaled e4m3 codes on the 5th-generation tensor cores, with one weight matrix or with the weights of
// one expert per run of rows:
//   y[m, n] = sum_b sx[m, b] sw[n / 128, b] sum_{k in b} x[m, k] w[n, k]  (+ bias[n])
//
// The power-of-two scales go into the instruction (tcgen05.mma kind::mxf8f6f4.block_scale): the sum runs over all of K
// in one fp32 accumulator and nothing has to be drained and scaled per block.  The instruction takes a scale for every 32
// features; a block of 128 uses the same byte of the scale words for its four instructions, so 512 features need one
// 32-bit word per row, four blocks' bytes.
//
// Operand roles as in k_gemm.cuh: 128 output channels are the MMA A operand (TMEM lanes), tokens the B operand
// (columns).  The extent in tokens is a field of the instruction, in steps of 16: a tile with few rows -- a decode
// step, the end of an expert's run -- costs what its rows cost, and no expert's rows have to be padded.
//
//   warp 0     TMA producer: 128-byte-swizzled K-major tiles of both operands into a ring of 6 to 10 stages
//   warp 1     allocates TMEM; one elected thread copies the scale words to TMEM (tcgen05.cp) and issues the MMAs
//   warps 2-3  scale producers: gather the scale words of 512 features of the tile's tokens and channels into the
//              order tcgen05.cp wants (row i of 32: rows i, i + 32, i + 64, i + 96), up to FP8G_SF_SLOTS steps ahead
//   warps 4-11 (GROUPS = 4: 4-19) epilogue: drain the finished accumulator while the next tile fills the other
// Every wait is bounded; when one expires the CTA raises the device status word, unwinds and frees its TMEM.
//
// PAIR = false: tiles of 128 channels x up to 128 tokens, one CTA each.  For few tiles the sum can be split over a
// cluster of 2, 4 or 8 CTAs (parameter `split`; one tile per cluster): each leaves its partial tile in its own shared
// memory, and each adds up a share of the tokens over all of them in rank order -- no atomics, a fixed order.
// PAIR = true: CTA pairs (cta_group::2), tiles of 256 channels x up to 256 tokens.  Two accumulators of 256 columns and
// the scales do not fit the 512 columns: the accumulators overlap in 32 columns, which the epilogue drains first; the
// next tile starts when they are free.
//
// What bounds it: large products the power limit (16384 x 14336 x 4096: 754 us = 2552 TFLOP/s at 990 W and about 1.1 GHz;
// without it, at 1.9 GHz, shared memory and the tensor pipe together, 537 clocks per 128 features of a 256 x 256 pair
// against the pipe's 512); few rows the issue and copy loops of the CTAs that have a tile, where tiles are fewer than SMs (1 x 4096 x
// 11008: 86 tiles of 32 steps at 330 clocks, 5.6 us, behind 3.2 of a launch with nothing to do: 10.0 us against 6.9 at the
// copy rate, with 62 SMs idle), else the weights' way from memory (320 rows over 64 experts of 2048 x 4096: 75 against 71).
// An fp32 output of more than 4096 features is read and written again for every further 4096: 16384 x 14336 x 4096 in 803 to
// 867 us where one accumulator would take 735.
#pragma once
#include "common.cuh"
#include "k_fp8_quant.cuh"
#include "ptx.cuh"

namespace stamp {

constexpr int FP8_MAX_EXPERTS = 1024;
constexpr int FP8G_BM = 128, FP8G_BK = 128;
constexpr int FP8G_RING_BYTES = 208 * 1024;            // operand stages: 6 of 128 token rows ... 10 of 32
constexpr int FP8G_MAX_STAGES = 10;
constexpr int FP8G_ACC_COLS = 128;                     // tensor-memory columns of a tile of one CTA
constexpr int FP8G_W_BYTES = FP8G_BM * FP8G_BK;
constexpr int FP8G_SF_SLOTS = 4;                       // steps of 512 features whose scale words are staged
constexpr int FP8G_TAIL_BOX = 32;
constexpr int FP8G_PART = FP8G_BM + 4;                 // FUSED: floats from one token to the next in a part of a split sum
constexpr int FP8G_MOST_GROUPS = 4;                    // epilogue warps come in groups of four, one for each quarter of the lanes
constexpr long long FP8G_WAIT_LIMIT = 4000000000LL;    // SM clocks (~2 s) before a wait gives up

struct Fp8GemmParams {
  const uint8_t* x;        // [M, K]
  const uint8_t* x_scale;  // [M, ks]
  const int* offsets;      // [E + 1] first row of every expert, or nullptr: one matrix for all rows
  const uint8_t* w;        // [E, N, K]
  const uint8_t* w_scale;  // [E, ceil(N / 128), ks]
  const float* bias;       // [E, N] or nullptr
  void* y;                 // [M, N] float or bf16
  int M, N, K, E, ks;
  int x_words;             // x_scale rows start on 4-byte boundaries
  int bn;                  // token rows of a tile: a multiple of 16, at most 128 (PAIR: 256)
  int stages, stage_bytes; // operand ring: 128 channels and the token rows that one CTA stages (bn; PAIR: bn / 2)
  int tail;                // tiles of up to this many staged rows (the ends of runs) are copied 32 rows at a time; 0: none
  int split;               // CTAs that share a tile's sum (PAIR: 1)
  int chunk;               // steps of 512 features that one accumulator sums (fp32 output), else all of them
  int band;                // channel tiles per raster band
  // FUSED only: what follows the sum
  int act;                 // stamp_activation
  const void* residual;    // [M, ldr] float or bf16, or nullptr
  int r_bf16;              // residual is bf16
  int words;               // four neighbouring channels of Y and of the residual are aligned words
  long ldr;
  uint8_t* y_scale;        // quantized output: [M, ceil(N / 128)]
};

template <bool PAIR>
struct Fp8Smem {
  static constexpr int BN = PAIR ? 256 : 128;          // token rows of the largest tile
  static constexpr int SF_SLOT = 512 + BN * 4;         // scale words of 512 features: channels, then tokens
  static constexpr int SF_OFFSET = FP8G_RING_BYTES;
  static constexpr int BAR_OFFSET = SF_OFFSET + FP8G_SF_SLOTS * SF_SLOT;
  static constexpr int NUM_BARS = 2 * FP8G_MAX_STAGES + 2 * FP8G_SF_SLOTS + 4; // full, empty, sffull, sfempty, tfull[2], tempty[2]
  static constexpr int TAB_OFFSET = BAR_OFFSET + NUM_BARS * 8 + 16;
  static constexpr int DYN_BYTES = TAB_OFFSET + 2 * (FP8_MAX_EXPERTS + 1) * 4 + 1024;
  // FUSED, quantized output: a barrier for each group of four epilogue warps, their maxima [group][buffer][quarter][token] and
  // the tokens' inverse scales [warp][token]
  static constexpr int EX_OFFSET = (TAB_OFFSET + 2 * 2 * 4 + 15) / 16 * 16;   // (one matrix: two entries of either table)
  static constexpr int EX_BYTES = FP8G_MOST_GROUPS * (8 + 2 * 4 * 32 * 4 + 4 * 32 * 4);
  static constexpr int FUSED_DYN_BYTES = EX_OFFSET + EX_BYTES + 1024;
  static_assert(DYN_BYTES <= 227 * 1024 && FUSED_DYN_BYTES <= 227 * 1024, "shared memory of one CTA");
  // tensor memory: second accumulator, then the two buffers of scale columns (4 for channels, BN / 32 for tokens)
  static constexpr int ACC1 = PAIR ? 224 : FP8G_ACC_COLS;
  static constexpr int SF_COL = PAIR ? 480 : 2 * FP8G_ACC_COLS;
  static constexpr int SF_COLS = 4 + BN / 32;
};

// One unit of work: up to BN rows of one expert's run times 128 (PAIR: 256) output channels.
struct Fp8Tile {
  int expert, ch_tile, row0, rows, n;   // n: rows rounded up to what an instruction takes
};
// Bands of `band` channel tiles; inside one, channel tiles vary fastest: CTAs running at the same time share token tiles,
// and the band's weights stay in L2 over an expert's token tiles.
__device__ __forceinline__ void fp8_raster(int tile, int band, int ch_tiles, int tok_tiles, int& ch_tile, int& tok_tile) {
  const int per_band = band * tok_tiles;
  const int b = tile / per_band, rem = tile - b * per_band;
  const int first = b * band, height = min(band, ch_tiles - first);
  tok_tile = rem / height;
  ch_tile = first + (rem - tok_tile * height);
}
__device__ __forceinline__ Fp8Tile fp8_tile(const Fp8GemmParams& p, const int* tile_start, const int* row_start, int experts, int tile,
                                            int ch_tiles, int tok_tiles) {
  Fp8Tile t;
  int tt;
  fp8_raster(tile, p.band, ch_tiles, tok_tiles, t.ch_tile, tt);
  int lo = 0, hi = experts;             // the expert whose tiles hold tt (empty runs have none)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (tile_start[mid] <= tt) lo = mid; else hi = mid;
  }
  t.expert = lo;
  t.row0 = row_start[lo] + (tt - tile_start[lo]) * p.bn;
  t.rows = min(p.bn, row_start[lo + 1] - t.row0);
  t.n = (t.rows + 15) & ~15;
  return t;
}

// FUSED: whether the block of 128 channels from `first` on keeps its order: it ends inside a run of 32 channels, or four
// channels of the output or the residual are no aligned word.
__device__ __forceinline__ bool fp8_plain_order(const Fp8GemmParams& p, int first) { return !p.words || ((p.N & 31) != 0 && first + FP8G_BM > p.N); }

// The scale bytes of `n` (1..4) consecutive blocks as one word.  Where there is none -- blocks past K, rows past the
// run, whose columns are not stored -- any finite scale does: 1.
__device__ __forceinline__ uint32_t fp8_scale_word(const uint8_t* ptr, int n, bool live) {
  uint32_t b[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) b[i] = (live && i < n) ? __ldg(ptr + i) : 0x7Fu;
  return b[0] | (b[1] << 8) | (b[2] << 16) | (b[3] << 24);
}

// The order in which the groups of epilogue warps (two, the plain form's halves, or four) drain an accumulator: chunks of 32
// columns, chunk c by group c % groups whichever accumulator it is.  A sum in several parts is added up in the output, accumulator
// after accumulator, and nothing orders the groups among each other: a chunk has to stay with one of them.  PAIR: the chunk whose
// columns the accumulators share, the eighth of the first and the first of the second, comes first; who has none of it hands the
// accumulator back at once.
__host__ __device__ constexpr int fp8_drain_chunks(int chunks, int group, int groups) { return (chunks - group + groups - 1) / groups; }
__host__ __device__ constexpr int fp8_drain_chunk(bool descending, int group, int i, int count, int groups) {
  return group + groups * (descending ? count - 1 - i : i);
}
__host__ __device__ constexpr int fp8_overlap_group(int accumulator, int groups) { return accumulator == 0 ? 7 % groups : 0; }
constexpr bool fp8_drain_order_holds(int groups) {
  for (int chunks = 1; chunks <= 8; ++chunks)
    for (int a = 0; a < 2; ++a) {
      unsigned taken = 0;
      for (int group = 0; group < groups; ++group) {
        const int count = fp8_drain_chunks(chunks, group, groups);
        for (int i = 0; i < count; ++i) {
          const int c = fp8_drain_chunk(a == 0, group, i, count, groups);
          if (c % groups != group || c < 0 || c >= chunks || (taken >> c & 1u) != 0u) return false;
          if (c == (a == 0 ? 7 : 0) && (group != fp8_overlap_group(a, groups) || i != 0)) return false;
          taken |= 1u << c;
        }
      }
      if (taken != (1u << chunks) - 1u) return false;
    }
  return true;
}
static_assert(fp8_drain_order_holds(2) && fp8_drain_order_holds(4), "every chunk once, by the same group in both accumulators, the shared columns first");

// Two adjacent channels of one token.
__device__ __forceinline__ void fp8_store2(float* y, float a, float b, bool both, bool vec) {
  if (vec && both) {
    *reinterpret_cast<float2*>(y) = make_float2(a, b);
  } else {
    y[0] = a;
    if (both) y[1] = b;
  }
}
__device__ __forceinline__ void fp8_store2(__nv_bfloat16* y, float a, float b, bool both, bool vec) {
  if (vec && both) {
    *reinterpret_cast<__nv_bfloat162*>(y) = __floats2bfloat162_rn(a, b);
  } else {
    y[0] = __float2bfloat16_rn(a);
    if (both) y[1] = __float2bfloat16_rn(b);
  }
}

// ---- what follows the sum in the fused form: activation, residual, quantization
// The activation of two sums at once, in packed fp32; two values of the special function unit for each.
//   LINEAR     none, or relu where `floor` is 0 instead of -inf (a NaN stays one).
//   SILU       v / (1 + exp(-v)): the exponent's product is held as head and tail, as in the gated quantizer; divisor and v are
//              both divided by four, since the reciprocal of a divisor from 2^126 on would be flushed to zero.  About 3 ulp.
//   GELU_TANH  (1 + tanh(u)) / 2 = 1 / (1 + exp(-2 u)), which does not cancel where tanh is near -1; 2 u is rounded three times, so
//              that the result is within about (5 |2 u| + 18) 2^-24 of itself.
//   GELU       v Phi(v), Phi(-x) = exp(-x^2 / 2) R(x) for x >= 0 (1 + erf would cancel in the lower tail).  R(x), half the scaled
//              complementary error function of x / sqrt 2, is t P(1 - 2 t) with t = 1 / (1 + x / 3): a least-squares fit of
//              degree 8, reweighted towards the smallest largest relative error (2^-23.3 for x <= 14, where exp(-x^2 / 2)
//              vanishes, with the coefficients rounded to fp32).  In fp32, a reciprocal off by an ulp included, R is within 2^-21; all in all 2^-20.
// An infinite sum comes out non-finite.
enum Fp8Act { FP8_LINEAR, FP8_GELU, FP8_GELU_TANH, FP8_SILU };
template <int ACT>
__device__ __forceinline__ float2 fp8_activate2(float2 v, float floor) {
  auto both = [](float x) { return make_float2(x, x); };
  if constexpr (ACT == FP8_GELU) {
    constexpr float P[9] = {0.243027896f, -0.169777423f, 0.0766731128f, -0.0157520343f, -0.00349331181f, 0.00230797403f, 0.000358678924f, -0.000301084074f, -8.89220537e-05f};
    constexpr float C = -0.721347520f, C_TAIL = -9.62981495e-9f, LN2 = 0.693147181f;   // -log2(e) / 2 and the rest of it
    const float2 x = make_float2(fminf(fabsf(v.x), 20.f), fminf(fabsf(v.y), 20.f));
    const float2 d = __ffma2_rn(x, both(1.f / 3.f), both(1.f));
    const float2 t = make_float2(ptx::rcp(d.x), ptx::rcp(d.y));
    const float2 u = __ffma2_rn(t, both(-2.f), both(1.f));
    float2 r = both(P[8]);
#pragma unroll
    for (int i = 7; i >= 0; --i) r = __ffma2_rn(r, u, both(P[i]));
    // exp(-x^2 / 2) = 2^head (1 + more)
    const float2 square = __fmul2_rn(x, x), rest = __ffma2_rn(x, x, __fmul2_rn(square, both(-1.f)));
    const float2 head = __fmul2_rn(square, both(C));
    float2 more = __ffma2_rn(square, both(C), __fmul2_rn(head, both(-1.f)));
    more = __ffma2_rn(rest, both(C), __ffma2_rn(square, both(C_TAIL), more));
    const float2 q = __fmul2_rn(__fmul2_rn(r, t), make_float2(ptx::ex2(head.x), ptx::ex2(head.y)));
    const float2 w = __fmul2_rn(v, __ffma2_rn(q, __fmul2_rn(more, both(LN2)), q));
    return make_float2(v.x > 0.f ? v.x - w.x : w.x, v.y > 0.f ? v.y - w.y : w.y);
  } else if constexpr (ACT == FP8_GELU_TANH) {
    constexpr float C = 1.5957691216f * 1.4426950409f;   // 2 sqrt(2 / pi) log2(e)
    const float2 a = __fmul2_rn(v, __ffma2_rn(__fmul2_rn(v, v), both(-0.044715f * C), both(-C)));
    const float2 d = __fadd2_rn(make_float2(ptx::ex2(a.x), ptx::ex2(a.y)), both(1.f));
    return __fmul2_rn(v, make_float2(ptx::rcp(d.x), ptx::rcp(d.y)));
  } else if constexpr (ACT == FP8_SILU) {
    constexpr float LOG2E = 1.44269504f, LOG2E_TAIL = 1.92596299e-8f, LN2 = 0.693147181f;
    const float2 x = make_float2(fminf(v.x, 90.f), fminf(v.y, 90.f));   // (inf would leave NaN below)
    const float2 head = __fmul2_rn(x, both(-LOG2E));
    const float2 tail = __ffma2_rn(x, both(-LOG2E), __fmul2_rn(head, both(-1.f)));
    const float2 more = __fmul2_rn(__ffma2_rn(x, both(-LOG2E_TAIL), tail), both(0.25f * LN2));
    const float2 p = make_float2(ptx::ex2(head.x), ptx::ex2(head.y));
    const float2 d = __ffma2_rn(p, __fadd2_rn(more, both(0.25f)), both(0.25f));   // (1 + exp(-v)) / 4
    return __fmul2_rn(__fmul2_rn(v, both(0.25f)), make_float2(ptx::rcp(d.x), ptx::rcp(d.y)));
  } else {
    return make_float2(ptx::max_nan(v.x, floor), ptx::max_nan(v.y, floor));
  }
}
// f(variant, floor) for a stamp_activation: one jump around whatever f does.
template <typename F>
__device__ __forceinline__ void fp8_with_activation(int act, F&& f) {
  const float none = -__int_as_float(0x7F800000);
  switch (act) {
    case STAMP_ACT_GELU: f(std::integral_constant<int, FP8_GELU>{}, none); break;
    case STAMP_ACT_GELU_TANH: f(std::integral_constant<int, FP8_GELU_TANH>{}, none); break;
    case STAMP_ACT_SILU: f(std::integral_constant<int, FP8_SILU>{}, none); break;
    default: f(std::integral_constant<int, FP8_LINEAR>{}, act == STAMP_ACT_RELU ? 0.f : none);
  }
}
// Four neighbouring channels of one token, stored as one aligned word.
__device__ __forceinline__ void fp8_store4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void fp8_store4(__nv_bfloat16* p, float4 v) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
__device__ __forceinline__ void fp8_put(float* p, float v) { *p = v; }
__device__ __forceinline__ void fp8_put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
// What a thread's columns are added to, as loaded: converted where it is used, so that no load waits for the one before.  A
// thread's tokens of 8 KU columns are 8 k + e from its first on; rows are `ld` elements apart and those below `left` exist (of
// the others the last one is loaded again; with none at all nothing is).
template <int KU>
__device__ __forceinline__ void fp8_load_tokens(const void* base, long at, long ld, bool bf16, int left, uint4 (&out)[2 * KU]) {
  if (left <= 0) return;
  const int most = left - 1;
  if (bf16) {
    const __nv_bfloat16* const p = static_cast<const __nv_bfloat16*>(base) + at;
#pragma unroll
    for (int j = 0; j < 2 * KU; ++j) {
      const uint2 u = *reinterpret_cast<const uint2*>(p + min((j >> 1) * 8 + (j & 1), most) * ld);
      out[j].x = u.x, out[j].y = u.y;
    }
  } else {
    const float* const p = static_cast<const float*>(base) + at;
#pragma unroll
    for (int j = 0; j < 2 * KU; ++j) out[j] = *reinterpret_cast<const uint4*>(p + min((j >> 1) * 8 + (j & 1), most) * ld);
  }
}
template <int KU>
__device__ __forceinline__ void fp8_add_tokens(const uint4 (&raw)[2 * KU], bool bf16, float (&v)[4][2 * KU]) {
  if (bf16) {
#pragma unroll
    for (int j = 0; j < 2 * KU; ++j) {
      v[0][j] += __uint_as_float(raw[j].x << 16), v[1][j] += __uint_as_float(raw[j].x & 0xFFFF0000u);
      v[2][j] += __uint_as_float(raw[j].y << 16), v[3][j] += __uint_as_float(raw[j].y & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 2 * KU; ++j) {
      v[0][j] += __uint_as_float(raw[j].x), v[1][j] += __uint_as_float(raw[j].y);
      v[2][j] += __uint_as_float(raw[j].z), v[3][j] += __uint_as_float(raw[j].w);
    }
  }
}
template <int KU, typename T>
__device__ __forceinline__ void fp8_store_tokens(T* p, long ld, int left, const float (&v)[4][2 * KU]) {
  T* q = p + ld;
#pragma unroll
  for (int k = 0; k < KU; ++k, p += 8 * ld, q += 8 * ld) {
    if (8 * k < left) fp8_store4(p, make_float4(v[0][2 * k], v[1][2 * k], v[2][2 * k], v[3][2 * k]));
    if (8 * k + 1 < left) fp8_store4(q, make_float4(v[0][2 * k + 1], v[1][2 * k + 1], v[2][2 * k + 1], v[3][2 * k + 1]));
  }
}
// 16 tokens at one channel, likewise; as loaded (bf16: in the upper half once it is used).
template <typename T>
__device__ __forceinline__ void fp8_load_column(const T* p, long ld, int left, uint32_t (&out)[16]) {
  if (left >= 16) {
#pragma unroll
    for (int j = 0; j < 16; ++j, p += ld) out[j] = *p;
  } else if (left > 0) {
    const int most = left - 1;
#pragma unroll
    for (int j = 0; j < 16; ++j) out[j] = p[min(j, most) * ld];
  }
}

// FUSED: y = act(sum + bias) + residual; TOut = uint8_t (FUSED only): the codes of act(sum + bias), the next product's
// operand.  A tile's 128 channels are one block of that operand, so its scale comes from the tile alone: the maximum over
// the lanes of a warp, then over the four warps that hold the block's channels, which exchange it in shared memory.
//
// FUSED reads the accumulator 16 lanes x 8 columns at a time (the 16x256b shape): a thread gets lanes l, l + 8, l + 16 and
// l + 24 of a warp's 32, at eight columns.  The weights' rows are copied in an order that makes these four neighbouring channels
// (a tensor map of four dimensions: channel 32 q + 4 g + c goes to row 32 q + 8 c + g of the tile), so that a thread stores whole
// words -- four channels of a token as 16, 8 or 4 bytes -- with no exchange between lanes, loads the residual likewise, and
// finds most of a token's maximum in its own registers.  With the plain epilogue's shape (a lane a channel, 32 columns), the
// exchange and the predicates of its stores made 16 instructions an output, 24 with gelu and codes: 80 us for 8192 x 1152 x
// 4608 with gelu to codes, two thirds of it the epilogue.
// A last block that ends inside a run of 32 channels, and all blocks where rows are not aligned, keep the plain order and shape:
// a lane a channel, outputs one by one, 32 lanes side by side (1797 x 2688 x 4463 in fp32 with a residual 67 us with the words'
// order and shape, whose four channels are then four stores 16 bytes apart).
//
// Device times, in us, in brackets the plain product's to bf16 or fp32 on the same box: 1 x 4096 x 11008 with bias and silu 11.3
// (10.6), 64 rows 12.2 (11.5), 128 rows 14.5 (13.0); 8192 x 4608 x 1152 with bias and a bf16 residual 42.7 (39.6), the residual's way from memory;
// 8192 x 1152 x 4608 with bias and gelu_tanh to codes 51 (41.3): a tile's nine steps of 128 features are summed before its 256 columns
// are drained, 21 warp instructions for 32 outputs in all, two values of the special function unit each, issue slots 46 % busy;
// 2048 x 4096 x 11008 with silu to codes 71 (69); 16384 x 14336 x 4096 in fp32 with a residual 966 to 990 (930), 870 before the power
// limit sets in.  In a stream of such calls all of the large ones are at that limit, 985 W, at 1.1 to 1.7 GHz.
// Tried: a long fp32 sum's parts added up in 128 registers a thread (960 for 966, but 84 for 76 where rows are
// not aligned: spills); tiles of 224 columns, whose accumulators share none (no difference).
//
// PARTS (codes): a sum of more than one accumulator's.  The fp32 form adds its parts up in the output; codes have no room for them, so a
// thread keeps its own, up to 128 of them, in local memory (128 KB of a CTA, which stay in L2) and quantizes with the last.  2048 x 11008 x
// 4096 102 us, in one accumulator 92; 16384 x 14336 x 4096 833 and 684 (fp32 output 927).
template <bool PAIR, typename TOut, bool FUSED = false, int GROUPS = 2, bool PARTS = false>
__global__ void __launch_bounds__(128 + 128 * GROUPS, 1)
    k_fp8_gemm(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x,
               const __grid_constant__ CUtensorMap tmap_x_tail, Fp8GemmParams p) {
  using SM = Fp8Smem<PAIR>;
  constexpr int BN = SM::BN;
  static_assert(GROUPS == 2 || (FUSED && GROUPS == FP8G_MOST_GROUPS), "groups of epilogue warps");
  static_assert(!PARTS || (FUSED && sizeof(TOut) == 1 && GROUPS == 2), "parts kept by the thread: of codes");
  constexpr int THREADS = 128 + 128 * GROUPS, EPI_WARPS = THREADS / 32 - 4;
  extern __shared__ uint8_t fp8g_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(fp8g_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + SM::BAR_OFFSET);
  uint64_t* empty = full + FP8G_MAX_STAGES;
  uint64_t* sffull = empty + FP8G_MAX_STAGES;
  uint64_t* sfempty = sffull + FP8G_SF_SLOTS;
  uint64_t* tfull = sfempty + FP8G_SF_SLOTS;
  uint64_t* tempty = tfull + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tempty + 2);
  volatile uint32_t* abort_word = tmem_slot + 1;
  int* tile_start = reinterpret_cast<int*>(smem + SM::TAB_OFFSET);
  int* row_start = tile_start + (FUSED ? 1 : FP8_MAX_EXPERTS) + 1;

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const bool clustered = PAIR || p.split > 1;
  const int rank = clustered ? static_cast<int>(ptx::cluster_ctarank()) : 0;
  const int per_tile = PAIR ? 2 : p.split;             // CTAs of a tile
  constexpr int CH_PER_TILE = PAIR ? 2 * FP8G_BM : FP8G_BM;
  const int ch_tiles = (p.N + CH_PER_TILE - 1) / CH_PER_TILE;
  // the part of K this CTA sums, in steps of 512 features (one scale word)
  const int num_kb = (p.K + FP8G_BK - 1) / FP8G_BK;
  const int steps = (num_kb + 3) / 4;
  const int split_rank = PAIR ? 0 : rank;
  const int step0 = steps * split_rank / p.split, step1 = steps * (split_rank + 1) / p.split;
  const int kb0 = step0 * 4, kb1 = min(step1 * 4, num_kb);

  if (threadIdx.x == 0) {
    for (int s = 0; s < FP8G_MAX_STAGES; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < FP8G_SF_SLOTS; ++a) {
      ptx::mbar_init(&sffull[a], PAIR ? 2 : 1);
      ptx::mbar_init(&sfempty[a], 1);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(&tfull[a], 1);
      ptx::mbar_init(&tempty[a], PAIR ? 2 * EPI_WARPS : EPI_WARPS);
    }
    if constexpr (sizeof(TOut) == 1) {
      for (int g = 0; g < GROUPS; ++g) ptx::mbar_init(reinterpret_cast<uint64_t*>(smem + SM::EX_OFFSET) + g, 4);
    }
    *abort_word = 0;
    ptx::fence_mbar_init();
    ptx::prefetch_tensormap(&tmap_w);
    ptx::prefetch_tensormap(&tmap_x);
    if (!FUSED && p.tail) ptx::prefetch_tensormap(&tmap_x_tail);
  }
  if (warp == 1) {
    if constexpr (PAIR) {
      ptx::tmem_alloc_pair(tmem_slot, 512);
      ptx::tmem_relinquish_pair();
    } else {
      ptx::tmem_alloc(tmem_slot, 512);
      ptx::tmem_relinquish();
    }
  }
  // Where every expert's rows and tiles start.  Offsets that are out of order or past the rows: no tile at all.
  if (p.offsets) {
    ptx::grid_dependency_wait();
    bool bad = false;
    for (int e = threadIdx.x; e <= p.E; e += THREADS) {
      const int o = __ldg(p.offsets + e);
      row_start[e] = o;
      bad |= o < 0 || o > p.M || (e == 0 ? o != 0 : o < __ldg(p.offsets + e - 1));
    }
    bad = __syncthreads_or(bad);
    if (bad && threadIdx.x == 0) raise_device_status(STAMP_ERR_INVALID_ARG);
    if (warp == 3) {
      int sum = 0;
      for (int e0 = 0; e0 < p.E; e0 += 32) {
        const int e = e0 + lane;
        int t = (e < p.E && !bad) ? (row_start[e + 1] - row_start[e] + p.bn - 1) / p.bn : 0;
        const int own = t;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int v = __shfl_up_sync(0xffffffffu, t, d);
          if (lane >= d) t += v;
        }
        if (e < p.E) tile_start[e] = sum + t - own;
        sum += __shfl_sync(0xffffffffu, t, 31);
      }
      if (lane == 0) tile_start[p.E] = sum;
    }
  } else if (threadIdx.x == 0) {
    row_start[0] = 0;
    row_start[1] = p.M;
    tile_start[0] = 0;
    tile_start[1] = (p.M + p.bn - 1) / p.bn;
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (clustered) ptx::cluster_sync();   // all barriers of the cluster are initialised before anyone signals another's
  ptx::tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const int tok_tiles = tile_start[p.E];
  const int num_tiles = ch_tiles * tok_tiles;
  const int tile0 = blockIdx.x / per_tile, tile_step = gridDim.x / per_tile;
  // Everything above may overlap the kernels before this one; codes and scales come from them.
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer
    if (ptx::elect_one()) {
      // barriers and stages by their shared-memory addresses; PAIR: all copies of the pair are counted on the even CTA's
      const uint32_t full0 = PAIR ? ptx::mapa(ptx::smem_u32(full), 0u) : ptx::smem_u32(full), ring = ptx::smem_u32(smem);
      uint32_t dst = ring, phase = 0, issued = 0;
      int stage = 0;
      bool ok = true, ready = false;   // ready: the next stage was seen to be free
      for (int tile = tile0; tile < num_tiles && ok; tile += tile_step) {
        const Fp8Tile t = fp8_tile(p, tile_start, row_start, p.E, tile, ch_tiles, tok_tiles);
        const int mine = PAIR ? t.n / 2 : t.n;   // token rows this CTA stages (copies bring whole boxes: more, not used)
        const int xrow = t.row0 + (PAIR ? rank * mine : 0);
        const int wrow = t.expert * p.N + t.ch_tile * CH_PER_TILE + (PAIR ? rank * FP8G_BM : 0);
        const int pieces = mine <= p.tail ? (mine + FP8G_TAIL_BOX - 1) / FP8G_TAIL_BOX : 0;
        const uint32_t bytes = pieces ? FP8G_W_BYTES + pieces * (FP8G_TAIL_BOX * FP8G_BK) : p.stage_bytes;
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!ready && !ptx::mbar_wait_bounded_sleepy(&empty[stage], phase ^ 1u, abort_word, FP8G_WAIT_LIMIT)) {
            ok = false;
            break;
          }
          const uint32_t bar = full0 + 8u * stage, ws = dst, xs = dst + FP8G_W_BYTES;
          if (!PAIR || rank == 0) ptx::mbar_arrive_expect_tx(&full[stage], PAIR ? 2 * bytes : bytes);
          ++issued;
          dst += p.stage_bytes;
          if (++stage == p.stages) {
            stage = 0;
            phase ^= 1u;
            dst = ring;
          }
          ready = ptx::mbar_test_wait(&empty[stage], phase ^ 1u);   // answered while the copies are issued
          if constexpr (FUSED) {
            if (fp8_plain_order(p, wrow)) ptx::tma_load_2d_at<PAIR>(ws, &tmap_x_tail, bar, kb * FP8G_BK, wrow);
            else ptx::tma_load_4d_at<PAIR>(ws, &tmap_w, bar, kb * FP8G_BK, 0, 0, wrow >> 5);
          } else {
            ptx::tma_load_2d_at<PAIR>(ws, &tmap_w, bar, kb * FP8G_BK, wrow);
          }
          if (pieces == 0) ptx::tma_load_2d_at<PAIR>(xs, &tmap_x, bar, kb * FP8G_BK, xrow);
          for (int i = 0; i < pieces; ++i)
            ptx::tma_load_2d_at<PAIR>(xs + i * (FP8G_TAIL_BOX * FP8G_BK), &tmap_x_tail, bar, kb * FP8G_BK, xrow + i * FP8G_TAIL_BOX);
        }
      }
      if (!ok) {
        *abort_word = 1;
        raise_device_status(STAMP_ERR_TIMEOUT);
        // let the copies in flight land before the shared memory goes away: the last fill of every stage
        for (uint32_t s = 0; s < static_cast<uint32_t>(p.stages) && s < issued; ++s) {
          const uint32_t parity = (issued - 1 - s) / p.stages & 1u;
          const long long t0 = clock64();
          // (the odd CTA of a pair has no barrier of its own to watch: it just gives its copies the time)
          while (((PAIR && rank != 0) || !ptx::mbar_try_wait(&full[s], parity)) && clock64() - t0 < 2000000LL) {
          }
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer (PAIR: the even CTA's, for both)
    if ((!PAIR || rank == 0) && ptx::elect_one()) {
      constexpr uint32_t idesc0 = ptx::make_mxf8_idesc(PAIR ? 2 * FP8G_BM : FP8G_BM);
      // the ring's stages by the lower words of their weight descriptors; the token rows lie FP8G_W_BYTES further
      const uint32_t first_low = ptx::sw128_desc_low(ptx::smem_u32(smem)), low_step = static_cast<uint32_t>(p.stage_bytes) >> 4;
      uint32_t low = first_low, phase = 0, scount = 0;
      int stage = 0, it = 0;
      bool ok = true, ready = false;   // ready: the operands of the next 128 features were seen to have arrived
      for (int tile = tile0; tile < num_tiles && ok; tile += tile_step) {
        const int n = fp8_tile(p, tile_start, row_start, p.E, tile, ch_tiles, tok_tiles).n;
        const uint32_t idesc = ptx::mxf8_idesc_with(idesc0, n);
        int in_chunk = 0;   // steps that are in the accumulator already
        for (int s = step0; s < step1 && ok; ++s, ++scount) {
          const int a = it & 1;
          // The scale words of this step, and their tensor-memory columns: two buffers, so the MMAs of the step before
          // the last have to be through (they are, long before the last one's are: the queue stays filled).
          const uint32_t slot = scount % FP8G_SF_SLOTS, before = scount - 2u;
          const uint32_t parity = (scount / FP8G_SF_SLOTS) & 1u;
          ok = (PAIR ? ptx::mbar_wait_bounded_cluster(&sffull[slot], parity, abort_word, FP8G_WAIT_LIMIT)
                     : ptx::mbar_wait_bounded(&sffull[slot], parity, abort_word, FP8G_WAIT_LIMIT)) &&
               (scount < 2u || ptx::mbar_wait_bounded(&sfempty[before % FP8G_SF_SLOTS], (before / FP8G_SF_SLOTS) & 1u, abort_word,
                                                      FP8G_WAIT_LIMIT));
          if (!ok) break;
          ptx::tc_fence_after();
          const uint32_t sfs = ptx::smem_u32(smem + SM::SF_OFFSET + slot * SM::SF_SLOT);
          const uint32_t sfa = tmem_base + SM::SF_COL + (scount & 1u) * SM::SF_COLS, sfb = sfa + 4;
          ptx::tmem_copy_scales<PAIR>(sfa, ptx::make_rows16_desc(sfs));
          ptx::tmem_copy_scales<PAIR>(sfb, ptx::make_rows16_desc(sfs + 512));
          if (PAIR && n > 128) ptx::tmem_copy_scales<PAIR>(sfb + 4, ptx::make_rows16_desc(sfs + 1024));
          if (in_chunk == 0) {
            // PAIR: the columns shared with the previous accumulator are drained (which implies that everything of the
            // one before it is); otherwise this accumulator's previous contents are
            ok = PAIR ? ptx::mbar_wait_bounded(&tempty[0], (it - 1) & 1, abort_word, FP8G_WAIT_LIMIT)
                      : ptx::mbar_wait_bounded(&tempty[a], ((it >> 1) & 1) ^ 1, abort_word, FP8G_WAIT_LIMIT);
            if (!ok) break;
            ptx::tc_fence_after();
          }
          const uint32_t tmem_d = tmem_base + static_cast<uint32_t>(a * SM::ACC1);
          const int blocks = min(4, num_kb - 4 * s);
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            if (b >= blocks) break;
            if (!ready && !ptx::mbar_wait_bounded(&full[stage], phase, abort_word, FP8G_WAIT_LIMIT)) {
              ok = false;
              break;
            }
            ptx::tc_fence_after();
            const uint32_t w_low = low, used = ptx::smem_u32(&empty[stage]);
            low += low_step;
            if (++stage == p.stages) {
              stage = 0;
              phase ^= 1u;
              low = first_low;
            }
            ready = ptx::mbar_test_wait(&full[stage], phase);   // answered while the instructions are issued
            ptx::mma_mxf8_128<PAIR>(tmem_d, w_low, w_low + (FP8G_W_BYTES >> 4), idesc | (static_cast<uint32_t>(b) << 4 | static_cast<uint32_t>(b) << 29),
                                    sfa, sfb, (in_chunk > 0 || b > 0) ? 1u : 0u, used);
          }
          if (!ok) break;
          if constexpr (PAIR) ptx::tc_commit_pair(&sfempty[slot], 3); else ptx::tc_commit(&sfempty[slot]);
          if (++in_chunk == p.chunk || s + 1 == step1) {
            if constexpr (PAIR) ptx::tc_commit_pair(&tfull[a], 3); else ptx::tc_commit(&tfull[a]);
            in_chunk = 0;
            ++it;
          }
        }
      }
      if (!ok) {
        *abort_word = 1;
        raise_device_status(STAMP_ERR_TIMEOUT);
      }
    }
  } else if (warp < 4) {
    // ------------------------------------------------------------------ scale producers: every other step each
    const uint32_t odd_step = warp & 1;
    const uint32_t sffull_bar0 = PAIR ? ptx::mapa(ptx::smem_u32(&sffull[0]), 0u) : 0u;
    const int ch_blocks = (p.N + FP8_BLOCK - 1) / FP8_BLOCK;
    uint32_t scount = 0;
    bool ok = true;
    for (int tile = tile0; tile < num_tiles && ok; tile += tile_step) {
      const Fp8Tile t = fp8_tile(p, tile_start, row_start, p.E, tile, ch_tiles, tok_tiles);
      // a CTA's 128 channels are one block of the weights' scales (a tile past the last channel takes the last block's)
      const int cb = min(t.ch_tile * (CH_PER_TILE / FP8_BLOCK) + (PAIR ? rank : 0), ch_blocks - 1);
      const uint8_t* wsc = p.w_scale + (static_cast<long>(t.expert) * ch_blocks + cb) * p.ks;
      const uint8_t* xsc = p.x_scale + static_cast<long>(t.row0) * p.ks;
      // Rows of scale bytes on word boundaries: one load per step.  Otherwise the two aligned words that hold the bytes,
      // where both are sure to lie within the scales (their eight bytes start at most three bytes before the first one
      // wanted: four rows of the table before the tile's and eight behind them are enough), or byte by byte.
      const int mode = p.x_words ? 0 : (t.row0 >= 4 && t.row0 + t.rows + 8 <= p.M) ? 1 : 2;
      // All loads of a step are issued before the first is used; they are in flight while the step waits for its slot.
      uint32_t ww, xw[BN / 32];
      auto load = [&](int s) {
        const int k = 4 * s, nk = min(4, p.ks - k);
        ww = fp8_scale_word(wsc + k, nk, true);
        const uint8_t* at = xsc + static_cast<long>(lane) * p.ks + k;
        const long step32 = 32L * p.ks;
        if (mode == 0) {
#pragma unroll
          for (int q = 0; q < BN / 32; ++q, at += step32)
            xw[q] = q * 32 + lane < t.rows ? __ldg(reinterpret_cast<const uint32_t*>(at)) : 0x7F7F7F7Fu;
        } else if (mode == 1) {
          uint32_t lo[BN / 32], hi[BN / 32];
#pragma unroll
          for (int q = 0; q < BN / 32; ++q) {
            const uint32_t* word = reinterpret_cast<const uint32_t*>(reinterpret_cast<uintptr_t>(at + q * step32) & ~uintptr_t(3));
            const bool live = q * 32 + lane < t.rows;
            lo[q] = live ? __ldg(word) : 0x7F7F7F7Fu;
            hi[q] = live ? __ldg(word + 1) : 0x7F7F7F7Fu;
          }
#pragma unroll
          for (int q = 0; q < BN / 32; ++q)
            xw[q] = __funnelshift_r(lo[q], hi[q], 8 * static_cast<uint32_t>(reinterpret_cast<uintptr_t>(at + q * step32) & 3));
        } else {
#pragma unroll
          for (int q = 0; q < BN / 32; ++q, at += step32) xw[q] = fp8_scale_word(at, nk, q * 32 + lane < t.rows);
        }
      };
      int s = step0 + static_cast<int>((scount ^ odd_step) & 1u);
      scount += s - step0;
      if (s < step1) load(s);
      for (; s < step1; s += 2, scount += 2) {
        const uint32_t slot = scount % FP8G_SF_SLOTS;
        if (!__all_sync(0xffffffffu, ptx::mbar_wait_bounded_sleepy(&sfempty[slot], ((scount / FP8G_SF_SLOTS) & 1u) ^ 1u, abort_word,
                                                                   FP8G_WAIT_LIMIT))) {
          ok = false;
          break;
        }
        uint8_t* dst = smem + SM::SF_OFFSET + slot * SM::SF_SLOT + lane * 16;
        *reinterpret_cast<uint4*>(dst) = make_uint4(ww, ww, ww, ww);
#pragma unroll
        for (int h = 0; h < BN / 128; ++h)
          *reinterpret_cast<uint4*>(dst + 512 + 512 * h) = make_uint4(xw[4 * h], xw[4 * h + 1], xw[4 * h + 2], xw[4 * h + 3]);
        ptx::fence_proxy_async_smem();   // tcgen05.cp reads them through the async proxy
        __syncwarp();
        if (lane == 0) {
          if constexpr (PAIR) ptx::mbar_arrive_cluster(sffull_bar0 + slot * 8u); else ptx::mbar_arrive(&sffull[slot]);
        }
        // (behind the arrival: with release semantics towards the cluster it would wait for loads in flight)
        if (s + 2 < step1) load(s + 2);
      }
      scount -= s - step1;   // steps of the tiles so far
    }
    if (!ok) {
      *abort_word = 1;
      if (lane == 0) raise_device_status(STAMP_ERR_TIMEOUT);
    }
  } else if constexpr (FUSED) {
    // ------------------------------------------------------------------ epilogue warps, with what follows the sum
    constexpr int G = GROUPS;
    const int quarter = warp & 3;          // TMEM lanes this warp may touch
    const int group = (warp - 4) >> 2;     // which chunks of 32 columns it takes: every G-th
    const int g4 = lane >> 2, col = 2 * (lane & 3);   // its channels; its tokens of a chunk: 8 k + col + e, k = 0..3, e = 0, 1
    const uint32_t tempty_bar0 = PAIR ? ptx::mapa(ptx::smem_u32(&tempty[0]), 0u) : 0u;
    TOut* const y = static_cast<TOut*>(p.y);
    // Hints that bring a tile's residual to L2, a tile ahead: a chunk's loads are too few to hide the way from memory.
    auto prefetch_residual = [&](int tile) {
      if (sizeof(TOut) == 1 || !p.residual || !(PAIR || p.split == 1) || tile >= num_tiles) return;
      const Fp8Tile t = fp8_tile(p, tile_start, row_start, p.E, tile, ch_tiles, tok_tiles);
      const int size = p.r_bf16 ? 2 : 4, first = (PAIR ? 2 * t.ch_tile + rank : t.ch_tile) * FP8G_BM, end = min(first + FP8G_BM, p.N);
      const char* const at = static_cast<const char*>(p.residual) + (static_cast<long>(t.row0) * p.ldr) * size;
      for (int r = (warp - 4) * 32 + lane; r < t.rows; r += 128 * G)
        for (int ch = first; ch < end; ch += 128 / size) ptx::prefetch_l2(at + (static_cast<long>(r) * p.ldr + ch) * size);
    };
    prefetch_residual(tile0);
    constexpr bool SUMMED = sizeof(TOut) == 4 || PARTS;   // of several accumulators, if need be
    float carried[PARTS ? BN / 32 / G : 1][32];           // PARTS: this thread's sums of the parts before, by chunk
    uint32_t exchanged = 0;   // maxima that this group has exchanged
    int it = 0;
    bool ok = true;
    for (int tile = tile0; tile < num_tiles && ok; tile += tile_step) {
      const Fp8Tile t = fp8_tile(p, tile_start, row_start, p.E, tile, ch_tiles, tok_tiles);
      const int block = PAIR ? 2 * t.ch_tile + rank : t.ch_tile;
      const bool plain = fp8_plain_order(p, block * FP8G_BM);
      // this thread's channels: four from ch on, or, in plain order, ch alone
      const int ch = block * FP8G_BM + quarter * 32 + (plain ? lane : 4 * g4);
      const bool have = ch < p.N;   // (all four or none)
      float bias[4] = {0.f, 0.f, 0.f, 0.f};
      if (p.bias) {
#pragma unroll
        for (int c = 0; c < 4; ++c) bias[c] = __ldg(p.bias + min(ch + c, p.N - 1));
#pragma unroll
        for (int c = 0; c < 4; ++c) bias[c] = have ? bias[c] : 0.f;
      }
      for (int c0 = step0; c0 < step1; c0 += p.chunk, ++it) {
        const int a = it & 1;
        const bool first = !SUMMED || c0 == step0, last = !SUMMED || c0 + p.chunk >= step1;
        // The bias goes in with the first part, the activation follows the last; without one the residual goes in with the
        // first part too: the output, which holds the parts, may be the residual's own memory.
        const bool whole = PAIR || p.split == 1;
        const bool add = sizeof(TOut) != 1 && p.residual && whole && (p.act == STAMP_ACT_NONE ? first : last);
        const int count = fp8_drain_chunks((t.n + 31) / 32, group, G);
        auto chunk_at = [&](int i) { return fp8_drain_chunk(PAIR && a == 0, group, i, count, G); };
        if (first) prefetch_residual(tile + tile_step);
        const uint32_t taddr = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + static_cast<uint32_t>(a * SM::ACC1);
        bool released = false;
        auto release = [&]() {
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            if constexpr (PAIR) ptx::mbar_arrive_cluster_relaxed(tempty_bar0); else ptx::mbar_arrive(&tempty[a]);
          }
          released = true;
        };
        // Waits for the sums.  PAIR: the chunk that overlaps the other accumulator is drained first; who has none of it hands back
        // at once.
        auto begin = [&]() {
          if (!__all_sync(0xffffffffu, ptx::mbar_wait_bounded_sleepy(&tfull[a], (it >> 1) & 1, abort_word, FP8G_WAIT_LIMIT))) {
            ok = false;
            return false;
          }
          ptx::tc_fence_after();
          if (PAIR && group != fp8_overlap_group(a, G)) release();
          return true;
        };
        // The largest magnitudes of a chunk's tokens over this warp's channels, one a lane, to those over the block's four warps:
        // scales to memory, inverse scales to this warp's shared memory.  False: the others have given up.
        auto exchange = [&](int tok, int mine, uint32_t amax) {
          uint8_t* const ex = smem + SM::EX_OFFSET;
          uint64_t* const bar = reinterpret_cast<uint64_t*>(ex) + group;
          uint32_t* const maxima = reinterpret_cast<uint32_t*>(ex + 8 * G) + (group * 2 + static_cast<int>(exchanged & 1u)) * 128;
          float* const inverse = reinterpret_cast<float*>(ex + 8 * G) + G * 256 + (warp - 4) * 32;
          maxima[quarter * 32 + mine] = amax;
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(bar);
          if (!__all_sync(0xffffffffu, ptx::mbar_wait_bounded(bar, exchanged & 1u, abort_word, FP8G_WAIT_LIMIT))) ok = false;
          ++exchanged;
          amax = 0;   // bits of magnitudes order like integers, NaNs above infinity
#pragma unroll
          for (int q = 0; q < 4; ++q) amax = max(amax, maxima[q * 32 + mine]);
          const Fp8Scale s = fp8_scale(amax);
          const int ks_out = (p.N + FP8_BLOCK - 1) / FP8_BLOCK;
          if (ok && quarter == 0 && tok + mine < t.rows && block < ks_out) p.y_scale[(t.row0 + static_cast<long>(tok + mine)) * ks_out + block] = s.byte;
          __syncwarp();   // (everyone has read the chunk's before)
          inverse[mine] = s.inverse;
          __syncwarp();
          return static_cast<const float*>(inverse);
        };
        const int act = last && whole ? p.act : STAMP_ACT_NONE;
        if (plain) {
          // A lane a channel, 16 tokens at a time (codes: all 32 of a chunk, for their maxima), what they are added to loaded one
          // step ahead.
          constexpr int W = sizeof(TOut) == 1 ? 32 : 16, STEPS = 32 / W;
          auto column_of = [&](int n) { return 32 * chunk_at(n / STEPS) + W * (n % STEPS); };
          uint32_t more[sizeof(TOut) == 1 ? 1 : 16], old[sizeof(TOut) == 4 ? 16 : 1];
          auto fetch = [&](int tok) {
            const int left = have ? t.rows - tok : 0;
            if constexpr (sizeof(TOut) != 1) {
              const long at = (t.row0 + static_cast<long>(tok)) * p.ldr + ch;
              if (add) {
                if (p.r_bf16) fp8_load_column(static_cast<const uint16_t*>(p.residual) + at, p.ldr, left, more);
                else fp8_load_column(static_cast<const uint32_t*>(p.residual) + at, p.ldr, left, more);
              }
            }
            if constexpr (sizeof(TOut) == 4) {
              if (!first) fp8_load_column(reinterpret_cast<const uint32_t*>(y) + (t.row0 + static_cast<long>(tok)) * p.N + ch, p.N, left, old);
            }
          };
          if (count > 0) fetch(column_of(0));
          auto drain = [&](auto variant, float floor) {
            for (int n = 0; n < count * STEPS; ++n) {
              const int tok = column_of(n), left = have ? t.rows - tok : 0;
              const bool last_of = n + 1 == (PAIR ? STEPS : count * STEPS);
              if (STEPS > 1 && tok >= t.rows) {   // (no such tokens, for anyone)
                if (!released && last_of) release();
                if (n + 1 < count * STEPS) fetch(column_of(n + 1));
                continue;
              }
              uint32_t r[W];
              float v[W];
              if constexpr (W == 32) ptx::tmem_ld_32x32b_x32(taddr + tok, r); else ptx::tmem_ld_32x32b_x16(taddr + tok, r);
              ptx::tmem_ld_wait();
              if (!released && last_of) release();
#pragma unroll
              for (int j = 0; j < W; ++j) v[j] = __uint_as_float(r[j]);
              if (!whole) {
                float* const part = reinterpret_cast<float*>(smem) + tok * FP8G_PART + (ch - block * FP8G_BM);
#pragma unroll
                for (int j = 0; j < W; ++j) part[j * FP8G_PART] = v[j];
                continue;
              }
              if constexpr (sizeof(TOut) == 4) {
                if (!first) {
#pragma unroll
                  for (int j = 0; j < W; ++j) v[j] += __uint_as_float(old[j]);
                }
              }
              if constexpr (PARTS) {
                float (&kept)[32] = carried[chunk_at(n) / G];
                if (!first) {
#pragma unroll
                  for (int j = 0; j < W; ++j) v[j] += kept[j];
                }
                if (!last) {
#pragma unroll
                  for (int j = 0; j < W; ++j) kept[j] = first ? v[j] + bias[0] : v[j];
                  continue;
                }
              }
#pragma unroll
              for (int j = 0; j < W; j += 2) {
                float2 x = make_float2(v[j], v[j + 1]);
                if (!SUMMED || first) x = __fadd2_rn(x, make_float2(bias[0], bias[0]));
                x = fp8_activate2<decltype(variant)::value>(x, floor);
                v[j] = x.x;
                v[j + 1] = x.y;
              }
              if constexpr (sizeof(TOut) != 1) {
                if (add) {
                  const int shift = p.r_bf16 ? 16 : 0;
#pragma unroll
                  for (int j = 0; j < W; ++j) v[j] += __uint_as_float(more[j] << shift);
                }
                if (n + 1 < count * STEPS) fetch(column_of(n + 1));
                TOut* out = y + (t.row0 + static_cast<long>(tok)) * p.N + ch;
                if (left >= W) {
#pragma unroll
                  for (int j = 0; j < W; ++j, out += p.N) fp8_put(out, v[j]);
                } else {
#pragma unroll
                  for (int j = 0; j < W; ++j, out += p.N)
                    if (j < left) fp8_put(out, v[j]);
                }
              } else {
                uint32_t amax = 0;   // (channels that do not exist are zeros)
#pragma unroll
                for (int j = 0; j < W; ++j) {
                  const uint32_t m = __float_as_uint(ptx::warp_max_abs(v[j]));
                  if (lane == j) amax = m;
                }
                const float* const inverse = exchange(tok, lane, amax);
                if (!ok) return;
                uint8_t* out = static_cast<uint8_t*>(p.y) + (t.row0 + static_cast<long>(tok)) * p.N + ch;
#pragma unroll
                for (int j = 0; j < W; j += 4, out += 4L * p.N) {
                  const uint32_t codes = ptx::cvt_e4m3x4(v[j] * inverse[j], v[j + 1] * inverse[j + 1], v[j + 2] * inverse[j + 2], v[j + 3] * inverse[j + 3]);
#pragma unroll
                  for (int k = 0; k < 4; ++k)
                    if (j + k < left) out[static_cast<long>(k) * p.N] = static_cast<uint8_t>(codes >> (8 * k));
                }
              }
            }
          };
          if (begin()) fp8_with_activation(act, drain);
          if (!released) release();
          if (!ok) break;
          continue;
        }
        // KU times eight columns at a time: codes all 32 of a chunk, for the tokens' maxima; bf16 pairs too, to have more loads in
        // flight; single CTAs, which often have few rows, and fp32, which has more to hold, 16.
        constexpr int KU = sizeof(TOut) == 1 || (PAIR && sizeof(TOut) == 2) ? 4 : 2, UNITS = 4 / KU;
        auto column_of = [&](int n) { return 32 * chunk_at(n / UNITS) + 8 * KU * (n % UNITS); };
        // What the columns add to is loaded ahead: for the first ones before the sums are waited for, then one step ahead.  Plain
        // loads: every element is read by the thread that writes it.
        uint4 res[sizeof(TOut) == 1 ? 1 : 2 * KU], before[sizeof(TOut) == 4 ? 2 * KU : 1];
        auto fetch = [&](int c) {
          const int tok = c + col, there = have ? t.rows - tok : 0;
          if constexpr (sizeof(TOut) != 1) {
            if (add) fp8_load_tokens<KU>(p.residual, (t.row0 + static_cast<long>(tok)) * p.ldr + ch, p.ldr, p.r_bf16, there, res);
          }
          if constexpr (sizeof(TOut) == 4) {
            if (!first) fp8_load_tokens<KU>(y, (t.row0 + static_cast<long>(tok)) * p.N + ch, p.N, false, there, before);
          }
        };
        if (count > 0) fetch(column_of(0));
        auto drain = [&](auto variant, float floor) {
          for (int n = 0; n < count * UNITS; ++n) {
            const int c = column_of(n), left = have ? t.rows - c - col : 0;   // tokens 8 k + e below `left` are stored
            const bool last_of = n + 1 == (PAIR ? UNITS : count * UNITS);
            if (UNITS > 1 && c >= t.rows) {   // (no such tokens, for anyone)
              if (!released && last_of) release();
              if (n + 1 < count * UNITS) fetch(column_of(n + 1));
              continue;
            }
            float v[4][2 * KU];
            {
              uint32_t lo[4 * KU], hi[4 * KU];
              ptx::tmem_ld_16x256b<KU>(taddr + c, lo);
              ptx::tmem_ld_16x256b<KU>(taddr + c + (16u << 16), hi);
              ptx::tmem_ld_wait();
#pragma unroll
              for (int k = 0; k < KU; ++k)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  v[0][2 * k + e] = __uint_as_float(lo[4 * k + e]);
                  v[1][2 * k + e] = __uint_as_float(lo[4 * k + 2 + e]);
                  v[2][2 * k + e] = __uint_as_float(hi[4 * k + e]);
                  v[3][2 * k + e] = __uint_as_float(hi[4 * k + 2 + e]);
                }
            }
            if (!released && last_of) release();
            if (!whole) {
              // this CTA's part of the sum, [token][channel], in the ring that nothing uses any more
              float* const part = reinterpret_cast<float*>(smem) + (c + col) * FP8G_PART + (ch - block * FP8G_BM);
              fp8_store_tokens<KU>(part, FP8G_PART, 8 * KU, v);
              continue;
            }
            if constexpr (sizeof(TOut) == 4) {
              if (!first) fp8_add_tokens<KU>(before, false, v);
            }
            if constexpr (PARTS) {
              float (&kept)[32] = carried[chunk_at(n) / G];
              if (!first) {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j >> 3][j & 7] += kept[j];
              }
              if (!last) {
#pragma unroll
                for (int j = 0; j < 32; ++j) kept[j] = first ? v[j >> 3][j & 7] + bias[j >> 3] : v[j >> 3][j & 7];
                continue;
              }
            }
            // (a part that is not the first has its bias already, one that is not the last gets no activation: LINEAR, floor -inf)
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
              for (int j = 0; j < 2 * KU; j += 2) {
                float2 r = make_float2(v[k][j], v[k][j + 1]);
                if (!SUMMED || first) r = __fadd2_rn(r, make_float2(bias[k], bias[k]));
                r = fp8_activate2<decltype(variant)::value>(r, floor);
                v[k][j] = r.x;
                v[k][j + 1] = r.y;
              }
            if constexpr (sizeof(TOut) != 1) {
              if (add) fp8_add_tokens<KU>(res, p.r_bf16, v);
              if (n + 1 < count * UNITS) fetch(column_of(n + 1));
              fp8_store_tokens<KU>(y + (t.row0 + static_cast<long>(c + col)) * p.N + ch, p.N, left, v);
            } else {
              // the largest magnitude of every token: over this thread's channels, the lanes that have the same tokens (each
              // step halves the tokens a lane looks after: lane -> one token), and the block's four warps
              uint32_t m[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) m[j] = __float_as_uint(ptx::max_abs_nan(ptx::max_abs_nan(v[0][j], v[1][j], v[2][j]), v[3][j], 0.f));
#pragma unroll
              for (int d = 16, half = 4; d >= 4; d >>= 1, half >>= 1) {
                const bool upper = (lane & d) != 0;
#pragma unroll
                for (int j = 0; j < half; ++j) {
                  const uint32_t other = __shfl_xor_sync(0xffffffffu, upper ? m[j] : m[j + half], d);
                  m[j] = max(upper ? m[j + half] : m[j], other);
                }
              }
              const int mine = ((lane >> 3) & 3) * 8 + col + ((lane >> 2) & 1);   // the token that is left
              const float* const inverse = exchange(c, mine, m[0]);
              if (!ok) return;
              uint32_t codes[8];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const float2 f = *reinterpret_cast<const float2*>(inverse + 8 * k + col);
                const float2 a01 = __fmul2_rn(make_float2(v[0][2 * k], v[0][2 * k + 1]), f), b01 = __fmul2_rn(make_float2(v[1][2 * k], v[1][2 * k + 1]), f);
                const float2 c01 = __fmul2_rn(make_float2(v[2][2 * k], v[2][2 * k + 1]), f), d01 = __fmul2_rn(make_float2(v[3][2 * k], v[3][2 * k + 1]), f);
                codes[2 * k] = ptx::cvt_e4m3x4(a01.x, b01.x, c01.x, d01.x);
                codes[2 * k + 1] = ptx::cvt_e4m3x4(a01.y, b01.y, c01.y, d01.y);
              }
              uint8_t* out = static_cast<uint8_t*>(p.y) + (t.row0 + static_cast<long>(c + col)) * p.N + ch;
              uint8_t* next = out + p.N;
#pragma unroll
              for (int k = 0; k < 4; ++k, out += 8L * p.N, next += 8L * p.N) {
                if (8 * k < left) *reinterpret_cast<uint32_t*>(out) = codes[2 * k];
                if (8 * k + 1 < left) *reinterpret_cast<uint32_t*>(next) = codes[2 * k + 1];
              }
            }
          }
        };
        if (begin()) fp8_with_activation(act, drain);
        if (!released) release();
        if (!ok) break;
      }
    }
    if (!ok) {
      *abort_word = 1;
      if (lane == 0) raise_device_status(STAMP_ERR_TIMEOUT);
    }
  } else if (warp >= 4) {
    // ------------------------------------------------------------------ epilogue warps
    const int quarter = warp & 3;          // TMEM lanes this warp may touch
    const int half = (warp - 4) >> 2;      // which half of the column chunks it takes
    const int row = quarter * 32 + lane;
    const uint32_t tempty_bar0 = PAIR ? ptx::mapa(ptx::smem_u32(&tempty[0]), 0u) : 0u;
    const bool vec = (reinterpret_cast<uintptr_t>(p.y) & (2 * sizeof(TOut) - 1)) == 0 && (p.N & 1) == 0;
    TOut* const y = static_cast<TOut*>(p.y);
    int it = 0;
    bool ok = true;
    for (int tile = tile0; tile < num_tiles && ok; tile += tile_step) {
      const Fp8Tile t = fp8_tile(p, tile_start, row_start, p.E, tile, ch_tiles, tok_tiles);
      const int ch = (PAIR ? 2 * t.ch_tile + rank : t.ch_tile) * FP8G_BM + row;
      float bias = 0.f;
      if (p.bias && ch < p.N) bias = __ldg(p.bias + static_cast<long>(t.expert) * p.N + ch);
      for (int c0 = step0; c0 < step1; c0 += p.chunk, ++it) {
        const int a = it & 1;
        if (!__all_sync(0xffffffffu, ptx::mbar_wait_bounded_sleepy(&tfull[a], (it >> 1) & 1, abort_word, FP8G_WAIT_LIMIT))) {
          ok = false;
          break;
        }
        ptx::tc_fence_after();
        const uint32_t taddr = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + static_cast<uint32_t>(a * SM::ACC1);
        bool released = false;
        auto release = [&]() {
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            if constexpr (PAIR) ptx::mbar_arrive_cluster_relaxed(tempty_bar0); else ptx::mbar_arrive(&tempty[a]);
          }
          released = true;
        };
        // PAIR: the chunk that overlaps the other accumulator first; who has none of it hands back at once
        if (PAIR && half != fp8_overlap_group(a, 2)) release();
        const int count = fp8_drain_chunks((t.n + 31) / 32, half, 2);
        for (int i = 0; i < count; ++i) {
          const int c = fp8_drain_chunk(PAIR && a == 0, half, i, count, 2);
          uint32_t r[32];
          ptx::tmem_ld_32x32b_x32(taddr + 32 * c, r);
          ptx::tmem_ld_wait();
          if (!released && (PAIR || i + 1 == count)) release();
          if (!PAIR && p.split > 1) {
            // this CTA's part of the sum, [token][channel], in the ring that nothing uses any more
            float* part = reinterpret_cast<float*>(smem);
#pragma unroll
            for (int j = 0; j < 32; ++j) part[(32 * c + j) * FP8G_BM + row] = __uint_as_float(r[j]);
            continue;
          }
          const int left = t.rows - 32 * c;
          if constexpr (sizeof(TOut) == 4) {
            TOut* out = y + static_cast<long>(t.row0 + 32 * c) * p.N + ch;
            if (c0 == step0) {
              if (ch < p.N) {
                if (left >= 32) {
#pragma unroll
                  for (int j = 0; j < 32; ++j, out += p.N) *out = __uint_as_float(r[j]) + bias;
                } else {
#pragma unroll
                  for (int j = 0; j < 32; ++j, out += p.N)
                    if (j < left) *out = __uint_as_float(r[j]) + bias;
                }
              }
            } else if (ch < p.N) {   // a later part of the sum: on top of this thread's own value of the parts before
              float before[32];
#pragma unroll
              for (int j = 0; j < 32; ++j) before[j] = j < left ? out[static_cast<long>(j) * p.N] : 0.f;
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (j < left) out[static_cast<long>(j) * p.N] = before[j] + __uint_as_float(r[j]);
            }
          } else {
            // Neighbouring lanes swap halves of a token pair: either then holds two adjacent channels of one token, the even
            // lane of the first, the odd lane of the second.
            const int odd = lane & 1, ch2 = ch & ~1;
            const uint32_t sel = odd ? 0x3276u : 0x5410u;
            TOut* out = y + static_cast<long>(t.row0 + 32 * c + odd) * p.N + ch2;
            uint32_t two[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const __nv_bfloat162 v = __floats2bfloat162_rn(__uint_as_float(r[2 * j]) + bias, __uint_as_float(r[2 * j + 1]) + bias);
              two[j] = *reinterpret_cast<const uint32_t*>(&v);
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) two[j] = __byte_perm(two[j], __shfl_xor_sync(0xffffffffu, two[j], 1), sel);
            if (vec && left >= 32) {
              if (ch2 < p.N) {
#pragma unroll
                for (int j = 0; j < 16; ++j, out += 2 * static_cast<long>(p.N)) *reinterpret_cast<uint32_t*>(out) = two[j];
              }
            } else {
#pragma unroll
              for (int j = 0; j < 16; ++j, out += 2 * static_cast<long>(p.N))
                if (2 * j + odd < left && ch2 < p.N) {
                  const __nv_bfloat162 v = *reinterpret_cast<const __nv_bfloat162*>(&two[j]);
                  if (vec) {
                    *reinterpret_cast<__nv_bfloat162*>(out) = v;
                  } else {
                    out[0] = v.x;
                    if (ch2 + 1 < p.N) out[1] = v.y;
                  }
                }
            }
          }
        }
        if (!released) release();
      }
    }
    if (!ok) {
      *abort_word = 1;
      if (lane == 0) raise_device_status(STAMP_ERR_TIMEOUT);
    }
  }

  ptx::tc_fence_before();
  __syncthreads();
  // Nobody lets go of its shared and tensor memory while a CTA of the cluster may still signal into it.
  if (clustered) ptx::cluster_sync();
  if (!PAIR && p.split > 1) {
    // every CTA adds up every split-th token of the tile over the cluster's partial sums, in rank order
    if (tile0 < num_tiles && *abort_word == 0) {
      const Fp8Tile t = fp8_tile(p, tile_start, row_start, p.E, tile0, ch_tiles, tok_tiles);
      const uint32_t part = ptx::smem_u32(smem);
      const bool vec = (reinterpret_cast<uintptr_t>(p.y) & (2 * sizeof(TOut) - 1)) == 0 && (p.N & 1) == 0;
      uint32_t part_of[8];
#pragma unroll
      for (int s = 0; s < 8; ++s) part_of[s] = ptx::mapa(part, static_cast<uint32_t>(min(s, p.split - 1)));
      const int c4 = 4 * lane, ch = t.ch_tile * FP8G_BM + c4;   // a warp takes a token, a lane four channels
      float bias[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) bias[i] = (p.bias && ch + i < p.N) ? __ldg(p.bias + static_cast<long>(t.expert) * p.N + ch + i) : 0.f;
      for (int tok = rank + warp * p.split; tok < t.rows; tok += THREADS / 32 * p.split) {
        float4 v[8];   // all in flight at once
#pragma unroll
        for (int s = 0; s < 8; ++s)
          if (s < p.split) v[s] = ptx::ld_dsmem_f4(part_of[s] + (tok * (FUSED ? FP8G_PART : FP8G_BM) + c4) * 4);
        float4 sum = v[0];
#pragma unroll
        for (int s = 1; s < 8; ++s)
          if (s < p.split) sum = make_float4(sum.x + v[s].x, sum.y + v[s].y, sum.z + v[s].z, sum.w + v[s].w);
        TOut* out = static_cast<TOut*>(p.y) + static_cast<long>(t.row0 + tok) * p.N + ch;
        if constexpr (FUSED) {
          float2 a, b;
          fp8_with_activation(p.act, [&](auto variant, float floor) {
            a = fp8_activate2<decltype(variant)::value>(make_float2(sum.x + bias[0], sum.y + bias[1]), floor);
            b = fp8_activate2<decltype(variant)::value>(make_float2(sum.z + bias[2], sum.w + bias[3]), floor);
          });
          float v[4] = {a.x, a.y, b.x, b.y};
          if constexpr (sizeof(TOut) == 1) {
            float most = 0.f;
#pragma unroll
            for (int i = 0; i < 4; i += 2) most = ptx::max_abs_nan(most, ch < p.N ? v[i] : 0.f, ch < p.N ? v[i + 1] : 0.f);
            const Fp8Scale s = fp8_scale(__float_as_uint(ptx::warp_max_abs(most)));
            const int ks_out = (p.N + FP8_BLOCK - 1) / FP8_BLOCK;
            if (lane == 0) p.y_scale[static_cast<long>(t.row0 + tok) * ks_out + t.ch_tile] = s.byte;
            if (ch < p.N)
              *reinterpret_cast<uint32_t*>(out) = ptx::cvt_e4m3x4(v[0] * s.inverse, v[1] * s.inverse, v[2] * s.inverse, v[3] * s.inverse);
          } else {
            if (p.residual) {
              const long at = (t.row0 + static_cast<long>(tok)) * p.ldr + ch;
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (ch + i < p.N) v[i] += p.r_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.residual)[at + i]) : static_cast<const float*>(p.residual)[at + i];
            }
            if (ch < p.N) fp8_store2(out, v[0], v[1], ch + 1 < p.N, vec);
            if (ch + 2 < p.N) fp8_store2(out + 2, v[2], v[3], ch + 3 < p.N, vec);
          }
        } else {
          if (ch < p.N) fp8_store2(out, sum.x + bias[0], sum.y + bias[1], ch + 1 < p.N, vec);
          if (ch + 2 < p.N) fp8_store2(out + 2, sum.z + bias[2], sum.w + bias[3], ch + 3 < p.N, vec);
        }
      }
    }
    ptx::cluster_sync();
  }
  if (warp == 1) {
    ptx::tc_fence_after();
    if constexpr (PAIR) ptx::tmem_dealloc_pair(tmem_base, 512); else ptx::tmem_dealloc(tmem_base, 512);
  }
}

}  // namespace stamp
