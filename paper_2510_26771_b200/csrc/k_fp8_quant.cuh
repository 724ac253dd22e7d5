// Quantizers to e4m3 codes with one power-of-two scale per block of 128 features: activations (a scale per token and
// block), the same behind a gated activation, and weights (a scale per block of 128 x 128).
//
// With a = max |x| over the block, the scale is s = 2^e, e the smallest integer >= -126 with a / s <= 448 (the largest
// e4m3 value, 1.75 * 2^8), and a code is x / s rounded to nearest even.  A power of two costs a floating-point code
// nothing but range (at most one binade of eighteen), and in return every step is exact: e follows from the exponent
// and mantissa bits of a, x / s is a multiplication by 2^-e without rounding, so a code is rounded once and does not
// depend on the order of any arithmetic.  The scale is stored as its biased exponent (e8m0), the form the tensor core's
// block-scaled product reads.  A block of zeros has scale 1.  A block that holds an infinity or a NaN has scale NaN
// (255) and NaN codes: what is computed from it is NaN instead of a finite number that hides it.
#pragma once
#include <type_traits>

#include "common.cuh"
#include "ptx.cuh"

namespace stamp {

constexpr int FP8_BLOCK = 128;      // features per scale
constexpr int FP8Q_THREADS = 256;

struct Fp8Scale {
  float inverse;   // 2^-e
  uint8_t byte;    // e + 127
};
// amax_bits: the largest |x| of the block as float bits (which order like unsigned integers, NaNs above infinity).
__device__ __forceinline__ Fp8Scale fp8_scale(uint32_t amax_bits) {
  Fp8Scale r;
  // biased exponent - 127 - 8, one more when the mantissa is above that of 1.75
  int e = static_cast<int>(amax_bits >> 23) - 135 + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  e = amax_bits == 0u ? 0 : max(e, -126);
  const bool finite = amax_bits < 0x7F800000u;
  r.inverse = __uint_as_float(finite ? static_cast<uint32_t>(127 - e) << 23 : 0x7FC00000u);
  r.byte = finite ? static_cast<uint8_t>(e + 127) : static_cast<uint8_t>(255);
  return r;
}

// Eight adjacent features of one row, as loaded and as floats.
template <typename T>
struct Fp8Raw;
template <>
struct Fp8Raw<__nv_bfloat16> {
  uint4 u;
  __device__ __forceinline__ void load(const __nv_bfloat16* p, bool live) {
    u = live ? __ldg(reinterpret_cast<const uint4*>(p)) : make_uint4(0u, 0u, 0u, 0u);
  }
  // all magnitudes at most 80 (a NaN may say either)
  __device__ __forceinline__ bool within80() const {
    const uint32_t m = ptx::max_abs_bf16x2(ptx::max_abs_bf16x2(u.x, u.y), ptx::max_abs_bf16x2(u.z, u.w)) & 0x7FFF7FFFu;
    return max(m & 0xFFFFu, m >> 16) <= 0x42A0u;
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
};
template <>
struct Fp8Raw<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p, bool live) {
    a = live ? __ldg(reinterpret_cast<const float4*>(p)) : make_float4(0.f, 0.f, 0.f, 0.f);
    b = live ? __ldg(reinterpret_cast<const float4*>(p) + 1) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  __device__ __forceinline__ bool within80() const {
    const float m = ptx::max_abs_nan(ptx::max_abs_nan(a.x, a.y, a.z), ptx::max_abs_nan(a.w, b.x, b.y), ptx::max_abs_nan(b.z, b.w, 0.f));
    return m <= 80.f;
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
};

__device__ __forceinline__ uint2 fp8_pack8(const float (&v)[8], float inverse) {
  const float2 i2 = make_float2(inverse, inverse);
  float2 s[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) s[i] = __fmul2_rn(make_float2(v[2 * i], v[2 * i + 1]), i2);
  return make_uint2(ptx::cvt_e4m3x4(s[0].x, s[0].y, s[1].x, s[1].y), ptx::cvt_e4m3x4(s[2].x, s[2].y, s[3].x, s[3].y));
}

// silu(g) * u = g / (1 + exp(-g)) * u, for two neighbours at once in packed fp32 instructions, to about an ulp of the
// IEEE operations in that order.  exp(-g) is 2^(-g log2 e), and what rounding that product would lose, the power would
// multiply by g.  So it is split: a bf16 gate (8 significant bits) times the first 16 bits of log2 e is exact, the rest of
// the constant, times ln 2, becomes a factor 1 + small; an fp32 gate's product is held as head and tail instead.  The
// quotient is g times the approximate reciprocal, corrected once by its remainder.  SMALL: |g| <= 80.  Otherwise the power
// is taken as 0 or infinite past +-90, an infinite divisor takes no correction (inf * 0), and gate and divisor are both
// divided by four: from 2^126 on (g = -87.34) the reciprocal of the divisor itself is subnormal, which the approximation
// returns as zero.  NaNs and infinities come out non-finite, as they do of the formula.
template <bool SMALL, bool BF16>
__device__ __forceinline__ float2 gated_silu2(float2 g, float2 u) {
  auto both = [](float v) { return make_float2(v, v); };
  const float2 x = SMALL ? g : make_float2(fminf(fmaxf(g.x, -90.f), 90.f), fminf(fmaxf(g.y, -90.f), 90.f));
  float2 head, more;   // exp(-x) = 2^head (1 + more)
  if constexpr (BF16) {
    head = __fmul2_rn(x, both(-47274.f / 32768.f));
    more = __fmul2_rn(x, both(-4.88843e-6f));         // (log2 e - 47274 / 32768) ln 2
  } else {
    constexpr float LOG2E = 1.44269504f, LOG2E_TAIL = 1.92596299e-8f, LN2 = 0.693147181f;
    head = __fmul2_rn(x, both(-LOG2E));
    const float2 tail = __ffma2_rn(x, both(-LOG2E), __fmul2_rn(x, both(LOG2E)));
    more = __fmul2_rn(__ffma2_rn(x, both(-LOG2E_TAIL), tail), both(LN2));
  }
  const float2 p = make_float2(ptx::ex2(head.x), ptx::ex2(head.y));
  // (p * more + p would be inf - inf where p is infinite)
  const float2 e = SMALL ? __ffma2_rn(p, more, p) : __fmul2_rn(p, __fadd2_rn(more, both(1.f)));
  // SMALL: g / (1 + e), otherwise both divided by four
  const float2 n = SMALL ? g : __fmul2_rn(g, both(0.25f));
  const float2 minus_d = SMALL ? __ffma2_rn(e, both(-1.f), both(-1.f)) : __ffma2_rn(e, both(-0.25f), both(-0.25f));
  const float2 r = make_float2(ptx::rcp(-minus_d.x), ptx::rcp(-minus_d.y));
  float2 q = __fmul2_rn(n, r);
  const float2 fixed = __ffma2_rn(__ffma2_rn(q, minus_d, n), r, q);
  if constexpr (SMALL) {
    q = fixed;
  } else {
    q.x = minus_d.x > -__int_as_float(0x7F800000) ? fixed.x : q.x;
    q.y = minus_d.y > -__int_as_float(0x7F800000) ? fixed.y : q.y;
  }
  return __fmul2_rn(q, u);
}

// n / d for n below 2^31: `magic` is 2^32 / d rounded up, so the product's upper half is the quotient or one above it.
__device__ __forceinline__ unsigned fp8_div(unsigned n, unsigned d, unsigned magic) {
  const unsigned q = d == 1u ? n : __umulhi(n, magic);
  return static_cast<int>(n - q * d) < 0 ? q - 1u : q;
}

// Both activation quantizers: a warp takes a chunk of a row, four blocks at a time.  Eight lanes own one block, lane l
// features [8 l, 8 l + 8) and [64 + 8 l, 72 + 8 l), so that the eight lanes' loads and stores are contiguous; the maximum
// takes three shuffles.  Where a lane's features lie follows from the row and the chunk, once for all blocks of a chunk.
struct Fp8Rows {
  int K, ks;                 // features of a row, blocks of a row
  unsigned chunks, magic;    // chunks of a row; fp8_div's magic for them
  unsigned items;            // rows x chunks
};
// One block: its codes (out: this lane's first feature, `left` features of the row from there on) and its scale.
__device__ __forceinline__ void fp8_quantize_block(const float (&v)[2][8], int left, uint8_t* out, uint8_t* scale) {
  float largest = 0.f;
#pragma unroll
  for (int i = 0; i < 16; i += 2) largest = ptx::max_abs_nan(largest, v[i >> 3][i & 7], v[i >> 3][(i & 7) + 1]);
  uint32_t amax = __float_as_uint(largest);
#pragma unroll
  for (int d = 1; d < 8; d <<= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, d));
  const Fp8Scale s = fp8_scale(amax);
  if (left > 0) {
    *reinterpret_cast<uint2*>(out) = fp8_pack8(v[0], s.inverse);
    if (left > 64) *reinterpret_cast<uint2*>(out + 64) = fp8_pack8(v[1], s.inverse);
    if ((threadIdx.x & 7u) == 0) *scale = s.byte;
  }
}

// Activations.
//   X       [T, ld]  rows of K features
//   rows    [M] source row of every output row, or nullptr for row m itself; an index outside [0, T) gives a row of
//           zeros and raises the device status word
//   codes   [M, K], scale [M, ks]
// A chunk is 4 U blocks, and a thread loads its part of all of them before it uses the first.  Bound by memory: 16384 x
// 14336 in 102 us, a little above the copy rate (a third of the traffic is writes, not half); fp32 rows in 165 us, likewise.
// A dispatch loads, reduces and converts a token once for each of its experts: 16384 rows of 4096 tokens of 2048 features
// take 12.1 us a call where a pass over memory would take 7.8 (fp32 17.2 and 10.3), 60 % of the issue slots and 40 % of the
// warps busy.  Where tokens and codes stay in L2 it is 9.8; there, with the place of every block found by itself, without
// regard to rows, 12.1 at 8.5 instructions a feature.
template <typename TIn, int U>
__global__ void __launch_bounds__(FP8Q_THREADS) k_fp8_quant(const TIn* __restrict__ X, long ld, const int* __restrict__ rows, int T,
                                                            Fp8Rows r, uint8_t* __restrict__ codes, uint8_t* __restrict__ scale) {
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int sub = (threadIdx.x >> 3) & 3, lane8 = threadIdx.x & 7;
  for (unsigned item = blockIdx.x * (FP8Q_THREADS / 32) + (threadIdx.x >> 5); item < r.items; item += gridDim.x * (FP8Q_THREADS / 32)) {
    const unsigned row = fp8_div(item, r.chunks, r.magic);
    const int block = static_cast<int>(item - row * r.chunks) * (4 * U) + sub, col = block * FP8_BLOCK + lane8 * 8;
    long src = row;
    bool valid = true;
    if (rows) {
      const int i = __ldg(rows + row);
      valid = i >= 0 && i < T;
      if (!valid) raise_device_status(STAMP_ERR_INVALID_ARG);
      src = valid ? i : 0;
    }
    const TIn* p = X + src * ld + col;
    const int left = r.K - col, have = valid ? left : 0;
    Fp8Raw<TIn> raw[U][2];
#pragma unroll
    for (int b = 0; b < U; ++b)
#pragma unroll
      for (int h = 0; h < 2; ++h) raw[b][h].load(p + (4 * b) * FP8_BLOCK + 64 * h, have > (4 * b) * FP8_BLOCK + 64 * h);
    uint8_t* out = codes + static_cast<long>(row) * r.K + col;
    uint8_t* sc = scale + static_cast<long>(row) * r.ks + block;
#pragma unroll
    for (int b = 0; b < U; ++b) {
      float v[2][8];
      raw[b][0].values(v[0]);
      raw[b][1].values(v[1]);
      fp8_quantize_block(v, left - (4 * b) * FP8_BLOCK, out + (4 * b) * FP8_BLOCK, sc + 4 * b);
    }
  }
}

// Behind a gated activation: X [M, ld] rows of K gates and K ups -> codes [M, K], scale [M, ks] of silu(gate) * up.
// A chunk is `quads` times four blocks, one after the other.  16384 x 4096 in 60 us, 86 % of the copy rate (56 without gates
// above 80, 91 for fp32 rows, at the copy rate): the arithmetic
// (15 instructions a feature, two of them on the special function unit, which is busy 58 % of the time) and the loads
// overlap across resident warps only, so it is one block at a time and more warps (two: 70 us against 61.5).  Copies through
// shared memory three blocks ahead, or two sets of registers in turn, cost more instructions or warps than they hide (3 %
// and 7 %); expf and the IEEE division in place of gated_silu2: 92 us.
template <typename TIn>
__global__ void __launch_bounds__(FP8Q_THREADS) k_fp8_gated_quant(const TIn* __restrict__ X, long ld, Fp8Rows r, int quads,
                                                                  uint8_t* __restrict__ codes, uint8_t* __restrict__ scale) {
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int sub = (threadIdx.x >> 3) & 3, lane8 = threadIdx.x & 7;
  for (unsigned item = blockIdx.x * (FP8Q_THREADS / 32) + (threadIdx.x >> 5); item < r.items; item += gridDim.x * (FP8Q_THREADS / 32)) {
    const unsigned row = fp8_div(item, r.chunks, r.magic);
    int quad = static_cast<int>(item - row * r.chunks) * quads;
    const int block = quad * 4 + sub, col = block * FP8_BLOCK + lane8 * 8;
    const TIn* p = X + static_cast<long>(row) * ld + col;
    uint8_t* out = codes + static_cast<long>(row) * r.K + col;
    uint8_t* sc = scale + static_cast<long>(row) * r.ks + block;
    int left = r.K - col;
    // (the warp's four blocks stay in the loop together: the shuffles are warp-wide)
    for (const int end = min(quad + quads, (r.ks + 3) / 4); quad < end; ++quad) {
      Fp8Raw<TIn> gate[2], up[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        gate[h].load(p + 64 * h, left > 64 * h);
        up[h].load(p + 64 * h + r.K, left > 64 * h);
      }
      float v[2][8];
      auto activate = [&](auto small) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float a[8], c[8];
          gate[h].values(a);
          up[h].values(c);
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            const float2 y = gated_silu2<decltype(small)::value, sizeof(TIn) == 2>(make_float2(a[i], a[i + 1]), make_float2(c[i], c[i + 1]));
            v[h][i] = y.x;
            v[h][i + 1] = y.y;
          }
        }
      };
      if (gate[0].within80() && gate[1].within80()) activate(std::true_type{}); else activate(std::false_type{});
      fp8_quantize_block(v, left, out, sc);
      p += 4 * FP8_BLOCK;
      out += 4 * FP8_BLOCK;
      sc += 4;
      left -= 4 * FP8_BLOCK;
    }
  }
}

// Weights (offline): one CTA per block of 128 output channels x 128 features of one matrix.  11008 x 4096 in 27 us (20.7 at
// the copy rate; fp32 37 and 34.5), 32 matrices of 4096 x 4096 in 267 (247; fp32 374 and 411).
//   W [E, N, K], codes [E, N, K], scale [E, ceil(N / 128), ceil(K / 128)]; grid (ceil(K / 128), ceil(N / 128), E)
template <typename TIn>
__global__ void __launch_bounds__(256) k_fp8_quant_weights(const TIn* __restrict__ W, int N, int K, uint8_t* __restrict__ codes,
                                                           uint8_t* __restrict__ scale) {
  __shared__ uint32_t smax[8];
  const int col = blockIdx.x * FP8_BLOCK + (threadIdx.x & 15) * 8;
  const int row0 = blockIdx.y * FP8_BLOCK + (threadIdx.x >> 4);
  const long base = static_cast<long>(blockIdx.z) * N * K + col;
  float v[8][8];
  uint32_t amax = 0;
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const int row = row0 + 16 * r;
    Fp8Raw<TIn> raw;
    raw.load(W + base + static_cast<long>(row) * K, row < N && col < K);
    raw.values(v[r]);
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = max(amax, absbits(v[r][i]));
  }
  amax = __reduce_max_sync(0xffffffffu, amax);
  if ((threadIdx.x & 31) == 0) smax[threadIdx.x >> 5] = amax;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) amax = max(amax, smax[w]);
  const Fp8Scale s = fp8_scale(amax);
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const int row = row0 + 16 * r;
    if (row < N && col < K) *reinterpret_cast<uint2*>(codes + base + static_cast<long>(row) * K) = fp8_pack8(v[r], s.inverse);
  }
  if (threadIdx.x == 0) scale[(static_cast<long>(blockIdx.z) * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x] = s.byte;
}

}  // namespace stamp
