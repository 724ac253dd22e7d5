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

// Eight adjacent features of one row as floats.
__device__ __forceinline__ void fp8_load8(const __nv_bfloat16* p, float (&v)[8]) {
  const uint4 u = __ldg(reinterpret_cast<const uint4*>(p));
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void fp8_load8(const float* p, float (&v)[8]) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ uint2 fp8_pack8(const float (&v)[8], float inverse) {
  uint2 r;
  r.x = ptx::cvt_e4m3x4(v[0] * inverse, v[1] * inverse, v[2] * inverse, v[3] * inverse);
  r.y = ptx::cvt_e4m3x4(v[4] * inverse, v[5] * inverse, v[6] * inverse, v[7] * inverse);
  return r;
}

// silu(g) * u.  Every operation is the IEEE-rounded one (expf's error is the only one above half an ulp).
__device__ __forceinline__ float gated_silu(float g, float u) { return __fmul_rn(__fdiv_rn(g, 1.0f + expf(-g)), u); }

// Activations.  Eight lanes own one block of a row: lane l holds features [8 l, 8 l + 8) and [64 + 8 l, 72 + 8 l), so
// that the eight lanes' loads and stores are contiguous; the maximum takes three shuffles.
//   X       [T, ld]  rows of K features (GATED: of 2 K, the gates first)
//   rows    [M] source row of every output row, or nullptr for row m itself; an index outside [0, T) gives a row of
//           zeros and raises the device status word
//   codes   [M, K], scale [M, ks], ks = ceil(K / 128), groups = M * ks
template <typename TIn, bool GATED>
__global__ void __launch_bounds__(FP8Q_THREADS) k_fp8_quant(const TIn* __restrict__ X, long ld, const int* __restrict__ rows, int T,
                                                            int K, unsigned ks, unsigned groups, uint8_t* __restrict__ codes,
                                                            uint8_t* __restrict__ scale) {
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const unsigned lane8 = threadIdx.x & 7u;
  const unsigned stride = gridDim.x * (FP8Q_THREADS / 8);
  // all four groups of a warp stay in the loop together: the shuffles are warp-wide
  for (unsigned g = blockIdx.x * (FP8Q_THREADS / 8) + (threadIdx.x >> 3); g - ((threadIdx.x >> 3) & 3u) < groups; g += stride) {
    const bool live = g < groups;
    const unsigned row = live ? g / ks : 0u;
    const int col = static_cast<int>(g - row * ks) * FP8_BLOCK + static_cast<int>(lane8) * 8;
    long src = row;
    bool valid = live;
    if (rows) {
      const int i = live ? __ldg(rows + row) : 0;
      valid = live && i >= 0 && i < T;
      if (live && !valid && lane8 == 0) raise_device_status(STAMP_ERR_INVALID_ARG);
      src = valid ? i : 0;
    }
    float v[2][8];
    uint32_t amax = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int c = col + 64 * h;
      if (valid && c < K) {
        fp8_load8(X + src * ld + c, v[h]);
        if constexpr (GATED) {
          float up[8];
          fp8_load8(X + src * ld + K + c, up);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[h][i] = gated_silu(v[h][i], up[i]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[h][i] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) amax = max(amax, absbits(v[h][i]));
    }
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, d));
    const Fp8Scale s = fp8_scale(amax);
    if (live) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (col + 64 * h < K)
          *reinterpret_cast<uint2*>(codes + static_cast<long>(row) * K + col + 64 * h) = fp8_pack8(v[h], s.inverse);
      if (lane8 == 0) scale[g] = s.byte;
    }
  }
}

// Weights (offline): one CTA per block of 128 output channels x 128 features of one matrix.
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
    if (row < N && col < K) {
      fp8_load8(W + base + static_cast<long>(row) * K, v[r]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[r][i] = 0.f;
    }
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
