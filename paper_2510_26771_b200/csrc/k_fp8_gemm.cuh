// Product of block-scaled e4m3 codes, with one weight matrix or with the weights of one expert per run of rows:
//   y[m, n] = sum_b sx[m, b] sw[n / 128, b] sum_{k in b} x[m, k] w[n, k]  (+ bias[n])
// Plain CUDA-core form: one thread per output, sixteen codes per load, a block's products summed in fp32 and scaled
// once per block.
#pragma once
#include <cuda_fp8.h>

#include "common.cuh"
#include "k_fp8_quant.cuh"
#include "ptx.cuh"

namespace stamp {

constexpr int FP8_MAX_EXPERTS = 1024;

struct Fp8GemmParams {
  const uint8_t* x;        // [M, K]
  const uint8_t* x_scale;  // [M, ks]
  const int* offsets;      // [E + 1] first row of every expert, or nullptr: one matrix for all rows
  const uint8_t* w;        // [E, N, K]
  const uint8_t* w_scale;  // [E, ceil(N / 128), ks]
  const float* bias;       // [E, N] or nullptr
  void* y;                 // [M, N] float or bf16
  int M, N, K, E, ks;
};

__device__ __forceinline__ float e8m0_value(uint8_t b) {
  return b == 255 ? __uint_as_float(0x7FC00000u) : b == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(static_cast<uint32_t>(b) << 23);
}
__device__ __forceinline__ void e4m3x4_values(uint32_t u, float (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(u >> (16 * i)), __NV_E4M3);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}

template <typename TOut>
__global__ void __launch_bounds__(256) k_fp8_product(Fp8GemmParams p) {
  const int n = blockIdx.x * 32 + (threadIdx.x & 31);
  for (long m = blockIdx.y * 8 + (threadIdx.x >> 5); m < p.M; m += gridDim.y * 8) {
    int e = 0;
    if (p.offsets) {
      if (p.offsets[0] != 0 || m >= p.offsets[p.E]) continue;
      int lo = 0, hi = p.E;   // the expert whose run holds row m
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.offsets[mid] <= m) lo = mid; else hi = mid;
      }
      e = lo;
    }
    if (n >= p.N) continue;
    const uint4* xr = reinterpret_cast<const uint4*>(p.x + m * p.K);
    const uint4* wr = reinterpret_cast<const uint4*>(p.w + (static_cast<long>(e) * p.N + n) * p.K);
    const uint8_t* ws = p.w_scale + (static_cast<long>(e) * ((p.N + 127) / 128) + n / 128) * p.ks;
    float y = 0.f;
    for (int b = 0; b < p.ks; ++b) {
      float part = 0.f;
      for (int c = b * 8; c < min((b + 1) * 8, p.K / 16); ++c) {
        const uint4 a = xr[c], w = wr[c];
        const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float av[4], wv[4];
          e4m3x4_values(aw[i], av);
          e4m3x4_values(ww[i], wv);
#pragma unroll
          for (int j = 0; j < 4; ++j) part = fmaf(av[j], wv[j], part);
        }
      }
      y = fmaf(part * e8m0_value(p.x_scale[m * p.ks + b]), e8m0_value(ws[b]), y);
    }
    if (p.bias) y += p.bias[static_cast<long>(e) * p.N + n];
    if constexpr (sizeof(TOut) == 2)
      static_cast<__nv_bfloat16*>(p.y)[m * p.N + n] = __float2bfloat16_rn(y);
    else
      static_cast<float*>(p.y)[m * p.N + n] = y;
  }
}

}  // namespace stamp
