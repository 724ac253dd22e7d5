// A whole expert layer for a few tokens, activations as they are:
//   h[m, f] = silu(g) u,  g = w_up[e, f] . x[rows[m]] + b_up[e, f],  u the same for row F + f      (e: the expert of row m)
//   y[t]    = residual[t] + sum over the rows m of token t of share[m] (w_down[e] h[m] + b_down[e])
#pragma once
#include <cuda_fp8.h>

#include "common.cuh"
#include "k_fp8_quant.cuh"
#include "ptx.cuh"

namespace stamp {

constexpr int EXPERT_FEW_TOKENS = 64;
constexpr int EXPERT_FEW_ROWS = 2048;
constexpr int EXPERT_MAX = 1024;

struct ExpertParams {
  const void* x;            // [T, ldx]
  long ldx;
  int x_bf16;
  const int* rows;          // [M] token of every row
  const float* share;       // [M]
  const int* offsets;       // [E + 1]
  const uint8_t *w_up, *up_scale, *w_down, *down_scale;   // [E, 2 F, K], [E, N, F]
  const float *up_bias, *down_bias;                       // [E, 2 F], [E, N] or nullptr
  const void* residual;     // [T, ldr] or nullptr
  long ldr;
  int r_bf16;
  int T, M, E, K, F, N;
  float* h;                 // [M, F]
  void* y;                  // [T, N]
};

__device__ __forceinline__ float expert_e4m3(uint8_t c) {
  __half_raw h = __nv_cvt_fp8_to_halfraw(c, __NV_E4M3);
  return __half2float(__half(h));
}
__device__ __forceinline__ float expert_scale(uint8_t b) { return b == 255 ? __int_as_float(0x7FC00000) : exp2f(static_cast<float>(b) - 127.f); }
__device__ __forceinline__ bool expert_offsets_ok(const ExpertParams& p) {
  bool bad = false;
  for (int e = threadIdx.x; e <= p.E; e += blockDim.x) {
    const int o = p.offsets[e];
    bad |= o < 0 || o > p.M || (e == 0 ? o != 0 : o < p.offsets[e - 1]);
  }
  bad = __syncthreads_or(bad);
  if (bad && threadIdx.x == 0) raise_device_status(STAMP_ERR_INVALID_ARG);
  return !bad;
}
__device__ __forceinline__ int expert_of(const ExpertParams& p, int m) {
  int lo = 0, hi = p.E;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p.offsets[mid] <= m) lo = mid; else hi = mid;
  }
  return lo;
}
__device__ __forceinline__ float expert_warp_sum(float v) {
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}

// One warp for each row and hidden channel.
__global__ void __launch_bounds__(256) k_expert_up_plain(ExpertParams p) {
  if (!expert_offsets_ok(p)) return;
  const int lane = threadIdx.x & 31, m = blockIdx.y, f = blockIdx.x * 8 + (threadIdx.x >> 5);
  if (m >= p.offsets[p.E] || f >= p.F) return;
  const int t = p.rows[m];
  if (t < 0 || t >= p.T) {
    if (lane == 0) raise_device_status(STAMP_ERR_INVALID_ARG);
    return;
  }
  const int e = expert_of(p, m), ks = (p.K + 127) / 128, nb = (2 * p.F + 127) / 128;
  float sum[2];
  for (int half = 0; half < 2; ++half) {
    const int ch = half * p.F + f;
    const uint8_t* w = p.w_up + (static_cast<long>(e) * 2 * p.F + ch) * p.K;
    const uint8_t* ws = p.up_scale + (static_cast<long>(e) * nb + ch / 128) * ks;
    float s = 0.f;
    for (int k = lane; k < p.K; k += 32) {
      const float x = p.x_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.x)[t * p.ldx + k]) : static_cast<const float*>(p.x)[t * p.ldx + k];
      s = fmaf(x, expert_e4m3(w[k]) * expert_scale(ws[k / 128]), s);
    }
    sum[half] = expert_warp_sum(s) + (p.up_bias ? p.up_bias[static_cast<long>(e) * 2 * p.F + ch] : 0.f);
  }
  if (lane == 0) p.h[static_cast<long>(m) * p.F + f] = sum[0] / (1.f + expf(-sum[0])) * sum[1];
}

// One warp for each token and output channel.
template <typename TOut>
__global__ void __launch_bounds__(256) k_expert_down_plain(ExpertParams p) {
  if (!expert_offsets_ok(p)) return;
  const int lane = threadIdx.x & 31, t = blockIdx.y, n = blockIdx.x * 8 + (threadIdx.x >> 5);
  if (n >= p.N) return;
  const int ks = (p.F + 127) / 128, nb = (p.N + 127) / 128;
  float y = 0.f;
  for (int m = 0; m < p.offsets[p.E]; ++m) {
    if (p.rows[m] != t) continue;
    const int e = expert_of(p, m);
    const uint8_t* w = p.w_down + (static_cast<long>(e) * p.N + n) * p.F;
    const uint8_t* ws = p.down_scale + (static_cast<long>(e) * nb + n / 128) * ks;
    float s = 0.f;
    for (int k = lane; k < p.F; k += 32) s = fmaf(p.h[static_cast<long>(m) * p.F + k], expert_e4m3(w[k]) * expert_scale(ws[k / 128]), s);
    y += p.share[m] * (expert_warp_sum(s) + (p.down_bias ? p.down_bias[static_cast<long>(e) * p.N + n] : 0.f));
  }
  if (lane == 0) {
    if (p.residual) {
      const long at = t * p.ldr + n;
      y += p.r_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.residual)[at]) : static_cast<const float*>(p.residual)[at];
    }
    TOut* out = static_cast<TOut*>(p.y) + static_cast<long>(t) * p.N + n;
    if constexpr (sizeof(TOut) == 2) *out = __float2bfloat16_rn(y); else *out = y;
  }
}

}  // namespace stamp
