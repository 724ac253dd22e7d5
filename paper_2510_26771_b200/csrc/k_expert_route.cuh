// Around the products of an expert layer: the router's choice, which gives the rows in expert order that the products take,
// and the way back, each token's rows weighted and summed.
//
// Choice: of a token's E logits the `top` largest, of equal ones the lower index, in falling order.  With m the largest and
// s_j = exp(l_j - m), the shares are s_j / sum of the chosen ones' (normalize), or s_j / sum of all.  A NaN is chosen last; a
// row with one has shares NaN.  A row of -inf alone (padding) has shares 0.
// Order: row (t, j) goes to place[t, j] = offsets[e] + how many (t', j') before it, in memory order, chose the same expert e.
#pragma once
#include "common.cuh"
#include "ptx.cuh"

namespace stamp {

constexpr int ROUTE_MAX_EXPERTS = 1024;
constexpr int ROUTE_MAX_TOP = 32;
constexpr int ROUTE_WARPS = 32;
constexpr int ROUTE_THREADS = 32 * ROUTE_WARPS;
constexpr int ROUTE_ONE_CTA_TOKENS = 128;   // up to here one CTA does it all in one launch

struct RouteParams {
  const void* logits;   // [T, ldl]
  long ldl;
  int T, E, top, normalize;
  int per_cta, per_warp;   // tokens; each CTA and warp has a run of them
  int* chosen;          // [T, top]
  float* share;         // [T, top]
  int* rows;            // [T * top] token of every row
  int* place;           // [T, top]
  int* offsets;         // [E + 1]
  float* row_share;     // [T * top]
  int* counts;          // [CTAs, E] rows of every expert from a CTA's tokens (more than one CTA)
};

// A float's bits so that they order as it does; -0 as 0, NaN below everything, 0 and 1 left free.
__device__ __forceinline__ uint32_t route_key(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  if ((b & 0x7FFFFFFFu) > 0x7F800000u) return 1u;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float route_value(uint32_t key) {
  if (key == 1u) return __int_as_float(0x7FC00000);
  return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}
__device__ __forceinline__ float route_load(const float* p) { return __ldg(p); }
__device__ __forceinline__ float route_load(const __nv_bfloat16* p) { return __bfloat162float(*p); }

// Exclusive sum over the CTA of one value per thread; `total` gets the sum.  scratch: 33 words.
__device__ __forceinline__ int route_scan(int v, int* scratch, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int sum = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, sum, d);
    if (lane >= d) sum += o;
  }
  __syncthreads();
  if (lane == 31) scratch[warp] = sum;
  __syncthreads();
  if (warp == 0) {
    int w = scratch[lane];
    const int own = w;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, w, d);
      if (lane >= d) w += o;
    }
    scratch[lane] = w - own;
    if (lane == 31) scratch[32] = w;
  }
  __syncthreads();
  total = scratch[32];
  return scratch[warp] + sum - v;
}

// Where the rows of this CTA's tokens go, given its experts' first places (base, shared memory) and each row's rank among the
// CTA's rows of the same expert (in place).
__device__ __forceinline__ void route_store(const RouteParams& p, const int* base) {
  const long first = static_cast<long>(blockIdx.x) * p.per_cta * p.top;
  const long last = min(first + static_cast<long>(p.per_cta) * p.top, static_cast<long>(p.T) * p.top);
  for (long i = first + threadIdx.x; i < last; i += ROUTE_THREADS) {
    const int at = base[p.chosen[i]] + p.place[i];
    p.place[i] = at;
    p.rows[at] = static_cast<int>(i / p.top);
    p.row_share[at] = p.share[i];
  }
}

// A warp takes one token after the other: PER logits a lane, expert 32 i + lane in register i.  Each warp counts its rows by
// expert in shared memory, and a row's rank is the count so far; the warps' counts are then summed in their order.
template <typename TIn, int PER>
__global__ void __launch_bounds__(ROUTE_THREADS) k_expert_choose(RouteParams p) {
  extern __shared__ int route_counts[];   // [ROUTE_WARPS][E] rows by warp and expert, then base [E]
  __shared__ int scratch[33];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int* const mine = route_counts + warp * p.E;
  for (int e = lane; e < p.E; e += 32) mine[e] = 0;
  __syncwarp();
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();

  const long cta_end = min((static_cast<long>(blockIdx.x) + 1) * p.per_cta, static_cast<long>(p.T));
  const long t0 = static_cast<long>(blockIdx.x) * p.per_cta + static_cast<long>(warp) * p.per_warp;
  for (long t = t0; t < min(t0 + p.per_warp, cta_end); ++t) {
    const TIn* at = static_cast<const TIn*>(p.logits) + t * p.ldl + lane;
    uint32_t key[PER];
    float l[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) l[i] = 32 * i + lane < p.E ? route_load(at + 32 * i) : -__int_as_float(0x7F800000);
    bool nan = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      key[i] = 32 * i + lane < p.E ? route_key(l[i]) : 0u;
      nan |= key[i] == 1u;
    }
    nan = __any_sync(0xffffffffu, nan);
    int expert = 0;        // lane j: choice j
    uint32_t best = 0u;
    for (int j = 0; j < p.top; ++j) {
      uint32_t most = key[0];
#pragma unroll
      for (int i = 1; i < PER; ++i) most = max(most, key[i]);
      most = __reduce_max_sync(0xffffffffu, most);
      int e = 0x7FFFFFFF;
#pragma unroll
      for (int i = PER - 1; i >= 0; --i)
        if (key[i] == most) e = 32 * i + lane;
      e = __reduce_min_sync(0xffffffffu, e);
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (32 * i + lane == e) key[i] = 0u;
      if (lane == j) expert = e, best = most;
    }
    const float largest = route_value(__shfl_sync(0xffffffffu, best, 0));
    const bool dead = !nan && largest == -__int_as_float(0x7F800000);
    const float weight = lane < p.top ? expf(route_value(best) - largest) : 0.f;
    float total = weight;
    if (!p.normalize) {
      total = 0.f;
#pragma unroll
      for (int i = 0; i < PER; ++i) total += expf(l[i] - largest);   // (lanes without an expert: exp(-inf))
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
    if (lane < p.top) {
      const long i = t * p.top + lane;
      p.chosen[i] = expert;
      p.share[i] = nan ? __int_as_float(0x7FC00000) : dead ? 0.f : weight / total;
      p.place[i] = mine[expert]++;   // (a token's choices differ)
    }
    __syncwarp();
  }
  __syncthreads();
  // rows of the warps before, by expert; and this CTA's
  int* const base = route_counts + ROUTE_WARPS * p.E;
  for (int e = threadIdx.x; e < p.E; e += ROUTE_THREADS) {
    int sum = 0;
#pragma unroll
    for (int w = 0; w < ROUTE_WARPS; ++w) {
      const int c = route_counts[w * p.E + e];
      route_counts[w * p.E + e] = sum;
      sum += c;
    }
    base[e] = sum;
    if (gridDim.x > 1) p.counts[static_cast<long>(blockIdx.x) * p.E + e] = sum;
  }
  __syncthreads();
  for (long t = t0; t < min(t0 + p.per_warp, cta_end); ++t)
    if (lane < p.top) p.place[t * p.top + lane] += mine[p.chosen[t * p.top + lane]];
  if (gridDim.x > 1) return;
  int total;
  const int e = threadIdx.x;
  static_assert(ROUTE_MAX_EXPERTS <= ROUTE_THREADS, "one thread for every expert");
  const int first = route_scan(e < p.E ? base[e] : 0, scratch, total);
  if (e < p.E) {
    base[e] = first;
    p.offsets[e] = first;
  }
  if (e == 0) p.offsets[p.E] = total;
  __syncthreads();
  route_store(p, base);
}

// The second launch where several CTAs chose: every expert's first place, from the counts of all CTAs; then the rows.
__global__ void __launch_bounds__(ROUTE_THREADS) k_expert_place(RouteParams p) {
  extern __shared__ int route_counts[];   // base [E], then sums [ROUTE_THREADS] twice
  __shared__ int scratch[33];
  int* const base = route_counts;
  int* const before_of = base + p.E;
  int* const all_of = before_of + ROUTE_THREADS;
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  // threads in groups of `width` >= E, each of which sums a share of the CTAs
  int width = 32;
  while (width < p.E) width *= 2;
  const int groups = ROUTE_THREADS / width, g = threadIdx.x / width, e = threadIdx.x % width;
  int before = 0, all = 0;   // rows of expert e from the CTAs before this one, and from all
  if (e < p.E) {
#pragma unroll 8
    for (int b = g; b < static_cast<int>(gridDim.x); b += groups) {
      const int c = __ldg(p.counts + static_cast<long>(b) * p.E + e);
      all += c;
      before += b < static_cast<int>(blockIdx.x) ? c : 0;
    }
  }
  before_of[threadIdx.x] = before;
  all_of[threadIdx.x] = all;
  __syncthreads();
  if (g == 0) {
    for (int o = 1; o < groups; ++o) {
      before += before_of[o * width + e];
      all += all_of[o * width + e];
    }
  } else {
    all = 0;
  }
  int total;
  const int first = route_scan(all, scratch, total);   // (thread e < E: expert e; the others add nothing)
  if (g == 0 && e < p.E) {
    base[e] = first + before;
    if (blockIdx.x == 0) p.offsets[e] = first;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) p.offsets[p.E] = total;
  __syncthreads();
  route_store(p, base);
}

// ---- the way back: out[t] = sum_j share[t, j] y[place[t, j]] + residual[t], in fp32 in the order of j, rounded once.
// A place outside [0, M) adds nothing and raises the device status word.
struct CombineParams {
  const void* y;          // [M, N]
  const int* place;       // [T, top]
  const float* share;     // [T, top]
  const void* residual;   // [T, ldr] or nullptr
  long ldr;
  int T, top, M, N;
  void* out;              // [T, N]
};
constexpr int COMBINE_THREADS = 128;

template <typename T, int V>
struct Packed {};
template <>
struct Packed<float, 4> { using type = float4; };
template <>
struct Packed<__nv_bfloat16, 4> { using type = uint2; };
template <>
struct Packed<float, 1> { using type = float; };
template <>
struct Packed<__nv_bfloat16, 1> { using type = __nv_bfloat16; };

__device__ __forceinline__ void unpack(const float4& u, float (&v)[4]) { v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w; }
__device__ __forceinline__ void unpack(const uint2& u, float (&v)[4]) {
  v[0] = __uint_as_float(u.x << 16), v[1] = __uint_as_float(u.x & 0xFFFF0000u);
  v[2] = __uint_as_float(u.y << 16), v[3] = __uint_as_float(u.y & 0xFFFF0000u);
}
__device__ __forceinline__ void unpack(const float& u, float (&v)[1]) { v[0] = u; }
__device__ __forceinline__ void unpack(const __nv_bfloat16& u, float (&v)[1]) { v[0] = __bfloat162float(u); }
__device__ __forceinline__ void pack(const float (&v)[4], float4& u) { u = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void pack(const float (&v)[4], uint2& u) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
  u = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
__device__ __forceinline__ void pack(const float (&v)[1], float& u) { u = v[0]; }
__device__ __forceinline__ void pack(const float (&v)[1], __nv_bfloat16& u) { u = __float2bfloat16_rn(v[0]); }

// A thread takes V neighbouring channels of one token; four of the token's rows are in flight at a time.
// grid (T, ceil(N / (COMBINE_THREADS V)))
template <typename TIn, typename TOut, int V>
__global__ void __launch_bounds__(COMBINE_THREADS) k_expert_combine(CombineParams p, int r_bf16) {
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const long t = blockIdx.x, c = (static_cast<long>(blockIdx.y) * COMBINE_THREADS + threadIdx.x) * V;
  if (c >= p.N) return;
  using In = typename Packed<TIn, V>::type;
  using Out = typename Packed<TOut, V>::type;
  float sum[V], v[V];
#pragma unroll
  for (int i = 0; i < V; ++i) sum[i] = 0.f;
  for (int j0 = 0; j0 < p.top; j0 += 4) {
    In raw[4];
    float share[4];
    bool live[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      live[j] = j0 + j < p.top;
      if (!live[j]) continue;
      const int at = __ldg(p.place + t * p.top + j0 + j);
      share[j] = __ldg(p.share + t * p.top + j0 + j);
      if (at < 0 || at >= p.M) {
        live[j] = false;
        raise_device_status(STAMP_ERR_INVALID_ARG);
        continue;
      }
      raw[j] = *reinterpret_cast<const In*>(static_cast<const TIn*>(p.y) + static_cast<long>(at) * p.N + c);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (!live[j]) continue;
      unpack(raw[j], v);
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] = fmaf(share[j], v[i], sum[i]);
    }
  }
  if (p.residual) {
    const long at = t * p.ldr + c;
    if (r_bf16)
      unpack(*reinterpret_cast<const typename Packed<__nv_bfloat16, V>::type*>(static_cast<const __nv_bfloat16*>(p.residual) + at), v);
    else
      unpack(*reinterpret_cast<const typename Packed<float, V>::type*>(static_cast<const float*>(p.residual) + at), v);
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] += v[i];
  }
  Out o;
  pack(sum, o);
  *reinterpret_cast<Out*>(static_cast<TOut*>(p.out) + t * p.N + c) = o;
}

}  // namespace stamp
