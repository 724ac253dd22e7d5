// A whole expert layer for a few tokens in two kernels, activations as they are:
//   h[m, f] = silu(g) u,  g = w_up[e, f] . x[rows[m]] + up_bias[e, f],  u the same for row F + f      (e: the expert of row m)
//   y[t]    = residual[t] + sum over the rows m of token t of share[m] (w_down[e] h[m] + down_bias[e])
//
// With few tokens a layer is the way of its weights from memory: each byte is read once and meets a handful of rows.  The
// weights are e4m3 already, so they go by TMA to shared memory and from there into the block-scaled tensor instruction
// (kind::mxf8f6f4, channels on the TMEM lanes, rows as columns) without passing a register.  The activations are not e4m3;
// quantizing them would be the layer's largest error and saves nothing here.  They are written as a sum of e4m3 terms
// instead, each with its own power-of-two scale for a block of 128:
//   v = c0 s + c1 s 2^-4 + c2 s 2^-9 + c3 s 2^-14,   s the quantizer's scale of the block, c_i the nearest e4m3 number to
//   what is left.  The first term is off by at most 2^-4 of v (16 s at the top of the range, hence the step to 2^-4), every
//   further one by 2^-5 of what was left: two terms hold the 8 significant bits of a bf16 value, three 2^-14, four 2^-19.  Values
//   more than 2^14 below their block's largest keep an error of 2^-24 of that.
// A term is a column of the product like any other row's, so the terms cost columns (16 at least in any case), not another
// pass over the weights; the epilogue adds them up.  bf16 tokens take two terms, fp32 ones four, the hidden values three for a
// bf16 output and four for an fp32 one.
//
//   warps 0-3   epilogue, one TMEM lane (output channel) a thread
//   warp 4      TMA producer: 128 channels x 128 features of weights (UP: of gates and of ups) into a ring of stages
//   warp 5      allocates TMEM, copies the scale words to it and issues the MMAs
//   warps 6-13  converters: the rows' terms and all scales.  As many warps for each stage of the ring as eight allow, always the
//               same ones: who fills a stage has filled it the time before too, so that the parity it waits for is never
//               an older one's, and it can load the stage's next rows as soon as it is through with the last
// Every wait is bounded; when one expires the CTA raises the device status word, unwinds and frees its TMEM.
//
// UP: a CTA takes one run (up to `cap` rows of one expert), 128 gates and the 128 ups that go with them, and, in a cluster of
// `split`, a share of the features; the partial sums are added over distributed shared memory in rank order.
// DOWN: a cluster takes 128 output channels and all runs; its CTAs share the sequence of all (run, 128 features).  A CTA adds
// each run's rows, weighted, to its tokens in shared memory in the order of the rows; the CTAs' sums are added in rank order,
// with the residual.  No atomics on results, nothing in memory but the hidden values, and every result repeats bit for bit.
// DOWN is launched as a programmatic dependent of UP: it needs less than half of an SM's shared memory, as UP does, so its
// first weights are on their way while UP's last CTAs run; only its converters wait for the hidden values.
#pragma once
#include "common.cuh"
#include "k_fp8_gemm.cuh"
#include "k_fp8_quant.cuh"
#include "ptx.cuh"

namespace stamp {

constexpr int EXPERT_FEW_TOKENS = 64;
constexpr int EXPERT_FEW_ROWS = 2048;
constexpr int EXPERT_MAX = 1024;
constexpr int EXPERT_CONVERTERS = 8;
constexpr int EXPERT_THREADS = 32 * (6 + EXPERT_CONVERTERS);
constexpr int EXPERT_MAX_STAGES = 8;
constexpr int EXPERT_W_BYTES = 128 * 128;
constexpr int EXPERT_SMEM = 112 * 1024;                 // of a CTA: two to an SM

struct ExpertParams {
  const void* x;            // [T, ldx] bf16 or float
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
  // one kernel's plan
  int terms, cap;           // terms of a row; rows of a run at most (a multiple of 8, terms * cap <= columns)
  int split;                // CTAs of a cluster
  int stages, stage_bytes;
};

template <bool UP>
struct ExpertSmem {
  static constexpr int COLUMNS = UP ? 64 : 96;          // of one accumulator
  static constexpr int SF_BYTES = UP ? 1536 : 1024;     // scale words of a stage: channels (UP: twice), then rows
  static constexpr int SF_COLS = SF_BYTES / 128;
  static constexpr int SF_COL = 2 * COLUMNS;            // tensor memory: two accumulators (UP: gates, ups), then the stages' scales
  static_assert(SF_COL + EXPERT_MAX_STAGES * SF_COLS <= 256, "half of the tensor memory: two CTAs to an SM");
  static constexpr int BARS = 2 * EXPERT_MAX_STAGES + 4;
  // after the ring and the scale words: barriers, [tmem, abort, runs, bad], run tables, DOWN: sums [T][128]
  __host__ __device__ static constexpr int tables(int max_runs) { return BARS * 8 + 16 + (max_runs * 8 + 15) / 16 * 16; }
  __host__ __device__ static int fixed(int max_runs, int T) { return 1024 + tables(max_runs) + (UP ? 0 : T * 512); }
};

// Runs at most: an expert's rows end in one part run, and no more experts than rows have any.
__host__ __device__ __forceinline__ int expert_max_runs(int M, int E, int cap) { return (E < M ? E : M) + M / cap; }

struct ExpertRun {
  int row0;
  uint16_t expert, n;
};

__device__ __forceinline__ float2 expert_e4m3x2(uint32_t two) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(two)));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// Four neighbouring features of a row, as loaded.
struct ExpertRaw {
  uint4 u;
  __device__ __forceinline__ void load(const void* base, long at, bool bf16, bool live) {
    u = make_uint4(0u, 0u, 0u, 0u);
    if (!live) return;
    if (bf16) {
      const uint2 v = __ldcg(reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(base) + at));
      u.x = v.x, u.y = v.y;
    } else {
      u = __ldcg(reinterpret_cast<const uint4*>(static_cast<const float*>(base) + at));
    }
  }
  __device__ __forceinline__ void values(bool bf16, float (&v)[4]) const {
    if (bf16) {
      v[0] = __uint_as_float(u.x << 16), v[1] = __uint_as_float(u.x & 0xFFFF0000u);
      v[2] = __uint_as_float(u.y << 16), v[3] = __uint_as_float(u.y & 0xFFFF0000u);
    } else {
      v[0] = __uint_as_float(u.x), v[1] = __uint_as_float(u.y), v[2] = __uint_as_float(u.z), v[3] = __uint_as_float(u.w);
    }
  }
};

// One row's 128 features (four a lane) as terms: codes to row `row` of the operand tile (128-byte rows, 128-byte swizzle) and,
// for each further term, `pitch` rows further; scale words to the order tmem_copy_scales wants.
__device__ __forceinline__ void expert_convert(const float (&value)[4], int terms, int row, int pitch, uint8_t* tile, uint8_t* words) {
  const int lane = threadIdx.x & 31;
  const float most = ptx::warp_max_abs(ptx::max_abs_nan(ptx::max_abs_nan(value[0], value[1], value[2]), value[3], 0.f));
  const Fp8Scale s = fp8_scale(__float_as_uint(most));
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = value[i] * s.inverse;
  uint32_t byte = s.byte, mine = 0u;
  uint8_t* out = tile + row * 128 + (((lane >> 2) ^ (row & 7)) << 4) + ((lane & 3) << 2);   // (pitch is a multiple of 8)
  for (int t = 0;;) {
    const uint32_t c = ptx::cvt_e4m3x4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<uint32_t*>(out) = c;
    if (lane == t) mine = byte;
    if (++t == terms) break;
    out += pitch * 128;
    // what is left, in units of the next term's scale (which stops at 2^-127; a NaN's terms are all NaN)
    const uint32_t shift = min(t == 1 ? 4u : 5u, byte);
    const float up = __uint_as_float((127u + shift) << 23);
    const float2 a = expert_e4m3x2(c), b = expert_e4m3x2(c >> 16);
    v[0] = (v[0] - a.x) * up, v[1] = (v[1] - a.y) * up, v[2] = (v[2] - b.x) * up, v[3] = (v[3] - b.y) * up;
    if (byte != 255u) byte -= shift;
  }
  if (lane < terms) {
    const int r = row + lane * pitch;
    *reinterpret_cast<uint32_t*>(words + ((r & 31) << 4) + ((r >> 5) << 2)) = mine * 0x01010101u;
  }
}

template <bool UP, typename TOut>
__global__ void __launch_bounds__(EXPERT_THREADS, 2)
    k_expert_layer(const __grid_constant__ CUtensorMap tmap, ExpertParams p) {
  using SM = ExpertSmem<UP>;
  extern __shared__ uint8_t expert_raw[];
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(expert_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* const words = smem + p.stages * p.stage_bytes;
  uint64_t* const full = reinterpret_cast<uint64_t*>(words + p.stages * SM::SF_BYTES);
  uint64_t* const empty = full + EXPERT_MAX_STAGES;
  uint64_t* const tfull = empty + EXPERT_MAX_STAGES;
  uint64_t* const tempty = tfull + 2;
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(tempty + 2);
  volatile uint32_t* const abort_word = tmem_slot + 1;
  int* const run_count = reinterpret_cast<int*>(tmem_slot + 2);   // -1: the offsets are out of order
  ExpertRun* const run_table = reinterpret_cast<ExpertRun*>(tmem_slot + 4);
  const int max_runs = expert_max_runs(p.M, p.E, p.cap);
  float* const sums = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(full) + SM::tables(max_runs));

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = p.split > 1 ? static_cast<int>(ptx::cluster_ctarank()) : 0;
  const int unit = blockIdx.x / p.split;
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      ptx::mbar_init(&full[s], 1 + EXPERT_CONVERTERS / p.stages);
      ptx::mbar_init(&empty[s], UP ? 2 : 1);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(&tfull[a], 1);
      ptx::mbar_init(&tempty[a], 4);
    }
    *abort_word = 0;
    ptx::fence_mbar_init();
    ptx::prefetch_tensormap(&tmap);
  }
  if (warp == 5) {
    ptx::tmem_alloc(tmem_slot, 256);
    ptx::tmem_relinquish();
  }
  if constexpr (!UP) {
    for (int i = threadIdx.x; i < p.T * 128; i += EXPERT_THREADS) sums[i] = 0.f;
  }
  // UP waits for what came before it.  DOWN starts when every CTA of UP has come past this point: what UP waited for is there
  // for DOWN too, and only the hidden values are to be waited for.  (Where no row exists, DOWN is alone and waits.)
  if (UP || p.M == 0) ptx::grid_dependency_wait();
  if constexpr (UP) ptx::grid_launch_dependents();
  if (warp == 4) {
    bool bad = false;
    int runs = 0;
    for (int e0 = 0; e0 < p.E; e0 += 32) {
      const int e = e0 + lane;
      const int first = e <= p.E ? __ldcg(p.offsets + e) : 0, last = e < p.E ? __ldcg(p.offsets + e + 1) : first;
      bad |= e < p.E && (first < 0 || last > p.M || last < first || (e == 0 && first != 0));
      if (__any_sync(0xffffffffu, bad)) {
        bad = true;
        break;
      }
      const int own = (last - first + p.cap - 1) / p.cap;
      int before = own;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, before, d);
        if (lane >= d) before += v;
      }
      const int at = runs + before - own;
      for (int i = 0; i < own; ++i)
        run_table[at + i] = ExpertRun{first + i * p.cap, static_cast<uint16_t>(e), static_cast<uint16_t>(min(p.cap, last - first - i * p.cap))};
      runs += __shfl_sync(0xffffffffu, before, 31);
    }
    if (lane == 0) {
      *run_count = bad ? -1 : runs;
      if (bad) raise_device_status(STAMP_ERR_INVALID_ARG);
    }
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int runs = *run_count;

  // What this CTA sums: UP one run's share of the features; DOWN its share of the sequence of (run, 128 features).
  const int blocks = ((UP ? p.K : p.F) + 127) / 128;                       // of one run
  const int tiles = UP ? (p.F + 127) / 128 : 1;
  const int run0 = UP ? unit / tiles : 0, tile = UP ? unit - run0 * tiles : unit;
  const bool idle = runs <= 0 || (UP && run0 >= runs);
  const long all = UP ? blocks : static_cast<long>(runs) * blocks, base = UP ? static_cast<long>(run0) * blocks : 0;
  const int u0 = idle ? 0 : static_cast<int>(base + all * rank / p.split), u1 = idle ? 0 : static_cast<int>(base + all * (rank + 1) / p.split);
  struct Segment {
    int kb0, kb1;
    ExpertRun run;
  };
  auto segment_at = [&](int u) {   // the part of one run that starts at u
    const int r = u / blocks, kb0 = u - r * blocks;
    return Segment{kb0, min(blocks, kb0 + u1 - u), run_table[r]};
  };
  const auto padded = [](int n) { return (n + 7) & ~7; };

  if (warp == 4) {
    // ------------------------------------------------------------------ TMA producer
    if (ptx::elect_one()) {
      int stage = 0;
      uint32_t phase = 0, issued = 0;
      bool ok = true;
      for (int u = u0; u < u1 && ok;) {
        const Segment g = segment_at(u);
        const int row = g.run.expert * (UP ? 2 * p.F : p.N) + tile * 128;
        for (int kb = g.kb0; kb < g.kb1; ++kb) {
          if (!ptx::mbar_wait_bounded_sleepy(&empty[stage], phase ^ 1u, abort_word, FP8G_WAIT_LIMIT)) {
            ok = false;
            break;
          }
          uint8_t* const dst = smem + stage * p.stage_bytes;
          ptx::mbar_arrive_expect_tx(&full[stage], (UP ? 2 : 1) * EXPERT_W_BYTES);
          ++issued;
          ptx::tma_load_2d(dst, &tmap, &full[stage], kb * 128, row);
          if constexpr (UP) ptx::tma_load_2d(dst + EXPERT_W_BYTES, &tmap, &full[stage], kb * 128, row + p.F);
          if (++stage == p.stages) stage = 0, phase ^= 1u;
        }
        u += g.kb1 - g.kb0;
      }
      if (!ok) {
        *abort_word = 1;
        raise_device_status(STAMP_ERR_TIMEOUT);
        // let the copies in flight land before the shared memory goes away (their barriers may lack the converters' arrival)
        const long long t0 = clock64();
        while (issued > 0 && clock64() - t0 < 2000000LL) {
        }
      }
    }
  } else if (warp == 5) {
    // ------------------------------------------------------------------ MMA issuer
    if (ptx::elect_one()) {
      constexpr uint32_t idesc0 = ptx::make_mxf8_idesc(128);
      int stage = 0, it = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int u = u0; u < u1 && ok; ++it) {
        const Segment g = segment_at(u);
        const uint32_t idesc = ptx::mxf8_idesc_with(idesc0, (p.terms * padded(g.run.n) + 15) & ~15);
        const int a = UP ? 0 : it & 1;
        if (!UP && !ptx::mbar_wait_bounded(&tempty[a], ((it >> 1) & 1) ^ 1, abort_word, FP8G_WAIT_LIMIT)) {
          ok = false;
          break;
        }
        ptx::tc_fence_after();
        const uint32_t acc = tmem + static_cast<uint32_t>(a * SM::COLUMNS);
        for (int kb = g.kb0; kb < g.kb1; ++kb) {
          if (!ptx::mbar_wait_bounded(&full[stage], phase, abort_word, FP8G_WAIT_LIMIT)) {
            ok = false;
            break;
          }
          ptx::tc_fence_after();
          const uint32_t w = ptx::smem_u32(smem + stage * p.stage_bytes), sf = ptx::smem_u32(words + stage * SM::SF_BYTES);
          const uint32_t sfc = tmem + static_cast<uint32_t>(SM::SF_COL + stage * SM::SF_COLS);
          const uint32_t bar = ptx::smem_u32(&empty[stage]), w_low = ptx::sw128_desc_low(w);
          ptx::tmem_copy_scales<false>(sfc, ptx::make_rows16_desc(sf));
          ptx::tmem_copy_scales<false>(sfc + 4, ptx::make_rows16_desc(sf + 512));
          if constexpr (UP) {
            ptx::tmem_copy_scales<false>(sfc + 8, ptx::make_rows16_desc(sf + 1024));
            const uint32_t x_low = w_low + (2 * EXPERT_W_BYTES >> 4);
            ptx::mma_mxf8_128<false>(acc, w_low, x_low, idesc, sfc, sfc + 8, kb > g.kb0 ? 1u : 0u, bar);
            ptx::mma_mxf8_128<false>(acc + SM::COLUMNS, w_low + (EXPERT_W_BYTES >> 4), x_low, idesc, sfc + 4, sfc + 8, kb > g.kb0 ? 1u : 0u, bar);
          } else {
            ptx::mma_mxf8_128<false>(acc, w_low, w_low + (EXPERT_W_BYTES >> 4), idesc, sfc, sfc + 4, kb > g.kb0 ? 1u : 0u, bar);
          }
          if (++stage == p.stages) stage = 0, phase ^= 1u;
        }
        if (!ok) break;
        ptx::tc_commit(&tfull[a]);
        u += g.kb1 - g.kb0;
      }
      if (!ok) {
        *abort_word = 1;
        raise_device_status(STAMP_ERR_TIMEOUT);
      }
    }
  } else if (warp >= 6) {
    // ------------------------------------------------------------------ converters
    if (!UP && p.M > 0) {
      ptx::grid_dependency_wait();
      ptx::grid_launch_dependents();
    }
    const int features = UP ? p.K : p.F;
    const bool bf16 = UP && p.x_bf16;
    const void* const src = UP ? p.x : p.h;
    const long ld = UP ? p.ldx : p.F;
    const uint8_t* const scales = UP ? p.up_scale : p.down_scale;
    const int scale_rows = ((UP ? 2 * p.F : p.N) + 127) / 128;
    const int up_first = UP ? (p.F + tile * 128) >> 7 : 0, up_rest = UP ? 128 - ((p.F + tile * 128) & 127) : 0;
    const int each = EXPERT_CONVERTERS / p.stages;   // warps of a stage; they share its rows
    const int stage = (warp - 6) / each, part = (warp - 6) % each;
    int i = 0, s = stage;   // steps before this segment; the next one that goes to this warp's stage
    uint32_t phase = 0;
    bool ok = true;
    for (int u = u0; u < u1 && ok && stage < p.stages;) {
      const Segment g = segment_at(u);
      const int n = g.run.n, pitch = padded(n);
      int token = -1;   // lane r: where row r of the run is read
      if (lane < n) {
        token = UP ? __ldcg(p.rows + g.run.row0 + lane) : g.run.row0 + lane;
        if (UP && (token < 0 || token >= p.T)) {
          if (tile == 0 && rank == 0 && warp == 6) raise_device_status(STAMP_ERR_INVALID_ARG);
          token = -1;
        }
      }
      const uint8_t* const sc = scales + static_cast<long>(g.run.expert) * scale_rows * blocks;
      for (; s < i + g.kb1 - g.kb0; s += p.stages, phase ^= 1u) {
        const int kb = g.kb0 + s - i;
        const int col = kb * 128 + lane * 4;
        // everything the stage needs is loaded before it is waited for, as far as eight rows for each warp
        ExpertRaw raw[8];
        auto load = [&](int r0) {
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            const int t = __shfl_sync(0xffffffffu, token, (r0 + r * each) & 31);
            raw[r].load(src, t * ld + col, bf16, r0 + r * each < n && t >= 0 && col < features);
          }
        };
        load(part);
        uint32_t w0, w1 = 0, w2 = 0;
        if constexpr (UP) {
          w0 = __ldcg(sc + static_cast<long>(tile) * blocks + kb);
          w1 = __ldcg(sc + static_cast<long>(up_first) * blocks + kb);
          w2 = __ldcg(sc + static_cast<long>(min(up_first + 1, scale_rows - 1)) * blocks + kb);
        } else {
          w0 = __ldcg(sc + static_cast<long>(tile) * blocks + kb);
        }
        if (!__all_sync(0xffffffffu, ptx::mbar_wait_bounded_sleepy(&empty[stage], phase ^ 1u, abort_word, FP8G_WAIT_LIMIT))) {
          ok = false;
          break;
        }
        uint8_t* const xt = smem + stage * p.stage_bytes + (UP ? 2 : 1) * EXPERT_W_BYTES;
        uint8_t* const sf = words + stage * SM::SF_BYTES;
        if (part == 0) {
          w0 *= 0x01010101u;
          *reinterpret_cast<uint4*>(sf + lane * 16) = make_uint4(w0, w0, w0, w0);
          if constexpr (UP) {
            // the ups may start inside a block of the scales
            w1 *= 0x01010101u, w2 *= 0x01010101u;
            *reinterpret_cast<uint4*>(sf + 512 + lane * 16) =
                make_uint4(lane < up_rest ? w1 : w2, lane + 32 < up_rest ? w1 : w2, lane + 64 < up_rest ? w1 : w2, lane + 96 < up_rest ? w1 : w2);
          }
        }
        for (int r0 = part; r0 < n;) {
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            if (r0 + r * each >= n) break;
            float v[4];
            raw[r].values(bf16, v);
            expert_convert(v, p.terms, r0 + r * each, pitch, xt, sf + SM::SF_BYTES - 512);
          }
          r0 += 8 * each;
          if (r0 < n) load(r0);
        }
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&full[stage]);
      }
      i += g.kb1 - g.kb0;
      u += g.kb1 - g.kb0;
    }
    if (!ok) {
      *abort_word = 1;
      if (lane == 0) raise_device_status(STAMP_ERR_TIMEOUT);
    }
  } else {
    // ------------------------------------------------------------------ epilogue warps
    const int ch = warp * 32 + lane;
    bool ok = true;
    int it = 0;
    // eight rows' sums at this thread's channel, their terms added up
    auto eight = [&](uint32_t acc, int pitch, float (&v)[8]) {
#pragma unroll
      for (int r = 0; r < 8; ++r) v[r] = 0.f;
      for (int t = p.terms - 1; t >= 0; --t) {   // the smallest first
        uint32_t c[8];
        ptx::tmem_ld_32x32b_x8(acc + t * pitch, c);
        ptx::tmem_ld_wait();
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r] += __uint_as_float(c[r]);
      }
    };
    for (int u = u0; u < u1; ++it) {
      const Segment g = segment_at(u);
      const int n = g.run.n, pitch = padded(n), a = UP ? 0 : it & 1;
      int token = -1;
      float share = 0.f;
      if (!UP && lane < n) {
        token = __ldcg(p.rows + g.run.row0 + lane);
        share = __ldcg(p.share + g.run.row0 + lane);
        if (token < 0 || token >= p.T) token = -1;
      }
      float bias = 0.f;   // (once for every row: with the run's first features)
      if (!UP && p.down_bias && g.kb0 == 0 && tile * 128 + ch < p.N) bias = __ldcg(p.down_bias + static_cast<long>(g.run.expert) * p.N + tile * 128 + ch);
      if (!__all_sync(0xffffffffu, ptx::mbar_wait_bounded_sleepy(&tfull[a], UP ? 0u : (it >> 1) & 1, abort_word, FP8G_WAIT_LIMIT))) {
        ok = false;
        break;
      }
      ptx::tc_fence_after();
      const uint32_t acc = tmem + (static_cast<uint32_t>(warp * 32) << 16) + static_cast<uint32_t>(a * SM::COLUMNS);
      for (int r0 = 0; r0 < n; r0 += 8) {
        if constexpr (UP) {
          // every CTA's part of the sums, [row][gates, ups], in the ring that nothing uses any more
          float* const part = reinterpret_cast<float*>(smem);
          float v[8], w[8];
          eight(acc + r0, pitch, v);
          eight(acc + SM::COLUMNS + r0, pitch, w);
#pragma unroll
          for (int r = 0; r < 8; ++r)
            if (r0 + r < n) {
              part[(r0 + r) * 256 + ch] = v[r];
              part[(r0 + r) * 256 + 128 + ch] = w[r];
            }
        } else {
          float v[8];
          eight(acc + r0, pitch, v);
          if (r0 + 8 >= n) {
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&tempty[a]);
          }
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            const int t = __shfl_sync(0xffffffffu, token, (r0 + r) & 31);
            const float s = __shfl_sync(0xffffffffu, share, (r0 + r) & 31);
            if (r0 + r < n && t >= 0) sums[t * 128 + ch] = fmaf(s, v[r] + bias, sums[t * 128 + ch]);
          }
        }
      }
      u += g.kb1 - g.kb0;
    }
    if (!ok) {
      *abort_word = 1;
      if (lane == 0) raise_device_status(STAMP_ERR_TIMEOUT);
    }
  }

  ptx::tc_fence_before();
  __syncthreads();
  if (p.split > 1) ptx::cluster_sync();
  // (a CTA that gave up leaves its outputs as they were)
  if (UP ? !idle && *abort_word == 0 : runs >= 0 && *abort_word == 0) {
    // the sums of the cluster's CTAs in rank order; every CTA takes every split-th row (UP) or token (DOWN)
    const uint32_t part = ptx::smem_u32(UP ? reinterpret_cast<float*>(smem) : sums);
    if constexpr (UP) {
      const ExpertRun run = run_table[run0];
      for (int i = threadIdx.x; i < (run.n - rank + p.split - 1) / p.split * 128; i += EXPERT_THREADS) {
        const int r = rank + (i >> 7) * p.split, ch = i & 127, f = tile * 128 + ch;
        float g = 0.f, u = 0.f;
        for (int s = 0; s < p.split; ++s) {
          const uint32_t at = (p.split > 1 ? ptx::mapa(part, s) : part) + (r * 256 + ch) * 4;
          g += p.split > 1 ? ptx::ld_dsmem_f1(at) : reinterpret_cast<const float*>(smem)[r * 256 + ch];
          u += p.split > 1 ? ptx::ld_dsmem_f1(at + 512) : reinterpret_cast<const float*>(smem)[r * 256 + 128 + ch];
        }
        if (f < p.F) {
          if (p.up_bias) {
            const float* const b = p.up_bias + static_cast<long>(run.expert) * 2 * p.F + f;
            g += __ldg(b);
            u += __ldg(b + p.F);
          }
          p.h[static_cast<long>(run.row0 + r) * p.F + f] = gated_silu2<false, false>(make_float2(g, g), make_float2(u, u)).x;
        }
      }
    } else {
      if (p.M > 0) ptx::grid_dependency_wait();   // (the tokens may be overwritten from here on)
      for (int i = threadIdx.x; i < (p.T - rank + p.split - 1) / p.split * 128; i += EXPERT_THREADS) {
        const int t = rank + (i >> 7) * p.split, ch = i & 127, c = tile * 128 + ch;
        float y = 0.f;
        for (int s = 0; s < p.split; ++s) y += p.split > 1 ? ptx::ld_dsmem_f1(ptx::mapa(part, s) + (t * 128 + ch) * 4) : sums[t * 128 + ch];
        if (c < p.N) {
          if (p.residual) {
            const long at = t * p.ldr + c;
            y += p.r_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.residual)[at]) : static_cast<const float*>(p.residual)[at];
          }
          TOut* const out = static_cast<TOut*>(p.y) + static_cast<long>(t) * p.N + c;
          if constexpr (sizeof(TOut) == 2) *out = __float2bfloat16_rn(y); else *out = y;
        }
      }
    }
  }
  // nobody lets go of its shared memory while another CTA may read it
  if (p.split > 1) ptx::cluster_sync();
  if (warp == 5) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, 256);
  }
}

}  // namespace stamp
