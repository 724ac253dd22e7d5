// A whole expert layer for a few tokens in two kernels, activations as they are:
//   h[m, f] = silu(g) u,  g = w_up[e, f] . x[rows[m]] + up_bias[e, f],  u the same for row F + f      (e: the expert of row m)
//   y[t]    = residual[t] + sum over the rows m of token t of share[m] (w_down[e] h[m] + down_bias[e])
//
// With few tokens a layer is the way of its weights from memory: each byte meets a handful of rows.  (An expert's weights are read
// once for every run of its rows: UP 16 of bf16 tokens or 8 of fp32 ones, DOWN 16; all but the first time mostly from L2.)  The
// weights are e4m3 already, so they go by TMA to shared memory and from there into the block-scaled tensor instruction
// (kind::mxf8f6f4, channels on the TMEM lanes, rows as columns) without passing a register.  The activations are not e4m3;
// quantizing them would be the layer's largest error and saves nothing here.  They are written as a sum of e4m3 terms
// instead, each with its own power-of-two scale for a block of 128:
//   v = c0 s + c1 s 2^-4 + c2 s 2^-9 + c3 s 2^-14 + c4 s 2^-19,   s the quantizer's scale of the block, c_i the nearest e4m3 number
//   to what is left.  The first term is off by at most 2^-4 of v (16 s at the top of the range, hence the step to 2^-4) and every further
//   one by 2^-5 of that: two terms hold the 8 significant bits of a bf16 value, four 2^-19, five the 24 bits of an fp32 one.  e4m3
//   numbers end in steps of 2^-9, so that two terms hold nothing below 2^-14 s (2^-21.8 of the block's largest value), four
//   nothing below 2^-24 s (2^-31.8), five nothing below 2^-29 s (2^-36.8).
// A term is a column of the product like any other row's, so the terms cost columns (16 at least in any case), not another
// pass over the weights; the epilogue adds them up.  bf16 tokens take two terms, fp32 ones five, the hidden values four: three, for a bf16
// output, would do with 1 % less time and leave one output in a hundred at its other neighbour.  UP leaves the hidden values as
// terms already, DOWN copies them like the weights.
//
//   warps 0-3   epilogue, one TMEM lane (output channel) a thread
//   warp 4      TMA producer: 128 channels x 128 features of weights (UP: of gates and of ups), DOWN: and of the rows' terms,
//               into a ring of stages
//   warp 5      allocates TMEM, copies the scale words to it and issues the MMAs
//   warps 6-13  (UP: 6-15) the scales, UP: and the tokens' terms.  Always the same warps for a stage of the ring: who fills it has filled
//               it the time before too, so that the parity it waits for is never an older one's, and it can load the stage's
//               next rows as soon as it is through with the last
// Every wait is bounded; when one expires the CTA raises the device status word, unwinds and frees its TMEM.
//
// UP: a tile is one run (up to `cap` rows of one expert) times 128 gates and the 128 ups that go with them.  One CTA an SM takes
// tile after tile, the epilogue of one beside the copies of the next.  Where there are few tiles a cluster of `split` CTAs
// takes one, each a share of the features; the partial sums are added over distributed shared memory in rank order.
// DOWN: a cluster takes 128 output channels and all runs; its CTAs share the sequence of all (run, 128 features).  A CTA adds
// each run's rows, weighted, to its tokens in shared memory in the order of the rows; the CTAs' sums are added in rank order,
// with the residual.  No atomics on results, nothing in memory but the hidden values, and every result repeats bit for bit.
// DOWN is launched as a programmatic dependent of UP: its first weights are on their way while UP's last CTAs run; only its
// copies of the hidden values and their scales wait.
//
// What bounds it.  Many experts: the weights' way from memory.  64 tokens, eight of 64 experts of 2048 x 2048: 805 MB, 125 us at the
// copy rate, in 143 (fp32 tokens 157: 8 rows a run, five terms each; UP 5.6 TB/s cold); 13 tokens, four of 32 experts of 4096 x 4096: 189 us
// where random choices reach some 26 of them (1.3 GB, 206 at the copy rate: reads alone go faster than the copy that the rate is from).  Few tiles:
// one chain of launch, first copies, terms, sums, exchange, hidden values, sums, exchange.  One token, four experts of 1152 x 2048: 28 MB,
// 4.4 us at the copy rate, in 16.4, where the two kernels alone and cold take 13 and 14.  Many rows for each of few experts: UP's runs, 55 tokens to
// all of 8 experts of 896 x 3456 64 us where the weights alone would take 11.6.
// Measured and not kept, us for what was kept then: tiles of 64 gates (171 for 150; one token 18.3 for 16); runs of 32 rows in UP (158 for
// 152); one CTA an SM with 200 KB in DOWN (160 for 147: clusters of eight find their SMs late); two CTAs an SM in UP, one tile each
// (187 for 150); hidden values in fp32, made into terms by DOWN (294 for 150); one kernel for both token types, which counts its terms as it
// runs (146 for 143; one token 16.9 for 16.4).
#pragma once
#include "common.cuh"
#include "k_fp8_gemm.cuh"
#include "k_fp8_quant.cuh"
#include "ptx.cuh"

namespace stamp {

constexpr int EXPERT_FEW_TOKENS = 64;
constexpr int EXPERT_FEW_ROWS = 2048;
constexpr int EXPERT_MAX = 1024;
constexpr int EXPERT_MAX_STAGES = 8, EXPERT_MAX_SPLIT = 16;
constexpr int EXPERT_W_BYTES = 128 * 128;
constexpr int EXPERT_H_TERMS = 4;                       // of a hidden value
// Blocks of 128 features that one accumulator sums at most: half as many as for the products' fp32 outputs, since three sums one after
// the other add up their errors.  13 tokens over 32 experts of 4096 x 4096 in bf16, fp32 output: 1.3e-6 of the result from 64 bits, with
// parts of 32 blocks 1.75e-6 and 0.3 % less time, in one part 2.8e-6.
constexpr int EXPERT_PART = 16;
constexpr int EXPERT_MAX_SMEM = 224 * 1024;             // of a CTA that has an SM to itself; two of half of it fit one
constexpr int EXPERT_H_BYTES = 2 * 8 * 128 * 4;         // UP: hidden values of eight rows on their way to terms, twice

struct ExpertParams {
  const void* x;            // [T, ldx] bf16 or float
  long ldx;
  const int* rows;          // [M] token of every row
  const float* share;       // [M]
  const int* offsets;       // [E + 1]
  const uint8_t *w_up, *up_scale, *w_down, *down_scale;   // [E, 2 F, K], [E, N, F]
  const float *up_bias, *down_bias;                       // [E, 2 F], [E, N] or nullptr
  const void* residual;     // [T, ldr] or nullptr
  long ldr;
  int r_bf16;
  int T, M, E, K, F, N;
  uint8_t* h;               // [terms][M, F] codes of the hidden values, terms of the DOWN kernel
  uint8_t* h_scale;         // [M, ceil(F / 128)] scale of a row's first term
  void* y;                  // [T, N]
  // one kernel's plan
  int cap;                  // rows of a run at most (a multiple of 8)
  int split;                // CTAs of a cluster
  int stages, stage_bytes;
};

// T: UP: the tokens' type, DOWN: the output's.
template <bool UP, typename T>
struct ExpertSmem {
  static constexpr int TERMS = !UP ? EXPERT_H_TERMS : sizeof(T) == 2 ? 2 : 5;   // of a row
  static constexpr int ROWS = UP && sizeof(T) == 4 ? 8 : 16;                    // of a run at most
  static constexpr int FILLERS = UP ? 10 : 8;           // warps that write scales (UP: and terms)
  static constexpr int THREADS = 32 * (6 + FILLERS);
  static constexpr int CTAS = UP ? 1 : 2;               // of an SM that the registers allow
  static constexpr int COLUMNS = (TERMS * ROWS + 15) / 16 * 16;   // of one sum
  static constexpr int ACC = UP ? 2 * COLUMNS : COLUMNS;   // tensor memory: two accumulators (UP: gates, ups), then the stages' scales
  static constexpr int SF_BYTES = UP ? 1536 : 1024;     // scale words of a stage: channels (UP: twice), then rows
  static constexpr int SF_COLS = SF_BYTES / 128, SF_COL = 2 * ACC;
  // Half of an SM's columns for every CTA, so that UP and DOWN, which waits for it, never wait for one another's.
  static constexpr int TMEM = 256, MAX_STAGES = UP && sizeof(T) == 4 ? 5 : EXPERT_MAX_STAGES;
  static_assert(SF_COL + MAX_STAGES * SF_COLS <= TMEM, "tensor memory of a CTA");
  static constexpr int BARS = 2 * EXPERT_MAX_STAGES + 6;
  // after the ring and the scale words: barriers, [tmem, abort, runs, -], run table, UP: hidden values, tokens [M], sums of the parts
  // before (PARTS) [row][gates, ups], DOWN: sums [T][128]
  static constexpr int CARRIED_BYTES = ROWS * 256 * 4;
  __host__ __device__ static constexpr int tables(int max_runs) { return BARS * 8 + 16 + (max_runs * 8 + 15) / 16 * 16; }
  __host__ __device__ static int fixed(int max_runs, int tokens, int M, bool parts) {
    return 1024 + tables(max_runs) + (UP ? EXPERT_H_BYTES + M * 4 + (parts ? CARRIED_BYTES : 0) : tokens * 512);
  }
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
template <typename T>
struct ExpertRaw;
template <>
struct ExpertRaw<__nv_bfloat16> {
  uint2 u;
  __device__ __forceinline__ void load(const void* base, long at, bool live) {
    u = live ? __ldcg(reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(base) + at)) : make_uint2(0u, 0u);
  }
  __device__ __forceinline__ void values(float (&v)[4]) const {
    v[0] = __uint_as_float(u.x << 16), v[1] = __uint_as_float(u.x & 0xFFFF0000u);
    v[2] = __uint_as_float(u.y << 16), v[3] = __uint_as_float(u.y & 0xFFFF0000u);
  }
};
template <>
struct ExpertRaw<float> {
  float4 u;
  __device__ __forceinline__ void load(const void* base, long at, bool live) {
    u = live ? __ldcg(reinterpret_cast<const float4*>(static_cast<const float*>(base) + at)) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  __device__ __forceinline__ void values(float (&v)[4]) const { v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w; }
};

// The scale of term t, from the first term's (which stops at 2^-127; a NaN's terms are all NaN).
__device__ __forceinline__ uint32_t expert_term_scale(uint32_t first, int t) {
  const uint32_t down = t == 0 ? 0u : 5u * t - 1u;
  return first == 255u ? 255u : first - min(first, down);
}
// 128 values of a row, four a lane, as terms: emit(t, codes) for each; returns the scale byte of the first.
template <int TERMS, typename Emit>
__device__ __forceinline__ uint32_t expert_terms(const float (&value)[4], Emit&& emit) {
  const float most = ptx::warp_max_abs(ptx::max_abs_nan(ptx::max_abs_nan(value[0], value[1], value[2]), value[3], 0.f));
  const Fp8Scale s = fp8_scale(__float_as_uint(most));
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = value[i] * s.inverse;
#pragma unroll
  for (int t = 0; t < TERMS; ++t) {
    const uint32_t c = ptx::cvt_e4m3x4(v[0], v[1], v[2], v[3]);
    emit(t, c);
    if (t + 1 == TERMS) break;
    // what is left, in units of the next term's scale
    const uint32_t shift = s.byte == 255 ? 0u : expert_term_scale(s.byte, t) - expert_term_scale(s.byte, t + 1);
    const float up = __uint_as_float((127u + shift) << 23);
    const float2 a = expert_e4m3x2(c), b = expert_e4m3x2(c >> 16);
    v[0] = (v[0] - a.x) * up, v[1] = (v[1] - a.y) * up, v[2] = (v[2] - b.x) * up, v[3] = (v[3] - b.y) * up;
  }
  return s.byte;
}
// Row i of a run, term t: its column.  Eight rows' first terms, then their second ones, and so on; then the next eight rows.
__device__ __forceinline__ int expert_column(int i, int t, int terms) { return (i & ~7) * terms + t * 8 + (i & 7); }
// The scale bytes of a row's terms, in the order that tmem_copy_scales wants.
__device__ __forceinline__ void expert_scale_words(uint8_t* words, int i, int t, int terms, uint32_t first) {
  const int r = expert_column(i, t, terms);
  *reinterpret_cast<uint32_t*>(words + ((r & 31) << 4) + ((r >> 5) << 2)) = expert_term_scale(first, t) * 0x01010101u;
}

// PARTS (UP): a CTA's share of the features is more than one accumulator sums.  (A kernel of its own: with the parts' branches in it
// the other takes 2 to 4 % longer, 55 tokens over 8 experts of 896 x 3456 70.5 us for 67.8.)
template <bool UP, typename T, bool PARTS = false>
__global__ void __launch_bounds__(ExpertSmem<UP, T>::THREADS, ExpertSmem<UP, T>::CTAS)
    k_expert_layer(const __grid_constant__ CUtensorMap tmap, const __grid_constant__ CUtensorMap tmap_h, ExpertParams p) {
  using SM = ExpertSmem<UP, T>;
  constexpr int TERMS = SM::TERMS;
  extern __shared__ uint8_t expert_raw[];
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(expert_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* const words = smem + p.stages * p.stage_bytes;
  uint64_t* const full = reinterpret_cast<uint64_t*>(words + p.stages * SM::SF_BYTES);
  uint64_t* const empty = full + EXPERT_MAX_STAGES;
  uint64_t* const tfull = empty + EXPERT_MAX_STAGES;
  uint64_t* const tempty = tfull + 2;
  uint64_t* const exchange = tempty + 2;   // (and one word to spare)
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(exchange + 2);
  volatile uint32_t* const abort_word = tmem_slot + 1;
  int* const run_count = reinterpret_cast<int*>(tmem_slot + 2);   // -1: the offsets are out of order
  ExpertRun* const run_table = reinterpret_cast<ExpertRun*>(tmem_slot + 4);
  const int max_runs = expert_max_runs(p.M, p.E, p.cap);
  float* const sums = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(full) + SM::tables(max_runs));
  float* const hidden = sums;
  int* const tokens = reinterpret_cast<int*>(hidden + EXPERT_H_BYTES / 4);
  float* const carried = reinterpret_cast<float*>(tokens + p.M);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = p.split > 1 ? static_cast<int>(ptx::cluster_ctarank()) : 0;
  const int unit = blockIdx.x / p.split;
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      ptx::mbar_init(&full[s], 1 + (UP ? SM::FILLERS / p.stages : 1));
      ptx::mbar_init(&empty[s], UP ? 2 : 1);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(&tfull[a], 1);
      ptx::mbar_init(&tempty[a], 4);
    }
    ptx::mbar_init(exchange, 4);
    *abort_word = 0;
    ptx::fence_mbar_init();
    ptx::prefetch_tensormap(&tmap);
    if constexpr (!UP) ptx::prefetch_tensormap(&tmap_h);
  }
  if (warp == 5) {
    ptx::tmem_alloc(tmem_slot, SM::TMEM);
    ptx::tmem_relinquish();
  }
  if constexpr (!UP) {
    for (int i = threadIdx.x; i < p.T * 128; i += SM::THREADS) sums[i] = 0.f;
  }
  // UP waits for what came before it.  DOWN starts when every CTA of UP has come past this point: what UP waited for is there
  // for DOWN too, and only the hidden values are to be waited for.  (Where no row exists, DOWN is alone and waits.)
  if (UP || p.M == 0) ptx::grid_dependency_wait();
  if constexpr (UP) {
    ptx::grid_launch_dependents();
    for (int m = threadIdx.x; m < p.M; m += SM::THREADS) tokens[m] = __ldcg(p.rows + m);
  }
  if (warp == 4) {
    bool bad = false;
    int runs = 0;
    for (int e0 = 0; e0 < p.E && !bad; e0 += 128) {
      int first[4], last[4];   // the loads of 128 experts at once
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = e0 + 32 * i + lane;
        first[i] = e < p.E ? __ldcg(p.offsets + e) : 0;
        last[i] = e < p.E ? __ldcg(p.offsets + e + 1) : 0;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = e0 + 32 * i + lane;
        bad |= first[i] < 0 || last[i] > p.M || last[i] < first[i] || (e == 0 && first[i] != 0);
        if (__any_sync(0xffffffffu, bad)) {
          bad = true;
          break;
        }
        if (e0 + 32 * i >= p.E) break;
        const int own = (last[i] - first[i] + p.cap - 1) / p.cap;
        int before = own;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int v = __shfl_up_sync(0xffffffffu, before, d);
          if (lane >= d) before += v;
        }
        const int at = runs + before - own;
        for (int j = 0; j < own; ++j)
          run_table[at + j] = ExpertRun{first[i] + j * p.cap, static_cast<uint16_t>(e), static_cast<uint16_t>(min(p.cap, last[i] - first[i] - j * p.cap))};
        runs += __shfl_sync(0xffffffffu, before, 31);
      }
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

  // What this CTA sums.  UP: its share of the features, one tile (run, 128 channels) after the other; DOWN: its share of the
  // sequence of (run, 128 features).  Either in parts of EXPERT_PART blocks: the tensor cores cut a running sum off instead of
  // rounding it, and what that loses grows with the number of additions.
  const int blocks = ((UP ? p.K : p.F) + 127) / 128;   // of one run
  const int tiles = UP ? (p.F + 127) / 128 : 1;
  int u0, u1, share0 = 0, share1 = blocks, parts = 1;
  if constexpr (UP) {
    if (p.split > 1) share0 = blocks * rank / p.split, share1 = blocks * (rank + 1) / p.split;
    if constexpr (PARTS) parts = (share1 - share0 + EXPERT_PART - 1) / EXPERT_PART;
    u0 = unit * parts;
    u1 = runs > 0 ? runs * tiles * parts : 0;
  } else {
    const int all = runs > 0 ? runs * blocks : 0, each = all / p.split, more = all - each * p.split;
    u0 = each * rank + min(rank, more);
    u1 = u0 + each + (rank < more ? 1 : 0);
  }
  struct Segment {
    int kb0, kb1, tile, next;
    ExpertRun run;
  };
  auto segment_at = [&](int u) {   // one part of a tile; the part of one run that starts at u
    if constexpr (UP) {
      const int step = static_cast<int>(gridDim.x) / p.split;
      if constexpr (PARTS) {
        const int t = u / parts, part = u - t * parts, r = t / tiles, kb0 = share0 + part * EXPERT_PART;
        return Segment{kb0, min(share1, kb0 + EXPERT_PART), t - r * tiles, part + 1 < parts ? u + 1 : (t + step) * parts, run_table[r]};
      } else {
        const int r = u / tiles;
        return Segment{share0, share1, u - r * tiles, u + step, run_table[r]};
      }
    } else {
      const int r = u / blocks, kb0 = u - r * blocks, kb1 = min(min(blocks, kb0 + EXPERT_PART), kb0 + u1 - u);
      return Segment{kb0, kb1, unit, u + kb1 - kb0, run_table[r]};
    }
  };
  const auto columns = [&](int n) { return TERMS * ((n + 7) & ~7); };

  // UP: four hidden values a lane of one row's 128, as terms (F is a multiple of 16: a lane's channels are all there or none)
  auto store_hidden = [&](float4 h, long row, int tile) {
    const int f = tile * 128 + lane * 4;
    const float v[4] = {h.x, h.y, h.z, h.w};
    const uint32_t first = expert_terms<EXPERT_H_TERMS>(v, [&](int t, uint32_t c) {
      if (f < p.F) *reinterpret_cast<uint32_t*>(p.h + (static_cast<long>(t) * p.M + row) * p.F + f) = c;
    });
    if (lane == 0) p.h_scale[row * tiles + tile] = static_cast<uint8_t>(first);
  };

  if (warp == 4) {
    // ------------------------------------------------------------------ TMA producer
    if (ptx::elect_one()) {
      int stage = 0, issued = 0;
      uint32_t phase = 0;
      bool ok = true;
      // DOWN: the weights of the first round go ahead of the hidden values, whose kernel may still run
      auto copy_hidden = [&](const Segment& g, int kb, int at) {
        for (int r = 0; r < g.run.n; r += 8)
          ptx::tma_load_3d(smem + at * p.stage_bytes + EXPERT_W_BYTES + r * TERMS * 128, &tmap_h, &full[at], kb * 128, g.run.row0 + r, 0);
      };
      auto first_hidden = [&]() {
        ptx::grid_dependency_wait();
        ptx::grid_launch_dependents();
        int at = 0;
        for (int u = u0; u < u1 && at < issued;) {
          const Segment g = segment_at(u);
          for (int kb = g.kb0; kb < g.kb1 && at < issued; ++kb) copy_hidden(g, kb, at++);
          u = g.next;
        }
      };
      for (int u = u0; u < u1 && ok;) {
        const Segment g = segment_at(u);
        const int row = g.run.expert * (UP ? 2 * p.F : p.N) + g.tile * 128;
        const uint32_t bytes = UP ? 2 * EXPERT_W_BYTES : EXPERT_W_BYTES + columns(g.run.n) * 128;
        for (int kb = g.kb0; kb < g.kb1; ++kb) {
          if (!UP && issued == p.stages) first_hidden();
          if (!ptx::mbar_wait_bounded_sleepy(&empty[stage], phase ^ 1u, abort_word, FP8G_WAIT_LIMIT)) {
            ok = false;
            break;
          }
          uint8_t* const dst = smem + stage * p.stage_bytes;
          ptx::mbar_arrive_expect_tx(&full[stage], bytes);
          ptx::tma_load_2d(dst, &tmap, &full[stage], kb * 128, row);
          if constexpr (UP) ptx::tma_load_2d(dst + EXPERT_W_BYTES, &tmap, &full[stage], kb * 128, row + p.F);
          if (!UP && issued >= p.stages) copy_hidden(g, kb, stage);
          ++issued;
          if (++stage == p.stages) stage = 0, phase ^= 1u;
        }
        u = g.next;
      }
      if (!UP && p.M > 0 && issued <= p.stages) first_hidden();
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
        const uint32_t idesc = ptx::mxf8_idesc_with(idesc0, (columns(g.run.n) + 15) & ~15);
        const int a = it & 1;
        if (!ptx::mbar_wait_bounded(&tempty[a], ((it >> 1) & 1) ^ 1, abort_word, FP8G_WAIT_LIMIT)) {
          ok = false;
          break;
        }
        ptx::tc_fence_after();
        const uint32_t acc = tmem + static_cast<uint32_t>(a * SM::ACC);
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
        u = g.next;
      }
      if (!ok) {
        *abort_word = 1;
        raise_device_status(STAMP_ERR_TIMEOUT);
      }
    }
  } else if (warp >= 6) {
    // ------------------------------------------------------------------ scales, UP: and the tokens' terms
    const uint8_t* const scales = UP ? p.up_scale : p.down_scale;
    const int scale_rows = ((UP ? 2 * p.F : p.N) + 127) / 128;
    const int each = UP ? SM::FILLERS / p.stages : 1;   // warps of a stage; they share its rows
    const int stage = (warp - 6) / each, part = (warp - 6) % each;
    uint8_t* const xt = smem + stage * p.stage_bytes + 2 * EXPERT_W_BYTES;
    uint8_t* const sf = words + stage * SM::SF_BYTES;
    uint8_t* const rf = sf + SM::SF_BYTES - 512;
    int i = 0, s = stage;   // steps before this segment; the next one that goes to this warp's stage
    uint32_t phase = 0;
    bool ok = true, waited = UP;
    for (int u = u0; u < u1 && ok && stage < p.stages;) {
      const Segment g = segment_at(u);
      const int n = g.run.n, up_first = UP ? (p.F + g.tile * 128) >> 7 : 0, up_rest = UP ? 128 - ((p.F + g.tile * 128) & 127) : 0;
      int token = -1;   // UP: lane r: the token of row r of the run
      if (UP && lane < n) {
        token = tokens[g.run.row0 + lane];
        if (token < 0 || token >= p.T) {
          if (g.tile == 0 && rank == 0 && warp == 6) raise_device_status(STAMP_ERR_INVALID_ARG);
          token = -1;
        }
      }
      const uint8_t* const sc = scales + static_cast<long>(g.run.expert) * scale_rows * blocks;
      for (; s < i + g.kb1 - g.kb0; s += p.stages, phase ^= 1u) {
        const int kb = g.kb0 + s - i;
        // everything the stage needs is loaded before it is waited for, UP: as far as eight rows for each warp
        uint32_t w0 = __ldcg(sc + static_cast<long>(g.tile) * blocks + kb), w1 = 0, w2 = 0;
        ExpertRaw<T> raw[8];
        auto load = [&](int r0) {
          const int col = kb * 128 + lane * 4;
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            const int t = __shfl_sync(0xffffffffu, token, (r0 + r * each) & 31);
            raw[r].load(p.x, t * p.ldx + col, r0 + r * each < n && t >= 0 && col < p.K);
          }
        };
        if constexpr (UP) {
          load(part);
          w1 = __ldcg(sc + static_cast<long>(up_first) * blocks + kb);
          w2 = __ldcg(sc + static_cast<long>(min(up_first + 1, scale_rows - 1)) * blocks + kb);
        } else {
          if (!waited) ptx::grid_dependency_wait();
          waited = true;
          w1 = lane < n ? __ldcg(p.h_scale + static_cast<long>(g.run.row0 + lane) * blocks + kb) : 0u;
        }
        if (!__all_sync(0xffffffffu, ptx::mbar_wait_bounded_sleepy(&empty[stage], phase ^ 1u, abort_word, FP8G_WAIT_LIMIT))) {
          ok = false;
          break;
        }
        w0 *= 0x01010101u;
        if (part == 0) *reinterpret_cast<uint4*>(sf + lane * 16) = make_uint4(w0, w0, w0, w0);
        if constexpr (UP) {
          if (part == 0) {
            // the ups may start inside a block of the scales
            w1 *= 0x01010101u, w2 *= 0x01010101u;
            *reinterpret_cast<uint4*>(sf + 512 + lane * 16) =
                make_uint4(lane < up_rest ? w1 : w2, lane + 32 < up_rest ? w1 : w2, lane + 64 < up_rest ? w1 : w2, lane + 96 < up_rest ? w1 : w2);
          }
          for (int r0 = part; r0 < n;) {
#pragma unroll
            for (int r = 0; r < 8; ++r) {
              const int row = r0 + r * each;
              if (row >= n) break;
              float v[4];
              raw[r].values(v);
              // (rows of 128 bytes, 128-byte swizzle; a term's columns are eight further)
              uint8_t* const out = xt + expert_column(row, 0, TERMS) * 128 + (((lane >> 2) ^ (row & 7)) << 4) + ((lane & 3) << 2);
              const uint32_t first = expert_terms<TERMS>(v, [&](int t, uint32_t c) { *reinterpret_cast<uint32_t*>(out + t * 1024) = c; });
              if (lane < TERMS) expert_scale_words(rf, row, lane, TERMS, first);
            }
            r0 += 8 * each;
            if (r0 < n) load(r0);
          }
        } else {
          if (lane < n) {
            for (int t = 0; t < TERMS; ++t) expert_scale_words(rf, lane, t, TERMS, w1);
          }
        }
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&full[stage]);
      }
      i += g.kb1 - g.kb0;
      u = g.next;
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
    // eight rows' sums at this thread's channel, their terms added up, the smallest first
    auto eight = [&](uint32_t acc, int r0, float (&v)[8]) {
      uint32_t c[TERMS][8];
#pragma unroll
      for (int t = 0; t < TERMS; ++t) ptx::tmem_ld_32x32b_x8(acc + r0 * TERMS + t * 8, c[t]);
      ptx::tmem_ld_wait();
#pragma unroll
      for (int r = 0; r < 8; ++r) v[r] = 0.f;
#pragma unroll
      for (int t = TERMS - 1; t >= 0; --t)
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r] += __uint_as_float(c[t][r]);
    };
    uint32_t exchanged = 0;
    for (int u = u0; u < u1 && ok; ++it) {
      const Segment g = segment_at(u);
      const int n = g.run.n, a = it & 1, c = g.tile * 128 + ch;   // this thread's channel
      int token = -1;
      float share = 0.f;
      if (!UP && lane < n) {
        token = __ldcg(p.rows + g.run.row0 + lane);
        share = __ldcg(p.share + g.run.row0 + lane);
        if (token < 0 || token >= p.T) token = -1;
      }
      float bias = 0.f;   // (once for every row: with the run's first features)
      float up_bias = 0.f;
      if (!UP && p.down_bias && g.kb0 == 0 && c < p.N) bias = __ldcg(p.down_bias + static_cast<long>(g.run.expert) * p.N + c);
      if (UP && p.up_bias && c < p.F && p.split == 1) {
        bias = __ldcg(p.up_bias + static_cast<long>(g.run.expert) * 2 * p.F + c);
        up_bias = __ldcg(p.up_bias + static_cast<long>(g.run.expert) * 2 * p.F + p.F + c);
      }
      if (!__all_sync(0xffffffffu, ptx::mbar_wait_bounded_sleepy(&tfull[a], (it >> 1) & 1, abort_word, FP8G_WAIT_LIMIT))) {
        ok = false;
        break;
      }
      ptx::tc_fence_after();
      const uint32_t acc = tmem + (static_cast<uint32_t>(warp * 32) << 16) + static_cast<uint32_t>(a * SM::ACC);
      for (int r0 = 0; r0 < n; r0 += 8) {
        float v[8], w[8];
        eight(acc, r0, v);
        if constexpr (UP) eight(acc + SM::COLUMNS, r0, w);
        if (r0 + 8 >= n) {
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&tempty[a]);
        }
        if constexpr (PARTS) {
          // (every value of the parts before is this thread's own)
          float* const before = carried + r0 * 256 + ch;
          if (g.kb0 > share0) {
#pragma unroll
            for (int r = 0; r < 8; ++r) v[r] += before[r * 256], w[r] += before[r * 256 + 128];
          }
          if (g.kb1 < share1) {
#pragma unroll
            for (int r = 0; r < 8; ++r) before[r * 256] = v[r], before[r * 256 + 128] = w[r];
            continue;
          }
        }
        if constexpr (!UP) {
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            const int t = __shfl_sync(0xffffffffu, token, (r0 + r) & 31);
            const float s = __shfl_sync(0xffffffffu, share, (r0 + r) & 31);
            if (r0 + r < n && t >= 0) sums[t * 128 + ch] = fmaf(s, v[r] + bias, sums[t * 128 + ch]);
          }
        } else if (p.split > 1) {
          // this CTA's part of the sums, [row][gates, ups], in the ring that nothing uses any more
          float* const part = reinterpret_cast<float*>(smem) + r0 * 256 + ch;
#pragma unroll
          for (int r = 0; r < 8; ++r)
            if (r0 + r < n) {
              part[r * 256] = v[r];
              part[r * 256 + 128] = w[r];
            }
        } else {
          // hidden values by channel to hidden values by row: over shared memory, two buffers in turn
          float* const at = hidden + (exchanged & 1u) * 1024;
#pragma unroll
          for (int r = 0; r < 8; r += 2) {
            const float2 h = gated_silu2<false, false>(make_float2(v[r] + bias, v[r + 1] + bias), make_float2(w[r] + up_bias, w[r + 1] + up_bias));
            at[r * 128 + ch] = c < p.F ? h.x : 0.f;
            at[r * 128 + 128 + ch] = c < p.F ? h.y : 0.f;
          }
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(exchange);
          if (!__all_sync(0xffffffffu, ptx::mbar_wait_bounded(exchange, exchanged & 1u, abort_word, FP8G_WAIT_LIMIT))) {
            ok = false;
            break;
          }
          ++exchanged;
          for (int r = warp; r < 8 && r0 + r < n; r += 4) store_hidden(*reinterpret_cast<const float4*>(at + r * 128 + lane * 4), g.run.row0 + r0 + r, g.tile);
        }
      }
      u = g.next;
    }
    if (!ok) {
      *abort_word = 1;
      if (lane == 0) raise_device_status(STAMP_ERR_TIMEOUT);
    }
  }

  // DOWN: the residual of the first token this warp writes is on its way while the cluster's CTAs wait for one another
  auto residual = [&](int t, int c) {
    const long at = t * p.ldr + c;
    return !p.residual || c >= p.N || t >= p.T ? 0.f
           : p.r_bf16                          ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.residual)[at])
                                               : static_cast<const float*>(p.residual)[at];
  };
  float ahead[UP ? 1 : 4];
  if constexpr (!UP) {
#pragma unroll
    for (int i = 0; i < 4; ++i) ahead[i] = residual(rank + warp * p.split, unit * 128 + lane * 4 + i);
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (p.split > 1) ptx::cluster_sync();
  // (a CTA that gave up leaves its outputs as they were)
  if (UP ? p.split > 1 && u0 < u1 && *abort_word == 0 : runs >= 0 && *abort_word == 0) {
    // the sums of the cluster's CTAs in rank order; every CTA takes every split-th row (UP) or token (DOWN)
    const uint32_t part = ptx::smem_u32(UP ? reinterpret_cast<float*>(smem) : sums);
    uint32_t part_of[EXPERT_MAX_SPLIT];
#pragma unroll
    for (int s = 0; s < EXPERT_MAX_SPLIT; ++s) part_of[s] = p.split > 1 ? ptx::mapa(part, static_cast<uint32_t>(min(s, p.split - 1))) : part;
    // four channels of one row from every CTA, four loads in flight at once
    auto total = [&](int at) {
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int s0 = 0; s0 < EXPERT_MAX_SPLIT; s0 += 4) {
        float4 v[4];
#pragma unroll
        for (int s = 0; s < 4; ++s)
          if (s0 + s < p.split)
            v[s] = p.split > 1 ? ptx::ld_dsmem_f4(part_of[s0 + s] + at * 4) : *reinterpret_cast<const float4*>((UP ? reinterpret_cast<const float*>(smem) : sums) + at);
#pragma unroll
        for (int s = 0; s < 4; ++s)
          if (s0 + s < p.split) sum = make_float4(sum.x + v[s].x, sum.y + v[s].y, sum.z + v[s].z, sum.w + v[s].w);
      }
      return sum;
    };
    if constexpr (UP) {
      // a warp takes a row, a lane four channels
      const Segment t = segment_at(u0);
      const int f = t.tile * 128 + lane * 4;
      for (int r = rank + warp * p.split; r < t.run.n; r += SM::THREADS / 32 * p.split) {
        float4 g = total(r * 256 + lane * 4), u = total(r * 256 + 128 + lane * 4);
        if (p.up_bias && f < p.F) {
          const float* const b = p.up_bias + static_cast<long>(t.run.expert) * 2 * p.F + f;
          g = make_float4(g.x + __ldg(b), g.y + __ldg(b + 1), g.z + __ldg(b + 2), g.w + __ldg(b + 3));
          u = make_float4(u.x + __ldg(b + p.F), u.y + __ldg(b + p.F + 1), u.z + __ldg(b + p.F + 2), u.w + __ldg(b + p.F + 3));
        }
        const float2 h0 = gated_silu2<false, false>(make_float2(g.x, g.y), make_float2(u.x, u.y));
        const float2 h1 = gated_silu2<false, false>(make_float2(g.z, g.w), make_float2(u.z, u.w));
        store_hidden(f < p.F ? make_float4(h0.x, h0.y, h1.x, h1.y) : make_float4(0.f, 0.f, 0.f, 0.f), t.run.row0 + r, t.tile);
      }
    } else {
      if (p.M > 0) ptx::grid_dependency_wait();   // (the tokens may be overwritten from here on)
      // a warp takes a token, a lane four channels
      const int c = unit * 128 + lane * 4;
      for (int t = rank + warp * p.split; t < p.T; t += SM::THREADS / 32 * p.split) {
        const float4 sum = total(t * 128 + lane * 4);
        const float y[4] = {sum.x, sum.y, sum.z, sum.w};
        T* const out = static_cast<T*>(p.y) + static_cast<long>(t) * p.N + c;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (c + i >= p.N) break;
          const float v = y[i] + (t == rank + warp * p.split ? ahead[i] : residual(t, c + i));
          if constexpr (sizeof(T) == 2) out[i] = __float2bfloat16_rn(v); else out[i] = v;
        }
      }
    }
  }
  // nobody lets go of its shared memory while another CTA may read it
  if (p.split > 1) ptx::cluster_sync();
  if (warp == 5) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, SM::TMEM);
  }
}

}  // namespace stamp
