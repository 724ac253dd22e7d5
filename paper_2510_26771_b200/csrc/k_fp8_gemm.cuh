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
//   warps 4-11 epilogue: drain the finished accumulator while the next tile fills the other
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
constexpr int FP8G_EPI_WARPS = 8;
constexpr int FP8G_THREADS = 128 + 32 * FP8G_EPI_WARPS;
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
  static_assert(DYN_BYTES <= 227 * 1024, "shared memory of one CTA");
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

// The scale bytes of `n` (1..4) consecutive blocks as one word.  Where there is none -- blocks past K, rows past the
// run, whose columns are not stored -- any finite scale does: 1.
__device__ __forceinline__ uint32_t fp8_scale_word(const uint8_t* ptr, int n, bool live) {
  uint32_t b[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) b[i] = (live && i < n) ? __ldg(ptr + i) : 0x7Fu;
  return b[0] | (b[1] << 8) | (b[2] << 16) | (b[3] << 24);
}

// The order in which the two halves of the epilogue warps drain an accumulator: chunks of 32 columns, chunk c by half c & 1
// whichever accumulator it is.  A sum in several parts is added up in the output, accumulator after accumulator, and
// nothing orders the halves among each other: a chunk has to stay with one of them.  PAIR: the chunk whose columns the
// accumulators share, the eighth of the first and the first of the second, comes first.
__host__ __device__ constexpr int fp8_drain_chunk(bool descending, int half, int i, int count) {
  return half + 2 * (descending ? count - 1 - i : i);
}
__host__ __device__ constexpr int fp8_overlap_half(int accumulator) { return accumulator == 0 ? 1 : 0; }
constexpr bool fp8_drain_order_holds() {
  for (int chunks = 1; chunks <= 8; ++chunks)
    for (int a = 0; a < 2; ++a) {
      unsigned taken = 0;
      for (int half = 0; half < 2; ++half) {
        const int count = (chunks - half + 1) / 2;
        for (int i = 0; i < count; ++i) {
          const int c = fp8_drain_chunk(a == 0, half, i, count);
          if ((c & 1) != half || c < 0 || c >= chunks || (taken >> c & 1u) != 0u) return false;
          if (c == (a == 0 ? 7 : 0) && (half != fp8_overlap_half(a) || i != 0)) return false;
          taken |= 1u << c;
        }
      }
      if (taken != (1u << chunks) - 1u) return false;
    }
  return true;
}
static_assert(fp8_drain_order_holds(), "every chunk once, by the same half in both accumulators, the shared columns first");

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

template <bool PAIR, typename TOut>
__global__ void __launch_bounds__(FP8G_THREADS, 1)
    k_fp8_gemm(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x,
               const __grid_constant__ CUtensorMap tmap_x_tail, Fp8GemmParams p) {
  using SM = Fp8Smem<PAIR>;
  constexpr int BN = SM::BN;
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
  int* row_start = tile_start + FP8_MAX_EXPERTS + 1;

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
      ptx::mbar_init(&tempty[a], PAIR ? 2 * FP8G_EPI_WARPS : FP8G_EPI_WARPS);
    }
    *abort_word = 0;
    ptx::fence_mbar_init();
    ptx::prefetch_tensormap(&tmap_w);
    ptx::prefetch_tensormap(&tmap_x);
    if (p.tail) ptx::prefetch_tensormap(&tmap_x_tail);
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
    for (int e = threadIdx.x; e <= p.E; e += FP8G_THREADS) {
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
          ptx::tma_load_2d_at<PAIR>(ws, &tmap_w, bar, kb * FP8G_BK, wrow);
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
        const int chunks = (t.n + 31) / 32;
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
        if (PAIR && half != fp8_overlap_half(a)) release();
        const int count = (chunks - half + 1) / 2;
        for (int i = 0; i < count; ++i) {
          const int c = fp8_drain_chunk(PAIR && a == 0, half, i, count);
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
      for (int tok = rank + warp * p.split; tok < t.rows; tok += FP8G_THREADS / 32 * p.split) {
        float4 v[8];   // all in flight at once
#pragma unroll
        for (int s = 0; s < 8; ++s)
          if (s < p.split) v[s] = ptx::ld_dsmem_f4(part_of[s] + (tok * FP8G_BM + c4) * 4);
        float4 sum = v[0];
#pragma unroll
        for (int s = 1; s < 8; ++s)
          if (s < p.split) sum = make_float4(sum.x + v[s].x, sum.y + v[s].y, sum.z + v[s].z, sum.w + v[s].w);
        TOut* out = static_cast<TOut*>(p.y) + static_cast<long>(t.row0 + tok) * p.N + ch;
        if (ch < p.N) fp8_store2(out, sum.x + bias[0], sum.y + bias[1], ch + 1 < p.N, vec);
        if (ch + 2 < p.N) fp8_store2(out + 2, sum.z + bias[2], sum.w + bias[3], ch + 3 < p.N, vec);
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
