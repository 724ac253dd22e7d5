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

// Experts of a row of counts: a multiple of four.
__host__ __device__ constexpr int route_pitch(int E) { return (E + 3) & ~3; }

struct RouteParams {
  const void* logits;   // [T, ldl]
  long ldl;
  int T, E, top, normalize;
  int vector;           // logits can be read 16 bytes (a lane's, if that is less) at a time
  int per_cta, per_warp;   // tokens; each CTA and warp has a run of them
  int* chosen;          // [T, top]
  float* share;         // [T, top]
  int* rows;            // [T * top] token of every row
  int* place;           // [T, top]
  int* offsets;         // [E + 1]
  float* row_share;     // [T * top]
  int* counts;          // [CTAs, route_pitch(E)] rows of every expert from a CTA's tokens (more than one CTA)
};

// A float's bits so that they order as it does; -0 as 0, NaN below everything, 0 left free.
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

// A logit and its expert, ordered: larger logits first, of equal ones the lower expert.  A bf16 logit has 16 bits, so both fit
// one word (the lower half counts experts downwards); an fp32 one takes two.  `none` comes behind everything.  set_finite leaves
// NaNs outside the infinities' range, where strange() finds them in a sorted list's ends; set gives them their place.
template <typename TIn>
struct RouteEntry;
template <>
struct RouteEntry<__nv_bfloat16> {
  uint32_t word;
  __device__ __forceinline__ void set(float logit, int e) { word = (route_key(logit) >> 16 << 16) | (0xFFFFu - e); }   // (a NaN: 0, with an expert)
  // two neighbouring logits, as loaded
  __device__ __forceinline__ static void set_finite(uint32_t two, int e, RouteEntry& a, RouteEntry& b) {
    const __nv_bfloat162 zero = __floats2bfloat162_rn(0.f, 0.f), sum = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&two), zero);
    const uint32_t v = *reinterpret_cast<const uint32_t*>(&sum);
    uint32_t sign;   // of each half, over all of its bits
    asm("prmt.b32 %0, %1, %1, 0xBB99;" : "=r"(sign) : "r"(v));
    const uint32_t key = v ^ (sign | 0x80008000u);
    a.word = __byte_perm(key, 0xFFFFu - e, 0x1054);
    b.word = (key & 0xFFFF0000u) | (0xFFFFu - e - 1u);
  }
  __device__ __forceinline__ static bool strange(const RouteEntry& first, const RouteEntry& last) {
    return first.word >= 0xFF810000u || last.word < 0x007F0000u;   // (infinity's upper half is 0xFF80, that of -infinity 0x007F)
  }
  __device__ __forceinline__ void none() { word = 0u; }
  __device__ __forceinline__ static void order(RouteEntry& a, RouteEntry& b) {
    const uint32_t hi = max(a.word, b.word);
    b.word = min(a.word, b.word);
    a.word = hi;
  }
  __device__ __forceinline__ RouteEntry best() const { return RouteEntry{__reduce_max_sync(0xffffffffu, word)}; }
  __device__ __forceinline__ bool is(const RouteEntry& o) const { return word == o.word; }
  __device__ __forceinline__ int expert() const { return 0xFFFF - (word & 0xFFFFu); }
  __device__ __forceinline__ float logit() const {
    const uint32_t key = word & 0xFFFF0000u;   // (the lower half of a negative float's key is all ones)
    return key == 0u ? __int_as_float(0x7FC00000) : __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key & 0xFFFF0000u);
  }
};
template <>
struct RouteEntry<float> {
  uint32_t key, e;
  __device__ __forceinline__ void set(float logit, int expert) { key = route_key(logit), e = expert; }
  __device__ __forceinline__ void set_finite(float logit, int expert) {
    const uint32_t b = __float_as_uint(logit + 0.f);
    key = b ^ (static_cast<uint32_t>(static_cast<int>(b) >> 31) | 0x80000000u), e = expert;
  }
  __device__ __forceinline__ static bool strange(const RouteEntry& first, const RouteEntry& last) {
    return first.key > 0xFF800000u || last.key < 0x007FFFFFu;
  }
  __device__ __forceinline__ void none() { key = 0u, e = 0x7FFFFFFFu; }
  __device__ __forceinline__ static void order(RouteEntry& a, RouteEntry& b) {
    const bool swap = a.key < b.key || (a.key == b.key && a.e > b.e);
    const RouteEntry c = a;
    a.key = swap ? b.key : c.key, a.e = swap ? b.e : c.e;
    b.key = swap ? c.key : b.key, b.e = swap ? c.e : b.e;
  }
  __device__ __forceinline__ RouteEntry best() const {
    const uint32_t most = __reduce_max_sync(0xffffffffu, key);
    return RouteEntry{most, __reduce_min_sync(0xffffffffu, key == most ? e : 0x7FFFFFFFu)};
  }
  __device__ __forceinline__ bool is(const RouteEntry& o) const { return e == o.e; }
  __device__ __forceinline__ int expert() const { return static_cast<int>(e); }
  __device__ __forceinline__ float logit() const { return route_value(key); }
};
// A lane's entries in order: sorting networks (of eight: two of four, then a merge).
template <typename T, int PER>
__device__ __forceinline__ void route_sort(RouteEntry<T> (&v)[PER]) {
  auto at = [&](int a, int b) { RouteEntry<T>::order(v[a], v[b]); };
  if constexpr (PER >= 2) {
#pragma unroll
    for (int i = 0; i < PER; i += 2) at(i, i + 1);
  }
  if constexpr (PER >= 4) {
#pragma unroll
    for (int i = 0; i < PER; i += 4) at(i, i + 2), at(i + 1, i + 3), at(i + 1, i + 2);
  }
  if constexpr (PER == 8) {
    at(0, 4), at(1, 5), at(2, 6), at(3, 7);
    at(2, 4), at(3, 5);
    at(1, 2), at(3, 4), at(5, 6);
  }
}
// PER neighbouring logits of a row, as loaded; beyond the row -inf.
template <typename T, int PER>
struct RouteLogits;
template <int PER>
struct RouteLogits<float, PER> {
  float v[PER];
  __device__ __forceinline__ void load(const float* p, int left, bool vector) {
    if (PER >= 4 && vector && left >= PER) {
#pragma unroll
      for (int i = 0; i < PER; i += 4) {
        const float4 u = __ldg(reinterpret_cast<const float4*>(p + i));
        v[i] = u.x, v[(i + 1) % PER] = u.y, v[(i + 2) % PER] = u.z, v[(i + 3) % PER] = u.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) v[i] = i < left ? __ldg(p + i) : -__int_as_float(0x7F800000);
    }
  }
  __device__ __forceinline__ float value(int i) const { return v[i]; }
  __device__ __forceinline__ void finite(RouteEntry<float> (&entry)[PER], int e) const {
#pragma unroll
    for (int i = 0; i < PER; ++i) entry[i].set_finite(v[i], e + i);
  }
};
template <int PER>
struct RouteLogits<__nv_bfloat16, PER> {
  uint32_t w[(PER + 1) / 2];
  __device__ __forceinline__ void load(const __nv_bfloat16* p, int left, bool vector) {
    if (PER >= 4 && vector && left >= PER) {
      if constexpr (PER == 8) {
        const uint4 u = __ldg(reinterpret_cast<const uint4*>(p));
        w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
      } else if constexpr (PER == 4) {
        const uint2 u = __ldg(reinterpret_cast<const uint2*>(p));
        w[0] = u.x, w[1] = u.y;
      }
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const uint32_t h = i < left ? *reinterpret_cast<const uint16_t*>(p + i) : 0xFF80u;
        w[i / 2] = i & 1 ? w[i / 2] | h << 16 : h;
      }
    }
  }
  __device__ __forceinline__ float value(int i) const { return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16); }
  __device__ __forceinline__ void finite(RouteEntry<__nv_bfloat16> (&entry)[PER], int e) const {
    RouteEntry<__nv_bfloat16> odd;
#pragma unroll
    for (int i = 0; i < PER; i += 2) RouteEntry<__nv_bfloat16>::set_finite(w[i / 2], e + i, entry[i], i + 1 < PER ? entry[(i + 1) % PER] : odd);
  }
};

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
struct RouteRow {
  long i, last;   // (token, choice) of this thread's next row, and the end of the CTA's
  int expert, rank;
  float share;
  __device__ __forceinline__ void load(const RouteParams& p) {
    if (i < last) expert = p.chosen[i], rank = p.place[i], share = p.share[i];
  }
};
__device__ __forceinline__ RouteRow route_first(const RouteParams& p) {
  const long first = static_cast<long>(blockIdx.x) * p.per_cta * p.top;
  RouteRow r{first + threadIdx.x, min(first + static_cast<long>(p.per_cta) * p.top, static_cast<long>(p.T) * p.top), 0, 0, 0.f};
  r.load(p);
  return r;
}
__device__ __forceinline__ void route_store(const RouteParams& p, const int* base, RouteRow r) {
  while (r.i < r.last) {
    const int at = base[r.expert] + r.rank;
    p.place[r.i] = at;
    p.rows[at] = static_cast<int>(static_cast<uint32_t>(r.i) / static_cast<uint32_t>(p.top));   // (T * top <= 2^30)
    p.row_share[at] = r.share;
    r.i += ROUTE_THREADS;
    r.load(p);
  }
}

// A warp takes one token after the other, the next one's logits on their way, a lane PER neighbouring experts: it sorts them
// once, then the lanes' first entries are compared `top` times, and the lane that had the best one moves up.  (Searching all
// entries every time took three times the instructions.  16384 tokens of 256 bf16 logits, top 8, both launches 16.3 us where 8.4 MB
// have to be read, 1.7 us: 390 instructions a token, eight of them warp-wide maxima that wait for one another with eight warps a scheduler to
// fill in, then the second launch; fp32 logits, whose entries take two words, 20.1 us.)  Up to eight
// choices are unrolled, so that only entries that can still be chosen move.  Above 256 experts (PER = 32, expert 32 i + lane in
// register i) sorting costs more than searching; that form spills, and takes 79 us for 16384 tokens of 384 experts, 107 of 1024.
// Each warp counts its rows by expert in shared memory, and a row's rank is the count so far; the warps' counts are then
// summed in their order.
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
  const long t1 = min(t0 + p.per_warp, cta_end);
  constexpr bool SORTED = PER <= 8;
  RouteLogits<TIn, SORTED ? PER : 1> next;   // (a token ahead)
  auto load = [&](long t) {
    if (SORTED && t < t1) next.load(static_cast<const TIn*>(p.logits) + t * p.ldl + lane * PER, p.E - lane * PER, p.vector);
  };
  load(t0);
  for (long t = t0; t < t1; ++t) {
    float l[SORTED ? 1 : PER];
    const auto now = next;
    load(t + 1);
    bool nan = false;
    int expert = 0;        // lane j: choice j and its logit
    float best = 0.f;
    if constexpr (SORTED) {
      RouteEntry<TIn> entry[PER], mine_of{};
      const bool full = p.E == 32 * PER;   // every lane has PER experts
      if (full) {
        now.finite(entry, lane * PER);
        route_sort<TIn, PER>(entry);
        nan = __any_sync(0xffffffffu, RouteEntry<TIn>::strange(entry[0], entry[PER - 1]));
      }
      if (!full || nan) {
        nan = false;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          entry[i].set(now.value(i), lane * PER + i);
          if (lane * PER + i >= p.E) entry[i].none();
          nan |= now.value(i) != now.value(i);
        }
        nan = __any_sync(0xffffffffu, nan);
        route_sort<TIn, PER>(entry);
      }
      auto take = [&](int j, int left) {   // choice j, with `left` entries of a lane to come into question after it
        const RouteEntry<TIn> first = entry[0].best();
        const bool up = entry[0].is(first);
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (i < left && up) {
            if (i + 1 < PER) entry[i] = entry[(i + 1) % PER];
            else entry[i].none();
          }
        if (lane == j) mine_of = first;
      };
      if (p.top <= 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (j >= p.top) break;
          take(j, 7 - j);
        }
      } else {
        for (int j = 0; j < p.top; ++j) take(j, PER);
      }
      expert = mine_of.expert();
      best = mine_of.logit();
    } else {
      const TIn* row = static_cast<const TIn*>(p.logits) + t * p.ldl;
      uint32_t key[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        l[i] = 32 * i + lane < p.E ? route_load(row + 32 * i + lane) : -__int_as_float(0x7F800000);
        key[i] = 32 * i + lane < p.E ? route_key(l[i]) : 0u;
        nan |= l[i] != l[i];
      }
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
        if (lane == j) expert = e, best = route_value(most);
      }
      nan = __any_sync(0xffffffffu, nan);
    }
    const float largest = __shfl_sync(0xffffffffu, best, 0);
    const bool dead = !nan && largest == -__int_as_float(0x7F800000);
    const float weight = lane < p.top ? expf(best - largest) : 0.f;
    float total = weight;
    if (!p.normalize) {
      total = 0.f;
#pragma unroll
      for (int i = 0; i < PER; ++i) total += expf((SORTED ? now.value(SORTED ? i : 0) : l[SORTED ? 0 : i]) - largest);   // (lanes without an expert: exp(-inf))
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
    if (gridDim.x > 1) p.counts[static_cast<long>(blockIdx.x) * route_pitch(p.E) + e] = sum;
  }
  if (gridDim.x > 1 && threadIdx.x >= p.E && threadIdx.x < route_pitch(p.E)) p.counts[static_cast<long>(blockIdx.x) * route_pitch(p.E) + threadIdx.x] = 0;
  __syncthreads();
  for (long i = t0 * p.top + lane; i < t1 * p.top; i += 32) p.place[i] += mine[p.chosen[i]];
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
  route_store(p, base, route_first(p));
}

// The second launch where several CTAs chose (about 5 us of the 16 above: two trips to the L2, one for the counts, one for the
// rows): every expert's first place, from the counts of all CTAs; then the rows.  The
// counts are padded to a multiple of four experts (`pitch`): a thread sums four experts over a share of the CTAs.
__global__ void __launch_bounds__(ROUTE_THREADS) k_expert_place(RouteParams p) {
  extern __shared__ int4 route_sums[];   // [groups][pitch / 4] rows of the CTAs before this one, then of all
  __shared__ int base[ROUTE_MAX_EXPERTS];
  __shared__ int scratch[33];
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int fours = route_pitch(p.E) / 4, groups = ROUTE_THREADS / fours, g = threadIdx.x / fours, i4 = threadIdx.x - g * fours;
  const RouteRow row = route_first(p);   // (on its way with the counts)
  int4 before = make_int4(0, 0, 0, 0), all = before;
  if (g < groups) {
#pragma unroll 10
    for (int b = g; b < static_cast<int>(gridDim.x); b += groups) {
      const int4 c = __ldg(reinterpret_cast<const int4*>(p.counts) + static_cast<long>(b) * fours + i4);
      all.x += c.x, all.y += c.y, all.z += c.z, all.w += c.w;
      if (b < static_cast<int>(blockIdx.x)) before.x += c.x, before.y += c.y, before.z += c.z, before.w += c.w;
    }
    route_sums[g * fours + i4] = before;
    route_sums[(groups + g) * fours + i4] = all;
  }
  __syncthreads();
  const int e = threadIdx.x;
  int mine = 0, sum = 0;
  if (e < p.E) {
    const int* const s = reinterpret_cast<const int*>(route_sums) + e;
    for (int o = 0; o < groups; ++o) {
      mine += s[o * fours * 4];
      sum += s[(groups + o) * fours * 4];
    }
  }
  int total;
  const int first = route_scan(sum, scratch, total);
  if (e < p.E) {
    base[e] = first + mine;
    if (blockIdx.x == 0) p.offsets[e] = first;
  }
  if (blockIdx.x == 0 && e == 0) p.offsets[p.E] = total;
  __syncthreads();
  route_store(p, base, row);
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

// V neighbouring channels as loaded and stored, 16 bytes at most a time.
template <typename T, int V>
struct Packed {
  static constexpr int BYTES = sizeof(T) * V, WORDS = (BYTES + 3) / 4;
  uint32_t w[WORDS];
  __device__ __forceinline__ void load(const void* base, long at) {
    const char* const p = static_cast<const char*>(base) + at * sizeof(T);
    if constexpr (BYTES % 16 == 0) {
#pragma unroll
      for (int i = 0; i < WORDS; i += 4) {
        const uint4 u = *reinterpret_cast<const uint4*>(p + i * 4);
        w[i] = u.x, w[i + 1] = u.y, w[i + 2] = u.z, w[i + 3] = u.w;
      }
    } else if constexpr (BYTES == 8) {
      const uint2 u = *reinterpret_cast<const uint2*>(p);
      w[0] = u.x, w[1] = u.y;
    } else if constexpr (BYTES == 4) {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
      w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
  }
  __device__ __forceinline__ float value(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
  }
  __device__ __forceinline__ static void store(void* base, long at, const float (&v)[V]) {
    T* const p = static_cast<T*>(base) + at;
    if constexpr (V == 1) {
      if constexpr (sizeof(T) == 4) *p = v[0];
      else *p = __float2bfloat16_rn(v[0]);
    } else {
      uint32_t u[WORDS];
#pragma unroll
      for (int i = 0; i < WORDS; ++i) {
        if constexpr (sizeof(T) == 4) {
          u[i] = __float_as_uint(v[i]);
        } else {
          const __nv_bfloat162 two = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
          u[i] = *reinterpret_cast<const uint32_t*>(&two);
        }
      }
      if constexpr (BYTES == 8) {
        *reinterpret_cast<uint2*>(p) = make_uint2(u[0], u[1]);
      } else {
#pragma unroll
        for (int i = 0; i < WORDS; i += 4) reinterpret_cast<uint4*>(p)[i / 4] = make_uint4(u[i], u[(i + 1) % WORDS], u[(i + 2) % WORDS], u[(i + 3) % WORDS]);
      }
    }
  }
};

// A thread takes V neighbouring channels of one token (rows off the words' alignment: V = 1 and U of them,
// COMBINE_THREADS apart); four of the token's rows are in flight at a time.  grid (T, ceil(N / (COMBINE_THREADS V U)))
template <typename TIn, typename TOut, int V, int U>
__global__ void __launch_bounds__(COMBINE_THREADS) k_expert_combine(CombineParams p, int r_bf16) {
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const long t = blockIdx.x, c0 = (static_cast<long>(blockIdx.y) * U * COMBINE_THREADS + threadIdx.x) * V;
  auto channel = [&](int u) { return c0 + u * COMBINE_THREADS; };
  // (the residual does not wait for the places)
  Packed<float, V> wide[U];
  Packed<__nv_bfloat16, V> narrow[U];
  float sum[U][V];
#pragma unroll
  for (int u = 0; u < U; ++u) {
#pragma unroll
    for (int i = 0; i < V; ++i) sum[u][i] = 0.f;
    if (!p.residual || channel(u) >= p.N) continue;
    if (r_bf16) narrow[u].load(p.residual, t * p.ldr + channel(u));
    else wide[u].load(p.residual, t * p.ldr + channel(u));
  }
  for (int j0 = 0; j0 < p.top; j0 += 4) {
    Packed<TIn, V> raw[4][U];
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
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (channel(u) < p.N) raw[j][u].load(p.y, static_cast<long>(at) * p.N + channel(u));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (!live[j]) continue;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i) sum[u][i] = fmaf(share[j], raw[j][u].value(i), sum[u][i]);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (channel(u) >= p.N) continue;
    if (p.residual) {
#pragma unroll
      for (int i = 0; i < V; ++i) sum[u][i] += r_bf16 ? narrow[u].value(i) : wide[u].value(i);
    }
    Packed<TOut, V>::store(p.out, t * p.N + channel(u), sum[u]);
  }
}

}  // namespace stamp
