// Log probabilities of given tokens, the distribution's entropy and its most
// probable tokens, from rows of logits read once.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "ifq_serve.h"

namespace ifq {
namespace {

// With c = scale * log2(e), M the row's largest logit, t = c * (x - M):
//   S = sum 2^t,  E = sum t 2^t
//   log p(x) = scale * (x - M) - ln S,  entropy = ln S - ln 2 * E / S
// Both terms of the entropy are positive, so nothing cancels. Parts of a row keep
// sums for a maximum of their own; with d = c * (M_part - M) their share is
// 2^d S and 2^d (E + d S). Differences are taken in halves and times twice the factor: x - M
// may leave fp32's range where scale * (x - M) does not. (x - M) / 2 is one operation,
// fma(x, 1/2, -M/2), with the bits of x - M wherever that is in the range.
//
// The top tokens go by a key of 64 bits: the value, as an integer of the same
// order, over the complement of the index, so that keys differ and equal values
// go by the lower index. Of 256 groups of values the k-th largest maximum is a bar that k
// values at least reach and few others: those are collected, and each one's place
// is the number of larger ones. A group is one lane's values, or those of two or four lanes
// beside one another: where all that counts lies in fewer groups than top tokens (rows of
// few values, all but a range of tokens masked), the bar is the masked ones' value and all
// others are ranked, each against each. us, and of unmasked rows: 96 x 50001 top 20 with 4096
// tokens in one range 398 and 17, 64 x 128000 top 64 497 and 20; 1000 x 1000 top 64 41.

struct LogprobArgs {
  const void* x;
  const int32_t* tokens;
  float* logprob;
  float* entropy;
  float* top_logprobs;
  int32_t* top_tokens;
  uint32_t* count;
  float* part;
  int64_t ld_x, ld_top;
  int64_t row0;                  // first row of this launch
  int32_t n, top, parts;
  int32_t chunks;                // of a row, each a wave's turn
  float scale2, c2;              // twice scale and c
};

constexpr float kLn2 = 0.69314718055994531f;
constexpr int kWaves = 4;
constexpr int kPartFloats = 4;   // M, S, E of a part ahead of its keys
constexpr int kMostParts = 32;   // of a row with top tokens
constexpr int kMore = 3;         // maxima that may reach the bar beyond the top ones; LDS for two workgroups

// The value of lane ^ D.
template <int D>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v) {
  if constexpr (D == 1) return __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, true);
  if constexpr (D == 2) return __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xF, 0xF, true);
  if constexpr (D == 4)          // 7 - i in eight lanes, then 3 - i in four
    return __builtin_amdgcn_update_dpp(
        0, __builtin_amdgcn_update_dpp(0, v, 0x141, 0xF, 0xF, true), 0x1B, 0xF, 0xF, true);
  if constexpr (D == 8) return __builtin_amdgcn_update_dpp(0, v, 0x128, 0xF, 0xF, true);
  if constexpr (D == 16) {
    const auto both = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return threadIdx.x & 16 ? both[0] : both[1];
  }
  const auto both = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return threadIdx.x & 32 ? both[0] : both[1];
}

template <int D>
__device__ __forceinline__ float lane_xor(float v) {
  return bits_f32(lane_xor<D>(f32_bits(v)));
}

// An integer of the same order; -0 equals 0.
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t b = f32_bits(v + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}

__device__ __forceinline__ float value_of(uint32_t order) {
  return bits_f32(order >> 31 ? order ^ 0x80000000u : ~order);
}

__device__ __forceinline__ uint64_t key_of(float v, int index) {
  return (uint64_t)order_of(v) << 32 | (uint32_t)~index;
}

__device__ __forceinline__ int index_of(uint64_t key) { return (int)~(uint32_t)key; }

// (v - from) / 2 for half = from / 2, without leaving fp32's range.
__device__ __forceinline__ float half_from(float v, float half) {
  return __builtin_fmaf(v, 0.5f, -half);
}

struct Sums {
  float m, s, e;
  // the sums as they go by a maximum that is as large at least
  __device__ __forceinline__ void to(float top, float c2) {
    const float r = top == -INFINITY ? 0.0f : top;
    // an empty part has no share (and its maximum none either)
    const float d = s == 0.0f ? 0.0f : c2 * half_from(m, 0.5f * r), f = __builtin_amdgcn_exp2f(d);
    e = f == 0.0f ? 0.0f : f * (e + d * s);    // a share of 0 adds nothing, also where d is -infinity
    s *= f;
    m = top;
  }
  __device__ __forceinline__ void add(Sums o, float c2) {
    const float top = fmaxf(m, o.m);
    to(top, c2);
    o.to(top, c2);
    s += o.s;
    e += o.e;
  }
  // over the lanes
  __device__ __forceinline__ void all(float c2) {
    float top = m;
    top = fmaxf(top, lane_xor<1>(top));
    top = fmaxf(top, lane_xor<2>(top));
    top = fmaxf(top, lane_xor<4>(top));
    top = fmaxf(top, lane_xor<8>(top));
    top = fmaxf(top, lane_xor<16>(top));
    top = fmaxf(top, lane_xor<32>(top));
    to(top, c2);
    s += lane_xor<1>(s), e += lane_xor<1>(e);
    s += lane_xor<2>(s), e += lane_xor<2>(e);
    s += lane_xor<4>(s), e += lane_xor<4>(e);
    s += lane_xor<8>(s), e += lane_xor<8>(e);
    s += lane_xor<16>(s), e += lane_xor<16>(e);
    s += lane_xor<32>(s), e += lane_xor<32>(e);
  }
};

// Indices of a lane's values: runs of W that follow one another.
template <typename T> constexpr int kRun = 16 / sizeof(T);
template <typename T>
__device__ __forceinline__ int index_in_turn(int i, int lane) {
  return i / kRun<T> * (64 * kRun<T>) + lane * kRun<T> + i % kRun<T>;
}

// Values of a turn that starts at `base`; -infinity from n on. Rows may begin at any
// element. The loads of a row's last turn do not wait for one another either: runs past the
// last whole one load that one again, and what is left of a run comes after.
template <typename T, int PER>
__device__ __forceinline__ void load_turn(const T* row, int base, int n, int lane, float* v) {
  constexpr int W = kRun<T>;
  T t[PER];
  if (base + 64 * PER <= n) {
#pragma unroll
    for (int i = 0; i < PER; i += W)
      __builtin_memcpy(t + i, row + base + index_in_turn<T>(i, lane), W * sizeof(T));
#pragma unroll
    for (int i = 0; i < PER; ++i) v[i] = (float)t[i];
    return;
  }
  const int rest = n % W, whole = n - rest;
#pragma unroll
  for (int i = 0; i < PER; ++i) v[i] = -INFINITY;
  if (whole) {
#pragma unroll
    for (int i = 0; i < PER; i += W)
      __builtin_memcpy(t + i, row + min(base + index_in_turn<T>(i, lane), whole - W), W * sizeof(T));
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (base + index_in_turn<T>(i - i % W, lane) < whole) v[i] = (float)t[i];
  }
#pragma unroll
  for (int i = 0; i < PER; i += W)
    if (rest && base + index_in_turn<T>(i, lane) == whole) {
#pragma unroll
      for (int j = 0; j < W - 1; ++j)
        if (j < rest) v[i + j] = (float)row[whole + j];
    }
}

// A turn's sums of a lane.
template <int PER>
__device__ __forceinline__ Sums sums_of(const float* v, float c2) {
  float m = v[0];
#pragma unroll
  for (int i = 1; i < PER; ++i) m = fmaxf(m, v[i]);
  Sums u = {m, 0.0f, 0.0f};
  const float half = m == -INFINITY ? 0.0f : 0.5f * m;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const float z = c2 * half_from(v[i], half), e = __builtin_amdgcn_exp2f(z);
    u.s += e;
    u.e = __builtin_fmaf(fmaxf(z, -1e4f), e, u.e);     // 0 where e is, z -infinity or not
  }
  return u;
}

// What a row's sums stand for. A row of -infinity alone has no probability anywhere (S is
// 0); with a NaN or an infinity in it (S is NaN) it has no distribution.
struct Row {
  bool none;
  float half, log;               // of the largest logit; of the sum
  __device__ __forceinline__ explicit Row(const Sums& t) {
    const bool empty = t.s == 0.0f;
    none = t.s != t.s;
    half = empty ? 0.0f : 0.5f * t.m;
    log = empty ? 0.0f : logf(t.s);
  }
  __device__ __forceinline__ float logprob(float v, float scale2) const {
    return scale2 * half_from(v, half) - log;
  }
};

// One lane's work.
template <typename T>
__device__ __forceinline__ void finish(const LogprobArgs& a, int64_t row, const T* x, const Sums& t) {
  const Row f(t);
  if (a.entropy) a.entropy[row] = t.s == 0.0f ? 0.0f : f.log - kLn2 * (t.e / t.s);
  if (a.logprob) {
    const int token = a.tokens[row];
    float p = 0.0f;
    if (token >= a.n) p = bits_f32(0x7FC00000u);
    else if (token >= 0) p = f.logprob((float)x[token], a.scale2);
    a.logprob[row] = p;
  }
}

// Without top tokens. One row or a part of it to a workgroup; its waves take turns of 64 *
// PER values, which stay in registers between the search for the largest and the sums. Bound
// by memory: 4000 x 32000 float32 87 us, 5.9 TB/s.
template <typename T, int PER>
__global__ __launch_bounds__(64 * kWaves) void logprobs(LogprobArgs a) {
  __shared__ Sums sums[kWaves];
  __shared__ int last;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t row = a.row0 + blockIdx.x / a.parts;
  const int own = blockIdx.x % a.parts;
  const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
  const int from = (int)((int64_t)a.chunks * own / a.parts);
  const int to = (int)((int64_t)a.chunks * (own + 1) / a.parts);
  Sums t = {-INFINITY, 0.0f, 0.0f};
  for (int chunk = from + wave; chunk < to; chunk += kWaves) {
    float v[PER];
    load_turn<T, PER>(x, chunk * (64 * PER), a.n, lane, v);
    t.add(sums_of<PER>(v, a.c2), a.c2);
  }
  t.all(a.c2);
  if (lane == 0) sums[wave] = t;
  __syncthreads();
  if (wave == 0) {
#pragma unroll
    for (int w = 1; w < kWaves; ++w) t.add(sums[w], a.c2);
  }
  if (a.parts > 1) {
    float* all = a.part + (int64_t)(row - a.row0) * a.parts * kPartFloats;
    if (threadIdx.x == 0) {
      put_pair(all + own * kPartFloats, t.m, t.s);
      put_pair(all + own * kPartFloats + 2, t.e, 0.0f);
    }
    if (!comes_last(a.count + row - a.row0, a.parts, &last)) return;
    t = {-INFINITY, 0.0f, 0.0f};
    if (lane < a.parts) {
      const f32x2 ms = get_pair(all + lane * kPartFloats), e = get_pair(all + lane * kPartFloats + 2);
      t = {ms[0], ms[1], e[0]};
    }
    t.all(a.c2);
  }
  if (threadIdx.x == 0) finish(a, row, x, t);
}

// A bar that k of 256 maxima reach and few more, by its bits from the top: the k-th
// largest one at most. Every wave finds it for itself.
__device__ __forceinline__ uint32_t bar_of(const uint32_t* maxima, int k, int lane) {
  uint32_t g[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) g[q] = maxima[64 * q + lane];
  // the bits that all of them share come first
  uint32_t high = max(max(g[0], g[1]), max(g[2], g[3])), low = min(min(g[0], g[1]), min(g[2], g[3]));
  high = max(high, lane_xor<1>(high)), low = min(low, lane_xor<1>(low));
  high = max(high, lane_xor<2>(high)), low = min(low, lane_xor<2>(low));
  high = max(high, lane_xor<4>(high)), low = min(low, lane_xor<4>(low));
  high = max(high, lane_xor<8>(high)), low = min(low, lane_xor<8>(low));
  high = max(high, lane_xor<16>(high)), low = min(low, lane_xor<16>(low));
  high = max(high, lane_xor<32>(high)), low = min(low, lane_xor<32>(low));
  high = __builtin_amdgcn_readfirstlane(high), low = __builtin_amdgcn_readfirstlane(low);
  if (high == low) return high;
  const int first = 31 - __builtin_clz(high ^ low);
  uint32_t bar = high & ~((2u << first) - 1);
  for (uint32_t bit = 1u << first; bit; bit >>= 1) {
    const uint32_t up = bar | bit;
    int reach = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) reach += __popcll(__ballot(g[q] >= up));
    if (reach >= k) bar = up;
    if (reach >= k && reach <= k + kMore) break;
  }
  return bar;
}

// Room in the list for the lanes of `some`; a lane's place.
__device__ __forceinline__ int places(int* count, uint64_t some, int lane) {
  int first = 0;
  if (lane == 0) first = atomicAdd(count, (int)__popcll(some));
  return __builtin_amdgcn_readfirstlane(first) + (int)__popcll(some & ((1ull << lane) - 1));
}

// Each key of a list at its place among the first k; a list of fewer leaves zeros. LANES lanes
// count for a key, eight others at a time each (in workgroups of 4 waves 4: 4000 x 4000 top 20
// 23.9 -> 22.5 us, but 1000 x 500 top 40 8.8 -> 9.8; of 16 one: four spilled registers, 2000 x 32000
// 55 -> 60). The list has kRankRun keys of 0 behind it.
constexpr int kRankRun = 32;
template <int LANES>
__device__ __forceinline__ void rank(const uint64_t* list, int count, int k, uint64_t* best) {
  const int part = threadIdx.x % LANES;
  for (int i = threadIdx.x / LANES; i < count; i += blockDim.x / LANES) {
    const uint64_t key = list[i];
    int place = 0;
    for (int j = 0; j < count; j += 8 * LANES) {
      uint64_t some[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) some[q] = list[j + 8 * part + q];
#pragma unroll
      for (int q = 0; q < 8; ++q) place += some[q] > key;
    }
    if (LANES >= 2) place += lane_xor<1>((uint32_t)place);
    if (LANES >= 4) place += lane_xor<2>((uint32_t)place);
    if (part == 0 && place < k) best[place] = key;
  }
}

// With top tokens. Every wave takes one turn, so that its values stay in registers until
// the bar is known; a chain of load, maxima, bar, list and places, for a row's parts twice (1 x
// 128000 top 20 10.7 us, 96 x 50001 top 5 without a join 13.1). Values above the bar are in k + kMore groups at most (where
// more maxima reach it, it is the k-th largest); of those equal to it a wave needs the
// k first ones only.
template <typename T, int PER, int WAVES>
__global__ __launch_bounds__(64 * WAVES, PER == 32 ? 8 : 4) void logprobs_top(LogprobArgs a) {
  typedef std::conditional_t<PER == 64, uint64_t, uint32_t> Bits;     // a lane's values
  constexpr int LANES = WAVES / 4;               // of a group
  constexpr int ABOVE = (64 + kMore) * LANES * PER;
  constexpr int LIST = std::max(ABOVE + 64 * WAVES, 64 * kMostParts);
  __shared__ Sums sums[WAVES];
  __shared__ uint32_t maxima[256];
  __shared__ uint64_t list[LIST + kRankRun], best[64];
  __shared__ int count, last;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t row = a.row0 + blockIdx.x / a.parts;
  const int own = blockIdx.x % a.parts, k = a.top;
  const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
  // parts of about the same size, so that the last one too has more groups than top tokens: with
  // fewer all its values are ranked (8 x 200000 top 33 310 us, 17 with this; 500 x 128000 top 20
  // 67.9 -> 69.7)
  const int from = a.chunks * own / a.parts, to = a.chunks * (own + 1) / a.parts;
  const int base = (from + wave) * (64 * PER);
  float v[PER];
  load_turn<T, PER>(x, base, min(a.n, to * (64 * PER)), lane, v);
  Sums t = sums_of<PER>(v, a.c2);
  uint32_t most = order_of(t.m);
  if (LANES >= 2) most = max(most, lane_xor<1>(most));
  if (LANES >= 4) most = max(most, lane_xor<2>(most));
  if (lane % LANES == 0) maxima[threadIdx.x / LANES] = most;
  if (threadIdx.x < 64) best[threadIdx.x] = 0;
  if (threadIdx.x == 0) count = 0;
  t.all(a.c2);
  if (lane == 0) sums[wave] = t;
  __syncthreads();
  {
    const float bar = value_of(bar_of(maxima, k, lane));
    Bits above = 0, equal = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      above |= v[i] > bar ? (Bits)1 << i : 0;
      equal |= v[i] == bar ? (Bits)1 << i : 0;
    }
    int ties = __popcll(equal);
    ties += lane_xor<1>((uint32_t)ties);
    ties += lane_xor<2>((uint32_t)ties);
    ties += lane_xor<4>((uint32_t)ties);
    ties += lane_xor<8>((uint32_t)ties);
    ties += lane_xor<16>((uint32_t)ties);
    ties += lane_xor<32>((uint32_t)ties);
    if (__builtin_amdgcn_readfirstlane(ties) <= 64) {
      above |= equal;
    } else {
      // in the order of their indices: run by run, lane by lane
      constexpr int W = kRun<T>;
      int taken = 0;
      for (int i = 0; i < PER && taken < k; i += W) {
        const uint32_t bits = (uint32_t)(equal >> i) & ((1u << W) - 1);
        int before = taken, all = 0;
#pragma unroll
        for (int j = 0; j < W; ++j) {
          const uint64_t with = __ballot(bits >> j & 1);
          before += __popcll(with & ((1ull << lane) - 1));
          all += __popcll(with);
        }
        for (int j = 0; j < W; ++j) {
          const bool mine = (bits >> j & 1) && before < k;
          const uint64_t some = __ballot(mine);
          if (!some) continue;
          const int place = places(&count, some, lane);
          if (mine) list[place] = key_of(bar, base + index_in_turn<T>(i, lane) + j);
          before += bits >> j & 1;
        }
        taken += all;
      }
    }
    while (const uint64_t some = __ballot(above != 0)) {
      const int i = above ? __ffsll((unsigned long long)above) - 1 : 0;
      float one = v[0];
#pragma unroll
      for (int j = 1; j < PER; ++j) one = i == j ? v[j] : one;
      const int place = places(&count, some, lane);
      if (above) list[place] = key_of(one, base + index_in_turn<T>(i, lane));
      above &= above - 1;
    }
  }
  __syncthreads();
  if (threadIdx.x < kRankRun) list[count + threadIdx.x] = 0;
  __syncthreads();
  rank<WAVES == 4 ? 4 : 1>(list, count, k, best);
  if (wave == 0) {
    t = {-INFINITY, 0.0f, 0.0f};
    if (lane < WAVES) t = sums[lane];
    t.all(a.c2);
  }
  __syncthreads();
  if (PER != 64 && a.parts > 1) {
    const int size = kPartFloats + 2 * k;
    float* all = a.part + (int64_t)(row - a.row0) * a.parts * size;
    if (wave == 0) {
      float* mine = all + (int64_t)own * size;
      if (lane == 0) put_pair(mine, t.m, t.s);
      if (lane == 1) put_pair(mine + 2, t.e, 0.0f);
      if (lane < k)
        put_pair(mine + kPartFloats + 2 * lane, bits_f32((uint32_t)best[lane]),
                 bits_f32((uint32_t)(best[lane] >> 32)));
    }
    if (!comes_last(a.count + row - a.row0, a.parts, &last)) return;
    // the parts' keys, a part to a wave at a time, and the same again
    constexpr int EACH = kMostParts / WAVES;
    f32x2 both[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i)                 // all on their way before one is looked at
      both[i] = get_pair(all + (int64_t)min(i * WAVES + wave, a.parts - 1) * size + kPartFloats +
                         2 * min(lane, k - 1));
    uint64_t keys[EACH];
    most = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const bool here = i * WAVES + wave < a.parts && lane < k;
      keys[i] = here ? (uint64_t)f32_bits(both[i][1]) << 32 | f32_bits(both[i][0]) : 0;
      most = max(most, (uint32_t)(keys[i] >> 32));
    }
    if (LANES >= 2) most = max(most, lane_xor<1>(most));
    if (LANES >= 4) most = max(most, lane_xor<2>(most));
    if (lane % LANES == 0) maxima[threadIdx.x / LANES] = most;
    if (threadIdx.x < 64) best[threadIdx.x] = 0;
    if (threadIdx.x == 0) count = 0;
    if (wave == 0) {
      t = {-INFINITY, 0.0f, 0.0f};
      if (lane < a.parts) {
        const f32x2 ms = get_pair(all + (int64_t)lane * size);
        const f32x2 e = get_pair(all + (int64_t)lane * size + 2);
        t = {ms[0], ms[1], e[0]};
      }
      t.all(a.c2);
    }
    __syncthreads();
    const uint32_t bar = bar_of(maxima, k, lane);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const bool mine = keys[i] && (uint32_t)(keys[i] >> 32) >= bar;
      const uint64_t some = __ballot(mine);
      if (!some) continue;
      const int place = places(&count, some, lane);
      if (mine) list[place] = keys[i];
    }
    __syncthreads();
    if (threadIdx.x < kRankRun) list[count + threadIdx.x] = 0;
    __syncthreads();
    rank<WAVES == 4 ? 4 : 1>(list, count, k, best);
    __syncthreads();
  }
  if (wave != 0) return;
  if (lane == 0) finish(a, row, x, t);
  if (lane < k) {
    const Row f(t);
    const uint64_t key = best[lane];
    a.top_logprobs[row * a.ld_top + lane] =
        f.none ? bits_f32(0x7FC00000u) : f.logprob(value_of((uint32_t)(key >> 32)), a.scale2);
    a.top_tokens[row * a.ld_top + lane] = f.none ? -1 : index_of(key);
  }
}

constexpr int kPer = 32;

// How a call is split: rows over launches, since there are 16384 counters of parts,
// and each row over workgroups.
struct Plan {
  int32_t per;                   // with top tokens, values a lane: 16 waves of 64 or 32, or 4 of 16
  int32_t parts;
  int64_t rows;                  // of a launch
};

Plan plan_of(const ifq_logprobs_desc& d) {
  Plan p = {16, 1, d.rows};
  if (d.top) {
    // 4096 values a workgroup spread a row widely; 32768 and 65536 spare the join of parts or
    // shorten it. us for 5 top tokens of bfloat16 rows, narrow and 64 values a lane: 16 x 33000
    // 10.1 and 12.0, 96 x 33000 12.7 and 12.4, 40 x 65500 13.8 and 12.0; two parts of 32768 in the
    // place of one of 65536: 256 x 33000 28 and 14, 1000 x 50001 98 and 58. Narrow and 32 values
    // beyond 65536: 14 x 66000 11.3 and 11.9, 40 x 66000 14.1 and 12.1, 40 x 128000 19.2 and 13.2.
    // There 64 values are slower again, with one workgroup on a CU and a join: 200 x 128000 32 and
    // 40, 1000 x 100000 100 and 157. Up to 8192: 1000 x 8000 narrow 22, 32 values 26.
    const int64_t narrow = (d.n + 4095) / 4096;
    if (d.n > 32768 && d.n <= 65536) p.per = narrow * d.rows > 640 ? 64 : 16;
    else if (d.n > 8192 && (d.n <= 32768 || narrow * d.rows > 400 || narrow > kMostParts))
      p.per = 32;
    p.parts = (int32_t)(p.per == 16 ? narrow : (d.n + 1024 * p.per - 1) / (1024 * p.per));
  } else {
    // a few workgroups for each CU, and a turn for each wave at least
    const int64_t turns = (d.n + 64 * kPer - 1) / (64 * kPer);
    const int64_t most = std::min<int64_t>(1024 / std::max<int64_t>(d.rows, 1), 64);
    p.parts = (int32_t)std::max<int64_t>(1, std::min(most, turns / kWaves));
  }
  const int64_t counters = kSplitCounterBytes / (int64_t)sizeof(uint32_t);
  if (p.parts > 1) p.rows = std::min(p.rows, counters);
  return p;
}

}  // namespace

size_t logprobs_workspace_bytes(const ifq_logprobs_desc& d) {
  if (d.rows == 0) return 0;
  const Plan p = plan_of(d);
  if (p.parts == 1) return 0;
  return kSplitCounterBytes + p.rows * p.parts * (kPartFloats + 2 * d.top) * sizeof(float);
}

int64_t logprobs_groups(const ifq_logprobs_desc& d) {
  const Plan p = plan_of(d);
  return p.rows * p.parts * (p.per > 16 ? 4 : 1);
}

hipError_t launch_logprobs(const ifq_logprobs_desc& d, const void* logits, const int32_t* tokens,
                           float* logprob, float* entropy, float* top_logprobs,
                           int32_t* top_tokens, void* ws, hipStream_t stream) {
  const Plan p = plan_of(d);
  LogprobArgs a;
  a.x = logits;
  a.tokens = tokens;
  a.logprob = logprob;
  a.entropy = entropy;
  a.top_logprobs = top_logprobs;
  a.top_tokens = top_tokens;
  a.count = static_cast<uint32_t*>(ws);
  a.part = ws ? reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + kSplitCounterBytes) : nullptr;
  a.ld_x = d.ld_x;
  a.ld_top = d.ld_top;
  a.n = (int32_t)d.n;
  a.top = d.top;
  a.parts = p.parts;
  const int turn = 64 * (d.top ? p.per : kPer);
  a.chunks = (int32_t)((d.n + turn - 1) / turn);
  a.scale2 = 2.0f * d.scale;
  a.c2 = a.scale2 * 1.4426950408889634f;
  for (int64_t row = 0; row < d.rows; row += p.rows) {
    a.row0 = row;
    const dim3 grid((uint32_t)(std::min(p.rows, d.rows - row) * p.parts));
    auto go = [&](auto zero) {
      typedef decltype(zero) T;
      if (!d.top)
        hipLaunchKernelGGL((logprobs<T, kPer>), grid, dim3(64 * kWaves), 0, stream, a);
      else if (p.per == 64)
        hipLaunchKernelGGL((logprobs_top<T, 64, 16>), grid, dim3(1024), 0, stream, a);
      else if (p.per == 32)
        hipLaunchKernelGGL((logprobs_top<T, 32, 16>), grid, dim3(1024), 0, stream, a);
      else
        hipLaunchKernelGGL((logprobs_top<T, 16, 4>), grid, dim3(256), 0, stream, a);
    };
    if (d.x_type == IFQ_TYPE_BF16) go(__bf16(0));
    else if (d.x_type == IFQ_TYPE_F16) go(_Float16(0));
    else go(0.0f);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

}  // namespace ifq
