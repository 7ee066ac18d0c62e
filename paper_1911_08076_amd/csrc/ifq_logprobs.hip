// Log probabilities of given tokens, the distribution's entropy and its most
// probable tokens, from rows of logits read once.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ifq_serve.h"

namespace ifq {
namespace {

// With c = scale * log2(e), M the row's largest logit, t = c * (x - M):
//   S = sum 2^t,  E = sum t 2^t
//   log p(x) = scale * (x - M) - ln S,  entropy = ln S - ln 2 * E / S
// Both terms of the entropy are positive, so nothing cancels. Parts of a row keep
// sums for a maximum of their own; with d = c * (M_part - M) their share is
// 2^d S and 2^d (E + d S).
//
// The top tokens go by a key of 64 bits: the value, as an integer of the same
// order, over the complement of the index, so that keys differ and equal values
// go by the lower index. A wave keeps its best 64 keys in order, one a lane.

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
  int32_t n, top, parts;
  int32_t chunks;                // of a row, each a wave's turn
  float scale, c;
};

constexpr float kLn2 = 0.69314718055994531f;
constexpr int kWaves = 4;
constexpr int kPer = 32;         // values of a lane in a turn
constexpr int kTurn = 64 * kPer;
constexpr int kPartFloats = 4;   // M, S, E of a part ahead of its keys

__device__ __forceinline__ uint64_t key_of(float v, int index) {
  const uint32_t b = f32_bits(v + 0.0f);                  // -0 equals 0
  const uint32_t order = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
  return (uint64_t)order << 32 | (uint32_t)~index;
}

__device__ __forceinline__ float value_of(uint64_t key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return bits_f32(o >> 31 ? o ^ 0x80000000u : ~o);
}

__device__ __forceinline__ int index_of(uint64_t key) { return (int)~(uint32_t)key; }

__device__ __forceinline__ uint64_t lane_key(uint64_t v, int lane) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane);
  return (uint64_t)hi << 32 | lo;
}

// The list with one more key in its place; what falls off the last lane is lost.
__device__ __forceinline__ uint64_t insert(uint64_t list, uint64_t key, int lane) {
  const int place = __popcll(__ballot(list > key));
  const uint64_t up = __shfl_up(list, 1);
  return lane < place ? list : lane == place ? key : up;
}

struct Sums {
  float m, s, e;
  // adds sums that go by another maximum
  __device__ __forceinline__ void add(const Sums& o, float c) {
    const float top = fmaxf(m, o.m), r = top == -INFINITY ? 0.0f : top;
    // an empty part has no share (and its maximum none either)
    const float d0 = s == 0.0f ? 0.0f : c * (m - r), d1 = o.s == 0.0f ? 0.0f : c * (o.m - r);
    const float f0 = __builtin_amdgcn_exp2f(d0), f1 = __builtin_amdgcn_exp2f(d1);
    // a share of 0 adds nothing, also where d is -infinity
    e = (f0 == 0.0f ? 0.0f : f0 * (e + d0 * s)) + (f1 == 0.0f ? 0.0f : f1 * (o.e + d1 * o.s));
    s = f0 * s + f1 * o.s;
    m = top;
  }
};

// Indices of a lane's values: runs of W that follow one another.
template <typename T> constexpr int kRun = 16 / sizeof(T);
template <typename T>
__device__ __forceinline__ int index_in_turn(int i, int lane) {
  return i / kRun<T> * (64 * kRun<T>) + lane * kRun<T> + i % kRun<T>;
}

// Values of a turn that starts at `base`; -infinity from n on. Rows may begin at any element.
template <typename T>
__device__ __forceinline__ void load_turn(const T* row, int base, int n, int lane, float* v) {
  constexpr int W = kRun<T>;
#pragma unroll
  for (int i = 0; i < kPer; i += W) {
    const int at = base + index_in_turn<T>(i, lane);
    if (at + W <= n) {
      T t[W];
      __builtin_memcpy(t, row + at, sizeof(t));
#pragma unroll
      for (int j = 0; j < W; ++j) v[i + j] = (float)t[j];
    } else {
#pragma unroll
      for (int j = 0; j < W; ++j) v[i + j] = at + j < n ? (float)row[at + j] : -INFINITY;
    }
  }
}

// Takes a turn's values into the wave's list.
template <typename T>
__device__ __forceinline__ uint64_t take_turn(uint64_t list, const float* v, int base, bool first,
                                              int top, int lane) {
  if (first) {
    // the lanes' largest, in order: a list that few of the others get into
    float best = v[0];
    int at = 0;
#pragma unroll
    for (int i = 1; i < kPer; ++i)
      if (v[i] > best) best = v[i], at = i;
    const uint64_t own = key_of(best, base + index_in_turn<T>(at, lane));
    int place = 0;
    for (int j = 0; j < 64; ++j) place += lane_key(own, j) > own;
    const int lo = __builtin_amdgcn_ds_permute(4 * place, (int)(uint32_t)own);
    const int hi = __builtin_amdgcn_ds_permute(4 * place, (int)(uint32_t)(own >> 32));
    list = (uint64_t)(uint32_t)hi << 32 | (uint32_t)lo;
    uint64_t bar = lane_key(list, top - 1);
    const float bar_v = value_of(bar);
    const int bar_i = index_of(bar) - base;
    uint32_t mask = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      mask |= (v[i] > bar_v || (v[i] == bar_v && index_in_turn<T>(i, lane) < bar_i)) ? 1u << i : 0;
    if (key_of(best, base + index_in_turn<T>(at, lane)) >= bar) mask &= ~(1u << at);  // there already
    while (__ballot(mask != 0)) {
      const int i = mask ? __ffs(mask) - 1 : 0;
      float x = v[0];
#pragma unroll
      for (int j = 1; j < kPer; ++j) x = i == j ? v[j] : x;
      const uint64_t key = mask ? key_of(x, base + index_in_turn<T>(i, lane)) : 0;
      uint64_t left = __ballot(mask != 0);
      while (left) {
        const int from = __ffsll((unsigned long long)left) - 1;
        left &= left - 1;
        const uint64_t one = lane_key(key, from);
        if (one > bar) {
          list = insert(list, one, lane);
          bar = lane_key(list, top - 1);
        }
      }
      mask &= mask - 1;
    }
    return list;
  }
  // later turns hold higher indices: equal values stay out
  uint64_t bar = lane_key(list, top - 1);
  const float bar_v = value_of(bar);
  uint32_t mask = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) mask |= v[i] > bar_v ? 1u << i : 0;
  while (__ballot(mask != 0)) {
    const int i = mask ? __ffs(mask) - 1 : 0;
    float x = v[0];
#pragma unroll
    for (int j = 1; j < kPer; ++j) x = i == j ? v[j] : x;
    const uint64_t key = mask ? key_of(x, base + index_in_turn<T>(i, lane)) : 0;
    uint64_t left = __ballot(mask != 0);
    while (left) {
      const int from = __ffsll((unsigned long long)left) - 1;
      left &= left - 1;
      const uint64_t one = lane_key(key, from);
      if (one > bar) {
        list = insert(list, one, lane);
        bar = lane_key(list, top - 1);
      }
    }
    mask &= mask - 1;
  }
  return list;
}

// One row or a part of it to a workgroup; its waves take turns of 64 * kPer values,
// which stay in registers between the search for the largest and the sums.
template <typename T, bool TOP>
__global__ __launch_bounds__(64 * kWaves) void logprobs(LogprobArgs a) {
  __shared__ Sums sums[kWaves];
  __shared__ uint64_t keys[kWaves * 64];
  __shared__ uint64_t best[64];
  __shared__ int last;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int row = blockIdx.x / a.parts, own = blockIdx.x % a.parts;
  const T* x = static_cast<const T*>(a.x) + (int64_t)row * a.ld_x;
  const int from = (int)((int64_t)a.chunks * own / a.parts);
  const int to = (int)((int64_t)a.chunks * (own + 1) / a.parts);
  Sums t = {-INFINITY, 0.0f, 0.0f};
  uint64_t list = 0;
  for (int chunk = from + wave; chunk < to; chunk += kWaves) {
    float v[kPer];
    load_turn(x, chunk * kTurn, a.n, lane, v);
    float m = v[0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) m = fmaxf(m, v[i]);
    Sums u = {m, 0.0f, 0.0f};
    const float r = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const float z = a.c * (v[i] - r), e = __builtin_amdgcn_exp2f(z);
      u.s += e;
      u.e = __builtin_fmaf(fmaxf(z, -1e4f), e, u.e);     // 0 where e is, z -infinity or not
    }
    t.add(u, a.c);
    if (TOP) list = take_turn<T>(list, v, chunk * kTurn, chunk == from + wave, a.top, lane);
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const Sums o = {__shfl_xor(t.m, d), __shfl_xor(t.s, d), __shfl_xor(t.e, d)};
    t.add(o, a.c);
  }
  if (lane == 0) sums[wave] = t;
  if (TOP) keys[threadIdx.x] = list;
  __syncthreads();
  t = sums[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) t.add(sums[w], a.c);
  const int top = TOP ? a.top : 0;
  if (TOP) {
    // a key's place among the waves' first `top`
    int place = lane < top && list ? 0 : 64;
    for (int w = 0; w < kWaves; ++w)
      for (int i = 0; i < top; ++i) place += keys[64 * w + i] > list;
    if (threadIdx.x < 64) best[threadIdx.x] = 0;
    __syncthreads();
    if (place < top) best[place] = list;
    __syncthreads();
  }
  if (a.parts > 1) {
    const int size = kPartFloats + 2 * top;
    float* mine = a.part + (int64_t)blockIdx.x * size;
    if (threadIdx.x == 0) {
      put_pair(mine, t.m, t.s);
      put_pair(mine + 2, t.e, 0.0f);
    }
    if (TOP && threadIdx.x < top)
      put_pair(mine + kPartFloats + 2 * threadIdx.x, bits_f32((uint32_t)best[threadIdx.x]),
               bits_f32((uint32_t)(best[threadIdx.x] >> 32)));
    if (!comes_last(a.count + row, a.parts, &last)) return;
    const float* all = a.part + (int64_t)row * a.parts * size;
    t = {-INFINITY, 0.0f, 0.0f};
    for (int p = 0; p < a.parts; ++p) {
      const f32x2 ms = get_pair(all + (int64_t)p * size), e = get_pair(all + (int64_t)p * size + 2);
      t.add({ms[0], ms[1], e[0]}, a.c);
    }
    if (TOP && wave == 0) {
      list = best[lane];
      for (int p = 0; p < a.parts; ++p) {
        if (p == own) continue;
        uint64_t key = 0;
        if (lane < top) {
          const f32x2 k = get_pair(all + (int64_t)p * size + kPartFloats + 2 * lane);
          key = (uint64_t)f32_bits(k[1]) << 32 | f32_bits(k[0]);
        }
        for (int i = 0; i < top; ++i) {
          const uint64_t one = lane_key(key, i);
          if (one <= lane_key(list, top - 1)) break;
          list = insert(list, one, lane);
        }
      }
      best[lane] = list;
    }
    __syncthreads();
  }
  // a row of -infinity alone has no probability anywhere; with a NaN or an
  // infinity in it (S is NaN) it has no distribution
  const bool empty = t.s == 0.0f;
  const float r = empty ? 0.0f : t.m, log = empty ? 0.0f : logf(t.s);
  if (threadIdx.x == 0) {
    if (a.entropy) a.entropy[row] = empty ? 0.0f : log - kLn2 * (t.e / t.s);
    if (a.logprob) {
      const int token = a.tokens[row];
      float p = 0.0f;
      if (token >= a.n) p = bits_f32(0x7FC00000u);
      else if (token >= 0) p = a.scale * ((float)x[token] - r) - log;
      a.logprob[row] = p;
    }
  }
  if (TOP && threadIdx.x < top) {
    const uint64_t key = best[threadIdx.x];
    const bool none = t.s != t.s;
    a.top_logprobs[row * a.ld_top + threadIdx.x] =
        none ? bits_f32(0x7FC00000u) : a.scale * (value_of(key) - r) - log;
    a.top_tokens[row * a.ld_top + threadIdx.x] = none ? -1 : index_of(key);
  }
}

int32_t parts_of(int64_t rows, int64_t n) {
  const int64_t chunks = (n + kTurn - 1) / kTurn;
  // a few workgroups for each CU, and a turn for each wave at least
  const int64_t most = std::min<int64_t>(1024 / std::max<int64_t>(rows, 1), 64);
  return (int32_t)std::max<int64_t>(1, std::min(most, chunks / kWaves));
}

}  // namespace

size_t logprobs_workspace_bytes(const ifq_logprobs_desc& d) {
  if (d.rows == 0) return 0;
  const int64_t parts = parts_of(d.rows, d.n);
  if (parts == 1) return 0;
  return kSplitCounterBytes + d.rows * parts * (kPartFloats + 2 * d.top) * sizeof(float);
}

int64_t logprobs_groups(const ifq_logprobs_desc& d) { return d.rows * parts_of(d.rows, d.n); }

hipError_t launch_logprobs(const ifq_logprobs_desc& d, const void* logits, const int32_t* tokens,
                           float* logprob, float* entropy, float* top_logprobs,
                           int32_t* top_tokens, void* ws, hipStream_t stream) {
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
  a.parts = parts_of(d.rows, d.n);
  a.chunks = (int32_t)((d.n + kTurn - 1) / kTurn);
  a.scale = d.scale;
  a.c = d.scale * 1.4426950408889634f;
  const dim3 grid((uint32_t)logprobs_groups(d)), block(64 * kWaves);
  auto go = [&](auto zero) {
    typedef decltype(zero) T;
    if (d.top) hipLaunchKernelGGL((logprobs<T, true>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((logprobs<T, false>), grid, block, 0, stream, a);
  };
  if (d.x_type == IFQ_TYPE_BF16) go(__bf16(0));
  else if (d.x_type == IFQ_TYPE_F16) go(_Float16(0));
  else go(0.0f);
  return hipGetLastError();
}

}  // namespace ifq
