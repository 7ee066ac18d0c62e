// Attention over a paged cache of 4-bit codes (its format: include/ifq.h,
// ifq_kv_desc).
//
// With row j standing for o_j + t_j * c_j, the codes enter the matrix
// instructions as they are and the offsets and steps are applied to sums:
//   q.k_j            = t_j * (q.(c_j - 8)) + (o_j + 8 t_j) * sum(q)
//   sum_j p_j v_j    = sum_j (p_j t_j) (c_j - 8) + sum_j p_j (o_j + 8 t_j)
// A code becomes the 16-bit float 16 + c by a shift, a mask and an or on two
// codes at once (the exponent of 16 leaves the mantissa to c); the remaining
// -24 is the accumulator's start -24 * sum(q) in the first product, and in
// the second -24 * sum of the factors, which one more matrix instruction adds
// up exactly as the others see them. Only q (as given) and p_j t_j are
// operands of 16 bits; p_j t_j goes in as the sum of two bfloat16 numbers, so
// that 16 bits of it are kept and its range is that of fp32.
//
// The first product is taken transposed (rows: tokens, columns: query rows),
// which leaves a lane with the tokens 16u + 4g + r of its query column: the
// tokens that it holds as the second product's operand, in the same order in
// which the values' codes are stored. Nothing moves between lanes.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ifq_serve.h"

namespace ifq {
namespace {

constexpr int64_t kTargetGroups = 2048;   // workgroups that split work aims at

struct AttnArgs {
  KvArgs c;
  const void* q;
  void* out;
  float* part;          // partial results of split sequences
  uint32_t* count;      // arrivals per unit of split work
  int64_t q_stride, o_stride;
  int32_t ratio;        // query heads per key/value head
  int32_t causal, window, sinks;
  float factor;         // scale * log2(e)
  int32_t row_blocks;   // blocks of a sequence's ratio * max_q query rows
  int32_t splits, chunk;  // parts at most, and steps of a part at least
};

template <typename T>
struct Half;
template <>
struct Half<__bf16> {
  typedef bf16x8 x8;
  // bits of 16.0 and where a code lies in the mantissa
  static constexpr uint32_t kBase = 0x41804180u, kMask = 0x00780078u;
  static constexpr int kAt = 3;
  static __device__ __forceinline__ f32x4 mfma(x8 a, x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Half<_Float16> {
  typedef f16x8 x8;
  static constexpr uint32_t kBase = 0x4C004C00u, kMask = 0x03C003C0u;
  static constexpr int kAt = 6;
  static __device__ __forceinline__ f32x4 mfma(x8 a, x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};

// Eight codes of a word (nibble p + 4h: element 2p + h) as 16 + c.
template <typename H>
__device__ __forceinline__ typename H::x8 codes8(uint32_t w) {
  u32x4 r;
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const int s = 4 * p - H::kAt;
    r[p] = ((s < 0 ? w << -s : w >> s) & H::kMask) | H::kBase;
  }
  return __builtin_bit_cast(typename H::x8, r);
}

// Eight fp32 numbers as the sums of two bfloat16 each: the upper half of the
// bits, and what remains, rounded.
__device__ __forceinline__ void split8(const float* x, u32x4& hi, u32x4& lo) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = f32_bits(x[2 * i]), b = f32_bits(x[2 * i + 1]);
    hi[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    bf16x2 r;
    r[0] = (__bf16)(x[2 * i] - bits_f32(a & 0xFFFF0000u));
    r[1] = (__bf16)(x[2 * i + 1] - bits_f32(b & 0xFFFF0000u));
    lo[i] = __builtin_bit_cast(uint32_t, r);
  }
}

// Over the four lanes that hold a column's tokens.
__device__ __forceinline__ float max_g(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum_g(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// What the query rows of a wave see: blocks of 32 positions, first those of
// the sinks, then those from the window's begin to the last position.
struct View {
  int32_t blocks, sink_blocks, first;   // first: block where the window begins
  __device__ __forceinline__ int block(int i) const {
    return i < sink_blocks ? i : i - sink_blocks + first;
  }
};

__device__ __forceinline__ View view_of(const AttnArgs& a, int p_lo, int p_hi) {
  View v = {0, 0, 0};
  if (p_hi < 0) return v;
  const int lo = a.window > 0 ? max(p_lo - a.window + 1, 0) : 0;
  v.first = lo / kCodeTokens;
  if (a.window > 0)
    v.sink_blocks = min((a.sinks + kCodeTokens - 1) / kCodeTokens, v.first);
  v.blocks = v.sink_blocks + p_hi / kCodeTokens - v.first + 1;
  return v;
}

// Where, in the order of the view's blocks, those that hold positions up to p end.
__device__ __forceinline__ int visible_end(const View& v, int p) {
  return p < 0 ? 0 : p / kCodeTokens < v.first ? v.blocks
                                                : v.sink_blocks + p / kCodeTokens - v.first + 1;
}

// A sequence's new tokens (queries) and cached tokens.
struct Seq {
  int32_t row, count, length, pos;     // pos: position of the first query
};

__device__ __forceinline__ Seq seq_of(const KvArgs& c, int b) {
  const int lo = min(max(c.offsets[b], 0), c.total_q);
  const int hi = min(max(c.offsets[b + 1], lo), c.total_q);
  Seq s;
  s.row = lo;
  s.count = min(hi - lo, c.max_q);
  s.length = min(max(c.lengths[b], 0), c.max_pages * c.page_tokens);
  s.pos = max(c.lengths[b], 0) - (hi - lo);
  return s;
}

// Running softmax and weighted sums of TILES x 16 query columns.
template <int D, int TILES>
struct State {
  f32x4 acc[TILES][D / 16];   // sums of factors * (16 + c): dims 16 x + 4g + r of a column
  f32x4 wsum[TILES];          // sums of the factors, the same in every row
  float m[TILES], mu[TILES];  // largest score so far, and the same or 0 where there is none
  float l[TILES], ob[TILES];  // this lane's sums of p and of p * (o + 8 t)
};

// A block's place: its page's head (page 0 where the cache has no such page,
// whose tokens are then hidden) and its first token there.
struct Place {
  const uint8_t* head;
  int32_t tp, j0;             // j0: position of the first token
  bool held;
};

__device__ __forceinline__ Place place_of(const KvArgs& c, const View& view, int i, int id,
                                          int64_t head_at, int per_page) {
  Place p;
  const int blk = view.block(i);
  p.held = id >= 0 && id < c.num_pages;
  p.head = c.cache + (p.held ? id : 0) * c.page_bytes + head_at;
  p.tp = (per_page & (per_page - 1)) ? blk % per_page : blk & (per_page - 1);
  p.tp *= kCodeTokens;
  p.j0 = blk * kCodeTokens;
  return p;
}

// Runs steps i = begin, begin + step .. below end of the view over the query
// columns, U blocks (U * i ..) at a step: column n stands for query row
// n % (16 / U) and sees only block n / (16 / U) of the U, so that with few
// rows all columns take part in the softmax. pos: the position of this lane's
// query in each tile. A step's loads are issued a step ahead: the keys' after
// their last use, the values' likewise.
template <typename T, int D, int U, int TILES>
__device__ __forceinline__ void attend(const AttnArgs& a, const View& view, int b, int hk,
                                       int begin, int end, int step,
                                       const typename Half<T>::x8 (&q)[TILES][D / 32],
                                       const int (&pos)[TILES], int p_lo, int p_hi,
                                       State<D, TILES>& s) {
  typedef Half<T> H;
  static_assert(U == 1 || TILES == 1, "");
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int mine = n / (16 / U);          // the block of the U that this column sees
  const KvArgs& c = a.c;
  float qc[TILES];      // factor * sum(q)
  f32x4 init[TILES];    // -24 * sum(q)
#pragma unroll
  for (int x = 0; x < TILES; ++x) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += (float)q[x][i][e];
    sum = sum_g(sum);
    qc[x] = sum * a.factor;
    init[x] = f32x4{-24.0f * sum, -24.0f * sum, -24.0f * sum, -24.0f * sum};
    s.m[x] = -__builtin_inff();
    s.mu[x] = s.l[x] = s.ob[x] = 0.0f;
    s.wsum[x] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int d = 0; d < D / 16; ++d) s.acc[x][d] = f32x4{0, 0, 0, 0};
  }
  if (begin >= end) return;
  const u32x4 ones = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
  const int per_page = c.page_tokens / kCodeTokens;
  const int32_t* table = c.pages + (int64_t)b * c.max_pages;
  const int64_t head_at = hk * c.head_bytes;
  const int last = view.blocks - 1;

  uint32_t kw[U][2][D / 32];
  u32x4 vw[U][D / 64], kp[2], vp[2];
  Place now[U], next[U];
  auto find = [&](int i, Place* p) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = min(U * i + u, last);
      p[u] = place_of(c, view, at, table[view.block(at) / per_page], head_at, per_page);
    }
  };
  auto load_keys = [&](const Place* p) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint32_t* src = reinterpret_cast<const uint32_t*>(
            p[u].head + (p[u].tp + 16 * t + n) * (D / 2) + g * (D / 8));
#pragma unroll
        for (int w = 0; w < D / 32; ++w) kw[u][t][w] = src[w];
      }
  };
  // the words of this column's tokens, of keys (part 0) or values
  auto load_words = [&](const Place* p, int part, u32x4* to) {
    const uint8_t* head = p[0].head;
    int tp = p[0].tp;
#pragma unroll
    for (int u = 1; u < U; ++u) {
      head = mine == u ? p[u].head : head;
      tp = mine == u ? p[u].tp : tp;
    }
    const uint8_t* src = head + c.page_tokens * (D + 4 * part) + 4 * (tp + 4 * g);
    to[0] = *reinterpret_cast<const u32x4*>(src);
    to[1] = *reinterpret_cast<const u32x4*>(src + 64);
  };
  auto load_values = [&](const Place* p) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int x = 0; x < D / 64; ++x)
        vw[u][x] = *reinterpret_cast<const u32x4*>(
            p[u].head + (c.page_tokens + p[u].tp) * (D / 2) + x * 1024 + lane * 16);
  };

  find(begin, now);
  load_keys(now);
  load_words(now, 0, kp);
  load_values(now);
  load_words(now, 1, vp);
  for (int i = begin; i < end; i += step) {
    const int ahead = min(i + step, end - 1);
    find(ahead, next);
    int j0 = now[0].j0;
    bool held = now[0].held && U * i <= last;
    bool masked = false;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool there = now[u].held && U * i + u <= last;
      masked |= !there || now[u].j0 + kCodeTokens - 1 > p_lo ||
                (a.window > 0 && now[u].j0 <= p_hi - a.window);
      if (u > 0) {
        j0 = mine == u ? now[u].j0 : j0;
        held = mine == u ? there : held;
      }
    }
    float sc[TILES][8];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x4 d[TILES];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        f32x4 e[TILES];
#pragma unroll
        for (int x = 0; x < TILES; ++x) e[x] = init[x];
#pragma unroll
        for (int w = 0; w < D / 32; ++w) {
          const typename H::x8 k = codes8<H>(kw[u][t][w]);
#pragma unroll
          for (int x = 0; x < TILES; ++x) e[x] = H::mfma(k, q[x][w], e[x]);
        }
#pragma unroll
        for (int x = 0; x < TILES; ++x)
#pragma unroll
          for (int r = 0; r < 4; ++r) d[x][r] = u == 0 || mine == u ? e[x][r] : d[x][r];
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float st = row_step(kp[t][r]), o = row_offset(kp[t][r]);
        const float f = st * a.factor, mid = __builtin_fmaf(8.0f, st, o);
#pragma unroll
        for (int x = 0; x < TILES; ++x) sc[x][4 * t + r] = __builtin_fmaf(d[x][r], f, mid * qc[x]);
      }
    }
    load_keys(next);
    load_words(next, 0, kp);
    float vt[8], vo[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      vt[e] = row_step(vp[e >> 2][e & 3]);
      vo[e] = __builtin_fmaf(8.0f, vt[e], row_offset(vp[e >> 2][e & 3]));
    }
    u32x4 hi[TILES], lo[TILES];
#pragma unroll
    for (int x = 0; x < TILES; ++x) {
      float tt[8], oo[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) tt[e] = vt[e], oo[e] = vo[e];
      if (masked) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int j = j0 + 16 * (e >> 2) + 4 * g + (e & 3);
          const bool sees = held && j <= pos[x] &&
                            (a.window == 0 || j > pos[x] - a.window || j < a.sinks);
          sc[x][e] = sees ? sc[x][e] : -__builtin_inff();
          // what a hidden row holds must not reach the sums, not even as 0 * NaN
          tt[e] = sees ? tt[e] : 0.0f;
          oo[e] = sees ? oo[e] : 0.0f;
        }
      }
      float top = sc[x][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top = fmaxf(top, sc[x][e]);
      // the maximum is raised only where a score passes it by 8 (a factor of
      // 256 in p): sums keep their precision, and they are seldom rescaled
      if (__ballot(top > s.m[x] + 8.0f)) {
        const float m = fmaxf(s.m[x], max_g(top));
        const float mu = m == -__builtin_inff() ? 0.0f : m;
        const float f = __builtin_amdgcn_exp2f(s.m[x] - mu);
        s.m[x] = m;
        s.mu[x] = mu;
        s.l[x] *= f;
        s.ob[x] *= f;
        s.wsum[x] *= f;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) s.acc[x][d] *= f;
      }
      float fac[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p = __builtin_amdgcn_exp2f(sc[x][e] - s.mu[x]);
        s.l[x] += p;
        s.ob[x] = __builtin_fmaf(p, oo[e], s.ob[x]);
        fac[e] = p * tt[e];
      }
      split8(fac, hi[x], lo[x]);
      const bf16x8 one = __builtin_bit_cast(bf16x8, ones);
      s.wsum[x] = Half<__bf16>::mfma(one, __builtin_bit_cast(bf16x8, hi[x]), s.wsum[x]);
      s.wsum[x] = Half<__bf16>::mfma(one, __builtin_bit_cast(bf16x8, lo[x]), s.wsum[x]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      bf16x8 fh[TILES], fl[TILES];
#pragma unroll
      for (int x = 0; x < TILES; ++x) {
        // block u counts for its own columns alone
        const uint32_t keep = U == 1 || mine == u ? 0xFFFFFFFFu : 0u;
        fh[x] = __builtin_bit_cast(bf16x8, hi[x] & keep);
        fl[x] = __builtin_bit_cast(bf16x8, lo[x] & keep);
      }
#pragma unroll
      for (int d = 0; d < D / 16; ++d) {
        const bf16x8 v = codes8<Half<__bf16>>(vw[u][d >> 2][d & 3]);
#pragma unroll
        for (int x = 0; x < TILES; ++x) {
          s.acc[x][d] = Half<__bf16>::mfma(v, fh[x], s.acc[x][d]);
          s.acc[x][d] = Half<__bf16>::mfma(v, fl[x], s.acc[x][d]);
        }
      }
    }
    load_values(next);
    load_words(next, 1, vp);
#pragma unroll
    for (int u = 0; u < U; ++u) now[u] = next[u];
  }
#pragma unroll
  for (int x = 0; x < TILES; ++x) {
    s.l[x] = sum_g(s.l[x]);
    s.ob[x] = sum_g(s.ob[x]);
  }
}

// Query row `row` of a sequence (row = token * ratio + head of the group) as
// this lane's operand column, and its position; rows past the last repeat it.
template <typename T, int D>
__device__ __forceinline__ void load_row(const AttnArgs& a, const Seq& s, int hk, int row,
                                         typename Half<T>::x8 (&q)[D / 32], int& pos) {
  const int g = (threadIdx.x & 63) >> 4;
  row = min(row, s.count * a.ratio - 1);
  const int token = row / a.ratio, h = hk * a.ratio + row % a.ratio;
  const T* src = static_cast<const T*>(a.q) + (int64_t)(s.row + token) * a.q_stride +
                 (int64_t)h * D + g * (D / 4);
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
    q[i] = *reinterpret_cast<const typename Half<T>::x8*>(src + 8 * i);
  pos = a.causal ? min(s.pos + token, s.length - 1) : s.length - 1;
}

template <typename T, int D>
__device__ __forceinline__ T* out_row(const AttnArgs& a, const Seq& s, int hk, int row) {
  return static_cast<T*>(a.out) + (int64_t)(s.row + row / a.ratio) * a.o_stride +
         (int64_t)(hk * a.ratio + row % a.ratio) * D;
}

template <typename T>
__device__ __forceinline__ void store4(T* p, f32x4 v) {
  typedef T t4 __attribute__((ext_vector_type(4)));
  *reinterpret_cast<t4*>(p) = t4{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
}

// Parts go through memory between workgroups whose caches do not see one
// another. Each number is written through to where all see it and read from
// there (accesses of agent scope), so that no workgroup has to write back or
// drop a whole cache for it: with fences around plain accesses 768 sequences
// and heads in two parts each took 382 us instead of 74 unsplit.
__device__ __forceinline__ void put_pair(float* p, float x, float y) {
  const uint64_t v = f32_bits(x) | (uint64_t)f32_bits(y) << 32;
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), v, __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ f32x2 get_pair(const float* p) {
  return __builtin_bit_cast(f32x2, __hip_atomic_load(reinterpret_cast<const uint64_t*>(p),
                                                     __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

__device__ __forceinline__ void put_sums(float* row, int d, f32x4 o) {
  put_pair(row + d, o[0], o[1]);
  put_pair(row + d + 2, o[2], o[3]);
}

// Joins the parts of a unit's rows in their order, in the workgroup that
// counts itself last. Called by all of a workgroup's threads after they have
// written its part ([rows][D + 4]: sums, then m and l).
template <typename T, int D, int ROWS>
__device__ __forceinline__ void join_parts(const AttnArgs& a, const Seq& s, int unit, int hk,
                                           int row0, int live, int parts) {
  __shared__ int last;
  // the part is in memory before the barrier, and so before the count
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0)
    last = atomicInc(a.count + unit, (uint32_t)(parts - 1)) == (uint32_t)(parts - 1);
  __syncthreads();
  if (!last) return;
  constexpr int LD = D + 4;
  const float* src = a.part + (int64_t)unit * a.splits * ROWS * LD;
  for (int i = threadIdx.x; i < live * (D / 4); i += 256) {
    const int r = i / (D / 4), d = i % (D / 4) * 4;
    float m = -__builtin_inff(), l = 0.0f;
    f32x4 o = {0, 0, 0, 0};
    for (int p = 0; p < parts; ++p) {
      const float* at = src + (int64_t)(p * ROWS + r) * LD;
      const f32x2 ml = get_pair(at + D), x = get_pair(at + d), y = get_pair(at + d + 2);
      const f32x4 v = {x[0], x[1], y[0], y[1]};
      const float top = fmaxf(m, ml[0]), mu = top == -__builtin_inff() ? 0.0f : top;
      const float f = __builtin_amdgcn_exp2f(m - mu), pf = __builtin_amdgcn_exp2f(ml[0] - mu);
      l = f * l + pf * ml[1];
      o = f * o + pf * v;
      m = top;
    }
    store4(out_row<T, D>(a, s, hk, row0 + r) + d, o * (l == 0.0f ? 0.0f : 1.0f / l));
  }
}

// Up to 16 / U query rows: the four waves of a workgroup take every fourth
// step of its part of the sequence for the same rows, and join their results
// in LDS.
template <typename T, int D, int U>
__global__ __launch_bounds__(256) void kv_attention_few(AttnArgs a) {
  constexpr int ROWS = 16 / U, LD = D + 4;
  __shared__ __align__(16) float osum[4][16][LD];
  __shared__ float ml[4][16][2];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int unit = blockIdx.x / a.splits, part = blockIdx.x % a.splits;
  const int hk = unit % a.c.kv_heads;
  const int rb = unit / a.c.kv_heads % a.row_blocks;
  const int b = unit / a.c.kv_heads / a.row_blocks;
  const Seq s = seq_of(a.c, b);
  const int rows = s.count * a.ratio, row0 = rb * ROWS;
  if (row0 >= rows) return;
  const int live = min(ROWS, rows - row0);
  const int p_lo = a.causal ? min(s.pos + row0 / a.ratio, s.length - 1) : s.length - 1;
  const int p_hi = a.causal ? min(s.pos + (row0 + live - 1) / a.ratio, s.length - 1)
                            : s.length - 1;
  const View view = view_of(a, p_lo, p_hi);
  // parts of `chunk` steps; longer ones where the sequence is longer than planned
  const int steps = (view.blocks + U - 1) / U;
  const int chunk = max(a.chunk, (steps + a.splits - 1) / a.splits);
  const int parts = max(1, (steps + chunk - 1) / chunk);
  if (part >= parts) return;
  typename Half<T>::x8 q[1][D / 32];
  int pos[1];
  load_row<T, D>(a, s, hk, row0 + n % ROWS, q[0], pos[0]);
  State<D, 1> st;
  attend<T, D, U, 1>(a, view, b, hk, part * chunk + wave, min(steps, (part + 1) * chunk), 4, q,
                     pos, p_lo, p_hi, st);
  const float corr = st.ob[0] - 24.0f * st.wsum[0][0];
#pragma unroll
  for (int d = 0; d < D / 16; ++d)
    *reinterpret_cast<f32x4*>(&osum[wave][n][16 * d + 4 * g]) = st.acc[0][d] + corr;
  if (g == 0) {
    ml[wave][n][0] = st.m[0];
    ml[wave][n][1] = st.l[0];
  }
  __syncthreads();
  float* dst = parts > 1 ? a.part + (int64_t)(unit * a.splits + part) * ROWS * LD : nullptr;
  for (int i = threadIdx.x; i < live * (D / 4); i += 256) {
    const int r = i / (D / 4), d = i % (D / 4) * 4;
    float m = -__builtin_inff();
#pragma unroll
    for (int w = 0; w < 4 * U; ++w) m = fmaxf(m, ml[w / U][w % U * ROWS + r][0]);
    const float mu = m == -__builtin_inff() ? 0.0f : m;
    float l = 0.0f;
    f32x4 o = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < 4 * U; ++w) {
      const int at = w % U * ROWS + r;
      const float f = __builtin_amdgcn_exp2f(ml[w / U][at][0] - mu);
      l += f * ml[w / U][at][1];
      o += f * *reinterpret_cast<const f32x4*>(&osum[w / U][at][d]);
    }
    if (parts > 1) {
      put_sums(dst + r * LD, d, o);
      if (d == 0) put_pair(dst + r * LD + D, m, l);
    } else {
      store4(out_row<T, D>(a, s, hk, row0 + r) + d, o * (l == 0.0f ? 0.0f : 1.0f / l));
    }
  }
  if (parts > 1) join_parts<T, D, ROWS>(a, s, unit, hk, row0, live, parts);
}

// Many query rows: each wave has TILES x 16 rows of its own and runs through
// all that they see of the workgroup's part. The last rows, which see most,
// come first.
template <typename T, int D, int TILES>
__global__ __launch_bounds__(256) void kv_attention_many(AttnArgs a) {
  constexpr int WROWS = 16 * TILES, ROWS = 4 * WROWS, LD = D + 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int unit = blockIdx.x / a.splits, part = blockIdx.x % a.splits;
  const int hk = unit % a.c.kv_heads;
  const int rb = a.row_blocks - 1 - unit / a.c.kv_heads % a.row_blocks;
  const int b = unit / a.c.kv_heads / a.row_blocks;
  const Seq s = seq_of(a.c, b);
  const int rows = s.count * a.ratio;
  if (rb * ROWS >= rows) return;
  // the split goes by what all of the workgroup's rows see
  const int live = min(ROWS, rows - rb * ROWS);
  const int g_lo = a.causal ? min(s.pos + rb * ROWS / a.ratio, s.length - 1) : s.length - 1;
  const int g_hi = a.causal ? min(s.pos + (rb * ROWS + live - 1) / a.ratio, s.length - 1)
                            : s.length - 1;
  const View all = view_of(a, g_lo, g_hi);
  const int chunk = max(a.chunk, (all.blocks + a.splits - 1) / a.splits);
  const int parts = max(1, (all.blocks + chunk - 1) / chunk);
  if (part >= parts) return;
  const int row0 = rb * ROWS + wave * WROWS;
  const int own = min(WROWS, rows - row0);
  if (own > 0) {
    const int p_lo = a.causal ? min(s.pos + row0 / a.ratio, s.length - 1) : s.length - 1;
    const int p_hi = a.causal ? min(s.pos + (row0 + own - 1) / a.ratio, s.length - 1)
                              : s.length - 1;
    typename Half<T>::x8 q[TILES][D / 32];
    int pos[TILES];
#pragma unroll
    for (int x = 0; x < TILES; ++x) load_row<T, D>(a, s, hk, row0 + 16 * x + n, q[x], pos[x]);
    State<D, TILES> st;
    attend<T, D, 1, TILES>(a, all, b, hk, part * chunk,
                           min(min(all.blocks, (part + 1) * chunk), visible_end(all, p_hi)), 1, q,
                           pos, p_lo, p_hi, st);
    float* dst = parts > 1 ? a.part + ((int64_t)(unit * a.splits + part) * ROWS +
                                       wave * WROWS) * LD : nullptr;
#pragma unroll
    for (int x = 0; x < TILES; ++x) {
      const int r = 16 * x + n;
      if (r < own) {
        const float corr = st.ob[x] - 24.0f * st.wsum[x][0];
        if (parts > 1) {
#pragma unroll
          for (int d = 0; d < D / 16; ++d)
            put_sums(dst + r * LD, 16 * d + 4 * g, st.acc[x][d] + corr);
          if (g == 0) put_pair(dst + r * LD + D, st.m[x], st.l[x]);
        } else {
          const float f = st.l[x] == 0.0f ? 0.0f : 1.0f / st.l[x];
          T* out = out_row<T, D>(a, s, hk, row0 + r) + 4 * g;
#pragma unroll
          for (int d = 0; d < D / 16; ++d) store4(out + 16 * d, (st.acc[x][d] + corr) * f);
        }
      }
    }
  }
  if (parts > 1) join_parts<T, D, ROWS>(a, s, unit, hk, rb * ROWS, live, parts);
}

// Which kernel, and how its work is split.
struct Plan {
  int32_t few;            // blocks of a step for few rows (U), 0: many rows
  int32_t tiles;          // tiles of 16 rows per wave, many rows
  int32_t row_blocks, splits, chunk;
  int64_t units;
  int32_t rows;           // per unit
};

Plan plan_of(const ifq_kv_desc& d) {
  Plan p;
  const int64_t rows = (int64_t)d.max_q * (d.heads / d.kv_heads);
  p.few = rows <= 4 && d.head_dim < 256 ? 4 : rows <= 8 ? 2 : rows <= 16 ? 1 : 0;
  p.tiles = d.head_dim == 256 ? 1 : 2;
  p.rows = p.few ? 16 / p.few : 64 * p.tiles;
  p.row_blocks = (int32_t)((rows + p.rows - 1) / p.rows);
  p.units = (int64_t)d.batch * d.kv_heads * p.row_blocks;
  // blocks that a unit may see, and steps of them
  int64_t blocks = ((int64_t)d.max_kv + kCodeTokens - 1) / kCodeTokens + 1;
  if (d.window > 0) {
    const int64_t seen = ((int64_t)d.window + d.max_q + kCodeTokens) / kCodeTokens +
                         (d.sinks + kCodeTokens - 1) / kCodeTokens + 1;
    blocks = std::min(blocks, seen);
  }
  const int64_t steps = p.few ? (blocks + p.few - 1) / p.few : blocks;
  const int64_t least = p.few ? 8 : 16;          // steps that are worth a workgroup
  const int64_t want = std::max<int64_t>(1, kTargetGroups / p.units);
  int64_t chunk = std::max(least, (steps + want - 1) / want);
  if (p.few) chunk = (chunk + 3) / 4 * 4;
  p.chunk = (int32_t)chunk;
  p.splits = (int32_t)std::max<int64_t>(1, (steps + chunk - 1) / chunk);
  // one arrival counter for each unit
  if (p.units * (int64_t)sizeof(uint32_t) > kSplitCounterBytes) p.splits = 1;
  return p;
}

template <typename T, int D>
hipError_t launch(const AttnArgs& a, const Plan& p, hipStream_t stream) {
  const dim3 grid((uint32_t)(p.units * p.splits)), block(256);
  constexpr int TILES = D == 256 ? 1 : 2;
  if (p.few == 4) {
    if constexpr (D < 256)
      hipLaunchKernelGGL((kv_attention_few<T, D, 4>), grid, block, 0, stream, a);
  } else if (p.few == 2) {
    hipLaunchKernelGGL((kv_attention_few<T, D, 2>), grid, block, 0, stream, a);
  } else if (p.few == 1) {
    hipLaunchKernelGGL((kv_attention_few<T, D, 1>), grid, block, 0, stream, a);
  } else {
    hipLaunchKernelGGL((kv_attention_many<T, D, TILES>), grid, block, 0, stream, a);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t launch(const AttnArgs& a, const Plan& p, int head_dim, hipStream_t stream) {
  if (head_dim == 64) return launch<T, 64>(a, p, stream);
  if (head_dim == 128) return launch<T, 128>(a, p, stream);
  return launch<T, 256>(a, p, stream);
}

}  // namespace

size_t kv_attention_workspace_bytes(const ifq_kv_desc& d) {
  const Plan p = plan_of(d);
  if (p.splits == 1) return 0;
  return kSplitCounterBytes +
         (size_t)p.units * p.splits * p.rows * (d.head_dim + 4) * sizeof(float);
}

hipError_t launch_kv_attention(const ifq_kv_desc& d, const void* q, const KvArgs& c, void* out,
                               void* ws, hipStream_t stream) {
  const Plan p = plan_of(d);
  AttnArgs a;
  a.c = c;
  a.q = q;
  a.out = out;
  a.count = static_cast<uint32_t*>(ws);
  a.part = ws ? reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + kSplitCounterBytes)
              : nullptr;
  a.q_stride = d.q_stride;
  a.o_stride = d.o_stride;
  a.ratio = d.heads / d.kv_heads;
  a.causal = d.causal;
  a.window = d.window;
  a.sinks = d.sinks;
  a.factor = d.scale * 1.4426950408889634f;
  a.row_blocks = p.row_blocks;
  a.splits = p.splits;
  a.chunk = p.chunk;
  if (p.units * p.splits > kMaxGroups) return hipErrorInvalidConfiguration;
  return d.type == IFQ_TYPE_BF16 ? launch<__bf16>(a, p, d.head_dim, stream)
                                 : launch<_Float16>(a, p, d.head_dim, stream);
}

}  // namespace ifq
