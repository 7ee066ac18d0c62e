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

#include "ifq_serve.h"

namespace ifq {
namespace {

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
  int32_t row_blocks;   // of a sequence's ratio * max_q query rows
  int32_t splits, chunk;
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
  const int lo = a.window > 0 ? max((int)max((int64_t)p_lo - a.window + 1, (int64_t)0), 0) : 0;
  v.first = lo / kCodeTokens;
  if (a.window > 0)
    v.sink_blocks = min((a.sinks + kCodeTokens - 1) / kCodeTokens, v.first);
  v.blocks = v.sink_blocks + p_hi / kCodeTokens - v.first + 1;
  return v;
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

// Running softmax and weighted sums of TILES x 16 query rows, a column each.
template <int D, int TILES>
struct State {
  f32x4 acc[TILES][D / 16];   // sums of factors * (16 + c): dims 16 x + 4g + r of a column
  f32x4 wsum[TILES];          // sums of the factors, the same in every row
  float m[TILES], mu[TILES];  // largest score so far, and the same or 0 where there is none
  float l[TILES], ob[TILES];  // this lane's sums of p and of p * (o + 8 t)
};

// Runs blocks begin + step * i (i = 0 ..) below end of the view over the
// query tiles. pos: the position of this lane's query in each tile.
template <typename T, int D, int TILES>
__device__ __forceinline__ void attend(const AttnArgs& a, const View& view, int b, int hk,
                                       int begin, int end, int step,
                                       const typename Half<T>::x8 (&q)[TILES][D / 32],
                                       const int (&pos)[TILES], int p_lo, int p_hi,
                                       State<D, TILES>& s) {
  typedef Half<T> H;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
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
  const u32x4 ones = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
  const int per_page = c.page_tokens / kCodeTokens;
  for (int i = begin; i < end; i += step) {
    const int blk = view.block(i);
    const int id = c.pages[(int64_t)b * c.max_pages + blk / per_page];
    const bool held = id >= 0 && id < c.num_pages;
    const uint8_t* head = c.cache + (held ? id : 0) * c.page_bytes + hk * c.head_bytes;
    const int tp = blk % per_page * kCodeTokens;
    // the block's words
    uint32_t kw[2][D / 32];
    u32x4 vw[D / 64], kp[2], vp[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint32_t* src = reinterpret_cast<const uint32_t*>(
          head + (tp + 16 * u + n) * (D / 2) + g * (D / 8));
#pragma unroll
      for (int w = 0; w < D / 32; ++w) kw[u][w] = src[w];
      const uint8_t* prm = head + c.page_tokens * D + 4 * (tp + 16 * u + 4 * g);
      kp[u] = *reinterpret_cast<const u32x4*>(prm);
      vp[u] = *reinterpret_cast<const u32x4*>(prm + 4 * c.page_tokens);
    }
#pragma unroll
    for (int x = 0; x < D / 64; ++x)
      vw[x] = *reinterpret_cast<const u32x4*>(head + (c.page_tokens + tp) * (D / 2) + x * 1024 +
                                              lane * 16);
    const int j0 = blk * kCodeTokens;
    const bool masked = !held || j0 + kCodeTokens - 1 > p_lo ||
                        (a.window > 0 && j0 <= p_hi - a.window);
#pragma unroll
    for (int x = 0; x < TILES; ++x) {
      float sc[8];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x4 d = init[x];
#pragma unroll
        for (int w = 0; w < D / 32; ++w) d = H::mfma(codes8<H>(kw[u][w]), q[x][w], d);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float t = row_step(kp[u][r]), o = row_offset(kp[u][r]);
          sc[4 * u + r] = __builtin_fmaf(d[r], t * a.factor, __builtin_fmaf(8.0f, t, o) * qc[x]);
        }
      }
      float vt[8], vo[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        vt[e] = row_step(vp[e >> 2][e & 3]);
        vo[e] = __builtin_fmaf(8.0f, vt[e], row_offset(vp[e >> 2][e & 3]));
      }
      if (masked) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int j = j0 + 16 * (e >> 2) + 4 * g + (e & 3);
          const bool sees = held && j <= pos[x] &&
                            (a.window == 0 || j > pos[x] - a.window || j < a.sinks);
          sc[e] = sees ? sc[e] : -__builtin_inff();
          // what a hidden row holds must not reach the sums, not even as 0 * NaN
          vt[e] = sees ? vt[e] : 0.0f;
          vo[e] = sees ? vo[e] : 0.0f;
        }
      }
      float top = sc[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top = fmaxf(top, sc[e]);
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
        const float p = __builtin_amdgcn_exp2f(sc[e] - s.mu[x]);
        s.l[x] += p;
        s.ob[x] = __builtin_fmaf(p, vo[e], s.ob[x]);
        fac[e] = p * vt[e];
      }
      u32x4 hi, lo;
      split8(fac, hi, lo);
      const bf16x8 fh = __builtin_bit_cast(bf16x8, hi), fl = __builtin_bit_cast(bf16x8, lo);
      const bf16x8 one = __builtin_bit_cast(bf16x8, ones);
      s.wsum[x] = Half<__bf16>::mfma(one, fh, s.wsum[x]);
      s.wsum[x] = Half<__bf16>::mfma(one, fl, s.wsum[x]);
#pragma unroll
      for (int d = 0; d < D / 16; ++d) {
        const bf16x8 v = codes8<Half<__bf16>>(vw[d >> 2][d & 3]);
        s.acc[x][d] = Half<__bf16>::mfma(v, fh, s.acc[x][d]);
        s.acc[x][d] = Half<__bf16>::mfma(v, fl, s.acc[x][d]);
      }
    }
  }
#pragma unroll
  for (int x = 0; x < TILES; ++x) {
    s.l[x] = sum_g(s.l[x]);
    s.ob[x] = sum_g(s.ob[x]);
  }
}

// Query rows row0 .. row0 + 15 of a sequence (row = token * ratio + head of the
// group) as operand columns; rows past the last repeat it.
template <typename T, int D>
__device__ __forceinline__ void load_rows(const AttnArgs& a, const Seq& s, int hk, int row,
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

// Few query rows: the four waves of a workgroup take every fourth block of its
// part of the sequence for the same 16 rows, and join their results in LDS;
// the parts of a split sequence are joined by the workgroup that ends last.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv_attention_split(AttnArgs a) {
  constexpr int PAD = D + 4;
  __shared__ __align__(16) float osum[4][16][PAD];
  __shared__ float ml[4][16][2];
  __shared__ int last;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int unit = blockIdx.x / a.splits, part = blockIdx.x % a.splits;
  const int hk = unit % a.c.kv_heads;
  const int rb = unit / a.c.kv_heads % a.row_blocks;
  const int b = unit / a.c.kv_heads / a.row_blocks;
  const Seq s = seq_of(a.c, b);
  const int rows = s.count * a.ratio, row0 = rb * 16;
  if (row0 >= rows) return;
  const int last_row = min(row0 + 15, rows - 1);
  const int p_lo = a.causal ? min(s.pos + row0 / a.ratio, s.length - 1) : s.length - 1;
  const int p_hi = a.causal ? min(s.pos + last_row / a.ratio, s.length - 1) : s.length - 1;
  const View view = view_of(a, p_lo, p_hi);
  // parts of `chunk` blocks; longer ones where the sequence is longer than planned
  const int chunk = max(a.chunk, (view.blocks + a.splits - 1) / a.splits);
  const int parts = max(1, (view.blocks + chunk - 1) / chunk);
  if (part >= parts) return;
  typename Half<T>::x8 q[1][D / 32];
  int pos[1];
  load_rows<T, D>(a, s, hk, row0 + n, q[0], pos[0]);
  State<D, 1> st;
  attend<T, D, 1>(a, view, b, hk, part * chunk + wave, min(view.blocks, (part + 1) * chunk), 4, q,
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
  float* dst = a.part + (int64_t)(unit * a.splits + part) * 16 * (D + 4);
  const int live = last_row - row0 + 1;
  for (int i = threadIdx.x; i < live * (D / 4); i += 256) {
    const int r = i / (D / 4), d = i % (D / 4) * 4;
    float m = ml[0][r][0];
#pragma unroll
    for (int w = 1; w < 4; ++w) m = fmaxf(m, ml[w][r][0]);
    const float mu = m == -__builtin_inff() ? 0.0f : m;
    float l = 0.0f;
    f32x4 o = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(ml[w][r][0] - mu);
      l += f * ml[w][r][1];
      o += f * *reinterpret_cast<const f32x4*>(&osum[w][r][d]);
    }
    if (parts > 1) {
      *reinterpret_cast<f32x4*>(dst + r * (D + 4) + d) = o;
      if (d == 0) {
        dst[r * (D + 4) + D] = m;
        dst[r * (D + 4) + D + 1] = l;
      }
    } else {
      const float f = l == 0.0f ? 0.0f : 1.0f / l;
      const int row = row0 + r;
      T* out = static_cast<T*>(a.out) + (int64_t)(s.row + row / a.ratio) * a.o_stride +
               (int64_t)(hk * a.ratio + row % a.ratio) * D + d;
#pragma unroll
      for (int e = 0; e < 4; ++e) out[e] = (T)(o[e] * f);
    }
  }
  if (parts == 1) return;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    last = atomicInc(a.count + unit, (uint32_t)(parts - 1)) == (uint32_t)(parts - 1);
    if (last) __threadfence();
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  const float* src = a.part + (int64_t)unit * a.splits * 16 * (D + 4);
  for (int i = threadIdx.x; i < live * (D / 4); i += 256) {
    const int r = i / (D / 4), d = i % (D / 4) * 4;
    float m = -__builtin_inff();
    for (int p = 0; p < parts; ++p) m = fmaxf(m, src[(p * 16 + r) * (D + 4) + D]);
    const float mu = m == -__builtin_inff() ? 0.0f : m;
    float l = 0.0f;
    f32x4 o = {0, 0, 0, 0};
    for (int p = 0; p < parts; ++p) {
      const float* at = src + (p * 16 + r) * (D + 4);
      const float f = __builtin_amdgcn_exp2f(at[D] - mu);
      l += f * at[D + 1];
      o += f * *reinterpret_cast<const f32x4*>(at + d);
    }
    const float f = l == 0.0f ? 0.0f : 1.0f / l;
    const int row = row0 + r;
    T* out = static_cast<T*>(a.out) + (int64_t)(s.row + row / a.ratio) * a.o_stride +
             (int64_t)(hk * a.ratio + row % a.ratio) * D + d;
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = (T)(o[e] * f);
  }
}

struct Plan {
  int32_t row_blocks, splits, chunk;
  int64_t units;
};

Plan plan_of(const ifq_kv_desc& d) {
  Plan p;
  const int64_t rows = (int64_t)d.max_q * (d.heads / d.kv_heads);
  p.row_blocks = (int32_t)((rows + 15) / 16);
  p.units = (int64_t)d.batch * d.kv_heads * p.row_blocks;
  p.splits = 1;
  p.chunk = INT32_MAX / 2;
  return p;
}

template <typename T>
hipError_t launch(const AttnArgs& a, int head_dim, int64_t groups, hipStream_t stream) {
  const dim3 grid((uint32_t)groups), block(256);
  if (head_dim == 64)
    hipLaunchKernelGGL((kv_attention_split<T, 64>), grid, block, 0, stream, a);
  else if (head_dim == 128)
    hipLaunchKernelGGL((kv_attention_split<T, 128>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((kv_attention_split<T, 256>), grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace

size_t kv_attention_workspace_bytes(const ifq_kv_desc& d) {
  const Plan p = plan_of(d);
  if (p.splits == 1) return 0;
  return kSplitCounterBytes + (size_t)p.units * p.splits * 16 * (d.head_dim + 4) * sizeof(float);
}

hipError_t launch_kv_attention(const ifq_kv_desc& d, const void* q, const KvArgs& c, void* out,
                               void* ws, hipStream_t stream) {
  const Plan p = plan_of(d);
  AttnArgs a;
  a.c = c;
  a.q = q;
  a.out = out;
  a.count = static_cast<uint32_t*>(ws);
  a.part = ws ? reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + kSplitCounterBytes) : nullptr;
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
  return d.type == IFQ_TYPE_BF16 ? launch<__bf16>(a, d.head_dim, p.units * p.splits, stream)
                                 : launch<_Float16>(a, d.head_dim, p.units * p.splits, stream);
}

}  // namespace ifq
