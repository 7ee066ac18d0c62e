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
//
// Rows of the softmax run with the largest score so far (State::raise) and all
// sums are fp32. A lane turns a code into an operand once for every 16 query
// columns; with few rows that work, not the products, stands beside the
// cache's bytes, with many it is shared through LDS.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "ifq_serve.h"

namespace ifq {
namespace {

constexpr double kSlots = 512;      // workgroups that run at once: two on a CU
constexpr double kPartSteps = 32;   // cost of a part and of joining it, in steps

struct AttnArgs {
  KvArgs c;
  const void* q;
  void* out;
  float* part;          // partial results of split sequences
  uint32_t* count;      // arrivals per unit of split work
  int64_t q_stride, o_stride;
  int32_t ratio;        // query heads per key/value head
  int32_t causal, window, sinks;
  int32_t sink_blocks;  // blocks of 32 positions that hold the sinks
  float factor;         // scale * log2(e)
  int32_t row_blocks;   // blocks of a sequence's ratio * max_q query rows
  FastDiv div_page;       // by the blocks of 32 tokens of a page
  int32_t splits, chunk;  // parts at most, and steps of a part at least
  // (sequence, row block, key/value head), the head fastest. A unit's parts are
  // `units` workgroups apart: the last parts, which only the longest sequences
  // have, would else fall to the same few XCDs (40 sequences of 100 to 5000
  // tokens in 4 parts: 33.6 us side by side, 20.2 so)
  int32_t units;
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

// What turns codes into 16 + c, kept in a scalar and a vector register: as
// constants they would be two literals, and the and and the or two
// instructions.
template <typename H>
struct Codes {
  uint32_t mask, base;
  __device__ __forceinline__ Codes() : mask(H::kMask), base(H::kBase) {
    asm("" : "+s"(mask));
    asm("" : "+v"(base));
  }
  // Eight codes of a word (nibble p + 4h: element 2p + h).
  __device__ __forceinline__ typename H::x8 operator()(uint32_t w) const {
    u32x4 r;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int s = 4 * p - H::kAt;
      r[p] = ((s < 0 ? w << -s : w >> s) & mask) | base;
    }
    return __builtin_bit_cast(typename H::x8, r);
  }
};

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
// the sinks, then those from the window's begin to the last position. p_lo and
// p_hi are the positions of the first and the last query, end the last position
// held: a sequence may be longer than its page table, and then the window may
// begin past it.
struct View {
  int32_t blocks, sink_blocks, first;   // first: block where the window begins
  __device__ __forceinline__ int block(int i) const {
    return i < sink_blocks ? i : i - sink_blocks + first;
  }
};

__device__ __forceinline__ View view_of(const AttnArgs& a, int p_lo, int p_hi, int end) {
  View v = {0, 0, 0};
  if (min(p_hi, end) < 0) return v;
  const int held = min(p_hi, end) / kCodeTokens + 1;       // blocks
  // queries before position 0 see nothing; without them no difference to a window
  // overflows, however wide it is
  const int lo = a.window > 0 ? max(max(p_lo, 0) - a.window + 1, 0) : 0;
  v.first = lo / kCodeTokens;
  if (a.window > 0) v.sink_blocks = min(a.sink_blocks, min(v.first, held));
  v.blocks = v.sink_blocks + max(held - v.first, 0);
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

// Running softmax and weighted sums of 16 query columns.
template <int D>
struct State {
  f32x4 acc[D / 16];   // sums of factors * (16 + c): dims 16 x + 4g + r of a column
  f32x4 wsum;          // sums of the factors, the same in every row
  float m, mu;         // largest score so far, and the same or 0 where there is none
  float l, ob;         // this lane's sums of p and of p * (o + 8 t)
  float qc;            // factor * sum(q)
  f32x4 init;          // -24 * sum(q)
  u32x4 ones;

  template <typename X8>
  __device__ __forceinline__ void begin(const X8 (&q)[D / 32], float factor) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += (float)q[i][e];
    sum = sum_g(sum);
    qc = sum * factor;
    init = f32x4{-24.0f * sum, -24.0f * sum, -24.0f * sum, -24.0f * sum};
    m = -__builtin_inff();
    mu = l = ob = 0.0f;
    wsum = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int d = 0; d < D / 16; ++d) acc[d] = f32x4{0, 0, 0, 0};
    ones = u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
    asm("" : "+v"(ones));        // in registers: not made anew for each use
  }

  // Raises the maximum for eight scores (as differences to mu).
  __device__ __forceinline__ void raise(float (&sc)[8]) {
    float top = sc[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) top = fmaxf(top, sc[e]);
    // the maximum is raised only where a score passes it by 8 (a factor of
    // 256 in p): sums keep their precision, and they are seldom rescaled
    const float none = -__builtin_inff();
    if (__ballot(top > (m == none ? none : 8.0f))) {
      const float most = fmaxf(m, max_g(top) + mu);
      const float mid = most == none ? 0.0f : most;
      const float f = __builtin_amdgcn_exp2f(m - mid), by = mid - mu;
#pragma unroll
      for (int e = 0; e < 8; ++e) sc[e] -= by;
      m = most;
      mu = mid;
      l *= f;
      ob *= f;
      wsum *= f;
#pragma unroll
      for (int d = 0; d < D / 16; ++d) acc[d] *= f;
    }
  }

  // Adds the scores' tokens, with values' steps vt and middles vm, to the sums
  // and leaves the factors p * vt as two bfloat16 each.
  __device__ __forceinline__ void take(const float (&sc)[8], const float (&vt)[8],
                                       const float (&vm)[8], u32x4& hi, u32x4& lo) {
    float fac[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float p = __builtin_amdgcn_exp2f(sc[e]);
      l += p;
      ob = __builtin_fmaf(p, vm[e], ob);
      fac[e] = p * vt[e];
    }
    split8(fac, hi, lo);
    const bf16x8 one = __builtin_bit_cast(bf16x8, ones);
    wsum = Half<__bf16>::mfma(one, __builtin_bit_cast(bf16x8, hi), wsum);
    wsum = Half<__bf16>::mfma(one, __builtin_bit_cast(bf16x8, lo), wsum);
  }
};

// Whether the query at position pos sees position j; end: the last position held.
__device__ __forceinline__ bool sees(const AttnArgs& a, int pos, int end, int j) {
  return j <= min(pos, end) && (a.window == 0 || j > max(pos, 0) - a.window || j < a.sinks);
}

// A block's place: its page's head (page 0 where the cache has no such page,
// whose tokens are then hidden) and its first token there.
struct Place {
  const uint8_t* head;
  int32_t tp, j0;             // j0: position of the first token
  bool held;
};

// One sequence's pages of one head.
struct Pages {
  const int32_t* ids;
  const uint8_t* cache;       // page 0's head
  int64_t page_bytes;
  FastDiv div;                // by the blocks of a page
  int32_t per_page, num_pages;

  __device__ __forceinline__ Pages(const AttnArgs& a, int b, int hk)
      : ids(a.c.pages + (int64_t)b * a.c.max_pages),
        cache(a.c.cache + hk * a.c.head_bytes),
        page_bytes(a.c.page_bytes),
        div(a.div_page),
        per_page(a.c.page_tokens / kCodeTokens),
        num_pages(a.c.num_pages) {}
  __device__ __forceinline__ int page(int blk) const {
    return (int)((__umulhi((uint32_t)blk, div.mul) + (uint32_t)blk) >> div.shift);
  }
  __device__ __forceinline__ int id(int blk) const { return ids[page(blk)]; }
  __device__ __forceinline__ Place place(int blk, int id, bool there) const {
    Place p;
    const bool has = id >= 0 && id < num_pages;
    p.head = cache + (has ? id : 0) * page_bytes;
    p.tp = (blk - page(blk) * per_page) * kCodeTokens;
    p.j0 = blk * kCodeTokens;
    p.held = has && there;
    return p;
  }
};

// One of the N places, chosen by a number that is no constant: field by field
// and by value, so that no array of places ends up in memory.
template <typename V>
__device__ __forceinline__ V choose(bool c, V a, V b) { return c ? a : b; }

template <int N>
__device__ __forceinline__ Place pick(const Place (&p)[N], int k) {
  Place r = p[0];
#pragma unroll
  for (int i = 1; i < N; ++i) {
    r.head = choose(k == i, p[i].head, r.head);
    r.tp = choose(k == i, p[i].tp, r.tp);
    r.j0 = choose(k == i, p[i].j0, r.j0);
    r.held = choose(k == i, p[i].held, r.held);
  }
  return r;
}

// Runs steps i = begin, begin + step .. below end of the view over 16 query
// columns, U blocks (U * i ..) at a step: column n stands for query row
// n % (16 / U) and sees only block n / (16 / U) of the U, so that with few
// rows all columns take part in the softmax. pos: the position of this lane's
// query; p_lo, p_hi and last_held: as for view_of. A step's loads are issued a step
// ahead: the keys' after their last use, the values' likewise.
template <typename T, int D, int U>
__device__ __forceinline__ void attend(const AttnArgs& a, const View& view, int b, int hk,
                                       int begin, int end, int step,
                                       const typename Half<T>::x8 (&q)[D / 32], int pos,
                                       int p_lo, int p_hi, int last_held, State<D>& s) {
  typedef Half<T> H;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int mine = n / (16 / U);          // the block of the U that this column sees
  const KvArgs& c = a.c;
  s.begin(q, a.factor);
  if (begin >= end) return;
  const Codes<H> kcodes;
  const Codes<Half<__bf16>> vcodes;
  const Pages pages(a, b, hk);
  const int last = view.blocks - 1;

  uint32_t kw[U][2][D / 32];
  u32x4 vw[U][D / 64], kp[2], vp[2];
  Place now[U], next[U];
  auto find = [&](int i, Place (&p)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int blk = view.block(min(U * i + u, last));
      p[u] = pages.place(blk, pages.id(blk), U * i + u <= last);
    }
  };
  auto load_keys = [&](const Place (&p)[U]) {
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
  auto load_words = [&](const Place (&p)[U], int part, u32x4 (&to)[2]) {
    const Place at = pick(p, mine);
    const uint8_t* src = at.head + c.page_tokens * (D + 4 * part) + 4 * (at.tp + 4 * g);
    to[0] = *reinterpret_cast<const u32x4*>(src);
    to[1] = *reinterpret_cast<const u32x4*>(src + 64);
  };
  auto load_values = [&](const Place (&p)[U]) {
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
    find(min(i + step, end - 1), next);
    const Place own = pick(now, mine);
    bool masked = false;
#pragma unroll
    for (int u = 0; u < U; ++u)
      masked |= !now[u].held || now[u].j0 + kCodeTokens - 1 > min(p_lo, last_held) ||
                (a.window > 0 && now[u].j0 <= p_hi - a.window);
    float sc[8];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x4 d;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        f32x4 e = s.init;
#pragma unroll
        for (int w = 0; w < D / 32; ++w) e = H::mfma(kcodes(kw[u][t][w]), q[w], e);
#pragma unroll
        for (int r = 0; r < 4; ++r) d[r] = u == 0 || mine == u ? e[r] : d[r];
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float st = row_step(kp[t][r]), mid = __builtin_fmaf(8.0f, st, row_offset(kp[t][r]));
        sc[4 * t + r] =
            __builtin_fmaf(d[r], st * a.factor, __builtin_fmaf(mid, s.qc, -s.mu));
      }
    }
    load_keys(next);
    load_words(next, 0, kp);
    float vt[8], vm[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      vt[e] = row_step(vp[e >> 2][e & 3]);
      vm[e] = __builtin_fmaf(8.0f, vt[e], row_offset(vp[e >> 2][e & 3]));
    }
    if (masked) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool ok =
            own.held && sees(a, pos, last_held, own.j0 + 16 * (e >> 2) + 4 * g + (e & 3));
        sc[e] = ok ? sc[e] : -__builtin_inff();
        // what a hidden row holds must not reach the sums, not even as 0 * NaN
        vt[e] = ok ? vt[e] : 0.0f;
        vm[e] = ok ? vm[e] : 0.0f;
      }
    }
    u32x4 hi, lo;
    s.raise(sc);
    s.take(sc, vt, vm, hi, lo);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // block u counts for its own columns alone
      const uint32_t keep = U == 1 || mine == u ? 0xFFFFFFFFu : 0u;
      const bf16x8 fh = __builtin_bit_cast(bf16x8, hi & keep);
      const bf16x8 fl = __builtin_bit_cast(bf16x8, lo & keep);
#pragma unroll
      for (int d = 0; d < D / 16; ++d) {
        const bf16x8 v = vcodes(vw[u][d >> 2][d & 3]);
        s.acc[d] = Half<__bf16>::mfma(v, fh, s.acc[d]);
        s.acc[d] = Half<__bf16>::mfma(v, fl, s.acc[d]);
      }
    }
    load_values(next);
    load_words(next, 1, vp);
#pragma unroll
    for (int u = 0; u < U; ++u) now[u] = next[u];
  }
  s.l = sum_g(s.l);
  s.ob = sum_g(s.ob);
}

// Position of query row `row` of a sequence (row = token * ratio + head of the
// group): where no mask is causal, the last.
__device__ __forceinline__ int position_of(const AttnArgs& a, const Seq& s, int row) {
  return a.causal ? s.pos + row / a.ratio : s.length - 1;
}

// A query row as this lane's operand column, and its position; rows past the
// last repeat it.
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
  pos = position_of(a, s, row);
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

__device__ __forceinline__ void put_sums(float* row, int d, f32x4 o) {
  put_pair(row + d, o[0], o[1]);
  put_pair(row + d + 2, o[2], o[3]);
}

// A row's result over some of its tokens: the largest score, the sum of p and
// four of the sums of p * v, relative to that score.
struct Result {
  float m, l;
  f32x4 o;
  __device__ __forceinline__ void add(float m2, float l2, f32x4 o2) {
    const float top = fmaxf(m, m2), mu = top == -__builtin_inff() ? 0.0f : top;
    const float f = __builtin_amdgcn_exp2f(m - mu), f2 = __builtin_amdgcn_exp2f(m2 - mu);
    l = f * l + f2 * l2;
    o = f * o + f2 * o2;
    m = top;
  }
};

// Joins the parts of a unit's rows in the workgroup that counts itself last.
// Called by all of a workgroup's threads after they have written its part
// ([rows][D + 4]: sums, then m and l). A thread takes four sums of a row at a
// time, and has 8 or 16 parts' loads in flight: eight parts where there are
// threads to spare, which then take a share of the parts each, else four parts
// of four rows (of 128 rows of 128 dims in two parts each in turn took 12 us).
// The order of all additions is the same in every call.
template <typename T, int D, int ROWS>
__device__ __forceinline__ void join_parts(const AttnArgs& a, const Seq& s, int unit, int hk,
                                           int row0, int live, int parts) {
  constexpr int LD = D + 4, AHEAD = 8, ITEMS = 4, EACH = 4;
  __shared__ int last;
  __shared__ Result share[256];
  if (!comes_last(a.count + unit, parts, &last)) return;
  const float* src = a.part + (int64_t)unit * a.splits * ROWS * LD;
  const int items = live * (D / 4);
  const Result none = {-__builtin_inff(), 0.0f, {0, 0, 0, 0}};
  auto store = [&](int r, int d, const Result& all) {
    store4(out_row<T, D>(a, s, hk, row0 + r) + d, all.o * (all.l == 0.0f ? 0.0f : 1.0f / all.l));
  };
  if (items > 256) {
    for (int i0 = threadIdx.x; i0 < items; i0 += 256 * ITEMS) {
      Result all[ITEMS];
      int at[ITEMS], dim[ITEMS];
#pragma unroll
      for (int u = 0; u < ITEMS; ++u) {
        const int i = min(i0 + 256 * u, items - 1);
        at[u] = i / (D / 4) * LD;
        dim[u] = i % (D / 4) * 4;
        all[u] = none;
      }
      for (int p0 = 0; p0 < parts; p0 += EACH) {
        f32x2 ml[ITEMS][EACH], x[ITEMS][EACH], y[ITEMS][EACH];
#pragma unroll
        for (int k = 0; k < EACH; ++k)
#pragma unroll
          for (int u = 0; u < ITEMS; ++u) {
            const float* row = src + (int64_t)min(p0 + k, parts - 1) * ROWS * LD + at[u];
            ml[u][k] = get_pair(row + D);
            x[u][k] = get_pair(row + dim[u]);
            y[u][k] = get_pair(row + dim[u] + 2);
          }
#pragma unroll
        for (int k = 0; k < EACH; ++k)
          if (p0 + k < parts)
#pragma unroll
            for (int u = 0; u < ITEMS; ++u)
              all[u].add(ml[u][k][0], ml[u][k][1],
                         f32x4{x[u][k][0], x[u][k][1], y[u][k][0], y[u][k][1]});
      }
#pragma unroll
      for (int u = 0; u < ITEMS; ++u)
        if (i0 + 256 * u < items) store(at[u] / LD, dim[u], all[u]);
    }
    return;
  }
  const int shares = 256 / items;
  const int i = (int)threadIdx.x % items, mine = (int)threadIdx.x / items;
  const bool on = mine < shares;
  const int r = i / (D / 4), d = i % (D / 4) * 4;
  Result all = none;
  for (int p0 = on ? mine : parts; p0 < parts; p0 += AHEAD * shares) {
    f32x2 ml[AHEAD], x[AHEAD], y[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const float* row = src + (int64_t)(min(p0 + k * shares, parts - 1) * ROWS + r) * LD;
      ml[k] = get_pair(row + D);
      x[k] = get_pair(row + d);
      y[k] = get_pair(row + d + 2);
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (p0 + k * shares < parts)
        all.add(ml[k][0], ml[k][1], f32x4{x[k][0], x[k][1], y[k][0], y[k][1]});
  }
  share[threadIdx.x] = all;
  __syncthreads();
  if (mine == 0) {
    for (int k = 1; k < shares; ++k) {
      const Result& more = share[threadIdx.x + k * items];
      all.add(more.m, more.l, more.o);
    }
    store(r, d, all);
  }
}

// Up to 16 / U query rows: the four waves of a workgroup take every fourth
// step of its part of the sequence for the same rows, and join their results
// in LDS. Bound by memory where all CUs have work: 5 sequences of up to 120001
// tokens, 8 heads of 128, 78.5 us, 4.8 TB/s (vector instructions take 40 % of the
// time, the products 17 %); 5 of up to 60000, 4 heads of 256, 62 us, 3.0 TB/s, with
// one workgroup on a CU. A step of a wave alone on its SIMD takes 2.4 us for 128
// tokens of 128 dims, which is what short sequences see: one of 1111 tokens takes
// 8.8 to 9.8 us on the GPU, where the shortest kernel takes 2: the step, then the
// join of three parts through memory. With all U blocks in one step of 16
// columns, rows in use grow from 16 / U to 16 in the softmax; a block's products
// still run over all 16 columns, at a quarter of their use for U = 4.
template <typename T, int D, int U>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void kv_attention_few(AttnArgs a) {
  constexpr int ROWS = 16 / U, LD = D + 4;
  __shared__ __align__(16) float osum[4][16][LD];
  __shared__ float ml[4][16][2];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int unit = blockIdx.x % a.units, part = blockIdx.x / a.units;
  const int hk = unit % a.c.kv_heads;
  const int rb = unit / a.c.kv_heads % a.row_blocks;
  const int b = unit / a.c.kv_heads / a.row_blocks;
  const Seq s = seq_of(a.c, b);
  const int rows = s.count * a.ratio, row0 = rb * ROWS;
  if (row0 >= rows) return;
  const int live = min(ROWS, rows - row0);
  const int p_lo = position_of(a, s, row0), p_hi = position_of(a, s, row0 + live - 1);
  const View view = view_of(a, p_lo, p_hi, s.length - 1);
  // parts of `chunk` steps; longer ones where the sequence is longer than planned
  const int steps = (view.blocks + U - 1) / U;
  const int chunk = max(a.chunk, (steps + a.splits - 1) / a.splits);
  const int parts = max(1, (steps + chunk - 1) / chunk);
  if (part >= parts) return;
  typename Half<T>::x8 q[D / 32];
  int pos;
  load_row<T, D>(a, s, hk, row0 + n % ROWS, q, pos);
  State<D> st;
  attend<T, D, U>(a, view, b, hk, part * chunk + wave, min(steps, (part + 1) * chunk), 4, q, pos,
                  p_lo, p_hi, s.length - 1, st);
  const float corr = st.ob - 24.0f * st.wsum[0];
#pragma unroll
  for (int d = 0; d < D / 16; ++d)
    *reinterpret_cast<f32x4*>(&osum[wave][n][16 * d + 4 * g]) = st.acc[d] + corr;
  if (g == 0) {
    ml[wave][n][0] = st.m;
    ml[wave][n][1] = st.l;
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

// The blocks of 32 tokens that many query rows take at a time, out of the
// 4-bit codes: matrix operands of 16 bytes per lane, and each row's step and
// middle, the keys' with the scores' factor.
template <int D>
struct Stage {
  static constexpr int TOKENS = D == 64 ? 128 : 64, BLOCKS = TOKENS / kCodeTokens;
  u32x4 k[TOKENS / 16][D / 32][64];
  u32x4 v[BLOCKS][D / 16][64];
  float kt[TOKENS], km[TOKENS], vt[TOKENS], vm[TOKENS];
};

// Many query rows: each wave has TILES x 16 of its own, and the workgroup
// runs through all that its rows see of its part. The codes become operands
// once for the workgroup, a quarter by each wave, in LDS, two stages in turn:
// while one is computed on, the next one's codes are on their way into
// registers. The last rows, which see most, come first.
// Bound by vector instructions beside the products: prompts of 900 to 2048
// tokens over up to 6100, 32 heads of 128, 412 us = 620 TFLOP/s of 4 D a pair
// (472 at first in a row of calls, as the clocks rise), with vector instructions at
// 56 % and products at 40 % of the cycles. 32 heads of 64: 332 us, 384 TFLOP/s; 16
// of 256, of which registers and LDS hold one query tile a wave and one workgroup a
// CU: 824 us, 310 TFLOP/s. The two halves of p t make 3 products' work of 2 (it buys
// 16 bits of p t and fp32's range). With the codes expanded by each wave for
// itself, without LDS, the first prompts took 772 us.
template <typename T, int D>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void kv_attention_many(AttnArgs a) {
  typedef Half<T> H;
  typedef Half<__bf16> B;
  typedef Stage<D> St;
  constexpr int TILES = D == 256 ? 1 : 2;
  constexpr int WROWS = 16 * TILES, ROWS = 4 * WROWS, LD = D + 4, NB = St::BLOCKS;
  constexpr int KPW = St::TOKENS / 64, VPW = NB * (D / 64) / 4;  // key tiles, value chunks per wave
  __shared__ __align__(16) St lds[2];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int unit = blockIdx.x % a.units, part = blockIdx.x / a.units;
  const KvArgs& c = a.c;
  const int hk = unit % c.kv_heads;
  const int rb = a.row_blocks - 1 - unit / c.kv_heads % a.row_blocks;
  const int b = unit / c.kv_heads / a.row_blocks;
  const Seq s = seq_of(c, b);
  const int rows = s.count * a.ratio;
  if (rb * ROWS >= rows) return;
  const int last_held = s.length - 1;
  const int live = min(ROWS, rows - rb * ROWS);
  const View view = view_of(a, position_of(a, s, rb * ROWS),
                            position_of(a, s, rb * ROWS + live - 1), last_held);
  const int steps = (view.blocks + NB - 1) / NB;
  const int chunk = max(a.chunk, (steps + a.splits - 1) / a.splits);
  const int parts = max(1, (steps + chunk - 1) / chunk);
  if (part >= parts) return;
  const int begin = part * chunk, end = min(steps, begin + chunk);
  const int row0 = rb * ROWS + wave * WROWS;
  const int own = min(WROWS, rows - row0);         // may be below 1: the wave only helps
  const int p_lo = own > 0 ? position_of(a, s, row0) : 0;
  const int p_hi = own > 0 ? position_of(a, s, row0 + own - 1) : -1;

  typename H::x8 q[TILES][D / 32];
  int pos[TILES];
  State<D> st[TILES];
#pragma unroll
  for (int x = 0; x < TILES; ++x) {
    load_row<T, D>(a, s, hk, row0 + 16 * x + n, q[x], pos[x]);
    st[x].begin(q[x], a.factor);
  }

  const Pages pages(a, b, hk);
  const int last = view.blocks - 1;
  auto block = [&](int step, int k) { return view.block(min(step * NB + k, last)); };
  const Codes<H> kcodes;
  const Codes<B> vcodes;
  uint32_t kw[KPW][D / 32], kprm, vprm;
  u32x4 vw[VPW];
  auto load = [&](const Place (&p)[NB]) {
#pragma unroll
    for (int x = 0; x < KPW; ++x) {
      const int t = wave * KPW + x;                // tile of 16 keys
      const Place at = pick(p, t >> 1);
      const uint32_t* src = reinterpret_cast<const uint32_t*>(
          at.head + (at.tp + 16 * (t & 1) + n) * (D / 2) + g * (D / 8));
#pragma unroll
      for (int w = 0; w < D / 32; ++w) kw[x][w] = src[w];
    }
#pragma unroll
    for (int x = 0; x < VPW; ++x) {
      const int t = wave * VPW + x;                // chunk of 32 values x 64 dims
      const Place at = pick(p, t / (D / 64));
      vw[x] = *reinterpret_cast<const u32x4*>(at.head + (c.page_tokens + at.tp) * (D / 2) +
                                              t % (D / 64) * 1024 + lane * 16);
    }
    // a word of a key and of a value for each of the first TOKENS threads
    const Place at = pick(p, (int)threadIdx.x / kCodeTokens % NB);
    const uint32_t* prm =
        reinterpret_cast<const uint32_t*>(at.head + c.page_tokens * D) + at.tp + (lane & 31);
    // what no sequence wrote may be anything: it counts as 0
    const bool there = at.held && at.j0 + (lane & 31) < s.length;
    kprm = there ? prm[0] : 0u;
    vprm = there ? prm[c.page_tokens] : 0u;
  };
  auto stage = [&](St& to) {
#pragma unroll
    for (int x = 0; x < KPW; ++x)
#pragma unroll
      for (int w = 0; w < D / 32; ++w)
        to.k[wave * KPW + x][w][lane] = __builtin_bit_cast(u32x4, kcodes(kw[x][w]));
#pragma unroll
    for (int x = 0; x < VPW; ++x) {
      const int t = wave * VPW + x;
#pragma unroll
      for (int d = 0; d < 4; ++d)
        to.v[t / (D / 64)][t % (D / 64) * 4 + d][lane] =
            __builtin_bit_cast(u32x4, vcodes(vw[x][d]));
    }
    if (threadIdx.x < St::TOKENS) {
      const float t = row_step(kprm), u = row_step(vprm);
      const float km = __builtin_fmaf(8.0f, t, row_offset(kprm));
      const float vm = __builtin_fmaf(8.0f, u, row_offset(vprm));
      // a value that is no number shows in its key's score instead, which a
      // mask hides where a factor of 0 would not
      const bool fine = vm - vm == 0.0f;
      to.kt[threadIdx.x] = t * a.factor;
      to.km[threadIdx.x] = fine ? km : __builtin_nanf("");
      to.vt[threadIdx.x] = fine ? u : 0.0f;
      to.vm[threadIdx.x] = fine ? vm : 0.0f;
    }
  };

  if (begin < end) {
    Place now[NB], next[NB];
    int id[NB];
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      const int blk = block(begin, k);
      now[k] = pages.place(blk, pages.id(blk), begin * NB + k <= last);
      id[k] = pages.id(block(min(begin + 1, end - 1), k));
    }
    load(now);
    stage(lds[begin & 1]);
    __syncthreads();
    for (int i = begin; i < end; ++i) {
      const bool more = i + 1 < end;
      if (more) {
#pragma unroll
        for (int k = 0; k < NB; ++k) {
          next[k] = pages.place(block(i + 1, k), id[k], (i + 1) * NB + k <= last);
          id[k] = pages.id(block(min(i + 2, end - 1), k));
        }
        load(next);
      }
      const St& from = lds[i & 1];
#pragma unroll
      for (int k = 0; k < NB; ++k) {
        const int j0 = now[k].j0;
        // blocks that none of the wave's rows sees
        if (!now[k].held || j0 > min(p_hi, last_held) ||
            (a.window > 0 && j0 + kCodeTokens - 1 <= max(p_lo, 0) - a.window && j0 >= a.sinks))
          continue;
        const bool masked = j0 + kCodeTokens - 1 > min(p_lo, last_held) ||
                            (a.window > 0 && j0 <= p_hi - a.window);
        float sc[TILES][8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          f32x4 d[TILES];
#pragma unroll
          for (int x = 0; x < TILES; ++x) d[x] = st[x].init;
#pragma unroll
          for (int w = 0; w < D / 32; ++w) {
            const typename H::x8 kk =
                __builtin_bit_cast(typename H::x8, from.k[2 * k + t][w][lane]);
#pragma unroll
            for (int x = 0; x < TILES; ++x) d[x] = H::mfma(kk, q[x][w], d[x]);
          }
          const int at = kCodeTokens * k + 16 * t + 4 * g;
          const f32x4 kt = *reinterpret_cast<const f32x4*>(&from.kt[at]);
          const f32x4 km = *reinterpret_cast<const f32x4*>(&from.km[at]);
#pragma unroll
          for (int x = 0; x < TILES; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              sc[x][4 * t + r] =
                  __builtin_fmaf(d[x][r], kt[r], __builtin_fmaf(km[r], st[x].qc, -st[x].mu));
        }
        if (masked) {
#pragma unroll
          for (int x = 0; x < TILES; ++x)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (!sees(a, pos[x], last_held, j0 + 16 * (e >> 2) + 4 * g + (e & 3)))
                sc[x][e] = -__builtin_inff();
        }
#pragma unroll
        for (int x = 0; x < TILES; ++x) st[x].raise(sc[x]);
        // no branch from here on, so that a tile's products run beside the next
        // tile's softmax
#pragma unroll
        for (int x = 0; x < TILES; ++x) {
          float vt[8], vm[8];
#pragma unroll
          for (int e = 0; e < 8; e += 4) {
            const int at = kCodeTokens * k + 4 * e + 4 * g;
            const f32x4 t = *reinterpret_cast<const f32x4*>(&from.vt[at]);
            const f32x4 o = *reinterpret_cast<const f32x4*>(&from.vm[at]);
#pragma unroll
            for (int r = 0; r < 4; ++r) vt[e + r] = t[r], vm[e + r] = o[r];
          }
          u32x4 hi, lo;
          st[x].take(sc[x], vt, vm, hi, lo);
#pragma unroll
          for (int d = 0; d < D / 16; ++d) {
            const bf16x8 v = __builtin_bit_cast(bf16x8, from.v[k][d][lane]);
            st[x].acc[d] = B::mfma(v, __builtin_bit_cast(bf16x8, hi), st[x].acc[d]);
            st[x].acc[d] = B::mfma(v, __builtin_bit_cast(bf16x8, lo), st[x].acc[d]);
          }
        }
      }
      if (more) {
        stage(lds[(i + 1) & 1]);
#pragma unroll
        for (int k = 0; k < NB; ++k) now[k] = next[k];
      }
      __syncthreads();
    }
  }
  float* dst = parts > 1 ? a.part + ((int64_t)(unit * a.splits + part) * ROWS +
                                     wave * WROWS) * LD : nullptr;
#pragma unroll
  for (int x = 0; x < TILES; ++x) {
    const int r = 16 * x + n;
    const float sum = sum_g(st[x].l), corr = sum_g(st[x].ob) - 24.0f * st[x].wsum[0];
    if (r >= own) continue;
    if (parts > 1) {
#pragma unroll
      for (int d = 0; d < D / 16; ++d)
        put_sums(dst + r * LD, 16 * d + 4 * g, st[x].acc[d] + corr);
      if (g == 0) put_pair(dst + r * LD + D, st[x].m, sum);
    } else {
      const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
      T* out = out_row<T, D>(a, s, hk, row0 + r) + 4 * g;
#pragma unroll
      for (int d = 0; d < D / 16; ++d) store4(out + 16 * d, (st[x].acc[d] + corr) * f);
    }
  }
  if (parts > 1) join_parts<T, D, ROWS>(a, s, unit, hk, rb * ROWS, live, parts);
}

// Blocks of 32 tokens that n tokens fill.
int64_t code_blocks(int64_t n) { return (n + kCodeTokens - 1) / kCodeTokens; }

// Which kernel, and how its work is split: by the longest of the sequences, for all
// of them. A prompt among single tokens takes these along as rows of the kernel for
// many (512 tokens beside 31 single ones over 32000: 3000 us; as two calls 26 and 202).
struct Plan {
  int32_t few;            // blocks of a step for few rows (U), 0: many rows
  int32_t row_blocks, splits, chunk;
  int64_t units;
  int32_t rows;           // per unit
};

Plan plan_of(const ifq_kv_desc& d) {
  Plan p;
  const int64_t rows = (int64_t)d.max_q * (d.heads / d.kv_heads);
  p.few = rows <= 4 && d.head_dim < 256 ? 4 : rows <= 8 ? 2 : rows <= 16 ? 1 : 0;
  p.rows = p.few ? 16 / p.few : d.head_dim == 256 ? 64 : 128;
  p.row_blocks = (int32_t)((rows + p.rows - 1) / p.rows);
  p.units = (int64_t)d.batch * d.kv_heads * p.row_blocks;
  // blocks that a unit may see, and steps of them
  int64_t blocks = code_blocks(d.max_kv) + 1;
  if (d.window > 0) {
    const int64_t seen = ((int64_t)d.window + d.max_q + kCodeTokens) / kCodeTokens +
                         code_blocks(d.sinks) + 1;
    blocks = std::min(blocks, seen);
  }
  const int64_t at_once = p.few ? p.few : d.head_dim == 64 ? 4 : 2;
  const int64_t steps = (blocks + at_once - 1) / at_once;
  int64_t parts = 1;
  if (p.few) {
    // With units * steps of work in parts of c steps over kSlots places, the
    // parts' own cost (kPartSteps steps' time each) and the last part's length add
    // up to units * steps * kPartSteps / (c * kSlots) + c, least at the root.
    const double c = std::sqrt((double)p.units * (double)steps * kPartSteps / kSlots);
    // At least a workgroup on each CU, as long as its waves have 128 x 128 values
    // each, since parts beside one another cost little more than one (16 sequences
    // of 1000 to 2100 tokens, 128 units: 16.6 us whole, 14.4 in two; one of 8000, 8
    // units: 11.8 in 8, 10.4 in 16; but one of 5000 with 64 dims 8.7 in 10, 9.6 in
    // 20). From 32 on joining them takes what they save (8 units of 64000 tokens:
    // 21.8 us in 32, 24.1 in 64).
    const int64_t worth = (steps * p.few * d.head_dim / 512 + 3) / 4;
    parts = std::max<int64_t>({1, (int64_t)((double)steps / c + 0.5),
                               std::min<int64_t>({(int64_t)kSlots / 2 / p.units, worth, 32})});
  } else {
    // us, as measured: a step of a workgroup alone on its CU or beside another that
    // has less to do, and joining parts of 128 rows of 128 dims. 300 queries of 20
    // heads of 64 over 4000 tokens: 128 us whole, 57 in 3, 42 in 8; 1000 over 2000, 8
    // heads of 64, 3 sequences: 68 whole, 48 in 3; 500 of 32 heads of 128 over 500:
    // 25 whole, 33 in two.
    const double step = d.head_dim == 64 ? 3.8 : d.head_dim == 128 ? 2.25 : 2.8;
    const double join = (double)std::min<int64_t>(rows, p.rows) * d.head_dim / (128 * 128);
    double least = 0.0;
    for (int64_t n = 1; n <= std::min<int64_t>(steps, 32); ++n) {
      const double groups = (double)(p.units * n) / 256;     // of a CU
      const double turns = groups <= 1 ? 1.0 : 0.75 * std::max(groups, 2.0);
      const double time = (double)((steps + n - 1) / n) * step * turns +
                          (n > 1 ? join * (11.0 + 2.0 * (double)n) : 0.0);
      if (n == 1 || time < least) least = time, parts = n;
    }
  }
  int64_t chunk = (steps + parts - 1) / parts;
  if (p.few) chunk = (chunk + 3) / 4 * 4;      // the four waves take a step each
  p.chunk = (int32_t)chunk;
  p.splits = (int32_t)((steps + chunk - 1) / chunk);
  // one arrival counter for each unit
  if (p.units * (int64_t)sizeof(uint32_t) > kSplitCounterBytes) p.splits = 1;
  return p;
}

template <typename T, int D>
hipError_t launch(const AttnArgs& a, const Plan& p, hipStream_t stream) {
  const dim3 grid((uint32_t)(p.units * p.splits)), block(256);
  if (p.few == 4) {
    if constexpr (D < 256)
      hipLaunchKernelGGL((kv_attention_few<T, D, 4>), grid, block, 0, stream, a);
  } else if (p.few == 2) {
    hipLaunchKernelGGL((kv_attention_few<T, D, 2>), grid, block, 0, stream, a);
  } else if (p.few == 1) {
    hipLaunchKernelGGL((kv_attention_few<T, D, 1>), grid, block, 0, stream, a);
  } else {
    hipLaunchKernelGGL((kv_attention_many<T, D>), grid, block, 0, stream, a);
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

const char* kv_attention_kernel_name(const ifq_kv_desc& d) {
  static const char* const names[3][4] = {
      {"kv_attention_many<64>", "kv_attention_few<64, 1>", "kv_attention_few<64, 2>",
       "kv_attention_few<64, 4>"},
      {"kv_attention_many<128>", "kv_attention_few<128, 1>", "kv_attention_few<128, 2>",
       "kv_attention_few<128, 4>"},
      {"kv_attention_many<256>", "kv_attention_few<256, 1>", "kv_attention_few<256, 2>", ""}};
  const Plan p = plan_of(d);
  return names[d.head_dim == 64 ? 0 : d.head_dim == 128 ? 1 : 2][p.few == 4 ? 3 : p.few];
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
  a.sink_blocks = (int32_t)code_blocks(d.sinks);
  a.factor = d.scale * 1.4426950408889634f;
  a.row_blocks = p.row_blocks;
  a.div_page = make_fastdiv((uint32_t)(d.page_tokens / kCodeTokens));
  a.units = (int32_t)p.units;
  a.splits = p.splits;
  a.chunk = p.chunk;
  if (p.units * p.splits > kMaxGroups) return hipErrorInvalidConfiguration;
  return d.type == IFQ_TYPE_BF16 ? launch<__bf16>(a, p, d.head_dim, stream)
                                 : launch<_Float16>(a, p, d.head_dim, stream);
}

}  // namespace ifq
