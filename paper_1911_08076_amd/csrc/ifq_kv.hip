// Append to, and read from, a paged cache of keys and values in 4-bit codes
// (its format: include/ifq.h, ifq_kv_desc).
//
// A value's code shares its word with those of seven other tokens, so the
// unit of writing is a block of 32 tokens of one head, which one workgroup
// owns: it codes the rows of the block's new tokens, gathers the values'
// codes in LDS and writes every word that holds a new token, with the old
// codes of the other tokens where not all eight are new.
//
// All is read and written once. 7 prompts of 129 to 3001 tokens, 16 heads of 64,
// take 27.5 us, 3.5 TB/s: vector instructions take 64 % of the cycles (the
// rotation, a division a value and the packing), and each workgroup goes
// through the chain offsets - page - row - code - word once. One token for each
// of 64 sequences takes 5.9 us, that chain alone.
#include <hip/hip_runtime.h>

#include "ifq_serve.h"

namespace ifq {
namespace {

struct AppendArgs {
  KvArgs c;
  const void* q;
  const void* k;
  const void* v;
  void* q_out;
  const float* cosines;
  const float* sines;
  int64_t q_stride, k_stride, v_stride;
  int32_t rot_dim, adjacent, rot_len;
  int32_t blocks;      // blocks of 32 tokens that max_q tokens may touch
  int32_t kv_groups;   // workgroups for keys and values; the others turn queries
};

template <typename T>
using vec8 = T __attribute__((ext_vector_type(8)));

template <typename T>
__device__ __forceinline__ void load8(const T* p, float* x) {
  const vec8<T> a = *reinterpret_cast<const vec8<T>*>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)a[i];
}

template <typename T>
__device__ __forceinline__ void store8(T* p, const float* x) {
  vec8<T> a;
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = (T)x[i];
  *reinterpret_cast<vec8<T>*>(p) = a;
}

// The new tokens of sequence b: their first row, how many, and the position
// of the first.
struct Span {
  int32_t row, count, pos;
};

__device__ __forceinline__ Span span_of(const KvArgs& c, int b) {
  const int lo = min(max(c.offsets[b], 0), c.total_q);
  const int hi = min(max(c.offsets[b + 1], lo), c.total_q);
  Span s;
  s.row = lo;
  s.count = min(hi - lo, c.max_q);
  s.pos = (int32_t)max((int64_t)c.lengths[b] - (hi - lo), (int64_t)INT32_MIN / 2);
  return s;
}

// Where the block of 32 positions from p (a multiple of 32 inside the table)
// of sequence b and head hk lies: its page's head, or NULL.
__device__ __forceinline__ uint8_t* head_of(const KvArgs& c, int b, int hk, int p) {
  const int id = c.pages[(int64_t)b * c.max_pages + p / c.page_tokens];
  if (id < 0 || id >= c.num_pages) return nullptr;
  return c.cache + id * c.page_bytes + hk * c.head_bytes;
}

// Dims 8c .. 8c+7 of the row at src, rotated by position pos: the pair of
// dim i (i < rot/2) is i + rot/2, or the neighbour.
template <typename T>
__device__ __forceinline__ void load_rotated(const AppendArgs& a, const T* src, int c, int pos,
                                             float* x) {
  load8(src + 8 * c, x);
  if (8 * c >= a.rot_dim || (uint32_t)pos >= (uint32_t)a.rot_len) return;
  const int half = a.rot_dim / 2;
  const int64_t t = (int64_t)pos * half;
  if (a.adjacent) {
    const f32x4 co = *reinterpret_cast<const f32x4*>(a.cosines + t + 4 * c);
    const f32x4 si = *reinterpret_cast<const f32x4*>(a.sines + t + 4 * c);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float u = x[2 * i], v = x[2 * i + 1];
      x[2 * i] = u * co[i] - v * si[i];
      x[2 * i + 1] = u * si[i] + v * co[i];
    }
    return;
  }
  const bool low = 8 * c < half;
  const int at = low ? 8 * c : 8 * c - half;
  float y[8];
  load8(src + (low ? 8 * c + half : 8 * c - half), y);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const f32x4 co = *reinterpret_cast<const f32x4*>(a.cosines + t + at + 4 * j);
    const f32x4 si = *reinterpret_cast<const f32x4*>(a.sines + t + at + 4 * j);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float u = x[4 * j + i], v = y[4 * j + i];
      x[4 * j + i] = low ? u * co[i] - v * si[i] : v * si[i] + u * co[i];
    }
  }
}

// Offset, step and codes of a row of which L lanes hold 8 dims each.
template <int L>
__device__ __forceinline__ uint32_t code_row(const float* x, uint32_t* code) {
  float lo = x[0], hi = x[0];
  bool fine = true;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo = fminf(lo, x[i]);
    hi = fmaxf(hi, x[i]);
    fine &= (f32_bits(x[i]) & 0x7F800000u) != 0x7F800000u;
  }
#pragma unroll
  for (int s = 1; s < L; s *= 2) {
    lo = fminf(lo, __shfl_xor(lo, s));
    hi = fmaxf(hi, __shfl_xor(hi, s));
    fine &= __shfl_xor((int)fine, s) != 0;
  }
  uint32_t o = f32_bits(lo);
  o = ((o >> 31) ? o + 0xFFFFu : o) & 0xFFFF0000u;           // down
  const float off = bits_f32(o);
  const float step = bits_f32((f32_bits((hi - off) / 15.0f) + 0xFFFFu) & 0xFFFF0000u);   // up
  // an offset or a step that leaves the range of fp32
  fine &= (o & 0x7F800000u) != 0x7F800000u && (f32_bits(step) & 0x7F800000u) != 0x7F800000u;
  if (!fine) {
#pragma unroll
    for (int i = 0; i < 8; ++i) code[i] = 0;
    return 0x7FC0u;                                          // NaN, step 0
  }
  // the quotients are those of a division; where the reciprocal and its products
  // are far from the ends of fp32, div_by gives the same in three operations
  const bool flat = step == 0.0f, plain = step > 0x1p-60f && step < 0x1p60f;
  const float inv = 1.0f / step;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float d = x[i] - off;
    const float c = plain ? div_by(d, step, inv) : flat ? 0.0f : d / step;
    code[i] = (uint32_t)fminf(fmaxf(__builtin_rintf(c), 0.0f), 15.0f);
  }
  return (o >> 16) | f32_bits(step);
}

// Keys and values: one workgroup per block of 32 tokens and head; queries:
// the workgroups after those, a row of D dims in D/8 lanes. Both in one launch:
// the queries' rows keep the memory busy while the blocks' chains run.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv_append(AppendArgs a) {
  constexpr int L = D / 8, ROWS = 256 / L;
  __shared__ __align__(16) uint8_t vcode[kCodeTokens][D];
  const int l = threadIdx.x % L, r = threadIdx.x / L;
  const KvArgs& c = a.c;
  if ((int)blockIdx.x >= a.kv_groups) {
    const int64_t i = (int64_t)(blockIdx.x - a.kv_groups) * ROWS + r;
    const int64_t t = i / c.heads;
    if (t >= c.total_q) return;
    // the sequence of row t: the last whose first row is not after it; a row's
    // lanes look at L sequences at a time (16 loads after one another, over
    // 65535 sequences, would take longer than all else here)
    int lo = 0;
    for (int n = c.batch; n > 1;) {
      const int step = (n + L - 1) / L;
      const bool before = l * step < n && c.offsets[lo + l * step] <= t;
      const uint64_t lanes =
          (__ballot(before) >> (threadIdx.x & 63 & ~(L - 1))) & ((1ull << L) - 1);
      const int to = max(__popcll(lanes) - 1, 0) * step;
      lo += to;
      n = min(step, n - to);
    }
    const Span s = span_of(c, lo);
    if (t < s.row || t >= s.row + s.count) return;           // a row of no sequence
    const int head = (int)(i - t * c.heads);
    const T* src = static_cast<const T*>(a.q) + t * a.q_stride + (int64_t)head * D;
    float x[8];
    load_rotated(a, src, l, s.pos + (int)(t - s.row), x);
    store8(static_cast<T*>(a.q_out) + i * D + 8 * l, x);
    return;
  }
  const int hk = blockIdx.x % c.kv_heads;
  const int bb = blockIdx.x / c.kv_heads;
  const int b = bb / a.blocks, blk = bb % a.blocks;
  const Span s = span_of(c, b);
  const int cap = c.max_pages * c.page_tokens;
  const int end = min(min(s.pos + s.count, cap), a.rot_dim ? a.rot_len : cap);
  const int first = max(s.pos, 0);
  const int64_t from = (int64_t)(first & ~(kCodeTokens - 1)) + kCodeTokens * blk;
  if (from >= end) return;
  const int p0 = (int)from;
  // new tokens of this block: lo .. hi-1
  const int lo = max(first - p0, 0), hi = min(end - p0, kCodeTokens);
  // A row's loads are on their way while its page is looked up, or the row
  // before it coded.
  float x[8], v[8];
  auto fetch = [&](int t) {
    if (t >= hi) return;
    const int64_t row = s.row + (p0 + t - s.pos);
    load8(static_cast<const T*>(a.v) + row * a.v_stride + (int64_t)hk * D + 8 * l, v);
    load_rotated(a, static_cast<const T*>(a.k) + row * a.k_stride + (int64_t)hk * D, l, p0 + t, x);
  };
  uint8_t* head = head_of(c, b, hk, p0);
  fetch(lo + r);
  if (!head) return;
  const int tp = p0 % c.page_tokens;
  uint32_t* words = reinterpret_cast<uint32_t*>(head);
  // The values' words of this block: which nibbles are new, and the old words,
  // asked for before the rows are coded. The old word is read in any case:
  // with a branch for words of new tokens alone, the compiler stored through an
  // index that the other lanes had not set.
  uint32_t* vw = words + c.page_tokens * (D / 8) + tp * (D / 8);
  const uint32_t fresh = hi > lo ? (0xFFFFFFFFu >> (32 - (hi - lo))) << lo : 0u;   // bit t: token t
  constexpr int WORDS = 4 * D / 256;
  uint32_t put[WORDS], old[WORDS];
#pragma unroll
  for (int k = 0; k < WORDS; ++k) {
    const int i = threadIdx.x + 256 * k, g = (i >> 6) & 3;
    put[k] = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      put[k] |= ((fresh >> (16 * (e >> 2) + 4 * g + (e & 3))) & 1u) * 15u
                << (4 * ((e >> 1) + 4 * (e & 1)));
    old[k] = vw[i];
  }
  for (int t = lo + r; t < hi; t += ROWS) {
    uint32_t code[8];
    uint32_t prm = code_row<L>(x, code);
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) w |= code[i] << (4 * ((i >> 1) + 4 * (i & 1)));
    words[(tp + t) * (D / 8) + l] = w;
    if (l == 0) words[c.page_tokens * (D / 4) + tp + t] = prm;
    prm = code_row<L>(v, code);
    if (l == 0) words[c.page_tokens * (D / 4) + c.page_tokens + tp + t] = prm;
    u32x2 bytes;
    bytes[0] = code[0] | code[1] << 8 | code[2] << 16 | code[3] << 24;
    bytes[1] = code[4] | code[5] << 8 | code[6] << 16 | code[7] << 24;
    *reinterpret_cast<u32x2*>(&vcode[t][8 * l]) = bytes;
    fetch(t + ROWS);
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < WORDS; ++k) {
    const int i = threadIdx.x + 256 * k;
    const int g = (i >> 6) & 3, n = (i >> 2) & 15, q = i & 3, dim = (i >> 8) * 64 + 16 * q + n;
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int t = 16 * (e >> 2) + 4 * g + (e & 3);
      w |= (uint32_t)(vcode[t][dim] & 15) << (4 * ((e >> 1) + 4 * (e & 1)));   // anything if old
    }
    if (put[k]) vw[i] = (old[k] & ~put[k]) | (w & put[k]);
  }
}

struct ReadArgs {
  KvArgs c;
  void* k_out;
  void* v_out;
  int32_t blocks;
};

// Rows read back: a workgroup per block of 32 tokens and head, D/8 lanes per
// row. The eight value words of a lane are shared with the lanes of the seven
// tokens beside it, which find them in the cache: 13.6 us for the same prompts,
// 3.3 TB/s; 3.3 us for a token each.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv_read(ReadArgs a) {
  constexpr int L = D / 8, ROWS = 256 / L;
  const int l = threadIdx.x % L, r = threadIdx.x / L;
  const KvArgs& c = a.c;
  const int hk = blockIdx.x % c.kv_heads;
  const int bb = blockIdx.x / c.kv_heads;
  const int b = bb / a.blocks, blk = bb % a.blocks;
  const Span s = span_of(c, b);
  // the span may begin before the sequence does, at a negative position
  const int64_t p0 = (int64_t)(s.pos & ~(kCodeTokens - 1)) + kCodeTokens * blk;
  if (p0 >= (int64_t)s.pos + s.count) return;
  const bool inside = p0 >= 0 && p0 < c.max_pages * c.page_tokens;
  const uint8_t* head = inside ? head_of(c, b, hk, (int)p0) : nullptr;
  const uint32_t* words = reinterpret_cast<const uint32_t*>(head);
  const int tp = inside ? (int)p0 % c.page_tokens : 0;
  for (int t = r; t < kCodeTokens; t += ROWS) {
    const int i = (int)(p0 + t - s.pos);
    if (i < 0 || i >= s.count) continue;
    float k[8], v[8];
    if (head) {
      const uint32_t* prm = words + c.page_tokens * (D / 4) + tp + t;
      const uint32_t kp = prm[0], vp = prm[c.page_tokens];
      const uint32_t kw = words[(tp + t) * (D / 8) + l];
      const uint32_t* vw = words + c.page_tokens * (D / 8) + tp * (D / 8);
      const int e = 4 * (t >> 4) + (t & 3), at = 4 * ((e >> 1) + 4 * (e & 1));
      const float ko = row_offset(kp), ks = row_step(kp), vo = row_offset(vp), vs = row_step(vp);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int dim = 8 * l + j;
        const uint32_t w = vw[(dim >> 6) * 256 + (((t & 15) >> 2) * 16 + (dim & 15)) * 4 +
                              ((dim & 63) >> 4)];
        k[j] = ko + ks * (float)((kw >> (4 * ((j >> 1) + 4 * (j & 1)))) & 15);
        v[j] = vo + vs * (float)((w >> at) & 15);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) k[j] = v[j] = 0.0f;
    }
    const int64_t row = ((int64_t)(s.row + i) * c.kv_heads + hk) * D + 8 * l;
    store8(static_cast<T*>(a.k_out) + row, k);
    store8(static_cast<T*>(a.v_out) + row, v);
  }
}

// Blocks of 32 positions that n consecutive ones may touch.
int blocks_of(int n) { return (n + kCodeTokens - 2) / kCodeTokens + 1; }

template <typename T>
hipError_t append(const AppendArgs& a, int head_dim, int64_t groups, hipStream_t stream) {
  const dim3 grid((uint32_t)groups), block(256);
  if (head_dim == 64) hipLaunchKernelGGL((kv_append<T, 64>), grid, block, 0, stream, a);
  else if (head_dim == 128) hipLaunchKernelGGL((kv_append<T, 128>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((kv_append<T, 256>), grid, block, 0, stream, a);
  return hipGetLastError();
}

template <typename T>
hipError_t read(const ReadArgs& a, int head_dim, int64_t groups, hipStream_t stream) {
  const dim3 grid((uint32_t)groups), block(256);
  if (head_dim == 64) hipLaunchKernelGGL((kv_read<T, 64>), grid, block, 0, stream, a);
  else if (head_dim == 128) hipLaunchKernelGGL((kv_read<T, 128>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((kv_read<T, 256>), grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_append(const ifq_kv_desc& d, const void* q, const void* k, const void* v,
                            const float* cosines, const float* sines, const KvArgs& c,
                            void* q_out, hipStream_t stream) {
  AppendArgs a;
  a.c = c;
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_out = q_out;
  a.cosines = cosines;
  a.sines = sines;
  a.q_stride = d.q_stride;
  a.k_stride = d.k_stride;
  a.v_stride = d.v_stride;
  a.rot_dim = d.rot_dim;
  a.adjacent = d.rot_adjacent;
  a.rot_len = d.rot_len;
  a.blocks = blocks_of(d.max_q);
  const int64_t kv = (int64_t)d.batch * a.blocks * d.kv_heads;
  const int64_t rows = 256 / (d.head_dim / 8);
  const int64_t qg = q ? ((int64_t)d.total_q * d.heads + rows - 1) / rows : 0;
  if (kv + qg > kMaxGroups) return hipErrorInvalidConfiguration;
  a.kv_groups = (int32_t)kv;
  return d.type == IFQ_TYPE_BF16 ? append<__bf16>(a, d.head_dim, kv + qg, stream)
                                 : append<_Float16>(a, d.head_dim, kv + qg, stream);
}

hipError_t launch_kv_read(const ifq_kv_desc& d, const KvArgs& c, void* k_out, void* v_out,
                          hipStream_t stream) {
  ReadArgs a;
  a.c = c;
  a.k_out = k_out;
  a.v_out = v_out;
  a.blocks = blocks_of(d.max_q);
  const int64_t groups = (int64_t)d.batch * a.blocks * d.kv_heads;
  if (groups > kMaxGroups) return hipErrorInvalidConfiguration;
  return d.type == IFQ_TYPE_BF16 ? read<__bf16>(a, d.head_dim, groups, stream)
                                 : read<_Float16>(a, d.head_dim, groups, stream);
}

}  // namespace ifq
