// Weights in 4-bit floats (e2m1) with a scale of a power of two per 32: the
// quantizer, its read-back, the product of 16-bit activations with such weights,
// and the gated product of a feed-forward block.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ifq_serve.h"

namespace ifq {
namespace {

typedef float v16f __attribute__((ext_vector_type(16)));

// Columns whose four scales lie together: a row's 64 bytes of codes.
constexpr int kF4Block = 128;

__device__ __forceinline__ float f4_scale(uint32_t byte) { return bits_f32(byte << 23); }

// --- quantizer ----------------------------------------------------------------

struct F4QuantArgs {
  const void* x;
  uint8_t* codes;
  uint32_t* scales;              // four bytes each
  int64_t ld_x, ld_codes;
  int32_t rows, k, kb;           // kb: blocks of 128 columns
  int32_t wide;                  // workgroups along k
};

constexpr float kF4MinTop = 0x1p-96f;
constexpr uint32_t kF4Inf = 0x7F800000u;

// Eight consecutive values of a row, which may begin at any element; zeros from k on.
template <typename T>
__device__ __forceinline__ void load8(const T* row, int c, int k, float* v) {
  if (c + 8 <= k) {
    T x[8];
    __builtin_memcpy(x, row + c, sizeof(x));
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)x[i];
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = c + i < k ? (float)row[c + i] : 0.0f;
}

// The scale's byte: the smallest e + 127 with top <= 7 * 2^e. With top = 1.f *
// 2^(E - 127) that is E - 2 where 1.f <= 1.75 and E - 1 above. Infinity and NaN
// (top goes by the bits of the magnitudes) give 255, NaN.
__device__ __forceinline__ uint32_t f4_byte(uint32_t top) {
  if (top >= kF4Inf) return 255u;
  return ((max(top, f32_bits(kF4MinTop)) + 0x1FFFFFu) >> 23) - 2;
}

// Four lanes hold a group of 32, sixteen the 128 columns of a row whose codes lie
// together; a workgroup takes 16 rows x 4 such blocks, so that the scales, which
// run along the rows, are written 64 bytes at a time. Bound by memory, as the read-back is:
// 64001 x 4096 float32 250 us each, 4.8 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void f4_quantize(F4QuantArgs a) {
  const int g = threadIdx.x >> 4, l = threadIdx.x & 15;
  const int bx = blockIdx.x % a.wide, by = blockIdx.x / a.wide;
  const int row = by * 16 + g;
  if (row >= a.rows) return;
  const T* src = static_cast<const T*>(a.x) + (int64_t)row * a.ld_x;
  uint8_t* dst = a.codes + (int64_t)row * a.ld_codes;
  const int k32 = (a.k + 31) & ~31;
  float v[4][8];
#pragma unroll
  for (int p = 0; p < 4; ++p) load8(src, (bx * 4 + p) * kF4Block + 8 * l, a.k, v[p]);
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const int b = bx * 4 + p, c = b * kF4Block + 8 * l;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, f32_bits(v[p][i]) & 0x7FFFFFFFu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    const uint32_t byte = f4_byte(top);
    const float s = f4_scale(byte);
    // x / 2^e to the nearest code, ties to the even one, beyond 6 to 6
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[p][0], v[p][1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[p][2], v[p][3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[p][4], v[p][5], s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[p][6], v[p][7], s, 3);
    if (byte == 255u) w = 0;
    if (c < k32) *reinterpret_cast<uint32_t*>(dst + c / 2) = w;
    // the four groups' bytes meet in the first lane
    uint32_t four = byte << (8 * (l >> 2));
    four |= (uint32_t)__shfl_xor((int)four, 4);
    four |= (uint32_t)__shfl_xor((int)four, 8);
    if (l == 0 && b < a.kb) a.scales[(int64_t)b * a.rows + row] = four;
  }
}

// Four values of two bytes of codes.
__device__ __forceinline__ void f4_values(uint32_t w, float s, float* v) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0);
  const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1);
  const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2);
  const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3);
  v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1];
  v[4] = c[0], v[5] = c[1], v[6] = d[0], v[7] = d[1];
}

// The read-back, in the quantizer's order.
template <typename T>
__global__ __launch_bounds__(256) void f4_dequantize(F4QuantArgs a, T* x) {
  const int g = threadIdx.x >> 4, l = threadIdx.x & 15;
  const int bx = blockIdx.x % a.wide, by = blockIdx.x / a.wide;
  const int row = by * 16 + g;
  if (row >= a.rows) return;
  T* dst = x + (int64_t)row * a.ld_x;
  const uint8_t* src = a.codes + (int64_t)row * a.ld_codes;
  uint32_t w[4], four[4];
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const int b = bx * 4 + p, c = b * kF4Block + 8 * l;
    w[p] = c < a.k ? *reinterpret_cast<const uint32_t*>(src + c / 2) : 0u;
    four[p] = b < a.kb ? a.scales[(int64_t)b * a.rows + row] : 0u;
  }
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const int c = (bx * 4 + p) * kF4Block + 8 * l;
    float v[8];
    f4_values(w[p], f4_scale(four[p] >> (8 * (l >> 2)) & 255u), v);
    T r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (T)v[i];
    if (c + 8 <= a.k) {
      __builtin_memcpy(dst + c, r, sizeof(r));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < a.k) dst[c + i] = r[i];
    }
  }
}

// --- products --------------------------------------------------------------------
//
// A conversion of two codes with their scale is one instruction, and every weight
// is then a 16-bit number without rounding (bfloat16 throughout fp32's range,
// float16 from 2^-24 to 65504): the products run on the 16-bit matrix
// instructions over the whole of k, their sums stay in fp32, and no scale is
// applied to a sum.
//
// The weights are the first operand: a lane's sums then belong to one row of
// activations. Which columns an instruction's operand holds is free as long as both
// agree: a lane takes 32 columns that follow one another, 16 bytes of codes under
// one scale, for four instructions.

struct F4MatmulArgs {
  const void* x;
  const uint8_t* w[2];           // the gate's and the other half's; a product has the second only
  const uint8_t* s[2];
  void* y;
  int64_t ld_x, ld_w, ld_y;
  int32_t m, n, k, kb;
  int32_t y_type, activation;
  int32_t groups_n;              // few rows: workgroups along n
  int32_t groups_m;              // tiles: workgroups along m
};

template <typename T> struct Half;
template <> struct Half<__bf16> {
  typedef bf16x8 x8;
  template <int I> static __device__ __forceinline__ bf16x2 pair(uint32_t w, float s) {
    return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, I);
  }
  static __device__ __forceinline__ f32x4 mma16(x8 a, x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ v16f mma32(x8 a, x8 b, v16f c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <> struct Half<_Float16> {
  typedef f16x8 x8;
  template <int I> static __device__ __forceinline__ f16x2 pair(uint32_t w, float s) {
    return __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, I);
  }
  static __device__ __forceinline__ f32x4 mma16(x8 a, x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ v16f mma32(x8 a, x8 b, v16f c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};

// Eight codes as an operand.
template <typename T>
__device__ __forceinline__ typename Half<T>::x8 operand(uint32_t w, float s) {
  const auto a = Half<T>::template pair<0>(w, s), b = Half<T>::template pair<1>(w, s),
             c = Half<T>::template pair<2>(w, s), d = Half<T>::template pair<3>(w, s);
  return typename Half<T>::x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The activation in fp32. Each form keeps its relative precision where it is small.
__device__ __forceinline__ f32x4 activate(f32x4 g, int kind) {
  f32x4 a, q;
  if (kind == IFQ_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = 0.5f * g[i] * erfcf(g[i] * -0.70710678118654752f);
    return q;
  }
  // g / (1 + e^a); g/2 (1 + tanh(u)) with a = -2u, u = sqrt(2/pi) (g + 0.044715 g^3)
#pragma unroll
  for (int i = 0; i < 4; ++i)
    a[i] = kind == IFQ_ACT_SILU ? -g[i]
                                : g[i] * (g[i] * g[i] * 0.044715f + 1.0f) * -1.5957691216057308f;
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = g[i] / (1.0f + expf(a[i]));
  // Beyond 88.7 e^a leaves fp32's range while the quotient is still in it: there the 1 does not
  // count, and it is g e^-64 e^(64 - a). Behind a branch, since few waves have such lanes
  if (__ballot(fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])) > 88.0f) != 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (a[i] > 88.0f) q[i] = g[i] * 1.6038108905486378e-28f * expf(64.0f - a[i]);
  }
  return q;
}

// Four sums of a row of y, or what is left of it; a row may begin at any element.
template <typename Y>
__device__ __forceinline__ void store4_as(void* y, int64_t at, f32x4 v, int left) {
  typedef Y t4 __attribute__((ext_vector_type(4)));
  typedef t4 any4 __attribute__((aligned(sizeof(Y))));
  Y* p = static_cast<Y*>(y) + at;
  const t4 r = {(Y)v[0], (Y)v[1], (Y)v[2], (Y)v[3]};
  if (left >= 4) {
    *reinterpret_cast<any4*>(p) = r;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) p[i] = r[i];
  }
}

__device__ __forceinline__ void store4(void* y, int type, int64_t at, f32x4 v, int left) {
  if (type == IFQ_TYPE_BF16) store4_as<__bf16>(y, at, v, left);
  else if (type == IFQ_TYPE_F16) store4_as<_Float16>(y, at, v, left);
  else store4_as<float>(y, at, v, left);
}

// Eight activations of a row from column c on; zeros from k on.
template <typename T>
__device__ __forceinline__ typename Half<T>::x8 load_x8(const T* row, int c, int k) {
  typename Half<T>::x8 v;
  if (c + 8 <= k) {
    __builtin_memcpy(&v, row + c, sizeof(v));
    return v;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = c + i < k ? row[c + i] : (T)0.0f;
  return v;
}

// A stage of LDS of a group of `wn` waves of few rows: x, and each wave's weights and scales.
constexpr int few_stage(int xr, int nt, int wn) { return 256 * xr + wn * (1024 * nt + 256); }
constexpr int kLdsBytes = 160 * 1024;

// Zeros: what loads past the end of a row read.
__device__ const u32x4 g_zero[1] = {};

// 16 bytes per lane straight into LDS at dst (uniform) + 16 * lane: from a
// pointer per lane, or from a uniform base and an offset per lane. The waits
// for them are the caller's. A load into LDS must not follow the write of M0
// directly: one wait state, which the compiler does not add inside asm.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_lds16(const void* src, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :: "s"(dst), "v"(src) : "memory", "m0");
}
__device__ __forceinline__ void load_lds16(const uint8_t* base, uint32_t off, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :: "s"(dst), "v"(off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void load_lds4(const void* src, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
               :: "s"(dst), "v"(src) : "memory", "m0");
}
#pragma clang diagnostic pop

// Waits until no more than `left` groups of LOADS loads are on their way.
template <int LOADS, int MOST>
__device__ __forceinline__ void wait_loads(int left) {
  if constexpr (MOST == 0) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  } else {
    if (left >= MOST) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(LOADS * MOST) : "memory");
    else wait_loads<LOADS, MOST - 1>(left);
  }
}

// A wave-uniform pointer that the compiler cannot tell for one.
__device__ __forceinline__ const uint8_t* uniform(const uint8_t* p) {
  const uint64_t v = (uint64_t)(uintptr_t)p;
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)v);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return reinterpret_cast<const uint8_t*>((uintptr_t)((uint64_t)hi << 32 | lo));
}

__device__ __forceinline__ int turned(int q) { return (q & 1) << 1 ^ (q >> 1 & 1) * 3; }

// Few activation rows. A workgroup takes 16 * NT * WN weight rows (of both halves
// together, where HALVES is 2) and XR activation rows. Its waves are groups of WN, which
// share their rows of x; a group takes every so many-th block of 128 columns, and the
// groups' sums are added in LDS in their order.
//
// All operands come through LDS, STAGES blocks of a group there at a time: then
// consecutive lanes read consecutive 16 bytes of a row, 64 of weights and 256 of x, where
// the operands' own order (16 lanes in 16 rows) takes a cycle for each lane (7 x 128000 x
// 4096 102 us, 32 x 4096 x 14336 34). Rows of weights lie 64 bytes apart with group c at
// place c ^ turned(r / 4), rows of x 256 with cell c at c ^ (r & 3) ^ 4 turned(r / 4): a
// read takes 16 lanes at a time (0-3, 12-15, 20-27 and so on), here rows 0-3 and 12-15
// of one group and 4-11 of the next, and these then spread over all 64 banks.
//
// DIRECT: x goes from memory into LDS; it needs 16-byte aligned rows of whole cells.
// Otherwise it goes through registers, and every block waits for all loads on their way: its
// own cells, those of the next block, just asked for, and the weights of every stage. Only other
// workgroups hide that. us with k of 4096 and of 4095: 7 x 4096 5.4 and 5.9, 24 x 4096 7.4 and
// 13.2, 41 x 4096 10.0 and 21.0, gated 7 x 9001 13.5 and 19.3, gated 41 x 9001 19.8 and 28.0.
//
// Up to some 16 rows bound by memory: 7 x 128000 x 4096 52.6 us (5.3 TB/s; the weights, 279 MB,
// do not stay in a cache), 1 x 4096 x 14336 8.1 (3.9 TB/s with the launch; its 31 MB stay in the
// last-level cache from one pass to the next, in a graph over 24 such matrices a pass takes 10.0 and
// with three 9.5). Beyond them a block's wait, reads from LDS, conversions and products
// follow one another: gated 41 x 9001 x 4008 18.8 us.
template <typename T, int XR, int NT, int WN, int STAGES, int HALVES, bool DIRECT>
__global__ __launch_bounds__(XR <= 16 ? 1024 : 512) void f4_matmul_few(F4MatmulArgs a) {
  constexpr int MT = (XR + 15) / 16, COLUMNS = 16 * NT / HALVES;
  constexpr int WB = 1024 * NT + 256, STAGE = few_stage(XR, NT, WN);
  constexpr int XL = XR / 4 / WN;                  // loads of 4 rows of x, for a wave
  static_assert(XL * 4 * WN == XR, "");
  constexpr int LOADS = NT + 1 + (DIRECT ? XL : 0);
  // a group of one wave loads a stage over as soon as it has read it, others after the next
  // barrier
  constexpr int AHEAD = WN == 1 ? STAGES : STAGES - 1;
  extern __shared__ __align__(16) uint8_t few_lds[];        // [group][STAGES][STAGE], then sums
  typedef typename Half<T>::x8 x8;
  const int groups = (blockDim.x >> 6) / WN;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = wave / WN, wn = wave % WN;
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int n0 = (blockIdx.x % a.groups_n * WN + wn) * COLUMNS;
  const int m0 = blockIdx.x / a.groups_n * XR;
  uint8_t* const own = few_lds + group * (STAGES * STAGE);
  const uint32_t to0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)own;
  // what this lane loads: group `piece` of row lane / 4, scales of row lane, and
  // cell `cell` of this wave's rows 4 i + lane / 16
  const int piece = (lane & 3) ^ turned(lane >> 4);
  const uint8_t* wp[NT];
#pragma unroll
  for (int z = 0; z < NT; ++z) {
    const int n = min(n0 + 16 * (z / HALVES) + (lane >> 2), a.n - 1);
    wp[z] = a.w[HALVES == 2 ? z % 2 : 1] + n * a.ld_w + 16 * piece;
  }
  const int sz = HALVES == 2 ? lane >> 4 & 1 : 1;
  const int sn = HALVES == 2 ? (lane >> 5) * 16 + (lane & 15) : lane;
  const uint8_t* sp = a.s[sz] + (int64_t)min(n0 + sn, a.n - 1) * 4;
  const uint8_t* xp[XL];
  int cell[XL];
#pragma unroll
  for (int i = 0; i < XL; ++i) {
    const int row = 4 * (XL * wn + i) + (lane >> 4);
    cell[i] = (lane & 15) ^ (row & 3) ^ 4 * turned(row >> 2);
    xp[i] = static_cast<const uint8_t*>(a.x) + min(m0 + row, a.m - 1) * a.ld_x * 2 + 16 * cell[i];
  }
  x8 held[DIRECT ? 1 : XL];
  auto load_x = [&](int b) {
    if constexpr (!DIRECT)
#pragma unroll
      for (int i = 0; i < XL; ++i)
        held[i] = load_x8(reinterpret_cast<const T*>(xp[i]) + (int64_t)b * kF4Block, 0,
                          a.k - b * kF4Block - 8 * cell[i]);
  };
  auto load = [&](int b, int turn) {
    const uint32_t to = to0 + turn * STAGE, tw = to + 256 * XR + WB * wn;
    const bool whole = (b + 1) * kF4Block <= a.k;
#pragma unroll
    for (int z = 0; z < NT; ++z) {
      const uint8_t* p = wp[z] + (int64_t)b * 64;
      load_lds16(whole || b * kF4Block + 32 * piece < a.k ? (const void*)p : g_zero,
                 tw + 1024 * z);
    }
    if (lane < 16 * NT) load_lds4(sp + (int64_t)b * a.n * 4, tw + 1024 * NT);
    if constexpr (DIRECT)
#pragma unroll
      for (int i = 0; i < XL; ++i) {
        const uint8_t* p = xp[i] + (int64_t)b * (2 * kF4Block);
        load_lds16(whole || b * kF4Block + 8 * cell[i] < a.k ? (const void*)p : g_zero,
                   to + 1024 * (XL * wn + i));
      }
  };
  f32x4 acc[NT][MT];
#pragma unroll
  for (int z = 0; z < NT; ++z)
#pragma unroll
    for (int x = 0; x < MT; ++x) acc[z][x] = f32x4{0, 0, 0, 0};
  const int mine = group < a.kb ? (a.kb - group + groups - 1) / groups : 0;     // blocks
  const int turns = WN == 1 ? mine : (a.kb + groups - 1) / groups;
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (i < mine) load(group + i * groups, i);
  if (mine) load_x(group);
  int turn = 0;
  for (int t = 0; t < turns; ++t, turn = turn + 1 == STAGES ? 0 : turn + 1) {
    const int b = group + t * groups;
    uint8_t* const xs = own + turn * STAGE;
    uint8_t* const ws = xs + 256 * XR + WB * wn;
    if constexpr (!DIRECT) {
      if (t < mine) {
#pragma unroll
        for (int i = 0; i < XL; ++i)
          *reinterpret_cast<x8*>(xs + 1024 * (XL * wn + i) + 16 * lane) = held[i];
        if (t + 1 < mine) load_x(b + groups);
      }
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    } else {
      wait_loads<LOADS, AHEAD - 1>(mine - 1 - t);
    }
    if constexpr (WN > 1) {
      // the stage is there for all its waves, and the last one is read
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (t + AHEAD < mine) load(b + AHEAD * groups, turn == 0 ? STAGES - 1 : turn - 1);
      if (t >= mine) break;                        // the last barrier of a group with a block less
    }
    // groups past k, whatever their bytes
    const uint32_t keep =
        (b + 1) * kF4Block <= a.k ? ~0u : ~0u >> (8 * (3 - (a.k - 1) % kF4Block / 32));
    x8 xv[MT][4];
#pragma unroll
    for (int x = 0; x < MT; ++x) {
      const int row = 16 * x + (XR < 16 ? r & (XR - 1) : r);
      const int swap = (row & 3) ^ 4 * turned(row >> 2);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        xv[x][e] = *reinterpret_cast<const x8*>(xs + 256 * row + 16 * ((4 * g + e) ^ swap));
    }
#pragma unroll
    for (int z = 0; z < NT; ++z) {
      const u32x4 words =
          *reinterpret_cast<const u32x4*>(ws + 1024 * z + 64 * r + 16 * (g ^ turned(r >> 2)));
      const uint32_t four = *reinterpret_cast<const uint32_t*>(ws + 1024 * NT + 4 * (16 * z + r));
      const float scale = f4_scale((four & keep) >> (8 * g) & 255u);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const x8 wv = operand<T>(words[e], scale);
#pragma unroll
        for (int x = 0; x < MT; ++x) acc[z][x] = Half<T>::mma16(wv, xv[x][e], acc[z][x]);
      }
    }
    if constexpr (WN == 1) {
      // read, before it is loaded over
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (t + AHEAD < mine) load(b + AHEAD * groups, turn);
    }
  }
  __syncthreads();                                 // the sums lie where the stages did
  f32x4* sums = reinterpret_cast<f32x4*>(few_lds);
#pragma unroll
  for (int z = 0; z < NT; ++z)
#pragma unroll
    for (int x = 0; x < MT; ++x) sums[((wave * NT + z) * MT + x) * 64 + lane] = acc[z][x];
  __syncthreads();
  for (int i = threadIdx.x; i < 64 * MT * NT / HALVES * WN; i += blockDim.x) {
    const int l = i & 63, x = (i >> 6) % MT, q = (i >> 6) / MT;       // q: 16 columns of y
    const int n = n0 - wn * COLUMNS + 16 * q + 4 * (l >> 4), m = m0 + 16 * x + (l & 15);
    if (m >= a.m || n >= a.n) continue;
    f32x4 v[HALVES];
#pragma unroll
    for (int z = 0; z < HALVES; ++z) {
      const f32x4* p = sums + ((HALVES * q + z) * MT + x) * 64 + l;
      v[z] = *p;
      for (int w = 1; w < groups; ++w) v[z] += p[w * WN * NT * MT * 64];
    }
    if constexpr (HALVES == 2) v[0] = activate(v[0], a.activation) * v[1];
    store4(a.y, a.y_type, m * a.ld_y + n, v[0], a.n - n);
  }
}

// Many activation rows: a workgroup takes 32 * MT of them, in LDS, and its WN
// waves 32 * NT weight rows each, which go from memory to registers, so that a code
// is converted once in the workgroup. Rows of x lie in LDS as 256 bytes a block of
// 128 columns, in 16-byte cells of which row r holds cell c at place c ^ (r & 15): the
// 16 rows of which a read takes a cell each at a time then spread over all 64
// banks. A lane of half h takes the groups 2 h and 2 h + 1 of its weight rows, and cells
// 8 h + 4 j + i of its activation rows beside word i of group 2 h + j.
//
// DIRECT: x goes from memory into LDS, two blocks in turn; it needs 16-byte aligned
// rows of whole cells. Otherwise it goes through registers.
//
// The matrix instructions are at work on 54 and 62 % of the cycles, at the 1.9 to 2.0 GHz that they
// leave; for the rest a block of 128 columns, of which one is on its way ahead, waits for its
// loads and the other waves, or converts. 2011 x 4096 x 14336 201 us (1.18 PFLOP/s), gated 3001 x
// 14336 x 4096 593 (1.19), beside the 1.26 of a long run of plain bfloat16 products.
template <typename T, int MT, int NT, int WN, int WK, int HALVES, bool DIRECT>
__global__ __launch_bounds__(64 * WN * WK, 2) void f4_matmul_tiled(F4MatmulArgs a) {
  constexpr int TM = 32 * MT, ROWS = TM / WN, LOADS = ROWS / 4;
  constexpr int TN = 32 * NT / HALVES;          // columns of y for a wave
  static_assert(TM % (4 * WN) == 0 && NT % HALVES == 0, "");
  __shared__ __align__(16) uint8_t lds[WK][2][TM][256];
  const int any = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave = any % WN, half = any / WN;
  const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
  // tiles that follow one another on an XCD share their weight rows
  const int each = (gridDim.x + 7) / 8, over = gridDim.x & 7;
  const int xcd = blockIdx.x & 7;
  const int tile = (over == 0 || xcd < over ? xcd * each : over * each + (xcd - over) * (each - 1)) +
                   (blockIdx.x >> 3);
  const int m0 = tile % a.groups_m * TM, n0 = tile / a.groups_m * (WN * TN) + wave * TN;

  const uint8_t* wp[NT];
  const uint8_t* sp[NT];
#pragma unroll
  for (int z = 0; z < NT; ++z) {
    const int n = min(n0 + 32 * (z / HALVES) + r, a.n - 1), from = HALVES == 2 ? z % 2 : 1;
    wp[z] = a.w[from] + n * a.ld_w + 32 * h;
    sp[z] = a.s[from] + (int64_t)n * 4 + 2 * h;
  }
  const int64_t sstep = (int64_t)a.n * 4;
  // this wave's rows of x
  const int x0 = min(m0 + ROWS * wave, a.m - 1);
  const uint8_t* xbase = uniform(static_cast<const uint8_t*>(a.x) + x0 * a.ld_x * 2);
  uint32_t xoff[LOADS];
  int cell[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int row = 4 * i + (lane >> 4);
    cell[i] = (lane & 15) ^ ((ROWS * wave + row) & 15);
    xoff[i] = DIRECT ? (uint32_t)(min(row, a.m - 1 - x0) * (int32_t)a.ld_x * 2) + 16 * cell[i] : 0;
  }
  const uint32_t to0 =
      (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)&lds[half][0][0][0] +
      ROWS * wave * 256;
  typename Half<T>::x8 held[DIRECT ? 1 : LOADS];
  auto load_x = [&](int b, int turn) {
    if constexpr (DIRECT) {
      const uint32_t to = to0 + turn * TM * 256;
      const uint8_t* base = xbase + (int64_t)b * 256;
      if ((b + 1) * kF4Block <= a.k) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load_lds16(base, xoff[i], to + 1024 * i);
      } else {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
          load_lds16(b * kF4Block + 8 * cell[i] < a.k ? (const void*)(base + xoff[i]) : g_zero,
                     to + 1024 * i);
      }
    } else {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int64_t row = min(x0 + 4 * i + (lane >> 4), a.m - 1);
        held[i] = load_x8(static_cast<const T*>(a.x) + row * a.ld_x, b * kF4Block + 8 * cell[i],
                          a.k);
      }
    }
  };
  auto store_x = [&](int turn) {
    if constexpr (!DIRECT)
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
        *reinterpret_cast<typename Half<T>::x8*>(
            &lds[half][turn][ROWS * wave + 4 * i + (lane >> 4)][16 * (lane & 15)]) = held[i];
  };
  u32x4 next[NT][2];
  uint32_t next_s[NT];
  auto load_w = [&](int b) {
    const bool whole = (b + 1) * kF4Block <= a.k;
#pragma unroll
    for (int z = 0; z < NT; ++z) {
      const uint8_t* p = wp[z] + (int64_t)b * 64;
      next_s[z] = *reinterpret_cast<const uint16_t*>(sp[z] + b * sstep);
      if (whole) {
        next[z][0] = *reinterpret_cast<const u32x4*>(p);
        next[z][1] = *reinterpret_cast<const u32x4*>(p + 16);
      } else {
        // groups past k: no codes, and not their scale
        const int c = b * kF4Block + 64 * h;
        next[z][0] = next[z][1] = u32x4{0, 0, 0, 0};
        if (c < a.k) next[z][0] = *reinterpret_cast<const u32x4*>(p);
        if (c + 32 < a.k) next[z][1] = *reinterpret_cast<const u32x4*>(p + 16);
        next_s[z] &= c + 32 < a.k ? 0xFFFFu : c < a.k ? 0xFFu : 0u;
      }
    }
  };
  v16f acc[MT][NT];
#pragma unroll
  for (int x = 0; x < MT; ++x)
#pragma unroll
    for (int z = 0; z < NT; ++z) acc[x][z] = v16f{};
  if (half < a.kb) {
    load_x(half, 0);
    load_w(half);
    store_x(0);
  }
  int turn = 0;
  for (int b0 = 0; b0 < a.kb; b0 += WK, turn ^= 1) {
    const int b = b0 + half;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (WK > 1 && b >= a.kb) break;              // the last wait of a group with a block less
    // taken before the next loads: the compiler's wait for these costs nothing here, and
    // later would count the loads into LDS
    u32x4 codes[NT][2];
    uint32_t scales[NT];
#pragma unroll
    for (int z = 0; z < NT; ++z) {
      codes[z][0] = next[z][0];
      codes[z][1] = next[z][1];
      scales[z] = next_s[z];
      asm volatile("" : "+v"(codes[z][0]), "+v"(codes[z][1]), "+v"(scales[z]));
    }
    const bool more = b + WK < a.kb;
    if (more) {
      load_x(b + WK, turn ^ 1);
      load_w(b + WK);
    }
    const uint8_t(*at)[256] = lds[half][turn];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        typename Half<T>::x8 xv[MT], wv[NT];
#pragma unroll
        for (int x = 0; x < MT; ++x)
          xv[x] = *reinterpret_cast<const typename Half<T>::x8*>(
              &at[32 * x + r][16 * ((8 * h + 4 * j + i) ^ (r & 15))]);
#pragma unroll
        for (int z = 0; z < NT; ++z)
          wv[z] = operand<T>(codes[z][j][i], f4_scale(scales[z] >> (8 * j) & 255u));
#pragma unroll
        for (int x = 0; x < MT; ++x)
#pragma unroll
          for (int z = 0; z < NT; ++z) acc[x][z] = Half<T>::mma32(wv[z], xv[x], acc[x][z]);
      }
    if (more) store_x(turn ^ 1);
  }
  if constexpr (WK > 1) {
    // the other groups' sums are added to the first's in their order
    constexpr int SIZE = MT * NT * 16 * 64 * WN;
    static_assert(sizeof(lds) >= sizeof(float) * SIZE * (WK - 1), "");
    __syncthreads();
    float* sums = reinterpret_cast<float*>(&lds[0][0][0][0]) + threadIdx.x % (64 * WN);
    if (half) {
#pragma unroll
      for (int x = 0; x < MT; ++x)
#pragma unroll
        for (int z = 0; z < NT; ++z)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            sums[(half - 1) * SIZE + ((x * NT + z) * 16 + e) * 64 * WN] = acc[x][z][e];
    }
    __syncthreads();
    if (half) return;
#pragma unroll
    for (int q = 0; q < WK - 1; ++q)
#pragma unroll
      for (int x = 0; x < MT; ++x)
#pragma unroll
        for (int z = 0; z < NT; ++z)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            acc[x][z][e] += sums[q * SIZE + ((x * NT + z) * 16 + e) * 64 * WN];
  }
#pragma unroll
  for (int x = 0; x < MT; ++x) {
    const int m = m0 + 32 * x + r;
    if (m >= a.m) continue;
#pragma unroll
    for (int z = 0; z < NT; z += HALVES)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int n = n0 + 32 * (z / HALVES) + 8 * e + 4 * h;
        if (n >= a.n) continue;
        f32x4 v, u;
#pragma unroll
        for (int q = 0; q < 4; ++q)
          v[q] = acc[x][z][4 * e + q], u[q] = acc[x][z + HALVES - 1][4 * e + q];
        if constexpr (HALVES == 2) v = activate(v, a.activation) * u;
        store4(a.y, a.y_type, m * a.ld_y + n, v, a.n - n);
      }
  }
}

int64_t ceil_of(int64_t a, int64_t b) { return (a + b - 1) / b; }

enum Way { kRows, kTiles };

// The kernels of few rows: rows of x, tiles of 16 weight rows of a wave, waves that share x,
// stages, halves. 24 rows of x beside 32 were not faster (24 x 14336 x 4096 11.9 and 10.4 us, 24 x
// 4096 x 14336 15.1 and 16.1).
#define IFQ_F4_FEW(F)                                                              \
  F(4, 1, 1, 4, 1) F(4, 2, 1, 4, 1) F(8, 1, 1, 4, 1) F(8, 2, 1, 4, 1)               \
  F(8, 2, 2, 4, 1) F(16, 1, 1, 3, 1) F(16, 2, 1, 3, 1) F(16, 2, 2, 4, 1)            \
  F(16, 2, 4, 4, 1) F(32, 2, 1, 2, 1) F(32, 2, 2, 3, 1) F(32, 2, 4, 3, 1)           \
  F(48, 2, 1, 2, 1) F(48, 2, 2, 3, 1) F(48, 2, 3, 3, 1) F(48, 2, 4, 3, 1)           \
  F(64, 2, 1, 2, 1) F(64, 2, 2, 3, 1) F(64, 2, 4, 3, 1)                             \
  F(4, 2, 1, 4, 2) F(8, 2, 1, 4, 2) F(8, 2, 2, 4, 2) F(16, 2, 1, 3, 2)              \
  F(16, 2, 2, 4, 2) F(16, 2, 4, 4, 2) F(32, 2, 1, 2, 2) F(32, 2, 2, 3, 2)           \
  F(32, 2, 4, 3, 2) F(48, 2, 1, 2, 2) F(48, 2, 2, 3, 2) F(48, 2, 3, 3, 2)           \
  F(48, 2, 4, 3, 2) F(64, 2, 1, 2, 2) F(64, 2, 2, 3, 2) F(64, 2, 4, 3, 2)

struct Few {
  int32_t xr, nt, wn, stages, halves;
  const char* name;
};

constexpr Few kFew[] = {
#define F(XR, NT, WN, ST, HV) \
  {XR, NT, WN, ST, HV, "f4_matmul_few<" #XR ", " #NT ", " #WN ", " #ST ", " #HV ">"},
    IFQ_F4_FEW(F)
#undef F
};

struct Plan {
  Way way;
  int32_t few;       // few rows: index in kFew
  int32_t shares;    // groups of waves that share k
  int64_t groups;    // workgroups
};

// LDS of a group of waves: its stages, and then its sums.
int few_lds_bytes(const Few& f) {
  return std::max(f.stages * few_stage(f.xr, f.nt, f.wn), (f.xr + 15) / 16 * f.nt * f.wn * 1024);
}

int64_t few_groups(const ifq_f4_matmul_desc& d, const Few& f) {
  return ceil_of(d.m, f.xr) * ceil_of(d.n, 16 * f.nt * f.wn / f.halves);
}

// Time in us of a kernel of few rows with k shared by `shares` groups of waves: a round of
// workgroups is its start and end and its turns, each as long as the loads on their way
// take or as what a CU's workgroups load (KB) and read in LDS. Fitted to 3900 times of
// 260 sizes (m up to 1300, n from 100 to 128000, k from 64 to 14336; DIRECT throughout) with
// 11 % between them on the mean. Among the kernels that plan_of admits the choice by it takes
// 1.5 % longer than the best, 35 % at worst (6 x 12717 x 10888 gated 54.6 and 42.1).
float few_time(const Few& f, int lds, int64_t groups, int64_t kb, int shares) {
  const int64_t each = (groups + 255) / 256;       // on the busiest CU
  const int64_t fit = std::max(1, std::min(kLdsBytes / (lds * shares), 16 / (shares * f.wn)));
  const int64_t at_once = std::min(fit, each), rounds = (each + at_once - 1) / at_once;
  const float load = (float)(shares * few_stage(f.xr, f.nt, f.wn)) / 1024;
  const float read = (float)(shares * f.wn * (f.xr + 4 * f.nt)) / 4;
  const float turn = std::max(1.43f / (float)(f.wn == 1 ? f.stages : f.stages - 1),
                              (float)at_once * (0.009f * load + 0.0045f * read));
  return 0.5f + (float)rounds * (2.4f + 0.023f * (float)(shares * f.wn * f.nt * ((f.xr + 15) / 16)) +
                                 (float)((kb + shares - 1) / shares) * turn);
}

// And of tiles of 128 rows, alone on a CU or in pairs.
float tiles_time(int64_t groups, int64_t kb, int shares) {
  if (shares == 2) return 9.8f + 2.8f * (float)((kb + 1) / 2);
  const int64_t rest = groups % 512;
  return 7.2f + 0.4f * (float)((groups + 511) / 512) +
         (float)kb * (3.2f * (float)(groups / 512) + (rest == 0 ? 0.0f : rest <= 256 ? 1.6f : 3.2f));
}

Plan plan_of(const ifq_f4_matmul_desc& d) {
  const int halves = d.activation ? 2 : 1;
  const int64_t kb = ceil_of(d.k, kF4Block);
  Plan p = {kTiles, 0, 1, ceil_of(d.m, 128) * ceil_of(d.n, 256 / halves)};
  if (p.groups <= 256 && kb >= 2) p.shares = 2;
  float best = d.m <= 32 ? 1e30f : tiles_time(p.groups, kb, p.shares);
  // As many rows of x as there are, or 48 and 64 of more. Fewer rows a workgroup, with more of
  // these, are not admitted, though by the estimate they would be faster where k is long or n
  // small: 64 x 4096 x 14336 17.9 us with 16 rows, 31.1 with 64 (which take 29.1; 96 rows
  // 26.9), 40 x 1000 x 4096 5.3 and 9.6. They have not been timed there.
  const int xr = d.m <= 4 ? 4 : d.m <= 8 ? 8 : d.m <= 64 ? (int)ceil_of(d.m, 16) * 16 : 0;
  for (int i = 0; i < (int)(sizeof(kFew) / sizeof(kFew[0])); ++i) {
    const Few& f = kFew[i];
    if (f.halves != halves || (xr ? f.xr != xr : f.xr < 48)) continue;
    const int lds = few_lds_bytes(f);
    const int64_t groups = few_groups(d, f);
    for (int shares = 8 / f.wn; shares >= 1; shares /= 2) {
      const int some = (int)std::min<int64_t>(std::min(shares, kLdsBytes / lds), kb);
      const float t = few_time(f, lds, groups, kb, some);
      if (t < best) best = t, p = {kRows, i, some, groups};
    }
  }
  return p;
}

template <typename T, int XR, int NT, int WN, int STAGES, int HALVES, bool DIRECT>
void few_of(F4MatmulArgs& a, const Plan& p, hipStream_t stream) {
  a.groups_n = (int32_t)ceil_of(a.n, 16 * NT * WN / HALVES);
  hipLaunchKernelGGL((f4_matmul_few<T, XR, NT, WN, STAGES, HALVES, DIRECT>),
                     dim3((uint32_t)p.groups), dim3(64 * WN * p.shares),
                     few_lds_bytes(kFew[p.few]) * p.shares, stream, a);
}

template <typename T, int HALVES, bool DIRECT>
void few(F4MatmulArgs& a, const Plan& p, hipStream_t stream) {
  int i = 0;
#define F(XR, NT, WN, ST, HV)                                                    \
  if constexpr (HV == HALVES)                                                    \
    if (p.few == i) return few_of<T, XR, NT, WN, ST, HV, DIRECT>(a, p, stream);  \
  ++i;
  IFQ_F4_FEW(F)
#undef F
}

template <typename T, int HALVES, bool DIRECT>
void tiled(F4MatmulArgs& a, const Plan& p, hipStream_t stream) {
  a.groups_m = (a.m + 127) / 128;
  const dim3 grid((uint32_t)p.groups);
  if (p.shares == 2)
    hipLaunchKernelGGL((f4_matmul_tiled<T, 4, 2, 4, 2, HALVES, DIRECT>), grid, dim3(512), 0,
                       stream, a);
  else
    hipLaunchKernelGGL((f4_matmul_tiled<T, 4, 2, 4, 1, HALVES, DIRECT>), grid, dim3(256), 0,
                       stream, a);
}

template <typename T, int HALVES>
void matmul(F4MatmulArgs& a, const Plan& p, hipStream_t stream) {
  // whole cells of 16 bytes, and the tiles' 32-bit offsets within their rows (the kernels of few
  // rows have 64-bit ones, and would not need the last condition)
  const bool direct = (reinterpret_cast<uintptr_t>(a.x) & 15) == 0 && a.ld_x % 8 == 0 &&
                      a.k % 8 == 0 && a.ld_x <= (1 << 22);
  if (p.way == kRows)
    return direct ? few<T, HALVES, true>(a, p, stream) : few<T, HALVES, false>(a, p, stream);
  if (direct) tiled<T, HALVES, true>(a, p, stream);
  else tiled<T, HALVES, false>(a, p, stream);
}

F4QuantArgs quant_args(const ifq_f4_weights_desc& d, const void* codes, const void* scales) {
  F4QuantArgs a;
  a.x = nullptr;
  a.codes = static_cast<uint8_t*>(const_cast<void*>(codes));
  a.scales = static_cast<uint32_t*>(const_cast<void*>(scales));
  a.ld_x = d.ld_x;
  a.ld_codes = d.ld_codes;
  a.rows = (int32_t)d.rows;
  a.k = (int32_t)d.k;
  a.kb = (int32_t)((d.k + kF4Block - 1) / kF4Block);
  a.wide = (a.kb + 3) / 4;
  return a;
}

dim3 quant_grid(const F4QuantArgs& a) {
  return dim3((uint32_t)((int64_t)a.wide * ((a.rows + 15) / 16)));
}

}  // namespace

int64_t f4_quant_groups(const ifq_f4_weights_desc& d) {
  return (d.rows + 15) / 16 * ((d.k + 4 * kF4Block - 1) / (4 * kF4Block));
}

hipError_t launch_f4_quantize(const ifq_f4_weights_desc& d, const void* x, void* codes,
                              void* scales, hipStream_t stream) {
  F4QuantArgs a = quant_args(d, codes, scales);
  a.x = x;
  const dim3 grid = quant_grid(a), block(256);
  if (d.x_type == IFQ_TYPE_BF16)
    hipLaunchKernelGGL((f4_quantize<__bf16>), grid, block, 0, stream, a);
  else if (d.x_type == IFQ_TYPE_F16)
    hipLaunchKernelGGL((f4_quantize<_Float16>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((f4_quantize<float>), grid, block, 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_f4_dequantize(const ifq_f4_weights_desc& d, const void* codes,
                                const void* scales, void* x, hipStream_t stream) {
  const F4QuantArgs a = quant_args(d, codes, scales);
  const dim3 grid = quant_grid(a), block(256);
  if (d.x_type == IFQ_TYPE_BF16)
    hipLaunchKernelGGL((f4_dequantize<__bf16>), grid, block, 0, stream, a,
                       static_cast<__bf16*>(x));
  else if (d.x_type == IFQ_TYPE_F16)
    hipLaunchKernelGGL((f4_dequantize<_Float16>), grid, block, 0, stream, a,
                       static_cast<_Float16*>(x));
  else
    hipLaunchKernelGGL((f4_dequantize<float>), grid, block, 0, stream, a,
                       static_cast<float*>(x));
  return hipGetLastError();
}

size_t f4_matmul_workspace_bytes(const ifq_f4_matmul_desc&) { return 0; }

int64_t f4_matmul_groups(const ifq_f4_matmul_desc& d) {
  if (d.m == 0 || d.n == 0) return 0;
  const Plan p = plan_of(d);
  const int waves = p.way == kRows ? p.shares * kFew[p.few].wn : 4 * p.shares;
  return ceil_of(p.groups * waves, 4);
}

const char* f4_matmul_kernel_name(const ifq_f4_matmul_desc& d) {
  if (d.m == 0 || d.n == 0) return "";
  const Plan p = plan_of(d);
  if (p.way == kRows) return kFew[p.few].name;
  if (p.shares == 2)
    return d.activation ? "f4_matmul_tiled<4, 2, 4, 2, 2>" : "f4_matmul_tiled<4, 2, 4, 2, 1>";
  return d.activation ? "f4_matmul_tiled<4, 2, 4, 1, 2>" : "f4_matmul_tiled<4, 2, 4, 1, 1>";
}

hipError_t launch_f4_matmul(const ifq_f4_matmul_desc& d, const void* x, const void* w_gate,
                            const void* gate_scales, const void* w, const void* w_scales,
                            void* y, void*, hipStream_t stream) {
  F4MatmulArgs a;
  a.x = x;
  a.w[0] = static_cast<const uint8_t*>(w_gate);
  a.w[1] = static_cast<const uint8_t*>(w);
  a.s[0] = static_cast<const uint8_t*>(gate_scales);
  a.s[1] = static_cast<const uint8_t*>(w_scales);
  a.y = y;
  a.ld_x = d.ld_x;
  a.ld_w = d.ld_w;
  a.ld_y = d.ld_y;
  a.m = (int32_t)d.m;
  a.n = (int32_t)d.n;
  a.k = (int32_t)d.k;
  a.kb = (int32_t)((d.k + kF4Block - 1) / kF4Block);
  a.y_type = d.y_type;
  a.activation = d.activation;
  const Plan p = plan_of(d);
  if (d.x_type == IFQ_TYPE_BF16) {
    if (d.activation) matmul<__bf16, 2>(a, p, stream);
    else matmul<__bf16, 1>(a, p, stream);
  } else {
    if (d.activation) matmul<_Float16, 2>(a, p, stream);
    else matmul<_Float16, 1>(a, p, stream);
  }
  return hipGetLastError();
}

}  // namespace ifq
