// Weights in 4-bit floats (e2m1) with a scale of a power of two per 32: the
// quantizer, its read-back, the product of 16-bit activations with such weights,
// and the gated product of a feed-forward block.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ifq_serve.h"

namespace ifq {
namespace {

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
// run along the rows, are written 64 bytes at a time.
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
  int32_t groups_n;              // workgroups along n
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
};
template <> struct Half<_Float16> {
  typedef f16x8 x8;
  template <int I> static __device__ __forceinline__ f16x2 pair(uint32_t w, float s) {
    return __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, I);
  }
  static __device__ __forceinline__ f32x4 mma16(x8 a, x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
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
__device__ __forceinline__ float activate(float g, int kind) {
  if (kind == IFQ_ACT_SILU) return g / (1.0f + expf(-g));
  if (kind == IFQ_ACT_GELU) return 0.5f * g * erfcf(g * -0.70710678118654752f);
  // g/2 (1 + tanh(u)) = g / (1 + e^-2u), u = sqrt(2/pi) (g + 0.044715 g^3)
  return g / (1.0f + expf(g * (g * g * 0.044715f + 1.0f) * -1.5957691216057308f));
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

// Few activation rows. A workgroup takes 16 weight rows (of each half, where
// HALVES is 2) and 16 * MT activation rows, its KS waves every KS-th block of 128
// columns; the waves' sums are added in LDS in their order.
template <typename T, int MT, int KS, int HALVES>
__global__ __launch_bounds__(64 * KS) void f4_matmul_few(F4MatmulArgs a) {
  __shared__ __align__(16) float sums[KS][HALVES][MT][64][4];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int n0 = blockIdx.x % a.groups_n * 16, m0 = blockIdx.x / a.groups_n * 16 * MT;
  const int wrow = min(n0 + r, a.n - 1);
  const T* xrow[MT];
#pragma unroll
  for (int x = 0; x < MT; ++x)
    xrow[x] = static_cast<const T*>(a.x) + (int64_t)min(m0 + 16 * x + r, a.m - 1) * a.ld_x;
  f32x4 acc[HALVES][MT];
#pragma unroll
  for (int z = 0; z < HALVES; ++z)
#pragma unroll
    for (int x = 0; x < MT; ++x) acc[z][x] = f32x4{0, 0, 0, 0};
  for (int b = wave; b < a.kb; b += KS) {
    const int c = b * kF4Block + 32 * g;
    u32x4 codes[HALVES];
    float scale[HALVES];
#pragma unroll
    for (int z = 0; z < HALVES; ++z) {
      const int from = z + 2 - HALVES;
      codes[z] = u32x4{0, 0, 0, 0};
      scale[z] = 0.0f;                       // a group past k, whatever its byte
      if (c < a.k) {
        codes[z] = *reinterpret_cast<const u32x4*>(a.w[from] + wrow * a.ld_w + c / 2);
        scale[z] = f4_scale(a.s[from][((int64_t)b * a.n + wrow) * 4 + g]);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      typename Half<T>::x8 xv[MT];
#pragma unroll
      for (int x = 0; x < MT; ++x) xv[x] = load_x8(xrow[x], c + 8 * i, a.k);
#pragma unroll
      for (int z = 0; z < HALVES; ++z) {
        const auto wv = operand<T>(codes[z][i], scale[z]);
#pragma unroll
        for (int x = 0; x < MT; ++x) acc[z][x] = Half<T>::mma16(wv, xv[x], acc[z][x]);
      }
    }
  }
#pragma unroll
  for (int z = 0; z < HALVES; ++z)
#pragma unroll
    for (int x = 0; x < MT; ++x) *reinterpret_cast<f32x4*>(sums[wave][z][x][lane]) = acc[z][x];
  __syncthreads();
  for (int i = threadIdx.x; i < 64 * MT; i += 64 * KS) {
    const int x = i >> 6, l = i & 63, n = n0 + 4 * (l >> 4), m = m0 + 16 * x + (l & 15);
    f32x4 v[HALVES];
#pragma unroll
    for (int z = 0; z < HALVES; ++z) {
      v[z] = *reinterpret_cast<const f32x4*>(sums[0][z][x][l]);
#pragma unroll
      for (int w = 1; w < KS; ++w) v[z] += *reinterpret_cast<const f32x4*>(sums[w][z][x][l]);
    }
    if (m < a.m && n < a.n) {
      if constexpr (HALVES == 2)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[0][e] = activate(v[0][e], a.activation) * v[1][e];
      store4(a.y, a.y_type, (int64_t)m * a.ld_y + n, v[0], a.n - n);
    }
  }
}

int64_t groups_of(int64_t m, int64_t n) { return (m + 31) / 32 * ((n + 15) / 16); }

template <typename T, int HALVES>
void few(F4MatmulArgs& a, hipStream_t stream) {
  a.groups_n = (a.n + 15) / 16;
  const dim3 grid((uint32_t)groups_of(a.m, a.n)), block(256);
  hipLaunchKernelGGL((f4_matmul_few<T, 2, 4, HALVES>), grid, block, 0, stream, a);
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
  return d.m == 0 || d.n == 0 ? 0 : groups_of(d.m, d.n);
}

const char* f4_matmul_kernel_name(const ifq_f4_matmul_desc& d) {
  if (d.m == 0 || d.n == 0) return "";
  return d.activation ? "f4_matmul_few<2, 4, 2>" : "f4_matmul_few<2, 4, 1>";
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
  if (d.x_type == IFQ_TYPE_BF16) {
    if (d.activation) few<__bf16, 2>(a, stream);
    else few<__bf16, 1>(a, stream);
  } else {
    if (d.activation) few<_Float16, 2>(a, stream);
    else few<_Float16, 1>(a, stream);
  }
  return hipGetLastError();
}

}  // namespace ifq
