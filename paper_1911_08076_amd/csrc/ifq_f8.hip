// Quantizer to 8-bit floats (e4m3) with a scale per block of 128 values, and
// the product of two such matrices.
#include <hip/hip_runtime.h>

#include "ifq_serve.h"

namespace ifq {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));

// --- quantizer ----------------------------------------------------------------

struct QuantArgs {
  const void* x;
  uint8_t* codes;
  float* scales;
  int64_t ld_x, ld_codes;
  int32_t rows, k, kb, rb;       // kb, rb: scale blocks along k and along the rows
};

constexpr float kMinTop = 0x1p-96f;
constexpr uint32_t kInfBits = 0x7F800000u;

// Eight consecutive values of a row, as fp32; zeros from k on.
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* row, int c, int k, float* v) {
  if (VEC && c + 8 <= k) {
    if constexpr (sizeof(T) == 4) {
      const f32x4 a = *reinterpret_cast<const f32x4*>(row + c);
      const f32x4 b = *reinterpret_cast<const f32x4*>(row + c + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
    } else {
      typedef T t8 __attribute__((ext_vector_type(8)));
      const t8 a = *reinterpret_cast<const t8*>(row + c);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = (float)a[i];
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = c + i < k ? (float)row[c + i] : 0.0f;
}

// Largest |v|, by the bits of the magnitudes, where infinity and NaN are the
// largest of all.
__device__ __forceinline__ uint32_t top8(const float* v) {
  uint32_t t = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) t = max(t, f32_bits(v[i]) & 0x7FFFFFFFu);
  return t;
}

__device__ __forceinline__ uint32_t max16(uint32_t t) {   // over 16 lanes
#pragma unroll
  for (int s = 1; s < 16; s *= 2) t = max(t, (uint32_t)__shfl_xor((int)t, s));
  return t;
}

// Codes of eight values: (x * 448/512) / (top / 512), in which nothing
// overflows; the division is correctly rounded (div_by), so that values
// exactly between two codes stay there and go to the even one.
__device__ __forceinline__ u32x2 codes8(const float* v, float top, bool fine) {
  const float d = top * 0x1p-9f, inv = 1.0f / d;
  float q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    // the correction would turn -0 into 0
    const float r = __builtin_copysignf(div_by(v[i] * 0.875f, d, inv), v[i]);
    q[i] = fine ? fminf(fmaxf(r, -448.0f), 448.0f) : 0.0f;
  }
  u32x2 w;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int t = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * i], q[4 * i + 1], 0, false);
    t = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * i + 2], q[4 * i + 3], t, true);
    w[i] = (uint32_t)t;
  }
  return w;
}

__device__ __forceinline__ float scale_of(uint32_t top) {
  return top >= kInfBits ? bits_f32(0x7FC00000u) : fmaxf(bits_f32(top), kMinTop) / 448.0f;
}

// A scale per row: 16 lanes hold a block of 128 values. ROWS = 16: a
// workgroup takes 16 rows x 4 blocks, so that the scales, which run along the
// rows, are written 64 bytes at a time; ROWS = 1: 16 blocks of one row.
template <typename T, bool VEC, int ROWS>
__global__ __launch_bounds__(256) void f8_quantize_rows(QuantArgs a) {
  constexpr int PER = ROWS == 16 ? 4 : 1;
  const int g = threadIdx.x >> 4, l = threadIdx.x & 15;
  const int row = ROWS == 16 ? blockIdx.y * 16 + g : blockIdx.y;
  const int b0 = ROWS == 16 ? blockIdx.x * PER : blockIdx.x * 16 + g;
  if (row >= a.rows) return;
  const T* src = static_cast<const T*>(a.x) + (int64_t)row * a.ld_x;
  uint8_t* dst = a.codes + (int64_t)row * a.ld_codes;
  const int k16 = (a.k + 15) & ~15;
  float v[PER][8];
#pragma unroll
  for (int p = 0; p < PER; ++p) load8<T, VEC>(src, (b0 + p) * kF8Block + 8 * l, a.k, v[p]);
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const int b = b0 + p, c = b * kF8Block + 8 * l;
    const uint32_t top = max16(top8(v[p]));
    const u32x2 w = codes8(v[p], fmaxf(bits_f32(top), kMinTop), top < kInfBits);
    if (c < k16) *reinterpret_cast<u32x2*>(dst + c) = w;
    if (l == 0 && b < a.kb) a.scales[(int64_t)b * a.rb + row] = scale_of(top);
  }
}

// A scale per 128 x 128: a workgroup holds the block in registers.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void f8_quantize_blocks(QuantArgs a) {
  __shared__ uint32_t part[4];
  const int g = threadIdx.x >> 4, l = threadIdx.x & 15;
  const int c = blockIdx.x * kF8Block + 8 * l;
  const int k16 = (a.k + 15) & ~15;
  float v[8][8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = blockIdx.y * kF8Block + 16 * i + g;
    if (row < a.rows) {
      load8<T, VEC>(static_cast<const T*>(a.x) + (int64_t)row * a.ld_x, c, a.k, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
    }
    top = max(top, top8(v[i]));
  }
  top = max16(top);
  top = max(top, (uint32_t)__shfl_xor((int)top, 16));
  top = max(top, (uint32_t)__shfl_xor((int)top, 32));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
  __syncthreads();
  top = max(max(part[0], part[1]), max(part[2], part[3]));
  const float t = fmaxf(bits_f32(top), kMinTop);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = blockIdx.y * kF8Block + 16 * i + g;
    if (row >= a.rows || c >= k16) continue;
    *reinterpret_cast<u32x2*>(a.codes + (int64_t)row * a.ld_codes + c) =
        codes8(v[i], t, top < kInfBits);
  }
  if (threadIdx.x == 0) a.scales[(int64_t)blockIdx.x * a.rb + blockIdx.y] = scale_of(top);
}

template <typename T, bool VEC>
void quantize(const QuantArgs& a, int block_rows, hipStream_t stream) {
  if (block_rows == 128) {
    hipLaunchKernelGGL((f8_quantize_blocks<T, VEC>), dim3(a.kb, a.rb), dim3(256), 0, stream, a);
  } else if (a.rows < 16) {
    hipLaunchKernelGGL((f8_quantize_rows<T, VEC, 1>), dim3((a.kb + 15) / 16, a.rows), dim3(256),
                       0, stream, a);
  } else {
    hipLaunchKernelGGL((f8_quantize_rows<T, VEC, 16>), dim3((a.kb + 3) / 4, (a.rows + 15) / 16),
                       dim3(256), 0, stream, a);
  }
}

template <typename T>
void quantize(const QuantArgs& a, int block_rows, hipStream_t stream) {
  const bool vec = reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && a.ld_x * sizeof(T) % 16 == 0;
  if (vec) quantize<T, true>(a, block_rows, stream);
  else quantize<T, false>(a, block_rows, stream);
}

// --- product --------------------------------------------------------------------

struct MatmulArgs {
  const uint8_t* a;
  const uint8_t* w;
  const float* sa;
  const float* sw;
  void* y;
  int64_t ld_a, ld_w, ld_y;
  int32_t m, n, k, kb, nb;
};

// 32 bytes of a row's codes; zeros from k on.
__device__ __forceinline__ v8i load32(const uint8_t* row, int c, int k) {
  v4i lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
  if (c < k) lo = *reinterpret_cast<const v4i*>(row + c);
  if (c + 16 < k) hi = *reinterpret_cast<const v4i*>(row + c + 16);
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Eight codes (two words) as 16-bit floats, which hold every e4m3 value.
__device__ __forceinline__ f16x8 halves(int a, int b) {
  const f16x2 x = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false);
  const f16x2 y = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true);
  const f16x2 z = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false);
  const f16x2 w = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true);
  return f16x8{x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
}

// 64 x 64 outputs per workgroup, 32 x 32 per wave: a lane of the weights'
// operand holds 32 bytes of a column's row, one of the activations' the same
// of an activation row, so a lane's sums all belong to one activation row and
// take its scale as one number. Every block of 128 is summed from zero and
// added with its scale. The products go through the 16-bit matrix
// instructions, whose sums are fp32: the 8-bit ones keep some 16 bits below
// the largest product (measured: 1.5e-5 of the result's norm over 128 normal
// values, against 1e-8).
template <typename T>
__global__ __launch_bounds__(256) void f8_matmul(MatmulArgs a) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int r = lane & 31, h = lane >> 5;
  const int n0 = blockIdx.x * 64 + (wave & 1) * 32, m0 = blockIdx.y * 64 + (wave >> 1) * 32;
  if (n0 >= a.n || m0 >= a.m) return;
  const int m = min(m0 + r, a.m - 1);
  const uint8_t* wrow = a.w + (int64_t)min(n0 + r, a.n - 1) * a.ld_w;
  const uint8_t* arow = a.a + (int64_t)m * a.ld_a;
  v16f acc = {};
  for (int b = 0; b < a.kb; ++b) {
    v16f part = {};
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int c = b * kF8Block + 64 * s + 32 * h;
      const v8i wv = load32(wrow, c, a.k), av = load32(arow, c, a.k);
#pragma unroll
      for (int t = 0; t < 8; t += 2)
        part = __builtin_amdgcn_mfma_f32_32x32x16_f16(halves(wv[t], wv[t + 1]),
                                                      halves(av[t], av[t + 1]), part, 0, 0, 0);
    }
    const float s = a.sa[(int64_t)b * a.m + m] * a.sw[(int64_t)b * a.nb + n0 / kF8Block];
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = __builtin_fmaf(part[i], s, acc[i]);
  }
  if (m0 + r >= a.m) return;
  T* y = static_cast<T*>(a.y) + (int64_t)m * a.ld_y;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int n = n0 + 8 * (i >> 2) + 4 * h + (i & 3);
    if (n < a.n) y[n] = (T)acc[i];
  }
}

}  // namespace

hipError_t launch_f8_quantize(const ifq_f8_quant_desc& d, const void* x, void* codes,
                              float* scales, hipStream_t stream) {
  QuantArgs a;
  a.x = x;
  a.codes = static_cast<uint8_t*>(codes);
  a.scales = scales;
  a.ld_x = d.ld_x;
  a.ld_codes = d.ld_codes;
  a.rows = (int32_t)d.rows;
  a.k = (int32_t)d.k;
  a.kb = (int32_t)((d.k + kF8Block - 1) / kF8Block);
  a.rb = (int32_t)((d.rows + d.block_rows - 1) / d.block_rows);
  if (d.x_type == IFQ_TYPE_BF16) quantize<__bf16>(a, d.block_rows, stream);
  else if (d.x_type == IFQ_TYPE_F16) quantize<_Float16>(a, d.block_rows, stream);
  else quantize<float>(a, d.block_rows, stream);
  return hipGetLastError();
}

size_t f8_matmul_workspace_bytes(const ifq_f8_matmul_desc& d) { return 0; }

hipError_t launch_f8_matmul(const ifq_f8_matmul_desc& d, const void* a_, const float* a_scales,
                            const void* w, const float* w_scales, void* y, void* ws,
                            hipStream_t stream) {
  MatmulArgs a;
  a.a = static_cast<const uint8_t*>(a_);
  a.w = static_cast<const uint8_t*>(w);
  a.sa = a_scales;
  a.sw = w_scales;
  a.y = y;
  a.ld_a = d.ld_a;
  a.ld_w = d.ld_w;
  a.ld_y = d.ld_y;
  a.m = (int32_t)d.m;
  a.n = (int32_t)d.n;
  a.k = (int32_t)d.k;
  a.kb = (a.k + kF8Block - 1) / kF8Block;
  a.nb = (a.n + kF8Block - 1) / kF8Block;
  const dim3 grid((a.n + 63) / 64, (a.m + 63) / 64);
  if (d.y_type == IFQ_TYPE_BF16)
    hipLaunchKernelGGL((f8_matmul<__bf16>), grid, dim3(256), 0, stream, a);
  else if (d.y_type == IFQ_TYPE_F16)
    hipLaunchKernelGGL((f8_matmul<_Float16>), grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((f8_matmul<float>), grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ifq
