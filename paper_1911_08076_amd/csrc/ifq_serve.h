// Internals of the operators for serving language models: the 8-bit float
// quantizer and block-scaled product (ifq_f8.hip), the paged cache of 4-bit
// codes (ifq_kv.hip) and attention over it (ifq_attn.hip). Arguments reach the
// launchers validated (ifq_serve.cpp).
#pragma once

#include <hip/hip_runtime.h>

#include "ifq.h"
#include "ifq_internal.h"

namespace ifq {

constexpr int kF8Block = 128;    // values under one scale of an 8-bit float row
constexpr int kCodeTokens = 32;  // tokens of one block of value codes in a page
constexpr int64_t kMaxGroups = (1 << 24) - 1;   // workgroups of 256 of one launch: 2^32 threads

struct KvArgs {
  const int32_t* offsets;        // [batch + 1] rows of the new tokens
  const int32_t* lengths;        // [batch] cached tokens, the new ones included
  const int32_t* pages;          // [batch][max_pages]
  uint8_t* cache;
  int64_t page_bytes, head_bytes;
  int32_t batch, total_q, max_q, heads, kv_heads, page_tokens, num_pages, max_pages;
};

hipError_t launch_f8_quantize(const ifq_f8_quant_desc& d, const void* x, void* codes,
                              float* scales, hipStream_t stream);

size_t f8_matmul_workspace_bytes(const ifq_f8_matmul_desc& d);
int64_t f8_matmul_groups(const ifq_f8_matmul_desc& d);   // workgroups of its launch
const char* f8_matmul_kernel_name(const ifq_f8_matmul_desc& d);
hipError_t launch_f8_matmul(const ifq_f8_matmul_desc& d, const void* a, const float* a_scales,
                            const void* w, const float* w_scales, void* y, void* ws,
                            hipStream_t stream);

hipError_t launch_kv_append(const ifq_kv_desc& d, const void* q, const void* k, const void* v,
                            const float* cosines, const float* sines, const KvArgs& a,
                            void* q_out, hipStream_t stream);
hipError_t launch_kv_read(const ifq_kv_desc& d, const KvArgs& a, void* k_out, void* v_out,
                          hipStream_t stream);

size_t kv_attention_workspace_bytes(const ifq_kv_desc& d);
const char* kv_attention_kernel_name(const ifq_kv_desc& d);
hipError_t launch_kv_attention(const ifq_kv_desc& d, const void* q, const KvArgs& a, void* out,
                               void* ws, hipStream_t stream);

#ifdef __HIPCC__
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bits_f32(uint32_t v) { return __builtin_bit_cast(float, v); }
__device__ __forceinline__ uint32_t f32_bits(float v) { return __builtin_bit_cast(uint32_t, v); }

// Offset and step of a cached row, two bfloat16 in a word.
__device__ __forceinline__ float row_offset(uint32_t w) { return bits_f32(w << 16); }
__device__ __forceinline__ float row_step(uint32_t w) { return bits_f32(w & 0xFFFF0000u); }

// Parts go through memory between workgroups whose caches do not see one
// another. Each number is written through to where all see it and read from
// there (accesses of agent scope), so that no workgroup has to write back or
// drop a whole cache for it: with fences around plain accesses an attention of
// 768 sequences and heads in two parts each took 382 us instead of 74 unsplit.
__device__ __forceinline__ void put_pair(float* p, float x, float y) {
  const uint64_t v = f32_bits(x) | (uint64_t)f32_bits(y) << 32;
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), v, __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ f32x2 get_pair(const float* p) {
  return __builtin_bit_cast(f32x2, __hip_atomic_load(reinterpret_cast<const uint64_t*>(p),
                                                     __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// Counts a workgroup of `parts` that has written its part of a unit's result;
// true in the one that comes last, which then may read all parts, and leaves
// the counter at 0. Called by all threads; flag is in LDS.
__device__ __forceinline__ bool comes_last(uint32_t* count, int parts, int* flag) {
  // the part is in memory before the barrier, and so before the count
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0)
    *flag = atomicInc(count, (uint32_t)(parts - 1)) == (uint32_t)(parts - 1);
  __syncthreads();
  return *flag != 0;
}

// x / d correctly rounded, given inv = 1 / d correctly rounded: the product
// is within an ulp, and its remainder, exact in the fma, corrects it.
__device__ __forceinline__ float div_by(float x, float d, float inv) {
  const float q = x * inv;
  return __builtin_fmaf(__builtin_fmaf(-q, d, x), inv, q);
}
#endif

}  // namespace ifq
