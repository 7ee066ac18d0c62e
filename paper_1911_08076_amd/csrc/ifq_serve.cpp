// Host side of the operators for serving language models (include/ifq.h):
// every argument is checked here before a launch.
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "ifq.h"
#include "ifq_internal.h"
#include "ifq_serve.h"

namespace {

ifq_status fail(ifq_status st, const char* fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  return ifq::set_error(st, buf);
}

ifq_status launched(hipError_t e, const char* what) {
  if (e == hipErrorInvalidConfiguration)     // more workgroups than a launch may have
    return fail(IFQ_ERR_UNSUPPORTED, "%s: too large for one launch", what);
  if (e != hipSuccess) return fail(IFQ_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return ifq::set_error(IFQ_OK, "");
}

// Sizes are kept where the kernels' 32-bit row and tile indexes hold them;
// byte offsets are 64-bit throughout.
constexpr int64_t kMaxRows = (int64_t)1 << 30;
constexpr int64_t kMaxStride = (int64_t)1 << 40;
constexpr int64_t kMaxProductStride = (int64_t)1 << 25;

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

size_t type_bytes(int32_t t) { return t == IFQ_TYPE_F32 ? 4 : 2; }

ifq_status check_quant(const ifq_f8_quant_desc* d) {
  if (!d) return fail(IFQ_ERR_INVALID_ARGUMENT, "quantize: desc is NULL");
  if (d->rows < 0 || d->k < 0 || d->rows > kMaxRows || d->k > kMaxRows)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "quantize: rows and k must be in 0..2^30");
  if (d->x_type != IFQ_TYPE_BF16 && d->x_type != IFQ_TYPE_F16 && d->x_type != IFQ_TYPE_F32)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "quantize: unknown type %d", d->x_type);
  if (d->block_rows != 1 && d->block_rows != 128)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "quantize: block_rows must be 1 or 128");
  if (d->ld_x < d->k || d->ld_codes < d->k || d->ld_x > kMaxStride || d->ld_codes > kMaxStride)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "quantize: a leading dimension is below k");
  if (d->ld_codes % 16)
    return fail(IFQ_ERR_UNSUPPORTED, "quantize: ld_codes must be a multiple of 16");
  return IFQ_OK;
}

ifq_status check_matmul(const ifq_f8_matmul_desc* d) {
  if (!d) return fail(IFQ_ERR_INVALID_ARGUMENT, "product: desc is NULL");
  if (d->m < 0 || d->n < 0 || d->k < 1 || d->m > kMaxRows || d->n > kMaxRows || d->k > kMaxRows)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "product: need m, n in 0..2^30 and k in 1..2^30");
  if (d->y_type != IFQ_TYPE_BF16 && d->y_type != IFQ_TYPE_F16 && d->y_type != IFQ_TYPE_F32)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "product: unknown type %d", d->y_type);
  if (d->reserved != 0)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "product: reserved must be 0");
  if (d->ld_a < d->k || d->ld_w < d->k || d->ld_y < d->n || d->ld_a > kMaxStride ||
      d->ld_w > kMaxStride || d->ld_y > kMaxStride)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "product: a leading dimension is below its row");
  if (d->k % 16 || d->ld_a % 16 || d->ld_w % 16)
    return fail(IFQ_ERR_UNSUPPORTED, "product: k, ld_a and ld_w must be multiples of 16");
  // 32-bit offsets within the rows of a tile
  if (d->ld_a > kMaxProductStride || d->ld_w > kMaxProductStride)
    return fail(IFQ_ERR_UNSUPPORTED, "product: ld_a and ld_w may be up to 2^25");
  if (ifq::f8_matmul_groups(*d) > ifq::kMaxGroups)
    return fail(IFQ_ERR_UNSUPPORTED, "product: m x n is too large for one launch");
  return IFQ_OK;
}

ifq_status check_kv(const ifq_kv_desc* d) {
  if (!d) return fail(IFQ_ERR_INVALID_ARGUMENT, "kv: desc is NULL");
  if (d->batch < 0 || d->total_q < 0 || d->max_q < 0 || d->max_kv < 0)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "kv: batch, total_q, max_q, max_kv must be >= 0");
  if (d->total_q > kMaxRows || d->max_q > d->total_q)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "kv: max_q must be at most total_q");
  if (d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "kv: heads must be a multiple of kv_heads");
  if (d->type != IFQ_TYPE_BF16 && d->type != IFQ_TYPE_F16)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "kv: type must be bf16 or f16");
  if (d->num_pages < 1 || d->max_pages < 1)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "kv: need num_pages and max_pages >= 1");
  if ((d->causal != 0 && d->causal != 1) || (d->rot_adjacent != 0 && d->rot_adjacent != 1))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "kv: causal and rot_adjacent must be 0 or 1");
  if (d->window < 0 || d->sinks < 0 || (d->window > 0 && !d->causal))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "kv: a window needs causal, window and sinks >= 0");
  if (d->rot_dim < 0 || d->rot_dim > d->head_dim || d->rot_len < 0)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "kv: rot_dim must be in 0..head_dim, rot_len >= 0");
  if (!(d->scale - d->scale == 0.0f))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "kv: scale must be finite");
  if (d->page_tokens < 32 || d->page_tokens > 4096 || d->page_tokens % 32)
    return fail(IFQ_ERR_UNSUPPORTED, "kv: page_tokens must be a multiple of 32 up to 4096");
  if (d->head_dim != 64 && d->head_dim != 128 && d->head_dim != 256)
    return fail(IFQ_ERR_UNSUPPORTED, "kv: head_dim must be 64, 128 or 256");
  if (d->rot_dim % 16) return fail(IFQ_ERR_UNSUPPORTED, "kv: rot_dim must be a multiple of 16");
  if ((int64_t)d->max_pages * d->page_tokens > kMaxRows)
    return fail(IFQ_ERR_UNSUPPORTED, "kv: a sequence may have up to 2^30 positions");
  if (d->batch > 65535 || (int64_t)d->heads * d->max_q > (int64_t)d->kv_heads * kMaxRows ||
      d->heads > 65535)
    return fail(IFQ_ERR_UNSUPPORTED, "kv: too many sequences or heads for one launch");
  return IFQ_OK;
}

ifq_status check_stride(int64_t stride, int64_t row, const char* name) {
  if (stride < row || stride > kMaxStride)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "kv: %s_stride is below its %lld elements", name,
                (long long)row);
  if (stride % 8)
    return fail(IFQ_ERR_UNSUPPORTED, "kv: %s_stride must be a multiple of 8", name);
  return IFQ_OK;
}

ifq_status check_batch(const int32_t* offsets, const int32_t* lengths, const int32_t* pages,
                       const void* cache) {
  if (!offsets || !lengths || !pages || !cache)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "kv: offsets, lengths, pages and cache are required");
  if (!aligned(offsets, 4) || !aligned(lengths, 4) || !aligned(pages, 4) || !aligned(cache, 16))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "kv: the cache must be 16-byte, the tables 4-byte "
                "aligned");
  return IFQ_OK;
}

bool known(int32_t t) { return t == IFQ_TYPE_BF16 || t == IFQ_TYPE_F16 || t == IFQ_TYPE_F32; }

// Bytes of a row of 4-bit codes.
int64_t code_bytes(int64_t k) { return (k + 31) / 32 * 16; }

ifq_status check_f4_weights(const ifq_f4_weights_desc* d) {
  if (!d) return fail(IFQ_ERR_INVALID_ARGUMENT, "f4 weights: desc is NULL");
  if (d->rows < 0 || d->k < 0 || d->rows > kMaxRows || d->k > kMaxRows)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "f4 weights: rows and k must be in 0..2^30");
  if (!known(d->x_type))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "f4 weights: unknown type %d", d->x_type);
  if (d->reserved != 0)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "f4 weights: reserved must be 0");
  if (d->ld_x < d->k || d->ld_codes < code_bytes(d->k) || d->ld_x > kMaxStride ||
      d->ld_codes > kMaxStride)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "f4 weights: a leading dimension is below its row");
  if (d->ld_codes % 16)
    return fail(IFQ_ERR_UNSUPPORTED, "f4 weights: ld_codes must be a multiple of 16");
  if (ifq::f4_quant_groups(*d) > ifq::kMaxGroups)
    return fail(IFQ_ERR_UNSUPPORTED, "f4 weights: rows x k is too large for one launch");
  return IFQ_OK;
}

ifq_status check_f4_pointers(const ifq_f4_weights_desc* d, const void* x, const void* codes,
                             const void* scales) {
  if (!x || !codes || !scales)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "f4 weights: x, codes and scales are required");
  if (!aligned(x, type_bytes(d->x_type)) || !aligned(codes, 16) || !aligned(scales, 4))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "f4 weights: x must be aligned to its element, codes "
                "to 16 bytes, scales to 4");
  return IFQ_OK;
}

ifq_status check_f4_matmul(const ifq_f4_matmul_desc* d, bool gated) {
  if (!d) return fail(IFQ_ERR_INVALID_ARGUMENT, "f4 product: desc is NULL");
  if (d->m < 0 || d->n < 0 || d->k < 1 || d->m > kMaxRows || d->n > kMaxRows || d->k > kMaxRows)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "f4 product: need m, n in 0..2^30 and k in 1..2^30");
  if (d->x_type != IFQ_TYPE_BF16 && d->x_type != IFQ_TYPE_F16)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "f4 product: x must be bf16 or f16");
  if (!known(d->y_type))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "f4 product: unknown type %d", d->y_type);
  if (gated ? d->activation < IFQ_ACT_SILU || d->activation > IFQ_ACT_GELU_TANH
            : d->activation != IFQ_ACT_NONE)
    return fail(IFQ_ERR_INVALID_ARGUMENT, gated ? "f4 gated product: unknown activation %d"
                                                : "f4 product: activation %d, none expected",
                d->activation);
  if (d->reserved != 0)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "f4 product: reserved must be 0");
  if (d->ld_x < d->k || d->ld_w < code_bytes(d->k) || d->ld_y < d->n || d->ld_x > kMaxStride ||
      d->ld_w > kMaxStride || d->ld_y > kMaxStride)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "f4 product: a leading dimension is below its row");
  if (d->ld_w % 16)
    return fail(IFQ_ERR_UNSUPPORTED, "f4 product: ld_w must be a multiple of 16");
  if (d->ld_w > kMaxProductStride)      // as for the 8-bit product; these kernels' offsets are 64-bit
    return fail(IFQ_ERR_UNSUPPORTED, "f4 product: ld_w may be up to 2^25");
  if (ifq::f4_matmul_groups(*d) > ifq::kMaxGroups)
    return fail(IFQ_ERR_UNSUPPORTED, "f4 product: m x n is too large for one launch");
  return IFQ_OK;
}

ifq_status f4_product(const ifq_f4_matmul_desc* d, bool gated, const void* x, const void* w_gate,
                      const void* gate_scales, const void* w, const void* w_scales, void* y,
                      void* ws, size_t ws_bytes, hipStream_t stream) {
  if (ifq_status st = check_f4_matmul(d, gated)) return st;
  if (d->m == 0 || d->n == 0) return ifq::set_error(IFQ_OK, "");
  if (!x || !w || !w_scales || !y || (gated && (!w_gate || !gate_scales)))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "f4 product: x, the weights, their scales and y are "
                "required");
  if (!aligned(x, 2) || !aligned(w, 16) || !aligned(w_gate, 16) || !aligned(w_scales, 4) ||
      !aligned(gate_scales, 4) || !aligned(y, type_bytes(d->y_type)))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "f4 product: weights must be 16-byte aligned, scales "
                "4-byte, x and y to their elements");
  const size_t need = ifq::f4_matmul_workspace_bytes(*d);
  if (need && (!ws || ws_bytes < need))
    return fail(IFQ_ERR_INSUFFICIENT_BUFFER, "f4 product: workspace of %zu bytes, %zu needed",
                ws ? ws_bytes : (size_t)0, need);
  if (need && !aligned(ws, 16))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "f4 product: the workspace must be 16-byte aligned");
  return launched(ifq::launch_f4_matmul(*d, x, w_gate, gate_scales, w, w_scales, y, ws, stream),
                  gated ? "f4_gated" : "f4_matmul");
}

ifq_status check_logprobs(const ifq_logprobs_desc* d) {
  if (!d) return fail(IFQ_ERR_INVALID_ARGUMENT, "logprobs: desc is NULL");
  if (d->rows < 0 || d->n < 1 || d->rows > kMaxRows || d->n > kMaxRows)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "logprobs: need rows in 0..2^30 and n in 1..2^30");
  if (!known(d->x_type))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "logprobs: unknown type %d", d->x_type);
  if (d->top < 0 || d->top > 64 || d->top > d->n)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "logprobs: top must be in 0..64 and at most n");
  if (!(d->scale > 0.0f && d->scale <= 0x1p64f))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "logprobs: scale must be above 0 and at most 2^64");
  if (d->reserved != 0)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "logprobs: reserved must be 0");
  if (d->ld_x < d->n || d->ld_top < d->top || d->ld_x > kMaxStride || d->ld_top > kMaxStride)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "logprobs: a leading dimension is below its row");
  if (d->top > 0 && d->n > ifq::kMostTopValues)
    return fail(IFQ_ERR_UNSUPPORTED, "logprobs: top tokens of up to 2^20 values");
  if (ifq::logprobs_groups(*d) > ifq::kMaxGroups)
    return fail(IFQ_ERR_UNSUPPORTED, "logprobs: too many rows for one launch");
  return IFQ_OK;
}

bool nothing(const ifq_kv_desc* d) { return d->batch == 0 || d->total_q == 0 || d->max_q == 0; }

int64_t head_bytes(const ifq_kv_desc* d) { return (int64_t)d->page_tokens * (d->head_dim + 8); }

ifq::KvArgs kv_args(const ifq_kv_desc* d, const int32_t* offsets, const int32_t* lengths,
                    const int32_t* pages, const void* cache) {
  ifq::KvArgs a;
  a.offsets = offsets;
  a.lengths = lengths;
  a.pages = pages;
  a.cache = static_cast<uint8_t*>(const_cast<void*>(cache));
  a.head_bytes = head_bytes(d);
  a.page_bytes = a.head_bytes * d->kv_heads;
  a.batch = d->batch;
  a.total_q = d->total_q;
  a.max_q = d->max_q;
  a.heads = d->heads;
  a.kv_heads = d->kv_heads;
  a.page_tokens = d->page_tokens;
  a.num_pages = d->num_pages;
  a.max_pages = d->max_pages;
  return a;
}

}  // namespace

extern "C" {

ifq_status ifq_f8_quantize(const ifq_f8_quant_desc* d, const void* x, void* codes, float* scales,
                           hipStream_t stream) {
  if (ifq_status st = check_quant(d)) return st;
  if (d->rows == 0 || d->k == 0) return ifq::set_error(IFQ_OK, "");
  if (!x || !codes || !scales)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "quantize: x, codes and scales are required");
  if (!aligned(x, type_bytes(d->x_type)) || !aligned(codes, 16) || !aligned(scales, 4))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "quantize: x must be aligned to its element, codes to "
                "16 bytes, scales to 4");
  return launched(ifq::launch_f8_quantize(*d, x, codes, scales, stream), "f8_quantize");
}

size_t ifq_f8_matmul_workspace_bytes(const ifq_f8_matmul_desc* d) {
  if (check_matmul(d) || d->m == 0 || d->n == 0) return 0;
  return ifq::f8_matmul_workspace_bytes(*d);
}

const char* ifq_f8_matmul_kernel_name(const ifq_f8_matmul_desc* d) {
  return check_matmul(d) ? "" : ifq::f8_matmul_kernel_name(*d);
}

ifq_status ifq_f8_matmul(const ifq_f8_matmul_desc* d, const void* a, const float* a_scales,
                         const void* w, const float* w_scales, void* y, void* ws,
                         size_t ws_bytes, hipStream_t stream) {
  if (ifq_status st = check_matmul(d)) return st;
  if (d->m == 0 || d->n == 0) return ifq::set_error(IFQ_OK, "");
  if (!a || !a_scales || !w || !w_scales || !y)
    return fail(IFQ_ERR_INVALID_ARGUMENT, "product: a, w, their scales and y are required");
  if (!aligned(a, 16) || !aligned(w, 16) || !aligned(a_scales, 4) || !aligned(w_scales, 4) ||
      !aligned(y, type_bytes(d->y_type)))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "product: a and w must be 16-byte aligned, scales "
                "4-byte, y to its element");
  const size_t need = ifq::f8_matmul_workspace_bytes(*d);
  if (need && (!ws || ws_bytes < need))
    return fail(IFQ_ERR_INSUFFICIENT_BUFFER, "product: workspace of %zu bytes, %zu needed",
                ws ? ws_bytes : (size_t)0, need);
  if (need && !aligned(ws, 16))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "product: the workspace must be 16-byte aligned");
  return launched(ifq::launch_f8_matmul(*d, a, a_scales, w, w_scales, y, ws, stream),
                  "f8_matmul");
}

size_t ifq_kv_cache_bytes(const ifq_kv_desc* d) {
  if (check_kv(d)) return 0;
  return (size_t)(head_bytes(d) * d->kv_heads) * (size_t)d->num_pages;
}

ifq_status ifq_kv_append(const ifq_kv_desc* d, const void* q, const void* k, const void* v,
                         const float* cosines, const float* sines, const int32_t* offsets,
                         const int32_t* lengths, const int32_t* pages, void* cache, void* q_out,
                         hipStream_t stream) {
  if (ifq_status st = check_kv(d)) return st;
  const int64_t qrow = (int64_t)d->heads * d->head_dim, krow = (int64_t)d->kv_heads * d->head_dim;
  if (q)
    if (ifq_status st = check_stride(d->q_stride, qrow, "q")) return st;
  if (ifq_status st = check_stride(d->k_stride, krow, "k")) return st;
  if (ifq_status st = check_stride(d->v_stride, krow, "v")) return st;
  if (nothing(d)) return ifq::set_error(IFQ_OK, "");
  if (ifq_status st = check_batch(offsets, lengths, pages, cache)) return st;
  if (!k || !v || (q == nullptr) != (q_out == nullptr))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "append: k and v are required, q_out goes with q");
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(q_out, 16))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "append: q, k, v and q_out must be 16-byte aligned");
  if ((d->rot_dim > 0) != (cosines != nullptr) || (d->rot_dim > 0) != (sines != nullptr))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "append: the rotation's tables go with rot_dim > 0");
  if (!aligned(cosines, 16) || !aligned(sines, 16))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "append: the rotation's tables must be 16-byte "
                "aligned");
  return launched(ifq::launch_kv_append(*d, q, k, v, cosines, sines,
                                        kv_args(d, offsets, lengths, pages, cache), q_out,
                                        stream), "kv_append");
}

ifq_status ifq_kv_read(const ifq_kv_desc* d, const int32_t* offsets, const int32_t* lengths,
                       const int32_t* pages, const void* cache, void* k_out, void* v_out,
                       hipStream_t stream) {
  if (ifq_status st = check_kv(d)) return st;
  if (nothing(d)) return ifq::set_error(IFQ_OK, "");
  if (ifq_status st = check_batch(offsets, lengths, pages, cache)) return st;
  if (!k_out || !v_out || !aligned(k_out, 16) || !aligned(v_out, 16))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "read: k_out and v_out are required, 16-byte aligned");
  return launched(ifq::launch_kv_read(*d, kv_args(d, offsets, lengths, pages, cache), k_out,
                                      v_out, stream), "kv_read");
}

size_t ifq_kv_attention_workspace_bytes(const ifq_kv_desc* d) {
  if (check_kv(d) || nothing(d)) return 0;
  return ifq::kv_attention_workspace_bytes(*d);
}

const char* ifq_kv_attention_kernel_name(const ifq_kv_desc* d) {
  return check_kv(d) || nothing(d) ? "" : ifq::kv_attention_kernel_name(*d);
}

ifq_status ifq_kv_attention(const ifq_kv_desc* d, const void* q, const int32_t* offsets,
                            const int32_t* lengths, const int32_t* pages, const void* cache,
                            void* out, void* ws, size_t ws_bytes, hipStream_t stream) {
  if (ifq_status st = check_kv(d)) return st;
  const int64_t row = (int64_t)d->heads * d->head_dim;
  if (ifq_status st = check_stride(d->q_stride, row, "q")) return st;
  if (ifq_status st = check_stride(d->o_stride, row, "o")) return st;
  if (nothing(d)) return ifq::set_error(IFQ_OK, "");
  if (ifq_status st = check_batch(offsets, lengths, pages, cache)) return st;
  if (!q || !out || !aligned(q, 16) || !aligned(out, 16))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "attention: q and out are required, 16-byte aligned");
  const size_t need = ifq::kv_attention_workspace_bytes(*d);
  if (need && (!ws || ws_bytes < need))
    return fail(IFQ_ERR_INSUFFICIENT_BUFFER, "attention: workspace of %zu bytes, %zu needed",
                ws ? ws_bytes : (size_t)0, need);
  if (need && !aligned(ws, 16))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "attention: the workspace must be 16-byte aligned");
  return launched(ifq::launch_kv_attention(*d, q, kv_args(d, offsets, lengths, pages, cache),
                                           out, ws, stream), "kv_attention");
}

ifq_status ifq_f4_quantize(const ifq_f4_weights_desc* d, const void* x, void* codes, void* scales,
                           hipStream_t stream) {
  if (ifq_status st = check_f4_weights(d)) return st;
  if (d->rows == 0 || d->k == 0) return ifq::set_error(IFQ_OK, "");
  if (ifq_status st = check_f4_pointers(d, x, codes, scales)) return st;
  return launched(ifq::launch_f4_quantize(*d, x, codes, scales, stream), "f4_quantize");
}

ifq_status ifq_f4_dequantize(const ifq_f4_weights_desc* d, const void* codes, const void* scales,
                             void* x, hipStream_t stream) {
  if (ifq_status st = check_f4_weights(d)) return st;
  if (d->rows == 0 || d->k == 0) return ifq::set_error(IFQ_OK, "");
  if (ifq_status st = check_f4_pointers(d, x, codes, scales)) return st;
  return launched(ifq::launch_f4_dequantize(*d, codes, scales, x, stream), "f4_dequantize");
}

size_t ifq_f4_matmul_workspace_bytes(const ifq_f4_matmul_desc* d) {
  return check_f4_matmul(d, false) ? 0 : ifq::f4_matmul_workspace_bytes(*d);
}

size_t ifq_f4_gated_workspace_bytes(const ifq_f4_matmul_desc* d) {
  return check_f4_matmul(d, true) ? 0 : ifq::f4_matmul_workspace_bytes(*d);
}

const char* ifq_f4_matmul_kernel_name(const ifq_f4_matmul_desc* d) {
  return check_f4_matmul(d, false) ? "" : ifq::f4_matmul_kernel_name(*d);
}

const char* ifq_f4_gated_kernel_name(const ifq_f4_matmul_desc* d) {
  return check_f4_matmul(d, true) ? "" : ifq::f4_matmul_kernel_name(*d);
}

ifq_status ifq_f4_matmul(const ifq_f4_matmul_desc* d, const void* x, const void* w,
                         const void* w_scales, void* y, void* ws, size_t ws_bytes,
                         hipStream_t stream) {
  return f4_product(d, false, x, nullptr, nullptr, w, w_scales, y, ws, ws_bytes, stream);
}

ifq_status ifq_f4_gated(const ifq_f4_matmul_desc* d, const void* x, const void* w_gate,
                        const void* gate_scales, const void* w_up, const void* up_scales,
                        void* y, void* ws, size_t ws_bytes, hipStream_t stream) {
  return f4_product(d, true, x, w_gate, gate_scales, w_up, up_scales, y, ws, ws_bytes, stream);
}

size_t ifq_logprobs_workspace_bytes(const ifq_logprobs_desc* d) {
  return check_logprobs(d) ? 0 : ifq::logprobs_workspace_bytes(*d);
}

ifq_status ifq_logprobs(const ifq_logprobs_desc* d, const void* logits, const int32_t* tokens,
                        float* logprob, float* entropy, float* top_logprobs, int32_t* top_tokens,
                        void* ws, size_t ws_bytes, hipStream_t stream) {
  if (ifq_status st = check_logprobs(d)) return st;
  if (d->rows == 0) return ifq::set_error(IFQ_OK, "");
  if (!logits || (tokens == nullptr) != (logprob == nullptr))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "logprobs: logits are required, logprob goes with "
                "tokens");
  if ((d->top > 0) != (top_logprobs != nullptr) || (d->top > 0) != (top_tokens != nullptr))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "logprobs: top_logprobs and top_tokens go with top > 0");
  if (!aligned(logits, type_bytes(d->x_type)) || !aligned(tokens, 4) || !aligned(logprob, 4) ||
      !aligned(entropy, 4) || !aligned(top_logprobs, 4) || !aligned(top_tokens, 4))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "logprobs: arrays must be aligned to their elements");
  const size_t need = ifq::logprobs_workspace_bytes(*d);
  if (need && (!ws || ws_bytes < need))
    return fail(IFQ_ERR_INSUFFICIENT_BUFFER, "logprobs: workspace of %zu bytes, %zu needed",
                ws ? ws_bytes : (size_t)0, need);
  if (need && !aligned(ws, 16))
    return fail(IFQ_ERR_INVALID_ARGUMENT, "logprobs: the workspace must be 16-byte aligned");
  return launched(ifq::launch_logprobs(*d, logits, tokens, logprob, entropy, top_logprobs,
                                       top_tokens, ws, stream), "logprobs");
}

}  // extern "C"
