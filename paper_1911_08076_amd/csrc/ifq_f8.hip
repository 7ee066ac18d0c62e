// Quantizer to 8-bit floats (e4m3) with a scale per block of 128 values, and
// the product of two such matrices.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "ifq_serve.h"

namespace ifq {
namespace {

typedef float v16f __attribute__((ext_vector_type(16)));

// --- quantizer ----------------------------------------------------------------

struct QuantArgs {
  const void* x;
  uint8_t* codes;
  float* scales;
  int64_t ld_x, ld_codes;
  int32_t rows, k, kb, rb;       // kb, rb: scale blocks along k and along the rows
  int32_t wide;                  // workgroups along k
};

constexpr float kMinTop = 0x1p-96f;
constexpr uint32_t kInfBits = 0x7F800000u;

// Eight consecutive values of a row, as fp32; zeros from k on. Rows may begin at
// any element: the copies become loads of 16 bytes whatever the address (rows of
// 4095 bfloat16 element by element, 8192 of them: 47 us instead of 21).
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

// A scale per row: 16 lanes hold a block of 128 values, read once and kept in
// registers between the search for the largest and the coding. ROWS = 16: a
// workgroup takes 16 rows x 4 blocks, so that the scales, which run along the
// rows, are written 64 bytes at a time; ROWS = 1: 16 blocks of one row.
// Bound by memory: 8192 x 14336 bfloat16 values 73 us, 4.9 TB/s (a copy reaches 4.6
// to 4.7; after some fifteen calls in a row 85 to 100 us), with vector instructions
// on 81 % of the cycles; one row of 4096 takes 2.1 us on the GPU, the latency of a
// launch.
template <typename T, int ROWS>
__global__ __launch_bounds__(256) void f8_quantize_rows(QuantArgs a) {
  constexpr int PER = ROWS == 16 ? 4 : 1;
  const int g = threadIdx.x >> 4, l = threadIdx.x & 15;
  const int bx = blockIdx.x % a.wide, by = blockIdx.x / a.wide;
  const int row = ROWS == 16 ? by * 16 + g : by;
  const int b0 = ROWS == 16 ? bx * PER : bx * 16 + g;
  if (row >= a.rows) return;
  const T* src = static_cast<const T*>(a.x) + (int64_t)row * a.ld_x;
  uint8_t* dst = a.codes + (int64_t)row * a.ld_codes;
  const int k16 = (a.k + 15) & ~15;
  float v[PER][8];
#pragma unroll
  for (int p = 0; p < PER; ++p) load8(src, (b0 + p) * kF8Block + 8 * l, a.k, v[p]);
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const int b = b0 + p, c = b * kF8Block + 8 * l;
    const uint32_t top = max16(top8(v[p]));
    const u32x2 w = codes8(v[p], fmaxf(bits_f32(top), kMinTop), top < kInfBits);
    if (c < k16) *reinterpret_cast<u32x2*>(dst + c) = w;
    if (l == 0 && b < a.kb) a.scales[(int64_t)b * a.rb + row] = scale_of(top);
  }
}

// A scale per 128 x 128: a workgroup holds the block in registers, 64 values to
// a thread, so that it too is read once. For weights, when they are loaded. Bound by
// memory: 14336 x 4096 bfloat16 values 38.7 us, 4.6 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void f8_quantize_blocks(QuantArgs a) {
  __shared__ uint32_t part[4];
  const int g = threadIdx.x >> 4, l = threadIdx.x & 15;
  const int bx = blockIdx.x % a.wide, by = blockIdx.x / a.wide;
  const int c = bx * kF8Block + 8 * l;
  const int k16 = (a.k + 15) & ~15;
  float v[8][8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = by * kF8Block + 16 * i + g;
    if (row < a.rows) {
      load8(static_cast<const T*>(a.x) + (int64_t)row * a.ld_x, c, a.k, v[i]);
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
    const int row = by * kF8Block + 16 * i + g;
    if (row >= a.rows || c >= k16) continue;
    *reinterpret_cast<u32x2*>(a.codes + (int64_t)row * a.ld_codes + c) =
        codes8(v[i], t, top < kInfBits);
  }
  if (threadIdx.x == 0) a.scales[(int64_t)bx * a.rb + by] = scale_of(top);
}

template <typename T>
hipError_t quantize(QuantArgs a, int block_rows, hipStream_t stream) {
  // Row by row where three quarters of its workgroups have work, or where rows
  // are few (us, row by row and 16 rows at a time: 16 x 4096 2.8 and 4.4, 1024 x
  // 14336 11.7 and 13.3, 8192 x 14336 72 and 75; but 8192 x 1000 10.1 and 9.3,
  // 8192 x 128 7.8 and 4.3)
  const int32_t per = (a.kb + 15) / 16;                // workgroups of a row
  const bool one = block_rows == 1 && (int64_t)a.rows * per <= kMaxGroups &&
                   (a.rows < 1024 || 4 * a.kb >= 3 * 16 * per);
  const int64_t high = block_rows == 128 ? a.rb : one ? a.rows : (a.rows + 15) / 16;
  a.wide = block_rows == 128 ? a.kb : one ? per : (a.kb + 3) / 4;
  if (a.wide * high > kMaxGroups) return hipErrorInvalidConfiguration;
  const dim3 grid((uint32_t)(a.wide * high)), block(256);
  if (block_rows == 128)
    hipLaunchKernelGGL((f8_quantize_blocks<T>), grid, block, 0, stream, a);
  else if (one)
    hipLaunchKernelGGL((f8_quantize_rows<T, 1>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((f8_quantize_rows<T, 16>), grid, block, 0, stream, a);
  return hipGetLastError();
}

// --- product --------------------------------------------------------------------
//
// The products go through the 16-bit matrix instructions, whose sums are fp32,
// as the definition has them for every type of y. The 8-bit ones would run at twice
// the rate, but keep some 16 bits below the largest product (1.5e-5 of the result's
// norm over 128 normal values, against 1e-8): below what rounds a bfloat16 or a
// float16 result, but not sums in fp32, so they are not used. Every e4m3 value is a
// 16-bit float, and a conversion of two codes is one instruction.
//
// The weights are the first operand and the activations the second: a lane's
// sums then belong to one activation row, whose scale is one number, and the
// weights' scale is the same for the whole wave. Every block of 128 is summed
// from zero and added with the product of its scales.

struct MatmulArgs {
  const uint8_t* a;
  const uint8_t* w;
  const float* sa;
  const float* sw;
  void* y;
  int64_t ld_a, ld_w, ld_y;
  int32_t m, n, k, kb, nb;
  int32_t splits;          // of k, where tiles of 64 x 64 are few
  uint32_t* count;
  float* part;
};

// Eight codes (two words) as 16-bit floats.
__device__ __forceinline__ f16x8 halves(uint32_t a, uint32_t b) {
  const f16x2 x = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false);
  const f16x2 y = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true);
  const f16x2 z = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false);
  const f16x2 w = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true);
  return f16x8{x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
}

// Adds the sum of a block of 128 times the block's two scales: as one factor, where
// fp32 holds sa * sw as a normal number. Where it is below those or infinite the
// larger scale comes first: the result may be well within the range all the same
// (scales of 2^-80 and 2^-65 with a sum of 2^20).
__device__ __forceinline__ bool out_of_range(float f) {
  return __builtin_amdgcn_classf(f, 0x2F4);       // not normal, and no NaN
}

struct Scales {
  float first, then;
  __device__ __forceinline__ Scales(float sa, float sw) {
    const float one = sa * sw;
    const bool out = out_of_range(one), a = __builtin_fabsf(sa) > __builtin_fabsf(sw);
    first = out ? (a ? sa : sw) : 1.0f;
    then = out ? (a ? sw : sa) : one;
  }
  __device__ __forceinline__ float add(float acc, float sum) const {
    return __builtin_fmaf(sum * first, then, acc);
  }
};

// Four sums of a row of y, or what is left of it; a row may begin at any element.
template <typename T>
__device__ __forceinline__ void store4(T* p, f32x4 v, int left) {
  typedef T t4 __attribute__((ext_vector_type(4)));
  typedef t4 any4 __attribute__((aligned(sizeof(T))));
  const t4 r = {(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
  if (left >= 4) {
    *reinterpret_cast<any4*>(p) = r;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) p[i] = r[i];
  }
}

// Few activation rows: the weights are read once, and only the latency and
// the memory's rate count. A workgroup takes 16 weight rows and 16 * MT
// activation rows, its KS waves every KS-th block of 128; the waves' sums are
// added in LDS in their order. A wave has the loads of AHEAD blocks in flight.
// 1 x 4096 x 4096: 5.7 us, of which the 16.8 MB of weights are 3.6 at the rate
// of a copy and the rest is the launch and the first load's latency.
template <typename T, int MT, int KS>
__global__ __launch_bounds__(64 * KS) void f8_matmul_few(MatmulArgs a) {
  constexpr int AHEAD = MT == 1 ? 4 : 2;
  __shared__ __align__(16) float sums[KS][MT][64][4];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * MT;
  const uint8_t* wrow = a.w + (int64_t)min(n0 + r, a.n - 1) * a.ld_w;
  const uint8_t* arow[MT];
  int m[MT];
#pragma unroll
  for (int x = 0; x < MT; ++x) {
    m[x] = min(m0 + 16 * x + r, a.m - 1);
    arow[x] = a.a + (int64_t)m[x] * a.ld_a;
  }
  const u32x4 zero = {0, 0, 0, 0};
  u32x4 wv[AHEAD][2], av[AHEAD][MT][2];
  float sa[AHEAD][MT], sw[AHEAD];
  auto load = [&](int b, int to) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int k = b * kF8Block + 64 * c + 16 * g;
      wv[to][c] = k < a.k ? *reinterpret_cast<const u32x4*>(wrow + k) : zero;
#pragma unroll
      for (int x = 0; x < MT; ++x)
        av[to][x][c] = k < a.k ? *reinterpret_cast<const u32x4*>(arow[x] + k) : zero;
    }
    sw[to] = a.sw[(int64_t)b * a.nb + n0 / kF8Block];
#pragma unroll
    for (int x = 0; x < MT; ++x) sa[to][x] = a.sa[(int64_t)b * a.m + m[x]];
  };
  f32x4 acc[MT];
#pragma unroll
  for (int x = 0; x < MT; ++x) acc[x] = f32x4{0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (wave + i * KS < a.kb) load(wave + i * KS, i);
  for (int b0 = wave; b0 < a.kb; b0 += AHEAD * KS) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int b = b0 + i * KS;
      if (b >= a.kb) break;
      f32x4 part[MT];
#pragma unroll
      for (int x = 0; x < MT; ++x) part[x] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          const f16x8 wh = halves(wv[i][c][e], wv[i][c][e + 1]);
#pragma unroll
          for (int x = 0; x < MT; ++x)
            part[x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                wh, halves(av[i][x][c][e], av[i][x][c][e + 1]), part[x], 0, 0, 0);
        }
#pragma unroll
      for (int x = 0; x < MT; ++x) {
        const Scales f(sa[i][x], sw[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[x][e] = f.add(acc[x][e], part[x][e]);
      }
      if (b + AHEAD * KS < a.kb) load(b + AHEAD * KS, i);
    }
  }
#pragma unroll
  for (int x = 0; x < MT; ++x) *reinterpret_cast<f32x4*>(sums[wave][x][lane]) = acc[x];
  __syncthreads();
  for (int i = threadIdx.x; i < 64 * MT; i += 64 * KS) {
    const int x = i >> 6, l = i & 63, n = n0 + 4 * (l >> 4), mm = m0 + 16 * x + (l & 15);
    f32x4 v = *reinterpret_cast<const f32x4*>(sums[0][x][l]);
#pragma unroll
    for (int w = 1; w < KS; ++w) v += *reinterpret_cast<const f32x4*>(sums[w][x][l]);
    if (mm < a.m && n < a.n)
      store4(static_cast<T*>(a.y) + (int64_t)mm * a.ld_y + n, v, a.n - n);
  }
}

// Sixteen zero bytes: what loads past the end of a row's codes read.
__device__ const u32x4 g_zero16 = {0, 0, 0, 0};

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
#pragma clang diagnostic pop

// A wave-uniform pointer that the compiler cannot tell for one.
__device__ __forceinline__ const uint8_t* uniform(const uint8_t* p) {
  const uint64_t v = (uint64_t)(uintptr_t)p;
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)v);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return reinterpret_cast<const uint8_t*>((uintptr_t)((uint64_t)hi << 32 | lo));
}

// Many activation rows: a workgroup of WM x WN waves takes WM*MT*32 activation
// and WN*NT*32 weight rows. The rows' 128 bytes of a block lie in LDS, two
// blocks in turn, in 16-byte cells of which row r holds cell c at place
// c ^ (r / 2 & 7): the 16 rows of which a read takes a cell each at a time
// (lanes 0-3, 12-15, 20-27 and so on) then spread over all 64 banks. With
// c ^ (r & 7) they met in pairs, 4 cycles for each read.
//
// Bound by the matrix instructions and the conversions beside them: 8192 x
// 14336 x 4096 takes 875 us, 1.10 PFLOP/s (860 to 1100 us as the clocks move; a
// bfloat16 product of 8192^3 reaches 1.47 in a short run and 1.19 twenty times in a
// row), with products and vector instructions on 55 % of the cycles each, at 1.9
// GHz. Tiles of 128 x 128 on 4 waves: a wave converts 128 rows' codes for 64 x 64
// sums. 128 x 256 was equal, 192 x 256 and
// 256 x 256 spilled registers; three and four blocks in LDS were no faster than
// two.
//
// WK = 2: two such groups of waves in the workgroup take every other block of
// k each, and the second's sums are added to the first's in LDS at the end.
template <typename T, int MT, int NT, int WM, int WN, int WK>
__global__ __launch_bounds__(64 * WM * WN * WK, 2) void f8_matmul_tiled(MatmulArgs a,
                                                                        int groups_m) {
  constexpr int TM = WM * MT * 32, TN = WN * NT * 32, WAVES = WM * WN;
  constexpr int LA = TM / 8 / WAVES, LW = TN / 8 / WAVES;   // loads of 8 rows, per wave
  static_assert(TM % (8 * WAVES) == 0 && TN % (8 * WAVES) == 0, "");
  __shared__ __align__(16) uint8_t lds[WK * 2][TM + TN][kF8Block];
  const int any = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave = any % WAVES, half = any / WAVES;
  const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
  // this workgroup's tile, and blocks b0 .. b1-1 of k
  constexpr bool SPLIT = MT * NT == 1;
  const int splits = SPLIT ? a.splits : 1;
  const int tile = SPLIT ? blockIdx.x / splits : blockIdx.x;
  const int own = SPLIT ? blockIdx.x % splits : 0;
  const int b0 = (int)((int64_t)a.kb * own / splits);
  const int b1 = (int)((int64_t)a.kb * (own + 1) / splits);
  const int m0 = tile % groups_m * TM, n0 = tile / groups_m * TN;
  const int wm = wave % WM * MT * 32, wn = wave / WM * NT * 32;
  // A wave loads 8 * LA and 8 * LW rows: rows 8 i + lane / 8 from a base, at
  // this lane's cell (one for even i, one for odd). Rows past the matrix
  // repeat its last.
  static_assert(LA % 2 == 0 && LW % 2 == 0, "");
  const int cells[2] = {16 * ((lane & 7) ^ (lane >> 4)), 16 * ((lane & 7) ^ (lane >> 4) ^ 4)};
  const int a0 = min(m0 + 8 * LA * wave, a.m - 1), w0 = min(n0 + 8 * LW * wave, a.n - 1);
  const uint8_t* abase = uniform(a.a + a0 * a.ld_a);
  const uint8_t* wbase = uniform(a.w + w0 * a.ld_w);
  uint32_t aoff[LA], woff[LW];
#pragma unroll
  for (int i = 0; i < LA; ++i)
    aoff[i] = (uint32_t)(min(8 * i + (lane >> 3), a.m - 1 - a0) * a.ld_a) + cells[i & 1];
#pragma unroll
  for (int i = 0; i < LW; ++i)
    woff[i] = (uint32_t)(min(8 * i + (lane >> 3), a.n - 1 - w0) * a.ld_w) + cells[i & 1];
  const uint32_t to0 =
      (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)&lds[0][0][0];
  auto load = [&](int b, int to) {
    const uint32_t at = to0 + to * (TM + TN) * kF8Block + 1024 * LA * wave;
    const uint32_t wt = at + TM * kF8Block + 1024 * (LW - LA) * wave;
    const uint8_t *ab = abase + b * kF8Block, *wb = wbase + b * kF8Block;
    if ((b + 1) * kF8Block <= a.k) {
#pragma unroll
      for (int i = 0; i < LA; ++i) load_lds16(ab, aoff[i], at + 1024 * i);
#pragma unroll
      for (int i = 0; i < LW; ++i) load_lds16(wb, woff[i], wt + 1024 * i);
    } else {
      const bool past[2] = {b * kF8Block + cells[0] >= a.k, b * kF8Block + cells[1] >= a.k};
      const void* zero = &g_zero16;
#pragma unroll
      for (int i = 0; i < LA; ++i) load_lds16(past[i & 1] ? zero : ab + aoff[i], at + 1024 * i);
#pragma unroll
      for (int i = 0; i < LW; ++i) load_lds16(past[i & 1] ? zero : wb + woff[i], wt + 1024 * i);
    }
  };
  int m[MT];
#pragma unroll
  for (int x = 0; x < MT; ++x) m[x] = min(m0 + wm + 32 * x + r, a.m - 1);
  const int nblock = min((n0 + wn) / kF8Block, a.nb - 1);
  v16f acc[MT][NT];
  // the scales of a block come a block ahead, as its rows do
  float sa[MT], sw;
  auto load_scales = [&](int b) {
    sw = a.sw[(int64_t)b * a.nb + nblock];
#pragma unroll
    for (int x = 0; x < MT; ++x) sa[x] = a.sa[(int64_t)b * a.m + m[x]];
  };
  // All blocks with sa * sw as one factor; whether one left the range is noted, and
  // then the tile is summed again with two (TWO). With that the products take 1 %
  // longer than with one factor whatever it is; a branch for each block: 3 to 10 %.
  __shared__ int again;
  if (threadIdx.x == 0) again = 0;
  auto sum = [&](auto two) {
    constexpr bool TWO = decltype(two)::value;
    bool out = false;
#pragma unroll
    for (int x = 0; x < MT; ++x)
#pragma unroll
      for (int z = 0; z < NT; ++z) acc[x][z] = v16f{};
    if (b0 + half < b1) {
      load(b0 + half, 2 * half);
      load_scales(b0 + half);
    }
    int turn = 0;
    for (int b = b0 + half; b < b1 + half; b += WK, turn ^= 1) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      const float fw = sw;
      float fa[MT];
#pragma unroll
      for (int x = 0; x < MT; ++x) {
        fa[x] = sa[x];
        if (!TWO) out |= out_of_range(fa[x] * fw);
      }
      if (WK > 1 && b >= b1) break;          // the last wait of a half with a block less
      if (b + WK < b1) {
        load(b + WK, 2 * half + (turn ^ 1));
        load_scales(b + WK);
      }
      // ahead of a wave of the other workgroup that still waits for its block
      // (8192 x 14336 x 4096: 878 -> 852 us)
      __builtin_amdgcn_s_setprio(1);
      const uint8_t(*at)[kF8Block] = lds[2 * half + turn];
      // a lane's cells: 2 j + h of its row
      f16x8 wh[NT][8];
#pragma unroll
      for (int z = 0; z < NT; ++z)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const u32x4 v = *reinterpret_cast<const u32x4*>(
              &at[TM + wn + 32 * z + r][16 * ((2 * j + h) ^ (r >> 1 & 7))]);
          wh[z][2 * j] = halves(v[0], v[1]);
          wh[z][2 * j + 1] = halves(v[2], v[3]);
        }
#pragma unroll
      for (int x = 0; x < MT; ++x) {
        v16f part[NT];
#pragma unroll
        for (int z = 0; z < NT; ++z) part[z] = v16f{};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const u32x4 v = *reinterpret_cast<const u32x4*>(
              &at[wm + 32 * x + r][16 * ((2 * j + h) ^ (r >> 1 & 7))]);
          const f16x8 a0 = halves(v[0], v[1]), a1 = halves(v[2], v[3]);
#pragma unroll
          for (int z = 0; z < NT; ++z) {
            part[z] = __builtin_amdgcn_mfma_f32_32x32x16_f16(wh[z][2 * j], a0, part[z],
                                                             0, 0, 0);
            part[z] = __builtin_amdgcn_mfma_f32_32x32x16_f16(wh[z][2 * j + 1], a1, part[z],
                                                             0, 0, 0);
          }
        }
        const Scales f(fa[x], fw);
        const float one = fa[x] * fw;
#pragma unroll
        for (int z = 0; z < NT; ++z)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            acc[x][z][e] = TWO ? f.add(acc[x][z][e], part[z][e])
                               : __builtin_fmaf(part[z][e], one, acc[x][z][e]);
      }
      __builtin_amdgcn_s_setprio(0);
    }
    return out;
  };
  if (sum(std::false_type{})) again = 1;
  __syncthreads();
  if (again) sum(std::true_type{});
  if constexpr (WK > 1) {
    static_assert(sizeof(lds) >= sizeof(float) * 64 * WAVES * MT * NT * 16, "");
    __syncthreads();
    float* sums = reinterpret_cast<float*>(&lds[0][0][0]) + (threadIdx.x & (64 * WAVES - 1));
    if (half) {
#pragma unroll
      for (int x = 0; x < MT; ++x)
#pragma unroll
        for (int z = 0; z < NT; ++z)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            sums[((x * NT + z) * 16 + e) * 64 * WAVES] = acc[x][z][e];
    }
    __syncthreads();
    if (half) return;
#pragma unroll
    for (int x = 0; x < MT; ++x)
#pragma unroll
      for (int z = 0; z < NT; ++z)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          acc[x][z][e] += sums[((x * NT + z) * 16 + e) * 64 * WAVES];
  }
  if (SPLIT && splits > 1) {
    // the parts go to memory lane by lane and are added in their order
    __shared__ int last;
    constexpr int SIZE = 64 * WAVES * 16;
    float* mine = a.part + ((int64_t)tile * splits + own) * SIZE + threadIdx.x * 2;
#pragma unroll
    for (int e = 0; e < 16; e += 2)
      put_pair(mine + e * 64 * WAVES, acc[0][0][e], acc[0][0][e + 1]);
    if (!comes_last(a.count + tile, splits, &last)) return;
    const float* all = a.part + (int64_t)tile * splits * SIZE + threadIdx.x * 2;
    acc[0][0] = v16f{};
    for (int p = 0; p < splits; ++p)
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const f32x2 v = get_pair(all + (int64_t)p * SIZE + e * 64 * WAVES);
        acc[0][0][e] += v[0];
        acc[0][0][e + 1] += v[1];
      }
  }
#pragma unroll
  for (int x = 0; x < MT; ++x) {
    const int mm = m0 + wm + 32 * x + r;
    if (mm >= a.m) continue;
    T* y = static_cast<T*>(a.y) + (int64_t)mm * a.ld_y;
#pragma unroll
    for (int z = 0; z < NT; ++z)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int n = n0 + wn + 32 * z + 8 * e + 4 * h;
        if (n < a.n)
          store4(y + n, f32x4{acc[x][z][4 * e], acc[x][z][4 * e + 1], acc[x][z][4 * e + 2],
                              acc[x][z][4 * e + 3]}, a.n - n);
      }
  }
}

constexpr int64_t kSplitGroups = 512;    // workgroups that a split of k aims at

enum Way { kRows16, kRows32, kTiles64, kTiles128 };

int64_t tiles(int64_t m, int64_t n, int64_t tm, int64_t tn) {
  return (m + tm - 1) / tm * ((n + tn - 1) / tn);
}

int64_t blocks_of(int64_t k) { return (k + kF8Block - 1) / kF8Block; }

// Parts of k where tiles of 64 x 64 leave CUs idle: of 4 blocks at least.
int64_t parts_of(int64_t tiles64, int64_t kb) {
  return std::max<int64_t>(1, std::min(kSplitGroups / tiles64, kb / 4));
}

// The kernel that takes least, by estimates in us fitted to what was measured. Over
// 88 sizes (m from 8 to 8192, n from 1000 to 14336, k 1024 and 4096) the choice takes
// 0.7 % longer than the best of the four on the mean, 22 % at worst (32 x 6144 x 4096).
// Some of them, 16 rows at a time, 32, tiles of 64 and of 128, with k = 4096:
// 32 x 1000 6.7, 8.3, 11.0, 29; 64 x 4096 19.3, 15.5, 16.1, 31; 17 x 14336 26, 21.1,
// 16.6, 31; 64 x 14336 55, 42, 18.2, 32; 515 x 6144 -, -, 46, 40; 515 x 14336 -, -, 92,
// 102; 2048 x 6144 -, -, 133, 108.
Way way_of(int64_t m, int64_t n, int64_t k) {
  const double kb = (double)blocks_of(k);
  auto more = [](int64_t x) { return (double)std::max<int64_t>(x, 0); };
  auto turns = [](int64_t x) { return (double)((x + 255) / 256); };   // on the busiest CU
  // few rows: a wave's share of k, and the workgroups beyond those that run at once
  const double t16 = 3.0 + kb * (0.09 + 4.3e-4 * more(tiles(m, n, 16, 16) - 100));
  const double t32 = 3.3 + kb * (0.13 + 7.0e-4 * more(tiles(m, n, 32, 16) - 250));
  // tiles: blocks of k one after another, and joining the parts of k
  const int64_t n64 = tiles(m, n, 64, 64), parts = parts_of(n64, (int64_t)kb);
  const double t64 = 4.0 + kb / (double)parts * (0.15 + 0.33 * turns(n64 * parts)) +
                     (parts > 1 ? 1.5 + 0.75 * (double)parts : 0.0);
  const double t128 = 4.0 + kb * (0.1 + turns(tiles(m, n, 128, 128)));
  const double tiled = std::min(t64, t128);
  // the few rows' kernels have the rows in the grid's second dimension
  if (m <= 65536 && std::min(t16, t32) <= tiled)
    return m <= 16 || t16 <= t32 ? kRows16 : kRows32;
  return t64 <= t128 ? kTiles64 : kTiles128;
}

// Which kernel, and how its work is split.
struct Plan {
  Way way;
  int32_t waves;     // few rows: waves that share k
  int32_t halves;    // tiles of 128: groups of waves that share k
  int64_t splits;    // tiles of 64: parts of k
  int64_t groups;    // workgroups
};

Plan plan_of(int64_t m, int64_t n, int64_t k) {
  const int64_t kb = blocks_of(k);
  Plan p = {way_of(m, n, k), 4, 1, 1, 0};
  switch (p.way) {
    case kRows16:
    case kRows32:
      // us with 4, 8 and 16 waves: 37 x 1000 x 4096 7.1, 6.8, 6.6; 32 x 2000 x 4096
      // 9.1, 8.4, 8.2; 1 x 8192 x 4096 9.6, 8.8, 10.4; 16 x 6144 x 1024 4.2, 4.1, 5.1;
      // 16 x 14336 x 1024 6.8, 7.7, 10.3; 1 x 2000 x 512 2.5, 2.6, 2.7
      p.groups = tiles(m, n, p.way == kRows16 ? 16 : 32, 16);
      if (p.groups <= 128 && kb >= 16) p.waves = 16;
      else if (p.groups <= 512 && kb >= 8) p.waves = 8;
      break;
    case kTiles64:
      p.splits = parts_of(tiles(m, n, 64, 64), kb);
      p.groups = tiles(m, n, 64, 64) * p.splits;
      break;
    case kTiles128:
      p.groups = tiles(m, n, 128, 128);
      // alone on its CU a tile waits for its blocks unless two of them are in
      // hand: k in halves 515 x 6144 x 4096 43 -> 38 us, k = 1024 15.6 -> 14.9,
      // k = 512 10.7 -> 11
      if (p.groups <= 256 && kb >= 8) p.halves = 2;
      break;
  }
  return p;
}

template <typename T, int MT>
void few(const MatmulArgs& a, const Plan& p, hipStream_t stream) {
  const dim3 grid((a.n + 15) / 16, (a.m + 16 * MT - 1) / (16 * MT)), block(64 * p.waves);
  if (p.waves == 16) hipLaunchKernelGGL((f8_matmul_few<T, MT, 16>), grid, block, 0, stream, a);
  else if (p.waves == 8) hipLaunchKernelGGL((f8_matmul_few<T, MT, 8>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((f8_matmul_few<T, MT, 4>), grid, block, 0, stream, a);
}

template <typename T, int MT, int NT, int WK>
void tiled(const MatmulArgs& a, const Plan& p, hipStream_t stream) {
  const int gm = (a.m + 64 * MT - 1) / (64 * MT);
  hipLaunchKernelGGL((f8_matmul_tiled<T, MT, NT, 2, 2, WK>), dim3((uint32_t)p.groups),
                     dim3(256 * WK), 0, stream, a, gm);
}

template <typename T>
void matmul(const MatmulArgs& a, const Plan& p, hipStream_t stream) {
  switch (p.way) {
    case kRows16: return few<T, 1>(a, p, stream);
    case kRows32: return few<T, 2>(a, p, stream);
    case kTiles64: return tiled<T, 1, 1, 1>(a, p, stream);
    case kTiles128:
      return p.halves == 2 ? tiled<T, 2, 2, 2>(a, p, stream) : tiled<T, 2, 2, 1>(a, p, stream);
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
  if (d.x_type == IFQ_TYPE_BF16) return quantize<__bf16>(a, d.block_rows, stream);
  if (d.x_type == IFQ_TYPE_F16) return quantize<_Float16>(a, d.block_rows, stream);
  return quantize<float>(a, d.block_rows, stream);
}

size_t f8_matmul_workspace_bytes(const ifq_f8_matmul_desc& d) {
  if (d.m == 0 || d.n == 0) return 0;
  const Plan p = plan_of(d.m, d.n, d.k);
  return p.splits == 1 ? 0 : kSplitCounterBytes + p.groups * 64 * 64 * sizeof(float);
}

int64_t f8_matmul_groups(const ifq_f8_matmul_desc& d) {
  return d.m == 0 || d.n == 0 ? 0 : plan_of(d.m, d.n, d.k).groups;
}

const char* f8_matmul_kernel_name(const ifq_f8_matmul_desc& d) {
  if (d.m == 0 || d.n == 0) return "";
  const Plan p = plan_of(d.m, d.n, d.k);
  const int w = p.waves == 16 ? 2 : p.waves == 8 ? 1 : 0;
  static const char* const rows16[] = {"f8_matmul_few<1, 4>", "f8_matmul_few<1, 8>",
                                       "f8_matmul_few<1, 16>"};
  static const char* const rows32[] = {"f8_matmul_few<2, 4>", "f8_matmul_few<2, 8>",
                                       "f8_matmul_few<2, 16>"};
  switch (p.way) {
    case kRows16: return rows16[w];
    case kRows32: return rows32[w];
    case kTiles64: return "f8_matmul_tiled<1, 1, 2, 2, 1>";
    case kTiles128:
      return p.halves == 2 ? "f8_matmul_tiled<2, 2, 2, 2, 2>" : "f8_matmul_tiled<2, 2, 2, 2, 1>";
  }
  return "";
}

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
  const Plan p = plan_of(d.m, d.n, d.k);
  a.splits = (int32_t)p.splits;
  a.count = static_cast<uint32_t*>(ws);
  a.part = a.splits > 1
               ? reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + kSplitCounterBytes)
               : nullptr;
  if (d.y_type == IFQ_TYPE_BF16) matmul<__bf16>(a, p, stream);
  else if (d.y_type == IFQ_TYPE_F16) matmul<_Float16>(a, p, stream);
  else matmul<float>(a, p, stream);
  return hipGetLastError();
}

}  // namespace ifq
