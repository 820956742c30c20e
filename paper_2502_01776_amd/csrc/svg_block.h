// Shared by the operators around the attention (gate + norm + modulation, microscaled 4-bit operands and products):
// element types, token matrices, the operand order of microscaled 4-bit matrices, sums over a wavefront.
#pragma once
#include <atomic>

#include "svg_internal.h"

namespace svg {

typedef unsigned block_u32x4 __attribute__((ext_vector_type(4)));
typedef float block_f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 block_bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 block_f16x8 __attribute__((ext_vector_type(8)));
typedef float block_f32x8 __attribute__((ext_vector_type(8)));

// ---- operand order ------------------------------------------------------------------------------------------------
// Piece 16 g + i of a tile holds row i, columns 32 g to 32 g + 31: what lane 16 g + i of a wavefront gives
// v_mfma_scale_f32_16x16x128_f8f6f4 as its 16 bytes, so one operand of one instruction is 1 KB in one run.
constexpr int kFp4Rows = 16;          // rows of a tile
constexpr int kFp4Cols = 128;         // columns of a tile
constexpr int kFp4Tile = 1024;        // bytes of a tile
constexpr int kFp4Group = 4;          // column tiles whose scale bytes share a word
__host__ __device__ inline long long fp4_row_tiles(long long rows) { return (rows + kFp4Rows - 1) / kFp4Rows; }
__host__ __device__ inline long long fp4_col_tiles(long long cols) { return (cols + 255) / 256 * 2; }
__host__ __device__ inline long long fp4_col_groups(long long cols) { return (fp4_col_tiles(cols) + kFp4Group - 1) / kFp4Group; }
inline size_t fp4_codes_bytes(long long rows, long long cols) { return (size_t)(fp4_row_tiles(rows) * fp4_col_tiles(cols)) * kFp4Tile; }
inline size_t fp4_scales_bytes(long long rows, long long cols) { return (size_t)(fp4_row_tiles(rows) * fp4_col_groups(cols)) * 256; }
constexpr long long kMaxTokenRows = 2147483584ll;      // 2^31 - 64
constexpr long long kMaxColumns = 1ll << 20;

// A token matrix after validation (svg_tokens_t).
struct Tokens {
  long long N;                  // tokens of one batch entry
  long long sb, sn, sh;         // strides in elements
  int D, type;
};

// Are runs of eight columns whole, contiguous and 16-byte aligned?
bool tokens_vectors(const Tokens& t, const void* x);

// Kernel launchers.  All arguments validated by the caller; rows > 0 except for the gradients.
// Has the call a form that writes 4-bit codes?
bool gate_norm_writes_codes(const svg_gate_norm_t& d, const void* x, const void* y, const void* r, const void* h);
int launch_gate_norm(const svg_gate_norm_t& d, const void* x, const void* y, void* r, void* h, void* codes, void* scales,
                     hipStream_t stream);
size_t gate_norm_workspace_bytes(const svg_gate_norm_t& d);
int launch_gate_norm_grad(const svg_gate_norm_t& d, const void* r, const void* y, const void* dr, const void* dh, void* dx, void* dy,
                          const svg_gate_norm_grads_t& grads, float* workspace, hipStream_t stream);
int launch_fp4_quantize(const Tokens& t, long long rows, int cols, const void* x, int activation, void* codes, void* scales,
                        hipStream_t stream);
int launch_fp4_dequantize(const Tokens& t, long long rows, int cols, const void* codes, const void* scales, void* x,
                          hipStream_t stream);
// Forms of a product: operands straight from memory for one, two (K over eight or four wavefronts) and four token tiles; output
// tiles of 64 x 128, 128 x 256 and 256 x 256.
enum class LinearForm : int { kRows1, kRows2Eight, kRows2, kRows4, kTiles64, kTiles128, kSquare };
// By row tiles of the tokens, pairs of column tiles of the output (of its whole operand where it is one) and column tiles of K.
LinearForm fp4_linear_form(long long m_tiles, long long pairs, int k_tiles, bool activation);
// tok and out, or codes and scales
int launch_fp4_linear(long long M, int N, int K, const void* a, const void* a_scales, const void* w, const void* w_scales,
                      const float* bias, int activation, const Tokens* tok, void* out, void* codes, void* scales,
                      hipStream_t stream);

// Lets a kernel take more than 64 KB of LDS; once for each GPU, because the call costs a microsecond.
inline hipError_t allow_lds(const void* kernel, int bytes, std::atomic<unsigned long long>& allowed) {
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess) return e;
  const unsigned long long bit = device < 64 ? 1ull << device : 0;
  if (allowed.load(std::memory_order_relaxed) & bit) return hipSuccess;
  e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) allowed.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

__host__ __device__ constexpr int type_bytes(int type) { return type == SVG_F32 ? 4 : 2; }

// ---- device helpers -------------------------------------------------------------------------------------------------
#if defined(__HIP_DEVICE_COMPILE__) || defined(__HIPCC__)

// One load of 16 bytes a lane from memory into LDS, lane l at lds_address + 16 l; as attn::load_to_lds, which takes two at a time.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_one_to_lds(const block_u32x4 rsrc, int voffset, int soffset, unsigned lds_address) {
  asm volatile("s_mov_b32 m0, %3\n\ts_nop 3\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds"
               :: "v"(voffset), "s"(rsrc), "s"(soffset), "s"(lds_address)
               : "memory", "m0");
}
#pragma clang diagnostic pop

// Sum and maximum over the 64 lanes, in all of them: inside the quarters by lane moves of the vector unit, over them by swaps.
template <class F>
__device__ __forceinline__ float wave_fold(float x, F f) {
  auto dpp = [](float v, auto ctrl) {
    return __uint_as_float((unsigned)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  x = f(x, dpp(x, std::integral_constant<int, 0x128>{}));      // rotated by 8, 4, 2 and 1 lanes inside the quarter
  x = f(x, dpp(x, std::integral_constant<int, 0x124>{}));
  x = f(x, dpp(x, std::integral_constant<int, 0x122>{}));
  x = f(x, dpp(x, std::integral_constant<int, 0x121>{}));
  const unsigned u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  x = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const unsigned w = __float_as_uint(x);
  const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float wave_sum(float x) {
  return wave_fold(x, [](float a, float b) { return a + b; });
}

// The larger of x over four neighbouring lanes, in all of them.
__device__ __forceinline__ unsigned quad_max(unsigned x) {
  x = max(x, (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0xb1, 0xf, 0xf, true));
  return max(x, (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x4e, 0xf, 0xf, true));
}

// Eight neighbouring elements from memory (16-byte aligned), as fp32.
template <int TYPE>
__device__ __forceinline__ void load8(const void* base, size_t element, float (&v)[8]) {
  if constexpr (TYPE == SVG_F32) {
    const block_f32x4* p = reinterpret_cast<const block_f32x4*>(static_cast<const float*>(base) + element);
    const block_f32x4 a = p[0], b = p[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
  } else if constexpr (TYPE == SVG_BF16) {
    const block_u32x4 a = *reinterpret_cast<const block_u32x4*>(static_cast<const unsigned short*>(base) + element);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(a[e] << 16);
      v[2 * e + 1] = __uint_as_float(a[e] & 0xffff0000u);
    }
  } else {
    const block_f16x8 a = *reinterpret_cast<const block_f16x8*>(static_cast<const unsigned short*>(base) + element);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)a[e];
  }
}
// From and to any element's address: the vector unit's loads and stores of 16 bytes need no alignment of their own.
typedef unsigned block_u32x4_of2 __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned block_u32x4_of4 __attribute__((ext_vector_type(4), aligned(4)));
template <int TYPE>
__device__ __forceinline__ void load8_any(const void* base, size_t element, float (&v)[8]) {
  if constexpr (TYPE == SVG_F32) {
    const block_u32x4_of4* p = reinterpret_cast<const block_u32x4_of4*>(static_cast<const float*>(base) + element);
    const block_u32x4 a = p[0], b = p[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = __uint_as_float(a[e]); v[4 + e] = __uint_as_float(b[e]); }
  } else {
    const block_u32x4 a = *reinterpret_cast<const block_u32x4_of2*>(static_cast<const unsigned short*>(base) + element);
    if constexpr (TYPE == SVG_BF16) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[2 * e] = __uint_as_float(a[e] << 16);
        v[2 * e + 1] = __uint_as_float(a[e] & 0xffff0000u);
      }
    } else {
      const block_f16x8 h = __builtin_bit_cast(block_f16x8, a);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (float)h[e];
    }
  }
}
// STREAM: rows that this launch does not look at again go past the caches.
template <int TYPE, bool STREAM = false>
__device__ __forceinline__ void store8_any(void* base, size_t element, const float (&v)[8]) {
  const block_f32x8 f = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
  auto put = [](const block_u32x4& x, auto* p) {
    if constexpr (STREAM) __builtin_nontemporal_store(x, p);
    else *p = x;
  };
  if constexpr (TYPE == SVG_F32) {
    block_u32x4_of4* p = reinterpret_cast<block_u32x4_of4*>(static_cast<float*>(base) + element);
    put(__builtin_bit_cast(block_u32x4, block_f32x4{v[0], v[1], v[2], v[3]}), p);
    put(__builtin_bit_cast(block_u32x4, block_f32x4{v[4], v[5], v[6], v[7]}), p + 1);
  } else {
    put(TYPE == SVG_BF16 ? __builtin_bit_cast(block_u32x4, __builtin_convertvector(f, block_bf16x8))
                         : __builtin_bit_cast(block_u32x4, __builtin_convertvector(f, block_f16x8)),
        reinterpret_cast<block_u32x4_of2*>(static_cast<unsigned short*>(base) + element));
  }
}
template <int TYPE>
__device__ __forceinline__ float load1(const void* base, size_t element) {
  if constexpr (TYPE == SVG_F32) return static_cast<const float*>(base)[element];
  else if constexpr (TYPE == SVG_BF16) return __uint_as_float((unsigned)static_cast<const unsigned short*>(base)[element] << 16);
  else return (float)static_cast<const _Float16*>(base)[element];
}
template <int TYPE>
__device__ __forceinline__ void store1(void* base, size_t element, float v) {
  if constexpr (TYPE == SVG_F32) static_cast<float*>(base)[element] = v;
  else if constexpr (TYPE == SVG_BF16) static_cast<__bf16*>(base)[element] = (__bf16)v;
  else static_cast<_Float16*>(base)[element] = (_Float16)v;
}

// silu(v) = v / (1 + e^-v);  the tanh form of GELU is v sigmoid(2 sqrt(2/pi) (v + 0.044715 v^3)).  The result is rounded next, to
// 16 or 4 bits mostly: base-2 exponential and reciprocal of the vector unit (one unit in the last place each).  The exponent's own rounding (its
// relative error is 1.3 x 2^-24 for silu, 7.3 x 2^-24 behind GELU's cubic) is an absolute one of the exponential's logarithm, so negative values far from zero are
// off by (1.3 |v| + 6) 2^-24 and (7.3 |z| + 6) 2^-24 of their size, positive ones by 8 x 2^-24.  The choice is made once for eight
// values: taken for each, its branches cost more than the arithmetic.
__device__ __forceinline__ void activate8(float (&v)[8], int activation) {
  constexpr float kLog2e = 1.4426950408889634f, kGelu = -1.5957691216057308f * kLog2e;
  auto gate = [](float x, float u) { return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u)); };
  if (activation == SVG_ACT_GELU_TANH) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = gate(v[e], v[e] * __builtin_fmaf(0.044715f * kGelu, v[e] * v[e], kGelu));
  } else if (activation == SVG_ACT_SILU) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = gate(v[e], -kLog2e * v[e]);
  }
}

// The bits of the largest magnitude of eight values; infinities and NaNs are above every finite value's.
__device__ __forceinline__ unsigned magnitude8(const float (&v)[8]) {
  unsigned m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(v[e]) & 0x7fffffffu);
  return m;
}
// The scale byte of a block whose largest magnitude has these bits: E + 127 with E = clamp(floor(log2) - 2, -127, 127).  The
// exponent field of a normal number is floor(log2) + 127; fields up to 2 (and subnormals) clamp to E = -127, 255 is infinity or NaN.
__device__ __forceinline__ unsigned fp4_scale(unsigned magnitude) {
  const unsigned field = magnitude >> 23;
  return field == 255u ? 255u : field > 2u ? field - 2u : 0u;
}
// Codes of eight values under a scale byte, the first in the lowest bits.  The conversion divides by the power of
// two in its scale operand's exponent field, rounds to nearest even and saturates.
__device__ __forceinline__ unsigned fp4_codes8(const float (&v)[8], unsigned scale) {
  const float s = __uint_as_float(scale << 23);
  unsigned c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], s, 3);
  return scale == 255u ? 0u : c;
}
#endif

}  // namespace svg
