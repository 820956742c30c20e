// Token matrices to and from microscaled 4-bit operands.  HBM-bound: 2 or 4 bytes an element in, 17/32 byte out.
//
// A lane takes eight neighbouring columns of a row (16 bytes of a 16-bit type), four neighbouring lanes one block of 32, so
// a wavefront reads 512 columns of a row in one run, the block's largest magnitude needs two lane moves
// and the codes of a lane are one word of the block's 16-byte piece.
#include <type_traits>

#include "svg_block.h"

namespace svg {

namespace {

struct QuantArgs {
  Tokens tok;
  const void* in;
  void* out;
  unsigned* codes;
  unsigned char* scales;
  long long rows;
  int cols, col_tiles, col_groups;
  int activation;
};

// One wavefront: a row tile's group of four column tiles.
template <int TYPE, bool VEC>
__global__ __launch_bounds__(256) void quantize_kernel(QuantArgs a) {
  const int lane = threadIdx.x & 63;
  const long long unit = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const long long rt = unit / a.col_groups;
  const int group = (int)(unit - rt * a.col_groups);
  if (rt * kFp4Rows >= a.rows) return;
  const int c0 = group * 512 + lane * 8;                 // this lane's columns
  const int ct = group * kFp4Group + (lane >> 4);        // their column tile
  const int g = (lane >> 2) & 3;                         // block of the tile
  const bool stored = ct < a.col_tiles;
  size_t col[8];
#pragma unroll
  for (int e = 0; e < (VEC ? 1 : 8); ++e) {
    const int c = c0 + e;
    col[e] = c < a.cols ? (size_t)(c / a.tok.D) * a.tok.sh + c % a.tok.D : 0;
  }
  for (int i = 0; i < kFp4Rows; ++i) {
    const long long row = rt * kFp4Rows + i;
    float v[8] = {};
    if (row < a.rows) {
      const long long b = row / a.tok.N;
      const size_t base = (size_t)b * a.tok.sb + (size_t)(row - b * a.tok.N) * a.tok.sn;
      if constexpr (VEC) {
        if (c0 < a.cols) load8<TYPE>(a.in, base + col[0], v);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c0 + e < a.cols) v[e] = load1<TYPE>(a.in, base + col[e]);
      }
      if (a.activation != SVG_ACT_NONE) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = activate(v[e], a.activation);      // act(0) = 0: the padding stays zero
      }
    }
    const unsigned scale = fp4_scale(quad_max(magnitude8(v)));
    if (stored) a.codes[((size_t)rt * a.col_tiles + ct) * 256 + g * 64 + i * 4 + (lane & 3)] = fp4_codes8(v, scale);
    if ((lane & 3) == 0) a.scales[(((size_t)rt * a.col_groups + group) * 64 + g * 16 + i) * 4 + (lane >> 4)] = (unsigned char)scale;
  }
}

template <int TYPE, bool VEC>
__global__ __launch_bounds__(256) void dequantize_kernel(QuantArgs a) {
  const int lane = threadIdx.x & 63;
  const long long unit = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const long long rt = unit / a.col_groups;
  const int group = (int)(unit - rt * a.col_groups);
  if (rt * kFp4Rows >= a.rows) return;
  const int c0 = group * 512 + lane * 8;
  const int ct = group * kFp4Group + (lane >> 4);
  const int g = (lane >> 2) & 3;
  if (c0 >= a.cols) return;
  size_t col[8];
#pragma unroll
  for (int e = 0; e < (VEC ? 1 : 8); ++e) {
    const int c = c0 + e;
    col[e] = c < a.cols ? (size_t)(c / a.tok.D) * a.tok.sh + c % a.tok.D : 0;
  }
  for (int i = 0; i < kFp4Rows; ++i) {
    const long long row = rt * kFp4Rows + i;
    if (row >= a.rows) return;
    const unsigned codes = a.codes[((size_t)rt * a.col_tiles + ct) * 256 + g * 64 + i * 4 + (lane & 3)];
    const unsigned scale = a.scales[(((size_t)rt * a.col_groups + group) * 64 + g * 16 + i) * 4 + (lane >> 4)];
    // code value times 2^(scale - 127) in two normal factors: the power itself may be subnormal
    const int half = (int)scale / 2;
    const float p = __uint_as_float((unsigned)(half + 64) << 23), q = __uint_as_float((unsigned)((int)scale - half + 63) << 23);
    float v[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const auto two = e == 0   ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 0)
                       : e == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 1)
                       : e == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 2)
                                : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 3);
      v[2 * e] = scale == 255u ? __builtin_nanf("") : two[0] * p * q;
      v[2 * e + 1] = scale == 255u ? __builtin_nanf("") : two[1] * p * q;
    }
    const long long b = row / a.tok.N;
    const size_t base = (size_t)b * a.tok.sb + (size_t)(row - b * a.tok.N) * a.tok.sn;
    if constexpr (VEC) {
      store8<TYPE>(a.out, base + col[0], v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c0 + e < a.cols) store1<TYPE>(a.out, base + col[e], v[e]);
    }
  }
}

template <bool QUANT>
int launch(const QuantArgs& a, bool vec, hipStream_t stream) {
  const long long units = fp4_row_tiles(a.rows) * a.col_groups;
  const long long blocks = (units + 3) / 4;
  if (blocks > 0xffffffll)                     // a launch has fewer than 2^32 threads
    return SVG_ERR_UNSUPPORTED;
  (void)hipGetLastError();
  auto go = [&](auto type) {
    constexpr int TYPE = decltype(type)::value;
    auto kernel = QUANT ? (vec ? quantize_kernel<TYPE, true> : quantize_kernel<TYPE, false>)
                        : (vec ? dequantize_kernel<TYPE, true> : dequantize_kernel<TYPE, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, stream, a);
  };
  if (a.tok.type == SVG_F32) go(std::integral_constant<int, SVG_F32>{});
  else if (a.tok.type == SVG_F16) go(std::integral_constant<int, SVG_F16>{});
  else go(std::integral_constant<int, SVG_BF16>{});
  return hip_status(hipGetLastError());
}

QuantArgs quant_args(const Tokens& t, long long rows, int cols, void* codes, void* scales) {
  QuantArgs a = {};
  a.tok = t;
  a.codes = static_cast<unsigned*>(codes);
  a.scales = static_cast<unsigned char*>(scales);
  a.rows = rows;
  a.cols = cols;
  a.col_tiles = (int)fp4_col_tiles(cols);
  a.col_groups = (int)fp4_col_groups(cols);
  return a;
}

}  // namespace

bool tokens_vectors(const Tokens& t, const void* x) {
  return t.D % 8 == 0 && t.sb % 8 == 0 && t.sn % 8 == 0 && t.sh % 8 == 0 && !misaligned16(x);
}

int launch_fp4_quantize(const Tokens& t, long long rows, int cols, const void* x, int activation, void* codes, void* scales,
                        hipStream_t stream) {
  QuantArgs a = quant_args(t, rows, cols, codes, scales);
  a.in = x;
  a.activation = activation;
  return launch<true>(a, tokens_vectors(t, x), stream);
}

int launch_fp4_dequantize(const Tokens& t, long long rows, int cols, const void* codes, const void* scales, void* x,
                          hipStream_t stream) {
  QuantArgs a = quant_args(t, rows, cols, const_cast<void*>(codes), const_cast<void*>(scales));
  a.out = x;
  return launch<false>(a, tokens_vectors(t, x), stream);
}

}  // namespace svg
