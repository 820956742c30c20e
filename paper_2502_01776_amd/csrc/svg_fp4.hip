// Token matrices to and from microscaled 4-bit operands.  HBM-bound: 2 or 4 bytes an element in, 17/32 byte out.
//
// A workgroup takes a row tile's group of four column tiles, each wavefront four of its rows at once.  A lane takes eight
// neighbouring columns (16 bytes of a 16-bit type) of each, four neighbouring lanes one block of 32: a wavefront
// reads 512 columns of a row in one run and the block's largest magnitude needs two lane moves.  The four lanes' codes of four rows
// are a square of words whose transpose gives every lane the whole 16-byte piece of one row.
// bf16, 32760 x 5120 as 40 heads: written in 86 us (4.9 TB/s), read back in 64 us (6.6 TB/s).
#include <algorithm>
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

// Where a lane's eight columns are: its wavefront's rows are r0 to r0 + 3 of a row tile.
struct Place {
  long long rt;
  int group, c0, ct, g, r0, lane;
  __device__ __forceinline__ Place(const QuantArgs& a) : lane(threadIdx.x & 63) {
    const unsigned unit = blockIdx.y * gridDim.x + blockIdx.x;
    rt = unit / (unsigned)a.col_groups;                  // behind the last row tile where the grid has a ragged second dimension
    group = (int)(unit - (unsigned)rt * (unsigned)a.col_groups);
    c0 = group * 512 + lane * 8;
    ct = group * kFp4Group + (lane >> 4);                // column tile
    g = (lane >> 2) & 3;                                 // block of the tile
    r0 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 4;
  }
  __device__ __forceinline__ long long row(int k) const { return rt * kFp4Rows + r0 + k; }
  // the piece of row k, in pieces of a tile
  __device__ __forceinline__ int piece(int k) const { return g * 16 + r0 + k; }
  __device__ __forceinline__ size_t code_words(const QuantArgs& a) const {
    return ((size_t)rt * a.col_tiles + ct) * 256 + piece(lane & 3) * 4;
  }
  __device__ __forceinline__ size_t scale_word(const QuantArgs& a) const { return ((size_t)rt * a.col_groups + group) * 64 + piece(lane & 3); }
};

// Elements from the first to row m's, and to a lane's columns.  RUNS: eight of them are neighbours wherever they all exist.
__device__ __forceinline__ size_t row_at(const QuantArgs& a, long long m) {
  const unsigned row = (unsigned)m, b = row / (unsigned)a.tok.N;
  return (size_t)b * a.tok.sb + (size_t)(row - b * (unsigned)a.tok.N) * a.tok.sn;
}
template <bool RUNS>
struct Columns {
  size_t at[RUNS ? 1 : 8];
  int here;                                              // how many exist
  __device__ __forceinline__ Columns(const QuantArgs& a, int c0) : here(a.cols - c0) {
#pragma unroll
    for (int e = 0; e < (RUNS ? 1 : 8); ++e) {
      const unsigned c = c0 + e, h = c / (unsigned)a.tok.D;
      at[e] = e < here ? (size_t)h * a.tok.sh + (c - h * (unsigned)a.tok.D) : 0;
    }
  }
  __device__ __forceinline__ size_t of(int e) const { return RUNS ? at[0] + e : at[RUNS ? 0 : e]; }
};

// w[r] of lane j in a quad -> w[j'] of lane r: word k of lane j becomes word j of lane k.
__device__ __forceinline__ void transpose_quads(unsigned (&w)[4]) {
  const int lane = threadIdx.x;
  auto exchange = [](unsigned& a, unsigned& b, bool odd, auto ctrl) {
    const unsigned got = (unsigned)__builtin_amdgcn_mov_dpp((int)(odd ? a : b), decltype(ctrl)::value, 0xf, 0xf, true);
    if (odd) a = got;
    else b = got;
  };
  using Next = std::integral_constant<int, 0xb1>;        // lanes 1, 0, 3, 2
  using Far = std::integral_constant<int, 0x4e>;         // lanes 2, 3, 0, 1
  exchange(w[0], w[1], lane & 1, Next{});
  exchange(w[2], w[3], lane & 1, Next{});
  exchange(w[0], w[2], lane & 2, Far{});
  exchange(w[1], w[3], lane & 2, Far{});
}

template <int TYPE, bool RUNS>
__global__ __launch_bounds__(256) void quantize_kernel(QuantArgs a) {
  const Place at(a);
  if (at.rt * kFp4Rows >= a.rows) return;
  const Columns<RUNS> col(a, at.c0);
  float v[4][8] = {};
#pragma unroll
  for (int k = 0; k < 4; ++k) {                          // all four rows' loads before the first use
    if (at.row(k) >= a.rows) continue;
    const size_t base = row_at(a, at.row(k));
    if (RUNS && col.here >= 8) {
      load8_any<TYPE>(a.in, base + col.of(0), v[k]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < col.here) v[k][e] = load1<TYPE>(a.in, base + col.of(e));
    }
  }
  if (a.activation != SVG_ACT_NONE) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (at.row(k) >= a.rows) break;                    // act(0) = 0: the padding stays zero
      activate8(v[k], a.activation);
    }
  }
  unsigned code[4], scale = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const unsigned s = fp4_scale(quad_max(magnitude8(v[k])));
    code[k] = fp4_codes8(v[k], s);
    if ((at.lane & 3) == k) scale = s;                   // a lane writes the scale of its own row
  }
  transpose_quads(code);
  if (at.ct < a.col_tiles)
    *reinterpret_cast<block_u32x4*>(a.codes + at.code_words(a)) = block_u32x4{code[0], code[1], code[2], code[3]};
  // the word of a piece: the bytes of four column tiles, which are 16 lanes apart
  scale <<= 8 * (at.lane >> 4);
  const auto x = __builtin_amdgcn_permlane16_swap(scale, scale, false, false);
  scale = x[0] | x[1];
  const auto y = __builtin_amdgcn_permlane32_swap(scale, scale, false, false);
  if (at.lane < 16) reinterpret_cast<unsigned*>(a.scales)[at.scale_word(a)] = y[0] | y[1];
}

template <int TYPE, bool RUNS>
__global__ __launch_bounds__(256) void dequantize_kernel(QuantArgs a) {
  const Place at(a);
  if (at.rt * kFp4Rows >= a.rows) return;
  const Columns<RUNS> col(a, at.c0);
  const bool there = at.ct < a.col_tiles;
  const block_u32x4 piece = there ? *reinterpret_cast<const block_u32x4*>(a.codes + at.code_words(a)) : block_u32x4{};
  const unsigned word = reinterpret_cast<const unsigned*>(a.scales)[at.scale_word(a)];
  unsigned code[4] = {piece[0], piece[1], piece[2], piece[3]};
  transpose_quads(code);
  const int mine = (int)(word >> (8 * (at.lane >> 4))) & 255;      // of the row of this lane's number in the quad
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int scale = k == 0   ? __builtin_amdgcn_mov_dpp(mine, 0x00, 0xf, 0xf, true)
                      : k == 1 ? __builtin_amdgcn_mov_dpp(mine, 0x55, 0xf, 0xf, true)
                      : k == 2 ? __builtin_amdgcn_mov_dpp(mine, 0xaa, 0xf, 0xf, true)
                               : __builtin_amdgcn_mov_dpp(mine, 0xff, 0xf, 0xf, true);
    if (at.row(k) >= a.rows) continue;
    // code value times 2^(scale - 127) in two normal factors: the power itself may be subnormal
    const int half = scale / 2;
    const float p = __uint_as_float((unsigned)(half + 64) << 23), q = __uint_as_float((unsigned)(scale - half + 63) << 23);
    float v[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const auto two = e == 0   ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[k], 1.0f, 0)
                       : e == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[k], 1.0f, 1)
                       : e == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[k], 1.0f, 2)
                                : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[k], 1.0f, 3);
      v[2 * e] = scale == 255 ? __builtin_nanf("") : two[0] * p * q;
      v[2 * e + 1] = scale == 255 ? __builtin_nanf("") : two[1] * p * q;
    }
    const size_t base = row_at(a, at.row(k));
    if (RUNS && col.here >= 8) {
      store8_any<TYPE>(a.out, base + col.of(0), v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < col.here) store1<TYPE>(a.out, base + col.of(e), v[e]);
    }
  }
}

template <bool QUANT>
int launch(const QuantArgs& a, hipStream_t stream) {
  const bool vec = a.tok.D == a.cols || a.tok.D % 8 == 0;
  const long long blocks = fp4_row_tiles(a.rows) * a.col_groups;
  if (blocks > 0x7fffffff) return SVG_ERR_UNSUPPORTED;         // more than the memory holds
  // a launch has fewer than 2^32 threads in one dimension
  const dim3 grid((unsigned)std::min(blocks, 1ll << 23), (unsigned)((blocks + (1ll << 23) - 1) >> 23));
  (void)hipGetLastError();
  auto go = [&](auto type) {
    constexpr int TYPE = decltype(type)::value;
    auto kernel = QUANT ? (vec ? quantize_kernel<TYPE, true> : quantize_kernel<TYPE, false>)
                        : (vec ? dequantize_kernel<TYPE, true> : dequantize_kernel<TYPE, false>);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a);
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
  return launch<true>(a, stream);
}

int launch_fp4_dequantize(const Tokens& t, long long rows, int cols, const void* codes, const void* scales, void* x,
                          hipStream_t stream) {
  QuantArgs a = quant_args(t, rows, cols, const_cast<void*>(codes), const_cast<void*>(scales));
  a.out = x;
  return launch<false>(a, stream);
}

}  // namespace svg
