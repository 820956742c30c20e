// Few rows of activations times 4-bit weights, out = act(in_act(x) w^T + bias), with the activations in full precision.
//
// The weights are dequantised in registers to bf16, which holds every 4-bit value under its power of two exactly, and go to
// v_mfma_f32_16x16x32_bf16 as the first operand: lane 16 q + i has row i's columns 32 q to 32 q + 31 of a column tile, 16 bytes in one load, and the
// order of columns inside a product is free as long as both operands have the same.  The activations are the second operand as sums of
// bf16 numbers, of which bf16 values take one, fp16 values two and fp32 values (and everything behind an activation) three: cut off after eight
// bits each, they are exact.  The parts of up to 16 rows lie side by side in the instruction's columns, which few rows would leave empty, so
// every product is exact and only the accumulation rounds.
//
// Bound: the weights' bytes, or the latency of a launch and a few trips to memory.
#include <algorithm>
#include <type_traits>

#include "svg_kv4.h"

namespace svg {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 8;
constexpr int kRowsAtATime = 16;
constexpr int kLds = 64 * 1024;          // of the activations; the sums take their place afterwards

struct RowsArgs {
  Tokens x_tok, out_tok;
  const void* x;
  void* out;
  const unsigned char* w;
  const unsigned* ws;
  const float* bias;
  int M, N, K;
  int kt, kg;                            // column tiles of K, and groups of four
  int n_tiles;                           // row tiles of w
  int m_each, parts;                     // rows of x in a launch's third dimension; bf16 numbers a value
  int chunk;                             // column tiles whose activations are in LDS at a time
  int in_activation, activation;
};

// Elements of token row m / column n from the first.
__device__ __forceinline__ size_t row_at(const Tokens& t, unsigned m) {
  const unsigned b = m / (unsigned)t.N;
  return (size_t)b * t.sb + (size_t)(m - b * (unsigned)t.N) * t.sn;
}
__device__ __forceinline__ size_t column_at(const Tokens& t, unsigned n) {
  const unsigned h = n / (unsigned)t.D;
  return (size_t)h * t.sh + (n - h * (unsigned)t.D);
}

// The eight weights of a word of codes under a power of two.
__device__ __forceinline__ block_bf16x8 weights8(unsigned code, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1),
               c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3);
  return block_bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A workgroup takes RT row tiles of the weights; its wavefronts share the columns and add up through LDS in the order of their number.
// CB: blocks of 16 columns of the instruction that the rows' parts take.
template <int TYPE, int RT, int CB>
__global__ __launch_bounds__(64 * kWaves) void rows_kernel(RowsArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  block_u32x4* const xs = reinterpret_cast<block_u32x4*>(lds);       // [column tile][step][q][column] pieces of eight
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i = lane & 15, q = lane >> 4;
  const int tile0 = blockIdx.x * RT;
  const int m0 = blockIdx.y * a.m_each;
  const int rows = min(a.m_each, a.M - m0), cols = rows * a.parts;

  const unsigned char* wp[RT];
  const unsigned* sp[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int tile = min(tile0 + r, a.n_tiles - 1);
    wp[r] = a.w + (size_t)tile * a.kt * kFp4Tile + lane * 16;
    sp[r] = a.ws + (size_t)tile * a.kg * 64 + lane;
  }
  int column[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) column[c] = min(16 * c + i, cols - 1);      // (columns that do not exist repeat the last one)
  f32x4 acc[RT][CB] = {};

  for (int k0 = 0; k0 < a.kt; k0 += a.chunk) {
    const int tiles = min(a.chunk, a.kt - k0);
    // this wavefront's column tiles of the chunk, and the first weights on their way before the activations are looked at
    const int first = k0 + tiles * wave / kWaves, last = k0 + tiles * (wave + 1) / kWaves;
    block_u32x4 codes[RT];
    unsigned scales[RT];
    auto load = [&](int k) {
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        codes[r] = __builtin_nontemporal_load(reinterpret_cast<const block_u32x4*>(wp[r] + (size_t)k * kFp4Tile));
        scales[r] = sp[r][(size_t)(k >> 2) * 64] >> (8 * (k & 3));
      }
    };
    if (first < last) load(first);
    if (k0 > 0) __syncthreads();
    // activations of the chunk: eight neighbouring columns of a row at a time
    const int runs = tiles * 16;
    for (int u = tid; u < runs * rows; u += 64 * kWaves) {
      const int m = u / runs, p = u - m * runs;           // piece p: columns 8 p .. of the chunk
      const int k = k0 * kFp4Cols + 8 * p;
      float v[8] = {};
      const size_t base = row_at(a.x_tok, (unsigned)(m0 + m));
      if (k + 8 <= a.K && (a.x_tok.D % 8 == 0 || a.x_tok.D == a.K)) {
        load8_any<TYPE>(a.x, base + column_at(a.x_tok, (unsigned)k), v);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (k + e < a.K) v[e] = load1<TYPE>(a.x, base + column_at(a.x_tok, (unsigned)(k + e)));
      }
      if (a.in_activation != SVG_ACT_NONE) activate8(v, a.in_activation);      // (act(0) = 0)
      // piece p of a tile: q = p / 4, step p % 4
      block_u32x4* const to = xs + ((size_t)((p >> 4) * 4 + (p & 3)) * 4 + ((p >> 2) & 3)) * cols + m * a.parts;
      for (int part = 0; part < a.parts; ++part) {
        block_u32x4 bits;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const unsigned lo = __float_as_uint(v[2 * e]), hi = __float_as_uint(v[2 * e + 1]);
          bits[e] = (lo >> 16) | (hi & 0xffff0000u);
        }
        to[part] = bits;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const unsigned u32 = __float_as_uint(v[e]);
          // what is left; an infinity or a NaN is whole in its first part
          v[e] = (u32 & 0x7f800000u) == 0x7f800000u ? 0.f : v[e] - __uint_as_float(u32 & 0xffff0000u);
        }
      }
    }
    __syncthreads();
    for (int k = first; k < last; ++k) {
      block_u32x4 now[RT];
      float scale[RT];
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        now[r] = codes[r];
        scale[r] = __uint_as_float((scales[r] & 255u) << 23);
      }
      if (k + 1 < last) load(k + 1);
      const block_u32x4* const from = xs + (size_t)(k - k0) * 16 * cols + q * cols;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        block_bf16x8 x[CB];
#pragma unroll
        for (int c = 0; c < CB; ++c) x[c] = __builtin_bit_cast(block_bf16x8, from[t * 4 * cols + column[c]]);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const block_bf16x8 w = weights8(now[r][t], scale[r]);
#pragma unroll
          for (int c = 0; c < CB; ++c) acc[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x[c], acc[r][c], 0, 0, 0);
        }
      }
    }
  }
  __syncthreads();
  // sums [wavefront][row tile][column][16 weights' rows]
  float* const sums = reinterpret_cast<float*>(lds);
  constexpr int SIZE = RT * CB * 256;
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int c = 0; c < CB; ++c) *reinterpret_cast<f32x4*>(sums + wave * SIZE + (r * CB + c) * 256 + i * 16 + 4 * q) = acc[r][c];
  __syncthreads();
  // eight neighbouring outputs a thread
  for (int u = tid; u < rows * RT * 2; u += 64 * kWaves) {
    const int m = u / (RT * 2), piece = u - m * (RT * 2);
    const int n = tile0 * 16 + 8 * piece;
    if (n >= a.N) continue;
    float v[8] = {};
    for (int part = a.parts - 1; part >= 0; --part) {      // the smallest first
      const int column = m * a.parts + part;
      const float* const from = sums + ((piece >> 1) * CB + (column >> 4)) * 256 + (column & 15) * 16 + 8 * (piece & 1);
      for (int w = 0; w < kWaves; ++w)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += from[w * SIZE + e];
    }
    if (a.bias)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += n + e < a.N ? a.bias[n + e] : 0.f;
    if (a.activation != SVG_ACT_NONE) activate8(v, a.activation);
    const size_t base = row_at(a.out_tok, (unsigned)(m0 + m));
    for (int e = 0; e < 8; ++e) {
      if (n + e >= a.N) break;
      const size_t at = base + column_at(a.out_tok, (unsigned)(n + e));
      float x = v[0];
#pragma unroll
      for (int y = 1; y < 8; ++y) x = y == e ? v[y] : x;
      if (a.out_tok.type == SVG_BF16) store1<SVG_BF16>(a.out, at, x);
      else if (a.out_tok.type == SVG_F16) store1<SVG_F16>(a.out, at, x);
      else store1<SVG_F32>(a.out, at, x);
    }
  }
}

}  // namespace

int launch_fp4_rows(const Tokens& x_tok, const void* x, int in_activation, long long M, int N, int K, const void* w, const void* w_scales,
                    const float* bias, int activation, const Tokens& out_tok, void* out, hipStream_t stream) {
  RowsArgs a = {};
  a.x_tok = x_tok;
  a.out_tok = out_tok;
  a.x = x;
  a.out = out;
  a.w = static_cast<const unsigned char*>(w);
  a.ws = static_cast<const unsigned*>(w_scales);
  a.bias = bias;
  a.M = (int)M;
  a.N = N;
  a.K = K;
  a.kt = (int)fp4_col_tiles(K);
  a.kg = (int)fp4_col_groups(K);
  a.n_tiles = (int)fp4_row_tiles(N);
  a.parts = in_activation != SVG_ACT_NONE || x_tok.type == SVG_F32 ? 3 : x_tok.type == SVG_F16 ? 2 : 1;
  a.m_each = (int)std::min<long long>(M, kRowsAtATime);
  a.in_activation = in_activation;
  a.activation = activation;
  const int cols = a.m_each * a.parts, blocks = (cols + 15) / 16;
  const int tile_bytes = cols * 256;                     // a column tile's activations in LDS
  a.chunk = std::max(1, std::min(a.kt, kLds / tile_bytes));
  const int rt = a.n_tiles >= 1024 && blocks < 3 ? 4 : a.n_tiles >= 512 ? 2 : 1;
  const int lds = std::max(a.chunk * tile_bytes, kWaves * rt * blocks * 1024);
  const dim3 grid((unsigned)((a.n_tiles + rt - 1) / rt), (unsigned)((M + a.m_each - 1) / a.m_each));
  (void)hipGetLastError();
  auto go = [&](auto type) {
    constexpr int TYPE = decltype(type)::value;
    auto with = [&](auto tiles) {
      constexpr int RT = decltype(tiles)::value;
      auto kernel = blocks == 1 ? rows_kernel<TYPE, RT, 1> : blocks == 2 ? rows_kernel<TYPE, RT, 2> : rows_kernel<TYPE, RT, 3>;
      hipLaunchKernelGGL(kernel, grid, dim3(64 * kWaves), (size_t)lds, stream, a);
    };
    if (rt == 4) with(std::integral_constant<int, 4>{});
    else if (rt == 2) with(std::integral_constant<int, 2>{});
    else with(std::integral_constant<int, 1>{});
  };
  if (x_tok.type == SVG_F32) go(std::integral_constant<int, SVG_F32>{});
  else if (x_tok.type == SVG_F16) go(std::integral_constant<int, SVG_F16>{});
  else go(std::integral_constant<int, SVG_BF16>{});
  return hip_status(hipGetLastError());
}

}  // namespace svg
