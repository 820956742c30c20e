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
#include <atomic>
#include <type_traits>
#include <utility>

#include "svg_kv4.h"

namespace svg {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 8;
constexpr int kRowsAtATime = 16;
constexpr int kLds = 152 * 1024;         // of the activations at the most; the sums take their place afterwards

// f(0), f(1), .. f(N - 1) with constants.
template <class F, int... I>
__device__ __forceinline__ void each_of(F f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void each(F f) { each_of(f, std::make_integer_sequence<int, N>{}); }

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
  int m_each, parts;                     // rows of x in a launch's second dimension; bf16 numbers a value
  int chunk;                             // column tiles whose activations are in LDS at a time
  int in_activation, activation;
  bool x_runs, out_runs;                 // are eight columns neighbours wherever they all exist?
  bool x_plain;                          // rows of x one step apart, columns in one run
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

// A barrier for what was written to LDS; what is on its way to registers stays so.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <class F>
__device__ __forceinline__ void by_type(int type, F f) {
  if (type == SVG_BF16) f(std::integral_constant<int, SVG_BF16>{});
  else if (type == SVG_F16) f(std::integral_constant<int, SVG_F16>{});
  else f(std::integral_constant<int, SVG_F32>{});
}

// WK wavefronts share the columns of K, every WK-th column tile each, whatever is in LDS at a time and however many rows there are: a row's sums do not
// depend on the others.  They add up through LDS in the order of their number.  The workgroup's kWaves / WK such groups take RT row tiles of
// the weights each.  CB: blocks of 16 columns of the instruction that the rows' parts take.
// A wavefront asks for its first activations, then for its first DEPTH column tiles, and only then looks at the activations: silu, its parts and
// the trip to LDS lie behind the weights' way.  (Loads arrive in order: activations asked for behind the weights would be waited for with them.)
// Measured with weights out of memory: 4 x 20480 x 5120, silu in front and GELU behind, 14.4 us among others (3.9 TB/s; 17.3 by itself, three tiles ahead 18, four
// 19.9), of which the activations take 3; one row without them 13.7 by itself, 5120 x 5120 7.2, 5120 x 256 3.7.  One row tile to a workgroup instead of
// five: 16.9 for one row, 36 for four.
template <int RT, int CB, int WK, int DEPTH>
__global__ __launch_bounds__(64 * kWaves, 2) void rows_kernel(RowsArgs a) {
  constexpr int GROUPS = kWaves / WK, UNITS = DEPTH == 1 ? 1 : 5;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  block_u32x4* const xs = reinterpret_cast<block_u32x4*>(lds);       // [column tile][step][q][column] pieces of eight
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wk = wave % WK, group = wave / WK;
  const int i = lane & 15, q = lane >> 4;
  const int tile0 = blockIdx.x * (RT * GROUPS);
  const int m0 = blockIdx.y * a.m_each;
  const int rows = min(a.m_each, a.M - m0), cols = rows * a.parts;

  // A chunk's activations in runs of eight neighbouring columns, row after row: run tid, and on in steps of the workgroup, without a division each.
  struct Run {
    int m, p;                                            // row, number in the row
    __device__ __forceinline__ void step(int rows_on, int runs_on, int runs) {
      p += runs_on;
      m += rows_on;
      if (p >= runs) {
        p -= runs;
        ++m;
      }
    }
  };
  auto x_at = [&](int m, int col) {
    return a.x_plain ? (size_t)(m0 + m) * a.x_tok.sn + col : row_at(a.x_tok, (unsigned)(m0 + m)) + column_at(a.x_tok, (unsigned)col);
  };
  block_u32x4 early[UNITS][2] = {};
  const int first_runs = min(a.chunk, a.kt) * 16, rows_on = 64 * kWaves / first_runs, runs_on = 64 * kWaves - rows_on * first_runs;
  const Run first_run = {tid / first_runs, tid % first_runs};
  {
    Run x = first_run;
    each<UNITS>([&](auto j) {
      if (x.m < rows && a.x_runs && 8 * x.p + 8 <= a.K) {
        const char* const from = static_cast<const char*>(a.x) + x_at(x.m, 8 * x.p) * type_bytes(a.x_tok.type);
        early[j][0] = *reinterpret_cast<const block_u32x4_of2*>(from);
        if (a.x_tok.type == SVG_F32) early[j][1] = *reinterpret_cast<const block_u32x4_of2*>(from + 16);
      }
      x.step(rows_on, runs_on, first_runs);
    });
  }

  const unsigned char* wp[RT];
  const unsigned* sp[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int tile = min(tile0 + group * RT + r, a.n_tiles - 1);
    wp[r] = a.w + (size_t)tile * a.kt * kFp4Tile + lane * 16;
    sp[r] = a.ws + (size_t)tile * a.kg * 64 + lane;
  }
  // tiles wk, wk + WK, ..
  block_u32x4 codes[DEPTH][RT];
  unsigned scales[DEPTH][RT];
  auto load = [&](auto slot, int k) {
    k = min(k, a.kt - 1);                                // (behind the last one: not looked at)
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      codes[slot][r] = *reinterpret_cast<const block_u32x4*>(wp[r] + (size_t)k * kFp4Tile);
      scales[slot][r] = sp[r][(size_t)(k >> 2) * 64];
    }
  };
  each<DEPTH>([&](auto d) { load(d, wk + WK * d); });
  // what this thread writes in the end: eight neighbouring outputs of a row, 16 rows at most
  const int out_m = tid / (RT * GROUPS * 2), out_piece = tid - out_m * (RT * GROUPS * 2), out_n = tile0 * 16 + 8 * out_piece;
  const bool writes = out_m < rows && out_n < a.N;
  float bias[8] = {};
  if (writes && a.bias)
#pragma unroll
    for (int e = 0; e < 8; ++e) bias[e] = a.bias[min(out_n + e, a.N - 1)];
  int column[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) column[c] = min(16 * c + i, cols - 1);      // (columns that do not exist repeat the last one)
  f32x4 acc[RT][CB] = {};

  // a run's values behind the activation, in parts, into LDS
  auto put = [&](const Run& x, float (&v)[8]) {
    if (a.in_activation != SVG_ACT_NONE) activate8(v, a.in_activation);      // (act(0) = 0)
    // run p of a tile: q = p / 4, step p % 4
    block_u32x4* const to = xs + (((x.p >> 4) * 4 + (x.p & 3)) * 4 + ((x.p >> 2) & 3)) * cols + x.m * a.parts;
    for (int part = 0; part < a.parts; ++part) {
      block_u32x4 bits;
#pragma unroll
      for (int e = 0; e < 4; ++e) bits[e] = __builtin_amdgcn_perm(__float_as_uint(v[2 * e + 1]), __float_as_uint(v[2 * e]), 0x07060302u);
      to[part] = bits;
      // what is left (of an infinity NaN)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] -= __uint_as_float(__float_as_uint(v[e]) & 0xffff0000u);
    }
  };
  auto put_rest = [&](int k0, int tiles, bool behind_early) {
    const int runs = tiles * 16, on = 64 * kWaves / runs;
    Run x = {tid / runs, tid % runs};
    for (int j = 0; x.m < rows; ++j, x.step(on, 64 * kWaves - on * runs, runs)) {
      const int col = k0 * kFp4Cols + 8 * x.p;
      const bool whole = a.x_runs && col + 8 <= a.K;
      if (behind_early && j < UNITS && whole) continue;
      float v[8] = {};
      by_type(a.x_tok.type, [&](auto type) {
        constexpr int TYPE = decltype(type)::value;
        if (whole) {
          load8_any<TYPE>(a.x, x_at(x.m, col), v);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (col + e < a.K) v[e] = load1<TYPE>(a.x, x_at(x.m, col + e));
        }
      });
      put(x, v);
    }
  };
  // The first chunk's stand in front of the loop: inside, the compiler would wait for everything that is on its way.
  {
    Run x = first_run;
    each<UNITS>([&](auto j) {
      if (x.m < rows && a.x_runs && 8 * x.p + 8 <= a.K) {
        float v[8];
        if (a.x_tok.type == SVG_F32) {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(early[j][e / 4][e % 4]);
        } else if (a.x_tok.type == SVG_BF16) {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(e % 2 ? early[j][0][e / 2] & 0xffff0000u : early[j][0][e / 2] << 16);
        } else {
          const block_f16x8 h = __builtin_bit_cast(block_f16x8, early[j][0]);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = (float)h[e];
        }
        put(x, v);
      }
      x.step(rows_on, runs_on, first_runs);
    });
  }
  if (first_runs * rows > 64 * kWaves * UNITS || !a.x_runs || a.K < a.kt * kFp4Cols) put_rest(0, min(a.chunk, a.kt), true);
  lds_barrier();

  int k = wk;                                            // the next column tile
  for (int k0 = 0;;) {
    const int tiles = min(a.chunk, a.kt - k0);
    auto take = [&](auto slot) {
      const block_u32x4* const from = xs + (size_t)(k - k0) * 16 * cols + q * cols;
      block_u32x4 now[RT];
      float scale[RT];
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        now[r] = codes[slot][r];
        scale[r] = __uint_as_float((scales[slot][r] >> (8 * (k & 3)) & 255u) << 23);
      }
      load(slot, k + WK * DEPTH);
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
      k += WK;
    };
    // a chunk has WK DEPTH column tiles or a multiple of them, but for the last one
    const int end = k0 + tiles;
    while (k < end)
      each<DEPTH>([&](auto d) {
        if (k < end) take(d);
      });
    k0 = end;
    if (k0 >= a.kt) break;
    __syncthreads();
    put_rest(k0, min(a.chunk, a.kt - k0), false);
    __syncthreads();
  }
  __syncthreads();
  // sums [wavefront of a group][group][row tile][block][column][16 weights' rows]
  float* const sums = reinterpret_cast<float*>(lds);
  constexpr int SIZE = GROUPS * RT * CB * 256;
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int c = 0; c < CB; ++c) *reinterpret_cast<f32x4*>(sums + wk * SIZE + ((group * RT + r) * CB + c) * 256 + i * 16 + 4 * q) = acc[r][c];
  __syncthreads();
  if (!writes) return;
  float v[8] = {};
  for (int part = a.parts - 1; part >= 0; --part) {      // the smallest first
    const int at = out_m * a.parts + part;
    const float* const from = sums + ((out_piece >> 1) * CB + (at >> 4)) * 256 + (at & 15) * 16 + 8 * (out_piece & 1);
#pragma unroll
    for (int w = 0; w < WK; ++w)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += from[w * SIZE + e];
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] += bias[e];
  if (a.activation != SVG_ACT_NONE) activate8(v, a.activation);
  const size_t base = row_at(a.out_tok, (unsigned)(m0 + out_m));
  by_type(a.out_tok.type, [&](auto type) {
    constexpr int TYPE = decltype(type)::value;
    if (out_n + 8 <= a.N && a.out_runs) {
      store8_any<TYPE>(a.out, base + column_at(a.out_tok, (unsigned)out_n), v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (out_n + e < a.N) store1<TYPE>(a.out, base + column_at(a.out_tok, (unsigned)(out_n + e)), v[e]);
    }
  });
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
  a.x_runs = x_tok.D % 8 == 0 || x_tok.D == K;
  a.x_plain = x_tok.D == K && (x_tok.N >= M || x_tok.sb == x_tok.N * x_tok.sn);
  a.out_runs = out_tok.D % 8 == 0 || out_tok.D == N;
  const int cols = a.m_each * a.parts, blocks = (cols + 15) / 16;
  const int tile_bytes = cols * 256;                     // a column tile's activations in LDS
  // few column tiles: two wavefronts share them (5120 x 256 7.4 -> 5.2 us); otherwise all eight
  const bool few = a.kt <= 4;
  // Row tiles of a workgroup: what keeps all compute units equally busy, and where that leaves a choice the most that gives each a workgroup, since
  // every workgroup makes its own parts of the activations.
  int rt = 1;
  if (!few) {
    auto blocks_of = [&](int r) { return (a.n_tiles + r - 1) / r; };
    auto rounds = [&](int r) { return (blocks_of(r) + 255) / 256 * r; };
    const bool heavy = (long long)a.kt * tile_bytes > 32768;
    for (int r = 2; r <= 5; ++r)
      if (rounds(r) < rounds(rt) || (rounds(r) == rounds(rt) && (heavy || blocks_of(r) >= 256))) rt = r;
  }
  // Activations that do not fit come in chunks: of whole turns of the wavefronts, one tile ahead instead of two where those are too long.
  int depth = 2;
  a.chunk = a.kt;
  if ((long long)a.kt * tile_bytes > kLds) {
    int turn = kWaves * depth;
    if (turn * tile_bytes > kLds) depth = 1, turn = kWaves;
    a.chunk = kLds / tile_bytes / turn * turn;
  }
  const int lds = std::max(a.chunk * tile_bytes, kWaves * rt * blocks * 1024);
  const int per_block = rt * (few ? 4 : 1);
  const dim3 grid((unsigned)((a.n_tiles + per_block - 1) / per_block), (unsigned)((M + a.m_each - 1) / a.m_each));
  (void)hipGetLastError();
  auto go = [&](auto block) {
    constexpr int CB = decltype(block)::value;
    static std::atomic<unsigned long long> allowed[2][6];      // GPUs on which a form may take this much LDS
    auto with = [&](auto tiles) {
      constexpr int RT = decltype(tiles)::value;
      const void* kernel = reinterpret_cast<const void*>(few ? rows_kernel<1, CB, 2, 2> : depth == 1 ? rows_kernel<RT, CB, 8, 1> : rows_kernel<RT, CB, 8, 2>);
      hipError_t e = lds > 65536 ? allow_lds(kernel, kLds, allowed[depth == 1][few ? 0 : RT]) : hipSuccess;
      void* args[] = {&a};
      if (e == hipSuccess) e = hipLaunchKernel(kernel, grid, dim3(64 * kWaves), args, (size_t)lds, stream);
      return e;
    };
    hipError_t e = hipSuccess;
    if (rt == 1) e = with(std::integral_constant<int, 1>{});
    else if (rt == 2) e = with(std::integral_constant<int, 2>{});
    else if (rt == 3) e = with(std::integral_constant<int, 3>{});
    else if (rt == 4) e = with(std::integral_constant<int, 4>{});
    else e = with(std::integral_constant<int, 5>{});
    return e;
  };
  const hipError_t e = blocks == 1 ? go(std::integral_constant<int, 1>{}) : blocks == 2 ? go(std::integral_constant<int, 2>{}) : go(std::integral_constant<int, 3>{});
  return hip_status(e != hipSuccess ? e : hipGetLastError());
}

}  // namespace svg
