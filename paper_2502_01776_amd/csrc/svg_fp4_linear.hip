// Products of microscaled 4-bit operands, out = act(a w^T + bias), on v_mfma_scale_f32_16x16x128_f8f6f4.
//
// The weights are the instruction's first operand and the activations its second, so a lane of the accumulator
// holds four neighbouring columns of one token.  Two products side by side take the 32 rows of a pair of weight tiles so that
// the lane has eight neighbouring columns, 8 q to 8 q + 7 for the lanes of quarter q: row 8 (i / 4) + 4 t + i % 4 is row i of product t.
// The pair is then one block of a 4-bit output, spread over the four lanes l, l^16, l^32, l^48.
#include <type_traits>
#include <utility>

#include "svg_attn_common.h"
#include "svg_block.h"

namespace svg {

namespace {

using attn::barrier_loads_done;
using attn::buffer_words;
using attn::load_to_lds;
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct LinearArgs {
  const unsigned char *a, *w;
  const unsigned *as, *ws;
  const float* bias;
  long long M;
  int N, kt, kg;                      // column tiles of K and groups of four of them
  long long m_tiles, n_tiles;         // row tiles of a and w
  int n_pairs;                        // pairs of column tiles (32 columns) that are computed
  int activation;
  Tokens tok;                         // output of the plain form
  void* out;
  unsigned* codes;                    // output of the quantising form
  unsigned char* scales;
  int out_tiles, out_groups;
};

__device__ __forceinline__ i32x8 operand(i32x4 x) { return __builtin_shufflevector(x, x, 0, 1, 2, 3, -1, -1, -1, -1); }

template <int STEP>
__device__ __forceinline__ f32x4 product(i32x4 w, i32x4 a, f32x4 c, unsigned ws, unsigned as) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(w), operand(a), c, 4, 4, STEP, (int)ws, STEP, (int)as);
}

// The largest of x over the lanes l, l^16, l^32, l^48, in all of them.
__device__ __forceinline__ unsigned quarter_max(unsigned x) {
  const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = max(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return max(b[0], b[1]);
}

// f(0), f(1), .. f(N - 1) with constants: what indexes accumulators has to be one, or they leave the registers.
template <class F, int... I>
__device__ __forceinline__ void each_of(F f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void each(F f) { each_of(f, std::make_integer_sequence<int, N>{}); }

enum Output { kAny, kVectors, kOperand };      // token matrix of any kind, of whole aligned runs of eight; a 4-bit operand

// The activations where the result is rounded next: base-2 exponential and reciprocal of the vector unit, a few units in the last place of fp32.
__device__ __forceinline__ float activate_fast(float v, int activation) {
  if (activation == SVG_ACT_NONE) return v;
  constexpr float kLog2e = 1.4426950408889634f;
  const float u = activation == SVG_ACT_SILU ? -kLog2e * v : -1.5957691216057308f * kLog2e * __builtin_fmaf(0.044715f * v * v, v, v);
  return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u));
}

// What the columns n to n + 7 of a pair have in common for all tokens.
template <Output OUT>
struct Columns {
  float bias[8];
  int n;
  size_t at[OUT == kAny ? 8 : 1];        // elements from a token's first
  __device__ __forceinline__ Columns(const LinearArgs& A, int n_) : n(n_) {
#pragma unroll
    for (int e = 0; e < 8; ++e) bias[e] = A.bias && n + e < A.N ? A.bias[n + e] : 0.f;
    if constexpr (OUT != kOperand) {
#pragma unroll
      for (int e = 0; e < (OUT == kAny ? 8 : 1); ++e) {
        const unsigned c = (unsigned)min(n + e, A.N - 1), h = c / (unsigned)A.tok.D;
        at[e] = (size_t)h * A.tok.sh + (c - h * (unsigned)A.tok.D);
      }
    }
  }
};

// Elements from the output's first to token m's.
__device__ __forceinline__ size_t token_at(const LinearArgs& A, long long m) {
  const unsigned row = (unsigned)min(m, A.M - 1), b = row / (unsigned)A.tok.N;
  return (size_t)b * A.tok.sb + (size_t)(row - b * (unsigned)A.tok.N) * A.tok.sn;
}

// Token m's eight columns to the output.  All 64 lanes call it together.
template <Output OUT>
__device__ __forceinline__ void finish(const LinearArgs& A, long long m, size_t row, const Columns<OUT>& col, f32x4 lo, f32x4 hi) {
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (e < 4 ? lo[e & 3] : hi[e & 3]) + col.bias[e];
  if (A.activation != SVG_ACT_NONE) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = activate_fast(v[e], A.activation);
  }
  const int n = col.n;
  if constexpr (OUT == kOperand) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = m < A.M && n + e < A.N ? v[e] : 0.f;      // the padding
    const unsigned s = fp4_scale(quarter_max(magnitude8(v)));
    const unsigned c = fp4_codes8(v, s);
    const long long rt = m / kFp4Rows;
    const int i = (int)(m % kFp4Rows), ct = n / kFp4Cols, g = (n >> 5) & 3;
    if (rt < A.m_tiles && ct < A.out_tiles) {
      A.codes[((size_t)rt * A.out_tiles + ct) * 256 + g * 64 + i * 4 + ((n >> 3) & 3)] = c;
      if ((n & 31) == 0) A.scales[(((size_t)rt * A.out_groups + ct / kFp4Group) * 64 + g * 16 + i) * 4 + ct % kFp4Group] = (unsigned char)s;
    }
  } else if constexpr (OUT == kVectors) {                   // N is a multiple of 8: D is
    if (m >= A.M || n >= A.N) return;
    const size_t at = row + col.at[0];
    if (A.tok.type == SVG_BF16) store8<SVG_BF16>(A.out, at, v);
    else if (A.tok.type == SVG_F16) store8<SVG_F16>(A.out, at, v);
    else store8<SVG_F32>(A.out, at, v);
  } else {
    if (m >= A.M) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (n + e >= A.N) continue;
      const size_t at = row + col.at[e];
      if (A.tok.type == SVG_BF16) store1<SVG_BF16>(A.out, at, v[e]);
      else if (A.tok.type == SVG_F16) store1<SVG_F16>(A.out, at, v[e]);
      else store1<SVG_F32>(A.out, at, v[e]);
    }
  }
}

// The accumulators of TM token tiles and TP pairs to the output.
template <Output OUT, int TM, int TP>
__device__ __forceinline__ void finish_all(const LinearArgs& A, long long m, int n, const f32x4 (&acc)[TM][TP][2]) {
  size_t row[TM];
  if constexpr (OUT != kOperand) each<TM>([&](auto x) { row[x] = token_at(A, m + x * kFp4Rows); });
  else each<TM>([&](auto x) { row[x] = 0; });
  each<TP>([&](auto y) {
    const Columns<OUT> col(A, n + y * 32);
    each<TM>([&](auto x) { finish<OUT>(A, m + x * kFp4Rows, row[x], col, acc[x][y][0], acc[x][y][1]); });
  });
}

// A wavefront computes MT token tiles times NP pairs of column tiles, operands straight from memory; WK wavefronts share
// the columns of K and add up through LDS in the order of their number.
template <int MT, int NP, int WK, Output OUT>
__global__ __launch_bounds__(64 * WK) void linear_rows_kernel(LinearArgs A) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int i = lane & 15, q = lane >> 4;
  const int m_blocks = (int)((A.m_tiles + MT - 1) / MT);
  const int mb = blockIdx.x % m_blocks, nb = blockIdx.x / m_blocks;
  const unsigned char* ap[MT];
  const unsigned* asp[MT];
  const unsigned char* wp[NP][2];
  const unsigned* wsp[NP][2];
#pragma unroll
  for (int x = 0; x < MT; ++x) {
    const long long t = min((long long)mb * MT + x, A.m_tiles - 1);
    ap[x] = A.a + (size_t)t * A.kt * kFp4Tile + lane * 16;
    asp[x] = A.as + (size_t)t * A.kg * 64 + lane;
  }
#pragma unroll
  for (int x = 0; x < NP; ++x)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int r = 8 * (i >> 2) + 4 * t + (i & 3);
      const long long tile = min((long long)(nb * NP + x) * 2 + (r >> 4), A.n_tiles - 1);
      const int piece = 16 * q + (r & 15);
      wp[x][t] = A.w + (size_t)tile * A.kt * kFp4Tile + piece * 16;
      wsp[x][t] = A.ws + (size_t)tile * A.kg * 64 + piece;
    }
  f32x4 acc[MT][NP][2] = {};
  for (int k = wave; k < A.kg; k += WK) {
    unsigned as[MT], ws[NP][2];
#pragma unroll
    for (int x = 0; x < MT; ++x) as[x] = asp[x][(size_t)k * 64];
#pragma unroll
    for (int x = 0; x < NP; ++x)
#pragma unroll
      for (int t = 0; t < 2; ++t) ws[x][t] = wsp[x][t][(size_t)k * 64];
    auto step = [&](auto j) {
      constexpr int J = decltype(j)::value;
      const size_t at = (size_t)(k * kFp4Group + J) * kFp4Tile;
      i32x4 av[MT], wv[NP][2];
#pragma unroll
      for (int x = 0; x < NP; ++x)
#pragma unroll
        for (int t = 0; t < 2; ++t) wv[x][t] = *reinterpret_cast<const i32x4*>(wp[x][t] + at);
#pragma unroll
      for (int x = 0; x < MT; ++x) av[x] = *reinterpret_cast<const i32x4*>(ap[x] + at);
#pragma unroll
      for (int x = 0; x < MT; ++x)
#pragma unroll
        for (int y = 0; y < NP; ++y)
#pragma unroll
          for (int t = 0; t < 2; ++t) acc[x][y][t] = product<J>(wv[y][t], av[x], acc[x][y][t], ws[y][t], as[x]);
    };
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
    if (k * kFp4Group + 2 < A.kt) {
      step(std::integral_constant<int, 2>{});
      step(std::integral_constant<int, 3>{});
    }
  }
  if constexpr (WK > 1) {
    __shared__ f32x4 part[WK][MT * NP * 2][64];
#pragma unroll
    for (int x = 0; x < MT * NP * 2; ++x) part[wave][x][lane] = acc[x / (NP * 2)][x / 2 % NP][x % 2];
    __syncthreads();
    // the pairs are dealt to the wavefronts
    for (int p = wave; p < MT * NP; p += WK) {
      f32x4 lo = part[0][2 * p][lane], hi = part[0][2 * p + 1][lane];
      for (int w = 1; w < WK; ++w) {
        lo += part[w][2 * p][lane];
        hi += part[w][2 * p + 1][lane];
      }
      const long long m = ((long long)mb * MT + p / NP) * kFp4Rows + i;
      const Columns<OUT> col(A, (nb * NP + p % NP) * 32 + 8 * q);
      finish<OUT>(A, m, OUT == kOperand ? 0 : token_at(A, m), col, lo, hi);
    }
  } else {
    finish_all<OUT, MT, NP>(A, (long long)mb * MT * kFp4Rows + i, nb * NP * 32 + 8 * q, acc);
  }
}

// Row of the weights' pair that lane 16 q + i gives product t.
__device__ __forceinline__ int pair_row(int i, int t) { return 8 * (i >> 2) + 4 * t + (i & 3); }

// One load of 16 bytes a lane from memory into LDS, lane l at lds_address + 16 l; as load_to_lds, which takes two at a time.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_one_to_lds(const attn::u32x4 rsrc, int voffset, int soffset, unsigned lds_address) {
  asm volatile("s_mov_b32 m0, %3\n\ts_nop 3\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds"
               :: "v"(voffset), "s"(rsrc), "s"(soffset), "s"(lds_address)
               : "memory", "m0");
}
#pragma clang diagnostic pop

// Waits until at most N of this wavefront's loads to LDS are outstanding and its own LDS reads have arrived.
template <int N>
__device__ __forceinline__ void wait_stage() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory"); }

// Output tiles of WM x WN wavefronts, each TM token tiles times TP pairs of column tiles, operands through LDS.
//
// One step is one column tile of K (128 columns) of every row tile: 1 KB an operand, moved from memory straight into LDS
// by loads of 1 KB, kStages - 1 steps ahead.  The lanes of a weight tile's load fetch the pieces in the order in which the products
// take the rows of a pair, so every LDS read is 1 KB in one run.  The scale bytes of four steps follow as one
// 256-byte run a row tile.
// A token operand is read where the last product that uses its predecessor has been issued, a pair of weight operands one
// pair ahead, so one set of token operands and two pairs of weights are all that is held beside the accumulators.  In front of the last pair of a
// step a wavefront waits for the loads of the next step and meets the others at the barrier, which also says that everybody has
// read the present stage; then it refills that stage.
constexpr int kStages = 4;

template <int TM, int TP, int WM, int WN>
struct TileShape {
  static constexpr int waves = WM * WN;
  static constexpr int m_tiles = TM * WM, n_tiles = 2 * TP * WN;     // row tiles of a workgroup
  static constexpr int tiles = m_tiles + n_tiles;
  static constexpr int loads = tiles / waves;                         // of a wavefront for one step
  static constexpr int scale_loads = (tiles * 256 / 1024 + waves - 1) / waves;
  static constexpr int lds = kStages * tiles * kFp4Tile + tiles * 256;
  static_assert(tiles % (2 * waves) == 0 && (tiles * 256) % (1024 * waves) == 0, "whole loads");
};

template <int TM, int TP, int WM, int WN, Output OUT>
__global__ __launch_bounds__(64 * WM * WN, 1) void linear_tile_kernel(LinearArgs A, int m_blocks, int n_blocks) {
  using Shape = TileShape<TM, TP, WM, WN>;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WM, wn = wave / WM;
  const int i = lane & 15, q = lane >> 4;
  int mb, nb;
  {
    // consecutive workgroups go to the 8 XCDs in turn: each takes a run of the tiles, in groups of 4 rows of tiles
    const int total = m_blocks * n_blocks, per = (total + 7) / 8;
    const int xcd = blockIdx.x & 7, at = xcd * per + (int)(blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || at >= total) return;
    const int group = at / (4 * n_blocks), rows = min(4, m_blocks - 4 * group), in = at - group * 4 * n_blocks;
    mb = 4 * group + in % rows;
    nb = in / rows;
  }
  // descriptors of this workgroup's row tiles; tiles behind the end of a matrix read as zeros
  const long long m0 = (long long)mb * Shape::m_tiles, n0 = (long long)nb * Shape::n_tiles;
  const int mv = (int)min((long long)Shape::m_tiles, A.m_tiles - m0);
  const int nv = (int)max(0ll, min((long long)Shape::n_tiles, A.n_tiles - n0));
  const unsigned tile_bytes = (unsigned)A.kt * kFp4Tile, scale_bytes = (unsigned)A.kg * 256;
  const bool weights = wave < Shape::waves / 2;                       // which operand this wavefront's loads fetch
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
  constexpr int kStageBytes = Shape::tiles * kFp4Tile;
  constexpr int kScales = kStages * kStageBytes;                      // where the scale bytes are
  static_assert(Shape::m_tiles == Shape::n_tiles, "half of the wavefronts load each operand");
  const int first = (wave % (Shape::waves / 2)) * Shape::loads;       // first row tile of its operand that this wavefront loads
  const auto rsrc = weights ? buffer_words(A.w + (size_t)n0 * tile_bytes, (unsigned)nv * tile_bytes)
                            : buffer_words(A.a + (size_t)m0 * tile_bytes, (unsigned)mv * tile_bytes);
  const auto rsrc_s = weights ? buffer_words(A.ws + (size_t)n0 * scale_bytes / 4, (unsigned)nv * scale_bytes)
                              : buffer_words(A.as + (size_t)m0 * scale_bytes / 4, (unsigned)mv * scale_bytes);
  int voff[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int r = pair_row(i, t);
    voff[t] = weights ? (r >> 4) * (int)tile_bytes + (16 * q + (r & 15)) * 16 : t * (int)tile_bytes + lane * 16;
  }
  // scale words of four row tiles in one load: lanes 16 t to 16 t + 15 fetch tile t's 256 bytes (the order of the pieces is put right by the reader)
  const int voff_s = (lane >> 4) * (int)scale_bytes + (lane & 15) * 16;
  auto load_step = [&](int k, int stage) {
    const int past = k < A.kt ? 0 : 0x40000000;                      // behind the last step: out of range, zeros without a fetch
#pragma unroll
    for (int x = 0; x < Shape::loads; x += 2) {
      const int so = (first + x) * (int)tile_bytes + k * kFp4Tile + past;
      load_to_lds(rsrc, voff[0], voff[1], so, so,
                  lds0 + stage * kStageBytes + (weights ? 0 : Shape::n_tiles * kFp4Tile) + (first + x) * kFp4Tile, kFp4Tile);
    }
  };
  auto load_scales = [&](int g) {
    const int past = g < A.kg ? 0 : 0x40000000;
#pragma unroll
    for (int x = 0; x < Shape::scale_loads; ++x) {
      const int tile = (wave % (Shape::waves / 2)) * Shape::scale_loads * 4 + x * 4;
      load_one_to_lds(rsrc_s, voff_s, tile * (int)scale_bytes + g * 256 + past,
                      lds0 + kScales + (weights ? 0 : Shape::n_tiles * 256) + tile * 256);
    }
  };
  // this wavefront's operands: weight tiles first, then token tiles
  const i32x4* const wl = reinterpret_cast<const i32x4*>(lds + wn * 2 * TP * kFp4Tile) + lane;
  const i32x4* const al = reinterpret_cast<const i32x4*>(lds + (Shape::n_tiles + wm * TM) * kFp4Tile) + lane;
  const unsigned* wsl[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int r = pair_row(i, t);
    wsl[t] = reinterpret_cast<const unsigned*>(lds + kScales + (wn * 2 * TP + (r >> 4)) * 256) + 16 * q + (r & 15);
  }
  const unsigned* const asl = reinterpret_cast<const unsigned*>(lds + kScales + (Shape::n_tiles + wm * TM) * 256) + lane;

  i32x4 wv[2][2], av[TM];
  unsigned ws[TP][2], as[TM];
  f32x4 acc[TM][TP][2] = {};
  auto read_pair = [&](int stage, int y, i32x4 (&w)[2]) {
#pragma unroll
    for (int t = 0; t < 2; ++t) w[t] = wl[stage * (kStageBytes / 16) + (2 * y + t) * 64];
  };
  auto read_token = [&](int stage, int x) { av[x] = al[stage * (kStageBytes / 16) + x * 64]; };
  auto read_scales = [&] {
#pragma unroll
    for (int y = 0; y < TP; ++y)
#pragma unroll
      for (int t = 0; t < 2; ++t) ws[y][t] = wsl[t][y * 128];
#pragma unroll
    for (int x = 0; x < TM; ++x) as[x] = asl[x * 64];
  };
  load_scales(0);
  load_step(0, 0);
  load_step(1, 1);
  load_step(2, 2);
  load_step(3, 3);
  wait_stage<3 * Shape::loads>();
  barrier_loads_done();
  read_scales();
  read_pair(0, 0, wv[0]);
#pragma unroll
  for (int x = 0; x < TM; ++x) read_token(0, x);
  static_assert(TP % 2 == 0, "the first pair of a step is in the first register pair");
  auto step = [&](auto j, int k, int g) {
    constexpr int J = decltype(j)::value;
    each<TP - 1>([&](auto yc) {
      constexpr int y = decltype(yc)::value;
      read_pair(J, y + 1, wv[(y + 1) & 1]);
#pragma unroll
      for (int x = 0; x < TM; ++x)
#pragma unroll
        for (int t = 0; t < 2; ++t) acc[x][y][t] = product<J>(wv[y & 1][t], av[x], acc[x][y][t], ws[y][t], as[x]);
    });
    // the loads of the two steps behind the next one, and this group's loads of the next scale bytes, may be outstanding
    wait_stage<2 * Shape::loads + (J == 1 || J == 2 ? Shape::scale_loads : 0)>();
    barrier_loads_done();
    if constexpr (J == 0) load_scales(g + 1);
    load_step(k + 4, J);
    constexpr int y = TP - 1;
    read_pair((J + 1) & 3, 0, wv[0]);
#pragma unroll
    for (int x = 0; x < TM; ++x) {
#pragma unroll
      for (int t = 0; t < 2; ++t) acc[x][y][t] = product<J>(wv[1][t], av[x], acc[x][y][t], ws[y][t], as[x]);
      read_token((J + 1) & 3, x);
    }
    if constexpr (J == 3) read_scales();
  };
  for (int g = 0; g < A.kg; ++g) {
    const int k = g * kFp4Group;
    step(std::integral_constant<int, 0>{}, k, g);
    step(std::integral_constant<int, 1>{}, k + 1, g);
    if (k + 2 < A.kt) {
      step(std::integral_constant<int, 2>{}, k + 2, g);
      step(std::integral_constant<int, 3>{}, k + 3, g);
    }
  }
  wait_stage<0>();                      // no load to LDS outlives the workgroup
  finish_all<OUT, TM, TP>(A, (m0 + wm * TM) * kFp4Rows + i, ((int)n0 / 2 + wn * TP) * 32 + 8 * q, acc);
}

template <int TM, int TP, int WM, int WN>
int launch_tiles(const LinearArgs& a, Output out, hipStream_t stream) {
  using Shape = TileShape<TM, TP, WM, WN>;
  const long long m_blocks = (a.m_tiles + Shape::m_tiles - 1) / Shape::m_tiles;
  const long long n_blocks = (2ll * a.n_pairs + Shape::n_tiles - 1) / Shape::n_tiles;
  const long long blocks = (m_blocks * n_blocks + 7) / 8 * 8;
  if (blocks > 0x7fffff) return SVG_ERR_UNSUPPORTED;
  auto kernel = out == kOperand   ? linear_tile_kernel<TM, TP, WM, WN, kOperand>
                : out == kVectors ? linear_tile_kernel<TM, TP, WM, WN, kVectors>
                                  : linear_tile_kernel<TM, TP, WM, WN, kAny>;
  (void)hipGetLastError();
  if (Shape::lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, Shape::lds);
    if (e != hipSuccess) return hip_status(e);
  }
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(64 * Shape::waves), Shape::lds, stream, a, (int)m_blocks, (int)n_blocks);
  return hip_status(hipGetLastError());
}

template <int MT, int NP, int WK>
int launch_rows(const LinearArgs& a, Output out, hipStream_t stream) {
  const long long blocks = (a.m_tiles + MT - 1) / MT * ((a.n_pairs + NP - 1) / NP);
  if (blocks > 0x7fffffll) return SVG_ERR_UNSUPPORTED;
  (void)hipGetLastError();
  auto kernel = out == kOperand ? linear_rows_kernel<MT, NP, WK, kOperand> : out == kVectors ? linear_rows_kernel<MT, NP, WK, kVectors> : linear_rows_kernel<MT, NP, WK, kAny>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(64 * WK), 0, stream, a);
  return hip_status(hipGetLastError());
}

}  // namespace

size_t fp4_linear_workspace_bytes(long long, long long, long long) { return 0; }

int launch_fp4_linear(long long M, int N, int K, const void* a, const void* a_scales, const void* w, const void* w_scales,
                      const float* bias, int activation, const Tokens* tok, void* out, void* codes, void* scales, void*,
                      hipStream_t stream) {
  LinearArgs A = {};
  A.a = static_cast<const unsigned char*>(a);
  A.w = static_cast<const unsigned char*>(w);
  A.as = static_cast<const unsigned*>(a_scales);
  A.ws = static_cast<const unsigned*>(w_scales);
  A.bias = bias;
  A.M = M;
  A.N = N;
  A.kt = (int)fp4_col_tiles(K);
  A.kg = (int)fp4_col_groups(K);
  A.m_tiles = fp4_row_tiles(M);
  A.n_tiles = fp4_row_tiles(N);
  A.n_pairs = codes ? (int)fp4_col_tiles(N) * 4 : (N + 31) / 32;
  A.activation = activation;
  if (tok) {
    A.tok = *tok;
    A.out = out;
  } else {
    A.codes = static_cast<unsigned*>(codes);
    A.scales = static_cast<unsigned char*>(scales);
    A.out_tiles = (int)fp4_col_tiles(N);
    A.out_groups = (int)fp4_col_groups(N);
  }
  const Output form = codes ? kOperand : tokens_vectors(*tok, out) ? kVectors : kAny;
  if (M <= 16) return launch_rows<1, 1, 8>(A, form, stream);
  if (M <= 512) return launch_rows<4, 1, 4>(A, form, stream);
  return launch_tiles<8, 2, 2, 4>(A, form, stream);
}

}  // namespace svg
