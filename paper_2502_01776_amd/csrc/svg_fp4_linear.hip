// Products of microscaled 4-bit operands, out = act(a w^T + bias), on v_mfma_scale_f32_16x16x128_f8f6f4.
//
// The weights are the instruction's first operand and the activations its second, so a lane of the accumulator
// holds four neighbouring columns of one token.  Two products side by side take the 32 rows of a pair of weight tiles so that
// the lane has eight neighbouring columns, 8 q to 8 q + 7 for the lanes of quarter q: row 8 (i / 4) + 4 t + i % 4 is row i of product t.
// The pair is then one block of a 4-bit output, spread over the four lanes l, l^16, l^32, l^48.
#include <algorithm>
#include <atomic>
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

constexpr long long kComputeUnits = 256;

// The output: a token matrix of any kind; one of whole aligned runs of eight columns in which a workgroup's tile spans less than 2^30 bytes;
// a 4-bit operand.
enum Output { kAny, kVectors, kOperand };

// The bias of the columns n to n + 3.
__device__ __forceinline__ f32x4 bias_of(const LinearArgs& A, int n) {
  f32x4 b;
#pragma unroll
  for (int e = 0; e < 4; ++e) b[e] = A.bias && n + e < A.N ? A.bias[n + e] : 0.f;
  return b;
}

// Elements from the output's first to token m's, and from a token's first to column n.
__device__ __forceinline__ size_t token_at(const LinearArgs& A, long long m) {
  const unsigned row = (unsigned)m, b = row / (unsigned)A.tok.N;
  return (size_t)b * A.tok.sb + (size_t)(row - b * (unsigned)A.tok.N) * A.tok.sn;
}
__device__ __forceinline__ size_t column_at(const LinearArgs& A, int n) {
  const unsigned h = (unsigned)n / (unsigned)A.tok.D;
  return (size_t)h * A.tok.sh + ((unsigned)n - h * (unsigned)A.tok.D);
}

// Writes accumulators: eight columns of a token a lane, tokens 16 a tile, columns 32 a pair.  m0, n0: the first token and column of the
// wavefront's tiles, the same in all lanes; TM, TP: their number.  Offsets inside the output are taken from a descriptor whose base is
// the wavefront's first element, in 32 bits, and what lies outside of the output is sent behind the descriptor's end, where stores have no effect.
template <Output OUT, int TM, int TP>
struct Writer {
  const LinearArgs& A;
  const long long m0;
  const int n0;
  const int i, q;
  static constexpr unsigned kOutside = 0x40000000;           // the descriptor's size: more than any tile spans
  __amdgpu_buffer_rsrc_t rsrc, rsrc_s;
  unsigned row[TM];                                     // bytes from the first token to this lane's of tile x
  bool inner;                                           // all tokens and columns exist
  long long rt0;

  __device__ __forceinline__ Writer(const LinearArgs& A_, long long m0_, int n0_) : A(A_), m0(m0_), n0(n0_), i(threadIdx.x & 15), q((threadIdx.x >> 4) & 3) {
    inner = m0 + TM * kFp4Rows <= A.M && n0 + TP * 32 <= A.N;
    if constexpr (OUT == kVectors) {
      const int size = type_bytes(A.tok.type);
      const size_t first = token_at(A, min(m0, A.M - 1)) + column_at(A, min(n0, A.N - 1));
      rsrc = __builtin_amdgcn_make_buffer_rsrc(static_cast<char*>(A.out) + first * size, 0, (int)kOutside, attn::kRsrcFlags);
      const size_t token0 = token_at(A, min(m0, A.M - 1));
      each<TM>([&](auto x) {
        const long long m = m0 + x * kFp4Rows + i;
        row[x] = m < A.M ? (unsigned)(token_at(A, m) - token0) * size : kOutside;
      });
    } else if constexpr (OUT == kOperand) {
      rt0 = m0 / kFp4Rows;
      rsrc = __builtin_amdgcn_make_buffer_rsrc(A.codes + (size_t)rt0 * A.out_tiles * 256, 0, (int)kOutside, attn::kRsrcFlags);
      rsrc_s = __builtin_amdgcn_make_buffer_rsrc(A.scales + (size_t)rt0 * A.out_groups * 256, 0, (int)kOutside, attn::kRsrcFlags);
    }
  }

  // the values of tile x and pair y; all 64 lanes call it together
  template <int X, int Y>
  __device__ __forceinline__ void write(f32x4 lo, f32x4 hi, unsigned col) const {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < 4 ? lo[e & 3] : hi[e & 3];
    if (A.activation != SVG_ACT_NONE) activate8(v, A.activation);
    const int n = n0 + Y * 32 + 8 * q;
    if constexpr (OUT == kOperand) {
      if (!inner) {                                     // the padding
        const bool token = m0 + X * kFp4Rows + i < A.M;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = token && n + e < A.N ? v[e] : 0.f;
      }
      const unsigned s = fp4_scale(quarter_max(magnitude8(v)));
      const unsigned c = fp4_codes8(v, s);
      const int block = n0 / 32 + Y, ct = block >> 2, g = block & 3;
      const bool there = rt0 + X < A.m_tiles && ct < A.out_tiles;
      __builtin_amdgcn_raw_buffer_store_b32(c, rsrc, i * 16 + q * 4, there ? X * A.out_tiles * 1024 + ct * 1024 + g * 256 : (int)kOutside, 0);
      __builtin_amdgcn_raw_buffer_store_b8((unsigned char)s, rsrc_s, (int)(i * 4 + (q ? kOutside : 0)),
                                           there ? X * A.out_groups * 256 + (ct >> 2) * 256 + g * 64 + (ct & 3) : (int)kOutside, 0);
    } else if constexpr (OUT == kVectors) {
      // Results are read by another pass, if at all from L2's far side: not kept in L2, where they would take the operands' place.
      constexpr int kStream = 2;
      const int at = (int)(row[X] + col);
      if (A.tok.type == SVG_F32) {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(attn::u32x4, f32x4{v[0], v[1], v[2], v[3]}), rsrc, at, 0, kStream);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(attn::u32x4, f32x4{v[4], v[5], v[6], v[7]}), rsrc, at, 16, kStream);
      } else {
        const block_f32x8 f = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
        const attn::u32x4 bits = A.tok.type == SVG_BF16 ? __builtin_bit_cast(attn::u32x4, __builtin_convertvector(f, block_bf16x8))
                                                        : __builtin_bit_cast(attn::u32x4, __builtin_convertvector(f, block_f16x8));
        __builtin_amdgcn_raw_buffer_store_b128(bits, rsrc, at, 0, kStream);
      }
    } else {
      const long long m = m0 + X * kFp4Rows + i;
      if (m >= A.M) return;
      const size_t first = token_at(A, m);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (n + e >= A.N) continue;
        const size_t at = first + column_at(A, n + e);
        if (A.tok.type == SVG_BF16) store1<SVG_BF16>(A.out, at, v[e]);
        else if (A.tok.type == SVG_F16) store1<SVG_F16>(A.out, at, v[e]);
        else store1<SVG_F32>(A.out, at, v[e]);
      }
    }
  }
  // bytes from the first column to this lane's of pair Y
  template <int Y>
  __device__ __forceinline__ unsigned column() const {
    if constexpr (OUT != kVectors) return 0;
    const int n = n0 + Y * 32 + 8 * q;                   // N is a multiple of 8: D is
    return n < A.N ? (unsigned)(column_at(A, n) - column_at(A, min(n0, A.N - 1))) * type_bytes(A.tok.type) : kOutside;
  }
  __device__ __forceinline__ void all(const f32x4 (&acc)[TM][TP][2]) const {
    each<TP>([&](auto y) {
      const unsigned col = column<y>();
      each<TM>([&](auto x) { write<x, y>(acc[x][y][0], acc[x][y][1], col); });
    });
  }
};

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
  f32x4 acc[MT][NP][2];
  // the first of the wavefronts that share K begins with the bias
  each<NP * 2>([&](auto n) {
    const f32x4 b = wave % WK == 0 ? bias_of(A, (nb * NP + n / 2) * 32 + 8 * q + n % 2 * 4) : f32x4{};
    each<MT>([&](auto x) { acc[x][n / 2][n % 2] = b; });
  });
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
    const Writer<OUT, 1, 1> out(A, ((long long)mb * MT + p / NP) * kFp4Rows, (nb * NP + p % NP) * 32);
    out.template write<0, 0>(lo, hi, out.template column<0>());
  }
}

// Row of the weights' pair that lane 16 q + i gives product t.
__device__ __forceinline__ int pair_row(int i, int t) { return 8 * (i >> 2) + 4 * t + (i & 3); }

// One load of 4 bytes a lane from memory into LDS, lane l at lds_address + 4 l; as load_to_lds, which takes two of 16 bytes.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_words_to_lds(const attn::u32x4 rsrc, int voffset, int soffset, unsigned lds_address) {
  asm volatile("s_mov_b32 m0, %3\n\ts_nop 3\n\tbuffer_load_dword %0, %1, %2 offen lds"
               :: "v"(voffset), "s"(rsrc), "s"(soffset), "s"(lds_address)
               : "memory", "m0");
}
#pragma clang diagnostic pop

// Waits until at most N of this wavefront's loads are outstanding and its LDS reads have arrived.
template <int N>
__device__ __forceinline__ void wait_stage() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory"); }

// Lets a kernel take more than 64 KB of LDS; once for each GPU, because the call costs a microsecond.
hipError_t allow_lds(const void* kernel, int bytes, std::atomic<unsigned long long>& allowed) {
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess) return e;
  const unsigned long long bit = device < 64 ? 1ull << device : 0;
  if (allowed.load(std::memory_order_relaxed) & bit) return hipSuccess;
  e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) allowed.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

// Output tiles of WM x WN wavefronts, each TM token tiles times TP pairs of column tiles.
//
// A step is one column tile of K (128 columns); four steps, whose scale bytes share a word, are a group.  The token operands,
// which the WN wavefronts of a row share, go straight from memory into LDS, a group ahead and in two halves of LDS in turn; the weight
// operands, which are a wavefront's own, go from memory into registers, a pair where the same pair has last been used two or
// eight steps earlier.  So LDS carries 8 KB a wavefront and step instead of 12, and one barrier a group is enough: in front of the last pair of a
// group a wavefront waits for the token operands of the next group and meets the others, which also says that the present
// half has been read.  A token operand is read where the last product that uses its predecessor has been issued.
template <int TM, int TP, int WM, int WN>
struct TileShape {
  static constexpr int waves = WM * WN;
  static constexpr int m_tiles = TM * WM, n_tiles = 2 * TP * WN;     // row tiles of a workgroup
  static constexpr int ahead = TM * TP <= 4 ? 8 : 2;                  // steps that the weights are asked for ahead: what the registers hold
  static constexpr int share = m_tiles / waves;                       // token tiles whose loads are a wavefront's
  static constexpr int stage = m_tiles * kFp4Tile;                    // LDS of a step's token operands
  static constexpr int half = kFp4Group * stage + m_tiles * 256;      // of a group's, with the scale bytes
  static constexpr int bias = 2 * half;                               // the bias of two output tiles in turn
  static constexpr int bias_bytes = n_tiles * kFp4Rows * 4;
  static constexpr int lds = bias + 2 * bias_bytes;
  static constexpr int per_unit = lds <= 81920 && waves <= 4 ? 2 : 1; // workgroups of a compute unit
  static_assert(share * waves == m_tiles && bias_bytes % 256 == 0, "whole loads");
};

template <int TM, int TP, int WM, int WN, Output OUT>
__global__ __launch_bounds__(64 * WM * WN, (TileShape<TM, TP, WM, WN>::per_unit * WM * WN / 4)) void
linear_tile_kernel(LinearArgs A, int m_blocks, int n_blocks) {
  using Shape = TileShape<TM, TP, WM, WN>;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WM, wn = wave / WM;
  const int i = lane & 15, q = lane >> 4;
  const unsigned tile_bytes = (unsigned)A.kt * kFp4Tile, scale_bytes = (unsigned)A.kg * 256;
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
  constexpr int kRows = 8;
  // Consecutive workgroups go to the 8 XCDs in turn: each XCD takes a run of the output tiles, in groups of 8 rows of
  // tiles, and deals them to its workgroups in turn.
  const int total = m_blocks * n_blocks, per = (total + 7) / 8;
  const int run_end = min(total, ((int)(blockIdx.x & 7) + 1) * per), run_step = (int)(gridDim.x >> 3);
  int at = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
  if (at >= run_end) return;

  long long m0, n0;                     // first row tiles
  attn::u32x4 rsrc_a, rsrc_as;
  __amdgpu_buffer_rsrc_t rsrc_w, rsrc_ws;
  // descriptors of the present output tile's operands; tiles behind the end of a matrix read as zeros
  auto open_tile = [&] {
    const int group = at / (kRows * n_blocks), rows = min(kRows, m_blocks - kRows * group), in = at - group * kRows * n_blocks;
    m0 = (long long)(kRows * group + in % rows) * Shape::m_tiles;
    n0 = (long long)(in / rows) * Shape::n_tiles;
    const unsigned mv = (unsigned)min((long long)Shape::m_tiles, A.m_tiles - m0);
    rsrc_a = buffer_words(A.a + (size_t)m0 * tile_bytes, mv * tile_bytes);
    rsrc_as = buffer_words(A.as + (size_t)m0 * scale_bytes / 4, mv * scale_bytes);
    const long long nw = n0 + wn * 2 * TP;                            // this wavefront's own
    const unsigned nv = (unsigned)max(0ll, min((long long)(2 * TP), A.n_tiles - nw));
    rsrc_w = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(A.w) + (size_t)(nv ? nw : 0) * tile_bytes, 0, (int)(nv * tile_bytes), attn::kRsrcFlags);
    rsrc_ws = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned*>(A.ws) + (size_t)(nv ? nw : 0) * scale_bytes / 4, 0, (int)(nv * scale_bytes), attn::kRsrcFlags);
  };
  constexpr int kPast = 0x40000000;     // added to an offset: out of range, zeros without a fetch
  // The token operands of group g, part by part (a pair of loads each), and their scale bytes.
  const int voff_a = lane * 16, voff_s = lane * 4;
  constexpr int kParts = Shape::share * kFp4Group / 2;
  auto load_tokens = [&](int g, int part) {
    const unsigned to = lds0 + (g & 1) * Shape::half;
    int so[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const int n = 2 * part + z, t = wave * Shape::share + n % Shape::share, k = g * kFp4Group + n / Shape::share;
      so[z] = t * (int)tile_bytes + k * kFp4Tile + (k < A.kt ? 0 : kPast);
    }
    const int t = wave * Shape::share + 2 * part % Shape::share, j = 2 * part / Shape::share;
    load_to_lds(rsrc_a, voff_a, voff_a, so[0], so[1], to + j * Shape::stage + t * kFp4Tile, Shape::share == 1 ? Shape::stage : kFp4Tile);
  };
  auto load_token_scales = [&](int g) {
    const unsigned to = lds0 + (g & 1) * Shape::half + kFp4Group * Shape::stage;
#pragma unroll
    for (int x = 0; x < Shape::share; ++x) {
      const int t = wave * Shape::share + x;
      load_words_to_lds(rsrc_as, voff_s, t * (int)scale_bytes + g * 256 + (g < A.kg ? 0 : kPast), to + t * 256);
    }
  };
  // the bias of the tile's columns, 64 a load; the wavefronts behind the last 64 load them again
  const auto rsrc_b = buffer_words(A.bias ? A.bias : reinterpret_cast<const float*>(A.w), A.bias ? (unsigned)A.N * 4 : 0);
  auto load_bias = [&](int turn) {
    const int part = wave % (Shape::bias_bytes / 256);
    load_words_to_lds(rsrc_b, lane * 4, (int)n0 * kFp4Rows * 4 + part * 256, lds0 + Shape::bias + turn * Shape::bias_bytes + part * 256);
  };
  // weights: the rows of a pair in the order of the products
  int voff_w[2], voff_ws[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int r = pair_row(i, t);
    voff_w[t] = (r >> 4) * (int)tile_bytes + (16 * q + (r & 15)) * 16;
    voff_ws[t] = (r >> 4) * (int)scale_bytes + (16 * q + (r & 15)) * 4;
  }
  constexpr int kAhead = Shape::ahead;
  i32x4 wv[kAhead][TP][2], av[TM];
  unsigned ws[TP][2], ws_next[TP][2], as[TM];
  f32x4 acc[TM][TP][2];
  auto load_pair = [&](int k, int y, i32x4 (&w)[2]) {
    const int so = 2 * y * (int)tile_bytes + k * kFp4Tile + (k < A.kt ? 0 : kPast);
#pragma unroll
    for (int t = 0; t < 2; ++t) w[t] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc_w, voff_w[t], so, 0));
  };
  auto load_weight_scales = [&](int g, unsigned (&s)[TP][2]) {
#pragma unroll
    for (int y = 0; y < TP; ++y)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        s[y][t] = __builtin_amdgcn_raw_buffer_load_b32(rsrc_ws, voff_ws[t], 2 * y * (int)scale_bytes + g * 256 + (g < A.kg ? 0 : kPast), 0);
  };
  auto load_first = [&](int turn) {
    load_bias(turn);
    load_token_scales(0);
#pragma unroll
    for (int p = 0; p < kParts; ++p) load_tokens(0, p);
    load_weight_scales(0, ws);
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
#pragma unroll
      for (int y = 0; y < TP; ++y) load_pair(k, y, wv[k][y]);
  };
  auto read_token = [&](int g, int j, int x) {
    av[x] = reinterpret_cast<const i32x4*>(lds + (g & 1) * Shape::half + j * Shape::stage + (wm * TM + x) * kFp4Tile)[lane];
  };
  auto read_scales = [&](int g) {
#pragma unroll
    for (int x = 0; x < TM; ++x)
      as[x] = reinterpret_cast<const unsigned*>(lds + (g & 1) * Shape::half + kFp4Group * Shape::stage + (wm * TM + x) * 256)[lane];
  };
  // step J of group g, whose number is odd if ODD
  auto step = [&](auto jc, auto odd, int g) {
    constexpr int J = decltype(jc)::value, W = (decltype(odd)::value * kFp4Group + J) % kAhead;
    const int k = g * kFp4Group + J;
    each<TP>([&](auto yc) {
      constexpr int y = decltype(yc)::value;
      if constexpr (y == TP - 1) __builtin_amdgcn_s_setprio(1);      // as in the larger tiles
      if constexpr (J == 3 && y == TP - 1) {
        // behind the next group's token operands only the scale words and weights of the steps 1 to 3 have been asked for
        wait_stage<8 * TP - 2>();
        barrier_loads_done();
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int x = 0; x < TM; ++x) {
#pragma unroll
        for (int t = 0; t < 2; ++t) acc[x][y][t] = product<J>(wv[W][y][t], av[x], acc[x][y][t], ws[y][t], as[x]);
        if constexpr (y == TP - 1) read_token(J == 3 ? g + 1 : g, (J + 1) & 3, x);
        // the next group's token operands in the first two steps, between the products
        if (y == 0 && J < 2 && x % 2 == 1) {
          constexpr int kSlots = TM / 2, kHere = (kParts + 1) / 2;
#pragma unroll
          for (int n = 0; n < kHere; ++n)
            if (n % kSlots == x / 2 && J * kHere + n < kParts) load_tokens(g + 1, J * kHere + n);
          if (x == TM - 1) {
            if constexpr (J == 0) load_token_scales(g + 1);
            if constexpr (J == 1) load_weight_scales(g + 1, ws_next);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      load_pair(k + kAhead, y, wv[W][y]);
      if constexpr (y == TP - 1) __builtin_amdgcn_s_setprio(0);
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (J == 3) {
      read_scales(g + 1);
#pragma unroll
      for (int y = 0; y < TP; ++y)
#pragma unroll
        for (int t = 0; t < 2; ++t) ws[y][t] = ws_next[y][t];
    }
  };
  open_tile();
  load_first(0);
  for (int turn = 0;; turn ^= 1) {
    wait_stage<(kAhead + 1) * TP * 2>();
    barrier_loads_done();
    read_scales(0);
#pragma unroll
    for (int x = 0; x < TM; ++x) read_token(0, 0, x);
    // the accumulators begin with the bias
    const float* const staged = reinterpret_cast<const float*>(lds + Shape::bias + turn * Shape::bias_bytes) + wn * TP * 32 + 8 * q;
    each<TP * 2>([&](auto n) {
      const f32x4 b = *reinterpret_cast<const f32x4*>(staged + n / 2 * 32 + n % 2 * 4);
      each<TM>([&](auto x) { acc[x][n / 2][n % 2] = b; });
    });
    int g = 0;
    const int whole = A.kt / kFp4Group;
    auto group = [&](auto odd, int g) {
      step(std::integral_constant<int, 0>{}, odd, g);
      step(std::integral_constant<int, 1>{}, odd, g);
      step(std::integral_constant<int, 2>{}, odd, g);
      step(std::integral_constant<int, 3>{}, odd, g);
    };
    auto half_group = [&](auto odd, int g) {        // kt is even
      step(std::integral_constant<int, 0>{}, odd, g);
      step(std::integral_constant<int, 1>{}, odd, g);
    };
    using Even = std::integral_constant<int, 0>;
    using Odd = std::integral_constant<int, 1>;
    const bool tail = A.kt % kFp4Group;
    if constexpr (kAhead <= kFp4Group) {
      for (; g < whole; ++g) group(Even{}, g);
      if (tail) half_group(Even{}, g);
    } else {
      for (; g + 1 < whole; g += 2) {
        group(Even{}, g);
        group(Odd{}, g + 1);
      }
      if (g < whole) {
        group(Even{}, g);
        if (tail) half_group(Odd{}, g + 1);
      } else if (tail) {
        half_group(Even{}, g);
      }
    }
    // No load to LDS outlives the workgroup, and LDS is everybody's again: the next tile's first group is on its way
    // while this one's results are written.
    wait_stage<0>();
    const Writer<OUT, TM, TP> out(A, (m0 + wm * TM) * kFp4Rows, ((int)n0 / 2 + wn * TP) * 32);
    at += run_step;
    const bool more = at < run_end;
    if (more) {
      barrier_loads_done();
      open_tile();
      load_first(turn ^ 1);
    }
    out.all(acc);
    if (!more) return;
  }
}

template <int TM, int TP, int WM, int WN>
int launch_tiles(const LinearArgs& a, Output out, hipStream_t stream) {
  using Shape = TileShape<TM, TP, WM, WN>;
  const long long m_blocks = (a.m_tiles + Shape::m_tiles - 1) / Shape::m_tiles;
  const long long n_blocks = (2ll * a.n_pairs + Shape::n_tiles - 1) / Shape::n_tiles;
  if (m_blocks * n_blocks > 0x7fffffff - 8) return SVG_ERR_UNSUPPORTED;
  const long long most = kComputeUnits * Shape::per_unit, blocks = std::min(most, (m_blocks * n_blocks + 7) / 8 * 8);
  auto kernel = out == kOperand   ? linear_tile_kernel<TM, TP, WM, WN, kOperand>
                : out == kVectors ? linear_tile_kernel<TM, TP, WM, WN, kVectors>
                                  : linear_tile_kernel<TM, TP, WM, WN, kAny>;
  static std::atomic<unsigned long long> allowed[3];
  (void)hipGetLastError();
  if (const hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), Shape::lds, allowed[out]); e != hipSuccess) return hip_status(e);
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(64 * Shape::waves), Shape::lds, stream, a, (int)m_blocks, (int)n_blocks);
  return hip_status(hipGetLastError());
}

// Output tiles of 256 x 256 for large products: eight wavefronts of 8 token tiles x 2 pairs, both operands through LDS in four stages of a
// step each, asked for four steps ahead; one barrier a step, in front of its last pair of products, behind which the loads of the
// stage that is free are issued between products.  The 128 x 64 outputs of a wavefront take 12 KB of LDS reads for 32 products.
// 32760 x 5120 x 20480: 1315 us into 4 bits and 1365 into bf16 rows, 5.2 and 5.0 PFLOP/s; the matrix units are busy 69 % of the cycles at 1.78 GHz
// (a loop of the same products from registers alone reaches 6.4 to 6.8 PFLOP/s on random operands, 9.5 on zeros: power).  32760 x 20480 x 5120: 1477 and
// 1527 us, behind GELU 1585 and 1608.
// What a round of tiles costs beside its K part (9 us) is largely the wait for the results of the tile before: their stores are issued behind the
// next tile's first loads, and the counts of its first steps are of loads alone, so the stores have to end first.
constexpr int kStages = 4;

template <int TM, int TP, int WM, int WN>
struct SquareShape {
  static constexpr int waves = WM * WN;
  static constexpr int m_tiles = TM * WM, n_tiles = 2 * TP * WN;     // row tiles of a workgroup
  static constexpr int tiles = m_tiles + n_tiles;
  static constexpr int loads = tiles / waves;                         // of a wavefront for one step
  static constexpr int scale_loads = (tiles * 256 / 1024 + waves - 1) / waves;
  static constexpr int bias_bytes = n_tiles * kFp4Rows * 4;
  static constexpr int lds = kStages * tiles * kFp4Tile + tiles * 256 + 2 * bias_bytes;
  static_assert(tiles % (2 * waves) == 0 && (tiles * 256) % (1024 * waves) == 0, "whole loads");
};

template <int TM, int TP, int WM, int WN, Output OUT>
__global__ __launch_bounds__(64 * WM * WN, 1) void linear_square_kernel(LinearArgs A, int m_blocks, int n_blocks) {
  using Shape = SquareShape<TM, TP, WM, WN>;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WM, wn = wave / WM;
  const int i = lane & 15, q = lane >> 4;
  const unsigned tile_bytes = (unsigned)A.kt * kFp4Tile, scale_bytes = (unsigned)A.kg * 256;
  const bool weights = wave < Shape::waves / 2;                       // which operand this wavefront's loads fetch
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
  constexpr int kStageBytes = Shape::tiles * kFp4Tile;
  constexpr int kScales = kStages * kStageBytes;                      // where the scale bytes are
  constexpr int kBias = kScales + Shape::tiles * 256;                 // and two tiles' bias in turn
  static_assert(Shape::m_tiles == Shape::n_tiles, "half of the wavefronts load each operand");
  const int first = (wave % (Shape::waves / 2)) * Shape::loads;       // first row tile of its operand that this wavefront loads
  // Consecutive workgroups go to the 8 XCDs in turn: each XCD takes a run of the output tiles, in groups of 4 rows of
  // tiles, and deals them to its workgroups in turn.
  const int total = m_blocks * n_blocks, per = (total + 7) / 8;
  const int run_end = min(total, ((int)(blockIdx.x & 7) + 1) * per), run_step = (int)(gridDim.x >> 3);
  int at = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
  long long m0, n0;
  attn::u32x4 rsrc, rsrc_s;
  auto open_tile = [&] {
    const int group = at / (4 * n_blocks), rows = min(4, m_blocks - 4 * group), in = at - group * 4 * n_blocks;
    m0 = (long long)(4 * group + in % rows) * Shape::m_tiles;
    n0 = (long long)(in / rows) * Shape::n_tiles;
    // descriptors of the row tiles; tiles behind the end of a matrix read as zeros
    const int mv = (int)min((long long)Shape::m_tiles, A.m_tiles - m0);
    const int nv = (int)max(0ll, min((long long)Shape::n_tiles, A.n_tiles - n0));
    rsrc = weights ? buffer_words(A.w + (size_t)n0 * tile_bytes, (unsigned)nv * tile_bytes)
                   : buffer_words(A.a + (size_t)m0 * tile_bytes, (unsigned)mv * tile_bytes);
    rsrc_s = weights ? buffer_words(A.ws + (size_t)n0 * scale_bytes / 4, (unsigned)nv * scale_bytes)
                     : buffer_words(A.as + (size_t)m0 * scale_bytes / 4, (unsigned)mv * scale_bytes);
  };
  int voff[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int r = pair_row(i, t);
    voff[t] = weights ? (r >> 4) * (int)tile_bytes + (16 * q + (r & 15)) * 16 : t * (int)tile_bytes + lane * 16;
  }
  // scale words of four row tiles in one load: lanes 16 t to 16 t + 15 fetch tile t's 256 bytes (the order of the pieces is put right by the reader)
  const int voff_s = (lane >> 4) * (int)scale_bytes + (lane & 15) * 16;
  auto load_pairs = [&](int k, int stage, int x) {
    const int past = k < A.kt ? 0 : 0x40000000;                      // behind the last step: out of range, zeros without a fetch
    const int so = (first + x) * (int)tile_bytes + k * kFp4Tile + past;
    load_to_lds(rsrc, voff[0], voff[1], so, so,
                lds0 + stage * kStageBytes + (weights ? 0 : Shape::n_tiles * kFp4Tile) + (first + x) * kFp4Tile, kFp4Tile);
  };
  auto load_step = [&](int k, int stage) {
#pragma unroll
    for (int x = 0; x < Shape::loads; x += 2) load_pairs(k, stage, x);
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
  // the bias of the tile's columns, 64 a load; the wavefronts behind the last 64 load them again
  const auto rsrc_b = buffer_words(A.bias ? A.bias : reinterpret_cast<const float*>(A.w), A.bias ? (unsigned)A.N * 4 : 0);
  auto load_bias = [&](int turn) {
    const int part = wave % (Shape::bias_bytes / 256);
    load_words_to_lds(rsrc_b, lane * 4, (int)n0 * kFp4Rows * 4 + part * 256, lds0 + kBias + turn * Shape::bias_bytes + part * 256);
  };
  auto load_first = [&](int turn) {
    load_scales(0);
    load_bias(turn);
#pragma unroll
    for (int k = 0; k < kStages; ++k) load_step(k, k);
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
  f32x4 acc[TM][TP][2];
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
  static_assert(TP % 2 == 0, "the first pair of a step is in the first register pair");
  auto step = [&](auto j, int k, int g) {
    constexpr int J = decltype(j)::value;
    each<TP - 1>([&](auto yc) {
      constexpr int y = decltype(yc)::value;
      read_pair(J, y + 1, wv[(y + 1) & 1]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int x = 0; x < TM; ++x)
#pragma unroll
        for (int t = 0; t < 2; ++t) acc[x][y][t] = product<J>(wv[y & 1][t], av[x], acc[x][y][t], ws[y][t], as[x]);
    });
    // The wavefront that meets the barrier first takes the matrix unit first behind it: the two of a SIMD then read
    // operands in turn (1.7 % of the time of 32760 x 5120 x 20480).
    __builtin_amdgcn_s_setprio(1);
    // the loads of the two steps behind the next one, and this group's loads of the next scale bytes, may be outstanding
    wait_stage<2 * Shape::loads + (J == 1 || J == 2 ? Shape::scale_loads : 0)>();
    barrier_loads_done();
    constexpr int y = TP - 1;
    read_pair((J + 1) & 3, 0, wv[0]);
#pragma unroll
    for (int x = 0; x < TM; ++x) {
#pragma unroll
      for (int t = 0; t < 2; ++t) acc[x][y][t] = product<J>(wv[1][t], av[x], acc[x][y][t], ws[y][t], as[x]);
      read_token((J + 1) & 3, x);
      // the loads between the products: in a row behind the barrier they would keep the matrix units waiting
      if (x == 0 && J == 0) load_scales(g + 1);
      if (x % 2 == 1 && x / 2 < Shape::loads / 2) load_pairs(k + 4, J, x - 1);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    if constexpr (J == 3) read_scales();
  };
  if (at >= run_end) return;
  open_tile();
  load_first(0);
  for (int turn = 0;; turn ^= 1) {
    wait_stage<(kStages - 1) * Shape::loads>();
    barrier_loads_done();
    read_scales();
    read_pair(0, 0, wv[0]);
#pragma unroll
    for (int x = 0; x < TM; ++x) read_token(0, x);
    const float* const staged = reinterpret_cast<const float*>(lds + kBias + turn * Shape::bias_bytes) + wn * TP * 32 + 8 * q;
    each<TP * 2>([&](auto n) {
      const f32x4 b = *reinterpret_cast<const f32x4*>(staged + n / 2 * 32 + n % 2 * 4);
      each<TM>([&](auto x) { acc[x][n / 2][n % 2] = b; });
    });
    int g = 0;
    for (; g < A.kt / kFp4Group; ++g) {
      const int k = g * kFp4Group;
      step(std::integral_constant<int, 0>{}, k, g);
      step(std::integral_constant<int, 1>{}, k + 1, g);
      step(std::integral_constant<int, 2>{}, k + 2, g);
      step(std::integral_constant<int, 3>{}, k + 3, g);
    }
    if (A.kt % kFp4Group) {             // half a group: kt is even
      step(std::integral_constant<int, 0>{}, g * kFp4Group, g);
      step(std::integral_constant<int, 1>{}, g * kFp4Group + 1, g);
    }
    // No load to LDS outlives the workgroup, and the stages are everybody's again: the next tile's first steps are on
    // their way while this one's results are written.
    wait_stage<0>();
    const Writer<OUT, TM, TP> out(A, (m0 + wm * TM) * kFp4Rows, ((int)n0 / 2 + wn * TP) * 32);
    at += run_step;
    const bool more = at < run_end;
    if (more) {
      barrier_loads_done();
      open_tile();
      load_first(turn ^ 1);
    }
    out.all(acc);
    if (!more) return;
  }
}

template <int TM, int TP, int WM, int WN>
int launch_square(const LinearArgs& a, Output out, hipStream_t stream) {
  using Shape = SquareShape<TM, TP, WM, WN>;
  const long long m_blocks = (a.m_tiles + Shape::m_tiles - 1) / Shape::m_tiles;
  const long long n_blocks = (2ll * a.n_pairs + Shape::n_tiles - 1) / Shape::n_tiles;
  if (m_blocks * n_blocks > 0x7fffffff - 8) return SVG_ERR_UNSUPPORTED;
  const long long most = kComputeUnits * (163840 / Shape::lds), blocks = std::min(most, (m_blocks * n_blocks + 7) / 8 * 8);
  auto kernel = out == kOperand   ? linear_square_kernel<TM, TP, WM, WN, kOperand>
                : out == kVectors ? linear_square_kernel<TM, TP, WM, WN, kVectors>
                                  : linear_square_kernel<TM, TP, WM, WN, kAny>;
  static std::atomic<unsigned long long> allowed[3];
  (void)hipGetLastError();
  if (const hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), Shape::lds, allowed[out]); e != hipSuccess) return hip_status(e);
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

int launch(const LinearArgs& a, Output form, hipStream_t stream) {
  switch (fp4_linear_form(a.m_tiles, a.n_pairs, a.kt, a.activation != SVG_ACT_NONE)) {
    case LinearForm::kRows1: return launch_rows<1, 1, 8>(a, form, stream);
    case LinearForm::kRows2Eight: return launch_rows<2, 1, 8>(a, form, stream);
    case LinearForm::kRows2: return launch_rows<2, 1, 4>(a, form, stream);
    case LinearForm::kRows4: return launch_rows<4, 1, 4>(a, form, stream);
    case LinearForm::kTiles64: return launch_tiles<4, 1, 1, 4>(a, form, stream);
    case LinearForm::kTiles128: return launch_tiles<8, 2, 1, 4>(a, form, stream);
    default: return launch_square<8, 2, 2, 4>(a, form, stream);
  }
}

}  // namespace

// Which form a product takes, by estimates of its time: what a round of workgroups needs is a part for its beginning and end, more of it
// with an activation, and one that grows with K.  A launch's workgroups of 256 x 256 run one to a compute unit, the smaller ones
// two, and one that has its compute unit to itself is faster.  In us, K in thousands:
//   256 x 256: 9 + 5.1 K a round of 256;  128 x 256: 9 + 5.35 K a round of 512, 6.1 + 3.44 K for a last one of up to 256;
//   64 x 128: 3.6 + 1.9 K, 85 % of it;  an activation: + 3.5, 3.5, 2.6, 0.5 (a fit over the products below; 2.0 to 2.7 in 40 rounds of 32760 x 20480 x 5120).
// Up to 64 tokens, or up to 400 workgroups of 64 tokens and 32 columns, operands straight from memory (K split over the wavefronts).
// us, 256 x 256 | 128 x 256 | 64 x 128 | straight (M x N x K), all forms in one run; between runs a time differs by up to 4 %:
//   64 x 5120 x 5120 30.3 22.9 12.5 9.3;  226 x 5120 x 4096 27.1 19.5 10.9 13.3;  226 x 1536 x 1536 15.8 11.3 6.9 6.4;
//   1573 x 512 x 512 11.3 8.6 6.0 5.9;  1573 x 1536 x 6144 34.3 25.4 16.8 26.7;  1573 x 6144 x 1536 17.3 17.2 18.0 26.6;
//   4096 x 1536 x 1536 17.0 12.4 13.5 17.5;  2048 x 5120 x 5120 33.3 34.5 36.6 63.3;  4096 x 5120 x 5120 73.4 60.2 77.8 117;
//   17776 x 512 x 8192 47.9 52.1 58.6 174;  32760 x 5120 x 20480 1376 1465 2246
// and behind GELU 500 x 10240 x 2560 22.9 17.2 15.2 25.2;  226 x 20480 x 5120 33.7 25.7 24.7 40.2;  1573 x 6144 x 1536 20.4 20.4 18.7 27.0;
//   8000 x 4096 x 1024 35.1 33.5 46.3 86.1;  32760 x 20480 x 5120 1569 1558 2212
// Straight, one token tile (K over 8 wavefronts), two (4, or 8 where there are fewer workgroups than compute units) and four (4):
//   16 x 5120 x 5120 7.1 7.8 (8: 7.5) 8.9;  32 x 5120 x 5120 9.6 7.9 (7.5) 8.9;  32 x 20480 x 5120 22.8 15.7 (19.5) 17.6
LinearForm fp4_linear_form(long long m, long long pairs, int kt, bool activation) {
  if (m == 1) return LinearForm::kRows1;
  if (m == 2) return pairs < kComputeUnits ? LinearForm::kRows2Eight : LinearForm::kRows2;
  if (m <= 4 || (m + 3) / 4 * pairs <= 400) return LinearForm::kRows4;
  auto tiles = [&](int m_tiles, int n_pairs) { return (m + m_tiles - 1) / m_tiles * ((pairs + n_pairs - 1) / n_pairs); };
  auto rounds = [](long long tiles, double whole, double alone) {
    const long long rest = tiles % (2 * kComputeUnits);
    return (double)(tiles / (2 * kComputeUnits)) * whole + (rest > kComputeUnits ? whole : rest ? alone : 0.0);
  };
  const double k = kt * 0.128, act = activation ? 1.0 : 0.0;
  const double square = (double)((tiles(16, 8) + kComputeUnits - 1) / kComputeUnits) * (9.0 + 3.5 * act + 5.1 * k);
  const double large = rounds(tiles(8, 8), 9.0 + 3.5 * act + 5.35 * k, 6.1 + 2.6 * act + 3.44 * k);
  const double one = 3.6 + 0.5 * act + 1.9 * k, small = rounds(tiles(4, 4), one, 0.85 * one);
  if (square <= large && square <= small) return LinearForm::kSquare;
  return large <= small ? LinearForm::kTiles128 : LinearForm::kTiles64;
}

namespace {
// Do the tokens of an output tile of 256 x 256 ascend in memory, and does it span less than 2^29 bytes?  (They may lie in as many batch entries.)
bool tile_spans_little(const Tokens& t, long long M, int N) {
  if (M > t.N && t.sb < (t.N - 1) * t.sn) return false;
  const long long tokens = std::min<long long>(M, 256), entries = std::min<long long>((M + t.N - 1) / t.N, (tokens + t.N - 1) / t.N + 1);
  const long long heads = std::min<long long>((N + t.D - 1) / t.D, 256 / t.D + 2);
  const __int128 span = (__int128)(entries - 1) * t.sb + (__int128)std::min(tokens, t.N) * t.sn + (__int128)(heads - 1) * t.sh + t.D;
  return span * 4 < (1 << 29);
}
}  // namespace

int launch_fp4_linear(long long M, int N, int K, const void* a, const void* a_scales, const void* w, const void* w_scales,
                      const float* bias, int activation, const Tokens* tok, void* out, void* codes, void* scales,
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
  const Output form = codes ? kOperand : tokens_vectors(*tok, out) && tile_spans_little(*tok, M, N) ? kVectors : kAny;
  return launch(A, form, stream);
}

}  // namespace svg
