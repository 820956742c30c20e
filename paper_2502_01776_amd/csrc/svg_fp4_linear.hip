// Products of microscaled 4-bit operands, out = act(a w^T + bias), on v_mfma_scale_f32_16x16x128_f8f6f4.
//
// The weights are the instruction's first operand and the activations its second, so a lane of the accumulator
// holds four neighbouring columns of one token.  Two products side by side take the 32 rows of a pair of weight tiles so that
// the lane has eight neighbouring columns, 8 q to 8 q + 7 for the lanes of quarter q: row 8 (i / 4) + 4 t + i % 4 is row i of product t.
// The pair is then one block of a 4-bit output, spread over the four lanes l, l^16, l^32, l^48.
#include <type_traits>

#include "svg_block.h"

namespace svg {

namespace {

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
  bool vec;
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

// Token m's columns n to n + 7 to the output.  All 64 lanes call it together.
template <bool QUANT>
__device__ __forceinline__ void finish(const LinearArgs& A, long long m, int n, f32x4 lo, f32x4 hi) {
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float b = A.bias && n + e < A.N ? A.bias[n + e] : 0.f;
    v[e] = activate((e < 4 ? lo[e & 3] : hi[e & 3]) + b, A.activation);
  }
  if constexpr (QUANT) {
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
  } else {
    if (m >= A.M || n >= A.N) return;
    const long long b = m / A.tok.N;
    const size_t base = (size_t)b * A.tok.sb + (size_t)(m - b * A.tok.N) * A.tok.sn;
    if (A.vec) {                                     // N is a multiple of 8 then: D is
      const size_t at = base + (size_t)(n / A.tok.D) * A.tok.sh + n % A.tok.D;
      if (A.tok.type == SVG_BF16) store8<SVG_BF16>(A.out, at, v);
      else if (A.tok.type == SVG_F16) store8<SVG_F16>(A.out, at, v);
      else store8<SVG_F32>(A.out, at, v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = n + e;
        if (c >= A.N) continue;
        const size_t at = base + (size_t)(c / A.tok.D) * A.tok.sh + c % A.tok.D;
        if (A.tok.type == SVG_BF16) store1<SVG_BF16>(A.out, at, v[e]);
        else if (A.tok.type == SVG_F16) store1<SVG_F16>(A.out, at, v[e]);
        else store1<SVG_F32>(A.out, at, v[e]);
      }
    }
  }
}

// A wavefront computes MT token tiles times NP pairs of column tiles, operands straight from memory; WK wavefronts share
// the columns of K and add up through LDS in the order of their number.
template <int MT, int NP, int WK, bool QUANT>
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
      finish<QUANT>(A, ((long long)mb * MT + p / NP) * kFp4Rows + i, (nb * NP + p % NP) * 32 + 8 * q, lo, hi);
    }
  } else {
#pragma unroll
    for (int x = 0; x < MT; ++x)
#pragma unroll
      for (int y = 0; y < NP; ++y)
        finish<QUANT>(A, ((long long)mb * MT + x) * kFp4Rows + i, (nb * NP + y) * 32 + 8 * q, acc[x][y][0], acc[x][y][1]);
  }
}

template <int MT, int NP, int WK>
int launch_rows(const LinearArgs& a, bool quant, hipStream_t stream) {
  const long long blocks = (a.m_tiles + MT - 1) / MT * ((a.n_pairs + NP - 1) / NP);
  if (blocks > 0x7fffffll) return SVG_ERR_UNSUPPORTED;
  (void)hipGetLastError();
  if (quant) hipLaunchKernelGGL((linear_rows_kernel<MT, NP, WK, true>), dim3((unsigned)blocks), dim3(64 * WK), 0, stream, a);
  else hipLaunchKernelGGL((linear_rows_kernel<MT, NP, WK, false>), dim3((unsigned)blocks), dim3(64 * WK), 0, stream, a);
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
    A.vec = tokens_vectors(*tok, out);
  } else {
    A.codes = static_cast<unsigned*>(codes);
    A.scales = static_cast<unsigned char*>(scales);
    A.out_tiles = (int)fp4_col_tiles(N);
    A.out_groups = (int)fp4_col_groups(N);
  }
  const bool quant = codes != nullptr;
  if (M <= 16) return launch_rows<1, 1, 8>(A, quant, stream);
  if (M <= 512) return launch_rows<4, 1, 4>(A, quant, stream);
  return launch_rows<8, 2, 1>(A, quant, stream);
}

}  // namespace svg
