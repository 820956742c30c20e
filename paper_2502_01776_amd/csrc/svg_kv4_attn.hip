// Attention of new queries over a cache of keys and values in 4 bits (svg_kv4_attn_fwd).
//
// With c = scale log2 e, one pass over the visible keys j in tiles of 64, in fp32:
//     p_ij = 2^(c q_i k_j - m_i),  l_i = sum_j p_ij,  o_i = sum_j p_ij v_j / l_i
// against a reference m_i that follows the largest score where it has to: when a lane's sum of a tile passes 2^13, the tile is taken again
// against its own maximum and what was summed is rescaled.  Both products are computed transposed on v_mfma_f32_16x16x32_bf16,
//     S^T = K Q^T      O^T += V^T P^T
// as in svg_attn_kernel.h: a lane has one query and four neighbouring keys of every 16, so that sums over keys stay in its registers and the
// weights are the second product's operand as they are.  The weights are rounded to bf16 for it; sums take them unrounded.
//
// Every 4-bit value under its power of two is a bf16 number, so keys and values are dequantised exactly (two a v_cvt_scalef32_pk_bf16_fp4) and the
// scores are exact products summed in fp32.  (The matrix instruction that takes 4-bit keys as they are, with a query as two 8-bit parts, made the form
// with 128 rows 5 % faster, but cuts what is 2^-14.5 below the largest of 128 products: scores off by 4e-6 of their size.)
//
// Two forms:
//  * 16 or 32 query rows: the wavefronts of a workgroup share them and split the keys, every one with its own tiles, straight
//    from memory into registers one tile ahead; no barrier before the results are merged through LDS.  Bound: HBM: one token of eight sequences over
//    up to 65536, 32 heads on 8 of 128 channels, 312 MB of cache: 61 us under the profiler, and 5 for the join; 68-74 in a graph, 4.2-4.6 TB/s (a large copy 4.7-4.9).
//  * 128 rows, 32 a wavefront: a tile of keys and values is dequantised once for all, a quarter by each wavefront, into LDS.  Bound: the matrix and the
//    vector unit in turns.  40 heads of 4680 rows and 128 channels over 32760 keys 2.78-2.83 ms, 1.06-1.07 PFLOP/s (matrix cores busy 44 % of the cycles, vector
//    instructions 48 %, workgroups on 94 % of the places); 48 heads of 4050 rows and 64 channels in a window of seven frames 690-740 us, 0.73-0.78 PFLOP/s (31, 57
//    and 87 %: two equal rounds of workgroups, of which those across two frames take a quarter longer).
// Few workgroups for the chip: the keys are cut into parts for several, whose results a second launch joins.
#include <algorithm>
#include <limits>
#include <type_traits>
#include <utility>

#include "svg_attn_common.h"
#include "svg_kv4.h"

namespace svg {

namespace {

using namespace attn;

constexpr int kTile = 64;              // keys of a tile
constexpr int kWaves = 4;
constexpr float kLowest = -3.40282347e38f;      // the first reference: no finite score is below it
constexpr float kFar = 1073741824.f;            // 2^30 (take_tile)
constexpr int kGroups = kTile / 16;    // 16-key groups of a tile: pages begin and end between them

// f(0), f(1), .. f(N - 1) with constants.
template <class F, int... I>
__device__ __forceinline__ void each_of(F f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void each(F f) { each_of(f, std::make_integer_sequence<int, N>{}); }

struct Kv4AttnArgs {
  Kv4 c;
  HeadRows q, o;
  const __bf16* qp;
  __bf16* op;
  float* lse;
  const int32_t *kv_len, *q_len;
  float* part;               // [part][head][row][D], and behind them (reference, sum) [part][head][row]; null: no sequence is cut
  float2* stats;
  int N, group, rows, tiles;
  int parts;                 // of all sequences together
  int reach;                 // an estimate of the keys that a row tile visits: parts are dealt by it, no result depends on it
  int causal, block, window, sink, capacity;
  float scale_log2;
};

// A sequence, and the keys that its query rows see.
struct Sequence {
  int kv, qn;
  __device__ __forceinline__ Sequence(const Kv4AttnArgs& a, int b) {
    kv = min(max(__builtin_amdgcn_readfirstlane(a.kv_len[b]), 0), a.capacity);
    qn = a.q_len ? min(max(__builtin_amdgcn_readfirstlane(a.q_len[b]), 0), a.N) : a.N;
  }
};
// Keys [begin, end), and of those in front of begin the first `sink`.
struct Visible {
  int begin, end;
};
__device__ __forceinline__ Visible visible(const Kv4AttnArgs& a, const Sequence& s, int n) {
  const int p = s.kv - s.qn + n;                         // may be negative: a query without a token of its own
  if (!a.causal && a.window < 0) return {0, s.kv};
  const int f = p >= 0 ? p / a.block : -1 - (-1 - p) / a.block;
  Visible v = {0, s.kv};
  if (a.causal) v.end = (int)max(0ll, min((long long)s.kv, (f + 1ll) * a.block));
  if (a.window >= 0) v.begin = (int)min((long long)s.kv, max(0ll, ((long long)f - a.window) * a.block));
  return v;
}
__device__ __forceinline__ bool sees(const Visible& v, int sink, int key) { return key < v.end && (key >= v.begin || key < sink); }

// The same for a row that is the same in all lanes.
__device__ __forceinline__ Visible visible_uniform(const Kv4AttnArgs& a, const Sequence& s, int n) {
  const Visible v = visible(a, s, n);
  return {__builtin_amdgcn_readfirstlane(v.begin), __builtin_amdgcn_readfirstlane(v.end)};
}

// The tiles of a range of rows, whose windows ascend: those of the sink, then those from the first row's begin to the last row's end.
struct Tiles {
  int sink_tiles, first, count;
  __device__ __forceinline__ Tiles(const Visible& lo, const Visible& hi, int sink) {
    sink_tiles = min(sink, hi.end) > 0 ? (min(sink, hi.end) + kTile - 1) / kTile : 0;
    first = max(lo.begin / kTile, sink_tiles);
    count = sink_tiles + max(0, (hi.end + kTile - 1) / kTile - first);
  }
  __device__ __forceinline__ int at(int t) const { return t < sink_tiles ? t : t - sink_tiles + first; }
};

// The keys of long sequences are cut into more parts than those of short ones: beside the one that each has, the parts are dealt by the number
// of tiles.  Up to 64 sequences, one to a lane; more are cut alike.
struct Part {
  int b;              // the sequence of a part, or -1
  int first, count;   // its sequence's parts
};
__device__ __forceinline__ Part parts_from(const Kv4AttnArgs& a, bool by_part, int x) {
  Part p;
  if (a.parts == a.c.B) return {x, x, 1};
  if (a.c.B > 64) {
    p.count = a.parts / a.c.B;
    p.b = by_part ? x / p.count : x;
    p.first = p.b * p.count;
    return p;
  }
  const int lane = threadIdx.x & 63;
  const int kv = lane < a.c.B ? min(min(max(a.kv_len[lane], 0), a.capacity), a.reach) : 0;
  const unsigned tiles = (unsigned)(kv + kTile - 1) / kTile;
  unsigned sum = tiles;                                  // (64 sequences of at most 2^24 tiles)
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const unsigned y = (unsigned)__shfl_up((int)sum, d, 64);
    if (lane >= d) sum += y;
  }
  const unsigned all = (unsigned)__builtin_amdgcn_readlane((int)sum, 63);
  const unsigned more = (unsigned)(a.parts - a.c.B);
  // where a sequence's parts begin: rounded down from the tiles in front of it
  auto begin = [&](int i, unsigned front) { return all ? i + (int)((unsigned long long)more * front / all) : i; };
  const int first = begin(lane, sum - tiles), end = lane < a.c.B ? begin(lane + 1, sum) : 0x7fffffff;
  const int b = by_part ? (int)__builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < a.c.B && end <= x)) : x;
  if (b >= a.c.B) return {-1, 0, 0};                     // (no keys at all: a part for each sequence)
  p.b = b;
  p.first = __builtin_amdgcn_readlane(first, b);
  p.count = __builtin_amdgcn_readlane(end, b) - p.first;
  return p;
}
// Where part `split` of `splits` of n tiles begins, in a scalar register (the division is the vector unit's).
__device__ __forceinline__ int part_of(int n, int split, int splits) {
  return __builtin_amdgcn_readfirstlane(splits == 1 ? n * split : (int)((unsigned)n * (unsigned long long)(unsigned)split / (unsigned)splits));
}

__device__ __forceinline__ float power_of(unsigned scale) { return __uint_as_float(scale << 23); }
// A block of values that are not finite: zeros in the product, NaN put into the results of the queries that see it afterwards, since a
// weight of zero does not take it away.
__device__ __forceinline__ bool not_finite(unsigned scale) { return scale >= 253; }

// Eight values of a word of codes.
__device__ __forceinline__ bf16x8 dequantise8(unsigned code, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1),
               c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Values in LDS: rows of D bf16, 32-byte slots swizzled with the row for the transposing read (svg_attn_kernel.h).
template <int D>
__device__ __forceinline__ int value_slot(int row, int slot) {
  return row * (2 * D) + ((slot ^ (D == 128 ? row & 7 : (row >> 1) & 3)) << 5);
}
// Keys in LDS: 16-byte pieces swizzled with the row, so that one piece of 16 rows lies on different banks.
template <int D>
__device__ __forceinline__ int key_piece(int row, int piece) {
  return row * (2 * D) + ((piece ^ (D == 128 ? row & 15 : (row >> 1) & 7)) << 4);
}

// (A row that has seen nothing yet is none: whatever it sees makes a new reference.)
__device__ __forceinline__ bool far_reference(float m) { return fabsf(m) >= kFar && m != kLowest; }

// Scores of rows with a far reference as what is left of them against it.
template <int QB>
__device__ __forceinline__ void far_scores(f32x4 (&s)[kGroups][QB], const float (&m)[QB], const float c) {
#pragma clang fp contract(off)
  const float inverse = 1.f / c;
#pragma unroll
  for (int kb = 0; kb < kGroups; ++kb)
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float left = s[kb][qb][j] * c - m[qb];
        s[kb][qb][j] = far_reference(m[qb]) ? left * inverse : s[kb][qb][j];
      }
}

// Online softmax of a wavefront's tile.  s: scores; on return p is the second product's operand.
// An exponent is c s - m in one rounding, against a reference m that is itself a rounded c s.  All weights of a row share the factor that this makes, 2^(2^-24 |m|)
// at the most, which leaves fp32's range where |m| is far beyond 2^30 (scores of hundreds of millions).  From there on c s is rounded first: neighbours are 64
// apart or more then, so the largest score's weight is one and the others' are none beside it.
// far_lanes: the wavefront's lanes of such rows.  (A comparison for each row and tile instead: 40 x 4680 rows over 32760 keys 2.78 -> 2.81 ms.)
template <int QB, int CB>
__device__ __forceinline__ void take_tile(f32x4 (&s)[kGroups][QB], bf16x8 (&p)[kGroups / 2][QB], float (&m)[QB], float (&l)[QB],
                                          f32x4 (&o)[CB][QB], const float c, unsigned long long& far_lanes) {
  float sum[QB];
  auto exponentials = [&](const float (&reference)[QB]) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      sum[qb] = 0.f;
#pragma unroll
      for (int ks = 0; ks < kGroups / 2; ++ks) {
        f32x8 e;
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * ks + j / 4][qb][j % 4], c, -reference[qb]));
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[qb] += e[j];
        // rounded here, not where they are used: eight fewer registers for every eight weights while the scores are still needed
        block_u32x4 bits = __builtin_bit_cast(block_u32x4, __builtin_convertvector(e, bf16x8));
        asm volatile("" : "+v"(bits));
        p[ks][qb] = __builtin_bit_cast(bf16x8, bits);
      }
    }
  };
  exponentials(m);
  bool over = false;
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) over |= sum[qb] > kLazySum;
  if (far_lanes | __builtin_amdgcn_ballot_w64(over)) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      float top = s[0][qb][0];
#pragma unroll
      for (int kb = 0; kb < kGroups; ++kb)
#pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, s[kb][qb][j]);
      const float reference = fmaxf(m[qb], quarters_max(top) * c);
      const float f = __builtin_amdgcn_exp2f(m[qb] - reference);
      m[qb] = reference;
      l[qb] *= f;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) o[cb][qb] *= f;
    }
    float reference[QB];
    bool far = false;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      reference[qb] = far_reference(m[qb]) ? 0.f : m[qb];
      far |= far_reference(m[qb]);
    }
    far_lanes = __builtin_amdgcn_ballot_w64(far);
    asm volatile("" : "+s"(far_lanes));                  // (known to be none, the compiler would double the exponentials, and spill)
    if (far_lanes) far_scores<QB>(s, m, c);
    exponentials(reference);
  }
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) l[qb] += sum[qb];
}

template <int QB>
__device__ __forceinline__ void mask_tile(f32x4 (&s)[kGroups][QB], const Visible (&v)[QB], int sink, int key0, unsigned missing, int g) {
#pragma unroll
  for (int kb = 0; kb < kGroups; ++kb)
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        s[kb][qb][j] = !(missing >> kb & 1) && sees(v[qb], sink, key0 + 16 * kb + 4 * g + j) ? s[kb][qb][j] : -INFINITY;
}

// NaN into the channels [32 block, + 32) of the queries that see this key.
template <int QB, int CB>
__device__ __forceinline__ void poison(f32x4 (&o)[CB][QB], const Visible (&v)[QB], int sink, int key, int block) {
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const bool hit = sees(v[qb], sink, key);
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
      if (cb >> 1 == block && hit) o[cb][qb] = f32x4{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
  }
}

// Query row m of a head of the cache: its token, and the query head.
struct Row {
  int n, head;
  __device__ __forceinline__ Row(const Kv4AttnArgs& a, int kvh, int m) {
    n = a.group == 1 ? m : m / a.group;
    head = kvh * a.group + (a.group == 1 ? 0 : m - n * a.group);
  }
};
// What this lane's rows see, one in each 16-query block from row m0 on; a row that does not exist sees nothing.  Taken anew where a tile needs
// it, behind an opaque m0, so that it does not occupy registers in the loop over tiles.
template <int QB>
struct Seen {
  Visible v[QB];
  __device__ __forceinline__ Seen(const Kv4AttnArgs& a, const Sequence& s, int m0) {
    asm volatile("" : "+s"(m0));
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const int n = Row(a, 0, m0 + 16 * qb + (int)(threadIdx.x & 15)).n;
      v[qb] = n < s.qn ? visible(a, s, n) : Visible{0, 0};
    }
  }
};

// This lane's query rows as the operand of the first product.  WIDE: the order of channels in which a lane's
// D / 4 neighbouring channels are its parts of the D / 32 products.
template <int D, int QB, bool WIDE>
struct Queries {
  bf16x8 q[QB][D / 32];
  __device__ __forceinline__ void load(const Kv4AttnArgs& a, const Sequence& s, int b, int kvh, int m0) {
    const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const Row row(a, kvh, m0 + 16 * qb + r);
      // (a row that does not exist has any query)
      const size_t at = (size_t)b * a.q.sb + (size_t)(row.n < s.qn ? row.n : 0) * a.q.sn + (size_t)row.head * a.q.sh;
#pragma unroll
      for (int st = 0; st < D / 32; ++st)
        q[qb][st] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const block_u32x4_of2*>(a.qp + at + (WIDE ? g * (D / 4) + st * 8 : st * 32 + g * 8)));
    }
  }
};

typedef unsigned u32x2_of2 __attribute__((ext_vector_type(2), aligned(2)));

// ---- few rows ------------------------------------------------------------------------------------------------------

// The pages of every fourth tile from t on, four 16-key groups each: 16 tiles at a time wait in a register, one group to a lane, the next 16 are on
// their way.
struct GroupPages {
  int now, ahead, taken;
  __device__ __forceinline__ int fetch(const Kv4AttnArgs& a, const Tiles& tiles, const int32_t* row, int t, int t1) const {
    const int lane = threadIdx.x & 63;
    t += kWaves * (lane >> 2);
    if (t >= t1) return -1;
    const int entry = (tiles.at(t) * kTile + 16 * (lane & 3)) >> a.c.page_log2;
    return entry < a.c.max_pages ? row[entry] : -1;
  }
  __device__ __forceinline__ void open(const Kv4AttnArgs& a, const Tiles& tiles, const int32_t* row, int t, int t1) {
    taken = 0;
    ahead = fetch(a, tiles, row, t, t1);
  }
  // the pages of the next tile, t being the first of all; -1: not there
  __device__ __forceinline__ void next(const Kv4AttnArgs& a, const Tiles& tiles, const int32_t* row, int t, int t1, int (&page)[kGroups]) {
    const int at = taken & 15;
    if (at == 0) {
      now = ahead;
      asm volatile("" : "+v"(now));       // the copy first: the next ones then go to the register they are waited for in
      ahead = fetch(a, tiles, row, t + kWaves * (taken + 16), t1);
    }
    ++taken;
#pragma unroll
    for (int kb = 0; kb < kGroups; ++kb) {
      const int x = __builtin_amdgcn_readlane(now, 4 * at + kb);
      page[kb] = (unsigned)x < (unsigned)a.c.pages ? x : -1;
    }
  }
};

// A wavefront's tile in registers, as it comes from memory: the keys are asked for where those in front have gone into the scores, the
// values where those in front have gone to LDS.
template <int D>
struct RawTile {
  static constexpr int kKeyWords = D / 32;               // words of codes a lane has of a key
  static constexpr int kValueLoads = D / 32;             // 16 bytes each
  unsigned k[kGroups][kKeyWords];
  block_u32x4 v[kValueLoads];
  unsigned char ks[kGroups], vs[kValueLoads];
  const unsigned char* group[kGroups];                   // the groups' keys; the same in all lanes
  const unsigned char* scales[kGroups];
  int key0;
  unsigned missing;

  __device__ __forceinline__ void place(const Kv4AttnArgs& a, const unsigned char* head_data, size_t page_step, int key, const int (&page)[kGroups]) {
    key0 = key;
    missing = 0;
#pragma unroll
    for (int kb = 0; kb < kGroups; ++kb) {
      missing |= page[kb] < 0 ? 1u << kb : 0u;
      const unsigned char* const record = head_data + (unsigned)max(page[kb], 0) * page_step;
      const unsigned at = (unsigned)(key + 16 * kb) & ((1u << a.c.page_log2) - 1);
      group[kb] = record + at * (D / 2);
      scales[kb] = record + (unsigned)a.c.key_scales() + at * (D / 32);
    }
  }
  __device__ __forceinline__ void load_keys() {
    const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
#pragma unroll
    for (int kb = 0; kb < kGroups; ++kb) {
      const unsigned char* const p = group[kb] + (unsigned)(r * (D / 2) + g * (D / 8));
      if constexpr (D == 128) {
        const block_u32x4 x = *reinterpret_cast<const block_u32x4*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) k[kb][e] = x[e];
      } else {
        const u32x2 x = *reinterpret_cast<const u32x2*>(p);
        k[kb][0] = x[0];
        k[kb][1] = x[1];
      }
      ks[kb] = scales[kb][(unsigned)(r * (D / 32) + (D == 128 ? g : g >> 1))];
    }
  }
  // load i: D = 128: 16 keys, four lanes each; D = 64: 32 keys, two lanes each
  __device__ __forceinline__ void load_value(const Kv4AttnArgs& a, int i) {
    const int lane = threadIdx.x & 63;
    const int v_codes = a.c.values(), v_scales = a.c.value_scales() - a.c.key_scales();
    if constexpr (D == 128) {
      v[i] = *reinterpret_cast<const block_u32x4*>(group[i] + v_codes + (unsigned)(lane * 16));
      vs[i] = (scales[i] + v_scales)[(unsigned)lane];
    } else {
      const unsigned char* const from = lane < 32 ? group[2 * i] : group[2 * i + 1];
      const unsigned char* const scale = lane < 32 ? scales[2 * i] : scales[2 * i + 1];
      v[i] = *reinterpret_cast<const block_u32x4*>(from + v_codes + (lane & 31) * 16);
      vs[i] = scale[v_scales + (lane & 31)];
    }
  }
};

// Wavefronts to a SIMD: enough that the others' work covers a trip to memory.
constexpr int rows_waves(int D, int QB) { return D == 64 ? (QB == 1 ? 4 : 3) : QB == 1 ? 3 : 2; }

template <int D, int QB>
__global__ __launch_bounds__(64 * kWaves, rows_waves(D, QB)) void kv4_rows_kernel(Kv4AttnArgs a) {
  constexpr int DS = D / 32, CB = D / 16, BM = 16 * QB;
  constexpr int STAGE = 32 * 2 * D;                      // half a tile of values
  constexpr int MERGE = BM * D * 4;                      // a wavefront's results
  constexpr int OWN = STAGE > MERGE ? STAGE : MERGE;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kWaves * OWN];
  __shared__ float2 merged[kWaves][BM];
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // parts innermost
  unsigned id = blockIdx.x;
  const int part = __builtin_amdgcn_readfirstlane(id % a.parts);
  id /= a.parts;
  const int tile_m = id % a.tiles;
  const int kvh = __builtin_amdgcn_readfirstlane(id / a.tiles);
  const Part cut = parts_from(a, true, part);
  const int b = __builtin_amdgcn_readfirstlane(cut.b);
  if (b < 0) return;
  const int m0 = __builtin_amdgcn_readfirstlane(tile_m * BM);
  const Sequence s(a, b);
  const int n0 = __builtin_amdgcn_readfirstlane(m0 / a.group);
  if (n0 >= s.qn) return;
  const int n1 = min((m0 + BM - 1) / a.group, s.qn - 1);
  const int sink = a.window >= 0 ? a.sink : 0;
  const Visible lo = visible_uniform(a, s, n0), hi = visible_uniform(a, s, n1);
  const Tiles tiles(lo, hi, sink);
  const int t0 = part_of(tiles.count, part - cut.first, cut.count), t1 = part_of(tiles.count, part - cut.first + 1, cut.count);
  const int32_t* const table_row = a.c.table + (size_t)b * a.c.max_pages;

  Queries<D, QB, true> rows;
  rows.load(a, s, b, kvh, m0);
  f32x4 o[CB][QB] = {};
  float m[QB], l[QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    m[qb] = kLowest;
    l[qb] = 0.f;
  }
  unsigned long long far_lanes = 0;
  unsigned char* const own = lds + wave * OWN;
  int v_off[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) v_off[cb] = value_slot<D>(4 * g + (r >> 2), cb) + ((r & 3) << 3);

  const unsigned char* const head_data = a.c.data + (size_t)kvh * a.c.record();
  const size_t page_step = (size_t)a.c.H * a.c.record();
  constexpr int LOADS = RawTile<D>::kValueLoads;
  RawTile<D> raw;
  GroupPages pages;
  const int first = t0 + wave;
  pages.open(a, tiles, table_row, first, t1);
  auto place = [&](int t) {
    int page[kGroups];
    pages.next(a, tiles, table_row, first, t1, page);
    raw.place(a, head_data, page_step, tiles.at(t) * kTile, page);
  };
  if (first < t1) {
    place(first);
    raw.load_keys();
#pragma unroll
    for (int i = 0; i < LOADS; ++i) raw.load_value(a, i);
  }
  for (int t = first; t < t1; t += kWaves) {
    const int key0 = raw.key0;
    const unsigned missing = raw.missing;
    f32x4 sc[kGroups][QB];
#pragma unroll
    for (int kb = 0; kb < kGroups; ++kb) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) sc[kb][qb] = f32x4{0.f, 0.f, 0.f, 0.f};
      const float scale = power_of(raw.ks[kb]);
#pragma unroll
      for (int st = 0; st < DS; ++st) {
        const bf16x8 k = dequantise8(raw.k[kb][st], scale);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) sc[kb][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, rows.q[qb][st], sc[kb][qb], 0, 0, 0);
      }
    }
    // (behind the last tile the same one again)
    place(min(t + kWaves, t1 - 1));
    raw.load_keys();
    const bool whole = key0 + kTile <= lo.end && (key0 >= hi.begin || key0 + kTile <= sink) && !missing;
    if (!whole) mask_tile<QB>(sc, Seen<QB>(a, s, m0).v, sink, key0, missing, g);
    bf16x8 p[kGroups / 2][QB];
    take_tile<QB, CB>(sc, p, m, l, o, a.scale_log2, far_lanes);
    // values that are not finite, and those that nobody sees, which may be anything
    unsigned long long odd[LOADS];
    bool any_odd = false;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int row = D == 128 ? 16 * i + (lane >> 2) : 32 * i + (lane >> 1);
      const bool gone = key0 + row >= hi.end || (missing >> (row >> 4) & 1) != 0;
      odd[i] = __builtin_amdgcn_ballot_w64(gone || not_finite(raw.vs[i]));
      if (odd[i]) {
        const bool bad = !gone && not_finite(raw.vs[i]);
        odd[i] = __builtin_amdgcn_ballot_w64(bad);
        any_odd |= odd[i] != 0;
        if (gone || bad) {
          raw.v[i] = block_u32x4{0, 0, 0, 0};
          raw.vs[i] = 127;
        }
      }
    }
#pragma unroll
    for (int ks = 0; ks < kGroups / 2; ++ks) {
#pragma unroll
      for (int x = 0; x < LOADS / 2; ++x) {
        const int i = ks * (LOADS / 2) + x;
        const int row = D == 128 ? 16 * x + (lane >> 2) : lane >> 1, block = D == 128 ? lane & 3 : lane & 1;
        const float scale = power_of(raw.vs[i]);
#pragma unroll
        for (int w = 0; w < 4; ++w)
          *reinterpret_cast<bf16x8*>(own + value_slot<D>(row, 2 * block + (w >> 1)) + (w & 1) * 16) = dequantise8(raw.v[i][w], scale);
        raw.load_value(a, i);
      }
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        const unsigned char* const src = own + v_off[cb];
        const i16x4 first_keys = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)src);
        const i16x4 second_keys = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(src + 16 * 2 * D));
        const bf16x8 v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(first_keys, second_keys, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) o[cb][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[ks][qb], o[cb][qb], 0, 0, 0);
      }
    }
    if (any_odd) {
#pragma unroll 1
      for (int i = 0; i < LOADS; ++i) {
        unsigned long long hits = 0;
#pragma unroll
        for (int x = 0; x < LOADS; ++x) hits = x == i ? odd[x] : hits;
        while (hits) {
          const int at = __builtin_ctzll(hits);
          hits &= hits - 1;
          poison<QB, CB>(o, Seen<QB>(a, s, m0).v, sink, key0 + (D == 128 ? 16 * i + (at >> 2) : 32 * i + (at >> 1)), D == 128 ? at & 3 : at & 1);
        }
      }
    }
  }

  // ---- the wavefronts' results joined
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) l[qb] = quarters_sum(l[qb]);
  if (g == 0)
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) merged[wave][16 * qb + r] = float2{m[qb], l[qb]};
  __syncthreads();
  float* const sums = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    float top = m[qb];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, merged[w][16 * qb + r].x);
    const float f = __builtin_amdgcn_exp2f(m[qb] - top);
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
      *reinterpret_cast<f32x4*>(sums + (wave * BM + 16 * qb + r) * D + ((4 * cb + g) ^ r) * 4) = o[cb][qb] * f;
  }
  __syncthreads();
  constexpr int PIECES = D / 4;
  const size_t first_row = ((size_t)part * a.c.H + kvh) * a.rows + m0;
  for (int u = threadIdx.x; u < BM * PIECES; u += 64 * kWaves) {
    const int row = u / PIECES, piece = u % PIECES;
    const int mm = m0 + row, n = mm / a.group;
    if (n >= s.qn) continue;
    float top = kLowest, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, merged[w][row].x);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += merged[w][row].y * __builtin_amdgcn_exp2f(merged[w][row].x - top);
    f32x4 x = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) x += *reinterpret_cast<const f32x4*>(sums + (w * BM + row) * D + (piece ^ (row & 15)) * 4);
    if (a.part != nullptr) {
      const size_t at = first_row + row;
      *reinterpret_cast<f32x4*>(a.part + at * D + piece * 4) = x;
      if (piece == 0) a.stats[at] = float2{top, sum};
      continue;
    }
    const int head = kvh * a.group + (mm - n * a.group);
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const bf16x4 y = __builtin_convertvector(x * inv, bf16x4);
    *reinterpret_cast<u32x2_of2*>(a.op + (size_t)b * a.o.sb + (size_t)n * a.o.sn + (size_t)head * a.o.sh + piece * 4) = __builtin_bit_cast(u32x2, y);
    if (piece == 0 && a.lse)
      a.lse[((size_t)b * a.c.H * a.group + head) * a.N + n] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
  }
}

// ---- many rows -----------------------------------------------------------------------------------------------------

// The pages of a wavefront's 16 keys of the tiles t0, t0 + 1, ..: 64 at a time wait in a register, one to a lane, the next 64 are on their way.
struct PageList {
  int now, ahead, taken;
  __device__ __forceinline__ int fetch(const Kv4AttnArgs& a, const Tiles& tiles, const int32_t* row, int t, int t1, int wave) const {
    t += (int)(threadIdx.x & 63);
    if (t >= t1) return -1;
    const int entry = (tiles.at(t) * kTile + 16 * wave) >> a.c.page_log2;
    return entry < a.c.max_pages ? row[entry] : -1;
  }
  __device__ __forceinline__ void open(const Kv4AttnArgs& a, const Tiles& tiles, const int32_t* row, int t0, int t1, int wave) {
    taken = 0;
    ahead = fetch(a, tiles, row, t0, t1, wave);
  }
  // the page of tile t0 + taken, or -1
  __device__ __forceinline__ int next(const Kv4AttnArgs& a, const Tiles& tiles, const int32_t* row, int t0, int t1, int wave) {
    const int lane = taken & 63;
    if (lane == 0) {
      now = ahead;
      asm volatile("" : "+v"(now));       // the copy first: the next 64 then go to the register they are waited for in
      ahead = fetch(a, tiles, row, t0 + taken + 64, t1, wave);
    }
    ++taken;
    const int page = __builtin_amdgcn_readlane(now, lane);
    return (unsigned)page < (unsigned)a.c.pages ? page : -1;
  }
};

// The loop is skewed by one tile, as in svg_attn_kernel.h: with the scores of tile j in registers a wavefront takes their exponentials and then issues
// the products of tile j + 1's scores and of tile j's output as one batch; the first operands of a batch are read in front of the exponentials, every
// other one behind the products.  Keys of tile j + 2 and values of j + 1 are dequantised into LDS meanwhile, those behind them are on their way
// from memory; one barrier a tile.  At D = 128 (40 x 4680 rows over 32760 keys, three runs each in turn) 2.80-2.81 ms; with batches that the compiler may
// reorder 3.02; without the wavefront's priority over its batch the same, at D = 64 (48 x 4050 rows in a window) 750-775 us for 716-765.
template <int D>
struct TileLds {
  static constexpr int HALF = kTile * 2 * D;             // a tile of keys, or of values
  __attribute__((aligned(1024))) unsigned char tiles[4 * HALF];      // keys, keys, values, values
  unsigned long long odd_values[2][kWaves];              // threads of a wavefront whose values are not finite
  unsigned flags[2][kWaves];                             // bit 0: the 16 keys' page is not there; bit 1: some value is not finite
};

// Row tile, part and head of the cache number `id`.
template <int D>
__device__ __forceinline__ void attend_tile(const Kv4AttnArgs& a, TileLds<D>& shared, unsigned id) {
  constexpr int QB = 2, DS = D / 32, CB = D / 16, BM = 32 * kWaves;
  constexpr int WORDS = D / 32;                          // words of codes that a thread stages of a tile's keys, and of its values
  constexpr int HALF = TileLds<D>::HALF;
  constexpr int NS = kGroups * DS, NV = kGroups / 2 * CB; // operands of the two products
  // Of them in registers, measured on the calls above: at D = 128 4 and 8 ahead alike, 12 2.86-2.90 ms; at D = 64 2 and 4 alike, 8 845-865 us.
  constexpr int AHEAD = D == 128 ? 8 : 4;
  // At D = 128 2.80-2.81 ms where one tile after the other takes 2.88-2.90; at D = 64 733-751 us skewed (with 8 ahead 919, two wavefronts to a SIMD 822) and
  // 716-765 not: alike, so the shorter program.
  constexpr bool SKEWED = D == 128;
  unsigned char* const lds = shared.tiles;
  auto& odd_values = shared.odd_values;
  auto& flags = shared.flags;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int tile_m = id % a.tiles;
  id /= a.tiles;
  const int part = __builtin_amdgcn_readfirstlane(id / a.c.H);
  const int kvh = __builtin_amdgcn_readfirstlane(id - part * a.c.H);
  const Part cut = parts_from(a, true, part);
  const int b = __builtin_amdgcn_readfirstlane(cut.b);
  if (b < 0) return;
  const int m0 = __builtin_amdgcn_readfirstlane(tile_m * BM);
  const Sequence s(a, b);
  const int n0 = __builtin_amdgcn_readfirstlane(m0 / a.group);
  if (n0 >= s.qn) return;
  const int n1 = min((m0 + BM - 1) / a.group, s.qn - 1);
  const int sink = a.window >= 0 ? a.sink : 0;
  const Visible lo = visible_uniform(a, s, n0), hi = visible_uniform(a, s, n1);
  const Tiles tiles(lo, hi, sink);
  const int t0 = part_of(tiles.count, part - cut.first, cut.count), t1 = part_of(tiles.count, part - cut.first + 1, cut.count);
  const int32_t* const table_row = a.c.table + (size_t)b * a.c.max_pages;
  // What this wavefront's rows see, all of them and any of them; of rows that do not exist nothing is written, whatever they see.  A wavefront
  // without rows stages its share and computes nothing.
  const int wm0 = m0 + 32 * wave, wn0 = __builtin_amdgcn_readfirstlane(wm0 / a.group), wn1 = min(__builtin_amdgcn_readfirstlane((wm0 + 31) / a.group), s.qn - 1);
  const bool active = wn0 < s.qn;
  const Visible wlo = visible_uniform(a, s, min(wn0, s.qn - 1)), whi = visible_uniform(a, s, wn1);

  Queries<D, QB, false> rows;
  rows.load(a, s, b, kvh, wm0);
  f32x4 o[CB][QB] = {}, sc[kGroups][QB];
  float m[QB], l[QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    m[qb] = kLowest;
    l[qb] = 0.f;
  }
  unsigned long long far_lanes = 0;

  // ---- staging: a wavefront has 16 keys of a tile, which are in one page; four threads a key
  struct Raw {
    unsigned w[WORDS];
    unsigned char scale;
  };
  // The wavefront's keys of a tile: the first of them, and where they lie; the same in all lanes.
  struct Place {
    int key;
    bool missing;
    const unsigned char *codes, *scales;               // of the keys; the values' lie a fixed distance behind
  };
  const int sub = tid & 3, stage_row = tid >> 2;
  const int code_at = (lane >> 2) * (D / 2) + sub * (D / 8), scale_at = (lane >> 2) * (D / 32) + (D == 128 ? sub : sub >> 1);
  const int v_codes = a.c.values(), v_scales = a.c.value_scales() - a.c.key_scales();
  const unsigned char* const head_data = a.c.data + (size_t)kvh * a.c.record();
  const size_t page_step = (size_t)a.c.H * a.c.record();
  PageList pages;
  pages.open(a, tiles, table_row, t0, t1, wave);
  // tile t0, t0 + 1, .. in turn
  int next_t = t0, next_key = tiles.at(t0) * kTile + 16 * wave;
  auto next_place = [&]() -> Place {
    Place x;
    const int page = pages.next(a, tiles, table_row, t0, t1, wave);
    x.key = __builtin_amdgcn_readfirstlane(next_key);
    x.missing = page < 0;
    const unsigned char* const record = head_data + (unsigned)max(page, 0) * page_step;
    const unsigned place = x.key & ((1 << a.c.page_log2) - 1);
    x.codes = record + place * (D / 2);
    x.scales = record + (unsigned)a.c.key_scales() + place * (D / 32);
    next_key = x.key + kTile;
    if (++next_t == tiles.sink_tiles) next_key = tiles.first * kTile + 16 * wave;
    return x;
  };
  auto load = [&](Raw& x, const unsigned char* codes, const unsigned char* scales) {
    if constexpr (D == 128) {
      const block_u32x4 y = *reinterpret_cast<const block_u32x4*>(codes + code_at);
#pragma unroll
      for (int e = 0; e < 4; ++e) x.w[e] = y[e];
    } else {
      const u32x2 y = *reinterpret_cast<const u32x2*>(codes + code_at);
      x.w[0] = y[0];
      x.w[1] = y[1];
    }
    x.scale = scales[scale_at];
  };
  // Keys that nobody sees may be anything: scores are replaced, so keys may be staged as they are.
  auto stage_k = [&](const Raw& x, int buffer) {
    const float scale = power_of(x.scale);
#pragma unroll
    for (int w = 0; w < WORDS; ++w)
      *reinterpret_cast<bf16x8*>(lds + buffer * HALF + key_piece<D>(stage_row, WORDS * sub + w)) = dequantise8(x.w[w], scale);
  };
  // A value that is not finite would not be taken away by its weight of zero.
  auto stage_v = [&](Raw& x, const Place& at, int buffer) {
    const bool gone = at.missing || at.key + (lane >> 2) >= hi.end;
    unsigned long long odd = __builtin_amdgcn_ballot_w64(gone || not_finite(x.scale));
    if (odd) {
      const bool bad = !gone && not_finite(x.scale);
      odd = __builtin_amdgcn_ballot_w64(bad);
      if (gone || bad) {
#pragma unroll
        for (int w = 0; w < WORDS; ++w) x.w[w] = 0;
        x.scale = 127;
      }
    }
    const float scale = power_of(x.scale);
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      const int piece = WORDS * sub + w;
      *reinterpret_cast<bf16x8*>(lds + (2 + buffer) * HALF + value_slot<D>(stage_row, piece >> 1) + (piece & 1) * 16) = dequantise8(x.w[w], scale);
    }
    if (lane == 0) {
      flags[buffer][wave] = (at.missing ? 1u : 0u) | (odd ? 2u : 0u);
      if (odd) odd_values[buffer][wave] = odd;
    }
  };

  int k_off[DS], v_off[CB];
#pragma unroll
  for (int st = 0; st < DS; ++st) k_off[st] = key_piece<D>(r, 4 * st + g);       // (16 rows on, the swizzle is the same)
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) v_off[cb] = value_slot<D>(4 * g + (r >> 2), cb) + ((r & 3) << 3);
  auto k_operand = [&](int buffer, int i) -> bf16x8 {
    return *reinterpret_cast<const bf16x8*>(lds + buffer * HALF + (i / DS) * 16 * 2 * D + k_off[i % DS]);
  };
  auto v_operand = [&](int buffer, int i) -> bf16x8 {
    const unsigned char* const src = lds + (2 + buffer) * HALF + (i / CB) * 32 * 2 * D + v_off[i % CB];
    const i16x4 first = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)src);
    const i16x4 second = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(src + 16 * 2 * D));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(first, second, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  bf16x8 operand[AHEAD];
  auto read_keys = [&](int buffer) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) operand[i] = k_operand(buffer, i);
  };
  // scores of the tile in `buffer`, whose first operands are in registers; the operands behind its own are the values in v_buffer
  auto scores = [&](int buffer, auto values, int v_buffer) {
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const bf16x8 k = operand[i % AHEAD];
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int qb = 0; qb < QB; ++qb)
        sc[i / DS][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, rows.q[qb][i % DS], i % DS ? sc[i / DS][qb] : f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
      if (i + AHEAD < NS) operand[i % AHEAD] = k_operand(buffer, i + AHEAD);
      else if constexpr (decltype(values)::value) operand[i % AHEAD] = v_operand(v_buffer, i + AHEAD - NS);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  if (t0 < t1) {
    // Tiles behind the last one are staged too, from any place, and never looked at.
    Raw k_raw, v_raw;
    Place p1 = next_place();
    load(k_raw, p1.codes, p1.scales);
    load(v_raw, p1.codes + v_codes, p1.scales + v_scales);
    int key0 = p1.key - 16 * wave;
    Place p2 = next_place();
    stage_k(k_raw, 0);
    load(k_raw, p2.codes, p2.scales);
    stage_v(v_raw, p1, 0);
    p1 = p2;
    load(v_raw, p1.codes + v_codes, p1.scales + v_scales);
    if constexpr (SKEWED) {
      p2 = next_place();
      stage_k(k_raw, 1);
      load(k_raw, p2.codes, p2.scales);
    }
    __syncthreads();
    if constexpr (SKEWED) {
      if (active) {
        read_keys(0);
        scores(0, std::false_type{}, 0);
      }
      __syncthreads();
    }

    auto needs = [&](int key) { return key < whi.end && (key + kTile > wlo.begin || key < sink); };
    // p1: the tile whose values are on their way; p2: the tile whose keys are, one behind it where the loop is skewed
    auto trip = [&](auto half) {
      constexpr int buffer = decltype(half)::value;
      const int next_key0 = p1.key - 16 * wave;
      const unsigned flag = flags[buffer][lane & 3];
      read_keys(SKEWED ? buffer ^ 1 : buffer);
      __builtin_amdgcn_sched_barrier(0);
      // the next tiles into LDS: their places were last read before the barrier
      stage_k(k_raw, SKEWED ? buffer : buffer ^ 1);
      stage_v(v_raw, p1, buffer ^ 1);
      if constexpr (!SKEWED) p2 = next_place();
      p1 = p2;
      load(v_raw, p1.codes + v_codes, p1.scales + v_scales);
      if constexpr (SKEWED) p2 = next_place();
      load(k_raw, p2.codes, p2.scales);
      __builtin_amdgcn_sched_barrier(0);
      // skewed, the scores are of the tile behind this one: a wavefront that needs one of the two takes both, with weights of zero for the other
      if (active && (needs(key0) || (SKEWED && needs(next_key0)))) {
        if constexpr (!SKEWED) {
          __builtin_amdgcn_s_setprio(1);
          scores(buffer, std::true_type{}, buffer);
          __builtin_amdgcn_s_setprio(0);
        }
        const unsigned gone = (unsigned)__builtin_amdgcn_ballot_w64((flag & 1) != 0) & 15u;
        const bool whole = key0 + kTile <= wlo.end && (key0 >= whi.begin || key0 + kTile <= sink) && !gone;
        if (!whole) mask_tile<QB>(sc, Seen<QB>(a, s, wm0).v, sink, key0, gone, g);
        bf16x8 p[kGroups / 2][QB];
        take_tile<QB, CB>(sc, p, m, l, o, a.scale_log2, far_lanes);
        __builtin_amdgcn_s_setprio(1);
        if constexpr (SKEWED) scores(buffer ^ 1, std::true_type{}, buffer);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const bf16x8 v = operand[(NS + i) % AHEAD];
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) o[i % CB][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[i / CB][qb], o[i % CB][qb], 0, 0, 0);
          if (i + AHEAD < NV) operand[(NS + i) % AHEAD] = v_operand(buffer, i + AHEAD);
          __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        if (__builtin_amdgcn_ballot_w64((flag & 2) != 0)) {
#pragma unroll 1
          for (int w = 0; w < kWaves; ++w) {
            unsigned long long hits = flags[buffer][w] & 2 ? odd_values[buffer][w] : 0;
            while (hits) {
              const int at = __builtin_ctzll(hits);
              hits &= hits - 1;
              poison<QB, CB>(o, Seen<QB>(a, s, wm0).v, sink, key0 + 16 * w + (at >> 2), D == 128 ? at & 3 : (at & 3) >> 1);
            }
          }
        }
      }
      key0 = next_key0;
      __syncthreads();
    };
    for (int t = t0;;) {
      trip(std::integral_constant<int, 0>{});
      if (++t >= t1) break;
      trip(std::integral_constant<int, 1>{});
      if (++t >= t1) break;
    }
  }

#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const float sum = quarters_sum(l[qb]);
    const Row row(a, kvh, wm0 + 16 * qb + r);
    if (row.n >= s.qn) continue;
    if (a.part != nullptr) {
      const size_t at = ((size_t)part * a.c.H + kvh) * a.rows + wm0 + 16 * qb + r;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) *reinterpret_cast<f32x4*>(a.part + at * D + 16 * cb + 4 * g) = o[cb][qb];
      if (g == 0) a.stats[at] = float2{m[qb], sum};
      continue;
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    __bf16* const to = a.op + (size_t)b * a.o.sb + (size_t)row.n * a.o.sn + (size_t)row.head * a.o.sh;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
      *reinterpret_cast<u32x2_of2*>(to + 16 * cb + 4 * g) = __builtin_bit_cast(u32x2, __builtin_convertvector(o[cb][qb] * inv, bf16x4));
    if (g == 0 && a.lse)
      a.lse[((size_t)b * a.c.H * a.group + row.head) * a.N + row.n] =
          sum == 0.f ? -INFINITY : (m[qb] + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
  }
}

// Neighbouring row tiles of a head on one XCD, whose L2 they share: an XCD has an eighth of them.
template <int D>
__global__ __launch_bounds__(64 * kWaves, D == 128 ? 2 : 3) void kv4_tiles_kernel(Kv4AttnArgs a) {
  __shared__ TileLds<D> shared;
  const unsigned all = (unsigned)a.c.H * (unsigned)a.tiles * (unsigned)a.parts, per_xcd = (all + 7) / 8;
  const unsigned id = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  if (blockIdx.x >> 3 < per_xcd && id < all) attend_tile<D>(a, shared, id);
}

// ---- parts of the keys joined -----------------------------------------------------------------------------------------

// D / 4 lanes have four channels each and GROUPS such sets of lanes a row, every GROUPS-th part each; they add up through LDS in the order of their
// number.  Eight sets where rows are few, so that all parts are on their way at once (64 parts of eight sequences' tokens 7 -> 4.8 us), else one.
template <int D, int GROUPS>
__global__ __launch_bounds__(256) void kv4_join_kernel(Kv4AttnArgs a) {
  constexpr int LANES = D / 4, ROWS = 256 / (LANES * GROUPS);
  __shared__ f32x4 part_o[GROUPS > 1 ? ROWS : 1][GROUPS][LANES];
  __shared__ float part_sum[GROUPS > 1 ? ROWS : 1][GROUPS];
  const int b = blockIdx.y;
  const Part cut = parts_from(a, false, b);
  const int piece = threadIdx.x % LANES, set = threadIdx.x / LANES % GROUPS, own = threadIdx.x / (LANES * GROUPS);
  const long long row = (long long)blockIdx.x * ROWS + own, of_sequence = (long long)a.c.H * a.rows;
  const int kvh = (int)(min(row, of_sequence - 1) / a.rows), m = (int)(min(row, of_sequence - 1) - (long long)kvh * a.rows);
  const Sequence s(a, b);
  const Row at(a, kvh, m);
  const bool there = row < of_sequence && at.n < s.qn;
  const size_t step = (size_t)a.c.H * a.rows, first = (size_t)cut.first * step + (size_t)kvh * a.rows + m;
  const int count = there ? cut.count : 0;
  // the reference of all parts, a part to a lane
  float top = kLowest;
  for (int x = piece; x < count; x += LANES) top = fmaxf(top, a.stats[first + x * step].x);
#pragma unroll
  for (int d = LANES / 2; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, LANES));
  float sum = 0.f;
  f32x4 o = {};
#pragma unroll 4
  for (int x = set; x < count; x += GROUPS) {
    const float2 st = a.stats[first + x * step];
    const f32x4 y = *reinterpret_cast<const f32x4*>(a.part + (first + x * step) * D + piece * 4);
    const float f = __builtin_amdgcn_exp2f(st.x - top);
    sum += st.y * f;
    o += y * f;
  }
  if constexpr (GROUPS > 1) {
    part_o[own][set][piece] = o;
    if (piece == 0) part_sum[own][set] = sum;
    __syncthreads();
    if (set > 0) return;
#pragma unroll
    for (int x = 1; x < GROUPS; ++x) {
      o += part_o[own][x][piece];
      sum += part_sum[own][x];
    }
  }
  if (!there) return;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  *reinterpret_cast<u32x2_of2*>(a.op + (size_t)b * a.o.sb + (size_t)at.n * a.o.sn + (size_t)at.head * a.o.sh + piece * 4) =
      __builtin_bit_cast(u32x2, __builtin_convertvector(o * inv, bf16x4));
  if (piece == 0 && a.lse)
    a.lse[((size_t)b * a.c.H * a.group + at.head) * a.N + at.n] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}

}  // namespace

// Which form, and in how many parts?  What is estimated to take the least time: with c workgroups on the fullest of 256 compute units and t
// turns of a workgroup (a tile for each of its four wavefronts, in the form with 128 rows one for all),
//     begin + begin_more c + t (turn + turn_more c)       microseconds,
// the last round of workgroups counted by its own c, and for parts the launch that joins them, 4.5 and what they take to write and read at 5 TB/s.
// Fitted to the times of 276 calls with 1 to 64 heads of 1 to 1000 rows over 300 to 60000 keys, each cut in up to eight ways: the way
// taken is within 15 % of the best of these ways, 2 % on the average (which says nothing of how far all of them are from a floor).  Measured, chosen way and its neighbours: 4 x 64 rows of 64 channels over 272 keys 7.2 us
// in tiles of 16 rows, 8.8 of 32; 24 x 48 of 128 over 20000 42 and 39; 24 x 226 of 128 over 12000 61 in tiles of 128, 81 of 32; 40 x 800 of 64 over 12000, which
// are 280 tiles of 128 for 768 places, 164 in tiles of 32, 185 of 128.  8 x 64 of 128 over 1000 keys 12.3 in four parts, 13.2 in one; 24 x 48 14.9 and 13.3.
struct FormTimes {
  float begin, begin_more, turn, turn_more;
};
constexpr FormTimes kFormTimes[3][2] = {      // tiles of 16, 32 and 128 rows; 64 and 128 channels
    {{3.7f, 1.23f, 0.87f, 0.34f}, {3.9f, 1.5f, 1.3f, 0.61f}},
    {{4.2f, 1.8f, 0.77f, 0.58f}, {5.f, 2.1f, 0.98f, 1.f}},
    {{7.1f, 1.f, 0.56f, 0.41f}, {9.1f, 0.6f, 1.01f, 0.4f}}};
constexpr int kUnits = 256;                   // compute units

Kv4Plan kv4_plan(const Kv4& c, const svg_kv4_attn_t& attn, long long N, int group) {
  Kv4Plan p = {};
  p.rows = (int)(N * group);
  // keys that a row tile visits, about (one across two blocks visits up to a block more)
  const long long capacity = (long long)c.max_pages << c.page_log2;
  long long keys = attn.max_kv > 0 ? std::min<long long>(attn.max_kv, capacity) : capacity;
  if (attn.window >= 0 && attn.causal) keys = std::min(keys, (attn.window + 1ll) * attn.block + std::min<long long>(attn.sink, keys) + 128);
  p.reach = (int)keys;
  const long long tiles = (keys + kTile - 1) / kTile;
  float best = std::numeric_limits<float>::infinity();
  auto consider = [&](int form, int rows, long long parts) {
    const FormTimes& x = kFormTimes[form][c.D == 128];
    const long long row_tiles = std::max(1, (p.rows + rows - 1) / rows), groups = c.H * row_tiles * parts;
    // Parts are dealt by length: fewer than two for each sequence cut only some of them, from there on none is much longer than the others.
    const long long cut = parts < 2ll * c.B ? std::min<long long>(parts, c.B) : parts, a_turn = (rows == 128 ? 1 : kWaves) * std::max(1ll, cut);
    const long long turns = (tiles * c.B + a_turn - 1) / a_turn;
    // (the forms with 16 and 32 rows slow down evenly with more workgroups, whether they are on the card or wait)
    const long long together = rows == 128 ? (c.D == 128 ? 2 : 3) * kUnits : std::max(groups, 1ll);
    const long long full = groups / together, rest = groups % together;
    auto on = [&](long long n) { return (float)((n + kUnits - 1) / kUnits); };
    float time = x.begin + x.begin_more * on(std::min(groups, together)) +
                 (float)turns * ((float)full * (x.turn + x.turn_more * on(together)) + (rest ? x.turn + x.turn_more * on(rest) : 0.f));
    if (parts > c.B) time += 4.5f + (float)parts * (float)c.H * (float)p.rows * (float)c.D * (8 / 5e6f);
    if (time < best) {
      best = time;
      p.tile = rows;
      p.tiles = (int)row_tiles;
      p.parts = (int)parts;
    }
  };
  constexpr int kRows[3] = {16, 32, 128};
  for (int form = 0; form < 3; ++form) {
    const int rows = kRows[form];
    // (32 rows for 16, or 128 for 64 and fewer, are never faster)
    if ((rows == 32 && p.rows <= 16) || (rows == 128 && p.rows <= 64)) continue;
    const long long each = (long long)c.H * std::max(1, (p.rows + rows - 1) / rows);
    // Beyond the calls that the times were fitted to (several sequences, whole rounds of workgroups) the form with more rows.  90 calls of 3 to 64 sequences of 33 to
    // 581 rows that this decides, both ways: the estimate's own choice takes 1.02 times as long on the geometric average, 0.64 to 1.35 (128 rows for 32: D = 64 0.98,
    // D = 128 1.05; 32 for 16: 1.02 and 0.99).
    if ((rows == 16 && p.rows > 16 && each * c.B > 4 * kUnits) || (rows == 32 && p.rows > 64 && each * c.B > 5 * kUnits)) continue;
    consider(form, rows, c.B);
    // parts for one, two or three workgroups to a compute unit, of a turn (128 rows: 8 tiles) at least
    const long long most = c.B * (rows == 128 ? tiles / 8 : (tiles + kWaves - 1) / kWaves);
    for (int places = kUnits; places <= (rows == 128 && c.D == 64 ? 3 : 2) * kUnits; places += kUnits) {
      long long parts = std::min(places / each, most);
      if (c.B > 64) parts -= parts % c.B;
      if (parts > c.B) consider(form, rows, parts);
    }
  }
  return p;
}

size_t kv4_workspace_bytes(const Kv4& c, const Kv4Plan& p) {
  return p.parts > c.B ? (size_t)p.parts * c.H * (size_t)p.rows * ((size_t)c.D * 4 + 8) : 0;
}

int launch_kv4_attn(const Kv4& c, const svg_kv4_attn_t& attn, const Kv4Plan& plan, const HeadRows& q, const void* qp, const HeadRows& o,
                    void* op, int group, float* lse, void* workspace, hipStream_t stream) {
  Kv4AttnArgs a = {};
  a.c = c;
  a.q = q;
  a.o = o;
  a.qp = static_cast<const __bf16*>(qp);
  a.op = static_cast<__bf16*>(op);
  a.lse = lse;
  a.kv_len = attn.kv_len;
  a.q_len = attn.q_len;
  a.N = plan.rows / group;
  a.group = group;
  a.rows = plan.rows;
  a.tiles = plan.tiles;
  a.parts = plan.parts;
  a.reach = plan.reach;
  if (plan.parts > c.B) {
    a.part = static_cast<float*>(workspace);
    a.stats = reinterpret_cast<float2*>(a.part + (size_t)plan.parts * c.H * plan.rows * c.D);
  }
  a.causal = attn.causal;
  a.block = attn.block;
  a.window = attn.window;
  a.sink = attn.sink;
  a.capacity = c.pages ? c.max_pages << c.page_log2 : 0;      // (without a pool there is nothing that a load could be sent to)
  const float scale = attn.softmax_scale > 0.f ? attn.softmax_scale : 1.f / sqrtf((float)c.D);
  a.scale_log2 = scale * 1.4426950408889634f;
  const long long blocks = (long long)c.H * plan.tiles * plan.parts;
  if (blocks > (1ll << 24) - 8) return SVG_ERR_UNSUPPORTED;      // a launch has fewer than 2^32 threads
  (void)hipGetLastError();
  const bool wide = c.D == 128;
  if (plan.tile == 128) {
    hipLaunchKernelGGL((wide ? kv4_tiles_kernel<128> : kv4_tiles_kernel<64>), dim3((unsigned)((blocks + 7) / 8 * 8)), dim3(64 * kWaves), 0, stream, a);
  } else if (plan.tile == 32)
    hipLaunchKernelGGL((wide ? kv4_rows_kernel<128, 2> : kv4_rows_kernel<64, 2>), dim3((unsigned)blocks), dim3(64 * kWaves), 0, stream, a);
  else
    hipLaunchKernelGGL((wide ? kv4_rows_kernel<128, 1> : kv4_rows_kernel<64, 1>), dim3((unsigned)blocks), dim3(64 * kWaves), 0, stream, a);
  if (plan.parts > c.B) {
    const long long rows = (long long)c.H * plan.rows;        // of a sequence
    const bool few = rows * c.B <= 2048;
    const int per_block = 256 / (c.D / 4) / (few ? 8 : 1);
    auto kernel = wide ? (few ? kv4_join_kernel<128, 8> : kv4_join_kernel<128, 1>) : few ? kv4_join_kernel<64, 8> : kv4_join_kernel<64, 1>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((rows + per_block - 1) / per_block), (unsigned)c.B), dim3(256), 0, stream, a);
  }
  return hip_status(hipGetLastError());
}

}  // namespace svg
