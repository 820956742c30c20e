// Gate, residual, norm and modulation between two branches of a layer, and its gradients.  HBM-bound: the forward pass
// reads x and y and writes r and h, the backward pass reads r, y, dr, dh and writes dx, dy; a row is read once and stays in
// registers from its statistics to its outputs.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "svg_attn_common.h"
#include "svg_block.h"

namespace svg {

namespace {

constexpr int kMaxWaves = 16;         // wavefronts of a workgroup
constexpr int kMaxChannels = 16384;
constexpr int kFewGroups = 8;

struct GateNormArgs {
  long long rows;
  int C, groups;
  int post, pre;
  float alpha, post_eps, eps;
  long long ld_x, ld_y, ld_r, ld_h, ld_mod;
  const float *gate, *scale, *shift;
  const int32_t* group_ptr;
  long long group_rows;               // rows of a group where there is no group_ptr
  const float *post_weight, *post_bias, *weight, *bias;
  const void *x, *y, *r_in, *dr, *dh;
  void *r, *h, *dx, *dy;
  unsigned* codes;
  unsigned char* scales;
  int col_tiles, col_groups;
  long long row_limit;                // rows, with a 4-bit output rounded up to whole tiles
  int strip;                          // neighbouring rows that a workgroup takes in turn
  int waves;                          // wavefronts of a workgroup
  float* partial;                     // backward: [slots][4][C]
};

// The group of a row: how many of the ends group_ptr[1 .. groups-1] are not above it; in range whatever the table holds.  end: the
// first row that may belong to another one.
__device__ __forceinline__ int group_of(const GateNormArgs& a, long long row, long long& end) {
  end = a.rows;
  if (a.groups == 1) return 0;
  if (!a.group_ptr) {
    const unsigned g = (unsigned)row / (unsigned)a.group_rows;
    end = (long long)(g + 1) * a.group_rows;
    return (int)g;
  }
  int lo = 0, hi = a.groups - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if ((long long)a.group_ptr[mid] <= row) lo = mid;
    else hi = mid - 1;
  }
  if (lo + 1 < a.groups) end = a.group_ptr[lo + 1];
  return lo;
}

// ---------------------------------------------------------------------------------------------------------------------
// A workgroup holds a row, eight neighbouring channels a lane and 512 a wavefront (VPL times), and takes the rows of a
// strip in turn.  Rows that are 16-byte aligned come through LDS: every wavefront asks
// for its part of the row D rows ahead, straight from memory into a ring of its own, so that 80 to 120 KB are on their way to a
// compute unit whatever registers the row in work needs.
// A ring is written and read by its own wavefront alone: no barrier, a count of its outstanding operations is enough.
// Rows of any other alignment come from the 16-byte granules that they touch: the granules of 504 channels fill the same 1 or 2 KB
// wherever the row begins, and are read out of LDS from its first byte on.  Rows that LDS has no place for, or of more channels than 16
// wavefronts of two such vectors hold, come in registers, one row ahead, in loads of eight elements at any address.
// (In registers, 32760 x 5119 takes 377 us forward and 1024 backward.)
constexpr int kSegment = 512;         // channels of a wavefront and vector
enum Form { kWhole, kShifted, kSingle };                  // aligned rows; granules in LDS; in registers
__host__ __device__ constexpr int segment(Form form) { return form == kShifted ? 504 : kSegment; }

// The lane's eight channels of one tensor in the ring.
template <int TYPE, bool ANY>
__device__ __forceinline__ void read_ring(const unsigned char* at, float (&x)[8]) {
  const int lane = threadIdx.x & 63;
  if constexpr (ANY) {                // lane 63 has none
    load8_any<TYPE>(at, (unsigned)min(lane, 62) * 8, x);
  } else if constexpr (TYPE == SVG_F32) {
    const block_f32x4* p = reinterpret_cast<const block_f32x4*>(at + lane * 32);
    const block_f32x4 lo = p[0], hi = p[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[e] = lo[e]; x[4 + e] = hi[e]; }
  } else if constexpr (TYPE == SVG_BF16) {
    const block_u32x4 w = *reinterpret_cast<const block_u32x4*>(at + lane * 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  } else {
    const block_f16x8 h = *reinterpret_cast<const block_f16x8*>(at + lane * 16);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)h[e];
  }
}

// A tensor's rows: the wavefront's part of one goes to the ring in loads of 1 KB; what is behind the last channel, or of a
// row that does not exist, arrives as zeros.
template <int TYPE, int VPL, Form FORM>
struct Rows {
  static constexpr int size = type_bytes(TYPE);
  static constexpr int loads = VPL * kSegment * 2 / 1024 * (size / 2);
  static constexpr int bytes = VPL * kSegment * size;
  const char* base;
  size_t step;                        // bytes of a row
  // bytes from the row's first granule to its first element
  __device__ __forceinline__ unsigned shift(long long row) const {
    return FORM == kShifted ? (unsigned)(reinterpret_cast<uintptr_t>(base) + (size_t)row * step) & 15u : 0u;
  }
  __device__ __forceinline__ void ask(long long row, bool there, int C, int waves, int wave, unsigned to) const {
    const unsigned past = there ? shift(row) : 0;         // granules lie in the allocation that their elements lie in
    const auto rsrc = attn::buffer_words(base + (there ? (size_t)row * step - past : 0),
                                         there && base ? (past + (unsigned)C * size + 3u) & ~3u : 0u);
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int v = 0; v < VPL; ++v)
#pragma unroll
      for (int l = 0; l < loads / VPL; ++l)
        load_one_to_lds(rsrc, lane * 16, (wave + v * waves) * segment(FORM) * size + l * 1024, to + v * kSegment * size + l * 1024);
  }
};

template <int VPL, Form FORM>
struct Lane {
  static constexpr int N = VPL * 8;
  static constexpr bool ANY = FORM != kWhole;
  int first, step, C;                 // channel of vector v, element e: first + v step + e
  __device__ __forceinline__ Lane(int C_, int waves, int wave) : step(waves * segment(FORM)), C(C_) {
    const int lane = threadIdx.x & 63;
    first = lane * 8 < segment(FORM) ? wave * segment(FORM) + lane * 8 : kMaxChannels;
  }
  __device__ __forceinline__ int at(int i) const { return first + i / 8 * step + i % 8; }
  __device__ __forceinline__ bool has(int i) const { return (ANY ? at(i) : at(i / 8 * 8)) < C; }
  __device__ __forceinline__ bool whole(int v) const { return at(v * 8) + (ANY ? 7 : 0) < C; }
  template <int TYPE>
  __device__ __forceinline__ void read(const unsigned char* ring, float (&x)[N]) const {
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      float t[8];
      read_ring<TYPE, ANY>(ring + v * kSegment * type_bytes(TYPE), t);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v * 8 + e] = !ANY || has(v * 8 + e) ? t[e] : 0.f;
    }
  }
  // Results of 16 bits are not kept in L2: a tensor of this size leaves it before it is read again.  Where a line is
  // written in parts (fp32: half of it by each store; rows off its borders), L2 has to join them.
  template <int TYPE>
  __device__ __forceinline__ void store(void* base, size_t row, const float (&x)[N]) const {
    char* const p = static_cast<char*>(base) + row * type_bytes(TYPE);
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      const unsigned c = (unsigned)at(v * 8);
      const float t[8] = {x[v * 8], x[v * 8 + 1], x[v * 8 + 2], x[v * 8 + 3], x[v * 8 + 4], x[v * 8 + 5], x[v * 8 + 6], x[v * 8 + 7]};
      if constexpr (ANY) {
        if (whole(v)) {
          store8_any<TYPE>(p, c, t);
        } else {
#pragma unroll
          for (int e = 0; e < 7; ++e)
            if (has(v * 8 + e)) store1<TYPE>(p, c + e, t[e]);
        }
      } else {
        if (!whole(v)) continue;
        block_u32x4* const q = reinterpret_cast<block_u32x4*>(p + c * (unsigned)type_bytes(TYPE));
        const block_f32x8 f = {t[0], t[1], t[2], t[3], t[4], t[5], t[6], t[7]};
        if constexpr (TYPE == SVG_F32) {
          q[0] = __builtin_bit_cast(block_u32x4, block_f32x4{f[0], f[1], f[2], f[3]});
          q[1] = __builtin_bit_cast(block_u32x4, block_f32x4{f[4], f[5], f[6], f[7]});
        } else if constexpr (TYPE == SVG_BF16) {
          __builtin_nontemporal_store(__builtin_bit_cast(block_u32x4, __builtin_convertvector(f, block_bf16x8)), q);
        } else {
          __builtin_nontemporal_store(__builtin_bit_cast(block_u32x4, __builtin_convertvector(f, block_f16x8)), q);
        }
      }
    }
  }
  // a parameter vector, or `otherwise` where there is none; zero where the row has no channel
  __device__ __forceinline__ void table(const float* base, size_t row, float otherwise, float (&x)[N]) const {
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      float t[8] = {};
      const unsigned c = (unsigned)at(v * 8);
      if (!base) {
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = has(v * 8 + e) ? otherwise : 0.f;
      } else if (whole(v)) {
        if constexpr (ANY) load8_any<SVG_F32>(base + row, c, t);
        else load8<SVG_F32>(base + row, c, t);
      } else if constexpr (ANY) {
#pragma unroll
        for (int e = 0; e < 7; ++e)
          if (has(v * 8 + e)) t[e] = base[row + c + e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v * 8 + e] = t[e];
    }
  }
};

// A lane's part of a row of any alignment, on its way into registers.  The lane that holds the row's end reads the row's last eight
// elements and moves them to their places when they are used: loads of single elements would have to be waited for at once.  Where
// some of the eight are another wavefront's, which may be writing the row in place, it takes its own one by one.
template <int TYPE, int VPL>
struct Coming {
  using Word = std::conditional_t<TYPE == SVG_F32, block_u32x4_of4, block_u32x4_of2>;
  static constexpr int kWords = TYPE == SVG_F32 ? 2 : 1;
  block_u32x4 w[VPL][kWords];
  __device__ __forceinline__ void ask(const void* base, size_t row, const Lane<VPL, kSingle>& lane) {
    const char* const p = static_cast<const char*>(base) + row * type_bytes(TYPE);
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      const int c = lane.at(v * 8);
#pragma unroll
      for (int k = 0; k < kWords; ++k) w[v][k] = block_u32x4{};
      if (base && c < lane.C) {
        if (c + 8 <= lane.C || c % kSegment) {
          const Word* const q = reinterpret_cast<const Word*>(p + (unsigned)min(c, lane.C - 8) * (unsigned)type_bytes(TYPE));
#pragma unroll
          for (int k = 0; k < kWords; ++k) w[v][k] = q[k];
        } else {
#pragma unroll
          for (int e = 0; e < 7; ++e) {
            if (c + e >= lane.C) continue;
            if constexpr (TYPE == SVG_F32) w[v][e / 4][e % 4] = reinterpret_cast<const unsigned*>(p)[c + e];
            else w[v][0][e / 2] |= (unsigned)reinterpret_cast<const unsigned short*>(p)[c + e] << (e % 2 * 16);
          }
        }
      }
    }
  }
  __device__ __forceinline__ void read(const Lane<VPL, kSingle>& lane, float (&x)[VPL * 8]) const {
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      float t[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (TYPE == SVG_F32) {
          t[e] = __uint_as_float(w[v][e / 4][e % 4]);
        } else {
          const unsigned bits = w[v][0][e / 2];
          if constexpr (TYPE == SVG_BF16) t[e] = __uint_as_float(e % 2 ? bits & 0xffff0000u : bits << 16);
          else t[e] = (float)__builtin_bit_cast(_Float16, (unsigned short)(e % 2 ? bits >> 16 : bits));
        }
      }
      if (lane.C % 8) {
        const int c = lane.at(v * 8), past = c < lane.C && c % kSegment ? max(c + 8 - lane.C, 0) : 0;
#pragma unroll
        for (int by = 4; by; by /= 2)
#pragma unroll
          for (int e = 0; e < 8; ++e) t[e] = past & by ? (e + by < 8 ? t[(e + by) & 7] : 0.f) : t[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v * 8 + e] = t[e];
    }
  }
};

// What the wavefronts of a workgroup tell each other through LDS: up to four numbers each.  Two sets of places in turn, so that one
// barrier a time is enough: a wavefront writes a place again only behind the next barrier.  The barrier is a bare one: it need not
// wait for rows on their way.
struct Meeting {
  block_f32x4 (*place)[kMaxWaves];
  int turn, waves, wave;              // wavefronts, this one's number

  // mine of all wavefronts, that of wavefront l in lane l and zeros behind them
  __device__ __forceinline__ block_f32x4 tell(block_f32x4 mine) {
    const int lane = threadIdx.x & 63;
    if (waves == 1) return lane == 0 ? mine : block_f32x4{};
    block_f32x4* const here = place[turn];
    if (lane == 0) here[wave] = mine;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    attn::barrier_loads_done();
    turn ^= 1;
    return lane < waves ? here[lane] : block_f32x4{};
  }
  __device__ __forceinline__ void sums(float& p, float& q) {
    p = wave_sum(p);
    q = wave_sum(q);
    if (waves == 1) return;
    const block_f32x4 all = tell({p, q, 0.f, 0.f});
    p = wave_sum(all[0]);
    q = wave_sum(all[1]);
  }
};

// A row's normalisation, v -> (v - mean) rho.  A wavefront takes the mean of its own n channels first and the squares of what is left
// then, and the wavefronts' pairs are joined by  sum of squares = sum over w of (squares_w + n_w (mean_w - mean)^2): a row far
// from zero loses nothing, and one meeting is enough.
template <int VPL, Form FORM>
__device__ __forceinline__ void own_statistics(const float (&v)[VPL * 8], int norm, const Lane<VPL, FORM>& lane, float inv_n, float& mean, float& squares) {
  mean = squares = 0.f;
  if (norm == SVG_NORM_NONE) return;
  if (norm == SVG_NORM_LAYER) {
#pragma unroll
    for (int i = 0; i < VPL * 8; ++i) mean += v[i];       // zeros where there is no channel
    mean = wave_sum(mean) * inv_n;
  }
#pragma unroll
  for (int i = 0; i < VPL * 8; ++i) {
    const float d = lane.has(i) ? v[i] - mean : 0.f;
    squares = __builtin_fmaf(d, d, squares);
  }
  squares = wave_sum(squares);
}
// mean_w and squares_w of wavefront w in lane w, n its channels there
__device__ __forceinline__ void join_statistics(float& mean, float& squares, float n, float inv) {
  const float all = wave_sum(n * mean) * inv, d = mean - all;
  squares = wave_sum(__builtin_fmaf(n * d, d, squares));
  mean = all;
}
template <int VPL, Form FORM>
__device__ __forceinline__ float apply_statistics(float (&v)[VPL * 8], int norm, float mean, float squares, float inv, float eps, const Lane<VPL, FORM>& lane) {
  if (norm == SVG_NORM_NONE) return 1.0f;
  const float rho = 1.0f / sqrtf(squares * inv + eps);
#pragma unroll
  for (int i = 0; i < VPL * 8; ++i) v[i] = lane.has(i) ? (v[i] - mean) * rho : 0.f;
  return rho;
}

template <int VPL, Form FORM>
struct Team {
  int wave;
  Lane<VPL, FORM> lane;
  Meeting meet;
  float inv_n, n_of_lane, inv;        // 1 / channels of this wavefront; channels of wavefront `lane`; 1 / C
  __device__ __forceinline__ Team(const GateNormArgs& a, block_f32x4 (*places)[kMaxWaves])
      : wave(__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6))), lane(a.C, a.waves, wave), meet{places, 0, a.waves, wave} {
    auto channels = [&](int w) {
      int n = 0;
      for (int v = 0; v < VPL; ++v) n += min(max(a.C - (w + v * a.waves) * segment(FORM), 0), segment(FORM));
      return (float)n;
    };
    inv_n = 1.0f / channels(wave);
    n_of_lane = (int)(threadIdx.x & 63) < a.waves ? channels(threadIdx.x & 63) : 0.f;
    inv = 1.0f / (float)a.C;
  }
  __device__ __forceinline__ float normalise(float (&v)[VPL * 8], int norm, float eps) {
    if (norm == SVG_NORM_NONE) return 1.0f;
    float mean, squares;
    own_statistics<VPL, FORM>(v, norm, lane, inv_n, mean, squares);
    const block_f32x4 all = meet.tell({mean, squares, 0.f, 0.f});
    mean = all[0];
    squares = all[1];
    join_statistics(mean, squares, n_of_lane, inv);
    return apply_statistics<VPL, FORM>(v, norm, mean, squares, inv, eps, lane);
  }
};

// Ends every load that the compiler knows of where a group begins.  It would wait for them, and with them for all rows on their way, where
// the paths with and without a new group meet, once a row.
__device__ __forceinline__ void wait_tables() { __builtin_amdgcn_s_waitcnt(0x0f70); }      // vmcnt(0)

// Waits until at most N of this wavefront's operations on memory are outstanding (they end in order).
template <int N>
__device__ __forceinline__ void wait_ring() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N < 63 ? N : 63) : "memory"); }

// The forward pass.  The tables of a group stay in registers, folded with the norms' weights: r = alpha x + (G1 yhat + G0),
// h = H1 rhat + H0.  With a 4-bit output five wavefronts a SIMD are asked for: the 101 registers that it takes otherwise leave a compute
// unit to one row of ten wavefronts (32760 x 5120 299 -> 245 us).  A spilt register in the loop would cost more: its reload waits for
// the rows on their way.
template <int TS, int TB, int VPL, int D, Form FORM, bool FP4>
__global__ __launch_bounds__(64 * kMaxWaves, FP4 && VPL == 1 ? 5 : 4) void gate_norm_kernel(GateNormArgs a) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  __shared__ block_f32x4 places[2][kMaxWaves];
  constexpr bool SINGLE = FORM == kSingle;
  Team<VPL, FORM> team(a, places);
  constexpr int N = VPL * 8;
  using X = Rows<TS, VPL, FORM>;
  using Y = Rows<TB, VPL, FORM>;
  const X xs{static_cast<const char*>(a.x), (size_t)a.ld_x * X::size};
  const Y ys{static_cast<const char*>(a.y), (size_t)a.ld_y * Y::size};
  constexpr int kSlot = X::bytes + Y::bytes, kLoads = X::loads + Y::loads;
  // stores of a row at least, where r and h (or its 4-bit form) are wanted: only the first vector is sure to have a channel
  constexpr int kStores = FORM == kWhole ? X::size / 2 + (FP4 ? 2 : 1) : 2;
  unsigned char* const ring = lds + (threadIdx.x >> 6) * (D * kSlot);
  const unsigned ring0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)ring);
  const long long r0 = (long long)blockIdx.x * a.strip;
  Coming<TS, VPL> next_x;
  Coming<TB, VPL> next_y;
  auto ask = [&](int k) {
    const bool there = k < a.strip && r0 + k < a.rows;
    if constexpr (SINGLE) {
      if (!there) return;
      next_x.ask(a.x, (size_t)(r0 + k) * a.ld_x, team.lane);
      next_y.ask(a.y, (size_t)(r0 + k) * a.ld_y, team.lane);
      return;
    }
    const unsigned to = ring0 + (unsigned)(k % (SINGLE ? 1 : D)) * kSlot;
    xs.ask(r0 + k, there, a.C, a.waves, team.wave, to);
    ys.ask(r0 + k, there, a.C, a.waves, team.wave, to + X::bytes);
  };
  const bool second = a.h || FP4, counted = a.r && (FP4 || a.h);
  float g1[N], g0[N], h1[N], h0[N];
  int group = -1;
  long long group_end = 0;
#pragma unroll
  for (int k = 0; k < (SINGLE ? 1 : D); ++k) ask(k);
  const int turns = (int)min((long long)a.strip, a.row_limit - r0);
  for (int k = 0; k < turns; ++k) {
    const long long row = r0 + k;
    const bool there = row < a.rows;
    // the tables' loads run beside those of the first rows
    if (there && row >= group_end) {
      const int now = group_of(a, row, group_end);
      if (now != group) {
        group = now;
        const size_t mod = (size_t)now * a.ld_mod;
        float t[N];
        if (a.y) {
          team.lane.table(a.gate, mod, 1.0f, g1);
          team.lane.table(a.post == SVG_NORM_LAYER ? a.post_bias : nullptr, 0, 0.0f, g0);
          team.lane.table(a.post != SVG_NORM_NONE ? a.post_weight : nullptr, 0, 1.0f, t);
#pragma unroll
          for (int i = 0; i < N; ++i) {
            g0[i] *= g1[i];
            g1[i] *= t[i];
          }
        }
        if (second) {
          team.lane.table(a.scale, mod, 0.0f, t);
          team.lane.table(a.pre != SVG_NORM_NONE ? a.weight : nullptr, 0, 1.0f, h1);
          team.lane.table(a.pre == SVG_NORM_LAYER ? a.bias : nullptr, 0, 0.0f, h0);
#pragma unroll
          for (int i = 0; i < N; ++i) {
            h0[i] *= 1.0f + t[i];
            h1[i] *= 1.0f + t[i];
          }
          team.lane.table(a.shift, mod, 0.0f, t);
#pragma unroll
          for (int i = 0; i < N; ++i) h0[i] += t[i];
        }
      }
      wait_tables();
    }
    float v[N], y[N];
    if constexpr (SINGLE) {
      next_x.read(team.lane, v);
      next_y.read(team.lane, y);
      ask(k + 1);
    } else {
      // row k's loads are in front of those of D - 1 rows and, from row D on, of D rows' stores
      if (counted && k >= D) wait_ring<(D - 1) * kLoads + D * kStores>();
      else wait_ring<(D - 1) * kLoads>();
      const unsigned char* const slot = ring + (unsigned)(k % D) * kSlot;
      team.lane.template read<TS>(slot + xs.shift(row), v);
      team.lane.template read<TB>(slot + X::bytes + ys.shift(row), y);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the slot has been read
      ask(k + D);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] *= a.alpha;
    if (a.y) {
      team.normalise(y, a.post, a.post_eps);
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += __builtin_fmaf(g1[i], y[i], g0[i]);
    }
    if (a.r && there) team.lane.template store<TS>(a.r, (size_t)row * a.ld_r, v);
    if (second) {
      team.normalise(v, a.pre, a.eps);
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = __builtin_fmaf(v[i], h1[i], h0[i]);
      if (a.h && there) team.lane.template store<TB>(a.h, (size_t)row * a.ld_h, v);
    }
    if constexpr (FP4) {
      const long long rt = row / kFp4Rows;
      const int i16 = (int)(row % kFp4Rows);
#pragma unroll
      for (int k8 = 0; k8 < VPL; ++k8) {
        float t[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = there && team.lane.has(k8 * 8) ? v[k8 * 8 + e] : 0.f;      // the padding
        const int c = team.lane.at(k8 * 8), ct = c / kFp4Cols, g = (c >> 5) & 3;
        const unsigned s = fp4_scale(quad_max(magnitude8(t)));
        if (ct < a.col_tiles) a.codes[((size_t)rt * a.col_tiles + ct) * 256 + g * 64 + i16 * 4 + ((c >> 3) & 3)] = fp4_codes8(t, s);
        if ((c & 31) == 0 && ct < a.col_groups * kFp4Group)
          a.scales[(((size_t)rt * a.col_groups + ct / kFp4Group) * 64 + g * 16 + i16) * 4 + ct % kFp4Group] = (unsigned char)s;
      }
    }
  }
  if constexpr (!SINGLE) wait_ring<0>();           // no load to LDS outlives the workgroup
}

// Gradients of a strip of rows.  What the parameters get are four sums over the rows of a group and channel:
//   S1 = sum dh, S2 = sum dh rhat, T1 = sum dR, T2 = sum dR yhat   (dR: gradient of r)
//   dshift = S1, dscale = weight S2 + bias S1, dgate = post_weight T2 + post_bias T1,
//   dweight = sum over g of (1 + scale) S2, dbias the same of S1, dpost_weight = sum over g of gate T2, dpost_bias of T1.
// They stay in registers while the strip is in one group and go to slot (workgroup + group), of which every pair that has
// rows has one of its own, because neither number ever falls along the rows.
template <int TS, int TB, int VPL, int D, Form FORM>
__global__ __launch_bounds__(64 * kMaxWaves) void gate_norm_grad_kernel(GateNormArgs a) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  __shared__ block_f32x4 places[2][kMaxWaves];
  constexpr bool SINGLE = FORM == kSingle;
  Team<VPL, FORM> team(a, places);
  constexpr int N = VPL * 8;
  using S = Rows<TS, VPL, FORM>;
  using B = Rows<TB, VPL, FORM>;
  const S rs{static_cast<const char*>(a.r_in), (size_t)a.ld_r * S::size}, drs{static_cast<const char*>(a.dr), (size_t)a.ld_r * S::size};
  const B ys{static_cast<const char*>(a.y), (size_t)a.ld_y * B::size}, dhs{static_cast<const char*>(a.dh), (size_t)a.ld_h * B::size};
  constexpr int kSlot = 2 * (S::bytes + B::bytes), kLoads = 2 * (S::loads + B::loads), kStores = FORM == kWhole ? S::size / 2 + 1 : 2;
  unsigned char* const ring = lds + (threadIdx.x >> 6) * (D * kSlot);
  const unsigned ring0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)ring);
  const long long r0 = (long long)blockIdx.x * a.strip;
  Coming<TS, VPL> next_r, next_dr;
  Coming<TB, VPL> next_y, next_dh;
  auto ask = [&](int k) {
    const bool there = k < a.strip && r0 + k < a.rows;
    if constexpr (SINGLE) {
      if (!there) return;
      next_r.ask(a.r_in, (size_t)(r0 + k) * a.ld_r, team.lane);
      next_dr.ask(a.dr, (size_t)(r0 + k) * a.ld_r, team.lane);
      next_y.ask(a.y, (size_t)(r0 + k) * a.ld_y, team.lane);
      next_dh.ask(a.dh, (size_t)(r0 + k) * a.ld_h, team.lane);
      return;
    }
    const unsigned to = ring0 + (unsigned)(k % (SINGLE ? 1 : D)) * kSlot;
    rs.ask(r0 + k, there, a.C, a.waves, team.wave, to);
    drs.ask(r0 + k, there, a.C, a.waves, team.wave, to + S::bytes);
    ys.ask(r0 + k, there, a.C, a.waves, team.wave, to + 2 * S::bytes);
    dhs.ask(r0 + k, there, a.C, a.waves, team.wave, to + 2 * S::bytes + B::bytes);
  };
  float s1[N] = {}, s2[N] = {}, t1[N] = {}, t2[N] = {};
  float e1[N], f1[N];                 // (1 + scale) weight, gate post_weight
  int group = -1;
  long long group_end = 0;
  auto flush = [&] {
    const size_t slot = (size_t)(blockIdx.x + (unsigned)group) * 4 * a.C;
    team.lane.template store<SVG_F32>(a.partial, slot, s1);
    team.lane.template store<SVG_F32>(a.partial, slot + a.C, s2);
    team.lane.template store<SVG_F32>(a.partial, slot + 2 * (size_t)a.C, t1);
    team.lane.template store<SVG_F32>(a.partial, slot + 3 * (size_t)a.C, t2);
  };
  const int pre = a.dh ? a.pre : SVG_NORM_NONE, post = a.y ? a.post : SVG_NORM_NONE;
  const bool counted = a.dx && a.dy;
#pragma unroll
  for (int k = 0; k < (SINGLE ? 1 : D); ++k) ask(k);
  const int turns = (int)min((long long)a.strip, a.rows - r0);
  for (int k = 0; k < turns; ++k) {
    const long long row = r0 + k;
    if (row >= group_end) {
      const int now = group_of(a, row, group_end);
      if (now != group) {
        if (group >= 0) {
          flush();
#pragma unroll
          for (int i = 0; i < N; ++i) s1[i] = s2[i] = t1[i] = t2[i] = 0.f;
        }
        group = now;
        const size_t mod = (size_t)now * a.ld_mod;
        float t[N];
        team.lane.table(a.scale, mod, 0.0f, e1);
        team.lane.table(a.pre != SVG_NORM_NONE ? a.weight : nullptr, 0, 1.0f, t);
#pragma unroll
        for (int i = 0; i < N; ++i) e1[i] = (1.0f + e1[i]) * t[i];
        team.lane.table(a.gate, mod, 1.0f, f1);
        team.lane.table(a.post != SVG_NORM_NONE ? a.post_weight : nullptr, 0, 1.0f, t);
#pragma unroll
        for (int i = 0; i < N; ++i) f1[i] *= t[i];
      }
      wait_tables();
    }
    float rhat[N], d[N], yhat[N], e[N];
    if constexpr (SINGLE) {
      next_r.read(team.lane, rhat);
      next_dr.read(team.lane, d);
      next_y.read(team.lane, yhat);
      next_dh.read(team.lane, e);
      ask(k + 1);
    } else {
      if (counted && k >= D) wait_ring<(D - 1) * kLoads + D * kStores>();
      else wait_ring<(D - 1) * kLoads>();
      const unsigned char* const slot = ring + (unsigned)(k % D) * kSlot;
      team.lane.template read<TS>(slot + rs.shift(row), rhat);
      team.lane.template read<TS>(slot + S::bytes + drs.shift(row), d);
      team.lane.template read<TB>(slot + 2 * S::bytes + ys.shift(row), yhat);
      team.lane.template read<TB>(slot + 2 * S::bytes + B::bytes + dhs.shift(row), e);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      ask(k + D);
    }
    // both normalisations' statistics in one meeting; a row that does not exist is zeros
    float rho = 1.0f, rho_y = 1.0f;
    if (pre != SVG_NORM_NONE || post != SVG_NORM_NONE) {
      float mr, sr, my, sy;
      own_statistics<VPL, FORM>(rhat, pre, team.lane, team.inv_n, mr, sr);
      own_statistics<VPL, FORM>(yhat, post, team.lane, team.inv_n, my, sy);
      const block_f32x4 all = team.meet.tell({mr, sr, my, sy});
      mr = all[0];
      sr = all[1];
      my = all[2];
      sy = all[3];
      if (pre != SVG_NORM_NONE) join_statistics(mr, sr, team.n_of_lane, team.inv);
      if (post != SVG_NORM_NONE) join_statistics(my, sy, team.n_of_lane, team.inv);
      rho = apply_statistics<VPL, FORM>(rhat, pre, mr, sr, team.inv, a.eps, team.lane);
      rho_y = apply_statistics<VPL, FORM>(yhat, post, my, sy, team.inv, a.post_eps, team.lane);
    }
    if (a.dh) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        s1[i] += e[i];
        s2[i] = __builtin_fmaf(e[i], rhat[i], s2[i]);
        e[i] *= e1[i];
      }
      if (pre != SVG_NORM_NONE) {
        float m1 = 0.f, m2 = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          m1 += e[i];
          m2 = __builtin_fmaf(e[i], rhat[i], m2);
        }
        team.meet.sums(m1, m2);
        m1 = pre == SVG_NORM_LAYER ? m1 * team.inv : 0.f;
        m2 *= team.inv;
        // places without a channel stay zero: they are part of the sums below
#pragma unroll
        for (int i = 0; i < N; ++i)
          d[i] = team.lane.has(i) ? __builtin_fmaf(rho, __builtin_fmaf(-rhat[i], m2, e[i] - m1), d[i]) : 0.f;
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) d[i] += e[i];
      }
    }
    if (a.dx) {
#pragma unroll
      for (int i = 0; i < N; ++i) e[i] = a.alpha * d[i];
      team.lane.template store<TS>(a.dx, (size_t)row * a.ld_x, e);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      t1[i] += d[i];
      t2[i] = __builtin_fmaf(d[i], yhat[i], t2[i]);
    }
    if (a.dy) {
#pragma unroll
      for (int i = 0; i < N; ++i) d[i] *= f1[i];
      if (post != SVG_NORM_NONE) {
        float m1 = 0.f, m2 = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          m1 += d[i];
          m2 = __builtin_fmaf(d[i], yhat[i], m2);
        }
        team.meet.sums(m1, m2);
        m1 = post == SVG_NORM_LAYER ? m1 * team.inv : 0.f;
        m2 *= team.inv;
#pragma unroll
        for (int i = 0; i < N; ++i) d[i] = rho_y * __builtin_fmaf(-yhat[i], m2, d[i] - m1);
      }
      team.lane.template store<TB>(a.dy, (size_t)row * a.ld_y, d);
    }
  }
  if constexpr (!SINGLE) wait_ring<0>();
  if (group >= 0) flush();
}

struct GradSumArgs {
  long long rows;
  int C, groups, strip, splits;
  const int32_t* group_ptr;
  long long group_rows;
  const float* partial;               // [slots][4][C]
  float* split;                       // [splits][groups][4][C]: sums of parts of the strips, where there is more than one
  float* total;                       // [groups][4][C], or null where no weight's gradient is wanted or the groups are few
  const float *post_weight, *post_bias, *weight, *bias;
  const float *gate, *scale;          // the forward pass's tables, [groups] rows of ld_mod
  long long ld_mod, ld_grad;
  float *dgate, *dscale, *dshift, *dpost_weight, *dpost_bias, *dweight, *dbias;
  bool has_post_weight, has_post_bias, has_weight, has_bias;        // does the norm have it?
};

constexpr int kSumLanes = 64;         // rows (slots, splits, groups) that are summed side by side
constexpr int kSumChannels = 16;

// Adds up the four sums of 16 channels over the workgroup's 64 rows of threads, in parts of `rows` of them (a multiple of 4):
// part p's result is in row p.
__device__ __forceinline__ void fold_rows(float (&s)[4], int rows = kSumLanes) {
  __shared__ float lds[kSumLanes / 4][4][kSumChannels];
  const int c = threadIdx.x % kSumChannels, wave = threadIdx.x >> 6, part = threadIdx.x / kSumChannels;
#pragma unroll
  for (int j = 0; j < 4; ++j) {       // the four rows of a wavefront
    const unsigned u = __float_as_uint(s[j]);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const unsigned v = __float_as_uint(__uint_as_float(a[0]) + __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    s[j] = __uint_as_float(b[0]) + __uint_as_float(b[1]);
  }
  if ((threadIdx.x & 63) < kSumChannels)
#pragma unroll
    for (int j = 0; j < 4; ++j) lds[wave][j][c] = s[j];
  __syncthreads();
  if (part * rows < kSumLanes)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s[j] = lds[part * rows / 4][j][c];
      for (int q = 1; q < rows / 4; ++q) s[j] += lds[part * rows / 4 + q][j][c];
    }
  __syncthreads();
}

// The gradients of group g, channel c, from its sums.
__device__ __forceinline__ void finish_group(const GradSumArgs& a, int g, int c, const float (&s)[4]) {
  const size_t at = (size_t)g * a.ld_grad + c;
  if (a.dshift) a.dshift[at] = s[0];
  if (a.dscale) a.dscale[at] = (a.weight ? a.weight[c] : 1.f) * s[1] + (a.bias ? a.bias[c] : 0.f) * s[0];
  if (a.dgate) a.dgate[at] = (a.post_weight ? a.post_weight[c] : 1.f) * s[3] + (a.post_bias ? a.post_bias[c] : 0.f) * s[2];
  if (a.total) {
#pragma unroll
    for (int j = 0; j < 4; ++j) a.total[((size_t)g * 4 + j) * a.C + c] = s[j];
  }
}

// Adds a group's sums under its modulation to those of the weights' gradients.
__device__ __forceinline__ void add_weights(const GradSumArgs& a, int g, int c, const float (&p)[4], float (&s)[4]) {
  const float scale = a.scale ? 1.0f + a.scale[(size_t)g * a.ld_mod + c] : 1.0f;
  const float gate = a.gate ? a.gate[(size_t)g * a.ld_mod + c] : 1.0f;
  s[0] = __builtin_fmaf(scale, p[0], s[0]);
  s[1] = __builtin_fmaf(scale, p[1], s[1]);
  s[2] = __builtin_fmaf(gate, p[2], s[2]);
  s[3] = __builtin_fmaf(gate, p[3], s[3]);
}
// What a norm does not have takes no part in the forward pass: its gradient is zero, whatever the sums hold.
__device__ __forceinline__ void write_weights(const GradSumArgs& a, int c, const float (&s)[4]) {
  if (a.dbias) a.dbias[c] = a.has_bias ? s[0] : 0.f;
  if (a.dweight) a.dweight[c] = a.has_weight ? s[1] : 0.f;
  if (a.dpost_bias) a.dpost_bias[c] = a.has_post_bias ? s[2] : 0.f;
  if (a.dpost_weight) a.dpost_weight[c] = a.has_post_weight ? s[3] : 0.f;
}

// The strips that have rows of group g: first to end - 1.
__device__ __forceinline__ void group_strips(const GradSumArgs& a, int g, long long& first, long long& end) {
  long long lo = 0, hi = a.rows;
  if (a.groups > 1) {
    if (a.group_ptr) {
      if (g > 0) lo = min(max((long long)a.group_ptr[g], 0ll), a.rows);
      if (g + 1 < a.groups) hi = min(max((long long)a.group_ptr[g + 1], 0ll), a.rows);
    } else {
      lo = g * a.group_rows;
      hi = lo + a.group_rows;
    }
  }
  first = lo < hi ? lo / a.strip : 0;
  end = lo < hi ? (hi - 1) / a.strip + 1 : 0;
}

// Few groups: their sums side by side, each by `lanes` rows of threads, from the strips' (or from the parts' where SPLIT), and all
// gradients from them.  One launch instead of two: 2971 x 1536 in four groups 15.6 -> 10.8 us.
template <bool SPLIT>
__global__ __launch_bounds__(kSumLanes* kSumChannels) void grad_few_kernel(GradSumArgs a, int lanes) {
  __shared__ float lds[kFewGroups][4][kSumChannels];
  const int i = threadIdx.x % kSumChannels, c = blockIdx.x * kSumChannels + i, k = threadIdx.x / kSumChannels, g = k / lanes;
  float s[4] = {};
  if (g < a.groups && c < a.C) {
    long long b = 0, end = a.splits;
    if constexpr (!SPLIT) group_strips(a, g, b, end);
#pragma unroll 4
    for (b += k % lanes; b < end; b += lanes) {
      const float* p = SPLIT ? a.split + ((size_t)b * a.groups + g) * 4 * a.C + c : a.partial + (size_t)(b + g) * 4 * a.C + c;
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] += p[(size_t)j * a.C];
    }
  }
  fold_rows(s, lanes);
  if (k < a.groups && c < a.C) {
    finish_group(a, k, c, s);
    float w[4] = {};
    add_weights(a, k, c, s, w);
#pragma unroll
    for (int j = 0; j < 4; ++j) lds[k][j][i] = w[j];
  }
  __syncthreads();
  if (k == 0 && c < a.C) {
    for (int j = 0; j < 4; ++j) s[j] = lds[0][j][i];
    for (int h = 1; h < a.groups; ++h)
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] += lds[h][j][i];
    write_weights(a, c, s);
  }
}

// The sums of a group from the slots of the strips that have rows of it; blockIdx.z: a part of the strips.
__global__ __launch_bounds__(kSumLanes* kSumChannels) void grad_groups_kernel(GradSumArgs a) {
  const int c = blockIdx.x * kSumChannels + threadIdx.x % kSumChannels, k = threadIdx.x / kSumChannels;
  for (int g = blockIdx.y; g < a.groups; g += gridDim.y) {
    long long first, end;
    group_strips(a, g, first, end);
    float s[4] = {};
    if (c < a.C) {
      const long long part = (end - first + a.splits - 1) / a.splits;
      const long long b1 = min(end, first + ((long long)blockIdx.z + 1) * part);
#pragma unroll 4
      for (long long b = first + blockIdx.z * part + k; b < b1; b += kSumLanes) {
        const float* p = a.partial + (size_t)(b + g) * 4 * a.C + c;
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] += p[(size_t)j * a.C];
      }
    }
    fold_rows(s);
    if (k == 0 && c < a.C) {
      if (a.splits == 1) {
        finish_group(a, g, c, s);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) a.split[(((size_t)blockIdx.z * a.groups + g) * 4 + j) * a.C + c] = s[j];
      }
    }
  }
}

// The parts' sums, and the gradients of the groups.
__global__ __launch_bounds__(kSumLanes* kSumChannels) void grad_splits_kernel(GradSumArgs a) {
  const int c = blockIdx.x * kSumChannels + threadIdx.x % kSumChannels, k = threadIdx.x / kSumChannels;
  for (int g = blockIdx.y; g < a.groups; g += gridDim.y) {
    float s[4] = {};
    if (c < a.C)
      for (int z = k; z < a.splits; z += kSumLanes)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] += a.split[(((size_t)z * a.groups + g) * 4 + j) * a.C + c];
    fold_rows(s);
    if (k == 0 && c < a.C) finish_group(a, g, c, s);
  }
}

// The weights' gradients of several groups: the groups' sums under their modulation.
__global__ __launch_bounds__(kSumLanes* kSumChannels) void grad_weights_kernel(GradSumArgs a) {
  const int c = blockIdx.x * kSumChannels + threadIdx.x % kSumChannels, k = threadIdx.x / kSumChannels;
  float s[4] = {};
  if (c < a.C)
    for (int g = k; g < a.groups; g += kSumLanes) {
      const float* t = a.total + (size_t)g * 4 * a.C + c;
      const float p[4] = {t[0], t[a.C], t[2 * (size_t)a.C], t[3 * (size_t)a.C]};
      add_weights(a, g, c, p, s);
    }
  fold_rows(s);
  if (k == 0 && c < a.C) write_weights(a, c, s);
}

// Wavefronts of a workgroup, vectors of a lane: 512 channels a wavefront and vector, one vector up to 8192 channels, two up to 16384.
struct RowShape { int waves, vpl; };
RowShape row_shape(int C, Form form = kWhole) {
  const int vectors = (C + segment(form) - 1) / segment(form), vpl = vectors <= kMaxWaves ? 1 : 2;
  return {(vectors + vpl - 1) / vpl, vpl};
}

// Rows that a workgroup has on their way, at `slot` bytes a wavefront and row: three, or what LDS holds; 0: not one.
constexpr int kRingBytes = 155 << 10;
int ring_depth(int waves, int slot) { return std::min(3, kRingBytes / (waves * slot)); }

// Rows of a strip, so that the workgroups that are resident at one time take them all.  `most`: wavefronts of a compute unit that
// the registers allow.  Forward, rows that make strips of two or three were slower one to a workgroup, by 18 % in bf16, 11 with an fp32 stream and 22
// with a 4-bit output in the geometric mean of 70 sizes each from 256 to 8192 channels (6 % faster to 39 % slower).
int strip_rows(long long rows, int waves, int most, int bytes) {
  const int resident = std::max(1, std::min(most / waves, bytes ? kRingBytes / bytes : most));
  return (int)std::max(1ll, (rows + 256ll * resident - 1) / (256ll * resident));
}

GateNormArgs gate_norm_args(const svg_gate_norm_t& d) {
  GateNormArgs a = {};
  a.rows = a.row_limit = d.rows;
  a.C = d.C; a.groups = d.groups;
  a.post = d.post_norm; a.pre = d.pre_norm;
  a.alpha = d.residual_scale; a.post_eps = d.post_eps; a.eps = d.eps;
  a.ld_x = d.ld_x ? d.ld_x : d.C; a.ld_y = d.ld_y ? d.ld_y : d.C;
  a.ld_r = d.ld_r ? d.ld_r : d.C; a.ld_h = d.ld_h ? d.ld_h : d.C;
  a.ld_mod = d.ld_mod ? d.ld_mod : d.C;
  a.gate = d.gate; a.scale = d.scale; a.shift = d.shift;
  a.group_ptr = d.group_ptr;
  a.group_rows = d.rows / d.groups;
  a.post_weight = d.post_weight; a.post_bias = d.post_bias; a.weight = d.weight; a.bias = d.bias;
  return a;
}

bool aligned(const GateNormArgs& a) {
  const void* all[] = {a.x, a.y, a.r_in, a.dr, a.dh, a.r, a.h, a.dx, a.dy, a.gate, a.scale, a.shift, a.post_weight, a.post_bias,
                       a.weight, a.bias};
  for (const void* p : all)
    if (misaligned16(p)) return false;
  return (a.C | a.ld_x | a.ld_y | a.ld_r | a.ld_h | a.ld_mod) % 8 == 0;
}

// f(stream type, branch type, vectors of a lane) as integral constants
template <class F>
void dispatch(const svg_gate_norm_t& d, int vpl, F f) {
  auto with_types = [&](auto v) {
    using BF = std::integral_constant<int, SVG_BF16>;
    using HF = std::integral_constant<int, SVG_F16>;
    using SF = std::integral_constant<int, SVG_F32>;
    if (d.stream_type == SVG_F32) {
      if (d.branch_type == SVG_F16) f(SF{}, HF{}, v);
      else f(SF{}, BF{}, v);
    } else {
      if (d.branch_type == SVG_F16) f(BF{}, HF{}, v);
      else f(BF{}, BF{}, v);
    }
  };
  if (vpl == 1) with_types(std::integral_constant<int, 1>{});
  else with_types(std::integral_constant<int, 2>{});
}
// How a call's rows come: form, wavefronts, rows ahead.
struct Way {
  Form form;
  RowShape row;
  int depth;
  int bytes(int element) const { return row.waves * depth * row.vpl * kSegment * element; }      // LDS of a workgroup
};
Way way(int C, bool whole, int bytes) {                  // bytes of an element of all tensors that are read
  auto depth = [&](const RowShape& r) { return ring_depth(r.waves, r.vpl * kSegment * bytes); };
  const Form form = whole ? kWhole : kShifted;
  const RowShape row = row_shape(C, form);
  if (row.waves <= kMaxWaves && depth(row)) return {form, row, depth(row)};
  return {kSingle, row_shape(C), 0};
}
// Gradients of two vectors a lane always come in registers: beside their sums and tables the 128 registers of 16 wavefronts hold no
// row, and what is spilt in front of a ring is read back behind its waits (bf16, 8200 x 12288 2634 us through the ring, 1408 in registers; 4000 x 9001
// 2971 and 617; fp32 stream, 8200 x 12288 6617 and 1749, 4000 x 16384 1229 and 1259).  Still 0.7 to 1 TB/s.
Way grad_way(int C, bool whole, int bytes) {
  const Way w = way(C, whole, bytes);
  return w.row.vpl == 1 ? w : Way{kSingle, row_shape(C), 0};
}
// f(form, depth) as integral constants
template <class F>
void with_way(const Way& w, F f) {
  auto with_form = [&](auto form) {
    if (w.depth == 1) f(form, std::integral_constant<int, 1>{});
    else if (w.depth == 2) f(form, std::integral_constant<int, 2>{});
    else f(form, std::integral_constant<int, 3>{});
  };
  if (w.form == kWhole) with_form(std::integral_constant<Form, kWhole>{});
  else if (w.form == kShifted) with_form(std::integral_constant<Form, kShifted>{});
  else f(std::integral_constant<Form, kSingle>{}, std::integral_constant<int, 0>{});
}

// Launches a kernel with `bytes` of dynamic LDS; more than 64 KB has to be allowed, once for each GPU, because the call costs a microsecond.
hipError_t launch_with_lds(void (*kernel)(GateNormArgs), std::atomic<unsigned long long>& allowed, dim3 grid, dim3 block, int bytes, hipStream_t stream,
                           const GateNormArgs& a) {
  if (bytes > 65536) {
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return e;
    const unsigned long long bit = device < 64 ? 1ull << device : 0;
    if (!(allowed.load(std::memory_order_relaxed) & bit)) {
      e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kRingBytes);
      if (e != hipSuccess) return e;
      allowed.fetch_or(bit, std::memory_order_relaxed);
    }
  }
  hipLaunchKernelGGL(kernel, grid, block, (unsigned)bytes, stream, a);
  return hipGetLastError();
}

constexpr int kGradLeast = 2;         // rows of a strip of the backward pass: its sums cost the traffic of two
struct GradShape {                    // by the descriptor alone: the workspace depends on it
  int strip, splits;
  long long strips;
};
GradShape grad_shape(const svg_gate_norm_t& d) {
  GradShape g;
  const int bytes = 2 * (type_bytes(d.stream_type) + 2);
  const Way w = grad_way(d.C, true, bytes);
  g.strip = std::max(strip_rows(d.rows, w.row.waves, 16, w.bytes(bytes)), kGradLeast);
  g.strips = (d.rows + g.strip - 1) / g.strip;
  // parts of the strips that are added up side by side: enough workgroups for the chip, at least 128 strips each
  const long long chunks = (d.C + kSumChannels - 1) / kSumChannels * (long long)(d.groups <= kFewGroups ? 1 : std::min(d.groups, 4096));
  const long long most = std::min<long long>(32, g.strips / std::max(1, std::min(d.groups, 64)) / 128);
  g.splits = (int)std::max<long long>(1, std::min<long long>(most, (256 + chunks - 1) / chunks));
  return g;
}

}  // namespace

size_t gate_norm_workspace_bytes(const svg_gate_norm_t& d) {
  const GradShape g = grad_shape(d);
  return (size_t)(g.strips + (long long)d.groups * (2 + (g.splits > 1 ? g.splits : 0))) * 4 * d.C * sizeof(float);
}

namespace {
GateNormArgs forward_args(const svg_gate_norm_t& d, const void* x, const void* y, const void* r, const void* h) {
  GateNormArgs a = gate_norm_args(d);
  a.x = x; a.y = y; a.r = const_cast<void*>(r); a.h = const_cast<void*>(h);
  return a;
}
}  // namespace

bool gate_norm_writes_codes(const svg_gate_norm_t& d, const void* x, const void* y, const void* r, const void* h) {
  return aligned(forward_args(d, x, y, r, h)) && d.C % 32 == 0;
}

int launch_gate_norm(const svg_gate_norm_t& d, const void* x, const void* y, void* r, void* h, void* codes, void* scales,
                     hipStream_t stream) {
  GateNormArgs a = forward_args(d, x, y, r, h);
  a.codes = static_cast<unsigned*>(codes);
  a.scales = static_cast<unsigned char*>(scales);
  a.col_tiles = (int)fp4_col_tiles(d.C);
  a.col_groups = (int)fp4_col_groups(d.C);
  const bool vec = aligned(a);
  if (codes) a.row_limit = fp4_row_tiles(d.rows) * kFp4Rows;
  const int bytes = type_bytes(d.stream_type) + 2;
  const Way w = way(d.C, vec, bytes);
  a.waves = w.row.waves;
  a.strip = strip_rows(a.row_limit, w.row.waves, 20, w.bytes(bytes));
  const dim3 grid((unsigned)((a.row_limit + a.strip - 1) / a.strip)), block((unsigned)(64 * w.row.waves));
  hipError_t e = hipSuccess;
  (void)hipGetLastError();
  dispatch(d, w.row.vpl, [&](auto ts, auto tb, auto vpl) {
    constexpr int TS = decltype(ts)::value, TB = decltype(tb)::value, VPL = decltype(vpl)::value;
    with_way(w, [&](auto form, auto depth) {
      constexpr Form FORM = decltype(form)::value;
      constexpr int D = decltype(depth)::value;
      static std::atomic<unsigned long long> allowed[2];
      constexpr bool F = FORM == kWhole;
      e = launch_with_lds(codes ? gate_norm_kernel<TS, TB, VPL, D, FORM, F> : gate_norm_kernel<TS, TB, VPL, D, FORM, false>, allowed[codes != nullptr],
                          grid, block, w.bytes(bytes), stream, a);
    });
  });
  return hip_status(e);
}

int launch_gate_norm_grad(const svg_gate_norm_t& d, const void* r, const void* y, const void* dr, const void* dh, void* dx, void* dy,
                          const svg_gate_norm_grads_t& grads, float* workspace, hipStream_t stream) {
  GateNormArgs a = gate_norm_args(d);
  a.r_in = r; a.y = y; a.dr = dr; a.dh = dh; a.dx = dx; a.dy = dy;
  a.partial = workspace;
  const GradShape g = grad_shape(d);
  const int bytes = 2 * (type_bytes(d.stream_type) + 2);
  const Way w = grad_way(d.C, aligned(a), bytes);
  a.waves = w.row.waves;
  a.strip = g.strip;
  (void)hipGetLastError();
  if (d.rows) {
    const dim3 grid((unsigned)g.strips), block((unsigned)(64 * w.row.waves));
    hipError_t e = hipSuccess;
    dispatch(d, w.row.vpl, [&](auto ts, auto tb, auto vpl) {
      constexpr int TS = decltype(ts)::value, TB = decltype(tb)::value, VPL = decltype(vpl)::value;
      with_way(w, [&](auto form, auto depth) {
        constexpr Form FORM = decltype(form)::value;
        constexpr int D = decltype(depth)::value;
        if constexpr (VPL == 1 || FORM == kSingle) {
          static std::atomic<unsigned long long> allowed;
          e = launch_with_lds(gate_norm_grad_kernel<TS, TB, VPL, D, FORM>, allowed, grid, block, w.bytes(bytes), stream, a);
        }
      });
    });
    if (e != hipSuccess) return hip_status(e);
  }
  GradSumArgs p = {};
  p.rows = d.rows; p.C = d.C; p.groups = d.groups;
  p.strip = g.strip; p.splits = g.splits;
  p.group_ptr = d.group_ptr; p.group_rows = a.group_rows;
  p.partial = workspace;
  const bool weights = grads.post_weight || grads.post_bias || grads.weight || grads.bias;
  float* const behind = workspace + (size_t)(g.strips + d.groups) * 4 * d.C;
  p.total = weights && d.groups > kFewGroups ? behind : nullptr;
  p.split = behind + (size_t)d.groups * 4 * d.C;
  // a missing norm's weight and bias take no part
  p.has_post_weight = d.post_norm != SVG_NORM_NONE;
  p.has_post_bias = d.post_norm == SVG_NORM_LAYER;
  p.has_weight = d.pre_norm != SVG_NORM_NONE;
  p.has_bias = d.pre_norm == SVG_NORM_LAYER;
  p.post_weight = p.has_post_weight ? d.post_weight : nullptr;
  p.post_bias = p.has_post_bias ? d.post_bias : nullptr;
  p.weight = p.has_weight ? d.weight : nullptr;
  p.bias = p.has_bias ? d.bias : nullptr;
  p.gate = d.gate; p.scale = d.scale;
  p.ld_mod = a.ld_mod;
  p.ld_grad = grads.ld_mod ? grads.ld_mod : d.C;
  p.dgate = grads.gate; p.dscale = grads.scale; p.dshift = grads.shift;
  p.dpost_weight = grads.post_weight; p.dpost_bias = grads.post_bias; p.dweight = grads.weight; p.dbias = grads.bias;
  if (!weights && !p.dgate && !p.dscale && !p.dshift) return SVG_OK;
  const unsigned chunks = (unsigned)((d.C + kSumChannels - 1) / kSumChannels), gy = (unsigned)std::min(d.groups, 4096);
  const dim3 threads(kSumLanes * kSumChannels);
  if (d.groups <= kFewGroups) {
    int lanes = kSumLanes;            // a power of two: whole wavefronts
    while (lanes * d.groups > kSumLanes) lanes /= 2;
    if (p.splits > 1) {
      hipLaunchKernelGGL(grad_groups_kernel, dim3(chunks, gy, (unsigned)p.splits), threads, 0, stream, p);
      hipLaunchKernelGGL(grad_few_kernel<true>, dim3(chunks), threads, 0, stream, p, lanes);
    } else {
      hipLaunchKernelGGL(grad_few_kernel<false>, dim3(chunks), threads, 0, stream, p, lanes);
    }
  } else {
    hipLaunchKernelGGL(grad_groups_kernel, dim3(chunks, gy, (unsigned)p.splits), threads, 0, stream, p);
    if (p.splits > 1) hipLaunchKernelGGL(grad_splits_kernel, dim3(chunks, gy), threads, 0, stream, p);
    if (p.total) hipLaunchKernelGGL(grad_weights_kernel, dim3(chunks), threads, 0, stream, p);
  }
  return hip_status(hipGetLastError());
}

}  // namespace svg
