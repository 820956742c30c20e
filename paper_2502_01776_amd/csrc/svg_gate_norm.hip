// Gate, residual, norm and modulation between two branches of a layer, and its gradients.  HBM-bound: the forward pass
// reads x and y and writes r and h, the backward pass reads r, y, dr, dh and writes dx, dy; a row is read once and stays in
// registers from its statistics to its outputs.
#include <type_traits>

#include "svg_block.h"

namespace svg {

namespace {

constexpr int kMaxWaves = 8;          // wavefronts that share a row

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
  int rows_per_block;
  float* partial;                     // backward: [slots][4][C]
};

// The group of a row: how many of the ends group_ptr[1 .. groups-1] are not above it.  In range whatever the table holds.
__device__ __forceinline__ int group_of(const GateNormArgs& a, long long row) {
  if (a.groups == 1) return 0;
  if (!a.group_ptr) return (int)(row / a.group_rows);
  int lo = 0, hi = a.groups - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if ((long long)a.group_ptr[mid] <= row) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// A wavefront's lanes hold VPL times eight channels of the row.  VEC: eight neighbours each; otherwise (rows that are not
// 16-byte aligned) neighbours are in neighbouring lanes.
template <int VPL, bool VEC>
struct Channels {
  int first, step, C;
  __device__ __forceinline__ Channels(int C_) : C(C_) {
    first = VEC ? (int)threadIdx.x * 8 : (int)threadIdx.x;
    step = VEC ? (int)blockDim.x * 8 : (int)blockDim.x;
  }
  __device__ __forceinline__ int at(int v, int e) const { return VEC ? first + v * step + e : first + (v * 8 + e) * step; }
  __device__ __forceinline__ bool has(int v, int e) const { return VEC ? first + v * step < C : at(v, e) < C; }

  // the row is the same for all lanes: its address stays in scalar registers
  template <int TYPE>
  static __device__ __forceinline__ const void* from(const void* base, size_t row) {
    return static_cast<const char*>(base) + row * (TYPE == SVG_F32 ? 4 : 2);
  }
  template <int TYPE>
  __device__ __forceinline__ void load(const void* base, size_t row, float (&x)[VPL * 8]) const {
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      float t[8] = {};
      if constexpr (VEC) {
        if (has(v, 0)) load8<TYPE>(from<TYPE>(base, row), (unsigned)at(v, 0), t);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (has(v, e)) t[e] = load1<TYPE>(from<TYPE>(base, row), (unsigned)at(v, e));
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v * 8 + e] = t[e];
    }
  }
  template <int TYPE>
  __device__ __forceinline__ void store(void* base, size_t row, const float (&x)[VPL * 8]) const {
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      if constexpr (VEC) {
        float t[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = x[v * 8 + e];
        if (has(v, 0)) store8<TYPE>(const_cast<void*>(from<TYPE>(base, row)), (unsigned)at(v, 0), t);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (has(v, e)) store1<TYPE>(const_cast<void*>(from<TYPE>(base, row)), (unsigned)at(v, e), x[v * 8 + e]);
      }
    }
  }
  // a parameter vector, or `otherwise` where there is none
  __device__ __forceinline__ void table(const float* base, size_t row, float otherwise, float (&x)[VPL * 8]) const {
    if (base) {
      load<SVG_F32>(base, row, x);
    } else {
#pragma unroll
      for (int i = 0; i < VPL * 8; ++i) x[i] = otherwise;
    }
  }
};

// Sums over the row: over the wavefront, then over the wavefronts of the workgroup through LDS.  Two sets of places in
// turn, so that one barrier a sum is enough: a wavefront writes a place again only behind the next barrier.
struct RowSum {
  float (*place)[kMaxWaves][2];
  int turn, waves;
  __device__ __forceinline__ void operator()(float& p, float& q) {
    p = wave_sum(p);
    q = wave_sum(q);
    if (waves == 1) return;
    if ((threadIdx.x & 63) == 0) {
      place[turn][threadIdx.x >> 6][0] = p;
      place[turn][threadIdx.x >> 6][1] = q;
    }
    __syncthreads();
    p = q = 0.f;
    for (int w = 0; w < waves; ++w) {
      p += place[turn][w][0];
      q += place[turn][w][1];
    }
    turn ^= 1;
  }
  __device__ __forceinline__ void operator()(float& p) {
    float none = 0.f;
    (*this)(p, none);
  }
};

// v -> (v - mean) * rho, returns rho.  The mean first and the squares of what is left then: a row far from zero loses nothing.
template <int VPL, bool VEC>
__device__ __forceinline__ float normalise(float (&v)[VPL * 8], int norm, float eps, const Channels<VPL, VEC>& ch, RowSum& sum) {
  if (norm == SVG_NORM_NONE) return 1.0f;
  const float inv = 1.0f / (float)ch.C;
  if (norm == SVG_NORM_LAYER) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < VPL * 8; ++i) m += v[i];
    sum(m);
    m *= inv;
#pragma unroll
    for (int i = 0; i < VPL * 8; ++i) v[i] = ch.has(i / 8, i % 8) ? v[i] - m : 0.f;
  }
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < VPL * 8; ++i) s = __builtin_fmaf(v[i], v[i], s);
  sum(s);
  const float rho = 1.0f / sqrtf(s * inv + eps);
#pragma unroll
  for (int i = 0; i < VPL * 8; ++i) v[i] *= rho;
  return rho;
}

template <int TS, int TB, int VPL, bool VEC, bool FP4>
__global__ __launch_bounds__(64 * kMaxWaves) void gate_norm_kernel(GateNormArgs a) {
  __shared__ float places[2][kMaxWaves][2];
  const Channels<VPL, VEC> ch(a.C);
  RowSum sum{places, 0, (int)(blockDim.x >> 6)};
  const long long r0 = (long long)blockIdx.x * a.rows_per_block;
  const long long r1 = min(r0 + a.rows_per_block, a.row_limit);
  for (long long row = r0; row < r1; ++row) {
    float v[VPL * 8] = {};
    if (row < a.rows) {
      const size_t mod = (size_t)group_of(a, row) * a.ld_mod;
      float t[VPL * 8];
      ch.template load<TS>(a.x, (size_t)row * a.ld_x, v);
#pragma unroll
      for (int i = 0; i < VPL * 8; ++i) v[i] *= a.alpha;
      if (a.y) {
        float y[VPL * 8];
        ch.template load<TB>(a.y, (size_t)row * a.ld_y, y);
        normalise(y, a.post, a.post_eps, ch, sum);
        if (a.post != SVG_NORM_NONE) {
          ch.table(a.post_weight, 0, 1.0f, t);
#pragma unroll
          for (int i = 0; i < VPL * 8; ++i) y[i] *= t[i];
          if (a.post == SVG_NORM_LAYER) {
            ch.table(a.post_bias, 0, 0.0f, t);
#pragma unroll
            for (int i = 0; i < VPL * 8; ++i) y[i] += t[i];
          }
        }
        ch.table(a.gate, mod, 1.0f, t);
#pragma unroll
        for (int i = 0; i < VPL * 8; ++i) v[i] = __builtin_fmaf(t[i], y[i], v[i]);
      }
      if (a.r) ch.template store<TS>(a.r, (size_t)row * a.ld_r, v);
      if (a.h || FP4) {
        normalise(v, a.pre, a.eps, ch, sum);
        if (a.pre != SVG_NORM_NONE) {
          ch.table(a.weight, 0, 1.0f, t);
#pragma unroll
          for (int i = 0; i < VPL * 8; ++i) v[i] *= t[i];
          if (a.pre == SVG_NORM_LAYER) {
            ch.table(a.bias, 0, 0.0f, t);
#pragma unroll
            for (int i = 0; i < VPL * 8; ++i) v[i] += t[i];
          }
        }
        float u[VPL * 8];
        ch.table(a.scale, mod, 0.0f, t);
        ch.table(a.shift, mod, 0.0f, u);
#pragma unroll
        for (int i = 0; i < VPL * 8; ++i) v[i] = __builtin_fmaf(v[i], 1.0f + t[i], u[i]);
        if (a.h) ch.template store<TB>(a.h, (size_t)row * a.ld_h, v);
      }
    }
    if constexpr (FP4) {
      const long long rt = row / kFp4Rows;
      const int i16 = (int)(row % kFp4Rows);
#pragma unroll
      for (int k = 0; k < VPL; ++k) {
        float t[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = v[k * 8 + e];
        const int c = ch.at(k, 0), ct = c / kFp4Cols, g = (c >> 5) & 3;
        const unsigned s = fp4_scale(quad_max(magnitude8(t)));
        if (ct < a.col_tiles) a.codes[((size_t)rt * a.col_tiles + ct) * 256 + g * 64 + i16 * 4 + ((c >> 3) & 3)] = fp4_codes8(t, s);
        if ((c & 31) == 0 && ct < a.col_groups * kFp4Group)
          a.scales[(((size_t)rt * a.col_groups + ct / kFp4Group) * 64 + g * 16 + i16) * 4 + ct % kFp4Group] = (unsigned char)s;
      }
    }
  }
}

// Gradients of a strip of rows.  What the parameters get are four sums over the rows of a group and channel:
//   S1 = sum dh, S2 = sum dh rhat, T1 = sum dR, T2 = sum dR yhat   (dR: gradient of r)
//   dshift = S1, dscale = weight S2 + bias S1, dgate = post_weight T2 + post_bias T1,
//   dweight = sum over g of (1 + scale) S2, dbias the same of S1, dpost_weight = sum over g of gate T2, dpost_bias of T1.
// They stay in registers while the strip is in one group and go to slot (workgroup + group), of which every pair that has
// rows has one of its own, because neither number ever falls along the rows.
template <int TS, int TB, int VPL, bool VEC>
__global__ __launch_bounds__(64 * kMaxWaves) void gate_norm_grad_kernel(GateNormArgs a) {
  __shared__ float places[2][kMaxWaves][2];
  const Channels<VPL, VEC> ch(a.C);
  RowSum sum{places, 0, (int)(blockDim.x >> 6)};
  constexpr int NC = VPL * 8;
  float s1[NC] = {}, s2[NC] = {}, t1[NC] = {}, t2[NC] = {};
  const float inv = 1.0f / (float)a.C;
  const long long r0 = (long long)blockIdx.x * a.rows_per_block;
  const long long r1 = min(r0 + a.rows_per_block, a.rows);
  int g = group_of(a, r0);
  auto flush = [&] {
    const size_t slot = (size_t)(blockIdx.x + (unsigned)g) * 4 * a.C;
    ch.template store<SVG_F32>(a.partial, slot, s1);
    ch.template store<SVG_F32>(a.partial, slot + a.C, s2);
    ch.template store<SVG_F32>(a.partial, slot + 2 * (size_t)a.C, t1);
    ch.template store<SVG_F32>(a.partial, slot + 3 * (size_t)a.C, t2);
  };
  for (long long row = r0; row < r1; ++row) {
    const int now = group_of(a, row);
    if (now != g) {
      flush();
      g = now;
#pragma unroll
      for (int i = 0; i < NC; ++i) s1[i] = s2[i] = t1[i] = t2[i] = 0.f;
    }
    const size_t mod = (size_t)g * a.ld_mod;
    float d[NC] = {}, t[NC];
    if (a.dr) ch.template load<TS>(a.dr, (size_t)row * a.ld_r, d);
    if (a.dh) {
      float hat[NC], e[NC];
      ch.template load<TS>(a.r_in, (size_t)row * a.ld_r, hat);
      ch.template load<TB>(a.dh, (size_t)row * a.ld_h, e);
      const float rho = normalise(hat, a.pre, a.eps, ch, sum);
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        s1[i] += e[i];
        s2[i] = __builtin_fmaf(e[i], hat[i], s2[i]);
      }
      ch.table(a.scale, mod, 0.0f, t);
#pragma unroll
      for (int i = 0; i < NC; ++i) e[i] *= 1.0f + t[i];
      if (a.pre != SVG_NORM_NONE) {
        ch.table(a.weight, 0, 1.0f, t);
        float m1 = 0.f, m2 = 0.f;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          e[i] *= t[i];
          m1 += e[i];
          m2 = __builtin_fmaf(e[i], hat[i], m2);
        }
        sum(m1, m2);
        m1 = a.pre == SVG_NORM_LAYER ? m1 * inv : 0.f;
        m2 *= inv;
#pragma unroll
        for (int i = 0; i < NC; ++i) d[i] = __builtin_fmaf(rho, __builtin_fmaf(-hat[i], m2, e[i] - m1), d[i]);
      } else {
#pragma unroll
        for (int i = 0; i < NC; ++i) d[i] += e[i];
      }
    }
    if (a.dx) {
#pragma unroll
      for (int i = 0; i < NC; ++i) t[i] = a.alpha * d[i];
      ch.template store<TS>(a.dx, (size_t)row * a.ld_x, t);
    }
    if (a.y || a.dy) {
      float hat[NC] = {}, rho = 1.0f;
      if (a.y) {
        ch.template load<TB>(a.y, (size_t)row * a.ld_y, hat);
        rho = normalise(hat, a.post, a.post_eps, ch, sum);
      }
      // the padding's d is not zero under a layer form of Pre, so it is kept out of the sums
#pragma unroll
      for (int i = 0; i < NC; ++i) d[i] = ch.has(i / 8, i % 8) ? d[i] : 0.f;
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        t1[i] += d[i];
        t2[i] = __builtin_fmaf(d[i], hat[i], t2[i]);
      }
      if (a.dy) {
        ch.table(a.gate, mod, 1.0f, t);
#pragma unroll
        for (int i = 0; i < NC; ++i) d[i] *= t[i];
        if (a.post != SVG_NORM_NONE) {
          ch.table(a.post_weight, 0, 1.0f, t);
          float m1 = 0.f, m2 = 0.f;
#pragma unroll
          for (int i = 0; i < NC; ++i) {
            d[i] *= t[i];
            m1 += d[i];
            m2 = __builtin_fmaf(d[i], hat[i], m2);
          }
          sum(m1, m2);
          m1 = a.post == SVG_NORM_LAYER ? m1 * inv : 0.f;
          m2 *= inv;
#pragma unroll
          for (int i = 0; i < NC; ++i) d[i] = rho * __builtin_fmaf(-hat[i], m2, d[i] - m1);
        }
        ch.template store<TB>(a.dy, (size_t)row * a.ld_y, d);
      }
    }
  }
  flush();
}

struct GradSumArgs {
  long long rows;
  int C, groups, rows_per_block;
  const int32_t* group_ptr;
  long long group_rows;
  const float* partial;               // [slots][4][C]
  float* total;                       // [groups][4][C], or null where no weight's gradient is wanted
  const float *post_weight, *post_bias, *weight, *bias;
  const float *gate, *scale;          // the forward pass's tables, [groups] rows of ld_mod
  long long ld_mod, ld_grad;
  float *dgate, *dscale, *dshift, *dpost_weight, *dpost_bias, *dweight, *dbias;
};

constexpr int kSumLanes = 16;         // rows (slots, groups) that are summed side by side
constexpr int kSumChannels = 64;

// Adds up the four sums of 64 channels over the workgroup's rows of threads; the result is in the first row.
__device__ __forceinline__ void fold_rows(float (&s)[4]) {
  __shared__ float lds[kSumLanes][4][kSumChannels];
  const int c = threadIdx.x % kSumChannels, k = threadIdx.x / kSumChannels;
#pragma unroll
  for (int j = 0; j < 4; ++j) lds[k][j][c] = s[j];
  __syncthreads();
  if (k == 0) {
    for (int q = 1; q < kSumLanes; ++q)
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] += lds[q][j][c];
  }
  __syncthreads();
}

// The sums of a group from the slots of the strips that have rows of it.
__global__ __launch_bounds__(kSumLanes* kSumChannels) void grad_groups_kernel(GradSumArgs a) {
  const int c = blockIdx.x * kSumChannels + threadIdx.x % kSumChannels, k = threadIdx.x / kSumChannels;
  for (int g = blockIdx.y; g < a.groups; g += gridDim.y) {
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
    float s[4] = {};
    if (lo < hi && c < a.C)
      for (long long b = lo / a.rows_per_block + k; b <= (hi - 1) / a.rows_per_block; b += kSumLanes) {
        const float* p = a.partial + (size_t)(b + g) * 4 * a.C + c;
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] += p[(size_t)j * a.C];
      }
    fold_rows(s);
    if (k == 0 && c < a.C) {
      const size_t at = (size_t)g * a.ld_grad + c;
      if (a.dshift) a.dshift[at] = s[0];
      if (a.dscale) a.dscale[at] = (a.weight ? a.weight[c] : 1.f) * s[1] + (a.bias ? a.bias[c] : 0.f) * s[0];
      if (a.dgate) a.dgate[at] = (a.post_weight ? a.post_weight[c] : 1.f) * s[3] + (a.post_bias ? a.post_bias[c] : 0.f) * s[2];
      if (a.total) {
#pragma unroll
        for (int j = 0; j < 4; ++j) a.total[((size_t)g * 4 + j) * a.C + c] = s[j];
      }
    }
  }
}

// The weights' gradients: the groups' sums under their modulation.
__global__ __launch_bounds__(kSumLanes* kSumChannels) void grad_weights_kernel(GradSumArgs a) {
  const int c = blockIdx.x * kSumChannels + threadIdx.x % kSumChannels, k = threadIdx.x / kSumChannels;
  float s[4] = {};
  if (c < a.C)
    for (int g = k; g < a.groups; g += kSumLanes) {
      const float* p = a.total + (size_t)g * 4 * a.C + c;
      const float scale = a.scale ? 1.0f + a.scale[(size_t)g * a.ld_mod + c] : 1.0f;
      const float gate = a.gate ? a.gate[(size_t)g * a.ld_mod + c] : 1.0f;
      s[0] = __builtin_fmaf(scale, p[0], s[0]);
      s[1] = __builtin_fmaf(scale, p[a.C], s[1]);
      s[2] = __builtin_fmaf(gate, p[2 * (size_t)a.C], s[2]);
      s[3] = __builtin_fmaf(gate, p[3 * (size_t)a.C], s[3]);
    }
  fold_rows(s);
  if (k == 0 && c < a.C) {
    if (a.dbias) a.dbias[c] = s[0];
    if (a.dweight) a.dweight[c] = s[1];
    if (a.dpost_bias) a.dpost_bias[c] = s[2];
    if (a.dpost_weight) a.dpost_weight[c] = s[3];
  }
}

// Wavefronts that share a row and vectors of a lane, 512 channels each: one vector up to 512 channels, two up to 8192, four up to 16384.
struct RowShape { int waves, vpl; };
RowShape row_shape(int C) {
  const int vectors = (C + 511) / 512;
  const int vpl = vectors == 1 ? 1 : vectors <= 2 * kMaxWaves ? 2 : 4;
  return {(vectors + vpl - 1) / vpl, vpl};
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

// f(stream type, branch type, vectors of a lane, whole vectors?) as integral constants
template <class F>
void dispatch(const svg_gate_norm_t& d, int vpl, bool vec, F f) {
  auto with_types = [&](auto v, auto whole) {
    using BF = std::integral_constant<int, SVG_BF16>;
    using HF = std::integral_constant<int, SVG_F16>;
    using SF = std::integral_constant<int, SVG_F32>;
    if (d.stream_type == SVG_F32) {
      if (d.branch_type == SVG_F16) f(SF{}, HF{}, v, whole);
      else f(SF{}, BF{}, v, whole);
    } else {
      if (d.branch_type == SVG_F16) f(BF{}, HF{}, v, whole);
      else f(BF{}, BF{}, v, whole);
    }
  };
  auto with_vectors = [&](auto whole) {
    if (vpl == 1) with_types(std::integral_constant<int, 1>{}, whole);
    else if (vpl == 2) with_types(std::integral_constant<int, 2>{}, whole);
    else with_types(std::integral_constant<int, 4>{}, whole);
  };
  if (vec) with_vectors(std::true_type{});
  else with_vectors(std::false_type{});
}

constexpr int kGradBlocks = 1024;     // strips of the backward pass
int grad_rows_per_block(long long rows) { return (int)((rows + kGradBlocks - 1) / kGradBlocks); }
long long grad_blocks(long long rows) {
  const long long r = grad_rows_per_block(rows);
  return r ? (rows + r - 1) / r : 0;
}

}  // namespace

size_t gate_norm_workspace_bytes(const svg_gate_norm_t& d) {
  return (size_t)(grad_blocks(d.rows) + 2 * (long long)d.groups) * 4 * d.C * sizeof(float);
}

int launch_gate_norm(const svg_gate_norm_t& d, const void* x, const void* y, void* r, void* h, void* codes, void* scales,
                     hipStream_t stream) {
  GateNormArgs a = gate_norm_args(d);
  a.x = x; a.y = y; a.r = r; a.h = h;
  a.codes = static_cast<unsigned*>(codes);
  a.scales = static_cast<unsigned char*>(scales);
  a.col_tiles = (int)fp4_col_tiles(d.C);
  a.col_groups = (int)fp4_col_groups(d.C);
  const bool vec = aligned(a);
  if (codes && (!vec || d.C % 32)) return SVG_ERR_UNSUPPORTED;
  if (codes) a.row_limit = fp4_row_tiles(d.rows) * kFp4Rows;
  a.rows_per_block = codes ? 4 : 1;
  while ((a.row_limit + a.rows_per_block - 1) / a.rows_per_block > 1 << 22) a.rows_per_block *= 2;      // a launch has fewer than 2^32 threads
  const RowShape s = row_shape(d.C);
  const long long blocks = (a.row_limit + a.rows_per_block - 1) / a.rows_per_block;
  (void)hipGetLastError();
  dispatch(d, s.vpl, vec, [&](auto ts, auto tb, auto vpl, auto whole) {
    constexpr int TS = decltype(ts)::value, TB = decltype(tb)::value, VPL = decltype(vpl)::value;
    constexpr bool VEC = decltype(whole)::value;
    if constexpr (VEC) {
      if (codes) {
        hipLaunchKernelGGL((gate_norm_kernel<TS, TB, VPL, true, true>), dim3((unsigned)blocks), dim3(64 * s.waves), 0, stream, a);
        return;
      }
    }
    hipLaunchKernelGGL((gate_norm_kernel<TS, TB, VPL, VEC, false>), dim3((unsigned)blocks), dim3(64 * s.waves), 0, stream, a);
  });
  return hip_status(hipGetLastError());
}

int launch_gate_norm_grad(const svg_gate_norm_t& d, const void* r, const void* y, const void* dr, const void* dh, void* dx, void* dy,
                          const svg_gate_norm_grads_t& grads, float* workspace, hipStream_t stream) {
  GateNormArgs a = gate_norm_args(d);
  a.r_in = r; a.y = y; a.dr = dr; a.dh = dh; a.dx = dx; a.dy = dy;
  a.partial = workspace;
  const bool vec = aligned(a);
  a.rows_per_block = grad_rows_per_block(d.rows);
  const RowShape s = row_shape(d.C);
  const long long blocks = grad_blocks(d.rows);
  (void)hipGetLastError();
  if (d.rows)
    dispatch(d, s.vpl, vec, [&](auto ts, auto tb, auto vpl, auto whole) {
      hipLaunchKernelGGL((gate_norm_grad_kernel<decltype(ts)::value, decltype(tb)::value, decltype(vpl)::value, decltype(whole)::value>),
                         dim3((unsigned)blocks), dim3(64 * s.waves), 0, stream, a);
    });
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_status(e);
  GradSumArgs p = {};
  p.rows = d.rows; p.C = d.C; p.groups = d.groups;
  p.rows_per_block = a.rows_per_block ? a.rows_per_block : 1;
  p.group_ptr = d.group_ptr; p.group_rows = a.group_rows;
  p.partial = workspace;
  const bool weights = grads.post_weight || grads.post_bias || grads.weight || grads.bias;
  p.total = weights ? workspace + (size_t)(blocks + d.groups) * 4 * d.C : nullptr;
  // a missing norm's weight and bias take no part
  p.post_weight = d.post_norm != SVG_NORM_NONE ? d.post_weight : nullptr;
  p.post_bias = d.post_norm == SVG_NORM_LAYER ? d.post_bias : nullptr;
  p.weight = d.pre_norm != SVG_NORM_NONE ? d.weight : nullptr;
  p.bias = d.pre_norm == SVG_NORM_LAYER ? d.bias : nullptr;
  p.gate = d.gate; p.scale = d.scale;
  p.ld_mod = a.ld_mod;
  p.ld_grad = grads.ld_mod ? grads.ld_mod : d.C;
  p.dgate = grads.gate; p.dscale = grads.scale; p.dshift = grads.shift;
  p.dpost_weight = grads.post_weight; p.dpost_bias = grads.post_bias; p.dweight = grads.weight; p.dbias = grads.bias;
  const unsigned chunks = (unsigned)((d.C + kSumChannels - 1) / kSumChannels);
  if (weights || p.dgate || p.dscale || p.dshift)
    hipLaunchKernelGGL(grad_groups_kernel, dim3(chunks, (unsigned)(d.groups < 4096 ? d.groups : 4096)), dim3(kSumLanes * kSumChannels), 0,
                       stream, p);
  if (weights) hipLaunchKernelGGL(grad_weights_kernel, dim3(chunks), dim3(kSumLanes * kSumChannels), 0, stream, p);
  return hip_status(hipGetLastError());
}

}  // namespace svg
