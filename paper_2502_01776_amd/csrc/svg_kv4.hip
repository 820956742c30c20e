// The 4-bit cache of keys and values: page tables and slots from the lengths, rows into the pages and out of them.
#include <algorithm>
#include <limits>
#include <type_traits>

#include "svg_kv4.h"

namespace svg {

namespace {

constexpr int kThreads = 256;

// ---- page tables -------------------------------------------------------------------------------------------------------
//
// With have_b and want_b the pages that sequence b holds and needs, sequence b gives back r_b = max(0, have_b - want_b) pages and
// takes g_b = max(0, want_b - have_b).  With sums R_b, G_b over the sequences in front of b and R, G over all of them, page j it gives back goes to
// stack[count + R_b + j - want_b], and page j it takes is stack[count + R - 1 - (G_b + j - have_b)]: below `count` the stack's own entry,
// from there on a page that some sequence gives back in the same call, found without the stack, so that nothing waits for another workgroup.
//
// A workgroup takes kTokens of one sequence's tokens and sums over all sequences by itself: 8 bytes a sequence out of L2
// instead of a launch in front.  The state (lengths, count) is written by the first workgroup, or by a launch of its own where it
// lies where others still read it.  Bound: latency of a launch and of three dependent trips to memory (one sequence 3.2 us); the slots' bytes for many tokens.
//
// kTokens is 512 as long as all workgroups are on the card at once (200 sequences of up to 1560 new tokens: 7.8 us, with 2048 8.6), else 2048:
// more workgroups would only repeat the sums.

constexpr int kTokens = 512, kTokensMany = 2048, kTogether = 8 * 256;

struct ResizeArgs {
  Kv4Resize r;
  int32_t* table;
  int B, log2, pages, max_pages;
  int each;             // tokens of a workgroup
  bool state;           // the first workgroup writes the state
};

struct Sequence {
  int len, wanted, have, want;
  bool bad;
  __device__ __forceinline__ Sequence(const ResizeArgs& a, int b) : len(a.r.lengths[b]), wanted(a.r.wanted[b]) {
    const int most = a.max_pages << a.log2;
    bad = len < 0 || len > most || wanted < 0 || wanted > most || (a.r.slots != nullptr && wanted - len > a.r.tokens);
    const int mask = (1 << a.log2) - 1;
    have = bad ? 0 : (len + mask) >> a.log2;
    want = bad ? 0 : (wanted + mask) >> a.log2;
  }
  __device__ __forceinline__ int back() const { return max(0, have - want); }
  __device__ __forceinline__ int take() const { return max(0, want - have); }
};

struct Totals {
  long long R, G, R_b, G_b;      // over all sequences, over those in front of b
  int status;
  int count;
};

// The sums that a call's totals are made of.
struct Sums {
  long long all_r, all_g, front_r, front_g;
  int bad;
};

__device__ __forceinline__ Totals totals(const ResizeArgs& a, int b, Sums* shared) {
  Sums t = {};
  const int count = *a.r.free_count;
  for (int s = threadIdx.x; s < a.B; s += kThreads) {
    const Sequence q(a, s);
    t.bad |= q.bad;
    t.all_r += q.back();
    t.all_g += q.take();
    t.front_r += s < b ? q.back() : 0;
    t.front_g += s < b ? q.take() : 0;
  }
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) {
    t.all_r += __shfl_xor(t.all_r, m, 64);
    t.all_g += __shfl_xor(t.all_g, m, 64);
    t.front_r += __shfl_xor(t.front_r, m, 64);
    t.front_g += __shfl_xor(t.front_g, m, 64);
    t.bad |= __shfl_xor(t.bad, m, 64);
  }
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = t;
  __syncthreads();
  t = shared[0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) {
    t.all_r += shared[w].all_r;
    t.all_g += shared[w].all_g;
    t.front_r += shared[w].front_r;
    t.front_g += shared[w].front_g;
    t.bad |= shared[w].bad;
  }
  const bool wrong = t.bad || count < 0 || count > a.pages || count + t.all_r > a.pages;
  return {t.all_r, t.all_g, t.front_r, t.front_g, wrong ? SVG_KV4_LENGTHS : t.all_g > count + t.all_r ? SVG_KV4_FULL : SVG_KV4_OK, count};
}

__device__ __forceinline__ void write_state(const ResizeArgs& a, const Totals& t) {
  for (int s = threadIdx.x; s < a.B; s += kThreads) a.r.new_lengths[s] = t.status == SVG_KV4_OK ? a.r.wanted[s] : a.r.lengths[s];
  if (threadIdx.x == 0) {
    *a.r.new_count = t.status == SVG_KV4_OK ? (int)(t.count + t.R - t.G) : t.count;
    *a.r.status = t.status;
  }
}

__global__ __launch_bounds__(kThreads) void resize_kernel(ResizeArgs a) {
  __shared__ Sums shared[kThreads / 64];
  __shared__ long long sums[kThreads / 64], running;
  const int b = blockIdx.x, part = blockIdx.y;
  const Sequence own(a, b);
  const Totals t = totals(a, b, shared);                 // (its barrier stands behind every read of the lengths)
  if (a.state && b == 0 && part == 0) write_state(a, t);
  const bool ok = t.status == SVG_KV4_OK;
  // tokens first .. last - 1 of the new ones are this workgroup's
  const long long first = (long long)part * a.each;
  const long long last = min(first + a.each, (long long)max(0, own.wanted - own.len));
  int32_t* const row = a.table + (size_t)b * a.max_pages;
  const int mask = (1 << a.log2) - 1;
  if (ok && part == 0)                                   // pages given back
    for (int j = own.want + threadIdx.x; j < own.have; j += kThreads) a.r.free_pages[t.count + t.R_b + (j - own.want)] = row[j];
  // (own.take() > 0: the row of a sequence that takes pages is written, one that gives pages back is only read)
  if (ok && own.take() > 0 && first < last) {
    // pages whose tokens are here; the first may be another workgroup's too, which writes the same
    const int j0 = max(own.have, (int)((own.len + first) >> a.log2)), j1 = min(own.want, (int)((own.len + last - 1) >> a.log2) + 1);
    const long long top = t.count + t.R - 1 - t.G_b + own.have;      // page j: stack[top - j]
    for (int j = j0 + threadIdx.x; j < j1; j += kThreads)
      if (top - j < t.count) row[j] = a.r.free_pages[top - j];
    // those that other sequences give back in this call: ranks (from the first page given back) top - count - j
    if (j0 < j1 && top - j0 >= t.count) {
      const long long lo = max(0ll, top - t.count - (j1 - 1)), hi = top - t.count - j0;
      if (threadIdx.x == 0) running = 0;
      for (int base = 0; base < a.B; base += kThreads) {
        const int s = base + threadIdx.x;
        int back = 0, want = 0;
        if (s < a.B) {
          const Sequence q(a, s);
          back = q.back();
          want = q.want;
        }
        // sum in front of each thread: inside the wavefront, then over the wavefronts
        long long sum = back;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const long long x = __shfl_up(sum, d, 64);
          if ((threadIdx.x & 63) >= d) sum += x;
        }
        __syncthreads();
        if ((threadIdx.x & 63) == 63) sums[threadIdx.x >> 6] = sum;
        __syncthreads();
        long long front = running;
        for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) front += sums[w];
        const long long end = front + sum, begin = end - back;
        for (long long rank = max(begin, lo); rank < min(end, hi + 1); ++rank)
          row[top - t.count - rank] = a.table[(size_t)s * a.max_pages + want + (rank - begin)];
        __syncthreads();
        if (threadIdx.x == kThreads - 1) running = end;
      }
    }
  }
  __syncthreads();                                       // the row's new entries can be read
  if (a.r.slots == nullptr) return;
  int64_t* const slots = a.r.slots + (size_t)b * a.r.tokens;
  const long long end = min(first + a.each, (long long)a.r.tokens);
  for (long long i = first + threadIdx.x; i < end; i += kThreads) {
    int64_t slot = -1;
    if (ok && i < last) {
      const int at = own.len + (int)i, page = row[at >> a.log2];
      if ((unsigned)page < (unsigned)a.pages) slot = ((int64_t)page << a.log2) + (at & mask);
    }
    slots[i] = slot;
  }
}

__global__ __launch_bounds__(kThreads) void resize_state_kernel(ResizeArgs a) {
  __shared__ Sums shared[kThreads / 64];
  const Totals t = totals(a, 0, shared);
  write_state(a, t);
}

// ---- rows into pages and out of them ---------------------------------------------------------------------------------
//
// A lane takes eight neighbouring elements of a row of keys and the same of values: D / 8 lanes a row, four of them a block of 32, whose largest
// magnitude needs two lane moves.  Bound: HBM (2 or 4 bytes an element in, 17/32 out; the other way round on the way back).  One row of each to a thread, and
// results past the caches: 40 heads of 4680 x 128 in bf16 written and read 45.8 us, 4.2 TB/s, a large copy 4.7; two rows to a thread 57.5, 48.6 with the
// stores alone changed, 52.5 with the rows alone; four rows 58.7.

struct RowsArgs {
  Kv4 c;
  HeadRows k, v;
  const void *kp, *vp;
  const int64_t* slots;
  long long rows;            // tokens
  unsigned units;            // rows of all heads
  bool heads_inner;          // neighbouring units are heads of one token, not tokens of one head
};

// Which row is unit u, and where is its record?
struct RowPlace {
  unsigned row, h;
  bool there;
  unsigned char* record;
  int place;
  size_t k_at, v_at;         // elements
  template <int D>
  __device__ __forceinline__ void find(const RowsArgs& a, unsigned u) {
    there = u < a.units;
    u = there ? u : 0;
    if (a.heads_inner) {
      row = u / (unsigned)a.c.H;
      h = u - row * (unsigned)a.c.H;
    } else {
      h = u / (unsigned)a.rows;
      row = u - h * (unsigned)a.rows;
    }
    const int64_t slot = a.slots[row];
    const long long page = slot >> a.c.page_log2;
    there = there && slot >= 0 && page < a.c.pages;
    place = (int)(slot & ((1 << a.c.page_log2) - 1));
    record = a.c.data + (size_t)((there ? page : 0) * a.c.H + h) * (size_t)a.c.record();
    const unsigned b = row / (unsigned)a.k.N, n = row - b * (unsigned)a.k.N;
    k_at = (size_t)b * a.k.sb + (size_t)n * a.k.sn + (size_t)h * a.k.sh;
    v_at = (size_t)b * a.v.sb + (size_t)n * a.v.sn + (size_t)h * a.v.sh;
  }
};

template <int D, int KT, int VT>
__global__ __launch_bounds__(kThreads) void write_kernel(RowsArgs a) {
  constexpr int LANES = D / 8, ROWS = kThreads / LANES;
  const int c = threadIdx.x % LANES;
  RowPlace at;
  at.template find<D>(a, (blockIdx.y * gridDim.x + blockIdx.x) * ROWS + threadIdx.x / LANES);
  float k[8] = {}, v[8] = {};
  if (at.there) {
    load8_any<KT>(a.kp, at.k_at + 8 * c, k);
    load8_any<VT>(a.vp, at.v_at + 8 * c, v);
  }
  unsigned ks = fp4_scale(quad_max(magnitude8(k))), vs = fp4_scale(quad_max(magnitude8(v)));
  const unsigned kc = fp4_codes8(k, ks), vc = fp4_codes8(v, vs);
  // a row's scale bytes as one word, or one half of it
  ks <<= 8 * (c >> 2);
  vs <<= 8 * (c >> 2);
#pragma unroll
  for (int m = 4; m < LANES; m <<= 1) {
    ks |= __shfl_xor(ks, m, 64);
    vs |= __shfl_xor(vs, m, 64);
  }
  if (!at.there) return;
  unsigned char* const codes = at.record + at.place * (D / 2) + 4 * c;
  *reinterpret_cast<unsigned*>(codes) = kc;
  *reinterpret_cast<unsigned*>(codes + a.c.values()) = vc;
  if (c < 2) {
    unsigned char* const scales = at.record + (c ? a.c.value_scales() : a.c.key_scales()) + at.place * (D / 32);
    const unsigned s = c ? vs : ks;
    if constexpr (D == 128) *reinterpret_cast<unsigned*>(scales) = s;
    else *reinterpret_cast<unsigned short*>(scales) = (unsigned short)s;
  }
}

// Eight values of a word of codes under a scale byte: the power of two in two normal factors, since it may be subnormal itself.
__device__ __forceinline__ void values8(unsigned code, unsigned scale, float (&v)[8]) {
  const unsigned half = scale / 2;
  const float p = __uint_as_float((half + 64) << 23), q = __uint_as_float((scale - half + 63) << 23);
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 1),
             c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 3);
  const float x[8] = {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = scale == 255 ? __builtin_nanf("") : x[e] * p * q;
}

template <int D, int KT, int VT>
__global__ __launch_bounds__(kThreads) void read_kernel(RowsArgs a, void* kp, void* vp) {
  constexpr int LANES = D / 8, ROWS = kThreads / LANES;
  const int c = threadIdx.x % LANES;
  RowPlace at;
  at.template find<D>(a, (blockIdx.y * gridDim.x + blockIdx.x) * ROWS + threadIdx.x / LANES);
  if (!at.there) return;
  const unsigned char* const codes = at.record + at.place * (D / 2) + 4 * c;
  const unsigned char* const scales = at.record + at.place * (D / 32) + (c >> 2);
  const unsigned kc = *reinterpret_cast<const unsigned*>(codes), vc = *reinterpret_cast<const unsigned*>(codes + a.c.values());
  const unsigned ks = scales[a.c.key_scales()], vs = scales[a.c.value_scales()];
  float v[8];
  values8(kc, ks, v);
  store8_any<KT, true>(kp, at.k_at + 8 * c, v);
  values8(vc, vs, v);
  store8_any<VT, true>(vp, at.v_at + 8 * c, v);
}

template <class F>
void by_type(int type, F f) {
  if (type == SVG_F32) f(std::integral_constant<int, SVG_F32>{});
  else if (type == SVG_F16) f(std::integral_constant<int, SVG_F16>{});
  else f(std::integral_constant<int, SVG_BF16>{});
}

template <class F>
int launch_rows(const Kv4& c, const HeadRows& k, const HeadRows& v, const int64_t* slots, long long rows, F go) {
  RowsArgs a = {};
  a.c = c;
  a.k = k;
  a.v = v;
  a.slots = slots;
  a.rows = rows;
  // from the layout that lies in memory: heads of a token side by side, or tokens of a head
  a.heads_inner = k.sh <= k.sn;
  const int per_block = kThreads / (c.D / 8);
  const long long all = rows * c.H;
  if (all > 0xfff00000ll) return SVG_ERR_UNSUPPORTED;          // (rows are counted in 32 bits, those of the last workgroups too)
  a.units = (unsigned)all;
  (void)hipGetLastError();
  // a launch has fewer than 2^32 threads in one dimension
  const long long blocks = (all + per_block - 1) / per_block, wide = std::min(blocks, 1ll << 23);
  go(a, dim3((unsigned)wide, (unsigned)((blocks + wide - 1) / wide)));
  return hip_status(hipGetLastError());
}

}  // namespace

int launch_kv4_resize(const Kv4& c, const Kv4Resize& r, bool in_place, hipStream_t stream) {
  ResizeArgs a = {r, c.table, c.B, c.page_log2, c.pages, c.max_pages, std::numeric_limits<int>::max(), false};
  unsigned parts = 1;
  if (r.slots && r.tokens > 0) {
    const long long tokens = r.tokens, fine = (tokens + kTokens - 1) / kTokens;
    // (a second dimension has at most 65535 workgroups)
    a.each = std::max(fine * c.B <= kTogether ? kTokens : kTokensMany, (int)((tokens + 65534) / 65535));
    parts = (unsigned)((tokens + a.each - 1) / a.each);
  }
  const bool one = (unsigned long long)c.B * parts <= 1;
  a.state = c.B > 0 && (one || !in_place);
  (void)hipGetLastError();
  if (c.B) hipLaunchKernelGGL(resize_kernel, dim3((unsigned)c.B, parts), dim3(kThreads), 0, stream, a);
  if (!a.state) hipLaunchKernelGGL(resize_state_kernel, dim3(1), dim3(kThreads), 0, stream, a);
  return hip_status(hipGetLastError());
}

int launch_kv4_write(const Kv4& c, const HeadRows& k, const void* kp, const HeadRows& v, const void* vp, const int64_t* slots, long long rows,
                     hipStream_t stream) {
  return launch_rows(c, k, v, slots, rows, [&](RowsArgs& a, dim3 grid) {
    a.kp = kp;
    a.vp = vp;
    by_type(k.type, [&](auto kt) {
      by_type(v.type, [&](auto vt) {
        constexpr int KT = decltype(kt)::value, VT = decltype(vt)::value;
        hipLaunchKernelGGL((c.D == 128 ? write_kernel<128, KT, VT> : write_kernel<64, KT, VT>), grid, dim3(kThreads), 0, stream, a);
      });
    });
  });
}

int launch_kv4_read(const Kv4& c, const HeadRows& k, void* kp, const HeadRows& v, void* vp, const int64_t* slots, long long rows,
                    hipStream_t stream) {
  return launch_rows(c, k, v, slots, rows, [&](RowsArgs& a, dim3 grid) {
    by_type(k.type, [&](auto kt) {
      by_type(v.type, [&](auto vt) {
        constexpr int KT = decltype(kt)::value, VT = decltype(vt)::value;
        hipLaunchKernelGGL((c.D == 128 ? read_kernel<128, KT, VT> : read_kernel<64, KT, VT>), grid, dim3(kThreads), 0, stream, a, kp, vp);
      });
    });
  });
}

}  // namespace svg
