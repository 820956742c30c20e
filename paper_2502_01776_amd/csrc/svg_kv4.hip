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
// With have_b and want_b the pages that sequence b holds and needs, b gives back those of its entries want_b .. have_b - 1 that name a page of the
// pool, r_b pages (an entry may be a page that is not there), and takes g_b = max(0, want_b - have_b).  With sums R_b, G_b over the sequences in front of
// b and R, G over all of them, the i-th page that it gives back goes to stack[count + R_b + i], and its entry j that is new gets
// stack[count + R - 1 - (G_b + j - have_b)]: below `count` the stack's own entry, from there on a page that some sequence gives back in the same call,
// found without the stack, so that nothing waits for another workgroup.
//
// A workgroup takes `each` of one sequence's tokens and makes the sums by itself: 8 bytes a sequence out of L2 instead of a launch in front.  R_b and R
// need the entries that are given back; a workgroup that neither gives nor takes does without where their number can not change the answer.
// A call that would grant a number outside of the pool grants nothing, so every workgroup looks at all that are taken from the
// stack.  The state (lengths, count) is written by the first workgroup, or by a launch of its own where it
// lies where others still read it.
//
// Bound: latency of a launch and of dependent trips to memory, then the slots' bytes, then what every workgroup reads for itself.  In a graph: one sequence
// 4.2 us; 200 sequences that grow by up to 1560 tokens 6.1, and 9.8 with every eighth cut off, 4800 pages given back; 200 that are cut off, 150000 pages given back,
// 62; 200 that grow by 30000 tokens in pages of 16, 190000 numbers looked at, 84.
//
// `each` is 512 as long as that makes at most two workgroups to a compute unit, else 2048: more would repeat the sums more often than they
// share the rest (32 sequences of 8000 new tokens 5.5 us, with 2048 6.2; 200 of 1560, every eighth cut off, 9.8, with 512 11.0).

constexpr int kTokens = 512, kTokensMany = 2048, kTogether = 2 * 256;
constexpr int kRun = 16;              // neighbouring entries of a row that a thread looks at together
constexpr int kList = 2 * kThreads * kRun;      // pages given back that a workgroup keeps

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

// The sums that a call's totals are made of.
struct Sums {
  long long back, take, front_take;
  int bad;
};

struct Shared {
  Sums sums[kThreads / 64];
  unsigned waves[kThreads / 64];
  unsigned end[kThreads];                                // runs of a round's sequences up to each
  int from[kThreads], to[kThreads];                      // their entries
  unsigned own;                                          // pages that sequence b gives back
  int list[kList];
};

// The sum of x over the threads up to this one; all: over the workgroup.
__device__ __forceinline__ unsigned running_sum(unsigned x, Shared& shared, unsigned* all) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const unsigned y = __shfl_up(x, d, 64);
    if ((threadIdx.x & 63) >= d) x += y;
  }
  __syncthreads();                                       // (what was there has been read)
  if ((threadIdx.x & 63) == 63) shared.waves[threadIdx.x >> 6] = x;
  __syncthreads();
  *all = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < (int)(threadIdx.x >> 6)) x += shared.waves[w];
    *all += shared.waves[w];
  }
  return x;
}

typedef int i32x4_of4 __attribute__((ext_vector_type(4), aligned(4)));

// The pages that sequences s0 .. s1 - 1 give back, sequences and entries ascending, up to number `last` of them at least.  A thread takes a run of up to kRun
// neighbours of a row, the workgroup a run to each thread a round.
// KEEP: they are counted, R in all and R_b of sequences in front of b (b's own in shared.own, which is zero before), and put into the list while they fit.
// Otherwise f(first, n) behind each round, with pages first .. first + n - 1 in the list.  All threads of the workgroup.
template <bool KEEP, class F>
__device__ __forceinline__ void given_back(const ResizeArgs& a, int s0, int s1, int b, long long last, Shared& shared, long long* R, long long* R_b, F f) {
  const size_t entries = (size_t)a.B * a.max_pages;
  *R = *R_b = 0;
  for (int base = s0; base < s1; base += kThreads) {
    int from = 0, to = 0;
    if (base + (int)threadIdx.x < s1) {
      const Sequence q(a, base + threadIdx.x);
      from = q.want;
      to = from + q.back();
    }
    unsigned runs;                                       // (at most 256 times 2^26 / kRun)
    const unsigned end = running_sum((unsigned)(to - from + kRun - 1) / kRun, shared, &runs);
    if (runs == 0) continue;
    shared.end[threadIdx.x] = end;                       // (the sum's barriers stand behind the reads of the round in front)
    shared.from[threadIdx.x] = from;
    shared.to[threadIdx.x] = to;
    __syncthreads();
    for (unsigned first = 0; first < runs; first += kThreads) {
      const unsigned run = first + threadIdx.x;
      int s = 0, n = 0, page[kRun] = {};
      size_t at = 0;                                     // of the run's first entry in the table
      if (run < runs) {
        // the first sequence whose runs end behind this one
#pragma unroll
        for (int step = kThreads / 2; step > 0; step >>= 1) s += shared.end[s + step - 1] <= run ? step : 0;
        const int entry = shared.from[s] + kRun * (int)(run - (s ? shared.end[s - 1] : 0));
        n = min(kRun, shared.to[s] - entry);
        at = (size_t)(base + s) * a.max_pages + entry;
      }
      // four at a time, also where the run ends between them; at the table's end one at a time
#pragma unroll
      for (int i = 0; i < kRun; i += 4) {
        if (__builtin_amdgcn_ballot_w64(i < n) == 0) continue;
        if (i < n) {
          if (at + i + 4 <= entries) {
            const i32x4_of4 y = *reinterpret_cast<const i32x4_of4*>(a.table + at + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) page[i + j] = y[j];
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) page[i + j] = i + j < n ? a.table[at + i + j] : -1;
          }
        }
      }
      unsigned there = 0;
#pragma unroll
      for (int i = 0; i < kRun; ++i) there |= i < n && (unsigned)page[i] < (unsigned)a.pages ? 1u << i : 0;
      // pages of the runs up to this one, and in the upper half of those in front of b (at most kThreads kRun each)
      const unsigned own = __builtin_popcount(there);
      if (KEEP && base + s == b && own) atomicAdd(&shared.own, own);
      unsigned all;
      const unsigned upto = running_sum(own | (base + s < b ? own : 0) << 16, shared, &all);
      if (!KEEP || *R + (all & 0xffff) <= kList) {
        unsigned to = (upto & 0xffff) - own + (KEEP ? (unsigned)*R : 0);
#pragma unroll
        for (int i = 0; i < kRun; ++i)
          if (there >> i & 1) shared.list[to++] = page[i];
      }
      if constexpr (!KEEP) {
        __syncthreads();
        f(*R, (int)(all & 0xffff));
      }
      *R += all & 0xffff;
      *R_b += all >> 16;
      if (*R > last) return;
    }
  }
}

struct Totals {
  long long R, G, R_b, G_b;      // over all sequences, over those in front of b
  int r_b;
  int status;
  int count;
};

// A thread's share of the sums.
__device__ __forceinline__ Sums share(const ResizeArgs& a, int b) {
  Sums t = {};
  for (int s = threadIdx.x; s < a.B; s += kThreads) {
    const Sequence q(a, s);
    t.bad |= q.bad;
    t.back += q.back();
    t.take += q.take();
    t.front_take += s < b ? q.take() : 0;
  }
  return t;
}

// exact: R and R_b are needed.
__device__ __forceinline__ Totals totals(const ResizeArgs& a, int b, Sums t, const int count, bool exact, Shared& shared) {
  if (threadIdx.x == 0) shared.own = 0;
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) {
    t.back += __shfl_xor(t.back, m, 64);
    t.take += __shfl_xor(t.take, m, 64);
    t.front_take += __shfl_xor(t.front_take, m, 64);
    t.bad |= __shfl_xor(t.bad, m, 64);
  }
  if ((threadIdx.x & 63) == 0) shared.sums[threadIdx.x >> 6] = t;
  __syncthreads();
  t = shared.sums[0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) {
    t.back += shared.sums[w].back;
    t.take += shared.sums[w].take;
    t.front_take += shared.sums[w].front_take;
    t.bad |= shared.sums[w].bad;
  }
  Totals r = {0, t.take, 0, t.front_take, 0, SVG_KV4_LENGTHS, count};
  if (t.bad || count < 0 || count > a.pages) return r;
  // At most t.back pages come back: the answer may be the same whatever their number.
  bool known = t.back == 0, count_them = !known && (exact || count + t.back > a.pages || r.G > count);
  for (;;) {
    if (count_them) {
      known = true;
      given_back<true>(a, 0, a.B, b, std::numeric_limits<long long>::max(), shared, &r.R, &r.R_b, [](long long, int) {});
    }
    if (count + r.R > a.pages) return r;
    if (r.G > count + r.R) {
      r.status = SVG_KV4_FULL;
      return r;
    }
    // the numbers that are taken from the stack (with R = 0 for an unknown one no fewer)
    int wrong = 0;
#pragma unroll 4
    for (int i = (int)max(0ll, count + r.R - r.G) + (int)threadIdx.x; i < count; i += kThreads)
      wrong |= (unsigned)a.r.free_pages[i] >= (unsigned)a.pages;
    wrong = __syncthreads_or(wrong);                     // (the list can be read)
    r.r_b = (int)shared.own;
    r.status = wrong ? SVG_KV4_PAGES : SVG_KV4_OK;
    if (!wrong || known) return r;
    count_them = true;
  }
}

// (behind the last read of the lengths)
__device__ __forceinline__ void write_state(const ResizeArgs& a, const Totals& t) {
  for (int s = threadIdx.x; s < a.B; s += kThreads) a.r.new_lengths[s] = t.status == SVG_KV4_OK ? a.r.wanted[s] : a.r.lengths[s];
  if (threadIdx.x == 0) {
    *a.r.new_count = t.status == SVG_KV4_OK ? (int)(t.count + t.R - t.G) : t.count;
    *a.r.status = t.status;
  }
}

__global__ __launch_bounds__(kThreads) void resize_kernel(ResizeArgs a) {
  __shared__ Shared shared;
  const int b = blockIdx.x, part = blockIdx.y;
  // (all loads in front of the first branch)
  const Sequence own(a, b);
  const int count = *a.r.free_count;
  const Sums sums = share(a, b);
  // tokens first .. last - 1 of the new ones are this workgroup's
  const long long first = (long long)part * a.each;
  const long long last = min(first + a.each, own.bad ? 0ll : (long long)max(0, own.wanted - own.len));
  // its new entries; the first may be another workgroup's too, which writes the same
  const int j0 = max(own.have, (int)((own.len + first) >> a.log2)), j1 = first < last ? min(own.want, (int)((own.len + last - 1) >> a.log2) + 1) : 0;
  const bool state = a.state && b == 0 && part == 0, gives = part == 0 && own.back() > 0, takes = j0 < j1;
  int32_t* const row = a.table + (size_t)b * a.max_pages;
  const int mask = (1 << a.log2) - 1;
  bool ok = false;
  if (first < last || gives || state) {                  // (the others have no slots to name)
    const Totals t = totals(a, b, sums, count, gives || takes || state, shared);
    ok = t.status == SVG_KV4_OK;
    // entry j: stack[top - j]; pages that other sequences give back in this call have the numbers (from the first one) top - count - j
    const long long top = t.count + t.R - 1 - t.G_b + own.have, lo = max(0ll, top - t.count - (j1 - 1)), hi = top - t.count - j0;
    if (ok && takes)
      for (int j = j0 + threadIdx.x; j < j1; j += kThreads)
        if (top - j < t.count) row[j] = a.r.free_pages[top - j];
    // Pages given back: this sequence's go to the stack, those that it takes into its row.  (The row of a sequence that takes pages is written, one that
    // gives pages back is only read.)
    if (ok && (gives ? t.r_b > 0 : takes && t.R > 0 && hi >= 0)) {
      auto put = [&](long long list, int n) {            // pages list .. list + n - 1 are in the list
        if (gives) {
          const long long from = max(t.R_b, list), to = min(t.R_b + t.r_b, list + n);
          for (long long i = from + threadIdx.x; i < to; i += kThreads) a.r.free_pages[t.count + i] = shared.list[i - list];
        } else {
          const long long from = max(lo, list), to = min(hi + 1, list + n);
          for (long long i = from + threadIdx.x; i < to; i += kThreads) row[top - t.count - i] = shared.list[i - list];
        }
      };
      long long all, front;
      if (t.R <= kList) put(0, (int)t.R);
      else
        given_back<false>(a, gives ? b : 0, gives ? b + 1 : a.B, b, gives ? t.r_b : hi, shared, &all, &front,
                          [&](long long first, int n) { put(first + (gives ? t.R_b : 0), n); });
    }
    __syncthreads();                                     // the row's new entries can be read, the lengths are not any more
    if (state) write_state(a, t);
  }
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
  __shared__ Shared shared;
  const Totals t = totals(a, 0, share(a, 0), *a.r.free_count, true, shared);
  __syncthreads();
  write_state(a, t);
}

// ---- rows into pages and out of them ---------------------------------------------------------------------------------
//
// A lane takes eight neighbouring elements of a row of keys and the same of values: D / 8 lanes a row, four of them a block of 32, whose largest
// magnitude needs two lane moves.  Bound: HBM (2 or 4 bytes an element in, 17/32 out; the other way round on the way back).  One row of each to a thread, and
// results past the caches: 40 heads of 4680 x 128 in bf16 written 22.5 us and read 18-19, 121 MB each, 5.4 and 6.3-6.7 TB/s (more than a large copy's 4.7-4.9: the
// caches hold part of it), 45.9 us as two calls; two rows to a thread 57.5, 48.6 with the stores alone changed, 52.5 with the rows alone; four rows 58.7.

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
