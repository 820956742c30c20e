// The cache of keys and values in 4 bits (svg_kv4_t): its layout and the kernels' launchers.
#pragma once
#include "svg_block.h"

namespace svg {

// A cache after validation.
struct Kv4 {
  unsigned char* data;
  int32_t* table;
  int B, H, D;
  int page_log2, pages, max_pages;
  // Bytes of a page's record for one head, and where its parts begin.
  __host__ __device__ long long record() const { return (long long)(D + D / 16) << page_log2; }
  __host__ __device__ int values() const { return (D / 2) << page_log2; }
  __host__ __device__ int key_scales() const { return D << page_log2; }
  __host__ __device__ int value_scales() const { return (D + D / 32) << page_log2; }
};

// Token rows of one tensor, as heads of the cache's dimension.
struct HeadRows {
  long long N, sb, sn, sh;      // tokens of a batch entry; strides in elements
  int type;
};

struct Kv4Resize {
  const int32_t *lengths, *wanted, *free_count;
  int32_t *free_pages, *new_lengths, *new_count, *status;
  int64_t* slots;
  int tokens;
};
// in_place: new_lengths is lengths or new_count is free_count
int launch_kv4_resize(const Kv4& c, const Kv4Resize& r, bool in_place, hipStream_t stream);
int launch_kv4_write(const Kv4& c, const HeadRows& k, const void* kp, const HeadRows& v, const void* vp, const int64_t* slots, long long rows,
                     hipStream_t stream);
int launch_kv4_read(const Kv4& c, const HeadRows& k, void* kp, const HeadRows& v, void* vp, const int64_t* slots, long long rows,
                    hipStream_t stream);

// How a call of the attention is cut (host function; sizes only).
struct Kv4Plan {
  int rows;              // query rows of a head of the cache: N times the query heads that share it
  int tile;              // rows of a workgroup: 16 or 32 (its wavefronts share the rows and split the keys) or 128 (32 rows a wavefront)
  int tiles;             // row tiles of a head of a sequence
  int parts;             // parts that the keys of all sequences are cut into, one each at least
  int reach;             // an estimate of the keys that a row tile visits: for dealing the parts only
};
Kv4Plan kv4_plan(const Kv4& c, const svg_kv4_attn_t& attn, long long N, int group);
size_t kv4_workspace_bytes(const Kv4& c, const Kv4Plan& plan);
int launch_kv4_attn(const Kv4& c, const svg_kv4_attn_t& attn, const Kv4Plan& plan, const HeadRows& q, const void* qp, const HeadRows& o,
                    void* op, int group, float* lse, void* workspace, hipStream_t stream);

// out = act(in_act(x) w^T + bias) of few rows (svg_fp4_rows.hip)
int launch_fp4_rows(const Tokens& x_tok, const void* x, int in_activation, long long M, int N, int K, const void* w, const void* w_scales,
                    const float* bias, int activation, const Tokens& out_tok, void* out, hipStream_t stream);

}  // namespace svg
