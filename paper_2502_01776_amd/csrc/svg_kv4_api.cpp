// C-ABI entry points of the 4-bit cache of keys and values and of few rows times 4-bit weights: argument checks, then the launchers.
#include "svg_checks.h"
#include "svg_kv4.h"

namespace {

using namespace svg::checks;

// The fields that every call looks at.
int check_cache(const svg_kv4_t* d, svg::Kv4* c) {
  if (!d || d->B < 0 || d->H < 1 || d->pages < 0 || d->max_pages < 0 || d->reserved != 0) return SVG_ERR_INVALID_ARG;
  if (d->page_size < 1 || (d->page_size & (d->page_size - 1))) return SVG_ERR_INVALID_ARG;
  if ((d->D != 64 && d->D != 128) || d->page_size < 16 || d->page_size > 65536 || d->B > 65536) return SVG_ERR_UNSUPPORTED;
  if ((long long)d->H * d->D > svg::kMaxColumns) return SVG_ERR_UNSUPPORTED;
  *c = svg::Kv4{static_cast<unsigned char*>(d->data), d->page_table, d->B, d->H, d->D, __builtin_ctz((unsigned)d->page_size), d->pages, d->max_pages};
  if ((__int128)c->record() * d->H * d->pages >= ((__int128)1 << 60)) return SVG_ERR_UNSUPPORTED;
  return SVG_OK;
}
size_t data_bytes(const svg::Kv4& c) { return (size_t)c.record() * c.H * c.pages; }
size_t table_bytes(const svg::Kv4& c) { return (size_t)c.B * c.max_pages * sizeof(int32_t); }
// Places of a sequence's tokens are 32-bit numbers with room for a block of 64 behind them.
bool places_fit(const svg::Kv4& c) { return ((long long)c.max_pages << c.page_log2) <= (1ll << 30); }

// A token matrix as heads of dimension D: [B,H,N,D], or H*D columns in one run.  Fills their number.
int check_heads(const svg_tokens_t* d, bool output, int D, svg::HeadRows* h, int* heads, long long* rows, Span* where, const void* p) {
  svg::Tokens t;
  long long cols;
  size_t bytes;
  const int rc = check_tokens(d, output, &t, rows, &cols, &bytes);
  if (rc != SVG_OK) return rc;
  if (d->D != D && (d->H != 1 || d->D % D)) return SVG_ERR_INVALID_ARG;
  if ((!p && *rows) || misaligned(p, svg::type_bytes(t.type))) return SVG_ERR_INVALID_ARG;      // (an empty tensor has no address)
  *heads = (int)(cols / D);
  *h = svg::HeadRows{t.N, t.sb, t.sn, d->D == D ? t.sh : D, t.type};
  // rows one step apart whose heads lie between one and the next are column slices; anything else is taken as one run
  const long long width = (long long)(*heads - 1) * h->sh + D;
  const bool even = d->B <= 1 || d->N <= 1 || t.sb == t.sn * d->N;
  const long long step = d->N > 1 ? t.sn : d->B > 1 ? t.sb : width;
  const size_t size = svg::type_bytes(t.type);
  *where = *rows && even && step >= width ? Span{reinterpret_cast<uintptr_t>(p), (size_t)*rows, (size_t)width * size, (size_t)step * size} : span(p, bytes);
  return SVG_OK;
}

// What a write and a read have in common.
struct Kv {
  svg::Kv4 c;
  svg::HeadRows k, v;
  Span where_k, where_v;
  long long rows;
};
int check_kv(const svg_kv4_t* cache, bool output, const svg_tokens_t* k_desc, const void* k, const svg_tokens_t* v_desc, const void* v,
             const int64_t* slots, Kv* a) {
  int rc = check_cache(cache, &a->c);
  if (rc != SVG_OK) return rc;
  int k_heads, v_heads;
  long long v_rows;
  if ((rc = check_heads(k_desc, output, a->c.D, &a->k, &k_heads, &a->rows, &a->where_k, k)) != SVG_OK) return rc;
  if ((rc = check_heads(v_desc, output, a->c.D, &a->v, &v_heads, &v_rows, &a->where_v, v)) != SVG_OK) return rc;
  if (k_heads != a->c.H || v_heads != a->c.H || k_desc->B != v_desc->B || k_desc->N != v_desc->N) return SVG_ERR_INVALID_ARG;
  if ((!slots && a->rows) || misaligned(slots, 8) || (!a->c.data && a->c.pages) || svg::misaligned16(a->c.data)) return SVG_ERR_INVALID_ARG;
  return SVG_OK;
}

struct Attn {
  svg::Kv4 c;
  svg::HeadRows q;
  Span where_q;
  int heads, group;
  svg::Kv4Plan plan;
};
int check_attn(const svg_kv4_t* cache, const svg_kv4_attn_t* attn, const svg_tokens_t* q_desc, const void* q, Attn* a) {
  int rc = check_cache(cache, &a->c);
  if (rc != SVG_OK) return rc;
  if (!attn || (attn->causal != 0 && attn->causal != 1) || attn->block < 1 || attn->sink < 0 || attn->max_kv < 0) return SVG_ERR_INVALID_ARG;
  // (a scale that is not a normal number beside the scores' would make 0 infinity of a masked one)
  if (!(attn->softmax_scale <= 0.f || (attn->softmax_scale >= 1.0e-30f && attn->softmax_scale <= 1.0e30f))) return SVG_ERR_INVALID_ARG;
  if (!places_fit(a->c)) return SVG_ERR_UNSUPPORTED;
  long long rows;
  if ((rc = check_heads(q_desc, false, a->c.D, &a->q, &a->heads, &rows, &a->where_q, q)) != SVG_OK) return rc;
  if (a->q.type != SVG_BF16) return SVG_ERR_UNSUPPORTED;
  if (q_desc->B != a->c.B || a->heads % a->c.H) return SVG_ERR_INVALID_ARG;
  a->group = a->heads / a->c.H;
  if (q_desc->N * a->group > (1ll << 30)) return SVG_ERR_UNSUPPORTED;
  a->plan = svg::kv4_plan(a->c, *attn, q_desc->N, a->group);
  return SVG_OK;
}

}  // namespace

extern "C" {

size_t svg_kv4_bytes(const svg_kv4_t* cache) {
  svg::Kv4 c;
  return check_cache(cache, &c) == SVG_OK ? data_bytes(c) : 0;
}

int svg_kv4_resize(const svg_kv4_t* cache, const int32_t* lengths, const int32_t* wanted, int32_t* free_pages, const int32_t* free_count,
                   int32_t* new_lengths, int32_t* new_count, int64_t* slots, int32_t tokens, int32_t* status, void* stream) {
  svg::Kv4 c;
  const int rc = check_cache(cache, &c);
  if (rc != SVG_OK) return rc;
  if (tokens < 0 || !free_count || !new_count || !status || (!free_pages && c.pages)) return SVG_ERR_INVALID_ARG;
  if (c.B && (!lengths || !wanted || !new_lengths || (!c.table && c.max_pages))) return SVG_ERR_INVALID_ARG;
  const void* words[] = {lengths, wanted, free_pages, free_count, new_lengths, new_count, status, c.table};
  for (const void* p : words)
    if (misaligned(p, 4)) return SVG_ERR_INVALID_ARG;
  if (misaligned(slots, 8)) return SVG_ERR_INVALID_ARG;
  if (!places_fit(c) || tokens > (1 << 30)) return SVG_ERR_UNSUPPORTED;
  const size_t each = (size_t)c.B * 4;
  const Span in[3] = {span(lengths, each), span(wanted, each), span(free_count, 4)};
  const Span out[6] = {span(new_lengths, each), span(new_count, 4), span(status, 4), span(slots, (size_t)c.B * (size_t)tokens * 8),
                       span(free_pages, (size_t)c.pages * 4), span(c.table, table_bytes(c))};
  for (int o = 0; o < 6; ++o) {
    for (int k = 0; k < 3; ++k)
      if (overlap(out[o], in[k]) && !(o == 0 && k == 0 && new_lengths == lengths) && !(o == 1 && k == 2 && new_count == free_count))
        return SVG_ERR_ALIAS;
    for (int k = o + 1; k < 6; ++k)
      if (overlap(out[o], out[k])) return SVG_ERR_ALIAS;
  }
  const svg::Kv4Resize r = {lengths, wanted, free_count, free_pages, new_lengths, new_count, status, slots, tokens};
  return svg::launch_kv4_resize(c, r, new_lengths == lengths || new_count == free_count, static_cast<hipStream_t>(stream));
}

int svg_kv4_write(const svg_kv4_t* cache, const svg_tokens_t* k_desc, const void* k, const svg_tokens_t* v_desc, const void* v,
                  const int64_t* slots, void* stream) {
  Kv a;
  const int rc = check_kv(cache, false, k_desc, k, v_desc, v, slots, &a);
  if (rc != SVG_OK) return rc;
  const Span data = span(a.c.data, data_bytes(a.c));
  if (overlap(data, a.where_k) || overlap(data, a.where_v) || overlap(data, span(slots, (size_t)a.rows * 8))) return SVG_ERR_ALIAS;
  if (!a.rows || !a.c.pages) return SVG_OK;
  return svg::launch_kv4_write(a.c, a.k, k, a.v, v, slots, a.rows, static_cast<hipStream_t>(stream));
}

int svg_kv4_read(const svg_kv4_t* cache, const int64_t* slots, const svg_tokens_t* k_desc, void* k, const svg_tokens_t* v_desc, void* v,
                 void* stream) {
  Kv a;
  const int rc = check_kv(cache, true, k_desc, k, v_desc, v, slots, &a);
  if (rc != SVG_OK) return rc;
  const Span in[2] = {span(a.c.data, data_bytes(a.c)), span(slots, (size_t)a.rows * 8)};
  for (const Span& i : in)
    if (overlap(i, a.where_k) || overlap(i, a.where_v)) return SVG_ERR_ALIAS;
  if (overlap(a.where_k, a.where_v)) return SVG_ERR_ALIAS;
  if (!a.rows || !a.c.pages) return SVG_OK;
  return svg::launch_kv4_read(a.c, a.k, k, a.v, v, slots, a.rows, static_cast<hipStream_t>(stream));
}

size_t svg_kv4_attn_workspace_bytes(const svg_kv4_t* cache, const svg_kv4_attn_t* attn, const svg_tokens_t* q_desc) {
  Attn a;
  const void* anywhere = reinterpret_cast<const void*>(uintptr_t{64});      // (the size does not depend on it)
  return check_attn(cache, attn, q_desc, anywhere, &a) == SVG_OK ? svg::kv4_workspace_bytes(a.c, a.plan) : 0;
}

int svg_kv4_attn_fwd(const svg_kv4_t* cache, const svg_kv4_attn_t* attn, const svg_tokens_t* q_desc, const void* q,
                     const svg_tokens_t* o_desc, void* o, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  Attn a;
  int rc = check_attn(cache, attn, q_desc, q, &a);
  if (rc != SVG_OK) return rc;
  svg::HeadRows out;
  Span where_o;
  int o_heads;
  long long o_rows;
  if ((rc = check_heads(o_desc, true, a.c.D, &out, &o_heads, &o_rows, &where_o, o)) != SVG_OK) return rc;
  if (out.type != SVG_BF16) return SVG_ERR_UNSUPPORTED;
  if (o_heads != a.heads || o_desc->B != q_desc->B || o_desc->N != q_desc->N || misaligned(lse, 4)) return SVG_ERR_INVALID_ARG;
  if (a.c.B && (!attn->kv_len || (!a.c.table && a.c.max_pages))) return SVG_ERR_INVALID_ARG;
  if ((!a.c.data && a.c.pages) || svg::misaligned16(a.c.data) || misaligned(a.c.table, 4) || misaligned(attn->kv_len, 4) || misaligned(attn->q_len, 4))
    return SVG_ERR_INVALID_ARG;
  const size_t need = svg::kv4_workspace_bytes(a.c, a.plan);
  if (need && (!workspace || workspace_bytes < need)) return SVG_ERR_WORKSPACE;
  if (svg::misaligned16(workspace)) return SVG_ERR_INVALID_ARG;
  const size_t each = (size_t)a.c.B * 4;
  const Span in[5] = {a.where_q, span(a.c.data, data_bytes(a.c)), span(a.c.table, table_bytes(a.c)), span(attn->kv_len, each), span(attn->q_len, each)};
  const Span outs[3] = {where_o, span(lse, (size_t)o_rows * o_heads * 4), span(workspace, need)};
  for (int x = 0; x < 3; ++x) {
    for (const Span& i : in)
      if (overlap(outs[x], i)) return SVG_ERR_ALIAS;
    for (int y = x + 1; y < 3; ++y)
      if (overlap(outs[x], outs[y])) return SVG_ERR_ALIAS;
  }
  if (!o_rows) return SVG_OK;
  return svg::launch_kv4_attn(a.c, *attn, a.plan, a.q, q, out, o, a.group, lse, workspace, static_cast<hipStream_t>(stream));
}

int svg_fp4_linear_rows(const svg_tokens_t* x_desc, const void* x, int in_activation, int64_t N, const void* w, const void* w_scales,
                        const float* bias, int activation, const svg_tokens_t* out_desc, void* out, void* stream) {
  svg::Tokens xt, ot;
  long long M, K, rows, cols;
  size_t x_bytes, out_bytes;
  int rc = check_tokens(x_desc, false, &xt, &M, &K, &x_bytes);
  if (rc != SVG_OK) return rc;
  if ((rc = check_tokens(out_desc, true, &ot, &rows, &cols, &out_bytes)) != SVG_OK) return rc;
  if (!activation_kind(in_activation) || !activation_kind(activation) || N < 1 || rows != M || cols != N) return SVG_ERR_INVALID_ARG;
  if ((M && (!x || !out)) || !w || !w_scales || misaligned(x, svg::type_bytes(xt.type)) || misaligned(out, svg::type_bytes(ot.type)))
    return SVG_ERR_INVALID_ARG;
  if (svg::misaligned16(w) || svg::misaligned16(w_scales) || misaligned(bias, 4)) return SVG_ERR_INVALID_ARG;
  if (M > 1024) return SVG_ERR_UNSUPPORTED;
  const Span in[4] = {span(x, x_bytes), span(w, svg::fp4_codes_bytes(N, K)), span(w_scales, svg::fp4_scales_bytes(N, K)),
                      span(bias, (size_t)N * sizeof(float))};
  for (const Span& i : in)
    if (overlap(i, span(out, out_bytes))) return SVG_ERR_ALIAS;
  if (!M) return SVG_OK;
  return svg::launch_fp4_rows(xt, x, in_activation, M, (int)N, (int)K, w, w_scales, bias, activation, ot, out, static_cast<hipStream_t>(stream));
}

}  // extern "C"
