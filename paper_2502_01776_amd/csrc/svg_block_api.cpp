// C-ABI entry points of the operators around the attention: argument checks, then the launchers.
#include <algorithm>
#include <array>

#include "svg_block.h"

namespace {

// `rows` runs of `width` bytes, `step` apart (width <= step).
struct Span {
  uintptr_t first;
  size_t rows, width, step;
  uintptr_t last() const { return first + (rows - 1) * step + width; }
};
Span span(const void* p, size_t bytes) { return {reinterpret_cast<uintptr_t>(p), p && bytes ? size_t{1} : size_t{0}, bytes, bytes}; }
Span row_span(const void* p, int64_t rows, int64_t C, int64_t ld, int type) {
  const size_t size = svg::type_bytes(type);
  return {reinterpret_cast<uintptr_t>(p), p ? (size_t)rows : 0, (size_t)C * size, (size_t)(ld ? ld : C) * size};
}
// Column slices of one tensor lie in each other's gaps: with one step, runs whose places modulo the step differ never meet.  Runs of
// different steps are taken to meet wherever the places between their first and last byte do.
bool overlap(const Span& a, const Span& b) {
  if (!a.rows || !b.rows || a.first >= b.last() || b.first >= a.last()) return false;
  if (a.rows > 1 && b.rows > 1 && a.step != b.step) return true;
  if (a.rows == 1 && b.rows == 1) return true;
  const size_t step = a.rows > 1 ? a.step : b.step;
  const size_t behind = b.first >= a.first ? (b.first - a.first) % step : (step - (a.first - b.first) % step) % step;
  return behind < a.width || behind + b.width > step;
}

bool float_type(int t) { return t == SVG_BF16 || t == SVG_F16 || t == SVG_F32; }
bool norm_kind(int n) { return n == SVG_NORM_NONE || n == SVG_NORM_RMS || n == SVG_NORM_LAYER; }
bool activation_kind(int a) { return a == SVG_ACT_NONE || a == SVG_ACT_SILU || a == SVG_ACT_GELU_TANH; }
bool misaligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) != 0; }

constexpr long long kMaxStride = 1ll << 40;

int check_gate_norm(const svg_gate_norm_t* d) {
  if (!d || d->rows < 0 || d->C < 1 || d->groups < 1 || d->reserved != 0) return SVG_ERR_INVALID_ARG;
  if (d->stream_type != SVG_BF16 && d->stream_type != SVG_F32) return SVG_ERR_INVALID_ARG;
  if (d->branch_type != SVG_BF16 && d->branch_type != SVG_F16) return SVG_ERR_INVALID_ARG;
  if (!norm_kind(d->post_norm) || !norm_kind(d->pre_norm)) return SVG_ERR_INVALID_ARG;
  if (!(d->eps >= 0.f) || !(d->post_eps >= 0.f)) return SVG_ERR_INVALID_ARG;
  const int64_t lds[] = {d->ld_x, d->ld_y, d->ld_r, d->ld_h, d->ld_mod};
  for (int64_t ld : lds)
    if (ld && (ld < d->C || ld > kMaxStride)) return SVG_ERR_INVALID_ARG;
  if (!d->group_ptr && d->rows % d->groups) return SVG_ERR_INVALID_ARG;
  const void* words[] = {d->gate, d->scale, d->shift, d->group_ptr, d->post_weight, d->post_bias, d->weight, d->bias};
  for (const void* p : words)
    if (misaligned(p, 4)) return SVG_ERR_INVALID_ARG;
  if (d->C > 16384 || d->rows > svg::kMaxTokenRows) return SVG_ERR_UNSUPPORTED;
  // the furthest element of every tensor, as in check_tokens
  for (int64_t ld : lds)
    if ((__int128)std::max<int64_t>(d->rows, d->groups) * ld >= ((__int128)1 << 60)) return SVG_ERR_UNSUPPORTED;
  return SVG_OK;
}

// The tables and weights of a descriptor.
constexpr int kParameters = 8;
std::array<Span, kParameters> parameter_spans(const svg_gate_norm_t& d) {
  auto table = [&](const float* p) { return row_span(p, d.groups, d.C, d.ld_mod, SVG_F32); };
  auto vector = [&](const float* p) { return row_span(p, 1, d.C, 0, SVG_F32); };
  return {table(d.gate), table(d.scale), table(d.shift), span(d.group_ptr, (size_t)(d.groups + 1ll) * sizeof(int32_t)),
          vector(d.post_weight), vector(d.post_bias), vector(d.weight), vector(d.bias)};
}

// Checks a token matrix; fills t, its rows and columns and the bytes it spans.  An output's elements must not share places.
int check_tokens(const svg_tokens_t* d, bool output, svg::Tokens* t, long long* rows, long long* cols, size_t* bytes) {
  if (!d || d->B < 0 || d->N < 0 || d->H < 1 || d->D < 1 || d->reserved != 0 || !float_type(d->type)) return SVG_ERR_INVALID_ARG;
  if (d->stride_b < 0 || d->stride_n < 0 || d->stride_h < 0) return SVG_ERR_INVALID_ARG;
  if (d->stride_b > kMaxStride || d->stride_n > kMaxStride || d->stride_h > kMaxStride) return SVG_ERR_INVALID_ARG;
  if (d->B > svg::kMaxTokenRows || d->N > svg::kMaxTokenRows || d->B * d->N > svg::kMaxTokenRows) return SVG_ERR_UNSUPPORTED;
  if ((long long)d->H * d->D > svg::kMaxColumns) return SVG_ERR_UNSUPPORTED;
  *rows = d->B * d->N;
  *cols = (long long)d->H * d->D;
  *t = svg::Tokens{d->N ? d->N : 1, d->B > 1 ? d->stride_b : 0, d->N > 1 ? d->stride_n : 0, d->H > 1 ? d->stride_h : 0, d->D, d->type};
  const long long size[3] = {d->B, d->N, d->H}, stride[3] = {t->sb, t->sn, t->sh};
  // furthest element; the strides are at most 2^40 and the sizes 2^31
  __int128 last = d->D - 1;
  for (int k = 0; k < 3; ++k) last += (__int128)(size[k] > 0 ? size[k] - 1 : 0) * stride[k];
  if (last >= ((__int128)1 << 60)) return SVG_ERR_UNSUPPORTED;
  *bytes = *rows ? (size_t)(last + 1) * svg::type_bytes(d->type) : 0;
  if (output && *rows) {
    // from the smallest stride up, each has to step over all that lies inside it
    bool done[3] = {};
    __int128 inside = d->D;
    for (int n = 0; n < 3; ++n) {
      int k = -1;
      for (int j = 0; j < 3; ++j)
        if (!done[j] && (k < 0 || (size[j] > 1 ? stride[j] : 0) < (size[k] > 1 ? stride[k] : 0))) k = j;
      done[k] = true;
      if (size[k] <= 1) continue;
      if (stride[k] < inside) return SVG_ERR_ALIAS;
      inside += (__int128)(size[k] - 1) * stride[k];
    }
  }
  return SVG_OK;
}

int check_linear(int64_t M, int64_t N, int64_t K, const void* a, const void* a_scales, const void* w, const void* w_scales,
                 const float* bias, int activation) {
  if (M < 0 || N < 1 || K < 1) return SVG_ERR_INVALID_ARG;
  if (M > svg::kMaxTokenRows || N > svg::kMaxColumns || K > svg::kMaxColumns) return SVG_ERR_UNSUPPORTED;
  if (!activation_kind(activation)) return SVG_ERR_INVALID_ARG;
  if (!a || !a_scales || !w || !w_scales || misaligned(bias, 4)) return SVG_ERR_INVALID_ARG;
  const void* p[] = {a, a_scales, w, w_scales};
  for (const void* x : p)
    if (svg::misaligned16(x)) return SVG_ERR_INVALID_ARG;
  return SVG_OK;
}

}  // namespace

extern "C" {

int svg_gate_norm_fwd(const svg_gate_norm_t* desc, const void* x, const void* y, void* r, void* h, void* codes, void* scales,
                      void* stream) {
  const int rc = check_gate_norm(desc);
  if (rc != SVG_OK) return rc;
  const svg_gate_norm_t& d = *desc;
  if (!x || (!r && !h && !codes) || (codes == nullptr) != (scales == nullptr)) return SVG_ERR_INVALID_ARG;
  const int sb = svg::type_bytes(d.stream_type), bb = svg::type_bytes(d.branch_type);
  if (misaligned(x, sb) || misaligned(r, sb) || misaligned(y, bb) || misaligned(h, bb)) return SVG_ERR_INVALID_ARG;
  if (svg::misaligned16(codes) || svg::misaligned16(scales)) return SVG_ERR_INVALID_ARG;
  const Span in[2] = {row_span(x, d.rows, d.C, d.ld_x, d.stream_type), row_span(y, d.rows, d.C, d.ld_y, d.branch_type)};
  const Span out[4] = {row_span(r, d.rows, d.C, d.ld_r, d.stream_type), row_span(h, d.rows, d.C, d.ld_h, d.branch_type),
                       span(codes, svg::fp4_codes_bytes(d.rows, d.C)), span(scales, svg::fp4_scales_bytes(d.rows, d.C))};
  if (codes && d.rows && !svg::gate_norm_writes_codes(d, x, y, r, h)) return SVG_ERR_UNSUPPORTED;
  const std::array<Span, kParameters> parameters = parameter_spans(d);
  const bool in_place = r == x && (d.ld_r ? d.ld_r : d.C) == (d.ld_x ? d.ld_x : d.C);
  for (int o = 0; o < 4; ++o) {
    for (int k = 0; k < 2; ++k)
      if (overlap(out[o], in[k]) && !(o == 0 && k == 0 && in_place)) return SVG_ERR_ALIAS;
    for (int k = o + 1; k < 4; ++k)
      if (overlap(out[o], out[k])) return SVG_ERR_ALIAS;
    for (const Span& p : parameters)
      if (overlap(out[o], p)) return SVG_ERR_ALIAS;
  }
  if (!d.rows) return SVG_OK;
  return svg::launch_gate_norm(d, x, y, r, h, codes, scales, static_cast<hipStream_t>(stream));
}

size_t svg_gate_norm_workspace_bytes(const svg_gate_norm_t* desc) {
  return check_gate_norm(desc) == SVG_OK ? svg::gate_norm_workspace_bytes(*desc) : 0;
}

int svg_gate_norm_bwd(const svg_gate_norm_t* desc, const void* r, const void* y, const void* dr, const void* dh, void* dx, void* dy,
                      const svg_gate_norm_grads_t* grads, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_gate_norm(desc);
  if (rc != SVG_OK) return rc;
  const svg_gate_norm_t& d = *desc;
  svg_gate_norm_grads_t none = {};
  const svg_gate_norm_grads_t& gr = grads ? *grads : none;
  if (gr.ld_mod && (gr.ld_mod < d.C || gr.ld_mod > kMaxStride)) return SVG_ERR_INVALID_ARG;
  if ((__int128)d.groups * gr.ld_mod >= ((__int128)1 << 60)) return SVG_ERR_UNSUPPORTED;
  float* const out_grads[7] = {gr.gate, gr.scale, gr.shift, gr.post_weight, gr.post_bias, gr.weight, gr.bias};
  bool any = dx || dy;
  for (const float* p : out_grads) {
    if (misaligned(p, 4)) return SVG_ERR_INVALID_ARG;
    any = any || p;
  }
  if (!any || (!dr && !dh)) return SVG_ERR_INVALID_ARG;
  // the stream is needed for the norm's statistics, the branch for its own norm's and for the gate's gradient
  if (dh && !r) return SVG_ERR_INVALID_ARG;
  if (!y && ((dy && d.post_norm != SVG_NORM_NONE) || gr.gate || gr.post_weight || gr.post_bias)) return SVG_ERR_INVALID_ARG;
  const int sb = svg::type_bytes(d.stream_type), bb = svg::type_bytes(d.branch_type);
  if (misaligned(r, sb) || misaligned(dr, sb) || misaligned(dx, sb) || misaligned(y, bb) || misaligned(dh, bb) || misaligned(dy, bb))
    return SVG_ERR_INVALID_ARG;
  const size_t need = svg::gate_norm_workspace_bytes(d);
  if (need && (!workspace || workspace_bytes < need)) return SVG_ERR_WORKSPACE;
  if (svg::misaligned16(workspace)) return SVG_ERR_INVALID_ARG;
  const int64_t lx = d.ld_x ? d.ld_x : d.C, ly = d.ld_y ? d.ld_y : d.C, lr = d.ld_r ? d.ld_r : d.C, lh = d.ld_h ? d.ld_h : d.C;
  const Span in[4] = {row_span(r, d.rows, d.C, lr, d.stream_type), row_span(y, d.rows, d.C, ly, d.branch_type),
                      row_span(dr, d.rows, d.C, lr, d.stream_type), row_span(dh, d.rows, d.C, lh, d.branch_type)};
  auto table = [&](const float* p) { return row_span(p, d.groups, d.C, gr.ld_mod, SVG_F32); };
  auto vector = [&](const float* p) { return row_span(p, 1, d.C, 0, SVG_F32); };
  const Span out[10] = {row_span(dx, d.rows, d.C, lx, d.stream_type), row_span(dy, d.rows, d.C, ly, d.branch_type), span(workspace, need),
                        table(gr.gate), table(gr.scale), table(gr.shift),
                        vector(gr.post_weight), vector(gr.post_bias), vector(gr.weight), vector(gr.bias)};
  const std::array<Span, kParameters> parameters = parameter_spans(d);
  for (int o = 0; o < 10; ++o) {
    for (int k = 0; k < 4; ++k) {
      const bool in_place = (o == 0 && k == 2 && dx == dr && lx == lr) || (o == 1 && k == 1 && dy == y) ||
                            (o == 1 && k == 3 && dy == dh && ly == lh);
      if (overlap(out[o], in[k]) && !in_place) return SVG_ERR_ALIAS;
    }
    for (int k = o + 1; k < 10; ++k)
      if (overlap(out[o], out[k])) return SVG_ERR_ALIAS;
    for (const Span& p : parameters)
      if (overlap(out[o], p)) return SVG_ERR_ALIAS;
  }
  return svg::launch_gate_norm_grad(d, r, y, dr, dh, dx, dy, gr, static_cast<float*>(workspace), static_cast<hipStream_t>(stream));
}

size_t svg_fp4_buffer_bytes(int64_t rows, int64_t cols, int which) {
  if (rows < 0 || rows > svg::kMaxTokenRows || cols < 1 || cols > svg::kMaxColumns) return 0;
  if (which == SVG_FP4_CODES) return svg::fp4_codes_bytes(rows, cols);
  if (which == SVG_FP4_SCALES) return svg::fp4_scales_bytes(rows, cols);
  return 0;
}

int svg_fp4_quantize(const svg_tokens_t* tokens, const void* x, int activation, void* codes, void* scales, void* stream) {
  svg::Tokens t;
  long long rows, cols;
  size_t bytes;
  const int rc = check_tokens(tokens, false, &t, &rows, &cols, &bytes);
  if (rc != SVG_OK) return rc;
  if (!activation_kind(activation) || !x || !codes || !scales || misaligned(x, svg::type_bytes(t.type))) return SVG_ERR_INVALID_ARG;
  if (svg::misaligned16(codes) || svg::misaligned16(scales)) return SVG_ERR_INVALID_ARG;
  const Span in = span(x, bytes), c = span(codes, svg::fp4_codes_bytes(rows, cols)), s = span(scales, svg::fp4_scales_bytes(rows, cols));
  if (overlap(in, c) || overlap(in, s) || overlap(c, s)) return SVG_ERR_ALIAS;
  if (!rows) return SVG_OK;
  return svg::launch_fp4_quantize(t, rows, (int)cols, x, activation, codes, scales, static_cast<hipStream_t>(stream));
}

int svg_fp4_dequantize(const svg_tokens_t* tokens, const void* codes, const void* scales, void* x, void* stream) {
  svg::Tokens t;
  long long rows, cols;
  size_t bytes;
  const int rc = check_tokens(tokens, true, &t, &rows, &cols, &bytes);
  if (rc != SVG_OK) return rc;
  if (!x || !codes || !scales || misaligned(x, svg::type_bytes(t.type))) return SVG_ERR_INVALID_ARG;
  if (svg::misaligned16(codes) || svg::misaligned16(scales)) return SVG_ERR_INVALID_ARG;
  const Span out = span(x, bytes);
  if (overlap(out, span(codes, svg::fp4_codes_bytes(rows, cols))) || overlap(out, span(scales, svg::fp4_scales_bytes(rows, cols))))
    return SVG_ERR_ALIAS;
  if (!rows) return SVG_OK;
  return svg::launch_fp4_dequantize(t, rows, (int)cols, codes, scales, x, static_cast<hipStream_t>(stream));
}

size_t svg_fp4_linear_workspace_bytes(int64_t, int64_t, int64_t) { return 0; }

int svg_fp4_linear(int64_t M, int64_t N, int64_t K, const void* a, const void* a_scales, const void* w, const void* w_scales,
                   const float* bias, int activation, const svg_tokens_t* out_desc, void* out, void*, size_t, void* stream) {
  int rc = check_linear(M, N, K, a, a_scales, w, w_scales, bias, activation);
  if (rc != SVG_OK) return rc;
  svg::Tokens t;
  long long rows, cols;
  size_t bytes;
  rc = check_tokens(out_desc, true, &t, &rows, &cols, &bytes);
  if (rc != SVG_OK) return rc;
  if (rows != M || cols != N || !out || misaligned(out, svg::type_bytes(t.type))) return SVG_ERR_INVALID_ARG;
  if (!M) return SVG_OK;
  const Span in[5] = {span(a, svg::fp4_codes_bytes(M, K)), span(a_scales, svg::fp4_scales_bytes(M, K)), span(w, svg::fp4_codes_bytes(N, K)),
                      span(w_scales, svg::fp4_scales_bytes(N, K)), span(bias, (size_t)N * sizeof(float))};
  for (const Span& i : in)
    if (overlap(i, span(out, bytes))) return SVG_ERR_ALIAS;
  return svg::launch_fp4_linear(M, (int)N, (int)K, a, a_scales, w, w_scales, bias, activation, &t, out, nullptr, nullptr,
                                static_cast<hipStream_t>(stream));
}

int svg_fp4_linear_quantize(int64_t M, int64_t N, int64_t K, const void* a, const void* a_scales, const void* w, const void* w_scales,
                            const float* bias, int activation, void* codes, void* scales, void*, size_t, void* stream) {
  int rc = check_linear(M, N, K, a, a_scales, w, w_scales, bias, activation);
  if (rc != SVG_OK) return rc;
  if (!codes || !scales || svg::misaligned16(codes) || svg::misaligned16(scales)) return SVG_ERR_INVALID_ARG;
  if (!M) return SVG_OK;
  const Span in[5] = {span(a, svg::fp4_codes_bytes(M, K)), span(a_scales, svg::fp4_scales_bytes(M, K)), span(w, svg::fp4_codes_bytes(N, K)),
                      span(w_scales, svg::fp4_scales_bytes(N, K)), span(bias, (size_t)N * sizeof(float))};
  const Span outs[2] = {span(codes, svg::fp4_codes_bytes(M, N)), span(scales, svg::fp4_scales_bytes(M, N))};
  for (const Span& o : outs)
    for (const Span& i : in)
      if (overlap(i, o)) return SVG_ERR_ALIAS;
  if (overlap(outs[0], outs[1])) return SVG_ERR_ALIAS;
  return svg::launch_fp4_linear(M, (int)N, (int)K, a, a_scales, w, w_scales, bias, activation, nullptr, nullptr, codes, scales,
                                static_cast<hipStream_t>(stream));
}

}  // extern "C"
