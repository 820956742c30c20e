// Checks of arguments that the entry points around the attention and of the 4-bit cache share (host code only).
#pragma once
#include "svg_block.h"

namespace svg {
namespace checks {

// `rows` runs of `width` bytes, `step` apart (width <= step).
struct Span {
  uintptr_t first;
  size_t rows, width, step;
  uintptr_t last() const { return first + (rows - 1) * step + width; }
};
inline Span span(const void* p, size_t bytes) { return {reinterpret_cast<uintptr_t>(p), p && bytes ? size_t{1} : size_t{0}, bytes, bytes}; }
inline Span row_span(const void* p, int64_t rows, int64_t C, int64_t ld, int type) {
  const size_t size = svg::type_bytes(type);
  return {reinterpret_cast<uintptr_t>(p), p ? (size_t)rows : 0, (size_t)C * size, (size_t)(ld ? ld : C) * size};
}
// Column slices of one tensor lie in each other's gaps: with one step, runs whose places modulo the step differ never meet.  Runs of
// different steps are taken to meet wherever the places between their first and last byte do.
inline bool overlap(const Span& a, const Span& b) {
  if (!a.rows || !b.rows || a.first >= b.last() || b.first >= a.last()) return false;
  if (a.rows > 1 && b.rows > 1 && a.step != b.step) return true;
  if (a.rows == 1 && b.rows == 1) return true;
  const size_t step = a.rows > 1 ? a.step : b.step;
  const size_t behind = b.first >= a.first ? (b.first - a.first) % step : (step - (a.first - b.first) % step) % step;
  return behind < a.width || behind + b.width > step;
}

inline bool float_type(int t) { return t == SVG_BF16 || t == SVG_F16 || t == SVG_F32; }
inline bool norm_kind(int n) { return n == SVG_NORM_NONE || n == SVG_NORM_RMS || n == SVG_NORM_LAYER; }
inline bool activation_kind(int a) { return a == SVG_ACT_NONE || a == SVG_ACT_SILU || a == SVG_ACT_GELU_TANH; }
inline bool misaligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) != 0; }

constexpr long long kMaxStride = 1ll << 40;

// Checks a token matrix; fills t, its rows and columns and the bytes it spans.  An output's elements must not share places.
inline int check_tokens(const svg_tokens_t* d, bool output, svg::Tokens* t, long long* rows, long long* cols, size_t* bytes) {
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

}  // namespace checks
}  // namespace svg
