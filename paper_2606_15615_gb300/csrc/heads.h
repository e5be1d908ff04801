// Heads of packed tokens (moeca_heads): what the kernels take, and the checks of the calls.
#pragma once

#include <numeric>

#include "calls.h"
#include "moeca_attention.h"

namespace moeca {

struct Heads {
  void* data;
  int64_t token_stride, head_stride;  // elements
  int heads;
};
inline Heads device_heads(const moeca_heads& h) { return {h.data, h.token_stride, h.head_stride, h.heads}; }

constexpr int64_t kMaxStride = int64_t(1) << 40;  // elements; with 2^20 heads, and tokens as checked, extents stay in 64 bits

// The bytes from the first value to the last.
inline Range heads_range(const moeca_heads& h, int64_t tokens, int dim, int64_t es) {
  if (tokens <= 0 || h.heads <= 0) return {nullptr, 0};
  return {h.data, ((tokens - 1) * h.token_stride + (h.heads - 1) * h.head_stride + dim) * es};
}

// What is wrong with heads (null: nothing).  Written heads must not overlap one another.
inline const char* bad_heads(const moeca_heads& h, int64_t tokens, int dim, int dtype, bool written) {
  if (h.heads < 0 || h.heads > (1 << 20)) return "heads: 0 .. 2^20 heads";
  if (tokens <= 0 || h.heads == 0) return nullptr;
  if (!h.data) return "heads: NULL";
  if (addr(h.data) % elem_size(dtype)) return "heads: not aligned to the type";
  if (h.token_stride < 0 || h.head_stride < 0 || h.token_stride > kMaxStride || h.head_stride > kMaxStride / h.heads ||
      h.token_stride > (int64_t(1) << 58) / tokens)
    return "heads: strides out of range";
  if (written) {
    const int64_t token = (h.heads - 1) * h.head_stride + dim, head = (tokens - 1) * h.token_stride + dim;
    const bool by_token = (h.heads == 1 || h.head_stride >= dim) && (tokens == 1 || h.token_stride >= token);
    const bool by_head = (tokens == 1 || h.token_stride >= dim) && (h.heads == 1 || h.head_stride >= head);
    if (!by_token && !by_head) return "heads: written heads overlap one another";
  }
  return nullptr;
}

inline bool same_heads(const moeca_heads& a, const moeca_heads& b) {
  return a.data == b.data && a.heads == b.heads && a.token_stride == b.token_stride && a.head_stride == b.head_stride;
}

// Whether two sets of heads (an, bn tokens of dim values) share a value.  Parts
// of one fused buffer do not, although their ranges do: within the common token or head
// stride, or the largest step that all strides are multiples of, they lie side by side.
inline bool heads_overlap(const moeca_heads& a, int64_t an, const moeca_heads& b, int64_t bn, int dim, int64_t es) {
  if (!overlap(heads_range(a, an, dim, es), heads_range(b, bn, dim, es))) return false;
  const auto apart = [&](int64_t stride, int64_t ea, int64_t eb) {
    // All of a lies in [0, ea) + multiples of the stride, all of b in [d, d + eb).
    if (stride <= 0 || ea > stride || eb > stride) return false;
    stride *= es;
    const int64_t gap = static_cast<int64_t>(addr(b.data) - addr(a.data)) % stride;
    const int64_t d = gap < 0 ? gap + stride : gap;
    return d >= ea * es && d + eb * es <= stride;
  };
  if (a.token_stride == b.token_stride &&
      apart(a.token_stride, (a.heads - 1) * a.head_stride + dim, (b.heads - 1) * b.head_stride + dim))
    return false;
  if (a.heads > 1 && a.head_stride == b.head_stride && b.heads > 1 &&
      apart(a.head_stride, (an - 1) * a.token_stride + dim, (bn - 1) * b.token_stride + dim))
    return false;
  // Heads start at multiples of what divides all strides.
  int64_t step = 0;
  const auto meet = [&](int64_t stride, int64_t n) {
    if (n > 1) step = std::gcd(step, stride);
  };
  meet(a.token_stride, an);
  meet(b.token_stride, bn);
  meet(a.head_stride, a.heads);
  meet(b.head_stride, b.heads);
  return !apart(step, dim, dim);
}
inline bool heads_overlap(const moeca_heads& a, int64_t an, const Range& r, int dim, int64_t es) {
  return overlap(heads_range(a, an, dim, es), r);
}

}  // namespace moeca
