// What the calls without a handle share: checks of their arguments on the host, and the launch's outcome.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "kernels.h"
#include "moeca.h"

namespace moeca {

constexpr int64_t kMaxRows = 0x7fffffff;
constexpr int kMaxWidth = 1 << 20, kMaxSlots = 16;

inline bool is_dtype(int d) { return d == MOECA_F32 || d == MOECA_BF16; }
inline int64_t elem_size(int d) { return d == MOECA_BF16 ? 2 : 4; }
inline uintptr_t addr(const void* p) { return reinterpret_cast<uintptr_t>(p); }

// A buffer's bytes: [from, from + bytes).
struct Range {
  const void* from;
  int64_t bytes;
};
inline Range rows_range(const void* p, int64_t rows, int64_t stride, int64_t row_bytes) {
  return {p, rows > 0 ? (rows - 1) * stride + row_bytes : 0};
}
inline bool overlap(const Range& a, const Range& b) {
  return a.from && b.from && a.bytes > 0 && b.bytes > 0 && addr(a.from) < addr(b.from) + b.bytes &&
         addr(b.from) < addr(a.from) + a.bytes;
}
// What is wrong with rows of values (null: nothing); `what` where there is no buffer.
inline const char* bad_values(const void* p, int64_t rows, int64_t stride, int width, int dtype, const char* what) {
  if (rows > 0 && !p) return what;
  if (addr(p) % elem_size(dtype)) return "a value buffer is not aligned to its type";
  if (stride < width || (rows > 0 && stride > INT64_MAX / 8 / rows)) return "a value stride is smaller than the width, or out of range";
  return nullptr;
}
inline moeca_status refuse(const char* why) {
  keep_call_error(why);
  return MOECA_ERR_INVALID_ARG;
}
// Runs a launch; nothing is thrown to the caller.
template <typename F>
moeca_status launched(F launch) {
  try {
    const cudaError_t e = launch();
    if (e == cudaSuccess) return MOECA_OK;
    cudaGetLastError();
    keep_call_error(cudaGetErrorString(e));
    return MOECA_ERR_CUDA;
  } catch (...) {
    keep_call_error("out of host memory");
    return MOECA_ERR_OOM;
  }
}
// Whether any buffer of `written` overlaps one of `read` or another one written.
template <int NW, int NR>
bool any_overlap(const Range (&written)[NW], const Range (&read)[NR]) {
  for (int i = 0; i < NW; ++i) {
    for (const Range& r : read)
      if (overlap(written[i], r)) return true;
    for (int j = 0; j < i; ++j)
      if (overlap(written[i], written[j])) return true;
  }
  return false;
}

}  // namespace moeca
