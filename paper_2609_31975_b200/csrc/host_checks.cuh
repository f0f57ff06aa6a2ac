// What the host side of the calls without a handle shares: checks of pointers, types and rows, and of outputs that lie over something
// else.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "sparse_ffn.h"

namespace sffn {
void note_cuda_error(cudaError_t e, const char* file, int line);  // api.cu

namespace host {

#define SFFN_CUDA(expr)                                  \
  do {                                                   \
    const cudaError_t e_ = (expr);                       \
    if (e_ != cudaSuccess) {                             \
      sffn::note_cuda_error(e_, SFFN_FILE, __LINE__);    \
      return SFFN_ERR_CUDA;                              \
    }                                                    \
  } while (0)

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }
inline size_t element(int dtype) { return dtype == SFFN_BF16 ? 2 : 4; }
inline bool storage_type(int dtype) { return dtype == SFFN_F32 || dtype == SFFN_BF16; }

inline int sm_count(int* n) {
  int dev = 0;
  SFFN_CUDA(cudaGetDevice(&dev));
  SFFN_CUDA(cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev));
  return SFFN_OK;
}

inline int check_rows(const void* p, int64_t ld, int64_t width, size_t esz) {
  if (ld < width) return SFFN_ERR_INVALID_ARG;
  return aligned(p, 16) && (ld * esz) % 16 == 0 && ld <= (1ll << 31) ? SFFN_OK : SFFN_ERR_UNSUPPORTED;
}

// A matrix's rows in memory, and whether any of them meets any row of another matrix's (what lies between rows does not count: two
// matrices may be columns of one).
struct Span {
  const void* p;
  int64_t rows, width, ld;  // bytes
};
inline bool meet(const Span& a, const Span& b) {
  if (!a.p || !b.p || a.rows <= 0 || b.rows <= 0 || a.width <= 0 || b.width <= 0) return false;
  const int64_t d = (int64_t)(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p));  // b's first byte, from a's
  if (d >= (a.rows - 1) * a.ld + a.width || -d >= (b.rows - 1) * b.ld + b.width) return false;
  if (a.ld == b.ld) {  // rows i of a and j of b meet where d - a.width < (i - j) ld < d + b.width
    const auto below = [](int64_t v, int64_t n) { return v >= 0 ? v / n : -((-v + n - 1) / n); };
    const int64_t least = below(d - a.width, a.ld) + 1, most = -below(-(d + b.width), a.ld) - 1;
    return (least > 1 - b.rows ? least : 1 - b.rows) <= (most < a.rows - 1 ? most : a.rows - 1);
  }
  for (int64_t i = 0, j = 0; i < a.rows && j < b.rows;) {
    if (i * a.ld + a.width <= d + j * b.ld) ++i;
    else if (d + j * b.ld + b.width <= i * a.ld) ++j;
    else return true;
  }
  return false;
}
// Whether an output of a call meets one of these inputs, or another output.
template <size_t kIn, size_t kOut>
bool outputs_meet(const Span (&in)[kIn], const Span (&out)[kOut]) {
  for (size_t o = 0; o < kOut; ++o) {
    for (const Span& i : in)
      if (meet(out[o], i)) return true;
    for (size_t q = o + 1; q < kOut; ++q)
      if (meet(out[o], out[q])) return true;
  }
  return false;
}
inline Span whole(const void* p, int64_t bytes) { return {p, 1, bytes, bytes}; }

}  // namespace host
}  // namespace sffn
