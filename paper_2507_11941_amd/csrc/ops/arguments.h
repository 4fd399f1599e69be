// What the host sides of the operators share: checks of arguments, types, parts of a workspace.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cstddef>

#include "../../../include/bpe_ops.h"
#include "element.h"

namespace bpe {

inline int launched() { return hipGetLastError() == hipSuccess ? BPE_OK : BPE_EHIP; }

inline size_t size_of(int dtype) { return dtype == BPE_F32 ? 4 : 2; }

inline bool is_type(int dtype) { return dtype == BPE_F32 || dtype == BPE_BF16 || dtype == BPE_F16; }

// Whether p may be used for n values of `size` bytes.
inline bool fits(const void* p, int64_t n, size_t size) { return (n == 0 || p) && ((uintptr_t)p & (size - 1)) == 0; }

// ... and, if there is one, an optional array.
inline bool aligned(const void* p, size_t size) { return ((uintptr_t)p & (size - 1)) == 0; }

inline bool is_matrix(const void* p, int dtype, int64_t rows, int64_t columns, int64_t stride) {
  return is_type(dtype) && columns >= 1 && columns <= BPE_MAX_COLUMNS && stride >= columns && stride < ((int64_t)1 << 40) &&
         fits(p, rows, size_of(dtype));
}

inline bool is_count(int64_t n) { return n >= 0 && n <= BPE_MAX_TOKENS; }

inline bool is_workspace(const void* p, size_t bytes, size_t need) { return p && ((uintptr_t)p & 255) == 0 && bytes >= need && need > 0; }

inline unsigned blocks(int64_t n, int64_t each) { return (unsigned)((n + each - 1) / each); }

// Calls f with a value of the type.
template <typename F>
inline void with_type(int dtype, F&& f) {
  if (dtype == BPE_F32) f(float{});
  else if (dtype == BPE_BF16) f(bf16{});
  else f(f16{});
}

inline size_t place(size_t& total, size_t bytes) {
  const size_t at = total;
  total += (bytes + 255) & ~(size_t)255;
  return at;
}

}  // namespace bpe
