// Host side of the 8-bit product (include/bpe_head.h): argument checks and the enqueue.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../../include/bpe_head.h"
#include "../ops/arguments.h"
#include "project_kernels.h"

using namespace bpe;

namespace {

template <typename T, int kMt, int kVt, int kWm, int kWv, int kStages>
void launch_tiles(ProjectArgs a, bool direct, T* out, hipStream_t stream) {
  constexpr int kTokens = 32 * kMt * kWm, kWords = 32 * kVt * kWv;
  a.token_tiles = blocks(a.n, kTokens);
  a.tiles = a.token_tiles * blocks(a.vocab, kWords);
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(a.tiles), dim3(64 * kWm * kWv), 0, stream, a, out);
  };
  if (direct) launch(project_kernel<T, kMt, kVt, kWm, kWv, kStages, true>);
  else launch(project_kernel<T, kMt, kVt, kWm, kWv, 2, false>);
}

template <typename T>
void launch_project(const ProjectArgs& a, T* out, hipStream_t stream) {
  const auto in_sixteens = [](const void* p, int64_t stride) { return (((uintptr_t)p | (uintptr_t)stride) & 15) == 0; };
  const bool direct = in_sixteens(a.q, a.q_stride) && in_sixteens(a.weight, a.weight_stride);
  if (a.n <= 32) launch_tiles<T, 1, 1, 1, 4, 4>(a, direct, out, stream);
  else if (a.n <= 64) launch_tiles<T, 2, 1, 1, 4, 3>(a, direct, out, stream);
  else if (a.n <= 128) launch_tiles<T, 2, 2, 2, 2, 2>(a, direct, out, stream);
  else launch_tiles<T, 4, 2, 2, 4, 2>(a, direct, out, stream);
}

bool is_bytes(const void* p, int64_t rows, int64_t columns, int64_t stride) {
  return stride >= columns && stride < ((int64_t)1 << 40) && fits(p, rows, 1);
}

}  // namespace

extern "C" {

int bpe_project_8bit(const int8_t* q, int64_t n, int64_t dim, int64_t q_stride, const float* scales, const int8_t* weight,
                     int64_t vocab, int64_t weight_stride, const float* weight_scales, void* out, int dtype, int64_t out_stride,
                     void* stream) {
  if (!is_count(n) || dim < 1 || dim > BPE_MAX_DIM_8BIT || !is_bytes(q, n, dim, q_stride) || !fits(scales, n, 4) || vocab < 1 ||
      vocab > BPE_MAX_COLUMNS || !is_bytes(weight, vocab, dim, weight_stride) || !fits(weight_scales, vocab, 4) ||
      !is_matrix(out, dtype, n, vocab, out_stride) || (double)n * (double)vocab > 1e13)
    return BPE_EINVAL;
  if (n == 0) return BPE_OK;
  ProjectArgs a{};
  a.q = q;
  a.scales = scales;
  a.weight = weight;
  a.weight_scales = weight_scales;
  a.n = n;
  a.vocab = vocab;
  a.q_stride = q_stride;
  a.weight_stride = weight_stride;
  a.out_stride = out_stride;
  a.dim = (int)dim;
  with_type(dtype, [&](auto type) {
    using T = decltype(type);
    launch_project(a, (T*)out, (hipStream_t)stream);
  });
  return launched();
}

}  // extern "C"
