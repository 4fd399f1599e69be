// Rows of an embedding, and their gradient.
#pragma once
#include "element.h"

namespace bpe {

__device__ inline int64_t rows_in_use(int64_t n, const int64_t* count) {
  return count ? min(n, max(*count, (int64_t)0)) : n;
}

// One workgroup a row.
template <typename T>
__global__ void __launch_bounds__(256) embed_kernel(const T* weight, int64_t vocab, int64_t dim, int64_t weight_stride,
                                                    const int32_t* ids, int64_t n, const int64_t* count, float scale, T* out,
                                                    int64_t out_stride) {
  const int64_t t = blockIdx.x;
  if (t >= rows_in_use(n, count)) return;
  const int32_t id = ids[t];
  const bool kept = id >= 0 && id < vocab;
  const T* from = weight + (kept ? id : 0) * weight_stride;
  T* to = out + t * out_stride;
  for (int64_t c = threadIdx.x; c < dim; c += 256) to[c] = from_float<T>(kept ? scale * to_float(from[c]) : 0.0f);
}

// One workgroup a row of the vocabulary: it looks through the ids and adds the rows that name it, in order.
template <typename T, typename O>
__global__ void __launch_bounds__(256) embed_grad_kernel(const T* grad, int64_t grad_stride, const int32_t* ids, int64_t n,
                                                         const int64_t* count, int64_t dim, float scale, int accumulate,
                                                         O* out, int64_t out_stride) {
  __shared__ int32_t found[256];
  const int64_t rows = rows_in_use(n, count);
  const int32_t v = (int32_t)blockIdx.x;
  O* to = out + (int64_t)v * out_stride;
  for (int64_t c0 = 0; c0 < dim; c0 += 256) {
    const int64_t c = c0 + threadIdx.x;
    float sum = 0.0f;
    bool any = false;
    for (int64_t t0 = 0; t0 < rows; t0 += 256) {
      const int64_t t = t0 + threadIdx.x;
      __syncthreads();
      found[threadIdx.x] = t < rows && ids[t] == v;
      __syncthreads();
      for (int i = 0; i < 256; ++i)
        if (found[i]) {
          any = true;
          if (c < dim) sum += to_float(grad[(t0 + i) * grad_stride + c]);
        }
    }
    if (c < dim && (any || !accumulate))
      to[c] = from_float<O>(any ? (accumulate ? to_float(to[c]) : 0.0f) + scale * sum : 0.0f);
  }
}

}  // namespace bpe
