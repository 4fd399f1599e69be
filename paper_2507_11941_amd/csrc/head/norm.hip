// Host side of the norms and of rows in 8 bits (include/bpe_head.h): argument checks and the enqueue.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../../include/bpe_head.h"
#include "../ops/arguments.h"
#include "norm_kernels.h"

using namespace bpe;

namespace {

constexpr int64_t kMostRows = (int64_t)1 << 21;             // workgroups of a launch
constexpr int64_t kGradRows = 256;                          // rows that are summed in 32 bits, at most

// Fewer rows than these have more threads, each with one vector.  One wave a row, and four, us (8 bits, the type, rows to 8 bits; in a graph):
// 61 rows of 2,048 bfloat16 5.3, 4.1, 3.9 and 3.7, 3.1, 3.1; 500 6.3, 4.6, 4.3 and 4.4, 3.6, 3.5; 1,000 6.6, 5.2, 4.3 and 5.6, 4.5, 4.4; 2,000
// 8.2, 7.0, 5.7 and 8.0, 6.6, 6.1; 4,000 13.3, 12.0, 8.4 and 14.7, 13.1, 9.6; of 700 columns 500 5.1, 4.0, 3.6 and 4.2, 3.4, 3.4, 2,000 6.2,
// 5.1, 4.4 and 6.5, 5.0, 5.1.
constexpr int64_t kFewRows = 1000;

// Calls f with the threads and vectors a lane of the smallest variant whose registers hold a row, or returns false.
template <typename T, typename F>
bool with_variant(int64_t n, int64_t dim, F&& f) {
  const int64_t vecs = dim / Vec<T>::kWidth;
  if (vecs <= 64) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
  else if (vecs <= 256 && n < kFewRows) f(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
  else if (vecs <= 64 * 4) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 4>{});
  else if (vecs <= 256 * 2) f(std::integral_constant<int, 256>{}, std::integral_constant<int, 2>{});
  else if (vecs <= 256 * 4) f(std::integral_constant<int, 256>{}, std::integral_constant<int, 4>{});
  else if (vecs <= 1024 * 2) f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
  else return false;
  return true;
}

// Calls f with a value of the type and one of the weights' type.
template <typename F>
void with_types(int dtype, int weight_dtype, F&& f) {
  with_type(dtype, [&](auto type) {
    if (weight_dtype == BPE_F32) f(type, float{});
    else if constexpr (!__is_same(decltype(type), float)) f(type, type);
  });
}

template <int kKind, typename T, typename W>
void launch_norm(NormArgs<T, W> a, int64_t n, hipStream_t stream) {
  for (a.first = 0; a.first < n; a.first += kMostRows) {
    const dim3 grid((unsigned)std::min(kMostRows, n - a.first));
    const bool held = with_variant<T>(n, a.dim, [&](auto threads, auto vecs) {
      hipLaunchKernelGGL((norm_kernel<T, W, kKind, threads.value, vecs.value>), grid, dim3(threads.value), 0, stream, a);
    });
    if (!held) hipLaunchKernelGGL((long_norm_kernel<T, W, kKind>), grid, dim3(1024), 0, stream, a);
  }
}

int64_t rows_of_group(int64_t n) {
  const int64_t groups = n >= 4096 ? 1024 : 512;
  return std::min(kGradRows, std::max<int64_t>(1, (n + groups - 1) / groups));
}

// The same for the gradient, whose threads hold more besides: one vector a lane where there are threads enough.
template <typename T, typename F>
bool with_grad_variant(int64_t dim, F&& f) {
  const int64_t vecs = dim / Vec<T>::kWidth;
  if (vecs <= 64) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
  else if (vecs <= 128) f(std::integral_constant<int, 128>{}, std::integral_constant<int, 1>{});
  else if (vecs <= 256) f(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
  else if (vecs <= 512) f(std::integral_constant<int, 512>{}, std::integral_constant<int, 1>{});
  else if (vecs <= 1024) f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 1>{});
  else return false;
  return true;
}

// Whether what is written at p begins where q does without lying as q does: its rows would lie over other rows of q.
bool crosses(const void* p, int64_t stride, const void* q, int64_t q_stride, int64_t n) { return p == q && n > 1 && stride != q_stride; }

// Arguments that the two forms of the norm share.
bool is_norm(const void* x, int dtype, int64_t n, int64_t dim, int64_t stride, const void* residual, int64_t residual_stride,
             const void* weight, int weight_dtype, float eps, const void* summed, int64_t summed_stride) {
  return is_count(n) && is_matrix(x, dtype, n, dim, stride) && (weight_dtype == BPE_F32 || weight_dtype == dtype) &&
         fits(weight, dim, size_of(weight_dtype)) && eps >= 0.0f && std::isfinite(eps) && !residual == !summed &&
         (!residual || (is_matrix(residual, dtype, n, dim, residual_stride) && is_matrix(summed, dtype, n, dim, summed_stride) &&
                        !crosses(summed, summed_stride, x, stride, n) && !crosses(summed, summed_stride, residual, residual_stride, n)));
}

template <typename T, typename W>
NormArgs<T, W> norm_args(const void* x, int64_t dim, int64_t stride, const void* residual, int64_t residual_stride, const void* weight,
                         float eps, void* summed, int64_t summed_stride) {
  NormArgs<T, W> a{};
  a.x = (const T*)x;
  a.residual = (const T*)residual;
  a.weight = (const W*)weight;
  a.summed = (T*)summed;
  a.stride = stride;
  a.residual_stride = residual_stride;
  a.summed_stride = summed_stride;
  a.dim = (int)dim;
  a.eps = eps;
  return a;
}

bool is_bytes(const void* p, int64_t rows, int64_t columns, int64_t stride) {
  return stride >= columns && stride < ((int64_t)1 << 40) && fits(p, rows, 1);
}

}  // namespace

extern "C" {

int bpe_add_norm(const void* x, int dtype, int64_t n, int64_t dim, int64_t stride, const void* residual, int64_t residual_stride,
                 const void* weight, int weight_dtype, float eps, void* summed, int64_t summed_stride, float* rstd, void* out,
                 int64_t out_stride, void* stream) {
  if (!is_norm(x, dtype, n, dim, stride, residual, residual_stride, weight, weight_dtype, eps, summed, summed_stride) ||
      !aligned(rstd, 4) || !is_matrix(out, dtype, n, dim, out_stride) || (summed && out == summed && n > 0) ||
      crosses(out, out_stride, x, stride, n) || (residual && crosses(out, out_stride, residual, residual_stride, n)))
    return BPE_EINVAL;
  with_types(dtype, weight_dtype, [&](auto type, auto weight_type) {
    using T = decltype(type);
    using W = decltype(weight_type);
    auto a = norm_args<T, W>(x, dim, stride, residual, residual_stride, weight, eps, summed, summed_stride);
    a.rstd = rstd;
    a.out = (T*)out;
    a.out_stride = out_stride;
    launch_norm<kNorm>(a, n, (hipStream_t)stream);
  });
  return launched();
}

int bpe_add_norm_8bit(const void* x, int dtype, int64_t n, int64_t dim, int64_t stride, const void* residual, int64_t residual_stride,
                      const void* weight, int weight_dtype, float eps, void* summed, int64_t summed_stride, int8_t* q,
                      int64_t q_stride, float* scales, void* stream) {
  if (!is_norm(x, dtype, n, dim, stride, residual, residual_stride, weight, weight_dtype, eps, summed, summed_stride) ||
      !is_bytes(q, n, dim, q_stride) || !fits(scales, n, 4))
    return BPE_EINVAL;
  with_types(dtype, weight_dtype, [&](auto type, auto weight_type) {
    using T = decltype(type);
    using W = decltype(weight_type);
    auto a = norm_args<T, W>(x, dim, stride, residual, residual_stride, weight, eps, summed, summed_stride);
    a.q = q;
    a.q_stride = q_stride;
    a.scales = scales;
    launch_norm<kNorm8>(a, n, (hipStream_t)stream);
  });
  return launched();
}

int bpe_quantize_rows(const void* x, int dtype, int64_t n, int64_t dim, int64_t stride, int8_t* q, int64_t q_stride, float* scales,
                      void* stream) {
  if (!is_count(n) || !is_matrix(x, dtype, n, dim, stride) || !is_bytes(q, n, dim, q_stride) || !fits(scales, n, 4)) return BPE_EINVAL;
  with_type(dtype, [&](auto type) {
    using T = decltype(type);
    auto a = norm_args<T, T>(x, dim, stride, nullptr, 0, nullptr, 0.0f, nullptr, 0);
    a.q = q;
    a.q_stride = q_stride;
    a.scales = scales;
    launch_norm<kRows8>(a, n, (hipStream_t)stream);
  });
  return launched();
}

size_t bpe_add_norm_grad_workspace_bytes(int64_t n, int64_t dim) {
  if (!is_count(n) || dim < 1 || dim > BPE_MAX_COLUMNS) return 0;
  const int64_t each = rows_of_group(n), groups = (n + each - 1) / each;
  size_t total = 0;
  place(total, (size_t)std::max<int64_t>(1, groups) * dim * 4);
  return total;
}

int bpe_add_norm_grad(const void* grad, int dtype, int64_t n, int64_t dim, int64_t grad_stride, const void* summed,
                      int64_t summed_stride, const void* weight, int weight_dtype, const float* rstd, const void* grad_summed,
                      int64_t grad_summed_stride, void* grad_x, int64_t grad_x_stride, void* grad_weight, int grad_weight_dtype,
                      int accumulate, void* workspace, size_t workspace_bytes, void* stream_ptr) {
  if (!is_count(n) || !is_matrix(grad, dtype, n, dim, grad_stride) || !is_matrix(summed, dtype, n, dim, summed_stride) ||
      (weight_dtype != BPE_F32 && weight_dtype != dtype) || !fits(weight, dim, size_of(weight_dtype)) || !fits(rstd, n, 4) ||
      (grad_summed && !is_matrix(grad_summed, dtype, n, dim, grad_summed_stride)) || !is_matrix(grad_x, dtype, n, dim, grad_x_stride) ||
      crosses(grad_x, grad_x_stride, grad, grad_stride, n) || (grad_summed && crosses(grad_x, grad_x_stride, grad_summed, grad_summed_stride, n)))
    return BPE_EINVAL;
  if (grad_weight && ((grad_weight_dtype != BPE_F32 && grad_weight_dtype != weight_dtype) || !aligned(grad_weight, size_of(grad_weight_dtype)) ||
                      !is_workspace(workspace, workspace_bytes, bpe_add_norm_grad_workspace_bytes(n, dim))))
    return BPE_EINVAL;
  const hipStream_t stream = (hipStream_t)stream_ptr;
  const int64_t each = rows_of_group(n), groups = (n + each - 1) / each;
  with_types(dtype, weight_dtype, [&](auto type, auto weight_type) {
    using T = decltype(type);
    using W = decltype(weight_type);
    NormGradArgs<T, W> a{};
    a.grad = (const T*)grad;
    a.summed = (const T*)summed;
    a.weight = (const W*)weight;
    a.rstd = rstd;
    a.grad_summed = (const T*)grad_summed;
    a.grad_x = (T*)grad_x;
    a.partial = grad_weight ? (float*)workspace : nullptr;
    a.grad_stride = grad_stride;
    a.summed_stride = summed_stride;
    a.grad_summed_stride = grad_summed_stride;
    a.grad_x_stride = grad_x_stride;
    a.n = n;
    a.dim = (int)dim;
    a.each = (int)each;
    if (n > 0) {
      const bool held = with_grad_variant<T>(dim, [&](auto threads, auto vecs) {
        hipLaunchKernelGGL((norm_grad_kernel<T, W, threads.value, vecs.value>), dim3((unsigned)groups), dim3(threads.value), 0, stream, a);
      });
      if (!held) {
        constexpr int64_t kMostGroups = 32768;
        if (a.partial)
          for (int64_t first = 0; first < groups; first += kMostGroups)
            hipLaunchKernelGGL((long_norm_partial_kernel<T, W>), dim3(blocks(dim, 256), (unsigned)std::min(kMostGroups, groups - first)),
                               dim3(256), 0, stream, a, first);
        for (int64_t first = 0; first < n; first += kMostRows)
          hipLaunchKernelGGL((long_norm_grad_kernel<T, W>), dim3((unsigned)std::min(kMostRows, n - first)), dim3(1024), 0, stream, a, first);
      }
    }
    if (grad_weight) {
      const auto join = [&](auto out_type) {
        using O = decltype(out_type);
        const unsigned columns = blocks(dim, 64);
        for (unsigned first = 0; first < columns; first += (unsigned)kMostRows)
          hipLaunchKernelGGL(norm_weight_kernel<O>, dim3(std::min((unsigned)kMostRows, columns - first)), dim3(1024), 0, stream, a.partial, groups,
                             (int)dim, accumulate, first, (O*)grad_weight);
      };
      if (grad_weight_dtype == BPE_F32) join(float{});
      else join(type);
    }
  });
  return launched();
}

}  // extern "C"
