// Host side of the adjustment of logits (include/bpe_head.h): argument checks and the enqueue.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../../include/bpe_head.h"
#include "../ops/arguments.h"
#include "adjust_kernels.h"

using namespace bpe;

namespace {

// Threads a stretch, sixteen columns each, by the mean of the histories: the more of them, the fewer stretches look through a history, and
// the later a workgroup's logits follow.  509 rows of 100,260 bfloat16 with 256, 512, 1,024 threads: histories of 100 tokens 33.7, 33.6,
// 36.5 us, of 1,000 37.1, 36.9, 40.3, of 4,000 (and masks) 46.7, 44.6, 46.1, of 16,000 72.6, 67.9, 64.6; 2,011 of 32,256 with 250 43.6,
// 44.6, 47.1; 32 of 100,260 with 10 5.2, 5.4, 5.7, with 1,000 7.2, 7.2, 7.5, with 16,000 10.3, 8.8, 7.9.  (Where the ids are a buffer that is
// not full, or histories share them, the mean is another, and the choice may be: results are the same.)
constexpr int64_t kLong = 2000, kLonger = 8000;

template <typename T, bool kGrad>
void launch_adjust(const T* in, const T* logits, T* out, AdjustArgs a, int64_t n, hipStream_t stream) {
  const bool in_place = in == out;
  const auto launch = [&](auto kernel, int threads) {
    const int64_t columns = (int64_t)threads * kAdjustEach;
    a.stretches = (unsigned)((a.vocab + columns - 1) / columns);
    const size_t shared = columns * (a.bias_begin ? 8 : a.begin ? 4 : 0);
    const int64_t rows = std::max<int64_t>(1, ((int64_t)1 << 21) / a.stretches);
    for (a.first = 0; a.first < n; a.first += rows)
      hipLaunchKernelGGL(kernel, dim3((unsigned)(std::min(rows, n - a.first) * a.stretches)), dim3(threads), shared, stream, in, logits, out, a);
  };
  const auto with_threads = [&](auto threads) {
    if (in_place) launch(adjust_kernel<T, kGrad, true, threads.value>, threads.value);
    else launch(adjust_kernel<T, kGrad, false, threads.value>, threads.value);
  };
  const int64_t history = a.begin ? a.n_ids / n : 0;
  if (history >= kLonger) with_threads(std::integral_constant<int, 1024>{});
  else if (history >= kLong) with_threads(std::integral_constant<int, 512>{});
  else with_threads(std::integral_constant<int, 256>{});
}

// A list's bounds: both or none, of an array that there is where it has elements.
bool is_list(const void* values, int64_t n, const int64_t* begin, const int64_t* end) {
  return !begin == !end && aligned(begin, 8) && aligned(end, 8) && n >= 0 && (!begin || (n < ((int64_t)1 << 40) && fits(values, n, 4)));
}

// (A null `state` beside masks: one for all, or one each.)
bool is_mask(const int32_t* mask, int64_t states, int64_t stride, const int32_t* state, int64_t n, int64_t vocab) {
  if (!mask) return true;
  return aligned(mask, 4) && states >= 1 && states <= BPE_MAX_TOKENS && stride >= (vocab + 31) / 32 && stride < ((int64_t)1 << 40) && aligned(state, 4) &&
         (state || states == 1 || states == n);
}

// Penalties and masks, which the gradient has too.
AdjustArgs adjust_args(int64_t vocab, int64_t stride, const int32_t* ids, int64_t n_ids, const int64_t* begin, const int64_t* end,
                       const float* penalties, float repetition, const int32_t* mask, int64_t states, int64_t mask_stride,
                       const int32_t* state, int64_t out_stride) {
  AdjustArgs a{};
  a.ids = ids;
  a.n_ids = n_ids;
  a.begin = begin;
  a.end = end;
  a.penalties = penalties;
  a.repetition = repetition;
  a.mask = (const uint8_t*)mask;
  a.states = states;
  a.mask_stride = mask_stride;
  a.state = state;
  a.stride = stride;
  a.out_stride = out_stride;
  a.vocab = vocab;
  return a;
}

// (Logits are multiplied by its reciprocal, which has to be an ordinary number too.)
bool is_repetition(float r) { return r >= 0x1p-126f && r <= 0x1p126f; }

}  // namespace

extern "C" {

int bpe_adjust_logits(const void* logits, int dtype, int64_t n, int64_t vocab, int64_t stride, const int32_t* ids, int64_t n_ids,
                      const int64_t* begin, const int64_t* end, const float* penalties, float repetition, float presence,
                      float frequency, const int32_t* bias_ids, const float* bias_values, int64_t n_biases,
                      const int64_t* bias_begin, const int64_t* bias_end, const int32_t* mask, int64_t states, int64_t mask_stride,
                      const int32_t* state, void* out, int64_t out_stride, void* stream) {
  if (!is_count(n) || !is_matrix(logits, dtype, n, vocab, stride) || !is_matrix(out, dtype, n, vocab, out_stride) ||
      (out == logits && n > 1 && out_stride != stride) || !is_list(ids, n_ids, begin, end) || !aligned(penalties, 4) ||
      !is_repetition(repetition) || !std::isfinite(presence) || !std::isfinite(frequency) ||
      !is_list(bias_ids, n_biases, bias_begin, bias_end) || !is_list(bias_values, n_biases, bias_begin, bias_end) ||
      !is_mask(mask, states, mask_stride, state, n, vocab))
    return BPE_EINVAL;
  if (n == 0) return BPE_OK;
  AdjustArgs a = adjust_args(vocab, stride, ids, n_ids, begin, end, penalties, repetition, mask, states, mask_stride, state, out_stride);
  a.presence = presence;
  a.frequency = frequency;
  a.bias_ids = bias_ids;
  a.bias_values = bias_values;
  a.n_biases = n_biases;
  a.bias_begin = bias_begin;
  a.bias_end = bias_end;
  with_type(dtype, [&](auto type) {
    using T = decltype(type);
    launch_adjust<T, false>((const T*)logits, nullptr, (T*)out, a, n, (hipStream_t)stream);
  });
  return launched();
}

int bpe_adjust_logits_grad(const void* grad, int dtype, int64_t n, int64_t vocab, int64_t grad_stride, const void* logits,
                           int64_t stride, const int32_t* ids, int64_t n_ids, const int64_t* begin, const int64_t* end,
                           const float* penalties, float repetition, const int32_t* mask, int64_t states, int64_t mask_stride,
                           const int32_t* state, void* out, int64_t out_stride, void* stream) {
  if (!is_count(n) || !is_matrix(grad, dtype, n, vocab, grad_stride) || !is_matrix(logits, dtype, n, vocab, stride) ||
      !is_matrix(out, dtype, n, vocab, out_stride) || (out == grad && n > 1 && out_stride != grad_stride) ||
      !is_list(ids, n_ids, begin, end) || !aligned(penalties, 4) || !is_repetition(repetition) ||
      !is_mask(mask, states, mask_stride, state, n, vocab))
    return BPE_EINVAL;
  if (n == 0) return BPE_OK;
  AdjustArgs a =
      adjust_args(vocab, grad_stride, ids, n_ids, begin, end, penalties, repetition, mask, states, mask_stride, state, out_stride);
  a.logits_stride = stride;
  with_type(dtype, [&](auto type) {
    using T = decltype(type);
    launch_adjust<T, true>((const T*)grad, (const T*)logits, (T*)out, a, n, (hipStream_t)stream);
  });
  return launched();
}

}  // extern "C"
