// Log-probabilities of tokens from logits, their gradient, and two losses made of them.
#pragma once
#include "element.h"

namespace bpe {

// The softmax statistics of some of a row's logits: their maximum and the sum of exp(x - maximum).
struct Stats {
  float m, s;
};

// What exponentials are taken against: the maximum, or 0 where there is nothing but -inf, whose exponentials are then 0.
__device__ inline float reference_of(float m) { return m == -INFINITY ? 0.0f : m; }

// exp(x - r).  The difference first: a multiple of the type's lowest value would be -inf, and -inf minus itself NaN.
__device__ inline float exp_of(float x, float r) { return __builtin_amdgcn_exp2f((x - r) * kLog2e); }

__device__ inline Stats join(Stats a, Stats b) {
  const float m = fmaxf(a.m, b.m), r = reference_of(m);
  return {m, a.s * exp_of(a.m, r) + b.s * exp_of(b.m, r)};
}

template <int kThreads>
__device__ inline Stats join_workgroup(Stats mine) {
  __shared__ Stats part[kThreads / 64];
  for (int d = 32; d >= 1; d >>= 1) mine = join(mine, {__shfl_xor(mine.m, d), __shfl_xor(mine.s, d)});
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = mine;
  __syncthreads();
  Stats all = part[0];
  for (int w = 1; w < kThreads / 64; ++w) all = join(all, part[w]);
  return all;
}

// The logarithm of a token's probability, in 64 bits: x - m is exact or nearly so, and the logarithm's rounding to 32 bits
// (5e-7 at 10) would be the largest error of a loss that adds up thousands of them.
__device__ inline double logprob_of(float x, Stats all) { return (double)(x - all.m) - log((double)all.s); }

enum RowKind { kRowLogprob, kRowStep, kRowPolicy };

struct RowArgs {
  const int32_t* targets;
  float* logprobs;            // null: not wanted
  float* lse;                 // null: not wanted
  double* logprobs64;         // null: not wanted
  const float* upstream;      // kRowStep
  int64_t grad_stride;
  // kRowPolicy
  const float* weight;        // of each row's loss; 0: not in a string
  const float* advantage;     // of each row
  const float* old;
  const float* reference;
  float low, high, kl_weight, scale;
  double* value;              // of each row: its share of the loss
};

// The loss of one token under the clipped policy, and its derivative with respect to the token's log-probability.
__device__ inline float policy_value(const RowArgs& a, int64_t t, double lp, float* slope) {
  const float advantage = a.advantage[t];
  const float ratio = expf((float)(lp - (double)a.old[t]));
  const float free = ratio * advantage, clipped = fminf(fmaxf(ratio, 1.0f - a.low), 1.0f + a.high) * advantage;
  float value = -fminf(free, clipped);
  *slope = free <= clipped ? -free : 0.0f;
  if (a.reference) {
    const float d = (float)((double)a.reference[t] - lp);
    value += a.kl_weight * (expm1f(d) - d);
    *slope -= a.kl_weight * expm1f(d);
  }
  return value;
}

// One workgroup a row: statistics, then what the row is for.
template <typename T, int kKind>
__global__ void __launch_bounds__(256) row_kernel(const T* logits, int64_t vocab, int64_t stride, RowArgs a, T* grad) {
  const int64_t t = blockIdx.x;
  const T* x = logits + t * stride;
  T* g = grad + t * a.grad_stride;
  const int32_t target = a.targets[t];
  const float weight = kKind == kRowPolicy ? a.weight[t] : 1.0f;
  const bool scored = target >= 0 && target < vocab && weight != 0.0f;
  if (!scored) {
    if (threadIdx.x == 0) {
      if (a.logprobs) a.logprobs[t] = 0.0f;
      if (a.lse) a.lse[t] = 0.0f;
      if (a.logprobs64) a.logprobs64[t] = 0.0;
      if (kKind == kRowPolicy) a.value[t] = 0.0;
    }
    if (kKind != kRowLogprob)
      for (int64_t j = threadIdx.x; j < vocab; j += 256) g[j] = from_float<T>(0.0f);
    return;
  }
  Stats mine = {-INFINITY, 0.0f};
  for (int64_t j = threadIdx.x; j < vocab; j += 256) mine = join(mine, {to_float(x[j]), 1.0f});
  const float at_target = to_float(x[target]);
  const Stats all = join_workgroup<256>(mine);
  const double lp = logprob_of(at_target, all);
  if (threadIdx.x == 0) {
    if (a.logprobs) a.logprobs[t] = (float)lp;
    if (a.lse) a.lse[t] = (float)((double)all.m + log((double)all.s));
    if (a.logprobs64) a.logprobs64[t] = lp;
  }
  if (kKind == kRowLogprob) return;
  float c = 0.0f;
  if (kKind == kRowStep) c = a.upstream[t];
  if (kKind == kRowPolicy) {
    float slope;
    const float value = policy_value(a, t, lp, &slope);
    if (threadIdx.x == 0) a.value[t] = (double)weight * value;
    c = a.scale * weight * slope;
  }
  if (c == 0.0f) {
    for (int64_t j = threadIdx.x; j < vocab; j += 256) g[j] = from_float<T>(0.0f);
    return;
  }
  const float share = -c / all.s;
  for (int64_t j = threadIdx.x; j < vocab; j += 256)
    g[j] = from_float<T>(j == target ? -c * expm1f((float)lp) : share * exp_of(to_float(x[j]), all.m));
}

template <typename T>
__global__ void __launch_bounds__(256) logprobs_grad_kernel(const T* logits, int64_t vocab, int64_t stride,
                                                            const int32_t* targets, const float* lse, const float* upstream,
                                                            T* grad, int64_t grad_stride) {
  const int64_t t = blockIdx.x;
  const T* x = logits + t * stride;
  T* g = grad + t * grad_stride;
  const int32_t target = targets[t];
  const float c = target >= 0 && target < vocab ? upstream[t] : 0.0f, l = c != 0.0f ? lse[t] : 0.0f;
  for (int64_t j = threadIdx.x; j < vocab; j += 256) {
    float d = 0.0f;
    if (c != 0.0f) d = j == target ? -c * expm1f(to_float(x[j]) - l) : -c * exp_of(to_float(x[j]), l);
    g[j] = from_float<T>(d);
  }
}

// ---- over strings --------------------------------------------------------------------------------------------

// String i's rows, as far as there are any.
__device__ inline void string_rows(const int64_t* offsets, int32_t i, int64_t n, int64_t* begin, int64_t* end) {
  *begin = min(max(offsets[i], (int64_t)0), n);
  *end = max(*begin, min(offsets[i + 1], n));
}

__device__ inline int32_t string_of(const int64_t* offsets, int32_t batch, int64_t t) {
  int32_t lo = 0, hi = batch;                              // the last string that begins at or before t
  while (lo < hi) {
    const int32_t mid = (lo + hi) >> 1;
    if (offsets[mid + 1] <= t) lo = mid + 1; else hi = mid;
  }
  return lo < batch && offsets[lo] <= t ? lo : -1;
}

__global__ void __launch_bounds__(256) next_tokens_kernel(const int32_t* ids, int64_t n, const int64_t* offsets, int32_t batch,
                                                          const int32_t* first, int32_t* targets) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t >= n) return;
  const int32_t i = string_of(offsets, batch, t);
  const bool scored = i >= 0 && t + 1 < n && t + 1 < offsets[i + 1] && (!first || t + 1 - offsets[i] >= first[i]);
  targets[t] = scored ? ids[t + 1] : -1;
}

template <typename V>
__device__ inline V sum_workgroup(V mine) {                 // of 256 threads, in a fixed order
  __shared__ V part[256];
  __syncthreads();
  part[threadIdx.x] = mine;
  __syncthreads();
  for (int d = 128; d >= 1; d >>= 1) {
    if ((int)threadIdx.x < d) part[threadIdx.x] += part[threadIdx.x + d];
    __syncthreads();
  }
  return part[0];
}

__device__ inline bool is_scored(const int32_t* targets, int64_t t, int64_t vocab) {
  return targets[t] >= 0 && targets[t] < vocab;
}

// One workgroup a pair; `upstream` is zero before.
__global__ void __launch_bounds__(256) pair_kernel(const double* logprobs, const int32_t* targets, int64_t n, int64_t vocab,
                                                   const int64_t* offsets, int32_t batch, const float* reference, float beta,
                                                   float smoothing, float scale, float* margins, double* losses, float* upstream) {
  const int32_t k = blockIdx.x;
  double sums[2];
  for (int side = 0; side < 2; ++side) {
    int64_t b, e;
    string_rows(offsets, 2 * k + side, n, &b, &e);
    double sum = 0.0;
    for (int64_t t = b + threadIdx.x; t < e; t += 256)
      if (is_scored(targets, t, vocab)) sum += logprobs[t] - (reference ? (double)reference[t] : 0.0);
    sums[side] = sum_workgroup(sum);
  }
  const double z = (double)beta * (sums[0] - sums[1]);
  // -log sigmoid(z) = max(-z, 0) + log(1 + exp(-|z|))
  const double tail = log1p(exp(-fabs(z)));
  const double loss = (1.0 - (double)smoothing) * (fmax(-z, 0.0) + tail) + (double)smoothing * (fmax(z, 0.0) + tail);
  const double slope = (double)smoothing - 1.0 / (1.0 + exp(z));
  const float c = (float)((double)scale * (double)beta * slope / (batch / 2));
  if (threadIdx.x == 0) {
    losses[k] = loss / (batch / 2);
    if (margins) margins[k] = (float)z;
  }
  for (int side = 0; side < 2; ++side) {
    int64_t b, e;
    string_rows(offsets, 2 * k + side, n, &b, &e);
    for (int64_t t = b + threadIdx.x; t < e; t += 256) upstream[t] = side ? -c : c;
  }
}

__global__ void __launch_bounds__(256) sum_kernel(const double* values, int64_t n, float* sum) {
  double mine = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += 256) mine += values[i];
  mine = sum_workgroup(mine);
  if (threadIdx.x == 0) *sum = (float)mine;
}

__global__ void __launch_bounds__(256) zero_kernel(float* values, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) values[i] = 0.0f;
}

// One workgroup: how many positions of each string are scored, and of all together (in counts[batch]).
__global__ void __launch_bounds__(256) count_kernel(const int32_t* targets, int64_t n, int64_t vocab, const int64_t* offsets,
                                                    int32_t batch, int32_t* counts) {
  int32_t all = 0;
  for (int32_t i = 0; i < batch; ++i) {
    int64_t b, e;
    string_rows(offsets, i, n, &b, &e);
    int32_t mine = 0;
    for (int64_t t = b + threadIdx.x; t < e; t += 256) mine += is_scored(targets, t, vocab);
    mine = sum_workgroup(mine);
    if (threadIdx.x == 0) counts[i] = mine;
    all += mine;
  }
  if (threadIdx.x == 0) counts[batch] = all;
}

__global__ void __launch_bounds__(256) weights_kernel(const int32_t* targets, int64_t n, int64_t vocab, const int64_t* offsets,
                                                      int32_t batch, const int32_t* counts, int by_string,
                                                      const float* advantages, int advantage_by_string, float* weight,
                                                      float* advantage) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t >= n) return;
  const int32_t i = string_of(offsets, batch, t);
  float w = 0.0f, a = 0.0f;
  if (i >= 0 && is_scored(targets, t, vocab)) {
    w = by_string ? (float)(1.0 / ((double)batch * counts[i])) : (float)(1.0 / counts[batch]);
    a = advantages[advantage_by_string ? i : t];
  }
  weight[t] = w;
  advantage[t] = a;
}

}  // namespace bpe
