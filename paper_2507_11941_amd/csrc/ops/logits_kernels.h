// Log-probabilities of tokens from logits, their gradient, and two losses made of them.
//
// All of it is bound by reading logits and writing gradients, so that what matters is how often a row passes: once for
// log-probabilities (a running maximum and sum), once in and once out for a gradient whose factor is known from the row itself (the
// row stays in registers between the two), and once more in where the factor needs other rows.  Measured on one MI355X, whose
// memory reads 6.2 to 6.3 TB/s, fills 6.9 to 7.3 and copies 5.0 (read and written):
//   log-probabilities of 8,191 rows of 100,260 bfloat16 (1.64 GB)            253 to 263 us from box to box, 6.2 to 6.5 TB/s
//   with the gradient, 8,209 rows of 32,256 bfloat16 (1.06 GB)               176 us, 6.0 TB/s
//   policy loss, 8,190 rows of 100,260 bfloat16 (2.86 GB)                    528 to 533 us, 5.4 TB/s
//   gradient from what was saved, 8,003 rows of 100,260 bfloat16 (2.78 GB)   507 to 519 us, 5.4 to 5.5 TB/s
// An exponential costs as much as four other instructions: of 16-bit logits the first of these keeps the vector units busy nine
// tenths of the time, and 32-bit ones, half as many a byte, come in at 6.3 TB/s.  Where a call moves more than the last-level
// cache holds, logits and gradients pass the caches by, which is how all but small calls come above the plain copy's rate; their
// stores write whole lines then.
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

// The same for term i of a sum.  log2 e lies between two 32-bit numbers, 1.34e-8 of itself above the one and 6.93e-8 below the
// other.  With the nearer one alone all terms would be too large, and log-probabilities 1e-7 too low on average, which strings add
// up; every sixth term takes the other, which makes up for it (a second product would cost 4 % of 8,191 x 100,260's 253 us).
__device__ inline float term_of(float x, float r, int i) {
  return __builtin_amdgcn_exp2f((x - r) * (i % 6 ? 1.44269502162933349609f : 1.44269514083862304688f));
}

// The same for a sum so far: log2 e in two parts.
__device__ inline float change_of(float m, float r) {
  const float d = m - r;
  return __builtin_amdgcn_exp2f(fmaf(d, kLog2e, d * 1.92596299112661746887e-8f));
}

// (Both sides the same whichever of them is whose: no product is fused with the addition.)
__device__ inline Stats join(Stats a, Stats b) {
#pragma clang fp contract(off)
  const float m = fmaxf(a.m, b.m), r = reference_of(m);
  return {m, a.s * change_of(a.m, r) + b.s * change_of(b.m, r)};
}

// Some more of a row's logits: one maximum and one change of reference for all of them.  Sums are in 32 bits: half of the terms are
// added to the sum so far, one after another.  That are 128 of them at most, and some ten steps join the lanes.
template <typename T, int kVecs>
__device__ inline void absorb(Stats& stats, const Vec<T>* v) {
  constexpr int kWidth = Vec<T>::kWidth;
  float m = stats.m;
#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
    float x[kWidth];
    v[k].get(x);
#pragma unroll
    for (int i = 0; i < kWidth; i += 2) m = max_of(m, x[i], x[i + 1]);
  }
  const float r = reference_of(m);
  float s0 = stats.s * change_of(stats.m, r), s1 = 0.0f;
#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
    float x[kWidth];
    v[k].get(x);
#pragma unroll
    for (int i = 0; i < kWidth; i += 2) {
      s0 += term_of(x[i], r, k * kWidth + i);
      s1 += term_of(x[i + 1], r, k * kWidth + i + 1);
    }
  }
  stats = {m, s0 + s1};
}

// The statistics of all threads' logits, in every thread, joined in a fixed order.
template <int kThreads>
__device__ inline Stats join_workgroup(Stats mine) {
  for (int d = 32; d >= 1; d >>= 1) mine = join(mine, {__shfl_xor(mine.m, d), __shfl_xor(mine.s, d)});
  if constexpr (kThreads > 64) {
    __shared__ Stats part[kThreads / 64];
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = mine;
    __syncthreads();
    mine = part[threadIdx.x & (kThreads / 64 - 1)];
    for (int d = kThreads / 128; d >= 1; d >>= 1) mine = join(mine, {__shfl_xor(mine.m, d), __shfl_xor(mine.s, d)});
  }
  return mine;
}

// The statistics of this thread's part of the elements [begin, end) of a row, 16 bytes a lane, four loads in flight.  With kEven
// nothing is done for the part of a step behind whole ones where there is none.
template <typename T, int kThreads, bool kOnce, bool kEven = false>
__device__ inline Stats stream(const T* x, int64_t begin, int64_t end) {
  constexpr int kWidth = Vec<T>::kWidth, kDeep = 4;
  Stats stats = {-INFINITY, 0.0f};
  const T* at = x + begin + (int64_t)threadIdx.x * kWidth;
  int64_t left = (end - begin) / kWidth;                    // whole vectors, and what is behind them
  const int rest = (int)((end - begin) % kWidth);
  for (; left >= kDeep * kThreads; left -= kDeep * kThreads, at += kDeep * kThreads * kWidth) {
    Vec<T> v[kDeep];
#pragma unroll
    for (int k = 0; k < kDeep; ++k) v[k] = Vec<T>::template load<kOnce>(at + k * kThreads * kWidth);
    absorb<T, kDeep>(stats, v);
  }
  if (kEven && left == 0 && rest == 0) return stats;
  Vec<T> v[kDeep];
#pragma unroll
  for (int k = 0; k < kDeep; ++k) {
    v[k] = Vec<T>::all(-INFINITY);
    if (k * kThreads + (int)threadIdx.x < left) v[k] = Vec<T>::template load<kOnce>(at + k * kThreads * kWidth);
  }
  absorb<T, kDeep>(stats, v);
  if ((int)threadIdx.x < rest) stats = join(stats, {to_float(x[end - rest + (int)threadIdx.x]), 1.0f});
  return stats;
}

// The same for any length.  Terms that are alike err alike, and of tens of millions of them added one after another 32 bits lose a
// thousandth: the sums of kStretch elements a thread, which are 128 additions, are added in 64 bits.
constexpr int kStretch = 256;

template <typename T, int kThreads, bool kOnce>
__device__ inline Stats stream_long(const T* x, int64_t begin, int64_t end) {
  double sum = 0.0;
  float m = -INFINITY;
  for (; begin < end; begin += kThreads * kStretch) {
    const Stats some = stream<T, kThreads, kOnce, true>(x, begin, min(end, begin + kThreads * kStretch));
    const float to = fmaxf(m, some.m), r = reference_of(to);
    sum = sum * (double)change_of(m, r) + (double)(some.s * change_of(some.m, r));
    m = to;
  }
  return {m, (float)sum};
}

// The logarithm of a token's probability.  The difference first, which is exact or nearly so: of logits that are all the type's
// lowest value m + log s keeps nothing of s.  The logarithm is 32-bit (1.4e-7 below its value on average, 2.4e-7 in the mean
// square), like that of reference and old log-probabilities from elsewhere, in whose differences to these its lean goes away again:
// margins of pairs of some hundreds of tokens come out 1e-5 of themselves from 64 bits, and 4e-6 from 32-bit torch on this device.
__device__ inline float logprob_of(float x, Stats all) { return (x - all.m) - logf(all.s); }

__device__ inline float lse_of(Stats all) { return all.m + logf(all.s); }

enum RowKind { kRowLogprob, kRowStep, kRowPolicy };

struct RowArgs {
  const int32_t* targets;
  float* logprobs;            // null: not wanted
  float* lse;                 // null: not wanted
  Stats* stats;               // null: not wanted; of scored rows
  const float* upstream;      // kRowStep
  int64_t grad_stride;
  bool once;                  // logits, and whole lines of the gradient, pass the caches by
  // kRowPolicy
  const float* weight;        // of each row's loss; 0: not scored
  const int32_t* scored;      // the numbers of scored rows whose sum the loss is divided by,
  int n_scored;               // if there are any of them
  const float* advantage;     // of each row
  const float* old;
  const float* reference;
  float low, high, kl_weight, scale;
  double* value;              // of each row: its share of the loss
};

// What a row has besides its logits.  Everything is read before the logits, side by side: read when the row's sums are there, it
// would be one more wait for memory while the row occupies its compute unit (policy loss of 8,000 rows of 12,000 bfloat16: 91 us
// instead of 84; 8,190 of 100,260: 589 instead of 585).
struct RowInputs {
  int32_t target;
  float weight, upstream, advantage, old, reference;
  int32_t counted, counted_more;                            // this lane's part of the number of scored rows
};

template <int kKind>
__device__ inline RowInputs inputs_of(const RowArgs& a, int64_t t) {
  RowInputs in{};
  in.target = a.targets[t];
  in.weight = kKind == kRowPolicy ? a.weight[t] : 1.0f;
  if constexpr (kKind == kRowStep) in.upstream = a.upstream[t];
  if constexpr (kKind == kRowPolicy) {
    in.advantage = a.advantage[t];
    in.old = a.old[t];
    if (a.reference) in.reference = a.reference[t];
    const int lane = threadIdx.x & 63;
    if (lane < a.n_scored) in.counted = a.scored[lane];
    for (int i = 64 + lane; i < a.n_scored; i += 64) in.counted_more += a.scored[i];
  }
  return in;
}

__device__ inline bool is_scored(const RowInputs& in, int64_t vocab) {
  return in.target >= 0 && in.target < vocab && in.weight != 0.0f;
}

// The loss of one token under the clipped policy, and its derivative with respect to the token's log-probability.  Comparisons that
// keep a NaN: fminf and fmaxf would put the bound in the place of a ratio that is none.  An advantage of 0 has no part in the loss,
// however large the ratio.
__device__ inline float policy_value(const RowArgs& a, const RowInputs& in, float lp, float* slope) {
  const float ratio = expf(lp - in.old), low = 1.0f - a.low, high = 1.0f + a.high;
  const float clipped = (ratio < low ? low : ratio > high ? high : ratio) * in.advantage;
  const float free = in.advantage == 0.0f ? clipped : ratio * in.advantage;
  float value = clipped < free ? -clipped : -free;
  *slope = clipped < free ? 0.0f : -free;
  if (a.reference) {
    const float d = in.reference - lp;
    value += a.kl_weight * (expm1f(d) - d);
    *slope -= a.kl_weight * expm1f(d);
  }
  return value;
}

// What a row's log-probability gives besides, by one wave: the outputs of thread 0, and the factor of the row's gradient.
template <int kKind>
__device__ inline float finish_row(const RowArgs& a, int64_t t, const RowInputs& in, Stats all, float lp) {
  if (threadIdx.x == 0) {
    if (a.logprobs) a.logprobs[t] = lp;
    if (a.lse) a.lse[t] = lse_of(all);
    if (a.stats) a.stats[t] = all;
  }
  if constexpr (kKind == kRowStep) return in.upstream;
  if constexpr (kKind == kRowPolicy) {
    float weight = in.weight, slope;
    if (a.n_scored > 0) {
      int32_t scored = in.counted + in.counted_more;
      for (int d = 32; d >= 1; d >>= 1) scored += __shfl_xor(scored, d);
      weight = 1.0f / (float)scored;
    }
    const float value = policy_value(a, in, lp, &slope);
    if (threadIdx.x == 0) a.value[t] = (double)weight * value;
    return a.scale * weight * slope;
  }
  return 0.0f;
}

template <int kKind>
__device__ inline void skip_row(const RowArgs& a, int64_t t) {
  if (threadIdx.x == 0) {
    if (a.logprobs) a.logprobs[t] = 0.0f;
    if (a.lse) a.lse[t] = 0.0f;
    if (kKind == kRowPolicy) a.value[t] = 0.0;
  }
}

// Zeros: whole lines, and the elements before and behind them.
template <typename T, int kThreads>
__device__ inline void zero_row(T* g, int64_t vocab, bool once) {
  constexpr int kWidth = Vec<T>::kWidth;
  const int head = head_of<kLine>(g, vocab);
  const int64_t whole = (vocab - head) / kWidth;
  if (once)
    for (int64_t j = threadIdx.x; j < whole; j += kThreads) Vec<T>::all(0.0f).template store<true>(g + head + j * kWidth);
  else
    for (int64_t j = threadIdx.x; j < whole; j += kThreads) Vec<T>::all(0.0f).store(g + head + j * kWidth);
  const int edges = (int)(vocab - whole * kWidth);
  for (int j = threadIdx.x; j < edges; j += kThreads) g[j < head ? j : whole * kWidth + j] = from_float<T>(0.0f);
}

// share x exp(x - reference) of the elements of a vector.
template <typename T>
__device__ inline Vec<T> grad_of(const Vec<T>& v, float reference, float share) {
  float x[Vec<T>::kWidth];
  v.get(x);
#pragma unroll
  for (int i = 0; i < Vec<T>::kWidth; ++i) x[i] = share * exp_of(x[i], reference);
  return Vec<T>::of(x);
}

// Log-probabilities alone, one workgroup a row: bound by memory (see above); a single row by its compute unit's exponentials, 9 us
// for 100,260.
template <typename T, int kThreads, bool kLong>
__global__ void __launch_bounds__(kThreads) logprobs_kernel(const T* logits, int64_t vocab, int64_t stride, int64_t first, RowArgs a) {
  const int64_t t = first + blockIdx.x;
  const RowInputs in = inputs_of<kRowLogprob>(a, t);
  if (!is_scored(in, vocab)) return skip_row<kRowLogprob>(a, t);
  const T* x = logits + t * stride;
  const float at_target = to_float(x[in.target]);
  Stats mine;
  if constexpr (kLong) mine = a.once ? stream_long<T, kThreads, true>(x, 0, vocab) : stream_long<T, kThreads, false>(x, 0, vocab);
  else mine = a.once ? stream<T, kThreads, true>(x, 0, vocab) : stream<T, kThreads, false>(x, 0, vocab);
  const Stats all = join_workgroup<kThreads>(mine);
  if (threadIdx.x == 0) finish_row<kRowLogprob>(a, t, in, all, logprob_of(at_target, all));
}

// Few rows: each is split among `parts` workgroups, whose statistics another kernel joins.
template <typename T, bool kLong>
__global__ void __launch_bounds__(256) logprobs_part_kernel(const T* logits, int64_t vocab, int64_t stride, const int32_t* targets,
                                                            unsigned parts, int64_t each, Stats* part) {
  const int64_t t = blockIdx.x / parts, begin = blockIdx.x % parts * each, end = min(vocab, begin + each);
  const int32_t target = targets[t];
  if (target < 0 || target >= vocab) return;
  const T* x = logits + t * stride;
  const Stats all = join_workgroup<256>(kLong ? stream_long<T, 256, false>(x, begin, end) : stream<T, 256, false>(x, begin, end));
  if (threadIdx.x == 0) part[blockIdx.x] = all;
}

// One wave a row.
template <typename T>
__global__ void __launch_bounds__(64) logprobs_join_kernel(const T* logits, int64_t vocab, int64_t stride, int parts,
                                                           const Stats* part, RowArgs a) {
  const int64_t t = blockIdx.x;
  const RowInputs in = inputs_of<kRowLogprob>(a, t);
  if (!is_scored(in, vocab)) return skip_row<kRowLogprob>(a, t);
  const float at_target = to_float(logits[t * stride + in.target]);
  Stats mine = {-INFINITY, 0.0f};
  for (int k = threadIdx.x; k < parts; k += 64) mine = join(mine, part[t * parts + k]);
  const Stats all = join_workgroup<64>(mine);
  if (threadIdx.x == 0) finish_row<kRowLogprob>(a, t, in, all, logprob_of(at_target, all));
}

// Log-probability and gradient of a row in one pass: the row stays in the workgroup's registers, kVecs x 16 bytes a lane, at most
// 128 registers in all.  One barrier for the statistics and one for the row's factor, which the first wave works out.  Workgroups of
// 512 threads share a compute unit by two, the one loading while the other stores; one of 1,024 has it to itself, and its loads,
// exponentials and stores follow each other (3,000 rows of 100,260 float32 in 430 us, 5.6 TB/s, of 128,256 bfloat16 in 309, 5.0).
// The last of a lane's vectors does not pass the caches by: the compiler makes one plain access of both branches' last.
template <typename T, int kKind, int kThreads, int kVecs>
__global__ void __launch_bounds__(kThreads, 4) row_kernel(const T* logits, int64_t vocab, int64_t stride, int64_t first, RowArgs a, T* grad) {
  constexpr int kWidth = Vec<T>::kWidth, kDeep = kVecs < 4 || (kVecs > 16 && sizeof(T) == 2) ? 2 : 4;
  __shared__ float factor[2];
  const int64_t t = first + blockIdx.x;
  T* g = grad + t * a.grad_stride;
  const RowInputs in = inputs_of<kKind>(a, t);
  if (!is_scored(in, vocab)) {
    skip_row<kKind>(a, t);
    return zero_row<T, kThreads>(g, vocab, a.once);
  }
  const T* x = logits + t * stride;
  // Whole vectors from the row's first line on; the elements before and behind them, at most one a thread.  (Not from the
  // gradient's first line on, which mostly is the same: sums would depend on where the gradient goes.)
  constexpr int kBytes = kThreads == 64 ? 64 : kLine;
  const int head = head_of<kBytes>(x, vocab), whole = ((int)vocab - head) / kWidth;
  const int edges = (int)vocab - whole * kWidth, lane_at = (int)threadIdx.x;
  const int edge_at = lane_at < head ? lane_at : whole * kWidth + lane_at;
  Vec<T> v[kVecs];
#pragma unroll
  for (int k = 0; k < kVecs; ++k) v[k] = Vec<T>::all(-INFINITY);
  if (a.once) {
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
      if (k * kThreads + lane_at < whole) v[k] = Vec<T>::template load<true>(x + head + (k * kThreads + lane_at) * kWidth);
  } else {
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
      if (k * kThreads + lane_at < whole) v[k] = Vec<T>::load(x + head + (k * kThreads + lane_at) * kWidth);
  }
  float edge = -INFINITY;
  if (lane_at < edges) edge = to_float(x[edge_at]);
  const float at_target = to_float(x[in.target]);
  Stats mine = {-INFINITY, 0.0f};
#pragma unroll
  for (int k = 0; k + kDeep <= kVecs; k += kDeep) absorb<T, kDeep>(mine, v + k);
  if constexpr (kVecs % kDeep) absorb<T, kVecs % kDeep>(mine, v + kVecs / kDeep * kDeep);
  const Stats all = join_workgroup<kThreads>(join(mine, {edge, 1.0f}));
  if (threadIdx.x < 64) {
    const float lp = logprob_of(at_target, all);
    const float c = finish_row<kKind>(a, t, in, all, lp);
    if (threadIdx.x == 0) {
      factor[0] = c;
      factor[1] = -c * expm1f(lp);                          // the gradient at the target: 1 - p without the cancellation
    }
  }
  __syncthreads();
  const float c = factor[0];
  if (c == 0.0f) return zero_row<T, kThreads>(g, vocab, a.once);
  const float share = -c / all.s;
  // (The logits are converted once more: kept as 32-bit numbers they would take twice the registers.)
#pragma unroll
  for (int k = 0; k < kVecs; ++k) asm("" : "+v"(v[k].w));
  if (a.once && head == head_of<kBytes>(g, vocab)) {
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
      if (k * kThreads + lane_at < whole) grad_of(v[k], all.m, share).template store<true>(g + head + (k * kThreads + lane_at) * kWidth);
  } else {
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
      if (k * kThreads + lane_at < whole) grad_of(v[k], all.m, share).store(g + head + (k * kThreads + lane_at) * kWidth);
  }
  if (lane_at < edges) g[edge_at] = from_float<T>(share * exp_of(edge, all.m));
  // The target's element once more, by the thread that has just written it.
  const int in_body = in.target - head;
  if (in_body >= 0 && in_body < whole * kWidth ? lane_at == in_body / kWidth % kThreads : lane_at < edges && edge_at == in.target)
    g[in.target] = from_float<T>(factor[1]);
}

// The same for rows that no workgroup's registers hold (over 400 KiB): they are read twice, first plainly, so that the second reading
// may find some of it in the caches (3,000 rows of 300,007 bfloat16: 826 us, 6.5 TB/s with both).
template <typename T, int kKind>
__global__ void __launch_bounds__(1024) long_row_kernel(const T* logits, int64_t vocab, int64_t stride, int64_t first, RowArgs a, T* grad) {
  constexpr int kWidth = Vec<T>::kWidth, kThreads = 1024;
  __shared__ float factor[2];
  const int64_t t = first + blockIdx.x;
  T* g = grad + t * a.grad_stride;
  const RowInputs in = inputs_of<kKind>(a, t);
  if (!is_scored(in, vocab)) {
    skip_row<kKind>(a, t);
    return zero_row<T, kThreads>(g, vocab, a.once);
  }
  const T* x = logits + t * stride;
  const float at_target = to_float(x[in.target]);
  const Stats all = join_workgroup<kThreads>(stream_long<T, kThreads, false>(x, 0, vocab));
  if (threadIdx.x < 64) {
    const float lp = logprob_of(at_target, all);
    const float c = finish_row<kKind>(a, t, in, all, lp);
    if (threadIdx.x == 0) {
      factor[0] = c;
      factor[1] = -c * expm1f(lp);                          // the gradient at the target: 1 - p without the cancellation
    }
  }
  __syncthreads();
  const float c = factor[0];
  if (c == 0.0f) return zero_row<T, kThreads>(g, vocab, a.once);
  const float share = -c / all.s;
  const int head = head_of<kLine>(g, vocab), lane_at = (int)threadIdx.x;
  const int64_t whole = (vocab - head) / kWidth, edges = vocab - whole * kWidth;
  if (a.once)
    for (int64_t j = lane_at; j < whole; j += kThreads)
      grad_of(Vec<T>::template load<true>(x + head + j * kWidth), all.m, share).template store<true>(g + head + j * kWidth);
  else
    for (int64_t j = lane_at; j < whole; j += kThreads)
      grad_of(Vec<T>::load(x + head + j * kWidth), all.m, share).store(g + head + j * kWidth);
  const int64_t edge_at = lane_at < head ? lane_at : whole * kWidth + lane_at;
  if (lane_at < edges) g[edge_at] = from_float<T>(share * exp_of(to_float(x[edge_at]), all.m));
  const int64_t in_body = in.target - head;
  if (in_body >= 0 && in_body < whole * kWidth ? lane_at == in_body / kWidth % kThreads : lane_at < edges && edge_at == in.target)
    g[in.target] = from_float<T>(factor[1]);
}

// The sum over a workgroup, in every thread, in a fixed order.
template <int kThreads, typename V>
__device__ inline V sum_workgroup(V mine) {
  __shared__ V part[kThreads / 64];
  for (int d = 32; d >= 1; d >>= 1) mine += __shfl_xor(mine, d);
  __syncthreads();                                          // (the last sum's parts are read)
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = mine;
  __syncthreads();
  V all = part[0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) all += part[w];
  return all;
}

// The sum of values, by one workgroup.
template <int kThreads>
__device__ inline void sum_values(const double* values, int64_t n, float* sum) {
  constexpr int kDeep = 16;
  double mine = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += kThreads * kDeep) {
    double v[kDeep];
#pragma unroll
    for (int k = 0; k < kDeep; ++k) v[k] = values[min(i + k * kThreads, n - 1)];       // (all reads side by side)
#pragma unroll
    for (int k = 0; k < kDeep; ++k) mine += i + k * kThreads < n ? v[k] : 0.0;
  }
  mine = sum_workgroup<kThreads>(mine);
  if (threadIdx.x == 0) *sum = (float)mine;
}

// The gradient from what was saved of each row: element by element, bound by memory.  A workgroup has up to 1,024 vectors of a row,
// one of its `parts`.  Saved is lse, the caller's, or, where it never leaves the library, `stats`: the maximum and the sum apart, as a
// 32-bit lse of logits about 10^4 says their sum to 10^-3 only, and of the type's lowest value nothing.  With `loss`, one workgroup
// more: the loss is the sum of the pairs' losses.
template <typename T, bool kOnce>
__global__ void __launch_bounds__(256) logprobs_grad_kernel(const T* logits, int64_t vocab, int64_t stride, int64_t first, unsigned parts,
                                                            const int32_t* targets, const float* lse, const Stats* stats,
                                                            const float* upstream, T* grad, int64_t grad_stride, const double* losses,
                                                            int32_t n_losses, float* loss) {
  if (blockIdx.x == gridDim.x - 1 && loss) return sum_values<256>(losses, n_losses, loss);
  constexpr int kWidth = Vec<T>::kWidth, kDeep = 4;
  const int64_t t = first + blockIdx.x / parts;
  const unsigned part = blockIdx.x % parts;
  const int32_t target = targets[t];
  const float c = target >= 0 && target < vocab ? upstream[t] : 0.0f;
  const T* x = logits + t * stride;
  T* g = grad + t * grad_stride;
  // Whole vectors from the first line of the gradient's row on; the first part has the elements before them, the last those behind.
  const int head = head_of<kLine>(g, vocab), at = threadIdx.x;
  const int64_t begin = head + (int64_t)part * (256 * kDeep * kWidth), left = max(vocab - begin, (int64_t)0);
  const int whole = (int)min(left / kWidth, (int64_t)(256 * kDeep));
  int64_t edge_at = -1;
  if (part == 0 && at < head) edge_at = at;
  else if (whole < 256 * kDeep) {
    const int64_t j = begin + whole * kWidth + at - (part == 0 ? head : 0);
    if (j < vocab) edge_at = j;
  }
  if (c == 0.0f) {
#pragma unroll
    for (int k = 0; k < kDeep; ++k)
      if (k * 256 + at < whole) Vec<T>::all(0.0f).template store<kOnce>(g + begin + (k * 256 + at) * kWidth);
    if (edge_at >= 0) g[edge_at] = from_float<T>(0.0f);
    return;
  }
  const Stats all = stats ? stats[t] : Stats{lse[t], 1.0f};
  const float share = -c / all.s;
  Vec<T> v[kDeep];
#pragma unroll
  for (int k = 0; k < kDeep; ++k)
    if (k * 256 + at < whole) v[k] = Vec<T>::template load<kOnce>(x + begin + (k * 256 + at) * kWidth);
  const int64_t in_body = target - begin;
  const bool here = in_body >= 0 && in_body < whole * kWidth ? in_body / kWidth % 256 == at : edge_at == target;
  float at_target = 0.0f;
  if (here) at_target = to_float(x[target]);
  if (edge_at >= 0) g[edge_at] = from_float<T>(share * exp_of(to_float(x[edge_at]), all.m));
#pragma unroll
  for (int k = 0; k < kDeep; ++k)
    if (k * 256 + at < whole) grad_of(v[k], all.m, share).template store<kOnce>(g + begin + (k * 256 + at) * kWidth);
  if (here) g[target] = from_float<T>(-c * expm1f(logprob_of(at_target, all)));
}

// ---- over strings --------------------------------------------------------------------------------------------

// String i's rows, as far as there are any.
__device__ inline void string_rows(const int64_t* offsets, int32_t i, int64_t n, int64_t* begin, int64_t* end) {
  *begin = min(max(offsets[i], (int64_t)0), n);
  *end = max(*begin, min(offsets[i + 1], n));
}

// The string of row t, -1 outside; t is the lane's number further than the wave's first row.  All lanes take part: 64 offsets
// are looked at together, so that up to 64 strings take one read, up to 4,096 two.  Lanes whose rows are in a later string than
// the first lane's look for it on their own.
__device__ inline int32_t string_of(const int64_t* offsets, int32_t batch, int64_t t, int lane) {
  const int64_t first = t - lane;
  int64_t lo = 0, hi = batch;                               // the first string that ends behind the wave's first row
  while (hi - lo > 0) {
    const int64_t step = (hi - lo + 63) / 64, at = lo + (lane + 1) * step - 1;
    const uint64_t ends_before = __ballot(at < hi && offsets[min(at, hi - 1) + 1] <= first);
    lo += (int64_t)__popcll(ends_before) * step;
    hi = min(hi, lo + step - 1);
  }
  if (lo < batch && offsets[lo + 1] <= t) {
    ++lo;
    hi = batch;
    while (lo < hi) {
      const int64_t mid = (lo + hi) >> 1;
      if (offsets[mid + 1] <= t) lo = mid + 1; else hi = mid;
    }
  }
  return lo < batch && offsets[lo] <= t ? (int32_t)lo : -1;
}

// A thread a position; 2.3 us for 301, 4.7 for 8,003: reads that wait for each other, the offsets, the string's prompt, the id.
__global__ void __launch_bounds__(256) next_tokens_kernel(const int32_t* ids, int64_t n, const int64_t* offsets, int32_t batch,
                                                          const int32_t* first, int32_t* targets) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int32_t i = string_of(offsets, batch, t, threadIdx.x & 63);
  if (t >= n) return;
  const bool scored = i >= 0 && t + 1 < n && t + 1 < offsets[i + 1] && (!first || t + 1 - offsets[i] >= first[i]);
  targets[t] = scored ? ids[t + 1] : -1;
}

__device__ inline bool is_scored(const int32_t* targets, int64_t t, int64_t vocab) {
  return targets[t] >= 0 && targets[t] < vocab;
}

// f(t) for the rows that are in no string.
template <int kThreads, typename F>
__device__ inline void rows_outside(const int64_t* offsets, int32_t batch, int64_t n, F&& f) {
  const int64_t begin = batch > 0 ? min(max(offsets[0], (int64_t)0), n) : n, end = batch > 0 ? min(offsets[batch], n) : n;
  for (int64_t t = threadIdx.x; t < begin; t += kThreads) f(t);
  for (int64_t t = max(begin, end) + threadIdx.x; t < n; t += kThreads) f(t);
}

// One workgroup a pair: both sides' sums, in 64 bits as there are thousands of terms of either sign, the loss, and the factor of
// each row's gradient.  One more: rows outside every string.  3 us for short strings, 6 for some hundreds of rows, again of waiting.
template <int kThreads>
__global__ void __launch_bounds__(kThreads) pair_kernel(const float* logprobs, const int32_t* targets, int64_t n, int64_t vocab,
                                                        const int64_t* offsets, int32_t batch, const float* reference, float beta,
                                                        float smoothing, float scale, float* margins, double* losses,
                                                        float* upstream) {
  const int32_t k = blockIdx.x;
  if (k == batch / 2) return rows_outside<kThreads>(offsets, batch, n, [&](int64_t t) { upstream[t] = 0.0f; });
  int64_t begin, middle, end, unused;
  string_rows(offsets, 2 * k, n, &begin, &middle);
  string_rows(offsets, 2 * k + 1, n, &unused, &end);
  constexpr int kDeep = 4;
  double sum = 0.0;
  for (int64_t t0 = begin + threadIdx.x; t0 < end; t0 += kThreads * kDeep) {
    int32_t target[kDeep];
    float lp[kDeep], ref[kDeep];
#pragma unroll
    for (int k = 0; k < kDeep; ++k) {                        // (all reads side by side)
      const int64_t t = min(t0 + k * kThreads, end - 1);
      target[k] = targets[t];
      lp[k] = logprobs[t];
      ref[k] = reference ? reference[t] : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < kDeep; ++k) {
      const int64_t t = t0 + k * kThreads;
      const double apart = (double)lp[k] - (double)ref[k];
      if (t < end && target[k] >= 0 && target[k] < vocab) sum += t < middle ? apart : -apart;
    }
  }
  const double z = (double)beta * sum_workgroup<kThreads>(sum);
  // -log sigmoid(z) = max(-z, 0) + log(1 + exp(-|z|)).  A masked target makes z infinite and one of the two terms with it: left out
  // where its weight is 0.  (tail is NaN where z is.)
  const double tail = log1p(exp(-fabs(z))), less = (double)smoothing;
  const double loss = tail + (less < 1.0 ? (1.0 - less) * fmax(-z, 0.0) : 0.0) + (less > 0.0 ? less * fmax(z, 0.0) : 0.0);
  const double slope = less - 1.0 / (1.0 + exp(z));
  const float c = (float)((double)scale * (double)beta * slope / (batch / 2));
  if (threadIdx.x == 0) {
    losses[k] = loss / (batch / 2);
    if (margins) margins[k] = (float)z;
  }
  for (int64_t t = begin + threadIdx.x; t < end; t += kThreads) upstream[t] = t < middle ? c : -c;
}

__global__ void __launch_bounds__(1024) sum_kernel(const double* values, int64_t n, float* sum) {
  sum_values<1024>(values, n, sum);
}

constexpr int kWeightWaves = 4;                              // waves of a workgroup
constexpr int kShortString = 1024;                           // positions that one wave goes over

// The weight of each scored position in its string's loss and its advantage; and the number of scored positions of this
// workgroup's strings.  `strings` of them, one a wave, or one where most are long; the whole workgroup goes over the long ones, one
// after the other.  The last workgroup: rows outside every string.  4 us for short strings, 8 for some of hundreds of positions:
// reads that wait for each other.
__global__ void __launch_bounds__(64 * kWeightWaves) weights_kernel(const int32_t* targets, int64_t n, int64_t vocab,
                                                                    const int64_t* offsets, int32_t batch, int by_string,
                                                                    const float* advantages, int advantage_by_string, float* weight,
                                                                    float* advantage, int32_t* scored, int strings) {
  constexpr int kThreads = 64 * kWeightWaves, kEach = kShortString / 64, kHalf = kEach / 2;
  if (blockIdx.x == gridDim.x - 1) return rows_outside<kThreads>(offsets, batch, n, [&](int64_t t) { weight[t] = 0.0f; });
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const auto weight_of = [&](int32_t count) { return by_string ? 1.0f / ((float)batch * (float)max(count, 1)) : 1.0f; };
  int32_t all = 0;                                           // of the waves' strings, in lane 0 of each; of long ones in thread 0
  const int short_string = strings == 1 ? 64 : kShortString;
  for (int32_t i0 = blockIdx.x * strings; i0 < batch; i0 += (gridDim.x - 1) * strings) {
    const int32_t i = i0 + wave;
    int64_t begin = 0, end = 0;
    if (wave < strings && i < batch) string_rows(offsets, i, n, &begin, &end);
    if (end - begin <= short_string) {
      bool is[kEach];
      float adv[kEach];
      int32_t count = 0;
#pragma unroll
      for (int k = 0; k < kEach; ++k) {                      // (all reads side by side)
        const int64_t t = begin + k * 64 + lane;
        is[k] = t < end && is_scored(targets, t, vocab);
        adv[k] = t < end ? advantages[advantage_by_string ? i : t] : 0.0f;
      }
#pragma unroll
      for (int k = 0; k < kEach; ++k) count += __popcll(__ballot(is[k]));
      const float w = weight_of(count);
#pragma unroll
      for (int k = 0; k < kEach; ++k) {
        const int64_t t = begin + k * 64 + lane;
        if (t >= end) continue;
        weight[t] = is[k] ? w : 0.0f;
        advantage[t] = adv[k];
      }
      if (lane == 0) all += count;
    }
    if (!__syncthreads_or(end - begin > short_string)) continue;
    for (int32_t j = i0; j < min(i0 + strings, batch); ++j) {
      string_rows(offsets, j, n, &begin, &end);
      if (end - begin <= short_string) continue;
      int32_t count = 0;
      for (int64_t t0 = begin + threadIdx.x; t0 < end; t0 += kThreads * kEach) {
        int32_t target[kEach];
#pragma unroll
        for (int k = 0; k < kEach; ++k) target[k] = targets[min(t0 + k * kThreads, end - 1)];
#pragma unroll
        for (int k = 0; k < kEach; ++k) count += t0 + k * kThreads < end && target[k] >= 0 && target[k] < vocab;
      }
      count = sum_workgroup<kThreads>(count);
      const float w = weight_of(count);
      for (int64_t t0 = begin + threadIdx.x; t0 < end; t0 += kThreads * kHalf) {
        int32_t target[kHalf];
        float adv[kHalf];
#pragma unroll
        for (int k = 0; k < kHalf; ++k) {
          const int64_t t = min(t0 + k * kThreads, end - 1);
          target[k] = targets[t];
          adv[k] = advantages[advantage_by_string ? j : t];
        }
#pragma unroll
        for (int k = 0; k < kHalf; ++k) {
          const int64_t t = t0 + k * kThreads;
          if (t >= end) continue;
          weight[t] = target[k] >= 0 && target[k] < vocab ? w : 0.0f;
          advantage[t] = adv[k];
        }
      }
      if (threadIdx.x == 0) all += count;
    }
  }
  all = sum_workgroup<kThreads>(lane == 0 ? all : 0);
  if (threadIdx.x == 0) scored[blockIdx.x] = all;
}

}  // namespace bpe
