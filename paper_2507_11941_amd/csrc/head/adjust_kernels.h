// Logits as a token is chosen from: penalties for tokens that a row's history holds, biases, masks; and the gradient.
//
// Bound by reading and writing the logits (509 rows of 100,260 bfloat16 under masks in 32.5 us, 6.3 TB/s), and, with histories of thousands
// of tokens, by looking through them.  A workgroup has a stretch of a row's columns: it counts the history's tokens among them in shared
// memory (whole numbers, so that the order of the additions does not matter) while its logits are on their way, and applies all of it to the
// logits in registers, which are rounded once.  A history is read once for each stretch of its row, from the caches.
#pragma once
#include "../ops/element.h"

namespace bpe {

constexpr int kAdjustEach = 16;                             // elements of a lane

struct AdjustArgs {
  const int32_t* ids;
  const int64_t* begin;       // null: no histories
  const int64_t* end;
  const float* penalties;     // null: those below for all rows
  const int32_t* bias_ids;
  const float* bias_values;
  const int64_t* bias_begin;  // null: no biases
  const int64_t* bias_end;
  const uint8_t* mask;        // null: none
  const int32_t* state;       // null: row t has mask t, or all have the only one
  int64_t n_ids, n_biases, states, mask_stride, stride, logits_stride, out_stride, vocab, first;
  float repetition, presence, frequency;
  unsigned stretches;
};

// A part of a list that lies within it.
struct Span {
  int64_t begin, end;
};

__device__ inline Span span_of(const int64_t* begin, const int64_t* end, int64_t t, int64_t n) {
  if (!begin) return {0, 0};
  return {max(begin[t], (int64_t)0), min(end[t], n)};
}

// f(place in the span, id - column) for the ids of a span that are among these columns; eight reads side by side.
template <int kThreads, typename F>
__device__ inline void for_ids(const int32_t* ids, Span s, int32_t column, int32_t columns, F&& f) {
  constexpr uint32_t kDeep = 8;
  const int32_t* p = ids + s.begin;
  const uint32_t count = (uint32_t)min(s.end - s.begin, (int64_t)0xfffffff0);
  const auto look = [&](uint32_t i, int32_t id) {
    const uint32_t at = (uint32_t)id - (uint32_t)column;     // (what is before the columns, negative ids among it, becomes large)
    if (at < (uint32_t)columns) f(i, at);
  };
  uint32_t first = 0;
  for (; count - first >= kDeep * kThreads; first += kDeep * kThreads) {
    int32_t id[kDeep];
#pragma unroll
    for (uint32_t k = 0; k < kDeep; ++k) id[k] = p[first + k * kThreads + threadIdx.x];
#pragma unroll
    for (uint32_t k = 0; k < kDeep; ++k) look(first + k * kThreads + threadIdx.x, id[k]);
  }
  // (The rest: places behind the end read the last id once more, and do not look at it.)
  const uint32_t left = count - first;
  int32_t id[kDeep];
#pragma unroll
  for (uint32_t k = 0; k < kDeep; ++k)
    if (k * kThreads < left) id[k] = p[first + min(k * kThreads + threadIdx.x, left - 1)];
#pragma unroll
  for (uint32_t k = 0; k < kDeep; ++k)
    if (k * kThreads < left) look(first + k * kThreads + threadIdx.x, k * kThreads + threadIdx.x < left ? id[k] : -1);
}

// The numbers of a lane's vector in shared memory.
template <int kWidth>
__device__ inline void numbers_of(const uint32_t* p, uint32_t (&c)[kWidth]) {
#pragma unroll
  for (int i = 0; i < kWidth; i += 4) {
    const Words w = *(const Words*)(p + i);
    for (int j = 0; j < 4; ++j) c[i + j] = w[j];
  }
}

// The first `valid` elements of a vector; all of them at once.
template <typename T>
__device__ inline void load_part(const T* p, int valid, float (&x)[Vec<T>::kWidth]) {
  if (valid == Vec<T>::kWidth) return Vec<T>::load(p).get(x);
  for (int i = 0; i < Vec<T>::kWidth; ++i) x[i] = i < valid ? to_float(p[i]) : 0.0f;
}

template <typename T>
__device__ inline void store_part(T* p, int valid, const float (&x)[Vec<T>::kWidth]) {
  if (valid == Vec<T>::kWidth) return Vec<T>::of(x).store(p);
  for (int i = 0; i < Vec<T>::kWidth; ++i)
    if (i < valid) p[i] = from_float<T>(x[i]);
}

// kGrad: `in` is the gradient of the adjusted logits, and `logits` are read where a token is in the history.  kInPlace: out is `in`,
// and vectors that do not change are neither read nor written.  Shared memory: a count for each column and, where there are biases,
// a place in the row's list of them.
template <typename T, bool kGrad, bool kInPlace, int kThreads>
__global__ void __launch_bounds__(kThreads) adjust_kernel(const T* in, const T* logits, T* out, AdjustArgs a) {
  constexpr int kWidth = Vec<T>::kWidth, kVecs = kAdjustEach / kWidth, kColumns = kThreads * kAdjustEach;
  extern __shared__ __attribute__((aligned(16))) uint32_t counts[];
  uint32_t* const places = counts + kColumns;
  const int64_t t = a.first + blockIdx.x / a.stretches;
  const int64_t column = (int64_t)(blockIdx.x % a.stretches) * kColumns;
  const int columns = (int)min((int64_t)kColumns, a.vocab - column), tid = threadIdx.x;
  const T* x = in + t * a.stride + column;

  Vec<T> v[kVecs];
  if constexpr (!kInPlace) {
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      const int at = (k * kThreads + tid) * kWidth;
      if (at + kWidth <= columns) v[k] = Vec<T>::load(x + at);
    }
  }
  const Span history = span_of(a.begin, a.end, t, a.n_ids), list = span_of(a.bias_begin, a.bias_end, t, a.n_biases);
  float repetition = a.repetition, presence = a.presence, frequency = a.frequency;
  if (a.penalties) {
    repetition = a.penalties[3 * t];
    presence = a.penalties[3 * t + 1];
    frequency = a.penalties[3 * t + 2];
  }
  const float reciprocal = 1.0f / repetition;                // (a second rounding for logits that are divided, and no division for each)
  const int64_t chosen = !a.mask ? -1 : a.state ? (int64_t)a.state[t] : a.states == 1 ? 0 : t;
  const bool masked = chosen >= 0 && chosen < a.states;
  uint32_t allowed[kVecs];
#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
    const int at = (k * kThreads + tid) * kWidth;
    allowed[k] = 255;
    if (masked && at < columns) allowed[k] = a.mask[chosen * a.mask_stride * 4 + (column + at) / 8] >> (at & 7);
  }

  const bool counted = history.begin < history.end, biased = !kGrad && list.begin < list.end;
  if (counted || biased) {                                   // (the same for the whole workgroup)
#pragma unroll
    for (int k = 0; k < kAdjustEach / 4; ++k) {
      if (counted) *(Words*)(counts + (k * kThreads + tid) * 4) = Words{0, 0, 0, 0};
      if (biased) *(Words*)(places + (k * kThreads + tid) * 4) = Words{0, 0, 0, 0};
    }
    __syncthreads();
    if (counted) for_ids<kThreads>(a.ids, history, (int32_t)column, columns, [&](uint32_t, uint32_t at) { atomicAdd(&counts[at], 1u); });
    if (biased)
      for_ids<kThreads>(a.bias_ids, list, (int32_t)column, columns,
                        [&](uint32_t i, uint32_t at) { atomicMax(&places[at], i + 1); });
    __syncthreads();
  }

#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
    const int at = (k * kThreads + tid) * kWidth, valid = min(kWidth, columns - at);
    if (valid <= 0) continue;
    uint32_t c[kWidth] = {}, place[kWidth] = {}, any = 0;
    if (counted) numbers_of<kWidth>(counts + at, c);
    if (biased) numbers_of<kWidth>(places + at, place);
#pragma unroll
    for (int i = 0; i < kWidth; ++i) any |= c[i] | place[i];
    const uint32_t all = (1u << valid) - 1, bits = allowed[k] & all;
    if (kInPlace && any == 0 && bits == all) continue;
    float y[kWidth] = {};
    if (bits != 0) {
      if (!kInPlace && valid == kWidth) v[k].get(y);
      else load_part(x + at, valid, y);
    }
    if constexpr (kGrad) {
      // (Logits by whole vectors where one has eight elements, by elements where it has four: 509 rows of 100,260 with 4,000 tokens of history
      // under masks 44.8 us for 48.3, with 16,000 70 for 80; in 32 bits with 1,000 86 for 78.)
      const T* from = logits + t * a.logits_stride + column + at;
      if (kWidth == 8 && any != 0 && bits != 0) {
        float was[kWidth];
        load_part(from, valid, was);
#pragma unroll
        for (int i = 0; i < kWidth; ++i) y[i] = c[i] ? y[i] * (was[i] > 0.0f ? reciprocal : repetition) : y[i];
      } else if (kWidth < 8 && any != 0) {
#pragma unroll
        for (int i = 0; i < kWidth; ++i)
          if (c[i] && (bits >> i & 1)) y[i] *= to_float(from[i]) > 0.0f ? reciprocal : repetition;
      }
    } else {
      // (Without branches for each element, of a long history's tokens some are among most waves' elements; one selection an element, and the
      // masks as bits: 509 rows of 100,260 with 4,000 tokens of history under masks 45.7 us -> 44.0, 2,011 of 32,256 with 250 45.6 -> 43.9.)
      if (any != 0) {
#pragma unroll
        for (int i = 0; i < kWidth; ++i) {
          const float factor = y[i] > 0.0f ? reciprocal : repetition, less = fmaf(frequency, (float)c[i], presence);
          const float changed = fmaf(y[i], factor, -less);
          y[i] = c[i] ? changed : y[i];
        }
      }
      if (biased) {
#pragma unroll
        for (int i = 0; i < kWidth; ++i)
          if (place[i]) y[i] += a.bias_values[list.begin + place[i] - 1];
      }
    }
#pragma unroll
    for (int i = 0; i < kWidth; ++i) {
      const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe((int)bits, i, 1), other = kGrad ? 0u : 0xff800000u;
      y[i] = __uint_as_float((__float_as_uint(y[i]) & keep) | (other & ~keep));
    }
    store_part(out + t * a.out_stride + column + at, valid, y);
  }
}

}  // namespace bpe
