// Root-mean-square norms of sums with the residual, into the type or into 8 bits, and their gradient; rows into 8 bits.
//
// All of it is bound by memory: a row is read once, stays in the registers of one workgroup while its sum of squares (and, for 8
// bits, its largest product) is joined, and is written once.  Sums are in 32 bits; a row whose squares leave their range is summed
// again in 64.  The gradient of the weights is summed over the rows of a workgroup in registers, at most kGradRows of them in 32
// bits, and over workgroups in 64 bits by a second kernel, in a fixed order.
#pragma once
#include "../ops/element.h"

namespace bpe {

// The weights of kWidth columns as 32-bit numbers.
template <int kWidth, typename W>
__device__ inline void load_weights(const W* p, float (&w)[kWidth]) {
#pragma unroll
  for (int i = 0; i < kWidth; i += Vec<W>::kWidth) {
    float part[Vec<W>::kWidth];
    Vec<W>::load(p + i).get(part);
#pragma unroll
    for (int j = 0; j < Vec<W>::kWidth; ++j) w[i + j] = part[j];
  }
}

// The sum over a workgroup and the largest value, in every thread, in a fixed order.
template <int kThreads>
__device__ inline float sum_all(float mine, float* part) {
  for (int d = 32; d >= 1; d >>= 1) mine += __shfl_xor(mine, d);
  if constexpr (kThreads > 64) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = mine;
    __syncthreads();
    mine = part[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) mine += part[w];
  }
  return mine;
}

template <int kThreads>
__device__ inline double sum_all(double mine, double* part) {
  for (int d = 32; d >= 1; d >>= 1) mine += __shfl_xor(mine, d);
  if constexpr (kThreads > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = mine;
    __syncthreads();
    mine = part[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) mine += part[w];
  }
  return mine;
}

template <int kThreads>
__device__ inline double largest_all(double mine, double* part) {
  for (int d = 32; d >= 1; d >>= 1) mine = fmax(mine, __shfl_xor(mine, d));
  if constexpr (kThreads > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = mine;
    __syncthreads();
    mine = part[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) mine = fmax(mine, part[w]);
  }
  return mine;
}

// A row's statistics: its sum of squares, 0 or NaN (NaN where the weights hold an infinity or NaN), and its largest |product|.
template <typename V>
struct RowSums {
  float squares, odd;
  V top;
};

template <bool kExact>
struct Largest {
  typedef float Type;
};
template <>
struct Largest<false> {
  typedef double Type;
};

__device__ inline float magnitude(float x) { return fabsf(x); }
__device__ inline double magnitude(double x) { return fabs(x); }
__device__ inline float larger(float a, float b) { return fmaxf(a, b); }
__device__ inline double larger(double a, double b) { return fmax(a, b); }

template <int kThreads, bool kTop, typename V>
__device__ inline RowSums<V> join_sums(RowSums<V> mine) {
  for (int d = 32; d >= 1; d >>= 1) {
    mine.squares += __shfl_xor(mine.squares, d);
    if constexpr (kTop) {
      mine.odd += __shfl_xor(mine.odd, d);
      mine.top = larger(mine.top, __shfl_xor(mine.top, d));
    }
  }
  if constexpr (kThreads > 64) {
    __shared__ RowSums<V> part[kThreads / 64];
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = mine;
    __syncthreads();
    mine = part[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) {
      mine.squares += part[w].squares;
      if constexpr (kTop) {
        mine.odd += part[w].odd;
        mine.top = larger(mine.top, part[w].top);
      }
    }
  }
  return mine;
}

// Whether a 32-bit sum of squares says what it should: neither beyond the type's range nor of squares below it.
__device__ inline bool in_range(float squares) { return squares > 1e-20f && squares < 1e37f; }

// A power of two that a row is multiplied by, and its factor divided by, where the factor is beyond the 32-bit numbers or among those that
// hold fewer bits.  A row of numbers about 2^-100 or smaller loses nothing by it; one of 2^100 or larger its elements' bits below 2^-149 + 32,
// of which its norm has none.
__device__ inline float lean_of(double root) { return root > 0x1p100 ? 0x1p64f : root < 0x1p-100 ? 0x1p-32f : 1.0f; }

enum NormKind { kNorm, kNorm8, kRows8 };

template <typename T, typename W>
struct NormArgs {
  const T* x;
  const T* residual;          // null: none
  const W* weight;
  T* summed;
  T* out;
  int8_t* q;
  float* rstd;                // kNorm: null: not wanted
  float* scales;
  int64_t stride, residual_stride, summed_stride, out_stride, q_stride, first;
  int dim;
  float eps;
};

// How products become 8-bit integers: by a 32-bit factor, or, where that says too little, by a 64-bit quotient.
struct Rounding {
  float factor;
  double top;
  bool slow;                  // of the whole row: its products are out of the 32-bit range
};

// The rounding and the scale of a row (see bpe_head.h); `root` is the norm's factor.
__device__ inline Rounding rounding_of(double top, double root, bool odd, float* scale) {
  Rounding r{0.0f, top, false};
  if (odd) {
    *scale = __builtin_nanf("");
    r.top = 1.0;
  } else if (top == 0.0) {
    *scale = 0.0f;
    r.top = 1.0;
  } else {
    *scale = (float)(top * root / 127.0);
    r.slow = !(top > 1e-30 && top < 1e30);
    if (!r.slow) r.factor = 127.0f / (float)top;
  }
  return r;
}

// s w 127 / top to the nearest integer, in the low byte of each number.  In 32 bits the quotient is off by at most three roundings of
// 127, 2.3e-5: only what lies within 1e-4 of the middle between two integers is computed in 64 bits, one vector of eight in six hundred.
// (Added to 1.5 x 2^23 a number is rounded to an integer, which the last bits of the sum hold.)
template <bool kWeights, int kWidth>
__device__ inline void to_8bit(const float (&s)[kWidth], const float (&w)[kWidth], const Rounding& r, bool odd, uint32_t (&q)[kWidth]) {
  constexpr float kInteger = 12582912.0f;
  float far = 0.0f;
#pragma unroll
  for (int i = 0; i < kWidth; ++i) {
    const float p = kWeights ? s[i] * w[i] : s[i], sum = fmaf(p, r.factor, kInteger);
    far = fmaxf(far, fabsf(fmaf(p, r.factor, kInteger - sum)));
    q[i] = __float_as_uint(sum);
  }
  if (r.slow || far > 0.4999f) {
#pragma unroll
    for (int i = 0; i < kWidth; ++i) {
      q[i] = (uint32_t)(int)rint((double)s[i] * (kWeights ? (double)w[i] : 1.0) * 127.0 / r.top);
      __builtin_amdgcn_sched_barrier(0);                     // (side by side these quotients would take all registers)
    }
  }
  if (odd) {
#pragma unroll
    for (int i = 0; i < kWidth; ++i) q[i] = 0;
  }
}

template <int kWidth>
__device__ inline void store_8bit(int8_t* p, const uint32_t (&q)[kWidth]) {
  typedef uint32_t Bytes __attribute__((ext_vector_type(kWidth / 4), aligned(1)));
  Bytes v;
#pragma unroll
  for (int i = 0; i < kWidth / 4; ++i) {
    // byte 0 of one number and byte 0 of the other, twice, then the two halves
    const uint32_t low = __builtin_amdgcn_perm(q[4 * i + 1], q[4 * i], 0x0c0c0400), high = __builtin_amdgcn_perm(q[4 * i + 3], q[4 * i + 2], 0x0c0c0400);
    const uint32_t all = low | high << 16;
    if constexpr (kWidth == 4) v = all;
    else v[i] = all;
  }
  *(Bytes*)p = v;
}

// One workgroup a row, which stays in registers: up to kVecs vectors a lane, and the elements behind whole vectors, one a thread.
template <typename T, typename W, int kKind, int kThreads, int kVecs>
__global__ void __launch_bounds__(kThreads) norm_kernel(NormArgs<T, W> a) {
  constexpr int kWidth = Vec<T>::kWidth;
  // kExact: products of 16-bit numbers have 32 bits at most, so that their largest is found in 32 bits where it is within their range.
  constexpr bool kEight = kKind != kNorm, kExact = kKind == kRows8 || (sizeof(T) == 2 && sizeof(W) == 2);
  const int64_t t = a.first + blockIdx.x;
  const int tid = threadIdx.x, whole = a.dim / kWidth, rest = a.dim % kWidth, edge_at = whole * kWidth + tid;
  const T* x = a.x + t * a.stride;
  Vec<T> v[kVecs];
  float w[kVecs][kWidth], edge = 0.0f, edge_w = 0.0f;
#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
    v[k] = Vec<T>::all(0.0f);
    if (k * kThreads + tid < whole) v[k] = Vec<T>::load(x + (k * kThreads + tid) * kWidth);
  }
  if (tid < rest) edge = to_float(x[edge_at]);
  if (a.residual) {
    const T* residual = a.residual + t * a.residual_stride;
    Vec<T> r[kVecs];
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      r[k] = Vec<T>::all(0.0f);
      if (k * kThreads + tid < whole) r[k] = Vec<T>::load(residual + (k * kThreads + tid) * kWidth);
    }
    if (tid < rest) edge = to_float(from_float<T>(edge + to_float(residual[edge_at])));
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      float s[kWidth], more[kWidth];
      v[k].get(s);
      r[k].get(more);
#pragma unroll
      for (int i = 0; i < kWidth; ++i) s[i] += more[i];
      v[k] = Vec<T>::of(s);
    }
  }
  if constexpr (kKind != kRows8) {
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
      if (k * kThreads + tid < whole) load_weights<kWidth>(a.weight + (k * kThreads + tid) * kWidth, w[k]);
      else
        for (int i = 0; i < kWidth; ++i) w[k][i] = 0.0f;
    if (tid < rest) edge_w = to_float(a.weight[edge_at]);
  } else {
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
      for (int i = 0; i < kWidth; ++i) w[k][i] = 1.0f;
    edge_w = 1.0f;
  }
  if (a.residual) {
    T* summed = a.summed + t * a.summed_stride;
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
      if (k * kThreads + tid < whole) v[k].store(summed + (k * kThreads + tid) * kWidth);
    if (tid < rest) summed[edge_at] = from_float<T>(edge);
  }

  typedef typename Largest<kExact>::Type Top;
  RowSums<Top> sums{edge * edge, kEight ? edge_w * 0.0f : 0.0f, kEight ? magnitude((Top)edge * (Top)edge_w) : (Top)0};
  if constexpr (kKind == kRows8) sums.odd = edge * 0.0f;
#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
    float s[kWidth];
    v[k].get(s);
#pragma unroll
    for (int i = 0; i < kWidth; ++i) {
      if constexpr (kKind != kRows8) sums.squares = fmaf(s[i], s[i], sums.squares);
      if constexpr (kEight) {
        sums.odd = fmaf(kKind == kRows8 ? s[i] : w[k][i], 0.0f, sums.odd);
        sums.top = larger(sums.top, magnitude((Top)s[i] * (Top)w[k][i]));
      }
    }
  }
  const RowSums<Top> all = join_sums<kThreads, kEight>(sums);
  // (Rows are converted once more: the 64-bit products, kept for where they are needed again, would take most registers.)
  if constexpr (kEight) {
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      asm("" : "+v"(v[k].w));
      if constexpr (kKind != kRows8) {
#pragma unroll
        for (int i = 0; i < kWidth; ++i) asm("" : "+v"(w[k][i]));
      }
    }
  }
  float root = 1.0f, lean = 1.0f;
  double root_64 = 1.0;
  bool odd = !(all.odd == 0.0f);
  if constexpr (kKind != kRows8) {
    if (in_range(all.squares)) {
      root = 1.0f / sqrtf(all.squares / (float)a.dim + a.eps);
      root_64 = root;
    } else {
      __shared__ double part[kThreads / 64];
      double mine = (double)edge * (double)edge;
      for (int k = 0; k < kVecs; ++k) {
        float s[kWidth];
        v[k].get(s);
        for (int i = 0; i < kWidth; ++i) mine += (double)s[i] * (double)s[i];
      }
      mine = sum_all<kThreads>(mine, part);
      odd = odd || !(mine < INFINITY);
      root_64 = 1.0 / sqrt(mine / (double)a.dim + (double)a.eps);
      root = (float)root_64;
      lean = lean_of(root_64);
    }
  }
  if constexpr (kKind == kNorm) {
    if (a.rstd && tid == 0) a.rstd[t] = root;
    T* out = a.out + t * a.out_stride;
    if (lean == 1.0f) {
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        if (k * kThreads + tid < whole) {
          float s[kWidth];
          v[k].get(s);
#pragma unroll
          for (int i = 0; i < kWidth; ++i) s[i] = s[i] * root * w[k][i];
          Vec<T>::of(s).store(out + (k * kThreads + tid) * kWidth);
        }
      }
      if (tid < rest) out[edge_at] = from_float<T>(edge * root * edge_w);
    } else {
      // (From memory, where each thread reads what it has read or written before: rare rows are to take no registers.  With the product by
      // `lean` in all rows 512 of 16,384 bfloat16 took 15.2 us for 12.5.)
      const T* from = a.residual ? a.summed + t * a.summed_stride : x;
      const float factor = (float)(root_64 / (double)lean);
#pragma unroll 1
      for (int i = 0; i < kVecs * kWidth; ++i) {
        const int j = (i / kWidth * kThreads + tid) * kWidth + i % kWidth;
        if (j < whole * kWidth) out[j] = from_float<T>(to_float(from[j]) * lean * factor * to_float(a.weight[j]));
      }
      if (tid < rest) out[edge_at] = from_float<T>(edge * lean * factor * edge_w);
    }
  } else {
    double top = all.top;
    if (kExact && kKind == kNorm8 && !(all.top > 1e-30f && all.top < 1e30f)) {       // (the same for the whole workgroup)
      __shared__ double part[kThreads / 64];
      double mine = fabs((double)edge * (double)edge_w);
      for (int k = 0; k < kVecs; ++k) {
        float s[kWidth];
        v[k].get(s);
        for (int i = 0; i < kWidth; ++i) mine = fmax(mine, fabs((double)s[i] * (double)w[k][i]));
      }
      top = largest_all<kThreads>(mine, part);
    }
    float scale;
    const Rounding r = rounding_of(top, root_64, odd, &scale);
    if (tid == 0) a.scales[t] = scale;
    int8_t* q = a.q + t * a.q_stride;
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      if (k * kThreads + tid < whole) {
        float s[kWidth];
        uint32_t to[kWidth];
        v[k].get(s);
        to_8bit<kKind != kRows8>(s, w[k], r, odd, to);
        store_8bit<kWidth>(q + (k * kThreads + tid) * kWidth, to);
      }
    }
    if (tid < rest) {
      const float s[1] = {edge}, one[1] = {edge_w};
      uint32_t to[1];
      to_8bit<kKind != kRows8>(s, one, r, odd, to);
      q[edge_at] = (int8_t)to[0];
    }
  }
}

// The same for rows that no workgroup's registers hold: they are read twice, element by element, and summed in 64 bits.
template <typename T, typename W, int kKind>
__global__ void __launch_bounds__(1024) long_norm_kernel(NormArgs<T, W> a) {
  constexpr int kThreads = 1024;
  constexpr bool kEight = kKind != kNorm;
  __shared__ double part[kThreads / 64];
  const int64_t t = a.first + blockIdx.x;
  const T* x = a.x + t * a.stride;
  const T* residual = a.residual ? a.residual + t * a.residual_stride : nullptr;
  T* summed = a.residual ? a.summed + t * a.summed_stride : nullptr;
  double squares = 0.0;
  RowSums<double> sums{0.0f, 0.0f, 0.0};
  for (int j = threadIdx.x; j < a.dim; j += kThreads) {
    float s = to_float(x[j]);
    if (residual) {
      const T rounded = from_float<T>(s + to_float(residual[j]));
      summed[j] = rounded;
      s = to_float(rounded);
    }
    squares += (double)s * (double)s;
    if constexpr (kEight) {
      const float w = kKind == kRows8 ? 1.0f : to_float(a.weight[j]);
      sums.odd += (kKind == kRows8 ? s : w) * 0.0f;
      sums.top = fmax(sums.top, fabs((double)s * (double)w));
    }
  }
  const RowSums<double> all = join_sums<kThreads, kEight>(sums);
  bool odd = !(all.odd == 0.0f);
  double root = 1.0;
  if constexpr (kKind != kRows8) {
    squares = sum_all<kThreads>(squares, part);
    odd = odd || !(squares < INFINITY);
    root = 1.0 / sqrt(squares / (double)a.dim + (double)a.eps);
  }
  const T* from = residual ? summed : x;                     // (each thread reads what it has written itself)
  if constexpr (kKind == kNorm) {
    if (a.rstd && threadIdx.x == 0) a.rstd[t] = (float)root;
    T* out = a.out + t * a.out_stride;
    const auto store = [&](float lean, float factor) {
      for (int j = threadIdx.x; j < a.dim; j += kThreads) out[j] = from_float<T>(to_float(from[j]) * lean * factor * to_float(a.weight[j]));
    };
    const float lean = lean_of(root);
    if (lean == 1.0f) store(1.0f, (float)root);
    else store(lean, (float)(root / (double)lean));
  } else {
    float scale;
    const Rounding r = rounding_of(all.top, root, odd, &scale);
    if (threadIdx.x == 0) a.scales[t] = scale;
    int8_t* q = a.q + t * a.q_stride;
    for (int j = threadIdx.x; j < a.dim; j += kThreads) {
      const float s[1] = {to_float(from[j])}, w[1] = {kKind == kRows8 ? 1.0f : to_float(a.weight[j])};
      uint32_t to[1];
      to_8bit<true>(s, w, r, odd, to);
      q[j] = (int8_t)to[0];
    }
  }
}

template <typename T, typename W>
struct NormGradArgs {
  const T* grad;
  const T* summed;
  const W* weight;
  const float* rstd;
  const T* grad_summed;       // null: none
  T* grad_x;
  float* partial;             // [groups][dim]; null: not wanted
  int64_t grad_stride, summed_stride, grad_summed_stride, grad_x_stride, n;
  int dim, each;              // each: rows of a group
};

// A workgroup has `each` rows, one after another, and its columns' part of the weights' gradient in registers.
template <typename T, typename W, int kThreads, int kVecs>
__global__ void __launch_bounds__(kThreads) norm_grad_kernel(NormGradArgs<T, W> a) {
  constexpr int kWidth = Vec<T>::kWidth;
  __shared__ float part[2][kThreads / 64];
  const int tid = threadIdx.x, whole = a.dim / kWidth, rest = a.dim % kWidth, edge_at = whole * kWidth + tid;
  const int64_t begin = (int64_t)blockIdx.x * a.each, end = min(a.n, begin + a.each);
  float w[kVecs][kWidth], total[kVecs][kWidth], edge_w = 0.0f, edge_total = 0.0f;
#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
#pragma unroll
    for (int i = 0; i < kWidth; ++i) w[k][i] = total[k][i] = 0.0f;
    if (k * kThreads + tid < whole) load_weights<kWidth>(a.weight + (k * kThreads + tid) * kWidth, w[k]);
  }
  if (tid < rest) edge_w = to_float(a.weight[edge_at]);
  // A row's vectors, of which the next row's are on their way while this one's sum is joined.
  Vec<T> next_g[kVecs], next_s[kVecs], next_more[kVecs];
  float next_edge_g = 0.0f, next_edge_s = 0.0f, next_edge_more = 0.0f, next_r = 0.0f;
#pragma unroll
  for (int k = 0; k < kVecs; ++k) next_g[k] = next_s[k] = next_more[k] = Vec<T>::all(0.0f);
  const auto load = [&](int64_t t) {
    const T *grad = a.grad + t * a.grad_stride, *summed = a.summed + t * a.summed_stride;
    const T* more = a.grad_summed ? a.grad_summed + t * a.grad_summed_stride : nullptr;
    next_r = a.rstd[t];
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      if (k * kThreads + tid < whole) {
        next_g[k] = Vec<T>::load(grad + (k * kThreads + tid) * kWidth);
        next_s[k] = Vec<T>::load(summed + (k * kThreads + tid) * kWidth);
        if (more) next_more[k] = Vec<T>::load(more + (k * kThreads + tid) * kWidth);
      }
    }
    if (tid < rest) {
      next_edge_g = to_float(grad[edge_at]);
      next_edge_s = to_float(summed[edge_at]);
      if (more) next_edge_more = to_float(more[edge_at]);
    }
  };
  load(begin);
  for (int64_t t = begin; t < end; ++t) {
    Vec<T> g[kVecs], s[kVecs], more[kVecs];
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      g[k] = next_g[k];
      s[k] = next_s[k];
      more[k] = next_more[k];
    }
    const float r = next_r, edge_g = next_edge_g, edge_h = next_edge_s * r, edge_more = next_edge_more;
    if (t + 1 < end) load(t + 1);
    float dot = edge_g * edge_w * edge_h;
    edge_total = fmaf(edge_g, edge_h, edge_total);
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      float x[kWidth], h[kWidth];
      g[k].get(x);
      s[k].get(h);
#pragma unroll
      for (int i = 0; i < kWidth; ++i) {
        const float gh = x[i] * (h[i] * r);
        dot = fmaf(gh, w[k][i], dot);
        total[k][i] += gh;
      }
    }
    // (Two sets of parts in turn: a wave that is a row ahead does not write into what others still read.)
    const float mean = sum_all<kThreads>(dot, part[t & 1]) / (float)a.dim;
    T* grad_x = a.grad_x + t * a.grad_x_stride;
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      if (k * kThreads + tid < whole) {
        float x[kWidth], h[kWidth], add[kWidth];
        g[k].get(x);
        s[k].get(h);
        more[k].get(add);
#pragma unroll
        for (int i = 0; i < kWidth; ++i) x[i] = fmaf(r, x[i] * w[k][i] - h[i] * r * mean, add[i]);
        Vec<T>::of(x).store(grad_x + (k * kThreads + tid) * kWidth);
      }
    }
    if (tid < rest) grad_x[edge_at] = from_float<T>(fmaf(r, edge_g * edge_w - edge_h * mean, edge_more));
  }
  if (!a.partial) return;
  float* to = a.partial + (int64_t)blockIdx.x * a.dim;
#pragma unroll
  for (int k = 0; k < kVecs; ++k)
    if (k * kThreads + tid < whole)
      for (int i = 0; i < kWidth; i += 4)
        Vec<float>::of({total[k][i], total[k][i + 1], total[k][i + 2], total[k][i + 3]}).store(to + (k * kThreads + tid) * kWidth + i);
  if (tid < rest) to[edge_at] = edge_total;
}

// Rows that no workgroup's registers hold: the gradient of each row's elements, read twice and summed in 64 bits, ...  (An element a lane, and
// with the weights' part three times through: 4,096 rows of 12,288 bfloat16 249 us, of 5,120 in 32 bits 111, where four matrices at 5 TB/s
// would take 81 and 67.)
template <typename T, typename W>
__global__ void __launch_bounds__(1024) long_norm_grad_kernel(NormGradArgs<T, W> a, int64_t first) {
  constexpr int kThreads = 1024;
  __shared__ double part[kThreads / 64];
  const int64_t t = first + blockIdx.x;
  const T *grad = a.grad + t * a.grad_stride, *summed = a.summed + t * a.summed_stride;
  const T* more = a.grad_summed ? a.grad_summed + t * a.grad_summed_stride : nullptr;
  T* grad_x = a.grad_x + t * a.grad_x_stride;
  const float r = a.rstd[t];
  double dot = 0.0;
  for (int j = threadIdx.x; j < a.dim; j += kThreads) dot += (double)(to_float(grad[j]) * to_float(a.weight[j])) * (double)(to_float(summed[j]) * r);
  const float mean = (float)(sum_all<kThreads>(dot, part) / (double)a.dim);
  for (int j = threadIdx.x; j < a.dim; j += kThreads) {
    const float add = more ? to_float(more[j]) : 0.0f;
    grad_x[j] = from_float<T>(fmaf(r, to_float(grad[j]) * to_float(a.weight[j]) - to_float(summed[j]) * r * mean, add));
  }
}

// ... and, before it (grad_x may be grad), a group's part of the weights' gradient, one column a thread.
template <typename T, typename W>
__global__ void __launch_bounds__(256) long_norm_partial_kernel(NormGradArgs<T, W> a, int64_t first) {
  const int64_t group = first + blockIdx.y, begin = group * a.each, end = min(a.n, begin + a.each);
  const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (j >= a.dim) return;
  float total = 0.0f;
  for (int64_t t = begin; t < end; ++t) total = fmaf(to_float(a.grad[t * a.grad_stride + j]), to_float(a.summed[t * a.summed_stride + j]) * a.rstd[t], total);
  a.partial[group * a.dim + j] = total;
}

// The weights' gradient from the groups' parts, added in 64 bits: 64 columns a workgroup, four a lane, and every 64th group for each
// sixteen lanes, so that a thread's reads are few and side by side.
template <typename O>
__global__ void __launch_bounds__(1024) norm_weight_kernel(const float* partial, int64_t groups, int dim, int accumulate, unsigned first, O* grad_weight) {
  __shared__ double part[16][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t begin = ((int64_t)first + blockIdx.x) * 64, j = begin + lane % 16 * 4;
  double total[4] = {0.0, 0.0, 0.0, 0.0};
  constexpr int kDeep = 8;
  for (int64_t i = wave * 4 + lane / 16; i < groups && j < dim; i += 64 * kDeep) {
    float v[kDeep][4];
#pragma unroll
    for (int k = 0; k < kDeep; ++k) {
      const float* p = partial + (i + 64 * k) * dim + j;
      for (int c = 0; c < 4; ++c) v[k][c] = 0.0f;
      if (i + 64 * k < groups) {
        if (j + 4 <= dim) Vec<float>::load(p).get(v[k]);
        else
          for (int c = 0; c < 4; ++c)
            if (j + c < dim) v[k][c] = p[c];
      }
    }
#pragma unroll
    for (int k = 0; k < kDeep; ++k)
      for (int c = 0; c < 4; ++c) total[c] += (double)v[k][c];
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    total[c] += __shfl_xor(total[c], 16);
    total[c] += __shfl_xor(total[c], 32);
    if (lane < 16) part[wave][lane * 4 + c] = total[c];
  }
  __syncthreads();
  const int64_t column = begin + threadIdx.x;
  if (threadIdx.x < 64 && column < dim) {
    double sum = part[0][threadIdx.x];
    for (int w = 1; w < 16; ++w) sum += part[w][threadIdx.x];
    if (accumulate) sum += (double)to_float(grad_weight[column]);
    grad_weight[column] = from_float<O>((float)sum);
  }
}

}  // namespace bpe
