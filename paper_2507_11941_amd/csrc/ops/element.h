// Types of the matrices that the operators on token batches read and write: float, bfloat16, half.  Everything is computed in
// 32 bits; a result is rounded once, to nearest even, where it is stored.
//
// Rows are read and written 16 bytes a lane, whatever their address: rows of a vocabulary of 100,260 tokens begin at every multiple
// of 8 bytes, and a view may begin at any element.  The hardware takes such addresses in global memory.  What is only read, and rows
// of an embedding, are taken from their first element on; what writes a gradient takes a row's vectors from its first whole line on,
// with a head and a tail of single elements, as stores that pass the caches by have to write whole lines.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bpe {

typedef __bf16 bf16;
typedef _Float16 f16;

template <typename T>
__device__ inline float to_float(T x) { return (float)x; }

template <typename T>
__device__ inline T from_float(float x) { return (T)x; }

constexpr float kLog2e = 1.44269504088896340736f;

typedef uint32_t Words __attribute__((ext_vector_type(4)));

// The same at any multiple of kBytes.
template <int kBytes>
struct At;
template <>
struct At<2> {
  typedef uint32_t Type __attribute__((ext_vector_type(4), aligned(2)));
};
template <>
struct At<4> {
  typedef uint32_t Type __attribute__((ext_vector_type(4), aligned(4)));
};

template <bool kValue>
struct Constant {
  static constexpr bool value = kValue;
};

constexpr int kLine = 128;                                   // bytes of a cache line

// How many of n elements lie before the first whole line of kBytes.
template <int kBytes, typename T>
__device__ inline int head_of(const T* p, int64_t n) {
  return (int)min((int64_t)(-(uintptr_t)p % kBytes / sizeof(T)), n);
}

// 16 bytes of a row.
template <typename T>
struct Vec {
  static constexpr int kWidth = 16 / sizeof(T);
  Words w;

  // With kOnce the access passes the caches by, as far as it can: for what nobody reads again soon.  Stores only where waves write
  // whole lines: parts of one go to memory each by themselves.
  template <bool kOnce = false>
  __device__ static Vec load(const T* p) {
    typedef typename At<sizeof(T)>::Type Here;
    if constexpr (kOnce) return {__builtin_nontemporal_load((const Here*)p)};
    else return {*(const Here*)p};
  }
  template <bool kOnce = false>
  __device__ void store(T* p) const {
    typedef typename At<sizeof(T)>::Type Here;
    if constexpr (kOnce) __builtin_nontemporal_store(w, (Here*)p);
    else *(Here*)p = w;
  }
  __device__ void get(float (&x)[kWidth]) const {
    if constexpr (sizeof(T) == 4) {
      for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
    } else if constexpr (__is_same(T, bf16)) {
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    } else {
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = (float)__builtin_bit_cast(f16, (uint16_t)w[i]);
        x[2 * i + 1] = (float)__builtin_bit_cast(f16, (uint16_t)(w[i] >> 16));
      }
    }
  }
  __device__ static Vec of(const float (&x)[kWidth]) {
    Vec v;
    if constexpr (sizeof(T) == 4) {
      for (int i = 0; i < 4; ++i) v.w[i] = __float_as_uint(x[i]);
    } else {
      for (int i = 0; i < 4; ++i)
        v.w[i] = (uint32_t)__builtin_bit_cast(uint16_t, (T)x[2 * i]) | (uint32_t)__builtin_bit_cast(uint16_t, (T)x[2 * i + 1]) << 16;
    }
    return v;
  }
  // Every element the same.
  __device__ static Vec all(float x) {
    float v[kWidth];
    for (int i = 0; i < kWidth; ++i) v[i] = x;
    return of(v);
  }
};

// The larger of three.  (fmaxf first quiets each operand that the compiler cannot tell to be no signalling NaN, an instruction
// more for each logit.)
__device__ inline float max_of(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

}  // namespace bpe
