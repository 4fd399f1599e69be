// Types of the matrices that the operators on token batches read and write: float, bfloat16, half.  Everything is computed in
// 32 bits; a result is rounded once, to nearest even, where it is stored.
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

}  // namespace bpe
