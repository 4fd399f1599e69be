// Logits from 8-bit rows and 8-bit weights: out[t][v] = scales[t] weight_scales[v] (sum over k of q[t][k] weight[v][k]).
//
// A workgroup has a tile of tokens x vocabulary and goes along the columns in steps of 128 bytes a row, which wait in shared memory in
// stages: while the matrix units work on one, the next are on their way.  The vocabulary is the matrix instruction's first operand,
// so that a lane holds four neighbours of a token's logits, and the tile goes to memory through shared memory, 16 bytes a lane.
#pragma once
#include "../ops/element.h"

namespace bpe {

typedef int Bytes16 __attribute__((ext_vector_type(4)));
typedef int Sums __attribute__((ext_vector_type(16)));

constexpr int kStep = 128;                                  // bytes of a row in a stage
constexpr int kXcds = 8;

__device__ __attribute__((aligned(16))) const uint32_t kZeros[4] = {0, 0, 0, 0};

struct ProjectArgs {
  const int8_t* q;
  const float* scales;
  const int8_t* weight;
  const float* weight_scales;
  int64_t n, vocab, q_stride, weight_stride, out_stride;
  int dim;
  unsigned token_tiles, tiles;                              // tiles: of the whole product
};

// Which tile a workgroup has.  Workgroups go round the eight dies; each die takes a stretch of the tiles of its own, in which up to
// kBand tiles of tokens share a tile of the vocabulary while it is in the die's cache.
struct Tile {
  unsigned token, word;
};

constexpr unsigned kBand = 8;

__device__ inline Tile tile_of(unsigned block, unsigned token_tiles, unsigned tiles) {
  const unsigned die = block % kXcds, share = tiles / kXcds, more = tiles % kXcds;
  const unsigned i = die * share + min(die, more) + block / kXcds;
  const unsigned words = tiles / token_tiles, band = i / (kBand * words), height = min(kBand, token_tiles - band * kBand);
  const unsigned in = i - band * kBand * words;
  return {band * kBand + in % height, in / height};
}

template <int kLeft>
__device__ inline void wait_and_meet() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLeft) : "memory");
}

// 16 bytes at any address.
__device__ inline Bytes16 load_bytes(const int8_t* p) {
  typedef int Here __attribute__((ext_vector_type(4), aligned(1)));
  return *(const Here*)p;
}

// The first `valid` of them, and zeros.
__device__ inline Bytes16 load_some_bytes(const int8_t* p, int valid) {
  if (valid >= 16) return load_bytes(p);
  Bytes16 v = {0, 0, 0, 0};
  for (int w = 0; w < 4; ++w)
    for (int i = 0; i < 4; ++i)
      if (4 * w + i < valid) v[w] |= (int)((uint32_t)(uint8_t)p[4 * w + i] << (8 * i));
  return v;
}

// kMt x kVt tiles of 32 x 32 a wave (tokens x vocabulary), kWm x kWv waves.  With kDirect rows begin at multiples of 16 bytes and go
// from memory into shared memory by themselves (all but a last step whose bytes are no multiple of 16); else through registers.
template <typename T, int kMt, int kVt, int kWm, int kWv, int kStages, bool kDirect>
__global__ void __launch_bounds__(64 * kWm * kWv) project_kernel(ProjectArgs a, T* out) {
  constexpr int kWaves = kWm * kWv, kThreads = 64 * kWaves, kTokens = 32 * kMt * kWm, kWords = 32 * kVt * kWv;
  constexpr int kRows = kTokens + kWords, kLoads = kRows / 8 / kWaves, kStage = kRows * kStep;
  static_assert(kRows % (8 * kWaves) == 0 && kTokens % 8 == 0);
  constexpr int kWidth = Vec<T>::kWidth, kOutRow = kWords * (int)sizeof(T) + 16, kOutBytes = 32 * kWm * kOutRow;
  __shared__ __attribute__((aligned(16))) int8_t shared[kStages * kStage > kOutBytes ? kStages * kStage : kOutBytes];
  const Tile tile = tile_of(blockIdx.x, a.token_tiles, a.tiles);
  const int64_t token = (int64_t)tile.token * kTokens, word = (int64_t)tile.word * kWords;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wave_token = wave / kWv * (32 * kMt), wave_word = wave % kWv * (32 * kVt);

  // Loading: a wave's instruction has eight rows of a stage.  The 16 bytes c of row r lie at place c ^ (r & 7) of the row, so that eight
  // lanes that read the same columns of eight rows meet all banks once.
  const int8_t* from[kLoads];
  const int chunk = (lane & 7) ^ (lane >> 3);
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int row = (wave * kLoads + i) * 8 + (lane >> 3);   // (rows behind the last are the last once more: nobody stores their logits)
    if (row < kTokens) from[i] = a.q + min(token + row, a.n - 1) * a.q_stride + chunk * 16;
    else from[i] = a.weight + min(word + row - kTokens, a.vocab - 1) * a.weight_stride + chunk * 16;
  }
  Bytes16 held[kDirect ? 1 : kLoads];
  const auto fetch = [&](int step) {
    int8_t* to = shared + step % kStages * kStage + wave * kLoads * 1024;
    const int left = a.dim - step * kStep - chunk * 16;      // bytes of the row from this lane's on
    if (a.dim - step * kStep >= kStep) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        if constexpr (kDirect)
          __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from[i] + step * kStep),
                                           (__attribute__((address_space(3))) void*)(to + i * 1024), 16, 0, 0);
        else held[i] = load_bytes(from[i] + step * kStep);
      }
    } else {
      if (kDirect && a.dim % 16 == 0) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int8_t* p = left > 0 ? from[i] + step * kStep : (const int8_t*)kZeros;
          __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p,
                                           (__attribute__((address_space(3))) void*)(to + i * 1024), 16, 0, 0);
        }
      } else {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const Bytes16 v = load_some_bytes(from[i] + step * kStep, left);
          if constexpr (kDirect) *(Bytes16*)(to + i * 1024 + lane * 16) = v;
          else held[i] = v;
        }
      }
    }
  };
  const auto commit = [&](int step) {
    if constexpr (!kDirect) {
      int8_t* to = shared + step % kStages * kStage + wave * kLoads * 1024 + lane * 16;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) *(Bytes16*)(to + i * 1024) = held[i];
    }
  };

  Sums sums[kMt][kVt];
#pragma unroll
  for (int m = 0; m < kMt; ++m)
#pragma unroll
    for (int v = 0; v < kVt; ++v) sums[m][v] = Sums{};

  const int steps = (a.dim + kStep - 1) / kStep;
  const int row = lane & 31, half = lane >> 5;
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s)
    if (s < steps) {
      fetch(s);
      commit(s);
    }
  for (int step = 0; step < steps; ++step) {
    if (!kDirect || kStages == 2 || step + kStages - 2 >= steps) wait_and_meet<0>();
    else wait_and_meet<(kStages - 2) * kLoads>();
    const bool more = step + kStages - 1 < steps;
    if (more) fetch(step + kStages - 1);
    const int8_t* stage = shared + step % kStages * kStage;
    const int8_t *tokens = stage + (wave_token + row) * kStep, *words = stage + (kTokens + wave_word + row) * kStep;
#pragma unroll
    for (int k = 0; k < kStep / 32; ++k) {
      const int at = ((2 * k + half) ^ (lane & 7)) * 16;
      Bytes16 t[kMt], w[kVt];
#pragma unroll
      for (int m = 0; m < kMt; ++m) t[m] = *(const Bytes16*)(tokens + m * 32 * kStep + at);
#pragma unroll
      for (int v = 0; v < kVt; ++v) w[v] = *(const Bytes16*)(words + v * 32 * kStep + at);
#pragma unroll
      for (int m = 0; m < kMt; ++m)
#pragma unroll
        for (int v = 0; v < kVt; ++v) sums[m][v] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[v], t[m], sums[m][v], 0, 0, 0);
    }
    if (more) commit(step + kStages - 1);
  }

  // Element 4 g + j of sums: vocabulary 8 g + 4 half + j, token `row` of the tile of 32 x 32.
  float word_scale[kVt][16];
#pragma unroll
  for (int v = 0; v < kVt; ++v)
#pragma unroll
    for (int i = 0; i < 16; ++i)
      word_scale[v][i] = a.weight_scales[min(word + wave_word + 32 * v + 8 * (i / 4) + 4 * half + i % 4, a.vocab - 1)];
  const int columns = (int)min((int64_t)kWords, a.vocab - word);
#pragma unroll
  for (int m = 0; m < kMt; ++m) {
    const float scale = a.scales[min(token + wave_token + 32 * m + row, a.n - 1)];
    __syncthreads();
    int8_t* to = shared + (wave / kWv * 32 + row) * kOutRow;
#pragma unroll
    for (int v = 0; v < kVt; ++v) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        T* p = (T*)to + wave_word + 32 * v + 8 * g + 4 * half;
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = (float)sums[m][v][4 * g + j] * scale * word_scale[v][4 * g + j];
        if constexpr (sizeof(T) == 4) {
          *(Words*)p = Vec<float>::of(x).w;
        } else {
          typedef T Four __attribute__((ext_vector_type(4)));
          *(Four*)p = Four{from_float<T>(x[0]), from_float<T>(x[1]), from_float<T>(x[2]), from_float<T>(x[3])};
        }
      }
    }
    __syncthreads();
    constexpr int kVecs = kWords / kWidth, kAtOnce = kThreads / kVecs;
    static_assert(kThreads % kVecs == 0);
    const int column = threadIdx.x % kVecs * kWidth;
#pragma unroll
    for (int r = 0; r < 32 * kWm; r += kAtOnce) {
      const int here = r + (int)threadIdx.x / kVecs;
      const int64_t t = token + here / 32 * (32 * kMt) + 32 * m + here % 32;
      if (here < 32 * kWm && t < a.n && column < columns) {
        Vec<T> v;
        v.w = *(const Words*)(shared + here * kOutRow + column * (int)sizeof(T));
        T* p = out + t * a.out_stride + word + column;
        if (column + kWidth <= columns) v.store(p);
        else {
          float x[kWidth];
          v.get(x);
          for (int i = 0; i < kWidth; ++i)
            if (column + i < columns) p[i] = from_float<T>(x[i]);
        }
      }
    }
  }
}

}  // namespace bpe
