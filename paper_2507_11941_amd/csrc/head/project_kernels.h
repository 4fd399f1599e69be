// Logits from 8-bit rows and 8-bit weights: out[t][v] = scales[t] weight_scales[v] (sum over k of q[t][k] weight[v][k]).
//
// A workgroup has a tile of tokens x vocabulary and goes along the columns in steps of 128 bytes a row, which wait in shared memory in
// stages: while the matrix units work on one, the next are on their way.  The vocabulary is the matrix instruction's first operand,
// so that a lane holds four neighbours of a token's logits, and these go to memory through shared memory, 16 bytes a lane.
//
// Measured on one MI355X, whose matrix units reach 3.5e15 operations/s on random bytes (they, too, lower the clock):
//   8,191 tokens x 2,048 into 100,260 bfloat16   1,620 to 1,760 us by the card, 1.9e15 to 2.1e15/s; 8,192 x 4,096 into 32,768 940 to 1,005 us, 2.3e15/s
//   (torch's product with 32-bit sums written: 2,008 and 1,017 us)
//   the same into 32-bit logits                   1,965 us, of which their 3.3 GB are 660 at 5 TB/s
//   8 tokens x 4,096 into 100,260                 70 us, 5.9 TB/s: the reading of the weights; 32 x 8,192 into 50,000 71 us, 5.7 TB/s
// What the first of these spent at 1,700, by leaving parts out: products and readings of shared memory alone 1,130 us, with the stages' transfers
// (13 GB through the second-level caches, 960 us alone) 1,380, with the conversion of the logits 1,500, the rest their stores; rows of
// 100,260 begin at multiples of 8 bytes, and of 100,352 the stores take 120 less.  Stages of 64 bytes, four of them instead of two of 128: 1,800
// (twice the requests); two workgroups of half the tile: 3,400 (half as much again to transfer); stores past the caches: 2,070 (parts of lines);
// offsets of loads worked out for each step: 1,830.
#pragma once
#include "../ops/element.h"

namespace bpe {

typedef int Bytes16 __attribute__((ext_vector_type(4)));
typedef int Sums __attribute__((ext_vector_type(16)));

constexpr int kXcds = 8;
constexpr int kStep = 128;                                  // bytes of a row in a stage

struct ProjectArgs {
  const int8_t* q;
  const float* scales;
  const int8_t* weight;
  const float* weight_scales;
  int64_t n, vocab, q_stride, weight_stride, out_stride;
  int dim;
  unsigned token_tiles, tiles;                              // tiles: of the whole product
  int words;                                                // of a tile for few tokens, at most its size
};

// Which tile a workgroup has.  Workgroups go round the eight dies; each die takes a stretch of the tiles of its own, in which up to
// kBand tiles of tokens share a tile of the vocabulary while it is in the die's cache.
struct Tile {
  unsigned token, word;
};

constexpr unsigned kBand = 4;

__device__ inline Tile tile_of(unsigned block, unsigned token_tiles, unsigned tiles) {
  const unsigned die = block % kXcds, share = tiles / kXcds, more = tiles % kXcds;
  const unsigned i = die * share + min(die, more) + block / kXcds;
  const unsigned words = tiles / token_tiles, band = i / (kBand * words), height = min(kBand, token_tiles - band * kBand);
  const unsigned in = i - band * kBand * words;
  return {band * kBand + in % height, in / height};
}

// Waits until at most kLeft of this wave's transfers are on their way (they end in the order of their beginning), then for all waves.
template <int kLeft>
__device__ inline void wait_and_meet() {
  static_assert(kLeft < 64);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((kLeft & 15) | 7 << 4 | (kLeft >> 4) << 14);     // ... and for its accesses to shared memory
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// From memory into shared memory, 16 or 4 bytes a lane, one lane behind the other from `to` on.
template <int kBytes>
__device__ inline void transfer(const void* from, void* to) {
  static_assert(kBytes == 16 || kBytes == 4);
  const auto* source = (const __attribute__((address_space(1))) void*)from;
  auto* target = (__attribute__((address_space(3))) void*)to;
  if constexpr (kBytes == 16) __builtin_amdgcn_global_load_lds(source, target, 16, 0, 0);
  else __builtin_amdgcn_global_load_lds(source, target, 4, 0, 0);
}

// How far the chunks of 16 bytes of a row are turned.
__device__ inline int turn(int row) { return row >> 1 & 7; }

// 16 bytes at any address.
__device__ inline Bytes16 load_bytes(const int8_t* p) {
  typedef int Here __attribute__((ext_vector_type(4), aligned(1)));
  return *(const Here*)p;
}

// The 16 bytes from `at` on of a row of `dim`; zeros from its end on, behind which nothing is read: the row's last 16 bytes, shifted.
__device__ inline Bytes16 load_end(const int8_t* row, int at, int dim) {
  Bytes16 v = {0, 0, 0, 0};
  if (at + 16 <= dim) return load_bytes(row + at);
  if (at >= dim) return v;
  if (dim >= 16) {
    const unsigned __int128 last = __builtin_bit_cast(unsigned __int128, load_bytes(row + dim - 16));
    return __builtin_bit_cast(Bytes16, last >> (8 * (at + 16 - dim)));
  }
#pragma unroll 1
  for (int i = 0; i < dim; ++i) {                            // (a row of fewer than 16 bytes: at is 0)
    const int b = (int)((uint32_t)(uint8_t)row[i] << (8 * (i & 3)));
    v[0] |= i >> 2 == 0 ? b : 0;
    v[1] |= i >> 2 == 1 ? b : 0;
    v[2] |= i >> 2 == 2 ? b : 0;
    v[3] |= i >> 2 == 3 ? b : 0;
  }
  return v;
}

// Where a row ends within 16 bytes or before them, its last 16 are taken instead, of tokens and weights alike; of the tokens' those are
// cleared that the 16 before them have as well: the mask of a word of them.
__device__ inline int keeps(int cleared, int word) {
  const int bytes = cleared - 4 * word;
  return bytes >= 4 ? 0 : bytes <= 0 ? -1 : -1 << (8 * bytes);
}

// kMt x kVt tiles of 32 x 32 a wave (tokens x vocabulary), kWm x kWv waves; kStages stages.  With kDirect rows
// begin at multiples of 4 bytes and have a multiple of 4, at least 16, and go from memory into shared memory by themselves; else through
// registers.  A workgroup has tiles gridDim.x apart, and the stages go on from one to the next: while a tile's logits are written, the
// next one's first stages are on their way.  (Behind the last tile stages are fetched once more, and not used: the loop has no branches.)
template <typename T, int kMt, int kVt, int kWm, int kWv, int kStages, bool kDirect>
__global__ void __launch_bounds__(64 * kWm * kWv) project_kernel(ProjectArgs a, T* out) {
  constexpr int kWaves = kWm * kWv, kTokens = 32 * kMt * kWm, kWords = 32 * kVt * kWv;
  constexpr int kRows = kTokens + kWords, kStage = kRows * kStep;
  constexpr int kChunks = kStep / 16, kAtOnce = 64 / kChunks, kLoads = kRows / kAtOnce / kWaves;      // chunks of a row; rows of a load
  constexpr int kParts = kStep / 32, kSets = kDirect ? 2 : 1;      // parts of a step: products of 32 bytes of each row
  static_assert(kRows % (kAtOnce * kWaves) == 0 && (kDirect || kStages == 2));
  constexpr int kOutTokens = kMt * kVt >= 8 ? 32 : 16;       // whose logits are in a wave's corner at once: what there is room for
  constexpr int kOutRow = 64 + 16;                           // 64 bytes of a token's logits, and room between rows
  constexpr int kStores = kMt * kVt * (int)sizeof(T);        // of a tile, by each wave
  constexpr int kScales = (kRows + 63) / 64 * 64, kScaleSets = kStages + 1;      // (with one step a tile, a wave may be at the one before)
  // (One array: of several the compiler knows which of them a transfer writes, and has every reading of that wait for it.)
  __shared__ __attribute__((aligned(16))) int8_t stages[kStages * kStage + kWaves * kOutTokens * kOutRow + kScaleSets * kScales * 4];
  int8_t* const corners = stages + kStages * kStage;
  float* const tile_scales = (float*)(corners + kWaves * kOutTokens * kOutRow);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wave_token = wave / kWv * (32 * kMt), wave_word = wave % kWv * (32 * kVt);
  const int steps = (a.dim + kStep - 1) / kStep, ragged = a.dim % kStep ? steps - 1 : -1;
  const int words = kTokens == 32 ? a.words : kWords;        // (few tokens: as many as share the work evenly)
  const unsigned mine = (a.tiles - blockIdx.x + gridDim.x - 1) / gridDim.x;
  // Workgroups begin at different columns, by thirty-seconds of a row, and go round: all at the same columns of rows of 4,096 bytes would
  // ask the same parts of memory at once.  Tiles of 64 x 64 for 8 tokens x 4,096 into 100,260: 84 us -> 76; 32 x 8,192 into 50,000: 94 -> 84;
  // of 256 x 256 for 4,096 x 4,096 into 65,536: 993 -> 960; 8,191 x 2,048 into 100,260: 1,680 -> 1,630.  (Small tiles with the large ones' places
  // 76, 87; large ones with the small ones' 980, 1,650.)
  const unsigned die = blockIdx.x % kXcds, begin = kMt * kVt >= 8 ? die * 4 + blockIdx.x / kXcds % 4 : die % 4 * 8;
  const int first_step = (int)(begin * (unsigned)steps / 32);

  // Loading.  The 16 bytes c of row r lie at place c ^ turn(r): shared memory serves sixteen lanes at a time from 64 banks, and so sixteen
  // rows of the same columns lie in 256 bytes once.
  // A load is of tokens or of weights alone, and, where the numbers of rows allow it, all of a wave's are.
  constexpr int kOwn = kRows / kWaves;
  constexpr bool kMixed = kTokens % kOwn != 0;
  static_assert(kTokens % kAtOnce == 0);
  const auto of_tokens = [&](int i) { return wave * kOwn + (kMixed ? i * kAtOnce : 0) < kTokens; };
  const int in_load = lane / kChunks;
  const auto place = [&](int i) { return ((lane % kChunks) ^ turn(wave * kOwn + i * kAtOnce + in_load)) * 16; };
  const int8_t* from[kMixed ? 2 : 1];                        // the tile's first row, of tokens and of weights or of this wave's
  const auto first_row = [&](int i) { return kMixed && !of_tokens(i) ? from[kMixed] : from[0]; };
  uint32_t offset[kLoads];                                   // of each load's row and this lane's place in it, from there
  Bytes16 held[kDirect ? 1 : kLoads];
  unsigned fetch_tile = 0;
  int fetch_step = first_step, fetch_stage = 0;
  const auto begin_fetch = [&] {
    if (fetch_step != first_step || fetch_tile >= mine) return;
    const Tile tile = tile_of(blockIdx.x + fetch_tile * gridDim.x, a.token_tiles, a.tiles);
    const int64_t token = (int64_t)tile.token * kTokens, word = (int64_t)tile.word * words;
    from[0] = kMixed || of_tokens(0) ? a.q + token * a.q_stride : a.weight + word * a.weight_stride;
    if (kMixed) from[kMixed] = a.weight + word * a.weight_stride;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {                       // (rows behind the last: the last once more, nobody stores their logits)
      const int64_t last = (of_tokens(i) ? a.n - token : min((int64_t)words, a.vocab - word)) - 1;
      const uint32_t stride = (uint32_t)(of_tokens(i) ? a.q_stride : a.weight_stride);
      offset[i] = (uint32_t)min((int64_t)(wave * kOwn - (of_tokens(i) ? 0 : kTokens) + in_load + i * kAtOnce), last) * stride + (uint32_t)place(i);
    }
    for (int i = wave * 64; i < kRows; i += kWaves * 64) {
      const int row = i + lane;
      const float* p = row < kTokens ? a.scales + min(token + row, a.n - 1) : a.weight_scales + min(word + row - kTokens, a.vocab - 1);
      transfer<4>(p, tile_scales + fetch_tile % kScaleSets * kScales + i);
    }
  };
  const auto fetch = [&] {
    int8_t* to = stages + fetch_stage * kStage + wave * kLoads * 1024;
    if (fetch_step != ragged) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        if constexpr (kDirect) transfer<16>(first_row(i) + fetch_step * kStep + offset[i], to + i * 1024);
        else held[i] = load_bytes(first_row(i) + fetch_step * kStep + offset[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int at = fetch_step * kStep + place(i);
        if constexpr (kDirect) transfer<16>(first_row(i) + (offset[i] - (uint32_t)place(i) + (uint32_t)min(at, a.dim - 16)), to + i * 1024);
        else held[i] = load_end(first_row(i) + (offset[i] - (uint32_t)place(i)), at, a.dim);
        if constexpr (!kDirect) __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  const auto end_fetch = [&] {
    if (++fetch_step == steps) fetch_step = 0;
    if (fetch_step == first_step) ++fetch_tile;
    fetch_stage = fetch_stage + 1 == kStages ? 0 : fetch_stage + 1;
  };
  const auto commit = [&](int stage) {
    if constexpr (!kDirect) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) *(Bytes16*)(stages + stage * kStage + (wave * kLoads + i) * 1024 + lane * 16) = held[i];
    }
  };

  Sums sums[kMt][kVt];
#pragma unroll
  for (int m = 0; m < kMt; ++m)
#pragma unroll
    for (int v = 0; v < kVt; ++v) sums[m][v] = Sums{};

  // The operands of a part, in two sets in turn (where registers have room): while one is multiplied, the next is read, also over the
  // end of a stage.
  const int row = lane & 31, half = lane >> 5;
  Bytes16 x[kSets][kMt], w[kSets][kVt];
  const auto read = [&](int stage, int part) {
    const int8_t* here = stages + stage * kStage + row * kStep + ((2 * part + half) ^ turn(row)) * 16;
#pragma unroll
    for (int v = 0; v < kVt; ++v) w[part % kSets][v] = *(const Bytes16*)(here + (kTokens + wave_word + v * 32) * kStep);
#pragma unroll
    for (int m = 0; m < kMt; ++m) x[part % kSets][m] = *(const Bytes16*)(here + (wave_token + m * 32) * kStep);
  };

#pragma unroll 1
  for (int s = 0; s < (kDirect ? kStages : kStages - 1); ++s) {
    begin_fetch();
    fetch();
    commit(s);
    end_fetch();
  }
  if constexpr (kDirect) {
    wait_and_meet<(kStages - 1) * kLoads>();
    read(0, 0);
  } else {
    wait_and_meet<0>();
  }
  int stage = 0, stored = 0;                                 // stored: of how many steps to come the stages are older than a whole tile's stores
  for (unsigned t = 0; t < mine; ++t) {
    const Tile tile = tile_of(blockIdx.x + t * gridDim.x, a.token_tiles, a.tiles);
    const int64_t token = (int64_t)tile.token * kTokens, word = (int64_t)tile.word * words;
#pragma unroll 1
    for (int count = 0, step = first_step; count < steps; ++count, step = step + 1 == steps ? 0 : step + 1) {
      const int next = stage + 1 == kStages ? 0 : stage + 1;
      if constexpr (!kDirect) begin_fetch();
#pragma unroll
      for (int part = 0; part < kParts; ++part) {
        if (kDirect && part + 1 < kParts) {
          read(stage, part + 1);
        } else if (kDirect) {
          // The next stage has come when all but the later ones' transfers have ended, and a tile's stores that came after those.  Then
          // all waves have read this one, whose place the stage after the last takes.
          if (stored > 0) wait_and_meet<(kStages - 2) * kLoads + kStores>();
          else wait_and_meet<(kStages - 2) * kLoads>();
          stored = stored > 0 ? stored - 1 : 0;
          read(next, 0);
          begin_fetch();
        } else {
          read(stage, part);
          if (part == 0) fetch();
        }
        __builtin_amdgcn_sched_barrier(0);
        if (kDirect && step == ragged) {                     // (nowhere, where rows fill their last step)
          const int cleared = step * kStep + (2 * part + half) * 16 + 16 - a.dim;
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int m = 0; m < kMt; ++m) x[part % kSets][m][i] &= keeps(cleared, i);
        }
#pragma unroll
        for (int m = 0; m < kMt; ++m)
#pragma unroll
          for (int v = 0; v < kVt; ++v) sums[m][v] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[part % kSets][v], x[part % kSets][m], sums[m][v], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        if (kDirect && part == kParts - 1) {                 // (behind the products: a wave waits while memory takes its transfers)
          fetch();
          end_fetch();
        }
      }
      if constexpr (!kDirect) {
        commit(next);
        end_fetch();
        wait_and_meet<0>();
      }
      stage = next;
    }

    // Element 4 g + j of sums: vocabulary 8 g + 4 half + j, token `row` of 32 x 32.  A wave's logits go through a corner of shared
    // memory of its own, 64 bytes of some tokens at a time; its accesses are in order by themselves.
    const float* scales = tile_scales + t % kScaleSets * kScales;
    int8_t* corner = corners + wave * kOutTokens * kOutRow;
    const bool whole = token + kTokens <= a.n && words == kWords && word + kWords <= a.vocab;
    constexpr int kWidth = Vec<T>::kWidth, kEights = 8 / (int)sizeof(T);           // groups of eight words in 64 bytes
#pragma unroll
    for (int m = 0; m < kMt; ++m) {
      const float scale = scales[wave_token + 32 * m + row];
#pragma unroll
      for (int first = 0; first < 4 * kVt; first += kEights) {
#pragma unroll
        for (int part = 0; part < 32 / kOutTokens; ++part) {
          if (kOutTokens == 32 || row / kOutTokens == part) {
#pragma unroll
            for (int i = 0; i < kEights; ++i) {
              const int v = (first + i) / 4, g = (first + i) % 4;
              const Words of = *(const Words*)(scales + kTokens + wave_word + 32 * v + 8 * g + 4 * half);
              float y[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) y[j] = (float)sums[m][v][4 * g + j] * scale * __uint_as_float(of[j]);
              T* p = (T*)(corner + row % kOutTokens * kOutRow) + 8 * i + 4 * half;
              if constexpr (sizeof(T) == 4) {
                *(Words*)p = Vec<float>::of(y).w;
              } else {
                typedef T Four __attribute__((ext_vector_type(4)));
                *(Four*)p = Four{from_float<T>(y[0]), from_float<T>(y[1]), from_float<T>(y[2]), from_float<T>(y[3])};
              }
            }
          }
          // (Lanes read what others have written: the compiler is not to keep what a lane has read before.)
          asm volatile("" ::: "memory");
#pragma unroll
          for (int i = 0; i < kOutTokens / 16; ++i) {
            const int r = lane / 4 + 16 * i, column = wave_word + 8 * first + lane % 4 * kWidth;
            Vec<T> y;
            y.w = *(const Words*)(corner + r * kOutRow + lane % 4 * 16);
            const int64_t to = token + wave_token + 32 * m + kOutTokens * part + r;
            T* p = out + to * a.out_stride + word + column;
            if (whole) {
              y.store(p);
            } else if (to < a.n) {
              float z[kWidth];
              y.get(z);
              const int64_t left = min((int64_t)words, a.vocab - word) - column;
              if (left >= kWidth) y.store(p);
              else
                for (int j = 0; j < kWidth; ++j)
                  if (j < left) p[j] = from_float<T>(z[j]);
            }
          }
          asm volatile("" ::: "memory");
        }
      }
#pragma unroll
      for (int v = 0; v < kVt; ++v) sums[m][v] = Sums{};
    }
    stored = whole ? kStages - 1 : 0;                        // (stages that were on their way before these stores)
  }
  wait_and_meet<0>();                                        // (nothing may come into shared memory when it is another workgroup's)
}

}  // namespace bpe
