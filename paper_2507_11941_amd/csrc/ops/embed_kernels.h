// Rows of an embedding, and their gradient.
#pragma once
#include <type_traits>

#include "element.h"
#include "sort_tokens.h"

namespace bpe {

__device__ inline int64_t rows_in_use(int64_t n, const int64_t* count) {
  return count ? min(n, max(*count, (int64_t)0)) : n;
}

// A lookup: a wave copies up to kVecs x 64 vectors of one row; a row takes `parts` waves.  Bound by memory: 40,961 rows of 2,048
// bfloat16 of an embedding of 132 MB, which the last-level cache holds, in 36 us, 9.3 TB/s read and written
// (42 us where what it writes takes that cache's place).
template <typename T, int kVecs>
__global__ void __launch_bounds__(256) embed_kernel(const T* weight, int64_t vocab, int64_t dim, int64_t weight_stride,
                                                    const int32_t* ids, int64_t first, int64_t n, unsigned parts, const int64_t* count,
                                                    float scale, T* out, int64_t out_stride, bool once) {
  constexpr int kWidth = Vec<T>::kWidth;
  const unsigned wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  const int64_t t = first + wave / parts, begin = (int64_t)(wave % parts) * (kVecs * 64 * kWidth);
  if (t >= rows_in_use(n, count)) return;
  const int32_t id = ids[t];
  const bool kept = id >= 0 && id < vocab;
  const int lane = threadIdx.x & 63;
  const int whole = (int)min((dim - begin) / kWidth, (int64_t)(kVecs * 64));
  const int64_t last = begin + whole * kWidth + lane;       // one of those behind the whole vectors
  const bool has_last = whole < kVecs * 64 && last < dim;
  const T* from = weight + (kept ? id : 0) * weight_stride;
  T* to = out + t * out_stride;
  Vec<T> v[kVecs];
  if (!kept) {
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
      if (k * 64 + lane < whole) Vec<T>::all(0.0f).store(to + begin + (k * 64 + lane) * kWidth);
    if (has_last) to[last] = from_float<T>(0.0f);
    return;
  }
#pragma unroll
  for (int k = 0; k < kVecs; ++k)
    if (k * 64 + lane < whole) v[k] = Vec<T>::load(from + begin + (k * 64 + lane) * kWidth);
  if (has_last) to[last] = from_float<T>(scale * to_float(from[last]));
  const auto write = [&](auto pass_by) {
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
      if (k * 64 + lane < whole) {
        float x[kWidth];
        v[k].get(x);
#pragma unroll
        for (int i = 0; i < kWidth; ++i) x[i] *= scale;
        Vec<T>::of(x).template store<pass_by.value>(to + begin + (k * 64 + lane) * kWidth);
      }
  };
  if (once) write(Constant<true>{});
  else write(Constant<false>{});
}

// ---- the gradient --------------------------------------------------------------------------------------------
//
// Positions come sorted by token, so that a token's rows are one run.  A wave has the runs of one chunk of up to 32 positions
// in 64 x (16 bytes) of the columns: a run belongs to the chunk in which it begins and is summed by its wave alone, also where
// it goes on into the next chunk, if it is no longer than a chunk.  A longer run is summed in pieces, one for each chunk that it
// touches, in 32 bits in the workspace, and another kernel adds those.  Which rows are added in which order follows from the
// sorted ids alone.
//
// Bound by memory: 65,536 rows of 2,048 bfloat16 into 100,260 rows of 32 bits, 1.08 GB, take 195 to 205 us (5.3 to 5.6 TB/s) after 26 us
// of sorting, and 10 us for the 184 tokens that have more than 32 rows.  Clearing the rows that no id names while the sort waits, before
// the sums, or between them changed nothing beyond 1 %: reads that follow 0.7 GB of writes wait for these to leave the caches.

constexpr int kChunk = 32;                                   // positions of a chunk at most: a wave's lanes hold it and the next

struct GradArgs {
  const uint32_t* keys;
  const uint32_t* positions;
  int64_t n;
  uint32_t vocab;
  int chunk;                                                 // positions of a chunk
  int64_t chunks;
  int64_t dim;
  unsigned tiles;                                            // of the columns
  int64_t grad_stride, out_stride;
  float scale;
  int accumulate;
  bool once;                                                 // grad's rows pass the caches by
  const uint8_t* present;                                    // whether there is a token; not used where it is accumulated
  uint32_t* long_runs;                                       // their number, cleared by the sort; then the chunks they begin in
  float* pieces;                                             // [chunks][2][dim]: of a run from before, of one that goes on
};

// A lane's columns: kWidth of them from `load` on.  Where a row does not end with a whole vector its last vector begins earlier,
// and the lane keeps only the columns from `own` on.  Rows narrower than a vector are one lane's, element by element.
struct Columns {
  int64_t load, own, end;
};

template <typename T>
__device__ inline Columns columns_of(int64_t tile, int64_t dim) {
  constexpr int kWidth = Vec<T>::kWidth;
  const int64_t own = (tile * 64 + (threadIdx.x & 63)) * kWidth;
  return {max((int64_t)0, min(own, dim - kWidth)), own, min(own + kWidth, dim)};
}

template <typename T, bool kOnce>
__device__ inline Vec<T> load_columns(const T* row, const Columns& c, int64_t dim) {
  if constexpr (kOnce) return Vec<T>::template load<true>(row + c.load);
  if (dim >= Vec<T>::kWidth) return Vec<T>::load(row + c.load);
  float x[Vec<T>::kWidth] = {};
  for (int i = 0; i < Vec<T>::kWidth; ++i)
    if (i < dim) x[i] = to_float(row[i]);
  return Vec<T>::of(x);
}

template <int kWidth, typename O>
__device__ inline void store_columns(O* row, const Columns& c, const float (&sum)[kWidth], float scale, int accumulate) {
  if (c.own >= c.end) return;
  if (c.load == c.own && c.end - c.own == kWidth) {
    float x[kWidth];
#pragma unroll
    for (int i = 0; i < kWidth; ++i) x[i] = scale * sum[i];
    constexpr int kOut = Vec<O>::kWidth;
#pragma unroll
    for (int h = 0; h < kWidth / kOut; ++h) {
      float y[kOut];
      if (accumulate) Vec<O>::load(row + c.own + h * kOut).get(y);
#pragma unroll
      for (int i = 0; i < kOut; ++i) y[i] = accumulate ? y[i] + x[h * kOut + i] : x[h * kOut + i];
      Vec<O>::of(y).store(row + c.own + h * kOut);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kWidth; ++i) {
    const int64_t col = c.load + i;
    if (col >= c.own && col < c.end) row[col] = from_float<O>((accumulate ? to_float(row[col]) : 0.0f) + scale * sum[i]);
  }
}

constexpr int kClear = 1024;                                 // vectors of a workgroup that clears

// Clears what there is of rows that no id names in one stretch of the matrix, whose last vector of a row may be a part of one.
// Workgroups that follow each other have stretches that do, 16 KiB each, as memory likes it best: 821 MB took 125 to 129 us for
// rows of 0.5, 2 and 8 KiB, with 4, 8 or 32 KiB each 150 to 170, with whole rows for a wave 118 to 150, with some rows each 150 to 180.
template <typename O>
__device__ inline void clear_stretch(O* out, const GradArgs& a, int64_t stretch) {
  constexpr int kOut = Vec<O>::kWidth;
  const uint32_t row_vecs = (uint32_t)((a.dim + kOut - 1) / kOut);
  const int64_t first_row = stretch * kClear / row_vecs;
  const uint32_t first = (uint32_t)(stretch * kClear - first_row * row_vecs);
  int64_t row[kClear / 256], column[kClear / 256];
  bool absent[kClear / 256];
#pragma unroll
  for (int k = 0; k < kClear / 256; ++k) {                   // (asked for side by side)
    const uint32_t at = first + k * 256 + threadIdx.x;
    row[k] = first_row + at / row_vecs;
    column[k] = (int64_t)(at % row_vecs) * kOut;
    absent[k] = row[k] < a.vocab;
    if (a.n > 0) absent[k] = !a.present[min(row[k], (int64_t)a.vocab - 1)] && absent[k];
  }
#pragma unroll
  for (int k = 0; k < kClear / 256; ++k) {
    if (!absent[k]) continue;
    O* to = out + row[k] * a.out_stride + column[k];
    if (column[k] + kOut <= a.dim)
      Vec<O>::all(0.0f).store(to);
    else
      for (int i = 0; i < (int)(a.dim - column[k]); ++i) to[i] = from_float<O>(0.0f);
  }
}

// The first `summing` workgroups sum, a wave a chunk in a tile of the columns, eight rows in flight; the others clear.
template <typename T, typename O>
__global__ void __launch_bounds__(256) embed_grad_kernel(const T* grad, O* out, GradArgs a, int64_t first, int64_t summing) {
  constexpr int kWidth = Vec<T>::kWidth, kDeep = 8;
  const int64_t group = first + blockIdx.x;
  if (group >= summing) return clear_stretch(out, a, group - summing);
  const int64_t wave = group * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int64_t c = wave / a.tiles, tile = wave % a.tiles, begin = c * a.chunk;
  if (begin >= a.n) return;
  const int size = (int)min((int64_t)a.chunk, a.n - begin);
  // Lane i: the chunk's position i, up to the next chunk's last; and the position a chunk before it.
  const int64_t mine = begin + lane;
  const bool in_reach = mine < a.n && lane < 2 * a.chunk;
  const uint32_t key = in_reach ? a.keys[mine] : 0xffffffffu;
  const uint32_t position = in_reach ? a.positions[mine] : 0u;
  const uint32_t earlier = lane < a.chunk && mine >= a.chunk ? a.keys[mine - a.chunk] : 0xffffffffu;
  const uint32_t first_key = __builtin_amdgcn_readlane(key, 0);
  if (first_key >= a.vocab) return;                          // nothing but padding from here on
  const Columns cols = columns_of<T>(tile, a.dim);
  float* head = a.pieces + 2 * c * a.dim;
  float* tail = head + a.dim;
  // What is ours: from `from` to `to` (numbers of lanes), the first `head_end` of it a piece of a run from before.
  int from = 0, head_end = 0;
  const uint64_t same = __ballot(key == first_key);
  const int first_end = (int)__builtin_ctzll(~same | ((uint64_t)1 << 63));        // where the first run ends, in reach
  if (begin > 0 && __builtin_amdgcn_readlane(earlier, a.chunk - 1) == first_key) {
    // how many of the positions before belong to it, up to a chunk
    const uint64_t back = __ballot(earlier == first_key) << (64 - a.chunk);
    const int before = (int)__builtin_clzll(~back);
    // It is long if its position number `chunk` exists: that many from its beginning, which may be before all we see.
    if (before >= a.chunk || first_end > a.chunk - before) head_end = min(first_end, size);
    from = min(first_end, size);
  }
  int to = size;                                             // where the last run that begins here ends
  bool tail_piece = false;
  const uint32_t last_key = __builtin_amdgcn_readlane(key, size - 1);
  int tail_begin = size;
  if (last_key < a.vocab && begin + size < a.n && __builtin_amdgcn_readlane(key, size) == last_key && from < size) {
    const uint64_t run = __ballot(key == last_key);
    tail_begin = (int)__builtin_ctzll(run);
    const int end = tail_begin + (int)__builtin_ctzll(~(run >> tail_begin) | ((uint64_t)1 << 63));
    if (end - tail_begin > a.chunk) {
      tail_piece = true;
      if (tile == 0 && lane == 0) a.long_runs[1 + atomicAdd(a.long_runs, 1u)] = (uint32_t)c;     // (in any order: each is summed by itself)
    } else {
      to = end;
    }
  }
  if (head_end > 0) from = 0;
  const int n_rows = min(to, (int)__builtin_ctzll(~__ballot(key < a.vocab) | ((uint64_t)1 << 63)));      // (padding is behind all tokens)
  float sum[kWidth] = {};
  for (int r0 = from; r0 < n_rows; r0 += kDeep) {
    Vec<T> v[kDeep];
    const auto row = [&](int k) {
      return grad + (int64_t)(uint32_t)__builtin_amdgcn_readlane(position, min(r0 + k, n_rows - 1)) * a.grad_stride;
    };
    if (a.once) {
#pragma unroll
      for (int k = 0; k < kDeep; ++k) v[k] = load_columns<T, true>(row(k), cols, a.dim);
    } else {
#pragma unroll
      for (int k = 0; k < kDeep; ++k) v[k] = load_columns<T, false>(row(k), cols, a.dim);
    }
#pragma unroll
    for (int k = 0; k < kDeep; ++k) {
      const int r = r0 + k;
      if (r >= n_rows) break;
      const uint32_t now = __builtin_amdgcn_readlane(key, r);
      float x[kWidth];
      v[k].get(x);
#pragma unroll
      for (int i = 0; i < kWidth; ++i) sum[i] += x[i];
      const bool last = r + 1 == n_rows || __builtin_amdgcn_readlane(key, min(r + 1, 63)) != now;
      if (!last) continue;
      if (r < head_end || (tail_piece && r >= tail_begin))
        store_columns(r < head_end ? head : tail, cols, sum, 1.0f, 0);
      else
        store_columns(out + (int64_t)now * a.out_stride, cols, sum, a.scale, a.accumulate);
#pragma unroll
      for (int i = 0; i < kWidth; ++i) sum[i] = 0.0f;
    }
  }
}

// Long runs: a workgroup for each and a tile of the columns, as far as there are workgroups.  Its four waves add a quarter of
// the pieces each.  With kLong, for what may be more than 256 pieces a wave, sums of 32 pieces, of which eight are read side by side,
// are added in 64 bits: of a token that occurs millions of times 32 bits lose a thousandth where its rows are alike.  (65,536 x 2,048
// bfloat16 of one token, accumulated: 129 us, in 32 bits 145; 1,000,000 x 64 float32 of 1,256 tokens 135 and 154.)
constexpr int kLongPieces = 4 * 256;

template <typename T, typename O, bool kLong>
__global__ void __launch_bounds__(256) embed_grad_join_kernel(O* out, GradArgs a) {
  constexpr int kWidth = Vec<T>::kWidth, kGroup = 32;
  using Sum = std::conditional_t<kLong, double, float>;
  __shared__ Sum part[4][64][kWidth];
  const int64_t tasks = (int64_t)a.long_runs[0] * a.tiles;
  for (int64_t task = blockIdx.x; task < tasks; task += gridDim.x) {
    const int64_t c = a.long_runs[1 + task / a.tiles], tile = task % a.tiles;
    const uint32_t key = a.keys[(c + 1) * a.chunk - 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // The chunks that it goes on into begin with it.
    int64_t pieces = 1;
    for (;;) {
      const int64_t at = (c + pieces + lane) * a.chunk;
      const uint64_t more = __ballot(at < a.n && a.keys[min(at, a.n - 1)] == key);
      pieces += more == ~(uint64_t)0 ? 64 : (int)__builtin_ctzll(~more);
      if (more != ~(uint64_t)0) break;
    }
    const int64_t each = (pieces + 3) / 4, last = min(pieces, (wave + 1) * each);
    const Columns cols = columns_of<T>(tile, a.dim);
    Sum sum[kWidth] = {};
    if (a.dim >= kWidth) {
      const auto add = [&](auto (&to)[kWidth], int64_t j) {
        const float* piece = a.pieces + (2 * (c + j) + (j == 0)) * a.dim + cols.load;
#pragma unroll
        for (int h = 0; h < kWidth; h += 4) {
          float x[4];
          Vec<float>::load(piece + h).get(x);
#pragma unroll
          for (int i = 0; i < 4; ++i) to[h + i] += x[i];
        }
      };
      int64_t j = wave * each;
      if constexpr (kLong) {
        for (; j + kGroup <= last; j += kGroup) {
          float some[kWidth] = {};
#pragma unroll 8
          for (int k = 0; k < kGroup; ++k) add(some, j + k);
#pragma unroll
          for (int i = 0; i < kWidth; ++i) sum[i] += some[i];
        }
      }
#pragma unroll 4
      for (; j < last; ++j) add(sum, j);
    } else if (cols.own < cols.end) {
      for (int64_t j = wave * each; j < last; ++j)
        for (int i = 0; i < kWidth; ++i)
          if (i < a.dim) sum[i] += a.pieces[(2 * (c + j) + (j == 0)) * a.dim + i];
    }
    __syncthreads();                                           // (what was joined before is read)
#pragma unroll
    for (int i = 0; i < kWidth; ++i) part[wave][lane][i] = sum[i];
    __syncthreads();
    if (wave == 0) {
      float all[kWidth];
#pragma unroll
      for (int i = 0; i < kWidth; ++i) all[i] = (float)(part[0][lane][i] + part[1][lane][i] + part[2][lane][i] + part[3][lane][i]);
      store_columns(out + (int64_t)key * a.out_stride, cols, all, a.scale, a.accumulate);
    }
  }
}

}  // namespace bpe
