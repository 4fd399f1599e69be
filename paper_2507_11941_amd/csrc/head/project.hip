// Host side of the 8-bit product (include/bpe_head.h): argument checks and the enqueue.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../../include/bpe_head.h"
#include "../ops/arguments.h"
#include "project_kernels.h"

using namespace bpe;

namespace {

// Tiles of tokens x vocabulary: by eight waves, one workgroup on a compute unit (256 x 256); by eight, two (128 x 128); by four, two
// (64 x 64); and by four, two (32 x 128), for few tokens.
enum Size { kLarge, kMiddle, kSmall, kFew };

constexpr struct {
  int tokens, words, at_once;
} kSizes[] = {{256, 256, 256}, {128, 128, 512}, {64, 64, 512}, {32, 128, 512}};

int64_t tiles_of(Size size, int64_t n, int64_t vocab) {
  return (n + kSizes[size].tokens - 1) / kSizes[size].tokens * ((vocab + kSizes[size].words - 1) / kSizes[size].words);
}

// How long tiles of a size take, in rounds of middle ones.  Large, middle, small tiles, us, of 2,048 columns into 100,260: 61 tokens 61, 39, 35;
// 128 64, 42, 51; 256 67, 70, 100; 384 137, 113, 160; 500 142, 154, 221; into 32,256: 61 31, 17, 14; 200 32, 23, 34; 1,000 70, 82, 130; 700
// tokens of 1,024 columns into 1,256 22, 9, 7.  64 tokens and fewer read the weights once either way.
double rounds_of(Size size, int64_t n, int64_t vocab) {
  constexpr double kRound[] = {1.7, 1.0, 0.8};
  return kRound[size] * (double)((tiles_of(size, n, vocab) + kSizes[size].at_once - 1) / kSizes[size].at_once);
}

Size size_of_tiles(int64_t n, int64_t vocab) {
  // (Tiles for few tokens where some compute unit would have two small ones.  Small and few, us: 8 tokens of 2,048 columns into 16,384 9.5, 9.7,
  // 20,480 11.7, 9.7, 32,000 13.0, 12.2; of 4,096 into 16,384 15.1, 15.6, 65,536 42.0, 40.8, 100,260 75.7, 76.7; of 768 into 50,257 11.9, 8.5;
  // 32 of 8,192 into 50,000 84, 75; 20 of 4,097 into 60,000 64, 40.)
  if (n <= 32 && tiles_of(kSmall, n, vocab) > 256) return kFew;
  if (n <= 64) return kSmall;
  Size best = kLarge;
  for (Size size : {kMiddle, kSmall})
    if (rounds_of(size, n, vocab) < rounds_of(best, n, vocab)) best = size;
  return best;
}

// As many workgroups as the chip holds at once go through the tiles.
template <typename T, Size kSize, int kMt, int kVt, int kWm, int kWv, int kStages>
void launch_tiles(ProjectArgs a, bool direct, T* out, hipStream_t stream) {
  static_assert(kSizes[kSize].tokens == 32 * kMt * kWm && kSizes[kSize].words == 32 * kVt * kWv);
  a.token_tiles = blocks(a.n, kSizes[kSize].tokens);
  a.tiles = (unsigned)tiles_of(kSize, a.n, a.vocab);
  // For few tokens a tile has as many words as make the last round of tiles a full one, if those are at least five eighths of it: 8 tokens of
  // 4,096 columns into 100,260 76 us -> 70, into 40,000 28.3 -> 26.0, 32 of 8,192 into 50,000 75.7 -> 71.4; with half a tile 8 of 4,096 into
  // 32,768 take 22.2, with all of it 21.3.
  if (kSize == kFew) {
    const int64_t places = ((int64_t)a.tiles + kSizes[kSize].at_once - 1) / kSizes[kSize].at_once * kSizes[kSize].at_once;
    const int words = (int)((a.vocab + places - 1) / places + 3) / 4 * 4;
    a.words = words * 8 >= kSizes[kSize].words * 5 ? words : kSizes[kSize].words;
    a.tiles = blocks(a.vocab, a.words);
  }
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(std::min(a.tiles, (unsigned)kSizes[kSize].at_once)), dim3(64 * kWm * kWv), 0, stream, a, out);
  };
  if (direct) launch(project_kernel<T, kMt, kVt, kWm, kWv, kStages, true>);
  else launch(project_kernel<T, kMt, kVt, kWm, kWv, 2, false>);
}

template <typename T>
void launch_size(Size size, const ProjectArgs& a, bool direct, T* out, hipStream_t stream) {
  if (size == kLarge) launch_tiles<T, kLarge, 4, 2, 2, 4, 2>(a, direct, out, stream);
  else if (size == kMiddle) launch_tiles<T, kMiddle, 2, 1, 2, 4, 2>(a, direct, out, stream);
  else if (size == kSmall) launch_tiles<T, kSmall, 1, 1, 2, 2, 4>(a, direct, out, stream);
  else launch_tiles<T, kFew, 1, 1, 1, 4, 3>(a, direct, out, stream);
}

template <typename T>
void launch_project(ProjectArgs a, T* out, hipStream_t stream) {
  const auto in_fours = [](const void* p, int64_t stride) { return (((uintptr_t)p | (uintptr_t)stride) & 3) == 0; };
  const bool direct = a.dim % 4 == 0 && a.dim >= 16 && in_fours(a.q, a.q_stride) && in_fours(a.weight, a.weight_stride);
  const Size size = size_of_tiles(a.n, a.vocab);
  // A last round that few workgroups have tiles of goes to smaller ones, in a second launch, where that takes less (500 tokens of 2,048
  // columns into 100,260, 3.06 rounds: 142 us -> 118).
  const int64_t token_tiles = (a.n + kSizes[size].tokens - 1) / kSizes[size].tokens, tiles = tiles_of(size, a.n, a.vocab);
  const int64_t whole = tiles / kSizes[size].at_once * kSizes[size].at_once / token_tiles * kSizes[size].words;
  if (size < kSmall && whole > 0 && whole < a.vocab) {
    const Size rest = size_of_tiles(a.n, a.vocab - whole);
    constexpr double kLaunch = 0.2;
    if (rest > size && rounds_of(size, a.n, whole) + rounds_of(rest, a.n, a.vocab - whole) + kLaunch < rounds_of(size, a.n, a.vocab)) {
      ProjectArgs last = a;
      last.vocab -= whole;
      last.weight += whole * a.weight_stride;
      last.weight_scales += whole;
      a.vocab = whole;
      launch_size(rest, last, direct, out + whole, stream);
    }
  }
  launch_size(size, a, direct, out, stream);
}

// (The rows of a tile are found by 32-bit offsets.)
bool is_bytes(const void* p, int64_t rows, int64_t columns, int64_t stride) {
  return stride >= columns && stride <= BPE_MAX_STRIDE_8BIT && fits(p, rows, 1);
}

}  // namespace

extern "C" {

int bpe_project_8bit(const int8_t* q, int64_t n, int64_t dim, int64_t q_stride, const float* scales, const int8_t* weight,
                     int64_t vocab, int64_t weight_stride, const float* weight_scales, void* out, int dtype, int64_t out_stride,
                     void* stream) {
  if (!is_count(n) || dim < 1 || dim > BPE_MAX_DIM_8BIT || !is_bytes(q, n, dim, q_stride) || !fits(scales, n, 4) || vocab < 1 ||
      vocab > BPE_MAX_COLUMNS || !is_bytes(weight, vocab, dim, weight_stride) || !fits(weight_scales, vocab, 4) ||
      !is_matrix(out, dtype, n, vocab, out_stride) || (double)n * (double)vocab > 1e13)
    return BPE_EINVAL;
  if (n == 0) return BPE_OK;
  ProjectArgs a{};
  a.q = q;
  a.scales = scales;
  a.weight = weight;
  a.weight_scales = weight_scales;
  a.n = n;
  a.vocab = vocab;
  a.q_stride = q_stride;
  a.weight_stride = weight_stride;
  a.out_stride = out_stride;
  a.dim = (int)dim;
  with_type(dtype, [&](auto type) {
    using T = decltype(type);
    launch_project(a, (T*)out, (hipStream_t)stream);
  });
  return launched();
}

}  // extern "C"
