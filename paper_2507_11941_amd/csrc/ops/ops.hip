// Host side of include/bpe_ops.h: argument checks and the enqueue of the operators on token batches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstddef>

#include "../../../include/bpe_ops.h"
#include "arguments.h"
#include "embed_kernels.h"
#include "logits_kernels.h"

using namespace bpe;

namespace {

// The parts of the workspace of the functions on logits.  `values` holds the rows' shares of the policy loss, 64 bits each, or the
// rows' statistics for the preference loss's gradient; `advantage` the rows' advantages, or the pairs' losses, 64 bits each.
struct LogitsWorkspace {
  size_t parts, logprobs, values, upstream, advantage, counts, total;
};

// Whether what n rows of so many elements read and write passes the caches by: where it is more than the last level holds, 256 MB.
// Passing by or not: a step of 8,209 rows of 32,256 bfloat16 181 and 204 us, 3,000 of 32,001 71 and 80, 1,600 (205 MB) 43 and 42, the
// gradient alone of 800 (102 MB) 23 and 19, after their log-probabilities 38 and 32; of 3,000 of 32,001 float32 122 and 151.  A lookup
// of 40,961 x 2,048 bfloat16 37 and 49, its gradient, of 65,536 rows, 241 and 266, of 10,000 x 1,024 float32 (41 MB) 50 and 48.
bool passes_by(int64_t n, int64_t columns, size_t element_bytes) {
  return (double)n * (double)columns * (double)element_bytes > 256e6;
}

// Whether rows begin with a line.
template <typename T>
bool rows_of_lines(const T* p, int64_t stride) {
  return aligned(p, kLine) && stride * (int64_t)sizeof(T) % kLine == 0;
}

constexpr unsigned kWeightGroups = 256;                     // workgroups that count scored positions

// Strings of 512 positions and more on average have more threads: 4 of 15,000 in 106 us a policy loss instead of 135 (of 1,256
// logits a position, whose reading and writing takes 60), 123 a preference loss instead of 163; 20 of 1,000 (2,000 logits) 46.7 and
// 47.4 instead of 51.3 and 48.8; 40 of 500 the same either way, 64 of 125 28.4 instead of 27.6 and 26.3 instead of 25.9.
bool long_strings(int64_t n, int32_t batch) { return batch > 0 && n / batch >= 512; }

// Few long rows are split among workgroups, as many as to make about kParts of them in all, and a second launch joins them.
// Each has 4 KiB of a row in one step.  Split and by one workgroup a row, us called one by one, where a launch costs the host 3.4, and
// in a graph:
//                 8 rows                   32 rows                  100 rows                 250 rows
//     63 KiB      12.4,  9.7;  5.8,  4.4   12.6,  9.6;  6.3,  4.8   12.7,  9.6;  8.2,  5.7   12.2,  9.4; 10.8,  6.9
//    196 KiB      12.1,  9.8;  6.2,  9.8   12.2, 10.4;  8.2, 10.4   11.9, 11.4; 11.6, 11.9   16.7, 14.9; 17.2, 15.3
//    392 KiB      11.9,  9.3;  6.5,  9.3   12.2, 12.9;  9.8, 13.0   13.3, 16.3; 13.6, 16.4   24.4, 21.3; 24.9, 21.7
//  3,906 KiB      12.8, 85.5; 13.2, 85.4   27.9, 88.4; 28.7, 89.4   75.2,  110; 78.1,  120
// So from 256 KiB on, where it gains called one by one and in a graph, but for the fewest rows, which lose a second launch as they are
// called; rows of 196 KiB gain in a graph alone, and are not split.
constexpr int64_t kParts = 1024;
constexpr int64_t kSplitBelow = 200, kSplitFrom = 64;       // rows; steps

bool splits_rows(int64_t n, int64_t steps) { return n < kSplitBelow && steps > kSplitFrom; }

// ... for the type with the longest rows.
size_t parts_bytes(int64_t n, int64_t vocab) {
  return n > 0 && splits_rows(n, (vocab + 1023) / 1024) ? (size_t)(n + kParts) * sizeof(Stats) : 0;
}

LogitsWorkspace logits_layout(int64_t n, int64_t vocab, int32_t batch) {
  LogitsWorkspace w{};
  w.parts = place(w.total, parts_bytes(n, vocab));
  w.logprobs = place(w.total, (size_t)n * 4);
  w.values = place(w.total, (size_t)n * 8);
  w.upstream = place(w.total, (size_t)n * 4);
  w.advantage = place(w.total, (size_t)std::max<int64_t>(n, batch) * 4);
  w.counts = place(w.total, kWeightGroups * 4);
  return w;
}

// Launches over n rows, `each` workgroups a row, of no more workgroups than a grid may have: f(first row, rows).
template <typename F>
void for_rows(int64_t n, int64_t each, F&& f) {
  const int64_t rows = std::max<int64_t>(1, ((int64_t)1 << 21) / each);
  for (int64_t first = 0; first < n; first += rows) f(first, std::min(rows, n - first));
}

// A wave of the lookup copies 4 KiB of a row where that makes at least this many waves, else 1 KiB.  Rows of 8 KiB, 1 KiB and 4
// KiB a wave: 32 rows 6.8 and 8.8 us, 2,048 9.6 and 10.1, 8,192 27.8 and 28.3, 40,961 115 and 108; 40,961 rows of 4 KiB 62.6 and 58.3.
constexpr int64_t kManyCopies = 32768;

template <typename T>
void launch_embed(const T* weight, int64_t vocab, int64_t dim, int64_t weight_stride, const int32_t* ids, int64_t n,
                  const int64_t* count, float scale, T* out, int64_t out_stride, hipStream_t stream) {
  const bool once = passes_by(n, dim, 2 * sizeof(T)) && rows_of_lines(out, out_stride);
  const auto launch = [&](auto kernel, int vecs) {
    const int64_t columns = (int64_t)vecs * 64 * Vec<T>::kWidth, parts = (dim + columns - 1) / columns;
    for_rows(n, parts, [&](int64_t first, int64_t rows) {
      hipLaunchKernelGGL(kernel, dim3(blocks(rows * parts, 4)), dim3(256), 0, stream, weight, vocab, dim, weight_stride, ids, first, n,
                         (unsigned)parts, count, scale, out, out_stride, once);
    });
  };
  if (n * ((dim + 256 * Vec<T>::kWidth - 1) / (256 * Vec<T>::kWidth)) >= kManyCopies) launch(embed_kernel<T, 4>, 4);
  else launch(embed_kernel<T, 1>, 1);
}

// The workspace of the embedding's gradient: keys and positions as they are and as the pass before left them.
struct EmbedWorkspace {
  size_t keys[2], positions[2], counts, present, long_runs, pieces, total;
  int chunk;
  int64_t chunks;
};

EmbedWorkspace embed_layout(int64_t n, int64_t vocab, int64_t dim) {
  EmbedWorkspace w{};
  // A chunk's rows are summed by one wave: fewer of them where there would be too few waves, more where runs would be cut into
  // more pieces than that needs.  Chunks of 8, 16 and 32: 2,003 rows of 2,048 columns 23.2, 26.0, 32.8 us, 8,192 37.6, 37.4, 41.7,
  // 30,000 71.2, 65.2, 63.0, 65,536 126, 103, 95; of 387 columns 8,192 34.7, 38.8, 48.6, 30,000 49.7, 45.6, 45.9.
  constexpr int64_t kEnoughWaves = 1536;
  const int64_t tiles = (dim + 511) / 512;
  w.chunk = kChunk;
  while (w.chunk > 8 && (n + w.chunk - 1) / w.chunk * tiles < kEnoughWaves) w.chunk /= 2;
  w.chunks = (n + w.chunk - 1) / w.chunk;
  for (int i = 0; i < 2; ++i) {
    w.keys[i] = place(w.total, (size_t)n * 4);
    w.positions[i] = place(w.total, (size_t)n * 4);
  }
  w.counts = place(w.total, (size_t)kSortGrid * kDigits * 4);
  w.present = place(w.total, (size_t)vocab);
  w.long_runs = place(w.total, ((size_t)w.chunks + 1) * 4);
  w.pieces = place(w.total, (size_t)w.chunks * 2 * dim * 4);
  return w;
}

// Positions by token, into keys[0] and positions[0] of the workspace; and which tokens there are, unless `present` is null.
void sort_tokens(const TokenKeys& in, char* ws, const EmbedWorkspace& w, uint8_t* present, hipStream_t stream) {
  int width = 1;
  while (in.vocab >> width) ++width;                        // of the largest key, which is `vocab`
  const int passes = (width + kDigitBits - 1) / kDigitBits, bits = (width + passes - 1) / passes;
  uint32_t *keys[2], *positions[2];
  for (int i = 0; i < 2; ++i) {
    keys[i] = (uint32_t*)(ws + w.keys[i]);
    positions[i] = (uint32_t*)(ws + w.positions[i]);
  }
  if (in.n <= kRankKeys && width + kRankBits <= 32) {
    const unsigned grid = std::max(blocks(in.n, kRankEach), blocks(in.vocab, kRankTokens));
    hipLaunchKernelGGL(sort_rank_kernel, dim3(grid), dim3(kRankThreads), 0, stream, in, (blocks(in.vocab, grid) + 15) & ~15u, keys[0],
                       positions[0], present, (uint32_t*)(ws + w.long_runs));
    return;
  }
  uint32_t* counts = (uint32_t*)(ws + w.counts);
  const int64_t most = (in.n + kSortGrid - 1) / kSortGrid, each = (most + kSortThreads - 1) / kSortThreads * kSortThreads;
  const dim3 grid(blocks(in.n, each));
  for (int p = 0; p < passes; ++p) {
    const int to = (passes - 1 - p) & 1, from = to ^ 1;
    const auto pass = [&](auto count, auto scatter) {
      hipLaunchKernelGGL(count, grid, dim3(kSortThreads), 0, stream, in, keys[from], p * bits, 1 << bits, each, counts, present,
                         (uint32_t*)(ws + w.long_runs));
      hipLaunchKernelGGL(scatter, grid, dim3(kSortThreads), 0, stream, in, keys[from], positions[from], p * bits, bits, each, counts,
                         keys[to], positions[to], present);
    };
    if (p == 0) pass(sort_count_kernel<true>, sort_scatter_kernel<true>);
    else pass(sort_count_kernel<false>, sort_scatter_kernel<false>);
  }
}

template <typename T, typename O>
void launch_embed_grad(const T* grad, O* out, GradArgs a, hipStream_t stream) {
  constexpr int64_t kMost = (int64_t)1 << 22;               // workgroups of a launch
  a.tiles = (unsigned)((a.dim + 64 * Vec<T>::kWidth - 1) / (64 * Vec<T>::kWidth));
  a.once = passes_by(a.n, a.dim, sizeof(T)) && a.dim >= Vec<T>::kWidth && rows_of_lines(grad, a.grad_stride);
  const int64_t summing = (a.chunks * a.tiles + 3) / 4, row_vecs = (a.dim + Vec<O>::kWidth - 1) / Vec<O>::kWidth;
  const int64_t groups = summing + (a.accumulate ? 0 : ((int64_t)a.vocab * row_vecs + kClear - 1) / kClear);
  for (int64_t first = 0; first < groups; first += kMost)
    hipLaunchKernelGGL((embed_grad_kernel<T, O>), dim3((unsigned)std::min(kMost, groups - first)), dim3(256), 0, stream, grad, out, a, first,
                       summing);
  const int64_t long_runs = a.n / (a.chunk + 1);            // at most
  const auto join = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>(2048, long_runs * a.tiles)), dim3(256), 0, stream, out, a);
  };
  if (a.chunks > kLongPieces) join(embed_grad_join_kernel<T, O, true>);
  else if (long_runs > 0) join(embed_grad_join_kernel<T, O, false>);
}

template <typename T>
void launch_logprobs(const T* logits, int64_t n, int64_t vocab, int64_t stride, RowArgs a, Stats* part, hipStream_t stream) {
  a.once = passes_by(n, vocab, sizeof(T));
  constexpr int64_t kStep = 256 * Vec<T>::kWidth;           // 4 KiB of a row
  const int64_t steps = (vocab + kStep - 1) / kStep;
  int64_t parts = splits_rows(n, steps) ? std::min(kParts / n, (steps + 1) / 2) : 1;
  const int64_t each = (steps + parts - 1) / parts * kStep;
  parts = (vocab + each - 1) / each;
  if (parts == 1) {
    for_rows(n, 1, [&](int64_t first, int64_t rows) {
      const auto launch = [&](auto kernel, int threads) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)rows), dim3(threads), 0, stream, logits, vocab, stride, first, a);
      };
      // The more threads a row has, the less of the chip is idle when the last of many rows end, and the more of a short row's time
      // goes into joining them.  8,191 rows of 200 KB with 256, 512, 1,024 threads: 277, 273, 263 us; of 129 KB 176, 173, 167; of
      // 64 KB 92.7, 89.5, 91.4; of 2.5 KB 19.6, 33.9, 67.7, with 64 threads 10.8.  Chosen by the length alone, which is not best for
      // all numbers of rows: 600 of 200 KB take 27.1, 29.9, 32.4, 1,021 41.1, 39.8, 43.5, 2,100 79.2, 78.3, 78.9, 3,000 107, 106, 105.
      if (vocab > 1024 * kStretch) launch(logprobs_kernel<T, 1024, true>, 1024);
      else if (steps >= 24) launch(logprobs_kernel<T, 1024, false>, 1024);
      else if (steps >= 4) launch(logprobs_kernel<T, 512, false>, 512);
      else if (steps >= 2) launch(logprobs_kernel<T, 256, false>, 256);
      else launch(logprobs_kernel<T, 64, false>, 64);
    });
    return;
  }
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)(n * parts)), dim3(256), 0, stream, logits, vocab, stride, a.targets, (unsigned)parts, each,
                       part);
  };
  if (each > 256 * kStretch) launch(logprobs_part_kernel<T, true>);
  else launch(logprobs_part_kernel<T, false>);
  hipLaunchKernelGGL(logprobs_join_kernel<T>, dim3((unsigned)n), dim3(64), 0, stream, logits, vocab, stride, (int)parts, part, a);
}

template <typename T, int kKind>
void launch_rows(const T* logits, int64_t n, int64_t vocab, int64_t stride, RowArgs a, T* grad, hipStream_t stream) {
  a.once = passes_by(n, vocab, 2 * sizeof(T));
  // The smallest variant whose registers hold a row: threads x vectors a lane.  (25 vectors are what 128 registers have room for,
  // and with 128 two workgroups of 512 threads share a compute unit, the one loading while the other stores; one of 1,024 is alone.)
  const int64_t vecs = vocab / Vec<T>::kWidth;
  for_rows(n, 1, [&](int64_t first, int64_t rows) {
    const auto launch = [&](auto kernel, int threads) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)rows), dim3(threads), 0, stream, logits, vocab, stride, first, a, grad);
    };
    if (vecs <= 64 * 8) launch(row_kernel<T, kKind, 64, 8>, 64);
    else if (vecs <= 256 * 8) launch(row_kernel<T, kKind, 256, 8>, 256);
    else if (vecs <= 256 * 16) launch(row_kernel<T, kKind, 256, 16>, 256);
    else if (vecs <= 512 * 16) launch(row_kernel<T, kKind, 512, 16>, 512);
    else if (vecs <= 512 * 25) launch(row_kernel<T, kKind, 512, 25>, 512);
    else if (vecs <= 1024 * 25) launch(row_kernel<T, kKind, 1024, 25>, 1024);
    else launch(long_row_kernel<T, kKind>, 1024);
  });
}

template <typename T>
void launch_grad(const T* logits, int64_t n, int64_t vocab, int64_t stride, const int32_t* targets, const float* lse,
                 const Stats* stats, const float* upstream, T* grad, int64_t grad_stride, hipStream_t stream,
                 const double* losses = nullptr, int32_t n_losses = 0, float* loss = nullptr) {
  const int64_t parts = (vocab / Vec<T>::kWidth + 1023) / 1024 + (vocab / Vec<T>::kWidth % 1024 == 0 && vocab % Vec<T>::kWidth);
  const auto launch = [&](auto kernel) {
    for_rows(n, parts, [&](int64_t first, int64_t rows) {
      float* const here = first == 0 ? loss : nullptr;
      hipLaunchKernelGGL(kernel, dim3((unsigned)(rows * parts + (here ? 1 : 0))), dim3(256), 0, stream, logits, vocab, stride, first,
                         (unsigned)parts, targets, lse, stats, upstream, grad, grad_stride, losses, n_losses, here);
    });
  };
  if (passes_by(n, vocab, 2 * sizeof(T))) launch(logprobs_grad_kernel<T, true>);
  else launch(logprobs_grad_kernel<T, false>);
}

}  // namespace

extern "C" {

int bpe_embed_tokens(const void* weight, int dtype, int64_t vocab, int64_t dim, int64_t weight_stride, const int32_t* ids,
                     int64_t n, const int64_t* count, float scale, void* out, int64_t out_stride, void* stream) {
  if (!is_count(n) || vocab < 1 || vocab > BPE_MAX_COLUMNS || !is_matrix(weight, dtype, vocab, dim, weight_stride) ||
      !is_matrix(out, dtype, n, dim, out_stride) || !fits(ids, n, 4) || !aligned(count, 8))
    return BPE_EINVAL;
  if (n == 0) return BPE_OK;
  with_type(dtype, [&](auto type) {
    using T = decltype(type);
    launch_embed((const T*)weight, vocab, dim, weight_stride, ids, n, count, scale, (T*)out, out_stride, (hipStream_t)stream);
  });
  return launched();
}

size_t bpe_embed_tokens_grad_workspace_bytes(int64_t n, int64_t vocab, int64_t dim) {
  if (!is_count(n) || vocab < 1 || vocab > BPE_MAX_COLUMNS || dim < 1 || dim > BPE_MAX_COLUMNS) return 0;
  return embed_layout(n, vocab, dim).total;
}

int bpe_embed_tokens_grad(const void* grad, int dtype, int64_t grad_stride, const int32_t* ids, int64_t n,
                          const int64_t* count, int64_t vocab, int64_t dim, float scale, int accumulate, void* grad_weight,
                          int out_dtype, int64_t out_stride, void* workspace, size_t workspace_bytes, void* stream) {
  if (!is_count(n) || vocab < 1 || vocab > BPE_MAX_COLUMNS || !is_matrix(grad, dtype, n, dim, grad_stride) ||
      !is_matrix(grad_weight, out_dtype, vocab, dim, out_stride) || (out_dtype != dtype && out_dtype != BPE_F32) ||
      !fits(ids, n, 4) || !aligned(count, 8) ||
      !is_workspace(workspace, workspace_bytes, bpe_embed_tokens_grad_workspace_bytes(n, vocab, dim)))
    return BPE_EINVAL;
  const EmbedWorkspace w = embed_layout(n, vocab, dim);
  char* ws = (char*)workspace;
  uint8_t* present = accumulate ? nullptr : (uint8_t*)(ws + w.present);
  if (n > 0) sort_tokens({ids, n, count, (uint32_t)vocab}, ws, w, present, (hipStream_t)stream);
  GradArgs a{};
  a.keys = (const uint32_t*)(ws + w.keys[0]);
  a.positions = (const uint32_t*)(ws + w.positions[0]);
  a.n = n;
  a.vocab = (uint32_t)vocab;
  a.chunk = w.chunk;
  a.chunks = w.chunks;
  a.dim = dim;
  a.grad_stride = grad_stride;
  a.out_stride = out_stride;
  a.scale = scale;
  a.accumulate = accumulate;
  a.present = present;
  a.long_runs = (uint32_t*)(ws + w.long_runs);
  a.pieces = (float*)(ws + w.pieces);
  with_type(dtype, [&](auto type) {
    using T = decltype(type);
    const auto launch = [&](auto out_type) {
      using O = decltype(out_type);
      launch_embed_grad((const T*)grad, (O*)grad_weight, a, (hipStream_t)stream);
    };
    if (out_dtype == BPE_F32) launch(float{});
    else launch(type);
  });
  return launched();
}

int bpe_next_tokens(const int32_t* ids, int64_t n, const int64_t* offsets, int32_t batch, const int32_t* first,
                    int32_t* targets, void* stream) {
  if (!is_count(n) || batch < 0 || !fits(ids, n, 4) || !offsets || !aligned(offsets, 8) || !aligned(first, 4) ||
      !fits(targets, n, 4))
    return BPE_EINVAL;
  if (n == 0) return BPE_OK;
  hipLaunchKernelGGL(next_tokens_kernel, dim3(blocks(n, 256)), dim3(256), 0, (hipStream_t)stream, ids, n, offsets, batch, first,
                     targets);
  return launched();
}

size_t bpe_loss_workspace_bytes(int64_t n, int64_t vocab, int32_t batch) {
  if (!is_count(n) || vocab < 1 || vocab > BPE_MAX_COLUMNS || batch < 0 || batch > BPE_MAX_STRINGS) return 0;
  return logits_layout(n, vocab, batch).total;
}

size_t bpe_token_logprobs_workspace_bytes(int64_t n, int64_t vocab) {
  if (!is_count(n) || vocab < 1 || vocab > BPE_MAX_COLUMNS) return 0;
  return parts_bytes(n, vocab);
}

int bpe_token_logprobs(const void* logits, int dtype, int64_t n, int64_t vocab, int64_t stride, const int32_t* targets,
                       float* logprobs, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  if (!is_count(n) || !is_matrix(logits, dtype, n, vocab, stride) || !fits(targets, n, 4) || !aligned(logprobs, 4) ||
      !aligned(lse, 4))
    return BPE_EINVAL;
  if (parts_bytes(n, vocab) && !is_workspace(workspace, workspace_bytes, parts_bytes(n, vocab))) return BPE_EINVAL;
  if (n == 0) return BPE_OK;
  RowArgs a{};
  a.targets = targets;
  a.logprobs = logprobs;
  a.lse = lse;
  with_type(dtype, [&](auto type) {
    using T = decltype(type);
    launch_logprobs((const T*)logits, n, vocab, stride, a, (Stats*)workspace, (hipStream_t)stream);
  });
  return launched();
}

int bpe_token_logprobs_grad(const void* logits, int dtype, int64_t n, int64_t vocab, int64_t stride, const int32_t* targets,
                            const float* lse, const float* upstream, void* grad, int64_t grad_stride, void* stream) {
  if (!is_count(n) || !is_matrix(logits, dtype, n, vocab, stride) || !is_matrix(grad, dtype, n, vocab, grad_stride) ||
      !fits(targets, n, 4) || !fits(lse, n, 4) || !fits(upstream, n, 4))
    return BPE_EINVAL;
  if (n == 0) return BPE_OK;
  with_type(dtype, [&](auto type) {
    using T = decltype(type);
    launch_grad((const T*)logits, n, vocab, stride, targets, lse, nullptr, upstream, (T*)grad, grad_stride, (hipStream_t)stream);
  });
  return launched();
}

int bpe_token_logprobs_and_grad(const void* logits, int dtype, int64_t n, int64_t vocab, int64_t stride,
                                const int32_t* targets, const float* upstream, float* logprobs, float* lse, void* grad,
                                int64_t grad_stride, void* stream) {
  if (!is_count(n) || !is_matrix(logits, dtype, n, vocab, stride) || !is_matrix(grad, dtype, n, vocab, grad_stride) ||
      !fits(targets, n, 4) || !fits(upstream, n, 4) || !aligned(logprobs, 4) || !aligned(lse, 4))
    return BPE_EINVAL;
  if (n == 0) return BPE_OK;
  RowArgs a{};
  a.targets = targets;
  a.logprobs = logprobs;
  a.lse = lse;
  a.upstream = upstream;
  a.grad_stride = grad_stride;
  with_type(dtype, [&](auto type) {
    using T = decltype(type);
    launch_rows<T, kRowStep>((const T*)logits, n, vocab, stride, a, (T*)grad, (hipStream_t)stream);
  });
  return launched();
}

int bpe_preference_loss(const void* logits, int dtype, int64_t n, int64_t vocab, int64_t stride, const int32_t* targets,
                        const int64_t* offsets, int32_t batch, const float* reference, float beta, float smoothing,
                        float scale, float* loss, float* margins, float* logprobs, void* grad, int64_t grad_stride,
                        void* workspace, size_t workspace_bytes, void* stream_ptr) {
  if (!is_count(n) || !is_matrix(logits, dtype, n, vocab, stride) || !is_matrix(grad, dtype, n, vocab, grad_stride) ||
      batch < 0 || batch > BPE_MAX_STRINGS || batch % 2 || !fits(targets, n, 4) || !offsets || !aligned(offsets, 8) || !aligned(reference, 4) ||
      !std::isfinite(beta) || !(smoothing >= 0.0f && smoothing <= 1.0f) || !std::isfinite(scale) || !loss || !aligned(loss, 4) ||
      !aligned(margins, 4) || !aligned(logprobs, 4) ||
      !is_workspace(workspace, workspace_bytes, bpe_loss_workspace_bytes(n, vocab, batch)))
    return BPE_EINVAL;
  const LogitsWorkspace w = logits_layout(n, vocab, batch);
  const hipStream_t stream = (hipStream_t)stream_ptr;
  char* ws = (char*)workspace;
  float* lp = logprobs ? logprobs : (float*)(ws + w.logprobs);
  double* losses = (double*)(ws + w.advantage);
  float* upstream = (float*)(ws + w.upstream);
  Stats* stats = (Stats*)(ws + w.values);
  RowArgs a{};
  a.targets = targets;
  a.logprobs = lp;
  a.stats = stats;
  with_type(dtype, [&](auto type) {
    using T = decltype(type);
    if (n > 0) launch_logprobs((const T*)logits, n, vocab, stride, a, (Stats*)(ws + w.parts), stream);
    const auto launch_pairs = [&](auto kernel, int threads) {
      hipLaunchKernelGGL(kernel, dim3(batch / 2 + 1), dim3(threads), 0, stream, lp, targets, n, vocab, offsets, batch, reference, beta,
                         smoothing, scale, margins, losses, upstream);
    };
    if (long_strings(n, batch)) launch_pairs(pair_kernel<1024>, 1024);
    else if (batch > 0 || n > 0) launch_pairs(pair_kernel<256>, 256);
    if (n > 0)
      launch_grad((const T*)logits, n, vocab, stride, targets, nullptr, stats, upstream, (T*)grad, grad_stride, stream, losses, batch / 2,
                  loss);
    else
      hipLaunchKernelGGL(sum_kernel, dim3(1), dim3(1024), 0, stream, losses, (int64_t)(batch / 2), loss);
  });
  return launched();
}

int bpe_policy_loss(const void* logits, int dtype, int64_t n, int64_t vocab, int64_t stride, const int32_t* targets,
                    const int64_t* offsets, int32_t batch, const float* old, const float* advantages,
                    int advantage_by_string, const float* reference, float clip_low, float clip_high, float kl_weight,
                    int by_string, float scale, float* loss, float* logprobs, void* grad, int64_t grad_stride,
                    void* workspace, size_t workspace_bytes, void* stream_ptr) {
  if (!is_count(n) || !is_matrix(logits, dtype, n, vocab, stride) || !is_matrix(grad, dtype, n, vocab, grad_stride) ||
      batch < 0 || batch > BPE_MAX_STRINGS || !fits(targets, n, 4) || !offsets || !aligned(offsets, 8) || !fits(old, n, 4) ||
      !fits(advantages, advantage_by_string ? batch : n, 4) || !aligned(reference, 4) || !(clip_low >= 0.0f && clip_low <= 1.0f) ||
      !(clip_high >= 0.0f && std::isfinite(clip_high)) || !(kl_weight >= 0.0f && std::isfinite(kl_weight)) || !std::isfinite(scale) ||
      !loss || !aligned(loss, 4) || !aligned(logprobs, 4) ||
      !is_workspace(workspace, workspace_bytes, bpe_loss_workspace_bytes(n, vocab, batch)))
    return BPE_EINVAL;
  const LogitsWorkspace w = logits_layout(n, vocab, batch);
  const hipStream_t stream = (hipStream_t)stream_ptr;
  char* ws = (char*)workspace;
  int32_t* counts = (int32_t*)(ws + w.counts);
  const int strings = long_strings(n, batch) ? 1 : kWeightWaves;
  const unsigned groups = std::min(kWeightGroups, blocks(batch, strings));
  RowArgs a{};
  a.targets = targets;
  a.logprobs = logprobs;
  a.grad_stride = grad_stride;
  a.weight = (float*)(ws + w.upstream);
  a.scored = counts;
  a.n_scored = by_string ? 0 : (int)groups;
  a.advantage = (float*)(ws + w.advantage);
  a.old = old;
  a.reference = kl_weight > 0.0f ? reference : nullptr;
  a.low = clip_low;
  a.high = clip_high;
  a.kl_weight = kl_weight;
  a.scale = scale;
  a.value = (double*)(ws + w.values);
  if (n > 0) {
    hipLaunchKernelGGL(weights_kernel, dim3(groups + 1), dim3(64 * kWeightWaves), 0, stream, targets, n, vocab, offsets, batch,
                       by_string, advantages, advantage_by_string, (float*)(ws + w.upstream), (float*)(ws + w.advantage), counts, strings);
    with_type(dtype, [&](auto type) {
      using T = decltype(type);
      launch_rows<T, kRowPolicy>((const T*)logits, n, vocab, stride, a, (T*)grad, stream);
    });
  }
  hipLaunchKernelGGL(sum_kernel, dim3(1), dim3(1024), 0, stream, a.value, n, loss);
  return launched();
}

}  // extern "C"
