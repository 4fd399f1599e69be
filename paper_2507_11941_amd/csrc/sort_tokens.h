// Positions sorted by token: a stable radix sort of n keys below 2^31, digits of at most 9 bits, lowest first.
//
// Every wave ranks 64 keys at a time: the lanes that hold the same digit find each other with one ballot per bit, the lowest of
// them takes their numbers from the wave's counter of the digit, and a scan over the workgroup's waves (and, through counts in
// memory, over the workgroups before it) says where each wave's numbers begin.  So equal digits keep their order, whatever the
// order in which waves run.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bpe {

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
constexpr int kSortGrid = 256;                               // workgroups at most

// Which tokens there are, a byte each: cleared before any is set.
__device__ inline void clear_present(uint8_t* present, uint32_t vocab, unsigned part, unsigned parts) {
  const uint4 none = {0, 0, 0, 0};
  for (uint32_t i = part * kSortThreads + threadIdx.x; i < (vocab + 15) / 16; i += parts * kSortThreads) ((uint4*)present)[i] = none;
}

// Where position t's key comes from: the ids, with `vocab` -- behind all tokens -- for padding and what is not in use.
struct TokenKeys {
  const int32_t* ids;
  int64_t n;
  const int64_t* count;
  uint32_t vocab;

  __device__ int64_t rows() const { return count ? min(n, max(*count, (int64_t)0)) : n; }
  __device__ uint32_t key(int64_t t, int64_t rows) const {
    const uint32_t id = t < rows ? (uint32_t)ids[t] : vocab;
    return min(id, vocab);                                   // (a negative id is a large number)
  }
};

// The number that this lane's digit has among the wave's so far; `counter`: the wave's, one for each digit.  Lanes with
// valid = false count nothing.  All lanes of the wave take part.
__device__ inline uint32_t wave_rank(uint32_t digit, int bits, bool valid, uint32_t* counter) {
  uint64_t peers = __ballot(valid);
  for (int b = 0; b < bits; ++b) {
    const bool bit = digit >> b & 1;
    const uint64_t set = __ballot(bit);
    peers &= bit ? set : ~set;
  }
  const int lane = threadIdx.x & 63, leader = peers ? __ffsll((unsigned long long)peers) - 1 : lane;
  uint32_t before = 0;
  if (valid && lane == leader) before = atomicAdd(&counter[digit], (uint32_t)__popcll(peers));
  before = __shfl(before, leader);
  return before + (uint32_t)__popcll(peers & (((uint64_t)1 << lane) - 1));
}

// Of the counts of kSortWaves waves for each digit: counts become places, beginning at base[digit], which moves on.
// All threads; the caller has synchronised before.
__device__ inline void places_of_waves(uint32_t (*counter)[kDigits], uint32_t* base, int digits) {
  for (int d = threadIdx.x; d < digits; d += kSortThreads) {
    uint32_t at = base[d];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t c = counter[w][d];
      counter[w][d] = at;
      at += c;
    }
    base[d] = at;
  }
}

// An exclusive scan over up to kDigits values in LDS by the first kDigits threads; all threads take part.
__device__ inline uint32_t scan_digits(uint32_t mine, uint32_t* wave_sum) {
  uint32_t sum = mine;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t other = __shfl_up(sum, d);
    if (lane >= d) sum += other;
  }
  if (lane == 63) wave_sum[wave] = sum;
  __syncthreads();
  uint32_t before = 0;
  for (int w = 0; w < wave; ++w) before += wave_sum[w];
  return before + sum - mine;
}

// Up to kEach x 1,024 keys (and a word that the caller needs cleared): one workgroup does all passes, the keys in its registers and LDS.
template <int kEach>
__global__ void __launch_bounds__(kSortThreads) sort_small_kernel(TokenKeys in, int bits, int passes, uint32_t* keys, uint32_t* positions,
                                                                  uint8_t* present, uint32_t* cleared) {
  __shared__ uint32_t counter[kSortWaves][kDigits];
  __shared__ uint32_t base[kDigits], wave_sum[kSortWaves];
  __shared__ uint32_t held[kEach * kSortThreads];
  __shared__ uint16_t held_at[kEach * kSortThreads];
  const int n = (int)in.n, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, first = wave * 64 * kEach + lane, digits = 1 << bits;
  const int64_t rows = in.rows();
  uint32_t key[kEach], at[kEach], rank[kEach];
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    at[e] = (uint32_t)(first + e * 64);
    key[e] = in.key(at[e], rows);
  }
  if (present) clear_present(present, in.vocab, 0, 1);
  if (threadIdx.x == 0) *cleared = 0;
  for (int p = 0; p < passes; ++p) {
    for (int d = lane; d < digits; d += 64) counter[wave][d] = 0;
    __syncthreads();
    if (p == 0 && present) {
#pragma unroll
      for (int e = 0; e < kEach; ++e)
        if (key[e] < in.vocab) present[key[e]] = 1;
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      rank[e] = wave_rank(key[e] >> (p * bits) & (digits - 1), bits, first + e * 64 < n, counter[wave]);
      __builtin_amdgcn_sched_barrier(0);                     // (side by side they take more registers than there are)
    }
    __syncthreads();
    uint32_t total = 0;
    if ((int)threadIdx.x < digits)
      for (int w = 0; w < kSortWaves; ++w) total += counter[w][threadIdx.x];
    const uint32_t before = scan_digits(total, wave_sum);
    if ((int)threadIdx.x < digits) base[threadIdx.x] = before;
    __syncthreads();
    places_of_waves(counter, base, digits);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      if (first + e * 64 < n) {
        const uint32_t to = counter[wave][key[e] >> (p * bits) & (digits - 1)] + rank[e];
        held[to] = key[e];
        held_at[to] = (uint16_t)at[e];
      }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      if (first + e * 64 < n) {
        key[e] = held[first + e * 64];
        at[e] = held_at[first + e * 64];
      }
  }
#pragma unroll
  for (int e = 0; e < kEach; ++e)
    if (first + e * 64 < n) {
      keys[first + e * 64] = key[e];
      positions[first + e * 64] = at[e];
    }
}

// A pass over more: each workgroup has the keys [its number x each, ...), `each` a multiple of 1,024.  First their counts.
template <bool kFirst>
__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(TokenKeys in, const uint32_t* keys_in, int shift, int digits, int64_t each,
                                                                  uint32_t* counts, uint8_t* present, uint32_t* cleared) {
  __shared__ uint32_t count[kDigits];
  for (int d = threadIdx.x; d < digits; d += kSortThreads) count[d] = 0;
  if (kFirst && present) clear_present(present, in.vocab, blockIdx.x, gridDim.x);
  if (kFirst && blockIdx.x == 0 && threadIdx.x == 0) *cleared = 0;
  __syncthreads();
  const int64_t begin = blockIdx.x * each, end = min(in.n, begin + each);
  const int64_t rows = kFirst ? in.rows() : 0;
  for (int64_t t = begin + threadIdx.x; t < end; t += kSortThreads) {
    const uint32_t key = kFirst ? in.key(t, rows) : keys_in[t];
    atomicAdd(&count[key >> shift & (digits - 1)], 1u);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += kSortThreads) counts[blockIdx.x * kDigits + d] = count[d];
}

// ... then their places: all smaller digits, the same digit of the workgroups before, and the numbers in this one.
template <bool kFirst>
__global__ void __launch_bounds__(kSortThreads) sort_scatter_kernel(TokenKeys in, const uint32_t* keys_in, const uint32_t* positions_in,
                                                                    int shift, int bits, int64_t each, const uint32_t* counts, uint32_t* keys,
                                                                    uint32_t* positions, uint8_t* present) {
  __shared__ uint32_t counter[kSortWaves][kDigits];
  __shared__ uint32_t base[kDigits], wave_sum[kSortWaves];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, digits = 1 << bits;
  // The counts of all workgroups, by as many threads for a digit as there are.
  const int digit = threadIdx.x & (digits - 1), share = threadIdx.x >> bits, shares = kSortThreads >> bits;
  uint32_t all = 0, before_me = 0;
  for (unsigned b0 = share; b0 < gridDim.x; b0 += 32 * shares) {
    uint32_t c[32];                                          // (side by side: they come from other XCDs' caches, 2 us a read)
#pragma unroll
    for (int i = 0; i < 32; ++i) c[i] = b0 + i * shares < gridDim.x ? counts[(b0 + i * shares) * kDigits + digit] : 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      all += c[i];
      before_me += b0 + i * shares < blockIdx.x ? c[i] : 0;
    }
  }
  uint32_t* part = &counter[0][0];                            // (its 8,192 words are not in use yet)
  part[threadIdx.x] = all;
  part[kSortThreads + threadIdx.x] = before_me;
  __syncthreads();
  uint32_t total = 0, earlier = 0;
  if ((int)threadIdx.x < digits)
    for (int h = 0; h < shares; ++h) {
      total += part[h * digits + threadIdx.x];
      earlier += part[kSortThreads + h * digits + threadIdx.x];
    }
  const uint32_t before = scan_digits(total, wave_sum);       // (synchronises)
  if ((int)threadIdx.x < digits) base[threadIdx.x] = before + earlier;
  const int64_t begin = blockIdx.x * each, end = min(in.n, begin + each);
  const int64_t rows = kFirst ? in.rows() : 0;
  for (int64_t t0 = begin; t0 < end; t0 += kSortThreads) {
    for (int d = lane; d < digits; d += 64) counter[wave][d] = 0;
    const int64_t t = t0 + threadIdx.x;
    const uint32_t key = kFirst ? in.key(t, rows) : t < end ? keys_in[t] : 0;
    const uint32_t at = kFirst ? (uint32_t)t : t < end ? positions_in[t] : 0;
    const uint32_t rank = wave_rank(key >> shift & (digits - 1), bits, t < end, counter[wave]);
    __syncthreads();
    places_of_waves(counter, base, digits);
    __syncthreads();
    if (t < end) {
      const uint32_t to = counter[wave][key >> shift & (digits - 1)] + rank;
      keys[to] = key;
      positions[to] = at;
      if (kFirst && present && key < in.vocab) present[key] = 1;
    }
    __syncthreads();
  }
}

}  // namespace bpe
