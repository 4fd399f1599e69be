// Positions sorted by token, equal tokens in their order: few keys by counting for each of them which are smaller, more by a radix
// sort of keys below 2^31, digits of at most 9 bits, lowest first.
//
// In the radix sort every wave ranks 64 keys at a time: the lanes that hold the same digit find each other with one ballot per bit, the lowest of
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

// Up to 8,192 keys below 2^19: a key's place is the number of smaller ones, keys and positions taken together as one number, so
// that no two are equal.  Every workgroup holds all of them in LDS and counts for 32, a wave for four at a time.  n^2 comparisons, but in
// one launch and with nobody to wait for: 1,000, 2,048, 4,096 and 8,192 keys in 4.5, 6.6, 12 and 16 us, where one workgroup that
// sorted them by digits took 7, 8.5, 18 and 22, and four launches that do take 8,193 in 21.  Each workgroup also marks which of its share of the tokens there are; and a word that the caller needs is cleared.
constexpr int kRankKeys = 8192, kRankThreads = 512, kRankWave = 4, kRankEach = kRankThreads / 64 * kRankWave, kRankTokens = 8192;
constexpr int kRankBits = 13;                                // of a position

__global__ void __launch_bounds__(kRankThreads) sort_rank_kernel(TokenKeys in, uint32_t share, uint32_t* keys, uint32_t* positions,
                                                                 uint8_t* present, uint32_t* cleared) {
  __shared__ __align__(16) uint32_t held[kRankKeys];
  __shared__ __align__(16) uint8_t mark[kRankTokens];
  const int n = (int)in.n, padded = (n + 255) & ~255;
  const int64_t rows = in.rows();
  uint32_t loaded[kRankKeys / kRankThreads];                  // (side by side)
#pragma unroll
  for (int k = 0; k < kRankKeys / kRankThreads; ++k) {
    const int i = k * kRankThreads + (int)threadIdx.x;
    loaded[k] = i < n ? (uint32_t)(i < rows ? in.ids[i] : -1) : 0;
  }
#pragma unroll
  for (int k = 0; k < kRankKeys / kRankThreads; ++k) {
    const int i = k * kRankThreads + (int)threadIdx.x;
    if (i < padded) held[i] = i < n ? min(loaded[k], in.vocab) << kRankBits | (uint32_t)i : 0xffffffffu;
  }
  if (present)
    for (uint32_t i = threadIdx.x; i < share / 4; i += kRankThreads) ((uint32_t*)mark)[i] = 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) *cleared = 0;
  __syncthreads();
  const uint32_t first_token = blockIdx.x * share;
  if (present)
    for (int i = threadIdx.x; i < n; i += kRankThreads) {
      const uint32_t token = held[i] >> kRankBits;
      if (token >= first_token && token - first_token < share) mark[token - first_token] = 1;
    }
  const int lane = threadIdx.x & 63, first = (int)(blockIdx.x * kRankThreads + threadIdx.x) / 64 * kRankWave;
  if (first < n) {
    uint32_t mine[kRankWave], smaller[kRankWave] = {};
#pragma unroll
    for (int k = 0; k < kRankWave; ++k) mine[k] = (uint32_t)__builtin_amdgcn_readfirstlane((int)held[min(first + k, n - 1)]);
    uint4 next = *(const uint4*)(held + 4 * lane);
    for (int i = 256; i <= padded; i += 256) {
      const uint4 other = next;
      next = *(const uint4*)(held + (min(i, padded - 256) + 4 * lane));
#pragma unroll
      for (int k = 0; k < kRankWave; ++k)                     // (counted by the scalar unit, beside the next comparison)
        smaller[k] += (uint32_t)(__popcll(__ballot(other.x < mine[k])) + __popcll(__ballot(other.y < mine[k])) +
                                 __popcll(__ballot(other.z < mine[k])) + __popcll(__ballot(other.w < mine[k])));
    }
    if (lane < kRankWave && first + lane < n) {
      uint32_t key = mine[0], to = smaller[0];
#pragma unroll
      for (int k = 1; k < kRankWave; ++k)
        if (lane == k) {
          key = mine[k];
          to = smaller[k];
        }
      keys[to] = key >> kRankBits;
      positions[to] = key & (kRankKeys - 1);
    }
  }
  __syncthreads();
  if (present)
    for (uint32_t i = 16 * threadIdx.x; i < share && first_token + i < in.vocab; i += 16 * kRankThreads)
      *(uint4*)(present + first_token + i) = *(const uint4*)(mark + i);
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
  const int64_t begin = blockIdx.x * each, end = min(in.n, begin + each);
  const int64_t rows = kFirst ? in.rows() : 0;
  const auto key_at = [&](int64_t t) { return t >= end ? 0 : kFirst ? in.key(t, rows) : keys_in[t]; };
  const auto position_at = [&](int64_t t) { return t >= end ? 0 : kFirst ? (uint32_t)t : positions_in[t]; };
  uint32_t key = key_at(begin + threadIdx.x), at = position_at(begin + threadIdx.x);     // (beside the counts, not after them)
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
  for (int64_t t0 = begin; t0 < end; t0 += kSortThreads) {
    for (int d = lane; d < digits; d += 64) counter[wave][d] = 0;
    const int64_t t = t0 + threadIdx.x;
    if (t0 > begin) {
      key = key_at(t);
      at = position_at(t);
    }
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
