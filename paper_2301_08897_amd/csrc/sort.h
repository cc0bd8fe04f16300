// sort.h -- a stable counting sort of items by a digit, as the order of tokens by
// expert and every pass of the sort of tokens by id. Internal to libscadles.
//
// A workgroup ranks a chunk of consecutive items. A wave takes 64 of them at a
// time and finds, one ballot for each bit of the digit, the lanes that hold the
// same digit; the lanes below in that set are the item's rank among the wave's,
// and the set's last lane moves the wave's count of the digit on. No rank depends
// on the order in which waves run, so the result is always the same.
// Chunks of up to a whole problem need one launch; else the chunks' counts are
// written, added up per digit over the chunks before (k_sort_scan), and read back
// as the chunk's first places.
#pragma once

#include "abi.h"
#include "frame.h"

namespace scadles {

constexpr int kSortBlock = 1024;
constexpr int kSortWaves = kSortBlock / 64;
constexpr uint32_t kSortDigits = 1025;       // 1024 experts and "missing", or 10 bits
constexpr uint32_t kSortRounds = 8;          // items of a lane, at most
constexpr uint32_t kSortChunk = kSortBlock * kSortRounds;
constexpr uint32_t kScanDigits = 64, kScanSlices = kSortBlock / 64;

inline uint32_t sort_bits(uint32_t digits)   // of digits 0 .. digits - 1
{
  uint32_t n = 0;
  while (n < 32 && (1ull << n) < digits) ++n;
  return n;
}

// What a workgroup keeps to rank its chunk.
struct SortLds {
  uint16_t count[kSortWaves][kSortDigits + 1];   // then: items of the digit in the waves before
  uint32_t first[kSortDigits + 1];               // where the chunk's items of the digit go
  uint32_t wave[kSortWaves];
};

// Exclusive prefix of x over the workgroup's threads; `total` receives the sum.
__device__ inline uint32_t block_prefix(uint32_t x, uint32_t* wave, uint32_t& total)
{
  const uint32_t lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  uint32_t sum = x;
#pragma unroll
  for (int step = 1; step < 64; step *= 2) {
    const uint32_t y = __shfl_up(sum, step, 64);
    if ((int)lane >= step) sum += y;
  }
  __syncthreads();
  if (lane == 63) wave[w] = sum;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int q = 0; q < kSortWaves; ++q) {
    const uint32_t n = wave[q];
    before += q < (int)w ? n : 0;
    all += n;
  }
  total = all;
  return before + sum - x;
}

// Ranks n items of a chunk, R of them a lane: lane l of wave w has items (w * R + r) *
// 64 + l. digit(i) is the digit of item i < n; `digits` at most kSortDigits. Gives each
// item's digit and its rank among the wave's of that digit, and leaves in s.count
// the items of the digit in the waves before, in `mine` (for thread x: digit x)
// the chunk's items of the digit. Digit 1024 has thread 0's `last`.
template <int R, class Digit>
__device__ inline void rank_chunk(SortLds& s, uint32_t n, uint32_t digits, uint32_t bits, Digit digit, uint32_t (&key)[R],
                                  uint32_t (&rank)[R], uint32_t& mine, uint32_t& last)
{
  const uint32_t lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  for (uint32_t i = threadIdx.x; i < kSortWaves * (kSortDigits + 1) / 2; i += kSortBlock) reinterpret_cast<uint32_t*>(s.count)[i] = 0;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const uint32_t i = (w * R + r) * 64 + lane;
    key[r] = i < n ? digit(i) : ~0u;
  }
  __syncthreads();
  volatile uint16_t* count = s.count[w];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool here = key[r] != ~0u;
    uint64_t same = __ballot(here);
    for (uint32_t b = 0; b < bits; ++b) {
      const uint64_t set = __ballot(here && (key[r] >> b & 1));
      same &= key[r] >> b & 1 ? set : ~set;
    }
    if (here) {
      const uint32_t before = count[key[r]];
      rank[r] = before + __popcll(same & ((1ull << lane) - 1));
      // every lane of the set has read the count before its last lane writes it: a
      // wave's LDS operations are carried out in order
      if ((same >> lane) >> 1 == 0) count[key[r]] = (uint16_t)(before + __popcll(same));
    }
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  auto column = [&](uint32_t d) {
    uint32_t sum = 0;
#pragma unroll
    for (int q = 0; q < kSortWaves; ++q) {
      const uint32_t x = s.count[q][d];
      s.count[q][d] = (uint16_t)sum;
      sum += x;
    }
    return sum;
  };
  mine = threadIdx.x < digits ? column(threadIdx.x) : 0;
  last = threadIdx.x == 0 && digits > 1024 ? column(1024) : 0;
}

// s.first for a chunk that is the whole problem; returns the number of items
// below digit 1024.
__device__ inline uint32_t first_of_all(SortLds& s, uint32_t mine)
{
  uint32_t total;
  s.first[threadIdx.x] = block_prefix(mine, s.wave, total);
  if (threadIdx.x == 0) s.first[1024] = total;
  __syncthreads();
  return total;
}

// s.first for chunk w of several: `before` are the items of each digit in the chunks
// before ([W][digits], after k_sort_scan), `all` those of all chunks.
__device__ inline void first_of_chunk(SortLds& s, const uint32_t* before, const uint32_t* all, uint32_t digits, uint32_t w)
{
  uint32_t total;
  const uint32_t x = threadIdx.x;
  const uint32_t at = block_prefix(x < digits ? all[x] : 0, s.wave, total);
  if (x < digits) s.first[x] = at + before[(uint64_t)w * digits + x];
  if (x == 0 && digits > 1024) s.first[1024] = total + before[(uint64_t)w * digits + 1024];
  __syncthreads();
}

// Counts the n items of a chunk into row[digits].
template <class Digit>
__device__ inline void count_chunk(uint32_t* lds, uint32_t n, uint32_t digits, Digit digit, uint32_t* row)
{
  for (uint32_t i = threadIdx.x; i < digits; i += kSortBlock) lds[i] = 0;
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < n; i += kSortBlock) atomicAdd(&lds[digit(i)], 1u);
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < digits; i += kSortBlock) row[i] = lds[i];
}

// count[W][digits] becomes the items of the digit in the chunks before; all[digits]
// the items of all. A workgroup takes 64 digits, its waves a slice of the chunks each.
void launch_sort_scan(uint32_t* count, uint32_t* all, uint32_t W, uint32_t digits, hipStream_t st);

// Items of a chunk for N items: so few that up to about 256 chunks take them, a
// chunk to a compute unit.
inline uint32_t sort_rounds(uint64_t N)
{
  uint32_t r = 1;
  while (r < kSortRounds && N > (uint64_t)r * kSortBlock * 256) r *= 2;
  return r;
}

// The most chunks of any sort of N items or fewer.
inline uint64_t sort_chunks(uint64_t N)
{
  const uint64_t few = div_up(N, kSortBlock), many = div_up(N, kSortChunk);
  return many > 256 ? many : few < 256 ? few : 256;
}

}  // namespace scadles
