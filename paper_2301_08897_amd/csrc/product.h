// product.h -- a 256 x 256 tile of a product of matrices of 16-bit floats with sums in
// float, on the matrix cores: D[m][n] = sum over pairs of planes, over k of
// A[m][k] B[n][k]. Internal to libscadles.
//
// Both operands are rows of adjacent k, 16-byte aligned, a multiple of 64 long. A
// workgroup of eight waves, two by four, has a tile; a wave 128 x 64 of it in 128
// accumulators. Steps of 64 k go straight from memory to LDS, the two operands' halves
// of a step (32 KiB each) in five places in turn: while a step is multiplied the next
// one's halves and the first half of the one behind it are on their way. A step's
// fragments are read at once, so that all of its products follow without a wait.
// 16384 x 1024 x 8192 takes 212 us, 1.30 PFLOP/s (a library product of those sizes 231; steps of 32,
// four ahead, 228; without the loads 165, without the products 157: what is left is
// the clock under load, and both at once).
// Rows that lie a power of two apart cost up to a tenth, so that whoever lays out an
// operand pads its rows.
// An LDS row is 128 bytes of one row of an operand, its eight 16-byte pieces permuted by
// the low bits of the row's number, so that eight lanes that read the same piece of
// neighbouring rows use every bank once. Which row of the operand lies in which LDS row is
// chosen for the stores: a lane's accumulators are four adjacent n, and of m groups of
// kGroup adjacent ones, the four groups of a column's lanes next to each other.
// Both are made on the way in, by what a lane loads.
#pragma once

#include <type_traits>

#include "pieces.h"

namespace scadles {

constexpr int kEdge = 256;                 // rows of A and of B in a tile
constexpr int kStep = 64;                  // k of a step
constexpr int kPlaces = 5;                 // halves of steps in LDS
constexpr int kProductBlock = 512;
constexpr uint32_t kComputeUnits = 256;
constexpr uint32_t kSideBytes = kEdge * kStep * 2;
constexpr uint32_t kProductLds = kPlaces * kSideBytes;

#if defined(__HIP_DEVICE_COMPILE__)
#define SHARED __attribute__((address_space(3)))
#else
#define SHARED
#endif

typedef _Float16 h8 __attribute__((ext_vector_type(8)));

// Element types.
struct BF16 {
  typedef b8 Fragment;
  typedef __bf16 Element;
  static __device__ inline f4 product(b8 x, b8 y, f4 sum) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, sum, 0, 0, 0); }
};
struct F16 {
  typedef h8 Fragment;
  typedef _Float16 Element;
  static __device__ inline f4 product(h8 x, h8 y, f4 sum) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, sum, 0, 0, 0); }
};

// Pairs of planes to multiply: pair i is plane (a >> 4 i) & 15 of A and of B alike.
struct Pairs {
  uint32_t n, a, b;
};

// An operand's part of a tile: the address of its first k in plane 0, the elements
// between planes, and this lane's four offsets in bytes (see lane_row_a, lane_piece).
struct Side {
  const uint16_t* base;
  uint64_t plane;
  uint32_t off[4];
};

// The LDS row that this lane fills in its turn `it`, and what it loads: a row of the
// tile and 16 bytes of its step.
__device__ inline uint32_t lane_slot(uint32_t it) { return (threadIdx.x >> 6) * 32 + it * 8 + (threadIdx.x & 63) / 8; }
template <int kGroup>
__device__ inline uint32_t lane_row_a(uint32_t it)
{
  const uint32_t x = lane_slot(it);
  return kGroup == 4 ? x : (x & 224) | (x >> 2 & 3) * 8 | (x >> 4 & 1) * 4 | (x & 3);
}
__device__ inline uint32_t lane_row_b(uint32_t it)
{
  const uint32_t x = lane_slot(it);
  return (x & 192) | (x & 15) * 4 | (x >> 4 & 3);
}
__device__ inline uint32_t lane_piece(uint32_t it) { return (threadIdx.x & 7) ^ (lane_slot(it) & 7); }

// Where a lane's accumulators lie in the tile: [i][j][e] is row lane_m(i) + e, column lane_n() + j.
template <int kGroup>
__device__ inline uint32_t lane_m(uint32_t i)
{
  const uint32_t q = threadIdx.x >> 4 & 3, w = (threadIdx.x >> 8) * 128;
  return kGroup == 4 ? w + i * 16 + q * 4 : w + i / 2 * 32 + q * 8 + i % 2 * 4;
}
__device__ inline uint32_t lane_n() { return (threadIdx.x >> 6 & 3) * 64 + (threadIdx.x & 15) * 4; }

// The workgroup's LDS from tile to tile. `begin` starts a tile's loads, `run` multiplies
// it; the next tile may begin as soon as run returns, without a barrier. All of the
// workgroup's lanes call them, with the same steps and pairs.
struct Pipe {
  char* lds;
  uint32_t fill, from;                     // the places that are filled and read next

  __device__ explicit Pipe(char* p) : lds(p), fill(0), from(0) {}

  static __device__ inline uint32_t turn(uint32_t& p)
  {
    const uint32_t here = p;
    p = p + kSideBytes == kProductLds ? 0 : p + kSideBytes;
    return here;
  }

  __device__ inline void load(const Side& s, uint32_t plane, uint32_t step)
  {
    const char* p = reinterpret_cast<const char*>(s.base + plane * s.plane + (uint64_t)step * kStep);
    char* to = lds + turn(fill) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 4096;
#pragma unroll
    for (int it = 0; it < 4; ++it)
      __builtin_amdgcn_global_load_lds((const GLOBAL void*)gptr(p + s.off[it]), (SHARED void*)(to + it * 1024), 16, 0, 0);
  }

  // What of a tile is loaded next: steps, counted over the pairs.
  struct Next {
    uint32_t pair, step;
    __device__ inline void advance(uint32_t steps)
    {
      if (++step == steps) {
        step = 0;
        ++pair;
      }
    }
  };
  Next next_a, next_b;

  __device__ inline void load_a(const Side& a, const Pairs& p, uint32_t steps)
  {
    load(a, p.a >> 4 * next_a.pair & 15, next_a.step);
    next_a.advance(steps);
  }
  __device__ inline void load_b(const Side& b, const Pairs& p, uint32_t steps)
  {
    load(b, p.b >> 4 * next_b.pair & 15, next_b.step);
    next_b.advance(steps);
  }

  __device__ inline void begin(const Side& a, const Side& b, uint32_t steps, const Pairs& pairs)
  {
    next_a = next_b = {0, 0};
    const uint32_t n = steps * pairs.n;
    if (n > 0) {
      load_a(a, pairs, steps);
      load_b(b, pairs, steps);
    }
    if (n > 1) load_a(a, pairs, steps);
  }

  // The tile's accumulators; steps may be 0. `loaded`: this wave has waited for the loads
  // of `begin` already.
  template <class E>
  __device__ inline void run(f4 (&acc)[8][4], const Side& a, const Side& b, uint32_t steps, const Pairs& pairs, bool loaded)
  {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = f4{0, 0, 0, 0};
    const uint32_t lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
    const uint32_t row_a = (threadIdx.x >> 8) * 128 + r, row_b = (threadIdx.x >> 6 & 3) * 64 + r;
    const uint32_t n = steps * pairs.n;
#pragma clang loop unroll(disable)
    for (uint32_t i = 0; i < n; ++i) {
      // the step's halves have come (the first half of the next one may be under way), and
      // every wave has read the step before, whose places are filled now
      if (i == 0 && loaded) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      else if (i + 1 < n) asm volatile("s_waitcnt vmcnt(4) lgkmcnt(0)" ::: "memory");
      else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (i + 1 < n) load_b(b, pairs, steps);
      if (i + 2 < n) load_a(a, pairs, steps);
      const char* pa = lds + turn(from) + row_a * 128;
      const char* pb = lds + turn(from) + row_b * 128;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t piece = ((k * 4 + q) ^ (r & 7)) * 16;
        typename E::Fragment x[8], y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = *(const typename E::Fragment*)(pb + j * 2048 + piece);
#pragma unroll
        for (int s = 0; s < 8; ++s) x[s] = *(const typename E::Fragment*)(pa + s * 2048 + piece);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < 8; ++s)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[s][j] = E::product(x[s], y[j], acc[s][j]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }

  // LDS that is free between run and the next tile's run, behind a barrier: the place that was read last.
  __device__ inline char* spare() const { return lds + (from ? from : kProductLds) - kSideBytes; }
};

}  // namespace scadles
