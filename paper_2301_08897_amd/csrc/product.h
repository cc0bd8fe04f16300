// product.h -- a 256 x 256 tile of a product of bfloat16 matrices with sums in float,
// on the matrix cores: D[m][n] = sum over pairs of planes, over k of A[m][k] B[n][k].
// Internal to libscadles.
//
// Both operands are rows of adjacent k, 16-byte aligned, a multiple of 64 long. A
// workgroup of eight waves, two by four, has a tile; a wave 128 x 64 of it in 128
// accumulators. 64 k of both operands (64 KiB) go straight from memory to LDS while
// the 64 before them are multiplied: two buffers, one barrier for each.
// LDS rows are 128 bytes; the eight 16-byte pieces of a row are permuted by bits of
// the row's number, so that eight lanes that read the same k of their rows use every
// bank once. The permutation is made on the way in, by which piece a lane loads.
// Which rows of a tile a lane holds is chosen for the stores: the accumulators of a
// lane are 32 adjacent m (a line of D's floats) of four adjacent n.
// Floats are sums of three bfloat16 planes; a product of two such matrices is the
// product of six pairs of planes, one after the other in the same accumulators.
#pragma once

#include "pieces.h"

namespace scadles {

constexpr int kEdge = 256;                 // rows of A and of B in a tile
constexpr int kStep = 64;                  // k of a step
constexpr int kProductBlock = 512;
constexpr uint32_t kSideBytes = kEdge * kStep * 2;
constexpr uint32_t kProductLds = 4 * kSideBytes;

#if defined(__HIP_DEVICE_COMPILE__)
#define SHARED __attribute__((address_space(3)))
#else
#define SHARED
#endif

// Pairs of planes to multiply: pair i is plane (a >> 4 i) & 15 of A and of B alike.
struct Pairs {
  uint32_t n, a, b;
};

// An operand's part of a tile: the address of its first k in plane 0, the elements
// between planes, and this lane's four offsets in it (see lane_row, lane_piece).
struct Side {
  const uint16_t* base;
  uint64_t plane;
  uint32_t off[4];
};

// The row of a tile, and the 16 bytes of it, that this lane loads in its turn `it`.
__device__ inline uint32_t lane_row(uint32_t it) { return (threadIdx.x >> 6) * 32 + it * 8 + (threadIdx.x & 63) / 8; }
__device__ inline uint32_t lane_piece_a(uint32_t it)
{
  const uint32_t row = lane_row(it);
  return (threadIdx.x & 7) ^ ((row & 3) | (row >> 5 & 1) << 2);
}
__device__ inline uint32_t lane_piece_b(uint32_t it) { return (threadIdx.x & 7) ^ (lane_row(it) >> 2 & 7); }

// Where a lane's accumulators lie in the tile: [i][j][e] is row m + 4 i + e, column n + j.
__device__ inline uint32_t lane_m() { return (threadIdx.x >> 8) * 128 + (threadIdx.x >> 4 & 3) * 32; }
__device__ inline uint32_t lane_n() { return (threadIdx.x >> 6 & 3) * 64 + (threadIdx.x & 15) * 4; }

__device__ inline void load_side(const Side& s, uint32_t plane, uint32_t step, char* lds)
{
  const char* p = reinterpret_cast<const char*>(s.base + plane * s.plane + (uint64_t)step * kStep);
  char* to = lds + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 4096;
#pragma unroll
  for (int it = 0; it < 4; ++it)
    __builtin_amdgcn_global_load_lds((const GLOBAL void*)gptr(p + s.off[it]), (SHARED void*)(to + it * 1024), 16, 0, 0);
}

// The tile's accumulators; steps may be 0. The workgroup's LDS is free afterwards.
__device__ inline void multiply(f4 (&acc)[8][4], const Side& a, const Side& b, uint32_t steps, const Pairs& pairs, char* lds)
{
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f4{0, 0, 0, 0};
  const uint32_t lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4, wm = threadIdx.x >> 8, wn = threadIdx.x >> 6 & 3;
  // the lane's rows of A are at + 4 i, of B at + j
  const uint32_t row_a = wm * 128 + (r >> 2) * 32 + (r & 3), row_b = wn * 64 + r * 4;
  const uint32_t swap_a = (r & 3) | (r >> 2 & 1) << 2, swap_b = r & 7;
  const uint32_t n = steps * pairs.n;
  uint32_t pair = 0, step = 0;
  auto load = [&](uint32_t i) {            // step i, counted over the pairs
    char* to = lds + (i & 1) * 2 * kSideBytes;
    load_side(a, pairs.a >> 4 * pair & 15, step, to);
    load_side(b, pairs.b >> 4 * pair & 15, step, to + kSideBytes);
    if (++step == steps) {
      step = 0;
      ++pair;
    }
  };
  if (n) load(0);
  for (uint32_t i = 0; i < n; ++i) {
    // the step's data have come, and every wave has read the step before
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (i + 1 < n) load(i + 1);
    const char* pa = lds + (i & 1) * 2 * kSideBytes + row_a * 128;
    const char* pb = lds + (i & 1) * 2 * kSideBytes + kSideBytes + row_b * 128;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      b8 x[8], y[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = *(const b8*)(pb + j * 128 + ((k * 4 + q) ^ swap_b) * 16);
#pragma unroll
      for (int s = 0; s < 8; ++s) x[s] = *(const b8*)(pa + s * 512 + ((k * 4 + q) ^ swap_a) * 16);
#pragma unroll
      for (int s = 0; s < 8; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[s][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[s], y[j], acc[s][j], 0, 0, 0);
    }
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// x as the sum of bfloat16 parts: each is the rest to nearest, so three hold all 24 bits.
// What is not finite is the first part alone.
__device__ inline uint16_t next_plane(float& x)
{
  uint32_t bits = __float_as_uint(x);
  uint16_t h = __builtin_bit_cast(uint16_t, (__bf16)x);
  if ((h & 0x7F80) == 0x7F80) {
    if ((bits & 0x7F800000) == 0x7F800000) {
      x = 0.0f;
      return h;
    }
    h = (uint16_t)(bits >> 16);            // rounding up would pass the largest value
  }
  x -= __uint_as_float((uint32_t)h << 16);
  return h;
}

}  // namespace scadles
