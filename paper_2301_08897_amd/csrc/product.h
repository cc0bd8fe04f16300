// product.h -- a 256 x 256 tile of a product of matrices of 16-bit floats with sums in
// float, on the matrix cores: D[m][n] = sum over pairs of planes, over k of
// A[m][k] B[n][k]. Internal to libscadles.
//
// Both operands are rows of adjacent k, 16-byte aligned, a multiple of 64 long. A
// workgroup of eight waves, two by four, has a tile; a wave 128 x 64 of it in 128
// accumulators.
// Steps of 64 k go straight from memory to LDS, the two operands' halves of a step (32
// KiB each) in five places in turn, up to one and a half steps ahead. A row's part of a step
// is a line of 128 bytes: loads to LDS reach 22 TB/s with those, 13 with 64 bytes of
// a row.
// The waves of a compute unit come out of a step's barrier together, so that what they read
// from LDS then is not hidden by each other's products (a third of the time). A step
// is four phases of 16 products, and every wave reads the fragments of a phase while
// it multiplies those of the one before; the barrier is before the last phase, when all
// of the step has been read.
// An LDS row is 128 bytes of one row of an operand, its eight 16-byte pieces permuted by
// the low bits of the row's number, so that eight lanes that read the same piece of
// neighbouring rows use every bank once. Which row of the operand lies in which LDS row is
// chosen for the stores: a lane's accumulators are four adjacent n, and of m groups of
// kGroup adjacent ones, the four groups of a column's lanes next to each other.
// Both are made on the way in, by what a lane loads.
// Rows that lie a power of two apart cost up to a tenth, so that whoever lays out an
// operand pads its rows.
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

// 16 bytes of every lane, at an offset of its own from a common address, to 1 KiB of LDS. It
// has no result, so that nothing can go wrong with registers; the builtin makes the
// compiler wait for all LDS reads before every product, where some of them suffice.
// The wait states are those between a lane's value becoming a scalar and its use as an address.
__device__ inline void load_lds(const char* base, uint32_t off, uint32_t lds)
{
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds) : "memory");
}

__device__ inline void workgroup_barrier()
{
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The workgroup's LDS from tile to tile. `begin` starts a tile's loads, `run` multiplies
// it; the next tile may begin as soon as run returns, without a barrier. All of the
// workgroup's lanes call them, with the same steps and pairs.
struct Pipe {
  char* lds;
  uint32_t start;                          // of this wave's rows in a place
  uint32_t fill, from;                     // the places that are filled and read next

  __device__ explicit Pipe(char* p)
      : lds(p), start((uint32_t)(uintptr_t)(SHARED char*)p + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 4096), fill(0), from(0)
  {
  }

  static __device__ inline uint32_t turn(uint32_t& p)
  {
    const uint32_t here = p;
    p = p + kSideBytes == kProductLds ? 0 : p + kSideBytes;
    return here;
  }

  // What of an operand is loaded next: the step, counted over the pairs, and its address.
  struct Next {
    const char* at;
    uint32_t pair, step;
  };
  Next a_next, b_next;

  static __device__ inline void enter(Next& x, const Side& s, uint32_t planes, uint32_t pair)
  {
    x = {reinterpret_cast<const char*>(s.base + (planes >> 4 * pair & 15) * s.plane), pair, 0};
  }

  __device__ inline void load(Next& x, const Side& s, uint32_t planes, uint32_t steps)
  {
    const uint32_t to = start + turn(fill);
#pragma unroll
    for (int it = 0; it < 4; ++it) load_lds(x.at, s.off[it], to + it * 1024);
    x.at += kStep * 2;
    if (++x.step == steps) enter(x, s, planes, x.pair + 1);
  }

  __device__ inline void begin(const Side& a, const Side& b, uint32_t steps, const Pairs& pairs)
  {
    enter(a_next, a, pairs.a, 0);
    enter(b_next, b, pairs.b, 0);
    const uint32_t n = steps * pairs.n;
    if (n > 0) {
      load(a_next, a, pairs.a, steps);
      load(b_next, b, pairs.b, steps);
    }
    if (n > 1) load(a_next, a, pairs.a, steps);
  }

  // The tile's accumulators; steps may be 0. `loaded`: this wave has waited for the loads
  // of `begin` already.
  template <class E>
  __device__ inline void run(f4 (&acc)[8][4], const Side& a, const Side& b, uint32_t steps, const Pairs& pairs, bool loaded)
  {
    typedef typename E::Fragment F;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = f4{0, 0, 0, 0};
    const uint32_t n = steps * pairs.n;
    if (n == 0) return;
    const uint32_t lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
    const uint32_t row_a = (threadIdx.x >> 8) * 16384 + r * 128, row_b = (threadIdx.x >> 6 & 3) * 8192 + r * 128;
    const uint32_t piece[2] = {(q ^ (r & 7)) * 16, ((4 + q) ^ (r & 7)) * 16};
    const char *pa, *pb;                   // the step that is read
    F low[4], high[4], y[2][4];
    auto next_step = [&] {
      pa = lds + turn(from) + row_a;
      pb = lds + turn(from) + row_b;
    };
    auto read_low = [&](auto k) {
#pragma unroll
      for (int j = 0; j < 4; ++j) y[k][j] = *(const F*)(pb + j * 2048 + piece[k]);
#pragma unroll
      for (int s = 0; s < 4; ++s) low[s] = *(const F*)(pa + s * 2048 + piece[k]);
      __builtin_amdgcn_sched_barrier(0);
    };
    auto read_high = [&](auto k) {
#pragma unroll
      for (int s = 0; s < 4; ++s) high[s] = *(const F*)(pa + (4 + s) * 2048 + piece[k]);
      __builtin_amdgcn_sched_barrier(0);
    };
    auto products = [&](const F (&x)[4], auto k, auto half) {
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[half * 4 + s][j] = E::product(x[s], y[k][j], acc[half * 4 + s][j]);
      __builtin_amdgcn_sched_barrier(0);
    };
    constexpr std::integral_constant<int, 0> k0;
    constexpr std::integral_constant<int, 1> k1;
    auto three_phases = [&] {
      read_high(k0);
      products(low, k0, k0);
      read_low(k1);
      products(high, k0, k1);
      read_high(k1);
      products(low, k1, k0);
    };
    // Scalar loads are waited for once, so that what is counted in the loop is LDS reads alone
    // and the waits can be for some of them.
    __builtin_amdgcn_s_waitcnt(0xC07F);
    if (!loaded) {
      if (n > 1) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    workgroup_barrier();
    if (n > 1) load(b_next, b, pairs.b, steps);
    if (n > 2) load(a_next, a, pairs.a, steps);
    next_step();
    read_low(k0);
    uint32_t i = 0;
#pragma clang loop unroll(disable)
    for (; i + 3 < n; ++i) {
      three_phases();
      // this wave has read all of the step, and the next one has come but for what others loaded
      // (the half behind it may be under way); behind the barrier both hold for all waves
      asm volatile("s_waitcnt vmcnt(4) lgkmcnt(0)" ::: "memory");
      workgroup_barrier();
      load(b_next, b, pairs.b, steps);
      load(a_next, a, pairs.a, steps);
      next_step();
      read_low(k0);
      products(high, k1, k1);
    }
#pragma clang loop unroll(disable)
    for (; i < n; ++i) {
      three_phases();
      if (i + 1 < n) {
        if (i + 2 < n) asm volatile("s_waitcnt vmcnt(4) lgkmcnt(0)" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        workgroup_barrier();
        if (i + 2 < n) load(b_next, b, pairs.b, steps);
        next_step();
        read_low(k0);
      }
      products(high, k1, k1);
    }
  }

  // LDS that is free between run and the next tile's run, behind a barrier: the place that was read last.
  __device__ inline char* spare() const { return lds + (from ? from : kProductLds) - kSideBytes; }
};

}  // namespace scadles
