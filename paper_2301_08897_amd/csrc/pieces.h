// pieces.h -- 16 bytes of a row of float or bfloat16 elements that starts at
// any address aligned to its elements (the memory system takes wide accesses
// at that alignment), and how a workgroup's lanes share the pieces of rows.
// Internal to libscadles.
#pragma once

#include "abi.h"
#include "frame.h"

namespace scadles {

typedef u4 u4at4 __attribute__((aligned(4)));
typedef u4 u4at2 __attribute__((aligned(2)));
typedef float f8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));

// What a type's 16 bytes are: N elements, as floats F.
template <class X>
struct Piece;
template <>
struct Piece<float> {
  static constexpr uint32_t N = 4;
  typedef f4 F;
  typedef u4at4 Any;
};
template <>
struct Piece<uint16_t> {     // bfloat16
  static constexpr uint32_t N = 8;
  typedef f8 F;
  typedef u4at2 Any;
};

// 16 bytes of a row of dim elements from element `at` on, as `settled` makes them: the row's last,
// incomplete piece is read as the 16 bytes that end with the row, which is one load for all
// lanes and no wait (single elements are waited for one row at a time). `at` may lie behind the row.
template <class X>
__device__ inline u4 load_raw(const X* row, uint32_t at, uint32_t dim)
{
  constexpr uint32_t N = Piece<X>::N;
  if (dim >= N) return *(const GLOBAL typename Piece<X>::Any*)gptr(row + (at < dim - N ? at : dim - N));
  u4 x = {0, 0, 0, 0};
#pragma unroll
  for (uint32_t q = 0; q < N - 1; ++q)
    if (q < dim) {
      if constexpr (sizeof(X) == 4) x[q] = __float_as_uint(gptr(row)[q]);
      else x[q / 2] |= (uint32_t)gptr(row)[q] << (q % 2 * 16);
    }
  return x;
}

// The elements from `at` < dim on; those behind the row are zero.
template <class X>
__device__ inline u4 settled(u4 x, uint32_t at, uint32_t dim)
{
  constexpr uint32_t N = Piece<X>::N;
  if (dim % N == 0 || dim < N) return x;
  const uint32_t extra = at + N > dim ? (at + N - dim) * (uint32_t)sizeof(X) * 8 : 0;      // bits in front
  const uint64_t lo = x[0] | (uint64_t)x[1] << 32, hi = x[2] | (uint64_t)x[3] << 32;
  const uint64_t low = extra == 0 ? lo : extra < 64 ? lo >> extra | hi << (64 - extra) : hi >> (extra & 63), high = extra < 64 ? hi >> extra : 0;
  return u4{(uint32_t)low, (uint32_t)(low >> 32), (uint32_t)high, (uint32_t)(high >> 32)};
}

template <class X>
__device__ inline u4 load_piece(const X* row, uint32_t at, uint32_t dim)
{
  return settled<X>(load_raw(row, at, dim), at, dim);
}

// The first k elements (all of them if there are N or more) to p.
template <class X>
__device__ inline void store_piece(X* p, u4 x, uint32_t k)
{
  typedef uint32_t u2 __attribute__((ext_vector_type(2)));
  typedef u2 u2any __attribute__((aligned(2)));
  typedef uint32_t u1any __attribute__((aligned(2)));
  if (k >= Piece<X>::N) {
    *(GLOBAL typename Piece<X>::Any*)gptr(p) = x;
    return;
  }
  uint32_t at = k & (8 / sizeof(X));             // the elements stored so far
  if (at) *(GLOBAL u2any*)gptr(p) = u2{x[0], x[1]};
  const uint32_t a = at ? x[2] : x[0], b = at ? x[3] : x[1];
  const bool one = k & (4 / sizeof(X));
  if (one) *(GLOBAL u1any*)gptr(p + at) = a;
  if constexpr (sizeof(X) == 2) {
    if (k & 1) gptr(p)[k - 1] = (uint16_t)(one ? b : a);
  }
}

// The same for data that is not read again soon.
template <class X>
__device__ inline void store_piece_once(X* p, u4 x, uint32_t k)
{
  if (k >= Piece<X>::N) __builtin_nontemporal_store((typename Piece<X>::Any)x, (GLOBAL typename Piece<X>::Any*)gptr(p));
  else store_piece(p, x, k);
}

template <class X>
__device__ inline typename Piece<X>::F unpack(u4 x)
{
  typename Piece<X>::F f;
  if constexpr (sizeof(X) == 4) {
#pragma unroll
    for (int q = 0; q < 4; ++q) f[q] = __uint_as_float(x[q]);
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      f[2 * q] = __uint_as_float(x[q] << 16);
      f[2 * q + 1] = __uint_as_float(x[q] & 0xFFFF0000u);
    }
  }
  return f;
}

// To bfloat16 to nearest, ties to even; floats as they are.
template <class X>
__device__ inline u4 pack(typename Piece<X>::F f)
{
  if constexpr (sizeof(X) == 4) return __builtin_bit_cast(u4, f);
  else return __builtin_bit_cast(u4, __builtin_convertvector(f, b8));
}

// A workgroup of kBlock lanes takes `rows` rows of `pieces` pieces each, piece by
// piece: place i is piece i % pieces of row i / pieces. The division is a
// multiplication, exact for i * pieces < 2^32; with rows = 1 it is not needed.
struct Share {
  uint32_t pieces, rows, magic;
};

// A piece for every lane of a workgroup.
inline Share share_rows(uint64_t rows, uint64_t pieces)
{
  uint64_t n = pieces > 1024 ? 1 : div_up(kBlock, pieces);
  if (n > rows) n = rows ? rows : 1;
  return {(uint32_t)pieces, (uint32_t)n, (uint32_t)(n == 1 ? 0 : div_up(1ull << 32, pieces))};
}

// A launch has fewer than 2^32 lanes: workgroups beyond these take their turn.
constexpr uint64_t kMostBlocks = 1u << 22;
inline uint32_t grid_of(uint64_t blocks) { return (uint32_t)(blocks < kMostBlocks ? blocks : kMostBlocks); }

// Calls f(row of the workgroup, piece) for every place of this lane.
template <class F>
__device__ inline void for_pieces(const Share& s, F f)
{
  for (uint32_t i = threadIdx.x; i < s.rows * s.pieces; i += kBlock) {
    const uint32_t r = s.rows == 1 ? 0u : s.pieces == 1 ? i : __umulhi(i, s.magic);
    f(r, i - r * s.pieces);
  }
}

// The same for all `rows` rows, f(row, piece): workgroup after workgroup of them.
template <class F>
__device__ inline void for_all_pieces(const Share& s, uint64_t rows, F f)
{
  for (uint64_t r0 = (uint64_t)blockIdx.x * s.rows; r0 < rows; r0 += (uint64_t)gridDim.x * s.rows)
    for_pieces(s, [&](uint32_t r, uint32_t g) {
      if (r0 + r < rows) f(r0 + r, g);
    });
}

// Bytes from the first to the last element of `rows` rows.
inline uint64_t rows_bytes(uint64_t rows, uint64_t dim, uint64_t ld, uint64_t esize) { return rows ? ((rows - 1) * ld + dim) * esize : 0; }

}  // namespace scadles
