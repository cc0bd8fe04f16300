// vec4.h -- four consecutive elements of a float or bfloat16 array that starts
// at any address aligned to its elements: the memory system takes wide accesses
// at that alignment. `k` elements (at least 4: all four) lie in the array; the
// others read as `fill` and are not written. Internal to libscadles.
#pragma once

#include "frame.h"

namespace scadles {

typedef f4 f4any __attribute__((aligned(4)));
typedef uint16_t h4any __attribute__((ext_vector_type(4), aligned(2)));

__device__ inline f4 widen(h4any h)
{
  f4 x;
#pragma unroll
  for (int q = 0; q < 4; ++q) x[q] = __uint_as_float((uint32_t)h[q] << 16);
  return x;
}

__device__ inline f4 load_some(const float* p, uint32_t k, float fill)
{
  f4 x = {fill, fill, fill, fill};
#pragma unroll
  for (uint32_t q = 0; q < 3; ++q)
    if (q < k) x[q] = gptr(p)[q];
  return x;
}

__device__ inline f4 load_some(const uint16_t* p, uint32_t k, float fill)
{
  f4 x = {fill, fill, fill, fill};
#pragma unroll
  for (uint32_t q = 0; q < 3; ++q)
    if (q < k) x[q] = __uint_as_float((uint32_t)gptr(p)[q] << 16);
  return x;
}

template <class T>
__device__ inline f4 load_f4(const T* p, uint32_t k, float fill = 0.0f)
{
  if (k < 4) return load_some(p, k, fill);
  if constexpr (sizeof(T) == 4) return *(const GLOBAL f4any*)gptr(p);
  else return widen(*(const GLOBAL h4any*)gptr(p));
}

// The same for data that is read once: it does not displace what the caches hold.
template <class T>
__device__ inline f4 load_once_f4(const T* p, uint32_t k, float fill = 0.0f)
{
  if (k < 4) return load_some(p, k, fill);
  if constexpr (sizeof(T) == 4) return (f4)__builtin_nontemporal_load((const GLOBAL f4any*)gptr(p));
  else return widen(__builtin_nontemporal_load((const GLOBAL h4any*)gptr(p)));
}

__device__ inline void store_f4(float* p, f4 x, uint32_t k)
{
  if (k >= 4) {
    *(GLOBAL f4any*)gptr(p) = x;
    return;
  }
#pragma unroll
  for (uint32_t q = 0; q < 3; ++q)
    if (q < k) gptr(p)[q] = x[q];
}

// To bfloat16, to nearest, ties to even.
__device__ inline void store_f4(uint16_t* p, f4 x, uint32_t k)
{
  h4any h;
#pragma unroll
  for (int q = 0; q < 4; ++q) h[q] = __builtin_bit_cast(uint16_t, (__bf16)x[q]);
  if (k >= 4) {
    *(GLOBAL h4any*)gptr(p) = h;
    return;
  }
#pragma unroll
  for (uint32_t q = 0; q < 3; ++q)
    if (q < k) gptr(p)[q] = h[q];
}

// The same for data that is not read again soon.
__device__ inline void store_once_f4(float* p, f4 x, uint32_t k)
{
  if (k >= 4) __builtin_nontemporal_store(x, (GLOBAL f4any*)gptr(p));
  else store_f4(p, x, k);
}

}  // namespace scadles
