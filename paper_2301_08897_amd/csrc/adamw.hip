// adamw.hip -- AdamW over many tensors at once, with moments in 32 bits or in
// blocks of 8-bit codes, and the gradients' global norm with the clip factor.
//
// Per element, t the step's number from 1, every operation rounded once to
// float (the same operations in the same order give the same bits anywhere):
//   g = grad * factor                       (the clip's factor, or none)
//   m = beta1 * m + (1 - beta1) * g
//   v = beta2 * v + (1 - beta2) * (g * g)
//   d = sqrt(v) * (1 / sqrt(1 - beta2^t)) + eps
//   p = p * (1 - lr * weight_decay) - (m / d) * (lr / (1 - beta1^t))
//
// Everything here reads and writes each element once and is bound by HBM: 28 B
// per element with 32-bit moments and float gradients, 16 B with 8-bit ones.
//
// 8-bit moments. Blocks of 256 consecutive elements of a tensor share one
// offset per moment. A float's upper bits, exponent and first three mantissa
// bits, number its "step" k = bits >> 20 of 0..2047; steps are 1/8 of an octave
// and order like the values. A code is the step relative to the block's
// largest: 127 steps below it for m (one bit is the sign), 255 for v, so both
// reach 15.9 octaves of m and of sqrt(v), and an update m / sqrt(v) stays
// bounded over the whole range. Below the range m becomes 0 and v the smallest
// code: a v that is not zero never becomes zero.
// The 20 bits dropped are rounded by a dither that is a Weyl sequence in the
// element's number and the step's. To the nearest, beta2 = 0.999 would move v
// by less than half a step and v would stand still; a random dither is right on
// average, but its errors add up over the ~1000 steps that v remembers, while
// those of a Weyl sequence mostly cancel. Simulated, the update against that of
// 32-bit moments, relative: 1.02 (nearest), 0.13 (random), 0.11 (Weyl) after
// 2000 steps, 0.66, 0.23 and 0.16 after 4000 more with gradients a tenth as
// large, in which Weyl's sqrt(v) falls 9% too far.
#include <cmath>
#include <cstring>

#include "abi.h"
#include "radix.h"
#include "vec4.h"

using namespace scadles;

namespace {

constexpr uint32_t kMoment = SCADLES_MOMENT_BLOCK;
constexpr uint32_t kPart = 4 * kBlock;     // elements of one workgroup's step: four per thread
constexpr uint32_t kChunk = 2 * kPart;     // elements of one record of the plan
// The norm's workgroups, at most: one per compute unit, of 1024 threads. Every
// workgroup counts itself in at one address when it is done, which takes 10 ns
// each (60 M floats: 48 us with 2048 workgroups of 256 threads, 40 us so). Where
// 256 workgroups of 256 threads take one chunk per wave, they are quicker to
// start (147 K floats: 4.6 us against 5.4).
constexpr uint32_t kNormBlocks = 256, kNormBlock = 1024, kNormSmall = 256;
constexpr uint32_t kPutTensors = 40;       // tensors of one launch's arguments
constexpr uint32_t kMagic = 0x5C4D0001u;
constexpr uint32_t kSpanM = 127, kSpanV = 255;
constexpr uint32_t kNoStep = 2040;         // steps from here on are infinities and NaN
// Multipliers of the Weyl sequences: the fractions of sqrt(5)/2, sqrt(3) and
// sqrt(2) in 32 bits.
constexpr uint32_t kWeylA = 0x9E3779B9u, kWeylB = 0xBB67AE85u, kWeylC = 0x6A09E667u;

struct Tensor {
  float* p;
  const void* g;
  void* m;
  void* v;
  uint16_t* copy;
  uint32_t* tops;
  uint64_t off;         // elements of the tensors before this one
  uint64_t n;
  uint32_t first;       // chunks of the tensors before this one
  float wd;
};

// A piece of a tensor, pointers at its first element.
struct alignas(16) Chunk {
  float* p;
  const void* g;
  void* m;
  void* v;
  uint16_t* copy;
  uint32_t* tops;
  uint64_t off;
  uint32_t n;           // 1 .. kChunk
  uint32_t i0;          // the first element's number in its tensor (modulo 2^32: it only feeds the dither)
  float wd;
  uint32_t pad[3];
};

// The plan's device memory: this header, the tensors, the chunks.
struct Head {
  uint32_t ticket;      // workgroups of the norm that are done
  uint32_t pad[63];
  double part[kNormBlocks];
};

struct PutArgs {
  Head* head;
  Tensor* to;
  uint32_t count;
  Tensor t[kPutTensors];
};

struct StepArgs {
  float b1, c1, b2, c2, eps, root, rate;   // c = 1 - beta, root = 1 / sqrt(1 - beta2^t), rate = lr / (1 - beta1^t)
  double lr;
  uint32_t um, uv;                         // the step's part of the dithers
};

__global__ void k_adamw_put(PutArgs a)
{
  const uint32_t* from = reinterpret_cast<const uint32_t*>(a.t);
  uint32_t* to = reinterpret_cast<uint32_t*>(a.to);
  for (uint32_t i = threadIdx.x; i < a.count * (sizeof(Tensor) / 4); i += blockDim.x) to[i] = from[i];
  if (threadIdx.x == 0) a.head->ticket = 0u;
}

template <class T>
__device__ inline T* step_by(T* p, uint64_t bytes)
{
  return p ? (T*)((uintptr_t)p + bytes) : nullptr;
}

// Every chunk's record, so that the kernels get all they need with one load.
__global__ __launch_bounds__(kBlock) void k_adamw_chunks(const Tensor* t, uint32_t count, Chunk* out, uint32_t chunks,
                                                         uint32_t gsize, uint32_t msize)
{
  const uint32_t c = blockIdx.x * kBlock + threadIdx.x;
  if (c >= chunks) return;
  uint32_t lo = 0, hi = count;             // the last tensor whose first chunk is at most c (empty ones have none)
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (t[mid].first <= c) lo = mid;
    else hi = mid;
  }
  const Tensor x = t[lo];
  const uint64_t e = (uint64_t)(c - x.first) * kChunk;
  const uint64_t left = x.n - e;
  Chunk r = {};
  r.p = step_by(x.p, e * 4);
  r.g = step_by(x.g, e * gsize);
  r.m = step_by(x.m, e * msize);
  r.v = step_by(x.v, e * msize);
  r.copy = step_by(x.copy, e * 2);
  r.tops = step_by(x.tops, e / kMoment * 4);
  r.off = x.off + e;
  r.n = left < kChunk ? (uint32_t)left : kChunk;
  r.i0 = (uint32_t)e;
  r.wd = x.wd;
  out[c] = r;
}

__device__ inline uint32_t load_codes(const uint8_t* p, uint32_t k)
{
  if (k >= 4) return __builtin_nontemporal_load((const GLOBAL uint32_t*)gptr(p));
  uint32_t c = 0;
  for (uint32_t q = 0; q < 3; ++q)
    if (q < k) c |= (uint32_t)gptr(p)[q] << (8 * q);
  return c;
}

__device__ inline void store_codes(uint8_t* p, uint32_t c, uint32_t k)
{
  if (k >= 4) {
    __builtin_nontemporal_store(c, (GLOBAL uint32_t*)gptr(p));
    return;
  }
  for (uint32_t q = 0; q < 3; ++q)
    if (q < k) gptr(p)[q] = (uint8_t)(c >> (8 * q));
}

// ---- 8-bit moments ----------------------------------------------------------------------------
__device__ inline uint32_t base_of(uint32_t top, uint32_t span) { return (top > span ? top : span) - span; }

template <bool kSigned>
__device__ inline float code_value(uint32_t code, uint32_t base)
{
  const uint32_t size = kSigned ? code & 127u : code;
  const uint32_t bits = size ? (size + base) << 20 : 0u;
  return __uint_as_float(kSigned ? bits | (code >> 7) << 31 : bits);
}

__device__ inline void decode_block(uint32_t cm, uint32_t cv, uint32_t top, f4& m, f4& v)
{
  const uint32_t bm = base_of(top & 0xFFFFu, kSpanM), bv = base_of(top >> 16, kSpanV);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    m[q] = code_value<true>(cm >> (8 * q) & 255u, bm);
    v[q] = code_value<false>(cv >> (8 * q) & 255u, bv);
  }
}

// The largest of the wave's values, two 16-bit halves at once, in every lane.
__device__ inline uint32_t wave_max_u16x2(uint32_t x)
{
  typedef uint16_t h2 __attribute__((ext_vector_type(2)));
  auto larger = [](uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(h2, a), __builtin_bit_cast(h2, b)));
  };
#define SCADLES_DPP(ctrl, rows) (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, rows, 0xF, false)
  x = larger(x, SCADLES_DPP(0xB1, 0xF));     // lanes 1 apart, 2 apart, the halves of 8, of 16
  x = larger(x, SCADLES_DPP(0x4E, 0xF));
  x = larger(x, SCADLES_DPP(0x141, 0xF));
  x = larger(x, SCADLES_DPP(0x140, 0xF));
  x = larger(x, SCADLES_DPP(0x142, 0xA));    // lane 15 of each row into the next, lane 31 into the upper half
  x = larger(x, SCADLES_DPP(0x143, 0xC));
#undef SCADLES_DPP
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

// Codes of the wave's block: four elements per lane (zero beyond the tensor's
// end), `um` and `uv` the dithers of the lane's first element before their
// shift. Returns the block's offsets, m's in the lower half.
__device__ inline uint32_t encode_block(f4 m, f4 v, uint32_t um, uint32_t uv, uint32_t& cm, uint32_t& cv)
{
  uint32_t km[4], kv[4], tm = 0, tv = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    km[q] = ((__float_as_uint(m[q]) & 0x7FFFFFFFu) + ((um + q * kWeylA) >> 12)) >> 20;
    kv[q] = ((__float_as_uint(v[q]) & 0x7FFFFFFFu) + ((uv + q * kWeylC) >> 12)) >> 20;
    tm = tm > km[q] ? tm : km[q];
    tv = tv > kv[q] ? tv : kv[q];
  }
  const uint32_t top = wave_max_u16x2(tm | tv << 16);
  tm = top & 0xFFFFu;
  tv = top >> 16;
  cm = cv = 0;
  if (tm >= kNoStep || tv >= kNoStep) {      // an infinity or NaN, or the largest floats rounded up
    bool bad = false;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      bad |= !(__builtin_fabsf(m[q]) < __builtin_inff()) | !(v[q] < __builtin_inff());
      km[q] = km[q] < kNoStep ? km[q] : kNoStep - 1u;
      kv[q] = kv[q] < kNoStep ? kv[q] : kNoStep - 1u;
    }
    if (__ballot(bad)) {                     // the whole block reads as NaN from now on
      cm = kSpanM * 0x01010101u;
      cv = kSpanV * 0x01010101u;
      return (kNoStep + 4u) | (kNoStep + 4u) << 16;
    }
    tm = tm < kNoStep ? tm : kNoStep - 1u;
    tv = tv < kNoStep ? tv : kNoStep - 1u;
  }
  const int bm = (int)base_of(tm, kSpanM), bv = (int)base_of(tv, kSpanV);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int a = (int)km[q] - bm, b = (int)kv[q] - bv;
    const uint32_t sa = a > 0 ? (uint32_t)a | (__float_as_uint(m[q]) >> 31) << 7 : 0u;
    const uint32_t sb = b > 1 ? (uint32_t)b : v[q] != 0.0f ? 1u : 0u;
    cm |= sa << (8 * q);
    cv |= sb << (8 * q);
  }
  return tm | tv << 16;
}

// ---- the step ---------------------------------------------------------------------------------
__device__ inline void adamw_element(float& p, float& m, float& v, float g, const StepArgs& a, float keep)
{
  m = a.b1 * m + a.c1 * g;
  v = a.b2 * v + a.c2 * (g * g);
  const float d = sqrtf(v) * a.root + a.eps;
  p = p * keep - (m / d) * a.rate;
}

// One float4 of each operand per thread and no loop, so that every load of the
// launch is independent, and every access past the caches: at the next step
// nothing of it would still be there. Both together: 5.5 TB/s on 143.7 M
// elements, 734 us; two float4 per thread in turn and plain accesses 788 us,
// either alone 786 to 853.
template <class G, bool kBits8, bool kClip>
__global__ __launch_bounds__(kBlock) void k_adamw(const Chunk* chunks, StepArgs a, const float* clip)
{
  const Chunk c = chunks[blockIdx.x / 2];
  float factor = 1.0f;
  if (kClip) {
    factor = clip[1];
    if (factor != factor) return;            // the norm is not finite: nothing changes
  }
  const float keep = (float)(1.0 - a.lr * (double)c.wd);
  const uint32_t e = blockIdx.x % 2 * kPart + threadIdx.x * 4;
  if ((e & ~(kMoment - 1)) >= c.n) return;   // whole waves: they share a block of 8-bit moments
  const uint32_t k = e < c.n ? c.n - e : 0u;
  f4 p = load_once_f4(c.p + e, k);
  const f4 g = load_once_f4((const G*)c.g + e, k);
  f4 m, v;
  uint32_t cm = 0, cv = 0;
  uint32_t* tops = nullptr;
  if (kBits8) {
    tops = c.tops + (blockIdx.x % 2 * kWaves + wave_id());
    cm = load_codes((const uint8_t*)c.m + e, k);
    cv = load_codes((const uint8_t*)c.v + e, k);
    decode_block(cm, cv, *gptr(tops), m, v);
  } else {
    m = load_once_f4((const float*)c.m + e, k);
    v = load_once_f4((const float*)c.v + e, k);
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    float pq = p[q], mq = m[q], vq = v[q];
    adamw_element(pq, mq, vq, kClip ? g[q] * factor : g[q], a, keep);
    p[q] = pq;
    m[q] = mq;
    v[q] = vq;
  }
  store_once_f4(c.p + e, p, k);
  if (c.copy) store_f4(c.copy + e, p, k);
  if (kBits8) {
#pragma unroll
    for (uint32_t q = 0; q < 4; ++q)
      if (q >= k) m[q] = v[q] = 0.0f;
    const uint32_t i = c.i0 + e;
    const uint32_t top = encode_block(m, v, i * kWeylA + a.um, i * kWeylC + a.uv, cm, cv);
    store_codes((uint8_t*)c.m + e, cm, k);
    store_codes((uint8_t*)c.v + e, cv, k);
    if (lane_id() == 0) *gptr(tops) = top;
  } else {
    store_once_f4((float*)c.m + e, m, k);
    store_once_f4((float*)c.v + e, v, k);
  }
}

// The moments' values, packed in the tensors' order, out of the states (kIn
// false) or into them. A wave takes half a chunk, all of its loads at once.
template <bool kBits8, bool kIn>
__global__ __launch_bounds__(kBlock) void k_adamw_moments(const Chunk* chunks, uint32_t count, float* pm, float* pv, uint32_t um,
                                                          uint32_t uv)
{
  constexpr uint32_t kLoads = kPart / kMoment;
  const uint32_t at = blockIdx.x * kWaves + wave_id();
  if (at / 2 >= count) return;
  const Chunk c = chunks[at / 2];
  float *xm = pm + c.off, *xv = pv + c.off;
  const uint32_t j0 = at % 2 * kLoads, e0 = lane_id() * 4;
  f4 m[kLoads], v[kLoads];
  uint32_t cm[kLoads], cv[kLoads], k[kLoads];
#pragma unroll
  for (uint32_t j = 0; j < kLoads; ++j) {
    const uint32_t e = (j0 + j) * kMoment + e0;
    k[j] = e < c.n ? c.n - e : 0u;
    if (kIn) {
      m[j] = load_once_f4(xm + e, k[j]);
      v[j] = load_once_f4(xv + e, k[j]);
    } else if (kBits8) {
      cm[j] = load_codes((const uint8_t*)c.m + e, k[j]);
      cv[j] = load_codes((const uint8_t*)c.v + e, k[j]);
    } else {
      m[j] = load_once_f4((const float*)c.m + e, k[j]);
      v[j] = load_once_f4((const float*)c.v + e, k[j]);
    }
  }
#pragma unroll
  for (uint32_t j = 0; j < kLoads; ++j) {
    const uint32_t e = (j0 + j) * kMoment + e0;
    if ((j0 + j) * kMoment >= c.n) return;
    if (kBits8 && kIn) {
      const uint32_t i = c.i0 + e;
      const uint32_t top = encode_block(m[j], v[j], i * kWeylA + um, i * kWeylC + uv, cm[j], cv[j]);
      store_codes((uint8_t*)c.m + e, cm[j], k[j]);
      store_codes((uint8_t*)c.v + e, cv[j], k[j]);
      if (e0 == 0) gptr(c.tops)[j0 + j] = top;
    } else if (kBits8) {
      decode_block(cm[j], cv[j], gptr(c.tops)[j0 + j], m[j], v[j]);
      store_f4(xm + e, m[j], k[j]);
      store_f4(xv + e, v[j], k[j]);
    } else {
      store_f4((kIn ? (float*)c.m : xm) + e, m[j], k[j]);
      store_f4((kIn ? (float*)c.v : xv) + e, v[j], k[j]);
    }
  }
}

// ---- the norm -----------------------------------------------------------------------------------
// Squares and sums in double. Workgroups sum their chunks in order, the last
// one to finish sums the workgroups' results in order, so the norm does not
// depend on the order in which they run.
template <int NT>
__device__ inline double norm_block_sum(double v, double* lds)
{
  v = wave_sum_f64(v);
  if (lane_id() == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lane_id() < NT / 64 ? lds[lane_id()] : 0.0;
  return wave_sum_f64(v);
}

template <class G, int NT>
__global__ __launch_bounds__(NT) void k_grad_norm(const Chunk* chunks, uint32_t count, Head* head, double max_norm,
                                                          float* out)
{
  __shared__ double s_sum[2][NT / 64];
  constexpr int kLoads = kChunk / 256;       // a wave takes a chunk, all of its loads at once
  double sum = 0.0;
  for (uint32_t i = blockIdx.x * (NT / 64) + wave_id(); i < count; i += gridDim.x * (NT / 64)) {
    const G* g = (const G*)chunks[i].g + lane_id() * 4;
    const uint32_t n = chunks[i].n;
    f4 x[kLoads];
    if (n == kChunk) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) x[j] = load_once_f4(g + j * 256, 4);
    } else {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const uint32_t e = j * 256 + lane_id() * 4;
        x[j] = load_once_f4(g + j * 256, e < n ? n - e : 0u);
      }
    }
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) sum = __builtin_fma((double)x[j][q], (double)x[j][q], sum);
  }
  sum = norm_block_sum<NT>(sum, s_sum[0]);
  if (threadIdx.x == 0) put(&head->part[blockIdx.x], sum);
  if (!block_is_last(&head->ticket, 1u, gridDim.x)) return;
  sum = 0.0;
  for (uint32_t i = threadIdx.x; i < gridDim.x; i += NT) sum += get(&head->part[i]);
  sum = norm_block_sum<NT>(sum, s_sum[1]);
  if (threadIdx.x) return;
  put(&head->ticket, 0u);
  const double norm = sqrt(sum);
  out[0] = (float)norm;
  out[1] = !(norm < __builtin_inf()) ? __builtin_nanf("") : norm > max_norm ? (float)(max_norm / norm) : 1.0f;
}

// ---- host side ------------------------------------------------------------------------------------
struct Layout {
  uint64_t chunks = 0, n = 0, tensors_at = sizeof(Head), chunks_at = 0, bytes = 0;
};

scadles_status measure(const scadles_adamw_tensor* t, uint32_t count, Layout& L)
{
  if (!t && count) return fail(SCADLES_EINVAL, "tensors is NULL");
  if (!count || count > (1u << 20)) return fail(SCADLES_EINVAL, "count = %u is outside [1, 2^20]", count);
  for (uint32_t i = 0; i < count; ++i) {
    if (t[i].n > 0xFFFFFFFFull) return fail(SCADLES_EINVAL, "tensor %u has more than 2^32 - 1 elements", i);
    L.chunks += div_up(t[i].n, kChunk);
    L.n += t[i].n;
  }
  if (L.chunks >= 1u << 23)                  // a launch counts its threads in 32 bits
    return fail(SCADLES_EINVAL, "the tensors have too many elements in all");
  L.chunks_at = div_up(L.tensors_at + count * sizeof(Tensor), 256) * 256;
  L.bytes = L.chunks_at + L.chunks * sizeof(Chunk);
  return SCADLES_OK;
}

scadles_status check_plan(const scadles_adamw_plan* plan)
{
  if (!plan || plan->magic != kMagic || !plan->table) return fail(SCADLES_EINVAL, "plan was not made by scadles_adamw_plan_build");
  return SCADLES_OK;
}

const Chunk* chunks_of(const scadles_adamw_plan* plan) { return reinterpret_cast<const Chunk*>((const char*)plan->table + plan->chunks_at); }

void dithers(uint64_t step, uint32_t& um, uint32_t& uv)
{
  um = (uint32_t)step * kWeylB;
  uv = (uint32_t)step * kWeylA;
}

template <class G>
void launch_norm(const Chunk* chunks, uint32_t count, Head* head, double max_norm, float* clip, hipStream_t s)
{
  const uint64_t small = div_up(count, kNormSmall / 64), blocks = div_up(count, kNormBlock / 64);
  if (small <= kNormBlocks)
    k_grad_norm<G, kNormSmall><<<small < 1 ? 1 : (uint32_t)small, kNormSmall, 0, s>>>(chunks, count, head, max_norm, clip);
  else
    k_grad_norm<G, kNormBlock><<<blocks < kNormBlocks ? (uint32_t)blocks : kNormBlocks, kNormBlock, 0, s>>>(chunks, count, head,
                                                                                                      max_norm, clip);
}

template <class G, bool kBits8>
void launch_step(const scadles_adamw_plan* plan, const StepArgs& a, const float* clip, hipStream_t s)
{
  const uint32_t grid = (uint32_t)(plan->chunks * (kChunk / kPart));
  if (clip) k_adamw<G, kBits8, true><<<grid, kBlock, 0, s>>>(chunks_of(plan), a, clip);
  else k_adamw<G, kBits8, false><<<grid, kBlock, 0, s>>>(chunks_of(plan), a, clip);
}

}  // namespace

extern "C" {

size_t scadles_adamw_plan_bytes(const scadles_adamw_tensor* tensors, uint32_t count)
{
  Layout L;
  return measure(tensors, count, L) ? 0 : (size_t)L.bytes;
}

scadles_status scadles_adamw_plan_build(const scadles_adamw_tensor* tensors, uint32_t count, int moment_bits, int grad_type,
                                        void* table, size_t table_bytes, scadles_adamw_plan* plan, void* stream)
{
  Layout L;
  if (scadles_status st = measure(tensors, count, L)) return st;
  if (moment_bits != 32 && moment_bits != 8) return fail(SCADLES_EINVAL, "moment_bits is %d, not 32 or 8", moment_bits);
  if (grad_type != SCADLES_F32 && grad_type != SCADLES_BF16) return fail(SCADLES_EINVAL, "unknown grad_type %d", grad_type);
  if (!plan) return fail(SCADLES_EINVAL, "plan is NULL");
  if (!table || !is_aligned(table, 256)) return fail(SCADLES_EWORKSPACE, "table must be 256-byte aligned and not NULL");
  if (table_bytes < L.bytes)
    return fail(SCADLES_EWORKSPACE, "table has %zu bytes, needs %zu", table_bytes, (size_t)L.bytes);
  const uint32_t gsize = grad_type == SCADLES_BF16 ? 2 : 4, msize = moment_bits / 8;
  for (uint32_t i = 0; i < count; ++i) {
    const scadles_adamw_tensor& t = tensors[i];
    if (!std::isfinite(t.weight_decay)) return fail(SCADLES_EINVAL, "tensor %u: weight_decay is not finite", i);
    if (t.n == 0) continue;
    if (!t.param || !t.grad || !t.m || !t.v) return fail(SCADLES_EINVAL, "tensor %u: param, grad, m and v must not be NULL", i);
    if ((moment_bits == 8) != (t.tops != nullptr))
      return fail(SCADLES_EINVAL, "tensor %u: tops is for 8-bit moments, and needed there", i);
    if (!is_aligned(t.param, 4) || !is_aligned(t.grad, gsize) || !is_aligned(t.m, 4) || !is_aligned(t.v, 4) ||
        !is_aligned(t.tops, 4) || !is_aligned(t.copy, 2))
      return fail(SCADLES_EINVAL, "tensor %u: a pointer is not aligned to its elements (8-bit moments: to 4 bytes)", i);
    const void* p[6] = {t.param, t.grad, t.m, t.v, t.tops, t.copy};
    const uint64_t b[6] = {t.n * 4, t.n * gsize, t.n * msize, t.n * msize, div_up(t.n, kMoment) * 4, t.n * 2};
    for (int x = 0; x < 6; ++x)
      for (int y = 0; y < x; ++y)
        if (bytes_overlap(p[x], b[x], p[y], b[y])) return fail(SCADLES_EINVAL, "tensor %u: two of its arrays overlap", i);
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  Head* head = static_cast<Head*>(table);
  Tensor* to = reinterpret_cast<Tensor*>((char*)table + L.tensors_at);
  uint64_t off = 0, first = 0;
  for (uint32_t i = 0; i < count;) {
    PutArgs a;
    a.head = head;
    a.to = to + i;
    for (a.count = 0; a.count < kPutTensors && i < count; ++a.count, ++i) {
      const scadles_adamw_tensor& t = tensors[i];
      a.t[a.count] = {t.param, t.grad, t.m, t.v, t.copy, t.tops, off, t.n, (uint32_t)first, t.weight_decay};
      off += t.n;
      first += div_up(t.n, kChunk);
    }
    k_adamw_put<<<1, kBlock, 0, s>>>(a);
  }
  if (L.chunks)
    k_adamw_chunks<<<(uint32_t)div_up(L.chunks, kBlock), kBlock, 0, s>>>(
        to, count, reinterpret_cast<Chunk*>((char*)table + L.chunks_at), (uint32_t)L.chunks, gsize, msize);
  if (scadles_status st = launch_status(hipGetLastError(), "adamw plan")) return st;
  plan->table = table;
  plan->chunks_at = L.chunks_at;
  plan->chunks = L.chunks;
  plan->n = L.n;
  plan->moment_bits = (uint32_t)moment_bits;
  plan->grad_type = (uint32_t)grad_type;
  plan->magic = kMagic;
  return SCADLES_OK;
}

scadles_status scadles_grad_norm(const scadles_adamw_plan* plan, double max_norm, float* clip, void* stream)
{
  if (scadles_status st = check_plan(plan)) return st;
  if (!(max_norm > 0.0)) return fail(SCADLES_EINVAL, "max_norm must be > 0");
  if (!clip || !is_aligned(clip, 4)) return fail(SCADLES_EINVAL, "clip must be 4-byte aligned and not NULL");
  hipStream_t s = static_cast<hipStream_t>(stream);
  const uint32_t count = (uint32_t)plan->chunks;
  Head* head = static_cast<Head*>(plan->table);
  if (plan->grad_type == SCADLES_BF16) launch_norm<uint16_t>(chunks_of(plan), count, head, max_norm, clip, s);
  else launch_norm<float>(chunks_of(plan), count, head, max_norm, clip, s);
  return launch_status(hipGetLastError(), "gradient norm");
}

scadles_status scadles_adamw_step(const scadles_adamw_plan* plan, const scadles_adamw_options* o, const float* clip, void* stream)
{
  if (scadles_status st = check_plan(plan)) return st;
  if (!o) return fail(SCADLES_EINVAL, "options is NULL");
  if (!std::isfinite(o->lr)) return fail(SCADLES_EINVAL, "lr is not finite");
  if (!(o->beta1 >= 0.0 && o->beta1 < 1.0) || !(o->beta2 >= 0.0 && o->beta2 < 1.0))
    return fail(SCADLES_EINVAL, "beta1 and beta2 must be in [0, 1)");
  if (!((float)o->eps > 0.0f) || !std::isfinite((float)o->eps)) return fail(SCADLES_EINVAL, "eps must be a float > 0");
  if (o->step == 0) return fail(SCADLES_EINVAL, "step counts from 1");
  if (clip && !is_aligned(clip, 4)) return fail(SCADLES_EINVAL, "clip must be 4-byte aligned");
  if (!plan->chunks) return SCADLES_OK;
  StepArgs a;
  const double t = (double)o->step;
  a.b1 = (float)o->beta1;
  a.c1 = (float)(1.0 - o->beta1);
  a.b2 = (float)o->beta2;
  a.c2 = (float)(1.0 - o->beta2);
  a.eps = (float)o->eps;
  a.root = (float)(1.0 / std::sqrt(1.0 - std::pow(o->beta2, t)));
  a.rate = (float)(o->lr / (1.0 - std::pow(o->beta1, t)));
  a.lr = o->lr;
  dithers(o->step, a.um, a.uv);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool half = plan->grad_type == SCADLES_BF16, small = plan->moment_bits == 8;
  if (half && small) launch_step<uint16_t, true>(plan, a, clip, s);
  else if (half) launch_step<uint16_t, false>(plan, a, clip, s);
  else if (small) launch_step<float, true>(plan, a, clip, s);
  else launch_step<float, false>(plan, a, clip, s);
  return launch_status(hipGetLastError(), "adamw step");
}

static scadles_status moments(const scadles_adamw_plan* plan, float* m, float* v, uint64_t step, bool in, void* stream)
{
  if (scadles_status st = check_plan(plan)) return st;
  if (!plan->chunks) return SCADLES_OK;
  if (!m || !v || !is_aligned(m, 4) || !is_aligned(v, 4)) return fail(SCADLES_EINVAL, "m and v must be 4-byte aligned and not NULL");
  if (bytes_overlap(m, plan->n * 4, v, plan->n * 4)) return fail(SCADLES_EINVAL, "m and v overlap");
  uint32_t um, uv;
  dithers(step, um, uv);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const uint32_t n = (uint32_t)plan->chunks, grid = (uint32_t)div_up(2 * (uint64_t)n, kWaves);
  const Chunk* c = chunks_of(plan);
  const bool small = plan->moment_bits == 8;
  if (small && in) k_adamw_moments<true, true><<<grid, kBlock, 0, s>>>(c, n, m, v, um, uv);
  else if (small) k_adamw_moments<true, false><<<grid, kBlock, 0, s>>>(c, n, m, v, um, uv);
  else if (in) k_adamw_moments<false, true><<<grid, kBlock, 0, s>>>(c, n, m, v, um, uv);
  else k_adamw_moments<false, false><<<grid, kBlock, 0, s>>>(c, n, m, v, um, uv);
  return launch_status(hipGetLastError(), "adamw moments");
}

scadles_status scadles_adamw_get_moments(const scadles_adamw_plan* plan, float* m, float* v, void* stream)
{
  return moments(plan, m, v, 0, false, stream);
}

scadles_status scadles_adamw_set_moments(const scadles_adamw_plan* plan, const float* m, const float* v, uint64_t step,
                                         void* stream)
{
  return moments(plan, const_cast<float*>(m), const_cast<float*>(v), step, true, stream);
}

}  // extern "C"
