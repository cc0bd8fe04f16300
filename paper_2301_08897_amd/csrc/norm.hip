// norm.hip -- layer norm and its gradients, those of the weights one per device.
//
//   h = (x - mean) rstd,  y = h weight + bias
//   d_x = rstd (w - mean(w) - h mean(w h)) with w = d_y weight
//   d_weight[d] = sum over device d's rows of d_y h,  d_bias[d] = sum of d_y
//
// Both directions read their rows once: a row lies in the registers of 16, 64 or
// 256 lanes, pieces of 16 bytes to a lane, so that the variance is a second pass
// over registers. A group of lanes takes row after row with the weights kept in
// registers; the backward pass keeps its columns' sums there too, adds
// those of a workgroup's groups in LDS, and k_norm_join adds the workgroups of a
// device. Rows that are too long for registers are read again from the cache,
// and their columns are summed by k_norm_columns.
// Both are bound by memory: of 131072 x 2048 bfloat16 the forward pass takes 190 us (5.6 TB/s),
// the backward pass of 32 devices 330 (4.9) and k_norm_join 12; of 64 x 256 floats each launch
// 3 to 6 us.
#include <cstring>

#include "pieces.h"
#include "vec4.h"

using namespace scadles;

namespace {

constexpr uint32_t kBackBlocks = 960;         // workgroups of a backward pass, about
constexpr uint32_t kForwardBlocks = 768;
constexpr uint32_t kJoinLanes = 64, kJoinSlices = 16;

// The weights and the rows that workgroups take.
struct Norm {
  const void *weight, *bias;
  uint64_t tokens;
  uint32_t dim, wide;         // wide: the weights are floats, else bfloat16
  float eps, inverse;         // 1 / dim
};

struct Split {
  uint64_t off[kMaxK + 1];    // device d's rows
  uint32_t first[kMaxK + 1];  // and workgroups
  uint32_t K;
};

struct Sums {
  float* w[kMaxK];
  float* b[kMaxK];
  uint32_t has_w, has_b;
};

template <class X>
__device__ inline typename Piece<X>::F weights_at(const void* p, uint32_t wide, uint32_t at, uint32_t left)
{
  typename Piece<X>::F f;
#pragma unroll
  for (uint32_t q = 0; q < Piece<X>::N; q += 4) {
    f4 x = {0, 0, 0, 0};
    if (q < left) x = wide ? load_f4((const float*)p + at + q, left - q) : load_f4((const uint16_t*)p + at + q, left - q);
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) f[q + e] = x[e];
  }
  return f;
}

// One step of a sum over lanes: what `kCtrl` brings from another lane, in the rows of
// 16 lanes that kRows names (0 elsewhere).
template <int kCtrl, int kRows>
__device__ inline float brought(float x)
{
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), kCtrl, kRows, 0xF, false));
}

// The sum of x over 16 lanes or a wave, the same in all of them.
template <int G>
__device__ inline float lanes_total(float x)
{
  x += brought<0xB1, 0xF>(x);      // lanes 1 apart
  x += brought<0x4E, 0xF>(x);      // 2 apart
  x += brought<0x141, 0xF>(x);     // the halves of 8
  x += brought<0x140, 0xF>(x);     // of 16
  if constexpr (G >= 64) {
    x += brought<0x142, 0xA>(x);   // the row before, in every second row
    x += brought<0x143, 0xC>(x);   // the lower half's last row, in the upper half
    x = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), 63));
  }
  return x;
}

// The sums of a and b over a group of G lanes; groups of more than a wave go through `lds`,
// which may be used again behind the next call with another one.
typedef float Sums2[2][kWaves];
template <int G>
__device__ inline void group_totals(float& a, float& b, Sums2& lds)
{
  a = lanes_total<G>(a);
  b = lanes_total<G>(b);
  if constexpr (G > 64) {
    if (threadIdx.x % 64 == 0) {
      lds[0][threadIdx.x / 64] = a;
      lds[1][threadIdx.x / 64] = b;
    }
    __syncthreads();
    a = b = 0.0f;
#pragma unroll
    for (int q = 0; q < G / 64; ++q) {
      a += lds[0][q];
      b += lds[1][q];
    }
  }
}

// The sum of x alike.
template <int G>
__device__ inline float group_total(float x, float* lds)
{
  x = lanes_total<G>(x);
  if constexpr (G > 64) {
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = x;
    __syncthreads();
    x = 0.0f;
#pragma unroll
    for (int q = 0; q < G / 64; ++q) x += lds[q];
  }
  return x;
}

template <class F>
__device__ inline F fused(F x, F y, F z)
{
  return __builtin_elementwise_fma(x, y, z);
}

template <class F>
__device__ inline float sum_of(F f, uint32_t n)
{
  float s = f[0];
#pragma unroll
  for (uint32_t q = 1; q < n; ++q) s += f[q];
  return s;
}

// The pieces of a row as loaded by load_raw; one branch for all of them.
template <class X, int G, int P>
__device__ inline void settle_row(u4 (&v)[P], uint32_t lane, uint32_t dim)
{
  if (dim % Piece<X>::N == 0) return;
#pragma unroll
  for (int j = 0; j < P; ++j) {
    const uint32_t at = (lane + j * G) * Piece<X>::N;
    if (at < dim) v[j] = settled<X>(v[j], at, dim);
  }
}

// A row in P pieces of each of G lanes.
template <class X, int G, int P>
__global__ __launch_bounds__(kBlock) void k_norm(Norm m, const X* x, uint64_t ld_x, X* y, uint64_t ld_y, float* mean_out, float* rstd_out)
{
  constexpr uint32_t N = Piece<X>::N;
  typedef typename Piece<X>::F F;
  __shared__ float lds[2][kWaves];
  const uint32_t lane = threadIdx.x % G, groups = kBlock / G;
  F w[P], b[P];
#pragma unroll
  for (int j = 0; j < P; ++j) {
    const uint32_t at = (lane + j * G) * N, left = at < m.dim ? m.dim - at : 0;
    w[j] = weights_at<X>(m.weight, m.wide, at, left);
    b[j] = m.bias ? weights_at<X>(m.bias, m.wide, at, left) : F{};
  }
  const uint64_t step = (uint64_t)gridDim.x * groups;
  u4 next[P];
  auto load = [&](uint64_t t) {
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const uint32_t at = (lane + j * G) * N;
      next[j] = t < m.tokens && at < m.dim ? load_raw(x + t * ld_x, at, m.dim) : u4{0, 0, 0, 0};
    }
  };
  uint64_t t = (uint64_t)blockIdx.x * groups + threadIdx.x / G;
  load(t);
  for (; t < m.tokens; t += step) {
    F v[P];
    float sum = 0.0f;
    settle_row<X, G, P>(next, lane, m.dim);
#pragma unroll
    for (int j = 0; j < P; ++j) {
      v[j] = unpack<X>(next[j]);
      sum += sum_of(v[j], N);
    }
    load(t + step);                // under this row's sums
    const float mean = group_total<G>(sum, lds[0]) * m.inverse;
    float square = 0.0f;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const uint32_t at = (lane + j * G) * N;
#pragma unroll
      for (uint32_t q = 0; q < N; ++q) {
        const float c = v[j][q] - mean;
        v[j][q] = c;
        square = at + q < m.dim ? __builtin_fmaf(c, c, square) : square;
      }
    }
    const float rstd = 1.0f / __builtin_sqrtf(group_total<G>(square, lds[1]) * m.inverse + m.eps);
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const uint32_t at = (lane + j * G) * N;
      if (at < m.dim) store_piece(y + t * ld_y + at, pack<X>(fused(v[j] * rstd, w[j], b[j])), m.dim - at);
    }
    if (lane == 0) {
      gptr(mean_out)[t] = mean;
      gptr(rstd_out)[t] = rstd;
    }
  }
}

// A row that is longer than that: a workgroup reads it three times.
template <class X>
__global__ __launch_bounds__(kBlock) void k_norm_long(Norm m, const X* x, uint64_t ld_x, X* y, uint64_t ld_y, float* mean_out, float* rstd_out)
{
  constexpr uint32_t N = Piece<X>::N;
  __shared__ float lds[2][kWaves];
  const uint64_t t = blockIdx.x;     // fewer than 2^24 rows this long fit in memory
  const X* row = x + t * ld_x;
  float sum = 0.0f, square = 0.0f;
  for (uint32_t at = threadIdx.x * N; at < m.dim; at += kBlock * N) sum += sum_of(unpack<X>(load_piece(row, at, m.dim)), N);
  const float mean = group_total<kBlock>(sum, lds[0]) * m.inverse;
  for (uint32_t at = threadIdx.x * N; at < m.dim; at += kBlock * N) {
    const auto v = unpack<X>(load_piece(row, at, m.dim));
#pragma unroll
    for (uint32_t q = 0; q < N; ++q) {
      const float c = v[q] - mean;
      square = at + q < m.dim ? __builtin_fmaf(c, c, square) : square;
    }
  }
  const float rstd = 1.0f / __builtin_sqrtf(group_total<kBlock>(square, lds[1]) * m.inverse + m.eps);
  for (uint32_t at = threadIdx.x * N; at < m.dim; at += kBlock * N) {
    const uint32_t left = m.dim - at;
    auto v = (unpack<X>(load_piece(row, at, m.dim)) - mean) * rstd * weights_at<X>(m.weight, m.wide, at, left);
    if (m.bias) v += weights_at<X>(m.bias, m.wide, at, left);
    store_piece(y + t * ld_y + at, pack<X>(v), left);
  }
  if (threadIdx.x == 0) {
    gptr(mean_out)[t] = mean;
    gptr(rstd_out)[t] = rstd;
  }
}

// ---- backward -------------------------------------------------------------------------------------

__device__ inline uint32_t device_of(const Split& s, uint32_t w)
{
  uint32_t d = 0;
  while (d + 1 < s.K && s.first[d + 1] <= w) ++d;
  return d;
}

// Where a workgroup's sums of a column go: to the device's, if it has no other
// workgroup, or to its place in the workspace.
__device__ inline float* sums_at(const Split& s, const Sums& o, uint32_t d, float* part, uint32_t width, uint32_t which)
{
  if (s.first[d + 1] - s.first[d] == 1) return which ? o.b[d] : o.w[d];
  return part + ((uint64_t)blockIdx.x * 2 + which) * width;
}

template <class X, int G, int P>
__global__ __launch_bounds__(kBlock) void k_norm_back(Norm m, Split s, Sums o, const X* x, uint64_t ld_x, const float* mean_in, const float* rstd_in,
                                                      const X* dy, uint64_t ld_dy, X* dx, uint64_t ld_dx, float* part, uint32_t width)
{
  constexpr uint32_t N = Piece<X>::N, groups = kBlock / G;
  typedef typename Piece<X>::F F;
  __shared__ Sums2 lds[2];
  uint32_t turn = 0;
  __shared__ F over[groups > 1 ? G * groups : 1];
  const uint32_t lane = threadIdx.x % G, group = threadIdx.x / G, d = device_of(s, blockIdx.x);
  // the device's workgroups take its rows in turn
  const uint64_t t0 = s.off[d] + (uint64_t)(blockIdx.x - s.first[d]) * groups + group, t1 = s.off[d + 1];
  const uint64_t step = (uint64_t)(s.first[d + 1] - s.first[d]) * groups;
  F w[P], sw[P], sb[P];
#pragma unroll
  for (int j = 0; j < P; ++j) {
    const uint32_t at = (lane + j * G) * N, left = at < m.dim ? m.dim - at : 0;
    w[j] = weights_at<X>(m.weight, m.wide, at, left);
    sw[j] = F{};
    sb[j] = F{};
  }
  u4 next_x[P], next_g[P];
  float next_mean = 0.0f, next_rstd = 0.0f;
  auto load = [&](uint64_t t) {
    const bool there = t < t1;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const uint32_t at = (lane + j * G) * N;
      const bool on = there && at < m.dim;
      next_x[j] = on ? load_raw(x + t * ld_x, at, m.dim) : u4{0, 0, 0, 0};
      next_g[j] = on ? load_raw(dy + t * ld_dy, at, m.dim) : u4{0, 0, 0, 0};
    }
    if (there) {
      next_mean = gptr(mean_in)[t];
      next_rstd = gptr(rstd_in)[t];
    }
  };
  load(t0);
  for (uint64_t t = t0; t < t1; t += step) {
    const float mean = next_mean, rstd = next_rstd;
    F h[P], g[P];
    float a = 0.0f, b = 0.0f;
    settle_row<X, G, P>(next_x, lane, m.dim);
    settle_row<X, G, P>(next_g, lane, m.dim);
#pragma unroll
    for (int j = 0; j < P; ++j) {
      h[j] = unpack<X>(next_x[j]);
      g[j] = unpack<X>(next_g[j]);
    }
    load(t + step);                // under this row's sums
#pragma unroll
    for (int j = 0; j < P; ++j) {       // what lies behind the row has d_y = 0 and adds nothing
      h[j] = (h[j] - mean) * rstd;
      sw[j] = fused(g[j], h[j], sw[j]);
      sb[j] += g[j];
      g[j] *= w[j];
#pragma unroll
      for (uint32_t q = 0; q < N; ++q) {
        a += g[j][q];
        b = __builtin_fmaf(g[j][q], h[j][q], b);
      }
    }
    group_totals<G>(a, b, lds[turn]);
    turn ^= 1;
    a *= m.inverse;
    b *= m.inverse;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const uint32_t at = (lane + j * G) * N;
      if (at < m.dim) store_piece(dx + t * ld_dx + at, pack<X>(fused(-h[j], F{} + b, g[j] - a) * rstd), m.dim - at);
    }
  }
  for (uint32_t which = 0; which < 2; ++which) {
    if (!(which ? o.has_b : o.has_w)) continue;
    float* to = sums_at(s, o, d, part, width, which);
#pragma unroll
    for (int j = 0; j < P; ++j) {
      F sum = which ? sb[j] : sw[j];
      if constexpr (groups > 1) {
        __syncthreads();
        over[group * G + lane] = sum;
        __syncthreads();
        for (uint32_t q = 1; q < groups; ++q) sum += group ? F{} : over[q * G + lane];
      }
      const uint32_t at = (lane + j * G) * N;
      if (group == 0)
#pragma unroll
        for (uint32_t q = 0; q < N; q += 4)
          if (at + q < m.dim) store_f4(to + at + q, f4{sum[q], sum[q + 1], sum[q + 2], sum[q + 3]}, m.dim - at - q);
    }
  }
}

template <class X>
__global__ __launch_bounds__(kBlock) void k_norm_back_long(Norm m, const X* x, uint64_t ld_x, const float* mean_in, const float* rstd_in,
                                                           const X* dy, uint64_t ld_dy, X* dx, uint64_t ld_dx)
{
  constexpr uint32_t N = Piece<X>::N;
  __shared__ float lds[2][kWaves];
  const uint64_t t = blockIdx.x;
  const float mean = gptr(mean_in)[t], rstd = gptr(rstd_in)[t];
  float a = 0.0f, b = 0.0f;
  auto both = [&](uint32_t at, auto& h, auto& g) {
    const uint32_t left = m.dim - at;
    h = (unpack<X>(load_piece(x + t * ld_x, at, m.dim)) - mean) * rstd;
    g = unpack<X>(load_piece(dy + t * ld_dy, at, m.dim)) * weights_at<X>(m.weight, m.wide, at, left);
  };
  typename Piece<X>::F h, g;
  for (uint32_t at = threadIdx.x * N; at < m.dim; at += kBlock * N) {
    both(at, h, g);
    a += sum_of(g, N);
    b += sum_of(g * h, N);
  }
  a = group_total<kBlock>(a, lds[0]) * m.inverse;
  b = group_total<kBlock>(b, lds[1]) * m.inverse;
  for (uint32_t at = threadIdx.x * N; at < m.dim; at += kBlock * N) {
    both(at, h, g);
    store_piece(dx + t * ld_dx + at, pack<X>((g - a - h * b) * rstd), m.dim - at);
  }
}

// The columns' sums of long rows: a lane has a piece of the columns.
template <class X>
__global__ __launch_bounds__(kBlock) void k_norm_columns(Norm m, Split s, Sums o, const X* x, uint64_t ld_x, const float* mean_in,
                                                         const float* rstd_in, const X* dy, uint64_t ld_dy, float* part, uint32_t width)
{
  constexpr uint32_t N = Piece<X>::N;
  typedef typename Piece<X>::F F;
  const uint32_t at = (blockIdx.y * kBlock + threadIdx.x) * N;
  if (at >= m.dim) return;
  const uint32_t left = m.dim - at, d = device_of(s, blockIdx.x);
  const uint64_t t0 = s.off[d] + (blockIdx.x - s.first[d]), step = s.first[d + 1] - s.first[d];
  F sw = {}, sb = {};
#pragma unroll 4
  for (uint64_t t = t0; t < s.off[d + 1]; t += step) {
    const F g = unpack<X>(load_piece(dy + t * ld_dy, at, m.dim));
    sw += g * ((unpack<X>(load_piece(x + t * ld_x, at, m.dim)) - gptr(mean_in)[t]) * gptr(rstd_in)[t]);
    sb += g;
  }
  for (uint32_t which = 0; which < 2; ++which) {
    if (!(which ? o.has_b : o.has_w)) continue;
    float* to = sums_at(s, o, d, part, width, which);
    const F sum = which ? sb : sw;
#pragma unroll
    for (uint32_t q = 0; q < N; q += 4)
      if (q < left) store_f4(to + at + q, f4{sum[q], sum[q + 1], sum[q + 2], sum[q + 3]}, left - q);
  }
}

// Adds the workgroups of a device: 64 columns, 16 slices of the workgroups. A device
// without rows gets zeros.
__global__ __launch_bounds__(kJoinLanes* kJoinSlices) void k_norm_join(Split s, Sums o, const float* part, uint32_t width, uint32_t dim)
{
  __shared__ float slice[kJoinSlices][kJoinLanes];
  const uint32_t d = blockIdx.y, which = blockIdx.z, lane = threadIdx.x % kJoinLanes, z = threadIdx.x / kJoinLanes;
  const uint32_t c = blockIdx.x * kJoinLanes + lane, lo = s.first[d], hi = s.first[d + 1];
  if (hi - lo == 1 || !(which ? o.has_b : o.has_w)) return;
  float sum = 0.0f;
  if (c < dim) {
#pragma unroll 8
    for (uint32_t w = lo + z; w < hi; w += kJoinSlices) sum += gptr(part)[((uint64_t)w * 2 + which) * width + c];
  }
  slice[z][lane] = sum;
  __syncthreads();
  if (z || c >= dim) return;
#pragma unroll
  for (uint32_t q = 1; q < kJoinSlices; ++q) sum += slice[q][lane];
  gptr(which ? o.b[d] : o.w[d])[c] = sum;
}

// ---- host -------------------------------------------------------------------------------------------

uint64_t size_of(int32_t type) { return type == SCADLES_BF16 ? 2 : 4; }

// Calls f with the lanes of a row and the pieces of a lane; false where the row is too
// long. `most` floats of a row to a lane.
template <class X, int kMost, class F>
bool with_row(uint32_t dim, F f)
{
  const uint32_t p = (uint32_t)div_up(dim, Piece<X>::N);
  constexpr int N = Piece<X>::N;
  auto go = [&](auto g, auto n) {
    if constexpr (n * N <= kMost) f(g, n);
    return n * N <= kMost;
  };
#define SCADLES_ROW(G, P) \
  if (p <= G * P && P * N <= kMost) return go(std::integral_constant<int, G>(), std::integral_constant<int, P>())
  SCADLES_ROW(16, 1);
  SCADLES_ROW(64, 1);
  SCADLES_ROW(64, 2);
  SCADLES_ROW(64, 4);
  SCADLES_ROW(256, 1);
  SCADLES_ROW(256, 2);
  SCADLES_ROW(256, 4);
  SCADLES_ROW(256, 8);
#undef SCADLES_ROW
  return false;
}

template <class X>
hipError_t forward(const Norm& m, const void* x, uint64_t ld_x, void* y, uint64_t ld_y, float* mean, float* rstd, hipStream_t st)
{
  const bool done = with_row<X, 32>(m.dim, [&](auto g, auto p) {
    uint64_t blocks = div_up(m.tokens, kBlock / g);
    if (blocks > kForwardBlocks) blocks = kForwardBlocks;
    k_norm<X, g, p><<<(uint32_t)blocks, kBlock, 0, st>>>(m, (const X*)x, ld_x, (X*)y, ld_y, mean, rstd);
  });
  if (!done) k_norm_long<X><<<(uint32_t)m.tokens, kBlock, 0, st>>>(m, (const X*)x, ld_x, (X*)y, ld_y, mean, rstd);
  return hipGetLastError();
}

// Rows of a workgroup: a few for every group of lanes, so that about kBackBlocks
// workgroups share them; returns the workgroups.
uint32_t split_rows(const scadles_batch* b, Split& s)
{
  std::memset(&s, 0, sizeof(s));
  s.K = b->devices;
  uint64_t per = div_up(b->tokens, kBackBlocks);
  if (per < 16) per = 16;
  uint64_t w = 0;
  for (uint32_t d = 0; d < s.K; ++d) {
    s.off[d] = b->tok_off[d];
    s.first[d] = (uint32_t)w;
    w += div_up(b->tok_off[d + 1] - b->tok_off[d], per);
  }
  s.off[s.K] = b->tokens;
  s.first[s.K] = (uint32_t)w;
  return (uint32_t)w;
}

uint32_t width_of(uint32_t dim) { return (uint32_t)div_up(dim, 4) * 4; }

template <class X>
hipError_t backward(const Norm& m, const Split& s, const Sums& o, uint32_t W, const void* x, uint64_t ld_x, const float* mean, const float* rstd,
                    const void* dy, uint64_t ld_dy, void* dx, uint64_t ld_dx, float* part, hipStream_t st)
{
  const uint32_t width = width_of(m.dim);
  if (W) {
    // 16 floats of a row to a lane, so that several workgroups share a compute unit (131072 x 2048
    // bfloat16: 330 us; 32 in a wave: 366), 32 for longer rows
    auto launch = [&](auto g, auto p) {
      k_norm_back<X, g, p><<<W, kBlock, 0, st>>>(m, s, o, (const X*)x, ld_x, mean, rstd, (const X*)dy, ld_dy, (X*)dx, ld_dx, part, width);
    };
    if (!with_row<X, 16>(m.dim, launch) && !with_row<X, 32>(m.dim, launch)) {
      k_norm_back_long<X><<<(uint32_t)m.tokens, kBlock, 0, st>>>(m, (const X*)x, ld_x, mean, rstd, (const X*)dy, ld_dy, (X*)dx, ld_dx);
      if (o.has_w || o.has_b)
        k_norm_columns<X><<<dim3(W, (uint32_t)div_up(div_up(m.dim, Piece<X>::N), kBlock)), kBlock, 0, st>>>(
            m, s, o, (const X*)x, ld_x, mean, rstd, (const X*)dy, ld_dy, part, width);
    }
  }
  bool join = false;
  for (uint32_t d = 0; d < s.K; ++d) join |= s.first[d + 1] - s.first[d] != 1;
  if (join && (o.has_w || o.has_b))
    k_norm_join<<<dim3((uint32_t)div_up(m.dim, kJoinLanes), s.K, 2), kJoinLanes * kJoinSlices, 0, st>>>(s, o, part, width, m.dim);
  return hipGetLastError();
}

scadles_status check_norm(const scadles_norm* n)
{
  if (!n) return fail(SCADLES_EINVAL, "norm is NULL");
  if (!n->dim || n->dim >= 1u << 24) return fail(SCADLES_EINVAL, "dim = %u is outside [1, 2^24)", n->dim);
  if ((n->type != SCADLES_F32 && n->type != SCADLES_BF16) || (n->weight_type != SCADLES_F32 && n->weight_type != SCADLES_BF16))
    return fail(SCADLES_EINVAL, "unknown type %d or weight_type %d", n->type, n->weight_type);
  if (!(n->eps - n->eps == 0.0f) || n->eps < 0.0f) return fail(SCADLES_EINVAL, "eps is negative or not finite");
  return SCADLES_OK;
}

// An array of an operator's call and its bytes.
struct Range {
  const void* p;
  uint64_t bytes;
};

bool any_overlap(const Range& a, std::initializer_list<Range> others)
{
  for (const Range& b : others)
    if (bytes_overlap(a.p, a.bytes, b.p, b.bytes)) return true;
  return false;
}

}  // namespace

extern "C" {

scadles_status scadles_layer_norm_forward(const scadles_norm* norm, uint64_t tokens, const void* x, uint64_t ld_x, const void* weight,
                                          const void* bias, void* y, uint64_t ld_y, float* mean, float* rstd, void* stream)
{
  if (scadles_status st = check_norm(norm)) return st;
  if (tokens > 0x7FFFFFFFull) return fail(SCADLES_EINVAL, "more than 2^31 - 1 tokens");
  if (!weight || (tokens && (!x || !y || !mean || !rstd))) return fail(SCADLES_EINVAL, "x, weight, y, mean and rstd must not be NULL");
  const uint64_t es = size_of(norm->type), wsz = size_of(norm->weight_type), dim = norm->dim;
  if (!is_aligned(x, es) || !is_aligned(y, es) || !is_aligned(weight, wsz) || !is_aligned(bias, wsz) || !is_aligned(mean, 4) || !is_aligned(rstd, 4))
    return fail(SCADLES_EINVAL, "an array is not aligned to its elements");
  if (ld_x < dim || ld_y < dim || ld_x >= 1ull << 31 || ld_y >= 1ull << 31)
    return fail(SCADLES_EINVAL, "ld_x or ld_y is smaller than dim, or 2^31 or more");
  const Range rx = {x, rows_bytes(tokens, dim, ld_x, es)}, rw = {weight, dim * wsz}, rb = {bias, dim * wsz};
  const Range ry = {y, rows_bytes(tokens, dim, ld_y, es)}, rm = {mean, tokens * 4}, rr = {rstd, tokens * 4};
  if (any_overlap(ry, {rx, rw, rb, rm, rr}) || any_overlap(rm, {rx, rw, rb, rr}) || any_overlap(rr, {rx, rw, rb}))
    return fail(SCADLES_EINVAL, "an output overlaps an input or another");
  if (!tokens) return SCADLES_OK;
  const Norm m = {weight, bias, tokens, norm->dim, norm->weight_type == SCADLES_F32, norm->eps, (float)(1.0 / (double)dim)};
  hipStream_t st = static_cast<hipStream_t>(stream);
  return launch_status(norm->type == SCADLES_BF16 ? forward<uint16_t>(m, x, ld_x, y, ld_y, mean, rstd, st)
                                                  : forward<float>(m, x, ld_x, y, ld_y, mean, rstd, st),
                       "layer norm forward");
}

size_t scadles_layer_norm_workspace_bytes(uint64_t tokens, uint32_t dim)
{
  if (tokens > 0x7FFFFFFFull || !dim || dim >= 1u << 24) return 0;
  const uint64_t W = (tokens / 16 < kBackBlocks ? tokens / 16 : kBackBlocks) + kMaxK;
  return (size_t)(W * 2 * width_of(dim) * 4);
}

scadles_status scadles_layer_norm_backward(const scadles_norm* norm, const scadles_batch* batch, const void* x, uint64_t ld_x, const void* weight,
                                           const float* mean, const float* rstd, const void* d_y, uint64_t ld_d_y, void* d_x, uint64_t ld_d_x,
                                           float* const* d_weight, float* const* d_bias, void* ws, size_t ws_bytes, void* stream)
{
  if (scadles_status st = check_norm(norm)) return st;
  if (scadles_status st = check_batch(batch)) return st;
  const uint64_t T = batch->tokens, dim = norm->dim, es = size_of(norm->type), wsz = size_of(norm->weight_type);
  if (!weight || (T && (!x || !d_y || !d_x || !mean || !rstd))) return fail(SCADLES_EINVAL, "x, weight, mean, rstd, d_y and d_x must not be NULL");
  if (!is_aligned(x, es) || !is_aligned(d_y, es) || !is_aligned(d_x, es) || !is_aligned(weight, wsz) || !is_aligned(mean, 4) || !is_aligned(rstd, 4))
    return fail(SCADLES_EINVAL, "an array is not aligned to its elements");
  for (uint64_t ld : {ld_x, ld_d_y, ld_d_x})
    if (ld < dim || ld >= 1ull << 31) return fail(SCADLES_EINVAL, "an ld is smaller than dim, or 2^31 or more");
  Split s;
  const uint32_t W = split_rows(batch, s);
  const uint64_t need = (uint64_t)W * 2 * width_of(norm->dim) * 4;
  if (!ws || !is_aligned(ws, 256)) return fail(SCADLES_EWORKSPACE, "workspace must be 256-byte aligned and not NULL");
  if (ws_bytes < need) return fail(SCADLES_EWORKSPACE, "workspace has %zu bytes, needs %zu", ws_bytes, (size_t)need);
  const Range rx = {x, rows_bytes(T, dim, ld_x, es)}, rw = {weight, dim * wsz}, rm = {mean, T * 4}, rr = {rstd, T * 4};
  const Range rg = {d_y, rows_bytes(T, dim, ld_d_y, es)}, ro = {d_x, rows_bytes(T, dim, ld_d_x, es)}, rs = {ws, need};
  if (any_overlap(ro, {rx, rw, rm, rr, rg, rs}) || any_overlap(rs, {rx, rw, rm, rr, rg}))
    return fail(SCADLES_EINVAL, "d_x or the workspace overlaps an input or the other");
  Sums o;
  std::memset(&o, 0, sizeof(o));
  o.has_w = d_weight != nullptr;
  o.has_b = d_bias != nullptr;
  for (uint32_t d = 0; d < batch->devices; ++d)
    for (int which = 0; which < 2; ++which) {
      if (!(which ? o.has_b : o.has_w)) continue;
      float* p = which ? d_bias[d] : d_weight[d];
      const Range r = {p, dim * 4};
      if (!p || !is_aligned(p, 4)) return fail(SCADLES_EINVAL, "a gradient of device %u is NULL or not 4-byte aligned", d);
      if (any_overlap(r, {rx, rw, rm, rr, rg, ro, rs})) return fail(SCADLES_EINVAL, "a gradient of device %u overlaps another array", d);
      for (uint32_t c = 0; c <= d; ++c)
        for (int other = 0; other < 2; ++other) {
          if ((c == d && other >= which) || !(other ? o.has_b : o.has_w)) continue;
          if (any_overlap(r, {{other ? d_bias[c] : d_weight[c], dim * 4}})) return fail(SCADLES_EINVAL, "gradients of devices %u and %u overlap", c, d);
        }
      (which ? o.b : o.w)[d] = p;
    }
  const Norm m = {weight, nullptr, T, norm->dim, norm->weight_type == SCADLES_F32, norm->eps, (float)(1.0 / (double)dim)};
  hipStream_t st = static_cast<hipStream_t>(stream);
  float* part = static_cast<float*>(ws);
  return launch_status(norm->type == SCADLES_BF16 ? backward<uint16_t>(m, s, o, W, x, ld_x, mean, rstd, d_y, ld_d_y, d_x, ld_d_x, part, st)
                                                  : backward<float>(m, s, o, W, x, ld_x, mean, rstd, d_y, ld_d_y, d_x, ld_d_x, part, st),
                       "layer norm backward");
}

}  // extern "C"
