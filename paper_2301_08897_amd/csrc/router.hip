// router.hip -- the router of a mixture of experts whose tokens lie on K devices:
// softmax, Top-k choice, gates, expert counts, the balance loss and the z loss
// over all devices, and the gradient of the logits.
//
// Row t of device d (weight w_d, n_d counted rows), E experts, k choices:
//   p = softmax(x), lse = log sum exp(x), S = the k largest x (ties: the lower index)
//   gate = p over S, or p over S divided by its sum
//   load_e = sum_d w_d / (k n_d) * c_de,   prob_e = sum_d w_d / n_d * sum_t p_te
//   balance = E sum_e load_e prob_e,       z = sum_d w_d / n_d * sum_t lse^2
// Backward (load is a constant), a and b the losses' incoming gradients:
//   dx = w_d / n_d * p (a E (load - sum_j load_j p_j) + 2 b lse) + the gates' part,
//   which is gate (dgate - sum gate dgate) over S, or p (dgate over S - sum gate dgate).
//
// Both directions read the logits once. A row lies in the registers of a group
// of G lanes, V elements each (see with_shape), so that its maximum, sums and
// choices are a few lane exchanges; a workgroup takes several rounds of 256 / G
// rows of one device and keeps the experts' probability sums in registers
// meanwhile.
#include <cmath>
#include <cstring>
#include <type_traits>

#include "abi.h"
#include "radix.h"
#include "vec4.h"

using namespace scadles;

namespace {

constexpr uint32_t kMaxChoices = SCADLES_ROUTER_MAX_K;
constexpr uint32_t kMaxExperts = SCADLES_ROUTER_MAX_EXPERTS;
constexpr uint32_t kFinishExperts = 16;    // experts of one workgroup of k_route_finish
constexpr int kFinishBlock = 1024;
constexpr int kFewLanes = 16;              // lanes per row from which choices are made by a threshold,
constexpr uint32_t few_from(int G) { return G < 64 ? 3 : 4; }    // if there are so many (see choose_few)
constexpr uint32_t kRouteBlocks = 1024;    // workgroups, at most, unless they would take
constexpr uint32_t kBackBlocks = 1280;     // the same for the backward pass, which has no sums
constexpr uint32_t kMaxRounds = 256;       // more rounds each than this: they sum probabilities in float
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// Where the rows lie and what workgroup takes which.
struct Rows {
  uint64_t off[kMaxK + 1];     // device d's rows are [off[d], off[d + 1])
  uint32_t first[kMaxK + 1];   // and its workgroups [first[d], first[d + 1])
  float w[kMaxK];
  uint64_t ld;                 // elements between rows of logits
  uint32_t E, k, K, per;       // per: rows of one workgroup
  uint32_t renormalise;
};

// What the workgroups leave for the sums over all rows.
struct Cell {
  uint32_t count;              // choices of an expert
  float prob;                  // and the sum of its probabilities
};

struct Parts {
  Cell* cell;                  // [W][E]
  double* z;                   // [W] sums of lse^2
  uint32_t* rows;              // [W] counted rows
  double* balance;             // [finishing workgroups]
  uint32_t* ticket;
  uint32_t W;
};

struct RouteOut {
  int32_t* idx;
  float* gate;
  float* lse;
  int32_t* counts;
  float* load;
  float* share;
  float* loss;
};

// ---- exchanges within a group of G lanes ------------------------------------------------------
template <int kCtrl>
__device__ inline uint32_t dpp(uint32_t x)
{
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kCtrl, 0xF, 0xF, true);
}

// Combines x over the group; every lane ends with the same value, in the same
// pattern of operations whatever the data. `step` combines with the lane that
// the given exchange names.
template <int G, class Step, class Far>
__device__ inline float group_reduce(float x, Step step, Far far)
{
  if constexpr (G >= 2) x = step(x, std::integral_constant<int, 0xB1>());    // lanes 1 apart
  if constexpr (G >= 4) x = step(x, std::integral_constant<int, 0x4E>());    // 2 apart
  if constexpr (G >= 8) x = step(x, std::integral_constant<int, 0x141>());   // the halves of 8
  if constexpr (G >= 16) x = step(x, std::integral_constant<int, 0x140>());  // of 16
  if constexpr (G >= 32) x = far(x, __shfl_xor(x, 16, 64));
  if constexpr (G >= 64) x = far(x, __shfl_xor(x, 32, 64));
  return x;
}

// One instruction with the exchange in it; the compiler would put a move and a
// second maximum (against signalling NaN) before it. It waits for x itself.
#define SCADLES_DPP_STEP(op, how) asm volatile("s_nop 1\n\t" op " %0, %1, %1 " how " row_mask:0xf bank_mask:0xf" : "=v"(y) : "v"(x))
#define SCADLES_DPP_OP(op)                                            \
  [](float x, auto ctrl) {                                            \
    float y;                                                          \
    if constexpr (ctrl == 0xB1) SCADLES_DPP_STEP(op, "quad_perm:[1,0,3,2]"); \
    else if constexpr (ctrl == 0x4E) SCADLES_DPP_STEP(op, "quad_perm:[2,3,0,1]"); \
    else if constexpr (ctrl == 0x141) SCADLES_DPP_STEP(op, "row_half_mirror"); \
    else SCADLES_DPP_STEP(op, "row_mirror");                          \
    return y;                                                         \
  }

template <int G>
__device__ inline float group_max(float x)
{
  return group_reduce<G>(x, SCADLES_DPP_OP("v_max_f32_dpp"), [](float a, float b) { return __builtin_fmaxf(a, b); });
}

template <int G>
__device__ inline float group_least(float x)
{
  return group_reduce<G>(x, SCADLES_DPP_OP("v_min_f32_dpp"), [](float a, float b) { return __builtin_fminf(a, b); });
}

template <int G>
__device__ inline float group_sum(float x)
{
  return group_reduce<G>(x, [](float a, auto ctrl) { return a + __uint_as_float(dpp<ctrl>(__float_as_uint(a))); },
                         [](float a, float b) { return a + b; });
}

template <int G>
__device__ inline uint32_t group_min(uint32_t x)
{
  auto least = [](uint32_t u, uint32_t v) { return __uint_as_float(u < v ? u : v); };
  return __float_as_uint(group_reduce<G>(__uint_as_float(x),
                                         [&](float a, auto ctrl) { return least(__float_as_uint(a), dpp<ctrl>(__float_as_uint(a))); },
                                         [&](float a, float b) { return least(__float_as_uint(a), __float_as_uint(b)); }));
}

// The sum of x over the lanes of a row of 16 that have the same place in their group.
template <int G>
__device__ inline float sum_over_row(float x)
{
  auto add = [](float a, uint32_t b) { return a + __uint_as_float(b); };
  if constexpr (G <= 8) x = add(x, dpp<0x128>(__float_as_uint(x)));    // turned by 8 lanes, by 4
  if constexpr (G <= 4) x = add(x, dpp<0x124>(__float_as_uint(x)));
  if constexpr (G <= 2) x = add(x, dpp<0x4E>(__float_as_uint(x)));
  if constexpr (G <= 1) x = add(x, dpp<0xB1>(__float_as_uint(x)));
  return x;
}

__device__ inline float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// exp(x - mid) of a row, as 2^(x log2 e - mid log2 e) with one rounding for the
// product and the difference; the rounding of mid log2 e is a factor of the
// whole row and cancels in its probabilities. Below kFar it is within 2^(1/16) of
// one (half a unit of a number below 2^21) and moves lse by less than lse's own
// rounding; beyond, where it would pass the range of a float, the exponential
// is that of the difference (`far`).
constexpr float kFar = 0x1p20f;

struct Exp {
  float mid, c;
  bool far;
  __device__ inline float operator()(float x) const
  {
    return far ? exp_of(x - mid) : __builtin_amdgcn_exp2f(__builtin_fmaf(x, kLog2e, -c));
  }
};

// Orders LDS accesses of the lanes of a wave, which run in step: only the
// compiler has to keep their order.
__device__ inline void wave_sync()
{
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The device whose workgroups include w, and the rows of that workgroup. Every
// lane loads a device's bounds, so that the arguments are waited for once.
struct Share {
  uint32_t d;
  uint64_t row0, row1;
};

__device__ inline uint64_t lane_value(uint64_t x, uint32_t l)
{
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, l);
}

__device__ inline Share share_of(const Rows& r, uint32_t w)
{
  const uint32_t l = lane_id(), dl = l < r.K ? l : r.K - 1;
  const uint32_t first = r.first[dl], next = r.first[dl + 1];
  const uint64_t begin = r.off[dl], end = r.off[dl + 1];
  Share s;
  s.d = (uint32_t)__builtin_popcountll(__ballot(l < r.K && next <= w));    // devices that end before w
  s.row0 = lane_value(begin, s.d) + (uint64_t)(w - (uint32_t)__builtin_amdgcn_readlane((int)first, s.d)) * r.per;
  const uint64_t stop = lane_value(end, s.d);
  s.row1 = s.row0 + r.per < stop ? s.row0 + r.per : stop;
  return s;
}

// Element i of a lane's V is expert 4 (G (i / 4) + lane) + i % 4: 16 bytes of
// every lane side by side.
template <int G>
__device__ constexpr uint32_t expert_at(int i) { return (uint32_t)(4 * G * (i / 4) + i % 4); }
template <int G>
__device__ inline uint32_t expert_of(uint32_t i, uint32_t l4) { return (i >> 2) * (4 * G) + (i & 3u) + l4; }

template <class X, int G, int V>
__device__ inline void load_row(float (&x)[V], const X* row, uint32_t l4, uint32_t E, bool on)
{
  if (!on) {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = -__builtin_inff();
    return;
  }
  const X* p = row + l4;
#pragma unroll
  for (int j = 0; j < V / 4; ++j) {
    uint32_t k = 4;
    if (expert_at<G>(4 * j + 4) > E) {         // not all lanes have four elements here
      const uint32_t e = expert_at<G>(4 * j) + l4;
      k = e < E ? E - e : 0u;
    }
    const f4 v = load_once_f4(p + expert_at<G>(4 * j), k, -__builtin_inff());
#pragma unroll
    for (int q = 0; q < 4; ++q) x[4 * j + q] = v[q];
  }
}

// ---- the sums over all rows ---------------------------------------------------------------------
// Experts [16 b, 16 b + 16), a line of the workgroups' results (8 experts and 512
// threads: 9.4 us for 256 experts, so 9.0). Every slice of 16 threads adds a run of the
// workgroups' results in order, kAhead loaded at once; then the slices are added
// in a fixed pattern.
struct FinishLds {
  static constexpr int NT = kFinishBlock;
  uint32_t first[kMaxK + 1];
  uint32_t rows[kMaxK];
  double scale[kMaxK];
  uint32_t count[kMaxK][kFinishExperts];
  double load[NT / 64][kFinishExperts], prob[NT / 64][kFinishExperts];
  double z[NT / 64];
};

// The device whose workgroups include w, from the table in LDS.
__device__ inline uint32_t device_in(const uint32_t* first, uint32_t K, uint32_t w)
{
  uint32_t lo = 0, hi = K;
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (first[mid] <= w) lo = mid;
    else hi = mid;
  }
  return lo;
}

__global__ __launch_bounds__(kFinishBlock) void k_route_finish(Rows r, Parts s, RouteOut o)
{
  __shared__ FinishLds m;
  constexpr uint32_t NT = kFinishBlock, kSlices = NT / kFinishExperts, kAhead = 16;
  const uint32_t b = blockIdx.x;
  const uint32_t tid = threadIdx.x;
  const uint32_t le = tid % kFinishExperts, slice = tid / kFinishExperts, e = b * kFinishExperts + le;
  const uint32_t w0 = (uint32_t)((uint64_t)s.W * slice / kSlices), w1 = (uint32_t)((uint64_t)s.W * (slice + 1) / kSlices);
  Cell ahead[kAhead];
  auto fetch = [&](uint32_t base) {
#pragma unroll
    for (uint32_t u = 0; u < kAhead; ++u) {
      ahead[u] = Cell{0u, 0.0f};
      if (e < r.E && base + u < w1) ahead[u] = s.cell[(uint64_t)(base + u) * r.E + e];
    }
  };
  fetch(w0);                                   // in flight while the devices' rows are counted
  const float weight = tid < r.K ? r.w[tid] : 0.0f;
  uint32_t n = tid < s.W ? s.rows[tid] : 0u;
  double z = tid < s.W && b == 0 ? s.z[tid] : 0.0;
  if (tid <= kMaxK) m.first[tid] = tid <= r.K ? r.first[tid] : ~0u;
  if (tid < kMaxK) m.rows[tid] = 0u;
  for (uint32_t i = tid; i < r.K * kFinishExperts; i += NT) (&m.count[0][0])[i] = 0u;
  __syncthreads();
  const uint32_t dev = device_in(m.first, r.K, tid < s.W ? tid : 0u);
  if (n) atomicAdd(&m.rows[dev], n);
  for (uint32_t w = tid + NT; w < s.W; w += NT)
    if ((n = s.rows[w])) atomicAdd(&m.rows[device_in(m.first, r.K, w)], n);
  __syncthreads();
  if (tid < r.K) {
    n = m.rows[tid];
    m.scale[tid] = n ? (double)weight / (double)n : 0.0;
    if (b == 0) o.share[tid] = n ? 1.0f / (float)n : 0.0f;
  }
  __syncthreads();
  double load = 0.0, prob = 0.0;
  if (e < r.E && w0 < w1) {
    uint32_t d = device_in(m.first, r.K, w0), end = m.first[d + 1], run = 0;
    double scale = m.scale[d];
    // kAhead results of one device at most are added in float
    auto flush = [&](float p, uint32_t c) {
      load = __builtin_fma(scale, (double)c, load);
      prob = __builtin_fma(scale, (double)p, prob);
      run += c;
    };
    for (uint32_t base = w0; base < w1; base += kAhead) {
      if (base != w0) fetch(base);
      float p = 0.0f;
      uint32_t c = 0;
      if (end >= w1 || base + kAhead <= end) {
#pragma unroll
        for (uint32_t u = 0; u < kAhead; ++u) {
          p += ahead[u].prob;
          c += ahead[u].count;
        }
      } else {
#pragma unroll
        for (uint32_t u = 0; u < kAhead; ++u) {
          if (base + u < w1 && base + u >= end) {
            flush(p, c);
            if (run) atomicAdd(&m.count[d][le], run);
            run = c = 0;
            p = 0.0f;
            while (base + u >= end) end = m.first[++d + 1];
            scale = m.scale[d];
          }
          p += ahead[u].prob;
          c += ahead[u].count;
        }
      }
      flush(p, c);
    }
    if (run) atomicAdd(&m.count[d][le], run);
  }
#pragma unroll
  for (int x = kFinishExperts; x < 64; x *= 2) {
    load += __shfl_xor(load, x, 64);
    prob += __shfl_xor(prob, x, 64);
  }
  if (lane_id() < kFinishExperts) {
    m.load[tid >> 6][le] = load;
    m.prob[tid >> 6][le] = prob;
  }
  if (b == 0) {
    z *= m.scale[dev];
    for (uint32_t w = tid + NT; w < s.W; w += NT) z = __builtin_fma(m.scale[device_in(m.first, r.K, w)], s.z[w], z);
    z = wave_sum_f64(z);
    if (lane_id() == 0) m.z[tid >> 6] = z;
  }
  __syncthreads();
  for (uint32_t i = tid; i < r.K * kFinishExperts; i += NT) {
    const uint32_t x = b * kFinishExperts + i % kFinishExperts;
    if (x < r.E) o.counts[(uint64_t)(i / kFinishExperts) * r.E + x] = (int32_t)m.count[i / kFinishExperts][i % kFinishExperts];
  }
  double balance = 0.0;
  if (tid < 64) {
    // lane tid takes expert tid % 16 of every fourth wave's sums
    load = prob = 0.0;
    for (uint32_t q = tid / kFinishExperts; q < NT / 64; q += 64 / kFinishExperts) {
      load += m.load[q][le];
      prob += m.prob[q][le];
    }
#pragma unroll
    for (int x = kFinishExperts; x < 64; x *= 2) {
      load += __shfl_xor(load, x, 64);
      prob += __shfl_xor(prob, x, 64);
    }
    load /= (double)r.k;
    if (tid < kFinishExperts && e < r.E) {
      o.load[e] = (float)load;
      balance = load * prob * (double)r.E;
    }
    balance = wave_sum_f64(balance);
    if (b == 0) {
      z = wave_sum_f64(tid < NT / 64 ? m.z[tid] : 0.0);
      if (tid == 0) o.loss[1] = (float)z;
    }
  }
  if (threadIdx.x == 0) put(&s.balance[blockIdx.x], balance);
  if (!block_is_last(s.ticket, 1u, gridDim.x) || threadIdx.x >= 64) return;
  double sum = 0.0;
  for (uint32_t i = threadIdx.x; i < gridDim.x; i += 64) sum += get(&s.balance[i]);
  sum = wave_sum_f64(sum);
  if (threadIdx.x == 0) o.loss[0] = (float)sum;
}

// ---- forward ------------------------------------------------------------------------------------
template <int G, int V>
struct RouteLds {
  static constexpr int kGroups = kBlock / G;
  static constexpr int kChoices = G * V < (int)kMaxChoices ? G * V : (int)kMaxChoices;
  uint32_t count[G * V];
  alignas(16) float row[kGroups][G * V];     // the groups' rows, at the end the groups' probability sums
  uint32_t idx[kGroups][kChoices];
  float ex[kGroups][kChoices];
  double z[kWaves];
  uint32_t rows[kWaves];
  static constexpr int kFewGroups = G >= kFewLanes ? kGroups : 1;      // of the choice by a threshold
  alignas(16) float top[kFewGroups][G];
  alignas(16) uint64_t few[kFewGroups][G];
  uint32_t at[kFewGroups][G];
  uint32_t nfew[kFewGroups];
};

// The k choices of every group's row of the wave, one after the other: k rounds
// of the largest value left, then the lowest index that has it. x is used up.
template <int G, int V>
__device__ inline void choose_in_turn(float (&x)[V], float mx, const Exp& ex, uint32_t k, uint32_t l4, uint32_t group, RouteLds<G, V>& m)
{
  for (uint32_t c = 0; c < k; ++c) {
    float top = mx;
    if (c) {
      top = x[0];
#pragma unroll
      for (int i = 1; i < V; ++i) top = __builtin_fmaxf(top, x[i]);
      top = group_max<G>(top);
    }
    uint32_t mine = V;                      // the lane's first element that has it
#pragma unroll
    for (int i = V - 1; i >= 0; --i) mine = x[i] == top ? (uint32_t)i : mine;
    const uint32_t e = mine < (uint32_t)V ? expert_of<G>(mine, l4) : ~0u, at = group_min<G>(e);
    const bool some = top > -__builtin_inff() && at != ~0u;
    if (c + 1 < k) {
      if (e != at) mine = V;
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] = (uint32_t)i == mine ? -__builtin_inff() : x[i];
    }
    if (l4 == 0) {
      m.idx[group][c] = some ? at : ~0u;
      m.ex[group][c] = some ? ex(top) : 0.0f;
      if (some) atomicAdd(&m.count[at], 1u);
    }
  }
}

// The same by a threshold: at least k lanes hold a value at or above the k-th
// largest of the lanes' maxima `top`, so the choices are among the values at or
// above it. Their experts are listed in LDS, one per lane, and ranked by
// counting the larger ones (of equal values, the lower index is the larger).
// False, with nothing chosen, where a row of the wave has more such values than
// lanes; rare as long as k is at most half the lanes (random logits: 10.6 values
// on average for 8 of 16 lanes, standard deviation 2). Comparisons are taken
// from the sign of a difference and gathered bit by bit: a compare's result
// would have to be waited for.
// 2^25 logits, 3, 4 and 8 choices so, and in turn: 38, 38, 44 and 41, 46, 68 us for
// 256 experts, 42, 42, 42 and 43, 49, 72 for 512, 52, 52, 52 and 46, 52, 77 for
// 1024; 8 choices of 128 experts 55 and 88; two of 256 37 and 37, of 1024 52 and 40.
template <int G, int V>
__device__ inline bool choose_few(const float (&x)[V], float top, const Exp& ex, uint32_t k, uint32_t l, uint32_t group, RouteLds<G, V>& m)
{
  auto append = [](uint32_t bits, float x) { return __builtin_amdgcn_alignbit(bits, __float_as_uint(x), 31); };
  top = __builtin_fmaxf(top, -__FLT_MAX__);                // an expert at -infinity is never chosen
  m.top[group][l] = top;
#pragma unroll
  for (int j = 0; j < V / 4; ++j)
    *reinterpret_cast<f4*>(&m.row[group][expert_at<G>(4 * j) + 4 * l]) = f4{x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]};
  m.few[group][l] = 0ull;
  if (l == 0) m.nfew[group] = 0u;
  wave_sync();
  uint32_t above = 0;
#pragma unroll
  for (int h = 0; h < G; h += 32) {
    uint32_t bits = 0;
#pragma unroll
    for (int j = h; j < h + 32 && j < G; j += 4) {
      const f4 t = *reinterpret_cast<const f4*>(&m.top[group][j]);
#pragma unroll
      for (int q = 0; q < 4; ++q) bits = append(bits, top - t[q]);
    }
    above += __builtin_popcount(bits);
  }
  float least = group_least<G>(above < k ? top : __builtin_inff());
  least = least == 0.0f ? -0.0f : least;                   // so that x - least is no -0 for an x of -0
  uint32_t below = 0;
#pragma unroll
  for (int i = V - 1; i >= 0; --i) below = append(below, x[i] - least);      // bit i: element i
  uint32_t mine = ~below & ((1u << V) - 1);
  const uint32_t n = __builtin_popcount(mine);
  uint32_t at = n ? atomicAdd(&m.nfew[group], n) : 0u;
  wave_sync();
  const uint32_t all = m.nfew[group];
  if (__ballot(all > (uint32_t)G)) return false;
  while (mine) {
    m.at[group][at++] = expert_of<G>((uint32_t)__builtin_ctz(mine), 4 * l);
    mine &= mine - 1;
  }
  if (l < k) {
    m.idx[group][l] = ~0u;
    m.ex[group][l] = 0.0f;
  }
  wave_sync();
  const bool some = l < all;
  const uint32_t e = some ? m.at[group][l] : 0u;
  const float value = m.row[group][e];
  const uint32_t u = __float_as_uint(value + 0.0f);        // -0 counts as 0; order of floats as integers
  const uint64_t key = some ? (uint64_t)(u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u)) << 32 | ~e : 0ull;
  if (some) m.few[group][l] = key;
  wave_sync();
  uint32_t rank = 0;
#pragma unroll 4
  for (int j = 0; j < G; ++j) rank += m.few[group][j] > key ? 1u : 0u;
  if (some && rank < k) {
    m.idx[group][rank] = e;
    m.ex[group][rank] = ex(value);
    atomicAdd(&m.count[e], 1u);
  }
  return true;
}

template <class X, int G, int V, bool kOne>
__global__ __launch_bounds__(kBlock, kOne ? 1 : V >= 16 ? 4 : 5) void k_route(Rows r, const X* logits, const uint8_t* valid, RouteOut o, Parts s)
{
  constexpr int kGroups = kBlock / G;
  __shared__ RouteLds<G, V> m;
  const uint32_t tid = threadIdx.x, l = tid % G, l4 = 4 * l, group = tid / G;
  const Share mine = share_of(r, blockIdx.x);
  const uint64_t row0 = mine.row0, row1 = mine.row1;
  for (uint32_t e = tid; e < G * V; e += kBlock) m.count[e] = 0u;
  if (blockIdx.x == 0 && tid == 0) *s.ticket = 0u;
  __syncthreads();
  float acc[V];
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] = 0.0f;
  double z = 0.0;
  uint32_t rows = 0;
  for (uint64_t base = row0 + wave_id() * (64 / G); base < row1; base += kGroups) {     // the wave's rows
    const uint64_t row = base + lane_id() / G;
    const bool on = row < row1 && (!valid || gptr(valid)[row]);
    float x[V];
    load_row<X, G, V>(x, logits + row * r.ld, l4, r.E, on);
    float top = x[0];
#pragma unroll
    for (int i = 1; i < V; ++i) top = __builtin_fmaxf(top, x[i]);
    const float mx = group_max<G>(top);
    // a row without a value above -inf sums to zero: it routes nowhere and is not counted
    const float mid = mx == -__builtin_inff() ? 0.0f : mx;
    float p[V], sum = 0.0f;
    const Exp ex = {mid, mid * kLog2e, !(__builtin_fabsf(mid) < kFar)};
    if (__ballot(ex.far)) {
#pragma unroll
      for (int i = 0; i < V; ++i) p[i] = ex(x[i]);
    } else {
      const Exp near = {mid, ex.c, false};
#pragma unroll
      for (int i = 0; i < V; ++i) p[i] = near(x[i]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) sum += p[i];
    sum = group_sum<G>(sum);
    const bool counted = !(sum == 0.0f);
    // sum is 1 to E, times the row's factor; reciprocal, exponential and logarithm are
    // the hardware's, within a unit: gates and lse are off by up to 1.4 times as much as
    // with exact ones (7.5e-8 against 5.3e-8 for 256 experts)
    const float inv = counted ? __builtin_amdgcn_rcpf(sum) : 0.0f;
    const float lse = counted ? mid + __builtin_amdgcn_logf(sum) * kLn2 : 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = __builtin_fmaf(p[i], inv, acc[i]);
    z += (double)lse * (double)lse;
    rows += (uint32_t)__builtin_popcountll(__ballot(counted)) / G;          // of the wave
    bool done = false;
    if constexpr (G >= kFewLanes)
      if (r.k >= few_from(G) && 2 * r.k <= G) done = choose_few<G, V>(x, top, ex, r.k, l, group, m);
    if (!done)
      choose_in_turn<G, V>(x, mx, ex, r.k, l4, group, m);
    wave_sync();
    float chosen = 0.0f;
    if (r.renormalise) {
      for (uint32_t c = l; c < r.k; c += G) chosen += m.ex[group][c];
      chosen = group_sum<G>(chosen);
    }
    float to_gate = inv;
    if (r.renormalise && sum < __builtin_inff()) to_gate = chosen > 0.0f ? __builtin_amdgcn_rcpf(chosen) : 0.0f;   // else NaN, as inv is
    if (row < row1) {
      for (uint32_t c = l; c < r.k; c += G) {
        o.idx[row * r.k + c] = (int32_t)m.idx[group][c];
        o.gate[row * r.k + c] = m.ex[group][c] * to_gate;
      }
      if (l == 0) o.lse[row] = lse;
    }
    wave_sync();
  }
  // the experts' sums of every 16 lanes (of a group, where it has more), then of the workgroup
  constexpr int kLanes = G < 16 ? 16 : G, kSums = kBlock / kLanes;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    acc[i] = sum_over_row<G>(acc[i]);
    if (tid % kLanes < G) m.row[tid / kLanes][expert_at<G>(i) + l4] = acc[i];
  }
  z = wave_sum_f64(l == 0 ? z : 0.0);
  if (lane_id() == 0) {
    m.z[wave_id()] = z;
    m.rows[wave_id()] = rows;
  }
  __syncthreads();
  double zs = 0.0, balance = 0.0;
  uint32_t n = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    zs += m.z[w];
    n += m.rows[w];
  }
  if (!kOne && tid == 0) {
    s.z[blockIdx.x] = zs;
    s.rows[blockIdx.x] = n;
  }
  const double scale = kOne && n ? (double)r.w[mine.d] / (double)n : 0.0;
  for (uint32_t e = tid; e < r.E; e += kBlock) {
    float sum = 0.0f;
#pragma unroll 4
    for (int g = 0; g < kSums; ++g) sum += m.row[g][e];
    if constexpr (kOne) {
      const double load = scale * (double)m.count[e] / (double)r.k;
      balance += load * scale * (double)sum * (double)r.E;
      o.load[e] = (float)load;
      for (uint32_t d = 0; d < r.K; ++d) o.counts[(uint64_t)d * r.E + e] = d == mine.d ? (int32_t)m.count[e] : 0;
    } else {
      s.cell[(uint64_t)blockIdx.x * r.E + e] = Cell{m.count[e], sum};
    }
  }
  if constexpr (kOne) {        // the only workgroup: it makes the sums over all rows itself
    for (uint32_t d = tid; d < r.K; d += kBlock) o.share[d] = d == mine.d && n ? 1.0f / (float)n : 0.0f;
    __shared__ double s_sum[kWaves];
    balance = block_sum_f64(balance, s_sum);
    if (tid == 0) {
      o.loss[0] = (float)balance;
      o.loss[1] = (float)(scale * zs);
    }
  }
}

// ---- backward -----------------------------------------------------------------------------------
template <class X, int G, int V>
__global__ __launch_bounds__(kBlock) void k_route_back(Rows r, const X* logits, RouteOut o, const float* dgate,
                                                       const float* dloss, X* dlogits, uint64_t ld_out)
{
  constexpr int kGroups = kBlock / G;
  __shared__ alignas(16) float s_part[kGroups][G * V];      // the gates' part of the group's row, zero elsewhere
  static_assert(__alignof__(s_part) >= sizeof(f4), "read by 16 bytes");
  const uint32_t tid = threadIdx.x, l = tid % G, l4 = 4 * l, group = tid / G;
  const Share mine = share_of(r, blockIdx.x);
  const uint64_t row0 = mine.row0, row1 = mine.row1;
  const float scale = r.w[mine.d] * o.share[mine.d];
  const float a = dloss ? dloss[0] * scale * (float)r.E : 0.0f, b2 = dloss ? 2.0f * dloss[1] * scale : 0.0f;
  float load[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t e = expert_at<G>(i) + l4;
    load[i] = e < r.E ? o.load[e] : 0.0f;
    s_part[group][e] = 0.0f;
  }
  wave_sync();
  for (uint64_t base = row0 + wave_id() * (64 / G); base < row1; base += kGroups) {     // the wave's rows
    const uint64_t row = base + lane_id() / G;
    const bool in = row < row1;
    const float lse = in ? o.lse[row] : 0.0f;
    // a choice's expert, or one past the experts for a missing choice: whatever idx
    // holds, nothing outside s_part is written
    auto chosen = [&](uint32_t c) {
      const uint32_t e = (uint32_t)o.idx[row * r.k + c];
      return e < r.E ? e : r.E;
    };
    const bool on = in && (chosen(0) < r.E || lse != lse);         // routed, or NaN
    float x[V];
    load_row<X, G, V>(x, logits + row * r.ld, l4, r.E, on);
    float sum = 0.0f, mean = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      x[i] = exp_of(x[i] - lse);
      sum += x[i];
      mean += x[i] * load[i];
    }
    sum = group_sum<G>(sum);
    mean = group_sum<G>(mean);
    float part = 0.0f;
    if (dgate) {
      for (uint32_t c = l; c < r.k; c += G)    // what is given for a choice that is missing does not count
        if (on && chosen(c) < r.E) part += o.gate[row * r.k + c] * dgate[row * r.k + c];
      part = group_sum<G>(part);
      for (uint32_t c = l; c < r.k; c += G) {
        const uint32_t e = on ? chosen(c) : r.E;
        if (e < r.E) s_part[group][e] = o.gate[row * r.k + c] * (dgate[row * r.k + c] - (r.renormalise ? part : 0.0f));
      }
      if (r.renormalise) part = 0.0f;
      wave_sync();
    }
    const float inv = on ? 1.0f / sum : 0.0f;   // lse is rounded: its error cancels
    const float all = b2 * lse - part - a * (mean * inv);
#pragma unroll
    for (int j = 0; j < V / 4; ++j) {
      const uint32_t e = expert_at<G>(4 * j) + l4;
      f4 dx;
#pragma unroll
      for (int q = 0; q < 4; ++q) dx[q] = on ? x[4 * j + q] * inv * (a * load[4 * j + q] + all) : 0.0f;
      if (dgate) {
        const f4 g = *reinterpret_cast<const f4*>(&s_part[group][e]);
#pragma unroll
        for (int q = 0; q < 4; ++q) dx[q] += g[q];
      }
      if (in && e < r.E) store_f4(dlogits + row * ld_out + e, dx, r.E - e);
    }
    if (dgate) {
      wave_sync();
      for (uint32_t c = l; c < r.k; c += G) {
        const uint32_t e = on ? chosen(c) : r.E;
        if (e < r.E) s_part[group][e] = 0.0f;
      }
      wave_sync();
    }
  }
}

// ---- host side ------------------------------------------------------------------------------------
// Lanes per row and elements per lane. The more elements a lane has, the fewer
// exchanges and rounds of choosing per row; the more lanes, the better their
// loads lie together, and from kFewLanes on choices can be made by a threshold.
// Forward with 2 choices, 2^25 logits: 8 experts by 1, 2 and 4 lanes 54, 66 and
// 112 us; 16 by 1, 2 and 4: 66, 49, 62; 32 by 2, 4 and 8: 58, 46, 62; 64 by 4, 8
// and 16: 41, 44, 63; 128 by 8 and 16: 37, 44, with 4, 5 and 8 choices 45, 51, 68
// and 49, 50, 55; 256 by 16 and 32: 37, 46. Backward (8 choices) 8 experts by 1,
// 2 and 4 lanes 486, 292 and 307 us; 16 by 1, 2 and 4: 280, 168, 173; 32 by 2, 4 and 8: 118, 88,
// 111; 64 by 4, 8 and 16: 68, 69, 111; 128 by 8 and 16: 55, 68; 256 by 16 and 32:
// 53, 68.
template <int G, int V, class F>
void shape(F f)
{
  f(std::integral_constant<int, G>(), std::integral_constant<int, V>());
}

template <class F>
void with_shape(uint32_t E, uint32_t k, F f)
{
  if (E <= 8) shape<1, 8>(f);
  else if (E <= 16) shape<2, 8>(f);
  else if (E <= 32) shape<4, 8>(f);
  else if (E <= 64) shape<4, 16>(f);
  else if (E <= 128 && k <= 4) shape<8, 16>(f);
  else if (E <= 128) shape<16, 8>(f);
  else if (E <= 256) shape<16, 16>(f);
  else if (E <= 512) shape<32, 16>(f);
  else shape<64, 16>(f);
}

template <class F>
void with_back_shape(uint32_t E, F f)
{
  if (E <= 8) shape<2, 4>(f);
  else if (E <= 16) shape<2, 8>(f);
  else if (E <= 32) shape<4, 8>(f);
  else if (E <= 64) shape<4, 16>(f);
  else if (E <= 128) shape<8, 16>(f);
  else if (E <= 256) shape<16, 16>(f);
  else if (E <= 512) shape<32, 16>(f);
  else shape<64, 16>(f);
}

// Rows that a workgroup takes at once.
uint32_t round_of(uint32_t E, uint32_t k)
{
  uint32_t n = 0;
  with_shape(E, k, [&](auto g, auto) { n = kBlock / g; });
  return n;
}

uint32_t back_round_of(uint32_t E)
{
  uint32_t n = 0;
  with_back_shape(E, [&](auto g, auto) { n = kBlock / g; });
  return n;
}

uint32_t blocks_for(const scadles_router* q, uint64_t per)
{
  uint64_t w = 0;
  for (uint32_t d = 0; d < q->devices; ++d) w += div_up(q->tok_off[d + 1] - q->tok_off[d], per);
  return (uint32_t)w;
}

// Rows of one workgroup, so that at most kRouteBlocks workgroups share them: that
// many fit the GPU at once, and a few more make the call take nearly twice as
// long. At least a round, then as many rows more as a wave takes at once.
uint64_t rows_for(const scadles_router* q, uint64_t round, uint32_t blocks)
{
  const uint64_t unit = round / kWaves, most = round * kMaxRounds;
  uint64_t n = div_up(div_up(q->tokens, blocks), round) * round;
  if (n >= 4 * round) n = div_up(div_up(q->tokens, blocks), unit) * unit;
  if (n < round) n = round;
  while (n < most && blocks_for(q, n) > blocks) n += n < 4 * round ? round : unit;
  return n < most ? n : most;
}

scadles_status check_router(const scadles_router* q)
{
  if (!q) return fail(SCADLES_EINVAL, "router is NULL");
  if (q->tokens > 0x7FFFFFFFull) return fail(SCADLES_EINVAL, "more than 2^31 - 1 tokens");
  if (!q->experts || q->experts > kMaxExperts) return fail(SCADLES_EINVAL, "experts = %u is outside [1, %u]", q->experts, kMaxExperts);
  if (!q->k || q->k > q->experts || q->k > kMaxChoices)
    return fail(SCADLES_EINVAL, "k = %u is outside [1, min(experts, %u)]", q->k, kMaxChoices);
  if (!q->devices || q->devices > kMaxK) return fail(SCADLES_EINVAL, "devices = %u is outside [1, %d]", q->devices, kMaxK);
  if (q->logits_type != SCADLES_F32 && q->logits_type != SCADLES_BF16)
    return fail(SCADLES_EINVAL, "unknown logits_type %d", q->logits_type);
  if (q->ld < q->experts) return fail(SCADLES_EINVAL, "ld is smaller than experts");
  if (!q->tok_off) return fail(SCADLES_EINVAL, "tok_off is NULL");
  if (q->tok_off[0] != 0 || q->tok_off[q->devices] != q->tokens) return fail(SCADLES_EINVAL, "tok_off must run from 0 to tokens");
  for (uint32_t d = 0; d < q->devices; ++d)
    if (q->tok_off[d + 1] < q->tok_off[d]) return fail(SCADLES_EINVAL, "tok_off must not decrease");
  if (!q->weights) return fail(SCADLES_EINVAL, "weights is NULL");
  for (uint32_t d = 0; d < q->devices; ++d)
    if (!std::isfinite(q->weights[d]) || q->weights[d] < 0.0f) return fail(SCADLES_EINVAL, "weight %u is negative or not finite", d);
  return SCADLES_OK;
}

// What the kernels need to know of the rows; returns the workgroups.
uint32_t make_rows(const scadles_router* q, uint32_t round, uint32_t blocks, Rows& r)
{
  std::memset(&r, 0, sizeof(r));
  r.per = (uint32_t)rows_for(q, round, blocks);
  r.E = q->experts;
  r.k = q->k;
  r.K = q->devices;
  r.ld = q->ld;
  r.renormalise = q->renormalise ? 1u : 0u;
  uint64_t w = 0;
  for (uint32_t d = 0; d < r.K; ++d) {
    r.off[d] = q->tok_off[d];
    r.first[d] = (uint32_t)w;
    r.w[d] = q->weights[d];
    w += div_up(q->tok_off[d + 1] - q->tok_off[d], r.per);
  }
  r.off[r.K] = q->tokens;
  r.first[r.K] = (uint32_t)w;
  return (uint32_t)w;
}

uint64_t take(uint64_t& at, uint64_t bytes)
{
  const uint64_t here = at;
  at = div_up(at + bytes, 256) * 256;
  return here;
}

// The workspace's pieces for W workgroups; returns its size.
uint64_t lay_out(uint32_t W, uint32_t E, char* ws, Parts& s)
{
  uint64_t at = 0;
  s.ticket = reinterpret_cast<uint32_t*>(ws + take(at, 256));
  s.balance = reinterpret_cast<double*>(ws + take(at, kMaxExperts / kFinishExperts * 8));
  s.z = reinterpret_cast<double*>(ws + take(at, (uint64_t)W * 8));
  s.rows = reinterpret_cast<uint32_t*>(ws + take(at, (uint64_t)W * 4));
  s.cell = reinterpret_cast<Cell*>(ws + take(at, (uint64_t)W * E * sizeof(Cell)));
  s.W = W;
  return at;
}

// A call without rows: nothing is counted.
__global__ void k_route_empty(Rows r, RouteOut o)
{
  for (uint32_t i = threadIdx.x; i < r.K * r.E; i += blockDim.x) o.counts[i] = 0;
  for (uint32_t i = threadIdx.x; i < r.E; i += blockDim.x) o.load[i] = 0.0f;
  for (uint32_t i = threadIdx.x; i < r.K; i += blockDim.x) o.share[i] = 0.0f;
  if (threadIdx.x < 2) o.loss[threadIdx.x] = 0.0f;
}

scadles_status check_out(const scadles_router* q, const scadles_router_out* o)
{
  if (!o) return fail(SCADLES_EINVAL, "out is NULL");
  if (q->tokens && (!o->idx || !o->gate || !o->lse)) return fail(SCADLES_EINVAL, "idx, gate and lse must not be NULL");
  if (!o->counts || !o->load || !o->share || !o->loss) return fail(SCADLES_EINVAL, "counts, load, share and loss must not be NULL");
  for (const void* p : {(const void*)o->idx, (const void*)o->gate, (const void*)o->lse, (const void*)o->counts, (const void*)o->load,
                        (const void*)o->share, (const void*)o->loss})
    if (!is_aligned(p, 4)) return fail(SCADLES_EINVAL, "an output is not 4-byte aligned");
  return SCADLES_OK;
}

// Elements from the first to the last of T rows.
uint64_t span_bytes(const scadles_router* q, uint64_t ld)
{
  return q->tokens ? ((q->tokens - 1) * ld + q->experts) * (q->logits_type == SCADLES_BF16 ? 2 : 4) : 0;
}

template <class X>
hipError_t launch_route(const Rows& r, const void* logits, const uint8_t* valid, const RouteOut& o, const Parts& s, hipStream_t st)
{
  with_shape(r.E, r.k, [&](auto g, auto v) {
    if (s.W == 1) k_route<X, g, v, true><<<1, kBlock, 0, st>>>(r, (const X*)logits, valid, o, s);
    else k_route<X, g, v, false><<<s.W, kBlock, 0, st>>>(r, (const X*)logits, valid, o, s);
  });
  if (s.W > 1) k_route_finish<<<(uint32_t)div_up(r.E, kFinishExperts), kFinishBlock, 0, st>>>(r, s, o);
  return hipGetLastError();
}

template <class X>
hipError_t launch_back(const Rows& r, uint32_t W, const void* logits, const RouteOut& o, const float* dgate, const float* dloss,
                       void* dlogits, uint64_t ld_out, hipStream_t st)
{
  with_back_shape(r.E, [&](auto g, auto v) {
    k_route_back<X, g, v><<<W, kBlock, 0, st>>>(r, (const X*)logits, o, dgate, dloss, (X*)dlogits, ld_out);
  });
  return hipGetLastError();
}

RouteOut outputs(const scadles_router_out* o)
{
  return {o->idx, o->gate, o->lse, o->counts, o->load, o->share, o->loss};
}

}  // namespace

extern "C" {

size_t scadles_router_workspace_bytes(uint64_t tokens, uint32_t experts, uint32_t devices)
{
  if (tokens > 0x7FFFFFFFull || !experts || experts > kMaxExperts || !devices || devices > kMaxK) return 0;
  // the most workgroups of any call of so many rows or fewer; every device's last one may be partly filled
  uint64_t round = round_of(experts, 1);       // the fewest rows of any k
  if (round_of(experts, kMaxChoices) < round) round = round_of(experts, kMaxChoices);
  const uint64_t few = tokens / round + devices;
  const uint64_t many = tokens / (round * kMaxRounds) + devices;
  const uint64_t W = few < kRouteBlocks ? few : many > kRouteBlocks ? many : kRouteBlocks;
  Parts s;
  return (size_t)lay_out((uint32_t)W, experts, nullptr, s);
}

scadles_status scadles_router_forward(const scadles_router* router, const void* logits, const uint8_t* valid,
                                      const scadles_router_out* out, void* ws, size_t ws_bytes, void* stream)
{
  if (scadles_status st = check_router(router)) return st;
  double total = 0.0;
  for (uint32_t d = 0; d < router->devices; ++d) total += (double)router->weights[d];
  if (std::fabs(total - 1.0) > (double)router->devices * std::ldexp(1.0, -23))
    return fail(SCADLES_EINVAL, "weights sum to %.17g, not 1 (Eqn 4a)", total);
  if (scadles_status st = check_out(router, out)) return st;
  const uint64_t esize = router->logits_type == SCADLES_BF16 ? 2 : 4, T = router->tokens;
  if (T && !logits) return fail(SCADLES_EINVAL, "logits is NULL");
  if (!is_aligned(logits, esize)) return fail(SCADLES_EINVAL, "logits is not aligned to its elements");
  Rows r;
  Parts s;
  const uint32_t W = make_rows(router, round_of(router->experts, router->k), kRouteBlocks, r);
  const uint64_t need = lay_out(W, router->experts, static_cast<char*>(ws), s);
  if (!ws || !is_aligned(ws, 256)) return fail(SCADLES_EWORKSPACE, "workspace must be 256-byte aligned and not NULL");
  if (ws_bytes < need) return fail(SCADLES_EWORKSPACE, "workspace has %zu bytes, needs %zu", ws_bytes, (size_t)need);
  const void* outs[7] = {out->idx, out->gate, out->lse, out->counts, out->load, out->share, out->loss};
  const uint64_t sizes[7] = {T * router->k * 4, T * router->k * 4, T * 4, (uint64_t)router->devices * router->experts * 4,
                             (uint64_t)router->experts * 4, (uint64_t)router->devices * 4, 8};
  for (int x = 0; x < 7; ++x) {
    if (bytes_overlap(outs[x], sizes[x], logits, span_bytes(router, router->ld)) || bytes_overlap(outs[x], sizes[x], valid, T) ||
        bytes_overlap(outs[x], sizes[x], ws, need))
      return fail(SCADLES_EINVAL, "an output overlaps an input or the workspace");
    for (int y = 0; y < x; ++y)
      if (bytes_overlap(outs[x], sizes[x], outs[y], sizes[y])) return fail(SCADLES_EINVAL, "two outputs overlap");
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  const RouteOut o = outputs(out);
  if (W == 0) {
    k_route_empty<<<1, kBlock, 0, st>>>(r, o);
    return launch_status(hipGetLastError(), "router forward");
  }
  return launch_status(esize == 2 ? launch_route<uint16_t>(r, logits, valid, o, s, st) : launch_route<float>(r, logits, valid, o, s, st),
                       "router forward");
}

scadles_status scadles_router_backward(const scadles_router* router, const void* logits, const scadles_router_out* out,
                                       const float* dgate, const float* dloss, void* dlogits, uint64_t ld_out, void* stream)
{
  if (scadles_status st = check_router(router)) return st;
  if (scadles_status st = check_out(router, out)) return st;
  const uint64_t esize = router->logits_type == SCADLES_BF16 ? 2 : 4, T = router->tokens;
  if (T && (!logits || !dlogits)) return fail(SCADLES_EINVAL, "logits and dlogits must not be NULL");
  if (!is_aligned(logits, esize) || !is_aligned(dlogits, esize))
    return fail(SCADLES_EINVAL, "logits or dlogits is not aligned to its elements");
  if (!is_aligned(dgate, 4) || !is_aligned(dloss, 4)) return fail(SCADLES_EINVAL, "dgate or dloss is not 4-byte aligned");
  if (ld_out < router->experts) return fail(SCADLES_EINVAL, "ld_out is smaller than experts");
  const uint64_t bytes = span_bytes(router, ld_out);
  const void* ins[8] = {logits, out->idx, out->gate, out->lse, out->load, out->share, dgate, dloss};
  const uint64_t sizes[8] = {span_bytes(router, router->ld), T * router->k * 4, T * router->k * 4, T * 4,
                             (uint64_t)router->experts * 4, (uint64_t)router->devices * 4, T * router->k * 4, 8};
  for (int x = 0; x < 8; ++x)
    if (bytes_overlap(dlogits, bytes, ins[x], sizes[x])) return fail(SCADLES_EINVAL, "dlogits overlaps an input");
  Rows r;
  const uint32_t W = make_rows(router, back_round_of(router->experts), kBackBlocks, r);
  if (W == 0) return SCADLES_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const RouteOut o = outputs(out);
  return launch_status(esize == 2 ? launch_back<uint16_t>(r, W, logits, o, dgate, dloss, dlogits, ld_out, st)
                                  : launch_back<float>(r, W, logits, o, dgate, dloss, dlogits, ld_out, st),
                       "router backward");
}

}  // extern "C"
