// cross_entropy.hip -- the cross entropy of a linear layer over a vocabulary, and its
// gradients, without the logits being kept.
//
//   z = weight x[t],  lse = log sum exp z,  nll = lse - z_target
//   G = softmax(z) - onehot,  d_x = c_t G weight,  d_weight[d] = c_d G^T x over device d
//
// Forward: k_logits multiplies tiles of 256 vocabulary entries by 256 tokens and leaves,
// in place of a tile's logits, each token's maximum and sum of exponentials over it;
// k_loss_rows joins the tiles of a token. Backward, for a piece of the vocabulary at a
// time: k_logits again, which now has lse and stores G of the piece both ways round,
// tokens by vocabulary for d_x and vocabulary by tokens for d_weight; then k_gradients,
// tiles of both products in one launch. x and weight are needed with the contraction's
// index adjacent, so that k_turn writes both transposed once per call.
//
// Types. bfloat16 x and weight are multiplied where they lie. With bfloat16 gradients G is rounded to
// bfloat16 too, 2^-8 of each value, so that each gradient is one product; with float gradients they
// are two and three, and a call takes 8.05 ms in place of 4.19 (below). The rounding of a target's
// probability minus one goes into all of a row's d_x. Errors of d_x and d_weight against 64 bits, 2048
// x 8192 x 512: 0.00168 where targets have a probability of 0, 0.0021 at 0.17, 0.0023 at 0.77, of which the
// outputs' own rounding is 0.00166. Float gradients are for those who want more.
// The logits of floats: x and weight are sums of two half floats (22 bits), scaled by powers of two
// by row, where the largest of a row comes to 2^13 .. 2^14. Three products of such parts, the fourth
// being below 2^-22 of the first, have the precision of sums in float, and what a row lacks is
// small beside its own largest.
// The gradients' products contract over rows, so that a scale would have to be common to rows that
// have nothing to do with each other: a masked entry's and the others', one device's tokens and
// another's. Their operands, and G, are three bfloat16 parts instead: all 24 bits of a float, at
// any magnitude (a probability of 1e-30 has as many as one of 1e-1), and six products, twice the three
// of half floats. The products are as many as the result's type asks for (x_pairs, w_pairs).
//
// Tokens are counted with every device's first one at a multiple of 64 (Tokens::place), so
// that a step of the product over tokens belongs to one device. A token that is
// not counted is a row of zeros wherever it is stored.
//
// A product's tiles are too few for the GPU where dim or a batch is small; its sum is then
// split into units of about the same length, whose sums k_join_x and k_join_weight add.
//
// Bound by the matrix cores. Traced, kernel by kernel: 8192 tokens, 65536 entries, 1024 bfloat16: forward 1038 us
// (1.06 PFLOP/s), then for each of 8 pieces 169 us for G (0.81: its exponentials and two copies) and 245 for
// both gradients (1.12), and 58 us to transpose x and weight, 4.42 ms with the losses; untraced a call is
// 4.19. With float gradients 315 for G in three parts and 575 for five products (1.20). 2039 x 20011 x 500
// floats: 166 us (246 TFLOP/s counted as products of floats), 246 and 670 (122).
#include <cmath>
#include <cstring>

#include "product.h"
#include "vec4.h"

using namespace scadles;

namespace {

// Of one plane of G and its transpose, about: three planes have pieces of the same length, since shorter ones
// cost the products more than G's memory does (8192 x 65536 x 1024 bfloat16 with float gradients: 8.05 ms; 256
// MiB for the three: 10.5. 2039 x 20011 x 500 floats: 1094 us, 1162; 14285 x 24630 x 64 floats: 4.68 ms, 4.52).
constexpr uint64_t kPieceBytes = 256ull << 20;
constexpr uint32_t kLeastPiece = 2048;            // vocabulary entries of a piece, at least
constexpr uint32_t kNone = ~0u;
constexpr uint32_t kMost = 1u << 22;              // tokens and vocabulary entries: 32-bit offsets within a tile
constexpr uint32_t kLeastSteps = 16;              // of a unit of a split sum, as long as its start and its store
constexpr int kParts = 3;                         // bfloat16 parts of a float
constexpr int kRowsBlock = 1024;
constexpr uint32_t kRowSlices = kRowsBlock / 64;

// The tokens and where they are counted.
struct Tokens {
  uint64_t off[kMaxK + 1];     // device d's tokens
  uint32_t place[kMaxK + 1];   // and their places, from a multiple of 64 on
  float weight[kMaxK];
  const void* target;
  uint32_t K, places, vocab, wide;
};

struct Where {
  int64_t t;                   // token, -1 where there is none
  uint32_t d;
};

__device__ inline Where token_at(const Tokens& a, uint32_t p)
{
  uint32_t d = 0;
  while (d + 1 < a.K && a.place[d + 1] <= p) ++d;
  const uint64_t t = a.off[d] + (p - a.place[d]);
  return {p < a.places && t < a.off[d + 1] ? (int64_t)t : -1, d};
}

// A token's target, kNone if it is not counted.
__device__ inline uint32_t target_of(const Tokens& a, int64_t t)
{
  const uint64_t v = a.wide ? gptr((const uint64_t*)a.target)[t] : (uint64_t)(int64_t)gptr((const int32_t*)a.target)[t];
  return v < a.vocab ? (uint32_t)v : kNone;
}

// An operand: rows of planes of 16-bit floats.
struct Matrix {
  const uint16_t* p;
  uint64_t plane;              // elements between planes
  uint64_t ld;
};

// Tiles in the order that workgroups take them: each XCD (every eighth workgroup) has a
// run of neighbouring tiles, columns of `rows` tiles at a time, so that its L2 serves the
// operands they share.
__device__ inline void tile_of(uint32_t id, uint32_t total, uint32_t rows, uint32_t columns, uint32_t& row, uint32_t& column)
{
  const uint32_t per = total / 8, more = total % 8, x = id % 8;
  const uint32_t at = x * per + (x < more ? x : more) + id / 8;
  constexpr uint32_t band = 4;
  const uint32_t b = at / (band * columns), first = b * band, height = rows - first < band ? rows - first : band;
  const uint32_t in = at - b * band * columns;
  row = first + in % height;
  column = in / height;
}

// ---- operands ---------------------------------------------------------------------------------

// The power of two that brings a largest magnitude, given by its bits, to 2^13 .. 2^14.
__device__ inline int scale_of(uint32_t top) { return top ? 13 + 127 - (int)(top >> 23) : 0; }

__device__ inline uint32_t finite_bits(float x)
{
  const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
  return b < 0x7F800000u ? b : 0u;
}

__device__ inline uint16_t bits_of(__bf16 x) { return __builtin_bit_cast(uint16_t, x); }
__device__ inline uint16_t bits_of(_Float16 x) { return __builtin_bit_cast(uint16_t, x); }

// The first part of x, which becomes the rest; what is not finite has no rest.
__device__ inline uint16_t half_part(float& x)
{
  const _Float16 h = (_Float16)x;
  const float rest = x - (float)h;
  x = rest - rest == 0.0f ? rest : 0.0f;
  return bits_of(h);
}

// The first part of x in bfloat16, which becomes the rest. A float beyond the largest bfloat16
// is not rounded to infinity; what is not finite has no rest.
__device__ inline uint16_t bf16_part(float& x)
{
  const uint32_t b = __float_as_uint(x);
  const bool beyond = (b & 0x7FFFFFFFu) - 0x7F7F8000u < 0x8000u;
  const __bf16 h = (__bf16)__uint_as_float(beyond ? b & 0xFFFF0000u : b);
  const float rest = x - (float)h;
  x = rest - rest == 0.0f ? rest : 0.0f;
  return bits_of(h);
}

// Rows of floats to rows of two planes, zeros behind dim, and the rows' powers of two: a wave
// has a row.
__global__ __launch_bounds__(kBlock) void k_planes(const float* x, uint64_t ld, uint32_t rows, uint32_t dim, uint32_t width, uint64_t stride,
                                                   uint16_t* out, uint64_t plane, int32_t* scale)
{
  const uint32_t r = blockIdx.x * kWaves + threadIdx.x / 64, lane = threadIdx.x % 64;
  if (r >= rows) return;
  const float* row = x + r * ld;
  uint32_t top = 0;
  for (uint32_t at = lane * 4; at < dim; at += 256) {
    const f4 v = load_f4(row + at, dim - at);
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, finite_bits(v[e]));
  }
#pragma unroll
  for (int step = 1; step < 64; step *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, step, 64));
  const int s = scale_of(top);
  if (lane == 0) gptr(scale)[r] = s;
  typedef uint32_t u2 __attribute__((ext_vector_type(2)));
  for (uint32_t at = lane * 4; at < width; at += 256) {
    const f4 v = at < dim ? load_f4(row + at, dim - at) : f4{0, 0, 0, 0};
    uint16_t h[2][4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float rest = ldexpf(v[e], s);
      h[0][e] = half_part(rest);
      h[1][e] = bits_of((_Float16)rest);
    }
#pragma unroll
    for (int n = 0; n < 2; ++n)
      *(GLOBAL u2*)gptr(out + n * plane + r * stride + at) = u2{h[n][0] | (uint32_t)h[n][1] << 16, h[n][2] | (uint32_t)h[n][3] << 16};
  }
}

// Rows of bfloat16 to rows of whole steps, 16-byte aligned, zeros behind dim.
__global__ __launch_bounds__(kBlock) void k_align(const uint16_t* x, uint64_t ld, uint64_t rows, uint32_t dim, uint32_t width, uint64_t stride,
                                                  uint16_t* out)
{
  const uint32_t per = width / 8;
  for (uint64_t i = (uint64_t)blockIdx.x * kBlock + threadIdx.x; i < rows * per; i += (uint64_t)gridDim.x * kBlock) {
    const uint64_t r = i / per;
    const uint32_t at = (uint32_t)(i - r * per) * 8;
    *(GLOBAL u4*)gptr(out + r * stride + at) = at < dim ? load_piece(x + r * ld, at, dim) : u4{0, 0, 0, 0};
  }
}

// The row of x that is row r of the transposed operand: a table's own row, or the token in
// a place if it is counted; -1 for zeros.
template <bool kTokens>
__device__ inline int64_t row_at(const Tokens& a, uint32_t r, uint32_t rows)
{
  if constexpr (!kTokens) return r < rows ? (int64_t)r : -1;
  const int64_t t = token_at(a, r).t;
  return t >= 0 && target_of(a, t) != kNone ? t : -1;
}

// Rows of X transposed to planes of bfloat16 [dim][stride], 64 x 64 at a time: kParts of floats.
template <class X, bool kTokens>
__global__ __launch_bounds__(kBlock) void k_turn(Tokens a, const X* x, uint64_t ld, uint32_t rows, uint32_t dim, uint64_t stride, uint16_t* out,
                                                 uint64_t plane)
{
  constexpr int kPlanes = sizeof(X) == 4 ? kParts : 1;
  __shared__ float tile[64][65];
  const uint32_t r0 = blockIdx.x * 64, c0 = blockIdx.y * 64;
  {
    const uint32_t r = threadIdx.x / 4, c = threadIdx.x % 4 * 16;
    const int64_t from = row_at<kTokens>(a, r0 + r, rows);
#pragma unroll
    for (uint32_t q = 0; q < 16; q += Piece<X>::N) {
      const uint32_t at = c0 + c + q;
      const u4 v = load_raw(x + (from >= 0 ? from : 0) * ld, at, dim);
      const auto f = unpack<X>(from >= 0 && at < dim ? settled<X>(v, at, dim) : u4{0, 0, 0, 0});
#pragma unroll
      for (uint32_t e = 0; e < Piece<X>::N; ++e) tile[r][c + q + e] = f[e];
    }
  }
  __syncthreads();
  const uint32_t c = threadIdx.x / 4, r = threadIdx.x % 4 * 16;
  if (c0 + c >= dim) return;
  uint32_t w[kPlanes][8];
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    float lo = tile[r + 2 * q][c], hi = tile[r + 2 * q + 1][c];
    if constexpr (kPlanes > 1) {
#pragma unroll
      for (int n = 0; n < kPlanes; ++n) {
        const uint32_t first = bf16_part(lo);
        w[n][q] = first | (uint32_t)bf16_part(hi) << 16;
      }
    } else {
      w[0][q] = bits_of((__bf16)lo) | (uint32_t)bits_of((__bf16)hi) << 16;
    }
  }
#pragma unroll
  for (int n = 0; n < kPlanes; ++n) {
    GLOBAL u4* to = (GLOBAL u4*)gptr(out + n * plane + (uint64_t)(c0 + c) * stride + r0 + r);
    to[0] = u4{w[n][0], w[n][1], w[n][2], w[n][3]};
    to[1] = u4{w[n][4], w[n][5], w[n][6], w[n][7]};
  }
}

// ---- logits -------------------------------------------------------------------------------------

// A tile's maximum and sum of exponentials for a token.
struct Part {
  float top, sum;
};

// What the logarithms that a largest one is taken from are counted from: it, or 0 if it is
// infinite, so that a logit of infinity gives an infinite sum and those of -infinity none.
__device__ inline float base_of(float top) { return __builtin_fabsf(top) == INFINITY ? 0.0f : top; }

struct Logits {
  Matrix w, x;                 // vocabulary and tokens
  const int32_t *w_scale, *x_scale;   // of half floats: the rows' powers of two
  uint32_t steps;
  Pairs pairs;
  uint32_t v0, v1;             // the vocabulary's piece
  uint32_t rows, columns;      // tiles
  // forward
  Part* part;                  // [tiles of the vocabulary][places]
  float* at_target;            // [places]
  // backward
  const float* lse;
  uint16_t *g, *gt;            // [places][g_stride], [piece][gt_stride]
  uint64_t g_stride, gt_stride, g_plane, gt_plane;
};

template <bool kExact>
__device__ inline float exp_of(float x)
{
  constexpr float log2e = 1.44269504088896340736f;
  if constexpr (kExact) {
    // 2^(x log2 e) with what the product's rounding and log2 e's leave: off by a step of the
    // result's, in a third of expf's instructions. Beyond 2^200, zero and infinity as they are.
    const float h = x * log2e, rest = __builtin_fmaf(x, log2e, -h) + x * 1.92596299e-8f, p = __builtin_amdgcn_exp2f(h);
    const float q = __builtin_fmaf(p, rest * 0.693147180559945f, p);
    return __builtin_fabsf(h) < 200.0f ? q : p;
  }
  else return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f);
}

// E: of x and weight. kOut: planes of G, one bfloat16 or its kParts.
template <bool kBack, class E, int kOut>
__global__ __launch_bounds__(kProductBlock, 2) void k_logits(Tokens a, Logits q)
{
  constexpr bool kHalf = std::is_same<E, F16>::value, kExact = kHalf || kOut > 1;
  __shared__ __attribute__((aligned(128))) char lds[kProductLds];
  Pipe pipe(lds);
  const uint32_t tiles = q.rows * q.columns;
  uint32_t m0, n0, tm;
  Side sa, sb;
  auto enter = [&](uint32_t id) {
    uint32_t tn;
    tile_of(id, tiles, q.rows, q.columns, tm, tn);
    m0 = q.v0 + tm * kEdge;
    n0 = tn * kEdge;
    sa.base = q.w.p + (uint64_t)m0 * q.w.ld;
    sa.plane = q.w.plane;
    const int64_t t0 = token_at(a, n0).t;       // there is one: a device's places begin with its tokens
    sb.base = q.x.p + (uint64_t)t0 * q.x.ld;
    sb.plane = q.x.plane;
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      const uint32_t r = lane_row_a<8>(it), last = q.v1 - 1 - m0;
      sa.off[it] = (uint32_t)((r < last ? r : last) * q.w.ld * 2) + lane_piece(it) * 16;
      const int64_t t = token_at(a, n0 + lane_row_b(it)).t;
      sb.off[it] = (uint32_t)((t < t0 ? 0 : t - t0) * q.x.ld * 2) + lane_piece(it) * 16;
    }
    pipe.begin(sa, sb, q.steps, q.pairs);
  };
  enter(blockIdx.x);
  bool loaded = false;
  for (uint32_t id = blockIdx.x; id < tiles; id += gridDim.x) {
    f4 acc[8][4];
    pipe.run<E>(acc, sa, sb, q.steps, q.pairs, loaded);
    const uint32_t first = m0, n = n0 + lane_n(), tile = tm, tokens = n0;
    if (id + gridDim.x < tiles) enter(id + gridDim.x);
    // the lane's tokens follow each other from a multiple of four on, so they are one device's
    const Where w = token_at(a, n);
    uint32_t target[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool on = w.t >= 0 && (uint64_t)w.t + j < a.off[w.d + 1];
      target[j] = on ? target_of(a, w.t + j) : kNone;
    }
    if constexpr (kHalf) {
      int s[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] = target[j] != kNone ? gptr(q.x_scale)[w.t + j] : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t v = first + lane_m<8>(i) + e;
          const int t = gptr(q.w_scale)[v < q.v1 ? v : q.v1 - 1];
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j][e] = ldexpf(acc[i][j][e], -(t + s[j]));
        }
    }
    if (first + kEdge > q.v1) {                   // behind the vocabulary
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (first + lane_m<8>(i) + e >= q.v1)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j][e] = -INFINITY;
    }
    // whether the lane has the target's logit, for a target of kNone never
    const uint32_t m = first + lane_m<8>(0);
    auto has = [&](uint32_t t) { return t - first < kEdge && (t - m) % 32 < 8 && (t - first) / 128 == (m - first) / 128; };
    if constexpr (!kBack) {
      Part* both = reinterpret_cast<Part*>(pipe.spare());   // [2][256]: of the waves' two rows
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (has(target[j])) {
          float z = 0.0f;
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) z = target[j] == first + lane_m<8>(i) + e ? acc[i][j][e] : z;
          gptr(q.at_target)[n + j] = z;
        }
        float top = acc[0][j][0], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) top = __builtin_fmaxf(top, acc[i][j][e]);
        const float from = base_of(top);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) sum += exp_of<kExact>(acc[i][j][e] - from);
#pragma unroll
        for (int step = 16; step < 64; step *= 2) {
          const float t = __shfl_xor(top, step, 64), s = __shfl_xor(sum, step, 64);
          const float most = __builtin_fmaxf(top, t), base = base_of(most);
          sum = sum * exp_of<kExact>(top - base) + s * exp_of<kExact>(t - base);
          top = most;
        }
        if ((threadIdx.x & 48) == 0) both[(threadIdx.x >> 8) * kEdge + lane_n() + j] = {top, sum};
      }
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");   // also for the next tile's loads, before the stores
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (threadIdx.x < kEdge && tokens + threadIdx.x < a.places) {
        const Part u = both[threadIdx.x], v = both[kEdge + threadIdx.x];
        const float most = __builtin_fmaxf(u.top, v.top), base = base_of(most);
        q.part[(uint64_t)tile * a.places + tokens + threadIdx.x] = {most, u.sum * exp_of<kExact>(u.top - base) + v.sum * exp_of<kExact>(v.top - base)};
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool on = target[j] != kNone;
        const float lse = on ? gptr(q.lse)[w.t + j] : 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][e] = exp_of<kExact>(acc[i][j][e] - lse);
        if (has(target[j])) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] -= target[j] == first + lane_m<8>(i) + e ? 1.0f : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][e] = on ? acc[i][j][e] : 0.0f;
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // for the next tile's loads, before the stores
      if (n < a.places) {                         // places are a multiple of 64
        // the rows of the piece have room for whole tiles
        uint16_t* g = q.g + (uint64_t)n * q.g_stride + (m - q.v0);
        uint16_t* gt = q.gt + (uint64_t)(m - q.v0) * q.gt_stride + n;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
#pragma unroll
          for (int pl = 0; pl < kOut; ++pl) {
            uint16_t h[4][8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              u4 x;
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const __bf16 part = (__bf16)acc[i + e / 4][j][e % 4];
                h[j][e] = bits_of(part);
                if (kOut > 1) acc[i + e / 4][j][e % 4] -= (float)part;
              }
#pragma unroll
              for (int e = 0; e < 4; ++e) x[e] = h[j][2 * e] | (uint32_t)h[j][2 * e + 1] << 16;
              *(GLOBAL u4*)gptr(g + pl * q.g_plane + j * q.g_stride + 16 * i) = x;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              typedef uint32_t u2 __attribute__((ext_vector_type(2)));
              const u2 x = {h[0][e] | (uint32_t)h[1][e] << 16, h[2][e] | (uint32_t)h[3][e] << 16};
              *(GLOBAL u2*)gptr(gt + pl * q.gt_plane + (16 * i + e) * q.gt_stride) = x;
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
    }
    loaded = true;
  }
}

// ---- losses -------------------------------------------------------------------------------------

// Sums over the counted tokens of 64 places.
struct Group {
  double nll;
  uint32_t rows, pad;
};

// Joins the vocabulary's tiles of 64 tokens, 16 slices of the tiles.
__global__ __launch_bounds__(kRowsBlock) void k_loss_rows(Tokens a, const Part* part, uint32_t tiles, const float* at_target, float* nll, float* lse,
                                                          Group* group)
{
  __shared__ Part slice[kRowSlices][64];
  const uint32_t lane = threadIdx.x & 63, s = threadIdx.x >> 6, p = blockIdx.x * 64 + lane;
  float top = -INFINITY, sum = 0.0f;
  auto add = [&](Part x) {
    const float most = __builtin_fmaxf(top, x.top), base = base_of(most);
    sum = sum * expf(top - base) + x.sum * expf(x.top - base);
    top = most;
  };
#pragma unroll 4
  for (uint32_t i = s; i < tiles; i += kRowSlices) add(part[(uint64_t)i * a.places + p]);
  slice[s][lane] = {top, sum};
  __syncthreads();
  if (s) return;
  for (uint32_t i = 1; i < kRowSlices; ++i) add(slice[i][lane]);
  const Where w = token_at(a, p);
  const bool on = w.t >= 0 && target_of(a, w.t) != kNone;
  const float l = top + logf(sum), loss = l - (on ? at_target[p] : 0.0f);
  if (w.t >= 0) {
    gptr(lse)[w.t] = on ? l : 0.0f;
    gptr(nll)[w.t] = on ? loss : 0.0f;
  }
  double total = on ? (double)loss : 0.0;
#pragma unroll
  for (int step = 1; step < 64; step *= 2) total += __shfl_xor(total, step, 64);
  const uint32_t rows = (uint32_t)__popcll(__ballot(on));
  if (lane == 0) group[blockIdx.x] = {total, rows, 0};
}

// Adds the groups of every device, a wave for each in turn, and the devices.
__global__ __launch_bounds__(kRowsBlock) void k_loss_devices(Tokens a, const Group* group, float* device_loss, float* share, float* loss)
{
  __shared__ double each[kMaxK];
  const uint32_t lane = threadIdx.x & 63;
  for (uint32_t d = threadIdx.x >> 6; d < a.K; d += kRowsBlock / 64) {
    double sum = 0.0;
    uint64_t rows = 0;
    for (uint32_t i = a.place[d] / 64 + lane; i < a.place[d + 1] / 64; i += 64) {
      sum += group[i].nll;
      rows += group[i].rows;
    }
#pragma unroll
    for (int step = 1; step < 64; step *= 2) {
      sum += __shfl_xor(sum, step, 64);
      rows += __shfl_xor(rows, step, 64);
    }
    if (lane == 0) {
      const double mean = rows ? sum / (double)rows : 0.0;
      gptr(share)[d] = rows ? (float)(1.0 / (double)rows) : 0.0f;
      gptr(device_loss)[d] = (float)mean;
      each[d] = (double)a.weight[d] * mean;
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double sum = 0.0;
    for (uint32_t d = 0; d < a.K; ++d) sum += each[d];
    gptr(loss)[0] = (float)sum;
  }
}

// ---- gradients ------------------------------------------------------------------------------------

struct Gradients {
  Matrix g, gt;                // [places][piece], [piece][places]
  Matrix wt, xt;               // [dim][vocabulary], [dim][places]
  const float *share, *d_loss;
  uint32_t v0, v1, dim;
  uint32_t steps;              // of the piece
  uint32_t rows;               // tiles of dim
  uint32_t x_columns, w_columns;
  Pairs x_pairs, w_pairs;
  // The units of a split sum, of so many steps each. d_x: x_units of them for every tile.
  // d_weight: units [w_first[d], w_first[d + 1]) for every tile of device d; where it has more
  // than one, their sums go to w_sum.
  uint32_t x_units, x_per, w_per;
  uint32_t w_first[kMaxK + 1];
  float* x_sum;                // [x_units][places][dim]: also of the pieces before
  float* w_sum;                // [units][piece][dim]
  uint64_t piece;
  void* d_x;
  uint64_t ld_d_x;
  void* d_weight[kMaxK];
  uint32_t first, last;        // whether the piece is
};

// What device d's sums are multiplied with; 0 where no rows are counted, whatever d_loss is.
__device__ inline float factor_of(const Tokens& a, const Gradients& q, uint32_t d)
{
  const float share = gptr(q.share)[d];
  return share == 0.0f ? 0.0f : a.weight[d] * share * (q.d_loss ? gptr(q.d_loss)[0] : 1.0f);
}

// X, W: d_x's and d_weight's elements.
template <class X, class W>
__global__ __launch_bounds__(kProductBlock, 2) void k_gradients(Tokens a, Gradients q)
{
  __shared__ __attribute__((aligned(128))) char lds[kProductLds];
  constexpr int kGroup = 4;
  const uint32_t x_tiles = q.rows * q.x_columns, w_tiles = q.rows * q.w_columns;
  const bool of_x = blockIdx.x < x_tiles * q.x_units;
  uint32_t tm, tn, d = 0, unit, steps;
  uint64_t k0 = 0;
  if (of_x) {
    unit = blockIdx.x / x_tiles;
    tile_of(blockIdx.x - unit * x_tiles, x_tiles, q.rows, q.x_columns, tm, tn);
    const uint32_t at = unit * q.x_per;
    steps = at >= q.steps ? 0 : q.steps - at < q.x_per ? q.steps - at : q.x_per;   // a shorter last piece
    k0 = (uint64_t)at * kStep;
  } else {
    const uint32_t id = blockIdx.x - x_tiles * q.x_units;
    unit = id / w_tiles;
    tile_of(id - unit * w_tiles, w_tiles, q.rows, q.w_columns, tm, tn);
    while (q.w_first[d + 1] <= unit) ++d;
    const uint32_t all = (a.place[d + 1] - a.place[d]) / kStep, at = (unit - q.w_first[d]) * q.w_per;
    steps = all - at < q.w_per ? all - at : q.w_per;
    k0 = a.place[d] + (uint64_t)at * kStep;
  }
  const Matrix &A = of_x ? q.wt : q.xt, &B = of_x ? q.g : q.gt;
  const uint32_t m0 = tm * kEdge, n0 = tn * kEdge, ends = of_x ? a.places : q.v1 - q.v0;
  Side sa, sb;
  sa.base = A.p + (uint64_t)m0 * A.ld + (of_x ? q.v0 : 0) + k0;
  sa.plane = A.plane;
  sb.base = B.p + (uint64_t)n0 * B.ld + k0;
  sb.plane = B.plane;
#pragma unroll
  for (int it = 0; it < 4; ++it) {
    const uint32_t ra = lane_row_a<kGroup>(it), rb = lane_row_b(it), last_m = q.dim - 1 - m0, last_n = ends - 1 - n0;
    sa.off[it] = (uint32_t)((ra < last_m ? ra : last_m) * A.ld * 2) + lane_piece(it) * 16;
    sb.off[it] = (uint32_t)((rb < last_n ? rb : last_n) * B.ld * 2) + lane_piece(it) * 16;
  }
  Pipe pipe(lds);
  f4 acc[8][4];
  const Pairs pairs = of_x ? q.x_pairs : q.w_pairs;
  pipe.begin(sa, sb, steps, pairs);
  pipe.run<BF16>(acc, sa, sb, steps, pairs, false);
  const uint32_t n = n0 + lane_n();
  if (of_x) {
    if (n >= a.places) return;
    const Where w = token_at(a, n);
    const float c = q.x_units == 1 && q.last && w.t >= 0 ? factor_of(a, q, w.d) : 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (w.t < 0 || (uint64_t)w.t + j >= a.off[w.d + 1]) break;
      const bool on = target_of(a, w.t + j) != kNone;
      float* sum = q.x_sum + ((uint64_t)unit * a.places + n + j) * q.dim;
      X* to = (X*)q.d_x + (uint64_t)(w.t + j) * q.ld_d_x;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t m = m0 + lane_m<kGroup>(i), left = q.dim - m;
        if (m >= q.dim) continue;
        f4 x = acc[i][j];
        if (!q.first) x += load_f4(sum + m, left);
        if (q.x_units > 1 || !q.last) store_f4(sum + m, x, left);
        else store_f4(to + m, on ? x * c : f4{0, 0, 0, 0}, left);
      }
    }
  } else {
    const bool whole = q.w_first[d + 1] - q.w_first[d] == 1;
    const float c = whole ? factor_of(a, q, d) : 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (n + j >= ends) break;
      W* to = (W*)q.d_weight[d] + (uint64_t)(q.v0 + n + j) * q.dim;
      float* sum = q.w_sum + ((uint64_t)unit * q.piece + n + j) * q.dim;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t m = m0 + lane_m<kGroup>(i), left = q.dim - m;
        if (m >= q.dim) continue;
        if (whole) store_f4(to + m, acc[i][j] * c, left);
        else store_f4(sum + m, acc[i][j], left);
      }
    }
  }
}

// Adds the units of d_x: a lane has four elements of a token.
template <class X>
__global__ __launch_bounds__(kBlock) void k_join_x(Tokens a, Gradients q, Share share)
{
  for_all_pieces(share, a.places, [&](uint64_t p, uint32_t g) {
    const Where w = token_at(a, (uint32_t)p);
    if (w.t < 0) return;
    const uint32_t m = g * 4, left = q.dim - m;
    f4 x = {0, 0, 0, 0};
    for (uint32_t u = 0; u < q.x_units; ++u) x += load_f4(q.x_sum + ((uint64_t)u * a.places + p) * q.dim + m, left);
    const bool on = target_of(a, w.t) != kNone;
    store_f4((X*)q.d_x + (uint64_t)w.t * q.ld_d_x + m, on ? x * factor_of(a, q, w.d) : f4{0, 0, 0, 0}, left);
  });
}

// Adds the units of d_weight of the devices that have several.
template <class W>
__global__ __launch_bounds__(kBlock) void k_join_weight(Tokens a, Gradients q, Share share)
{
  const uint32_t d = blockIdx.y, lo = q.w_first[d], hi = q.w_first[d + 1];
  if (hi - lo == 1) return;
  const float c = factor_of(a, q, d);
  for_all_pieces(share, q.v1 - q.v0, [&](uint64_t v, uint32_t g) {
    const uint32_t m = g * 4, left = q.dim - m;
    f4 x = {0, 0, 0, 0};
    for (uint32_t u = lo; u < hi; ++u) x += load_f4(q.w_sum + ((uint64_t)u * q.piece + v) * q.dim + m, left);
    store_f4((W*)q.d_weight[d] + (q.v0 + v) * q.dim + m, x * c, left);
  });
}

// ---- host -------------------------------------------------------------------------------------------

uint64_t size_of(int32_t type) { return type == SCADLES_BF16 ? 2 : 4; }
uint64_t round_up(uint64_t x, uint64_t to) { return div_up(x, to) * to; }

// Elements between rows of n, a multiple of 64: an odd number of 128-byte lines.
uint64_t stride_of(uint64_t n) { return n / 64 % 2 ? n : n + 64; }

scadles_status check_ce(const scadles_cross_entropy* ce)
{
  if (!ce) return fail(SCADLES_EINVAL, "cross_entropy is NULL");
  if (!ce->vocab || ce->vocab > kMost) return fail(SCADLES_EINVAL, "vocab = %llu is outside [1, 2^22]", (unsigned long long)ce->vocab);
  if (!ce->dim || ce->dim > 65536) return fail(SCADLES_EINVAL, "dim = %u is outside [1, 65536]", ce->dim);
  if ((ce->type != SCADLES_F32 && ce->type != SCADLES_BF16) || (ce->grad_type != SCADLES_F32 && ce->grad_type != SCADLES_BF16))
    return fail(SCADLES_EINVAL, "unknown type %d or grad_type %d", ce->type, ce->grad_type);
  if (ce->target_bytes != 4 && ce->target_bytes != 8) return fail(SCADLES_EINVAL, "target_bytes must be 4 or 8");
  return SCADLES_OK;
}

// The places of the tokens.
void make_tokens(const scadles_cross_entropy* ce, const scadles_batch* b, const float* weights, const void* target, Tokens& a)
{
  std::memset(&a, 0, sizeof(a));
  a.K = b->devices;
  a.target = target;
  a.vocab = (uint32_t)ce->vocab;
  a.wide = ce->target_bytes == 8;
  uint64_t p = 0;
  for (uint32_t d = 0; d < a.K; ++d) {
    a.off[d] = b->tok_off[d];
    a.place[d] = (uint32_t)p;
    a.weight[d] = weights ? weights[d] : 1.0f;
    p += round_up(b->tok_off[d + 1] - b->tok_off[d], 64);
  }
  a.off[a.K] = b->tokens;
  a.place[a.K] = (uint32_t)p;
  a.places = (uint32_t)p;
}

// Whether a matrix can be multiplied where it is.
bool is_operand(const scadles_cross_entropy* ce, const void* p, uint64_t ld)
{
  return ce->type == SCADLES_BF16 && ce->dim % kStep == 0 && ld % 8 == 0 && is_aligned(p, 16) && ld <= 1u << 22;
}

// The products of parts that a gradient of a type has, of x or weight (A) and G (B), the greatest last.
// Float gradients: all but those of 2^-24 of the first and less, six, or three of bfloat16 x and weight.
// bfloat16 gradients, whose own rounding is 2^-8: those down to 2^-8, which leave 2^-16; of bfloat16 x and
// weight, two, or one if all gradients are bfloat16 and G is rounded like them.
Pairs pairs_of(const scadles_cross_entropy* ce, int32_t type)
{
  if (ce->type == SCADLES_F32) return type == SCADLES_F32 ? Pairs{6, 0x001102, 0x010120} : Pairs{3, 0x001, 0x010};
  if (type == SCADLES_F32) return {3, 0, 0x012};
  return ce->grad_type == SCADLES_F32 ? Pairs{2, 0, 0x01} : Pairs{1, 0, 0};
}

// How a call is done, and its arrays in the workspace.
struct Plan {
  bool half;                   // x and weight in half floats for the logits
  uint32_t planes;             // 2 of these, else 1
  uint32_t t_planes, g_planes; // of x and weight transposed and of G: kParts of floats, else 1
  uint64_t x_width, x_stride;  // of their rows
  uint64_t vocab_width, wt_stride, xt_stride;
  uint64_t piece, g_stride;    // vocabulary entries at a time
  uint32_t x_units, x_per, w_per, w_units;
  uint16_t *x, *w, *xt, *wt, *g, *gt;
  int32_t *x_scale, *w_scale;
  Part* part;
  float *at_target, *x_sum, *w_sum;
  Group* group;
  uint64_t bytes;
};

// Vocabulary entries of a piece: as many rows of tiles as a plane of G's share of kPieceBytes
// holds, or a few less where the tiles then come in whole rounds of the compute units.
uint64_t piece_of(uint64_t vocab, uint64_t places)
{
  const uint64_t row = places * 2 * kEdge, columns = div_up(places, kEdge), all = div_up(vocab, kEdge);
  uint64_t most = row ? kPieceBytes / 2 / row : all;
  if (most < kLeastPiece / kEdge) most = kLeastPiece / kEdge;
  if (most >= all) return all * kEdge;
  uint64_t best = most;
  double full = 0.0;
  for (uint64_t r = most; 2 * r >= most && r; --r) {
    const uint64_t tiles = r * columns;
    const double f = (double)tiles / (double)round_up(tiles, kComputeUnits);
    if (f > full * 1.02) {
      full = f;
      best = r;
    }
  }
  return best * kEdge;
}

void plan_call(const scadles_cross_entropy* ce, const Tokens& a, bool backward, bool own_x, bool own_w, char* ws, Plan& p)
{
  std::memset(&p, 0, sizeof(p));
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) {
    const uint64_t here = at;
    at = round_up(at + bytes, 256);
    return ws + here;
  };
  const uint64_t tokens = a.off[a.K], places = a.places, V = ce->vocab;
  p.half = ce->type == SCADLES_F32;
  p.planes = p.half ? 2 : 1;
  p.x_width = round_up(ce->dim, kStep);
  p.x_stride = stride_of(p.x_width);
  if (!own_x) p.x = (uint16_t*)take(tokens * p.x_stride * 2 * p.planes);
  if (!own_w) p.w = (uint16_t*)take(V * p.x_stride * 2 * p.planes);
  if (p.half) {
    p.x_scale = (int32_t*)take(tokens * 4);
    p.w_scale = (int32_t*)take(V * 4);
  }
  if (!backward) {
    p.part = (Part*)take(div_up(V, kEdge) * places * sizeof(Part));
    p.at_target = (float*)take(places * 4);
    p.group = (Group*)take(places / 64 * sizeof(Group));
    p.bytes = at;
    return;
  }
  p.t_planes = p.half ? kParts : 1;
  p.g_planes = p.half || ce->grad_type == SCADLES_F32 ? kParts : 1;
  p.vocab_width = round_up(V, kStep);
  p.wt_stride = stride_of(p.vocab_width);
  p.xt_stride = stride_of(places);
  p.piece = piece_of(V, places);
  p.g_stride = stride_of(p.piece);
  p.xt = (uint16_t*)take(ce->dim * p.xt_stride * 2 * p.t_planes);
  p.wt = (uint16_t*)take(ce->dim * p.wt_stride * 2 * p.t_planes);
  p.g = (uint16_t*)take(places * p.g_stride * 2 * p.g_planes);
  p.gt = (uint16_t*)take(p.piece * p.xt_stride * 2 * p.g_planes);
  // units: each about the 256th part of a piece's steps
  const uint32_t x_pairs = pairs_of(ce, ce->type).n, w_pairs = pairs_of(ce, ce->grad_type).n;
  const uint64_t rows = div_up(ce->dim, kEdge), steps = (p.piece < V ? p.piece : p.vocab_width) / kStep;
  const uint64_t x_all = rows * div_up(places, kEdge) * steps * x_pairs, w_tiles = rows * div_up(p.piece, kEdge);
  const uint64_t w_all = w_tiles * (places / kStep) * w_pairs;
  uint64_t per = div_up(x_all + w_all, kComputeUnits);
  if (per < kLeastSteps) per = kLeastSteps;
  p.x_units = (uint32_t)div_up(steps * x_pairs, per);
  p.x_per = (uint32_t)div_up(steps, p.x_units);
  p.x_units = (uint32_t)div_up(steps, p.x_per);
  p.w_per = (uint32_t)div_up(per, w_pairs);
  bool several = false;
  for (uint32_t d = 0; d < a.K; ++d) {
    const uint64_t n = div_up((a.place[d + 1] - a.place[d]) / kStep, p.w_per);
    p.w_units += (uint32_t)(n ? n : 1);
    several |= n > 1;
  }
  if (p.piece < V || p.x_units > 1) p.x_sum = (float*)take(p.x_units * places * ce->dim * 4);
  if (several) p.w_sum = (float*)take(p.w_units * p.piece * ce->dim * 4);
  p.bytes = at;
}

scadles_status check_arrays(const scadles_cross_entropy* ce, const scadles_batch* b, const float* weights, const void* x, uint64_t ld_x,
                            const void* weight, uint64_t ld_w, const void* target, const scadles_cross_entropy_out* out)
{
  const uint64_t es = size_of(ce->type);
  if (b->tokens > kMost) return fail(SCADLES_EINVAL, "more than 2^22 tokens");
  if (weights)
    for (uint32_t d = 0; d < b->devices; ++d)
      if (!std::isfinite(weights[d]) || weights[d] < 0.0f) return fail(SCADLES_EINVAL, "weight %u is negative or not finite", d);
  if (!weight || (b->tokens && (!x || !target))) return fail(SCADLES_EINVAL, "x, weight and target must not be NULL");
  if (!is_aligned(x, es) || !is_aligned(weight, es) || !is_aligned(target, ce->target_bytes))
    return fail(SCADLES_EINVAL, "x, weight or target is not aligned to its elements");
  if (ld_x < ce->dim || ld_w < ce->dim || ld_x >= 1ull << 31 || ld_w >= 1ull << 31)
    return fail(SCADLES_EINVAL, "ld_x or ld_weight is smaller than dim, or 2^31 or more");
  if (!out) return fail(SCADLES_EINVAL, "out is NULL");
  if (!out->lse && b->tokens) return fail(SCADLES_EINVAL, "lse is NULL");
  if (!out->share) return fail(SCADLES_EINVAL, "share is NULL");
  if (!is_aligned(out->lse, 4) || !is_aligned(out->share, 4)) return fail(SCADLES_EINVAL, "lse or share is not 4-byte aligned");
  return SCADLES_OK;
}

scadles_status check_space(const void* ws, size_t ws_bytes, uint64_t need)
{
  if (!ws || !is_aligned(ws, 256)) return fail(SCADLES_EWORKSPACE, "workspace must be 256-byte aligned and not NULL");
  if (ws_bytes < need) return fail(SCADLES_EWORKSPACE, "workspace has %zu bytes, needs %zu", ws_bytes, (size_t)need);
  return SCADLES_OK;
}

struct Range {
  const void* p;
  uint64_t bytes;
};

// An operand of the logits: where it is, or in planes.
Matrix operand(const scadles_cross_entropy* ce, const Plan& p, const void* x, uint64_t ld, uint64_t rows, uint16_t* to, int32_t* scale, hipStream_t st)
{
  if (!to) return {(const uint16_t*)x, 0, ld};
  const uint64_t plane = rows * p.x_stride;
  if (rows) {
    if (p.half)
      k_planes<<<(uint32_t)div_up(rows, kWaves), kBlock, 0, st>>>((const float*)x, ld, (uint32_t)rows, ce->dim, (uint32_t)p.x_width, p.x_stride, to,
                                                                  plane, scale);
    else
      k_align<<<grid_of(div_up(rows * (p.x_width / 8), kBlock)), kBlock, 0, st>>>((const uint16_t*)x, ld, rows, ce->dim, (uint32_t)p.x_width,
                                                                                  p.x_stride, to);
  }
  return {to, plane, p.x_stride};
}

void prepare(Logits& q, const scadles_cross_entropy* ce, const Tokens& a, const Plan& p, const void* x, uint64_t ld_x, const void* weight,
             uint64_t ld_w, hipStream_t st)
{
  std::memset(&q, 0, sizeof(q));
  q.x = operand(ce, p, x, ld_x, a.off[a.K], p.x, p.x_scale, st);
  q.w = operand(ce, p, weight, ld_w, ce->vocab, p.w, p.w_scale, st);
  q.x_scale = p.x_scale;
  q.w_scale = p.w_scale;
  q.steps = (uint32_t)(p.x_width / kStep);
  q.pairs = p.half ? Pairs{3, 0x010, 0x001} : Pairs{1, 0, 0};
  q.columns = (uint32_t)div_up(a.places, kEdge);
}

uint32_t blocks_for(const Logits& q)
{
  const uint32_t tiles = q.rows * q.columns;
  return tiles < kComputeUnits ? tiles : kComputeUnits;
}

hipError_t forward(const scadles_cross_entropy* ce, const Tokens& a, const Plan& p, const void* x, uint64_t ld_x, const void* weight, uint64_t ld_w,
                   const scadles_cross_entropy_out* out, hipStream_t st)
{
  if (a.places) {
    Logits q;
    prepare(q, ce, a, p, x, ld_x, weight, ld_w, st);
    q.v1 = a.vocab;
    q.rows = (uint32_t)div_up(a.vocab, kEdge);
    q.part = p.part;
    q.at_target = p.at_target;
    if (p.half) k_logits<false, F16, 1><<<blocks_for(q), kProductBlock, 0, st>>>(a, q);
    else k_logits<false, BF16, 1><<<blocks_for(q), kProductBlock, 0, st>>>(a, q);
    k_loss_rows<<<a.places / 64, kRowsBlock, 0, st>>>(a, p.part, q.rows, p.at_target, out->nll, out->lse, p.group);
  }
  k_loss_devices<<<1, kRowsBlock, 0, st>>>(a, p.group, out->device_loss, out->share, out->loss);
  return hipGetLastError();
}

// The operands of the gradients' products, transposed.
template <class X>
void turn(const scadles_cross_entropy* ce, const Tokens& a, const Plan& p, const void* x, uint64_t ld_x, const void* weight, uint64_t ld_w,
          bool tokens, hipStream_t st)
{
  const uint32_t dim = ce->dim, down = (uint32_t)div_up(dim, 64), V = (uint32_t)ce->vocab, T = (uint32_t)a.off[a.K];
  k_turn<X, false><<<dim3((uint32_t)(p.vocab_width / 64), down), kBlock, 0, st>>>(a, (const X*)weight, ld_w, V, dim, p.wt_stride, p.wt, dim * p.wt_stride);
  if (tokens) k_turn<X, true><<<dim3(a.places / 64, down), kBlock, 0, st>>>(a, (const X*)x, ld_x, T, dim, p.xt_stride, p.xt, dim * p.xt_stride);
}

template <class X, class W>
hipError_t backward(const scadles_cross_entropy* ce, const Tokens& a, const Plan& p, const void* x, uint64_t ld_x, const void* weight, uint64_t ld_w,
                    const scadles_cross_entropy_out* out, const float* d_loss, void* d_x, uint64_t ld_d_x, void* const* d_weight, hipStream_t st)
{
  constexpr int kOut = sizeof(X) == 4 || sizeof(W) == 4 ? kParts : 1;
  typedef typename std::conditional<sizeof(X) == 4, F16, BF16>::type In;
  const uint32_t dim = ce->dim;
  Logits q;
  std::memset(&q, 0, sizeof(q));
  if (a.places) {
    prepare(q, ce, a, p, x, ld_x, weight, ld_w, st);
    turn<X>(ce, a, p, x, ld_x, weight, ld_w, d_weight != nullptr, st);
  }
  q.lse = out->lse;
  q.g = p.g;
  q.gt = p.gt;
  q.g_stride = p.g_stride;
  q.gt_stride = p.xt_stride;
  q.g_plane = a.places * p.g_stride;
  q.gt_plane = p.piece * p.xt_stride;
  Gradients r;
  std::memset(&r, 0, sizeof(r));
  r.g = {p.g, q.g_plane, p.g_stride};
  r.gt = {p.gt, q.gt_plane, p.xt_stride};
  r.wt = {p.wt, dim * p.wt_stride, p.wt_stride};
  r.xt = {p.xt, dim * p.xt_stride, p.xt_stride};
  r.share = out->share;
  r.d_loss = d_loss;
  r.dim = dim;
  r.rows = (uint32_t)div_up(dim, kEdge);
  r.x_columns = q.columns;
  r.x_pairs = pairs_of(ce, ce->type);
  r.w_pairs = pairs_of(ce, ce->grad_type);
  r.x_units = p.x_units;
  r.x_per = p.x_per;
  r.w_per = p.w_per;
  for (uint32_t d = 0; d < a.K; ++d) {
    const uint64_t n = div_up((a.place[d + 1] - a.place[d]) / kStep, p.w_per);
    r.w_first[d + 1] = r.w_first[d] + (uint32_t)(n ? n : 1);
    if (d_weight) r.d_weight[d] = d_weight[d];
  }
  r.x_sum = p.x_sum;
  r.w_sum = p.w_sum;
  r.piece = p.piece;
  r.d_x = d_x;
  r.ld_d_x = ld_d_x;
  const uint32_t quads = (uint32_t)div_up(dim, 4);
  for (uint64_t v0 = 0; v0 < a.vocab; v0 += p.piece) {
    const uint64_t v1 = a.vocab - v0 < p.piece ? a.vocab : v0 + p.piece;
    q.v0 = r.v0 = (uint32_t)v0;
    q.v1 = r.v1 = (uint32_t)v1;
    q.rows = (uint32_t)div_up(v1 - v0, kEdge);
    r.steps = (uint32_t)div_up(v1 - v0, kStep);
    // the last piece may be shorter: as many units as the others', some of them without steps
    r.w_columns = d_weight ? q.rows : 0;
    r.first = v0 == 0;
    r.last = v1 == a.vocab;
    if (a.places) k_logits<true, In, kOut><<<blocks_for(q), kProductBlock, 0, st>>>(a, q);
    const uint64_t units = (uint64_t)r.rows * r.x_columns * r.x_units + (uint64_t)r.rows * r.w_columns * r.w_first[a.K];
    if (units) k_gradients<X, W><<<(uint32_t)units, kProductBlock, 0, st>>>(a, r);
    if (d_weight && p.w_sum) {
      const Share share = share_rows(v1 - v0, quads);
      k_join_weight<W><<<dim3(grid_of(div_up(v1 - v0, share.rows)), a.K), kBlock, 0, st>>>(a, r, share);
    }
  }
  if (r.x_units > 1 && a.places) {
    const Share share = share_rows(a.places, quads);
    k_join_x<X><<<grid_of(div_up(a.places, share.rows)), kBlock, 0, st>>>(a, r, share);
  }
  return hipGetLastError();
}

}  // namespace

extern "C" {

size_t scadles_cross_entropy_workspace_bytes(const scadles_cross_entropy* ce, const scadles_batch* batch, int backward)
{
  if (check_ce(ce) || check_batch(batch) || batch->tokens > kMost) return 0;
  Tokens a;
  Plan p;
  make_tokens(ce, batch, nullptr, nullptr, a);
  plan_call(ce, a, backward != 0, false, false, nullptr, p);
  return (size_t)(p.bytes < 256 ? 256 : p.bytes);
}

scadles_status scadles_cross_entropy_forward(const scadles_cross_entropy* ce, const scadles_batch* batch, const float* weights, const void* x,
                                             uint64_t ld_x, const void* weight, uint64_t ld_weight, const void* target,
                                             const scadles_cross_entropy_out* out, void* ws, size_t ws_bytes, void* stream)
{
  if (scadles_status st = check_ce(ce)) return st;
  if (scadles_status st = check_batch(batch)) return st;
  if (!weights) return fail(SCADLES_EINVAL, "weights is NULL");
  if (scadles_status st = check_arrays(ce, batch, weights, x, ld_x, weight, ld_weight, target, out)) return st;
  if ((batch->tokens && !out->nll) || !out->device_loss || !out->loss) return fail(SCADLES_EINVAL, "nll, device_loss and loss must not be NULL");
  if (!is_aligned(out->nll, 4) || !is_aligned(out->device_loss, 4) || !is_aligned(out->loss, 4))
    return fail(SCADLES_EINVAL, "an output is not 4-byte aligned");
  Tokens a;
  make_tokens(ce, batch, weights, target, a);
  Plan p;
  const uint64_t T = batch->tokens, K = batch->devices, es = size_of(ce->type);
  plan_call(ce, a, false, is_operand(ce, x, ld_x), is_operand(ce, weight, ld_weight), (char*)ws, p);
  const uint64_t need = p.bytes;
  if (scadles_status st = check_space(ws, ws_bytes, need)) return st;
  const Range at[9] = {{out->nll, T * 4}, {out->lse, T * 4}, {out->device_loss, K * 4}, {out->share, K * 4}, {out->loss, 4}, {ws, need},
                       {x, rows_bytes(T, ce->dim, ld_x, es)}, {weight, rows_bytes(ce->vocab, ce->dim, ld_weight, es)}, {target, T * ce->target_bytes}};
  for (int i = 0; i < 6; ++i)
    for (int j = i + 1; j < 9; ++j)
      if (bytes_overlap(at[i].p, at[i].bytes, at[j].p, at[j].bytes)) return fail(SCADLES_EINVAL, "an output overlaps an input, the workspace or another");
  hipStream_t st = static_cast<hipStream_t>(stream);
  return launch_status(forward(ce, a, p, x, ld_x, weight, ld_weight, out, st), "cross entropy forward");
}

scadles_status scadles_cross_entropy_backward(const scadles_cross_entropy* ce, const scadles_batch* batch, const float* weights, const void* x,
                                              uint64_t ld_x, const void* weight, uint64_t ld_weight, const void* target,
                                              const scadles_cross_entropy_out* out, const float* d_loss, void* d_x, uint64_t ld_d_x,
                                              void* const* d_weight, void* ws, size_t ws_bytes, void* stream)
{
  if (scadles_status st = check_ce(ce)) return st;
  if (scadles_status st = check_batch(batch)) return st;
  if (scadles_status st = check_arrays(ce, batch, weights, x, ld_x, weight, ld_weight, target, out)) return st;
  const uint64_t T = batch->tokens, K = batch->devices, es = size_of(ce->type), gs = size_of(ce->grad_type);
  if (T && !d_x) return fail(SCADLES_EINVAL, "d_x is NULL");
  if (!is_aligned(d_x, es) || !is_aligned(d_loss, 4)) return fail(SCADLES_EINVAL, "d_x or d_loss is not aligned to its elements");
  if (ld_d_x < ce->dim || ld_d_x >= 1ull << 31) return fail(SCADLES_EINVAL, "ld_d_x is smaller than dim, or 2^31 or more");
  Tokens a;
  make_tokens(ce, batch, weights, target, a);
  Plan p;
  plan_call(ce, a, true, is_operand(ce, x, ld_x), is_operand(ce, weight, ld_weight), (char*)ws, p);
  const uint64_t need = p.bytes;
  if (scadles_status st = check_space(ws, ws_bytes, need)) return st;
  const Range in[6] = {{x, rows_bytes(T, ce->dim, ld_x, es)}, {weight, rows_bytes(ce->vocab, ce->dim, ld_weight, es)}, {target, T * ce->target_bytes},
                       {out->lse, T * 4}, {out->share, K * 4}, {d_loss, 4}};
  const Range own[2] = {{ws, need}, {d_x, rows_bytes(T, ce->dim, ld_d_x, es)}};
  if (bytes_overlap(own[0].p, own[0].bytes, own[1].p, own[1].bytes)) return fail(SCADLES_EINVAL, "d_x overlaps the workspace");
  for (const Range& o : own)
    for (const Range& i : in)
      if (bytes_overlap(o.p, o.bytes, i.p, i.bytes)) return fail(SCADLES_EINVAL, "d_x or the workspace overlaps an input");
  const uint64_t bytes = ce->vocab * ce->dim * gs;
  for (uint32_t d = 0; d < K && d_weight; ++d) {
    const void* w = d_weight[d];
    if (!w || !is_aligned(w, gs)) return fail(SCADLES_EINVAL, "gradient %u is NULL or not aligned to its elements", d);
    for (const Range& i : in)
      if (bytes_overlap(w, bytes, i.p, i.bytes)) return fail(SCADLES_EINVAL, "gradient %u overlaps an input", d);
    for (const Range& o : own)
      if (bytes_overlap(w, bytes, o.p, o.bytes)) return fail(SCADLES_EINVAL, "gradient %u overlaps d_x or the workspace", d);
    for (uint32_t c = 0; c < d; ++c)
      if (bytes_overlap(w, bytes, d_weight[c], bytes)) return fail(SCADLES_EINVAL, "gradients %u and %u overlap", c, d);
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool b = ce->type == SCADLES_BF16, gb = ce->grad_type == SCADLES_BF16;
  auto go = [&](auto f) { return f(ce, a, p, x, ld_x, weight, ld_weight, out, d_loss, d_x, ld_d_x, d_weight, st); };
  return launch_status(b ? (gb ? go(backward<uint16_t, uint16_t>) : go(backward<uint16_t, float>))
                         : (gb ? go(backward<float, uint16_t>) : go(backward<float, float>)),
                       "cross entropy backward");
}

}  // extern "C"
