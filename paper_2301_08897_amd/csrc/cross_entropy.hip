// cross_entropy.hip -- the cross entropy of a linear layer over a vocabulary, and its
// gradients, without the logits being kept.
//
//   z = weight x[t],  lse = log sum exp z,  nll = lse - z_target
//   G = c_t (softmax(z) - onehot),  d_x = G weight,  d_weight[d] = G^T x over device d
//
// Forward: k_logits multiplies a tile of 256 vocabulary entries by 256 tokens and leaves,
// in place of its logits, each token's maximum and sum of exponentials over the tile;
// k_loss_rows joins the tiles of a token. Backward, for a piece of the vocabulary at a
// time: k_logits again, which now has lse and stores G of the piece both ways round,
// tokens by vocabulary for d_x and vocabulary by tokens for d_weight; then k_gradients,
// tiles of both products in one launch. x and weight are needed with the contraction's
// index adjacent, so that k_turn writes both transposed once per call.
//
// Tokens are counted with every device's first one at a multiple of 64 (Tokens::place), so
// that a step of the product over tokens belongs to one device. A token that is
// not counted is a row of zeros wherever it is stored.
#include <cmath>
#include <cstring>

#include "product.h"
#include "vec4.h"

using namespace scadles;

namespace {

constexpr uint64_t kPieceBytes = 256ull << 20;    // of G and its transpose
constexpr uint32_t kLeastPiece = 2048;            // vocabulary entries of a piece, at least
constexpr uint32_t kNone = ~0u;
constexpr uint32_t kMost = 1u << 22;                // tokens and vocabulary entries: 32-bit offsets within a tile
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

// An operand: rows of bfloat16 planes.
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

// Rows of X to rows of planes, zeros behind dim.
template <class X>
__global__ __launch_bounds__(kBlock) void k_planes(const X* x, uint64_t ld, uint64_t rows, uint32_t dim, uint32_t width, uint32_t planes,
                                                   uint16_t* out, uint64_t plane)
{
  const uint32_t per = width / 8;
  const uint64_t i = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
  if (i >= rows * per) return;
  const uint64_t r = i / per;
  const uint32_t at = (uint32_t)(i - r * per) * 8;
  float v[8];
#pragma unroll
  for (uint32_t q = 0; q < 8; q += Piece<X>::N) {
    const uint32_t k = at + q < dim ? dim - at - q : 0;
    const auto f = unpack<X>(load_piece(x + r * ld + at + q, k));
#pragma unroll
    for (uint32_t e = 0; e < Piece<X>::N; ++e) v[q + e] = f[e];
  }
  for (uint32_t n = 0; n < planes; ++n) {
    u4 w;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t lo = next_plane(v[2 * q]), hi = next_plane(v[2 * q + 1]);
      w[q] = lo | hi << 16;
    }
    *(GLOBAL u4*)gptr(out + n * plane + r * width + at) = w;
  }
}

// Rows of X transposed to planes [dim][width], 64 x 64 at a time. The rows are those of
// a table (kTokens false: `rows` of them, then zeros) or the tokens in their places, zeros
// where there is none or it is not counted.
template <class X, bool kTokens>
__global__ __launch_bounds__(kBlock) void k_turn(Tokens a, const X* x, uint64_t ld, uint64_t rows, uint32_t dim, uint64_t width, uint32_t planes,
                                                 uint16_t* out, uint64_t plane)
{
  __shared__ float tile[64][65];
  const uint64_t r0 = (uint64_t)blockIdx.x * 64;
  const uint32_t c0 = blockIdx.y * 64;
  {
    const uint32_t r = threadIdx.x / 4, c = threadIdx.x % 4 * 16;
    int64_t from = r0 + r < rows ? (int64_t)(r0 + r) : -1;
    if constexpr (kTokens) {
      from = token_at(a, (uint32_t)(r0 + r)).t;
      if (from >= 0 && target_of(a, from) == kNone) from = -1;
    }
#pragma unroll
    for (uint32_t q = 0; q < 16; q += Piece<X>::N) {
      const uint32_t at = c0 + c + q, k = from >= 0 && at < dim ? dim - at : 0;
      const auto f = unpack<X>(load_piece(x + (from >= 0 ? from : 0) * ld + at, k));
#pragma unroll
      for (uint32_t e = 0; e < Piece<X>::N; ++e) tile[r][c + q + e] = f[e];
    }
  }
  __syncthreads();
  const uint32_t c = threadIdx.x / 4, r = threadIdx.x % 4 * 16;
  if (c0 + c >= dim) return;
  float v[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) v[e] = tile[r + e][c];
  for (uint32_t n = 0; n < planes; ++n) {
    u4 w[2];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const uint32_t lo = next_plane(v[2 * q]), hi = next_plane(v[2 * q + 1]);
      w[q / 4][q % 4] = lo | hi << 16;
    }
    GLOBAL u4* to = (GLOBAL u4*)gptr(out + n * plane + (uint64_t)(c0 + c) * width + r0 + r);
    to[0] = w[0];
    to[1] = w[1];
  }
}

// ---- logits -------------------------------------------------------------------------------------

// A tile's maximum and sum of exponentials for a token.
struct Part {
  float top, sum;
};

struct Logits {
  Matrix w, x;                 // vocabulary and tokens
  uint32_t steps;
  Pairs pairs;
  uint32_t v0, v1;             // the vocabulary's piece
  uint32_t rows, columns;      // tiles
  // forward
  Part* part;                  // [tiles of the vocabulary][places]
  float* at_target;            // [places]
  // backward
  const float *lse, *share, *d_loss;
  uint16_t *g, *gt;            // [places][piece], [piece][places]
  uint64_t plane;              // elements between their planes
  uint32_t piece;
};

template <bool kExact>
__device__ inline float exp_of(float x)
{
  if constexpr (kExact) return expf(x);
  else return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f);
}

// kExact: G in three planes, and exponentials to all of a float's bits.
template <bool kBack, bool kExact>
__global__ __launch_bounds__(kProductBlock, 2) void k_logits(Tokens a, Logits q)
{
  __shared__ __attribute__((aligned(128))) char lds[kProductLds];
  uint32_t tm, tn;
  tile_of(blockIdx.x, q.rows * q.columns, q.rows, q.columns, tm, tn);
  const uint32_t m0 = q.v0 + tm * kEdge, n0 = tn * kEdge;
  Side sa, sb;
  sa.base = q.w.p + (uint64_t)m0 * q.w.ld;
  sa.plane = q.w.plane;
  const int64_t first = token_at(a, n0).t;      // a tile begins with a device's tokens or within them
  const int64_t t0 = first < 0 ? 0 : first;
  sb.base = q.x.p + (uint64_t)t0 * q.x.ld;
  sb.plane = q.x.plane;
#pragma unroll
  for (int it = 0; it < 4; ++it) {
    const uint32_t r = lane_row(it), last = q.v1 - 1 - m0;
    sa.off[it] = (uint32_t)((r < last ? r : last) * q.w.ld * 2) + lane_piece_a(it) * 16;
    const int64_t t = token_at(a, n0 + r).t;
    sb.off[it] = (uint32_t)((t < t0 ? 0 : t - t0) * q.x.ld * 2) + lane_piece_b(it) * 16;
  }
  f4 acc[8][4];
  multiply(acc, sa, sb, q.steps, q.pairs, lds);

  // the lane's tokens follow each other from a multiple of four on, so they are one device's
  const uint32_t m = m0 + lane_m(), n = n0 + lane_n();
  const Where w = token_at(a, n);
  uint32_t target[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const bool on = w.t >= 0 && (uint64_t)w.t + j < a.off[w.d + 1];
    target[j] = on ? target_of(a, w.t + j) : kNone;
  }
  if (m0 + kEdge > q.v1) {                        // behind the vocabulary
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (m + 4 * i + e >= q.v1)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j][e] = -INFINITY;
  }
  if constexpr (!kBack) {
    Part* both = reinterpret_cast<Part*>(lds);   // [2][256]: of the waves' two rows
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (target[j] - m < 32) {                  // this lane has the target's logit
        float z = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) z = target[j] - m == 4 * i + e ? acc[i][j][e] : z;
        gptr(q.at_target)[n + j] = z;
      }
      float top = acc[0][j][0], sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = __builtin_fmaxf(top, acc[i][j][e]);
      const float from = top == -INFINITY ? 0.0f : top;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += exp_of<kExact>(acc[i][j][e] - from);
#pragma unroll
      for (int step = 16; step < 64; step *= 2) {
        const float t = __shfl_xor(top, step, 64), s = __shfl_xor(sum, step, 64);
        const float most = __builtin_fmaxf(top, t), base = most == -INFINITY ? 0.0f : most;
        sum = sum * exp_of<kExact>(top - base) + s * exp_of<kExact>(t - base);
        top = most;
      }
      if ((threadIdx.x & 48) == 0) both[(threadIdx.x >> 8) * kEdge + lane_n() + j] = {top, sum};
    }
    __syncthreads();
    if (threadIdx.x < kEdge && n0 + threadIdx.x < a.places) {
      const Part u = both[threadIdx.x], v = both[kEdge + threadIdx.x];
      const float most = __builtin_fmaxf(u.top, v.top), base = most == -INFINITY ? 0.0f : most;
      q.part[(uint64_t)tm * a.places + n0 + threadIdx.x] = {most, u.sum * exp_of<kExact>(u.top - base) + v.sum * exp_of<kExact>(v.top - base)};
    }
  } else {
    if (n >= a.places) return;                   // places are a multiple of 64
    const float c = w.t < 0 ? 0.0f : a.weight[w.d] * gptr(q.share)[w.d] * (q.d_loss ? gptr(q.d_loss)[0] : 1.0f);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool on = target[j] != kNone;
      const float lse = on ? gptr(q.lse)[w.t + j] : 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = exp_of<kExact>(acc[i][j][e] - lse);
      if (target[j] - m < 32) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][e] -= target[j] - m == 4 * i + e ? 1.0f : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = on ? acc[i][j][e] * c : 0.0f;
    }
    // the rows of the piece have room for whole tiles
    uint16_t* g = q.g + (uint64_t)n * q.piece + (m - q.v0);
    uint16_t* gt = q.gt + (uint64_t)(m - q.v0) * a.places + n;
    constexpr int planes = kExact ? 3 : 1;
#pragma unroll
    for (int i = 0; i < 8; i += 2)
#pragma unroll
      for (int pl = 0; pl < planes; ++pl) {
        uint16_t h[4][8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          u4 x;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float rest = acc[i + e / 4][j][e % 4];
            h[j][e] = kExact ? next_plane(rest) : __builtin_bit_cast(uint16_t, (__bf16)rest);
            acc[i + e / 4][j][e % 4] = rest;
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = h[j][2 * e] | (uint32_t)h[j][2 * e + 1] << 16;
          *(GLOBAL u4*)gptr(g + pl * q.plane + j * (uint64_t)q.piece + 4 * i) = x;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          typedef uint32_t u2 __attribute__((ext_vector_type(2)));
          const u2 x = {h[0][e] | (uint32_t)h[1][e] << 16, h[2][e] | (uint32_t)h[3][e] << 16};
          *(GLOBAL u2*)gptr(gt + pl * q.plane + (4 * i + e) * (uint64_t)a.places) = x;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
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
    const float most = __builtin_fmaxf(top, x.top), base = most == -INFINITY ? 0.0f : most;
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
  uint32_t v0, v1, dim;
  uint32_t steps;              // of the piece
  uint32_t rows;               // tiles of dim
  uint32_t x_columns, w_columns;
  Pairs x_pairs, w_pairs;
  float* sum;                  // [places][dim]: d_x of the pieces before
  void* d_x;
  uint64_t ld_d_x;
  void* d_weight[kMaxK];
  uint32_t first, last;        // whether the piece is
};

template <class X, class W>
__global__ __launch_bounds__(kProductBlock, 2) void k_gradients(Tokens a, Gradients q)
{
  __shared__ __attribute__((aligned(128))) char lds[kProductLds];
  const uint32_t x_tiles = q.rows * q.x_columns, w_tiles = q.rows * q.w_columns;
  const bool of_x = blockIdx.x < x_tiles;
  uint32_t tm, tn, d = 0, steps = q.steps;
  uint64_t k0 = 0;
  if (of_x) {
    tile_of(blockIdx.x, x_tiles, q.rows, q.x_columns, tm, tn);
  } else {
    const uint32_t id = blockIdx.x - x_tiles;
    d = id / w_tiles;
    tile_of(id - d * w_tiles, w_tiles, q.rows, q.w_columns, tm, tn);
    k0 = a.place[d];
    steps = (a.place[d + 1] - a.place[d]) / kStep;
  }
  const Matrix &A = of_x ? q.wt : q.xt, &B = of_x ? q.g : q.gt;
  const uint32_t m0 = tm * kEdge, n0 = tn * kEdge, ends = of_x ? a.places : (q.v1 - q.v0);
  Side sa, sb;
  sa.base = A.p + (uint64_t)m0 * A.ld + (of_x ? q.v0 : k0);
  sa.plane = A.plane;
  sb.base = B.p + (uint64_t)n0 * B.ld + k0;
  sb.plane = B.plane;
#pragma unroll
  for (int it = 0; it < 4; ++it) {
    const uint32_t r = lane_row(it), last_m = q.dim - 1 - m0, last_n = ends - 1 - n0;
    sa.off[it] = (uint32_t)((r < last_m ? r : last_m) * A.ld * 2) + lane_piece_a(it) * 16;
    sb.off[it] = (uint32_t)((r < last_n ? r : last_n) * B.ld * 2) + lane_piece_b(it) * 16;
  }
  f4 acc[8][4];
  multiply(acc, sa, sb, steps, of_x ? q.x_pairs : q.w_pairs, lds);
  const uint32_t m = m0 + lane_m(), n = n0 + lane_n();
  if (m >= q.dim) return;
  if (of_x) {
    if (n >= a.places) return;
    const Where w = token_at(a, n);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (w.t < 0 || (uint64_t)w.t + j >= a.off[w.d + 1]) break;
      const bool on = target_of(a, w.t + j) != kNone;
      float* sum = q.sum + (uint64_t)(n + j) * q.dim + m;
      X* to = (X*)q.d_x + (uint64_t)(w.t + j) * q.ld_d_x + m;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t left = q.dim - m - 4 * i;
        if (m + 4 * i >= q.dim) break;
        f4 x = acc[i][j];
        if (!q.first) x += load_f4(sum + 4 * i, left);
        if (!q.last) store_f4(sum + 4 * i, x, left);
        else store_f4(to + 4 * i, on ? x : f4{0, 0, 0, 0}, left);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (n + j >= ends) break;
      W* to = (W*)q.d_weight[d] + (uint64_t)(q.v0 + n + j) * q.dim + m;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (m + 4 * i < q.dim) store_f4(to + 4 * i, acc[i][j], q.dim - m - 4 * i);
    }
  }
}

// ---- host -------------------------------------------------------------------------------------------

uint64_t size_of(int32_t type) { return type == SCADLES_BF16 ? 2 : 4; }
uint64_t round_up(uint64_t x, uint64_t to) { return div_up(x, to) * to; }

// The products of a matrix of one plane or three with one of `b` planes: all of one
// plane's, or six of the nine of three parts each; the largest last.
Pairs pairs_of(uint32_t a, uint32_t b)
{
  if (a == 3) return {6, 0x010210, 0x001012};
  return b == 3 ? Pairs{3, 0, 0x012} : Pairs{1, 0, 0};
}

// What a call's arrays need in the workspace.
struct Plan {
  uint64_t x_width;            // elements of a row of x's and weight's planes
  uint64_t vocab_width;        // of weight transposed
  uint32_t planes;             // of x and weight
  uint32_t g_planes;
  uint32_t piece;              // vocabulary entries at a time
  uint64_t places;
  // addresses
  uint16_t *x, *w, *xt, *wt, *g, *gt;
  Part* part;
  float *at_target, *sum;
  Group* group;
};

uint64_t plan_call(const scadles_cross_entropy* ce, uint64_t tokens, uint64_t places, bool backward, bool own_x, bool own_w, char* ws, Plan& p)
{
  std::memset(&p, 0, sizeof(p));
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) {
    const uint64_t here = at;
    at = round_up(at + bytes, 256);
    return ws + here;
  };
  p.planes = ce->type == SCADLES_F32 ? 3 : 1;
  p.g_planes = ce->type == SCADLES_F32 || ce->grad_type == SCADLES_F32 ? 3 : 1;
  p.x_width = round_up(ce->dim, kStep);
  p.vocab_width = round_up(ce->vocab, kStep);
  p.places = places;
  if (!own_x) p.x = (uint16_t*)take(tokens * p.x_width * 2 * p.planes);
  if (!own_w) p.w = (uint16_t*)take(ce->vocab * p.x_width * 2 * p.planes);
  if (!backward) {
    p.part = (Part*)take(div_up(ce->vocab, kEdge) * places * sizeof(Part));
    p.at_target = (float*)take(places * 4);
    p.group = (Group*)take(places / 64 * sizeof(Group));
    return at;
  }
  // G takes at most half of kPieceBytes, or kLeastPiece entries; the pieces are about equal
  const uint64_t row = places * 2 * p.g_planes, all = round_up(ce->vocab, kEdge);
  uint64_t piece = row ? kPieceBytes / 2 / row / kEdge * kEdge : all, bytes = kPieceBytes / 2;
  if (piece < kLeastPiece) {
    piece = kLeastPiece;
    bytes = kLeastPiece * row;
  }
  if (bytes > all * row) bytes = all * row;
  p.piece = (uint32_t)round_up(div_up(ce->vocab, div_up(ce->vocab, piece)), kEdge);
  p.xt = (uint16_t*)take(ce->dim * places * 2 * p.planes);
  p.wt = (uint16_t*)take(ce->dim * p.vocab_width * 2 * p.planes);
  p.g = (uint16_t*)take(bytes);
  p.gt = (uint16_t*)take(bytes);
  if (piece < ce->vocab) p.sum = (float*)take(places * ce->dim * 4);
  return at;
}

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

template <class X>
Matrix operand(const void* x, uint64_t ld, uint64_t rows, const scadles_cross_entropy* ce, const Plan& p, uint16_t* to, hipStream_t st)
{
  if (!to) return {(const uint16_t*)x, 0, ld};
  const uint64_t plane = rows * p.x_width;
  if (rows)
    k_planes<X><<<(uint32_t)div_up(rows * (p.x_width / 8), kBlock), kBlock, 0, st>>>((const X*)x, ld, rows, ce->dim, (uint32_t)p.x_width, p.planes,
                                                                                    to, plane);
  return {to, plane, p.x_width};
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

template <class X>
void prepare(Logits& q, const scadles_cross_entropy* ce, const Tokens& a, const Plan& p, const void* x, uint64_t ld_x, const void* weight,
             uint64_t ld_w, hipStream_t st)
{
  std::memset(&q, 0, sizeof(q));
  q.x = operand<X>(x, ld_x, a.off[a.K], ce, p, p.x, st);
  q.w = operand<X>(weight, ld_w, ce->vocab, ce, p, p.w, st);
  q.steps = (uint32_t)(p.x_width / kStep);
  q.pairs = pairs_of(p.planes, p.planes);
  q.columns = (uint32_t)div_up(a.places, kEdge);
}

template <class X>
hipError_t forward(const scadles_cross_entropy* ce, const Tokens& a, const Plan& p, const void* x, uint64_t ld_x, const void* weight, uint64_t ld_w,
                   const scadles_cross_entropy_out* out, hipStream_t st)
{
  if (a.places) {
    Logits q;
    prepare<X>(q, ce, a, p, x, ld_x, weight, ld_w, st);
    q.v1 = a.vocab;
    q.rows = (uint32_t)div_up(a.vocab, kEdge);
    q.part = p.part;
    q.at_target = p.at_target;
    k_logits<false, sizeof(X) == 4><<<q.rows * q.columns, kProductBlock, 0, st>>>(a, q);
    k_loss_rows<<<a.places / 64, kRowsBlock, 0, st>>>(a, p.part, q.rows, p.at_target, out->nll, out->lse, p.group);
  }
  k_loss_devices<<<1, kRowsBlock, 0, st>>>(a, p.group, out->device_loss, out->share, out->loss);
  return hipGetLastError();
}

template <class X, class W>
hipError_t backward(const scadles_cross_entropy* ce, const Tokens& a, const Plan& p, const void* x, uint64_t ld_x, const void* weight, uint64_t ld_w,
                    const scadles_cross_entropy_out* out, const float* d_loss, void* d_x, uint64_t ld_d_x, void* const* d_weight, hipStream_t st)
{
  Logits q;
  prepare<X>(q, ce, a, p, x, ld_x, weight, ld_w, st);
  q.lse = out->lse;
  q.share = out->share;
  q.d_loss = d_loss;
  q.g = p.g;
  q.gt = p.gt;
  q.plane = p.places * p.piece;
  q.piece = p.piece;
  Gradients r;
  std::memset(&r, 0, sizeof(r));
  const uint32_t dim = ce->dim, down = (uint32_t)div_up(dim, 64);
  if (a.places) {
    k_turn<X, false><<<dim3((uint32_t)(p.vocab_width / 64), down), kBlock, 0, st>>>(a, (const X*)weight, ld_w, ce->vocab, dim, p.vocab_width, p.planes,
                                                                                   p.wt, dim * p.vocab_width);
    if (d_weight)
      k_turn<X, true><<<dim3((uint32_t)(p.places / 64), down), kBlock, 0, st>>>(a, (const X*)x, ld_x, a.off[a.K], dim, p.places, p.planes, p.xt,
                                                                               dim * p.places);
  }
  r.g = {p.g, q.plane, p.piece};
  r.gt = {p.gt, q.plane, p.places};
  r.wt = {p.wt, dim * p.vocab_width, p.vocab_width};
  r.xt = {p.xt, dim * p.places, p.places};
  r.dim = dim;
  r.rows = (uint32_t)div_up(dim, kEdge);
  r.x_columns = q.columns;
  r.x_pairs = pairs_of(p.planes, sizeof(X) == 4 ? 3 : 1);
  r.w_pairs = pairs_of(p.planes, sizeof(X) == 4 || sizeof(W) == 4 ? 3 : 1);
  r.sum = p.sum;
  r.d_x = d_x;
  r.ld_d_x = ld_d_x;
  for (uint32_t d = 0; d < a.K && d_weight; ++d) r.d_weight[d] = d_weight[d];
  for (uint32_t v0 = 0; v0 < a.vocab; v0 += p.piece) {
    const uint32_t v1 = a.vocab - v0 < p.piece ? a.vocab : v0 + p.piece;
    q.v0 = r.v0 = v0;
    q.v1 = r.v1 = v1;
    q.rows = (uint32_t)div_up(v1 - v0, kEdge);
    r.steps = (uint32_t)div_up(v1 - v0, kStep);
    r.w_columns = d_weight ? q.rows : 0;
    r.first = v0 == 0;
    r.last = v1 == a.vocab;
    if (a.places) k_logits<true, sizeof(X) == 4 || sizeof(W) == 4><<<q.rows * q.columns, kProductBlock, 0, st>>>(a, q);
    const uint64_t tiles = (uint64_t)r.rows * r.x_columns + (uint64_t)r.rows * r.w_columns * a.K;
    if (tiles) k_gradients<X, W><<<(uint32_t)tiles, kProductBlock, 0, st>>>(a, r);
  }
  return hipGetLastError();
}

}  // namespace

extern "C" {

size_t scadles_cross_entropy_workspace_bytes(const scadles_cross_entropy* ce, uint64_t tokens, uint32_t devices, int backward)
{
  if (check_ce(ce) || tokens > kMost || !devices || devices > kMaxK) return 0;
  Plan p;
  const uint64_t places = round_up(tokens, 64) + (uint64_t)(devices - 1) * 64;
  const uint64_t n = plan_call(ce, tokens, places, backward != 0, false, false, nullptr, p);
  return (size_t)(n < 256 ? 256 : n);
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
  const uint64_t need = plan_call(ce, T, a.places, false, is_operand(ce, x, ld_x), is_operand(ce, weight, ld_weight), (char*)ws, p);
  if (scadles_status st = check_space(ws, ws_bytes, need)) return st;
  const Range at[9] = {{out->nll, T * 4}, {out->lse, T * 4}, {out->device_loss, K * 4}, {out->share, K * 4}, {out->loss, 4}, {ws, need},
                       {x, rows_bytes(T, ce->dim, ld_x, es)}, {weight, rows_bytes(ce->vocab, ce->dim, ld_weight, es)}, {target, T * ce->target_bytes}};
  for (int i = 0; i < 6; ++i)
    for (int j = i + 1; j < 9; ++j)
      if (bytes_overlap(at[i].p, at[i].bytes, at[j].p, at[j].bytes)) return fail(SCADLES_EINVAL, "an output overlaps an input, the workspace or another");
  hipStream_t st = static_cast<hipStream_t>(stream);
  return launch_status(ce->type == SCADLES_BF16 ? forward<uint16_t>(ce, a, p, x, ld_x, weight, ld_weight, out, st)
                                                : forward<float>(ce, a, p, x, ld_x, weight, ld_weight, out, st),
                       "cross entropy forward");
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
  const uint64_t need = plan_call(ce, T, a.places, true, is_operand(ce, x, ld_x), is_operand(ce, weight, ld_weight), (char*)ws, p);
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
