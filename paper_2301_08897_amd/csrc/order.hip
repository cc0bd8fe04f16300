// order.hip -- tokens sorted by expert and back: the order of the choices by
// (expert, device, token), the experts' input rows, the sum of the experts'
// outputs times the gates, and the gradients of both.
//
//   rows[pos[t][c]] = x[t]                       dispatch
//   out[t] = sum_c gate[t][c] rows[pos[t][c]]    combine (dispatch's gradient without gates)
//   d_rows[pos[t][c]] = gate[t][c] d_out[t],  d_gate[t][c] = d_out[t] . rows[pos[t][c]]
//
// The sort is the stable counting sort of sort.h with the expert as the digit.
// Chunks do not cross devices where there are several, so that the counts of
// the chunks before a device's first one are the bounds by expert and device;
// a call of one chunk searches them in its sorted items.
// All of it is bound by memory: a row of x is read once and stored k times, and
// rows are summed with the loads of all k choices in flight. 32768 tokens of 2048 bfloat16
// with 8 of 256 experts: sort 20 us in three launches, dispatch 204 (5.9 TB/s), combine 271
// (4.5), its gradients 455 (5.0), dispatch's 220 (5.5). Up to 8192 choices: one launch of 4.5 us.
#include <cstring>

#include "pieces.h"
#include "sort.h"

using namespace scadles;

namespace {

constexpr uint32_t kMaxChoices = SCADLES_ROUTER_MAX_K;
constexpr uint32_t kMaxExperts = SCADLES_ROUTER_MAX_EXPERTS;

// The chunks of a sort: device d's items are [off[d], off[d + 1]), its chunks
// [first[d], first[d + 1]) of `per` items.
struct Chunks {
  uint64_t off[kMaxK + 1];
  uint32_t first[kMaxK + 1];
  uint32_t K, per;
};

__device__ inline uint32_t find_device(const Chunks& c, uint32_t w)
{
  uint32_t d = 0;
  while (d + 1 < c.K && c.first[d + 1] <= w) ++d;
  return d;
}

// A chunk's first item and how many it has.
__device__ inline uint64_t chunk_start(const Chunks& c, uint32_t w, uint32_t& n)
{
  const uint32_t d = find_device(c, w);
  const uint64_t at = c.off[d] + (uint64_t)(w - c.first[d]) * c.per, left = c.off[d + 1] - at;
  n = left < c.per ? (uint32_t)left : c.per;
  return at;
}

__device__ inline uint32_t expert_of(const int32_t* idx, uint64_t i, uint32_t E)
{
  const uint32_t e = (uint32_t)gptr(idx)[i];
  return e < E ? e : E;
}

__global__ __launch_bounds__(kSortBlock) void k_order_count(Chunks c, const int32_t* idx, uint32_t E, uint32_t* count)
{
  __shared__ uint32_t lds[kSortDigits + 1];
  uint32_t n;
  const uint64_t at = chunk_start(c, blockIdx.x, n);
  count_chunk(lds, n, E + 1, [&](uint32_t i) { return expert_of(idx, at + i, E); }, count + (uint64_t)blockIdx.x * (E + 1));
}

// The chunk's items to their places. The only chunk (kOne) finds the first places and
// the bounds itself; else they come from k_sort_scan's sums.
template <int R, bool kOne>
__global__ __launch_bounds__(kSortBlock) void k_order_place(Chunks c, const int32_t* idx, uint32_t E, uint32_t bits, const uint32_t* before,
                                                            const uint32_t* all, int32_t* pos, int32_t* src, int32_t* bounds)
{
  __shared__ SortLds s;
  __shared__ uint16_t sorted[kOne ? R * kSortBlock : 1];
  uint32_t n = kOne ? (uint32_t)c.off[c.K] : 0;
  const uint64_t at = kOne ? 0 : chunk_start(c, blockIdx.x, n);
  uint32_t key[R], rank[R], mine, last;
  rank_chunk<R>(s, n, E + 1, bits, [&](uint32_t i) { return expert_of(idx, at + i, E); }, key, rank, mine, last);
  uint32_t there;
  if constexpr (kOne) {
    // the missing choices are digit E: with E < 1024 they are among the digits summed
    first_of_all(s, threadIdx.x == E ? 0 : mine);
    there = s.first[1024];
    if (threadIdx.x == 0) s.first[E] = there;
    __syncthreads();
  } else {
    first_of_chunk(s, before, all, E + 1, blockIdx.x);
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (key[r] == ~0u) continue;
    const uint32_t i = ((threadIdx.x >> 6) * R + r) * 64 + (threadIdx.x & 63);
    const uint32_t p = s.first[key[r]] + s.count[threadIdx.x >> 6][key[r]] + rank[r];
    const bool missing = key[r] == E;
    gptr(pos)[at + i] = missing ? -1 : (int32_t)p;
    gptr(src)[p] = missing ? -1 : (int32_t)(at + i);
    if constexpr (kOne) sorted[p] = (uint16_t)i;
  }
  if (kOne || blockIdx.x == 0) {
    if constexpr (kOne) __syncthreads();
    for (uint32_t x = threadIdx.x; x <= E * c.K; x += kSortBlock) {
      const uint32_t e = x / c.K, d = x - e * c.K;
      uint32_t b;
      if constexpr (kOne) {                     // the first of the expert's items that is not of a device before
        uint32_t lo = e < E ? s.first[e] : there, hi = e < E ? (e + 1 == E ? there : s.first[e + 1]) : there;
        while (lo < hi) {
          const uint32_t mid = (lo + hi) / 2;
          if (sorted[mid] < c.off[d]) lo = mid + 1;
          else hi = mid;
        }
        b = lo;
      } else {                                  // s.first is chunk 0's: the first of all
        b = s.first[e];
        if (d) {
          const uint32_t w = c.first[d];
          b += w < c.first[c.K] ? before[(uint64_t)w * (E + 1) + e] : all[e];
        }
      }
      gptr(bounds)[x] = (int32_t)b;
    }
  }
}

__global__ void k_order_empty(int32_t* bounds, uint32_t n)
{
  for (uint32_t x = blockIdx.x * blockDim.x + threadIdx.x; x < n; x += gridDim.x * blockDim.x) gptr(bounds)[x] = 0;
}

// ---- rows -----------------------------------------------------------------------------------------

// The choices of the tokens, and the tokens that a workgroup takes.
struct Move {
  const int32_t* pos;
  uint64_t tokens;
  uint32_t rows;             // tokens * k: what pos may name
  uint32_t dim;
  Share share;
};

// The rows of a token's choices c0 .. c0 + C - 1, kNoRow where there is none: read before what
// lies there, so that one wait is for all of them.
constexpr uint32_t kNoRow = ~0u;
template <int C>
__device__ inline void rows_of(const Move& m, uint64_t t, uint32_t k, uint32_t c0, uint32_t (&p)[C])
{
#pragma unroll
  for (int c = 0; c < C; ++c) p[c] = (uint32_t)gptr(m.pos)[t * k + (c0 + c < k ? c0 + c : k - 1)];
#pragma unroll
  for (int c = 0; c < C; ++c) p[c] = c0 + c < k && p[c] < m.rows ? p[c] : kNoRow;
}

// A piece of a token's row is loaded once and stored k times.
template <class X>
__global__ __launch_bounds__(kBlock) void k_dispatch(Move m, uint32_t k, const X* x, uint64_t ld_x, X* rows, uint64_t ld_rows)
{
  for_all_pieces(m.share, m.tokens, [&](uint64_t t, uint32_t g) {
    const uint32_t at = g * Piece<X>::N, left = m.dim - at;
    const u4 v = load_piece(x + t * ld_x, at, m.dim);
    for (uint32_t c = 0; c < k; ++c) {          // eight positions at once: 214 us instead of 203
      uint32_t p[1];
      rows_of<1>(m, t, k, c, p);
      if (p[0] != kNoRow) store_piece(rows + (uint64_t)p[0] * ld_rows + at, v, left);
    }
  });
}

// Up to C choices at once, so that their loads are in flight together.
template <class X, int C, bool kGate>
__global__ __launch_bounds__(kBlock) void k_combine(Move m, uint32_t k, const X* rows, uint64_t ld_rows, const float* gate, X* out,
                                                    uint64_t ld_out)
{
  for_all_pieces(m.share, m.tokens, [&](uint64_t t, uint32_t g) {
    const uint32_t at = g * Piece<X>::N, left = m.dim - at;
    typename Piece<X>::F sum = {};
    for (uint32_t c0 = 0; c0 < k; c0 += C) {
      u4 v[C];
      float w[C];
      uint32_t p[C];
      rows_of<C>(m, t, k, c0, p);
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (p[c] != kNoRow) {
          v[c] = load_raw(rows + (uint64_t)p[c] * ld_rows, at, m.dim);
          w[c] = kGate ? gptr(gate)[t * k + c0 + c] : 1.0f;
        }
      if (m.dim % Piece<X>::N) {     // one branch for all of them
#pragma unroll
        for (int c = 0; c < C; ++c)
          if (p[c] != kNoRow) v[c] = settled<X>(v[c], at, m.dim);
      }
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (p[c] != kNoRow) sum += kGate ? unpack<X>(v[c]) * w[c] : unpack<X>(v[c]);
    }
    store_piece_once(out + t * ld_out + at, pack<X>(sum), left);   // leaves the caches to the rows: a fifth less time
  });
}

// A group of G lanes has a token: its pieces of d_out are multiplied with the same of
// every choice's row and scaled into d_rows; the products are added over the lanes
// at the end. d_rows may be the rows: a piece is read before it is written, by the same lane
// (what the load of a row's last piece sees of the one before is dropped).
template <class X, int C, int G>
__global__ __launch_bounds__(kBlock) void k_combine_back(Move m, uint32_t k, const X* d_out, uint64_t ld_d_out, const X* rows,
                                                         uint64_t ld_rows, const float* gate, X* d_rows, uint64_t ld_d_rows, float* d_gate)
{
  const uint32_t lane = threadIdx.x % G;
  const uint64_t stride = (uint64_t)gridDim.x * (kBlock / G);
  for (uint64_t t = (uint64_t)blockIdx.x * (kBlock / G) + threadIdx.x / G; t < m.tokens; t += stride)
    for (uint32_t c0 = 0; c0 < k; c0 += C) {
      uint32_t p[C];
      float w[C], sum[C];
      rows_of<C>(m, t, k, c0, p);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        w[c] = p[c] != kNoRow ? gptr(gate)[t * k + c0 + c] : 0.0f;
        sum[c] = 0.0f;
      }
      for (uint32_t at = lane * Piece<X>::N; at < m.dim; at += G * Piece<X>::N) {
        const uint32_t left = m.dim - at;
        const u4 up = load_raw(d_out + t * ld_d_out, at, m.dim);
        u4 v[C];
        if (d_gate) {
#pragma unroll
          for (int c = 0; c < C; ++c)
            if (p[c] != kNoRow) v[c] = load_raw(rows + (uint64_t)p[c] * ld_rows, at, m.dim);
        }
        const auto g = unpack<X>(settled<X>(up, at, m.dim));
        if (d_gate) {
#pragma unroll
          for (int c = 0; c < C; ++c)
            if (p[c] != kNoRow) {
              const auto y = unpack<X>(settled<X>(v[c], at, m.dim));
#pragma unroll
              for (uint32_t q = 0; q < Piece<X>::N; ++q) sum[c] = __builtin_fmaf(g[q], y[q], sum[c]);
            }
        }
        if (d_rows) {
#pragma unroll
          for (int c = 0; c < C; ++c)
            if (p[c] != kNoRow) store_piece_once(d_rows + (uint64_t)p[c] * ld_d_rows + at, pack<X>(g * w[c]), left);
        }
      }
      if (d_gate) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
          for (int step = 1; step < G; step *= 2) sum[c] += __shfl_xor(sum[c], step, 64);
          if (lane == 0 && c0 + c < k) gptr(d_gate)[t * k + c0 + c] = p[c] != kNoRow ? sum[c] : 0.0f;
        }
      }
    }
}

// ---- host -------------------------------------------------------------------------------------------

// Chunks of rounds * 1024 items that do not cross devices; returns how many.
uint32_t make_chunks(const scadles_batch* b, uint32_t k, uint32_t rounds, Chunks& c)
{
  std::memset(&c, 0, sizeof(c));
  c.K = b->devices;
  c.per = rounds * kSortBlock;
  uint64_t w = 0;
  for (uint32_t d = 0; d < c.K; ++d) {
    c.off[d] = b->tok_off[d] * k;
    c.first[d] = (uint32_t)w;
    w += div_up((b->tok_off[d + 1] - b->tok_off[d]) * k, c.per);
  }
  c.off[c.K] = b->tokens * k;
  c.first[c.K] = (uint32_t)w;
  return (uint32_t)w;
}

uint64_t sort_bytes(uint64_t chunks, uint32_t digits) { return div_up((chunks + 1) * digits * 4, 256) * 256; }

template <bool kOne>
void place(uint32_t rounds, uint32_t W, const Chunks& c, const int32_t* idx, uint32_t E, const uint32_t* before, const uint32_t* all,
           int32_t* pos, int32_t* src, int32_t* bounds, hipStream_t st)
{
  const uint32_t bits = sort_bits(E + 1);
  if (rounds == 1) k_order_place<1, kOne><<<W, kSortBlock, 0, st>>>(c, idx, E, bits, before, all, pos, src, bounds);
  else if (rounds == 2) k_order_place<2, kOne><<<W, kSortBlock, 0, st>>>(c, idx, E, bits, before, all, pos, src, bounds);
  else if (rounds <= 4) k_order_place<4, kOne><<<W, kSortBlock, 0, st>>>(c, idx, E, bits, before, all, pos, src, bounds);
  else k_order_place<8, kOne><<<W, kSortBlock, 0, st>>>(c, idx, E, bits, before, all, pos, src, bounds);
}

scadles_status check_order(const scadles_order* o)
{
  if (!o) return fail(SCADLES_EINVAL, "order is NULL");
  if (!o->k || o->k > kMaxChoices) return fail(SCADLES_EINVAL, "k = %u is outside [1, %u]", o->k, kMaxChoices);
  if (o->tokens > 0x7FFFFFFFull / o->k) return fail(SCADLES_EINVAL, "tokens * k is above 2^31 - 1");
  if (!o->dim || o->dim >= 1u << 24) return fail(SCADLES_EINVAL, "dim = %u is outside [1, 2^24)", o->dim);
  if (o->type != SCADLES_F32 && o->type != SCADLES_BF16) return fail(SCADLES_EINVAL, "unknown type %d", o->type);
  if (o->tokens && !o->pos) return fail(SCADLES_EINVAL, "pos is NULL");
  if (!is_aligned(o->pos, 4)) return fail(SCADLES_EINVAL, "pos is not 4-byte aligned");
  return SCADLES_OK;
}

uint64_t esize(const scadles_order* o) { return o->type == SCADLES_BF16 ? 2 : 4; }

// One array of rows.
struct Span {
  const void* p;
  uint64_t rows, ld;
  const char* name;
};

scadles_status check_span(const scadles_order* o, const Span& s)
{
  if (o->tokens && !s.p) return fail(SCADLES_EINVAL, "%s is NULL", s.name);
  if (!is_aligned(s.p, esize(o))) return fail(SCADLES_EINVAL, "%s is not aligned to its elements", s.name);
  if (s.ld < o->dim) return fail(SCADLES_EINVAL, "the ld of %s is smaller than dim", s.name);
  if (s.ld >= 1ull << 31) return fail(SCADLES_EINVAL, "the ld of %s is 2^31 or more", s.name);
  return SCADLES_OK;
}

bool spans_overlap(const scadles_order* o, const Span& a, const Span& b)
{
  return bytes_overlap(a.p, rows_bytes(a.rows, o->dim, a.ld, esize(o)), b.p, rows_bytes(b.rows, o->dim, b.ld, esize(o)));
}

bool overlaps(const scadles_order* o, const Span& a, const void* p, uint64_t bytes)
{
  return bytes_overlap(a.p, rows_bytes(a.rows, o->dim, a.ld, esize(o)), p, bytes);
}

// A lane has one piece of one token (of 32768 x 2048 bfloat16 in 8 rows each, four pieces: dispatch 232
// us instead of 202, combine 284 instead of 269, its backward pass's sums 231 instead of 219).
Move make_move(const scadles_order* o, uint64_t n)
{
  return {o->pos, o->tokens, (uint32_t)(o->tokens * o->k), o->dim, share_rows(o->tokens, div_up(o->dim, n))};
}

template <class X>
void dispatch(const scadles_order* o, const void* x, uint64_t ld_x, void* rows, uint64_t ld_rows, hipStream_t st)
{
  const Move m = make_move(o, Piece<X>::N);
  k_dispatch<X><<<grid_of(div_up(o->tokens, m.share.rows)), kBlock, 0, st>>>(m, o->k, (const X*)x, ld_x, (X*)rows, ld_rows);
}

template <class X, int C>
void combine_of(const scadles_order* o, const void* rows, uint64_t ld_rows, const float* gate, void* out, uint64_t ld_out, hipStream_t st)
{
  const Move m = make_move(o, Piece<X>::N);
  const uint32_t W = grid_of(div_up(o->tokens, m.share.rows));
  if (gate) k_combine<X, C, true><<<W, kBlock, 0, st>>>(m, o->k, (const X*)rows, ld_rows, gate, (X*)out, ld_out);
  else k_combine<X, C, false><<<W, kBlock, 0, st>>>(m, o->k, (const X*)rows, ld_rows, gate, (X*)out, ld_out);
}

template <class X>
void combine(const scadles_order* o, const void* rows, uint64_t ld_rows, const float* gate, void* out, uint64_t ld_out, hipStream_t st)
{
  if (o->k == 1) combine_of<X, 1>(o, rows, ld_rows, gate, out, ld_out, st);
  else if (o->k == 2) combine_of<X, 2>(o, rows, ld_rows, gate, out, ld_out, st);
  else if (o->k <= 4) combine_of<X, 4>(o, rows, ld_rows, gate, out, ld_out, st);
  else combine_of<X, 8>(o, rows, ld_rows, gate, out, ld_out, st);
}

template <class X, int C>
void combine_back_of(const scadles_order* o, const void* d_out, uint64_t ld_d_out, const void* rows, uint64_t ld_rows, const float* gate,
                     void* d_rows, uint64_t ld_d_rows, float* d_gate, hipStream_t st)
{
  const Move m = make_move(o, Piece<X>::N);
  auto go = [&](auto kernel, uint32_t G) {
    kernel<<<grid_of(div_up(o->tokens, kBlock / G)), kBlock, 0, st>>>(m, o->k, (const X*)d_out, ld_d_out, (const X*)rows, ld_rows, gate,
                                                                       (X*)d_rows, ld_d_rows, d_gate);
  };
  if (m.share.pieces <= 8) go(k_combine_back<X, C, 8>, 8);
  else if (m.share.pieces <= 32) go(k_combine_back<X, C, 32>, 32);
  else go(k_combine_back<X, C, 64>, 64);
}

template <class X>
void combine_back(const scadles_order* o, const void* d_out, uint64_t ld_d_out, const void* rows, uint64_t ld_rows, const float* gate,
                  void* d_rows, uint64_t ld_d_rows, float* d_gate, hipStream_t st)
{
  auto of = [&](auto f) { f(o, d_out, ld_d_out, rows, ld_rows, gate, d_rows, ld_d_rows, d_gate, st); };
  if (o->k == 1) of(combine_back_of<X, 1>);
  else if (o->k == 2) of(combine_back_of<X, 2>);
  else if (o->k <= 4) of(combine_back_of<X, 4>);
  else of(combine_back_of<X, 8>);
}

}  // namespace

namespace scadles {

__global__ __launch_bounds__(kSortBlock) void k_sort_scan(uint32_t* count, uint32_t* all, uint32_t W, uint32_t digits)
{
  __shared__ uint32_t part[kScanSlices][kScanDigits];
  const uint32_t lane = threadIdx.x % kScanDigits, s = threadIdx.x / kScanDigits;
  const uint32_t d = blockIdx.x * kScanDigits + lane, per = (W + kScanSlices - 1) / kScanSlices;
  const uint32_t lo = s * per < W ? s * per : W, hi = lo + per < W ? lo + per : W;
  uint32_t sum = 0;
  if (d < digits) {
#pragma unroll 8
    for (uint32_t w = lo; w < hi; ++w) sum += count[(uint64_t)w * digits + d];
  }
  part[s][lane] = sum;
  __syncthreads();
  uint32_t at = 0, total = 0;
  for (uint32_t q = 0; q < kScanSlices; ++q) {
    const uint32_t x = part[q][lane];
    at += q < s ? x : 0;
    total += x;
  }
  if (d >= digits) return;
  if (s == 0) all[d] = total;
  for (uint32_t w0 = lo; w0 < hi; w0 += 8) {        // eight loads before the stores that follow them
    uint32_t x[8];
#pragma unroll
    for (uint32_t q = 0; q < 8; ++q) x[q] = w0 + q < hi ? count[(uint64_t)(w0 + q) * digits + d] : 0;
#pragma unroll
    for (uint32_t q = 0; q < 8; ++q)
      if (w0 + q < hi) {
        count[(uint64_t)(w0 + q) * digits + d] = at;
        at += x[q];
      }
  }
}

void launch_sort_scan(uint32_t* count, uint32_t* all, uint32_t W, uint32_t digits, hipStream_t st)
{
  k_sort_scan<<<(uint32_t)div_up(digits, kScanDigits), kSortBlock, 0, st>>>(count, all, W, digits);
}

scadles_status check_batch(const scadles_batch* b)
{
  if (!b) return fail(SCADLES_EINVAL, "batch is NULL");
  if (b->tokens > 0x7FFFFFFFull) return fail(SCADLES_EINVAL, "more than 2^31 - 1 tokens");
  if (!b->devices || b->devices > kMaxK) return fail(SCADLES_EINVAL, "devices = %u is outside [1, %d]", b->devices, kMaxK);
  if (!b->tok_off) return fail(SCADLES_EINVAL, "tok_off is NULL");
  if (b->tok_off[0] != 0 || b->tok_off[b->devices] != b->tokens) return fail(SCADLES_EINVAL, "tok_off must run from 0 to tokens");
  for (uint32_t d = 0; d < b->devices; ++d)
    if (b->tok_off[d + 1] < b->tok_off[d]) return fail(SCADLES_EINVAL, "tok_off must not decrease");
  return SCADLES_OK;
}

}  // namespace scadles

extern "C" {

size_t scadles_order_workspace_bytes(uint64_t tokens, uint32_t experts, uint32_t k)
{
  if (!experts || experts > kMaxExperts || !k || k > kMaxChoices || k > experts || tokens > 0x7FFFFFFFull / k) return 0;
  // every device's last chunk may be partly filled
  return (size_t)sort_bytes(sort_chunks(tokens * k) + kMaxK, experts + 1);
}

scadles_status scadles_order_sort(const scadles_batch* batch, const int32_t* idx, uint32_t experts, uint32_t k, int32_t* pos, int32_t* src,
                                  int32_t* bounds, void* ws, size_t ws_bytes, void* stream)
{
  if (scadles_status st = check_batch(batch)) return st;
  if (!experts || experts > kMaxExperts) return fail(SCADLES_EINVAL, "experts = %u is outside [1, %u]", experts, kMaxExperts);
  if (!k || k > experts || k > kMaxChoices) return fail(SCADLES_EINVAL, "k = %u is outside [1, min(experts, %u)]", k, kMaxChoices);
  if (batch->tokens > 0x7FFFFFFFull / k) return fail(SCADLES_EINVAL, "tokens * k is above 2^31 - 1");
  const uint64_t N = batch->tokens * k, cells = (uint64_t)experts * batch->devices + 1;
  if (N && (!idx || !pos || !src)) return fail(SCADLES_EINVAL, "idx, pos and src must not be NULL");
  if (!bounds) return fail(SCADLES_EINVAL, "bounds is NULL");
  for (const void* p : {(const void*)idx, (const void*)pos, (const void*)src, (const void*)bounds})
    if (!is_aligned(p, 4)) return fail(SCADLES_EINVAL, "idx, pos, src or bounds is not 4-byte aligned");
  Chunks c;
  const bool one = N <= kSortChunk;
  const uint32_t rounds = one ? (uint32_t)div_up(N, kSortBlock) : sort_rounds(N);
  const uint32_t W = make_chunks(batch, k, one && rounds ? rounds : sort_rounds(N), c);
  const uint64_t need = one ? 0 : sort_bytes(W, experts + 1);
  if (!ws || !is_aligned(ws, 256)) return fail(SCADLES_EWORKSPACE, "workspace must be 256-byte aligned and not NULL");
  if (ws_bytes < need) return fail(SCADLES_EWORKSPACE, "workspace has %zu bytes, needs %zu", ws_bytes, (size_t)need);
  const void* at[5] = {pos, src, bounds, ws, idx};
  const uint64_t size[5] = {N * 4, N * 4, cells * 4, need, N * 4};
  for (int x = 0; x < 3; ++x)
    for (int y = x + 1; y < 5; ++y)
      if (bytes_overlap(at[x], size[x], at[y], size[y])) return fail(SCADLES_EINVAL, "an output overlaps an input, the workspace or another");
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (N == 0) {
    k_order_empty<<<(uint32_t)div_up(cells, kBlock), kBlock, 0, st>>>(bounds, (uint32_t)cells);
  } else if (one) {
    place<true>(rounds, 1, c, idx, experts, nullptr, nullptr, pos, src, bounds, st);
  } else {
    uint32_t* all = static_cast<uint32_t*>(ws);
    uint32_t* count = all + experts + 1;
    k_order_count<<<W, kSortBlock, 0, st>>>(c, idx, experts, count);
    launch_sort_scan(count, all, W, experts + 1, st);
    place<false>(rounds, W, c, idx, experts, count, all, pos, src, bounds, st);
  }
  return launch_status(hipGetLastError(), "order sort");
}

scadles_status scadles_dispatch(const scadles_order* order, const void* x, uint64_t ld_x, void* rows, uint64_t ld_rows, void* stream)
{
  if (scadles_status st = check_order(order)) return st;
  const uint64_t T = order->tokens;
  const Span in = {x, T, ld_x, "x"}, out = {rows, T * order->k, ld_rows, "rows"};
  for (const Span& s : {in, out})
    if (scadles_status st = check_span(order, s)) return st;
  if (spans_overlap(order, in, out) || overlaps(order, out, order->pos, T * order->k * 4)) return fail(SCADLES_EINVAL, "rows overlaps an input");
  if (!T) return SCADLES_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (order->type == SCADLES_BF16) dispatch<uint16_t>(order, x, ld_x, rows, ld_rows, st);
  else dispatch<float>(order, x, ld_x, rows, ld_rows, st);
  return launch_status(hipGetLastError(), "dispatch");
}

scadles_status scadles_combine(const scadles_order* order, const void* rows, uint64_t ld_rows, const float* gate, void* out, uint64_t ld_out,
                               void* stream)
{
  if (scadles_status st = check_order(order)) return st;
  const uint64_t T = order->tokens;
  const Span in = {rows, T * order->k, ld_rows, "rows"}, to = {out, T, ld_out, "out"};
  for (const Span& s : {in, to})
    if (scadles_status st = check_span(order, s)) return st;
  if (!is_aligned(gate, 4)) return fail(SCADLES_EINVAL, "gate is not 4-byte aligned");
  if (spans_overlap(order, in, to) || overlaps(order, to, order->pos, T * order->k * 4) || overlaps(order, to, gate, T * order->k * 4))
    return fail(SCADLES_EINVAL, "out overlaps an input");
  if (!T) return SCADLES_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (order->type == SCADLES_BF16) combine<uint16_t>(order, rows, ld_rows, gate, out, ld_out, st);
  else combine<float>(order, rows, ld_rows, gate, out, ld_out, st);
  return launch_status(hipGetLastError(), "combine");
}

scadles_status scadles_combine_backward(const scadles_order* order, const void* d_out, uint64_t ld_d_out, const void* rows, uint64_t ld_rows,
                                        const float* gate, void* d_rows, uint64_t ld_d_rows, float* d_gate, void* stream)
{
  if (scadles_status st = check_order(order)) return st;
  const uint64_t T = order->tokens, n = T * order->k;
  const Span up = {d_out, T, ld_d_out, "d_out"}, in = {rows, n, ld_rows, "rows"}, to = {d_rows, n, ld_d_rows, "d_rows"};
  for (const Span& s : {up, in})
    if (scadles_status st = check_span(order, s)) return st;
  if (d_rows) {
    if (scadles_status st = check_span(order, to)) return st;
    if ((spans_overlap(order, to, in) && (d_rows != rows || ld_d_rows != ld_rows)) || spans_overlap(order, to, up) ||
        overlaps(order, to, order->pos, n * 4) || overlaps(order, to, gate, n * 4) || overlaps(order, to, d_gate, n * 4))
      return fail(SCADLES_EINVAL, "d_rows overlaps an input or d_gate");
  }
  if (T && !gate) return fail(SCADLES_EINVAL, "gate is NULL");
  if (!is_aligned(gate, 4) || !is_aligned(d_gate, 4)) return fail(SCADLES_EINVAL, "gate or d_gate is not 4-byte aligned");
  if (overlaps(order, up, d_gate, n * 4) || overlaps(order, in, d_gate, n * 4) || bytes_overlap(d_gate, n * 4, order->pos, n * 4) ||
      bytes_overlap(d_gate, n * 4, gate, n * 4))
    return fail(SCADLES_EINVAL, "d_gate overlaps an input");
  if (!T || (!d_rows && !d_gate)) return SCADLES_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (order->type == SCADLES_BF16) combine_back<uint16_t>(order, d_out, ld_d_out, rows, ld_rows, gate, d_rows, ld_d_rows, d_gate, st);
  else combine_back<float>(order, d_out, ld_d_out, rows, ld_rows, gate, d_rows, ld_d_rows, d_gate, st);
  return launch_status(hipGetLastError(), "combine backward");
}

}  // extern "C"
