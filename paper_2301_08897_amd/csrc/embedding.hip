// embedding.hip -- rows of a table by token, times a scale, and the gradients of
// the table, one per device, by sorted tokens.
//
//   out[t] = scale weight[id_t]
//   d_weight[d][v] = scale sum over device d's tokens t of id v of d_out[t]
//
// The tokens are sorted by id, with sort.h's stable counting sort by digits of up
// to 10 bits; tokens of one id stay in their order, so those of one device follow
// each other and a run of equal (id, device), a cell, is one row of one gradient.
// k_embed_sum adds the rows of 32 sorted tokens at a time, a lane for each piece
// of 16 bytes, and writes the cells that lie within its 32; a cell that goes
// on beyond them leaves the parts in the workspace, which k_embed_join adds.
// The rows without a token are set to zero by further workgroups of the same
// launch, which search the sorted tokens for their ids. So every element of a
// gradient is written once, and nothing depends on the order of workgroups.
// Bound by memory: 131072 tokens of 1024 bfloat16 take 88 us to look up, 31 to sort (two passes of three
// launches), 146 to add into floats that are there and 29 to join; four tables of 50001 x 515 floats with
// 8190 tokens 91 us to write (4.7 TB/s), the sort 27. A sort's and a join's launches are bound by
// their few dependent loads each.
#include <cstring>

#include "pieces.h"
#include "sort.h"
#include "vec4.h"

using namespace scadles;

namespace {

constexpr uint32_t kRun = 32;                 // sorted tokens that a lane adds
constexpr uint32_t kSortOne = 4 * kSortBlock; // tokens of a sort in one launch
constexpr uint32_t kFillIds = 256;            // ids of a workgroup that writes zeros, at most
constexpr uint32_t kNone = ~0u;
constexpr int kJoinBlock = 1024;
constexpr uint32_t kJoins = 1u << 21;         // workgroups of a launch that joins

// Where ids come from: the caller's tokens, or an earlier pass.
struct Ids {
  const void* tokens;
  const uint32_t* id;         // of an earlier pass, or NULL
  const uint32_t* src;
  uint32_t wide, vocab;
};

// A token's id, `vocab` for padding.
__device__ inline uint32_t token_id(const Ids& a, uint64_t t)
{
  const uint64_t v = a.wide ? gptr((const uint64_t*)a.tokens)[t] : (uint64_t)(int64_t)gptr((const int32_t*)a.tokens)[t];
  return v < a.vocab ? (uint32_t)v : a.vocab;
}

__device__ inline uint32_t id_at(const Ids& a, uint64_t i) { return a.id ? gptr(a.id)[i] : token_id(a, i); }

// The devices' rows and gradients.
struct Grads {
  uint64_t off[kMaxK + 1];
  void* w[kMaxK];
  uint32_t K, vocab, dim;
  float scale;
};

__device__ inline uint32_t cell_of(const Grads& g, uint32_t id, uint32_t t)
{
  if (id == g.vocab) return kNone;
  uint32_t d = 0;
  while (d + 1 < g.K && g.off[d + 1] <= t) ++d;
  return d * g.vocab + id;
}

// ---- forward ------------------------------------------------------------------------------------

// kWhole: rows are whole pieces, and nothing is decided for the last one (131072 x 1024 bfloat16: 88
// us, else 96).
template <class X, bool kWhole>
__global__ __launch_bounds__(kBlock) void k_embed(Ids a, uint64_t tokens, Share share, uint32_t dim, float scale, const X* weight,
                                                  uint64_t ld_w, X* out, uint64_t ld_out)
{
  for_all_pieces(share, tokens, [&](uint64_t t, uint32_t g) {
    constexpr uint32_t N = Piece<X>::N;
    const uint32_t at = g * N, id = token_id(a, t);
    const X* row = weight + (uint64_t)id * ld_w;
    u4 v = {0, 0, 0, 0};
    if (id < a.vocab) v = pack<X>(unpack<X>(kWhole ? load_piece(row + at, 0, N) : load_piece(row, at, dim)) * scale);
    store_piece(out + t * ld_out + at, v, kWhole ? N : dim - at);
  });
}

// ---- tokens sorted by id ----------------------------------------------------------------------------

// Up to 4096 tokens in one workgroup, pass after pass in LDS.
template <int R>
__global__ __launch_bounds__(kSortBlock) void k_ids_one(Ids a, Grads g, uint32_t n, uint32_t passes, uint32_t bits, uint32_t* cell,
                                                        uint32_t* src)
{
  __shared__ SortLds s;
  __shared__ uint32_t id[R * kSortBlock];
  __shared__ uint16_t from[R * kSortBlock];
  for (uint32_t i = threadIdx.x; i < n; i += kSortBlock) {
    id[i] = token_id(a, i);
    from[i] = (uint16_t)i;
  }
  __syncthreads();
  for (uint32_t pass = 0; pass < passes; ++pass) {
    uint32_t key[R], rank[R], mine, last, mine_id[R], mine_from[R];
    rank_chunk<R>(s, n, 1u << bits, bits, [&](uint32_t i) { return id[i] >> pass * bits & ((1u << bits) - 1); }, key, rank, mine, last);
    first_of_all(s, mine);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const uint32_t i = ((threadIdx.x >> 6) * R + r) * 64 + (threadIdx.x & 63);
      if (key[r] == ~0u) continue;
      mine_id[r] = id[i];
      mine_from[r] = from[i];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (key[r] == ~0u) continue;
      const uint32_t p = s.first[key[r]] + s.count[threadIdx.x >> 6][key[r]] + rank[r];
      id[p] = mine_id[r];
      from[p] = (uint16_t)mine_from[r];
    }
    __syncthreads();
  }
  for (uint32_t i = threadIdx.x; i < n; i += kSortBlock) {
    gptr(cell)[i] = cell_of(g, id[i], from[i]);
    gptr(src)[i] = from[i];
  }
}

__global__ __launch_bounds__(kSortBlock) void k_ids_count(Ids a, uint64_t n, uint32_t per, uint32_t shift, uint32_t bits, uint32_t* count)
{
  __shared__ uint32_t lds[kSortDigits + 1];
  const uint64_t at = (uint64_t)blockIdx.x * per, left = n - at;
  count_chunk(lds, left < per ? (uint32_t)left : per, 1u << bits, [&](uint32_t i) { return id_at(a, at + i) >> shift & ((1u << bits) - 1); },
              count + ((uint64_t)blockIdx.x << bits));
}

// One pass; the last one gives the cells in place of the ids.
template <int R>
__global__ __launch_bounds__(kSortBlock) void k_ids_place(Ids a, Grads g, uint64_t n, uint32_t shift, uint32_t bits, const uint32_t* before,
                                                          const uint32_t* all, uint32_t* id, uint32_t* src, uint32_t is_last)
{
  __shared__ SortLds s;
  const uint32_t per = R * kSortBlock;
  const uint64_t at = (uint64_t)blockIdx.x * per, left = n - at;
  uint32_t key[R], rank[R], mine, last;
  rank_chunk<R>(s, left < per ? (uint32_t)left : per, 1u << bits, bits,
                [&](uint32_t i) { return id_at(a, at + i) >> shift & ((1u << bits) - 1); }, key, rank, mine, last);
  first_of_chunk(s, before, all, 1u << bits, blockIdx.x);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (key[r] == ~0u) continue;
    const uint64_t i = at + ((threadIdx.x >> 6) * R + r) * 64 + (threadIdx.x & 63);
    const uint32_t p = s.first[key[r]] + s.count[threadIdx.x >> 6][key[r]] + rank[r];
    const uint32_t v = id_at(a, i), t = a.id ? gptr(a.src)[i] : (uint32_t)i;
    gptr(id)[p] = is_last ? cell_of(g, v, t) : v;
    gptr(src)[p] = t;
  }
}

// ---- sums -----------------------------------------------------------------------------------------------

// N sums into a row of a gradient at element `at`, `left` of them.
template <class X, class W>
__device__ inline void write_grad(W* row, uint32_t left, typename Piece<X>::F sum, bool add)
{
#pragma unroll
  for (uint32_t q = 0; q < Piece<X>::N; q += 4) {
    if (q >= left) break;
    f4 x = {sum[q], sum[q + 1], sum[q + 2], sum[q + 3]};
    if (add) x += load_f4(row + q, left - q);
    store_f4(row + q, x, left - q);
  }
}

// What the launch of the sums does: workgroups [0, sums) add, `chunks` of them beside
// each other in lanes of `lanes`; the rest write zeros, `per` ids of a device each.
struct Sums {
  uint32_t n, sums, lanes, columns, chunks;      // chunks: groups of kRun sorted tokens
  uint32_t per, device_groups, magic;            // magic: x * magic >> 32 is x / dim for x < per * dim
};

template <class W>
__device__ inline void fill_rows(const Grads& g, const Sums& m, uint32_t b, const uint32_t* cell, uint8_t* hit, uint32_t* range)
{
  const uint32_t d = b / m.device_groups, a = (b - d * m.device_groups) * m.per;
  const uint32_t ids = g.vocab - a < m.per ? g.vocab - a : m.per;
  if (threadIdx.x < m.per) hit[threadIdx.x] = 0;
  if (threadIdx.x < 128) {                      // the sorted tokens of these ids: a wave for each end
    const uint32_t want = a + (threadIdx.x < 64 ? 0 : ids), lane = threadIdx.x & 63;
    uint32_t lo = 0, hi = m.n;                  // 64 places of the range are looked at at once
    while (lo < hi) {
      const uint32_t step = (hi - lo + 63) / 64, at = lo + lane * step;
      const uint32_t c = at < hi ? gptr(cell)[at] : kNone;
      const uint32_t below = (uint32_t)__popcll(__ballot(c != kNone && c % g.vocab < want));
      if (below == 0) break;                    // lo itself is not below
      const uint32_t last = lo + (below - 1) * step;
      hi = last + step < hi ? last + step : hi;
      lo = last + 1;
    }
    if (lane == 0) range[threadIdx.x >> 6] = lo;
  }
  __syncthreads();
  for (uint32_t i = range[0] + threadIdx.x; i < range[1]; i += kBlock) {
    const uint32_t c = gptr(cell)[i];
    if (c / g.vocab == d) hit[c % g.vocab - a] = 1;
  }
  __syncthreads();
  // the rows follow each other: aligned words of 16 bytes where both their ends lie in rows
  // without a token, single elements elsewhere
  constexpr uint32_t N = 16 / sizeof(W);
  W* w = (W*)g.w[d] + (uint64_t)a * g.dim;
  const uint32_t n = ids * g.dim, skip = (uint32_t)((16 - (uintptr_t)w % 16) % 16 / sizeof(W));
  auto row = [&](uint32_t i) { return m.per == 1 ? 0u : g.dim == 1 ? i : __umulhi(i, m.magic); };
  for (uint32_t i = threadIdx.x; i <= (n + N - 1) / N; i += kBlock) {
    // word i begins N elements before the next; the first one may begin before the rows
    const int32_t lo = (int32_t)(i * N) + (int32_t)skip - (int32_t)N;
    if (lo >= 0 && lo + N <= n && !hit[row(lo)] && !hit[row(lo + N - 1)] && row(lo + N - 1) - row(lo) <= 1) {
      *(GLOBAL u4*)gptr(w + lo) = u4{0, 0, 0, 0};
      continue;
    }
    for (uint32_t e = 0; e < N; ++e) {
      const int32_t at = lo + (int32_t)e;
      if (at >= 0 && (uint32_t)at < n && !hit[row(at)]) gptr(w)[at] = 0;
    }
  }
}

template <class X, class W, bool kAdd>
__global__ __launch_bounds__(kBlock) void k_embed_sum(Grads g, Sums m, const uint32_t* cell, const uint32_t* src, const X* d_out, uint64_t ld,
                                                      float* part, uint32_t width)
{
  typedef typename Piece<X>::F F;
  if constexpr (!kAdd) {
    __shared__ uint8_t hit[kFillIds];
    __shared__ uint32_t range[2];
    if (blockIdx.x >= m.sums) {
      for (uint32_t b = blockIdx.x - m.sums; b < m.device_groups * g.K; b += gridDim.x - m.sums) {
        fill_rows<W>(g, m, b, cell, hit, range);
        __syncthreads();
      }
      return;
    }
  }
  const uint32_t column = blockIdx.x % m.columns, chunk = blockIdx.x / m.columns * (kBlock / m.lanes) + threadIdx.x / m.lanes;
  const uint32_t at = (column * m.lanes + threadIdx.x % m.lanes) * Piece<X>::N;
  if (chunk >= m.chunks || at >= g.dim) return;
  const uint32_t left = g.dim - at, i0 = chunk * kRun, i1 = i0 + kRun < m.n ? i0 + kRun : m.n;
  uint32_t now = gptr(cell)[i0];
  bool before = i0 && gptr(cell)[i0 - 1] == now;
  F sum = {};
  auto done = [&](bool after) {
    if (now == kNone) return;
    if (before || after) {
      float* p = part + ((uint64_t)chunk * 2 + (before ? 0 : 1)) * width + at;
#pragma unroll
      for (uint32_t q = 0; q < Piece<X>::N; q += 4) *(GLOBAL f4*)gptr(p + q) = f4{sum[q], sum[q + 1], sum[q + 2], sum[q + 3]};
    } else {
      const uint32_t d = now / g.vocab;
      write_grad<X>((W*)g.w[d] + (uint64_t)(now - d * g.vocab) * g.dim + at, left, sum * g.scale, kAdd);
    }
  };
  for (uint32_t i = i0; i < i1; i += 8) {
    uint32_t c[8];
    u4 v[8];
#pragma unroll
    for (uint32_t q = 0; q < 8; ++q) {
      c[q] = i + q < i1 ? gptr(cell)[i + q] : kNone;
      // padding's rows are read too, so that no load waits for another's branch
      v[q] = load_raw(d_out + (uint64_t)(i + q < i1 ? gptr(src)[i + q] : 0) * ld, at, g.dim);
    }
#pragma unroll
    for (uint32_t q = 0; q < 8; ++q) {
      if (i + q >= i1) break;
      if (c[q] != now) {
        done(false);
        now = c[q];
        before = false;
        sum = F{};
      }
      if (c[q] != kNone) sum += unpack<X>(settled<X>(v[q], at, g.dim));
    }
  }
  done(i1 < m.n && gptr(cell)[i1] == now);
}

// The cells that begin in a chunk of sorted tokens and go on behind it. The workgroup's
// lanes share the columns, and the chunks of a long cell in slices.
template <class X, class W, bool kAdd>
__global__ __launch_bounds__(kJoinBlock) void k_embed_join(Grads g, Sums m, uint32_t block, const uint32_t* cell, const float* part, uint32_t width)
{
  typedef typename Piece<X>::F F;
  __shared__ F slice[kJoinBlock];
  block += blockIdx.x;
  const uint32_t column = block % m.columns, chunk = block / m.columns;
  const uint32_t first = (chunk + 1) * kRun;             // of the next chunk; the last chunk has no workgroup here
  const uint32_t now = gptr(cell)[first];
  if (now == kNone || gptr(cell)[first - 1] != now) return;
  if (gptr(cell)[chunk * kRun] == now && chunk && gptr(cell)[chunk * kRun - 1] == now) return;   // began before
  uint32_t lo = chunk + 1, hi = m.chunks;                // chunks [chunk + 1, hi) begin with it
  while (lo < hi) {
    const uint32_t mid = (lo + hi) / 2;
    if (gptr(cell)[mid * kRun] == now) lo = mid + 1;
    else hi = mid;
  }
  const uint32_t lane = threadIdx.x % m.lanes, s = threadIdx.x / m.lanes, slices = kJoinBlock / m.lanes;
  const uint32_t at = (column * m.lanes + lane) * Piece<X>::N;
  F sum = {};
  if (at < g.dim) {
#pragma unroll 4
    for (uint32_t j = chunk + s; j < hi; j += slices) {
      const float* p = part + ((uint64_t)j * 2 + (j == chunk ? 1 : 0)) * width + at;
#pragma unroll
      for (uint32_t q = 0; q < Piece<X>::N; q += 4) {
        const f4 x = *(const GLOBAL f4*)gptr(p + q);
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) sum[q + e] += x[e];
      }
    }
  }
  slice[threadIdx.x] = sum;
  __syncthreads();
  if (s || at >= g.dim) return;
  for (uint32_t q = 1; q < slices; ++q) sum += slice[q * m.lanes + lane];
  const uint32_t d = now / g.vocab;
  write_grad<X>((W*)g.w[d] + (uint64_t)(now - d * g.vocab) * g.dim + at, g.dim - at, sum * g.scale, kAdd);
}

// ---- host -------------------------------------------------------------------------------------------------

// The workspace's pieces.
struct Space {
  uint32_t *cell, *src, *id, *id_src, *count, *all;
  float* part;
};

uint32_t passes_of(uint64_t vocab, uint32_t& bits)
{
  uint32_t total = 0;
  while (total < 32 && (1ull << total) < vocab + 1) ++total;   // padding is id `vocab`
  const uint32_t passes = (uint32_t)div_up(total, 10);
  bits = (uint32_t)div_up(total, passes);
  return passes;
}

uint32_t width_of(uint32_t dim) { return (uint32_t)div_up(dim, 8) * 8; }

uint64_t lay_out(uint64_t n, uint64_t vocab, uint32_t dim, char* ws, Space& s)
{
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) {
    const uint64_t here = at;
    at = div_up(at + bytes, 256) * 256;
    return ws + here;
  };
  uint32_t bits;
  passes_of(vocab, bits);
  s.cell = (uint32_t*)take(n * 4);
  s.src = (uint32_t*)take(n * 4);
  s.id = s.id_src = s.count = s.all = nullptr;
  if (n > kSortOne) {
    const uint64_t W = sort_chunks(n);
    s.id = (uint32_t*)take(n * 4);
    s.id_src = (uint32_t*)take(n * 4);
    s.all = (uint32_t*)take(4ull << bits);
    s.count = (uint32_t*)take((W * 4) << bits);
  }
  s.part = (float*)take(div_up(n, kRun) * 2 * width_of(dim) * 4);
  return at;
}

scadles_status check_embedding(const scadles_embedding* e, uint32_t devices)
{
  if (!e) return fail(SCADLES_EINVAL, "embedding is NULL");
  if (!e->vocab || e->vocab >= 0xFFFFFFFFull || e->vocab * devices >= 0xFFFFFFFFull)
    return fail(SCADLES_EINVAL, "vocab = %llu is 0, or 2^32 - 1 or more over all devices", (unsigned long long)e->vocab);
  if (!e->dim || e->dim >= 1u << 24) return fail(SCADLES_EINVAL, "dim = %u is outside [1, 2^24)", e->dim);
  if ((e->type != SCADLES_F32 && e->type != SCADLES_BF16) || (e->grad_type != SCADLES_F32 && e->grad_type != SCADLES_BF16))
    return fail(SCADLES_EINVAL, "unknown type %d or grad_type %d", e->type, e->grad_type);
  if (e->token_bytes != 4 && e->token_bytes != 8) return fail(SCADLES_EINVAL, "token_bytes must be 4 or 8");
  if (!(e->scale - e->scale == 0.0f)) return fail(SCADLES_EINVAL, "scale is not finite");
  return SCADLES_OK;
}

uint64_t size_of(int32_t type) { return type == SCADLES_BF16 ? 2 : 4; }

template <class X>
hipError_t forward(const scadles_embedding* e, uint64_t tokens, const void* ids, const void* weight, uint64_t ld_w, void* out, uint64_t ld_out,
                   hipStream_t st)
{
  const Ids a = {ids, nullptr, nullptr, e->token_bytes == 8, (uint32_t)e->vocab};
  const Share share = share_rows(tokens, div_up(e->dim, Piece<X>::N));
  auto go = [&](auto kernel) {
    kernel<<<grid_of(div_up(tokens, share.rows)), kBlock, 0, st>>>(a, tokens, share, e->dim, e->scale, (const X*)weight, ld_w, (X*)out, ld_out);
  };
  if (e->dim % Piece<X>::N) go(k_embed<X, false>);
  else go(k_embed<X, true>);
  return hipGetLastError();
}

void sort_ids(const scadles_embedding* e, const Grads& g, const void* tokens, uint64_t n, const Space& s, hipStream_t st)
{
  uint32_t bits;
  const uint32_t passes = passes_of(e->vocab, bits);
  Ids a = {tokens, nullptr, nullptr, e->token_bytes == 8, (uint32_t)e->vocab};
  if (n <= kSortOne) {
    const uint32_t N = (uint32_t)n;
    if (n <= kSortBlock) k_ids_one<1><<<1, kSortBlock, 0, st>>>(a, g, N, passes, bits, s.cell, s.src);
    else if (n <= 2 * kSortBlock) k_ids_one<2><<<1, kSortBlock, 0, st>>>(a, g, N, passes, bits, s.cell, s.src);
    else k_ids_one<4><<<1, kSortBlock, 0, st>>>(a, g, N, passes, bits, s.cell, s.src);
    return;
  }
  const uint32_t R = sort_rounds(n), W = (uint32_t)div_up(n, (uint64_t)R * kSortBlock);
  for (uint32_t p = 0; p < passes; ++p) {
    // passes write to the two pairs in turn, the last one to cell and src
    const bool here = (passes - p) % 2 == 1;
    uint32_t *id = here ? s.cell : s.id, *src = here ? s.src : s.id_src;
    k_ids_count<<<W, kSortBlock, 0, st>>>(a, n, R * kSortBlock, p * bits, bits, s.count);
    launch_sort_scan(s.count, s.all, W, 1u << bits, st);
    const uint32_t last = p + 1 == passes;
    if (R == 1) k_ids_place<1><<<W, kSortBlock, 0, st>>>(a, g, n, p * bits, bits, s.count, s.all, id, src, last);
    else if (R == 2) k_ids_place<2><<<W, kSortBlock, 0, st>>>(a, g, n, p * bits, bits, s.count, s.all, id, src, last);
    else if (R == 4) k_ids_place<4><<<W, kSortBlock, 0, st>>>(a, g, n, p * bits, bits, s.count, s.all, id, src, last);
    else k_ids_place<8><<<W, kSortBlock, 0, st>>>(a, g, n, p * bits, bits, s.count, s.all, id, src, last);
    a.id = id;
    a.src = src;
  }
}

template <class X, class W>
hipError_t sums(const Grads& g, uint64_t n, const Space& s, const void* d_out, uint64_t ld, int accumulate, hipStream_t st)
{
  Sums m;
  std::memset(&m, 0, sizeof(m));
  const uint32_t pieces = (uint32_t)div_up(g.dim, Piece<X>::N);
  m.n = (uint32_t)n;
  m.lanes = 8;
  while (m.lanes < kBlock && m.lanes < pieces) m.lanes *= 2;
  m.columns = (uint32_t)div_up(pieces, m.lanes);
  m.chunks = (uint32_t)div_up(n, kRun);
  m.sums = (uint32_t)div_up(m.chunks, kBlock / m.lanes) * m.columns;
  uint64_t fills = 0;
  if (!accumulate) {
    // 64 KiB of rows to a workgroup, and 8 KiB for a few tokens, whose search is short: those under
    // way then write next to each other (65536 x 1024 floats, 100 tokens: 61 us a call; 64 KiB: 76. Four
    // tables of 50001 x 515 floats, 8190 tokens: 91 us, 16 KiB: 99, 8 KiB: 148)
    const uint64_t row = (uint64_t)g.dim * sizeof(W);
    uint64_t per = (n <= 4096 ? 8u << 10 : 64u << 10) / row;
    per = per < 1 ? 1 : per > kFillIds ? kFillIds : per;
    if (per > g.vocab) per = g.vocab;
    m.per = (uint32_t)per;
    m.device_groups = (uint32_t)div_up(g.vocab, per);
    m.magic = (uint32_t)(g.dim == 1 ? 0 : div_up(1ull << 32, g.dim));
    fills = grid_of((uint64_t)m.device_groups * g.K);
  }
  const uint32_t width = width_of(g.dim);
  if (m.sums > kMostBlocks) return hipErrorInvalidValue;      // more than 2^19 MB of rows
  if (m.sums + fills) {
    const uint32_t blocks = (uint32_t)(m.sums + fills);
    if (accumulate) k_embed_sum<X, W, true><<<blocks, kBlock, 0, st>>>(g, m, s.cell, s.src, (const X*)d_out, ld, s.part, width);
    else k_embed_sum<X, W, false><<<blocks, kBlock, 0, st>>>(g, m, s.cell, s.src, (const X*)d_out, ld, s.part, width);
  }
  const uint64_t joins = (uint64_t)(m.chunks ? m.chunks - 1 : 0) * m.columns;
  for (uint64_t at = 0; at < joins; at += kJoins) {
    const uint32_t blocks = (uint32_t)(joins - at < kJoins ? joins - at : kJoins), b = (uint32_t)at;
    if (accumulate) k_embed_join<X, W, true><<<blocks, kJoinBlock, 0, st>>>(g, m, b, s.cell, s.part, width);
    else k_embed_join<X, W, false><<<blocks, kJoinBlock, 0, st>>>(g, m, b, s.cell, s.part, width);
  }
  return hipGetLastError();
}

}  // namespace

extern "C" {

scadles_status scadles_embedding_forward(const scadles_embedding* e, uint64_t tokens, const void* ids, const void* weight, uint64_t ld_weight,
                                         void* out, uint64_t ld_out, void* stream)
{
  if (scadles_status st = check_embedding(e, 1)) return st;
  if (tokens > 0x7FFFFFFFull) return fail(SCADLES_EINVAL, "more than 2^31 - 1 tokens");
  if (!weight || (tokens && (!ids || !out))) return fail(SCADLES_EINVAL, "ids, weight and out must not be NULL");
  const uint64_t es = size_of(e->type);
  if (!is_aligned(ids, e->token_bytes) || !is_aligned(weight, es) || !is_aligned(out, es))
    return fail(SCADLES_EINVAL, "ids, weight or out is not aligned to its elements");
  if (ld_weight < e->dim || ld_out < e->dim || ld_weight >= 1ull << 31 || ld_out >= 1ull << 31)
    return fail(SCADLES_EINVAL, "ld_weight or ld_out is smaller than dim, or 2^31 or more");
  const uint64_t bytes = rows_bytes(tokens, e->dim, ld_out, es);
  if (bytes_overlap(out, bytes, weight, rows_bytes(e->vocab, e->dim, ld_weight, es)) || bytes_overlap(out, bytes, ids, tokens * e->token_bytes))
    return fail(SCADLES_EINVAL, "out overlaps an input");
  if (!tokens) return SCADLES_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  return launch_status(e->type == SCADLES_BF16 ? forward<uint16_t>(e, tokens, ids, weight, ld_weight, out, ld_out, st)
                                               : forward<float>(e, tokens, ids, weight, ld_weight, out, ld_out, st),
                       "embedding forward");
}

size_t scadles_embedding_workspace_bytes(uint64_t tokens, uint64_t vocab, uint32_t dim)
{
  if (tokens > 0x7FFFFFFFull || !vocab || vocab >= 0xFFFFFFFFull || !dim || dim >= 1u << 24) return 0;
  Space s;
  const uint64_t n = lay_out(tokens, vocab, dim, nullptr, s);
  return (size_t)(n < 256 ? 256 : n);
}

scadles_status scadles_embedding_backward(const scadles_embedding* e, const scadles_batch* batch, const void* ids, const void* d_out,
                                          uint64_t ld_d_out, void* const* d_weight, int accumulate, void* ws, size_t ws_bytes, void* stream)
{
  if (scadles_status st = check_batch(batch)) return st;
  if (scadles_status st = check_embedding(e, batch->devices)) return st;
  const uint64_t n = batch->tokens, es = size_of(e->type), gs = size_of(e->grad_type);
  if (n && (!ids || !d_out)) return fail(SCADLES_EINVAL, "ids and d_out must not be NULL");
  if (!is_aligned(ids, e->token_bytes) || !is_aligned(d_out, es)) return fail(SCADLES_EINVAL, "ids or d_out is not aligned to its elements");
  if (ld_d_out < e->dim || ld_d_out >= 1ull << 31) return fail(SCADLES_EINVAL, "ld_d_out is smaller than dim, or 2^31 or more");
  if (!d_weight) return fail(SCADLES_EINVAL, "d_weight is NULL");
  Space s;
  const uint64_t need = lay_out(n, e->vocab, e->dim, static_cast<char*>(ws), s);
  if (!ws || !is_aligned(ws, 256)) return fail(SCADLES_EWORKSPACE, "workspace must be 256-byte aligned and not NULL");
  if (ws_bytes < need) return fail(SCADLES_EWORKSPACE, "workspace has %zu bytes, needs %zu", ws_bytes, (size_t)need);
  Grads g;
  std::memset(&g, 0, sizeof(g));
  const uint64_t bytes = e->vocab * e->dim * gs;
  for (uint32_t d = 0; d < batch->devices; ++d) {
    const void* w = d_weight[d];
    if (!w || !is_aligned(w, gs)) return fail(SCADLES_EINVAL, "gradient %u is NULL or not aligned to its elements", d);
    if (bytes_overlap(w, bytes, ids, n * e->token_bytes) || bytes_overlap(w, bytes, d_out, rows_bytes(n, e->dim, ld_d_out, es)) ||
        bytes_overlap(w, bytes, ws, need))
      return fail(SCADLES_EINVAL, "gradient %u overlaps an input or the workspace", d);
    for (uint32_t c = 0; c < d; ++c)
      if (bytes_overlap(w, bytes, d_weight[c], bytes)) return fail(SCADLES_EINVAL, "gradients %u and %u overlap", c, d);
    g.w[d] = d_weight[d];
    g.off[d] = batch->tok_off[d];
  }
  if (bytes_overlap(ws, need, ids, n * e->token_bytes) || bytes_overlap(ws, need, d_out, rows_bytes(n, e->dim, ld_d_out, es)))
    return fail(SCADLES_EINVAL, "the workspace overlaps an input");
  g.K = batch->devices;
  g.off[g.K] = n;
  g.vocab = (uint32_t)e->vocab;
  g.dim = e->dim;
  g.scale = e->scale;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (n) sort_ids(e, g, ids, n, s, st);
  const bool b = e->type == SCADLES_BF16, gb = e->grad_type == SCADLES_BF16;
  const hipError_t err = b ? (gb ? sums<uint16_t, uint16_t>(g, n, s, d_out, ld_d_out, accumulate, st)
                                 : sums<uint16_t, float>(g, n, s, d_out, ld_d_out, accumulate, st))
                           : (gb ? sums<float, uint16_t>(g, n, s, d_out, ld_d_out, accumulate, st)
                                 : sums<float, float>(g, n, s, d_out, ld_d_out, accumulate, st));
  return launch_status(err, "embedding backward");
}

}  // extern "C"
