// Embedding: rows of a table, scaled, and the table's gradient.
//
//   out[i] = s table[id_i],   grad_table[v] = s sum over {i : id_i = v} of grad_out[i]
//
// The gradient adds each row's positions in an order that the ids alone fix: positions
// are sorted by id (a stable radix sort of up to 9 bits a pass), every wave sums the
// runs of equal ids among 16 or 32 sorted positions, whatever their rows, and the sums of
// ids that go on past a wave's positions are joined by a second kernel.  The sums of a
// frequent token are so spread over the chip; its join (one block for 256 to 512 values of
// the row, a term for every 16 or 32 positions) and the block that clears its neighbours (it
// reads their ids once) still grow with its count.  Rows that no token names are cleared beside
// the sums.  Both directions are bound by memory: the gradient writes all V rows.
//
// 32768 tokens (frequencies 1 / rank) in 50001 rows of 1024 in bf16: lookup 21 us (67 MB
// written), sort 2 x (3 + 6) us, sums and clearing 30 us (67 MB read from cache, 102 MB
// written), join 7 us; 86 us with the launches' gaps.  With a block a row of the table,
// whatever its count, the sums alone took 342 us (the first token has 2700 positions).
#include "seq_common.h"

namespace dendsn_seq {
namespace {

constexpr int kThreads = 256;
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kBits = 9, kRadix = 1 << kBits;  // most bits of a pass
constexpr int kMaxTiles = 512;                 // sorting blocks, at most
constexpr int kOneBlock = 1024;                // positions that one block sorts alone (7 us, in two launches
                                               // 4 + 4; 2048: 12, 4.7 + 5)
constexpr int kCountAll = 4096;                // positions that every sorting block counts for itself (a pass
                                               // 5.8 us, with a launch that counts 2.4 + 4.8; 8192: 8.6, 3 + 5.7)
constexpr int kRows = 32;                      // table rows of a clearing block

template <typename ID>
__device__ __forceinline__ uint32_t key_of(const ID* ids, int64_t i, uint32_t V) {
  const int64_t id = int64_t(ids[i]);
  return id >= 0 && id < int64_t(V) ? uint32_t(id) : V;  // V: no row
}

// A wave a row: 64 lanes over its values, VEC a lane.  Bound by the rows' bytes, 64 rows by
// the launch (2.7 us).
template <typename IO, typename ID, int VEC>
__global__ void __launch_bounds__(kThreads) embed_fwd_kernel(const ID* ids, const IO* table, IO* out, int64_t n,
                                                             uint32_t V, int64_t D, int64_t ldt, int64_t ldo,
                                                             float scale) {
  const int lane = threadIdx.x & 63;
  const int64_t i = int64_t(blockIdx.x) * (kThreads / 64) + (threadIdx.x >> 6);
  if (i >= n) return;
  const uint32_t key = __builtin_amdgcn_readfirstlane(key_of(ids, i, V));
  const IO* row = table + int64_t(key) * ldt;
  IO* to = out + i * ldo;
  for (int64_t d0 = lane * VEC; d0 < D; d0 += 64 * VEC) {
    const int64_t d = min(d0, D - VEC);  // (a row's last lane shares values with the one before)
    Pack<IO, VEC> v;
    if (key < V) {
      v = *reinterpret_cast<const Pack<IO, VEC>*>(row + d);
#pragma unroll
      for (int k = 0; k < VEC; ++k) v.v[k] = narrow<IO>(scale * widen(v.v[k]));
    } else {
#pragma unroll
      for (int k = 0; k < VEC; ++k) v.v[k] = narrow<IO>(0.0f);
    }
    *reinterpret_cast<Pack<IO, VEC>*>(to + d) = v;
  }
}

// ---------------------------------------------------------------------------
// Sort
// ---------------------------------------------------------------------------
struct SortArgs {
  const void* ids;              // first pass
  const uint32_t *key_in, *at_in;
  uint32_t *key_out, *at_out;
  uint32_t* hist;               // [tiles][kRadix]
  int64_t n, tile;              // tile: positions of a block, a multiple of kSortThreads
  uint32_t V, ntiles;
  int shift, bits, passes;
};

template <typename ID, bool FIRST>
__device__ __forceinline__ uint32_t sort_key(const SortArgs& p, int64_t i) {
  return FIRST ? key_of(static_cast<const ID*>(p.ids), i, p.V) : p.key_in[i];
}

// A pass's counts of each tile.  (Counted by the pass before as it places the keys,
// with global atomics, frequent ids made that pass 11 us slower; this launch is 3 us.)
template <typename ID, bool FIRST>
__global__ void __launch_bounds__(kSortThreads) embed_hist_kernel(SortArgs p) {
  __shared__ uint32_t h[kRadix];
  const int tid = threadIdx.x;
  if (tid < kRadix) h[tid] = 0;
  __syncthreads();
  const int64_t lo = blockIdx.x * p.tile, hi = min(lo + p.tile, p.n);
  const uint32_t mask = (1u << p.bits) - 1;
  for (int64_t i = lo + tid; i < hi; i += kSortThreads) atomicAdd(&h[(sort_key<ID, FIRST>(p, i) >> p.shift) & mask], 1u);
  __syncthreads();
  if (tid < kRadix) p.hist[int64_t(blockIdx.x) * kRadix + tid] = h[tid];
}

struct SortShared {
  uint32_t base[kRadix], count[kSortWaves][kRadix], sums[kRadix / 64], part[4][2][kRadix];
};

// base[d] = positions before this tile's first of digit d, from the digits' totals and
// their counts in the tiles before.  total, before: of digit tid < kRadix.
__device__ __forceinline__ void sort_bases(SortShared& s, uint32_t total, uint32_t before) {
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  uint32_t sum = total;  // of the wave's digits up to this one
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t add = __shfl_up(sum, d);
    if (lane >= d) sum += add;
  }
  if (lane == 63 && w < kRadix / 64) s.sums[w] = sum;
  __syncthreads();
  if (tid < kRadix) {
#pragma unroll
    for (int q = 0; q < kRadix / 64; ++q)
      if (q < w) sum += s.sums[q];
    s.base[tid] = sum - total + before;
  }
}

// Moves the positions [lo, hi) to their places, in their order.
template <typename ID, bool FIRST>
__device__ __forceinline__ void sort_move(const SortArgs& p, SortShared& s, int64_t lo, int64_t hi) {
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const uint32_t mask = (1u << p.bits) - 1;
  for (int64_t i0 = lo; i0 < hi; i0 += kSortThreads) {
    for (int d = tid; d < kSortWaves * kRadix; d += kSortThreads) (&s.count[0][0])[d] = 0;
    __syncthreads();
    const int64_t i = i0 + tid;
    const bool in = i < hi;
    const uint32_t key = in ? sort_key<ID, FIRST>(p, i) : 0;
    const uint32_t at = in ? (FIRST ? uint32_t(i) : p.at_in[i]) : 0;
    const uint32_t digit = (key >> p.shift) & mask;
    uint64_t same = __ballot(in);
    for (int b = 0; b < p.bits; ++b) {
      const bool set = (digit >> b) & 1;
      const uint64_t votes = __ballot(set);
      same &= set ? votes : ~votes;
    }
    const uint32_t rank = __popcll(same & ((uint64_t(1) << lane) - 1));
    if (in && rank == 0) s.count[w][digit] = __popcll(same);
    __syncthreads();
    if (tid < kRadix) {  // a digit's counts become the places of the waves' first
      uint32_t sum = s.base[tid];
#pragma unroll
      for (int q = 0; q < kSortWaves; ++q) {
        const uint32_t c = s.count[q][tid];
        s.count[q][tid] = sum;
        sum += c;
      }
      s.base[tid] = sum;
    }
    __syncthreads();
    if (in) {
      const uint32_t to = s.count[w][digit] + rank;
      p.key_out[to] = key;
      p.at_out[to] = at;
    }
    __syncthreads();
  }
}

// A block a tile: bases from all tiles' counts, then the tile's positions moved in order.
// Bound by latency (6 us for 32 tiles of 1024): counts, ranks and stores follow each other.
// COUNTED: embed_hist_kernel has counted the tiles; else each block counts all positions.
template <typename ID, bool FIRST, bool COUNTED>
__global__ void __launch_bounds__(kSortThreads) embed_scatter_kernel(SortArgs p) {
  __shared__ SortShared s;
  const int tid = threadIdx.x;
  const int64_t lo = blockIdx.x * p.tile;
  uint32_t tt = 0, bb = 0;
  if (COUNTED) {
    const int q = tid >> 8, d = (tid & 255) * 2;
    uint2 total = make_uint2(0, 0), before = make_uint2(0, 0);
#pragma unroll 8
    for (uint32_t t = q; t < p.ntiles; t += 4) {
      const uint2 c = *reinterpret_cast<const uint2*>(p.hist + int64_t(t) * kRadix + d);
      total.x += c.x, total.y += c.y;
      if (t < blockIdx.x) before.x += c.x, before.y += c.y;
    }
    *reinterpret_cast<uint2*>(&s.part[q][0][d]) = total;
    *reinterpret_cast<uint2*>(&s.part[q][1][d]) = before;
    __syncthreads();
    if (tid < kRadix) {
#pragma unroll
      for (int k = 0; k < 4; ++k) tt += s.part[k][0][tid], bb += s.part[k][1][tid];
    }
  } else {
    if (tid < kRadix) s.part[0][0][tid] = s.part[0][1][tid] = 0;
    __syncthreads();
    const uint32_t mask = (1u << p.bits) - 1;
#pragma unroll 8
    for (int64_t i = tid; i < p.n; i += kSortThreads)
      atomicAdd(&s.part[0][i < lo][(sort_key<ID, FIRST>(p, i) >> p.shift) & mask], 1u);
    __syncthreads();
    if (tid < kRadix) bb = s.part[0][1][tid], tt = s.part[0][0][tid] + bb;
  }
  sort_bases(s, tt, bb);
  sort_move<ID, FIRST>(p, s, lo, min(lo + p.tile, p.n));
}

// Few positions: one block makes all passes.  buf: the two buffers in turn.
template <typename ID>
__global__ void __launch_bounds__(kSortThreads) embed_sort_kernel(SortArgs p, uint32_t* key0, uint32_t* at0,
                                                                  uint32_t* key1, uint32_t* at1) {
  __shared__ SortShared s;
  const int tid = threadIdx.x;
  const uint32_t mask = (1u << p.bits) - 1;
  for (int k = 0; k < p.passes; ++k) {
    p.shift = k * p.bits;
    p.key_in = k & 1 ? key1 : key0;
    p.at_in = k & 1 ? at1 : at0;
    p.key_out = k & 1 ? key0 : key1;
    p.at_out = k & 1 ? at0 : at1;
    __syncthreads();  // the last pass's places are written (a block's barrier orders its memory)
    if (tid < kRadix) s.part[0][0][tid] = 0;
    __syncthreads();
    for (int64_t i = tid; i < p.n; i += kSortThreads) {
      const uint32_t key = k ? sort_key<ID, false>(p, i) : sort_key<ID, true>(p, i);
      atomicAdd(&s.part[0][0][(key >> p.shift) & mask], 1u);
    }
    __syncthreads();
    sort_bases(s, tid < kRadix ? s.part[0][0][tid] : 0, 0);
    if (k) sort_move<ID, false>(p, s, 0, p.n);
    else sort_move<ID, true>(p, s, 0, p.n);
  }
}

// ---------------------------------------------------------------------------
// Sums
// ---------------------------------------------------------------------------
struct SumArgs {
  const uint32_t *key, *at;  // sorted
  const void* grad;
  void* table;
  float* part;               // [runs][2][D]: sums of the ids that a run begins and ends in the middle of
  int64_t n, D, ldg, ldt;
  int64_t runs, sum_blocks;
  int chunks;                // waves along a row
  int log_run;               // of the sorted positions of a wave
  uint32_t V;
  float scale;
};

// First sorted position in [lo, lo + len) whose key is at least `key` (lo + len: none), by
// one wave: 64 candidates a step.
__device__ __forceinline__ int64_t lower_bound(const uint32_t* keys, int64_t lo, int64_t len, uint32_t key, int lane) {
  while (len > 0) {
    const int64_t step = ceil_div(len, 64);
    const int64_t i = lo + int64_t(lane) * step;
    const bool below = i < lo + len && keys[i] < key;
    const int below_n = __popcll(__ballot(below));
    if (below_n == 0) return lo;
    // candidate below_n - 1 is below, the next one is not
    const int64_t last = lo + int64_t(below_n - 1) * step;
    const int64_t end = min(last + step, lo + len);
    lo = last + 1;
    len = end - lo;
  }
  return lo;
}

template <typename IO, int VEC>
__device__ __forceinline__ void store_row(const SumArgs& p, uint32_t v, int64_t d, const float (&acc)[VEC]) {
  Pack<IO, VEC> o;
#pragma unroll
  for (int k = 0; k < VEC; ++k) o.v[k] = narrow<IO>(p.scale * acc[k]);
  *reinterpret_cast<Pack<IO, VEC>*>(static_cast<IO*>(p.table) + int64_t(v) * p.ldt + d) = o;
}

// A wave: a run of sorted positions by 64 VEC values of a row.
template <typename IO, int VEC>
__device__ __forceinline__ void sum_run(const SumArgs& p, int64_t run, int chunk, int lane) {
  constexpr int U = 8;  // loads in flight
  const int64_t i0 = run << p.log_run;
  const int count = int(min(int64_t(1) << p.log_run, p.n - i0));
  const int64_t mine = i0 + min(lane, count - 1);
  const uint32_t key = p.key[mine], at = p.at[mine];
  const uint32_t prev = i0 > 0 ? p.key[i0 - 1] : ~0u, next = i0 + count < p.n ? p.key[i0 + count] : ~0u;
  const int64_t d0 = (int64_t(chunk) * 64 + lane) * VEC;
  const bool on = d0 < p.D;
  const int64_t d = on ? min(d0, p.D - VEC) : 0;  // (a row's last lane shares values with the one before)
  const IO* grad = static_cast<const IO*>(p.grad) + d;
  const bool inside = __builtin_amdgcn_readlane(key, 0) == prev;  // the first id began before
  bool first = true;
  float acc[VEC] = {};
  for (int j0 = 0; j0 < count; j0 += U) {
    Pack<IO, VEC> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)  // past the end: the last position again, dropped below
      v[u] = *reinterpret_cast<const Pack<IO, VEC>*>(grad + int64_t(__builtin_amdgcn_readlane(at, min(j0 + u, count - 1))) * p.ldg);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u;
      if (j >= count) break;
      const uint32_t k = __builtin_amdgcn_readlane(key, j);
      if (k >= p.V) return;  // the rest name no row
#pragma unroll
      for (int e = 0; e < VEC; ++e) acc[e] += widen(v[u].v[e]);
      const uint32_t after = j + 1 < count ? __builtin_amdgcn_readlane(key, j + 1) : next;
      const bool last = j + 1 == count;
      if (k != after || last) {
        const bool begun = first && inside, goes_on = last && k == after;
        if (on) {
          if (!begun && !goes_on) {
            store_row<IO, VEC>(p, k, d, acc);
          } else {
            Pack<float, VEC> o;
#pragma unroll
            for (int e = 0; e < VEC; ++e) o.v[e] = acc[e];
            *reinterpret_cast<Pack<float, VEC>*>(p.part + (run * 2 + (begun ? 0 : 1)) * p.D + d) = o;
          }
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] = 0.0f;
        first = false;
      }
    }
  }
}

// The first sum_blocks blocks sum runs, the others clear the rows that no token names.
template <typename IO, int VEC>
__global__ void __launch_bounds__(kThreads) embed_sum_kernel(SumArgs p) {
  __shared__ int64_t bounds[2];
  __shared__ uint32_t named;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (blockIdx.x < p.sum_blocks) {
    const int64_t unit = int64_t(blockIdx.x) * (kThreads / 64) + w;
    if (unit < p.runs * p.chunks) sum_run<IO, VEC>(p, unit / p.chunks, int(unit % p.chunks), lane);
    return;
  }
  const uint32_t v0 = uint32_t(blockIdx.x - p.sum_blocks) * kRows;
  const uint32_t rows = min(uint32_t(kRows), p.V - v0);
  if (threadIdx.x == 0) named = 0;
  if (w < 2) {
    const int64_t at = lower_bound(p.key, 0, p.n, v0 + (w ? rows : 0), lane);
    if (lane == 0) bounds[w] = at;
  }
  __syncthreads();
  for (int64_t i = bounds[0] + threadIdx.x; i < bounds[1]; i += kThreads) {
    const uint32_t k = p.key[i];
    if (i == bounds[0] || p.key[i - 1] != k) atomicOr(&named, 1u << (k - v0));
  }
  __syncthreads();
  const uint32_t have = named;
  Pack<IO, VEC> zero;  // +0, not the scale's product with it: a negative one has -0
#pragma unroll
  for (int k = 0; k < VEC; ++k) zero.v[k] = narrow<IO>(0.0f);
  for (uint32_t r = w; r < rows; r += kThreads / 64) {
    if (have >> r & 1) continue;
    IO* row = static_cast<IO*>(p.table) + int64_t(v0 + r) * p.ldt;
    for (int64_t d = lane * VEC; d < p.D; d += 64 * VEC) *reinterpret_cast<Pack<IO, VEC>*>(row + min(d, p.D - VEC)) = zero;
  }
}

// Ids whose positions go on past a run: the block of the run that they begin in adds
// the runs' sums, each of its waves a share.  Bound by the most frequent id (7 us for 84
// runs), whose sums are read eight at a time by each wave.
template <typename IO, int VEC>
__global__ void __launch_bounds__(kThreads) embed_join_kernel(SumArgs p) {
  constexpr int W = kThreads / 64, U = 8;
  __shared__ float join[W][64 * VEC];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t run = blockIdx.x, i0 = run << p.log_run, i1 = (run + 1) << p.log_run;  // (i1 < n: the last run has no block)
  const uint32_t k = p.key[i1 - 1];
  if (k >= p.V || p.key[i1] != k || (i0 > 0 && p.key[i0 - 1] == k)) return;
  const int64_t end = lower_bound(p.key, i1, p.n - i1, k + 1, lane);
  const int64_t runs = ((end - 1) >> p.log_run) - run;  // that go on
  const int64_t each = ceil_div(runs, W), lo = min(run + 1 + w * each, run + 1 + runs), hi = min(lo + each, run + 1 + runs);
  const int64_t d0 = (int64_t(blockIdx.y) * 64 + lane) * VEC, d = min(d0, p.D - VEC);
  const bool on = d0 < p.D;
  float acc[VEC] = {};
  if (on) {
    if (w == 0) {
      const auto v = *reinterpret_cast<const Pack<float, VEC>*>(p.part + (run * 2 + 1) * p.D + d);
#pragma unroll
      for (int e = 0; e < VEC; ++e) acc[e] = v.v[e];
    }
    for (int64_t r = lo; r < hi; r += U) {
      Pack<float, VEC> v[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        v[u] = *reinterpret_cast<const Pack<float, VEC>*>(p.part + min(r + u, hi - 1) * 2 * p.D + d);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (r + u < hi)
#pragma unroll
          for (int e = 0; e < VEC; ++e) acc[e] += v[u].v[e];
    }
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) join[w][e * 64 + lane] = acc[e];
  __syncthreads();
  if (w == 0 && on) {
#pragma unroll
    for (int q = 1; q < W; ++q)
#pragma unroll
      for (int e = 0; e < VEC; ++e) acc[e] += join[q][e * 64 + lane];
    store_row<IO, VEC>(p, k, d, acc);
  }
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
dendsn_status check_cfg(const dendsn_embed_cfg* c) {
  if (!c) return fail(DENDSN_E_INVALID, "cfg is NULL");
  // a launch has fewer than 2^32 threads: 64 of them a token, 16 a row of the table
  if (c->n < 0 || c->n > (int64_t(1) << 25)) return fail(DENDSN_E_INVALID, "n must be in [0, 2^25]");
  if (c->V < 0 || c->V > (int64_t(1) << 27)) return fail(DENDSN_E_INVALID, "V must be in [0, 2^27]");
  if (c->D < 0 || c->D >= (int64_t(1) << 22)) return fail(DENDSN_E_INVALID, "D must be in [0, 2^22)");
  if (c->ld_table < c->D || c->ld_table > kMaxElems) return fail(DENDSN_E_INVALID, "ld_table must be >= D");
  if (c->ld_out < 0 || c->ld_out > kMaxElems) return fail(DENDSN_E_INVALID, "ld_out negative or too large");
  if (!small_product(c->V, c->ld_table) || !small_product(c->n, c->ld_out) || !small_product(c->n, c->D))
    return fail(DENDSN_E_INVALID, "V * ld_table, n * ld_out or n * D too large");
  if (c->io != DENDSN_IO_F32 && c->io != DENDSN_IO_BF16) return fail(DENDSN_E_INVALID, "bad io");
  if (c->index != DENDSN_INDEX_I32 && c->index != DENDSN_INDEX_I64) return fail(DENDSN_E_INVALID, "bad index");
  if (!isfinite(c->scale)) return fail(DENDSN_E_INVALID, "scale must be finite");
  return DENDSN_OK;
}

size_t esize(const dendsn_embed_cfg* c) { return c->io == DENDSN_IO_BF16 ? 2 : 4; }

// 16 bytes a lane, but for rows that are shorter.
bool wide(const dendsn_embed_cfg* c) { return c->D >= int64_t(16 / esize(c)); }

// Blocks of embed_sum_kernel: a launch has fewer than 2^32 threads.
dendsn_status check_sums(const dendsn_embed_cfg* c) {
  if (ceil_div(c->n, 32) * ceil_div(c->D, 64) > (int64_t(1) << 25))
    return fail(DENDSN_E_UNSUPPORTED, "n * D must be at most 2^36");
  return DENDSN_OK;
}

struct Layout {
  size_t key[2], at[2], hist, part, total;
  int64_t tile, runs;
  uint32_t ntiles;
  int bits, passes, log_run;
};

Layout layout(const dendsn_embed_cfg* c) {
  Layout l;
  Carve cv;
  int bits = 1;  // of the keys 0 .. V
  while (bits < 32 && (uint64_t(c->V) >> bits) != 0) ++bits;
  l.passes = int(ceil_div(bits, kBits));
  l.bits = int(ceil_div(bits, l.passes));
  const int64_t n = c->n > 0 ? c->n : 1;
  l.tile = round_up(ceil_div(n, kMaxTiles), kSortThreads);
  l.ntiles = uint32_t(ceil_div(n, l.tile));
  // Runs of 32, or of 16 where those are fewer waves than four a CU: 8192 positions of 513
  // in fp32 (768 waves) sums and join 11 + 4 us, of 16 7 + 5; 32768 of 1024 in bf16 (2048
  // waves) 25 + 8, of 16 26 + 13.
  const int64_t chunks = ceil_div(c->D, wide(c) ? 64 * int64_t(16 / esize(c)) : 64);
  l.log_run = ceil_div(n, 32) * chunks < 1024 ? 4 : 5;
  l.runs = ceil_div(n, int64_t(1) << l.log_run);
  for (int i = 0; i < 2; ++i) {
    l.key[i] = cv.take(size_t(n) * 4);
    l.at[i] = cv.take(size_t(n) * 4);
  }
  l.hist = cv.take(size_t(l.ntiles) * kRadix * 4);
  l.part = cv.take(size_t(l.runs) * 2 * size_t(c->D) * 4);
  l.total = cv.at;
  return l;
}

// Sorts the positions by id; returns which of the two buffers holds the result.
template <typename ID>
int sort(const dendsn_embed_cfg* c, const Layout& l, const void* ids, char* ws, hipStream_t stream) {
  uint32_t *key[2], *at[2];
  for (int i = 0; i < 2; ++i) {
    key[i] = reinterpret_cast<uint32_t*>(ws + l.key[i]);
    at[i] = reinterpret_cast<uint32_t*>(ws + l.at[i]);
  }
  SortArgs s{};
  s.ids = ids; s.n = c->n; s.tile = l.tile; s.V = uint32_t(c->V); s.ntiles = l.ntiles;
  s.bits = l.bits; s.passes = l.passes;
  const dim3 grid(l.ntiles), block(kSortThreads);
  if (c->n <= kOneBlock) {
    embed_sort_kernel<ID><<<dim3(1), block, 0, stream>>>(s, key[0], at[0], key[1], at[1]);
    return l.passes & 1;
  }
  s.hist = reinterpret_cast<uint32_t*>(ws + l.hist);
  for (int k = 0; k < l.passes; ++k) {
    s.shift = k * l.bits;
    s.key_in = key[k & 1]; s.at_in = at[k & 1];
    s.key_out = key[~k & 1]; s.at_out = at[~k & 1];
    if (c->n <= kCountAll) {
      if (k == 0) embed_scatter_kernel<ID, true, false><<<grid, block, 0, stream>>>(s);
      else embed_scatter_kernel<ID, false, false><<<grid, block, 0, stream>>>(s);
    } else if (k == 0) {
      embed_hist_kernel<ID, true><<<grid, block, 0, stream>>>(s);
      embed_scatter_kernel<ID, true, true><<<grid, block, 0, stream>>>(s);
    } else {
      embed_hist_kernel<ID, false><<<grid, block, 0, stream>>>(s);
      embed_scatter_kernel<ID, false, true><<<grid, block, 0, stream>>>(s);
    }
  }
  return l.passes & 1;
}

template <typename IO, int VEC>
void sums(SumArgs a, hipStream_t stream) {
  a.chunks = int(ceil_div(a.D, 64 * VEC));
  a.sum_blocks = ceil_div(a.runs * a.chunks, kThreads / 64);
  embed_sum_kernel<IO, VEC>
      <<<dim3(unsigned(a.sum_blocks + ceil_div(a.V, kRows))), dim3(kThreads), 0, stream>>>(a);
  if (a.runs > 1)
    embed_join_kernel<IO, VEC><<<dim3(unsigned(a.runs - 1), unsigned(a.chunks)), dim3(kThreads), 0, stream>>>(a);
}

template <typename IO, typename ID>
void forward(const dendsn_embed_cfg* c, const void* ids, const void* table, void* out, hipStream_t stream) {
  const dim3 grid(unsigned(ceil_div(c->n, kThreads / 64))), block(kThreads);
  constexpr int VEC = 16 / sizeof(IO);
  const auto* i = static_cast<const ID*>(ids);
  const auto* t = static_cast<const IO*>(table);
  auto* o = static_cast<IO*>(out);
  if (wide(c))
    embed_fwd_kernel<IO, ID, VEC><<<grid, block, 0, stream>>>(i, t, o, c->n, uint32_t(c->V), c->D, c->ld_table, c->ld_out, c->scale);
  else
    embed_fwd_kernel<IO, ID, 1><<<grid, block, 0, stream>>>(i, t, o, c->n, uint32_t(c->V), c->D, c->ld_table, c->ld_out, c->scale);
}

}  // namespace
}  // namespace dendsn_seq

using namespace dendsn_seq;

extern "C" {

dendsn_status dendsn_embed_forward(const dendsn_embed_cfg* cfg, const void* ids, const void* table, void* out,
                                   hipStream_t stream) {
  clear_error();
  const dendsn_status st = check_cfg(cfg);
  if (st != DENDSN_OK) return st;
  const bool none = cfg->n == 0 || cfg->D == 0;
  const size_t isz = cfg->index == DENDSN_INDEX_I64 ? 8 : 4, esz = esize(cfg);
  if (!none && (!ids || !out)) return fail(DENDSN_E_INVALID, "ids or out is NULL");
  if (!none && cfg->V > 0 && !table) return fail(DENDSN_E_INVALID, "table is NULL");
  if (!aligned(ids, isz) || !aligned(table, esz) || !aligned(out, esz))
    return fail(DENDSN_E_INVALID, "ids, table or out misaligned");
  if (cfg->n > 1 && cfg->ld_out < cfg->D) return fail(DENDSN_E_INVALID, "ld_out must be >= D");
  if (none) return DENDSN_OK;
  const bool l = cfg->index == DENDSN_INDEX_I64;
  if (cfg->io == DENDSN_IO_BF16)
    l ? forward<bf16_t, int64_t>(cfg, ids, table, out, stream) : forward<bf16_t, int32_t>(cfg, ids, table, out, stream);
  else
    l ? forward<float, int64_t>(cfg, ids, table, out, stream) : forward<float, int32_t>(cfg, ids, table, out, stream);
  return launched("embedding forward");
}

dendsn_status dendsn_embed_workspace_bytes(const dendsn_embed_cfg* cfg, size_t* bytes) {
  clear_error();
  dendsn_status st = check_cfg(cfg);
  if (st == DENDSN_OK) st = check_sums(cfg);
  if (st != DENDSN_OK) return st;
  if (!bytes) return fail(DENDSN_E_INVALID, "bytes is NULL");
  *bytes = layout(cfg).total;
  return DENDSN_OK;
}

dendsn_status dendsn_embed_backward(const dendsn_embed_cfg* cfg, const void* ids, const void* grad_out,
                                    void* grad_table, void* workspace, size_t workspace_bytes,
                                    hipStream_t stream) {
  clear_error();
  dendsn_status st = check_cfg(cfg);
  if (st == DENDSN_OK) st = check_sums(cfg);
  if (st != DENDSN_OK) return st;
  const bool none = cfg->V == 0 || cfg->D == 0;
  const size_t isz = cfg->index == DENDSN_INDEX_I64 ? 8 : 4, esz = esize(cfg);
  if (!none && !grad_table) return fail(DENDSN_E_INVALID, "grad_table is NULL");
  if (!none && cfg->n > 0 && (!ids || !grad_out)) return fail(DENDSN_E_INVALID, "ids or grad_out is NULL");
  if (!aligned(ids, isz) || !aligned(grad_out, esz) || !aligned(grad_table, esz))
    return fail(DENDSN_E_INVALID, "ids, grad_out or grad_table misaligned");
  const Layout l = layout(cfg);
  st = check_workspace(workspace, workspace_bytes, l.total, "dendsn_embed_workspace_bytes");
  if (st != DENDSN_OK) return st;
  if (none) return DENDSN_OK;

  char* ws = static_cast<char*>(workspace);
  int cur = 0;
  if (cfg->n > 0)
    cur = cfg->index == DENDSN_INDEX_I64 ? sort<int64_t>(cfg, l, ids, ws, stream) : sort<int32_t>(cfg, l, ids, ws, stream);
  SumArgs a{};
  a.runs = cfg->n > 0 ? l.runs : 0;
  a.log_run = l.log_run;
  a.key = reinterpret_cast<const uint32_t*>(ws + l.key[cur]);
  a.at = reinterpret_cast<const uint32_t*>(ws + l.at[cur]);
  a.grad = grad_out; a.table = grad_table;
  a.part = reinterpret_cast<float*>(ws + l.part);
  a.n = cfg->n; a.D = cfg->D; a.ldg = cfg->ld_out; a.ldt = cfg->ld_table; a.V = uint32_t(cfg->V); a.scale = cfg->scale;
  const bool w = wide(cfg);
  if (cfg->io == DENDSN_IO_BF16)
    w ? sums<bf16_t, 8>(a, stream) : sums<bf16_t, 1>(a, stream);
  else
    w ? sums<float, 4>(a, stream) : sums<float, 1>(a, stream);
  return launched("embedding backward");
}

}  // extern "C"
