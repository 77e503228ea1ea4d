// Embedding: rows of a table, scaled, and the table's gradient.
//
//   out[i] = s table[id_i],   grad_table[v] = s sum over {i : id_i = v} of grad_out[i]
//
// The gradient adds each row's positions in ascending order, so that it does not
// depend on scheduling: positions are sorted by id (a stable radix sort of up to 9
// bits a pass), rows of 64 sorted positions that all hold one id are summed first
// (frequent tokens), and then every row of the table is written once, +0 or the sum
// of its first loose positions, its whole rows of 64 and its last loose positions.
// Both directions are bound by memory: the gradient writes all V rows.
#include "seq_common.h"

namespace dendsn_seq {
namespace {

constexpr int kThreads = 256;
constexpr int kBits = 9, kRadix = 1 << kBits;  // most bits of a pass
constexpr int kChunk = 2048;                   // positions of a sorting block, at least
constexpr int kMaxTiles = 512;                 // sorting blocks, at most
constexpr int kRun = 64;                       // sorted positions of a partial sum
constexpr int kRows = 32;                      // table rows of a block
constexpr int kRowWaves = 8;
constexpr int kLight = 16;  // a row of at most so many positions is one wave's

template <typename ID>
__device__ __forceinline__ uint32_t key_of(const ID* ids, int64_t i, uint32_t V) {
  const int64_t id = int64_t(ids[i]);
  return id >= 0 && id < int64_t(V) ? uint32_t(id) : V;  // V: no row
}

// A wave a row: 64 lanes over its values, VEC a lane.
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
  for (int64_t d = lane * VEC; d < D; d += 64 * VEC) {
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
  int64_t n, tile;              // tile: positions of a block, a multiple of kThreads
  uint32_t V, ntiles;
  int shift, bits;
};

template <typename ID, bool FIRST>
__device__ __forceinline__ uint32_t sort_key(const SortArgs& p, int64_t i) {
  return FIRST ? key_of(static_cast<const ID*>(p.ids), i, p.V) : p.key_in[i];
}

template <typename ID, bool FIRST>
__global__ void __launch_bounds__(kThreads) embed_hist_kernel(SortArgs p) {
  __shared__ uint32_t h[kRadix];
  for (int d = threadIdx.x; d < kRadix; d += kThreads) h[d] = 0;
  __syncthreads();
  const int64_t lo = blockIdx.x * p.tile, hi = min(lo + p.tile, p.n);
  const uint32_t mask = (1u << p.bits) - 1;
  for (int64_t i = lo + threadIdx.x; i < hi; i += kThreads)
    atomicAdd(&h[(sort_key<ID, FIRST>(p, i) >> p.shift) & mask], 1u);
  __syncthreads();
  for (int d = threadIdx.x; d < kRadix; d += kThreads) p.hist[int64_t(blockIdx.x) * kRadix + d] = h[d];
}

template <typename ID, bool FIRST>
__global__ void __launch_bounds__(kThreads) embed_scatter_kernel(SortArgs p) {
  constexpr int W = kThreads / 64;
  __shared__ uint32_t base[kRadix], count[W][kRadix], sums[kThreads];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  // where this block's first position of each digit goes: digits before it in all
  // blocks, and the digit itself in the blocks before
  uint32_t total[2] = {0, 0}, before[2] = {0, 0};
  for (uint32_t t = 0; t < p.ntiles; ++t) {
    const uint2 c = *reinterpret_cast<const uint2*>(p.hist + int64_t(t) * kRadix + 2 * tid);
    total[0] += c.x;
    total[1] += c.y;
    if (t < blockIdx.x) before[0] += c.x, before[1] += c.y;
  }
  sums[tid] = total[0] + total[1];
  __syncthreads();
  for (int s = 1; s < kThreads; s <<= 1) {
    const uint32_t add = tid >= s ? sums[tid - s] : 0;
    __syncthreads();
    sums[tid] += add;
    __syncthreads();
  }
  const uint32_t first = sums[tid] - total[0] - total[1];
  base[2 * tid] = first + before[0];
  base[2 * tid + 1] = first + total[0] + before[1];
  const uint32_t mask = (1u << p.bits) - 1;
  const int64_t lo = blockIdx.x * p.tile, hi = min(lo + p.tile, p.n);
  for (int64_t i0 = lo; i0 < hi; i0 += kThreads) {
    for (int d = tid; d < W * kRadix; d += kThreads) (&count[0][0])[d] = 0;
    __syncthreads();
    const int64_t i = i0 + tid;
    const bool in = i < hi;
    const uint32_t key = in ? sort_key<ID, FIRST>(p, i) : 0;
    const uint32_t digit = (key >> p.shift) & mask;
    uint64_t same = __ballot(in);
    for (int b = 0; b < p.bits; ++b) {
      const bool set = (digit >> b) & 1;
      const uint64_t votes = __ballot(set);
      same &= set ? votes : ~votes;
    }
    const uint32_t rank = __popcll(same & ((uint64_t(1) << lane) - 1));
    if (in && rank == 0) count[w][digit] = __popcll(same);
    __syncthreads();
    if (in) {
      uint32_t to = base[digit] + rank;
      for (int q = 0; q < w; ++q) to += count[q][digit];
      p.key_out[to] = key;
      p.at_out[to] = FIRST ? uint32_t(i) : p.at_in[i];
    }
    __syncthreads();
    for (int d = tid; d < kRadix; d += kThreads) {
      uint32_t add = 0;
#pragma unroll
      for (int q = 0; q < W; ++q) add += count[q][d];
      base[d] += add;
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// Sums
// ---------------------------------------------------------------------------
struct SumArgs {
  const uint32_t *key, *at;  // sorted
  const void* grad;
  void* table;
  float* part;               // [n / kRun][D]
  int64_t n, D, ldg, ldt;
  uint32_t V;
  float scale;
};

template <typename IO, int VEC>
__device__ __forceinline__ void add_rows(float (&acc)[VEC], const SumArgs& p, int64_t from, int64_t to, int64_t d) {
  const IO* grad = static_cast<const IO*>(p.grad);
  constexpr int U = 8;  // loads in flight
  for (int64_t i = from; i < to; i += U) {
    Pack<IO, VEC> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)  // past the end: the last row again, dropped below
      v[u] = *reinterpret_cast<const Pack<IO, VEC>*>(grad + int64_t(p.at[min(i + u, to - 1)]) * p.ldg + d);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u < to)
#pragma unroll
        for (int k = 0; k < VEC; ++k) acc[k] += widen(v[u].v[k]);
  }
}

template <int VEC>
__device__ __forceinline__ void add_parts(float (&acc)[VEC], const SumArgs& p, int64_t from, int64_t to, int64_t d) {
  constexpr int U = 4;
  for (int64_t i = from; i < to; i += U) {
    Pack<float, VEC> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = *reinterpret_cast<const Pack<float, VEC>*>(p.part + min(i + u, to - 1) * p.D + d);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u < to)
#pragma unroll
        for (int k = 0; k < VEC; ++k) acc[k] += v[u].v[k];
  }
}

// The sum of kRun sorted positions, where they all hold one id.
template <typename IO, int VEC>
__global__ void __launch_bounds__(64) embed_part_kernel(SumArgs p) {
  const int64_t j = blockIdx.x;
  const uint32_t key = p.key[j * kRun];
  if (key >= p.V || key != p.key[j * kRun + kRun - 1]) return;
  const int64_t d = (int64_t(blockIdx.y) * 64 + threadIdx.x) * VEC;
  if (d >= p.D) return;
  float acc[VEC] = {};
  add_rows<IO, VEC>(acc, p, j * kRun, (j + 1) * kRun, d);
  Pack<float, VEC> o;
#pragma unroll
  for (int k = 0; k < VEC; ++k) o.v[k] = acc[k];
  *reinterpret_cast<Pack<float, VEC>*>(p.part + j * p.D + d) = o;
}

// First sorted position whose key is at least `key`, by one wave: 64 candidates a step.
__device__ __forceinline__ int64_t lower_bound(const uint32_t* keys, int64_t n, uint32_t key, int lane) {
  int64_t lo = 0, len = n;  // the answer lies in [lo, lo + len]
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

// kRows rows of the table: a wave for a row of few positions, the whole block for a
// row of many.
template <typename IO, int VEC>
__global__ void __launch_bounds__(kRowWaves * 64) embed_rows_kernel(SumArgs p) {
  __shared__ int64_t bounds[2];
  __shared__ int64_t start[kRows + 1];
  __shared__ float join[kRowWaves][64 * VEC];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const uint32_t v0 = blockIdx.x * uint32_t(kRows);
  const uint32_t rows = min(uint32_t(kRows), p.V - v0);
  if (w < 2) {
    const int64_t at = lower_bound(p.key, p.n, v0 + (w ? rows : 0), lane);
    if (lane == 0) bounds[w] = at;
  }
  __syncthreads();
  const int64_t lo = bounds[0], hi = bounds[1];
  if (threadIdx.x <= kRows) start[threadIdx.x] = hi;
  __syncthreads();
  for (int64_t i = lo + threadIdx.x; i < hi; i += kRowWaves * 64) {
    const uint32_t k = p.key[i];
    uint32_t v = i > lo ? p.key[i - 1] + 1 : v0;  // rows up to k start here
    for (; v <= k; ++v) start[v - v0] = i;
  }
  __syncthreads();
  for (uint32_t r = w; r < rows; r += kRowWaves) {
    const int64_t s = start[r], e = start[r + 1];
    if (e - s > kLight) continue;
    for (int64_t d = lane * VEC; d < p.D; d += 64 * VEC) {
      float acc[VEC] = {};
      add_rows<IO, VEC>(acc, p, s, e, d);
      store_row<IO, VEC>(p, v0 + r, d, acc);
    }
  }
  for (uint32_t r = 0; r < rows; ++r) {
    const int64_t s = start[r], e = start[r + 1];
    if (e - s <= kLight) continue;
    // whole runs [b0, b1) of kRun, loose positions before and after
    const int64_t b0 = ceil_div(s, kRun), b1 = max(b0, e / kRun);
    const int64_t head = min(b0 * kRun, e), tail = max(b1 * kRun, head);
    const int64_t ph = ceil_div(head - s, kRowWaves), pp = ceil_div(b1 - b0, kRowWaves);
    const int64_t pt = ceil_div(e - tail, kRowWaves);
    for (int64_t c = 0; c < p.D; c += 64 * VEC) {
      const int64_t d = c + lane * VEC;
      float acc[VEC] = {};
      if (d < p.D) {
        add_rows<IO, VEC>(acc, p, min(s + w * ph, head), min(s + (w + 1) * ph, head), d);
        if (b1 * kRun <= e) add_parts<VEC>(acc, p, min(b0 + w * pp, b1), min(b0 + (w + 1) * pp, b1), d);
        add_rows<IO, VEC>(acc, p, min(tail + w * pt, e), min(tail + (w + 1) * pt, e), d);
      }
#pragma unroll
      for (int k = 0; k < VEC; ++k) join[w][k * 64 + lane] = acc[k];
      __syncthreads();
      if (w == 0 && d < p.D) {
#pragma unroll
        for (int q = 1; q < kRowWaves; ++q)
#pragma unroll
          for (int k = 0; k < VEC; ++k) acc[k] += join[q][k * 64 + lane];
        store_row<IO, VEC>(p, v0 + r, d, acc);
      }
      __syncthreads();
    }
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

// 16 bytes a lane where every row allows it, else element by element.
bool wide(const dendsn_embed_cfg* c, const void* a, const void* b) {
  const int64_t m = int64_t(16 / esize(c));
  return aligned(a, 16) && aligned(b, 16) && c->D % m == 0 && c->ld_table % m == 0 && c->ld_out % m == 0;
}

struct Layout {
  size_t key[2], at[2], hist, part, total;
  int64_t tile;
  uint32_t ntiles;
};

Layout layout(const dendsn_embed_cfg* c) {
  Layout l;
  Carve cv;
  l.tile = round_up(ceil_div(c->n > 0 ? c->n : 1, kMaxTiles), kThreads);
  if (l.tile < kChunk) l.tile = kChunk;
  l.ntiles = uint32_t(ceil_div(c->n > 0 ? c->n : 1, l.tile));
  for (int i = 0; i < 2; ++i) {
    l.key[i] = cv.take(size_t(c->n) * 4);
    l.at[i] = cv.take(size_t(c->n) * 4);
  }
  l.hist = cv.take(size_t(l.ntiles) * kRadix * 4);
  l.part = cv.take(size_t(c->n / kRun) * size_t(c->D) * 4);
  l.total = cv.at;
  return l;
}

template <typename ID>
void sort_pass(const SortArgs& a, bool first, hipStream_t stream) {
  const dim3 grid(a.ntiles), block(kThreads);
  if (first) {
    embed_hist_kernel<ID, true><<<grid, block, 0, stream>>>(a);
    embed_scatter_kernel<ID, true><<<grid, block, 0, stream>>>(a);
  } else {
    embed_hist_kernel<ID, false><<<grid, block, 0, stream>>>(a);
    embed_scatter_kernel<ID, false><<<grid, block, 0, stream>>>(a);
  }
}

template <typename IO, int VEC>
void sums(const SumArgs& a, hipStream_t stream) {
  if (a.n >= kRun)
    embed_part_kernel<IO, VEC>
        <<<dim3(unsigned(a.n / kRun), unsigned(ceil_div(a.D, 64 * VEC))), dim3(64), 0, stream>>>(a);
  embed_rows_kernel<IO, VEC><<<dim3(unsigned(ceil_div(a.V, kRows))), dim3(kRowWaves * 64), 0, stream>>>(a);
}

template <typename IO, typename ID>
void forward(const dendsn_embed_cfg* c, const void* ids, const void* table, void* out, hipStream_t stream) {
  const dim3 grid(unsigned(ceil_div(c->n, kThreads / 64))), block(kThreads);
  constexpr int VEC = 16 / sizeof(IO);
  const auto* i = static_cast<const ID*>(ids);
  const auto* t = static_cast<const IO*>(table);
  auto* o = static_cast<IO*>(out);
  if (wide(c, table, out))
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
  const dendsn_status st = check_cfg(cfg);
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
  SortArgs s{};
  s.ids = ids;
  s.hist = reinterpret_cast<uint32_t*>(ws + l.hist);
  s.n = cfg->n; s.tile = l.tile; s.V = uint32_t(cfg->V); s.ntiles = l.ntiles;
  int bits = 1;  // of the keys 0 .. V
  while (bits < 32 && (uint64_t(cfg->V) >> bits) != 0) ++bits;
  const int passes = int(ceil_div(bits, kBits));
  s.bits = int(ceil_div(bits, passes));
  int cur = 0;
  if (cfg->n > 0) {
    for (int k = 0; k < passes; ++k) {
      s.shift = k * s.bits;
      s.key_in = reinterpret_cast<const uint32_t*>(ws + l.key[cur]);
      s.at_in = reinterpret_cast<const uint32_t*>(ws + l.at[cur]);
      cur ^= 1;
      s.key_out = reinterpret_cast<uint32_t*>(ws + l.key[cur]);
      s.at_out = reinterpret_cast<uint32_t*>(ws + l.at[cur]);
      cfg->index == DENDSN_INDEX_I64 ? sort_pass<int64_t>(s, k == 0, stream) : sort_pass<int32_t>(s, k == 0, stream);
    }
  }
  SumArgs a{};
  a.key = reinterpret_cast<const uint32_t*>(ws + l.key[cur]);
  a.at = reinterpret_cast<const uint32_t*>(ws + l.at[cur]);
  a.grad = grad_out; a.table = grad_table;
  a.part = reinterpret_cast<float*>(ws + l.part);
  a.n = cfg->n; a.D = cfg->D; a.ldg = cfg->ld_out; a.ldt = cfg->ld_table; a.V = uint32_t(cfg->V); a.scale = cfg->scale;
  const bool w = wide(cfg, grad_out, grad_table);
  if (cfg->io == DENDSN_IO_BF16)
    w ? sums<bf16_t, 8>(a, stream) : sums<bf16_t, 1>(a, stream);
  else
    w ? sums<float, 4>(a, stream) : sums<float, 1>(a, stream);
  return launched("embedding backward");
}

}  // extern "C"
