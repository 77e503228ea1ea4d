// Softmax cross entropy of a linear readout over a vocabulary.
//
//   z = s H W^T,  lse = log sum_v exp z_v,  loss = lse - z_target
//   dz = r s (softmax(z) - onehot(target)),  dH = dz W,  dW = dz^T H
//
// The rows go through in pieces whose logits fit a bounded scratch.  Of a piece, the
// first product leaves each row's maximum and sum of exponentials over every tile of
// the vocabulary (and, for the gradient, its fp32 logits); the tiles' statistics are
// joined into the row's; the gradient of the logits, without the rows' common factor (see
// ce_unit_kernel), is rounded to bf16 once and enters the two other products, dW summed
// over the pieces in fp32.  The three products carry the time: 2 N V D operations each.
//
// 8192 rows, 128000 classes, 2048 features in bf16, 11.7 ms: logits 4.02 ms (1070 TF with
// their 4.2 GB of stores; 1275 TF without), dz 1.21 ms (5.2 TB/s), dH 2.92 ms (1470 TF), dW
// 3.52 ms (1220 TF); the card's power limit holds the clock at 1.8 to 1.95 GHz throughout.
// A library product of 8192^3 reaches 1510 TF, of dW's form 1060.
#include "seq_gemm.h"

namespace dendsn_seq {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kMostThreads = int64_t(1) << 31;  // of a launch (it has fewer than 2^32)
constexpr int64_t kPieceBytes = int64_t(4) << 30;  // of a piece's logits with their gradient, and of its packed rows

__device__ __forceinline__ int64_t target_of(const void* t, int wide, int64_t i) {
  return wide ? static_cast<const int64_t*>(t)[i] : int64_t(static_cast<const int32_t*>(t)[i]);
}

// ---------------------------------------------------------------------------
// Operands as bf16 planes
// ---------------------------------------------------------------------------
struct PackArgs {
  const void* src;
  uint16_t* dst;
  const void* targets;  // rows without a target become zero (NULL: none)
  int64_t rows, cols, ld, cols_p, plane, V;
  int wide, planes;
  int64_t first;  // thread of the launch's first
};

// v as three bf16 that add up to it: each the nearest to what the ones before leave, so that
// the second is at most 2^-8 and the third 2^-17 of v's power of two, with either sign (cut
// off, they would be twice and four times that, all of v's sign, and so would what the
// products of lower planes lose).  Infinities and NaN are in the first alone, and not in its
// finite copy.
__device__ __forceinline__ void split3(float v, uint16_t& a, uint16_t& finite, uint16_t& b, uint16_t& c) {
  const uint32_t u = __float_as_uint(v);
  if ((u & 0x7F800000u) == 0x7F800000u) {
    a = uint16_t(u >> 16);
    if (u & 0x7FFFFFu) a |= 0x40;  // a NaN stays one without its low bits
    finite = b = c = 0;
    return;
  }
  constexpr float kMost = 3.38953139e38f;  // of bf16: beyond it the nearest would be infinite
  a = finite = bf16_bits(__builtin_amdgcn_fmed3f(v, -kMost, kMost));
  const float r1 = v - __uint_as_float(uint32_t(a) << 16);
  b = bf16_bits(r1);
  const float r2 = r1 - __uint_as_float(uint32_t(b) << 16);
  c = uint16_t(__float_as_uint(r2) >> 16);  // (at most eight bits are left)
}

__device__ __forceinline__ void store8(uint16_t* to, const uint16_t (&x)[8]) {
  uint4 q;
  q.x = x[0] | uint32_t(x[1]) << 16;
  q.y = x[2] | uint32_t(x[3]) << 16;
  q.z = x[4] | uint32_t(x[5]) << 16;
  q.w = x[6] | uint32_t(x[7]) << 16;
  *reinterpret_cast<uint4*>(to) = q;
}

// Eight values a thread.
template <typename IO>
__global__ void __launch_bounds__(kThreads) ce_pack_kernel(PackArgs p) {
  const int64_t chunks = p.cols_p / 8, id = p.first + int64_t(blockIdx.x) * kThreads + threadIdx.x;
  const int64_t row = id / chunks, d = id % chunks * 8;
  if (row >= p.rows) return;
  bool keep = true;
  if (p.targets) {
    const int64_t t = target_of(p.targets, p.wide, row);
    keep = t >= 0 && t < p.V;
  }
  const IO* src = static_cast<const IO*>(p.src) + row * p.ld + d;
  float v[8] = {};
  if (keep && d + 8 <= p.cols) {
    const auto x = *reinterpret_cast<const Pack<IO, 8>*>(src);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = widen(x.v[k]);
  } else if (keep) {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (d + k < p.cols) v[k] = widen(src[k]);
  }
  uint16_t* dst = p.dst + row * p.cols_p + d;
  uint16_t a[8], f[8], b[8], c[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (p.planes == 1) a[k] = bf16_bits(v[k]);
    else split3(v[k], a[k], f[k], b[k], c[k]);
  }
  store8(dst, a);
  if (p.planes == 3) {
    store8(dst + p.plane, b);
    store8(dst + 2 * p.plane, c);
    store8(dst + kFinite * p.plane, f);
  }
}

// ---------------------------------------------------------------------------
// The products
// ---------------------------------------------------------------------------
// exp(a - b): the difference first, which is exact where it matters (a scaled maximum
// would be rounded, by hundredths for logits of 10^4).  The argument of exp2 is rounded once: a
// probability p is off by p |log p| 2^-24, at most 0.37 x 2^-24.
__device__ __forceinline__ float exp_diff(float a, float b) {
  return __builtin_amdgcn_exp2f(1.44269504f * (a - b));
}

// What the exponentials of a row are taken from: its maximum, kept finite, since infinity
// less itself is none (minus infinity then gives a sum of 0, plus infinity an infinite one).
__device__ __forceinline__ float anchor(float top) { return __builtin_amdgcn_fmed3f(top, -3.40282347e38f, 3.40282347e38f); }

struct LogitArgs {
  GemmArgs g;
  float scale;
  float2* stats;   // [M][tiles_n] maximum and sum of exponentials
  float* z;        // hidden weight^T in panels of 64 classes, NULL: not kept
  float* chosen;   // [M] the target's (where z is not kept)
  const void* targets;
  int64_t zrows, zcols;  // rows of a panel, classes of all
  int wide;
};

// Over the four lane groups of a wave that hold one row.
template <typename F>
__device__ __forceinline__ float over_groups(float v, F f) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Each row's maximum and sum of exponentials over a wave's columns n0 + 16 i + 0..3 of its
// tile (those below N; WHOLE: all of them), times scale >= 0, to to[16 j].
template <bool WHOLE, int FN, int FM>
__device__ __forceinline__ void row_statistics(const f32x4 (&acc)[FN][FM], int64_t n0, int64_t N, float scale, float2* to,
                                               int lane) {
  const float c = 1.44269504f * scale;
  const auto in = [&](int i, int r) { return WHOLE || n0 + 16 * i + r < N; };
#pragma unroll
  for (int j = 0; j < FM; ++j) {
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) top = fmaxf(top, in(i, r) ? acc[i][j][r] : -INFINITY);
    top = over_groups(top, [](float a, float b) { return fmaxf(a, b); });
    const float ref = anchor(top);
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        // (the difference first: see exp_diff)
        sum += in(i, r) ? __builtin_amdgcn_exp2f(c * (acc[i][j][r] - ref)) : 0.0f;
    sum = over_groups(sum, [](float a, float b) { return a + b; });
    // (of a finite maximum: with no class of its own and a scale of 0 the other would be NaN)
    if (lane < 16) to[16 * j] = make_float2(scale * ref, sum);
  }
}

// A block takes tiles in turn: the next one's first stages are fetched while it works
// out this one's statistics.  Where the logits are kept it has one tile: its fetches
// would wait for its stores (vmcnt counts both, in order), which a new block's do not.
template <int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(WM * WN * 64) ce_logits_kernel(LogitArgs) {
  using G = Gemm<BM, BN, WM, WN, false, false, false>;
  // (one array: with two, the compiler tells reads of one from DMA into the other, and
  // makes every read of a stage wait for all DMA in flight)
  __shared__ __align__(1024) char lds[2 * G::kStage + G::kNotes];
  float2(*part)[BM] = reinterpret_cast<float2(*)[BM]>(lds + 2 * G::kStage);
  G gemm(lds);
  const int lane = gemm.lane, wm = gemm.w / WN, wn = gemm.w % WN;
  int tm, tn;
  tile_of(arguments<GemmArgs>(), blockIdx.x, tm, tn);
  gemm.begin(tm, tn, 0);
  G::landed();
  block_barrier();
  for (uint32_t id = blockIdx.x;; ) {
    f32x4 acc[G::FN][G::FM];
    gemm.run(acc);
    const LogitArgs& p = arguments<LogitArgs>();
    const uint32_t tiles = scalar(p.g.tiles_m * p.g.tiles_n);
    const float scale = p.scale;
    const int64_t m0 = int64_t(tm) * BM, n0 = int64_t(tn) * BN + wn * G::TN + 4 * (lane >> 4);
    const bool whole = int64_t(tn + 1) * BN <= p.g.N;
    const int this_tn = tn;
    id += gridDim.x;
    if (id < tiles) {
      tile_of(p.g, id, tm, tn);
      gemm.begin(tm, tn, 0);
    }
    const int r0 = wm * G::TM + (lane & 15);
    if (p.chosen) {
#pragma unroll
      for (int j = 0; j < G::FM; ++j) {
        const int64_t m = m0 + r0 + 16 * j;
        const int64_t at = (m < p.g.M ? target_of(p.targets, p.wide, m) : -1) - n0;
        if (at < 0 || at >= p.g.N - n0) continue;
#pragma unroll
        for (int i = 0; i < G::FN; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (at == 16 * i + r) p.chosen[m] = acc[i][j][r];
      }
    }
    if (p.z) {
      // (a column past zcols is in no panel)
      float* z = p.z + (n0 / kStep * p.zrows + m0 + r0) * kStep + n0 % kStep;
#pragma unroll
      for (int j = 0; j < G::FM; ++j)
#pragma unroll
        for (int i = 0; i < G::FN; ++i) {
          static_assert(G::TN == kStep, "a wave's columns are one panel's");
          if (n0 < p.zcols) *reinterpret_cast<f32x4*>(z + 16 * j * kStep + 16 * i) = acc[i][j];
        }
    }
    if (scale < 0.0f) {  // the largest logit belongs to the smallest product
#pragma unroll
      for (int j = 0; j < G::FM; ++j)
#pragma unroll
        for (int i = 0; i < G::FN; ++i) acc[i][j] = -acc[i][j];
    }
    if (whole) row_statistics<true>(acc, n0, p.g.N, fabsf(scale), part[wn] + r0, lane);
    else row_statistics<false>(acc, n0, p.g.N, fabsf(scale), part[wn] + r0, lane);
    if (id < tiles) G::landed();
    else __builtin_amdgcn_s_waitcnt(0xC07F);  // (lgkmcnt 0: the logits need not have arrived)
    block_barrier();
    for (int r = threadIdx.x; r < BM; r += WM * WN * 64) {
      if (m0 + r >= p.g.M) continue;
      float2 a = part[0][r];
#pragma unroll
      for (int q = 1; q < WN; ++q) {
        const float2 b = part[q][r];
        const float top = fmaxf(a.x, b.x), ref = anchor(top);
        a = make_float2(top, a.y * exp_diff(a.x, ref) + b.y * exp_diff(b.x, ref));
      }
      p.stats[(m0 + r) * p.g.tiles_n + this_tn] = a;
    }
    if (id >= tiles) break;
  }
}

// ---------------------------------------------------------------------------
// Few rows: the weights are streamed once
// ---------------------------------------------------------------------------
struct ScoreArgs {
  const void *h, *w;
  const void* targets;
  float2* stats;   // [M][gridDim.x]
  float* chosen;   // [M]
  float* z;        // as LogitArgs
  int64_t ldh, ldw, M, V, K, zrows;
  float scale;
  int wide;
};

constexpr int kScoreWaves = 8;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// 16 bytes a lane of either operand: 32 k of bf16, or four times 4 k of fp32.
template <typename IO>
__device__ __forceinline__ f32x4 multiply16(u32x4 a, u32x4 b, f32x4 acc) {
  if constexpr (sizeof(IO) == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[k]), __uint_as_float(b[k]), acc, 0, 0, 0);
    return acc;
  }
}

// A block takes V / gridDim.x classes, sixteen at a time; wave w takes the k of its U
// units of 64 (lane group q the 16 k from 16 q on, in both operands, so that whole lines of
// the weights are read at once).  The rows of hidden, MF times sixteen, stay in
// registers; the waves' sums meet in LDS, where wave f keeps the statistics of rows
// 16 f .. 16 f + 15.  Bound by the weights' bytes: two groups of classes are in flight.
template <typename IO, int MF, int U>
__global__ void __launch_bounds__(kScoreWaves * 64) ce_score_kernel(ScoreArgs p) {
  constexpr int E = 16 / sizeof(IO), L = 16 / E;  // values of a load, loads of a unit
  __shared__ f32x4 part[2][kScoreWaves][MF][64];
  const int lane = threadIdx.x & 63, w = scalar(int(threadIdx.x >> 6)), i = lane & 15, q = lane >> 4;
  int64_t n0 = p.V * blockIdx.x / gridDim.x, n1 = p.V * (blockIdx.x + 1) / gridDim.x;
  if (p.z) {  // whole sixteens, so that a lane's four lie together in a panel
    const int64_t units = ceil_div(p.V, 16);
    n0 = units * blockIdx.x / gridDim.x * 16;
    n1 = min(units * (blockIdx.x + 1) / gridDim.x * 16, p.V);
  }
  const int k0 = w * U * kStep + q * 16;
  u32x4 hf[MF][L * U];
#pragma unroll
  for (int f = 0; f < MF; ++f)
#pragma unroll
    for (int e = 0; e < L * U; ++e) {
      const int k = k0 + e / L * kStep + e % L * E;
      const int64_t m = 16 * f + i;
      hf[f][e] = u32x4{0, 0, 0, 0};
      if (m < p.M && k < p.K) hf[f][e] = *reinterpret_cast<const u32x4*>(static_cast<const IO*>(p.h) + m * p.ldh + k);
    }
  struct Group {
    u32x4 v[L * U];
  };
  auto fetch = [&](Group& g, int64_t n) {  // classes n .. n + 15; past n1 and past K: zero
    const int64_t rows = n1 - n;
    const int64_t bytes = rows > 0 ? ((rows - 1) * p.ldw + p.K) * int64_t(sizeof(IO)) : 0;
    const int records = scalar(int(bytes < 0x7FFFFFF0 ? bytes : 0x7FFFFFF0));
    const rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char*>(scalar(reinterpret_cast<const char*>(static_cast<const IO*>(p.w) + n * p.ldw))), 0, records, 0x00020000);
#pragma unroll
    for (int e = 0; e < L * U; ++e) {
      const int k = k0 + e / L * kStep + e % L * E;
      const uint32_t off = k < p.K && i < rows ? uint32_t(i * p.ldw + k) * uint32_t(sizeof(IO)) : 0x80000000u;
      g.v[e] = __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0);
    }
  };
  float top = -INFINITY, sum = 0.0f;
  const int64_t m = 16 * w + i;  // (of a wave below MF)
  const int64_t target = w < MF && m < p.M ? target_of(p.targets, p.wide, m) : -1;
  auto group = [&](Group& g, int64_t n, int buf) {
    f32x4 acc[MF];
#pragma unroll
    for (int f = 0; f < MF; ++f) acc[f] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int e = 0; e < L * U; ++e)
#pragma unroll
      for (int f = 0; f < MF; ++f) acc[f] = multiply16<IO>(g.v[e], hf[f][e], acc[f]);
    fetch(g, n + 32);
#pragma unroll
    for (int f = 0; f < MF; ++f) part[buf][w][f][lane] = acc[f];
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt 0
    block_barrier();
    if (w < MF) {
      f32x4 z = part[buf][0][w][lane];
#pragma unroll
      for (int o = 1; o < kScoreWaves; ++o) z += part[buf][o][w][lane];
      float most = top;
      if (p.z && m < p.M) *reinterpret_cast<f32x4*>(p.z + (n / kStep * p.zrows + m) * kStep + n % kStep + 4 * q) = z;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t v = n + 4 * q + r;
        if (p.chosen && v == target && v < n1) p.chosen[m] = z[r];  // (past n1: another block's)
        z[r] = v < n1 ? p.scale * z[r] : -INFINITY;
        most = fmaxf(most, z[r]);
      }
      const float ref = anchor(most);
      sum *= exp_diff(top, ref);
#pragma unroll
      for (int r = 0; r < 4; ++r) sum += exp_diff(z[r], ref);
      top = most;
    }
  };
  Group ga, gb;
  fetch(ga, n0);
  fetch(gb, n0 + 16);
  for (int64_t n = n0; n < n1; n += 32) {
    group(ga, n, 0);
    if (n + 16 < n1) group(gb, n + 16, 1);
  }
  if (w < MF) {
    const float most = over_groups(top, [](float a, float b) { return fmaxf(a, b); });
    const float ref = anchor(most);
    sum = over_groups(sum * exp_diff(top, ref), [](float a, float b) { return a + b; });
    if (lane < 16 && m < p.M) p.stats[m * gridDim.x + blockIdx.x] = make_float2(most, sum);
  }
}

struct GradArgs {
  GemmArgs g;
  const float* unit;     // what dz leaves out (NULL: 1), times scale
  float scale;
  void* out;             // io
  float* part;           // fp32: [splits][M][N] (splits > 1), or [M][N] summed over pieces
  const void* targets;   // rows without a target are +0 (NULL: none)
  int64_t ld, V;
  int wide, io;          // io: dendsn_io
  int add, keep;         // add the sum of the pieces before; keep it (else the result is whole)
};

typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) { return uint32_t(bf16_bits(a)) | uint32_t(bf16_bits(b)) << 16; }

// Eight neighbours of a row, of which those below N are there; rows of any alignment.
__device__ __forceinline__ void store8(void* out, int io, int64_t at, int64_t n, int64_t N, const float (&v)[8]) {
  if (io == DENDSN_IO_BF16) {
    uint16_t* o = static_cast<uint16_t*>(out) + at;
    if (n + 8 <= N) {
      *reinterpret_cast<u32x4_any*>(o) = u32x4_any{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
      return;
    }
#pragma unroll
    for (int r = 0; r < 8; ++r)
      if (n + r < N) o[r] = bf16_bits(v[r]);
  } else {
    float* o = static_cast<float*>(out) + at;
    if (n + 8 <= N) {
      *reinterpret_cast<f32x4_any*>(o) = f32x4_any{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<f32x4_any*>(o + 4) = f32x4_any{v[4], v[5], v[6], v[7]};
      return;
    }
#pragma unroll
    for (int r = 0; r < 8; ++r)
      if (n + r < N) o[r] = v[r];
  }
}

// dH (dz by rows, sums over the classes) or, XCOL, dW (dz by columns, sums over the rows).
// As many blocks as the chip holds take tiles in turn: the next tile's first stages are on
// their way while this one is written.
template <int BM, int BN, int WM, int WN, bool XCOL>
__global__ void __launch_bounds__(WM * WN * 64) ce_grad_kernel(GradArgs) {
  using G = Gemm<BM, BN, WM, WN, XCOL, true, true>;  // X: dz, in panels
  __shared__ __align__(1024) char lds[2 * G::kStage];
  G gemm(lds);
  const int lane = gemm.lane, wm = gemm.w / WN, wn = gemm.w % WN;
  int tm, tn, split;
  auto begin = [&](const GemmArgs& g, uint32_t id) {
    const uint32_t tiles = uint32_t(g.tiles_m) * uint32_t(g.tiles_n);
    split = scalar(int(id / tiles));
    tile_of(g, id % tiles, tm, tn);
    gemm.begin(tm, tn, split);
  };
  begin(arguments<GemmArgs>(), blockIdx.x);
  G::landed();
  block_barrier();
  for (uint32_t id = blockIdx.x;; ) {
    f32x4 acc[G::FN][G::FM];
    gemm.run(acc);
    const GradArgs& p = arguments<GradArgs>();
    const uint32_t units = scalar(p.g.tiles_m * p.g.tiles_n * p.g.splits);
    const int64_t N = p.g.N;
    const float unit = p.unit ? *p.unit * p.scale : p.scale;
    const int64_t m0 = int64_t(tm) * BM + wm * G::TM + (lane & 15);
    const int64_t n0 = int64_t(tn) * BN + wn * G::TN + 8 * (lane >> 4);
    const int this_split = split;
    id += gridDim.x;
    if (id < units) begin(p.g, id);
    G::landed();
    block_barrier();
#pragma unroll
    for (int j = 0; j < G::FM; ++j) {
      const int64_t m = m0 + 16 * j;
      if (m >= p.g.M) continue;
      bool zero = false;
      if (p.targets) {
        const int64_t t = target_of(p.targets, p.wide, m);
        zero = t < 0 || t >= p.V;
      }
#pragma unroll
      for (int i = 0; i < G::FN; i += 2) {
        const int64_t n = n0 + 16 * i;
        if (n >= N) continue;
        float v[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r] = zero ? 0.0f : acc[i + r / 4][j][r % 4];
        if (p.g.splits > 1) {
          store8(p.part, DENDSN_IO_F32, (int64_t(this_split) * p.g.M + m) * N + n, n, N, v);
          continue;
        }
        if (p.add) {
#pragma unroll
          for (int r = 0; r < 8; ++r)
            if (n + r < N) v[r] += p.part[m * N + n + r];
        }
        if (p.keep) {
          store8(p.part, DENDSN_IO_F32, m * N + n, n, N, v);
        } else {
#pragma unroll
          for (int r = 0; r < 8; ++r) v[r] = v[r] == 0.0f ? 0.0f : unit * v[r];
          store8(p.out, p.io, m * p.ld + n, n, N, v);
        }
      }
    }
    if (id >= units) break;
  }
}

// The splits of a product joined, in their order.  Bound by memory (4096 x 1024 of 4 parts
// 14 us), most of it in cache.
struct JoinArgs {
  const float *part, *unit;
  void* out;
  int64_t M, N, ld;
  float scale;
  int splits, io;
};

// VEC: values of a thread (4 where N is a multiple of it).  U: loads in flight, 16 of many
// splits (256 of 8 x 512: 13 us, with 8 17; but 3 of 10000 x 512 20 against 15).
template <int VEC, int U>
__global__ void __launch_bounds__(kThreads) ce_join_splits_kernel(JoinArgs p) {
  const int64_t at = (int64_t(blockIdx.x) * kThreads + threadIdx.x) * VEC;
  if (at >= p.M * p.N) return;
  const float unit = p.unit ? *p.unit * p.scale : p.scale;
  const float* from = p.part + at;
  float s[VEC] = {};
  for (int k0 = 0; k0 < p.splits; k0 += U) {
    Pack<float, VEC> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      v[u] = *reinterpret_cast<const Pack<float, VEC>*>(from + int64_t(min(k0 + u, p.splits - 1)) * p.M * p.N);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (k0 + u < p.splits)
#pragma unroll
        for (int e = 0; e < VEC; ++e) s[e] += v[u].v[e];
  }
  const int64_t to = at / p.N * p.ld + at % p.N;
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const float g = s[e] == 0.0f ? 0.0f : unit * s[e];
    if (p.io == DENDSN_IO_BF16) static_cast<uint16_t*>(p.out)[to + e] = bf16_bits(g);
    else static_cast<float*>(p.out)[to + e] = g;
  }
}

// ---------------------------------------------------------------------------
// Rows
// ---------------------------------------------------------------------------
struct LossArgs {
  const float2* stats;
  const float* z;       // kept logits, or
  const float* chosen;  // the target's
  const void* targets;
  float *loss, *lse;
  float2* norm;         // [M] what the gradient reads: what exponentials are taken from, one over their sum (or NULL)
  int64_t M, zrows, V;
  float scale;
  int tiles, wide;
};

// A wave a row: joins the tiles' statistics (8192 rows of 500: 19 us).  The gradient gets the
// maximum and the sum apart, and the loss its difference from the maximum first: in lse, their sum,
// logits of 4e4 leave the probabilities 0.2 % of their own rounding.
__global__ void __launch_bounds__(kThreads) ce_loss_kernel(LossArgs p) {
  const int lane = threadIdx.x & 63;
  const int64_t m = int64_t(blockIdx.x) * (kThreads / 64) + (threadIdx.x >> 6);
  if (m >= p.M) return;
  const int64_t t = target_of(p.targets, p.wide, m);
  const bool keep = t >= 0 && t < p.V;
  float top = -INFINITY;
  for (int i = lane; i < p.tiles; i += 64) top = fmaxf(top, p.stats[m * p.tiles + i].x);
#pragma unroll
  for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  const float ref = anchor(top);
  float sum = 0.0f;
  for (int i = lane; i < p.tiles; i += 64) {
    const float2 s = p.stats[m * p.tiles + i];
    sum += s.y * exp_diff(s.x, ref);  // (a tile at minus infinity: 0 times 0)
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) {
    const float log_sum = logf(sum);
    const float z = !keep ? 0.0f : p.scale * (p.z ? p.z[(t / kStep * p.zrows + m) * kStep + t % kStep] : p.chosen[m]);
    p.loss[m] = keep ? (ref - z) + log_sum : 0.0f;
    if (p.lse) p.lse[m] = keep ? ref + log_sum : 0.0f;
    if (p.norm) p.norm[m] = make_float2(ref, 1.0f / sum);
  }
}

// The largest weight of a row with a target: dz is formed in its units.  Rows of one
// weight (a mean) would otherwise all carry that number's own rounding to bf16, up to
// 0.4 % the same way in every sum; in units of it they carry none.
struct UnitArgs {
  const float* row_weight;
  const void* targets;
  float* unit;
  int64_t N, V;
  int wide;
};

__global__ void __launch_bounds__(1024) ce_unit_kernel(UnitArgs p) {
  __shared__ float most[16];
  float top = 0.0f;
  for (int64_t i = threadIdx.x; i < p.N; i += 1024) {
    const int64_t t = target_of(p.targets, p.wide, i);
    if (t >= 0 && t < p.V) top = fmaxf(top, fabsf(p.row_weight[i]));
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  if (threadIdx.x % 64 == 0) most[threadIdx.x / 64] = top;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int q = 1; q < 16; ++q) top = fmaxf(top, most[q]);
    *p.unit = top > 0.0f && top < INFINITY ? top : 1.0f;
  }
}

struct DzArgs {
  const float *z, *row_weight, *unit;
  const float2* norm;  // as LossArgs
  const void* targets;
  uint16_t* dz;
  int64_t M, rows, blocks, plane, V;  // rows of a panel; blocks along the rows
  int64_t ld;                         // dz: elements between rows of a panel
  float scale;
  int wide, planes;
};

constexpr int kDzRows = 128;  // rows of a block, of one panel

// dz = (r / unit) (softmax(s z) - onehot); +0 in rows without a target, past V, and in the
// rows past M that the last stage of dW's sum reads.  In bf16 dz takes the place of the
// logits (ld = 128: the first half of each row's 64 fp32): the eight lanes that write a
// row are those that have read it, in one wave.  Bound by memory: 5.2 TB/s.
__global__ void __launch_bounds__(kThreads) ce_dz_kernel(DzArgs p) {
  const int64_t panel = blockIdx.x / p.blocks, r0 = blockIdx.x % p.blocks * kDzRows;
  const int64_t v0 = panel * kStep + threadIdx.x % 8 * 8;
#pragma unroll
  for (int it = 0; it < kDzRows / 32; ++it) {
    const int64_t m = r0 + it * 32 + threadIdx.x / 8;
    if (m >= round_up(p.M, kStep)) return;
    const int64_t t = m < p.M ? target_of(p.targets, p.wide, m) : -1;
    const bool keep = t >= 0 && t < p.V;
    const float c = keep && p.row_weight ? p.row_weight[m] / *p.unit : 1.0f;
    const float2 norm = keep ? p.norm[m] : make_float2(0.0f, 0.0f);
    const int64_t row = panel * p.rows + m, at = row * p.ld + threadIdx.x % 8 * 8;
    const f32x4* z = reinterpret_cast<const f32x4*>(p.z + row * kStep + threadIdx.x % 8 * 8);
    const f32x4 za = __builtin_nontemporal_load(z), zb = __builtin_nontemporal_load(z + 1);
    uint16_t a[8], f, b[8], d[8];  // (dz is finite wherever the loss is: no copy)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float zk = k < 4 ? za[k & 3] : zb[k & 3];
      float g = 0.0f;
      if (keep && v0 + k < p.V) {
        g = exp_diff(p.scale * zk, norm.x) * norm.y;
        if (v0 + k == t) g -= 1.0f;
        g *= c;
      }
      if (p.planes == 1) a[k] = bf16_bits(g);
      else split3(g, a[k], f, b[k], d[k]);
    }
    store8(p.dz + at, a);
    if (p.planes == 3) store8(p.dz + p.plane + at, b), store8(p.dz + 2 * p.plane + at, d);
  }
}

// Both gradients of few rows in fp32: the weights are read, and their gradient written, once.
struct FewArgs {
  const void *h, *w, *targets;
  const float *z, *row_weight;
  const float2* norm;  // as LossArgs
  float *part, *gw;  // dH: [gridDim.y][M][D], without the scale
  int64_t ldh, ldw, ldg, M, V, D, zrows, panels, each;  // each: panels of a block
  float scale;
  int wide;
};

// A block takes a run of panels of 64 classes by 256 features, a wave 64 of them, four
// neighbours a lane.  The panel's dz is formed in LDS; a wave's sixteen classes of weights
// enter its sums for dH (over the classes: k is a class), and meet the rows of hidden, MF
// times sixteen, that stay in registers (k is a row) for their own gradient, which is
// written at once.  Bound by the weights' bytes and, from 32 rows on, by the fp32 matrix
// instructions.  50000 classes, 512 features: 8 rows 38 us (205 MB, 5.4 TB/s), 32 rows 58,
// 64 rows 130 (50 TF; a block a CU, for its registers); as planes laid out and three
// products of tiles 220, 210 and 220.  More rows go through the tiles.
template <int MF>
__global__ void __launch_bounds__(256, MF == 4 ? 1 : 2) ce_few_grad_kernel(FewArgs p) {
  __shared__ float dz[16 * MF][kStep + 4];  // (rows four banks apart)
  const int tid = threadIdx.x, lane = tid & 63, w = scalar(tid >> 6), i = lane & 15, q = lane >> 4;
  const int64_t d = int64_t(blockIdx.x) * 256 + w * 64 + 4 * i;
  const bool on = d < p.D;  // (and then all four)
  auto keeps = [&](int64_t m) {
    const int64_t t = m < p.M ? target_of(p.targets, p.wide, m) : -1;
    return t >= 0 && t < p.V;
  };
  f32x4 hf[4 * MF], acc[MF][4];
#pragma unroll
  for (int s = 0; s < 4 * MF; ++s) {
    const int64_t m = 4 * s + q;
    hf[s] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (on && keeps(m)) hf[s] = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.h) + m * p.ldh + d);
  }
#pragma unroll
  for (int f = 0; f < MF; ++f)
#pragma unroll
    for (int c = 0; c < 4; ++c) acc[f][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int64_t k0 = blockIdx.y * p.each, k1 = min(k0 + p.each, p.panels);
  const int64_t end = min(k1 * kStep, p.V);
  f32x4 wf[2][4];  // sixteen classes, and those after them
  auto fetch = [&](f32x4 (&to)[4], int64_t v0) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int64_t v = v0 + 4 * t + q;
      to[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if (on && v < end) to[t] = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.w) + v * p.ldw + d);
    }
  };
  fetch(wf[0], k0 * kStep);
  for (int64_t k = k0; k < k1; ++k) {
    const int64_t v0 = k * kStep;
    __syncthreads();  // (the last panel's dz is read)
#pragma unroll
    for (int f = 0; f < MF; ++f) {
      const int64_t m = 16 * f + tid / 16, v = v0 + tid % 16 * 4;
      const int64_t t = m < p.M ? target_of(p.targets, p.wide, m) : -1;
      f32x4 g{0.0f, 0.0f, 0.0f, 0.0f};
      if (t >= 0 && t < p.V) {
        const f32x4 z = *reinterpret_cast<const f32x4*>(p.z + (k * p.zrows + m) * kStep + tid % 16 * 4);
        const float2 norm = p.norm[m];
        const float r = p.row_weight ? p.row_weight[m] : 1.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (v + e < p.V) g[e] = r * (exp_diff(p.scale * z[e], norm.x) * norm.y - (v + e == t ? 1.0f : 0.0f));
      }
      *reinterpret_cast<f32x4*>(&dz[16 * f + tid / 16][tid % 16 * 4]) = g;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      f32x4 o[4];
      fetch(wf[~u & 1], v0 + 16 * (u + 1));
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int f = 0; f < MF; ++f) {
          const float a = dz[16 * f + i][16 * u + 4 * t + q];
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[f][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, wf[u & 1][t][c], acc[f][c], 0, 0, 0);
        }
#pragma unroll
      for (int s = 0; s < 4 * MF; ++s) {
        const float a = dz[4 * s + q][16 * u + i];
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, hf[s][c], o[c], 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t v = v0 + 16 * u + 4 * q + r;
        f32x4 g;
#pragma unroll
        for (int c = 0; c < 4; ++c) g[c] = o[c][r] == 0.0f ? 0.0f : p.scale * o[c][r];
        if (on && v < p.V) *reinterpret_cast<f32x4_any*>(p.gw + v * p.ldg + d) = g;
      }
      __builtin_amdgcn_sched_barrier(0);  // (no later classes' loads before: the registers do not reach)
    }
  }
#pragma unroll
  for (int f = 0; f < MF; ++f)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t m = 16 * f + 4 * q + r;
      if (!on || m >= p.M) continue;
      f32x4 g{0.0f, 0.0f, 0.0f, 0.0f};
      if (keeps(m)) {
#pragma unroll
        for (int c = 0; c < 4; ++c) g[c] = acc[f][c][r];
      }
      *reinterpret_cast<f32x4*>(p.part + (int64_t(blockIdx.y) * p.M + m) * p.D + d) = g;
    }
}

// The gradient of the weights of no rows.
__global__ void __launch_bounds__(kThreads) ce_zero_kernel(void* out, int64_t rows, int64_t cols, int64_t ld, int io) {
  for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < rows * cols; i += int64_t(gridDim.x) * kThreads) {
    const int64_t at = i / cols * ld + i % cols;
    if (io == DENDSN_IO_BF16) static_cast<uint16_t*>(out)[at] = 0;
    else static_cast<float*>(out)[at] = 0.0f;
  }
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
dendsn_status check_cfg(const dendsn_ce_cfg* c) {
  if (!c) return fail(DENDSN_E_INVALID, "cfg is NULL");
  if (c->N < 0 || c->N > (int64_t(1) << 26)) return fail(DENDSN_E_INVALID, "N must be in [0, 2^26]");
  if (c->V < 1 || c->V > (int64_t(1) << 24)) return fail(DENDSN_E_INVALID, "V must be in [1, 2^24]");
  if (c->D < 1 || c->D > (int64_t(1) << 20)) return fail(DENDSN_E_INVALID, "D must be in [1, 2^20]");
  const int64_t ld[4] = {c->ld_hidden, c->ld_grad_hidden, c->ld_weight, c->ld_grad_weight};
  for (int i = 0; i < 4; ++i) {
    if (ld[i] < c->D) return fail(DENDSN_E_INVALID, "every stride must be >= D");
    if (!small_product(i < 2 ? c->N : c->V, ld[i])) return fail(DENDSN_E_INVALID, "a stride is too large");
  }
  if (c->io != DENDSN_IO_F32 && c->io != DENDSN_IO_BF16) return fail(DENDSN_E_INVALID, "bad io");
  if (c->index != DENDSN_INDEX_I32 && c->index != DENDSN_INDEX_I64) return fail(DENDSN_E_INVALID, "bad index");
  if (!isfinite(c->logit_scale)) return fail(DENDSN_E_INVALID, "logit_scale must be finite");
  return DENDSN_OK;
}

constexpr int kBig = 256;  // tile of a product, both ways
constexpr int64_t kMaxParts = 128;  // of a sum over k

struct Plan {
  int planes;
  int64_t Dp, Vp;      // rows of packed operands, of logits
  int64_t piece, pieces, rows;  // rows: of a panel
  int logits, dh_tile, dw_tile;  // rows of the products' tiles: 256 x 256, 192 x 256, 128 x 128
  int splits, dw_splits;         // of their sums: dH, dW
  int64_t few;                   // panels of a block of ce_few_grad_kernel
  size_t h, w, stats, z, dz, chosen, norm, unit, dh, dw, total;
};

// Rows that can be read in chunks of 16 bytes, near enough for a descriptor.
bool rows16(const dendsn_ce_cfg* c, const void* p, int64_t ld) {
  const int64_t m = c->io == DENDSN_IO_BF16 ? 8 : 4;
  return aligned(p, 16) && c->D % m == 0 && ld % m == 0 && ld <= kMaxLd;
}

// The kernel for few rows, if one is made for these sizes: MF times sixteen rows, U units
// of 64 k a wave, as far as the registers reach.  2048 features, 50001 classes in bf16: 8
// rows 33 us, 32 rows 35 us; the tiles, which split no sum over k, 53 and 41 us (and fp32
// would be laid out in planes first).  With the logits kept for training, 64 rows of 32000
// classes and 1024 features: 19 us against 22; 32 rows of 50000 in fp32: 70 us against 137;
// 32 rows of 5000 classes and 1500 features in fp32: 31 against 107, and 20 of layout.
// launch = false: only says whether.
template <typename IO>
bool launch_score(const ScoreArgs& a, bool launch, unsigned grid, hipStream_t stream) {
  constexpr bool BF = sizeof(IO) == 2;
  const int64_t mf = ceil_div(a.M, 16), u = ceil_div(a.K, kStep * kScoreWaves);
  const dim3 g(grid), b(kScoreWaves * 64);
#define DENDSN_SCORE(MF, U)                                         \
  if (mf <= MF && u <= U) {                                         \
    if (launch) ce_score_kernel<IO, MF, U><<<g, b, 0, stream>>>(a); \
    return true;                                                    \
  }
  DENDSN_SCORE(1, 1) DENDSN_SCORE(1, 2) DENDSN_SCORE(1, 4)
  DENDSN_SCORE(2, 1) DENDSN_SCORE(2, 2)
  DENDSN_SCORE(4, 1)
  if constexpr (BF) {
    DENDSN_SCORE(1, 8) DENDSN_SCORE(2, 4) DENDSN_SCORE(4, 2)
  } else {
    DENDSN_SCORE(2, 3) DENDSN_SCORE(4, 2)
  }
#undef DENDSN_SCORE
  return false;
}

// Which kernels read the operands, by where they lie.
struct Route {
  bool streamed;        // logits of few rows, from one stream over the weights
  bool few_back;        // and their gradients, from another
  bool pack_h, pack_w;  // operands are laid out for the products (bf16 as they lie: by the DMA)
};

Route route_of(const dendsn_ce_cfg* c, bool train, const void* hidden, const void* weight) {
  const bool bf = c->io == DENDSN_IO_BF16, h = rows16(c, hidden, c->ld_hidden), w = rows16(c, weight, c->ld_weight);
  Route r{};
  if (c->N <= 64 && h && w) {
    ScoreArgs a{};
    a.M = c->N;
    a.K = c->D;
    r.streamed = bf ? launch_score<bf16_t>(a, false, 1, nullptr) : launch_score<float>(a, false, 1, nullptr);
    r.few_back = train && !bf;
  }
  const bool products = !r.streamed || (train && !r.few_back);
  r.pack_w = products && !(bf && w);
  r.pack_h = products && !(bf && h && !train);  // (training clears the rows without a target)
  return r;
}

// The tile of a product of M x N.  A CU works through a 256 tile at 0.6 of the time of
// four 128 tiles (its fragments are read from LDS half as often): in units of one 256 tile
// a CU, rounds of 256 tiles against 0.4 a round of 128 tiles.  Measured, 1024 x 10000 x
// 512 in fp32 (160 tiles of 256 or 632 of 128): logits 78 us against 107; dW (80 or 316)
// 138 us against 115.
int tile_for(int64_t M, int64_t N) {
  const int64_t big = ceil_div(ceil_div(M, 256) * ceil_div(N, 256), 256);
  const int64_t small = ceil_div(ceil_div(M, 128) * ceil_div(N, 128), 256);
  return 5 * big <= 2 * small ? 256 : 128;
}

// The logits' tile, whose sum is not split: also 192 x 256, at 0.85 of a 256 tile's time.
// 1024 x 10000 x 512 in fp32 (240 tiles of it, or 160): 71 us against 82; 2048 x 10000 x
// 512 in bf16 (440, or 320) 43 against 50; 4096 x 4000 x 1024 (352, or 256) 58 against 41.
int logits_tile(int64_t M, int64_t V) {
  const int tile = tile_for(M, V);
  const int64_t big = ceil_div(ceil_div(M, 256) * ceil_div(V, 256), 256);
  const int64_t mid = ceil_div(ceil_div(M, 192) * ceil_div(V, 256), 256);
  const int64_t small = ceil_div(ceil_div(M, 128) * ceil_div(V, 128), 256);
  return 85 * mid < (tile == 256 ? 100 * big : 40 * small) ? 192 : tile;
}

// The tile of a gradient's product, and the parts that its sum of `steps` stages is cut
// into, by an estimate in us: a stage of a full chip takes 1.6 in 256 tiles, 0.64 a round of
// 256 tiles of 128 (0.85 where there is one round: nothing shares a CU then); parts are
// written and joined at 4 TB/s, by a launch of 5.  At least eight stages a part.  Measured,
// the kernel and the join: dW of 1024 rows, 10000 x 512 in fp32 in three parts 85, whole (128
// tiles) 110; of 8192 rows, 1000 x 256 in bf16 28 and 93; dH of 64 rows, 32000 x 1024 in bf16
// in 32 parts of 128 tiles 32; of 4096 in four of 256 254.
struct Split {
  int tile, parts;
};

Split split_of(int64_t M, int64_t N, int64_t steps, bool whole) {
  Split best{};
  double least = 0.0;
  for (int tile : {256, 128}) {
    const int64_t tiles = ceil_div(M, tile) * ceil_div(N, tile);
    for (int64_t fill : {0, 256, 512}) {  // blocks
      int64_t parts = fill / tiles;
      if (parts > kMaxParts) parts = kMaxParts;
      if (parts > steps / 8) parts = steps / 8;
      if (parts < 1 || whole) parts = 1;
      const int64_t each = ceil_div(steps, parts), rounds = ceil_div(tiles * parts, 256);
      parts = ceil_div(steps, each);
      double us = double(each) * (tile == 256 ? 1.6 * double(rounds) : rounds == 1 ? 0.85 : 0.64 * double(rounds));
      if (parts > 1) us += double(2 * parts + 1) * double(M) * double(N) * 1e-6 + 5.0;
      if (!best.tile || us < least) best = Split{tile, int(parts)}, least = us;
    }
  }
  return best;
}

// Of a route, or of all that the operands' places may lead to.
Plan make_plan(const dendsn_ce_cfg* c, bool train, const Route* r) {
  Plan p{};
  p.planes = c->io == DENDSN_IO_BF16 ? 1 : 3;
  p.Dp = round_up(c->D, kStep);
  p.Vp = round_up(c->V, kStep);
  // a row's logits, with their gradient in their place (fp32: beside them, in planes)
  const int64_t logits_row = train ? p.Vp * (p.planes == 1 ? 4 : 10) : ceil_div(c->V, 64) * 8;
  const int64_t packed_row = p.Dp * (p.planes == 1 ? 2 : 8);
  const int64_t per_row = logits_row > packed_row ? logits_row : packed_row;
  int64_t most = kPieceBytes / per_row / kBig * kBig;
  if (most < kBig) most = kBig;
  if (most > kMaxPanelRows) most = kMaxPanelRows;
  const int64_t N = c->N > 0 ? c->N : 1;
  p.pieces = ceil_div(N, most);
  p.piece = p.pieces > 1 ? round_up(ceil_div(N, p.pieces), kBig) : N;
  p.pieces = ceil_div(N, p.piece);
  p.logits = logits_tile(p.piece, c->V);
  p.rows = round_up(p.piece, kBig);
  if (p.logits == 192) p.rows = round_up(p.piece, 192) > p.rows ? round_up(p.piece, 192) : p.rows;
  Carve cv;
  if (!r || r->pack_h) p.h = cv.take(size_t(p.planes == 3 ? 4 : 1) * size_t(p.piece) * size_t(p.Dp) * 2);
  if (!r || r->pack_w) p.w = cv.take(size_t(p.planes == 3 ? 4 : 1) * size_t(c->V) * size_t(p.Dp) * 2);
  p.stats = cv.take(size_t(p.piece) * size_t(ceil_div(c->V, 64)) * 8);
  p.chosen = cv.take(size_t(p.piece) * 4);
  p.unit = cv.take(4);
  p.splits = 1;
  if (train) {
    p.norm = cv.take(size_t(p.piece) * 8);
    p.z = cv.take(size_t(p.rows) * size_t(p.Vp) * 4);
    p.dz = p.z;
    if (p.planes == 3 && !(r && r->few_back)) p.dz = cv.take(size_t(p.planes) * size_t(p.rows) * size_t(p.Vp) * 2);
    const int64_t planes = p.planes == 3 ? 6 : 1;
    const Split dh = split_of(p.piece, c->D, ceil_div(c->V, kStep) * planes, false);
    const Split dw = split_of(c->V, c->D, ceil_div(p.piece, kStep) * planes, p.pieces > 1);
    p.dh_tile = dh.tile, p.splits = dh.parts;
    p.dw_tile = dw.tile, p.dw_splits = dw.parts;
    int64_t dh_parts = p.splits > 1 && !(r && r->few_back) ? p.splits : 0;
    if (r ? r->few_back : p.planes == 3 && c->N <= 64) {  // two blocks a CU
      const int64_t panels = p.Vp / kStep, columns = ceil_div(c->D, 256);
      const int64_t parts = columns < 512 ? 512 / columns : 1;
      p.few = ceil_div(panels, parts);
      if (ceil_div(panels, p.few) > dh_parts) dh_parts = ceil_div(panels, p.few);
    }
    p.dh = cv.take(size_t(dh_parts) * size_t(p.piece) * size_t(c->D) * 4);
    const int dw_parts = r && r->few_back ? 0 : p.dw_splits > 1 ? p.dw_splits : p.pieces > 1 ? 1 : 0;
    p.dw = cv.take(size_t(dw_parts) * size_t(c->V) * size_t(c->D) * 4);
  }
  p.total = cv.at;
  return p;
}

void finish(GemmArgs& g, int planes, int tile, int splits) {
  g.planes = planes;
  g.tiles_m = int(ceil_div(g.M, tile));
  g.tiles_n = int(ceil_div(g.N, tile == 192 ? 256 : tile));
  g.splits = splits;
  g.per = int(ceil_div(g.K, kStep));
  g.steps = g.per * (planes == 3 ? 6 : 1);
  g.each = (g.steps + splits - 1) / splits;
}

void pack(PackArgs a, bool bf, hipStream_t stream) {
  const int64_t threads = a.rows * (a.cols_p / 8);
  for (a.first = 0; a.first < threads; a.first += kMostThreads) {
    const int64_t n = threads - a.first < kMostThreads ? threads - a.first : kMostThreads;
    const dim3 g(unsigned(ceil_div(n, kThreads))), b(kThreads);
    if (bf) ce_pack_kernel<bf16_t><<<g, b, 0, stream>>>(a);
    else ce_pack_kernel<float><<<g, b, 0, stream>>>(a);
  }
}

// As many blocks as the 256 CUs hold at a time, a multiple of the eight XCDs: a block's
// tiles then stay on its XCD.
unsigned grid_of(const GemmArgs& g, int tile, bool all) {
  const int64_t units = int64_t(g.tiles_m) * g.tiles_n * g.splits, most = tile == 128 ? 512 : 256;
  return unsigned(all || units < most ? units : most);
}

void join_splits(const GradArgs& g, int splits, hipStream_t stream) {
  const JoinArgs j{g.part, g.unit, g.out, g.g.M, g.g.N, g.ld, g.scale, splits, g.io};
  const bool four = j.N % 4 == 0;
  const dim3 grid(unsigned(ceil_div(j.M * j.N, kThreads * (four ? 4 : 1)))), b(kThreads);
  if (splits > 32) {
    if (four) ce_join_splits_kernel<4, 16><<<grid, b, 0, stream>>>(j);
    else ce_join_splits_kernel<1, 16><<<grid, b, 0, stream>>>(j);
  } else if (four) {
    ce_join_splits_kernel<4, 8><<<grid, b, 0, stream>>>(j);
  } else {
    ce_join_splits_kernel<1, 8><<<grid, b, 0, stream>>>(j);
  }
}

dendsn_status run(const dendsn_ce_cfg* c, bool train, const void* hidden, const void* weight, const void* targets,
                  const float* row_weight, float* loss, float* lse, void* grad_hidden, void* grad_weight,
                  char* ws, const Route& route, const Plan& p, hipStream_t stream) {
  const size_t esz = c->io == DENDSN_IO_BF16 ? 2 : 4;
  const int wide = c->index == DENDSN_INDEX_I64;
  const size_t isz = wide ? 8 : 4;
  const bool bf = c->io == DENDSN_IO_BF16;
  // Few rows: at most as many blocks as there is room for statistics, a CU each.
  const unsigned blocks = unsigned(ceil_div(c->V, kStep) < 256 ? ceil_div(c->V, kStep) : 256);
  if (route.streamed) {
    const ScoreArgs a{hidden, weight, targets, reinterpret_cast<float2*>(ws + p.stats),
                      train ? nullptr : reinterpret_cast<float*>(ws + p.chosen),
                      train ? reinterpret_cast<float*>(ws + p.z) : nullptr,
                      c->ld_hidden, c->ld_weight, c->N, c->V, c->D, p.rows, c->logit_scale, wide};
    if (bf) launch_score<bf16_t>(a, true, blocks, stream);
    else launch_score<float>(a, true, blocks, stream);
  }
  Operand w{static_cast<const uint16_t*>(weight), c->ld_weight, 0, 0, c->V, c->D};  // (bf16, where a product reads it)
  if (route.pack_w) {
    PackArgs a{weight, reinterpret_cast<uint16_t*>(ws + p.w), nullptr, c->V, c->D, c->ld_weight, p.Dp, c->V * p.Dp, c->V, wide, p.planes};
    pack(a, bf, stream);
    w = Operand{a.dst, p.Dp, a.plane, kFinite * a.plane, c->V, p.Dp};
  }
  float* unit = nullptr;
  if (train && row_weight && !route.few_back) {
    unit = reinterpret_cast<float*>(ws + p.unit);
    ce_unit_kernel<<<dim3(1), dim3(1024), 0, stream>>>(UnitArgs{row_weight, targets, unit, c->N, c->V, wide});
  }
  for (int64_t r0 = 0; r0 < c->N; r0 += p.piece) {
    const int64_t M = c->N - r0 < p.piece ? c->N - r0 : p.piece;
    const void* hp = static_cast<const char*>(hidden) + size_t(r0) * size_t(c->ld_hidden) * esz;
    const void* tp = static_cast<const char*>(targets) + size_t(r0) * isz;
    Operand h{static_cast<const uint16_t*>(hp), c->ld_hidden, 0, 0, M, c->D};  // (as w)
    if (route.pack_h) {
      PackArgs a{hp, reinterpret_cast<uint16_t*>(ws + p.h), tp, M, c->D, c->ld_hidden, p.Dp, M * p.Dp, c->V, wide, p.planes};
      pack(a, bf, stream);
      h = Operand{a.dst, p.Dp, a.plane, kFinite * a.plane, M, p.Dp};
    }
    LogitArgs l{};
    l.g.x = h; l.g.y = w;
    l.g.M = M; l.g.N = c->V; l.g.K = c->D;
    finish(l.g, p.planes, p.logits, 1);
    l.scale = c->logit_scale;
    l.stats = reinterpret_cast<float2*>(ws + p.stats);
    l.z = train ? reinterpret_cast<float*>(ws + p.z) : nullptr;
    l.chosen = train ? nullptr : reinterpret_cast<float*>(ws + p.chosen);
    l.targets = tp; l.zrows = p.rows; l.zcols = p.Vp; l.wide = wide;
    const dim3 lg(grid_of(l.g, p.logits, train));
    if (route.streamed) l.g.tiles_n = int(blocks);
    else if (p.logits == 256) ce_logits_kernel<256, 256, 2, 4><<<lg, dim3(512), 0, stream>>>(l);
    else if (p.logits == 192) ce_logits_kernel<192, 256, 2, 4><<<lg, dim3(512), 0, stream>>>(l);
    else ce_logits_kernel<128, 128, 2, 2><<<lg, dim3(256), 0, stream>>>(l);

    LossArgs s{};
    s.stats = l.stats; s.z = l.z; s.chosen = l.chosen; s.targets = tp;
    s.loss = loss + r0;
    s.lse = lse ? lse + r0 : nullptr;
    s.norm = train ? reinterpret_cast<float2*>(ws + p.norm) : nullptr;
    s.M = M; s.zrows = p.rows; s.V = c->V; s.scale = c->logit_scale; s.tiles = l.g.tiles_n; s.wide = wide;
    ce_loss_kernel<<<dim3(unsigned(ceil_div(M, kThreads / 64))), dim3(kThreads), 0, stream>>>(s);
    if (!train) continue;
    if (route.few_back) {
      FewArgs a{hidden, weight, targets, l.z, row_weight, s.norm, reinterpret_cast<float*>(ws + p.dh), static_cast<float*>(grad_weight),
                c->ld_hidden, c->ld_weight, c->ld_grad_weight, M, c->V, c->D, p.rows, p.Vp / kStep, p.few, c->logit_scale, wide};
      const dim3 grid(unsigned(ceil_div(c->D, 256)), unsigned(ceil_div(a.panels, a.each))), b(256);
      if (M <= 16) ce_few_grad_kernel<1><<<grid, b, 0, stream>>>(a);
      else if (M <= 32) ce_few_grad_kernel<2><<<grid, b, 0, stream>>>(a);
      else ce_few_grad_kernel<4><<<grid, b, 0, stream>>>(a);
      GradArgs g{};
      g.g.M = M; g.g.N = c->D;
      g.out = grad_hidden; g.part = a.part; g.scale = c->logit_scale; g.ld = c->ld_grad_hidden; g.io = c->io;
      join_splits(g, int(grid.y), stream);
      continue;
    }

    DzArgs z{};
    z.z = l.z; z.norm = s.norm; z.row_weight = row_weight ? row_weight + r0 : nullptr;
    z.unit = unit; z.targets = tp;
    z.dz = reinterpret_cast<uint16_t*>(ws + p.dz);
    z.M = M; z.rows = p.rows; z.blocks = ceil_div(round_up(M, kStep), kDzRows);
    z.ld = p.planes == 1 ? 2 * kStep : kStep; z.plane = p.rows * p.Vp; z.V = c->V; z.scale = c->logit_scale; z.wide = wide; z.planes = p.planes;
    ce_dz_kernel<<<dim3(unsigned(z.blocks * (p.Vp / kStep))), dim3(kThreads), 0, stream>>>(z);

    GradArgs gh{};
    gh.g.x = Operand{z.dz, z.ld, z.plane, 0, M, p.Vp, p.rows};
    gh.g.y = w;
    gh.g.M = M; gh.g.N = c->D; gh.g.K = c->V;
    finish(gh.g, p.planes, p.dh_tile, p.splits);
    gh.out = static_cast<char*>(grad_hidden) + size_t(r0) * size_t(c->ld_grad_hidden) * esz;
    gh.part = reinterpret_cast<float*>(ws + p.dh);
    gh.unit = unit; gh.scale = c->logit_scale;
    gh.targets = tp; gh.ld = c->ld_grad_hidden; gh.V = c->V; gh.wide = wide; gh.io = c->io;
    const dim3 hg(grid_of(gh.g, p.dh_tile, false));
    if (p.dh_tile == 256) ce_grad_kernel<256, 256, 2, 4, false><<<hg, dim3(512), 0, stream>>>(gh);
    else ce_grad_kernel<128, 128, 2, 2, false><<<hg, dim3(256), 0, stream>>>(gh);
    if (p.splits > 1) join_splits(gh, p.splits, stream);

    GradArgs gw{};
    gw.g.x = Operand{z.dz, z.ld, z.plane, 0, M, p.Vp, p.rows};
    gw.g.y = h;
    gw.g.M = c->V; gw.g.N = c->D; gw.g.K = M;
    finish(gw.g, p.planes, p.dw_tile, p.dw_splits);
    gw.unit = unit; gw.scale = c->logit_scale;
    gw.out = grad_weight; gw.ld = c->ld_grad_weight; gw.io = c->io;
    gw.part = reinterpret_cast<float*>(ws + p.dw);
    gw.add = r0 > 0; gw.keep = r0 + M < c->N;
    const dim3 wg(grid_of(gw.g, p.dw_tile, false));
    if (p.dw_tile == 256) ce_grad_kernel<256, 256, 2, 4, true><<<wg, dim3(512), 0, stream>>>(gw);
    else ce_grad_kernel<128, 128, 2, 2, true><<<wg, dim3(256), 0, stream>>>(gw);
    if (p.dw_splits > 1) join_splits(gw, p.dw_splits, stream);
  }
  return launched("linear cross entropy");
}

dendsn_status check_args(const dendsn_ce_cfg* c, const void* hidden, const void* weight, const void* targets,
                         const float* loss, const float* lse) {
  const size_t isz = c->index == DENDSN_INDEX_I64 ? 8 : 4, esz = c->io == DENDSN_IO_BF16 ? 2 : 4;
  if (c->N > 0 && (!hidden || !targets || !loss)) return fail(DENDSN_E_INVALID, "hidden, targets or loss is NULL");
  if (!weight) return fail(DENDSN_E_INVALID, "weight is NULL");
  if (!aligned(hidden, esz) || !aligned(weight, esz) || !aligned(targets, isz) || !aligned(loss, 4) || !aligned(lse, 4))
    return fail(DENDSN_E_INVALID, "hidden, weight, targets, loss or lse misaligned");
  return DENDSN_OK;
}

}  // namespace
}  // namespace dendsn_seq

using namespace dendsn_seq;

extern "C" {

dendsn_status dendsn_ce_workspace_bytes(const dendsn_ce_cfg* cfg, int32_t train, size_t* bytes) {
  clear_error();
  const dendsn_status st = check_cfg(cfg);
  if (st != DENDSN_OK) return st;
  if (!bytes) return fail(DENDSN_E_INVALID, "bytes is NULL");
  *bytes = make_plan(cfg, train != 0, nullptr).total;
  return DENDSN_OK;
}

dendsn_status dendsn_ce_workspace_bytes_at(const dendsn_ce_cfg* cfg, int32_t train, const void* hidden,
                                           const void* weight, size_t* bytes) {
  clear_error();
  const dendsn_status st = check_cfg(cfg);
  if (st != DENDSN_OK) return st;
  if (!bytes) return fail(DENDSN_E_INVALID, "bytes is NULL");
  const Route r = route_of(cfg, train != 0, hidden, weight);
  *bytes = make_plan(cfg, train != 0, &r).total;
  return DENDSN_OK;
}

dendsn_status dendsn_ce_forward(const dendsn_ce_cfg* cfg, const void* hidden, const void* weight,
                                const void* targets, float* loss, float* lse, void* workspace,
                                size_t workspace_bytes, hipStream_t stream) {
  clear_error();
  dendsn_status st = check_cfg(cfg);
  if (st == DENDSN_OK) st = check_args(cfg, hidden, weight, targets, loss, lse);
  if (st != DENDSN_OK) return st;
  const Route r = route_of(cfg, false, hidden, weight);
  const Plan p = make_plan(cfg, false, &r);
  st = check_workspace(workspace, workspace_bytes, p.total, "dendsn_ce_workspace_bytes_at");
  if (st != DENDSN_OK || cfg->N == 0) return st;
  return run(cfg, false, hidden, weight, targets, nullptr, loss, lse, nullptr, nullptr, static_cast<char*>(workspace),
             r, p, stream);
}

dendsn_status dendsn_ce_train(const dendsn_ce_cfg* cfg, const void* hidden, const void* weight,
                              const void* targets, const float* row_weight, float* loss, float* lse,
                              void* grad_hidden, void* grad_weight, void* workspace, size_t workspace_bytes,
                              hipStream_t stream) {
  clear_error();
  dendsn_status st = check_cfg(cfg);
  if (st == DENDSN_OK) st = check_args(cfg, hidden, weight, targets, loss, lse);
  if (st != DENDSN_OK) return st;
  const size_t esz = cfg->io == DENDSN_IO_BF16 ? 2 : 4;
  if ((cfg->N > 0 && !grad_hidden) || !grad_weight) return fail(DENDSN_E_INVALID, "grad_hidden or grad_weight is NULL");
  if (!aligned(grad_hidden, esz) || !aligned(grad_weight, esz) || !aligned(row_weight, 4))
    return fail(DENDSN_E_INVALID, "grad_hidden, grad_weight or row_weight misaligned");
  const Route r = route_of(cfg, true, hidden, weight);
  const Plan p = make_plan(cfg, true, &r);
  st = check_workspace(workspace, workspace_bytes, p.total, "dendsn_ce_workspace_bytes_at");
  if (st != DENDSN_OK) return st;
  if (cfg->N == 0) {
    const int64_t blocks = ceil_div(cfg->V * cfg->D, kThreads);
    ce_zero_kernel<<<dim3(unsigned(blocks < 4096 ? blocks : 4096)), dim3(kThreads), 0, stream>>>(grad_weight, cfg->V, cfg->D, cfg->ld_grad_weight, cfg->io);
    return launched("linear cross entropy");
  }
  return run(cfg, true, hidden, weight, targets, row_weight, loss, lse, grad_hidden, grad_weight,
             static_cast<char*>(workspace), r, p, stream);
}

}  // extern "C"
