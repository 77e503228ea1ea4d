// bf16 matrix products for gfx950: C[m, n] = sum over k of X[m, k] Y[n, k], fp32 sums.
//
// Each operand lies in memory either with k adjacent ("K rows": X[m][k]) or with
// its other index adjacent ("K columns": X[k][m]); both are staged in LDS as they
// lie, by LDS-DMA of 16 bytes a lane, two stages deep, and reach the matrix
// instructions through 16-byte reads or, for K columns, transposing reads.  The
// 16-byte chunks of a stage are permuted so that neither kind of read meets a bank
// twice: the DMA writes LDS linearly, so each lane fetches the chunk that belongs at
// its place.  Buffer descriptors bound every access: rows, columns and k past an
// operand's end read as zero.
//
// fp32 operands come as three bf16 planes that add up to them exactly (8 bits of
// the significand each); the six products of planes that matter at fp32 precision
// (those of at most two steps down) run as one longer sum over k.  The products with a
// lower plane take the first plane from a copy without infinities: a lower plane is
// often 0, and 0 times infinity is no part of the sum.
#pragma once

#include "seq_common.h"

namespace dendsn_seq {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __amdgpu_buffer_rsrc_t rsrc_t;
typedef __attribute__((address_space(3))) void lds_void_t;

constexpr int kStep = 64;   // k of a stage
constexpr int kFinite = 3;  // the first plane without infinities, as a plane's number

struct Operand {
  const uint16_t* p;
  int64_t ld;      // elements between rows as they lie
  int64_t plane;   // elements between planes
  int64_t finite;  // elements from the first plane to its copy without infinities
  int64_t rows, cols;  // as they lie
};

struct GemmArgs {
  Operand x, y;
  int64_t M, N, K;
  int planes;       // 1 or 3
  int tiles_m, tiles_n;
  int splits;       // blocks along k of a tile
  int64_t steps;    // stages of the whole sum
};

// Rows of an operand may be this far apart: 256 of them lie within a descriptor.
constexpr int64_t kMaxLd = int64_t(1) << 21;

__device__ __forceinline__ void dma16(rsrc_t r, uint32_t off, void* lds) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_t*)lds, 16, off, 0, 0, 0);
}

// A barrier that leaves loads in flight; no memory access of the program moves across it.
__device__ __forceinline__ void block_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// One operand's side of a block: R rows (K rows) or columns (K columns) of its stage.
template <int R, int NW, bool KCOL>
struct Side {
  static constexpr int kBytes = R * kStep * 2;
  static constexpr int kLoads = kBytes / (1024 * NW);  // DMA instructions of a wave
  static_assert(kLoads >= 1 && kBytes % (1024 * NW) == 0, "a stage is whole DMA instructions");
  static constexpr int kRowBytes = KCOL ? R * 2 : kStep * 2;

  const char* base;
  int64_t left;          // bytes from base to the operand's end
  int64_t ldb;           // bytes between rows
  int64_t plane, finite; // bytes between planes, and to the copy of the first one
  int64_t per_step;      // bytes from stage to stage
  uint32_t off[kLoads];
  uint32_t tail;         // bit i: load i of a K-rows stage reads past the last k in the last step

  __device__ __forceinline__ void init(const Operand& o, int64_t r0, int w, int lane) {
    ldb = o.ld * 2;
    plane = o.plane * 2;
    finite = o.finite * 2;
    const int64_t at = KCOL ? r0 * 2 : r0 * ldb;
    base = reinterpret_cast<const char*>(o.p) + at;
    left = ((o.rows - 1) * o.ld + o.cols) * 2 - at;
    per_step = KCOL ? kStep * ldb : kStep * 2;
    tail = 0;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int b = (w * kLoads + i) * 1024 + lane * 16;
      const int row = b / kRowBytes, chunk = b % kRowBytes / 16;
      const int logical = chunk ^ swizzle(row);
      off[i] = uint32_t(row * ldb) + logical * 16;
      if (!KCOL && logical * 8 >= int((o.cols - 1) % kStep + 1)) tail |= 1u << i;
    }
  }
  static __device__ __forceinline__ int swizzle(int row) {
    return KCOL ? 2 * ((row & 3) | ((row >> 3) & 1) << 2) : row & 7;
  }
  // The stage of step `step` of plane `pl` (kFinite: of the first one's copy); `last`: the
  // last step of a plane's k.
  __device__ __forceinline__ void fetch(char* lds, int pl, int64_t step, bool last, int w) const {
    const int64_t skip = (pl == kFinite ? finite : pl * plane) + step * per_step;
    int64_t n = left - step * per_step;
    n = n < 0 ? 0 : n > 0x7FFFFFF0 ? 0x7FFFFFF0 : n;
    const rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base + skip), 0, int(n), 0x00020000);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      uint32_t o = off[i];
      if (!KCOL && last && (tail >> i & 1)) o = 0x80000000u;
      dma16(r, o, lds + (w * kLoads + i) * 1024);
    }
  }
};

// A lane's addresses of its fragments in a stage: rows (or columns) r0 + 16 f + (lane & 15),
// k = 32 s + 8 (lane >> 4) .. + 7.
template <int R, int F, bool KCOL>
struct Frags {
  uint32_t at[KCOL ? F : 2];
  __device__ __forceinline__ void init(int r0, int lane) {
    const int q = lane >> 4, i = lane & 15;
    if (KCOL) {
      const int k = q * 8 + (i >> 2);
      const int fp = (i >> 2) | (q & 1) << 2;
#pragma unroll
      for (int f = 0; f < F; ++f) at[f] = k * (R * 2) + ((r0 / 16 + f) ^ fp) * 32 + (i & 3) * 8;
    } else {
#pragma unroll
      for (int s = 0; s < 2; ++s) at[s] = (r0 + i) * (kStep * 2) + (((s * 4 + q) ^ (i & 7)) * 16);
    }
  }
  __device__ __forceinline__ bf16x8 read(const char* lds, int f, int s) const {
    if (KCOL) {
      const char* p = lds + at[f] + s * (32 * R * 2);
      typedef __attribute__((address_space(3))) s16x4* ptr;
      const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(p));
      const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(p + 4 * R * 2));
      typedef short s16x8 __attribute__((ext_vector_type(8)));
      const s16x8 v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
      return __builtin_bit_cast(bf16x8, v);
    }
    return *reinterpret_cast<const bf16x8*>(lds + at[s] + f * (16 * kStep * 2));
  }
};

// Which tile a block works on: neighbours along the launch order go to the eight
// XCDs in turn, so each XCD takes a contiguous run of tiles, in groups of eight
// rows of tiles (the run's operands then fit its L2).
__device__ __forceinline__ void tile_of(const GemmArgs& g, int64_t id, int& tm, int& tn) {
  constexpr int kXcd = 8, kGroup = 8;
  const int64_t tiles = int64_t(g.tiles_m) * g.tiles_n;
  const int64_t q = tiles / kXcd, rem = tiles % kXcd;
  const int64_t x = id % kXcd, k = id / kXcd;
  const int64_t t = x * q + (x < rem ? x : rem) + k;
  const int64_t width = int64_t(kGroup) * g.tiles_n;
  const int64_t grp = t / width;
  const int first = int(grp) * kGroup;
  const int size = g.tiles_m - first < kGroup ? g.tiles_m - first : kGroup;
  const int64_t in = t - grp * width;
  tm = first + int(in % size);
  tn = int(in / size);
}

// The planes of the s-th product of an fp32 pair, smallest first.
__device__ __forceinline__ void planes_of(int s, int& px, int& py) {
  constexpr uint32_t xs = 0x031132, ys = 0x013123;  // (2,F) (F,2) (1,1) (1,F) (F,1) (0,0)
  px = xs >> (4 * s) & 15;
  py = ys >> (4 * s) & 15;
}

// The product of one tile.  acc[i][j]: lane l holds rows m = 16 j + (l & 15) and
// columns n = 16 i + 4 (l >> 4) + 0..3 of the wave's tile.
template <int BM, int BN, int WM, int WN, bool XCOL, bool YCOL>
struct Gemm {
  static constexpr int NW = WM * WN, TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
  using SX = Side<BM, NW, XCOL>;
  using SY = Side<BN, NW, YCOL>;
  static constexpr int kStage = SX::kBytes + SY::kBytes;

  static __device__ __forceinline__ void run(const GemmArgs& g, char* lds, int tm, int tn, int split,
                                             f32x4 (&acc)[FN][FM]) {
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = w / WN, wn = w % WN;
    SX sx;
    SY sy;
    sx.init(g.x, int64_t(tm) * BM, w, lane);
    sy.init(g.y, int64_t(tn) * BN, w, lane);
    Frags<BM, FM, XCOL> fx;
    Frags<BN, FN, YCOL> fy;
    fx.init(wm * TM, lane);
    fy.init(wn * TN, lane);
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
      for (int j = 0; j < FM; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const int64_t per = ceil_div(g.K, kStep);  // stages of one product of planes
    const int64_t each = ceil_div(g.steps, g.splits);
    const int64_t s0 = split * each, s1 = s0 + each < g.steps ? s0 + each : g.steps;
    int prod = int(s0 / per);
    int64_t k = s0 % per;
    auto fetch = [&](char* to) {
      int px = 0, py = 0;
      if (g.planes == 3) planes_of(prod, px, py);
      sx.fetch(to, px, k, k == per - 1, w);
      sy.fetch(to + SX::kBytes, py, k, k == per - 1, w);
      if (++k == per) k = 0, ++prod;
    };
    if (s0 < s1) fetch(lds);
    for (int64_t s = s0; s < s1; ++s) {
      const int buf = int(s - s0) & 1;
      // this wave's part of the stage is there (vmcnt 0) and its reads of the other one are
      // done (lgkmcnt 0); past the barrier, so are every wave's
      __builtin_amdgcn_s_waitcnt(0x0070);
      block_barrier();
      if (s + 1 < s1) fetch(lds + (buf ^ 1) * kStage);
      const char* cx = lds + buf * kStage;
      const char* cy = cx + SX::kBytes;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        bf16x8 xf[FM], yf[FN];
#pragma unroll
        for (int i = 0; i < FN; ++i) yf[i] = fy.read(cy, i, h);
#pragma unroll
        for (int j = 0; j < FM; ++j) xf[j] = fx.read(cx, j, h);
#pragma unroll
        for (int j = 0; j < FM; ++j)
#pragma unroll
          for (int i = 0; i < FN; ++i)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(yf[i], xf[j], acc[i][j], 0, 0, 0);
      }
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt 0: past the barrier, the stages may be reused
    block_barrier();
  }
};

}  // namespace dendsn_seq
