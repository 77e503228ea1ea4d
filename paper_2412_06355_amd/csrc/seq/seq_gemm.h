// bf16 matrix products for gfx950: C[m, n] = sum over k of X[m, k] Y[n, k], fp32 sums.
//
// Each operand lies in memory either with k adjacent ("K rows": X[m][k]) or with
// its other index adjacent ("K columns": X[k][m]); both are staged in LDS as they
// lie, by LDS-DMA of 16 bytes a lane, two stages deep, and reach the matrix
// instructions through 16-byte reads or, for K columns, transposing reads.  A wave holds
// the fragments of half a stage while it reads those of the next half, and the block
// meets once a stage, between the halves, with products on both sides of the barrier;
// the products of a half go in rounds with its reads and fetches between them.  The
// 16-byte chunks of a stage are permuted so that reads spread over the banks (those of K
// columns in eights meet some twice, a quarter of their cycles: see Frags): the DMA writes
// LDS linearly, so each lane fetches the chunk that belongs at its place.  Buffer descriptors bound every access: rows, columns and k past an
// operand's end read as zero.
//
// fp32 operands come as three bf16 planes that add up to them exactly, each the nearest
// to what is left; the six products of planes of at most two steps down run as one longer
// sum over k (the other three are at most 2^-24 of a product, with either sign).  The
// products with a lower plane take the first plane from a copy without infinities: a lower plane is
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

// An operand as it lies: rows of cols elements, ld apart; or, in panels, columns in
// groups of 64, each group a matrix of its own of `height` rows ld apart (all of which
// exist; cols is a multiple of 64).  Panels keep what a stage reads of a wide matrix in a
// few pages, whichever way the product runs.
struct Operand {
  const uint16_t* p;
  int64_t ld;
  int64_t plane;   // elements between planes
  int64_t finite;  // elements from the first plane to its copy without infinities
  int64_t rows, cols;
  int64_t height;
};

struct GemmArgs {
  Operand x, y;
  int64_t M, N, K;
  int planes;       // 1 or 3
  int tiles_m, tiles_n;
  int splits;       // blocks along k of a tile
  int steps;        // stages of the whole sum
  int per, each;    // stages of one product of planes, of a split
};

// Rows of an operand may be this far apart: a stage's 256 lie within a descriptor.
constexpr int64_t kMaxLd = int64_t(1) << 21;
constexpr int64_t kMaxPanelRows = int64_t(1) << 20;

__device__ __forceinline__ void dma16(rsrc_t r, uint32_t off, uint32_t soff, void* lds) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_t*)lds, 16, off, soff, 0, 0);
}

// A barrier that leaves loads in flight; no memory access of the program moves across it.
__device__ __forceinline__ void block_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Values that are the same in every lane, put where the compiler sees it (scalar
// registers): results of divisions are not.
__device__ __forceinline__ int scalar(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t scalar(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane(uint32_t(v)), hi = __builtin_amdgcn_readfirstlane(uint32_t(uint64_t(v) >> 32));
  return int64_t(uint64_t(hi) << 32 | lo);
}
__device__ __forceinline__ const char* scalar(const char* p) {
  return reinterpret_cast<const char*>(scalar(reinterpret_cast<int64_t>(p)));
}

// The kernel's arguments, read again where they are used.  Held from the start of a kernel
// they would take the scalar registers that its main loop needs.
template <typename T>
__device__ __forceinline__ const T& arguments() {
  typedef const __attribute__((address_space(4))) T* ptr;
  ptr p = (ptr)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const T*)p;
}

// One operand's side of a block: R rows (K rows) or columns (K columns) of its stages.
// A stage is fetched through a descriptor that stays put while a scalar offset moves.
// EIGHTS: as Frags.
template <int R, int NW, bool KCOL, bool PANEL, bool EIGHTS>
struct Side {
  static constexpr int kBytes = R * kStep * 2;
  static constexpr int kLoads = kBytes / (1024 * NW);  // DMA instructions of a wave
  static_assert(kLoads >= 1 && kBytes % (1024 * NW) == 0, "a stage is whole DMA instructions");
  static constexpr int kRowBytes = KCOL ? R * 2 : kStep * 2;  // in LDS
  static constexpr uint32_t kRebase = 1u << 29;

  const char* base;
  int64_t left;         // bytes from base to the operand's end
  uint32_t step, soff;  // bytes from stage to stage, from base to the stage
  int records;
  uint32_t off[kLoads];
  uint32_t tail;        // bit i: load i of a K-rows stage is past the last k in the last stage

  __device__ __forceinline__ void init(const Operand& o, int w, int lane) {
    const int64_t ldb = o.ld * 2, panel = o.height * ldb;
    step = uint32_t(scalar(int(KCOL ? kStep * ldb : PANEL ? panel : kStep * 2)));
    tail = 0;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int b = (w * kLoads + i) * 1024 + lane * 16;
      const int row = b / kRowBytes, chunk = (b % kRowBytes / 16) ^ swizzle(row);
      off[i] = uint32_t(row * ldb) + (PANEL && KCOL ? uint32_t(chunk / 8 * panel) + chunk % 8 * 16 : chunk * 16);
      if (!KCOL && !PANEL && chunk * 8 >= int((o.cols - 1) % kStep + 1)) tail |= 1u << i;
    }
  }
  static __device__ __forceinline__ int swizzle(int row) {
    return !KCOL ? row & 7 : EIGHTS ? 4 * (row & 3) : 2 * ((row & 3) | ((row >> 3) & 1) << 2);
  }
  __device__ __forceinline__ void place() {
    const int hi = int(left >> 32);  // (a 64-bit comparison would be a vector instruction)
    const uint32_t lo = uint32_t(left);
    records = scalar(hi < 0 ? 0 : hi > 0 || lo > 0x7FFFFFF0u ? 0x7FFFFFF0 : int(lo));
  }
  // Goes to stage `s` of plane `pl` (kFinite: of the first one's copy) at row or column r0.
  __device__ __forceinline__ void seek(const Operand& o, int r0, int pl, int s) {
    const int64_t ldb = o.ld * 2, panel = o.height * ldb;
    const int64_t at = PANEL ? (KCOL ? r0 / kStep * panel : r0 * ldb) : KCOL ? r0 * 2 : r0 * ldb;
    const int64_t total = PANEL ? (o.cols / kStep - 1) * panel + (o.height - 1) * ldb + kStep * 2
                                : ((o.rows - 1) * o.ld + o.cols) * 2;
    const int64_t skip = at + int64_t(s) * step;
    base = scalar(reinterpret_cast<const char*>(o.p + (pl == kFinite ? o.finite : pl * o.plane)) + skip);
    left = scalar(total - skip);
    soff = 0;
    place();
#pragma unroll
    for (int i = 0; i < kLoads; ++i) off[i] &= 0x7FFFFFFFu;
  }
  __device__ __forceinline__ void next() { soff += step; }
  __device__ __forceinline__ void rebase() {
    base += soff;
    left -= soff;
    soff = 0;
    place();
  }
  // The stage that comes is the last of its plane: what lies past the last k is out of
  // every descriptor's reach.
  __device__ __forceinline__ void last() {
    // (no branch: lanes differ, and with one the loop's uniform state would go to vectors)
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      if (!KCOL && !PANEL) off[i] |= (tail >> i & 1) << 31;
  }
  __device__ __forceinline__ rsrc_t descriptor(bool live) const {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(scalar(base)), 0, scalar(live ? records : 0), 0x00020000);
  }
  __device__ __forceinline__ void fetch(rsrc_t r, char* lds, int i, int w) const {
    dma16(r, off[i], scalar(int(soff)), lds + (w * kLoads + i) * 1024);
  }
};

// Four rows of 16 elements, a lane's pointer at 4 of them, come as 16 columns of four.
// (The qualifier is what tells the compiler which memory the builtin reads; without it
// every such read waited for all DMA in flight, whatever it was writing.)
__device__ __forceinline__ s16x4 read_transposed(const char* __restrict__ p) {
  typedef __attribute__((address_space(3))) s16x4* ptr;
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(p));
}

// A lane's addresses of its fragments in a stage: rows (or columns) r0 + 16 f + (lane & 15),
// k = 32 s + 8 (lane >> 4) .. + 7.  EIGHTS (K columns): two fragments together take 32
// columns, of which fragment f has the fours of parity f & 1: a lane's results of the two
// are eight neighbours, so that a product of few stages (64 rows, 32000 x 1024 of them
// written in bf16: 27 us, with four neighbours 34) writes whole lines.
template <int R, int F, bool KCOL, bool EIGHTS>
struct Frags {
  uint32_t at[KCOL ? F : 2];
  __device__ __forceinline__ void init(int r0, int lane) {
    const int q = lane >> 4, i = lane & 15;
    if (KCOL) {
      const int k = q * 8 + (i >> 2);
      const int fp = (i >> 2) | (q & 1) << 2;
#pragma unroll
      for (int f = 0; f < F; ++f)
        at[f] = EIGHTS ? k * (R * 2) + ((r0 / 8 + f / 2 * 4 + (i & 3)) ^ (i >> 2) * 4) * 16 + f % 2 * 8
                       : k * (R * 2) + ((r0 / 16 + f) ^ fp) * 32 + (i & 3) * 8;
    } else {
#pragma unroll
      for (int s = 0; s < 2; ++s) at[s] = (r0 + i) * (kStep * 2) + (((s * 4 + q) ^ (i & 7)) * 16);
    }
  }
  __device__ __forceinline__ bf16x8 read(const char* lds, int f, int s) const {
    if (KCOL) {
      const char* p = lds + at[f] + s * (32 * R * 2);
      const s16x4 a = read_transposed(p), b = read_transposed(p + 4 * R * 2);
      typedef short s16x8 __attribute__((ext_vector_type(8)));
      const s16x8 v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
      return __builtin_bit_cast(bf16x8, v);
    }
    return *reinterpret_cast<const bf16x8*>(lds + at[s] + f * (16 * kStep * 2));
  }
};

// The tile of a unit of work: neighbours go to the eight XCDs in turn, so each XCD takes
// a contiguous run of tiles, in groups of eight rows of tiles (what the run reads at a
// time then fits its L2).
__device__ __forceinline__ void tile_of(const GemmArgs& g, uint32_t id, int& tm, int& tn) {
  constexpr uint32_t kXcd = 8, kGroup = 8;
  const uint32_t tiles = uint32_t(g.tiles_m) * uint32_t(g.tiles_n);
  const uint32_t q = tiles / kXcd, rem = tiles % kXcd;
  const uint32_t x = id % kXcd, k = id / kXcd;
  const uint32_t t = x * q + (x < rem ? x : rem) + k;
  const uint32_t width = kGroup * uint32_t(g.tiles_n);
  const uint32_t grp = t / width, in = t - grp * width;
  const uint32_t first = grp * kGroup, left = uint32_t(g.tiles_m) - first;
  const uint32_t size = left < kGroup ? left : kGroup;
  tm = scalar(int(first + in % size));
  tn = scalar(int(in / size));
}

// The planes of the s-th product of an fp32 pair, smallest first.
__device__ __forceinline__ void planes_of(int s, int& px, int& py) {
  constexpr uint32_t xs = 0x031132, ys = 0x013123;  // (2,F) (F,2) (1,1) (1,F) (F,1) (0,0)
  px = xs >> (4 * s) & 15;
  py = ys >> (4 * s) & 15;
}

// The product of one tile.  acc[i][j]: lane l holds rows m = 16 j + (l & 15) and
// columns n = 16 i + 4 (l >> 4) + 0..3 of the wave's tile; with YCOL, in i's pairs,
// n = 32 (i / 2) + 8 (l >> 4) + 4 (i % 2) + 0..3.
template <int BM, int BN, int WM, int WN, bool XCOL, bool XPANEL, bool YCOL>
struct Gemm {
  static constexpr int NW = WM * WN, TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
  using SX = Side<BM, NW, XCOL, XPANEL, false>;
  using SY = Side<BN, NW, YCOL, false, YCOL>;
  static constexpr int kStage = SX::kBytes + SY::kBytes;
  static constexpr int kLoads = SX::kLoads + SY::kLoads;
  static constexpr int kNotes = WN * BM * 8;  // bytes past the stages for the kernel's own use
  static_assert(FM % 2 == 0 && FN <= FM / 2 * 2, "half of a wave's rounds read all fragments");

  // (the kernel's arguments begin with the GemmArgs)
  char* lds;  // two stages
  int lane, w, per, s0, s1, prod, k, m0, n0;
  SX sx;
  SY sy;
  Frags<BM, FM, XCOL, false> fx;
  Frags<BN, FN, YCOL, YCOL> fy;

  __device__ __forceinline__ explicit Gemm(char* stages) : lds(stages) {
    const GemmArgs& g = arguments<GemmArgs>();
    lane = threadIdx.x & 63;
    w = scalar(int(threadIdx.x >> 6));
    fx.init(w / WN * TM, lane);
    fy.init(w % WN * TN, lane);
    sx.init(g.x, w, lane);
    sy.init(g.y, w, lane);
    per = scalar(g.per);
  }

  // Starts on a tile: its first two stages are on their way.
  __device__ __forceinline__ void begin(int tm, int tn, int split) {
    const GemmArgs& g = arguments<GemmArgs>();
    s0 = scalar(split * g.each);
    s1 = scalar(min(s0 + g.each, g.steps));
    prod = scalar(s0 / per);
    k = s0 - prod * per;
    m0 = tm * BM;
    n0 = tn * BN;
    seek();
    fetch(sx.descriptor(s0 < s1), sy.descriptor(s0 < s1), lds, 0, kLoads);
    next();
    fetch(sx.descriptor(s0 + 1 < s1), sy.descriptor(s0 + 1 < s1), lds + kStage, 0, kLoads);
    next();
  }

  __device__ __forceinline__ void seek() {
    const GemmArgs& g = arguments<GemmArgs>();
    int px = 0, py = 0;
    if (g.planes == 3) planes_of(prod, px, py);
    sx.seek(g.x, m0, px, k);
    sy.seek(g.y, n0, py, k);
    if (k == per - 1) sx.last(), sy.last();
  }
  __device__ __forceinline__ void next() {
    ++k;
    sx.next();
    sy.next();
    if (k >= per - 1 || max(sx.soff, sy.soff) >= SX::kRebase) {  // seldom
      if (k == per) {
        ++prod;
        k = 0;
        if (prod < 6) seek();
      } else {
        sx.rebase();
        sy.rebase();
        if (k == per - 1) sx.last(), sy.last();
      }
    }
  }
  // Loads [lo, hi) of a stage.
  __device__ __forceinline__ void fetch(rsrc_t rx, rsrc_t ry, char* to, int lo, int hi) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      if (i < lo || i >= hi) continue;
      if (i < SX::kLoads) sx.fetch(rx, to, i, w);
      else sy.fetch(ry, to + SX::kBytes, i - SX::kLoads, w);
    }
  }
  // What round j of FM reads of a half: all of it in the first half of the rounds.
  __device__ __forceinline__ void read(const char* from, int h, int j, bf16x8 (&xf)[FM], bf16x8 (&yf)[FN]) const {
    if (j >= FM / 2) return;
#pragma unroll
    for (int i = 0; i < FN; ++i)
      if (i / ((FN + FM / 2 - 1) / (FM / 2)) == j) yf[i] = fy.read(from + SX::kBytes, i, h);
    xf[2 * j] = fx.read(from, 2 * j, h);
    xf[2 * j + 1] = fx.read(from, 2 * j + 1, h);
  }

  // The tile's product.  Before: this wave's vmcnt was 0 after begin(), and the block met.
  // After: the stages may be overwritten.
  __device__ __forceinline__ void run(f32x4 (&acc)[FN][FM]) {
    bf16x8 xa[FM], ya[FN], xb[FM], yb[FN];  // fragments of a stage's first and second 32 k
    auto multiply = [&](int j, const bf16x8 (&xf)[FM], const bf16x8 (&yf)[FN]) {
#pragma unroll
      for (int i = 0; i < FN; ++i)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(yf[i], xf[j], acc[i][j], 0, 0, 0);
    };
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
      for (int j = 0; j < FM; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < FM / 2; ++j) read(lds, 0, j, xa, ya);
#pragma nounroll
    for (int s = s0; s < s1; ++s) {
      char* now = lds + ((s - s0) & 1) * kStage;
      char* then = lds + (~(s - s0) & 1) * kStage;
#pragma unroll
      for (int j = 0; j < FM; ++j) {
        read(now, 1, j, xb, yb);
        multiply(j, xa, ya);
        __builtin_amdgcn_sched_barrier(0);
      }
      // the next stage is there (vmcnt 0; the tile's second one was before) and this one is
      // in registers (lgkmcnt 0); past the barrier that holds for every wave, so this stage's
      // place takes the stage after next (past the last one: nothing, by an empty descriptor)
      if (s > s0) __builtin_amdgcn_s_waitcnt(0x0070);
      else __builtin_amdgcn_s_waitcnt(0xC07F);
      block_barrier();
      __builtin_amdgcn_sched_barrier(0);
      const rsrc_t rx = sx.descriptor(s + 2 < s1), ry = sy.descriptor(s + 2 < s1);
#pragma unroll
      for (int j = 0; j < FM; ++j) {
        read(then, 0, j, xa, ya);
        fetch(rx, ry, now, j * kLoads / FM, (j + 1) * kLoads / FM);
        multiply(j, xb, yb);
        __builtin_amdgcn_sched_barrier(0);
      }
      next();
    }
    __builtin_amdgcn_s_waitcnt(0x0070);
    block_barrier();
  }

  // This wave's share of the stages that begin() fetched has landed, and what it wrote to
  // LDS is there.
  static __device__ __forceinline__ void landed() { __builtin_amdgcn_s_waitcnt(0x0070); }
};

}  // namespace dendsn_seq
