// Gated delta rule: forward and backward over chunks of 64 steps, and one-token step.
//
// Of a head's steps i in a chunk that starts from state S, with G_i the sum of g up to i,
// D_ij = exp(G_i - G_j) for j <= i, and u_i = b_i (v_i - a_i S[i-1]^T k_i) the values that
// are added,
//
//   (I + A) U = R,  A_ij = b_i D_ij k_i.k_j (j < i),  R_i = b_i (v_i - e^G_i S^T k_i)
//   o_i = scale e^G_i S^T q_i + sum_j P_ij u_j,       P_ij = scale D_ij q_i.k_j (j <= i)
//   S'  = e^G_63 S + sum_i e^(G_63 - G_i) k_i u_i^T
//
// and back, from dS' and do, with T = (I + A)^-1,
//
//   dU = P^T do + e^(G_63 - G) K dS',   dR = T^T dU,   dv = b dR
//   dS = e^G_63 dS' + Q^T (scale e^G do) - K^T (b e^G dR)
//   dq = scale e^G do S^T + E K,        E_ij = scale D_ij do_i.u_j (j <= i)
//   dk = b X + Y,  X = F K - e^G dR S^T,  F_ij = -D_ij dR_i.u_j (j < i)
//   Y = e^(G_63 - G) U dS'^T + E^T Q + (b F)^T K
//   db_i = dR_i.v_i + k_i.X_i
//   dg_t = sum over i >= t of (q_i.dq_i + b_i k_i.X_i - k_i.Y_i)
//          + sum over all i of e^(G_63 - G_i) k_i.(dS' u_i) + e^G_63 <S, dS'>
//
// where E's diagonal, which has no decay, is left out of the products (its parts of the two sums
// would cancel) and added to dq and dk at the end, and what dS' gives is summed over i < t.
//
// T and P are of a chunk alone and are computed for all chunks at once (local); the states go
// chunk by chunk, 32 columns of v a block (scan, and back: back_scan, which leaves dR and dS');
// the gradients of q, k, g and b are again of a chunk alone (back_local).
//
// Products are matrix instructions of 16 x 16.  In bf16 the inputs are operands as they are;
// everything computed on the way is a sum of bf16 values: of three in the scans, whose states
// are outputs in fp32 (s_last off by 0.8 to 1.5e-7 of a head's norm, grad_s0 by 1.5 to 2.3e-7; s_last by
// 3.5e-6 with two), of two where all ends in bf16.  In fp32 the fp32 instruction is used.  States and
// values that the backward reads are kept in fp32.
//
// 8192 steps of 4 sequences, 16 heads of 128 x 128, bf16, under a profiler: local 190 us twice (400 MB
// written: 3.5 TB/s), scan 620, back_scan 740, back_local 605 (2.7 GB: 4.3 TB/s, bound by memory).
// The scans have one block a CU, whose three barriers a chunk let nothing saturate (matrix units
// 13 % busy, LDS 30 %, HBM 2.6 TB/s): without its loads the scan takes 356 us, without stores of
// states too 327.  Tried: fewer dependent matrix instructions in a row (no gain, spills), 16-byte
// stores of turned states (no gain), stores past the caches (no gain), two blocks of 16 columns a CU
// (916 us).  One token of 64 requests,
// 16 heads of 128 x 128: 23 us a call for 135 MB.
#include "dendsn_block.h"
#include "seq_common.h"

namespace dendsn_seq {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kC = 64;          // steps of a chunk
constexpr int kThreads = 256;

constexpr double kForget = -200.0;  // exp of it is 0 in fp32

struct DeltaArgs {
  const void *q, *k, *v, *g, *beta, *go;
  const float *s0, *gs_last, *state_in;
  const int32_t* lengths;
  void *o, *gq, *gk, *gv, *gg, *gbeta;
  float *s_last, *gs0;
  float *ck_s, *ck_u;       // [batch][H][nc]: [KP][Vp], [64][Vp]
  void *tm, *pm;            // [batch][H][nc]: planes of [64][64]
  float* dec;               // [batch][H][nc]: [3][64]
  float *dr, *ds;           // as ck_u and ck_s
  float *part_q, *part_k;   // [T][batch][H][K] where heads are shared
  int64_t q_t, q_b, q_h, k_t, k_b, k_h, v_t, v_b, v_h, g_t, g_b, g_h, beta_t, beta_b, beta_h, o_t, o_b, o_h;
  int64_t go_t, go_b, go_h;
  float *maps, *seg_in;     // [batch][H][segs]: [KP][Vp + KP], [KP][Vp]
  int32_t T, batch, H, Hk, K, V, nc, Vp;
  int32_t segs, per, pass;  // segments of the steps, chunks of one, and what a scan does (Pass)
  float scale;
};

// A long sequence of few heads is cut into segments that go at once: the first pass starts each
// from S = 0 beside K columns of the identity, which gives it as a map S -> M S + N of what enters
// it; the maps are composed (delta_join_states); the second pass starts from the states.
enum Pass { kWhole, kMaps, kStates };

// ---------------------------------------------------------------------------
// Operands.  A fragment is a lane's eight values of one row (or column): row
// lane % 16, places 8 (lane / 16) to + 7 of 32 along the sum.
// ---------------------------------------------------------------------------
struct F32 {
  using IO = float;
  using Word = float;
  static constexpr int planes = 1;
};
template <int P> struct Bf {
  using IO = bf16_t;
  using Word = __bf16;
  static constexpr int planes = P;
};

template <class M> struct Exact;  // of inputs
template <class M> struct Both;   // of what was computed: a sum of planes
template <> struct Both<F32> { f32x8 v; };
template <> struct Exact<F32> : Both<F32> {};
template <int P> struct Exact<Bf<P>> { bf16x8 h; };
template <int P> struct Both<Bf<P>> { bf16x8 p[P]; };

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// The Q largest orders of planes, the smallest first; Q of 0: all.
template <int Q = 0, int P>
__device__ __forceinline__ void mma(f32x4& c, const Exact<Bf<P>>& a, const Exact<Bf<P>>& b) { c = mfma(a.h, b.h, c); }
template <int Q = 0, int P>
__device__ __forceinline__ void mma(f32x4& c, const Exact<Bf<P>>& a, const Both<Bf<P>>& b) {
#pragma unroll
  for (int j = (Q ? Q : P) - 1; j >= 0; --j) c = mfma(a.h, b.p[j], c);
}
template <int Q = 0, int P>
__device__ __forceinline__ void mma(f32x4& c, const Both<Bf<P>>& a, const Exact<Bf<P>>& b) {
#pragma unroll
  for (int j = (Q ? Q : P) - 1; j >= 0; --j) c = mfma(a.p[j], b.h, c);
}
template <int Q = 0, int P>
__device__ __forceinline__ void mma(f32x4& c, const Both<Bf<P>>& a, const Both<Bf<P>>& b) {
#pragma unroll
  for (int n = (Q ? Q : P) - 1; n >= 0; --n)
#pragma unroll
    for (int j = 0; j <= n; ++j) c = mfma(a.p[j], b.p[n - j], c);
}
template <int Q = 0>
__device__ __forceinline__ void mma(f32x4& c, const Both<F32>& a, const Both<F32>& b) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j], b.v[j], c, 0, 0, 0);
}

__device__ __forceinline__ void both_of(f32x8 x, Both<F32>& f) { f.v = x; }
template <int P>
__device__ __forceinline__ void both_of(f32x8 x, Both<Bf<P>>& f) {
#pragma unroll
  for (int j = 0; j < P; ++j) {
    f.p[j] = __builtin_convertvector(x, bf16x8);
    if (j + 1 < P) x -= __builtin_convertvector(f.p[j], f32x8);
  }
}

// Eight values of a row as they are stored.
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
template <typename IO> struct Eight;
template <> struct Eight<float> {
  typedef f32x8 Vec;
  typedef f32x8 Any __attribute__((aligned(4)));  // anywhere in memory
  static __device__ __forceinline__ float bits(float v) { return v; }
  static __device__ __forceinline__ float wide(float v) { return v; }
};
template <> struct Eight<bf16_t> {
  typedef u16x8 Vec;
  typedef u16x8 Any __attribute__((aligned(2)));
  static __device__ __forceinline__ uint16_t bits(bf16_t v) { return v.bits; }
  static __device__ __forceinline__ float wide(uint16_t v) { return widen(bf16_t{v}); }
};

// The value `at` places behind a base that is the same in all lanes: 64 steps of a tensor span
// less than 2^31 bytes, and addresses are a scalar and 32 bits.
template <typename T>
__device__ __forceinline__ const T& behind(const T* base, uint32_t at) {
  return *reinterpret_cast<const T*>(reinterpret_cast<const char*>(base) + uint32_t(at * uint32_t(sizeof(T))));
}
template <typename T>
__device__ __forceinline__ T& behind(T* base, uint32_t at) {
  return *reinterpret_cast<T*>(reinterpret_cast<char*>(base) + uint32_t(at * uint32_t(sizeof(T))));
}

// Stores by a descriptor drop what lies at 2^31 and beyond: a condition is an offset, and no branch
// comes between the stores and what they are counted with.
typedef __amdgpu_buffer_rsrc_t rsrc_t;
constexpr uint32_t kNowhere = 0x80000000u;
__device__ __forceinline__ rsrc_t stores_to(void* base, bool there = true) {
  return __builtin_amdgcn_make_buffer_rsrc(base, 0, there ? int(kNowhere) : 0, 0x00020000);
}
__device__ __forceinline__ void put_at(rsrc_t to, uint32_t at, float v, float) {
  __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), to, at, 0, 0);
}
__device__ __forceinline__ void put_at(rsrc_t to, uint32_t at, float v, bf16_t) {
  __builtin_amdgcn_raw_buffer_store_b16(bf16_bits(v), to, at, 0, 0);
}

// Eight places from k0 on of the row of K that starts `row` places behind base, without a branch a
// lane: what lies past K has some other value of the row.  odd (K is no multiple of 8): value
// by value.
template <typename IO>
__device__ __forceinline__ typename Eight<IO>::Vec load8(const IO* base, uint32_t row, int k0, int K, bool odd) {
  typename Eight<IO>::Vec r;
  if (!odd) {
    r = *reinterpret_cast<const typename Eight<IO>::Any*>(&behind(base, row + (k0 < K ? k0 : 0)));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = Eight<IO>::bits(behind(base, row + min(k0 + j, K - 1)));
  }
  return r;
}
// The same with zeros past K.
template <typename V>
__device__ __forceinline__ void cut8(V& r, int k0, int K) {
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = k0 + j < K ? r[j] : 0;
}
template <class M>
__device__ __forceinline__ Exact<M> exact_of(typename Eight<typename M::IO>::Vec r) {
  Exact<M> f;
  if constexpr (M::planes == 1) f.v = r;
  else f.h = __builtin_bit_cast(bf16x8, r);
  return f;
}
template <class M>
__device__ __forceinline__ Both<M> load_both(const float* p) {  // 16-byte aligned
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
  Both<M> f;
  both_of(__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7), f);
  return f;
}

// Matrices in LDS, rows along the sum; padded, so that a fragment's read meets a bank twice at most.
// (Without meeting any twice, by exchanged pieces, the scans are no faster: 625 for 623 us.)
template <class M, int ROWS, int COLS> struct Mat;  // of computed values
template <int ROWS, int COLS> struct Mat<F32, ROWS, COLS> {
  static constexpr int kLd = COLS + 4;
  float v[ROWS * kLd];
  __device__ __forceinline__ Both<F32> frag(int row, int col) const {
    const int lane = threadIdx.x & 63;
    return load_both<F32>(v + (row + lane % 16) * kLd + col + lane / 16 * 8);
  }
  __device__ __forceinline__ void put4(int row, int col, f32x4 x) { *reinterpret_cast<f32x4*>(v + row * kLd + col) = x; }
  __device__ __forceinline__ void put(int row, int col, float x) { v[row * kLd + col] = x; }
};
template <int P, int ROWS, int COLS> struct Mat<Bf<P>, ROWS, COLS> {
  static constexpr int kLd = COLS + 8;
  __bf16 v[P][ROWS * kLd];
  __device__ __forceinline__ Both<Bf<P>> frag(int row, int col) const {
    const int lane = threadIdx.x & 63, at = (row + lane % 16) * kLd + col + lane / 16 * 8;
    Both<Bf<P>> f;
#pragma unroll
    for (int j = 0; j < P; ++j) f.p[j] = *reinterpret_cast<const bf16x8*>(v[j] + at);
    return f;
  }
  __device__ __forceinline__ void put4(int row, int col, f32x4 x) {
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const bf16x4 a = __builtin_convertvector(x, bf16x4);
      *reinterpret_cast<bf16x4*>(v[j] + row * kLd + col) = a;
      if (j + 1 < P) x -= __builtin_convertvector(a, f32x4);
    }
  }
  __device__ __forceinline__ void put(int row, int col, float x) {
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const __bf16 a = static_cast<__bf16>(x);
      v[j][row * kLd + col] = a;
      if (j + 1 < P) x -= static_cast<float>(a);
    }
  }
};
template <class M, int ROWS, int COLS> struct MatX;  // of inputs
template <int ROWS, int COLS> struct MatX<F32, ROWS, COLS> {
  static constexpr int kLd = COLS + 4;
  float v[ROWS * kLd];
  __device__ __forceinline__ Exact<F32> frag(int row, int col) const {
    const int lane = threadIdx.x & 63;
    Exact<F32> f;
    f.v = load_both<F32>(v + (row + lane % 16) * kLd + col + lane / 16 * 8).v;
    return f;
  }
  __device__ __forceinline__ void put4(int row, int col, float a, float b, float c, float d) {
    *reinterpret_cast<f32x4*>(v + row * kLd + col) = f32x4{a, b, c, d};
  }
  __device__ __forceinline__ f32x4 get4(int row, int col) const { return *reinterpret_cast<const f32x4*>(v + row * kLd + col); }
};
template <int P, int ROWS, int COLS> struct MatX<Bf<P>, ROWS, COLS> {
  static constexpr int kLd = COLS + 8;
  __bf16 h[ROWS * kLd];
  __device__ __forceinline__ Exact<Bf<P>> frag(int row, int col) const {
    const int lane = threadIdx.x & 63;
    return Exact<Bf<P>>{*reinterpret_cast<const bf16x8*>(h + (row + lane % 16) * kLd + col + lane / 16 * 8)};
  }
  __device__ __forceinline__ void put4(int row, int col, uint16_t a, uint16_t b, uint16_t c, uint16_t d) {
    *reinterpret_cast<uint2*>(h + row * kLd + col) = uint2{a | uint32_t(b) << 16, c | uint32_t(d) << 16};
  }
  __device__ __forceinline__ f32x4 get4(int row, int col) const {
    return __builtin_convertvector(*reinterpret_cast<const bf16x4*>(h + row * kLd + col), f32x4);
  }
};

// dst[d][t] = rows[t][d]: 64 steps (n of which are there), D of ROWS places.  A thread has a
// block of 4 x 8, in registers between the two.
template <class M, int ROWS> struct Turn {
  using IO = typename M::IO;
  static_assert(2 * ROWS <= kThreads, "one block a thread");
  // (with fewer blocks than 256 threads several have the same one)
  __device__ __forceinline__ static int tid() { return threadIdx.x % (2 * ROWS); }
  typename Eight<IO>::Vec r[4];
  uint32_t at[4];  // the four rows
  // steps past the n-th have the n-th's values
  __device__ __forceinline__ void place(uint32_t stride, int n) {
#pragma unroll
    for (int x = 0; x < 4; ++x) at[x] = uint32_t(min(tid() % 16 * 4 + x, n - 1)) * stride;
  }
  __device__ __forceinline__ void load(const IO* rows, int D, bool odd) {
#pragma unroll
    for (int x = 0; x < 4; ++x) r[x] = load8(rows, at[x], tid() / 16 * 8, D, odd);
  }
  __device__ __forceinline__ void put(MatX<M, ROWS, kC>& dst, int D) {
    const int t = tid() % 16 * 4, d = tid() / 16 * 8;
    if (D < ROWS) {
#pragma unroll
      for (int x = 0; x < 4; ++x) cut8(r[x], d, D);
    }
#pragma unroll
    for (int y = 0; y < 8; ++y) dst.put4(d + y, t, r[0][y], r[1][y], r[2][y], r[3][y]);
  }
};

// A barrier for what is in LDS: loads and stores of device memory stay in flight.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// T and P in memory: planes of [64][64], as operands of their rows.
template <class M, int Q = M::planes>
__device__ __forceinline__ Both<M> load_planes(const typename M::Word* p, int row, int col) {
  const int at = row * kC + col;
  Both<M> f;
  if constexpr (M::planes == 1) {
    f = load_both<M>(p + at);
  } else {
#pragma unroll
    for (int j = 0; j < Q; ++j) f.p[j] = *reinterpret_cast<const bf16x8*>(p + j * kC * kC + at);
  }
  return f;
}
__device__ __forceinline__ int length_of(const DeltaArgs& a, int b) {
  if (!a.lengths) return a.T;
  const int n = a.lengths[b];
  return n < 0 ? 0 : n > a.T ? a.T : n;
}

// exp of a difference of sums, whose rounding to fp32 would be off by more than the result's.
__device__ __forceinline__ float exp_of(double x) {
  const float f = float(x), e = expf(f);
  return fmaf(e, float(x - double(f)), e);
}

// G_i of lane i's step: sums of a chunk's logarithms, in 64 bits (their differences count).
template <typename IO>
__device__ __forceinline__ double chunk_sum(const DeltaArgs& a, int b, int h, int t0, int n) {
  const int i = threadIdx.x & 63;
  double G = 0.0;
  if (i < n) {
    G = double(widen(static_cast<const IO*>(a.g)[int64_t(t0 + i) * a.g_t + b * a.g_b + h * a.g_h]));
    G = G < kForget ? kForget : G;  // (NaN stays)
  }
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    const double up = __shfl_up(G, s);
    if (i >= s) G += up;
  }
  return G;
}

// ---------------------------------------------------------------------------
// local: T and P (BACK: turned) and the decays of one chunk.  Wave w has steps 16 w to + 15
// of A and P.  T by blocks of 16: those on the diagonal by substitution, a column a lane; then
// T_ij = -T_ii sum over k from j to i - 1 of A_ik T_kj, a diagonal of blocks at a time, in fp32.
// Both squares are written whole, with all planes: what the scans do not read of them (the quarter that
// is 0, forward P's third plane) is some 150 of the 409 MB of the longest case forward, 100 back.
// ---------------------------------------------------------------------------
// Eight values of a row of T or P from LDS, as planes in memory.
template <class M>
__device__ __forceinline__ void store_planes8(typename M::Word* p, int row, int col, f32x8 x) {
  if constexpr (M::planes == 1) {
    *reinterpret_cast<f32x8*>(p + row * kC + col) = x;
  } else {
#pragma unroll
    for (int j = 0; j < M::planes; ++j) {
      const bf16x8 a = __builtin_convertvector(x, bf16x8);
      *reinterpret_cast<bf16x8*>(p + j * kC * kC + row * kC + col) = a;
      x -= __builtin_convertvector(a, f32x8);
    }
  }
}

template <class M, int KP, bool BACK>
__global__ __launch_bounds__(kThreads, M::planes == 1 && KP > 64 ? 2 : 3) void delta_local_kernel(DeltaArgs a) {
  using IO = typename M::IO;
  using Word = typename M::Word;
  constexpr int KS = KP / 32, kLd = kC + 4;
  const int lane = threadIdx.x & 63, w = threadIdx.x / 64, r = lane % 16, q4 = lane / 16;
  const int c = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const int t0 = c * kC, n = min(length_of(a, b) - t0, kC);
  if (n <= 0) return;
  __shared__ double sg[kC];
  __shared__ float sb[kC];
  __shared__ __align__(16) float sa[kC][kLd], st[kC][kLd], sm[4][16][17];  // A and later P, T
  const int64_t at = (int64_t(b) * a.H + h) * a.nc + c;
  const int hk = h / (a.H / a.Hk), row = 16 * w + r;
  const IO* kp = static_cast<const IO*>(a.k) + t0 * a.k_t + b * a.k_b + hk * a.k_h;
  const IO* qp = static_cast<const IO*>(a.q) + t0 * a.q_t + b * a.q_b + hk * a.q_h;
  const bool odd = a.K % 8;
  typename Eight<IO>::Vec kr[3][KS], own[KS], qr[KS];  // rows of the blocks before, of the wave's own
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    qr[s] = load8(qp, uint32_t(min(row, n - 1)) * uint32_t(a.q_t), s * 32 + q4 * 8, a.K, odd);
    own[s] = load8(kp, uint32_t(min(row, n - 1)) * uint32_t(a.k_t), s * 32 + q4 * 8, a.K, odd);
#pragma unroll
    for (int bj = 0; bj < 3; ++bj)
      if (bj < w) kr[bj][s] = load8(kp, uint32_t(min(16 * bj + r, n - 1)) * uint32_t(a.k_t), s * 32 + q4 * 8, a.K, odd);
  }
  if (w == 3) {  // (the wave with the most products waits least)
    const double G = chunk_sum<IO>(a, b, h, t0, n);
    const double last = __shfl(G, 63);
    const float beta = lane < n ? widen(static_cast<const IO*>(a.beta)[int64_t(t0 + lane) * a.beta_t + b * a.beta_b + h * a.beta_h]) : 0.0f;
    float* dec = a.dec + at * 3 * kC;
    dec[lane] = exp_of(G);
    dec[kC + lane] = exp_of(last - G);
    dec[2 * kC + lane] = beta;
    sg[lane] = G;
    sb[lane] = beta;
  }
  if (a.K < KP) {
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      cut8(qr[s], s * 32 + q4 * 8, a.K);
      cut8(own[s], s * 32 + q4 * 8, a.K);
#pragma unroll
      for (int bj = 0; bj < 3; ++bj)
        if (bj < w) cut8(kr[bj][s], s * 32 + q4 * 8, a.K);
    }
  }
  f32x4 kk[4], qk[4];  // of the blocks before, and last of the wave's own
#pragma unroll
  for (int bj = 0; bj < 4; ++bj) {
    kk[bj] = qk[bj] = f32x4{0, 0, 0, 0};
    if (bj < w || bj == 3) {
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const Exact<M> f = exact_of<M>(bj < 3 ? kr[bj < 3 ? bj : 0][s] : own[s]);
        mma(kk[bj], exact_of<M>(own[s]), f);
        mma(qk[bj], exact_of<M>(qr[s]), f);
      }
    }
  }
  __syncthreads();
  const int i0 = 16 * w + q4 * 4;
  f32x4 P[4];
#pragma unroll
  for (int bj = 0; bj < 4; ++bj) {
    const int j = 16 * bj + r;
    f32x4 A = {0, 0, 0, 0};
    P[bj] = f32x4{0, 0, 0, 0};
    if (bj <= w) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int i = i0 + x;
        const float d = j <= i ? exp_of(sg[i] - sg[j]) : 0.0f;
        A[x] = j < i ? sb[i] * d * (bj < w ? kk[bj][x] : kk[3][x]) : 0.0f;
        P[bj][x] = j <= i ? a.scale * d * (bj < w ? qk[bj][x] : qk[3][x]) : 0.0f;
      }
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      sa[i0 + x][j] = A[x];
      if (bj > w) st[i0 + x][j] = 0.0f;
    }
  }
  __syncthreads();
  {  // the block on the diagonal: lane r has column r, each quarter of the wave writes four rows
    float t[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float s = i == r ? 1.0f : 0.0f;
#pragma unroll
      for (int j = 0; j < i; ++j) s = fmaf(-sa[16 * w + i][16 * w + j], t[j], s);
      t[i] = s;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i / 4 == q4) st[16 * w + i][16 * w + r] = t[i];
  }
  __syncthreads();
#pragma unroll
  for (int d = 1; d < 4; ++d) {
    if (w + d < 4) {
      const int i = 16 * (w + d), j = 16 * w;
      f32x4 m = {0, 0, 0, 0}, t = {0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < 16 * d; k += 4) m = __builtin_amdgcn_mfma_f32_16x16x4f32(sa[i + r][j + k + q4], st[j + k + q4][j + r], m, 0, 0, 0);
#pragma unroll
      for (int x = 0; x < 4; ++x) sm[w][q4 * 4 + x][r] = m[x];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int k = 0; k < 16; k += 4) t = __builtin_amdgcn_mfma_f32_16x16x4f32(st[i + r][i + k + q4], sm[w][k + q4][r], t, 0, 0, 0);
#pragma unroll
      for (int x = 0; x < 4; ++x) st[i + q4 * 4 + x][j + r] = -t[x];
    }
    __syncthreads();
  }
#pragma unroll
  for (int bj = 0; bj < 4; ++bj) {
    const int j = 16 * bj + r;
    if (BACK) *reinterpret_cast<f32x4*>(&sa[j][i0]) = P[bj];
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (!BACK) sa[i0 + x][j] = P[bj][x];
  }
  __syncthreads();
  Word* pm = static_cast<Word*>(a.pm) + at * M::planes * kC * kC;
  Word* tm = static_cast<Word*>(a.tm) + at * M::planes * kC * kC;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int e = u * kThreads + threadIdx.x, i = e / 8, j = e % 8 * 8;
    f32x8 x, y;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      x[k] = BACK ? st[j + k][i] : st[i][j + k];
      y[k] = sa[i][j + k];
    }
    store_planes8<M>(tm, i, j, x);
    store_planes8<M>(pm, i, j, y);
  }
}

// ---------------------------------------------------------------------------
// scan: states and outputs, chunk after chunk, BV columns of v a block of two groups of four
// waves.  The first has the chain: wave w has steps 16 w to + 15 of R and U, and a quarter of the
// state's rows, which stay in its registers.  The second has q's products, the outputs, and
// turns the next chunk's k over.  Three barriers a chunk: the state, R and U go through LDS.
// What a chunk reads is fetched two chunks ahead, into the registers that are free again; the
// barriers wait for LDS alone.  A wave waits for a load by the number of loads and stores behind it,
// on the path that has the fewest: so each is issued in every chunk (past the end the last one's
// again), and stores that are not wanted go nowhere.
// ---------------------------------------------------------------------------
constexpr int kScanThreads = 512;

// Blocks go to the eight XCDs in turn, each of which has a cache of its own: the blocks of one
// head (and segment), which read the same q, k, T and P, are eight apart.
struct ScanBlock {
  int v0, bh, seg;
};
__device__ __forceinline__ ScanBlock scan_block(const DeltaArgs& a, int KP, int BV) {
  const int cols = (a.Vp + (a.pass == kMaps ? KP : 0)) / BV, m = blockIdx.x / 8, heads = a.batch * a.H;
  const int group = m / cols * 8 + blockIdx.x % 8, seg = group / heads;
  return {m % cols * BV, seg < a.segs ? group - seg * heads : -1, seg};
}

template <class M, int KP, int BV>
struct ScanLds {
  MatX<M, KP, kC> kt[2];
  Mat<M, BV, KP> st;
  Mat<M, BV, kC> rt, ut, us;
};

template <class M, int KP, int BV, bool ODD>
__global__ __launch_bounds__(kScanThreads) void delta_scan_kernel(DeltaArgs a) {
  using IO = typename M::IO;
  using Word = typename M::Word;
  using E = Eight<IO>;
  constexpr int KS = KP / 32, MT = KP / 64, NV = BV / 16;  // MT: row tiles of the state of a wave
  extern __shared__ __align__(16) char lds[];
  ScanLds<M, KP, BV>& s = *reinterpret_cast<ScanLds<M, KP, BV>*>(lds);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), w = wave % 4, r = lane % 16, q4 = lane / 16;
  const bool chain = wave < 4;
  const ScanBlock at_block = scan_block(a, KP, BV);
  const int v0 = at_block.v0, bh = at_block.bh, part = at_block.seg;
  if (bh < 0) return;
  const int b = bh / a.H, h = bh - b * a.H, hk = h / (a.H / a.Hk);
  const int len = __builtin_amdgcn_readfirstlane(length_of(a, b)), chunks = (len + kC - 1) / kC;
  const int row = 16 * w + r, i0 = 16 * w + q4 * 4;
  const bool maps = a.pass == kMaps;
  const int c0 = part * a.per, c1 = min(chunks, c0 + a.per);  // the segment's chunks
  const int64_t first = int64_t(bh) * a.nc + c0, seg = int64_t(bh) * a.segs + part;
  // the next chunk's, in turn
  const IO* kc = static_cast<const IO*>(a.k) + b * a.k_b + hk * a.k_h + c0 * kC * a.k_t;
  const IO* qc = static_cast<const IO*>(a.q) + b * a.q_b + hk * a.q_h + c0 * kC * a.q_t;
  const IO* vc = static_cast<const IO*>(a.v) + b * a.v_b + h * a.v_h + c0 * kC * a.v_t;
  const Word* tm = static_cast<const Word*>(a.tm) + first * M::planes * kC * kC;
  const Word* pm = static_cast<const Word*>(a.pm) + first * M::planes * kC * kC;
  const float* dec = a.dec + first * 3 * kC;
  // this chunk's
  IO* oc = static_cast<IO*>(a.o) + b * a.o_b + h * a.o_h + c0 * kC * a.o_t;
  const bool keep = a.ck_s && !maps;
  float* ck_s = a.ck_s + first * KP * a.Vp;
  float* ck_u = a.ck_u + first * kC * a.Vp;

  // Rows past the sequence's end are read as its last one, columns past K and V as some other: their
  // betas are 0, their rows of the state stay 0 (Turn), their values are set to 0.  Where K is no
  // multiple of 8, eight values may reach into the row behind, if there is one, and are cut off.
  uint32_t vat[NV];
  bool vin[NV], step_by_step = false;
#pragma unroll
  for (int nt = 0; nt < NV; ++nt) {
    vin[nt] = v0 + nt * 16 + r < a.V;
    vat[nt] = vin[nt] ? v0 + nt * 16 + r : 0;
  }
  uint32_t at_k, at_q, at_v[4];
  Turn<M, KP> turn;
  auto place = [&](int c) {  // where the rows of chunk c lie: of all but the last the same
    const int n = min(len - c * kC, kC);
    at_k = uint32_t(min(row, n - 1)) * uint32_t(a.k_t);
    at_q = uint32_t(min(row, n - 1)) * uint32_t(a.q_t);
#pragma unroll
    for (int x = 0; x < 4; ++x) at_v[x] = uint32_t(min(i0 + x, n - 1)) * uint32_t(a.v_t);
    turn.place(a.k_t, n);
    if (ODD) step_by_step = c + 1 >= chunks || a.k_t < a.K + 8 || a.q_t < a.K + 8;
  };
  auto row8 = [&](const IO* base, uint32_t at, int k) { return load8(base, at, k * 32 + q4 * 8, a.K, ODD && step_by_step); };
  auto load_square = [&](Both<M>(&f)[2], const Word* m, auto planes) {  // rows of T or P, which are lower
    constexpr int Q = decltype(planes)::value;
    f[0] = load_planes<M, Q>(m, row, q4 * 8);
    if (w >= 2) f[1] = load_planes<M, Q>(m, row, 32 + q4 * 8);
  };
  constexpr std::integral_constant<int, M::planes> kAll{};
  constexpr std::integral_constant<int, M::planes < 2 ? 1 : 2> kTwo{};  // of what enters o alone
  auto next = [&](int c) {  // what is loaded from now on is of chunk c
    kc += kC * a.k_t;
    qc += kC * a.q_t;
    vc += kC * a.v_t;
    tm += M::planes * kC * kC;
    pm += M::planes * kC * kC;
    dec += 3 * kC;
    if (c + 1 == chunks) place(c);
  };
  auto two_by_two = [&](auto&& step) {  // (buffers are registers: which one has to be known when it is compiled)
    for (int c = c0; c < c1; c += 2) {
      step(std::integral_constant<int, 0>{}, c);
      if (c + 1 < c1) step(std::integral_constant<int, 1>{}, c + 1);
    }
  };
  auto cut = [&](Exact<M>& f, int k) {
    if (ODD) {
      typename E::Vec x = __builtin_bit_cast(typename E::Vec, f);
      cut8(x, k * 32 + q4 * 8, a.K);
      f = exact_of<M>(x);
    }
  };

  if (chain) {
    // the state: rows 16 (MT w + m) + 4 q4 + x, columns 16 nt + r
    f32x4 S[MT][NV];
    auto state_at = [&](int m, int nt, int x) { return (int64_t(bh) * a.K + (MT * w + m) * 16 + q4 * 4 + x) * a.V + v0 + nt * 16 + r; };
    auto state_in = [&](int m, int nt, int x) { return (MT * w + m) * 16 + q4 * 4 + x < a.K && vin[nt]; };
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int nt = 0; nt < NV; ++nt)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int d = (MT * w + m) * 16 + q4 * 4 + x, v = v0 + nt * 16 + r;
          if (maps) S[m][nt][x] = d == v - a.Vp ? 1.0f : 0.0f;
          else if (a.pass == kStates && part > 0) S[m][nt][x] = a.seg_in[(seg * KP + d) * a.Vp + v];
          else S[m][nt][x] = a.s0 && state_in(m, nt, x) ? a.s0[state_at(m, nt, x)] : 0.0f;
        }
    auto put_state = [&]() {
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int nt = 0; nt < NV; ++nt) s.st.put4(nt * 16 + r, (MT * w + m) * 16 + q4 * 4, S[m][nt]);
    };
    struct Chunk {
      Exact<M> kf[KS];
      Both<M> tf[2];
      f32x4 eg, tail, beta;
      float whole;
      IO vv[NV][4];
    } in[2];
    auto load_k = [&](Chunk& n) {
#pragma unroll
      for (int k = 0; k < KS; ++k) n.kf[k] = exact_of<M>(row8(kc, at_k, k));
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int nt = 0; nt < NV; ++nt) n.vv[nt][x] = behind(vc, at_v[x] + vat[nt]);
    };
    auto load_dec = [&](Chunk& n) {
      n.eg = *reinterpret_cast<const f32x4*>(dec + i0);
      n.tail = *reinterpret_cast<const f32x4*>(dec + kC + i0);
      n.beta = *reinterpret_cast<const f32x4*>(dec + 2 * kC + i0);
      n.whole = dec[kC - 1];
    };
    if (c0 < c1) {
      place(c0);
      load_k(in[0]);
      load_square(in[0].tf, tm, kAll);
      load_dec(in[0]);
      if (c0 + 1 < c1) next(c0 + 1);
      load_k(in[1]);
      load_square(in[1].tf, tm, kAll);
      load_dec(in[1]);
      put_state();
    }
    lds_barrier();
    two_by_two([&](auto buffer, int c) {
      Chunk& n = in[decltype(buffer)::value];
      const bool more = c + 2 < c1;
#pragma unroll
      for (int k = 0; k < KS; ++k) cut(n.kf[k], k);
      if (more) next(c + 2);
      f32x4 ks[NV];
#pragma unroll
      for (int nt = 0; nt < NV; ++nt) ks[nt] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int nt = 0; nt < NV; ++nt) mma(ks[nt], n.kf[k], s.st.frag(nt * 16, k * 32));
#pragma unroll
      for (int nt = 0; nt < NV; ++nt) {
        f32x4 R;
#pragma unroll
        for (int x = 0; x < 4; ++x) R[x] = n.beta[x] * ((vin[nt] ? widen(n.vv[nt][x]) : 0.0f) - n.eg[x] * ks[nt][x]);
        s.rt.put4(nt * 16 + r, i0, R);
      }
      load_k(n);
      {
        const rsrc_t to = stores_to(ck_s, keep);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int nt = 0; nt < NV; ++nt)
#pragma unroll
            for (int x = 0; x < 4; ++x)
              put_at(to, 4 * (uint32_t((MT * w + m) * 16 + q4 * 4 + x) * uint32_t(a.Vp) + v0 + nt * 16 + r), S[m][nt][x], 0.0f);
        ck_s += KP * a.Vp;
      }
      lds_barrier();
      f32x4 U[NV];
#pragma unroll
      for (int nt = 0; nt < NV; ++nt) {
        U[nt] = f32x4{0, 0, 0, 0};
        mma(U[nt], n.tf[0], s.rt.frag(nt * 16, 0));
        if (w >= 2) mma(U[nt], n.tf[1], s.rt.frag(nt * 16, 32));
        s.us.put4(nt * 16 + r, i0, n.tail * U[nt]);
        s.ut.put4(nt * 16 + r, i0, U[nt]);
      }
      load_square(n.tf, tm, kAll);
      {
        const rsrc_t to = stores_to(ck_u, keep);
#pragma unroll
        for (int nt = 0; nt < NV; ++nt)
#pragma unroll
          for (int x = 0; x < 4; ++x) put_at(to, 4 * (uint32_t(i0 + x) * uint32_t(a.Vp) + v0 + nt * 16 + r), U[nt][x], 0.0f);
        ck_u += kC * a.Vp;
      }
      lds_barrier();
#pragma unroll
      for (int nt = 0; nt < NV; ++nt)
#pragma unroll
        for (int m = 0; m < MT; ++m) S[m][nt] *= n.whole;
      load_dec(n);
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int nt = 0; nt < NV; ++nt) {
          const Both<M> f = s.us.frag(nt * 16, k * 32);
#pragma unroll
          for (int m = 0; m < MT; ++m) mma(S[m][nt], s.kt[decltype(buffer)::value].frag((MT * w + m) * 16, k * 32), f);
        }
      put_state();  // (all have read the one before)
      lds_barrier();
    });
    if (maps) {
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int nt = 0; nt < NV; ++nt)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            a.maps[(seg * KP + (MT * w + m) * 16 + q4 * 4 + x) * (a.Vp + KP) + v0 + nt * 16 + r] = S[m][nt][x];
    } else if (a.s_last && (c0 < c1 ? c1 == chunks : c0 == 0)) {  // the segment with the sequence's end
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int nt = 0; nt < NV; ++nt)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            if (state_in(m, nt, x)) a.s_last[state_at(m, nt, x)] = S[m][nt][x];
    }
  } else if (maps) {
    if (c0 < c1) {
      place(c0);
      turn.load(kc, a.K, ODD && step_by_step);
      turn.put(s.kt[0], a.K);
      if (c0 + 1 < c1) next(c0 + 1);
      turn.load(kc, a.K, ODD && step_by_step);
    }
    lds_barrier();
    two_by_two([&](auto buffer, int c) {
      if (c + 2 < c1) next(c + 2);
      lds_barrier();
      turn.put(s.kt[1 - decltype(buffer)::value], a.K);
      turn.load(kc, a.K, ODD && step_by_step);
      lds_barrier();
      lds_barrier();
    });
  } else {
    struct Chunk {
      Exact<M> qf[KS];
      Both<M> pf[2];
      f32x4 eg;
    } in[2];
    auto load_q = [&](Chunk& n) {
#pragma unroll
      for (int k = 0; k < KS; ++k) n.qf[k] = exact_of<M>(row8(qc, at_q, k));
      n.eg = *reinterpret_cast<const f32x4*>(dec + i0);
    };
    if (c0 < c1) {
      place(c0);
      turn.load(kc, a.K, ODD && step_by_step);
      load_q(in[0]);
      load_square(in[0].pf, pm, kTwo);
      turn.put(s.kt[0], a.K);
      if (c0 + 1 < c1) next(c0 + 1);
      turn.load(kc, a.K, ODD && step_by_step);
      load_q(in[1]);
      load_square(in[1].pf, pm, kTwo);
    }
    lds_barrier();
    two_by_two([&](auto buffer, int c) {
      Chunk& m = in[decltype(buffer)::value];
      const int n = min(len - c * kC, kC);
      const bool more = c + 2 < c1;
#pragma unroll
      for (int k = 0; k < KS; ++k) cut(m.qf[k], k);
      if (more) next(c + 2);
      f32x4 o[NV];
#pragma unroll
      for (int nt = 0; nt < NV; ++nt) o[nt] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int nt = 0; nt < NV; ++nt) mma<2>(o[nt], m.qf[k], s.st.frag(nt * 16, k * 32));
#pragma unroll
      for (int nt = 0; nt < NV; ++nt) o[nt] *= a.scale * m.eg;
      load_q(m);
      lds_barrier();
      turn.put(s.kt[1 - decltype(buffer)::value], a.K);
      turn.load(kc, a.K, ODD && step_by_step);
      lds_barrier();
#pragma unroll
      for (int nt = 0; nt < NV; ++nt) {
        mma<2>(o[nt], m.pf[0], s.ut.frag(nt * 16, 0));
        if (w >= 2) mma<2>(o[nt], m.pf[1], s.ut.frag(nt * 16, 32));
      }
      load_square(m.pf, pm, kTwo);
      const rsrc_t to = stores_to(oc);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const uint32_t at = i0 + x < n ? uint32_t(i0 + x) * uint32_t(a.o_t * sizeof(IO)) : kNowhere;
#pragma unroll
        for (int nt = 0; nt < NV; ++nt) put_at(to, vin[nt] ? at + vat[nt] * uint32_t(sizeof(IO)) : kNowhere, o[nt][x], IO{});
      }
      oc += kC * a.o_t;
      lds_barrier();
    });
    if (part > 0) return;  // steps past the end
    IO* ob = static_cast<IO*>(a.o) + b * a.o_b + h * a.o_h;
    for (int64_t u = threadIdx.x - kThreads; u < int64_t(a.T - len) * BV; u += kThreads)
      if (v0 + u % BV < a.V) ob[(len + u / BV) * a.o_t + v0 + u % BV] = IO{};
  }
}

// ---------------------------------------------------------------------------
// back_scan: the states' gradients, from the last chunk down; dR, dv.  As the scan; here the
// first group has dU and dR, the second the state's gradient and the turned q and k.
// ---------------------------------------------------------------------------
template <class M, int KP, int BV>
struct BackLds {
  MatX<M, KP, kC> kt[2], qt;
  MatX<M, BV, kC> ot;
  Mat<M, BV, KP> st;
  Mat<M, BV, kC> os, ut, rt;
};

template <class M, int KP, int BV, bool ODD>
__global__ __launch_bounds__(kScanThreads) void delta_back_scan_kernel(DeltaArgs a) {
  using IO = typename M::IO;
  using Word = typename M::Word;
  using E = Eight<IO>;
  constexpr int KS = KP / 32, MT = KP / 64, NV = BV / 16;
  extern __shared__ __align__(16) char lds[];
  BackLds<M, KP, BV>& s = *reinterpret_cast<BackLds<M, KP, BV>*>(lds);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), w = wave % 4, r = lane % 16, q4 = lane / 16;
  const ScanBlock at_block = scan_block(a, KP, BV);
  const int v0 = at_block.v0, bh = at_block.bh, part = at_block.seg;
  if (bh < 0) return;
  const int b = bh / a.H, h = bh - b * a.H, hk = h / (a.H / a.Hk);
  const int len = __builtin_amdgcn_readfirstlane(length_of(a, b)), chunks = (len + kC - 1) / kC;
  const bool maps = a.pass == kMaps;
  const int c0 = part * a.per, c1 = min(chunks, c0 + a.per), end = max(c1 - 1, 0);  // the segment's chunks
  const int row = 16 * w + r, i0 = 16 * w + q4 * 4;
  const int64_t gv_t = int64_t(a.batch) * a.H * a.V, top = int64_t(bh) * a.nc + end, seg = int64_t(bh) * a.segs + part;
  // of the chunk that is loaded next
  const IO* kc = static_cast<const IO*>(a.k) + b * a.k_b + hk * a.k_h + end * kC * a.k_t;
  const IO* qc = static_cast<const IO*>(a.q) + b * a.q_b + hk * a.q_h + end * kC * a.q_t;
  const IO* goc = static_cast<const IO*>(a.go) + b * a.go_b + h * a.go_h + end * kC * a.go_t;
  const Word* tm = static_cast<const Word*>(a.tm) + top * M::planes * kC * kC;
  const Word* pm = static_cast<const Word*>(a.pm) + top * M::planes * kC * kC;
  const float* dec = a.dec + top * 3 * kC;
  uint32_t vat[NV];
  bool vin[NV], step_by_step = false;
#pragma unroll
  for (int nt = 0; nt < NV; ++nt) {
    vin[nt] = v0 + nt * 16 + r < a.V;
    vat[nt] = vin[nt] ? v0 + nt * 16 + r : 0;
  }
  uint32_t at_k, at_go[4];
  Turn<M, KP> kturn, qturn;
  auto place = [&](int c) {  // of all but the last, which comes first, the same
    const int n = min(len - c * kC, kC);
    at_k = uint32_t(min(row, n - 1)) * uint32_t(a.k_t);
#pragma unroll
    for (int x = 0; x < 4; ++x) at_go[x] = uint32_t(min(i0 + x, n - 1)) * uint32_t(a.go_t);
    kturn.place(a.k_t, n);
    qturn.place(a.q_t, n);
    if (ODD) step_by_step = c + 1 >= chunks || a.k_t < a.K + 8 || a.q_t < a.K + 8;
  };
  auto next = [&](int c) {
    kc -= kC * a.k_t;
    qc -= kC * a.q_t;
    goc -= kC * a.go_t;
    tm -= M::planes * kC * kC;
    pm -= M::planes * kC * kC;
    dec -= 3 * kC;
    if (c + 2 == c1) place(c);
  };
  if (c0 < c1) place(end);
  auto two_by_two = [&](auto&& step) {
    for (int c = c1 - 1; c >= c0; c -= 2) {
      step(std::integral_constant<int, 0>{}, c);
      if (c > c0) step(std::integral_constant<int, 1>{}, c - 1);
    }
  };

  if (wave < 4) {
    struct Chunk {
      Exact<M> kf[KS];
      Both<M> tf[2], pf[2];
      f32x4 eg, tail, beta;
    } in[2];
    IO go[NV][4];
    IO* gvc = static_cast<IO*>(a.gv) + int64_t(bh) * a.V + end * kC * gv_t;
    float* drc = a.dr + top * kC * a.Vp;
    auto load_k = [&](Chunk& n) {
#pragma unroll
      for (int k = 0; k < KS; ++k) n.kf[k] = exact_of<M>(load8(kc, at_k, k * 32 + q4 * 8, a.K, ODD && step_by_step));
    };
    auto load_go = [&]() {
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int nt = 0; nt < NV; ++nt) go[nt][x] = behind(goc, at_go[x] + vat[nt]);
    };
    auto load_square = [&](Both<M>(&f)[2], const Word* m) {  // rows of T or P turned, which are upper
      if (w < 2) f[0] = load_planes<M>(m, row, q4 * 8);
      f[1] = load_planes<M>(m, row, 32 + q4 * 8);
    };
    auto load_dec = [&](Chunk& n) {
      n.eg = *reinterpret_cast<const f32x4*>(dec + i0);
      n.tail = *reinterpret_cast<const f32x4*>(dec + kC + i0);
      n.beta = *reinterpret_cast<const f32x4*>(dec + 2 * kC + i0);
    };
    auto put_go = [&](const Chunk& n, int c) {
#pragma unroll
      for (int nt = 0; nt < NV; ++nt) {
        f32x4 os;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          if (c * kC + i0 + x >= len || !vin[nt]) go[nt][x] = IO{};
          os[x] = a.scale * n.eg[x] * widen(go[nt][x]);
        }
        s.ot.put4(nt * 16 + r, i0, E::bits(go[nt][0]), E::bits(go[nt][1]), E::bits(go[nt][2]), E::bits(go[nt][3]));
        s.os.put4(nt * 16 + r, i0, os);
      }
    };
    if (c0 < c1) {
      load_go();
      load_dec(in[0]);
      load_k(in[0]);
      load_square(in[0].pf, pm);
      load_square(in[0].tf, tm);
      put_go(in[0], end);
      if (c0 + 1 < c1) next(end - 1);
      load_go();
      load_dec(in[1]);
      load_k(in[1]);
      load_square(in[1].pf, pm);
      load_square(in[1].tf, tm);
    }
    lds_barrier();
    two_by_two([&](auto buffer, int c) {
      Chunk& m = in[decltype(buffer)::value];
      const int n = min(len - c * kC, kC);
      const bool more = c > c0 + 1;
      if (ODD) {
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          typename E::Vec x = __builtin_bit_cast(typename E::Vec, m.kf[k]);
          cut8(x, k * 32 + q4 * 8, a.K);
          m.kf[k] = exact_of<M>(x);
        }
      }
      if (more) next(c - 2);
      f32x4 U[NV];
#pragma unroll
      for (int nt = 0; nt < NV; ++nt) U[nt] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int nt = 0; nt < NV; ++nt) mma(U[nt], m.kf[k], s.st.frag(nt * 16, k * 32));
#pragma unroll
      for (int nt = 0; nt < NV; ++nt) {
        U[nt] *= m.tail;
        if (w < 2) mma(U[nt], m.pf[0], s.ot.frag(nt * 16, 0));
        mma(U[nt], m.pf[1], s.ot.frag(nt * 16, 32));
        s.ut.put4(nt * 16 + r, i0, U[nt]);
      }
      load_k(m);
      load_square(m.pf, pm);
      lds_barrier();
      f32x4 R[NV];
#pragma unroll
      for (int nt = 0; nt < NV; ++nt) {
        R[nt] = f32x4{0, 0, 0, 0};
        if (w < 2) mma(R[nt], m.tf[0], s.ut.frag(nt * 16, 0));
        mma(R[nt], m.tf[1], s.ut.frag(nt * 16, 32));
        s.rt.put4(nt * 16 + r, i0, -m.eg * m.beta * R[nt]);
      }
      load_square(m.tf, tm);
      const rsrc_t to_dr = stores_to(drc, !maps), to_gv = stores_to(gvc, !maps);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const uint32_t at = i0 + x < n ? uint32_t(i0 + x) * uint32_t(gv_t * sizeof(IO)) : kNowhere;
#pragma unroll
        for (int nt = 0; nt < NV; ++nt) {
          put_at(to_dr, 4 * (uint32_t(i0 + x) * uint32_t(a.Vp) + v0 + nt * 16 + r), R[nt][x], 0.0f);
          put_at(to_gv, vin[nt] ? at + vat[nt] * uint32_t(sizeof(IO)) : kNowhere, m.beta[x] * R[nt][x], IO{});
        }
      }
      gvc -= kC * gv_t;
      drc -= kC * a.Vp;
      load_dec(m);
      lds_barrier();
      put_go(in[1 - decltype(buffer)::value], c - 1);
      load_go();
      lds_barrier();
    });
    if (maps || part > 0) return;
    IO* gvb = static_cast<IO*>(a.gv) + int64_t(bh) * a.V;
    for (int64_t u = threadIdx.x; u < int64_t(a.T - len) * BV; u += kThreads)  // steps past the end
      if (v0 + u % BV < a.V) gvb[(len + u / BV) * gv_t + v0 + u % BV] = IO{};
  } else {
    f32x4 S[MT][NV];  // dS'
    auto state_at = [&](int m, int nt, int x) { return (int64_t(bh) * a.K + (MT * w + m) * 16 + q4 * 4 + x) * a.V + v0 + nt * 16 + r; };
    auto state_in = [&](int m, int nt, int x) { return (MT * w + m) * 16 + q4 * 4 + x < a.K && vin[nt]; };
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int nt = 0; nt < NV; ++nt)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int d = (MT * w + m) * 16 + q4 * 4 + x, v = v0 + nt * 16 + r;
          if (maps) S[m][nt][x] = d == v - a.Vp ? 1.0f : 0.0f;
          else if (a.pass == kStates && part + 1 < a.segs) S[m][nt][x] = a.seg_in[(seg * KP + d) * a.Vp + v];
          else S[m][nt][x] = a.gs_last && state_in(m, nt, x) ? a.gs_last[state_at(m, nt, x)] : 0.0f;
        }
    auto put_state = [&]() {
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int nt = 0; nt < NV; ++nt) s.st.put4(nt * 16 + r, (MT * w + m) * 16 + q4 * 4, S[m][nt]);
    };
    float whole[2] = {0.0f, 0.0f};
    float* dsc = a.ds + top * KP * a.Vp;
    if (c0 < c1) {
      kturn.load(kc, a.K, ODD && step_by_step);
      qturn.load(qc, a.K, ODD && step_by_step);
      whole[0] = dec[kC - 1];
      put_state();
      kturn.put(s.kt[0], a.K);
      qturn.put(s.qt, a.K);
      if (c0 + 1 < c1) next(end - 1);
      kturn.load(kc, a.K, ODD && step_by_step);
      qturn.load(qc, a.K, ODD && step_by_step);
      whole[1] = dec[kC - 1];
    }
    lds_barrier();
    two_by_two([&](auto buffer, int c) {
      constexpr int kNow = decltype(buffer)::value;
      const bool more = c > c0 + 1;
      if (more) next(c - 2);
      const rsrc_t to = stores_to(dsc, !maps);
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int nt = 0; nt < NV; ++nt) {
#pragma unroll
          for (int x = 0; x < 4; ++x)
            put_at(to, 4 * (uint32_t((MT * w + m) * 16 + q4 * 4 + x) * uint32_t(a.Vp) + v0 + nt * 16 + r), S[m][nt][x], 0.0f);
          S[m][nt] *= whole[kNow];
        }
      dsc -= KP * a.Vp;
      whole[kNow] = dec[kC - 1];
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int nt = 0; nt < NV; ++nt) {
          const Both<M> f = s.os.frag(nt * 16, k * 32);
#pragma unroll
          for (int m = 0; m < MT; ++m) mma(S[m][nt], s.qt.frag((MT * w + m) * 16, k * 32), f);
        }
      lds_barrier();
      // (q's products are done; k's of this chunk are not)
      kturn.put(s.kt[1 - kNow], a.K);
      qturn.put(s.qt, a.K);
      kturn.load(kc, a.K, ODD && step_by_step);
      qturn.load(qc, a.K, ODD && step_by_step);
      lds_barrier();
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int nt = 0; nt < NV; ++nt) {
          const Both<M> f = s.rt.frag(nt * 16, k * 32);
#pragma unroll
          for (int m = 0; m < MT; ++m) mma(S[m][nt], s.kt[kNow].frag((MT * w + m) * 16, k * 32), f);
        }
      put_state();
      lds_barrier();
    });
    if (maps) {
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int nt = 0; nt < NV; ++nt)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            a.maps[(seg * KP + (MT * w + m) * 16 + q4 * 4 + x) * (a.Vp + KP) + v0 + nt * 16 + r] = S[m][nt][x];
    } else if (a.gs0 && part == 0) {
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int nt = 0; nt < NV; ++nt)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            if (state_in(m, nt, x)) a.gs0[state_at(m, nt, x)] = S[m][nt][x];
    }
  }
}

// ---------------------------------------------------------------------------
// join_states: the states that enter the segments, S = M S + N from one to the next (back: from
// the last down), 16 columns of v a block, in fp32.  A wave has a quarter of the rows; the next
// segment's map is on its way meanwhile.
// ---------------------------------------------------------------------------
template <int KP>
__global__ __launch_bounds__(kThreads) void delta_join_states_kernel(DeltaArgs a, const float* from, bool back) {
  constexpr int KS = KP / 32, MT = KP / 64;
  __shared__ __align__(16) Mat<F32, 16, KP> st;
  const int lane = threadIdx.x & 63, w = threadIdx.x / 64, r = lane % 16, q4 = lane / 16;
  const int v = blockIdx.x * 16 + r, bh = blockIdx.y, ld = a.Vp + KP;
  auto map_of = [&](int n) { return a.maps + (int64_t(bh) * a.segs + (back ? a.segs - 1 - n : n)) * KP * ld; };
  f32x4 S[MT], N[MT];
  Both<F32> mf[MT][KS];
  auto load = [&](int n) {
    const float* map = map_of(n);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
#pragma unroll
      for (int k = 0; k < KS; ++k) mf[m][k] = load_both<F32>(map + int64_t((MT * w + m) * 16 + r) * ld + a.Vp + k * 32 + q4 * 8);
#pragma unroll
      for (int x = 0; x < 4; ++x) N[m][x] = map[int64_t((MT * w + m) * 16 + q4 * 4 + x) * ld + v];
    }
  };
  load(0);
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int d = (MT * w + m) * 16 + q4 * 4 + x;
      S[m][x] = from && d < a.K && v < a.V ? from[(int64_t(bh) * a.K + d) * a.V + v] : 0.0f;
    }
  for (int n = 0; n + 1 < a.segs; ++n) {
#pragma unroll
    for (int m = 0; m < MT; ++m) st.put4(r, (MT * w + m) * 16 + q4 * 4, S[m]);
    lds_barrier();
#pragma unroll
    for (int m = 0; m < MT; ++m) S[m] = N[m];
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const Both<F32> f = st.frag(0, k * 32);
#pragma unroll
      for (int m = 0; m < MT; ++m) mma(S[m], mf[m][k], f);
    }
    load(n + 2 < a.segs ? n + 1 : n);
    float* to = a.seg_in + (int64_t(bh) * a.segs + (back ? a.segs - 2 - n : n + 1)) * KP * a.Vp;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int x = 0; x < 4; ++x) to[int64_t((MT * w + m) * 16 + q4 * 4 + x) * a.Vp + v] = S[m][x];
    lds_barrier();
  }
}

// ---------------------------------------------------------------------------
// back_local: gradients of q, k, g and beta of one chunk.  Wave w has steps 16 w to + 15; sums over v
// go 32 columns at a time, through LDS, whose place E, then F, and the turned q and k take
// afterwards: two blocks a CU, one of which computes while the other waits for memory.
// ---------------------------------------------------------------------------
constexpr int kVpad = 32;      // columns of v at a time; rows in memory are filled up to a multiple
constexpr int kLocalThreads = 256;

template <class M, int KP>
struct LocalLds {
  union {
    struct {
      Mat<M, KP, kVpad> s0, ds;
      Mat<M, kC, kVpad> u;
    } a;
    struct {
      MatX<M, KP, kC> kt, qt;
      Mat<M, kC, kC> e, et;  // later F and b F
    } b;
  };
  double g[kC];
  float dg[kC], kx[kC], kd[kC], rv[kC], diag[kC], part[4];
};

template <class M, int KP>
__global__ __launch_bounds__(kLocalThreads, M::planes == 1 ? 1 : 2) void delta_back_local_kernel(DeltaArgs a) {
  using IO = typename M::IO;
  constexpr int NT = KP / 16, kQuads = KP * kVpad / 4 / kLocalThreads;  // f32x4 of a state a thread
  extern __shared__ __align__(16) char lds[];
  LocalLds<M, KP>& s = *reinterpret_cast<LocalLds<M, KP>*>(lds);
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane % 16, q4 = lane / 16;
  const int c = blockIdx.x, h = blockIdx.y, b = blockIdx.z, share = a.H / a.Hk, hk = h / share;
  const int len = length_of(a, b), t0 = c * kC, n = min(len - t0, kC), there = min(a.T - t0, kC);
  const int64_t bh = int64_t(b) * a.H + h, at = bh * a.nc + c;
  // gradients are contiguous; those of shared heads are summed by a kernel of their own
  const int64_t tk = int64_t(a.batch) * a.Hk * a.K, th = int64_t(a.batch) * a.H;
  float* part_q = share > 1 ? a.part_q + (t0 * th + bh) * a.K : nullptr;
  float* part_k = share > 1 ? a.part_k + (t0 * th + bh) * a.K : nullptr;
  IO* gq = static_cast<IO*>(a.gq) + t0 * tk + (int64_t(b) * a.Hk + hk) * a.K;
  IO* gk = static_cast<IO*>(a.gk) + t0 * tk + (int64_t(b) * a.Hk + hk) * a.K;
  IO* gg = static_cast<IO*>(a.gg) + t0 * th + bh;
  IO* gbeta = static_cast<IO*>(a.gbeta) + t0 * th + bh;
  auto put_qk = [&](int i, int d, float q, float k) {
    if (share > 1) {
      part_q[i * th * a.K + d] = q;
      part_k[i * th * a.K + d] = k;
    } else {
      gq[i * tk + d] = narrow<IO>(q);
      gk[i * tk + d] = narrow<IO>(k);
    }
  };
  // steps past the end
  for (int u = threadIdx.x + max(n, 0) * a.K; u < there * a.K; u += kLocalThreads) put_qk(u / a.K, u % a.K, 0.0f, 0.0f);
  for (int i = threadIdx.x + max(n, 0); i < there; i += kLocalThreads) gg[i * th] = gbeta[i * th] = IO{};
  if (n <= 0) return;

  const IO* kb = static_cast<const IO*>(a.k) + t0 * a.k_t + b * a.k_b + hk * a.k_h;
  const IO* qb = static_cast<const IO*>(a.q) + t0 * a.q_t + b * a.q_b + hk * a.q_h;
  const IO* vb = static_cast<const IO*>(a.v) + t0 * a.v_t + b * a.v_b + h * a.v_h;
  const IO* gob = static_cast<const IO*>(a.go) + t0 * a.go_t + b * a.go_b + h * a.go_h;
  const float *ck_s = a.ck_s + at * KP * a.Vp, *ds = a.ds + at * KP * a.Vp, *ck_u = a.ck_u + at * kC * a.Vp, *dr = a.dr + at * kC * a.Vp;
  const float* dec = a.dec + at * 3 * kC;
  const int row = 16 * w + r, i0 = 16 * w + q4 * 4;
  const float whole = dec[kC - 1];

  {
    const double G = chunk_sum<IO>(a, b, h, t0, n);
    if (w == 0) s.g[lane] = G;
  }
  f32x4 dq[NT], X[NT], Y[NT], e[4], f[4];
#pragma unroll
  for (int t = 0; t < NT; ++t) dq[t] = X[t] = Y[t] = f32x4{0, 0, 0, 0};
#pragma unroll
  for (int t = 0; t < 4; ++t) e[t] = f[t] = f32x4{0, 0, 0, 0};
  float rv = 0.0f, sds = 0.0f;  // dR.v of row `row` (a quarter of it), <S, dS'>
  for (int v0 = 0; v0 < a.Vp; v0 += kVpad) {
    f32x4 ps[kQuads], pd[kQuads], pu[2];
#pragma unroll
    for (int u = 0; u < kQuads; ++u) {
      const uint32_t i = u * kLocalThreads + threadIdx.x, from = i / 8 * uint32_t(a.Vp) + v0 + i % 8 * 4;
      ps[u] = *reinterpret_cast<const f32x4*>(&behind(ck_s, from));
      pd[u] = *reinterpret_cast<const f32x4*>(&behind(ds, from));
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint32_t i = u * kLocalThreads + threadIdx.x;
      pu[u] = *reinterpret_cast<const f32x4*>(&behind(ck_u, i / 8 * uint32_t(a.Vp) + v0 + i % 8 * 4));
    }
    // (values past V meet zeros, of U, S and dR; rows past the end are the last one's, but for do)
    typename Eight<IO>::Vec po = load8(gob, uint32_t(min(row, n - 1)) * uint32_t(a.go_t), v0 + q4 * 8, a.V, a.V % 8);
    const typename Eight<IO>::Vec pv = load8(vb, uint32_t(min(row, n - 1)) * uint32_t(a.v_t), v0 + q4 * 8, a.V, a.V % 8);
    const f32x8 pr = *reinterpret_cast<const f32x8*>(&behind(dr, uint32_t(row) * uint32_t(a.Vp) + v0 + q4 * 8));
    if (v0 > 0) lds_barrier();
#pragma unroll
    for (int u = 0; u < kQuads; ++u) {
      const int i = u * kLocalThreads + threadIdx.x;
      sds += (ps[u][0] * pd[u][0] + ps[u][1] * pd[u][1]) + (ps[u][2] * pd[u][2] + ps[u][3] * pd[u][3]);
      s.a.s0.put4(i / 8, i % 8 * 4, ps[u]);
      s.a.ds.put4(i / 8, i % 8 * 4, pd[u]);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int i = u * kLocalThreads + threadIdx.x;
      s.a.u.put4(i / 8, i % 8 * 4, pu[u]);
    }
    if (row >= n) po = 0;
    const Exact<M> of = exact_of<M>(po);
#pragma unroll
    for (int j = 0; j < 8; ++j) rv = fmaf(pr[j], Eight<IO>::wide(pv[j]), rv);
    Both<M> rf;
    both_of(pr, rf);
    lds_barrier();
    const Both<M> uf = s.a.u.frag(16 * w, 0);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const Both<M> sf = s.a.s0.frag(t * 16, 0);
      mma(dq[t], of, sf);
      mma(X[t], rf, sf);
      mma(Y[t], uf, s.a.ds.frag(t * 16, 0));
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      if (t <= w) {
        const Both<M> u2 = s.a.u.frag(t * 16, 0);
        mma(e[t], of, u2);
        mma(f[t], rf, u2);
      }
    }
  }
  Turn<M, KP> kturn, qturn;
  kturn.place(a.k_t, n);
  kturn.load(kb, a.K, a.K % 8);
  qturn.place(a.q_t, n);
  qturn.load(qb, a.K, a.K % 8);
  rv += __shfl_xor(rv, 16);
  rv += __shfl_xor(rv, 32);
  if (q4 == 0) s.rv[row] = rv;
#pragma unroll
  for (int x = 32; x > 0; x /= 2) sds += __shfl_xor(sds, x);
  if (lane == 0) s.part[w] = whole * sds;
  const f32x4 eg = *reinterpret_cast<const f32x4*>(dec + i0), tail = *reinterpret_cast<const f32x4*>(dec + kC + i0),
              beta = *reinterpret_cast<const f32x4*>(dec + 2 * kC + i0);
  lds_barrier();
  kturn.put(s.b.kt, a.K);
  qturn.put(s.b.qt, a.K);
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int j = 16 * t + r;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int i = i0 + x;
      const float d = j < i ? exp_of(s.g[i] - s.g[j]) : 0.0f;
      if (i == j) s.diag[i] = a.scale * e[t][x];
      e[t][x] = j < i ? a.scale * d * e[t][x] : 0.0f;
      f[t][x] = j < i ? -d * f[t][x] : 0.0f;
      s.b.e.put(i, j, e[t][x]);
    }
    s.b.et.put4(j, i0, e[t]);
  }
  lds_barrier();
  f32x4 kd = {0, 0, 0, 0}, Y2[NT];  // k.Y of dS' alone; the rest of Y
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    dq[t] *= a.scale * eg;
    X[t] *= -eg;
    Y[t] *= tail;
    Y2[t] = f32x4{0, 0, 0, 0};
    kd += s.b.kt.get4(t * 16 + r, i0) * Y[t];
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const Both<M> ef = s.b.e.frag(16 * w, k * 32), etf = s.b.et.frag(16 * w, k * 32);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      mma(dq[t], ef, s.b.kt.frag(t * 16, k * 32));
      mma(Y2[t], etf, s.b.qt.frag(t * 16, k * 32));
    }
  }
  lds_barrier();
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int j = 16 * t + r;
#pragma unroll
    for (int x = 0; x < 4; ++x) s.b.e.put(i0 + x, j, f[t][x]);
    s.b.et.put4(j, i0, beta * f[t]);
  }
  lds_barrier();
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const Both<M> ff = s.b.e.frag(16 * w, k * 32), ftf = s.b.et.frag(16 * w, k * 32);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const Exact<M> kf = s.b.kt.frag(t * 16, k * 32);
      mma(X[t], ff, kf);
      mma(Y2[t], ftf, kf);
    }
  }
  const f32x4 diag = *reinterpret_cast<const f32x4*>(s.diag + i0);
  f32x4 dg = {0, 0, 0, 0}, kx = {0, 0, 0, 0};
  const bool full = n == kC && a.K == KP && share == 1;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int d = t * 16 + r;
    const f32x4 k = s.b.kt.get4(d, i0), q = s.b.qt.get4(d, i0);
    dg += q * dq[t] - k * Y2[t];
    kx += k * X[t];
    const f32x4 gqv = dq[t] + diag * k, gkv = (beta * X[t] + Y[t]) + (Y2[t] + diag * q);
    if (full) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        behind(gq, uint32_t(i0 + x) * uint32_t(tk) + d) = narrow<IO>(gqv[x]);
        behind(gk, uint32_t(i0 + x) * uint32_t(tk) + d) = narrow<IO>(gkv[x]);
      }
    } else {
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (i0 + x < n && d < a.K) put_qk(i0 + x, d, gqv[x], gkv[x]);
    }
  }
  dg += beta * kx;
#pragma unroll
  for (int m = 8; m > 0; m /= 2)
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      dg[x] += __shfl_xor(dg[x], m);
      kx[x] += __shfl_xor(kx[x], m);
      kd[x] += __shfl_xor(kd[x], m);
    }
  if (r == 0) {
    *reinterpret_cast<f32x4*>(&s.dg[i0]) = dg;
    *reinterpret_cast<f32x4*>(&s.kx[i0]) = kx;
    *reinterpret_cast<f32x4*>(&s.kd[i0]) = kd;
  }
  lds_barrier();
  if (w == 0) {
    // sums from the last step down and from the first up, in 64 bits: terms cancel
    double after = s.dg[lane], upto = s.kd[lane];
    const double own = upto;
#pragma unroll
    for (int x = 1; x < 64; x *= 2) {
      const double down = __shfl_down(after, x), up = __shfl_up(upto, x);
      if (lane + x < 64) after += down;
      if (lane >= x) upto += up;
    }
    const double held = (double(s.part[0]) + double(s.part[1])) + (double(s.part[2]) + double(s.part[3]));
    if (lane < n) {
      gg[lane * th] = narrow<IO>(float(after + (upto - own) + held));
      gbeta[lane * th] = narrow<IO>(s.rv[lane] + s.kx[lane]);
    }
  }
}

// Gradients of heads of q and k that several heads of v share.
template <typename IO>
__global__ __launch_bounds__(256) void delta_join_kernel(const float* pq, const float* pk, IO* gq, IO* gk, int64_t rows, int K, int share) {
  for (int64_t u = int64_t(blockIdx.x) * 256 + threadIdx.x; u < rows * K; u += int64_t(gridDim.x) * 256) {
    const int64_t row = u / K, from = (row * share) * K + u % K;
    float q = 0.0f, k = 0.0f;
    for (int s = 0; s < share; ++s) {
      q += pq[from + int64_t(s) * K];
      k += pk[from + int64_t(s) * K];
    }
    gq[u] = narrow<IO>(q);
    gk[u] = narrow<IO>(k);
  }
}

// ---------------------------------------------------------------------------
// One token.  S^T k and S^T q come from one pass over the state, in registers:
// o = scale (a S^T q + (q.k) u).  Bound by the state's bytes.
// ---------------------------------------------------------------------------
constexpr int kStepV = 32;  // columns of a block

struct DeltaStepArgs {
  const void *q, *k, *v, *g, *beta;
  const int32_t* slots;
  float* state;
  void* o;
  int64_t q_b, q_h, k_b, k_h, v_b, v_h, g_b, g_h, beta_b, beta_h, o_b, o_h, n_slots;
  int32_t H, share, K, V;
  float scale;
};

template <typename IO>
__global__ __launch_bounds__(kThreads) void delta_step_kernel(DeltaStepArgs a) {
  const int h = blockIdx.y, b = blockIdx.z, hk = h / a.share;
  const int vl = threadIdx.x % 8 * 4, kl = threadIdx.x / 8, v = blockIdx.x * kStepV + vl;
  const int left = a.V - v;  // columns from this lane's first on
  IO* op = static_cast<IO*>(a.o) + b * a.o_b + h * a.o_h + v;
  const int64_t slot = a.slots ? a.slots[b] : b;
  if (slot < 0 || slot >= a.n_slots) {
    if (kl == 0)
      for (int x = 0; x < 4; ++x)
        if (x < left) op[x] = IO{};
    return;
  }
  float* S = a.state + ((slot * a.H + h) * a.K) * a.V + v;
  const IO* qp = static_cast<const IO*>(a.q) + b * a.q_b + hk * a.q_h;
  const IO* kp = static_cast<const IO*>(a.k) + b * a.k_b + hk * a.k_h;
  const float gl = widen(static_cast<const IO*>(a.g)[b * a.g_b + h * a.g_h]);
  const float decay = expf(gl < float(kForget) ? float(kForget) : gl), beta = widen(static_cast<const IO*>(a.beta)[b * a.beta_b + h * a.beta_h]);
  float s[4][4], kk[4];
  float sk[4] = {0, 0, 0, 0}, sq[4] = {0, 0, 0, 0}, qk = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int d = kl + 32 * i;
    const bool ok = d < a.K;
    kk[i] = ok ? widen(kp[d]) : 0.0f;
    const float q = ok ? widen(qp[d]) : 0.0f;
    if (ok && left >= 4) {
      const Pack<float, 4> p = *reinterpret_cast<const Pack<float, 4>*>(S + int64_t(d) * a.V);
#pragma unroll
      for (int x = 0; x < 4; ++x) s[i][x] = p.v[x];
    } else {
#pragma unroll
      for (int x = 0; x < 4; ++x) s[i][x] = ok && x < left ? S[int64_t(d) * a.V + x] : 0.0f;
    }
    qk = fmaf(q, kk[i], qk);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      s[i][x] *= decay;
      sk[x] = fmaf(kk[i], s[i][x], sk[x]);
      sq[x] = fmaf(q, s[i][x], sq[x]);
    }
  }
#pragma unroll
  for (int m = 8; m < 64; m *= 2) {
    qk += __shfl_xor(qk, m);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      sk[x] += __shfl_xor(sk[x], m);
      sq[x] += __shfl_xor(sq[x], m);
    }
  }
  __shared__ float red[4][8][9];
  const int w = threadIdx.x / 64, j = threadIdx.x % 8;
  if ((threadIdx.x & 63) < 8) {
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      red[w][j][x] = sk[x];
      red[w][j][4 + x] = sq[x];
    }
    red[w][j][8] = qk;
  }
  __syncthreads();
  qk = (red[0][j][8] + red[1][j][8]) + (red[2][j][8] + red[3][j][8]);
  const IO* vp = static_cast<const IO*>(a.v) + b * a.v_b + h * a.v_h + v;
  float u[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    sk[x] = (red[0][j][x] + red[1][j][x]) + (red[2][j][x] + red[3][j][x]);
    sq[x] = (red[0][j][4 + x] + red[1][j][4 + x]) + (red[2][j][4 + x] + red[3][j][4 + x]);
    u[x] = x < left ? beta * (widen(vp[x]) - sk[x]) : 0.0f;
    if (kl == 0 && x < left) op[x] = narrow<IO>(a.scale * fmaf(qk, u[x], sq[x]));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int d = kl + 32 * i;
    if (d >= a.K) continue;
    Pack<float, 4> p;
#pragma unroll
    for (int x = 0; x < 4; ++x) p.v[x] = fmaf(kk[i], u[x], s[i][x]);
    if (left >= 4) {
      *reinterpret_cast<Pack<float, 4>*>(S + int64_t(d) * a.V) = p;
    } else {
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (x < left) S[int64_t(d) * a.V + x] = p.v[x];
    }
  }
}

__global__ __launch_bounds__(256) void delta_copy_kernel(const float* from, float* to, int64_t n) {
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256) to[i] = from ? from[i] : 0.0f;
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
bool empty(const dendsn_delta_cfg* c) { return c->T == 0 || c->batch == 0 || c->H == 0; }
int64_t states(const dendsn_delta_cfg* c) { return c->batch * c->H * c->K * c->V; }
int kp_of(const dendsn_delta_cfg* c) { return c->K <= 64 ? 64 : 128; }

bool strides_fit(const dendsn_delta_cfg* c, int64_t t, int64_t b, int64_t h) {
  return t >= 0 && b >= 0 && h >= 0 && small_product(c->T, t) && small_product(c->batch, b) && small_product(c->H, h);
}

dendsn_status check_cfg(const dendsn_delta_cfg* c) {
  if (!c) return fail(DENDSN_E_INVALID, "cfg is NULL");
  if (c->T < 0 || c->T > (int64_t(1) << 24)) return fail(DENDSN_E_INVALID, "T must be in [0, 2^24]");
  if (c->batch < 0 || c->batch > 65535) return fail(DENDSN_E_INVALID, "batch must be in [0, 65535]");
  if (c->H < 0 || c->H > 65535) return fail(DENDSN_E_INVALID, "H must be in [0, 65535]");
  if (c->Hk < 0 || (c->H > 0 && (c->Hk < 1 || c->H % c->Hk)))
    return fail(DENDSN_E_INVALID, "H must be a multiple of Hk >= 1");
  if (c->K < 1 || c->V < 1 || c->V > 65536) return fail(DENDSN_E_INVALID, "K or V out of range");
  if (c->K > 128) return fail(DENDSN_E_UNSUPPORTED, "K must be <= 128");
  if (c->io != DENDSN_IO_F32 && c->io != DENDSN_IO_BF16) return fail(DENDSN_E_INVALID, "bad io");
  if (!isfinite(c->scale)) return fail(DENDSN_E_INVALID, "scale must be finite");
  // a chunk's states and the padding of V
  if (!small_product(c->batch * c->H * 128, round_up(c->T + kC, kC)) ||
      !small_product(c->batch * c->H * 128 * round_up(c->T + kC, kC) / kC * 4, round_up(c->V, kVpad)))
    return fail(DENDSN_E_INVALID, "T * batch * H * V too large");
  const int64_t s[21] = {c->q_t, c->q_b, c->q_h, c->k_t, c->k_b, c->k_h, c->v_t, c->v_b, c->v_h, c->g_t, c->g_b, c->g_h,
                         c->beta_t, c->beta_b, c->beta_h, c->o_t, c->o_b, c->o_h, c->grad_o_t, c->grad_o_b, c->grad_o_h};
  for (int i = 0; i < 21; i += 3)
    if (!strides_fit(c, s[i], s[i + 1], s[i + 2])) return fail(DENDSN_E_INVALID, "a stride is negative or too large");
  return DENDSN_OK;
}

// What holds for whole sequences besides.
dendsn_status check_sequences(const dendsn_delta_cfg* c) {
  const dendsn_status st = check_cfg(c);
  if (st != DENDSN_OK) return st;
  // a launch has fewer than 2^32 threads: blocks of 512, 16 columns of v or more
  if (round_up(c->batch * c->H, 8) > (int64_t(1) << 22) / (round_up(c->V, kVpad) / 16))
    return fail(DENDSN_E_UNSUPPORTED, "batch * H * V too large");
  // 64 steps of a tensor lie within 2^31 bytes (gradients are contiguous)
  const int64_t s[7] = {c->q_t, c->k_t, c->v_t, c->g_t, c->beta_t, c->o_t, c->grad_o_t};
  int64_t most = c->batch * c->H * (c->V > c->K ? c->V : c->K);
  for (int64_t t : s) most = t > most ? t : most;
  if (c->T > 1 && most >= (int64_t(1) << 31) / kC / (c->io == DENDSN_IO_BF16 ? 2 : 4))
    return fail(DENDSN_E_UNSUPPORTED, "64 steps of a tensor span 2^31 bytes or more");
  return DENDSN_OK;
}

// Whether the rows [V] of an output at these strides lie apart: taken from the nearest to
// the farthest, each dimension steps over all that the nearer ones span.
bool rows_apart(const dendsn_delta_cfg* c, int64_t t, int64_t b, int64_t h) {
  int64_t n[3] = {c->T, c->batch, c->H}, s[3] = {t, b, h}, span = c->V;
  for (int pass = 0; pass < 3; ++pass) {
    int least = -1;
    for (int i = 0; i < 3; ++i)
      if (n[i] > 1 && (least < 0 || s[i] < s[least])) least = i;
    if (least < 0) break;
    if (s[least] < span) return false;
    span += s[least] * (n[least] - 1);
    n[least] = 1;
  }
  return true;
}

struct DeltaPlan {
  int64_t nc, items, Vp;
  int KP;
  size_t ck_u, ckpt;                               // offset of the values, whole size
  int segs, per;                                   // of the steps, and chunks of one
  size_t tm, pm, dec, maps, seg_in, dr, ds, part_q, part_k;  // of the scratch
  size_t forward, backward;
};

constexpr int64_t kCus = 256;
using Wide = Bf<3>;    // of the scans: their states are outputs in fp32
using Narrow = Bf<2>;  // of what ends in bf16

DeltaPlan make_plan(const dendsn_delta_cfg* c) {
  DeltaPlan p{};
  if (empty(c)) return p;
  p.nc = ceil_div(c->T, kC);
  p.items = p.nc * c->batch * c->H;
  p.Vp = round_up(c->V, kVpad);
  p.KP = kp_of(c);
  Carve k;
  k.take(size_t(p.items) * p.KP * p.Vp * 4);
  p.ck_u = k.take(size_t(p.items) * kC * p.Vp * 4);
  p.ckpt = k.at;
  Carve w;
  const size_t square = size_t(kC) * kC * (c->io == DENDSN_IO_BF16 ? 2 * Wide::planes : 4);
  p.tm = w.take(size_t(p.items) * square);
  p.pm = w.take(size_t(p.items) * square);
  p.dec = w.take(size_t(p.items) * 3 * kC * 4);
  // With few heads the steps are cut into segments: the number that takes the fewest rounds of chunks,
  // a CU having one block (here: of 16 columns) at a time, where each chunk goes through both passes and
  // a join takes about
  // a chunk's time (16384 steps of 4 heads, bf16, forward: 626 us whole).
  const int64_t heads = c->batch * c->H, states = p.Vp / 16 * heads, maps = (p.Vp + p.KP) / 16 * heads;
  int64_t segs = 1, least = p.nc * ceil_div(states, kCus);
  for (int64_t n = 2; n <= 64 && 4 * n <= p.nc; ++n) {
    const int64_t rounds = ceil_div(p.nc, n) * (ceil_div(states * n, kCus) + ceil_div(maps * n, kCus)) + n;
    if (rounds < least) segs = n, least = rounds;
  }
  p.per = int(ceil_div(p.nc, segs));
  p.segs = int(ceil_div(p.nc, p.per));
  if (p.segs > 1) {
    p.maps = w.take(size_t(c->batch) * c->H * p.segs * p.KP * (p.Vp + p.KP) * 4);
    p.seg_in = w.take(size_t(c->batch) * c->H * p.segs * p.KP * p.Vp * 4);
  }
  p.forward = w.at;
  p.dr = w.take(size_t(p.items) * kC * p.Vp * 4);
  p.ds = w.take(size_t(p.items) * p.KP * p.Vp * 4);
  if (c->H != c->Hk) {
    p.part_q = w.take(size_t(c->T) * c->batch * c->H * c->K * 4);
    p.part_k = w.take(size_t(c->T) * c->batch * c->H * c->K * 4);
  }
  p.backward = w.at;
  return p;
}

void fill_args(const dendsn_delta_cfg* c, const DeltaPlan& p, void* workspace, DeltaArgs& a) {
  a.q_t = c->q_t; a.q_b = c->q_b; a.q_h = c->q_h; a.k_t = c->k_t; a.k_b = c->k_b; a.k_h = c->k_h;
  a.v_t = c->v_t; a.v_b = c->v_b; a.v_h = c->v_h; a.g_t = c->g_t; a.g_b = c->g_b; a.g_h = c->g_h;
  a.beta_t = c->beta_t; a.beta_b = c->beta_b; a.beta_h = c->beta_h; a.o_t = c->o_t; a.o_b = c->o_b; a.o_h = c->o_h;
  a.go_t = c->grad_o_t; a.go_b = c->grad_o_b; a.go_h = c->grad_o_h;
  a.T = int32_t(c->T); a.batch = int32_t(c->batch); a.H = int32_t(c->H); a.Hk = int32_t(c->Hk);
  a.K = int32_t(c->K); a.V = int32_t(c->V); a.nc = int32_t(p.nc); a.Vp = int32_t(p.Vp); a.scale = c->scale;
  char* w = static_cast<char*>(workspace);
  a.tm = w + p.tm;
  a.pm = w + p.pm;
  a.dec = reinterpret_cast<float*>(w + p.dec);
  a.maps = reinterpret_cast<float*>(w + p.maps);
  a.seg_in = reinterpret_cast<float*>(w + p.seg_in);
  a.segs = p.segs; a.per = p.per;
  a.dr = reinterpret_cast<float*>(w + p.dr);
  a.ds = reinterpret_cast<float*>(w + p.ds);
  a.part_q = reinterpret_cast<float*>(w + p.part_q);
  a.part_k = reinterpret_cast<float*>(w + p.part_k);
}

// A kernel whose LDS passes the default limit has to be told once a device; the call is cheap.
template <typename F>
bool allow_lds(F* kernel, size_t bytes) {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, int(bytes)) == hipSuccess;
}

// A scan over the steps at once, or over segments of them: their maps, the states that enter, the rest.
template <int KP, typename K>
void scan_passes(K kernel, size_t bytes, int BV, DeltaArgs a, const float* from, bool back, hipStream_t stream) {
  const int64_t heads = int64_t(a.batch) * a.H;
  auto grid = [&](int64_t cols) { return dim3(unsigned(cols / BV * round_up(heads * a.segs, 8))); };
  a.pass = kWhole;
  if (a.segs > 1) {
    a.pass = kMaps;
    kernel<<<grid(a.Vp + KP), dim3(kScanThreads), bytes, stream>>>(a);
    delta_join_states_kernel<KP><<<dim3(unsigned(a.Vp / 16), unsigned(heads)), dim3(kThreads), 0, stream>>>(a, from, back);
    a.pass = kStates;
  }
  kernel<<<grid(a.Vp), dim3(kScanThreads), bytes, stream>>>(a);
}

template <class M, int KP, int BV, bool ODD>
dendsn_status launch_scan(const DeltaArgs& a, hipStream_t stream) {
  const dim3 heads(unsigned(a.nc), unsigned(a.H), unsigned(a.batch));
  constexpr size_t bytes = sizeof(ScanLds<M, KP, BV>);
  static_assert(bytes <= 160 * 1024, "LDS of a CU");
  if (!allow_lds(delta_scan_kernel<M, KP, BV, ODD>, bytes)) return fail(DENDSN_E_HIP, "delta forward: %zu bytes of LDS refused", bytes);
  delta_local_kernel<M, KP, false><<<heads, dim3(kThreads), 0, stream>>>(a);
  scan_passes<KP>(delta_scan_kernel<M, KP, BV, ODD>, bytes, BV, a, a.s0, false, stream);
  return launched("delta forward");
}

template <class M, int KP, int BV, bool ODD>
dendsn_status launch_back_scan(const DeltaArgs& a, hipStream_t stream) {
  const dim3 heads(unsigned(a.nc), unsigned(a.H), unsigned(a.batch));
  constexpr size_t bytes = sizeof(BackLds<M, KP, BV>);
  static_assert(bytes <= 160 * 1024, "LDS of a CU");
  if (!allow_lds(delta_back_scan_kernel<M, KP, BV, ODD>, bytes)) return fail(DENDSN_E_HIP, "delta backward: %zu bytes of LDS refused", bytes);
  delta_local_kernel<M, KP, true><<<heads, dim3(kThreads), 0, stream>>>(a);
  scan_passes<KP>(delta_back_scan_kernel<M, KP, BV, ODD>, bytes, BV, a, a.gs_last, true, stream);
  return launched("delta backward");
}

template <class M, int KP>
dendsn_status launch_back_local(const DeltaArgs& a, hipStream_t stream) {
  using IO = typename M::IO;
  const dim3 heads(unsigned(a.nc), unsigned(a.H), unsigned(a.batch));
  constexpr size_t bytes = sizeof(LocalLds<M, KP>);
  static_assert(bytes <= 160 * 1024, "LDS of a CU");
  if (!allow_lds(delta_back_local_kernel<M, KP>, bytes)) return fail(DENDSN_E_HIP, "delta backward: %zu bytes of LDS refused", bytes);
  delta_back_local_kernel<M, KP><<<heads, dim3(kLocalThreads), bytes, stream>>>(a);
  if (a.H != a.Hk) {
    const int64_t rows = int64_t(a.T) * a.batch * a.Hk, blocks = ceil_div(rows * a.K, 256);
    delta_join_kernel<IO><<<dim3(unsigned(blocks < 65536 ? blocks : 65536)), dim3(256), 0, stream>>>(
        a.part_q, a.part_k, static_cast<IO*>(a.gq), static_cast<IO*>(a.gk), rows, a.K, a.H / a.Hk);
  }
  return launched("delta backward");
}

// 32 columns of v a block where that gives each CU one, else 16: what a chunk reads of q, k, T and P
// is half as much a column, but a block's chunk takes longer (16 and 32, forward and back, bf16, heads
// of 128 x 128: 32 heads of 2048 steps 102 + 116 and 129 + 155 us, 64 of 8192 steps 955 + 1023 and
// 646 + 741).  Between, from 33 to 63 such heads, 16 columns take two rounds of blocks where 32 take
// one; no measurement stands for that range, and by these figures 32 would be the faster there.
template <class M, class L, int KP, bool ODD>
dendsn_status launch(const DeltaArgs& a, bool back, hipStream_t stream) {
  const bool wide = int64_t(a.Vp / 32) * a.batch * a.H >= 256;
  if (!back) return wide ? launch_scan<M, KP, 32, ODD>(a, stream) : launch_scan<M, KP, 16, ODD>(a, stream);
  const dendsn_status st = wide ? launch_back_scan<M, KP, 32, ODD>(a, stream) : launch_back_scan<M, KP, 16, ODD>(a, stream);
  return st != DENDSN_OK ? st : launch_back_local<L, KP>(a, stream);
}

template <class M, class L>
dendsn_status launch(const DeltaArgs& a, bool back, hipStream_t stream) {
  if (a.K % 8) return a.K <= 64 ? launch<M, L, 64, true>(a, back, stream) : launch<M, L, 128, true>(a, back, stream);
  return a.K <= 64 ? launch<M, L, 64, false>(a, back, stream) : launch<M, L, 128, false>(a, back, stream);
}

dendsn_status launch(const dendsn_delta_cfg* c, const DeltaArgs& a, bool back, hipStream_t stream) {
  return c->io == DENDSN_IO_BF16 ? launch<Wide, Narrow>(a, back, stream) : launch<F32, F32>(a, back, stream);
}

dendsn_status copy_states(const dendsn_delta_cfg* c, const float* from, float* to, hipStream_t stream, const char* what) {
  const int64_t n = states(c), blocks = ceil_div(n, 256);
  if (!to || n == 0) return DENDSN_OK;
  delta_copy_kernel<<<dim3(unsigned(blocks < 4096 ? blocks : 4096)), dim3(256), 0, stream>>>(from, to, n);
  return launched(what);
}

}  // namespace
}  // namespace dendsn_seq

using namespace dendsn_seq;

extern "C" {

dendsn_status dendsn_delta_ckpt_bytes(const dendsn_delta_cfg* cfg, size_t* bytes) {
  clear_error();
  const dendsn_status st = check_sequences(cfg);
  if (st != DENDSN_OK) return st;
  if (!bytes) return fail(DENDSN_E_INVALID, "bytes is NULL");
  *bytes = make_plan(cfg).ckpt;
  return DENDSN_OK;
}

dendsn_status dendsn_delta_workspace_bytes(const dendsn_delta_cfg* cfg, int32_t backward, size_t* bytes) {
  clear_error();
  const dendsn_status st = check_sequences(cfg);
  if (st != DENDSN_OK) return st;
  if (!bytes) return fail(DENDSN_E_INVALID, "bytes is NULL");
  const DeltaPlan p = make_plan(cfg);
  *bytes = backward ? p.backward : p.forward;
  return DENDSN_OK;
}

dendsn_status dendsn_delta_forward(const dendsn_delta_cfg* cfg, const void* q, const void* k, const void* v,
                                   const void* g, const void* beta, const float* s0, const int32_t* lengths, void* o,
                                   float* s_last, void* ckpt, void* workspace, size_t workspace_bytes,
                                   hipStream_t stream) {
  clear_error();
  dendsn_status st = check_sequences(cfg);
  if (st != DENDSN_OK) return st;
  const size_t esz = cfg->io == DENDSN_IO_BF16 ? 2 : 4;
  const bool none = empty(cfg);
  if (!none && (!q || !k || !v || !g || !beta || !o)) return fail(DENDSN_E_INVALID, "q, k, v, g, beta or o is NULL");
  if (!aligned(q, esz) || !aligned(k, esz) || !aligned(v, esz) || !aligned(g, esz) || !aligned(beta, esz) || !aligned(o, esz))
    return fail(DENDSN_E_INVALID, "q, k, v, g, beta or o misaligned");
  if (!aligned(s0, 4) || !aligned(lengths, 4) || !aligned(s_last, 4)) return fail(DENDSN_E_INVALID, "s0, lengths or s_last misaligned");
  if (!aligned(ckpt, 16)) return fail(DENDSN_E_INVALID, "ckpt must be 16-byte aligned");
  if (!none && !rows_apart(cfg, cfg->o_t, cfg->o_b, cfg->o_h)) return fail(DENDSN_E_INVALID, "rows of o overlap");
  if (none) return copy_states(cfg, s0, s_last, stream, "delta forward");
  const DeltaPlan p = make_plan(cfg);
  st = check_workspace(workspace, workspace_bytes, p.forward, "dendsn_delta_workspace_bytes");
  if (st != DENDSN_OK) return st;
  DeltaArgs a{};
  fill_args(cfg, p, workspace, a);
  a.q = q; a.k = k; a.v = v; a.g = g; a.beta = beta; a.s0 = s0; a.lengths = lengths; a.o = o; a.s_last = s_last;
  if (ckpt) {
    a.ck_s = static_cast<float*>(ckpt);
    a.ck_u = reinterpret_cast<float*>(static_cast<char*>(ckpt) + p.ck_u);
  }
  return launch(cfg, a, false, stream);
}

dendsn_status dendsn_delta_backward(const dendsn_delta_cfg* cfg, const void* q, const void* k, const void* v,
                                    const void* g, const void* beta, const int32_t* lengths, const void* ckpt,
                                    const void* grad_o, const float* grad_s_last, void* grad_q, void* grad_k,
                                    void* grad_v, void* grad_g, void* grad_beta, float* grad_s0, void* workspace,
                                    size_t workspace_bytes, hipStream_t stream) {
  clear_error();
  dendsn_status st = check_sequences(cfg);
  if (st != DENDSN_OK) return st;
  const size_t esz = cfg->io == DENDSN_IO_BF16 ? 2 : 4;
  const bool none = empty(cfg);
  if (!none && (!q || !k || !v || !g || !beta || !grad_o)) return fail(DENDSN_E_INVALID, "q, k, v, g, beta or grad_o is NULL");
  if (!none && (!grad_q || !grad_k || !grad_v || !grad_g || !grad_beta)) return fail(DENDSN_E_INVALID, "a gradient of an input is NULL");
  if (!none && !ckpt) return fail(DENDSN_E_INVALID, "ckpt is NULL");
  if (!aligned(q, esz) || !aligned(k, esz) || !aligned(v, esz) || !aligned(g, esz) || !aligned(beta, esz) || !aligned(grad_o, esz))
    return fail(DENDSN_E_INVALID, "q, k, v, g, beta or grad_o misaligned");
  if (!aligned(grad_q, esz) || !aligned(grad_k, esz) || !aligned(grad_v, esz) || !aligned(grad_g, esz) || !aligned(grad_beta, esz))
    return fail(DENDSN_E_INVALID, "a gradient of an input is misaligned");
  if (!aligned(grad_s_last, 4) || !aligned(lengths, 4) || !aligned(grad_s0, 4))
    return fail(DENDSN_E_INVALID, "grad_s_last, lengths or grad_s0 misaligned");
  if (!aligned(ckpt, 16)) return fail(DENDSN_E_INVALID, "ckpt must be 16-byte aligned");
  if (none) return copy_states(cfg, grad_s_last, grad_s0, stream, "delta backward");
  const DeltaPlan p = make_plan(cfg);
  st = check_workspace(workspace, workspace_bytes, p.backward, "dendsn_delta_workspace_bytes");
  if (st != DENDSN_OK) return st;
  DeltaArgs a{};
  fill_args(cfg, p, workspace, a);
  a.q = q; a.k = k; a.v = v; a.g = g; a.beta = beta; a.lengths = lengths; a.go = grad_o; a.gs_last = grad_s_last;
  a.gq = grad_q; a.gk = grad_k; a.gv = grad_v; a.gg = grad_g; a.gbeta = grad_beta; a.gs0 = grad_s0;
  a.ck_s = static_cast<float*>(const_cast<void*>(ckpt));
  a.ck_u = reinterpret_cast<float*>(static_cast<char*>(const_cast<void*>(ckpt)) + p.ck_u);
  return launch(cfg, a, true, stream);
}

dendsn_status dendsn_delta_step(const dendsn_delta_cfg* cfg, const void* q, const void* k, const void* v,
                                const void* g, const void* beta, int64_t n_slots, const int32_t* slots, float* state,
                                void* o, hipStream_t stream) {
  clear_error();
  const dendsn_status st = check_cfg(cfg);
  if (st != DENDSN_OK) return st;
  if (cfg->T != 1) return fail(DENDSN_E_INVALID, "T must be 1");
  const size_t esz = cfg->io == DENDSN_IO_BF16 ? 2 : 4;
  const bool none = empty(cfg);
  if (n_slots < 0 || !small_product(n_slots, cfg->H * cfg->K * cfg->V)) return fail(DENDSN_E_INVALID, "n_slots negative or too large");
  if (!slots && n_slots < cfg->batch) return fail(DENDSN_E_INVALID, "without slots, n_slots must be >= batch");
  if (!none && (!q || !k || !v || !g || !beta || !o)) return fail(DENDSN_E_INVALID, "q, k, v, g, beta or o is NULL");
  if (!none && n_slots > 0 && !state) return fail(DENDSN_E_INVALID, "state is NULL");
  if (!aligned(q, esz) || !aligned(k, esz) || !aligned(v, esz) || !aligned(g, esz) || !aligned(beta, esz) || !aligned(o, esz))
    return fail(DENDSN_E_INVALID, "q, k, v, g, beta or o misaligned");
  if (!aligned(slots, 4) || !aligned(state, 4)) return fail(DENDSN_E_INVALID, "slots or state misaligned");
  if (!none && !rows_apart(cfg, cfg->o_t, cfg->o_b, cfg->o_h)) return fail(DENDSN_E_INVALID, "rows of o overlap");
  if (none) return DENDSN_OK;
  const DeltaStepArgs a{q, k, v, g, beta, slots, state, o, cfg->q_b, cfg->q_h, cfg->k_b, cfg->k_h, cfg->v_b, cfg->v_h,
                        cfg->g_b, cfg->g_h, cfg->beta_b, cfg->beta_h, cfg->o_b, cfg->o_h, n_slots,
                        int32_t(cfg->H), int32_t(cfg->H / cfg->Hk), int32_t(cfg->K), int32_t(cfg->V), cfg->scale};
  const dim3 grid(unsigned(ceil_div(cfg->V, kStepV)), unsigned(cfg->H), unsigned(cfg->batch));
  if (cfg->io == DENDSN_IO_BF16) delta_step_kernel<bf16_t><<<grid, dim3(kThreads), 0, stream>>>(a);
  else delta_step_kernel<float><<<grid, dim3(kThreads), 0, stream>>>(a);
  return launched("delta step");
}

}  // extern "C"
