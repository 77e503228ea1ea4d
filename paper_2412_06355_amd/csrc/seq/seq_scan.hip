// Gated leaky scan: forward, backward and one-token step.
//
//   a = sigmoid(g) or g,  w = 1 - a or 1,  h[t] = a[t] h[t-1] + w[t] x[t]
//   lam[t] = dh[t] + c[t],  c[t-1] = a[t] lam[t],  c[T] = dh_last
//   dx = w lam,  da = lam (h[t-1] - (leaky ? x : 0)),  dg = da a (1 - a) or da,  dh0 = c[0]
//
// Both recurrences are linear, so a run of steps acts on what enters it as
// (A, B): out = A in + B, A the product of the run's a.  A block owns 64 lanes of
// VEC channels of one sequence and walks its steps tile by tile; a tile is W waves
// of L steps, each wave's run composed in registers, the waves' runs joined
// through LDS (one barrier a tile), the state carried in registers.  Every input
// is read once.  With few channels the steps are also split over S blocks: a first
// kernel composes each block's run, and the scan starts from the runs before it.
//
// Bound by memory: bytes read once, written once, and the checkpoints (1/64 of a fp32
// state a step).  8192 steps, 8 sequences, 4096 channels in bf16: both together 826 us
// (5.2 TB/s, as a copy; under a profiler 341 and 575).  64 steps, 32 sequences: 33 us, 12.5
// and 22 under a profiler.
#include "seq_common.h"

namespace dendsn_seq {
namespace {

constexpr int kW = 8;          // waves of a block
constexpr int kL = 8;          // steps of a wave in a tile
constexpr int kTile = kW * kL; // steps between checkpoints
constexpr int kMaxSplit = 64;  // most blocks along the steps

struct ScanArgs {
  const void *x, *g, *gh;
  const float *h0, *ckpt_in, *gh_last;
  const int32_t* lengths;
  void *h, *gx, *gg;
  float *h_last, *ckpt, *gh0;
  void* runs;  // [S][batch][D] composed runs of the split (Run)
  int64_t D, x_t, x_b, g_t, g_b, h_t, h_b, gh_t, gh_b, gx_t, gx_b, gg_t, gg_b;
  int32_t T, batch, ntiles, per;  // per: tiles of a block of the split
};

// The decay and its complement, each to (|g| + 6) 2^-24 of itself: |g| 2^-24 is the rounding of
// the exponential's argument, which the smaller of the two alone carries.
template <bool SIG>
__device__ __forceinline__ void decay(float g, float& a, float& na) {
  if (SIG) {
    // e = exp(-|g|), in [0, 1]; the exponential instruction flushes results below 2^-126,
    // which a gate's gradient would lose: there its argument is raised and the result lowered
    const float y = -1.44269504f * fabsf(g);
    const bool low = y < -126.0f;
    const float e = __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f(low ? y + 64.0f : y), low ? -64 : 0);
    const float s = 1.0f + e;
    float r = __builtin_amdgcn_rcpf(s);
    r = fmaf(fmaf(-s, r, 1.0f), r, r);  // a long memory multiplies the decay's rounding
    const float q = e * r;
    a = g >= 0.0f ? r : q;
    na = g >= 0.0f ? q : r;
  } else {
    a = g;
    na = 1.0f - g;
  }
}

// A run of steps: it takes a state s to A s + b.  Sigmoid decays are at most 1, and their
// product is a number.  Decays that are given have any size: 512 steps of 1.25, or two of
// 1e20, would make A infinite, and A times a state of 0 NaN, where the recurrence has 0.  Their
// product carries its exponent beside a mantissa (16384 steps of 2000 channels in bf16, forward
// and backward: 191 us, without 184; with exponents only in tiles that need them 191 too).
template <bool SIG>
struct Run {
  float a, b;
  __device__ __forceinline__ void one() { a = 1.0f; }
  __device__ __forceinline__ void times(float f) { a *= f; }
  __device__ __forceinline__ void settle() {}
  __device__ __forceinline__ void times(const Run& r) { a *= r.a; }
  __device__ __forceinline__ float plus(float s, float add) const { return fmaf(a, s, add); }  // A s + add
  __device__ __forceinline__ float of(float s) const { return plus(s, b); }
};

template <>
struct Run<false> {
  float a, b;
  int32_t e;  // A = a 2^e
  __device__ __forceinline__ void one() { a = 1.0f, e = 0; }
  // (a halves with each at most: settle() after some eights of them)
  __device__ __forceinline__ void times(float f) {
    a *= __builtin_amdgcn_frexp_mantf(f);
    e += __builtin_amdgcn_frexp_expf(f);
  }
  // (an exponent past 2^28 is no state's any more, and 32 bits would overflow)
  __device__ __forceinline__ void settle() {
    constexpr int32_t kMost = 1 << 28;
    e = max(-kMost, min(kMost, e + __builtin_amdgcn_frexp_expf(a)));
    a = __builtin_amdgcn_frexp_mantf(a);
  }
  __device__ __forceinline__ void times(const Run& r) {  // both settled
    a *= r.a;
    e += r.e;
    settle();
  }
  __device__ __forceinline__ float plus(float s, float add) const {
    return __builtin_amdgcn_ldexpf(a * __builtin_amdgcn_frexp_mantf(s), e + __builtin_amdgcn_frexp_expf(s)) + add;
  }
  __device__ __forceinline__ float of(float s) const { return plus(s, b); }
};

// VEC values at d of the row that starts `off` elements into an array (off is the same in
// every lane, d a lane's).
template <typename IO, int VEC>
__device__ __forceinline__ Pack<IO, VEC> load_row(const void* base, int64_t off, int d) {
  return *reinterpret_cast<const Pack<IO, VEC>*>(static_cast<const IO*>(base) + off + d);
}
template <typename IO, int VEC>
__device__ __forceinline__ void store_row(void* base, int64_t off, int d, const Pack<IO, VEC>& v) {
  *reinterpret_cast<Pack<IO, VEC>*>(static_cast<IO*>(base) + off + d) = v;
}

__device__ __forceinline__ int seq_length(const ScanArgs& p, int b) {
  if (!p.lengths) return p.T;
  return max(0, min(p.T, p.lengths[b]));
}

// A barrier for what waves wrote to LDS: loads and stores of global memory stay in flight.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt 0
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Composes the run of one block of the split: (A, B) over its steps, forward
// (u = w x) or backward (c[t-1] = a[t] (dh[t] + c[t])).  16384 steps of 2000 channels in
// bf16 (131 MB): 38 us forward, 32 us backward.  The scan then reads the same bytes from
// the 256 MB cache; blocks that wait for the runs before them instead of this kernel
// (one read of the inputs) took 83 + 140 us for both scans, against 89 + 119 with it.
template <typename IO, int VEC, bool SIG, bool LEAKY, bool BWD>
__global__ void __launch_bounds__(kW * 64) scan_runs_kernel(ScanArgs p) {
  __shared__ Run<SIG> sh[kW][64 * VEC];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int b = blockIdx.y;
  const int seg = BWD ? int(blockIdx.z) + 1 : int(blockIdx.z);  // the first (last) block's run feeds nobody
  const int d0 = int((blockIdx.x * 64 + lane) * VEC);
  const bool on = d0 < p.D;
  const int d = on ? min(d0, int(p.D) - VEC) : 0;  // (an odd row's last lane shares a channel)
  const int len = seq_length(p, b);
  const int lo = seg * p.per * kTile, hi = min(min(lo + p.per * kTile, p.T), len);
  // wave w composes the steps [s0, s1)
  const int each = p.per * kL;
  const int s0 = lo + w * each, s1 = min(s0 + each, hi);
  const int64_t xb = b * (BWD ? p.gh_b : p.x_b), gb = b * p.g_b;
  const void* xs = BWD ? p.gh : p.x;
  const int64_t xt = BWD ? p.gh_t : p.x_t;
  Run<SIG> r[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) r[v].one(), r[v].b = 0.0f;
  const int n = s1 - s0;
  for (int j0 = 0; j0 < n; j0 += kL) {  // (loads further ahead than this measured no faster)
    Pack<IO, VEC> rx[kL], rg[kL];
#pragma unroll
    for (int j = 0; j < kL; ++j) {
      const int i = min(j0 + j, n - 1);
      const int64_t t = BWD ? s1 - 1 - i : s0 + i;
      rx[j] = load_row<IO, VEC>(xs, t * xt + xb, d);
      rg[j] = load_row<IO, VEC>(p.g, t * p.g_t + gb, d);
    }
#pragma unroll
    for (int j = 0; j < kL; ++j) {
      const bool in = j0 + j < n;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        float a, na;
        decay<SIG>(widen(rg[j].v[v]), a, na);
        const float xv = widen(rx[j].v[v]);
        const float next = BWD ? a * (xv + r[v].b) : fmaf(a, r[v].b, LEAKY ? na * xv : xv);
        r[v].b = in ? next : r[v].b;
        r[v].times(in ? a : 1.0f);
      }
    }
#pragma unroll
    for (int v = 0; v < VEC; ++v) r[v].settle();
  }
#pragma unroll
  for (int v = 0; v < VEC; ++v) sh[w][v * 64 + lane] = r[v];
  __syncthreads();
  if (w == 0 && on) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      Run<SIG> c = sh[BWD ? kW - 1 : 0][v * 64 + lane];
      for (int k = 1; k < kW; ++k) {
        const Run<SIG> next = sh[BWD ? kW - 1 - k : k][v * 64 + lane];
        c.b = next.of(c.b);
        c.times(next);
      }
      static_cast<Run<SIG>*>(p.runs)[(int64_t(seg) * p.batch + b) * p.D + d + v] = c;
    }
  }
}

// What enters block `to` of the split, from what entered block `from`: the runs between,
// in the order of `step`, sixteen (of three words: eight) at a time in flight.
template <int VEC, bool SIG>
__device__ __forceinline__ void enter(float (&carry)[VEC], const Run<SIG>* runs, int64_t lanes, int from, int to, int step) {
  constexpr int U = SIG ? 16 : 8;
  for (int s0 = from; s0 != to; s0 += step * min(U, (to - s0) * step)) {
    Run<SIG> r[U][VEC];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = (to - s0) * step > u ? s0 + u * step : s0;
#pragma unroll
      for (int v = 0; v < VEC; ++v) r[u][v] = runs[s * lanes + v];
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if ((to - s0) * step > u)
#pragma unroll
        for (int v = 0; v < VEC; ++v) carry[v] = r[u][v].of(carry[v]);
  }
}

// Two tiles' inputs are in flight while a third is worked on; a wave's eight steps are
// composed, the eight waves' runs exchanged, and the states written from registers.
// W > 0: all steps are one tile of W waves, kW / W of them (of other channels) a block, and
// nothing is in flight beside it.  With blocks of a tile, as for long sequences, 256
// sequences of 4096 channels in bf16 took 56 us forward and 134 backward for one step, 10
// and 14 so; 64 steps of 512 x 1000 in fp32 115 and 181, 90 and 162 so.
template <typename IO, int VEC, bool SIG, bool LEAKY, int W>
__global__ void __launch_bounds__(kW * 64, W || sizeof(IO) == 2 ? 4 : 2) scan_fwd_kernel(ScanArgs p) {
  constexpr bool ONE = W > 0;
  constexpr int N = ONE ? W : kW;  // waves of a tile
  __shared__ Run<SIG> sh[ONE ? 1 : 2][kW][64 * VEC];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int w = N < kW ? wave % N : wave, first = N < kW ? wave - w : 0;  // in its tile; its tile's first
  const int b = blockIdx.y, seg = blockIdx.z;
  const int d0 = int(((N < kW ? blockIdx.x * (kW / N) + wave / N : blockIdx.x) * 64 + lane) * VEC);
  const bool on = d0 < p.D;
  const int d = on ? min(d0, int(p.D) - VEC) : 0;  // (an odd row's last lane shares a channel)
  const int len = seq_length(p, b);
  const int64_t xb = b * p.x_b, gb = b * p.g_b, hb = b * p.h_b;
  const int64_t bd = int64_t(b) * p.D + d, lanes = int64_t(p.batch) * p.D;

  float carry[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) carry[v] = p.h0 ? p.h0[bd + v] : 0.0f;
  if (!ONE) enter<VEC, SIG>(carry, static_cast<const Run<SIG>*>(p.runs) + bd, lanes, 0, seg, 1);

  const int k0 = ONE ? 0 : seg * p.per, k1 = ONE ? 1 : min(k0 + p.per, p.ntiles);
  struct Raw {
    Pack<IO, VEC> x[kL], g[kL];
  };
  auto fetch = [&](Raw& r, int k) {  // rows past the end read the last row again
    const int t0 = k * kTile + w * kL;
    if (k < k1 && t0 < len) {
#pragma unroll
      for (int j = 0; j < kL; ++j) {
        const int64_t t = min(t0 + j, p.T - 1);
        r.x[j] = load_row<IO, VEC>(p.x, t * p.x_t + xb, d);
        r.g[j] = load_row<IO, VEC>(p.g, t * p.g_t + gb, d);
      }
    }
  };
  // WHOLE: all of the wave's steps belong to the sequence
  auto tile = [&](auto whole, Raw& raw, int k, int buf) {
    constexpr bool WHOLE = decltype(whole)::value;
    const int t0 = k * kTile + w * kL;
    // what takes the state before the wave's steps to the one after step j, A s + b; where decays
    // are given, the state before that step (the products of several may be no numbers)
    float P[kL][VEC], H[kL][VEC];
    Run<SIG> run[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) run[v].one(), run[v].b = 0.0f;
#pragma unroll
    for (int j = 0; j < kL; ++j) {
      const bool in = WHOLE || t0 + j < len;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        float a, na;
        decay<SIG>(widen(raw.g[j].v[v]), a, na);
        const float xv = widen(raw.x[j].v[v]);
        const float u = LEAKY ? na * xv : xv, next = fmaf(a, run[v].b, u);
        run[v].times(in ? a : 1.0f);
        run[v].b = in ? next : run[v].b;
        P[j][v] = SIG ? run[v].a : in ? a : 1.0f;
        H[j][v] = SIG ? run[v].b : in ? u : 0.0f;
      }
    }
    if (!ONE) fetch(raw, k + 2);
    if (N > 1) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) sh[buf][wave][v * 64 + lane] = run[v];
      lds_barrier();
    }
    float in[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      if (w == 0 && on && p.ckpt) p.ckpt[int64_t(k) * lanes + bd + v] = carry[v];
      in[v] = carry[v];
#pragma unroll
      for (int q = 0; q < N; ++q) {
        const Run<SIG> r = N > 1 ? sh[buf][first + q][v * 64 + lane] : run[v];
        if (q == w) in[v] = carry[v];
        carry[v] = r.of(carry[v]);
      }
    }
    if (on) {
#pragma unroll
      for (int j = 0; j < kL; ++j) {
        const int t = t0 + j;
        Pack<IO, VEC> o;
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          const float state = fmaf(P[j][v], in[v], H[j][v]);
          if (!SIG) in[v] = state;
          o.v[v] = narrow<IO>(WHOLE || t < len ? state : 0.0f);
        }
        if (WHOLE || t < p.T) store_row<IO, VEC>(p.h, t * p.h_t + hb, d, o);
      }
    }
  };
  auto either = [&](Raw& raw, int k, int buf) {
    if (k * kTile + (w + 1) * kL <= len) tile(std::true_type{}, raw, k, buf);
    else tile(std::false_type{}, raw, k, buf);
  };
  Raw ra, rb;  // a tile's loads are two tiles ahead of its use
  fetch(ra, k0);
  if (ONE) {
    either(ra, 0, 0);
  } else {
    fetch(rb, k0 + 1);
    for (int k = k0; k < k1; k += 2) {
      either(ra, k, 0);
      if (k + 1 < k1) either(rb, k + 1, 1);
    }
  }
  if (w == 0 && on && p.h_last && k1 == p.ntiles && k0 < k1) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) p.h_last[bd + v] = carry[v];
  }
}

// From the last tile to the first: the tile's states are computed again from its
// checkpoint, so that h is not read (it would cost as much as x, and is rounded in bf16),
// the gradient's runs are exchanged beside the states', and the next tile's inputs are in
// flight meanwhile.
template <typename IO, int VEC, bool SIG, bool LEAKY, int W>
__global__ void __launch_bounds__(kW * 64, 2) scan_bwd_kernel(ScanArgs p) {
  constexpr bool ONE = W > 0;  // as in the forward
  constexpr int N = ONE ? W : kW, S = ONE ? 1 : 2;
  __shared__ Run<SIG> shH[S][kW][64 * VEC];  // the states' runs; the gradient's have their products
  __shared__ float shC[S][kW][64 * VEC];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int w = N < kW ? wave % N : wave, first = N < kW ? wave - w : 0;  // in its tile; its tile's first
  const int b = blockIdx.y, seg = blockIdx.z;
  const int d0 = int(((N < kW ? blockIdx.x * (kW / N) + wave / N : blockIdx.x) * 64 + lane) * VEC);
  const bool on = d0 < p.D;
  const int d = on ? min(d0, int(p.D) - VEC) : 0;  // (an odd row's last lane shares a channel)
  const int len = seq_length(p, b);
  const int64_t xb = b * p.x_b, gb = b * p.g_b, ghb = b * p.gh_b, gxb = b * p.gx_b, ggb = b * p.gg_b;
  const int64_t bd = int64_t(b) * p.D + d, lanes = int64_t(p.batch) * p.D;

  float carry[VEC];  // c of the tile's last step
#pragma unroll
  for (int v = 0; v < VEC; ++v) carry[v] = p.gh_last ? p.gh_last[bd + v] : 0.0f;
  if (!ONE) enter<VEC, SIG>(carry, static_cast<const Run<SIG>*>(p.runs) + bd, lanes, int(gridDim.z) - 1, seg, -1);

  const int k0 = ONE ? 0 : seg * p.per, k1 = ONE ? 1 : min(k0 + p.per, p.ntiles);
  struct Raw {
    Pack<IO, VEC> x[kL], g[kL], h[kL];
    float start[VEC];
  };
  auto fetch = [&](Raw& r, int k) {
    if (k < k0) return;
    const int t0 = k * kTile + w * kL;
#pragma unroll
    for (int v = 0; v < VEC; ++v) r.start[v] = p.ckpt_in[int64_t(k) * lanes + bd + v];
    if (t0 < len) {
#pragma unroll
      for (int j = 0; j < kL; ++j) {
        const int64_t t = min(t0 + j, p.T - 1);
        r.x[j] = load_row<IO, VEC>(p.x, t * p.x_t + xb, d);
        r.g[j] = load_row<IO, VEC>(p.g, t * p.g_t + gb, d);
        r.h[j] = load_row<IO, VEC>(p.gh, t * p.gh_t + ghb, d);
      }
    }
  };
  auto tile = [&](auto whole, Raw& raw, int k, int buf) {
    constexpr bool WHOLE = decltype(whole)::value;
    const int t0 = k * kTile + w * kL;
    float a[kL][VEC], na[kL][VEC], x[kL][VEC], dh[kL][VEC];
    Run<SIG> H[VEC];
    float C[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) H[v].one(), H[v].b = 0.0f, C[v] = 0.0f;
#pragma unroll
    for (int j = 0; j < kL; ++j) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const bool in = WHOLE || t0 + j < len;
        float av, nav;
        decay<SIG>(widen(raw.g[j].v[v]), av, nav);
        a[j][v] = in ? av : 1.0f;
        na[j][v] = in ? nav : 0.0f;
        x[j][v] = in ? widen(raw.x[j].v[v]) : 0.0f;
        dh[j][v] = in ? widen(raw.h[j].v[v]) : 0.0f;
        H[v].times(a[j][v]);
        H[v].b = fmaf(a[j][v], H[v].b, LEAKY ? na[j][v] * x[j][v] : x[j][v]);
      }
    }
#pragma unroll
    for (int j = kL - 1; j >= 0; --j) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) C[v] = a[j][v] * (dh[j][v] + C[v]);
    }
    float hin[VEC], cin[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      hin[v] = raw.start[v];
      if (N > 1) {
        shH[buf][wave][v * 64 + lane] = H[v];
        shC[buf][wave][v * 64 + lane] = C[v];
      }
    }
    if (!ONE) fetch(raw, k - 1);
    if (N > 1) lds_barrier();
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      const int at = v * 64 + lane;
#pragma unroll
      for (int q = 0; q < N - 1; ++q)
        if (q < w) hin[v] = shH[buf][first + q][at].of(hin[v]);
      cin[v] = carry[v];
#pragma unroll
      for (int q = N - 1; q >= 0; --q) {
        if (q == w) cin[v] = carry[v];
        carry[v] = N > 1 ? shH[buf][first + q][at].plus(carry[v], shC[buf][first + q][at]) : H[v].plus(carry[v], C[v]);
      }
    }
    float before[kL][VEC];
#pragma unroll
    for (int j = 0; j < kL; ++j) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        before[j][v] = hin[v];
        hin[v] = fmaf(a[j][v], hin[v], LEAKY ? na[j][v] * x[j][v] : x[j][v]);
      }
    }
#pragma unroll
    for (int j = kL - 1; j >= 0; --j) {
      const int t = t0 + j;
      Pack<IO, VEC> ox, og;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const float lam = dh[j][v] + cin[v];
        cin[v] = a[j][v] * lam;
        float da = lam * (LEAKY ? before[j][v] - x[j][v] : before[j][v]);
        if (SIG) da *= a[j][v] * na[j][v];
        ox.v[v] = narrow<IO>(WHOLE || t < len ? (LEAKY ? na[j][v] * lam : lam) : 0.0f);
        og.v[v] = narrow<IO>(WHOLE || t < len ? da : 0.0f);
      }
      if (on && (WHOLE || t < p.T)) {
        store_row<IO, VEC>(p.gx, t * p.gx_t + gxb, d, ox);
        store_row<IO, VEC>(p.gg, t * p.gg_t + ggb, d, og);
      }
    }
  };
  auto either = [&](Raw& raw, int k, int buf) {
    if (k * kTile + (w + 1) * kL <= len) tile(std::true_type{}, raw, k, buf);
    else tile(std::false_type{}, raw, k, buf);
  };
  Raw raw;  // (two tiles ahead, as in the forward, the registers do not reach)
  fetch(raw, k1 - 1);
  for (int k = k1 - 1; k >= k0; --k) either(raw, k, ONE ? 0 : k & 1);
  if (w == 0 && on && p.gh0 && seg == 0) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) p.gh0[bd + v] = carry[v];
  }
}

struct StepArgs {
  const void *x, *g;
  const int32_t* slots;
  float* state;
  void* h;
  int64_t D, x_b, g_b, h_b, n_slots;
};

// One token of each request: VEC channels a thread, the state read and written
// where it lies.  64 requests of 4096 channels move 3.7 MB in 2.7 us, a launch's latency.
template <typename IO, int VEC, bool SIG, bool LEAKY>
__global__ void __launch_bounds__(256) scan_step_kernel(StepArgs p) {
  const int64_t d = (int64_t(blockIdx.x) * 256 + threadIdx.x) * VEC;
  const int b = blockIdx.y;
  if (d >= p.D) return;
  const int64_t slot = p.slots ? int64_t(p.slots[b]) : b;
  const bool live = slot >= 0 && slot < p.n_slots;
  Pack<IO, VEC> o;
#pragma unroll
  for (int v = 0; v < VEC; ++v) o.v[v] = narrow<IO>(0.0f);
  if (live) {
    const Pack<IO, VEC> rx = load_row<IO, VEC>(p.x, b * p.x_b, int(d)), rg = load_row<IO, VEC>(p.g, b * p.g_b, int(d));
    auto* st = reinterpret_cast<Pack<float, VEC>*>(p.state + slot * p.D + d);
    Pack<float, VEC> s = *st;
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      float a, na;
      decay<SIG>(widen(rg.v[v]), a, na);
      const float xv = widen(rx.v[v]);
      s.v[v] = fmaf(a, s.v[v], LEAKY ? na * xv : xv);
      o.v[v] = narrow<IO>(s.v[v]);
    }
    *st = s;
  }
  *reinterpret_cast<Pack<IO, VEC>*>(static_cast<IO*>(p.h) + b * p.h_b + d) = o;
}

// T = 0: the state passes through.
__global__ void __launch_bounds__(256) scan_copy_kernel(const float* from, float* to, int64_t n) {
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256)
    to[i] = from ? from[i] : 0.0f;
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
bool rows_apart(const dendsn_scan_cfg* c, int64_t st, int64_t sb) {
  // every two rows of [T, batch] are at least D apart
  if (c->T > 1 && st < c->D) return false;
  if (c->batch > 1 && sb < c->D) return false;
  if (c->T <= 1 || c->batch <= 1) return true;
  return st >= (c->batch - 1) * sb + c->D || sb >= (c->T - 1) * st + c->D;
}

bool strides_fit(const dendsn_scan_cfg* c, int64_t st, int64_t sb) {
  return st >= 0 && sb >= 0 && st <= kMaxElems && sb <= kMaxElems && small_product(c->T, st) &&
         small_product(c->batch, sb);
}

bool empty(const dendsn_scan_cfg* c) { return c->T == 0 || c->batch == 0 || c->D == 0; }

dendsn_status check_cfg(const dendsn_scan_cfg* c) {
  if (!c) return fail(DENDSN_E_INVALID, "cfg is NULL");
  if (c->T < 0 || c->T > (int64_t(1) << 30)) return fail(DENDSN_E_INVALID, "T must be in [0, 2^30]");
  if (c->batch < 0 || c->batch > 65535) return fail(DENDSN_E_INVALID, "batch must be in [0, 65535]");
  // a launch has fewer than 2^32 threads along the channels: eight of them each
  if (c->D < 0 || c->D > (int64_t(1) << 27)) return fail(DENDSN_E_INVALID, "D must be in [0, 2^27]");
  if (c->io != DENDSN_IO_F32 && c->io != DENDSN_IO_BF16) return fail(DENDSN_E_INVALID, "bad io");
  if (c->gate != DENDSN_GATE_SIGMOID && c->gate != DENDSN_GATE_DECAY) return fail(DENDSN_E_INVALID, "bad gate");
  if (c->leaky != 0 && c->leaky != 1) return fail(DENDSN_E_INVALID, "leaky must be 0 or 1");
  if (!small_product(c->batch * c->D, c->T)) return fail(DENDSN_E_INVALID, "T * batch * D too large");
  const int64_t s[12] = {c->x_t, c->x_b, c->g_t, c->g_b, c->h_t, c->h_b, c->grad_h_t, c->grad_h_b,
                         c->grad_x_t, c->grad_x_b, c->grad_g_t, c->grad_g_b};
  for (int i = 0; i < 12; i += 2)
    if (!strides_fit(c, s[i], s[i + 1])) return fail(DENDSN_E_INVALID, "a stride is negative or too large");
  return DENDSN_OK;
}

struct Plan {
  int vec;
  int64_t groups;  // blocks along the channels
  int ntiles, per, S;
  int one;         // waves of the only tile; 0: several tiles
};

// Lanes of two channels (4 or 8 bytes a lane).  With fewer blocks than CUs the steps are
// split, to kFill blocks (16384 steps of 2000 channels, forward and backward with kFill of
// 256 / 512 / 1024: 242 / 228 / 243 us).
constexpr int64_t kCus = 256, kFill = 512;

Plan make_plan(const dendsn_scan_cfg* c) {
  Plan p;
  p.vec = c->D >= 2 ? 2 : 1;
  p.groups = ceil_div(c->D, 64 * p.vec);
  p.ntiles = int(ceil_div(c->T, kTile));
  p.one = c->T > kTile ? 0 : c->T > 4 * kL ? 8 : c->T > 2 * kL ? 4 : c->T > kL ? 2 : 1;
  const int64_t blocks = p.groups * c->batch;
  int64_t S = blocks >= kCus ? 1 : ceil_div(kFill, blocks);
  S = S < kMaxSplit ? S : kMaxSplit;
  // a block of the split has two tiles at least
  S = S < p.ntiles / 2 ? S : p.ntiles / 2;
  if (S < 1) S = 1;
  p.per = int(ceil_div(p.ntiles, S));
  p.S = int(ceil_div(p.ntiles, p.per));
  return p;
}

size_t runs_bytes(const dendsn_scan_cfg* c) {
  const Plan p = make_plan(c);
  const size_t run = c->gate == DENDSN_GATE_SIGMOID ? sizeof(Run<true>) : sizeof(Run<false>);
  return p.S > 1 ? size_t(p.S) * size_t(c->batch) * size_t(c->D) * run : 0;
}

size_t ckpt_bytes(const dendsn_scan_cfg* c) {
  return empty(c) ? 0 : size_t(ceil_div(c->T, kTile)) * size_t(c->batch) * size_t(c->D) * sizeof(float);
}

template <typename F>
void dispatch(const dendsn_scan_cfg* c, bool wide, F&& f) {
  auto flags = [&](auto io, auto vec) {
    using IO = decltype(io);
    constexpr int V = decltype(vec)::value;
    if (c->gate == DENDSN_GATE_SIGMOID) {
      if (c->leaky) f.template operator()<IO, V, true, true>();
      else f.template operator()<IO, V, true, false>();
    } else {
      if (c->leaky) f.template operator()<IO, V, false, true>();
      else f.template operator()<IO, V, false, false>();
    }
  };
  auto width = [&](auto io) {
    if (wide) flags(io, std::integral_constant<int, 2>{});
    else flags(io, std::integral_constant<int, 1>{});
  };
  if (c->io == DENDSN_IO_BF16) width(bf16_t{});
  else width(float{});
}

struct LaunchFwd {
  ScanArgs a;
  Plan p;
  hipStream_t stream;
  template <typename IO, int V, bool SIG, bool LEAKY>
  void operator()() const {
    const dim3 block(kW * 64);
    if (p.S > 1)
      scan_runs_kernel<IO, V, SIG, LEAKY, false><<<dim3(unsigned(p.groups), a.batch, p.S - 1), block, 0, stream>>>(a);
    const dim3 grid(unsigned(ceil_div(p.groups, p.one ? kW / p.one : 1)), a.batch, p.S);
    if (p.one == 1) scan_fwd_kernel<IO, V, SIG, LEAKY, 1><<<grid, block, 0, stream>>>(a);
    else if (p.one == 2) scan_fwd_kernel<IO, V, SIG, LEAKY, 2><<<grid, block, 0, stream>>>(a);
    else if (p.one == 4) scan_fwd_kernel<IO, V, SIG, LEAKY, 4><<<grid, block, 0, stream>>>(a);
    else if (p.one == 8) scan_fwd_kernel<IO, V, SIG, LEAKY, 8><<<grid, block, 0, stream>>>(a);
    else scan_fwd_kernel<IO, V, SIG, LEAKY, 0><<<grid, block, 0, stream>>>(a);
  }
};

struct LaunchBwd {
  ScanArgs a;
  Plan p;
  hipStream_t stream;
  template <typename IO, int V, bool SIG, bool LEAKY>
  void operator()() const {
    const dim3 block(kW * 64);
    if (p.S > 1)
      scan_runs_kernel<IO, V, SIG, LEAKY, true><<<dim3(unsigned(p.groups), a.batch, p.S - 1), block, 0, stream>>>(a);
    const dim3 grid(unsigned(ceil_div(p.groups, p.one ? kW / p.one : 1)), a.batch, p.S);
    if (p.one == 1) scan_bwd_kernel<IO, V, SIG, LEAKY, 1><<<grid, block, 0, stream>>>(a);
    else if (p.one == 2) scan_bwd_kernel<IO, V, SIG, LEAKY, 2><<<grid, block, 0, stream>>>(a);
    else if (p.one == 4) scan_bwd_kernel<IO, V, SIG, LEAKY, 4><<<grid, block, 0, stream>>>(a);
    else if (p.one == 8) scan_bwd_kernel<IO, V, SIG, LEAKY, 8><<<grid, block, 0, stream>>>(a);
    else scan_bwd_kernel<IO, V, SIG, LEAKY, 0><<<grid, block, 0, stream>>>(a);
  }
};

struct LaunchStep {
  StepArgs a;
  int64_t batch;
  hipStream_t stream;
  template <typename IO, int V, bool SIG, bool LEAKY>
  void operator()() const {
    scan_step_kernel<IO, V, SIG, LEAKY>
        <<<dim3(unsigned(ceil_div(a.D, 256 * V)), unsigned(batch)), dim3(256), 0, stream>>>(a);
  }
};

}  // namespace
}  // namespace dendsn_seq

using namespace dendsn_seq;

extern "C" {

dendsn_status dendsn_scan_ckpt_bytes(const dendsn_scan_cfg* cfg, size_t* bytes) {
  clear_error();
  const dendsn_status st = check_cfg(cfg);
  if (st != DENDSN_OK) return st;
  if (!bytes) return fail(DENDSN_E_INVALID, "bytes is NULL");
  *bytes = ckpt_bytes(cfg);
  return DENDSN_OK;
}

dendsn_status dendsn_scan_workspace_bytes(const dendsn_scan_cfg* cfg, int32_t backward, size_t* bytes) {
  clear_error();
  const dendsn_status st = check_cfg(cfg);
  if (st != DENDSN_OK) return st;
  if (!bytes) return fail(DENDSN_E_INVALID, "bytes is NULL");
  (void)backward;  // both directions split alike
  *bytes = empty(cfg) ? 0 : runs_bytes(cfg);
  return DENDSN_OK;
}

dendsn_status dendsn_scan_forward(const dendsn_scan_cfg* cfg, const void* x, const void* g, const float* h0,
                                  const int32_t* lengths, void* h, float* h_last, float* ckpt, void* workspace,
                                  size_t workspace_bytes, hipStream_t stream) {
  clear_error();
  dendsn_status st = check_cfg(cfg);
  if (st != DENDSN_OK) return st;
  const bool none = empty(cfg);
  const size_t esz = cfg->io == DENDSN_IO_BF16 ? 2 : 4;
  if (!none && (!x || !g || !h)) return fail(DENDSN_E_INVALID, "x, g or h is NULL");
  if (!aligned(x, esz) || !aligned(g, esz) || !aligned(h, esz)) return fail(DENDSN_E_INVALID, "x, g or h misaligned");
  if (!aligned(h0, 4) || !aligned(lengths, 4) || !aligned(h_last, 4))
    return fail(DENDSN_E_INVALID, "h0, lengths or h_last misaligned");
  if (!aligned(ckpt, 16)) return fail(DENDSN_E_INVALID, "ckpt must be 16-byte aligned");
  if (!none && !rows_apart(cfg, cfg->h_t, cfg->h_b)) return fail(DENDSN_E_INVALID, "rows of h overlap");
  if (none) {
    const int64_t lanes = cfg->batch * cfg->D;
    if (h_last && lanes) {
      scan_copy_kernel<<<dim3(unsigned(ceil_div(lanes, 256) < 4096 ? ceil_div(lanes, 256) : 4096)), dim3(256), 0, stream>>>(h0, h_last, lanes);
      return launched("scan forward");
    }
    return DENDSN_OK;
  }
  st = check_workspace(workspace, workspace_bytes, runs_bytes(cfg), "dendsn_scan_workspace_bytes");
  if (st != DENDSN_OK) return st;
  LaunchFwd f{{}, make_plan(cfg), stream};
  ScanArgs& a = f.a;
  a.x = x; a.g = g; a.h0 = h0; a.lengths = lengths; a.h = h; a.h_last = h_last; a.ckpt = ckpt;
  a.runs = workspace;
  a.D = cfg->D; a.T = int32_t(cfg->T); a.batch = int32_t(cfg->batch); a.ntiles = f.p.ntiles; a.per = f.p.per;
  a.x_t = cfg->x_t; a.x_b = cfg->x_b; a.g_t = cfg->g_t; a.g_b = cfg->g_b; a.h_t = cfg->h_t; a.h_b = cfg->h_b;
  dispatch(cfg, f.p.vec == 2, f);
  return launched("scan forward");
}

dendsn_status dendsn_scan_backward(const dendsn_scan_cfg* cfg, const void* x, const void* g,
                                   const int32_t* lengths, const float* ckpt, const void* grad_h,
                                   const float* grad_h_last, void* grad_x, void* grad_g, float* grad_h0,
                                   void* workspace, size_t workspace_bytes, hipStream_t stream) {
  clear_error();
  dendsn_status st = check_cfg(cfg);
  if (st != DENDSN_OK) return st;
  const bool none = empty(cfg);
  const size_t esz = cfg->io == DENDSN_IO_BF16 ? 2 : 4;
  if (!none && (!x || !g || !grad_h || !grad_x || !grad_g))
    return fail(DENDSN_E_INVALID, "x, g, grad_h, grad_x or grad_g is NULL");
  if (!none && !ckpt) return fail(DENDSN_E_INVALID, "ckpt is NULL");
  if (!aligned(x, esz) || !aligned(g, esz) || !aligned(grad_h, esz) || !aligned(grad_x, esz) || !aligned(grad_g, esz))
    return fail(DENDSN_E_INVALID, "x, g, grad_h, grad_x or grad_g misaligned");
  if (!aligned(grad_h_last, 4) || !aligned(lengths, 4) || !aligned(grad_h0, 4))
    return fail(DENDSN_E_INVALID, "grad_h_last, lengths or grad_h0 misaligned");
  if (!aligned(ckpt, 16)) return fail(DENDSN_E_INVALID, "ckpt must be 16-byte aligned");
  if (!none && (!rows_apart(cfg, cfg->grad_x_t, cfg->grad_x_b) || !rows_apart(cfg, cfg->grad_g_t, cfg->grad_g_b)))
    return fail(DENDSN_E_INVALID, "rows of grad_x or of grad_g overlap");
  if (none) {
    const int64_t lanes = cfg->batch * cfg->D;
    if (grad_h0 && lanes) {
      scan_copy_kernel<<<dim3(unsigned(ceil_div(lanes, 256) < 4096 ? ceil_div(lanes, 256) : 4096)), dim3(256), 0, stream>>>(grad_h_last, grad_h0, lanes);
      return launched("scan backward");
    }
    return DENDSN_OK;
  }
  st = check_workspace(workspace, workspace_bytes, runs_bytes(cfg), "dendsn_scan_workspace_bytes");
  if (st != DENDSN_OK) return st;
  LaunchBwd f{{}, make_plan(cfg), stream};
  ScanArgs& a = f.a;
  a.x = x; a.g = g; a.gh = grad_h; a.lengths = lengths; a.ckpt_in = ckpt; a.gh_last = grad_h_last;
  a.gx = grad_x; a.gg = grad_g; a.gh0 = grad_h0;
  a.runs = workspace;
  a.D = cfg->D; a.T = int32_t(cfg->T); a.batch = int32_t(cfg->batch); a.ntiles = f.p.ntiles; a.per = f.p.per;
  a.x_t = cfg->x_t; a.x_b = cfg->x_b; a.g_t = cfg->g_t; a.g_b = cfg->g_b;
  a.gh_t = cfg->grad_h_t; a.gh_b = cfg->grad_h_b; a.gx_t = cfg->grad_x_t; a.gx_b = cfg->grad_x_b;
  a.gg_t = cfg->grad_g_t; a.gg_b = cfg->grad_g_b;
  dispatch(cfg, f.p.vec == 2, f);
  return launched("scan backward");
}

dendsn_status dendsn_scan_step(const dendsn_scan_cfg* cfg, const void* x, const void* g, int64_t n_slots,
                               const int32_t* slots, float* state, void* h, hipStream_t stream) {
  clear_error();
  dendsn_status st = check_cfg(cfg);
  if (st != DENDSN_OK) return st;
  if (cfg->T != 1) return fail(DENDSN_E_INVALID, "T must be 1");
  const bool none = empty(cfg);
  const size_t esz = cfg->io == DENDSN_IO_BF16 ? 2 : 4;
  if (n_slots < 0 || !small_product(n_slots, cfg->D)) return fail(DENDSN_E_INVALID, "n_slots negative or too large");
  if (!slots && n_slots < cfg->batch) return fail(DENDSN_E_INVALID, "without slots, n_slots must be >= batch");
  if (!none && (!x || !g || !h)) return fail(DENDSN_E_INVALID, "x, g or h is NULL");
  if (!none && n_slots > 0 && !state) return fail(DENDSN_E_INVALID, "state is NULL");
  if (!aligned(x, esz) || !aligned(g, esz) || !aligned(h, esz)) return fail(DENDSN_E_INVALID, "x, g or h misaligned");
  if (!aligned(slots, 4) || !aligned(state, 4)) return fail(DENDSN_E_INVALID, "slots or state misaligned");
  if (!none && !rows_apart(cfg, cfg->h_t, cfg->h_b)) return fail(DENDSN_E_INVALID, "rows of h overlap");
  if (none) return DENDSN_OK;
  // (no lane shares a channel here: its state is read and written)
  const bool wide = cfg->D % 2 == 0;
  LaunchStep f{{x, g, slots, state, h, cfg->D, cfg->x_b, cfg->g_b, cfg->h_b, n_slots}, cfg->batch, stream};
  dispatch(cfg, wide, f);
  return launched("scan step");
}

}  // extern "C"
