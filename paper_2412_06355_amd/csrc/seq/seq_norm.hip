// Root-mean-square norm of rows, or of their sum with a residual stream: forward (rows in io, or
// in 8 bits with a scale each) and backward.
//
//   s = x + residual,  rstd = (mean s^2 + eps)^-1/2,  y = s rstd w
//   dx = rstd (w dy - hat mean(w dy hat)) + dsum,  hat = s rstd;   dw = sum over rows of dy hat
//
// Bound by memory: every row is read once and kept in registers between the sum and the output,
// up to four packs of 16 bytes a lane; TPR lanes have a row, as many as its length needs (of 16, a
// wave's others have other rows).  What a row of more than 4 x 1024 packs has left is read again.
// The backward's blocks walk rows and keep their part of dw in registers; parts are joined in
// the blocks' order, so results do not depend on timing.
//
// 16384 rows of 4096 in bf16 with the stream: forward 126 us (4.3 TB/s), backward 119 us (4.5 TB/s)
// and 7 for the parts' sum; registers for as many packs as the row has instead of four: backward
// 187 -> 119.  4096 rows of 16384, of 1024 lanes each: 139 (3.9) and 119 (4.5).  8192 rows of 2048 to
// e4m3: 35 us (3.3 TB/s), where a device copy of as many bytes takes 24.  Why is not settled: rows of fp32
// go at a copy's rate in the same kernel (16384 of 2048: 83 us, 5.2 TB/s), so it is not memory; the same
// rows to bf16, without a second reduction and divisions, take 37 (3.7 TB/s), so it is not those alone;
// 16384 of 4096 to e4m3 take 121 (3.9 TB/s), so the launch's length is a part.
#include "dendsn_block.h"
#include "seq_common.h"

namespace dendsn_seq {
namespace {

constexpr int kMost = 4;  // packs of a lane that may be kept in registers
constexpr float kTop = 448.0f;  // the largest e4m3 value

template <typename IO> constexpr int kV = 16 / int(sizeof(IO));

struct NormArgs {
  const void *x, *residual, *w, *gy, *gsum;
  const float* rstd_in;
  void *y, *sum, *gx;
  float *rstd, *scale, *part;
  int64_t ld_x, ld_residual, ld_y, ld_sum, ld_gy, ld_gsum, ld_gx;
  int32_t N, D;
  float eps;
};

// Values [base, base + V) of a row of D, 0 past its end.
template <typename IO, int V>
__device__ __forceinline__ void load_row(const IO* row, int base, int D, float (&out)[V]) {
  if (base + V <= D) {
    const Pack<IO, V> p = *reinterpret_cast<const Pack<IO, V>*>(row + base);
#pragma unroll
    for (int j = 0; j < V; ++j) out[j] = widen(p.v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) out[j] = base + j < D ? widen(row[base + j]) : 0.0f;
  }
}
template <typename IO, int V>
__device__ __forceinline__ void store_row(IO* row, int base, int D, const float (&v)[V]) {
  if (base + V <= D) {
    Pack<IO, V> p;
#pragma unroll
    for (int j = 0; j < V; ++j) p.v[j] = narrow<IO>(v[j]);
    *reinterpret_cast<Pack<IO, V>*>(row + base) = p;
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (base + j < D) row[base + j] = narrow<IO>(v[j]);
  }
}

// Over the TPR lanes of a row; every lane has the result.
template <int TPR, bool MAX>
__device__ __forceinline__ float over_row(float v, float* red) {
#pragma unroll
  for (int m = (TPR < 64 ? TPR : 64) / 2; m > 0; m /= 2) {
    const float o = __shfl_xor(v, m);
    v = MAX ? fmaxf(v, o) : v + o;
  }
  if (TPR > 64) {
    __syncthreads();  // the last result is read
    if ((threadIdx.x & 63) == 0) red[threadIdx.x / 64] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < TPR / 64; ++i) v = MAX ? fmaxf(v, red[i]) : v + red[i];
  }
  return v;
}

__device__ __forceinline__ uint32_t e4m3_pair(float a, float b, float scale) {
  a /= scale;
  b /= scale;
  // (comparisons, so that NaN stays)
  a = a > kTop ? kTop : a < -kTop ? -kTop : a;
  b = b > kTop ? kTop : b < -kTop ? -kTop : b;
  return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false)) & 0xffffu;
}

template <int V>
__device__ __forceinline__ void store_e4m3(uint8_t* row, int base, int D, const float (&v)[V], float scale) {
  Pack<uint8_t, V> p;
#pragma unroll
  for (int j = 0; j < V; j += 2) {
    const uint32_t two = e4m3_pair(v[j], v[j + 1], scale);
    p.v[j] = uint8_t(two);
    p.v[j + 1] = uint8_t(two >> 8);
  }
  if (base + V <= D) {
    *reinterpret_cast<Pack<uint8_t, V>*>(row + base) = p;
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (base + j < D) row[base + j] = p.v[j];
  }
}

template <typename IO, int TPR, int kE, bool E4M3>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_fwd_kernel(NormArgs a) {
  constexpr int V = kV<IO>, kBlock = TPR > 256 ? TPR : 256;
  __shared__ float red[TPR > 64 ? TPR / 64 : 1];
  const int t = threadIdx.x % TPR;
  const int64_t n = int64_t(blockIdx.x) * (kBlock / TPR) + threadIdx.x / TPR;
  if (n >= a.N) return;
  const IO* x = static_cast<const IO*>(a.x) + n * a.ld_x;
  const IO* res = a.residual ? static_cast<const IO*>(a.residual) + n * a.ld_residual : nullptr;
  const IO* w = static_cast<const IO*>(a.w);
  IO* sum = a.sum ? static_cast<IO*>(a.sum) + n * a.ld_sum : nullptr;
  auto row_of = [&](int base, float (&s)[V]) {
    load_row<IO, V>(x, base, a.D, s);
    if (res) {
      float r[V];
      load_row<IO, V>(res, base, a.D, r);
#pragma unroll
      for (int j = 0; j < V; ++j) s[j] += r[j];
    }
  };
  float s[kE][V], ss = 0.0f;
#pragma unroll
  for (int e = 0; e < kE; ++e) {
    const int base = (e * TPR + t) * V;
#pragma unroll
    for (int j = 0; j < V; ++j) s[e][j] = 0.0f;
    if (base < a.D) row_of(base, s[e]);
  }
#pragma unroll
  for (int e = 0; e < kE; ++e)
#pragma unroll
    for (int j = 0; j < V; ++j) ss = fmaf(s[e][j], s[e][j], ss);
  if (TPR == 1024) {
    for (int base = (kE * TPR + t) * V; base < a.D; base += TPR * V) {
      float r[V];
      row_of(base, r);
#pragma unroll
      for (int j = 0; j < V; ++j) ss = fmaf(r[j], r[j], ss);
    }
  }
  const float rstd = 1.0f / sqrtf(over_row<TPR, false>(ss, red) / float(a.D) + a.eps);
  if (a.rstd && t == 0) a.rstd[n] = rstd;
  auto normed = [&](int base, float (&r)[V]) {  // s, then y
    if (sum) store_row<IO, V>(sum, base, a.D, r);
    float g[V];
    if (w) load_row<IO, V>(w, base, a.D, g);
#pragma unroll
    for (int j = 0; j < V; ++j) r[j] = r[j] * rstd * (w ? g[j] : 1.0f);
  };
  if (!E4M3) {
    IO* y = static_cast<IO*>(a.y) + n * a.ld_y;
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const int base = (e * TPR + t) * V;
      if (base < a.D) {
        normed(base, s[e]);
        store_row<IO, V>(y, base, a.D, s[e]);
      }
    }
    if (TPR == 1024) {
      for (int base = (kE * TPR + t) * V; base < a.D; base += TPR * V) {
        float r[V];
        row_of(base, r);
        normed(base, r);
        store_row<IO, V>(y, base, a.D, r);
      }
    }
  } else {
    uint8_t* y = static_cast<uint8_t*>(a.y) + n * a.ld_y;
    float top = 0.0f;
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const int base = (e * TPR + t) * V;
      if (base < a.D) {
        normed(base, s[e]);
#pragma unroll
        for (int j = 0; j < V; ++j) top = fmaxf(top, fabsf(s[e][j]));
      }
    }
    if (TPR == 1024) {
      for (int base = (kE * TPR + t) * V; base < a.D; base += TPR * V) {
        float r[V];
        row_of(base, r);
        normed(base, r);
#pragma unroll
        for (int j = 0; j < V; ++j) top = fmaxf(top, fabsf(r[j]));
      }
    }
    float scale = over_row<TPR, true>(top, red) / kTop;
    scale = scale > 0.0f ? scale : 1.0f;
    if (t == 0) a.scale[n] = scale;
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const int base = (e * TPR + t) * V;
      if (base < a.D) store_e4m3<V>(y, base, a.D, s[e], scale);
    }
    if (TPR == 1024) {
      for (int base = (kE * TPR + t) * V; base < a.D; base += TPR * V) {
        float r[V];
        row_of(base, r);
        normed(base, r);
        store_e4m3<V>(y, base, a.D, r, scale);
      }
    }
  }
}

// hat is of the row that is given: of the sum that the forward stored, which has io's bits, or (RES) of
// x + residual, formed again as the forward had it, for one more row read.  What y and rstd are the norm
// of is the second; in bf16 the first moves every hat by up to 2^-8 of itself, and grad_weight by about as
// much as its own rounding does (4096 rows of 512: off by 2.5e-3 in norm, not 1.6e-3).  The choice is the
// caller's: 16384 rows of 4096 in bf16 take 120 us the first way, 146 the second.
template <typename IO, int TPR, int kE, bool W, bool RES>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_bwd_kernel(NormArgs a) {
  constexpr int V = kV<IO>, kBlock = TPR > 256 ? TPR : 256, kRows = kBlock / TPR;
  __shared__ float red[TPR > 64 ? TPR / 64 : 1];
  __shared__ float join[W && kRows > 1 ? kE * V * TPR : 1];
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const IO* w = static_cast<const IO*>(a.w);
  float* part = W ? a.part + int64_t(blockIdx.x) * a.D : nullptr;
  float dw[kE][V];
#pragma unroll
  for (int e = 0; e < kE; ++e)
#pragma unroll
    for (int j = 0; j < V; ++j) dw[e][j] = 0.0f;
  bool first = true;
  for (int64_t n = int64_t(blockIdx.x) * kRows + sub; n < a.N; n += int64_t(gridDim.x) * kRows) {
    const IO* x = static_cast<const IO*>(a.x) + n * a.ld_x;
    const IO* res = RES ? static_cast<const IO*>(a.residual) + n * a.ld_residual : nullptr;
    const IO* gy = static_cast<const IO*>(a.gy) + n * a.ld_gy;
    const IO* gs = a.gsum ? static_cast<const IO*>(a.gsum) + n * a.ld_gsum : nullptr;
    IO* gx = static_cast<IO*>(a.gx) + n * a.ld_gx;
    const float rstd = a.rstd_in[n];
    // hat, w dy (and dy hat into dw) of one pack
    auto pack_of = [&](int base, float (&hat)[V], float (&g)[V], float (&d)[V]) {
      load_row<IO, V>(x, base, a.D, hat);
      load_row<IO, V>(gy, base, a.D, g);
      if (RES) {
        float r[V];
        load_row<IO, V>(res, base, a.D, r);
#pragma unroll
        for (int j = 0; j < V; ++j) hat[j] += r[j];
      }
      float ww[V];
      if (W) load_row<IO, V>(w, base, a.D, ww);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        hat[j] *= rstd;
        if (W) {
          d[j] = fmaf(g[j], hat[j], d[j]);
          g[j] *= ww[j];
        }
      }
    };
    float hat[kE][V], g[kE][V], along = 0.0f;
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const int base = (e * TPR + t) * V;
#pragma unroll
      for (int j = 0; j < V; ++j) hat[e][j] = g[e][j] = 0.0f;
      if (base < a.D) pack_of(base, hat[e], g[e], dw[e]);
    }
#pragma unroll
    for (int e = 0; e < kE; ++e)
#pragma unroll
      for (int j = 0; j < V; ++j) along = fmaf(hat[e][j], g[e][j], along);
    if (TPR == 1024) {
      for (int base = (kE * TPR + t) * V; base < a.D; base += TPR * V) {
        float h1[V], g1[V], d1[V];
#pragma unroll
        for (int j = 0; j < V; ++j) d1[j] = !W || first || base + j >= a.D ? 0.0f : part[base + j];
        pack_of(base, h1, g1, d1);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          along = fmaf(h1[j], g1[j], along);
          if (W && base + j < a.D) part[base + j] = d1[j];
        }
      }
    }
    along = over_row<TPR, false>(along, red) / float(a.D);
    auto put = [&](int base, const float (&hat)[V], const float (&g)[V]) {
      float r[V], o[V];
      if (gs) load_row<IO, V>(gs, base, a.D, r);
#pragma unroll
      for (int j = 0; j < V; ++j) o[j] = fmaf(rstd, g[j] - hat[j] * along, gs ? r[j] : 0.0f);
      store_row<IO, V>(gx, base, a.D, o);
    };
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const int base = (e * TPR + t) * V;
      if (base < a.D) put(base, hat[e], g[e]);
    }
    if (TPR == 1024) {
      for (int base = (kE * TPR + t) * V; base < a.D; base += TPR * V) {
        float h1[V], g1[V], d1[V] = {};
        pack_of(base, h1, g1, d1);
        put(base, h1, g1);
      }
    }
    first = false;
  }
  if (!W) return;
  if (kRows > 1) {
    // the block's rows in their order
    for (int s = 0; s < kRows; ++s) {
      if (sub == s) {
#pragma unroll
        for (int e = 0; e < kE; ++e)
#pragma unroll
          for (int j = 0; j < V; ++j) {
            float& to = join[(e * V + j) * TPR + t];
            to = s == 0 ? dw[e][j] : to + dw[e][j];
          }
      }
      __syncthreads();
    }
    for (int i = threadIdx.x; i < a.D; i += kBlock) {
      const int p = i / V;
      part[i] = join[(p / TPR * V + i % V) * TPR + p % TPR];
    }
  } else {
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const int base = (e * TPR + t) * V;
      if (base < a.D) store_row<float, V>(part, base, a.D, dw[e]);
    }
  }
}

// dw from the blocks' parts: 32 columns a block, eight sums a column.
template <typename IO>
__global__ __launch_bounds__(256) void norm_join_kernel(const float* part, IO* gw, int64_t D, int parts) {
  __shared__ float red[8][33];
  const int c = threadIdx.x % 32, g = threadIdx.x / 32;
  const int64_t d = int64_t(blockIdx.x) * 32 + c;
  float s = 0.0f;
  if (d < D) {
#pragma unroll 8
    for (int i = g; i < parts; i += 8) s += part[i * D + d];
  }
  red[g][c] = s;
  __syncthreads();
  if (g == 0 && d < D) {
#pragma unroll
    for (int i = 1; i < 8; ++i) s += red[i][c];
    gw[d] = narrow<IO>(s);
  }
}

dendsn_status check_cfg(const dendsn_norm_cfg* c) {
  if (!c) return fail(DENDSN_E_INVALID, "cfg is NULL");
  if (c->N < 0 || c->N > INT32_MAX) return fail(DENDSN_E_INVALID, "N must be in [0, 2^31)");
  if (c->D < 1 || c->D > (int64_t(1) << 22)) return fail(DENDSN_E_INVALID, "D must be in [1, 2^22]");
  if (c->io != DENDSN_IO_F32 && c->io != DENDSN_IO_BF16) return fail(DENDSN_E_INVALID, "bad io");
  if (!(c->eps >= 0.0f) || !isfinite(c->eps)) return fail(DENDSN_E_INVALID, "eps must be finite and >= 0");
  const int64_t in[4] = {c->ld_x, c->ld_residual, c->ld_grad_y, c->ld_grad_sum}, out[3] = {c->ld_y, c->ld_sum, c->ld_grad_x};
  for (int64_t s : in)
    if (s < 0 || !small_product(c->N, s)) return fail(DENDSN_E_INVALID, "a stride is negative or too large");
  for (int64_t s : out)
    if (s < c->D || !small_product(c->N, s)) return fail(DENDSN_E_INVALID, "the stride of an output is below D or too large");
  return DENDSN_OK;
}

struct Shape {
  int lanes, packs;  // of a row, of a lane
};
Shape shape_of(const dendsn_norm_cfg* c) {
  const int64_t n = ceil_div(c->D, c->io == DENDSN_IO_BF16 ? 8 : 4);
  const int lanes = n <= 16 * kMost ? 16 : n <= 64 * kMost ? 64 : n <= 256 * kMost ? 256 : 1024;
  return {lanes, n <= lanes ? 1 : n <= 2 * lanes ? 2 : kMost};
}

// Blocks of the backward: four of 256 threads a CU, or one of 1024.
int64_t parts_of(const dendsn_norm_cfg* c) {
  const int lanes = shape_of(c).lanes, rows = lanes < 256 ? 256 / lanes : 1;
  const int64_t blocks = ceil_div(c->N, rows), most = lanes == 1024 ? 256 : 1024;
  return blocks < most ? blocks : most;
}

template <typename F>
void dispatch(Shape s, F&& f) {
  auto packs = [&](auto lanes) {
    if (s.packs == 1) f(lanes, std::integral_constant<int, 1>{});
    else if (s.packs == 2) f(lanes, std::integral_constant<int, 2>{});
    else f(lanes, std::integral_constant<int, kMost>{});
  };
  if (s.lanes == 16) packs(std::integral_constant<int, 16>{});
  else if (s.lanes == 64) packs(std::integral_constant<int, 64>{});
  else if (s.lanes == 256) packs(std::integral_constant<int, 256>{});
  else packs(std::integral_constant<int, 1024>{});
}

// A launch has at most 2^31 threads: with more rows there are several.
template <typename IO, bool E4M3>
void launch_forward(const NormArgs& whole, Shape s, hipStream_t stream) {
  const int threads = s.lanes > 256 ? s.lanes : 256, rows = threads / s.lanes;
  const int64_t most = (int64_t(1) << 31) / threads * rows;
  auto from = [](auto* p, int64_t at) { return p ? p + at : p; };
  for (int64_t n0 = 0; n0 < whole.N; n0 += most) {
    NormArgs a = whole;
    a.N = int32_t(whole.N - n0 < most ? whole.N - n0 : most);
    a.x = static_cast<const IO*>(a.x) + n0 * a.ld_x;
    a.residual = from(static_cast<const IO*>(a.residual), n0 * a.ld_residual);
    a.y = static_cast<char*>(a.y) + n0 * a.ld_y * (E4M3 ? 1 : int64_t(sizeof(IO)));
    a.sum = from(static_cast<IO*>(a.sum), n0 * a.ld_sum);
    a.rstd = from(a.rstd, n0);
    a.scale = from(a.scale, n0);
    const dim3 grid(unsigned(ceil_div(a.N, rows))), block(threads);
    dispatch(s, [&](auto lanes, auto packs) {
      norm_fwd_kernel<IO, decltype(lanes)::value, decltype(packs)::value, E4M3><<<grid, block, 0, stream>>>(a);
    });
  }
}

template <typename IO, bool W>
void launch_backward(const NormArgs& a, Shape s, int64_t blocks, hipStream_t stream) {
  const dim3 grid{unsigned(blocks)}, block(s.lanes > 256 ? s.lanes : 256);
  dispatch(s, [&](auto lanes, auto packs) {
    if (a.residual) norm_bwd_kernel<IO, decltype(lanes)::value, decltype(packs)::value, W, true><<<grid, block, 0, stream>>>(a);
    else norm_bwd_kernel<IO, decltype(lanes)::value, decltype(packs)::value, W, false><<<grid, block, 0, stream>>>(a);
  });
}

dendsn_status forward(const dendsn_norm_cfg* cfg, const void* x, const void* residual, const void* weight, void* y,
                      float* scale, void* sum, float* rstd, bool e4m3, hipStream_t stream) {
  clear_error();
  const dendsn_status st = check_cfg(cfg);
  if (st != DENDSN_OK) return st;
  const size_t esz = cfg->io == DENDSN_IO_BF16 ? 2 : 4;
  // (x's rows may be one, or overlap)
  const int64_t x_bytes = ((cfg->N - 1) * cfg->ld_x + cfg->D) * int64_t(esz), y_bytes = cfg->N * cfg->D * (e4m3 ? 1 : int64_t(esz));
  if (cfg->N > 0 && x_bytes + y_bytes > (int64_t(1) << 39))
    return fail(DENDSN_E_UNSUPPORTED, "x and y of more than 2^39 bytes");
  if (cfg->N > 0 && (!x || !y || (e4m3 && !scale))) return fail(DENDSN_E_INVALID, e4m3 ? "x, y or scale is NULL" : "x or y is NULL");
  if (!aligned(x, esz) || !aligned(residual, esz) || !aligned(weight, esz) || !aligned(sum, esz) || (!e4m3 && !aligned(y, esz)))
    return fail(DENDSN_E_INVALID, "x, residual, weight, y or sum misaligned");
  if (!aligned(scale, 4) || !aligned(rstd, 4)) return fail(DENDSN_E_INVALID, "scale or rstd misaligned");
  if (cfg->N == 0) return DENDSN_OK;
  NormArgs a{};
  a.x = x; a.residual = residual; a.w = weight; a.y = y; a.sum = sum; a.rstd = rstd; a.scale = scale;
  a.ld_x = cfg->ld_x; a.ld_residual = cfg->ld_residual; a.ld_y = cfg->ld_y; a.ld_sum = cfg->ld_sum;
  a.N = int32_t(cfg->N); a.D = int32_t(cfg->D); a.eps = cfg->eps;
  const Shape shape = shape_of(cfg);
  if (cfg->io == DENDSN_IO_BF16) e4m3 ? launch_forward<bf16_t, true>(a, shape, stream) : launch_forward<bf16_t, false>(a, shape, stream);
  else e4m3 ? launch_forward<float, true>(a, shape, stream) : launch_forward<float, false>(a, shape, stream);
  return launched("norm forward");
}

}  // namespace
}  // namespace dendsn_seq

using namespace dendsn_seq;

extern "C" {

dendsn_status dendsn_norm_forward(const dendsn_norm_cfg* cfg, const void* x, const void* residual, const void* weight,
                                  void* y, void* sum, float* rstd, hipStream_t stream) {
  return forward(cfg, x, residual, weight, y, nullptr, sum, rstd, false, stream);
}

dendsn_status dendsn_norm_forward_e4m3(const dendsn_norm_cfg* cfg, const void* x, const void* residual,
                                       const void* weight, void* y, float* scale, void* sum, float* rstd,
                                       hipStream_t stream) {
  return forward(cfg, x, residual, weight, y, scale, sum, rstd, true, stream);
}

dendsn_status dendsn_norm_workspace_bytes(const dendsn_norm_cfg* cfg, size_t* bytes) {
  clear_error();
  const dendsn_status st = check_cfg(cfg);
  if (st != DENDSN_OK) return st;
  if (!bytes) return fail(DENDSN_E_INVALID, "bytes is NULL");
  *bytes = size_t(parts_of(cfg)) * size_t(cfg->D) * sizeof(float);
  return DENDSN_OK;
}

dendsn_status dendsn_norm_backward(const dendsn_norm_cfg* cfg, const void* x, const void* weight, const float* rstd,
                                   const void* grad_y, const void* grad_sum, void* grad_x, void* grad_weight,
                                   void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return dendsn_norm_backward_residual(cfg, x, nullptr, weight, rstd, grad_y, grad_sum, grad_x, grad_weight, workspace,
                                       workspace_bytes, stream);
}

dendsn_status dendsn_norm_backward_residual(const dendsn_norm_cfg* cfg, const void* x, const void* residual,
                                            const void* weight, const float* rstd, const void* grad_y,
                                            const void* grad_sum, void* grad_x, void* grad_weight, void* workspace,
                                            size_t workspace_bytes, hipStream_t stream) {
  clear_error();
  dendsn_status st = check_cfg(cfg);
  if (st != DENDSN_OK) return st;
  const size_t esz = cfg->io == DENDSN_IO_BF16 ? 2 : 4;
  if (cfg->N > 0 && (!x || !rstd || !grad_y || !grad_x)) return fail(DENDSN_E_INVALID, "x, rstd, grad_y or grad_x is NULL");
  if (weight && !grad_weight) return fail(DENDSN_E_INVALID, "grad_weight is NULL");
  if (!aligned(x, esz) || !aligned(residual, esz) || !aligned(weight, esz) || !aligned(grad_y, esz) ||
      !aligned(grad_sum, esz) || !aligned(grad_x, esz) || !aligned(grad_weight, esz) || !aligned(rstd, 4))
    return fail(DENDSN_E_INVALID, "x, residual, weight, rstd, grad_y, grad_sum, grad_x or grad_weight misaligned");
  if (weight) {
    st = check_workspace(workspace, workspace_bytes, size_t(parts_of(cfg)) * size_t(cfg->D) * sizeof(float),
                         "dendsn_norm_workspace_bytes");
    if (st != DENDSN_OK) return st;
  }
  if (cfg->N == 0 && !weight) return DENDSN_OK;
  NormArgs a{};
  a.x = x; a.residual = residual; a.w = weight; a.rstd_in = rstd; a.gy = grad_y; a.gsum = grad_sum; a.gx = grad_x;
  a.part = static_cast<float*>(workspace);
  a.ld_x = cfg->ld_x; a.ld_residual = cfg->ld_residual; a.ld_gy = cfg->ld_grad_y; a.ld_gsum = cfg->ld_grad_sum; a.ld_gx = cfg->ld_grad_x;
  a.N = int32_t(cfg->N); a.D = int32_t(cfg->D);
  const Shape shape = shape_of(cfg);
  const int64_t parts = parts_of(cfg);
  const bool bf16 = cfg->io == DENDSN_IO_BF16;
  if (parts) {
    if (weight) bf16 ? launch_backward<bf16_t, true>(a, shape, parts, stream) : launch_backward<float, true>(a, shape, parts, stream);
    else bf16 ? launch_backward<bf16_t, false>(a, shape, parts, stream) : launch_backward<float, false>(a, shape, parts, stream);
  }
  if (weight) {  // of no rows: +0
    const dim3 grid(unsigned(ceil_div(cfg->D, 32)));
    if (bf16) norm_join_kernel<bf16_t><<<grid, dim3(256), 0, stream>>>(a.part, static_cast<bf16_t*>(grad_weight), cfg->D, int(parts));
    else norm_join_kernel<float><<<grid, dim3(256), 0, stream>>>(a.part, static_cast<float*>(grad_weight), cfg->D, int(parts));
  }
  return launched("norm backward");
}

}  // extern "C"
