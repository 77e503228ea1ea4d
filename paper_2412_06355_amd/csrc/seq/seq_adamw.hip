// AdamW over many tensors, states in fp32 or in 8 bits.
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
//   p = p - lr (wd p + (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps))
//
// Bound by memory: 28 bytes a value with states in fp32, bf16 gradients and copies, 16 with
// states in 8 bits.  The tensors' pointers are kernel arguments, 40 tensors a launch: nothing
// is copied to the device, and a captured step holds them.  A block has 8192 values of one
// tensor, a wave 256 at a time, which is also the block of values that share a scale in 8 bits:
// its largest magnitude is found within the wave.  Two rounds' loads are issued together, without
// conditions where a round is whole (1683 -> 1589 us below).
//
// 292M values in 122 tensors, bf16 gradients and copies: 1589 us with fp32 states (5.15 TB/s, a copy's
// rate), 961 to 975 us in 8 bits (4.9 TB/s; its 70 vector instructions a value take nearly as long:
// with a second root and a division 1056).
//
// In 8 bits a value is rounded down or up at random, so that its mean is kept.  v changes by a
// thousandth a step, e4m3 values lie an eighth to a sixteenth apart: rounded to the nearest, v
// would never move.  What is held is the root of v, whose range is half v's in binades; one
// that is not 0 stays at least at the smallest code, so that m / root stays bounded.  Whether a
// value goes down or up hangs on its last bit, so what decides it is computed as it is written:
// products and sums rounded one by one, a value over its scale to the nearest.
#include <cfloat>

#include "dendsn_block.h"
#include "seq_common.h"

namespace dendsn_seq {
namespace {

constexpr int kTensors = 40;      // of a launch
constexpr int kGroup = 256;       // values of a wave's round, and of a scale
constexpr int kGroups = 32;       // of a block
constexpr int kWaves = 4;
constexpr float kTop = 448.0f;    // the largest e4m3 value
constexpr int64_t kMaxBlocks = int64_t(1) << 23;  // of a launch: fewer than 2^32 threads

struct Tensor {
  float* p;
  const void* g;
  void *m, *v;
  float *ms, *vs;
  bf16_t* copy;
  int64_t n;
  uint32_t first;    // block
  uint32_t bf16;     // gradients
};

struct Batch {
  Tensor t[kTensors];
  int32_t count, base;  // base: the first one's place in the list
  float b1, c1, b2, c2, lr, eps, wd, fix1, fix2;  // c = 1 - b, fix = 1 - b^step
  double log_b1, log_b2;
  uint32_t step, seed_lo, seed_hi;
  const int32_t* step_dev;
  const float* grad_scale;
};

// A bijection of 32 bits: rounds of folding the high half down and an odd product.  The first and the last
// multiplier are those of a published 32-bit hash (C. Wellons, "Prospecting for Hash Functions", 2018),
// found there by search; the one between is 2^32 over the golden ratio.
__device__ __forceinline__ uint32_t mix(uint32_t h) {
  h = (h ^ (h >> 16)) * 0x7FEB352Du;
  h = (h ^ (h >> 16)) * 0x9E3779B1u;
  h = (h ^ (h >> 16)) * 0x846CA68Bu;
  return h ^ (h >> 16);
}

// |y| <= 448 rounded to one of its two e4m3 neighbours by u in [0, 1).
__device__ __forceinline__ float round_at(float size, float u) {
  const uint32_t binade = __float_as_uint(fmaxf(size, 0.015625f)) & 0x7f800000u;
  const float step = __uint_as_float(binade) * 0.125f, inv = __uint_as_float(0x7f000000u - binade) * 8.0f;
  return floorf(size * inv + u) * step;
}

struct Scale {
  float scale, inv;
};
// Of values whose largest magnitude is top: that times 1 / 448 as fp32 has it.  (So does torch divide by a
// number on the GPU; the quotient, which is another number for half of all blocks, would decide other
// roundings than those formulas in torch do.)  Scales stay normal numbers, so that they can be
// inverted: values below 2^-117 are of no account.
__device__ __forceinline__ Scale scale_of(float top) {
  const float s = top > 0.0f ? fmaxf(top * (1.0f / kTop), 0x1p-126f) : 1.0f;
  return {s, 1.0f / s};
}

// x / s.scale, rounded once: the reciprocal's product, and what is left of x times it.
__device__ __forceinline__ float in_units(float x, Scale s) {
  const float q = x * s.inv;
  return fmaf(fmaf(-q, s.scale, x), s.inv, q);
}

__device__ __forceinline__ float over_wave(float v) {
#pragma unroll
  for (int m = 32; m > 0; m /= 2) v = fmaxf(v, __shfl_xor(v, m));
  return v;
}

// V values of which `left` are there; FULL: all.
template <bool FULL, typename T, int V>
__device__ __forceinline__ Pack<T, V> load_some(const T* p, int left) {
  Pack<T, V> r{};
  if (FULL || left >= V) {
    r = *reinterpret_cast<const Pack<T, V>*>(p);
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (j < left) r.v[j] = p[j];
  }
  return r;
}
template <bool FULL, typename T, int V>
__device__ __forceinline__ void store_some(T* p, int left, const Pack<T, V>& r) {
  if (FULL || left >= V) {
    *reinterpret_cast<Pack<T, V>*>(p) = r;
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (j < left) p[j] = r.v[j];
  }
}

__device__ __forceinline__ void codes_of(const Pack<uint8_t, 4>& c, float (&out)[4]) {
  const uint32_t w = c.v[0] | c.v[1] << 8 | c.v[2] << 16 | uint32_t(c.v[3]) << 24;
  out[0] = __builtin_amdgcn_cvt_f32_fp8(w, 0);
  out[1] = __builtin_amdgcn_cvt_f32_fp8(w, 1);
  out[2] = __builtin_amdgcn_cvt_f32_fp8(w, 2);
  out[3] = __builtin_amdgcn_cvt_f32_fp8(w, 3);
}
__device__ __forceinline__ Pack<uint8_t, 4> codes(const float (&v)[4]) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], w, true);
  return Pack<uint8_t, 4>{{uint8_t(w), uint8_t(w >> 8), uint8_t(w >> 16), uint8_t(uint32_t(w) >> 24)}};
}

template <bool E4M3>
__global__ __launch_bounds__(kWaves * 64) void adamw_kernel(const Batch a) {
  int at = 0;
  for (int half = 32; half > 0; half /= 2)  // the last tensor whose first block is not past this one
    if (at + half < a.count && a.t[at + half].first <= blockIdx.x) at += half;
  const Tensor& t = a.t[at];
  const int lane = threadIdx.x & 63;
  const int64_t n = t.n;
  float fix1 = a.fix1, fix2 = a.fix2;
  uint32_t step = a.step;
  if (a.step_dev) {
    step = uint32_t(*a.step_dev);
    fix1 = float(-expm1(double(step) * a.log_b1));
    fix2 = float(-expm1(double(step) * a.log_b2));
  }
  const float inv1 = 1.0f / fix1, inv_root = sqrtf(1.0f / fix2);
  const float gs = a.grad_scale ? *a.grad_scale : 1.0f;
  const uint32_t key = mix(a.seed_lo ^ mix(a.seed_hi ^ mix(step ^ mix(uint32_t(a.base + at) + 1u))));
  const int64_t from = int64_t(blockIdx.x - t.first) * (kGroup * kGroups);
  // a lane's four values of a round
  struct Values {
    Pack<float, 4> p, m, v, g;
    Pack<bf16_t, 4> gh;
    Pack<uint8_t, 4> cm, cv;
    float ms, vs;
  };
  auto left_of = [&](int64_t i) { return int(n - i < 4 ? n - i < 0 ? 0 : n - i : 4); };
  auto load = [&](auto full, int r) {
    constexpr bool F = decltype(full)::value;
    Values x;
    const int64_t g0 = from + r * kGroup, i = g0 + lane * 4;
    const int left = F ? 4 : left_of(i);
    x.p = load_some<F, float, 4>(t.p + i, left);
    if (t.bf16) x.gh = load_some<F, bf16_t, 4>(static_cast<const bf16_t*>(t.g) + i, left);
    else x.g = load_some<F, float, 4>(static_cast<const float*>(t.g) + i, left);
    if (E4M3) {
      x.cm = load_some<F, uint8_t, 4>(static_cast<const uint8_t*>(t.m) + i, left);
      x.cv = load_some<F, uint8_t, 4>(static_cast<const uint8_t*>(t.v) + i, left);
      x.ms = t.ms[g0 / kGroup];
      x.vs = t.vs[g0 / kGroup];
    } else {
      x.m = load_some<F, float, 4>(static_cast<const float*>(t.m) + i, left);
      x.v = load_some<F, float, 4>(static_cast<const float*>(t.v) + i, left);
    }
    return x;
  };
  auto compute = [&](auto full, int r, const Values& x) {
    constexpr bool F = decltype(full)::value;
    const int64_t g0 = from + r * kGroup, i = g0 + lane * 4;
    const int left = F ? 4 : left_of(i);
    const Pack<float, 4> p = x.p;
    float g[4], m[4], v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) g[j] = (t.bf16 ? widen(x.gh.v[j]) : x.g.v[j]) * gs;
    if (E4M3) {
      codes_of(x.cm, m);
      codes_of(x.cv, v);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        m[j] *= x.ms;
        v[j] *= x.vs;
        v[j] *= v[j];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        m[j] = x.m.v[j];
        v[j] = x.v.v[j];
      }
    }
    Pack<float, 4> np;
    float root[4];
    Pack<bf16_t, 4> copy;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m[j] = a.b1 * m[j] + a.c1 * g[j];
      v[j] = a.b2 * v[j] + a.c2 * g[j] * g[j];
      // (the update needs no last bit: the root of v is taken once, the quotient is a reciprocal's)
      root[j] = sqrtf(v[j]);
      const float to = (m[j] * inv1) * __builtin_amdgcn_rcpf(fmaf(root[j], inv_root, a.eps));
      np.v[j] = p.v[j] - a.lr * fmaf(a.wd, p.v[j], to);
      copy.v[j] = narrow<bf16_t>(np.v[j]);
    }
    store_some<F, float, 4>(t.p + i, left, np);
    if (t.copy) store_some<F, bf16_t, 4>(t.copy + i, left, copy);
    if (E4M3) {
      float tm = 0.0f, tv = 0.0f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] = root[j];
        tm = fmaxf(tm, fabsf(m[j]));
        tv = fmaxf(tv, v[j]);
      }
      const Scale sm = scale_of(over_wave(tm)), sv = scale_of(over_wave(tv));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t bits = mix(uint32_t(i + j) ^ (key + uint32_t(uint64_t(i + j) >> 32)));
        // (comparisons, so that NaN stays)
        float um = in_units(fabsf(m[j]), sm), uv = in_units(v[j], sv);
        um = um > kTop ? kTop : um;
        uv = uv > kTop ? kTop : uv;
        const float u1 = float(bits & 0xffffu) * 0x1p-16f, u2 = float(bits >> 16) * 0x1p-16f;
        const float cm = round_at(um, u1), cv = round_at(uv, u2);
        m[j] = copysignf(cm, m[j]);
        v[j] = uv > 0.0f && cv < 0x1p-9f ? 0x1p-9f : cv;
      }
      store_some<F, uint8_t, 4>(static_cast<uint8_t*>(t.m) + i, left, codes(m));
      store_some<F, uint8_t, 4>(static_cast<uint8_t*>(t.v) + i, left, codes(v));
      if (lane == 0) {
        t.ms[g0 / kGroup] = sm.scale;
        t.vs[g0 / kGroup] = sv.scale;
      }
    } else {
      store_some<F, float, 4>(static_cast<float*>(t.m) + i, left, Pack<float, 4>{{m[0], m[1], m[2], m[3]}});
      store_some<F, float, 4>(static_cast<float*>(t.v) + i, left, Pack<float, 4>{{v[0], v[1], v[2], v[3]}});
    }
  };
  int r = threadIdx.x / 64;
  for (; r + kWaves < kGroups && from + (r + kWaves + 1) * kGroup <= n; r += 2 * kWaves) {  // two rounds' loads at once
    const Values x = load(std::true_type{}, r), y = load(std::true_type{}, r + kWaves);
    compute(std::true_type{}, r, x);
    compute(std::true_type{}, r + kWaves, y);
  }
  for (; r < kGroups && from + r * kGroup < n; r += kWaves) compute(std::false_type{}, r, load(std::false_type{}, r));
}

dendsn_status check_tensor(const dendsn_adamw_cfg* c, const dendsn_adamw_tensor& t, int64_t i) {
  const long long at = i;
  if (t.n < 0 || t.n > (int64_t(1) << 34)) return fail(DENDSN_E_INVALID, "tensor %lld: n must be in [0, 2^34]", at);
  if (t.grad_io != DENDSN_IO_F32 && t.grad_io != DENDSN_IO_BF16) return fail(DENDSN_E_INVALID, "tensor %lld: bad grad_io", at);
  if (t.n == 0) return DENDSN_OK;
  const bool e4m3 = c->state == DENDSN_STATE_E4M3;
  if (!t.param || !t.grad || !t.m || !t.v) return fail(DENDSN_E_INVALID, "tensor %lld: param, grad, m or v is NULL", at);
  if (e4m3 && (!t.m_scale || !t.v_scale)) return fail(DENDSN_E_INVALID, "tensor %lld: m_scale or v_scale is NULL", at);
  if (!aligned(t.param, 4) || !aligned(t.grad, t.grad_io == DENDSN_IO_BF16 ? 2 : 4) || !aligned(t.copy, 2) ||
      !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4) || (!e4m3 && (!aligned(t.m, 4) || !aligned(t.v, 4))))
    return fail(DENDSN_E_INVALID, "tensor %lld: an array is misaligned", at);
  return DENDSN_OK;
}

}  // namespace
}  // namespace dendsn_seq

using namespace dendsn_seq;

extern "C" dendsn_status dendsn_adamw_step(const dendsn_adamw_cfg* cfg, const dendsn_adamw_tensor* tensors,
                                           int64_t count, int64_t step, const int32_t* step_dev,
                                           const float* grad_scale, uint64_t seed, hipStream_t stream) {
  clear_error();
  if (!cfg) return fail(DENDSN_E_INVALID, "cfg is NULL");
  if (!isfinite(cfg->lr) || !(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0) || !(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0))
    return fail(DENDSN_E_INVALID, "lr must be finite, the betas in [0, 1)");
  if (!(cfg->eps >= 0.0) || !isfinite(cfg->eps) || !(cfg->weight_decay >= 0.0) || !isfinite(cfg->weight_decay))
    return fail(DENDSN_E_INVALID, "eps and weight_decay must be finite and >= 0");
  if (cfg->state != DENDSN_STATE_F32 && cfg->state != DENDSN_STATE_E4M3) return fail(DENDSN_E_INVALID, "bad state");
  if (count < 0 || count > (int64_t(1) << 20)) return fail(DENDSN_E_INVALID, "count must be in [0, 2^20]");
  if (count > 0 && !tensors) return fail(DENDSN_E_INVALID, "tensors is NULL");
  if (step < 1 || step > INT32_MAX) return fail(DENDSN_E_INVALID, "step must be in [1, 2^31)");
  if (!aligned(step_dev, 4) || !aligned(grad_scale, 4)) return fail(DENDSN_E_INVALID, "step_dev or grad_scale misaligned");
  for (int64_t i = 0; i < count; ++i) {
    const dendsn_status st = check_tensor(cfg, tensors[i], i);
    if (st != DENDSN_OK) return st;
  }
  Batch a{};
  a.b1 = float(cfg->beta1); a.c1 = float(1.0 - cfg->beta1);
  a.b2 = float(cfg->beta2); a.c2 = float(1.0 - cfg->beta2);
  a.lr = float(cfg->lr); a.wd = float(cfg->weight_decay);
  // (the reciprocal takes what is below the normal numbers for 0: an eps that is not 0 stays one of them)
  a.eps = cfg->eps > 0.0 && cfg->eps < FLT_MIN ? FLT_MIN : float(cfg->eps);
  a.log_b1 = log(cfg->beta1); a.log_b2 = log(cfg->beta2);
  a.fix1 = float(-expm1(double(step) * a.log_b1)); a.fix2 = float(-expm1(double(step) * a.log_b2));
  a.step = uint32_t(step); a.seed_lo = uint32_t(seed); a.seed_hi = uint32_t(seed >> 32);
  a.step_dev = step_dev; a.grad_scale = grad_scale;
  int64_t blocks = 0;
  for (int64_t i = 0; i <= count; ++i) {
    const int64_t more = i < count ? ceil_div(tensors[i].n, kGroup * kGroups) : 0;
    if (i == count || a.count == kTensors || blocks + more > kMaxBlocks) {
      if (blocks > 0) {
        if (cfg->state == DENDSN_STATE_E4M3) adamw_kernel<true><<<dim3(unsigned(blocks)), dim3(kWaves * 64), 0, stream>>>(a);
        else adamw_kernel<false><<<dim3(unsigned(blocks)), dim3(kWaves * 64), 0, stream>>>(a);
        const dendsn_status st = launched("adamw");
        if (st != DENDSN_OK) return st;
      }
      a.count = 0;
      blocks = 0;
    }
    if (i == count) break;
    const dendsn_adamw_tensor& t = tensors[i];
    if (a.count == 0) a.base = int32_t(i);
    a.t[a.count++] = Tensor{t.param, t.grad, t.m, t.v, t.m_scale, t.v_scale, static_cast<bf16_t*>(t.copy), t.n,
                            uint32_t(blocks), uint32_t(t.grad_io == DENDSN_IO_BF16)};
    blocks += more;
  }
  return DENDSN_OK;
}
