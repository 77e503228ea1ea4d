// What the token-sequence operators share: error reporting, argument helpers,
// element types and their wide loads.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "dendsn_seq.h"

namespace dendsn_seq {

// Records a description for dendsn_seq_last_error() and returns the status.  The text
// lives in a fixed buffer: a C entry point throws nothing, out of memory included.
dendsn_status fail(dendsn_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
void clear_error();
dendsn_status launched(const char* what);  // DENDSN_E_HIP if the last launch failed

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
__host__ __device__ inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
__host__ __device__ inline int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

constexpr int64_t kMaxElems = int64_t(1) << 46;  // of one tensor, strides included

// a * b <= kMaxElems for non-negative a, b.
inline bool small_product(int64_t a, int64_t b) { return a == 0 || b == 0 || a <= kMaxElems / b; }

// Carves 256-byte aligned arrays out of a workspace.
struct Carve {
  size_t at = 0;
  size_t take(size_t bytes) {
    const size_t o = at;
    at += (bytes + 255) / 256 * 256;
    return o;
  }
};

dendsn_status check_workspace(const void* ws, size_t have, size_t need, const char* query);

// ---------------------------------------------------------------------------
// bf16 storage: 16 bits, widened exactly, narrowed round-to-nearest-even (NaN
// stays NaN) by the hardware conversion.
// ---------------------------------------------------------------------------
struct bf16_t {
  uint16_t bits;
};

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16_t v) { return __uint_as_float(uint32_t(v.bits) << 16); }

__device__ __forceinline__ uint16_t bf16_bits(float v) {
  const __bf16 b = static_cast<__bf16>(v);
  return __builtin_bit_cast(uint16_t, b);
}

template <typename IO>
__device__ __forceinline__ IO narrow(float v);
template <>
__device__ __forceinline__ float narrow<float>(float v) { return v; }
template <>
__device__ __forceinline__ bf16_t narrow<bf16_t>(float v) { return bf16_t{bf16_bits(v)}; }

// V adjacent elements, moved by one load or store.  The address need be no multiple of
// more than an element's size: the memory pipe takes any, so odd rows go as wide as even
// ones.
template <typename IO, int V>
struct __attribute__((packed, aligned(sizeof(IO)))) Pack {
  IO v[V];
};

}  // namespace dendsn_seq
