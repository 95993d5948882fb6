// Rows of 32- and 16-bit floating-point values, read and written in vectors and computed with in fp32: what the kernels of the
// sequence operators (layernorm.hip, recurrence.hip, ffn.hip, ffn_grad.hip) share.
#pragma once
#include "common.h"

template <typename T, int N> using emc2_vec = T __attribute__((ext_vector_type(N)));
template <int N> using emc2_fvec = emc2_vec<float, N>;

// N values at p, which lies on a multiple of their size (of 16 bytes where they take more), as floats; and back, one rounding to
// nearest even each.
template <int N, typename T> __device__ __forceinline__ emc2_fvec<N> emc2_load(const T* p) {
  return __builtin_convertvector(*reinterpret_cast<const emc2_vec<T, N>*>(p), emc2_fvec<N>);
}
template <int N, typename T> __device__ __forceinline__ void emc2_store(T* p, emc2_fvec<N> v) {
  *reinterpret_cast<emc2_vec<T, N>*>(p) = __builtin_convertvector(v, emc2_vec<T, N>);
}
// N floats of a parameter vector that lies on a multiple of 16 bytes (4 where N is 1)
template <int N> __device__ __forceinline__ emc2_fvec<N> emc2_load_params(const float* p) {
  if constexpr (N <= 4) {
    return *reinterpret_cast<const emc2_fvec<N>*>(p);
  } else {
    emc2_fvec<N> v;
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const emc2_fvec<4> q = *reinterpret_cast<const emc2_fvec<4>*>(p + i);
      v[i] = q[0], v[i + 1] = q[1], v[i + 2] = q[2], v[i + 3] = q[3];
    }
    return v;
  }
}
template <int N> __device__ __forceinline__ void emc2_store_params(float* p, emc2_fvec<N> v) {
  if constexpr (N <= 4) {
    *reinterpret_cast<emc2_fvec<N>*>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<emc2_fvec<4>*>(p + i) = emc2_fvec<4>{v[i], v[i + 1], v[i + 2], v[i + 3]};
  }
}

// Rows that a call deals with: the device count, if it is given, kept within the capacity.
__device__ __forceinline__ int32_t emc2_row_count(const int32_t* d_n, int64_t capacity) {
  if (!d_n) return (int32_t)capacity;
  const int32_t n = *d_n;
  return n < 0 ? 0 : n < capacity ? n : (int32_t)capacity;
}

// The logistic function s = 1 / (1 + exp(-z)) and 1 - s = exp(-z) / (1 + exp(-z)), each to a few ulp: 1 - s is not taken from s, which
// would leave nothing of it where s is near 1.  Where exp(-z) is beyond the range s is 0 and 1 - s is 1; NaN passes through.
// EXACT (32-bit values): the exponent's product with log2(e) is carried to twice the precision, which matters beyond |z| of about 8.
template <bool EXACT> __device__ __forceinline__ void emc2_logistic(float z, float& s, float& rest) {
  const float log2e = 1.44269504088896341f;
  const float t = -z * log2e;
  float e = __builtin_amdgcn_exp2f(t);
  if constexpr (EXACT) {
    const float low = __builtin_fmaf(-z, log2e, -t) - z * 1.92596299112661746e-8f;
    e = t > -126.0f && t < 126.0f ? __builtin_fmaf(e, low * 0.693147180559945309f, e) : e;
  }
  s = __builtin_amdgcn_rcpf(1.0f + e);
  rest = t > 126.0f ? 1.0f : e * s;
}

// True if the rows at p, `pitch` elements apart, can be moved in pieces of 16 bytes (p may be null).
static inline bool emc2_wide_rows(const void* p, int64_t pitch, size_t size) {
  return ((uintptr_t)p & 15) == 0 && (pitch * (int64_t)size) % 16 == 0;
}
// Null, misaligned or overlapping-by-pitch rows are refused; p may be null if it is optional or there are no rows.
static inline bool emc2_rows_ok(const void* p, int64_t pitch, int32_t channels, size_t size, bool optional) {
  if (!p) return optional;
  return ((uintptr_t)p % size) == 0 && pitch >= channels && pitch <= (1ll << 40);
}
static inline size_t emc2_size_of(emc2_dtype dtype) { return dtype == EMC2_F32 ? 4 : 2; }
static inline bool emc2_is_float(emc2_dtype dtype) { return dtype == EMC2_F32 || dtype == EMC2_F16 || dtype == EMC2_BF16; }
