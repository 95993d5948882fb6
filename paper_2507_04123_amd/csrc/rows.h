// Rows of 32- and 16-bit floating-point values, read and written in vectors and computed with in fp32: what the kernels of the
// sequence operators (layernorm.hip, recurrence.hip, ffn.hip, ffn_grad.hip) share.
#pragma once
#include "common.h"

template <typename T, int N> using emc2_vec = T __attribute__((ext_vector_type(N)));
template <int N> using emc2_fvec = emc2_vec<float, N>;

// N values at p as they lie in memory, anywhere: the target's vector loads and stores need no more than the alignment of a value, so rows of odd
// lengths and pitches move in 16-byte pieces too.
template <typename T, int N> struct emc2_anywhere { typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T)))); };
template <int N, typename T> __device__ __forceinline__ emc2_vec<T, N> emc2_piece(const T* p) {
  return *reinterpret_cast<const typename emc2_anywhere<T, N>::type*>(p);
}
// The same as floats; and back, one rounding to nearest even each.
template <int N, typename T> __device__ __forceinline__ emc2_fvec<N> emc2_load(const T* p) {
  return __builtin_convertvector(emc2_piece<N>(p), emc2_fvec<N>);
}
template <int N, typename T> __device__ __forceinline__ void emc2_store(T* p, emc2_fvec<N> v) {
  *reinterpret_cast<typename emc2_anywhere<T, N>::type*>(p) = __builtin_convertvector(v, emc2_vec<T, N>);
}

// Rows that a call deals with: the device count, if it is given, kept within the capacity.
__device__ __forceinline__ int32_t emc2_row_count(const int32_t* d_n, int64_t capacity) {
  if (!d_n) return (int32_t)capacity;
  const int32_t n = *d_n;
  return n < 0 ? 0 : n < capacity ? n : (int32_t)capacity;
}

// A launch of as many blocks as a call needs.  An axis of a grid has fewer than 2^32 threads: more than 2^21 blocks lie in lines of 2^21.
constexpr int64_t kEmc2BlocksALine = 1 << 21;
static inline dim3 emc2_grid(int64_t blocks) {
  return blocks <= kEmc2BlocksALine ? dim3((unsigned)blocks) : dim3((unsigned)kEmc2BlocksALine, (unsigned)((blocks + kEmc2BlocksALine - 1) / kEmc2BlocksALine));
}
__device__ __forceinline__ int64_t emc2_block() { return blockIdx.y * kEmc2BlocksALine + blockIdx.x; }

// The logistic function s = 1 / (1 + exp(-z)) and 1 - s = exp(-z) / (1 + exp(-z)), each to a few ulp: 1 - s is not taken from s, which
// would leave nothing of it where s is near 1.  Where exp(-z) is beyond the range s is 0 and 1 - s is 1; NaN passes through.
// EXACT (32-bit values): the exponent's product with log2(e) is carried to twice the precision, which matters beyond |z| of about 8.
template <bool EXACT> __device__ __forceinline__ float emc2_exp_of_minus(float z, float& t) {
  const float log2e = 1.44269504088896341f;
  t = -z * log2e;
  float e = __builtin_amdgcn_exp2f(t);
  if constexpr (EXACT) {
    const float low = __builtin_fmaf(-z, log2e, -t) - z * 1.92596299112661746e-8f;
    e = t > -126.0f && t < 126.0f ? __builtin_fmaf(e, low * 0.693147180559945309f, e) : e;
  }
  return e;
}
template <bool EXACT> __device__ __forceinline__ void emc2_logistic(float z, float& s, float& rest) {
  float t;
  const float e = emc2_exp_of_minus<EXACT>(z, t);
  s = __builtin_amdgcn_rcpf(1.0f + e);
  rest = t > 126.0f ? 1.0f : e * s;
}
template <bool EXACT> __device__ __forceinline__ float emc2_logistic(float z) {
  float t;
  return __builtin_amdgcn_rcpf(1.0f + emc2_exp_of_minus<EXACT>(z, t));
}

// Null, misaligned or overlapping-by-pitch rows are refused; p may be null if it is optional or there are no rows.
static inline bool emc2_rows_ok(const void* p, int64_t pitch, int32_t channels, size_t size, bool optional) {
  if (!p) return optional;
  return ((uintptr_t)p % size) == 0 && pitch >= channels && pitch <= (1ll << 40);
}
static inline size_t emc2_size_of(emc2_dtype dtype) { return dtype == EMC2_F32 ? 4 : 2; }
static inline bool emc2_is_float(emc2_dtype dtype) { return dtype == EMC2_F32 || dtype == EMC2_F16 || dtype == EMC2_BF16; }
