// Gated feed-forward network: the matrix-core fragments that its forward pass (ffn.hip) and its gradients (ffn_grad.hip) share.
//   G = x Wg, U = x Wu, H = act(G) * U, y = H Wd;   x [n][C], Wg and Wu [C][F], Wd [F][C]
// Everything is computed in tiles of 32 rows (voxels) by 32 hidden units with v_mfma_f32_32x32 (16 products deep for 16-bit values, 2
// for fp32).  A fragment is what one lane group of 64 holds of a 32-wide operand: lane l holds line l % 32 and, of the KF values
// along the contraction, PER = 16 bytes' worth: with half = l / 32 those at PER * half + e (e = 0 .. PER - 1).
// A result tile leaves lane l with column l % 32 and rows 8 j + 4 half + i in register 4 j + i.  Read as a fragment, its registers
// PER m .. PER m + PER - 1 are values hidden_of(m, half, e) along its rows: a product's result is the next product's operand
// without leaving the registers, if the other operand (packed weights) has its values in that order.  So H, dG and dU never leave the chip.
#pragma once
#include "rows.h"

template <typename T> struct emc2_tile {
  static constexpr int kPer = 16 / sizeof(T);       // values of a fragment in a lane
  static constexpr int kDeep = 2 * kPer;            // and along the contraction (KF)
  typedef emc2_vec<T, kPer> frag;
};
typedef emc2_fvec<16> emc2_acc;

template <typename T> __device__ __forceinline__ emc2_acc emc2_mma(emc2_vec<T, 16 / sizeof(T)> a, emc2_vec<T, 16 / sizeof(T)> b, emc2_acc c) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
  } else if constexpr (__is_same(T, _Float16)) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
}

// Place along a result tile's rows of value e of fragment m made of its registers.
template <typename T> __host__ __device__ __forceinline__ constexpr int emc2_hidden_of(int m, int half, int e) {
  return emc2_tile<T>::kDeep * m + 8 * (e / 4) + 4 * half + e % 4;
}

// Packed weights: for every slice of 32 hidden units (an even number of slices) six groups of width / KF fragments (width: C rounded up to 32s, zeros beyond C and F):
enum emc2_ffn_group {   // the forward pass takes the first three, dx the last five, the weights' gradients the three from EMC2_FFN_GATE on
  EMC2_FFN_DOWN,        // Wd: line = channel (fragment ct * 32 / KF + m: channels 32 ct ..), along = hidden units in the order of a result tile
  EMC2_FFN_GATE,        // Wg: line = hidden unit, along = channel
  EMC2_FFN_UP,          // Wu: the same
  EMC2_FFN_DOWN_T,      // Wd: the same
  EMC2_FFN_GATE_T,      // Wg: line = channel, along = hidden units in the order of a result tile
  EMC2_FFN_UP_T,        // Wu: the same
  EMC2_FFN_GROUPS
};

template <typename T> __device__ __forceinline__ typename emc2_tile<T>::frag emc2_zero_frag() { return typename emc2_tile<T>::frag(T(0)); }

// The fragment of row `row`, along channels kk KF ..; zero beyond the rows and channels.  WIDE: rows are whole pieces of 16 bytes.
template <typename T, bool WIDE>
__device__ __forceinline__ typename emc2_tile<T>::frag emc2_row_frag(const T* p, int64_t ld, int64_t row, int32_t n, int32_t channels, int kk, int half) {
  typedef emc2_tile<T> M;
  const int c = kk * M::kDeep + half * M::kPer;
  typename M::frag f = emc2_zero_frag<T>();
  if (row < n && c < channels) {
    const T* q = p + row * ld + c;
    if (WIDE || c + M::kPer <= channels) {
      f = emc2_piece<M::kPer>(q);
    } else {
#pragma unroll
      for (int e = 0; e < M::kPer; ++e)
        if (c + e < channels) f[e] = q[e];
    }
  }
  return f;
}

// The fragments of a row: kept in registers, or (wide rows of fp32, which would take half of them) read again for every use.
template <typename T, int CT, bool WIDE> struct emc2_row {
  typedef emc2_tile<T> M;
  static constexpr int KK = 32 * CT / M::kDeep;
  static constexpr bool kKept = sizeof(T) * CT <= 16;
  typename M::frag f[kKept ? KK : 1];
  const T* p;
  int64_t ld, row;
  int32_t n, channels;
  int half;
  __device__ __forceinline__ void set(const void* p_, int64_t ld_, int64_t row_, int32_t n_, int32_t channels_, int half_) {
    p = (const T*)p_, ld = ld_, row = row_, n = n_, channels = channels_, half = half_;
    if constexpr (kKept) {
#pragma unroll
      for (int k = 0; k < KK; ++k) f[k] = emc2_row_frag<T, WIDE>(p, ld, row, n, channels, k, half);
    }
  }
  // before a loop's turn: what is read again is not moved out of the loop
  __device__ __forceinline__ void again() {
    if constexpr (!kKept) asm volatile("" : "+v"(p));
  }
  __device__ __forceinline__ typename M::frag operator[](int k) const {
    if constexpr (kKept) return f[k];
    else return emc2_row_frag<T, WIDE>(p, ld, row, n, channels, k, half);
  }
};

// act(g) of either activation as g s, s = logistic(z): SiLU z = g, GELU (its tanh form) z = sqrt(8 / pi) (g + 0.044715 g^3); and the slope
// s + g s (1 - s) dz/dg (1 - s is taken from s here: where nothing is left of it, the slope is s; g^2 is held finite for that).
template <bool EXACT, bool GELU> __device__ __forceinline__ float emc2_activate(float g) {
  return g * emc2_logistic<EXACT>(GELU ? 1.5957691216057308f * (g + 0.044715f * g * g * g) : g);
}
template <bool EXACT, bool GELU> __device__ __forceinline__ float emc2_activate(float g, float& slope) {
  const float sq = GELU ? __builtin_fminf(g * g, 1e30f) : 0.0f;
  const float s = emc2_logistic<EXACT>(GELU ? g * __builtin_fmaf(sq, 0.0713548163f, 1.5957691216057308f) : g), a = g * s;
  const float rest = GELU ? (1.0f - s) * __builtin_fmaf(sq, 0.2140644488f, 1.5957691216057308f) : 1.0f - s;
  slope = __builtin_fmaf(a, rest, s);
  return a;
}
// Two neighbouring values of a result tile, registers r and r + 1 (r even), into the fragments made of it: P = 1 rounded, P = 2 also what the rounding
// leaves over, in fragments of its own, whose products with the same operand make up for it.
template <typename T> __device__ __forceinline__ void emc2_put_pair(typename emc2_tile<T>::frag* f, int r, emc2_vec<T, 2> v) {
  constexpr int kPer = emc2_tile<T>::kPer;
  if constexpr (sizeof(T) == 2) {
    emc2_vec<uint32_t, 4> w = __builtin_bit_cast(emc2_vec<uint32_t, 4>, f[r / kPer]);
    w[r % kPer / 2] = __builtin_bit_cast(uint32_t, v);
    f[r / kPer] = __builtin_bit_cast(typename emc2_tile<T>::frag, w);
  } else {
    f[r / kPer][r % kPer] = v[0], f[r / kPer][r % kPer + 1] = v[1];
  }
}
template <typename T> __device__ __forceinline__ void emc2_put_pair(typename emc2_tile<T>::frag* f, int r, float a, float b) {
  emc2_put_pair<T>(f, r, __builtin_convertvector((emc2_fvec<2>{a, b}), emc2_vec<T, 2>));
}
template <typename T, int P, int MM>
__device__ __forceinline__ void emc2_put_pair(typename emc2_tile<T>::frag (&f)[P][MM], int r, float a, float b) {
  const emc2_vec<T, 2> v = __builtin_convertvector((emc2_fvec<2>{a, b}), emc2_vec<T, 2>);
  emc2_put_pair<T>(f[0], r, v);
  if constexpr (P == 2) {
    const emc2_fvec<2> q = __builtin_convertvector(v, emc2_fvec<2>);
    emc2_put_pair<T>(f[1], r, __builtin_convertvector((emc2_fvec<2>{a - q[0], b - q[1]}), emc2_vec<T, 2>));
  }
}

// Rows up to which 16-bit hidden values and their gradients are held in two parts (P = 2), the rounded value and what that leaves over: results are as near as
// with fp32 hidden values.  One part adds an error as large as the result's own rounding (1.4 times the plain one's over many values, up to twice over those of
// a few rows).  A second product each is hidden by the latency of small calls and not by the products of large ones.  us, one part / two: forward, 24 rows x 128 x 512 f16
// 8.5 / 8.9, 300 x 256 x 1024 27 / 31, 16 k x 128 x 512 18 / 20 (bf16), 300 k 162 / 185 (f16) and 139 / 166 (bf16); with gradients, 24 rows x 128 x 512 f16 40 / 42,
// 2 k x 64 x 256 29 / 29, 2 k x 128 x 512 bf16 49 / 51, 2 k x 256 x 512 f16 141 / 158, 100 k x 64 x 256 bf16 106 / 122 (forward in one part).
constexpr int64_t kFfnRestRows = 2048;

// Arguments of a launch.
struct emc2_ffn_args {
  const void *x, *res, *dy, *packed;
  void* y;                    // forward: the result; backward: dx
  float* partial;             // weight gradients of every part of the rows
  const int32_t* d_n;
  int64_t ld_x, ld_res, ld_dy, ld_y, capacity;
  int32_t channels, hidden, slices, parts;
};

static inline int emc2_ffn_tiles(int32_t channels) {        // 32-wide tiles of channels that the kernels are made for
  const int t = (channels + 31) / 32;
  return t <= 4 ? t : t <= 6 ? 6 : 8;
}
static inline int32_t emc2_ffn_slices(int32_t hidden) { return (hidden + 63) / 64 * 2; }
constexpr int kFfnMaxChannels = 256, kFfnMaxHidden = 1 << 16;

// Calls f with a value of the type, and as constants the number of tiles, whether the activation is GELU and whether rows are whole pieces of 16 bytes.
template <int N> struct emc2_const { static constexpr int value = N; };
template <typename F> void emc2_ffn_dispatch(emc2_dtype dtype, int tiles, bool gelu, bool wide, F&& f) {
  const auto by_act = [&](auto type, auto count) {
    if (gelu && wide) f(type, count, emc2_const<1>(), emc2_const<1>());
    else if (gelu) f(type, count, emc2_const<1>(), emc2_const<0>());
    else if (wide) f(type, count, emc2_const<0>(), emc2_const<1>());
    else f(type, count, emc2_const<0>(), emc2_const<0>());
  };
  const auto by_tiles = [&](auto type) {
    switch (tiles) {
      case 1: return by_act(type, emc2_const<1>());
      case 2: return by_act(type, emc2_const<2>());
      case 3: return by_act(type, emc2_const<3>());
      case 4: return by_act(type, emc2_const<4>());
      case 6: return by_act(type, emc2_const<6>());
      default: return by_act(type, emc2_const<8>());
    }
  };
  if (dtype == EMC2_F32) by_tiles(float());
  else if (dtype == EMC2_F16) by_tiles(_Float16());
  else by_tiles(__bf16());
}
emc2_status emc2_ffn_check(emc2_ctx* ctx, const char* what, emc2_dtype dtype, int32_t activation, int64_t capacity, int32_t channels,
                           int32_t hidden, const void* packed);
