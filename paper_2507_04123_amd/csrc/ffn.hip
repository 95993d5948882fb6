// Gated feed-forward network, forward pass and the order of its weights (ffn.h has the mathematics and the fragments).
// A wave keeps its 32 rows of x and of y's sums in registers and walks the hidden units in slices of 32: two products for G and U, the
// activation, H rounded to the operands' type (the matrix cores multiply 16-bit values; its error is that of the result's own rounding),
// and the product with the slice's lines of Wd.
#include "ffn.h"

namespace {

constexpr int kThreads = 256;

template <typename T, int CT>
__global__ void __launch_bounds__(kThreads) k_ffn(const emc2_ffn_args a) {
  typedef emc2_tile<T> M;
  typedef typename M::frag frag;
  constexpr int KK = 32 * CT / M::kDeep, MM = 32 / M::kDeep;
  const int32_t n = emc2_row_count(a.d_n, a.capacity);
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int64_t row = ((int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)) * 32 + (lane & 31);
  if (row - (lane & 31) >= n) return;
  emc2_row<T, CT> x;
  x.set(a.x, a.ld_x, row, n, a.wide, a.channels, half);
  emc2_acc y[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) y[c] = 0.0f;
  const frag* w = (const frag*)a.packed + lane;
  for (int32_t s = 0; s < a.slices; ++s, w += EMC2_FFN_GROUPS * KK * 64) {
    emc2_acc g = 0.0f, u = 0.0f;
    x.again();
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      g = emc2_mma<T>(w[(EMC2_FFN_GATE * KK + k) * 64], x[k], g);
      u = emc2_mma<T>(w[(EMC2_FFN_UP * KK + k) * 64], x[k], u);
    }
    frag h[MM];
#pragma unroll
    for (int m = 0; m < MM; ++m)
#pragma unroll
      for (int e = 0; e < M::kPer; ++e) {
        const int r = m * M::kPer + e;
        h[m][e] = (T)(emc2_activate<sizeof(T) == 4>(a.gelu, g[r]) * u[r]);
      }
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int m = 0; m < MM; ++m) y[c] = emc2_mma<T>(w[(EMC2_FFN_DOWN * KK + c * MM + m) * 64], h[m], y[c]);
  }
  if (row >= n) return;
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int at = 32 * c + 8 * j + 4 * half;
      emc2_fvec<4> v = {y[c][4 * j], y[c][4 * j + 1], y[c][4 * j + 2], y[c][4 * j + 3]};
      T* out = (T*)a.y + row * a.ld_y + at;
      const T* res = (const T*)a.res + row * a.ld_res + at;
      if (a.wide) {
        if (at >= a.channels) continue;
        if (a.res) v += emc2_load<4>(res);
        emc2_store<4>(out, v);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (at + i < a.channels) out[i] = (T)(v[i] + (a.res ? (float)res[i] : 0.0f));
      }
    }
}

// One lane's 16 bytes of a fragment a thread.
template <typename T>
__global__ void __launch_bounds__(kThreads) k_ffn_pack(const T* __restrict__ wg, const T* __restrict__ wu, const T* __restrict__ wd,
                                                       int32_t channels, int32_t hidden, int32_t tiles, int64_t pieces, T* __restrict__ packed) {
  typedef emc2_tile<T> M;
  const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (at >= pieces) return;
  const int kk = 32 * tiles / M::kDeep, mm = 32 / M::kDeep;
  const int lane = (int)(at & 63), half = lane >> 5, line = lane & 31;
  const int64_t frag = at >> 6;
  const int k = (int)(frag % kk), group = (int)(frag / kk % EMC2_FFN_GROUPS);
  const int32_t f0 = (int32_t)(frag / kk / EMC2_FFN_GROUPS) * 32;
  const bool along_channels = group == EMC2_FFN_GATE || group == EMC2_FFN_UP || group == EMC2_FFN_DOWN_T;
  const T* w = group == EMC2_FFN_GATE || group == EMC2_FFN_GATE_T ? wg : group == EMC2_FFN_UP || group == EMC2_FFN_UP_T ? wu : wd;
  const bool by_hidden = w == wd;                          // Wd has its lines by hidden unit, Wg and Wu by channel
  typename M::frag v = emc2_zero_frag<T>();
#pragma unroll
  for (int e = 0; e < M::kPer; ++e) {
    const int32_t c = along_channels ? k * M::kDeep + half * M::kPer + e : k / mm * 32 + line;
    const int32_t f = f0 + (along_channels ? line : emc2_hidden_of<T>(k % mm, half, e));
    if (c < channels && f < hidden) v[e] = by_hidden ? w[(int64_t)f * channels + c] : w[(int64_t)c * hidden + f];
  }
  *reinterpret_cast<typename M::frag*>(packed + at * M::kPer) = v;
}

int64_t packed_values(int32_t channels, int32_t hidden) {
  return (int64_t)EMC2_FFN_GROUPS * 32 * emc2_ffn_tiles(channels) * 32 * ((hidden + 31) / 32);
}

}  // namespace

emc2_status emc2_ffn_check(emc2_ctx* ctx, const char* what, emc2_dtype dtype, int32_t activation, int64_t capacity, int32_t channels,
                           int32_t hidden, const void* packed) {
  if (!emc2_is_float(dtype)) return emc2_fail(ctx, EMC2_ERR_UNSUPPORTED, "%s: dtype must be F32, F16 or BF16", what);
  if (channels < 1 || channels > kFfnMaxChannels || hidden < 1 || hidden > kFfnMaxHidden)
    return emc2_fail(ctx, EMC2_ERR_UNSUPPORTED, "%s: channels outside [1, %d] or hidden outside [1, %d]", what, kFfnMaxChannels, kFfnMaxHidden);
  if (activation != EMC2_ACT_SILU && activation != EMC2_ACT_GELU)
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: activation must be EMC2_ACT_SILU or EMC2_ACT_GELU", what);
  if (capacity < 0 || capacity > (1ll << 30)) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: capacity outside [0, 2^30]", what);
  if (!packed || ((uintptr_t)packed & 15)) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: packed weights null or not 16-byte aligned", what);
  return EMC2_OK;
}

extern "C" int64_t emc2_ffn_packed_size(emc2_dtype dtype, int32_t channels, int32_t hidden) {
  if (!emc2_is_float(dtype) || channels < 1 || channels > kFfnMaxChannels || hidden < 1 || hidden > kFfnMaxHidden) return -1;
  return packed_values(channels, hidden);
}

extern "C" emc2_status emc2_ffn_pack(emc2_ctx* ctx, emc2_dtype dtype, const void* d_wg, const void* d_wu, const void* d_wd, int32_t channels,
                                     int32_t hidden, void* d_packed, void* stream) {
  if (!ctx) return EMC2_ERR_INVALID_ARG;
  const emc2_status st = emc2_ffn_check(ctx, "emc2_ffn_pack", dtype, EMC2_ACT_SILU, 0, channels, hidden, d_packed);
  if (st != EMC2_OK) return st;
  const size_t size = emc2_size_of(dtype);
  if (!d_wg || !d_wu || !d_wd || (uintptr_t)d_wg % size || (uintptr_t)d_wu % size || (uintptr_t)d_wd % size)
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_ffn_pack: weights null or misaligned");
  const int tiles = emc2_ffn_tiles(channels);
  const int64_t pieces = packed_values(channels, hidden) / (16 / (int64_t)size);
  const dim3 grid((unsigned)emc2_div_up(pieces, kThreads));
  hipStream_t s = (hipStream_t)stream;
  if (dtype == EMC2_F32)
    hipLaunchKernelGGL(k_ffn_pack<float>, grid, dim3(kThreads), 0, s, (const float*)d_wg, (const float*)d_wu, (const float*)d_wd, channels,
                       hidden, tiles, pieces, (float*)d_packed);
  else if (dtype == EMC2_F16)
    hipLaunchKernelGGL(k_ffn_pack<_Float16>, grid, dim3(kThreads), 0, s, (const _Float16*)d_wg, (const _Float16*)d_wu, (const _Float16*)d_wd,
                       channels, hidden, tiles, pieces, (_Float16*)d_packed);
  else
    hipLaunchKernelGGL(k_ffn_pack<__bf16>, grid, dim3(kThreads), 0, s, (const __bf16*)d_wg, (const __bf16*)d_wu, (const __bf16*)d_wd, channels,
                       hidden, tiles, pieces, (__bf16*)d_packed);
  return emc2_check_hip(ctx, hipGetLastError(), "emc2_ffn_pack launch");
}

extern "C" emc2_status emc2_ffn(emc2_ctx* ctx, emc2_dtype dtype, int32_t activation, const void* d_x, int64_t ld_x, const void* d_packed,
                                const void* d_res, int64_t ld_res, const int32_t* d_n, int64_t capacity, int32_t channels, int32_t hidden,
                                void* d_y, int64_t ld_y, void* stream) {
  if (!ctx) return EMC2_ERR_INVALID_ARG;
  const emc2_status st = emc2_ffn_check(ctx, "emc2_ffn", dtype, activation, capacity, channels, hidden, d_packed);
  if (st != EMC2_OK) return st;
  const size_t size = emc2_size_of(dtype);
  const bool none = capacity == 0;
  if (!emc2_rows_ok(d_x, ld_x, channels, size, none) || !emc2_rows_ok(d_y, ld_y, channels, size, none) ||
      !emc2_rows_ok(d_res, ld_res, channels, size, true))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_ffn: null or misaligned rows, or a pitch below the channels");
  if (none) return EMC2_OK;
  emc2_ffn_args a = {};
  a.x = d_x, a.res = d_res, a.packed = d_packed, a.y = d_y, a.d_n = d_n, a.ld_x = ld_x, a.ld_res = ld_res, a.ld_y = ld_y;
  a.capacity = capacity, a.channels = channels, a.hidden = hidden, a.slices = (hidden + 31) / 32, a.gelu = activation == EMC2_ACT_GELU;
  a.wide = channels % (16 / size) == 0 && emc2_wide_rows(d_x, ld_x, size) && emc2_wide_rows(d_y, ld_y, size) &&
           (!d_res || emc2_wide_rows(d_res, ld_res, size));
  emc2_ffn_dispatch(dtype, emc2_ffn_tiles(channels), [&](auto type, auto tiles) {
    using T = decltype(type);
    constexpr int CT = decltype(tiles)::value;
    hipLaunchKernelGGL((k_ffn<T, CT>), dim3((unsigned)emc2_div_up(capacity, 128)), dim3(kThreads), 0, (hipStream_t)stream, a);
  });
  return emc2_check_hip(ctx, hipGetLastError(), "emc2_ffn launch");
}
