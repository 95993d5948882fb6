// Gradients of the gated feed-forward network (ffn.h has the mathematics of the forward pass and the fragments).
//   dH = dy Wd^T, dU = dH act(G), dG = dH U act'(G);   dx = dG Wg^T + dU Wu^T;   dWg = x^T dG, dWu = x^T dU, dWd = H^T dy
// G, U and dH are computed again in both kernels rather than stored: a slice of 32 hidden units costs 3 products per pass, and storing H, dG
// and dU would move six times n F values.
// k_ffn_dx works like the forward pass: hidden units along the lanes' registers, rows along the lanes.
// k_ffn_dw has them the other way round (rows along the registers), which is what a contraction over rows takes: dG, dU and H are its operands as
// they are.  x and dy have to be turned round for it: a product with the identity does that on the matrix cores, exactly.  Each wave sums
// its slice of 32 hidden units over a part of the rows; the parts are added by k_ffn_sum in a fixed order (fp32, no atomics).
#include "ffn.h"

namespace {

constexpr int kThreads = 256;

template <typename T, int CT>
__global__ void __launch_bounds__(kThreads) k_ffn_dx(const emc2_ffn_args a) {
  typedef emc2_tile<T> M;
  typedef typename M::frag frag;
  constexpr int KK = 32 * CT / M::kDeep, MM = 32 / M::kDeep;
  const int32_t n = emc2_row_count(a.d_n, a.capacity);
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int64_t row = ((int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)) * 32 + (lane & 31);
  if (row - (lane & 31) >= n) return;
  emc2_row<T, CT> x, dy;
  x.set(a.x, a.ld_x, row, n, a.wide, a.channels, half);
  dy.set(a.dy, a.ld_dy, row, n, a.wide, a.channels, half);
  emc2_acc dx[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) dx[c] = 0.0f;
  const frag* w = (const frag*)a.packed + lane;
  for (int32_t s = 0; s < a.slices; ++s, w += EMC2_FFN_GROUPS * KK * 64) {
    emc2_acc g = 0.0f, u = 0.0f, dh = 0.0f;
    x.again(), dy.again();
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      g = emc2_mma<T>(w[(EMC2_FFN_GATE * KK + k) * 64], x[k], g);
      u = emc2_mma<T>(w[(EMC2_FFN_UP * KK + k) * 64], x[k], u);
      dh = emc2_mma<T>(w[(EMC2_FFN_DOWN_T * KK + k) * 64], dy[k], dh);
    }
    frag dg[MM], du[MM];
#pragma unroll
    for (int m = 0; m < MM; ++m)
#pragma unroll
      for (int e = 0; e < M::kPer; ++e) {
        const int r = m * M::kPer + e;
        float slope;
        const float act = emc2_activate<sizeof(T) == 4>(a.gelu, g[r], slope);
        dg[m][e] = (T)(dh[r] * u[r] * slope);
        du[m][e] = (T)(dh[r] * act);
      }
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int m = 0; m < MM; ++m) {
        dx[c] = emc2_mma<T>(w[(EMC2_FFN_GATE_T * KK + c * MM + m) * 64], dg[m], dx[c]);
        dx[c] = emc2_mma<T>(w[(EMC2_FFN_UP_T * KK + c * MM + m) * 64], du[m], dx[c]);
      }
  }
  if (row >= n) return;
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int at = 32 * c + 8 * j + 4 * half;
      const emc2_fvec<4> v = {dx[c][4 * j], dx[c][4 * j + 1], dx[c][4 * j + 2], dx[c][4 * j + 3]};
      T* out = (T*)a.y + row * a.ld_y + at;
      if (a.wide) {
        if (at < a.channels) emc2_store<4>(out, v);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (at + i < a.channels) out[i] = (T)v[i];
      }
    }
}

// Fragments of a tile's 32 columns of x or dy, rows along the lanes' registers: the rows' fragments times the identity.
template <typename T, int CT, int MM>
__device__ __forceinline__ void turned(const emc2_row<T, CT>& rows, int first, const typename emc2_tile<T>::frag (&one)[MM],
                                       typename emc2_tile<T>::frag (&out)[MM]) {
  emc2_acc t = 0.0f;
#pragma unroll
  for (int m = 0; m < MM; ++m) t = emc2_mma<T>(rows[first + m], one[m], t);
#pragma unroll
  for (int m = 0; m < MM; ++m)
#pragma unroll
    for (int e = 0; e < emc2_tile<T>::kPer; ++e) out[m][e] = (T)t[m * emc2_tile<T>::kPer + e];
}

// Partial sums [part][slice][3][C / 32][64 lanes][16]: of a tile of dWg, dWu (rows: channels, columns: hidden units) and of dWd (rows: hidden
// units, columns: channels).  C0: the first of the CB tiles of channels whose sums the launch takes.
template <typename T, int CT, int C0, int CB>
__global__ void __launch_bounds__(kThreads, 1) k_ffn_dw(const emc2_ffn_args a) {
  typedef emc2_tile<T> M;
  typedef typename M::frag frag;
  constexpr int KK = 32 * CT / M::kDeep, MM = 32 / M::kDeep;
  const int32_t n = emc2_row_count(a.d_n, a.capacity);
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int64_t wave = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  const int32_t s = (int32_t)(wave % a.slices), part = (int32_t)(wave / a.slices);
  if (part >= a.parts) return;
  const frag* w = (const frag*)a.packed + (int64_t)s * EMC2_FFN_GROUPS * KK * 64 + lane;
  frag one[MM];
#pragma unroll
  for (int m = 0; m < MM; ++m)
#pragma unroll
    for (int e = 0; e < M::kPer; ++e) one[m][e] = (T)(m * M::kDeep + half * M::kPer + e == (lane & 31) ? 1.0f : 0.0f);
  emc2_acc dwg[CB], dwu[CB], dwd[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) dwg[c] = 0.0f, dwu[c] = 0.0f, dwd[c] = 0.0f;
  for (int64_t tile = part; tile * 32 < n; tile += a.parts) {
    const int64_t row = tile * 32 + (lane & 31);
    if constexpr (sizeof(T) * CT > 8) asm volatile("" : "+v"(w));   // too many weights to keep in registers: loaded again for every tile
    emc2_row<T, CT> x, dy;
    x.set(a.x, a.ld_x, row, n, a.wide, a.channels, half);
    dy.set(a.dy, a.ld_dy, row, n, a.wide, a.channels, half);
    emc2_acc g = 0.0f, u = 0.0f, dh = 0.0f;
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      g = emc2_mma<T>(x[k], w[(EMC2_FFN_GATE * KK + k) * 64], g);
      u = emc2_mma<T>(x[k], w[(EMC2_FFN_UP * KK + k) * 64], u);
      dh = emc2_mma<T>(dy[k], w[(EMC2_FFN_DOWN_T * KK + k) * 64], dh);
    }
    frag h[MM], dg[MM], du[MM];
#pragma unroll
    for (int m = 0; m < MM; ++m)
#pragma unroll
      for (int e = 0; e < M::kPer; ++e) {
        const int r = m * M::kPer + e;
        float slope;
        const float act = emc2_activate<sizeof(T) == 4>(a.gelu, g[r], slope);
        h[m][e] = (T)(act * u[r]);
        dg[m][e] = (T)(dh[r] * u[r] * slope);
        du[m][e] = (T)(dh[r] * act);
      }
#pragma unroll
    for (int c = 0; c < CB; ++c) {
      frag t[MM];
      turned<T, CT, MM>(x, (C0 + c) * MM, one, t);
#pragma unroll
      for (int m = 0; m < MM; ++m) dwg[c] = emc2_mma<T>(t[m], dg[m], dwg[c]), dwu[c] = emc2_mma<T>(t[m], du[m], dwu[c]);
      turned<T, CT, MM>(dy, (C0 + c) * MM, one, t);
#pragma unroll
      for (int m = 0; m < MM; ++m) dwd[c] = emc2_mma<T>(h[m], t[m], dwd[c]);
    }
  }
  emc2_acc* out = (emc2_acc*)a.partial + (((int64_t)part * a.slices + s) * 3 * CT + C0) * 64 + lane;
#pragma unroll
  for (int c = 0; c < CB; ++c) out[c * 64] = dwg[c], out[(CT + c) * 64] = dwu[c], out[(2 * CT + c) * 64] = dwd[c];
}

// Adds the parts, four values a thread, and puts them where they belong.
template <typename T>
__global__ void __launch_bounds__(kThreads) k_ffn_sum(const float4* __restrict__ partial, int32_t parts, int32_t slices, int32_t tiles,
                                                      int32_t channels, int32_t hidden, T* __restrict__ dwg, T* __restrict__ dwu,
                                                      T* __restrict__ dwd) {
  const int64_t quads = (int64_t)slices * 3 * tiles * 64 * 4, at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (at >= quads) return;
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
  for (int32_t p = 0; p < parts; ++p) {
    const float4 q = partial[p * quads + at];
    s.x += q.x, s.y += q.y, s.z += q.z, s.w += q.w;
  }
  const int j = (int)(at & 3), lane = (int)(at >> 2 & 63);
  const int64_t rest = at >> 8;
  const int tile = (int)(rest % tiles), which = (int)(rest / tiles % 3);
  const int32_t slice = (int32_t)(rest / tiles / 3);
  const int32_t row = 8 * j + 4 * (lane >> 5), col = lane & 31;
  const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int32_t c = tile * 32 + (which == 2 ? col : row + i), f = slice * 32 + (which == 2 ? row + i : col);
    if (c < channels && f < hidden) {
      if (which == 2) dwd[(int64_t)f * channels + c] = (T)v[i];
      else (which ? dwu : dwg)[(int64_t)c * hidden + f] = (T)v[i];
    }
  }
}

// Parts that the rows are cut into: enough that every SIMD has a wave, none without rows.
int32_t parts_of(int64_t capacity, int32_t hidden) {
  const int64_t slices = (hidden + 31) / 32, aim = emc2_div_up(1024, slices), tiles = emc2_div_up(capacity, 32);
  const int64_t parts = aim < tiles ? aim : tiles;
  return (int32_t)(parts < 1 ? 1 : parts);
}

}  // namespace

extern "C" int64_t emc2_ffn_work(emc2_dtype dtype, int64_t capacity, int32_t channels, int32_t hidden) {
  if (!emc2_is_float(dtype) || channels < 1 || channels > kFfnMaxChannels || hidden < 1 || hidden > kFfnMaxHidden || capacity < 0 ||
      capacity > (1ll << 30))
    return -1;
  return (int64_t)parts_of(capacity, hidden) * 3 * 32 * emc2_ffn_tiles(channels) * 32 * ((hidden + 31) / 32) * (int64_t)sizeof(float);
}

extern "C" emc2_status emc2_ffn_backward(emc2_ctx* ctx, emc2_dtype dtype, int32_t activation, const void* d_x, int64_t ld_x,
                                         const void* d_packed, const void* d_dy, int64_t ld_dy, const int32_t* d_n, int64_t capacity,
                                         int32_t channels, int32_t hidden, void* d_dx, int64_t ld_dx, void* d_dwg, void* d_dwu, void* d_dwd,
                                         void* d_work, int64_t work_bytes, void* stream) {
  if (!ctx) return EMC2_ERR_INVALID_ARG;
  const emc2_status st = emc2_ffn_check(ctx, "emc2_ffn_backward", dtype, activation, capacity, channels, hidden, d_packed);
  if (st != EMC2_OK) return st;
  const size_t size = emc2_size_of(dtype);
  const bool none = capacity == 0;
  if (!emc2_rows_ok(d_x, ld_x, channels, size, none) || !emc2_rows_ok(d_dy, ld_dy, channels, size, none) ||
      !emc2_rows_ok(d_dx, ld_dx, channels, size, none))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_ffn_backward: null or misaligned rows, or a pitch below the channels");
  if (!d_dwg || !d_dwu || !d_dwd || (uintptr_t)d_dwg % size || (uintptr_t)d_dwu % size || (uintptr_t)d_dwd % size)
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_ffn_backward: weight gradients null or misaligned");
  if (work_bytes < emc2_ffn_work(dtype, capacity, channels, hidden) || !d_work || ((uintptr_t)d_work & 15))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_ffn_backward: work buffer null, not 16-byte aligned or smaller than emc2_ffn_work");
  emc2_ffn_args a = {};
  a.x = d_x, a.dy = d_dy, a.packed = d_packed, a.y = d_dx, a.partial = (float*)d_work, a.d_n = d_n, a.ld_x = ld_x, a.ld_dy = ld_dy, a.ld_y = ld_dx;
  a.capacity = capacity, a.channels = channels, a.hidden = hidden, a.slices = (hidden + 31) / 32, a.gelu = activation == EMC2_ACT_GELU;
  a.parts = parts_of(capacity, hidden);
  a.wide = channels % (16 / size) == 0 && emc2_wide_rows(d_x, ld_x, size) && emc2_wide_rows(d_dy, ld_dy, size) && emc2_wide_rows(d_dx, ld_dx, size);
  hipStream_t s = (hipStream_t)stream;
  const int tiles = emc2_ffn_tiles(channels);
  const dim3 dw_grid((unsigned)emc2_div_up((int64_t)a.parts * a.slices, kThreads / 64));
  emc2_ffn_dispatch(dtype, tiles, [&](auto type, auto count) {
    using T = decltype(type);
    constexpr int CT = decltype(count)::value, CB = CT > 4 ? CT / 2 : CT;
    // the weights' launches first: dx may lie where dy did
    hipLaunchKernelGGL((k_ffn_dw<T, CT, 0, CB>), dw_grid, dim3(kThreads), 0, s, a);
    if constexpr (CB < CT) hipLaunchKernelGGL((k_ffn_dw<T, CT, CB, CB>), dw_grid, dim3(kThreads), 0, s, a);
    if (!none) hipLaunchKernelGGL((k_ffn_dx<T, CT>), dim3((unsigned)emc2_div_up(capacity, 128)), dim3(kThreads), 0, s, a);
    hipLaunchKernelGGL(k_ffn_sum<T>, dim3((unsigned)emc2_div_up((int64_t)a.slices * 3 * CT * 256, kThreads)), dim3(kThreads), 0, s,
                       (const float4*)d_work, a.parts, a.slices, CT, channels, hidden, (T*)d_dwg, (T*)d_dwu, (T*)d_dwd);
  });
  return emc2_check_hip(ctx, hipGetLastError(), "emc2_ffn_backward launch");
}
