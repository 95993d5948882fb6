// Gated feed-forward network, forward pass and the order of its weights (ffn.h has the mathematics and the fragments).
// A wave keeps its 32 rows of x and of y's sums in registers and walks the hidden units in slices of 32: two products for G and U, the
// activation, H rounded to the operands' type (the matrix cores multiply 16-bit values; up to kFfnRestRows rows in two parts), and the product with the
// slice's lines of Wd.  What is beyond f16's range (65504) is not finite.
#include "ffn.h"

namespace {

constexpr int kThreads = 256;
// Up to here a block has 32 rows and its waves share the slices out (k_ffn_few), beyond it a wave has 32 rows of its own (k_ffn).
// us, few / many at 8 k, 16 k, 24 k and 64 k rows: f16 64 x 256 5.3 / 9.6, 7.4 / 9.9, 10.4 / 10.2, 22 / 15; f16 128 x 512 11 / 18, 18 / 19, 26 / 19,
// 65 / 36; f16 256 x 512 20 / 40, 38 / 42, 55 / 44, 143 / 90; f32 48 x 200 12 / 30, 20 / 31, 29 / 32, 69 / 60.
constexpr int64_t kFewRows = 16384;
static_assert(kFfnRestRows <= kFewRows, "two parts: in the form for few rows only");

// Four neighbouring values of a result's row, from channel `at` on.
template <typename T, bool WIDE> __device__ __forceinline__ void put(const emc2_ffn_args& a, int64_t row, int at, emc2_fvec<4> v) {
  T* out = (T*)a.y + row * a.ld_y + at;
  const T* res = (const T*)a.res + row * a.ld_res + at;
  if (at + 4 <= a.channels) {
    if (a.res) v += emc2_load<4>(res);
    emc2_store<4>(out, v);
  } else if constexpr (!WIDE) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (at + i < a.channels) out[i] = (T)(v[i] + (a.res ? (float)res[i] : 0.0f));
  }
}

// H's registers r and r + 1, as operands
template <typename T, bool GELU, int P, int MM>
__device__ __forceinline__ void hidden(const emc2_acc& g, const emc2_acc& u, int r, typename emc2_tile<T>::frag (&h)[P][MM]) {
  constexpr bool kExact = sizeof(T) == 4;
  emc2_put_pair<T, P, MM>(h, r, emc2_activate<kExact, GELU>(g[r]) * u[r], emc2_activate<kExact, GELU>(g[r + 1]) * u[r + 1]);
}

template <bool GATES, bool ACT, bool DOWN> struct Stages { static constexpr bool gates = GATES, act = ACT, down = DOWN; };
template <int V> struct Now { static constexpr int value = V; };

// Waves a SIMD of the kernel below: two where 256 registers hold x, y's sums, and G and U twice
template <typename T, int CT> constexpr int kFfnWaves = sizeof(T) * CT <= 8 ? 2 : 1;

// Many rows: a block of four waves has 128 rows and passes the weights, slice by slice, through LDS, where all waves read them.  Turn t multiplies
// slice t's gates, activates slice t - 1 and multiplies slice t - 2's way down: three independent strands, so that the vector ALU's
// activation (an exponential and a reciprocal an element) runs under the matrix cores' products.  The loads of turn t + 1's
// weights are under way meanwhile.  300 k x 128 x 512 f16 160 to 166 us, 720 TFLOP/s: a fragment from LDS (128 bytes a clock) feeds one product of a wave,
// which takes about as long as its reading, and 2344 blocks, two a CU at once, leave the fifth round half empty.  Measured and not better: 64 rows
// a wave (fragments feed two products, one wave a SIMD) 211, eight waves a block with the weights two turns ahead 180, Wd's lines past LDS 244.
constexpr int kManyWaves = 4;
template <typename T, int CT, bool GELU, bool WIDE>
__global__ void __launch_bounds__(64 * kManyWaves, (kFfnWaves<T, CT>)) k_ffn(const emc2_ffn_args a) {
  typedef emc2_tile<T> M;
  typedef typename M::frag frag;
  constexpr int W = kManyWaves, KK = 32 * CT / M::kDeep, MM = 32 / M::kDeep;
  __shared__ frag ring[2][3 * KK * 64];    // lines down, then gates (two products' fragments)
  const int32_t n = emc2_row_count(a.d_n, a.capacity);
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((int64_t)blockIdx.x * W * 32 >= n) return;
  const int64_t row = ((int64_t)blockIdx.x * W + wave) * 32 + (lane & 31);
  emc2_row<T, CT, WIDE> x;
  x.set(a.x, a.ld_x, row, n, a.channels, half);
  emc2_acc y[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) y[c] = 0.0f;
  emc2_acc g[2], u[2];                   // of the slice whose gates were multiplied last, and of this turn's
  frag h[2][1][MM];                      // likewise
  const frag* packed = (const frag*)a.packed + lane;
  // A turn's weights, fragment by fragment over the waves: gates of slice t + 1 and lines down of slice t - 1, by way of registers (loads
  // straight into LDS are waited for, all of them, before the next read of LDS).
  constexpr int kStaged = (3 * KK + W - 1) / W;
  frag staged[kStaged];
  const auto fetch = [&](int32_t t) {
#pragma unroll
    for (int i = 0; i < kStaged; ++i) {                    // (beyond the last fragment or slice: the last one again, which hurts nobody)
      const int f = min(wave + i * W, 3 * KK - 1), ahead = min(f / KK, 1);
      const int32_t slice = max(0, min(t - 1 + 2 * ahead, a.slices - 1));
      staged[i] = packed[((int64_t)slice * EMC2_FFN_GROUPS * KK + f) * 64];
    }
  };
  const auto keep = [&](int buf) {
#pragma unroll
    for (int i = 0; i < kStaged; ++i) ring[buf][min(wave + i * W, 3 * KK - 1) * 64 + lane] = staged[i];
  };
  const auto all_here = [] { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
  // one turn: of slices t, t - 1 and t - 2 (parity NOW = t % 2), whichever there are
  const auto turn = [&](auto stages, auto parity, int32_t t) {
    constexpr bool kGates = decltype(stages)::gates, kAct = decltype(stages)::act, kDown = decltype(stages)::down;
    constexpr int now = decltype(parity)::value;
    all_here();
    fetch(t);
    __builtin_amdgcn_sched_barrier(0);
    const frag* w = ring[now] + lane;
    x.again();
    if constexpr (kGates) g[now] = 0.0f, u[now] = 0.0f;
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      if constexpr (kGates) {
        g[now] = emc2_mma<T>(w[(KK + k) * 64], x[k], g[now]);
        u[now] = emc2_mma<T>(w[(2 * KK + k) * 64], x[k], u[now]);
      }
      if constexpr (kDown) y[k / MM] = emc2_mma<T>(w[k * 64], h[now][0][k % MM], y[k / MM]);
      if constexpr (kAct) {
#pragma unroll
        for (int r = 8 * k / KK; r < 8 * (k + 1) / KK; ++r) hidden<T, GELU, 1, MM>(g[now ^ 1], u[now ^ 1], 2 * r, h[now ^ 1]);
      }
    }
    if constexpr (kGates && kAct && kDown && sizeof(T) == 2) {
      // the order that the scheduler is to find: the next fragments ahead (two k's, one where registers are short), and after every product
      // its share of the activation
      __builtin_amdgcn_sched_group_barrier(0x100, CT == 6 ? 3 : 6, 0);
#pragma unroll
      for (int i = 0; i < 3 * KK; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x400, (32 + 3 * KK - 1) / (3 * KK), 0);
        __builtin_amdgcn_sched_group_barrier(0x002, (72 + 3 * KK - 1) / (3 * KK), 0);
        if (i % 3 == 2) __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    keep(now ^ 1);
  };
  fetch(-1);
  keep(0);
  turn(Stages<true, false, false>(), Now<0>(), 0);         // slices come in pairs, the second one of zeros where F ends in the first
  turn(Stages<true, true, false>(), Now<1>(), 1);
  for (int32_t t = 2; t < a.slices; t += 2) {
    turn(Stages<true, true, true>(), Now<0>(), t);
    turn(Stages<true, true, true>(), Now<1>(), t + 1);
  }
  turn(Stages<false, true, true>(), Now<0>(), a.slices);
  turn(Stages<false, false, true>(), Now<1>(), a.slices + 1);
  if (row >= n) return;
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      put<T, WIDE>(a, row, 32 * c + 8 * j + 4 * half, emc2_fvec<4>{y[c][4 * j], y[c][4 * j + 1], y[c][4 * j + 2], y[c][4 * j + 3]});
}

// Few rows: a block has 32 of them, its waves share the slices out, each reading its own from memory at once, and their sums meet in LDS.
template <int CT, bool WIDE> constexpr int kFewWaves = CT == 8 && !WIDE ? 4 : 8;   // (four: rows value by value take more registers)
template <typename T, int CT, bool GELU, bool WIDE, int P>
__global__ void __launch_bounds__((64 * kFewWaves<CT, WIDE>)) k_ffn_few(const emc2_ffn_args a) {
  typedef emc2_tile<T> M;
  typedef typename M::frag frag;
  constexpr int KK = 32 * CT / M::kDeep, MM = 32 / M::kDeep;
  constexpr int kWaves = kFewWaves<CT, WIDE>;
  constexpr bool kAhead = P == 2 && CT <= 4;               // the lines down are requested before the activation, where registers allow it
  __shared__ emc2_fvec<4> part[kWaves][4][64];
  const int32_t n = emc2_row_count(a.d_n, a.capacity);
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (emc2_block() * 32 >= n) return;
  const int64_t row = emc2_block() * 32 + (lane & 31);
  emc2_row<T, CT, WIDE> x;
  x.set(a.x, a.ld_x, row, n, a.channels, half);
  emc2_acc y[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) y[c] = 0.0f;
  for (int32_t s = wave; s < a.slices; s += kWaves) {
    const frag* w = (const frag*)a.packed + (int64_t)s * EMC2_FFN_GROUPS * KK * 64 + lane;
    x.again();
    emc2_acc g = 0.0f, u = 0.0f;
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      g = emc2_mma<T>(w[(EMC2_FFN_GATE * KK + k) * 64], x[k], g);
      u = emc2_mma<T>(w[(EMC2_FFN_UP * KK + k) * 64], x[k], u);
    }
    frag h[P][MM], down[kAhead ? KK : 1];
    if constexpr (kAhead) {
#pragma unroll
      for (int k = 0; k < KK; ++k) down[k] = w[(EMC2_FFN_DOWN * KK + k) * 64];
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int r = 0; r < 16; r += 2) hidden<T, GELU, P, MM>(g, u, r, h);
    if constexpr (CT == 8) __builtin_amdgcn_sched_barrier(0);   // no loads further ahead: registers
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      if constexpr (!kAhead) down[0] = w[(EMC2_FFN_DOWN * KK + k) * 64];
#pragma unroll
      for (int p = 0; p < P; ++p) y[k / MM] = emc2_mma<T>(down[kAhead ? k : 0], h[p][k % MM], y[k / MM]);
    }
  }
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    if (c) __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j) part[wave][j][lane] = emc2_fvec<4>{y[c][4 * j], y[c][4 * j + 1], y[c][4 * j + 2], y[c][4 * j + 3]};
    __syncthreads();
    if (wave < 4 && row < n) {
      emc2_fvec<4> v = part[0][wave][lane];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) v += part[w][wave][lane];
      put<T, WIDE>(a, row, 32 * c + 8 * wave + 4 * half, v);
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
  return (int64_t)EMC2_FFN_GROUPS * 32 * emc2_ffn_tiles(channels) * 32 * emc2_ffn_slices(hidden);
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
  a.capacity = capacity, a.channels = channels, a.hidden = hidden, a.slices = emc2_ffn_slices(hidden);
  const bool wide = channels % (16 / size) == 0;
  emc2_ffn_dispatch(dtype, emc2_ffn_tiles(channels), activation == EMC2_ACT_GELU, wide, [&](auto type, auto tiles, auto gelu, auto pieces) {
    using T = decltype(type);
    constexpr int CT = decltype(tiles)::value;
    constexpr bool G = decltype(gelu)::value, W = decltype(pieces)::value;
    const auto few = [&](auto parts) {
      hipLaunchKernelGGL((k_ffn_few<T, CT, G, W, decltype(parts)::value>), emc2_grid(emc2_div_up(capacity, 32)), dim3(64 * kFewWaves<CT, W>), 0,
                         (hipStream_t)stream, a);
    };
    if constexpr (sizeof(T) == 2)
      if (capacity <= kFfnRestRows) return few(emc2_const<2>());
    // fp32 rows of over 64 channels would leave a SIMD one wave of k_ffn.  us, few / many, 96 x 384 at 16 k, 32 k and 64 k rows: 42 / 67, 79 / 72, 155 / 142: the
    // form for few rows takes them all, and a tenth longer than it might from 32 k rows on
    constexpr bool kFew = sizeof(T) * CT > 8 && sizeof(T) == 4;
    if (kFew || capacity <= kFewRows) few(emc2_const<1>());
    else if constexpr (!kFew)
      hipLaunchKernelGGL((k_ffn<T, CT, G, W>), dim3((unsigned)emc2_div_up(capacity, 32 * kManyWaves)), dim3(64 * kManyWaves), 0, (hipStream_t)stream, a);
  });
  return emc2_check_hip(ctx, hipGetLastError(), "emc2_ffn launch");
}
