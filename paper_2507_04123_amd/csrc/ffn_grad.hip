// Gradients of the gated feed-forward network (ffn.h has the mathematics of the forward pass and the fragments).
//   dH = dy Wd^T, dU = dH act(G), dG = dH U act'(G);   dx = dG Wg^T + dU Wu^T;   dWg = x^T dG, dWu = x^T dU, dWd = H^T dy
// G, U and dH are computed again in both kernels rather than stored: a slice of 32 hidden units costs 3 products per pass, and storing H, dG
// and dU would move six times n F values.  dG, dU and H are rounded to the operands' type for their products, up to kFfnRestRows rows in two parts; f16 ones lose
// places below 6e-5 all the same.
// k_ffn_dx works like the forward pass: hidden units along the lanes' registers, rows along the lanes.
// k_ffn_dw has them the other way round (rows along the registers), which is what a contraction over rows takes: dG, dU and H are its operands as
// they are.  x and dy have to be turned round for it: a product with the identity does that on the matrix cores, exactly (of finite values).  Each block sums
// its slice of 32 hidden units over a part of the rows; the parts are added by k_ffn_sum in a fixed order (fp32, no atomics).
#include "ffn.h"

namespace {

constexpr int kThreads = 256;

// Four neighbouring values of dx's row, from channel `at` on.
template <typename T, bool WIDE> __device__ __forceinline__ void put_dx(const emc2_ffn_args& a, int64_t row, int at, emc2_fvec<4> v) {
  T* out = (T*)a.y + row * a.ld_y + at;
  if (at + 4 <= a.channels) {
    emc2_store<4>(out, v);
  } else if constexpr (!WIDE) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (at + i < a.channels) out[i] = (T)v[i];
  }
}

// Many rows: every wave has 32 rows of its own and walks all slices, whose weights pass through LDS for the whole block; the next
// slice's are on their way meanwhile.  Wide rows of 16 bits take this form whatever their number; the others beyond the power of two that is nearest to where both
// take as long.
// us, the form below (whose waves split the slices) / this one at 16 k, 32 k and 64 k rows: f16 64 x 256 11 / 12, 22 / 13, 39 / 21;
// f16 128 x 512 27 / 42, 51 / 46, 99 / 54; f16 256 x 512 122 / 71, 199 / 76, 353 / 147 (2 k rows 79 / 67);
// f32 96 x 384 67 / 106, 129 / 113, 250 / 217 (at 32 k rows, the limit of these two, 5 and 16 us are lost).  At 300 k x 128 x 512 f16 256 us, 770 TFLOP/s: like the forward pass, bound by the weights' way out of LDS
// (a wave's fragment feeds one product) and the products themselves.
template <typename T, int CT> constexpr bool kDxMany = sizeof(T) * CT <= 16;              // LDS has room for two slices' weights
template <typename T, int CT> constexpr bool kDxFew = sizeof(T) == 4 || CT <= 4;
template <typename T, int CT> constexpr int64_t kDxFewRows = !kDxFew<T, CT> ? 0 : sizeof(T) * CT < 8 ? 16384 : 32768;
static_assert(kFfnRestRows <= 16384, "two parts: this form has the types that have no other one");
template <typename T, int CT> constexpr int kDxManyASimd = sizeof(T) * CT <= 8 ? 2 : 1;   // waves a SIMD that the registers are enough for
template <typename T, int CT> constexpr int kDxManyWaves = sizeof(T) * CT <= 4 || sizeof(T) * CT > 8 ? 4 : 8;   // (and the fragments under way are fewer a wave)
template <typename T, int CT, bool GELU, bool WIDE, int P>
__global__ void __launch_bounds__((64 * kDxManyWaves<T, CT>), (kDxManyASimd<T, CT>)) k_ffn_dx_many(const emc2_ffn_args a) {
  typedef emc2_tile<T> M;
  typedef typename M::frag frag;
  constexpr int W = kDxManyWaves<T, CT>, KK = 32 * CT / M::kDeep, MM = 32 / M::kDeep, kStaged = (3 * KK + W - 1) / W;
  constexpr bool kExact = sizeof(T) == 4, kShort = sizeof(T) * CT == 16;   // registers are short: weights no further ahead
  __shared__ frag ring[2][5 * KK * 64];
  const int32_t n = emc2_row_count(a.d_n, a.capacity);
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((int64_t)blockIdx.x * W * 32 >= n) return;
  const int64_t row = ((int64_t)blockIdx.x * W + wave) * 32 + (lane & 31);
  emc2_row<T, CT, WIDE> x, dy;
  x.set(a.x, a.ld_x, row, n, a.channels, half);
  dy.set(a.dy, a.ld_dy, row, n, a.channels, half);
  emc2_acc dx[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) dx[c] = 0.0f;
  const frag* packed = (const frag*)a.packed + EMC2_FFN_GATE * KK * 64 + lane;
  frag staged[kStaged];
  // fragments FROM .. TO - 1 of a slice (beyond the last one: the last one again)
  const auto place = [&](int i, int from, int to) { return min(from + wave + i * W, to - 1); };
  const auto fetch = [&](int32_t s, int from, int to) {
#pragma unroll
    for (int i = 0; i < (to - from + W - 1) / W; ++i)
      staged[i] = packed[((int64_t)min(s, a.slices - 1) * EMC2_FFN_GROUPS * KK + place(i, from, to)) * 64];
  };
  const auto keep = [&](int buf, int from, int to) {
#pragma unroll
    for (int i = 0; i < (to - from + W - 1) / W; ++i) ring[buf][place(i, from, to) * 64 + lane] = staged[i];
  };
  fetch(0, 0, 3 * KK);
  keep(0, 0, 3 * KK);
  fetch(0, 3 * KK, 5 * KK);
  keep(0, 3 * KK, 5 * KK);
  for (int32_t s = 0; s < a.slices; ++s) {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    fetch(s + 1, 0, 3 * KK);
    __builtin_amdgcn_sched_barrier(0);
    const frag* w = ring[s & 1] + lane;
    emc2_acc g = 0.0f, u = 0.0f, dh = 0.0f;
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      g = emc2_mma<T>(w[k * 64], x[k], g);
      u = emc2_mma<T>(w[(KK + k) * 64], x[k], u);
      dh = emc2_mma<T>(w[(2 * KK + k) * 64], dy[k], dh);
      if constexpr (kShort) if (k % 8 == 7) __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_sched_barrier(0);
    keep((s + 1) & 1, 0, 3 * KK);
    fetch(s + 1, 3 * KK, 5 * KK);
    frag dg[P][MM], du[P][MM];
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      float slope[2];
      const float act[2] = {emc2_activate<kExact, GELU>(g[r], slope[0]), emc2_activate<kExact, GELU>(g[r + 1], slope[1])};
      emc2_put_pair<T, P, MM>(dg, r, dh[r] * u[r] * slope[0], dh[r + 1] * u[r + 1] * slope[1]);
      emc2_put_pair<T, P, MM>(du, r, dh[r] * act[0], dh[r + 1] * act[1]);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < KK; ++k) {
#pragma unroll
      for (int p = 0; p < P; ++p) {
        dx[k / MM] = emc2_mma<T>(w[(3 * KK + k) * 64], dg[p][k % MM], dx[k / MM]);
        dx[k / MM] = emc2_mma<T>(w[(4 * KK + k) * 64], du[p][k % MM], dx[k / MM]);
      }
      if constexpr (kShort) if (k % 8 == 7) __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_sched_barrier(0);
    keep((s + 1) & 1, 3 * KK, 5 * KK);
  }
  if (row >= n) return;
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      put_dx<T, WIDE>(a, row, 32 * c + 8 * j + 4 * half, emc2_fvec<4>{dx[c][4 * j], dx[c][4 * j + 1], dx[c][4 * j + 2], dx[c][4 * j + 3]});
}

// A block has 32 rows; its waves (eight, or four where x, dy and dx's sums take over half of a SIMD's registers) share the slices out, each
// reading its own weights from memory at once, and their sums meet in LDS.
template <typename T, int CT> constexpr int kDxWaves = sizeof(T) == 4 && CT == 4 ? 4 : 8;
template <typename T, int CT, bool GELU, bool WIDE, int P>
__global__ void __launch_bounds__((64 * kDxWaves<T, CT>)) k_ffn_dx(const emc2_ffn_args a) {
  typedef emc2_tile<T> M;
  typedef typename M::frag frag;
  constexpr int KK = 32 * CT / M::kDeep, MM = 32 / M::kDeep;
  constexpr bool kExact = sizeof(T) == 4;
  constexpr int kWaves = kDxWaves<T, CT>;
  __shared__ emc2_fvec<4> part[kWaves][4][64];
  const int32_t n = emc2_row_count(a.d_n, a.capacity);
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (emc2_block() * 32 >= n) return;
  const int64_t row = emc2_block() * 32 + (lane & 31);
  emc2_row<T, CT, WIDE> x, dy;
  x.set(a.x, a.ld_x, row, n, a.channels, half);
  dy.set(a.dy, a.ld_dy, row, n, a.channels, half);
  emc2_acc dx[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) dx[c] = 0.0f;
  for (int32_t s = wave; s < a.slices; s += kWaves) {
    const frag* w = (const frag*)a.packed + (int64_t)s * EMC2_FFN_GROUPS * KK * 64 + lane;
    x.again(), dy.again();
    emc2_acc g = 0.0f, u = 0.0f, dh = 0.0f;
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      g = emc2_mma<T>(w[(EMC2_FFN_GATE * KK + k) * 64], x[k], g);
      u = emc2_mma<T>(w[(EMC2_FFN_UP * KK + k) * 64], x[k], u);
      dh = emc2_mma<T>(w[(EMC2_FFN_DOWN_T * KK + k) * 64], dy[k], dh);
    }
    frag dg[P][MM], du[P][MM];
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      float slope[2];
      const float act[2] = {emc2_activate<kExact, GELU>(g[r], slope[0]), emc2_activate<kExact, GELU>(g[r + 1], slope[1])};
      emc2_put_pair<T, P, MM>(dg, r, dh[r] * u[r] * slope[0], dh[r + 1] * u[r + 1] * slope[1]);
      emc2_put_pair<T, P, MM>(du, r, dh[r] * act[0], dh[r + 1] * act[1]);
    }
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      const frag gate = w[(EMC2_FFN_GATE_T * KK + k) * 64], up = w[(EMC2_FFN_UP_T * KK + k) * 64];
#pragma unroll
      for (int p = 0; p < P; ++p) {
        dx[k / MM] = emc2_mma<T>(gate, dg[p][k % MM], dx[k / MM]);
        dx[k / MM] = emc2_mma<T>(up, du[p][k % MM], dx[k / MM]);
      }
    }
  }
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    if (c) __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j) part[wave][j][lane] = emc2_fvec<4>{dx[c][4 * j], dx[c][4 * j + 1], dx[c][4 * j + 2], dx[c][4 * j + 3]};
    __syncthreads();
    const int at = 32 * c + 8 * wave + 4 * half;
    if (wave < 4 && row < n) {
      emc2_fvec<4> v = part[0][wave][lane];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) v += part[w][wave][lane];
      put_dx<T, WIDE>(a, row, at, v);
    }
  }
}

// Fragments of a tile's 32 columns of x or dy, rows along the lanes' registers: the rows' fragments times the identity.
template <typename T, int CT, bool WIDE, int MM>
__device__ __forceinline__ void turned(const emc2_row<T, CT, WIDE>& rows, int first, const typename emc2_tile<T>::frag (&one)[MM],
                                       typename emc2_tile<T>::frag (&out)[MM]) {
  emc2_acc t = 0.0f;
#pragma unroll
  for (int m = 0; m < MM; ++m) t = emc2_mma<T>(rows[first + m], one[m], t);
#pragma unroll
  for (int r = 0; r < 16; r += 2) emc2_put_pair<T>(out, r, t[r], t[r + 1]);
}

// Partial sums [part][slice][3][C / 32][64 lanes][16]: of a tile of dWg, dWu (rows: channels, columns: hidden units) and of dWd (rows: hidden
// units, columns: channels), the CB tiles of channels from C0 on.  A block has one slice, whose weights lie in LDS, and one part of the rows, which
// its four waves share out.  16-bit values: 100 k x 64 x 256 in 40 us, 300 k x 128 x 512 in 510: 490 and 460 TFLOP/s without
// the turning.  For every 32 products at 64 channels there are 200 plain and 32 slow vector instructions of activation, slopes and roundings.  Measured and
// not better: the next tile's rows on their way during the activation (within 4 %, or no registers for it), the turning spread over the
// activation (up to 9 % slower), a part's slices on one XCD (up to 10 % slower).
// Waves a SIMD: two where the sums are few.
template <typename T, int CT> constexpr int kDwWaves = sizeof(T) * CT <= 4 ? 2 : 1;   // (parts_of counts on it)
template <typename T, int CT, bool GELU, bool WIDE, int C0, int CB, int P>
__global__ void __launch_bounds__(kThreads, (kDwWaves<T, CT>)) k_ffn_dw(const emc2_ffn_args a) {
  typedef emc2_tile<T> M;
  typedef typename M::frag frag;
  constexpr int KK = 32 * CT / M::kDeep, MM = 32 / M::kDeep, kWaves = kThreads / 64;
  constexpr int kWavesASimd = kDwWaves<T, CT>;
  constexpr bool kExact = sizeof(T) == 4;
  __shared__ frag w[3 * KK * 64];
  __shared__ emc2_fvec<4> meet[kWaves][4][64];
  const int32_t n = emc2_row_count(a.d_n, a.capacity);
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t s = blockIdx.x % a.slices, part = blockIdx.x / a.slices;
  {
    const frag* from = (const frag*)a.packed + ((int64_t)s * EMC2_FFN_GROUPS + EMC2_FFN_GATE) * KK * 64;
    for (int i = threadIdx.x; i < 3 * KK * 64; i += kThreads) w[i] = from[i];
  }
  __syncthreads();
  frag one[MM];
#pragma unroll
  for (int m = 0; m < MM; ++m)
#pragma unroll
    for (int e = 0; e < M::kPer; ++e) one[m][e] = (T)(m * M::kDeep + half * M::kPer + e == (lane & 31) ? 1.0f : 0.0f);
  emc2_acc dwg[CB], dwu[CB], dwd[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) dwg[c] = 0.0f, dwu[c] = 0.0f, dwd[c] = 0.0f;
  const int32_t step = a.parts * kWaves;
  for (int64_t tile = (int64_t)part * kWaves + wave; tile * 32 < n; tile += step) {
    const int64_t row = tile * 32 + (lane & 31);
    emc2_row<T, CT, WIDE> x, dy;
    x.set(a.x, a.ld_x, row, n, a.channels, half);
    dy.set(a.dy, a.ld_dy, row, n, a.channels, half);
    int at = lane;
    asm volatile("" : "+v"(at));                           // the weights are read from LDS each time: registers have no room for them
    emc2_acc g = 0.0f, u = 0.0f, dh = 0.0f;
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      g = emc2_mma<T>(x[k], w[k * 64 + at], g);
      u = emc2_mma<T>(x[k], w[(KK + k) * 64 + at], u);
      dh = emc2_mma<T>(dy[k], w[(2 * KK + k) * 64 + at], dh);
    }
    frag h[P][MM], dg[P][MM], du[P][MM];
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      float slope[2];
      const float act[2] = {emc2_activate<kExact, GELU>(g[r], slope[0]), emc2_activate<kExact, GELU>(g[r + 1], slope[1])};
      emc2_put_pair<T, P, MM>(h, r, act[0] * u[r], act[1] * u[r + 1]);
      emc2_put_pair<T, P, MM>(dg, r, dh[r] * u[r] * slope[0], dh[r + 1] * u[r + 1] * slope[1]);
      emc2_put_pair<T, P, MM>(du, r, dh[r] * act[0], dh[r + 1] * act[1]);
    }
    // tile 2 c of x and 2 c + 1 of dy, each turned one step ahead of its products
    frag t[2][MM];
    turned<T, CT, WIDE, MM>(x, C0 * MM, one, t[0]);
#pragma unroll
    for (int i = 0; i < 2 * CB; ++i) {
      const int c = i / 2;
      if (i + 1 < 2 * CB) {
        if (i % 2) turned<T, CT, WIDE, MM>(x, (C0 + c + 1) * MM, one, t[(i + 1) % 2]);
        else turned<T, CT, WIDE, MM>(dy, (C0 + c) * MM, one, t[(i + 1) % 2]);
      }
#pragma unroll
      for (int m = 0; m < MM; ++m) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
          if (i % 2) dwd[c] = emc2_mma<T>(h[p][m], t[1][m], dwd[c]);
          else dwg[c] = emc2_mma<T>(t[0][m], dg[p][m], dwg[c]), dwu[c] = emc2_mma<T>(t[0][m], du[p][m], dwu[c]);
        }
      }
      if constexpr (kWavesASimd == 1) __builtin_amdgcn_sched_barrier(0);   // no further ahead: registers
    }
  }
  emc2_fvec<4>* out = (emc2_fvec<4>*)a.partial + ((int64_t)part * a.slices + s) * 3 * CT * 256;
  const auto put = [&](int which, const emc2_acc (&sums)[CB]) {
#pragma unroll
    for (int c = 0; c < CB; ++c) {
      const emc2_acc& t = sums[c];
      if (which + c) __syncthreads();
#pragma unroll
      for (int j = 0; j < 4; ++j) meet[wave][j][lane] = emc2_fvec<4>{t[4 * j], t[4 * j + 1], t[4 * j + 2], t[4 * j + 3]};
      __syncthreads();
      // registers 4 wave .. 4 wave + 3 of every lane
      out[((which * CT + C0 + c) * 64 + lane) * 4 + wave] = meet[0][wave][lane] + meet[1][wave][lane] + meet[2][wave][lane] + meet[3][wave][lane];
    }
  };
  put(0, dwg);
  put(1, dwu);
  // A value of dy that is not finite makes its turned row NaN, 0 times it being that, in all columns of the tile: then the wave sums dWd once more,
  // with dy's values read one by one where they belong.  (One of x leaves no gradient of its row finite in any column.)  Here, where the
  // other sums' registers are free, it costs the loop above none.
  bool nan = false;
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int r = 0; r < 16; ++r) nan |= dwd[c][r] != dwd[c][r];
  if (__any(nan)) {
#pragma unroll
    for (int c = 0; c < CB; ++c) dwd[c] = 0.0f;
    for (int64_t tile = (int64_t)part * kWaves + wave; tile * 32 < n; tile += step) {
      // channels and rows that are not there take the last one's values: they meet weights and hidden values of 0, or are not kept
      const int64_t row = tile * 32 + (lane & 31), most = n - 1;
      const T* x = (const T*)a.x + min(row, most) * a.ld_x;
      int at = lane, channel = half * M::kPer;
      asm volatile("" : "+v"(at), "+v"(channel));
      emc2_acc g = 0.0f, u = 0.0f;
#pragma unroll
      for (int k = 0; k < KK; ++k) {
        frag v;
#pragma unroll
        for (int e = 0; e < M::kPer; ++e) v[e] = x[min(channel + k * M::kDeep + e, a.channels - 1)];
        if (row > most) v = emc2_zero_frag<T>();
        g = emc2_mma<T>(v, w[k * 64 + at], g);
        u = emc2_mma<T>(v, w[(KK + k) * 64 + at], u);
        __builtin_amdgcn_sched_barrier(0);
      }
      frag h[P][MM];
#pragma unroll
      for (int r = 0; r < 16; r += 2)
        emc2_put_pair<T, P, MM>(h, r, emc2_activate<kExact, GELU>(g[r]) * u[r], emc2_activate<kExact, GELU>(g[r + 1]) * u[r + 1]);
#pragma unroll
      for (int c = 0; c < CB; ++c) {
        const T* dy = (const T*)a.dy + min(32 * (C0 + c) + (at & 31), a.channels - 1);
#pragma unroll
        for (int m = 0; m < MM; ++m) {
          frag t;
#pragma unroll
          for (int e = 0; e < M::kPer; ++e) t[e] = dy[min(tile * 32 + emc2_hidden_of<T>(m, half, e), most) * a.ld_dy];
#pragma unroll
          for (int p = 0; p < P; ++p) dwd[c] = emc2_mma<T>(h[p][m], t, dwd[c]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }
  put(2, dwd);
}

// Adds the parts, four values a thread, and puts them where they belong.  Eight threads share a sum's parts out (500 parts of 32 x 128 values:
// 9.0 us by one thread, 5.3 by eight; 61 parts of 64 x 256 values with their loads in a row 5.5, together 5.0) and meet in LDS, always in the same order.
constexpr int kSumThreads = 8;
template <typename T>
__global__ void __launch_bounds__(kThreads) k_ffn_sum(const float4* __restrict__ partial, int32_t parts, int32_t slices, int32_t tiles,
                                                      int32_t channels, int32_t hidden, T* __restrict__ dwg, T* __restrict__ dwu,
                                                      T* __restrict__ dwd) {
  constexpr int kSums = kThreads / kSumThreads;
  __shared__ float4 meet[kSumThreads][kSums];
  const int64_t quads = (int64_t)slices * 3 * tiles * 64 * 4, at = (int64_t)blockIdx.x * kSums + threadIdx.x % kSums;
  const int mine = threadIdx.x / kSums;
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);              // (768 sums a tile and slice: no block has fewer than kSums)
  for (int32_t p = mine; p < parts; p += kSumThreads * 8) {    // eight loads under way, beyond the last part of the last one again
    float4 q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = partial[min(p + kSumThreads * i, parts - 1) * quads + at];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (p + kSumThreads * i < parts) s.x += q[i].x, s.y += q[i].y, s.z += q[i].z, s.w += q[i].w;
  }
  meet[mine][threadIdx.x % kSums] = s;
  __syncthreads();
  if (mine) return;
#pragma unroll
  for (int i = 1; i < kSumThreads; ++i) {
    const float4 q = meet[i][threadIdx.x];
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

// Parts that the rows are cut into.  The chip holds kDwWaves blocks a CU; a launch takes as many rounds of them as it needs, each as long as a
// wave's tiles of rows and about one tile's time for the weights and the sums.  The best of one to three rounds, then the fewest parts with as many
// tiles a wave.  us, k_ffn_dw with four blocks more than two rounds / this: 32000 x 96 x 384 f32 250 / 173, f16 58 / 38.
constexpr int64_t kMostRounds = 3;
int64_t room_of(emc2_dtype dtype, int32_t channels) { return 256 * (emc2_size_of(dtype) * emc2_ffn_tiles(channels) <= 4 ? 2 : 1); }
int32_t parts_of(emc2_dtype dtype, int64_t capacity, int32_t channels, int32_t hidden) {
  const int64_t slices = (hidden + 31) / 32, tiles = emc2_div_up(capacity, 32), waves = kThreads / 64, room = room_of(dtype, channels);
  int64_t best = 1, cost = INT64_MAX;
  for (int64_t rounds = 1; rounds <= kMostRounds; ++rounds) {
    const int64_t most = room * rounds / slices, turns = emc2_div_up(tiles, waves * (most ? most : 1));
    const int64_t parts = turns ? emc2_div_up(tiles, waves * turns) : 1, c = emc2_div_up(parts * slices, room) * (turns + 1);
    if (c < cost) best = parts, cost = c;
  }
  return (int32_t)best;
}
// As many parts as a call of up to that many rows may have: more rows may well have fewer parts, and a buffer for them has to serve both.
int64_t most_parts(emc2_dtype dtype, int64_t capacity, int32_t channels, int32_t hidden) {
  const int64_t room = kMostRounds * room_of(dtype, channels) / ((hidden + 31) / 32), blocks = emc2_div_up(emc2_div_up(capacity, 32), kThreads / 64);
  const int64_t parts = room < blocks ? room : blocks;
  return parts < 1 ? 1 : parts;
}

}  // namespace

extern "C" int64_t emc2_ffn_work(emc2_dtype dtype, int64_t capacity, int32_t channels, int32_t hidden) {
  if (!emc2_is_float(dtype) || channels < 1 || channels > kFfnMaxChannels || hidden < 1 || hidden > kFfnMaxHidden || capacity < 0 ||
      capacity > (1ll << 30))
    return -1;
  return most_parts(dtype, capacity, channels, hidden) * 3 * 32 * emc2_ffn_tiles(channels) * 32 * ((hidden + 31) / 32) * (int64_t)sizeof(float);
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
  a.capacity = capacity, a.channels = channels, a.hidden = hidden, a.slices = (hidden + 31) / 32;
  a.parts = parts_of(dtype, capacity, channels, hidden);
  const bool wide = channels % (16 / size) == 0;
  hipStream_t s = (hipStream_t)stream;
  const int tiles = emc2_ffn_tiles(channels);
  const dim3 dw_grid((unsigned)((int64_t)a.parts * a.slices));
  emc2_ffn_dispatch(dtype, tiles, activation == EMC2_ACT_GELU, wide, [&](auto type, auto count, auto gelu, auto pieces) {
    using T = decltype(type);
    constexpr bool G = decltype(gelu)::value;
    constexpr int CT = decltype(count)::value, CB = CT > 4 ? CT / 2 : CT;   // (the sums of more tiles of channels leave no registers)
    const auto launch = [&](auto whole, auto parts) {
      constexpr bool W = decltype(whole)::value;
      constexpr int P = decltype(parts)::value;
      // the weights' launches first: dx may lie where dy did
      hipLaunchKernelGGL((k_ffn_dw<T, CT, G, W, 0, CB, P>), dw_grid, dim3(kThreads), 0, s, a);
      if constexpr (CB < CT) hipLaunchKernelGGL((k_ffn_dw<T, CT, G, W, CB, CT - CB, P>), dw_grid, dim3(kThreads), 0, s, a);
      // (two parts are for fewer rows than need a choice of forms)
      constexpr bool kMany = kDxMany<T, CT> && (P == 1 || !kDxFew<T, CT>);
      if constexpr (kMany) {
        constexpr int kWaves = kDxManyWaves<T, CT>;
        if (capacity > kDxFewRows<T, CT>)
          hipLaunchKernelGGL((k_ffn_dx_many<T, CT, G, W, P>), dim3((unsigned)emc2_div_up(capacity, 32 * kWaves)), dim3(64 * kWaves), 0, s, a);
      }
      if constexpr (kDxFew<T, CT>) {
        if (!none && !(kMany && capacity > kDxFewRows<T, CT>))
          hipLaunchKernelGGL((k_ffn_dx<T, CT, G, W, P>), emc2_grid(emc2_div_up(capacity, 32)), dim3(64 * kDxWaves<T, CT>), 0, s, a);
      }
    };
    if constexpr (sizeof(T) == 2) {
      if (capacity <= kFfnRestRows) launch(emc2_const<0>(), emc2_const<2>());   // (one form for whole pieces and others)
      else launch(pieces, emc2_const<1>());
    } else {
      launch(pieces, emc2_const<1>());
    }
    hipLaunchKernelGGL(k_ffn_sum<T>, dim3((unsigned)((int64_t)a.slices * 3 * CT * 256 / (kThreads / kSumThreads))), dim3(kThreads), 0, s,
                       (const float4*)d_work, a.parts, a.slices, CT, channels, hidden, (T*)d_dwg, (T*)d_dwu, (T*)d_dwd);
  });
  return emc2_check_hip(ctx, hipGetLastError(), "emc2_ffn_backward launch");
}
