// Selective state space scan along the rows of packed sequences, and its form for one row per sequence.
//   D_t = softplus(dt_t + dt_bias);  h_t[c][n] = exp(D_t[c] A[c][n]) h_{t-1}[c][n] + D_t[c] x_t[c] B_t[n];  y_t[c] = sum over n of C_t[n] h_t[c][n] + skip[c] x_t[c]
// Rows map a state h to exp(A D) h + add, and runs of rows to exp(A (sum of D)) h + total: of a run, one sum a channel and one total a state are kept.
// A long list of rows is cut into chunks that are worked on side by side: a first launch walks every chunk from a state of zeros (k_scan_totals), a second
// composes the totals of spans of eight chunks (k_scan_enter), the third walks every chunk from the state that enters it (k_scan).  Short calls do all of it in
// one block a slice of the channels (k_scan_short).  A sequence's first row takes the given state whatever lies before it, so sequences of any length share
// a chunk, and nothing from one reaches another.
// A lane holds S states of a channel and walks rows one after the other; x and dt of the next rows are on their way in registers, B and C, which all channels
// share, pass through LDS as floats.  The order of composition is fixed: equal inputs give equal bits.  States are fp32.
// The issue of vector instructions bounds both walks of long lists: 613,217 rows of 64 channels by 16 states in f16 take the totals 137 us, k_scan 167 us, with
// the vector units busy 85 and 88 % of the time; a row's 64 x 16 states take 108 and 131 issue slots, 80 and 96 of them for the recurrence (an exponential is two).  Rows
// without sequence ends go in straight-line code without masks (an infinite gain excepted where lanes have states that are none); against one code for all rows 299 -> 273 us
// for the call.  The sums over states on the small matrix instructions: 172 -> 211 us.  B and C read from LDS ahead of the exponentials: no change.
#include "selective_walk.h"

namespace {

// Third launch: the rows.  Blocks as in the first; those behind them deal with sequences without rows.
template <typename T, int S, int P> __global__ void __launch_bounds__(64 * kChunkWaves, 4) k_scan(const ScanArgs a) {
  __shared__ float lds[kChunkWaves * 2 * kBatch * S * P];
  const Walk w(a.offsets, a.n_seq, a.capacity, a.backwards);
  if ((int32_t)blockIdx.x >= a.row_blocks) return hand_on(a, w, a.h0, a.last);
  const States<S, P> t(a, blockIdx.y);
  const int64_t k = (int64_t)blockIdx.x * kChunkWaves + t.wave, row0 = k * a.chunk;
  if (row0 >= w.n) return;
  float a2[S], h[S], flow[S], sum;
  bool begun, ended;
  decays(a, t, a2);
  entering<0, S>(a, t, a2, (int32_t)k, spans_of(a, w.n), h);
  walk<kRun, T, S, P>(a, w, t, a2, (int32_t)row0, row0 + a.chunk < w.n ? (int32_t)row0 + a.chunk : w.n, lds + t.wave * 2 * kBatch * S * P, h, sum, begun, flow,
                      ended);
}

// Short calls: one block a slice of the channels does all three, with four states a lane.
constexpr int kShortWaves = 16;
constexpr int short_waves(int p) { return p < 16 ? kShortWaves : kShortWaves / 2; }   // 64 KiB of LDS at most
template <typename T, int P> __global__ void __launch_bounds__(64 * kShortWaves) k_scan_short(const ScanArgs a) {
  constexpr int S = 4, kOwn = 2 * kBatch * S * P;
  extern __shared__ float lds[];                           // [waves][kOwn], then totals [waves][S][64], then sums [waves][64]
  const Walk w(a.offsets, a.n_seq, a.capacity, a.backwards);
  report_rows(a.offsets, a.n_seq, a.capacity, a.flags);
  if ((int32_t)blockIdx.x >= a.row_blocks) return hand_on(a, w, a.h0, a.last);
  const States<S, P> t(a, blockIdx.y);
  const int waves = blockDim.x >> 6;
  float* const totals = lds + waves * kOwn;
  float* const sums = totals + waves * S * 64;
  const int64_t row0 = (int64_t)t.wave * a.chunk;
  const int32_t end = row0 + a.chunk < w.n ? (int32_t)row0 + a.chunk : w.n;
  float a2[S], h[S], flow[S], sum = 0.0f;
  bool begun = false, ended = false;
  decays(a, t, a2);
#pragma unroll
  for (int s = 0; s < S; ++s) h[s] = 0.0f;
  if (waves > 1) {
    if (row0 < w.n && t.wave < waves - 1) walk<kTotals, T, S, P>(a, w, t, a2, (int32_t)row0, end, lds + t.wave * kOwn, h, sum, begun, flow, ended);
#pragma unroll
    for (int s = 0; s < S; ++s) totals[(t.wave * S + s) * 64 + t.lane] = h[s];
    sums[t.wave * 64 + t.lane] = begun ? -1.0f : sum;
    __syncthreads();
#pragma unroll
    for (int s = 0; s < S; ++s) h[s] = 0.0f;
    for (int m = 0; m < t.wave; ++m) {
      float v[S];
#pragma unroll
      for (int s = 0; s < S; ++s) v[s] = totals[(m * S + s) * 64 + t.lane];
      through<S>(a2, sums[m * 64 + t.lane], v, h);
    }
  }
  if (row0 < w.n) walk<kRun, T, S, P>(a, w, t, a2, (int32_t)row0, end, lds + t.wave * kOwn, h, sum, begun, flow, ended);
}

// One row per sequence: a lane has four states.
constexpr int kStepThreads = 256;
template <typename T, int P>
__global__ void __launch_bounds__(kStepThreads) k_scan_step(const ScanArgs a, const float* h_in, float* h_out, int64_t rows) {
  constexpr int S = 4;
  const int64_t i = emc2_block() * kStepThreads + threadIdx.x, at = i / P, all = rows * a.channels;
  const bool in = at < all;
  const int64_t line = in ? at : all - 1, row = line / a.channels;   // lanes beyond the last take part in sums and write nothing
  const int32_t c = (int32_t)(line - row * a.channels), first = (int32_t)(i % P) * S, left = a.states - first, there = left < 0 ? 0 : left < S ? left : S;
  float d, slope;
  const float x = (float)((const T*)a.x + row * a.ld_x)[c];
  step_of<sizeof(T) == 4>((float)((const T*)a.dt + row * a.ld_dt)[c] + (a.dt_bias ? a.dt_bias[c] : 0.0f), d, slope);
  const float* const p = h_in + line * a.states + first;
  const float* const decay = a.a + (int64_t)c * a.states + first;
  const T* const b = (const T*)a.b + row * a.ld_b + first;
  const T* const cc = (const T*)a.c + row * a.ld_c + first;
  float h[S], y = 0.0f;
  if (there == S) {
    const emc2_fvec<4> before = emc2_load<4>(p), rate = emc2_load<4>(decay), bv = emc2_load<4>(b), cv = emc2_load<4>(cc);
#pragma unroll
    for (int s = 0; s < S; ++s) {
      h[s] = __builtin_fmaf(__builtin_amdgcn_exp2f(d * (rate[s] * kLog2e)), before[s], d * x * bv[s]);
      y = __builtin_fmaf(cv[s], h[s], y);
    }
  } else {
#pragma unroll
    for (int s = 0; s < S; ++s)
      if (s < there) {
        h[s] = __builtin_fmaf(__builtin_amdgcn_exp2f(d * (decay[s] * kLog2e)), p[s], d * x * (float)b[s]);
        y = __builtin_fmaf((float)cc[s], h[s], y);
      }
  }
  y = lane_sum<P>(y);
  if (!in) return;
  float* const to = h_out + line * a.states + first;
  if (there == S) {
    emc2_store<4>(to, emc2_fvec<4>{h[0], h[1], h[2], h[3]});
  } else {
#pragma unroll
    for (int s = 0; s < S; ++s)
      if (s < there) to[s] = h[s];
  }
  if (first == 0) ((T*)a.y + row * a.ld_y)[c] = (T)(a.skip ? y + a.skip[c] * x : y);
}

// Short calls have four states a lane (short chains).
template <typename F> void with_short_form(int32_t states, F&& f) {
  if (states <= 4) return f(Form<4, 1>());
  if (states <= 8) return f(Form<4, 2>());
  if (states <= 16) return f(Form<4, 4>());
  if (states <= 32) return f(Form<4, 8>());
  f(Form<4, 16>());
}

// Rows up to which one block a slice deals with all.  us of the GPU in one launch and in three (of a call alone from Python, which issues one in 10 and three in 15),
// bf16: 128 channels by 16 states, 256 rows 15.5 and 16.7 (34 and 36), 288 rows 17.0 and 16.3, 320 rows 19.2 and 16.8 (38 and 36), 512 rows 24 and 17 (43 and 36); 64 by 64,
// 320 rows 20 and 24 (38 and 44), 448 rows 26 and 24; 2048 by 16, 320 rows 20 and 39, 512 rows 26 and 44.  So up to 16 states the two meet at about 280 rows (alone:
// 310), with more states or thousands of channels later; the constant lies between.
constexpr int64_t kShortRows = 320;
int64_t hand_on_blocks(int32_t n_seq, int32_t slices, bool any) {
  const int64_t b = any ? emc2_div_up(n_seq, 16ll * slices) : 0;
  return b < 1024 ? b : 1024;
}

}  // namespace

emc2_status emc2_scan_check(emc2_ctx* ctx, const char* what, emc2_dtype dtype, int64_t capacity, int32_t channels, int32_t states) {
  if (!emc2_is_float(dtype)) return emc2_fail(ctx, EMC2_ERR_UNSUPPORTED, "%s: dtype must be F32, F16 or BF16", what);
  if (channels < 1 || channels > (1 << 16)) return emc2_fail(ctx, EMC2_ERR_UNSUPPORTED, "%s: channels outside [1, 2^16]", what);
  if (states < 1 || states > kMaxStates) return emc2_fail(ctx, EMC2_ERR_UNSUPPORTED, "%s: states outside [1, %d]", what, kMaxStates);
  if (capacity < 0 || capacity > (1ll << 30)) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: rows outside [0, 2^30]", what);
  return EMC2_OK;
}

extern "C" emc2_status emc2_selective_scan(emc2_ctx* ctx, emc2_dtype dtype, const void* d_x, int64_t ld_x, const void* d_dt, int64_t ld_dt,
                                           const float* d_a, const void* d_b, int64_t ld_b, const void* d_c, int64_t ld_c, const float* d_skip,
                                           const float* d_dt_bias, const int32_t* d_offsets, int32_t n_seq, int64_t capacity, int32_t channels,
                                           int32_t states, int32_t backwards, const float* d_h0, void* d_y, int64_t ld_y, float* d_last,
                                           void* d_work, int64_t work_bytes, void* stream) {
  if (!ctx) return EMC2_ERR_INVALID_ARG;
  const char* const what = "emc2_selective_scan";
  const emc2_status st = emc2_scan_check(ctx, what, dtype, capacity, channels, states);
  if (st != EMC2_OK) return st;
  if (n_seq < 1 || n_seq > (1 << 30) || !d_offsets) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: offsets null or n_seq outside [1, 2^30]", what);
  const size_t size = emc2_size_of(dtype);
  const bool none = capacity == 0;
  const int64_t kept = (int64_t)n_seq * channels * states;
  if (!d_a) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: null argument", what);
  if (!rows_ok(d_x, ld_x, channels, size, none) || !rows_ok(d_dt, ld_dt, channels, size, none) || !rows_ok(d_b, ld_b, states, size, none) ||
      !rows_ok(d_c, ld_c, states, size, none) || !rows_ok(d_y, ld_y, channels, size, none))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: null or misaligned rows, or a pitch below the values of a row or beyond 2^26", what);
  const emc2_rows y = {d_y, ld_y, channels}, own[] = {{d_x, ld_x, channels}, {d_dt, ld_dt, channels}}, shared[] = {{d_b, ld_b, states}, {d_c, ld_c, states}};
  if (!emc2_results_ok(&y, 1, own, 2, capacity, size, true) || !emc2_results_ok(&y, 1, shared, 2, capacity, size, false))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: d_y overlaps d_b or d_c, or d_x or d_dt at another place or pitch", what);
  if (!emc2_apart(d_last, kept, d_h0, kept)) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: d_last must not overlap d_h0", what);
  const emc2_scan_plan p = emc2_plan_scan(capacity, channels, states, false);
  const bool small = capacity <= kShortRows;
  const int64_t need = small ? 0 : emc2_scan_totals_size(p.chunks, channels, states) * (int64_t)sizeof(float);
  if (work_bytes < need || (need && (!d_work || ((uintptr_t)d_work & 15))))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: work buffer null, misaligned or smaller than emc2_selective_scan_work", what);
  ScanArgs a = {};
  a.x = d_x, a.dt = d_dt, a.b = d_b, a.c = d_c, a.a = d_a, a.skip = d_skip, a.dt_bias = d_dt_bias, a.h0 = d_h0, a.offsets = d_offsets, a.y = d_y;
  a.last = d_last, a.flags = ctx->dev_words, a.ld_x = ld_x, a.ld_dt = ld_dt, a.ld_b = ld_b, a.ld_c = ld_c, a.ld_y = ld_y;
  a.capacity = (int32_t)capacity, a.channels = channels, a.states = states, a.n_seq = n_seq, a.backwards = backwards != 0;
  hipStream_t s = (hipStream_t)stream;
  if (small) {
    with_type(dtype, [&](auto type) {
      using T = decltype(type);
      with_short_form(states, [&](auto form) {
        using F = decltype(form);
        // chunks of whole batches, as many waves as they make
        const int64_t per = emc2_div_up(emc2_div_up(capacity, short_waves(F::p)), kBatch) * kBatch;
        a.chunk = (int32_t)(per < kBatch ? kBatch : per);
        const int64_t waves = emc2_div_up(capacity, a.chunk) < 1 ? 1 : emc2_div_up(capacity, a.chunk);
        const int32_t slices = (int32_t)emc2_div_up(channels, 64 / F::p);
        a.row_blocks = 1;
        const dim3 grid((unsigned)(1 + hand_on_blocks(n_seq, slices, d_last)), (unsigned)slices);
        hipLaunchKernelGGL((k_scan_short<T, F::p>), grid, dim3((unsigned)(64 * waves)),
                           (size_t)(waves * (2 * kBatch * 4 * F::p + 5 * 64) * sizeof(float)), s, a);
      });
    });
    return emc2_check_hip(ctx, hipGetLastError(), "emc2_selective_scan launch");
  }
  emc2_place_totals(a, 0, (float*)d_work, p);
  a.chunk = p.chunk, a.row_blocks = p.spans;
  emc2_scan_totals(a, dtype, p, false, s);
  with_type(dtype, [&](auto type) {
    using T = decltype(type);
    with_form(states, p.lanes, [&](auto form) {
      using F = decltype(form);
      const int32_t slices = (int32_t)emc2_div_up(channels, 64 / F::p);
      const dim3 grid((unsigned)(p.spans + hand_on_blocks(n_seq, slices, d_last)), (unsigned)slices);
      hipLaunchKernelGGL((k_scan<T, F::s, F::p>), grid, dim3(64 * kChunkWaves), 0, s, a);
    });
  });
  return emc2_check_hip(ctx, hipGetLastError(), "emc2_selective_scan launch");
}

extern "C" emc2_status emc2_selective_scan_step(emc2_ctx* ctx, emc2_dtype dtype, const void* d_x, int64_t ld_x, const void* d_dt, int64_t ld_dt,
                                                const float* d_a, const void* d_b, int64_t ld_b, const void* d_c, int64_t ld_c,
                                                const float* d_skip, const float* d_dt_bias, const float* d_h, int64_t rows, int32_t channels,
                                                int32_t states, float* d_h_out, void* d_y, int64_t ld_y, void* stream) {
  if (!ctx) return EMC2_ERR_INVALID_ARG;
  const char* const what = "emc2_selective_scan_step";
  const emc2_status st = emc2_scan_check(ctx, what, dtype, rows, channels, states);
  if (st != EMC2_OK) return st;
  if (rows == 0) return EMC2_OK;
  const size_t size = emc2_size_of(dtype);
  const int64_t kept = rows * channels * states;
  if (!d_a || !d_h || !d_h_out) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: null argument", what);
  if (!emc2_rows_ok(d_x, ld_x, channels, size, false) || !emc2_rows_ok(d_dt, ld_dt, channels, size, false) ||
      !emc2_rows_ok(d_b, ld_b, states, size, false) || !emc2_rows_ok(d_c, ld_c, states, size, false) || !emc2_rows_ok(d_y, ld_y, channels, size, false))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: null or misaligned rows, or a pitch below the values of a row", what);
  const emc2_rows y = {d_y, ld_y, channels}, own[] = {{d_x, ld_x, channels}, {d_dt, ld_dt, channels}}, shared[] = {{d_b, ld_b, states}, {d_c, ld_c, states}};
  if (!emc2_results_ok(&y, 1, own, 2, rows, size, true) || !emc2_results_ok(&y, 1, shared, 2, rows, size, false) ||
      (d_h != d_h_out && !emc2_apart(d_h, kept, d_h_out, kept)))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: d_y overlaps an input, or d_h_out d_h, at another place or pitch", what);
  ScanArgs a = {};
  a.x = d_x, a.dt = d_dt, a.b = d_b, a.c = d_c, a.a = d_a, a.skip = d_skip, a.dt_bias = d_dt_bias, a.y = d_y;
  a.ld_x = ld_x, a.ld_dt = ld_dt, a.ld_b = ld_b, a.ld_c = ld_c, a.ld_y = ld_y, a.channels = channels, a.states = states;
  with_type(dtype, [&](auto type) {
    using T = decltype(type);
    with_short_form(states, [&](auto form) {
      constexpr int P = decltype(form)::p;
      hipLaunchKernelGGL((k_scan_step<T, P>), emc2_grid(emc2_div_up(rows * channels * P, kStepThreads)), dim3(kStepThreads), 0, (hipStream_t)stream, a, d_h,
                         d_h_out, rows);
    });
  });
  return emc2_check_hip(ctx, hipGetLastError(), "emc2_selective_scan_step launch");
}
