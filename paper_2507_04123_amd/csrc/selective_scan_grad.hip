// Gradients of the selective state space scan.
//   g_t = C_t dy_t + a_{t+1} g_{t+1} (+ dlast behind the last row), a = exp(D A): the gradient of the state h_t
//   dC_t = sum over channels of dy h_t;  dB_t = sum over channels of g D x;  dx = skip dy + D sum over states of g B
//   dD = sum over states of (g a h_{t-1}) A + x sum of g B;  ddt = dD softplus';  dA = sum over rows of g a h_{t-1} D;  dskip = sum of dy x;  dh0 = a_1 g_1
// g runs against h with the same factors.  The first launch (selective_scan_totals.hip) walks every chunk of rows once for the totals of both directions and writes the
// state before every eight rows; the second finds what enters the spans of chunks from either side; the third (k_scan_grad) walks a chunk's batches of eight
// rows from the last to the first: forward through a batch, whose states stay in registers, then back through it with the decays made again.  Nothing is kept from the forward pass.
// A block has up to eight waves, all with the same rows, each with a slice of the channels: sums over channels, dB and dC, are taken over a wave's lanes by
// swaps that halve the number of values with every step, over the waves through LDS.  Wider rows have several such blocks, whose sums are added in a last launch.
// Weights' gradients stay in registers along a chunk and are added over chunks by halves.  No atomics, no order that may change: equal inputs give equal bits.
// Vector issue bounds it: 200,003 rows of 128 channels by 16 states in bf16 take the first launch 147 us, k_scan_grad 413 us, 237 issue slots a row of 32 channels (the recurrence
// about 130 of them, its decays made twice included; the sums over channels about 40), the units busy 76 % of the time at the two waves a SIMD that a batch's states leave room for.  Eight states a lane with the decays kept beside them: one wave, 538 us; four states
// a lane: 528 us, for what belongs to the channel is repeated in more lanes.
#include "column_sums.h"
#include "selective_scan.h"

namespace {

// Sums of v[s] over the lanes that differ in channel only.  Bits 5 and 4 (S = 8: and 3) of the lane choose between halves of what is left until one value is;
// the other channel bits add.
template <int S, int P> __device__ __forceinline__ float channel_sum(const float (&v)[S], int lane) {
  float w[S / 2];
#pragma unroll
  for (int s = 0; s < S / 2; ++s) w[s] = swapped_sum32(v[s], v[s + S / 2]);
#pragma unroll
  for (int s = 0; s < S / 4; ++s) w[s] = swapped_sum16(w[s], w[s + S / 4]);
  float r = w[0];
  if constexpr (S == 8) {
    const bool high = lane & 8;
    r = (high ? w[1] : w[0]) + moved<0x128>(high ? w[0] : w[1]);     // row_ror:8, which is lane ^ 8
    if constexpr (P <= 4) r += moved<0x1B>(moved<0x141>(r));         // lane ^ 7, then lane ^ 3
  } else {
    if constexpr (P <= 8) r += moved<0x128>(r);
    if constexpr (P <= 4) r += moved<0x124>(r);                      // row_ror:4: as good as lane ^ 4 by now
  }
  if constexpr (P <= 2) r += moved<0x4E>(r);
  if constexpr (P == 1) r += moved<0xB1>(r);
  return r;
}
template <int S> __device__ __forceinline__ int kept_state(int lane) {
  return S == 8 ? (lane >> 5) * 4 + (lane >> 4 & 1) * 2 + (lane >> 3 & 1) : (lane >> 5) * 2 + (lane >> 4 & 1);
}
// Lanes that write: one of those that hold the same value.
template <int S, int P> __device__ __forceinline__ bool writes(int lane) { return (lane & (S == 8 ? 7 : 15) & ~(P - 1)) == 0; }

constexpr int grad_waves(int width) { return width <= 32 ? 8 : 4; }

template <typename T, int S, int P> __global__ void __launch_bounds__(64 * grad_waves(S * P), 2) k_scan_grad(const ScanArgs a) {
  constexpr bool kKeep = S == 4;                           // decays stay in registers, too; otherwise they are made again
  constexpr int kWidth = S * P, kPair = 2 * kBatch * kWidth, Q = Slots<P>::Q, R = Slots<P>::R;
  constexpr bool kExact = sizeof(T) == 4;
  extern __shared__ float lds[];                           // B and C of two batches [2][kPair], zeros [kPair], then the waves' sums for two batches [2][waves][kPair]
  const Walk w(a.offsets, a.n_seq, a.capacity, a.backwards);
  if (a.capacity == 0) report_rows(a.offsets, a.n_seq, a.capacity, a.flags);   // (otherwise the totals' launch has done so)
  if ((int32_t)blockIdx.x >= a.row_blocks) return hand_on(a, w, a.dlast, a.dh0);
  const int waves = blockDim.x >> 6;
  const States<S, P> t(a, blockIdx.y * waves + (threadIdx.x >> 6));
  const int q = t.part % Q;
  const int64_t first = (int64_t)blockIdx.x * a.chunk;
  float* const line = a.partial + (int64_t)blockIdx.x * ((int64_t)a.channels * (a.states + 2));
  float a2[S], flow[S], enter[S], dA[S], dskip = 0.0f, dbias = 0.0f;
  decays(a, t, a2);
#pragma unroll
  for (int s = 0; s < S; ++s) dA[s] = 0.0f;
  if (first < w.n) {
    const int32_t row0 = (int32_t)first, end = first + a.chunk < w.n ? row0 + a.chunk : w.n;
    const int32_t spans = spans_of(a, w.n);
    entering<0, S>(a, t, a2, blockIdx.x, spans, enter);
    entering<1, S>(a, t, a2, blockIdx.x, spans, flow);
    const float bias = a.dt_bias ? a.dt_bias[t.channel] : 0.0f, skip = a.skip ? a.skip[t.channel] : 0.0f;
    const bool idle = __any(!t.in), ragged = a.states != kWidth || idle;
    Cursor at;
    Staged<T, kWidth, 2> bc;
    constexpr bool kSoon = Staged<T, kWidth, 2>::kMine <= 2;   // B and C are requested with the rows; wide ones, which would take 16 registers, when they are due
    Column<T, P> x, v, dy;
    float before[S], before_s;
    const Line<const T> xs(w, (const T*)a.x, a.ld_x), vs(w, (const T*)a.dt, a.ld_dt), dys(w, (const T*)a.dy, a.ld_dy);
    const Line<const T> bs(w, (const T*)a.b, a.ld_b), cs(w, (const T*)a.c, a.ld_c);
    const Line<T> dxs(w, (T*)a.y, a.ld_y), ddts(w, (T*)a.ddt, a.ld_ddt);
    const int32_t bytes = t.channel * (int32_t)sizeof(T);
    bc.open(bs, cs, threadIdx.x, blockDim.x);
    const auto fetch = [&](int32_t r0) {
      if constexpr (kSoon) bc.fetch(bs, cs, r0, end, a.states);
      x.fetch(xs, bytes, q, r0, w.n);
      v.fetch(vs, bytes, q, r0, w.n);
      dy.fetch(dys, bytes, q, r0, w.n);
      t.load(a, a.batch_h + (int64_t)(r0 / kBatch) * a.channels * a.states, before);
      before_s = a.batch_s[(int64_t)(r0 / kBatch) * a.channels + t.channel];
    };
    const int32_t last = row0 + (end - row0 - 1) / kBatch * kBatch;
    for (int i = threadIdx.x; i < kPair; i += blockDim.x) lds[2 * kPair + i] = 0.0f;
    fetch(last);
    at.fill(w, w.n_seq < 64 ? 0 : w.find(last, t.lane) - 31, t.lane);
    if constexpr (!kSoon) bc.fetch(bs, cs, last, end, a.states);
    bc.put(lds + (last / kBatch & 1) * kPair);
    __syncthreads();
    for (int32_t r0 = last; r0 >= row0; r0 -= kBatch) {
      const int turn = r0 / kBatch & 1;
      const float* const now = lds + (t.in ? turn : 2) * kPair + t.first;
      float* const sums = lds + 3 * kPair + (turn * waves + t.wave) * kPair + t.first + kept_state<S>(t.lane);
      float d[R], xv[R], dyv[R], slope[R], gb[R], dd[R], h[S];
#pragma unroll
      for (int j = 0; j < R; ++j) {
        step_of<kExact>((float)v.v[j] + bias, d[j], slope[j]);
        xv[j] = (float)x.v[j], dyv[j] = (float)dy.v[j];
        gb[j] = 0.0f, dd[j] = 0.0f;
      }
      // Lanes without a channel, which take part in the sums over channels, have rows of zeros, B and C too: what they have read is channel 0's, and another block may
      // be writing its gradients there.
      if (idle && !t.in) {
#pragma unroll
        for (int j = 0; j < R; ++j) d[j] = 0.0f, xv[j] = 0.0f, dyv[j] = 0.0f;
        before_s = 0.0f;
      }
#pragma unroll
      for (int s = 0; s < S; ++s) h[s] = enter[s];
      through<S>(a2, before_s, before, h);
      fetch(r0 > row0 ? r0 - kBatch : row0);               // (unconditional: what it replaces need not be kept for a second way)
      at.before(w, r0, t.lane);
      const Rows<P> dx_rows(dxs, bytes, q, r0, w.n), ddt_rows(ddts, bytes, q, r0, w.n);
      const auto finish = [&](int j, float row_gb, float row_dd) __attribute__((always_inline)) {
        const float dv = __builtin_fmaf(row_dd, 0.693147180559945309f, row_gb * xv[j]) * slope[j];
        float dx = d[j] * row_gb;
        if (a.skip) dx = __builtin_fmaf(skip, dyv[j], dx);
        if (j * Q + q < end - r0) {
          dskip = __builtin_fmaf(dyv[j], xv[j], dskip);
          dbias += dv;
          if (t.in && t.part < Q) dx_rows.template store<T>(j, q, (T)dx), ddt_rows.template store<T>(j, q, (T)dv);
        }
      };
      // PLAIN: all rows are there, none begins or ends a sequence, and nothing infinite has to be kept out of states that are none.
      const auto rows = [&](auto plain) __attribute__((always_inline)) {
        constexpr bool PLAIN = decltype(plain)::value;
        float prev[kBatch][S], keep[kKeep ? kBatch : 1][S];
        int32_t seq[kBatch];
        uint32_t begins = 0, ends = 0;
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          const int32_t r = r0 + i;
          if (!PLAIN && r >= end) break;
          const float di = a_row<PLAIN>(of_row<P>(d, i)), gi = di * of_row<P>(xv, i), dyi = of_row<P>(dyv, i);
          if constexpr (!PLAIN) {
            if (r >= at.next) {
              at.locate(w, r, t.lane);
              t.load_or_zero(a, a.h0, w.number(at.j), h);
              begins |= 1u << i;
            }
            seq[i] = w.number(at.j);
            if (r + 1 >= at.next) ends |= 1u << i;
          }
          float b[S];
          from_lds<S>(now + i * kWidth, b);
#pragma unroll
          for (int s = 0; s < S; ++s) {
            prev[i][s] = h[s];
            const float one = __builtin_amdgcn_exp2f(di * a2[s]);
            if constexpr (kKeep) keep[i][s] = one;
            b[s] *= gi;
            if (!PLAIN) b[s] = s < t.there ? b[s] : 0.0f;
            h[s] = __builtin_fmaf(one, h[s], b[s]);
            b[s] = dyi * h[s];
          }
          const float dC = channel_sum<S, P>(b, t.lane);
          if (writes<S, P>(t.lane)) sums[(kBatch + i) * kWidth] = dC;
        }
#pragma unroll
        for (int i = kBatch - 1; i >= 0; --i) {
          const int32_t r = r0 + i;
          if (!PLAIN && r >= end) continue;
          const float di = a_row<PLAIN>(of_row<P>(d, i)), gi = di * of_row<P>(xv, i), dyi = of_row<P>(dyv, i);
          if (!PLAIN && (ends >> i & 1)) t.load_or_zero(a, a.dlast, seq[i], flow);
          float b[S], c[S], sum_gb = 0.0f, sum_dd = 0.0f;
          from_lds<S>(now + i * kWidth, b);
          from_lds<S>(now + (kBatch + i) * kWidth, c);
#pragma unroll
          for (int s = 0; s < S; ++s) {
            float g = __builtin_fmaf(c[s], dyi, flow[s]);
            if (!PLAIN) g = s < t.there ? g : 0.0f;
            sum_gb = __builtin_fmaf(g, b[s], sum_gb);
            flow[s] = (kKeep ? keep[kKeep ? i : 0][s] : __builtin_amdgcn_exp2f(di * a2[s])) * g;
            const float e = flow[s] * prev[i][s];          // reaches the exponent
            sum_dd = __builtin_fmaf(e, a2[s], sum_dd);
            dA[s] = __builtin_fmaf(e, di, dA[s]);
            b[s] = g * gi;
          }
          const float dB = channel_sum<S, P>(b, t.lane);
          if (writes<S, P>(t.lane)) sums[i * kWidth] = dB;
          sum_gb = lane_sum<P>(sum_gb), sum_dd = lane_sum<P>(sum_dd);
          if constexpr (Q == 1) {
            finish(i, sum_gb, sum_dd);
          } else {
            gb[i / Q] = q == i % Q ? sum_gb : gb[i / Q];
            dd[i / Q] = q == i % Q ? sum_dd : dd[i / Q];
          }
          if (!PLAIN && (begins >> i & 1) && a.dh0 && t.in) t.store(a, a.dh0, seq[i], flow);
        }
      };
      bool plain = r0 + kBatch <= end && r0 + kBatch < at.next;
      if (plain && ragged) {
        float gain[R];
#pragma unroll
        for (int j = 0; j < R; ++j) gain[j] = d[j] * xv[j];
        plain = !any_infinite(gain) && !any_infinite(dyv);
      }
      if (plain) rows(Yes());
      else rows(No());
      if constexpr (Q > 1) {
#pragma unroll
        for (int j = 0; j < R; ++j) finish(j, gb[j], dd[j]);
      }
      // the next batch's B and C to the other half, this one's sums over the waves out of theirs
      if constexpr (!kSoon) bc.fetch(bs, cs, r0 > row0 ? r0 - kBatch : row0, end, a.states);
      if (r0 > row0) bc.put(lds + (turn ^ 1) * kPair);
      __syncthreads();
      for (int e = threadIdx.x; e < kPair; e += blockDim.x) {
        const int n = e % kWidth, i = e / kWidth % kBatch, which = e / (kWidth * kBatch);
        const int32_t r = r0 + i;
        float all = 0.0f;
        for (int m = 0; m < waves; ++m) all += lds[3 * kPair + (turn * waves + m) * kPair + e];
        if (n < a.states && r < end) {
          if (gridDim.y > 1) a.partial_bc[(((int64_t)blockIdx.y * a.capacity + r) * 2 + which) * a.states + n] = all;
          else if (which == 0) ((T*)a.db + w.row(r) * a.ld_db)[n] = (T)all;
          else ((T*)a.dc + w.row(r) * a.ld_dc)[n] = (T)all;
        }
      }
    }
  }
  // rows of the channel's lanes; lanes beyond the first Q have the same again
  dskip = lane_sum<Q>(dskip), dbias = lane_sum<Q>(dbias);
  if (t.in) {
    t.store(a, line, 0, dA);
    if (t.part == 0) {
      line[(int64_t)a.channels * a.states + t.channel] = dskip;
      line[(int64_t)a.channels * (a.states + 1) + t.channel] = dbias;
    }
  }
}

// dB and dC from the sums of the parts of the channels, in their order.
constexpr int kSumThreads = 256;
template <typename T> __global__ void __launch_bounds__(kSumThreads) k_scan_grad_bc(const ScanArgs a, int32_t parts) {
  const Walk w(a.offsets, a.n_seq, a.capacity, a.backwards);
  const int64_t i = emc2_block() * kSumThreads + threadIdx.x, pair = i / a.states, r = pair >> 1;
  if (r >= w.n) return;
  const int32_t n = (int32_t)(i - pair * a.states);
  const int64_t line = (int64_t)a.capacity * 2 * a.states;
  float all = 0.0f;
  for (int32_t p = 0; p < parts; ++p) all += a.partial_bc[p * line + i];
  if (pair & 1) ((T*)a.dc + w.row((int32_t)r) * a.ld_dc)[n] = (T)all;
  else ((T*)a.db + w.row((int32_t)r) * a.ld_db)[n] = (T)all;
}

template <typename F> void with_grad_form(int32_t states, int32_t lanes, F&& f) {
  if (states <= 4) return f(Form<4, 1>());
  if (states <= 8) return f(Form<4, 2>());
  if (states <= 16) return lanes == 4 ? f(Form<4, 4>()) : f(Form<8, 2>());
  if (states <= 32) return f(Form<8, 4>());
  f(Form<8, 8>());
}
// Slices of the channels, waves of a block, blocks side by side.
struct Cut { int32_t slices, waves, parts; };
Cut cut_of(int32_t channels, int32_t states, int32_t lanes) {
  Cut c;
  with_grad_form(states, lanes, [&](auto form) {
    using F = decltype(form);
    c.slices = (int32_t)emc2_div_up(channels, 64 / F::p);
    const int32_t most = grad_waves(F::s * F::p);
    c.parts = (int32_t)emc2_div_up(c.slices, most);
    c.waves = (int32_t)emc2_div_up(c.slices, c.parts);
  });
  return c;
}
int64_t shared_size(int64_t capacity, int32_t states, int64_t parts) { return parts > 1 ? parts * capacity * 2 * states : 0; }
// Floats of scratch: totals of both directions, states before batches, weights' sums, sums of dB and dC.
int64_t grad_size(int64_t capacity, int64_t chunks, int32_t channels, int32_t states, int64_t shared) {
  return 2 * emc2_scan_totals_size(chunks, channels, states) + emc2_div_up(capacity, kBatch) * channels * (states + 1) +
         (chunks > 1 ? chunks : 1) * channels * (states + 2) + shared;
}

}  // namespace

extern "C" int64_t emc2_selective_scan_work(emc2_dtype dtype, int64_t capacity, int32_t channels, int32_t states) {
  if (!emc2_is_float(dtype) || channels < 1 || channels > (1 << 16) || states < 1 || states > kMaxStates || capacity < 0 || capacity > (1ll << 30)) return -1;
  const int64_t forward = emc2_scan_totals_size(emc2_plan_scan(capacity, channels, states, false).most, channels, states);
  const emc2_scan_plan p = emc2_plan_scan(capacity, channels, states, true);
  // fewer rows may have more lanes a channel, and so more parts to sum
  const int64_t few = kFewWaveRows / emc2_div_up((int64_t)channels * 4, 64), narrow = shared_size(capacity < few ? capacity : few, states, cut_of(channels, states, 4).parts),
                now = shared_size(capacity, states, cut_of(channels, states, p.lanes).parts), grad = grad_size(capacity, p.most, channels, states, narrow > now ? narrow : now);
  return (forward > grad ? forward : grad) * (int64_t)sizeof(float);
}

extern "C" emc2_status emc2_selective_scan_backward(
    emc2_ctx* ctx, emc2_dtype dtype, const void* d_x, int64_t ld_x, const void* d_dt, int64_t ld_dt, const float* d_a, const void* d_b, int64_t ld_b,
    const void* d_c, int64_t ld_c, const float* d_skip, const float* d_dt_bias, const int32_t* d_offsets, int32_t n_seq, int64_t capacity,
    int32_t channels, int32_t states, int32_t backwards, const float* d_h0, const void* d_dy, int64_t ld_dy, const float* d_dlast, void* d_dx,
    int64_t ld_dx, void* d_ddt, int64_t ld_ddt, float* d_da, void* d_db, int64_t ld_db, void* d_dc, int64_t ld_dc, float* d_dskip,
    float* d_ddt_bias, float* d_dh0, void* d_work, int64_t work_bytes, void* stream) {
  if (!ctx) return EMC2_ERR_INVALID_ARG;
  const char* const what = "emc2_selective_scan_backward";
  const emc2_status st = emc2_scan_check(ctx, what, dtype, capacity, channels, states);
  if (st != EMC2_OK) return st;
  if (n_seq < 1 || n_seq > (1 << 30) || !d_offsets) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: offsets null or n_seq outside [1, 2^30]", what);
  const size_t size = emc2_size_of(dtype);
  const bool none = capacity == 0;
  const int64_t kept = (int64_t)n_seq * channels * states;
  if (!d_a || !d_da || (!d_skip && d_dskip)) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: null argument", what);
  if (!rows_ok(d_x, ld_x, channels, size, none) || !rows_ok(d_dt, ld_dt, channels, size, none) ||
      !rows_ok(d_b, ld_b, states, size, none) || !rows_ok(d_c, ld_c, states, size, none) ||
      !rows_ok(d_dy, ld_dy, channels, size, none) || !rows_ok(d_dx, ld_dx, channels, size, none) ||
      !rows_ok(d_ddt, ld_ddt, channels, size, none) || !rows_ok(d_db, ld_db, states, size, none) ||
      !rows_ok(d_dc, ld_dc, states, size, none))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: null or misaligned rows, or a pitch below the values of a row or beyond 2^26", what);
  const emc2_rows outs[] = {{d_dx, ld_dx, channels}, {d_ddt, ld_ddt, channels}, {d_db, ld_db, states}, {d_dc, ld_dc, states}},
                  own[] = {{d_x, ld_x, channels}, {d_dt, ld_dt, channels}, {d_dy, ld_dy, channels}}, shared[] = {{d_b, ld_b, states}, {d_c, ld_c, states}};
  if (!emc2_results_ok(outs, 4, shared, 2, capacity, size, false) || !emc2_results_ok(outs, 2, own, 3, capacity, size, true) ||
      !emc2_results_ok(outs + 2, 2, own, 3, capacity, size, false))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: results overlap each other or inputs (only d_dx and d_ddt may lie where d_x, d_dt or d_dy do)", what);
  if (!emc2_apart(d_dh0, kept, d_dlast, kept) || !emc2_apart(d_dh0, kept, d_h0, kept))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: d_dh0 must not overlap d_dlast or d_h0", what);
  const emc2_scan_plan p = emc2_plan_scan(capacity, channels, states, true);
  const Cut cut = cut_of(channels, states, p.lanes);
  if (work_bytes < grad_size(capacity, p.chunks, channels, states, shared_size(capacity, states, cut.parts)) * (int64_t)sizeof(float) || !d_work || ((uintptr_t)d_work & 15))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: work buffer null, misaligned or smaller than emc2_selective_scan_work", what);
  ScanArgs a = {};
  a.x = d_x, a.dt = d_dt, a.b = d_b, a.c = d_c, a.dy = d_dy, a.a = d_a, a.skip = d_skip, a.dt_bias = d_dt_bias, a.h0 = d_h0, a.dlast = d_dlast;
  a.offsets = d_offsets, a.y = d_dx, a.ddt = d_ddt, a.db = d_db, a.dc = d_dc, a.dh0 = d_dh0, a.flags = ctx->dev_words;
  a.ld_x = ld_x, a.ld_dt = ld_dt, a.ld_b = ld_b, a.ld_c = ld_c, a.ld_dy = ld_dy, a.ld_y = ld_dx, a.ld_ddt = ld_ddt, a.ld_db = ld_db, a.ld_dc = ld_dc;
  a.capacity = (int32_t)capacity, a.channels = channels, a.states = states, a.n_seq = n_seq, a.backwards = backwards != 0, a.chunk = p.chunk;
  float* place = emc2_place_totals(a, 1, emc2_place_totals(a, 0, (float*)d_work, p), p);
  a.batch_h = place, place += emc2_div_up(capacity, kBatch) * channels * states;
  a.batch_s = place, place += emc2_div_up(capacity, kBatch) * channels;
  a.row_blocks = p.chunks > 1 ? p.chunks : 1;
  a.partial = place, place += (int64_t)a.row_blocks * channels * (states + 2);
  a.partial_bc = place;
  hipStream_t s = (hipStream_t)stream;
  if (capacity > 0) emc2_scan_totals(a, dtype, p, true, s);
  const int64_t more = d_dh0 ? emc2_div_up(n_seq, 16ll * cut.parts) : 0;
  with_type(dtype, [&](auto type) {
    using T = decltype(type);
    with_grad_form(states, p.lanes, [&](auto form) {
      using F = decltype(form);
      const dim3 grid((unsigned)(a.row_blocks + (more < 1024 ? more : 1024)), (unsigned)cut.parts);
      hipLaunchKernelGGL((k_scan_grad<T, F::s, F::p>), grid, dim3((unsigned)(64 * cut.waves)),
                         (size_t)((3 + 2 * cut.waves) * 2 * kBatch * F::s * F::p * sizeof(float)), s, a);
    });
    if (cut.parts > 1 && capacity > 0)
      hipLaunchKernelGGL((k_scan_grad_bc<T>), emc2_grid(emc2_div_up(capacity * 2 * states, kSumThreads)), dim3(kSumThreads), 0, s, a, cut.parts);
  });
  Columns c = {};
  const int32_t cn = channels * states;
  c.parts = a.partial, c.lines = a.row_blocks, c.width = cn + 2 * channels;
  c.to[0] = d_da, c.end[0] = cn, c.to[1] = d_dskip, c.end[1] = cn + channels, c.to[2] = d_ddt_bias, c.end[2] = c.width;
  emc2_column_sums(c, s);
  return emc2_check_hip(ctx, hipGetLastError(), "emc2_selective_scan_backward launch");
}
