// A wave's walk along the rows of a chunk of the selective scan, for the launches that make totals (selective_scan_totals.hip) and results (selective_scan.hip).
#pragma once
#include "selective_scan.h"

namespace {

enum { kTotals = 0, kGradTotals = 1, kRun = 2 };

// Walks rows [row0, end) of a chunk, a wave alone, with LDS of its own (lds [2][kBatch][WIDTH]).  kTotals: h becomes what the chunk makes of it, sum the sum of its
// steps and `begun` whether a sequence begins in it.  kGradTotals: also what flows out of the chunk towards earlier rows, from none behind it (flow), and whether
// a sequence ends in it (ended); the states before every batch are written.  kRun: writes y and the last states.
template <int MODE, typename T, int S, int P>
__device__ __forceinline__ void walk(const ScanArgs& a, const Walk& w, const States<S, P>& t, const float (&a2)[S], int32_t row0, int32_t end, float* lds,
                                     float (&h)[S], float& sum, bool& begun, float (&flow)[S], bool& ended) {
  constexpr int kWidth = S * P, kArrays = MODE == kTotals ? 1 : 2, Q = Slots<P>::Q, R = Slots<P>::R;
  constexpr bool kExact = sizeof(T) == 4;
  const int q = t.part % Q;
  Staged<T, kWidth, kArrays> bc;
  constexpr bool kSoon = sizeof(T) == 2 || Staged<T, kWidth, kArrays>::kMine == 1;   // B and C are requested with the rows; wide ones, for lack of registers, when due
  Column<T, P> x, v, dy;
  const Line<const T> xs(w, (const T*)a.x, a.ld_x), vs(w, (const T*)a.dt, a.ld_dt), dys(w, (const T*)a.dy, a.ld_dy);
  const Line<const T> bs(w, (const T*)a.b, a.ld_b), cs(w, (const T*)a.c, a.ld_c);
  const Line<T> ys(w, (T*)a.y, a.ld_y);
  const int32_t bytes = t.channel * (int32_t)sizeof(T);
  bc.open(bs, cs, t.lane, 64);
  const auto fetch = [&](int32_t r0) {
    if constexpr (kSoon) bc.fetch(bs, cs, r0, end, a.states);
    x.fetch(xs, bytes, q, r0, w.n);
    v.fetch(vs, bytes, q, r0, w.n);
    if constexpr (MODE == kGradTotals) dy.fetch(dys, bytes, q, r0, w.n);
  };
  fetch(row0);
  const float bias = a.dt_bias ? a.dt_bias[t.channel] : 0.0f;
  const float skip = MODE == kRun && a.skip ? a.skip[t.channel] : 0.0f;
  const bool ragged = a.states != kWidth || __any(!t.in);
  Cursor at;
  at.open(w, row0, t.lane);
  float decay[S];                                          // kGradTotals: of all rows so far
  if constexpr (MODE == kGradTotals) {
#pragma unroll
    for (int s = 0; s < S; ++s) decay[s] = 1.0f, flow[s] = 0.0f;
    ended = false;
  }
  for (int32_t r0 = row0; r0 < end; r0 += kBatch) {
    if constexpr (!kSoon) bc.fetch(bs, cs, r0, end, a.states);
    bc.put(lds);
    float d[R], xv[R], y[R], dyv[R];
#pragma unroll
    for (int j = 0; j < R; ++j) {
      float slope;
      step_of<kExact>((float)v.v[j] + bias, d[j], slope);
      xv[j] = (float)x.v[j], y[j] = 0.0f, dyv[j] = 0.0f;
      if constexpr (MODE == kGradTotals) dyv[j] = (float)dy.v[j];
    }
    fetch(r0 + kBatch < end ? r0 + kBatch : r0);           // (unconditional: what it replaces need not be kept for a second way)
    if constexpr (MODE == kGradTotals) {
      if (t.in) {
        t.store(a, a.batch_h, r0 / kBatch, h);
        if (t.part == 0) a.batch_s[(int64_t)(r0 / kBatch) * a.channels + t.channel] = begun ? -1.0f : sum;
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const Rows<P> y_rows(ys, bytes, q, r0, w.n);
    // One row; returns what its states add to y.  PLAIN: it begins and ends no sequence, and its gain is finite where lanes have states that are none (an infinite
    // gain stays out of those; a NaN is in the channel's other states too).  LIVE (kGradTotals): it adds to the flow; without PLAIN that is looked at here.
    const auto row = [&](auto plain, auto live, int i, float di, float xi, float dyi) __attribute__((always_inline)) {
      constexpr bool PLAIN = decltype(plain)::value, LIVE = decltype(live)::value;
      const float gi = di * xi;
      if (!PLAIN && r0 + i >= at.next) {                   // a sequence begins
        at.locate(w, r0 + i, t.lane);
        t.load_or_zero(a, a.h0, w.number(at.j), h);
        begun = true;
      }
      float b[S], keep[S];
      int32_t there = t.there;
      if (!PLAIN && MODE == kGradTotals) asm volatile("" : "+v"(there));   // (compared anew in every row: masks kept for all would take the registers)
      from_lds<S>(lds + i * kWidth + t.first, b);
#pragma unroll
      for (int s = 0; s < S; ++s) {
        b[s] *= gi;
        if (!PLAIN) b[s] = s < there ? b[s] : 0.0f;
        keep[s] = __builtin_amdgcn_exp2f(di * a2[s]);
        h[s] = __builtin_fmaf(keep[s], h[s], b[s]);
      }
      float all = 0.0f;
      if constexpr (MODE != kRun) {
        sum += di;
#pragma unroll
        for (int s = 0; s < S; ++s) row_ends_with(h[s]);
      }
      if constexpr (MODE == kGradTotals) {
        if (PLAIN ? LIVE : !ended) {
          float c[S];
          from_lds<S>(lds + (kBatch + i) * kWidth + t.first, c);
#pragma unroll
          for (int s = 0; s < S; ++s) {
            decay[s] *= keep[s];
            flow[s] = __builtin_fmaf(decay[s], c[s] * dyi, flow[s]);
            row_ends_with(flow[s]);
          }
          if (!PLAIN && r0 + i + 1 >= at.next) {           // a sequence ends
            float l[S];
            t.load_or_zero(a, a.dlast, w.number(at.j), l);
#pragma unroll
            for (int s = 0; s < S; ++s) flow[s] = __builtin_fmaf(decay[s], l[s], flow[s]);
            ended = true;
          }
        }
      }
      if constexpr (MODE == kRun) {
        float c[S], part[4] = {Q == 1 && a.skip ? skip * xi : 0.0f, 0.0f, 0.0f, 0.0f};
        from_lds<S>(lds + (kBatch + i) * kWidth + t.first, c);
#pragma unroll
        for (int s = 0; s < S; ++s) part[s & 3] = __builtin_fmaf(c[s], h[s], part[s & 3]);
        all = lane_sum<P>((part[0] + part[1]) + (part[2] + part[3]));
        if constexpr (Q == 1) {
          if (t.in) y_rows.template store<T>(i, q, (T)all);
        }
        if (!PLAIN && r0 + i + 1 >= at.next && a.last && t.in) t.store(a, a.last, w.number(at.j), h);
      }
      return all;
    };
    const auto rows = [&](auto live) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const float di = a_row<1 + decltype(live)::value>(of_row<P>(d, i));
        const float all = row(Yes(), live, i, di, of_row<P>(xv, i), MODE == kGradTotals ? of_row<P>(dyv, i) : 0.0f);
        if constexpr (MODE == kRun && Q > 1) {
          y[i / Q] = q == i % Q ? all : y[i / Q];
          row_ends_with(y[i / Q]);
        }
      }
    };
    bool plain = r0 + kBatch <= end && r0 + kBatch < at.next;
    if (plain && ragged) {
      float gain[R];
#pragma unroll
      for (int j = 0; j < R; ++j) gain[j] = t.in ? d[j] * xv[j] : 0.0f;   // (lanes without a channel read channel 0's rows, which another block may be writing)
      plain = !any_infinite(gain);
    }
    if (plain) {
      if (MODE == kGradTotals && !ended) rows(Yes());
      else rows(No());
    } else if constexpr (MODE != kGradTotals) {
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        if (r0 + i >= end) break;
        const float di = a_row<0>(of_row<P>(d, i)), all = row(No(), No(), i, di, of_row<P>(xv, i), 0.0f);
        if constexpr (MODE == kRun && Q > 1) y[i / Q] = q == i % Q ? all : y[i / Q];
      }
    } else {
      // In one copy of the row's code, which leaves registers for decays and flows: the lane's values move down behind each row; after all of them they are
      // where they were.
#pragma unroll 1
      for (int i = 0; i < kBatch; ++i) {
        if (r0 + i < end) {
          const auto mine = [&](float v) { return Q == 1 ? v : __shfl(v, (t.lane & ~(Q - 1)) | (i & (Q - 1)), 64); };
          row(No(), No(), i, a_row<0>(mine(d[0])), mine(xv[0]), mine(dyv[0]));
        }
        if ((i & (Q - 1)) == Q - 1) {
          const float d0 = d[0], x0 = xv[0], dy0 = dyv[0];
#pragma unroll
          for (int j = 0; j + 1 < R; ++j) d[j] = d[j + 1], xv[j] = xv[j + 1], dyv[j] = dyv[j + 1];
          d[R - 1] = d0, xv[R - 1] = x0, dyv[R - 1] = dy0;
        }
      }
    }
    if constexpr (MODE == kRun && Q > 1) {
      if (t.in && t.part < Q) {
#pragma unroll
        for (int j = 0; j < R; ++j)
          if (j * Q + q < end - r0) y_rows.template store<T>(j, q, (T)(a.skip ? __builtin_fmaf(skip, xv[j], y[j]) : y[j]));
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// States a lane and lanes a channel: long lists as emc2_scan_lanes says, short calls four states (short chains).
template <typename F> void with_form(int32_t states, int32_t lanes, F&& f) {
  if (states <= 4) return f(Form<4, 1>());
  if (states <= 8) return lanes == 2 ? f(Form<4, 2>()) : f(Form<8, 1>());
  if (states <= 16) return lanes == 4 ? f(Form<4, 4>()) : lanes == 2 ? f(Form<8, 2>()) : f(Form<16, 1>());
  if (states <= 32) return lanes == 4 ? f(Form<8, 4>()) : f(Form<16, 2>());
  f(Form<16, 4>());
}
}  // namespace
