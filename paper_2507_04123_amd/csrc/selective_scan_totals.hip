// The selective scan's first two launches: the totals of chunks of rows, in one direction or both, and what enters the spans of eight chunks (selective_scan.hip).
#include "selective_walk.h"

namespace {

// First launch: every chunk from a state of zeros, and what spans of eight chunks make of it.  Block (span, slice of the channels), a wave a chunk.
template <bool GRAD, typename T, int S, int P> __global__ void __launch_bounds__(64 * kChunkWaves, GRAD ? 2 : 4) k_scan_totals(const ScanArgs a) {
  constexpr int kWidth = S * P, kOwn = (GRAD ? 2 : 1) * kBatch * kWidth, kLine = 64 * S;   // a wave's LDS; its total
  __shared__ float lds[kChunkWaves * (kOwn > kLine ? kOwn : kLine)];
  __shared__ float sums[kChunkWaves][64];
  const Walk w(a.offsets, a.n_seq, a.capacity, a.backwards);
  report_rows(a.offsets, a.n_seq, a.capacity, a.flags);
  const States<S, P> t(a, blockIdx.y);
  const int64_t k = (int64_t)blockIdx.x * kChunkWaves + t.wave, row0 = k * a.chunk;
  if ((int64_t)blockIdx.x * kChunkWaves * a.chunk >= w.n) return;
  float a2[S], h[S], flow[S], sum = 0.0f;
  bool begun = false, ended = false;
  decays(a, t, a2);
#pragma unroll
  for (int s = 0; s < S; ++s) h[s] = 0.0f, flow[s] = 0.0f;
  if (row0 < w.n)
    walk<GRAD ? kGradTotals : kTotals, T, S, P>(a, w, t, a2, (int32_t)row0, row0 + a.chunk < w.n ? (int32_t)row0 + a.chunk : w.n, lds + t.wave * kOwn, h, sum,
                                                begun, flow, ended);
#pragma unroll
  for (int dir = 0; dir < (GRAD ? 2 : 1); ++dir) {
    const float s0 = (dir == 0 ? begun : ended) ? -1.0f : sum;
    const float(&mine)[S] = dir == 0 ? h : flow;
    __syncthreads();                                       // all waves are through with their rows, or the direction before
#pragma unroll
    for (int s = 0; s < S; ++s) lds[(t.wave * S + s) * 64 + t.lane] = mine[s];
    sums[t.wave][t.lane] = s0;
    __syncthreads();
    // what the chunks before this one make together, in the order of the direction; behind the last of them, the span
    float all[S], total = 0.0f;
#pragma unroll
    for (int s = 0; s < S; ++s) all[s] = 0.0f;
    const int before = dir == 0 ? t.wave : kChunkWaves - 1 - t.wave;
    for (int m = 0; m < before; ++m) {
      const int from = dir == 0 ? m : kChunkWaves - 1 - m;
      float v[S];
#pragma unroll
      for (int s = 0; s < S; ++s) v[s] = lds[(from * S + s) * 64 + t.lane];
      const float one = sums[from][t.lane];
      through<S>(a2, one, v, all);
      total = one < 0.0f ? -1.0f : total < 0.0f ? total : total + one;
    }
    if (t.in && row0 < w.n) {
      t.store(a, a.chunk_h[dir], k, all);
      if (t.part == 0) a.chunk_s[dir][k * a.channels + t.channel] = total;
    }
    if (before == kChunkWaves - 1 && t.in) {
      through<S>(a2, s0, mine, all);
      t.store(a, a.span_h[dir], blockIdx.x, all);
      if (t.part == 0) a.span_s[dir][(int64_t)blockIdx.x * a.channels + t.channel] = s0 < 0.0f ? -1.0f : total < 0.0f ? total : total + s0;
    }
  }
}

// Second launch: what enters every span.  A block has 32 states of the line [channels][states] and 32 runs of spans; a thread composes its run and, from what
// enters it, walks it again, out of registers.  blockIdx.y: the direction.
constexpr int kRuns = 32, kRunSpans = kMaxSpans / kRuns;
__global__ void __launch_bounds__(32 * kRuns) k_scan_enter(const ScanArgs a) {
  __shared__ float part_p[kRuns][33], part_h[kRuns][33];
  const int32_t rows = a.offsets[a.n_seq], n = rows < 0 ? 0 : rows < a.capacity ? rows : a.capacity;
  const int32_t spans = spans_of(a, n), per = (spans + kRuns - 1) / kRuns;
  const int col = threadIdx.x & 31, run = threadIdx.x >> 5, dir = blockIdx.y;
  const int64_t line = (int64_t)a.channels * a.states, at = (int64_t)blockIdx.x * 32 + col, mine = at < line ? at : line - 1;
  const float* const span_s = dir == 0 ? a.span_s[0] : a.span_s[1];
  const float* const span_h = dir == 0 ? a.span_h[0] : a.span_h[1];
  float* const enter = dir == 0 ? a.enter[0] : a.enter[1];
  const float a2 = a.a[mine] * kLog2e;
  const int32_t c = (int32_t)(mine / a.states), from = run * per;
  float p[kRunSpans], h[kRunSpans];
#pragma unroll
  for (int i = 0; i < kRunSpans; ++i) {
    const int32_t m = from + i;
    const bool there = i < per && m < spans;
    const int64_t span = there ? (dir == 0 ? m : spans - 1 - m) : 0;
    p[i] = there ? span_s[span * a.channels + c] : 0.0f;
    h[i] = there ? span_h[span * line + mine] : 0.0f;
  }
  // products of decays; a run in which a sequence begins has -1
  float all_p = 1.0f, all_h = 0.0f;
#pragma unroll
  for (int i = 0; i < kRunSpans; ++i) {
    p[i] = p[i] < 0.0f ? -1.0f : __builtin_amdgcn_exp2f(a2 * p[i]);
    all_h = p[i] < 0.0f ? h[i] : __builtin_fmaf(p[i], all_h, h[i]);
    all_p = p[i] < 0.0f || all_p < 0.0f ? -1.0f : all_p * p[i];
  }
  part_p[run][col] = all_p, part_h[run][col] = all_h;
  __syncthreads();
  float state = 0.0f;
  for (int m = 0; m < run; ++m) state = part_p[m][col] < 0.0f ? part_h[m][col] : __builtin_fmaf(part_p[m][col], state, part_h[m][col]);
#pragma unroll
  for (int i = 0; i < kRunSpans; ++i) {
    const int32_t m = from + i;
    if (i < per && m < spans && at < line) enter[(int64_t)(dir == 0 ? m : spans - 1 - m) * line + at] = state;
    state = p[i] < 0.0f ? h[i] : __builtin_fmaf(p[i], state, h[i]);
  }
}

}  // namespace

void emc2_scan_totals(const ScanArgs& a, emc2_dtype dtype, const emc2_scan_plan& p, bool grad, hipStream_t stream) {
  with_type(dtype, [&](auto type) {
    using T = decltype(type);
    const auto launch = [&](auto form, auto both) {
      using F = decltype(form);
      hipLaunchKernelGGL((k_scan_totals<decltype(both)::value, T, F::s, F::p>), dim3((unsigned)p.spans, (unsigned)emc2_div_up(a.channels, 64 / F::p)),
                         dim3(64 * kChunkWaves), 0, stream, a);
    };
    with_form(a.states, p.lanes, [&](auto form) {
      if (grad) launch(form, Yes());
      else launch(form, No());
    });
  });
  if (p.spans > 1)
    hipLaunchKernelGGL(k_scan_enter, dim3((unsigned)emc2_div_up((int64_t)a.channels * a.states, 32), grad ? 2u : 1u), dim3(32 * kRuns), 0, stream, a);
}
