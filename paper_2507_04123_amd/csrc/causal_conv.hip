// Short causal convolution, channel by channel, along the rows of packed sequences; its gradients and its form for one row per sequence.
//   z_t = bias + sum over k < TAPS of w[k] x_{t-k},   y_t = silu(z_t) or z_t;   x before the first row: the caller's rows kept of before, or 0
//   dz_t = dy_t act'(z_t);  dx_t = sum over k of w[k] dz_{t+k} (rows of the same sequence; + dlast on the TAPS - 1 last);  dw[k] = sum of dz_t x_{t-k}
// A thread has N neighbouring channels of a run of rows.  Forward: it requests all rows of its run and the TAPS - 1 before it at once and goes through
// them with the taps in registers: the rows that neighbouring runs share come out of the caches, so memory sees every row once.  Gradients: it walks its run
// and the TAPS - 1 rows behind it with the last TAPS rows and the unfinished dx in registers; each dz is added to the TAPS rows before it.  Most waves see no
// end of a sequence and go without masks; the others know each row's depth in its sequence.
// Weights' gradients stay in registers while a thread walks its runs, are joined over a block in LDS and over blocks by a second launch in a fixed order.
// The rows that a sequence keeps (its last TAPS - 1, or what is left of the given ones) are written by blocks of their own.
// Memory bounds the forward pass: 613,217 rows of 96 f16 values in 45 to 54 us, 5.2 to 4.3 TB/s.  The gradients have as many bytes to move as vector instructions to
// issue and, of 4 values a thread, registers for three waves a SIMD: 200,003 rows of 160 bf16 values, 4 taps, 50 us (3.9 TB/s; 2 values a thread 76; 8 rows under way
// instead of 4: 62, at two waves).
#include "column_sums.h"
#include "rows.h"
#include "sequences.h"

namespace {

constexpr int kConvThreads = 256;
constexpr int kMaxTaps = 8;
constexpr int kRows = 8;                 // of a thread, forward
constexpr int kBatch = 4;                // rows that a thread of the backward pass has under way
constexpr int kMaxRun = 60, kMinRun = 8; // rows of a thread, backward
constexpr int64_t kGradBlocks = 2048;    // of the backward pass
constexpr int64_t kAtOnce = 768;         // of them on the chip together: the registers leave room for three on a CU

struct ConvArgs {
  const void *x, *dy;
  const float *w, *bias, *before, *dlast;      // bias, before, dlast may be null
  const int32_t* offsets;
  void* y;                                     // forward: y; backward: dx
  float *last, *dbefore, *partial;             // last, dbefore may be null; partial [blocks][(taps + 1) * channels]
  int32_t* flags;
  int64_t ld_x, ld_dy, ld_y;
  int32_t capacity, channels, n_seq, backwards, silu;
  int32_t pieces, runs_a_block, run;           // pieces of N channels in a block's slice; runs side by side in a block; rows of a run (backward)
  int32_t row_blocks;                          // blocks that walk rows; those behind them deal with states
};

// What a thread is: its piece of channels and its run's place among the block's.
template <int N> struct Lane {
  int32_t channel, twice;                      // first channel; a last piece that would pass the channels begins `twice` earlier
  int32_t group, first_group, last_group;      // of its wave
  bool in;
  __device__ __forceinline__ explicit Lane(const ConvArgs& a) {
    const int32_t t = threadIdx.x;
    group = t / a.pieces;
    const int32_t c = ((int32_t)blockIdx.y * a.pieces + (t - group * a.pieces)) * N;
    in = group < a.runs_a_block && c < a.channels;
    twice = in && c + N > a.channels ? c + N - a.channels : 0;
    channel = in ? c - twice : 0;
    const int32_t w = __builtin_amdgcn_readfirstlane(t & ~63);
    first_group = w / a.pieces;
    last_group = (w + 63) / a.pieces < a.runs_a_block ? (w + 63) / a.pieces : a.runs_a_block - 1;
    if (first_group > last_group) first_group = last_group;
  }
};

template <int N> __device__ __forceinline__ emc2_fvec<N> state_row(const float* p, const ConvArgs& a, int32_t taps, int32_t seq, int32_t i, int32_t c) {
  return p ? emc2_load<N>(p + ((int64_t)seq * (taps - 1) + i) * a.channels + c) : emc2_fvec<N>(0.0f);
}

template <bool EXACT, int N> __device__ __forceinline__ emc2_fvec<N> silu(emc2_fvec<N> z) {
#pragma unroll
  for (int e = 0; e < N; ++e) z[e] *= emc2_logistic<EXACT>(z[e]);
  return z;
}
template <bool EXACT, int N> __device__ __forceinline__ emc2_fvec<N> silu_slope(emc2_fvec<N> z) {
#pragma unroll
  for (int e = 0; e < N; ++e) {
    float on, off;
    emc2_logistic<EXACT>(z[e], on, off);
    z[e] = on * (1.0f + z[e] * off);
  }
  return z;
}

// Sequences that the rows [lo, hi) touch, by the whole wave; alone: they are rows of one sequence with none of its begin or end between them.
struct Reach { int32_t first, last; bool alone; };
__device__ __forceinline__ Reach reach(const Walk& w, int32_t lo, int32_t hi) {
  const int lane = threadIdx.x & 63;
  const int32_t from = lo > 0 ? lo : 0, to = hi < w.n ? hi : w.n;
  Reach r;
  r.first = w.find(from, lane);
  r.alone = lo >= w.start(r.first) && hi <= w.start(r.first + 1);
  r.last = r.alone || to <= from ? r.first : w.find(to - 1, lane);
  return r;
}

// The rows that sequences keep: a thread has a channel of a sequence.  Row i of them (oldest first) is row length - (TAPS - 1) + i of the sequence, or one of those
// before it.
template <typename T, int TAPS> __device__ __forceinline__ void keep_last(const ConvArgs& a, const Walk& w) {
  const int64_t all = (int64_t)a.n_seq * a.channels, step = (int64_t)(gridDim.x - a.row_blocks) * gridDim.y * kConvThreads;
  for (int64_t i = (((int64_t)blockIdx.x - a.row_blocks) * gridDim.y + blockIdx.y) * kConvThreads + threadIdx.x; i < all; i += step) {
    const int32_t j = (int32_t)(i / a.channels), c = (int32_t)(i - (int64_t)j * a.channels), seq = w.number(j);
    const int32_t start = w.start(j), length = max(w.start(j + 1) - start, 0);
    const int64_t kept = (int64_t)seq * (TAPS - 1) * a.channels + c;
    float v[TAPS - 1];
#pragma unroll
    for (int k = 0; k < TAPS - 1; ++k) {
      const int32_t at = length - (TAPS - 1) + k;
      v[k] = 0.0f;
      if (at >= 0) v[k] = (float)((const T*)a.x)[w.row(start + at) * a.ld_x + c];
      else if (a.before) v[k] = a.before[kept + (int64_t)(at + TAPS - 1) * a.channels];
    }
#pragma unroll
    for (int k = 0; k < TAPS - 1; ++k) a.last[kept + (int64_t)k * a.channels] = v[k];
  }
}

template <typename T, int N, int TAPS>
__global__ void __launch_bounds__(kConvThreads) k_causal_conv(const ConvArgs a) {
  const Walk w(a.offsets, a.n_seq, a.capacity, a.backwards);
  report_rows(a.offsets, a.n_seq, a.capacity, a.flags);
  if ((int32_t)blockIdx.x >= a.row_blocks) return keep_last<T, TAPS>(a, w);
  const int64_t block_row = (int64_t)blockIdx.x * a.runs_a_block * kRows;
  if (block_row >= w.n) return;
  const Lane<N> t(a);
  const int32_t row0 = (int32_t)block_row + t.group * kRows, wave0 = (int32_t)block_row + t.first_group * kRows,
                wave1 = (int32_t)block_row + (t.last_group + 1) * kRows;
  if (wave0 >= w.n) return;
  emc2_vec<T, N> x[kRows + TAPS - 1];                      // x[i]: row row0 - (TAPS - 1) + i; rows that are none read valid places
#pragma unroll
  for (int i = 0; i < kRows + TAPS - 1; ++i) {
    const int32_t r = row0 - (TAPS - 1) + i;
    x[i] = emc2_piece<N>((const T*)a.x + w.row(r < 0 ? 0 : r < w.n ? r : w.n - 1) * a.ld_x + t.channel);
  }
  emc2_fvec<N> taps[TAPS], bias = emc2_fvec<N>(0.0f);
#pragma unroll
  for (int k = 0; k < TAPS; ++k) taps[k] = emc2_load<N>(a.w + (int64_t)k * a.channels + t.channel);
  if (a.bias) bias = emc2_load<N>(a.bias + t.channel);
  const Reach q = reach(w, wave0 - (TAPS - 1), wave1);
  if (!t.in || row0 >= w.n) return;
  if (q.alone) {
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      emc2_fvec<N> z = bias;
#pragma unroll
      for (int k = 0; k < TAPS; ++k) z += taps[k] * __builtin_convertvector(x[i + TAPS - 1 - k], emc2_fvec<N>);
      if (a.silu) z = silu<sizeof(T) == 4, N>(z);
      emc2_store<N>((T*)a.y + w.row(row0 + i) * a.ld_y + t.channel, z);
    }
    return;
  }
  int32_t j = w.find_between(row0, q.first, q.last), start = w.start(j), next = w.start(j + 1);
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int32_t r = row0 + i;
    if (r >= w.n) break;
    if (r >= next) {
      j = w.find_between(r, j, q.last);
      start = w.start(j), next = w.start(j + 1);
    }
    const int32_t depth = r > start ? r - start : 0;
    emc2_fvec<N> z = bias;
#pragma unroll
    for (int k = 0; k < TAPS; ++k) {
      emc2_fvec<N> v = __builtin_convertvector(x[i + TAPS - 1 - k], emc2_fvec<N>);
      if (k > depth) v = state_row<N>(a.before, a, TAPS, w.number(j), TAPS - 1 + depth - k, t.channel);
      z += taps[k] * v;
    }
    if (a.silu) z = silu<sizeof(T) == 4, N>(z);
    emc2_store<N>((T*)a.y + w.row(r) * a.ld_y + t.channel, z);
  }
}

// Gradients of the rows before the first: a thread has a channel of a sequence, whose first TAPS - 1 rows are all that they reach.
template <typename T, int TAPS> __device__ __forceinline__ void before_grad(const ConvArgs& a, const Walk& w) {
  const int64_t all = (int64_t)a.n_seq * a.channels, step = (int64_t)(gridDim.x - a.row_blocks) * gridDim.y * kConvThreads;
  for (int64_t i = (((int64_t)blockIdx.x - a.row_blocks) * gridDim.y + blockIdx.y) * kConvThreads + threadIdx.x; i < all; i += step) {
    const int32_t j = (int32_t)(i / a.channels), c = (int32_t)(i - (int64_t)j * a.channels), seq = w.number(j);
    const int32_t start = w.start(j), length = max(w.start(j + 1) - start, 0);
    const int64_t kept = (int64_t)seq * (TAPS - 1) * a.channels + c;
    float x[2 * (TAPS - 1)], dz[TAPS - 1], taps[TAPS], v[TAPS - 1];   // x: the rows before, oldest first, and the first rows
#pragma unroll
    for (int k = 0; k < TAPS; ++k) taps[k] = a.w[(int64_t)k * a.channels + c];
#pragma unroll
    for (int p = 0; p < TAPS - 1; ++p) {
      x[p] = a.before ? a.before[kept + (int64_t)p * a.channels] : 0.0f;
      x[TAPS - 1 + p] = p < length ? (float)((const T*)a.x)[w.row(start + p) * a.ld_x + c] : 0.0f;
      dz[p] = p < length ? (float)((const T*)a.dy)[w.row(start + p) * a.ld_dy + c] : 0.0f;
      v[p] = a.dlast && p >= length ? a.dlast[kept + (int64_t)(p - length) * a.channels] : 0.0f;
    }
    if (a.silu) {
      const float bias = a.bias ? a.bias[c] : 0.0f;
#pragma unroll
      for (int p = 0; p < TAPS - 1; ++p) {
        float z = bias;
#pragma unroll
        for (int k = 0; k < TAPS; ++k) z += taps[k] * x[TAPS - 1 + p - k];
        if (p < length) dz[p] *= silu_slope<sizeof(T) == 4, 1>(emc2_fvec<1>(z))[0];
      }
    }
#pragma unroll
    for (int k = 0; k < TAPS - 1; ++k) {                     // row k reaches rows p of the sequence, TAPS - 1 - k + p rows behind it
#pragma unroll
      for (int p = 0; p <= k; ++p) v[k] += p < length ? taps[TAPS - 1 - k + p] * dz[p] : 0.0f;
      a.dbefore[kept + (int64_t)k * a.channels] = v[k];
    }
  }
}

// One run of rows [row0, end) and the TAPS - 1 behind it.
template <bool MASKED, typename T, int N, int TAPS>
__device__ __forceinline__ void walk_run(const ConvArgs& a, const Walk& w, const Lane<N>& t, const Reach& q, int32_t row0, int32_t end,
                                         const emc2_fvec<N> (&taps)[TAPS], emc2_fvec<N> bias, emc2_fvec<N> (&dw)[TAPS], emc2_fvec<N>& db) {
  emc2_fvec<N> xs[TAPS], dx[TAPS];                         // x_{t-k} and the unfinished dx_{t-k}
#pragma unroll
  for (int k = 0; k < TAPS; ++k) xs[k] = 0.0f, dx[k] = 0.0f;
  int32_t j = 0, depth = 0, next = 0;
  if constexpr (MASKED) {
    j = w.find_between(row0, q.first, q.last);
    depth = max(row0 - w.start(j), 0) - 1, next = w.start(j + 1);  // of the row before row0
  }
#pragma unroll
  for (int k = 1; k < TAPS; ++k) {                         // the rows before row0, as x_{t-k} of row0 - 1 before its first move
    if (!MASKED || k <= depth + 1) xs[k - 1] = emc2_load<N>((const T*)a.x + w.row(row0 - k) * a.ld_x + t.channel);
    else xs[k - 1] = state_row<N>(a.before, a, TAPS, w.number(j), TAPS + depth - k, t.channel);
  }
  emc2_vec<T, N> x[kBatch], dy[kBatch];
  const auto fetch = [&](int32_t r) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int64_t at = w.row(r + i < w.n ? r + i : w.n - 1);
      x[i] = emc2_piece<N>((const T*)a.x + at * a.ld_x + t.channel);
      dy[i] = emc2_piece<N>((const T*)a.dy + at * a.ld_dy + t.channel);
    }
  };
  fetch(row0);
  for (int32_t r0 = row0; r0 < end + TAPS - 1; r0 += kBatch) {
    emc2_fvec<N> xv[kBatch], dyv[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) xv[i] = __builtin_convertvector(x[i], emc2_fvec<N>), dyv[i] = __builtin_convertvector(dy[i], emc2_fvec<N>);
    if (r0 + kBatch < end + TAPS - 1) fetch(r0 + kBatch);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int32_t r = r0 + i;
#pragma unroll
      for (int k = TAPS - 1; k > 0; --k) xs[k] = xs[k - 1], dx[k] = dx[k - 1];
      xs[0] = xv[i], dx[0] = 0.0f;
      const bool there = !MASKED || r < w.n;
      if constexpr (MASKED) {
        ++depth;
        if (there && r >= next) {                          // a sequence begins
          j = w.find_between(r, j, q.last);
          depth = 0, next = w.start(j + 1);
#pragma unroll
          for (int k = 1; k < TAPS; ++k) xs[k] = state_row<N>(a.before, a, TAPS, w.number(j), TAPS - 1 - k, t.channel);
        }
        if (there && a.dlast && (uint32_t)(next - 1 - r) < (uint32_t)(TAPS - 1)) dx[0] = state_row<N>(a.dlast, a, TAPS, w.number(j), TAPS - 2 - (next - 1 - r), t.channel);
      }
      emc2_fvec<N> dz = dyv[i];
      if (a.silu) {
        emc2_fvec<N> z = bias;
#pragma unroll
        for (int k = 0; k < TAPS; ++k) z += taps[k] * xs[k];
        dz *= silu_slope<sizeof(T) == 4, N>(z);
      }
#pragma unroll
      for (int k = 0; k < TAPS; ++k)
        if (!MASKED || (there && k <= depth)) dx[k] += taps[k] * dz;
      if (r < end) {
        db += dz;
#pragma unroll
        for (int k = 0; k < TAPS; ++k) dw[k] += dz * xs[k];
      }
      const int32_t out = r - (TAPS - 1);
      if (out >= row0 && out < end) emc2_store<N>((T*)a.y + w.row(out) * a.ld_y + t.channel, dx[TAPS - 1]);
    }
  }
}

template <typename T, int N, int TAPS>
__global__ void __launch_bounds__(kConvThreads) k_causal_conv_grad(const ConvArgs a) {
  __shared__ emc2_fvec<N> part[TAPS + 1][kConvThreads / 2];
  const Walk w(a.offsets, a.n_seq, a.capacity, a.backwards);
  report_rows(a.offsets, a.n_seq, a.capacity, a.flags);
  if ((int32_t)blockIdx.x >= a.row_blocks) return before_grad<T, TAPS>(a, w);
  const Lane<N> t(a);
  emc2_fvec<N> taps[TAPS], bias = emc2_fvec<N>(0.0f), dw[TAPS], db = emc2_fvec<N>(0.0f);
#pragma unroll
  for (int k = 0; k < TAPS; ++k) taps[k] = emc2_load<N>(a.w + (int64_t)k * a.channels + t.channel), dw[k] = 0.0f;
  if (a.bias) bias = emc2_load<N>(a.bias + t.channel);
  const int64_t step = (int64_t)a.row_blocks * a.runs_a_block * a.run;
  for (int64_t block_row = (int64_t)blockIdx.x * a.runs_a_block * a.run; block_row < w.n; block_row += step) {
    const int64_t row0 = block_row + (int64_t)t.group * a.run, wave0 = block_row + (int64_t)t.first_group * a.run,
                  wave1 = block_row + (int64_t)(t.last_group + 1) * a.run + TAPS - 1;
    if (wave0 >= w.n) break;
    const Reach q = reach(w, (int32_t)wave0 - (TAPS - 1), wave1 < 0x7fffffff ? (int32_t)wave1 : 0x7fffffff);
    if (!t.in || row0 >= w.n) continue;
    const int32_t end = row0 + a.run < w.n ? (int32_t)row0 + a.run : w.n;
    if (q.alone) walk_run<false, T, N, TAPS>(a, w, t, q, (int32_t)row0, end, taps, bias, dw, db);
    else walk_run<true, T, N, TAPS>(a, w, t, q, (int32_t)row0, end, taps, bias, dw, db);
  }
  // The block's sums: the upper half of the runs side by side hands its sums to the lower until one is left.
  for (int32_t m = a.runs_a_block; m > 1;) {
    const int32_t half = (m + 1) / 2;
    if (t.in && t.group >= half && t.group < m) {
#pragma unroll
      for (int k = 0; k <= TAPS; ++k) part[k][threadIdx.x - half * a.pieces] = k < TAPS ? dw[k < TAPS ? k : 0] : db;
    }
    __syncthreads();
    if (t.in && t.group + half < m) {
#pragma unroll
      for (int k = 0; k < TAPS; ++k) dw[k] += part[k][threadIdx.x];
      db += part[TAPS][threadIdx.x];
    }
    __syncthreads();
    m = half;
  }
  if (!t.in || t.group > 0) return;
  float* const line = a.partial + (int64_t)blockIdx.x * (TAPS + 1) * a.channels + t.channel;
#pragma unroll
  for (int k = 0; k <= TAPS; ++k)
#pragma unroll
    for (int e = 0; e < N; ++e)                            // (a piece moved back leaves its neighbour's channels to that one)
      if (e >= t.twice) line[(int64_t)k * a.channels + e] = k < TAPS ? dw[k < TAPS ? k : 0][e] : db[e];
}

// One row per sequence, one value a thread: the rows kept move up by one.
template <typename T>
__global__ void __launch_bounds__(kConvThreads) k_causal_conv_step(const T* x, int64_t ld_x, const float* w, const float* bias, const float* state,
                                                                   float* state_out, T* y, int64_t ld_y, int64_t rows, int32_t channels,
                                                                   int32_t taps, int32_t act) {
  const int64_t i = emc2_block() * kConvThreads + threadIdx.x;
  if (i >= rows * channels) return;
  const int64_t row = i / channels;
  const int32_t c = (int32_t)(i - row * channels);
  float v[kMaxTaps];
#pragma unroll
  for (int k = 0; k < kMaxTaps - 1; ++k) v[k] = k < taps - 1 ? state[(row * (taps - 1) + k) * channels + c] : 0.0f;   // oldest first
  const float now = (float)x[row * ld_x + c];
  float z = bias ? bias[c] : 0.0f;
  z += w[c] * now;
#pragma unroll
  for (int k = 0; k < kMaxTaps - 1; ++k)
    if (k < taps - 1) z += w[(int64_t)(taps - 1 - k) * channels + c] * v[k];
  v[kMaxTaps - 1] = 0.0f;
#pragma unroll
  for (int k = 0; k < kMaxTaps - 1; ++k)
    if (k < taps - 1) state_out[(row * (taps - 1) + k) * channels + c] = k + 1 < taps - 1 ? v[k + 1] : now;
  if (act) z = silu<sizeof(T) == 4, 1>(emc2_fvec<1>(z))[0];
  y[row * ld_y + c] = (T)z;
}

// How a call is cut: values a piece, slices of the channels, pieces of a slice, runs side by side in a block.
struct Plan { int n; int32_t slices, pieces, runs; };
Plan plan_of(int whole, int32_t channels) {
  Plan p;
  p.n = channels >= whole ? whole : 1;
  const int32_t pieces = (channels + p.n - 1) / p.n;
  p.slices = (pieces + 63) / 64;
  p.pieces = (pieces + p.slices - 1) / p.slices;
  p.runs = kConvThreads / p.pieces;
  return p;
}
// Values a piece: 16 bytes, half of that where eight taps of as many values would leave registers for one wave a SIMD (613,217 rows of 96 f16 values: 54 us, 84 with
// whole pieces; six taps 51 and 47).
constexpr int whole_forward(size_t size, int32_t taps) { return size == 4 || taps == kMaxTaps ? 4 : 8; }
constexpr int kWholeGrad = 4;
// Blocks that write the states: a channel of a sequence a thread, as many blocks as keep the chip busy at most.
int64_t state_blocks(int32_t n_seq, int32_t channels, int32_t slices, bool any) {
  if (!any) return 0;
  const int64_t b = emc2_div_up((int64_t)n_seq * channels, (int64_t)kConvThreads * slices);
  return b < 2048 ? b : 2048;
}
// Rows of a run: as many as leave every block that the chip holds at once its share, so that no second round of blocks runs half empty
// (200,003 rows of 160 bf16 values: 56 us with runs of 32, 49 with runs of 44).  No longer than 60: rows under way lie ever further apart, which costs more than
// the rows between runs, read twice, do (613,217 rows of 96: 95 us with runs of 28 to 60, 104 with 100, 116 with 128).
int32_t run_of(int64_t capacity, const Plan& p) {
  const int64_t threads = kAtOnce * kConvThreads / (p.pieces * p.slices), per = emc2_div_up(capacity, threads < 1 ? 1 : threads);
  return (int32_t)(per < kMinRun ? kMinRun : per < kMaxRun ? (per + kBatch - 1) / kBatch * kBatch : kMaxRun);
}
int64_t grad_blocks(int64_t runs, const Plan& p) {
  const int64_t blocks = emc2_div_up(runs, p.runs), most = kGradBlocks / p.slices > 1 ? kGradBlocks / p.slices : 1;
  return blocks < 1 ? 1 : blocks < most ? blocks : most;
}

template <typename F> void with_type(emc2_dtype dtype, F&& f) {
  if (dtype == EMC2_F32) f(float());
  else if (dtype == EMC2_F16) f(_Float16());
  else f(__bf16());
}
template <int K> struct Taps { static constexpr int k = K; };
template <typename F> void with_taps(int32_t taps, F&& f) {
  switch (taps) {
    case 2: return f(Taps<2>());
    case 3: return f(Taps<3>());
    case 4: return f(Taps<4>());
    case 5: return f(Taps<5>());
    case 6: return f(Taps<6>());
    case 7: return f(Taps<7>());
    default: return f(Taps<8>());
  }
}

constexpr int32_t kMaxConvChannels = 1 << 16;
emc2_status check(emc2_ctx* ctx, const char* what, emc2_dtype dtype, int64_t capacity, int32_t channels, int32_t taps) {
  if (!emc2_is_float(dtype)) return emc2_fail(ctx, EMC2_ERR_UNSUPPORTED, "%s: dtype must be F32, F16 or BF16", what);
  if (channels < 1 || channels > kMaxConvChannels) return emc2_fail(ctx, EMC2_ERR_UNSUPPORTED, "%s: channels outside [1, 2^16]", what);
  if (taps < 2 || taps > kMaxTaps) return emc2_fail(ctx, EMC2_ERR_UNSUPPORTED, "%s: taps outside [2, %d]", what, kMaxTaps);
  if (capacity < 0 || capacity > (1ll << 30)) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: rows outside [0, 2^30]", what);
  return EMC2_OK;
}
emc2_status check_offsets(emc2_ctx* ctx, const char* what, const void* offsets, int32_t n_seq) {
  if (n_seq < 1 || n_seq > (1 << 30) || !offsets) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: offsets null or n_seq outside [1, 2^30]", what);
  return EMC2_OK;
}

}  // namespace

extern "C" emc2_status emc2_causal_conv(emc2_ctx* ctx, emc2_dtype dtype, const void* d_x, int64_t ld_x, const float* d_w, const float* d_bias,
                                        int32_t silu, const int32_t* d_offsets, int32_t n_seq, int64_t capacity, int32_t channels, int32_t taps,
                                        int32_t backwards, const float* d_before, void* d_y, int64_t ld_y, float* d_last, void* stream) {
  if (!ctx) return EMC2_ERR_INVALID_ARG;
  const char* const what = "emc2_causal_conv";
  emc2_status st = check(ctx, what, dtype, capacity, channels, taps);
  if (st == EMC2_OK) st = check_offsets(ctx, what, d_offsets, n_seq);
  if (st != EMC2_OK) return st;
  const size_t size = emc2_size_of(dtype);
  const bool none = capacity == 0;
  const int64_t kept = (int64_t)n_seq * (taps - 1) * channels;
  if (!d_w) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: null argument", what);
  if (!emc2_rows_ok(d_x, ld_x, channels, size, none) || !emc2_rows_ok(d_y, ld_y, channels, size, none))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: null or misaligned rows, or a pitch below the channels", what);
  if (!emc2_apart({d_y, ld_y, channels}, {d_x, ld_x, channels}, capacity, size) || !emc2_apart(d_last, kept, d_before, kept))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: d_y must not overlap d_x, nor d_last d_before", what);
  const Plan p = plan_of(whole_forward(size, taps), channels);
  ConvArgs a = {};
  a.x = d_x, a.w = d_w, a.bias = d_bias, a.before = d_before, a.offsets = d_offsets, a.y = d_y, a.last = d_last, a.flags = ctx->dev_words;
  a.ld_x = ld_x, a.ld_y = ld_y, a.capacity = (int32_t)capacity, a.channels = channels, a.n_seq = n_seq, a.backwards = backwards != 0;
  a.silu = silu != 0, a.pieces = p.pieces, a.runs_a_block = p.runs;
  a.row_blocks = (int32_t)emc2_div_up(capacity, (int64_t)p.runs * kRows);
  int64_t blocks = a.row_blocks + state_blocks(n_seq, channels, p.slices, d_last);
  if (blocks == 0) a.row_blocks = 1, blocks = 1;           // a block that reports rows beyond the capacity
  const dim3 grid((unsigned)blocks, (unsigned)p.slices);
  with_type(dtype, [&](auto type) {
    using T = decltype(type);
    with_taps(taps, [&](auto k) {
      constexpr int K = decltype(k)::k, N = whole_forward(sizeof(T), K);
      if (p.n > 1) hipLaunchKernelGGL((k_causal_conv<T, N, K>), grid, dim3(kConvThreads), 0, (hipStream_t)stream, a);
      else hipLaunchKernelGGL((k_causal_conv<T, 1, K>), grid, dim3(kConvThreads), 0, (hipStream_t)stream, a);
    });
  });
  return emc2_check_hip(ctx, hipGetLastError(), "emc2_causal_conv launch");
}

extern "C" int64_t emc2_causal_conv_work(emc2_dtype dtype, int64_t capacity, int32_t channels, int32_t taps) {
  if (!emc2_is_float(dtype) || channels < 1 || channels > kMaxConvChannels || taps < 2 || taps > kMaxTaps || capacity < 0 || capacity > (1ll << 30))
    return -1;
  const Plan p = plan_of(kWholeGrad, channels);
  return grad_blocks(emc2_div_up(capacity, kMinRun), p) * (taps + 1) * channels * (int64_t)sizeof(float);
}

extern "C" emc2_status emc2_causal_conv_backward(emc2_ctx* ctx, emc2_dtype dtype, const void* d_x, int64_t ld_x, const float* d_w,
                                                 const float* d_bias, int32_t silu, const int32_t* d_offsets, int32_t n_seq, int64_t capacity,
                                                 int32_t channels, int32_t taps, int32_t backwards, const float* d_before, const void* d_dy,
                                                 int64_t ld_dy, const float* d_dlast, void* d_dx, int64_t ld_dx, float* d_dw, float* d_dbias,
                                                 float* d_dbefore, void* d_work, int64_t work_bytes, void* stream) {
  if (!ctx) return EMC2_ERR_INVALID_ARG;
  const char* const what = "emc2_causal_conv_backward";
  emc2_status st = check(ctx, what, dtype, capacity, channels, taps);
  if (st == EMC2_OK) st = check_offsets(ctx, what, d_offsets, n_seq);
  if (st != EMC2_OK) return st;
  const size_t size = emc2_size_of(dtype);
  const bool none = capacity == 0;
  const int64_t kept = (int64_t)n_seq * (taps - 1) * channels;
  if (!d_w || !d_dw) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: null argument", what);
  if (!emc2_rows_ok(d_x, ld_x, channels, size, none) || !emc2_rows_ok(d_dy, ld_dy, channels, size, none) ||
      !emc2_rows_ok(d_dx, ld_dx, channels, size, none))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: null or misaligned rows, or a pitch below the channels", what);
  if (!emc2_apart({d_dx, ld_dx, channels}, {d_x, ld_x, channels}, capacity, size) ||
      !emc2_apart({d_dx, ld_dx, channels}, {d_dy, ld_dy, channels}, capacity, size) || !emc2_apart(d_dbefore, kept, d_before, kept) ||
      !emc2_apart(d_dbefore, kept, d_dlast, kept))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: d_dx must not overlap d_x or d_dy, nor d_dbefore d_before or d_dlast", what);
  if (work_bytes < emc2_causal_conv_work(dtype, capacity, channels, taps) || !d_work || ((uintptr_t)d_work & 15))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: work buffer null, misaligned or smaller than emc2_causal_conv_work", what);
  const Plan p = plan_of(kWholeGrad, channels);
  ConvArgs a = {};
  a.x = d_x, a.dy = d_dy, a.w = d_w, a.bias = d_bias, a.before = d_before, a.dlast = d_dlast, a.offsets = d_offsets, a.y = d_dx;
  a.dbefore = d_dbefore, a.partial = (float*)d_work, a.flags = ctx->dev_words, a.ld_x = ld_x, a.ld_dy = ld_dy, a.ld_y = ld_dx;
  a.capacity = (int32_t)capacity, a.channels = channels, a.n_seq = n_seq, a.backwards = backwards != 0, a.silu = silu != 0;
  a.pieces = p.pieces, a.runs_a_block = p.runs, a.run = run_of(capacity, p);
  a.row_blocks = (int32_t)grad_blocks(emc2_div_up(capacity, a.run), p);
  const dim3 grid((unsigned)(a.row_blocks + state_blocks(n_seq, channels, p.slices, d_dbefore)), (unsigned)p.slices);
  with_type(dtype, [&](auto type) {
    using T = decltype(type);
    with_taps(taps, [&](auto k) {
      constexpr int K = decltype(k)::k;
      if (p.n > 1) hipLaunchKernelGGL((k_causal_conv_grad<T, kWholeGrad, K>), grid, dim3(kConvThreads), 0, (hipStream_t)stream, a);
      else hipLaunchKernelGGL((k_causal_conv_grad<T, 1, K>), grid, dim3(kConvThreads), 0, (hipStream_t)stream, a);
    });
  });
  Columns c = {};
  c.parts = a.partial, c.lines = a.row_blocks, c.width = (taps + 1) * channels;
  c.to[0] = d_dw, c.end[0] = taps * channels, c.to[1] = d_dbias, c.end[1] = c.end[2] = c.width;
  emc2_column_sums(c, (hipStream_t)stream);
  return emc2_check_hip(ctx, hipGetLastError(), "emc2_causal_conv_backward launch");
}

extern "C" emc2_status emc2_causal_conv_step(emc2_ctx* ctx, emc2_dtype dtype, const void* d_x, int64_t ld_x, const float* d_w,
                                             const float* d_bias, int32_t silu, const float* d_state, int64_t rows, int32_t channels,
                                             int32_t taps, float* d_state_out, void* d_y, int64_t ld_y, void* stream) {
  if (!ctx) return EMC2_ERR_INVALID_ARG;
  const char* const what = "emc2_causal_conv_step";
  const emc2_status st = check(ctx, what, dtype, rows, channels, taps);
  if (st != EMC2_OK) return st;
  const size_t size = emc2_size_of(dtype);
  const int64_t kept = rows * (taps - 1) * channels;
  if (rows == 0) return EMC2_OK;
  if (!d_w || !d_state || !d_state_out) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: null argument", what);
  if (!emc2_rows_ok(d_x, ld_x, channels, size, false) || !emc2_rows_ok(d_y, ld_y, channels, size, false))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: null or misaligned rows, or a pitch below the channels", what);
  const emc2_rows out = {d_y, ld_y, channels}, in = {d_x, ld_x, channels};
  if (!emc2_results_ok(&out, 1, &in, 1, rows, size, true) || (d_state != d_state_out && !emc2_apart(d_state, kept, d_state_out, kept)))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: d_y overlaps d_x, or d_state_out d_state, at another place or pitch", what);
  with_type(dtype, [&](auto type) {
    using T = decltype(type);
    hipLaunchKernelGGL((k_causal_conv_step<T>), emc2_grid(emc2_div_up(rows * channels, kConvThreads)), dim3(kConvThreads), 0, (hipStream_t)stream,
                       (const T*)d_x, ld_x, d_w, d_bias, d_state, d_state_out, (T*)d_y, ld_y, rows, channels, taps, (int32_t)(silu != 0));
  });
  return emc2_check_hip(ctx, hipGetLastError(), "emc2_causal_conv_step launch");
}
