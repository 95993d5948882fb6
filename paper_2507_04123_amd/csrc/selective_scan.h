// What the kernels of the selective scan (selective_scan.hip, selective_scan_totals.hip, selective_scan_grad.hip) share: how states lie over lanes, the rows' way into registers and
// LDS, steps and decays, and the totals of runs of rows.
#pragma once
#include "lane_sums.h"
#include "rows.h"
#include "sequences.h"

struct emc2_scan_args {
  const void *x, *dt, *b, *c, *dy;
  const float *a, *skip, *dt_bias, *h0, *dlast;   // skip, dt_bias, h0, dlast may be null
  const int32_t* offsets;
  void *y, *ddt, *db, *dc;                     // y: forward: y; backward: dx
  float *last, *dh0;                           // may be null
  // of chunks: what those before them in their span make of a state of zeros; of spans: what they make of it (forward; in gradients also of the flow towards
  // earlier rows); what enters each span; the state before every batch
  float *chunk_s[2], *chunk_h[2], *span_s[2], *span_h[2], *enter[2], *batch_s, *batch_h;
  float *partial, *partial_bc;                 // weights' sums per chunk; sums of dB and dC per part of the channels
  int32_t* flags;
  int64_t ld_x, ld_dt, ld_b, ld_c, ld_dy, ld_y, ld_ddt, ld_db, ld_dc;
  int32_t capacity, channels, states, n_seq, backwards;
  int32_t chunk, row_blocks;                   // rows of a chunk; blocks that walk rows
};

namespace {

constexpr int kBatch = 8;                // rows under way together
constexpr int kChunkWaves = 8;           // chunks side by side in a block of the launch that reduces them: a block's total stands for them ("span")
// Chunks of a call times slices of its channels at most: as many waves as the chip holds at once of the forward pass, and of the gradients, whose waves have
// twice the registers (forward and gradients with the forward pass' cut and with its own: 200,003 rows of 128 channels by 16 states in bf16 783 and 747 us, 30,011 rows of
// 90 channels by 12 states in fp32 215 and 217).
constexpr int kMaxChunks = 4096, kMaxChunksGrad = 2048;
// A chunk has 16 rows at least, or 8 while that makes no more chunks than this, two waves a SIMD (128 channels by 16 states in bf16, 2000 rows forward and gradients
// 35 and 69 us with 16 and 32 rows, 27 and 40 with 8; 12,000 rows forward 39 us with 8 rows, 35 with 16).
constexpr int kFewChunks = 2048;
constexpr int kMaxSpans = kMaxChunks / kChunkWaves;
constexpr int kMaxStates = 64;

typedef emc2_scan_args ScanArgs;

// A lane has S neighbouring states of one channel; P lanes side by side have a channel's states, 64 / P channels lie in a wave.
template <int S, int P> struct States {
  static constexpr int kWidth = S * P, kChannels = 64 / P;
  int32_t lane, wave, part, channel, first, there;   // first: of its states; there: how many of them there are (0 without a channel)
  bool in;
  __device__ __forceinline__ States(const ScanArgs& a, int32_t slice) {
    lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    part = lane & (P - 1);
    channel = slice * kChannels + lane / P;
    in = channel < a.channels;
    if (!in) channel = 0;
    first = part * S;
    const int32_t left = a.states - first;
    there = !in || left < 0 ? 0 : left < S ? left : S;
  }
  // The lane's values of a line [channels][states].
  __device__ __forceinline__ void load(const ScanArgs& a, const float* line, float (&v)[S]) const {
    const float* const p = line + (int64_t)channel * a.states + first;
    if (there == S) {
#pragma unroll
      for (int i = 0; i < S; i += 4) {
        const emc2_fvec<4> q = emc2_load<4>(p + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i + e] = q[e];
      }
    } else {
#pragma unroll
      for (int i = 0; i < S; ++i) v[i] = i < there ? p[i] : 0.0f;
    }
  }
  __device__ __forceinline__ void load_or_zero(const ScanArgs& a, const float* lines, int64_t line, float (&v)[S]) const {
    if (lines) return load(a, lines + line * a.channels * a.states, v);
#pragma unroll
    for (int i = 0; i < S; ++i) v[i] = 0.0f;
  }
  __device__ __forceinline__ void store(const ScanArgs& a, float* lines, int64_t line, const float (&v)[S]) const {
    float* const p = lines + (line * a.channels + channel) * a.states + first;
    if (there == S) {
#pragma unroll
      for (int i = 0; i < S; i += 4) emc2_store<4>(p + i, emc2_fvec<4>{v[i], v[i + 1], v[i + 2], v[i + 3]});
    } else {
#pragma unroll
      for (int i = 0; i < S; ++i)
        if (i < there) p[i] = v[i];
    }
  }
};

// Steps: softplus(v) = log(1 + e), e = exp(v), and its slope e / (1 + e).  u = 1 + e is rounded; log(1 + e) = log(u) + (e - (u - 1)) / u to second order, so
// that steps far below 1 keep their places.  Beyond 20 the logarithm is v itself, to 2e-9.
template <bool EXACT> __device__ __forceinline__ void step_of(float v, float& d, float& slope) {
  float t;
  const float e = emc2_exp_of_minus<EXACT>(-v, t), u = 1.0f + e, r = __builtin_amdgcn_rcpf(u);
  const float l = __builtin_fmaf(__builtin_amdgcn_logf(u), 0.693147180559945309f, (e - (u - 1.0f)) * r);
  d = v > 20.0f ? v : l;
  slope = v > 20.0f ? 1.0f : e * r;
}
constexpr float kLog2e = 1.44269504088896341f;

// Sequences from a row on, by a window of 64 starts in the wave's lanes.
struct Cursor {
  int32_t j, next;                       // the sequence at hand and the row at which the one behind it starts
  int32_t base, mine;                    // of the window: its first sequence, the lane's start
  __device__ __forceinline__ void fill(const Walk& w, int32_t from, int lane) {
    base = from > 0 ? from : 0;
    mine = base + lane <= w.n_seq ? w.start(base + lane) : 0x7fffffff;
  }
  __device__ __forceinline__ int count(const Walk& w, int32_t r, int lane) const { return __popcll(__ballot(base + lane < w.n_seq && mine <= r)); }
  // The sequence of row r in [0, n).
  __device__ __forceinline__ void locate(const Walk& w, int32_t r, int lane) {
    int c = count(w, r, lane);
    if ((c == 0 && base > 0) || c == 64) {
      fill(w, w.find(r, lane) - 31, lane);
      c = count(w, r, lane);
    }
    c = c < 1 ? 1 : c < 63 ? c : 63;
    j = __builtin_amdgcn_readfirstlane(base + c - 1);
    next = __builtin_amdgcn_readlane(mine, c);
  }
  // Before row r: a sequence that starts with it is still to come.
  __device__ __forceinline__ void open(const Walk& w, int32_t r, int lane) {
    fill(w, w.n_seq < 64 ? 0 : w.find(r, lane) - 31, lane);
    before(w, r, lane);
  }
  __device__ __forceinline__ void before(const Walk& w, int32_t r, int lane) {
    locate(w, r, lane);
    if (__builtin_amdgcn_readlane(mine, j - base) >= r) next = r;
  }
};

// Rows of an operand in the order of a walk: row r lies r steps behind the first.
template <typename T> struct Line {
  T* first;
  int64_t step;                          // values; negative when the walk runs backwards
  __device__ __forceinline__ Line(const Walk& w, T* p, int64_t ld) : first(p + w.row(0) * ld), step(w.backwards ? -ld : ld) {}
};
// How a batch's rows lie over the lanes of a channel: of its first Q lanes (four at most) lane q has rows q, q + Q, ...; what belongs to a row and a channel is
// loaded, computed and stored by that lane alone and handed to the others where they need it.
template <int P> struct Slots {
  static constexpr int Q = P < 4 ? P : 4, R = kBatch / Q;
};
// Row i's value, from the lane that has it.
template <int P> __device__ __forceinline__ float of_row(const float (&v)[Slots<P>::R], int i) {
  constexpr int Q = Slots<P>::Q;
  if constexpr (Q == 1) return v[i];
  if constexpr (Q == 2) return i % 2 ? moved<0xF5>(v[i / 2]) : moved<0xA0>(v[i / 2]);
  const float own = v[i / Q];
  return i % 4 == 0 ? moved<0x00>(own) : i % 4 == 1 ? moved<0x55>(own) : i % 4 == 2 ? moved<0xAA>(own) : moved<0xFF>(own);
}
// The rows of the batch at r0 as a buffer, for accesses whose address is a scalar offset a row and a 32-bit one a lane (sums of 64 bits a lane cost several
// instructions each).  Rows beyond the last of n have its place.
template <int P> struct Rows {
  static constexpr int Q = Slots<P>::Q;
  __amdgpu_buffer_rsrc_t buffer;
  int32_t last, at0, step, lane;         // the last row; bytes to the first row, and from one to the next; the lane's own offset
  template <typename T> __device__ __forceinline__ Rows(const Line<T>& l, int32_t bytes, int q, int32_t r0, int32_t n) {
    last = n - 1 - r0 < kBatch - 1 ? n - 1 - r0 : kBatch - 1;
    const int32_t low = l.step < 0 ? last : 0;             // the row of the lowest address
    step = (int32_t)l.step * (int32_t)sizeof(T);
    at0 = low * -step;
    buffer = __builtin_amdgcn_make_buffer_rsrc((void*)(l.first + (r0 + low) * l.step), 0, -1, 0x00027000);
    if constexpr (Q > 1) {
      if (last == kBatch - 1) {
        lane = bytes + (l.step < 0 ? q - (Q - 1) : q) * step;
        if (l.step < 0) at0 += (Q - 1) * step;
        return;
      }
    }
    lane = bytes;
  }
  // Offsets of a slot's row: of the lane and of all.
  __device__ __forceinline__ int32_t of_lane(int slot, int q) const {
    if constexpr (Q > 1) {
      if (last < kBatch - 1) return lane + at0 + (slot * Q + q < last ? slot * Q + q : last) * step;
    }
    return lane;
  }
  __device__ __forceinline__ int32_t of_all(int slot) const {
    if constexpr (Q > 1) return last < kBatch - 1 ? 0 : at0 + slot * Q * step;
    return at0 + (slot < last ? slot : last) * step;
  }
  template <typename T> __device__ __forceinline__ T load(int slot, int q) const {
    if constexpr (sizeof(T) == 2) {
      const unsigned short v = __builtin_amdgcn_raw_buffer_load_b16(buffer, of_lane(slot, q), of_all(slot), 0);
      return __builtin_bit_cast(T, v);
    } else {
      const unsigned v = __builtin_amdgcn_raw_buffer_load_b32(buffer, of_lane(slot, q), of_all(slot), 0);
      return __builtin_bit_cast(T, v);
    }
  }
  template <typename T> __device__ __forceinline__ void store(int slot, int q, T v) const {
    if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, v), buffer, of_lane(slot, q), of_all(slot), 0);
    else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, v), buffer, of_lane(slot, q), of_all(slot), 0);
  }
};
constexpr int64_t kMaxPitch = 1 << 26;   // a batch's offsets stay below 2^31 bytes

// B and C of a batch, ARRAYS of them: pieces of PV values in registers on their way from memory, floats in LDS.  `threads` threads, at least 64, share them out.
template <typename T, int WIDTH, int ARRAYS> struct Staged {
  static constexpr int kWhole = 16 / sizeof(T), PV = kWhole < WIDTH ? kWhole : WIDTH, kARow = WIDTH / PV, kAll = ARRAYS * kBatch * kARow,
                       kMine = (kAll + 63) / 64;
  emc2_vec<T, PV> v[kMine];
  int32_t off[kMine];                    // a piece's place behind its array's first row of a batch, in values
  int32_t thread, threads;
  __device__ __forceinline__ int array(int q) const { return (q * threads + thread) / (kBatch * kARow); }
  __device__ __forceinline__ int row(int q) const { return (q * threads + thread) / kARow % kBatch; }
  __device__ __forceinline__ int state(int q) const { return (q * threads + thread) % kARow * PV; }
  __device__ __forceinline__ void open(const Line<const T>& b, const Line<const T>& c, int thread_, int threads_) {
    thread = thread_, threads = threads_;
#pragma unroll
    for (int q = 0; q < kMine; ++q) off[q] = row(q) * (int32_t)(array(q) ? c.step : b.step) + state(q);
  }
  // Rows of the batch at r0 that are none (at `end` or beyond) and states that are none become 0.
  __device__ __forceinline__ void fetch(const Line<const T>& b, const Line<const T>& c, int32_t r0, int32_t end, int32_t states) {
    const T *const b0 = b.first + r0 * b.step, *const c0 = c.first + r0 * c.step;
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
      v[q] = (T)0.0f;
      if (q * threads + thread < kAll && row(q) < end - r0) {
        const T* const p = (ARRAYS > 1 && array(q) ? c0 : b0) + off[q];
        const int there = states - state(q);
        if (there >= PV) {
          v[q] = emc2_piece<PV>(p);
        } else {
#pragma unroll
          for (int e = 0; e < PV; ++e)
            if (e < there) v[q][e] = p[e];
        }
      }
    }
  }
  __device__ __forceinline__ void put(float* to) const {   // to [ARRAYS][kBatch][WIDTH]
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
      const int id = q * threads + thread;
      if (id < kAll) {
        const emc2_fvec<PV> f = __builtin_convertvector(v[q], emc2_fvec<PV>);
#pragma unroll
        for (int e = 0; e < PV; e += 4) *reinterpret_cast<emc2_fvec<4>*>(to + id * PV + e) = emc2_fvec<4>{f[e], f[e + 1], f[e + 2], f[e + 3]};
      }
    }
  }
};
// A row's step, at the row's begin in one of the forms of a loop over rows: what is made of it, and the reads of LDS behind it, do not move in front of this
// (all rows' decays and reads at once, or those that several forms have in common in front of all of them, would take all registers).
template <int FORM> __device__ __forceinline__ float a_row(float d) {
  asm volatile("; row %1" : "+v"(d) : "i"(FORM) : "memory");
  return d;
}
// A value that a row ends with: it is made before the next row begins, and does not wait, with all that it needs, until it is used.
__device__ __forceinline__ void row_ends_with(float& v) { asm volatile("" : "+v"(v)); }
template <int S> __device__ __forceinline__ void from_lds(const float* p, float (&v)[S]) {
#pragma unroll
  for (int i = 0; i < S; i += 4) {
    const emc2_fvec<4> q = *reinterpret_cast<const emc2_fvec<4>*>(p + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[i + e] = q[e];
  }
}

// Whether any of the values is infinite.  (A NaN may be overlooked.)
template <int R> __device__ __forceinline__ bool any_infinite(const float (&v)[R]) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < R; ++i) m = fmaxf(m, fabsf(v[i]));
  return __any(m > 3.402823466e38f);
}

// Values of one channel in a lane's rows of a batch; rows that are none have the last one's.
template <typename T, int P> struct Column {
  T v[Slots<P>::R];
  __device__ __forceinline__ void fetch(const Line<const T>& l, int32_t bytes, int q, int32_t r0, int32_t n) {
    const Rows<P> rows(l, bytes, q, r0, n);
#pragma unroll
    for (int j = 0; j < Slots<P>::R; ++j) v[j] = rows.template load<T>(j, q);
  }
};

// A times log2(e): the rows' decays are powers of two.  States that are none have any value below 0: their decays end with an infinite step as all others do (0 would make
// them NaN), so that they stay 0.
template <int S, typename Lanes> __device__ __forceinline__ void decays(const ScanArgs& a, const Lanes& t, float (&a2)[S]) {
  t.load(a, a.a, a2);
#pragma unroll
  for (int s = 0; s < S; ++s) a2[s] = s < t.there ? a2[s] * kLog2e : -1.0f;
}

// `h` behind a run of rows that multiply a state by exp(A s) and add `t`; s < 0: a sequence begins in the run, and nothing from before it is left.
template <int S> __device__ __forceinline__ void through(const float (&a2)[S], float s, const float (&t)[S], float (&h)[S]) {
#pragma unroll
  for (int i = 0; i < S; ++i) h[i] = s < 0.0f ? t[i] : __builtin_fmaf(__builtin_amdgcn_exp2f(a2[i] * s), h[i], t[i]);
}

// Spans that n rows make.
__device__ __forceinline__ int32_t spans_of(const ScanArgs& a, int32_t n) {
  const int32_t chunks = (int32_t)(((int64_t)n + a.chunk - 1) / a.chunk);
  return (chunks + kChunkWaves - 1) / kChunkWaves;
}

// The state that enters chunk `k` (direction 0), or the flow that enters it from later rows (1): what enters its span, behind the chunks of the span before it.
template <int DIR, int S, typename Lanes>
__device__ __forceinline__ void entering(const ScanArgs& a, const Lanes& t, const float (&a2)[S], int32_t k, int32_t spans, float (&h)[S]) {
  float v[S];
  t.load(a, a.chunk_h[DIR] + (int64_t)k * a.channels * a.states, v);
  const float s = t.in ? a.chunk_s[DIR][(int64_t)k * a.channels + t.channel] : 0.0f;
  if (spans > 1) t.load(a, a.enter[DIR] + (int64_t)(k / kChunkWaves) * a.channels * a.states, h);
  else {
#pragma unroll
    for (int i = 0; i < S; ++i) h[i] = 0.0f;
  }
  through<S>(a2, s, v, h);
}

// Sequences without rows hand their states on; blocks of their own, a sequence at a time.
__device__ __forceinline__ void hand_on(const ScanArgs& a, const Walk& w, const float* from, float* to) {
  const int64_t size = (int64_t)a.channels * a.states, step = (int64_t)(gridDim.x - a.row_blocks) * gridDim.y;
  for (int64_t j = (int64_t)(blockIdx.x - a.row_blocks) * gridDim.y + blockIdx.y; j < a.n_seq; j += step) {
    if (w.start((int32_t)j + 1) > w.start((int32_t)j)) continue;
    const int64_t at = w.number((int32_t)j) * size;
    for (int64_t i = threadIdx.x; i < size; i += blockDim.x) to[at + i] = from ? from[at + i] : 0.0f;
  }
}

inline bool rows_ok(const void* p, int64_t pitch, int32_t width, size_t size, bool optional) {
  return emc2_rows_ok(p, pitch, width, size, optional) && (!p || pitch <= kMaxPitch);
}
template <typename F> void with_type(emc2_dtype dtype, F&& f) {
  if (dtype == EMC2_F32) f(float());
  else if (dtype == EMC2_F16) f(_Float16());
  else f(__bf16());
}
template <bool V> struct Flag { static constexpr bool value = V; };
typedef Flag<true> Yes;
typedef Flag<false> No;
template <int S, int P> struct Form { static constexpr int s = S, p = P; };

}  // namespace

// Lanes a channel that walk long lists (host), and so states a lane.  Fewer states a lane are a shorter row, but more lanes repeat what belongs to the channel: it is best
// while the chip is not full (128 channels by 16 states in bf16, forward and gradients: 2000 rows 26 and 40 us with one lane, 20 and 32 with four; 20,000 rows 50 and 97,
// 43 and 88; 80,000 rows 90 and 242, 109 and 272) and wherever lanes would be idle otherwise (100,000 rows of 16 channels 75 and 131 us with one lane, 36 and 79 with four).
constexpr int64_t kFewWaveRows = 160000;
static inline int32_t emc2_scan_lanes(int64_t capacity, int32_t channels, int32_t states) {
  const int32_t fewest = states <= 16 ? 1 : states <= 32 ? 2 : 4, most = states <= 4 ? 1 : states <= 8 ? 2 : 4;
  constexpr int kCost[3] = {16, 10, 7};  // of a wave's row, with the fewest lanes and with twice and four times as many
  int32_t best = fewest;
  int64_t least = -1;
  for (int32_t lanes = fewest, i = 0; lanes <= most; lanes *= 2, ++i) {
    const int64_t slices = emc2_div_up((int64_t)channels * lanes, 64);
    if (least < 0 || slices * kCost[i] < least) best = lanes, least = slices * kCost[i];
    else if (capacity * slices <= kFewWaveRows) best = lanes;
  }
  return best;
}

// How a call is cut (host): by the waves that a chunk's channels fill (100,000 rows of 128 channels by 32 states, gradients 556 us; cut as for 16 states 603).
struct emc2_scan_plan {
  int32_t lanes;                         // a channel's
  int32_t chunk, chunks, spans;          // rows of a chunk; chunks and spans of the capacity
  int64_t most;                          // chunks that no call of up to that many rows exceeds
};
static inline emc2_scan_plan emc2_plan_scan(int64_t capacity, int32_t channels, int32_t states, bool grad) {
  emc2_scan_plan p;
  p.lanes = emc2_scan_lanes(capacity, channels, states);
  const int64_t slices = emc2_div_up((int64_t)channels * p.lanes, 64), all = grad ? kMaxChunksGrad : kMaxChunks;
  const int64_t room = slices < all ? all / slices : 1, few = slices < kFewChunks ? kFewChunks / slices : 1;
  const int64_t per = emc2_div_up(capacity, room), least = capacity <= few * kBatch ? kBatch : 2 * kBatch;
  const int64_t eights = emc2_div_up(capacity, kBatch), sixteens = emc2_div_up(eights, 2);
  p.chunk = (int32_t)(per < least ? least : emc2_div_up(per, kBatch) * kBatch);
  p.chunks = (int32_t)emc2_div_up(capacity, p.chunk);
  p.spans = (int32_t)emc2_div_up(p.chunks, kChunkWaves);
  p.most = eights < few ? eights : sixteens < few ? few : sixteens < room ? sixteens : room;
  return p;
}
// Totals of chunks and spans in one direction, and what enters the spans: floats.
static inline int64_t emc2_scan_totals_size(int64_t chunks, int32_t channels, int32_t states) {
  const int64_t spans = emc2_div_up(chunks, kChunkWaves);
  return ((chunks + spans) * (states + 1) + spans * states) * channels;
}
static inline float* emc2_place_totals(ScanArgs& a, int dir, float* at, const emc2_scan_plan& p) {
  const int64_t c = a.channels, cn = c * a.states;
  a.chunk_h[dir] = at, at += p.chunks * cn;
  a.span_h[dir] = at, at += p.spans * cn;
  a.enter[dir] = at, at += p.spans * cn;
  a.chunk_s[dir] = at, at += p.chunks * c;
  a.span_s[dir] = at, at += p.spans * c;
  return at;
}
// Launches the reduction of chunks and what enters the spans (selective_scan_totals.hip); `grad`: of both directions, with the states before every batch.
void emc2_scan_totals(const ScanArgs& a, emc2_dtype dtype, const emc2_scan_plan& p, bool grad, hipStream_t stream);
// Refuses what both directions refuse.
emc2_status emc2_scan_check(emc2_ctx* ctx, const char* what, emc2_dtype dtype, int64_t capacity, int32_t channels, int32_t states);
