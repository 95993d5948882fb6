// Gated linear recurrence along the rows of packed sequences, its gradients and its form for one row per sequence.
//   a_t = logistic(gate_t),  h_t = a_t h_{t-1} + (1 - a_t) x_t                 per channel, h_0 given or 0
//   u_t = dy_t + a_{t+1} u_{t+1} (+ dlast behind the last row);  dx_t = (1 - a_t) u_t,  dgate_t = u_t (h_{t-1} - x_t) a_t (1 - a_t),
//   dh_0 = a_1 u_1
// Row t maps the state h -> A h + B, and maps compose: any run of rows is one such pair per channel, so a long sequence is cut into
// blocks of rows that are worked on side by side.  A first launch reduces every block to its pair (k_recurrence_totals), the second
// composes the pairs of the blocks before its own into the state that enters it and then walks its rows (k_recurrence).  A sequence's
// first row begins a new map (A = -0, B = the given state), so sequences of any length share a block and none is padded.
// The gradients' u runs the other way with the same factors: the first launch reduces both directions at once, the second walks a block's
// tiles from the last to the first, with the state that enters every tile known from the first launch.
// A thread holds R consecutive rows of N neighbouring channels in registers; maps are composed over a wave's
// row groups by shuffles, over waves through LDS.  The order of composition is fixed: equal inputs give equal bits.  Maps and states are fp32.
// The map that begins a sequence drops what lies before it, whatever that holds: an infinity or NaN in one sequence never reaches another one.
// Its factor is -0, which no product of gates is: within a sequence a NaN or infinity travels on to the end, also where the gates' product is 0.
// Bound by memory, and close behind by the logistic function's two slow instructions an element.  Rows are read by both launches: 613 k x 64 f16 in
// eight sequences 99 us, 4.0 TB/s of both launches' bytes (the second finds much of its input in the last cache); 150 k x 96 fp32 in 9001 sequences 87 us,
// 3.3 TB/s; forward pass and gradients of 200 k x 128 bf16 176 us, 3.8 TB/s (over the same inputs again and again 88, 72 and 166).
#include "rows.h"

namespace {

constexpr int kMaxTiles = 32;        // tiles of a wave's run (forward) or of a block (gradients)
constexpr int kSlice = 64;           // channels of a block at most
// Waves of a block, rows of a thread and blocks aimed at: the second launch's blocks compose the maps of all others, which costs 1024 of them 20 us;
// blocks of eight waves need half as many.  us, 613 k x 64 f16 forward / 150 k x 96 fp32 in 9001 sequences forward / 200 k x 128 bf16 with gradients, over
// the same inputs each time: as below 88 / 72 / 166; 256 blocks 92 / 83 / 219, 1024 105 / 87 / 203; forward of 4 waves 98 / 80, of 2 rows 96 / 75, of
// 8 rows 98 / 96; gradients of 8 waves 194, of 2 rows 198, of 8 rows 202.
constexpr int kStepThreads = 256;    // of the kernels of one value or piece a thread
constexpr int kWavesForward = 8, kWavesGrad = 4, kRowsForward = 4, kRowsGrad = 4, kBlocks = 512;

struct Args {
  const void *x, *gate, *dy;
  const float *h0, *dlast;           // dlast: gradient of the last states
  const int32_t* offsets;
  void *y, *dgate;                   // y: forward: the states; backward: dx
  float *last, *dh0;
  float2 *block_f, *block_r, *tile_f;  // maps [blocks or tiles][width]; width: channels rounded up to whole slices
  int32_t* flags;
  int64_t ld_x, ld_gate, ld_dy, ld_y, ld_dgate;
  int32_t capacity, channels, width, n_seq, tiles, backwards;
  int32_t lane_shift;                // a row group is 2^lane_shift lanes wide
};

// Rows are counted in the direction of the scan: row r lies at r, or at n - 1 - r when the scan runs backwards; sequence j of the
// scan is then the caller's sequence n_seq - 1 - j.  Offsets are held within the rows, whatever they say.
__device__ __forceinline__ int32_t rows_of(const Args& a) {
  const int32_t n = a.offsets[a.n_seq];
  return n < 0 ? 0 : n < a.capacity ? n : a.capacity;
}
__device__ __forceinline__ int32_t start_of(const Args& a, int32_t n, int32_t j) {   // j in [0, n_seq]
  const int32_t o = a.offsets[a.backwards ? a.n_seq - j : j];
  const int32_t in = o < 0 ? 0 : o < n ? o : n;
  return a.backwards ? n - in : in;
}
__device__ __forceinline__ int32_t seq_of(const Args& a, int32_t j) { return a.backwards ? a.n_seq - 1 - j : j; }

// More rows than the buffers hold are left out and reported.
__device__ __forceinline__ void report(const Args& a) {
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0 && a.offsets[a.n_seq] > a.capacity) atomicOr(a.flags, EMC2_DEVFLAG_CAPACITY);
}

// The first j >= `j` whose sequence starts at `row` or later (n_seq if there is none), by the whole wave.
__device__ __forceinline__ int32_t seek(const Args& a, int32_t n, int32_t j, int32_t row, int lane) {
  while (true) {
    const bool below = j + lane < a.n_seq && start_of(a, n, j + lane) < row;
    const unsigned long long m = ~__ballot(below);
    if (m) return j + __builtin_ctzll(m);
    j += 64;
  }
}
__device__ __forceinline__ int32_t seek_far(const Args& a, int32_t n, int32_t row, int lane) {
  int32_t lo = 0, hi = a.n_seq;
  while (hi - lo > 64) {                 // the answer lies in [lo, hi]; every turn leaves at most a 64th of that
    const int32_t step = (hi - lo) / 64;
    const unsigned long long m = ~__ballot(start_of(a, n, lo + (lane + 1) * step - 1) < row);
    const int c = m ? __builtin_ctzll(m) : 64;
    if (c < 64) hi = lo + (c + 1) * step - 1;
    lo += c * step;
  }
  return seek(a, n, lo, row, lane);
}

// The first sequence from a tile's first row on, for tiles in falling order.
struct Falling {
  int32_t j = 0, next = -1, before = 0x7fffffff;           // its number and start; the start of the one before it
  __device__ __forceinline__ void move(const Args& a, int32_t n, int32_t row0, int lane) {
    if (before < row0) return;
    j = row0 > 0 ? seek_far(a, n, row0, lane) : 0;
    next = start_of(a, n, j);
    before = j > 0 ? start_of(a, n, j - 1) : -1;
  }
};

// Where sequences start and end within a wave's rows of a tile: per row the caller's number of the sequence that starts or ends there,
// or -1.  Returns false, and writes nothing, where none does (next: the first start at or after the rows' first, also the end of
// the sequence that runs there).
__device__ __forceinline__ bool mark(const Args& a, int32_t n, int32_t row0, int rows, int32_t& j, int32_t& next, int32_t* starts,
                                     int32_t* ends, int lane) {
  if (next < row0) {
    j = seek(a, n, j, row0, lane);
    next = start_of(a, n, j);
  }
  if (next > row0 + rows) return false;
  for (int i = lane; i < rows; i += 64) starts[i] = ends[i] = -1;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (lane == 0 && j > 0 && next > row0 && next <= row0 + rows) ends[next - 1 - row0] = seq_of(a, j - 1);
  for (int32_t k = j;; k += 64) {
    const int32_t s = k + lane;
    bool here = false;
    if (s < a.n_seq) {
      const int32_t p = start_of(a, n, s), q = start_of(a, n, s + 1);
      here = p >= row0 && p < row0 + rows;
      if (here && q > p) {
        starts[p - row0] = seq_of(a, s);
        if (q <= row0 + rows) ends[q - 1 - row0] = seq_of(a, s);
      }
    }
    if (!__any(here)) break;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  return true;
}

// A map h -> A h + B of N channels, and what it makes of a state.
template <int N> struct Map { emc2_fvec<N> A, B; };
constexpr float kBegins = -0.0f;     // A of a map that drops the state before it; gates are >= +0, and so are their products
__device__ __forceinline__ bool begins(float A) { return __float_as_uint(A) == 0x80000000u; }
__device__ __forceinline__ float apply(float A, float B, float h) { return begins(A) ? B : __builtin_fmaf(A, h, B); }
template <int N> __device__ __forceinline__ emc2_fvec<N> apply(const Map<N>& m, emc2_fvec<N> h) {
#pragma unroll
  for (int e = 0; e < N; ++e) h[e] = apply(m.A[e], m.B[e], h[e]);
  return h;
}
// `second` after `first`.  A second map that drops the state stays one, even if the first one's factor is NaN.
__device__ __forceinline__ float2 then(float2 first, float2 second) {
  return make_float2(begins(second.x) ? kBegins : first.x * second.x, apply(second.x, second.y, first.y));
}
template <int N> __device__ __forceinline__ Map<N> then(const Map<N>& first, const Map<N>& second) {
  Map<N> m;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const float2 q = then(make_float2(first.A[e], first.B[e]), make_float2(second.A[e], second.B[e]));
    m.A[e] = q.x, m.B[e] = q.y;
  }
  return m;
}
template <int N> __device__ __forceinline__ Map<N> nothing() { return {emc2_fvec<N>(1.0f), emc2_fvec<N>(0.0f)}; }
template <int N> __device__ __forceinline__ Map<N> from_below(const Map<N>& m, int d) {
  Map<N> o;
#pragma unroll
  for (int e = 0; e < N; ++e) o.A[e] = __shfl_up(m.A[e], d, 64), o.B[e] = __shfl_up(m.B[e], d, 64);
  return o;
}
template <int N> __device__ __forceinline__ Map<N> from_above(const Map<N>& m, int d) {
  Map<N> o;
#pragma unroll
  for (int e = 0; e < N; ++e) o.A[e] = __shfl_down(m.A[e], d, 64), o.B[e] = __shfl_down(m.B[e], d, 64);
  return o;
}

// What a thread is: its wave, its row group within the wave, its channels.
struct Place {
  int lane, wave, group, groups, column;   // column: the first of its channels within the slice
  int32_t channel;                         // and of all
  int twice;                               // a last piece that would pass the channels begins so many earlier: its first values are another's
  bool in;                                 // it has channels
};
template <int N> __device__ __forceinline__ Place place_of(const Args& a) {
  Place p;
  p.lane = threadIdx.x & 63;
  p.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  p.group = p.lane >> a.lane_shift;
  p.groups = 64 >> a.lane_shift;
  p.column = (p.lane & ((1 << a.lane_shift) - 1)) * N;
  p.channel = (int32_t)blockIdx.y * (N << a.lane_shift) + p.column;
  p.in = p.channel < a.channels;
  p.twice = p.in && p.channel + N > a.channels ? p.channel + N - a.channels : 0;
  p.channel -= p.twice;
  return p;
}

// A thread's own values of a row, to p.
template <int N, typename T> __device__ __forceinline__ void put(T* p, emc2_fvec<N> v, const Place& t) {
  if (N == 1 || t.twice == 0) return emc2_store<N>(p, v);
#pragma unroll
  for (int e = 1; e < N; ++e)
    if (e >= t.twice) p[e] = (T)v[e];
}

// R consecutive rows of a thread as they lie in memory; rows past the last and channels that are none read valid places.
template <typename T, int N, int R> struct Rows { emc2_vec<T, N> v[R]; };
template <typename T, int N, int R>
__device__ __forceinline__ Rows<T, N, R> fetch(const Args& a, const void* p, int64_t ld, int32_t n, int64_t row, const Place& t) {
  Rows<T, N, R> r;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int64_t k = row + i < n ? row + i : n - 1;
    r.v[i] = emc2_piece<N>((const T*)p + (a.backwards ? n - 1 - k : k) * ld + (t.in ? t.channel : 0));
  }
  return r;
}

// a and 1 - a of a gate's row
template <typename T, int N> __device__ __forceinline__ void open(emc2_vec<T, N> gate, emc2_fvec<N>& keep, emc2_fvec<N>& take) {
  const emc2_fvec<N> g = __builtin_convertvector(gate, emc2_fvec<N>);
#pragma unroll
  for (int e = 0; e < N; ++e) {
    float s, r;
    emc2_logistic<sizeof(T) == 4>(g[e], s, r);
    keep[e] = s, take[e] = r;
  }
}

template <int N> __device__ __forceinline__ emc2_fvec<N> state_or_zero(const float* p, const Args& a, int32_t seq, const Place& t) {
  return p && t.in ? emc2_load<N>(p + (int64_t)seq * a.channels + t.channel) : emc2_fvec<N>(0.0f);
}

// The map of a thread's rows, first to last, from their factors and offsets.
template <int N, int R>
__device__ __forceinline__ Map<N> run_forward(const Args& a, const emc2_fvec<N> (&keep)[R], const emc2_fvec<N> (&add)[R], bool marked,
                                              const int32_t* starts, const Place& t) {
  Map<N> m = nothing<N>();
  if (!marked) {
#pragma unroll
    for (int i = 0; i < R; ++i) m.A *= keep[i], m.B = keep[i] * m.B + add[i];
  } else {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int32_t s = starts[i];
      if (s >= 0) m = {emc2_fvec<N>(kBegins), state_or_zero<N>(a.h0, a, s, t)};
      m.A *= keep[i], m.B = keep[i] * m.B + add[i];
    }
  }
  return m;
}
// The map of what flows towards earlier rows (a_t u_t), last to first.
template <int N, int R>
__device__ __forceinline__ Map<N> run_backward(const Args& a, const emc2_fvec<N> (&keep)[R], const emc2_fvec<N> (&dy)[R], bool marked,
                                               const int32_t* ends, const Place& t) {
  Map<N> m = nothing<N>();
#pragma unroll
  for (int i = R - 1; i >= 0; --i) {
    if (marked) {
      const int32_t s = ends[i];
      if (s >= 0) m = {emc2_fvec<N>(kBegins), state_or_zero<N>(a.dlast, a, s, t)};
    }
    m.A *= keep[i], m.B = keep[i] * (dy[i] + m.B);
  }
  return m;
}

// Rows past the last change nothing: a = 1, nothing added.
template <int N, int R> __device__ __forceinline__ void blank(int32_t n, int32_t row, emc2_fvec<N> (&keep)[R], emc2_fvec<N> (&add)[R]) {
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (row + i >= n) keep[i] = 1.0f, add[i] = 0.0f;
}

// First launch of the forward pass: the maps of every wave's run of rows and of every block.  A wave walks `tiles` tiles, a tile being R rows in every
// row group of the wave, from the last to the first: the second launch, whose blocks lie on the same XCDs, begins with what was read
// last.  The next tile's rows are on their way while one is worked on.
template <typename T, int N, int R>
__global__ void __launch_bounds__(64 * kWavesForward) k_recurrence_totals(const Args a) {
  constexpr int kWaves = kWavesForward;
  __shared__ float2 total[kWaves][kSlice];
  __shared__ int32_t starts[kWaves][64 * R], ends[kWaves][64 * R];
  const Place t = place_of<N>(a);
  const int32_t n = rows_of(a), rows = t.groups * R;
  report(a);
  const int64_t first = ((int64_t)blockIdx.x * kWaves + t.wave) * a.tiles * rows;
  if ((int64_t)blockIdx.x * kWaves * a.tiles * rows >= n) return;
  const int slice = N << a.lane_shift;
  Map<N> run = nothing<N>();
  if (first < n) {
    const int32_t here = (int32_t)((n - first + rows - 1) / rows), tiles = here < a.tiles ? here : a.tiles;
    const int64_t mine = first + (int64_t)(tiles - 1) * rows + t.group * R;
    Rows<T, N, R> x = fetch<T, N, R>(a, a.x, a.ld_x, n, mine, t), g = fetch<T, N, R>(a, a.gate, a.ld_gate, n, mine, t);
    Falling at;
    for (int32_t k = tiles - 1; k >= 0; --k) {
      const int64_t row0 = first + (int64_t)k * rows;
      const int32_t row = (int32_t)row0 + t.group * R;
      emc2_fvec<N> keep[R], add[R];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        emc2_fvec<N> take;
        open<T, N>(g.v[i], keep[i], take);
        add[i] = take * __builtin_convertvector(x.v[i], emc2_fvec<N>);
      }
      if (k > 0) {
        x = fetch<T, N, R>(a, a.x, a.ld_x, n, (int64_t)row - rows, t);
        g = fetch<T, N, R>(a, a.gate, a.ld_gate, n, (int64_t)row - rows, t);
      }
      at.move(a, n, (int32_t)row0, t.lane);
      const bool marked = mark(a, n, (int32_t)row0, rows, at.j, at.next, starts[t.wave], ends[t.wave], t.lane);
      if (row0 + rows > n) blank<N, R>(n, row, keep, add);
      Map<N> m = run_forward<N, R>(a, keep, add, marked, &starts[t.wave][t.group * R], t);
      for (int dist = 1 << a.lane_shift; dist < 64; dist <<= 1) m = then<N>(m, from_above<N>(m, dist));
      run = then<N>(m, run);                               // (of the first row group; the others' are not used)
    }
  }
  if (t.group == 0) {
#pragma unroll
    for (int e = 0; e < N; ++e) total[t.wave][t.column + e] = make_float2(run.A[e], run.B[e]);
  }
  __syncthreads();
  if ((int)threadIdx.x < slice) {
    const int64_t place = (int64_t)blockIdx.y * slice + threadIdx.x;
    float2 block = make_float2(1.0f, 0.0f);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float2 m = total[w][threadIdx.x];
      a.tile_f[((int64_t)blockIdx.x * kWaves + w) * a.width + place] = m;
      block = then(block, m);
    }
    a.block_f[(int64_t)blockIdx.x * a.width + place] = block;
  }
}

// First launch of the gradients: the maps of every block in both directions, and the forward one of every tile.  Block (b, slice) has `tiles` tiles
// of rows, a tile being R rows in every row group of the block.
template <typename T, int N, int R>
__global__ void __launch_bounds__(64 * kWavesGrad) k_recurrence_grad_totals(const Args a) {
  constexpr int kWaves = kWavesGrad;
  __shared__ float2 total[2][2][kWaves][kSlice];
  __shared__ int32_t starts[kWaves][64 * R], ends[kWaves][64 * R];
  const Place t = place_of<N>(a);
  const int32_t n = rows_of(a);
  report(a);
  const int32_t tile_rows = kWaves * t.groups * R;
  const int64_t first = (int64_t)blockIdx.x * a.tiles * tile_rows;
  if (first >= n) return;
  const int slice = N << a.lane_shift;
  const int64_t mine = first + (t.wave * t.groups + t.group) * R;
  Rows<T, N, R> x = fetch<T, N, R>(a, a.x, a.ld_x, n, mine, t), g = fetch<T, N, R>(a, a.gate, a.ld_gate, n, mine, t),
                d = fetch<T, N, R>(a, a.dy, a.ld_dy, n, mine, t);
  int32_t j = 0, next = -1;
  if (first > 0) j = seek_far(a, n, (int32_t)first, t.lane);
  float2 block_f = make_float2(1.0f, 0.0f), block_r = block_f;
  for (int32_t k = 0; k < a.tiles; ++k) {
    const int64_t row0 = first + (int64_t)k * tile_rows + t.wave * t.groups * R;
    if (first + (int64_t)k * tile_rows >= n) break;
    const int32_t row = (int32_t)row0 + t.group * R;
    Map<N> f = nothing<N>(), r = nothing<N>();
    emc2_fvec<N> keep[R], add[R], dy[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      emc2_fvec<N> take;
      open<T, N>(g.v[i], keep[i], take);
      add[i] = take * __builtin_convertvector(x.v[i], emc2_fvec<N>);
      dy[i] = __builtin_convertvector(d.v[i], emc2_fvec<N>);
    }
    if (k + 1 < a.tiles && first + (int64_t)(k + 1) * tile_rows < n) {
      x = fetch<T, N, R>(a, a.x, a.ld_x, n, (int64_t)row + tile_rows, t);
      g = fetch<T, N, R>(a, a.gate, a.ld_gate, n, (int64_t)row + tile_rows, t);
      d = fetch<T, N, R>(a, a.dy, a.ld_dy, n, (int64_t)row + tile_rows, t);
    }
    if (row0 < n) {
      const bool marked = mark(a, n, (int32_t)row0, t.groups * R, j, next, starts[t.wave], ends[t.wave], t.lane);
      if (row0 + t.groups * R > n) blank<N, R>(n, row, keep, add), blank<N, R>(n, row, keep, dy);
      f = run_forward<N, R>(a, keep, add, marked, &starts[t.wave][t.group * R], t);
      r = run_backward<N, R>(a, keep, dy, marked, &ends[t.wave][t.group * R], t);
      for (int dist = 1 << a.lane_shift; dist < 64; dist <<= 1) {     // the wave's first row group ends with all of them
        f = then<N>(f, from_above<N>(f, dist));
        r = then<N>(from_above<N>(r, dist), r);
      }
    }
    if (t.group == 0) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        total[k & 1][0][t.wave][t.column + e] = make_float2(f.A[e], f.B[e]);
        total[k & 1][1][t.wave][t.column + e] = make_float2(r.A[e], r.B[e]);
      }
    }
    __syncthreads();
    if ((int)threadIdx.x < slice) {
      const int c = threadIdx.x;
      float2 tile = total[k & 1][0][0][c];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) tile = then(tile, total[k & 1][0][w][c]);
      block_f = then(block_f, tile);
      a.tile_f[((int64_t)blockIdx.x * a.tiles + k) * a.width + blockIdx.y * slice + c] = tile;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) block_r = then(total[k & 1][1][w][c], block_r);   // of the flow towards earlier rows, the later rows come first
    }
  }
  if ((int)threadIdx.x < slice) {
    a.block_f[(int64_t)blockIdx.x * a.width + blockIdx.y * slice + threadIdx.x] = block_f;
    a.block_r[(int64_t)blockIdx.x * a.width + blockIdx.y * slice + threadIdx.x] = block_r;
  }
}

// What a run of blocks makes of a state of zeros, per channel of the slice, into enter[]: blocks [lo, hi) in rising order, or (FALLING) from
// hi - 1 down to lo.  The block's threads take a part of the run each.  Ends with a barrier.
template <bool FALLING, int WAVES>
__device__ __forceinline__ void compose(const float2* __restrict__ maps, int32_t width, int32_t column, int slice, int32_t lo, int32_t hi,
                                        float2* part, float* enter) {
  const int c = threadIdx.x & (slice - 1), seg = threadIdx.x / slice, segs = 64 * WAVES / slice;
  const int32_t count = hi > lo ? hi - lo : 0, per = (count + segs - 1) / segs;
  const int32_t from = seg * per < count ? seg * per : count, to = from + per < count ? from + per : count;
  float2 all = make_float2(1.0f, 0.0f);
  constexpr int kAtOnce = 16;
  for (int32_t i = from; i < to; i += kAtOnce) {
    float2 m[kAtOnce];
#pragma unroll
    for (int q = 0; q < kAtOnce; ++q) {
      const int32_t k = i + q < to ? i + q : to - 1;
      m[q] = maps[(int64_t)(FALLING ? hi - 1 - k : lo + k) * width + column + c];
    }
#pragma unroll
    for (int q = 0; q < kAtOnce; ++q)
      if (i + q < to) all = then(all, m[q]);
  }
  part[threadIdx.x] = all;
  __syncthreads();
  if (seg == 0) {
    float h = 0.0f;
    for (int s = 0; s < segs; ++s) h = apply(part[s * slice + c].x, part[s * slice + c].y, h);
    enter[c] = h;
  }
  __syncthreads();
}

// Sequences without rows leave the state they were given.  The blocks and their waves share the sequences out; a wave looks at up to 64 at once and, where
// any is empty, copies their states of the slice's channels, eight loads under way.
__device__ __forceinline__ void pass_empty(const Args& a, int32_t n, const float* from, float* to, int slice) {
  if (!to) return;
  const int32_t per = (int32_t)(((int64_t)a.n_seq + gridDim.x - 1) / gridDim.x), waves = blockDim.x >> 6;
  const int32_t even = (per + waves - 1) / waves, each = even < 64 ? even : 64;
  const int64_t lo = (int64_t)blockIdx.x * per, hi = lo + per < a.n_seq ? lo + per : a.n_seq;
  const int lane = threadIdx.x & 63, shift = __builtin_ctz(slice);
  for (int64_t j0 = lo + (threadIdx.x >> 6) * each; j0 < hi; j0 += waves * each) {
    const int64_t j = j0 + lane;
    const unsigned long long empty = __ballot(lane < each && j < hi && start_of(a, n, (int32_t)j + 1) <= start_of(a, n, (int32_t)j));
    if (!empty) continue;
    for (int i0 = 0; i0 * 64 < each * slice; i0 += 8) {
      float v[8];
      int64_t at[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int q = (i0 + i) * 64 + lane, m = q >> shift;                // sequence of the wave's and, below it, channel of the slice
        const int32_t c = (int32_t)blockIdx.y * slice + (q & (slice - 1));
        const bool here = m < each && (empty >> (m & 63) & 1) && c < a.channels;
        at[i] = here ? (int64_t)seq_of(a, (int32_t)(j0 + m)) * a.channels + c : -1;
        v[i] = here && from ? from[at[i]] : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (at[i] >= 0) to[at[i]] = v[i];
    }
  }
}

// Second launch: the rows.  A block of one wave (calls of a few tiles) needs no first launch.
template <typename T, int N, int R>
__global__ void __launch_bounds__(64 * kWavesForward) k_recurrence(const Args a) {
  constexpr int kWaves = kWavesForward;
  __shared__ int32_t starts[kWaves][64 * R], ends[kWaves][64 * R];
  __shared__ float2 part[64 * kWaves];
  __shared__ float enter[kSlice];
  const Place t = place_of<N>(a);
  const int32_t n = rows_of(a), rows = t.groups * R, waves = blockDim.x >> 6;
  if (waves == 1) report(a);
  const int slice = N << a.lane_shift;
  const int64_t first = ((int64_t)blockIdx.x * waves + t.wave) * a.tiles * rows;
  if ((int64_t)blockIdx.x * waves * a.tiles * rows >= n) return pass_empty(a, n, a.h0, a.last, slice);
  const int64_t mine = first + t.group * R;
  Rows<T, N, R> x = fetch<T, N, R>(a, a.x, a.ld_x, n, mine, t), g = fetch<T, N, R>(a, a.gate, a.ld_gate, n, mine, t);
  emc2_fvec<N> h = emc2_fvec<N>(0.0f);                     // the state that enters the tile
  int32_t j = 0, next = -1;
  if (first > 0 && first < n) j = seek_far(a, n, (int32_t)first, t.lane);
  if (waves > 1) {
    compose<false, kWaves>(a.block_f, a.width, blockIdx.y * slice, slice, 0, blockIdx.x, part, enter);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      h[e] = enter[t.column + e];
      float2 m[kWaves - 1];
#pragma unroll
      for (int w = 0; w < kWaves - 1; ++w) m[w] = a.tile_f[((int64_t)blockIdx.x * kWaves + w) * a.width + blockIdx.y * slice + t.column + e];
#pragma unroll
      for (int w = 0; w < kWaves - 1; ++w)
        if (w < t.wave) h[e] = apply(m[w].x, m[w].y, h[e]);
    }
  }
  for (int32_t k = 0; k < a.tiles; ++k) {
    const int64_t row0 = first + (int64_t)k * rows;
    if (row0 >= n) break;
    const int32_t row = (int32_t)row0 + t.group * R;
    emc2_fvec<N> keep[R], add[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      emc2_fvec<N> take;
      open<T, N>(g.v[i], keep[i], take);
      add[i] = take * __builtin_convertvector(x.v[i], emc2_fvec<N>);
    }
    if (k + 1 < a.tiles && row0 + rows < n) {
      x = fetch<T, N, R>(a, a.x, a.ld_x, n, (int64_t)row + rows, t);
      g = fetch<T, N, R>(a, a.gate, a.ld_gate, n, (int64_t)row + rows, t);
    }
    const bool marked = mark(a, n, (int32_t)row0, rows, j, next, starts[t.wave], ends[t.wave], t.lane);
    if (row0 + rows > n) blank<N, R>(n, row, keep, add);
    Map<N> m = run_forward<N, R>(a, keep, add, marked, &starts[t.wave][t.group * R], t);
    // maps of all rows of the wave up to the group's last; then of those before its first
    for (int dist = 1 << a.lane_shift; dist < 64; dist <<= 1) {
      const Map<N> before = from_below<N>(m, dist);
      if (t.lane >= dist) m = then<N>(before, m);
    }
    m = from_below<N>(m, 1 << a.lane_shift);
    if (t.group > 0) h = apply<N>(m, h);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int32_t r = row + i;
      if (marked && starts[t.wave][t.group * R + i] >= 0) h = state_or_zero<N>(a.h0, a, starts[t.wave][t.group * R + i], t);
      h = keep[i] * h + add[i];
      if (r < n && t.in) {
        put<N>((T*)a.y + (int64_t)(a.backwards ? n - 1 - r : r) * a.ld_y + t.channel, h, t);
        if (marked && a.last && ends[t.wave][t.group * R + i] >= 0)
          put<N>(a.last + (int64_t)ends[t.wave][t.group * R + i] * a.channels + t.channel, h, t);
      }
    }
#pragma unroll
    for (int e = 0; e < N; ++e) h[e] = __shfl(h[e], t.lane | (64 - (1 << a.lane_shift)), 64);   // the last row group's: enters the next tile
  }
  pass_empty(a, n, a.h0, a.last, slice);                   // (last: it waits for what it loads)
}

template <typename T, int N, int R>
__global__ void __launch_bounds__(64 * kWavesGrad) k_recurrence_grad(const Args a) {
  constexpr int kWaves = kWavesGrad;
  __shared__ float2 total[2][2][kWaves][kSlice];
  __shared__ int32_t starts[kWaves][64 * R], ends[kWaves][64 * R];
  __shared__ float2 part[64 * kWaves];
  __shared__ float enter[kMaxTiles][kSlice], enter_r[kSlice];
  const Place t = place_of<N>(a);
  const int32_t n = rows_of(a);
  report(a);
  const int slice = N << a.lane_shift;
  const int32_t tile_rows = kWaves * t.groups * R, block_rows = a.tiles * tile_rows;
  const int64_t first = (int64_t)blockIdx.x * block_rows;
  pass_empty(a, n, a.dlast, a.dh0, slice);
  if (first >= n) return;
  const int32_t here = (int32_t)((n - first + tile_rows - 1) / tile_rows), tiles = here < a.tiles ? here : a.tiles;
  const int64_t mine = first + (int64_t)(tiles - 1) * tile_rows + (t.wave * t.groups + t.group) * R;
  Rows<T, N, R> xv = fetch<T, N, R>(a, a.x, a.ld_x, n, mine, t), g = fetch<T, N, R>(a, a.gate, a.ld_gate, n, mine, t),
                d = fetch<T, N, R>(a, a.dy, a.ld_dy, n, mine, t);
  Falling at;
  emc2_fvec<N> flow = emc2_fvec<N>(0.0f);                  // what flows into the tile from later rows
  const int32_t blocks = (int32_t)(((int64_t)n + block_rows - 1) / block_rows);
  if (blocks > 1 || tiles > 1) {
    compose<false, kWaves>(a.block_f, a.width, blockIdx.y * slice, slice, 0, blockIdx.x, part, enter[0]);
    compose<true, kWaves>(a.block_r, a.width, blockIdx.y * slice, slice, blockIdx.x + 1, blocks, part, enter_r);
    if ((int)threadIdx.x < slice) {
      float h = enter[0][threadIdx.x];
      for (int32_t k = 1; k < tiles; ++k) {
        const float2 q = a.tile_f[((int64_t)blockIdx.x * a.tiles + k - 1) * a.width + blockIdx.y * slice + threadIdx.x];
        enter[k][threadIdx.x] = h = apply(q.x, q.y, h);
      }
    }
#pragma unroll
    for (int e = 0; e < N; ++e) flow[e] = enter_r[t.column + e];
  } else if ((int)threadIdx.x < slice) {
    enter[0][threadIdx.x] = 0.0f;
  }
  for (int32_t k = tiles - 1; k >= 0; --k) {
    const int64_t row0 = first + (int64_t)k * tile_rows + t.wave * t.groups * R;
    const int32_t row = (int32_t)row0 + t.group * R;
    emc2_fvec<N> keep[R], take[R], x[R], dy[R];
    Map<N> f = nothing<N>(), r = nothing<N>();
    bool marked = false;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      open<T, N>(g.v[i], keep[i], take[i]);
      x[i] = __builtin_convertvector(xv.v[i], emc2_fvec<N>);
      dy[i] = __builtin_convertvector(d.v[i], emc2_fvec<N>);
    }
    if (k > 0) {
      xv = fetch<T, N, R>(a, a.x, a.ld_x, n, (int64_t)row - tile_rows, t);
      g = fetch<T, N, R>(a, a.gate, a.ld_gate, n, (int64_t)row - tile_rows, t);
      d = fetch<T, N, R>(a, a.dy, a.ld_dy, n, (int64_t)row - tile_rows, t);
    }
    if (row0 < n) {
      at.move(a, n, (int32_t)row0, t.lane);
      marked = mark(a, n, (int32_t)row0, t.groups * R, at.j, at.next, starts[t.wave], ends[t.wave], t.lane);
      emc2_fvec<N> add[R];
#pragma unroll
      for (int i = 0; i < R; ++i) add[i] = take[i] * x[i];
      if (row0 + t.groups * R > n) blank<N, R>(n, row, keep, add), blank<N, R>(n, row, keep, dy);
      f = run_forward<N, R>(a, keep, add, marked, &starts[t.wave][t.group * R], t);
      r = run_backward<N, R>(a, keep, dy, marked, &ends[t.wave][t.group * R], t);
    }
    for (int dist = 1 << a.lane_shift; dist < 64; dist <<= 1) {
      const Map<N> below = from_below<N>(f, dist), above = from_above<N>(r, dist);
      if (t.lane >= dist) f = then<N>(below, f);
      if (t.lane + dist < 64) r = then<N>(above, r);
    }
    if (t.group == t.groups - 1) {
#pragma unroll
      for (int e = 0; e < N; ++e) total[k & 1][0][t.wave][t.column + e] = make_float2(f.A[e], f.B[e]);
    }
    if (t.group == 0) {
#pragma unroll
      for (int e = 0; e < N; ++e) total[k & 1][1][t.wave][t.column + e] = make_float2(r.A[e], r.B[e]);
    }
    f = from_below<N>(f, 1 << a.lane_shift), r = from_above<N>(r, 1 << a.lane_shift);
    if (t.group == 0) f = nothing<N>();
    if (t.group == t.groups - 1) r = nothing<N>();
    __syncthreads();
    emc2_fvec<N> h, u = flow;                              // what enters the thread's rows from either side
#pragma unroll
    for (int e = 0; e < N; ++e) h[e] = enter[k][t.column + e];
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
      if (w < t.wave) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float2 q = total[k & 1][0][w][t.column + e];
          h[e] = apply(q.x, q.y, h[e]);
        }
      }
#pragma unroll
    for (int w = kWaves - 1; w >= 0; --w) {
      if (w == t.wave) u = flow;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float2 q = total[k & 1][1][w][t.column + e];
        flow[e] = apply(q.x, q.y, flow[e]);
      }
    }
    if (row0 < n) {
      h = apply<N>(f, h), u = apply<N>(r, u);
      emc2_fvec<N> prev[R];                                // h_{t-1}
#pragma unroll
      for (int i = 0; i < R; ++i) {
        if (marked && starts[t.wave][t.group * R + i] >= 0) h = state_or_zero<N>(a.h0, a, starts[t.wave][t.group * R + i], t);
        prev[i] = h;
        h = keep[i] * h + take[i] * x[i];
      }
#pragma unroll
      for (int i = R - 1; i >= 0; --i) {
        const int32_t at = row + i;
        if (marked && ends[t.wave][t.group * R + i] >= 0) u = state_or_zero<N>(a.dlast, a, ends[t.wave][t.group * R + i], t);
        const emc2_fvec<N> du = dy[i] + u;
        if (at < n) u = keep[i] * du;
        if (at < n && t.in) {
          const int64_t place = a.backwards ? n - 1 - at : at;
          put<N>((T*)a.y + place * a.ld_y + t.channel, take[i] * du, t);
          put<N>((T*)a.dgate + place * a.ld_dgate + t.channel, (prev[i] - x[i]) * (keep[i] * take[i]) * du, t);
          if (marked && a.dh0 && starts[t.wave][t.group * R + i] >= 0)
            put<N>(a.dh0 + (int64_t)starts[t.wave][t.group * R + i] * a.channels + t.channel, u, t);
        }
      }
    }
  }
}

// One row per sequence: N channels of a row a thread.
template <typename T, int N>
__global__ void __launch_bounds__(kStepThreads) k_recurrence_step(const T* x, int64_t ld_x, const T* gate, int64_t ld_gate, const float* h_in,
                                                                  float* h_out, T* y, int64_t ld_y, int64_t rows, int32_t channels) {
  const int32_t pieces = (channels + N - 1) / N;
  const int64_t i = emc2_block() * kStepThreads + threadIdx.x;
  if (i >= rows * pieces) return;
  const int64_t row = i / pieces;
  const int32_t c = (int32_t)(i - row * pieces) * N;
  if (c + N <= channels) {
    emc2_fvec<N> keep, take;
    open<T, N>(emc2_piece<N>(gate + row * ld_gate + c), keep, take);
    const emc2_fvec<N> h = keep * emc2_load<N>(h_in + row * channels + c) + take * emc2_load<N>(x + row * ld_x + c);
    emc2_store<N>(h_out + row * channels + c, h);
    emc2_store<N>(y + row * ld_y + c, h);
  } else {                                                 // the row's last, incomplete piece: states may be in place, so value by value
    for (int32_t k = c; k < channels; ++k) {
      float keep, take;
      emc2_logistic<sizeof(T) == 4>((float)gate[row * ld_gate + k], keep, take);
      const float h = keep * h_in[row * channels + k] + take * (float)x[row * ld_x + k];
      h_out[row * channels + k] = h;
      y[row * ld_y + k] = (T)h;
    }
  }
}

// How a call is cut: row groups, tiles a block, blocks, and the pieces of the work buffer.
struct Plan {
  int n, lane_shift, slices;
  int32_t tiles, blocks, width;
  bool totals;                       // a first launch is needed
  int64_t bytes, most;               // of scratch: what the call takes, and what no call of up to that many rows takes more than
};
Plan plan_of(emc2_dtype dtype, int64_t capacity, int32_t channels, bool grad) {
  Plan p = {};
  p.n = channels >= 4 ? 4 : 1;       // pieces of four values, wherever they lie
  const int pieces = (channels + p.n - 1) / p.n, most = dtype == EMC2_F32 ? 3 : 4;     // row groups of 128 bytes at most
  while (p.lane_shift < most && (1 << p.lane_shift) < pieces) ++p.lane_shift;
  const int slice = p.n << p.lane_shift, groups = 64 >> p.lane_shift;
  p.slices = (channels + slice - 1) / slice;
  p.width = p.slices * slice;
  // A call of a few tiles is one launch: the forward pass's of one wave, which walks them, the gradients' of one block and one tile.
  const int64_t small = emc2_div_up(capacity, grad ? kWavesGrad * groups * kRowsGrad : groups * kRowsForward);
  if (small <= (grad ? 1 : 4)) {
    p.tiles = small < 1 ? 1 : (int32_t)small, p.blocks = 1;
    return p;
  }
  // Others have about 512 blocks, two for every CU, each with a whole number of tiles for every wave.
  const int64_t tiles = emc2_div_up(capacity, groups * (grad ? kWavesGrad * kRowsGrad : kWavesForward * kRowsForward));
  const int64_t aim = kBlocks / p.slices > 1 ? kBlocks / p.slices : 1, per = emc2_div_up(tiles, aim);
  p.tiles = (int32_t)(per < kMaxTiles ? per : kMaxTiles);
  p.blocks = (int32_t)emc2_div_up(tiles, p.tiles);
  p.totals = true;
  const int64_t line = p.width * (int64_t)sizeof(float2);
  p.bytes = p.blocks * line * (grad ? 2 + p.tiles : 1 + kWavesForward);
  // blocks may become fewer as rows become more; what bounds them does not
  const int64_t some = tiles < aim ? tiles : aim, full = emc2_div_up(tiles, kMaxTiles), blocks = some > full ? some : full;
  p.most = line * (grad ? 2 * blocks + tiles + p.tiles - 1 : (1 + kWavesForward) * blocks);
  return p;
}

// Blocks of the launch that walks the rows: where they are fewer than the CUs, more for the sequences' states that are only handed on (to: where),
// eight sequences each.  8 rows x 128 in 4096 sequences 788 us with one block, whose one wave copied row by row, 24 so; blocks beyond the CUs' number make
// 150 k x 96 fp32 in 9001 sequences 7 us slower.
int64_t blocks_with_states(const Plan& p, int32_t n_seq, const void* to) {
  const int64_t room = 256 / p.slices, some = to ? emc2_div_up(n_seq, 8) : 0, more = some < room ? some : room;
  return more > p.blocks ? more : p.blocks;
}

template <typename F> void with_type(emc2_dtype dtype, int n, F&& f) {
  const auto by_length = [&](auto type) {
    if (n == 4) f(type, emc2_fvec<4>());
    else f(type, emc2_fvec<1>());
  };
  if (dtype == EMC2_F32) by_length(float());
  else if (dtype == EMC2_F16) by_length(_Float16());
  else by_length(__bf16());
}
template <typename V> constexpr int kLength = sizeof(V) / sizeof(float);

__global__ void __launch_bounds__(kStepThreads) k_frame_offsets(const int4* __restrict__ coords, const int32_t* __restrict__ d_n, int64_t capacity,
                                                            int32_t n_batch, int32_t* __restrict__ offsets) {
  const int64_t b = (int64_t)blockIdx.x * kStepThreads + threadIdx.x;
  if (b > n_batch) return;
  int32_t lo = 0, hi = emc2_row_count(d_n, capacity);
  if (b == n_batch) lo = hi;                               // every row, also one whose frame id is out of range, belongs to some frame
  if (b == 0) hi = 0;
  while (lo < hi) {                                        // the first row of a frame >= b
    const int32_t mid = lo + (hi - lo) / 2;
    if (coords[mid].x < b) lo = mid + 1;
    else hi = mid;
  }
  offsets[b] = lo;
}

emc2_status check(emc2_ctx* ctx, const char* what, emc2_dtype dtype, int64_t capacity, int32_t channels, int32_t n_seq, const void* offsets) {
  if (!emc2_is_float(dtype)) return emc2_fail(ctx, EMC2_ERR_UNSUPPORTED, "%s: dtype must be F32, F16 or BF16", what);
  if (channels < 1 || channels > (1 << 16)) return emc2_fail(ctx, EMC2_ERR_UNSUPPORTED, "%s: channels outside [1, 2^16]", what);
  if (capacity < 0 || capacity > (1ll << 30)) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: capacity outside [0, 2^30]", what);
  if (n_seq < 1 || n_seq > (1 << 30) || !offsets) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: offsets null or n_seq outside [1, 2^30]", what);
  return EMC2_OK;
}
bool aligned(const void* p) { return ((uintptr_t)p & 15) == 0; }
// States [n_seq][channels] of both lie apart: one sequence's are read by some waves while others write another's.
bool apart(const float* p, const float* q, int32_t n_seq, int32_t channels) {
  const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q, size = (uintptr_t)n_seq * channels * sizeof(float);
  return !p || !q || a + size <= b || b + size <= a;
}

}  // namespace

extern "C" emc2_status emc2_frame_offsets(emc2_ctx* ctx, const int32_t* d_coords, const int32_t* d_n, int64_t capacity, int32_t n_batch,
                                          int32_t* d_offsets, void* stream) {
  if (!ctx) return EMC2_ERR_INVALID_ARG;
  if (!d_offsets || (!d_coords && capacity > 0)) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_frame_offsets: null argument");
  if (capacity < 0 || capacity > (1ll << 30) || n_batch < 1 || n_batch > (1 << 30))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_frame_offsets: capacity outside [0, 2^30] or n_batch outside [1, 2^30]");
  if (!aligned(d_coords)) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_frame_offsets: d_coords must be 16-byte aligned");
  hipLaunchKernelGGL(k_frame_offsets, dim3((unsigned)emc2_div_up((int64_t)n_batch + 1, kStepThreads)), dim3(kStepThreads), 0, (hipStream_t)stream,
                     (const int4*)d_coords, d_n, capacity, n_batch, d_offsets);
  return emc2_check_hip(ctx, hipGetLastError(), "emc2_frame_offsets launch");
}

extern "C" int64_t emc2_recurrence_work(emc2_dtype dtype, int64_t capacity, int32_t channels) {
  if (!emc2_is_float(dtype) || channels < 1 || channels > (1 << 16) || capacity < 0 || capacity > (1ll << 30)) return -1;
  const int64_t forward = plan_of(dtype, capacity, channels, false).most, grad = plan_of(dtype, capacity, channels, true).most;
  return forward > grad ? forward : grad;
}

extern "C" emc2_status emc2_recurrence(emc2_ctx* ctx, emc2_dtype dtype, const void* d_x, int64_t ld_x, const void* d_gate, int64_t ld_gate,
                                       const int32_t* d_offsets, int32_t n_seq, int64_t capacity, int32_t channels, int32_t backwards,
                                       const float* d_h0, void* d_y, int64_t ld_y, float* d_last, void* d_work, int64_t work_bytes,
                                       void* stream) {
  if (!ctx) return EMC2_ERR_INVALID_ARG;
  const emc2_status st = check(ctx, "emc2_recurrence", dtype, capacity, channels, n_seq, d_offsets);
  if (st != EMC2_OK) return st;
  const size_t size = emc2_size_of(dtype);
  const bool none = capacity == 0;
  if (!emc2_rows_ok(d_x, ld_x, channels, size, none) || !emc2_rows_ok(d_gate, ld_gate, channels, size, none) ||
      !emc2_rows_ok(d_y, ld_y, channels, size, none))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_recurrence: null or misaligned rows, or a pitch below the channels");
  if (!apart(d_h0, d_last, n_seq, channels)) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_recurrence: d_last must not overlap d_h0");
  const Plan p = plan_of(dtype, capacity, channels, false);
  if (work_bytes < p.bytes || (p.bytes && (!d_work || !aligned(d_work))))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_recurrence: work buffer null, misaligned or smaller than emc2_recurrence_work");
  Args a = {};
  a.x = d_x, a.gate = d_gate, a.h0 = d_h0, a.offsets = d_offsets, a.y = d_y, a.last = d_last, a.block_f = (float2*)d_work;
  a.tile_f = a.block_f + (int64_t)p.blocks * p.width;
  a.flags = ctx->dev_words, a.ld_x = ld_x, a.ld_gate = ld_gate, a.ld_y = ld_y, a.capacity = (int32_t)capacity, a.channels = channels;
  a.width = p.width, a.n_seq = n_seq, a.tiles = p.tiles, a.backwards = backwards != 0, a.lane_shift = p.lane_shift;
  const dim3 grid((unsigned)p.blocks, (unsigned)p.slices), rows_grid((unsigned)blocks_with_states(p, n_seq, d_last), (unsigned)p.slices);
  with_type(dtype, p.n, [&](auto type, auto length) {
    using T = decltype(type);
    constexpr int N = kLength<decltype(length)>;
    if (p.totals) hipLaunchKernelGGL((k_recurrence_totals<T, N, kRowsForward>), grid, dim3(64 * kWavesForward), 0, (hipStream_t)stream, a);
    hipLaunchKernelGGL((k_recurrence<T, N, kRowsForward>), rows_grid, dim3(p.totals ? 64 * kWavesForward : 64), 0, (hipStream_t)stream, a);
  });
  return emc2_check_hip(ctx, hipGetLastError(), "emc2_recurrence launch");
}

extern "C" emc2_status emc2_recurrence_backward(emc2_ctx* ctx, emc2_dtype dtype, const void* d_x, int64_t ld_x, const void* d_gate,
                                                int64_t ld_gate, const int32_t* d_offsets, int32_t n_seq, int64_t capacity, int32_t channels,
                                                int32_t backwards, const float* d_h0, const void* d_dy, int64_t ld_dy, const float* d_dlast,
                                                void* d_dx, int64_t ld_dx, void* d_dgate, int64_t ld_dgate, float* d_dh0, void* d_work,
                                                int64_t work_bytes, void* stream) {
  if (!ctx) return EMC2_ERR_INVALID_ARG;
  const emc2_status st = check(ctx, "emc2_recurrence_backward", dtype, capacity, channels, n_seq, d_offsets);
  if (st != EMC2_OK) return st;
  const size_t size = emc2_size_of(dtype);
  const bool none = capacity == 0;
  if (!emc2_rows_ok(d_x, ld_x, channels, size, none) || !emc2_rows_ok(d_gate, ld_gate, channels, size, none) ||
      !emc2_rows_ok(d_dy, ld_dy, channels, size, none) || !emc2_rows_ok(d_dx, ld_dx, channels, size, none) ||
      !emc2_rows_ok(d_dgate, ld_dgate, channels, size, none))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_recurrence_backward: null or misaligned rows, or a pitch below the channels");
  if (!apart(d_dlast, d_dh0, n_seq, channels))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_recurrence_backward: d_dh0 must not overlap d_dlast");
  const Plan p = plan_of(dtype, capacity, channels, true);
  if (work_bytes < p.bytes || (p.bytes && (!d_work || !aligned(d_work))))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_recurrence_backward: work buffer null, misaligned or smaller than emc2_recurrence_work");
  Args a = {};
  a.x = d_x, a.gate = d_gate, a.dy = d_dy, a.h0 = d_h0, a.dlast = d_dlast, a.offsets = d_offsets, a.y = d_dx, a.dgate = d_dgate, a.dh0 = d_dh0;
  a.block_f = (float2*)d_work, a.block_r = a.block_f + (int64_t)p.blocks * p.width, a.tile_f = a.block_r + (int64_t)p.blocks * p.width;
  a.flags = ctx->dev_words, a.ld_x = ld_x, a.ld_gate = ld_gate, a.ld_dy = ld_dy, a.ld_y = ld_dx, a.ld_dgate = ld_dgate;
  a.capacity = (int32_t)capacity, a.channels = channels, a.width = p.width, a.n_seq = n_seq, a.tiles = p.tiles;
  a.backwards = backwards != 0, a.lane_shift = p.lane_shift;
  const dim3 grid((unsigned)p.blocks, (unsigned)p.slices), rows_grid((unsigned)blocks_with_states(p, n_seq, d_dh0), (unsigned)p.slices);
  with_type(dtype, p.n, [&](auto type, auto length) {
    using T = decltype(type);
    constexpr int N = kLength<decltype(length)>;
    if (p.totals) hipLaunchKernelGGL((k_recurrence_grad_totals<T, N, kRowsGrad>), grid, dim3(64 * kWavesGrad), 0, (hipStream_t)stream, a);
    hipLaunchKernelGGL((k_recurrence_grad<T, N, kRowsGrad>), rows_grid, dim3(64 * kWavesGrad), 0, (hipStream_t)stream, a);
  });
  return emc2_check_hip(ctx, hipGetLastError(), "emc2_recurrence_backward launch");
}

extern "C" emc2_status emc2_recurrence_step(emc2_ctx* ctx, emc2_dtype dtype, const void* d_x, int64_t ld_x, const void* d_gate, int64_t ld_gate,
                                            const float* d_h, int64_t rows, int32_t channels, float* d_h_out, void* d_y, int64_t ld_y,
                                            void* stream) {
  if (!ctx) return EMC2_ERR_INVALID_ARG;
  if (!emc2_is_float(dtype)) return emc2_fail(ctx, EMC2_ERR_UNSUPPORTED, "emc2_recurrence_step: dtype must be F32, F16 or BF16");
  if (channels < 1 || channels > (1 << 16)) return emc2_fail(ctx, EMC2_ERR_UNSUPPORTED, "emc2_recurrence_step: channels outside [1, 2^16]");
  if (rows < 0 || rows > (1ll << 30)) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_recurrence_step: rows outside [0, 2^30]");
  const size_t size = emc2_size_of(dtype);
  if (rows == 0) return EMC2_OK;
  if (!d_h || !d_h_out) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_recurrence_step: null argument");
  if (!emc2_rows_ok(d_x, ld_x, channels, size, false) || !emc2_rows_ok(d_gate, ld_gate, channels, size, false) ||
      !emc2_rows_ok(d_y, ld_y, channels, size, false))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_recurrence_step: null or misaligned rows, or a pitch below the channels");
  const int n = channels >= 4 ? 4 : 1;
  const int64_t blocks = emc2_div_up(rows * emc2_div_up(channels, n), kStepThreads);
  with_type(dtype, n, [&](auto type, auto length) {
    using T = decltype(type);
    constexpr int N = kLength<decltype(length)>;
    hipLaunchKernelGGL((k_recurrence_step<T, N>), emc2_grid(blocks), dim3(kStepThreads), 0, (hipStream_t)stream, (const T*)d_x, ld_x,
                       (const T*)d_gate, ld_gate, d_h, d_h_out, (T*)d_y, ld_y, rows, channels);
  });
  return emc2_check_hip(ctx, hipGetLastError(), "emc2_recurrence_step launch");
}
