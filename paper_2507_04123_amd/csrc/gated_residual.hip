// From a block's result to the next block's input: the norm behind the block, its gate, the scale of the residual branch, the residual sum and the norm
// before the next block in one pass; and the gradients.
//   s = x + scale * act * (b rb) * post,   y = (s rs) * next,   act = silu(gate) or 1,   r? = 1 / sqrt(mean over the row of ?^2 + eps)
// A row lies in the registers of L neighbouring lanes (row_lanes.h): everything is read once, both sums of squares are fp32 butterflies, y is taken from s
// before s is rounded.
//   S = dsum + rs (q - sh mean(q sh)),  q = dy next, sh = s rs            the gradient that reaches s, and so x: dx = S
//   R = S scale;  dgate = R bh post act';  db = rb (d - bh mean(d bh)),  d = R act post, bh = b rb
//   dnext = sum over rows of dy sh;  dpost = scale sum of S act bh;  dscale = sum of S act bh post
// The backward pass computes s again from x, b and gate, which it needs in registers anyway: as many bytes as reading s, and no rounding of s in it.
// Columns' sums stay in each lane's registers while its block walks the rows; the blocks' sums are added by a second launch in a fixed order (fp32
// throughout, no atomics: equal inputs give equal bits).
// Memory bounds both: 613,217 rows of 64 f16 values forward 76 us, 5.1 TB/s, 240,001 rows of 128 bf16 values backward 94 us, 5.2 TB/s.  The next row requested ahead
// changes nothing (95 us) and takes registers that wide rows do not have.
#include "row_lanes.h"

namespace {

struct JoinArgs {
  const void *x, *branch, *gate, *dsum, *dy;   // gate, dsum and dy may be null
  const float *post, *scale, *next;            // next: null without y
  const int32_t* d_n;
  void *sum, *y;                               // y may be null
  void *dx, *dbranch, *dgate;
  float* partial;                              // [blocks][2 * channels + 1]
  int64_t ld_x, ld_branch, ld_gate, ld_dsum, ld_dy, ld_sum, ld_y, ld_dx, ld_dbranch, ld_dgate, capacity;
  int32_t channels;
  float eps, inv_channels;
};

template <int N, int V> struct Row { emc2_fvec<N> v[V]; };
// A lane's vectors of a row, zeros where there are none (no row, or no such operand).
template <typename T, int N, int L, int V, bool MOVED>
__device__ __forceinline__ Row<N, V> fetch(const void* p, int64_t ld, int64_t row, bool there, const Places<N, L, V, MOVED>& at) {
  Row<N, V> r;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    r.v[v] = 0.0f;
    if (there && at.at[v] >= 0) r.v[v] = emc2_load<N>((const T*)p + row * ld + at.at[v]);
  }
  return r;
}
template <typename T, int N, int L, int V, bool MOVED>
__device__ __forceinline__ void put(void* p, int64_t ld, int64_t row, const Row<N, V>& r, const Places<N, L, V, MOVED>& at) {
#pragma unroll
  for (int v = 0; v < V; ++v)
    if (at.at[v] >= 0) emc2_store<N>((T*)p + row * ld + at.at[v], r.v[v]);
}
template <int N, int L, int V, bool MOVED>
__device__ __forceinline__ float mean_of_products(const Row<N, V>& a, const Row<N, V>& b, const Places<N, L, V, MOVED>& at, float inv) {
  emc2_fvec<N> p[V];
#pragma unroll
  for (int v = 0; v < V; ++v) p[v] = a.v[v] * b.v[v];
  return lane_sum<L>(at.sum(p)) * inv;
}

// N values a vector, L lanes a row, V vectors a lane, U rows of a lane under way together
template <typename T, int N, int L, int V, int U, bool MOVED>
__global__ void __launch_bounds__(kThreads, V == 1 ? 4 : 2) k_gated_residual(const JoinArgs a) {
  const int32_t n = emc2_row_count(a.d_n, a.capacity);
  constexpr int kGroups = kThreads / L;
  const int64_t first = emc2_block() * (kGroups * U) + threadIdx.x / L;
  if (emc2_block() * (kGroups * U) >= n) return;
  const Places<N, L, V, MOVED> p(a.channels, threadIdx.x % L);
  Row<N, V> x[U], b[U], g[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t row = first + u * kGroups;
    b[u] = fetch<T>(a.branch, a.ld_branch, row, row < n, p);
    g[u] = fetch<T>(a.gate, a.ld_gate, row, a.gate && row < n, p);
    x[u] = fetch<T>(a.x, a.ld_x, row, row < n, p);
  }
  const Row<N, V> post = fetch<float>(a.post, 0, 0, true, p), next = fetch<float>(a.next, 0, 0, a.next, p);
  const float scale = *a.scale;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t row = first + u * kGroups;
    const float rb = 1.0f / __builtin_sqrtf(mean_of_products(b[u], b[u], p, a.inv_channels) + a.eps);
    Row<N, V> s;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      emc2_fvec<N> t = b[u].v[v] * rb * post.v[v];
      if (a.gate) {
#pragma unroll
        for (int e = 0; e < N; ++e) t[e] *= g[u].v[v][e] * emc2_logistic<sizeof(T) == 4>(g[u].v[v][e]);
      }
      s.v[v] = x[u].v[v] + scale * t;
    }
    if (row < n) put<T>(a.sum, a.ld_sum, row, s, p);
    if (!a.y) continue;
    const float rs = 1.0f / __builtin_sqrtf(mean_of_products(s, s, p, a.inv_channels) + a.eps);
#pragma unroll
    for (int v = 0; v < V; ++v) s.v[v] = s.v[v] * rs * next.v[v];
    if (row < n) put<T>(a.y, a.ld_y, row, s, p);
  }
}

template <typename T, int N, int L, int V, bool MOVED>
__global__ void __launch_bounds__(kThreads, V == 1 ? 4 : 2) k_gated_residual_grad(const JoinArgs a) {
  const int32_t n = emc2_row_count(a.d_n, a.capacity);
  constexpr int kGroups = kThreads / L;
  const Places<N, L, V, MOVED> p(a.channels, threadIdx.x % L);
  const Row<N, V> post = fetch<float>(a.post, 0, 0, true, p), next = fetch<float>(a.next, 0, 0, a.next, p);
  const float scale = *a.scale;
  Row<N, V> sum_post, sum_next;
  float sum_scale = 0.0f;
#pragma unroll
  for (int v = 0; v < V; ++v) sum_post.v[v] = 0.0f, sum_next.v[v] = 0.0f;
  const int64_t step = (int64_t)gridDim.x * kGroups;
  for (int64_t row = (int64_t)blockIdx.x * kGroups + threadIdx.x / L; row < n; row += step) {
    Row<N, V> b = fetch<T>(a.branch, a.ld_branch, row, true, p), g = fetch<T>(a.gate, a.ld_gate, row, a.gate, p);
    Row<N, V> s = fetch<T>(a.x, a.ld_x, row, true, p), S = fetch<T>(a.dsum, a.ld_dsum, row, a.dsum, p);
    Row<N, V> dy = fetch<T>(a.dy, a.ld_dy, row, a.dy, p), act, slope;
    const float rb = 1.0f / __builtin_sqrtf(mean_of_products(b, b, p, a.inv_channels) + a.eps);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      b.v[v] *= rb;                                        // bh
      act.v[v] = 1.0f, slope.v[v] = 0.0f;
      if (a.gate) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          float on, off;
          const float z = g.v[v][e];
          emc2_logistic<sizeof(T) == 4>(z, on, off);
          act.v[v][e] = z * on;
          slope.v[v][e] = on * (1.0f + z * off);
        }
      }
      s.v[v] += scale * (b.v[v] * post.v[v] * act.v[v]);
    }
    if (a.dy) {
      const float rs = 1.0f / __builtin_sqrtf(mean_of_products(s, s, p, a.inv_channels) + a.eps);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        s.v[v] *= rs;                                      // sh
        sum_next.v[v] += dy.v[v] * s.v[v];
        dy.v[v] *= next.v[v];                              // q
      }
      const float m = mean_of_products(dy, s, p, a.inv_channels);
#pragma unroll
      for (int v = 0; v < V; ++v) S.v[v] += (dy.v[v] - s.v[v] * m) * rs;
    }
    Row<N, V> t, d;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      t.v[v] = S.v[v] * b.v[v];
      sum_post.v[v] += t.v[v] * act.v[v];
      d.v[v] = S.v[v] * scale * post.v[v] * act.v[v];
      g.v[v] = t.v[v] * scale * post.v[v] * slope.v[v];    // dgate
      t.v[v] *= act.v[v] * post.v[v];
    }
    sum_scale += p.sum(t.v);
    const float m = mean_of_products(d, b, p, a.inv_channels);
#pragma unroll
    for (int v = 0; v < V; ++v) d.v[v] = (d.v[v] - b.v[v] * m) * rb;
    put<T>(a.dx, a.ld_dx, row, S, p);
    put<T>(a.dbranch, a.ld_dbranch, row, d, p);
    if (a.gate) put<T>(a.dgate, a.ld_dgate, row, g, p);
  }
  // The block's sums: over a wave's groups by a butterfly, over the waves through LDS, one half of the channels' vectors at a time.
  __shared__ float part[kThreads / 64][L * N];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  float* const line = a.partial + (int64_t)blockIdx.x * (2 * a.channels + 1);
#pragma unroll
  for (int which = 0; which < 2; ++which)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      emc2_fvec<N> s = which ? sum_next.v[v] : sum_post.v[v];
#pragma unroll
      for (int d = L; d < 64; d <<= 1)
#pragma unroll
        for (int e = 0; e < N; ++e) s[e] += __shfl_xor(s[e], d, 64);
      __syncthreads();
      if (lane < L) {
#pragma unroll
        for (int e = 0; e < N; ++e) part[wave][lane * N + e] = s[e];
      }
      __syncthreads();
      for (int i = threadIdx.x; i < L * N; i += kThreads) {
        const int32_t from = (v * L + i / N) * N, at = from + N <= a.channels ? from : a.channels - N, c = at + i % N;
        float all = part[0][i];
#pragma unroll
        for (int w = 1; w < kThreads / 64; ++w) all += part[w][i];
        if (from < a.channels && c >= from) line[which * a.channels + c] = all;   // a vector moved back leaves its neighbour's channels to that one
      }
    }
  sum_scale = lane_sum<64>(sum_scale);
  __syncthreads();
  if (lane == 0) part[wave][0] = sum_scale;
  __syncthreads();
  if (threadIdx.x == 0) {
    float all = part[0][0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) all += part[w][0];
    line[2 * a.channels] = all;
  }
}

// Lanes of a row at least (500,000 rows of 16 bf16 values forward and backward 29 and 63 us with eight, 16 and 30 with two).
constexpr int kLeastLanes = 2;
// Blocks of the backward pass, each walking the rows in steps of all blocks: as many as the chip holds at once with the registers of 16-bit rows.  A few more
// run alone at the end: 240,001 rows of 128 bf16 values 102 us (4.8 TB/s) with 1024, 108 with 1792, 114 with 1536, 134 with 1280; fp32 rows, whose kernels
// leave room for more blocks, 205 us with any of these.  60,000 rows of 1000 bf16 values: 267 us with 512, 335 with 768.
constexpr int64_t kGradBlocks = 1024;
constexpr int64_t grad_blocks(int vectors) { return vectors == 1 ? kGradBlocks : 512; }

emc2_status check(emc2_ctx* ctx, const char* what, emc2_dtype dtype, int64_t capacity, int32_t channels, float eps) {
  if (!emc2_is_float(dtype)) return emc2_fail(ctx, EMC2_ERR_UNSUPPORTED, "%s: dtype must be F32, F16 or BF16", what);
  if (channels < 1 || channels > kMaxChannels) return emc2_fail(ctx, EMC2_ERR_UNSUPPORTED, "%s: channels outside [1, %d]", what, kMaxChannels);
  if (capacity < 0 || capacity > (1ll << 30)) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: capacity outside [0, 2^30]", what);
  if (!(eps >= 0.0f)) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "%s: eps must not be negative", what);
  return EMC2_OK;
}

}  // namespace

extern "C" emc2_status emc2_gated_residual(emc2_ctx* ctx, emc2_dtype dtype, const void* d_x, int64_t ld_x, const void* d_branch,
                                           int64_t ld_branch, const void* d_gate, int64_t ld_gate, const float* d_post, const float* d_scale,
                                           const float* d_next, float eps, const int32_t* d_n, int64_t capacity, int32_t channels, void* d_sum,
                                           int64_t ld_sum, void* d_y, int64_t ld_y, void* stream) {
  if (!ctx) return EMC2_ERR_INVALID_ARG;
  const emc2_status st = check(ctx, "emc2_gated_residual", dtype, capacity, channels, eps);
  if (st != EMC2_OK) return st;
  const size_t size = emc2_size_of(dtype);
  const bool none = capacity == 0;
  if (!d_post || !d_scale) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_gated_residual: null argument");
  if (!none && !d_y != !d_next) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_gated_residual: d_y and d_next go together");
  if (!emc2_rows_ok(d_x, ld_x, channels, size, none) || !emc2_rows_ok(d_branch, ld_branch, channels, size, none) ||
      !emc2_rows_ok(d_gate, ld_gate, channels, size, true) || !emc2_rows_ok(d_sum, ld_sum, channels, size, none) ||
      !emc2_rows_ok(d_y, ld_y, channels, size, true))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_gated_residual: null or misaligned rows, or a pitch below the channels");
  const emc2_rows outs[] = {{d_sum, ld_sum, channels}, {d_y, ld_y, channels}};
  const emc2_rows ins[] = {{d_x, ld_x, channels}, {d_branch, ld_branch, channels}, {d_gate, ld_gate, channels}};
  if (!emc2_results_ok(outs, 2, ins, 3, capacity, size, true))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_gated_residual: results overlap each other, or inputs at another place or pitch");
  if (none) return EMC2_OK;
  JoinArgs a = {};
  a.x = d_x, a.branch = d_branch, a.gate = d_gate, a.post = d_post, a.scale = d_scale, a.next = d_next, a.d_n = d_n, a.sum = d_sum, a.y = d_y;
  a.ld_x = ld_x, a.ld_branch = ld_branch, a.ld_gate = ld_gate, a.ld_sum = ld_sum, a.ld_y = ld_y, a.capacity = capacity, a.channels = channels;
  a.eps = eps, a.inv_channels = 1.0f / (float)channels;
  with_type<kLeastLanes>(dtype, shape_of(dtype, channels, kLeastLanes), [&](auto form, auto type) {
    using F = decltype(form);
    using T = decltype(type);
    constexpr int U = F::u > 1 ? F::u / 2 : 1;             // three operands of each row
    hipLaunchKernelGGL((k_gated_residual<T, F::n, F::l, F::v, U, F::moved>), emc2_grid(emc2_div_up(capacity, kThreads / F::l * U)),
                       dim3(kThreads), 0, (hipStream_t)stream, a);
  });
  return emc2_check_hip(ctx, hipGetLastError(), "emc2_gated_residual launch");
}

extern "C" int64_t emc2_gated_residual_work(emc2_dtype dtype, int64_t capacity, int32_t channels) {
  if (!emc2_is_float(dtype) || channels < 1 || channels > kMaxChannels || capacity < 0 || capacity > (1ll << 30)) return -1;
  const int64_t blocks = emc2_div_up(capacity, 8) > 1 ? emc2_div_up(capacity, 8) : 1;   // a block has eight rows at least
  return (blocks < kGradBlocks ? blocks : kGradBlocks) * (2 * channels + 1) * (int64_t)sizeof(float);
}

extern "C" emc2_status emc2_gated_residual_backward(
    emc2_ctx* ctx, emc2_dtype dtype, const void* d_x, int64_t ld_x, const void* d_branch, int64_t ld_branch, const void* d_gate,
    int64_t ld_gate, const float* d_post, const float* d_scale, const float* d_next, float eps, const void* d_dsum, int64_t ld_dsum,
    const void* d_dy, int64_t ld_dy, const int32_t* d_n, int64_t capacity, int32_t channels, void* d_dx, int64_t ld_dx, void* d_dbranch,
    int64_t ld_dbranch, void* d_dgate, int64_t ld_dgate, float* d_dpost, float* d_dscale, float* d_dnext, void* d_work, int64_t work_bytes,
    void* stream) {
  if (!ctx) return EMC2_ERR_INVALID_ARG;
  const emc2_status st = check(ctx, "emc2_gated_residual_backward", dtype, capacity, channels, eps);
  if (st != EMC2_OK) return st;
  const size_t size = emc2_size_of(dtype);
  const bool none = capacity == 0;
  if (!d_post || !d_scale || !d_dpost || !d_dscale) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_gated_residual_backward: null argument");
  if (!d_next != !d_dnext || (!none && (!d_gate != !d_dgate || !d_dy != !d_next || (!d_dy && !d_dsum))))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_gated_residual_backward: d_gate and d_dgate go together, so do d_dy, d_next and d_dnext; one of d_dsum and d_dy is needed");
  if (!emc2_rows_ok(d_x, ld_x, channels, size, none) || !emc2_rows_ok(d_branch, ld_branch, channels, size, none) ||
      !emc2_rows_ok(d_gate, ld_gate, channels, size, true) || !emc2_rows_ok(d_dsum, ld_dsum, channels, size, true) ||
      !emc2_rows_ok(d_dy, ld_dy, channels, size, true) || !emc2_rows_ok(d_dx, ld_dx, channels, size, none) ||
      !emc2_rows_ok(d_dbranch, ld_dbranch, channels, size, none) || !emc2_rows_ok(d_dgate, ld_dgate, channels, size, true))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_gated_residual_backward: null or misaligned rows, or a pitch below the channels");
  const emc2_rows outs[] = {{d_dx, ld_dx, channels}, {d_dbranch, ld_dbranch, channels}, {d_dgate, ld_dgate, channels}};
  const emc2_rows ins[] = {{d_x, ld_x, channels}, {d_branch, ld_branch, channels}, {d_gate, ld_gate, channels}, {d_dsum, ld_dsum, channels},
                           {d_dy, ld_dy, channels}};
  if (!emc2_results_ok(outs, 3, ins, 5, capacity, size, true))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_gated_residual_backward: results overlap each other, or inputs at another place or pitch");
  if (work_bytes < emc2_gated_residual_work(dtype, capacity, channels) || !d_work || ((uintptr_t)d_work & 15))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_gated_residual_backward: work buffer null, misaligned or smaller than emc2_gated_residual_work");
  JoinArgs a = {};
  a.x = d_x, a.branch = d_branch, a.gate = d_gate, a.dsum = d_dsum, a.dy = d_dy, a.post = d_post, a.scale = d_scale, a.next = d_next, a.d_n = d_n;
  a.dx = d_dx, a.dbranch = d_dbranch, a.dgate = d_dgate, a.partial = (float*)d_work;
  a.ld_x = ld_x, a.ld_branch = ld_branch, a.ld_gate = ld_gate, a.ld_dsum = ld_dsum, a.ld_dy = ld_dy, a.ld_dx = ld_dx, a.ld_dbranch = ld_dbranch;
  a.ld_dgate = ld_dgate, a.capacity = capacity, a.channels = channels, a.eps = eps, a.inv_channels = 1.0f / (float)channels;
  hipStream_t s = (hipStream_t)stream;
  int64_t blocks = 1;
  with_type<kLeastLanes>(dtype, shape_of(dtype, channels, kLeastLanes), [&](auto form, auto type) {
    using F = decltype(form);
    using T = decltype(type);
    blocks = emc2_div_up(capacity, kThreads / F::l * 2);
    blocks = blocks < 1 ? 1 : blocks < grad_blocks(F::v) ? blocks : grad_blocks(F::v);
    hipLaunchKernelGGL((k_gated_residual_grad<T, F::n, F::l, F::v, F::moved>), dim3((unsigned)blocks), dim3(kThreads), 0, s, a);
  });
  Columns c = {};
  c.parts = a.partial, c.lines = (int32_t)blocks, c.width = 2 * channels + 1, c.factor = d_scale;
  c.to[0] = d_dpost, c.end[0] = channels, c.to[1] = d_dnext, c.end[1] = 2 * channels, c.to[2] = d_dscale, c.end[2] = 2 * channels + 1;
  emc2_column_sums(c, s);
  return emc2_check_hip(ctx, hipGetLastError(), "emc2_gated_residual_backward launch");
}
