// Layer norm over the channels of feature rows, and its gradients.
//   y = (s - mean) * rstd * gamma + beta,   rstd = 1 / sqrt(var + eps), var the mean of (s - mean)^2, s = x or x + residual
// A row lies in the registers of L neighbouring lanes, V vectors of 16 bytes each: it is read once, the mean is summed first
// and the squares about it second (no difference of two large sums), both in fp32 with a butterfly over the L lanes.
//   dx = rstd (q - mean(q) - xh mean(q xh)) + add,  q = dy gamma, xh = (x - mean) rstd;   dgamma = sum over rows of dy xh, dbeta of dy
// The backward pass takes mean and rstd from the row again, which it needs in registers anyway: nothing is kept from the forward
// pass.  The weights' sums stay in each lane's registers while its block walks the rows; the blocks' sums are added by a second
// launch in a fixed order (fp32 throughout, no atomics: equal inputs give equal bits).
// Both are bound by memory: 613 k x 64 f16 with residual and sum 63 us, 5.0 TB/s of what it has to move (a copy of that size reaches 5.0); forward and
// backward pass of 240 k x 128 bf16 68 us, 4.5 TB/s.
#include "row_lanes.h"

namespace {

struct NormArgs {
  const void *x, *res, *dy;      // res: forward: the residual; backward: added to dx.  May be null
  const float *gamma, *beta;
  const int32_t* d_n;
  void *y, *sum;                 // y: forward: the result; backward: dx
  float* partial;                // [blocks][2][channels]
  int64_t ld_x, ld_res, ld_dy, ld_y, ld_sum, capacity;
  int32_t channels;
  float eps, inv_channels;
};

// N values a vector, L lanes a row, V vectors a lane, U rows of a lane under way together
template <typename T, int N, int L, int V, int U, bool MOVED>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 5 : 4) k_layernorm(const NormArgs a) {
  const int32_t n = emc2_row_count(a.d_n, a.capacity);
  constexpr int kGroups = kThreads / L;
  const int64_t first = emc2_block() * (kGroups * U) + threadIdx.x / L;
  if (emc2_block() * (kGroups * U) >= n) return;
  const Places<N, L, V, MOVED> p(a.channels, threadIdx.x % L);
  emc2_fvec<N> x[U][V];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t row = first + u * kGroups;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      x[u][v] = 0.0f;
      if (row < n && p.at[v] >= 0) x[u][v] = emc2_load<N>((const T*)a.x + row * a.ld_x + p.at[v]);
    }
  }
  if (a.res) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t row = first + u * kGroups;
      if (row >= n) break;
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (p.at[v] >= 0) x[u][v] += emc2_load<N>((const T*)a.res + row * a.ld_res + p.at[v]);
      if (a.sum) {                                         // rounded for the caller, not for the norm; after all of the row's loads
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (p.at[v] >= 0) emc2_store<N>((T*)a.sum + row * a.ld_sum + p.at[v], x[u][v]);
      }
    }
  }
  emc2_fvec<N> gamma[V], beta[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    gamma[v] = 0.0f, beta[v] = 0.0f;
    if (p.at[v] >= 0) gamma[v] = emc2_load<N>(a.gamma + p.at[v]), beta[v] = emc2_load<N>(a.beta + p.at[v]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t row = first + u * kGroups;
    const float mean = lane_sum<L>(p.sum(x[u])) * a.inv_channels;
    emc2_fvec<N> sq[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      x[u][v] -= mean;
      sq[v] = p.at[v] >= 0 ? x[u][v] * x[u][v] : emc2_fvec<N>(0.0f);
    }
    const float rstd = 1.0f / __builtin_sqrtf(lane_sum<L>(p.sum(sq)) * a.inv_channels + a.eps);
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (row < n && p.at[v] >= 0) emc2_store<N>((T*)a.y + row * a.ld_y + p.at[v], x[u][v] * rstd * gamma[v] + beta[v]);
  }
}

template <typename T, int N, int L, int V, bool MOVED>
__global__ void __launch_bounds__(kThreads, V == 1 ? 5 : 2) k_layernorm_grad(const NormArgs a, float* __restrict__ dgamma, float* __restrict__ dbeta) {
  const int32_t n = emc2_row_count(a.d_n, a.capacity);
  constexpr int kGroups = kThreads / L;
  const Places<N, L, V, MOVED> p(a.channels, threadIdx.x % L);
  emc2_fvec<N> gamma[V], sum_g[V], sum_b[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    gamma[v] = 0.0f, sum_g[v] = 0.0f, sum_b[v] = 0.0f;
    if (p.at[v] >= 0) gamma[v] = emc2_load<N>(a.gamma + p.at[v]);
  }
  const int64_t step = (int64_t)gridDim.x * kGroups;
  for (int64_t row = (int64_t)blockIdx.x * kGroups + threadIdx.x / L; row < n; row += step) {
    emc2_fvec<N> x[V], dy[V], t[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      x[v] = 0.0f, dy[v] = 0.0f;
      if (p.at[v] >= 0) {
        x[v] = emc2_load<N>((const T*)a.x + row * a.ld_x + p.at[v]);
        dy[v] = emc2_load<N>((const T*)a.dy + row * a.ld_dy + p.at[v]);
      }
    }
    const float mean = lane_sum<L>(p.sum(x)) * a.inv_channels;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      x[v] = p.at[v] >= 0 ? x[v] - mean : emc2_fvec<N>(0.0f);
      t[v] = x[v] * x[v];
    }
    const float rstd = 1.0f / __builtin_sqrtf(lane_sum<L>(p.sum(t)) * a.inv_channels + a.eps);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      x[v] *= rstd;                                        // xh
      sum_g[v] += dy[v] * x[v];
      sum_b[v] += dy[v];
      dy[v] *= gamma[v];
      t[v] = dy[v] * x[v];
    }
    const float mean_q = lane_sum<L>(p.sum(dy)) * a.inv_channels;
    const float mean_qx = lane_sum<L>(p.sum(t)) * a.inv_channels;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      t[v] = (dy[v] - mean_q - x[v] * mean_qx) * rstd;
      if (a.res && p.at[v] >= 0) t[v] += emc2_load<N>((const T*)a.res + row * a.ld_res + p.at[v]);
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (p.at[v] >= 0) emc2_store<N>((T*)a.y + row * a.ld_y + p.at[v], t[v]);
  }
  // The block's sums: over a wave's groups by a butterfly, over the waves through LDS, one half of the channels' vectors at a time.
  __shared__ float part[kThreads / 64][L * N];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
  for (int which = 0; which < 2; ++which)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      emc2_fvec<N> s = which ? sum_b[v] : sum_g[v];
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
        if (from < a.channels && c >= from) {                // a vector moved back leaves its neighbour's channels to that one
          if (gridDim.x == 1) (which ? dbeta : dgamma)[c] = all;
          else a.partial[((int64_t)blockIdx.x * 2 + which) * a.channels + c] = all;
        }
      }
    }
}

// dgamma and dbeta from the blocks' sums: 32 columns a block, 32 threads a column, each with eight loads under way (beyond the last sum: of the last one
// again, not counted; 1251 sums of 180 columns 4.9 us, 0.5 more with the last ones loaded in a row).  Added by halves: of 1280 sums none has more than
// 13 additions behind it.
__global__ void __launch_bounds__(1024) k_layernorm_weights(const float* __restrict__ partial, int32_t blocks, int32_t channels,
                                                            float* __restrict__ dgamma, float* __restrict__ dbeta) {
  __shared__ float part[32][33];
  const int col = blockIdx.x * 32 + (threadIdx.x & 31), seg = threadIdx.x >> 5;
  float s = 0.0f;
  if (col < 2 * channels) {
    for (int b = seg; b < blocks; b += 32 * 8) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = partial[(int64_t)min(b + 32 * i, blocks - 1) * 2 * channels + col];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = b + 32 * i < blocks ? v[i] : 0.0f;
      s += sum_by_halves(v);
    }
  }
  part[seg][threadIdx.x & 31] = s;
  __syncthreads();
  if (seg == 0 && col < 2 * channels) {
    float v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = part[i][threadIdx.x];
    (col < channels ? dgamma[col] : dbeta[col - channels]) = sum_by_halves(v);
  }
}

// Blocks of the backward pass, each walking the rows in steps of all blocks: about as many as the chip holds at once (a lane's sums and one row of 16
// bytes leave room for five or six a CU, several vectors a lane for three), one row a lane at a time.  us with the forward pass, 240 k x 128 bf16 / 600 k x 64 f16:
// 1280 or 1536 blocks 69 / 81, 1024 of two rows at a time 76 / 85, 1024 of four 94 / 106; several vectors a lane, 30 k x 1024 bf16 / 20 k x 768 f32 /
// 60 k x 600 f16: 512 blocks 71 / 55 / 130, 768 65 / 56 / 107, 1024 74 / 59 / 133, 1280 71 / 60 / 122.
constexpr int64_t kGradBlocks = 1280;
constexpr int64_t grad_blocks(int vectors) { return vectors == 1 ? kGradBlocks : 768; }

}  // namespace

extern "C" emc2_status emc2_layernorm(emc2_ctx* ctx, emc2_dtype dtype, const void* d_x, int64_t ld_x, const void* d_res, int64_t ld_res,
                                      const float* d_gamma, const float* d_beta, float eps, const int32_t* d_n, int64_t capacity,
                                      int32_t channels, void* d_sum, int64_t ld_sum, void* d_y, int64_t ld_y, void* stream) {
  if (!ctx) return EMC2_ERR_INVALID_ARG;
  if (!emc2_is_float(dtype)) return emc2_fail(ctx, EMC2_ERR_UNSUPPORTED, "emc2_layernorm: dtype must be F32, F16 or BF16");
  if (channels < 1 || channels > kMaxChannels)
    return emc2_fail(ctx, EMC2_ERR_UNSUPPORTED, "emc2_layernorm: channels outside [1, %d]", kMaxChannels);
  if (capacity < 0 || capacity > (1ll << 30)) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_layernorm: capacity outside [0, 2^30]");
  if (!(eps >= 0.0f)) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_layernorm: eps must not be negative");
  const size_t size = emc2_size_of(dtype);
  const bool none = capacity == 0;
  if (!d_gamma || !d_beta || (d_sum && !d_res)) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_layernorm: null argument");
  if (!emc2_rows_ok(d_x, ld_x, channels, size, none) || !emc2_rows_ok(d_y, ld_y, channels, size, none) ||
      !emc2_rows_ok(d_res, ld_res, channels, size, true) || !emc2_rows_ok(d_sum, ld_sum, channels, size, true))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_layernorm: null or misaligned rows, or a pitch below the channels");
  if (none) return EMC2_OK;
  NormArgs a = {};
  a.x = d_x, a.res = d_res, a.gamma = d_gamma, a.beta = d_beta, a.d_n = d_n, a.y = d_y, a.sum = d_sum;
  a.ld_x = ld_x, a.ld_res = ld_res, a.ld_y = ld_y, a.ld_sum = ld_sum, a.capacity = capacity, a.channels = channels;
  a.eps = eps, a.inv_channels = 1.0f / (float)channels;
  with_type(dtype, shape_of(dtype, channels), [&](auto form, auto type) {
    using F = decltype(form);
    using T = decltype(type);
    const int64_t rows = kThreads / F::l * F::u;
    hipLaunchKernelGGL((k_layernorm<T, F::n, F::l, F::v, F::u, F::moved>), emc2_grid(emc2_div_up(capacity, rows)), dim3(kThreads), 0,
                       (hipStream_t)stream, a);
  });
  return emc2_check_hip(ctx, hipGetLastError(), "emc2_layernorm launch");
}

extern "C" int64_t emc2_layernorm_work(emc2_dtype dtype, int64_t capacity, int32_t channels) {
  if (!emc2_is_float(dtype) || channels < 1 || channels > kMaxChannels || capacity < 0 || capacity > (1ll << 30)) return -1;
  const int64_t blocks = emc2_div_up(capacity, 8);         // a block has eight rows at least
  return (blocks < kGradBlocks ? blocks : kGradBlocks) * 2 * channels * (int64_t)sizeof(float);
}

extern "C" emc2_status emc2_layernorm_backward(emc2_ctx* ctx, emc2_dtype dtype, const void* d_x, int64_t ld_x, const void* d_dy, int64_t ld_dy,
                                               const void* d_add, int64_t ld_add, const float* d_gamma, float eps, const int32_t* d_n,
                                               int64_t capacity, int32_t channels, void* d_dx, int64_t ld_dx, float* d_dgamma,
                                               float* d_dbeta, void* d_work, int64_t work_bytes, void* stream) {
  if (!ctx) return EMC2_ERR_INVALID_ARG;
  if (!emc2_is_float(dtype)) return emc2_fail(ctx, EMC2_ERR_UNSUPPORTED, "emc2_layernorm_backward: dtype must be F32, F16 or BF16");
  if (channels < 1 || channels > kMaxChannels)
    return emc2_fail(ctx, EMC2_ERR_UNSUPPORTED, "emc2_layernorm_backward: channels outside [1, %d]", kMaxChannels);
  if (capacity < 0 || capacity > (1ll << 30))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_layernorm_backward: capacity outside [0, 2^30]");
  if (!(eps >= 0.0f)) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_layernorm_backward: eps must not be negative");
  const size_t size = emc2_size_of(dtype);
  const bool none = capacity == 0;
  if (!d_gamma || !d_dgamma || !d_dbeta) return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_layernorm_backward: null argument");
  if (!emc2_rows_ok(d_x, ld_x, channels, size, none) || !emc2_rows_ok(d_dy, ld_dy, channels, size, none) ||
      !emc2_rows_ok(d_dx, ld_dx, channels, size, none) || !emc2_rows_ok(d_add, ld_add, channels, size, true))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_layernorm_backward: null or misaligned rows, or a pitch below the channels");
  if (work_bytes < emc2_layernorm_work(dtype, capacity, channels) || (!none && (!d_work || ((uintptr_t)d_work & 3))))
    return emc2_fail(ctx, EMC2_ERR_INVALID_ARG, "emc2_layernorm_backward: work buffer null, misaligned or smaller than emc2_layernorm_work");
  NormArgs a = {};
  a.x = d_x, a.res = d_add, a.dy = d_dy, a.gamma = d_gamma, a.d_n = d_n, a.y = d_dx, a.partial = (float*)d_work;
  a.ld_x = ld_x, a.ld_res = ld_add, a.ld_dy = ld_dy, a.ld_y = ld_dx, a.capacity = capacity, a.channels = channels;
  a.eps = eps, a.inv_channels = 1.0f / (float)channels;
  hipStream_t s = (hipStream_t)stream;
  int64_t blocks = 1;
  with_type(dtype, shape_of(dtype, channels), [&](auto form, auto type) {
    using F = decltype(form);
    using T = decltype(type);
    blocks = emc2_div_up(capacity, kThreads / F::l * 2);
    blocks = blocks < 1 ? 1 : blocks < grad_blocks(F::v) ? blocks : grad_blocks(F::v);
    hipLaunchKernelGGL((k_layernorm_grad<T, F::n, F::l, F::v, F::moved>), dim3((unsigned)blocks), dim3(kThreads), 0, s, a, d_dgamma, d_dbeta);
  });
  if (blocks > 1)
    hipLaunchKernelGGL(k_layernorm_weights, dim3((unsigned)emc2_div_up(2 * channels, 32)), dim3(1024), 0, s, a.partial, (int32_t)blocks,
                       channels, d_dgamma, d_dbeta);
  return emc2_check_hip(ctx, hipGetLastError(), "emc2_layernorm_backward launch");
}
