// Rows of up to 1024 channels in the registers of neighbouring lanes, for operators that need sums over a whole row (layernorm.hip, gated_residual.hip),
// and the sums of their weights' gradients.
#pragma once
#include "column_sums.h"
#include "lane_sums.h"
#include "rows.h"

namespace {

constexpr int kThreads = 256;
constexpr int kMaxChannels = 1024;

// A lane's vectors: vector v begins at channel at[v] (-1: there is none).  A row whose length is no multiple of N (MOVED) ends with a vector moved
// back over its neighbour: the first twice[v] of its values are that one's too, computed alike by both and counted by one.
template <int N, int L, int V, bool MOVED> struct Places {
  int32_t at[V], twice[V];
  __device__ __forceinline__ Places(int32_t channels, int sub) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int32_t c = (v * L + sub) * N;
      at[v] = c >= channels ? -1 : !MOVED || c + N <= channels ? c : channels - N;
      twice[v] = at[v] >= 0 ? c - at[v] : 0;
    }
  }
  // The sum of the values that the lane counts.
  __device__ __forceinline__ float sum(const emc2_fvec<N> (&x)[V]) const {
    float s = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < N; ++e) s += MOVED && e < twice[v] ? 0.0f : x[v][e];
    return s;
  }
};

// How the rows of a call lie over the lanes, `least` of them at least: vectors of 16 bytes, single values where a row has not even one.
struct Shape { bool wide, moved; int lanes, vectors; };
Shape shape_of(emc2_dtype dtype, int32_t channels, int least = 8) {
  const int whole = dtype == EMC2_F32 ? 4 : 8, per = channels >= whole ? whole : 1;
  const int pieces = (channels + per - 1) / per;
  int lanes = least;
  while (lanes < 64 && lanes < pieces) lanes *= 2;
  int vectors = 1;
  while (vectors * lanes < pieces) vectors *= 2;
  return {per > 1, channels % per != 0, lanes, vectors};
}

// Calls f with the compile-time form (values a vector, lanes, vectors, rows at a time) of a shape.  Against one value a lane where rows are not whole
// vectors: 200 k x 47 f16 forward and backward 94 us, 32 with a last vector moved back.
template <int N, int L, int V, int U, bool MOVED = false> struct Form {
  static constexpr int n = N, l = L, v = V, u = U;
  static constexpr bool moved = MOVED;
};
template <int N, bool MOVED, int LEAST, typename F> void with_form(const Shape& s, F&& f) {
  if constexpr (LEAST <= 2) {
    if (s.lanes == 2) return f(Form<N, 2, 1, 4, MOVED>());
    if (s.lanes == 4) return f(Form<N, 4, 1, 4, MOVED>());
  }
  switch (s.lanes) {
    case 8: return f(Form<N, 8, 1, 4, MOVED>());
    case 16: return f(Form<N, 16, 1, 4, MOVED>());
    case 32: return f(Form<N, 32, 1, 4, MOVED>());
  }
  switch (s.vectors) {
    case 1: return f(Form<N, 64, 1, 2, MOVED>());
    case 2: return f(Form<N, 64, 2, 1, MOVED>());
  }
  if constexpr (N == 4) return f(Form<N, 64, 4, 1, MOVED>());
}
template <typename T, int LEAST, typename F> void with_type(const Shape& s, F&& f) {
  constexpr int N = 16 / sizeof(T);
  const auto with_T = [&](auto form) { f(form, T()); };
  if (!s.wide) with_T(Form<1, 8, 1, 4>());
  else if (s.moved) with_form<N, true, LEAST>(s, with_T);
  else with_form<N, false, LEAST>(s, with_T);
}
template <int LEAST = 8, typename F> void with_type(emc2_dtype dtype, const Shape& s, F&& f) {
  if (dtype == EMC2_F32) with_type<float, LEAST>(s, f);
  else if (dtype == EMC2_F16) with_type<_Float16, LEAST>(s, f);
  else with_type<__bf16, LEAST>(s, f);
}

}  // namespace
