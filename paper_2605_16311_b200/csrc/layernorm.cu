// Layer norm over the last axis, forward and backward, with one weight gradient per worker.
//
//   forward   s = x + residual,  y = (s - mean) rstd gamma + beta
//   backward  xhat = (s - mean) rstd,  d = dy gamma,  dx = rstd (d - mean(d) - xhat mean(d xhat)) + dsum,
//             dgamma_k = sum_rows dy xhat,  dbeta_k = sum_rows dy
//
// A row is held in the registers of T threads, E entries each (T = 4 .. 1024): it is read once, and the variance is the
// mean of the squared differences from the mean that is already known, so nothing cancels.  Rows beyond 1024 x 16
// entries are passed over several times instead (the second and later passes find them in the caches).
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <new>

#include "../../include/signmuon.h"
#include "common.cuh"

using namespace signmuon;

namespace {

constexpr int WIDE_THREADS = 1024;
constexpr int COLUMN_THREADS = 256;

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(bf16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(bf16* p, float x) { *p = __float2bfloat16_rn(x); }
template <typename AT> __device__ __forceinline__ float rounded(float x);
template <> __device__ __forceinline__ float rounded<float>(float x) { return x; }
template <> __device__ __forceinline__ float rounded<bf16>(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }

template <typename AT> struct Unit { static constexpr int N = 16 / sizeof(AT); };   // entries of a 16-byte access

// N neighbouring entries from an address that is aligned to them all (at most 16 bytes are needed).
template <int N>
__device__ __forceinline__ void load_unit(const float* p, float* x) {
#pragma unroll
  for (int q = 0; q < N / 4; ++q) {
    const float4 a = reinterpret_cast<const float4*>(p)[q];
    x[4 * q] = a.x; x[4 * q + 1] = a.y; x[4 * q + 2] = a.z; x[4 * q + 3] = a.w;
  }
}
template <int N>
__device__ __forceinline__ void load_unit(const bf16* p, float* x) {
  uint32_t w[N / 2];
  if constexpr (N == 8) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
  } else {
    const uint2 a = *reinterpret_cast<const uint2*>(p);
    w[0] = a.x; w[1] = a.y;
  }
#pragma unroll
  for (int e = 0; e < N / 2; ++e) {
    x[2 * e] = __uint_as_float(w[e] << 16);
    x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
  }
}
__device__ __forceinline__ void store_unit(float* p, const float* x) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
}
__device__ __forceinline__ void store_unit(bf16* p, const float* x) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                                            pack_bf16x2(x[6], x[7]));
}

// A thread's E entries of a row of `cols`: units of 16 bytes, T units apart, or (VEC false) single entries T apart.
template <typename AT, int T, int E, bool VEC>
__device__ __forceinline__ int column(int t, int e) {
  constexpr int U = Unit<AT>::N;
  return VEC ? ((e / U) * T + t) * U + e % U : e * T + t;
}
template <typename AT, int T, int E, bool VEC>
__device__ __forceinline__ void load_row(const AT* p, int t, int cols, float (&x)[E]) {
  constexpr int U = Unit<AT>::N;
  if constexpr (VEC) {
#pragma unroll
    for (int e = 0; e < E; e += U) {
      const int c = column<AT, T, E, VEC>(t, e);
      if (c < cols) load_unit<U>(p + c, x + e);
      else for (int u = 0; u < U; ++u) x[e + u] = 0.f;
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = column<AT, T, E, VEC>(t, e);
      x[e] = c < cols ? as_float(p[c]) : 0.f;
    }
  }
}
template <typename AT, int T, int E, bool VEC>
__device__ __forceinline__ void store_row(AT* p, int t, int cols, const float (&x)[E]) {
  constexpr int U = Unit<AT>::N;
  if constexpr (VEC) {
#pragma unroll
    for (int e = 0; e < E; e += U) {
      const int c = column<AT, T, E, VEC>(t, e);
      if (c < cols) store_unit(p + c, x + e);
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = column<AT, T, E, VEC>(t, e);
      if (c < cols) put(p + c, x[e]);
    }
  }
}
// gamma or beta (either type; null: the neutral value) at a thread's entries
template <typename AT, int T, int E, bool VEC, typename WT>
__device__ __forceinline__ void load_weights_as(const WT* p, int t, int cols, float (&x)[E]) {
  constexpr int U = Unit<AT>::N;
  if constexpr (VEC) {
#pragma unroll
    for (int e = 0; e < E; e += U) {
      const int c = column<AT, T, E, VEC>(t, e);
      if (c < cols) load_unit<U>(p + c, x + e);
      else for (int u = 0; u < U; ++u) x[e + u] = 0.f;
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = column<AT, T, E, VEC>(t, e);
      x[e] = c < cols ? as_float(p[c]) : 0.f;
    }
  }
}
template <typename AT, int T, int E, bool VEC>
__device__ __forceinline__ void load_weights(const void* p, bool is_bf16, float neutral, int t, int cols, float (&x)[E]) {
  if (!p) {
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = neutral;
  } else if (is_bf16) {
    load_weights_as<AT, T, E, VEC>(static_cast<const bf16*>(p), t, cols, x);
  } else {
    load_weights_as<AT, T, E, VEC>(static_cast<const float*>(p), t, cols, x);
  }
}

// Sums over the T threads of a row; every thread gets the result.  `part` is shared memory for T / 32 values that no
// other sum in flight uses.
template <int T, int N>
__device__ __forceinline__ void row_sum(float (&x)[N], float* part, int t) {
#pragma unroll
  for (int o = (T < 32 ? T : 32) / 2; o > 0; o >>= 1)
#pragma unroll
    for (int n = 0; n < N; ++n) x[n] += __shfl_xor_sync(0xffffffffu, x[n], o);
  if constexpr (T > 32) {
    constexpr int W = T / 32;
    if ((t & 31) == 0)
#pragma unroll
      for (int n = 0; n < N; ++n) part[n * W + (t >> 5)] = x[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float r = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) r += part[n * W + w];
      x[n] = r;
    }
  }
}

struct Forward {
  const void *x, *residual, *gamma, *beta;
  void *y, *sum;
  float *mean, *rstd;
  int64_t ld_x, ld_residual, ld_y, ld_sum;
  int64_t rows, cols;
  int32_t weight_bf16;
  float eps, inv_cols;
};

template <int T> struct Group { static constexpr int THREADS = T <= 32 ? 128 : T, ROWS = THREADS / T; };

template <typename AT, int T, int E, bool VEC>
__global__ void __launch_bounds__(Group<T>::THREADS) forward_kernel(const Forward a) {
  __shared__ float part[2][T > 32 ? T / 32 : 1];
  wait_for_stream();
  let_next_begin();
  const int t = threadIdx.x % T, cols = (int)a.cols;
  const int64_t row = (int64_t)blockIdx.x * Group<T>::ROWS + threadIdx.x / T;
  const bool live = row < a.rows;
  float x[E] = {};
  if (live) {
    load_row<AT, T, E, VEC>(static_cast<const AT*>(a.x) + row * a.ld_x, t, cols, x);
    if (a.residual) {
      float r[E];
      load_row<AT, T, E, VEC>(static_cast<const AT*>(a.residual) + row * a.ld_residual, t, cols, r);
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = rounded<AT>(x[e] + r[e]);
      store_row<AT, T, E, VEC>(static_cast<AT*>(a.sum) + row * a.ld_sum, t, cols, x);
    }
  }
  float s[1] = {0.f};
#pragma unroll
  for (int e = 0; e < E; ++e) s[0] += x[e];
  row_sum<T>(s, part[0], t);
  const float mean = s[0] * a.inv_cols;
  s[0] = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    x[e] -= mean;
    s[0] = column<AT, T, E, VEC>(t, e) < cols ? fmaf(x[e], x[e], s[0]) : s[0];
  }
  row_sum<T>(s, part[1], t);
  if (!live) return;
  const float rstd = rsqrtf(fmaf(s[0], a.inv_cols, a.eps));
  float g[E], b[E];
  load_weights<AT, T, E, VEC>(a.gamma, a.weight_bf16, 1.f, t, cols, g);
  load_weights<AT, T, E, VEC>(a.beta, a.weight_bf16, 0.f, t, cols, b);
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = fmaf(x[e] * rstd, g[e], b[e]);
  store_row<AT, T, E, VEC>(static_cast<AT*>(a.y) + row * a.ld_y, t, cols, x);
  if (t == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
}

// ---- rows through shared memory.  Every thread copies its own units of the rows to come with cp.async and reads back only
// what it copied, so a stage needs no barrier: waiting for one's own copies is enough.  DEPTH rows of a group are in
// flight while one is worked on, whatever the registers allow.
__device__ __forceinline__ void copy16(void* shared, const void* global) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(shared)), "l"(global) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A thread's units of one row of one array inside a stage; NT threads lie side by side.
template <typename AT, int T, int E, int NT>
__device__ __forceinline__ void copy_row(uint4* stage, const AT* p, int t, int cols) {
  constexpr int U = Unit<AT>::N;
#pragma unroll
  for (int v = 0; v < E / U; ++v) {
    const int c = (v * T + t) * U;
    if (c < cols) copy16(stage + v * NT + threadIdx.x, p + c);
  }
}
__device__ __forceinline__ void unpack_unit(uint4 a, const float*, float_pair* x) {
  x[0] = pair_of(__uint_as_float(a.x), __uint_as_float(a.y));
  x[1] = pair_of(__uint_as_float(a.z), __uint_as_float(a.w));
}
__device__ __forceinline__ void unpack_unit(uint4 a, const bf16*, float_pair* x) {
  x[0] = pair_of_bf16x2(a.x);
  x[1] = pair_of_bf16x2(a.y);
  x[2] = pair_of_bf16x2(a.z);
  x[3] = pair_of_bf16x2(a.w);
}
__device__ __forceinline__ uint4 packed_unit(const float*, const float_pair* x) {
  const float2 a = halves(x[0]), b = halves(x[1]);
  return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
}
__device__ __forceinline__ uint4 packed_unit(const bf16*, const float_pair* x) {
  return make_uint4(pack_bf16x2(x[0]), pack_bf16x2(x[1]), pack_bf16x2(x[2]), pack_bf16x2(x[3]));
}
template <typename AT, int T, int E, int NT>
__device__ __forceinline__ void read_row(const uint4* stage, float_pair (&x)[E / 2]) {
  constexpr int U = Unit<AT>::N;
#pragma unroll
  for (int v = 0; v < E / U; ++v) unpack_unit(stage[v * NT + threadIdx.x], static_cast<const AT*>(nullptr), x + v * U / 2);
}
template <typename AT, int T, int E>
__device__ __forceinline__ void write_row(AT* p, int t, int cols, const float_pair (&x)[E / 2]) {
  constexpr int U = Unit<AT>::N;
#pragma unroll
  for (int v = 0; v < E / U; ++v) {
    const int c = (v * T + t) * U;
    if (c < cols) *reinterpret_cast<uint4*>(p + c) = packed_unit(static_cast<const AT*>(nullptr), x + v * U / 2);
  }
}
// The units behind a row's end are never copied: they hold zeros from the start.
template <typename AT, int T, int E, int NT>
__device__ __forceinline__ void clear_tail(uint4* ring, int planes, int t, int cols) {
  constexpr int U = Unit<AT>::N;
#pragma unroll
  for (int v = 0; v < E / U; ++v)
    if ((v * T + t) * U >= cols)
      for (int i = 0; i < planes; ++i) ring[(i * (E / U) + v) * NT + threadIdx.x] = make_uint4(0, 0, 0, 0);
}
// Weights as float32, laid so that a warp's 16-byte reads fall into different banks.
template <typename AT, int T, int E>
__device__ __forceinline__ void keep_weights(float* kept, const void* p, bool is_bf16, float neutral, int t, int cols) {
  float w[E];
  load_weights<AT, T, E, true>(p, is_bf16, neutral, t, cols, w);
#pragma unroll
  for (int e = 0; e < E; e += 4) *reinterpret_cast<float4*>(kept + (e / 4 * T + t) * 4) = make_float4(w[e], w[e + 1], w[e + 2], w[e + 3]);
}
struct Pairs { float_pair a, b; };
template <int T>
__device__ __forceinline__ Pairs kept_weights(const float* kept, int t, int e) {
  const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(kept + (e / 4 * T + t) * 4);
  return {q.x, q.y};
}

// ARRAYS: x, or x and the residual.  With a third row in flight x alone would leave room for fewer thread blocks (768
// columns: 24.3 us for 44 k rows with three, 22.0 us with two); x and residual are faster with three (16.4 us, 18.0 us).
template <typename AT, int T, int E, int ARRAYS> struct ForwardRing {
  static constexpr int NT = T < 256 ? 256 / T * T : T, GROUPS = NT / T;
  static constexpr int DEPTH = sizeof(AT) == 2 && ARRAYS == 2 ? 3 : 2;
  static constexpr size_t STAGE = (size_t)ARRAYS * NT * E * sizeof(AT);
  static constexpr size_t BYTES = DEPTH * STAGE + 2 * T * E * sizeof(float);
};

// Sums over the T threads of group `g` of a block (T a multiple of 32); every thread gets them.  `part`: T / 32 values
// (each sum) of shared memory that no other sum in flight uses.
template <int T>
__device__ __forceinline__ float joined(const float* part) {
  constexpr int W = T / 32;
  float r = 0.f;
  if constexpr (W >= 4) {
#pragma unroll
    for (int w = 0; w < W; w += 4) {
      const float4 q = *reinterpret_cast<const float4*>(part + w);
      r += (q.x + q.y) + (q.z + q.w);
    }
  } else {
#pragma unroll
    for (int w = 0; w < W; ++w) r += part[w];
  }
  return r;
}
template <int T>
__device__ __forceinline__ void group_barrier(int g) { asm volatile("bar.sync %0, %1;" ::"r"(g + 1), "n"(T) : "memory"); }

template <int T>
__device__ __forceinline__ float group_sum(float x, float* part, int t, int g) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if constexpr (T > 32) {
    if ((t & 31) == 0) part[t >> 5] = x;
    group_barrier<T>(g);
    x = joined<T>(part);
  }
  return x;
}
// Two sums at once: the first exchange leaves one of them to each half of the warp.
template <int T>
__device__ __forceinline__ float2 group_sum(float x, float y, float* part, int t, int g) {
  const bool upper = t & 16;
  float r = (upper ? y : x) + __shfl_xor_sync(0xffffffffu, upper ? x : y, 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) r += __shfl_xor_sync(0xffffffffu, r, o);
  if constexpr (T > 32) {
    if ((t & 15) == 0) part[(upper ? T / 32 : 0) + (t >> 5)] = r;
    group_barrier<T>(g);
    return make_float2(joined<T>(part), joined<T>(part + T / 32));
  }
  return make_float2(__shfl_sync(0xffffffffu, r, 0), __shfl_sync(0xffffffffu, r, 16));
}

// Bound by the memory: 16384 x 768 bf16 with the residual's sum (101 MB) in 18.9 us, 5.3 TB/s (16.0 us where y and s are written
// over themselves in the L2 cache); 24.9 us without the ring.  Rows of one warp need no barrier; wider ones lose 5 to 30 % to
// the two barriers a row (8192 bf16 columns without a residual: 4.3 TB/s).
template <typename AT, int T, int E, int ARRAYS>
__global__ void __launch_bounds__(ForwardRing<AT, T, E, ARRAYS>::NT) forward_ring_kernel(const Forward a) {
  using R = ForwardRing<AT, T, E, ARRAYS>;
  constexpr int NT = R::NT, DEPTH = R::DEPTH, U = Unit<AT>::N;
  extern __shared__ uint4 shared[];
  __shared__ __align__(16) float part[R::GROUPS][2][T > 32 ? T / 32 : 1];
  wait_for_stream();
  let_next_begin();
  const int t = threadIdx.x % T, g = threadIdx.x / T, cols = (int)a.cols;
  constexpr int PLANE = NT * E / U, stage = ARRAYS * PLANE;                    // units of one array's rows in a stage, and of all
  float* gamma = reinterpret_cast<float*>(shared + DEPTH * stage);
  float* beta = gamma + T * E;
  const int64_t groups = (int64_t)gridDim.x * R::GROUPS;
  const int64_t first = (int64_t)blockIdx.x * R::GROUPS + g;
  const auto fetch = [&](int64_t row, int slot) {
    if (row < a.rows) {
      copy_row<AT, T, E, NT>(shared + slot * stage, static_cast<const AT*>(a.x) + row * a.ld_x, t, cols);
      if (ARRAYS == 2)
        copy_row<AT, T, E, NT>(shared + slot * stage + PLANE, static_cast<const AT*>(a.residual) + row * a.ld_residual, t, cols);
    }
    copies_commit();
  };
#pragma unroll
  for (int d = 0; d < DEPTH; ++d) fetch(first + d * groups, d);
  clear_tail<AT, T, E, NT>(shared, DEPTH * ARRAYS, t, cols);
  if (g == 0) {
    keep_weights<AT, T, E>(gamma, a.gamma, a.weight_bf16, 1.f, t, cols);
    keep_weights<AT, T, E>(beta, a.beta, a.weight_bf16, 0.f, t, cols);
  }
  __syncthreads();
  int slot = 0;
  for (int64_t row = first; row < a.rows; row += groups, slot = slot + 1 == DEPTH ? 0 : slot + 1) {
    copies_wait<DEPTH - 1>();
    float_pair x[E / 2];
    read_row<AT, T, E, NT>(shared + slot * stage, x);
    if constexpr (ARRAYS == 2) {
      float_pair r[E / 2];
      read_row<AT, T, E, NT>(shared + slot * stage + PLANE, r);
      AT* sum = static_cast<AT*>(a.sum) + row * a.ld_sum;
#pragma unroll
      for (int v = 0; v < E / U; ++v) {
#pragma unroll
        for (int i = v * U / 2; i < (v + 1) * U / 2; ++i) x[i] = pair_add(x[i], r[i]);
        const uint4 q = packed_unit(static_cast<const AT*>(nullptr), x + v * U / 2);
        const int c = (v * T + t) * U;
        if (c < cols) *reinterpret_cast<uint4*>(sum + c) = q;
        unpack_unit(q, static_cast<const AT*>(nullptr), x + v * U / 2);         // what is normalised is the rounded sum
      }
    }
    fetch(row + DEPTH * groups, slot);
    float_pair s = 0;
#pragma unroll
    for (int i = 0; i < E / 2; ++i) s = pair_add(s, x[i]);
    float2 h = halves(s);
    const float mean = group_sum<T>(h.x + h.y, part[g][0], t, g) * a.inv_cols;
    const float_pair off = pair_of(-mean);
    s = 0;
#pragma unroll
    for (int v = 0; v < E / U; ++v)
      if ((v * T + t) * U < cols)
#pragma unroll
        for (int i = v * U / 2; i < (v + 1) * U / 2; ++i) {
          x[i] = pair_add(x[i], off);
          s = pair_fma(x[i], x[i], s);
        }
    h = halves(s);
    const float rstd = rsqrtf(fmaf(group_sum<T>(h.x + h.y, part[g][1], t, g), a.inv_cols, a.eps));
    const float_pair by = pair_of(rstd);
#pragma unroll
    for (int e = 0; e < E; e += 4) {
      const Pairs p = kept_weights<T>(gamma, t, e), q = kept_weights<T>(beta, t, e);
      x[e / 2] = pair_fma(pair_mul(x[e / 2], by), p.a, q.a);
      x[e / 2 + 1] = pair_fma(pair_mul(x[e / 2 + 1], by), p.b, q.b);
    }
    write_row<AT, T, E>(static_cast<AT*>(a.y) + row * a.ld_y, t, cols, x);
    if (t == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
  copies_wait<0>();
}

// N neighbouring entries: one unit of 16 bytes, or a single entry.
template <int N, typename AT>
__device__ __forceinline__ void load_some(const AT* p, float (&x)[N]) {
  if constexpr (N == 1) x[0] = as_float(*p);
  else load_unit<N>(p, x);
}
template <int N, typename AT>
__device__ __forceinline__ void store_some(AT* p, const float (&x)[N]) {
  if constexpr (N == 1) put(p, x[0]);
  else store_unit(p, x);
}
template <int N>
__device__ __forceinline__ void load_some_weights(const void* p, bool is_bf16, float neutral, int64_t c, float (&x)[N]) {
  if (!p) {
#pragma unroll
    for (int u = 0; u < N; ++u) x[u] = neutral;
  } else if (is_bf16) {
    load_some<N>(static_cast<const bf16*>(p) + c, x);
  } else {
    load_some<N>(static_cast<const float*>(p) + c, x);
  }
}

// A row of any length: three passes by one thread block.  A thread meets the same entries in every pass, so s may be
// read back from where it was written, and y may lie on x.
template <typename AT, int N>
__global__ void __launch_bounds__(WIDE_THREADS) forward_wide_kernel(const Forward a) {
  __shared__ float part[2][WIDE_THREADS / 32];
  wait_for_stream();
  let_next_begin();
  const int t = threadIdx.x;
  const int64_t row = blockIdx.x;
  const AT* x = static_cast<const AT*>(a.x) + row * a.ld_x;
  const AT* r = a.residual ? static_cast<const AT*>(a.residual) + row * a.ld_residual : nullptr;
  AT* total = a.residual ? static_cast<AT*>(a.sum) + row * a.ld_sum : nullptr;
  float s[1] = {0.f}, v[N], w[N];
  for (int64_t c = t * N; c < a.cols; c += WIDE_THREADS * N) {
    load_some<N>(x + c, v);
    if (r) {
      load_some<N>(r + c, w);
#pragma unroll
      for (int u = 0; u < N; ++u) v[u] = rounded<AT>(v[u] + w[u]);
      store_some<N>(total + c, v);
    }
#pragma unroll
    for (int u = 0; u < N; ++u) s[0] += v[u];
  }
  const AT* from = r ? total : x;
  row_sum<WIDE_THREADS>(s, part[0], t);
  const float mean = s[0] * a.inv_cols;
  s[0] = 0.f;
  for (int64_t c = t * N; c < a.cols; c += WIDE_THREADS * N) {
    load_some<N>(from + c, v);
#pragma unroll
    for (int u = 0; u < N; ++u) s[0] = fmaf(v[u] - mean, v[u] - mean, s[0]);
  }
  row_sum<WIDE_THREADS>(s, part[1], t);
  const float rstd = rsqrtf(fmaf(s[0], a.inv_cols, a.eps));
  AT* y = static_cast<AT*>(a.y) + row * a.ld_y;
  for (int64_t c = t * N; c < a.cols; c += WIDE_THREADS * N) {
    float g[N], b[N];
    load_some<N>(from + c, v);
    load_some_weights<N>(a.gamma, a.weight_bf16, 1.f, c, g);
    load_some_weights<N>(a.beta, a.weight_bf16, 0.f, c, b);
#pragma unroll
    for (int u = 0; u < N; ++u) v[u] = fmaf((v[u] - mean) * rstd, g[u], b[u]);
    store_some<N>(y + c, v);
  }
  if (t == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
}

struct Backward {
  const void *dy, *s, *gamma, *dsum;
  const float *mean, *rstd;
  void *dx, *dgamma, *dbeta;
  float* partials;               // [workers][parts][2][padded], used when parts > 1
  int64_t padded;                // cols rounded up to four
  int64_t ld_dy, ld_s, ld_dsum, ld_dx, dgamma_stride, dbeta_stride;
  int64_t rows_each, cols;       // rows of a worker
  int32_t parts;                 // thread blocks that share a worker's rows
  int32_t weight_bf16, grad_bf16;
  float inv_cols;
};

__device__ __forceinline__ void put_gradient(void* p, bool is_bf16, int64_t i, float x) {
  if (is_bf16) put(static_cast<bf16*>(p) + i, x);
  else put(static_cast<float*>(p) + i, x);
}

template <int T> struct BackGroup { static constexpr int THREADS = T <= 32 ? 256 : T, ROWS = THREADS / T; };

// dx, and in every thread the sums of its columns over the rows of the block.
template <typename AT, int T, int E, bool VEC>
__global__ void __launch_bounds__(BackGroup<T>::THREADS) backward_kernel(const Backward a) {
  constexpr int ROWS = BackGroup<T>::ROWS;
  constexpr int WARPS = BackGroup<T>::THREADS / 32;
  __shared__ float part[2][T > 32 ? 2 * (T / 32) : 1];
  __shared__ float sums[T <= 32 ? 2 * 32 * E : 1];       // (T <= 32: the warps' columns are joined here)
  wait_for_stream();
  let_next_begin();
  const int t = threadIdx.x % T, cols = (int)a.cols;
  const int worker = blockIdx.x / a.parts, piece = blockIdx.x % a.parts;
  float g[E], dg[E] = {}, db[E] = {};
  load_weights<AT, T, E, VEC>(a.gamma, a.weight_bf16, 1.f, t, cols, g);
  int flip = 0;
  for (int64_t first = (int64_t)piece * ROWS; first < a.rows_each; first += (int64_t)a.parts * ROWS, flip ^= 1) {
    const int64_t mine = first + threadIdx.x / T;
    const bool live = mine < a.rows_each;
    const int64_t row = (int64_t)worker * a.rows_each + mine;
    float x[E] = {}, d[E] = {}, mean = 0.f, rstd = 0.f;
    if (live) {
      load_row<AT, T, E, VEC>(static_cast<const AT*>(a.s) + row * a.ld_s, t, cols, x);
      load_row<AT, T, E, VEC>(static_cast<const AT*>(a.dy) + row * a.ld_dy, t, cols, d);
      mean = a.mean[row];
      rstd = a.rstd[row];
    }
    float c[2] = {0.f, 0.f};
#pragma unroll
    for (int e = 0; e < E; ++e) {
      x[e] = (x[e] - mean) * rstd;
      dg[e] = fmaf(d[e], x[e], dg[e]);
      db[e] += d[e];
      d[e] *= g[e];                                    // (entries behind the row's end are zeros in d)
      c[0] += d[e];
      c[1] = fmaf(d[e], x[e], c[1]);
    }
    row_sum<T>(c, part[flip], t);
    if (!live) continue;
    c[0] *= a.inv_cols;
    c[1] *= a.inv_cols;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = (d[e] - c[0] - x[e] * c[1]) * rstd;
    if (a.dsum) {
      load_row<AT, T, E, VEC>(static_cast<const AT*>(a.dsum) + row * a.ld_dsum, t, cols, d);
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] += d[e];
    }
    store_row<AT, T, E, VEC>(static_cast<AT*>(a.dx) + row * a.ld_dx, t, cols, x);
  }
  if constexpr (T <= 32) {
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int o = T; o < 32; o <<= 1) {
        dg[e] += __shfl_xor_sync(0xffffffffu, dg[e], o);
        db[e] += __shfl_xor_sync(0xffffffffu, db[e], o);
      }
    const int lane = threadIdx.x & 31;
    for (int w = 0; w < WARPS; ++w) {                  // in the order of the warps
      if ((int)(threadIdx.x >> 5) == w && lane < T) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int at = e * 32 + lane;
          sums[at] = dg[e] + (w ? sums[at] : 0.f);
          sums[32 * E + at] = db[e] + (w ? sums[32 * E + at] : 0.f);
        }
      }
      __syncthreads();
    }
    if (threadIdx.x >= T) return;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      dg[e] = sums[e * 32 + lane];
      db[e] = sums[32 * E + e * 32 + lane];
    }
  }
  float* out = a.partials + ((int64_t)worker * a.parts + piece) * 2 * a.padded;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int c = column<AT, T, E, VEC>(t, e);
    if (c >= cols) continue;
    if (a.parts > 1) {
      out[c] = dg[e];
      out[a.padded + c] = db[e];
    } else {
      if (a.dgamma) put_gradient(a.dgamma, a.grad_bf16, worker * a.dgamma_stride + c, dg[e]);
      if (a.dbeta) put_gradient(a.dbeta, a.grad_bf16, worker * a.dbeta_stride + c, db[e]);
    }
  }
}

template <typename AT, int T, int E> struct BackwardRing {
  static constexpr int NT = E == 24 ? 384 : 512, GROUPS = NT / T;      // (24 entries: up to 168 registers a thread, 16: 128)
  static constexpr int BLOCKS = E == 8 ? 2 : 1;                        // of an SM
  static constexpr int DEPTH = 2;
  static constexpr size_t bytes(int arrays) {
    const size_t ring = (size_t)DEPTH * arrays * NT * E * sizeof(AT), join = GROUPS > 1 ? (size_t)GROUPS * 2 * T * E * sizeof(float) : 0;
    return (ring > join ? ring : join) + T * E * sizeof(float);
  }
};

// As backward_kernel, with the rows to come in flight through shared memory.  Every thread keeps the sums of its columns in
// registers (2 E of them), which leaves 12 to 16 warps an SM: too few to hide a row's two sums behind other rows entirely.
// 16384 x 768 bf16 with dsum (101 MB): 22.5 us with the joining kernel, 4.5 TB/s; 16384 x 4096 (403 MB): 77.4 us, 5.2 TB/s.
// Several groups share a thread block so that one leaves a single row of partial sums (1024 columns: 48 us with 64 threads a
// block, 39 us so).
template <typename AT, int T, int E>
__global__ void __launch_bounds__(BackwardRing<AT, T, E>::NT, BackwardRing<AT, T, E>::BLOCKS) backward_ring_kernel(const Backward a) {
  using R = BackwardRing<AT, T, E>;
  constexpr int NT = R::NT, GROUPS = R::GROUPS, DEPTH = R::DEPTH, U = Unit<AT>::N;
  extern __shared__ uint4 shared[];
  __shared__ __align__(16) float part[2][GROUPS][T > 32 ? 2 * (T / 32) : 1];
  wait_for_stream();
  let_next_begin();
  const int t = threadIdx.x % T, g = threadIdx.x / T, cols = (int)a.cols;
  const int worker = blockIdx.x / a.parts, piece = blockIdx.x % a.parts;
  constexpr int PLANE = NT * E / U;
  const int arrays = a.dsum ? 3 : 2, stage = arrays * PLANE;
  float* gamma = reinterpret_cast<float*>(shared);
  uint4* ring = shared + T * E / 4;
  const int64_t row0 = (int64_t)worker * a.rows_each, step = (int64_t)a.parts * GROUPS;
  const int64_t first = (int64_t)piece * GROUPS + g;
  const auto fetch = [&](int64_t mine, int slot) {
    if (mine < a.rows_each) {
      const int64_t row = row0 + mine;
      copy_row<AT, T, E, NT>(ring + slot * stage, static_cast<const AT*>(a.s) + row * a.ld_s, t, cols);
      copy_row<AT, T, E, NT>(ring + slot * stage + PLANE, static_cast<const AT*>(a.dy) + row * a.ld_dy, t, cols);
      if (arrays == 3)
        copy_row<AT, T, E, NT>(ring + slot * stage + 2 * PLANE, static_cast<const AT*>(a.dsum) + row * a.ld_dsum, t, cols);
    }
    copies_commit();
  };
#pragma unroll
  for (int d = 0; d < DEPTH; ++d) fetch(first + d * step, d);
  clear_tail<AT, T, E, NT>(ring, DEPTH * arrays, t, cols);
  if (g == 0) keep_weights<AT, T, E>(gamma, a.gamma, a.weight_bf16, 1.f, t, cols);
  __syncthreads();
  float_pair dg[E / 2] = {}, db[E / 2] = {};
  float mean = 0.f, rstd = 0.f;
  if (first < a.rows_each) {
    mean = a.mean[row0 + first];
    rstd = a.rstd[row0 + first];
  }
  int slot = 0, flip = 0;
  for (int64_t mine = first; mine < a.rows_each; mine += step, slot = slot + 1 == DEPTH ? 0 : slot + 1, flip ^= 1) {
    const int64_t row = row0 + mine;
    float next_mean = 0.f, next_rstd = 0.f;
    if (mine + step < a.rows_each) {
      next_mean = a.mean[row + step];
      next_rstd = a.rstd[row + step];
    }
    copies_wait<DEPTH - 1>();
    float_pair x[E / 2], d[E / 2];
    read_row<AT, T, E, NT>(ring + slot * stage, x);
    read_row<AT, T, E, NT>(ring + slot * stage + PLANE, d);
    float_pair c0 = 0, c1 = 0;
    const float_pair off = pair_of(-mean), by = pair_of(rstd);
#pragma unroll
    for (int e = 0; e < E; e += 4) {
      const Pairs w = kept_weights<T>(gamma, t, e);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int i = e / 2 + u;
        x[i] = pair_mul(pair_add(x[i], off), by);
        dg[i] = pair_fma(d[i], x[i], dg[i]);
        db[i] = pair_add(db[i], d[i]);
        d[i] = pair_mul(d[i], u ? w.b : w.a);          // (entries behind the row's end are zeros in d)
        c0 = pair_add(c0, d[i]);
        c1 = pair_fma(d[i], x[i], c1);
      }
    }
    const float2 h0 = halves(c0), h1 = halves(c1);
    const float2 c = group_sum<T>(h0.x + h0.y, h1.x + h1.y, part[flip][g], t, g);
    const float_pair less = pair_of(-c.x * a.inv_cols), along = pair_of(-c.y * a.inv_cols);
    if (arrays == 3) {
      float_pair r[E / 2];
      read_row<AT, T, E, NT>(ring + slot * stage + 2 * PLANE, r);
#pragma unroll
      for (int i = 0; i < E / 2; ++i) x[i] = pair_fma(pair_fma(x[i], along, pair_add(d[i], less)), by, r[i]);
    } else {
#pragma unroll
      for (int i = 0; i < E / 2; ++i) x[i] = pair_mul(pair_fma(x[i], along, pair_add(d[i], less)), by);
    }
    fetch(mine + DEPTH * step, slot);
    write_row<AT, T, E>(static_cast<AT*>(a.dx) + row * a.ld_dx, t, cols, x);
    mean = next_mean;
    rstd = next_rstd;
  }
  copies_wait<0>();
  const bool direct = a.parts == 1;
  float* out = a.partials + ((int64_t)worker * a.parts + piece) * 2 * a.padded;
  if constexpr (GROUPS > 1) {                          // the groups' sums, joined in their order
    float* join = reinterpret_cast<float*>(ring);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; e += 4) {
      const int c = column<AT, T, E, true>(t, e);
      *reinterpret_cast<ulonglong2*>(join + (g * 2 + 0) * T * E + c) = make_ulonglong2(dg[e / 2], dg[e / 2 + 1]);
      *reinterpret_cast<ulonglong2*>(join + (g * 2 + 1) * T * E + c) = make_ulonglong2(db[e / 2], db[e / 2 + 1]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * T * E; i += NT) {
      const int c = i % (T * E), which = i / (T * E);
      if (c >= cols) continue;
      float r = 0.f;
#pragma unroll
      for (int k = 0; k < GROUPS; ++k) r += join[(k * 2 + which) * T * E + c];
      if (!direct) out[which * a.padded + c] = r;
      else if (void* to = which ? a.dbeta : a.dgamma) put_gradient(to, a.grad_bf16, worker * (which ? a.dbeta_stride : a.dgamma_stride) + c, r);
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = column<AT, T, E, true>(t, e);
      if (c >= cols) continue;
      const float2 p = halves(dg[e / 2]), q = halves(db[e / 2]);
      const float x = e & 1 ? p.y : p.x, y = e & 1 ? q.y : q.x;
      if (!direct) {
        out[c] = x;
        out[a.padded + c] = y;
      } else {
        if (a.dgamma) put_gradient(a.dgamma, a.grad_bf16, worker * a.dgamma_stride + c, x);
        if (a.dbeta) put_gradient(a.dbeta, a.grad_bf16, worker * a.dbeta_stride + c, y);
      }
    }
  }
}

// Joins the partial sums of a worker in the order of its thread blocks.  Block: 32 x 4 columns x 8 runs of parts.
__global__ void __launch_bounds__(256) join_kernel(const Backward a) {
  __shared__ float4 part[8][32];
  const int64_t c = ((int64_t)blockIdx.x * 32 + threadIdx.x) * 4;
  const int worker = blockIdx.y, which = blockIdx.z;
  float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
  wait_for_stream();
  let_next_begin();
  if (c < a.cols) {
    const float* p = a.partials + ((int64_t)worker * a.parts * 2 + which) * a.padded + c;
#pragma unroll 4
    for (int i = threadIdx.y; i < a.parts; i += 8) {
      const float4 q = *reinterpret_cast<const float4*>(p + (int64_t)i * 2 * a.padded);
      r.x += q.x; r.y += q.y; r.z += q.z; r.w += q.w;
    }
  }
  part[threadIdx.y][threadIdx.x] = r;
  __syncthreads();
  void* out = which ? a.dbeta : a.dgamma;
  const int64_t column = (int64_t)blockIdx.x * 128 + threadIdx.y * 32 + threadIdx.x;       // the first four warps: a column each
  if (threadIdx.y >= 4 || column >= a.cols || !out) return;
  const float* q = reinterpret_cast<const float*>(part) + threadIdx.y * 32 + threadIdx.x;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) sum += q[i * 128];
  put_gradient(out, a.grad_bf16, worker * (which ? a.dbeta_stride : a.dgamma_stride) + column, sum);
}

// Rows too long for a thread to hold its columns' sums beside them: the sums first (dx may lie on dy), N columns a thread,
// then dx, which finds dy and s in the caches where they fit.
template <typename AT, int N>
__global__ void __launch_bounds__(COLUMN_THREADS) columns_kernel(const Backward a) {
  wait_for_stream();
  let_next_begin();
  const int64_t c = ((int64_t)blockIdx.x * COLUMN_THREADS + threadIdx.x) * N;
  if (c >= a.cols) return;
  const int piece = blockIdx.y;
  const int64_t worker = blockIdx.z;
  float dg[N] = {}, db[N] = {};
#pragma unroll 4
  for (int64_t mine = piece; mine < a.rows_each; mine += a.parts) {
    const int64_t row = worker * a.rows_each + mine;
    float d[N], x[N];
    load_some<N>(static_cast<const AT*>(a.dy) + row * a.ld_dy + c, d);
    load_some<N>(static_cast<const AT*>(a.s) + row * a.ld_s + c, x);
    const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      dg[u] = fmaf(d[u], (x[u] - mean) * rstd, dg[u]);
      db[u] += d[u];
    }
  }
  float* out = a.partials + (worker * a.parts + piece) * 2 * a.padded + c;
#pragma unroll
  for (int u = 0; u < N; ++u) {
    if (a.parts > 1) {
      out[u] = dg[u];
      out[a.padded + u] = db[u];
    } else {
      if (a.dgamma) put_gradient(a.dgamma, a.grad_bf16, worker * a.dgamma_stride + c + u, dg[u]);
      if (a.dbeta) put_gradient(a.dbeta, a.grad_bf16, worker * a.dbeta_stride + c + u, db[u]);
    }
  }
}
// dx of a row that a thread block holds
template <typename AT, int T, int E, bool VEC>
__global__ void __launch_bounds__(T) dx_kernel(const Backward a) {
  __shared__ float part[2 * (T / 32)];
  wait_for_stream();
  let_next_begin();
  const int t = threadIdx.x, cols = (int)a.cols;
  const int64_t row = blockIdx.x;
  float x[E], d[E], g[E], c[2] = {0.f, 0.f};
  load_row<AT, T, E, VEC>(static_cast<const AT*>(a.s) + row * a.ld_s, t, cols, x);
  load_row<AT, T, E, VEC>(static_cast<const AT*>(a.dy) + row * a.ld_dy, t, cols, d);
  load_weights<AT, T, E, VEC>(a.gamma, a.weight_bf16, 1.f, t, cols, g);
  const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    x[e] = (x[e] - mean) * rstd;
    d[e] *= g[e];
    c[0] += d[e];
    c[1] = fmaf(d[e], x[e], c[1]);
  }
  row_sum<T>(c, part, t);
  c[0] *= a.inv_cols;
  c[1] *= a.inv_cols;
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = (d[e] - c[0] - x[e] * c[1]) * rstd;
  if (a.dsum) {
    load_row<AT, T, E, VEC>(static_cast<const AT*>(a.dsum) + row * a.ld_dsum, t, cols, d);
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] += d[e];
  }
  store_row<AT, T, E, VEC>(static_cast<AT*>(a.dx) + row * a.ld_dx, t, cols, x);
}
// ... and of a row of any length
template <typename AT, int N>
__global__ void __launch_bounds__(WIDE_THREADS) dx_wide_kernel(const Backward a) {
  __shared__ float part[2 * (WIDE_THREADS / 32)];
  wait_for_stream();
  let_next_begin();
  const int t = threadIdx.x;
  const int64_t row = blockIdx.x;
  const AT* s = static_cast<const AT*>(a.s) + row * a.ld_s;
  const AT* dy = static_cast<const AT*>(a.dy) + row * a.ld_dy;
  const float mean = a.mean[row], rstd = a.rstd[row];
  float c[2] = {0.f, 0.f}, d[N], x[N], g[N];
  for (int64_t i = t * N; i < a.cols; i += WIDE_THREADS * N) {
    load_some<N>(dy + i, d);
    load_some<N>(s + i, x);
    load_some_weights<N>(a.gamma, a.weight_bf16, 1.f, i, g);
#pragma unroll
    for (int u = 0; u < N; ++u) {
      c[0] += d[u] * g[u];
      c[1] = fmaf(d[u] * g[u], (x[u] - mean) * rstd, c[1]);
    }
  }
  row_sum<WIDE_THREADS>(c, part, t);
  c[0] *= a.inv_cols;
  c[1] *= a.inv_cols;
  AT* dx = static_cast<AT*>(a.dx) + row * a.ld_dx;
  const AT* more = a.dsum ? static_cast<const AT*>(a.dsum) + row * a.ld_dsum : nullptr;
  for (int64_t i = t * N; i < a.cols; i += WIDE_THREADS * N) {
    load_some<N>(dy + i, d);
    load_some<N>(s + i, x);
    load_some_weights<N>(a.gamma, a.weight_bf16, 1.f, i, g);
#pragma unroll
    for (int u = 0; u < N; ++u) x[u] = (d[u] * g[u] - c[0] - (x[u] - mean) * rstd * c[1]) * rstd;
    if (more) {
      load_some<N>(more + i, d);
#pragma unroll
      for (int u = 0; u < N; ++u) x[u] += d[u];
    }
    store_some<N>(dx + i, x);
  }
}

// rows: of a thread block at a time.  shared: dynamic shared memory (0: a kernel that loads its rows directly); limit: the most
// that any call asks of this kernel.  The limit that the runtime keeps belongs to the kernel and the device, whichever context
// sets it: it is always set to `limit`, so that no call takes away what another one needs.
struct Choice {
  void* fn;
  int threads, rows;
  size_t shared, limit;
  bool wide;
};
template <typename AT, int T, int E, bool VEC>
Choice forward_choice() { return {(void*)forward_kernel<AT, T, E, VEC>, Group<T>::THREADS, Group<T>::ROWS, 0, 0, false}; }
template <typename AT, int T, int E>
Choice forward_ring(int arrays) {
  using One = ForwardRing<AT, T, E, 1>;
  using Two = ForwardRing<AT, T, E, 2>;
  if (arrays == 1) return {(void*)forward_ring_kernel<AT, T, E, 1>, One::NT, One::GROUPS, One::BYTES, One::BYTES, false};
  return {(void*)forward_ring_kernel<AT, T, E, 2>, Two::NT, Two::GROUPS, Two::BYTES, Two::BYTES, false};
}

template <typename AT, bool VEC>
Choice choose_forward(int64_t cols) {
  if (cols <= 4 * 8) return forward_choice<AT, 4, 8, VEC>();
  if (cols <= 8 * 8) return forward_choice<AT, 8, 8, VEC>();
  if (cols <= 16 * 8) return forward_choice<AT, 16, 8, VEC>();
  if (cols <= 32 * 8) return forward_choice<AT, 32, 8, VEC>();
  if constexpr (!VEC) {       // single entries: more threads with fewer of them (1001 columns: 13.4 us, 16.7 us at 32 x 32)
    if (cols <= 32 * 12) return forward_choice<AT, 32, 12, VEC>();
    if (cols <= 64 * 8) return forward_choice<AT, 64, 8, VEC>();
    if (cols <= 64 * 12) return forward_choice<AT, 64, 12, VEC>();
    if (cols <= 128 * 8) return forward_choice<AT, 128, 8, VEC>();
    if (cols <= 128 * 12) return forward_choice<AT, 128, 12, VEC>();
    if (cols <= 256 * 8) return forward_choice<AT, 256, 8, VEC>();
    if (cols <= 256 * 12) return forward_choice<AT, 256, 12, VEC>();
    if (cols <= 512 * 8) return forward_choice<AT, 512, 8, VEC>();
    if (cols <= 512 * 12) return forward_choice<AT, 512, 12, VEC>();
    if (cols <= 1024 * 8) return forward_choice<AT, 1024, 8, VEC>();
    if (cols <= 1024 * 12) return forward_choice<AT, 1024, 12, VEC>();
    if (cols <= 1024 * 16) return forward_choice<AT, 1024, 16, VEC>();
    return {(void*)forward_wide_kernel<AT, 1>, WIDE_THREADS, 1, 0, 0, true};
  } else {
    if (cols <= 32 * 16) return forward_choice<AT, 32, 16, true>();
    if (cols <= 32 * 24) return forward_choice<AT, 32, 24, true>();
    if (cols <= 32 * 32) return forward_choice<AT, 32, 32, true>();
    if (cols <= 128 * 16) return forward_choice<AT, 128, 16, true>();
    if (cols <= 256 * 16) return forward_choice<AT, 256, 16, true>();
    if (cols <= 512 * 16) return forward_choice<AT, 512, 16, true>();
    if (cols <= 1024 * 16) return forward_choice<AT, 1024, 16, true>();
    return {(void*)forward_wide_kernel<AT, Unit<AT>::N>, WIDE_THREADS, 1, 0, 0, true};
  }
}
// (aligned rows of 129 .. 8192 entries)
template <typename AT>
Choice choose_forward_ring(int64_t cols, int arrays) {
  if (cols <= 32 * 8) return forward_ring<AT, 32, 8>(arrays);
  if (cols <= 32 * 16) return forward_ring<AT, 32, 16>(arrays);
  if (cols <= 32 * 24) return forward_ring<AT, 32, 24>(arrays);
  if (cols <= 32 * 32) return forward_ring<AT, 32, 32>(arrays);
  if (cols <= 128 * 16) return forward_ring<AT, 128, 16>(arrays);
  if (cols <= 256 * 16) return forward_ring<AT, 256, 16>(arrays);
  return forward_ring<AT, 512, 16>(arrays);
}

template <typename AT, int T, int E, bool VEC>
Choice backward_choice() { return {(void*)backward_kernel<AT, T, E, VEC>, BackGroup<T>::THREADS, BackGroup<T>::ROWS, 0, 0, false}; }
template <typename AT, int T, int E>
Choice backward_ring(int arrays) {
  using R = BackwardRing<AT, T, E>;
  return {(void*)backward_ring_kernel<AT, T, E>, R::NT, R::GROUPS, R::bytes(arrays), R::bytes(3), false};
}

template <typename AT, bool VEC>
Choice choose_backward(int64_t cols, int arrays) {
  if (cols <= 4 * 8) return backward_choice<AT, 4, 8, VEC>();
  if (cols <= 8 * 8) return backward_choice<AT, 8, 8, VEC>();
  if (cols <= 16 * 8) return backward_choice<AT, 16, 8, VEC>();
  if (cols > 1024 * 16) return {(void*)dx_wide_kernel<AT, VEC ? Unit<AT>::N : 1>, WIDE_THREADS, 1, 0, 0, true};
  if (cols > 512 * 16) return {(void*)dx_kernel<AT, 1024, 16, VEC>, 1024, 1, 0, 0, true};
  if constexpr (VEC) {
    if (cols <= 32 * 8) return backward_ring<AT, 32, 8>(arrays);
    if (cols <= 32 * 16) return backward_ring<AT, 32, 16>(arrays);
    if (cols <= 32 * 24) return backward_ring<AT, 32, 24>(arrays);
    if (cols <= 64 * 16) return backward_ring<AT, 64, 16>(arrays);
    if (cols <= 128 * 16) return backward_ring<AT, 128, 16>(arrays);
    if (cols <= 256 * 16) return backward_ring<AT, 256, 16>(arrays);
    return backward_ring<AT, 512, 16>(arrays);
  } else {
    if (cols <= 32 * 8) return backward_choice<AT, 32, 8, false>();
    if (cols <= 32 * 12) return backward_choice<AT, 32, 12, false>();
    if (cols <= 64 * 8) return backward_choice<AT, 64, 8, false>();
    if (cols <= 64 * 12) return backward_choice<AT, 64, 12, false>();
    if (cols <= 128 * 8) return backward_choice<AT, 128, 8, false>();
    if (cols <= 128 * 12) return backward_choice<AT, 128, 12, false>();
    if (cols <= 256 * 8) return backward_choice<AT, 256, 8, false>();
    if (cols <= 256 * 12) return backward_choice<AT, 256, 12, false>();
    if (cols <= 512 * 8) return backward_choice<AT, 512, 8, false>();
    if (cols <= 512 * 12) return backward_choice<AT, 512, 12, false>();
    return backward_choice<AT, 1024, 8, false>();
  }
}

constexpr int64_t MOST_PARTS = 148 * 8, PARTIAL_BYTES = int64_t(32) << 20;

bool is_dtype(int32_t d) { return d == SIGNMUON_F32 || d == SIGNMUON_BF16; }
int entry_bytes(int32_t dtype) { return dtype == SIGNMUON_BF16 ? 2 : 4; }

}  // namespace

struct signmuon_layernorm {
  signmuon_layernorm_config cfg;
  int64_t max_parts = 1;         // thread blocks over all workers that may leave partial sums
  size_t workspace_bytes = 0;
  float* workspace = nullptr;
  bool bound = false;
  int sms = 0;
  std::atomic<int> sticky{SIGNMUON_OK};
  // Thread blocks of a kernel that an SM holds, asked of the runtime once for each kind of call; 0: not yet.  Threads that ask
  // at once get the same answer.
  enum Kind { FORWARD, FORWARD_RESIDUAL, BACKWARD, BACKWARD_DSUM, BACKWARD_SINGLE, KINDS };
  std::atomic<int> fits[KINDS] = {};

  // Also allows the kernel its dynamic shared memory.  0: the runtime refused.
  int resident(const Choice& k, int kind) {
    int blocks = fits[kind].load(std::memory_order_acquire);
    if (blocks) return blocks;
    if ((k.limit && cudaFuncSetAttribute(k.fn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)k.limit) != cudaSuccess) ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&blocks, k.fn, k.threads, k.shared) != cudaSuccess || blocks < 1)
      return 0;
    fits[kind].store(blocks, std::memory_order_release);
    return blocks;
  }
};

extern "C" {

int signmuon_layernorm_create(const signmuon_layernorm_config* config, signmuon_layernorm** out) {
  if (!out) return SIGNMUON_ERR_INVALID_ARG;
  *out = nullptr;
  if (!config || !is_dtype(config->act_dtype) || !is_dtype(config->weight_dtype) || !is_dtype(config->grad_dtype) ||
      config->num_workers < 1 || config->num_workers > 65535 || !(config->eps >= 0) || !std::isfinite(config->eps))
    return SIGNMUON_ERR_INVALID_ARG;
  if (config->cols < 1 || config->cols > (int64_t(1) << 24)) return SIGNMUON_ERR_BAD_SHAPE;
  signmuon_layernorm* c = new (std::nothrow) signmuon_layernorm();
  if (!c) return SIGNMUON_ERR_NO_MEMORY;
  c->cfg = *config;
  const int64_t bytes = 2 * ((config->cols + 3) / 4 * 4) * (int64_t)sizeof(float);
  c->max_parts = std::max<int64_t>(1, std::min(MOST_PARTS, PARTIAL_BYTES / bytes));
  c->workspace_bytes = (size_t)((c->max_parts * bytes + 255) / 256 * 256);
  *out = c;
  return SIGNMUON_OK;
}

int signmuon_layernorm_workspace_bytes(const signmuon_layernorm* c, size_t* workspace) {
  if (!c || !workspace) return SIGNMUON_ERR_INVALID_ARG;
  *workspace = c->workspace_bytes;
  return SIGNMUON_OK;
}

int signmuon_layernorm_bind(signmuon_layernorm* c, void* dev_workspace, size_t workspace_bytes, void*) {
  if (!c || (!dev_workspace && workspace_bytes)) return SIGNMUON_ERR_INVALID_ARG;
  if (dev_workspace && workspace_bytes < c->workspace_bytes) return SIGNMUON_ERR_BUFFER_TOO_SMALL;
  if (reinterpret_cast<uintptr_t>(dev_workspace) & 255) return SIGNMUON_ERR_MISALIGNED;
  int dev = 0, major = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
    cudaGetLastError();
    return SIGNMUON_ERR_CUDA;
  }
  if (major != 10) return SIGNMUON_ERR_UNSUPPORTED_ARCH;
  c->sms = sms;
  for (auto& f : c->fits) f = 0;
  c->workspace = static_cast<float*>(dev_workspace);
  c->bound = true;
  c->sticky = SIGNMUON_OK;
  return SIGNMUON_OK;
}

int signmuon_layernorm_forward(signmuon_layernorm* c, const signmuon_layernorm_forward_args* args, void* cuda_stream) {
  if (!c || !args) return SIGNMUON_ERR_INVALID_ARG;
  if (!c->bound) return SIGNMUON_ERR_NOT_BOUND;
  if (c->sticky != SIGNMUON_OK) return c->sticky;
  const signmuon_layernorm_forward_args& q = *args;
  const int64_t cols = c->cfg.cols;
  if (q.rows < 0 || q.rows > INT32_MAX) return SIGNMUON_ERR_BAD_SHAPE;
  if (q.rows == 0) return SIGNMUON_OK;
  if (!q.x || !q.y || (q.residual && !q.sum)) return SIGNMUON_ERR_INVALID_ARG;
  Forward a = {};
  a.x = q.x; a.residual = q.residual; a.gamma = q.gamma; a.beta = q.beta; a.y = q.y; a.sum = q.sum;
  a.mean = q.mean; a.rstd = q.rstd;
  a.ld_x = q.ld_x ? q.ld_x : cols;
  a.ld_residual = q.ld_residual ? q.ld_residual : cols;
  a.ld_y = q.ld_y ? q.ld_y : cols;
  a.ld_sum = q.ld_sum ? q.ld_sum : cols;
  if (a.ld_x < cols || a.ld_y < cols || (q.residual && (a.ld_residual < cols || a.ld_sum < cols))) return SIGNMUON_ERR_BAD_SHAPE;
  a.rows = q.rows;
  a.cols = cols;
  a.weight_bf16 = c->cfg.weight_dtype == SIGNMUON_BF16;
  a.eps = c->cfg.eps;
  a.inv_cols = (float)(1.0 / (double)cols);
  const int ab = entry_bytes(c->cfg.act_dtype), wb = entry_bytes(c->cfg.weight_dtype), unit = 16 / ab;
  const auto at = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
  const uintptr_t acts = at(q.x) | at(q.y) | (q.residual ? at(q.residual) | at(q.sum) : 0);
  const uintptr_t weights = at(q.gamma) | at(q.beta);
  if (acts % ab || weights % wb || (at(q.mean) | at(q.rstd)) % 4) return SIGNMUON_ERR_MISALIGNED;
  const int64_t distances = a.ld_x | a.ld_y | (q.residual ? a.ld_residual | a.ld_sum : 0);
  const bool vec = (acts | weights) % 16 == 0 && (distances | cols) % unit == 0;
  const bool half = c->cfg.act_dtype == SIGNMUON_BF16;
  Choice f = half ? (vec ? choose_forward<bf16, true>(cols) : choose_forward<bf16, false>(cols))
                  : (vec ? choose_forward<float, true>(cols) : choose_forward<float, false>(cols));
  int64_t grid = (q.rows + f.rows - 1) / f.rows;
  cudaError_t e = cudaSuccess;
  if (vec && cols > 16 * 8 && cols <= 512 * 16) {
    const int arrays = q.residual ? 2 : 1;
    const Choice ring = half ? choose_forward_ring<bf16>(cols, arrays) : choose_forward_ring<float>(cols, arrays);
    const int64_t blocks = (int64_t)c->resident(ring, arrays == 2 ? c->FORWARD_RESIDUAL : c->FORWARD) * c->sms;
    if (blocks == 0) e = cudaErrorUnknown;
    else if (q.rows > 2 * blocks * ring.rows) {       // every group meets three rows or more: fetching ahead pays
      f = ring;
      grid = blocks;
    }
  }
  void* params[] = {&a};
  if (e == cudaSuccess)
    e = launch_early(f.fn, dim3((unsigned)grid), dim3(f.threads), f.shared, params, reinterpret_cast<cudaStream_t>(cuda_stream));
  if (e != cudaSuccess) {
    cudaGetLastError();
    c->sticky = SIGNMUON_ERR_CUDA;
  }
  return c->sticky;
}

int signmuon_layernorm_backward(signmuon_layernorm* c, const signmuon_layernorm_backward_args* args, void* cuda_stream) {
  if (!c || !args) return SIGNMUON_ERR_INVALID_ARG;
  if (!c->bound || !c->workspace) return SIGNMUON_ERR_NOT_BOUND;
  if (c->sticky != SIGNMUON_OK) return c->sticky;
  const signmuon_layernorm_backward_args& q = *args;
  const int64_t cols = c->cfg.cols, workers = c->cfg.num_workers;
  if (q.rows < 0 || q.rows > INT32_MAX) return SIGNMUON_ERR_BAD_SHAPE;
  if (q.rows % workers) return SIGNMUON_ERR_INVALID_ARG;
  if (q.rows && (!q.dy || !q.s || !q.mean || !q.rstd || !q.dx)) return SIGNMUON_ERR_INVALID_ARG;
  Backward a = {};
  a.dy = q.dy; a.s = q.s; a.gamma = q.gamma; a.dsum = q.dsum; a.mean = q.mean; a.rstd = q.rstd;
  a.dx = q.dx; a.dgamma = q.dgamma; a.dbeta = q.dbeta;
  a.partials = c->workspace;
  a.ld_dy = q.ld_dy ? q.ld_dy : cols;
  a.ld_s = q.ld_s ? q.ld_s : cols;
  a.ld_dsum = q.ld_dsum ? q.ld_dsum : cols;
  a.ld_dx = q.ld_dx ? q.ld_dx : cols;
  a.dgamma_stride = q.dgamma_stride ? q.dgamma_stride : cols;
  a.dbeta_stride = q.dbeta_stride ? q.dbeta_stride : cols;
  if (a.ld_dy < cols || a.ld_s < cols || a.ld_dx < cols || (q.dsum && a.ld_dsum < cols) || (q.dgamma && a.dgamma_stride < cols) ||
      (q.dbeta && a.dbeta_stride < cols))
    return SIGNMUON_ERR_BAD_SHAPE;
  a.rows_each = q.rows / workers;
  a.cols = cols;
  a.padded = (cols + 3) / 4 * 4;
  a.weight_bf16 = c->cfg.weight_dtype == SIGNMUON_BF16;
  a.grad_bf16 = c->cfg.grad_dtype == SIGNMUON_BF16;
  a.inv_cols = (float)(1.0 / (double)cols);
  const int ab = entry_bytes(c->cfg.act_dtype), wb = entry_bytes(c->cfg.weight_dtype), gb = entry_bytes(c->cfg.grad_dtype);
  const int unit = 16 / ab;
  const auto at = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
  const uintptr_t acts = at(q.dy) | at(q.s) | at(q.dx) | at(q.dsum);
  if (acts % ab || at(q.gamma) % wb || (at(q.dgamma) | at(q.dbeta)) % gb || (at(q.mean) | at(q.rstd)) % 4)
    return SIGNMUON_ERR_MISALIGNED;
  const int64_t distances = a.ld_dy | a.ld_s | a.ld_dx | (q.dsum ? a.ld_dsum : 0);
  const bool vec = (acts | at(q.gamma)) % 16 == 0 && (distances | cols) % unit == 0;
  const bool half = c->cfg.act_dtype == SIGNMUON_BF16;
  const int arrays = q.dsum ? 3 : 2;
  const Choice f = half ? (vec ? choose_backward<bf16, true>(cols, arrays) : choose_backward<bf16, false>(cols, arrays))
                        : (vec ? choose_backward<float, true>(cols, arrays) : choose_backward<float, false>(cols, arrays));
  const bool weights = q.dgamma || q.dbeta;
  // One wave of thread blocks, every group with a row at least; the columns' kernel shares a row out over several.  Where the
  // workers do not divide the wave, the SMs that are left over have nothing to do, and from half a wave on there is one thread
  // block a worker: 14.8 k rows of 768 take 19.1 us for 64 workers, 21.4 us for 75, 18.4 us for 100, 17.2 us for 148.
  const int64_t across = COLUMN_THREADS * (vec ? unit : 1), side = (cols + across - 1) / across;
  const int blocks = f.wide ? 8 : c->resident(f, !vec ? c->BACKWARD_SINGLE : q.dsum ? c->BACKWARD_DSUM : c->BACKWARD);
  const int64_t target = std::min<int64_t>(c->max_parts, f.wide ? (c->sms * 8 + side - 1) / side : (int64_t)c->sms * blocks);
  // rows of a part: the columns' kernel writes two floats for each that it sums; up to three rows a group stay with one thread
  // block, since two more rows cost it less than the launch of the joining kernel
  const int64_t least = f.wide ? 16 : a.rows_each <= 3 * f.rows ? 3 * f.rows : f.rows;
  const int64_t most = (a.rows_each + least - 1) / least;
  a.parts = (int32_t)std::max<int64_t>(1, std::min(target / workers, most));
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  void* params[] = {&a};
  cudaError_t e = blocks ? cudaSuccess : cudaErrorUnknown;
  if (e != cudaSuccess) {
  } else if (f.wide) {
    if (weights) {
      void* columns = half ? (vec ? (void*)columns_kernel<bf16, 8> : (void*)columns_kernel<bf16, 1>)
                           : (vec ? (void*)columns_kernel<float, 4> : (void*)columns_kernel<float, 1>);
      const dim3 grid((unsigned)side, (unsigned)a.parts, (unsigned)workers);
      e = launch_early(columns, grid, dim3(COLUMN_THREADS), 0, params, stream);
    }
    if (e == cudaSuccess && q.rows) e = launch_early(f.fn, dim3((unsigned)q.rows), dim3(f.threads), 0, params, stream);
  } else if (q.rows || weights) {
    e = launch_early(f.fn, dim3((unsigned)(workers * a.parts)), dim3(f.threads), f.shared, params, stream);
  }
  if (e == cudaSuccess && weights && a.parts > 1)
    e = launch_early((void*)join_kernel, dim3((unsigned)((cols + 127) / 128), (unsigned)workers, 2), dim3(32, 8), 0, params, stream);
  if (e != cudaSuccess) {
    cudaGetLastError();
    c->sticky = SIGNMUON_ERR_CUDA;
  }
  return c->sticky;
}

void signmuon_layernorm_destroy(signmuon_layernorm* c) { delete c; }

}  // extern "C"
