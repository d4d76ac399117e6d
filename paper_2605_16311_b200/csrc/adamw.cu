// AdamW over many tensors at once, with states in 32 or in 8 bits, and the norm of the mean gradient.
//
//   g = (scale / M) sum_k G_k
//   m <- b1 m + (1 - b1) g,   v <- b2 v + (1 - b2) g^2
//   W <- (1 - lr wd) W - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Every warp owns one block of 256 consecutive entries of one tensor at a time, which is also the block that shares a
// scale when the states are held in 8 bits.  The table of tensors (pointers, sizes, decay) travels in the kernel's
// parameters: nothing is uploaded and nothing is kept from one call for the next, so a call may name new tensors every
// time and can be captured in a CUDA graph.  The step number t and the powers of the betas live in the state buffer and
// are advanced by the last block of a step, so that a replayed graph goes on counting.
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "../../include/signmuon.h"
#include "common.cuh"

using namespace signmuon;

namespace {

constexpr int BLOCK = 256;                    // entries of a warp's unit of work, and of a scale of the 8-bit states
constexpr int THREADS = 256;
constexpr int WARPS = THREADS / 32;
constexpr int SPAN = BLOCK * WARPS;           // entries between two blocks of a warp in a tile
// A thread block's unit of work, a tile, is one block a warp.  Where the ring of the 8-bit states serves (below), it is two
// or, where the shared memory has room for them (bf16 weights and gradients), four blocks a warp.
__host__ __device__ constexpr int passes_of(int ring) { return ring ? ring : 1; }
// The ring pays from this many blocks on (2 M entries): 2.4 M float32 entries take 9.5 us with it and 10.6 us without, 1.2 M
// 6.8 and 6.0 us, 20 k 4.8 and 3.5 us.
constexpr int64_t RING_BLOCKS = 8192;
constexpr size_t HEADER_BYTES = 256;
constexpr int64_t MAX_ENTRIES = int64_t(1) << 40;
constexpr int MAX_GRID = 148 * 16;            // partial sums of the norm that one launch may write
constexpr float E4M3_MAX = 448.f;
constexpr float E4M3_LEAST = 0x1p-9f;         // least positive E4M3 number
constexpr float TINY = 0x1p-100f;             // a block whose largest value is below this is held as zeros

// First bytes of the state buffer.  The factors are those of the NEXT step.
struct Header {
  int64_t step;                               // steps taken
  double pow_one, pow_two;                    // b1^(step + 1), b2^(step + 1)
  float inv_correction;                       // 1 / (1 - b1^(step + 1))
  float inv_root_correction;                  // 1 / sqrt(1 - b2^(step + 1))
  uint32_t ticket;                            // blocks of the running step that have finished
};

struct Tensor {
  void* w;
  const void* g;
  int64_t numel;
  int64_t grad_stride;                        // entries between two workers' gradients
  int64_t state_at;                           // first entry inside the state regions (a multiple of BLOCK)
  uint32_t tile0;                             // first tile of the launch that belongs to this tensor
  float decay;
  uint32_t kind;                              // KIND_*
  uint32_t reserved;
};
enum : uint32_t { KIND_W_BF16 = 1, KIND_G_BF16 = 2, KIND_VEC = 4 };

template <int CAP>
struct Table {
  Tensor t[CAP];
  int32_t n;
};

struct Step {
  uint8_t* state;
  int64_t m_at, v_at, ms_at, vs_at, master_at;   // byte offsets of the state regions
  const float* scale;                            // optional device scalar
  uint32_t tiles;
  int32_t workers;
  int32_t block_bytes;                           // room of a block in the ring
  float lr, b1, omb1, b2, omb2, eps, inv_workers;
  float minus_zero;                              // (product() below)
  float fast_above;                              // (8-bit states) blocks whose largest v is above this take their roots from roots_of
  double beta_one, beta_two;
  int32_t advance;                               // the launch that ends the step
};

struct Norm {
  double* partials;                              // this launch's first partial sum
  const double* all;                             // every launch's
  uint32_t n_all;
  uint32_t* ticket;
  float* out;
  uint32_t tiles;
  int32_t workers;
  float inv_workers, max_norm;
  int32_t last;
};

// The entries of a warp's block that a lane holds.  OCTET: eight neighbours, one 16-byte access of bf16.  QUAD: twice four,
// two 16-byte accesses of float32 that lie side by side over the warp (eight neighbours would touch half a sector each: with
// more than 64 KB an SM in flight, the other half was fetched again - a step on 33.5 M float32 entries took 174 us, not 148).
// SCALAR: every 32nd, for tensors that are not aligned and for their ends.
enum Layout { SCALAR, OCTET, QUAD };
__device__ __forceinline__ int scalar_entry(int lane, int j) { return j * 32 + lane; }

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(bf16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(bf16* p, float x) { *p = __float2bfloat16_rn(x); }

// Eight entries of a lane as they were loaded, so that many loads can be in flight at four or eight registers each.
template <typename T> struct Raw;
template <> struct Raw<float> { float4 a, b; };
template <> struct Raw<bf16> { uint2 a, b; };
template <Layout L>
__device__ __forceinline__ Raw<float> load_raw(const float* p, int lane) {
  static_assert(L == QUAD, "float32 is read by fours");
  return {__ldcs(reinterpret_cast<const float4*>(p) + lane), __ldcs(reinterpret_cast<const float4*>(p) + 32 + lane)};
}
template <Layout L>
__device__ __forceinline__ Raw<bf16> load_raw(const bf16* p, int lane) {
  if constexpr (L == QUAD) return {__ldcs(reinterpret_cast<const uint2*>(p) + lane), __ldcs(reinterpret_cast<const uint2*>(p) + 32 + lane)};
  const uint4 v = __ldcs(reinterpret_cast<const uint4*>(p) + lane);
  return {make_uint2(v.x, v.y), make_uint2(v.z, v.w)};
}
__device__ __forceinline__ void unpack(const Raw<float>& r, float (&x)[8]) {
  x[0] = r.a.x; x[1] = r.a.y; x[2] = r.a.z; x[3] = r.a.w; x[4] = r.b.x; x[5] = r.b.y; x[6] = r.b.z; x[7] = r.b.w;
}
__device__ __forceinline__ void unpack(const Raw<bf16>& r, float (&x)[8]) {
  const uint32_t w[4] = {r.a.x, r.a.y, r.b.x, r.b.y};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(w[e] << 16);
    x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
  }
}
template <Layout L, typename T>
__device__ __forceinline__ void load(const T* p, int lane, int valid, float (&x)[8]) {
  if constexpr (L != SCALAR) {
    unpack(load_raw<L>(p, lane), x);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = scalar_entry(lane, j) < valid ? as_float(__ldcs(p + scalar_entry(lane, j))) : 0.f;
  }
}
__device__ __forceinline__ void store_quads(float* p, int lane, const float (&x)[8]) {
  __stcs(reinterpret_cast<float4*>(p) + lane, make_float4(x[0], x[1], x[2], x[3]));
  __stcs(reinterpret_cast<float4*>(p) + 32 + lane, make_float4(x[4], x[5], x[6], x[7]));
}
__device__ __forceinline__ void store_quads(bf16* p, int lane, const float (&x)[8]) {
  __stcs(reinterpret_cast<uint2*>(p) + lane, make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])));
  __stcs(reinterpret_cast<uint2*>(p) + 32 + lane, make_uint2(pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])));
}
template <Layout L, typename T>
__device__ __forceinline__ void store(T* p, int lane, int valid, const float (&x)[8]) {
  if constexpr (L != SCALAR) {
    store_quads(p, lane, x);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (scalar_entry(lane, j) < valid) put(p + scalar_entry(lane, j), x[j]);
  }
}

// Adds N workers' gradients, all of them in flight together.
template <int N, typename GT, Layout L>
__device__ __forceinline__ void add_gradients(const GT* g, int64_t stride, int lane, int valid, float (&x)[8]) {
  float y[8];
  if constexpr (L != SCALAR) {
    Raw<GT> r[N];
#pragma unroll
    for (int k = 0; k < N; ++k) r[k] = load_raw<L>(g + k * stride, lane);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      unpack(r[k], y);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] += y[j];
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      load<L>(g + k * stride, lane, valid, y);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] += y[j];
    }
  }
}
// Sum of the workers' gradients, in their order.  Groups of 16 (eight in float32, for the registers' sake) are in flight
// together, then what is left by halves: a loop unrolled by four would take the last three of 16 workers one latency each
// (the norm of 39.4 M entries of 16 workers: 201 us then, 192 us so; 25 small tensors: 5.3 and 4.9 us).
template <typename GT, Layout L>
__device__ __forceinline__ void sum_gradients(const GT* g, int64_t stride, int workers, int lane, int valid, float (&x)[8]) {
  constexpr int MOST = L == SCALAR ? 1 : sizeof(GT) == 2 ? 16 : 8;
  if (workers == 1) {                    // (straight, so that what the caller loads next is in flight beside it)
    load<L>(g, lane, valid, x);
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = 0.f;
  int k = workers;
#pragma unroll 1
  for (; k >= MOST; k -= MOST, g += MOST * stride) add_gradients<MOST, GT, L>(g, stride, lane, valid, x);
  if constexpr (MOST > 8)
    if (k & 8) { add_gradients<8, GT, L>(g, stride, lane, valid, x); g += 8 * stride; }
  if constexpr (MOST > 4)
    if (k & 4) { add_gradients<4, GT, L>(g, stride, lane, valid, x); g += 4 * stride; }
  if constexpr (MOST > 2)
    if (k & 2) { add_gradients<2, GT, L>(g, stride, lane, valid, x); g += 2 * stride; }
  if constexpr (MOST > 1)
    if (k & 1) add_gradients<1, GT, L>(g, stride, lane, valid, x);
}

// What a step's launch derives from its scalars.
struct Factors {
  float gs;              // scale / M
  float step_size;       // lr / (1 - b1^t)
  float inv_root;        // 1 / sqrt(1 - b2^t)
  bool first;            // t == 1: master weights come from W
};

// W's new value.  Root, reciprocal and product are approximate to 2^-22.  The second moment may be denormal (gradients of
// 1e-18 and less) and still count beside a small eps; the denominator is at least eps, which is no less than 2^-120.
__device__ __forceinline__ float root_of(float v) {
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float inverse(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float updated(float w, float m, float root, float keep, const Step& s, const Factors& f) {
  return fmaf(-f.step_size, m * inverse(fmaf(root, f.inv_root, s.eps)), fmaf(keep, w, w));
}

// ---- states in 32 bits
template <typename WT, typename GT, bool MASTER, Layout L>
__device__ __forceinline__ void update_block32(const Tensor& t, const Step& s, const Factors& f, int64_t at, int valid, int lane) {
  float g[8], m[8], v[8], w[8];
  const int64_t sat = t.state_at + at;
  WT* wp = static_cast<WT*>(t.w) + at;
  float* mp = reinterpret_cast<float*>(s.state + s.m_at) + sat;
  float* vp = reinterpret_cast<float*>(s.state + s.v_at) + sat;
  float* master = MASTER ? reinterpret_cast<float*>(s.state + s.master_at) + sat : nullptr;
  const GT* gp = static_cast<const GT*>(t.g) + at;
  sum_gradients<GT, L>(gp, t.grad_stride, s.workers, lane, valid, g);
  if (MASTER && !f.first) load<L>(master, lane, valid, w);
  else load<L>(wp, lane, valid, w);
  load<L>(mp, lane, valid, m);
  load<L>(vp, lane, valid, v);
  const float keep = -s.lr * t.decay;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float x = g[j] * f.gs;
    m[j] = fmaf(s.b1, m[j], s.omb1 * x);
    v[j] = fmaf(s.b2, v[j], s.omb2 * (x * x));
    w[j] = updated(w[j], m[j], root_of(v[j]), keep, s, f);
  }
  if (MASTER) store<L>(master, lane, valid, w);
  store<L>(wp, lane, valid, w);
  store<L>(mp, lane, valid, m);
  store<L>(vp, lane, valid, v);
}

// ---- states in 8 bits: a block's values are E4M3 numbers times the block's scale (largest magnitude / 448).
__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return (uint32_t)hi << 16 | lo;
}
__device__ __forceinline__ void from_e4m3x4(uint32_t v, float* x) {
  uint32_t lo, hi;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"((uint16_t)(v & 0xffffu)));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"((uint16_t)(v >> 16)));
  asm("{.reg .f16 a, b; mov.b32 {a, b}, %2; cvt.f32.f16 %0, a; cvt.f32.f16 %1, b;}" : "=f"(x[0]), "=f"(x[1]) : "r"(lo));
  asm("{.reg .f16 a, b; mov.b32 {a, b}, %2; cvt.f32.f16 %0, a; cvt.f32.f16 %1, b;}" : "=f"(x[2]), "=f"(x[3]) : "r"(hi));
}
template <Layout L>
__device__ __forceinline__ uint2 load_codes(const uint8_t* p, int lane) {
  if constexpr (L == QUAD) return make_uint2(__ldcs(reinterpret_cast<const uint32_t*>(p) + lane), __ldcs(reinterpret_cast<const uint32_t*>(p) + 32 + lane));
  // (a block's codes are whole in the state buffer, also behind a tensor's end)
  return make_uint2(p[lane] | p[32 + lane] << 8 | p[64 + lane] << 16 | (uint32_t)p[96 + lane] << 24,
                    p[128 + lane] | p[160 + lane] << 8 | p[192 + lane] << 16 | (uint32_t)p[224 + lane] << 24);
}
template <Layout L>
__device__ __forceinline__ void store_codes(uint8_t* p, int lane, uint2 codes) {
  const uint32_t a = codes.x, b = codes.y;
  if constexpr (L == QUAD) {
    __stcs(reinterpret_cast<uint32_t*>(p) + lane, a);
    __stcs(reinterpret_cast<uint32_t*>(p) + 32 + lane, b);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      p[32 * j + lane] = (uint8_t)(a >> 8 * j);
      p[128 + 32 * j + lane] = (uint8_t)(b >> 8 * j);
    }
  }
}
// Correctly rounded roots of a pair in (2^-100, 2^120), and 0 of 0.  Newton's step for x^2 = v from an approximate root x:
// the residual v - x^2 is exact in a fused multiply-add, and what the step leaves of the error, its square, never decides the
// last bit: every float32 in the range was compared with __fsqrt_rn on a B200.  (2^-126 is added where 0 would divide: smaller
// v lose digits, below 2^-117 more than 2^-20 of the root, but never more than 2^-63.  The codes do not see that: such an entry
// is held as the least positive number beside the block's largest, which is above 2^-60.  W's step does not either while that
// error over the root's correction is at most 2^-23 of eps; for a smaller eps the roots are taken one by one: fast_above is
// infinite then.  It is a constant of the launch: a flag in a register took 320 us for 157 M entries, this 309 us.)
__device__ __forceinline__ float_pair roots_of(float_pair v) {
  const float2 a = halves(pair_add(v, pair_of(0x1p-126f)));
  float y0, y1;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y0) : "f"(a.x));
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y1) : "f"(a.y));
  const float_pair y = pair_of(y0, y1), x = pair_mul(v, y);
  return pair_fma(pair_fma(x, pair_mul(x, pair_of(-1.f)), v), pair_mul(y, pair_of(0.5f)), x);
}
__device__ __noinline__ float root_of_any(float v) { return __fsqrt_rn(v); }

// The update of a block from what was loaded, by LANES lanes with 2 N entries each (LANES 16: a half warp, with another block
// in the other half).  Everything that reaches the state is rounded operation by operation (no fused multiply-add, correctly
// rounded root and quotients): the next codes follow from the inputs bit for bit in any float32 restatement of the formulas.
// A code that fell to the other side would be 6 % off in every step that follows.  Arithmetic runs on pairs: with 10 bytes an
// entry to move, the issue of instructions counts as much as the memory does.
//   in: g gradient sums, w weights, mc and rc codes (four a word), ms and rs scales
//   out: w new weights, mc and rc new codes; one lane in LANES holds each new scale (store_scales)
template <int N> struct Entries {
  float_pair g[N], w[N];
  uint32_t mc[N / 2], rc[N / 2];
  float ms, rs;
};
// Largest magnitude over the values of a warp, or of each half of it; NaN if one is NaN.  redux takes the halves one after
// the other.  Where issue bounds the kernel (bf16, 157 M entries) that costs: 299 us, 282 us with shuffles.  Where the memory
// does (float32 weights or master copies, 39.4 M entries) the shuffles only let the warps crowd it: 116 us, 108 us with redux.
enum Reduce { REDUX, SHUFFLE };
template <int N, int LANES, Reduce R>
__device__ __forceinline__ float largest(const float_pair (&x)[N], int lane) {
  float t;
  const float2 a = halves(x[0]);
  asm("max.NaN.abs.f32 %0, %1, %2, %2;" : "=f"(t) : "f"(a.x), "f"(a.y));
#pragma unroll
  for (int j = 1; j < N; ++j) {
    const float2 b = halves(x[j]);
    asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(t) : "f"(b.x), "f"(b.y));
  }
  if constexpr (R == REDUX) {
    asm("redux.sync.max.abs.NaN.f32 %0, %1, %2;" : "=f"(t) : "f"(t), "r"(LANES == 32 ? 0xffffffffu : 0xffffu << (lane & 16)));
  } else {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) {
      const float u = __shfl_xor_sync(0xffffffffu, t, o);
      asm("max.NaN.f32 %0, %0, %1;" : "+f"(t) : "f"(u));
    }
  }
  return t;
}
template <int N, int LANES, Reduce R>
__device__ __forceinline__ float update_entries(Entries<N>& x, const Tensor& t, const Step& s, const Factors& f, int lane) {
  // a product that the assembler cannot merge with the addition behind it (it does not know that the third operand is -0)
  const float_pair none = pair_of(s.minus_zero);
  const auto product = [&](float_pair a, float_pair b) { return pair_fma(a, b, none); };
  const float_pair m_scale = pair_of(x.ms), r_scale = pair_of(x.rs), gs = pair_of(f.gs);
  const float_pair b1 = pair_of(s.b1), omb1 = pair_of(s.omb1), b2 = pair_of(s.b2), omb2 = pair_of(s.omb2);
  float_pair m[N], r[N];
#pragma unroll
  for (int j = 0; j < N; j += 2) {
    float mq[4], rq[4];
    from_e4m3x4(x.mc[j / 2], mq);
    from_e4m3x4(x.rc[j / 2], rq);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float_pair y = pair_mul(x.g[j + i], gs);
      m[j + i] = pair_add(product(b1, pair_mul(pair_of(mq[2 * i], mq[2 * i + 1]), m_scale)), product(omb1, y));
      const float_pair a = pair_mul(pair_of(rq[2 * i], rq[2 * i + 1]), r_scale);
      r[j + i] = pair_add(product(b2, pair_mul(a, a)), product(omb2, pair_mul(y, y)));
    }
  }
  const float vt = largest<N, LANES, R>(r, lane);
  float rt;
  if (__all_sync(0xffffffffu, vt > s.fast_above && vt < 0x1p120f)) {
    rt = halves(roots_of(pair_of(vt))).x;
#pragma unroll
    for (int j = 0; j < N; ++j) r[j] = roots_of(r[j]);
  } else {
    rt = root_of_any(vt);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float2 v = halves(r[j]);
      r[j] = pair_of(root_of_any(v.x), root_of_any(v.y));
    }
  }
  const float_pair inv_root = pair_of(f.inv_root), eps = pair_of(s.eps), down = pair_of(-f.step_size), less = pair_of(-s.lr * t.decay);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const float2 den = halves(pair_fma(r[j], inv_root, eps));
    const float_pair step = pair_mul(m[j], pair_of(inverse(den.x), inverse(den.y)));
    x.w[j] = pair_fma(down, step, pair_fma(less, x.w[j], x.w[j]));
  }
  // 448 / top and top / 448 of both: one division, by four lanes
  const float mt = largest<N, LANES, R>(m, lane), top = lane & 1 ? rt : mt;
  const float quotient = top < TINY ? 0.f : __fdiv_rn(lane & 2 ? top : E4M3_MAX, lane & 2 ? E4M3_MAX : top);
  const int first = LANES == 32 ? 0 : lane & 16;
  const float_pair mi = pair_of(__shfl_sync(0xffffffffu, quotient, first)), ri = pair_of(__shfl_sync(0xffffffffu, quotient, first + 1));
  const float least = rt < TINY ? 0.f : E4M3_LEAST;
#pragma unroll
  for (int j = 0; j < N; j += 2) {
    float mx[4], rx[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float2 a = halves(pair_mul(m[j + i], mi)), b = halves(pair_mul(r[j + i], ri)), q = halves(r[j + i]);
      mx[2 * i] = a.x; mx[2 * i + 1] = a.y;
      // a positive root never becomes zero: m over it would explode
      rx[2 * i] = q.x > 0.f ? fmaxf(b.x, least) : b.x;
      rx[2 * i + 1] = q.y > 0.f ? fmaxf(b.y, least) : b.y;
    }
    x.mc[j / 2] = to_e4m3x4(mx[0], mx[1], mx[2], mx[3]);
    x.rc[j / 2] = to_e4m3x4(rx[0], rx[1], rx[2], rx[3]);
  }
  return quotient;                                    // lanes 2 and 3 of the group: the new scales of m and of r
}
template <int LANES>
__device__ __forceinline__ void store_scales(const Step& s, int64_t block, int lane, float quotient) {
  if ((lane & (LANES - 2)) == 2) reinterpret_cast<float*>(s.state + (lane & 1 ? s.vs_at : s.ms_at))[block] = quotient;
}
template <typename WT, typename GT, bool MASTER, Layout L>
__device__ __forceinline__ void update_block8(const Tensor& t, const Step& s, const Factors& f, int64_t at, int valid, int lane) {
  const int64_t sat = t.state_at + at;
  uint8_t* mp = s.state + s.m_at + sat;
  uint8_t* rp = s.state + s.v_at + sat;
  WT* wp = static_cast<WT*>(t.w) + at;
  float* master = MASTER ? reinterpret_cast<float*>(s.state + s.master_at) + sat : nullptr;
  Entries<4> x;
  float g[8], w[8];
  const uint2 mc = load_codes<L>(mp, lane), rc = load_codes<L>(rp, lane);
  x.ms = __ldcs(reinterpret_cast<const float*>(s.state + s.ms_at) + sat / BLOCK);
  x.rs = __ldcs(reinterpret_cast<const float*>(s.state + s.vs_at) + sat / BLOCK);
  if (MASTER && !f.first) load<L>(master, lane, valid, w);
  else load<L>(wp, lane, valid, w);
  sum_gradients<GT, L>(static_cast<const GT*>(t.g) + at, t.grad_stride, s.workers, lane, valid, g);
  x.mc[0] = mc.x; x.mc[1] = mc.y;
  x.rc[0] = rc.x; x.rc[1] = rc.y;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x.g[j] = pair_of(g[2 * j], g[2 * j + 1]);
    x.w[j] = pair_of(w[2 * j], w[2 * j + 1]);
  }
  const float quotient = update_entries<4, 32, REDUX>(x, t, s, f, lane);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 q = halves(x.w[j]);
    w[2 * j] = q.x; w[2 * j + 1] = q.y;
  }
  if (MASTER) store<L>(master, lane, valid, w);
  store<L>(wp, lane, valid, w);
  store_codes<L>(mp, lane, make_uint2(x.mc[0], x.mc[1]));
  store_codes<L>(rp, lane, make_uint2(x.rc[0], x.rc[1]));
  store_scales<32>(s, sat / BLOCK, lane, quotient);
}

// A warp's part of a tile, or what the tensor's end leaves of it.
template <int BITS, int PASSES, typename WT, typename GT, bool MASTER, bool VEC>
__device__ __forceinline__ void update_warp(const Tensor& t, const Step& s, const Factors& f, int64_t at, int lane) {
#pragma unroll 1
  for (int n = 0; n < PASSES; ++n, at += SPAN) {
    if (at >= t.numel) return;
    const bool whole = at + BLOCK <= t.numel;
    const int valid = whole ? BLOCK : (int)(t.numel - at);
    if (VEC && whole) {
      if constexpr (BITS == 8) update_block8<WT, GT, MASTER, QUAD>(t, s, f, at, valid, lane);
      else update_block32<WT, GT, MASTER, QUAD>(t, s, f, at, valid, lane);
    } else {
      if constexpr (BITS == 8) update_block8<WT, GT, MASTER, SCALAR>(t, s, f, at, valid, lane);
      else update_block32<WT, GT, MASTER, SCALAR>(t, s, f, at, valid, lane);
    }
  }
}

// ---- 8-bit states, aligned tensors, few workers: a warp's blocks of the next tile are on their way through shared memory
// (cp.async, 16 bytes a lane side by side) while it works on this one.  The warps share nothing, so no barrier is needed.
// What a block brings: weights, every worker's gradients, the codes of m and of r.
__device__ __forceinline__ void copy16(void* shared, const void* global) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(shared)), "l"(global) : "memory");
}
constexpr int STAGES = 2;
constexpr size_t RING_LIMIT = 100 * 1024;     // two thread blocks an SM
struct Ahead {
  int tensor;
  int64_t at;
  bool ready;                                 // the warp's blocks of the tile are on their way, or there
  float scale;                                // lane 2 n: m's scale in block n, lane 2 n + 1: r's
};
// 256 entries of 2 or 4 bytes
__device__ __forceinline__ void copy_block(uint8_t* to, const char* from, bool wide, int lane) {
  copy16(to + lane * 16, from + lane * 16);
  if (wide) copy16(to + 512 + lane * 16, from + 512 + lane * 16);
}
template <bool MASTER, int PASSES>
__device__ __forceinline__ void fetch_tile(const Tensor& t, const Step& s, const Factors& f, uint8_t* stage, int lane, Ahead& a) {
  a.ready = (t.kind & KIND_VEC) && a.at + (PASSES - 1) * SPAN + BLOCK <= t.numel;
  if (!a.ready) return;
  const int64_t sat = t.state_at + a.at;
  const bool half = t.kind & KIND_W_BF16, from_master = MASTER && half && !f.first;
  const bool wide_w = from_master || !half, wide_g = !(t.kind & KIND_G_BF16);
  const char* w = from_master ? reinterpret_cast<const char*>(s.state + s.master_at) + sat * 4
                              : static_cast<const char*>(t.w) + a.at * (half ? 2 : 4);
  const char* g = static_cast<const char*>(t.g) + a.at * (wide_g ? 4 : 2);
  const uint8_t* codes = s.state + (lane < 16 ? s.m_at : s.v_at) + sat + (lane & 15) * 16;
  // (through L1: a line holds the scales that the thread block's other warps read)
  a.scale = *(reinterpret_cast<const float*>(s.state + (lane & 1 ? s.vs_at : s.ms_at)) + sat / BLOCK + (lane / 2 % PASSES) * (SPAN / BLOCK));
#pragma unroll
  for (int n = 0; n < PASSES; ++n, stage += s.block_bytes) {
    uint8_t* to = stage;
    copy16(to + lane * 16, codes + n * SPAN);
    to += 512;
    copy_block(to, w + n * SPAN * (wide_w ? 4 : 2), wide_w, lane);
    to += wide_w ? 1024 : 512;
    copy_block(to, g + n * SPAN * (wide_g ? 4 : 2), wide_g, lane);
    for (int k = 1; k < s.workers; ++k) {
      to += wide_g ? 1024 : 512;
      copy_block(to, g + (k * t.grad_stride + n * SPAN) * (wide_g ? 4 : 2), wide_g, lane);
    }
  }
}
// A lane's 16 entries of a block that a half warp works on (l: the lane in it): twice eight neighbours (OCTET) or four times
// four (QUAD), so that the half warp's accesses lie side by side.
template <Layout L>
__device__ __forceinline__ void read_block(const uint8_t* from, bool wide, int l, float_pair (&x)[8]) {
  if (wide) {
    const ulonglong2* p = reinterpret_cast<const ulonglong2*>(from);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const ulonglong2 v = p[L == QUAD ? 16 * i + l : 32 * (i / 2) + 2 * l + i % 2];
      x[2 * i] = v.x; x[2 * i + 1] = v.y;
    }
    return;
  }
  uint32_t v[8];
  if constexpr (L == QUAD) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint2 q = reinterpret_cast<const uint2*>(from)[16 * i + l];
      v[2 * i] = q.x; v[2 * i + 1] = q.y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint4 q = reinterpret_cast<const uint4*>(from)[16 * i + l];
      v[4 * i] = q.x; v[4 * i + 1] = q.y; v[4 * i + 2] = q.z; v[4 * i + 3] = q.w;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = pair_of_bf16x2(v[i]);
}
template <Layout L>
__device__ __forceinline__ void read_codes(const uint8_t* from, int l, uint32_t (&c)[4]) {
  if constexpr (L == QUAD) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = reinterpret_cast<const uint32_t*>(from)[16 * i + l];
  } else {
    const uint2 a = reinterpret_cast<const uint2*>(from)[l], b = reinterpret_cast<const uint2*>(from)[16 + l];
    c[0] = a.x; c[1] = a.y; c[2] = b.x; c[3] = b.y;
  }
}
template <Layout L>
__device__ __forceinline__ void write_codes(uint8_t* to, int l, const uint32_t (&c)[4]) {
  if constexpr (L == QUAD) {
#pragma unroll
    for (int i = 0; i < 4; ++i) __stcs(reinterpret_cast<uint32_t*>(to) + 16 * i + l, c[i]);
  } else {
    __stcs(reinterpret_cast<uint2*>(to) + l, make_uint2(c[0], c[1]));
    __stcs(reinterpret_cast<uint2*>(to) + 16 + l, make_uint2(c[2], c[3]));
  }
}
__device__ __forceinline__ void write_floats(float* to, int l, const float_pair (&x)[8]) {      // (QUAD)
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 a = halves(x[2 * i]), b = halves(x[2 * i + 1]);
    __stcs(reinterpret_cast<float4*>(to) + 16 * i + l, make_float4(a.x, a.y, b.x, b.y));
  }
}
template <Layout L>
__device__ __forceinline__ void write_bf16(bf16* to, int l, const float_pair (&x)[8]) {
  uint32_t v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = pack_bf16x2(x[i]);
  if constexpr (L == QUAD) {
#pragma unroll
    for (int i = 0; i < 4; ++i) __stcs(reinterpret_cast<uint2*>(to) + 16 * i + l, make_uint2(v[2 * i], v[2 * i + 1]));
  } else {
    __stcs(reinterpret_cast<uint4*>(to) + l, make_uint4(v[0], v[1], v[2], v[3]));
    __stcs(reinterpret_cast<uint4*>(to) + 16 + l, make_uint4(v[4], v[5], v[6], v[7]));
  }
}
// Two blocks at a time, one a half warp: what a block costs whatever its size (the scales, the addresses) is paid once for both.
template <typename WT, bool MASTER, int PASSES>
__device__ __forceinline__ void finish_tile(const Tensor& t, const Step& s, const Factors& f, const uint8_t* stage, int lane, const Ahead& a) {
  constexpr Layout L = sizeof(WT) == 4 || MASTER ? QUAD : OCTET;    // by what is stored
  const int half = lane >> 4, l = lane & 15;
  const bool wide_w = sizeof(WT) == 4 || (MASTER && !f.first), wide_g = !(t.kind & KIND_G_BF16);
#pragma unroll 1
  for (int i = 0; i < PASSES; i += 2) {
    const int n = i + half;                                         // this lane's block
    const uint8_t* from = stage + n * s.block_bytes;
    Entries<8> x;
    read_codes<L>(from, l, x.mc);
    read_codes<L>(from + 256, l, x.rc);
    from += 512;
    read_block<L>(from, wide_w, l, x.w);
    from += wide_w ? 1024 : 512;
    read_block<L>(from, wide_g, l, x.g);
    for (int k = 1; k < s.workers; ++k) {
      float_pair y[8];
      from += wide_g ? 1024 : 512;
      read_block<L>(from, wide_g, l, y);
#pragma unroll
      for (int j = 0; j < 8; ++j) x.g[j] = pair_add(x.g[j], y[j]);
    }
    x.ms = __shfl_sync(0xffffffffu, a.scale, 2 * n);
    x.rs = __shfl_sync(0xffffffffu, a.scale, 2 * n + 1);
    const float quotient = update_entries<8, 16, L == QUAD ? REDUX : SHUFFLE>(x, t, s, f, lane);
    const int64_t at = a.at + n * SPAN, sat = t.state_at + at;
    if (MASTER) write_floats(reinterpret_cast<float*>(s.state + s.master_at) + sat, l, x.w);
    if constexpr (sizeof(WT) == 4) write_floats(static_cast<float*>(t.w) + at, l, x.w);
    else write_bf16<L>(static_cast<bf16*>(t.w) + at, l, x.w);
    write_codes<L>(s.state + s.m_at + sat, l, x.mc);
    write_codes<L>(s.state + s.v_at + sat, l, x.rc);
    store_scales<16>(s, sat / BLOCK, lane, quotient);
  }
}

template <int CAP>
__device__ __forceinline__ int find_tensor(const Table<CAP>& tab, uint32_t tile) {
  int lo = 0, hi = tab.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (tab.t[mid].tile0 <= tile) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ Header header_of(int64_t step, double pow_one, double pow_two) {
  return {step, pow_one, pow_two, (float)(1.0 / (1.0 - pow_one)), (float)(1.0 / sqrt(1.0 - pow_two)), 0};
}

template <int BITS, int PASSES, bool MASTER>
__device__ __forceinline__ void update_tile(const Tensor& t, const Step& s, const Factors& f, int64_t at, int lane) {
#define SIGNMUON_CASE(K, WT, GT, MS, VEC) \
  case K: update_warp<BITS, PASSES, WT, GT, MS, VEC>(t, s, f, at, lane); break
  switch (t.kind) {
    SIGNMUON_CASE(0, float, float, false, false);
    SIGNMUON_CASE(KIND_VEC, float, float, false, true);
    SIGNMUON_CASE(KIND_G_BF16, float, bf16, false, false);
    SIGNMUON_CASE(KIND_G_BF16 | KIND_VEC, float, bf16, false, true);
    SIGNMUON_CASE(KIND_W_BF16, bf16, float, MASTER, false);
    SIGNMUON_CASE(KIND_W_BF16 | KIND_VEC, bf16, float, MASTER, true);
    SIGNMUON_CASE(KIND_W_BF16 | KIND_G_BF16, bf16, bf16, MASTER, false);
    SIGNMUON_CASE(KIND_W_BF16 | KIND_G_BF16 | KIND_VEC, bf16, bf16, MASTER, true);
  }
#undef SIGNMUON_CASE
}
// (what the ring leaves over - unaligned tensors and tails - must not cost it registers)
template <int PASSES, bool MASTER>
__device__ __noinline__ void update_rest(const Tensor& t, const Step& s, const Factors& f, int64_t at, int lane) {
  update_tile<8, PASSES, MASTER>(t, s, f, at, lane);
}

// One pass over everything.  What bounds it (a plain copy moves 6.46 TB/s here):
// - 32 bits: the memory.  25.5 M float32 entries with 4 workers (1.02 GB): 159 us, 6.4 TB/s; 39.4 M bf16 entries with master
//   weights (1.10 GB): 176 us, 6.3 TB/s.  Three thread blocks an SM keep 72 to 96 KB in flight; with two the latter takes 201
//   us, with four 186 us.
// - 8 bits: bf16, the issue of instructions, about 40 an entry for its 10 bytes.  157 M entries (1.58 GB): 309 us, 5.1 TB/s
//   (273 us in a run so short that the clock stays high).  The root and the separate roundings of the exact codes are a fifth of
//   the work (252 us without, before the last steps; but then one code in 10^5 differs from the formula's).
//   float32 weights: the memory (39.4 M entries with one worker: 103 us, 6.2 TB/s).
// - 8 bits without the ring, large sets (two float32 gradients beside float32 weights or master copies, five bf16 gradients and
//   more): the latency of a block's loads, with nothing of the warp in flight beside them.  39.4 M entries take 188 us with two
//   float32 gradients (4.2 TB/s), 185 us with five and with eight bf16 ones (3.8 and 5.1 TB/s), 267 us with 16 (5.9 TB/s).
// - small sets: latency.  19 k entries of 25 tensors with 16 workers: 3.4 us a step, launched back to back.
template <int BITS, bool MASTER, int RING, int CAP>
__global__ void __launch_bounds__(THREADS, BITS == 8 ? 2 : 3) adamw_kernel(const __grid_constant__ Table<CAP> tab, const __grid_constant__ Step s) {
  wait_for_stream();
  Header* h = reinterpret_cast<Header*>(s.state);
  const float scale = s.scale ? __ldcg(s.scale) : 1.f;      // (not __ldg: the kernel before this one may write it while this one runs)
  const Factors f = {scale * s.inv_workers, s.lr * __ldcg(&h->inv_correction), __ldcg(&h->inv_root_correction), __ldcg(&h->step) == 0};
  if (!(fabsf(scale) <= 3.402823466e38f)) return;       // not finite: the step is skipped, t does not advance
  constexpr int PASSES = passes_of(RING), TILE = SPAN * PASSES;
  const int lane = threadIdx.x & 31;
  const int at_warp = (threadIdx.x >> 5) * BLOCK;
  if constexpr (RING > 0) {
    extern __shared__ __align__(16) uint8_t ring[];
    const int stage = PASSES * s.block_bytes;
    uint8_t* mine = ring + (threadIdx.x >> 5) * STAGES * stage;
    Ahead next = {};
    if (blockIdx.x < s.tiles) {
      next.tensor = find_tensor(tab, blockIdx.x);
      next.at = (int64_t)(blockIdx.x - tab.t[next.tensor].tile0) * TILE + at_warp;
      fetch_tile<MASTER, PASSES>(tab.t[next.tensor], s, f, mine, lane, next);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    int slot = 0;
    for (uint32_t tile = blockIdx.x; tile < s.tiles; tile += gridDim.x, slot ^= 1) {
      const Ahead now = next;
      const uint32_t then = tile + gridDim.x;
      if (then < s.tiles) {                           // (the tensors lie in the order of their tiles)
        while (next.tensor + 1 < tab.n && tab.t[next.tensor + 1].tile0 <= then) ++next.tensor;
        next.at = (int64_t)(then - tab.t[next.tensor].tile0) * TILE + at_warp;
        fetch_tile<MASTER, PASSES>(tab.t[next.tensor], s, f, mine + (slot ^ 1) * stage, lane, next);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
      asm volatile("cp.async.wait_group 1;" ::: "memory");
      __syncwarp();                                   // the lanes read what others copied
      const Tensor& t = tab.t[now.tensor];
      if (!now.ready) update_rest<PASSES, MASTER>(t, s, f, now.at, lane);
      else if (t.kind & KIND_W_BF16) finish_tile<bf16, MASTER, PASSES>(t, s, f, mine + slot * stage, lane, now);
      else finish_tile<float, false, PASSES>(t, s, f, mine + slot * stage, lane, now);
      __syncwarp();                                   // read before it is copied over
    }
  } else {
    for (uint32_t tile = blockIdx.x; tile < s.tiles; tile += gridDim.x) {
      const Tensor& t = tab.t[find_tensor(tab, tile)];
      update_tile<BITS, PASSES, MASTER>(t, s, f, (int64_t)(tile - t.tile0) * TILE + at_warp, lane);
    }
  }
  if (!s.advance) return;
  // The block that finishes last advances the step: every block has read the header by then.  The last warp, which has
  // least to do in a small tile, works out the next header beforehand.
  Header next;
  if (threadIdx.x == THREADS - 32) next = header_of(__ldcg(&h->step) + 1, __ldcg(&h->pow_one) * s.beta_one, __ldcg(&h->pow_two) * s.beta_two);
  __syncthreads();
  if (threadIdx.x == THREADS - 32 && atomicAdd(&h->ticket, 1u) == gridDim.x - 1) *h = next;
}

__global__ void set_header_kernel(Header* h, int64_t step, double pow_one, double pow_two) { *h = header_of(step, pow_one, pow_two); }

// Sum of the squares of the mean gradient over a warp's blocks of a tile.  Few workers' gradients are few loads a block: four
// blocks are loaded together for one worker, two for two or three.
constexpr int NORM_PASSES = 4, NORM_TILE = NORM_PASSES * SPAN;
__device__ __forceinline__ float square_of(float (&g)[8], float by) {
  float q = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    g[j] *= by;
    q = fmaf(g[j], g[j], q);
  }
  return q;
}
template <int N, typename GT>
__device__ __forceinline__ double squares_together(const GT* g, const Norm& s, int64_t stride, int lane) {
  constexpr int TOGETHER = N == 1 ? 4 : 2;
  double sum = 0.0;
#pragma unroll
  for (int first = 0; first < NORM_PASSES; first += TOGETHER) {
    Raw<GT> r[TOGETHER * N];
#pragma unroll
    for (int i = 0; i < TOGETHER * N; ++i) r[i] = load_raw<sizeof(GT) == 4 ? QUAD : OCTET>(g + (first + i / N) * SPAN + (i % N) * stride, lane);
#pragma unroll
    for (int n = 0; n < TOGETHER; ++n) {
      float x[8], y[8];
      unpack(r[n * N], x);
#pragma unroll
      for (int k = 1; k < N; ++k) {
        unpack(r[n * N + k], y);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] += y[j];
      }
      sum += (double)square_of(x, s.inv_workers);
    }
  }
  return sum;
}
template <typename GT>
__device__ __forceinline__ double squares(const Tensor& t, const GT* g, const Norm& s, int64_t at, int lane) {
  double sum = 0.0;
  if (s.workers <= 3 && (t.kind & KIND_VEC) && at + (NORM_PASSES - 1) * SPAN + BLOCK <= t.numel)
    return s.workers == 1 ? squares_together<1>(g + at, s, 0, lane)
         : s.workers == 2 ? squares_together<2>(g + at, s, t.grad_stride, lane) : squares_together<3>(g + at, s, t.grad_stride, lane);
#pragma unroll 1
  for (int n = 0; n < NORM_PASSES && at < t.numel; ++n, at += SPAN) {
    const int valid = t.numel - at < BLOCK ? (int)(t.numel - at) : BLOCK;
    float x[8];
    if (valid == BLOCK && (t.kind & KIND_VEC)) sum_gradients<GT, sizeof(GT) == 4 ? QUAD : OCTET>(g + at, t.grad_stride, s.workers, lane, valid, x);
    else sum_gradients<GT, SCALAR>(g + at, t.grad_stride, s.workers, lane, valid, x);
    sum += (double)square_of(x, s.inv_workers);
  }
  return sum;
}

// Bound by the memory: 39.4 M bf16 entries of 16 workers (1.26 GB) in 194 us, 6.5 TB/s (reading alone can be faster than a
// copy).  19 k entries of 25 tensors: 4.9 us, most of it the two latencies of the last block's turn.
// Sum of the squares of the mean gradient: float32 over a thread's 8 entries of a block, double from there on; the
// partial sums are added in the order of their blocks, whichever block comes last.
template <int CAP>
__global__ void __launch_bounds__(THREADS) grad_norm_kernel(const __grid_constant__ Table<CAP> tab, const __grid_constant__ Norm s) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  double sum = 0.0;
  wait_for_stream();
  for (uint32_t tile = blockIdx.x; tile < s.tiles; tile += gridDim.x) {
    const Tensor& t = tab.t[find_tensor(tab, tile)];
    int64_t at = (int64_t)(tile - t.tile0) * NORM_TILE + warp * BLOCK;
    if (t.kind & KIND_G_BF16) sum += squares(t, static_cast<const bf16*>(t.g), s, at, lane);
    else sum += squares(t, static_cast<const float*>(t.g), s, at, lane);
  }
  __shared__ double part[THREADS];
  __shared__ bool is_last;
  const auto reduce = [&](double x) -> double {      // over the thread block, in a fixed order; valid in thread 0
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    __syncthreads();
    if (lane == 0) part[warp] = x;
    __syncthreads();
    double r = 0.0;
    if (threadIdx.x == 0)
      for (int i = 0; i < WARPS; ++i) r += part[i];
    return r;
  };
  sum = reduce(sum);
  if (threadIdx.x == 0) {
    s.partials[blockIdx.x] = sum;
    is_last = false;
    if (s.last) {
      __threadfence();
      is_last = atomicAdd(s.ticket, 1u) == gridDim.x - 1;
      __threadfence();
    }
  }
  __syncthreads();
  if (!is_last) return;
  sum = 0.0;
  for (uint32_t i = threadIdx.x; i < s.n_all; i += THREADS) sum += __ldcg(s.all + i);
  sum = reduce(sum);
  if (threadIdx.x == 0) {
    *s.ticket = 0;
    const float norm = (float)sqrt(sum);
    s.out[0] = norm;
    // not finite: the coefficient is NaN, and a step that takes it as its scale is skipped
    s.out[1] = !(norm <= 3.402823466e38f) ? __int_as_float(0x7fffffff) : norm > s.max_norm ? s.max_norm / norm : 1.f;
  }
}

inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

constexpr int SMALL = 32, LARGE = 512;      // tensors in one launch's table: 1.8 KB or 28 KB of kernel parameters

}  // namespace

struct signmuon_adamw {
  signmuon_adamw_config cfg;
  std::vector<signmuon_adamw_param> params;
  std::vector<Tensor> tensors;              // what does not change from call to call
  std::vector<uint32_t> norm_tile0;         // their first tiles in the norm's launches
  struct Launch { size_t first, count; uint32_t tiles, norm_tiles; };
  std::vector<Launch> launches;
  int64_t padded = 0;                       // entries of a state region
  bool master = false;
  size_t region[SIGNMUON_ADAMW_MASTER_WEIGHT + 1] = {}, region_bytes[SIGNMUON_ADAMW_MASTER_WEIGHT + 1] = {};
  size_t state_bytes = 0, workspace_bytes = 0;
  bool bound = false;
  uint8_t* state = nullptr;
  uint8_t* workspace = nullptr;
  int grid_step = 0, grid_norm = 0;
  int block_bytes = 0;                      // of a block in the step's ring in shared memory, for the widest tensor
  int ring = 0;                             // blocks of a warp that the ring holds a stage (0: no ring)
  int tile = 0;
  size_t shared = 0;                        // of the step's kernel
  int sticky = SIGNMUON_OK;
};

namespace {

int entry_bytes(int32_t dtype) { return dtype == SIGNMUON_BF16 ? 2 : 4; }
bool is_dtype(int32_t d) { return d == SIGNMUON_F32 || d == SIGNMUON_BF16; }

// Fills a launch's table with the call's pointers.  weights may be null (norm).
template <int CAP>
int fill(const signmuon_adamw* c, const signmuon_adamw::Launch& l, void* const* weights, const void* const* grads,
         Table<CAP>& tab) {
  tab.n = (int32_t)l.count;
  for (size_t i = 0; i < l.count; ++i) {
    const size_t p = l.first + i;
    Tensor t = c->tensors[p];
    t.w = weights ? weights[p] : nullptr;
    t.g = grads[p];
    if (!weights) t.tile0 = c->norm_tile0[p];
    if (t.numel > 0) {
      const int gb = entry_bytes(c->params[p].grad_dtype), wb = entry_bytes(c->params[p].weight_dtype);
      const uintptr_t g = reinterpret_cast<uintptr_t>(t.g), w = reinterpret_cast<uintptr_t>(t.w);
      if (!t.g || (weights && !t.w)) return SIGNMUON_ERR_INVALID_ARG;
      if (g % gb || w % wb) return SIGNMUON_ERR_MISALIGNED;
      const bool strides = c->cfg.num_workers == 1 || (t.grad_stride * gb) % 16 == 0;
      if (g % 16 == 0 && w % 16 == 0 && strides) t.kind |= KIND_VEC;
    }
    tab.t[i] = t;
  }
  return SIGNMUON_OK;
}

template <int CAP>
void* step_kernel(const signmuon_adamw* c) {
  if (c->cfg.state_bits == 32)
    return c->master ? (void*)adamw_kernel<32, true, 0, CAP> : (void*)adamw_kernel<32, false, 0, CAP>;
  if (c->ring == 4) return (void*)adamw_kernel<8, false, 4, CAP>;        // (a master copy makes a block too large for four)
  if (c->ring == 2) return c->master ? (void*)adamw_kernel<8, true, 2, CAP> : (void*)adamw_kernel<8, false, 2, CAP>;
  return c->master ? (void*)adamw_kernel<8, true, 0, CAP> : (void*)adamw_kernel<8, false, 0, CAP>;
}

template <int CAP>
int launch_step(signmuon_adamw* c, const signmuon_adamw::Launch& l, void* const* weights, const void* const* grads, Step& s,
                cudaStream_t stream) {
  Table<CAP> tab;
  if (const int e = fill(c, l, weights, grads, tab)) return e;
  s.tiles = l.tiles;
  void* args[] = {&tab, &s};
  const unsigned grid = std::max(1u, std::min<unsigned>(l.tiles, c->grid_step));
  const cudaError_t e = launch_early(step_kernel<CAP>(c), dim3(grid), dim3(THREADS), c->shared, args, stream);
  return e == cudaSuccess ? SIGNMUON_OK : SIGNMUON_ERR_CUDA;
}

template <int CAP>
int launch_norm(signmuon_adamw* c, const signmuon_adamw::Launch& l, const void* const* grads, Norm& s, cudaStream_t stream) {
  Table<CAP> tab;
  if (const int e = fill(c, l, nullptr, grads, tab)) return e;
  s.tiles = l.norm_tiles;
  const unsigned grid = std::max(1u, std::min<unsigned>(l.norm_tiles, c->grid_norm));
  s.n_all += grid;
  void* args[] = {&tab, &s};
  const cudaError_t e = launch_early((void*)grad_norm_kernel<CAP>, dim3(grid), dim3(THREADS), 0, args, stream);
  s.partials += grid;
  return e == cudaSuccess ? SIGNMUON_OK : SIGNMUON_ERR_CUDA;
}

}  // namespace

extern "C" {

int signmuon_adamw_create(const signmuon_adamw_config* config, signmuon_adamw** out) {
  if (!out) return SIGNMUON_ERR_INVALID_ARG;
  *out = nullptr;
  if (!config || config->num_params < 1 || !config->params) return SIGNMUON_ERR_INVALID_ARG;
  const signmuon_adamw_config& g = *config;
  if (g.num_workers < 1 || g.num_workers > 255 || (g.state_bits != 32 && g.state_bits != 8) ||
      (g.flags & ~SIGNMUON_ADAMW_FLAG_MASTER) || !std::isfinite(g.lr) || !(g.beta_one >= 0 && g.beta_one < 1) ||
      !(g.beta_two >= 0 && g.beta_two < 1) || !(g.eps >= 0x1p-120) || !(g.eps <= 1))
    return SIGNMUON_ERR_INVALID_ARG;
  for (int32_t p = 0; p < g.num_params; ++p) {
    const signmuon_adamw_param& q = g.params[p];
    if (!is_dtype(q.weight_dtype) || !is_dtype(q.grad_dtype) || !(q.weight_decay >= 0) || !std::isfinite(q.weight_decay))
      return SIGNMUON_ERR_INVALID_ARG;
    if (q.numel < 0 || q.numel > MAX_ENTRIES || q.grad_stride < 0 || q.grad_stride > MAX_ENTRIES ||
        (q.grad_stride != 0 && q.grad_stride < q.numel))
      return SIGNMUON_ERR_BAD_SHAPE;
  }
  signmuon_adamw* c = nullptr;
  try {
    c = new signmuon_adamw();
    c->cfg = g;
    c->params.assign(g.params, g.params + g.num_params);
    c->cfg.params = nullptr;
    for (const signmuon_adamw_param& q : c->params) {
      const bool wide_w = q.weight_dtype == SIGNMUON_F32 || (g.flags & SIGNMUON_ADAMW_FLAG_MASTER);
      c->block_bytes = std::max(c->block_bytes, 512 + (wide_w ? 1024 : 512) + g.num_workers * (q.grad_dtype == SIGNMUON_F32 ? 1024 : 512));
    }
    int64_t blocks = 0;
    for (const signmuon_adamw_param& q : c->params) blocks += (q.numel + BLOCK - 1) / BLOCK;
    for (int passes = 4; passes >= 2 && g.state_bits == 8 && blocks >= RING_BLOCKS && c->ring == 0; passes /= 2)
      if ((size_t)WARPS * STAGES * passes * c->block_bytes <= RING_LIMIT) c->ring = passes;
    c->shared = (size_t)WARPS * STAGES * c->ring * c->block_bytes;
    c->tile = SPAN * passes_of(c->ring);
    for (const signmuon_adamw_param& q : c->params) {
      if (c->launches.empty() || c->launches.back().count == LARGE) c->launches.push_back({c->tensors.size(), 0, 0, 0});
      signmuon_adamw::Launch& l = c->launches.back();
      Tensor t = {};
      t.numel = q.numel;
      t.grad_stride = q.grad_stride ? q.grad_stride : q.numel;
      t.state_at = c->padded;
      t.tile0 = l.tiles;
      t.decay = (float)q.weight_decay;
      t.kind = (q.weight_dtype == SIGNMUON_BF16 ? KIND_W_BF16 : 0) | (q.grad_dtype == SIGNMUON_BF16 ? KIND_G_BF16 : 0);
      if (q.weight_dtype == SIGNMUON_BF16 && (g.flags & SIGNMUON_ADAMW_FLAG_MASTER)) c->master = true;
      c->tensors.push_back(t);
      c->padded += (int64_t)round_up(q.numel, BLOCK);
      const int64_t tiles = l.tiles + (q.numel + c->tile - 1) / c->tile;
      if (c->padded > MAX_ENTRIES || tiles > INT32_MAX) { delete c; return SIGNMUON_ERR_BAD_SHAPE; }
      l.tiles = (uint32_t)tiles;
      c->norm_tile0.push_back(l.norm_tiles);
      l.norm_tiles += (uint32_t)((q.numel + NORM_TILE - 1) / NORM_TILE);
      l.count += 1;
    }
  } catch (const std::bad_alloc&) {
    delete c;
    return SIGNMUON_ERR_NO_MEMORY;
  }
  const size_t n = (size_t)c->padded, blocks = n / BLOCK, per = g.state_bits == 32 ? 4 : 1;
  size_t at = 0;
  const auto add = [&](int what, size_t bytes) {
    c->region[what] = at;
    c->region_bytes[what] = bytes;
    at += round_up(bytes, 256);
  };
  add(SIGNMUON_ADAMW_HEADER, HEADER_BYTES);
  add(SIGNMUON_ADAMW_FIRST_MOMENT, n * per);
  add(SIGNMUON_ADAMW_SECOND_MOMENT, n * per);
  add(SIGNMUON_ADAMW_FIRST_SCALE, g.state_bits == 8 ? blocks * 4 : 0);
  add(SIGNMUON_ADAMW_SECOND_SCALE, g.state_bits == 8 ? blocks * 4 : 0);
  add(SIGNMUON_ADAMW_MASTER_WEIGHT, c->master ? n * 4 : 0);
  c->state_bytes = at;
  c->workspace_bytes = 256 + round_up(c->launches.size() * MAX_GRID * sizeof(double), 256);
  *out = c;
  return SIGNMUON_OK;
}

int signmuon_adamw_state_bytes(const signmuon_adamw* c, size_t* state, size_t* workspace) {
  if (!c) return SIGNMUON_ERR_INVALID_ARG;
  if (state) *state = c->state_bytes;
  if (workspace) *workspace = c->workspace_bytes;
  return SIGNMUON_OK;
}

int signmuon_adamw_state_segment(const signmuon_adamw* c, int32_t what, int32_t param, size_t* byte_offset, size_t* bytes) {
  if (!c || what < SIGNMUON_ADAMW_HEADER || what > SIGNMUON_ADAMW_MASTER_WEIGHT || param < -1 ||
      param >= (int32_t)c->params.size() || (what == SIGNMUON_ADAMW_HEADER && param >= 0))
    return SIGNMUON_ERR_INVALID_ARG;
  if (c->region_bytes[what] == 0 && c->padded > 0) return SIGNMUON_ERR_INVALID_ARG;   // this context has no such state
  size_t off = c->region[what], size = c->region_bytes[what];
  if (param >= 0) {
    const Tensor& t = c->tensors[param];
    const bool scales = what == SIGNMUON_ADAMW_FIRST_SCALE || what == SIGNMUON_ADAMW_SECOND_SCALE;
    const size_t per = what == SIGNMUON_ADAMW_MASTER_WEIGHT || c->cfg.state_bits == 32 ? 4 : 1;
    off += scales ? (size_t)t.state_at / BLOCK * 4 : (size_t)t.state_at * per;
    size = scales ? round_up(t.numel, BLOCK) / BLOCK * 4 : (size_t)t.numel * per;
  }
  if (byte_offset) *byte_offset = off;
  if (bytes) *bytes = size;
  return SIGNMUON_OK;
}

int signmuon_adamw_set_step(signmuon_adamw* c, int64_t step, void* cuda_stream) {
  if (!c || step < 0) return SIGNMUON_ERR_INVALID_ARG;
  if (!c->bound) return SIGNMUON_ERR_NOT_BOUND;
  if (c->sticky != SIGNMUON_OK) return c->sticky;
  set_header_kernel<<<1, 1, 0, reinterpret_cast<cudaStream_t>(cuda_stream)>>>(
      reinterpret_cast<Header*>(c->state), step, std::pow(c->cfg.beta_one, (double)step + 1),
      std::pow(c->cfg.beta_two, (double)step + 1));
  if (cudaGetLastError() != cudaSuccess) c->sticky = SIGNMUON_ERR_CUDA;
  return c->sticky;
}

int signmuon_adamw_bind(signmuon_adamw* c, void* dev_state, size_t state_bytes, void* dev_workspace, size_t workspace_bytes,
                        int zero_state, void* cuda_stream) {
  if (!c || !dev_state || !dev_workspace) return SIGNMUON_ERR_INVALID_ARG;
  if (state_bytes < c->state_bytes || workspace_bytes < c->workspace_bytes) return SIGNMUON_ERR_BUFFER_TOO_SMALL;
  if ((reinterpret_cast<uintptr_t>(dev_state) | reinterpret_cast<uintptr_t>(dev_workspace)) & 255) return SIGNMUON_ERR_MISALIGNED;
  int dev = 0, major = 0, sms = 0, occ_step = 0, occ_norm = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
    cudaGetLastError();
    return SIGNMUON_ERR_CUDA;
  }
  if (major != 10) return SIGNMUON_ERR_UNSUPPORTED_ARCH;
  const bool small = c->params.size() <= SMALL;
  void* step = small ? step_kernel<SMALL>(c) : step_kernel<LARGE>(c);
  void* norm = small ? (void*)grad_norm_kernel<SMALL> : (void*)grad_norm_kernel<LARGE>;
  // The limit of dynamic shared memory belongs to the kernel and the device, not to this context: always the most that any
  // context asks of it, so that none lowers it under another.
  if ((c->shared && cudaFuncSetAttribute(step, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)RING_LIMIT) != cudaSuccess) ||
      cudaOccupancyMaxActiveBlocksPerMultiprocessor(&occ_step, step, THREADS, c->shared) != cudaSuccess ||
      cudaOccupancyMaxActiveBlocksPerMultiprocessor(&occ_norm, norm, THREADS, 0) != cudaSuccess) {
    cudaGetLastError();
    return SIGNMUON_ERR_CUDA;
  }
  c->grid_step = std::max(1, occ_step * sms);
  c->grid_norm = std::max(1, std::min(occ_norm * sms, MAX_GRID));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (cudaMemsetAsync(dev_workspace, 0, 256, s) != cudaSuccess ||
      (zero_state && cudaMemsetAsync(dev_state, 0, c->state_bytes, s) != cudaSuccess)) {
    c->sticky = SIGNMUON_ERR_CUDA;
    return c->sticky;
  }
  c->state = static_cast<uint8_t*>(dev_state);
  c->workspace = static_cast<uint8_t*>(dev_workspace);
  c->bound = true;
  c->sticky = SIGNMUON_OK;
  return zero_state ? signmuon_adamw_set_step(c, 0, cuda_stream) : SIGNMUON_OK;
}

int signmuon_adamw_step(signmuon_adamw* c, void* const* weights, const void* const* grads, double lr, const float* dev_scale,
                        void* cuda_stream) {
  if (!c || !weights || !grads || std::isnan(lr) || std::isinf(lr)) return SIGNMUON_ERR_INVALID_ARG;
  if (!c->bound) return SIGNMUON_ERR_NOT_BOUND;
  if (c->sticky != SIGNMUON_OK) return c->sticky;
  if (reinterpret_cast<uintptr_t>(dev_scale) & 3) return SIGNMUON_ERR_MISALIGNED;
  Step s = {};
  s.state = c->state;
  s.m_at = (int64_t)c->region[SIGNMUON_ADAMW_FIRST_MOMENT];
  s.v_at = (int64_t)c->region[SIGNMUON_ADAMW_SECOND_MOMENT];
  s.ms_at = (int64_t)c->region[SIGNMUON_ADAMW_FIRST_SCALE];
  s.vs_at = (int64_t)c->region[SIGNMUON_ADAMW_SECOND_SCALE];
  s.master_at = (int64_t)c->region[SIGNMUON_ADAMW_MASTER_WEIGHT];
  s.scale = dev_scale;
  s.workers = c->cfg.num_workers;
  s.block_bytes = c->block_bytes;
  // the factors are rounded to float32 once, from doubles: 1 - float(0.999) would be off by 1e-5 of its value
  s.lr = (float)(lr < 0 ? c->cfg.lr : lr);
  s.beta_one = c->cfg.beta_one;
  s.beta_two = c->cfg.beta_two;
  s.b1 = (float)s.beta_one;
  s.b2 = (float)s.beta_two;
  s.omb1 = (float)(1 - s.beta_one);
  s.omb2 = (float)(1 - s.beta_two);
  s.eps = (float)c->cfg.eps;
  s.minus_zero = -0.f;
  s.fast_above = c->cfg.eps >= 0x1p-40 / std::sqrt(1 - s.beta_two) ? 0x1p-60f : INFINITY;      // (the correction is largest at t = 1)
  s.inv_workers = (float)(1.0 / s.workers);
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (c->launches.size() > 1) {              // a pointer that is refused is refused before the first launch
    Table<LARGE> tab;
    for (const auto& l : c->launches)
      if (const int e = fill(c, l, weights, grads, tab)) return e;
  }
  for (size_t i = 0; i < c->launches.size(); ++i) {
    const auto& l = c->launches[i];
    s.advance = i + 1 == c->launches.size();
    const int e = c->params.size() <= SMALL ? launch_step<SMALL>(c, l, weights, grads, s, stream)
                                            : launch_step<LARGE>(c, l, weights, grads, s, stream);
    if (e == SIGNMUON_ERR_CUDA) { cudaGetLastError(); c->sticky = e; }
    if (e != SIGNMUON_OK) return e;
  }
  return SIGNMUON_OK;
}

int signmuon_adamw_grad_norm(signmuon_adamw* c, const void* const* grads, float max_norm, float* dev_out, void* cuda_stream) {
  if (!c || !grads || !dev_out || !(max_norm > 0)) return SIGNMUON_ERR_INVALID_ARG;
  if (!c->bound) return SIGNMUON_ERR_NOT_BOUND;
  if (c->sticky != SIGNMUON_OK) return c->sticky;
  if (reinterpret_cast<uintptr_t>(dev_out) & 3) return SIGNMUON_ERR_MISALIGNED;
  Norm s = {};
  s.ticket = reinterpret_cast<uint32_t*>(c->workspace);
  s.all = s.partials = reinterpret_cast<double*>(c->workspace + 256);
  s.out = dev_out;
  s.workers = c->cfg.num_workers;
  s.inv_workers = (float)(1.0 / s.workers);
  s.max_norm = max_norm;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (c->launches.size() > 1) {
    Table<LARGE> tab;
    for (const auto& l : c->launches)
      if (const int e = fill(c, l, nullptr, grads, tab)) return e;
  }
  for (size_t i = 0; i < c->launches.size(); ++i) {
    const auto& l = c->launches[i];
    s.last = i + 1 == c->launches.size();
    const int e = c->params.size() <= SMALL ? launch_norm<SMALL>(c, l, grads, s, stream) : launch_norm<LARGE>(c, l, grads, s, stream);
    if (e == SIGNMUON_ERR_CUDA) { cudaGetLastError(); c->sticky = e; }
    if (e != SIGNMUON_OK) return e;
  }
  return SIGNMUON_OK;
}

int signmuon_adamw_launches_per_step(const signmuon_adamw* c, int32_t* launches) {
  if (!c || !launches) return SIGNMUON_ERR_INVALID_ARG;
  *launches = (int32_t)c->launches.size();
  return SIGNMUON_OK;
}

void signmuon_adamw_destroy(signmuon_adamw* c) { delete c; }

}  // extern "C"
