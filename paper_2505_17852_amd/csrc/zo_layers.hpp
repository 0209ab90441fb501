// Launchers of the layers' kernels (host side) and what their kernels share.
// Every launcher only enqueues on `stream`; the C ABI layer has checked its
// arguments.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/zo_layers.h"
#include "zo_common.hpp"
#include "zo_rng.hpp"

namespace zo {

// ---- values of either type ----

template <typename T>
__device__ __forceinline__ float to_f32(T x) {
  if constexpr (sizeof(T) == 2) return bf16_to_f32(x);
  else return x;
}
// Two fp32 values to packed bf16, each to nearest even.
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
  typedef float f2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2){lo, hi}, bf2));
}
template <typename T>
__device__ __forceinline__ T from_f32(float x) {
  if constexpr (sizeof(T) == 2) return (uint16_t)bf16_pair(x, 0.0f);
  else return x;
}

// N consecutive values at p, which needs no more than its type's alignment (gfx950
// loads and stores 16 bytes at any address of 4-byte words, and at odd ones).
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Run {
  T v[N];
};
template <typename T, int N>
__device__ __forceinline__ void load_run(const T* p, float* out) {
  const Run<T, N> r = *(const Run<T, N>*)p;
#pragma unroll
  for (int e = 0; e < N; ++e) out[e] = to_f32(r.v[e]);
}
template <typename T, int N>
__device__ __forceinline__ void store_run(T* p, const float* in) {
  if constexpr (sizeof(T) == 2) {
    typedef Run<uint32_t, N / 2> Words;
    struct __attribute__((packed, aligned(2))) Any { Words w; } a;
#pragma unroll
    for (int e = 0; e < N / 2; ++e) a.w.v[e] = bf16_pair(in[2 * e], in[2 * e + 1]);
    *(Any*)p = a;
  } else {
    Run<T, N> r;
#pragma unroll
    for (int e = 0; e < N; ++e) r.v[e] = in[e];
    *(Run<T, N>*)p = r;
  }
}

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
// 16 bytes at p, which is aligned to its type.
template <typename T>
__device__ __forceinline__ u4 load16(const T* p) {
  struct __attribute__((packed, aligned(sizeof(T)))) Any { u4 v; };
  return ((const Any*)p)->v;
}
// Drops the first n values (fewer than 16 bytes hold), zeros after the rest: the end of a row,
// read with the 16 bytes that end there.
template <typename T>
__device__ __forceinline__ u4 drop(u4 v, int n) {
  int words = n;
  if constexpr (sizeof(T) == 2) {
    words = n >> 1;
    if (n & 1) v = u4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
  }
  if (words & 1) v = u4{v[1], v[2], v[3], 0};
  if (words & 2) v = u4{v[2], v[3], 0, 0};
  return v;
}

// ---- linear attention (k_linattn.hip, k_linattn_step.hip) ----

// The nearest finite value: an infinite state takes no correction (which would make it NaN).
__device__ __forceinline__ float finite(float s) {
  constexpr float kMax = 3.40282347e38f;
  return __builtin_amdgcn_fmed3f(s, -kMax, kMax);
}

// gamma = high + low. A state that takes gamma at every token would drift by gamma's rounding, thousands of times half a
// unit in the last place (6e-5 after 2,000 tokens), so it is held in two parts, from its value in 64 bits.
struct Gamma {
  float high, low;
  __device__ __forceinline__ explicit Gamma(float log_decay) {
    const double gamma = exp((double)log_decay);
    high = (float)gamma;
    low = high < __builtin_inff() ? (float)(gamma - (double)high) : 0.0f;
  }
  // gamma s + add
  __device__ __forceinline__ float times(float s, float add) const { return fmaf(high, s, fmaf(low, finite(s), add)); }
};

struct Heads {
  const void* p;
  int64_t b, t, h;  // strides in elements
};

// One pass of the recurrence. Forward in time, for every sequence, output head and position:
//   R_t = gamma R_{t-1} + upd sum_s y_t z_t^T,   out_t = carry gamma R_{t-1}^T x_t + ...
// The forward pass and the three gradients are all of this form (see k_linattn.hip).
struct LinPass {
  Heads x, y, z;        // x: the reader [out heads][dx]; y [dx] and z [dz]: the summed products
  void* out;            // [out heads][dz]
  int64_t ob, ot, oh;
  int dx, dz;
  int heads;            // out heads per state (forward: the query heads that read it; backward: 1)
  int sources;          // y/z heads summed into one state (forward: 1; backward: those query heads)
  int reverse;
  int state_t;          // the states' array is [dz][dx] instead of [dx][dz]
  float score, carry, upd;
  const float* init;    // [B][states][..] or nullptr
  float* fin;           // or nullptr
};
constexpr int kLinPasses = 3;
struct LinCall {
  LinPass pass[kLinPasses];
  int npasses;
  int B, T, kv_heads, share;  // share: query heads per key/value head
  int dtype;
  const float* log_decay;
  const int32_t* lengths;
  void* work;
};
size_t linattn_workspace(const zo_linattn& s, bool backward);
hipError_t launch_linattn(const LinCall& c, hipStream_t s);

struct LinStep {
  Heads q, k, v;
  void* o;
  int64_t ob, oh;
  int B, q_heads, kv_heads, dk, dv, dtype;
  float scale;
  const float* log_decay;
  float* state;
  int32_t n_slots;
  const int32_t* slots;
};
hipError_t launch_linattn_step(const LinStep& a, hipStream_t s);

// ---- layer norm (k_norm.hip) ----

struct NormArgs {
  int xdtype, wdtype;
  int64_t rows, D;
  const void* x;
  int64_t xs;
  const void* w;
  const void* b;        // forward
  float eps;            // forward
  void* y;              // forward: y; backward: dx
  int64_t ys;
  const void* dy;       // backward
  int64_t dys;
  float* mean;
  float* rstd;
  float* dw;
  float* db;
  float* partial;       // workspace
};
size_t norm_workspace(int64_t rows, int64_t D);
hipError_t launch_norm(const NormArgs& a, hipStream_t s);
hipError_t launch_norm_backward(const NormArgs& a, hipStream_t s);

// ---- AdamW (k_adamw.hip) ----

hipError_t launch_adamw(const zo_adamw_config& cfg, const zo_adamw_tensor* t, int32_t n, void* m, void* v,
                        float* ms, float* vs, const float* grad_scale, int32_t* skipped, hipStream_t s);
hipError_t launch_adamw_moments(int64_t n, const void* m, const void* v, const float* ms, const float* vs, float* mo,
                                float* vo, hipStream_t s);

}  // namespace zo
