// AdamW over many tensors in one launch (of up to kTensors tensors, whose
// addresses travel in the launch's arguments: nothing is copied or kept).
//
// Per value: m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2 and
// p = p keep - lr (m c1) / (sqrt(v c2) + eps), c1 and c2 the bias corrections.
// Everything is read once and written once, so the step is bound by memory; a
// thread takes 8 consecutive values, whose six 16-byte loads are in flight
// together. 1.2e9 parameters (bf16, 32-bit moments): 26.7 GB in 5.24 ms, 5.1 TB/s (a copy of
// 4 GiB: 4.75).
//
// 8-bit moments: 32 lanes hold one block of 256 values, whose maxima they find
// by lane exchanges; codes are the nearest in the square root of the first
// moment and the fourth root of the second (relative steps of 1.6% at the
// block's maximum, and a range of 1.6e4 and 4e9 below it). The code of a value
// near a rounding boundary depends on the last bit of the moment, so moments and
// codes are those of the definition's operations, one IEEE rounding each, without
// contraction. Roots and quotients of that kind take ten instructions and
// more; a code is first found from the hardware's approximate ones and worked out again only where it lies
// within 2^-11 of a boundary, which their error cannot reach across: 1 / top is within 2^-22 (a subnormal one; 2^-24
// otherwise), products within 2^-24, a root within 2^-23 and half of what lies under it, so that a code is known to
// 2^-21 relative, the definition's own operations to 2^-22, together at most 255 x 2^-20 = 2^-12 apart
// (128 million parameters: 0.53 -> 0.31 to 0.34 ms, 4 TB/s; decoding the
// moments for the caller 0.20 ms, 6.3 TB/s).
#include <hip/hip_runtime.h>

#include <cmath>

#include "zo_layers.hpp"

namespace zo {
namespace {

constexpr int kTensors = 64;
constexpr int kThreads = 256;
constexpr int kPer = 8;                       // values per thread
constexpr int64_t kChunk = kThreads * kPer;   // values per workgroup

struct Entry {
  void* p;
  const void* g;
  int64_t n;
  int64_t off;
  int64_t first;  // the tensor's first workgroup
  float keep;
  int16_t pbf, gbf;
};
struct Args {
  Entry e[kTensors];
  int n;
  float b1, omb1, b2, omb2, c1, c2, eps, lr;
  void* m;
  void* v;
  float* ms;
  float* vs;
  const float* grad_scale;
  int32_t* skipped;
};

template <typename T>
__device__ __forceinline__ void load8(const T* p, int64_t left, float* out) {
  if (left >= kPer) {
    load_run<T, kPer>(p, out);
  } else {
#pragma unroll
    for (int e = 0; e < kPer; ++e) out[e] = e < left ? to_f32(p[e]) : 0.0f;
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int64_t left, const float* in) {
  if (left >= kPer) {
    store_run<T, kPer>(p, in);
  } else {
#pragma unroll
    for (int e = 0; e < kPer; ++e)
      if (e < left) p[e] = from_f32<T>(in[e]);
  }
}

// The largest |x| of a block's 256 values (32 lanes of 8): as bit patterns, so
// that a NaN is larger than everything; what is not finite becomes NaN.
__device__ __forceinline__ float block_top(const float* x) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < kPer; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
#pragma unroll
  for (int d = 16; d; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d, 32));
  return top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : __uint_as_float(top);
}

__device__ __forceinline__ float decode_m(int c, float top) {
#pragma clang fp contract(off)
  const float part = (float)c * (float)(1.0 / 127.0);
  return part * fabsf(part) * top;
}
__device__ __forceinline__ float decode_v(int c, float top) {
#pragma clang fp contract(off)
  float part = (float)c * (float)(1.0 / 255.0);
  part = part * part;
  return part * part * top;
}
constexpr float kNear = 0x1p-11f;

// Whether the nearest whole number of t, at most 255 and known to 2^-20 relative, is certain (not of a NaN).
__device__ __forceinline__ bool certain(float t) { return fabsf(t - rintf(t)) < 0.5f - kNear; }

__device__ __noinline__ float exact_code(float x, float top, int root) {
#pragma clang fp contract(off)
  const float share = x / top;
  float r = sqrtf(share >= 0.0f ? share : 0.0f);
  if (root == 4) r = sqrtf(r);
  return rintf(r * (root == 4 ? 255.0f : 127.0f));
}
// inv: 1 / top.
__device__ __forceinline__ int encode_m(float m, float top, float inv) {
  const float t = __builtin_amdgcn_sqrtf(fabsf(m) * inv) * 127.0f;
  float code = rintf(t);
  if (!certain(t)) code = exact_code(fabsf(m), top, 2);
  return m < 0.0f ? -(int)code : (int)code;
}
__device__ __forceinline__ int encode_v(float v, float top, float inv) {
  const float t = __builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(v * inv)) * 255.0f;
  float code = rintf(t);
  if (!certain(t)) code = exact_code(v, top, 4);
  return v > 0.0f ? max((int)code, 1) : 0;
}

// m / (sqrt(v) + eps). It is scaled by lr, far below the parameter: the approximate root and reciprocal serve. They
// take subnormal numbers for zero, so small ones (and the quotient's sides alike) are scaled up by a power of two first.
__device__ __forceinline__ float quotient(float m, float v, float eps) {
#pragma clang fp contract(off)
  const bool low = v < 0x1p-96f;
  const float den = __builtin_amdgcn_sqrtf(low ? v * 0x1p64f : v) * (low ? 0x1p-32f : 1.0f) + eps;
  const float up = den < 0x1p-64f ? 0x1p64f : 1.0f;
  return (m * up) * __builtin_amdgcn_rcpf(den * up);
}

template <int bits>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const Args a) {
#pragma clang fp contract(off)
  const int64_t blk = block_id();
  const float gs = a.grad_scale ? *a.grad_scale : 1.0f;
  const bool skip = !(fabsf(gs) < __builtin_inff());
  if (a.skipped && blk == 0 && threadIdx.x == 0) *a.skipped = skip ? 1 : 0;
  if (skip) return;
  int lo = 0, hi = a.n - 1;  // the last entry whose first workgroup is not past this one
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.e[mid].first <= blk) lo = mid;
    else hi = mid - 1;
  }
  const Entry& t = a.e[lo];
  const int64_t j = (blk - t.first) * kChunk + threadIdx.x * kPer;
  const int64_t left = t.n - j;
  // a block's 32 lanes stay together: all of them leave, or none
  if ((j & ~(int64_t)(ZO_ADAMW_BLOCK - 1)) >= t.n) return;
  float p[kPer], g[kPer], m[kPer], v[kPer];
  if (t.gbf) load8((const uint16_t*)t.g + j, left, g);
  else load8((const float*)t.g + j, left, g);
  if (t.pbf) load8((const uint16_t*)t.p + j, left, p);
  else load8((const float*)t.p + j, left, p);
  const int64_t s = t.off + j;
  float mtop = 0, vtop = 0;
  if constexpr (bits == 8) {
    // the moments' blocks are whole in memory; values past the tensor's end count as zeros
    const uint2 mc = *(const uint2*)((const int8_t*)a.m + s), vc = *(const uint2*)((const uint8_t*)a.v + s);
    mtop = a.ms[s / ZO_ADAMW_BLOCK];
    vtop = a.vs[s / ZO_ADAMW_BLOCK];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const uint32_t mw = e < 4 ? mc.x : mc.y, vw = e < 4 ? vc.x : vc.y;
      m[e] = e < left ? decode_m((int8_t)(mw >> (8 * (e & 3))), mtop) : 0.0f;
      v[e] = e < left ? decode_v((uint8_t)(vw >> (8 * (e & 3))), vtop) : 0.0f;
    }
  } else {
    load8((const float*)a.m + s, left, m);
    load8((const float*)a.v + s, left, v);
  }
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const float ge = a.grad_scale ? g[e] * gs : g[e];
    m[e] = m[e] * a.b1 + ge * a.omb1;
    v[e] = v[e] * a.b2 + (ge * ge) * a.omb2;
    p[e] = p[e] * t.keep - quotient(m[e] * a.c1, v[e] * a.c2, a.eps) * a.lr;
  }
  if (t.pbf) store8((uint16_t*)t.p + j, left, p);
  else store8((float*)t.p + j, left, p);
  if constexpr (bits == 8) {
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      m[e] = e < left ? m[e] : 0.0f;
      v[e] = e < left ? v[e] : 0.0f;
    }
    mtop = block_top(m);
    vtop = block_top(v);
    const float minv = 1.0f / mtop, vinv = 1.0f / vtop;
    uint2 mc{0, 0}, vc{0, 0};
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      uint32_t& mw = e < 4 ? mc.x : mc.y;
      uint32_t& vw = e < 4 ? vc.x : vc.y;
      mw |= (uint32_t)(uint8_t)encode_m(m[e], mtop, minv) << (8 * (e & 3));
      vw |= (uint32_t)(uint8_t)encode_v(v[e], vtop, vinv) << (8 * (e & 3));
    }
    *(uint2*)((int8_t*)a.m + s) = mc;
    *(uint2*)((uint8_t*)a.v + s) = vc;
    if ((threadIdx.x & 31) == 0) {
      a.ms[s / ZO_ADAMW_BLOCK] = mtop;
      a.vs[s / ZO_ADAMW_BLOCK] = vtop;
    }
  } else {
    store8((float*)a.m + s, left, m);
    store8((float*)a.v + s, left, v);
  }
}

// The values that 8-bit moments stand for: 4 a thread.
__global__ __launch_bounds__(kThreads) void adamw_moments_kernel(int64_t n, const uint8_t* m, const uint8_t* v,
                                                                 const float* ms, const float* vs, float* mo,
                                                                 float* vo) {
  const int64_t j = (block_id() * kThreads + threadIdx.x) * 4;
  if (j >= n) return;
  const uint32_t mc = *(const uint32_t*)(m + j), vc = *(const uint32_t*)(v + j);
  const float mt = ms[j / ZO_ADAMW_BLOCK], vt = vs[j / ZO_ADAMW_BLOCK];
  float4 mf, vf;
  mf.x = decode_m((int8_t)mc, mt);
  mf.y = decode_m((int8_t)(mc >> 8), mt);
  mf.z = decode_m((int8_t)(mc >> 16), mt);
  mf.w = decode_m((int8_t)(mc >> 24), mt);
  vf.x = decode_v((uint8_t)vc, vt);
  vf.y = decode_v((uint8_t)(vc >> 8), vt);
  vf.z = decode_v((uint8_t)(vc >> 16), vt);
  vf.w = decode_v((uint8_t)(vc >> 24), vt);
  *(float4*)(mo + j) = mf;
  *(float4*)(vo + j) = vf;
}

}  // namespace

hipError_t launch_adamw(const zo_adamw_config& cfg, const zo_adamw_tensor* t, int32_t n, void* m, void* v,
                        float* ms, float* vs, const float* grad_scale, int32_t* skipped, hipStream_t st) {
  Args a;
  a.b1 = (float)cfg.beta1;
  a.omb1 = (float)(1.0 - cfg.beta1);
  a.b2 = (float)cfg.beta2;
  a.omb2 = (float)(1.0 - cfg.beta2);
  a.c1 = (float)(1.0 / (1.0 - std::pow(cfg.beta1, (double)cfg.step)));
  a.c2 = (float)(1.0 / (1.0 - std::pow(cfg.beta2, (double)cfg.step)));
  a.eps = (float)cfg.eps;
  a.lr = (float)cfg.lr;
  a.m = m;
  a.v = v;
  a.ms = ms;
  a.vs = vs;
  a.grad_scale = grad_scale;
  a.skipped = skipped;
  // without a value to update the first launch still reports whether the step was skipped
  for (int32_t i = 0, launched = 0; i < n || (skipped && !launched); ++launched) {
    a.n = 0;
    int64_t blocks = 0;
    for (; i < n && a.n < kTensors; ++i) {
      if (t[i].n == 0) continue;
      Entry& e = a.e[a.n++];
      e.p = t[i].param;
      e.g = t[i].grad;
      e.n = t[i].n;
      e.off = t[i].state_offset;
      e.first = blocks;
      e.keep = (float)(1.0 - cfg.lr * t[i].weight_decay);
      e.pbf = t[i].pdtype == ZO_WBF16;
      e.gbf = t[i].gdtype == ZO_WBF16;
      blocks += (t[i].n + kChunk - 1) / kChunk;
    }
    if (a.n == 0) {
      if (!a.skipped || launched) break;
      // an entry of no values: its workgroup leaves at once
      a.e[a.n++] = Entry{nullptr, nullptr, 0, 0, 0, 1.0f, 0, 0};
      blocks = 1;
    }
    const dim3 grid = wide_grid(blocks);
    if (cfg.state_bits == 8) adamw_kernel<8><<<grid, kThreads, 0, st>>>(a);
    else adamw_kernel<32><<<grid, kThreads, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.skipped = nullptr;
  }
  return hipSuccess;
}

hipError_t launch_adamw_moments(int64_t n, const void* m, const void* v, const float* ms, const float* vs, float* mo,
                                float* vo, hipStream_t st) {
  if (n == 0) return hipSuccess;
  adamw_moments_kernel<<<wide_grid((n / 4 + kThreads - 1) / kThreads), kThreads, 0, st>>>(
      n, (const uint8_t*)m, (const uint8_t*)v, ms, vs, mo, vo);
  return hipGetLastError();
}

}  // namespace zo
