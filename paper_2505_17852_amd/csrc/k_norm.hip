// Layer norm, forward and backward, over rows of D values.
//
// forward   mean and variance of the row (two passes over values held in
//           registers: the variance is of x - mean, so a large mean costs no
//           precision), y = (x - mean) rstd w + b
// backward  g = dy w, xhat = (x - mean) rstd,
//           dx = rstd (g - avg(g) - xhat avg(g xhat)),
//           dw = sum dy xhat, db = sum dy over the rows
//
// Both are bound by memory: each input is read once and each output written
// once. A row belongs to 64 or 256 threads, the fewest that hold it in 16
// registers each (a wave exchanges its sums without a barrier; more threads
// leave fewer loads per thread in flight), or to 1,024 threads with 8 each (16
// do not fit the registers of so many). Rows beyond 8,192 values are read again
// for every pass (the loop kernels).
//
// 65,536 rows of 4,096 (bf16), forward and backward with the weight's gradients: 2.7 GB in 0.51 ms, 5.2 TB/s (a
// copy of 4 GiB: 4.75); without the next row's loads ahead and with the weights read for every row
// 0.76 ms. 4,097 rows of 1,003 (fp32): 25 us, three launches of 9, 13 and 4 us.
//
// The weight's gradients: a workgroup of the backward pass walks over many rows
// and keeps its threads' columns' sums in registers; the workgroups' sums go to
// the workspace, and a second launch adds them, in workgroup order: the same
// bits every time, no atomics.
#include <hip/hip_runtime.h>

#include "zo_layers.hpp"

namespace zo {
namespace {

constexpr int kMaxParts = 512;  // workgroups of a backward pass
constexpr int kLoopThreads = 1024;

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d, 64);
  return x;
}

// Sums of N values over the TPR threads of a row; `buf` alternates between two
// arrays of a wave's sums, so that one barrier per call is enough.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&s)[N], float (*buf)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] = wave_sum(s[i]);
  if constexpr (TPR > 64) {
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) buf[w][i] = s[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      s[i] = 0;
#pragma unroll
      for (int k = 0; k < TPR / 64; ++k) s[i] += buf[k][i];
    }
  }
}

// Values of a row per thread.
template <int TPR>
constexpr int vals_of() { return TPR > 256 ? 8 : 16; }

// A thread's values of a row: runs of VEC at (c TPR + lane) VEC.
template <typename T>
constexpr int vec_of() { return sizeof(T) == 2 ? 8 : 4; }

// A row as it lies in memory, on its way to a thread's registers, 16 bytes a run. No branch stands around a load, so
// that the next row's loads stay in flight while this one is worked on: runs past the end repeat the
// last 16 bytes, and the run that the row ends in (D not a multiple of VEC) is the last 16 bytes,
// moved down when it is used. D is VEC at least, but for short rows.
template <typename T, int TPR, bool even>
struct RawRow {
  static constexpr int VEC = vec_of<T>(), N = vals_of<TPR>() / VEC;
  u4 v[N];
  __device__ __forceinline__ void load(const T* p, int lane, int D) {
    if (even || D >= VEC) {
#pragma unroll
      for (int c = 0; c < N; ++c) v[c] = load16(p + min((c * TPR + lane) * VEC, D - VEC));
    } else {
      T few[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) few[e] = p[min(e, D - 1)];
#pragma unroll
      for (int c = 0; c < N; ++c) v[c] = __builtin_bit_cast(u4, few);
    }
  }
  // fp32, zeros past the row's end
  __device__ __forceinline__ void get(int lane, int D, float* out) const {
#pragma unroll
    for (int c = 0; c < N; ++c) {
      const int j = (c * TPR + lane) * VEC;
      u4 run = v[c];
      if constexpr (!even) run = drop<T>(run, D >= VEC ? min(max(j - (D - VEC), 0), VEC - 1) : 0);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const uint32_t word = sizeof(T) == 4 ? run[e] : e & 1 ? run[e / 2] & 0xffff0000u : run[e / 2] << 16;
        out[c * VEC + e] = (even ? j : j + e) < D ? __uint_as_float(word) : 0.0f;
      }
    }
  }
};
// Weights, read once per workgroup, in the runs of x.
template <typename T, int TPR, int VEC>
__device__ __forceinline__ void load_row(const T* p, int lane, int D, float* out) {
#pragma unroll
  for (int c = 0; c < vals_of<TPR>() / VEC; ++c) {
    const int j = (c * TPR + lane) * VEC;
    if (j + VEC <= D) {
      load_run<T, VEC>(p + j, out + c * VEC);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) out[c * VEC + e] = j + e < D ? to_f32(p[j + e]) : 0.0f;
    }
  }
}

template <typename T, int TPR, int VEC>
__device__ __forceinline__ void store_row(T* p, int lane, int D, const float* in) {
  constexpr int kVals = vals_of<TPR>();
#pragma unroll
  for (int c = 0; c < kVals / VEC; ++c) {
    const int j = (c * TPR + lane) * VEC;
    if (j + VEC <= D) {
      store_run<T, VEC>(p + j, in + c * VEC);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (j + e < D) p[j + e] = from_f32<T>(in[c * VEC + e]);
    }
  }
}

// Rows per workgroup at a time: waves of their own rows where one wave holds a row.
template <int TPR>
constexpr int threads_of() { return TPR > 256 ? TPR : 256; }
template <int TPR>
constexpr int rows_of() { return threads_of<TPR>() / TPR; }

template <typename T, typename W, int TPR, bool even>
__global__ __launch_bounds__(threads_of<TPR>()) void norm_kernel(NormArgs a) {
  constexpr int VEC = vec_of<T>(), RPB = rows_of<TPR>(), kVals = vals_of<TPR>();
  __shared__ float buf[2][TPR / 64][1];
  const int lane = threadIdx.x % TPR, D = (int)a.D;
  const int64_t step = (int64_t)gridDim.x * RPB;
  int64_t r = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
  RawRow<T, TPR, even> raw;
  if (r < a.rows) raw.load((const T*)a.x + r * a.xs, lane, D);
  float w[kVals], b[kVals];
#pragma unroll
  for (int i = 0; i < kVals; ++i) {
    w[i] = 1.0f;
    b[i] = 0.0f;
  }
  if (a.w) load_row<W, TPR, VEC>((const W*)a.w, lane, D, w);
  if (a.b) load_row<W, TPR, VEC>((const W*)a.b, lane, D, b);
  for (; r < a.rows; r += step) {
    float x[kVals];
    raw.get(lane, D, x);
    raw.load((const T*)a.x + (r + step < a.rows ? r + step : r) * a.xs, lane, D);
    float s[1] = {0};
#pragma unroll
    for (int i = 0; i < kVals; ++i) s[0] += x[i];
    row_sums<TPR, 1>(s, buf[0]);
    const float mean = s[0] / (float)D;
    s[0] = 0;
#pragma unroll
    for (int c = 0; c < kVals / VEC; ++c)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        float& v = x[c * VEC + e];
        const int j = (c * TPR + lane) * VEC;
        v = (even ? j : j + e) < D ? v - mean : 0.0f;
        s[0] += v * v;
      }
    row_sums<TPR, 1>(s, buf[1]);
    const float rstd = 1.0f / sqrtf(s[0] / (float)D + a.eps);
#pragma unroll
    for (int i = 0; i < kVals; ++i) x[i] = x[i] * rstd * w[i] + b[i];
    store_row<T, TPR, VEC>((T*)a.y + r * a.ys, lane, D, x);
    if (a.mean && lane == 0) {
      a.mean[r] = mean;
      a.rstd[r] = rstd;
    }
  }
}

template <typename T, typename W, int TPR, bool even>
__global__ __launch_bounds__(threads_of<TPR>()) void norm_backward_kernel(NormArgs a) {
  constexpr int VEC = vec_of<T>(), RPB = rows_of<TPR>(), NT = threads_of<TPR>(), kVals = vals_of<TPR>();
  __shared__ float buf[2][TPR / 64][2];
  __shared__ float join[RPB > 1 ? kVals * NT : 1];
  const int lane = threadIdx.x % TPR, D = (int)a.D;
  const int64_t step = (int64_t)gridDim.x * RPB;
  int64_t r = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
  RawRow<T, TPR, even> rx, rdy;
  float mean = 0, rstd = 0;
  const auto load = [&](int64_t r) {
    rx.load((const T*)a.x + r * a.xs, lane, D);
    rdy.load((const T*)a.dy + r * a.dys, lane, D);
    mean = a.mean[r];
    rstd = a.rstd[r];
  };
  if (r < a.rows) load(r);
  float w[kVals], dw[kVals], db[kVals];
#pragma unroll
  for (int i = 0; i < kVals; ++i) {
    w[i] = 1.0f;
    dw[i] = 0.0f;
    db[i] = 0.0f;
  }
  if (a.w) load_row<W, TPR, VEC>((const W*)a.w, lane, D, w);
  int turn = 0;
  for (; r < a.rows; r += step) {
    float x[kVals], dy[kVals];
    rx.get(lane, D, x);
    rdy.get(lane, D, dy);
    const float rs = rstd;
    // zero past the row's end too: a large mean times rstd may not be finite where no value is
#pragma unroll
    for (int c = 0; c < kVals / VEC; ++c)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        float& v = x[c * VEC + e];
        const int j = (c * TPR + lane) * VEC;
        v = (even ? j : j + e) < D ? (v - mean) * rs : 0.0f;
      }
    // the next row's loads before this one's sums (the last row has none: itself once more, in place or not)
    load(r + step < a.rows ? r + step : r);
    float s[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < kVals; ++i) {
      db[i] += dy[i];
      dw[i] += dy[i] * x[i];
      dy[i] *= w[i];
      s[0] += dy[i];
      s[1] += dy[i] * x[i];
    }
    row_sums<TPR, 2>(s, buf[turn]);
    turn ^= 1;
    const float m0 = s[0] / (float)D, m1 = s[1] / (float)D;
#pragma unroll
    for (int i = 0; i < kVals; ++i) x[i] = rs * (dy[i] - m0 - x[i] * m1);
    store_row<T, TPR, VEC>((T*)a.y + r * a.ys, lane, D, x);
  }
  if (!a.partial) return;
  // the workgroup's sums: [workgroup][dw, db][D]
  float* part = a.partial + (int64_t)blockIdx.x * 2 * D;
  if constexpr (RPB > 1) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kVals; ++i) join[i * NT + threadIdx.x] = q ? db[i] : dw[i];
      __syncthreads();
      if (threadIdx.x < TPR)
#pragma unroll
        for (int i = 0; i < kVals; ++i) {
          float& v = q ? db[i] : dw[i];
          v = 0;
#pragma unroll
          for (int k = 0; k < RPB; ++k) v += join[i * NT + k * TPR + threadIdx.x];
        }
    }
    if (threadIdx.x >= TPR) return;
  }
  store_row<float, TPR, VEC>(part, lane, D, dw);
  store_row<float, TPR, VEC>(part + D, lane, D, db);
}

// Adds the workgroups' sums: 64 columns by 16 shares of the workgroups, then the shares (a tree, so that no chain of
// loads is longer than 32).
__global__ __launch_bounds__(1024) void norm_sums_kernel(const float* partial, int parts, int64_t D, float* dw,
                                                         float* db) {
  __shared__ float join[16][64];
  float* out = blockIdx.z ? db : dw;
  if (!out) return;
  const int c = threadIdx.x & 63, share = threadIdx.x >> 6;
  const int64_t j = block_id() * 64 + c;
  float s = 0;
  if (j < D) {
    const float* p = partial + blockIdx.z * D + j;
#pragma unroll 8
    for (int k = share; k < parts; k += 16) s += p[(int64_t)k * 2 * D];
  }
  join[share][c] = s;
  __syncthreads();
#pragma unroll
  for (int half = 8; half; half >>= 1) {
    if (share < half) join[share][c] += join[share + half][c];
    __syncthreads();
  }
  if (share == 0 && j < D) out[j] = join[0][c];
}

// Rows of any length: a workgroup per row, every pass reads the row again.
template <typename T, typename W>
__global__ __launch_bounds__(kLoopThreads) void norm_loop_kernel(NormArgs a) {
  __shared__ float buf[2][kLoopThreads / 64][1];
  for (int64_t r = block_id(); r < a.rows; r += (int64_t)gridDim.x * gridDim.y) {
    const T* x = (const T*)a.x + r * a.xs;
    float s[1] = {0};
    for (int64_t j = threadIdx.x; j < a.D; j += kLoopThreads) s[0] += to_f32(x[j]);
    row_sums<kLoopThreads, 1>(s, buf[0]);
    const float mean = s[0] / (float)a.D;
    s[0] = 0;
    for (int64_t j = threadIdx.x; j < a.D; j += kLoopThreads) {
      const float v = to_f32(x[j]) - mean;
      s[0] += v * v;
    }
    row_sums<kLoopThreads, 1>(s, buf[1]);
    const float rstd = 1.0f / sqrtf(s[0] / (float)a.D + a.eps);
    T* y = (T*)a.y + r * a.ys;
    for (int64_t j = threadIdx.x; j < a.D; j += kLoopThreads) {
      const float w = a.w ? to_f32(((const W*)a.w)[j]) : 1.0f, b = a.b ? to_f32(((const W*)a.b)[j]) : 0.0f;
      y[j] = from_f32<T>((to_f32(x[j]) - mean) * rstd * w + b);
    }
    if (a.mean && threadIdx.x == 0) {
      a.mean[r] = mean;
      a.rstd[r] = rstd;
    }
  }
}
template <typename T, typename W>
__global__ __launch_bounds__(kLoopThreads) void norm_backward_loop_kernel(NormArgs a) {
  __shared__ float buf[2][kLoopThreads / 64][2];
  int turn = 0;
  for (int64_t r = block_id(); r < a.rows; r += (int64_t)gridDim.x * gridDim.y) {
    const T *x = (const T*)a.x + r * a.xs, *dy = (const T*)a.dy + r * a.dys;
    const float mean = a.mean[r], rstd = a.rstd[r];
    float s[2] = {0, 0};
    for (int64_t j = threadIdx.x; j < a.D; j += kLoopThreads) {
      const float g = to_f32(dy[j]) * (a.w ? to_f32(((const W*)a.w)[j]) : 1.0f);
      s[0] += g;
      s[1] += g * ((to_f32(x[j]) - mean) * rstd);
    }
    row_sums<kLoopThreads, 2>(s, buf[turn]);
    turn ^= 1;
    const float m0 = s[0] / (float)a.D, m1 = s[1] / (float)a.D;
    T* dx = (T*)a.y + r * a.ys;
    for (int64_t j = threadIdx.x; j < a.D; j += kLoopThreads) {
      const float g = to_f32(dy[j]) * (a.w ? to_f32(((const W*)a.w)[j]) : 1.0f);
      dx[j] = from_f32<T>(rstd * (g - m0 - (to_f32(x[j]) - mean) * rstd * m1));
    }
  }
}
// Column sums of long rows, before dx is written (it may replace dy or x): a
// thread per column and share of the rows.
template <typename T>
__global__ __launch_bounds__(256) void norm_columns_kernel(NormArgs a, int parts) {
  const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (j >= a.D) return;
  float dw = 0, db = 0;
  for (int64_t r = blockIdx.y; r < a.rows; r += parts) {
    const float g = to_f32(((const T*)a.dy)[r * a.dys + j]);
    db += g;
    dw += g * ((to_f32(((const T*)a.x)[r * a.xs + j]) - a.mean[r]) * a.rstd[r]);
  }
  float* part = a.partial + (int64_t)blockIdx.y * 2 * a.D;
  part[j] = dw;
  part[a.D + j] = db;
}

int row_threads(int64_t D) { return D <= 1024 ? 64 : D <= 4096 ? 256 : D <= 8192 ? 1024 : 0; }

// Workgroups of a backward pass, each with sums of its own.
int parts_of(int64_t rows, int64_t D) {
  const int tpr = row_threads(D);
  const int64_t need = tpr == 64 ? (rows + 3) / 4 : rows;
  return (int)(need < kMaxParts ? need : kMaxParts);
}

// Workgroups of a forward pass: each keeps weight and bias for all its rows.
constexpr int kMaxForward = 2048;

template <typename T, typename W, bool even>
hipError_t forward_as(const NormArgs& a, hipStream_t s) {
  const int tpr = row_threads(a.D);
  const int64_t need = tpr == 64 ? (a.rows + 3) / 4 : a.rows;
  const unsigned grid = (unsigned)(need < kMaxForward ? need : kMaxForward);
  if (tpr == 64) norm_kernel<T, W, 64, even><<<grid, 256, 0, s>>>(a);
  else if (tpr == 256) norm_kernel<T, W, 256, even><<<grid, 256, 0, s>>>(a);
  else if (tpr == 1024) norm_kernel<T, W, 1024, even><<<grid, 1024, 0, s>>>(a);
  else norm_loop_kernel<T, W><<<wide_grid(a.rows), kLoopThreads, 0, s>>>(a);
  return hipGetLastError();
}
template <typename T, typename W>
hipError_t forward(const NormArgs& a, hipStream_t s) {
  return a.D % vec_of<T>() == 0 ? forward_as<T, W, true>(a, s) : forward_as<T, W, false>(a, s);
}

template <typename T, typename W, bool even>
void backward_as(const NormArgs& a, int parts, hipStream_t s) {
  const int tpr = row_threads(a.D);
  if (tpr == 64) norm_backward_kernel<T, W, 64, even><<<parts, 256, 0, s>>>(a);
  else if (tpr == 256) norm_backward_kernel<T, W, 256, even><<<parts, 256, 0, s>>>(a);
  else if (tpr == 1024) norm_backward_kernel<T, W, 1024, even><<<parts, 1024, 0, s>>>(a);
  else {
    if (a.partial) norm_columns_kernel<T><<<dim3((unsigned)((a.D + 255) / 256), parts), 256, 0, s>>>(a, parts);
    norm_backward_loop_kernel<T, W><<<wide_grid(a.rows), kLoopThreads, 0, s>>>(a);
  }
}
template <typename T, typename W>
hipError_t backward(const NormArgs& a, hipStream_t s) {
  const int parts = parts_of(a.rows, a.D);
  if (a.rows) {
    if (a.D % vec_of<T>() == 0) backward_as<T, W, true>(a, parts, s);
    else backward_as<T, W, false>(a, parts, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.dw || a.db) {
    dim3 grid = wide_grid((a.D + 63) / 64);  // (rows of 2^28 values and more: 2^32 threads)
    grid.z = 2;
    norm_sums_kernel<<<grid, 1024, 0, s>>>(a.partial, parts, a.D, a.dw, a.db);
  }
  return hipGetLastError();
}

template <typename F>
hipError_t by_type(const NormArgs& a, F f) {
  const bool xb = a.xdtype == ZO_WBF16, wb = a.wdtype == ZO_WBF16;
  if (xb) return wb ? f((uint16_t*)nullptr, (uint16_t*)nullptr) : f((uint16_t*)nullptr, (float*)nullptr);
  return wb ? f((float*)nullptr, (uint16_t*)nullptr) : f((float*)nullptr, (float*)nullptr);
}

}  // namespace

size_t norm_workspace(int64_t rows, int64_t D) { return (size_t)parts_of(rows, D) * 2 * (size_t)D * sizeof(float); }

hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  return by_type(a, [&](auto t, auto w) {
    return forward<std::remove_pointer_t<decltype(t)>, std::remove_pointer_t<decltype(w)>>(a, s);
  });
}

hipError_t launch_norm_backward(const NormArgs& a, hipStream_t s) {
  return by_type(a, [&](auto t, auto w) {
    return backward<std::remove_pointer_t<decltype(t)>, std::remove_pointer_t<decltype(w)>>(a, s);
  });
}

}  // namespace zo
