// Linear attention, one token for each sequence: S = gamma S + k v^T,
// o = scale S^T q, the state read once and written once. That traffic, 8 bytes
// per value of the state, is all the time there is (2 to 5 operations a value),
// so the layout serves it: a workgroup holds all rows of 64 columns of one
// state, 16 lanes by 16 bytes to a row, all of a thread's loads (up to 16) in
// flight before the first is used. The state stays in registers for every query
// head that reads it; their sums over the rows go through lane exchanges and
// LDS. 224 sequences, 32 states of 128 x 128 each: 0.95 GB in 187 us, 5.05 TB/s (a
// copy of 4 GiB: 4.75); 4 sequences of 8 states: 5.6 us, a launch and one trip to memory.
#include <hip/hip_runtime.h>

#include "zo_layers.hpp"

namespace zo {
namespace {

constexpr int kCols = 64;      // columns of a workgroup
constexpr int kRowGroups = 16; // thread t: columns 4 (t % 16) .., rows t / 16 + 16 i
constexpr int kHeads = 4;      // query heads per turn

template <typename T, int ROWS>
__global__ __launch_bounds__(256) void linattn_step_kernel(LinStep a) {
  __shared__ float ks[ROWS * kRowGroups];
  __shared__ float qs[kHeads][ROWS * kRowGroups];
  __shared__ float part[kHeads][4][kCols];
  const int tid = threadIdx.x, c4 = (tid & 15) * 4, rg = tid >> 4;
  const int slices = (a.dv + kCols - 1) / kCols;
  const int64_t blk = block_id(), bh = blk / slices;
  const int b = (int)(bh / a.kv_heads), h = (int)(bh % a.kv_heads);
  if (b >= a.B) return;  // the last row of a wide grid
  const int col = (int)(blk % slices) * kCols;
  const int groups = a.q_heads / a.kv_heads;
  T* o = (T*)a.o + b * a.ob + (int64_t)h * groups * a.oh + col;
  const int64_t slot = a.slots ? a.slots[b] : b;
  if (slot < 0 || slot >= a.n_slots) {
    const float nothing = slot == -1 ? 0.0f : __builtin_nanf("");
    if (tid < kCols && col + tid < a.dv)
      for (int g = 0; g < groups; ++g) o[g * a.oh + tid] = from_f32<T>(nothing);
    return;
  }
  float* S = a.state + (slot * a.kv_heads + h) * (int64_t)a.dk * a.dv + col + c4;
  const int left = a.dv - col - c4;  // columns of this thread that exist: 4 or fewer
  float s[ROWS][4];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int r = rg + kRowGroups * i;
    if (r < a.dk && left >= 4) {
      load_run<float, 4>(S + (int64_t)r * a.dv, s[i]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) s[i][e] = r < a.dk && e < left ? S[(int64_t)r * a.dv + e] : 0.0f;
    }
  }
  const T* k = (const T*)a.k.p + b * a.k.b + h * a.k.h;
  const T* v = (const T*)a.v.p + b * a.v.b + h * a.v.h + col + c4;
  float vs[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) vs[e] = e < left ? to_f32(v[e]) : 0.0f;
  for (int d = tid; d < ROWS * kRowGroups; d += 256) ks[d] = d < a.dk ? to_f32(k[d]) : 0.0f;
  const Gamma gamma(a.log_decay[h]);
  for (int g0 = 0; g0 < groups; g0 += kHeads) {
    const int n = min(kHeads, groups - g0);
    for (int i = 0; i < n; ++i) {
      const T* q = (const T*)a.q.p + b * a.q.b + (int64_t)(h * groups + g0 + i) * a.q.h;
      for (int d = tid; d < ROWS * kRowGroups; d += 256) qs[i][d] = d < a.dk ? to_f32(q[d]) : 0.0f;
    }
    __syncthreads();
    if (g0 == 0) {
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        const int r = rg + kRowGroups * i;
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][e] = gamma.times(s[i][e], ks[r] * vs[e]);
        if (r < a.dk && left >= 4) {
          store_run<float, 4>(S + (int64_t)r * a.dv, s[i]);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (r < a.dk && e < left) S[(int64_t)r * a.dv + e] = s[i][e];
        }
      }
    }
    for (int i = 0; i < n; ++i) {
      float acc[4] = {0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < ROWS; ++j) {
        const float q = qs[i][rg + kRowGroups * j];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = fmaf(q, s[j][e], acc[e]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc[e] += __shfl_xor(acc[e], 16, 64);
        acc[e] += __shfl_xor(acc[e], 32, 64);
        if ((tid & 63) < 16) part[i][tid >> 6][c4 + e] = acc[e];
      }
    }
    __syncthreads();
    for (int x = tid; x < n * kCols; x += 256) {
      const int i = x / kCols, c = x % kCols;
      if (col + c < a.dv)
        o[(g0 + i) * a.oh + c] =
            from_f32<T>(a.scale * ((part[i][0][c] + part[i][1][c]) + (part[i][2][c] + part[i][3][c])));
    }
  }
}

template <typename T>
hipError_t launch(const LinStep& a, hipStream_t s) {
  const int slices = (a.dv + kCols - 1) / kCols;
  const dim3 grid = wide_grid((int64_t)a.B * a.kv_heads * slices);
  if (a.dk <= 64) linattn_step_kernel<T, 4><<<grid, 256, 0, s>>>(a);
  else if (a.dk <= 128) linattn_step_kernel<T, 8><<<grid, 256, 0, s>>>(a);
  else linattn_step_kernel<T, 16><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_linattn_step(const LinStep& a, hipStream_t s) {
  if (a.B == 0) return hipSuccess;
  return a.dtype == ZO_WBF16 ? launch<uint16_t>(a, s) : launch<float>(a, s);
}

}  // namespace zo
