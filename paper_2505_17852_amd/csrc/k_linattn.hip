// Linear attention with a decay for each head over whole sequences.
//
// The forward pass and the three gradients are one recurrence with different
// operands, forward or backward in time (S' = S^T):
//   o   S  = gamma S + k v^T,             o  = scale S^T q         forward
//   dq  S' = gamma S' + v k^T,            dq = scale S'^T do       forward
//   dv  R  = gamma (R + scale q do^T),    dv = (R + scale q do^T)^T k     backward, sum over query heads
//   dk  R' = gamma (R' + scale do q^T),   dk = (R' + scale do q^T)^T v    backward, sum over query heads
// so a pass reads x (the reader), y and z (the products' sides) and writes out
// [positions][dz], with the state R [dx][dz]; a workgroup takes one sequence,
// one output head and a slice of the columns dz.
#include <hip/hip_runtime.h>

#include "zo_layers.hpp"

namespace zo {
namespace {

constexpr int kCols = 64;
constexpr int kRowGroups = 16;

// Position by position: the state in registers (thread t: columns 4 (t % 16) ..,
// rows t / 16 + 16 i).
template <typename T, int ROWS>
__global__ __launch_bounds__(256) void linattn_token_kernel(LinCall c) {
  __shared__ float xs[ROWS * kRowGroups];
  __shared__ float ys[ROWS * kRowGroups];
  __shared__ float part[4][kCols];
  const LinPass& a = c.pass[blockIdx.z];
  const int tid = threadIdx.x, c4 = (tid & 15) * 4, rg = tid >> 4;
  const int slices = (a.dz + kCols - 1) / kCols;
  const int64_t blk = block_id(), bh = blk / slices;
  const int b = (int)(bh / a.out_heads), h = (int)(bh % a.out_heads);
  if (b >= c.B) return;
  const int col = (int)(blk % slices) * kCols;
  const int state = h / a.share;  // the key/value head
  const int n = c.lengths ? min(max(c.lengths[b], 0), c.T) : c.T;
  T* out = (T*)a.out + b * a.ob + h * a.oh + col;
  const float gamma = expf(c.log_decay[state]);
  const int64_t state_at = ((int64_t)b * c.kv_heads + state) * a.dx * a.dz;
  float s[ROWS][4];
#pragma unroll
  for (int i = 0; i < ROWS; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = rg + kRowGroups * i, z = col + c4 + e;
      s[i][e] = a.init && r < a.dx && z < a.dz ? a.init[state_at + (a.state_t ? (int64_t)z * a.dx + r : (int64_t)r * a.dz + z)] : 0.0f;
    }
  for (int t = n; t < c.T; ++t)
    if (tid < kCols && col + tid < a.dz) out[t * a.ot + tid] = from_f32<T>(0.0f);
  for (int u = 0; u < n; ++u) {
    const int64_t t = a.reverse ? n - 1 - u : u;
    if (!a.reverse)
#pragma unroll
      for (int i = 0; i < ROWS; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][e] *= gamma;
    for (int src = 0; src < a.sources; ++src) {
      const int yh = state * a.sources + src;
      __syncthreads();
      for (int d = tid; d < ROWS * kRowGroups; d += 256) {
        ys[d] = d < a.dx ? to_f32(((const T*)a.y.p)[b * a.y.b + t * a.y.t + yh * a.y.h + d]) : 0.0f;
        if (src == 0) xs[d] = d < a.dx ? to_f32(((const T*)a.x.p)[b * a.x.b + t * a.x.t + h * a.x.h + d]) : 0.0f;
      }
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int z = col + c4 + e;
        const float zv = z < a.dz ? a.upd * to_f32(((const T*)a.z.p)[b * a.z.b + t * a.z.t + yh * a.z.h + z]) : 0.0f;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) s[i][e] = fmaf(ys[rg + kRowGroups * i], zv, s[i][e]);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float acc = 0;
#pragma unroll
      for (int i = 0; i < ROWS; ++i) acc = fmaf(xs[rg + kRowGroups * i], s[i][e], acc);
      acc += __shfl_xor(acc, 16, 64);
      acc += __shfl_xor(acc, 32, 64);
      if ((tid & 63) < 16) part[tid >> 6][c4 + e] = acc;
    }
    __syncthreads();
    if (tid < kCols && col + tid < a.dz)
      out[t * a.ot + tid] = from_f32<T>(a.carry * ((part[0][tid] + part[1][tid]) + (part[2][tid] + part[3][tid])));
    if (a.reverse)
#pragma unroll
      for (int i = 0; i < ROWS; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][e] *= gamma;
  }
  if (a.fin && h % a.share == 0)
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = rg + kRowGroups * i, z = col + c4 + e;
        if (r < a.dx && z < a.dz) a.fin[state_at + (a.state_t ? (int64_t)z * a.dx + r : (int64_t)r * a.dz + z)] = s[i][e];
      }
}

template <typename T>
hipError_t launch(const LinCall& c, hipStream_t st) {
  int64_t blocks = 0;
  int dx = 0;
  for (int i = 0; i < c.npasses; ++i) {
    const LinPass& p = c.pass[i];
    blocks = std::max(blocks, (int64_t)c.B * p.out_heads * ((p.dz + kCols - 1) / kCols));
    dx = std::max(dx, p.dx);
  }
  dim3 grid = wide_grid(blocks);
  grid.z = c.npasses;
  if (dx <= 64) linattn_token_kernel<T, 4><<<grid, 256, 0, st>>>(c);
  else if (dx <= 128) linattn_token_kernel<T, 8><<<grid, 256, 0, st>>>(c);
  else linattn_token_kernel<T, 16><<<grid, 256, 0, st>>>(c);
  return hipGetLastError();
}

}  // namespace

size_t linattn_workspace(const zo_linattn&, bool) { return 0; }

hipError_t launch_linattn(const LinCall& c, hipStream_t s) {
  if (c.B == 0) return hipSuccess;
  return c.dtype == ZO_WBF16 ? launch<uint16_t>(c, s) : launch<float>(c, s);
}

}  // namespace zo
