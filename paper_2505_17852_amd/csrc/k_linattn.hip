// Linear attention with a decay for each head over whole sequences.
//
// The forward pass and the three gradients are one recurrence with different
// operands, forward or backward in time (S' = S^T):
//   o   S  = gamma S + k v^T,             o  = scale S^T q         forward
//   dq  S' = gamma S' + v k^T,            dq = scale S'^T do       forward
//   dv  R  = gamma (R + scale q do^T),    dv = (R + scale q do^T)^T k     backward, sum over query heads
//   dk  R' = gamma (R' + scale do q^T),   dk = (R' + scale do q^T)^T v    backward, sum over query heads
// so a pass reads x (the reader), y and z (the products' sides) and writes out
// [positions][dz], with the state R [dx][dz].
//
// In chunks of 64 positions (counted in the pass's direction; off = 1 forward,
// 0 backward, where the state that is carried has decayed already):
//   P_ij  = score gamma^(i-j) (x_i . y_j)   for j <= i
//   out_i = sum_j P_ij z_j + carry gamma^(i+off) R^T x_i
//   R     = gamma^64 R + sum_j upd gamma^(64-off-j) y_j z_j^T
// every sum a matrix product. A workgroup of four waves walks over the chunks of
// one sequence, head and slice of 64 or 128 columns of z with R in its accumulators:
// x, y, z are read and out is written once per slice (the slices and passes of a
// state run next to each other on one XCD, whose L2 serves the second reading).
// Wave w has the chunk's rows 16 w .. 16 w + 15 and a quarter of R's columns (so that only a quarter of z is
// scaled by each).
//
// Operands. MFMA 16x16: A and B have the same lane layout, lane l = row (or column)
// l % 16, contraction index group l / 16; the result has column l % 16 and
// rows 4 (l / 16) + r. Scores are formed as P^T (y x^T), so that a lane holds
// P_ij of its row i = l % 16 for 4 positions j of each tile of 16: taken in that order of j,
// the accumulators are the next product's operand as they are. The other operand of
// the sums over j (columns of y and z by rows j) is read from row-major LDS tiles in the
// same order: with the transposing LDS load (bf16), or by words (fp32). out is
// formed transposed too, so that a lane holds 4 neighbouring columns of one row.
//
// Precision: fp32 accumulators and state. With bf16 inputs P, and R where x reads it, meet
// them as two bf16 parts each, which leave out 2^-16 at most: the outputs' error is that of their own
// rounding (one part each adds another of that size: 1.4 times the error, for a tenth less time, a sixth where
// slices have 128 columns). The state's own sum takes gamma^(..) z in
// three bf16 parts, all of its fp32 value, since what is lost there would stay for all later
// positions. fp32 runs on fp32 MFMAs throughout.
//
// Slices of 128 columns: both parts of all of R would leave LDS for one workgroup per CU, so x
// reads 64 columns at a time, with two barriers more.
//
// Positions past a sequence's length are never read. P of later positions is set
// to zero, not multiplied by it; a z that is not finite would still turn those zeros
// into NaN, so chunks that hold one (seen when it is staged) take z without it
// and add its products to the rows that it reaches.
//
// Few sequences: where the workgroups would not fill the chip the positions are split
// into segments; a first launch runs only the state's sum of every segment
// but the last, a second adds the segments up, and the main launch starts each
// segment from its own state.
//
// What bounds it. bf16, 16 sequences of 1,024 positions, 32 heads of 128: the forward pass moves its 0.54 GB in
// 0.16 ms (3.4 TB/s, a large copy reaches 4.75); the backward pass reads nine tensors for the four it needs
// (its three passes share most of that in L2) and takes 0.43 ms. There and on shorter or
// fewer sequences (32 ragged ones of up to 777 positions, 16 heads of 64: 40 us, 2.1 TB/s; one of 8,192, 32 heads of
// 128: 0.13 ms) it is a workgroup's chain per chunk - loads, LDS, four dependent products, two barriers (four with
// slices of 128) - at the workgroups that fit a CU: two, by registers and LDS, three where states have 64 rows. The
// matrix pipes are busy for a third of the cycles. fp32 waits in the same way, for the fp32 MFMAs (1/16 of the bf16 rate)
// of the waves with most score tiles and at one or two workgroups a CU: 64 sequences of 256 positions, 4 heads of
// 64, forward and backward 87 us, 43 TFLOP/s of the recurrence's own operations, the pipes busy for 36 and 49%.
#include <hip/hip_runtime.h>

#include "zo_layers.hpp"

namespace zo {
namespace {

constexpr int kChunk = 64;    // positions
constexpr int kThreads = 256;
constexpr int kXcds = 8;
constexpr int kParts = 3;     // bf16 parts of the decayed z in the state's sum

typedef float f4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));

// Positions of a pass are split into `segments` of `length` (a multiple of kChunk).
struct Plan {
  int segments;
  int length;
  int64_t groups;            // (sequence, key/value head, segment)
  int members;               // workgroups of a group: (pass, head, slice)
  float* states[kLinPasses]; // [B][kv_heads][segments - 1][dx][dz]
};

// The contraction block of one operand register set (4 VGPRs a lane).
template <typename T>
struct Op;
template <>
struct Op<uint16_t> {
  static constexpr int KB = 32;
  typedef b8 Frag;
  // c[e] += a[e] b
  template <int N>
  static __device__ __forceinline__ void mma(const Frag (&a)[N], Frag b, f4* c) {
#pragma unroll
    for (int e = 0; e < N; ++e) c[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[e], b, c[e], 0, 0, 0);
  }
  // contraction along a row: 8 values from index 8 g
  static __device__ __forceinline__ Frag along(const uint16_t* row, int g) { return *(const Frag*)(row + 8 * g); }
  // contraction over rows: rows 4 g .. 4 g + 3 of each of two tiles of 16 rows, column l % 16
  static constexpr int TILES = 2;
  static __device__ __forceinline__ Frag down(const uint16_t* tile0, const uint16_t* tile1, int stride, int g, int m) {
    typedef __attribute__((address_space(3))) s4 Lds;
    const int at = (4 * g + (m >> 2)) * stride + 4 * (m & 3);
    const s4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(tile0 + at));
    const s4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(tile1 + at));
    return __builtin_bit_cast(Frag, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};
template <>
struct Op<float> {
  static constexpr int KB = 16;
  typedef f4 Frag;
  // (the N accumulators in turn, so that no product waits for the one before it: 16 sequences of 300 positions, 16
  // heads of 128, backward 233 -> 222 us)
  template <int N>
  static __device__ __forceinline__ void mma(const Frag (&a)[N], Frag b, f4* c) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int e = 0; e < N; ++e) c[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e][s], b[s], c[e], 0, 0, 0);
  }
  static __device__ __forceinline__ Frag along(const float* row, int g) { return *(const Frag*)(row + 4 * g); }
  static constexpr int TILES = 1;
  static __device__ __forceinline__ Frag down(const float* tile, const float*, int stride, int g, int m) {
    Frag f;
#pragma unroll
    for (int s = 0; s < 4; ++s) f[s] = tile[(4 * g + s) * stride + m];
    return f;
  }
};

// The first d (fewer than 16 bytes hold) values of a row, then zeros.
template <typename T>
__device__ __forceinline__ u4 load_few(const T* p, int d) {
  u4 v = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < (int)(16 / sizeof(T)); ++e)
    if (e < d) {
      if constexpr (sizeof(T) == 2) v[e / 2] |= (uint32_t)p[e] << (16 * (e & 1));
      else v[e] = __float_as_uint(p[e]);
    }
  return v;
}
// Gathers, over words of values, the sign bit of each whose exponent is all ones.
template <typename T>
__device__ __forceinline__ uint32_t not_finite(u4 v) {
  uint32_t bad = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    bad |= sizeof(T) == 2 ? (v[e] & 0x7fff7fffu) + 0x00800080u : (v[e] & 0x7fffffffu) + 0x00800000u;
  return bad & (sizeof(T) == 2 ? 0x80008000u : 0x80000000u);
}
template <typename T>
__device__ __forceinline__ typename Op<T>::Frag only_finite(typename Op<T>::Frag f) {
  u4 v = __builtin_bit_cast(u4, f);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (sizeof(T) == 2) {
      if ((v[e] & 0x7f80u) == 0x7f80u) v[e] &= 0xffff0000u;
      if ((v[e] & 0x7f800000u) == 0x7f800000u) v[e] &= 0x0000ffffu;
    } else {
      if ((v[e] & 0x7f800000u) == 0x7f800000u) v[e] = 0;
    }
  }
  return __builtin_bit_cast(typename Op<T>::Frag, v);
}

// Four values as bf16, and what that leaves out of each.
__device__ __forceinline__ uint2 halves(const f4& x, float* rest) {
  const uint2 p{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
  rest[0] = x[0] - __uint_as_float(p.x << 16);
  rest[1] = x[1] - __uint_as_float(p.x & 0xffff0000u);
  rest[2] = x[2] - __uint_as_float(p.y << 16);
  rest[3] = x[3] - __uint_as_float(p.y & 0xffff0000u);
  return p;
}

// A value that all lanes share, in a scalar register.
__device__ __forceinline__ float scalar(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(x)));
}

// gamma^n; gamma^0 is 1 whatever gamma.
__device__ __forceinline__ float decay(float lg, int n) { return n == 0 ? 1.0f : exp2f(lg * (float)n); }

// The positions of a chunk in memory: position i (counted in the pass's direction) at
// base + row(i), an offset of 32 bits, so that a chunk's loads share one scalar base.
template <typename T>
struct Rows {
  const T* first;   // position 0
  int64_t stride;   // in the pass's direction
  uint32_t step;    // |stride|
  bool down;
  __device__ __forceinline__ Rows(const T* p, int64_t s, bool reverse, int origin)
      : first(p + origin * s), stride(reverse ? -s : s), step((uint32_t)(s < 0 ? -s : s)), down((s < 0) != reverse) {}
  __device__ __forceinline__ const T* base(int start) const {
    return first + (start + (down ? kChunk - 1 : 0)) * stride;
  }
  __device__ __forceinline__ uint32_t row(int i) const { return (uint32_t)(down ? kChunk - 1 - i : i) * step; }
};

// A tile of 64 positions by COLS columns (the first d of which exist) on its way from memory
// to LDS, 16 bytes per thread and step. Rows before the first position (`lead` of them)
// repeat it (no branch around a load: the loads stay in flight together) and are put down as
// zeros; columns past d are never put down (they are cleared beforehand).
template <typename T, int COLS, bool even>
struct Staged {
  static constexpr int EL = 16 / sizeof(T), PER_ROW = COLS / EL, STEP = kThreads / PER_ROW;
  // rows lie 8 banks (bf16: the transposing loads' width) or 4 (fp32) past a multiple of all 64
  static constexpr int N = kChunk / STEP, STRIDE = COLS + (sizeof(T) == 2 ? 16 : 4);
  u4 v[N];
  uint32_t at[N];
  __device__ __forceinline__ void aim(const Rows<T>& m, int lead, int d) {
    const int q = (int)threadIdx.x % PER_ROW * EL, r = (int)threadIdx.x / PER_ROW;
#pragma unroll
    for (int i = 0; i < N; ++i) at[i] = m.row(max(r + STEP * i, lead)) + max(min(q, d - EL), 0);
  }
  __device__ __forceinline__ void fetch(const T* base, int d) {
    if (even || d >= EL) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = load16(base + at[i]);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = load_few(base + at[i], d);
    }
  }
  __device__ __forceinline__ void put(T* tile, int lead, int d) {
    const int q = (int)threadIdx.x % PER_ROW * EL, r = (int)threadIdx.x / PER_ROW;
    if (!even && d >= EL) {
      const int n = max(q - (d - EL), 0);
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = drop<T>(v[i], n);
    }
    if (lead)
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (r + STEP * i < lead) v[i] = u4{0, 0, 0, 0};
    if (q < d)
#pragma unroll
      for (int i = 0; i < N; ++i) *(u4*)(tile + (r + STEP * i) * STRIDE + q) = v[i];
  }
  __device__ __forceinline__ static void clear(T* tile) {
    for (int i = threadIdx.x; i < kChunk * STRIDE / EL; i += kThreads) *(u4*)(tile + i * EL) = u4{0, 0, 0, 0};
  }
  __device__ __forceinline__ bool any_not_finite() const {
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) bad |= not_finite<T>(v[i]);
    return bad != 0;
  }
};

// Stores a wave's 16 rows of 64 columns (d of which exist): lane l holds columns 16 j + 4 (l / 16) .. of row l % 16.
// bf16: lanes of neighbouring groups swap halves, so that each stores 16 bytes and a row 64 in one instruction.
template <typename T, bool even>
__device__ __forceinline__ void store_rows(const f4 (&acc)[4], T* row, bool exists, int d, int g) {
  if constexpr (sizeof(T) == 2 && even) {
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
      u4 v;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const auto s = __builtin_amdgcn_permlane16_swap(bf16_pair(acc[j][2 * e], acc[j][2 * e + 1]),
                                                        bf16_pair(acc[j + 1][2 * e], acc[j + 1][2 * e + 1]), false, false);
        v[e] = s[0];
        v[2 + e] = s[1];
      }
      // groups 0 and 2 now hold columns 0 .. 7 and 8 .. 15 of tile j, groups 1 and 3 of tile j + 1
      const int at = 16 * j + 16 * (g & 1) + 4 * (g & 2);
      struct __attribute__((packed, aligned(sizeof(T)))) Any { u4 v; };
      if (exists && at < d) ((Any*)(row + at))->v = v;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int at = 16 * j + 4 * g;
      if (exists && (even ? at < d : at + 4 <= d)) {
        store_run<T, 4>(row + at, (const float*)&acc[j]);
      } else if (!even && exists) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (at + e < d) row[at + e] = from_f32<T>(acc[j][e]);
      }
    }
  }
}

// Waves per SIMD: bf16 states of 64 rows leave room for three (64 sequences of 1,024 positions, 16 heads of 64, backward:
// 307 us, with two 320; of 60, whose loads take more registers, 417 and 414: two).
template <typename T, int DX, int SL, bool even, bool state_only>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 && DX == 64 && even ? 3 : (sizeof(T) == 2 ? DX < 256 : DX < 128) ? 2 : 1) void linattn_chunk_kernel(LinCall c, Plan pl) {
  typedef Op<T> O;
  typedef typename O::Frag Frag;
  typedef Staged<T, DX, even> Y;
  typedef Staged<T, SL, even> Z;
  constexpr int EL = 16 / sizeof(T), KB = O::KB;
  constexpr int YS = Y::STRIDE, ZS = Z::STRIDE;
  constexpr int NX = DX / KB, NJ = kChunk / KB;        // operand sets along a row of x, over the chunk's positions
  constexpr int MT = DX / 16, NW = SL / 64;           // tiles of 16: R's rows, a wave's of its columns (w, w + 4)
  constexpr int FP = sizeof(T) == 2 ? 2 : 1;          // parts of P, and of R where x reads it
  constexpr int RC = FP == 2 ? 64 : SL;               // columns of R that x reads at a time
  __shared__ __align__(16) T ys[kChunk * YS];
  __shared__ __align__(16) T zs[kChunk * ZS];
  __shared__ __align__(16) T rs[state_only ? 1 : FP * RC * YS];  // R^T where x reads it
  __shared__ int bad[2];

  // groups go round the XCDs (workgroup i runs on XCD i % 8), the members of one stay together
  const int64_t id = block_id(), turn = id / kXcds;
  const int64_t group = turn / pl.members * kXcds + id % kXcds;
  if (group >= pl.groups) return;
  int member = (int)(turn % pl.members), pass = 0;
  for (;; ++pass) {
    const int n = (state_only ? 1 : c.pass[pass].heads) * ((c.pass[pass].dz + SL - 1) / SL);
    if (member < n) break;
    member -= n;
  }
  const LinPass& a = c.pass[pass];
  const int slices = (a.dz + SL - 1) / SL;
  const int col = member % slices * SL;
  const int seg = (int)(group % (pl.segments - (state_only ? 1 : 0)));
  const int64_t bh = group / (pl.segments - (state_only ? 1 : 0));
  const int b = (int)(bh / c.kv_heads), kvh = (int)(bh % c.kv_heads);
  const int h = kvh * a.heads + member / slices;

  const int n = c.lengths ? min(max(c.lengths[b], 0), c.T) : c.T;
  const int r0 = seg * pl.length, r1 = min(n, r0 + pl.length);  // the segment's positions
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = lane >> 4, m = lane & 15;

  const float lg = c.log_decay[kvh] * 1.44269504088896340736f;
  const int off = a.reverse ? 0 : 1;

  T* out = (T*)a.out + b * a.ob + (int64_t)h * a.oh;
  if constexpr (state_only) {
    if (r0 + pl.length > n) return;  // no position follows it
  } else {
    const int end = min(c.T, r0 + pl.length), width = min(SL, a.dz - col);
    for (int t = max(r0, n) + w; t < end; t += kThreads / 64)
      for (int d = lane; d < width; d += 64) out[t * a.ot + col + d] = from_f32<T>(0.0f);
    if (r0 >= n && seg > 0) return;
  }

  // R: rows 16 i + 4 g + r, columns col + 64 u + 16 w + m
  f4 R[NW][MT];
  const int rz = col + 16 * w + m;
  const float* from = nullptr;
  {
    bool turned = false;
    if (seg == 0) {
      if (a.init) from = a.init + bh * a.dx * a.dz;
      turned = a.state_t;
    } else if (!state_only) {
      from = pl.states[pass] + (bh * (pl.segments - 1) + seg - 1) * a.dx * a.dz;
    }
#pragma unroll
    for (int u = 0; u < NW; ++u)
#pragma unroll
      for (int i = 0; i < MT; ++i) R[u][i] = f4{0, 0, 0, 0};
    if (from) {
      const int sx = turned ? 1 : a.dz, sz = turned ? a.dx : 1;
#pragma unroll
      for (int u = 0; u < NW; ++u) {
        const int z = rz + 64 * u;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) R[u][i][r] = from[min(16 * i + 4 * g + r, a.dx - 1) * sx + min(z, a.dz - 1) * sz];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (16 * i + 4 * g + r >= a.dx || z >= a.dz) R[u][i][r] = 0.0f;
      }
    }
  }

  // Factors of the scores and of z. The first chunk may begin before the segment, by
  // `lead` rows of zeros, so that all others are whole and these never change.
  const int row = 16 * w + m;
  const int lead0 = (kChunk - (r1 - r0) % kChunk) % kChunk;
  // Scores go by tiles of 16 positions backwards from the wave's own: tile t holds positions 16 (w - t) .., all of
  // them before the rows for t >= 1 (none at all for t > w). Each factor is a product of two powers, both of
  // exponents >= 0 (no overflow however strong the decay), one by lane and one by tile.
  float own_f[4], far_f[4], pos_f[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int apart = m - 4 * g - r;
    own_f[r] = state_only ? 0.0f : a.score * decay(lg, max(apart, 0));
    far_f[r] = state_only ? 0.0f : a.score * decay(lg, apart + 16);
    pos_f[r] = a.upd * decay(lg, 16 - off - 4 * g - r);
  }
  const float tile_f[4] = {1.0f, scalar(decay(lg, 16)), scalar(decay(lg, 32)), scalar(decay(lg, 48))};
  // of the carried state: what reaches a row, and what is left after the chunk
  float xf = a.carry * decay(lg, max(row - lead0, 0) + off), rf = scalar(decay(lg, kChunk - lead0));

  // the next step's y and z, the next chunk's x (whose values past dx meet zeros of y and R)
  const int origin = a.reverse ? n - 1 : 0, zd = min(SL, a.dz - col);
  const Rows<T> yr((const T*)a.y.p + b * a.y.b + (int64_t)kvh * a.sources * a.y.h, a.y.t, a.reverse, origin);
  const Rows<T> zr((const T*)a.z.p + b * a.z.b + (int64_t)kvh * a.sources * a.z.h + col, a.z.t, a.reverse, origin);
  const Rows<T> xr((const T*)a.x.p + b * a.x.b + (int64_t)h * a.x.h, a.x.t, a.reverse, origin);
  // The loads of the next step go out once this one's tiles are in LDS, or, where the registers of two waves
  // per SIMD do not hold them beside the output, once that is stored.
  constexpr bool late = sizeof(T) == 2 && SL == 128;
  // Whether the first chunk's products with a state of zero and the last one's sum that nothing reads are left out
  // (the branches cost the kernel that is short of registers more than two of its many chunks' products).
  constexpr bool ends = !late;
  // (kept in scalar registers: loads of arguments inside the loop would wait for the LDS too)
  int64_t yh = a.y.h, zh = a.z.h, out_turn = a.reverse ? -a.ot : a.ot;
  T* outp = out + origin * a.ot + col;
  int sources = a.sources, dxn = a.dx;
  const bool fin = a.fin != nullptr;
  asm volatile("" : "+s"(yh), "+s"(zh), "+s"(out_turn), "+s"(outp), "+s"(sources), "+s"(dxn));
  Y yn;
  Z zn;
  Frag xn[NX];
  uint32_t xat = 0;
  const auto aim = [&](int lead) {
    yn.aim(yr, lead, a.dx);
    zn.aim(zr, lead, zd);
    if constexpr (!state_only) xat = xr.row(max(row, lead));
  };
  const auto fetch_x = [&](int start) {
    const T* x = xr.base(start);
    if (even || dxn >= EL) {
#pragma unroll
      for (int i = 0; i < NX; ++i)
        xn[i] = __builtin_bit_cast(Frag, load16(x + (xat + (uint32_t)min(i * KB + KB / 4 * g, dxn - EL))));
    } else {
#pragma unroll
      for (int i = 0; i < NX; ++i) xn[i] = __builtin_bit_cast(Frag, load_few(x + xat, i * KB + KB / 4 * g == 0 ? a.dx : 0));
    }
  };

  if (r0 < r1) {
    aim(lead0);
    yn.fetch(yr.base(r0 - lead0), a.dx);
    zn.fetch(zr.base(r0 - lead0), zd);
    if constexpr (!state_only) fetch_x(r0 - lead0);
  }
  if (tid < 2) bad[tid] = 0;
  if (a.dx < DX) Y::clear(ys);
  if (zd < SL) Z::clear(zs);
  __syncthreads();
  static_assert(SL == 64 || SL == 128, "one part of the output, or two (and then one source: acc holds one part)");
  f4 acc[4];
  // bf16: 64 columns of R as two parts, the second of what the first left out
  const auto put_r = [&](int u) {
    T* to = rs + (16 * w + m) * YS + 4 * g;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      float rest[4];
      const uint2 high = halves(R[u][i], rest);
      *(uint2*)(to + 16 * i) = high;
      *(uint2*)(to + 64 * YS + 16 * i) = uint2{bf16_pair(rest[0], rest[1]), bf16_pair(rest[2], rest[3])};
    }
  };
  int src = 0, turn_of = 0;
  for (int start = r0 - lead0; start < r1; turn_of ^= 1) {
    const int lead = max(r0 - start, 0);
    yn.put(ys, lead, dxn);
    zn.put(zs, lead, zd);
    if constexpr (!state_only) {
      if (zn.any_not_finite()) bad[turn_of] = 1;
      if (src == 0) {
        if constexpr (FP == 2) {
          put_r(0);
        } else {
#pragma unroll
          for (int u = 0; u < NW; ++u)
#pragma unroll
            for (int i = 0; i < MT; ++i)
              store_run<T, 4>(rs + (64 * u + 16 * w + m) * YS + 16 * i + 4 * g, (const float*)&R[u][i]);
        }
      }
    }
    __syncthreads();
    const bool flagged = !state_only && bad[turn_of];
    if (tid == 0) bad[turn_of ^ 1] = 0;
    // the loads of the next step, or once more this one's after the last
    const bool last_src = src == sources - 1;
    const int next = last_src && start + kChunk < r1 ? start + kChunk : start, next_src = last_src ? 0 : src + 1;
    if (next > start && lead) {
      int none = 0;
      asm volatile("" : "+v"(none));  // (worked out here, not held in registers from before the loop)
      aim(none);
    }
    if constexpr (!late) {
      yn.fetch(yr.base(next) + next_src * yh, dxn);
      zn.fetch(zr.base(next) + next_src * zh, zd);
    }
    if constexpr (!state_only) {
      if constexpr (!even) {
        if (a.dx >= EL)
#pragma unroll
          for (int i = 0; i < NX; ++i)
            if ((i + 1) * KB > a.dx - EL)
              xn[i] = __builtin_bit_cast(Frag, drop<T>(__builtin_bit_cast(u4, xn[i]), min(max(i * KB + KB / 4 * g - (a.dx - EL), 0), EL - 1)));
      }
      f4 P[4];
      // (bf16: all four tiles, also those past the wave's rows: there the wave with most of them is what the others
      // wait for. fp32, whose products take 16 times as long: two or four.)
      constexpr bool all = sizeof(T) == 2;
      const auto y_of = [&](int t, int i) { return O::along(ys + 16 * ((w - t) & 3) * YS + m * YS + i * KB, g); };
#pragma unroll
      for (int t = 0; t < 4; ++t) P[t] = f4{0, 0, 0, 0};
      if constexpr (all) {
#pragma unroll
        for (int i = 0; i < NX; ++i) O::mma({y_of(0, i), y_of(1, i), y_of(2, i), y_of(3, i)}, xn[i], P);
      } else {
#pragma unroll
        for (int i = 0; i < NX; ++i) O::mma({y_of(0, i), y_of(1, i)}, xn[i], P);
        if (w >= 2)
#pragma unroll
          for (int i = 0; i < NX; ++i) O::mma({y_of(2, i), y_of(3, i)}, xn[i], P + 2);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) P[0][r] = 4 * g + r <= m ? P[0][r] * own_f[r] : 0.0f;
#pragma unroll
      for (int t = 1; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) P[t][r] = t <= w ? P[t][r] * far_f[r] * tile_f[t - 1] : 0.0f;
      Frag pb[FP][NJ];
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        if constexpr (FP == 2) {
          float rest[8];
          const uint2 a = halves(P[2 * j], rest), b = halves(P[2 * j + 1], rest + 4);
          pb[0][j] = __builtin_bit_cast(Frag, u4{a.x, a.y, b.x, b.y});
          pb[1][j] = __builtin_bit_cast(Frag, u4{bf16_pair(rest[0], rest[1]), bf16_pair(rest[2], rest[3]),
                                                 bf16_pair(rest[4], rest[5]), bf16_pair(rest[6], rest[7])});
        } else {
          pb[0][j] = P[j];
        }
      }
      // the output, 64 columns at a time
#pragma unroll
      for (int part = 0; part < SL / 64; ++part) {
        if (FP == 2 && part > 0) {  // (slices of 128 have one source)
          __syncthreads();
          put_r(part);
          __syncthreads();
        }
        if (src == 0) {
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[j] = f4{0, 0, 0, 0};
        }
        if (src == 0 && (!ends || start > r0 - lead0 || from)) {
#pragma unroll
          for (int i = 0; i < NX; ++i)
#pragma unroll
            for (int q = 0; q < FP; ++q) {
              const auto r_of = [&](int j) {
                return O::along(rs + ((FP == 2 ? 64 * q : 64 * part) + 16 * j + m) * YS + i * KB, g);
              };
              O::mma({r_of(0), r_of(1), r_of(2), r_of(3)}, xn[i], acc);
            }
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[j] *= xf;
        }
        // tile t of the scores meets the rows of z of its positions
        const auto z_of = [&](int k, int j) {
          const auto tile = [&](int t) { return zs + 16 * ((w - t) & 3) * ZS + 64 * part + 16 * j; };
          return O::down(tile(k * O::TILES), tile(k * O::TILES + 1), ZS, g, m);
        };
        if (!flagged) {
#pragma unroll
          for (int k = 0; k < NJ; ++k)
            if (all || k < 2 || w >= 2) {
              const Frag z[4] = {z_of(k, 0), z_of(k, 1), z_of(k, 2), z_of(k, 3)};
#pragma unroll
              for (int q = 0; q < FP; ++q) O::mma(z, pb[q][k], acc);
            }
        } else {
#pragma unroll
          for (int k = 0; k < NJ; ++k) {
            const Frag z[4] = {only_finite<T>(z_of(k, 0)), only_finite<T>(z_of(k, 1)), only_finite<T>(z_of(k, 2)),
                               only_finite<T>(z_of(k, 3))};
#pragma unroll
            for (int q = 0; q < FP; ++q) O::mma(z, pb[q][k], acc);
          }
          // the products of z that are not finite, for the rows they reach
          constexpr int WORDS = 4 * NJ;
          int zat = 64 * part + 4 * g;
          asm volatile("" : "+v"(zat));  // (keeps this path's addresses out of the others' registers)
#pragma unroll 1
          for (int at = 0; at < kChunk; ++at) {
            // P of position at: in lanes of group (at / 4) % 4, values 4 t + at % 4 of the operands
            const int t = w - (at >> 4), value = (t & 3) * 4 + (at & 3), want = sizeof(T) == 2 ? value >> 1 : value;
            float p = 0;
#pragma unroll
            for (int q = 0; q < FP; ++q) {
              uint32_t word = 0;
#pragma unroll
              for (int e = 0; e < WORDS; ++e) word = e == want ? __builtin_bit_cast(u4, pb[q][e >> 2])[e & 3] : word;
              word = (uint32_t)__shfl((int)word, m + 16 * ((at >> 2) & 3), 64);
              p += __uint_as_float(sizeof(T) == 4 ? word : at & 1 ? word & 0xffff0000u : word << 16);
            }
#pragma unroll
            for (int d = 0; d < 16; ++d) {
              const float v = to_f32(zs[at * ZS + zat + 16 * (d >> 2) + (d & 3)]);
              if (at <= row && !(fabsf(v) < __builtin_inff())) acc[d >> 2][d & 3] += p * v;
            }
          }
        }
        if (last_src)
          store_rows<T, even>(acc, outp + (start + row) * out_turn + 64 * part, row >= lead, zd - 64 * part, g);
      }
      fetch_x(next);
    }
    if constexpr (late) {
      yn.fetch(yr.base(next) + next_src * yh, dxn);
      zn.fetch(zr.base(next) + next_src * zh, zd);
    }
    // the state after the chunk
    const bool read = state_only || !ends || start + kChunk < r1 || fin;
    if (read && src == 0)
#pragma unroll
      for (int u = 0; u < NW; ++u)
#pragma unroll
        for (int i = 0; i < MT; ++i) R[u][i] *= rf;
    if (read)
#pragma unroll
    for (int k = 0; k < NJ; ++k) {
      // gamma^(..) z; in bf16 parts, the next one of what the last left out
      constexpr int PARTS = sizeof(T) == 2 ? kParts : 1;
      Frag part[NW][PARTS];
#pragma unroll
      for (int u = 0; u < NW; ++u) {
        const T* zt = zs + k * KB * ZS + 64 * u + 16 * w;
        const Frag own = O::down(zt, zt + 16 * ZS, ZS, g, m);
        if constexpr (sizeof(T) == 2) {
          const u4 raw = __builtin_bit_cast(u4, own);
          float rest[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float f = tile_f[3 - 2 * k - (e >> 1)];
            rest[2 * e] = __uint_as_float(raw[e] << 16) * (pos_f[2 * e & 3] * f);
            rest[2 * e + 1] = __uint_as_float(raw[e] & 0xffff0000u) * (pos_f[(2 * e + 1) & 3] * f);
          }
#pragma unroll
          for (int q = 0; q < PARTS; ++q) {
            u4 p;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              p[e] = bf16_pair(rest[2 * e], rest[2 * e + 1]);
              rest[2 * e] -= __uint_as_float(p[e] << 16);
              rest[2 * e + 1] -= __uint_as_float(p[e] & 0xffff0000u);
            }
            part[u][q] = __builtin_bit_cast(Frag, p);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) part[u][0][e] = own[e] * (pos_f[e] * tile_f[3 - k]);
        }
      }
      // four tiles of rows in turn: a product's accumulator is four products old
#pragma unroll
      for (int i = 0; i < MT; i += 4) {
        Frag y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const T* yt = ys + k * KB * YS + 16 * (i + e);
          y[e] = O::down(yt, yt + 16 * YS, YS, g, m);
        }
#pragma unroll
        for (int q = 0; q < PARTS; ++q)
#pragma unroll
          for (int u = 0; u < NW; ++u) O::mma(y, part[u][q], &R[u][i]);
      }
    }
    __syncthreads();
    src = next_src;
    if (last_src) {
      if (lead) {
        float l = lg;
        asm volatile("" : "+v"(l));
        xf = a.carry * decay(l, row + off);
        rf = scalar(decay(l, kChunk));
      }
      start += kChunk;
    }
  }

  float* to = nullptr;
  bool turned = false;
  if constexpr (state_only) {
    to = pl.states[pass] + (bh * (pl.segments - 1) + seg) * a.dx * a.dz;
  } else if (a.fin && r1 == n && h == kvh * a.heads) {  // the segment of the last position (the first one of none)
    to = a.fin + bh * a.dx * a.dz;
    turned = a.state_t;
  }
  if (to)
#pragma unroll
    for (int u = 0; u < NW; ++u)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int x = 16 * i + 4 * g + r, z = rz + 64 * u;
          if (x < a.dx && z < a.dz) to[turned ? z * a.dx + x : x * a.dz + z] = R[u][i][r];
        }
}

// Few positions: one after another, the state in registers (thread t: columns 4 (t % 16) .., rows t / 16 + 16 i of 64
// columns), everything in fp32. A chunk of 64 would be mostly zeros, in a workgroup that takes a third of a CU or
// all of it. All positions are read at once, and their outputs' sums joined at once.
// One to four positions, 256 sequences of 32 heads of 128: without states 0.04 to 0.09 ms (bf16) against 0.15 in
// chunks, fp32 0.04 to 0.10 against 0.34; with states 0.21 to 0.24 against 0.40, fp32 0.21 to 0.26 against 0.90.
// Eight take 0.17 against 0.15 (bf16; fp32 0.18 against 0.34).
constexpr int kFew = 4;         // positions
constexpr int kFewPairs = 16;   // positions times y/z heads
template <typename T, int ROWS, int PAIRS>
__global__ __launch_bounds__(kThreads) void linattn_few_kernel(LinCall c) {
  constexpr int GROUPS = 16, DX = ROWS * GROUPS;
  __shared__ float xs[kFew][DX];
  __shared__ float ys[PAIRS][DX];
  __shared__ float part[kFew][4][64];
  const LinPass& a = c.pass[blockIdx.z];
  const int tid = threadIdx.x, c4 = (tid & 15) * 4, rg = tid >> 4;
  const int slices = (a.dz + 63) / 64, heads = c.kv_heads * a.heads;
  const int64_t blk = block_id(), bh = blk / slices;
  const int b = (int)(bh / heads), h = (int)(bh % heads);
  if (b >= c.B) return;
  const int col = (int)(blk % slices) * 64, kvh = h / a.heads;
  const int n = c.lengths ? min(max(c.lengths[b], 0), c.T) : c.T;
  const T* x = (const T*)a.x.p + b * a.x.b + h * a.x.h;
  const T* y = (const T*)a.y.p + b * a.y.b + (int64_t)kvh * a.sources * a.y.h;
  const T* z = (const T*)a.z.p + b * a.z.b + (int64_t)kvh * a.sources * a.z.h + col + c4;
  T* out = (T*)a.out + b * a.ob + h * a.oh + col;
  const int left = a.dz - col - c4;  // columns of this thread that exist: 4 or fewer
  const int64_t state_at = ((int64_t)b * c.kv_heads + kvh) * a.dx * a.dz;
  const int sx = a.state_t ? 1 : a.dz, sz = a.state_t ? a.dx : 1;
  float s[ROWS][4];
#pragma unroll
  for (int i = 0; i < ROWS; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) s[i][e] = 0.0f;
  // A state handed from call to call would drift by gamma's rounding: one of its n decays, as it is read (forward) or
  // written (backward), takes gamma's lower part for all of them (at every position that takes a tenth more time).
  float gamma = decay(c.log_decay[kvh] * 1.44269504088896340736f, 1), lower = 0.0f;
  if (a.init) {
    const Gamma both(c.log_decay[kvh]);
    gamma = both.high;
    lower = (float)n * both.low;
  }
  const auto aged = [&](float v, bool now) { return now ? fmaf(gamma, v, lower * finite(v)) : v; };
  const bool before = n > 0 && !a.reverse, after = n > 0 && a.reverse;
  const bool whole = left >= 4 && !a.state_t;  // a thread's four values lie together
  if (a.init && whole) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) load_run<float, 4>(a.init + state_at + min(rg + GROUPS * i, a.dx - 1) * sx + col + c4, s[i]);
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[i][e] = rg + GROUPS * i < a.dx ? aged(s[i][e], before) : 0.0f;
  } else if (a.init) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = rg + GROUPS * i;
        const float v = a.init[state_at + min(r, a.dx - 1) * sx + min(col + c4 + e, a.dz - 1) * sz];
        s[i][e] = r < a.dx && e < left ? aged(v, before) : 0.0f;
      }
  }
  for (int at = tid; at < n * DX; at += kThreads) {
    const int u = at / DX, d = at % DX, t = a.reverse ? n - 1 - u : u;
    xs[u][d] = d < a.dx ? to_f32(x[t * a.x.t + d]) : 0.0f;
  }
  for (int at = tid; at < n * a.sources * DX; at += kThreads) {
    const int p = at / DX, d = at % DX, u = p / a.sources, t = a.reverse ? n - 1 - u : u;
    ys[p][d] = d < a.dx ? to_f32(y[t * a.y.t + (p % a.sources) * a.y.h + d]) : 0.0f;
  }
  __syncthreads();
  for (int u = 0; u < n; ++u) {
    const int64_t t = a.reverse ? n - 1 - u : u;
    if (before && u > 0)
#pragma unroll
      for (int i = 0; i < ROWS; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][e] *= gamma;
    for (int q = 0; q < a.sources; ++q) {
      float zv[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) zv[e] = e < left ? a.upd * to_f32(z[t * a.z.t + q * a.z.h + e]) : 0.0f;
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        const float yv = ys[u * a.sources + q][rg + GROUPS * i];
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][e] = fmaf(yv, zv[e], s[i][e]);
      }
    }
    float acc[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const float xv = xs[u][rg + GROUPS * i];
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = fmaf(xv, s[i][e], acc[e]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      acc[e] += __shfl_xor(acc[e], 16, 64);
      acc[e] += __shfl_xor(acc[e], 32, 64);
      if ((tid & 63) < 16) part[u][tid >> 6][c4 + e] = acc[e];
    }
    if (after && u < n - 1)
#pragma unroll
      for (int i = 0; i < ROWS; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][e] *= gamma;
  }
  __syncthreads();
  for (int at = tid; at < c.T * 64; at += kThreads) {
    const int u = at / 64, d = at % 64;
    if (col + d >= a.dz) continue;
    const int64_t t = u >= n ? u : a.reverse ? n - 1 - u : u;  // positions past the length in their own order
    out[t * a.ot + d] = from_f32<T>(
        u < n ? a.carry * ((part[u][0][d] + part[u][1][d]) + (part[u][2][d] + part[u][3][d])) : 0.0f);
  }
  if (!a.fin || h != kvh * a.heads) return;
#pragma unroll
  for (int i = 0; i < ROWS; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) s[i][e] = aged(s[i][e], after);
  if (whole) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
      if (rg + GROUPS * i < a.dx) store_run<float, 4>(a.fin + state_at + (rg + GROUPS * i) * sx + col + c4, s[i]);
  } else {
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = rg + GROUPS * i;
        if (r < a.dx && e < left) a.fin[state_at + r * sx + (col + c4 + e) * sz] = s[i][e];
      }
  }
}

template <typename T, int PAIRS>
hipError_t launch_few(const LinCall& c, int dx, hipStream_t st) {
  int64_t blocks = 0;
  for (int i = 0; i < c.npasses; ++i)
    blocks = std::max(blocks, (int64_t)c.B * c.kv_heads * c.pass[i].heads * ((c.pass[i].dz + 63) / 64));
  dim3 grid = wide_grid(blocks);
  grid.z = c.npasses;
  if (dx <= 64) linattn_few_kernel<T, 4, PAIRS><<<grid, kThreads, 0, st>>>(c);
  else if (dx <= 128) linattn_few_kernel<T, 8, PAIRS><<<grid, kThreads, 0, st>>>(c);
  else linattn_few_kernel<T, 16, PAIRS><<<grid, kThreads, 0, st>>>(c);
  return hipGetLastError();
}

// Adds up the segments' states: state_s = gamma^length state_(s-1) + its own sum.
__global__ __launch_bounds__(kThreads) void linattn_scan_kernel(LinCall c, Plan pl) {
  const int pass = blockIdx.z;
  const int per = c.pass[pass].dx * c.pass[pass].dz;
  const int64_t blk = block_id();
  const int parts = (per + kThreads - 1) / kThreads;
  const int64_t bh = blk / parts;
  if (bh >= (int64_t)c.B * c.kv_heads) return;
  const int e = (int)(blk % parts) * kThreads + threadIdx.x;
  if (e >= per) return;
  const int b = (int)(bh / c.kv_heads);
  const int n = c.lengths ? min(max(c.lengths[b], 0), c.T) : c.T;
  const int whole = min(n / pl.length, pl.segments - 1);  // segments whose sums exist
  const float gamma = decay(c.log_decay[bh % c.kv_heads] * 1.44269504088896340736f, pl.length);
  float* p = pl.states[pass] + bh * (pl.segments - 1) * per + e;
  // (eight loads in flight at a time)
  float s = 0;
  for (int i = 0; i < whole; i += 8) {
    float u[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) u[k] = p[(int64_t)min(i + k, whole - 1) * per];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (i + k < whole) {
        s = i + k == 0 ? u[k] : fmaf(gamma, s, u[k]);
        p[(int64_t)(i + k) * per] = s;
      }
  }
}

// Segments of a call: enough workgroups for two on every CU, none shorter than four chunks; one where 256 workgroups
// are there already (the states' pass over y and z costs more than the shorter chain saves: 512 workgroups, bf16, 32
// sequences of 777, 16 heads on 4 states of 64: 49 us, in two segments 57; of 2,048, 16 heads of 64: 130 and 170).
void split(int64_t workgroups, int T, int* segments, int* length) {
  int64_t s = workgroups >= 256 || workgroups == 0 ? 1 : (512 + workgroups - 1) / workgroups;
  const int64_t most = T / (4 * kChunk);
  if (s > most) s = most;
  if (s < 1) s = 1;
  *length = (int)(((T + s - 1) / s + kChunk - 1) / kChunk * kChunk);
  if (*length == 0) *length = kChunk;
  *segments = T > 0 ? (T + *length - 1) / *length : 1;
}

template <typename T, int DX, int SL, bool even>
hipError_t launch_chunks(const LinCall& c, Plan pl, hipStream_t st) {
  const int64_t states = (int64_t)c.B * c.kv_heads;
  const auto grid = [&](int64_t groups, int members) {
    return wide_grid((groups + kXcds - 1) / kXcds * kXcds * members);
  };
  int slices = 0, members = 0, most = 0;
  for (int i = 0; i < c.npasses; ++i) {
    const LinPass& p = c.pass[i];
    slices += (p.dz + SL - 1) / SL;
    members += p.heads * ((p.dz + SL - 1) / SL);
    most = std::max(most, p.dx * p.dz);
  }
  if constexpr (SL == 64) {  // (slices of 128 come with 256 workgroups and more, and those in one segment)
    if (pl.segments > 1) {
      pl.groups = states * (pl.segments - 1);
      pl.members = slices;
      linattn_chunk_kernel<T, DX, SL, even, true><<<grid(pl.groups, slices), kThreads, 0, st>>>(c, pl);
      hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      if (pl.segments > 2) {
        dim3 g = wide_grid(states * ((most + kThreads - 1) / kThreads));
        g.z = c.npasses;
        linattn_scan_kernel<<<g, kThreads, 0, st>>>(c, pl);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
      }
    }
  }
  pl.groups = states * pl.segments;
  pl.members = members;
  linattn_chunk_kernel<T, DX, SL, even, false><<<grid(pl.groups, members), kThreads, 0, st>>>(c, pl);
  return hipGetLastError();
}

template <typename T, bool even>
hipError_t launch(const LinCall& c, const Plan& pl, int dx, int slice, hipStream_t st) {
  if (dx <= 64) return launch_chunks<T, 64, 64, even>(c, pl, st);
  if (dx > 128) return launch_chunks<T, 256, 64, even>(c, pl, st);
  return slice == 128 ? launch_chunks<T, 128, 128, even>(c, pl, st) : launch_chunks<T, 128, 64, even>(c, pl, st);
}

// Columns of z per workgroup: 128 where states have more than 64 rows and columns and no more
// than 128 rows (x and y are then read once, and the scores formed once; 16 sequences of 1,024 positions, 32 heads
// of 128, forward and backward: 0.58 ms against 0.62), 64 otherwise, where several query heads
// add to one output, and where the states are too few to give every CU one (half the workgroups would be left).
int slice_of(int64_t states, int dk, int dv, int share, bool backward) {
  if ((backward ? states : states * share) < 256 || (backward && share > 1)) return 64;
  const int dx = backward ? std::max(dk, dv) : dk, dz = backward ? std::min(dk, dv) : dv;
  return dx > 64 && dx <= 128 && dz > 64 ? 128 : 64;
}

void plan_segments(int B, int kv_heads, int share, int dk, int dv, int T, bool backward, Plan* pl) {
  const int sl = slice_of((int64_t)B * kv_heads, dk, dv, share, backward), nk = (dk + sl - 1) / sl, nv = (dv + sl - 1) / sl;
  const int64_t per_state = backward ? (int64_t)share * nk + nk + nv : (int64_t)share * nv;
  split((int64_t)B * kv_heads * per_state, T, &pl->segments, &pl->length);
}

}  // namespace

size_t linattn_workspace(const zo_linattn& s, bool backward) {
  Plan pl{};
  plan_segments(s.batch, s.kv_heads, s.q_heads / s.kv_heads, s.key_dim, s.value_dim, s.length, backward, &pl);
  return (size_t)(backward ? 3 : 1) * s.batch * s.kv_heads * (pl.segments - 1) * s.key_dim * s.value_dim *
         sizeof(float);
}

hipError_t launch_linattn(const LinCall& c, hipStream_t s) {
  if (c.B == 0) return hipSuccess;
  const LinPass& p = c.pass[0];
  const bool backward = c.npasses > 1;
  Plan pl{};
  const int dk = backward ? p.dz : p.dx, dv = backward ? p.dx : p.dz, sl = slice_of((int64_t)c.B * c.kv_heads, dk, dv, c.share, backward);
  plan_segments(c.B, c.kv_heads, c.share, dk, dv, c.T, backward, &pl);
  bool even = true;
  int64_t pairs = 0;
  int dx = 0;
  for (int i = 0; i < c.npasses; ++i) {
    pl.states[i] = (float*)c.work + (int64_t)i * c.B * c.kv_heads * (pl.segments - 1) * p.dx * p.dz;
    dx = std::max(dx, c.pass[i].dx);
    pairs = std::max(pairs, (int64_t)c.T * c.pass[i].sources);
    const int el = c.dtype == ZO_WBF16 ? 8 : 4;
    even &= c.pass[i].dx % el == 0 && c.pass[i].dz % el == 0;
  }
  const bool few = c.T <= kFew && pairs <= kFewPairs;
  if (few && pairs <= kFew) return c.dtype == ZO_WBF16 ? launch_few<uint16_t, kFew>(c, dx, s) : launch_few<float, kFew>(c, dx, s);
  if (few)
    return c.dtype == ZO_WBF16 ? launch_few<uint16_t, kFewPairs>(c, dx, s) : launch_few<float, kFewPairs>(c, dx, s);
  if (c.dtype == ZO_WBF16)
    return even ? launch<uint16_t, true>(c, pl, dx, sl, s) : launch<uint16_t, false>(c, pl, dx, sl, s);
  return even ? launch<float, true>(c, pl, dx, sl, s) : launch<float, false>(c, pl, dx, sl, s);
}

}  // namespace zo
