// C ABI entry points of the layers (zo_layers.h): argument validation on the
// host, then kernel launches on the caller's stream. Nothing here allocates
// device memory.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <initializer_list>
#include <utility>

#include "zo_error.hpp"
#include "zo_layers.hpp"
#include "zo_profile.hpp"

namespace {

using zo::aligned16;
using zo::device_status;
using zo::fail;
using zo::ok;

bool is_type(int32_t t) { return t == ZO_WFP32 || t == ZO_WBF16; }
size_t type_bytes(int32_t t) { return t == ZO_WBF16 ? 2 : 4; }
bool aligned_for(const void* p, int32_t t) { return ((uintptr_t)p & (type_bytes(t) - 1)) == 0; }
bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }

int check_linattn(const zo_linattn* s) {
  if (!s) return fail(ZO_EINVAL, "shape is NULL");
  if (s->batch < 0 || s->length < 0) return fail(ZO_EINVAL, "batch and length must be >= 0");
  if (s->length > 1 << 30) return fail(ZO_ESHAPE, "length must be <= 2^30");
  if (s->q_heads < 1 || s->kv_heads < 1 || s->q_heads % s->kv_heads)
    return fail(ZO_EINVAL, "q_heads (%d) must be a positive multiple of kv_heads (%d)", s->q_heads, s->kv_heads);
  if (s->key_dim < 1 || s->value_dim < 1) return fail(ZO_EINVAL, "key_dim and value_dim must be >= 1");
  if (s->key_dim > ZO_LINATTN_MAX_DIM || s->value_dim > ZO_LINATTN_MAX_DIM)
    return fail(ZO_ESHAPE, "key_dim (%d) and value_dim (%d) must be <= %d", s->key_dim, s->value_dim,
                ZO_LINATTN_MAX_DIM);
  if (!is_type(s->dtype)) return fail(ZO_EINVAL, "unknown dtype %d", s->dtype);
  if (!std::isfinite(s->scale)) return fail(ZO_EINVAL, "scale must be finite");
  if ((int64_t)s->batch * s->q_heads > (int64_t)1 << 31) return fail(ZO_ESHAPE, "batch * q_heads too many");
  return ZO_OK;
}

// A tensor of `positions` positions that is read or written (its elements exist when `any`).
int check_heads(const zo_heads* h, const char* name, int32_t dtype, bool any, int32_t positions) {
  if (!h) return fail(ZO_EINVAL, "%s is NULL", name);
  if (any && !h->data) return fail(ZO_EINVAL, "%s has no data", name);
  if (!aligned_for(h->data, dtype)) return fail(ZO_EINVAL, "%s is not aligned to its type", name);
  // the kernels reach the 64 positions of a chunk with 32-bit offsets; one position, or none, has no distance
  if (positions < 2) return ZO_OK;
  if (h->position_stride > ZO_LINATTN_MAX_STRIDE || h->position_stride < -ZO_LINATTN_MAX_STRIDE)
    return fail(ZO_ESHAPE, "%s: position strides must stay within 2^24", name);
  return ZO_OK;
}

zo::Heads heads(const zo_heads* h, int32_t positions) {
  return zo::Heads{h->data, h->batch_stride, positions < 2 ? 0 : h->position_stride, h->head_stride};
}

int check_state(const float* s, const char* name) {
  return aligned4(s) ? ZO_OK : fail(ZO_EINVAL, "%s is not aligned to its type", name);
}

// Whether two buffers of all sequences' states share memory.
bool overlap(const zo_linattn& s, const float* a, const float* b) {
  const uint64_t bytes = (uint64_t)s.batch * s.kv_heads * s.key_dim * s.value_dim * sizeof(float);
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a && b && (x < y ? y - x : x - y) < bytes;
}

int check_workspace(const zo_linattn* s, bool backward, const void* workspace, size_t bytes) {
  const size_t need = zo::linattn_workspace(*s, backward);
  if (bytes < need) return fail(ZO_ENOMEM, "workspace of %zu bytes < %zu required", bytes, need);
  if (need && !workspace) return fail(ZO_EINVAL, "workspace is NULL");
  if (!aligned16(workspace)) return fail(ZO_EINVAL, "workspace must be 16-byte aligned");
  return ZO_OK;
}

// A tensor in memory: size[i] values stride[i] apart in each dimension; those of size 1 are left out.
struct Strided {
  static constexpr int kDims = 4;
  const char* name;
  uintptr_t data;
  int64_t element;
  int dims = 0;
  int64_t size[kDims], stride[kDims];
  bool empty = false;
  uintptr_t begin, end;  // of the memory between its first and its last value

  Strided(const char* n, const void* p, int32_t type, std::initializer_list<std::pair<int64_t, int64_t>> all)
      : name(n), data((uintptr_t)p), element((int64_t)type_bytes(type)) {
    begin = data;
    end = data + (uintptr_t)element;
    for (const auto& d : all) {
      if (d.first == 0) empty = true;
      if (d.first < 2) continue;
      size[dims] = d.first;
      stride[dims++] = d.second;
      const uintptr_t reach = (uintptr_t)(d.first - 1) * (uintptr_t)d.second * (uintptr_t)element;
      (d.second < 0 ? begin : end) += reach;
    }
    for (int i = 1; i < dims; ++i)  // by distance, the nearest first
      for (int j = i; j > 0 && std::abs(stride[j]) < std::abs(stride[j - 1]); --j) {
        std::swap(stride[j], stride[j - 1]);
        std::swap(size[j], size[j - 1]);
      }
  }
  // Every value between the first and the last belongs to it.
  bool dense() const {
    int64_t next = 1;
    for (int i = 0; i < dims; ++i) {
      if (std::abs(stride[i]) != next) return false;
      next *= size[i];
    }
    return true;
  }
  bool in_one_place() const {
    for (int i = 0; i < dims; ++i)
      if (stride[i] == 0) return true;
    return false;
  }
};

// Whether sum_i x_i stride_i = distance for some x_i within (-b.size_i, a.size_i), i < dims.
bool meet(const Strided& a, const Strided& b, int dims, int64_t distance, int* tries) {
  if (dims == 0) return distance == 0;
  if (--*tries < 0) return false;
  const int i = dims - 1;
  int64_t low = 0, high = 0;  // what the nearer dimensions can add
  for (int j = 0; j < i; ++j) {
    const int64_t x = (a.size[j] - 1) * a.stride[j], y = (b.size[j] - 1) * a.stride[j];
    low -= std::max(y, -x);
    high += std::max(x, -y);
  }
  const int64_t s = a.stride[i];
  int64_t from = (distance - high) / s - 1, to = (distance - low) / s + 1;
  if (from > to) std::swap(from, to);
  from = std::max(from - 1, -(b.size[i] - 1));
  to = std::min(to + 1, a.size[i] - 1);
  for (int64_t x = from; x <= to && *tries >= 0; ++x) {
    const int64_t left = distance - x * s;
    if (left >= low && left <= high && meet(a, b, i, left, tries)) return true;
  }
  return false;
}

// Whether two tensors are known to share a value: they begin at the same one, both fill the memory that they span, or
// their strides are the same (slices of one buffer). Others whose spans cross may lie between each other's values.
bool share(const Strided& a, const Strided& b) {
  if (a.empty || b.empty || a.begin >= b.end || b.begin >= a.end) return false;
  if (a.data == b.data || (a.dense() && b.dense())) return true;
  if (a.dims != b.dims || a.element != b.element) return false;
  for (int i = 0; i < a.dims; ++i)
    if (a.stride[i] != b.stride[i] || a.stride[i] == 0) return false;
  int tries = 1024;  // (nested strides take a few)
  return meet(a, b, a.dims, ((int64_t)(b.data - a.data)) / a.element, &tries);
}

// Outputs share nothing with inputs, with one another, or within themselves.
int check_apart(std::initializer_list<Strided> outputs, std::initializer_list<Strided> inputs) {
  for (const Strided* o = outputs.begin(); o != outputs.end(); ++o) {
    if (!o->empty && o->in_one_place()) return fail(ZO_EINVAL, "%s: values of an output lie in one place (stride 0)", o->name);
    for (const Strided& x : inputs)
      if (share(*o, x)) return fail(ZO_EINVAL, "%s and %s share memory", o->name, x.name);
    for (const Strided* p = outputs.begin(); p != o; ++p)
      if (share(*o, *p)) return fail(ZO_EINVAL, "%s and %s share memory", o->name, p->name);
  }
  return ZO_OK;
}

Strided strided(const char* name, const zo_heads* h, const zo_linattn& s, int32_t positions, bool query, bool key) {
  return Strided(name, h->data, s.dtype,
                 {{s.batch, h->batch_stride},
                  {positions, h->position_stride},
                  {query ? s.q_heads : s.kv_heads, h->head_stride},
                  {key ? s.key_dim : s.value_dim, 1}});
}

// Ranges [begin, end) of memory, to be checked for overlaps: one comparison each where they come in order (views of one
// vector, moments one after another), sorted otherwise.
class Ranges {
 public:
  explicit Ranges(int32_t n) : at_(n <= kFew ? few_ : (Range*)std::malloc(sizeof(Range) * (size_t)n)) {}
  ~Ranges() {
    if (at_ != few_) std::free(at_);
  }
  bool ready() const { return at_ != nullptr; }
  void add(uint64_t begin, uint64_t bytes) { at_[n_++] = Range{begin, begin + bytes}; }
  bool overlap() {
    if (in_order()) return false;
    std::sort(at_, at_ + n_, [](const Range& a, const Range& b) { return a.begin < b.begin; });
    return !in_order();
  }

 private:
  struct Range {
    uint64_t begin, end;
  };
  static constexpr int32_t kFew = 64;
  Range few_[kFew];
  Range* at_;
  int32_t n_ = 0;
  bool in_order() const {
    for (int32_t i = 1; i < n_; ++i)
      if (at_[i].begin < at_[i - 1].end) return false;
    return true;
  }
};

}  // namespace

extern "C" {

size_t zo_linear_attention_workspace_bytes(const zo_linattn* shape, int32_t backward) {
  if (check_linattn(shape)) return 0;
  return zo::linattn_workspace(*shape, backward != 0);
}

int zo_linear_attention(const zo_linattn* shape, const zo_heads* q, const zo_heads* k, const zo_heads* v,
                        const zo_heads* o, const float* log_decay, const int32_t* lengths,
                        const float* initial_state, float* final_state, void* workspace, size_t ws_bytes,
                        void* stream) {
  zo::PhaseRange range("zo_linear_attention");
  int st = check_linattn(shape);
  if (st) return st;
  const zo_linattn& s = *shape;
  const bool any = s.batch > 0 && s.length > 0;
  if ((st = check_heads(q, "q", s.dtype, any, s.length)) || (st = check_heads(k, "k", s.dtype, any, s.length)) ||
      (st = check_heads(v, "v", s.dtype, any, s.length)) || (st = check_heads(o, "o", s.dtype, any, s.length)) ||
      (st = check_state(log_decay, "log_decay")) || (st = check_state(initial_state, "initial_state")) ||
      (st = check_state(final_state, "final_state")) || (st = check_workspace(shape, false, workspace, ws_bytes)))
    return st;
  if (!log_decay) return fail(ZO_EINVAL, "log_decay is NULL");
  if (((uintptr_t)lengths & 3u) != 0) return fail(ZO_EINVAL, "lengths is not aligned to its type");
  if (overlap(s, final_state, initial_state))
    return fail(ZO_EINVAL, "final_state and initial_state must be different buffers");
  if ((st = check_apart({strided("o", o, s, s.length, true, false)},
                        {strided("q", q, s, s.length, true, true), strided("k", k, s, s.length, false, true),
                         strided("v", v, s, s.length, false, false)})))
    return st;
  zo::LinCall c{};
  zo::LinPass& p = c.pass[0];
  p.x = heads(q, s.length);
  p.y = heads(k, s.length);
  p.z = heads(v, s.length);
  p.out = o->data;
  p.ob = o->batch_stride;
  p.ot = s.length < 2 ? 0 : o->position_stride;
  p.oh = o->head_stride;
  p.dx = s.key_dim;
  p.dz = s.value_dim;
  p.heads = s.q_heads / s.kv_heads;
  p.sources = 1;
  p.score = p.carry = s.scale;
  p.upd = 1.0f;
  p.init = initial_state;
  p.fin = final_state;
  c.npasses = 1;
  c.B = s.batch;
  c.T = s.length;
  c.kv_heads = s.kv_heads;
  c.share = s.q_heads / s.kv_heads;
  c.dtype = s.dtype;
  c.log_decay = log_decay;
  c.lengths = lengths;
  c.work = workspace;
  return device_status(zo::launch_linattn(c, (hipStream_t)stream), "zo_linear_attention");
}

int zo_linear_attention_backward(const zo_linattn* shape, const zo_heads* dout, const zo_heads* q,
                                 const zo_heads* k, const zo_heads* v, const zo_heads* dq, const zo_heads* dk,
                                 const zo_heads* dv, const float* log_decay, const int32_t* lengths,
                                 const float* initial_state, const float* dfinal_state, float* dinitial_state,
                                 void* workspace, size_t ws_bytes, void* stream) {
  zo::PhaseRange range("zo_linear_attention_backward");
  int st = check_linattn(shape);
  if (st) return st;
  const zo_linattn& s = *shape;
  const bool any = s.batch > 0 && s.length > 0;
  if ((st = check_heads(dout, "dout", s.dtype, any, s.length)) || (st = check_heads(q, "q", s.dtype, any, s.length)) ||
      (st = check_heads(k, "k", s.dtype, any, s.length)) || (st = check_heads(v, "v", s.dtype, any, s.length)) ||
      (st = check_heads(dq, "dq", s.dtype, any, s.length)) || (st = check_heads(dk, "dk", s.dtype, any, s.length)) ||
      (st = check_heads(dv, "dv", s.dtype, any, s.length)) || (st = check_state(log_decay, "log_decay")) ||
      (st = check_state(initial_state, "initial_state")) || (st = check_state(dfinal_state, "dfinal_state")) ||
      (st = check_state(dinitial_state, "dinitial_state")) ||
      (st = check_workspace(shape, true, workspace, ws_bytes)))
    return st;
  if (!log_decay) return fail(ZO_EINVAL, "log_decay is NULL");
  if (((uintptr_t)lengths & 3u) != 0) return fail(ZO_EINVAL, "lengths is not aligned to its type");
  if (overlap(s, dinitial_state, dfinal_state))
    return fail(ZO_EINVAL, "dinitial_state and dfinal_state must be different buffers");
  if ((st = check_apart({strided("dq", dq, s, s.length, true, true), strided("dk", dk, s, s.length, false, true),
                         strided("dv", dv, s, s.length, false, false)},
                        {strided("dout", dout, s, s.length, true, false), strided("q", q, s, s.length, true, true),
                         strided("k", k, s, s.length, false, true), strided("v", v, s, s.length, false, false)})))
    return st;
  const int share = s.q_heads / s.kv_heads;
  zo::LinCall c{};
  // dq: forward in time, the transposed state
  zo::LinPass& a = c.pass[0];
  a.x = heads(dout, s.length);
  a.y = heads(v, s.length);
  a.z = heads(k, s.length);
  a.out = dq->data;
  a.ob = dq->batch_stride;
  a.ot = s.length < 2 ? 0 : dq->position_stride;
  a.oh = dq->head_stride;
  a.dx = s.value_dim;
  a.dz = s.key_dim;
  a.heads = share;
  a.sources = 1;
  a.state_t = 1;
  a.score = a.carry = s.scale;
  a.upd = 1.0f;
  a.init = initial_state;
  // dv: backward in time, the gradient of the state
  zo::LinPass& d = c.pass[1];
  d.x = heads(k, s.length);
  d.y = heads(q, s.length);
  d.z = heads(dout, s.length);
  d.out = dv->data;
  d.ob = dv->batch_stride;
  d.ot = s.length < 2 ? 0 : dv->position_stride;
  d.oh = dv->head_stride;
  d.dx = s.key_dim;
  d.dz = s.value_dim;
  d.heads = 1;
  d.sources = share;
  d.reverse = 1;
  d.score = d.upd = s.scale;
  d.carry = 1.0f;
  d.init = dfinal_state;
  d.fin = dinitial_state;
  // dk: backward in time, its transpose
  zo::LinPass& e = c.pass[2];
  e = d;
  e.x = heads(v, s.length);
  e.y = heads(dout, s.length);
  e.z = heads(q, s.length);
  e.out = dk->data;
  e.ob = dk->batch_stride;
  e.ot = s.length < 2 ? 0 : dk->position_stride;
  e.oh = dk->head_stride;
  e.dx = s.value_dim;
  e.dz = s.key_dim;
  e.state_t = 1;
  e.fin = nullptr;
  c.npasses = 3;
  c.B = s.batch;
  c.T = s.length;
  c.kv_heads = s.kv_heads;
  c.share = s.q_heads / s.kv_heads;
  c.dtype = s.dtype;
  c.log_decay = log_decay;
  c.lengths = lengths;
  c.work = workspace;
  return device_status(zo::launch_linattn(c, (hipStream_t)stream), "zo_linear_attention_backward");
}

int zo_linear_attention_step(const zo_linattn* shape, const zo_heads* q, const zo_heads* k, const zo_heads* v,
                             const zo_heads* o, const float* log_decay, float* state, int32_t n_slots,
                             const int32_t* slots, void* stream) {
  zo::PhaseRange range("zo_linear_attention_step");
  int st = check_linattn(shape);
  if (st) return st;
  const zo_linattn& s = *shape;
  const bool any = s.batch > 0;
  if ((st = check_heads(q, "q", s.dtype, any, 1)) || (st = check_heads(k, "k", s.dtype, any, 1)) ||
      (st = check_heads(v, "v", s.dtype, any, 1)) || (st = check_heads(o, "o", s.dtype, any, 1)) ||
      (st = check_state(log_decay, "log_decay")) || (st = check_state(state, "state")))
    return st;
  if (!log_decay || (!state && n_slots > 0)) return fail(ZO_EINVAL, "a required pointer is NULL");
  if (n_slots < 0 || (!slots && n_slots < s.batch))
    return fail(ZO_EINVAL, "n_slots (%d) must be >= 0, and >= batch (%d) without slots", n_slots, s.batch);
  if (((uintptr_t)slots & 3u) != 0) return fail(ZO_EINVAL, "slots is not aligned to its type");
  if ((st = check_apart({strided("o", o, s, 1, true, false)}, {strided("q", q, s, 1, true, true),
                                                               strided("k", k, s, 1, false, true),
                                                               strided("v", v, s, 1, false, false)})))
    return st;
  zo::LinStep a{};
  a.q = heads(q, 1);
  a.k = heads(k, 1);
  a.v = heads(v, 1);
  a.o = o->data;
  a.ob = o->batch_stride;
  a.oh = o->head_stride;
  a.B = s.batch;
  a.q_heads = s.q_heads;
  a.kv_heads = s.kv_heads;
  a.dk = s.key_dim;
  a.dv = s.value_dim;
  a.dtype = s.dtype;
  a.scale = s.scale;
  a.log_decay = log_decay;
  a.state = state;
  a.n_slots = n_slots;
  a.slots = slots;
  return device_status(zo::launch_linattn_step(a, (hipStream_t)stream), "zo_linear_attention_step");
}

static int check_norm(int32_t xdtype, int32_t wdtype, int64_t rows, int64_t D) {
  if (!is_type(xdtype) || !is_type(wdtype)) return fail(ZO_EINVAL, "unknown dtype (%d, %d)", xdtype, wdtype);
  if (rows < 0 || D < 1) return fail(ZO_EINVAL, "rows must be >= 0 and D >= 1");
  if (D > (int64_t)1 << 30) return fail(ZO_ESHAPE, "D must be <= 2^30");
  if (rows > (int64_t)1 << 36) return fail(ZO_ESHAPE, "rows must be <= 2^36");
  return ZO_OK;
}

// Rows out over rows in: the same ones, or apart.
static int check_rows(const char* out, const void* y, int64_t ys, const char* in, const void* x, int64_t xs, int32_t type,
                      int64_t rows, int64_t D) {
  const bool same = y == x && (ys == xs || rows < 2);
  const Strided o(out, y, type, {{rows, ys}, {D, 1}}), i(in, x, type, {{rows, xs}, {D, 1}});
  return same ? check_apart({o}, {}) : check_apart({o}, {i});
}

int zo_layer_norm(int32_t xdtype, int32_t wdtype, int64_t rows, int64_t D, const void* x, int64_t x_stride,
                  const void* weight, const void* bias, float eps, void* y, int64_t y_stride, float* mean,
                  float* rstd, void* stream) {
  zo::PhaseRange range("zo_layer_norm");
  int st = check_norm(xdtype, wdtype, rows, D);
  if (st) return st;
  if (rows > 0 && (!x || !y)) return fail(ZO_EINVAL, "a required pointer is NULL");
  if (!mean != !rstd) return fail(ZO_EINVAL, "mean and rstd go together");
  if (!(eps >= 0.0f) || !std::isfinite(eps)) return fail(ZO_EINVAL, "eps must be finite and >= 0");
  if (!aligned_for(x, xdtype) || !aligned_for(y, xdtype) || !aligned_for(weight, wdtype) ||
      !aligned_for(bias, wdtype) || !aligned4(mean) || !aligned4(rstd))
    return fail(ZO_EINVAL, "a buffer is not aligned to its type");
  if ((st = check_rows("y", y, y_stride, "x", x, x_stride, xdtype, rows, D))) return st;
  zo::NormArgs a{};
  a.xdtype = xdtype;
  a.wdtype = wdtype;
  a.rows = rows;
  a.D = D;
  a.x = x;
  a.xs = x_stride;
  a.w = weight;
  a.b = bias;
  a.eps = eps;
  a.y = y;
  a.ys = y_stride;
  a.mean = mean;
  a.rstd = rstd;
  return device_status(zo::launch_norm(a, (hipStream_t)stream), "zo_layer_norm");
}

size_t zo_layer_norm_workspace_bytes(int64_t rows, int64_t D) {
  return check_norm(ZO_WFP32, ZO_WFP32, rows, D) ? 0 : zo::norm_workspace(rows, D);
}

int zo_layer_norm_backward(int32_t xdtype, int32_t wdtype, int64_t rows, int64_t D, const void* dy,
                           int64_t dy_stride, const void* x, int64_t x_stride, const void* weight,
                           const float* mean, const float* rstd, void* dx, int64_t dx_stride, float* dweight,
                           float* dbias, void* workspace, size_t ws_bytes, void* stream) {
  zo::PhaseRange range("zo_layer_norm_backward");
  int st = check_norm(xdtype, wdtype, rows, D);
  if (st) return st;
  if (rows > 0 && (!dy || !x || !mean || !rstd || !dx)) return fail(ZO_EINVAL, "a required pointer is NULL");
  if (!aligned_for(x, xdtype) || !aligned_for(dy, xdtype) || !aligned_for(dx, xdtype) ||
      !aligned_for(weight, wdtype) || !aligned4(mean) || !aligned4(rstd) || !aligned4(dweight) || !aligned4(dbias))
    return fail(ZO_EINVAL, "a buffer is not aligned to its type");
  const bool sums = dweight || dbias;
  if (sums) {
    const size_t need = zo::norm_workspace(rows, D);
    if (ws_bytes < need) return fail(ZO_ENOMEM, "workspace of %zu bytes < %zu required", ws_bytes, need);
    if (need && !workspace) return fail(ZO_EINVAL, "workspace is NULL");
    if (!aligned16(workspace)) return fail(ZO_EINVAL, "workspace must be 16-byte aligned");
  }
  if ((st = check_rows("dx", dx, dx_stride, "dy", dy, dy_stride, xdtype, rows, D)) ||
      (st = check_rows("dx", dx, dx_stride, "x", x, x_stride, xdtype, rows, D)))
    return st;
  zo::NormArgs a{};
  a.xdtype = xdtype;
  a.wdtype = wdtype;
  a.rows = rows;
  a.D = D;
  a.x = x;
  a.xs = x_stride;
  a.w = weight;
  a.y = dx;
  a.ys = dx_stride;
  a.dy = dy;
  a.dys = dy_stride;
  a.mean = const_cast<float*>(mean);
  a.rstd = const_cast<float*>(rstd);
  a.dw = dweight;
  a.db = dbias;
  a.partial = sums ? (float*)workspace : nullptr;
  return device_status(zo::launch_norm_backward(a, (hipStream_t)stream), "zo_layer_norm_backward");
}

int zo_adamw(const zo_adamw_config* cfg, const zo_adamw_tensor* tensors, int32_t n_tensors, void* m, void* v,
             float* m_scale, float* v_scale, const float* grad_scale, int32_t* skipped_out, void* stream) {
  zo::PhaseRange range("zo_adamw");
  if (!cfg) return fail(ZO_EINVAL, "cfg is NULL");
  if (!std::isfinite(cfg->lr) || !(cfg->eps >= 0.0) || !std::isfinite(cfg->eps))
    return fail(ZO_EINVAL, "lr must be finite, eps finite and >= 0");
  if (!(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0) || !(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0))
    return fail(ZO_EINVAL, "beta1 and beta2 must lie in [0, 1)");
  if (cfg->step < 1) return fail(ZO_EINVAL, "step must be >= 1");
  if (cfg->state_bits != 32 && cfg->state_bits != 8) return fail(ZO_EINVAL, "state_bits must be 32 or 8");
  if (n_tensors < 0 || (n_tensors > 0 && !tensors)) return fail(ZO_EINVAL, "n_tensors < 0, or tensors is NULL");
  bool any = false;
  Ranges params(n_tensors), moments(n_tensors);
  if (!params.ready() || !moments.ready()) return fail(ZO_ENOMEM, "no host memory for %d tensors", n_tensors);
  for (int32_t i = 0; i < n_tensors; ++i) {
    const zo_adamw_tensor& t = tensors[i];
    if (t.n < 0 || t.n > (int64_t)1 << 40) return fail(ZO_EINVAL, "tensor %d: n must lie in [0, 2^40]", i);
    if (!is_type(t.pdtype) || !is_type(t.gdtype)) return fail(ZO_EINVAL, "tensor %d: unknown dtype", i);
    if (t.n > 0 && (!t.param || !t.grad)) return fail(ZO_EINVAL, "tensor %d: param or grad is NULL", i);
    if (!aligned_for(t.param, t.pdtype) || !aligned_for(t.grad, t.gdtype))
      return fail(ZO_EINVAL, "tensor %d is not aligned to its type", i);
    if (t.state_offset < 0 || t.state_offset % ZO_ADAMW_BLOCK)
      return fail(ZO_EINVAL, "tensor %d: state_offset must be a multiple of %d", i, ZO_ADAMW_BLOCK);
    if (!std::isfinite(t.weight_decay)) return fail(ZO_EINVAL, "tensor %d: weight_decay must be finite", i);
    if (t.n == 0) continue;
    any = true;
    params.add((uint64_t)(uintptr_t)t.param, (uint64_t)t.n * type_bytes(t.pdtype));
    moments.add((uint64_t)t.state_offset, (uint64_t)((t.n + ZO_ADAMW_BLOCK - 1) / ZO_ADAMW_BLOCK * ZO_ADAMW_BLOCK));
  }
  // a launch updates all tensors in no order
  if (params.overlap()) return fail(ZO_EINVAL, "the param buffers of two tensors overlap");
  if (moments.overlap()) return fail(ZO_EINVAL, "the moments of two tensors overlap");
  if (any && (!m || !v)) return fail(ZO_EINVAL, "m or v is NULL");
  if (!aligned16(m) || !aligned16(v)) return fail(ZO_EINVAL, "m and v must be 16-byte aligned");
  if (cfg->state_bits == 8) {
    if (any && (!m_scale || !v_scale)) return fail(ZO_EINVAL, "8-bit moments need m_scale and v_scale");
  } else if (m_scale || v_scale) {
    return fail(ZO_EINVAL, "32-bit moments take no m_scale or v_scale");
  }
  if (!aligned4(m_scale) || !aligned4(v_scale) || !aligned4(grad_scale) || !aligned4(skipped_out))
    return fail(ZO_EINVAL, "a buffer is not aligned to its type");
  return device_status(zo::launch_adamw(*cfg, tensors, n_tensors, m, v, m_scale, v_scale, grad_scale, skipped_out,
                                        (hipStream_t)stream),
                       "zo_adamw");
}

int zo_adamw_moments(int64_t n, const void* m, const void* v, const float* m_scale, const float* v_scale,
                     float* m_out, float* v_out, void* stream) {
  zo::PhaseRange range("zo_adamw_moments");
  if (n < 0 || n % ZO_ADAMW_BLOCK) return fail(ZO_EINVAL, "n must be a multiple of %d", ZO_ADAMW_BLOCK);
  if (n > (int64_t)1 << 40) return fail(ZO_EINVAL, "n must be <= 2^40");
  if (n && (!m || !v || !m_scale || !v_scale || !m_out || !v_out))
    return fail(ZO_EINVAL, "a required pointer is NULL");
  if (!aligned16(m) || !aligned16(v) || !aligned16(m_out) || !aligned16(v_out) || !aligned4(m_scale) ||
      !aligned4(v_scale))
    return fail(ZO_EINVAL, "m, v, m_out and v_out must be 16-byte aligned");
  return device_status(zo::launch_adamw_moments(n, m, v, m_scale, v_scale, m_out, v_out, (hipStream_t)stream),
                       "zo_adamw_moments");
}

}  // extern "C"
