// C entries of rotary positions and of the token cache: argument checks, then one
// launcher each.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "fd_error.h"
#include "fd_token.h"

using fd::fail;

namespace {

constexpr double kTwoPi = 6.28318530717958647693;

int kind_of(int32_t dtype) { return dtype == FD_DTYPE_F16 ? 0 : dtype == FD_DTYPE_BF16 ? 1 : dtype == FD_DTYPE_F32 ? 2 : -1; }
int elem_size(int32_t dtype) { return dtype == FD_DTYPE_F32 ? 4 : 2; }

// Checks a rotation for vectors of head_dim elements (coords given apart).
fd_status check_rope(const fd_rope* r, int32_t head_dim, fd::RopeArgs* out) {
  if (r->struct_size != sizeof(fd_rope))
    return fail(FD_ERR_INVALID_ARGUMENT, "fd_rope struct_size %u != %zu", r->struct_size, sizeof(fd_rope));
  if (r->rot_dim < 0 || r->rot_dim % 2 || r->rot_dim > head_dim)
    return fail(FD_ERR_INVALID_ARGUMENT, "rot_dim %d must be even and in [0, head_dim %d]", r->rot_dim, head_dim);
  if (r->layout != FD_ROPE_INTERLEAVED && r->layout != FD_ROPE_HALF)
    return fail(FD_ERR_INVALID_ARGUMENT, "unknown rotary layout %d", r->layout);
  if (r->n_axes < 1 || r->n_axes > 4)
    return fail(FD_ERR_INVALID_ARGUMENT, "n_axes %d outside [1, 4]", r->n_axes);
  if (r->rot_dim > 0 && !r->freq) return fail(FD_ERR_INVALID_ARGUMENT, "fd_rope.freq is NULL");
  if ((uintptr_t)r->freq % 8 || (uintptr_t)r->axis % 4)
    return fail(FD_ERR_INVALID_ARGUMENT, "fd_rope.freq must be 8-byte aligned, axis 4-byte aligned");
  if (!std::isfinite(r->magnitude)) return fail(FD_ERR_INVALID_ARGUMENT, "fd_rope.magnitude is not finite");
  out->freq = r->freq;
  out->axis = r->axis;
  out->axes = r->n_axes;
  out->half = r->rot_dim / 2;
  out->interleaved = r->layout == FD_ROPE_INTERLEAVED;
  out->mag = r->magnitude;
  out->sign = r->inverse ? -1.f : 1.f;
  return FD_OK;
}

// Strides of rows that the kernels read and write 16 bytes at a time (those of
// extents of one are never stepped by).
bool strides_ok(const int64_t* s, std::initializer_list<int64_t> extents, int head_dim, int es) {
  for (int64_t e : extents) {
    if (e > 1 && (*s < head_dim || *s >= (int64_t)1 << 48 || *s * es % 16)) return false;
    ++s;
  }
  return true;
}

// Whether two rows of `width` elements at these strides (at least width where the extent is above
// one) share an element. Layouts that nest, as views of one tensor do, are seen at once; for
// others the distances along all axes but the longest are gone through, and the nearest
// steps of that one back.
bool rows_overlap(std::initializer_list<int64_t> strides, std::initializer_list<int64_t> extents, int64_t width) {
  struct Axis { int64_t stride, extent; } ax[3];
  int n = 0;
  for (auto s = strides.begin(), e = extents.begin(); s != strides.end(); ++s, ++e)
    if (*e > 1) ax[n++] = {*s, *e};
  std::sort(ax, ax + n, [](const Axis& a, const Axis& b) { return a.stride < b.stride; });
  __int128 span = width;
  bool nested = true;
  for (int i = 0; i < n; ++i) {
    nested = nested && ax[i].stride >= span;
    span += (__int128)(ax[i].extent - 1) * ax[i].stride;
  }
  if (nested) return false;
  std::sort(ax, ax + n, [](const Axis& a, const Axis& b) { return a.extent > b.extent; });
  const Axis b = n > 1 ? ax[1] : Axis{0, 1}, c = n > 2 ? ax[2] : Axis{0, 1};
  for (int64_t i = 0; i < b.extent; ++i)
    for (int64_t j = 1 - c.extent; j < c.extent; ++j) {
      const __int128 off = (__int128)i * b.stride + (__int128)j * c.stride;
      const __int128 k = off / ax[0].stride;  // and its neighbours
      for (int d = -1; d <= 1; ++d) {
        const __int128 x = off - (k + d) * ax[0].stride;
        const bool far = k + d >= ax[0].extent || k + d <= -(__int128)ax[0].extent;
        if (!far && x < width && -x < width && (i || j || k + d)) return true;
      }
    }
  return false;
}

fd_status check_cache(const fd_token_cache* c, fd::TokenCacheArgs* a) {
  if (!c) return fail(FD_ERR_INVALID_ARGUMENT, "cache is NULL");
  if (c->struct_size != sizeof(fd_token_cache))
    return fail(FD_ERR_INVALID_ARGUMENT, "fd_token_cache struct_size %u != %zu", c->struct_size, sizeof(fd_token_cache));
  if (kind_of(c->dtype) < 0) return fail(FD_ERR_INVALID_ARGUMENT, "unknown dtype %d", c->dtype);
  if (c->batch < 1 || c->groups < 1 || c->capacity < 1)
    return fail(FD_ERR_INVALID_ARGUMENT, "batch, groups and capacity must be positive");
  if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128)
    return fail(FD_ERR_UNSUPPORTED, "token cache head_dim %d (32, 64 or 128)", c->head_dim);
  if (c->capacity > FD_TOKEN_MAX_CAPACITY || (int64_t)c->batch * c->groups > 65535)
    return fail(FD_ERR_UNSUPPORTED, "capacity above 2^24, or more than 65535 (request, group) pairs");
  if (!c->k || !c->v || !c->pos || !c->weight) return fail(FD_ERR_INVALID_ARGUMENT, "NULL pointer in the cache");
  if (((uintptr_t)c->k | (uintptr_t)c->v) % 16 || ((uintptr_t)c->pos | (uintptr_t)c->weight) % 4)
    return fail(FD_ERR_INVALID_ARGUMENT, "k and v must be 16-byte aligned, pos and weight 4-byte aligned");
  const int es = elem_size(c->dtype);
  const auto extents = {(int64_t)c->batch, (int64_t)c->groups, (int64_t)c->capacity};
  if (!strides_ok(c->k_stride, extents, c->head_dim, es) || !strides_ok(c->v_stride, extents, c->head_dim, es))
    return fail(FD_ERR_INVALID_ARGUMENT, "cache strides must be at least head_dim and whole 16 bytes");
  if (c->capacity > 1 && (c->k_stride[2] * es >= 1 << 24 || c->v_stride[2] * es >= 1 << 24))
    return fail(FD_ERR_UNSUPPORTED, "slot strides must be below 2^24 bytes");
  a->k = c->k;
  a->v = c->v;
  a->pos = c->pos;
  a->weight = c->weight;
  for (int i = 0; i < 3; ++i) {
    a->ks[i] = c->k_stride[i];
    a->vs[i] = c->v_stride[i];
  }
  a->B = c->batch;
  a->G = c->groups;
  a->C = c->capacity;
  a->D = c->head_dim;
  return FD_OK;
}

fd_status launched(hipError_t e, const char* what) {
  return e == hipSuccess ? FD_OK : fail(FD_ERR_DEVICE, "%s launch failed: %s", what, hipGetErrorString(e));
}

}  // namespace

extern "C" {

fd_status fd_rope_frequencies(int32_t rot_dim, double theta, int32_t scaling, double factor, double trained_length,
                              double fast_turns, double slow_turns, double* freq, float* magnitude) {
  if (rot_dim < 2 || rot_dim % 2 || rot_dim > 512)
    return fail(FD_ERR_INVALID_ARGUMENT, "rot_dim %d must be even and in [2, 512]", rot_dim);
  if (!freq || !magnitude) return fail(FD_ERR_INVALID_ARGUMENT, "NULL pointer");
  if (!(theta > 1.0) || !std::isfinite(theta)) return fail(FD_ERR_INVALID_ARGUMENT, "theta must be finite and > 1");
  if (scaling < FD_ROPE_SCALE_NONE || scaling > FD_ROPE_SCALE_BANDS)
    return fail(FD_ERR_INVALID_ARGUMENT, "unknown rotary scaling %d", scaling);
  if (scaling != FD_ROPE_SCALE_NONE && (!(factor >= 1.0) || !std::isfinite(factor)))
    return fail(FD_ERR_INVALID_ARGUMENT, "scaling factor must be finite and >= 1");
  const bool bands = scaling == FD_ROPE_SCALE_BANDS;
  if (bands && (!(trained_length > 0.0) || !std::isfinite(trained_length) || !(slow_turns >= 0.0) ||
                !(fast_turns > slow_turns) || !std::isfinite(fast_turns)))
    return fail(FD_ERR_INVALID_ARGUMENT, "bands need trained_length > 0 and fast_turns > slow_turns >= 0");
  const int half = rot_dim / 2;
  const double base = scaling == FD_ROPE_SCALE_BASE && half > 1 ? theta * std::pow(factor, (double)half / (half - 1)) : theta;
  for (int i = 0; i < half; ++i) {
    double f = std::pow(base, -(double)i / half);
    if (scaling == FD_ROPE_SCALE_LINEAR) f /= factor;
    if (bands) {
      double keep = (trained_length * f / kTwoPi - slow_turns) / (fast_turns - slow_turns);
      keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
      f = keep * f + (1.0 - keep) * f / factor;
    }
    freq[i] = f;
  }
  *magnitude = bands ? (float)(1.0 + 0.1 * std::log(factor)) : 1.f;
  return FD_OK;
}

fd_status fd_rope_device(const fd_rope* rope, const void* x, int32_t dtype, int64_t tokens, int32_t heads,
                         int32_t head_dim, int64_t x_token_stride, int64_t x_head_stride, const int32_t* coords,
                         void* out, int64_t out_token_stride, int64_t out_head_stride, void* stream) {
  if (!rope) return fail(FD_ERR_INVALID_ARGUMENT, "rope is NULL");
  const int kind = kind_of(dtype);
  if (kind < 0) return fail(FD_ERR_INVALID_ARGUMENT, "unknown dtype %d", dtype);
  if (tokens < 0 || tokens > 0x7FFFFFFF || heads < 1 || heads > 65536 || head_dim < 1 || head_dim > 512)
    return fail(FD_ERR_INVALID_ARGUMENT, "tokens in [0, 2^31), heads in [1, 65536] and head_dim in [1, 512] required");
  fd::RopeArgs r;
  const fd_status st = check_rope(rope, head_dim, &r);
  if (st != FD_OK) return st;
  fd::RopeRows w;
  w.x = x;
  w.out = out;
  w.tokens = tokens;
  w.heads = heads;
  w.dim = head_dim;
  w.x_token = x_token_stride;
  w.x_head = x_head_stride;
  w.o_token = out_token_stride;
  w.o_head = out_head_stride;
  for (int64_t s : {x_token_stride, x_head_stride, out_token_stride, out_head_stride})
    if (s < 0 || s >= (int64_t)1 << 48) return fail(FD_ERR_INVALID_ARGUMENT, "strides must be in [0, 2^48)");
  if ((tokens > 1 && out_token_stride < head_dim) || (heads > 1 && out_head_stride < head_dim) ||
      rows_overlap({out_token_stride, out_head_stride}, {tokens, heads}, head_dim))
    return fail(FD_ERR_INVALID_ARGUMENT, "rows of out overlap");
  if (x == out && ((tokens > 1 && x_token_stride != out_token_stride) || (heads > 1 && x_head_stride != out_head_stride)))
    return fail(FD_ERR_INVALID_ARGUMENT, "in place needs the same strides for x and out");
  if (tokens == 0) return FD_OK;
  if (!x || !out || (r.half > 0 && !coords)) return fail(FD_ERR_INVALID_ARGUMENT, "NULL pointer");
  if (((uintptr_t)x | (uintptr_t)out) % elem_size(dtype) || (uintptr_t)coords % 4)
    return fail(FD_ERR_INVALID_ARGUMENT, "misaligned pointer");
  r.coords = coords;
  return launched(fd::rope_rows(r, w, kind, (hipStream_t)stream), "rotary");
}

// Sizes of a choice of slots.
static fd_status check_slots(int32_t batch, int32_t groups, int32_t capacity, int32_t n) {
  if (batch < 1 || groups < 1 || capacity < 1 || n < 0)
    return fail(FD_ERR_INVALID_ARGUMENT, "batch, groups and capacity must be positive, n >= 0");
  if (capacity > FD_TOKEN_MAX_CAPACITY || (int64_t)batch * groups > 65535)
    return fail(FD_ERR_UNSUPPORTED, "capacity above 2^24, or more than 65535 (request, group) pairs");
  if (n > capacity || n > fd::kMaxSlotTokens)
    return fail(FD_ERR_INVALID_ARGUMENT, "%d new tokens exceed the capacity %d or 65536", n, capacity);
  return FD_OK;
}

fd_status fd_token_slots_workspace(int32_t batch, int32_t groups, int32_t capacity, int32_t n, size_t* bytes) {
  const fd_status st = check_slots(batch, groups, capacity, n);
  if (st != FD_OK) return st;
  if (!bytes) return fail(FD_ERR_INVALID_ARGUMENT, "NULL pointer");
  *bytes = (size_t)fd::token_slots_workspace(batch, groups, capacity, n);
  return FD_OK;
}

fd_status fd_token_slots_device(const int32_t* slot_pos, const float* weight, int32_t batch, int32_t groups,
                                int32_t capacity, const int32_t* pos, int32_t n, int32_t keep_first,
                                int32_t keep_recent, int32_t* slots, void* workspace, size_t workspace_bytes,
                                void* stream) {
  const fd_status st = check_slots(batch, groups, capacity, n);
  if (st != FD_OK) return st;
  if (keep_first < 0 || keep_recent < 0) return fail(FD_ERR_INVALID_ARGUMENT, "keep_first and keep_recent must be >= 0");
  if (n == 0) return FD_OK;
  if (!slot_pos || !weight || !pos || !slots) return fail(FD_ERR_INVALID_ARGUMENT, "NULL pointer");
  if (((uintptr_t)slot_pos | (uintptr_t)weight | (uintptr_t)pos | (uintptr_t)slots) % 4)
    return fail(FD_ERR_INVALID_ARGUMENT, "misaligned pointer");
  const int64_t need = fd::token_slots_workspace(batch, groups, capacity, n);
  if (need > 0 && (!workspace || (uintptr_t)workspace % 4 || workspace_bytes < (size_t)need))
    return fail(FD_ERR_INVALID_ARGUMENT, "workspace of %zu bytes, %lld needed (4-byte aligned)", workspace_bytes,
                (long long)need);
  fd::TokenSlots a;
  a.slot_pos = slot_pos;
  a.weight = weight;
  a.pos = pos;
  a.slots = slots;
  a.B = batch;
  a.G = groups;
  a.C = capacity;
  a.n = n;
  a.keep_first = keep_first;
  a.keep_recent = keep_recent;
  a.ws = workspace;
  return launched(fd::token_slots(a, (hipStream_t)stream), "slot choice");
}

fd_status fd_token_append_device(const fd_token_cache* cache, const fd_rope* rope, const void* k,
                                 const int64_t k_stride[3], const void* v, const int64_t v_stride[3], int32_t n,
                                 const int32_t* pos, const int32_t* coords, const int32_t* slots, void* stream) {
  fd::TokenCacheArgs c;
  fd_status st = check_cache(cache, &c);
  if (st != FD_OK) return st;
  fd::RopeArgs r;
  if (rope && (st = check_rope(rope, c.D, &r)) != FD_OK) return st;
  if (n < 0 || (int64_t)c.B * n > 0x7FFFFFFF)
    return fail(FD_ERR_INVALID_ARGUMENT, "n >= 0 and batch x n below 2^31 required");
  if (n == 0) return FD_OK;
  for (const int64_t* x : {c.ks, c.vs})
    if (rows_overlap({x[0], x[1], x[2]}, {c.B, c.G, c.C}, c.D))
      return fail(FD_ERR_INVALID_ARGUMENT, "rows of the cache overlap");
  if (!k || !v || !k_stride || !v_stride || !pos || !slots) return fail(FD_ERR_INVALID_ARGUMENT, "NULL pointer");
  if (r.half > 0 && !coords && r.axes != 1)
    return fail(FD_ERR_INVALID_ARGUMENT, "coords may be NULL only for one axis (then pos turns the keys)");
  const int es = elem_size(cache->dtype);
  if (((uintptr_t)k | (uintptr_t)v) % 16 || ((uintptr_t)pos | (uintptr_t)coords | (uintptr_t)slots) % 4)
    return fail(FD_ERR_INVALID_ARGUMENT, "k and v must be 16-byte aligned, pos, coords and slots 4-byte aligned");
  const auto extents = {(int64_t)c.B, (int64_t)n, (int64_t)c.G};
  if (!strides_ok(k_stride, extents, c.D, es) || !strides_ok(v_stride, extents, c.D, es))
    return fail(FD_ERR_INVALID_ARGUMENT, "strides of k and v must be at least head_dim and whole 16 bytes");
  r.coords = coords ? coords : pos;
  fd::TokenAppend a;
  a.k = k;
  a.v = v;
  for (int i = 0; i < 3; ++i) {
    a.ks[i] = k_stride[i];
    a.vs[i] = v_stride[i];
  }
  a.n = n;
  a.pos = pos;
  a.slots = slots;
  return launched(fd::token_append(c, r, a, kind_of(cache->dtype), (hipStream_t)stream), "append");
}

// Sizes of an attention call that the launches can index.
static fd_status check_attend(const fd::TokenCacheArgs& c, int32_t heads, int32_t n) {
  if (heads < 1 || heads % c.G) return fail(FD_ERR_INVALID_ARGUMENT, "heads %d must be a multiple of groups %d", heads, c.G);
  if (n < 0) return fail(FD_ERR_INVALID_ARGUMENT, "n must be >= 0");
  const int64_t rows = (int64_t)n * (heads / c.G), bg = (int64_t)c.B * c.G;
  if (heads / c.G > 256) return fail(FD_ERR_UNSUPPORTED, "more than 256 heads a group");
  if (rows > (int64_t)1 << 24 || bg * rows > (int64_t)1 << 28 || bg * c.C > (int64_t)1 << 31)
    return fail(FD_ERR_UNSUPPORTED,
                "n x heads / groups above 2^24, batch x n x heads above 2^28, or batch x groups x capacity above 2^31");
  return FD_OK;
}

fd_status fd_token_attend_workspace(const fd_token_cache* cache, int32_t heads, int32_t n, int32_t weights,
                                    size_t* bytes) {
  fd::TokenCacheArgs c;
  fd_status st = check_cache(cache, &c);
  if (st != FD_OK) return st;
  if ((st = check_attend(c, heads, n)) != FD_OK) return st;
  if (!bytes) return fail(FD_ERR_INVALID_ARGUMENT, "NULL pointer");
  *bytes = n == 0 ? 0 : (size_t)fd::token_attend_plan(c, n, heads / c.G, kind_of(cache->dtype), weights != 0).bytes;
  return FD_OK;
}

fd_status fd_token_attend_device(const fd_token_cache* cache, const void* q, const int64_t q_stride[3], int32_t heads,
                                 int32_t n, const int32_t* pos, float scale, int32_t causal, void* out,
                                 const int64_t out_stride[3], float* lse, float decay, float* weight_out,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  fd::TokenCacheArgs c;
  fd_status st = check_cache(cache, &c);
  if (st != FD_OK) return st;
  if ((st = check_attend(c, heads, n)) != FD_OK) return st;
  // (the kernels take powers of two: scale log2 e, which need not be finite where scale is)
  if (!std::isfinite(scale * 1.44269504f) || !(scale > 0.f))
    return fail(FD_ERR_INVALID_ARGUMENT, "scale must be > 0, and scale / ln 2 finite in fp32");
  if (!std::isfinite(decay)) return fail(FD_ERR_INVALID_ARGUMENT, "decay must be finite");
  if ((uintptr_t)weight_out % 4 || (uintptr_t)lse % 4)
    return fail(FD_ERR_INVALID_ARGUMENT, "lse and weight_out must be 4-byte aligned");
  const int kind = kind_of(cache->dtype), rep = heads / c.G;
  fd::TokenAttend a;
  fd::TokenAttendPlan plan;
  a.n = n;
  a.rep = rep;
  a.scale = scale;
  a.causal = causal != 0;
  a.lse = lse;
  a.weight_out = weight_out;
  a.decay = decay;
  if (n > 0) {
    if (!q || !out || !q_stride || !out_stride || !pos) return fail(FD_ERR_INVALID_ARGUMENT, "NULL pointer");
    const int es = elem_size(cache->dtype);
    const auto extents = {(int64_t)c.B, (int64_t)n, (int64_t)heads};
    if (((uintptr_t)q | (uintptr_t)out) % 16 || (uintptr_t)pos % 4)
      return fail(FD_ERR_INVALID_ARGUMENT, "q and out must be 16-byte aligned, pos 4-byte aligned");
    if (!strides_ok(q_stride, extents, c.D, es) || !strides_ok(out_stride, extents, c.D, es))
      return fail(FD_ERR_INVALID_ARGUMENT, "strides of q and out must be at least head_dim and whole 16 bytes");
    if (rows_overlap({out_stride[0], out_stride[1], out_stride[2]}, {c.B, n, heads}, c.D))
      return fail(FD_ERR_INVALID_ARGUMENT, "rows of out overlap");
    plan = fd::token_attend_plan(c, n, rep, kind, weight_out != nullptr);
    const int64_t need = plan.bytes;
    if (need > 0 && (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < (size_t)need))
      return fail(FD_ERR_INVALID_ARGUMENT, "workspace of %zu bytes, %lld needed (16-byte aligned)", workspace_bytes,
                  (long long)need);
    a.q = q;
    a.out = out;
    for (int i = 0; i < 3; ++i) {
      a.qs[i] = q_stride[i];
      a.os[i] = out_stride[i];
    }
    a.pos = pos;
    a.ws = workspace;
  }
  return launched(fd::token_attend(c, a, plan, kind, (hipStream_t)stream), "token attention");
}

}  // extern "C"
