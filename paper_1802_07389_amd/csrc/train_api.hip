// train_api.hip -- host side of the training-step operators of include/tlc.h:
// argument checks, their context's workspace and the launches on its stream.
#include <math.h>

#include <new>
#include <type_traits>
#include <vector>

#include "api_common.hpp"
#include "train_internal.h"
#include "typed_io.hpp"

using namespace tlc;

namespace {

// Staging slots of the lists' pieces, in two groups: one event after a group's
// last call guards the group (an event a call cost the host more than the
// pieces).
constexpr int kGroups = 2, kGroupSlots = 4;
constexpr size_t kMaxListValues = (size_t)1 << 40;

bool known_type(int type) { return type == TLC_F32 || type == TLC_BF16 || type == TLC_F16; }

// Bytes from the first to the last value of `count` rows; false: beyond the
// address space.
bool rows_extent(size_t count, size_t dim, size_t stride, size_t value, size_t* bytes) {
  *bytes = 0;
  if (count == 0 || dim == 0) return true;
  size_t v = 0;
  return !__builtin_mul_overflow(count - 1, stride, &v) && !__builtin_add_overflow(v, dim, &v) &&
         !__builtin_mul_overflow(v, value, bytes);
}

}  // namespace

struct tlc_train {
  hipStream_t stream = nullptr;
  int device = 0;
  size_t max_tokens = 0, max_rows = 0, max_dim = 0, max_tensors = 0;
  bool broken = false;
  // device workspace (one allocation)
  void* ws = nullptr;
  double* partials = nullptr;
  Piece* pieces = nullptr;  // a long list's, for its clipping
  GradWork grad = {};
  // pinned: the sticky index flag and the staging slots of the pieces
  uint32_t* bad = nullptr;
  uint32_t* bad_dev = nullptr;
  Piece* staging = nullptr;
  Piece* staging_dev = nullptr;  // the same, as the device addresses it
  size_t slot_pieces = 0;
  hipEvent_t group_done[kGroups] = {};
  bool group_used[kGroups] = {};
  int slot_next = 0;
  // host tables, reserved at creation so that the calls do not allocate
  std::vector<Span> spans, spans_ok;
};

namespace {

int check_usable(tlc_train* c, const char* fn) {
  if (!c) return fail(TLC_E_INVALID, "%s: NULL context", fn);
  if (c->broken) return fail(TLC_E_DEVICE, "%s: context unusable after a device error", fn);
  return TLC_OK;
}

int launched(tlc_train* c, hipError_t e, const char* what) {
  if (e == hipSuccess) return TLC_OK;
  c->broken = true;
  return hip_fail(e, what);
}

int check_table(const char* fn, size_t rows, size_t dim, int ids_type, int value_type,
                size_t count, float scale) {
  if (rows == 0 || rows > TLC_MAX_ROWS)
    return fail(TLC_E_INVALID, "%s: rows = %zu not in [1, %d]", fn, rows, TLC_MAX_ROWS);
  if (dim == 0 || dim > TLC_MAX_DIM)
    return fail(TLC_E_INVALID, "%s: dim = %zu not in [1, %d]", fn, dim, TLC_MAX_DIM);
  if (count > INT32_MAX) return fail(TLC_E_INVALID, "%s: %zu tokens", fn, count);
  if (ids_type != TLC_I32 && ids_type != TLC_I64)
    return fail(TLC_E_INVALID, "%s: unknown type of ids %d", fn, ids_type);
  if (!known_type(value_type))
    return fail(TLC_E_INVALID, "%s: unknown type %d", fn, value_type);
  if (!isfinite(scale))
    return fail(TLC_E_INVALID, "%s: scale %g is not finite", fn, (double)scale);
  return TLC_OK;
}

// The next pinned slot: a group's first one waits for the group's last calls.
int take_slot(tlc_train* c, Piece** host, const Piece** dev) {
  const int slot = c->slot_next, group = slot / kGroupSlots;
  if (slot % kGroupSlots == 0 && c->group_used[group]) {
    const hipError_t e = hipEventSynchronize(c->group_done[group]);
    if (e != hipSuccess) return hip_fail(e, "hipEventSynchronize(staging)");
    c->group_used[group] = false;
  }
  *host = c->staging + (size_t)slot * c->slot_pieces;
  *dev = c->staging_dev + (size_t)slot * c->slot_pieces;
  return TLC_OK;
}

// After the kernels that read the slot are queued.
int leave_slot(tlc_train* c) {
  const int slot = c->slot_next, group = slot / kGroupSlots;
  c->slot_next = (slot + 1) % (kGroups * kGroupSlots);
  if (c->slot_next % kGroupSlots != 0) return TLC_OK;
  const hipError_t e = hipEventRecord(c->group_done[group], c->stream);
  if (e != hipSuccess) return launched(c, e, "hipEventRecord(staging)");
  c->group_used[group] = true;
  return TLC_OK;
}

// A call on a list of tensors.  clip: they are scaled into outs, or in place
// (outs NULL).
struct ListCall {
  size_t count;
  const void* const* tensors;
  const int* types;
  const size_t* ns;
  tlc_norm_result* result;
  bool clip;
  float* const* outs;
  size_t total = 0;  // values; set by check_list
};

int check_list(tlc_train* c, const char* fn, ListCall* l) {
  int st = check_usable(c, fn);
  if (st) return st;
  if (!l->result) return fail(TLC_E_INVALID, "%s: NULL result", fn);
  if (l->count && (!l->tensors || !l->types || !l->ns))
    return fail(TLC_E_INVALID, "%s: NULL argument", fn);
  if (l->count > c->max_tensors)
    return fail(TLC_E_INVALID, "%s: %zu tensors exceed the context's %zu", fn, l->count,
                c->max_tensors);
  c->spans.clear();
  add_span(c->spans, l->result, sizeof(*l->result), true);
  for (size_t i = 0; i < l->count; ++i) {
    const size_t n = l->ns[i];
    if (n == 0) continue;
    if (!known_type(l->types[i]))
      return fail(TLC_E_INVALID, "%s: tensor %zu: unknown type %d", fn, i, l->types[i]);
    if (n > TLC_MAX_N)
      return fail(TLC_E_INVALID, "%s: tensor %zu: n = %zu too large", fn, i, n);
    if (!l->tensors[i] || (l->outs && !l->outs[i]))
      return fail(TLC_E_INVALID, "%s: tensor %zu: NULL pointer", fn, i);
    const size_t bytes = n * type_bytes(l->types[i]);
    l->total += n;
    const bool in_place =
        l->clip &&
        (!l->outs || ((const void*)l->outs[i] == l->tensors[i] && l->types[i] == TLC_F32));
    add_span(c->spans, l->tensors[i], bytes, in_place);
    if (l->clip && !in_place) add_span(c->spans, l->outs[i], n * 4, true);
  }
  if (l->total > kMaxListValues)
    return fail(TLC_E_INVALID, "%s: %zu values exceed %zu", fn, l->total, kMaxListValues);
  if (spans_conflict_cached(c->spans, c->spans_ok))
    return fail(TLC_E_INVALID, "%s: a written buffer overlaps another one", fn);
  return TLC_OK;
}

ArgList arg_list(const ListCall& l) {
  ArgList r = {};
  r.own_type = l.clip && !l.outs;
  r.len = piece_values(l.total, l.count);
  for (size_t i = 0; i < l.count; ++i) {
    if (l.ns[i] == 0) continue;
    ListTensor& e = r.tensors[r.count++];
    e.x = l.tensors[i];
    e.out = l.outs ? (void*)l.outs[i] : (void*)l.tensors[i];
    e.n = (uint32_t)l.ns[i];
    e.piece0_type = r.n | (uint32_t)l.types[i] << 30;
    r.n += (uint32_t)ceil_div(l.ns[i], r.len);
  }
  return r;
}

PinnedList pinned_list(const ListCall& l, Piece* host, const Piece* dev, Piece* copy) {
  PinnedList r = {};
  r.copy = copy;
  r.own_type = l.clip && !l.outs;
  r.pieces = dev;
  const size_t len = piece_values(l.total, l.count);
  for (size_t i = 0; i < l.count; ++i) {
    const size_t size = type_bytes(l.types[i]);
    for (size_t k = 0; k < l.ns[i]; k += len) {
      Piece& p = host[r.n++];
      p.x = (const uint8_t*)l.tensors[i] + k * size;
      p.out = l.outs ? (void*)(l.outs[i] + k) : (void*)p.x;
      p.n = (uint32_t)std::min<size_t>(len, l.ns[i] - k);
      p.type = (uint32_t)l.types[i];
    }
  }
  return r;
}

// Checks the call, then has `run` queue its kernels on the list.
template <class F>
int run_list(tlc_train* c, const char* fn, ListCall l, F&& run) {
  int st = check_list(c, fn, &l);
  if (st) return st;
  DeviceScope dev(c->device);
  st = dev.status();
  if (st) return st;
  if (l.count <= kArgTensors) return launched(c, run(arg_list(l)), fn);
  // a replay would read the slot after later calls have filled it again
  hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
  const hipError_t e = hipStreamIsCapturing(c->stream, &capture);
  if (e != hipSuccess) return hip_fail(e, "hipStreamIsCapturing");
  if (capture != hipStreamCaptureStatusNone)
    return fail(TLC_E_INVALID, "%s: a list of %zu tensors cannot be captured (%u at most)", fn,
                l.count, kArgTensors);
  Piece* host = nullptr;
  const Piece* pieces = nullptr;
  st = take_slot(c, &host, &pieces);
  if (!st) st = launched(c, run(pinned_list(l, host, pieces, l.clip ? c->pieces : nullptr)), fn);
  return st ? st : leave_slot(c);
}

int check_clip(const char* fn, float max_norm) {
  if (!(isfinite(max_norm) && max_norm >= 0.0f))
    return fail(TLC_E_INVALID, "%s: max_norm %g is not finite and >= 0", fn, (double)max_norm);
  return TLC_OK;
}

}  // namespace

TLC_API int tlc_train_create(tlc_train** out, size_t max_tokens, size_t max_rows, size_t max_dim,
                             size_t max_tensors, void* hip_stream) {
  if (!out) return fail(TLC_E_INVALID, "tlc_train_create: ctx pointer is NULL");
  *out = nullptr;
  if (max_tokens > INT32_MAX || max_rows > TLC_MAX_ROWS || max_dim > TLC_MAX_DIM ||
      max_tensors > TLC_MAX_TENSORS)
    return fail(TLC_E_INVALID,
                "tlc_train_create: %zu tokens, %zu rows, %zu values a row or %zu tensors are too "
                "many",
                max_tokens, max_rows, max_dim, max_tensors);
  tlc_train* c = new (std::nothrow) tlc_train();
  if (!c) return fail(TLC_E_DEVICE, "tlc_train_create: out of host memory");
  c->stream = (hipStream_t)hip_stream;
  c->max_tokens = max_tokens;
  c->max_rows = max_rows;
  c->max_dim = max_dim;
  c->max_tensors = max_tensors;
  hipError_t e = hipGetDevice(&c->device);
  if (e != hipSuccess) {
    delete c;
    return hip_fail(e, "hipGetDevice");
  }
  c->slot_pieces = max_tensors > kArgTensors ? kNormBlocks + max_tensors : 0;
  // layout: partial sums | a long list's pieces | sorted tokens, twice | counts of the sort |
  //         touched rows | partial rows
  size_t off = round_up(kNormBlocks * sizeof(double), 256);
  const size_t off_pieces = off;
  off = round_up(off + c->slot_pieces * sizeof(Piece), 256);
  size_t off_sort[4];
  for (size_t& o : off_sort) {
    o = off;
    off = round_up(off + max_tokens * sizeof(uint32_t), 256);
  }
  const size_t off_counts = off;
  off = round_up(off + kSortPasses * ceil_div(max_tokens, kSortTile) * kDigits * sizeof(uint32_t),
                 256);
  const size_t off_touched = off;
  off = round_up(off + max_rows, 256);
  const size_t off_parts = off;
  off = round_up(off + ceil_div(max_tokens, kSumMinTokens * kSumWaves) * 2 * max_dim *
                           sizeof(float), 256);
  e = hipMalloc(&c->ws, off);
  if (e == hipSuccess) e = hipMemset((uint8_t*)c->ws + off_touched, 0, max_rows);
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e == hipSuccess) e = hipHostMalloc((void**)&c->bad, 256, hipHostMallocDefault);
  if (e == hipSuccess) e = hipHostGetDevicePointer((void**)&c->bad_dev, c->bad, 0);
  if (e == hipSuccess && c->slot_pieces)
    e = hipHostMalloc((void**)&c->staging, kGroups * kGroupSlots * c->slot_pieces * sizeof(Piece),
                      hipHostMallocDefault);
  if (e == hipSuccess && c->staging)
    e = hipHostGetDevicePointer((void**)&c->staging_dev, c->staging, 0);
  for (int i = 0; i < kGroups && e == hipSuccess; ++i)
    e = hipEventCreateWithFlags(&c->group_done[i], hipEventDisableTiming);
  if (e != hipSuccess) {
    tlc_train_destroy(c);
    return hip_fail(e, "tlc_train_create: workspace");
  }
  *c->bad = 0u;
  uint8_t* base = (uint8_t*)c->ws;
  c->partials = (double*)base;
  c->pieces = (Piece*)(base + off_pieces);
  for (int i = 0; i < 2; ++i) {
    c->grad.keys[i] = (uint32_t*)(base + off_sort[i]);
    c->grad.pos[i] = (uint32_t*)(base + off_sort[2 + i]);
  }
  c->grad.counts = (uint32_t*)(base + off_counts);
  c->grad.touched = base + off_touched;
  c->grad.parts = (float*)(base + off_parts);
  try {
    c->spans.reserve(2 * max_tensors + 1);
    c->spans_ok.reserve(2 * max_tensors + 1);
  } catch (...) {
    tlc_train_destroy(c);
    return fail(TLC_E_DEVICE, "tlc_train_create: out of host memory");
  }
  *out = c;
  return TLC_OK;
}

TLC_API int tlc_train_destroy(tlc_train* c) {
  if (!c) return TLC_OK;
  DeviceScope dev(c->device);
  (void)hipStreamSynchronize(c->stream);
  for (int i = 0; i < kGroups; ++i)
    if (c->group_done[i]) (void)hipEventDestroy(c->group_done[i]);
  if (c->staging) (void)hipHostFree(c->staging);
  if (c->bad) (void)hipHostFree(c->bad);
  if (c->ws) (void)hipFree(c->ws);
  delete c;
  return TLC_OK;
}

TLC_API int tlc_train_sync(tlc_train* c) {
  if (!c) return fail(TLC_E_INVALID, "tlc_train_sync: NULL context");
  DeviceScope dev(c->device);
  int st = dev.status();
  if (st) return st;
  const hipError_t e = hipStreamSynchronize(c->stream);
  if (e != hipSuccess) return hip_fail(e, "hipStreamSynchronize");
  volatile uint32_t* bad = c->bad;
  if (*bad) {
    *bad = 0u;
    return fail(TLC_E_INDEX, "a token id is outside the embedding table");
  }
  return TLC_OK;
}

// ---------------------------------------------------------------- embedding
TLC_API int tlc_embedding(tlc_train* c, const void* table, int table_type, size_t rows,
                          size_t dim, size_t table_stride, const void* ids, int ids_type,
                          size_t count, float scale, void* out, int out_type,
                          size_t out_stride) {
  const char* fn = "tlc_embedding";
  int st = check_usable(c, fn);
  if (st) return st;
  st = check_table(fn, rows, dim, ids_type, table_type, count, scale);
  if (st) return st;
  if (!known_type(out_type)) return fail(TLC_E_INVALID, "%s: unknown type %d", fn, out_type);
  if (count == 0) return TLC_OK;
  if (!table || !ids || !out) return fail(TLC_E_INVALID, "%s: NULL device pointer", fn);
  if (out_stride < dim)
    return fail(TLC_E_INVALID, "%s: out_stride %zu below dim %zu", fn, out_stride, dim);
  size_t table_bytes = 0, out_bytes = 0;
  if (!rows_extent(rows, dim, table_stride, type_bytes(table_type), &table_bytes) ||
      !rows_extent(count, dim, out_stride, type_bytes(out_type), &out_bytes))
    return fail(TLC_E_INVALID, "%s: strides beyond the address space", fn);
  if (overlap(out, out_bytes, table, table_bytes) ||
      overlap(out, out_bytes, ids, count * (ids_type == TLC_I64 ? 8 : 4)))
    return fail(TLC_E_INVALID, "%s: out overlaps the table or the ids", fn);
  DeviceScope dev(c->device);
  st = dev.status();
  if (st) return st;
  EmbArgs a = {};
  a.x = table;
  a.ids = ids;
  a.out = out;
  a.x_stride = table_stride;
  a.out_stride = out_stride;
  a.count = (uint32_t)count;
  a.rows = (uint32_t)rows;
  a.dim = (uint32_t)dim;
  a.scale = scale;
  a.bad = c->bad_dev;
  return launched(c, launch_embedding(a, table_type, ids_type, out_type, c->stream), fn);
}

TLC_API int tlc_embedding_grad(tlc_train* c, const void* grad, int grad_type, size_t grad_stride,
                               const void* ids, int ids_type, size_t count, size_t rows,
                               size_t dim, float scale, int64_t padding_id, float* out,
                               size_t out_stride, int accumulate) {
  const char* fn = "tlc_embedding_grad";
  int st = check_usable(c, fn);
  if (st) return st;
  st = check_table(fn, rows, dim, ids_type, grad_type, count, scale);
  if (st) return st;
  if (count > c->max_tokens || rows > c->max_rows || dim > c->max_dim)
    return fail(TLC_E_INVALID,
                "%s: %zu tokens, %zu rows of %zu exceed the context's %zu, %zu of %zu", fn, count,
                rows, dim, c->max_tokens, c->max_rows, c->max_dim);
  if (!out || (count && (!grad || !ids)))
    return fail(TLC_E_INVALID, "%s: NULL device pointer", fn);
  if (out_stride < dim)
    return fail(TLC_E_INVALID, "%s: out_stride %zu below dim %zu", fn, out_stride, dim);
  size_t grad_bytes = 0, out_bytes = 0;
  if (!rows_extent(count, dim, grad_stride, type_bytes(grad_type), &grad_bytes) ||
      !rows_extent(rows, dim, out_stride, 4, &out_bytes))
    return fail(TLC_E_INVALID, "%s: strides beyond the address space", fn);
  if (overlap(out, out_bytes, grad, grad_bytes) ||
      overlap(out, out_bytes, ids, count * (ids_type == TLC_I64 ? 8 : 4)))
    return fail(TLC_E_INVALID, "%s: out overlaps the gradient or the ids", fn);
  if (count == 0 && accumulate) return TLC_OK;
  DeviceScope dev(c->device);
  st = dev.status();
  if (st) return st;
  EmbArgs a = {};
  a.x = grad;
  a.ids = ids;
  a.out = out;
  a.x_stride = grad_stride;
  a.out_stride = out_stride;
  a.count = (uint32_t)count;
  a.rows = (uint32_t)rows;
  a.dim = (uint32_t)dim;
  a.scale = scale;
  a.padding = padding_id;
  a.wide_ids = ids_type == TLC_I64;
  a.bad = c->bad_dev;
  return launched(c, launch_embedding_grad(a, grad_type, accumulate != 0, c->grad,
                                           c->stream), fn);
}

// ---------------------------------------------------------------- norm, clip
TLC_API int tlc_grad_norm(tlc_train* c, size_t count, const void* const* tensors,
                          const int* types, const size_t* ns, tlc_norm_result* result) {
  return run_list(c, "tlc_grad_norm", ListCall{count, tensors, types, ns, result, false, nullptr},
                  [&](const auto& list) {
                    const hipError_t e = launch_sumsq(list, true, c->partials, c->stream);
                    if (e != hipSuccess) return e;
                    return launch_norm_finish(c->partials, norm_blocks(list.n), result, c->stream);
                  });
}

TLC_API int tlc_clip(tlc_train* c, size_t count, const void* const* tensors, const int* types,
                     const size_t* ns, float max_norm, tlc_norm_result* result,
                     float* const* outs) {
  const int st = check_clip("tlc_clip", max_norm);
  if (st) return st;
  return run_list(c, "tlc_clip", ListCall{count, tensors, types, ns, result, true, outs},
                  [&](const auto& list) {
                    return launch_clip(list, nullptr, 0, max_norm, result, c->stream);
                  });
}

TLC_API int tlc_clip_grad_norm(tlc_train* c, size_t count, const void* const* tensors,
                               const int* types, const size_t* ns, float max_norm,
                               tlc_norm_result* result, float* const* outs) {
  const int st = check_clip("tlc_clip_grad_norm", max_norm);
  if (st) return st;
  return run_list(c, "tlc_clip_grad_norm",
                  ListCall{count, tensors, types, ns, result, true, outs},
                  [&](const auto& list) {
                    const hipError_t e = launch_sumsq(list, false, c->partials, c->stream);
                    if (e != hipSuccess) return e;
                    auto again = list;
                    if constexpr (std::is_same_v<decltype(again), PinnedList>)
                      again.pieces = again.copy;
                    return launch_clip(again, c->partials, norm_blocks(list.n), max_norm, result,
                                       c->stream);
                  });
}
