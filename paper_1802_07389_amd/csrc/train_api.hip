// train_api.hip -- host side of the training-step operators of include/tlc.h:
// argument checks, their context's workspace and the launches on its stream.
#include <math.h>

#include <new>
#include <vector>

#include "api_common.hpp"
#include "train_internal.h"
#include "typed_io.hpp"

using namespace tlc;

namespace {

constexpr int kSlots = 4;
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
  GradWork grad = {};
  // pinned: the sticky index flag and the staging slots of the pieces
  uint32_t* bad = nullptr;
  uint32_t* bad_dev = nullptr;
  Piece* staging = nullptr;
  Piece* staging_dev = nullptr;  // the same, as the device addresses it
  size_t slot_pieces = 0;
  hipEvent_t slot_done[kSlots] = {};
  bool slot_used[kSlots] = {};
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

// A pinned slot, free once the kernels of its last call have run.
int take_slot(tlc_train* c, int* slot) {
  *slot = c->slot_next;
  c->slot_next = (*slot + 1) % kSlots;
  if (c->slot_used[*slot]) {
    const hipError_t e = hipEventSynchronize(c->slot_done[*slot]);
    if (e != hipSuccess) return hip_fail(e, "hipEventSynchronize(staging)");
    c->slot_used[*slot] = false;
  }
  return TLC_OK;
}

// Checks a list of tensors and cuts it into pieces: into l's table, or into a
// pinned slot (*slot, to be held after the kernels that read it; else -1).
// clip: the tensors are scaled into outs, or in place (outs NULL).
int cut_list(tlc_train* c, const char* fn, size_t count, const void* const* tensors,
             const int* types, const size_t* ns, tlc_norm_result* result, bool clip,
             float* const* outs, ListArgs* l, int* slot) {
  *slot = -1;
  int st = check_usable(c, fn);
  if (st) return st;
  if (!result) return fail(TLC_E_INVALID, "%s: NULL result", fn);
  if (count && (!tensors || !types || !ns)) return fail(TLC_E_INVALID, "%s: NULL argument", fn);
  if (count > c->max_tensors)
    return fail(TLC_E_INVALID, "%s: %zu tensors exceed the context's %zu", fn, count,
                c->max_tensors);
  size_t total = 0, total_bytes = 0;
  c->spans.clear();
  add_span(c->spans, result, sizeof(*result), true);
  for (size_t i = 0; i < count; ++i) {
    if (ns[i] == 0) continue;
    if (!known_type(types[i]))
      return fail(TLC_E_INVALID, "%s: tensor %zu: unknown type %d", fn, i, types[i]);
    if (ns[i] > TLC_MAX_N)
      return fail(TLC_E_INVALID, "%s: tensor %zu: n = %zu too large", fn, i, ns[i]);
    if (!tensors[i] || (outs && !outs[i]))
      return fail(TLC_E_INVALID, "%s: tensor %zu: NULL pointer", fn, i);
    total += ns[i];
    const size_t bytes = ns[i] * type_bytes(types[i]);
    total_bytes += bytes;
    const bool in_place =
        clip && (!outs || ((const void*)outs[i] == tensors[i] && types[i] == TLC_F32));
    add_span(c->spans, tensors[i], bytes, in_place);
    if (clip && !in_place) add_span(c->spans, outs[i], ns[i] * 4, true);
  }
  if (total > kMaxListValues)
    return fail(TLC_E_INVALID, "%s: %zu values exceed %zu", fn, total, kMaxListValues);
  if (spans_conflict_cached(c->spans, c->spans_ok))
    return fail(TLC_E_INVALID, "%s: a written buffer overlaps another one", fn);
  l->own_type = clip && !outs;
  l->stream = total_bytes > kCacheBytes;
  l->len = (uint32_t)(std::max<size_t>(1, ceil_div(ceil_div(total, kNormBlocks), kPieceValues)) *
                      kPieceValues);
  if (count <= kArgTensors) {
    for (size_t i = 0; i < count; ++i) {
      if (ns[i] == 0) continue;
      ListTensor& e = l->tensors[l->count++];
      e.x = tensors[i];
      e.out = outs ? (void*)outs[i] : (void*)tensors[i];
      e.n = (uint32_t)ns[i];
      e.piece0_type = l->n | (uint32_t)types[i] << 30;
      l->n += (uint32_t)ceil_div(ns[i], l->len);
    }
    return TLC_OK;
  }
  st = take_slot(c, slot);
  if (st) return st;
  Piece* host = c->staging + (size_t)*slot * c->slot_pieces;
  l->pieces = c->staging_dev + (size_t)*slot * c->slot_pieces;
  for (size_t i = 0; i < count; ++i) {
    const size_t size = type_bytes(types[i]);
    for (size_t k = 0; k < ns[i]; k += l->len) {
      Piece& p = host[l->n++];
      p.x = (const uint8_t*)tensors[i] + k * size;
      p.out = outs ? (void*)(outs[i] + k) : (void*)p.x;
      p.n = (uint32_t)std::min<size_t>(l->len, ns[i] - k);
      p.type = (uint32_t)types[i];
    }
  }
  return TLC_OK;
}

// The staging slot is free again once the kernels queued so far have run.
int hold_slot(tlc_train* c, int slot) {
  if (slot < 0) return TLC_OK;
  const hipError_t e = hipEventRecord(c->slot_done[slot], c->stream);
  if (e != hipSuccess) return launched(c, e, "hipEventRecord(staging)");
  c->slot_used[slot] = true;
  return TLC_OK;
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
  // layout: partial sums | sorted tokens, twice | counts of the sort |
  //         touched rows | partial rows
  size_t off = round_up(kNormBlocks * sizeof(double), 256);
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
    e = hipHostMalloc((void**)&c->staging, kSlots * c->slot_pieces * sizeof(Piece),
                      hipHostMallocDefault);
  if (e == hipSuccess && c->staging)
    e = hipHostGetDevicePointer((void**)&c->staging_dev, c->staging, 0);
  for (int i = 0; i < kSlots && e == hipSuccess; ++i)
    e = hipEventCreateWithFlags(&c->slot_done[i], hipEventDisableTiming);
  if (e != hipSuccess) {
    tlc_train_destroy(c);
    return hip_fail(e, "tlc_train_create: workspace");
  }
  *c->bad = 0u;
  uint8_t* base = (uint8_t*)c->ws;
  c->partials = (double*)base;
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
  for (int i = 0; i < kSlots; ++i)
    if (c->slot_done[i]) (void)hipEventDestroy(c->slot_done[i]);
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
  const char* fn = "tlc_grad_norm";
  ListArgs l = {};
  int slot = -1;
  int st = cut_list(c, fn, count, tensors, types, ns, result, false, nullptr, &l, &slot);
  if (st) return st;
  DeviceScope dev(c->device);
  st = dev.status();
  if (st) return st;
  st = launched(c, launch_sumsq(l, c->partials, c->stream), fn);
  if (!st)
    st = launched(c, launch_norm_finish(c->partials, norm_blocks(l.n), result, c->stream), fn);
  return st ? st : hold_slot(c, slot);
}

TLC_API int tlc_clip(tlc_train* c, size_t count, const void* const* tensors, const int* types,
                     const size_t* ns, float max_norm, tlc_norm_result* result,
                     float* const* outs) {
  const char* fn = "tlc_clip";
  ListArgs l = {};
  int slot = -1;
  int st = check_clip(fn, max_norm);
  if (!st) st = cut_list(c, fn, count, tensors, types, ns, result, true, outs, &l, &slot);
  if (st) return st;
  DeviceScope dev(c->device);
  st = dev.status();
  if (st) return st;
  st = launched(c, launch_clip(l, nullptr, 0, max_norm, result, c->stream), fn);
  return st ? st : hold_slot(c, slot);
}

TLC_API int tlc_clip_grad_norm(tlc_train* c, size_t count, const void* const* tensors,
                               const int* types, const size_t* ns, float max_norm,
                               tlc_norm_result* result, float* const* outs) {
  const char* fn = "tlc_clip_grad_norm";
  ListArgs l = {};
  int slot = -1;
  int st = check_clip(fn, max_norm);
  if (!st) st = cut_list(c, fn, count, tensors, types, ns, result, true, outs, &l, &slot);
  if (st) return st;
  DeviceScope dev(c->device);
  st = dev.status();
  if (st) return st;
  st = launched(c, launch_sumsq(l, c->partials, c->stream), fn);
  if (!st)
    st = launched(c, launch_clip(l, c->partials, norm_blocks(l.n), max_norm, result, c->stream),
                  fn);
  return st ? st : hold_slot(c, slot);
}
