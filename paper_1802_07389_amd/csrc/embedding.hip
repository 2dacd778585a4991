// embedding.hip -- the lookup of embedding rows with scaling, and the gradient
// of the table.
#include "device_common.hpp"
#include "train_internal.h"
#include "typed_io.hpp"

namespace tlc {
namespace {

// A token's row, or -1 for an id outside the table.
template <class Id>
__device__ __forceinline__ int64_t token_row(const void* ids, uint32_t t, uint32_t rows) {
  const int64_t id = static_cast<const Id*>(ids)[t];
  return id >= 0 && id < (int64_t)rows ? id : -1;
}

}  // namespace

// One block per token.
template <class In, class Id, class Out>
__global__ __launch_bounds__(kEmbThreads) void tlc_embedding_kernel(EmbArgs a) {
  for (uint32_t t = blockIdx.x; t < a.count; t += gridDim.x) {
    const int64_t row = token_row<Id>(a.ids, t, a.rows);
    if (row < 0 && threadIdx.x == 0) host_put(a.bad, 1u);
    const In* x = static_cast<const In*>(a.x) + (row < 0 ? 0 : row) * a.x_stride;
    Out* out = static_cast<Out*>(a.out) + t * a.out_stride;
    for (uint32_t k = threadIdx.x; k < a.dim; k += kEmbThreads)
      out[k] = row < 0 ? (Out)0.0f : round_to<Out>(a.scale * (float)x[k]);
  }
}

// Rows without a token: zeros everywhere, before the sums are written.
__global__ __launch_bounds__(kEmbThreads) void tlc_embedding_grad_fill_kernel(EmbArgs a) {
  float* out = static_cast<float*>(a.out);
  for (uint32_t v = blockIdx.x; v < a.rows; v += gridDim.x)
    for (uint32_t k = threadIdx.x; k < a.dim; k += kEmbThreads) out[v * a.out_stride + k] = 0.0f;
}

// One wave per token: the wave of an id's first token adds up all of its
// tokens' rows, found 64 ids at a time.
template <class In, class Id>
__global__ __launch_bounds__(kEmbThreads) void tlc_embedding_grad_kernel(EmbArgs a,
                                                                         bool accumulate) {
  const uint32_t lane = threadIdx.x & 63u;
  const Id* ids = static_cast<const Id*>(a.ids);
  const In* x = static_cast<const In*>(a.x);
  const uint32_t waves = gridDim.x * (kEmbThreads / 64);
  for (uint32_t t = blockIdx.x * (kEmbThreads / 64) + (threadIdx.x >> 6); t < a.count;
       t += waves) {
    const int64_t id = ids[t];
    if (id == a.padding && id >= 0) continue;
    if (id < 0 || id >= (int64_t)a.rows) {
      if (lane == 0) host_put(a.bad, 1u);
      continue;
    }
    bool first = true;
    for (uint32_t b = 0; b < t && first; b += 64)
      first = __ballot(b + lane < t && ids[b + lane] == id) == 0;
    if (!first) continue;
    float* out = static_cast<float*>(a.out) + (uint64_t)id * a.out_stride;
    for (uint32_t k0 = 0; k0 < a.dim; k0 += 64) {
      const uint32_t k = k0 + lane;
      float sum = 0.0f;
      for (uint32_t b = t & ~63u; b < a.count; b += 64) {
        uint64_t m = __ballot(b + lane < a.count && ids[b + lane] == id);
        for (; m; m &= m - 1) {
          const uint32_t u = b + (uint32_t)__builtin_ctzll(m);
          if (k < a.dim) sum += (float)x[u * a.x_stride + k];
        }
      }
      if (k < a.dim) out[k] = accumulate ? out[k] + a.scale * sum : a.scale * sum;
    }
  }
}

namespace {

template <class In, class Id>
hipError_t embedding_out(const EmbArgs& a, int out_type, uint32_t grid, hipStream_t st) {
  switch (out_type) {
    case TLC_F32:
      launch_k(tlc_embedding_kernel<In, Id, float>, grid, kEmbThreads, st, a);
      break;
    case TLC_BF16:
      launch_k(tlc_embedding_kernel<In, Id, bf16_t>, grid, kEmbThreads, st, a);
      break;
    default:
      launch_k(tlc_embedding_kernel<In, Id, f16_t>, grid, kEmbThreads, st, a);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_embedding(const EmbArgs& a, int table_type, int ids_type, int out_type,
                            hipStream_t st) {
  const uint32_t grid = std::min(a.count, 1u << 20);
  return with_type(table_type, [&](auto in) {
    using In = decltype(in);
    return ids_type == TLC_I64 ? embedding_out<In, int64_t>(a, out_type, grid, st)
                               : embedding_out<In, int32_t>(a, out_type, grid, st);
  });
}

hipError_t launch_embedding_grad(const EmbArgs& a, int grad_type, int ids_type, bool accumulate,
                                 hipStream_t st) {
  if (!accumulate) {
    launch_k(tlc_embedding_grad_fill_kernel, std::min(a.rows, 1u << 14), kEmbThreads, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.count == 0) return hipSuccess;
  const uint32_t grid = std::min((a.count + 3) / 4, 1u << 20);
  return with_type(grad_type, [&](auto in) {
    using In = decltype(in);
    if (ids_type == TLC_I64)
      launch_k(tlc_embedding_grad_kernel<In, int64_t>, grid, kEmbThreads, st, a, accumulate);
    else
      launch_k(tlc_embedding_grad_kernel<In, int32_t>, grid, kEmbThreads, st, a, accumulate);
    return hipGetLastError();
  });
}

}  // namespace tlc
