// embedding.hip -- the lookup of embedding rows with scaling:
//   out[t, :] = round(scale * table[ids[t], :])
// What bounds it: the rows read (common ones from the caches) and out written
// once.  65536 tokens of 2048 bf16 values from 131072 rows take 75 us (268 MB
// written, about 88 MB of distinct rows: 4.8 TB/s, a large copy's rate), a few
// tokens one launch.
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

// One pass over the output in packs of V values, kUnits of a thread 256 packs
// apart: the ids of all of them are asked for first, then their rows, then the
// products stored, streaming, so that rows asked for again keep the caches (65536
// tokens of 1024 fp32 values: 78 us, without the hint 89; of 2048 bf16 values with
// one pack a thread 82, two 75, four 77, eight 80; a block per token, value by
// value, 194; 2 to 32 MB looked up and read by the next kernel take the same with
// and without the hint).  A row that is no whole number of packs ends with a pack
// moved back to end with it (its values are written twice, alike).
template <class In, class Id, class Out, int V, int kUnits>
__global__ __launch_bounds__(kEmbThreads) void tlc_embedding_kernel(EmbArgs a, Divider packs,
                                                                    uint32_t slice) {
  const uint32_t t0 = blockIdx.y * slice;
  const uint32_t units = umin32(slice, a.count - t0) * packs.d;  // below 2^31
  const uint32_t u0 = blockIdx.x * (kEmbThreads * kUnits) + threadIdx.x;
  uint32_t t[kUnits], k[kUnits];
  int64_t row[kUnits];
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const uint32_t u = u0 + i * kEmbThreads;
    t[i] = quotient(umin32(u, units - 1), packs);
    k[i] = umin32((umin32(u, units - 1) - t[i] * packs.d) * V, a.dim - V);
    t[i] += t0;
    row[i] = token_row<Id>(a.ids, t[i], a.rows);
  }
  Pack<In, V> x[kUnits];
#pragma unroll
  for (int i = 0; i < kUnits; ++i)
    x[i] = load_pack<In, V>(static_cast<const In*>(a.x) + (row[i] < 0 ? 0 : row[i]) * a.x_stride +
                            k[i]);
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    if (u0 + i * kEmbThreads >= units) break;
    Pack<Out, V> o;
#pragma unroll
    for (int e = 0; e < V; ++e) o.set(e, row[i] < 0 ? 0.0f : a.scale * x[i].get(e));
    store_pack<Out, V, true>(static_cast<Out*>(a.out) + t[i] * a.out_stride + k[i], o);
    if (row[i] < 0 && k[i] == 0) host_put(a.bad, 1u);
  }
}

namespace {

template <class In, class Id, class Out, int V>
hipError_t embedding_packs(const EmbArgs& a, hipStream_t st) {
  const uint32_t packs = (a.dim + V - 1) / V;
  const uint32_t slice = std::min(a.count, (uint32_t)((1u << 31) - 1) / packs);
  const uint32_t slices = (a.count + slice - 1) / slice;
  const uint32_t units = slice * packs;
  constexpr int kUnits = 2;
  // A call that two packs a thread leave without a block for every CU takes
  // one each.
  if ((units + kEmbThreads * kUnits - 1) / (kEmbThreads * kUnits) < kCus) {
    launch_k(tlc_embedding_kernel<In, Id, Out, V, 1>,
             dim3((units + kEmbThreads - 1) / kEmbThreads, slices), kEmbThreads, st, a,
             divider(packs), slice);
  } else {
    launch_k(tlc_embedding_kernel<In, Id, Out, V, kUnits>,
             dim3((units + kEmbThreads * kUnits - 1) / (kEmbThreads * kUnits), slices),
             kEmbThreads, st, a, divider(packs), slice);
  }
  return hipGetLastError();
}

// 16 bytes of the output a pack, so that a wave's stores fill whole lines (bf16
// rows to fp32 in packs of eight, two stores a lane: 162 instead of 145 us for
// 65536 tokens of 2048); rows shorter than a pack, value by value.
template <class In, class Id, class Out>
hipError_t embedding_rows(const EmbArgs& a, hipStream_t st) {
  constexpr int V = 16 / sizeof(Out);
  return a.dim >= V ? embedding_packs<In, Id, Out, V>(a, st)
                    : embedding_packs<In, Id, Out, 1>(a, st);
}

}  // namespace

hipError_t launch_embedding(const EmbArgs& a, int table_type, int ids_type, int out_type,
                            hipStream_t st) {
  return with_type(table_type, [&](auto in) {
    return with_type(out_type, [&](auto out) {
      using In = decltype(in);
      using Out = decltype(out);
      return ids_type == TLC_I64 ? embedding_rows<In, int64_t, Out>(a, st)
                                 : embedding_rows<In, int32_t, Out>(a, st);
    });
  });
}

}  // namespace tlc
