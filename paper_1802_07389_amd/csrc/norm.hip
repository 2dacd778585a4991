// norm.hip -- the global norm of a list of tensors, and their clipping.
//
//   sumsq = sum x^2,  norm = sqrt(sumsq),  coef = norm > max ? max / norm : 1,  out = coef * x
//
// What bounds it: the values read once for the norm, and once more to be clipped,
// for which the last-level cache keeps what it can.  Squares and sums are in 64
// bits: the conversions and multiply-adds hide behind the loads (2^28 fp32 values
// in 159 us, 6.7 TB/s; with fp32 sums as fast, 480M bf16 values 150 against 144),
// no value overflows, and the order of the sums is fixed by the sizes (another one
// changes the last of 53 bits, so seldom the norm's 24).  A partial sum a block and a second launch that adds
// them: letting the block that is done last do so costs every block a fence and
// an addition to one word (2^28 values 247 us, 25M 113 against 20).
#include <type_traits>

#include "device_common.hpp"
#include "train_internal.h"
#include "typed_io.hpp"

namespace tlc {
namespace {

// Block-wide sum in a fixed order; every thread gets it.  Uses lds[kWaves]
// and one barrier; callers that use lds again barrier first.
__device__ __forceinline__ double block_sum(double v, double* lds) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63u) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  double r = lds[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) r += lds[w];
  return r;
}

__device__ __forceinline__ double sum_partials(const double* partials, uint32_t np, double* lds) {
  double v = 0.0;
  for (uint32_t i = threadIdx.x; i < np; i += kNormThreads) v += partials[i];
  return block_sum(v, lds);
}

// Piece p of a list.
__device__ __forceinline__ Piece piece_of(const PinnedList& list, uint32_t p) {
  return list.pieces[p];
}
__device__ __forceinline__ Piece piece_of(const ArgList& list, uint32_t p) {
  const uint32_t lane = threadIdx.x & 63u;
  uint32_t t = 0;  // tensors whose first piece is at most p
  for (uint32_t c = 0; c < list.count; c += 64)
    t += (uint32_t)__popcll(__ballot(
        c + lane < list.count && (list.tensors[c + lane].piece0_type & 0x3fffffffu) <= p));
  const ListTensor& e = list.tensors[uniform32(t) - 1];
  const uint64_t first = (uint64_t)(p - (e.piece0_type & 0x3fffffffu)) * list.len;
  Piece r;
  r.type = e.piece0_type >> 30;
  const uint32_t size = r.type == TLC_F32 ? 4 : 2;
  r.x = static_cast<const uint8_t*>(e.x) + first * size;
  r.out = static_cast<uint8_t*>(e.out) + first * (list.own_type ? size : 4);
  r.n = (uint32_t)umin64(list.len, e.n - first);
  return r;
}

// What the norm leaves for the clipping that follows it in the same call.
__device__ __forceinline__ void keep_piece(const PinnedList& list, uint32_t i, const Piece& p) {
  if (list.copy && threadIdx.x == 0) list.copy[i] = p;
}
__device__ __forceinline__ void keep_piece(const ArgList&, uint32_t, const Piece&) {}

constexpr uint32_t kUnits = 8;  // packs of a thread in flight

// kStream: nothing of the list is read again.
template <class T, bool kStream>
__device__ __forceinline__ double piece_sumsq(const Piece& p) {
  constexpr int V = 16 / sizeof(T);
  const T* x = static_cast<const T*>(p.x);
  const uint32_t packs = p.n / V;
  double v[4] = {0.0, 0.0, 0.0, 0.0};
  for (uint32_t u0 = threadIdx.x; u0 < packs; u0 += kNormThreads * kUnits) {
    Pack<T, V> r[kUnits];
#pragma unroll
    for (uint32_t i = 0; i < kUnits; ++i) {
      const uint32_t u = u0 + i * kNormThreads;
      r[i] = load_pack<T, V, kStream>(x + umin32(u, packs - 1) * V);
      if (u >= packs) r[i] = {};
    }
#pragma unroll
    for (uint32_t i = 0; i < kUnits; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const double d = (double)r[i].get(e);
        v[e & 3] = __builtin_fma(d, d, v[e & 3]);
      }
  }
  if (threadIdx.x < p.n - packs * V) {
    const double d = (double)(float)x[packs * V + threadIdx.x];
    v[0] = __builtin_fma(d, d, v[0]);
  }
  return (v[0] + v[1]) + (v[2] + v[3]);
}

// The second read of the values, from the piece's end: what the first one left
// in the last-level cache is its ends.  This call reads and writes nothing again
// after it, and its accesses say so (100M fp32 values: 236 us with both reads
// hinted, 249 with neither, 203 with this one alone).  The encode that reads the
// clipped values next does not pay for the stores' hint: bf16 values clipped and
// encoded, hinted | not, 1M 34 | 34 us, 16M 103 | 107, 40M 229 | 230, 100M 482 | 501.
template <class T, class Out>
__device__ __forceinline__ void piece_scale(const Piece& p, float coef) {
  // 16 bytes of what is stored: a wave's stores fill whole lines
  constexpr int V = 16 / sizeof(Out);
  const T* x = static_cast<const T*>(p.x);
  Out* out = static_cast<Out*>(p.out);
  const uint32_t packs = p.n / V;
  constexpr uint32_t kStep = kNormThreads * kUnits;
  for (uint32_t c = (packs + kStep - 1) / kStep; c-- > 0;) {
    const uint32_t u0 = c * kStep + threadIdx.x;
    Pack<T, V> r[kUnits];
#pragma unroll
    for (uint32_t i = 0; i < kUnits; ++i)
      r[i] = load_pack<T, V, true>(x + umin32(u0 + i * kNormThreads, packs - 1) * V);
#pragma unroll
    for (uint32_t i = 0; i < kUnits; ++i) {
      const uint32_t u = u0 + i * kNormThreads;
      if (u >= packs) break;
      Pack<Out, V> o;
#pragma unroll
      for (int e = 0; e < V; ++e) o.set(e, coef * r[i].get(e));
      store_pack<Out, V, true>(out + u * V, o);
    }
  }
  if (threadIdx.x < p.n - packs * V) {
    const uint32_t i = packs * V + threadIdx.x;
    out[i] = round_to<Out>(coef * (float)x[i]);
  }
}

}  // namespace

// Partial sums of squares, eight packs of 16 bytes a thread in flight.
template <class List, bool kStream>
__global__ __launch_bounds__(kNormThreads) void tlc_sumsq_kernel(List list,
                                                                 double* __restrict__ partials) {
  __shared__ double lds[kWaves];
  const uint32_t p0 = (uint32_t)((uint64_t)blockIdx.x * list.n / gridDim.x);
  const uint32_t p1 = (uint32_t)((uint64_t)(blockIdx.x + 1) * list.n / gridDim.x);
  double v = 0.0;
  for (uint32_t i = p0; i < p1; ++i) {
    const Piece p = piece_of(list, i);
    keep_piece(list, i, p);
    if (p.type == TLC_F32)
      v += piece_sumsq<float, kStream>(p);
    else if (p.type == TLC_BF16)
      v += piece_sumsq<bf16_t, kStream>(p);
    else
      v += piece_sumsq<f16_t, kStream>(p);
  }
  v = block_sum(v, lds);
  if (threadIdx.x == 0) partials[blockIdx.x] = v;
}

__global__ __launch_bounds__(kNormThreads) void tlc_norm_finish_kernel(
    const double* __restrict__ partials, uint32_t np, tlc_norm_result* __restrict__ result) {
  __shared__ double lds[kWaves];
  const double sumsq = sum_partials(partials, np, lds);
  if (threadIdx.x != 0) return;
  result->sumsq = sumsq;
  put_result(result, clip_of(sumsq, INFINITY));
}

// The clipped tensors.  Out: float, or void: the tensors' own types.  100M bf16
// values to fp32: 161 us with the norm (200 MB read twice, 400 MB written); 335
// tensors of 1.7M values in all 13 us, of which two launches and a read of the
// pieces over the bus are most.
template <class List, class Out>
__global__ __launch_bounds__(kNormThreads) void tlc_clip_kernel(
    List list, const double* __restrict__ partials, uint32_t np, float max_norm,
    tlc_norm_result* __restrict__ result) {
  constexpr bool kOwn = __is_same(Out, void);
  __shared__ double lds[kWaves];
  const uint32_t p0 = (uint32_t)((uint64_t)blockIdx.x * list.n / gridDim.x);
  const uint32_t p1 = (uint32_t)((uint64_t)(blockIdx.x + 1) * list.n / gridDim.x);
  // asked for before the sums are there: it may be in host memory
  Piece p = {};
  if (p0 < p1) p = piece_of(list, p0);
  // sumsq is read by every block; the first one writes the rest
  const double sumsq = partials ? sum_partials(partials, np, lds) : result->sumsq;
  const Clip c = clip_of(sumsq, max_norm);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (partials) result->sumsq = sumsq;
    put_result(result, c);
  }
  if (!c.finite || (kOwn && c.coef == 1.0f)) return;
  for (uint32_t i = p0; i < p1; ++i) {
    if (i > p0) p = piece_of(list, i);
    if (p.type == TLC_F32)
      piece_scale<float, float>(p, c.coef);
    else if (p.type == TLC_BF16)
      piece_scale<bf16_t, std::conditional_t<kOwn, bf16_t, float>>(p, c.coef);
    else
      piece_scale<f16_t, std::conditional_t<kOwn, f16_t, float>>(p, c.coef);
  }
}

template <class List>
hipError_t launch_sumsq(const List& list, bool read_once, double* partials, hipStream_t st) {
  if (list.n == 0) return hipSuccess;
  if (read_once)
    launch_k(tlc_sumsq_kernel<List, true>, norm_blocks(list.n), kNormThreads, st, list, partials);
  else
    launch_k(tlc_sumsq_kernel<List, false>, norm_blocks(list.n), kNormThreads, st, list, partials);
  return hipGetLastError();
}

hipError_t launch_norm_finish(const double* partials, uint32_t np, tlc_norm_result* result,
                              hipStream_t st) {
  launch_k(tlc_norm_finish_kernel, 1, kNormThreads, st, partials, np, result);
  return hipGetLastError();
}

namespace {

template <class Out, class List>
void launch_clip_to(const List& list, const double* partials, uint32_t np, float max_norm,
                    tlc_norm_result* result, hipStream_t st) {
  const uint32_t grid = std::max(1u, norm_blocks(list.n));
  launch_k(tlc_clip_kernel<List, Out>, grid, kNormThreads, st, list, partials, np, max_norm,
           result);
}

}  // namespace

template <class List>
hipError_t launch_clip(const List& list, const double* partials, uint32_t np, float max_norm,
                       tlc_norm_result* result, hipStream_t st) {
  if (list.own_type)
    launch_clip_to<void>(list, partials, np, max_norm, result, st);
  else
    launch_clip_to<float>(list, partials, np, max_norm, result, st);
  return hipGetLastError();
}

template hipError_t launch_sumsq(const PinnedList&, bool, double*, hipStream_t);
template hipError_t launch_sumsq(const ArgList&, bool, double*, hipStream_t);
template hipError_t launch_clip(const PinnedList&, const double*, uint32_t, float,
                                tlc_norm_result*, hipStream_t);
template hipError_t launch_clip(const ArgList&, const double*, uint32_t, float, tlc_norm_result*,
                                hipStream_t);

}  // namespace tlc
