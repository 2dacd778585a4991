// norm.hip -- the global norm of a list of tensors, and their clipping.
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

struct Clip {
  float norm, coef;
  bool finite;
};
__device__ __forceinline__ Clip clip_of(double sumsq, float max_norm) {
  const double norm = sqrt(sumsq);
  Clip c;
  c.finite = sumsq <= DBL_MAX;  // false for NaN too
  c.norm = (float)norm;
  c.coef = !c.finite ? __builtin_nanf("")
                     : (norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.0f);
  return c;
}

__device__ __forceinline__ void put_result(tlc_norm_result* r, double sumsq, Clip c) {
  r->sumsq = sumsq;
  r->norm = c.norm;
  r->coef = c.coef;
  r->status = c.finite ? TLC_OK : TLC_E_NONFINITE;
  r->reserved = 0u;
}

template <class T>
__device__ __forceinline__ double piece_sumsq(const Piece& p) {
  const T* x = static_cast<const T*>(p.x);
  double v = 0.0;
  for (uint32_t i = threadIdx.x; i < p.n; i += kNormThreads) {
    const double d = (double)(float)x[i];
    v += d * d;
  }
  return v;
}

template <class T, class Out>
__device__ __forceinline__ void piece_scale(const Piece& p, float coef) {
  const T* x = static_cast<const T*>(p.x);
  Out* out = static_cast<Out*>(p.out);
  for (uint32_t i = threadIdx.x; i < p.n; i += kNormThreads) out[i] = round_to<Out>(coef * (float)x[i]);
}

}  // namespace

__global__ __launch_bounds__(kNormThreads) void tlc_sumsq_kernel(const Piece* __restrict__ pieces,
                                                                 uint32_t n,
                                                                 double* __restrict__ partials) {
  __shared__ double lds[kWaves];
  const uint32_t p0 = (uint32_t)((uint64_t)blockIdx.x * n / gridDim.x);
  const uint32_t p1 = (uint32_t)((uint64_t)(blockIdx.x + 1) * n / gridDim.x);
  double v = 0.0;
  for (uint32_t i = p0; i < p1; ++i) {
    const Piece p = pieces[i];
    if (p.type == TLC_F32)
      v += piece_sumsq<float>(p);
    else if (p.type == TLC_BF16)
      v += piece_sumsq<bf16_t>(p);
    else
      v += piece_sumsq<f16_t>(p);
  }
  v = block_sum(v, lds);
  if (threadIdx.x == 0) partials[blockIdx.x] = v;
}

__global__ __launch_bounds__(kNormThreads) void tlc_norm_finish_kernel(
    const double* __restrict__ partials, uint32_t np, tlc_norm_result* __restrict__ result) {
  __shared__ double lds[kWaves];
  const double sumsq = sum_partials(partials, np, lds);
  if (threadIdx.x == 0) put_result(result, sumsq, clip_of(sumsq, INFINITY));
}

__global__ __launch_bounds__(kNormThreads) void tlc_clip_kernel(
    const Piece* __restrict__ pieces, uint32_t n, const double* __restrict__ partials, uint32_t np,
    float max_norm, bool own_type, tlc_norm_result* __restrict__ result) {
  __shared__ double lds[kWaves];
  // sumsq is read by every block; block 0 writes it back as it is
  const double sumsq = partials ? sum_partials(partials, np, lds) : result->sumsq;
  const Clip c = clip_of(sumsq, max_norm);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (partials) {
      put_result(result, sumsq, c);
    } else {
      result->norm = c.norm;
      result->coef = c.coef;
      result->status = c.finite ? TLC_OK : TLC_E_NONFINITE;
      result->reserved = 0u;
    }
  }
  if (!c.finite || (own_type && c.coef == 1.0f)) return;
  const uint32_t p0 = (uint32_t)((uint64_t)blockIdx.x * n / gridDim.x);
  const uint32_t p1 = (uint32_t)((uint64_t)(blockIdx.x + 1) * n / gridDim.x);
  for (uint32_t i = p0; i < p1; ++i) {
    const Piece p = pieces[i];
    if (p.type == TLC_F32)
      piece_scale<float, float>(p, c.coef);
    else if (p.type == TLC_BF16)
      own_type ? piece_scale<bf16_t, bf16_t>(p, c.coef) : piece_scale<bf16_t, float>(p, c.coef);
    else
      own_type ? piece_scale<f16_t, f16_t>(p, c.coef) : piece_scale<f16_t, float>(p, c.coef);
  }
}

hipError_t launch_sumsq(const Piece* pieces, uint32_t n, double* partials, hipStream_t st) {
  if (n) launch_k(tlc_sumsq_kernel, norm_blocks(n), kNormThreads, st, pieces, n, partials);
  return hipGetLastError();
}

hipError_t launch_norm_finish(const double* partials, uint32_t np, tlc_norm_result* result,
                              hipStream_t st) {
  launch_k(tlc_norm_finish_kernel, 1, kNormThreads, st, partials, np, result);
  return hipGetLastError();
}

hipError_t launch_clip(const Piece* pieces, uint32_t n, const double* partials, uint32_t np,
                       float max_norm, bool own_type, tlc_norm_result* result, hipStream_t st) {
  launch_k(tlc_clip_kernel, std::max(1u, norm_blocks(n)), kNormThreads, st, pieces, n, partials,
           np, max_norm, own_type, result);
  return hipGetLastError();
}

}  // namespace tlc
