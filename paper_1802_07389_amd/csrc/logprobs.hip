// logprobs.hip -- log probabilities of given tokens with entropy and the most
// likely alternatives, and their gradient.  Of a row of logits x, scale s, target t:
//   m = max x,  l = ln sum exp(s (x - m)),  logprob = s (x_t - m) - l
//   H = l - sum p s (x - m),  p = exp(s (x - m) - l)
//   dx_j = s (a (1[j = t] - p_j) - b p_j (ln p_j + H))   of their gradients a, b
// What bounds it: the logits read once (and, for the gradient, its values written
// once).
#include <float.h>
#include <math.h>

#include "device_common.hpp"
#include "train_internal.h"
#include "typed_io.hpp"

namespace tlc {
namespace {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
// Exponents are clamped here where they multiply a probability of 0: a logit of
// -inf adds 0 * kFar and not 0 * -inf.
constexpr float kFar = -1e30f;

// A row's target: its column, kNoTarget where the call has none, kLeftOut where
// it is the ignored id or outside the vocabulary.
constexpr int64_t kNoTarget = -1, kLeftOut = -2;
__device__ __forceinline__ int64_t target_of(const LogitArgs& a, uint32_t row, bool report) {
  if (!a.targets) return kNoTarget;
  const int64_t id = a.wide_ids ? static_cast<const int64_t*>(a.targets)[row]
                                : static_cast<const int32_t*>(a.targets)[row];
  if (id == a.ignore) return kLeftOut;
  if (id >= 0 && id < (int64_t)a.vocab) return id;
  if (report) host_put(a.bad, 1u);
  return kLeftOut;
}

// Sums of a part of a row, by its largest logit m (-FLT_MAX where there is none
// above it, so that differences of -inf do not arise): s0 = sum e, s1 = sum e t with
// t = (x - m) c, e = 2^t, c = s log2(e).  NaN and +inf make s0 NaN.
__device__ __forceinline__ float exp2_of(float t) { return __builtin_amdgcn_exp2f(t); }
__device__ __forceinline__ LogitPart rebased(LogitPart p, float m, float c) {
  const float d = fmaxf((p.m - m) * c, kFar), f = exp2_of(d);
  return LogitPart{m, f * p.s0, f * (p.s1 + d * p.s0)};
}
__device__ __forceinline__ LogitPart merged(LogitPart a, LogitPart b, float c) {
  const float m = fmaxf(a.m, b.m);
  a = rebased(a, m, c);
  b = rebased(b, m, c);
  return LogitPart{m, a.s0 + b.s0, a.s1 + b.s1};
}

constexpr int kLogWaves = kLogThreads / 64;

// Of a whole block, the same in every thread.  Uses lds[kLogWaves] and one
// barrier.
__device__ __forceinline__ LogitPart block_merged(LogitPart p, float c, LogitPart* lds) {
  float m = p.m;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  p = rebased(p, m, c);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    p.s0 += __shfl_xor(p.s0, d);
    p.s1 += __shfl_xor(p.s1, d);
  }
  if ((threadIdx.x & 63u) == 0) lds[threadIdx.x >> 6] = p;
  __syncthreads();
  LogitPart r = lds[0];
#pragma unroll
  for (int w = 1; w < kLogWaves; ++w) r = merged(r, lds[w], c);
  return r;
}

// Packs of V neighbouring columns; the last one of a row that is no whole number
// of them is moved back to end with it, and its first `skip` columns are not its
// own.
template <class T, int V>
struct RowPacks {
  const T* x;
  uint32_t vocab;
  __device__ __forceinline__ uint32_t start(uint32_t p) const {
    return umin32(p * V, vocab - V);
  }
  // Pack p with the columns that are not its own set to -inf; all of them where
  // p >= end.
  __device__ __forceinline__ Pack<T, V> load(uint32_t p, uint32_t end) const {
    const uint32_t q = umin32(p, end - 1), k = start(q);
    Pack<T, V> r = load_pack<T, V>(x + k);
    const uint32_t skip = p < end ? q * V - k : V;
#pragma unroll
    for (int e = 0; e < V; ++e)
      if ((uint32_t)e < skip) r.set(e, -INFINITY);
    return r;
  }
};

// Logits in their order as whole numbers (no NaN; both zeroes alike), above the
// column's complement: keys are unique, and the lowest of equal logits is first.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t column) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  const uint32_t order = (u >> 31) ? ~u : u | 0x80000000u;
  return ((uint64_t)order << 32) | (uint32_t)~column;
}
__device__ __forceinline__ float key_logit(uint64_t key) {
  const uint32_t order = (uint32_t)(key >> 32);
  return __uint_as_float((order >> 31) ? order & 0x7fffffffu : ~order);
}

// The block's selection of the largest keys.
constexpr uint32_t kFewKeys = kLogThreads;
struct TopLds {
  uint64_t keys[kLogThreads];
  uint64_t found[kFewKeys + kLogThreads * 8];
  uint64_t best[TLC_MAX_TOP];
  uint64_t least;  // found keys below it are not among the largest
  uint32_t from[TLC_MAX_TOP];
  uint32_t count;
};

// How many of keys[0, n) are above `key`.
__device__ __forceinline__ uint32_t rank_of(const uint64_t* keys, uint32_t n, uint64_t key) {
  uint32_t r = 0;
  for (uint32_t j = 0; j < n; ++j) r += keys[j] > key;
  return r;
}

__device__ __forceinline__ void put_key(TopLds& l, uint64_t key) {
  if (key >= l.least) l.found[atomicAdd(&l.count, 1u)] = key;
}

// best: the `top` largest of the found keys, in order; they stay as the found
// ones.  All threads; begins after a barrier and ends with one.
__device__ __forceinline__ void keep_best(TopLds& l, uint32_t n, uint32_t top) {
  for (uint32_t j = threadIdx.x; j < n; j += kLogThreads) {
    const uint64_t key = l.found[j];
    const uint32_t r = rank_of(l.found, n, key);
    if (r < top) l.best[r] = key;
  }
  __syncthreads();
  const uint32_t kept = umin32(n, top);
  if (threadIdx.x < kept) l.found[threadIdx.x] = l.best[threadIdx.x];
  if (threadIdx.x == 0) {
    l.count = kept;
    if (n >= top) l.least = l.best[top - 1];
  }
  __syncthreads();
}

// After a round that adds at most eight keys a thread.
__device__ __forceinline__ void end_round(TopLds& l, uint32_t top) {
  __syncthreads();
  const uint32_t n = l.count;
  __syncthreads();
  if (n > kFewKeys) keep_best(l, n, top);
}

// The row's statistics from the merged sums.
__device__ __forceinline__ tlc_token_result result_of(LogitPart p, float scale, bool has_target,
                                                      float x) {
  tlc_token_result r;
  if (!(p.s0 >= 0.0f)) {  // NaN or +inf among the logits
    r.logprob = r.entropy = r.max = r.log_sum = __builtin_nanf("");
  } else if (p.s0 == 0.0f) {  // nothing above -inf
    r.logprob = has_target ? -INFINITY : 0.0f;
    r.entropy = 0.0f;
    r.max = r.log_sum = -INFINITY;
  } else {
    r.max = p.m;
    r.log_sum = logf(p.s0);
    r.entropy = fmaxf(r.log_sum - kLn2 * (p.s1 / p.s0), 0.0f);
    r.logprob = has_target ? (x - p.m) * scale - r.log_sum : 0.0f;
  }
  return r;
}

// What a row gets that is left out.
__device__ __forceinline__ void put_left_out(const TokenArgs& a, uint32_t row) {
  if (threadIdx.x == 0) a.results[row] = tlc_token_result{0.0f, 0.0f, 0.0f, 0.0f};
  if (threadIdx.x < a.top) {
    a.top_logprobs[(uint64_t)row * a.top + threadIdx.x] = 0.0f;
    a.top_ids[(uint64_t)row * a.top + threadIdx.x] = -1;
  }
}

__device__ __forceinline__ void put_top(const TokenArgs& a, uint32_t row, const uint64_t* best,
                                        const tlc_token_result& r) {
  if (threadIdx.x >= a.top) return;
  const uint64_t at = (uint64_t)row * a.top + threadIdx.x;
  if (r.max != r.max) {
    a.top_logprobs[at] = r.max;
    a.top_ids[at] = -1;
    return;
  }
  const uint64_t key = best[threadIdx.x];
  a.top_logprobs[at] =
      r.max == -INFINITY ? -INFINITY : (key_logit(key) - r.max) * a.scale - r.log_sum;
  a.top_ids[at] = (int32_t)~(uint32_t)key;
}

constexpr uint32_t kLogUnits = 4;  // packs of a thread in flight
constexpr uint32_t kLogChunk = kLogThreads * kLogUnits;

struct Lane {
  LogitPart p;
  float best;      // largest logit of the thread, and the chunk that had it first
  uint32_t chunk;
};

template <class T, int V, bool kTop>
__device__ __forceinline__ void add_chunk(Lane& l, const Pack<T, V> (&r)[kLogUnits], float c,
                                          uint32_t chunk) {
  float mx = r[0].get(0);
#pragma unroll
  for (uint32_t u = 0; u < kLogUnits; ++u)
#pragma unroll
    for (int e = 0; e < V; ++e) mx = fmaxf(mx, r[u].get(e));
  if (kTop && mx > l.best) {
    l.best = mx;
    l.chunk = chunk;
  }
  l.p = rebased(l.p, fmaxf(l.p.m, mx), c);
#pragma unroll
  for (uint32_t u = 0; u < kLogUnits; ++u)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float t = (r[u].get(e) - l.p.m) * c, w = exp2_of(t);
      l.p.s0 += w;
      l.p.s1 = __builtin_fmaf(w, fmaxf(t, kFar), l.p.s1);
    }
}

// The `top` largest keys of packs [p0, p0 + n) into lds.best (fewer where there
// are fewer columns: lds.count).  A thread's columns hold one of them only if the
// thread's largest is among the `top` largest of all threads', so that `top` threads'
// columns are read again, and of them the keys from the least of those on are
// ranked.
template <class T, int V>
__device__ __forceinline__ void select_top(const RowPacks<T, V>& row, uint32_t p0, uint32_t n,
                                           const Lane& l, uint32_t top, TopLds& lds) {
  const uint32_t tid = threadIdx.x, end = p0 + n;
  uint64_t key = 0;
  if (tid < n) {
    uint32_t at = ~0u;
#pragma unroll
    for (uint32_t u = kLogUnits; u-- > 0;) {
      const uint32_t p = p0 + l.chunk * kLogChunk + u * kLogThreads + tid;
      const Pack<T, V> r = row.load(p, end);
      const uint32_t k = row.start(umin32(p, end - 1));
#pragma unroll
      for (int e = V - 1; e >= 0; --e)
        if (p < end && k + e >= p * V && r.get(e) == l.best) at = k + e;
    }
    key = key_of(l.best, at);
  }
  lds.keys[tid] = key;
  if (tid == 0) {
    lds.count = 0;
    lds.least = 0;
  }
  __syncthreads();
  const uint32_t threads = umin32(umin32(n, kLogThreads), top);
  const uint32_t r = rank_of(lds.keys, kLogThreads, key);
  if (key != 0 && r < threads) {
    lds.from[r] = tid;
    if (r == top - 1) lds.least = key;
  }
  __syncthreads();
  const uint32_t each = (n + kLogThreads - 1) / kLogThreads;  // packs of a thread
  for (uint32_t w0 = 0; w0 < threads * each; w0 += kLogThreads) {
    const uint32_t w = w0 + tid, s = w / each;
    const uint32_t i = s < threads ? lds.from[s] + (w - s * each) * kLogThreads : n;
    if (i < n) {
      const uint32_t p = p0 + i, k = row.start(p);
      const Pack<T, V> x = load_pack<T, V>(row.x + k);
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (k + e >= p * V) put_key(lds, key_of(x.get(e), k + e));
    }
    end_round(lds, top);
  }
  keep_best(lds, lds.count, top);
}

}  // namespace

// A block reads a row, or one of `parts` parts of it, whose sums and keys
// tlc_token_join_kernel puts together.
template <class T, int V, bool kTop>
__global__ __launch_bounds__(kLogThreads) void tlc_token_logprobs_kernel(TokenArgs a) {
  __shared__ LogitPart sums[kLogWaves];
  __shared__ TopLds lds;
  const uint32_t packs = (a.vocab + V - 1) / V, full = a.vocab / V;
  const float c = a.scale * kLog2e;
  const uint64_t blocks = (uint64_t)a.count * a.parts;
  for (uint64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
    const uint32_t row = (uint32_t)(b / a.parts), part = (uint32_t)(b - (uint64_t)row * a.parts);
    const int64_t target = target_of(a, row, a.parts == 1 && threadIdx.x == 0);
    if (target == kLeftOut) {
      if (a.parts == 1) put_left_out(a, row);
      continue;
    }
    const RowPacks<T, V> xs{static_cast<const T*>(a.x) + row * a.stride, a.vocab};
    const uint32_t p0 = part * a.part_packs, end = umin32(p0 + a.part_packs, packs);
    const float x = target >= 0 ? (float)xs.x[target] : 0.0f;
    Lane l{{-FLT_MAX, 0.0f, 0.0f}, -INFINITY, 0u};
    const uint32_t n = end - p0, whole = (umin32(end, full) - p0) / kLogChunk;
    uint32_t i = 0;
    Pack<T, V> r[kLogUnits];
    for (; i < whole; ++i) {
#pragma unroll
      for (uint32_t u = 0; u < kLogUnits; ++u)
        r[u] = load_pack<T, V>(
            xs.x + (p0 + i * kLogChunk + u * kLogThreads + threadIdx.x) * V);
      add_chunk<T, V, kTop>(l, r, c, i);
    }
    for (; i * kLogChunk < n; ++i) {
#pragma unroll
      for (uint32_t u = 0; u < kLogUnits; ++u)
        r[u] = xs.load(p0 + i * kLogChunk + u * kLogThreads + threadIdx.x, end);
      add_chunk<T, V, kTop>(l, r, c, i);
    }
    const LogitPart sum = block_merged(l.p, c, sums);
    const bool ordered = sum.s0 >= 0.0f;  // no NaN
    if (kTop && ordered) select_top(xs, p0, n, l, a.top, lds);
    if (a.parts == 1) {
      const tlc_token_result res = result_of(sum, a.scale, target >= 0, x);
      if (threadIdx.x == 0) a.results[row] = res;
      if (kTop) put_top(a, row, lds.best, res);
    } else {
      if (threadIdx.x == 0) a.part[b] = sum;
      if (kTop && threadIdx.x < a.top)
        a.keys[b * a.top + threadIdx.x] =
            ordered && threadIdx.x < lds.count ? lds.best[threadIdx.x] : 0;
    }
    __syncthreads();
  }
}

// The parts of a row put together, a block each.
template <class T>
__global__ __launch_bounds__(kLogThreads) void tlc_token_join_kernel(TokenArgs a) {
  __shared__ LogitPart sums[kLogWaves];
  __shared__ TopLds lds;
  const uint32_t row = blockIdx.x, tid = threadIdx.x;
  const int64_t target = target_of(a, row, tid == 0);
  if (target == kLeftOut) {
    put_left_out(a, row);
    return;
  }
  const uint64_t first = (uint64_t)row * a.parts;
  const float c = a.scale * kLog2e;
  const float x = target >= 0 ? (float)(static_cast<const T*>(a.x) + row * a.stride)[target] : 0.0f;
  LogitPart p{-FLT_MAX, 0.0f, 0.0f};
  if (tid < a.parts) p = a.part[first + tid];
  const LogitPart sum = block_merged(p, c, sums);
  const tlc_token_result res = result_of(sum, a.scale, target >= 0, x);
  if (tid == 0) a.results[row] = res;
  if (a.top == 0) return;
  if (sum.s0 >= 0.0f) {
    // the first `deep` keys of `lists` parts are `top` keys or more, none below the
    // least of their deep-th ones
    const uint32_t deep = (a.top + a.parts - 1) / a.parts, lists = (a.top + deep - 1) / deep;
    const uint64_t* keys = a.keys + first * a.top;
    const uint64_t key = tid < a.parts ? keys[tid * a.top + deep - 1] : 0;
    lds.keys[tid] = key;
    if (tid == 0) {
      lds.count = 0;
      lds.least = 1;  // 0: no key
    }
    __syncthreads();
    if (key != 0 && rank_of(lds.keys, a.parts, key) == lists - 1) lds.least = key;
    __syncthreads();
    const uint32_t n = a.parts * a.top;
    for (uint32_t i0 = 0; i0 < n; i0 += kLogThreads * 8) {
#pragma unroll
      for (uint32_t u = 0; u < 8; ++u) {
        const uint32_t i = i0 + u * kLogThreads + tid;
        if (i < n) put_key(lds, keys[i]);
      }
      end_round(lds, a.top);
    }
    keep_best(lds, lds.count, a.top);
  }
  put_top(a, row, lds.best, res);
}

// The gradient, kGradUnits packs of a row a thread; rows that are left out, or
// have nothing above -inf, get zeroes and are not read.
constexpr uint32_t kGradUnits = 4;
template <class In, class Out, int V, bool kEntropy>
__global__ __launch_bounds__(kLogThreads) void tlc_token_grad_kernel(TokenGradArgs a) {
  const uint32_t full = a.vocab / V, rest = a.vocab - full * V;
  const uint64_t blocks = (uint64_t)a.count * a.slices;
  const float c = a.scale * kLog2e;
  for (uint64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
    const uint32_t row = (uint32_t)(b / a.slices), slice = (uint32_t)(b - (uint64_t)row * a.slices);
    const int64_t target = target_of(a, row, slice == 0 && threadIdx.x == 0);
    const In* x = static_cast<const In*>(a.x) + row * a.stride;
    Out* out = static_cast<Out*>(a.out) + row * a.out_stride;
    const tlc_token_result res = a.results[row];
    const bool live = target != kLeftOut && res.max != -INFINITY;
    const float ga = live && a.grad_logprob ? a.grad_logprob[row] : 0.0f;
    const float gb = kEntropy && live ? a.grad_entropy[row] : 0.0f;
    const float fa = -(ga * a.scale), fb = -(gb * a.scale), ls2 = res.log_sum * kLog2e;
    const auto grad = [&](float v, uint32_t k) {
      const float z = v - res.max;
      const float p = exp2_of(z * c - ls2);
      float bonus = 0.0f;
      if (kEntropy) bonus = fb * (fmaxf(z * a.scale - res.log_sum, kFar) + res.entropy);
      if ((int64_t)k == target)  // a (1 - p), without the loss of 1 - p near 1
        return fa * expm1f(z * a.scale - res.log_sum) + bonus * p;
      return (fa + bonus) * p;
    };
    const uint32_t u0 = slice * (kLogThreads * kGradUnits) + threadIdx.x;
    Pack<In, V> r[kGradUnits] = {};
    if (live)
#pragma unroll
      for (uint32_t i = 0; i < kGradUnits; ++i) {
        const uint32_t u = u0 + i * kLogThreads;
        if (u < full) r[i] = load_pack<In, V>(x + u * V);
      }
#pragma unroll
    for (uint32_t i = 0; i < kGradUnits; ++i) {
      const uint32_t u = u0 + i * kLogThreads;
      if (u >= full) break;
      Pack<Out, V> o;
#pragma unroll
      for (int e = 0; e < V; ++e) o.set(e, live ? grad(r[i].get(e), u * V + e) : 0.0f);
      store_pack<Out, V>(out + u * V, o);
    }
    if (slice + 1 == a.slices && threadIdx.x < rest) {
      const uint32_t k = full * V + threadIdx.x;
      out[k] = round_to<Out>(live ? grad((float)x[k], k) : 0.0f);
    }
  }
}

namespace {

constexpr uint64_t kMostBlocks = 1u << 22;

template <class T, int V>
hipError_t logprobs_packs(const TokenArgs& a, hipStream_t st) {
  const uint64_t blocks = std::min((uint64_t)a.count * a.parts, kMostBlocks);
  if (a.top)
    launch_k(tlc_token_logprobs_kernel<T, V, true>, (uint32_t)blocks, kLogThreads, st, a);
  else
    launch_k(tlc_token_logprobs_kernel<T, V, false>, (uint32_t)blocks, kLogThreads, st, a);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && a.parts > 1) {
    launch_k(tlc_token_join_kernel<T>, a.count, kLogThreads, st, a);
    e = hipGetLastError();
  }
  return e;
}

template <class T>
hipError_t logprobs_rows(TokenArgs a, hipStream_t st) {
  constexpr int V = 16 / sizeof(T);
  const uint32_t packs = a.vocab < V ? a.vocab : (a.vocab + V - 1) / V;
  a.parts = logit_parts(a.count, packs);
  a.part_packs = (packs + a.parts - 1) / a.parts;
  a.parts = (packs + a.part_packs - 1) / a.part_packs;
  return a.vocab < V ? logprobs_packs<T, 1>(a, st) : logprobs_packs<T, V>(a, st);
}

template <class In, class Out>
hipError_t grad_rows(TokenGradArgs a, hipStream_t st) {
  constexpr int V = 16 / sizeof(Out);
  const uint32_t each = kLogThreads * kGradUnits;
  a.slices = std::max(1u, (a.vocab / V + each - 1) / each);
  const uint32_t blocks = (uint32_t)std::min((uint64_t)a.count * a.slices, kMostBlocks);
  if (a.grad_entropy)
    launch_k(tlc_token_grad_kernel<In, Out, V, true>, blocks, kLogThreads, st, a);
  else
    launch_k(tlc_token_grad_kernel<In, Out, V, false>, blocks, kLogThreads, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_token_logprobs(const TokenArgs& a, int type, hipStream_t st) {
  return with_type(type, [&](auto t) { return logprobs_rows<decltype(t)>(a, st); });
}

hipError_t launch_token_grad(const TokenGradArgs& a, int type, int out_type, hipStream_t st) {
  return with_type(type, [&](auto in) {
    return with_type(out_type,
                     [&](auto out) { return grad_rows<decltype(in), decltype(out)>(a, st); });
  });
}

}  // namespace tlc
