// logprobs.hip -- log probabilities of given tokens with entropy and the most
// likely alternatives, and their gradient.  Of a row of logits x, scale s, target t:
//   m = max x,  l = ln sum exp(s (x - m)),  logprob = s (x_t - m) - l
//   H = l - sum p s (x - m),  p = exp(s (x - m) - l)
//   dx_j = s (a (1[j = t] - p_j) - b p_j (ln p_j + H))   of their gradients a, b
// What bounds it: the logits read once (8192 x 65536 bf16 values, 966 MB, 144 us:
// 6.7 TB/s; what the cache holds also by its arithmetic), and for the gradient its
// values written once (8192 x 131072, 4.08 GB, 660 us: 6.2 TB/s); of few rows the
// chain of a launch, the loads, and the choice of alternatives (1 x 32768 with twenty
// 10 us, 64 x 131072 fp32 15.4, without alternatives 6 and 8).
#include <float.h>
#include <math.h>

#include <type_traits>

#include "device_common.hpp"
#include "train_internal.h"
#include "typed_io.hpp"

namespace tlc {
namespace {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
// Exponents are clamped here where they multiply a probability of 0: a logit of
// -inf adds 0 * kFar and not 0 * -inf.
constexpr float kFar = -1e30f;
// ln p that the gradient multiplies by p: below it p is 0 (2^-149 is exp(-103.3)),
// and the factors, below 2^109, times it stay finite.
constexpr float kGone = -128.0f;
constexpr float kFarRef = 65536.0f;  // m c below it, which fp32 rounds by 2^-8 at most

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
// f (x - m), rounded as the two steps: the difference is formed of halves, as it may be
// beyond fp32 where the product is not.
__device__ __forceinline__ float scaled_difference(float x, float m, float f) {
  return __builtin_fmaf(x, 0.5f, m * -0.5f) * (f * 2.0f);
}
__device__ __forceinline__ LogitPart rebased(LogitPart p, float m, float c) {
  const float d = fmaxf(scaled_difference(p.m, m, c), kFar), f = exp2_of(d);
  return LogitPart{m, f * p.s0, f * (p.s1 + d * p.s0)};
}
__device__ __forceinline__ LogitPart merged(LogitPart a, LogitPart b, float c) {
  const float m = fmaxf(a.m, b.m);
  a = rebased(a, m, c);
  b = rebased(b, m, c);
  return LogitPart{m, a.s0 + b.s0, a.s1 + b.s1};
}

// The larger of three.  (fmaxf() has the compiler quiet every operand first: two
// instructions more a value.)  NaN may get lost here; the sums keep it.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// Of a whole block, the same in every thread.  Uses lds[kThreads / 64] and one
// barrier.
template <int kThreads>
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
  if constexpr (kThreads == 64) return p;
  if ((threadIdx.x & 63u) == 0) lds[threadIdx.x >> 6] = p;
  __syncthreads();
  LogitPart r = lds[0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) r = merged(r, lds[w], c);
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

// The block's selection of the largest keys: rounds of kRoundKeys a thread at
// most, after kFewKeys at most.  (16.9 KB of 256 threads: nine blocks a CU.)
constexpr uint32_t kFewKeys = 256, kRoundKeys = 4;
// Parts whose segments are looked at together; a wave's rows have one.
template <int kThreads>
constexpr uint32_t kLiveParts = kThreads == 64 ? 1 : 8;
template <int kThreads>
struct TopLds {
  uint64_t keys[kThreads];
  uint64_t found[kFewKeys + kThreads * kRoundKeys];
  uint64_t best[TLC_MAX_TOP];
  uint16_t live[kThreads * kLiveParts<kThreads>];  // part * kThreads + thread, of 256 parts at most
  uint64_t least;
  uint32_t found_count, live_count;
};

// How many of keys[0, n) are above `key`.
__device__ __forceinline__ uint32_t rank_of(const uint64_t* keys, uint32_t n, uint64_t key) {
  uint32_t r = 0, j = 0;
  for (; j + 8 <= n; j += 8) {
    uint64_t k[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) k[i] = keys[j + i];
#pragma unroll
    for (int i = 0; i < 8; ++i) r += k[i] > key;
  }
  for (; j < n; ++j) r += keys[j] > key;
  return r;
}

// best: the `top` largest of the n found keys, in order; they stay as the found
// ones.  All threads; begins after a barrier and ends with one.
template <int kThreads>
__device__ __forceinline__ void keep_best(TopLds<kThreads>& l, uint32_t n, uint32_t top) {
  for (uint32_t j = threadIdx.x; j < n; j += kThreads) {
    const uint64_t key = l.found[j];
    const uint32_t r = rank_of(l.found, n, key);
    if (r < top) l.best[r] = key;
  }
  __syncthreads();
  const uint32_t kept = umin32(n, top);
  if (threadIdx.x < kept) l.found[threadIdx.x] = l.best[threadIdx.x];
  if (threadIdx.x == 0) l.found_count = kept;
  __syncthreads();
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
    r.logprob = has_target ? scaled_difference(x, p.m, scale) - r.log_sum : 0.0f;
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

// A row's results, with its best keys in LDS.
__device__ __forceinline__ void put_row(const TokenArgs& a, uint32_t row, LogitPart sum,
                                        int64_t target, float x, const uint64_t* best) {
  const tlc_token_result r = result_of(sum, a.scale, target >= 0, x);
  if (threadIdx.x == 0) a.results[row] = r;
  if (threadIdx.x >= a.top) return;
  const uint64_t at = (uint64_t)row * a.top + threadIdx.x;
  if (r.max != r.max) {
    a.top_logprobs[at] = r.max;
    a.top_ids[at] = -1;
    return;
  }
  const uint64_t key = best[threadIdx.x];
  a.top_logprobs[at] =
      r.max == -INFINITY ? -INFINITY
                         : scaled_difference(key_logit(key), r.max, a.scale) - r.log_sum;
  a.top_ids[at] = (int32_t)~(uint32_t)key;
}

struct Lane {
  LogitPart p;
  float best;     // largest logit of the thread, and the pack that had it first
  uint32_t pack;
};

// Packs first, first + kThreads, ... of a thread, kUnits of them; of a masked one
// the first `skip` columns are not its own (V: none is).
//
// Exponents are one fused x c - R, by R = m c rounded, and the sums are corrected
// for R - m c once: a value takes its conversion, half a maximum, a multiply-add,
// 2^t (a quarter of the others' rate), an addition and a multiply-add (with a
// difference, a product and a clamp in place of the first multiply-add 1001 x 30011
// fp16 values took 16.2 us instead of 14.9).  Where an exponent is not finite
// (masked entries, or what is NaN in the end) or R so large that the correction is,
// the wave takes the sums again with differences of x and m: no chunk pays for it
// before it holds such a value.  Chunks of masked entries alone are passed over.
template <class T, int V, bool kTop, int kThreads, bool kMasked, uint32_t kUnits>
__device__ __forceinline__ void add_packs(Lane& l, const Pack<T, V> (&r)[kUnits], float c,
                                          uint32_t first, uint32_t skip) {
  if (kMasked && skip >= V) return;
  const auto own = [&](int e) { return !kMasked || (uint32_t)e >= skip; };
  const auto seen = [&](uint32_t u, int e) { return own(e) ? r[u].get(e) : -INFINITY; };
  float most = -INFINITY;
#pragma unroll
  for (uint32_t u = 0; u < kUnits; ++u) {
    float pm = seen(u, 0);
#pragma unroll
    for (int e = 1; e < V; e += 2) pm = max3(pm, seen(u, e), seen(u, e + 1 < V ? e + 1 : e));
    if (kTop && pm > l.best) {
      l.best = pm;
      l.pack = first + u * kThreads;
    }
    most = max3(most, pm, pm);
  }
  if (__ballot(most != -INFINITY) == 0) {  // masked entries add nothing; but NaN is no maximum
    bool only = true;
#pragma unroll
    for (uint32_t u = 0; u < kUnits; ++u)
#pragma unroll
      for (int e = 0; e < V; ++e) only &= !own(e) || r[u].get(e) == -INFINITY;
    if (__ballot(!only) == 0) return;
  }
  const float m = fmaxf(l.p.m, most), ref = m * c;
  float d = __builtin_fmaf(-m, c, ref), s0 = 0.0f, s1 = 0.0f;
#pragma unroll
  for (uint32_t u = 0; u < kUnits; ++u)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float t = own(e) ? __builtin_fmaf(r[u].get(e), c, -ref) : kFar, w = exp2_of(t);
      s0 += w;
      s1 = __builtin_fmaf(w, t, s1);
    }
  if (__ballot(!(s1 == s1 && fabsf(ref) < kFarRef)) != 0) {
    d = s0 = s1 = 0.0f;
#pragma unroll
    for (uint32_t u = 0; u < kUnits; ++u)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float t = own(e) ? scaled_difference(r[u].get(e), m, c) : kFar, w = exp2_of(t);
        s0 += w;
        s1 = __builtin_fmaf(w, fmaxf(t, kFar), s1);
      }
  }
  const float f = exp2_of(d);
  l.p = rebased(l.p, m, c);
  l.p.s0 += f * s0;
  l.p.s1 += f * (s1 + d * s0);
}

// A segment: the columns of one thread of one part; its key is that of its
// largest logit, with the pack that had it first in the column's place (0: no
// columns).  own: the keys of this thread's segments of the first kLiveParts
// parts; seg(j, own) those of the parts from j on.
//
// The `top` largest keys of the row's columns into lds.best.  Groups of segments
// (four neighbouring threads' where `top` is small beside 64, else a thread's)
// have their largest keys ranked.  The top-th of these is the key of a column, so a
// column below it is not among the `top` largest, and a segment below it has none of
// them: the others, about `top`, are read again.  (Twenty alternatives of 1001 x 30011
// fp16 values cost 6 of 21 us; with every thread's largest logit ranked instead of
// the quads' 8.5 of 24.5.)
template <class T, int V, int kThreads, class Seg>
__device__ __forceinline__ void select_top(const RowPacks<T, V>& row, const TokenArgs& a,
                                           uint32_t packs, uint64_t (&own)[kLiveParts<kThreads>],
                                           Seg&& seg, TopLds<kThreads>& lds) {
  const uint32_t tid = threadIdx.x, top = a.top;
  const bool quads = kThreads > 64 && top <= kQuadTop;
  uint64_t key = 0;
  for (uint32_t j0 = 0; j0 < a.parts; j0 += kLiveParts<kThreads>) {
    if (j0 > 0) seg(j0, own);
#pragma unroll
    for (uint32_t j = 0; j < kLiveParts<kThreads>; ++j) key = own[j] > key ? own[j] : key;
  }
  if (quads) {
#pragma unroll
    for (int d = 1; d < 4; d <<= 1) {
      const uint64_t k = __shfl_xor(key, d);
      key = k > key ? k : key;
    }
    if ((tid & 3u) == 0) lds.keys[tid >> 2] = key;
  } else {
    lds.keys[tid] = key;
  }
  if (tid == 0) {
    lds.found_count = lds.live_count = 0;
    lds.least = 0;
  }
  __syncthreads();
  // the top-th largest key; 0 where there are fewer
  uint64_t least;
  if (kThreads == 64 || quads) {  // every wave for itself
    const uint64_t k = lds.keys[tid & 63u];
    const uint64_t who = __ballot(k != 0 && rank_of(lds.keys, 64, k) == top - 1);
    const int lane = __ffsll((unsigned long long)who) - 1;
    least = who == 0 ? 0
                     : (uint64_t)(uint32_t)__shfl((int)(uint32_t)k, lane) |
                           (uint64_t)(uint32_t)__shfl((int)(uint32_t)(k >> 32), lane) << 32;
  } else {
    if (key != 0 && rank_of(lds.keys, kThreads, key) == top - 1) lds.least = key;
    __syncthreads();
    least = lds.least;
  }
  // the same as a column's key, of the last column that its pack may have
  const uint64_t floor =
      least == 0 ? 0 : (least >> 32 << 32) | (uint32_t)~(~(uint32_t)least * V + (V - 1));
  const uint32_t each = (a.part_packs + kThreads - 1) / kThreads;  // packs of a segment
  for (uint32_t j0 = 0; j0 < a.parts; j0 += kLiveParts<kThreads>) {
    if (a.parts > kLiveParts<kThreads>) seg(j0, own);
#pragma unroll
    for (uint32_t j = 0; j < kLiveParts<kThreads>; ++j)
      if (own[j] != 0 && own[j] >= least)
        lds.live[atomicAdd(&lds.live_count, 1u)] = (uint16_t)((j0 + j) * kThreads + tid);
    __syncthreads();
    const uint32_t items = lds.live_count * each;
    for (uint32_t w0 = 0; w0 < items; w0 += kThreads) {
      const uint32_t w = w0 + tid;
      uint32_t p = packs, k = 0;
      Pack<T, V> x = {};
      if (w < items) {
        const uint32_t s = w / each, part = lds.live[s] / kThreads;
        const uint32_t i = lds.live[s] - part * kThreads + (w - s * each) * kThreads;
        if (i < a.part_packs) p = part * a.part_packs + i;
        if (p < packs) {
          k = row.start(p);
          x = load_pack<T, V>(row.x + k);
        }
      }
#pragma unroll
      for (int e0 = 0; e0 < V; e0 += kRoundKeys) {
        if (p < packs)
#pragma unroll
          for (int e = e0; e < V && e < e0 + (int)kRoundKeys; ++e) {
            const uint64_t c = key_of(x.get(e), k + e);
            if (k + e >= p * V && c >= floor) lds.found[atomicAdd(&lds.found_count, 1u)] = c;
          }
        __syncthreads();
        const uint32_t n = lds.found_count;
        __syncthreads();
        if (n > kFewKeys) keep_best(lds, n, top);
      }
    }
    if (tid == 0) lds.live_count = 0;
    __syncthreads();
  }
  keep_best(lds, lds.found_count, top);
}

// Stores and loads of what blocks hand to one another: they go to where all of the
// card's caches meet, so that a block which has waited for its stores may count
// itself as done without a fence (a fence writes back a whole L2; with one, and the
// rows' counters side by side, 64 rows of 131072 fp32 values in 512 blocks took 14.4
// instead of 8.0 us).
template <class W>
__device__ __forceinline__ void hand_over(W* p, W v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <class W>
__device__ __forceinline__ W take_over(const W* p) {
  return __hip_atomic_load(const_cast<W*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

}  // namespace

// A block reads a row, or one of `parts` parts of it; the last of a row's blocks
// puts the parts together.
template <class T, int V, bool kTop, int kThreads, uint32_t kUnits, bool kStream>
__global__ __launch_bounds__(kThreads) void tlc_token_logprobs_kernel(TokenArgs a) {
  constexpr uint32_t kChunk = kThreads * kUnits;
  __shared__ LogitPart sums[kThreads / 64];
  __shared__ std::conditional_t<kTop, TopLds<kThreads>, uint64_t> lds;
  __shared__ uint32_t last;
  const uint32_t packs = (a.vocab + V - 1) / V, full = a.vocab / V;
  const float c = a.scale * kLog2e;
  const uint64_t blocks = (uint64_t)a.count * a.parts;
  for (uint64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
    const uint32_t row = (uint32_t)(b / a.parts), part = (uint32_t)(b - (uint64_t)row * a.parts);
    const int64_t target = target_of(a, row, part == 0 && threadIdx.x == 0);
    if (target == kLeftOut) {
      if (part == 0) put_left_out(a, row);
      continue;
    }
    const RowPacks<T, V> xs{static_cast<const T*>(a.x) + row * a.stride, a.vocab};
    const uint32_t p0 = part * a.part_packs, end = umin32(p0 + a.part_packs, packs);
    const float x = target >= 0 ? (float)xs.x[target] : 0.0f;
    Lane l{{-FLT_MAX, 0.0f, 0.0f}, -INFINITY, p0 + threadIdx.x};
    const uint32_t n = end - p0, own_full = umin32(end, full) - p0;
    uint32_t i = 0;
    for (; i + kChunk <= own_full; i += kChunk) {
      const uint32_t p = p0 + i + threadIdx.x;
      Pack<T, V> r[kUnits];
#pragma unroll
      for (uint32_t u = 0; u < kUnits; ++u)
        r[u] = load_pack<T, V, kStream>(xs.x + (p + u * kThreads) * V);
      add_packs<T, V, kTop, kThreads, false>(l, r, c, p, 0);
    }
    if (i < n) {  // packs of the last columns, asked for before any is taken
      const uint32_t p = p0 + i + threadIdx.x;
      Pack<T, V> r[kUnits][1];
#pragma unroll
      for (uint32_t u = 0; u < kUnits; ++u)
        r[u][0] = load_pack<T, V>(xs.x + xs.start(umin32(p + u * kThreads, end - 1)));
#pragma unroll
      for (uint32_t u = 0; u < kUnits; ++u) {
        const uint32_t q = p + u * kThreads;
        if (i + (u + 1) * kThreads <= own_full)
          add_packs<T, V, kTop, kThreads, false>(l, r[u], c, q, 0);
        else if (i + u * kThreads < n)
          add_packs<T, V, kTop, kThreads, true>(l, r[u], c, q,
                                                q < end ? q * V - xs.start(q) : V);
      }
    }
    LogitPart sum = block_merged<kThreads>(l.p, c, sums);
    const uint64_t key = threadIdx.x < n ? key_of(l.best, l.pack) : 0;
    const uint64_t first = (uint64_t)row * a.parts;
    const uint64_t* const keys = a.keys + first * kThreads + threadIdx.x;
    const auto seg = [&](uint32_t j0, uint64_t(&own)[kLiveParts<kThreads>]) {
#pragma unroll
      for (uint32_t j = 0; j < kLiveParts<kThreads>; ++j)
        own[j] = take_over(keys + umin32(j0 + j, a.parts - 1) * kThreads);
#pragma unroll
      for (uint32_t j = 0; j < kLiveParts<kThreads>; ++j)
        if (j0 + j >= a.parts) own[j] = 0;
    };
    uint64_t own[kLiveParts<kThreads>] = {key};
    if (a.parts > 1) {
      if (threadIdx.x == 0) {
        hand_over(&a.part[b].m, sum.m);
        hand_over(&a.part[b].s0, sum.s0);
        hand_over(&a.part[b].s1, sum.s1);
      }
      if (kTop) hand_over(a.keys + b * kThreads + threadIdx.x, key);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (threadIdx.x == 0)
        last = __hip_atomic_fetch_add(a.tickets + row * kTicketWords, 1u, __ATOMIC_RELAXED,
                                      __HIP_MEMORY_SCOPE_AGENT) == a.parts - 1;
      __syncthreads();
      if (!last) continue;
      if (threadIdx.x == 0) a.tickets[row * kTicketWords] = 0u;
      if (kTop) seg(0, own);
      LogitPart p{-FLT_MAX, 0.0f, 0.0f};
      for (uint32_t j = threadIdx.x; j < a.parts; j += kThreads) {
        const LogitPart* q = a.part + first + j;
        p = merged(p, LogitPart{take_over(&q->m), take_over(&q->s0), take_over(&q->s1)}, c);
      }
      sum = block_merged<kThreads>(p, c, sums);
    }
    if constexpr (kTop)
      if (sum.s0 >= 0.0f) select_top(xs, a, packs, own, seg, lds);  // no NaN
    if constexpr (kTop)
      put_row(a, row, sum, target, x, lds.best);
    else
      put_row(a, row, sum, target, x, nullptr);
    __syncthreads();
  }
}

namespace {

// What the gradient needs of a row.
struct GradRow {
  int64_t target;
  float fa, fb;  // -scale times the gradients of the log probability and the entropy
  float unit;    // of fa and fb
  float max, log_sum, entropy;
  bool live;     // else zeroes, taken at x = 0: the row is not read
};
template <bool kEntropy>
__device__ __forceinline__ GradRow grad_row(const TokenGradArgs& a, uint32_t row, bool report) {
  GradRow r;
  r.target = target_of(a, row, report);
  const tlc_token_result res = a.results[row];
  const float ga = a.grad_logprob ? a.grad_logprob[row] : 0.0f;
  const float gb = kEntropy ? a.grad_entropy[row] : 0.0f;
  r.live = r.target != kLeftOut && res.max != -INFINITY;
  if (!r.live) return GradRow{-1, 0.0f, 0.0f, 1.0f, 0.0f, 0.0f, 0.0f, false};  // 0 at x = 0
  // factors near fp32's end and beyond it are held as multiples of 2^80, as what p
  // leaves of them may be small (infinite ones are not: theirs is infinite)
  const float most = fmaxf(fabsf(ga), fabsf(gb));
  const bool large = most <= FLT_MAX && most * a.scale > 0x1p100f;
  const float s = large ? a.scale * 0x1p-80f : a.scale;
  r.unit = large ? 0x1p80f : 1.0f;
  r.fa = -(ga * s);
  r.fb = -(gb * s);
  r.max = res.max;
  r.log_sum = res.log_sum;
  r.entropy = res.entropy;
  return r;
}

template <bool kEntropy>
__device__ __forceinline__ float grad_of(const GradRow& r, float scale, float x, bool is_target) {
  const float p = exp2_of(scaled_difference(x, r.max, scale * kLog2e) - r.log_sum * kLog2e);
  const float z = scaled_difference(x, r.max, scale);
  float bonus = 0.0f;
  if (kEntropy) bonus = r.fb * (fmaxf(z - r.log_sum, kGone) + r.entropy);
  // a (1 - p) without a difference: near p = 1 as exact as log_sum, whose sum holds the
  // largest logit's own 1, and so to 2^-24 of each addition, absolute
  if (is_target)
    return (r.fa * expm1f(z - r.log_sum) + bonus * p) * r.unit;
  return (r.fa + bonus) * p * r.unit;
}

template <class In, class Out, int V, bool kEntropy>
__device__ __forceinline__ Pack<Out, V> grad_pack(const GradRow& r, float scale,
                                                  const Pack<In, V>& x, uint32_t k) {
  Pack<Out, V> o;
  const uint32_t at = (uint32_t)(r.target - (int64_t)k);  // V and above: another pack's
#pragma unroll
  for (int e = 0; e < V; ++e) o.set(e, grad_of<kEntropy>(r, scale, x.get(e), false));
  if (at < V && r.target >= 0)
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (at == (uint32_t)e) o.set(e, grad_of<kEntropy>(r, scale, x.get(e), true));
  return o;
}

}  // namespace

// The gradient of a slice of a row, kGradUnits packs a thread (two: 8192 x 131072
// bf16 values 664 us, 6.1 TB/s; one 897, four 723, eight 763).
template <class In, class Out, int V, bool kEntropy, bool kStream>
__global__ __launch_bounds__(kLogThreads) void tlc_token_grad_kernel(TokenGradArgs a) {
  const uint32_t full = a.vocab / V, rest = a.vocab - full * V;
  const uint64_t blocks = (uint64_t)a.count * a.slices;
  for (uint64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
    const uint32_t row = (uint32_t)(b / a.slices), slice = (uint32_t)(b - (uint64_t)row * a.slices);
    const GradRow g = grad_row<kEntropy>(a, row, slice == 0 && threadIdx.x == 0);
    const In* x = static_cast<const In*>(a.x) + row * a.stride;
    Out* out = static_cast<Out*>(a.out) + row * a.out_stride;
    const uint32_t u0 = slice * (kLogThreads * kGradUnits) + threadIdx.x;
    Pack<In, V> r[kGradUnits] = {};
    if (g.live)
#pragma unroll
      for (uint32_t i = 0; i < kGradUnits; ++i) {
        const uint32_t u = u0 + i * kLogThreads;
        if (u < full) r[i] = load_pack<In, V, kStream>(x + u * V);
      }
#pragma unroll
    for (uint32_t i = 0; i < kGradUnits; ++i) {
      const uint32_t u = u0 + i * kLogThreads;
      if (u >= full) break;
      store_pack<Out, V, kStream>(out + u * V,
                                  grad_pack<In, Out, V, kEntropy>(g, a.scale, r[i], u * V));
    }
    if (slice + 1 == a.slices && threadIdx.x < rest) {
      const uint32_t k = full * V + threadIdx.x;
      Pack<In, 1> one = {};
      if (g.live) one.v = x[k];
      out[k] = grad_pack<In, Out, 1, kEntropy>(g, a.scale, one, k).v;
    }
  }
}

// Of short rows (16384 x 1024 bf16 values 13.7 us, a block each 20; 8192 x 2048 fp32
// values 22.7 | 21): their packs one after the other, the last one of a row shorter
// where it is no whole number of them.
template <class In, class Out, int V, bool kEntropy>
__global__ __launch_bounds__(kLogThreads) void tlc_token_grad_short_kernel(TokenGradArgs a,
                                                                           Divider packs) {
  const uint32_t u = blockIdx.x * kLogThreads + threadIdx.x;
  const uint32_t row = quotient(u, packs);
  if (row >= a.rows) return;
  const uint32_t k = (u - row * packs.d) * V;
  const GradRow g = grad_row<kEntropy>(a, a.row0 + row, k == 0);
  const In* x = static_cast<const In*>(a.x) + (uint64_t)(a.row0 + row) * a.stride + k;
  Out* out = static_cast<Out*>(a.out) + (uint64_t)(a.row0 + row) * a.out_stride + k;
  if (k + V <= a.vocab) {
    Pack<In, V> r = {};
    if (g.live) r = load_pack<In, V>(x);
    store_pack<Out, V>(out, grad_pack<In, Out, V, kEntropy>(g, a.scale, r, k));
    return;
  }
#pragma unroll
  for (uint32_t e = 0; e < V; ++e) {
    if (k + e >= a.vocab) break;
    Pack<In, 1> one = {};
    if (g.live) one.v = x[e];
    out[e] = grad_pack<In, Out, 1, kEntropy>(g, a.scale, one, k + e).v;
  }
}

namespace {

constexpr uint64_t kMostBlocks = 1u << 22;


template <class T, int V, int kThreads, uint32_t kUnits, bool kStream>
hipError_t logprobs_blocks(TokenArgs a, uint32_t packs, hipStream_t st) {
  a.parts = kThreads == 64 ? 1 : logit_parts(a.count, packs);  // (64: a.keys holds none)
  a.part_packs = (packs + a.parts - 1) / a.parts;
  a.parts = (packs + a.part_packs - 1) / a.part_packs;
  const uint32_t blocks = (uint32_t)std::min((uint64_t)a.count * a.parts, kMostBlocks);
  if (a.top)
    launch_k(tlc_token_logprobs_kernel<T, V, true, kThreads, kUnits, kStream>, blocks, kThreads,
             st, a);
  else
    launch_k(tlc_token_logprobs_kernel<T, V, false, kThreads, kUnits, kStream>, blocks, kThreads,
             st, a);
  return hipGetLastError();
}

template <class T>
hipError_t logprobs_rows(const TokenArgs& a, hipStream_t st) {
  constexpr int V = 16 / sizeof(T);
  const uint32_t packs = (a.vocab + V - 1) / V;
  if (a.vocab < V) return logprobs_blocks<T, 1, 64, 1, false>(a, a.vocab, st);
  if (wave_rows(a.count, packs, a.top))
    return packs <= 2 * 64 ? logprobs_blocks<T, V, 64, 2, false>(a, packs, st)
                           : logprobs_blocks<T, V, 64, 4, false>(a, packs, st);
  if ((uint64_t)a.count * packs * 16 >= kStreamBytes)
    return logprobs_blocks<T, V, kLogThreads, 8, true>(a, packs, st);
  return packs <= 2 * kLogThreads ? logprobs_blocks<T, V, kLogThreads, 2, false>(a, packs, st)
                                  : logprobs_blocks<T, V, kLogThreads, 4, false>(a, packs, st);
}

template <class In, class Out, bool kEntropy>
hipError_t grad_rows(TokenGradArgs a, hipStream_t st) {
  constexpr int V = 16 / sizeof(Out);
  const uint32_t packs = (a.vocab + V - 1) / V;
  if (packs <= kShortPacks) {
    const Divider d = divider(packs);
    const uint32_t most = ((1u << 31) - kLogThreads) / packs;  // rows of a launch
    for (a.row0 = 0; a.row0 < a.count; a.row0 += a.rows) {
      a.rows = std::min(a.count - a.row0, most);
      launch_k(tlc_token_grad_short_kernel<In, Out, V, kEntropy>,
               (a.rows * packs + kLogThreads - 1) / kLogThreads, kLogThreads, st, a, d);
    }
    return hipGetLastError();
  }
  const uint32_t each = kLogThreads * kGradUnits;
  a.slices = (a.vocab / V + each - 1) / each;
  const uint32_t blocks = (uint32_t)std::min((uint64_t)a.count * a.slices, kMostBlocks);
  if ((uint64_t)a.count * a.vocab * sizeof(Out) >= kStreamBytes)
    launch_k(tlc_token_grad_kernel<In, Out, V, kEntropy, true>, blocks, kLogThreads, st, a);
  else
    launch_k(tlc_token_grad_kernel<In, Out, V, kEntropy, false>, blocks, kLogThreads, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_token_logprobs(const TokenArgs& a, int type, hipStream_t st) {
  return with_type(type, [&](auto t) { return logprobs_rows<decltype(t)>(a, st); });
}

hipError_t launch_token_grad(const TokenGradArgs& a, int type, int out_type, hipStream_t st) {
  return with_type(type, [&](auto in) {
    return with_type(out_type, [&](auto out) {
      return a.grad_entropy ? grad_rows<decltype(in), decltype(out), true>(a, st)
                            : grad_rows<decltype(in), decltype(out), false>(a, st);
    });
  });
}

}  // namespace tlc
