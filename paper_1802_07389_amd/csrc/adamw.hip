// adamw.hip -- one step of AdamW over a list of tensors, every operation rounded
// to fp32:
//   g' = coef g,  m' = m + (g' - m) c1,  v' = v + (g' g' - v) c2
//   p' = p - (a (m' / (sqrt(v') r + eps)) + w p)
// with c = 1 - beta, a = lr / (1 - beta1^t), r = 1 / sqrt(1 - beta2^t), w = lr decay.
// States of 8 bits hold 256 values by one scale, m as OCP E4M3 and v as OCP E5M2.
// What bounds it: every tensor read and written once (28 bytes an fp32 value of
// fp32 states, 16 of 8 bits): 148 tensors of 100M fp32 weights with bf16 gradients
// 503 us (5.2 TB/s), of 8-bit states, whose blocks begin within lines, 312 (4.5 TB/s); one
// tensor 484 and 290.  Raw square roots and quotients changed neither.  335 tensors of
// 1.7M values 14 us, of which one launch and the read of the pieces over the bus are 8.
#include <math.h>

#include <type_traits>

#include "device_common.hpp"
#include "train_internal.h"
#include "typed_io.hpp"

namespace tlc {
namespace {

struct Factors {
  float rate, root, decay, coef;
  uint32_t step;  // its low word
  bool skip;
};

// The step's factors, in 64 bits until they are complete.
__device__ __forceinline__ Factors factors_of(const AdamArgs& a, int64_t step) {
  const double lr = a.lr * (double)a.clock->lr_scale, t = (double)step;
  Factors f;
  f.rate = (float)(lr / -expm1(t * a.log_beta1));
  f.root = (float)(1.0 / sqrt(-expm1(t * a.log_beta2)));
  f.decay = (float)(lr * a.decay);
  f.coef = 1.0f;
  f.step = (uint32_t)step;
  f.skip = false;
  if (a.result) {
    const Clip c = clip_of(a.result->sumsq, a.max_norm);
    f.coef = c.coef;
    f.skip = !c.finite;
  }
  return f;
}

__device__ __forceinline__ float adam_step(float p, float g, float& m, float& v,
                                           const AdamArgs& a, const Factors& f) {
  m = m + (g - m) * a.c1;
  v = v + (g * g - v) * a.c2;
  const float u = m / (sqrtf(v) * f.root + a.eps);
  return p - (f.rate * u + f.decay * p);
}

constexpr int V = 4;  // neighbouring values of a thread
constexpr uint32_t kStride = kAdamThreads * V;
static_assert(kStride == kAdamUnit, "a unit is a pack of every thread");

// Values k to k + 3 of x, those from n on 0.  No load waits for a condition: at
// the end a pack is moved back to end with the values, and its own ones shifted
// down; of fewer values than a pack, value by value.
template <bool kFull, bool kStream, class T>
__device__ __forceinline__ Pack<T, V> load_some(const void* x, uint32_t k, uint32_t n) {
  const T* p = static_cast<const T*>(x);
  if (kFull) return load_pack<T, V, kStream>(p + k);
  Pack<T, V> r;
  if (n < V) {
#pragma unroll
    for (uint32_t e = 0; e < V; ++e) {
      r.v[e] = p[umin32(k + e, n - 1)];
      if (k + e >= n) r.v[e] = T();
    }
    return r;
  }
  const uint32_t at = umin32(k, n - V), skip = k - at;
  const Pack<T, V> c = load_pack<T, V>(p + at);
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (uint32_t e = 0; e < V; ++e) {
      r.v[e] = T();
#pragma unroll
      for (uint32_t s = V - e; s-- > 0;) r.v[e] = skip == s ? c.v[e + s] : r.v[e];
    }
  } else {
    using Word = std::conditional_t<sizeof(T) == 2, uint64_t, uint32_t>;
    const Word w = skip < V ? __builtin_bit_cast(Word, c.v) >> (8 * sizeof(T) * skip) : 0;
    r.v = __builtin_bit_cast(decltype(r.v), w);
  }
  return r;
}
template <bool kFull, bool kStream, class T>
__device__ __forceinline__ void store_some(void* x, uint32_t k, uint32_t n, const Pack<T, V>& r) {
  T* p = static_cast<T*>(x);
  if (kFull || k + V <= n) {
    store_pack<T, V, kStream>(p + k, r);
    return;
  }
#pragma unroll
  for (uint32_t e = 0; e < V; ++e)
    if (k + e < n) p[k + e] = r.v[e];
}

// The code of y >= 0 in a format of kMantissa bits with smallest exponent kLowest
// (below it steps are even) and largest code kMost: the codes joined by straight
// lines make y a place between two of them, which `dither` (of the 23 - kMantissa
// bits that are cut off) carries to the upper one as often as y is near it.  At
// least `least`.
template <int kMantissa, int kLowest, uint32_t kMost>
__device__ __forceinline__ uint32_t fp8_code(float y, uint32_t dither, uint32_t least) {
  constexpr int kCut = 23 - kMantissa;
  constexpr float kUnit = 1.0f / (float)(1ull << -kLowest);  // 2^kLowest
  constexpr float kFine = (float)(1ull << (kMantissa - kLowest + kCut));
  const uint32_t fine = __float_as_uint(y) - ((uint32_t)(126 + kLowest) << 23);
  const uint32_t small = (uint32_t)(fminf(y, kUnit) * kFine);
  return umin32(umax32(((y < kUnit ? small : fine) + dither) >> kCut, least), kMost);
}

// A block's scale from its largest magnitude (as bits): its share of the
// format's largest number (inv_most: 1 / that), at least 2^-126 so that it
// divides; NaN where a value is NaN or infinite.
__device__ __forceinline__ float scale_of_max(uint32_t bits, float inv_most) {
  if (bits == 0) return 0.0f;
  if (bits >= 0x7f800000u) return __builtin_nanf("");
  return fmaxf(__uint_as_float(bits) * inv_most, 0x1p-126f);
}

// x / s of many x >= 0 by one s, rounded as a division: the residual of a quotient
// that is within a unit in the last place, times the rounded reciprocal, corrects
// it (Markstein, IBM J. Res. Dev. 34, 1990), and one such step before brings the product with
// the reciprocal there.  Residuals are exact where they do not underflow: of x below
// 2^-102, whose quotient no code tells from 0 for s from 2^-64 on; for other s, a
// division.
struct Divisor {
  float s, r;
  bool exact;
  __device__ __forceinline__ explicit Divisor(float scale)
      : s(scale), r(1.0f / scale), exact(scale >= 0x1p-64f && scale <= 0x1p100f) {}
  __device__ __forceinline__ float of(float x) const {
    float q = x * r;
    q = __builtin_fmaf(__builtin_fmaf(-q, s, x), r, q);
    return __builtin_fmaf(__builtin_fmaf(-q, s, x), r, q);
  }
};

// The first two powers of the inverse plastic number, as fractions of 2^32: of
// value k in step t the dither is the fraction of k / rho + t / rho^2, which is
// spread evenly over neighbours and over steps.
constexpr uint32_t kDitherK = 0xC13FA9A9u, kDitherT = 0x91E10DA5u;

// What a thread reads of a chunk.
template <class P, class G, int kBits, uint32_t kSteps>
struct Chunk {
  Pack<P, V> p[kSteps];
  Pack<G, V> g[kSteps];
  Pack<std::conditional_t<kBits == 32, float, uint8_t>, V> m[kSteps], v[kSteps];
  float sm[kSteps], sv[kSteps];
};

template <bool kFull, bool kStream, class P, class G, int kBits, uint32_t kSteps>
__device__ __forceinline__ void load_chunk(Chunk<P, G, kBits, kSteps>& c, const AdamPiece& t,
                                           uint32_t k0) {
  using S = std::conditional_t<kBits == 32, float, uint8_t>;
#pragma unroll
  for (uint32_t u = 0; u < kSteps; ++u) {
    const uint32_t k = k0 + u * kStride + threadIdx.x * V;
    c.p[u] = load_some<kFull, kStream, P>(t.p, k, t.n);
    c.g[u] = load_some<kFull, kStream, G>(t.g, k, t.n);
    c.m[u] = load_some<kFull, kStream, S>(t.m, k, t.n);
    c.v[u] = load_some<kFull, kStream, S>(t.v, k, t.n);
    if constexpr (kBits == 8) {
      // (a wave beyond the end takes the last block's: its values are 0)
      const uint32_t b = umin32(k, t.n - 1) / TLC_STATE_BLOCK;
      c.sm[u] = t.scales[b * 2];
      c.sv[u] = t.scales[b * 2 + 1];
    }
  }
}

template <bool kFull, bool kStream, class P, class G, int kBits, uint32_t kSteps>
__device__ __forceinline__ void step_chunk(const Chunk<P, G, kBits, kSteps>& c,
                                           const AdamPiece& t, uint32_t k0, const AdamArgs& a,
                                           const Factors& f) {
  using S = std::conditional_t<kBits == 32, float, uint8_t>;
#pragma unroll
  for (uint32_t u = 0; u < kSteps; ++u) {
    const uint32_t k = k0 + u * kStride + threadIdx.x * V;
    float m[V], v[V];
    if constexpr (kBits == 32) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        m[e] = c.m[u].get(e);
        v[e] = c.v[u].get(e);
      }
    } else {
      const int wm = __builtin_bit_cast(int, c.m[u].v), wv = __builtin_bit_cast(int, c.v[u].v);
      const auto m01 = __builtin_amdgcn_cvt_pk_f32_fp8(wm, false);
      const auto m23 = __builtin_amdgcn_cvt_pk_f32_fp8(wm, true);
      const auto v01 = __builtin_amdgcn_cvt_pk_f32_bf8(wv, false);
      const auto v23 = __builtin_amdgcn_cvt_pk_f32_bf8(wv, true);
      const float cm[V] = {m01[0], m01[1], m23[0], m23[1]};
      const float cv[V] = {v01[0], v01[1], v23[0], v23[1]};
#pragma unroll
      for (int e = 0; e < V; ++e) {
        m[e] = cm[e] * c.sm[u];
        v[e] = cv[e] * c.sv[u];
      }
    }
    Pack<P, V> q;
    Pack<float, V> d;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float old = c.p[u].get(e);
      q.set(e, adam_step(old, f.coef * c.g[u].get(e), m[e], v[e], a, f));
      d.set(e, q.get(e) - old);
    }
    store_some<kFull, kStream, P>(t.p, k, t.n, q);
    if (t.delta) store_some<kFull, kStream, float>(t.delta, k, t.n, d);
    Pack<S, V> pm, pv;
    if constexpr (kBits == 32) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        pm.set(e, m[e]);
        pv.set(e, v[e]);
      }
    } else {
      uint32_t mm = 0, mv = 0;  // (values beyond the end are 0)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        mm = umax32(mm, abs_bits(m[e]));
        mv = umax32(mv, abs_bits(v[e]));
      }
      const float sm = scale_of_max(wave_max(mm), 1.0f / 448.0f);  // the wave's, in scalars
      const float sv = scale_of_max(wave_max(mv), 1.0f / 57344.0f);
      float ym[V], yv[V];
      const Divisor dm(sm), dv(sv);
      if (dm.exact && dv.exact) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          ym[e] = dm.of(fabsf(m[e]));
          yv[e] = dv.of(v[e]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          ym[e] = sm > 0.0f ? fabsf(m[e]) / sm : 0.0f;
          yv[e] = sv > 0.0f ? v[e] / sv : 0.0f;
        }
      }
      uint32_t wm = 0, wv = 0;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const uint32_t h = (t.k0 + k + e) * kDitherK + f.step * kDitherT;
        // a nonzero v stays one
        const uint32_t qm = fp8_code<3, -6, 126>(ym[e], h >> 12, 0u);
        const uint32_t qv = fp8_code<2, -14, 123>(yv[e], (h ^ 0x80000000u) >> 11,
                                                  umin32(__float_as_uint(v[e]), 1u));
        wm |= (qm | (__float_as_uint(m[e]) >> 24 & 0x80u)) << (8 * e);
        wv |= qv << (8 * e);
      }
      if (!(sm >= 0.0f)) wm = 0;
      if (!(sv >= 0.0f)) wv = 0;
      pm.v = __builtin_bit_cast(decltype(pm.v), wm);
      pv.v = __builtin_bit_cast(decltype(pv.v), wv);
      if (k % TLC_STATE_BLOCK == 0 && (kFull || k < t.n)) {
        t.scales[k / TLC_STATE_BLOCK * 2] = sm;
        t.scales[k / TLC_STATE_BLOCK * 2 + 1] = sv;
      }
    }
    store_some<kFull, kStream, S>(t.m, k, t.n, pm);
    store_some<kFull, kStream, S>(t.v, k, t.n, pv);
  }
}

// Piece i of a list, with pointers to its values.
__device__ __forceinline__ AdamPiece piece_of(const AdamPinned& list, uint32_t i) {
  return list.pieces[i];
}
__device__ __forceinline__ AdamPiece piece_of(const AdamList& list, uint32_t i) {
  const uint32_t lane = threadIdx.x & 63u;
  const uint32_t s = (uint32_t)__popcll(__ballot(
      lane < list.count && (list.tensors[lane].piece0_types & 0xfffffffu) <= i));
  const AdamTensor& t = list.tensors[uniform32(s) - 1];
  return adam_piece(t, t.piece0_types >> 28, (i - (t.piece0_types & 0xfffffffu)) * list.len,
                    list.len, list.state_bytes);
}

// Whether this block is the last one to have read the clock, whose value `step`
// is here.  Blocks count themselves in groups, and the last of each group the
// groups: one word for all took 8 ns a block (977 blocks of 1024 values 16.8 us).
__device__ __forceinline__ bool last_to_read(uint32_t* tickets, int64_t step) {
  uint32_t one = 1u;
  asm volatile("" : "+v"(one) : "v"((uint32_t)step));  // the read is done before the count
  const uint32_t groups = umin32(gridDim.x, kTicketGroups), g = blockIdx.x % groups;
  uint32_t* mine = tickets + (1 + g) * kTicketWords;
  if (atomicAdd(mine, one) != (gridDim.x - g + groups - 1) / groups - 1) return false;
  *mine = 0u;
  if (atomicAdd(tickets, 1u) != groups - 1) return false;
  *tickets = 0u;
  return true;
}

constexpr uint32_t kLine = 128;

// A piece of n values of fp32 states without its first `head`.
__device__ __forceinline__ AdamPiece adam_rest(AdamPiece t, uint32_t head, uint32_t n, uint32_t p,
                                               uint32_t g) {
  t.p = static_cast<uint8_t*>(t.p) + head * p;
  t.g = static_cast<const uint8_t*>(t.g) + head * g;
  t.m = static_cast<float*>(t.m) + head;
  t.v = static_cast<float*>(t.v) + head;
  t.delta = t.delta ? t.delta + head : nullptr;
  t.n = n - head;
  t.k0 += head;
  return t;
}

template <int kBits>
struct Step {
  const AdamArgs& a;
  Factors* shared;
  Factors f;
  bool ready = false;

  // The step's factors, which wave 0 has left in LDS.
  __device__ __forceinline__ void wait() {
    if (ready) return;
    __syncthreads();
    f = *shared;
    ready = true;
  }

  template <class P, class G, uint32_t kSteps, bool kFull, bool kStream = false>
  __device__ __forceinline__ void chunk(const AdamPiece& t, uint32_t k) {
    Chunk<P, G, kBits, kSteps> c;
    load_chunk<kFull, kStream>(c, t, k);
    wait();
    if (f.skip) {
      // a change of nothing, so that the codec is not given the last step's
      if (t.delta)
#pragma unroll
        for (uint32_t u = 0; u < kSteps; ++u)
          store_some<kFull, kStream, float>(t.delta, k + u * kStride + threadIdx.x * V, t.n, {});
      return;
    }
    step_chunk<kFull, kStream>(c, t, k, a, f);
  }

  template <class P, class G>
  __device__ __forceinline__ void piece(AdamPiece t) {
    constexpr uint32_t kSteps = adam_steps(kBits);
    uint32_t k = 0;
    if constexpr (kBits == 32) {
      // Pieces of a list larger than the last-level cache go on from where a line of p
      // begins: the states of a flat buffer's tensors begin lines there too.  Whole
      // lines are written, and where all of them do, past the cache (148 tensors of
      // 100M values at odd offsets, 2048 pieces: 571 us without, 549 with whole lines,
      // 525 past the cache; partial lines past the cache 640).  8-bit blocks stay where
      // they are.
      if (a.stream && t.n >= kSteps * kStride) {  // (more values than a head has)
        const uint32_t head = (uint32_t)(-reinterpret_cast<uintptr_t>(t.p) % kLine) / sizeof(P);
        if (head) {
          const uint32_t n = t.n;
          t.n = head;
          chunk<P, G, 1, false>(t, 0);
          t = adam_rest(t, head, n, sizeof(P), sizeof(G));
        }
        if ((reinterpret_cast<uintptr_t>(t.p) | reinterpret_cast<uintptr_t>(t.m) |
             reinterpret_cast<uintptr_t>(t.v) | reinterpret_cast<uintptr_t>(t.delta)) % kLine == 0)
          for (; t.n - k >= kSteps * kStride; k += kSteps * kStride)
            chunk<P, G, kSteps, true, true>(t, k);
      }
    }
    for (; t.n - k >= kSteps * kStride; k += kSteps * kStride) chunk<P, G, kSteps, true>(t, k);
    for (; t.n - k >= kStride; k += kStride) chunk<P, G, 1, true>(t, k);
    if (k < t.n) chunk<P, G, 1, false>(t, k);
  }
  template <class P>
  __device__ __forceinline__ void piece(const AdamPiece& t) {
    const uint32_t type = t.types >> 2;
    if (type == TLC_F32)
      piece<P, float>(t);
    else if (type == TLC_BF16)
      piece<P, bf16_t>(t);
    else
      piece<P, f16_t>(t);
  }
};

}  // namespace

template <class List, int kBits>
__global__ __launch_bounds__(kAdamThreads) void tlc_adamw_kernel(List list, AdamArgs a) {
  __shared__ Factors shared;
  const uint32_t i0 = (uint32_t)((uint64_t)blockIdx.x * list.n / gridDim.x);
  const uint32_t i1 = (uint32_t)((uint64_t)(blockIdx.x + 1) * list.n / gridDim.x);
  AdamPiece t = {};
  if (i0 < i1) t = piece_of(list, i0);  // asked for first: it may be in host memory
  if (threadIdx.x == 0) {
    const int64_t step = a.clock->step + 1;
    shared = factors_of(a, step);
    if (a.result && blockIdx.x == 0) put_result(a.result, clip_of(a.result->sumsq, a.max_norm));
    // (counted before the factors are released, which wait for it; it needs the clock's
    // read alone)
    if (a.tickets && last_to_read(a.tickets, step) && !shared.skip) a.clock->step = step;
  }
  Step<kBits> s{a, &shared, {}};
  for (uint32_t i = i0; i < i1; ++i) {
    if (i > i0) t = piece_of(list, i);
    const uint32_t type = t.types & 3u;
    if (type == TLC_F32)
      s.template piece<float>(t);
    else if (type == TLC_BF16)
      s.template piece<bf16_t>(t);
    else
      s.template piece<f16_t>(t);
  }
}

template <class List>
hipError_t launch_adamw(const List& list, const AdamArgs& a, int state_type, hipStream_t st) {
  const uint32_t grid = std::max(1u, std::min(list.n, kAdamPieces));
  if (state_type == TLC_STATE_8BIT)
    launch_k(tlc_adamw_kernel<List, 8>, grid, kAdamThreads, st, list, a);
  else
    launch_k(tlc_adamw_kernel<List, 32>, grid, kAdamThreads, st, list, a);
  return hipGetLastError();
}

template hipError_t launch_adamw(const AdamList&, const AdamArgs&, int, hipStream_t);
template hipError_t launch_adamw(const AdamPinned&, const AdamArgs&, int, hipStream_t);

}  // namespace tlc
