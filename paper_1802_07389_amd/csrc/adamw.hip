// adamw.hip -- one step of AdamW over a list of tensors, every operation rounded
// to fp32:
//   g' = coef g,  m' = m + (g' - m) c1,  v' = v + (g' g' - v) c2
//   p' = p - (a (m' / (sqrt(v') r + eps)) + w p)
// with c = 1 - beta, a = lr / (1 - beta1^t), r = 1 / sqrt(1 - beta2^t), w = lr decay.
// States of 8 bits hold 256 values by one scale, m as OCP E4M3 and v as OCP E5M2.
// What bounds it: every tensor read and written once (28 bytes an fp32 value of
// fp32 states, 16 of 8 bits).
#include <math.h>

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

// Values k to k + 3 of x, those from n on 0.
template <class T>
__device__ __forceinline__ Pack<T, V> load_some(const T* x, uint32_t k, uint32_t n) {
  if (n - k >= V) return load_pack<T, V>(x + k);
  Pack<T, V> r = {};
#pragma unroll
  for (uint32_t e = 0; e < V; ++e)
    if (e < n - k) r.v[e] = x[k + e];
  return r;
}
template <class T>
__device__ __forceinline__ void store_some(T* x, uint32_t k, uint32_t n, const Pack<T, V>& r) {
  if (n - k >= V) {
    store_pack<T, V>(x + k, r);
    return;
  }
#pragma unroll
  for (uint32_t e = 0; e < V; ++e)
    if (e < n - k) x[k + e] = r.v[e];
}

// Four codes as one word, those from n on 0.
__device__ __forceinline__ uint32_t load_codes(const uint8_t* x, uint32_t k, uint32_t n) {
  if (n - k >= V) return ld_word(x + k);
  uint32_t w = 0;
#pragma unroll
  for (uint32_t e = 0; e < V; ++e)
    if (e < n - k) w |= (uint32_t)x[k + e] << (8 * e);
  return w;
}
__device__ __forceinline__ void store_codes(uint8_t* x, uint32_t k, uint32_t n, uint32_t w) {
  if (n - k >= V) {
    st_word(x + k, w);
    return;
  }
#pragma unroll
  for (uint32_t e = 0; e < V; ++e)
    if (e < n - k) x[k + e] = (uint8_t)(w >> (8 * e));
}

// The code of y >= 0 in a format of kMantissa bits with smallest exponent kLowest
// (below it steps are even) and largest code kMost: the codes joined by straight
// lines make y a place between two of them, which `dither` (of the 23 - kMantissa
// bits that are cut off) carries to the upper one as often as y is near it.
template <int kMantissa, int kLowest, uint32_t kMost>
__device__ __forceinline__ uint32_t fp8_code(float y, uint32_t dither) {
  constexpr int kCut = 23 - kMantissa;
  constexpr float kUnit = 1.0f / (float)(1ull << -kLowest);  // 2^kLowest
  const uint32_t fine =
      ((__float_as_uint(y) + dither) >> kCut) - ((uint32_t)(126 + kLowest) << kMantissa);
  constexpr float kFine = (float)(1ull << (kMantissa - kLowest + kCut));
  const uint32_t small = ((uint32_t)(fminf(y, kUnit) * kFine) + dither) >> kCut;
  return umin32(y < kUnit ? small : fine, kMost);
}

// A block's scale from its largest magnitude (as bits): its share of the
// format's largest number (inv_most: 1 / that), at least 2^-126 so that it
// divides; NaN where a value is NaN or infinite.
__device__ __forceinline__ float scale_of_max(uint32_t bits, float inv_most) {
  if (bits == 0) return 0.0f;
  if (bits >= 0x7f800000u) return __builtin_nanf("");
  return fmaxf(__uint_as_float(bits) * inv_most, 0x1p-126f);
}

constexpr uint32_t kDitherK = 0xC13FA9A9u, kDitherT = 0x91E10DA5u;

// A piece of a tensor: its values from k0 on.
struct AdamPiece {
  void* p;
  const void* g;
  void* m;
  void* v;
  float* scales;
  float* delta;
  uint32_t k0, n;
};

// Values k to k + 3 of a piece.
template <class P, class G, int kBits>
__device__ __forceinline__ void step_four(const AdamPiece& t, uint32_t k, const AdamArgs& a,
                                          const Factors& f) {
  const bool in = k < t.n;  // of 8 bits the whole wave stays for its block's largest
  if (kBits == 32 && !in) return;
  float m[V] = {}, v[V] = {};
  Pack<P, V> p = {};
  Pack<G, V> g = {};
  if (in) {
    p = load_some(static_cast<const P*>(t.p), k, t.n);
    g = load_some(static_cast<const G*>(t.g), k, t.n);
    if constexpr (kBits == 32) {
      const Pack<float, V> pm = load_some(static_cast<const float*>(t.m), k, t.n);
      const Pack<float, V> pv = load_some(static_cast<const float*>(t.v), k, t.n);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        m[e] = pm.get(e);
        v[e] = pv.get(e);
      }
    } else {
      const int wm = (int)load_codes(static_cast<const uint8_t*>(t.m), k, t.n);
      const int wv = (int)load_codes(static_cast<const uint8_t*>(t.v), k, t.n);
      const float* s = t.scales + k / TLC_STATE_BLOCK * 2;
      const float sm = s[0], sv = s[1];
      m[0] = __builtin_amdgcn_cvt_f32_fp8(wm, 0) * sm;
      m[1] = __builtin_amdgcn_cvt_f32_fp8(wm, 1) * sm;
      m[2] = __builtin_amdgcn_cvt_f32_fp8(wm, 2) * sm;
      m[3] = __builtin_amdgcn_cvt_f32_fp8(wm, 3) * sm;
      v[0] = __builtin_amdgcn_cvt_f32_bf8(wv, 0) * sv;
      v[1] = __builtin_amdgcn_cvt_f32_bf8(wv, 1) * sv;
      v[2] = __builtin_amdgcn_cvt_f32_bf8(wv, 2) * sv;
      v[3] = __builtin_amdgcn_cvt_f32_bf8(wv, 3) * sv;
    }
  }
  Pack<P, V> q;
  Pack<float, V> d;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const float old = p.get(e);
    q.set(e, adam_step(old, f.coef * g.get(e), m[e], v[e], a, f));
    d.set(e, q.get(e) - old);
  }
  if (in) {
    store_some(static_cast<P*>(t.p), k, t.n, q);
    if (t.delta) store_some(t.delta, k, t.n, d);
  }
  if constexpr (kBits == 32) {
    Pack<float, V> pm, pv;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      pm.set(e, m[e]);
      pv.set(e, v[e]);
    }
    store_some(static_cast<float*>(t.m), k, t.n, pm);
    store_some(static_cast<float*>(t.v), k, t.n, pv);
  } else {
    uint32_t mm = 0, mv = 0;
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (k + e < t.n) {  // beyond the end nothing is held
        mm = umax32(mm, abs_bits(m[e]));
        mv = umax32(mv, abs_bits(v[e]));
      }
    const float sm = scale_of_max(wave_max(mm), 1.0f / 448.0f);
    const float sv = scale_of_max(wave_max(mv), 1.0f / 57344.0f);
    uint32_t wm = 0, wv = 0;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const uint32_t h = (t.k0 + k + e) * kDitherK + f.step * kDitherT;
      const float ym = sm > 0.0f ? fabsf(m[e]) / sm : 0.0f;
      const float yv = sv > 0.0f ? v[e] / sv : 0.0f;
      uint32_t qm = fp8_code<3, -6, 126>(ym, h >> 12);
      uint32_t qv = fp8_code<2, -14, 123>(yv, (h ^ 0x80000000u) >> 11);
      qm |= __float_as_uint(m[e]) >> 31 << 7;
      if (qv == 0 && v[e] > 0.0f) qv = 1;  // a nonzero v stays one
      if (!(sm >= 0.0f)) qm = 0;
      if (!(sv >= 0.0f)) qv = 0;
      wm |= qm << (8 * e);
      wv |= qv << (8 * e);
    }
    if (in) {
      store_codes(static_cast<uint8_t*>(t.m), k, t.n, wm);
      store_codes(static_cast<uint8_t*>(t.v), k, t.n, wv);
      if (k % TLC_STATE_BLOCK == 0) {
        t.scales[k / TLC_STATE_BLOCK * 2] = sm;
        t.scales[k / TLC_STATE_BLOCK * 2 + 1] = sv;
      }
    }
  }
}

template <class P, class G, int kBits>
__device__ __forceinline__ void step_piece(const AdamTensor& t, uint32_t k0, uint32_t len,
                                           const AdamArgs& a, const Factors& f) {
  constexpr uint32_t kState = kBits == 32 ? 4 : 1;
  AdamPiece r;
  r.p = static_cast<P*>(t.p) + k0;
  r.g = static_cast<const G*>(t.g) + k0;
  r.m = static_cast<uint8_t*>(t.m) + (uint64_t)k0 * kState;
  r.v = static_cast<uint8_t*>(t.v) + (uint64_t)k0 * kState;
  r.scales = t.scales + k0 / TLC_STATE_BLOCK * 2;
  r.delta = t.delta ? t.delta + k0 : nullptr;
  r.k0 = k0;
  r.n = umin32(len, t.n - k0);
  for (uint32_t k = 0; k < r.n; k += kAdamThreads * V)
    step_four<P, G, kBits>(r, k + threadIdx.x * V, a, f);
}

}  // namespace

template <int kBits>
__global__ __launch_bounds__(kAdamThreads) void tlc_adamw_kernel(AdamList list, AdamArgs a) {
  __shared__ Factors shared;
  if (threadIdx.x == 0) {
    const int64_t step = a.clock->step + 1;
    shared = factors_of(a, step);
    if (a.result && blockIdx.x == 0) put_result(a.result, clip_of(a.result->sumsq, a.max_norm));
    if (a.ticket) {
      // the block that is last to have read the clock sets it; the read is done
      // when its value is added
      uint32_t one = 1u;
      asm volatile("" : "+v"(one) : "v"((uint32_t)step), "v"(shared.coef));
      if (atomicAdd(a.ticket, one) == gridDim.x - 1) {
        if (!shared.skip) a.clock->step = step;
        *a.ticket = 0u;
      }
    }
  }
  __syncthreads();
  const Factors f = shared;
  const uint32_t lane = threadIdx.x & 63u;
  for (uint32_t i = blockIdx.x; i < list.n; i += gridDim.x) {
    const uint32_t s = (uint32_t)__popcll(__ballot(
        lane < list.count && (list.tensors[lane].piece0_types & 0xfffffffu) <= i));
    const AdamTensor& t = list.tensors[uniform32(s) - 1];
    const uint32_t k0 = (i - (t.piece0_types & 0xfffffffu)) * list.len;
    if (f.skip) {
      // a change of nothing, so that the codec is not given the last step's
      const uint32_t n = umin32(list.len, t.n - k0);
      if (t.delta)
        for (uint32_t k = threadIdx.x; k < n; k += kAdamThreads) t.delta[(uint64_t)k0 + k] = 0.0f;
      continue;
    }
    const auto with = [&](auto p, auto g) {
      step_piece<decltype(p), decltype(g), kBits>(t, k0, list.len, a, f);
    };
    const auto with_p = [&](auto p) {
      const uint32_t type = t.piece0_types >> 30;
      if (type == TLC_F32)
        with(p, float());
      else if (type == TLC_BF16)
        with(p, bf16_t());
      else
        with(p, f16_t());
    };
    const uint32_t type = (t.piece0_types >> 28) & 3u;
    if (type == TLC_F32)
      with_p(float());
    else if (type == TLC_BF16)
      with_p(bf16_t());
    else
      with_p(f16_t());
  }
}

hipError_t launch_adamw(const AdamList& list, const AdamArgs& a, int state_type, hipStream_t st) {
  const uint32_t grid = std::max(1u, std::min(list.n, kNormBlocks));
  if (state_type == TLC_STATE_8BIT)
    launch_k(tlc_adamw_kernel<8>, grid, kAdamThreads, st, list, a);
  else
    launch_k(tlc_adamw_kernel<32>, grid, kAdamThreads, st, list, a);
  return hipGetLastError();
}

}  // namespace tlc
