// embedding_grad.hip -- the gradient of an embedding table: the tokens sorted
// by their rows, and every row's sum over its run of tokens.
//
//   out[v, :] = (accumulate ? out[v, :] : 0) + scale * sum grad[t, :], ids[t] == v
//
// What bounds it: grad read once and out written once.  The tokens' numbers are
// sorted (stably, so that a row adds its tokens in their order) by counting
// passes over the digits of their rows; a wave then takes a fixed number of
// sorted tokens and a slab of columns, holds the running sum of a run in
// registers, and joins what a run leaves in several waves through LDS and, past
// a block, through partial rows in the workspace.  So a row that has half of all
// tokens is spread over the chip like any other, no atomics order anything,
// and the bits depend on the sizes and ids alone.  Rows without a token are
// zeroed by blocks beside the sorting ones, which leave the memory idle.
#include "device_common.hpp"
#include "train_internal.h"
#include "typed_io.hpp"

namespace tlc {
namespace {

constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortItems = kSortTile / kSortThreads;

// The key a token is sorted by: its row, or `rows` (after all others) where it
// adds nothing.
template <class Id>
__device__ __forceinline__ uint32_t token_key(const EmbArgs& a, uint32_t t) {
  const int64_t id = static_cast<const Id*>(a.ids)[t];
  if (id >= 0 && id == a.padding) return a.rows;
  if (id < 0 || id >= (int64_t)a.rows) {
    host_put(a.bad, 1u);
    return a.rows;
  }
  return (uint32_t)id;
}

// Zeroes the rows of block b of the fill that no token touched.
template <uint32_t kBlock>
__device__ __forceinline__ void fill_rows(const FillArgs& f, uint32_t b) {
  const uint64_t r0 = (uint64_t)b * f.block_rows;
  const uint32_t n = (uint32_t)umin64(f.block_rows, f.rows - r0) * f.packs.d;
  float* out = f.out + r0 * f.out_stride;
  for (uint32_t u = threadIdx.x; u < n; u += kBlock) {
    const uint32_t r = quotient(u, f.packs);
    if (f.touched[r0 + r]) continue;
    float* o = out + r * f.out_stride;
    const uint32_t j = u - r * f.packs.d;
    if (f.dim >= 4)
      st4(o + umin32(j * 4, f.dim - 4), make_float4(0.0f, 0.0f, 0.0f, 0.0f));
    else
      o[j] = 0.0f;
  }
}

}  // namespace

// The keys, the counts of every tile's first digits, and the rows that any
// token touches (touched NULL: not wanted).  Clears the counts of the passes
// after the first (next1, next2: may be NULL).
template <class Id>
__global__ __launch_bounds__(kSortThreads) void tlc_token_count_kernel(
    EmbArgs a, uint32_t* __restrict__ keys, uint8_t* __restrict__ touched,
    uint32_t* __restrict__ counts, uint32_t* __restrict__ next1, uint32_t* __restrict__ next2,
    uint32_t digits) {
  __shared__ uint32_t n[kSortMaxDigits];
  for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) n[d] = 0u;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const uint32_t t = blockIdx.x * kSortTile + i * kSortThreads + threadIdx.x;
    if (t >= a.count) break;
    const uint32_t key = token_key<Id>(a, t);
    keys[t] = key;
    if (touched && key < a.rows) touched[key] = 1;
    atomicAdd(&n[key & (digits - 1)], 1u);
  }
  __syncthreads();
  const uint64_t at = (uint64_t)blockIdx.x * digits;
  for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) {
    counts[at + d] = n[d];
    if (next1) next1[at + d] = 0u;
    if (next2) next2[at + d] = 0u;
  }
}

// One pass: the tile's keys go where the counts of all tiles send them, those
// of equal digits in their order.  A wave ranks 64 neighbouring keys at a time
// by the ballots of their digits' bits.  Counts the next pass's digits (by the
// tile that a key goes to), one addition for all neighbours that share digit and
// tile.  Blocks from `tiles` on fill rows instead.
__global__ __launch_bounds__(kSortThreads) void tlc_token_sort_kernel(SortArgs s, FillArgs f) {
  __shared__ uint16_t wave_n[kSortWaves][kSortMaxDigits];
  __shared__ uint32_t base[kSortMaxDigits];
  __shared__ uint32_t scan_lds[kSortWaves];
  if (blockIdx.x >= s.tiles) {
    fill_rows<kSortThreads>(f, f.block0 + blockIdx.x - s.tiles);
    return;
  }
  const uint32_t lane = threadIdx.x & 63u, wid = threadIdx.x >> 6;
  const uint32_t digits = 1u << s.bits;
  constexpr uint32_t kPer = kSortMaxDigits / kSortThreads;
  // where the tile's keys of every digit start
  uint32_t before[kPer];
#pragma unroll
  for (uint32_t i = 0; i < kPer; ++i) {
    const uint32_t d = threadIdx.x + i * kSortThreads;
    before[i] = 0;
    if (d >= digits) break;
    uint32_t total = 0;
#pragma unroll 8
    for (uint32_t t = 0; t < s.tiles; ++t) {
      const uint32_t v = s.counts[(uint64_t)t * digits + d];
      before[i] += t < blockIdx.x ? v : 0u;
      total += v;
    }
    base[d] = total;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) wave_n[w][d] = 0;
  }
  __syncthreads();
  const uint32_t d0 = threadIdx.x * kPer;
  uint32_t own[kPer], sum = 0;
#pragma unroll
  for (uint32_t i = 0; i < kPer; ++i) {
    own[i] = d0 + i < digits ? base[d0 + i] : 0u;
    sum += own[i];
  }
  uint32_t excl = block_scan_u32<kSortWaves>(sum, scan_lds).excl;
#pragma unroll
  for (uint32_t i = 0; i < kPer; ++i) {
    if (d0 + i < digits) base[d0 + i] = excl;
    excl += own[i];
  }
  // rank within the wave
  const uint32_t t0 = blockIdx.x * kSortTile + wid * (64 * kSortItems) + lane;
  uint32_t key[kSortItems], pos[kSortItems], rank[kSortItems];
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const uint32_t t = t0 + i * 64;
    key[i] = t < s.count ? s.keys_in[t] : 0u;
    pos[i] = t < s.count && s.pos_in ? s.pos_in[t] : t;
  }
  const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const bool in = t0 + i * 64 < s.count;
    const uint32_t d = (key[i] >> s.shift) & (digits - 1);
    uint64_t same = __ballot(in);
    for (uint32_t b = 0; b < s.bits; ++b) {
      const uint64_t m = __ballot((d >> b) & 1u);
      same &= (d >> b) & 1u ? m : ~m;
    }
    if (in) rank[i] = wave_n[wid][d] + (uint32_t)__popcll(same & below);
    // every lane has read the count before the run's first lane raises it
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (in && (same & below) == 0) wave_n[wid][d] += (uint16_t)__popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
#pragma unroll
  for (uint32_t i = 0; i < kPer; ++i) {
    const uint32_t d = threadIdx.x + i * kSortThreads;
    if (d >= digits) break;
    uint32_t n = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t v = wave_n[w][d];
      wave_n[w][d] = (uint16_t)n;
      n += v;
    }
    base[d] += before[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const bool in = t0 + i * 64 < s.count;
    const uint32_t d = (key[i] >> s.shift) & (digits - 1);
    const uint32_t to = in ? base[d] + wave_n[wid][d] + rank[i] : 0u;
    if (in) {
      s.keys_out[to] = key[i];
      s.pos_out[to] = pos[i];
    }
    if (s.next) {
      const uint32_t nd = (key[i] >> (s.shift + s.bits)) & ((1u << s.next_bits) - 1);
      // lanes of one digit go to neighbouring places: their tiles differ by
      // at most one, so that the tile's parity tells them apart
      const uint32_t word = d | nd << s.bits;
      uint64_t same = __ballot(in);
      for (uint32_t b = 0; b < s.bits + s.next_bits; ++b) {
        const uint64_t m = __ballot((word >> b) & 1u);
        same &= (word >> b) & 1u ? m : ~m;
      }
      const uint32_t odd = (to / kSortTile) & 1u;
      const uint64_t m = __ballot(odd);
      same &= odd ? m : ~m;
      if (in && (same & below) == 0)
        atomicAdd(&s.next[((uint64_t)(to / kSortTile) << s.next_bits) + nd],
                  (uint32_t)__popcll(same));
    }
  }
}

namespace {

// V columns of one run's sum.
template <int V>
struct Sum {
  float v[V];
  __device__ __forceinline__ void add(const float* p) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] += p[i];
  }
};

template <int V>
__device__ __forceinline__ void put_floats(float* p, const float* v) {
  Pack<float, V> o;
#pragma unroll
  for (int i = 0; i < V; ++i) o.set(i, v[i]);
  store_pack<float, V>(p, o);
}

// A row's final values: the scale once, on the whole sum.
template <int V>
__device__ __forceinline__ void put_row(const EmbArgs& a, uint32_t row, uint32_t k, const float* v,
                                        bool accumulate) {
  float* p = static_cast<float*>(a.out) + row * a.out_stride + k;
  Pack<float, V> o;
  if (accumulate) {
    o = load_pack<float, V>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) o.set(i, o.get(i) + a.scale * v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) o.set(i, a.scale * v[i]);
  }
  store_pack<float, V>(p, o);
}

}  // namespace

// Every wave: `per_wave` sorted tokens (at most 64) of one slab of columns.  Its
// runs are summed eight rows at a time; one that neither began before the wave
// nor goes on after it is final.  The others' parts meet in LDS: the wave where a
// run begins adds the parts of the block's later waves, and leaves the sum as
// the block's tail if the run goes on in the next block; what the block adds to
// a run that began earlier is its head.
template <class In, int V>
__global__ __launch_bounds__(kSumThreads) void tlc_embedding_grad_sum_kernel(EmbArgs a, SumArgs s,
                                                                             bool accumulate,
                                                                             FillArgs f) {
  constexpr int kRows = 8;  // rows in flight
  __shared__ float lds[kSumWaves][64 * V];
  __shared__ uint32_t lds_head[kSumWaves];  // 1: has a head; 2: the run goes on
  if (blockIdx.x >= s.blocks * s.slabs) {
    fill_rows<kSumThreads>(f, f.block0 + blockIdx.x - s.blocks * s.slabs);
    return;
  }
  const uint32_t lane = threadIdx.x & 63u, wid = uniform32(threadIdx.x >> 6);
  const uint32_t block = blockIdx.x / s.slabs, slab = blockIdx.x % s.slabs;
  // packs of the slab; the last of a row is moved back to end with it, beside
  // the pack that it overlaps (both lanes load before either stores)
  const uint32_t p0 = (uint32_t)((uint64_t)slab * s.packs / s.slabs);
  const uint32_t p1 = (uint32_t)((uint64_t)(slab + 1) * s.packs / s.slabs);
  const bool in = p0 + lane < p1;
  const uint32_t k = umin32((p0 + lane) * V, a.dim - V);
  const uint32_t c0 = umin32((block * kSumWaves + wid) * s.per_wave, a.count);
  const uint32_t c1 = umin32(c0 + s.per_wave, a.count);
  const uint32_t key = c0 + lane < c1 ? s.keys[c0 + lane] : a.rows;
  const uint32_t pos = c0 + lane < c1 ? s.pos[c0 + lane] : 0u;
  const uint32_t prev = c0 > 0 && c0 < c1 ? s.keys[c0 - 1] : a.rows;
  const uint32_t next = c1 < a.count ? s.keys[c1] : a.rows;
  const uint32_t n = (uint32_t)__popcll(__ballot(key < a.rows));
  const In* x = static_cast<const In*>(a.x) + k;
  Sum<V> sum = {};
  uint32_t cur = uniform32(key);
  bool first = n > 0 && uniform32(prev) == cur;  // the run began before
  uint32_t head = first ? 1u : 0u;
  for (uint32_t e = 0; e < n; e += kRows) {
    Pack<In, V> r[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const uint32_t t =
          (uint32_t)__builtin_amdgcn_readlane((int)pos, (int)umin32(e + i, n - 1));
      if (in) r[i] = load_pack<In, V>(x + (uint64_t)t * a.x_stride);
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      if (e + i >= n) break;
      const uint32_t row = (uint32_t)__builtin_amdgcn_readlane((int)key, (int)(e + i));
      if (row != cur) {
        if (in) {
          if (first)
            put_floats<V>(&lds[wid][lane * V], sum.v);
          else
            put_row<V>(a, cur, k, sum.v, accumulate);
        }
        first = false;
        cur = row;
        sum = {};
      }
      if (in) {
#pragma unroll
        for (int c = 0; c < V; ++c) sum.v[c] += r[i].get(c);
      }
    }
  }
  const bool on = n > 0 && uniform32(next) == cur;
  const bool tail = on && !first;
  if (n > 0 && in) {
    if (first)
      put_floats<V>(&lds[wid][lane * V], sum.v);
    else if (!on)
      put_row<V>(a, cur, k, sum.v, accumulate);
  }
  if (first && on) head = 3u;
  if (lane == 0) lds_head[wid] = head;
  __syncthreads();
  float* parts = s.parts + (uint64_t)block * 2 * a.dim + k;
  if (tail) {
    bool ends = false;
    for (uint32_t w = wid + 1; w < kSumWaves && !ends; ++w) {
      if (in) sum.add(&lds[w][lane * V]);
      ends = lds_head[w] == 1u;
    }
    if (in) {
      if (ends)
        put_row<V>(a, cur, k, sum.v, accumulate);
      else
        put_floats<V>(parts + a.dim, sum.v);
    }
  }
  if (wid == 0 && lds_head[0]) {
    sum = {};
    uint32_t w = 0;
    do {
      if (in) sum.add(&lds[w][lane * V]);
    } while (lds_head[w] == 3u && ++w < kSumWaves);
    if (in) put_floats<V>(parts, sum.v);
  }
}

// Runs that go on past a block: the block where one begins adds its tail and
// the heads of the blocks after it, in their order.  Also leaves the
// touched rows' marks as they were before the call.
template <int V>
__global__ __launch_bounds__(kJoinThreads) void tlc_embedding_grad_join_kernel(
    EmbArgs a, SumArgs s, bool accumulate, uint8_t* __restrict__ touched) {
  constexpr int kParts = 8;  // partial rows in flight
  constexpr uint32_t kWavesJ = kJoinThreads / 64;
  __shared__ float lds[kWavesJ][64 * V];
  __shared__ uint32_t heads;
  const uint32_t lane = threadIdx.x & 63u, wid = uniform32(threadIdx.x >> 6);
  const uint32_t len = s.per_wave * kSumWaves;
  const uint32_t c0 = blockIdx.x * len, c1 = umin32(c0 + len, a.count);
  if (touched && blockIdx.y == 0)
    for (uint32_t c = c0 + threadIdx.x; c < c1; c += kJoinThreads)
      if (s.keys[c] < a.rows) touched[s.keys[c]] = 0;
  if (c1 >= a.count) return;
  const uint32_t row = uniform32(s.keys[c1 - 1]);
  if (row >= a.rows || uniform32(s.keys[c1]) != row) return;
  if (c0 > 0 && uniform32(s.keys[c0 - 1]) == row) return;
  if (threadIdx.x == 0) heads = 0;
  __syncthreads();
  uint32_t mine = 0;
  for (uint32_t b = blockIdx.x + 1 + threadIdx.x; b < s.blocks; b += kJoinThreads) {
    if (s.keys[b * len] != row) break;
    ++mine;
  }
  if (mine) atomicAdd(&heads, mine);
  __syncthreads();
  const uint32_t n = 1 + uniform32(heads);  // the tail, then the heads
  const uint32_t per = (n + kWavesJ - 1) / kWavesJ;
  const uint32_t i0 = umin32(wid * per, n), i1 = umin32(i0 + per, n);
  const uint32_t packs = (a.dim + V - 1) / V, slabs = (packs + 63) / 64;
  for (uint32_t slab = blockIdx.y; slab < slabs; slab += gridDim.y) {
    const uint32_t p0 = (uint32_t)((uint64_t)slab * packs / slabs);
    const uint32_t p1 = (uint32_t)((uint64_t)(slab + 1) * packs / slabs);
    const bool in = p0 + lane < p1;
    const uint32_t k = umin32((p0 + lane) * V, a.dim - V);
    const float* parts = s.parts + (uint64_t)blockIdx.x * 2 * a.dim + k;
    Sum<V> sum = {};
    if (in) {
      for (uint32_t i = i0; i < i1; i += kParts) {
        Pack<float, V> r[kParts];
#pragma unroll
        for (int j = 0; j < kParts; ++j) {
          const uint32_t at = umin32(i + j, i1 - 1);
          r[j] = load_pack<float, V>(parts + (at ? (uint64_t)at * 2 : 1) * a.dim);
        }
#pragma unroll
        for (int j = 0; j < kParts; ++j) {
#pragma unroll
          for (int c = 0; c < V; ++c) sum.v[c] += i + j < i1 ? r[j].get(c) : 0.0f;
        }
      }
      put_floats<V>(&lds[wid][lane * V], sum.v);
    }
    __syncthreads();
    if (wid == 0 && in) {
      for (uint32_t w = 1; w < kWavesJ && w * per < n; ++w) sum.add(&lds[w][lane * V]);
      put_row<V>(a, row, k, sum.v, accumulate);
    }
    __syncthreads();
  }
}

namespace {

template <class In, int V>
void launch_sum(const EmbArgs& a, SumArgs s, bool accumulate, const FillArgs& f, uint32_t fill,
                hipStream_t st) {
  launch_k(tlc_embedding_grad_sum_kernel<In, V>, s.blocks * s.slabs + fill, kSumThreads, st, a, s,
           accumulate, f);
}

}  // namespace

hipError_t launch_embedding_grad(const EmbArgs& a, int grad_type, int ids_type, bool accumulate,
                                 const GradWork& w, hipStream_t st) {
  FillArgs f = {};
  uint32_t fill = 0;  // blocks that zero rows
  if (!accumulate) {
    const uint32_t packs = a.dim >= 4 ? (a.dim + 3) / 4 : a.dim;
    f.out = static_cast<float*>(a.out);
    f.out_stride = a.out_stride;
    f.touched = w.touched;
    f.rows = a.rows;
    f.dim = a.dim;
    f.packs = divider(packs);
    f.block_rows = std::max(1u, kFillPacks / packs);
    fill = (a.rows + f.block_rows - 1) / f.block_rows;
  }
  // passes of equal digits over the bits of 0 .. rows
  const uint32_t bits = 32 - (uint32_t)__builtin_clz(a.rows);
  const uint32_t passes = (bits + kSortMaxBits - 1) / kSortMaxBits;
  const uint32_t digit = (bits + passes - 1) / passes;
  const uint32_t tiles = (a.count + kSortTile - 1) / kSortTile;
  if (tiles) {
    uint8_t* touched = accumulate ? nullptr : w.touched;
    uint32_t* next1 = passes > 1 ? w.counts[1] : nullptr;
    uint32_t* next2 = passes > 2 ? w.counts[2] : nullptr;
    if (ids_type == TLC_I64)
      launch_k(tlc_token_count_kernel<int64_t>, tiles, kSortThreads, st, a, w.keys[0], touched,
               w.counts[0], next1, next2, 1u << digit);
    else
      launch_k(tlc_token_count_kernel<int32_t>, tiles, kSortThreads, st, a, w.keys[0], touched,
               w.counts[0], next1, next2, 1u << digit);
  }
  for (uint32_t p = 0; p < passes; ++p) {
    SortArgs s = {};
    s.keys_in = w.keys[p & 1];
    s.pos_in = p ? w.pos[p & 1] : nullptr;
    s.keys_out = w.keys[(p + 1) & 1];
    s.pos_out = w.pos[(p + 1) & 1];
    s.counts = w.counts[p];
    s.next = p + 1 < passes ? w.counts[p + 1] : nullptr;
    s.count = a.count;
    s.tiles = tiles;
    s.shift = p * digit;
    s.bits = digit;
    s.next_bits = digit;
    // the rest of the fill goes beside the last pass where no sums follow
    const uint32_t beside = tiles ? std::min(fill, kFillBeside) : fill;
    if (tiles + beside) launch_k(tlc_token_sort_kernel, tiles + beside, kSortThreads, st, s, f);
    f.block0 += beside;
    fill -= beside;
  }
  if (tiles == 0) return hipGetLastError();
  SumArgs s = {};
  s.keys = w.keys[passes & 1];
  s.pos = w.pos[passes & 1];
  s.parts = w.parts;
  const uint32_t pack = grad_type == TLC_F32 ? 4 : 8;
  s.packs = a.dim >= pack ? (a.dim + pack - 1) / pack : a.dim;
  s.slabs = (s.packs + 63) / 64;
  s.per_wave = sum_per_wave(a.count, s.slabs);
  s.blocks = (a.count + s.per_wave * kSumWaves - 1) / (s.per_wave * kSumWaves);
  with_type(grad_type, [&](auto in) {
    using In = decltype(in);
    if (a.dim >= 16 / sizeof(In))
      launch_sum<In, 16 / sizeof(In)>(a, s, accumulate, f, fill, st);
    else
      launch_sum<In, 1>(a, s, accumulate, f, fill, st);
  });
  uint8_t* touched = accumulate ? nullptr : w.touched;
  if (s.blocks > 1 || touched) {
    if (a.dim >= 4)
      launch_k(tlc_embedding_grad_join_kernel<4>,
               dim3(s.blocks, std::min((a.dim + 255) / 256, 8u)), kJoinThreads, st, a, s,
               accumulate, touched);
    else
      launch_k(tlc_embedding_grad_join_kernel<1>, dim3(s.blocks, 1), kJoinThreads, st, a, s,
               accumulate, touched);
  }
  return hipGetLastError();
}

}  // namespace tlc
