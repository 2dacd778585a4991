// train_internal.h -- definitions shared by the kernels of the training step
// (embedding tables, gradient norm, token log probabilities, AdamW) and their host
// side (not part of the public ABI).
#pragma once

#include <float.h>

#include "tlc_internal.h"
#include "typed_io.hpp"

namespace tlc {

constexpr uint32_t kEmbThreads = 256;

// One call on a table.
struct EmbArgs {
  const void* x;      // the table, or the tokens' gradients
  const void* ids;
  void* out;
  uint64_t x_stride, out_stride;  // values
  uint32_t count, rows, dim;
  float scale;
  int64_t padding;    // gradient: tokens of this id add nothing
  bool wide_ids;      // gradient: ids are int64
  uint32_t* bad;      // pinned host word: set where an id is outside the table
};

hipError_t launch_embedding(const EmbArgs& a, int table_type, int ids_type, int out_type,
                            hipStream_t st);

// The gradient's sort by digits of the tokens' rows (heights below 2^18 in two
// passes).  Up to kSmallTokens tokens every block of the sums sorts them in LDS;
// more are sorted first, in tiles of two tokens a thread, from kTile4Tokens on of
// four: small tiles fill the chip, but every tile's block reads the counts of all,
// or all have to be scanned (two | four a thread, 8 fp32 values a token added:
// 30000 tokens 33 | 35 us, 65536 34 | 36, 130000 52 | 47, 500000 94 | 94, 2000000
// 252 | 249; of one value 2^24 1.70 | 1.56 ms, 2^27 13.7 | 12.5; sixteen a thread 50
// us for 30000, 0.26 ms for 2000000, 11.7 ms for 2^27).
constexpr uint32_t kDigitBits = 9;
constexpr uint32_t kDigits = 1u << kDigitBits;
constexpr uint32_t kSortThreads = 512;
constexpr uint32_t kSortTile = kSortThreads * 2;  // the smallest
constexpr uint32_t kSmallThreads = 512;
// (One launch | sorted first, 512 bf16 values a token added: 1000 tokens of common
// ids 8.6 | 18.0 us, of three ids in all 12.9 | 17.6; 2000 tokens 13.2 | 19.3 and
// 19.9 | 18.5.  The host does not know the ids; with twice as many tokens the wave
// that has a common id to itself takes longer than the sort.)
constexpr uint32_t kSmallTokens = kSmallThreads * 4;
constexpr uint32_t kSortPasses = 4;  // at most, of 31 bits
// Up to kNextTiles tiles a pass counts the next one's digits, which saves that
// pass's count (10000 tokens 30 | 33 us).  Its counters are in LDS, which leaves
// fewer blocks a CU to fill beside: with room for 28 tiles 16384 tokens of 1024
// values, 65536 rows set, take 67 instead of 62 us.
constexpr uint32_t kNextTiles = 16;
constexpr uint32_t kXcds = 8;
constexpr uint32_t kTile4Tokens = 1u << 16;
// Above kScanTiles tiles a launch of its own turns a pass's counts into their
// prefixes, so that what the blocks read does not grow with the square of the
// tiles (every block reading all counts | prefixes, two passes over tokens of one
// value: 200000 tokens, 98 tiles, 52 | 54 us; 500000 88 | 83; in tiles of sixteen a
// thread, 2^20 tokens 145 | 145, 2^21 244 | 235, 2^24 2.15 | 1.54 ms, 2^27 102 | 11.7).
constexpr uint32_t kScanTiles = 128;
constexpr uint32_t kScanDigits = 16;  // of a block: 64 bytes of every tile's counts
constexpr uint32_t kScanThreads = 512;
struct SortArgs {
  const uint32_t* keys_in;
  const uint32_t* pos_in;  // NULL: the tokens in their order
  uint32_t* keys_out;
  uint32_t* pos_out;
  uint32_t* counts;  // per tile and digit
  uint32_t* totals;  // per digit; counts then hold prefixes.  NULL: they are counts
  uint32_t* next;    // the next pass's, or NULL
  uint32_t count, tiles, shift;
  uint32_t clear;    // tables to clear behind counts
};
// Zeroes for the rows that no token touches.
struct FillArgs {
  float* out;
  uint64_t out_stride;
  const uint8_t* touched;
  uint64_t rows;
  uint32_t dim;
  Divider packs;     // float4s (or, of shorter rows, floats) of a row
  uint32_t blocks;   // of the launch
  // beside the sort: tiles of kSortThreads packs at most
  uint32_t tiles, tile0, tile1;  // all, and the launch's
  uint32_t tile_rows;            // rows of a tile (1 where a row has several)
  Divider row_tiles;             // tiles of a row
  // few tokens: groups of rows, `stride` groups from one of a block's to the next
  Divider group, stride;
};
constexpr uint32_t kFillBlocks = 1u << 20;  // of a launch
// Above so many values to set, few tokens are sorted first too: the sort is over
// before the zeroes are written, which tiles do faster than blocks that look at
// all ids (one launch | sorted first, 1000 tokens: 41 MB 12.9 | 24.4 us, 102 MB
// 23.6 | 32.0, 205 MB 44 | 45, 410 MB 85 | 75, 1065 MB 225 | 174).
constexpr uint64_t kSmallFillValues = 50000000;
constexpr uint32_t kSmallFillBlocks = 1024;
constexpr uint32_t kSmallFillRows = 8192;   // of a block
// The sums: kSumWaves waves of a block, each per_wave sorted tokens.
constexpr uint32_t kSumThreads = 256;
constexpr uint32_t kSumWaves = kSumThreads / 64;
constexpr uint32_t kSumMinTokens = 16, kSumMaxTokens = 64;  // of a wave
constexpr uint32_t kJoinThreads = 256;
struct SumArgs {
  const uint32_t* keys;  // sorted; `rows` and above: adds nothing
  const uint32_t* pos;
  float* parts;          // per block of tokens: head, tail (dim values each)
  uint32_t packs, slabs, blocks;
  uint32_t per_wave;     // sorted tokens (few tokens: of a block)
};
inline uint32_t sum_per_wave(uint32_t count, uint32_t slabs) {
  const uint64_t each = (uint64_t)count * slabs / 4096 / 8 * 8;
  return (uint32_t)std::min<uint64_t>(std::max<uint64_t>(each, kSumMinTokens), kSumMaxTokens);
}
// Device memory of the gradient; touched is zero between calls.
struct GradWork {
  uint32_t* keys[2];
  uint32_t* pos[2];
  uint32_t* counts;  // kSortPasses tables
  uint8_t* touched;
  float* parts;
};
hipError_t launch_embedding_grad(const EmbArgs& a, int grad_type, bool accumulate,
                                 const GradWork& w, hipStream_t st);

// A list of tensors is cut into pieces of one length (the last of a tensor
// shorter), a block each up to kNormBlocks of them; of more (very many tensors) a
// block takes consecutive ones.
struct Piece {
  const void* x;
  void* out;
  uint32_t n;
  uint32_t type;
};
static_assert(sizeof(Piece) == 24, "Piece is 24 bytes");
constexpr uint32_t kNormThreads = 256;
constexpr uint32_t kNormBlocks = 2048;   // eight blocks on every CU
constexpr uint32_t kPieceValues = 4096;  // pieces are multiples of this
// Values of a piece: so that `count` tensors of `total` values in all make at most
// kNormBlocks pieces (half as many tensors: kNormBlocks / 2 pieces more than
// tensors).  Blocks with two pieces where others have one held up all: 148
// tensors of 100M bf16 values 79 instead of 36 us.
inline uint32_t piece_values(size_t total, size_t count) {
  const size_t most = kNormBlocks - std::min<size_t>(count, kNormBlocks / 2);
  const size_t units = (total + most * kPieceValues - 1) / (most * kPieceValues);
  return (uint32_t)(std::max<size_t>(units, 1) * kPieceValues);
}

// How the kernels are given a list: up to kArgTensors tensors with their
// arguments, and a block finds its piece there; of more, the pieces are read in
// pinned host memory.
constexpr uint32_t kArgTensors = TLC_CAPTURE_TENSORS;
struct ListTensor {
  const void* x;
  void* out;
  uint32_t n;
  uint32_t piece0_type;  // its first piece, type in the top two bits
};
struct PinnedList {
  const Piece* pieces;
  // device memory where the norm leaves the pieces for the clipping, which then
  // need not wait for the bus (335 tensors 14.3 -> 12.9 us); NULL: no clipping
  Piece* copy;
  uint32_t n;     // pieces
  bool own_type;  // clipping: out is of x's type (else fp32)
};
struct ArgList {
  uint32_t count, n;  // tensors, pieces
  uint32_t len;       // values of a piece
  bool own_type;
  ListTensor tensors[kArgTensors];
};
static_assert(sizeof(ArgList) <= 3328, "kernel arguments end at 4096 bytes");

// The partial sums of the blocks (one double each) over `pieces` pieces.
inline uint32_t norm_blocks(uint32_t pieces) {
  return pieces < kNormBlocks ? pieces : kNormBlocks;
}
// read_once: no clipping follows in the same call.
template <class List>
hipError_t launch_sumsq(const List& list, bool read_once, double* partials, hipStream_t st);
// Their sum into the result.
hipError_t launch_norm_finish(const double* partials, uint32_t np, tlc_norm_result* result,
                              hipStream_t st);
// The clipped tensors, from the partial sums or (partials NULL) from
// result->sumsq.
template <class List>
hipError_t launch_clip(const List& list, const double* partials, uint32_t np, float max_norm,
                       tlc_norm_result* result, hipStream_t st);

// What a norm makes of the values.
struct Clip {
  float norm, coef;
  bool finite;
};
__device__ __forceinline__ Clip clip_of(double sumsq, float max_norm) {
  const double norm = sqrt(sumsq);
  Clip c;
  c.finite = sumsq >= 0.0 && sumsq <= DBL_MAX;  // false for NaN too
  c.norm = (float)norm;
  c.coef = !c.finite ? __builtin_nanf("")
                     : (norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.0f);
  return c;
}

__device__ __forceinline__ void put_result(tlc_norm_result* r, Clip c) {
  r->norm = c.norm;
  r->coef = c.coef;
  r->status = c.finite ? TLC_OK : TLC_E_NONFINITE;
  r->reserved = 0u;
}

// Words from one counter of blocks to the next: each has a cache line of its own,
// where atomics come one after the other.
constexpr uint32_t kTicketWords = 32;

// ---- token log probabilities
constexpr uint32_t kLogThreads = 256;
// A row, or a part of one: its largest logit (at least -FLT_MAX) and sums by it.
struct LogitPart {
  float m, s0, s1;
};
struct LogitArgs {
  const void* x;
  uint64_t stride;  // values
  uint32_t count, vocab;
  float scale;
  const void* targets;  // NULL: none
  bool wide_ids;        // targets are int64
  int64_t ignore;
  uint32_t* bad;        // pinned host word: set where a target is outside the vocabulary
};
struct TokenArgs : LogitArgs {
  tlc_token_result* results;
  uint32_t top;
  float* top_logprobs;
  int32_t* top_ids;
  // rows cut into parts: the parts' sums and a key for each of their threads
  uint32_t parts, part_packs;
  LogitPart* part;
  uint64_t* keys;
  uint32_t* tickets;  // of a row's blocks that are done; zero between calls
};
// Packs of 16 bytes a row.  Short rows take a wave each (8192 rows of 2048 fp32
// values 12.7 us, in blocks 17; with five alternatives 17.7 | 48.6), longer ones where
// there are many or no alternatives are asked for (packs up to kManyPacks: 4096 rows
// of 8192 bf16 values with twenty 22.9 | 34.5, 64 such rows 11.1 | 7.5).  More than
// kWaveTop alternatives are half of a wave's lanes, whose largest then say little of long
// segments: their rows take a block each.  That costs short rows much (4096 rows of 4096
// bf16 values with 32 | 33 alternatives 16 | 48 us, 16384 of 64 values 24 | 150): of rows
// of 64 packs and fewer, whose columns all fit in `found`, a wave has not been measured.
constexpr uint32_t kWavePacks = 512, kManyPacks = 1024, kManyRows = 2048, kWaveTop = 32;
inline bool wave_rows(uint32_t count, uint32_t packs, uint32_t top) {
  return top <= kWaveTop &&
         (packs <= kWavePacks || (packs <= kManyPacks && (top == 0 || count >= kManyRows)));
}
// Parts of a row: where the rows alone leave CUs idle, as many as make kLogBlocks
// blocks, of kPartPacks packs at least (1 row of 131072 fp32 values with twenty
// alternatives 11.3 us; in parts of half | a quarter 12.4 | 16; 64 such rows 15.6, in 1024
// blocks 19.9: the last block of a row reads a key for each thread of the others).
constexpr uint32_t kLogBlocks = 512, kLogMaxParts = 256, kPartPacks = 4096;
inline uint32_t logit_parts(uint32_t count, uint32_t packs) {
  const uint32_t want = std::min(kLogBlocks / count, kLogMaxParts);
  return std::max(1u, std::min(want, packs / kPartPacks));
}
// Groups of four threads' segments: up to so many alternatives.
constexpr uint32_t kQuadTop = 32;
// Logits of the last-level cache's size and more are read past it, eight packs of
// a thread in flight (8192 rows of 65536 bf16 values, 966 MB: 143 us, 6.75 TB/s;
// through the cache 158, with four packs 165, past it 148; 64 rows of 131072 fp32
// values, which the cache holds, 18.7 | 19.8 past it).  Gradients of that size are
// read and written past it (8192 x 131072 bf16 values 662 | 677 us).
constexpr uint64_t kStreamBytes = 256u << 20;
hipError_t launch_token_logprobs(const TokenArgs& a, int type, hipStream_t st);

struct TokenGradArgs : LogitArgs {
  const tlc_token_result* results;
  const float* grad_logprob;  // NULL: zeroes
  const float* grad_entropy;  // NULL: zeroes
  void* out;
  uint64_t out_stride;
  uint32_t slices;            // blocks of a row
  uint32_t row0, rows;        // of short rows, a launch's
};
constexpr uint32_t kGradUnits = 2, kShortPacks = 256;

hipError_t launch_token_grad(const TokenGradArgs& a, int type, int out_type, hipStream_t st);

// ---- AdamW
constexpr uint32_t kAdamThreads = 256;
constexpr uint32_t kAdamTensors = 64;  // of a launch
// Packs of four values a thread has in flight: a wave's are whole blocks of 8-bit
// states (100M values, two | four: 590 | 569 us of 32 bits, 330 | 332 of 8, one
// 363; few values, which have no wave to spare, in short pieces one at a time).
constexpr uint32_t kAdamUnit = kAdamThreads * 4;
constexpr uint32_t adam_steps(int bits) { return bits == 32 ? 4 : 2; }
// A block takes a piece, or of very many several.  Pieces are multiples of
// kAdamUnit values, so that few values still fill the chip (1000003 of 8 bits 7.5 us,
// in pieces of 4096 9.8); in pinned memory no shorter than what a block has in flight,
// as a piece takes 3 ns of the bus (335 tensors of 1.7M values, pieces of 1024 | 2048 | 4096: 18.8 | 16.4
// | 14.4 us of 32 bits, 18.3 | 16.4 | 17.2 of 8).  Large lists make kAdamPieces of
// them or fewer, pinned ones kAdamPinned (one tensor of 100M, 2048 | 4096 | 8192 | 16384
// pieces: 505 | 493 | 485 | 488 us; 148 tensors 523 | 503 | 512 | 508).
constexpr uint32_t kAdamPieces = 8192, kAdamPinned = 4096;
inline uint32_t adam_piece_values(size_t total, size_t count, size_t unit, size_t pieces) {
  const size_t most = pieces - std::min<size_t>(count, pieces / 2);
  const size_t units = (total + most * unit - 1) / (most * unit);
  return (uint32_t)(std::max<size_t>(units, 1) * unit);
}
struct AdamTensor {
  void* p;
  const void* g;
  void* m;
  void* v;
  float* scales;  // states in 8 bits: two floats a block
  float* delta;   // or NULL
  uint32_t n;
  uint32_t piece0_types;  // its first piece, p's type in bits 28 and 29, g's in 30 and 31
};
struct AdamList {
  uint32_t count, n;  // tensors, pieces
  uint32_t len;       // values of a piece
  uint32_t state_bytes;  // of a value of m or v
  AdamTensor tensors[kAdamTensors];
};
// A piece with pointers to its values, which begin at value k0 of their tensor.
struct AdamPiece {
  void* p;
  const void* g;
  void* m;
  void* v;
  float* scales;
  float* delta;
  uint32_t n, k0;
  uint32_t types;  // p's in bits 0 and 1, g's in 2 and 3
  uint32_t reserved;
};
static_assert(sizeof(AdamPiece) == 64, "AdamPiece is 64 bytes");
__host__ __device__ inline AdamPiece adam_piece(const AdamTensor& t, uint32_t types, uint32_t k0,
                                                uint32_t len, uint32_t state_bytes) {
  AdamPiece r;
  r.p = (uint8_t*)t.p + (uint64_t)k0 * ((types & 3u) == TLC_F32 ? 4 : 2);
  r.g = (const uint8_t*)t.g + (uint64_t)k0 * ((types >> 2) == TLC_F32 ? 4 : 2);
  r.m = (uint8_t*)t.m + (uint64_t)k0 * state_bytes;
  r.v = (uint8_t*)t.v + (uint64_t)k0 * state_bytes;
  r.scales = t.scales ? t.scales + k0 / TLC_STATE_BLOCK * 2 : nullptr;
  r.delta = t.delta ? t.delta + k0 : nullptr;
  r.n = len < t.n - k0 ? len : t.n - k0;
  r.k0 = k0;
  r.types = types;
  r.reserved = 0u;
  return r;
}
// More tensors than a launch's arguments hold: their pieces in pinned host memory.
struct AdamPinned {
  const AdamPiece* pieces;
  uint32_t n;
};
struct AdamArgs {
  double lr, log_beta1, log_beta2, decay;
  float c1, c2;  // 1 - beta
  float eps, max_norm;
  tlc_adamw_clock* clock;
  tlc_norm_result* result;  // NULL: no clipping
  bool stream;              // the list is larger than the last-level cache
  uint32_t* tickets;        // the step's last launch: counts its blocks; else NULL
};
// The counters: of the groups, and of each group's blocks; zero between calls.
constexpr uint32_t kTicketGroups = 64;
constexpr size_t kTicketBytes = (1 + kTicketGroups) * kTicketWords * sizeof(uint32_t);
static_assert(sizeof(AdamList) + sizeof(AdamArgs) <= 3840, "kernel arguments end at 4096 bytes");
template <class List>
hipError_t launch_adamw(const List& list, const AdamArgs& a, int state_type, hipStream_t st);

}  // namespace tlc
