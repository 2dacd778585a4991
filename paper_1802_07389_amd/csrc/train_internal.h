// train_internal.h -- definitions shared by the kernels of the embedding
// tables and of the gradient norm and their host side (not part of the public
// ABI).
#pragma once

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

}  // namespace tlc
