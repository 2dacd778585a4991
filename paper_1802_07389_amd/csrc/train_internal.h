// train_internal.h -- definitions shared by the kernels of the embedding
// tables and of the gradient norm and their host side (not part of the public
// ABI).
#pragma once

#include "tlc_internal.h"

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
  uint32_t* bad;      // pinned host word: set where an id is outside the table
};

hipError_t launch_embedding(const EmbArgs& a, int table_type, int ids_type, int out_type,
                            hipStream_t st);
hipError_t launch_embedding_grad(const EmbArgs& a, int grad_type, int ids_type, bool accumulate,
                                 hipStream_t st);

// A list of tensors is cut into pieces of one length (the last of a tensor
// shorter).  A block takes consecutive pieces.
struct Piece {
  const void* x;
  void* out;
  uint32_t n;
  uint32_t type;
};
static_assert(sizeof(Piece) == 24, "Piece is 24 bytes");
constexpr uint32_t kNormThreads = 256;
constexpr uint32_t kNormBlocks = 2048;    // eight blocks on every CU
constexpr uint64_t kPieceValues = 4096;   // pieces are multiples of this

// The partial sums of the blocks (one double each) over `pieces` pieces.
inline uint32_t norm_blocks(uint32_t pieces) {
  return pieces < kNormBlocks ? pieces : kNormBlocks;
}
hipError_t launch_sumsq(const Piece* pieces, uint32_t n, double* partials, hipStream_t st);
// Their sum into the result.
hipError_t launch_norm_finish(const double* partials, uint32_t np, tlc_norm_result* result,
                              hipStream_t st);
// The clipped tensors, from the partial sums or (partials NULL) from
// result->sumsq.  own_type: in place in the pieces' own types.
hipError_t launch_clip(const Piece* pieces, uint32_t n, const double* partials, uint32_t np,
                       float max_norm, bool own_type, tlc_norm_result* result, hipStream_t st);

}  // namespace tlc
