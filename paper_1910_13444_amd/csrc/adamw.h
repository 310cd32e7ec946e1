// The gradients' norm and the AdamW step over many tensors (adamw.hip).
#pragma once
#include "common.h"

namespace pigan {

// Calls that move more leave nothing for the next one in the last-level cache (256 MiB).
constexpr double STREAM_BYTES = 192.0 * 1048576.0;
constexpr int QBLOCK = 256;      // elements that share the scale of an 8-bit state
constexpr int PIECE = 1024;      // elements of a tensor that a block takes, four a thread

// A tensor as the kernels see it; `state` is its first element in the flat states.
struct TensorEntry {
  float* p; const void* g; void* copy;
  int64_t n; int64_t state;
  double decay;
  int32_t g_dt; int32_t copy_dt;
};

// A piece of work: elements [piece * PIECE, ...) of tensor `tensor`.
struct TensorPiece { uint32_t tensor; uint32_t piece; };

// Memory [from, to) of a table's tensors.
struct Extent { uint64_t from; uint64_t to; };

// A table, in host memory and, byte for byte, in device memory: the header, the
// entries, the pieces, and, for the host's checks of a call's other operands, what the
// tensors' outputs (parameters, copies, states) and their gradients take, joined and in
// the order of the addresses.
struct TableHeader {
  uint64_t magic;
  int32_t n_tensors; int32_t bits;      // bits 0: gradients alone
  int64_t n_pieces; int64_t states;     // elements of a flat state
  int64_t entries_at; int64_t pieces_at; int64_t bytes;
  void* m; void* v; float* m_scale; float* v_scale;
  int64_t elements; int64_t g_bytes; int64_t copy_bytes;
  int64_t extents_at; int64_t n_written; int64_t n_read;
};
constexpr uint64_t TABLE_MAGIC = 0x656c626174676970ull;

struct AdamwArgs {
  const TensorEntry* entries; const TensorPiece* pieces;
  void* m; void* v; float* m_scale; float* v_scale;
  double lr, b1, b2, nb1, nb2, eps, scale, c1, c2;   // nb = 1 - b
  const float* coef;        // multiplies scale, or null
  const double* corr;       // {c1, c2} on the device, or null
  const int32_t* skip;
  bool stream;              // past the caches
};

hipError_t launch_adamw(const AdamwArgs& a, int bits, int64_t n_pieces, hipStream_t st);
// ++*step unless *skip, and corr = {1 / (1 - b1^step), 1 / (1 - b2^step)}
hipError_t launch_adamw_begin(double b1, double b2, int32_t* step, const int32_t* skip, double* corr, hipStream_t st);

// partial sums of the gradients' norm
int64_t grad_norm_blocks(int64_t n_pieces);
hipError_t launch_grad_norm(const TensorEntry* entries, const TensorPiece* pieces, int64_t n_pieces, double max_norm,
                            double scale, double* part, float* norm, float* coef, int32_t* nonfinite, hipStream_t st);

hipError_t launch_state_values(int64_t n, const int8_t* m, const float* m_scale, const uint8_t* v, const float* v_scale,
                               float* m_out, float* v_out, hipStream_t st);

}  // namespace pigan
