// Internal interface of the model-side operators (model_api.cpp and the
// embedding, linear and clip kernels).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "dattri.h"
#include "row_grid.h"

namespace dattri {

// ------------------------------------------------------------- embedding
hipError_t launch_embedding(int elt, const void* table, int64_t ld_table, int64_t vocab, int64_t d, const void* tokens,
                            int token_bytes, int64_t n, float scale, void* out, int64_t ld_out, hipStream_t s);

// Workspace of the table gradient: byte offsets of two (key, position) buffers,
// the digit counts and the partial sums of long runs.
struct EmbGradLayout {
  size_t off_key[2], off_pos[2], off_hist, off_part, total;
};
EmbGradLayout embedding_grad_layout(int64_t n, int64_t vocab, int64_t d);
hipError_t launch_embedding_grad(int elt, const void* grad_out, int64_t ld_grad, const void* tokens, int token_bytes,
                                 int64_t n, float scale, int64_t vocab, int64_t d, float* grad_table, int64_t ld_table,
                                 bool accumulate, uint8_t* ws, hipStream_t s);

// ---------------------------------------------------------------- linear
// C[m][n] = sum_k A(m, k) B(n, k) with an epilogue.  An operand is stored
// [rows of k] (k contiguous) or [k rows of its index] (k strided):
//   forward       A = X (contiguous),  B = W (contiguous), m: row,   n: d_out, k: d_in
//   input grad    A = G (contiguous),  B = W (strided),    m: row,   n: d_in,  k: d_out
//   weight grad   A = G (strided),     B = X (strided),    m: d_out, n: d_in,  k: row
struct GemmArgs {
  const void* A;
  const void* B;
  int64_t lda, ldb;
  int M, N, K;
  const void* bias;  // forward
  const void* R;
  int64_t ldr;
  void* Z;  // forward: kept pre-activation (or null); input grad: read
  int64_t ldz;
  void* out;  // Y; D (or null); dW
  int64_t ldo;
  void* out2;  // input grad: P (or null)
  int64_t ldo2;
  int act;
  int accumulate;  // weight grad
  int vec;         // rows of the epilogue's buffers start on four elements
};
size_t linear_workspace_need(dattri_linear_op op, int64_t rows, int64_t d_in, int64_t d_out, int elt, bool aligned);
// aligned: both operands' pointers and strides on 16 bytes; dbias (weight grad):
// null or the bias gradient; a.out may then be null.
hipError_t launch_linear(dattri_linear_op op, int elt, bool aligned, GemmArgs a, float* dbias, uint8_t* ws,
                         hipStream_t s);

// The form for a few rows (linear_few.hip): whether a call takes it, its launch
// (aligned: rows of X and W on 16 bytes).
bool linear_few(dattri_linear_op op, int64_t rows, int64_t d_out);
hipError_t launch_linear_few(int elt, const GemmArgs& a, bool aligned, hipStream_t s);

// ------------------------------------------------------------------ clip
constexpr int kClipTensors = 128;    // tensors per launch (their list is a kernel argument)
constexpr int kClipChunk = 16384;    // elements per unit of work
constexpr int kClipMost = (1 << 24) - 1;  // chunks per launch: 256 threads for each fit 32 bits
constexpr int kClipGroups = 2048;    // most workgroups of the norm's launch, each writing one partial sum
struct ClipTensor {
  const void* src;
  void* dst;           // null: norm only
  int64_t size_flags;  // elements << 2 | dst is float32 << 1 | src is float32
};
struct ClipList {
  int n, pad;
  ClipTensor t[kClipTensors];
  int first[kClipTensors + 1];  // first chunk of each tensor, then the number of chunks
};
static_assert(sizeof(ClipList) <= 3840, "kernel argument size");
// stream: loads past the caches
hipError_t launch_clip_squares(const ClipList& l, int groups, double* partials, bool stream, hipStream_t s);
hipError_t launch_clip_norm(const double* partials, int n_partials, float max_norm, float* norm_coef, hipStream_t s);
hipError_t launch_clip_scale(const ClipList& l, const float* norm_coef, bool stream, hipStream_t s);

}  // namespace dattri
