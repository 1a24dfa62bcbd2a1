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

// --------------------------------------------------------------- experts
// A product of rows sorted by expert: rows [offsets[e], offsets[e + 1]) meet
// expert e's weight.  GemmArgs hold expert 0's weight, bias and weight gradient
// and the whole buffers' rows.
struct ExpertArgs {
  const void* offsets;  // [experts + 1] integers of offset_bytes
  int offset_bytes, experts;
  int rows;
  int64_t stride;  // elements between two experts' weights, or weight gradients
};
size_t expert_workspace_need(dattri_linear_op op, int64_t rows, int64_t experts, int64_t d_in, int64_t d_out, int elt,
                             bool aligned);
// aligned: both operands readable in 16-byte pieces; a.out may be null beside dbias (weight grad).
hipError_t launch_expert(dattri_linear_op op, int elt, bool aligned, GemmArgs a, ExpertArgs x, float* dbias,
                         uint8_t* ws, hipStream_t s);

// ----------------------------------------------------------------- 8 bits
// Scales of an 8-bit product: x [rows][ldx], w [blocks of 128 outputs][ldw], one
// for every 128 of k.
struct Scales8 {
  const float *x, *w;
  int64_t ldx, ldw;
};
size_t linear8_workspace_need(int64_t rows, int64_t d_in, int64_t d_out, int elt, bool aligned);
// As the forward product: A = X, B = W, one byte per element; elt is that of bias, R, Y and Z.
hipError_t launch_linear8(int elt, bool aligned, GemmArgs a, const Scales8& sc, uint8_t* ws, hipStream_t s);
hipError_t launch_quantize_rows(int elt, const void* X, int64_t ldx, int64_t rows, int64_t d, uint8_t* Q, int64_t ldq,
                                float* S, int64_t lds, hipStream_t s);
hipError_t launch_quantize_weight(int elt, const void* W, int64_t ldw, int64_t rows, int64_t d, uint8_t* Q, int64_t ldq,
                                  float* S, int64_t lds, hipStream_t s);

// ------------------------------------------------------------------ norm
struct NormArgs {
  const void *X, *R, *W;  // R may be null
  int64_t ldx, ldr, rows;
  int d;
  float eps;
  void *Y, *H;  // may be null
  int64_t ldy, ldh;
  uint8_t* Q;  // may be null, with S
  float* S;
  int64_t ldq, lds;
};
hipError_t launch_rms_norm(int elt, const NormArgs& a, hipStream_t s);
struct NormGradArgs {
  const void *G, *H, *W, *P;  // P may be null
  int64_t ldg, ldh, ldp, rows;
  int d;
  float eps;
  void* D;
  int64_t ldd;
  float* U;  // [rows], set by the launch
};
struct NormGradLayout {
  size_t off_part, total;
};
NormGradLayout norm_grad_layout(int64_t rows, int64_t d, bool weight);
// dw: null or the weight's gradient
hipError_t launch_norm_grad(int elt, NormGradArgs a, float* dw, bool accumulate, uint8_t* ws, hipStream_t s);

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
