// C ABI of the model-side operators: argument checks, workspace layout and
// launches of embedding, linear and clipping kernels.
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "api_common.h"
#include "dattri.h"
#include "model_checks.h"
#include "model_ops.h"

using namespace dattri;

namespace {

constexpr int64_t kClipStream = (int64_t)256 << 20;  // bytes (gradients and other buffers written) that no cache holds

dattri_status check_tokens(const void* tokens, int32_t token_bytes, int64_t n) {
  if (token_bytes != 4 && token_bytes != 8)
    return fail(DATTRI_E_INVALID_ARG, "token_bytes must be 4 or 8 (got %d)", token_bytes);
  if (n > 0 && !tokens) return fail(DATTRI_E_INVALID_ARG, "tokens is NULL");
  if ((uintptr_t)tokens % token_bytes) return fail(DATTRI_E_INVALID_ARG, "tokens is not aligned to its elements");
  return DATTRI_OK;
}

dattri_status check_linear_sizes(int64_t rows, int64_t d_in, int64_t d_out, dattri_dtype dtype, int* elt) {
  dattri_status st = elt_of(dtype, elt);
  if (st == DATTRI_OK) st = check_count("rows", rows);
  if (st == DATTRI_OK) st = check_width("d_in", d_in);
  if (st == DATTRI_OK) st = check_width("d_out", d_out);
  return st;
}

}  // namespace

extern "C" {

dattri_status dattri_embedding(const void* table, int64_t ld_table, int64_t vocab, int64_t d, dattri_dtype dtype,
                               const void* tokens, int32_t token_bytes, int64_t n, float scale, void* out,
                               int64_t ld_out, void* stream) {
  reset_error();
  int elt;
  TRY(elt_of(dtype, &elt));
  TRY(check_count("vocab", vocab));
  TRY(check_count("n", n));
  TRY(check_width("d", d));
  TRY(check_rows("table", table, &ld_table, n > 0 ? vocab : 0, d, elt, true));
  TRY(check_rows("out", out, &ld_out, n, d, elt, true));
  TRY(check_tokens(tokens, token_bytes, n));
  TRY(check_apart(Span("out", out, n, d, ld_out, elt),
                  {Span("table", table, vocab, d, ld_table, elt), Span("tokens", tokens, n * token_bytes)}));
  if (n == 0) return DATTRI_OK;
  HIP_TRY(launch_embedding(elt, table, ld_table, vocab, d, tokens, token_bytes, n, scale, out, ld_out,
                           (hipStream_t)stream));
  return DATTRI_OK;
}

dattri_status dattri_embedding_grad_workspace_bytes(int64_t n, int64_t vocab, int64_t d, size_t* bytes) {
  reset_error();
  if (!bytes) return fail(DATTRI_E_INVALID_ARG, "bytes is NULL");
  TRY(check_count("n", n));
  TRY(check_count("vocab", vocab));
  TRY(check_width("d", d));
  *bytes = embedding_grad_layout(n, vocab, d).total;
  return DATTRI_OK;
}

dattri_status dattri_embedding_grad(const void* grad_out, int64_t ld_grad, dattri_dtype dtype, const void* tokens,
                                    int32_t token_bytes, int64_t n, float scale, int64_t vocab, int64_t d,
                                    float* grad_table, int64_t ld_table, int32_t accumulate, void* workspace,
                                    size_t ws_bytes, void* stream) {
  reset_error();
  int elt;
  TRY(elt_of(dtype, &elt));
  TRY(check_count("n", n));
  TRY(check_count("vocab", vocab));
  TRY(check_width("d", d));
  TRY(check_rows("grad_out", grad_out, &ld_grad, n, d, elt, true));
  TRY(check_rows("grad_table", grad_table, &ld_table, vocab, d, 4, true));
  TRY(check_tokens(tokens, token_bytes, n));
  const size_t need = embedding_grad_layout(n, vocab, d).total;
  TRY(check_workspace(workspace, ws_bytes, need));
  {
    const Span g("grad_out", grad_out, n, d, ld_grad, elt), t("tokens", tokens, n * token_bytes),
        out("grad_table", grad_table, vocab, d, ld_table, 4);
    TRY(check_apart(out, {g, t}));
    TRY(check_apart(Span("workspace", workspace, (int64_t)need), {g, t, out}));
  }
  HIP_TRY(launch_embedding_grad(elt, grad_out, ld_grad, tokens, token_bytes, n, scale, vocab, d, grad_table, ld_table,
                                accumulate != 0, (uint8_t*)workspace, (hipStream_t)stream));
  return DATTRI_OK;
}

dattri_status dattri_linear_workspace_bytes(dattri_linear_op op, int64_t rows, int64_t d_in, int64_t d_out,
                                            dattri_dtype dtype, int32_t aligned, size_t* bytes) {
  reset_error();
  int elt;
  if (!bytes) return fail(DATTRI_E_INVALID_ARG, "bytes is NULL");
  if ((int)op < DATTRI_LINEAR_FORWARD || (int)op > DATTRI_LINEAR_WEIGHT_GRAD)
    return fail(DATTRI_E_INVALID_ARG, "unknown linear op %d", (int)op);
  TRY(check_linear_sizes(rows, d_in, d_out, dtype, &elt));
  *bytes = linear_workspace_need(op, rows, d_in, d_out, elt, aligned != 0);
  return DATTRI_OK;
}

dattri_status dattri_linear(const void* X, int64_t ld_x, const void* W, int64_t ld_w, const void* bias, dattri_act act,
                            const void* R, int64_t ld_r, void* Y, int64_t ld_y, void* Z, int64_t ld_z, int64_t rows,
                            int64_t d_in, int64_t d_out, dattri_dtype dtype, void* workspace, size_t ws_bytes,
                            void* stream) {
  reset_error();
  int elt;
  TRY(check_linear_sizes(rows, d_in, d_out, dtype, &elt));
  TRY(check_act(act));
  TRY(check_rows("X", X, &ld_x, rows, d_in, elt, true));
  TRY(check_rows("W", W, &ld_w, d_out, d_in, elt, true));
  TRY(check_rows("R", R, &ld_r, rows, d_out, elt, false));
  TRY(check_rows("Y", Y, &ld_y, rows, d_out, elt, true));
  TRY(check_rows("Z", Z, &ld_z, rows, d_out, elt, false));
  if ((uintptr_t)bias % elt) return fail(DATTRI_E_INVALID_ARG, "bias is not aligned to its elements");
  if (R && R == Y && ld_r != ld_y) return fail(DATTRI_E_INVALID_ARG, "Y may be R only with the same row stride");
  const bool aligned = on_16(X, ld_x, W, ld_w, elt);
  const size_t need = linear_workspace_need(DATTRI_LINEAR_FORWARD, rows, d_in, d_out, elt, aligned);
  TRY(check_workspace(workspace, ws_bytes, need));
  {
    const Span x("X", X, rows, d_in, ld_x, elt), w("W", W, d_out, d_in, ld_w, elt), b("bias", bias, d_out * elt),
        r("R", R, rows, d_out, ld_r, elt), y("Y", Y, rows, d_out, ld_y, elt), z("Z", Z, rows, d_out, ld_z, elt);
    TRY(check_apart(y, {x, w, b, z}, &r));
    TRY(check_apart(z, {x, w, b, r}));
    TRY(check_apart(Span("workspace", workspace, (int64_t)need), {x, w, b, r, y, z}));
  }
  if (rows == 0) return DATTRI_OK;
  GemmArgs a = {};
  a.A = X;
  a.B = W;
  a.lda = ld_x;
  a.ldb = ld_w;
  a.M = (int)rows;
  a.N = (int)d_out;
  a.K = (int)d_in;
  a.bias = bias;
  a.R = R;
  a.ldr = ld_r;
  a.Z = Z;
  a.ldz = ld_z;
  a.out = Y;
  a.ldo = ld_y;
  a.act = act;
  HIP_TRY(launch_linear(DATTRI_LINEAR_FORWARD, elt, aligned, a, nullptr, (uint8_t*)workspace, (hipStream_t)stream));
  return DATTRI_OK;
}

dattri_status dattri_linear_input_grad(const void* G, int64_t ld_g, const void* W, int64_t ld_w, const void* R,
                                       int64_t ld_r, dattri_act act, const void* Z, int64_t ld_z, void* D, int64_t ld_d,
                                       void* P, int64_t ld_p, int64_t rows, int64_t d_in, int64_t d_out,
                                       dattri_dtype dtype, void* workspace, size_t ws_bytes, void* stream) {
  reset_error();
  int elt;
  TRY(check_linear_sizes(rows, d_in, d_out, dtype, &elt));
  TRY(check_act(act));
  TRY(check_rows("G", G, &ld_g, rows, d_out, elt, true));
  TRY(check_rows("W", W, &ld_w, d_out, d_in, elt, true));
  TRY(check_rows("R", R, &ld_r, rows, d_in, elt, false));
  TRY(check_rows("Z", Z, &ld_z, rows, d_in, elt, P && act != DATTRI_ACT_NONE));
  TRY(check_rows("D", D, &ld_d, rows, d_in, elt, false));
  TRY(check_rows("P", P, &ld_p, rows, d_in, elt, false));
  if (rows > 0 && !D && !P) return fail(DATTRI_E_INVALID_ARG, "nothing to compute: D and P are NULL");
  if (D && D == P) return fail(DATTRI_E_INVALID_ARG, "D and P must be different buffers");
  if (R && ((R == D && ld_r != ld_d) || (R == P && ld_r != ld_p)))
    return fail(DATTRI_E_INVALID_ARG, "D or P may be R only with the same row stride");
  if (Z && ((Z == P && ld_z != ld_p) || Z == D))
    return fail(DATTRI_E_INVALID_ARG, "P may be Z only with the same row stride, D may not");
  const bool aligned = on_16(G, ld_g, W, ld_w, elt);
  const size_t need = linear_workspace_need(DATTRI_LINEAR_INPUT_GRAD, rows, d_in, d_out, elt, aligned);
  TRY(check_workspace(workspace, ws_bytes, need));
  {
    const Span g("G", G, rows, d_out, ld_g, elt), w("W", W, d_out, d_in, ld_w, elt), r("R", R, rows, d_in, ld_r, elt),
        z("Z", act == DATTRI_ACT_NONE || !P ? nullptr : Z, rows, d_in, ld_z, elt), d("D", D, rows, d_in, ld_d, elt),
        p("P", P, rows, d_in, ld_p, elt);
    TRY(check_apart(d, {g, w, z, p}, &r));
    TRY(check_apart(p, {g, w}, &r, &z));
    TRY(check_apart(Span("workspace", workspace, (int64_t)need), {g, w, r, z, d, p}));
  }
  if (rows == 0) return DATTRI_OK;
  GemmArgs a = {};
  a.A = G;
  a.B = W;
  a.lda = ld_g;
  a.ldb = ld_w;
  a.M = (int)rows;
  a.N = (int)d_in;
  a.K = (int)d_out;
  a.R = R;
  a.ldr = ld_r;
  a.Z = const_cast<void*>(Z);
  a.ldz = ld_z;
  a.out = D;
  a.ldo = ld_d;
  a.out2 = P;
  a.ldo2 = ld_p;
  a.act = act;
  HIP_TRY(launch_linear(DATTRI_LINEAR_INPUT_GRAD, elt, aligned, a, nullptr, (uint8_t*)workspace,
                        (hipStream_t)stream));
  return DATTRI_OK;
}

dattri_status dattri_linear_weight_grad(const void* G, int64_t ld_g, const void* X, int64_t ld_x, float* dW,
                                        int64_t ld_dw, float* dbias, int32_t accumulate, int64_t rows, int64_t d_in,
                                        int64_t d_out, dattri_dtype dtype, void* workspace, size_t ws_bytes,
                                        void* stream) {
  reset_error();
  int elt;
  TRY(check_linear_sizes(rows, d_in, d_out, dtype, &elt));
  TRY(check_rows("G", G, &ld_g, rows, d_out, elt, true));
  TRY(check_rows("X", X, &ld_x, rows, d_in, elt, dW != nullptr));
  TRY(check_rows("dW", dW, &ld_dw, d_out, d_in, 4, false));
  if ((uintptr_t)dbias % 4) return fail(DATTRI_E_INVALID_ARG, "dbias is not aligned to its elements");
  if (!dW && !dbias) return fail(DATTRI_E_INVALID_ARG, "nothing to compute: dW and dbias are NULL");
  const bool aligned = !dW || on_16(G, ld_g, X, ld_x, elt);  // bias alone: no operands
  const size_t need = linear_workspace_need(DATTRI_LINEAR_WEIGHT_GRAD, rows, d_in, d_out, elt, aligned);
  TRY(check_workspace(workspace, ws_bytes, need));
  {
    const Span g("G", G, rows, d_out, ld_g, elt), x("X", dW ? X : nullptr, rows, d_in, ld_x, elt),
        w("dW", dW, d_out, d_in, ld_dw, 4), b("dbias", dbias, d_out * 4);
    TRY(check_apart(w, {g, x, b}));
    TRY(check_apart(b, {g, x}));
    TRY(check_apart(Span("workspace", workspace, (int64_t)need), {g, x, w, b}));
  }
  if (rows == 0 && accumulate) return DATTRI_OK;
  GemmArgs a = {};
  a.A = G;
  a.B = X;
  a.lda = ld_g;
  a.ldb = ld_x;
  a.M = (int)d_out;
  a.N = (int)d_in;
  a.K = (int)rows;
  a.out = dW;
  a.ldo = ld_dw;
  a.accumulate = accumulate != 0;
  HIP_TRY(launch_linear(DATTRI_LINEAR_WEIGHT_GRAD, elt, aligned, a, dbias, (uint8_t*)workspace, (hipStream_t)stream));
  return DATTRI_OK;
}

}  // extern "C"

namespace {

// Walks the tensors in launches of at most kClipTensors of them and at most
// kClipMost chunks; `visit(list, groups)` gets each (with src, dst, dtypes when given).
template <class F>
dattri_status clip_launches(const void* const* grads, const int64_t* sizes, const dattri_dtype* dtypes,
                            void* const* outs, const dattri_dtype* out_dtypes, int64_t n_tensors, F visit) {
  ClipList l;
  l.n = l.pad = 0;
  l.first[0] = 0;
  auto flush = [&]() -> dattri_status {
    if (l.n == 0) return DATTRI_OK;
    const dattri_status st = visit(l, std::min(l.first[l.n], kClipGroups));
    l.n = 0;
    return st;
  };
  for (int64_t i = 0; i < n_tensors; ++i) {
    const int64_t chunks = (sizes[i] + kClipChunk - 1) / kClipChunk;
    if (chunks == 0) continue;
    if (l.n == kClipTensors || (l.n > 0 && l.first[l.n] + chunks > kClipMost)) TRY(flush());
    ClipTensor& t = l.t[l.n];
    t.src = grads ? grads[i] : nullptr;
    t.dst = outs ? outs[i] : nullptr;
    t.size_flags = sizes[i] << 2 | (out_dtypes && out_dtypes[i] == DATTRI_F32 ? 2 : 0) |
                   (dtypes && dtypes[i] == DATTRI_F32 ? 1 : 0);
    l.first[l.n + 1] = l.first[l.n] + (int)chunks;
    ++l.n;
  }
  return flush();
}

dattri_status clip_sizes(const int64_t* sizes, int64_t n_tensors, int64_t* partials) {
  if (n_tensors < 0) return fail(DATTRI_E_INVALID_ARG, "n_tensors must be >= 0");
  if (n_tensors > INT32_MAX / kClipGroups * (int64_t)kClipTensors)
    return fail(DATTRI_E_UNSUPPORTED, "%lld tensors are too many", (long long)n_tensors);
  if (n_tensors > 0 && !sizes) return fail(DATTRI_E_INVALID_ARG, "sizes is NULL");
  for (int64_t i = 0; i < n_tensors; ++i) {
    if (sizes[i] < 0) return fail(DATTRI_E_INVALID_ARG, "size of tensor %lld is negative", (long long)i);
    if (sizes[i] > (int64_t)kClipChunk * kClipMost)
      return fail(DATTRI_E_UNSUPPORTED, "tensor %lld has too many elements", (long long)i);
  }
  int64_t n = 0;
  const dattri_status st = clip_launches(nullptr, sizes, nullptr, nullptr, nullptr, n_tensors,
                                         [&](const ClipList&, int groups) {
                                           n += groups;
                                           return DATTRI_OK;
                                         });
  *partials = n;
  return st;
}

// A scaled tensor may lie in no other tensor of the call, and in its own source
// only if it is that: sources and outputs in the order of their addresses, no
// output in front of an end and nothing in front of an output's.
dattri_status clip_apart(const void* const* grads, const int64_t* sizes, const dattri_dtype* dtypes, void* const* outs,
                         const dattri_dtype* out_dtypes, int64_t n_tensors, const Span& norm_coef,
                         const Span& workspace) {
  TRY(check_apart(workspace, {norm_coef}));
  struct Piece {
    uintptr_t at, end;
    int64_t tensor;
    bool operator<(const Piece& o) const { return at < o.at; }
  };
  const std::unique_ptr<Piece[]> all(new (std::nothrow) Piece[2 * n_tensors + 1]);
  if (!all) return fail(DATTRI_E_UNSUPPORTED, "no host memory for a list of %lld tensors", (long long)n_tensors);
  Piece *src = all.get(), *src_end = src, *dst = src + n_tensors, *dst_end = dst;
  for (int64_t i = 0; i < n_tensors; ++i) {
    if (sizes[i] == 0) continue;
    const uintptr_t p = (uintptr_t)grads[i], q = outs ? (uintptr_t)outs[i] : 0;
    const int64_t bytes = sizes[i] * (dtypes[i] == DATTRI_F32 ? 4 : 2);
    if (p != q) *src_end++ = Piece{p, p + bytes, i};
    if (outs) *dst_end++ = Piece{q, q + sizes[i] * (out_dtypes[i] == DATTRI_F32 ? 4 : 2), i};
    for (const Span* o : {&norm_coef, &workspace})
      for (const Piece* e : {p != q ? src_end - 1 : nullptr, outs ? dst_end - 1 : nullptr})
        if (e && e->at < (uintptr_t)o->end() && (uintptr_t)o->at < e->end)
          return fail(DATTRI_E_INVALID_ARG, "tensor %lld overlaps %s", (long long)i, o->what);
  }
  if (!outs) return DATTRI_OK;
  if (!std::is_sorted(src, src_end)) std::sort(src, src_end);
  if (!std::is_sorted(dst, dst_end)) std::sort(dst, dst_end);
  Piece read{0, 0, -1}, written{0, 0, -1};  // the ones that reach furthest
  while (src != src_end || dst != dst_end) {
    const bool w = src == src_end || (dst != dst_end && dst->at < src->at);
    const Piece& e = w ? *dst++ : *src++;
    const Piece* hit = e.at < written.end ? &written : w && e.at < read.end ? &read : nullptr;
    if (hit)
      return fail(DATTRI_E_INVALID_ARG, "tensors %lld and %lld overlap and one of them is written",
                  (long long)hit->tensor, (long long)e.tensor);
    Piece& reach = w ? written : read;
    if (e.end > reach.end) reach = e;
  }
  return DATTRI_OK;
}

}  // namespace

extern "C" {

dattri_status dattri_clip_workspace_bytes(const int64_t* sizes, int64_t n_tensors, size_t* bytes) {
  reset_error();
  if (!bytes) return fail(DATTRI_E_INVALID_ARG, "bytes is NULL");
  int64_t n;
  TRY(clip_sizes(sizes, n_tensors, &n));
  *bytes = align_up(std::max<size_t>((size_t)n * 8, kAlign));
  return DATTRI_OK;
}

dattri_status dattri_clip_gradients(const void* const* grads, const int64_t* sizes, const dattri_dtype* dtypes,
                                    void* const* outs, const dattri_dtype* out_dtypes, int64_t n_tensors,
                                    float max_norm, float* norm_coef, void* workspace, size_t ws_bytes, void* stream) {
  reset_error();
  int64_t n_partials;
  TRY(clip_sizes(sizes, n_tensors, &n_partials));
  if (!(max_norm >= 0.f)) return fail(DATTRI_E_INVALID_ARG, "max_norm must be >= 0");
  if (!norm_coef) return fail(DATTRI_E_INVALID_ARG, "norm_coef is NULL");
  if ((uintptr_t)norm_coef % 4) return fail(DATTRI_E_INVALID_ARG, "norm_coef is not aligned to its elements");
  if (n_tensors > 0 && (!grads || !dtypes)) return fail(DATTRI_E_INVALID_ARG, "grads or dtypes is NULL");
  if (!outs != !out_dtypes) return fail(DATTRI_E_INVALID_ARG, "outs and out_dtypes go together");
  for (int64_t i = 0; i < n_tensors; ++i) {
    int elt, oelt = 0;
    TRY(elt_of(dtypes[i], &elt));
    if (outs) TRY(elt_of(out_dtypes[i], &oelt));
    if (sizes[i] == 0) continue;
    if (!grads[i] || (outs && !outs[i]))
      return fail(DATTRI_E_INVALID_ARG, "tensor %lld has elements and a NULL pointer", (long long)i);
    if ((uintptr_t)grads[i] % elt || (outs && (uintptr_t)outs[i] % oelt))
      return fail(DATTRI_E_INVALID_ARG, "tensor %lld is not aligned to its elements", (long long)i);
    if (outs && outs[i] == grads[i] && elt != oelt)
      return fail(DATTRI_E_INVALID_ARG, "tensor %lld is scaled in place with another type", (long long)i);
  }
  TRY(check_workspace(workspace, ws_bytes, align_up(std::max<size_t>((size_t)n_partials * 8, kAlign))));
  TRY(clip_apart(grads, sizes, dtypes, outs, out_dtypes, n_tensors, Span("norm_coef", norm_coef, 8),
                 Span("workspace", workspace, n_partials * 8)));
  hipStream_t s = (hipStream_t)stream;
  double* partials = (double*)workspace;
  int64_t bytes = 0;
  for (int64_t i = 0; i < n_tensors; ++i)
    bytes += sizes[i] * ((dtypes[i] == DATTRI_F32 ? 4 : 2) + (!outs || outs[i] == grads[i] ? 0 : out_dtypes[i] == DATTRI_F32 ? 4 : 2));
  int at = 0;
  TRY(clip_launches(grads, sizes, dtypes, outs, out_dtypes, n_tensors,
                    [&](const ClipList& l, int groups) -> dattri_status {
                      HIP_TRY(launch_clip_squares(l, groups, partials + at, bytes > kClipStream, s));
                      at += groups;
                      return DATTRI_OK;
                    }));
  HIP_TRY(launch_clip_norm(partials, at, max_norm, norm_coef, s));
  if (!outs) return DATTRI_OK;
  return clip_launches(grads, sizes, dtypes, outs, out_dtypes, n_tensors,
                       [&](const ClipList& l, int) -> dattri_status {
                         HIP_TRY(launch_clip_scale(l, norm_coef, bytes > kClipStream, s));
                         return DATTRI_OK;
                       });
}

}  // extern "C"
