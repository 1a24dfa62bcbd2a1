// C ABI of the norm, the 8-bit rows, weights and products, and the experts'
// linear layers: argument checks, workspace layout and launches.
#include <algorithm>
#include <cmath>

#include "api_common.h"
#include "dattri.h"
#include "model_checks.h"
#include "model_ops.h"

using namespace dattri;

namespace {

int64_t groups_of(int64_t d) { return (d + 127) / 128; }

// 8-bit values and their scales: `rows` rows of d columns, `srows` rows of scales.
dattri_status check_8bit(const char* what, const void* q, int64_t* ldq, const void* s, int64_t* lds, int64_t rows,
                         int64_t srows, int64_t d) {
  TRY(check_rows(what, q, ldq, rows, d, 1, true));
  return check_rows("scales", s, lds, srows, groups_of(d), 4, true);
}

dattri_status check_eps(float eps) {
  if (!(eps >= 0.f) || std::isinf(eps)) return fail(DATTRI_E_INVALID_ARG, "eps must be finite and >= 0");
  return DATTRI_OK;
}

dattri_status check_experts(int64_t experts, int64_t d_out, const void* offsets, int32_t offset_bytes, bool needed) {
  if (experts < 1) return fail(DATTRI_E_INVALID_ARG, "experts must be >= 1 (got %lld)", (long long)experts);
  if (experts > 65535) return fail(DATTRI_E_UNSUPPORTED, "%lld experts are more than 65535", (long long)experts);
  TRY(check_count("experts * d_out", experts * d_out));
  if (!needed) return DATTRI_OK;
  if (offset_bytes != 4 && offset_bytes != 8)
    return fail(DATTRI_E_INVALID_ARG, "offset_bytes must be 4 or 8 (got %d)", offset_bytes);
  if (!offsets) return fail(DATTRI_E_INVALID_ARG, "offsets is NULL");
  if ((uintptr_t)offsets % offset_bytes)
    return fail(DATTRI_E_INVALID_ARG, "offsets is not aligned to its elements");
  return DATTRI_OK;
}

dattri_status check_product(int64_t rows, int64_t d_in, int64_t d_out, dattri_dtype dtype, int* elt) {
  TRY(elt_of(dtype, elt));
  TRY(check_count("rows", rows));
  TRY(check_width("d_in", d_in));
  return check_width("d_out", d_out);
}

dattri_status check_bias(const char* what, const void* p, int elt) {
  if ((uintptr_t)p % elt) return fail(DATTRI_E_INVALID_ARG, "%s is not aligned to its elements", what);
  return DATTRI_OK;
}

}  // namespace

extern "C" {

dattri_status dattri_rms_norm(const void* X, int64_t ld_x, const void* R, int64_t ld_r, const void* W, float eps,
                              void* Y, int64_t ld_y, void* H, int64_t ld_h, void* Q, int64_t ld_q, float* S,
                              int64_t ld_s, int64_t rows, int64_t d, dattri_dtype dtype, void* stream) {
  reset_error();
  int elt;
  TRY(elt_of(dtype, &elt));
  TRY(check_count("rows", rows));
  TRY(check_width("d", d));
  TRY(check_eps(eps));
  TRY(check_rows("X", X, &ld_x, rows, d, elt, true));
  TRY(check_rows("R", R, &ld_r, rows, d, elt, false));
  TRY(check_rows("Y", Y, &ld_y, rows, d, elt, false));
  TRY(check_rows("H", H, &ld_h, rows, d, elt, false));
  if (!W) return fail(DATTRI_E_INVALID_ARG, "W is NULL");
  TRY(check_bias("W", W, elt));
  if (rows > 0 && !Y && !Q) return fail(DATTRI_E_INVALID_ARG, "nothing to compute: Y and Q are NULL");
  if (!Q != !S) return fail(DATTRI_E_INVALID_ARG, "Q and S go together");
  if (H && !R) return fail(DATTRI_E_INVALID_ARG, "H without R would be X");
  TRY(check_rows("Q", Q, &ld_q, rows, d, 1, false));
  TRY(check_rows("S", S, &ld_s, rows, groups_of(d), 4, false));
  {
    const Span x("X", X, rows, d, ld_x, elt), r("R", R, rows, d, ld_r, elt), w("W", W, d * elt),
        y("Y", Y, rows, d, ld_y, elt), h("H", H, rows, d, ld_h, elt), q("Q", Q, rows, d, ld_q, 1),
        s("S", S, rows, groups_of(d), ld_s, 4);
    TRY(check_apart(y, {w, h, q, s}, &x, &r));
    TRY(check_apart(h, {w, q, s}, &x, &r));
    TRY(check_apart(q, {x, r, w, s}));
    TRY(check_apart(s, {x, r, w}));
  }
  if (rows == 0) return DATTRI_OK;
  NormArgs a = {};
  a.X = X;
  a.R = R;
  a.W = W;
  a.ldx = ld_x;
  a.ldr = ld_r;
  a.rows = rows;
  a.d = (int)d;
  a.eps = eps;
  a.Y = Y;
  a.H = H;
  a.ldy = ld_y;
  a.ldh = ld_h;
  a.Q = (uint8_t*)Q;
  a.S = S;
  a.ldq = ld_q;
  a.lds = ld_s;
  HIP_TRY(launch_rms_norm(elt, a, (hipStream_t)stream));
  return DATTRI_OK;
}

dattri_status dattri_rms_norm_grad_workspace_bytes(int64_t rows, int64_t d, dattri_dtype dtype, int32_t weight,
                                                   size_t* bytes) {
  reset_error();
  int elt;
  if (!bytes) return fail(DATTRI_E_INVALID_ARG, "bytes is NULL");
  TRY(elt_of(dtype, &elt));
  TRY(check_count("rows", rows));
  TRY(check_width("d", d));
  *bytes = norm_grad_layout(rows, d, weight != 0).total;
  return DATTRI_OK;
}

dattri_status dattri_rms_norm_grad(const void* G, int64_t ld_g, const void* H, int64_t ld_h, const void* W, float eps,
                                   const void* P, int64_t ld_p, void* D, int64_t ld_d, float* dW, int32_t accumulate,
                                   int64_t rows, int64_t d, dattri_dtype dtype, void* workspace, size_t ws_bytes,
                                   void* stream) {
  reset_error();
  int elt;
  TRY(elt_of(dtype, &elt));
  TRY(check_count("rows", rows));
  TRY(check_width("d", d));
  TRY(check_eps(eps));
  TRY(check_rows("G", G, &ld_g, rows, d, elt, true));
  TRY(check_rows("H", H, &ld_h, rows, d, elt, true));
  TRY(check_rows("P", P, &ld_p, rows, d, elt, false));
  TRY(check_rows("D", D, &ld_d, rows, d, elt, true));
  if (!W) return fail(DATTRI_E_INVALID_ARG, "W is NULL");
  TRY(check_bias("W", W, elt));
  TRY(check_bias("dW", dW, 4));
  const size_t need = norm_grad_layout(rows, d, dW != nullptr).total;
  TRY(check_workspace(workspace, ws_bytes, need));
  {
    const Span g("G", G, rows, d, ld_g, elt), h("H", H, rows, d, ld_h, elt), w("W", W, d * elt),
        p("P", P, rows, d, ld_p, elt), out("D", D, rows, d, ld_d, elt), dw("dW", dW, d * 4);
    TRY(check_apart(out, {g, h, w, dw}, &p));
    TRY(check_apart(dw, {g, h, w, p}));
    TRY(check_apart(Span("workspace", workspace, (int64_t)need), {g, h, w, p, out, dw}));
  }
  if (rows == 0 && (!dW || accumulate)) return DATTRI_OK;
  NormGradArgs a = {};
  a.G = G;
  a.H = H;
  a.W = W;
  a.P = P;
  a.ldg = ld_g;
  a.ldh = ld_h;
  a.ldp = ld_p;
  a.rows = rows;
  a.d = (int)d;
  a.eps = eps;
  a.D = D;
  a.ldd = ld_d;
  HIP_TRY(launch_norm_grad(elt, a, dW, accumulate != 0, (uint8_t*)workspace, (hipStream_t)stream));
  return DATTRI_OK;
}

dattri_status dattri_quantize_rows(const void* X, int64_t ld_x, int64_t rows, int64_t d, dattri_dtype dtype, void* Q,
                                   int64_t ld_q, float* S, int64_t ld_s, void* stream) {
  reset_error();
  int elt;
  TRY(elt_of(dtype, &elt));
  TRY(check_count("rows", rows));
  TRY(check_width("d", d));
  TRY(check_rows("X", X, &ld_x, rows, d, elt, true));
  TRY(check_8bit("Q", Q, &ld_q, S, &ld_s, rows, rows, d));
  {
    const Span x("X", X, rows, d, ld_x, elt), q("Q", Q, rows, d, ld_q, 1), s("S", S, rows, groups_of(d), ld_s, 4);
    TRY(check_apart(q, {x, s}));
    TRY(check_apart(s, {x}));
  }
  if (rows == 0) return DATTRI_OK;
  HIP_TRY(launch_quantize_rows(elt, X, ld_x, rows, d, (uint8_t*)Q, ld_q, S, ld_s, (hipStream_t)stream));
  return DATTRI_OK;
}

dattri_status dattri_quantize_weight(const void* W, int64_t ld_w, int64_t d_out, int64_t d_in, dattri_dtype dtype,
                                     void* Q, int64_t ld_q, float* S, int64_t ld_s, void* stream) {
  reset_error();
  int elt;
  TRY(elt_of(dtype, &elt));
  TRY(check_width("d_out", d_out));
  TRY(check_width("d_in", d_in));
  TRY(check_rows("W", W, &ld_w, d_out, d_in, elt, true));
  TRY(check_8bit("Q", Q, &ld_q, S, &ld_s, d_out, groups_of(d_out), d_in));
  {
    const Span w("W", W, d_out, d_in, ld_w, elt), q("Q", Q, d_out, d_in, ld_q, 1),
        s("S", S, groups_of(d_out), groups_of(d_in), ld_s, 4);
    TRY(check_apart(q, {w, s}));
    TRY(check_apart(s, {w}));
  }
  HIP_TRY(launch_quantize_weight(elt, W, ld_w, d_out, d_in, (uint8_t*)Q, ld_q, S, ld_s, (hipStream_t)stream));
  return DATTRI_OK;
}

dattri_status dattri_linear_scaled_workspace_bytes(int64_t rows, int64_t d_in, int64_t d_out, dattri_dtype dtype,
                                                 int32_t aligned, size_t* bytes) {
  reset_error();
  int elt;
  if (!bytes) return fail(DATTRI_E_INVALID_ARG, "bytes is NULL");
  TRY(check_product(rows, d_in, d_out, dtype, &elt));
  *bytes = linear8_workspace_need(rows, d_in, d_out, elt, aligned != 0);
  return DATTRI_OK;
}

dattri_status dattri_linear_scaled(const void* X, int64_t ld_x, const float* SX, int64_t ld_sx, const void* W,
                                 int64_t ld_w, const float* SW, int64_t ld_sw, const void* bias, dattri_act act,
                                 const void* R, int64_t ld_r, void* Y, int64_t ld_y, void* Z, int64_t ld_z,
                                 int64_t rows, int64_t d_in, int64_t d_out, dattri_dtype dtype, void* workspace,
                                 size_t ws_bytes, void* stream) {
  reset_error();
  int elt;
  TRY(check_product(rows, d_in, d_out, dtype, &elt));
  TRY(check_act(act));
  TRY(check_8bit("X", X, &ld_x, SX, &ld_sx, rows, rows, d_in));
  TRY(check_8bit("W", W, &ld_w, SW, &ld_sw, d_out, groups_of(d_out), d_in));
  TRY(check_rows("R", R, &ld_r, rows, d_out, elt, false));
  TRY(check_rows("Y", Y, &ld_y, rows, d_out, elt, true));
  TRY(check_rows("Z", Z, &ld_z, rows, d_out, elt, false));
  TRY(check_bias("bias", bias, elt));
  const bool aligned = on_16(X, ld_x, W, ld_w, 1);
  const size_t need = linear8_workspace_need(rows, d_in, d_out, elt, aligned);
  TRY(check_workspace(workspace, ws_bytes, need));
  {
    const Span x("X", X, rows, d_in, ld_x, 1), sx("SX", SX, rows, groups_of(d_in), ld_sx, 4),
        w("W", W, d_out, d_in, ld_w, 1), sw("SW", SW, groups_of(d_out), groups_of(d_in), ld_sw, 4),
        b("bias", bias, d_out * elt), r("R", R, rows, d_out, ld_r, elt), y("Y", Y, rows, d_out, ld_y, elt),
        z("Z", Z, rows, d_out, ld_z, elt);
    TRY(check_apart(y, {x, sx, w, sw, b, z}, &r));
    TRY(check_apart(z, {x, sx, w, sw, b, r}));
    TRY(check_apart(Span("workspace", workspace, (int64_t)need), {x, sx, w, sw, b, r, y, z}));
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
  HIP_TRY(launch_linear8(elt, aligned, a, Scales8{SX, SW, ld_sx, ld_sw}, (uint8_t*)workspace, (hipStream_t)stream));
  return DATTRI_OK;
}

dattri_status dattri_expert_linear_workspace_bytes(dattri_linear_op op, int64_t rows, int64_t experts, int64_t d_in,
                                                   int64_t d_out, dattri_dtype dtype, int32_t aligned,
                                                   size_t* bytes) {
  reset_error();
  int elt;
  if (!bytes) return fail(DATTRI_E_INVALID_ARG, "bytes is NULL");
  if ((int)op < DATTRI_LINEAR_FORWARD || (int)op > DATTRI_LINEAR_WEIGHT_GRAD)
    return fail(DATTRI_E_INVALID_ARG, "unknown linear op %d", (int)op);
  TRY(check_product(rows, d_in, d_out, dtype, &elt));
  TRY(check_experts(experts, d_out, nullptr, 0, false));
  *bytes = expert_workspace_need(op, rows, experts, d_in, d_out, elt, aligned != 0);
  return DATTRI_OK;
}

dattri_status dattri_expert_linear(const void* X, int64_t ld_x, const void* W, int64_t ld_w, const void* bias,
                                   const void* offsets, int32_t offset_bytes, dattri_act act, const void* R,
                                   int64_t ld_r, void* Y, int64_t ld_y, void* Z, int64_t ld_z, int64_t rows,
                                   int64_t experts, int64_t d_in, int64_t d_out, dattri_dtype dtype, void* workspace,
                                   size_t ws_bytes, void* stream) {
  reset_error();
  int elt;
  TRY(check_product(rows, d_in, d_out, dtype, &elt));
  TRY(check_experts(experts, d_out, offsets, offset_bytes, true));
  TRY(check_act(act));
  TRY(check_rows("X", X, &ld_x, rows, d_in, elt, true));
  TRY(check_rows("W", W, &ld_w, experts * d_out, d_in, elt, true));
  TRY(check_rows("R", R, &ld_r, rows, d_out, elt, false));
  TRY(check_rows("Y", Y, &ld_y, rows, d_out, elt, true));
  TRY(check_rows("Z", Z, &ld_z, rows, d_out, elt, false));
  TRY(check_bias("bias", bias, elt));
  const bool aligned = on_16(X, ld_x, W, ld_w, elt);
  const size_t need = expert_workspace_need(DATTRI_LINEAR_FORWARD, rows, experts, d_in, d_out, elt, aligned);
  TRY(check_workspace(workspace, ws_bytes, need));
  {
    const Span x("X", X, rows, d_in, ld_x, elt), w("W", W, experts * d_out, d_in, ld_w, elt),
        b("bias", bias, experts * d_out * elt), o("offsets", offsets, (experts + 1) * offset_bytes),
        r("R", R, rows, d_out, ld_r, elt), y("Y", Y, rows, d_out, ld_y, elt), z("Z", Z, rows, d_out, ld_z, elt);
    TRY(check_apart(y, {x, w, b, o, z}, &r));
    TRY(check_apart(z, {x, w, b, o, r}));
    TRY(check_apart(Span("workspace", workspace, (int64_t)need), {x, w, b, o, r, y, z}));
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
  HIP_TRY(launch_expert(DATTRI_LINEAR_FORWARD, elt, aligned, a,
                        ExpertArgs{offsets, offset_bytes, (int)experts, (int)rows, ld_w * d_out}, nullptr,
                        (uint8_t*)workspace, (hipStream_t)stream));
  return DATTRI_OK;
}

dattri_status dattri_expert_linear_input_grad(const void* G, int64_t ld_g, const void* W, int64_t ld_w,
                                              const void* offsets, int32_t offset_bytes, const void* R, int64_t ld_r,
                                              dattri_act act, const void* Z, int64_t ld_z, void* D, int64_t ld_d,
                                              void* P, int64_t ld_p, int64_t rows, int64_t experts, int64_t d_in,
                                              int64_t d_out, dattri_dtype dtype, void* workspace, size_t ws_bytes,
                                              void* stream) {
  reset_error();
  int elt;
  TRY(check_product(rows, d_in, d_out, dtype, &elt));
  TRY(check_experts(experts, d_out, offsets, offset_bytes, true));
  TRY(check_act(act));
  TRY(check_rows("G", G, &ld_g, rows, d_out, elt, true));
  TRY(check_rows("W", W, &ld_w, experts * d_out, d_in, elt, true));
  TRY(check_rows("R", R, &ld_r, rows, d_in, elt, false));
  TRY(check_rows("Z", Z, &ld_z, rows, d_in, elt, P && act != DATTRI_ACT_NONE));
  TRY(check_rows("D", D, &ld_d, rows, d_in, elt, false));
  TRY(check_rows("P", P, &ld_p, rows, d_in, elt, false));
  if (rows > 0 && !D && !P) return fail(DATTRI_E_INVALID_ARG, "nothing to compute: D and P are NULL");
  const bool aligned = on_16(G, ld_g, W, ld_w, elt);
  const size_t need = expert_workspace_need(DATTRI_LINEAR_INPUT_GRAD, rows, experts, d_in, d_out, elt, aligned);
  TRY(check_workspace(workspace, ws_bytes, need));
  {
    const Span g("G", G, rows, d_out, ld_g, elt), w("W", W, experts * d_out, d_in, ld_w, elt),
        o("offsets", offsets, (experts + 1) * offset_bytes), r("R", R, rows, d_in, ld_r, elt),
        z("Z", act == DATTRI_ACT_NONE || !P ? nullptr : Z, rows, d_in, ld_z, elt), d("D", D, rows, d_in, ld_d, elt),
        p("P", P, rows, d_in, ld_p, elt);
    TRY(check_apart(d, {g, w, o, z, p}, &r));
    TRY(check_apart(p, {g, w, o}, &r, &z));
    TRY(check_apart(Span("workspace", workspace, (int64_t)need), {g, w, o, r, z, d, p}));
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
  HIP_TRY(launch_expert(DATTRI_LINEAR_INPUT_GRAD, elt, aligned, a,
                        ExpertArgs{offsets, offset_bytes, (int)experts, (int)rows, ld_w * d_out}, nullptr,
                        (uint8_t*)workspace, (hipStream_t)stream));
  return DATTRI_OK;
}

dattri_status dattri_expert_linear_weight_grad(const void* G, int64_t ld_g, const void* X, int64_t ld_x,
                                               const void* offsets, int32_t offset_bytes, float* dW, int64_t ld_dw,
                                               float* dbias, int32_t accumulate, int64_t rows, int64_t experts,
                                               int64_t d_in, int64_t d_out, dattri_dtype dtype, void* workspace,
                                               size_t ws_bytes, void* stream) {
  reset_error();
  int elt;
  TRY(check_product(rows, d_in, d_out, dtype, &elt));
  TRY(check_experts(experts, d_out, offsets, offset_bytes, true));
  TRY(check_rows("G", G, &ld_g, rows, d_out, elt, true));
  TRY(check_rows("X", X, &ld_x, rows, d_in, elt, dW != nullptr));
  TRY(check_rows("dW", dW, &ld_dw, experts * d_out, d_in, 4, false));
  TRY(check_bias("dbias", dbias, 4));
  if (!dW && !dbias) return fail(DATTRI_E_INVALID_ARG, "nothing to compute: dW and dbias are NULL");
  const bool aligned = !dW || on_16(G, ld_g, X, ld_x, elt);  // bias alone: no operands
  const size_t need = expert_workspace_need(DATTRI_LINEAR_WEIGHT_GRAD, rows, experts, d_in, d_out, elt, aligned);
  TRY(check_workspace(workspace, ws_bytes, need));
  {
    const Span g("G", G, rows, d_out, ld_g, elt), x("X", dW ? X : nullptr, rows, d_in, ld_x, elt),
        o("offsets", offsets, (experts + 1) * offset_bytes), w("dW", dW, experts * d_out, d_in, ld_dw, 4),
        b("dbias", dbias, experts * d_out * 4);
    TRY(check_apart(w, {g, x, o, b}));
    TRY(check_apart(b, {g, x, o}));
    TRY(check_apart(Span("workspace", workspace, (int64_t)need), {g, x, o, w, b}));
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
  HIP_TRY(launch_expert(DATTRI_LINEAR_WEIGHT_GRAD, elt, aligned, a,
                        ExpertArgs{offsets, offset_bytes, (int)experts, (int)rows, ld_dw * d_out}, dbias,
                        (uint8_t*)workspace, (hipStream_t)stream));
  return DATTRI_OK;
}

}  // extern "C"
