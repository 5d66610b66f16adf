// The gated feed-forward block on matrices as a program trains them: plain, row-major, nothing packed or kept.
//   forward    G = X Wg, U = X Wu, H = G / (1 + e^-G) * U (Eq. 3 line 1), rounded to the type; Y = base + H Wd
//   backward   from G and U as they were stored: dH = dY Wd^T (never stored), with s = 1 / (1 + e^-G)
//              dG = dH U s (1 + G (1 - s)), dU = dH G s, rounded; dX = dx_base + dG Wg^T + dU Wu^T;
//              dWg = X^T dG, dWu = X^T dU, dWd = H^T dY
// Two launches forward and four backward (and one before each product whose operands are copied, one behind each that splits K): both projections, the activation and the product in one,
// its gradient behind the product that makes dH, dX one product over twice the width, and the two gradients that share X
// one launch.  Bound by the matrix cores (4096 tokens of 4096 x 14336 in bf16: 780 + 365 us forward, 460 + 775 + 735 + 380 backward, 1.24 to 1.36
// PFLOP/s but for dH's product, whose results are four times as large as its operands' shares) and by the weights' way out of memory with few
// tokens (one token of 4096 x 11008: 32 + 19 us, 5.6 and 4.8 TB/s).
#include <algorithm>

#include "../../include/cmoe.h"
#include "cmoe_internal.h"
#include "matmul.h"
#include "operator_args.h"

namespace cmoe {
namespace {

constexpr int64_t MOST = 1 << 20;          // tokens and widths: element offsets stay below 2^40, a tile's byte offsets below 2^31

int check_sizes(const char* what, int32_t dtype, int64_t tokens, int32_t d, int32_t d_ff) {
  if (dtype != CMOE_F32 && dtype != CMOE_BF16) return fail(CMOE_EINVAL, "%s: dtype must be CMOE_F32 or CMOE_BF16", what);
  if (tokens < 0 || tokens > MOST || d < 1 || d > MOST || d_ff < 1 || d_ff > MOST)
    return fail(CMOE_EINVAL, "%s: need 0 <= tokens <= 2^20 and widths from 1 to 2^20", what);
  return CMOE_OK;
}

size_t forward_bytes(int dtype, int64_t t, int64_t d, int64_t f) {
  return std::max(matmul_workspace_bytes(PRODUCT_GATED, dtype, t, f, d), matmul_workspace_bytes(PRODUCT_DOWN, dtype, t, d, f));
}
size_t backward_bytes(int dtype, int64_t t, int64_t d, int64_t f) {
  return std::max({matmul_workspace_bytes(PRODUCT_DGATED, dtype, t, f, d), matmul_workspace_bytes(PRODUCT_DX, dtype, t, d, f),
                   matmul_workspace_bytes(PRODUCT_DW, dtype, d, f, t), matmul_workspace_bytes(PRODUCT_DW, dtype, f, d, t)});
}

int check_workspace(const char* what, const void* ws, uint64_t have, size_t need) {
  if (need == 0) return CMOE_OK;
  if (!ws || (uintptr_t)ws % 16 != 0) return fail(CMOE_EINVAL, "%s: the workspace is null or not aligned to 16 bytes", what);
  if (have < need) return fail(CMOE_EINVAL, "%s: the workspace has %llu bytes and needs %llu", what, (unsigned long long)have, (unsigned long long)need);
  return CMOE_OK;
}

int launched(const char* what, hipError_t e) { return e == hipSuccess ? CMOE_OK : fail(CMOE_EHIP, "%s: %s", what, hipGetErrorString(e)); }

}  // namespace
}  // namespace cmoe

extern "C" size_t cmoe_ffn_forward_workspace_bytes(int64_t tokens, int32_t d, int32_t d_ff, int32_t dtype) {
  using namespace cmoe;
  return check_sizes("cmoe_ffn_forward", dtype, tokens, d, d_ff) ? 0 : forward_bytes(dtype, tokens, d, d_ff);
}

extern "C" int cmoe_ffn_forward(const cmoe_ffn_forward_args* args, void* hip_stream) {
  using namespace cmoe;
  const char* what = "cmoe_ffn_forward";
  if (!args || args->struct_bytes != (int32_t)sizeof(*args)) return fail(CMOE_EINVAL, "%s: the arguments are null or a struct of another version", what);
  const auto& a = *args;
  if (int rc = check_sizes(what, a.dtype, a.tokens, a.d, a.d_ff)) return rc;
  if (!a.gate != !a.up) return fail(CMOE_EINVAL, "%s: gate and up are given together", what);
  if (a.tokens == 0) return CMOE_OK;
  if (!a.x || !a.w_gate || !a.w_up || !a.w_down || !a.hidden || !a.y) return fail(CMOE_EINVAL, "%s: x, a weight, hidden or y is null", what);
  const size_t es = elem_size(a.dtype);
  const uint64_t td = (uint64_t)a.tokens * a.d * es, tf = (uint64_t)a.tokens * a.d_ff * es, df = (uint64_t)a.d * a.d_ff * es;
  const size_t need = forward_bytes(a.dtype, a.tokens, a.d, a.d_ff);
  if (int rc = check_workspace(what, a.workspace, a.workspace_bytes, need)) return rc;
  if (int rc = check_operands(what, {{"x", a.x, td, es}, {"w_gate", a.w_gate, df, es}, {"w_up", a.w_up, df, es}, {"w_down", a.w_down, df, es}, {"base", a.base, td, es, true}},
                              {{"y", a.y, td, es, true}, {"hidden", a.hidden, tf, es}, {"gate", a.gate, tf, es}, {"up", a.up, tf, es}, {"the workspace", need ? a.workspace : nullptr, need, 16}}))
    return rc;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  MatArgs p = {};
  p.a = a.x, p.lda = a.d, p.b = a.w_gate, p.b2 = a.w_up, p.ldb = a.d_ff;
  p.m = (int)a.tokens, p.n = a.d_ff, p.k = a.d;
  p.c = a.hidden, p.c2 = a.gate, p.c3 = a.up, p.ldc = a.d_ff;
  if (hipError_t e = matmul(PRODUCT_GATED, a.dtype, p, a.workspace, need, s)) return launched(what, e);
  MatArgs q = {};
  q.a = a.hidden, q.lda = a.d_ff, q.b = a.w_down, q.ldb = a.d;
  q.m = (int)a.tokens, q.n = a.d, q.k = a.d_ff;
  q.c = a.y, q.e1 = a.base, q.ldc = a.d;
  return launched(what, matmul(PRODUCT_DOWN, a.dtype, q, a.workspace, need, s));
}

extern "C" size_t cmoe_ffn_backward_workspace_bytes(int64_t tokens, int32_t d, int32_t d_ff, int32_t dtype) {
  using namespace cmoe;
  return check_sizes("cmoe_ffn_backward", dtype, tokens, d, d_ff) ? 0 : backward_bytes(dtype, tokens, d, d_ff);
}

extern "C" int cmoe_ffn_backward(const cmoe_ffn_backward_args* args, void* hip_stream) {
  using namespace cmoe;
  const char* what = "cmoe_ffn_backward";
  if (!args || args->struct_bytes != (int32_t)sizeof(*args)) return fail(CMOE_EINVAL, "%s: the arguments are null or a struct of another version", what);
  const auto& a = *args;
  if (int rc = check_sizes(what, a.dtype, a.tokens, a.d, a.d_ff)) return rc;
  if (a.dx_base && !a.dx) return fail(CMOE_EINVAL, "%s: dx_base without dx", what);
  if (a.tokens > 0) {
    if (!a.dy || !a.gate || !a.up || !a.w_down || !a.dgate || !a.dup) return fail(CMOE_EINVAL, "%s: dy, gate, up, w_down, dgate or dup is null", what);
    if (a.dx && (!a.w_gate || !a.w_up)) return fail(CMOE_EINVAL, "%s: dx needs w_gate and w_up", what);
    if ((a.dw_gate || a.dw_up) && !a.x) return fail(CMOE_EINVAL, "%s: dw_gate and dw_up need x", what);
    if (a.dw_down && !a.hidden) return fail(CMOE_EINVAL, "%s: dw_down needs hidden", what);
  }
  const size_t es = elem_size(a.dtype);
  const uint64_t td = (uint64_t)a.tokens * a.d * es, tf = (uint64_t)a.tokens * a.d_ff * es, df = (uint64_t)a.d * a.d_ff * es;
  const size_t need = backward_bytes(a.dtype, a.tokens, a.d, a.d_ff);
  if (int rc = check_workspace(what, a.workspace, a.workspace_bytes, need)) return rc;
  const void* ws = need ? a.workspace : nullptr;
  // dgate and dup over gate and up, and dx over dx_base, each in its own launch
  if (int rc = check_operands(what,
                              {{"dy", a.dy, td, es}, {"x", a.x, td, es}, {"gate", a.gate, tf, es, true}, {"up", a.up, tf, es, true}, {"hidden", a.hidden, tf, es},
                               {"w_gate", a.w_gate, df, es}, {"w_up", a.w_up, df, es}, {"w_down", a.w_down, df, es}, {"dx_base", a.dx_base, td, es}},
                              {{"dgate", a.dgate, tf, es, true}, {"dup", a.dup, tf, es, true}, {"dw_gate", a.dw_gate, df, es}, {"dw_up", a.dw_up, df, es},
                               {"dw_down", a.dw_down, df, es}, {"the workspace", ws, need, 16}}))
    return rc;
  if (int rc = check_operands(what,
                              {{"dy", a.dy, td, es}, {"x", a.x, td, es}, {"gate", a.gate, tf, es}, {"up", a.up, tf, es}, {"hidden", a.hidden, tf, es}, {"w_gate", a.w_gate, df, es},
                               {"w_up", a.w_up, df, es}, {"w_down", a.w_down, df, es}, {"dx_base", a.dx_base, td, es, true}, {"dgate", a.dgate, tf, es}, {"dup", a.dup, tf, es},
                               {"dw_gate", a.dw_gate, df, es}, {"dw_up", a.dw_up, df, es}, {"dw_down", a.dw_down, df, es}, {"the workspace", ws, need, 16}},
                              {{"dx", a.dx, td, es, true}}))
    return rc;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (a.tokens > 0) {
    MatArgs p = {};
    p.a = a.dy, p.lda = a.d, p.b = a.w_down, p.ldb = a.d;
    p.m = (int)a.tokens, p.n = a.d_ff, p.k = a.d;
    p.e1 = a.gate, p.e2 = a.up, p.c = a.dgate, p.c2 = a.dup, p.ldc = a.d_ff;
    if (hipError_t e = matmul(PRODUCT_DGATED, a.dtype, p, a.workspace, need, s)) return launched(what, e);
    if (a.dx) {
      MatArgs q = {};
      q.a = a.dgate, q.a2 = a.dup, q.lda = a.d_ff, q.b = a.w_gate, q.b2 = a.w_up, q.ldb = a.d_ff;
      q.m = (int)a.tokens, q.n = a.d, q.k = a.d_ff;
      q.c = a.dx, q.e1 = a.dx_base, q.ldc = a.d;
      if (hipError_t e = matmul(PRODUCT_DX, a.dtype, q, a.workspace, need, s)) return launched(what, e);
    }
  }
  auto weights = [&](const void* left, int m, const void* right, const void* right2, int n, void* c, void* c2) {
    MatArgs q = {};
    q.a = left, q.lda = m, q.b = right, q.b2 = right2, q.ldb = n;
    q.m = m, q.n = n, q.k = (int)a.tokens;
    q.c = c, q.c2 = c2, q.ldc = n, q.alpha = 1.0f;
    return matmul(PRODUCT_DW, a.dtype, q, a.workspace, need, s);
  };
  if (a.dw_gate && a.dw_up) {
    if (hipError_t e = weights(a.x, a.d, a.dgate, a.dup, a.d_ff, a.dw_gate, a.dw_up)) return launched(what, e);
  } else if (a.dw_gate || a.dw_up) {
    if (hipError_t e = weights(a.x, a.d, a.dw_gate ? a.dgate : a.dup, nullptr, a.d_ff, a.dw_gate ? a.dw_gate : a.dw_up, nullptr)) return launched(what, e);
  }
  if (a.dw_down)
    if (hipError_t e = weights(a.hidden, a.d_ff, a.dy, nullptr, a.d, a.dw_down, nullptr)) return launched(what, e);
  return CMOE_OK;
}
