// Softmax cross entropy of a head over a vocabulary, without its logits in memory.
//   forward    z = X W^T in registers: every tile leaves the largest logit m of its columns of a row and the sum of
//              exp(z - m), and the target's logit; lse = log sum exp z over the ranges, loss = lse - z[target], 0 without a target
//   backward   in pieces of the vocabulary: z once more, dZ = weight * (exp(z - lse) - [target]) of a piece in the type, then
//              dX += dZ W (fp32 between the pieces) and dW = scale * dZ^T X, complete for the piece's rows
// What a piece costs beside its products is dX's sums, read and written, so pieces are as wide as 128 MB of dZ allow:
// it is read twice soon after it is written, and this part's last cache holds 256 MB.
// dW takes x from a copy without the rows of tokens that have no target: what such a row holds (padding, NaN) would reach every row of dW as 0 times it.
// Bound by the matrix cores (8192 tokens of 4096 over 131072 in bf16: forward 6.5 ms, 1.35 PFLOP/s; per piece of 8192 entries 440 us of logits, 420 of dX,
// 370 of dW) and by the vocabulary's way out of memory with few tokens (one token over 32768: 45 us, 5.9 TB/s).
// `scale` and the factor on the device are applied to the sums in fp32, and not to dZ: what all tokens share would round the entries of all targets,
// which are all close to -scale, to the same side.
#include <algorithm>

#include "../../include/cmoe.h"
#include "cmoe_internal.h"
#include "matmul_device.h"
#include "operator_args.h"

namespace cmoe {
namespace {

constexpr int64_t MOST = 1 << 20;
constexpr int64_t PIECE_BYTES = 128 << 20;
constexpr int64_t PIECE_LEAST = 1024;

int check_sizes(const char* what, int32_t dtype, int64_t tokens, int32_t d, int32_t vocab) {
  if (dtype != CMOE_F32 && dtype != CMOE_BF16) return fail(CMOE_EINVAL, "%s: dtype must be CMOE_F32 or CMOE_BF16", what);
  if (tokens < 0 || tokens > MOST || d < 1 || d > MOST || vocab < 1 || vocab > MOST)
    return fail(CMOE_EINVAL, "%s: need 0 <= tokens <= 2^20, d and vocab from 1 to 2^20", what);
  return CMOE_OK;
}

size_t round16(size_t n) { return (n + 15) / 16 * 16; }

// How many vocabulary entries a piece may have for the copies of their rows, where operands may be copied, to stay below 256 MB (up to a width of
// 8192); all of them otherwise.
int64_t copied_piece(int dtype, int64_t t, int64_t d, int64_t vocab, const LogitsPlan& plan) {
  const int64_t most = std::max<int64_t>(4096, ((int64_t)1 << 35) / t / 256 * 256);      // (a launch has fewer than 2^32 threads)
  if (plan.in_place) return std::min(vocab, most);
  return std::min({vocab, most, std::max<int64_t>(4096, ((int64_t)1 << (dtype == CMOE_F32 ? 25 : 27)) / d / 256 * 256)});
}

struct ForwardSpace {
  LogitsPlan plan;
  int64_t piece, last;                     // entries of a piece, and of the last one
  size_t picked, product, total;           // offsets of the targets' logits and of the products' workspace; the ranges at 0
  ForwardSpace(int dtype, int64_t t, int64_t d, int64_t vocab) {
    plan = logits_plan(dtype, t, vocab, d);
    piece = copied_piece(dtype, t, d, vocab, plan);
    const int64_t pieces = (vocab - 1) / piece;              // but the last
    last = vocab - pieces * piece;
    const int64_t ranges = pieces * lse_ranges(dtype, t, piece, d, plan) + lse_ranges(dtype, t, last, d, plan);
    picked = round16((size_t)ranges * t * sizeof(float2));
    product = picked + round16((size_t)t * 4);
    total = product + std::max(matmul_workspace_bytes(PRODUCT_LSE, dtype, t, piece, d, &plan), matmul_workspace_bytes(PRODUCT_LSE, dtype, t, last, d, &plan));
  }
};

struct BackwardSpace {
  LogitsPlan plan;
  int64_t piece, ld;                       // vocabulary entries of a piece, elements of a row of dZ
  size_t acc, rows, product, total;        // offsets of dX's sums, of x's rows that count and of the products' workspace; dZ at 0
  BackwardSpace(int dtype, int64_t t, int64_t d, int64_t vocab) {
    plan = logits_plan(dtype, t, vocab, d);
    piece = std::max(PIECE_LEAST, PIECE_BYTES / (int64_t)elem_size(dtype) / std::max<int64_t>(t, 1) / 256 * 256);
    piece = std::min(piece, copied_piece(dtype, t, d, vocab, plan));
    ld = (piece + 7) / 8 * 8;
    acc = round16((size_t)t * ld * elem_size(dtype));
    rows = acc + (piece < vocab ? round16((size_t)t * d * 4) : 0);
    product = rows + round16((size_t)t * d * elem_size(dtype));
    size_t most = 0;
    const int64_t last = vocab - (vocab - 1) / piece * piece;
    for (int64_t w : {piece, last}) {
      const int64_t padded = (w + 7) / 8 * 8;
      most = std::max({most, matmul_workspace_bytes(PRODUCT_DLOGITS, dtype, t, padded, d, &plan), matmul_workspace_bytes(PRODUCT_DHEAD, dtype, t, d, padded),
                       matmul_workspace_bytes(PRODUCT_DW, dtype, w, d, t)});
    }
    total = product + most;
  }
};

// A row's ranges joined: ROWS rows to a workgroup, its threads over the ranges, then in LDS.
template <int ROWS>
__global__ __launch_bounds__(256) void head_finish(const float2* part, int ranges, const float* picked, const int32_t* ids, int vocab, int64_t tokens, float* loss,
                                                   float* lse) {
  __shared__ float2 joined[256];
  constexpr int GROUPS = 256 / ROWS;
  const int r = threadIdx.x % ROWS, g = threadIdx.x / ROWS;
  const int64_t row = (int64_t)blockIdx.x * ROWS + r;
  float2 mine = {-INFINITY, 0.0f};
  if (row < tokens) {
#pragma unroll 4
    for (int i = g; i < ranges; i += GROUPS) mine = join_ranges(mine, part[(int64_t)i * tokens + row]);
  }
  joined[threadIdx.x] = mine;
  for (int half = GROUPS / 2; half > 0; half /= 2) {
    __syncthreads();
    if (g < half) joined[threadIdx.x] = mine = join_ranges(mine, joined[threadIdx.x + half * ROWS]);
  }
  if (g == 0 && row < tokens) {
    const float rest = logf(mine.y);
    if (lse) lse[row] = mine.x + rest;
    // (not lse - picked: a target that is nearly certain has a loss far below the rounding of lse)
    if (loss) loss[row] = (uint32_t)ids[row] < (uint32_t)vocab ? (mine.x - picked[row]) + rest : 0.0f;
  }
}

// x without the rows of tokens that have no target.  A thread per eight columns.
template <typename T>
__global__ __launch_bounds__(256) void head_rows(const T* x, const int32_t* ids, int vocab, int64_t tokens, int d, T* out) {
  const uint32_t per_row = (uint32_t)(d + 7) >> 3;
  const uint64_t first = (uint64_t)blockIdx.x * 256;
  const uint64_t row0 = first / per_row;
  const uint32_t c0 = (uint32_t)(first - row0 * per_row) + threadIdx.x;
  const int64_t row = row0 + c0 / per_row;
  if (row >= tokens) return;
  const int col = (int)(c0 % per_row) * 8, n = d - col;
  float v[8];
  load8(x + row * d + col, n, v);
  const bool has = (uint32_t)ids[row] < (uint32_t)vocab;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = has ? v[e] : 0.0f;
  store8(out + row * d + col, n, v);
}

int check_workspace(const char* what, const void* ws, uint64_t have, size_t need) {
  if (!ws || (uintptr_t)ws % 16 != 0) return fail(CMOE_EINVAL, "%s: the workspace is null or not aligned to 16 bytes", what);
  if (have < need) return fail(CMOE_EINVAL, "%s: the workspace has %llu bytes and needs %llu", what, (unsigned long long)have, (unsigned long long)need);
  return CMOE_OK;
}

int launched(const char* what, hipError_t e) { return e == hipSuccess ? CMOE_OK : fail(CMOE_EHIP, "%s: %s", what, hipGetErrorString(e)); }

}  // namespace
}  // namespace cmoe

extern "C" size_t cmoe_head_loss_forward_workspace_bytes(int64_t tokens, int32_t d, int32_t vocab, int32_t dtype) {
  using namespace cmoe;
  return check_sizes("cmoe_head_loss_forward", dtype, tokens, d, vocab) || tokens == 0 ? 0 : ForwardSpace(dtype, tokens, d, vocab).total;
}

extern "C" int cmoe_head_loss_forward(const cmoe_head_loss_forward_args* args, void* hip_stream) {
  using namespace cmoe;
  const char* what = "cmoe_head_loss_forward";
  if (!args || args->struct_bytes != (int32_t)sizeof(*args)) return fail(CMOE_EINVAL, "%s: the arguments are null or a struct of another version", what);
  const auto& a = *args;
  if (int rc = check_sizes(what, a.dtype, a.tokens, a.d, a.vocab)) return rc;
  if (a.tokens == 0) return CMOE_OK;
  if (!a.x || !a.weight || !a.ids) return fail(CMOE_EINVAL, "%s: x, weight or ids is null", what);
  if (!a.loss && !a.lse) return fail(CMOE_EINVAL, "%s: neither loss nor lse is given", what);
  const size_t es = elem_size(a.dtype);
  const ForwardSpace ws(a.dtype, a.tokens, a.d, a.vocab);
  if (int rc = check_workspace(what, a.workspace, a.workspace_bytes, ws.total)) return rc;
  const uint64_t rows = (uint64_t)a.tokens * 4;
  if (int rc = check_operands(what, {{"x", a.x, (uint64_t)a.tokens * a.d * es, es}, {"weight", a.weight, (uint64_t)a.vocab * a.d * es, es}, {"ids", a.ids, rows, 4}},
                              {{"loss", a.loss, rows, 4}, {"lse", a.lse, rows, 4}, {"the workspace", a.workspace, ws.total, 16}}))
    return rc;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  char* base = static_cast<char*>(a.workspace);
  float2* part = static_cast<float2*>(a.workspace);
  float* picked = reinterpret_cast<float*>(base + ws.picked);
  int ranges = 0;
  for (int64_t first = 0; first < a.vocab; first += ws.piece) {
    MatArgs p = {};
    p.a = a.x, p.lda = a.d, p.b = static_cast<const char*>(a.weight) + (size_t)first * a.d * es, p.ldb = a.d;
    p.m = (int)a.tokens, p.n = (int)std::min(ws.piece, a.vocab - first), p.k = a.d;
    p.ids = a.ids, p.vocab = a.vocab, p.col0 = (int)first;
    p.logits = ws.plan;
    p.part = part + (size_t)ranges * a.tokens, p.picked = picked;
    int more = 0;
    if (hipError_t e = matmul(PRODUCT_LSE, a.dtype, p, base + ws.product, ws.total - ws.product, s, &more)) return launched(what, e);
    ranges += more;
  }
  // few rows: all threads to a row; many: neighbouring threads read neighbouring rows, 64 bytes of them (8192 rows of 1024 ranges: 256 bytes 61 us)
  auto finish = [&](auto kernel, int rows_of) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)((a.tokens + rows_of - 1) / rows_of)), dim3(256), 0, s, part, ranges, picked, a.ids, a.vocab, a.tokens, a.loss, a.lse);
  };
  if (a.tokens <= 512) finish(head_finish<1>, 1);
  else finish(head_finish<8>, 8);
  return launched(what, hipGetLastError());
}

extern "C" size_t cmoe_head_loss_backward_workspace_bytes(int64_t tokens, int32_t d, int32_t vocab, int32_t dtype) {
  using namespace cmoe;
  return check_sizes("cmoe_head_loss_backward", dtype, tokens, d, vocab) || tokens == 0 ? 0 : BackwardSpace(dtype, tokens, d, vocab).total;
}

extern "C" int cmoe_head_loss_backward(const cmoe_head_loss_backward_args* args, void* hip_stream) { return cmoe_head_loss_backward_scaled(args, nullptr, hip_stream); }

extern "C" int cmoe_head_loss_backward_scaled(const cmoe_head_loss_backward_args* args, const float* factor, void* hip_stream) {
  using namespace cmoe;
  const char* what = "cmoe_head_loss_backward";
  if (!args || args->struct_bytes != (int32_t)sizeof(*args)) return fail(CMOE_EINVAL, "%s: the arguments are null or a struct of another version", what);
  const auto& a = *args;
  if (int rc = check_sizes(what, a.dtype, a.tokens, a.d, a.vocab)) return rc;
  if (!a.dx && !a.dweight) return fail(CMOE_EINVAL, "%s: neither dx nor dweight is given", what);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const size_t es = elem_size(a.dtype);
  MatArgs w = {};
  w.b = a.x, w.ldb = a.d, w.n = a.d, w.k = (int)a.tokens, w.ldc = a.d, w.alpha = a.scale;
  if (a.tokens == 0) {                     // nothing to learn: a gradient of zeros
    if (!a.dweight) return CMOE_OK;
    if (int rc = check_operands(what, {}, {{"dweight", a.dweight, (uint64_t)a.vocab * a.d * es, es}})) return rc;
    w.m = a.vocab, w.lda = a.vocab, w.c = a.dweight;
    return launched(what, matmul(PRODUCT_DW, a.dtype, w, nullptr, 0, s));
  }
  if (!a.x || !a.weight || !a.ids || !a.lse) return fail(CMOE_EINVAL, "%s: x, weight, ids or lse is null", what);
  const BackwardSpace ws(a.dtype, a.tokens, a.d, a.vocab);
  if (int rc = check_workspace(what, a.workspace, a.workspace_bytes, ws.total)) return rc;
  const uint64_t rows = (uint64_t)a.tokens * 4, td = (uint64_t)a.tokens * a.d * es, vd = (uint64_t)a.vocab * a.d * es;
  if (int rc = check_operands(what, {{"x", a.x, td, es}, {"weight", a.weight, vd, es}, {"ids", a.ids, rows, 4}, {"lse", a.lse, rows, 4}, {"dloss", a.dloss, rows, 4},
                                     {"factor", factor, 4, 4}},
                              {{"dx", a.dx, td, es}, {"dweight", a.dweight, vd, es}, {"the workspace", a.workspace, ws.total, 16}}))
    return rc;
  char* base = static_cast<char*>(a.workspace);
  w.factor = factor;                       // (not without tokens: the zeros above are zeros whatever it is)
  if (a.dweight) {
    w.b = base + ws.rows;
    const unsigned groups = (unsigned)((a.tokens * ((a.d + 7) / 8) + 255) / 256);
    if (a.dtype == CMOE_BF16)
      hipLaunchKernelGGL(head_rows<bf16_t>, dim3(groups), dim3(256), 0, s, (const bf16_t*)a.x, a.ids, a.vocab, a.tokens, a.d, (bf16_t*)(base + ws.rows));
    else hipLaunchKernelGGL(head_rows<float>, dim3(groups), dim3(256), 0, s, (const float*)a.x, a.ids, a.vocab, a.tokens, a.d, (float*)(base + ws.rows));
    if (hipError_t e = hipGetLastError()) return launched(what, e);
  }
  void* const room = base + ws.product;
  const size_t room_bytes = ws.total - ws.product;
  for (int64_t first = 0; first < a.vocab; first += ws.piece) {
    const int n = (int)std::min<int64_t>(ws.piece, a.vocab - first), padded = (n + 7) / 8 * 8;
    const char* rows_of_w = static_cast<const char*>(a.weight) + (size_t)first * a.d * es;
    MatArgs p = {};
    p.a = a.x, p.lda = a.d, p.b = rows_of_w, p.ldb = a.d;
    p.m = (int)a.tokens, p.n = padded, p.n_b = n, p.k = a.d;
    p.c = base, p.ldc = ws.ld;
    p.ids = a.ids, p.vocab = a.vocab, p.col0 = (int)first, p.lse = a.lse, p.dloss = a.dloss;
    p.logits = ws.plan;
    if (hipError_t e = matmul(PRODUCT_DLOGITS, a.dtype, p, room, room_bytes, s)) return launched(what, e);
    if (a.dx) {
      MatArgs q = {};
      q.a = base, q.lda = ws.ld, q.b = rows_of_w, q.ldb = a.d;
      q.m = (int)a.tokens, q.n = a.d, q.k = padded, q.k_b = n;
      q.acc = reinterpret_cast<float*>(base + ws.acc), q.first = first == 0, q.last = first + n == a.vocab;
      q.c = a.dx, q.ldc = a.d, q.alpha = a.scale, q.factor = factor;
      if (hipError_t e = matmul(PRODUCT_DHEAD, a.dtype, q, room, room_bytes, s)) return launched(what, e);
    }
    if (a.dweight) {
      w.a = base, w.lda = ws.ld, w.m = n, w.m_a = padded;
      w.c = static_cast<char*>(a.dweight) + (size_t)first * a.d * es;
      if (hipError_t e = matmul(PRODUCT_DW, a.dtype, w, room, room_bytes, s)) return launched(what, e);
    }
  }
  return CMOE_OK;
}
