// Low-rank adapters of many requests beside a shared projection, forward and backward.  Token t has adapter k = ids[t]:
//   u = A_k drop(x)                     [rank], fp32
//   y = base + scale_k * B_k u
//   v = scale_k * B_k^T dy              [rank], fp32
//   dx = dx_base + drop's mask and scale on A_k^T v
//   dA_k = sum over its tokens of v drop(x)^T,   dB_k = scale_k * sum over its tokens of dy u^T
#include <hip/hip_runtime.h>
#include <algorithm>

#include "../../include/cmoe.h"
#include "cmoe_internal.h"
#include "dropout_device.h"
#include "operator_args.h"

namespace cmoe {

constexpr int MAX_RANK = 64;

// The adapter of a token, or -1.
__device__ __forceinline__ int adapter_of(const int32_t* ids, int64_t t, int n_adapters) {
  const int k = ids ? ids[t] : 0;
  return k >= 0 && k < n_adapters ? k : -1;
}

// u[t][j] = scale * sum over i of drop(x[t][i]) w_k[j][i], w_k [rank][d] or, TRANSPOSED, [d][rank]: a wave per element.
template <typename T, bool TRANSPOSED>
__global__ __launch_bounds__(256) void contract_kernel(const T* x, const T* w, const float* scale, const int32_t* ids, float* u, int64_t tokens, int d,
                                                       int rank, int n_adapters, Drop drop) {
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int64_t t = unit / rank;
  const int j = (int)(unit % rank);
  if (t >= tokens) return;
  const int k = adapter_of(ids, t, n_adapters);
  float sum = 0.0f;
  if (k >= 0) {
    const int per_row = (d + 7) >> 3;
    for (int c = lane; c < per_row; c += 64) {
      const int n = d - c * 8;
      float v[8], m[8];
      load8(x + t * d + c * 8, n, v);
      if (drop.limit) drop8(v, drop, (uint64_t)t * per_row + c);
      if (!TRANSPOSED) load8(w + ((int64_t)k * rank + j) * d + c * 8, n, m);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (TRANSPOSED) m[e] = e < n ? Elem<T>::ld(w + ((int64_t)k * d + c * 8 + e) * rank + j) : 0.0f;
        sum += v[e] * m[e];
      }
    }
    sum = wave_sum(sum);
    if (scale) sum *= scale[k];
  }
  if (lane == 0) u[t * rank + j] = sum;
}

// y[t][o] = base[t][o] + drop(scale * sum over j of u[t][j] w_k[o][j]): a thread per eight outputs.
template <typename T, bool TRANSPOSED>
__global__ __launch_bounds__(256) void expand_kernel(const float* u, const T* w, const float* scale, const int32_t* ids, const T* base, T* y,
                                                     int64_t tokens, int d, int rank, int n_adapters, Drop drop) {
  const int per_row = (d + 7) >> 3;
  const int64_t unit = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t t = unit / per_row;
  const int c = (int)(unit % per_row), n = d - c * 8;
  if (t >= tokens) return;
  const int k = adapter_of(ids, t, n_adapters);
  float v[8], o[8] = {};
  if (k >= 0) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (e >= n) continue;
      for (int j = 0; j < rank; ++j)
        o[e] += u[t * rank + j] * Elem<T>::ld(w + (TRANSPOSED ? ((int64_t)k * rank + j) * d + c * 8 + e : ((int64_t)k * d + c * 8 + e) * rank + j));
      if (scale) o[e] *= scale[k];
    }
    if (drop.limit) drop8(o, drop, (uint64_t)t * per_row + c);
  }
  if (base) {
    load8(base + t * d + c * 8, n, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] += v[e];
  }
  store8(y + t * d + c * 8, n, o);
}

// g_k[j][i] (TRANSPOSED: [i][j]) = scale * sum over the adapter's tokens of u[t][j] drop(x[t][i]): a thread per element.
template <typename T, bool TRANSPOSED>
__global__ __launch_bounds__(256) void outer_kernel(const float* u, const T* x, const float* scale, const int32_t* ids, float* g, int64_t tokens,
                                                    int d, int rank, int n_adapters, Drop drop) {
  const int i = blockIdx.x * 256 + threadIdx.x, j = blockIdx.y, k = blockIdx.z;
  if (i >= d) return;
  const int per_row = (d + 7) >> 3;
  float sum = 0.0f;
  bool any = false;                               // (an adapter without tokens: 0, whatever its scale)
  for (int64_t t = 0; t < tokens; ++t) {
    if (adapter_of(ids, t, n_adapters) != k) continue;
    any = true;
    float v = Elem<T>::ld(x + t * d + i);
    if (drop.limit) v = drop_keeps(drop, philox_words(drop, (uint64_t)t * per_row + (i >> 3)), i & 7) ? v * drop.scale : 0.0f;
    sum += u[t * rank + j] * v;
  }
  if (scale && any) sum *= scale[k];
  g[TRANSPOSED ? ((int64_t)k * d + i) * rank + j : ((int64_t)k * rank + j) * d + i] = sum;
}

template <typename T>
static void launch_adapters_forward(const cmoe_adapters_forward_args& p, const Drop& drop, hipStream_t s) {
  float* u = p.u ? p.u : (float*)p.workspace;
  const unsigned units = (unsigned)((p.tokens * p.rank + 3) / 4);
  hipLaunchKernelGGL((contract_kernel<T, false>), dim3(units), dim3(256), 0, s, (const T*)p.x, (const T*)p.a, (const float*)nullptr, p.ids, u, p.tokens,
                     p.d_in, p.rank, p.n_adapters, drop);
  const unsigned blocks = (unsigned)((p.tokens * ((p.d_out + 7) / 8) + 255) / 256);
  hipLaunchKernelGGL((expand_kernel<T, false>), dim3(blocks), dim3(256), 0, s, u, (const T*)p.b, p.scale, p.ids, (const T*)p.base, (T*)p.y, p.tokens,
                     p.d_out, p.rank, p.n_adapters, Drop{});
}

template <typename T>
static void launch_adapters_backward(const cmoe_adapters_backward_args& p, const Drop& drop, hipStream_t s) {
  float* v = (float*)p.workspace;
  if (p.tokens > 0 && (p.dx || p.da)) {
    const unsigned units = (unsigned)((p.tokens * p.rank + 3) / 4);
    hipLaunchKernelGGL((contract_kernel<T, true>), dim3(units), dim3(256), 0, s, (const T*)p.dy, (const T*)p.b, p.scale, p.ids, v, p.tokens, p.d_out,
                       p.rank, p.n_adapters, Drop{});
  }
  if (p.tokens > 0 && p.dx) {
    const unsigned blocks = (unsigned)((p.tokens * ((p.d_in + 7) / 8) + 255) / 256);
    hipLaunchKernelGGL((expand_kernel<T, true>), dim3(blocks), dim3(256), 0, s, v, (const T*)p.a, (const float*)nullptr, p.ids, (const T*)p.dx_base,
                       (T*)p.dx, p.tokens, p.d_in, p.rank, p.n_adapters, drop);
  }
  if (p.da)
    hipLaunchKernelGGL((outer_kernel<T, false>), dim3((p.d_in + 255) / 256, p.rank, p.n_adapters), dim3(256), 0, s, v, (const T*)p.x, (const float*)nullptr,
                       p.ids, p.da, p.tokens, p.d_in, p.rank, p.n_adapters, drop);
  if (p.db)
    hipLaunchKernelGGL((outer_kernel<T, true>), dim3((p.d_out + 255) / 256, p.rank, p.n_adapters), dim3(256), 0, s, p.u, (const T*)p.dy, p.scale, p.ids,
                       p.db, p.tokens, p.d_out, p.rank, p.n_adapters, Drop{});
}

static int check_adapters(const char* what, int dtype, int64_t tokens, int d_in, int d_out, int rank, int n_adapters) {
  if (dtype != CMOE_F32 && dtype != CMOE_BF16) return fail(CMOE_EINVAL, "%s: dtype must be CMOE_F32 or CMOE_BF16", what);
  if (d_in < 1 || d_out < 1 || d_in > (1 << 24) || d_out > (1 << 24)) return fail(CMOE_EINVAL, "%s: d_in and d_out must be 1 to 2^24", what);
  if (rank < 1 || rank > MAX_RANK) return fail(CMOE_EINVAL, "%s: rank must be 1 to %d", what, MAX_RANK);
  if (n_adapters < 1 || n_adapters > 65535) return fail(CMOE_EINVAL, "%s: n_adapters must be 1 to 65535", what);
  if (tokens < 0 || tokens > (1 << 20)) return fail(CMOE_EINVAL, "%s: tokens must be 0 to 2^20", what);
  return CMOE_OK;
}

}  // namespace cmoe

extern "C" size_t cmoe_adapters_forward_workspace_bytes(int64_t tokens, int32_t d_in, int32_t d_out, int32_t rank, int32_t n_adapters, int32_t dtype) {
  using namespace cmoe;
  if (check_adapters("cmoe_adapters_forward_workspace_bytes", dtype, tokens, d_in, d_out, rank, n_adapters)) return 0;
  return (size_t)tokens * rank * sizeof(float);
}

extern "C" int cmoe_adapters_forward(const cmoe_adapters_forward_args* p, void* hip_stream) {
  using namespace cmoe;
  const char* what = "cmoe_adapters_forward";
  if (!p || p->struct_bytes != sizeof(*p)) return fail(CMOE_EINVAL, "%s: the arguments are null or of another version", what);
  if (int rc = check_adapters(what, p->dtype, p->tokens, p->d_in, p->d_out, p->rank, p->n_adapters)) return rc;
  Drop drop;
  if (int rc = make_drop(what, p->p, p->seed, p->offset, &drop)) return rc;
  if (p->tokens == 0) return CMOE_OK;
  if (!p->x || !p->y || !p->a || !p->b || !p->scale) return fail(CMOE_EINVAL, "%s: x, a, b, scale or y is null", what);
  if (!p->u && (!p->workspace || p->workspace_bytes < cmoe_adapters_forward_workspace_bytes(p->tokens, p->d_in, p->d_out, p->rank, p->n_adapters, p->dtype)))
    return fail(CMOE_EINVAL, "%s: the workspace is missing or too small", what);
  const size_t es = elem_size(p->dtype);
  const uint64_t t = p->tokens, in = t * p->d_in * es, out = t * p->d_out * es, n = p->n_adapters;
  const Operand y{"y", p->y, out, es};
  if (int rc = check_operands(what, {{"base", p->base, out, es}}, {y}, true)) return rc;
  if (int rc = check_operands(what, {{"x", p->x, in, es}, {"a", p->a, n * p->rank * p->d_in * es, es}, {"b", p->b, n * p->d_out * p->rank * es, es},
                                     {"scale", p->scale, n * 4, 4}, {"ids", p->ids, t * 4, 4}},
                              {y, {"u", p->u, t * p->rank * 4, 4}, {"workspace", p->workspace, p->workspace_bytes, 16}}, false))
    return rc;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  p->dtype == CMOE_BF16 ? launch_adapters_forward<bf16_t>(*p, drop, s) : launch_adapters_forward<float>(*p, drop, s);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CMOE_OK : fail(CMOE_EHIP, "%s: %s", what, hipGetErrorString(e));
}

extern "C" size_t cmoe_adapters_backward_workspace_bytes(int64_t tokens, int32_t d_in, int32_t d_out, int32_t rank, int32_t n_adapters, int32_t dtype) {
  using namespace cmoe;
  if (check_adapters("cmoe_adapters_backward_workspace_bytes", dtype, tokens, d_in, d_out, rank, n_adapters)) return 0;
  return (size_t)tokens * rank * sizeof(float);
}

extern "C" int cmoe_adapters_backward(const cmoe_adapters_backward_args* p, void* hip_stream) {
  using namespace cmoe;
  const char* what = "cmoe_adapters_backward";
  if (!p || p->struct_bytes != sizeof(*p)) return fail(CMOE_EINVAL, "%s: the arguments are null or of another version", what);
  if (int rc = check_adapters(what, p->dtype, p->tokens, p->d_in, p->d_out, p->rank, p->n_adapters)) return rc;
  Drop drop;
  if (int rc = make_drop(what, p->p, p->seed, p->offset, &drop)) return rc;
  if (p->tokens > 0 && (!p->dy || !p->a || !p->b || !p->scale)) return fail(CMOE_EINVAL, "%s: dy, a, b or scale is null", what);
  if (p->tokens > 0 && ((p->da && !p->x) || (p->db && !p->u))) return fail(CMOE_EINVAL, "%s: da needs x, db needs u", what);
  if (p->tokens > 0 && (!p->workspace || p->workspace_bytes < cmoe_adapters_backward_workspace_bytes(p->tokens, p->d_in, p->d_out, p->rank, p->n_adapters, p->dtype)))
    return fail(CMOE_EINVAL, "%s: the workspace is missing or too small", what);
  const size_t es = elem_size(p->dtype);
  const uint64_t t = p->tokens, in = t * p->d_in * es, out = t * p->d_out * es, n = p->n_adapters, wa = n * p->rank * p->d_in, wb = n * p->d_out * p->rank;
  const Operand dx{"dx", p->dx, in, es};
  if (int rc = check_operands(what, {{"dx_base", p->dx_base, in, es}}, {dx}, true)) return rc;
  if (int rc = check_operands(what, {{"dy", p->dy, out, es}, {"x", p->x, in, es}, {"u", p->u, t * p->rank * 4, 4}, {"a", p->a, wa * es, es}, {"b", p->b, wb * es, es},
                                     {"scale", p->scale, n * 4, 4}, {"ids", p->ids, t * 4, 4}},
                              {dx, {"da", p->da, wa * 4, 4}, {"db", p->db, wb * 4, 4}, {"workspace", p->workspace, p->workspace_bytes, 16}}, false))
    return rc;
  if (p->tokens == 0 && !p->da && !p->db) return CMOE_OK;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  p->dtype == CMOE_BF16 ? launch_adapters_backward<bf16_t>(*p, drop, s) : launch_adapters_backward<float>(*p, drop, s);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CMOE_OK : fail(CMOE_EHIP, "%s: %s", what, hipGetErrorString(e));
}
