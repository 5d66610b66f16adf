// Layer norm and its root-mean-square form, with the dropout and the residual addition in front of it, forward and backward.
//   s = drop(x) + residual            rounded to the batch's type where it is stored, and normalised as stored
//   y = (s - mean) * rstd * w + bias  rstd = 1 / sqrt(mean((s - mean)^2) + eps); the rms form has mean = 0
// Backward, with g = dy * w and h = (s - mean) * rstd:
//   ds = rstd * (g - mean(g) - h * mean(g * h)) + dsum     (the rms form has no mean(g))
//   dresidual = ds,  dx = drop's mask and scale on ds,  dw = sum over rows of dy * h,  dbias = sum over rows of dy
// Statistics, sums and gradients of the weights are fp32; the mask is computed again from its counters.
#include <hip/hip_runtime.h>
#include <cmath>

#include "../../include/cmoe.h"
#include "cmoe_internal.h"
#include "fragments_device.h"
#include "operator_args.h"

namespace cmoe {

constexpr int NORM_MAX_COLS = 32768;

// Sums over the 16 lanes of a row, or over a wave, in every lane: additions in DPP operands, no trip through LDS.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float dpp_f32(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float row16_sum(float v) {
  v += dpp_f32<0x128>(v);      // rotations by 8, 4, 2, 1
  v += dpp_f32<0x124>(v);
  v += dpp_f32<0x122>(v);
  v += dpp_f32<0x121>(v);
  return v;
}
__device__ __forceinline__ float wave64_sum(float v) {
  v = row16_sum(v);
  v += dpp_f32<0x142, 0xa>(v);      // last lane of rows 0, 2 into rows 1, 3
  v += dpp_f32<0x143, 0xc>(v);      // ... of row 1 into rows 2, 3
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// N sums over the LANES threads that share a row, in all of them.  More than a wave: through `part`, which the caller has to
// alternate between two buffers, since one barrier lies between writing and reading and none after.
template <int LANES, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*part)[16]) {
  if constexpr (LANES == 16) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = row16_sum(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave64_sum(v[i]);
    if constexpr (LANES > 64) {
      const int wave = threadIdx.x >> 6, first = threadIdx.x / LANES * (LANES / 64);
      if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) part[i][wave] = v[i];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) {
        v[i] = part[i][first];
#pragma unroll
        for (int w = 1; w < LANES / 64; ++w) v[i] += part[i][first + w];
      }
    }
  }
}

template <typename T>
struct NormForward {
  const T* x;
  const T* residual;      // or null
  T* sum;                 // or null
  T* y;
  const T* w;             // or null: 1
  const T* bias;          // or null: 0
  float* mean;            // or null
  float* rstd;            // or null
  int64_t rows;
  int cols;
  float eps;
  Drop drop;
};

// A row of LANES threads; a thread holds CH chunks of eight elements, LANES chunks apart, in registers from the one time they
// are read to the one time they are written: the variance is taken around the mean without a second pass over memory.  Bound by memory:
// 8192 rows of 4096 with a residual, bf16, 268 MB in 51 us (5.3 TB/s; a copy of that size 5.4).  A single row is a chain of latencies
// (3.4 us), behind 3 us of the launch on the host and 3.5 us of the binding.
template <typename T, int LANES, int CH, bool LAYER>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void norm_forward_kernel(NormForward<T> a) {
  constexpr int ROWS = LANES >= 256 ? 1 : 256 / LANES;
  __shared__ float part[2][1][16];
  const int lane = threadIdx.x % LANES;
  const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
  if (row >= a.rows) return;                      // (rows that share a workgroup need no barrier)
  const int per_row = (a.cols + 7) >> 3;
  const int64_t base = row * a.cols;
  float v[CH][8];
  float total[1] = {0.0f};
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = i * LANES + lane;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] = 0.0f;
    if (c < per_row) {
      const int n = a.cols - c * 8;
      load8(a.x + base + c * 8, n, v[i]);
      float r[8];
      if (a.residual) load8(a.residual + base + c * 8, n, r);
      if (a.drop.limit) drop8(v[i], a.drop, (uint64_t)row * per_row + c);
      if (a.residual) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] += r[e];
      }
      if (a.sum) {
        store8(a.sum + base + c * 8, n, v[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = as_stored<T>(v[i][e]);
      }
    }
    if (LAYER) {
#pragma unroll
      for (int e = 0; e < 8; ++e) total[0] += v[i][e];
    }
  }
  const float inv_cols = 1.0f / a.cols;
  float mean = 0.0f;
  if (LAYER) {
    row_sums<LANES>(total, part[0]);
    mean = total[0] * inv_cols;
  }
  float sq[1] = {0.0f};
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = i * LANES + lane;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[i][e] -= mean;
      sq[0] += c * 8 + e < a.cols ? v[i][e] * v[i][e] : 0.0f;
    }
  }
  row_sums<LANES>(sq, part[1]);
  const float rstd = 1.0f / sqrtf(sq[0] * inv_cols + a.eps);
  if (lane == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = i * LANES + lane;
    if (c >= per_row) continue;
    const int n = a.cols - c * 8;
    float w[8], b[8];
    if (a.w) load8(a.w + c * 8, n, w);
    if (a.bias) load8(a.bias + c * 8, n, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float h = v[i][e] * rstd;
      v[i][e] = (a.w ? h * w[e] : h) + (a.bias ? b[e] : 0.0f);
    }
    store8(a.y + base + c * 8, n, v[i]);
  }
}

template <typename T>
struct NormBackward {
  const T* dy;
  const T* s;
  const T* dsum;          // or null
  const T* w;             // or null: 1
  const float* mean;      // or null: 0
  const float* rstd;
  T* dx;
  T* dresidual;           // or null
  float* partials;        // [workgroup][dw, dbias][cols], or null
  int64_t rows;
  int cols;
  int sums;               // 1: dw alone, 2: dbias too
  Drop drop;
};

// Rows of a workgroup; the threads of a row are LANES, those of a workgroup 256 at least.
template <int LANES>
constexpr int BACKWARD_ROWS = LANES >= 256 ? 1 : 256 / LANES;

// A workgroup takes every grid'th set of rows and keeps its share of the sums over rows in registers, in the same columns for every row,
// so the sums over rows cost one row of partial sums per workgroup.  All that a row reads is loaded while the row before it is worked
// on: a row has a reduction in its middle, which nothing else would cover (4096 rows of 4096, bf16, all operands: 59 -> 32 us, 168 MB at
// 5.3 TB/s).  Beyond 8192 columns a workgroup of 1024 threads has more than one chunk per thread and 128 registers for each: nothing is loaded
// ahead, the weights are read for every row, and what does not fit is spilled (two chunks: 3 to 30 registers; four: 142 to 195).  All
// operands: bf16 2048 x 8192 without spills 168 MB in 38 us; of 336 MB each (62 us at 5.4 TB/s) bf16 2048 x 16384 102, 1024 x 32768 279, fp32
// 1024 x 16384 90, 512 x 32768 202.
template <typename T, int LANES, int CH, bool LAYER, int EDGE>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void norm_backward_kernel(NormBackward<T> a) {
  constexpr int ROWS = BACKWARD_ROWS<LANES>;
  constexpr bool AHEAD = CH == 1;
  __shared__ float part[2][2][16];
  __shared__ float joined[ROWS > 1 ? 2 : 1][ROWS > 1 ? 2048 : 1];
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  const int per_row = (a.cols + 7) >> 3;
  const int64_t size = a.rows * a.cols;
  const float inv_cols = 1.0f / a.cols;
  float dw[CH][8], db[CH][8], w[8];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[i][e] = db[i][e] = 0.0f;
  }
  auto load_weight = [&](int i) {
    const int c = (i * LANES + lane) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = 1.0f;
    if (a.w) unpack(load_at<EDGE>(a.w, c, a.cols - c, a.cols), w);
  };
  if (AHEAD) load_weight(0);
  Frag<T> dy[CH], s[CH], dsum[CH];
  float mean = 0.0f, rstd = 0.0f;
  auto load = [&](int64_t row) {
    row = min(row, a.rows - 1);
    if (LAYER) mean = a.mean[row];
    rstd = a.rstd[row];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = (i * LANES + lane) * 8, n = a.cols - c;
      dy[i] = load_at<EDGE>(a.dy, row * a.cols + c, n, size);
      s[i] = load_at<EDGE>(a.s, row * a.cols + c, n, size);
      if (a.dsum) dsum[i] = load_at<EDGE>(a.dsum, row * a.cols + c, n, size);
    }
  };
  int buffer = 0;
  int64_t row0 = (int64_t)blockIdx.x * ROWS;
  if (AHEAD) load(row0 + group);
  for (; row0 < a.rows; row0 += (int64_t)gridDim.x * ROWS, buffer ^= 1) {
    const int64_t row = row0 + group;
    const bool valid = row < a.rows;
    if (!AHEAD) load(row);
    const float r = rstd;
    float g[CH][8], h[CH][8], t[2] = {0.0f, 0.0f};
    Frag<T> past[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int n = valid ? a.cols - (i * LANES + lane) * 8 : 0;
      keep_first(dy[i], n);
      keep_first(s[i], n);
      unpack(dy[i], g[i]);
      unpack(s[i], h[i]);
      past[i] = dsum[i];
      if (!AHEAD) load_weight(i);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        h[i][e] = (h[i][e] - mean) * r;
        dw[i][e] += g[i][e] * h[i][e];
        db[i][e] += g[i][e];
        g[i][e] *= w[e];
        t[0] += g[i][e] * h[i][e];
        t[1] += g[i][e];
      }
    }
    if (AHEAD) load(row0 + (int64_t)gridDim.x * ROWS + group);
    row_sums<LANES>(t, part[buffer]);
    const float mgh = t[0] * inv_cols, mg = LAYER ? t[1] * inv_cols : 0.0f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = i * LANES + lane, n = a.cols - c * 8;
      float o[8], past_f[8];
      unpack(past[i], past_f);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        o[e] = (g[i][e] - mg - h[i][e] * mgh) * r;
        if (a.dsum) o[e] += past_f[e];
      }
      if (!valid || n <= 0) continue;
      const int64_t at = row * a.cols + c * 8;
      if (a.dresidual) store_at<EDGE>(a.dresidual + at, n, o);
      if (a.drop.limit) drop8(o, a.drop, (uint64_t)row * per_row + c);
      store_at<EDGE>(a.dx + at, n, o);
    }
  }
  if (!a.partials) return;
  float* p = a.partials + (int64_t)blockIdx.x * a.sums * a.cols;
  if constexpr (ROWS > 1) {
    // the groups' sums, added in their order by the first
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      joined[0][(group * LANES + lane) * 8 + e] = dw[0][e];
      joined[1][(group * LANES + lane) * 8 + e] = db[0][e];
    }
    __syncthreads();
    if (group > 0) return;
    for (int k = 1; k < ROWS; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dw[0][e] += joined[0][(k * LANES + lane) * 8 + e];
        db[0][e] += joined[1][(k * LANES + lane) * 8 + e];
      }
  }
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = (i * LANES + lane) * 8;
    store_at<RAGGED>(p + c, a.cols - c, dw[i]);
    if (a.sums == 2) store_at<RAGGED>(p + a.cols + c, a.cols - c, db[i]);
  }
}

// out[c] = the sum of n rows of partial sums, in a fixed order: 64 columns per workgroup, each wave a sixteenth of the rows (512 rows of
// two times 4096 columns 4.8 us; by four waves 7.1).
__global__ __launch_bounds__(1024) void sum_rows_kernel(const float* __restrict__ partials, int n, int cols, int sums, float* dw, float* dbias) {
  __shared__ float part[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int which = blockIdx.y;
  const int c = blockIdx.x * 64 + lane;
  const int per = (n + 15) / 16, first = wave * per, last = min(n, first + per);
  float t = 0.0f;
  if (c < cols) {
    const float* p = partials + (int64_t)which * cols + c;
#pragma unroll 8
    for (int r = first; r < last; ++r) t += p[(int64_t)r * sums * cols];
  }
  part[wave][lane] = t;
  __syncthreads();
  if (wave > 0 || c >= cols) return;
  for (int k = 1; k < 16; ++k) t += part[k][lane];
  (which ? dbias : dw)[c] = t;
}

// Threads per row and chunks per thread.
struct NormShape { int lanes, chunks; };
static NormShape norm_shape(int cols) {
  const int per_row = (cols + 7) / 8;
  if (per_row <= 16) return {16, 1};
  if (per_row <= 64) return {64, 1};
  if (per_row <= 128) return {64, 2};
  if (per_row <= 256) return {256, 1};
  if (per_row <= 512) return {256, 2};
  if (per_row <= 1024) return {256, 4};
  if (per_row <= 2048) return {1024, 2};
  return {1024, 4};
}

// f(lanes, chunks) with the shape as compile-time constants
template <typename F>
static void with_norm_shape(int cols, F&& f) {
  const NormShape s = norm_shape(cols);
#define CMOE_NORM_SHAPE(L, C) if (s.lanes == L && s.chunks == C) return f(std::integral_constant<int, L>{}, std::integral_constant<int, C>{});
  CMOE_NORM_SHAPE(16, 1)
  CMOE_NORM_SHAPE(64, 1)
  CMOE_NORM_SHAPE(64, 2)
  CMOE_NORM_SHAPE(256, 1)
  CMOE_NORM_SHAPE(256, 2)
  CMOE_NORM_SHAPE(256, 4)
  CMOE_NORM_SHAPE(1024, 2)
  CMOE_NORM_SHAPE(1024, 4)
#undef CMOE_NORM_SHAPE
}

static int rows_per_block(int lanes) { return lanes >= 256 ? 1 : 256 / lanes; }

// The backward pass keeps the columns' sums beside what it loads ahead: one chunk per thread as long as a workgroup has the threads.
static NormShape backward_shape(int cols) {
  const int per_row = (cols + 7) / 8;
  for (const int lanes : {16, 64, 128, 256, 512, 1024})
    if (per_row <= lanes) return {lanes, 1};
  return {1024, per_row <= 2048 ? 2 : 4};
}

// f(lanes, chunks, edge)
template <typename F>
static void with_backward_shape(int cols, F&& f) {
  const NormShape s = backward_shape(cols);
  const auto whole = std::integral_constant<int, WHOLE>{};
  const auto ragged = std::integral_constant<int, RAGGED>{};
  if (cols < 8) return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{}, std::integral_constant<int, TINY>{});
#define CMOE_NORM_SHAPE(L, C) \
  if (s.lanes == L && s.chunks == C) { \
    if (cols % 8 == 0) return f(std::integral_constant<int, L>{}, std::integral_constant<int, C>{}, whole); \
    return f(std::integral_constant<int, L>{}, std::integral_constant<int, C>{}, ragged); \
  }
  CMOE_NORM_SHAPE(16, 1)
  CMOE_NORM_SHAPE(64, 1)
  CMOE_NORM_SHAPE(128, 1)
  CMOE_NORM_SHAPE(256, 1)
  CMOE_NORM_SHAPE(512, 1)
  CMOE_NORM_SHAPE(1024, 1)
  CMOE_NORM_SHAPE(1024, 2)
  CMOE_NORM_SHAPE(1024, 4)
#undef CMOE_NORM_SHAPE
}

// Workgroups of the backward pass: enough to fill the chip, few enough that their partial sums stay small beside the rows.
static int backward_blocks(int64_t rows, int cols) {
  const int per = rows_per_block(backward_shape(cols).lanes);
  return (int)std::min<int64_t>((rows + per - 1) / per, 512);
}

template <typename T>
static void launch_forward(const cmoe_norm_forward_args& p, const Drop& drop, hipStream_t s) {
  const NormForward<T> a{(const T*)p.x, (const T*)p.residual, (T*)p.sum_out, (T*)p.y, (const T*)p.weight, (const T*)p.bias,
                         p.mean, p.rstd, p.rows, p.cols, p.eps, drop};
  with_norm_shape(p.cols, [&](auto lanes, auto chunks) {
    constexpr int L = decltype(lanes)::value, C = decltype(chunks)::value;
    const int per = rows_per_block(L);
    const dim3 grid((unsigned)((p.rows + per - 1) / per)), block(L > 256 ? L : 256);
    if (p.form == CMOE_NORM_LAYER) hipLaunchKernelGGL((norm_forward_kernel<T, L, C, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((norm_forward_kernel<T, L, C, false>), grid, block, 0, s, a);
  });
}

template <typename T>
static void launch_backward(const cmoe_norm_backward_args& p, const Drop& drop, int blocks, hipStream_t s) {
  const NormBackward<T> a{(const T*)p.dy, (const T*)p.s, (const T*)p.dsum, (const T*)p.weight, p.form == CMOE_NORM_LAYER ? p.mean : nullptr, p.rstd,
                          (T*)p.dx, (T*)p.dresidual, p.dweight ? (float*)p.workspace : nullptr, p.rows, p.cols, p.dbias ? 2 : 1, drop};
  with_backward_shape(p.cols, [&](auto lanes, auto chunks, auto edge) {
    constexpr int L = decltype(lanes)::value, C = decltype(chunks)::value, E = decltype(edge)::value;
    const dim3 grid((unsigned)blocks), block(L > 256 ? L : 256);
    if (p.form == CMOE_NORM_LAYER) hipLaunchKernelGGL((norm_backward_kernel<T, L, C, true, E>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((norm_backward_kernel<T, L, C, false, E>), grid, block, 0, s, a);
  });
}

static int check_norm(const char* what, int dtype, int form, int64_t rows, int cols) {
  if (dtype != CMOE_F32 && dtype != CMOE_BF16) return fail(CMOE_EINVAL, "%s: dtype must be CMOE_F32 or CMOE_BF16", what);
  if (form != CMOE_NORM_LAYER && form != CMOE_NORM_RMS) return fail(CMOE_EINVAL, "%s: form must be CMOE_NORM_LAYER or CMOE_NORM_RMS", what);
  if (cols < 1 || cols > NORM_MAX_COLS) return fail(CMOE_EINVAL, "%s: cols must be 1 to %d", what, NORM_MAX_COLS);
  // a launch has fewer than 2^32 threads
  if (rows < 0 || rows > (int64_t)0xfffffc00 / norm_shape(cols).lanes) return fail(CMOE_EINVAL, "%s: rows are negative or too many", what);
  return CMOE_OK;
}

}  // namespace cmoe

extern "C" int cmoe_norm_forward(const cmoe_norm_forward_args* p, void* hip_stream) {
  using namespace cmoe;
  const char* what = "cmoe_norm_forward";
  if (!p || p->struct_bytes != sizeof(*p)) return fail(CMOE_EINVAL, "%s: the arguments are null or of another version", what);
  if (int rc = check_norm(what, p->dtype, p->form, p->rows, p->cols)) return rc;
  if (!(p->eps >= 0.0f) || !std::isfinite(p->eps)) return fail(CMOE_EINVAL, "%s: eps must be finite and not negative", what);
  Drop drop;
  if (int rc = make_drop(what, p->p, p->seed, p->offset, &drop)) return rc;
  if (p->rows == 0) return CMOE_OK;
  if (!p->x || !p->y) return fail(CMOE_EINVAL, "%s: x or y is null", what);
  const size_t es = elem_size(p->dtype);
  const uint64_t batch = (uint64_t)p->rows * p->cols * es, row = (uint64_t)p->cols * es, stat = (uint64_t)p->rows * 4;
  if (int rc = check_operands(what, {{"x", p->x, batch, es, true}, {"residual", p->residual, batch, es, true}, {"weight", p->weight, row, es}, {"bias", p->bias, row, es}},
                              {{"y", p->y, batch, es, true}, {"sum_out", p->sum_out, batch, es, true}, {"mean", p->mean, stat, 4}, {"rstd", p->rstd, stat, 4}}))
    return rc;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  p->dtype == CMOE_BF16 ? launch_forward<bf16_t>(*p, drop, s) : launch_forward<float>(*p, drop, s);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CMOE_OK : fail(CMOE_EHIP, "%s: %s", what, hipGetErrorString(e));
}

extern "C" size_t cmoe_norm_backward_workspace_bytes(int64_t rows, int32_t cols) {
  using namespace cmoe;
  if (rows < 0 || cols < 1 || cols > NORM_MAX_COLS) return 0;
  return (size_t)backward_blocks(rows, cols) * 2 * cols * sizeof(float);
}

extern "C" int cmoe_norm_backward(const cmoe_norm_backward_args* p, void* hip_stream) {
  using namespace cmoe;
  const char* what = "cmoe_norm_backward";
  if (!p || p->struct_bytes != sizeof(*p)) return fail(CMOE_EINVAL, "%s: the arguments are null or of another version", what);
  if (int rc = check_norm(what, p->dtype, p->form, p->rows, p->cols)) return rc;
  Drop drop;
  if (int rc = make_drop(what, p->p, p->seed, p->offset, &drop)) return rc;
  if (p->dbias && !p->dweight) return fail(CMOE_EINVAL, "%s: dbias without dweight", what);
  if (p->rows > 0 && (!p->dy || !p->s || !p->dx || !p->rstd || (p->form == CMOE_NORM_LAYER && !p->mean)))
    return fail(CMOE_EINVAL, "%s: dy, s, dx, rstd or the layer form's mean is null", what);
  const size_t es = elem_size(p->dtype);
  const uint64_t batch = (uint64_t)p->rows * p->cols * es, row = (uint64_t)p->cols * es, stat = (uint64_t)p->rows * 4;
  if (p->dweight && p->rows > 0 && (!p->workspace || p->workspace_bytes < cmoe_norm_backward_workspace_bytes(p->rows, p->cols)))
    return fail(CMOE_EINVAL, "%s: the workspace is missing or too small", what);
  if (int rc = check_operands(what, {{"dy", p->dy, batch, es, true}, {"s", p->s, batch, es, true}, {"dsum", p->dsum, batch, es, true}, {"weight", p->weight, row, es},
                                     {"mean", p->mean, stat, 4}, {"rstd", p->rstd, stat, 4}},
                              {{"dx", p->dx, batch, es, true}, {"dresidual", p->dresidual, batch, es, true}, {"dweight", p->dweight, (uint64_t)p->cols * 4, 4},
                               {"dbias", p->dbias, (uint64_t)p->cols * 4, 4}, {"workspace", p->workspace, p->workspace_bytes, 16}}))
    return rc;
  if (p->rows == 0 && !p->dweight) return CMOE_OK;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int blocks = backward_blocks(p->rows, p->cols);
  if (blocks > 0) p->dtype == CMOE_BF16 ? launch_backward<bf16_t>(*p, drop, blocks, s) : launch_backward<float>(*p, drop, blocks, s);
  if (p->dweight)      // (no rows: the sums are zeros)
    hipLaunchKernelGGL(sum_rows_kernel, dim3((p->cols + 63) / 64, p->dbias ? 2 : 1), dim3(1024), 0, s, (const float*)p->workspace,
                       blocks, p->cols, p->dbias ? 2 : 1, p->dweight, p->dbias);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CMOE_OK : fail(CMOE_EHIP, "%s: %s", what, hipGetErrorString(e));
}
