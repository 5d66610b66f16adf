// The norm of a list of tensors together, and the tensors scaled so that it is at most a given one:
//   n = sqrt(sum over all tensors of v^2),  c = min(1, max_norm / (n + eps)), 1 where n + eps is 0,  out = c v
// Squares and sums are fp64: a bf16 or fp32 gradient's square neither overflows nor vanishes there, and the vector units do a
// conversion and an fp64 multiply-add per element in a fraction of the time that memory takes for it.  Every workgroup sums one run of one
// tensor and leaves the sum at its own place; in the second launch every workgroup adds all places in the same order.  No
// atomics, so the same tensors give the same bits.  Bound by memory: 1.08 G elements in bf16, 2.2 GB, are read in 415 us (5.2 TB/s) and read and written
// in 845 (5.1); small lists by the host, 0.45 to 0.7 us a tensor, with kernels of 3 and 5 us.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <vector>

#include "../../include/cmoe.h"
#include "cmoe_internal.h"
#include "dropout_device.h"
#include "operator_args.h"

namespace cmoe {
namespace {

constexpr int PER_LAUNCH = 120;            // tensors whose description fits a launch's arguments (4 KB)
constexpr int64_t RUN = 16384;             // elements of a workgroup's shortest run
constexpr int64_t RUNS = 2048;             // about how many workgroups share a long list

struct Listed {
  const void* g;
  void* out;
  int64_t n;                               // negative: ~n elements of fp32
  uint32_t first;                          // its first workgroup, of this launch
  uint32_t unused;
};
struct List {
  Listed t[PER_LAUNCH];
  int64_t run;
  int32_t count;
  uint32_t groups;                         // workgroups of this launch
  uint32_t place;                          // of the first one's sum
  uint32_t places;                         // of all launches
};
static_assert(sizeof(List) <= 4000, "kernel arguments");

// The tensor of a workgroup: the last one that begins at or before it.
__device__ __forceinline__ int listed_of(const List& list, uint32_t group) {
  int lo = 0, hi = list.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (list.t[mid].first <= group) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ double add_all(double v, double* shared) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
  __syncthreads();
  return shared[0] + shared[1] + shared[2] + shared[3];
}

template <typename T>
__device__ __forceinline__ double squares(const T* g, int64_t n) {
  double sum = 0.0;
  constexpr int AHEAD = 4;
  int64_t at = (int64_t)threadIdx.x * 8;
  for (; at + (AHEAD - 1) * 2048 + 8 <= n; at += AHEAD * 2048) {
    float v[AHEAD][8];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) load8(g + at + a * 2048, 8, v[a]);
#pragma unroll
    for (int a = 0; a < AHEAD; ++a)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fma((double)v[a][e], (double)v[a][e], sum);
  }
  for (; at < n; at += 2048) {
    float v[8];
    load8(g + at, (int)(n - at < 8 ? n - at : 8), v);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fma((double)v[e], (double)v[e], sum);
  }
  return sum;
}

__global__ __launch_bounds__(256) void clip_squares(List list, double* places) {
  __shared__ double shared[4];
  const Listed& t = list.t[listed_of(list, blockIdx.x)];
  const int64_t n = t.n < 0 ? ~t.n : t.n, from = (int64_t)(blockIdx.x - t.first) * list.run;
  const int64_t mine = min(list.run, n - from);
  const double sum = t.n < 0 ? squares(static_cast<const float*>(t.g) + from, mine) : squares(static_cast<const bf16_t*>(t.g) + from, mine);
  const double all = add_all(sum, shared);
  if (threadIdx.x == 0) places[list.place + blockIdx.x] = all;
}

template <typename T>
__device__ __forceinline__ void scale_run(const T* g, T* out, int64_t n, float pre, float c) {
  constexpr int AHEAD = 4;
  int64_t at = (int64_t)threadIdx.x * 8;
  for (; at + (AHEAD - 1) * 2048 + 8 <= n; at += AHEAD * 2048) {
    float v[AHEAD][8];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) load8(g + at + a * 2048, 8, v[a]);
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[a][e] = v[a][e] * pre * c;
      store8(out + at + a * 2048, 8, v[a]);
    }
  }
  for (; at < n; at += 2048) {
    float v[8];
    const int left = (int)(n - at < 8 ? n - at : 8);
    load8(g + at, left, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = v[e] * pre * c;
    store8(out + at, left, v);
  }
}

__global__ __launch_bounds__(256) void clip_scale(List list, const double* places, float max_norm, float eps, float* norm) {
  __shared__ double shared[4];
  double sum = 0.0;
  for (uint32_t i = threadIdx.x; i < list.places; i += 256) sum += places[i];
  const double n = sqrt(add_all(sum, shared));
  if (list.place == 0 && blockIdx.x == 0 && threadIdx.x == 0) norm[0] = (float)n;
  const double over = n + (double)eps;
  const double ratio = over == 0.0 ? 1.0 : (double)max_norm / over;        // (zeros stay zeros, whatever the limit)
  // a norm that is no number makes every gradient none; without a limit nothing is looked at
  // A factor near fp32's smallest numbers or below them would have few bits left: 2^-64 of it goes to the gradient first, exactly (what falls
  // below the normal numbers there, under 2^-62, would come to less than 2^-162, and that is zero).
  const float pre = ratio < 0x1p-100 ? 0x1p-64f : 1.0f;
  const float c = max_norm == INFINITY || ratio >= 1.0 ? 1.0f : (float)(ratio / (double)pre);
  // (from the list's end on: what the first launch read last may still be in a cache)
  const uint32_t group = list.groups - 1 - blockIdx.x;
  const Listed& t = list.t[listed_of(list, group)];
  if (c == 1.0f && t.out == t.g) return;
  const int64_t count = t.n < 0 ? ~t.n : t.n, from = (int64_t)(group - t.first) * list.run;
  const int64_t mine = min(list.run, count - from);
  if (t.n < 0) scale_run(static_cast<const float*>(t.g) + from, static_cast<float*>(t.out) + from, mine, pre, c);
  else scale_run(static_cast<const bf16_t*>(t.g) + from, static_cast<bf16_t*>(t.out) + from, mine, pre, c);
}

__global__ void clip_nothing(float* norm) { norm[0] = 0.0f; }

// Elements of a run, and all runs; -1: a tensor's size or type is not one, -2: too many.
int64_t runs_of(const cmoe_gradient* list, int32_t count, int64_t* run) {
  int64_t total = 0;
  for (int i = 0; i < count; ++i) {
    if (list[i].elements < 0 || list[i].elements > ((int64_t)1 << 40) || (list[i].dtype != CMOE_F32 && list[i].dtype != CMOE_BF16)) return -1;
    total += list[i].elements;
    if (total > ((int64_t)1 << 44)) return -2;
  }
  *run = std::max(RUN, (total / RUNS + RUN - 1) / RUN * RUN);
  int64_t runs = 0;
  for (int i = 0; i < count; ++i) runs += (list[i].elements + *run - 1) / *run;
  return runs;
}

}  // namespace
}  // namespace cmoe

extern "C" size_t cmoe_clip_gradients_workspace_bytes(const cmoe_gradient* list, int32_t count) {
  int64_t run;
  const int64_t runs = list && count > 0 && count <= 65536 ? cmoe::runs_of(list, count, &run) : 0;
  return runs > 0 ? (size_t)runs * sizeof(double) : 0;
}

extern "C" int cmoe_clip_gradients(const cmoe_gradient* list, int32_t count, float max_norm, float eps, float* norm, void* workspace, size_t workspace_bytes,
                                   void* hip_stream) {
  using namespace cmoe;
  const char* what = "cmoe_clip_gradients";
  if (count < 0 || count > 65536 || (count > 0 && !list)) return fail(CMOE_EINVAL, "%s: need a list of 0 to 65536 tensors", what);
  if (!(max_norm >= 0.0f) || !(eps >= 0.0f) || !std::isfinite(eps)) return fail(CMOE_EINVAL, "%s: max_norm and eps must not be negative, eps finite", what);
  if (!norm || (uintptr_t)norm % 4 != 0) return fail(CMOE_EINVAL, "%s: norm is null or not aligned to 4 bytes", what);
  int64_t run = RUN;
  const int64_t runs = runs_of(list, count, &run);
  if (runs < 0) return fail(CMOE_EINVAL, "%s: a tensor's size or dtype is not one, or there are too many elements", what);
  if (runs > 0 && (!workspace || (uintptr_t)workspace % 8 != 0 || workspace_bytes < (size_t)runs * sizeof(double)))
    return fail(CMOE_EINVAL, "%s: the workspace is null, not aligned to 8 bytes or has less than %lld bytes", what, (long long)(runs * sizeof(double)));
  // Outputs overlap nothing but, in place, their own tensor.  In the order of the addresses, whoever overlaps somebody overlaps the one that
  // reaches furthest before it.
  struct Span {
    uint64_t from, to;
    bool written;
  };
  try {
    std::vector<Span> spans;
    spans.reserve(2 * (size_t)count + 2);
    for (int i = 0; i < count; ++i) {
      const cmoe_gradient& t = list[i];
      if (t.elements == 0) continue;
      const uint64_t es = elem_size(t.dtype), bytes = t.elements * es, g = (uint64_t)(uintptr_t)t.g, out = (uint64_t)(uintptr_t)t.out;
      if (!t.g || !t.out || g % es || out % es) return fail(CMOE_EINVAL, "%s: tensor %d is null or not aligned", what, i);
      spans.push_back({out, out + bytes, true});
      if (out != g) spans.push_back({g, g + bytes, false});
    }
    spans.push_back({(uint64_t)(uintptr_t)norm, (uint64_t)(uintptr_t)norm + 4, true});
    if (runs > 0) spans.push_back({(uint64_t)(uintptr_t)workspace, (uint64_t)(uintptr_t)workspace + runs * 8, true});
    std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.from < b.from; });
    uint64_t read_to = 0, written_to = 0;
    for (const Span& q : spans) {
      if (q.from < written_to || (q.written && q.from < read_to)) return fail(CMOE_EINVAL, "%s: an output overlaps another tensor", what);
      (q.written ? written_to : read_to) = std::max(q.written ? written_to : read_to, q.to);
    }
  } catch (const std::exception&) {
    return fail(CMOE_ENOMEM, "%s: no host memory", what);
  }
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (runs == 0) {
    hipLaunchKernelGGL(clip_nothing, dim3(1), dim3(1), 0, s, norm);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CMOE_OK : fail(CMOE_EHIP, "%s: %s", what, hipGetErrorString(e));
  }
  double* places = static_cast<double*>(workspace);
  for (int pass = 0; pass < 2; ++pass) {
    List l = {};
    l.run = run;
    l.places = (uint32_t)runs;
    auto launch = [&]() {
      if (l.count == 0) return hipSuccess;
      if (pass == 0) hipLaunchKernelGGL(clip_squares, dim3(l.groups), dim3(256), 0, s, l, places);
      else hipLaunchKernelGGL(clip_scale, dim3(l.groups), dim3(256), 0, s, l, places, max_norm, eps, norm);
      l.place += l.groups;
      l.groups = 0;
      l.count = 0;
      return hipGetLastError();
    };
    for (int i = 0; i < count; ++i) {
      if (list[i].elements == 0) continue;
      Listed& t = l.t[l.count++];
      t.g = list[i].g;
      t.out = list[i].out;
      t.n = list[i].dtype == CMOE_F32 ? ~list[i].elements : list[i].elements;
      t.first = l.groups;
      l.groups += (uint32_t)((list[i].elements + run - 1) / run);
      if (l.count == PER_LAUNCH)
        if (hipError_t e = launch()) return fail(CMOE_EHIP, "%s: %s", what, hipGetErrorString(e));
    }
    if (hipError_t e = launch()) return fail(CMOE_EHIP, "%s: %s", what, hipGetErrorString(e));
  }
  return CMOE_OK;
}
