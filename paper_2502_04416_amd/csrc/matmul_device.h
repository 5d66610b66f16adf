// Kernels of the products in matmul.h.
//
// matmul_any: both types, any alignment and size, operands through registers with every chunk's end checked.
#pragma once
#include <type_traits>

#include "device_utils.h"
#include "dropout_device.h"
#include "gemm_device.h"
#include "matmul.h"

namespace cmoe {

template <typename T> __device__ __forceinline__ float exp_of(float x);
template <> __device__ __forceinline__ float exp_of<float>(float x) { return expf(x); }
// The hardware exponential: the error, |x| 2^-24 relative, is far below the rounding to bf16 that follows.
template <> __device__ __forceinline__ float exp_of<bf16_t>(float x) { return __expf(x); }
template <typename T> __device__ __forceinline__ float sigmoid_of(float x) { return 1.0f / (1.0f + exp_of<T>(-x)); }

// ---- what happens to eight consecutive columns of a row of the result ---------------------------------------------
// put: n of them exist; v, and for DUAL w, hold the sums.

template <typename T, bool SEGS, bool PAIR>
struct EpiStore {                                             // PRODUCT_DOWN, PRODUCT_DX, PRODUCT_DW
  static constexpr bool DUAL = false, SEGMENTS = SEGS, PAIRED = PAIR, RANGES = false;
  typedef T type;
  static __device__ __forceinline__ void put(const MatArgs& p, int z, int64_t row, int col, int n, float (&v)[8], float (&)[8]) {
    const int64_t at = row * p.ldc + col;
    if (PAIR) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= p.alpha;
    } else if (p.e1) {
      float base[8];
      load8(static_cast<const T*>(p.e1) + at, n, base);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += base[e];
    }
    store8(static_cast<T*>(PAIR && z ? p.c2 : p.c) + at, n, v);
  }
};

template <typename T>
struct EpiGated {
  static constexpr bool DUAL = true, SEGMENTS = false, PAIRED = false, RANGES = false;
  typedef T type;
  static __device__ __forceinline__ void put(const MatArgs& p, int, int64_t row, int col, int n, float (&v)[8], float (&w)[8]) {
    const int64_t at = row * p.ldc + col;
    if (p.c2) {
      store8(static_cast<T*>(p.c2) + at, n, v);
      store8(static_cast<T*>(p.c3) + at, n, w);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = v[e] * sigmoid_of<T>(v[e]) * w[e];
    store8(static_cast<T*>(p.c) + at, n, v);
  }
};

template <typename T>
struct EpiDGated {
  static constexpr bool DUAL = false, SEGMENTS = false, PAIRED = false, RANGES = false;
  typedef T type;
  static __device__ __forceinline__ void put(const MatArgs& p, int, int64_t row, int col, int n, float (&v)[8], float (&)[8]) {
    const int64_t at = row * p.ldc + col;
    float g[8], u[8];
    load8(static_cast<const T*>(p.e1) + at, n, g);
    load8(static_cast<const T*>(p.e2) + at, n, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float s = sigmoid_of<T>(g[e]);
      u[e] *= v[e] * s * (1.0f + g[e] * (1.0f - s));
      g[e] *= v[e] * s;
    }
    store8(static_cast<T*>(p.c) + at, n, u);
    store8(static_cast<T*>(p.c2) + at, n, g);
  }
};

template <typename T>
struct EpiDLogits {
  static constexpr bool DUAL = false, SEGMENTS = false, PAIRED = false, RANGES = false;
  typedef T type;
  static __device__ __forceinline__ void put(const MatArgs& p, int, int64_t row, int col, int n, float (&v)[8], float (&)[8]) {
    const int id = p.ids[row];
    const float lse = p.lse[row], weight = p.dloss ? p.dloss[row] : 1.0f;
    const bool has = (unsigned)id < (unsigned)p.vocab;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = exp_of<T>(v[e] - lse) - (id == p.col0 + col + e ? 1.0f : 0.0f);
      v[e] = has && col + e < p.n_b ? d * weight : 0.0f;     // (columns behind the vocabulary are zeros)
    }
    store8(static_cast<T*>(p.c) + row * p.ldc + col, n, v);
  }
};

template <typename T>
struct EpiDHead {
  static constexpr bool DUAL = false, SEGMENTS = false, PAIRED = false, RANGES = false;
  typedef T type;
  static __device__ __forceinline__ void put(const MatArgs& p, int, int64_t row, int col, int n, float (&v)[8], float (&)[8]) {
    float* acc = p.acc + row * p.n + col;
    if (!p.first) {
      float before[8];
      load8(acc, n, before);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += before[e];
    }
    if (p.last) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= p.alpha;
      store8(static_cast<T*>(p.c) + row * p.ldc + col, n, v);
    } else {
      store8(acc, n, v);
    }
  }
};

template <typename T>
struct EpiLse {
  static constexpr bool DUAL = false, SEGMENTS = false, PAIRED = false, RANGES = true;
  typedef T type;
  static __device__ __forceinline__ void put(const MatArgs&, int, int64_t, int, int, float (&)[8], float (&)[8]) {}
};

// The largest of two, and the exponentials summed below it.  An empty range is (-inf, 0).
__device__ __forceinline__ float2 join_ranges(float2 a, float2 b) {
  const float top = fmaxf(a.x, b.x);
  if (top == -INFINITY) return float2{top, a.y + b.y};
  return float2{top, a.y * __expf(a.x - top) + b.y * __expf(b.x - top)};
}

// Rows of a wave's tile, reduced over its columns where they are: a lane holds columns kq * 4 .. + 3 of every block of 16 in row r16.
// A NaN among the logits makes the sum NaN (fmaxf passes it over).
template <int MB, int NB>
__device__ __forceinline__ void put_ranges(const MatArgs& p, const floatx4_t (&acc)[MB][NB], int64_t row0, int col0, int range) {
  const int lane = threadIdx.x & 63, r16 = lane & 15, kq = lane >> 4;
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) {
    const int64_t row = row0 + mb * 16 + r16;
    const bool in = row < p.m;
    const int want = (int)((uint32_t)(in ? p.ids[row] : -1) - (uint32_t)(p.col0 + col0 + kq * 4));
    float top = -INFINITY;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool there = col0 + nb * 16 + kq * 4 + i < p.n;
        if (there) top = fmaxf(top, acc[mb][nb][i]);
        if (there && want == nb * 16 + i) p.picked[row] = acc[mb][nb][i];
      }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float from = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float e = __expf(acc[mb][nb][i] - from);
        sum += col0 + nb * 16 + kq * 4 + i < p.n ? e : 0.0f;
      }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (in && kq == 0) p.part[(int64_t)range * p.m + row] = float2{top, sum};
  }
}

// A wave's tile [MB * 16][NB * 16] from its accumulators to eight columns of a row per lane, 32 rows at a time through a strip of LDS
// that is the wave's own.
template <int MB, int NB>
constexpr int strip_floats() { return (MB > 1 ? 32 : 16) * (NB * 16 + 4); }

template <int MB, int NB, class EPI>
__device__ __forceinline__ void put_tile(const MatArgs& p, const floatx4_t (&acc)[MB][NB], float* strip, int z, int part, int64_t row0, int col0) {
  constexpr int RB = MB > 1 ? 2 : 1, TN = NB * 16, LD = TN + 4;
  constexpr int OUT = EPI::DUAL ? TN / 2 : TN, CH = OUT / 8;
  static_assert(MB % RB == 0, "rows of a strip");
  const int lane = threadIdx.x & 63, r16 = lane & 15, kq = lane >> 4;
  float* slab = p.k_split > 1 ? p.slab + ((int64_t)part * p.m) * (EPI::DUAL ? 2 * p.n : p.n) : nullptr;
#pragma unroll
  for (int mb = 0; mb < MB; mb += RB) {
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) *reinterpret_cast<floatx4_t*>(strip + (r * 16 + r16) * LD + nb * 16 + kq * 4) = acc[mb + r][nb];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 2
    for (int q = lane; q < RB * 16 * CH; q += 64) {
      const int rr = q / CH, cc = q % CH * 8;
      const int64_t row = row0 + mb * 16 + rr;
      const int col = col0 + cc;
      float v[8], w[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const floatx4_t f = *reinterpret_cast<const floatx4_t*>(strip + rr * LD + cc + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * h + e] = f[e];
        if (EPI::DUAL) {
          const floatx4_t g = *reinterpret_cast<const floatx4_t*>(strip + rr * LD + OUT + cc + 4 * h);
#pragma unroll
          for (int e = 0; e < 4; ++e) w[4 * h + e] = g[e];
        }
      }
      if (row >= p.m || col >= p.n) continue;
      const int n = p.n - col;
      if (slab) {
        float* to = slab + row * (EPI::DUAL ? 2 * p.n : p.n) + col;
        store8(to, n, v);
        if (EPI::DUAL) store8(to + p.n, n, w);
      } else {
        EPI::put(p, z, row, col, n, v, w);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// The parts of a K split, added in order.
template <class EPI>
__global__ __launch_bounds__(256) void matmul_finish(MatArgs p) {
  const int per_row = (p.n + 7) >> 3;
  const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = q / per_row;
  if (row >= p.m) return;
  const int col = (int)(q - row * per_row) * 8, n = p.n - col;
  const int64_t cols = EPI::DUAL ? 2 * (int64_t)p.n : p.n;
  const float* from = p.slab + row * cols + col;
  float v[8], w[8];
  load8(from, n, v);
  if (EPI::DUAL) load8(from + p.n, n, w);
  for (int s = 1; s < p.k_split; ++s) {
    float t[8];
    from += p.m * cols;
    load8(from, n, t);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += t[e];
    if (EPI::DUAL) {
      load8(from + p.n, n, t);
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] += t[e];
    }
  }
  EPI::put(p, 0, row, col, n, v, w);
}

// Which tile a workgroup has.  Workgroup b runs on XCD b % 8, each of which works through a run of the list, so that tiles that share
// an operand meet in one L2; inside the list the row tile runs fastest in bands of eight.  Behind the tiles of one part of K come those of the next.
struct TileAt {
  int mt, nt, part;
};
__device__ __forceinline__ bool find_tile(const MatArgs& p, int n_mt, int n_nt, TileAt* at) {
  const int tiles = n_mt * n_nt, total = tiles * p.k_split;
  const int chunk = (total + 7) >> 3;
  const int item = (blockIdx.x & 7) * chunk + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= chunk || item >= total) return false;
  at->part = item / tiles;
  const int local = item - at->part * tiles;
  constexpr int BAND = 8;
  const int band = local / (BAND * n_nt), rem = local - band * (BAND * n_nt);
  const int rows = min(n_mt - band * BAND, BAND);
  at->mt = band * BAND + rem % rows;
  at->nt = rem / rows;
  return true;
}
inline __host__ int grid_of(int64_t tiles, int k_split) { return (int)((tiles * k_split + 7) / 8 * 8); }

// ---- any size, alignment and type -----------------------------------------------------------------------------------

// Operands go through registers into LDS in rows of 64 bytes of K, whichever way they lie in memory, padded by 16 bytes: the 16 rows of
// a read then fall into different banks.  One K step is loaded while the one before it is multiplied.
template <typename T> struct AnyStep;
template <> struct AnyStep<float> { static constexpr int K = 16, E = 4, LD = 20; };
template <> struct AnyStep<bf16_t> { static constexpr int K = 32, E = 8, LD = 40; };

template <typename T>
struct Chunk {
  T v[AnyStep<T>::E];
};
template <typename T>
__device__ __forceinline__ Chunk<T> load_chunk(const T* p, int n) {
  constexpr int E = AnyStep<T>::E;
  if (n >= E) return __builtin_bit_cast(Chunk<T>, *reinterpret_cast<const Bytes16<T>*>(p));
  Chunk<T> c;
#pragma unroll
  for (int e = 0; e < E; ++e) c.v[e] = e < n ? p[e] : (T)0;
  return c;
}

template <typename T, int BM, int BN, int WGM, int WGN>
constexpr size_t mat_any_bytes() {
  const size_t strips = (size_t)WGM * WGN * strip_floats<BM / WGM / 16, BN / WGN / 16>() * 4, tiles = 2 * (size_t)(BM + BN) * AnyStep<T>::LD * sizeof(T);
  return strips > tiles ? strips : tiles;
}

template <int BM, int BN, int WGM, int WGN, bool ACOL, bool BCOL, class EPI>
__global__ __launch_bounds__(WGM* WGN * 64) void matmul_any(MatArgs p) {
  typedef typename EPI::type T;
  constexpr int NT = WGM * WGN * 64, K = AnyStep<T>::K, E = AnyStep<T>::E, LD = AnyStep<T>::LD, KC = K / E;
  constexpr int TM = BM / WGM, TN = BN / WGN, MB = TM / 16, NB = TN / 16;
  constexpr int A_N = (BM * KC + NT - 1) / NT, B_N = (BN * KC + NT - 1) / NT;   // chunks per thread and step
  static_assert(BM % 16 == 0 && BN % 64 == 0 && (BM * KC) % 64 == 0, "whole waves load");
  extern __shared__ __attribute__((aligned(16))) char any_smem[];
  T* const tiles = reinterpret_cast<T*>(any_smem);

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WGN, wn = wave % WGN, r16 = lane & 15, kq = lane >> 4;
  TileAt at;
  constexpr int BNO = EPI::DUAL ? BN / 2 : BN;
  if (!find_tile(p, (p.m + BM - 1) / BM, (p.n + BNO - 1) / BNO, &at)) return;
  const int z = blockIdx.y;
  const int row_first = at.mt * BM, col_first = at.nt * BNO;
  const int seg_steps = (p.k + K - 1) / K;
  const int all = EPI::SEGMENTS ? 2 * seg_steps : seg_steps;
  const int per = (all + p.k_split - 1) / p.k_split;
  const int k_begin = min(at.part * per, all), k_end = min(k_begin + per, all);

  Chunk<T> ra[A_N], rb[B_N];
  auto fetch = [&](auto col_tag, int c, int rows, const T* base, int64_t ld, int first, int size, int k_size, int k0) {
    Chunk<T> out = {};
    if constexpr (decltype(col_tag)::value) {                // chunk c: K row c / (rows / E), E columns
      const int kr = c / (rows / E), col = first + c % (rows / E) * E;
      if (k0 + kr < k_size && col < size) out = load_chunk<T>(base + (int64_t)(k0 + kr) * ld + col, size - col);
    } else {
      const int row = first + c / KC, k = k0 + c % KC * E;
      if (row < size && k < k_size) out = load_chunk<T>(base + (int64_t)row * ld + k, k_size - k);
    }
    return out;
  };
  auto load = [&](int s) {
    const bool second = EPI::SEGMENTS && s >= seg_steps;
    const int k0 = (second ? s - seg_steps : s) * K;
    const T* a = static_cast<const T*>(second ? p.a2 : p.a);
    const T* b = static_cast<const T*>(second || (EPI::PAIRED && z) ? p.b2 : p.b);
#pragma unroll
    for (int i = 0; i < A_N; ++i)
      if (BM * KC >= NT || tid < BM * KC) ra[i] = fetch(std::bool_constant<ACOL>{}, tid + i * NT, BM, a, p.lda, row_first, p.m_a, p.k, k0);
#pragma unroll
    for (int i = 0; i < B_N; ++i) {
      int c = tid + i * NT;
      const T* from = b;
      // DUAL: the tile's first half from B, its second from B2, the same columns of both
      if (EPI::DUAL && c >= BN * KC / 2) {
        c -= BN * KC / 2;
        from = static_cast<const T*>(p.b2);
      }
      rb[i] = fetch(std::bool_constant<BCOL>{}, c, EPI::DUAL ? BN / 2 : BN, from, p.ldb, col_first, p.n_b, p.k_b, k0);
    }
  };
  auto place = [&](auto col_tag, const Chunk<T>& v, int c, int rows, T* to) {
    if constexpr (decltype(col_tag)::value) {
      const int kr = c / (rows / E), col = c % (rows / E) * E;
#pragma unroll
      for (int e = 0; e < E; ++e) to[(col + e) * LD + kr] = v.v[e];
    } else {
      *reinterpret_cast<Chunk<T>*>(__builtin_assume_aligned(to + (c / KC) * LD + c % KC * E, 16)) = v;
    }
  };
  auto store = [&](int buf) {
    T* ta = tiles + buf * (BM + BN) * LD;
    T* tb = ta + BM * LD;
#pragma unroll
    for (int i = 0; i < A_N; ++i)
      if (BM * KC >= NT || tid < BM * KC) place(std::bool_constant<ACOL>{}, ra[i], tid + i * NT, BM, ta);
#pragma unroll
    for (int i = 0; i < B_N; ++i) {
      const int c = tid + i * NT;
      const bool up = EPI::DUAL && c >= BN * KC / 2;
      place(std::bool_constant<BCOL>{}, rb[i], up ? c - BN * KC / 2 : c, EPI::DUAL ? BN / 2 : BN, up ? tb + BN / 2 * LD : tb);
    }
  };

  floatx4_t acc[MB][NB];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) acc[mb][nb] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
  auto b_row = [&](int nb) {
    if (!EPI::DUAL) return wn * TN + nb * 16;
    return (nb / (NB / 2)) * (BN / 2) + wn * (TN / 2) + nb % (NB / 2) * 16;
  };
  if (k_begin < k_end) load(k_begin);
  int buf = 0;
  for (int s = k_begin; s < k_end; ++s) {
    store(buf);
    __syncthreads();                                         // (the reads of this buffer, two steps ago, lie before the last barrier)
    if (s + 1 < k_end) load(s + 1);
    const T* ta = tiles + buf * (BM + BN) * LD;
    const T* tb = ta + BM * LD;
    if constexpr (sizeof(T) == 4) {
      // K in the order of the reads: MFMA i takes elements 4 kq + i of both operands
      floatx4_t fa[MB], fb[NB];
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) fa[mb] = *reinterpret_cast<const floatx4_t*>(ta + (wm * TM + mb * 16 + r16) * LD + kq * 4);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) fb[nb] = *reinterpret_cast<const floatx4_t*>(tb + (b_row(nb) + r16) * LD + kq * 4);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) acc[mb][nb] = __builtin_amdgcn_mfma_f32_16x16x4f32(fb[nb][i], fa[mb][i], acc[mb][nb], 0, 0, 0);
    } else {
      bf16x8_t fa[MB], fb[NB];
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) fa[mb] = *reinterpret_cast<const bf16x8_t*>(ta + (wm * TM + mb * 16 + r16) * LD + kq * 8);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) fb[nb] = *reinterpret_cast<const bf16x8_t*>(tb + (b_row(nb) + r16) * LD + kq * 8);
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) acc[mb][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[nb], fa[mb], acc[mb][nb], 0, 0, 0);
    }
    buf ^= 1;
  }
  const int64_t row0 = row_first + wm * TM;
  if constexpr (EPI::RANGES) {
    put_ranges<MB, NB>(p, acc, row0, col_first + wn * TN, at.nt * WGN + wn);
  } else {
    __syncthreads();
    put_tile<MB, NB, EPI>(p, acc, reinterpret_cast<float*>(any_smem) + wave * strip_floats<MB, NB>(), z, at.part, row0, col_first + wn * (EPI::DUAL ? TN / 2 : TN));
  }
}

}  // namespace cmoe
