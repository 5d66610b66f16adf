// Kernels of the products in matmul.h.
//
// matmul_ring: bf16, both operands read 16 bytes at a time (widths that are multiples of 8, addresses of 16).  Bound by the matrix cores under
// the power limit with tiles of 256 x 256 (0.69 us a step of 32 K, 1.25 to 1.37 PFLOP/s in launches of whole rounds at 4096 x 14336 x 4096;
// other places of the reads and loads among the MFMAs change half a per cent), by what a CU takes in with smaller ones (62 KB a us).  The ring of
// gemm_bf16.hip with operands as they lie in a program's tensors: K steps of 32, global memory straight to LDS by buffer loads, STAGES
// - 1 steps in flight, the fragments of the next step read from LDS while this one is multiplied out of registers.  A
// stage holds an operand
//   by rows     in blocks of 16 rows x 32 K (1 KB: one load instruction of a wave, one operand of an MFMA), or
//   by columns  in panels of 32 K x 64 columns (4 KB: four load instructions of 8 K x 128 bytes): the 16 x 16 corners of an MFMA's
//               operand are turned on the way out of LDS by ds_read_b64_tr_b16, whose 16 lanes read 4 rows of K of 16 columns
//               (32 bytes each) and receive 4 K of one column each; two of them make an operand.
// Both are XOR-swizzled on the global side so that the lanes of a read fall into different banks: 16-byte chunks of a block's row
// with (row >> 2) & 3; 32-byte chunks of a panel's row k with bits 1 and 3 of k (bit 0 chooses the half of the 256-byte bank line,
// bit 2 is the other read).
//
// fp32 on the ring: an operand is copied into three planes of bf16 that hold its 24 bits (matmul_prepare; each plane is what is left, rounded to
// nearest, so that the rests have either sign and the planes' sum is the value).  A stage holds a step of all planes, and six products of planes are
// summed; the three that are left out, of the smaller planes, come to less than 2^-24 of the product, to either side: a product is as exact as an
// fp32 one (2^-24 at most for the last sum; planes that are cut have left-out products of the product's own sign: 0.65 x 2^-24 short on average, up to
// 7.8).  That holds from 2^-110 on (below it the last plane falls under bf16's smallest number).  Infinities become NaN.  Such a product runs at a sixth of
// the bf16 rate, above 200 TFLOP/s, where the fp32 matrix instructions have 157 at most.  bf16 operands at odd addresses or of odd
// widths are copied into one plane.
//
// matmul_any: both types, any alignment and size, operands through registers with every chunk's end checked: what is too small to be worth copying.
// fp32: 114 TFLOP/s on the fp32 matrix instructions at 2048 x 4096 x 2048, 44 where there are 1.5 tiles to a CU (517 x 1379 x 515: 33 us).
#pragma once
#include <type_traits>
#include <utility>

#include "device_utils.h"
#include "dropout_device.h"
#include "gemm_device.h"
#include "matmul.h"

namespace cmoe {

constexpr float LOG2E = 1.44269504088896341f;
// exp(x - from), 1 where they are equal: the difference is taken first, or the product's rounding would be an error of every exponential of a row.
template <typename T> __device__ __forceinline__ float exp_from(float x, float from);
template <> __device__ __forceinline__ float exp_from<float>(float x, float from) { return expf(x - from); }
// (the hardware's power of two: 1.3 x 2^-24 |x - from| relative, of logits that are sums in fp32 of thousands of products and
// no more exact.  expf: head-sized steps 2 to 2.5 per cent longer, 8192 tokens over 131072 entries 27.0 -> 27.7 ms)
template <> __device__ __forceinline__ float exp_from<bf16_t>(float x, float from) { return __builtin_amdgcn_exp2f((x - from) * LOG2E); }
template <typename T> __device__ __forceinline__ float sigmoid_of(float x);
template <> __device__ __forceinline__ float sigmoid_of<float>(float x) { return 1.0f / (1.0f + expf(-x)); }
// (the hardware's reciprocal: one unit in the last place of fp32, and the result is rounded to bf16; a division is ten instructions)
template <> __device__ __forceinline__ float sigmoid_of<bf16_t>(float x) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-x * LOG2E)); }

// ---- what happens to eight consecutive columns of a row of the result ---------------------------------------------
// hold: what it reads of global memory for them (n of them exist); put: with v, and for DUAL w, the sums.

// Eight values as they lie in memory.
template <typename T>
struct Raw8 {
  uint32_t w[2 * sizeof(T)];
};
template <typename T>
__device__ __forceinline__ void hold8(const T* p, int n, Raw8<T>& r) {
  if (n >= 8) {
#pragma unroll
    for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
      const Bytes16<T> b = *reinterpret_cast<const Bytes16<T>*>(p + 16 / sizeof(T) * h);
#pragma unroll
      for (int e = 0; e < 4; ++e) r.w[4 * h + e] = b.w[e];
    }
  } else {
    float v[8];
    load8(p, n, v);
#pragma unroll
    for (int e = 0; e < 2 * (int)sizeof(T); ++e) r.w[e] = sizeof(T) == 4 ? __float_as_uint(v[e]) : pack_bf16(v[2 * (e & 3)], v[2 * (e & 3) + 1]);
  }
}
template <typename T>
__device__ __forceinline__ float held(const Raw8<T>& r, int e) {
  if (sizeof(T) == 4) return __uint_as_float(r.w[e & (2 * sizeof(T) - 1)]);
  return __uint_as_float(e & 1 ? r.w[e >> 1] & 0xffff0000u : r.w[e >> 1] << 16);
}

__device__ __forceinline__ float alpha_of(const MatArgs& p) { return p.factor ? p.alpha * *p.factor : p.alpha; }

template <typename T, bool SEGS, bool PAIR>
struct EpiStore {                                             // PRODUCT_DOWN, PRODUCT_DX, PRODUCT_DW
  static constexpr bool LOGITS = false, DUAL = false, SEGMENTS = SEGS, PAIRED = PAIR, RANGES = false;
  typedef T type;
  struct Held {
    Raw8<T> base;
    float alpha;
  };
  static __device__ __forceinline__ void hold(const MatArgs& p, int64_t row, int col, int n, Held& h) {
    if (PAIR) h.alpha = alpha_of(p);
    else if (p.e1) hold8(static_cast<const T*>(p.e1) + row * p.ldc + col, n, h.base);
  }
  static __device__ __forceinline__ void put(const MatArgs& p, int z, int64_t row, int col, int n, float (&v)[8], float (&)[8], const Held& h) {
    if (PAIR) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= h.alpha;
    } else if (p.e1) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += held(h.base, e);
    }
    store8(static_cast<T*>(PAIR && z ? p.c2 : p.c) + row * p.ldc + col, n, v);
  }
};

struct HeldNothing {};

template <typename T>
struct EpiGated {
  static constexpr bool LOGITS = false, DUAL = true, SEGMENTS = false, PAIRED = false, RANGES = false;
  typedef T type;
  typedef HeldNothing Held;
  static __device__ __forceinline__ void hold(const MatArgs&, int64_t, int, int, Held&) {}
  static __device__ __forceinline__ void put(const MatArgs& p, int, int64_t row, int col, int n, float (&v)[8], float (&w)[8], const Held&) {
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
  static constexpr bool LOGITS = false, DUAL = false, SEGMENTS = false, PAIRED = false, RANGES = false;
  typedef T type;
  struct Held {
    Raw8<T> gate, up;
  };
  static __device__ __forceinline__ void hold(const MatArgs& p, int64_t row, int col, int n, Held& h) {
    const int64_t at = row * p.ldc + col;
    hold8(static_cast<const T*>(p.e1) + at, n, h.gate);
    hold8(static_cast<const T*>(p.e2) + at, n, h.up);
  }
  static __device__ __forceinline__ void put(const MatArgs& p, int, int64_t row, int col, int n, float (&v)[8], float (&)[8], const Held& h) {
    const int64_t at = row * p.ldc + col;
    float dg[8], du[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float g = held(h.gate, e), s = sigmoid_of<T>(g);
      dg[e] = held(h.up, e) * v[e] * s * (1.0f + g * (1.0f - s));
      du[e] = g * v[e] * s;
    }
    store8(static_cast<T*>(p.c) + at, n, dg);
    store8(static_cast<T*>(p.c2) + at, n, du);
  }
};

template <typename T>
struct EpiDLogits {
  static constexpr bool LOGITS = true, DUAL = false, SEGMENTS = false, PAIRED = false, RANGES = false;
  typedef T type;
  struct Held {
    int id;
    float lse, weight;
  };
  static __device__ __forceinline__ void hold(const MatArgs& p, int64_t row, int, int, Held& h) {
    h.id = p.ids[row];
    h.lse = p.lse[row];
    h.weight = p.dloss ? p.dloss[row] : 1.0f;
  }
  static __device__ __forceinline__ void put(const MatArgs& p, int, int64_t row, int col, int n, float (&v)[8], float (&)[8], const Held& h) {
    const bool has = (unsigned)h.id < (unsigned)p.vocab;
    const unsigned at = (unsigned)(h.id - p.col0 - col);     // of the target among the eight
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = exp_from<T>(v[e], h.lse);
    if (at < 8u) {                                           // (few waves have one)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] -= at == (unsigned)e ? 1.0f : 0.0f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = has ? v[e] * h.weight : 0.0f;
    if (col + 8 > p.n_b) {                                   // columns behind the vocabulary are zeros
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = col + e < p.n_b ? v[e] : 0.0f;
    }
    store8(static_cast<T*>(p.c) + row * p.ldc + col, n, v);
  }
};

template <typename T>
struct EpiDHead {
  static constexpr bool LOGITS = false, DUAL = false, SEGMENTS = false, PAIRED = false, RANGES = false;
  typedef T type;
  struct Held {
    Raw8<float> before;
    float alpha;
  };
  static __device__ __forceinline__ void hold(const MatArgs& p, int64_t row, int col, int n, Held& h) {
    if (!p.first) hold8(p.acc + row * p.n + col, n, h.before);
    if (p.last) h.alpha = alpha_of(p);
  }
  static __device__ __forceinline__ void put(const MatArgs& p, int, int64_t row, int col, int n, float (&v)[8], float (&)[8], const Held& h) {
    if (!p.first) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += held(h.before, e);
    }
    if (p.last) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= h.alpha;
      store8(static_cast<T*>(p.c) + row * p.ldc + col, n, v);
    } else {
      store8(p.acc + row * p.n + col, n, v);
    }
  }
};

template <typename T>
struct EpiLse {
  static constexpr bool LOGITS = true, DUAL = false, SEGMENTS = false, PAIRED = false, RANGES = true;
  typedef T type;
  typedef HeldNothing Held;
  static __device__ __forceinline__ void hold(const MatArgs&, int64_t, int, int, Held&) {}
  static __device__ __forceinline__ void put(const MatArgs&, int, int64_t, int, int, float (&)[8], float (&)[8], const Held&) {}
};

// The largest of two, and the exponentials summed below it.  An empty range is (-inf, 0).  (expf, of bf16 logits too: a range's factor is an error
// of its whole sum, and a power of two of (x - from) log2 e would be off by |x - from| roundings, 14 at -13.)
__device__ __forceinline__ float2 join_ranges(float2 a, float2 b) {
  const float top = fmaxf(a.x, b.x);
  if (top == -INFINITY) return float2{top, a.y + b.y};
  return float2{top, a.y * expf(a.x - top) + b.y * expf(b.x - top)};
}

// Rows of a wave's tile, reduced over its columns where they are: a lane holds columns kq * 4 .. + 3 of every block of 16 in row r16.
// A NaN among the logits makes the sum NaN (fmaxf passes it over).  The vector units' time for this is a CU's own, nothing else runs beside it: whole
// tiles look for no edge, and rows whose target is in other columns for no target.
template <typename T, bool WHOLE, int MB, int NB>
__device__ __forceinline__ void put_rows(const MatArgs& p, const floatx4_t (&acc)[MB][NB], int64_t row0, int col0, int range) {
  const int lane = threadIdx.x & 63, r16 = lane & 15, kq = lane >> 4;
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) {
    const int64_t row = row0 + mb * 16 + r16;
    const bool in = WHOLE || row < p.m;
    const int want = (int)((uint32_t)(in ? p.ids[row] : -1) - (uint32_t)(p.col0 + col0 + kq * 4));
    if ((unsigned)want < (unsigned)(NB * 16)) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (want == nb * 16 + i && (WHOLE || col0 + nb * 16 + kq * 4 + i < p.n)) p.picked[row] = acc[mb][nb][i];
    }
    auto there = [&](int nb, int i) { return WHOLE || col0 + nb * 16 + kq * 4 + i < p.n; };
    float top = -INFINITY;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = there(nb, i) ? fmaxf(top, acc[mb][nb][i]) : top;
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float from = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float e = exp_from<T>(acc[mb][nb][i], from);
        sum += there(nb, i) ? e : 0.0f;
      }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (in && kq == 0) p.part[(int64_t)range * p.m + row] = float2{top, sum};
  }
}
template <typename T, int MB, int NB>
__device__ __forceinline__ void put_ranges(const MatArgs& p, const floatx4_t (&acc)[MB][NB], int64_t row0, int col0, int range) {
  if (row0 + MB * 16 <= p.m && col0 + NB * 16 <= p.n) put_rows<T, true>(p, acc, row0, col0, range);
  else put_rows<T, false>(p, acc, row0, col0, range);
}

// Which tile a workgroup has.  Workgroup b runs on XCD b % 8, each of which works through a run of the list, so that tiles that share
// an operand meet in one L2; inside the list the row tile runs fastest in bands of eight.  The last p.full .. tiles, which would not fill the
// chip, are given to p.k_split workgroups each, a range of K to every one: behind the parts of one range come those of the next.
struct TileAt {
  int mt, nt, z;
  int part;                  // of p.k_split
  int slot;                  // among the tiles that are split; -1: this one is not
};
__device__ __forceinline__ void tile_of(const MatArgs& p, int tile, int n_mt, int n_nt, TileAt* at) {
  const int each = n_mt * n_nt;
  at->z = tile >= each;
  const int local = tile - at->z * each;
  constexpr int BAND = 8;
  const int band = local / (BAND * n_nt), rem = local - band * (BAND * n_nt);
  const int rows = min(n_mt - band * BAND, BAND);
  at->mt = band * BAND + rem % rows;
  at->nt = rem / rows;
}
__device__ __forceinline__ bool find_tile(const MatArgs& p, int n_mt, int n_nt, TileAt* at) {
  const int b = blockIdx.x;
  int tile;
  at->part = 0;
  at->slot = -1;
  if (b < p.full) {
    tile = (b & 7) * (p.full >> 3) + (b >> 3);
  } else {
    const int rest = n_mt * n_nt * p.zs - p.full, items = rest * p.k_split, chunk = (items + 7) >> 3;
    const int item = (b & 7) * chunk + ((b - p.full) >> 3);
    if (((b - p.full) >> 3) >= chunk || item >= items) return false;
    at->part = item / rest;
    const int slot = item - at->part * rest;
    if (p.k_split > 1) at->slot = slot;
    tile = p.full + slot;
  }
  tile_of(p, tile, n_mt, n_nt, at);
  return true;
}

// A wave's tile [MB * 16][NB * 16] from its accumulators to eight columns of a row per lane, 32 rows at a time through a strip of LDS
// that is the wave's own.
template <int MB, int NB>
constexpr int strip_floats() { return (MB > 1 ? 32 : 16) * (NB * 16 + 4); }

template <int MB, int NB, class EPI>
__device__ __forceinline__ void put_tile(const MatArgs& p, const floatx4_t (&acc)[MB][NB], float* strip, const TileAt& at, int wave_row, int wave_col, int64_t row0,
                                         int col0) {
  constexpr int RB = MB > 1 ? 2 : 1, TN = NB * 16, LD = TN + 4;
  constexpr int OUT = EPI::DUAL ? TN / 2 : TN, CH = OUT / 8, TURNS = RB * 16 * CH / 64;
  static_assert(MB % RB == 0 && RB * 16 * CH % 64 == 0, "rows of a strip");
  const int lane = threadIdx.x & 63, r16 = lane & 15, kq = lane >> 4;
  if (at.slot >= 0) {
    // a part of a tile: its sums as they are, the tile's rows one after the other
    float* slab = p.slab + ((int64_t)(at.slot * p.k_split + at.part) * p.bm + wave_row) * p.bn;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int col = EPI::DUAL ? nb / (NB / 2) * (p.bn / 2) + wave_col + nb % (NB / 2) * 16 : wave_col + nb * 16;
        *reinterpret_cast<floatx4_t*>(slab + (mb * 16 + r16) * p.bn + col + kq * 4) = acc[mb][nb];
      }
    return;
  }
  if constexpr (EPI::RANGES) return;                         // (whole tiles of logits are reduced where they are)
  auto stage = [&](int mb) {
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) *reinterpret_cast<floatx4_t*>(strip + (r * 16 + r16) * LD + nb * 16 + kq * 4) = acc[mb + r][nb];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };
  auto take = [&](int rr, int cc, float (&v)[8], float (&w)[8]) {
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
  };
  if (row0 + MB * 16 <= p.m && col0 + OUT <= p.n) {
    // A tile that is whole: nothing has to be asked for every row, and what the rows of a strip read is under way before the strip is written.
    typename EPI::Held held[TURNS];
    const int rr0 = lane / CH, cc = lane % CH * 8;
#pragma unroll
    for (int mb = 0; mb < MB; mb += RB) {
#pragma unroll
      for (int t = 0; t < TURNS; ++t) EPI::hold(p, row0 + mb * 16 + rr0 + t * (64 / CH), col0 + cc, 8, held[t]);
      stage(mb);
#pragma unroll
      for (int t = 0; t < TURNS; ++t) {
        float v[8], w[8];
        take(rr0 + t * (64 / CH), cc, v, w);
        EPI::put(p, at.z, row0 + mb * 16 + rr0 + t * (64 / CH), col0 + cc, 8, v, w, held[t]);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    return;
  }
#pragma unroll
  for (int mb = 0; mb < MB; mb += RB) {
    stage(mb);
#pragma unroll 1
    for (int q = lane; q < RB * 16 * CH; q += 64) {
      const int rr = q / CH, cc = q % CH * 8;
      const int64_t row = row0 + mb * 16 + rr;
      const int col = col0 + cc;
      float v[8], w[8];
      take(rr, cc, v, w);
      if (row >= p.m || col >= p.n) continue;
      typename EPI::Held held;
      EPI::hold(p, row, col, p.n - col, held);
      EPI::put(p, at.z, row, col, p.n - col, v, w, held);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// The parts of the tiles that are split, added in order: a thread per eight columns, gridDim.y parts of a tile.  Bound by memory: 128 tiles of 256 x
// 256 in two parts 13.5 us (80 MB), a few small ones 4 (a launch).
template <class EPI>
__global__ __launch_bounds__(256) void matmul_finish(MatArgs p) {
  const int bno = EPI::DUAL ? p.bn / 2 : p.bn, per_row = bno >> 3;
  const int q = blockIdx.y * 256 + threadIdx.x, rr = q / per_row, cc = q % per_row * 8;
  TileAt at;
  tile_of(p, p.full + blockIdx.x, (p.m + p.bm - 1) / p.bm, (p.n + bno - 1) / bno, &at);
  const int64_t row = (int64_t)at.mt * p.bm + rr;
  const int col = at.nt * bno + cc, n = p.n - col;
  if (rr >= p.bm || row >= p.m || col >= p.n) return;
  const int64_t each = (int64_t)p.bm * p.bn;
  const float* from = p.slab + blockIdx.x * p.k_split * each + rr * p.bn + cc;
  float v[8], w[8];
  typename EPI::Held held;
  EPI::hold(p, row, col, n, held);
  load8(from, 8, v);
  if (EPI::DUAL) load8(from + bno, 8, w);
#pragma unroll 2
  for (int s = 1; s < p.k_split; ++s) {
    float t[8];
    from += each;
    load8(from, 8, t);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += t[e];
    if (EPI::DUAL) {
      load8(from + bno, 8, t);
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] += t[e];
    }
  }
  EPI::put(p, at.z, row, col, n, v, w, held);
}

// The same of logits: a wave per row of a tile, its columns' largest and sum as the first of the ranges that the tile has, the others empty.
template <typename T>
__global__ __launch_bounds__(256) void matmul_finish_ranges(MatArgs p, int ranges) {
  const int lane = threadIdx.x & 63, rr = blockIdx.y * 4 + (threadIdx.x >> 6);
  TileAt at;
  tile_of(p, p.full + blockIdx.x, (p.m + p.bm - 1) / p.bm, (p.n + p.bn - 1) / p.bn, &at);
  const int64_t row = (int64_t)at.mt * p.bm + rr;
  if (rr >= p.bm || row >= p.m) return;
  const int64_t each = (int64_t)p.bm * p.bn;
  const float* from = p.slab + (int64_t)blockIdx.x * p.k_split * each + rr * p.bn;
  const int want = (int)((uint32_t)p.ids[row] - (uint32_t)(p.col0 + at.nt * p.bn));
  float2 mine = {-INFINITY, 0.0f};
  for (int c = lane; c < p.bn; c += 64) {
    float v = from[c];
    for (int s = 1; s < p.k_split; ++s) v += from[s * each + c];
    if (at.nt * p.bn + c >= p.n) break;
    if (want == c) p.picked[row] = v;
    // (a NaN is passed over by the maximum and makes the sum one)
    const float top = fmaxf(mine.x, v);
    mine.y = (mine.y > 0.0f ? mine.y * exp_from<T>(mine.x, top) : mine.y) + (top == -INFINITY && v == v ? 0.0f : exp_from<T>(v, top));
    mine.x = top;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) mine = join_ranges(mine, float2{__shfl_xor(mine.x, d), __shfl_xor(mine.y, d)});
  if (lane < ranges) p.part[((int64_t)at.nt * ranges + lane) * p.m + row] = lane == 0 ? mine : float2{-INFINITY, 0.0f};
}

// ---- operands copied for the ring ---------------------------------------------------------------------------------------

struct Copied {
  const void* from;          // [rows, cols], rows `ld` apart
  bf16_t* to;                // [planes][rows][pitch], zeros behind the columns
  int64_t ld, rows;
  int cols, pitch;
  uint32_t first, unused;    // its first workgroup
};
struct CopyArgs {
  Copied op[4];
  int n;
};

// A thread per eight columns.  Bound by memory: 4118 x 2880 and 716 x 2880 in fp32, 139 MB read and written, in 22 us.
template <typename T>
__global__ __launch_bounds__(256) void matmul_prepare(CopyArgs args) {
  int which = 0;
  for (int i = 1; i < args.n; ++i)
    if (args.op[i].first <= blockIdx.x) which = i;
  const Copied& op = args.op[which];
  const uint32_t per_row = (uint32_t)op.pitch >> 3;
  const uint64_t chunk = (uint64_t)(blockIdx.x - op.first) * 256;
  const uint64_t row0 = chunk / per_row;
  const uint32_t c0 = (uint32_t)(chunk - row0 * per_row) + threadIdx.x;
  const int64_t row = row0 + c0 / per_row;
  if (row >= op.rows) return;
  const int col = (int)(c0 % per_row) * 8, n = op.cols - col;
  float v[8] = {};
  if (n > 0) load8(static_cast<const T*>(op.from) + row * op.ld + col, n, v);
  bf16_t* to = op.to + row * op.pitch + col;
  if constexpr (sizeof(T) == 2) {
    store8(to, 8, v);
  } else {
    float top[8], mid[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      top[e] = as_stored<bf16_t>(v[e]);
      // (above bf16's largest number fp32 has some that would be rounded to infinity: their first plane is cut)
      if (isinf(top[e]) && !isinf(v[e])) top[e] = __uint_as_float(__float_as_uint(v[e]) & 0xffff0000u);
      // (an infinity or NaN is passed on as NaN: its rest is NaN)
      const float rest = v[e] - top[e];
      mid[e] = as_stored<bf16_t>(rest);
      v[e] = rest - mid[e];
    }
    const int64_t plane = op.rows * op.pitch;
    store8(to, 8, top);
    store8(to + plane, 8, mid);
    store8(to + 2 * plane, 8, v);
  }
}

// ---- the ring -------------------------------------------------------------------------------------------------------

typedef short shortx4_t __attribute__((ext_vector_type(4)));

// `__restrict__` is not for the programmer: inlined, it leaves the read with an alias scope, and the compiler then does not take it to wait for
// every load into LDS that is under way (vmcnt(0) in front of each read, 0.4 of the rate; it takes ordinary reads so by their
// type).  What they have to wait for is waited for by hand at the barrier of a step.
__device__ __forceinline__ shortx4_t read_turned(const bf16_t* __restrict__ at) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4_t*)(at));
#else
  return shortx4_t{};
#endif
}

// Eight K of a column: two reads, the second `further` elements on.
__device__ __forceinline__ bf16x8_t read_turned2(const bf16_t* at, int further) {
  union { shortx4_t h[2]; bf16x8_t v; } u;
  u.h[0] = read_turned(at);
  u.h[1] = read_turned(at + further);
  return u.v;
}

constexpr int mat_ring_elems(int bm, int bn, int stages, int planes) { return stages * planes * (bm + bn) * BK; }
template <class EPI>
constexpr int planes_of() { return sizeof(typename EPI::type) == 4 ? 3 : 1; }
template <int BM, int BN, int STAGES, int WGM, int WGN, class EPI>
constexpr size_t mat_ring_bytes() {
  const int strips = WGM * WGN * strip_floats<BM / WGM / 16, BN / WGN / 16>() * 4, ring = mat_ring_elems(BM, BN, STAGES, planes_of<EPI>()) * 2;
  return ring > strips ? ring : strips;
}

constexpr int FEW_ROWS = 64;                                 // whose products are bound by the other operand's way out of memory

// f(0), f(1) ... with indices that are constants: more of them than the compiler unrolls of a loop.
template <int N, class F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void each_index(F&& f) {
  each_of<N>(f, std::make_integer_sequence<int, N>{});
}

// The pairs of planes of two fp32 operands whose products count; the last one's sums are by far the largest and are kept apart from the others'.
constexpr int PAIRS = 6;
constexpr int kPairA[PAIRS] = {0, 1, 2, 0, 1, 0}, kPairB[PAIRS] = {2, 1, 0, 1, 0, 0};

template <int BM, int BN, int STAGES, int WGM, int WGN, bool ACOL, bool BCOL, class EPI>
__global__ __launch_bounds__(WGM* WGN * 64)
__attribute__((amdgpu_waves_per_eu(mat_ring_elems(BM, BN, STAGES, planes_of<EPI>()) * 2 <= 80 * 1024 ? 2 : 1))) void matmul_ring(MatArgs p) {
  constexpr int NW = WGM * WGN;
  constexpr int TM = BM / WGM, TN = BN / WGN, MB = TM / 16, NB = TN / 16;
  constexpr int PL = planes_of<EPI>();
  constexpr int A_CH = BM / 16 / NW, B_CH = BN / 16 / NW, LPT = PL * (A_CH + B_CH);   // load instructions per wave and step
  constexpr int A_ELEMS = PL * BM * BK, STAGE_ELEMS = PL * (BM + BN) * BK;
  constexpr int SEGS = EPI::SEGMENTS ? 2 : 1;                                  // parts of K one after the other
  static_assert(NW == 4 && BM % 64 == 0 && BN % 64 == 0, "a wave loads whole blocks and panels");
  static_assert((!ACOL || TM % 64 == 0) && (!BCOL || EPI::DUAL || TN % 64 == 0), "panels belong to one wave column");
  static_assert(!EPI::DUAL || (BCOL && BN % 128 == 0 && (TN / 2) % 32 == 0), "gate and up panels alternate");
  static_assert(STAGES >= 3 && (STAGES - 1) * LPT < 64, "ring depth");
  extern __shared__ __attribute__((aligned(16))) bf16_t smem[];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WGN, wn = wave % WGN;
  const int r16 = lane & 15, kq = lane >> 4;

  TileAt at;
  constexpr int BNO = EPI::DUAL ? BN / 2 : BN;               // columns of the result in a tile
  if (!find_tile(p, (p.m + BM - 1) / BM, (p.n + BNO - 1) / BNO, &at)) return;
  const int z = at.z;
  const int row_first = at.mt * BM, col_first = at.nt * BNO;
  const int seg_steps = (p.k + BK - 1) / BK;                 // steps of a part of K
  const int all = SEGS * seg_steps;
  const int per = at.slot < 0 ? all : (all + p.k_split - 1) / p.k_split;
  const int k_begin = min(at.part * per, all), KT = min(per, all - k_begin);

  // Lanes' offsets in bytes from the operand's place of a step; DMA_NONE: zeros.  By rows: load i of a wave is block wave + 4 i,
  // lane l its row l / 4 and chunk (l % 4) ^ (row >> 2) & 3.  By columns: load i is a quarter of panel i, lane l row l / 8 of
  // it and the 16-byte chunk that the swizzle puts at l % 8.
  const int coff = ((lane & 3) ^ ((lane >> 4) & 3)) << 3;
  const int pk = wave * 8 + (lane >> 3);                     // row of a panel
  const int pcol = ((((lane & 7) >> 1) ^ (((pk >> 1) & 1) | (((pk >> 3) & 1) << 1))) << 4) + ((lane & 1) << 3);
  uint32_t a_off[A_CH], b_off[B_CH];
#pragma unroll
  for (int i = 0; i < A_CH; ++i) {
    if (ACOL) a_off[i] = row_first + i * 64 + pcol < p.m_a ? (uint32_t)((pk * p.lda + i * 64 + pcol) * 2) : DMA_NONE;
    else a_off[i] = row_first + (wave + i * NW) * 16 + (lane >> 2) < p.m_a ? (uint32_t)((((wave + i * NW) * 16 + (lane >> 2)) * p.lda + coff) * 2) : DMA_NONE;
  }
#pragma unroll
  for (int i = 0; i < B_CH; ++i) {
    const int panel = EPI::DUAL ? i >> 1 : i;
    if (BCOL) b_off[i] = col_first + panel * 64 + pcol < p.n_b ? (uint32_t)((pk * p.ldb + panel * 64 + pcol) * 2) : DMA_NONE;
    else b_off[i] = col_first + (wave + i * NW) * 16 + (lane >> 2) < p.n_b ? (uint32_t)((((wave + i * NW) * 16 + (lane >> 2)) * p.ldb + coff) * 2) : DMA_NONE;
  }
  const bool k_past = (seg_steps - 1) * BK + coff >= p.k;    // of a part's last step, by rows

  // The step that is fetched next: part of K, step in it, and where its operands lie.  Where there are few rows the columns' tiles share
  // next to nothing, and each 256 columns begin K at a place of their own: rows of B a power of two apart would otherwise ask the same few
  // channels of the memory at the same time.  (By the column and not the tile: a logit has the same bits in the forward and in the backward pass.)
  constexpr bool TURNS = !ACOL && !BCOL && SEGS == 1;
  const int turn = TURNS && p.m <= FEW_ROWS && KT > 0 ? (p.col0 + col_first) / 256 * 5 % KT : 0;
  int f_left = KT, f_seg = SEGS > 1 && seg_steps > 0 ? k_begin / seg_steps : 0, f_step = k_begin - f_seg * seg_steps + turn;
  const bf16_t *f_a, *f_b, *f_b2 = nullptr;
  auto place_of = [&]() {
    const bool second = EPI::SEGMENTS && f_seg > 0;
    f_a = uniform_ptr(static_cast<const bf16_t*>(second ? p.a2 : p.a) + (ACOL ? row_first + f_step * BK * p.lda : row_first * p.lda + f_step * BK));
    const int64_t at_b = BCOL ? col_first + f_step * BK * p.ldb : col_first * p.ldb + f_step * BK;
    f_b = uniform_ptr(static_cast<const bf16_t*>(second || (EPI::PAIRED && z) ? p.b2 : p.b) + at_b);
    if (EPI::DUAL) f_b2 = uniform_ptr(static_cast<const bf16_t*>(p.b2) + at_b);
  };
  place_of();
  auto advance = [&]() {
    --f_left;
    if (++f_step == seg_steps && SEGS > 1) {
      f_step = 0;
      f_seg = f_seg + 1 < SEGS ? f_seg + 1 : 0;              // (behind the last part nothing is read)
      place_of();
    } else if (TURNS && f_step == k_begin + KT) {
      f_step = k_begin;
      place_of();
    } else {
      f_a += ACOL ? BK * p.lda : BK;
      f_b += BCOL ? BK * p.ldb : BK;
      if (EPI::DUAL) f_b2 += BK * p.ldb;
    }
  };
  // Lanes outside of an operand ask for nothing; the buffer's size is what the rows of a step by columns hold, so that K past its end is
  // zeros, and nothing behind the last step.
  auto fetch = [&](auto col_tag, const bf16_t* base, int64_t ld, int k, uint32_t off, bf16_t* dst) {
    uint32_t size = DMA_NONE;
    if constexpr (decltype(col_tag)::value) {
      const int rows = min(k - f_step * BK, BK);
      size = rows > 0 ? (uint32_t)(rows * ld * 2) : 0;
    } else {
      off = f_step == seg_steps - 1 && k_past ? DMA_NONE : off;
    }
    dma16_buffer(base, __builtin_amdgcn_readfirstlane(f_left > 0 ? size : 0), off, 0, dst);
  };
  auto issue = [&](int slot, int i) {                        // load i of the step fetched next
    const int plane = i / (A_CH + B_CH), q = i % (A_CH + B_CH);
    bf16_t* st = smem + slot * STAGE_ELEMS;
    if (q < A_CH) {
      fetch(std::bool_constant<ACOL>{}, PL > 1 ? uniform_ptr(f_a + plane * p.a_plane) : f_a, p.lda, p.k, a_off[q],
            st + plane * BM * BK + (ACOL ? q * 2048 + wave * 512 : (wave + q * NW) * BLK));
    } else {
      const int j = q - A_CH;
      const bf16_t* base = EPI::DUAL && (j & 1) ? f_b2 : f_b;
      fetch(std::bool_constant<BCOL>{}, PL > 1 ? uniform_ptr(base + plane * p.b_plane) : base, p.ldb, p.k_b, b_off[j],
            st + A_ELEMS + plane * BN * BK + (BCOL ? j * 2048 + wave * 512 : (wave + j * NW) * BLK));
    }
  };

  // fragments: of a block row r16, chunk kq; of a panel columns r16 of a block of 16, K kq * 8 .. + 7 in two reads
  const int frag = r16 * BK + ((kq ^ (r16 >> 2)) << 3);
  const int tj = r16 >> 2;                                   // K row of a read that the lane asks for
  const int swz = ((tj >> 1) & 1) | ((kq & 1) << 1);
  int turned[4];                                             // by block of 16 columns of a panel (DUAL, TN 64: from the wave's first on)
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int cb = (c + (EPI::DUAL ? wn * (TN / 32) : 0)) & 3;
    turned[c] = (kq * 8 + tj) * 64 + ((cb ^ swz) << 4) + ((r16 & 3) << 2);
  }
  int turned_a[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) turned_a[c] = (kq * 8 + tj) * 64 + ((c ^ swz) << 4) + ((r16 & 3) << 2);

  floatx4_t acc[MB][NB], low[PL > 1 ? MB : 1][PL > 1 ? NB : 1];               // low: of the pairs of planes but the last
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        acc[mb][nb][i] = 0.0f;
        if (PL > 1) low[mb][nb][i] = 0.0f;
      }

  bf16x8_t af[2][PL * MB], wf[2][PL * NB];
  auto load_frag = [&](int slot, int f, int set) {           // of every plane B's fragments first, then A's
    const int plane = f / (NB + MB), g = f % (NB + MB);
    const bf16_t* st = smem + slot * STAGE_ELEMS;
    if (g < NB) {
      const bf16_t* tb = st + A_ELEMS + plane * BN * BK;
      bf16x8_t& to = wf[set][plane * NB + g];
      if constexpr (!BCOL) to = *reinterpret_cast<const bf16x8_t*>(tb + (wn * NB + g) * BLK + frag);
      else if constexpr (EPI::DUAL) {
        const int which = g / (NB / 2), c = g % (NB / 2);    // panel of the wave's column block, in gate / up pairs
        to = read_turned2(tb + ((wn * (NB / 2) / 4 + c / 4) * 2 + which) * 2048 + turned[c % 4], 4 * 64);
      } else to = read_turned2(tb + (wn * (NB / 4) + g / 4) * 2048 + turned[g % 4], 4 * 64);
    } else {
      const bf16_t* ta = st + plane * BM * BK;
      const int q = g - NB;
      if constexpr (!ACOL) af[set][plane * MB + q] = *reinterpret_cast<const bf16x8_t*>(ta + (wm * MB + q) * BLK + frag);
      else af[set][plane * MB + q] = read_turned2(ta + (wm * (MB / 4) + q / 4) * 2048 + turned_a[q % 4], 4 * 64);
    }
  };
  static_assert(!EPI::DUAL || NB / 2 == 2 || NB / 2 % 4 == 0, "a wave's gate columns are whole panels, or half of one");

  constexpr int NM = (PL > 1 ? PAIRS : 1) * MB * NB, NF = PL * (MB + NB), ND = LPT;
  static_assert(ND <= NM, "at most one load instruction after an MFMA");
#pragma unroll
  for (int st = 0; st < STAGES; ++st) {
#pragma unroll
    for (int i = 0; i < ND; ++i) issue(st, i);
    advance();
  }
  wait_vmcnt<(STAGES - 1) * ND>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int f = 0; f < NF; ++f) load_frag(0, f, 0);

  int slot = 0;
  auto step = [&](auto set_tag, auto wait_tag) {
    constexpr int SET = decltype(set_tag)::value;
    constexpr bool WAIT = decltype(wait_tag)::value;
    // this wave's loads of the next step have landed and its reads of this one have returned: behind the barrier the next step may be
    // read and this one's slot refilled (a bare barrier: __syncthreads() would drain every load)
    wait_vmcnt<(STAGES - 2) * ND>();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const int next = slot + 1 == STAGES ? 0 : slot + 1;
    each_index<NM>([&](auto m_tag) {
      constexpr int m = decltype(m_tag)::value, pair = m / (MB * NB), mb = m / NB % MB, nb = m % NB;
      constexpr int pa = PL > 1 ? kPairA[pair] : 0, pb = PL > 1 ? kPairB[pair] : 0;
      floatx4_t& sum = PL > 1 && pair < PAIRS - 1 ? low[PL > 1 ? mb : 0][PL > 1 ? nb : 0] : acc[mb][nb];
      __builtin_amdgcn_sched_barrier(0);
      mfma_acc<WAIT && m == NM - 1>(sum, wf[SET][pb * NB + nb], af[SET][pa * MB + mb]);
      __builtin_amdgcn_sched_barrier(0);
      // the fragments of the next step in the first three quarters of the MFMAs, the load instructions spread over all
      constexpr int f0 = (m * NF * 4 + NM * 3 - 1) / (NM * 3), f1 = ((m + 1) * NF * 4 + NM * 3 - 1) / (NM * 3);
#pragma unroll
      for (int f = f0; f < (f1 < NF ? f1 : NF); ++f) load_frag(next, f, SET ^ 1);
      // (load i follows MFMA i NM / ND, each another one since there are no more loads than MFMAs)
      constexpr int i = (m * ND + NM - 1) / NM;
      if constexpr (i < ND && i * NM / ND == m) issue(slot, i);
    });
    advance();
    __builtin_amdgcn_sched_barrier(0);
    slot = next;
  };
  // Logits of few rows, which one token's loss hangs on: sums of 512 K each, added up beside, have a third of the rounding of one chain (4096 K:
  // 3e-6 of a logit of 16 or so before).  Smaller tiles have the registers for it, larger ones are not taken for few rows.
  constexpr bool BESIDE = EPI::LOGITS && PL == 1 && BM * BN <= 128 * 128;
  floatx4_t beside[BESIDE ? MB : 1][BESIDE ? NB : 1] = {};
  const bool few = BESIDE && p.m <= FEW_ROWS;
  int ks = 0;
  for (; ks + 1 < KT; ks += 2) {
    step(std::integral_constant<int, 0>{}, std::false_type{});
    step(std::integral_constant<int, 1>{}, std::true_type{});
    if constexpr (BESIDE) {
      if (few && (ks & 14) == 14) {
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            beside[mb][nb] += acc[mb][nb];
            acc[mb][nb] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
          }
      }
    }
  }
  if (ks < KT) step(std::integral_constant<int, 0>{}, std::true_type{});
  if constexpr (BESIDE) {
    if (few) {
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) acc[mb][nb] += beside[mb][nb];
    }
  }
  if constexpr (PL > 1) {
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) acc[mb][nb] += low[mb][nb];
  }
  __builtin_amdgcn_sched_barrier(0);
  wait_vmcnt<0>();                                           // (no load into LDS may outlive the workgroup)
  const int64_t row0 = row_first + wm * TM;
  if (EPI::RANGES && at.slot < 0) {
    put_ranges<typename EPI::type>(p, acc, row0, col_first + wn * TN, at.nt * WGN + wn);
  } else {
    __syncthreads();                                         // every wave has left the ring
    put_tile<MB, NB, EPI>(p, acc, reinterpret_cast<float*>(smem) + wave * strip_floats<MB, NB>(), at, wm * TM, wn * (EPI::DUAL ? TN / 2 : TN), row0,
                          col_first + wn * (EPI::DUAL ? TN / 2 : TN));
  }
}

// ---- any size, alignment and type -----------------------------------------------------------------------------------

// Steps of 128 bytes of K, through registers: two steps are under way while a third is multiplied out of LDS, since a step is shorter than the
// memory's latency.  An operand by rows lies in LDS in rows of 128 bytes padded by 16 (16 rows of a ds_read_b128 in different banks);
// by columns as in memory, a row per K, and an MFMA's operand is taken down a column: in fp32 one value per K (rows padded so that four
// K apart is a quarter of the banks apart), in bf16 turned by ds_read_b64_tr_b16 (four K at eight banks from one another).
template <typename T>
struct Any {
  static constexpr int E = 16 / sizeof(T), K = 128 / sizeof(T), KC = 8;      // values of a chunk, K of a step, chunks of a row
  static constexpr int ROW = K + E;                                          // pitch of an operand by rows
  static constexpr int pitch(int cols) { return sizeof(T) == 4 ? cols + 4 : cols + 16; }
  static constexpr int elems(bool columns, int size) { return columns ? K * pitch(size) : size * ROW; }
};

// A chunk's 16 bytes, loaded from where they all lie in the operand (which has at least that many), up to E - 1 elements before the chunk's
// place at the operand's end; and what of it counts, moved into place.  The loads have no branch around them: one would wait for each.
template <typename T>
struct Chunk {
  uint32_t w[4];
};
template <typename T>
__device__ __forceinline__ void keep(Chunk<T>& c, int shift, int n) {
  if constexpr (sizeof(T) == 4) {
    if (shift & 2) c.w[0] = c.w[2], c.w[1] = c.w[3];
    if (shift & 1) c.w[0] = c.w[1], c.w[1] = c.w[2], c.w[2] = c.w[3];
#pragma unroll
    for (int e = 0; e < 4; ++e) c.w[e] = e < n ? c.w[e] : 0;
  } else {
    if (shift & 4) c.w[0] = c.w[2], c.w[1] = c.w[3];
    if (shift & 2) c.w[0] = c.w[1], c.w[1] = c.w[2], c.w[2] = c.w[3];
    if (shift & 1) {
#pragma unroll
      for (int e = 0; e < 3; ++e) c.w[e] = c.w[e] >> 16 | c.w[e + 1] << 16;
      c.w[3] >>= 16;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) c.w[e] = n >= 2 * e + 2 ? c.w[e] : n == 2 * e + 1 ? c.w[e] & 0xffffu : 0;
  }
}

template <typename T, int BM, int BN, int WGM, int WGN, bool ACOL, bool BCOL>
constexpr size_t mat_any_bytes() {
  const size_t strips = (size_t)WGM * WGN * strip_floats<BM / WGM / 16, BN / WGN / 16>() * 4;
  const size_t tiles = 2 * (size_t)(Any<T>::elems(ACOL, BM) + Any<T>::elems(BCOL, BN)) * sizeof(T);
  return strips > tiles ? strips : tiles;
}

template <int BM, int BN, int WGM, int WGN, bool ACOL, bool BCOL, class EPI>
__global__ __launch_bounds__(WGM* WGN * 64) void matmul_any(MatArgs p) {
  typedef typename EPI::type T;
  typedef Any<T> S;
  constexpr int NT = WGM * WGN * 64, K = S::K, E = S::E, KC = S::KC;
  constexpr int TM = BM / WGM, TN = BN / WGN, MB = TM / 16, NB = TN / 16;
  constexpr int A_N = BM * KC / NT, B_N = BN * KC / NT;                      // chunks per thread and step
  constexpr int A_ELEMS = S::elems(ACOL, BM), STAGE = A_ELEMS + S::elems(BCOL, BN);
  static_assert(BM * KC % NT == 0 && BN * KC % NT == 0, "every thread loads");
  extern __shared__ __attribute__((aligned(16))) char any_smem[];
  T* const tiles = reinterpret_cast<T*>(any_smem);

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WGN, wn = wave % WGN, r16 = lane & 15, kq = lane >> 4;
  TileAt at;
  constexpr int BNO = EPI::DUAL ? BN / 2 : BN;
  if (!find_tile(p, (p.m + BM - 1) / BM, (p.n + BNO - 1) / BNO, &at)) return;
  const int z = at.z;
  const int row_first = at.mt * BM, col_first = at.nt * BNO;
  const int seg_steps = (p.k + K - 1) / K;
  const int all = EPI::SEGMENTS ? 2 * seg_steps : seg_steps;
  const int per = at.slot < 0 ? all : (all + p.k_split - 1) / p.k_split;
  const int k_begin = min(at.part * per, all), k_end = min(k_begin + per, all);

  static_assert(!EPI::DUAL || BN * KC / 2 % NT == 0, "a thread's chunk is of one of the two");
  Chunk<T> ra[2][A_N], rb[2][B_N];
  // An operand's step: by columns its chunk c is K row c / (size / E) and E columns of it, by rows row c / KC and E of its K.  `off`: the
  // chunk from the step's place on; `last`: where the operand's last 16 bytes begin from there (before it, where a step ends with the operand).
  struct Place {
    int64_t at;
    int last;
  };
  auto place_of = [&](auto col_tag, int64_t ld, int first, int there, int k_there, int k0) {
    constexpr bool COL = decltype(col_tag)::value;
    const int64_t at = COL ? k0 * ld + first : first * ld + k0, total = COL ? (k_there - 1) * ld + there : (there - 1) * ld + k_there;
    return Place{at, (int)min(total - E - at, (int64_t)0x3fffffff)};
  };
  auto off_of = [&](auto col_tag, int c, int size, int64_t ld) {
    return decltype(col_tag)::value ? c / (size / E) * (int)ld + c % (size / E) * E : c / KC * (int)ld + c % KC * E;
  };
  auto fetch = [&](const T* base, int off, const Place& at) {
    const Bytes16<T> b = *reinterpret_cast<const Bytes16<T>*>(base + at.at + min(off, at.last));
    return Chunk<T>{{b.w[0], b.w[1], b.w[2], b.w[3]}};
  };
  auto k_of = [&](int s, bool* second) {
    *second = EPI::SEGMENTS && s >= seg_steps;
    return (*second ? s - seg_steps : s) * K;
  };
  auto load = [&](int s, int set) {
    if (s >= k_end) return;
    bool second;
    const int k0 = k_of(s, &second);
    const T* a = static_cast<const T*>(second ? p.a2 : p.a);
    const T* b = static_cast<const T*>(second || (EPI::PAIRED && z) ? p.b2 : p.b);
    const Place pa = place_of(std::bool_constant<ACOL>{}, p.lda, row_first, p.m_a, p.k, k0), pb = place_of(std::bool_constant<BCOL>{}, p.ldb, col_first, p.n_b, p.k_b, k0);
#pragma unroll
    for (int i = 0; i < A_N; ++i) ra[set][i] = fetch(a, off_of(std::bool_constant<ACOL>{}, tid + i * NT, BM, p.lda), pa);
#pragma unroll
    for (int i = 0; i < B_N; ++i) {
      const bool up = EPI::DUAL && i * NT >= BN * KC / 2;    // DUAL: the first half of the chunks from B, the second from B2, the same columns of both
      rb[set][i] = fetch(up ? static_cast<const T*>(p.b2) : b, off_of(std::bool_constant<BCOL>{}, tid + (up ? i * NT - BN * KC / 2 : i * NT), BNO, p.ldb), pb);
    }
  };
  auto place = [&](auto col_tag, Chunk<T> v, int c, int size, int pitch, int64_t ld, const Place& at, int left, int k_left, T* to) {
    constexpr bool COL = decltype(col_tag)::value;
    const int r = COL ? c / (size / E) : c / KC, e = COL ? c % (size / E) * E : c % KC * E;
    if (left < size || k_left < K) {                         // (uniform) the step reaches past the operand: what of the chunk counts
      const int off = r * (int)ld + e;
      keep(v, max(off - at.last, 0), r < (COL ? k_left : left) ? (COL ? left : k_left) - e : 0);
    }
    *reinterpret_cast<Chunk<T>*>(__builtin_assume_aligned(to + (COL ? r * pitch + e : r * S::ROW + e), 16)) = v;
  };
  auto store = [&](int s, int buf, int set) {
    T* ta = tiles + buf * STAGE;
    T* tb = ta + A_ELEMS;
    bool second;
    const int k0 = k_of(s, &second);
    const Place pa = place_of(std::bool_constant<ACOL>{}, p.lda, row_first, p.m_a, p.k, k0), pb = place_of(std::bool_constant<BCOL>{}, p.ldb, col_first, p.n_b, p.k_b, k0);
#pragma unroll
    for (int i = 0; i < A_N; ++i) place(std::bool_constant<ACOL>{}, ra[set][i], tid + i * NT, BM, S::pitch(BM), p.lda, pa, p.m_a - row_first, p.k - k0, ta);
#pragma unroll
    for (int i = 0; i < B_N; ++i) {
      const bool up = EPI::DUAL && i * NT >= BN * KC / 2;
      place(std::bool_constant<BCOL>{}, rb[set][i], tid + (up ? i * NT - BN * KC / 2 : i * NT), BNO, S::pitch(BN), p.ldb, pb, p.n_b - col_first, p.k_b - k0,
            up ? tb + (BCOL ? BNO : BNO * S::ROW) : tb);
    }
  };
  auto b_first = [&](int nb) {                               // first column, in the tile, of a wave's block
    if (!EPI::DUAL) return wn * TN + nb * 16;
    return (nb / (NB / 2)) * BNO + wn * (TN / 2) + nb % (NB / 2) * 16;
  };

  floatx4_t acc[MB][NB];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) acc[mb][nb] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
  auto multiply = [&](int buf) {
    const T* ta = tiles + buf * STAGE;
    const T* tb = ta + A_ELEMS;
    if constexpr (sizeof(T) == 4) {
      // 16 of K at a time: MFMA i takes K 4 kq + i of both operands
      auto four = [&](auto col_tag, const T* t, int first, int pitch, int k) {
        floatx4_t v;
        if constexpr (decltype(col_tag)::value) {
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = t[(k + kq * 4 + i) * pitch + first + r16];
        } else {
          v = *reinterpret_cast<const floatx4_t*>(t + (first + r16) * S::ROW + k + kq * 4);
        }
        return v;
      };
#pragma unroll
      for (int k = 0; k < K; k += 16) {
        floatx4_t fa[MB], fb[NB];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) fa[mb] = four(std::bool_constant<ACOL>{}, ta, wm * TM + mb * 16, S::pitch(BM), k);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) fb[nb] = four(std::bool_constant<BCOL>{}, tb, b_first(nb), S::pitch(BN), k);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) acc[mb][nb] = __builtin_amdgcn_mfma_f32_16x16x4f32(fb[nb][i], fa[mb][i], acc[mb][nb], 0, 0, 0);
      }
    } else {
      auto eight = [&](auto col_tag, const T* t, int first, int pitch, int k) {
        if constexpr (decltype(col_tag)::value) return read_turned2(t + (k + kq * 8 + (r16 >> 2)) * pitch + first + (r16 & 3) * 4, 4 * pitch);
        else return *reinterpret_cast<const bf16x8_t*>(t + (first + r16) * S::ROW + k + kq * 8);
      };
#pragma unroll
      for (int k = 0; k < K; k += 32) {
        bf16x8_t fa[MB], fb[NB];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) fa[mb] = eight(std::bool_constant<ACOL>{}, ta, wm * TM + mb * 16, S::pitch(BM), k);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) fb[nb] = eight(std::bool_constant<BCOL>{}, tb, b_first(nb), S::pitch(BN), k);
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) acc[mb][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[nb], fa[mb], acc[mb][nb], 0, 0, 0);
      }
    }
  };
  // sums of at most 512 K (fp32: 128 MFMAs) in one chain, added up beside
  constexpr int CHAIN = 512 / K;
  floatx4_t beside[MB][NB] = {};
  load(k_begin, 0);
  load(k_begin + 1, 1);
  for (int s = k_begin; s < k_end; s += 2) {
    if (s > k_begin && (s - k_begin) % CHAIN == 0) {
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          beside[mb][nb] += acc[mb][nb];
          acc[mb][nb] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }
    store(s, 0, 0);
    __syncthreads();                                         // (a buffer's reads lie before the barrier of the step between)
    load(s + 2, 0);
    multiply(0);
    if (s + 1 < k_end) {
      store(s + 1, 1, 1);
      __syncthreads();
      load(s + 3, 1);
      multiply(1);
    }
  }
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) acc[mb][nb] += beside[mb][nb];
  const int64_t row0 = row_first + wm * TM;
  if (EPI::RANGES && at.slot < 0) {
    put_ranges<typename EPI::type>(p, acc, row0, col_first + wn * TN, at.nt * WGN + wn);
  } else {
    __syncthreads();
    put_tile<MB, NB, EPI>(p, acc, reinterpret_cast<float*>(any_smem) + wave * strip_floats<MB, NB>(), at, wm * TM, wn * (EPI::DUAL ? TN / 2 : TN), row0,
                          col_first + wn * (EPI::DUAL ? TN / 2 : TN));
  }
}

}  // namespace cmoe
