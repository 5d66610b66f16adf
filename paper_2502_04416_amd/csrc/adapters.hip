// Low-rank adapters of many requests beside a shared projection, forward and backward.  Token t has adapter k = ids[t]:
//   u = A_k drop(x)                     [rank], fp32
//   y = base + scale_k * B_k u
//   v = scale_k * B_k^T dy              [rank], fp32
//   dx = dx_base + drop's mask and scale on A_k^T v
//   dA_k = sum over its tokens of v drop(x)^T,   dB_k = scale_k * sum over its tokens of dy u^T
// The batches are read and written once and the adapters are small beside them, so all of it is bound by memory; the products run
// on the matrix cores to stay out of the way, bf16 ones with factors kept in fp32 (u, v) entering as two or three bf16 terms.
#include <hip/hip_runtime.h>
#include <algorithm>

#include "../../include/cmoe.h"
#include "cmoe_internal.h"
#include "dropout_device.h"
#include "operator_args.h"

namespace cmoe {

constexpr int MAX_RANK = 64;
constexpr int MAX_ADAPTERS = 12287;      // a wave's counts of them fit LDS

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// ---- operands of the matrix instructions ---------------------------------------------------------------------------
// Eight consecutive values along the contracted axis of one row: lane l holds row l & 15, values (l >> 4) * 8 on.  A product of
// two operands leaves column l & 15 (of the second) and rows (l >> 4) * 4 + i (of the first) in lane l.
template <typename T> struct Frag;
template <> struct Frag<bf16_t> { uint32_t w[4]; };
template <> struct Frag<float> { float w[8]; };

__device__ __forceinline__ void mma(f32x4& acc, const Frag<bf16_t>& rows, const Frag<bf16_t>& cols) {
  acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, rows), __builtin_bit_cast(bf16x8, cols), acc, 0, 0, 0);
}
// (eight steps of four: both operands number the contracted axis alike, so its order is free)
__device__ __forceinline__ void mma(f32x4& acc, const Frag<float>& rows, const Frag<float>& cols) {
#pragma unroll
  for (int j = 0; j < 8; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(rows.w[j], cols.w[j], acc, 0, 0, 0);
}

__device__ __forceinline__ Frag<bf16_t> load_frag(const bf16_t* p) {
  return __builtin_bit_cast(Frag<bf16_t>, *reinterpret_cast<const Bytes16<bf16_t>*>(p));
}
__device__ __forceinline__ Frag<float> load_frag(const float* p) {
  Frag<float> f;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const Bytes16<float> b = *reinterpret_cast<const Bytes16<float>*>(p + 4 * h);
#pragma unroll
    for (int e = 0; e < 4; ++e) f.w[4 * h + e] = __uint_as_float(b.w[e]);
  }
  return f;
}
// The first n values (none if n <= 0), then zeros.
__device__ __forceinline__ Frag<bf16_t> load_frag(const bf16_t* p, int n) {
  if (n >= 8) return load_frag(p);
  Frag<bf16_t> f;
#pragma unroll
  for (int e = 0; e < 4; ++e) f.w[e] = (2 * e < n ? (uint32_t)p[2 * e] : 0u) | (2 * e + 1 < n ? (uint32_t)p[2 * e + 1] << 16 : 0u);
  return f;
}
__device__ __forceinline__ Frag<float> load_frag(const float* p, int n) {
  if (n >= 8) return load_frag(p);
  Frag<float> f;
#pragma unroll
  for (int e = 0; e < 8; ++e) f.w[e] = e < n ? p[e] : 0.0f;
  return f;
}

// What dropout drops becomes 0 (its scale is applied to the products in fp32, so that bf16 values stay as they are).
__device__ __forceinline__ void mask_frag(Frag<bf16_t>& f, const Drop& d, const uint4& words) {
#pragma unroll
  for (int e = 0; e < 4; ++e) f.w[e] &= (drop_keeps(d, words, 2 * e) ? 0xffffu : 0u) | (drop_keeps(d, words, 2 * e + 1) ? 0xffff0000u : 0u);
}
__device__ __forceinline__ void mask_frag(Frag<float>& f, const Drop& d, const uint4& words) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f.w[e] = drop_keeps(d, words, e) ? f.w[e] : 0.0f;
}

// Eight rows of eight values to eight columns.
__device__ __forceinline__ void transpose(const Frag<bf16_t> (&rows)[8], Frag<bf16_t> (&cols)[8]) {
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      cols[2 * d].w[a] = __builtin_amdgcn_perm(rows[2 * a + 1].w[d], rows[2 * a].w[d], 0x05040100u);
      cols[2 * d + 1].w[a] = __builtin_amdgcn_perm(rows[2 * a + 1].w[d], rows[2 * a].w[d], 0x07060302u);
    }
}
__device__ __forceinline__ void transpose(const Frag<float> (&rows)[8], Frag<float> (&cols)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e)
#pragma unroll
    for (int j = 0; j < 8; ++j) cols[e].w[j] = rows[j].w[e];
}

// fp32 values as a sum of operands.  bf16: the upper eight bits of the significand, then those of what is left, the last term
// rounded: two terms carry 16 bits (outputs that are themselves rounded to bf16), three all 24 (gradients of the weights, which
// stay fp32).  What is left of an infinity would be NaN: 0.  fp32 needs one term.
template <typename T> struct Terms { static constexpr int OUTPUT = 1, GRADIENT = 1; };
template <> struct Terms<bf16_t> { static constexpr int OUTPUT = 2, GRADIENT = 3; };

template <int N>
__device__ __forceinline__ void split(const float (&v)[8], Frag<bf16_t> (&f)[N]) {
  float rest[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) rest[e] = v[e];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (i < N - 1) {
#pragma unroll
      for (int e = 0; e < 4; ++e) f[i].w[e] = __builtin_amdgcn_perm(__float_as_uint(rest[2 * e + 1]), __float_as_uint(rest[2 * e]), 0x07060302u);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float left = rest[e] - __uint_as_float(__float_as_uint(rest[e]) & 0xffff0000u);
        rest[e] = left == left ? left : 0.0f;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) f[i].w[e] = (uint32_t)f32_to_bf16(rest[2 * e]) | ((uint32_t)f32_to_bf16(rest[2 * e + 1]) << 16);
    }
  }
}
__device__ __forceinline__ void split(const float (&v)[8], Frag<float> (&f)[1]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f[0].w[e] = v[e];
}

__device__ __forceinline__ void unpack(const Frag<bf16_t>& f, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[2 * e] = __uint_as_float(f.w[e] << 16);
    v[2 * e + 1] = __uint_as_float(f.w[e] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack(const Frag<float>& f, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = f.w[e];
}

// The adapter of a token, or -1.
__device__ __forceinline__ int adapter_of(const int32_t* ids, int64_t t, int n_adapters) {
  const int k = ids ? ids[t] : 0;
  return k >= 0 && k < n_adapters ? k : -1;
}

// ---- u and y -------------------------------------------------------------------------------------------------------

template <typename T>
struct TileArgs {
  const T* x;             // [tokens, d_in]
  const T* a;             // [n][rank][d_in]
  const T* b;             // [n][d_out][rank]
  const float* scale;
  const int32_t* ids;
  const T* base;          // or null
  T* y;
  float* u;               // or null
  int64_t tokens;
  int d_in, d_out, rank, n_adapters;
  int slices;             // workgroups that share a tile, each with its part of the columns of y
  Drop drop;
};

constexpr int SCAN_TOKENS = 512;         // a workgroup of the scanning form looks at one id per thread

// A tile is 16 tokens.  Its workgroup first contracts x with the adapter's rows: the waves take turns along the width, 64 values at a
// time, and their sums meet in LDS; then each wave expands u to its own columns, on to base, straight from memory to memory.
// SCAN: workgroup b is for the adapter of token b, if b is the first of its adapter's tokens or the 16th, 32nd ... after it; it finds
// up to 16 of them itself.  Weights are then read once per 16 tokens of an adapter whatever the order, as decode batches need it,
// where every token may have another.  Otherwise 16 consecutive tokens, and one pass for each adapter among them: prompts and
// training batches come as runs, so that most tiles have one.
// Without EXPAND: u * scale alone (v of the backward pass).
template <typename T, int R16, bool SCAN, bool EXPAND>
__global__ __launch_bounds__(R16 == 4 ? 512 : 1024) void tile_kernel(TileArgs<T> g) {
  constexpr int WAVES = R16 == 4 ? 8 : 16;
  constexpr int CHUNKS = (R16 + 1) / 2;                      // operands along the rank
  constexpr int NT = Terms<T>::OUTPUT;
  constexpr int LD = R16 * 16 + 4;
  __shared__ float sums[WAVES][R16 * 4 * 64];
  __shared__ float us[16][LD];
  __shared__ int token[16], id[16], found[16], counts[2][16], n_found;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, m = lane & 15, q = lane >> 4;
  if (SCAN) {
    const int me = blockIdx.x;
    const int k = adapter_of(g.ids, me, g.n_adapters);
    if (tid < 16) {
      token[tid] = me;
      id[tid] = tid == 0 ? k : -2;
    }
    const bool mine = tid < g.tokens && k >= 0 && adapter_of(g.ids, tid, g.n_adapters) == k;
    const uint64_t votes = __ballot(mine);
    if (lane == 0) counts[0][wave] = __popcll(votes);
    __syncthreads();
    int before = 0, before_me = 0;                           // of this thread, of the workgroup's token
    for (int w = 0; w < wave; ++w) before += counts[0][w];
    before += __popcll(votes & ((1ull << lane) - 1));
    if (tid == me) counts[1][0] = before;
    __syncthreads();
    before_me = counts[1][0];
    if (k >= 0) {
      if (before_me & 15) return;
      if (mine && tid >= me && before - before_me < 16) {
        token[before - before_me] = tid;
        id[before - before_me] = k;
      }
    }
    if (tid == 0) {
      found[0] = k;
      n_found = k >= 0;
    }
  } else if (tid < 64) {
    const int64_t t = (int64_t)blockIdx.x * 16 + m;
    const bool valid = t < g.tokens;
    const int k = valid ? adapter_of(g.ids, t, g.n_adapters) : -2;
    bool first = k >= 0 && lane < 16;
#pragma unroll
    for (int i = 0; i < 15; ++i) {
      const int other = __shfl(k, i, 64);                    // (by all lanes, before the comparison)
      first = first && !(i < m && other == k);
    }
    const uint64_t votes = __ballot(first);
    if (lane < 16) {
      token[m] = valid ? m : 0;
      id[m] = k;
    }
    if (first) found[__popcll(votes & ((1ull << lane) - 1))] = k;
    if (lane == 0) n_found = __popcll(votes);
  }
  for (int i = tid; i < 16 * LD; i += WAVES * 64) (&us[0][0])[i] = 0.0f;
  __syncthreads();
  const int64_t t0 = SCAN ? 0 : (int64_t)blockIdx.x * 16;
  const int64_t my_token = t0 + token[m];
  const int my_id = id[m], n_distinct = n_found;

  // u: rows are tokens, columns are the rank.  A row or column that is none reads another's values, and its results are not used.
  for (int f = 0; f < n_distinct; ++f) {
    const int k = found[f];
    const T* x = g.x + my_token * g.d_in + q * 8;
    const T* a[R16];
#pragma unroll
    for (int r = 0; r < R16; ++r) a[r] = g.a + ((int64_t)k * g.rank + min(r * 16 + m, g.rank - 1)) * g.d_in + q * 8;
    const int per_row = (g.d_in + 7) >> 3;
    const uint64_t chunk0 = (uint64_t)my_token * per_row + q;
    f32x4 acc[R16];
#pragma unroll
    for (int r = 0; r < R16; ++r) acc[r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int full = g.d_in / 64;
    constexpr int DEPTH = R16 == 1 ? 4 : 2;                  // turns whose loads are in flight together
    int s = wave;
    for (; s + (DEPTH - 1) * WAVES < full; s += DEPTH * WAVES) {
      Frag<T> xf[DEPTH][2], af[DEPTH][2][R16];
#pragma unroll
      for (int i = 0; i < DEPTH; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int at = (s + i * WAVES) * 64 + h * 32;
          xf[i][h] = load_frag(x + at);
#pragma unroll
          for (int r = 0; r < R16; ++r) af[i][h][r] = load_frag(a[r] + at);
        }
#pragma unroll
      for (int i = 0; i < DEPTH; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (g.drop.limit) mask_frag(xf[i][h], g.drop, philox_words(g.drop, chunk0 + (s + i * WAVES) * 8 + h * 4));
#pragma unroll
          for (int r = 0; r < R16; ++r) mma(acc[r], xf[i][h], af[i][h][r]);
        }
    }
    for (; s * 64 < g.d_in; s += WAVES) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int at = s * 64 + h * 32, n = g.d_in - at - q * 8;
        Frag<T> xf = load_frag(x + at, n);
        if (g.drop.limit) mask_frag(xf, g.drop, philox_words(g.drop, chunk0 + s * 8 + h * 4));
#pragma unroll
        for (int r = 0; r < R16; ++r) mma(acc[r], xf, load_frag(a[r] + at, n));
      }
    }
#pragma unroll
    for (int r = 0; r < R16; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) sums[wave][(r * 4 + i) * 64 + lane] = acc[r][i];
    __syncthreads();
    for (int v = tid; v < R16 * 256; v += WAVES * 64) {
      const int l = v & 63, row = (l >> 4) * 4 + ((v >> 6) & 3), col = (v >> 8) * 16 + (l & 15);
      float t = sums[0][v];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) t += sums[w][v];
      if (g.drop.limit) t *= g.drop.scale;
      if (id[row] == k && col < g.rank) us[row][col] = t;
    }
    __syncthreads();
  }

  if (g.u && blockIdx.y == 0)
    for (int v = tid; v < 16 * g.rank; v += WAVES * 64) {
      const int row = v / g.rank, col = v % g.rank;
      if (id[row] > -2) g.u[(t0 + token[row]) * g.rank + col] = EXPAND ? us[row][col] : (id[row] >= 0 ? us[row][col] * g.scale[id[row]] : 0.0f);
    }
  if (!EXPAND) return;

  // y: rows are 16 columns of y, columns are tokens.  Two products' rows are dealt so that a lane ends with eight consecutive
  // columns of its token.  The contracted axis is the rank in chunks of eight; the last chunk of a rank that is no multiple
  // of eight reaches back, with zeros in u where it overlaps.
  const int units = (g.d_out + 31) >> 5;
  const int first = (int)((int64_t)units * blockIdx.y / g.slices), last = (int)((int64_t)units * (blockIdx.y + 1) / g.slices);
  const int chunks = (g.rank + 7) >> 3;
  Frag<T> uf[CHUNKS][NT];
  int have = -1;
  for (int unit = first + wave; unit < last; unit += WAVES) {
    const int o0 = unit * 32;
    const int64_t at = my_token * g.d_out + o0 + q * 8;
    const int n = g.d_out - o0 - q * 8;
    float v[8] = {};
    if (g.base && n > 0) load8(g.base + at, n, v);
    for (int f = 0; f < n_distinct; ++f) {
      const int k = found[f];
      f32x4 acc[2] = {f32x4{0.0f, 0.0f, 0.0f, 0.0f}, f32x4{0.0f, 0.0f, 0.0f, 0.0f}};
      Frag<T> bf[2][CHUNKS];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int o = min(o0 + (m >> 2) * 8 + e * 4 + (m & 3), g.d_out - 1);
        const T* row = g.b + ((int64_t)k * g.d_out + o) * g.rank;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
          bf[e][c] = g.rank >= 8 ? load_frag(row + min((c * 4 + q) * 8, g.rank - 8)) : load_frag(row, c * 4 + q == 0 ? g.rank : 0);
      }
      if (have != f) {
        have = f;
        const float scale = g.scale[k];
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
          const int chunk = c * 4 + q, from = max(min(chunk * 8, g.rank - 8), 0);
          float t[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) t[j] = chunk < chunks && from + j >= chunk * 8 && my_id == k ? us[m][from + j] * scale : 0.0f;
          split(t, uf[c]);
        }
      }
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int p = 0; p < NT; ++p)
#pragma unroll
          for (int e = 0; e < 2; ++e) mma(acc[e], bf[e][c], uf[c][p]);
      // (added by choice, not as a product with 0: a token does not see what another's adapter holds)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += my_id == k ? acc[e >> 2][e & 3] : 0.0f;
    }
    if (my_id == -2 || n <= 0) continue;
    store8(g.y + at, n, v);
  }
}

// ---- backward: order of the tokens, b transposed -------------------------------------------------------------------

// order: the tokens by adapter, in their order within one, those without an adapter last; start[k]: adapter k's first place, start[n]:
// that of the tokens without one, start[n + 1] = tokens.  One workgroup; each wave counts and places a range of tokens of its own.
__global__ __launch_bounds__(1024) void order_kernel(const int32_t* ids, int tokens, int n_adapters, int32_t* order, int32_t* start) {
  extern __shared__ int32_t cursor[];                        // [wave][n + 1]
  __shared__ int32_t totals[1024], carry;
  const int n_waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, bins = n_adapters + 1;
  for (int i = threadIdx.x; i < n_waves * bins; i += blockDim.x) cursor[i] = 0;
  if (threadIdx.x == 0) carry = 0;
  __syncthreads();
  const int per = (((tokens + n_waves - 1) / n_waves) + 63) & ~63;
  const int first = min(wave * per, tokens), last = min(first + per, tokens);
  volatile int32_t* mine = cursor + wave * bins;             // (written by one lane, read by others of its wave)
  auto bin_of = [&](int t) {
    const int k = adapter_of(ids, t, n_adapters);
    return k < 0 ? n_adapters : k;
  };
  // f(place among the wave's lanes with this bin, how many, bin) once per lane that holds a token
  auto by_bin = [&](int t, auto f) {
    const int bin = t < last ? bin_of(t) : -1;
    uint64_t left = __ballot(bin >= 0);
    while (left) {
      const int b = __builtin_amdgcn_readlane(bin, __ffsll((unsigned long long)left) - 1);
      const uint64_t same = __ballot(bin == b);
      if (bin == b) f(__popcll(same & ((1ull << lane) - 1)), __popcll(same), b);
      left &= ~same;
    }
  };
  for (int t = first + lane; t - lane < last; t += 64)
    by_bin(t, [&](int place, int n, int b) {
      if (place == 0) mine[b] = mine[b] + n;
    });
  __syncthreads();
  for (int b0 = 0; b0 < bins; b0 += blockDim.x) {
    const int b = b0 + threadIdx.x;
    int total = 0;
    if (b < bins)
      for (int w = 0; w < n_waves; ++w) total += cursor[w * bins + b];
    const int upto = wave_incl_scan(total);
    if (lane == 63) totals[wave] = upto;
    __syncthreads();
    int at = carry + upto - total;
    for (int w = 0; w < wave; ++w) at += totals[w];
    __syncthreads();
    if (threadIdx.x == blockDim.x - 1) carry = at + total;
    if (b < bins) {
      start[b] = at;
      for (int w = 0; w < n_waves; ++w) {
        const int n = cursor[w * bins + b];
        cursor[w * bins + b] = at;
        at += n;
      }
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) start[bins] = tokens;
  for (int t = first + lane; t - lane < last; t += 64)
    by_bin(t, [&](int place, int n, int b) {
      const int at = mine[b];
      order[at + place] = t;
      if (place == 0) mine[b] = at + n;
    });
}

// bt[k][j][o] = b[k][o][j]: 64 columns o of one adapter per workgroup, through LDS.
template <typename T>
__global__ __launch_bounds__(256) void transpose_kernel(const T* b, T* bt, int d_out, int rank) {
  __shared__ T tile[MAX_RANK][64 + 2];
  const int k = blockIdx.y, o0 = blockIdx.x * 64, n = min(64, d_out - o0);
  const T* from = b + ((int64_t)k * d_out + o0) * rank;
  for (int i = threadIdx.x; i < n * rank; i += 256) tile[i % rank][i / rank] = from[i];
  __syncthreads();
  for (int i = threadIdx.x; i < rank * 64; i += 256)
    if ((i & 63) < n) bt[((int64_t)k * rank + (i >> 6)) * d_out + o0 + (i & 63)] = tile[i >> 6][i & 63];
}

// ---- backward: dx and the gradients of the weights -----------------------------------------------------------------

template <typename T>
struct OuterArgs {
  const T* x;             // [tokens, d]: x for da and dx, dy for db
  const float* v;         // [tokens, rank]: v, or u
  const T* a;             // dx: [n][rank][d]
  const T* base;          // dx_base or null
  T* dx;
  float* partials;        // [slot][rank][d]
  const int32_t* order;
  const int32_t* start;
  int tokens, d, rank, n_adapters;
  int chunk;              // places of the order per workgroup
  Drop drop;
};

// A workgroup has 128 columns and a chunk of the places in the order of adapters; its four waves take turns of 32 tokens.  A lane reads
// eight columns of eight tokens and turns them in its registers into eight operands whose contracted axis is the tokens: operand e's
// row m is column 8 m + e.  So nothing goes through LDS, every load and store is 16 bytes of a row, and the columns that a lane reads
// of a token are those that it writes of dx: one evaluation of the mask serves both.  The sums over tokens of an adapter within the
// chunk go to a slot of their own (slots are numbered chunk + adapter: of two slots in the order one number differs), and
// are added in the order of chunks by the kernel below.
template <typename T, int R16, bool DX, bool GRAD>
__global__ __launch_bounds__(256) void outer_kernel(OuterArgs<T> g) {
  constexpr int CHUNKS = (R16 + 1) / 2;
  constexpr int NT = Terms<T>::OUTPUT, NG = Terms<T>::GRADIENT;
  __shared__ float sums[GRAD ? 3 * 64 * 32 : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, q = lane >> 4;
  const int c0 = blockIdx.x * 128 + m * 8;                   // the lane's columns
  const int n = g.d - c0;
  const int per_row = (g.d + 7) >> 3;
  const int chunk0 = blockIdx.y * g.chunk, chunk1 = min(chunk0 + g.chunk, g.tokens);
  const int chunks = (g.rank + 7) >> 3;
  // the adapter of the chunk's first place: the last one that starts at or before it (empty ones start where the next does)
  int k = 0;
  {
    int hi = g.n_adapters;                                   // start[n_adapters]: tokens without an adapter
    while (k < hi) {
      const int mid = (k + hi + 1) >> 1;
      if (g.start[mid] <= chunk0) k = mid;
      else hi = mid - 1;
    }
  }
  for (int p0 = chunk0; p0 < chunk1; ++k) {
    const int p1 = min(g.start[k + 1], chunk1);
    if (p1 <= p0) continue;
    const bool none = k == g.n_adapters;
    if (none && !DX) return;
    f32x4 acc[GRAD ? R16 : 1][8];
    Frag<T> af[DX ? CHUNKS : 1][8];
    if (GRAD) {
#pragma unroll
      for (int r = 0; r < R16; ++r)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[r][e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    if (DX && !none) {
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) {
        Frag<T> rows[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int r = (c * 4 + q) * 8 + j;
          rows[j] = load_frag(g.a + ((int64_t)k * g.rank + min(r, g.rank - 1)) * g.d + c0, r < g.rank ? n : 0);
        }
        transpose(rows, af[c]);
      }
    }
    for (int p = p0 + wave * 32; p < p1; p += 128) {
      int64_t t[8];                                          // places q * 4 + 0..3 and 16 + q * 4 + 0..3; a place past the end: none
      bool valid[8];
      Frag<T> rows[8], base[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int at = p + (j >> 2) * 16 + q * 4 + (j & 3);
        valid[j] = at < p1;
        t[j] = g.order[min(at, p1 - 1)];
      }
      if (GRAD || DX) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (GRAD) rows[j] = load_frag(g.x + t[j] * g.d + c0, valid[j] && !none ? n : 0);
          if (DX) base[j] = load_frag((g.base ? g.base : g.a) + (g.base ? t[j] * g.d + c0 : 0), g.base && valid[j] ? n : 0);
        }
      }
      uint4 words[8];
      if (g.drop.limit) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          words[j] = philox_words(g.drop, (uint64_t)t[j] * per_row + (c0 >> 3));
          if (GRAD) mask_frag(rows[j], g.drop, words[j]);
        }
      }
      if (GRAD && !none) {
        Frag<T> cols[8];
        transpose(rows, cols);
#pragma unroll
        for (int r = 0; r < R16; ++r) {
          float f[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j] = valid[j] && r * 16 + m < g.rank ? g.v[t[j] * g.rank + r * 16 + m] : 0.0f;
          Frag<T> vf[NG];
          split(f, vf);
#pragma unroll
          for (int i = 0; i < NG; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) mma(acc[r][e], cols[e], vf[i]);
        }
      }
      if (DX) {
        f32x4 out[2][8];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int e = 0; e < 8; ++e) out[s][e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (!none) {
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const int at = p + s * 16 + m;
            const int64_t row = (int64_t)g.order[min(at, p1 - 1)] * g.rank;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
              float f[8];
              Frag<T> vf[NT];
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                const int r = (c * 4 + q) * 8 + j;
                f[j] = r < g.rank ? g.v[row + r] : 0.0f;
              }
              split(f, vf);
#pragma unroll
              for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) mma(out[s][e], vf[i], af[c][e]);
            }
          }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (!valid[j] || n <= 0) continue;
          float o[8], b[8];
          unpack(base[j], b);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float d = out[j >> 2][e][j & 3];
            if (g.drop.limit) d = drop_keeps(g.drop, words[j], e) ? d * g.drop.scale : 0.0f;
            o[e] = none ? b[e] : b[e] + d;
          }
          store8(g.dx + t[j] * g.d + c0, n, o);
        }
      }
    }
    if (GRAD && !none) {
      float* slot = g.partials + (int64_t)(blockIdx.y + k) * g.rank * g.d;
#pragma unroll
      for (int r = 0; r < R16; ++r) {
        __syncthreads();
        if (wave > 0) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[((wave - 1) * 32 + e * 4 + i) * 64 + lane] = acc[r][e][i];
        }
        __syncthreads();
        if (wave == 0 && r * 16 + m < g.rank) {
          // the lane's rank is r * 16 + m; its columns q * 32 + i * 8 + e
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              o[e] = acc[r][e][i] + sums[(e * 4 + i) * 64 + lane] + sums[(32 + e * 4 + i) * 64 + lane] + sums[(64 + e * 4 + i) * 64 + lane];
              if (g.drop.limit) o[e] *= g.drop.scale;
            }
            const int c = blockIdx.x * 128 + q * 32 + i * 8;
            if (c < g.d) store8(slot + (int64_t)(r * 16 + m) * g.d + c, g.d - c, o);
          }
        }
      }
    }
    p0 = p1;
  }
}

// out = the slots of an adapter added in the order of chunks (0 without one), times the adapter's scale if there is one.
// TRANSPOSED: out is [n][d][rank].
__global__ __launch_bounds__(256) void sum_slots_kernel(const float* partials, const int32_t* start, const float* scale, float* out, int d, int rank, int chunk,
                                                        int transposed) {
  const int k = blockIdx.y;
  const int64_t size = (int64_t)rank * d, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= size) return;
  const int p0 = start[k], p1 = start[k + 1];
  float t = 0.0f;
  if (p1 > p0) {
    for (int c = p0 / chunk; c <= (p1 - 1) / chunk; ++c) t += partials[(int64_t)(c + k) * size + i];
    if (scale) t *= scale[k];
  }
  out[k * size + (transposed ? (i % d) * rank + i / d : i)] = t;
}

// f(R16) with the rank in blocks of 16 as a compile-time constant
template <typename F>
static void with_rank(int rank, F&& f) {
  if (rank <= 16) f(std::integral_constant<int, 1>{});
  else if (rank <= 32) f(std::integral_constant<int, 2>{});
  else f(std::integral_constant<int, 4>{});
}

template <typename T, bool EXPAND>
static void launch_tiles(TileArgs<T> g, hipStream_t s) {
  const int units = EXPAND ? (g.d_out + 31) / 32 : 1;
  const bool scan = g.tokens <= SCAN_TOKENS;
  const int64_t tiles = scan ? g.tokens : (g.tokens + 15) / 16;
  g.slices = EXPAND ? (int)std::max<int64_t>(1, std::min<int64_t>(256 / tiles, (units + 15) / 16)) : 1;
  with_rank(g.rank, [&](auto r) {
    constexpr int R = decltype(r)::value;
    const dim3 grid((unsigned)tiles, g.slices), block(R == 4 ? 512 : 1024);
    if (scan) hipLaunchKernelGGL((tile_kernel<T, R, true, EXPAND>), grid, block, 0, s, g);
    else hipLaunchKernelGGL((tile_kernel<T, R, false, EXPAND>), grid, block, 0, s, g);
  });
}

template <typename T>
static void launch_adapters_forward(const cmoe_adapters_forward_args& p, const Drop& drop, hipStream_t s) {
  launch_tiles<T, true>(TileArgs<T>{(const T*)p.x, (const T*)p.a, (const T*)p.b, p.scale, p.ids, (const T*)p.base, (T*)p.y, p.u, p.tokens, p.d_in, p.d_out,
                                    p.rank, p.n_adapters, 1, drop}, s);
}

// Workspace of the backward pass: order and starts, v, b transposed, slots of da's and db's partial sums.
struct BackwardLayout {
  int chunk, chunks;
  size_t order, start, v, bt, da, db, total;
};
static BackwardLayout backward_layout(int64_t tokens, int d_in, int d_out, int rank, int n_adapters, int dtype) {
  BackwardLayout l{};
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t o = off; off = (off + bytes + 255) & ~(size_t)255; return o; };
  l.chunk = 256;
  l.chunks = (int)((tokens + l.chunk - 1) / l.chunk);
  l.order = take(sizeof(int32_t) * tokens);
  l.start = take(sizeof(int32_t) * (n_adapters + 2));
  l.v = take(sizeof(float) * tokens * rank);
  l.bt = take(elem_size(dtype) * n_adapters * rank * d_out);
  l.da = take(sizeof(float) * (l.chunks + n_adapters) * rank * d_in);
  l.db = take(sizeof(float) * (l.chunks + n_adapters) * rank * d_out);
  l.total = off;
  return l;
}

template <typename T>
static void launch_adapters_backward(const cmoe_adapters_backward_args& p, const Drop& drop, hipStream_t s) {
  const BackwardLayout l = backward_layout(p.tokens, p.d_in, p.d_out, p.rank, p.n_adapters, p.dtype);
  char* ws = (char*)p.workspace;
  int32_t *order = (int32_t*)(ws + l.order), *start = (int32_t*)(ws + l.start);
  float *v = (float*)(ws + l.v), *da = (float*)(ws + l.da), *db = (float*)(ws + l.db);
  T* bt = (T*)(ws + l.bt);
  const int n_waves = std::min(16, (MAX_ADAPTERS + 1) / (p.n_adapters + 1));
  hipLaunchKernelGGL(order_kernel, dim3(1), dim3(64 * n_waves), sizeof(int32_t) * n_waves * (p.n_adapters + 1), s, p.ids, (int)p.tokens, p.n_adapters, order, start);
  if (p.tokens > 0 && (p.dx || p.da)) {
    hipLaunchKernelGGL(transpose_kernel<T>, dim3((p.d_out + 63) / 64, p.n_adapters), dim3(256), 0, s, (const T*)p.b, bt, p.d_out, p.rank);
    launch_tiles<T, false>(TileArgs<T>{(const T*)p.dy, bt, nullptr, p.scale, p.ids, nullptr, nullptr, v, p.tokens, p.d_out, 0, p.rank, p.n_adapters, 1, Drop{}}, s);
  }
  with_rank(p.rank, [&](auto r) {
    constexpr int R = decltype(r)::value;
    if (l.chunks > 0 && (p.dx || p.da)) {
      const OuterArgs<T> g{(const T*)p.x, v, (const T*)p.a, (const T*)p.dx_base, (T*)p.dx, da, order, start, (int)p.tokens, p.d_in, p.rank, p.n_adapters, l.chunk, drop};
      const dim3 grid((p.d_in + 127) / 128, l.chunks);
      if (p.dx && p.da) hipLaunchKernelGGL((outer_kernel<T, R, true, true>), grid, dim3(256), 0, s, g);
      else if (p.dx) hipLaunchKernelGGL((outer_kernel<T, R, true, false>), grid, dim3(256), 0, s, g);
      else hipLaunchKernelGGL((outer_kernel<T, R, false, true>), grid, dim3(256), 0, s, g);
    }
    if (l.chunks > 0 && p.db) {
      const OuterArgs<T> g{(const T*)p.dy, p.u, nullptr, nullptr, nullptr, db, order, start, (int)p.tokens, p.d_out, p.rank, p.n_adapters, l.chunk, Drop{}};
      hipLaunchKernelGGL((outer_kernel<T, R, false, true>), dim3((p.d_out + 127) / 128, l.chunks), dim3(256), 0, s, g);
    }
  });
  if (p.da)
    hipLaunchKernelGGL(sum_slots_kernel, dim3((unsigned)(((int64_t)p.rank * p.d_in + 255) / 256), p.n_adapters), dim3(256), 0, s, da, start, (const float*)nullptr, p.da,
                       p.d_in, p.rank, l.chunk, 0);
  if (p.db)
    hipLaunchKernelGGL(sum_slots_kernel, dim3((unsigned)(((int64_t)p.rank * p.d_out + 255) / 256), p.n_adapters), dim3(256), 0, s, db, start, p.scale, p.db, p.d_out,
                       p.rank, l.chunk, 1);
}

static int check_adapters(const char* what, int dtype, int64_t tokens, int d_in, int d_out, int rank, int n_adapters) {
  if (dtype != CMOE_F32 && dtype != CMOE_BF16) return fail(CMOE_EINVAL, "%s: dtype must be CMOE_F32 or CMOE_BF16", what);
  if (d_in < 1 || d_out < 1 || d_in > (1 << 24) || d_out > (1 << 24)) return fail(CMOE_EINVAL, "%s: d_in and d_out must be 1 to 2^24", what);
  if (rank < 1 || rank > MAX_RANK) return fail(CMOE_EINVAL, "%s: rank must be 1 to %d", what, MAX_RANK);
  if (n_adapters < 1 || n_adapters > MAX_ADAPTERS) return fail(CMOE_EINVAL, "%s: n_adapters must be 1 to %d", what, MAX_ADAPTERS);
  if (tokens < 0 || tokens > (1 << 20)) return fail(CMOE_EINVAL, "%s: tokens must be 0 to 2^20", what);
  return CMOE_OK;
}

}  // namespace cmoe

extern "C" size_t cmoe_adapters_forward_workspace_bytes(int64_t tokens, int32_t d_in, int32_t d_out, int32_t rank, int32_t n_adapters, int32_t dtype) {
  using namespace cmoe;
  if (check_adapters("cmoe_adapters_forward_workspace_bytes", dtype, tokens, d_in, d_out, rank, n_adapters)) return 0;
  return 0;
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
  return backward_layout(tokens, d_in, d_out, rank, n_adapters, dtype).total;
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
  if ((p->tokens > 0 || p->da || p->db) && (!p->workspace || p->workspace_bytes < cmoe_adapters_backward_workspace_bytes(p->tokens, p->d_in, p->d_out, p->rank, p->n_adapters, p->dtype)))
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
