// Low-rank adapters of many requests beside a shared projection, forward and backward.  Token t has adapter k = ids[t]:
//   u = A_k drop(x)                     [rank], fp32
//   y = base + scale_k * B_k u
//   v = scale_k * B_k^T dy              [rank], fp32
//   dx = dx_base + drop's mask and scale on A_k^T v
//   dA_k = sum over its tokens of v drop(x)^T,   dB_k = scale_k * sum over its tokens of dy u^T
// The batches are read and written once and the adapters are small beside them, so all of it is bound by memory; the products run
// on the matrix cores to stay out of the way, bf16 ones with factors kept in fp32 (u, v) entering as three bf16 terms.
#include <hip/hip_runtime.h>
#include <algorithm>

#include "../../include/cmoe.h"
#include "cmoe_internal.h"
#include "fragments_device.h"
#include "operator_args.h"

namespace cmoe {

constexpr int MAX_RANK = 64;
constexpr int MAX_WIDTH = 1 << 20;       // of SCAN_TOKENS rows an offset fits 31 bits of bytes
constexpr int MAX_ADAPTERS = 8191;       // a wave's counts of them fit LDS

// The adapter of a token, or -1.
__device__ __forceinline__ int adapter_of(const int32_t* ids, int64_t t, int n_adapters) {
  const int k = ids ? ids[t] : 0;
  return k >= 0 && k < n_adapters ? k : -1;
}

// A value of which the compiler takes nothing for granted: what is computed from it stays where it is used.  (It computes the addresses of
// all loads of a loop ahead of it otherwise, 64 bits of each, and spills them.)
__device__ __forceinline__ int here(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// The number of the wave in the workgroup, known to be the same in its lanes.
__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

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
  float* u;               // [tokens, ldu] or null
  int64_t tokens;
  int d_in, d_out, rank, n_adapters;
  int ldu;                // at least the rank: zeros from there on
  int slices;             // workgroups that share a tile, each with its part of the columns of y
  Drop drop;
};

constexpr int SCAN_TOKENS = 512;         // a workgroup of the scanning form looks at one id per thread

// Waves of a workgroup, and units of 32 columns of y that a wave has in flight at once.
template <int R16, bool SCAN>
constexpr int TILE_WAVES = R16 == 1 || (R16 == 2 && SCAN) ? 16 : 8;
template <typename T, int R16>
constexpr int UNITS_AT_ONCE = R16 == 4 || sizeof(T) == 4 ? 1 : 2;

// A tile is 16 MT tokens.  Its workgroup first contracts x with the adapter's rows: the waves take turns along the width, 64 values each
// time, each a part of its own, and their sums meet in LDS; then each wave expands u to its own columns, on to base, straight from memory to memory.
// SCAN: workgroup b is for the adapter of token b, if b is the first of its adapter's tokens or the 16th, 32nd ... after it; it finds
// up to 16 of them itself.  Weights are then read once per 16 tokens of an adapter whatever the order, as decode batches need it,
// where every token may have another.  Otherwise consecutive tokens, and one pass for each adapter among them, shared by gridDim.z
// workgroups: prompts and training batches come as runs, so that most tiles have one, and the tiles with two are not the last to end.
// A row or column of a product that is no token, rank or column of y reads another's values, and its results are not used: a token
// does not see what another's adapter holds.
// Without EXPAND: u * scale alone (v of the backward pass).
// One launch, since a second costs what the sums of u take to meet.  4096 tokens, 4096 wide, rank 8, bf16 with dropout: 29 us for 101 MB (a
// copy 19), of which the launch is 3, the first latencies 3, and the generator 7 in a part that waits for x meanwhile.  2048 tokens of
// eleven adapters of rank 32: 22.8 us; 64 tokens of 35 adapters, 4096 by 11008, rank 16: 13.9 us for 18 MB; one token 8.9 us.  What bounds
// the small ones is one round trip after another (ids, x and a, b) and the fetching of code that runs once.
template <typename T, int R16, int MT, bool SCAN, bool EXPAND, int EDGE>
__global__ __launch_bounds__((TILE_WAVES<R16, SCAN>) * 64, R16 == 4 ? 2 : 4) void tile_kernel(TileArgs<T> g) {
  constexpr int WAVES = TILE_WAVES<R16, SCAN>, M = 16 * MT;
  constexpr int CHUNKS = (R16 + 1) / 2;                      // operands along the rank
  constexpr int NT = TERMS<T>;
  constexpr int LD = CHUNKS * 32 + 16 / sizeof(T);
  __shared__ float sums[WAVES][MT * R16 * 4 * 64];
  __shared__ __align__(16) T us[EXPAND ? NT : 1][M][LD];    // scale * u, in terms
  __shared__ int token[M], id[M], found[M], counts[2][16], n_found;
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id(), m = lane & 15, q = lane >> 4;
  const int row = lane >> 2, part_q = lane & 3;              // row and chunk of a lane as rows are loaded and stored
  const Lanes lanes = lane_orders();
  const int z = gridDim.z - 1 - blockIdx.z;                  // (the few tiles with a second adapter begin with it)
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
    const int place = lane & (M - 1);
    const int64_t t = (int64_t)blockIdx.x * M + place;
    const bool valid = t < g.tokens;
    const int k = valid ? adapter_of(g.ids, t, g.n_adapters) : -2;
    bool first = k >= 0 && lane < M;
#pragma unroll
    for (int i = 0; i < M - 1; ++i) {
      const int other = __shfl(k, i, 64);                    // (by all lanes, before the comparison)
      first = first && !(i < place && other == k);
    }
    const uint64_t votes = __ballot(first);
    if (lane < M) {
      token[place] = valid ? place : (int)(g.tokens - 1 - (int64_t)blockIdx.x * M);
      id[place] = k;
    }
    if (first) found[__popcll(votes & ((1ull << lane) - 1))] = k;
    if (lane == 0) n_found = __popcll(votes);
  }
  if (EXPAND && R16 == 1)                                    // (an operand is 32 values along the rank)
    for (int i = tid; i < (int)sizeof(us) / 4; i += WAVES * 64) reinterpret_cast<uint32_t*>(us)[i] = 0;
  __syncthreads();
  const int64_t t0 = SCAN ? 0 : (int64_t)blockIdx.x * M;
  const int n_distinct = __builtin_amdgcn_readfirstlane(n_found);
  int row_token[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) row_token[t] = token[t * 16 + row];

  // What the expansion reads, UNITS units of 32 columns of y at a time (past the wave's last unit: its values).
  constexpr int UNITS = UNITS_AT_ONCE<T, R16>;
  const int units = (g.d_out + 31) >> 5;
  const int part = blockIdx.y * WAVES + wave, parts = g.slices * WAVES;
  const int first = (int)((int64_t)units * part / parts), last = (int)((int64_t)units * (part + 1) / parts);      // of the wave
  const int64_t y_size = g.tokens * g.d_out, b_size = (int64_t)g.n_adapters * g.d_out * g.rank;
  const int b_at = ((row >> 2) * 8 + (row & 3)) * g.rank + part_q * 8;
  const T* base = g.base ? g.base : g.y;                     // (without one the values are not used)
  auto load_units = [&](int unit, int k, Frag<T> (&basef)[UNITS][MT], Frag<T> (&bf)[UNITS][2][CHUNKS]) {
    const int b_here = here(b_at);
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int o0 = min(unit + i, last - 1) * 32;
      const int64_t y0 = t0 * g.d_out + o0, b0 = ((int64_t)max(k, 0) * g.d_out + o0) * g.rank;
#pragma unroll
      for (int t = 0; t < MT; ++t) basef[i][t] = load_near<EDGE>(base + y0, here(row_token[t]) * g.d_out + part_q * 8, g.d_out - o0 - part_q * 8, y_size - y0);
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) bf[i][e][c] = load_near<EDGE>(g.b + b0, b_here + e * 4 * g.rank + c * 32, g.rank - (c * 4 + part_q) * 8, b_size - b0);
    }
  };

  // Turns along the width are DEPTH at a time; past the wave's last turn its values, as zeros.  The other waves cover a turn's latency, and
  // code costs time to fetch (kernels of some us are mostly run once through): 2 rather than 4 at one block of ranks, 30.4 -> 28.8 us for
  // 4096 tokens, 13.7 -> 10.8 for 40 of odd widths; 1 rather than 2 at four, 30.5 -> 25.7 for 1024 tokens.
  constexpr int DEPTH = MT == 1 && R16 == 1 && sizeof(T) == 2 ? 2 : 1;
  const int full = g.d_in / 64;                              // whole turns
  const int turns = (full + WAVES - 1) / WAVES, turn0 = min(wave * turns, full), turn1 = min(turn0 + turns, full);
  auto turn = [&](int s, int i) { return min(s + (i >> 1), turn1 - 1) * 64 + (i & 1) * 32; };

  // A pass per adapter, of those among the tile's tokens that are this workgroup's; the first takes the tokens without one along.
  for (int f = z; f < n_distinct || f == 0; f += gridDim.z) {
    const int k = f < n_distinct ? __builtin_amdgcn_readfirstlane(found[f]) : -1;
    if (k >= 0) {
      // u: rows are tokens, columns are the rank
      const float scale = g.scale[k];
      const T* x = g.x + t0 * g.d_in;
      const T* a = g.a + (int64_t)k * g.rank * g.d_in;
      int x_at[MT];
#pragma unroll
      for (int t = 0; t < MT; ++t) x_at[t] = here(row_token[t] * g.d_in + part_q * 8);
      int a_at[R16];
#pragma unroll
      for (int r = 0; r < R16; ++r) a_at[r] = here(min(r * 16 + row, g.rank - 1) * g.d_in + part_q * 8);
      auto chunk0 = [&](int t) { return (uint64_t)(t0 + here(row_token[t])) * ((g.d_in + 7) >> 3) + part_q; };
      f32x4 acc[MT][R16];
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int r = 0; r < R16; ++r) acc[t][r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
      for (int s = turn0; s < turn1; s += DEPTH) {
        Frag<T> xf[MT][2 * DEPTH], af[2 * DEPTH][R16];
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int i = 0; i < 2 * DEPTH; ++i) xf[t][i] = load_from(x + turn(s, i), x_at[t]);
#pragma unroll
        for (int i = 0; i < 2 * DEPTH; ++i)
#pragma unroll
          for (int r = 0; r < R16; ++r) af[i][r] = load_from(a + turn(s, i), a_at[r]);
        if (g.drop.limit) {
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            uint32_t kept[(DEPTH + 1) / 2];
            const uint64_t chunk = chunk0(t);
            kept_bits(g.drop, kept, [&](int j) { return chunk + (turn(s, j) >> 3); });
            mask_frags(xf[t], kept);
          }
        }
#pragma unroll
        for (int i = 0; i < 2 * DEPTH; ++i) {
          Frag<T> xo[MT];
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            if (i > 1) keep_all(xf[t][i], less_mask(s + (i >> 1), turn1));
            xo[t] = exchange(xf[t][i], lanes.operand);
          }
#pragma unroll
          for (int r = 0; r < R16; ++r) {
            const Frag<T> ao = exchange(af[i][r], lanes.operand);
#pragma unroll
            for (int t = 0; t < MT; ++t) mma(acc[t][r], xo[t], ao);
          }
        }
      }
      if (wave == WAVES - 1 && (g.d_in & 63)) {             // the rest of the width
        Frag<T> ar[2][R16];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int n = g.d_in - full * 64 - h * 32 - part_q * 8, at = rest_base(g.d_in, h);
#pragma unroll
          for (int r = 0; r < R16; ++r) {
            ar[h][r] = load_near<EDGE>(a + at, a_at[r], n, rest_left((int64_t)(g.n_adapters - k) * g.rank, g.d_in, h));
            keep_first(ar[h][r], n);
          }
        }
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          Frag<T> xr[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int n = g.d_in - full * 64 - h * 32 - part_q * 8, at = rest_base(g.d_in, h);
            xr[h] = load_near<EDGE>(x + at, x_at[t], n, rest_left(g.tokens - t0, g.d_in, h));
            keep_first(xr[h], n);
          }
          if (g.drop.limit) {
            uint32_t kept[1];
            const uint64_t chunk = chunk0(t);
            kept_bits(g.drop, kept, [&](int j) { return chunk + full * 8 + (j & 1) * 4; });
            mask_frags(xr, kept);
          }
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < R16; ++r) mma(acc[t][r], exchange(xr[h], lanes.operand), exchange(ar[h][r], lanes.operand));
        }
      }
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int r = 0; r < R16; ++r)
#pragma unroll
          for (int i = 0; i < 4; ++i) sums[wave][((t * R16 + r) * 4 + i) * 64 + lane] = acc[t][r][i];
      __syncthreads();
      for (int v = tid; v < MT * R16 * 256; v += WAVES * 64) {
        const int l = v & 63, row = v / (R16 * 256) * 16 + (l >> 4) * 4 + ((v >> 6) & 3), col = (v >> 8) % R16 * 16 + (l & 15);
        float t = sums[0][v];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) t += sums[w][v];
        if (g.drop.limit) t *= g.drop.scale;
        if (col >= g.rank) t = 0.0f;
        if (g.u && blockIdx.y == 0 && col < g.ldu && id[row] == k) g.u[(t0 + token[row]) * g.ldu + col] = EXPAND ? t : t * scale;
        if (EXPAND) split(t * scale, &us[0][row][col], M * LD);
      }
      __syncthreads();
    }
    if (f == 0 && g.u && blockIdx.y == 0)
      for (int v = tid; v < M * g.ldu; v += WAVES * 64)
        if (id[v / g.ldu] == -1) g.u[(t0 + token[v / g.ldu]) * g.ldu + v % g.ldu] = 0.0f;
    if (!EXPAND) continue;

    // y: rows are 16 columns of y, columns are tokens, the contracted axis the rank.  Two products' rows are dealt so that a lane ends
    // with eight consecutive columns of its token.
    Frag<T> uf[MT][CHUNKS][NT];
    uint32_t has[MT];
    bool stores[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int p = 0; p < NT; ++p) uf[t][c][p] = *reinterpret_cast<const Frag<T>*>(&us[p][t * 16 + m][(c * 4 + q) * 8]);
      const int row_id = id[t * 16 + row];
      has[t] = id[t * 16 + m] == k && k >= 0 ? ~0u : 0u;
      stores[t] = row_id == k || (f == 0 && row_id == -1);
    }
    const uint32_t has_base = g.base ? ~0u : 0u;
    uint32_t along[CHUNKS];                                  // chunks of the rank
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) along[c] = less_mask((c * 4 + part_q) * 8, g.rank);
#pragma unroll 1
    for (int unit = first; unit < last; unit += UNITS) {
      Frag<T> basef[UNITS][MT], bf[UNITS][2][CHUNKS];
      load_units(unit, k, basef, bf);
      f32x4 acc[UNITS][MT][2];
#pragma unroll
      for (int i = 0; i < UNITS; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
          for (int t = 0; t < MT; ++t) acc[i][t][e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int c = 0; c < CHUNKS; ++c) {
            if (EDGE == WHOLE) keep_all(bf[i][e][c], along[c]);
            const Frag<T> bo = exchange(bf[i][e][c], lanes.operand);
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
              for (int p = 0; p < NT; ++p) mma(acc[i][t][e], bo, uf[t][c][p]);
          }
        }
      Frag<T> yf[UNITS][MT];
#pragma unroll
      for (int i = 0; i < UNITS; ++i)
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          float v[8], o[8];
          unpack(exchange(basef[i][t], lanes.operand), o);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = keep(acc[i][t][e >> 2][e & 3], has[t]) + keep(o[e], has_base);
          pack(v, yf[i][t]);
          yf[i][t] = exchange(yf[i][t], lanes.rows);
        }
#pragma unroll
      for (int i = 0; i < UNITS; ++i)
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          const int o0 = (unit + i) * 32;
          if (stores[t] && unit + i < last)
            store_frag<EDGE>(g.y + t0 * g.d_out + o0 + here(row_token[t]) * g.d_out + part_q * 8, g.d_out - o0 - part_q * 8, yf[i][t]);
        }
    }
  }
}

// ---- backward: order of the tokens, b transposed -------------------------------------------------------------------

constexpr int HELD = 8;                  // ids that a thread of the ordering workgroup keeps between its two looks at them

// order: the tokens by adapter, in their order within one, those without an adapter last; start[k]: adapter k's first place, start[n]:
// that of the tokens without one, start[n + 1] = tokens.  One workgroup; each wave counts and places a range of tokens of its own.
__device__ void order_tokens(const int32_t* ids, int tokens, int n_adapters, int n_waves, int32_t* order, int32_t* start, int32_t* cursor) {
  __shared__ int32_t totals[16], carry;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, bins = n_adapters + 1;
  for (int i = threadIdx.x; i < n_waves * bins; i += 1024) cursor[i] = 0;
  if (threadIdx.x == 0) carry = 0;
  const int per = (((tokens + n_waves - 1) / n_waves) + 63) & ~63;
  const int first = wave < n_waves ? min(wave * per, tokens) : tokens, last = min(first + per, tokens);
  volatile int32_t* mine = cursor + wave * bins;             // (written by one lane, read by others of its wave)
  auto bin_of = [&](int t) {
    if (t >= last) return -1;
    const int k = adapter_of(ids, t, n_adapters);
    return k < 0 ? n_adapters : k;
  };
  int held[HELD];
#pragma unroll
  for (int i = 0; i < HELD; ++i) held[i] = bin_of(first + i * 64 + lane);
  __syncthreads();
  // f(place among the wave's lanes with this bin, how many, bin) once per lane that holds a token
  auto by_bin = [&](int bin, auto f) {
    uint64_t left = __ballot(bin >= 0);
    while (left) {
      const int b = __builtin_amdgcn_readlane(bin, __ffsll((unsigned long long)left) - 1);
      const uint64_t same = __ballot(bin == b);
      if (bin == b) f(__popcll(same & ((1ull << lane) - 1)), __popcll(same), b);
      left &= ~same;
    }
  };
  auto all = [&](auto f) {                                   // f(token, bin) of every 64 tokens of the wave, in order
#pragma unroll
    for (int i = 0; i < HELD; ++i)
      if (first + i * 64 < last) f(first + i * 64 + lane, held[i]);
    for (int t = first + HELD * 64; t < last; t += 64) f(t + lane, bin_of(t + lane));
  };
  all([&](int, int bin) {
    by_bin(bin, [&](int place, int n, int b) {
      if (place == 0) mine[b] = mine[b] + n;
    });
  });
  __syncthreads();
  for (int b0 = 0; b0 < bins; b0 += 1024) {
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
    if (threadIdx.x == 1023) carry = at + total;
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
  all([&](int t, int bin) {
    by_bin(bin, [&](int place, int n, int b) {
      const int at = mine[b];
      order[at + place] = t;
      if (place == 0) mine[b] = at + n;
    });
  });
}

// 4096 tokens: 8 us, of which the order takes 6.5.  The first workgroup orders the tokens; the next ones transpose b, bt[k][j][o] = b[k][o][j], 64 columns o of one adapter at a time through
// LDS; the others leave dropout's mask, a byte per chunk.  (The order is a chain of latencies, so the rest is done beside it.)
template <typename T>
__global__ __launch_bounds__(1024) void arrange_kernel(const int32_t* ids, int tokens, int n_adapters, int n_waves, int32_t* order, int32_t* start, const T* b,
                                                       T* bt, int d_out, int rank, int transposes, Drop drop, uint8_t* kept, int64_t chunks) {
  extern __shared__ int32_t cursor[];                        // [wave][n + 1]
  __shared__ T tile[MAX_RANK][64 + 4 / sizeof(T)];
  if (blockIdx.x == 0) {
    order_tokens(ids, tokens, n_adapters, n_waves, order, start, cursor);
    return;
  }
  if ((int)blockIdx.x > transposes) {
    const int64_t step = (int64_t)(gridDim.x - 1 - transposes) * 1024;
    for (int64_t c = (int64_t)(blockIdx.x - 1 - transposes) * 1024 + threadIdx.x; c < chunks; c += step) {
      const uint4 words = philox_words(drop, c);
      uint32_t bits = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) bits |= drop_keeps(drop, words, e) ? 1u << e : 0u;
      kept[c] = (uint8_t)bits;
    }
    return;
  }
  const int per = transposes / n_adapters, k = (blockIdx.x - 1) / per;
  if (n_adapters > 1) {                                      // (a bank holds more adapters than a batch has)
    bool used = false;
#pragma unroll 4
    for (int t = threadIdx.x; t < tokens; t += 1024) used |= adapter_of(ids, t, n_adapters) == k;
    if (!__syncthreads_or(used)) return;
  }
  for (int o0 = (blockIdx.x - 1) % per * 64; o0 < d_out; o0 += per * 64) {
    const int n = min(64, d_out - o0);
    const T* from = b + ((int64_t)k * d_out + o0) * rank;
    for (int i = threadIdx.x; i < n * rank; i += 1024) tile[i % rank][i / rank] = from[i];
    __syncthreads();
    for (int i = threadIdx.x; i < rank * 64; i += 1024)
      if ((i & 63) < n) bt[((int64_t)k * rank + (i >> 6)) * d_out + o0 + (i & 63)] = tile[i >> 6][i & 63];
    __syncthreads();
  }
}

// ---- backward: dx and the gradients of the weights -----------------------------------------------------------------

// Dropout of a batch as the arranging launch leaves it, a bit per element: both dx and da need the mask, and ten rounds of the generator
// twice would be 15 of the 25 us that their memory traffic takes (4096 tokens, 4096 wide).
struct Mask {
  const uint8_t* kept;    // [tokens][ceil(d / 8)], or null
  float scale;
};

template <typename T>
struct GradArgs {         // da from x and v, db from dy and u
  const T* x;             // [tokens, d]
  const float* v;         // [tokens, ldv]
  float* slots;           // [slot][rank][d]
  int d, ldv;
  Mask mask;
};

template <typename T>
struct DxArgs {
  const float* v;         // [tokens, ldv], ldv a multiple of eight with zeros past the rank
  const T* a;             // [n][rank][d]
  const T* base;          // or null
  T* dx;
  int d, ldv;
  Mask mask;
};

struct OrderArgs {
  const int32_t* ids;
  const int32_t* order;
  const int32_t* start;
  int64_t tokens;
  int rank, n_adapters;
  int chunk;              // places of the order per workgroup, CHUNK_MAX at most
};

constexpr int CHUNK_MAX = 512;

// A workgroup of the gradients and of dx has 128 columns and a chunk of the places in the order of adapters, and takes it adapter by
// adapter, its four waves in turns.  A lane holds eight columns, m * 8 on, of several tokens, so that every load and store is 16 bytes of a
// row.  (Two kernels: one for both needed 246 registers; up to rank 16 the gradients need 130, three waves per SIMD, and dx 170.)
struct Places {
  const int32_t* token;   // LDS
  int first, last;        // of the chunk
};
__device__ __forceinline__ Places load_places(const OrderArgs& w, int chunk, int32_t* token) {
  const Places at{token, chunk * w.chunk, (int)min((int64_t)(chunk + 1) * w.chunk, w.tokens)};
  for (int i = threadIdx.x; i < at.last - at.first; i += 256) token[i] = w.order[at.first + i];
  __syncthreads();
  return at;
}

// Sums over tokens, 32 in a turn, the lane's at places q * 4 + 0..3 and 16 + q * 4 + 0..3: the lane turns its eight rows in registers into eight operands whose contracted axis is the tokens (operand e's row m
// is column 8 m + e), so nothing goes through LDS.  An adapter's sums within the chunk go to a slot of their own (numbered chunk +
// adapter: of two neighbours in the order one number is larger), and are added in the order of chunks by the kernel below.  Bound by
// memory: 4096 tokens, da and db 4096 wide at rank 8, 67 MB in 18.5 us.
template <typename T, int R16, int EDGE>
__device__ __forceinline__ void grad_segment(const GradArgs<T>& g, const OrderArgs& w, const Places& at, int slab, int k, int p0, int p1, float* sums) {
  constexpr int NG = TERMS<T>;
  const int lane = threadIdx.x & 63, wave = wave_id(), m = lane & 15, q = lane >> 4;
  const int c0 = slab * 128 + m * 8, n = g.d - c0, per_row = (g.d + 7) >> 3;
  f32x4 acc[R16][8];
#pragma unroll
  for (int r = 0; r < R16; ++r)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[r][e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
  for (int p = p0 + wave * 32; p < p1; p += 128) {
    auto place = [&](int j) { return p + (j >> 2) * 16 + q * 4 + (j & 3); };
    Frag<T> rows[8];
    uint32_t kept[8];
    float f[R16][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {                            // (past the end: the last one's values, with 0 in v)
      const int64_t t = at.token[min(place(j), p1 - 1) - at.first];
      rows[j] = load_at<EDGE>(g.x, t * g.d + c0, n, w.tokens * g.d);
      if (g.mask.kept) kept[j] = g.mask.kept[t * per_row + min(c0 >> 3, per_row - 1)];
#pragma unroll
      for (int r = 0; r < R16; ++r) f[r][j] = g.v[t * g.ldv + min(r * 16 + m, w.rank - 1)];
    }
    if (g.mask.kept) {
#pragma unroll
      for (int j = 0; j < 8; ++j) mask_frag<0>(rows[j], kept[j]);
    }
    Frag<T> cols[8];
    transpose(rows, cols);
#pragma unroll
    for (int r = 0; r < R16; ++r) {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[r][j] = keep(f[r][j], less_mask_apart(place(j), p1));
      Frag<T> vf[NG];
      split(f[r], vf);
#pragma unroll
      for (int i = 0; i < NG; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) mma(acc[r][e], cols[e], vf[i]);
    }
  }
  float* slot = g.slots + (int64_t)(blockIdx.y + k) * w.rank * g.d;
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
    if (wave == 0 && r * 16 + m < w.rank) {
      // the lane's rank is r * 16 + m; its columns q * 32 + i * 8 + e
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          o[e] = acc[r][e][i] + sums[(e * 4 + i) * 64 + lane] + sums[(32 + e * 4 + i) * 64 + lane] + sums[(64 + e * 4 + i) * 64 + lane];
          if (g.mask.kept) o[e] *= g.mask.scale;
        }
        const int c = slab * 128 + q * 32 + i * 8;
        store_at<EDGE>(slot + (int64_t)(r * 16 + m) * g.d + c, g.d - c, o);
      }
    }
  }
}

// Slabs of da, then of db.
template <typename T, int R16, int EDGE>
__global__ __launch_bounds__(256) void grad_kernel(GradArgs<T> da, GradArgs<T> db, OrderArgs w, int slabs_da) {
  __shared__ float sums[3 * 64 * 32];
  __shared__ int32_t token[CHUNK_MAX];
  const Places at = load_places(w, blockIdx.y, token);
  const bool first = (int)blockIdx.x < slabs_da;
  for (int p0 = at.first; p0 < at.last;) {
    const int id = adapter_of(w.ids, token[p0 - at.first], w.n_adapters);
    if (id < 0) break;                                       // (they are the last)
    const int p1 = min(w.start[id + 1], at.last);
    grad_segment<T, R16, EDGE>(first ? da : db, w, at, blockIdx.x - (first ? 0 : slabs_da), id, p0, p1, sums);
    p0 = p1;
  }
}

// dx: rows are tokens, 16 in a turn, columns those of dx, dealt so that a lane ends with eight consecutive ones of four tokens; the adapter's
// rows are turned in registers once.
template <typename T, int R16, int EDGE>
__device__ __forceinline__ void dx_segment(const DxArgs<T>& g, const OrderArgs& w, const Places& at, int slab, int k, int p0, int p1) {
  constexpr int CHUNKS = (R16 + 1) / 2, NT = TERMS<T>;
  const int lane = threadIdx.x & 63, wave = wave_id(), m = lane & 15, q = lane >> 4;
  const int c0 = slab * 128 + m * 8, n = g.d - c0, per_row = (g.d + 7) >> 3;
  const bool none = k < 0;                                   // dx = base
  const uint32_t with = none ? 0u : ~0u;
  Frag<T> af[CHUNKS][8];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    Frag<T> rows[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int r = (c * 4 + q) * 8 + j;
      rows[j] = load_at<EDGE>(g.a, ((int64_t)(none ? 0 : k) * w.rank + min(r, w.rank - 1)) * g.d + c0, n, (int64_t)w.n_adapters * w.rank * g.d);
      keep_all(rows[j], less_mask_apart(r, w.rank));
    }
    transpose(rows, af[c]);
  }
#pragma unroll 1
  for (int p = p0 + wave * 16; p < p1; p += 64) {
    Frag<T> base[4];
    uint32_t kept[4];
    float h[CHUNKS][8];
    int64_t row[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t t = at.token[min(p + q * 4 + i, p1 - 1) - at.first];
      row[i] = t * g.d + c0;
      if (g.base) base[i] = load_at<EDGE>(g.base, row[i], n, w.tokens * g.d);
      if (g.mask.kept) kept[i] = g.mask.kept[t * per_row + min(c0 >> 3, per_row - 1)];
    }
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) load8(g.v + (int64_t)at.token[min(p + m, p1 - 1) - at.first] * g.ldv + min((c * 4 + q) * 8, g.ldv - 8), 8, h[c]);
    f32x4 out[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      Frag<T> vf[NT];
      split(h[c], vf);
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) mma(out[e], vf[i], af[c][e]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (p + q * 4 + i >= p1) continue;
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        o[e] = keep(out[e][i], with);
        if (g.mask.kept) o[e] = __uint_as_float(__float_as_uint(o[e] * g.mask.scale) & (uint32_t)__builtin_amdgcn_sbfe(kept[i], e, 1));
      }
      if (g.base) {
        float b[8];
        unpack(base[i], b);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] += b[e];
      }
      store_at<EDGE>(g.dx + row[i], n, o);
    }
  }
}

struct SumArgs {
  const float* da_slots;
  const float* db_slots;
  const float* scale;
  float* da;              // [n][rank][d_in]
  float* db;              // [n][d_out][rank]
  int d_in, d_out;
  int blocks_in, blocks;  // workgroups per adapter: of da, of both
};

constexpr int SUM_COLUMNS = 32;          // of db per workgroup

// Slots of an adapter added in the order of chunks (0 without one); db times the adapter's scale, and turned in LDS, since its rows are along
// the rank (written as they are read, 4 bytes a row, they took 40 us of 2048 tokens' training step at rank 64, eight adapters).
__device__ __forceinline__ void sum_slots(const SumArgs& g, const OrderArgs& w, int k, int b, float* tile) {
  const bool first = b < g.blocks_in;
  const int d = first ? g.d_in : g.d_out;
  const int64_t size = (int64_t)w.rank * d;
  const int p0 = w.start[k], p1 = w.start[k + 1];
  const int c0 = p0 / w.chunk, n = p1 > p0 ? (p1 - 1) / w.chunk - c0 + 1 : 0;
  const float* slots = (first ? g.da_slots : g.db_slots) + (int64_t)(c0 + k) * size;
  if (first) {
    const int64_t i = ((int64_t)b * 256 + threadIdx.x) * 4;
    const int left = (int)min(size - i, (int64_t)4);
    if (left <= 0) return;
    float t[4] = {};
    if (left == 4) {
#pragma unroll 8
      for (int c = 0; c < n; ++c) {
        const Bytes16<float> v = *reinterpret_cast<const Bytes16<float>*>(slots + c * size + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] += __uint_as_float(v.w[e]);
      }
      *reinterpret_cast<Bytes16<float>*>(g.da + k * size + i) = __builtin_bit_cast(Bytes16<float>, t);
    } else {
      for (int e = 0; e < left; ++e) {
        float last = 0.0f;
        for (int c = 0; c < n; ++c) last += slots[c * size + i + e];
        g.da[k * size + i + e] = last;
      }
    }
    return;
  }
  const int o0 = (b - g.blocks_in) * SUM_COLUMNS, columns = min(SUM_COLUMNS, d - o0);
  const float scale = n > 0 ? g.scale[k] : 0.0f;
  for (int i = threadIdx.x; i < w.rank * SUM_COLUMNS; i += 256) {
    const int r = i / SUM_COLUMNS, o = i % SUM_COLUMNS;
    if (o >= columns) continue;
    const float* from = slots + (int64_t)r * d + o0 + o;
    float t = 0.0f;
#pragma unroll 8
    for (int c = 0; c < n; ++c) t += from[c * size];
    tile[o * (w.rank + 1) + r] = n > 0 ? t * scale : 0.0f;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < w.rank * columns; i += 256) g.db[k * size + (int64_t)o0 * w.rank + i] = tile[i / w.rank * (w.rank + 1) + i % w.rank];
}

// A row of workgroups per adapter: of a bank of thousands, all in one row would be more threads than a launch's axis holds (2^32).
__global__ __launch_bounds__(256) void sum_kernel(SumArgs sums, OrderArgs w) {
  __shared__ float tile[SUM_COLUMNS * (MAX_RANK + 1)];
  sum_slots(sums, w, blockIdx.y, blockIdx.x, tile);
}

// What is left once the slots are written: dx, which only needs v, and the sums of the slots, which are short beside it (together 20 us for
// 4096 tokens of 4096 at rank 8, of 72 MB).
template <typename T, int R16, int EDGE>
__global__ __launch_bounds__(256) void finish_kernel(DxArgs<T> dx, SumArgs sums, OrderArgs w, int sum_blocks, int slabs) {
  __shared__ int32_t token[CHUNK_MAX];
  __shared__ float tile[SUM_COLUMNS * (MAX_RANK + 1)];
  if ((int)blockIdx.x < sum_blocks) return sum_slots(sums, w, blockIdx.x / sums.blocks, blockIdx.x % sums.blocks, tile);
  const int block = blockIdx.x - sum_blocks, slab = block % slabs;
  const Places at = load_places(w, block / slabs, token);
  for (int p0 = at.first; p0 < at.last;) {
    const int id = adapter_of(w.ids, token[p0 - at.first], w.n_adapters);
    const int p1 = min(w.start[id < 0 ? w.n_adapters + 1 : id + 1], at.last);
    dx_segment<T, R16, EDGE>(dx, w, at, slab, id, p0, p1);
    p0 = p1;
  }
}

// f(R16) with the rank in blocks of 16 as a compile-time constant
template <typename F>
static void with_rank(int rank, F&& f) {
  if (rank <= 16) f(std::integral_constant<int, 1>{});
  else if (rank <= 32) f(std::integral_constant<int, 2>{});
  else f(std::integral_constant<int, 4>{});
}

// f(R16, EDGE): ... and how rows end (fragments_device.h).  A width or buffer below eight values is nothing to be fast at: one form.
template <typename F>
static void with_shape(int rank, bool whole, bool tiny, F&& f) {
  if (tiny) return f(std::integral_constant<int, 4>{}, std::integral_constant<int, TINY>{});
  with_rank(rank, [&](auto r) {
    if (whole) f(r, std::integral_constant<int, WHOLE>{});
    else f(r, std::integral_constant<int, RAGGED>{});
  });
}

template <typename T, bool EXPAND>
static void launch_tiles(TileArgs<T> g, hipStream_t s) {
  const int units = EXPAND ? (g.d_out + 31) / 32 : 1;
  const bool scan = g.tokens <= SCAN_TOKENS;
  const bool whole = g.d_in % 8 == 0 && (!EXPAND || (g.d_out % 8 == 0 && g.rank % 8 == 0));
  const bool tiny = g.d_in < 8 || (EXPAND && std::min(g.tokens * g.d_out, (int64_t)g.n_adapters * g.d_out * g.rank) < 8);
  with_shape(g.rank, whole, tiny, [&](auto r, auto edge) {
    constexpr int R = decltype(r)::value, E = decltype(edge)::value;
    // Wide adapters are read once for 32 tokens where such tiles still fill the chip (rank 64, 4096 wide, us with 16 / 32: 8192 tokens
    // of one adapter 77 / 63, of eight 98 / 89; 2048 tokens 21.5 / 23.5 and 32 / 38).
    const bool tall = R == 4 && !scan && g.tokens >= 256 * 32;
    const int64_t rows = tall ? 32 : 16, tiles = scan ? g.tokens : (g.tokens + rows - 1) / rows;
    // Parts of y's columns, as many as fill the chip if every tile has tokens.  (Each contracts x again, and workgroups that find none of
    // their own are not free: eight parts for 256 tokens of one adapter, 15 -> 61 us.)
    g.slices = EXPAND ? (int)std::max<int64_t>(1, std::min<int64_t>(256 / tiles, (units + 15) / 16)) : 1;
    const dim3 grid((unsigned)tiles, g.slices, scan ? 1 : std::min(g.n_adapters, 2)), block((scan ? TILE_WAVES<R, true> : TILE_WAVES<R, false>) * 64);
    if (scan) hipLaunchKernelGGL((tile_kernel<T, R, 1, true, EXPAND, E>), grid, block, 0, s, g);
    else if (tall) hipLaunchKernelGGL((tile_kernel<T, R, R == 4 ? 2 : 1, false, EXPAND, E>), grid, block, 0, s, g);
    else hipLaunchKernelGGL((tile_kernel<T, R, 1, false, EXPAND, E>), grid, block, 0, s, g);
  });
}

template <typename T>
static void launch_adapters_forward(const cmoe_adapters_forward_args& p, const Drop& drop, hipStream_t s) {
  launch_tiles<T, true>(TileArgs<T>{(const T*)p.x, (const T*)p.a, (const T*)p.b, p.scale, p.ids, (const T*)p.base, (T*)p.y, p.u, p.tokens, p.d_in, p.d_out,
                                    p.rank, p.n_adapters, p.rank, 1, drop}, s);
}

// Workspace of the backward pass: order and starts, v, b transposed, slots of da's and db's partial sums.
struct BackwardLayout {
  int chunk, chunks, ldv;
  size_t order, start, v, bt, kept, da, db, total;
};
static BackwardLayout backward_layout(int64_t tokens, int d_in, int d_out, int rank, int n_adapters, int dtype) {
  BackwardLayout l{};
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t o = off; off = (off + bytes + 255) & ~(size_t)255; return o; };
  // Long chunks leave fewer partial sums, short ones more workgroups: about 1024 of them, of one to four turns per wave.
  const int64_t slabs = 2 * ((d_in + 127) / 128) + (d_out + 127) / 128;
  for (l.chunk = 128; l.chunk < CHUNK_MAX && tokens * slabs > 1024 * 2 * l.chunk;) l.chunk *= 2;
  l.ldv = (rank + 7) & ~7;
  l.chunks = (int)((tokens + l.chunk - 1) / l.chunk);
  l.order = take(sizeof(int32_t) * tokens);
  l.start = take(sizeof(int32_t) * (n_adapters + 2));
  l.v = take(sizeof(float) * tokens * l.ldv);
  l.bt = take(elem_size(dtype) * n_adapters * rank * d_out);
  l.kept = take(tokens * ((d_in + 7) / 8));
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
  const bool needs_v = p.tokens > 0 && (p.dx || p.da);
  const int n_waves = std::min(16, (MAX_ADAPTERS + 1) / (p.n_adapters + 1));
  const int transposes = needs_v ? std::min((p.d_out + 63) / 64, std::max(1, 512 / p.n_adapters)) * p.n_adapters : 0;
  const int64_t chunks = needs_v && drop.limit ? p.tokens * ((p.d_in + 7) / 8) : 0;
  const int masks = (int)std::min<int64_t>((chunks + 1023) / 1024, 1024);
  uint8_t* kept = (uint8_t*)(ws + l.kept);
  const Mask mask{chunks > 0 ? kept : nullptr, drop.scale};
  hipLaunchKernelGGL(arrange_kernel<T>, dim3(1 + transposes + masks), dim3(1024), sizeof(int32_t) * n_waves * (p.n_adapters + 1), s, p.ids, (int)p.tokens,
                     p.n_adapters, n_waves, order, start, (const T*)p.b, bt, p.d_out, p.rank, transposes, drop, kept, chunks);
  if (needs_v)
    launch_tiles<T, false>(TileArgs<T>{(const T*)p.dy, bt, nullptr, p.scale, p.ids, nullptr, nullptr, v, p.tokens, p.d_out, 0, p.rank, p.n_adapters, l.ldv, 1, Drop{}}, s);
  const DxArgs<T> dx{v, (const T*)p.a, (const T*)p.dx_base, (T*)p.dx, p.d_in, l.ldv, mask};
  const GradArgs<T> ga{(const T*)p.x, v, da, p.d_in, l.ldv, mask}, gb{(const T*)p.dy, p.u, db, p.d_out, p.rank, Mask{}};
  const OrderArgs w{p.ids, order, start, p.tokens, p.rank, p.n_adapters, l.chunk};
  const int slabs = (p.d_in + 127) / 128, slabs_da = p.da ? slabs : 0, slabs_db = p.db ? (p.d_out + 127) / 128 : 0;
  if (p.tokens > 0 && slabs_da + slabs_db > 0) {
    const bool whole = (!p.da || p.d_in % 8 == 0) && (!p.db || p.d_out % 8 == 0), tiny = (p.da && p.d_in < 8) || (p.db && p.d_out < 8);
    with_shape(p.rank, whole, tiny, [&](auto r, auto edge) {
      hipLaunchKernelGGL((grad_kernel<T, decltype(r)::value, decltype(edge)::value>), dim3(slabs_da + slabs_db, l.chunks), dim3(256), 0, s, ga, gb, w, slabs_da);
    });
  }
  const int blocks_in = p.da ? (int)(((int64_t)p.rank * p.d_in + 1023) / 1024) : 0, blocks_out = p.db ? (p.d_out + SUM_COLUMNS - 1) / SUM_COLUMNS : 0;
  const SumArgs sums{da, db, p.scale, p.da, p.db, p.d_in, p.d_out, blocks_in, blocks_in + blocks_out};
  int sum_blocks = sums.blocks * p.n_adapters;
  // Beside dx there is room for two or three workgroups on a CU.  Where the sums alone are many times that, a launch of their own, of eight
  // (us of both: 34 adapters of rank 24, 2368 by 8896, 128 tokens 50 / 36; eight of rank 64, 4096 wide, 2048 tokens 42 / 40; one of rank 8,
  // 160 workgroups, 19.6 beside dx and 2 more apart).
  if (sum_blocks > 2048) {
    hipLaunchKernelGGL(sum_kernel, dim3(sums.blocks, p.n_adapters), dim3(256), 0, s, sums, w);
    sum_blocks = 0;
  }
  const int dx_blocks = p.dx ? slabs * l.chunks : 0;
  if (sum_blocks + dx_blocks > 0)
    with_shape(p.rank, p.d_in % 8 == 0, p.d_in < 8, [&](auto r, auto edge) {
      hipLaunchKernelGGL((finish_kernel<T, decltype(r)::value, decltype(edge)::value>), dim3(sum_blocks + dx_blocks), dim3(256), 0, s, dx, sums, w, sum_blocks, slabs);
    });
}

static int check_adapters(const char* what, int dtype, int64_t tokens, int d_in, int d_out, int rank, int n_adapters) {
  if (dtype != CMOE_F32 && dtype != CMOE_BF16) return fail(CMOE_EINVAL, "%s: dtype must be CMOE_F32 or CMOE_BF16", what);
  if (d_in < 1 || d_out < 1 || d_in > MAX_WIDTH || d_out > MAX_WIDTH) return fail(CMOE_EINVAL, "%s: d_in and d_out must be 1 to %d", what, MAX_WIDTH);
  if (rank < 1 || rank > MAX_RANK) return fail(CMOE_EINVAL, "%s: rank must be 1 to %d", what, MAX_RANK);
  if (n_adapters < 1 || n_adapters > MAX_ADAPTERS) return fail(CMOE_EINVAL, "%s: n_adapters must be 1 to %d", what, MAX_ADAPTERS);
  if (tokens < 0 || tokens > (1 << 20)) return fail(CMOE_EINVAL, "%s: tokens must be 0 to 2^20", what);
  return CMOE_OK;
}

}  // namespace cmoe

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
  if (int rc = check_operands(what, {{"x", p->x, in, es}, {"a", p->a, n * p->rank * p->d_in * es, es}, {"b", p->b, n * p->d_out * p->rank * es, es},
                                     {"scale", p->scale, n * 4, 4}, {"ids", p->ids, t * 4, 4}, {"base", p->base, out, es, true}},
                              {{"y", p->y, out, es, true}, {"u", p->u, t * p->rank * 4, 4}}))
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
  if (int rc = check_operands(what, {{"dy", p->dy, out, es}, {"x", p->x, in, es}, {"u", p->u, t * p->rank * 4, 4}, {"a", p->a, wa * es, es}, {"b", p->b, wb * es, es},
                                     {"scale", p->scale, n * 4, 4}, {"ids", p->ids, t * 4, 4}, {"dx_base", p->dx_base, in, es, true}},
                              {{"dx", p->dx, in, es, true}, {"da", p->da, wa * 4, 4}, {"db", p->db, wb * 4, 4}, {"workspace", p->workspace, p->workspace_bytes, 16}}))
    return rc;
  if (p->tokens == 0 && !p->da && !p->db) return CMOE_OK;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  p->dtype == CMOE_BF16 ? launch_adapters_backward<bf16_t>(*p, drop, s) : launch_adapters_backward<float>(*p, drop, s);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CMOE_OK : fail(CMOE_EHIP, "%s: %s", what, hipGetErrorString(e));
}
