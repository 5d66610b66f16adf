// Eight values of a row per lane, in registers as they are stored: how rows are read and written, and operands of the matrix instructions.
#pragma once
#include "dropout_device.h"
#include "row_reads.h"

namespace cmoe {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

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
// All ones where a < b (both far from the ends of the type).  Values are chosen by masks, not by conditions, throughout: of a condition on
// loaded values the compiler made a branch for each, with a wait of its own.
__device__ __forceinline__ uint32_t less_mask(int a, int b) { return (uint32_t)((a - b) >> 31); }
// ... that is not to be merged with others: of the products of two sets of masks it made conditions again, hundreds of them, in scalar
// registers that it had to spill.
__device__ __forceinline__ uint32_t less_mask_apart(int a, int b) {
  uint32_t mask = less_mask(a, b);
  asm("" : "+v"(mask));
  return mask;
}
__device__ __forceinline__ uint32_t choose(uint32_t mask, uint32_t a, uint32_t b) { return (a & mask) | (b & ~mask); }

// Values from the s-th on, zeros after the last (any s >= 0).
__device__ __forceinline__ void shift_down(Frag<bf16_t>& f, int s) {
  const uint32_t four = less_mask(3, s & 4), two = less_mask(1, s & 2), one = less_mask(0, s & 1), any = less_mask(s, 8);
  f.w[0] = choose(four, f.w[2], f.w[0]);
  f.w[1] = choose(four, f.w[3], f.w[1]);
  f.w[2] &= ~four;
  f.w[3] &= ~four;
#pragma unroll
  for (int i = 0; i < 4; ++i) f.w[i] = choose(two, i < 3 ? f.w[i + 1] : 0u, f.w[i]);
#pragma unroll
  for (int i = 0; i < 4; ++i) f.w[i] = choose(one, (f.w[i] >> 16) | (i < 3 ? f.w[i + 1] << 16 : 0u), f.w[i]) & any;
}
__device__ __forceinline__ void shift_down(Frag<float>& f, int s) {
  const uint32_t any = less_mask(s, 8);
  uint32_t w[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(f.w[e]);
#pragma unroll
  for (int step = 4; step > 0; step >>= 1) {
    const uint32_t by = less_mask(0, s & step);
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = choose(by, e + step < 8 ? w[e + step] : 0u, w[e]);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) f.w[e] = __uint_as_float(w[e] & any);
}
// The first n values, zeros after them.
__device__ __forceinline__ void keep_first(Frag<bf16_t>& f, int n) {
#pragma unroll
  for (int e = 0; e < 4; ++e) f.w[e] &= choose(0xffffu, less_mask(2 * e, n), less_mask(2 * e + 1, n));
}
__device__ __forceinline__ void keep_first(Frag<float>& f, int n) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f.w[e] = __uint_as_float(__float_as_uint(f.w[e]) & less_mask(e, n));
}
// All of them or zeros.
__device__ __forceinline__ void keep_all(Frag<bf16_t>& f, uint32_t mask) {
#pragma unroll
  for (int e = 0; e < 4; ++e) f.w[e] &= mask;
}
__device__ __forceinline__ void keep_all(Frag<float>& f, uint32_t mask) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f.w[e] = __uint_as_float(__float_as_uint(f.w[e]) & mask);
}
__device__ __forceinline__ float keep(float v, uint32_t mask) { return __uint_as_float(__float_as_uint(v) & mask); }

// How eight values of a row are read, of which n (it may be 0 or less, or more than 8) belong to it:
//   WHOLE   rows are a multiple of eight values: n >= 8, or n <= 0 and the result is not used
//   RAGGED  the buffer has eight values at least: eight that do not pass its end, moved into place, zeros from the n-th on
//   TINY    one by one
// The first two have no branch, so that a caller's loads are all in flight before the first is waited for.
enum { WHOLE, RAGGED, TINY };

template <typename T>
__device__ __forceinline__ Frag<T> load_tiny(const T* p, int n) {
  Frag<T> f = {};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (e >= n) continue;
    if constexpr (sizeof(T) == 2) f.w[e >> 1] |= (uint32_t)p[e] << (16 * (e & 1));
    else f.w[e] = p[e];
  }
  return f;
}

// From an address that is the same for the whole wave and an offset of the lane (values, below 2^31 bytes): one register, where a
// 64-bit address of its own for every load under way took more than the loads' results.  left: from base to the buffer's end; WHOLE
// adds the offset unsigned, so eight at least.
template <typename T>
__device__ __forceinline__ Frag<T> load_from(const T* base, uint32_t at) {
  return load_frag(reinterpret_cast<const T*>(reinterpret_cast<const char*>(base) + (uint32_t)(at * sizeof(T))));
}
template <int EDGE, typename T>
__device__ __forceinline__ Frag<T> load_near(const T* base, int at, int n, int64_t left) {
  if constexpr (EDGE == TINY) return load_tiny(base + at, tiny_count(at, n, left));
  const int from = near_first(at, left);
  if constexpr (EDGE == WHOLE) return load_from(base, (uint32_t)from);
  Frag<T> f = load_frag(base + from);
  shift_down(f, at - from);
  keep_first(f, n);
  return f;
}

// From any place of a buffer of `size` values.
template <int EDGE, typename T>
__device__ __forceinline__ Frag<T> load_at(const T* p, int64_t at, int n, int64_t size) {
  if constexpr (EDGE == TINY) return load_tiny(p + at, n);
  if constexpr (EDGE == WHOLE) return load_frag(p + (n > 0 ? at : 0));
  const int64_t from = n > 0 ? min(at, size - 8) : 0;
  Frag<T> f = load_frag(p + from);
  asm("" : "+v"(n));                                         // (as less_mask_apart)
  shift_down(f, n > 0 ? (int)(at - from) : 8);
  keep_first(f, n);
  return f;
}

// What dropout drops becomes 0 (its scale is applied to the products in fp32, so that bf16 values stay as they are).
// kept: a bit per value, from bit AT on.
template <int AT>
__device__ __forceinline__ void mask_frag(Frag<bf16_t>& f, uint32_t kept) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    f.w[e] &= ((uint32_t)__builtin_amdgcn_sbfe(kept, AT + 2 * e, 1) & 0xffffu) | ((uint32_t)__builtin_amdgcn_sbfe(kept, AT + 2 * e + 1, 1) & 0xffff0000u);
}
template <int AT>
__device__ __forceinline__ void mask_frag(Frag<float>& f, uint32_t kept) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f.w[e] = __uint_as_float(__float_as_uint(f.w[e]) & (uint32_t)__builtin_amdgcn_sbfe(kept, AT + e, 1));
}

// ... of N operands, four to a word.
template <int I = 0, typename T, int N, int W>
__device__ __forceinline__ void mask_frags(Frag<T> (&f)[N], const uint32_t (&kept)[W]) {
  mask_frag<(I & 3) * 8>(f[I], kept[I >> 2]);
  if constexpr (I + 1 < N) mask_frags<I + 1>(f, kept);
}

// The bits of 4 * N chunks, chunk(j) the j-th one's number, 32 to a word.  A loop, not N copies of the generator: the kernels are
// short-lived, and what they fetch as code counts (eight copies, beside the code of three forms of rows, made a kernel for dx and the gradients
// of 4096 tokens 55 us long that took 44 with a loop and one form).
template <int N, typename F>
__device__ __forceinline__ void kept_bits(const Drop& d, uint32_t (&kept)[N], F&& chunk) {
  const uint32_t rest = 65536u - d.limit;                    // a half word is at least the limit where the sum carries
#pragma unroll
  for (int i = 0; i < N; ++i) {
    uint32_t bits = 0;
#pragma unroll 1
    for (int j = 0; j < 4; ++j) {
      const uint4 words = philox_words(d, chunk(i * 4 + j));
      uint32_t b = 0;
#pragma unroll
      for (int e = 7; e >= 0; --e) {
        const uint32_t w = e < 2 ? words.x : e < 4 ? words.y : e < 6 ? words.z : words.w;
        b = (b << 1) | ((((e & 1) ? w >> 16 : w & 0xffffu) + rest) >> 16);
      }
      bits |= b << (8 * j);
    }
    kept[i] = bits;
  }
}

// A load whose neighbouring lanes are on different rows moves 18 bytes a cycle into a CU, one whose lanes 4 r to 4 r + 3 hold row r's four
// chunks 55 (measured, from the L2 cache): so rows are loaded and stored in the second order and exchanged with the operands', 16 q + r,
// between the lanes.
struct Lanes {
  int operand, rows;      // byte addresses of the lanes to take from
};
__device__ __forceinline__ Lanes lane_orders() {
  const int l = threadIdx.x & 63;
  return Lanes{((l & 15) * 4 + (l >> 4)) * 4, ((l & 3) * 16 + (l >> 2)) * 4};
}
template <typename T>
__device__ __forceinline__ Frag<T> exchange(const Frag<T>& f, int from) {
  Frag<T> out;
#pragma unroll
  for (int e = 0; e < (int)(sizeof(f.w) / 4); ++e)
    out.w[e] = __builtin_bit_cast(decltype(f.w[0] + f.w[0]), __builtin_amdgcn_ds_bpermute(from, __builtin_bit_cast(int, f.w[e])));
  return out;
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

// fp32 values as a sum of operands.  bf16: the upper eight bits of the significand, then those of what is left, then the rest: three terms
// carry all 24, so that a product is that of the fp32 values, also where an output is a small difference of its base and the adapter's
// part.  (Two terms, 16 bits, are no faster to speak of: us per training step of 4096 tokens, 4096 wide, rank 8, 85.4 / 85.9 with three;
// 2048 tokens at rank 64 160.4 / 162.5; 2048 tokens of prompts at rank 32 21.8 / 22.3.)  What is left of an infinity would be NaN: 0.  (An infinity
// in the other factor times a term that is 0 is NaN all the same: not finite either way.)  fp32 needs one term.
template <typename T> constexpr int TERMS = sizeof(T) == 2 ? 3 : 1;

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
      for (int e = 0; e < 4; ++e) f[i].w[e] = pack_bf16(rest[2 * e], rest[2 * e + 1]);
    }
  }
}
__device__ __forceinline__ void split(const float (&v)[8], Frag<float> (&f)[1]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f[0].w[e] = v[e];
}
// ... of one value, stored `stride` apart.
__device__ __forceinline__ void split(float v, bf16_t* to, int stride) {
  float rest = v;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    if (i < 2) {
      to[i * stride] = (bf16_t)(__float_as_uint(rest) >> 16);
      const float left = rest - __uint_as_float(__float_as_uint(rest) & 0xffff0000u);
      rest = left == left ? left : 0.0f;
    } else {
      to[i * stride] = f32_to_bf16(rest);
    }
  }
}
__device__ __forceinline__ void split(float v, float* to, int) { *to = v; }

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

// Eight values as they are stored.
__device__ __forceinline__ void pack(const float (&v)[8], Frag<bf16_t>& f) {
#pragma unroll
  for (int e = 0; e < 4; ++e) f.w[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
}
__device__ __forceinline__ void pack(const float (&v)[8], Frag<float>& f) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f.w[e] = v[e];
}
template <int EDGE>
__device__ __forceinline__ void store_frag(bf16_t* p, int n, const Frag<bf16_t>& f) {
  if (n >= 8 || (EDGE == WHOLE && n > 0)) {
    *reinterpret_cast<Bytes16<bf16_t>*>(p) = __builtin_bit_cast(Bytes16<bf16_t>, f);
  } else if (EDGE != WHOLE) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = (bf16_t)(f.w[e >> 1] >> (16 * (e & 1)));
  }
}
template <int EDGE>
__device__ __forceinline__ void store_frag(float* p, int n, const Frag<float>& f) {
  if (n > 0) store8(p, EDGE == WHOLE ? 8 : n, f.w);
}

// Eight values to a row of which n are left.
template <int EDGE, typename T>
__device__ __forceinline__ void store_at(T* p, int n, const float (&v)[8]) {
  if (n > 0) store8(p, EDGE == WHOLE ? 8 : n, v);
}

}  // namespace cmoe
