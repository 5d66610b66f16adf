// Dropout from a counter-based generator, and chunks of eight elements in registers: what the norm, dropout and adapter kernels share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/cmoe.h"
#include "device_utils.h"

namespace cmoe {

// The mask of a [rows, cols] batch is a function of (seed, offset) and the element's place, so it is never stored: eight
// consecutive elements of a row share one counter, (number of the chunk in the batch, offset), and take one half word each of
// its four random words (the low half first).  An element is kept where its half word is at least `limit`, and multiplied by
// `scale` = 65536 / (65536 - limit).
struct Drop {
  uint32_t k0, k1, o0, o1;
  uint32_t limit;            // 0: keep everything (the kernels run their form without a mask); 65536: keep nothing
  float scale;
};

// Philox-4x32 with ten rounds (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3, SC 2011).
__device__ __forceinline__ uint4 philox_words(const Drop& d, uint64_t chunk) {
  uint32_t c0 = (uint32_t)chunk, c1 = (uint32_t)(chunk >> 32), c2 = d.o0, c3 = d.o1, k0 = d.k0, k1 = d.k1;
#pragma unroll
  for (int round = 0; round < 10; ++round) {
    const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0;
    c2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
    c1 = (uint32_t)p1;
    c3 = (uint32_t)p0;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}

__device__ __forceinline__ bool drop_keeps(const Drop& d, const uint4& words, int e) {
  const uint32_t w = e < 2 ? words.x : e < 4 ? words.y : e < 6 ? words.z : words.w;
  return ((e & 1) ? (w >> 16) : (w & 0xffffu)) >= d.limit;
}

// A dropped element is 0 whatever it was (NaN and infinities too).
__device__ __forceinline__ void drop8(float (&v)[8], const Drop& d, uint64_t chunk) {
  const uint4 words = philox_words(d, chunk);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = drop_keeps(d, words, e) ? v[e] * d.scale : 0.0f;
}

// Sixteen bytes at any address an element may have: the memory system of this part takes wide accesses that are not aligned,
// so rows of odd width need no path of their own, only their last chunk does.
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Bytes16 { uint32_t w[4]; };

// Eight consecutive elements, or the first n of them and zeros (n >= 1).
__device__ __forceinline__ void load8(const bf16_t* p, int n, float (&v)[8]) {
  if (n >= 8) {
    const Bytes16<bf16_t> b = *reinterpret_cast<const Bytes16<bf16_t>*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(b.w[e] << 16);
      v[2 * e + 1] = __uint_as_float(b.w[e] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? bf16_to_f32(p[e]) : 0.0f;
  }
}
__device__ __forceinline__ void load8(const float* p, int n, float (&v)[8]) {
  if (n >= 8) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const Bytes16<float> b = *reinterpret_cast<const Bytes16<float>*>(p + 4 * h);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * h + e] = __uint_as_float(b.w[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? p[e] : 0.0f;
  }
}

// Two values rounded to bf16 by one conversion.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}

__device__ __forceinline__ void store8(bf16_t* p, int n, const float (&v)[8]) {
  if (n >= 8) {
    Bytes16<bf16_t> b;
#pragma unroll
    for (int e = 0; e < 4; ++e) b.w[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
    *reinterpret_cast<Bytes16<bf16_t>*>(p) = b;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = f32_to_bf16(v[e]);
  }
}
__device__ __forceinline__ void store8(float* p, int n, const float (&v)[8]) {
  if (n >= 8) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      Bytes16<float> b;
#pragma unroll
      for (int e = 0; e < 4; ++e) b.w[e] = __float_as_uint(v[4 * h + e]);
      *reinterpret_cast<Bytes16<float>*>(p + 4 * h) = b;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = v[e];
  }
}

// What a value becomes when it is stored as a T and read again.
template <typename T> __device__ __forceinline__ float as_stored(float v);
template <> __device__ __forceinline__ float as_stored<float>(float v) { return v; }
template <> __device__ __forceinline__ float as_stored<bf16_t>(float v) { return bf16_to_f32(f32_to_bf16(v)); }

}  // namespace cmoe
