// Eight elements of a row, bf16 or fp32, on their way through a lane: streamed (non-temporal), as no byte is used twice.
// Internal to the library.
#pragma once

#include "kv4.h"

namespace cs {

template <bool kBf16>
struct Eight;
template <>
struct Eight<true> {                     // eight bf16: one 16-byte vector
  u32x4 v;
  __device__ __forceinline__ void load(const uint16_t* p) { v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)); }
  __device__ __forceinline__ void get(float* f) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void copy_to(uint16_t* p) const { __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p)); }      // (bit for bit)
  static __device__ __forceinline__ void store(uint16_t* p, const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32v2 x = {f[2 * i], f[2 * i + 1]};
      w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16v2));
    }
    __builtin_nontemporal_store(u32x4{w[0], w[1], w[2], w[3]}, reinterpret_cast<u32x4*>(p));
  }
};
template <>
struct Eight<false> {
  u32x4 v, w;
  __device__ __forceinline__ void load(const float* p) {
    v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + 4));
  }
  __device__ __forceinline__ void get(float* f) const {
    f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    f[4] = __uint_as_float(w.x); f[5] = __uint_as_float(w.y); f[6] = __uint_as_float(w.z); f[7] = __uint_as_float(w.w);
  }
  __device__ __forceinline__ void copy_to(float* p) const {
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(p + 4));
  }
  static __device__ __forceinline__ void store(float* p, const float* f) {
    __builtin_nontemporal_store(u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])},
                                reinterpret_cast<u32x4*>(p));
    __builtin_nontemporal_store(u32x4{__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])},
                                reinterpret_cast<u32x4*>(p + 4));
  }
};

}  // namespace cs
