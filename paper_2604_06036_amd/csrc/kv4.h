// 4-bit cache rows on gfx950: blocks of 32 elements along head_dim, each element sign + three magnitude bits
// ({0, .5, 1, 1.5, 2, 3, 4, 6}), one power of two (8 bits, biased by 127; 255: the block holds no numbers) per block.
// Internal to the library.
#pragma once

#include "common.h"

namespace cs {

typedef __attribute__((ext_vector_type(2))) float f32v2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16v2;

constexpr int kKv4Block = 32;            // elements that share a scale
constexpr int64_t kMostThreads = 0xffffffffll;   // of a launch, along one axis of its grid
constexpr uint32_t kKv4NoNumber = 255;   // scale byte of a block that held a NaN or an infinity
constexpr uint32_t kKv4Large = 253;      // least scale byte of a block with elements past the largest finite number

// Scale byte of a block whose largest magnitude has the given fp32 bits: the least power of two s with amax <= 7 s.
// (7 is as far above 6, the largest value, as 5 is above 4, so that saturating it costs no more than the rounding between
// 4 and 6; and 7 is no value of the grid: rows that are turned again never have their maximum on the border.)
__device__ __forceinline__ uint32_t kv4_scale_byte(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return kKv4NoNumber;
  const int e = static_cast<int>((amax_bits + 0x1fffffu) >> 23) - 2;
  return e < 1 ? 1u : static_cast<uint32_t>(e);
}

// The scale as a number (bytes 1..254; 0 is read as 1).
__device__ __forceinline__ float kv4_scale(uint32_t byte) { return __uint_as_float((byte ? byte : 1u) << 23); }

// Eight values -> eight codes (element 0 in the lowest nibble): nearest, ties to the even code, saturating at 6.
__device__ __forceinline__ uint32_t kv4_pack8(const float* x, float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
  return w;
}

// Eight codes -> fp32 (exact).
__device__ __forceinline__ void kv4_unpack8(uint32_t w, float scale, float* x) {
  const f32v2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0);
  const f32v2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
  const f32v2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2);
  const f32v2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
  x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
  x[4] = c.x; x[5] = c.y; x[6] = d.x; x[7] = d.y;
}

// Eight codes -> eight bf16 (exact: a value has one fraction bit).
__device__ __forceinline__ u32x4 kv4_unpack8_bf16(uint32_t w, float scale) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3))};
}

__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Element strides of a 4-bit pool: whole blocks.
inline bool kv4_strides(int64_t a, int64_t b, int64_t c) { return a % kKv4Block == 0 && b % kKv4Block == 0 && c % kKv4Block == 0; }

}  // namespace cs
