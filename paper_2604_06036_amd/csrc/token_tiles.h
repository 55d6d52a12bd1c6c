// Tiles of consecutive query tokens of one stream, and lane exchanges of the kernels that take them.  Internal to the library.
#pragma once

#include "common.h"

namespace cs {

struct TokenTile {
  int stream, first, count;              // its stream, its first token, how many (1 .. tile)
};

// Sum over the lanes up to and with this one.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);      // row_shr:1, 2, 4, 8: inside each 16 lanes
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // row_bcast:15: lane 15 to the second 16, 47 to the fourth
  return v + __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);      // row_bcast:31: lane 31 to the upper half
}

// Tile `target` of the launch's order: stream by stream, `tile` tokens each, a stream's last tile holding what is left.  cu_q's
// tokens from n_q on do not exist.  Every wave scans the streams for itself, 64 at a time; false: there are fewer tiles.
__device__ __forceinline__ bool find_token_tile(const int32_t* __restrict__ cu_q, int n_streams, int64_t n_q, int tile, int target, TokenTile* t) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int s0 = 0; s0 < n_streams; s0 += 64) {
    const int s = s0 + lane;
    int a = 0, n = 0;
    if (s < n_streams) {
      a = cu_q[s];
      n = max(0, min(cu_q[s + 1], static_cast<int>(n_q)) - a);
    }
    const int tiles = (n + tile - 1) / tile;
    const int incl = wave_scan(tiles);
    const int total = __builtin_amdgcn_readlane(incl, 63);
    if (target >= before + total) {
      before += total;
      continue;
    }
    const int l = __builtin_amdgcn_readfirstlane(__ffsll(static_cast<unsigned long long>(__ballot(before + incl > target))) - 1);
    const int skip = (target - before - __builtin_amdgcn_readlane(incl - tiles, l)) * tile;
    t->stream = s0 + l;
    t->first = __builtin_amdgcn_readlane(a, l) + skip;
    t->count = min(tile, __builtin_amdgcn_readlane(n, l) - skip);
    return true;
  }
  return false;
}

// Tiles that n_q tokens of n_streams streams make at most: every stream one of a single token, the other tokens in whole ones.
inline int64_t most_token_tiles(int64_t n_q, int32_t n_streams, int tile) {
  const int64_t one = n_q < n_streams ? n_q : n_streams;
  return one + (n_q - one) / tile;
}

// What an operation makes of a value and the one of lane ^ 32, lane ^ 16: the swaps leave both lanes' values in both lanes.
template <class F>
__device__ __forceinline__ float with_lane32(float x, const F& f) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <class F>
__device__ __forceinline__ float with_lane16(float x, const F& f) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float plus(float a, float b) { return a + b; }
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float smaller(float a, float b) { return fminf(a, b); }

template <int kCtrl>
__device__ __forceinline__ uint32_t lane_dpp(uint32_t x) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), kCtrl, 0xf, 0xf, true));
}

// Largest of the wave, or of its aligned groups of `kLanes` lanes.
template <int kLanes>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
  if (kLanes > 1) x = max(x, lane_dpp<0xb1>(x));
  if (kLanes > 2) x = max(x, lane_dpp<0x4e>(x));
  if (kLanes > 4) x = max(x, lane_dpp<0x141>(x));
  if (kLanes > 8) x = max(x, lane_dpp<0x140>(x));
  if (kLanes > 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max(r[0], r[1]);
  }
  if (kLanes > 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    x = max(r[0], r[1]);
  }
  return x;
}

}  // namespace cs
