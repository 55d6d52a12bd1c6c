// Which cache entries stay when a window is cut to a budget, and the row lists of the repacking, gfx950.
//
// Per stream: the first n_first and last n_last entries, then those of the largest accumulated weight, ties to the lowest
// index, NaN last, up to the budget; kept in their order.  One workgroup a stream: weights become unsigned integers of the same
// order, four passes of 256 LDS counters find the smallest kept one and how many of its equals stay, and a pass in index order
// places what is kept by counting across lanes and waves.  All of it is integer work: bit exact, the same from run to run.
#include "common.h"

namespace {

struct Params {
  const float* __restrict__ weight;
  const int32_t* __restrict__ kv_len;
  const int32_t* __restrict__ bt_old;
  const int32_t* __restrict__ bt_new;
  int32_t* __restrict__ kept;
  int32_t* __restrict__ src_slot;
  int32_t* __restrict__ dst_slot;
  int32_t* __restrict__ delta;
  int32_t* __restrict__ kv_len_new;
  float* __restrict__ weight_new;
  int32_t max_blocks_old, max_blocks_new, budget, n_first, n_last, renumber;
};

constexpr int kThreads = 1024;

// Unsigned integers in the order of the weights: NaN, then -inf .. +inf (-0 and +0 alike), then what stays whatever its weight.
__device__ __forceinline__ uint32_t rank_of(float w, bool fixed) {
  if (fixed) return 0xffffffffu;
  const uint32_t u = __float_as_uint(w);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0;
  if ((u & 0x7fffffffu) == 0) return 0x80000000u;
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kThreads) void plan_evict_kernel(Params p) {
  __shared__ int s_hist[256];
  __shared__ int s_digit, s_left;
  __shared__ int s_wave[2][kThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, stream = blockIdx.x;
  const int row_old = p.max_blocks_old * CS_KV_BLOCK;
  const int n = max(0, min(p.kv_len[stream], row_old)), keep = min(n, p.budget);
  const float* weight = p.weight + static_cast<int64_t>(stream) * row_old;
  const int first = p.n_first, last = max(0, n - min(p.n_last, n));
  auto rank = [&](int j) __attribute__((always_inline)) { return rank_of(weight[j], j < first || j >= last); };

  // ---- the smallest rank that stays, and how many entries of that rank
  uint32_t prefix = 0, mask = 0;
  int left = keep;                       // entries still to find among those that share the prefix
  if (keep < n && keep > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) s_hist[tid] = 0;
      __syncthreads();
      for (int j = tid; j < n; j += kThreads) {
        const uint32_t r = rank(j);
        if ((r & mask) == prefix) atomicAdd(&s_hist[(r >> shift) & 255u], 1);
      }
      __syncthreads();
      if (tid < 64) {                    // from the largest digit down: the digit at which `left` is reached
        int c[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          c[i] = s_hist[255 - 4 * tid - i];
          sum += c[i];
        }
        int incl = sum;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const int up = __shfl_up(incl, d);
          if (tid >= d) incl += up;
        }
        int before = incl - sum;
        if (before < left && left <= incl) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (before < left && left <= before + c[i]) {
              s_digit = 255 - 4 * tid - i;
              s_left = left - before;
            }
            before += c[i];
          }
        }
      }
      __syncthreads();
      prefix |= static_cast<uint32_t>(s_digit) << shift;
      mask |= 255u << shift;
      left = s_left;
      __syncthreads();
    }
  }

  // ---- lists, in index order
  const int64_t list = static_cast<int64_t>(stream) * p.budget;
  const int32_t* ids_old = p.bt_old + static_cast<int64_t>(stream) * p.max_blocks_old;
  const int32_t* ids_new = p.bt_new + static_cast<int64_t>(stream) * p.max_blocks_new;
  float* weight_new = p.weight_new ? p.weight_new + static_cast<int64_t>(stream) * p.max_blocks_new * CS_KV_BLOCK : nullptr;
  int at0 = 0, equal0 = 0;               // kept entries and entries of the smallest rank before this round
  for (int j0 = 0; j0 < n && keep > 0; j0 += kThreads) {
    const int j = j0 + tid;
    const uint32_t r = j < n ? rank(j) : 0u;
    const bool above = j < n && (keep == n || r > prefix), equal = j < n && keep < n && r == prefix;
    const uint64_t lower = (1ull << lane) - 1, eq = __ballot(equal);
    if (lane == 0) s_wave[0][wave] = __popcll(eq);
    __syncthreads();
    int eq_before = equal0, eq_all = equal0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
      const int c = s_wave[0][w];
      if (w < wave) eq_before += c;
      eq_all += c;
    }
    const bool stays = above || (equal && eq_before + __popcll(eq & lower) < left);
    const uint64_t st = __ballot(stays);
    if (lane == 0) s_wave[1][wave] = __popcll(st);
    __syncthreads();
    int at = at0, all = at0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
      const int c = s_wave[1][w];
      if (w < wave) at += c;
      all += c;
    }
    at += __popcll(st & lower);
    if (stays) {
      p.kept[list + at] = j;
      p.src_slot[list + at] = ids_old[j / CS_KV_BLOCK] * CS_KV_BLOCK + j % CS_KV_BLOCK;
      p.dst_slot[list + at] = ids_new[at / CS_KV_BLOCK] * CS_KV_BLOCK + at % CS_KV_BLOCK;
      p.delta[list + at] = p.renumber ? at - j : 0;
      if (weight_new) weight_new[at] = weight[j];
    }
    at0 = all;
    equal0 = eq_all;
  }
  for (int i = keep + tid; i < p.budget; i += kThreads) {
    p.kept[list + i] = -1;
    p.src_slot[list + i] = -1;
    p.dst_slot[list + i] = -1;
    p.delta[list + i] = 0;
  }
  if (tid == 0) p.kv_len_new[stream] = keep;
}

}  // namespace

extern "C" int cs_plan_evict(const float* weight, const int32_t* kv_len, const int32_t* block_table_old, int32_t max_blocks_old,
                             const int32_t* block_table_new, int32_t max_blocks_new, int32_t n_streams, int32_t budget, int32_t n_first,
                             int32_t n_last, int32_t renumber, int32_t* kept, int32_t* src_slot, int32_t* dst_slot, int32_t* delta,
                             int32_t* kv_len_new, float* weight_new, void* stream) {
  if (n_streams < 0 || budget < 1 || n_first < 0 || n_last < 0 || max_blocks_old < 1 || max_blocks_new < 1) return CS_EINVAL;
  if (max_blocks_old > 0x7fffffff / CS_KV_BLOCK - kThreads || max_blocks_new > 0x7fffffff / CS_KV_BLOCK - kThreads) return CS_EUNSUPPORTED;
  // what may stay has to fit a row of the new table
  if ((budget < max_blocks_old * CS_KV_BLOCK ? budget : max_blocks_old * CS_KV_BLOCK) > max_blocks_new * CS_KV_BLOCK) return CS_EINVAL;
  if (n_streams == 0) return CS_OK;
  if (!weight || !kv_len || !block_table_old || !block_table_new || !kept || !src_slot || !dst_slot || !delta || !kv_len_new) return CS_EINVAL;
  Params p;
  p.weight = weight;
  p.kv_len = kv_len;
  p.bt_old = block_table_old;
  p.bt_new = block_table_new;
  p.kept = kept;
  p.src_slot = src_slot;
  p.dst_slot = dst_slot;
  p.delta = delta;
  p.kv_len_new = kv_len_new;
  p.weight_new = weight_new;
  p.max_blocks_old = max_blocks_old;
  p.max_blocks_new = max_blocks_new;
  p.budget = budget;
  p.n_first = n_first;
  p.n_last = n_last;
  p.renumber = renumber;
  hipLaunchKernelGGL(plan_evict_kernel, dim3(static_cast<unsigned>(n_streams)), dim3(kThreads), 0, cs::as_stream(stream), p);
  return cs::note_hip(hipGetLastError());
}
