// Which cache entries stay when a window is cut to a budget, and the row lists of the repacking, gfx950.
//
// Per stream: the first n_first and last n_last entries, then those of the largest accumulated weight, ties to the lowest
// index, NaN last, up to the budget; kept in their order.  One workgroup a stream, a run of neighbouring entries a wave: weights
// become unsigned integers of the same order, held in registers (up to 24 a thread), three passes of LDS counters over 11, 11 and
// 10 bits find the smallest kept one and how many of its equals stay, and every wave counts the larger and the equal ones
// before its own and places what it keeps.  (11 bits hold the exponent and two more, so that sums of softmax weights, within a few
// powers of two of each other, spread over enough counters.)  What is kept passes through a list in LDS, so that the lists in memory
// are written in whole lines: a quarter of a wave's lanes storing to five of them took a third of the time.
// All of it is integer work: bit exact, the same from run to run.  One cache of 919 entries takes 6.2 us on the card: a launch, 14 barriers
// (four a pass, two for the lists) and one trip to memory.  64 of up to 17,630 cut to 4,096 take 22.6 us (their bytes 1.8; 46.5 with every
// pass reading memory), on a quarter of the card: the 64 CUs' vector units work 58 % of that time, LDS 16 % (a quarter of that conflicts
// of the counters), and waves wait half of theirs.  A stream of 60,000 entries, past what registers hold, takes 83 us in its one workgroup.
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

constexpr int kWaves = kThreads / 64, kBins = 2048;

// Entries a thread holds; HELD 0: any number, read anew in every pass.
template <int HELD>
__global__ __launch_bounds__(kThreads) void plan_evict_kernel(Params p) {
  // counters of the passes, then the list of what is kept
  __shared__ __attribute__((aligned(16))) char s_mem[kBins * 4 > HELD * kThreads * 2 ? kBins * 4 : HELD * kThreads * 2];
  int* const s_bins = reinterpret_cast<int*>(s_mem);
  uint16_t* const s_list = reinterpret_cast<uint16_t*>(s_mem);
  __shared__ int s_wave[kWaves], s_above[kWaves], s_equal[kWaves];
  __shared__ int s_digit, s_left;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), stream = blockIdx.x;
  const int row_old = p.max_blocks_old * CS_KV_BLOCK;
  const int n = max(0, min(p.kv_len[stream], row_old)), keep = min(n, p.budget);
  const float* weight = p.weight + static_cast<int64_t>(stream) * row_old;
  const int first = p.n_first, last = max(0, n - min(p.n_last, n));
  const int rounds = (n + kThreads - 1) / kThreads;        // of 64 entries a wave
  const int j0 = wave * rounds * 64 + lane;                // entry i of a thread: j0 + 64 i
  const int32_t* ids_old = p.bt_old + static_cast<int64_t>(stream) * p.max_blocks_old;
  const int32_t* ids_new = p.bt_new + static_cast<int64_t>(stream) * p.max_blocks_new;
  uint32_t held[HELD ? HELD : 1];
  if (HELD) {
    float w[HELD ? HELD : 1];
#pragma unroll
    for (int i = 0; i < HELD; ++i) w[i] = i < rounds && j0 + 64 * i < n ? weight[j0 + 64 * i] : 0.0f;
#pragma unroll
    for (int i = 0; i < HELD; ++i) held[i] = rank_of(w[i], j0 + 64 * i < first || j0 + 64 * i >= last);
  }
  constexpr int kAtOnce = 8;             // entries that a thread asks for together where it holds none
  auto each = [&](auto f) __attribute__((always_inline)) {
    if (HELD) {
#pragma unroll
      for (int i = 0; i < HELD; ++i)
        if (i < rounds) f(i, held[HELD ? i : 0]);
    } else {
      for (int i0 = 0; i0 < rounds; i0 += kAtOnce) {
        float w[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) w[k] = weight[min(j0 + 64 * (i0 + k), n - 1)];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
          const int j = j0 + 64 * (i0 + k);
          if (i0 + k < rounds) f(i0 + k, rank_of(w[k], j < first || j >= last));
        }
      }
    }
  };

  // ---- the smallest rank that stays, and how many entries of that rank
  uint32_t prefix = 0, mask = 0;
  int left = keep;                       // entries still to find among those that share the prefix
  if (keep < n && keep > 0) {
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
      s_bins[tid] = 0;
      s_bins[kThreads + tid] = 0;
      __syncthreads();
      each([&](int i, uint32_t r) __attribute__((always_inline)) {
        if (j0 + 64 * i >= n) return;
        if ((r & mask) == prefix) atomicAdd(&s_bins[(r >> shift) & ((1u << bits) - 1)], 1);
      });
      __syncthreads();
      // from the largest digit down, two digits a thread: the one at which `left` is reached
      const int d = kBins - 1 - 2 * tid, c0 = s_bins[d], c1 = s_bins[d - 1];
      int incl = c0 + c1;
#pragma unroll
      for (int k = 1; k < 64; k <<= 1) {
        const int up = __shfl_up(incl, k);
        if (lane >= k) incl += up;
      }
      if (lane == 63) s_wave[wave] = incl;
      __syncthreads();
      int before = incl - c0 - c1;
#pragma unroll
      for (int k = 0; k < kWaves; ++k) before += k < wave ? s_wave[k] : 0;
      if (before < left && left <= before + c0 + c1) {     // (one thread)
        const bool second = left > before + c0;
        s_digit = second ? d - 1 : d;
        s_left = left - before - (second ? c0 : 0);
      }
      __syncthreads();
      prefix |= static_cast<uint32_t>(s_digit) << shift;
      mask |= ((1u << bits) - 1) << shift;
      left = s_left;
    }
  }

  // ---- lists, in index order: before an entry stay the larger ones before it, and of its equals no more than `left`
  const bool all = keep == n;
  auto marks = [&](int i, uint32_t r, uint64_t* above, uint64_t* equal) __attribute__((always_inline)) {
    const bool there = j0 + 64 * i < n;
    *above = __ballot(there && (all || r > prefix));
    *equal = __ballot(there && !all && r == prefix);
  };
  int above = 0, equal = 0;
  each([&](int i, uint32_t r) __attribute__((always_inline)) {
    uint64_t a, e;
    marks(i, r, &a, &e);
    above += __popcll(a);
    equal += __popcll(e);
  });
  if (lane == 0) {
    s_above[wave] = above;
    s_equal[wave] = equal;
  }
  __syncthreads();                       // (the counters have been read, too)
  above = equal = 0;
#pragma unroll
  for (int k = 0; k < kWaves; ++k) {
    above += k < wave ? s_above[k] : 0;
    equal += k < wave ? s_equal[k] : 0;
  }
  const int64_t list = static_cast<int64_t>(stream) * p.budget;
  float* weight_new = p.weight_new ? p.weight_new + static_cast<int64_t>(stream) * p.max_blocks_new * CS_KV_BLOCK : nullptr;
  auto put = [&](int at, int j, int old_id, int new_id, float x) __attribute__((always_inline)) {
    p.kept[list + at] = j;
    p.src_slot[list + at] = old_id * CS_KV_BLOCK + j % CS_KV_BLOCK;
    p.dst_slot[list + at] = new_id * CS_KV_BLOCK + at % CS_KV_BLOCK;
    p.delta[list + at] = p.renumber ? at - j : 0;
    if (weight_new) weight_new[at] = x;
  };
  const uint64_t lower = (1ull << lane) - 1;
  if (keep > 0)
    each([&](int i, uint32_t r) __attribute__((always_inline)) {
      uint64_t a, e;
      marks(i, r, &a, &e);
      const int before = equal + __popcll(e & lower), j = j0 + 64 * i;
      if ((a >> lane & 1) || ((e >> lane & 1) && before < left)) {
        const int at = above + __popcll(a & lower) + min(before, left);
        if (HELD) s_list[at] = static_cast<uint16_t>(j);
        else put(at, j, ids_old[j / CS_KV_BLOCK], ids_new[at / CS_KV_BLOCK], weight[j]);
      }
      above += __popcll(a);
      equal += __popcll(e);
    });
  if (HELD) {                            // four entries of a thread at once
    __syncthreads();
    for (int i0 = tid; i0 < keep; i0 += 4 * kThreads) {
      int j[4], id_old[4], id_new[4];
      float x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = min(i0 + k * kThreads, keep - 1);
        j[k] = s_list[i];
        id_old[k] = ids_old[j[k] / CS_KV_BLOCK];
        id_new[k] = ids_new[i / CS_KV_BLOCK];
        x[k] = weight_new ? weight[j[k]] : 0.0f;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i0 + k * kThreads < keep) put(i0 + k * kThreads, j[k], id_old[k], id_new[k], x[k]);
    }
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
  if (max_blocks_old > 0x7fffffff / CS_KV_BLOCK - kThreads || max_blocks_new > 0x7fffffff / CS_KV_BLOCK - kThreads || budget > (1 << 30) ||
      n_streams >= (1 << 22))              // (2^32 threads)
    return CS_EUNSUPPORTED;
  // what may stay has to fit a row of the new table
  if ((budget < max_blocks_old * CS_KV_BLOCK ? budget : max_blocks_old * CS_KV_BLOCK) > max_blocks_new * CS_KV_BLOCK) return CS_EINVAL;
  if (n_streams == 0) return CS_OK;
  if (!weight || !kv_len || !block_table_old || !block_table_new || !kept || !src_slot || !dst_slot || !delta || !kv_len_new) return CS_EINVAL;
  if (kv_len_new == kv_len || weight_new == weight) return CS_EINVAL;
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
  const dim3 grid(static_cast<unsigned>(n_streams));
  hipStream_t st = cs::as_stream(stream);
  const int entries = max_blocks_old * CS_KV_BLOCK;        // of the widest row there may be
  if (entries <= kThreads) hipLaunchKernelGGL(plan_evict_kernel<1>, grid, dim3(kThreads), 0, st, p);
  else if (entries <= 4 * kThreads) hipLaunchKernelGGL(plan_evict_kernel<4>, grid, dim3(kThreads), 0, st, p);
  else if (entries <= 12 * kThreads) hipLaunchKernelGGL(plan_evict_kernel<12>, grid, dim3(kThreads), 0, st, p);
  else if (entries <= 24 * kThreads) hipLaunchKernelGGL(plan_evict_kernel<24>, grid, dim3(kThreads), 0, st, p);
  else hipLaunchKernelGGL(plan_evict_kernel<0>, grid, dim3(kThreads), 0, st, p);
  return cs::note_hip(hipGetLastError());
}
