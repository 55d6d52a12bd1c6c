// Which cache entries stay when a window is cut to a budget, and the row lists of the repacking, gfx950.
//
// Per stream: the first n_first and last n_last entries, then those of the largest accumulated weight, ties to the lowest
// index, NaN last, up to the budget; kept in their order.  One workgroup a stream: weights become unsigned integers of the same
// order, held in registers (up to 32 a thread), three passes of LDS counters over 11, 11 and 10 bits find the smallest kept one and
// how many of its equals stay, and one count of the larger and of the equal ones before every entry places what is kept.
// (11 bits hold the exponent and two more, so that sums of softmax weights, within a few powers of two of each other, spread over
// enough counters.)  All of it is integer work: bit exact, the same from run to run.  Latency bounds it: MEASURED
#include "common.h"

namespace {

struct Params {
  const float* __restrict__ weight;
  const int32_t* __restrict__ kv_len;
  const int32_t* __restrict__ bt_old;
  const int32_t* __restrict__ bt_new;
  int32_t* kept;                         // (written, and read back by other threads of the workgroup)
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
  constexpr int ROUNDS = HELD ? HELD : 32;                 // entries of a thread that are placed at once
  __shared__ int s_bins[kBins];
  __shared__ int s_wave[kWaves];
  __shared__ int s_digit, s_left;
  __shared__ int s_above[ROUNDS * kWaves], s_equal[ROUNDS * kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, stream = blockIdx.x;
  const int row_old = p.max_blocks_old * CS_KV_BLOCK;
  const int n = max(0, min(p.kv_len[stream], row_old)), keep = min(n, p.budget);
  const float* weight = p.weight + static_cast<int64_t>(stream) * row_old;
  const int first = p.n_first, last = max(0, n - min(p.n_last, n));
  const int rounds = (n + kThreads - 1) / kThreads;
  auto rank_at = [&](int j) __attribute__((always_inline)) { return rank_of(weight[j], j < first || j >= last); };
  uint32_t held[HELD ? HELD : 1];
  if (HELD) {
    float w[HELD ? HELD : 1];
#pragma unroll
    for (int i = 0; i < HELD; ++i) w[i] = i * kThreads + tid < n ? weight[i * kThreads + tid] : 0.0f;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      const int j = i * kThreads + tid;
      held[i] = rank_of(w[i], j < first || j >= last);
    }
  }
  auto rank = [&](int i, int j) __attribute__((always_inline)) { return HELD ? held[HELD ? i : 0] : rank_at(j); };

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
      auto count = [&](int i) __attribute__((always_inline)) {
        const int j = i * kThreads + tid;
        if (j >= n) return;
        const uint32_t r = rank(i, j);
        if ((r & mask) == prefix) atomicAdd(&s_bins[(r >> shift) & ((1u << bits) - 1)], 1);
      };
      if (HELD) {
#pragma unroll
        for (int i = 0; i < HELD; ++i)
          if (i < rounds) count(i);
      } else {
        for (int i = 0; i < rounds; ++i) count(i);
      }
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
      for (int w = 0; w < kWaves; ++w) before += w < wave ? s_wave[w] : 0;
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
  const int64_t list = static_cast<int64_t>(stream) * p.budget;
  const int32_t* ids_old = p.bt_old + static_cast<int64_t>(stream) * p.max_blocks_old;
  const int32_t* ids_new = p.bt_new + static_cast<int64_t>(stream) * p.max_blocks_new;
  float* weight_new = p.weight_new ? p.weight_new + static_cast<int64_t>(stream) * p.max_blocks_new * CS_KV_BLOCK : nullptr;
  const bool all = keep == n;
  int above0 = 0, equal0 = 0;            // before this lot of entries
  for (int i0 = 0; i0 < rounds && keep > 0; i0 += ROUNDS) {
    auto marks = [&](int i, uint64_t* above, uint64_t* equal) __attribute__((always_inline)) {
      const int j = (i0 + i) * kThreads + tid;
      const uint32_t r = j < n ? rank(i, j) : 0u;
      *above = __ballot(j < n && (all || r > prefix));
      *equal = __ballot(j < n && !all && r == prefix);
    };
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) {
      uint64_t a = 0, e = 0;
      if (i0 + i < rounds) marks(i, &a, &e);
      if (lane == 0) {
        s_above[i * kWaves + wave] = __popcll(a);
        s_equal[i * kWaves + wave] = __popcll(e);
      }
    }
    __syncthreads();
    // exclusive sums over (round, wave), by the first wave, ROUNDS * kWaves / 64 neighbours a lane
    constexpr int PER = (ROUNDS * kWaves + 63) / 64;
    if (wave == 0) {
      int ca[PER], ce[PER], sa = 0, se = 0;
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        const int x = lane * PER + k;
        ca[k] = x < ROUNDS * kWaves ? s_above[x] : 0;
        ce[k] = x < ROUNDS * kWaves ? s_equal[x] : 0;
        sa += ca[k];
        se += ce[k];
      }
      int ia = sa, ie = se;
#pragma unroll
      for (int k = 1; k < 64; k <<= 1) {
        const int ua = __shfl_up(ia, k), ue = __shfl_up(ie, k);
        if (lane >= k) {
          ia += ua;
          ie += ue;
        }
      }
      ia += above0 - sa;
      ie += equal0 - se;
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        const int x = lane * PER + k;
        if (x < ROUNDS * kWaves) {
          s_above[x] = ia;
          s_equal[x] = ie;
        }
        ia += ca[k];
        ie += ce[k];
      }
      if (lane == 63) {
        s_digit = ia;
        s_left = ie;
      }
    }
    __syncthreads();
    const uint64_t lower = (1ull << lane) - 1;
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) {
      if (i0 + i >= rounds) break;
      uint64_t a, e;
      marks(i, &a, &e);
      const int before = s_equal[i * kWaves + wave] + __popcll(e & lower);
      const bool stays = (a >> lane & 1) || ((e >> lane & 1) && before < left);
      if (stays) {
        const int j = (i0 + i) * kThreads + tid;
        const int at = s_above[i * kWaves + wave] + __popcll(a & lower) + min(before, left);
        p.kept[list + at] = j;
      }
    }
    above0 = s_digit;
    equal0 = s_left;
    if (!HELD) __syncthreads();
  }
  // slots of what is kept, in its order: four entries of a thread at once
  __syncthreads();
  for (int i0 = 0; i0 < p.budget; i0 += 4 * kThreads) {
    int j[4], id_old[4], id_new[4];
    float w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = i0 + k * kThreads + tid;
      j[k] = i < keep ? p.kept[list + i] : -1;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      id_old[k] = j[k] < 0 ? 0 : ids_old[j[k] / CS_KV_BLOCK];
      id_new[k] = j[k] < 0 ? 0 : ids_new[(i0 + k * kThreads + tid) / CS_KV_BLOCK];
      w[k] = j[k] < 0 ? 0.0f : weight[j[k]];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = i0 + k * kThreads + tid;
      if (i >= p.budget) break;
      const bool none = j[k] < 0;
      if (none) p.kept[list + i] = -1;
      p.src_slot[list + i] = none ? -1 : id_old[k] * CS_KV_BLOCK + j[k] % CS_KV_BLOCK;
      p.dst_slot[list + i] = none ? -1 : id_new[k] * CS_KV_BLOCK + i % CS_KV_BLOCK;
      p.delta[list + i] = none || !p.renumber ? 0 : i - j[k];
      if (weight_new && !none) weight_new[i] = w[k];
    }
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
  const dim3 grid(static_cast<unsigned>(n_streams));
  hipStream_t st = cs::as_stream(stream);
  const int entries = max_blocks_old * CS_KV_BLOCK;        // of the widest row there may be
  if (entries <= kThreads) hipLaunchKernelGGL(plan_evict_kernel<1>, grid, dim3(kThreads), 0, st, p);
  else if (entries <= 4 * kThreads) hipLaunchKernelGGL(plan_evict_kernel<4>, grid, dim3(kThreads), 0, st, p);
  else if (entries <= 16 * kThreads) hipLaunchKernelGGL(plan_evict_kernel<16>, grid, dim3(kThreads), 0, st, p);
  else if (entries <= 32 * kThreads) hipLaunchKernelGGL(plan_evict_kernel<32>, grid, dim3(kThreads), 0, st, p);
  else hipLaunchKernelGGL(plan_evict_kernel<0>, grid, dim3(kThreads), 0, st, p);
  return cs::note_hip(hipGetLastError());
}
