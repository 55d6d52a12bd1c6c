// Attention weight that every cache entry received, summed over queries and query heads, gfx950.
//
// weight[s][j] = decay weight[s][j] + sum_{t, h} exp(scale q[t][h] . K_j - lse[t][h]) over the queries t of stream s that see j.
// A wave holds 64 keys (32 of an fp32 cache) as matrix operands in registers for the whole launch, so that a key is read and,
// from a 4-bit cache, converted once; query rows pass through LDS in steps of 32.  With S = Q K^T a lane owns one key and 16
// rows: weights add up in a register, in a fixed order, and no two lanes add to the same place.  Shares of a stream's rows and
// kv heads leave partial sums that a last launch adds in order, so results are the same bits from run to run.
// Without statistics from the caller the same kernel computes S^T = K Q^T first (operands swapped: a lane owns one query and
// 16 keys), which gives a row's maximum and sum over the workgroup's keys in registers; a second launch joins the key ranges.
// fp32 operands are sums of three bf16 numbers: three products for 4-bit keys (exact in bf16), six for fp32 keys.
// 16 streams of up to 389 queries of 28 heads over up to 1,100 4-bit entries take 46 to 49 us, 437 to 466 TFLOP/s: while CUs are busy their
// matrix units work 27 % and their vector units 50 % of the time (an exponential, a product and an add per row and key), a wave's one
// after the other, and a wave waits half of its own time.  64 queries over 17,630 16-bit entries with statistics to find first (two sweeps)
// take 52 to 55 us: matrix units 15 and 20 %, vector units 41 and 43 %, 828 workgroups on the 512 places that the statistics kernel's
// registers leave, and on 768 for the weights.  2,082 queries over 17,630 entries with statistics at hand: 288 to 301 us.
#include <math.h>

#include <type_traits>

#include "kv4.h"

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;

struct Params {
  const void* __restrict__ q;
  const float* __restrict__ lse;         // natural logarithms [n_q][n_q_heads]
  const void* __restrict__ k;
  const uint8_t* __restrict__ k_scales;
  const int32_t* __restrict__ cu_q;
  const int32_t* __restrict__ q_pos;
  const int32_t* __restrict__ kv_len;
  const int32_t* __restrict__ block_table;
  const float* weight_in;
  float* weight_out;
  float* ws_lse;                         // [n_q][n_q_heads]
  cs::f32v2* ws_stat;                    // [n_q][n_q_heads][key_tiles]: maximum (log2 units), sum
  float* ws_part;                        // [chunks][n_kv_heads][n_streams][max_blocks * 16]
  int64_t n_q, stride_slot, stride_head;
  int32_t max_blocks, n_streams, n_q_heads, n_kv_heads, group, key_tiles, chunks, shares_per_xcd;
  uint32_t group_inv;                    // 2^32 / group, rounded up (group 1: 0): rows below 2^28 are divided by a high product
  float scale_log2e, decay;
};

constexpr int kStep = 32;                // query rows of a step
// Steps of a stream that a workgroup sorts out (those that see no key of its tile are left out); of a share, that it does not sort:
// 4 streams of 424 queries over 919 entries take 29 us at 8, 33 at 2, the prefill of 16 streams 49 us at 8, 53 at 64.
constexpr int kListed = 2048, kFewSteps = 8;
// Workgroups wanted, steps that a share of a stream's rows has at least.  16 streams of 389 queries over 1,100 entries: 49 us, 58 with
// half as many workgroups, 48 with twice (4 x 424 x 919: 29, 25 and 29.5); 64 queries over 17,630 entries: 55 us at 4 steps, 59 at 2, 60 at 8.
constexpr int kGroups = 1536, kLeast = 4;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

constexpr int keys_per_wave(int cache) { return cache == CS_F32 ? 32 : 64; }
constexpr int keys_per_tile(int cache) { return 4 * keys_per_wave(cache); }

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const cs::f32v2 v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, cs::bf16v2));
}

// The next bf16 part of eight numbers, taken off them.
__device__ __forceinline__ cs::u32x4 next_part(float* x) {
  cs::u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w[i] = pack2(x[2 * i], x[2 * i + 1]);
    x[2 * i] -= __uint_as_float(w[i] << 16);
    x[2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u);
  }
  return w;
}

__device__ __forceinline__ int token_of(const Params& p, int row) { return p.group_inv ? static_cast<int>(__umulhi(static_cast<uint32_t>(row), p.group_inv)) : row; }

__device__ __forceinline__ int stream_entries(const Params& p, int s) { return min(p.kv_len[s], p.max_blocks * CS_KV_BLOCK); }

template <int D, int CACHE, int QP, bool STATS>
__global__ __launch_bounds__(256) void attn_weights_kernel(Params p) {
  constexpr int STEPS = D / 16, KP = CACHE == CS_F32 ? 3 : 1, KB = keys_per_wave(CACHE) / 32;
  constexpr int TILE = keys_per_tile(CACHE);
  constexpr int QROW = D + 8;                              // padded LDS row
  constexpr int CHUNKS = kStep * D / 8 / 256;              // 8-element pieces of a step's rows a thread moves (D 64: 1, D 128: 2)
  constexpr int EB = CACHE == CS_BF16 ? 2 : 4;             // bytes of a key's element (caches that are not of 4 bits)
  constexpr int KROW = D * EB + 16;                        // padded LDS row of a key on its way, bytes
  constexpr int Q_BYTES = 2 * QP * kStep * QROW * 2, K_BYTES = CACHE == CS_KV4 ? 0 : 4 * 32 * KROW;
  __shared__ __attribute__((aligned(16))) char s_mem[Q_BYTES > K_BYTES ? Q_BYTES : K_BYTES];
  uint16_t (*const s_q)[QP][kStep * QROW] = reinterpret_cast<uint16_t (*)[QP][kStep * QROW]>(s_mem);
  __shared__ __attribute__((aligned(16))) float s_lse[2][kStep];
  __shared__ __attribute__((aligned(16))) int s_pos[2][kStep];
  __shared__ int s_none;                                   // whether a row's statistics were no number
  __shared__ float s_m[2][4][kStep], s_l[2][4][kStep];
  __shared__ uint16_t s_list[kListed];
  __shared__ uint32_t s_bits[kListed / 32];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 31, h = lane >> 5;
  // ---- which keys, which rows
  // (workgroups go round the eight XCDs: where there are enough, the key tiles that read the same rows follow each other on one)
  int kt, share_of;
  if (p.shares_per_xcd) {
    const int turn = static_cast<int>(blockIdx.x / 8);
    kt = turn % p.key_tiles;
    share_of = turn / p.key_tiles * 8 + static_cast<int>(blockIdx.x % 8);
  } else {
    kt = static_cast<int>(blockIdx.x) % p.key_tiles;
    share_of = static_cast<int>(blockIdx.x) / p.key_tiles;
  }
  const int chunk = share_of % p.chunks, kvh = share_of / p.chunks % p.n_kv_heads, stream = share_of / p.chunks / p.n_kv_heads;
  if (stream >= p.n_streams) return;
  const int entries = stream_entries(p, stream), q0 = p.cu_q[stream];
  const int rows = max(0, min(p.cu_q[stream + 1], static_cast<int>(p.n_q)) - q0) * p.group;
  if (kt * TILE >= entries) return;
  const int steps = (rows + kStep - 1) / kStep;
  const int tile0 = kt * TILE, key0 = tile0 + wave * 32 * KB;

  // ---- keys, asked for before the steps are looked over.  4-bit: lane n is a key, of whose elements it takes 64 i + 32 h + 0..31, one
  // block.  Others: whole rows by neighbouring lanes, to change places in LDS (16 bytes of each of 32 rows a load would cost the
  // address unit four times as much).
  const int32_t* ids = p.block_table + static_cast<int64_t>(stream) * p.max_blocks;
  constexpr int LANES = D * EB / 16, ROWS = 64 / LANES;    // lanes of a row, rows of a load
  constexpr int RAW = CACHE == CS_KV4 ? D / 64 : 32 / ROWS;
  cs::u32x4 k_raw[KB][RAW];
  uint32_t k_scale[KB];
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
    k_scale[kb] = 0;
    if (CACHE == CS_KV4) {
      const int key = min(key0 + 32 * kb + n, entries - 1);
      const int64_t at = (static_cast<int64_t>(ids[key / CS_KV_BLOCK]) * CS_KV_BLOCK + key % CS_KV_BLOCK) * p.stride_slot + static_cast<int64_t>(kvh) * p.stride_head;
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        k_raw[kb][i] = *reinterpret_cast<const cs::u32x4*>(static_cast<const char*>(p.k) + at / 2 + 32 * i + 16 * h);
        k_scale[kb] |= static_cast<uint32_t>(p.k_scales[at / cs::kKv4Block + 2 * i + h]) << (8 * i);
      }
    } else {
#pragma unroll
      for (int j = 0; j < RAW; ++j) {
        const int key = min(key0 + 32 * kb + ROWS * j + lane / LANES, entries - 1);
        const int64_t at = (static_cast<int64_t>(ids[key / CS_KV_BLOCK]) * CS_KV_BLOCK + key % CS_KV_BLOCK) * p.stride_slot + static_cast<int64_t>(kvh) * p.stride_head;
        k_raw[kb][j] = *reinterpret_cast<const cs::u32x4*>(static_cast<const char*>(p.k) + at * EB + 16 * (lane % LANES));
      }
    }
  }

  // ---- the steps with a row that sees a key of the tile; shares are of those.  Of all steps where they are more than the list holds, or
  // so few that sorting them out (2 us) takes longer than passing over what sees nothing.
  const bool listed = steps <= kListed && steps > kFewSteps * p.chunks;
  int n_active = steps;
  if (listed) {
    if (tid < kListed / 32) s_bits[tid] = 0;
    __syncthreads();
    for (int t = tid; t * p.group < rows; t += 256) {      // a token's rows lie in one step, or two
      if (p.q_pos[q0 + t] >= tile0) {
        const int s0 = t * p.group / kStep, s1 = (t * p.group + p.group - 1) / kStep;
        atomicOr(&s_bits[s0 / 32], 1u << (s0 % 32));
        if (s1 != s0) atomicOr(&s_bits[s1 / 32], 1u << (s1 % 32));
      }
    }
    __syncthreads();
    n_active = 0;
    for (int s0 = 0; s0 < steps; s0 += 64) {               // (every wave writes the same list)
      const int st = s0 + lane;
      const uint64_t in = static_cast<uint64_t>(s_bits[s0 / 32 + 1]) << 32 | s_bits[s0 / 32];
      if (in >> lane & 1) s_list[n_active + __popcll(in & ((1ull << lane) - 1))] = static_cast<uint16_t>(st);
      n_active += __popcll(in);
    }
    n_active = __builtin_amdgcn_readfirstlane(n_active);
    __syncthreads();
  }
  const int share = (n_active + p.chunks - 1) / p.chunks;
  const int step_begin = chunk * share, step_end = min(n_active, step_begin + share);
  auto step_at = [&](int i) __attribute__((always_inline)) { return listed ? static_cast<int>(s_list[i]) : i; };

  // ---- query rows: asked for AHEAD steps ahead (a step takes a fraction of their latency)
  constexpr int AHEAD = QP == 1 ? 4 : 2;
  constexpr int QB = QP == 1 ? 2 : 4;                      // bytes of an element
  const char* const q_base = static_cast<const char*>(p.q) + (static_cast<int64_t>(q0) * p.n_q_heads + kvh * p.group) * (D * QB);
  const float* const lse_base = STATS ? nullptr : p.lse + static_cast<int64_t>(q0) * p.n_q_heads + kvh * p.group;
  const uint32_t tok_bytes = static_cast<uint32_t>(p.n_q_heads) * (D * QB);
  cs::u32x4 raw[AHEAD][CHUNKS][QP == 1 ? 1 : 2];
  int next_pos[AHEAD];
  float next_lse[AHEAD];
  auto request = [&](int index, int at) __attribute__((always_inline)) {
    const int step = step_at(index);
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int c = tid + 256 * i, r = min(step * kStep + c / (D / 8), rows - 1), tok = token_of(p, r);
      const char* src = q_base + static_cast<uint64_t>(tok) * tok_bytes + ((r - tok * p.group) * D + 8 * (c % (D / 8))) * QB;
      raw[at][i][0] = *reinterpret_cast<const cs::u32x4*>(src);
      if (QP != 1) raw[at][i][QP == 1 ? 0 : 1] = *reinterpret_cast<const cs::u32x4*>(src + 16);
    }
    if (tid < kStep) {                                     // (used as they come when the step's turn is there: no wait in between)
      const int r = min(step * kStep + tid, rows - 1), tok = token_of(p, r);
      next_pos[at] = p.q_pos[q0 + tok];
      if (!STATS) next_lse[at] = lse_base[static_cast<int64_t>(tok) * p.n_q_heads + (r - tok * p.group)];
    }
  };
  // (STATS) a step's maxima and sums of the four waves joined, left for the launch that joins key ranges
  auto join = [&](int index, int buf) __attribute__((always_inline)) {
    const int r = step_at(index) * kStep + tid;
    if (tid < kStep && r < rows) {
      float m = s_m[buf][0][tid];
#pragma unroll
      for (int w = 1; w < 4; ++w) m = fmaxf(m, s_m[buf][w][tid]);
      float l = 0.0f;
#pragma unroll
      for (int w = 0; w < 4; ++w) l += m == -INFINITY ? s_l[buf][w][tid] : s_l[buf][w][tid] * __builtin_amdgcn_exp2f(s_m[buf][w][tid] - m);
      const int tok = token_of(p, r);
      p.ws_stat[(static_cast<int64_t>(q0 + tok) * p.n_q_heads + kvh * p.group + (r - tok * p.group)) * p.key_tiles + kt] = cs::f32v2{m, l};
    }
  };

  // ---- keys as operands: elements 64 i + 32 h + 8 w + 0..7 in step 4 i + w
  bf16x8 kf[KP][KB][STEPS];
  auto unpack = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      char* const mine = s_mem + wave * 32 * KROW;         // (a wave's own; its LDS operations keep their order)
      if (CACHE != CS_KV4) {
#pragma unroll
        for (int j = 0; j < RAW; ++j)
          *reinterpret_cast<cs::u32x4*>(mine + (ROWS * j + lane / LANES) * KROW + 16 * (lane % LANES)) = k_raw[kb][j];
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      }
#pragma unroll
      for (int i = 0; i < D / 64; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const char* at = mine + n * KROW + (64 * i + 32 * h + 8 * w) * EB;
          if (CACHE == CS_KV4) {
            const uint32_t e = k_scale[kb] >> (8 * i) & 255u;
            kf[0][kb][4 * i + w] = __builtin_bit_cast(bf16x8, cs::kv4_unpack8_bf16(k_raw[kb][CACHE == CS_KV4 ? i : 0][w], cs::kv4_scale(e)));
          } else if (CACHE == CS_BF16) {
            kf[0][kb][4 * i + w] = *reinterpret_cast<const bf16x8*>(at);
          } else {
            const cs::u32x4 lo = *reinterpret_cast<const cs::u32x4*>(at), hi = *reinterpret_cast<const cs::u32x4*>(at + 16);
            float x[8];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              x[c] = __uint_as_float(lo[c]);
              x[4 + c] = __uint_as_float(hi[c]);
            }
#pragma unroll
            for (int part = 0; part < KP; ++part) kf[part][kb][4 * i + w] = __builtin_bit_cast(bf16x8, next_part(x));
          }
        }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    }
    if (CACHE == CS_KV4) {                                 // (blocks without numbers: rare)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < D / 64; ++i)
          if (__builtin_expect((k_scale[kb] >> (8 * i) & 255u) == cs::kKv4NoNumber, 0)) {
#pragma unroll
            for (int w = 0; w < 4; ++w) kf[0][kb][4 * i + w] = __builtin_bit_cast(bf16x8, cs::u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u});
          }
    }
  };

  float acc[KB] = {};
  auto do_step = [&](int step, auto stage) __attribute__((always_inline)) {
    constexpr int at_stage = decltype(stage)::value, buf = at_stage & 1;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int c = tid + 256 * i, at = (c / (D / 8)) * QROW + 8 * (c % (D / 8));
      if (QP == 1) {
        *reinterpret_cast<cs::u32x4*>(&s_q[buf][0][at]) = raw[at_stage][i][0];
      } else {
        float x[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = __uint_as_float(raw[at_stage][i][0][e]);
          x[4 + e] = __uint_as_float(raw[at_stage][i][QP == 1 ? 0 : 1][e]);
        }
#pragma unroll
        for (int part = 0; part < QP; ++part) *reinterpret_cast<cs::u32x4*>(&s_q[buf][part][at]) = next_part(x);
      }
    }
    if (tid < kStep) {
      // rows past the last, like those of a negative position, see nothing
      const int pos = step_at(step) * kStep + tid < rows ? min(next_pos[at_stage], entries - 1) : -1;
      s_pos[buf][tid] = pos;
      if (!STATS) {                                        // (+inf: such a row's weights are 0 here, those of keys past its position too)
        const bool none = pos >= 0 && !(next_lse[at_stage] > -INFINITY);
        s_lse[buf][tid] = none ? INFINITY : pos >= 0 ? next_lse[at_stage] * kLog2e : 0.0f;
        if (__builtin_expect(none, 0)) s_none = 1;
      }
    }
    if (step + AHEAD < step_end) request(step + AHEAD, at_stage);
    __syncthreads();
    if (STATS && step > step_begin) join(step - 1, buf ^ 1);

    const int my_pos = s_pos[buf][n];
    const bool sees = __any(my_pos >= key0);               // some row of the step sees a key of this wave
    const bool masked = __any(my_pos < key0 + 32 * KB - 1);
    if (sees) {
      f32x16 s[KB] = {};
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        bf16x8 qf[QP];
#pragma unroll
        for (int part = 0; part < QP; ++part) qf[part] = *reinterpret_cast<const bf16x8*>(&s_q[buf][part][n * QROW + 64 * (st / 4) + 32 * h + 8 * (st % 4)]);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int a = 0; a < QP; ++a)
#pragma unroll
            for (int b = 0; b < KP; ++b)
              if (a + b < 3)                               // (what the others add is below fp32's last bit)
                s[kb] = STATS ? __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[b][kb][st], qf[a], s[kb], 0, 0, 0)
                              : __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[a], kf[b][kb][st], s[kb], 0, 0, 0);
      }
      if (STATS) {
        float m = -INFINITY, l = 0.0f;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            s[kb][r] *= p.scale_log2e;
          }
        if (masked) {
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (key0 + 32 * kb + 8 * (r / 4) + 4 * h + r % 4 > my_pos) s[kb][r] = -INFINITY;
        }
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) m = fmaxf(m, s[kb][r]);
        m = fmaxf(m, __shfl_xor(m, 32));
        const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) l += __builtin_amdgcn_exp2f(s[kb][r] - base);
        l += __shfl_xor(l, 32);
        if (h == 0) {
          s_m[buf][wave][n] = m;
          s_l[buf][wave][n] = l;
        }
      } else {
        if (masked) {                                      // weights of keys that a row does not see: exp2 of -inf
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const cs::u32x4 pos = *reinterpret_cast<const cs::u32x4*>(&s_pos[buf][8 * g + 4 * h]);
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (key0 + 32 * kb + n > static_cast<int>(pos[i])) s[kb][4 * g + i] = -INFINITY;
          }
        }
        float sum[KB] = {};
#pragma unroll
        for (int g = 0; g < 4; ++g) {                      // rows 8 g + 4 h + 0..3
          const cs::u32x4 lse = *reinterpret_cast<const cs::u32x4*>(&s_lse[buf][8 * g + 4 * h]);
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[kb] += __builtin_amdgcn_exp2f(fmaf(s[kb][4 * g + i], p.scale_log2e, -__uint_as_float(lse[i])));
        }
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) acc[kb] += sum[kb];
      }
    } else if (STATS && h == 0) {
      s_m[buf][wave][n] = -INFINITY;
      s_l[buf][wave][n] = 0.0f;
    }
  };
  if (tid == 0) s_none = 0;                                // (written by this wave alone)
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (step_begin + i < step_end) request(step_begin + i, i);
  unpack();
  if (CACHE != CS_KV4) __syncthreads();                    // (what the keys passed through becomes the rows')
  for (int step = step_begin; step < step_end; step += AHEAD) {
    do_step(step, std::integral_constant<int, 0>());
    if (step + 1 < step_end) do_step(step + 1, std::integral_constant<int, 1>());
    if constexpr (AHEAD == 4) {
      if (step + 2 < step_end) do_step(step + 2, std::integral_constant<int, 2>());
      if (step + 3 < step_end) do_step(step + 3, std::integral_constant<int, 3>());
    }
  }
  if (STATS) {
    if (step_begin < step_end) {
      __syncthreads();
      join(step_end - 1, (step_end - 1 - step_begin) & 1);
    }
    return;
  }
  // Rows without statistics (rare) are looked up again: what they see, and nothing else, becomes NaN.
  if (step_begin < step_end && __builtin_expect(__builtin_amdgcn_readfirstlane(s_none), 0))
    for (int i = step_begin; i < step_end; ++i) {
      const int r = min(step_at(i) * kStep + n, rows - 1), tok = token_of(p, r);
      const int pos = min(p.q_pos[q0 + tok], entries - 1);
      const bool none = pos >= 0 && !(lse_base[static_cast<int64_t>(tok) * p.n_q_heads + (r - tok * p.group)] > -INFINITY);
      for (uint32_t left = static_cast<uint32_t>(__ballot(none)); left; left &= left - 1) {
        const int last = __builtin_amdgcn_readlane(pos, __ffs(left) - 1);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
          if (key0 + 32 * kb + n <= last) acc[kb] = NAN;
      }
    }
  float* part = p.ws_part + ((static_cast<int64_t>(chunk) * p.n_kv_heads + kvh) * p.n_streams + stream) * (static_cast<int64_t>(p.max_blocks) * CS_KV_BLOCK);
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
    const float both = acc[kb] + __shfl_xor(acc[kb], 32);
    const int key = key0 + 32 * kb + n;
    if (h == 0 && key < entries) part[key] = both;
  }
}

// log-sum-exp of every query row from its key ranges' maxima and sums: a wave a row, ranges dealt to its lanes.
__global__ __launch_bounds__(256) void attn_weights_join_kernel(Params p, int tile) {
  const int lane = threadIdx.x & 63;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (i >= p.n_q * p.n_q_heads) return;
  const int tok = static_cast<int>(i / p.n_q_heads);
  int lo = 0, hi = p.n_streams;                            // the last stream that starts at or before the token
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (p.cu_q[mid] <= tok) lo = mid;
    else hi = mid;
  }
  if (tok < p.cu_q[lo] || tok >= p.cu_q[lo + 1]) return;
  const int pos = min(p.q_pos[tok], stream_entries(p, lo) - 1);
  if (pos < 0) return;
  float m = -INFINITY, l = 0.0f;
  auto add = [&](float pm, float pl) __attribute__((always_inline)) {
    const float top = fmaxf(m, pm);
    l = (m == -INFINITY ? l : l * __builtin_amdgcn_exp2f(m - top)) + (pm == -INFINITY ? pl : pl * __builtin_amdgcn_exp2f(pm - top));
    m = top;
  };
  const cs::f32v2* part = p.ws_stat + i * p.key_tiles;
  for (int kt = lane; kt <= pos / tile; kt += 64) {
    const cs::f32v2 x = part[kt];
    add(x.x, x.y);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const float pm = __shfl_xor(m, d), pl = __shfl_xor(l, d);
    add(pm, pl);
  }
  if (lane == 0) p.ws_lse[i] = ((m == -INFINITY ? 0.0f : m) + __builtin_amdgcn_logf(l)) * kLn2;
}

// Partial sums of shares and kv heads, added in order to what earlier calls left.
__global__ __launch_bounds__(256) void attn_weights_sum_kernel(Params p) {
  const int64_t row = static_cast<int64_t>(p.max_blocks) * CS_KV_BLOCK, all = row * p.n_streams;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= all) return;
  const int stream = static_cast<int>(i / row);
  if (i - stream * row >= stream_entries(p, stream)) return;
  float sum = 0.0f;
  const int parts = p.chunks * p.n_kv_heads;
  for (int c0 = 0; c0 < parts; c0 += 8) {                  // (eight under way at once, added in order)
    float x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = c0 + k < parts ? p.ws_part[(c0 + k) * all + i] : 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += x[k];
  }
  if (p.weight_in && p.decay != 0.0f) sum = fmaf(p.decay, p.weight_in[i], sum);
  p.weight_out[i] = sum;
}

struct Layout {
  int key_tiles, chunks;
  size_t lse, stat, part, total;
};
Layout layout(int64_t n_q, int32_t n_streams, int32_t n_q_heads, int32_t n_kv_heads, int32_t max_blocks, int tile) {
  Layout w;
  const int64_t entries = static_cast<int64_t>(max_blocks) * CS_KV_BLOCK;
  w.key_tiles = static_cast<int>((entries + tile - 1) / tile);
  // Shares of a stream's rows: until kGroups workgroups are under way, but at least kLeast steps of rows each.
  const int64_t jobs = static_cast<int64_t>(w.key_tiles) * n_streams * n_kv_heads;
  const int64_t steps = (n_q * (n_q_heads / n_kv_heads) / (n_streams > 0 ? n_streams : 1) + kStep - 1) / kStep;
  int64_t c = jobs > 0 ? kGroups / jobs : 1;
  if (c > steps / kLeast) c = steps / kLeast;
  w.chunks = static_cast<int>(c < 1 ? 1 : c);
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  w.lse = 0;
  w.stat = up(static_cast<size_t>(n_q) * n_q_heads * 4);
  w.part = w.stat + up(static_cast<size_t>(n_q) * n_q_heads * w.key_tiles * 8);
  w.total = w.part + up(static_cast<size_t>(w.chunks) * n_kv_heads * n_streams * entries * 4);
  return w;
}

template <int D, int CACHE, int QP>
int launch(Params p, const Layout& w, bool have_lse, hipStream_t st) {
  const int64_t shares = static_cast<int64_t>(p.n_streams) * p.n_kv_heads * w.chunks;
  p.shares_per_xcd = shares >= 64;       // (few shares would load the XCDs unevenly)
  const int64_t jobs = (p.shares_per_xcd ? (shares + 7) / 8 * 8 : shares) * w.key_tiles;
  if (jobs > cs::kMostThreads / 256) return CS_EUNSUPPORTED;
  const dim3 grid(static_cast<unsigned>(jobs));
  const int64_t all = static_cast<int64_t>(p.max_blocks) * CS_KV_BLOCK * p.n_streams;
  if (!have_lse) {
    hipLaunchKernelGGL((attn_weights_kernel<D, CACHE, QP, true>), grid, dim3(256), 0, st, p);
    hipLaunchKernelGGL(attn_weights_join_kernel, dim3(static_cast<unsigned>((p.n_q * p.n_q_heads + 3) / 4)), dim3(256), 0, st, p, keys_per_tile(CACHE));
    p.lse = p.ws_lse;
  }
  hipLaunchKernelGGL((attn_weights_kernel<D, CACHE, QP, false>), grid, dim3(256), 0, st, p);
  hipLaunchKernelGGL(attn_weights_sum_kernel, dim3(static_cast<unsigned>((all + 255) / 256)), dim3(256), 0, st, p);
  return cs::note_hip(hipGetLastError());
}

}  // namespace

// (sized for the smaller tiles of an fp32 cache, whatever the cache)
extern "C" size_t cs_attn_weights_workspace(int64_t n_q, int32_t n_streams, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_blocks) {
  (void)head_dim;
  if (n_q < 1 || n_streams < 1 || n_q_heads < 1 || n_kv_heads < 1 || max_blocks < 1) return 0;
  const Layout a = layout(n_q, n_streams, n_q_heads, n_kv_heads, max_blocks, keys_per_tile(CS_F32));
  const Layout b = layout(n_q, n_streams, n_q_heads, n_kv_heads, max_blocks, keys_per_tile(CS_BF16));
  return a.total > b.total ? a.total : b.total;
}

extern "C" int cs_attn_weights(const void* q, const float* lse, const void* k_cache_layer, const uint8_t* k_scales_layer, const int32_t* cu_q,
                               const int32_t* q_pos, const int32_t* kv_len, const int32_t* block_table, int32_t max_blocks, int32_t block_size,
                               const float* weight_in, float* weight_out, float decay, int64_t n_q, int32_t n_streams, int32_t n_q_heads,
                               int32_t n_kv_heads, int32_t head_dim, int64_t stride_slot, int64_t stride_head, float softmax_scale, int32_t dtype,
                               int32_t cache_dtype, void* workspace, size_t workspace_bytes, void* stream) {
  if (n_q < 0 || n_streams < 0 || n_q_heads < 1 || n_kv_heads < 1 || head_dim < 1 || max_blocks < 0 || stride_slot < 0 || stride_head < 0)
    return CS_EINVAL;
  if (n_q_heads % n_kv_heads) return CS_EINVAL;
  if (!(softmax_scale > 0.0f && softmax_scale <= 3.0e38f) || !(decay >= 0.0f && decay <= 1.0f)) return CS_EINVAL;
  if (dtype != CS_F32 && dtype != CS_BF16) return CS_EUNSUPPORTED;
  if (cache_dtype != CS_KV4 && cache_dtype != dtype) return CS_EUNSUPPORTED;
  if ((head_dim != 64 && head_dim != 128) || block_size != CS_KV_BLOCK || n_q_heads / n_kv_heads > 16) return CS_EUNSUPPORTED;
  const int unit = cache_dtype == CS_KV4 ? cs::kKv4Block : cache_dtype == CS_BF16 ? 8 : 4;
  if (stride_slot % unit || stride_head % unit) return CS_EUNSUPPORTED;
  if (n_q > 0x7fffffffll / n_q_heads || n_q * (n_q_heads / n_kv_heads) >= (1 << 28) || max_blocks > 0x7fffffff / CS_KV_BLOCK - 256)
    return CS_EUNSUPPORTED;
  if (static_cast<int64_t>(max_blocks) * CS_KV_BLOCK * n_streams > cs::kMostThreads - 255) return CS_EUNSUPPORTED;
  if (!lse && n_q * n_q_heads > (cs::kMostThreads - 255) / 64) return CS_EUNSUPPORTED;     // (a wave a row joins the statistics)
  if (n_streams == 0) return CS_OK;
  if (!kv_len || !weight_out || max_blocks < 1) return CS_EINVAL;
  if (n_q == 0) {                        // earlier weights fade
    Params p = {};
    p.kv_len = kv_len;
    p.weight_in = weight_in;
    p.weight_out = weight_out;
    p.max_blocks = max_blocks;
    p.n_streams = n_streams;
    p.decay = decay;
    const int64_t all = static_cast<int64_t>(max_blocks) * CS_KV_BLOCK * n_streams;
    hipLaunchKernelGGL(attn_weights_sum_kernel, dim3(static_cast<unsigned>((all + 255) / 256)), dim3(256), 0, cs::as_stream(stream), p);
    return cs::note_hip(hipGetLastError());
  }
  if (!q || !k_cache_layer || !cu_q || !q_pos || !block_table) return CS_EINVAL;
  if (cache_dtype == CS_KV4 && !k_scales_layer) return CS_EINVAL;
  if (!cs::aligned16(q) || !cs::aligned16(k_cache_layer)) return CS_EUNSUPPORTED;
  const size_t need = cs_attn_weights_workspace(n_q, n_streams, n_q_heads, n_kv_heads, head_dim, max_blocks);
  if (!workspace || workspace_bytes < need || !cs::aligned16(workspace)) return CS_EWORKSPACE;

  const Layout w = layout(n_q, n_streams, n_q_heads, n_kv_heads, max_blocks, keys_per_tile(cache_dtype));
  Params p;
  p.q = q;
  p.lse = lse;
  p.k = k_cache_layer;
  p.k_scales = k_scales_layer;
  p.cu_q = cu_q;
  p.q_pos = q_pos;
  p.kv_len = kv_len;
  p.block_table = block_table;
  p.weight_in = weight_in;
  p.weight_out = weight_out;
  p.ws_lse = reinterpret_cast<float*>(static_cast<char*>(workspace) + w.lse);
  p.ws_stat = reinterpret_cast<cs::f32v2*>(static_cast<char*>(workspace) + w.stat);
  p.ws_part = reinterpret_cast<float*>(static_cast<char*>(workspace) + w.part);
  p.n_q = n_q;
  p.stride_slot = stride_slot;
  p.stride_head = stride_head;
  p.max_blocks = max_blocks;
  p.n_streams = n_streams;
  p.n_q_heads = n_q_heads;
  p.n_kv_heads = n_kv_heads;
  p.group = n_q_heads / n_kv_heads;
  p.group_inv = p.group == 1 ? 0u : static_cast<uint32_t>(((1ull << 32) + p.group - 1) / p.group);
  p.key_tiles = w.key_tiles;
  p.chunks = w.chunks;
  p.scale_log2e = softmax_scale * kLog2e;
  p.decay = decay;
  hipStream_t st = cs::as_stream(stream);
  const bool have = lse != nullptr;
  if (head_dim == 128) {
    if (cache_dtype == CS_F32) return launch<128, CS_F32, 3>(p, w, have, st);
    if (cache_dtype == CS_BF16) return launch<128, CS_BF16, 1>(p, w, have, st);
    return dtype == CS_BF16 ? launch<128, CS_KV4, 1>(p, w, have, st) : launch<128, CS_KV4, 3>(p, w, have, st);
  }
  if (cache_dtype == CS_F32) return launch<64, CS_F32, 3>(p, w, have, st);
  if (cache_dtype == CS_BF16) return launch<64, CS_BF16, 1>(p, w, have, st);
  return dtype == CS_BF16 ? launch<64, CS_KV4, 1>(p, w, have, st) : launch<64, CS_KV4, 3>(p, w, have, st);
}
