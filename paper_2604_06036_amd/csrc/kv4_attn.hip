// Causal attention of a batch's queries over the 4-bit window cache, gfx950: windows, questions and single tokens.
//
// out[t][h] = sum_j softmax_j(scale q[t][h] . K_j) V_j over the entries j <= q_pos[t] of the query's stream.
// A "row" is one (query token, query head of a kv group) pair, so that a tile of keys serves all heads of the group.  A
// workgroup takes 128 rows, 32 a wave, and sweeps the stream's entries in tiles of 64:
//   codes     16 bytes a lane (one block of 32 elements) in registers, asked for a tile ahead, to bf16 in LDS by the
//             conversion instruction (exact: a 4-bit value times a power of two has one fraction bit);
//   S^T = K Q^T      v_mfma_f32_32x32x16_bf16: a lane owns one query and 16 of 32 keys;
//   softmax          one pass, running maximum and sum in fp32; the reference maximum is raised when a tile exceeds it by
//                    more than 2^8, so that accumulators are rarely scaled;
//   O^T += V^T P^T   P^T is in operand layout as it is, V^T comes from the row-major tile by the transposing LDS read.
// fp32 queries: a query is the sum of three bf16 numbers (8 + 8 + 8 bits), so is a weight, and keys and values are bf16
// numbers, so three matrix instructions in place of one give scores and sums of fp32 accuracy.
#include <math.h>

#include <type_traits>

#include "kv4.h"

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

struct Params {
  const void* __restrict__ q;
  const uint8_t* __restrict__ k_codes;
  const uint8_t* __restrict__ k_scales;
  const uint8_t* __restrict__ v_codes;
  const uint8_t* __restrict__ v_scales;
  const int32_t* __restrict__ cu_q;
  const int32_t* __restrict__ q_pos;
  const int32_t* __restrict__ kv_len;
  const int32_t* __restrict__ block_table;
  void* __restrict__ out;
  float* __restrict__ lse;
  int64_t n_q, stride_slot, stride_head;
  int32_t max_blocks, n_streams, n_q_heads, n_kv_heads, group;
  float scale_log2e;
};

constexpr int kRows = 128;               // rows of a workgroup
constexpr int kKeys = 64;                // entries of a tile
constexpr float kSlack = 8.0f;           // log2 of how far weights may exceed the reference maximum's

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const cs::f32v2 v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, cs::bf16v2));
}

// The stream and row tile of the `target`-th row tile of the launch.  Every wave scans the streams for itself.
struct Tile {
  int stream, index, n_tiles, q0, rows;      // rows: of the whole stream
};
template <int ROWS>
__device__ __forceinline__ bool find_tile(const Params& p, int target, Tile* t) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int s0 = 0; s0 < p.n_streams; s0 += 64) {
    const int s = s0 + lane;
    int a = 0, n = 0;
    if (s < p.n_streams) {
      a = p.cu_q[s];
      n = max(0, min(p.cu_q[s + 1], static_cast<int>(p.n_q)) - a);
    }
    const int tiles = (n * p.group + ROWS - 1) / ROWS;
    int incl = tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int up = __shfl_up(incl, d);
      if (lane >= d) incl += up;
    }
    const int total = __shfl(incl, 63);
    if (target < before + total) {
      const uint64_t past = __ballot(before + incl > target);
      const int l = __ffsll(static_cast<unsigned long long>(past)) - 1;
      t->stream = s0 + l;
      t->n_tiles = __shfl(tiles, l);
      t->index = target - (before + __shfl(incl, l) - t->n_tiles);
      t->q0 = __shfl(a, l);
      t->rows = __shfl(n, l) * p.group;
      return true;
    }
    before += total;
  }
  return false;
}

// PARTS: bf16 numbers that a query and a weight are the sum of (1: bf16 queries, 3: fp32).
template <int D, int PARTS>
__global__ __launch_bounds__(256) void kv4_attn_kernel(Params p) {
  constexpr int STEPS = D / 16, DB = D / 32;
  constexpr int KROW = D + 8, VROW = D + 32;               // LDS rows, padded so that the reads below meet no bank twice
  constexpr int CHUNKS = kKeys * DB;                       // blocks of 32 elements of a tile, keys or values
  constexpr int MINE = 2 * CHUNKS / 256;                   // ... of a thread (D 128: one of each; D 64: one of either)
  __shared__ __attribute__((aligned(16))) uint16_t s_k[kKeys * KROW];
  __shared__ __attribute__((aligned(16))) uint16_t s_v[kKeys * VROW];
  __shared__ uint8_t s_vscale[kKeys][DB];
  __shared__ int s_last[4];
  __shared__ int s_nan;

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 31, h = lane >> 5;
  Tile t;
  if (!find_tile<kRows>(p, blockIdx.x, &t)) return;
  const int kvh = blockIdx.y;
  const int entries = min(p.kv_len[t.stream], p.max_blocks * CS_KV_BLOCK);
  if (entries <= 0) return;
  if (tid == 0) s_nan = 0;

  // ---- this lane's query
  const int row0 = (t.n_tiles - 1 - t.index) * kRows + wave * 32;     // the longest sweeps first
  const int row = min(row0 + n, t.rows - 1);
  const int tok = t.q0 + row / p.group, head = kvh * p.group + row % p.group;
  const bool live = row0 + n < t.rows;
  const int pos = min(p.q_pos[tok], entries - 1);
  bf16x8 qf[PARTS][STEPS];
  {
    const int64_t at = (static_cast<int64_t>(tok) * p.n_q_heads + head) * D + 8 * h;
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      if (PARTS == 1) {
        qf[0][st] = *reinterpret_cast<const bf16x8*>(static_cast<const uint16_t*>(p.q) + at + 16 * st);
      } else {
        float x[8];
        const cs::u32x4 a = *reinterpret_cast<const cs::u32x4*>(static_cast<const float*>(p.q) + at + 16 * st);
        const cs::u32x4 b = *reinterpret_cast<const cs::u32x4*>(static_cast<const float*>(p.q) + at + 16 * st + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = __uint_as_float(a[i]);
          x[4 + i] = __uint_as_float(b[i]);
        }
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
          cs::u32x4 w;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            w[i] = pack2(x[2 * i], x[2 * i + 1]);
            x[2 * i] -= __uint_as_float(w[i] << 16);
            x[2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u);
          }
          qf[part][st] = __builtin_bit_cast(bf16x8, w);
        }
      }
    }
  }

  // ---- how far the workgroup's rows see, and this wave's
  int wave_last = live ? pos : -1, wave_first = live ? pos : 0x7fffffff;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    wave_last = max(wave_last, __shfl_xor(wave_last, d));
    wave_first = min(wave_first, __shfl_xor(wave_first, d));
  }
  if (lane == 0) s_last[wave] = wave_last;
  __syncthreads();
  const int last = max(max(s_last[0], s_last[1]), max(s_last[2], s_last[3]));
  const int n_tiles = (last + kKeys) / kKeys;              // (no entry seen: last -1, no tile)

  // ---- tile requests
  const int32_t* ids = p.block_table + static_cast<int64_t>(t.stream) * p.max_blocks;
  cs::u32x4 code[MINE];
  uint32_t scale[MINE];
  auto request = [&](int kt) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
      const int c = tid + 256 * i, of_v = c >= CHUNKS, cc = c - (of_v ? CHUNKS : 0);
      const int key = min(kt * kKeys + cc / DB, last);     // past the frontier: the frontier's row (what lies there may be nothing)
      const int64_t at = (static_cast<int64_t>(ids[key / CS_KV_BLOCK]) * CS_KV_BLOCK + key % CS_KV_BLOCK) * p.stride_slot +
                         static_cast<int64_t>(kvh) * p.stride_head + (cc % DB) * cs::kKv4Block;
      code[i] = *reinterpret_cast<const cs::u32x4*>((of_v ? p.v_codes : p.k_codes) + at / 2);
      scale[i] = (of_v ? p.v_scales : p.k_scales)[at / cs::kKv4Block];
    }
  };
  if (n_tiles > 0) request(0);

  f32x16 o[DB] = {};
  float m = -INFINITY, l = 0.0f;                           // reference maximum (raw score), this lane's share of the sum
  for (int kt = 0; kt < n_tiles; ++kt) {
    // ---- codes -> bf16 tile
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
      const int c = tid + 256 * i, of_v = c >= CHUNKS, cc = c - (of_v ? CHUNKS : 0);
      const int r = cc / DB, b = cc % DB;
      uint16_t* dst = of_v ? s_v + r * VROW + 32 * b : s_k + r * KROW + 32 * b;
      const bool none = scale[i] == cs::kKv4NoNumber;
      const float sc = cs::kv4_scale(scale[i]);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        cs::u32x4 x = cs::kv4_unpack8_bf16(code[i][w], sc);
        // keys that are no numbers poison the scores of the queries that see them; values must not meet a weight of 0
        if (none) x = of_v ? cs::u32x4{0, 0, 0, 0} : cs::u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
        *reinterpret_cast<cs::u32x4*>(dst + 8 * w) = x;
      }
      if (of_v) {
        s_vscale[r][b] = static_cast<uint8_t>(scale[i]);
        if (none) s_nan = 1;
      }
    }
    __syncthreads();
    if (kt + 1 < n_tiles) request(kt + 1);

    const int key0 = kt * kKeys;
    if (key0 <= wave_last) {
      // ---- S^T
      f32x16 s[2] = {};
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
          const bf16x8 kf = *reinterpret_cast<const bf16x8*>(s_k + (32 * kb + n) * KROW + 16 * st + 8 * h);
#pragma unroll
          for (int part = 0; part < PARTS; ++part) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[part][st], s[kb], 0, 0, 0);
        }
      // ---- masks, maximum
      if (key0 + kKeys - 1 > wave_first) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (key0 + 32 * kb + 8 * (r / 4) + 4 * h + r % 4 > pos) s[kb][r] = -INFINITY;
      }
      float top = s[0][0];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[kb][r]);
      top = fmaxf(top, __shfl_xor(top, 32));
      if (__any((top - m) * p.scale_log2e > kSlack || m == -INFINITY)) {
        const float raised = fmaxf(m, top);
        const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - raised) * p.scale_log2e);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[db][r] *= f;
        l *= f;
        m = raised;
      }
      const float base = m == -INFINITY ? 0.0f : -m * p.scale_log2e;
      // ---- weights
      bf16x8 pf[PARTS][4];
#pragma unroll
      for (int st = 0; st < 4; ++st) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] = __builtin_amdgcn_exp2f(fmaf(s[st / 2][8 * (st & 1) + i], p.scale_log2e, base));
          l += x[i];
        }
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
          cs::u32x4 w;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            w[i] = pack2(x[2 * i], x[2 * i + 1]);
            if (PARTS > 1) {
              x[2 * i] -= __uint_as_float(w[i] << 16);
              x[2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u);
            }
          }
          pf[part][st] = __builtin_bit_cast(bf16x8, w);
        }
      }
      // ---- O^T: of the 16 keys of a step a lane holds 4 h + 0..3 and 8 + 4 h + 0..3
      const int i16 = lane & 15, gid = (lane >> 4) & 1;
#pragma unroll
      for (int st = 0; st < 4; ++st)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const uint16_t* at = s_v + (16 * st + 4 * h + (i16 >> 2)) * VROW + 32 * db + 16 * gid + 4 * (i16 & 3);
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 8 * VROW));
          const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
          for (int part = 0; part < PARTS; ++part) o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[part][st], o[db], 0, 0, 0);
        }
      if (s_nan) {                                         // (a tile so far held a value block without numbers)
        for (int r = 0; r < kKeys; ++r)
#pragma unroll
          for (int db = 0; db < DB; ++db)
            if (s_vscale[r][db] == cs::kKv4NoNumber && key0 + r <= pos) {
#pragma unroll
              for (int i = 0; i < 16; ++i) o[db][i] = NAN;
            }
      }
    }
    __syncthreads();
  }

  // ---- results
  l += __shfl_xor(l, 32);
  if (!live) return;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;           // a row that sees nothing is 0
  const int64_t at = (static_cast<int64_t>(tok) * p.n_q_heads + head) * D;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int d = 32 * db + 8 * g + 4 * h;
      float x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = o[db][4 * g + i] * inv;
      if (PARTS == 1)
        *reinterpret_cast<cs::u32x2*>(static_cast<uint16_t*>(p.out) + at + d) = cs::u32x2{pack2(x[0], x[1]), pack2(x[2], x[3])};
      else
        *reinterpret_cast<cs::u32x4*>(static_cast<float*>(p.out) + at + d) =
            cs::u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    }
  if (p.lse && h == 0)
    p.lse[static_cast<int64_t>(tok) * p.n_q_heads + head] =
        l == 0.0f ? -INFINITY : (m * p.scale_log2e + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

}  // namespace

extern "C" size_t cs_kv4_window_attn_workspace(int64_t n_q, int32_t n_streams, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                               int32_t max_blocks) {
  (void)n_q; (void)n_streams; (void)n_q_heads; (void)n_kv_heads; (void)head_dim; (void)max_blocks;
  return 0;
}

extern "C" int cs_kv4_window_attn(const void* q, const uint8_t* k_codes_layer, const uint8_t* k_scales_layer, const uint8_t* v_codes_layer,
                                  const uint8_t* v_scales_layer, const int32_t* cu_q, const int32_t* q_pos, const int32_t* kv_len,
                                  const int32_t* block_table, int32_t max_blocks, int32_t block_size, void* out, float* lse, int64_t n_q,
                                  int32_t n_streams, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t stride_slot,
                                  int64_t stride_head, float softmax_scale, int32_t dtype, void* workspace, size_t workspace_bytes,
                                  void* stream) {
  if (n_q < 0 || n_streams < 0 || n_q_heads < 1 || n_kv_heads < 1 || head_dim < 1 || max_blocks < 0 || stride_slot < 0 || stride_head < 0)
    return CS_EINVAL;
  if (n_q_heads % n_kv_heads) return CS_EINVAL;
  if (!(softmax_scale > 0.0f && softmax_scale <= 3.0e38f)) return CS_EINVAL;
  if (dtype != CS_F32 && dtype != CS_BF16) return CS_EUNSUPPORTED;
  if ((head_dim != 64 && head_dim != 128) || block_size != CS_KV_BLOCK || n_q_heads / n_kv_heads > 16 || n_kv_heads > 65535) return CS_EUNSUPPORTED;
  if (!cs::kv4_strides(stride_slot, stride_head, 0)) return CS_EUNSUPPORTED;
  if (n_q > 0x7fffffffll / 16 || max_blocks > 0x7fffffff / CS_KV_BLOCK) return CS_EUNSUPPORTED;
  if (n_q == 0 || n_streams == 0) return CS_OK;
  if (!q || !k_codes_layer || !k_scales_layer || !v_codes_layer || !v_scales_layer || !cu_q || !q_pos || !kv_len || !block_table || !out || max_blocks < 1)
    return CS_EINVAL;
  if (!cs::aligned16(q) || !cs::aligned16(out) || !cs::aligned16(k_codes_layer) || !cs::aligned16(v_codes_layer)) return CS_EUNSUPPORTED;
  const size_t need = cs_kv4_window_attn_workspace(n_q, n_streams, n_q_heads, n_kv_heads, head_dim, max_blocks);
  if (need && (!workspace || workspace_bytes < need || !cs::aligned16(workspace))) return CS_EWORKSPACE;

  Params p;
  p.q = q;
  p.k_codes = k_codes_layer;
  p.k_scales = k_scales_layer;
  p.v_codes = v_codes_layer;
  p.v_scales = v_scales_layer;
  p.cu_q = cu_q;
  p.q_pos = q_pos;
  p.kv_len = kv_len;
  p.block_table = block_table;
  p.out = out;
  p.lse = lse;
  p.n_q = n_q;
  p.stride_slot = stride_slot;
  p.stride_head = stride_head;
  p.max_blocks = max_blocks;
  p.n_streams = n_streams;
  p.n_q_heads = n_q_heads;
  p.n_kv_heads = n_kv_heads;
  p.group = n_q_heads / n_kv_heads;
  p.scale_log2e = softmax_scale * 1.4426950408889634f;
  const int64_t tiles = n_q * p.group / kRows + (n_streams < n_q ? n_streams : n_q);
  const dim3 grid(static_cast<unsigned>(tiles), static_cast<unsigned>(n_kv_heads));
  hipStream_t st = cs::as_stream(stream);
  if (head_dim == 128 && dtype == CS_BF16) hipLaunchKernelGGL((kv4_attn_kernel<128, 1>), grid, dim3(256), 0, st, p);
  else if (head_dim == 128) hipLaunchKernelGGL((kv4_attn_kernel<128, 3>), grid, dim3(256), 0, st, p);
  else if (dtype == CS_BF16) hipLaunchKernelGGL((kv4_attn_kernel<64, 1>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((kv4_attn_kernel<64, 3>), grid, dim3(256), 0, st, p);
  return cs::note_hip(hipGetLastError());
}
