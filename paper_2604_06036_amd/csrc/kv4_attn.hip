// Causal attention of a batch's queries over the 4-bit window cache, gfx950: windows, questions and single tokens.
//
// out[t][h] = sum_j softmax_j(scale q[t][h] . K_j) V_j over the entries j <= q_pos[t] of the query's stream.
// A "row" is one (query token, query head of a kv group) pair, so that a tile of keys serves all heads of the group.  Keys
// pass in tiles of 64, 32 at a time:
//   S^T = K Q^T      v_mfma_f32_32x32x16_bf16, a lane owns one query and 16 of 32 keys.  Keys are converted to bf16, which
//                    is exact (a 4-bit value has one fraction bit).  fp32 queries are the sum of three bf16 numbers (8 + 8 + 8
//                    bits).  (v_mfma_scale_f32_32x32x64 would take the codes as they lie in the cache, against queries in 8-bit
//                    parts; but it drops what lies 2^14 below the largest product of an instruction, measured on integers:
//                    one large channel would cost the scores their low bits, 4e-5 of a score of 1 for normal data.)
//   softmax          one pass, running maximum and sum in fp32; the reference maximum is raised when a tile exceeds it by
//                    more than 2^8, so that accumulators are rarely scaled.  Weights are rounded to bf16 (fp32 queries:
//                    three bf16 parts); the sums of the statistics are over the unrounded ones.
//   O^T += V^T P^T   v_mfma_f32_32x32x16_bf16: P^T is in operand layout as it is, values are converted to bf16 on their way
//                    into LDS and come back by its transposing read.
// Many rows a stream (rows kernel): four waves of 32 rows share a tile in LDS.  Few rows (keys kernel): every wave holds the
// same 32 rows and takes tiles of its own, with nothing but its own values in LDS; the waves join their results at the end.
// Where there are few workgroups, the sweep of a row tile is cut into pieces of entries, whose results a second launch joins.
#include <math.h>

#include <type_traits>

#include "kv4.h"

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
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
  float* __restrict__ ws_ml;             // [jobs][rows][2]: reference maximum (raw score), sum; jobs are (kv head, row tile, piece)
  float* __restrict__ ws_o;              // [jobs][rows][D]: sums, not divided
  int64_t n_q, stride_slot, stride_head;
  int32_t max_blocks, n_streams, n_q_heads, n_kv_heads, group;
  int32_t row_tiles, pieces, jobs, jobs_per_xcd;
  float scale_log2e;
};

constexpr int kKeys = 64;                // entries of a tile
constexpr int kRowsMany = 128;           // rows of a workgroup of the rows kernel
constexpr int kRowsFew = 32;             // ... of the keys kernel
constexpr float kSlack = 8.0f;           // log2 of how far weights may exceed the reference maximum's
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const cs::f32v2 v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, cs::bf16v2));
}

__device__ __forceinline__ float other_half(float x) {     // the value of lane ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
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
    const int total = __builtin_amdgcn_readlane(incl, 63);
    if (target < before + total) {
      const uint64_t past = __ballot(before + incl > target);
      const int l = __builtin_amdgcn_readfirstlane(__ffsll(static_cast<unsigned long long>(past)) - 1);
      t->stream = s0 + l;
      t->n_tiles = __builtin_amdgcn_readlane(tiles, l);
      t->index = target - (before + __builtin_amdgcn_readlane(incl, l) - t->n_tiles);
      t->q0 = __builtin_amdgcn_readlane(a, l);
      t->rows = __builtin_amdgcn_readlane(n, l) * p.group;
      return true;
    }
    before += total;
  }
  return false;
}

// Workgroup -> (kv head, row tile, piece).  Workgroups go round the eight XCDs, so an XCD is given a run of neighbouring
// jobs: row tiles of the same stream and kv head meet in its L2.
struct Job {
  int kvh, tile, piece, index;
};
__device__ __forceinline__ bool job_of(const Params& p, Job* j) {
  const int i = static_cast<int>(blockIdx.x % 8) * p.jobs_per_xcd + static_cast<int>(blockIdx.x / 8);
  if (static_cast<int>(blockIdx.x / 8) >= p.jobs_per_xcd || i >= p.jobs) return false;
  j->index = i;
  j->piece = i % p.pieces;
  const int kt = i / p.pieces;
  j->tile = kt % p.row_tiles;
  j->kvh = kt / p.row_tiles;
  return true;
}

// ---- a lane's query: PARTS bf16 numbers an element (1: bf16 queries, 3: fp32), elements 64 i + 32 h + 8 w + 0..7 of its row in operand
// (i, w), h being which half of the wave: the order in which a lane holds the codes of whole 32-element blocks
template <int D, int PARTS>
struct Query {
  bf16x8 part[PARTS][D / 64][4];

  __device__ __forceinline__ void load(const void* q, int64_t at, int h) {
#pragma unroll
    for (int i = 0; i < D / 64; ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int64_t from = at + 64 * i + 32 * h + 8 * w;
        if (PARTS == 1) {
          part[0][i][w] = *reinterpret_cast<const bf16x8*>(static_cast<const uint16_t*>(q) + from);
          continue;
        }
        const float* src = static_cast<const float*>(q) + from;
        const cs::u32x4 a = *reinterpret_cast<const cs::u32x4*>(src), b = *reinterpret_cast<const cs::u32x4*>(src + 4);
        float x[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = __uint_as_float(a[e]);
          x[4 + e] = __uint_as_float(b[e]);
        }
#pragma unroll
        for (int k = 0; k < PARTS; ++k) {
          cs::u32x4 c;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            c[e] = pack2(x[2 * e], x[2 * e + 1]);
            x[2 * e] -= __uint_as_float(c[e] << 16);
            x[2 * e + 1] -= __uint_as_float(c[e] & 0xffff0000u);
          }
          part[k][i][w] = __builtin_bit_cast(bf16x8, c);
        }
      }
  }

  __device__ __forceinline__ void step(f32x16& s, const bf16x8& keys, int i, int w) const {
#pragma unroll
    for (int k = PARTS - 1; k >= 0; --k) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(keys, part[k][i][w], s, 0, 0, 0);
  }

  // S^T of 32 keys in LDS: `keys` is the lane's row
  __device__ __forceinline__ f32x16 scores(const uint16_t* keys, int h) const {
    f32x16 s = {};
#pragma unroll
    for (int i = 0; i < D / 64; ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w) step(s, *reinterpret_cast<const bf16x8*>(keys + 64 * i + 32 * h + 8 * w), i, w);
    return s;
  }

  // ... of codes in registers: blocks 2 i + h of the lane's key, their scales in bytes 0 and 2 of `scales`
  __device__ __forceinline__ f32x16 scores(const cs::u32x4 (&codes)[D / 64], uint32_t scales) const {
    f32x16 s = {};
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const uint32_t e = (scales >> (16 * i)) & 255u;
      const float sc = cs::kv4_scale(e == cs::kKv4NoNumber ? 1u : e);
#pragma unroll
      for (int w = 0; w < 4; ++w) step(s, __builtin_bit_cast(bf16x8, cs::kv4_unpack8_bf16(codes[i][w], sc)), i, w);
    }
    return s;
  }
};

// ---- running softmax and sums of a lane's query over half tiles of 32 keys
template <int D, int PARTS>
struct Sums {
  static constexpr int DB = D / 32;
  f32x16 o[DB];
  float m, l;                            // reference maximum (raw score), the lane's share of the sum

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = f32x16{};
    m = -INFINITY;
    l = 0.0f;
  }

  // Weights of the scores of keys key0 + 8 (r / 4) + 4 h + r % 4 for a query that sees up to `pos`.
  __device__ __forceinline__ void weights(f32x16 s, int key0, int pos, bool masked, int h, float c, bf16x8 (&pf)[PARTS][2]) {
    if (masked) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (key0 + 8 * (r / 4) + 4 * h + r % 4 > pos) s[r] = -INFINITY;
    }
    float top = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
    top = fmaxf(top, other_half(top));
    if (__any((top - m) * c > kSlack || m == -INFINITY)) {
      const float raised = fmaxf(m, top);
      const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - raised) * c);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[db][r] *= f;
      l *= f;
      m = raised;
    }
    const float base = m == -INFINITY ? 0.0f : -m * c;
    float sum = 0.0f;
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = __builtin_amdgcn_exp2f(fmaf(s[8 * st + i], c, base));
        sum += x[i];
      }
#pragma unroll
      for (int k = 0; k < PARTS; ++k) {
        cs::u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w[i] = pack2(x[2 * i], x[2 * i + 1]);
          if (PARTS > 1) {
            x[2 * i] -= __uint_as_float(w[i] << 16);
            x[2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u);
          }
        }
        pf[k][st] = __builtin_bit_cast(bf16x8, w);
      }
    }
    l += sum;
  }

  // Values of 32 keys, row-major bf16 in LDS with rows of VROW elements.  Of the 16 keys of a step a lane's weights are of
  // 4 h + 0..3 and 8 + 4 h + 0..3; the transposing read gives 16 lanes four rows of 16 elements.
  template <int VROW>
  __device__ __forceinline__ void add(const uint16_t* v, const bf16x8 (&pf)[PARTS][2], int lane) {
    const int h = lane >> 5, i16 = lane & 15, gid = (lane >> 4) & 1;
    const uint16_t* base = v + (4 * h + (i16 >> 2)) * VROW + 16 * gid + 4 * (i16 & 3);
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const uint16_t* at = base + 16 * st * VROW + 32 * db;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 8 * VROW));
        const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int k = PARTS - 1; k >= 0; --k) o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[k][st], o[db], 0, 0, 0);
      }
  }

  // A value block without numbers (its place in LDS holds zeros) reaches the queries that see its key.
  __device__ __forceinline__ void poison(int db, bool sees) {
#pragma unroll
    for (int b = 0; b < DB; ++b)
      if (b == db && sees) {
#pragma unroll
        for (int r = 0; r < 16; ++r) o[b][r] = NAN;
      }
  }
};

// A block of 32 values -> bf16 in LDS; zeros for a block without numbers, which is reported.
__device__ __forceinline__ bool put_values(uint16_t* dst, const cs::u32x4& code, uint32_t scale) {
  const bool none = scale == cs::kKv4NoNumber;
  const float sc = cs::kv4_scale(none ? 1u : scale);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    cs::u32x4 x = cs::kv4_unpack8_bf16(code[w], sc);
    if (none) x = cs::u32x4{0, 0, 0, 0};
    *reinterpret_cast<cs::u32x4*>(dst + 8 * w) = x;
  }
  return none;
}

// A block of 32 keys' elements -> bf16 in LDS; NaN for a block without numbers.
__device__ __forceinline__ void put_keys(uint16_t* dst, const cs::u32x4& code, uint32_t scale) {
  const bool none = scale == cs::kKv4NoNumber;
  const float sc = cs::kv4_scale(none ? 1u : scale);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    cs::u32x4 x = cs::kv4_unpack8_bf16(code[w], sc);
    if (none) x = cs::u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
    *reinterpret_cast<cs::u32x4*>(dst + 8 * w) = x;
  }
}

__device__ __forceinline__ void store4(void* out, int64_t at, const float* x, bool bf16) {
  if (bf16)
    *reinterpret_cast<cs::u32x2*>(static_cast<uint16_t*>(out) + at) = cs::u32x2{pack2(x[0], x[1]), pack2(x[2], x[3])};
  else
    *reinterpret_cast<cs::u32x4*>(static_cast<float*>(out) + at) =
        cs::u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
}

__device__ __forceinline__ float log_sum(float m, float l, float c) { return l == 0.0f ? -INFINITY : (m * c + __builtin_amdgcn_logf(l)) * kLn2; }

// Scale bytes of a cache row, from element `at` on (any alignment): block 2 i + h of the row in byte 2 i.
template <int D>
__device__ __forceinline__ uint32_t row_scales(const uint8_t* scales, int64_t at, int h) {
  if (D == 128) {
    uint32_t w;
    __builtin_memcpy(&w, scales + at / cs::kKv4Block, 4);
    return w >> (8 * h);
  }
  return scales[at / cs::kKv4Block + h];
}

// ------------------------------------------------------------------------------------------
// Many rows: four waves of 32 rows share the tiles of a sweep.  Codes are asked for a tile ahead into registers (16 bytes a
// lane: one block) and put into LDS as bf16, in two stages, so that a tile costs one barrier.
template <int D, int PARTS>
__global__ __launch_bounds__(256) void kv4_rows_kernel(Params p) {
  constexpr int DB = D / 32;
  constexpr int KROW = D + 8, VROW = D + 32;               // padded: reads of eight rows, and the transposing ones, meet no bank twice
  constexpr int CHUNKS = kKeys * DB, MINE = 2 * CHUNKS / 256;      // blocks of a tile's keys (or values), blocks a thread moves
  __shared__ __attribute__((aligned(16))) uint16_t s_k[2][kKeys * KROW];
  __shared__ __attribute__((aligned(16))) uint16_t s_v[2][kKeys * VROW];
  __shared__ uint8_t s_vs[2][CHUNKS];
  __shared__ int s_last[4];
  __shared__ int s_nan;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
  Job job;
  Tile t;
  if (!job_of(p, &job) || !find_tile<kRowsMany>(p, job.tile, &t)) return;
  const int kvh = job.kvh;
  const int entries = min(p.kv_len[t.stream], p.max_blocks * CS_KV_BLOCK);
  if (entries <= 0) return;
  if (tid == 0) s_nan = 0;

  // ---- this lane's query
  const int row0 = (t.n_tiles - 1 - t.index) * kRowsMany + wave * 32;     // the longest sweeps first
  const int row = min(row0 + n, t.rows - 1);
  const int tok = t.q0 + row / p.group, head = kvh * p.group + row % p.group;
  const bool live = row0 + n < t.rows;
  const int pos = min(p.q_pos[tok], entries - 1);
  const int64_t at_q = (static_cast<int64_t>(tok) * p.n_q_heads + head) * D;
  Query<D, PARTS> query;
  query.load(p.q, at_q, h);

  // ---- how far the workgroup's rows see, and this wave's
  int wave_last = live ? pos : -1, wave_first = live ? pos : 0x7fffffff;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    wave_last = max(wave_last, __shfl_xor(wave_last, d));
    wave_first = min(wave_first, __shfl_xor(wave_first, d));
  }
  wave_last = __builtin_amdgcn_readfirstlane(wave_last);
  wave_first = __builtin_amdgcn_readfirstlane(wave_first);
  if (lane == 0) s_last[wave] = wave_last;
  __syncthreads();
  const int last = max(max(s_last[0], s_last[1]), max(s_last[2], s_last[3]));
  const int all_tiles = (last + kKeys) / kKeys;            // (no entry seen: last -1, no tile)
  const int share = (all_tiles + p.pieces - 1) / p.pieces;
  const int kt0 = min(all_tiles, job.piece * share), kt1 = min(all_tiles, kt0 + share);

  // ---- tile requests
  const int32_t* ids = p.block_table + static_cast<int64_t>(t.stream) * p.max_blocks;
  cs::u32x4 code[MINE];
  uint32_t scale[MINE];
  int id[MINE];
  auto key_of = [&](int kt, int i) __attribute__((always_inline)) {        // past the frontier: the frontier's row (what lies there may be nothing)
    const int c = tid + 256 * i;
    return min(kt * kKeys + (c >= CHUNKS ? c - CHUNKS : c) / DB, last);
  };
  auto request_id = [&](int kt) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < MINE; ++i) id[i] = ids[key_of(kt, i) / CS_KV_BLOCK];
  };
  auto request = [&](int kt) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
      const int c = tid + 256 * i, of_v = c >= CHUNKS;
      const int64_t at = (static_cast<int64_t>(id[i]) * CS_KV_BLOCK + key_of(kt, i) % CS_KV_BLOCK) * p.stride_slot +
                         static_cast<int64_t>(kvh) * p.stride_head + (c % DB) * cs::kKv4Block;
      code[i] = *reinterpret_cast<const cs::u32x4*>((of_v ? p.v_codes : p.k_codes) + at / 2);
      scale[i] = (of_v ? p.v_scales : p.k_scales)[at / cs::kKv4Block];
    }
  };
  auto put = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
      const int c = tid + 256 * i, of_v = c >= CHUNKS, cc = c - (of_v ? CHUNKS : 0), r = cc / DB, b = cc % DB;
      if (of_v) {
        if (put_values(&s_v[buf][r * VROW + 32 * b], code[i], scale[i])) s_nan = 1;
        s_vs[buf][cc] = static_cast<uint8_t>(scale[i]);
      } else {
        put_keys(&s_k[buf][r * KROW + 32 * b], code[i], scale[i]);
      }
    }
  };

  Sums<D, PARTS> sums;
  sums.clear();
  if (kt0 < kt1) {
    request_id(kt0);
    request(kt0);
    if (kt0 + 1 < kt1) request_id(kt0 + 1);
    put(0);
    if (kt0 + 1 < kt1) request(kt0 + 1);
    if (kt0 + 2 < kt1) request_id(kt0 + 2);
    __syncthreads();
  }
  for (int kt = kt0; kt < kt1; ++kt) {
    const int buf = (kt - kt0) & 1;
    const int key0 = kt * kKeys;
    if (key0 <= wave_last) {
      const bool two = key0 + 32 <= wave_last;             // (the second half's scores beside the first half's softmax)
      f32x16 s0 = query.scores(&s_k[buf][n * KROW], h), s1;
      if (two) s1 = query.scores(&s_k[buf][(32 + n) * KROW], h);
      bf16x8 pf[PARTS][2];
      sums.weights(s0, key0, pos, key0 + 31 > wave_first, h, p.scale_log2e, pf);
      sums.template add<VROW>(&s_v[buf][0], pf, lane);
      if (two) {
        sums.weights(s1, key0 + 32, pos, key0 + 63 > wave_first, h, p.scale_log2e, pf);
        sums.template add<VROW>(&s_v[buf][32 * VROW], pf, lane);
      }
    }
    if (s_nan) {                                           // (a tile so far held a value block without numbers)
      for (int c = 0; c < CHUNKS; ++c)
        if (s_vs[buf][c] == cs::kKv4NoNumber) sums.poison(c % DB, kt * kKeys + c / DB <= pos);
    }
    if (kt + 1 < kt1) put(buf ^ 1);
    if (kt + 2 < kt1) request(kt + 2);
    if (kt + 3 < kt1) request_id(kt + 3);
    __syncthreads();
  }

  // ---- results
  sums.l += other_half(sums.l);
  if (p.pieces > 1) {                                      // the row tile's other pieces are joined to it by a launch of its own
    const int64_t r = static_cast<int64_t>(job.index) * kRowsMany + wave * 32 + n;
    if (h == 0) *reinterpret_cast<cs::f32v2*>(p.ws_ml + 2 * r) = cs::f32v2{sums.m, sums.l};
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4*>(p.ws_o + r * D + 32 * db + 8 * g + 4 * h) =
            f32x4{sums.o[db][4 * g], sums.o[db][4 * g + 1], sums.o[db][4 * g + 2], sums.o[db][4 * g + 3]};
    return;
  }
  if (!live) return;
  const float inv = sums.l == 0.0f ? 0.0f : 1.0f / sums.l;       // a row that sees nothing is 0
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = sums.o[db][4 * g + i] * inv;
      store4(p.out, at_q + 32 * db + 8 * g + 4 * h, x, PARTS == 1);
    }
  if (p.lse && h == 0) p.lse[static_cast<int64_t>(tok) * p.n_q_heads + head] = log_sum(sums.m, sums.l, p.scale_log2e);
}

// ------------------------------------------------------------------------------------------
// Few rows: WAVES waves hold the same 32 rows and take every WAVES-th tile of the sweep, each for itself: a wave's keys go
// from memory into operand registers, its values through its own 32 rows of LDS.  No barrier before the end.
template <int D, int PARTS, int WAVES>
__global__ __launch_bounds__(64 * WAVES, D == 128 && PARTS == 3 ? 1 : 2) void kv4_keys_kernel(Params p) {
  constexpr int DB = D / 32, KI = D / 64;
  constexpr int VROW = D + 32;
  constexpr int VC = kKeys * DB / 64;                      // value blocks of a tile that a lane moves (an even number)
  constexpr int OROW = 64 + 4;                             // padded rows of the join, 64 columns at a time
  constexpr int V_BYTES = WAVES * 32 * VROW * 2, O_BYTES = WAVES * 32 * OROW * 4;
  __shared__ __attribute__((aligned(16))) uint8_t s_mem[V_BYTES > O_BYTES ? V_BYTES : O_BYTES];
  __shared__ float s_m[WAVES][32], s_l[WAVES][32], s_sum[32];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
  Job job;
  Tile t;
  if (!job_of(p, &job) || !find_tile<kRowsFew>(p, job.tile, &t)) return;
  const int kvh = job.kvh;
  const int entries = min(p.kv_len[t.stream], p.max_blocks * CS_KV_BLOCK);
  if (entries <= 0) return;
  const int row0 = (t.n_tiles - 1 - t.index) * kRowsFew;
  const int row = min(row0 + n, t.rows - 1);
  const int tok = t.q0 + row / p.group, head = kvh * p.group + row % p.group;
  const bool live = row0 + n < t.rows;
  const int pos = min(p.q_pos[tok], entries - 1);
  Query<D, PARTS> query;
  query.load(p.q, (static_cast<int64_t>(tok) * p.n_q_heads + head) * D, h);
  int last = live ? pos : -1, first = live ? pos : 0x7fffffff;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    last = max(last, __shfl_xor(last, d));
    first = min(first, __shfl_xor(first, d));
  }
  last = __builtin_amdgcn_readfirstlane(last);
  first = __builtin_amdgcn_readfirstlane(first);
  const int all_tiles = (last + kKeys) / kKeys;
  const int share = (all_tiles + p.pieces - 1) / p.pieces;
  const int kt0 = min(all_tiles, job.piece * share), kt1 = min(all_tiles, kt0 + share);

  // ---- a tile's blocks: 16 rows each, the same for all lanes; rows past the frontier are the frontier's
  const int32_t* ids = p.block_table + static_cast<int64_t>(t.stream) * p.max_blocks;
  const int last_block = max(last, 0) / CS_KV_BLOCK, last_row = max(last, 0) % CS_KV_BLOCK;
  const int64_t head_at = static_cast<int64_t>(kvh) * p.stride_head;
  cs::u32x4 kc[2][KI], vc[VC];
  uint32_t ks[2];
  int id[4];
  uint32_t vs[VC];
  auto request_ids = [&](int kt) __attribute__((always_inline)) {
#pragma unroll
    for (int b = 0; b < 4; ++b) id[b] = ids[min(4 * kt + b, last_block)];
  };
  // keys and values 32 kb .. of tile kt: cache blocks 2 kb and 2 kb + 1 of its four
  auto request = [&](int kt, int kb) __attribute__((always_inline)) {
    int64_t base[2];
    int cap[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      base[b] = static_cast<int64_t>(id[2 * kb + b]) * CS_KV_BLOCK * p.stride_slot + head_at;
      cap[b] = 4 * kt + 2 * kb + b >= last_block ? last_row : CS_KV_BLOCK - 1;
    }
    const int64_t at = (n < 16 ? base[0] : base[1]) + min(n & 15, n < 16 ? cap[0] : cap[1]) * p.stride_slot;
#pragma unroll
    for (int i = 0; i < KI; ++i) kc[kb][i] = *reinterpret_cast<const cs::u32x4*>(p.k_codes + (at + 64 * i + 32 * h) / 2);
    ks[kb] = row_scales<D>(p.k_scales, at, h);
#pragma unroll
    for (int i = 0; i < VC / 2; ++i) {
      const int r = lane / DB + i * (64 / DB);             // D 128: row of cache block i; D 64: of either
      const int64_t at_v = (r < 16 ? base[0] : base[1]) + min(r & 15, r < 16 ? cap[0] : cap[1]) * p.stride_slot + (lane % DB) * cs::kKv4Block;
      vc[kb * (VC / 2) + i] = *reinterpret_cast<const cs::u32x4*>(p.v_codes + at_v / 2);
      vs[kb * (VC / 2) + i] = p.v_scales[at_v / cs::kKv4Block];
    }
  };

  Sums<D, PARTS> sums;
  sums.clear();
  uint16_t* const v_mine = reinterpret_cast<uint16_t*>(s_mem) + wave * 32 * VROW;
  if (kt0 + wave < kt1) {
    request_ids(kt0 + wave);
    request(kt0 + wave, 0);
    request(kt0 + wave, 1);
  }
  for (int kt = kt0 + wave; kt < kt1; kt += WAVES) {
    const bool more = kt + WAVES < kt1;
    if (more) request_ids(kt + WAVES);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const int key0 = kt * kKeys + 32 * kb;
      // (LDS operations of a wave keep their order: the reads of the half before are done when these writes are)
      uint64_t none[VC / 2];
#pragma unroll
      for (int i = 0; i < VC / 2; ++i) {
        const bool b = put_values(v_mine + (lane / DB + i * (64 / DB)) * VROW + 32 * (lane % DB), vc[kb * (VC / 2) + i], vs[kb * (VC / 2) + i]);
        none[i] = __ballot(b);
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      f32x16 s = query.scores(kc[kb], ks[kb]);
      // (a key without numbers: rare, and its column of the scores is one lane's query for all lanes)
      const bool bad = (ks[kb] & 255u) == cs::kKv4NoNumber || (D == 128 && (ks[kb] >> 16 & 255u) == cs::kKv4NoNumber);
      for (uint64_t left = __ballot(bad); left; left &= left - 1) {
        const int key = (__ffsll(static_cast<unsigned long long>(left)) - 1) & 31;
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (8 * (r / 4) + 4 * h + r % 4 == key) s[r] = NAN;
      }
      if (more) request(kt + WAVES, kb);
      bf16x8 pf[PARTS][2];
      sums.weights(s, key0, pos, key0 + 31 > first, h, p.scale_log2e, pf);
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      sums.template add<VROW>(v_mine, pf, lane);
#pragma unroll
      for (int i = 0; i < VC / 2; ++i)
        for (uint64_t left = none[i]; left; left &= left - 1) {
          const int b = __ffsll(static_cast<unsigned long long>(left)) - 1;
          sums.poison(b % DB, key0 + b / DB + i * (64 / DB) <= pos);
        }
    }
  }

  // ---- the waves' results, joined: 64 columns of the output at a time
  sums.l += other_half(sums.l);
  if (h == 0) {
    s_m[wave][n] = sums.m;
    s_l[wave][n] = sums.l;
  }
  __syncthreads();
  float m = s_m[0][n];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) m = fmaxf(m, s_m[w][n]);
  float l = 0.0f;
  const float f = sums.m == -INFINITY ? (sums.l == 0.0f ? 0.0f : 1.0f) : __builtin_amdgcn_exp2f((sums.m - m) * p.scale_log2e);
#pragma unroll
  for (int w = 0; w < WAVES; ++w) l += s_m[w][n] == -INFINITY ? s_l[w][n] : s_l[w][n] * __builtin_amdgcn_exp2f((s_m[w][n] - m) * p.scale_log2e);
  float* const s_o = reinterpret_cast<float*>(s_mem);
  const int64_t job_row = static_cast<int64_t>(job.index) * kRowsFew;
  if (wave == 0 && h == 0) {
    if (p.pieces > 1) *reinterpret_cast<cs::f32v2*>(p.ws_ml + 2 * (job_row + n)) = cs::f32v2{m, l};
    else if (p.lse && live) p.lse[static_cast<int64_t>(tok) * p.n_q_heads + head] = log_sum(m, l, p.scale_log2e);
  }
  for (int half = 0; half < D / 64; ++half) {
    if (half) __syncthreads();
#pragma unroll
    for (int db = 0; db < 2; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (half == 0 ? sums.o[db][4 * g + i] : sums.o[DB == 4 ? 2 + db : db][4 * g + i]) * f;
        *reinterpret_cast<f32x4*>(s_o + (wave * 32 + n) * OROW + 32 * db + 8 * g + 4 * h) = x;
      }
    if (half == 0 && wave == 0 && h == 0) s_sum[n] = l;
    __syncthreads();
    for (int c = tid; c < 32 * 16; c += 64 * WAVES) {      // four columns of a row
      const int r = c / 16, d = 4 * (c % 16);
      if (row0 + r >= t.rows) continue;
      f32x4 x = *reinterpret_cast<const f32x4*>(s_o + r * OROW + d);
#pragma unroll
      for (int w = 1; w < WAVES; ++w) x += *reinterpret_cast<const f32x4*>(s_o + (w * 32 + r) * OROW + d);
      if (p.pieces > 1) {
        *reinterpret_cast<f32x4*>(p.ws_o + (job_row + r) * D + 64 * half + d) = x;
      } else {
        const float sum = s_sum[r], inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        const float y[4] = {x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv};
        const int rr = row0 + r;
        store4(p.out, (static_cast<int64_t>(t.q0 + rr / p.group) * p.n_q_heads + kvh * p.group + rr % p.group) * D + 64 * half + d, y, PARTS == 1);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------
// The pieces of a row tile's sweep, joined: a thread four columns of a row.
template <int D, int ROWS>
__global__ __launch_bounds__(256) void kv4_join_kernel(Params p, int bf16) {
  constexpr int PER_ROW = D / 4, AT_ONCE = 256 / PER_ROW;
  const int kvh = blockIdx.y;
  Tile t;
  if (!find_tile<ROWS>(p, blockIdx.x, &t)) return;
  if (min(p.kv_len[t.stream], p.max_blocks * CS_KV_BLOCK) <= 0) return;
  const int row0 = (t.n_tiles - 1 - t.index) * ROWS, d = 4 * (threadIdx.x % PER_ROW);
  const int64_t job0 = (static_cast<int64_t>(kvh) * p.row_tiles + blockIdx.x) * p.pieces;
  for (int r = blockIdx.z * AT_ONCE + threadIdx.x / PER_ROW; r < ROWS && row0 + r < t.rows; r += AT_ONCE * gridDim.z) {
    float m = -INFINITY, l = 0.0f;
    f32x4 o = {};
    for (int k = 0; k < p.pieces; ++k) {
      const int64_t at = (job0 + k) * ROWS + r;
      const cs::f32v2 ml = *reinterpret_cast<const cs::f32v2*>(p.ws_ml + 2 * at);
      if (ml.y == 0.0f) continue;        // (a piece without entries that the row sees; its sums are 0, or were not written)
      const float top = fmaxf(m, ml.x);
      const float fo = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - top) * p.scale_log2e);      // (sums are 0 there)
      const float fn = ml.x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((ml.x - top) * p.scale_log2e);
      const f32x4 x = *reinterpret_cast<const f32x4*>(p.ws_o + at * D + d);
      o = o * fo + x * fn;
      l = l * fo + ml.y * fn;
      m = top;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const int row = row0 + r, tok = t.q0 + row / p.group, head = kvh * p.group + row % p.group;
    const float y[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
    store4(p.out, (static_cast<int64_t>(tok) * p.n_q_heads + head) * D + d, y, bf16);
    if (p.lse && d == 0) p.lse[static_cast<int64_t>(tok) * p.n_q_heads + head] = log_sum(m, l, p.scale_log2e);
  }
}

// ---- which kernel, how many pieces
struct Route {
  bool few;
  int rows, waves;
  int64_t row_tiles, pieces, jobs;
  size_t ml, total;
};
Route route(int64_t n_q, int32_t n_streams, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_blocks) {
  Route r;
  const int group = n_q_heads / n_kv_heads;
  const int64_t busy = n_streams < n_q ? n_streams : n_q;
  r.few = n_q * group <= 64 * busy;
  r.rows = r.few ? kRowsFew : kRowsMany;
  r.row_tiles = n_q * group / r.rows + busy;               // no less than the row tiles there are, whatever cu_q says
  const int64_t jobs = r.row_tiles * n_kv_heads, tiles = (static_cast<int64_t>(max_blocks) * CS_KV_BLOCK + kKeys - 1) / kKeys;
  r.waves = 4;
  const int64_t least = r.few ? 8 : 6;                     // tiles that make a piece worth its share of the join
  r.pieces = (r.few ? 1024 : 512) / jobs;
  if (r.pieces > tiles / least) r.pieces = tiles / least;
  if (r.pieces > 64) r.pieces = 64;
  if (r.pieces < 1) r.pieces = 1;
  if (r.few && r.pieces == 1 && jobs <= 256) r.waves = 8;
  r.jobs = jobs * r.pieces;
  r.ml = r.pieces > 1 ? (static_cast<size_t>(r.jobs) * r.rows * 8 + 255) / 256 * 256 : 0;
  r.total = r.pieces > 1 ? r.ml + static_cast<size_t>(r.jobs) * r.rows * head_dim * 4 : 0;
  return r;
}

template <int D, int PARTS>
int launch(const Params& p, const Route& r, hipStream_t st) {
  const dim3 grid(static_cast<unsigned>(p.jobs_per_xcd * 8));
  if (!r.few) hipLaunchKernelGGL((kv4_rows_kernel<D, PARTS>), grid, dim3(256), 0, st, p);
  else if (r.waves == 8 && !(D == 128 && PARTS == 3))      // (whose registers a wave a SIMD takes)
    hipLaunchKernelGGL((kv4_keys_kernel<D, D == 128 ? 1 : PARTS, 8>), grid, dim3(512), 0, st, p);
  else hipLaunchKernelGGL((kv4_keys_kernel<D, PARTS, 4>), grid, dim3(256), 0, st, p);
  if (r.pieces > 1) {
    const dim3 all(static_cast<unsigned>(r.row_tiles), static_cast<unsigned>(p.n_kv_heads), r.few ? 2 : 8);
    if (r.few) hipLaunchKernelGGL((kv4_join_kernel<D, kRowsFew>), all, dim3(256), 0, st, p, PARTS == 1);
    else hipLaunchKernelGGL((kv4_join_kernel<D, kRowsMany>), all, dim3(256), 0, st, p, PARTS == 1);
  }
  return cs::note_hip(hipGetLastError());
}

}  // namespace

extern "C" size_t cs_kv4_window_attn_workspace(int64_t n_q, int32_t n_streams, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                               int32_t max_blocks) {
  if (n_q < 1 || n_streams < 1 || n_q_heads < 1 || n_kv_heads < 1 || n_q_heads < n_kv_heads || head_dim < 1 || max_blocks < 1) return 0;
  return route(n_q, n_streams, n_q_heads, n_kv_heads, head_dim, max_blocks).total;
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
  if (n_q > 0x7fffffffll / 16 || max_blocks > 0x7fffffff / CS_KV_BLOCK - kKeys) return CS_EUNSUPPORTED;
  if (n_q == 0 || n_streams == 0) return CS_OK;
  if (!q || !k_codes_layer || !k_scales_layer || !v_codes_layer || !v_scales_layer || !cu_q || !q_pos || !kv_len || !block_table || !out || max_blocks < 1)
    return CS_EINVAL;
  if (!cs::aligned16(q) || !cs::aligned16(out) || !cs::aligned16(k_codes_layer) || !cs::aligned16(v_codes_layer)) return CS_EUNSUPPORTED;
  const Route r = route(n_q, n_streams, n_q_heads, n_kv_heads, head_dim, max_blocks);
  if (r.jobs > 0x7fffffffll - 64) return CS_EUNSUPPORTED;
  if (r.total && (!workspace || workspace_bytes < r.total || !cs::aligned16(workspace))) return CS_EWORKSPACE;

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
  p.ws_ml = static_cast<float*>(workspace);
  p.ws_o = r.total ? reinterpret_cast<float*>(static_cast<char*>(workspace) + r.ml) : nullptr;
  p.n_q = n_q;
  p.stride_slot = stride_slot;
  p.stride_head = stride_head;
  p.max_blocks = max_blocks;
  p.n_streams = n_streams;
  p.n_q_heads = n_q_heads;
  p.n_kv_heads = n_kv_heads;
  p.group = n_q_heads / n_kv_heads;
  p.row_tiles = static_cast<int32_t>(r.row_tiles);
  p.pieces = static_cast<int32_t>(r.pieces);
  p.jobs = static_cast<int32_t>(r.jobs);
  p.jobs_per_xcd = static_cast<int32_t>((r.jobs + 7) / 8);
  p.scale_log2e = softmax_scale * 1.4426950408889634f;
  hipStream_t st = cs::as_stream(stream);
  if (head_dim == 128) return dtype == CS_BF16 ? launch<128, 1>(p, r, st) : launch<128, 3>(p, r, st);
  return dtype == CS_BF16 ? launch<64, 1>(p, r, st) : launch<64, 3>(p, r, st);
}
