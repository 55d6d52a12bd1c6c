// Causal attention of a batch's queries over the 4-bit window cache, gfx950: windows, questions and single tokens.
//
// out[t][h] = sum_j softmax_j(scale q[t][h] . K_j) V_j over the entries j <= q_pos[t] of the query's stream.
// A "row" is one (query token, query head of a kv group) pair, so that a tile of keys serves all heads of the group.  Keys
// pass in tiles of 64 (rows kernel at head_dim 128: of 32), 32 at a time:
//   S^T = K Q^T      v_mfma_f32_32x32x16_bf16, a lane owns one query and 16 of 32 keys.  Keys are converted to bf16, which
//                    is exact (a 4-bit value has one fraction bit).  fp32 queries are the sum of three bf16 numbers (8 + 8 + 8
//                    bits).  (v_mfma_scale_f32_32x32x64 would take the codes as they lie in the cache, against queries in 8-bit
//                    parts; but it drops what lies 2^14 below the largest product of an instruction, measured on integers:
//                    one large channel would cost the scores their low bits, 4e-5 of a score of 1 for normal data.)
//   softmax          one pass, running maximum and sum in fp32; the reference maximum is raised when a tile exceeds it by
//                    more than 2^8, so that accumulators are rarely scaled.  Weights are rounded to bf16, which the products
//                    take (half a step is 2^-8 of a weight; outputs are 0.0023 off in relative norm, 0.0017 if only they were
//                    rounded; a second part would cost as many products again); fp32 queries: three bf16 parts.  The sums of
//                    the statistics are over the unrounded ones.
//   O^T += V^T P^T   v_mfma_f32_32x32x16_bf16: P^T is in operand layout as it is, values are converted to bf16 on their way
//                    into LDS and come back by its transposing read.
// Many rows a stream (rows kernel): four waves of 32 rows share a tile in LDS.  Few rows (keys kernel): every wave holds the
// same 16 rows (16x16x32 instructions) and takes tiles of its own, with nothing but its own values in LDS; the waves join their
// results at the end.  Where there are few workgroups, the sweep of a row tile is cut into pieces of entries, whose results a second
// launch joins.
// Bounds.  Rows kernel: products and vector work (unpacking, softmax) of a wave follow each other; of the time that CUs are busy the matrix
// units work 34 %, the vector units 49 %, LDS 36 % (a quarter of that is conflicts).  32 streams of up to 389 tokens of 28 heads over up to
// 1,100 entries take 115 to 123 us, 690 to 737 TFLOP/s (a large product of the library reaches 1,200).  Keys kernel: memory; 64 streams of
// one token of 32 heads over up to 17,630 entries, 8 kv heads, take 198 us and read 982 MB, 4.9 TB/s, as fast as a large copy.
// One token over one window of 919 entries takes 9 us: a chain of one tile a wave, the join of eight waves and a launch.
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
  float* __restrict__ ws_ml;             // [jobs][rows][2]: reference maximum (raw score), sum; jobs are (row tile, piece, kv head)
  float* __restrict__ ws_o;              // [jobs][rows][D]: sums, not divided
  int64_t n_q, stride_slot, stride_head;
  int32_t max_blocks, n_streams, n_q_heads, n_kv_heads, group;
  int32_t pieces;
  float scale_log2e;
};

constexpr int kKeys = 64;                // entries of a tile
constexpr int kRowsMany = 128;           // rows of a workgroup of the rows kernel
constexpr int kRowsFew = 16;             // ... of the keys kernel
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

__device__ __forceinline__ float other_quarter(float x) {  // the value of lane ^ 16
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 16) ? r[0] : r[1]);
}

// Eight numbers as sums of PARTS bf16 numbers, the first being the rounded ones.
template <int PARTS>
__device__ __forceinline__ void split8(float (&x)[8], bf16x8 (&part)[PARTS]) {
#pragma unroll
  for (int k = 0; k < PARTS; ++k) {
    cs::u32x4 c;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      c[e] = pack2(x[2 * e], x[2 * e + 1]);
      if (k + 1 < PARTS) {
        x[2 * e] -= __uint_as_float(c[e] << 16);
        x[2 * e + 1] -= __uint_as_float(c[e] & 0xffff0000u);
      }
    }
    part[k] = __builtin_bit_cast(bf16x8, c);
  }
}

// Eight elements of a query: bf16 (PARTS 1) or fp32.
template <int PARTS>
__device__ __forceinline__ void load_parts(const void* q, int64_t at, bf16x8 (&part)[PARTS]) {
  if constexpr (PARTS == 1) {
    part[0] = *reinterpret_cast<const bf16x8*>(static_cast<const uint16_t*>(q) + at);
  } else {
    const float* src = static_cast<const float*>(q) + at;
    const cs::u32x4 a = *reinterpret_cast<const cs::u32x4*>(src), b = *reinterpret_cast<const cs::u32x4*>(src + 4);
    float x[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = __uint_as_float(a[e]);
      x[4 + e] = __uint_as_float(b[e]);
    }
    split8<PARTS>(x, part);
  }
}

// Codes of EL elements of a row: a 32-element block, or half of one.
template <int EL>
struct Codes {
  typedef typename std::conditional<EL == 32, cs::u32x4, cs::u32x2>::type V;
  V v;
  __device__ __forceinline__ void load(const uint8_t* base, uint32_t off) { v = *reinterpret_cast<const V*>(base + off); }
  __device__ __forceinline__ uint32_t word(int w) const { return v[w]; }
};

// The stream and row tile of place `target` in the launch's order.  Up to 64 streams: every stream's last row tile, then every
// stream's last but one, and so on, so that the longest sweeps start first and the launch ends on short ones; more: stream
// by stream.  Every wave scans the streams for itself.
struct Tile {
  int stream, row0, q0, rows;            // first row of the tile in the stream's rows; rows of the whole stream
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
    int l, from_end;                     // the lane of the stream, the tile's distance from the stream's last one
    if (p.n_streams <= 64) {
      uint64_t live = __ballot(tiles > 0);
      int rank = 0, left = target;
      while (left >= __popcll(live)) {
        if (live == 0) return false;
        left -= __popcll(live);
        live = __ballot(tiles > ++rank);
      }
      const bool mine = (live >> lane & 1) && __popcll(live & ((1ull << lane) - 1)) == left;
      l = __ffsll(static_cast<unsigned long long>(__ballot(mine))) - 1;
      from_end = rank;
    } else {
      int incl = tiles;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int up = __shfl_up(incl, d);
        if (lane >= d) incl += up;
      }
      const int total = __builtin_amdgcn_readlane(incl, 63);
      if (target >= before + total) {
        before += total;
        continue;
      }
      l = __ffsll(static_cast<unsigned long long>(__ballot(before + incl > target))) - 1;
      from_end = target - (before + __builtin_amdgcn_readlane(incl - tiles, __builtin_amdgcn_readfirstlane(l)));
    }
    l = __builtin_amdgcn_readfirstlane(l);
    t->stream = s0 + l;
    t->row0 = (__builtin_amdgcn_readlane(tiles, l) - 1 - __builtin_amdgcn_readfirstlane(from_end)) * ROWS;
    t->q0 = __builtin_amdgcn_readlane(a, l);
    t->rows = __builtin_amdgcn_readlane(n, l) * p.group;
    return true;
  }
  return false;
}

// Workgroup -> (row tile, piece, kv head), the kv head changing fastest: workgroups go round the eight XCDs, so that with four or
// eight kv heads an XCD's L2 serves one of them.
struct Job {
  int kvh, tile, piece, index;
};
__device__ __forceinline__ Job job_of(const Params& p) {
  Job j;
  j.index = static_cast<int>(blockIdx.x);
  j.kvh = j.index % p.n_kv_heads;
  const int i = j.index / p.n_kv_heads;
  j.piece = i % p.pieces;
  j.tile = i / p.pieces;
  return j;
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
        bf16x8 parts[PARTS];
        load_parts<PARTS>(q, at + 64 * i + 32 * h + 8 * w, parts);
#pragma unroll
        for (int k = 0; k < PARTS; ++k) part[k][i][w] = parts[k];
      }
  }

  __device__ __forceinline__ void step(f32x16& s, const bf16x8& keys, int i, int w) const {
#pragma unroll
    for (int k = PARTS - 1; k >= 0; --k) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(keys, part[k][i][w], s, 0, 0, 0);
  }

  // S^T of 32 keys in LDS: `keys` is the lane's row
  __device__ __forceinline__ f32x16 scores(const uint16_t* keys, int h) const {
    f32x16 s = {};
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int i = 0; i < D / 64; ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w) step(s, *reinterpret_cast<const bf16x8*>(keys + 64 * i + 32 * h + 8 * w), i, w);
    __builtin_amdgcn_s_setprio(0);
    return s;
  }
};

// ---- running softmax and sums of a lane's query over half tiles of 32 keys
template <int D, int PARTS>
struct Sums {
  static constexpr int DB = D / 32;
  f32x16 o[DB];
  float m, l;                            // reference maximum (raw score), the lane's share of the sum
  uint32_t bad;                          // 32-column parts of the sums that a value without numbers has reached

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = f32x16{};
    m = -INFINITY;
    l = 0.0f;
    bad = 0;
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
      bf16x8 parts[PARTS];
      split8<PARTS>(x, parts);
#pragma unroll
      for (int k = 0; k < PARTS; ++k) pf[k][st] = parts[k];
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

  // A value block without numbers (its place in LDS holds zeros) reaches the queries that see its key: noted, and put into
  // the sums at the end.
  __device__ __forceinline__ void poison(int db, bool sees) { bad |= sees ? 1u << db : 0u; }

  __device__ __forceinline__ void finish() {
    l += other_half(l);
    if (__builtin_expect(__any(bad != 0), 0)) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
        if (bad >> db & 1) {
#pragma unroll
          for (int r = 0; r < 16; ++r) o[db][r] = NAN;
        }
    }
  }
};

// A block of 32 elements -> bf16 in LDS.  A block without numbers becomes NaN (keys) or zeros (values, which must not meet a weight of
// 0; infinite elements of values become zeros as well, and such blocks are reported).  KIND 0: keys, rows 16 bytes past a multiple of the
// banks' width.  Values: 1: rows 64 bytes past one, 2: 32 bytes; there blocks of neighbouring rows share banks, and lanes of different
// rows write a block's four pieces in different orders (by two bits of `row`, or the second one).
template <int KIND>
__device__ __forceinline__ bool put_block(uint16_t* dst, const cs::u32x4& code, uint32_t scale, int row) {
  const bool odd_one = scale >= (KIND == 0 ? cs::kKv4NoNumber : cs::kKv4Large);
  const float sc = cs::kv4_scale(odd_one ? 1u : scale);
  cs::u32x4 c = code;
  const int turn = KIND == 1 ? row & 3 : KIND == 2 ? (row >> 1) & 1 : 0;       // c[w] = code[w ^ turn]
  if (KIND != 0) {
    const bool odd = turn & 1;
    c = cs::u32x4{odd ? c.y : c.x, odd ? c.x : c.y, odd ? c.w : c.z, odd ? c.z : c.w};
  }
  if (KIND == 1) {
    const bool high = turn & 2;
    c = cs::u32x4{high ? c.z : c.x, high ? c.w : c.y, high ? c.x : c.z, high ? c.y : c.w};
  }
#pragma unroll
  for (int w = 0; w < 4; ++w) *reinterpret_cast<cs::u32x4*>(dst + 8 * (w ^ turn)) = cs::kv4_unpack8_bf16(c[w], sc);
  if (__builtin_expect(odd_one, 0)) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t none = KIND != 0 ? 0u : 0x7fc07fc0u;
      cs::u32x4 x = {none, none, none, none};
      if (KIND != 0 && scale != cs::kKv4NoNumber) {
        x = cs::kv4_unpack8_bf16(code[w], cs::kv4_scale(scale));
#pragma unroll
        for (int e = 0; e < 4; ++e)
          x[e] = ((x[e] & 0x7fffu) == 0x7f80u ? 0u : x[e] & 0xffffu) | ((x[e] & 0x7fff0000u) == 0x7f800000u ? 0u : x[e] & 0xffff0000u);
      }
      *reinterpret_cast<cs::u32x4*>(dst + 8 * w) = x;
    }
  }
  return odd_one;
}

// What element e of a block of values adds to a sum past the products: an infinity, or 0.  (Scale 253: 4 and 6 times 2^126 are past
// the largest finite number, 254: 2 times 2^127 and more.)
__device__ __forceinline__ float infinity_of(const cs::u32x4& code, uint32_t scale, int e) {
  const uint32_t word = e < 16 ? (e < 8 ? code.x : code.y) : (e < 24 ? code.z : code.w), c = word >> (4 * (e & 7)) & 15u;
  if ((c & 7u) < (scale == cs::kKv4Large ? 6u : 4u)) return 0.0f;
  return c & 8u ? -INFINITY : INFINITY;
}

// Where a sweep has met infinite values (rare), it looks them up again: f(entry, block, codes, scale) for every block of the entries begin
// .. end - 1 that may hold some, the whole wave at once.
template <int DB, class F>
__device__ __forceinline__ void each_large_block(const Params& p, const int32_t* ids, int kvh, int begin, int end, F f) {
  const int mine = static_cast<int>(threadIdx.x & 63) / DB, block = static_cast<int>(threadIdx.x & 63) % DB;
  for (int key0 = begin; key0 < end; key0 += 64 / DB) {
    const int key = min(key0 + mine, end - 1);
    const int64_t at = (static_cast<int64_t>(ids[key / CS_KV_BLOCK]) * CS_KV_BLOCK + key % CS_KV_BLOCK) * p.stride_slot +
                       static_cast<int64_t>(kvh) * p.stride_head + block * cs::kKv4Block;
    const uint32_t scale = p.v_scales[at / cs::kKv4Block];
    const cs::u32x4 code = *reinterpret_cast<const cs::u32x4*>(p.v_codes + at / 2);
    for (uint64_t left = __ballot(scale >= cs::kKv4Large && scale != cs::kKv4NoNumber && key == key0 + mine); left; left &= left - 1) {
      const int l = __ffsll(static_cast<unsigned long long>(left)) - 1;
      cs::u32x4 c;
#pragma unroll
      for (int w = 0; w < 4; ++w) c[w] = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(code[w]), l));
      f(key0 + l / DB, l % DB, c, static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(scale), l)));
    }
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

// ------------------------------------------------------------------------------------------
// Many rows: four waves of 32 rows share the tiles of a sweep, 32 keys (head_dim 64: 64).  A thread moves one block of 32 elements a
// tile, the first two waves keys, the others values: asked for a tile ahead into registers, put into LDS as bf16, in two
// stages, so that a tile costs one barrier.
template <int D, int PARTS>
__global__ __launch_bounds__(256, PARTS == 1 ? 3 : D == 64 ? 2 : 1) void kv4_rows_kernel(Params p) {
  constexpr int DB = D / 32;
  constexpr int T = 128 / DB;                              // keys of a tile
  constexpr int KROW = D + 8, VROW = D + 32;               // padded: reads of eight rows, and the transposing ones, start in banks of their own
  __shared__ __attribute__((aligned(16))) uint16_t s_k[2][T * KROW];
  __shared__ __attribute__((aligned(16))) uint16_t s_v[2][T * VROW];
  __shared__ uint8_t s_vs[2][128];
  __shared__ int s_last[4];
  __shared__ uint32_t s_odd;                               // values met so far: 1: without numbers, 2: infinite

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
  const Job job = job_of(p);
  Tile t;
  if (!find_tile<kRowsMany>(p, job.tile, &t)) return;
  const int kvh = job.kvh;
  const int entries = min(p.kv_len[t.stream], p.max_blocks * CS_KV_BLOCK);
  if (entries <= 0) return;
  if (tid == 0) s_odd = 0;

  // ---- this lane's query
  const int row0 = t.row0 + wave * 32;
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
  const int last = __builtin_amdgcn_readfirstlane(max(max(s_last[0], s_last[1]), max(s_last[2], s_last[3])));
  const int all_tiles = (last + T) / T;                    // (no entry seen: last -1, no tile)
  const int share = (all_tiles + p.pieces - 1) / p.pieces;
  const int kt0 = min(all_tiles, job.piece * share), kt1 = min(all_tiles, kt0 + share);

  // ---- tile requests
  const int32_t* ids = p.block_table + static_cast<int64_t>(t.stream) * p.max_blocks;
  const bool of_v = wave >= 2;
  const uint8_t* codes = of_v ? p.v_codes : p.k_codes;
  const uint8_t* scales = of_v ? p.v_scales : p.k_scales;
  const int my_row = (tid & 127) / DB, my_block = tid % DB;
  // (a thread's place in cache block 0, in the frontier's row of it, and what a block adds: stride_slot < 2^26)
  const int64_t head_at = static_cast<int64_t>(kvh) * p.stride_head + my_block * cs::kKv4Block;
  const int64_t at_row = static_cast<int64_t>(my_row % CS_KV_BLOCK) * p.stride_slot + head_at;
  const int64_t at_last = static_cast<int64_t>(max(last, 0) % CS_KV_BLOCK) * p.stride_slot + head_at;
  const uint32_t code_step = static_cast<uint32_t>(p.stride_slot * CS_KV_BLOCK / 2), scale_step = static_cast<uint32_t>(p.stride_slot / 2);
  const uint8_t* const my_code = codes + at_row / 2;
  const uint8_t* const my_scale = scales + at_row / cs::kKv4Block;
  // Two tiles are under way while one is computed on: a tile of 32 keys takes less time than its codes.
  cs::u32x4 code[2];
  uint32_t scale[2];
  // A wave's rows lie in one cache block (head_dim 64: two): its id is the same in all lanes, and a scalar load keeps out of the
  // queue of vector loads, in which waiting for it would be waiting for the codes asked for before.
  const int last_block = max(last, 0) / CS_KV_BLOCK, first_block = (wave & 1) * (T / CS_KV_BLOCK / 2);
  int id[2];
  auto request_id = [&](int kt) __attribute__((always_inline)) {
#pragma unroll
    for (int b = 0; b < T / CS_KV_BLOCK / 2; ++b) id[b] = ids[min(kt * (T / CS_KV_BLOCK) + first_block + b, last_block)];
  };
  // rows past the frontier are the frontier's row (what lies there may be nothing)
  auto request = [&](int kt, int at) __attribute__((always_inline)) {
    const uint8_t *c = my_code, *s = my_scale;
    if (kt * T + T - 1 > last && kt * T + my_row > last) {
      c = codes + at_last / 2;
      s = scales + at_last / cs::kKv4Block;
    }
    const uint32_t block = static_cast<uint32_t>(T == 64 && lane >= 32 ? id[T == 64 ? 1 : 0] : id[0]);
    code[at] = *reinterpret_cast<const cs::u32x4*>(c + static_cast<uint64_t>(block) * code_step);
    scale[at] = s[static_cast<uint64_t>(block) * scale_step];
  };
  auto put = [&](int buf) __attribute__((always_inline)) {       // tile kt0 + k: stage k & 1 of the registers and of LDS
    if (of_v) {
      if (put_block<1>(&s_v[buf][my_row * VROW + 32 * my_block], code[buf], scale[buf], my_row))
        atomicOr(&s_odd, scale[buf] == cs::kKv4NoNumber ? 1u : 2u);
      s_vs[buf][tid & 127] = static_cast<uint8_t>(scale[buf]);
    } else {
      put_block<0>(&s_k[buf][my_row * KROW + 32 * my_block], code[buf], scale[buf], my_row);
    }
  };

  Sums<D, PARTS> sums;
  sums.clear();
  auto tile = [&](int kt, auto stage) __attribute__((always_inline)) {
    constexpr int buf = decltype(stage)::value;
    const uint32_t odd = s_odd;                            // (read ahead of the products)
#pragma unroll
    for (int kb = 0; kb < T / 32; ++kb) {
      const int key0 = kt * T + 32 * kb;
      if (key0 > wave_last) continue;
      bf16x8 pf[PARTS][2];
      sums.weights(query.scores(&s_k[buf][(32 * kb + n) * KROW], h), key0, pos, key0 + 31 > wave_first, h, p.scale_log2e, pf);
      __builtin_amdgcn_s_setprio(1);                       // (products before other waves' vector work: 2-3 % for these and the scores)
      sums.template add<VROW>(&s_v[buf][32 * kb * VROW], pf, lane);
      __builtin_amdgcn_s_setprio(0);
    }
    if (__builtin_expect(__builtin_amdgcn_readfirstlane(odd) & 1u, 0)) {      // (a tile so far held a value block without numbers)
      for (int c = 0; c < 128; ++c)
        if (s_vs[buf][c] == cs::kKv4NoNumber) sums.poison(c % DB, kt * T + c / DB <= pos);
    }
    // (requests past the end made the last tile's instead, so that a wait for one is not a wait for all, were level or 2 % slower)
    if (kt + 1 < kt1) put(buf ^ 1);
    if (kt + 3 < kt1) request(kt + 3, buf ^ 1);
    if (kt + 4 < kt1) request_id(kt + 4);
    __syncthreads();
  };
  if (kt0 < kt1) {
    request_id(kt0);
    request(kt0, 0);
    if (kt0 + 1 < kt1) {
      request_id(kt0 + 1);
      request(kt0 + 1, 1);
    }
    if (kt0 + 2 < kt1) request_id(kt0 + 2);
    put(0);
    if (kt0 + 2 < kt1) request(kt0 + 2, 0);
    if (kt0 + 3 < kt1) request_id(kt0 + 3);
    __syncthreads();
  }
  for (int kt = kt0; kt < kt1; kt += 2) {
    tile(kt, std::integral_constant<int, 0>());
    if (kt + 1 < kt1) tile(kt + 1, std::integral_constant<int, 1>());
  }

  // ---- results
  sums.finish();
  if (__builtin_expect(__builtin_amdgcn_readfirstlane(s_odd) & 2u, 0))
    each_large_block<DB>(p, ids, kvh, kt0 * T, min(kt1 * T, last + 1), [&](int key, int block, const cs::u32x4& c, uint32_t sc) __attribute__((always_inline)) {
      if (key > pos) return;
#pragma unroll
      for (int db = 0; db < DB; ++db)
        if (db == block) {
#pragma unroll
          for (int r = 0; r < 16; ++r) sums.o[db][r] += infinity_of(c, sc, 8 * (r / 4) + 4 * h + r % 4);
        }
    });
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
// Few rows: WAVES waves hold the same 16 rows and take every WAVES-th tile of the sweep, each for itself: a wave's keys go
// from memory into operand registers, its values through its own 32 rows of LDS.  No barrier before the end.
// v_mfma_f32_16x16x32_bf16: lane l is query l % 16; of a 16-key cache block it holds, as an operand, key l % 16 and a quarter of
// its elements (head_dim 128: one 32-element block, so that a wave reads a cache block in one load), and of the scores keys
// 4 (l / 16) + 0..3.
template <int D, int PARTS, int WAVES>
__global__ __launch_bounds__(64 * WAVES, PARTS == 1 ? 3 : 2) void kv4_keys_kernel(Params p) {
  constexpr int DB = D / 32, EL = D / 4, SW = EL / 8;      // blocks of a row; elements of a lane's key; steps of a key's sum
  constexpr int VROW = D + 16;                             // padded: eight rows of 32 bytes start in banks of their own (counted: two fifths of its LDS cycles are conflicts all the same)
  constexpr int VC = 32 * DB / 64;                         // value blocks of 32 keys that a lane moves
  constexpr int OROW = D + 4;
  constexpr int BYTES = 32 * VROW * 2 > 16 * OROW * 4 ? 32 * VROW * 2 : 16 * OROW * 4;
  __shared__ __attribute__((aligned(16))) uint8_t s_mem[WAVES][BYTES];
  __shared__ float s_m[WAVES][16], s_l[WAVES][16], s_sum[16];
  __shared__ int s_pos[16], s_large[WAVES];                // positions of the rows; whether a wave met infinite values

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
  const Job job = job_of(p);
  Tile t;
  if (!find_tile<kRowsFew>(p, job.tile, &t)) return;
  const int kvh = job.kvh;
  const int entries = min(p.kv_len[t.stream], p.max_blocks * CS_KV_BLOCK);
  if (entries <= 0) return;
  const int row = min(t.row0 + n, t.rows - 1);
  const int tok = t.q0 + row / p.group, head = kvh * p.group + row % p.group;
  const bool live = t.row0 + n < t.rows;
  const int pos = min(p.q_pos[tok], entries - 1);

  // ---- the lane's query: elements EL g + 8 w + 0..7 in step w
  bf16x8 qf[PARTS][SW];
  {
    const int64_t at = (static_cast<int64_t>(tok) * p.n_q_heads + head) * D + EL * g;
#pragma unroll
    for (int w = 0; w < SW; ++w) {
      bf16x8 parts[PARTS];
      load_parts<PARTS>(p.q, at + 8 * w, parts);
#pragma unroll
      for (int k = 0; k < PARTS; ++k) qf[k][w] = parts[k];
    }
  }
  int last = live ? pos : -1, first = live ? pos : 0x7fffffff;
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) {
    last = max(last, __shfl_xor(last, d));
    first = min(first, __shfl_xor(first, d));
  }
  last = __builtin_amdgcn_readfirstlane(last);
  first = __builtin_amdgcn_readfirstlane(first);
  const int all_tiles = (last + kKeys) / kKeys;
  const int share = (all_tiles + p.pieces - 1) / p.pieces;
  const int kt0 = min(all_tiles, job.piece * share), kt1 = min(all_tiles, kt0 + share);

  // ---- a tile is four cache blocks; their ids, and so the addresses of their first rows, are the same in all lanes
  const int32_t* ids = p.block_table + static_cast<int64_t>(t.stream) * p.max_blocks;
  const int last_block = max(last, 0) / CS_KV_BLOCK, last_row = max(last, 0) % CS_KV_BLOCK;
  const uint32_t row_bytes = static_cast<uint32_t>(p.stride_slot / 2), row_scales = static_cast<uint32_t>(p.stride_slot / cs::kKv4Block);
  const int64_t head_at = static_cast<int64_t>(kvh) * p.stride_head;
  const uint8_t *k_head = p.k_codes + head_at / 2, *v_head = p.v_codes + head_at / 2;
  const uint8_t *ks_head = p.k_scales + head_at / cs::kKv4Block, *vs_head = p.v_scales + head_at / cs::kKv4Block;
  const int v_row = lane / DB, v_block = lane % DB;        // D 128: row of a cache block; D 64: of a pair of them
  Codes<EL> kc[4];
  cs::u32x4 vc[2][VC];
  uint32_t ks[4], vs[2][VC];
  int id[4];
  auto request_ids = [&](int kt) __attribute__((always_inline)) {
#pragma unroll
    for (int b = 0; b < 4; ++b) id[b] = ids[min(4 * kt + b, last_block)];
  };
  // keys and values 32 kb .. of tile kt; rows past the frontier are the frontier's row (what lies there may be nothing)
  auto request = [&](int kt, int kb) __attribute__((always_inline)) {
    uint64_t at[2], at_s[2];
    int cap[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      at[b] = static_cast<uint64_t>(static_cast<uint32_t>(id[2 * kb + b])) * (CS_KV_BLOCK * row_bytes);
      at_s[b] = static_cast<uint64_t>(static_cast<uint32_t>(id[2 * kb + b])) * (CS_KV_BLOCK * row_scales);
      cap[b] = 4 * kt + 2 * kb + b >= last_block ? last_row : CS_KV_BLOCK - 1;
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint32_t r = min(n, cap[b]);
      kc[2 * kb + b].load(k_head + at[b], r * row_bytes + g * (EL / 2));
      ks[2 * kb + b] = (ks_head + at_s[b])[r * row_scales + g * EL / cs::kKv4Block];
    }
#pragma unroll
    for (int i = 0; i < VC; ++i) {
      if constexpr (DB == 4) {
        const uint32_t r = min(v_row, cap[i]);
        vc[kb][i] = *reinterpret_cast<const cs::u32x4*>(v_head + at[i] + (r * row_bytes + v_block * 16));
        vs[kb][i] = (vs_head + at_s[i])[r * row_scales + v_block];
      } else {
        const bool second = v_row >= CS_KV_BLOCK;
        const uint32_t r = min(v_row % CS_KV_BLOCK, second ? cap[1] : cap[0]);
        vc[kb][i] = *reinterpret_cast<const cs::u32x4*>(v_head + (second ? at[1] : at[0]) + (r * row_bytes + v_block * 16));
        vs[kb][i] = (vs_head + (second ? at_s[1] : at_s[0]))[r * row_scales + v_block];
      }
    }
  };

  f32x4 o[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) o[i] = f32x4{};
  float m = -INFINITY, l = 0.0f;                           // reference maximum (raw score), the lane's share of the sum
  bool large = false;                                      // infinite values met
  uint32_t bad = 0;                                        // 32-column parts of the sums that a value without numbers has reached
  uint16_t* const v_mine = reinterpret_cast<uint16_t*>(s_mem[wave]);
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
      // ---- values to LDS (the operations of a wave on it keep their order: the reads of the half before are done by then)
      uint64_t none[VC];
#pragma unroll
      for (int i = 0; i < VC; ++i) {
        const int r = DB == 4 ? v_row + CS_KV_BLOCK * i : v_row;
        none[i] = __ballot(put_block<2>(v_mine + r * VROW + 32 * v_block, vc[kb][i], vs[kb][i], v_row));
        if (__builtin_expect(none[i] != 0, 0)) {
          const uint64_t without = __ballot(vs[kb][i] == cs::kKv4NoNumber);
          large |= none[i] != without;
          none[i] = without;
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      // ---- S^T
      f32x4 s[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        s[b] = f32x4{};
        const uint32_t e = ks[2 * kb + b];
        const float sc = cs::kv4_scale(e == cs::kKv4NoNumber ? 1u : e);
#pragma unroll
        for (int w = 0; w < SW; ++w) {
          const bf16x8 kf = __builtin_bit_cast(bf16x8, cs::kv4_unpack8_bf16(kc[2 * kb + b].word(w), sc));
#pragma unroll
          for (int k = PARTS - 1; k >= 0; --k) s[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[k][w], s[b], 0, 0, 0);
        }
        // (a key without numbers: rare)
        for (uint64_t left = __ballot(e == cs::kKv4NoNumber); left; left &= left - 1) {
          const int key = (__ffsll(static_cast<unsigned long long>(left)) - 1) & 15;
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (4 * g + r == key) s[b][r] = NAN;
        }
      }
      if (more) request(kt + WAVES, kb);
      if (key0 + 31 > first) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (key0 + 16 * b + 4 * g + r > pos) s[b][r] = -INFINITY;
      }
      // ---- softmax
      float top = s[0][0];
#pragma unroll
      for (int r = 1; r < 8; ++r) top = fmaxf(top, s[r / 4][r % 4]);
      top = fmaxf(top, other_quarter(top));
      top = fmaxf(top, other_half(top));
      if (__any((top - m) * p.scale_log2e > kSlack || m == -INFINITY)) {
        const float raised = fmaxf(m, top);
        const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - raised) * p.scale_log2e);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[i] *= f;
        l *= f;
        m = raised;
      }
      const float base = m == -INFINITY ? 0.0f : -m * p.scale_log2e;
      float x[8], sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = __builtin_amdgcn_exp2f(fmaf(s[i / 4][i % 4], p.scale_log2e, base));
        sum += x[i];
      }
      l += sum;
      bf16x8 pf[PARTS];
      split8<PARTS>(x, pf);
      // ---- O^T: a lane's weights are of keys 4 g + 0..3 of either cache block
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      const uint16_t* v_at = v_mine + (4 * g + (n >> 2)) * VROW + 4 * (n & 3);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(v_at + 16 * i));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(v_at + 16 * i + 16 * VROW));
        const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int k = PARTS - 1; k >= 0; --k) o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[k], o[i], 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < VC; ++i)
        for (uint64_t left = none[i]; left; left &= left - 1) {
          const int b = __ffsll(static_cast<unsigned long long>(left)) - 1;
          if (key0 + b / DB + CS_KV_BLOCK * i <= pos) bad |= 1u << (b % DB);
        }
    }
  }

  // ---- the waves' results, joined
  l += other_quarter(l);
  l += other_half(l);
  if (__builtin_expect(__any(bad != 0), 0)) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
      if (bad >> (i / 2) & 1) o[i] = f32x4{NAN, NAN, NAN, NAN};
  }
  if (g == 0) {
    s_m[wave][n] = m;
    s_l[wave][n] = l;
  }
  if (lane == 0) s_large[wave] = large;
  if (wave == 0 && g == 0) s_pos[n] = live ? pos : -1;
  __syncthreads();
  float top = s_m[0][n], sum = 0.0f;
#pragma unroll
  for (int w = 1; w < WAVES; ++w) top = fmaxf(top, s_m[w][n]);
#pragma unroll
  for (int w = 0; w < WAVES; ++w) sum += s_m[w][n] == -INFINITY ? s_l[w][n] : s_l[w][n] * __builtin_amdgcn_exp2f((s_m[w][n] - top) * p.scale_log2e);
  const float f = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - top) * p.scale_log2e);      // (sums are 0, or NaN, where m is -inf)
  float* const s_o = reinterpret_cast<float*>(s_mem[wave]);
#pragma unroll
  for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4*>(s_o + n * OROW + 16 * i + 4 * g) = o[i] * f;
  const int64_t job_row = static_cast<int64_t>(job.index) * kRowsFew;
  if (wave == 0 && g == 0) {
    s_sum[n] = sum;
    if (p.pieces > 1) *reinterpret_cast<cs::f32v2*>(p.ws_ml + 2 * (job_row + n)) = cs::f32v2{top, sum};
    else if (p.lse && live) p.lse[static_cast<int64_t>(tok) * p.n_q_heads + head] = log_sum(top, sum, p.scale_log2e);
  }
  __syncthreads();
  int any_large = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) any_large |= s_large[w];
  for (int c = tid; c < 16 * D / 4; c += 64 * WAVES) {     // four columns of a row
    const int r = c / (D / 4), d = 4 * (c % (D / 4)), rr = t.row0 + r;
    f32x4 y = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(s_mem[0]) + r * OROW + d);
#pragma unroll
    for (int w = 1; w < WAVES; ++w) y += *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(s_mem[w]) + r * OROW + d);
    if (__builtin_expect(__builtin_amdgcn_readfirstlane(any_large), 0)) {
      const int sees = s_pos[r];
      each_large_block<DB>(p, ids, kvh, kt0 * kKeys, min(kt1 * kKeys, last + 1), [&](int key, int block, const cs::u32x4& codes, uint32_t sc) __attribute__((always_inline)) {
        if (key > sees || d / 32 != block) return;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] += infinity_of(codes, sc, d % 32 + i);
      });
    }
    if (rr >= t.rows) continue;
    if (p.pieces > 1) {
      *reinterpret_cast<f32x4*>(p.ws_o + (job_row + r) * D + d) = y;
    } else {
      const float inv = s_sum[r] == 0.0f ? 0.0f : 1.0f / s_sum[r];
      const float z[4] = {y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv};
      store4(p.out, (static_cast<int64_t>(t.q0 + rr / p.group) * p.n_q_heads + kvh * p.group + rr % p.group) * D + d, z, PARTS == 1);
    }
  }
}

// ------------------------------------------------------------------------------------------
// The pieces of a row tile's sweep, joined: a thread four columns of a row.  SLICED: the workgroup's eight (head_dim 64: sixteen) groups
// of lanes that make a row share the pieces of one row, and meet in LDS.
template <int D, int ROWS, bool SLICED>
__global__ __launch_bounds__(256) void kv4_join_kernel(Params p, int bf16) {
  constexpr int PER_ROW = D / 4, GROUPS = 256 / PER_ROW;
  __shared__ __attribute__((aligned(16))) float s_o[SLICED ? GROUPS : 1][D];
  __shared__ float s_m[GROUPS], s_l[GROUPS];
  const int kvh = blockIdx.y, grp = threadIdx.x / PER_ROW, d = 4 * (threadIdx.x % PER_ROW);
  Tile t;
  if (!find_tile<ROWS>(p, blockIdx.x, &t)) return;
  if (min(p.kv_len[t.stream], p.max_blocks * CS_KV_BLOCK) <= 0) return;
  const int r = SLICED ? static_cast<int>(blockIdx.z) : static_cast<int>(blockIdx.z) * GROUPS + grp;
  const bool live = r < ROWS && t.row0 + r < t.rows;
  if (SLICED && !live) return;
  const int64_t job0 = static_cast<int64_t>(blockIdx.x) * p.pieces * p.n_kv_heads + kvh;
  float m = -INFINITY, l = 0.0f;
  f32x4 o = {};
  auto add = [&](float pm, float pl, const f32x4& x) __attribute__((always_inline)) {
    const float top = fmaxf(m, pm);
    const float fo = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - top) * p.scale_log2e);      // (sums are 0 there)
    const float fn = pm == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((pm - top) * p.scale_log2e);
    o = o * fo + x * fn;
    l = l * fo + pl * fn;
    m = top;
  };
  constexpr int STEP = SLICED ? GROUPS : 1;
  if (live)
    for (int k0 = SLICED ? grp : 0; k0 < p.pieces; k0 += 4 * STEP) {       // (four under way at once)
      cs::f32v2 ml[4];
      f32x4 x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int64_t at = (job0 + static_cast<int64_t>(min(k0 + k * STEP, p.pieces - 1)) * p.n_kv_heads) * ROWS + r;
        ml[k] = *reinterpret_cast<const cs::f32v2*>(p.ws_ml + 2 * at);
        x[k] = *reinterpret_cast<const f32x4*>(p.ws_o + at * D + d);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k0 + k * STEP < p.pieces && ml[k].y != 0.0f) add(ml[k].x, ml[k].y, x[k]);      // (0: a piece without entries that the row sees)
    }
  if (SLICED) {
    *reinterpret_cast<f32x4*>(&s_o[SLICED ? grp : 0][d]) = o;
    if (d == 0) {
      s_m[grp] = m;
      s_l[grp] = l;
    }
    __syncthreads();
    if (grp != 0) return;
    for (int g = 1; g < GROUPS; ++g)
      if (s_l[g] != 0.0f) add(s_m[g], s_l[g], *reinterpret_cast<const f32x4*>(&s_o[SLICED ? g : 0][d]));
  }
  if (!live) return;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  const int row = t.row0 + r, tok = t.q0 + row / p.group, head = kvh * p.group + row % p.group;
  const float y[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
  store4(p.out, (static_cast<int64_t>(tok) * p.n_q_heads + head) * D + d, y, bf16);
  if (p.lse && d == 0) p.lse[static_cast<int64_t>(tok) * p.n_q_heads + head] = log_sum(m, l, p.scale_log2e);
}

// ---- which kernel, how many pieces
// Tiles that make a piece worth its share of the join, of the keys and the rows kernel.  4 kv heads of 7 query heads, head_dim 128, calls
// back to back: one token over 919 entries takes 9.5 to 9.9 us uncut (8), 11.7 to 13.6 in pieces (6), over 1,500 12.1 to 12.6 at 8 and
// 11.5 at 16, over 17,630 14.0 and 17.1;
// 424 tokens over 919 take 30.5 us at 6, 28.8 at 4, 31.4 at 3.
constexpr int kLeastFew = 8, kLeastMany = 4;
// Pieces above which a workgroup shares a row's: 64 tokens over 17,630 entries (48 pieces) take 45.6 us, 61 us with one thread walking
// all pieces of its columns; 7 streams of 40 tokens over up to 5,000 (9 pieces) 57 us shared, 52 us walked.
constexpr int kSliced = 16;
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
  // The keys kernel up to four of its row tiles a stream: 8 tokens of 7 heads (56 rows) over 17,630 entries take 18.9 us in it, 22.1 us
  // in the rows kernel; 16 tokens (112 rows) 26.7 and 24.0 us, 64 streams of those over 4,000 151 and 135.
  r.few = n_q * group <= 64 * busy;
  r.rows = r.few ? kRowsFew : kRowsMany;
  r.row_tiles = n_q * group / r.rows + busy;               // no less than the row tiles there are, whatever cu_q says
  const int64_t jobs = r.row_tiles * n_kv_heads, tiles = (static_cast<int64_t>(max_blocks) * CS_KV_BLOCK + kKeys - 1) / kKeys;
  r.waves = 4;
  const int64_t least = r.few ? kLeastFew : kLeastMany;
  // Pieces for two rounds of what the card holds at once (keys: 4 waves each; half of it costs 14.2 -> 15.8 us for 16 tokens of 16
  // streams, twice it changes nothing) and three workgroups a CU (rows; of fp32 queries two fit: 64 tokens over 17,630 entries take 45 us, with half as
  // many 47.8, with twice 51).  The rows kernel counts the row tiles that streams of one length would have (64 streams of 16 tokens over
  // 4,000: 97 us, 135 by the bound on any lengths); the keys kernel the bound (64 streams of a token over 8,000: 103 us, 116 us).
  const int64_t even = (n_q * group + busy * r.rows - 1) / (busy * r.rows) * busy * n_kv_heads;     // jobs of streams of one length
  r.pieces = (r.few ? 1024 : 768) / (!r.few && even < jobs ? even : jobs);
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
  const dim3 grid(static_cast<unsigned>(r.jobs));
  if (!r.few) hipLaunchKernelGGL((kv4_rows_kernel<D, PARTS>), grid, dim3(256), 0, st, p);
  else if (r.waves == 8) hipLaunchKernelGGL((kv4_keys_kernel<D, PARTS, 8>), grid, dim3(512), 0, st, p);
  else hipLaunchKernelGGL((kv4_keys_kernel<D, PARTS, 4>), grid, dim3(256), 0, st, p);
  if (r.pieces > 1) {
    const unsigned tiles = static_cast<unsigned>(r.row_tiles), heads = static_cast<unsigned>(p.n_kv_heads);
    constexpr int at_once = 256 / (D / 4);
    const dim3 whole(tiles, heads, (r.rows + at_once - 1) / at_once), sliced(tiles, heads, r.rows);
    if (r.few && r.pieces > kSliced) hipLaunchKernelGGL((kv4_join_kernel<D, kRowsFew, true>), sliced, dim3(256), 0, st, p, PARTS == 1);
    else if (r.few) hipLaunchKernelGGL((kv4_join_kernel<D, kRowsFew, false>), whole, dim3(256), 0, st, p, PARTS == 1);
    else if (r.pieces > kSliced) hipLaunchKernelGGL((kv4_join_kernel<D, kRowsMany, true>), sliced, dim3(256), 0, st, p, PARTS == 1);
    else hipLaunchKernelGGL((kv4_join_kernel<D, kRowsMany, false>), whole, dim3(256), 0, st, p, PARTS == 1);
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
  if (!cs::kv4_strides(stride_slot, stride_head, 0) || stride_slot >= (1 << 26)) return CS_EUNSUPPORTED;
  if (n_q >= (1 << 26) || max_blocks > 0x7fffffff / CS_KV_BLOCK - kKeys) return CS_EUNSUPPORTED;
  if (n_q == 0 || n_streams == 0) return CS_OK;
  if (!q || !k_codes_layer || !k_scales_layer || !v_codes_layer || !v_scales_layer || !cu_q || !q_pos || !kv_len || !block_table || !out || max_blocks < 1)
    return CS_EINVAL;
  if (!cs::aligned16(q) || !cs::aligned16(out) || !cs::aligned16(k_codes_layer) || !cs::aligned16(v_codes_layer)) return CS_EUNSUPPORTED;
  const Route r = route(n_q, n_streams, n_q_heads, n_kv_heads, head_dim, max_blocks);
  if (r.jobs > cs::kMostThreads / 512) return CS_EUNSUPPORTED;
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
  p.pieces = static_cast<int32_t>(r.pieces);
  p.scale_log2e = softmax_scale * 1.4426950408889634f;
  hipStream_t st = cs::as_stream(stream);
  if (head_dim == 128) return dtype == CS_BF16 ? launch<128, 1>(p, r, st) : launch<128, 3>(p, r, st);
  return dtype == CS_BF16 ? launch<64, 1>(p, r, st) : launch<64, 3>(p, r, st);
}
