// Attention over the blocks that were selected for each query, paged 16-bit or fp32 cache, gfx950: single tokens, questions, windows.
//
//     out[t][h] = sum_j softmax_j(scale q[t][h] . K_j) V_j    over the entries j <= q_pos[t] of the blocks listed for (t, kv head of h)
//
// A row is one (query token, query head of the kv group) pair; 16 rows are a tile: as many tokens of a stream as fit, T = 16 / group (one
// token where its heads fill the tile).  A workgroup takes a tile and a kv head, or a piece of its sweep:
//   lists      the tokens' lists become one ascending list of different blocks, each with a mask of the tokens that read it: every
//              element counts the ones before it (at most 256 of them, in LDS), so the caller's order does not matter and an
//              index that stands twice counts once
//   S^T        = K Q^T over 16 keys (bf16: v_mfma_f32_16x16x32_bf16, fp32: v_mfma_f32_16x16x4_f32), keys straight from memory in operand
//              layout; a lane owns one row and 4 keys
//   softmax    one pass, running maximum and sum in fp32; the reference is raised when a tile exceeds it by more than 2^8.  It is held as the
//              rounded exponent that it stands for, m = round(scale log2(e) s): weights are 2^(scale log2(e) s - m), with one rounding, and
//              what was summed against another m is taken over by 2^(m - m'), so that no rounding of m reaches the result.
//              bf16: weights are rounded to bf16, which the products take (half a step is 2^-8 of a weight); their sum is not
//   O^T       += V^T P^T; P^T is in operand layout as it is.  bf16 values pass through a wave's own part of LDS, whose transposing read
//              gives the operand; fp32 values come from memory in operand layout
// The waves of a workgroup take key tiles in turn and join their results at the end; pieces are joined by a second launch.  Few rows are bound
// by latency (a token over 16 blocks of 64: 10.6 us, both launches), many tokens of their own windows by memory (64 tokens, 278 MB: 53 us,
// 5.2 TB/s), fp32 by latency with 4 waves a SIMD (1,011 tokens of 16 heads of 64 on 4, 24 blocks of 16: 44 us; keys asked for a step ahead cost
// registers, hence waves: 52; rows shared through LDS as below: 48).
//
// Entries that a query does not see have weight 0, and values there may be anything: addresses stop at the last entry that a token of the
// tile sees, and where a sum comes out as no number or infinite, the sweep is done again token by token with the values that the token
// does not see as 0.
#include <math.h>

#include <type_traits>

#include "kv4.h"
#include "lds_rows.h"
#include "token_tiles.h"

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;

struct Params {
  const void* __restrict__ q;
  const void* __restrict__ k;
  const void* __restrict__ v;
  const int32_t* __restrict__ cu_q;
  const int32_t* __restrict__ q_pos;
  const int32_t* __restrict__ kv_len;
  const int32_t* __restrict__ block_table;
  const int32_t* __restrict__ selected;  // [n_q][n_kv_heads][n_select]
  void* __restrict__ out;
  float* __restrict__ lse;
  float* __restrict__ ws_ml;             // [tile][kv head][piece][16][2]: reference exponent, sum
  float* __restrict__ ws_o;              // [tile][kv head][piece][16][D]: sums, not divided
  int64_t n_q, stride_slot, stride_head;
  int32_t max_blocks, n_streams, n_q_heads, n_kv_heads, group, tile, n_select, cache_blocks, pieces;
  float scale_log2e, scale_rest;         // scale log2(e), and what its rounding left
};

constexpr int kRows = 16;
constexpr int kMostListed = 256;         // list elements of a tile
constexpr float kSlack = 8.0f;           // log2 of how far weights may exceed the reference maximum's
constexpr float kFar = 1e18f;            // a score, and a factor, past which the factor's rounding is left alone: products stay finite
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const cs::f32v2 v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, cs::bf16v2));
}

__device__ __forceinline__ void store4(void* out, int64_t at, const float* x, bool bf16) {
  if (bf16)
    *reinterpret_cast<cs::u32x2*>(static_cast<uint16_t*>(out) + at) = cs::u32x2{pack2(x[0], x[1]), pack2(x[2], x[3])};
  else
    *reinterpret_cast<cs::u32x4*>(static_cast<float*>(out) + at) =
        cs::u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
}

__device__ __forceinline__ float log_sum(float m, float l) { return l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2; }

// ---- where the 16 keys of a group lie
struct Group {
  int first;                             // first entry
  int mask;                              // tokens that read it (0: past the list)
  int64_t at;                            // element offset of row 0 of its cache block, kv head included
  int top;                               // rows from here on are row `top`: past the last entry that is seen
};

// Sixteen rows' sums, and what a lane's row has seen: o holds channels as the kind of cache has them.
template <int D>
struct Sums {
  f32x4 o[D / 16];
  float m, l;                            // reference exponent, sum of weights 2^(exponent - m)
};

// ---- bf16: 16 * GROUPS keys a step
template <int D, int GROUPS = 4>
struct Bf16 {
  static constexpr bool kBf16 = true;
  static constexpr int KB = GROUPS;      // groups a step
  static constexpr int VROW = D + 16;    // of LDS: the transposing reads of 16 rows spread over the banks
  static constexpr int kLds = KB * 16 * VROW * 2;      // bytes a wave
  bf16x8 query[D / 32];

  __device__ __forceinline__ void load_query(const void* q, int64_t row, int g) {
#pragma unroll
    for (int s = 0; s < D / 32; ++s) query[s] = *reinterpret_cast<const bf16x8*>(static_cast<const uint16_t*>(q) + row + 32 * s + 8 * g);
  }

  struct Tile {
    bf16x8 k[KB][D / 32];
    cs::u32x4 v[KB][D / 32];
  };

  __device__ __forceinline__ void load(const Params& p, const Group (&gr)[KB], Tile& t, int lane) const {
    const int r16 = lane & 15, g = lane >> 4;
    constexpr int LR = D / 8;            // lanes of a row of values
    constexpr int RL = 64 / LR;
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      const uint16_t* k = static_cast<const uint16_t*>(p.k) + gr[b].at + static_cast<int64_t>(min(r16, gr[b].top)) * p.stride_slot + 8 * g;
#pragma unroll
      for (int s = 0; s < D / 32; ++s) t.k[b][s] = *reinterpret_cast<const bf16x8*>(k + 32 * s);
    }
#pragma unroll
    for (int b = 0; b < KB; ++b) {
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        const int r = i * RL + lane / LR;
        t.v[b][i] = *reinterpret_cast<const cs::u32x4*>(static_cast<const uint16_t*>(p.v) + gr[b].at +
                                                        static_cast<int64_t>(min(r, gr[b].top)) * p.stride_slot + lane % LR * 8);
      }
    }
  }

  __device__ __forceinline__ void scores(const Tile& t, f32x4 (&s)[KB]) const {
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      s[b] = f32x4{};
#pragma unroll
      for (int i = 0; i < D / 32; ++i) s[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(t.k[b][i], query[i], s[b], 0, 0, 0);
    }
  }

  // only: the token whose unseen values are taken as 0 (limit[b]: its last entry in group b), or nobody's
  __device__ __forceinline__ void add(const Tile& t, const Group (&gr)[KB], const f32x4 (&w)[KB], Sums<D>& sums, uint8_t* lds, int lane, bool careful,
                                      const int (&limit)[KB]) const {
    constexpr int LR = D / 8, RL = 64 / LR;
    const int r16 = lane & 15, g = lane >> 4;
    uint16_t* v = reinterpret_cast<uint16_t*>(lds);
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        const int r = i * RL + lane / LR;
        cs::u32x4 x = t.v[b][i];
        if (careful && gr[b].first + r > limit[b]) x = cs::u32x4{0, 0, 0, 0};
        *reinterpret_cast<cs::u32x4*>(v + (16 * b + r) * VROW + lane % LR * 8) = x;
      }
    // Of the 32 keys of a product a lane's weights are of 4 g + 0..3 of two groups; the transposing read gives 16 lanes four rows of
    // 16 elements.
    const uint16_t* at = v + (4 * g + (r16 >> 2)) * VROW + 4 * (r16 & 3);
#pragma unroll
    for (int st = 0; st < KB / 2; ++st) {
      const cs::u32x4 pw = {pack2(w[2 * st][0], w[2 * st][1]), pack2(w[2 * st][2], w[2 * st][3]), pack2(w[2 * st + 1][0], w[2 * st + 1][1]),
                            pack2(w[2 * st + 1][2], w[2 * st + 1][3])};
      const bf16x8 pf = __builtin_bit_cast(bf16x8, pw);
#pragma unroll
      for (int db = 0; db < D / 16; ++db) {
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 32 * st * VROW + 16 * db));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + (32 * st + 16) * VROW + 16 * db));
        const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        sums.o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf, sums.o[db], 0, 0, 0);
      }
    }
  }

  // Channels of o[i][0..3]: 16 i + 4 g + 0..3.
  template <class F>
  static __device__ __forceinline__ void each4(const Sums<D>& s, int g, const F& f) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      const float x[4] = {s.o[i][0], s.o[i][1], s.o[i][2], s.o[i][3]};
      f(16 * i + 4 * g, x);
    }
  }
};

// ---- fp32: 32 keys a step
template <int D>
struct F32 {
  static constexpr bool kBf16 = false;
  static constexpr int KB = 2;
  static constexpr int kLds = 0;
  f32x4 query[D / 16];

  __device__ __forceinline__ void load_query(const void* q, int64_t row, int g) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) query[s] = *reinterpret_cast<const f32x4*>(static_cast<const float*>(q) + row + 16 * s + 4 * g);
  }

  struct Tile {
    f32x4 k[KB][D / 16];
    f32x4 v[KB][4][D / 64];
  };

  __device__ __forceinline__ void load(const Params& p, const Group (&gr)[KB], Tile& t, int lane) const {
    const int r16 = lane & 15, g = lane >> 4;
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      const float* k = static_cast<const float*>(p.k) + gr[b].at + static_cast<int64_t>(min(r16, gr[b].top)) * p.stride_slot + 4 * g;
#pragma unroll
      for (int s = 0; s < D / 16; ++s) t.k[b][s] = *reinterpret_cast<const f32x4*>(k + 16 * s);
    }
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float* v = static_cast<const float*>(p.v) + gr[b].at + static_cast<int64_t>(min(4 * g + r, gr[b].top)) * p.stride_slot + 4 * r16;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) t.v[b][r][j] = *reinterpret_cast<const f32x4*>(v + 64 * j);
      }
  }

  // The sum over channels may run in any order: element e of the lanes' vectors is one step of it, and a sum of its own, since four short
  // sums round less than a long one.
  __device__ __forceinline__ void scores(const Tile& t, f32x4 (&s)[KB]) const {
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      f32x4 part[4] = {};
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) part[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(t.k[b][i][e], query[i][e], part[e], 0, 0, 0);
      s[b] = (part[0] + part[1]) + (part[2] + part[3]);
    }
  }

  __device__ __forceinline__ void add(const Tile& t, const Group (&gr)[KB], const f32x4 (&w)[KB], Sums<D>& sums, uint8_t*, int lane, bool careful,
                                      const int (&limit)[KB]) const {
    const int g = lane >> 4;
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const bool none = careful && gr[b].first + 4 * g + r > limit[b];
#pragma unroll
        for (int j = 0; j < D / 64; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            sums.o[4 * j + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(none ? 0.0f : t.v[b][r][j][e], w[b][r], sums.o[4 * j + e], 0, 0, 0);
      }
  }

  // Channels of o[4 j + 0..3][r]: 64 j + 16 g + 4 r + 0..3.
  template <class F>
  static __device__ __forceinline__ void each4(const Sums<D>& s, int g, const F& f) {
#pragma unroll
    for (int j = 0; j < D / 64; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float x[4] = {s.o[4 * j][r], s.o[4 * j + 1][r], s.o[4 * j + 2][r], s.o[4 * j + 3][r]};
        f(64 * j + 16 * g + 4 * r, x);
      }
  }
};

// ---- one pass of a wave over groups of keys
// 16 rows' sums over groups g0, g0 + KB .. of every `stride` from `begin` on; locate(g0, gr) says where they lie.  A lane's row belongs to the token of
// mask bit `bit` and sees up to entry `pos`.  careful: values past only_pos, or in blocks that the token of mask bit `only` does not read, are
// taken as 0 (the sums of other tokens' rows are then worth nothing).
template <class Kind, int D, class Locate>
__device__ __forceinline__ void sweep(const Params& p, const Kind& kind, const Locate& locate, int begin, int stride, int n_groups, int bit, int pos, bool careful,
                                      int only, int only_pos, uint8_t* lds, int lane, Sums<D>& sums) {
  constexpr int KB = Kind::KB;
  const int g = lane >> 4;
  const float c = p.scale_log2e;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) sums.o[i] = f32x4{};
  sums.m = -INFINITY;
  sums.l = 0.0f;
  for (int g0 = begin; g0 < n_groups; g0 += stride) {
    Group gr[KB];
    locate(g0, gr);
    typename Kind::Tile tl;
    kind.load(p, gr, tl, lane);
    f32x4 s[KB];
    kind.scores(tl, s);
    float high = -INFINITY;
    int limit[KB];
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      limit[b] = gr[b].mask >> only & 1 ? only_pos : -1;
      const int lim = (gr[b].mask >> bit & 1) && (!careful || bit == only) ? pos : -1;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (gr[b].first + 4 * g + r > lim) s[b][r] = -INFINITY;
        high = fmaxf(high, s[b][r]);
      }
    }
    // (the row's lanes hold different keys; they share a maximum, and look at each other's only to raise it.  -inf - -inf: no)
    if (__any(fmaf(high, c, -sums.m) > kSlack)) {
      high = cs::with_lane32(cs::with_lane16(high, cs::larger), cs::larger);
      const float raised = fmaxf(sums.m, high * c);
      const float f = sums.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sums.m - raised);
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) sums.o[i][r] *= f;
      sums.l *= f;
      sums.m = raised;
    }
    const float base = sums.m == -INFINITY ? 0.0f : -sums.m;
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float e = fmaf(s[b][r], c, base);
        // (fp32: with the rounded factor alone a score of 20 would be off by 1e-6; what is infinite stays so)
        if constexpr (!Kind::kBf16) e = fmaf(__builtin_amdgcn_fmed3f(s[b][r], -kFar, kFar), p.scale_rest, e);
        s[b][r] = __builtin_amdgcn_exp2f(e);
        sums.l += s[b][r];
      }
    kind.add(tl, gr, s, sums, lds, lane, careful, limit);
  }
}

constexpr int kJoinBatch = 8;
// What is joined: results of R rows, `ml` [way][R][2] and `o` [way][R][D].  A thread takes four channels of a row, kJoinBatch ways at a time.
template <int D, int R>
__device__ __forceinline__ void join_rows(const float* ml, const float* o, int ways, int row, int ch, float* m_out, float* l_out, float (&x)[4]) {
  float m = -INFINITY, l = 0.0f;
  x[0] = x[1] = x[2] = x[3] = 0.0f;
  for (int w0 = 0; w0 < ways; w0 += kJoinBatch) {
    cs::f32v2 stat[kJoinBatch];
    f32x4 v[kJoinBatch];
#pragma unroll
    for (int i = 0; i < kJoinBatch; ++i) {
      const int w = min(w0 + i, ways - 1);
      stat[i] = *reinterpret_cast<const cs::f32v2*>(ml + (w * R + row) * 2);
      v[i] = *reinterpret_cast<const f32x4*>(o + (w * R + row) * D + ch);
    }
    float high = m;
#pragma unroll
    for (int i = 0; i < kJoinBatch; ++i) high = fmaxf(high, stat[i].x);
    const float back = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - high);      // (without a maximum there are only zeros, or what is no number)
    l *= back;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] *= back;
    m = high;
#pragma unroll
    for (int i = 0; i < kJoinBatch; ++i) {
      if (w0 + i >= ways) break;
      const float f = stat[i].x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(stat[i].x - m);
      l = fmaf(stat[i].y, f, l);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = fmaf(v[i][e], f, x[e]);
    }
  }
  *m_out = m;
  *l_out = l;
}

template <int D>
__device__ __forceinline__ void write_row(const Params& p, int tok, int head, int ch, float m, float l, float (&x)[4], bool bf16) {
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] *= inv;
  store4(p.out, (static_cast<int64_t>(tok) * p.n_q_heads + head) * D + ch, x, bf16);
  if (ch == 0 && p.lse) p.lse[static_cast<int64_t>(tok) * p.n_q_heads + head] = log_sum(m, l);
}

// (fp32, head_dim 64: 128 registers, four waves a SIMD; without the bound 139 and 51 us where it takes 44)
template <class Kind, int D, int NW>
__global__ __launch_bounds__(64 * NW, !Kind::kBf16 && D == 64 ? 4 : 1) void selected_attn_kernel(Params p) {
  constexpr int KB = Kind::KB;
  constexpr int kJoin = NW > 1 ? NW * kRows * (D + 2) * 4 : 16;          // results of the waves, where values were
  constexpr int kBytes = NW * Kind::kLds > kJoin ? NW * Kind::kLds : kJoin;
  __shared__ __attribute__((aligned(16))) uint8_t s_mem[kBytes];
  __shared__ __attribute__((aligned(16))) int s_key[kMostListed], s_sorted[kMostListed], s_tok[kMostListed], s_list[kMostListed], s_mask[kMostListed];
  __shared__ int s_count;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, g = lane >> 4;
  const int kvh = static_cast<int>(blockIdx.x % p.n_kv_heads);
  const int job = static_cast<int>(blockIdx.x / p.n_kv_heads), piece = job % p.pieces, tile = job / p.pieces;
  cs::TokenTile t;
  if (!cs::find_token_tile(p.cu_q, p.n_streams, p.n_q, p.tile, tile, &t)) return;
  const int size = p.cache_blocks * CS_KV_BLOCK;
  const int n_keys = t.count * p.n_select;
  const auto listed = [&](int i) __attribute__((always_inline)) {
    return i < n_keys ? p.selected[(static_cast<int64_t>(t.first + i / p.n_select) * p.n_kv_heads + kvh) * p.n_select + i % p.n_select] : -1;
  };
  const int mine = listed(lane);         // (asked for with the length and the position)
  const int entries = min(p.kv_len[t.stream], p.max_blocks * CS_KV_BLOCK);
  const int first_pos = p.q_pos[t.first];
  if (entries <= 0) return;              // (such a stream's rows are left as they were)

  // ---- the tile's lists as one
  int n_blocks;
  const auto usable = [&](int block, int pos) __attribute__((always_inline)) {
    const int last = min(pos, entries - 1);
    return block >= 0 && last >= 0 && block <= last / size ? block : 0x7fffffff;
  };
  const int key0 = usable(mine, first_pos);
  const int before0 = __builtin_amdgcn_update_dpp(-1, key0, 0x138, 0xf, 0xf, false);      // of the lane before (wave_shr:1)
  if (t.count == 1 && n_keys <= 64 && __all(key0 > before0 || key0 == 0x7fffffff)) {
    // One token whose list ascends, as a selection leaves it: every wave writes it for itself (what the others write is the same).
    s_list[lane] = key0;
    s_mask[lane] = 1;
    n_blocks = __popcll(__ballot(key0 != 0x7fffffff));
  } else {
    for (int i = tid; i < kMostListed; i += 64 * NW) s_key[i] = i < n_keys ? usable(listed(i), p.q_pos[t.first + i / p.n_select]) : 0x7fffffff;
    __syncthreads();
    const int padded = (n_keys + 3) & ~3;
    for (int i = tid; i < padded; i += 64 * NW) {
      const int key = s_key[i];
      int rank = 0;
      for (int j = 0; j < padded; j += 4) {
        const cs::u32x4 other = *reinterpret_cast<const cs::u32x4*>(s_key + j);
  #pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int o = static_cast<int>(other[e]);
          rank += o < key || (o == key && j + e < i) ? 1 : 0;
        }
      }
      s_sorted[rank] = key;
      s_tok[rank] = i / p.n_select;
    }
    __syncthreads();
    if (wave == 0) {
      int base = 0;
      for (int i0 = 0; i0 < padded; i0 += 64) {
        const int i = i0 + lane;
        const int key = i < padded ? s_sorted[i] : 0x7fffffff;
        const bool first = key != 0x7fffffff && (i == 0 || s_sorted[i - 1] != key);
        const uint64_t all = __ballot(first);
        if (first) {
          int mask = 0;
          for (int j = i; j < padded && s_sorted[j] == key; ++j) mask |= 1 << s_tok[j];
          const int at = base + __popcll(all & ((1ull << lane) - 1));
          s_list[at] = key;
          s_mask[at] = mask;
        }
        base += __popcll(all);
      }
      if (lane == 0) s_count = base;
    }
    __syncthreads();
    n_blocks = __builtin_amdgcn_readfirstlane(s_count);
  }
  const int n_groups = n_blocks * p.cache_blocks;

  // ---- the lane's row
  const int tau = r16 / p.group;
  const bool live = tau < t.count && r16 < p.tile * p.group;
  const int tok = t.first + (live ? tau : 0), head = kvh * p.group + (live ? r16 % p.group : 0);
  const int pos = live ? min(p.q_pos[tok], entries - 1) : -1;
  const int top = __builtin_amdgcn_readfirstlane(static_cast<int>(cs::lanes_max<64>(static_cast<uint32_t>(max(pos, 0)))));      // last entry that anyone sees
  Kind kind;
  kind.load_query(p.q, (static_cast<int64_t>(tok) * p.n_q_heads + head) * D, g);
  const int32_t* ids = p.block_table + static_cast<int64_t>(t.stream) * p.max_blocks;
  const int64_t head_at = static_cast<int64_t>(kvh) * p.stride_head;
  uint8_t* lds = s_mem + wave * Kind::kLds;

  const auto locate = [&](int first_group, Group (&gr)[KB]) __attribute__((always_inline)) {
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      const bool there = first_group + b < n_groups;
      const int gi = there ? first_group + b : first_group;
      const int u = gi / p.cache_blocks;
      gr[b].first = (__builtin_amdgcn_readfirstlane(s_list[u]) * p.cache_blocks + (gi - u * p.cache_blocks)) * CS_KV_BLOCK;
      gr[b].mask = there ? __builtin_amdgcn_readfirstlane(s_mask[u]) : 0;
      const int cb = min(gr[b].first, top) / CS_KV_BLOCK;
      gr[b].at = static_cast<int64_t>(ids[cb]) * CS_KV_BLOCK * p.stride_slot + head_at;
      gr[b].top = min(CS_KV_BLOCK - 1, top - cb * CS_KV_BLOCK);
    }
  };

  Sums<D> sums;
  const int begin = (piece * NW + wave) * KB, stride = p.pieces * NW * KB;
  sweep<Kind, D>(p, kind, locate, begin, stride, n_groups, tau, pos, false, 0, 0, lds, lane, sums);
  bool odd = false;
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) odd |= (__float_as_uint(sums.o[i][r]) & 0x7f800000u) == 0x7f800000u;
  if (__builtin_expect(__any(odd), 0)) {
    Sums<D> kept = sums;
    for (int only = 0; only < t.count; ++only) {
      sweep<Kind, D>(p, kind, locate, begin, stride, n_groups, tau, pos, true, only, min(p.q_pos[t.first + only], entries - 1), lds, lane, sums);
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) kept.o[i][r] = tau == only ? sums.o[i][r] : kept.o[i][r];
      kept.m = tau == only ? sums.m : kept.m;
      kept.l = tau == only ? sums.l : kept.l;
    }
    sums = kept;
  }
  sums.l = cs::with_lane32(cs::with_lane16(sums.l, cs::plus), cs::plus);

  // ---- results
  const int64_t at_job = (static_cast<int64_t>(tile) * p.n_kv_heads + kvh) * p.pieces + piece;
  if constexpr (NW == 1) {
    if (p.pieces == 1) {
      if (live) {
        Kind::each4(sums, g, [&](int ch, const float (&x)[4]) __attribute__((always_inline)) {
          float y[4] = {x[0], x[1], x[2], x[3]};
          write_row<D>(p, tok, head, ch, sums.m, sums.l, y, Kind::kBf16);
        });
      }
    } else {
      if (g == 0) *reinterpret_cast<cs::f32v2*>(p.ws_ml + (at_job * kRows + r16) * 2) = cs::f32v2{sums.m, sums.l};
      Kind::each4(sums, g, [&](int ch, const float (&x)[4]) __attribute__((always_inline)) {
        *reinterpret_cast<f32x4*>(p.ws_o + (at_job * kRows + r16) * D + ch) = f32x4{x[0], x[1], x[2], x[3]};
      });
    }
  } else {
    __syncthreads();                     // (values of other waves are no longer read)
    float* s_o = reinterpret_cast<float*>(s_mem);
    float* s_ml = s_o + NW * kRows * D;
    if (g == 0) *reinterpret_cast<cs::f32v2*>(s_ml + (wave * kRows + r16) * 2) = cs::f32v2{sums.m, sums.l};
    Kind::each4(sums, g, [&](int ch, const float (&x)[4]) __attribute__((always_inline)) {
      *reinterpret_cast<f32x4*>(s_o + (wave * kRows + r16) * D + ch) = f32x4{x[0], x[1], x[2], x[3]};
    });
    __syncthreads();
    for (int i = tid; i < kRows * (D / 4); i += 64 * NW) {
      const int row = i / (D / 4), ch = i % (D / 4) * 4;
      if (row >= t.count * p.group) continue;
      float m, l, x[4];
      join_rows<D, kRows>(s_ml, s_o, NW, row, ch, &m, &l, x);
      if (p.pieces == 1) {
        write_row<D>(p, t.first + row / p.group, kvh * p.group + row % p.group, ch, m, l, x, Kind::kBf16);
      } else {
        if (ch == 0) *reinterpret_cast<cs::f32v2*>(p.ws_ml + (at_job * kRows + row) * 2) = cs::f32v2{m, l};
        *reinterpret_cast<f32x4*>(p.ws_o + (at_job * kRows + row) * D + ch) = f32x4{x[0], x[1], x[2], x[3]};
      }
    }
  }
}

// The pieces of a tile and kv head, joined: R rows a tile, four channels of one a thread.
template <int D, int R>
__global__ __launch_bounds__(256) void selected_join_kernel(Params p, int bf16) {
  const int kvh = static_cast<int>(blockIdx.x % p.n_kv_heads), tile = static_cast<int>(blockIdx.x / p.n_kv_heads);
  cs::TokenTile t;
  if (!cs::find_token_tile(p.cu_q, p.n_streams, p.n_q, p.tile, tile, &t)) return;
  if (min(p.kv_len[t.stream], p.max_blocks * CS_KV_BLOCK) <= 0) return;
  const int64_t at_job = (static_cast<int64_t>(tile) * p.n_kv_heads + kvh) * p.pieces;
  const int i = blockIdx.y * 256 + threadIdx.x, row = i / (D / 4), ch = i % (D / 4) * 4;
  if (row >= t.count * p.group) return;
  float m, l, x[4];
  join_rows<D, R>(p.ws_ml + at_job * R * 2, p.ws_o + at_job * R * D, p.pieces, row, ch, &m, &l, x);
  write_row<D>(p, t.first + row / p.group, kvh * p.group + row % p.group, ch, m, l, x, bf16 != 0);
}

// ------------------------------------------------------------------------------------------
// Many tokens a stream, bf16.  Neighbouring tokens read much the same blocks, so a workgroup takes as many as its four waves hold, 16
// rows each (a token's heads may lie in two waves), and moves every block that any of them reads through LDS once, 32 keys a step.  A wave
// skips the steps that none of its tokens reads.
//   S^T = K Q^T, O^T += V^T P^T      v_mfma_f32_16x16x32_bf16; a lane owns one row and 4 of 16 keys
// Rows go from memory to LDS directly (global_load_lds_dwordx4: lane l lands at base + 16 l), a step ahead, in two stages, one barrier a
// step.  Lanes choose which 16-byte chunk of a row they fetch, so that reads spread over the banks: row r of keys holds chunk c at place
// c ^ row_place(r), of values at c ^ v_place(r).
// Bound by the length of a step's chain (gate, scores, softmax, sums) with the four waves a SIMD that registers and LDS allow: 2,082 tokens of 28
// heads of 128 on 4 over 16 blocks of 64 each take 90 us; matrix instructions are busy for 20 of them, vector instructions for 32, and LDS
// reads for 21; what the workgroups move from L2, 1.32 GB, takes 34 at 64 bytes a clock and CU.  Deeper or wider did worse, since it costs waves (when this kernel took 112 to 116): three stages 152, a wave's scores a step
// ahead of its sums 171, 64 keys a step 126, 32 rows a wave 130.
constexpr int kStepKeys = 32, kStepGroups = kStepKeys / CS_KV_BLOCK;
constexpr int kRowsWave = kRows, kRowsWaves = 4, kRowsGroup = kRowsWave * kRowsWaves;
constexpr int kRowsListed = 512;         // list elements of a workgroup's tokens
constexpr int kChunk = 1024;             // blocks whose readers are collected at once
constexpr int kStages = 2;
constexpr int kPlaces = 64;              // groups whose places are looked up at once, a lane each

// Tokens of a workgroup: as many as fit, and as masks of 32 bits hold.
inline int rows_tokens(int group) { return kRowsGroup / group < 32 ? kRowsGroup / group : 32; }

template <int D>
__device__ __forceinline__ int v_place(int r) { return D == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3); }

// kPaired: the groups of a step are of one listed block (those of an even number of cache blocks).  Five workgroups a CU at head_dim 64 (32
// streams of up to 389 tokens: four 86 us, five 81).
template <int D, bool kPaired>
__global__ __launch_bounds__(64 * kRowsWaves, D == 64 ? 5 : 4) void selected_rows_kernel(Params p) {
  constexpr int DB = D / 16, STEPS = D / 32;
  constexpr int kTensor = kStepKeys * D * 2;               // bytes of a step's keys, or values
  constexpr int kStage = 2 * kTensor;
  constexpr int kParts = kTensor / 1024;                   // requests for a step's keys, and as many for its values
  constexpr int kAsks = kParts / kRowsWaves;               // ... of a wave
  static_assert(kRowsWaves == 2 * kStepGroups && kAsks >= 1, "a wave asks for half a group");
  typedef Bf16<D, 2> Again;
  constexpr int kBytes = kStages * kStage;
  constexpr int kAgainWaves = kBytes / Again::kLds < kRowsWaves ? kBytes / Again::kLds : kRowsWaves;
  static_assert(kBytes >= kChunk * 4, "readers are collected where tiles are later");
  __shared__ __attribute__((aligned(16))) uint8_t s_mem[kBytes];
  __shared__ int s_list[kRowsListed];
  __shared__ uint32_t s_mask[kRowsListed];
  __shared__ int s_odd;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, g = lane >> 4;
  const int kvh = static_cast<int>(blockIdx.x % p.n_kv_heads);
  const int job = static_cast<int>(blockIdx.x / p.n_kv_heads), piece = job % p.pieces, tile = job / p.pieces;
  cs::TokenTile t;
  if (!cs::find_token_tile(p.cu_q, p.n_streams, p.n_q, p.tile, tile, &t)) return;
  const int entries = min(p.kv_len[t.stream], p.max_blocks * CS_KV_BLOCK);
  if (entries <= 0) return;
  const int size = p.cache_blocks * CS_KV_BLOCK;

  // ---- the blocks that the tokens read, ascending, each with the mask of its readers
  constexpr int kHeld = (kRowsListed + 64 * kRowsWaves - 1) / (64 * kRowsWaves);
  const int n_keys = t.count * p.n_select;
  int held[kHeld];
  int top = 0;                           // last entry that anyone sees
  for (int i = lane; i < t.count; i += 64) top = max(top, min(p.q_pos[t.first + i], entries - 1));
  top = __builtin_amdgcn_readfirstlane(static_cast<int>(cs::lanes_max<64>(static_cast<uint32_t>(top))));
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int at = i * 64 * kRowsWaves + tid;
    held[i] = -1;
    if (at < n_keys) {
      const int tok = t.first + at / p.n_select;
      const int last = min(p.q_pos[tok], entries - 1);
      const int block = p.selected[(static_cast<int64_t>(tok) * p.n_kv_heads + kvh) * p.n_select + at % p.n_select];
      if (block >= 0 && last >= 0 && block <= last / size) held[i] = block;
    }
  }
  uint32_t* readers = reinterpret_cast<uint32_t*>(s_mem);
  const int candidates = top / size + 1;
  int count = 0;
  for (int c0 = 0; c0 < candidates; c0 += kChunk) {
    for (int i = tid; i < kChunk; i += 64 * kRowsWaves) readers[i] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (held[i] >= c0 && held[i] < c0 + kChunk) atomicOr(&readers[held[i] - c0], 1u << ((i * 64 * kRowsWaves + tid) / p.n_select));
    __syncthreads();
    const int here = min(kChunk, candidates - c0);
    for (int i0 = 0; i0 < here; i0 += 64) {                // (every wave counts, the first one writes)
      const uint32_t mask = i0 + lane < here ? readers[i0 + lane] : 0;
      const uint64_t all = __ballot(mask != 0);
      if (wave == 0 && mask) {
        const int at = count + __popcll(all & ((1ull << lane) - 1));
        s_list[at] = c0 + i0 + lane;
        s_mask[at] = mask;
      }
      count += __popcll(all);
    }
    __syncthreads();
  }
  // this piece's groups, whole steps
  const int all_groups = __builtin_amdgcn_readfirstlane(count) * p.cache_blocks;
  const int a_piece = ((all_groups + kStepGroups - 1) / kStepGroups + p.pieces - 1) / p.pieces * kStepGroups;
  const int begin = min(piece * a_piece, all_groups), n_groups = min(begin + a_piece, all_groups);

  // ---- the lane's row
  const int in_group = wave * kRowsWave + r16, bit = in_group / p.group;      // bit: the token, of the workgroup's
  const bool live = bit < t.count;
  const uint32_t my_bit = live ? 1u << bit : 0;
  const int tok = t.first + (live ? bit : 0), head = kvh * p.group + (live ? in_group % p.group : 0);
  const int pos = live ? min(p.q_pos[tok], entries - 1) : -1;
  const int bits0 = wave * kRowsWave / p.group, bits1 = min((wave * kRowsWave + kRowsWave - 1) / p.group, t.count - 1);       // the wave's tokens
  const uint32_t wave_mask = bits1 < bits0 ? 0u : (~0u >> (31 - (bits1 - bits0))) << bits0;
  int least = live ? pos : 0x7fffffff;                     // how far all of them see
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) least = min(least, __shfl_xor(least, d));
  least = __builtin_amdgcn_readfirstlane(least);
  const int64_t at_q = (static_cast<int64_t>(tok) * p.n_q_heads + head) * D;
  bf16x8 query[STEPS];
#pragma unroll
  for (int s = 0; s < STEPS; ++s) query[s] = *reinterpret_cast<const bf16x8*>(static_cast<const uint16_t*>(p.q) + at_q + 32 * s + 8 * g);

  const int32_t* ids = p.block_table + static_cast<int64_t>(t.stream) * p.max_blocks;
  const int64_t head_at = static_cast<int64_t>(kvh) * p.stride_head;
  const float c = p.scale_log2e;
  constexpr float kNone = 3.402823466e38f;                 // the constant without a maximum: any score is a reason to raise it, and -inf has weight 0

  // ---- this wave's part of a step's requests: half the rows of a group
  constexpr int LR = D / 8, RL = 64 / LR;                  // lanes of a row, rows of a request
  const uint32_t mem = __builtin_amdgcn_readfirstlane(cs::lds_address(s_mem));
  const uint32_t row_bytes = static_cast<uint32_t>(p.stride_slot * 2);
  const auto row_of = [&](int j) __attribute__((always_inline)) { return 8 * (wave & 1) + j * RL + lane / LR; };
  const auto k_part = [&](int j) __attribute__((always_inline)) { return 16u * (lane % LR ^ cs::row_place<D>(row_of(j))); };
  const auto v_part = [&](int j) __attribute__((always_inline)) { return 16u * (lane % LR ^ v_place<D>(row_of(j))); };
  uint32_t k_off[kAsks], v_off[kAsks];
#pragma unroll
  for (int j = 0; j < kAsks; ++j) {
    k_off[j] = row_of(j) * row_bytes + k_part(j);
    v_off[j] = row_of(j) * row_bytes + v_part(j);
  }
  // A lane's group, of those whose places are at hand: first entry, readers, last row, offset in bytes of its cache block.
  int at_first = 0, at_last = 0;
  uint32_t at_mask = 0, at_low = 0, at_high = 0;
  const auto request = [&](int i, int stage) __attribute__((always_inline)) {
    const int from = kStepGroups * i + (wave >> 1);
    const uint64_t off64 = static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(at_high), from))) << 32 |
                           static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(at_low), from));
    const int last = __builtin_amdgcn_readlane(at_last, from);
    const char* k = static_cast<const char*>(p.k) + off64;
    const char* v = static_cast<const char*>(p.v) + off64;
    const uint32_t to = mem + stage * kStage + wave * (1024 * kAsks);
    if (last == CS_KV_BLOCK - 1) {
#pragma unroll
      for (int j = 0; j < kAsks; ++j) {
        cs::to_lds(k_off[j], k, to + 1024 * j);
        cs::to_lds(v_off[j], v, to + kTensor + 1024 * j);
      }
    } else {                             // (rows past the last entry that anyone sees are that one)
#pragma unroll
      for (int j = 0; j < kAsks; ++j) {
        const uint32_t off = min(row_of(j), last) * row_bytes;
        cs::to_lds(off + k_part(j), k, to + 1024 * j);
        cs::to_lds(off + v_part(j), v, to + kTensor + 1024 * j);
      }
    }
  };

  Sums<D> sums;
#pragma unroll
  for (int db = 0; db < DB; ++db) sums.o[db] = f32x4{};
  sums.m = -INFINITY;
  float base = kNone;                    // the exponents' constant: - m
  float total[4] = {};                   // sums of weights
  // the lane's places in the first stage
  const int v_row = 4 * g + (r16 >> 2);
  uint32_t k_at[STEPS], v_at[DB];        // (LDS addresses, kept from being worked out again at every use)
#pragma unroll
  for (int j = 0; j < STEPS; ++j) {
    k_at[j] = mem + r16 * D * 2 + 16 * ((4 * j + g) ^ cs::row_place<D>(r16));
    asm("" : "+v"(k_at[j]));
  }
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    v_at[db] = mem + kTensor + v_row * D * 2 + 16 * ((r16 >> 1) & 1) + 8 * (r16 & 1) + 16 * ((2 * db) ^ v_place<D>(v_row));
    asm("" : "+v"(v_at[db]));
  }
  const auto compute = [&](int i, auto which) __attribute__((always_inline)) {
    constexpr int kHere = decltype(which)::value * kStage;
    int first[kStepGroups];
    bool reads[kStepGroups];
#pragma unroll
    for (int b = 0; b < kStepGroups; ++b) {
      first[b] = kPaired && b ? first[0] + CS_KV_BLOCK : __builtin_amdgcn_readlane(at_first, kStepGroups * i + b);
      reads[b] = kPaired && b ? reads[0] : (static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(at_mask), kStepGroups * i + b)) & my_bit) != 0;
    }
    __builtin_amdgcn_s_setprio(1);       // (before waves that wait or ask: 98 -> 94 us)
    f32x4 s[kStepGroups] = {};
#pragma unroll
    for (int j = 0; j < STEPS; ++j)
#pragma unroll
      for (int b = 0; b < kStepGroups; ++b)
        s[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*((lds_bf16x8*)static_cast<uintptr_t>(k_at[j]) + (kHere + b * 16 * D * 2) / 16), query[j], s[b], 0, 0, 0);
    // A group that the lane's token does not read has the exponent -inf; only a group that ends behind one of the tokens is masked key
    // by key.
    if (max(first[0], first[1]) + CS_KV_BLOCK - 1 > least) {
#pragma unroll
      for (int b = 0; b < kStepGroups; ++b) {
        const int lim = pos - first[b] - 4 * g;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (r > lim) s[b][r] = -INFINITY;
      }
    }
    float high = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), s[0][2]), s[0][3]);
    if constexpr (kPaired) {
      high = fmaxf(fmaxf(fmaxf(high, s[1][0]), fmaxf(s[1][1], s[1][2])), s[1][3]);
      high = reads[0] ? high : -INFINITY;
    } else {
      const float other = fmaxf(fmaxf(fmaxf(s[1][0], s[1][1]), s[1][2]), s[1][3]);
      high = fmaxf(reads[0] ? high : -INFINITY, reads[1] ? other : -INFINITY);
    }
    if (__any(fmaf(high, c, base) > kSlack)) {             // (as above)
      high = cs::with_lane32(cs::with_lane16(high, cs::larger), cs::larger);
      const float raised = fmaxf(sums.m, high * c);
      const float f = sums.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sums.m - raised);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 4; ++r) sums.o[db][r] *= f;
#pragma unroll
      for (int r = 0; r < 4; ++r) total[r] *= f;
      sums.m = raised;
      base = fminf(-raised, kNone);
    }
    // of the 32 keys of a product a lane's weights are of 4 g + 0..3 of two groups; a row's place does not change 16 rows further
#pragma unroll
    for (int st = 0; st < kStepGroups / 2; ++st) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int b = 2 * st + e / 4;
        x[e] = __builtin_amdgcn_exp2f(fmaf(s[b][e % 4], c, reads[b] ? base : -INFINITY));
        total[e % 4] += x[e];
      }
      const bf16x8 pf = __builtin_bit_cast(bf16x8, cs::u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])});
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        lds_s16x4* at = (lds_s16x4*)static_cast<uintptr_t>(v_at[db]) + (kHere + 32 * st * D * 2) / 8;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at + 16 * D * 2 / 8);
        const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        sums.o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf, sums.o[db], 0, 0, 0);
      }
    }
    __builtin_amdgcn_s_setprio(0);
  };

  // ---- the steps, kPlaces groups at a time
  for (int g0 = begin; g0 < n_groups; g0 += kPlaces) {
    const int here = min(kPlaces, n_groups - g0), steps = (here + kStepGroups - 1) / kStepGroups;
    const int gi = g0 + min(lane, here - 1), u = gi / p.cache_blocks;
    at_first = (s_list[u] * p.cache_blocks + (gi - u * p.cache_blocks)) * CS_KV_BLOCK;
    at_mask = lane < here ? s_mask[u] : 0;
    const int cb = min(at_first, top) / CS_KV_BLOCK;
    const uint64_t off64 = static_cast<uint64_t>((static_cast<int64_t>(ids[cb]) * CS_KV_BLOCK * p.stride_slot + head_at) * 2);
    at_low = static_cast<uint32_t>(off64);
    at_high = static_cast<uint32_t>(off64 >> 32);
    at_last = min(CS_KV_BLOCK - 1, top - cb * CS_KV_BLOCK);
    // (bit i: whether a token of this wave reads something of step i)
    const uint64_t groups = __ballot((at_mask & wave_mask) != 0), active = groups | groups >> 1;
    __syncthreads();                     // (the stages are free)
    request(0, 0);
    const auto step = [&](int i, auto which) __attribute__((always_inline)) {
      cs::rows_gate();
      if (i + 1 < steps) request(i + 1, 1 - decltype(which)::value);       // (into the stage that everyone has read a step ago)
      if (active >> (kStepGroups * i) & 1) compute(i, which);
    };
    for (int i = 0; i < steps; i += 2) {
      step(i, std::integral_constant<int, 0>());
      if (i + 1 < steps) step(i + 1, std::integral_constant<int, 1>());
    }
  }
  sums.l = cs::with_lane32(cs::with_lane16((total[0] + total[1]) + (total[2] + total[3]), cs::plus), cs::plus);

  // ---- results; where something is no number or infinite, again token by token, the waves in turn
  const int64_t at_row = ((static_cast<int64_t>(tile) * p.n_kv_heads + kvh) * p.pieces + piece) * kRowsGroup;
  const auto leave = [&](int token, int row, int ch, const Sums<D>& of, float (&y)[4]) __attribute__((always_inline)) {
    if (p.pieces == 1) {
      write_row<D>(p, token, kvh * p.group + row % p.group, ch, of.m, of.l, y, true);
    } else {
      if (ch == 0) *reinterpret_cast<cs::f32v2*>(p.ws_ml + (at_row + row) * 2) = cs::f32v2{of.m, of.l};
      *reinterpret_cast<f32x4*>(p.ws_o + (at_row + row) * D + ch) = f32x4{y[0], y[1], y[2], y[3]};
    }
  };
  if (tid == 0) s_odd = 0;
  bool odd = false;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 4; ++r) odd |= (__float_as_uint(sums.o[db][r]) & 0x7f800000u) == 0x7f800000u;
  __syncthreads();
  if (__builtin_expect(__any(odd), 0)) s_odd = 1;
  __syncthreads();
  if (__builtin_expect(s_odd, 0)) {
    if (wave >= kAgainWaves) return;
    uint8_t* lds = s_mem + wave * Again::kLds;
    const auto locate = [&](int first_group, Group (&gr)[2]) __attribute__((always_inline)) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const bool there = first_group + b < n_groups;
        const int gi = there ? first_group + b : first_group, u = gi / p.cache_blocks;
        gr[b].first = (__builtin_amdgcn_readfirstlane(s_list[u]) * p.cache_blocks + (gi - u * p.cache_blocks)) * CS_KV_BLOCK;
        gr[b].mask = there ? __builtin_amdgcn_readfirstlane(static_cast<int>(s_mask[u])) : 0;
        const int cb = min(gr[b].first, top) / CS_KV_BLOCK;
        gr[b].at = static_cast<int64_t>(ids[cb]) * CS_KV_BLOCK * p.stride_slot + head_at;
        gr[b].top = min(CS_KV_BLOCK - 1, top - cb * CS_KV_BLOCK);
      }
    };
    for (int i = wave; i < t.count; i += kAgainWaves) {
      const int tok1 = t.first + i, pos1 = min(p.q_pos[tok1], entries - 1);
      const bool live1 = r16 < p.group;
      const int head1 = kvh * p.group + (live1 ? r16 : 0);
      Again kind;
      kind.load_query(p.q, (static_cast<int64_t>(tok1) * p.n_q_heads + head1) * D, g);
      Sums<D> one;
      sweep<Again, D>(p, kind, locate, begin, 2, n_groups, i, live1 ? pos1 : -1, true, i, pos1, lds, lane, one);
      one.l = cs::with_lane32(cs::with_lane16(one.l, cs::plus), cs::plus);
      if (live1) {
        Again::each4(one, g, [&](int ch, const float (&x)[4]) __attribute__((always_inline)) {
          float y[4] = {x[0], x[1], x[2], x[3]};
          leave(tok1, i * p.group + r16, ch, one, y);
        });
      }
    }
    return;
  }
  if (!live) return;
  Again::each4(sums, g, [&](int ch, const float (&x)[4]) __attribute__((always_inline)) {
    float y[4] = {x[0], x[1], x[2], x[3]};
    leave(tok, in_group, ch, sums, y);
  });
}

// ---- shapes: tokens of a tile, and pieces of a sweep
int tile_of(int32_t group, int32_t n_select) {
  const int by_rows = kRows / group, by_lists = kMostListed / n_select;
  return by_rows < by_lists ? by_rows : by_lists;
}

struct Shape {
  bool rows;                             // the kernel for many tokens a stream
  int tile, pieces, waves;
  int64_t tiles;
  size_t partials;                       // bytes of the pieces' results
};
// Pieces, so that few tokens fill the card too.  A token over 16 / 32 blocks of 64: one piece 20 us, at most 4 11.4 / 14.9, 8 10.7 / 12.3.
// 9 tokens over 16 blocks each, in the rows kernel: one piece 54 us, 8 17; 256 tokens 70 and 34; 1,024 tokens (two pieces) 80 and 75.
constexpr int kMostPieces = 8;
constexpr int kGroupsWanted = 512;       // workgroups wanted of the few-rows kernel
constexpr int kRowsWanted = 1024;        // ... of the rows kernel, as many as are on the card at once (512: 1,024 tokens 84 us; 2,048: 2,082 tokens 125)
constexpr int kRowsSteps = 4;            // steps of a piece of its sweep at least (2: the same)
// Tokens a stream, on average, from which bf16 takes the rows kernel.  Few rows / rows kernel: one token 10.6 / 11.6 us, two 15.4 / 13.5; 16
// streams of 2 tokens 22.3 / 18.9, of 8 30.6 / 25.5; 64 streams of 8 96 / 76.  (8 tokens of a stream over 8 blocks of 16 keys: 14.2 / 15.1.)
constexpr int kManyTokens = 2;
int most_pieces(int32_t sel_block, int32_t n_select, bool rows) {
  const int64_t entries = static_cast<int64_t>(n_select) * sel_block;
  const int64_t steps = rows ? entries / (kStepKeys * kRowsSteps) : (entries + 63) / 64;      // (rows: lists that are all alike)
  return static_cast<int>(steps < 1 ? 1 : steps < kMostPieces ? steps : kMostPieces);
}
int pieces_of(int64_t jobs, int most, bool rows) {
  const int64_t spare = (rows ? kRowsWanted : kGroupsWanted) / jobs;
  return static_cast<int>(spare < 1 ? 1 : spare < most ? spare : most);
}
int rows_tile_of(int32_t group, int32_t n_select) {
  const int all = rows_tokens(group), by_lists = kRowsListed / n_select;
  return all < by_lists ? all : by_lists;
}
size_t partials_of(int64_t jobs, int pieces, int32_t head_dim, bool rows) {
  return pieces == 1 ? 0 : static_cast<size_t>(jobs) * pieces * (rows ? kRowsGroup : kRows) * (head_dim + 2) * sizeof(float);
}

Shape shape_of(int64_t n_q, int32_t n_streams, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t sel_block, int32_t n_select, bool bf16,
               int64_t stride_slot) {
  Shape s;
  const int group = n_q_heads / n_kv_heads;
  s.rows = bf16 && n_q >= static_cast<int64_t>(kManyTokens) * n_streams && stride_slot < 1ll << 26;      // (offsets of a cache block in 32 bits)
  s.tile = s.rows ? rows_tile_of(group, n_select) : tile_of(group, n_select);
  s.tiles = cs::most_token_tiles(n_q, n_streams, s.tile);
  const int64_t jobs = s.tiles * n_kv_heads;
  s.pieces = pieces_of(jobs, most_pieces(sel_block, n_select, s.rows), s.rows);
  const int64_t each = ((static_cast<int64_t>(n_select) * sel_block + 63) / 64 + s.pieces - 1) / s.pieces;      // steps of a piece, few rows
  s.waves = each >= 4 ? 4 : each >= 2 ? 2 : 1;
  s.partials = partials_of(jobs, s.pieces, head_dim, s.rows);
  return s;
}

// Bytes that any call of up to n_q tokens and n_streams streams uses: fewer tokens are swept in more pieces, so this is the most over all
// numbers of tiles (they go up one by one with the tokens, and down with the streams).
size_t most_partials(int64_t n_q, int32_t n_streams, int32_t n_kv_heads, int32_t head_dim, int tile, int most, bool rows) {
  const int64_t tiles = cs::most_token_tiles(n_q, n_streams, tile), in_pieces = (rows ? kRowsWanted : kGroupsWanted) / (2 * static_cast<int64_t>(n_kv_heads));
  size_t bytes = 0;
  for (int64_t t = 1; t <= tiles && t <= in_pieces; ++t) {
    const size_t here = partials_of(t * n_kv_heads, pieces_of(t * n_kv_heads, most, rows), head_dim, rows);
    bytes = here > bytes ? here : bytes;
  }
  return bytes;
}

}  // namespace

extern "C" size_t cs_selected_attn_workspace(int64_t n_q, int32_t n_streams, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                             int32_t sel_block, int32_t n_select) {
  if (n_q < 1 || n_streams < 1 || n_kv_heads < 1 || n_q_heads < 1 || n_q_heads % n_kv_heads || n_q_heads / n_kv_heads > kRows) return 0;
  if (sel_block < 1 || n_select < 1 || n_select > CS_SELECT_MOST || head_dim < 1 || n_q >= 1ll << 26) return 0;
  // (either type's, and either kernel's)
  const int group = n_q_heads / n_kv_heads;
  const size_t few = most_partials(n_q, n_streams, n_kv_heads, head_dim, tile_of(group, n_select), most_pieces(sel_block, n_select, false), false);
  if (n_q < kManyTokens) return few;
  const size_t rows = most_partials(n_q, n_streams, n_kv_heads, head_dim, rows_tile_of(group, n_select), most_pieces(sel_block, n_select, true), true);
  return rows > few ? rows : few;
}

extern "C" int cs_selected_attn(const void* q, const void* k_cache_layer, const void* v_cache_layer, const int32_t* cu_q, const int32_t* q_pos,
                                const int32_t* kv_len, const int32_t* block_table, int32_t max_blocks, int32_t block_size,
                                const int32_t* selected, int32_t sel_block, int32_t n_select, void* out, float* lse, int64_t n_q,
                                int32_t n_streams, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t stride_slot,
                                int64_t stride_head, float softmax_scale, int32_t dtype, void* workspace, size_t workspace_bytes,
                                void* stream) {
  if (n_q < 0 || n_streams < 0 || n_kv_heads < 1 || n_q_heads < 1 || n_q_heads % n_kv_heads || max_blocks < 1 || sel_block < 1 || n_select < 1)
    return CS_EINVAL;
  if (stride_slot < 0 || stride_head < 0 || !(softmax_scale > 0.0f && softmax_scale <= 3.0e38f)) return CS_EINVAL;
  if (dtype != CS_F32 && dtype != CS_BF16) return CS_EUNSUPPORTED;
  if ((head_dim != 64 && head_dim != 128) || block_size != CS_KV_BLOCK || n_q_heads / n_kv_heads > kRows) return CS_EUNSUPPORTED;
  if (sel_block % CS_KV_BLOCK || sel_block > CS_SELECT_BLOCK_MOST || n_select > CS_SELECT_MOST || n_kv_heads > 65535 || max_blocks > (1 << 27) - 65)
    return CS_EUNSUPPORTED;
  if (n_q >= 1ll << 26) return CS_EUNSUPPORTED;
  const int elems = dtype == CS_BF16 ? 8 : 4;
  if (stride_slot % elems || stride_head % elems) return CS_EUNSUPPORTED;
  if (n_q == 0 || n_streams == 0) return CS_OK;
  if (!q || !k_cache_layer || !v_cache_layer || !cu_q || !q_pos || !kv_len || !block_table || !selected || !out) return CS_EINVAL;
  if (!cs::aligned16(q) || !cs::aligned16(k_cache_layer) || !cs::aligned16(v_cache_layer) || !cs::aligned16(out)) return CS_EUNSUPPORTED;
  const Shape s = shape_of(n_q, n_streams, n_q_heads, n_kv_heads, head_dim, sel_block, n_select, dtype == CS_BF16, stride_slot);
  if (s.partials && (!workspace || !cs::aligned16(workspace) || workspace_bytes < s.partials)) return CS_EWORKSPACE;
  const int64_t groups = s.tiles * n_kv_heads * s.pieces;
  if (groups > cs::kMostThreads / 512) return CS_EUNSUPPORTED;
  Params p;
  p.q = q;
  p.k = k_cache_layer;
  p.v = v_cache_layer;
  p.cu_q = cu_q;
  p.q_pos = q_pos;
  p.kv_len = kv_len;
  p.block_table = block_table;
  p.selected = selected;
  p.out = out;
  p.lse = lse;
  p.ws_o = static_cast<float*>(workspace);
  p.ws_ml = s.partials ? p.ws_o + groups * (s.rows ? kRowsGroup : kRows) * head_dim : nullptr;
  p.n_q = n_q;
  p.stride_slot = stride_slot;
  p.stride_head = stride_head;
  p.max_blocks = max_blocks;
  p.n_streams = n_streams;
  p.n_q_heads = n_q_heads;
  p.n_kv_heads = n_kv_heads;
  p.group = n_q_heads / n_kv_heads;
  p.tile = s.tile;
  p.n_select = n_select;
  p.cache_blocks = sel_block / CS_KV_BLOCK;
  p.pieces = s.pieces;
  const double scale = static_cast<double>(softmax_scale) * 1.4426950408889634;
  p.scale_log2e = static_cast<float>(scale < 3.4e38 ? scale : 3.4e38);
  p.scale_rest = p.scale_log2e < kFar ? static_cast<float>(scale - p.scale_log2e) : 0.0f;
  hipStream_t st = cs::as_stream(stream);
  const dim3 grid(static_cast<unsigned>(groups));
#define CS_LAUNCH_SELECTED(KIND, D)                                                                                        \
  do {                                                                                                                     \
    if (s.waves == 4) hipLaunchKernelGGL((selected_attn_kernel<KIND<D>, D, 4>), grid, dim3(256), 0, st, p);                \
    else if (s.waves == 2) hipLaunchKernelGGL((selected_attn_kernel<KIND<D>, D, 2>), grid, dim3(128), 0, st, p);           \
    else hipLaunchKernelGGL((selected_attn_kernel<KIND<D>, D, 1>), grid, dim3(64), 0, st, p);                              \
  } while (0)
  if (s.rows) {
    const bool paired = p.cache_blocks % kStepGroups == 0;
    if (head_dim == 128 && paired) hipLaunchKernelGGL((selected_rows_kernel<128, true>), grid, dim3(64 * kRowsWaves), 0, st, p);
    else if (head_dim == 128) hipLaunchKernelGGL((selected_rows_kernel<128, false>), grid, dim3(64 * kRowsWaves), 0, st, p);
    else if (paired) hipLaunchKernelGGL((selected_rows_kernel<64, true>), grid, dim3(64 * kRowsWaves), 0, st, p);
    else hipLaunchKernelGGL((selected_rows_kernel<64, false>), grid, dim3(64 * kRowsWaves), 0, st, p);
  } else if (dtype == CS_BF16) {
    if (head_dim == 128) CS_LAUNCH_SELECTED(Bf16, 128);
    else CS_LAUNCH_SELECTED(Bf16, 64);
  } else {
    if (head_dim == 128) CS_LAUNCH_SELECTED(F32, 128);
    else CS_LAUNCH_SELECTED(F32, 64);
  }
#undef CS_LAUNCH_SELECTED
  if (s.pieces > 1) {
    const int status = cs::note_hip(hipGetLastError());
    if (status != CS_OK) return status;
    const int rows = s.rows ? kRowsGroup : kRows;
    const dim3 joins(static_cast<unsigned>(s.tiles * n_kv_heads), static_cast<unsigned>(rows * (head_dim / 4) / 256));
    const int bf16 = dtype == CS_BF16;
    if (head_dim == 128 && s.rows) hipLaunchKernelGGL((selected_join_kernel<128, kRowsGroup>), joins, dim3(256), 0, st, p, bf16);
    else if (head_dim == 128) hipLaunchKernelGGL((selected_join_kernel<128, kRows>), joins, dim3(256), 0, st, p, bf16);
    else if (s.rows) hipLaunchKernelGGL((selected_join_kernel<64, kRowsGroup>), joins, dim3(256), 0, st, p, bf16);
    else hipLaunchKernelGGL((selected_join_kernel<64, kRows>), joins, dim3(256), 0, st, p, bf16);
  }
  return cs::note_hip(hipGetLastError());
}
