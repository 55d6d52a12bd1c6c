// Which blocks of a long cache a query reads, gfx950: bounds of the keys of every block, and the choice by a bound on the products
// with them.
//
// Bounds.  A block of `sel_block` entries of a stream and kv head is described by its channels' largest and smallest key as whole numbers
// of a power of two:  hi_c = ceil(max_j K_jc / 2^k),  lo_c = floor(min_j K_jc / 2^k),  k the least with all |.| <= 127.  Largest and
// smallest know no rounding and no order of sums, so the numbers are the same however they are found.
//
// Choice.  The heads of a query token and kv head become whole numbers too, qc = q / 2^f rounded to nearest (f the least with all |qc| <=
// 127), and a block's score is
//     2^k max_h sum_c max(qc_hc hi_c, qc_hc lo_c)      >= every q_h . K_j of the block, up to the rounding of q
// The sum over c is  q+ . hi + q- . lo  with q+ = max(qc, 0), q- = min(qc, 0): a matrix product of bytes over 2 d, exact in 32 bits.  The
// scores that are compared are one power of two times whole numbers below 2^21, exact in fp32: lists are the same on any machine, in any order.
#include <math.h>

#include <atomic>
#include <type_traits>

#include "kv4.h"
#include "lds_rows.h"
#include "token_tiles.h"

namespace {

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(16))) int i32x16;

constexpr uint32_t kNoNumber = 255;      // scale byte of a block that holds a NaN or an infinity
constexpr int kLeast = 32;               // least scale byte: powers below 2^-95 are not needed, and scores stay normal numbers

// Scale byte of numbers whose largest magnitude has the given fp32 bits: the least k >= kLeast - 127 with amax <= 127 * 2^k, biased by 127.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return kNoNumber;
  const int e = static_cast<int>((amax_bits + 0x1ffffu) >> 23) - 6;
  return e < kLeast ? kLeast : static_cast<uint32_t>(e);
}
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }      // 2^-k

// ------------------------------------------------------------------------------------------ bounds

struct BoundsParams {
  const void* __restrict__ k;
  const int32_t* __restrict__ from;      // nullptr: all blocks
  const int32_t* __restrict__ kv_len;
  const int32_t* __restrict__ block_table;
  int8_t* __restrict__ bounds;           // [n_streams][n_kv_heads][n_sel][2][head_dim]
  uint8_t* __restrict__ scales;          // [n_streams][n_kv_heads][n_sel]
  int64_t stride_slot, stride_head;
  int32_t max_blocks, n_streams, n_kv_heads, n_sel, cache_blocks;      // cache_blocks: of a block
  int32_t walkers;                       // waves that share the blocks of a stream and kv head
};

// Waves at most: as good as one a block (32 windows, 28,000 blocks of 64 keys: 8,192 waves 102 us, 16,384 96, one a block 91), or, where only
// the blocks from `from` on are made, as few as fill the card, since most find nothing to do (32 tokens: 16,384 waves 12.3 us, 2,048 5.8, 1,024
// 4.4, 512 4.4).
constexpr int kManyWaves = 1 << 20, kFewWaves = 1024;
// A wave takes a block, lanes side by side on a row's channels, and goes on with the block `walkers` further.  Largest, smallest and greatest
// magnitude are kept while the rows pass, UC cache blocks asked for at once; lanes that hold other rows of the same channels are joined at
// the end.  Bound by memory: 32 windows of 17,630 entries at most, 4 heads of 128, 446 MB, take 91 us, 4.9 TB/s (a large copy: 5.1); in
// fp32, 892 MB, 164 us.
template <bool kBf16, int D, int UC>
__global__ __launch_bounds__(256) void key_bounds_kernel(BoundsParams p) {
  using Elem = typename std::conditional<kBf16, uint16_t, float>::type;
  constexpr int VE = kBf16 ? 8 : 4;      // elements a lane
  constexpr int LR = D / VE;             // lanes a row
  constexpr int RL = 64 / LR;            // rows a load
  constexpr int NL = CS_KV_BLOCK / RL;   // loads a cache block
  const int lane = threadIdx.x & 63;
  const uint32_t unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);      // (below 2^26 * 4)
  const uint32_t rest = unit / static_cast<uint32_t>(p.n_kv_heads);
  const int kvh = static_cast<int>(unit - rest * p.n_kv_heads), stream = static_cast<int>(rest / static_cast<uint32_t>(p.walkers));
  const int walker = static_cast<int>(rest - static_cast<uint32_t>(stream) * p.walkers);
  if (stream >= p.n_streams) return;
  const int entries = min(p.kv_len[stream], p.max_blocks * CS_KV_BLOCK);
  const int size = p.cache_blocks * CS_KV_BLOCK;
  const int first = p.from ? max(p.from[stream], 0) / size : 0;
  const int32_t* ids = p.block_table + static_cast<int64_t>(stream) * p.max_blocks;
  const int row = lane / LR, c = lane % LR;
  const Elem* base = static_cast<const Elem*>(p.k) + static_cast<int64_t>(kvh) * p.stride_head + c * VE;
  for (int64_t b = static_cast<int64_t>(first) + walker; b * size < entries; b += p.walkers) {
    const int begin = static_cast<int>(b) * size, last = min(entries - begin, size) - 1;      // last: of the block's entries
    float hi[VE], lo[VE];
    uint32_t amax = 0;
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      hi[e] = -INFINITY;
      lo[e] = INFINITY;
    }
    for (int cb0 = 0; cb0 * CS_KV_BLOCK <= last; cb0 += UC) {
      cs::u32x4 v[UC][NL];
#pragma unroll
      for (int u = 0; u < UC; ++u) {
        // (rows past the last one are that one again: it changes nothing)
        const int cb = min((cb0 + u) * CS_KV_BLOCK, last) / CS_KV_BLOCK;
        const int64_t at = static_cast<int64_t>(ids[begin / CS_KV_BLOCK + cb]) * CS_KV_BLOCK;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          const int r = min((cb0 + u) * CS_KV_BLOCK + i * RL + row, last) - cb * CS_KV_BLOCK;
          v[u][i] = *reinterpret_cast<const cs::u32x4*>(base + (at + r) * p.stride_slot);
        }
      }
#pragma unroll
      for (int u = 0; u < UC; ++u)
#pragma unroll
        for (int i = 0; i < NL; ++i)
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            const uint32_t w = v[u][i][kBf16 ? e / 2 : e];
            const uint32_t bits = kBf16 ? (e & 1 ? w & 0xffff0000u : w << 16) : w;
            amax = max(amax, bits & 0x7fffffffu);
            hi[e] = fmaxf(hi[e], __uint_as_float(bits));
            lo[e] = fminf(lo[e], __uint_as_float(bits));
          }
    }
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      if (LR <= 8) {
        hi[e] = fmaxf(hi[e], __uint_as_float(cs::lane_dpp<0x128>(__float_as_uint(hi[e]))));      // lane ^ 8
        lo[e] = fminf(lo[e], __uint_as_float(cs::lane_dpp<0x128>(__float_as_uint(lo[e]))));
      }
      if (LR <= 16) {
        hi[e] = cs::with_lane16(hi[e], cs::larger);
        lo[e] = cs::with_lane16(lo[e], cs::smaller);
      }
      hi[e] = cs::with_lane32(hi[e], cs::larger);
      lo[e] = cs::with_lane32(lo[e], cs::smaller);
    }
    const uint32_t byte = scale_byte(cs::lanes_max<64>(amax));
    const float inv = inverse_scale(byte == kNoNumber ? 127u : byte);
    const int64_t at = (static_cast<int64_t>(stream) * p.n_kv_heads + kvh) * p.n_sel + b;
    if (lane == 0) p.scales[at] = static_cast<uint8_t>(byte);
    if (row > 1) continue;               // the first row of lanes writes the upper bounds, the second the lower ones
    uint32_t word[VE / 4] = {};
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      // (a number that 2^-k takes below the smallest one still lies past 0)
      const float x = row == 0 ? hi[e] : -lo[e];
      int code = static_cast<int>(ceilf(x * inv));
      if (x > 0.0f) code = max(code, 1);
      if (row != 0) code = -code;
      if (byte == kNoNumber) code = 0;
      word[e / 4] |= (static_cast<uint32_t>(code) & 0xffu) << (8 * (e % 4));
    }
    int8_t* dst = p.bounds + at * 2 * D + row * D + c * VE;
    if constexpr (VE == 8) *reinterpret_cast<cs::u32x2*>(dst) = cs::u32x2{word[0], word[1]};
    else *reinterpret_cast<uint32_t*>(dst) = word[0];
  }
}

// ------------------------------------------------------------------------------------------ choice

struct SelectParams {
  const void* __restrict__ q;
  const int8_t* __restrict__ bounds;
  const uint8_t* __restrict__ scales;
  const int32_t* __restrict__ cu_q;
  const int32_t* __restrict__ q_pos;
  const int32_t* __restrict__ kv_len;
  int32_t* __restrict__ selected;        // [n_q][n_kv_heads][n_select]
  int64_t n_q;
  int32_t max_blocks, n_streams, n_q_heads, n_kv_heads, group, n_sel, size, n_select, n_first, n_last, tile, pitch;
};

// Which kernel: workgroups of 16 waves share a tile's blocks out among themselves, as long as all of them are on the card at once (two a
// CU); past that pairs of waves with rows of their own do more for what they read.  28 on 4 heads, 276 blocks, wide / pairs: 64 tokens 7.5 /
// 12.2 us, 256 8.1 / 12.4, 512 12.0 / 12.8, 768 (the first over 512 workgroups) 16.6 / 12.7, 1,024 20.8 / 13.0.  And a pair needs
// the scores of two tokens at once: 1,250 blocks, 1,024 tokens 50 / 64 us (pairs of one token each), 938 blocks, 2,082 tokens 81 / 61 us.
constexpr int kWideGroups = 512;
constexpr int kPairTokens = 2, kPairBlocks = 1024;
constexpr int kMostBlocks = 32768;       // whose scores a workgroup holds in LDS for one token
constexpr int kTileScores = 8192;        // ... for a tile of tokens

// Scores in the order of unsigned numbers; every one is past 0.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr uint32_t kOdd = 0xfffffffeu;    // ... of a block that holds what is no number

// The largest T with at least `wanted` (> 0) scores >= T, and how many are > T.  `at(c)` is the lane's score of chunk c, 0 where it has none.
// Found bit by bit from the first one in which the scores differ, counting by ballots.  C: chunks, or 0: counted when the kernel runs.
template <int C, class F>
__device__ __forceinline__ void threshold(const F& at, int chunks, int wanted, uint32_t* t_out, int* above_out) {
  if (C) chunks = C;
  uint32_t high = 0, low = 0xffffffffu;
#pragma unroll(C ? C : 1)
  for (int c = 0; c < chunks; ++c) {
    const uint32_t x = at(c);
    high = max(high, x);
    low = min(low, x ? x : 0xffffffffu);
  }
  high = __builtin_amdgcn_readfirstlane(cs::lanes_max<64>(high));
  low = ~__builtin_amdgcn_readfirstlane(cs::lanes_max<64>(~low));
  const int first_bit = 31 - __clz(high ^ low);        // (-1: all are equal)
  uint32_t t = first_bit < 0 ? high : high & ~(0xffffffffu >> (31 - first_bit));
  for (int bit = first_bit; bit >= 0; --bit) {
    const uint32_t cand = t | 1u << bit;
    int count = 0;
#pragma unroll(C ? C : 1)
    for (int c = 0; c < chunks; ++c) count += __popcll(__ballot(at(c) >= cand));
    if (count >= wanted) {
      t = cand;
      if (count == wanted) break;
    }
  }
  int above = 0;
#pragma unroll(C ? C : 1)
  for (int c = 0; c < chunks; ++c) above += __popcll(__ballot(at(c) > t));
  *t_out = t;
  *above_out = above;
}

// The query's list from the scores of its n blocks, more than n_select: those of the first n_first, the last n_last, and the n_select -
// n_first - n_last largest of the others, of which `above` are > t and the lowest ones = t follow.  Fixed blocks have the score 0.
template <int C, class F>
__device__ __forceinline__ void write_list(const F& at, int n, int n_first, int n_last, int n_select, uint32_t t, int above, int32_t* out, int lane) {
  const int chunks = C ? C : (n + 63) / 64;
  int ties = n_select - n_first - n_last - above, place = 0;
  const uint64_t below = (1ull << lane) - 1;
#pragma unroll(C ? C : 1)
  for (int c = 0; c < chunks; ++c) {
    const uint32_t x = at(c);
    const int block = c * 64 + lane;
    const bool fixed = block < n && (block < n_first || block >= n - n_last);
    const uint64_t equal = __ballot(x == t);
    const bool taken = fixed || x > t || (x == t && __popcll(equal & below) < ties);
    const uint64_t all = __ballot(taken);
    if (taken) out[place + __popcll(all & below)] = block;
    place += __popcll(all);
    ties -= min(ties, __popcll(equal));
  }
}

// The same from scores in registers.  kNarrow, where a few are wanted of many: a bound is found first, from the lanes' largest scores alone;
// what passes it moves into one register a lane, and the threshold is found there.  `score`: the row in LDS, not needed any more.  (1,563
// blocks 22.7 -> 19.9 us; with 276 blocks it costs more than it saves, and in the kernel for many tokens registers.)
constexpr int kNarrowChunks = 12;        // chunks from which it is taken (64 tokens, 768 blocks, 12 chunks: 13.0 us without, 11.8 with)
constexpr int kFewWanted = 32, kSpare = 8;             // of 64 places; largest scores that may pass the bound beside those wanted
template <int C, bool kNarrow, class F>
__device__ __forceinline__ void write_list_held(const F& key, int n, int n_first, int n_last, int n_select, uint32_t* score, int32_t* out, int lane) {
  uint32_t held[C];
#pragma unroll
  for (int c = 0; c < C; ++c) held[c] = key(c * 64 + lane);
  const auto at = [&](int c) __attribute__((always_inline)) { return held[c]; };
  const int wanted = n_select - n_first - n_last;
  uint32_t t = 0xffffffffu;                            // (nothing is wanted)
  int above = 0, passed = 65;
  if (kNarrow && wanted > 0 && wanted <= kFewWanted) {
    uint32_t most = held[0];
#pragma unroll
    for (int c = 1; c < C; ++c) most = max(most, held[c]);
    const uint32_t high = __builtin_amdgcn_readfirstlane(cs::lanes_max<64>(most));
    const uint32_t low = ~__builtin_amdgcn_readfirstlane(cs::lanes_max<64>(~most));
    const int first_bit = 31 - __clz(high ^ low);
    uint32_t bound = first_bit < 0 ? high : high & ~(0xffffffffu >> (31 - first_bit));
    for (int bit = first_bit; bit >= 0; --bit) {
      const uint32_t cand = bound | 1u << bit;
      const int count = __popcll(__ballot(most >= cand));
      if (count >= wanted) {
        bound = cand;
        if (count <= wanted + kSpare) break;
      }
    }
    passed = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) passed += __popcll(__ballot(held[c] >= bound));
    if (passed <= 64) {
      const uint64_t below = (1ull << lane) - 1;
      int place = 0;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const uint64_t all = __ballot(held[c] >= bound);
        if (held[c] >= bound) score[place + __popcll(all & below)] = held[c];
        place += __popcll(all);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");              // (a wave's LDS operations are in order)
      const uint32_t x = lane < passed ? score[lane] : 0u;
      threshold<1>([&](int) __attribute__((always_inline)) { return x; }, 1, wanted, &t, &above);
      t = max(t, bound);                 // (below it are others)
      above = __popcll(__ballot(x > t));
    }
  }
  if (passed > 64 && wanted > 0) threshold<C>(at, C, wanted, &t, &above);
  write_list<C>(at, n, n_first, n_last, n_select, t, above, out, lane);
}

constexpr int kWide = 16;                // waves of a workgroup that takes few tokens
constexpr int kRowsWaves = 8, kPairs = kRowsWaves / 2;     // ... many
static_assert(kPairs * kPairTokens * kPairBlocks == kTileScores, "what a pair holds at least");

// Tokens whose heads, padded to GP, are 32 rows (8 at most).
template <int GP>
constexpr int kTokens = 32 / GP < 8 ? 32 / GP : 8;

// Whole numbers of a token's heads: 16 bytes a lane are asked for, then written to the token's rows of 32 in LDS, q+ and q- behind one another.
// Token k of the 32 rows is pair k / 2 of half k % 2: registers GP (k / 2) + slot of the lanes of that half, rows 8 (r / 4) + 4 half + r % 4.
template <bool kBf16, int D, int GP>
struct Query {
  static constexpr int VE = kBf16 ? 8 : 4, CHUNKS = D / VE, HELD = (GP * CHUNKS + 63) / 64, QROW = 2 * D + 16;
  cs::u32x4 v[HELD];

  static __device__ __forceinline__ uint32_t number(const cs::u32x4& x, int e) {
    const uint32_t w = x[kBf16 ? e / 2 : e];
    return kBf16 ? (e & 1 ? w & 0xffff0000u : w << 16) : w;
  }
  static constexpr float kWhole = 12582912.0f;
  static __device__ __forceinline__ uint32_t lowest_bytes(const uint32_t (&x)[4]) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(x[3], x[2], 0x0c0c0400), __builtin_amdgcn_perm(x[1], x[0], 0x0c0c0400), 0x05040100);
  }
  __device__ __forceinline__ void ask(const SelectParams& p, int tok, int kvh, int lane) {
    const int64_t from = (static_cast<int64_t>(tok) * p.n_q_heads + static_cast<int64_t>(kvh) * p.group) * D;
#pragma unroll
    for (int j = 0; j < HELD; ++j) {
      const int c = j * 64 + lane, head = min(c / CHUNKS, p.group - 1);      // (past the group: its last head again)
      const int64_t at = from + head * D + c % CHUNKS * VE;
      if constexpr (kBf16) v[j] = *reinterpret_cast<const cs::u32x4*>(static_cast<const uint16_t*>(p.q) + at);
      else v[j] = *reinterpret_cast<const cs::u32x4*>(static_cast<const float*>(p.q) + at);
    }
  }
  __device__ __forceinline__ void put(uint8_t* rows, int k, int lane) const {
    uint32_t amax = 0;
#pragma unroll
    for (int j = 0; j < HELD; ++j)
#pragma unroll
      for (int e = 0; e < VE; ++e) amax = max(amax, number(v[j], e) & 0x7fffffffu);
    const uint32_t byte = scale_byte(cs::lanes_max<64>(amax));
    const float inv = byte == kNoNumber ? 0.0f : inverse_scale(byte);
#pragma unroll
    for (int j = 0; j < HELD; ++j) {
      const int c = j * 64 + lane, slot = c / CHUNKS;
      if (slot >= GP) continue;
      // A sum with 1.5 x 2^23 rounds to a whole number, whose lowest byte is the code.  (A query that holds what is no number: 0 throughout.)
      uint32_t up[VE / 4], down[VE / 4];
#pragma unroll
      for (int w = 0; w < VE / 4; ++w) {
        uint32_t u[4], d[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float code = byte == kNoNumber ? kWhole : fmaf(__uint_as_float(number(v[j], 4 * w + e)), inv, kWhole);
          u[e] = __float_as_uint(fmaxf(code, kWhole));
          d[e] = __float_as_uint(fminf(code, kWhole));
        }
        up[w] = lowest_bytes(u);
        down[w] = lowest_bytes(d);
      }
      const int r = GP * (k / 2) + slot, row = 8 * (r / 4) + 4 * (k % 2) + r % 4;
      uint8_t* dst = rows + row * QROW + c % CHUNKS * VE;
      if constexpr (VE == 8) {
        *reinterpret_cast<cs::u32x2*>(dst) = cs::u32x2{up[0], up[1]};
        *reinterpret_cast<cs::u32x2*>(dst + D) = cs::u32x2{down[0], down[1]};
      } else {
        *reinterpret_cast<uint32_t*>(dst) = up[0];
        *reinterpret_cast<uint32_t*>(dst + D) = down[0];
      }
    }
  }
};

// Scores of a lane's block for the tokens of 32 rows, from the products with all of their heads: f(token, score).
template <int GP, class F>
__device__ __forceinline__ void each_score(const i32x16& acc, uint32_t byte, int h, const F& f) {
  const float scale = __uint_as_float((byte - 21u) << 23);               // 2^(k - 21)
#pragma unroll
  for (int g = 0; g < (kTokens<GP> + 1) / 2; ++g) {
    int top = acc[g * GP];
#pragma unroll
    for (int i = 1; i < GP; ++i) top = max(top, acc[g * GP + i]);
    f(2 * g + h, byte == kNoNumber ? kOdd : ordered(static_cast<float>(top) * scale));
  }
}

// Candidates of the tile's token `lane` (0: none, or no such token).
__device__ __forceinline__ int candidates_of(const SelectParams& p, const cs::TokenTile& t, int lane) {
  const int entries = min(p.kv_len[t.stream], p.max_blocks * CS_KV_BLOCK);
  const int last = lane < t.count ? min(p.q_pos[t.first + lane], entries - 1) : -1;
  return last < 0 ? 0 : last / p.size + 1;
}

// The list of token `tok` from its scores, by a wave.  kMost: blocks that it may be among (0: any number).
template <int kMost>
__device__ __forceinline__ void select_token(const SelectParams& p, uint32_t* score, int tok, int kvh, int n, int lane) {
  int32_t* out = p.selected + (static_cast<int64_t>(tok) * p.n_kv_heads + kvh) * p.n_select;
  if (n <= p.n_select) {
    for (int c = lane; c < p.n_select; c += 64) out[c] = c < n ? c : -1;
    return;
  }
  const auto key = [&](int b) __attribute__((always_inline)) -> uint32_t { return b < p.n_first || b >= n - p.n_last ? 0u : score[b]; };
  // As many registers as the list has chunks of 64 blocks, by a rule that leaves no window out: every number up to 8, then 12, 16, 24, 32, so
  // that less than half again of what is counted is padding.  2,082 tokens, powers of two alone / this: 192 blocks 16.4 / 15.8 us, 276 23.3 /
  // 19.5, 384 28.4 / 26.2, 448 29.7 / 28.4, 768 54.2 / 49.8; a token among 1,536 blocks 19.4 / 18.3.
#define CS_LIST(C) write_list_held<C, kMost == 0 && (C >= kNarrowChunks)>(key, n, p.n_first, p.n_last, p.n_select, score, out, lane)
  if (n <= 128) CS_LIST(2);
  else if (n <= 192) CS_LIST(3);
  else if (n <= 256) CS_LIST(4);
  else if (n <= 320) CS_LIST(5);
  else if (n <= 384) CS_LIST(6);
  else if (n <= 448) CS_LIST(7);
  else if (n <= 512) CS_LIST(8);
  else if (n <= 768) CS_LIST(12);
  else if (kMost == 1024 || n <= 1024) CS_LIST(16);
  else if (n <= 1536) CS_LIST(24);
  else if (n <= 2048) CS_LIST(32);
  else {
    const auto at = [&](int c) __attribute__((always_inline)) { return key(c * 64 + lane); };
    uint32_t t = 0xffffffffu;            // (nothing is wanted)
    int above = 0;
    const int wanted = p.n_select - p.n_first - p.n_last;
    if (wanted > 0) threshold<0>(at, (n + 63) / 64, wanted, &t, &above);
    write_list<0>(at, n, p.n_first, p.n_last, p.n_select, t, above, out, lane);
  }
#undef CS_LIST
}

// Few tokens: a workgroup takes those of 32 rows and a kv head, its 16 waves the blocks in turn, 32 columns at a time; then each wave the
// list of a token.  Bound by latency, of launch, queries, bounds, counting one after the other: a token among 276 blocks 6.6 us, 64 tokens 7.5, a
// token among 1,563 blocks 19.9.  Rows are (token, head), the heads of a token padded to GP by the last of them and spread so that they are
// neighbouring registers of a lane.
template <bool kBf16, int D, int GP>
__global__ __launch_bounds__(64 * kWide) void select_blocks_kernel(SelectParams p) {
  typedef Query<kBf16, D, GP> Q;
  constexpr int STEPS = 2 * D / 32;
  __shared__ __attribute__((aligned(16))) uint8_t s_q[32 * Q::QROW];
  extern __shared__ __attribute__((aligned(16))) uint32_t s_score[];      // [tile][pitch]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
  const int kvh = static_cast<int>(blockIdx.x % p.n_kv_heads);
  cs::TokenTile t;
  if (!cs::find_token_tile(p.cu_q, p.n_streams, p.n_q, p.tile, static_cast<int>(blockIdx.x / p.n_kv_heads), &t)) return;
  if (wave < t.count) {
    Q q;
    q.ask(p, t.first + wave, kvh, lane);
    q.put(s_q, wave, lane);
  }
  const int candidates = candidates_of(p, t, lane);
  const int most = __builtin_amdgcn_readfirstlane(static_cast<int>(cs::lanes_max<64>(static_cast<uint32_t>(candidates))));
  __syncthreads();

  if (most > p.n_select) {               // (rows without a token hold anything: nobody reads their scores)
    i32x4 a[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) a[s] = *reinterpret_cast<const i32x4*>(s_q + n * Q::QROW + 32 * s + 16 * h);
    const int64_t head_at = (static_cast<int64_t>(t.stream) * p.n_kv_heads + kvh) * p.n_sel;
    for (int b0 = wave * 32; b0 < most; b0 += 32 * kWide) {
      const int block = min(b0 + n, most - 1);
      const int8_t* from = p.bounds + (head_at + block) * 2 * D + 16 * h;
      const uint32_t byte = p.scales[head_at + block];
      i32x4 b[STEPS];
#pragma unroll
      for (int s = 0; s < STEPS; ++s) b[s] = *reinterpret_cast<const i32x4*>(from + 32 * s);
      i32x16 acc = {};
#pragma unroll
      for (int s = 0; s < STEPS; ++s) acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[s], b[s], acc, 0, 0, 0);
      each_score<GP>(acc, byte, h, [&](int tok, uint32_t x) __attribute__((always_inline)) {
        if (b0 + n < most && tok < t.count) s_score[tok * p.pitch + block] = x;
      });
    }
  }
  __syncthreads();
  if (wave < t.count) select_token<0>(p, s_score + wave * p.pitch, t.first + wave, kvh, __builtin_amdgcn_readlane(candidates, wave), lane);
}

// Many tokens: two waves of a workgroup share 32 rows, four pairs take 64 columns a step, one wave of a pair the first 32 of them, the
// other the others.  Columns pass through LDS once, a step ahead; the second stage and the scores take the queries' place.  Then each wave
// makes the lists of every second token of its pair.  2,082 tokens of 28 heads on 4, 276 blocks: 20 us, of which the lists take 8 (scalar
// counting), the products 6, the queries 3; every wave with 32 rows of its own 23.
template <bool kBf16, int D, int GP>
__global__ __launch_bounds__(64 * kRowsWaves) void select_rows_kernel(SelectParams p) {
  typedef Query<kBf16, D, GP> Q;
  constexpr int STEPS = 2 * D / 32;
  constexpr int kStage = 64 * 2 * D, kParts = kStage / 1024 / kRowsWaves;    // bytes of 64 blocks, requests of a wave for them
  constexpr int LR = 2 * D / 16, RL = 64 / LR;             // lanes of a block, blocks of a request
  // a stage, then the queries [pairs][32 rows], or the other stage and the scores [tile][pitch]
  extern __shared__ __attribute__((aligned(16))) uint8_t s_mem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
  const int kvh = static_cast<int>(blockIdx.x % p.n_kv_heads);
  cs::TokenTile t;
  if (!cs::find_token_tile(p.cu_q, p.n_streams, p.n_q, p.tile, static_cast<int>(blockIdx.x / p.n_kv_heads), &t)) return;
  const int pair = wave >> 1, half = wave & 1;
  const int first = pair * (p.tile / kPairs), mine = min(p.tile / kPairs, t.count - first);      // the pair's tokens (fewer than one: none)
  const int64_t head_at = (static_cast<int64_t>(t.stream) * p.n_kv_heads + kvh) * p.n_sel;
  const char* bounds = reinterpret_cast<const char*>(p.bounds + head_at * 2 * D);
  const uint32_t to = __builtin_amdgcn_readfirstlane(cs::lds_address(s_mem)) + wave * kParts * 1024;
  const auto request = [&](int i) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < kParts; ++j) {
      const int row = (wave * kParts + j) * RL + lane / LR;
      cs::to_lds(static_cast<uint32_t>(min(64 * i + row, p.n_sel - 1)) * (2 * D) + 16 * (lane % LR ^ cs::row_place<D>(row)), bounds, to + (i & 1) * kStage + 1024 * j);
    }
  };
  request(0);                            // (before anything else: it lands while the queries are looked at)
  const int candidates = candidates_of(p, t, lane);
  uint8_t* rows = s_mem + kStage + pair * 32 * Q::QROW;
  for (int i0 = half; i0 < mine; i0 += 4) {
    Q q[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) q[i].ask(p, t.first + first + min(i0 + 2 * i, mine - 1), kvh, lane);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (i0 + 2 * i < mine) q[i].put(rows, i0 + 2 * i, lane);
  }
  const int most = __builtin_amdgcn_readfirstlane(static_cast<int>(cs::lanes_max<64>(static_cast<uint32_t>(candidates))));
  __syncthreads();
  i32x4 a[STEPS];
#pragma unroll
  for (int s = 0; s < STEPS; ++s) a[s] = *reinterpret_cast<const i32x4*>(rows + n * Q::QROW + 32 * s + 16 * h);
  uint32_t* score = reinterpret_cast<uint32_t*>(s_mem + 2 * kStage) + first * p.pitch;

  const int steps = most > p.n_select ? (most + 63) / 64 : 0;
  for (int i = 0; i < steps; ++i) {
    const int block = 64 * i + 32 * half + n;
    const uint32_t byte = p.scales[head_at + min(block, most - 1)];
    cs::rows_gate();                     // (the first one: everyone holds its queries)
    if (i + 1 < steps) request(i + 1);
    const uint8_t* b = s_mem + (i & 1) * kStage + (32 * half + n) * 2 * D;
    i32x16 acc = {};
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
      acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[s], *reinterpret_cast<const i32x4*>(b + 16 * ((2 * s + h) ^ cs::row_place<D>(n))), acc, 0, 0, 0);
    each_score<GP>(acc, byte, h, [&](int tok, uint32_t x) __attribute__((always_inline)) {
      if (block < most && tok < mine) score[tok * p.pitch + block] = x;
    });
  }
  cs::rows_gate();                       // (also where no step has waited for the first request)
  for (int i = half; i < mine; i += 2) select_token<kPairBlocks>(p, score + i * p.pitch, t.first + first + i, kvh, __builtin_amdgcn_readlane(candidates, first + i), lane);
}

// LDS that a workgroup of many tokens takes: a stage, then the queries, or the other stage and the scores.
constexpr size_t rows_lds(int head_dim, size_t scores) {
  const size_t stage = 64 * 2 * static_cast<size_t>(head_dim), queries = static_cast<size_t>(kPairs) * 32 * (2 * head_dim + 16);
  return stage + (queries > stage + scores ? queries : stage + scores);
}
constexpr size_t kMostLdsWide = kMostBlocks * sizeof(uint32_t);
template <int D>
constexpr size_t kMostLdsRows = rows_lds(D, kTileScores * sizeof(uint32_t));

// A kernel's limit on the LDS of a launch is the process's: it is raised once a device, to the most that any call takes, since a limit of one
// call's own could be lowered by another thread's between this and the launch.
template <void (*kKernel)(SelectParams), size_t kMostLds>
int launch(const SelectParams& p, dim3 grid, int threads, size_t lds, hipStream_t st) {
  if (lds > 32 * 1024) {
    static std::atomic<uint64_t> raised{0};                // a bit a device
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    const uint64_t bit = device < 64 ? 1ull << device : 0;
    if (e == hipSuccess && !(raised.load(std::memory_order_acquire) & bit)) {
      e = hipFuncSetAttribute(reinterpret_cast<const void*>(kKernel), hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kMostLds));
      if (e == hipSuccess) raised.fetch_or(bit, std::memory_order_release);
    }
    if (e != hipSuccess) return cs::note_hip(e);
  }
  hipLaunchKernelGGL(kKernel, grid, dim3(threads), lds, st, p);
  return cs::note_hip(hipGetLastError());
}

}  // namespace

extern "C" int cs_key_bounds(const void* k_cache_layer, const int32_t* from, const int32_t* kv_len, const int32_t* block_table,
                             int32_t max_blocks, int32_t block_size, int32_t sel_block, int8_t* bounds, uint8_t* scales,
                             int32_t n_streams, int32_t n_kv_heads, int32_t head_dim, int64_t stride_slot, int64_t stride_head,
                             int32_t dtype, void* stream) {
  if (n_streams < 0 || n_kv_heads < 1 || max_blocks < 1 || sel_block < 1 || stride_slot < 0 || stride_head < 0) return CS_EINVAL;
  if (dtype != CS_F32 && dtype != CS_BF16) return CS_EUNSUPPORTED;
  if ((head_dim != 64 && head_dim != 128) || block_size != CS_KV_BLOCK) return CS_EUNSUPPORTED;
  if (sel_block % CS_KV_BLOCK || sel_block > CS_SELECT_BLOCK_MOST || n_kv_heads > 65535 || max_blocks > (1 << 27) - 65) return CS_EUNSUPPORTED;
  const int elems = dtype == CS_BF16 ? 8 : 4;
  if (stride_slot % elems || stride_head % elems) return CS_EUNSUPPORTED;
  if (n_streams == 0) return CS_OK;
  if (!k_cache_layer || !kv_len || !block_table || !bounds || !scales) return CS_EINVAL;
  if (!cs::aligned16(k_cache_layer) || !cs::aligned16(bounds)) return CS_EUNSUPPORTED;
  BoundsParams p;
  p.k = k_cache_layer;
  p.from = from;
  p.kv_len = kv_len;
  p.block_table = block_table;
  p.bounds = bounds;
  p.scales = scales;
  p.stride_slot = stride_slot;
  p.stride_head = stride_head;
  p.max_blocks = max_blocks;
  p.n_streams = n_streams;
  p.n_kv_heads = n_kv_heads;
  p.cache_blocks = sel_block / CS_KV_BLOCK;
  p.n_sel = (max_blocks + p.cache_blocks - 1) / p.cache_blocks;
  const int64_t pairs = static_cast<int64_t>(n_streams) * n_kv_heads;
  const int64_t wanted = ((from ? kFewWaves : kManyWaves) + pairs - 1) / pairs;
  p.walkers = static_cast<int32_t>(wanted < p.n_sel ? wanted : p.n_sel);
  const int64_t groups = (pairs * p.walkers + 3) / 4;
  if (groups > cs::kMostThreads / 256) return CS_EUNSUPPORTED;
  const dim3 grid(static_cast<unsigned>(groups));
  hipStream_t st = cs::as_stream(stream);
#define CS_LAUNCH_BOUNDS(BF16, D)                                                                                           \
  do {                                                                                                                      \
    if (p.cache_blocks == 1) hipLaunchKernelGGL((key_bounds_kernel<BF16, D, 1>), grid, dim3(256), 0, st, p);                \
    else if (p.cache_blocks == 2) hipLaunchKernelGGL((key_bounds_kernel<BF16, D, 2>), grid, dim3(256), 0, st, p);           \
    else hipLaunchKernelGGL((key_bounds_kernel<BF16, D, 4>), grid, dim3(256), 0, st, p);                                    \
  } while (0)
  if (dtype == CS_BF16) {
    if (head_dim == 128) CS_LAUNCH_BOUNDS(true, 128);
    else CS_LAUNCH_BOUNDS(true, 64);
  } else {
    if (head_dim == 128) CS_LAUNCH_BOUNDS(false, 128);
    else CS_LAUNCH_BOUNDS(false, 64);
  }
#undef CS_LAUNCH_BOUNDS
  return cs::note_hip(hipGetLastError());
}

extern "C" size_t cs_select_blocks_workspace(int64_t, int32_t, int32_t, int32_t, int32_t, int32_t, int32_t) { return 0; }

extern "C" int cs_select_blocks(const void* q, const int8_t* bounds, const uint8_t* scales, const int32_t* cu_q, const int32_t* q_pos,
                                const int32_t* kv_len, int32_t max_blocks, int32_t sel_block, int32_t n_select, int32_t n_first,
                                int32_t n_last, int32_t* selected, int64_t n_q, int32_t n_streams, int32_t n_q_heads, int32_t n_kv_heads,
                                int32_t head_dim, int32_t dtype, void* workspace, size_t workspace_bytes, void* stream) {
  (void)workspace;
  (void)workspace_bytes;
  if (n_q < 0 || n_streams < 0 || n_kv_heads < 1 || n_q_heads < 1 || n_q_heads % n_kv_heads || max_blocks < 1 || sel_block < 1) return CS_EINVAL;
  if (n_select < 1 || n_first < 0 || n_last < 0 || static_cast<int64_t>(n_first) + n_last > n_select) return CS_EINVAL;
  if (dtype != CS_F32 && dtype != CS_BF16) return CS_EUNSUPPORTED;
  if ((head_dim != 64 && head_dim != 128) || n_q_heads / n_kv_heads > 16) return CS_EUNSUPPORTED;
  if (sel_block % CS_KV_BLOCK || sel_block > CS_SELECT_BLOCK_MOST || n_kv_heads > 65535 || max_blocks > (1 << 27) - 65) return CS_EUNSUPPORTED;
  if (n_select > CS_SELECT_MOST || n_q >= 1ll << 26) return CS_EUNSUPPORTED;
  const int32_t per = sel_block / CS_KV_BLOCK, n_sel = (max_blocks + per - 1) / per;
  if (n_sel > kMostBlocks) return CS_EUNSUPPORTED;
  if (n_q == 0 || n_streams == 0) return CS_OK;
  if (!q || !bounds || !scales || !cu_q || !q_pos || !kv_len || !selected) return CS_EINVAL;
  if (!cs::aligned16(q) || !cs::aligned16(bounds)) return CS_EUNSUPPORTED;
  SelectParams p;
  p.q = q;
  p.bounds = bounds;
  p.scales = scales;
  p.cu_q = cu_q;
  p.q_pos = q_pos;
  p.kv_len = kv_len;
  p.selected = selected;
  p.n_q = n_q;
  p.max_blocks = max_blocks;
  p.n_streams = n_streams;
  p.n_q_heads = n_q_heads;
  p.n_kv_heads = n_kv_heads;
  p.group = n_q_heads / n_kv_heads;
  p.n_sel = n_sel;
  p.size = sel_block;
  p.n_select = n_select;
  p.n_first = n_first;
  p.n_last = n_last;
  int gp = 1;
  while (gp < p.group) gp *= 2;
  p.pitch = n_sel;
  const int tok = 32 / gp < 8 ? 32 / gp : 8;
  p.tile = tok;
  while (p.tile > 1 && static_cast<int64_t>(p.tile) * p.pitch > kTileScores) p.tile /= 2;
  const bool many = cs::most_token_tiles(n_q, n_streams, p.tile) * n_kv_heads > kWideGroups && n_sel <= kPairBlocks;
  if (many) {
    p.tile = kPairs * tok;
    while (static_cast<int64_t>(p.tile) * p.pitch > kTileScores) p.tile /= 2;
  }
  const int64_t tiles = cs::most_token_tiles(n_q, n_streams, p.tile), groups = tiles * n_kv_heads;
  if (groups > cs::kMostThreads / 1024) return CS_EUNSUPPORTED;
  const dim3 grid(static_cast<unsigned>(groups));
  const size_t scores = static_cast<size_t>(p.tile) * p.pitch * sizeof(uint32_t), lds = many ? rows_lds(head_dim, scores) : scores;
  hipStream_t st = cs::as_stream(stream);
#define CS_LAUNCH_SELECT(BF16, D, GP)                                                                                  \
  do {                                                                                                                 \
    if (many) return launch<select_rows_kernel<BF16, D, GP>, kMostLdsRows<D>>(p, grid, 64 * kRowsWaves, lds, st);      \
    return launch<select_blocks_kernel<BF16, D, GP>, kMostLdsWide>(p, grid, 64 * kWide, lds, st);                      \
  } while (0)
#define CS_LAUNCH_SELECT_GROUP(BF16, D)              \
  do {                                               \
    if (gp == 1) CS_LAUNCH_SELECT(BF16, D, 1);       \
    else if (gp == 2) CS_LAUNCH_SELECT(BF16, D, 2);  \
    else if (gp == 4) CS_LAUNCH_SELECT(BF16, D, 4);  \
    else if (gp == 8) CS_LAUNCH_SELECT(BF16, D, 8);  \
    else CS_LAUNCH_SELECT(BF16, D, 16);              \
  } while (0)
  if (dtype == CS_BF16) {
    if (head_dim == 128) CS_LAUNCH_SELECT_GROUP(true, 128);
    else CS_LAUNCH_SELECT_GROUP(true, 64);
  } else {
    if (head_dim == 128) CS_LAUNCH_SELECT_GROUP(false, 128);
    else CS_LAUNCH_SELECT_GROUP(false, 64);
  }
#undef CS_LAUNCH_SELECT_GROUP
#undef CS_LAUNCH_SELECT
}
