// Rows on their way into, inside and out of the window cache: rotary embedding of fresh queries and keys (one position, or
// one per axis: time, height, width) with the refresh write, position correction of 4-bit rows, and 4-bit rows as numbers.
//
// All three are single passes that memory bounds.  Rotation: a lane owns eight pairs of a token and evaluates their cosines
// and sines once (double precision, 30 fused operations a pair), then turns them in every head of its share; so the angles
// cost a few instructions a head.  4-bit blocks are 32 elements, so four lanes (pairs half a head apart) or two (neighbouring
// pairs) agree on a block's largest magnitude by lane exchanges, and nothing passes through LDS.
#include <type_traits>

#include "kv4.h"
#include "rope.h"

namespace {

constexpr int kPairs = 8;                // pairs a lane owns
// Workgroups wanted of the rotary write.  22,804 tokens of 32 + 2 x 8 heads of 128 take 112 us, 4.4 TB/s (a large copy reaches 4.1 to
// 5.0).  With their rows read back as numbers: 141 us at 4,096, 155 at 1,024 or 2,048, 153 at 16,384.
// A thread still takes up to four heads with one evaluation of its angles as long as two workgroups a CU are left: 3,000 tokens
// of 28 + 2 x 4 heads 27.6 -> 19.2 us with the rows read back, 7,000 39.4 -> 35.8 (six heads: 20.4 and 37.0; four workgroups a CU: 20.9, 35.5).
// A token alone is 5 us, and 13 to 18 from the host with its row read back.
constexpr int kRopeGroups = 4096, kRopeHeads = 4, kRopeEnough = 512;

template <bool kBf16>
struct Eight;
template <>
struct Eight<true> {                     // eight bf16: one 16-byte vector
  cs::u32x4 v;
  __device__ __forceinline__ void load(const uint16_t* p) { v = __builtin_nontemporal_load(reinterpret_cast<const cs::u32x4*>(p)); }
  __device__ __forceinline__ void get(float* f) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ void store(uint16_t* p, const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const cs::f32v2 x = {f[2 * i], f[2 * i + 1]};
      w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, cs::bf16v2));
    }
    __builtin_nontemporal_store(cs::u32x4{w[0], w[1], w[2], w[3]}, reinterpret_cast<cs::u32x4*>(p));
  }
};
template <>
struct Eight<false> {
  cs::u32x4 v, w;
  __device__ __forceinline__ void load(const float* p) {
    v = __builtin_nontemporal_load(reinterpret_cast<const cs::u32x4*>(p));
    w = __builtin_nontemporal_load(reinterpret_cast<const cs::u32x4*>(p + 4));
  }
  __device__ __forceinline__ void get(float* f) const {
    f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    f[4] = __uint_as_float(w.x); f[5] = __uint_as_float(w.y); f[6] = __uint_as_float(w.z); f[7] = __uint_as_float(w.w);
  }
  static __device__ __forceinline__ void store(float* p, const float* f) {
    __builtin_nontemporal_store(cs::u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])},
                                reinterpret_cast<cs::u32x4*>(p));
    __builtin_nontemporal_store(cs::u32x4{__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])},
                                reinterpret_cast<cs::u32x4*>(p + 4));
  }
};

// Largest of the lanes of a quad (kLanes 4) or of a pair (2).
template <int kLanes>
__device__ __forceinline__ uint32_t near_max(uint32_t x) {
  x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0xb1, 0xf, 0xf, true)));      // lane ^ 1
  if (kLanes == 4) x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x4e, 0xf, 0xf, true)));   // lane ^ 2
  return x;
}

struct RopeWriteParams {
  cs::RopeAngles rope;
  const void* q;
  void* q_out;                           // may be q
  const void* __restrict__ k_new;
  const void* __restrict__ v_new;
  const int32_t* __restrict__ slot;
  void* __restrict__ k_cache;
  void* __restrict__ v_cache;
  uint8_t* __restrict__ k_scales;
  uint8_t* __restrict__ v_scales;
  int64_t n_tok, stride_q, stride_q_out, stride_k, stride_v, stride_slot, stride_head;
  int32_t n_q_heads, n_kv_heads, head_dim, lanes_per_tok, heads_per_thread;
};

// Grid: x over (token, eight pairs), y over shares of the n_q_heads + 2 n_kv_heads heads of a token (queries, keys, values).
template <bool kBf16, int kStyle, bool kFour>
__global__ __launch_bounds__(256) void rope_write_kernel(RopeWriteParams p) {
  using Elem = typename std::conditional<kBf16, uint16_t, float>::type;
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  const int64_t tok = unit / p.lanes_per_tok;
  if (tok >= p.n_tok) return;            // (whole tokens: the lanes of a block leave together)
  const int j = static_cast<int>(unit - tok * p.lanes_per_tok);
  const int half = p.head_dim / 2;
  const int off_a = kStyle == CS_ROPE_HALF_SPLIT ? j * kPairs : 2 * j * kPairs;
  const int off_b = kStyle == CS_ROPE_HALF_SPLIT ? half + j * kPairs : 2 * j * kPairs + kPairs;
  const int h_begin = blockIdx.y * p.heads_per_thread;
  const int h_end = min(p.n_q_heads + 2 * p.n_kv_heads, h_begin + p.heads_per_thread);
  const int first_v = p.n_q_heads + p.n_kv_heads;
  const int slot = h_end > p.n_q_heads ? p.slot[tok] : -1;

  float cn[kPairs], sn[kPairs];
  const bool turned = p.rope.pos != nullptr && h_begin < first_v;
  if (turned) cs::rope_row<kPairs>(p.rope, tok, j * kPairs, cn, sn);

  constexpr int kBatch = kBf16 ? 4 : 2;
  for (int h0 = h_begin; h0 < h_end; h0 += kBatch) {
    Eight<kBf16> a[kBatch], b[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int h = h0 + i;
      if (h < h_end && (h < p.n_q_heads || slot >= 0)) {
        const Elem* src = h < p.n_q_heads ? static_cast<const Elem*>(p.q) + tok * p.stride_q + static_cast<int64_t>(h) * p.head_dim
                          : h < first_v   ? static_cast<const Elem*>(p.k_new) + tok * p.stride_k + static_cast<int64_t>(h - p.n_q_heads) * p.head_dim
                                          : static_cast<const Elem*>(p.v_new) + tok * p.stride_v + static_cast<int64_t>(h - first_v) * p.head_dim;
        a[i].load(src + off_a);
        b[i].load(src + off_b);
      }
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int h = h0 + i;
      if (!(h < h_end && (h < p.n_q_heads || slot >= 0))) continue;
      float fa[kPairs], fb[kPairs];
      a[i].get(fa);
      b[i].get(fb);
      if (turned && h < first_v) {
        float ya[kPairs], yb[kPairs];
        if (kStyle == CS_ROPE_HALF_SPLIT) {
#pragma unroll
          for (int e = 0; e < kPairs; ++e) cs::rope_turn(fa[e], fb[e], cn[e], sn[e], &ya[e], &yb[e]);
        } else {
#pragma unroll
          for (int e = 0; e < kPairs / 2; ++e) {
            cs::rope_turn(fa[2 * e], fa[2 * e + 1], cn[e], sn[e], &ya[2 * e], &ya[2 * e + 1]);
            cs::rope_turn(fb[2 * e], fb[2 * e + 1], cn[kPairs / 2 + e], sn[kPairs / 2 + e], &yb[2 * e], &yb[2 * e + 1]);
          }
        }
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
          fa[e] = ya[e];
          fb[e] = yb[e];
        }
      }
      if (h < p.n_q_heads) {
        Elem* dst = static_cast<Elem*>(p.q_out) + tok * p.stride_q_out + static_cast<int64_t>(h) * p.head_dim;
        Eight<kBf16>::store(dst + off_a, fa);
        Eight<kBf16>::store(dst + off_b, fb);
        continue;
      }
      const bool is_v = h >= first_v;
      const int64_t at = static_cast<int64_t>(slot) * p.stride_slot + static_cast<int64_t>(is_v ? h - first_v : h - p.n_q_heads) * p.stride_head;
      if (!kFour) {
        Elem* dst = static_cast<Elem*>(is_v ? p.v_cache : p.k_cache) + at;
        Eight<kBf16>::store(dst + off_a, fa);
        Eight<kBf16>::store(dst + off_b, fb);
      } else {
        uint32_t ma = 0, mb = 0;
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
          ma = max(ma, cs::abs_bits(fa[e]));
          mb = max(mb, cs::abs_bits(fb[e]));
        }
        uint8_t* codes = static_cast<uint8_t*>(is_v ? p.v_cache : p.k_cache);
        uint8_t* scales = is_v ? p.v_scales : p.k_scales;
        if (kStyle == CS_ROPE_HALF_SPLIT) {        // two blocks, four lanes each
          const uint32_t ea = cs::kv4_scale_byte(near_max<4>(ma)), eb = cs::kv4_scale_byte(near_max<4>(mb));
          *reinterpret_cast<uint32_t*>(codes + (at + off_a) / 2) = cs::kv4_pack8(fa, cs::kv4_scale(ea));
          *reinterpret_cast<uint32_t*>(codes + (at + off_b) / 2) = cs::kv4_pack8(fb, cs::kv4_scale(eb));
          if ((j & 3) == 0) {
            scales[(at + off_a) / cs::kKv4Block] = static_cast<uint8_t>(ea);
            scales[(at + off_b) / cs::kKv4Block] = static_cast<uint8_t>(eb);
          }
        } else {                                   // one block, two lanes
          const uint32_t e = cs::kv4_scale_byte(near_max<2>(max(ma, mb)));
          const float s = cs::kv4_scale(e);
          *reinterpret_cast<cs::u32x2*>(codes + (at + off_a) / 2) = cs::u32x2{cs::kv4_pack8(fa, s), cs::kv4_pack8(fb, s)};
          if ((j & 1) == 0) scales[(at + off_a) / cs::kKv4Block] = static_cast<uint8_t>(e);
        }
      }
    }
  }
}

struct GatherParams {
  const uint8_t* __restrict__ codes[2];
  const uint8_t* __restrict__ scales[2];
  void* __restrict__ out[2];
  const int32_t* __restrict__ slot;
  int64_t n_rows, stride_layer, stride_slot, stride_head, n_units;     // n_units: eight elements each, all layers
  int32_t n_kv_heads, lanes_per_head;
};

// A lane turns four bytes of codes into eight numbers; units run in the output's order, so stores are linear.  Bound by them: 15,023
// rows of 28 layers, 4 heads of 128, keys and values, take 253 us, 4.3 TB/s.
template <bool kBf16>
__global__ __launch_bounds__(256) void kv4_gather_kernel(GatherParams p) {
  using Elem = typename std::conditional<kBf16, uint16_t, float>::type;
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  if (unit >= p.n_units) return;
  const int which = blockIdx.y;
  const int64_t rh = unit / p.lanes_per_head;
  const int j = static_cast<int>(unit - rh * p.lanes_per_head);
  const int64_t lr = rh / p.n_kv_heads;
  const int head = static_cast<int>(rh - lr * p.n_kv_heads);
  const int64_t layer = lr / p.n_rows, row = lr - layer * p.n_rows;
  const int sl = p.slot[row];
  if (sl < 0) return;
  const int64_t at = layer * p.stride_layer + static_cast<int64_t>(sl) * p.stride_slot + static_cast<int64_t>(head) * p.stride_head + 8 * j;
  const uint32_t w = *reinterpret_cast<const uint32_t*>(p.codes[which] + at / 2);
  const uint32_t e = p.scales[which][at / cs::kKv4Block];
  float x[8];
  cs::kv4_unpack8(w, cs::kv4_scale(e), x);
  if (e == cs::kKv4NoNumber) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = NAN;
  }
  Eight<kBf16>::store(static_cast<Elem*>(p.out[which]) + unit * 8, x);
}

struct Kv4RerotateParams {
  cs::RopeAngles rope;
  uint8_t* k_codes;
  uint8_t* k_scales;
  uint8_t* v_codes;
  uint8_t* v_scales;
  const int32_t* __restrict__ src_slot;
  const int32_t* __restrict__ dst_slot;        // nullptr: in place, keys only
  int64_t n_rows, stride_layer, stride_slot, stride_head;
  int32_t n_layers, n_kv_heads, head_dim, lanes_per_head, layers_per_block, rows_per_block, scale_width;
};

// A workgroup evaluates the angles of its rows once, into LDS (all heads and layers of a row turn by them).  A lane owns 32 pairs of
// a row and head, two blocks, in every layer of its share: 16-byte loads, and a block's largest magnitude is the lane's own.
// Bound by memory, and by its requests where rows are not neighbours: 15,023 rows of 28 layers, 4 heads of 128, move at 4.2 TB/s
// (110 us) in a slot-major cache and 3.6 (127 us) head-major where slots run on within cache blocks, as a refresh plan's do.  Slots drawn
// one by one, nearer to an eviction's: 116 to 126 us slot-major, whose rows are 256 bytes of codes, and 264 head-major, 64 bytes.
// 2,051 rows take 48 us with the gather behind them; 58 at 128 workgroups, 54 at 256 or 1,024, 62 at 2,048, 50 then at 512.
constexpr int kAngleRows = 4096;         // (row, pair) places in LDS
constexpr int kRerotateGroups = 512;     // workgroups wanted

template <int kStyle>
__global__ __launch_bounds__(256) void kv4_rerotate_kernel(Kv4RerotateParams p) {
  constexpr int N = cs::kKv4Block;
  extern __shared__ __attribute__((aligned(16))) float s_angle[];       // [rows][2 * pairs + 4]: cosine, sine
  const int half = p.head_dim / 2, pitch = 2 * half + 4, tid = threadIdx.x;
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * p.rows_per_block;
  const int rows = static_cast<int>(min(static_cast<int64_t>(p.rows_per_block), p.n_rows - row0));
  for (int i = tid; i < rows * half; i += 256) {
    const int r = i / half, c = i - r * half;
    float cn, sn;
    cs::rope_row<1>(p.rope, row0 + r, c, &cn, &sn);
    *reinterpret_cast<cs::f32v2*>(s_angle + r * pitch + 2 * c) = cs::f32v2{cn, sn};
  }
  __syncthreads();
  const int units_per_row = p.n_kv_heads * p.lanes_per_head;
  const int l_begin = blockIdx.y * p.layers_per_block, l_end = min(p.n_layers, l_begin + p.layers_per_block);
  for (int unit = tid; unit < rows * units_per_row; unit += 256) {
    const int r = unit / units_per_row;
    const int rem = unit - r * units_per_row;
    const int head = rem / p.lanes_per_head;
    const int j = rem - head * p.lanes_per_head;
    const int src = p.src_slot[row0 + r];
    const int dst = p.dst_slot ? p.dst_slot[row0 + r] : src;
    if (src < 0 || dst < 0) continue;
    float cn[N], sn[N];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const cs::u32x4 v = *reinterpret_cast<const cs::u32x4*>(s_angle + r * pitch + 2 * j * N + 4 * i);
      cn[2 * i] = __uint_as_float(v.x);
      sn[2 * i] = __uint_as_float(v.y);
      cn[2 * i + 1] = __uint_as_float(v.z);
      sn[2 * i + 1] = __uint_as_float(v.w);
    }
    // Blocks that nothing turns keep their codes: a sine of 0 would carry what is no number into the partner block.  (A sine of
    // 0 means a cosine of 1: no multiple of pi but 0 is a number of 64 bits.)
    uint32_t sines = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) sines |= cs::abs_bits(sn[i]);
    const bool still = sines == 0;

    const int off_a = kStyle == CS_ROPE_HALF_SPLIT ? j * N : 2 * j * N;
    const int off_b = kStyle == CS_ROPE_HALF_SPLIT ? p.head_dim / 2 + j * N : 2 * j * N + N;
    const int at_a = p.scale_width == 1 ? 0 : 8 * (off_a / N), at_b = p.scale_width == 1 ? 8 : 8 * (off_b / N);
    const int64_t from = static_cast<int64_t>(src) * p.stride_slot + static_cast<int64_t>(head) * p.stride_head;
    const int64_t to = static_cast<int64_t>(dst) * p.stride_slot + static_cast<int64_t>(head) * p.stride_head;
    for (int l = l_begin; l < l_end; ++l) {
      const int64_t s = static_cast<int64_t>(l) * p.stride_layer + from, d = static_cast<int64_t>(l) * p.stride_layer + to;
      const cs::u32x4 wa = *reinterpret_cast<const cs::u32x4*>(p.k_codes + (s + off_a) / 2);
      const cs::u32x4 wb = *reinterpret_cast<const cs::u32x4*>(p.k_codes + (s + off_b) / 2);
      uint32_t ks = 0, vs = 0;           // scale bytes of the head where they are few, else the lane's two
      auto scales = [&](const uint8_t* from_scales) __attribute__((always_inline)) {
        if (p.scale_width == 4) return *reinterpret_cast<const uint32_t*>(from_scales + s / N);
        if (p.scale_width == 2) return static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(from_scales + s / N));
        return static_cast<uint32_t>(from_scales[(s + off_a) / N]) | static_cast<uint32_t>(from_scales[(s + off_b) / N]) << 8;
      };
      ks = scales(p.k_scales);
      const uint32_t ea = ks >> at_a & 0xffu, eb = ks >> at_b & 0xffu;
      cs::u32x4 va, vb;
      if (p.dst_slot) {
        va = *reinterpret_cast<const cs::u32x4*>(p.v_codes + (s + off_a) / 2);
        vb = *reinterpret_cast<const cs::u32x4*>(p.v_codes + (s + off_b) / 2);
        vs = scales(p.v_scales);
      }
      uint32_t na = ea, nb = eb;
      cs::u32x4 oa = wa, ob = wb;
      if (!still) {
        float a[N], b[N];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          cs::kv4_unpack8(wa[i], cs::kv4_scale(ea), a + 8 * i);
          cs::kv4_unpack8(wb[i], cs::kv4_scale(eb), b + 8 * i);
        }
        if (ea == cs::kKv4NoNumber || eb == cs::kKv4NoNumber) {
#pragma unroll
          for (int i = 0; i < N; ++i) {
            if (ea == cs::kKv4NoNumber) a[i] = NAN;
            if (eb == cs::kKv4NoNumber) b[i] = NAN;
          }
        }
        uint32_t ma = 0, mb = 0;
        if (kStyle == CS_ROPE_HALF_SPLIT) {
#pragma unroll
          for (int i = 0; i < N; ++i) cs::rope_turn(a[i], b[i], cn[i], sn[i], &a[i], &b[i]);
        } else {
#pragma unroll
          for (int i = 0; i < N / 2; ++i) {
            cs::rope_turn(a[2 * i], a[2 * i + 1], cn[i], sn[i], &a[2 * i], &a[2 * i + 1]);
            cs::rope_turn(b[2 * i], b[2 * i + 1], cn[N / 2 + i], sn[N / 2 + i], &b[2 * i], &b[2 * i + 1]);
          }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
          ma = max(ma, cs::abs_bits(a[i]));
          mb = max(mb, cs::abs_bits(b[i]));
        }
        na = cs::kv4_scale_byte(ma);
        nb = cs::kv4_scale_byte(mb);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          oa[i] = cs::kv4_pack8(a + 8 * i, cs::kv4_scale(na));
          ob[i] = cs::kv4_pack8(b + 8 * i, cs::kv4_scale(nb));
        }
      }
      *reinterpret_cast<cs::u32x4*>(p.k_codes + (d + off_a) / 2) = oa;
      *reinterpret_cast<cs::u32x4*>(p.k_codes + (d + off_b) / 2) = ob;
      if (p.dst_slot) {
        *reinterpret_cast<cs::u32x4*>(p.v_codes + (d + off_a) / 2) = va;
        *reinterpret_cast<cs::u32x4*>(p.v_codes + (d + off_b) / 2) = vb;
      }
      uint32_t kn = na << at_a | nb << at_b;
      if (p.scale_width == 4) {          // two lanes a head: one writes the keys' scales, one the values'
        kn |= static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(kn), 0xb1, 0xf, 0xf, true));       // lane ^ 1
        if (j == 0 || p.dst_slot) *reinterpret_cast<uint32_t*>((j == 0 ? p.k_scales : p.v_scales) + d / N) = j == 0 ? kn : vs;
      } else if (p.scale_width == 2) {
        *reinterpret_cast<uint16_t*>(p.k_scales + d / N) = static_cast<uint16_t>(kn);
        if (p.dst_slot) *reinterpret_cast<uint16_t*>(p.v_scales + d / N) = static_cast<uint16_t>(vs);
      } else {
        p.k_scales[(d + off_a) / N] = static_cast<uint8_t>(na);
        p.k_scales[(d + off_b) / N] = static_cast<uint8_t>(nb);
        if (p.dst_slot) {
          p.v_scales[(d + off_a) / N] = static_cast<uint8_t>(vs);
          p.v_scales[(d + off_b) / N] = static_cast<uint8_t>(vs >> 8);
        }
      }
    }
  }
}

}  // namespace

extern "C" int cs_rope_refresh_scatter(const void* q, void* q_out, const void* k_new, const void* v_new, const int32_t* slot,
                                       const int32_t* pos, const uint8_t* axis_of_pair, void* k_cache_layer, void* v_cache_layer,
                                       uint8_t* k_scales_layer, uint8_t* v_scales_layer, int64_t n_tok, int32_t n_q_heads,
                                       int32_t n_kv_heads, int32_t head_dim, int64_t stride_q, int64_t stride_k, int64_t stride_v,
                                       int64_t stride_slot, int64_t stride_head, float rope_base, int32_t rope_style,
                                       int32_t dtype, int32_t cache_dtype, void* stream) {
  if (n_tok < 0 || n_q_heads < 0 || n_kv_heads < 0 || n_q_heads + static_cast<int64_t>(n_kv_heads) < 1 || head_dim < 1) return CS_EINVAL;
  if (stride_q < 0 || stride_k < 0 || stride_v < 0 || stride_slot < 0 || stride_head < 0) return CS_EINVAL;
  if (dtype != CS_F32 && dtype != CS_BF16) return CS_EUNSUPPORTED;
  if (rope_style != CS_ROPE_HALF_SPLIT && rope_style != CS_ROPE_INTERLEAVED) return CS_EUNSUPPORTED;
  if (head_dim % 16 != 0 || head_dim > 2 * cs::kRopeMaxPairs) return CS_EUNSUPPORTED;
  if (n_q_heads > 65535 || n_kv_heads > 32767) return CS_EUNSUPPORTED;
  const bool four = cache_dtype == CS_KV4;
  const int elems = dtype == CS_BF16 ? 8 : 4;              // elements per 16-byte vector
  const int64_t q_row = static_cast<int64_t>(n_q_heads) * head_dim, kv_row = static_cast<int64_t>(n_kv_heads) * head_dim;
  if (n_q_heads > 0) {
    if (!pos && n_tok > 0) return CS_EINVAL;               // queries are only turned
    if (stride_q % elems) return CS_EUNSUPPORTED;
    if (n_tok > 1 && stride_q < q_row) return CS_EINVAL;
  }
  if (n_kv_heads > 0) {
    if (!four && cache_dtype != dtype) return CS_EUNSUPPORTED;
    if (four && head_dim % 64) return CS_EUNSUPPORTED;
    if (stride_k % elems || stride_v % elems) return CS_EUNSUPPORTED;
    if (four ? !cs::kv4_strides(stride_slot, stride_head, 0) : (stride_slot % elems || stride_head % elems)) return CS_EUNSUPPORTED;
    if (n_tok > 1 && (stride_k < kv_row || stride_v < kv_row)) return CS_EINVAL;
  }
  if (pos && !(rope_base > 0.0f && rope_base <= 3.0e38f)) return CS_EINVAL;
  if (n_tok == 0) return CS_OK;
  if (n_q_heads > 0) {
    if (!q || !q_out) return CS_EINVAL;
    if (!cs::aligned16(q) || !cs::aligned16(q_out)) return CS_EUNSUPPORTED;
  }
  if (n_kv_heads > 0) {
    if (!k_new || !v_new || !slot || !k_cache_layer || !v_cache_layer) return CS_EINVAL;
    if (four && (!k_scales_layer || !v_scales_layer)) return CS_EINVAL;
    if (!cs::aligned16(k_new) || !cs::aligned16(v_new) || !cs::aligned16(k_cache_layer) || !cs::aligned16(v_cache_layer)) return CS_EUNSUPPORTED;
  }

  RopeWriteParams p;
  cs::rope_angles(&p.rope, pos, axis_of_pair, rope_base, head_dim);
  p.q = q;
  p.q_out = q_out;
  p.k_new = k_new;
  p.v_new = v_new;
  p.slot = slot;
  p.k_cache = k_cache_layer;
  p.v_cache = v_cache_layer;
  p.k_scales = k_scales_layer;
  p.v_scales = v_scales_layer;
  p.n_tok = n_tok;
  p.stride_q = stride_q;
  p.stride_q_out = q_out == q ? stride_q : q_row;
  p.stride_k = stride_k;
  p.stride_v = stride_v;
  p.stride_slot = stride_slot;
  p.stride_head = stride_head;
  p.n_q_heads = n_q_heads;
  p.n_kv_heads = n_kv_heads;
  p.head_dim = head_dim;
  p.lanes_per_tok = head_dim / 2 / kPairs;
  if (n_tok > (cs::kMostThreads - 255) / p.lanes_per_tok) return CS_EUNSUPPORTED;
  const int64_t blocks_x = (n_tok * p.lanes_per_tok + 255) / 256;
  // Heads a thread turns with one evaluation of its angles: all of them where the tokens alone fill the card, fewer below (shares: at
  // most kRopeGroups, along the grid's second axis).
  const int heads = n_q_heads + 2 * n_kv_heads;
  const int64_t shares = blocks_x >= kRopeGroups ? 1 : (kRopeGroups + blocks_x - 1) / blocks_x;
  p.heads_per_thread = static_cast<int32_t>(shares >= heads ? 1 : (heads + shares - 1) / shares);
  while (p.heads_per_thread < kRopeHeads && blocks_x * ((heads + p.heads_per_thread) / (p.heads_per_thread + 1)) >= kRopeEnough) ++p.heads_per_thread;
  const dim3 grid(static_cast<unsigned>(blocks_x), static_cast<unsigned>((heads + p.heads_per_thread - 1) / p.heads_per_thread));
  hipStream_t st = cs::as_stream(stream);
  const bool half_split = rope_style == CS_ROPE_HALF_SPLIT, bf16 = dtype == CS_BF16;
#define CS_LAUNCH_ROPE(BF16, STYLE)                                                                          \
  do {                                                                                                       \
    if (four) hipLaunchKernelGGL((rope_write_kernel<BF16, STYLE, true>), grid, dim3(256), 0, st, p);         \
    else hipLaunchKernelGGL((rope_write_kernel<BF16, STYLE, false>), grid, dim3(256), 0, st, p);             \
  } while (0)
  if (bf16 && half_split) CS_LAUNCH_ROPE(true, CS_ROPE_HALF_SPLIT);
  else if (bf16) CS_LAUNCH_ROPE(true, CS_ROPE_INTERLEAVED);
  else if (half_split) CS_LAUNCH_ROPE(false, CS_ROPE_HALF_SPLIT);
  else CS_LAUNCH_ROPE(false, CS_ROPE_INTERLEAVED);
#undef CS_LAUNCH_ROPE
  return cs::note_hip(hipGetLastError());
}

extern "C" int cs_kv4_gather(const uint8_t* k_codes, const uint8_t* k_scales, const uint8_t* v_codes, const uint8_t* v_scales,
                             const int32_t* slot, int64_t n_rows, int32_t n_layers, int32_t n_kv_heads, int32_t head_dim,
                             int64_t stride_layer, int64_t stride_slot, int64_t stride_head, void* k_out, void* v_out,
                             int32_t dtype, void* stream) {
  if (n_rows < 0 || n_layers < 0 || n_kv_heads < 1 || head_dim < 1) return CS_EINVAL;
  if (stride_layer < 0 || stride_slot < 0 || stride_head < 0) return CS_EINVAL;
  if (dtype != CS_F32 && dtype != CS_BF16) return CS_EUNSUPPORTED;
  if (head_dim % 64 || head_dim > 2 * cs::kRopeMaxPairs || !cs::kv4_strides(stride_layer, stride_slot, stride_head)) return CS_EUNSUPPORTED;
  if (n_rows == 0 || n_layers == 0) return CS_OK;
  if (!slot || (!k_out && !v_out)) return CS_EINVAL;
  if (k_out && (!k_codes || !k_scales)) return CS_EINVAL;
  if (v_out && (!v_codes || !v_scales)) return CS_EINVAL;
  if (!cs::aligned16(k_out) || !cs::aligned16(v_out) || !cs::aligned16(k_out ? k_codes : nullptr) || !cs::aligned16(v_out ? v_codes : nullptr))
    return CS_EUNSUPPORTED;
  GatherParams p;
  int n = 0;
  if (k_out) {
    p.codes[n] = k_codes;
    p.scales[n] = k_scales;
    p.out[n++] = k_out;
  }
  if (v_out) {
    p.codes[n] = v_codes;
    p.scales[n] = v_scales;
    p.out[n++] = v_out;
  }
  p.slot = slot;
  p.n_rows = n_rows;
  p.stride_layer = stride_layer;
  p.stride_slot = stride_slot;
  p.stride_head = stride_head;
  p.n_kv_heads = n_kv_heads;
  p.lanes_per_head = head_dim / 8;
  if (n_rows > (cs::kMostThreads - 255) / n_layers / n_kv_heads / p.lanes_per_head) return CS_EUNSUPPORTED;
  p.n_units = n_rows * n_layers * n_kv_heads * p.lanes_per_head;
  const int64_t blocks = (p.n_units + 255) / 256;
  const dim3 grid(static_cast<unsigned>(blocks), n);
  if (dtype == CS_BF16) hipLaunchKernelGGL(kv4_gather_kernel<true>, grid, dim3(256), 0, cs::as_stream(stream), p);
  else hipLaunchKernelGGL(kv4_gather_kernel<false>, grid, dim3(256), 0, cs::as_stream(stream), p);
  return cs::note_hip(hipGetLastError());
}

extern "C" int cs_kv4_rerotate(uint8_t* k_codes, uint8_t* k_scales, uint8_t* v_codes, uint8_t* v_scales, const int32_t* src_slot,
                               const int32_t* dst_slot, const int32_t* delta, const uint8_t* axis_of_pair, int64_t n_rows,
                               int32_t n_layers, int32_t n_kv_heads, int32_t head_dim, int64_t stride_layer, int64_t stride_slot,
                               int64_t stride_head, float rope_base, int32_t rope_style, void* stream) {
  if (n_rows < 0 || n_layers < 0 || n_kv_heads < 1 || head_dim < 1) return CS_EINVAL;
  if (stride_layer < 0 || stride_slot < 0 || stride_head < 0) return CS_EINVAL;
  if (!(rope_base > 0.0f && rope_base <= 3.0e38f)) return CS_EINVAL;
  if (rope_style != CS_ROPE_HALF_SPLIT && rope_style != CS_ROPE_INTERLEAVED) return CS_EUNSUPPORTED;
  if (head_dim % 64 || head_dim > 2 * cs::kRopeMaxPairs || !cs::kv4_strides(stride_layer, stride_slot, stride_head)) return CS_EUNSUPPORTED;
  if (n_rows == 0 || n_layers == 0) return CS_OK;
  if (!k_codes || !k_scales || !src_slot || !delta) return CS_EINVAL;
  if (dst_slot && (!v_codes || !v_scales)) return CS_EINVAL;
  if (!cs::aligned16(k_codes) || (dst_slot && !cs::aligned16(v_codes))) return CS_EUNSUPPORTED;
  Kv4RerotateParams p;
  cs::rope_angles(&p.rope, delta, axis_of_pair, rope_base, head_dim);
  p.k_codes = k_codes;
  p.k_scales = k_scales;
  p.v_codes = v_codes;
  p.v_scales = v_scales;
  p.src_slot = src_slot;
  p.dst_slot = dst_slot;
  p.n_rows = n_rows;
  p.stride_layer = stride_layer;
  p.stride_slot = stride_slot;
  p.stride_head = stride_head;
  p.n_layers = n_layers;
  p.n_kv_heads = n_kv_heads;
  p.head_dim = head_dim;
  p.lanes_per_head = head_dim / 64;
  // Scale bytes move as one word a row and head where they lie as one (head_dim 64 and 128): 15,023 rows of 28 layers,
  // 4 heads of 128 each, in slots drawn one by one, take 265 us head-major and 120 us slot-major, with single bytes 297 and 125.
  const int64_t strides = stride_layer | stride_slot | stride_head;
  const uintptr_t scales = reinterpret_cast<uintptr_t>(k_scales) | (dst_slot ? reinterpret_cast<uintptr_t>(v_scales) : 0);
  const int width = 2 * p.lanes_per_head;
  p.scale_width = width <= 4 && strides / cs::kKv4Block % width == 0 && scales % width == 0 ? width : 1;
  const int units = n_kv_heads * p.lanes_per_head, places = kAngleRows / (head_dim / 2);
  p.rows_per_block = units >= 256 ? 1 : 256 / units < places ? 256 / units : places;
  if (n_rows > cs::kMostThreads / 256 * p.rows_per_block) return CS_EUNSUPPORTED;
  const int64_t blocks_x = (n_rows + p.rows_per_block - 1) / p.rows_per_block;
  // Layers of a workgroup: all of them where the rows alone fill the card.
  const int64_t shares = blocks_x >= kRerotateGroups ? 1 : (kRerotateGroups + blocks_x - 1) / blocks_x;
  p.layers_per_block = static_cast<int32_t>(shares >= n_layers ? 1 : (n_layers + shares - 1) / shares);
  const int64_t blocks_y = (n_layers + p.layers_per_block - 1) / p.layers_per_block;
  if (blocks_y > 65535) return CS_EUNSUPPORTED;
  const dim3 grid(static_cast<unsigned>(blocks_x), static_cast<unsigned>(blocks_y));
  const size_t lds = static_cast<size_t>(p.rows_per_block) * (head_dim + 4) * sizeof(float);
  if (rope_style == CS_ROPE_HALF_SPLIT) hipLaunchKernelGGL(kv4_rerotate_kernel<CS_ROPE_HALF_SPLIT>, grid, dim3(256), lds, cs::as_stream(stream), p);
  else hipLaunchKernelGGL(kv4_rerotate_kernel<CS_ROPE_INTERLEAVED>, grid, dim3(256), lds, cs::as_stream(stream), p);
  return cs::note_hip(hipGetLastError());
}
