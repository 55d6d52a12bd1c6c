// Fresh tokens of a layer on their way into the window cache: queries and keys normed head by head and rotated, in one pass with
// the refresh write.
//
//     y = w x / sqrt(mean(x^2) + eps)           over a head's d elements
//     (a, b) -> (a c - b s, b c + a s)          for the pairs of the first `rotary_dim` elements, c, s = amplitude * cos, sin(pos f_i)
//
// A lane owns 16 elements of a token's heads: eight pairs of the rotated part (8 and 8 elements, half a rotated part apart or
// neighbours), or 16 neighbours past it.  It evaluates its cosines and sines once (double precision) and keeps them for every head of
// its share; a head's lanes lie in one row of 16 of the wave, so the sum of squares is up to four lane exchanges, and nothing passes through
// LDS.  Bound by memory: 22,804 tokens of 32 + 8 heads of 128 take 127 us, 4.4 TB/s (a large copy: 5.1),
// in fp32 262 us, 4.3 TB/s; one token of 28 + 4 heads 4.4 us.
#include <math.h>

#include <type_traits>

#include "rope.h"
#include "vec8.h"

namespace {

using cs::Eight;

constexpr int kPairs = 8;                // pairs a lane owns
// Workgroups wanted, heads a thread takes with one evaluation of its angles even so, and workgroups enough: as the write without norms.
constexpr int kGroups = 4096, kHeads = 4, kEnough = 512;

struct NormRopeParams {
  const void* q;
  void* q_out;                           // may be q
  const void* __restrict__ k_new;
  const void* __restrict__ v_new;
  const void* __restrict__ q_weight;     // [head_dim], nullptr: not normed
  const void* __restrict__ k_weight;
  const int32_t* __restrict__ slot;
  const int32_t* __restrict__ pos;       // [n_tok], or [n_tok][3] with axis_of_pair; nullptr: not rotated
  const uint8_t* __restrict__ axis_of_pair;
  const float* __restrict__ inv_freq;    // [rotary_dim / 2]
  void* __restrict__ k_cache;
  void* __restrict__ v_cache;
  int64_t n_tok, stride_q, stride_q_out, stride_k, stride_v, stride_slot, stride_head;
  int32_t n_q_heads, n_kv_heads, head_dim, rotary_dim, lanes_per_tok, heads_per_thread;      // lanes_per_tok: a power of two, 16 at most
  float eps, amplitude;
};

// Sum over the lanes of a token: aligned groups of 1, 2, 4, 8 or 16.
__device__ __forceinline__ float token_sum(float x, int lanes) {
  const auto add = [&](auto ctrl) __attribute__((always_inline)) {
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  if (lanes > 1) add(std::integral_constant<int, 0xb1>());       // lane ^ 1
  if (lanes > 2) add(std::integral_constant<int, 0x4e>());       // lane ^ 2
  if (lanes > 4) add(std::integral_constant<int, 0x141>());      // 7 - lane of eight: the other four's sum
  if (lanes > 8) add(std::integral_constant<int, 0x140>());      // 15 - lane of sixteen: the other eight's
  return x;
}

// Grid: x over (token, lane of the token), y over shares of the n_q_heads + 2 n_kv_heads heads of a token (queries, keys, values).
template <bool kBf16, int kStyle>
__global__ __launch_bounds__(256) void norm_rope_write_kernel(NormRopeParams p) {
  using Elem = typename std::conditional<kBf16, uint16_t, float>::type;
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  const int64_t tok = unit / p.lanes_per_tok;
  if (tok >= p.n_tok) return;            // (whole tokens: the lanes of a head leave together)
  const int j = static_cast<int>(unit) & (p.lanes_per_tok - 1);
  const bool mine = j < p.head_dim / 16;                          // (head_dim / 16 need not be a power of two)
  const bool rotated = j < p.rotary_dim / 16;
  const bool apart = kStyle == CS_ROPE_HALF_SPLIT && rotated;
  const int off_a = apart ? j * kPairs : 2 * j * kPairs;
  const int off_b = apart ? p.rotary_dim / 2 + j * kPairs : 2 * j * kPairs + kPairs;
  const int h_begin = blockIdx.y * p.heads_per_thread;
  const int h_end = min(p.n_q_heads + 2 * p.n_kv_heads, h_begin + p.heads_per_thread);
  const int first_v = p.n_q_heads + p.n_kv_heads;
  const int slot = h_end > p.n_q_heads ? p.slot[tok] : -1;

  float cn[kPairs], sn[kPairs];
  const bool turned = p.pos != nullptr && rotated && h_begin < first_v;
  if (turned) {
    const int64_t at = p.axis_of_pair ? 3 * tok : tok;
    const int p0 = p.pos[at], p1 = p.axis_of_pair ? p.pos[at + 1] : p0, p2 = p.axis_of_pair ? p.pos[at + 2] : p0;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const int axis = p.axis_of_pair ? p.axis_of_pair[j * kPairs + i] : 0;
      const int at_pos = axis == 0 ? p0 : axis == 1 ? p1 : p2;
      cs::sincos_rounded(static_cast<double>(at_pos) * static_cast<double>(p.inv_freq[j * kPairs + i]), &sn[i], &cn[i]);
      cn[i] *= p.amplitude;
      sn[i] *= p.amplitude;
    }
  }
  // weights of the kind of head at hand (queries first)
  float wa[kPairs], wb[kPairs];
  int held = -1;                         // 0: queries', 1: keys'
  const float share = 1.0f / static_cast<float>(p.head_dim);

  constexpr int kBatch = kBf16 ? 4 : 2;
  for (int h0 = h_begin; h0 < h_end; h0 += kBatch) {
    Eight<kBf16> a[kBatch], b[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int h = h0 + i;
      if (mine && h < h_end && (h < p.n_q_heads || slot >= 0)) {
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
      if (!(h < h_end && (h < p.n_q_heads || slot >= 0))) continue;        // (the same for all lanes of a token)
      if (h >= first_v) {                // (as they are: a conversion would make a signalling NaN a quiet one)
        if (mine) {
          Elem* dst = static_cast<Elem*>(p.v_cache) + static_cast<int64_t>(slot) * p.stride_slot + static_cast<int64_t>(h - first_v) * p.stride_head;
          a[i].copy_to(dst + off_a);
          b[i].copy_to(dst + off_b);
        }
        continue;
      }
      float fa[kPairs], fb[kPairs];
      a[i].get(fa);
      b[i].get(fb);
      const void* weight = h < p.n_q_heads ? p.q_weight : p.k_weight;
      if (weight) {
        const int kind = h < p.n_q_heads ? 0 : 1;
        if (held != kind && mine) {
          Eight<kBf16> w;
          w.load(static_cast<const Elem*>(weight) + off_a);
          w.get(wa);
          w.load(static_cast<const Elem*>(weight) + off_b);
          w.get(wb);
        }
        held = kind;
        float ss = 0.0f;
#pragma unroll
        for (int e = 0; e < kPairs; ++e) ss = fmaf(fa[e], fa[e], fmaf(fb[e], fb[e], ss));
        ss = token_sum(mine ? ss : 0.0f, p.lanes_per_tok);
        float eps = p.eps;
        if (__builtin_expect(!(ss < INFINITY), 0)) {
          // squares past the largest number (or what is none): the same with all elements 2^-70 times as large, and eps with their squares
          eps *= 0x1p-140f;
          ss = 0.0f;
#pragma unroll
          for (int e = 0; e < kPairs; ++e) {
            fa[e] *= 0x1p-70f;
            fb[e] *= 0x1p-70f;
            ss = fmaf(fa[e], fa[e], fmaf(fb[e], fb[e], ss));
          }
          ss = token_sum(mine ? ss : 0.0f, p.lanes_per_tok);
        }
        const float r = __builtin_amdgcn_rsqf(fmaf(ss, share, eps));
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
          fa[e] = fa[e] * r * wa[e];
          fb[e] = fb[e] * r * wb[e];
        }
      }
      if (turned) {
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
      if (!mine) continue;
      Elem* dst;
      if (h < p.n_q_heads) {
        dst = static_cast<Elem*>(p.q_out) + tok * p.stride_q_out + static_cast<int64_t>(h) * p.head_dim;
      } else {
        dst = static_cast<Elem*>(p.k_cache) + static_cast<int64_t>(slot) * p.stride_slot + static_cast<int64_t>(h - p.n_q_heads) * p.stride_head;
      }
      Eight<kBf16>::store(dst + off_a, fa);
      Eight<kBf16>::store(dst + off_b, fb);
    }
  }
}

}  // namespace

extern "C" int cs_norm_rope_refresh_scatter(const void* q, void* q_out, const void* k_new, const void* v_new, const void* q_weight,
                                            const void* k_weight, const int32_t* slot, const int32_t* pos, const uint8_t* axis_of_pair,
                                            const float* inv_freq, void* k_cache_layer, void* v_cache_layer, int64_t n_tok, int32_t n_q_heads,
                                            int32_t n_kv_heads, int32_t head_dim, int32_t rotary_dim, int64_t stride_q, int64_t stride_k,
                                            int64_t stride_v, int64_t stride_slot, int64_t stride_head, float norm_eps, float amplitude,
                                            int32_t rope_style, int32_t dtype, void* stream) {
  if (n_tok < 0 || n_q_heads < 0 || n_kv_heads < 0 || n_q_heads + static_cast<int64_t>(n_kv_heads) < 1 || head_dim < 1) return CS_EINVAL;
  if (stride_q < 0 || stride_k < 0 || stride_v < 0 || stride_slot < 0 || stride_head < 0) return CS_EINVAL;
  if (rotary_dim < 0 || rotary_dim > head_dim) return CS_EINVAL;
  if (dtype != CS_F32 && dtype != CS_BF16) return CS_EUNSUPPORTED;
  if (rope_style != CS_ROPE_HALF_SPLIT && rope_style != CS_ROPE_INTERLEAVED) return CS_EUNSUPPORTED;
  if (head_dim % 16 != 0 || head_dim > 2 * cs::kRopeMaxPairs || rotary_dim % 16 != 0) return CS_EUNSUPPORTED;
  if (n_q_heads > 65535 || n_kv_heads > 32767) return CS_EUNSUPPORTED;
  const int elems = dtype == CS_BF16 ? 8 : 4;              // elements per 16-byte vector
  const int64_t q_row = static_cast<int64_t>(n_q_heads) * head_dim, kv_row = static_cast<int64_t>(n_kv_heads) * head_dim;
  if (n_q_heads > 0) {
    if (stride_q % elems) return CS_EUNSUPPORTED;
    if (n_tok > 1 && stride_q < q_row) return CS_EINVAL;
  }
  if (n_kv_heads > 0) {
    if (stride_k % elems || stride_v % elems || stride_slot % elems || stride_head % elems) return CS_EUNSUPPORTED;
    if (n_tok > 1 && (stride_k < kv_row || stride_v < kv_row)) return CS_EINVAL;
  }
  // (the least eps: squares below the smallest number are then nothing beside it)
  if ((q_weight || k_weight) && !(norm_eps >= 1e-30f && norm_eps <= 3.0e38f)) return CS_EINVAL;
  if (pos && !(amplitude >= -3.0e38f && amplitude <= 3.0e38f)) return CS_EINVAL;
  if (n_tok == 0) return CS_OK;
  if (pos && rotary_dim > 0 && !inv_freq) return CS_EINVAL;
  if (n_q_heads > 0) {
    if (!q || !q_out) return CS_EINVAL;
    if (!cs::aligned16(q) || !cs::aligned16(q_out) || !cs::aligned16(q_weight)) return CS_EUNSUPPORTED;
  }
  if (n_kv_heads > 0) {
    if (!k_new || !v_new || !slot || !k_cache_layer || !v_cache_layer) return CS_EINVAL;
    if (!cs::aligned16(k_new) || !cs::aligned16(v_new) || !cs::aligned16(k_weight) || !cs::aligned16(k_cache_layer) || !cs::aligned16(v_cache_layer))
      return CS_EUNSUPPORTED;
  }

  NormRopeParams p;
  p.q = q;
  p.q_out = q_out;
  p.k_new = k_new;
  p.v_new = v_new;
  p.q_weight = q_weight;
  p.k_weight = k_weight;
  p.slot = slot;
  p.pos = pos;
  p.axis_of_pair = axis_of_pair;
  p.inv_freq = inv_freq;
  p.k_cache = k_cache_layer;
  p.v_cache = v_cache_layer;
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
  p.rotary_dim = rotary_dim;
  p.eps = norm_eps;
  p.amplitude = amplitude;
  p.lanes_per_tok = 1;
  while (p.lanes_per_tok < head_dim / 16) p.lanes_per_tok *= 2;
  if (n_tok > (cs::kMostThreads - 255) / p.lanes_per_tok) return CS_EUNSUPPORTED;
  const int64_t blocks_x = (n_tok * p.lanes_per_tok + 255) / 256;
  const int heads = n_q_heads + 2 * n_kv_heads;
  const int64_t shares = blocks_x >= kGroups ? 1 : (kGroups + blocks_x - 1) / blocks_x;
  p.heads_per_thread = static_cast<int32_t>(shares >= heads ? 1 : (heads + shares - 1) / shares);
  while (p.heads_per_thread < kHeads && blocks_x * ((heads + p.heads_per_thread) / (p.heads_per_thread + 1)) >= kEnough) ++p.heads_per_thread;
  const dim3 grid(static_cast<unsigned>(blocks_x), static_cast<unsigned>((heads + p.heads_per_thread - 1) / p.heads_per_thread));
  hipStream_t st = cs::as_stream(stream);
  const bool half_split = rope_style == CS_ROPE_HALF_SPLIT, bf16 = dtype == CS_BF16;
  if (bf16 && half_split) hipLaunchKernelGGL((norm_rope_write_kernel<true, CS_ROPE_HALF_SPLIT>), grid, dim3(256), 0, st, p);
  else if (bf16) hipLaunchKernelGGL((norm_rope_write_kernel<true, CS_ROPE_INTERLEAVED>), grid, dim3(256), 0, st, p);
  else if (half_split) hipLaunchKernelGGL((norm_rope_write_kernel<false, CS_ROPE_HALF_SPLIT>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((norm_rope_write_kernel<false, CS_ROPE_INTERLEAVED>), grid, dim3(256), 0, st, p);
  return cs::note_hip(hipGetLastError());
}
