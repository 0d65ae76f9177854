// rope_kernels.hip -- rotary positions of queries and keys, and the append that
// applies them on the way into the cache (gfx950).
//
// Pair i of the first rot_dim channels of a head, (a, b), turns by the angle
// t = pos[axis[i]] freq[i]:
//     a' = a cos t - b sin t,   b' = b cos t + a sin t,
// both times the rotation's magnitude; the channels past rot_dim stay.  The
// angle is taken in turns, pos x (freq / 2 pi), as one fp64 product whose nearest
// whole number is dropped, so that a position of 2^31 still has its angle to
// 2^-22 of a turn and near ones to fp32's last place; sine and cosine, and the
// products, are fp32; one rounding to bf16 at the end.  The compiler contracts
// nothing here by itself, so that both kernels turn a pair to the same bits.
//
// A lane holds 16 channels of a head: 8 pairs, which are chunks c and
// c + rot_dim / 16 (halves) or 2c and 2c + 1 (adjacent pairs) of 8 channels.
#include <algorithm>

#include "hwkv_internal.h"
#include "kv_format.h"
#include "kv_rows8.h"

namespace hwkv {
namespace {

struct Turn {
  float cos[8], sin[8];
};

// Cosines and sines of pairs 8c .. 8c + 7 at the token's positions.
__device__ __forceinline__ Turn turns_of(const RopeTable &t, const int32_t *pos, int64_t stride, int c) {
  Turn r;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma clang fp contract(off)
    const double x = (double)pos[t.axis[8 * c + i] * stride] * t.turns[8 * c + i];
    const float f = 2.0f * (float)(x - __builtin_rint(x));
    sincospif(f, &r.sin[i], &r.cos[i]);
    r.sin[i] *= t.magnitude;
    r.cos[i] *= t.magnitude;
  }
  return r;
}

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{lo, hi}, b2));
}

__device__ __forceinline__ float half_of(uint4 x, int i) {
  const uint32_t w = i < 2 ? x.x : i < 4 ? x.y : i < 6 ? x.z : x.w;
  return bf16_bits_to_f32(i & 1 ? w >> 16 : w & 0xffffu);
}

// The lane's two chunks x, y turned.
__device__ __forceinline__ void turn(const Turn &t, bool halves, uint4 &x, uint4 &y) {
  float a[8], b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    // halves: pair i is element i of both chunks; pairs: 2i and 2i + 1 of x | y
    const float u = halves ? half_of(x, i) : half_of(i < 4 ? x : y, 2 * i % 8);
    const float v = halves ? half_of(y, i) : half_of(i < 4 ? x : y, 2 * i % 8 + 1);
    a[i] = fmaf(u, t.cos[i], -__fmul_rn(v, t.sin[i]));
    b[i] = fmaf(v, t.cos[i], __fmul_rn(u, t.sin[i]));
  }
  if (halves) {
    x = make_uint4(bf16_pair(a[0], a[1]), bf16_pair(a[2], a[3]), bf16_pair(a[4], a[5]), bf16_pair(a[6], a[7]));
    y = make_uint4(bf16_pair(b[0], b[1]), bf16_pair(b[2], b[3]), bf16_pair(b[4], b[5]), bf16_pair(b[6], b[7]));
  } else {
    x = make_uint4(bf16_pair(a[0], b[0]), bf16_pair(a[1], b[1]), bf16_pair(a[2], b[2]), bf16_pair(a[3], b[3]));
    y = make_uint4(bf16_pair(a[4], b[4]), bf16_pair(a[5], b[5]), bf16_pair(a[6], b[6]), bf16_pair(a[7], b[7]));
  }
}

// First channels of the lane's two chunks (lane c of a head's D / 16).
struct Chunks {
  int x, y;
};
__device__ __forceinline__ Chunks chunks_of(const RopeTable &t, int c) {
  const int n = t.rot_dim / 16;
  if (c < n && t.pairs == HWKV_ROPE_HALF) return {8 * c, 8 * (c + n)};
  return {16 * c, 16 * c + 8};
}

template <int D>
__global__ __launch_bounds__(256) void rope(RopeArgs a) {
  constexpr int NL = D / 16;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t tok = i / NL;
  const int c = (int)(i % NL);
  if (tok >= a.n) return;
  const Chunks ch = chunks_of(a.rope, c);
  const bool turns = c < a.rope.rot_dim / 16, halves = a.rope.pairs == HWKV_ROPE_HALF;
  Turn t;
  if (turns) t = turns_of(a.rope, a.pos + tok, a.n, c);
  const int h1 = min(a.n_q + a.n_k, (int)(blockIdx.y + 1) * a.heads_per);
  for (int h = blockIdx.y * a.heads_per; h < h1; ++h) {
    const bool isq = h < a.n_q;
    const int hh = isq ? h : h - a.n_q;
    const uint16_t *from = isq ? a.q + tok * a.q_stride : a.k + tok * a.k_stride;
    uint16_t *to = isq ? a.q_out + tok * a.n_q * D : a.k_out + tok * a.n_k * D;
    from += hh * D;
    to += hh * D;
    uint4 x = *reinterpret_cast<const uint4 *>(from + ch.x);
    uint4 y = *reinterpret_cast<const uint4 *>(from + ch.y);
    if (turns) turn(t, halves, x, y);
    *reinterpret_cast<uint4 *>(to + ch.x) = x;
    *reinterpret_cast<uint4 *>(to + ch.y) = y;
  }
}

// D / 16 lanes for each row of a sequence: its q heads, then k, then v.
template <int D, int F>
__global__ __launch_bounds__(256) void append_rope(AppendRopeArgs a) {
  constexpr int NL = D / 16;
  constexpr int EB = KvFormat<F>::kBytes;
  constexpr int LB = 8 * EB;
  const int rows = a.n_heads * (a.group + 2);
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int c = (int)(i % NL);
  const int b = (int)(i / NL / rows), row = (int)(i / NL % rows);
  if (b >= a.n_seqs) return;
  const int nq = a.n_heads * a.group;
  const bool isq = row < nq, isk = !isq && row < nq + a.n_heads;
  const int h = isq ? row : isk ? row - nq : row - nq - a.n_heads;
  const uint16_t *from = isq ? a.q + b * a.q_stride : isk ? a.k + b * a.k_stride : a.v + b * a.v_stride;
  from += h * D;
  const bool turns = (isq || isk) && c < a.rope.rot_dim / 16;
  const Chunks ch = isq || isk ? chunks_of(a.rope, c) : Chunks{16 * c, 16 * c + 8};
  uint4 x = *reinterpret_cast<const uint4 *>(from + ch.x);
  uint4 y = *reinterpret_cast<const uint4 *>(from + ch.y);
  if (turns) turn(turns_of(a.rope, a.pos + b, a.pos_stride, c), a.rope.pairs == HWKV_ROPE_HALF, x, y);
  if (isq) {
    uint16_t *to = a.q_out + b * a.q_out_stride + h * D;
    *reinterpret_cast<uint4 *>(to + ch.x) = x;
    *reinterpret_cast<uint4 *>(to + ch.y) = y;
    return;
  }
  // the row's place in the cache
  const ItemHead &hd = a.head[h];
  const int pos = a.len[b];
  const int slot = hd.window == 0 || pos < a.n_sinks ? pos : a.n_sinks + (pos - a.n_sinks) % hd.window;
  uint8_t *const cache = static_cast<uint8_t *>(a.cache);
  int64_t at, soff = 0;      // first element of the K tiles or V rows; the scale pairs
  int r = slot;
  if (hd.page0 >= 0) {
    const int64_t pg = a.page_table[hd.page0 + b * a.max_pages + slot / kPageTokens];
    const int64_t base = a.pool_off + pg * page_elems<F>(D);
    at = base + (isk ? 0 : kPageTokens * D);
    soff = base + 2 * kPageTokens * D;
    r = slot % kPageTokens;
  } else {
    at = (isk ? hd.k_off : hd.v_off) + (int64_t)b * hd.cap_pad * D;
    if constexpr (F == HWKV_KV_I8) soff = (int64_t)hd.s_off128 * 128 + (int64_t)b * hd.cap_pad * kRowScaleBytes;
  }
  uint8_t *const to = cache + (at + (isk ? (int64_t)(r / kTile) * kTile * D : (int64_t)r * D)) * EB;
  uint32_t e = 0;
  if constexpr (F == HWKV_KV_I8) {
    e = row_scale(group_max<NL>(max(top8(x), top8(y))));
    if (c == 0) cache[soff + (int64_t)r * kRowScaleBytes + (isk ? 0 : 1)] = (uint8_t)e;
  }
  auto put = [&](int first, uint4 w) {
    typename KvFormat<F>::Chunk code;
    if constexpr (F == HWKV_KV_I8)
      code = encode8_row(w, e);
    else
      code = encode8<F>(w, isk ? hd.k_scale : hd.v_scale);
    const int g = first / 8;
    store_chunk<F>(to + (isk ? (g * kTile + r % kTile) * LB : g * LB), code);
  };
  put(ch.x, x);
  put(ch.y, y);
}

template <int D>
hipError_t launch_rope_d(const RopeArgs &a, hipStream_t s) {
  constexpr int NL = D / 16;
  const int heads = a.n_q + a.n_k;
  const dim3 grid((unsigned)((a.n * NL + 255) / 256), (unsigned)((heads + a.heads_per - 1) / a.heads_per));
  hipLaunchKernelGGL(rope<D>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

template <int D, int F>
hipError_t launch_append_rope_df(const AppendRopeArgs &a, hipStream_t s) {
  const int64_t lanes = (int64_t)a.n_seqs * a.n_heads * (a.group + 2) * (D / 16);
  hipLaunchKernelGGL((append_rope<D, F>), dim3((unsigned)((lanes + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_append_rope_d(int fmt, const AppendRopeArgs &a, hipStream_t s) {
  switch (fmt) {
    case HWKV_KV_BF16: return launch_append_rope_df<D, HWKV_KV_BF16>(a, s);
    case HWKV_KV_F16: return launch_append_rope_df<D, HWKV_KV_F16>(a, s);
    case HWKV_KV_FP8_E4M3: return launch_append_rope_df<D, HWKV_KV_FP8_E4M3>(a, s);
    case HWKV_KV_I8: return launch_append_rope_df<D, HWKV_KV_I8>(a, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t launch_rope(int D, const RopeArgs &a, hipStream_t s) {
  switch (D) {
    case 64: return launch_rope_d<64>(a, s);
    case 128: return launch_rope_d<128>(a, s);
    case 256: return launch_rope_d<256>(a, s);
    default: return hipErrorInvalidValue;
  }
}

hipError_t launch_append_rope(int fmt, int D, const AppendRopeArgs &a, hipStream_t s) {
  switch (D) {
    case 64: return launch_append_rope_d<64>(fmt, a, s);
    case 128: return launch_append_rope_d<128>(fmt, a, s);
    case 256: return launch_append_rope_d<256>(fmt, a, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace hwkv
