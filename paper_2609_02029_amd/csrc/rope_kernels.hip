// rope_kernels.hip -- rotary positions of queries and keys, and the append that
// applies them on the way into the cache (gfx950).
//
// Pair i of the first rot_dim channels of a head, (a, b), turns by the angle
// t = pos[axis[i]] freq[i]:
//     a' = a cos t - b sin t,   b' = b cos t + a sin t,
// both times the rotation's magnitude; the channels past rot_dim stay.  The
// angle is taken in turns, pos x (freq / 2 pi), with freq / 2 pi as a double and
// the float that it leaves (2^-77 of it), and the product as an fp64 one, whose
// nearest whole number is dropped, and its own rest: up to 2^49 turns (a position
// of 2^31 at a frequency of 10^6) the fraction has fp32's last place.  (The fp64
// product alone is off by 2^-23 turns at 2^31 x 3 radians, 2^-4 at 2^31 x 10^6.)
// Sine and cosine, and the products, are fp32; one rounding to bf16 at the end.
// The compiler contracts nothing here by itself, so that both kernels turn a pair
// to the same bits.
//
// A lane holds 16 channels of a head: 8 pairs, which are chunks c and
// c + rot_dim / 16 (halves) or 2c and 2c + 1 (adjacent pairs) of 8 channels.
#include <algorithm>

#include "hwkv_internal.h"
#include "kv_format.h"
#include "kv_rows8.h"

namespace hwkv {
namespace {

typedef unsigned int u4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint4 chunk(u4 x) { return make_uint4(x.x, x.y, x.z, x.w); }

// Cosine and sine of pair p at the token's positions.
__device__ __forceinline__ void cos_sin(const RopeTable &t, const int32_t *pos, int64_t stride, int p,
                                        float *c, float *s) {
#pragma clang fp contract(off)
  const double at = pos[t.axis[p] * stride], x = at * t.turns[p];
  const double rest = __builtin_fma(at, t.turns[p], -x) + at * (double)t.turns_low[p];
  const float f = 2.0f * (float)((x - __builtin_rint(x)) + rest);
  float sn, cn;
  sincospif(f, &sn, &cn);
  *s = sn * t.magnitude;
  *c = cn * t.magnitude;
}

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{lo, hi}, b2));
}

__device__ __forceinline__ float half_of(u4 x, int i) {
  return bf16_bits_to_f32(i & 1 ? x[i / 2] >> 16 : x[i / 2] & 0xffffu);
}

// The lane's two chunks x, y turned by the cosines and sines of its 8 pairs.
__device__ __forceinline__ void turn(const float *cos, const float *sin, bool halves, u4 &x, u4 &y) {
  float a[8], b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    // halves: pair i is element i of both chunks; pairs: 2i and 2i + 1 of x | y
    const float u = halves ? half_of(x, i) : half_of(i < 4 ? x : y, 2 * i % 8);
    const float v = halves ? half_of(y, i) : half_of(i < 4 ? x : y, 2 * i % 8 + 1);
    a[i] = fmaf(u, cos[i], -__fmul_rn(v, sin[i]));
    b[i] = fmaf(v, cos[i], __fmul_rn(u, sin[i]));
  }
  if (halves) {
    x = u4{bf16_pair(a[0], a[1]), bf16_pair(a[2], a[3]), bf16_pair(a[4], a[5]), bf16_pair(a[6], a[7])};
    y = u4{bf16_pair(b[0], b[1]), bf16_pair(b[2], b[3]), bf16_pair(b[4], b[5]), bf16_pair(b[6], b[7])};
  } else {
    x = u4{bf16_pair(a[0], b[0]), bf16_pair(a[1], b[1]), bf16_pair(a[2], b[2]), bf16_pair(a[3], b[3])};
    y = u4{bf16_pair(a[4], b[4]), bf16_pair(a[5], b[5]), bf16_pair(a[6], b[6]), bf16_pair(a[7], b[7])};
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

// One workgroup: tokens_per tokens and heads_per of their heads.  Each thread
// works out one cosine and sine at a time into LDS; then D / 16 lanes take a row,
// rows in memory order, U rows of each lane in flight.
template <int D>
__global__ __launch_bounds__(256) void rope(RopeArgs a) {
  constexpr int NL = D / 16, RW = 256 / NL;      // lanes per row, rows at a time
  constexpr int U = 2;
  __shared__ __attribute__((aligned(16))) float cs[2][kRopeTokens * kMaxPairs];
  const int64_t tok0 = (int64_t)blockIdx.x * a.tokens_per;
  const int toks = (int)min((int64_t)a.tokens_per, a.n - tok0);
  const int h0 = blockIdx.y * a.heads_per, heads = min(a.heads_per, a.n_q + a.n_k - h0);
  const int pairs = a.rope.rot_dim / 2;
  const int c = threadIdx.x % NL;
  const Chunks ch = chunks_of(a.rope, c);
  const bool turns = c < pairs / 8, halves = a.rope.pairs == HWKV_ROPE_HALF;
  auto row_at = [&](int r, const uint16_t *q, int64_t qs, const uint16_t *k, int64_t ks) {
    const int t = r / heads, h = h0 + r - t * heads;
    const int64_t tok = tok0 + t;
    return h < a.n_q ? q + tok * qs + h * D : k + tok * ks + (h - a.n_q) * D;
  };
  const int rows = toks * heads;
  for (int r0 = threadIdx.x / NL; r0 < rows || r0 < RW; r0 += U * RW) {
    u4 x[U], y[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (r0 + i * RW >= rows) break;
      const uint16_t *from = row_at(r0 + i * RW, a.q, a.q_stride, a.k, a.k_stride);
      x[i] = *reinterpret_cast<const u4 *>(from + ch.x);
      y[i] = *reinterpret_cast<const u4 *>(from + ch.y);
    }
    if (r0 < RW) {                               // once, behind the first rows' loads
      for (int i = threadIdx.x; i < toks * pairs; i += 256) {
        const int t = i / pairs, p = i - t * pairs;
        cos_sin(a.rope, a.pos + tok0 + t, a.pos_stride, p, &cs[0][i], &cs[1][i]);
      }
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int r = r0 + i * RW;
      if (r >= rows) break;
      if (turns) {
        const int at = r / heads * pairs + 8 * c;
        turn(&cs[0][at], &cs[1][at], halves, x[i], y[i]);
      }
      uint16_t *to = const_cast<uint16_t *>(
          row_at(r, a.q_out, (int64_t)a.n_q * D, a.k_out, (int64_t)a.n_k * D));
      *reinterpret_cast<u4 *>(to + ch.x) = x[i];
      *reinterpret_cast<u4 *>(to + ch.y) = y[i];
    }
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
  u4 x = *reinterpret_cast<const u4 *>(from + ch.x);
  u4 y = *reinterpret_cast<const u4 *>(from + ch.y);
  if (turns) {
    float cs[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) cos_sin(a.rope, a.pos + b, a.pos_stride, 8 * c + i, &cs[i], &sn[i]);
    turn(cs, sn, a.rope.pairs == HWKV_ROPE_HALF, x, y);
  }
  if (isq) {
    uint16_t *to = a.q_out + b * a.q_out_stride + h * D;
    *reinterpret_cast<u4 *>(to + ch.x) = x;
    *reinterpret_cast<u4 *>(to + ch.y) = y;
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
    e = row_scale(group_max<NL>(max(top8(chunk(x)), top8(chunk(y)))));
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
  put(ch.x, chunk(x));
  put(ch.y, chunk(y));
}

// A workgroup takes two rounds of rows (of RW), in as many tokens as that is, and
// fewer where that leaves less than 1,024 workgroups; below 256 tokens one round.
// us a call, 1 / 2 / 4 / 8 tokens a workgroup: 32,768 tokens of 40 heads of 128 126 /
// 125 / 128 / 132 (5.4 TB/s; 162 with a wavefront's lanes on 8 tokens and every lane
// its own cosines), of 28 of 256 167 / 171 / 182 / 190, of 10 of 64 57 / 35 / 24 / 19.
// One token of 40 heads 2.8, in one workgroup 3.1.
template <int D>
hipError_t launch_rope_d(RopeArgs a, hipStream_t s) {
  constexpr int RW = 256 * 16 / D;
  const int heads = a.n_q + a.n_k;
  const int64_t rounds = std::max(1, (2 * RW + heads / 2) / heads);
  a.tokens_per = (int32_t)std::min<int64_t>({rounds, std::max<int64_t>(1, a.n / 1024), kRopeTokens});
  a.heads_per = a.n < 256 ? std::min(heads, RW) : heads;
  const dim3 grid((unsigned)((a.n + a.tokens_per - 1) / a.tokens_per),
                  (unsigned)((heads + a.heads_per - 1) / a.heads_per));
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
