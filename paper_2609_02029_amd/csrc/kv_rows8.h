// kv_rows8.h -- the int8 cache format (HWKV_KV_I8): codes with one
// power-of-two scale for each token row of a KV head, K and V apart (gfx950).
//
// A row whose largest magnitude lies in [2^(e - 127), 2^(e - 126)) is held as
// its scale byte e and the codes round(x 2^(133 - e)), to nearest even, clamped
// to +-127: the value of a code c is c 2^(e - 133).  e is the bf16 exponent
// field of the largest magnitude (1 for a row of zeros and subnormals), so both
// the quotient and the value are exact, and every value is a bf16 value: prefill
// attention and the calibration replay stage codes as bf16 without rounding.
// The scale is the row's own because a ring slot is overwritten one token at a
// time: a scale shared by several tokens would have to change under the codes
// of those that stay, and what is stored would depend on the chunking.  A row
// that holds an infinity or a NaN has e = 255 and codes 0: 0 x 2^128 makes every
// one of its values NaN where it is used.
//
// Error: half a step of 2^-6 of the row's power of two, at most 2^-7 of its
// largest magnitude.  On unit normal rows of 128 channels that is 41 dB below
// the values, against 32 dB for fp8 codes under a well-chosen scale; a row with
// loud channels loses to fp8 in the others (29 dB with two eight times louder).
//
// Layout: codes as in an fp8 cache (K tiles slot-minor, V rows); the scale bytes
// as pairs (K's, V's) in slot order, in an area after every unit's codes
// ([unit][seq][cap_pad][2]), or behind the V rows of a page ([256][2]).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "hwkv_internal.h"
#include "kv_format.h"

namespace hwkv {

template <>
struct KvFormat<HWKV_KV_I8> {
  static constexpr int kBytes = 1;
  using Chunk = uint2;
};

// Elements of one page of a paged unit: K tiles, V rows, scale pairs.
template <int F>
constexpr int page_elems(int D) {
  return 2 * kPageTokens * D + (F == HWKV_KV_I8 ? kRowScaleBytes * kPageTokens : 0);
}

// The largest of 8 bf16 magnitudes, as bits (infinity and NaN are the largest).
__device__ __forceinline__ uint32_t top8(uint4 x) {
  auto hi = [](uint32_t w) { return max((w >> 16) & 0x7fffu, w & 0x7fffu); };
  return max(max(hi(x.x), hi(x.y)), max(hi(x.z), hi(x.w)));
}

// The scale byte of a row whose largest magnitude has these bf16 bits.
__device__ __forceinline__ uint32_t row_scale(uint32_t top) { return max(top >> 7, 1u); }

// 8 codes of a row with scale byte e.
__device__ __forceinline__ uint2 encode8_row(uint4 x, uint32_t e) {
  const int up = 133 - (int)e;
  auto code = [&](uint32_t bits) -> uint32_t {
    const float y = __builtin_rintf(ldexpf(bf16_bits_to_f32(bits), up));
    return (uint32_t)(int)fminf(fmaxf(y, -127.0f), 127.0f) & 0xffu;
  };
  auto four = [&](uint32_t a, uint32_t b) {
    return code(a & 0xffffu) | code(a >> 16) << 8 | code(b & 0xffffu) << 16 | code(b >> 16) << 24;
  };
  if (e == 255u) return make_uint2(0u, 0u);
  return make_uint2(four(x.x, x.y), four(x.z, x.w));
}

// 8 codes of a row with scale byte e as 8 bf16 values (exact).
__device__ __forceinline__ uint4 widen8_row(uint2 c, uint32_t e) {
  auto val = [&](uint32_t w, int i) -> uint32_t {
    const float v = (float)(int)(int8_t)(w >> (8 * i));
    // 0 x infinity: the NaN of a row that is not finite
    const float y = e == 255u ? __builtin_nanf("") : ldexpf(v, (int)e - 133);
    return __builtin_bit_cast(uint32_t, y) >> 16;
  };
  auto two = [&](uint32_t w, int i) { return val(w, i) | val(w, i + 1) << 16; };
  return make_uint4(two(c.x, 0), two(c.x, 2), two(c.y, 0), two(c.y, 2));
}

// The largest of `v` over groups of N lanes (a power of two).
template <int N>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
#pragma unroll
  for (int off = 1; off < N; off <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, off));
  return v;
}

}  // namespace hwkv
