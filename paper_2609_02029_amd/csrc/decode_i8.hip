// decode_i8.hip -- split phase of the decode attention over int8 caches
// (kv_rows8.h; gfx950, wave64), with the work decomposition, fused append and
// partial format of decode_split.h.
//
// With the codes c and scale bytes e of the rows,
//     z_s = scale 2^(eK_s - 133) q.cK_s,   out = sum_s p_s 2^(eV_s - 133) cV_s / sum_s p_s,
// p_s = 2^(z_s - m).  A wave takes whole 64-slot tiles with an online softmax of
// its own: q.k with a lane per slot, p.v with a lane on D / 64 channels.
#include "decode_split.h"
#include "kv_rows8.h"

namespace hwkv {
namespace {

template <int D, int G>
__global__ __launch_bounds__(kWaves * 64) void decode_i8(DecodeArgs a) {
  constexpr int NC = D / 8;            // chunks per row
  constexpr int CPL = D / 64;          // channels per lane of the value product
  __shared__ __attribute__((aligned(16))) float q_s[G * D];
  __shared__ float w_s[kWaves][64 * G];
  __shared__ float acc_s[kWaves][G * D];
  __shared__ float m_s[kWaves][G], l_s[kWaves][G];

  const DecodeItems &it = a.it;
  const int blk = blockIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int item = __builtin_amdgcn_readfirstlane(__popcll(__ballot(it.split_begin[lane] <= blk)) - 1);
  const int j = blk - it.split_begin[item];
  const int nwg = it.split_begin[item + 1] - it.split_begin[item];
  const int nv = it.n_valid[item], new_slot = it.new_slot[item], pto = it.pto[item];
  const int n_tiles = (nv + 63) / 64;
  uint8_t *const cache = static_cast<uint8_t *>(a.cache);
  // K tile, V rows and scale pairs of tile t
  struct Tile {
    uint8_t *k, *v, *s;
  };
  auto tile = [&](int t) -> Tile {
    if (pto >= 0) {
      constexpr int TPP = kPageTokens / 64;
      const int64_t pg = a.page_table[pto + t / TPP];
      uint8_t *const p = cache + a.pool_off + pg * page_elems<HWKV_KV_I8>(D);
      return {p + t % TPP * 64 * D, p + (kPageTokens + t % TPP * 64) * D,
              p + 2 * kPageTokens * D + t % TPP * 64 * kRowScaleBytes};
    }
    return {cache + it.k_off[item] + (int64_t)t * 64 * D, cache + it.v_off[item] + (int64_t)t * 64 * D,
            cache + it.s_off[item] + t * 64 * kRowScaleBytes};
  };
  // logical tile 0 is the tile that holds new_slot (see decode_split)
  const int tile_new = new_slot >= 0 ? new_slot / 64 : 0;
  auto phys = [&](int lt) { return lt == 0 ? tile_new : (lt == tile_new ? 0 : lt); };
  if (new_slot >= 0 && j == 0 && wave == 0) {
    const Tile t = tile(tile_new);
    const int g = lane % NC, r = new_slot % 64;
    const uint16_t *from = (lane < NC ? a.k_new : a.v_new) + (size_t)it.kv_row[item] * D + g * 8;
    uint4 x = make_uint4(0u, 0u, 0u, 0u);
    if (lane < 2 * NC) x = *reinterpret_cast<const uint4 *>(from);
    const uint32_t e = row_scale(group_max<NC>(top8(x)));
    if (lane < 2 * NC) {
      store_chunk<HWKV_KV_I8>(lane < NC ? t.k + (g * 64 + r) * 8 : t.v + r * D + g * 8, encode8_row(x, e));
      if (g == 0) t.s[r * kRowScaleBytes + lane / NC] = (uint8_t)e;
    }
  }
  for (int i = threadIdx.x; i < G * D; i += kWaves * 64)
    q_s[i] = bf16_bits_to_f32(a.q[(size_t)it.q_row[item] * D + i]);
  // only this workgroup reads the new slot in this launch (see decode_split)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
  __syncthreads();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");

  float m[G], l[G], acc[G][CPL];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    m[g] = -1e30f;
    l[g] = 0.f;
#pragma unroll
    for (int e = 0; e < CPL; ++e) acc[g][e] = 0.f;
  }
  for (int lt = j + wave * nwg; lt < n_tiles; lt += kWaves * nwg) {
    const int pt = phys(lt);
    const Tile t = tile(pt);
    const bool valid = 64 * pt + lane < nv;
    float z[G];
#pragma unroll
    for (int g = 0; g < G; ++g) z[g] = 0.f;
    for (int c = 0; c < NC; ++c) {
      const uint2 x = *reinterpret_cast<const uint2 *>(t.k + (c * 64 + lane) * 8);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float k = (float)(int8_t)((i < 4 ? x.x : x.y) >> (8 * (i & 3)));
#pragma unroll
        for (int g = 0; g < G; ++g) z[g] = fmaf(k, q_s[g * D + c * 8 + i], z[g]);
      }
    }
    const uint32_t pair = *reinterpret_cast<const uint16_t *>(t.s + lane * kRowScaleBytes);
    const float ks = __uint_as_float((pair & 255u) << 23), vs = __uint_as_float((pair >> 8) << 23);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      z[g] = valid ? z[g] * ks * (a.scale_log2 * 0.015625f) : -INFINITY;
      const float mn = fmaxf(m[g], wave_max(z[g]));
      const float alpha = exp2f(m[g] - mn);
      m[g] = mn;
      l[g] *= alpha;
#pragma unroll
      for (int e = 0; e < CPL; ++e) acc[g][e] *= alpha;
      const float p = exp2f(z[g] - mn);
      l[g] += p;
      w_s[wave][lane * G + g] = valid ? p * vs : 0.f;
    }
    wave_lds_order();
    const int rows = min(64, nv - 64 * pt);
    for (int r = 0; r < rows; ++r) {
      float v[CPL];
#pragma unroll
      for (int e = 0; e < CPL; ++e) v[e] = (float)(int8_t)t.v[r * D + lane * CPL + e];
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int e = 0; e < CPL; ++e) acc[g][e] = fmaf(w_s[wave][r * G + g], v[e], acc[g][e]);
    }
    wave_lds_order();
  }
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const float lg = wave_sum(l[g]);
    if (lane == 0) {
      m_s[wave][g] = m[g];
      l_s[wave][g] = lg;
    }
#pragma unroll
    for (int e = 0; e < CPL; ++e) acc_s[wave][g * D + lane * CPL + e] = acc[g][e] * 0.015625f;
  }
  __syncthreads();
  const size_t part = (size_t)(it.ws_split0 + blk) * G;
  for (int i = threadIdx.x; i < G * D; i += kWaves * 64) {
    const int g = i / D, c = i % D;
    float M = m_s[0][g], L = 0.f, A = 0.f;
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, m_s[w][g]);
    for (int w = 0; w < kWaves; ++w) {
      const float f = exp2f(m_s[w][g] - M);
      L += l_s[w][g] * f;
      A += acc_s[w][i] * f;
    }
    if (nwg == 1) {
      a.out[((size_t)it.q_row[item] + g) * D + c] = A / L;
    } else {
      a.part_acc[(part + g) * D + c] = A;
      if (c == 0) {
        a.part_ml[(part + g) * 2] = M;
        a.part_ml[(part + g) * 2 + 1] = L;
      }
    }
  }
}

template <int D, int G>
struct I8Launch {
  static hipError_t run(const DecodeArgs &a, int n, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
    hipExtLaunchKernelGGL((decode_i8<D, G>), dim3(n), dim3(kWaves * 64), 0, s, e0, e1, 0, a);
    return hipGetLastError();
  }
};

}  // namespace

hipError_t launch_decode_i8(int D, int G, const DecodeArgs &a, int n_splits, hipStream_t s,
                            hipEvent_t e0, hipEvent_t e1) {
  return dispatch_dg<I8Launch>(D, G, a, n_splits, s, e0, e1);
}

}  // namespace hwkv
