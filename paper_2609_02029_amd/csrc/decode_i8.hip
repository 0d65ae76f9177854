// decode_i8.hip -- split phase of the decode attention over int8 caches
// (kv_rows8.h; gfx950, matrix cores), with the work decomposition, fused append
// and partial format of decode_split.h.
//
// With the codes c and scale bytes e of the rows,
//     z_s = scale 2^(eK_s - 133) q.cK_s,
//     out = sum_s p_s 2^(eV_s - 133) cV_s / sum_s p_s,   p_s = 2^(z_s - m) in base 2.
//
// Wave w of the workgroup takes slots [16w, 16w + 16) of every tile and all of
// their channels, with an online softmax of its own.  Per tile:
//   q.c    v_mfma_i32_16x16x64_i8 on the codes as they are stored: A = K (16
//          slots x 64 channels: lane (g, r) holds chunks 8m + g and 8m + 4 + g of
//          slot r), B = q as a whole number of 22 bits and a sign in three signed
//          digits of 8 bits, one product each.  Products and sums are exact; the
//          digits' sums meet in fp32.  Lane (g, c) ends with the logits of slots
//          4g .. 4g + 3 for head c mod 8 (mod 4 up to 4 heads): the columns repeat
//          the heads.
//   p.c    v_mfma_f32_16x16x16_bf16: A = the weights p_s 2^(eV_s - 151) as three bf16
//          terms, each the rounded rest of those before it (2^-27 of a weight is
//          left behind; two terms leave 2^-18 and cost 2.5e-6 of the output, a tenth
//          of that is fp32's).  The terms of a head are rows of their own, so that
//          up to 4 heads take one product for all three, 6 and 8 a second for the
//          third.  B = V (16 slots x 16 channels): a lane reads 4 channels of its 4
//          rows as words and widens them (one conversion a code, half a packing),
//          which transposes them on the way.
// A code thus costs 1.5 vector instructions for V and none for K, against 0.5 and
// 0.5 plus a byte read each in decode_mfma.
//
// What bounds it: HBM, as long as loads stay in flight.  A wave's slices of K, V
// and the scale pairs go from global memory straight into its own part of LDS
// (buffer_load ... lds) in a ring of ST stages; a stage is read into registers
// whole (48 of them at head_dim 256) and its loads for ST tiles on are issued
// before anything is computed, so ST tiles of a wave are always in flight: 66 KB
// a workgroup, two workgroups per CU.  No barrier falls inside the walk.
#include "decode_split.h"
#include "kv_rows8.h"

namespace hwkv {
namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));

// 16 bytes (4 with DWORD) per lane from a buffer into LDS, at 16 (4) x lane of
// lds_block; past the descriptor's range zeros arrive.  The load has no
// destination register, and the kernel waits for it itself (wait_vm): as a
// builtin it would make the compiler wait for every load in flight before each
// LDS read.
template <bool DWORD>
__device__ __forceinline__ void stage_lds(__amdgpu_buffer_rsrc_t r, uint32_t lds_block, int voffset,
                                          int soffset) {
  if constexpr (DWORD)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen nt lds" ::"s"(lds_block),
                 "v"(voffset), "s"(r), "s"(soffset)
                 : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen nt lds" ::"s"(lds_block),
                 "v"(voffset), "s"(r), "s"(soffset)
                 : "memory", "m0");
}

// At most LEFT vector memory operations of the wave are still in flight.
template <int LEFT>
__device__ __forceinline__ void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"i"(LEFT) : "memory");
}

// Two bf16 of the signed bytes E of two words, low first (exact).
template <int E>
__device__ __forceinline__ uint32_t codes_bf16x2(uint32_t x, uint32_t y) {
  const f32x2_t f = {(float)(int)(int8_t)(x >> (8 * E)), (float)(int)(int8_t)(y >> (8 * E))};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));
}

template <int D, int G>
__global__ __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(2)))
void decode_i8(DecodeArgs a) {
  static_assert(G <= 8, "heads and their second terms share 16 rows");
  constexpr int NC = D / 8;            // chunks per row
  constexpr int KM = D / 64;           // 64-channel products of q.c
  constexpr int VB = D / 16;           // 16-channel blocks of the output
  constexpr int ST = 512 / D;          // stages of a wave's ring
  constexpr int KB = 16 * D;           // a stage: K slice, V rows, scale pairs
  constexpr int SB = 2 * KB + 256;
  constexpr int LOADS = 2 * KB / 1024 + 1;
  constexpr int WB = ST * SB;          // a wave's ring; its acc in the epilogue
  constexpr int HC = G <= 4 ? 4 : 8;   // columns, and rows of a term
  static_assert(WB >= G * D * 4, "the acc rows fit the ring");
  __shared__ __attribute__((aligned(1024))) uint8_t ring[kWaves * WB];
  __shared__ __attribute__((aligned(16))) uint8_t digits[3 * G * D];
  __shared__ float zs_s[G];
  __shared__ float sml[kWaves][2][8];

  const DecodeItems &it = a.it;
  const int blk = blockIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int g4 = lane >> 4, l16 = lane & 15;
  // the item: one round of lane loads, as in decode_split
  static_assert(kMaxItems == 64, "one lane per item");
  const int sb_l = it.split_begin[lane], sb1_l = it.split_begin[lane + 1];
  const int nv_l = it.n_valid[lane], ns_l = it.new_slot[lane], pto_l = it.pto[lane];
  const int qrow_l = it.q_row[lane];
  const int64_t koff_l = it.k_off[lane], voff_l = it.v_off[lane], soff_l = it.s_off[lane];
  const int item = __builtin_amdgcn_readfirstlane(__popcll(__ballot(sb_l <= blk)) - 1);
  auto pick = [&](int v) { return __builtin_amdgcn_readlane(v, item); };
  auto pick64 = [&](int64_t v) {
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)v, item);
    const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)v >> 32), item);
    return (int64_t)(((uint64_t)hi << 32) | lo);
  };
  const int j = blk - pick(sb_l);
  const int nwg = pick(sb1_l) - pick(sb_l);
  const int nv = pick(nv_l), new_slot = pick(ns_l), pto = pick(pto_l), q_row = pick(qrow_l);
  const int n_tiles = (nv + 63) / 64;
  uint8_t *const cache = static_cast<uint8_t *>(a.cache);
  uint8_t *const pool = cache + a.pool_off;
  uint8_t *const kbase = cache + pick64(koff_l), *const vbase = cache + pick64(voff_l),
                *const sbase = cache + pick64(soff_l);
  // K tile, V rows and scale pairs of physical tile t
  struct Tile {
    uint8_t *k, *v, *s;
  };
  auto tile = [&](int t) -> Tile {
    constexpr int TPP = kPageTokens / 64;
    if (pto >= 0) {
      // (a scalar load: a vector one would wait for every load in flight)
      const int64_t pg = ((const __attribute__((address_space(4))) int32_t *)a.page_table)[pto + t / TPP];
      uint8_t *const p = pool + pg * page_elems<HWKV_KV_I8>(D);
      return {p + t % TPP * 64 * D, p + (kPageTokens + t % TPP * 64) * D,
              p + 2 * kPageTokens * D + t % TPP * 64 * kRowScaleBytes};
    }
    return {kbase + (int64_t)t * 64 * D, vbase + (int64_t)t * 64 * D, sbase + t * 64 * kRowScaleBytes};
  };
  // logical tile 0 is the tile that holds new_slot (see decode_split)
  const int tile_new = new_slot >= 0 ? new_slot / 64 : 0;
  auto phys = [&](int lt) {
    return __builtin_amdgcn_readfirstlane(lt == 0 ? tile_new : (lt == tile_new ? 0 : lt));
  };

  // per-lane load offsets.  K: load n takes chunks 8n .. 8n + 7 of the wave's 16
  // slots, 128 bytes each.  V: the LDS row 4i + g holds row 4g + i, its 16-byte
  // pieces rotated so that the four rows a group of lanes reads together lie in
  // different banks.  Scale pairs: 32 bytes, lanes 0 .. 7; the others are out of
  // range.
  const uint32_t ring0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)ring + wave * WB;
  const int kl = lane / 8 * 512 + 128 * wave + lane % 8 * 16;
  constexpr int PCS = D / 16;          // 16-byte pieces of a V row
  const int vdr = lane / PCS, vpc = lane % PCS;   // row and piece of LDS within a load
  auto piece_xor = [](int g) { return D == 256 ? 4 * g : D == 128 ? 4 * (g >> 1) : 0; };
  int vl[KB / 1024];
#pragma unroll
  for (int n = 0; n < KB / 1024; ++n) {
    const int dr = n * (1024 / D) + vdr, g = dr % 4;
    vl[n] = (16 * wave + 4 * g + dr / 4) * D + (vpc ^ piece_xor(g)) * 16;
  }
  const int sl = lane < 8 ? 32 * wave + 4 * lane : 1 << 20;
  auto issue = [&](int lt, int stage) {
    const bool has = lt < n_tiles;
    const int t = has ? phys(lt) : 0;
    const Tile at = tile(t);
    const int rows = min(64, nv - 64 * t);
    const __amdgpu_buffer_rsrc_t kr = make_rsrc(at.k, has ? (uint32_t)(64 * D) : 0u);
    const __amdgpu_buffer_rsrc_t vr = make_rsrc(at.v, has ? (uint32_t)(rows * D) : 0u);
    const __amdgpu_buffer_rsrc_t sr = make_rsrc(at.s, has ? (uint32_t)(64 * kRowScaleBytes) : 0u);
    const uint32_t to = ring0 + stage * SB;
#pragma unroll
    for (int n = 0; n < KB / 1024; ++n) stage_lds<false>(kr, to + n * 1024, kl, n * 4096);
#pragma unroll
    for (int n = 0; n < KB / 1024; ++n) stage_lds<false>(vr, to + KB + n * 1024, vl[n], 0);
    stage_lds<true>(sr, to + 2 * KB, sl, 0);
  };

  const bool writes_new = __builtin_amdgcn_readfirstlane((int)(new_slot >= 0 && j == 0)) != 0;
  if (writes_new && wave == 0) {
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
  // q: 8 channels a thread, as digits in the order the products read them; a
  // head is scaled by the power of two that puts its largest |q| in [2^21, 2^22),
  // less where the logit scale that takes it back would leave fp32's range
  const bool has_q = threadIdx.x < G * NC;
  uint4 q8 = make_uint4(0u, 0u, 0u, 0u);
  if (has_q) q8 = *reinterpret_cast<const uint4 *>(a.q + (size_t)q_row * D + threadIdx.x * 8);
  if (!writes_new) {
#pragma unroll
    for (int s = 0; s < ST; ++s) issue(j + s * nwg, s);
  }
  {
    const uint32_t top = group_max<NC>(top8(q8));
    int ez;
    (void)frexpf(a.scale_log2, &ez);
    const int sh = top ? min(148 - (int)max(top >> 7, 1u), ez + 110) : 0;
    const uint32_t w[4] = {q8.x, q8.y, q8.z, q8.w};
    uint32_t d[3][2] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t b = i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
      int x = top >= 0x7f80u ? 0 : (int)__builtin_rintf(ldexpf(bf16_bits_to_f32(b), sh));
#pragma unroll
      for (int t = 0; t < 3; ++t) {
        d[t][i / 4] |= (uint32_t)(x & 255) << (8 * (i % 4));
        x = (x - (int)(int8_t)x) >> 8;
      }
    }
    if (has_q) {
      const int h = threadIdx.x / NC, c = threadIdx.x % NC;
      const int at = h * D + c / 8 * 64 + c % 4 * 16 + c % 8 / 4 * 8;
#pragma unroll
      for (int t = 0; t < 3; ++t)
        *reinterpret_cast<uint2 *>(digits + t * G * D + at) = make_uint2(d[t][0], d[t][1]);
      // (2^-6: codes count 2^(e - 133), the bits of 2^(e - 127) are e << 23; a
      // head that is not finite has NaN for its logits)
      if (c == 0) zs_s[h] = top >= 0x7f80u ? __builtin_nanf("") : ldexpf(a.scale_log2, -6 - sh);
    }
  }
  // only this workgroup reads the new slot in this launch (see decode_split)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
  __syncthreads();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
  if (writes_new) {
#pragma unroll
    for (int s = 0; s < ST; ++s) issue(j + s * nwg, s);
  }

  const int hc = l16 % HC, term = l16 / HC;
  i32x4_t qd[3][KM];
#pragma unroll
  for (int t = 0; t < 3; ++t)
#pragma unroll
    for (int m = 0; m < KM; ++m) {
      qd[t][m] = *reinterpret_cast<const i32x4_t *>(digits + t * G * D + (hc < G ? hc : 0) * D + m * 64 + g4 * 16);
      if (hc >= G) qd[t][m] = i32x4_t{0, 0, 0, 0};
    }
  const float zs = hc < G ? zs_s[hc] : 0.f;

  // the lane's head: running shift m (base 2, lazily raised: the weights stay
  // below 2^8) and the sum of its slots' weights
  float m = -1e30f, lsum = 0.0f;
  f32x4_t o[VB];
#pragma unroll
  for (int vb = 0; vb < VB; ++vb) o[vb] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  const uint8_t *const mine = ring + wave * WB;
  int stage = 0;
  for (int lt = j; lt < n_tiles; lt += nwg) {
    // the stage's loads have landed; all of it goes into registers, and its
    // loads for ST tiles on are issued
    wait_vm<(ST - 1) * LOADS>();
    const uint8_t *const sp = mine + stage * SB;
    i32x4_t kc[KM];
#pragma unroll
    for (int i = 0; i < KM; ++i) {
      const uint2 x = *reinterpret_cast<const uint2 *>(sp + (8 * i + g4) * 128 + l16 * 8);
      const uint2 y = *reinterpret_cast<const uint2 *>(sp + (8 * i + 4 + g4) * 128 + l16 * 8);
      kc[i] = i32x4_t{(int)x.x, (int)x.y, (int)y.x, (int)y.y};
    }
    uint32_t vc[KM][4];
#pragma unroll
    for (int n = 0; n < KM; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        vc[n][i] = *reinterpret_cast<const uint32_t *>(
            sp + KB + (4 * i + g4) * D + (((4 * n + l16 / 4) ^ piece_xor(g4)) * 16) + l16 % 4 * 4);
    const uint2 pairs = *reinterpret_cast<const uint2 *>(sp + 2 * KB + 8 * g4);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    issue(lt + ST * nwg, stage);
    stage = stage + 1 == ST ? 0 : stage + 1;

    i32x4_t s[3];
#pragma unroll
    for (int t = 0; t < 3; ++t) {
      s[t] = i32x4_t{0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < KM; ++i) s[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(kc[i], qd[t][i], s[t], 0, 0, 0);
    }
    // online softmax of the lane's head over its four slots
    const int slot0 = 64 * phys(lt) + 16 * wave + 4 * g4;
    float z[4], vs[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t pr = (i < 2 ? pairs.x : pairs.y) >> (16 * (i & 1));
      const bool valid = slot0 + i < nv;
      const float sum = fmaf((float)s[2][i], 65536.0f, fmaf((float)s[1][i], 256.0f, (float)s[0][i]));
      z[i] = valid ? sum * __uint_as_float((pr & 255u) << 23) * zs : -INFINITY;
      vs[i] = valid ? __uint_as_float((pr << 15) & 0x7f800000u) : 0.f;
    }
    float mx = fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]));
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    if (__any(mx > m + 8.0f)) {
      const float mn = fmaxf(m, mx);
      const float alpha = exp2f(m - mn);
      m = mn;
      lsum *= alpha;
      // acc rows 4 g + r are heads (4 g + r) mod HC
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float al = __shfl(alpha, (4 * g4 + r) % HC);
#pragma unroll
        for (int vb = 0; vb < VB; ++vb) o[vb][r] *= al;
      }
    }
    // 2^-24 keeps the weights of the largest rows in range
    float w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p = exp2f(z[i] - m);
      lsum += p;
      w[i] = p * 0x1p-24f * vs[i];
    }
    u32x2_t t0, t1, t2;
    t0.x = pack_bf16x2(w[0], w[1]);
    t0.y = pack_bf16x2(w[2], w[3]);
    const float r[4] = {w[0] - bf_lo(t0.x), w[1] - bf_hi(t0.x), w[2] - bf_lo(t0.y), w[3] - bf_hi(t0.y)};
    t1.x = pack_bf16x2(r[0], r[1]);
    t1.y = pack_bf16x2(r[2], r[3]);
    t2.x = pack_bf16x2(r[0] - bf_lo(t1.x), r[1] - bf_hi(t1.x));
    t2.y = pack_bf16x2(r[2] - bf_lo(t1.y), r[3] - bf_hi(t1.y));
    const u32x2_t none = {0u, 0u};
    const u32x2_t pw = term == 0 ? t0 : term == 1 ? t1 : term == 2 ? t2 : none;
    const u32x2_t pl = term == 0 ? t2 : none;      // 6 and 8 heads: the third term
    static_for<4>([&](auto ec) {
      constexpr int e = decltype(ec)::value;
#pragma unroll
      for (int n = 0; n < KM; ++n) {
        const u32x2_t v = {codes_bf16x2<e>(vc[n][0], vc[n][1]), codes_bf16x2<e>(vc[n][2], vc[n][3])};
        o[4 * n + e] = mfma_pv(pw, v, o[4 * n + e]);
        if constexpr (HC == 8) o[4 * n + e] = mfma_pv(pl, v, o[4 * n + e]);
      }
    });
  }

  // ---- the workgroup's partial: every wave's (m, l, acc) in its own ring
  // (after the last, empty, loads have landed), then an exact merge
  wait_vm<0>();
  float lt = lsum + __shfl_xor(lsum, 16);
  lt += __shfl_xor(lt, 32);
  if (lane < G) {
    sml[wave][0][lane] = m;
    sml[wave][1][lane] = lt;
  }
  float *const accw = reinterpret_cast<float *>(ring + wave * WB);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int h = 4 * g4 + r;
#pragma unroll
    for (int n = 0; n < KM; ++n) {
      f32x4_t x;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = o[4 * n + e][r];
        if constexpr (HC == 4) x[e] += __shfl_xor(x[e], 16);
        x[e] += __shfl_xor(x[e], 32);
      }
      if (h < G) *reinterpret_cast<f32x4_t *>(accw + h * D + 64 * n + 4 * l16) = x;
    }
  }
  __syncthreads();

  const int pidx = it.ws_split0 + blk;
  for (int idx = threadIdx.x; idx < G * D / 4; idx += kWaves * 64) {
    const int h = idx / (D / 4), c = (idx % (D / 4)) * 4;
    float M = sml[0][0][h];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, sml[w][0][h]);
    float L = 0.f;
    f32x4_t A = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = exp2f(sml[w][0][h] - M);
      const f32x4_t x = *reinterpret_cast<const f32x4_t *>(ring + w * WB + ((size_t)h * D + c) * 4);
      L += sml[w][1][h] * f;
      A += x * f;
    }
    const float back = 0x1p18f;        // 2^24 of the weights, 2^-6 of the codes
    if (nwg == 1) {
      __builtin_nontemporal_store(A * (back / L),
                                  reinterpret_cast<f32x4_t *>(&a.out[((size_t)q_row + h) * D + c]));
    } else {
      __builtin_nontemporal_store(
          A * back, reinterpret_cast<f32x4_t *>(&a.part_acc[((size_t)pidx * G + h) * D + c]));
      if (c == 0)
        __builtin_nontemporal_store(
            f32x2_t{M, L}, reinterpret_cast<f32x2_t *>(&a.part_ml[((size_t)pidx * G + h) * 2]));
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
