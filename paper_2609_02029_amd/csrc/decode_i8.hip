// decode_i8.hip -- decode attention over int8 caches (kv_rows8.h; gfx950, matrix
// cores): with the work decomposition, fused append and partials of
// decode_split.h, or (ITEM) with those of decode_item.h, whose one launch takes
// the items of up to 192 sequences, whole or in shares.
//
// With the codes c and scale bytes e of the rows,
//     z_s = scale 2^(eK_s - 133) q.cK_s,
//     out = sum_s p_s 2^(eV_s - 133) cV_s / sum_s p_s,   p_s = 2^(z_s - m) in base 2.
//
// Wave w of the workgroup takes slots [16w, 16w + 16) of every tile and all of
// their channels, two tiles at a time, with an online softmax of its own:
//   q.c    v_mfma_i32_16x16x64_i8 on the codes as they are stored: A = K (16
//          slots x 64 channels: lane (g, r) holds chunks 8m + g and 8m + 4 + g of
//          slot r), B = q as a whole number of 22 bits and a sign in three signed
//          digits of 8 bits, one product each.  Products and sums are exact; the
//          digits' sums meet in fp32.  The 16 columns repeat the heads (c mod 8, or
//          mod 4 up to 4 heads), and half of them take the second tile's logits:
//          lane (g, c) has slots 4g .. 4g + 3 of one head and one tile.
//   p.c    v_mfma_f32_16x16x32_bf16 over both tiles' slots: A = the weights
//          p_s 2^(eV_s - 139) as three bf16 terms, each the rounded rest of those
//          before it (2^-27 of a weight is left behind; two terms leave 2^-18 and
//          cost 2.5e-6 of the output, ten times what fp32 does).  The terms of a head
//          are rows of their own, whose other tile's half comes from the lane that
//          has it, so that up to 4 heads take one product for all three, 6 and 8 a
//          second for the third.  B = V: a lane reads 4 channels of its rows as words
//          and widens them (one conversion a code, half a packing), which
//          transposes them on the way.
// A code thus costs 1.5 vector instructions for V and none for K, against 0.5 and
// 0.5 plus a byte read each in decode_mfma; two tiles at a time halve the softmax
// (one tile: 31 us against 27 for 32 sequences of 3,000 tokens, 64 x 8, 8 KV heads).
//
// What bounds it: HBM, as long as loads stay in flight.  A wave's slices of K, V
// and the scale pairs go from global memory straight into its own part of LDS
// (buffer_load ... lds); a pair of tiles is read into registers whole (64 of them
// at head_dim 256) and the next pair's loads are issued before anything is
// computed, so two tiles of every wave are always in flight: 66 KB a workgroup at
// head_dim 256, two workgroups per CU (more at 64 and 128: rings of four and eight
// tiles, which left room for two, were slower by 1 to 20 %).  No barrier falls
// inside the walk.  16 sequences of 16K to 64K tokens, 256 x 6: 530 MB in 90 us, 5.9
// TB/s; a launch costs about 6 us beyond its bytes.
#include <algorithm>
#include <cfloat>

#include "decode_split.h"
#include "kv_rows8.h"
#include "lds_loads.h"

namespace hwkv {
namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));

// The value of lane c + N of the lane's 16 (modulo 16).
template <int N>
__device__ __forceinline__ uint32_t from_ahead(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x120 + 16 - N, 0xf, 0xf, true);   // row_ror
}

template <int D, int G, bool ITEM>
__global__ __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(2)))
void decode_i8(std::conditional_t<ITEM, ItemArgs, DecodeArgs> a) {
  static_assert(G <= 8, "heads and their second terms share 16 rows");
  constexpr int NC = D / 8;            // chunks per row
  constexpr int KM = D / 64;           // 64-channel products of q.c
  constexpr int VB = D / 16;           // 16-channel blocks of the output
  constexpr int KB = 16 * D;           // a wave's part of a tile: K slice, V rows,
  constexpr int SB = 2 * KB + 256;     //   scale pairs
  constexpr int WB = 2 * SB;           //   of two tiles; its acc in the epilogue
  static_assert(WB >= 16 * D * 4, "16 acc rows");
  constexpr int HC = G <= 4 ? 4 : 8;   // columns, and rows of a term
  __shared__ __attribute__((aligned(1024))) uint8_t area[kWaves * WB];
  __shared__ __attribute__((aligned(16))) uint8_t digits[3 * G * D];
  __shared__ f32x2_t zs_s[G];
  __shared__ float sml[kWaves][2][8];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int g4 = lane >> 4, l16 = lane & 15;
  // The item: its rows (K, V and scale pairs, or pages from page-table entry pto
  // on), the slot that takes a new token (-1: none), its q and k_new / v_new rows;
  // this workgroup's tiles lt = first, first + step, ... < last; where it leaves
  // its result (whole: the output; else partial part).
  int nv, new_slot, pto, first, step, last;
  int64_t koff, voff, soff;
  size_t q_row, kv_row, part;
  bool whole;
  if constexpr (ITEM) {
    // as in decode_item
    const int run = blockIdx.x / a.n_seqs;
    const int rank = __builtin_amdgcn_readfirstlane(__popcll(__ballot(a.wg_begin[lane] <= run)) - 1);
    const int h = a.head_order[rank];
    const int split = run - a.wg_begin[rank];
    int si = blockIdx.x - run * a.n_seqs;
    if (a.rotate) {
      si -= run % a.n_seqs;
      si += si < 0 ? a.n_seqs : 0;
    }
    const int b = a.seq[si], n = a.len[si];
    const ItemHead &hd = a.head[h];
    nv = min(n, hd.cap);
    const int all_tiles = (nv + 63) / 64;
    // an item of more than tiles_per_wg tiles in equal shares (none of them empty)
    const int splits = (all_tiles + a.tiles_per_wg - 1) / a.tiles_per_wg;
    if (split >= splits) return;                 // uniform: a shorter item
    const int share = (all_tiles + splits - 1) / splits;
    first = split * share;
    step = 1;
    last = min(all_tiles, first + share);
    whole = last - first == all_tiles;
    pto = hd.page0 >= 0 ? hd.page0 + b * a.max_pages : -1;
    koff = hd.k_off + (int64_t)b * hd.cap_pad * D;
    voff = hd.v_off + (int64_t)b * hd.cap_pad * D;
    soff = (int64_t)hd.s_off128 * 128 + (int64_t)b * hd.cap_pad * kRowScaleBytes;
    q_row = ((size_t)b * a.n_kv_heads + h) * G;
    kv_row = (size_t)b * a.n_kv_heads + h;
    part = (size_t)(a.part_begin[rank] + split * a.part_seqs[rank] + si);
    const int pos = n - 1;
    const int slot = hd.window == 0 || pos < a.n_sinks ? pos : a.n_sinks + (pos - a.n_sinks) % hd.window;
    new_slot = a.k_new && slot / 64 >= first && slot / 64 < last ? slot : -1;
  } else {
    // one round of lane loads, as in decode_split
    static_assert(kMaxItems == 64, "one lane per item");
    const DecodeItems &it = a.it;
    const int blk = blockIdx.x;
    const int sb_l = it.split_begin[lane], sb1_l = it.split_begin[lane + 1];
    const int nv_l = it.n_valid[lane], ns_l = it.new_slot[lane], pto_l = it.pto[lane];
    const int qrow_l = it.q_row[lane], kvrow_l = it.kv_row[lane];
    const int64_t koff_l = it.k_off[lane], voff_l = it.v_off[lane], soff_l = it.s_off[lane];
    const int item = __builtin_amdgcn_readfirstlane(__popcll(__ballot(sb_l <= blk)) - 1);
    auto pick = [&](int v) { return __builtin_amdgcn_readlane(v, item); };
    auto pick64 = [&](int64_t v) {
      const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)v, item);
      const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)v >> 32), item);
      return (int64_t)(((uint64_t)hi << 32) | lo);
    };
    first = blk - pick(sb_l);
    step = pick(sb1_l) - pick(sb_l);
    nv = pick(nv_l);
    last = (nv + 63) / 64;
    whole = step == 1;
    new_slot = pick(ns_l);
    pto = pick(pto_l);
    koff = pick64(koff_l);
    voff = pick64(voff_l);
    soff = pick64(soff_l);
    q_row = pick(qrow_l);
    kv_row = pick(kvrow_l);
    part = it.ws_split0 + blk;
  }
  uint8_t *const cache = static_cast<uint8_t *>(a.cache);
  uint8_t *const pool = cache + a.pool_off;
  uint8_t *const kbase = cache + koff, *const vbase = cache + voff, *const sbase = cache + soff;
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
  // split: logical tile 0 is the tile that holds new_slot (see decode_split)
  const int tile_new = new_slot >= 0 ? new_slot / 64 : 0;
  auto phys = [&](int lt) {
    if constexpr (ITEM) return lt;
    return __builtin_amdgcn_readfirstlane(lt == 0 ? tile_new : (lt == tile_new ? 0 : lt));
  };

  // per-lane load offsets.  K: load n takes chunks 8n .. 8n + 7 of the wave's 16
  // slots, 128 bytes each.  V: the LDS row 4i + g holds row 4g + i, its 16-byte
  // pieces rotated so that the four rows a group of lanes reads together lie in
  // different banks.  Scale pairs: 32 bytes, lanes 0 .. 7; the others are out of
  // range.
  const uint32_t area0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)area + wave * WB;
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
  auto issue = [&](int lt, int half) {
    const bool has = lt < last;
    const int t = phys(has ? lt : first);
    const Tile at = tile(t);
    const int rows = min(64, nv - 64 * t);
    const __amdgpu_buffer_rsrc_t kr = make_rsrc(at.k, has ? (uint32_t)(64 * D) : 0u);
    const __amdgpu_buffer_rsrc_t vr = make_rsrc(at.v, has ? (uint32_t)(rows * D) : 0u);
    const __amdgpu_buffer_rsrc_t sr = make_rsrc(at.s, has ? (uint32_t)(64 * kRowScaleBytes) : 0u);
    const uint32_t to = area0 + half * SB;
#pragma unroll
    for (int n = 0; n < KB / 1024; ++n) stage_lds<false>(kr, to + n * 1024, kl, n * 4096);
#pragma unroll
    for (int n = 0; n < KB / 1024; ++n) stage_lds<false>(vr, to + KB + n * 1024, vl[n], 0);
    stage_lds<true>(sr, to + 2 * KB, sl, 0);
  };
  const bool writes_new =
      __builtin_amdgcn_readfirstlane((int)(new_slot >= 0 && (ITEM || first == 0))) != 0;
  if (writes_new && wave == 0) {
    const Tile t = tile(tile_new);
    const int g = lane % NC, r = new_slot % 64;
    const uint16_t *from = (lane < NC ? a.k_new : a.v_new) + kv_row * D + g * 8;
    uint4 x = make_uint4(0u, 0u, 0u, 0u);
    if (lane < 2 * NC) x = *reinterpret_cast<const uint4 *>(from);
    const uint32_t e = row_scale(group_max<NC>(top8(x)));
    if (lane < 2 * NC) {
      store_chunk<HWKV_KV_I8>(lane < NC ? t.k + (g * 64 + r) * 8 : t.v + r * D + g * 8, encode8_row(x, e));
      if (g == 0) t.s[r * kRowScaleBytes + lane / NC] = (uint8_t)e;
    }
  }
  // q: 8 channels a thread, as digits in the order the products read them; a
  // head is scaled by the power of two that puts its largest |q| in [2^21, 2^22)
  const bool has_q = threadIdx.x < G * NC;
  uint4 q8 = make_uint4(0u, 0u, 0u, 0u);
  if (has_q) q8 = *reinterpret_cast<const uint4 *>(a.q + q_row * D + threadIdx.x * 8);
  if (!writes_new) {
    issue(first, 0);
    issue(first + step, 1);
  }
  {
    const uint32_t top = group_max<NC>(top8(q8));
    const int sh = 148 - (int)max(top >> 7, 1u);
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
      // What takes this back, and 2^-6 (codes count 2^(e - 133), the bits of 2^(e -
      // 127) are e << 23), in two factors around the row's own, so that no step
      // leaves fp32's range where q.k does not.  A head that is not finite has NaN
      // for its logits.
      if (c == 0) {
        const int back = -6 - sh, near = min(max(back, -60), 60);
        zs_s[h] = f32x2_t{ldexpf(1.0f, near),
                          top >= 0x7f80u ? __builtin_nanf("") : ldexpf(a.scale_log2, back - near)};
      }
    }
  }
  // only this workgroup reads the new slot in this launch (see decode_split)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
  __syncthreads();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
  if (writes_new) {
    issue(first, 0);
    issue(first + step, 1);
  }

  const int hc = l16 % HC, u = l16 / HC;
  i32x4_t qd[3][KM];
#pragma unroll
  for (int t = 0; t < 3; ++t)
#pragma unroll
    for (int m = 0; m < KM; ++m) {
      qd[t][m] = *reinterpret_cast<const i32x4_t *>(digits + t * G * D + (hc < G ? hc : 0) * D + m * 64 + g4 * 16);
      if (hc >= G) qd[t][m] = i32x4_t{0, 0, 0, 0};
    }
  const f32x2_t zs = hc < G ? zs_s[hc] : f32x2_t{0.f, 0.f};

  // the lane's head: running shift m (base 2, lazily raised: the weights stay
  // below 2^8; it begins below every finite logit) and the sum of its slots' weights
  float m = -FLT_MAX, lsum = 0.0f;
  f32x4_t o[VB];
#pragma unroll
  for (int vb = 0; vb < VB; ++vb) o[vb] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  // this lane's column: which of the pair's two tiles, and the term its weights
  // take as a row of A
  const bool second = u & 1;
  const uint8_t *const sp = area + wave * WB;
  for (int lt = first; lt < last; lt += 2 * step) {
    // the pair's loads have landed; all of it goes into registers, and the next
    // pair's loads are issued
    wait_loads();
    i32x4_t kc[2][KM];
    uint32_t vc[2][KM][4];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < KM; ++i) {
        const uint8_t *const k = sp + b * SB + (8 * i + g4) * 128 + l16 * 8;
        const uint2 x = *reinterpret_cast<const uint2 *>(k), y = *reinterpret_cast<const uint2 *>(k + 512);
        kc[b][i] = i32x4_t{(int)x.x, (int)x.y, (int)y.x, (int)y.y};
#pragma unroll
        for (int n = 0; n < 4; ++n)
          vc[b][i][n] = *reinterpret_cast<const uint32_t *>(
              sp + b * SB + KB + (4 * n + g4) * D + (((4 * i + l16 / 4) ^ piece_xor(g4)) * 16) + l16 % 4 * 4);
      }
    const uint2 pairs = *reinterpret_cast<const uint2 *>(sp + (second ? SB : 0) + 2 * KB + 8 * g4);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    issue(lt + 2 * step, 0);
    issue(lt + 3 * step, 1);

    f32x4_t sum;
    {
      i32x4_t s[2][3];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int t = 0; t < 3; ++t) {
          s[b][t] = i32x4_t{0, 0, 0, 0};
#pragma unroll
          for (int i = 0; i < KM; ++i)
            s[b][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(kc[b][i], qd[t][i], s[b][t], 0, 0, 0);
        }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int s0 = second ? s[1][0][i] : s[0][0][i], s1 = second ? s[1][1][i] : s[0][1][i],
                  s2 = second ? s[1][2][i] : s[0][2][i];
        sum[i] = fmaf((float)s2, 65536.0f, fmaf((float)s1, 256.0f, (float)s0));
      }
    }
    // online softmax of the lane's head over its four slots of its tile
    const int ta = 64 * phys(lt), tb = lt + step < last ? 64 * phys(lt + step) : nv;
    const int slot0 = (second ? tb : ta) + 16 * wave + 4 * g4;
    float z[4], vs[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t pr = (i < 2 ? pairs.x : pairs.y) >> (16 * (i & 1));
      const bool valid = slot0 + i < nv;
      z[i] = valid ? sum[i] * zs.x * __uint_as_float((pr & 255u) << 23) * zs.y : -INFINITY;
      vs[i] = valid ? __uint_as_float((pr << 15) & 0x7f800000u) : 0.f;
    }
    float mx = max_of_rows(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])));
    mx = fmaxf(mx, __uint_as_float(from_ahead<HC>(__float_as_uint(mx))));
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
    // 2^-12 centres the range: value rows from 2^-98 (below, the third term and then
    // the second are lost) to 2^108 (above, long sums overflow)
    float w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p = exp2f(z[i] - m);
      lsum += p;
      w[i] = p * 0x1p-12f * vs[i];
    }
    u32x2_t t[4];
    t[0] = u32x2_t{pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3])};
    const float r[4] = {w[0] - bf_lo(t[0].x), w[1] - bf_hi(t[0].x), w[2] - bf_lo(t[0].y), w[3] - bf_hi(t[0].y)};
    t[1] = u32x2_t{pack_bf16x2(r[0], r[1]), pack_bf16x2(r[2], r[3])};
    t[2] = u32x2_t{pack_bf16x2(r[0] - bf_lo(t[1].x), r[1] - bf_hi(t[1].x)),
                   pack_bf16x2(r[2] - bf_lo(t[1].y), r[3] - bf_hi(t[1].y))};
    t[3] = u32x2_t{0u, 0u};
    // Row l16 of A is term u of the lane's head over both tiles: its own tile's
    // words, and the other's from the lane HC ahead, which holds that tile
    auto both = [&](u32x2_t own, u32x2_t sent) {
      const u32x2_t got = {from_ahead<HC>(sent.x), from_ahead<HC>(sent.y)};
      return second ? u32x4_t{got.x, got.y, own.x, own.y} : u32x4_t{own.x, own.y, got.x, got.y};
    };
    u32x4_t pw, pl;
    if constexpr (HC == 4) {
      pw = both(u == 0 ? t[0] : u == 1 ? t[1] : u == 2 ? t[2] : t[3],
                u == 1 ? t[0] : u == 2 ? t[1] : u == 3 ? t[2] : t[3]);
    } else {
      pw = both(u == 0 ? t[0] : t[1], u == 0 ? t[1] : t[0]);
      pl = both(t[2], t[2]);
      if (u != 0) pl = u32x4_t{0u, 0u, 0u, 0u};
    }
    static_for<4>([&](auto ec) {
      constexpr int e = decltype(ec)::value;
#pragma unroll
      for (int n = 0; n < KM; ++n) {
        const u32x4_t v = {codes_bf16x2<e>(vc[0][n][0], vc[0][n][1]), codes_bf16x2<e>(vc[0][n][2], vc[0][n][3]),
                           codes_bf16x2<e>(vc[1][n][0], vc[1][n][1]), codes_bf16x2<e>(vc[1][n][2], vc[1][n][3])};
        o[4 * n + e] = mfma_kq(pw, v, o[4 * n + e]);
        if constexpr (HC == 8) o[4 * n + e] = mfma_kq(pl, v, o[4 * n + e]);
      }
    });
  }

  // ---- the workgroup's result: every wave's (m, l, acc) in its own area (after
  // the last, empty, loads have landed), then an exact merge
  wait_loads();
  float lt = lsum + __shfl_xor(lsum, 16);
  lt += __shfl_xor(lt, 32);
  lt += __shfl_xor(lt, HC);            // the other tiles of the pairs
  if (lane < G) {
    sml[wave][0][lane] = m;
    sml[wave][1][lane] = lt;
  }
  // (all 16 rows, a head's terms among them: the merge adds them as it reads)
  float *const accw = reinterpret_cast<float *>(area + wave * WB);
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int n = 0; n < KM; ++n)
      *reinterpret_cast<f32x4_t *>(accw + (4 * g4 + r) * D + 64 * n + 4 * l16) =
          f32x4_t{o[4 * n][r], o[4 * n + 1][r], o[4 * n + 2][r], o[4 * n + 3][r]};
  __syncthreads();

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
      L += sml[w][1][h] * f;
      f32x4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < (HC == 4 ? 3 : 2); ++t)
        x += *reinterpret_cast<const f32x4_t *>(area + w * WB + ((t * HC + h) * D + c) * 4);
      A += x * f;
    }
    const float back = 0x1p6f;         // 2^12 of the weights, 2^-6 of the codes
    if (whole) {
      __builtin_nontemporal_store(A * (back / L),
                                  reinterpret_cast<f32x4_t *>(&a.out[(q_row + h) * D + c]));
    } else {
      __builtin_nontemporal_store(
          A * back, reinterpret_cast<f32x4_t *>(&a.part_acc[(part * G + h) * D + c]));
      if (c == 0)
        __builtin_nontemporal_store(
            f32x2_t{M, L}, reinterpret_cast<f32x2_t *>(&a.part_ml[(part * G + h) * 2]));
    }
  }
}

// Merge of split items, one workgroup per (item, q head): rows of D / 4 lanes take
// every R-th split, a lane 4 channels, and meet in LDS.  (item_merge walks an
// item's splits on one such row: 38 us for 300 of them.)
template <int D, int G>
__global__ __launch_bounds__(256) void i8_merge(ItemArgs a) {
  constexpr int LPR = D / 4, R = 256 / LPR;
  constexpr int U = 4;                           // splits per round, loads in flight
  __shared__ __attribute__((aligned(16))) f32x4_t acc_s[256];
  __shared__ float m_s[R], l_s[R];
  const int rank = blockIdx.y / G, g = blockIdx.y % G, si = blockIdx.x;
  if (si >= a.part_seqs[rank]) return;           // uniform: not split
  const int h = a.head_order[rank], b = a.seq[si];
  const int tiles = (min(a.len[si], a.head[h].cap) + 63) / 64;
  const int ns = (tiles + a.tiles_per_wg - 1) / a.tiles_per_wg;
  const int row = threadIdx.x / LPR, c = threadIdx.x % LPR * 4;
  const size_t p0 = (size_t)(a.part_begin[rank] + si) * G + g;
  const size_t step = (size_t)a.part_seqs[rank] * G;   // the next split's partial
  float M = -FLT_MAX, L = 0.f;
  f32x4_t A = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = row; j0 < ns; j0 += U * R) {
    f32x2_t ml[U];
    f32x4_t x[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const size_t p = p0 + (size_t)min(j0 + i * R, ns - 1) * step;
      ml[i] = *reinterpret_cast<const f32x2_t *>(a.part_ml + p * 2);
      x[i] = *reinterpret_cast<const f32x4_t *>(a.part_acc + p * D + c);
    }
    float Mn = M;
#pragma unroll
    for (int i = 0; i < U; ++i) Mn = fmaxf(Mn, ml[i].x);
    const float f = exp2f(M - Mn);
    L *= f;
    A *= f;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const float e = j0 + i * R < ns ? exp2f(ml[i].x - Mn) : 0.f;
      L += ml[i].y * e;
      A += x[i] * e;
    }
    M = Mn;
  }
  acc_s[threadIdx.x] = A;
  if (c == 0) {
    m_s[row] = M;
    l_s[row] = L;
  }
  __syncthreads();
  if (row > 0) return;
  const int rows = min(R, ns);                   // those that had a split
  for (int r = 1; r < rows; ++r) M = fmaxf(M, m_s[r]);
  L = 0.f;
  A = f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int r = 0; r < rows; ++r) {
    const float f = exp2f(m_s[r] - M);
    L += l_s[r] * f;
    A += acc_s[r * LPR + threadIdx.x] * f;
  }
  *reinterpret_cast<f32x4_t *>(a.out + (((size_t)b * a.n_kv_heads + h) * G + g) * D + c) = A * (1.0f / L);
}

template <int D, int G>
struct I8Launch {
  static hipError_t run(const DecodeArgs &a, int n, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
    hipExtLaunchKernelGGL((decode_i8<D, G, false>), dim3(n), dim3(kWaves * 64), 0, s, e0, e1, 0, a);
    return hipGetLastError();
  }
};

template <int D, int G>
struct I8ItemLaunch {
  static hipError_t run(const ItemArgs &a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
    hipExtLaunchKernelGGL((decode_i8<D, G, true>), dim3(a.n_seqs * a.wg_begin[a.n_kv_heads]),
                          dim3(kWaves * 64), 0, s, e0, e1, 0, a);
    return hipGetLastError();
  }
};

template <int D, int G>
struct I8MergeLaunch {
  static hipError_t run(const ItemArgs &a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
    int most = 0;                    // split items of a head
    for (int r = 0; r < a.n_kv_heads; ++r) most = std::max(most, (int)a.part_seqs[r]);
    hipExtLaunchKernelGGL((i8_merge<D, G>), dim3(most, a.n_kv_heads * G), dim3(256), 0, s, e0, e1, 0, a);
    return hipGetLastError();
  }
};

}  // namespace

hipError_t launch_decode_i8(int D, int G, const DecodeArgs &a, int n_splits, hipStream_t s,
                            hipEvent_t e0, hipEvent_t e1) {
  return dispatch_dg<I8Launch>(D, G, a, n_splits, s, e0, e1);
}

hipError_t launch_decode_i8_item(int D, int G, const ItemArgs &a, hipStream_t s, hipEvent_t e0,
                                 hipEvent_t e1) {
  return dispatch_dg<I8ItemLaunch>(D, G, a, s, e0, e1);
}

hipError_t launch_i8_merge(int D, int G, const ItemArgs &a, hipStream_t s, hipEvent_t e0,
                           hipEvent_t e1) {
  return dispatch_dg<I8MergeLaunch>(D, G, a, s, e0, e1);
}

}  // namespace hwkv
