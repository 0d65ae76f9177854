// decode_shared.h -- decode attention of sequences that share pages of a paged
// cache (gfx950, matrix cores), for every cache format; instantiated once per
// format by decode_shared_<format>.hip.
//
// The sequences of a fork hold the same pages up to where they parted.  An item of
// work is a run of rows of one KV head and the query columns that see all of them:
//   a block   the pages that a group of sequences shares, with the q heads of all of
//             its members (up to 64 columns), so that a row is read once for them;
//   an own    a sequence's rows from there on, a window's rows, or all the rows of
//             a sequence that shares nothing, with its own q heads.
// Every item is split over workgroups, workgroup j of n taking its tiles of 64 rows
// j, j + n, ..; each leaves (m, l, acc) of its columns, and shared_merge adds, for
// every q head of a sequence, the parts of its block and its own:
//     out = sum_j acc_j 2^(m_j - M) / sum_j l_j 2^(m_j - M),  M = max m_j.
//
// A wavefront has 16 columns (so that its accumulators take 64 registers at head_dim
// 256, whatever the block) and a part of every tile's rows, with an online softmax of
// its own; the waves of a column group meet in LDS at the end.
//   z = K q   v_mfma_f32_16x16x32: A = K (16 rows x 32 channels; lane (g, r) holds
//             8 channels of row r as they lie in the K tile), B = the columns of q.
//             Lane (g, c) ends with rows 4g .. 4g + 3 of column c.
//   acc += V p  the same shape, transposed: A = V (lane (g, r): rows 4g .. 4g + 3 of
//             channel r), B = the weights as lane (g, c) formed them.  The weights
//             enter as terms, each the rounded rest of those before it, so that they
//             keep fp32's precision: three of bf16 (2^-27 is left), or two of
//             binary16 over binary16 values (2^-22).  The 32 places of a product hold
//             two terms of 16 rows over the same V, or the third of two times 16 rows.
// Rows go from memory straight into LDS, 64 KB of K and V at a time (a stage of one to
// four tiles).  With one column group (CW = 1) four waves share out a tile's rows and
// each loads, and reads into registers whole, its own: no barrier falls inside the
// walk, the next stage's loads are issued before anything is computed, and two
// workgroups fit a CU.  With two or four (32, 64 columns) eight waves share the rows,
// in two stages that barriers hand over, one workgroup per CU.
#pragma once

#include <cfloat>

#include "decode_split.h"
#include "kv_rows8.h"
#include "lds_loads.h"

namespace hwkv {
namespace {

typedef _Float16 h16x8_t __attribute__((ext_vector_type(8)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

// D += A B over 32 places, operands of the format's 16-bit type.
template <int F>
__device__ __forceinline__ f32x4_t product(u32x4_t a, u32x4_t b, f32x4_t c) {
  if constexpr (F == HWKV_KV_F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h16x8_t, a), __builtin_bit_cast(h16x8_t, b), c,
                                                  0, 0, 0);
  else
    return mfma_kq(a, b, c);
}

// Two codes of 8 bits (bytes E of two words) as two bf16 values.
template <int F, int E>
__device__ __forceinline__ uint32_t pair_of_codes(uint32_t x, uint32_t y) {
  if constexpr (F == HWKV_KV_I8) return codes_bf16x2<E>(x, y);
  else return fp8x2_bf16x2<false>(__builtin_amdgcn_perm(y, x, 0x0c0c0400u + E * 0x0101u));
}

// Eight consecutive codes as 8 bf16 values.
template <int F>
__device__ __forceinline__ u32x4_t widen_codes(u32x2_t c) {
  if constexpr (F == HWKV_KV_I8) {
    auto two = [](uint32_t w, int e) {
      const f32x2_t f = {(float)(int)(int8_t)(w >> (8 * e)), (float)(int)(int8_t)(w >> (8 * e + 8))};
      return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));
    };
    return u32x4_t{two(c.x, 0), two(c.x, 2), two(c.y, 0), two(c.y, 2)};
  } else {
    return u32x4_t{fp8x2_bf16x2<false>(c.x), fp8x2_bf16x2<true>(c.x), fp8x2_bf16x2<false>(c.y),
                   fp8x2_bf16x2<true>(c.y)};
  }
}

// Tiles of a stage.
constexpr int shared_tiles(int row_bytes) { return row_bytes >= 512 ? 1 : row_bytes >= 256 ? 2 : 4; }

// All but the last N vector memory operations of the wave are done.
template <int N>
__device__ __forceinline__ void wait_all_but() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// The wave's LDS reads are done.
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// A barrier that leaves loads in flight.
__device__ __forceinline__ void meet() { asm volatile("s_barrier" ::: "memory"); }

constexpr int shared_threads(int CW) { return CW == 1 ? 256 : 512; }

template <int D, int F, int CW>
__global__ __launch_bounds__(shared_threads(CW)) __attribute__((amdgpu_waves_per_eu(2)))
void decode_shared(SharedArgs a) {
  constexpr bool CODES = KvFormat<F>::kBytes == 1, I8 = F == HWKV_KV_I8, F16 = F == HWKV_KV_F16;
  constexpr bool ALONE = CW == 1;      // a wave reads only what it has loaded
  constexpr int EB = KvFormat<F>::kBytes;
  constexpr int WAVES = shared_threads(CW) / 64;
  constexpr int NC = D / 8;            // chunks of a row
  constexpr int KS = D / 32;           // products over the channels
  constexpr int VB = D / 16;           // channel blocks
  constexpr int ROW = D * EB;
  constexpr int PCS = ROW / 16;        // 16-byte pieces of a V row
  constexpr int NT = shared_tiles(ROW);
  constexpr int KB = 64 * ROW;         // K, or V, of a tile
  constexpr int TB = 2 * KB + (I8 ? 1024 : 0);   // and scale pairs
  constexpr int STAGE = NT * TB, BUFS = ALONE ? 1 : 2;
  constexpr int LDS = NT * KB / 1024 / WAVES;    // a wave's loads of K, and of V, of a stage
  constexpr int LOADS = 2 * LDS + (I8 ? NT : 0);
  constexpr int PARTS = NT * 4;        // 16-row parts of a stage,
  constexpr int P = ALONE ? NT : 2;    // that a wave computes at a time
  constexpr int CB = 16 * CW;          // columns
  static_assert(BUFS * STAGE >= WAVES * 16 * D * 4, "16 columns of acc a wave, at the end");
  static_assert(STAGE >= CB * D * 2, "the columns of q");
  __shared__ __attribute__((aligned(1024))) uint8_t area[BUFS * STAGE];
  __shared__ __attribute__((aligned(16))) u32x4_t q_s[ALONE ? KS * 64 : 1];
  __shared__ float back_s[CB][2];      // what a column's logits are multiplied by
  __shared__ float sml[WAVES][2][16];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int g4 = lane >> 4, l16 = lane & 15;
  // ---- the item
  const int rank = __builtin_amdgcn_readfirstlane(__popcll(__ballot(a.wg_begin[lane] <= (int)blockIdx.x)) - 1);
  const ItemHead &hd = a.head[rank];
  const int h = a.head_id[rank];
  const int local = blockIdx.x - a.wg_begin[rank];
  int first, count, row0, end, j, nwg;
  bool block = false;
  if (rank < a.n_full) {
    int item = -1;
#pragma unroll
    for (int i = 0; i < kSharedItems; i += 64)
      item += __popcll(__ballot((int)a.item_begin[i + lane] <= local));
    item = __builtin_amdgcn_readfirstlane(item);
    j = local - a.item_begin[item];
    nwg = a.item_begin[item + 1] - a.item_begin[item];
    block = item < a.n_blocks;
    first = block ? a.block_first[item] : item - a.n_blocks;
    count = block ? a.block_count[item] : 1;
    row0 = 0;
    end = a.len[first];
    if (block) {
      end = a.block_pages[item] * kPageTokens;
    } else if (a.seq_block[first] != kNoBlock) {
      row0 = a.block_pages[a.seq_block[first]] * kPageTokens;
    }
  } else {
    first = local % a.n_seqs;
    j = local / a.n_seqs;
    count = 1;
    row0 = 0;
    end = min(a.len[first], hd.cap);
    nwg = ((end + 63) / 64 + a.tiles_per_wg - 1) / a.tiles_per_wg;
    if (j >= nwg) return;              // uniform: a shorter sequence
  }
  const int ncols = count * a.group;
  // Waves share out the columns in groups of 16, and with those of their group the
  // parts: RW waves take `per` each, wave rw from part rw * per on.
  const int RW = ALONE ? 4 : ncols <= 16 ? 8 : ncols <= 32 ? 4 : 2;
  const int cw = wave / RW, rw = wave % RW;
  const int per = ALONE ? NT : max(PARTS / RW, 1);
  const bool busy = ALONE || (16 * cw < ncols && rw * per < PARTS);
  const int tile0 = row0 / 64, n_tiles = (end - row0 + 63) / 64;
  const int b0 = a.seq[first];
  const int pto = hd.page0 >= 0 ? hd.page0 + b0 * a.max_pages : -1;
  const uint8_t *const cache = static_cast<const uint8_t *>(a.cache);
  const uint8_t *const pool = cache + a.pool_off * EB;
  const int64_t rows0 = (int64_t)b0 * hd.cap_pad;
  const uint8_t *const kbase = cache + (hd.k_off + rows0 * D) * EB, *const vbase = cache + (hd.v_off + rows0 * D) * EB;
  const uint8_t *const sbase = I8 ? cache + (int64_t)hd.s_off128 * 128 + rows0 * kRowScaleBytes : cache;

  // The workgroup's i-th tile is tile0 + j + i nwg.  Lane i mod 64 holds its page (a
  // lookup for every tile, in front of its loads, is a round trip to the L2 each).
  int pages = 0;
  auto look_up = [&](int i0) {
    const int t = tile0 + min(j + (i0 + lane) * nwg, n_tiles - 1);
    if (pto >= 0) pages = a.page_table[pto + t / (kPageTokens / 64)];
    // (waited for here, once in 64 tiles, and not wherever it is read)
    asm volatile("" : "+v"(pages));
  };
  struct Tile {
    const uint8_t *k, *v, *s;
  };
  auto tile = [&](int i) -> Tile {
    constexpr int TPP = kPageTokens / 64;
    const int t = tile0 + j + i * nwg;
    if (pto >= 0) {
      const int64_t pg = __builtin_amdgcn_readlane(pages, i & 63);
      const uint8_t *const p = pool + pg * page_elems<F>(D) * EB;
      return {p + t % TPP * KB, p + kPageTokens * ROW + t % TPP * KB,
              p + 2 * kPageTokens * ROW + t % TPP * 64 * kRowScaleBytes};
    }
    return {kbase + (int64_t)t * KB, vbase + (int64_t)t * KB, sbase + t * 64 * kRowScaleBytes};
  };
  // ---- loads, 1 KB each.  K as it lies in the tile; ALONE, the wave's 16 rows of every
  // chunk, chunk by chunk.  V row by row, each row's pieces turned (by 32 bytes from row
  // to row at 16 bits) so that the rows that are read together lie in different banks;
  // of codes, LDS row 4i + g of 16 holds row 4g + i.
  auto piece_xor = [](int r) {
    if constexpr (CODES) return D == 256 ? 4 * (r & 3) : D == 128 ? 4 * ((r & 3) >> 1) : 0;
    return D == 64 ? 2 * (r >> 1 & 3) : 2 * (r & 7);
  };
  constexpr int RPL = 1024 / ROW;      // V rows of a load
  constexpr int TK = KB / 1024;        // loads of a tile's K, or V
  const uint32_t area0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)area;
  // the lane's place in load n of a tile's V (ALONE: of its 16 rows)
  auto v_offset = [&](int n) {
    const int r = n * RPL + lane / PCS;
    const int at = CODES ? (r & ~15) + 4 * (r & 3) + (r >> 2 & 3) : r;
    return at * ROW + ((lane % PCS) ^ piece_xor(r)) * 16;
  };
  const int kl = !ALONE ? lane * 16
                 : CODES ? lane / 8 * 512 + 128 * wave + lane % 8 * 16 : g4 * 1024 + (16 * wave + l16) * 16;
  int vl[LDS];
#pragma unroll
  for (int n = 0; n < LDS; ++n)
    vl[n] = ALONE ? 16 * wave * ROW + v_offset(n % (LDS / NT)) : v_offset((wave + WAVES * n) % TK);
  const int sl = lane < 32 ? 4 * lane : 1 << 20;
  // The loads of tiles i0 .. i0 + NT - 1; of those past the last nothing is read.
  auto issue = [&](int i0, int buf) {
    if (i0 % 64 == 0 && j + i0 * nwg < n_tiles) look_up(i0);
    const uint32_t to = area0 + buf * STAGE;
    struct Part {
      Tile at;
      int rows;
    };
    auto of = [&](int t) -> Part {
      const int lt = j + (i0 + t) * nwg;
      const Tile at = tile(i0 + t);
      return {at, lt < n_tiles ? min(64, end - 64 * (tile0 + lt)) : 0};
    };
    if constexpr (ALONE) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const Part x = of(t);
        const __amdgpu_buffer_rsrc_t kr = make_rsrc(x.at.k, x.rows > 0 ? (uint32_t)KB : 0u);
        const __amdgpu_buffer_rsrc_t vr = make_rsrc(x.at.v, (uint32_t)(x.rows * ROW));
        const uint32_t into = to + t * TB + wave * (KB / 4);
#pragma unroll
        for (int n = 0; n < TK / 4; ++n) stage_lds<false>(kr, into + n * 1024, kl, n * 4096);
#pragma unroll
        for (int n = 0; n < TK / 4; ++n) stage_lds<false>(vr, into + KB + n * 1024, vl[n], 0);
        // (every wave has the tile's pairs, in a place of its own)
        if constexpr (I8)
          stage_lds<true>(make_rsrc(x.at.s, x.rows > 0 ? 64u * kRowScaleBytes : 0u), to + t * TB + 2 * KB + wave * 256, sl,
                          0);
      }
    } else {
#pragma unroll
      for (int n = 0; n < LDS; ++n) {
        const int t = __builtin_amdgcn_readfirstlane((wave + WAVES * n) / TK), i = (wave + WAVES * n) % TK;
        const Part x = of(t);
        const __amdgpu_buffer_rsrc_t kr = make_rsrc(x.at.k, x.rows > 0 ? (uint32_t)KB : 0u);
        const __amdgpu_buffer_rsrc_t vr = make_rsrc(x.at.v, (uint32_t)(x.rows * ROW));
        const uint32_t into = __builtin_amdgcn_readfirstlane(to + t * TB + i * 1024);
        stage_lds<false>(kr, into, kl, __builtin_amdgcn_readfirstlane(i * 1024));
        stage_lds<false>(vr, into + KB, vl[n], 0);
      }
      // (every wave loads all pairs, the same bytes to the same place, so that the
      // waves have equal numbers of loads)
      if constexpr (I8)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const Part x = of(t);
          stage_lds<true>(make_rsrc(x.at.s, x.rows > 0 ? 64u * kRowScaleBytes : 0u), to + t * TB + 2 * KB, sl, 0);
        }
    }
  };
  issue(0, 0);

  // ---- q: column c is q head c mod G of the block's member c / G.  Over binary16
  // and int8 rows a column is scaled by a power of two, that of its largest |q|: to
  // [2^14, 2^15), so that binary16 holds it, or to [1, 2), so that sums over codes
  // stay in fp32's range.
  u32x4_t *const q_at = ALONE ? q_s : reinterpret_cast<u32x4_t *>(area + (BUFS - 1) * STAGE);
  for (int i = threadIdx.x; i < CB * NC; i += WAVES * 64) {
    const int c = i / NC, ch = i % NC;
    uint4 x = make_uint4(0u, 0u, 0u, 0u);
    if (c < ncols) {
      const int64_t row = (int64_t)a.seq[first + c / a.group] * a.n_q_heads + h * a.group + c % a.group;
      x = *reinterpret_cast<const uint4 *>(a.q + row * D + ch * 8);
    }
    u32x4_t y = {x.x, x.y, x.z, x.w};
    float near = a.scale_log2, rest = 1.0f;
    if constexpr (F16 || I8) {
      const uint32_t top = group_max<NC>(top8(x));
      const int sh = (F16 ? 141 : 127) - (int)max(top >> 7, 1u);
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float lo = ldexpf(bf_lo(w[k]), sh), hi = ldexpf(bf_hi(w[k]), sh);
        if constexpr (F16) {
          const f16x2_t v = {(_Float16)lo, (_Float16)hi};
          y[k] = __builtin_bit_cast(uint32_t, v);
        } else {
          y[k] = pack_bf16x2(lo, hi);
        }
      }
      // (codes count 2^(e - 133), the bits of 2^(e - 127) are e << 23; in two factors
      // around the row's own, so that no step leaves fp32's range)
      const int back = (I8 ? -6 : 0) - sh, mid = min(max(back, -60), 60);
      near = ldexpf(1.0f, mid);
      rest = top >= 0x7f80u ? __builtin_nanf("") : ldexpf(a.scale_log2, back - mid);
    } else if constexpr (F == HWKV_KV_FP8_E4M3) {
      near *= hd.k_scale;
    }
    q_at[(c / 16 * KS + ch / 4) * 64 + ch % 4 * 16 + c % 16] = y;
    if (ch == 0) {
      back_s[c][0] = near;
      back_s[c][1] = rest;
    }
  }
  // (the barriers of this phase wait for LDS alone: the first stage stays in flight)
  wait_reads();
  meet();
  u32x4_t q[KS];
#pragma unroll
  for (int i = 0; i < KS; ++i) q[i] = q_at[(cw * KS + i) * 64 + lane];
  const float near = back_s[16 * cw + l16][0], rest = back_s[16 * cw + l16][1];
  if constexpr (!ALONE) {
    wait_reads();
    meet();
    issue(NT, 1);
  }

  // ---- the walk.  m: running shift of the lane's column (base 2), raised where a
  // logit passes it by 8, so that weights stay below 2^8; it begins below every
  // finite logit.
  float m = -FLT_MAX, lsum = 0.0f;
  f32x4_t o[VB];
#pragma unroll
  for (int vb = 0; vb < VB; ++vb) o[vb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  int buf = 0;
  for (int i0 = 0; j + i0 * nwg < n_tiles; i0 += NT) {
    wait_all_but<(BUFS - 1) * LOADS>();
    if constexpr (!ALONE) meet();
    const uint8_t *const sp = area + buf * STAGE;
    for (int s0 = 0; busy && s0 < per; s0 += P) {
      // its parts s0 .. s0 + P - 1: rows [16 part, + 16) of tile t (ALONE: part `wave`
      // of every tile)
      u32x4_t kf[CODES ? 1 : P][KS];
      u32x2_t kc[CODES ? P : 1][KS];
      u32x2_t vf[CODES ? 1 : P][VB];
      uint32_t vc[CODES ? P : 1][CODES ? D / 64 : 1][4];
      u32x2_t pairs[P];
      int left[P];                     // of the lane's rows, from its first on
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int x = rw * per + min(s0 + p, per - 1);
        const int t = ALONE ? p : x / 4, part = ALONE ? wave : x % 4;
        const uint8_t *const at = sp + t * TB;
        const int lt = j + (i0 + t) * nwg;
        left[p] = lt < n_tiles && s0 + p < per ? end - (64 * (tile0 + lt) + 16 * part + 4 * g4) : 0;
        if constexpr (I8)
          pairs[p] = *reinterpret_cast<const u32x2_t *>(at + 2 * KB + (ALONE ? wave * 256 : 0) + 32 * part + 8 * g4);
        const uint8_t *const v = at + KB + part * (KB / 4);
        if constexpr (CODES) {
#pragma unroll
          for (int i = 0; i < KS; ++i)
            kc[p][i] = *reinterpret_cast<const u32x2_t *>(
                ALONE ? at + wave * (KB / 4) + (4 * i + g4) * 128 + l16 * 8 : at + (4 * i + g4) * 512 + part * 128 + l16 * 8);
#pragma unroll
          for (int i = 0; i < D / 64; ++i)
#pragma unroll
            for (int n = 0; n < 4; ++n)
              vc[p][i][n] = *reinterpret_cast<const uint32_t *>(v + (4 * n + g4) * D +
                                                                ((4 * i + l16 / 4) ^ piece_xor(g4)) * 16 + l16 % 4 * 4);
        } else {
#pragma unroll
          for (int i = 0; i < KS; ++i)
            kf[p][i] = *reinterpret_cast<const u32x4_t *>(
                ALONE ? at + wave * (KB / 4) + i * 1024 + lane * 16 : at + (4 * i + g4) * 1024 + part * 256 + l16 * 16);
          // (16 lanes read 4 rows of 16 channels, 8 bytes each, and receive 4 rows of one)
          const int r = 4 * g4 + l16 / 4;
#pragma unroll
          for (int vb = 0; vb < VB; ++vb)
            vf[p][vb] = __builtin_bit_cast(
                u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                             (lds_s16x4_t *)(uint8_t __attribute__((address_space(3))) *)(
                                 v + r * ROW + ((2 * vb) ^ piece_xor(r)) * 16 + l16 % 4 * 8)));
        }
      }
      if constexpr (ALONE) {
        wait_reads();
        issue(i0 + NT, 0);
      }

      // logits (a product that adds to the one before it waits out its latency: two
      // sums where there is one part)
      constexpr int CH = P == 1 ? 2 : 1;
      f32x4_t z[P], zz[P][CH];
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int c = 0; c < CH; ++c) zz[p][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < KS; ++i)
#pragma unroll
        for (int p = 0; p < P; ++p) {
          if constexpr (CODES) zz[p][i % CH] = product<F>(widen_codes<F>(kc[p][i]), q[i], zz[p][i % CH]);
          else zz[p][i % CH] = product<F>(kf[p][i], q[i], zz[p][i % CH]);
        }
#pragma unroll
      for (int p = 0; p < P; ++p) {
        z[p] = zz[p][0];
        if constexpr (CH == 2) z[p] += zz[p][1];
      }
      // (rows past the item's end have no weight)
      float top = -FLT_MAX;
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x = z[p][i] * near;
          if constexpr (I8) x *= __uint_as_float(((i < 2 ? pairs[p].x : pairs[p].y) >> (16 * (i & 1)) & 255u) << 23);
          if constexpr (I8 || F16) x *= rest;
          z[p][i] = i < left[p] ? x : -INFINITY;
          top = fmaxf(top, z[p][i]);
        }
      top = max_of_rows(top);
      if (__any(top > m + 8.0f)) {
        const float mn = fmaxf(m, top), f = exp2f(m - mn);
        m = mn;
        lsum *= f;
#pragma unroll
        for (int vb = 0; vb < VB; ++vb) o[vb] *= f;
      }
      u32x2_t term[P][F16 ? 2 : 3];
#pragma unroll
      for (int p = 0; p < P; ++p) {
        float w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w[i] = __builtin_amdgcn_exp2f(z[p][i] - m);
          lsum += w[i];
          if constexpr (F16) w[i] *= 0x1p7f;       // clear of binary16's subnormals
          // 2^-12 centres the range of weights times row scales
          if constexpr (I8) {
            const uint32_t pr = (i < 2 ? pairs[p].x : pairs[p].y) >> (16 * (i & 1));
            w[i] = i < left[p] ? w[i] * 0x1p-12f * __uint_as_float((pr << 15) & 0x7f800000u) : 0.f;
          }
        }
        if constexpr (F16) {
          const f16x2_t a0 = {(_Float16)w[0], (_Float16)w[1]}, a1 = {(_Float16)w[2], (_Float16)w[3]};
          const f16x2_t r0 = {(_Float16)(w[0] - (float)a0.x), (_Float16)(w[1] - (float)a0.y)},
                        r1 = {(_Float16)(w[2] - (float)a1.x), (_Float16)(w[3] - (float)a1.y)};
          term[p][0] = u32x2_t{__builtin_bit_cast(uint32_t, a0), __builtin_bit_cast(uint32_t, a1)};
          term[p][1] = u32x2_t{__builtin_bit_cast(uint32_t, r0), __builtin_bit_cast(uint32_t, r1)};
        } else {
#pragma unroll
          for (int k = 0; k < 3; ++k) {
            const u32x2_t x = {pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3])};
            term[p][k] = x;
            w[0] -= bf_lo(x.x);
            w[1] -= bf_hi(x.x);
            w[2] -= bf_lo(x.y);
            w[3] -= bf_hi(x.y);
          }
        }
      }
      // values: term by term over two parts; of a single part, the first two terms over
      // the same V, then the third.  (The product of 16 places takes as long as that of
      // 32; and compiled right behind one of 32 into the same accumulator, with no wait
      // between, it gave wrong sums.)
      constexpr int TERMS = F16 ? 2 : 3, STEPS = P == 1 ? TERMS - 1 : TERMS;
      auto add = [&](int step, int vb, const u32x2_t (&v)[P]) {
        if constexpr (P == 1) {
          const u32x2_t x = term[0][2 * step], y = step == 0 ? term[0][1] : u32x2_t{0u, 0u};
          o[vb] = product<F>(u32x4_t{v[0].x, v[0].y, v[0].x, v[0].y}, u32x4_t{x.x, x.y, y.x, y.y}, o[vb]);
        } else {
#pragma unroll
          for (int p = 0; p < P; p += 2) {
            const u32x2_t x = term[p][step], y = term[p + 1][step];
            o[vb] = product<F>(u32x4_t{v[p].x, v[p].y, v[p + 1].x, v[p + 1].y}, u32x4_t{x.x, x.y, y.x, y.y}, o[vb]);
          }
        }
      };
      if constexpr (CODES) {
        static_for<4>([&](auto ec) {
          constexpr int e = decltype(ec)::value;
          u32x2_t v[D / 64][P];
#pragma unroll
          for (int i = 0; i < D / 64; ++i)
#pragma unroll
            for (int p = 0; p < P; ++p)
              v[i][p] = u32x2_t{pair_of_codes<F, e>(vc[p][i][0], vc[p][i][1]), pair_of_codes<F, e>(vc[p][i][2], vc[p][i][3])};
#pragma unroll
          for (int step = 0; step < STEPS; ++step)
#pragma unroll
            for (int i = 0; i < D / 64; ++i) add(step, 4 * i + e, v[i]);
        });
      } else {
        u32x2_t v[VB][P];
#pragma unroll
        for (int vb = 0; vb < VB; ++vb)
#pragma unroll
          for (int p = 0; p < P; ++p) v[vb][p] = vf[p][vb];
        // (in runs of 8 blocks: a product that adds to the one before it waits)
#pragma unroll
        for (int v0 = 0; v0 < VB; v0 += 8)
#pragma unroll
          for (int step = 0; step < STEPS; ++step)
#pragma unroll
            for (int vb = v0; vb < VB && vb < v0 + 8; ++vb) add(step, vb, v[vb]);
      }
    }
    if constexpr (!ALONE) {
      wait_reads();
      meet();                          // nobody reads this stage any more
      issue(i0 + 2 * NT, buf);
      buf ^= 1;
    }
  }

  // ---- the workgroup's result: every wave's acc in an area of its own (after the
  // last, empty, loads have landed), 4 channels q of column c at place c ^ q of 16,
  // then an exact merge of a column group's waves
  wait_loads();
  __syncthreads();
  lsum += __shfl_xor(lsum, 16);
  lsum += __shfl_xor(lsum, 32);
  if (g4 == 0) {
    sml[wave][0][l16] = m;
    sml[wave][1][l16] = lsum;
  }
  constexpr int AW = 16 * D * 4;
  f32x4_t *const mine = reinterpret_cast<f32x4_t *>(area + wave * AW);
  if constexpr (CODES) {
    // (channel 64i + 16g + 4k + e lies in block 4i + e)
#pragma unroll
    for (int i = 0; i < D / 64; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int at = 16 * i + 4 * g4 + k;
        mine[at * 16 + (l16 ^ (at & 15))] = f32x4_t{o[4 * i][k], o[4 * i + 1][k], o[4 * i + 2][k], o[4 * i + 3][k]};
      }
  } else {
#pragma unroll
    for (int vb = 0; vb < VB; ++vb) {
      const int at = 4 * vb + g4;
      mine[at * 16 + (l16 ^ (at & 15))] = o[vb];
    }
  }
  __syncthreads();
  const float back = I8 ? 0x1p6f : F16 ? 0x1p-7f : F == HWKV_KV_FP8_E4M3 ? hd.v_scale : 1.0f;
  const bool whole = nwg == 1 && !block && (rank >= a.n_full || a.seq_block[first] == kNoBlock);
  const size_t part = block ? (size_t)rank * a.block_wgs + local : blockIdx.x;
  for (int idx = threadIdx.x; idx < ncols * (D / 4); idx += WAVES * 64) {
    const int col = idx / (D / 4), at = idx % (D / 4), c = col % 16, w0 = col / 16 * RW;
    float M = sml[w0][0][c];
    for (int w = 1; w < RW; ++w) M = fmaxf(M, sml[w0 + w][0][c]);
    float L = 0.f;
    f32x4_t A = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int w = 0; w < RW; ++w) {
      const float f = exp2f(sml[w0 + w][0][c] - M);
      L += sml[w0 + w][1][c] * f;
      A += reinterpret_cast<const f32x4_t *>(area + (w0 + w) * AW)[at * 16 + (c ^ (at & 15))] * f;
    }
    if (whole) {
      const int64_t row = (int64_t)b0 * a.n_q_heads + h * a.group + col;
      *reinterpret_cast<f32x4_t *>(a.out + row * D + 4 * at) = A * (back / L);
      continue;
    }
    const size_t row = block ? part * CB + col : part * a.group + col;
    *reinterpret_cast<f32x4_t *>((block ? a.block_acc : a.own_acc) + row * D + 4 * at) = A * back;
    if (at == 0) *reinterpret_cast<f32x2_t *>((block ? a.block_ml : a.own_ml) + row * 2) = f32x2_t{M, L};
  }
}

template <int D, int F, int CW>
hipError_t launch_shared(const SharedArgs &a, hipStream_t s) {
  hipLaunchKernelGGL((decode_shared<D, F, CW>), dim3((unsigned)a.wg_begin[a.n_heads]), dim3(shared_threads(CW)), 0, s,
                     a);
  return hipGetLastError();
}

}  // namespace

template <int F>
hipError_t launch_decode_shared_fmt(int D, int n_col_groups, const SharedArgs &a, hipStream_t s) {
#define HWKV_SHARED(DD)                                              \
  switch (n_col_groups) {                                            \
    case 1: return launch_shared<DD, F, 1>(a, s);                    \
    case 2: return launch_shared<DD, F, 2>(a, s);                    \
    case 4: return launch_shared<DD, F, 4>(a, s);                    \
    default: return hipErrorInvalidValue;                            \
  }
  switch (D) {
    case 64: HWKV_SHARED(64)
    case 128: HWKV_SHARED(128)
    case 256: HWKV_SHARED(256)
    default: return hipErrorInvalidValue;
  }
#undef HWKV_SHARED
}

}  // namespace hwkv
