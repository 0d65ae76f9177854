// decode_shared.h -- decode attention of sequences that share pages of a paged
// cache (gfx950, matrix cores), for every cache format; instantiated once per
// format by decode_shared_<format>.hip.
//
// The sequences of a fork hold the same pages up to where they parted.  An item of
// work is a run of rows of one KV head and the query columns that see all of them:
//   a block   the pages that a group of sequences shares, with the q heads of all of
//             its members, in groups of 16 columns;
//   an own    a sequence's rows from there on, a window's rows, or all the rows of
//             a sequence that shares nothing, with its own q heads.
// Every item is split over workgroups, workgroup j of n taking its tiles of 64 rows
// j, j + n, ..; each leaves (m, l, acc) of its columns, and shared_merge adds, for
// every q head of a sequence, the parts of its block and its own:
//     out = sum_j acc_j 2^(m_j - M) / sum_j l_j 2^(m_j - M),  M = max m_j.
//
// A workgroup has N groups of 16 columns, 1 to 3 (a block of more is read once for every
// N); a wavefront has a quarter of every tile's rows and all of these columns, with an
// online softmax of its own, and the four meet in LDS at the end.
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
// four tiles).  Each wave loads, and reads into registers, its own rows: no barrier
// falls inside the walk.  N = 1: one stage, whose successor's loads are issued as soon as
// it is in registers, and two workgroups a CU.  N > 1: two stages, one workgroup a CU,
// and up to 512 registers a wave: at head_dim 256 the accumulators take 64 N, and V is
// read only after the logits (before them the kernel of three groups spilled, and each
// spilled register's load waited for all rows in flight: 265 us instead of 91).
//
// What bounds it: HBM at 16 bits, as long as a block's rows are read once: 4 KV heads of
// 256 x 6, all full, 112,000 rows (476 MB) with 2, 5 and 8 sequences (1, 2 and 3 column
// groups) take 82.6, 85.5 and 98.6 us, 5.8 to 4.8 TB/s.  Column groups in workgroups of
// their own, side by side on the same L2, took 115 and 150 us: the L2 gave a third of the
// rows a second time, and the rest came from memory again.  At 8 bits (238 MB) the
// widening of codes and the products: fp8 50, 55 and 71 us, int8 53, 64 and 81.
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

// Eight consecutive codes as 8 bf16 values; of int8 in the order 0 4 1 5 2 6 3 7 (which
// widens a code with 1.5 instructions, not 2.5; q's channels lie alike).
template <int F>
__device__ __forceinline__ u32x4_t widen_codes(u32x2_t c) {
  if constexpr (F == HWKV_KV_I8)
    return u32x4_t{codes_bf16x2<0>(c.x, c.y), codes_bf16x2<1>(c.x, c.y), codes_bf16x2<2>(c.x, c.y),
                   codes_bf16x2<3>(c.x, c.y)};
  else
    return u32x4_t{fp8x2_bf16x2<false>(c.x), fp8x2_bf16x2<true>(c.x), fp8x2_bf16x2<false>(c.y),
                   fp8x2_bf16x2<true>(c.y)};
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

template <int D, int F, int N>
__global__ __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(N == 1 ? 2 : 1, N == 1 ? 2 : 1)))
void decode_shared(SharedArgs a) {
  constexpr bool CODES = KvFormat<F>::kBytes == 1, I8 = F == HWKV_KV_I8, F16 = F == HWKV_KV_F16;
  constexpr int EB = KvFormat<F>::kBytes;
  constexpr int NC = D / 8;            // chunks of a row
  constexpr int KS = D / 32;           // products over the channels
  constexpr int VB = D / 16;           // channel blocks
  constexpr int ROW = D * EB;
  constexpr int PCS = ROW / 16;        // 16-byte pieces of a V row
  constexpr int P = shared_tiles(ROW); // tiles of a stage; a wave has 16 rows of each
  constexpr int KB = 64 * ROW;         // K, or V, of a tile
  constexpr int TB = 2 * KB + (I8 ? 1024 : 0);   // and scale pairs
  constexpr int BUFS = N == 1 ? 1 : 2, STAGE = P * TB;
  static_assert(kWaves == 4, "16 rows of a tile a wave");
  static_assert(STAGE >= kWaves * 16 * D * 4, "16 columns of acc a wave, at the end");
  __shared__ __attribute__((aligned(1024))) uint8_t area[BUFS * STAGE];
  __shared__ __attribute__((aligned(16))) u32x4_t q_s[N * KS * 64];
  __shared__ float back_s[N * 16][2];      // what a column's logits are multiplied by
  __shared__ float sml[kWaves][2][16];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int g4 = lane >> 4, l16 = lane & 15;
  // ---- the item
  int rank = __builtin_amdgcn_readfirstlane(__popcll(__ballot(a.wg_begin[lane] <= (int)blockIdx.x)) - 1);
  const bool block = rank < 0;
  int first, count = 1, row0 = 0, end, j, nwg, col0 = 0;
  if (rank < a.n_full) {
    const int local = block ? (int)blockIdx.x : blockIdx.x - a.wg_begin[rank] + a.block_wgs;
    const int heads = block ? a.n_full : 1;      // that share item_begin's range
    int item = -1;
#pragma unroll
    for (int i = 0; i < kSharedItems; i += 64)
      item += __popcll(__ballot(a.item_begin[i + lane] * heads <= local));
    item = __builtin_amdgcn_readfirstlane(item);
    nwg = a.item_begin[item + 1] - a.item_begin[item];
    j = local - a.item_begin[item] * heads;
    if (block) {
      // (the heads' workgroups in one row, eight of a column group after eight of
      // another)
      first = a.block_first[item];
      count = a.block_count[item];
      end = a.block_pages[item] * kPageTokens;
      const int turns = (count * a.group + 16 * N - 1) / (16 * N), round = j / (8 * turns), at = j - round * 8 * turns;
      nwg /= turns;
      const int n = min(8, nwg * heads - 8 * round);
      j = 8 * round + at % n;
      col0 = at / n * (16 * N);
      rank = j / nwg;
      j -= rank * nwg;
    } else {
      first = item - a.n_blocks;
      end = a.len[first];
      if (a.seq_block[first] != kNoBlock) row0 = a.block_pages[a.seq_block[first]] * kPageTokens;
    }
  } else {
    const int local = blockIdx.x - a.wg_begin[rank];
    first = local % a.n_seqs;
    j = local / a.n_seqs;
    end = min(a.len[first], a.head[rank].cap);
    nwg = ((end + 63) / 64 + a.tiles_per_wg - 1) / a.tiles_per_wg;
    if (j >= nwg) return;              // uniform: a shorter sequence
  }
  const ItemHead &hd = a.head[rank];
  const int h = a.head_id[rank];
  const int ncols = min(16 * N, count * a.group - col0);
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
  // ---- loads, 1 KB each: the wave's 16 rows of every chunk of K, chunk by chunk, and
  // its rows of V, each row's pieces turned (by 32 bytes from row to row at 16 bits) so
  // that the rows that are read together lie in different banks; of codes, LDS row
  // 4i + g of 16 holds row 4g + i.
  auto piece_xor = [](int r) {
    if constexpr (CODES) return D == 256 ? 4 * (r & 3) : D == 128 ? 4 * ((r & 3) >> 1) : 0;
    return D == 64 ? 2 * (r >> 1 & 3) : 2 * (r & 7);
  };
  constexpr int RPL = 1024 / ROW;      // V rows of a load
  constexpr int LOADS = KB / 4096;     // the wave's loads of a tile's K, or V
  const uint32_t area0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)area + wave * (KB / 4);
  const int kl = CODES ? lane / 8 * 512 + 128 * wave + lane % 8 * 16 : g4 * 1024 + (16 * wave + l16) * 16;
  int vl[LOADS];
#pragma unroll
  for (int n = 0; n < LOADS; ++n) {
    const int r = n * RPL + lane / PCS, row = CODES ? 4 * (r & 3) + (r >> 2) : r;
    vl[n] = (16 * wave + row) * ROW + ((lane % PCS) ^ piece_xor(r)) * 16;
  }
  const int sl = lane < 32 ? 4 * lane : 1 << 20;
  // The loads of tiles i0 .. i0 + P - 1; of those past the last nothing is read.
  auto issue = [&](int i0, int buf) {
    if (i0 % 64 == 0 && j + i0 * nwg < n_tiles) look_up(i0);
#pragma unroll
    for (int t = 0; t < P; ++t) {
      const int lt = j + (i0 + t) * nwg, rows = lt < n_tiles ? min(64, end - 64 * (tile0 + lt)) : 0;
      const Tile at = tile(i0 + t);
      const __amdgpu_buffer_rsrc_t kr = make_rsrc(at.k, rows > 0 ? (uint32_t)KB : 0u);
      const __amdgpu_buffer_rsrc_t vr = make_rsrc(at.v, (uint32_t)(rows * ROW));
      const uint32_t into = area0 + buf * STAGE + t * TB;
#pragma unroll
      for (int n = 0; n < LOADS; ++n) stage_lds<false>(kr, into + n * 1024, kl, n * 4096);
#pragma unroll
      for (int n = 0; n < LOADS; ++n) stage_lds<false>(vr, into + KB + n * 1024, vl[n], 0);
      // (every wave has the tile's pairs, in a place of its own)
      if constexpr (I8)
        stage_lds<true>(make_rsrc(at.s, rows > 0 ? 64u * kRowScaleBytes : 0u),
                        into - wave * (KB / 4 - 256) + 2 * KB, sl, 0);
    }
  };
  issue(0, 0);
  if constexpr (BUFS == 2) issue(P, 1);

  // ---- q: column c is q head c mod G of the block's member c / G.  Over binary16
  // and int8 rows a column is scaled by a power of two, that of its largest |q|: to
  // [2^14, 2^15), so that binary16 holds it, or to [1, 2), so that sums over codes
  // stay in fp32's range.
  for (int i = threadIdx.x; i < N * 16 * NC; i += kWaves * 64) {
    const int c = i / NC, ch = i % NC;
    uint4 x = make_uint4(0u, 0u, 0u, 0u);
    if (c < ncols) {
      const int col = col0 + c;
      const int64_t row = (int64_t)a.seq[first + col / a.group] * a.n_q_heads + h * a.group + col % a.group;
      x = *reinterpret_cast<const uint4 *>(a.q + row * D + ch * 8);
    }
    u32x4_t y = {x.x, x.y, x.z, x.w};
    float near = a.scale_log2, rest = 1.0f;
    if constexpr (F16 || I8) {
      const uint32_t top = group_max<NC>(top8(x));
      const int sh = (F16 ? 141 : 127) - (int)max(top >> 7, 1u);
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
      float f[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] = ldexpf(k % 2 ? bf_hi(w[k / 2]) : bf_lo(w[k / 2]), sh);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (F16) {
          const f16x2_t v = {(_Float16)f[2 * k], (_Float16)f[2 * k + 1]};
          y[k] = __builtin_bit_cast(uint32_t, v);
        } else {
          y[k] = pack_bf16x2(f[k], f[k + 4]);
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
    q_s[(c / 16 * KS + ch / 4) * 64 + ch % 4 * 16 + c % 16] = y;
    if (ch == 0) {
      back_s[c][0] = near;
      back_s[c][1] = rest;
    }
  }
  // (the barriers of this phase wait for LDS alone: the first stage stays in flight)
  wait_reads();
  meet();
  u32x4_t q[N == 1 ? KS : 1];
  float near[N], rest[N];
  if constexpr (N == 1)
#pragma unroll
    for (int i = 0; i < KS; ++i) q[i] = q_s[i * 64 + lane];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    near[n] = back_s[16 * n + l16][0];
    rest[n] = back_s[16 * n + l16][1];
  }

  // ---- the walk.  m: running shift of the lane's column (base 2), raised where a
  // logit passes it by 8, so that weights stay below 2^8; it begins below every
  // finite logit.
  float m[N], lsum[N];
  f32x4_t o[N][VB];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    m[n] = -FLT_MAX;
    lsum[n] = 0.0f;
#pragma unroll
    for (int vb = 0; vb < VB; ++vb) o[n][vb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  // a stage, for the first GN groups
  auto stage = [&](auto gn, int i0, int buf) {
    constexpr int GN = decltype(gn)::value;
    const uint8_t *const at = area + buf * STAGE;
    wait_all_but<(BUFS - 1) * P * (2 * LOADS + I8)>();
    u32x4_t kf[CODES ? 1 : P][KS];
    u32x2_t kc[CODES ? P : 1][KS];
    u32x2_t vf[CODES ? 1 : P][VB];
    uint32_t vc[CODES ? P : 1][CODES ? D / 64 : 1][4];
    u32x2_t pairs[P];
    int left[P];                       // of the lane's rows, from its first on
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const uint8_t *const k = at + p * TB + wave * (KB / 4);
      const int lt = j + (i0 + p) * nwg;
      left[p] = lt < n_tiles ? end - (64 * (tile0 + lt) + 16 * wave + 4 * g4) : 0;
      if constexpr (I8)
        pairs[p] = *reinterpret_cast<const u32x2_t *>(at + p * TB + 2 * KB + wave * 256 + 32 * wave + 8 * g4);
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        if constexpr (CODES) kc[p][i] = *reinterpret_cast<const u32x2_t *>(k + (4 * i + g4) * 128 + l16 * 8);
        else kf[p][i] = *reinterpret_cast<const u32x4_t *>(k + i * 1024 + lane * 16);
      }
    }
    auto read_v = [&]() {
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const uint8_t *const v = at + p * TB + wave * (KB / 4) + KB;
        if constexpr (CODES) {
#pragma unroll
          for (int i = 0; i < D / 64; ++i)
#pragma unroll
            for (int n = 0; n < 4; ++n)
              vc[p][i][n] = *reinterpret_cast<const uint32_t *>(v + (4 * n + g4) * D +
                                                                ((4 * i + l16 / 4) ^ piece_xor(g4)) * 16 + l16 % 4 * 4);
        } else {
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
      wait_reads();
      issue(i0 + BUFS * P, buf);
    };
    if constexpr (N == 1) read_v();

    // logits (a product that adds to the one before it waits out its latency: two
    // sums where there are no others)
    constexpr int CH = P * GN == 1 ? 2 : 1;
    f32x4_t z[GN][P], zz[GN][P][CH];
#pragma unroll
    for (int n = 0; n < GN; ++n)
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int c = 0; c < CH; ++c) zz[n][p][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      u32x4_t k[P];
#pragma unroll
      for (int p = 0; p < P; ++p) {
        if constexpr (CODES) k[p] = widen_codes<F>(kc[p][i]);
        else k[p] = kf[p][i];
      }
#pragma unroll
      for (int n = 0; n < GN; ++n) {
        u32x4_t qn;
        if constexpr (N == 1) qn = q[i];
        else qn = q_s[(n * KS + i) * 64 + lane];
#pragma unroll
        for (int p = 0; p < P; ++p) zz[n][p][i % CH] = product<F>(k[p], qn, zz[n][p][i % CH]);
      }
    }
    // (rows past the item's end have no weight)
    float top[GN];
    bool raise = false;
#pragma unroll
    for (int n = 0; n < GN; ++n) {
      top[n] = -FLT_MAX;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        z[n][p] = zz[n][p][0];
        if constexpr (CH == 2) z[n][p] += zz[n][p][1];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x = z[n][p][i] * near[n];
          if constexpr (I8) x *= __uint_as_float(((i < 2 ? pairs[p].x : pairs[p].y) >> (16 * (i & 1)) & 255u) << 23);
          if constexpr (I8 || F16) x *= rest[n];
          z[n][p][i] = i < left[p] ? x : -INFINITY;
          top[n] = fmaxf(top[n], z[n][p][i]);
        }
      }
      top[n] = max_of_rows(top[n]);
      raise |= top[n] > m[n] + 8.0f;
    }
    if (__any(raise)) {
#pragma unroll
      for (int n = 0; n < GN; ++n) {
        const float mn = fmaxf(m[n], top[n]), f = exp2f(m[n] - mn);
        m[n] = mn;
        lsum[n] *= f;
#pragma unroll
        for (int vb = 0; vb < VB; ++vb) o[n][vb] *= f;
      }
    }
    u32x2_t term[GN][P][F16 ? 2 : 3];
#pragma unroll
    for (int n = 0; n < GN; ++n)
#pragma unroll
      for (int p = 0; p < P; ++p) {
        float w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w[i] = __builtin_amdgcn_exp2f(z[n][p][i] - m[n]);
          lsum[n] += w[i];
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
          term[n][p][0] = u32x2_t{__builtin_bit_cast(uint32_t, a0), __builtin_bit_cast(uint32_t, a1)};
          term[n][p][1] = u32x2_t{__builtin_bit_cast(uint32_t, r0), __builtin_bit_cast(uint32_t, r1)};
        } else {
#pragma unroll
          for (int k = 0; k < 3; ++k) {
            const u32x2_t x = {pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3])};
            term[n][p][k] = x;
            w[0] -= bf_lo(x.x);
            w[1] -= bf_hi(x.x);
            w[2] -= bf_lo(x.y);
            w[3] -= bf_hi(x.y);
          }
        }
      }
    if constexpr (N > 1) {
      __builtin_amdgcn_sched_barrier(0);
      read_v();
    }
    // values: term by term over two parts; of a single part, the first two terms over
    // the same V, then the third.  (The product of 16 places takes as long as that of
    // 32; and compiled right behind one of 32 into the same accumulator, with no wait
    // between, it gave wrong sums.)
    constexpr int TERMS = F16 ? 2 : 3, STEPS = P == 1 ? TERMS - 1 : TERMS;
    auto add = [&](int n, int step, int vb, const u32x2_t (&v)[P]) {
      if constexpr (P == 1) {
        const u32x2_t x = term[n][0][2 * step], y = step == 0 ? term[n][0][1] : u32x2_t{0u, 0u};
        o[n][vb] = product<F>(u32x4_t{v[0].x, v[0].y, v[0].x, v[0].y}, u32x4_t{x.x, x.y, y.x, y.y}, o[n][vb]);
      } else {
#pragma unroll
        for (int p = 0; p < P; p += 2) {
          const u32x2_t x = term[n][p][step], y = term[n][p + 1][step];
          o[n][vb] = product<F>(u32x4_t{v[p].x, v[p].y, v[p + 1].x, v[p + 1].y}, u32x4_t{x.x, x.y, y.x, y.y}, o[n][vb]);
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
          for (int n = 0; n < GN; ++n)
#pragma unroll
            for (int i = 0; i < D / 64; ++i) add(n, step, 4 * i + e, v[i]);
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
        for (int n = 0; n < GN; ++n)
#pragma unroll
          for (int step = 0; step < STEPS; ++step)
#pragma unroll
            for (int vb = v0; vb < VB && vb < v0 + 8; ++vb) add(n, step, vb, v[vb]);
    }
  };
  const auto walk = [&](auto gn) {
    int buf = 0;
    for (int i0 = 0; j + i0 * nwg < n_tiles; i0 += P) {
      stage(gn, i0, buf);
      if constexpr (BUFS == 2) buf ^= 1;
    }
  };
  if (N > 1 && ncols <= 16) walk(std::integral_constant<int, 1>{});
  else walk(std::integral_constant<int, N>{});

  // ---- the workgroup's result, a column group at a time: every wave's acc in an area of
  // its own (after the last, empty, loads have landed), 4 channels q of column c at
  // place c ^ q of 16, then an exact merge of the waves
  wait_loads();
  constexpr int AW = 16 * D * 4;
  f32x4_t *const mine = reinterpret_cast<f32x4_t *>(area + wave * AW);
  const float back = I8 ? 0x1p6f : F16 ? 0x1p-7f : F == HWKV_KV_FP8_E4M3 ? hd.v_scale : 1.0f;
  const bool whole = nwg == 1 && !block && (rank >= a.n_full || a.seq_block[first] == kNoBlock);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (16 * n >= ncols) break;
    __syncthreads();
    lsum[n] += __shfl_xor(lsum[n], 16);
    lsum[n] += __shfl_xor(lsum[n], 32);
    if (g4 == 0) {
      sml[wave][0][l16] = m[n];
      sml[wave][1][l16] = lsum[n];
    }
    if constexpr (CODES) {
      // (channel 64i + 16g + 4k + e lies in block 4i + e)
#pragma unroll
      for (int i = 0; i < D / 64; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int at = 16 * i + 4 * g4 + k;
          mine[at * 16 + (l16 ^ (at & 15))] =
              f32x4_t{o[n][4 * i][k], o[n][4 * i + 1][k], o[n][4 * i + 2][k], o[n][4 * i + 3][k]};
        }
    } else {
#pragma unroll
      for (int vb = 0; vb < VB; ++vb) {
        const int at = 4 * vb + g4;
        mine[at * 16 + (l16 ^ (at & 15))] = o[n][vb];
      }
    }
    __syncthreads();
    for (int idx = threadIdx.x; idx < min(16, ncols - 16 * n) * (D / 4); idx += kWaves * 64) {
      const int c = idx / (D / 4), at = idx % (D / 4);
      float M = sml[0][0][c];
      for (int w = 1; w < kWaves; ++w) M = fmaxf(M, sml[w][0][c]);
      float L = 0.f;
      f32x4_t A = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = exp2f(sml[w][0][c] - M);
        L += sml[w][1][c] * f;
        A += reinterpret_cast<const f32x4_t *>(area + w * AW)[at * 16 + (c ^ (at & 15))] * f;
      }
      if (whole) {
        const int64_t row = (int64_t)b0 * a.n_q_heads + h * a.group + c;
        *reinterpret_cast<f32x4_t *>(a.out + row * D + 4 * at) = A * (back / L);
        continue;
      }
      const size_t row = block ? (size_t)blockIdx.x * (16 * N) + 16 * n + c : (size_t)blockIdx.x * a.group + c;
      *reinterpret_cast<f32x4_t *>((block ? a.block_acc : a.own_acc) + row * D + 4 * at) = A * back;
      if (at == 0) *reinterpret_cast<f32x2_t *>((block ? a.block_ml : a.own_ml) + row * 2) = f32x2_t{M, L};
    }
  }
}

template <int D, int F>
hipError_t launch_shared(const SharedArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)a.wg_begin[a.n_heads]);
  switch (a.col_groups) {
    case 1: hipLaunchKernelGGL((decode_shared<D, F, 1>), grid, dim3(kWaves * 64), 0, s, a); break;
    case 2: hipLaunchKernelGGL((decode_shared<D, F, 2>), grid, dim3(kWaves * 64), 0, s, a); break;
    case 3: hipLaunchKernelGGL((decode_shared<D, F, 3>), grid, dim3(kWaves * 64), 0, s, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace

template <int F>
hipError_t launch_decode_shared_fmt(int D, const SharedArgs &a, hipStream_t s) {
  switch (D) {
    case 64: return launch_shared<64, F>(a, s);
    case 128: return launch_shared<128, F>(a, s);
    case 256: return launch_shared<256, F>(a, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace hwkv
