// decode_shared_merge.hip -- the merge of decode attention over shared pages
// (decode_shared.h), and the launchers of both phases.
#include <cfloat>

#include "decode_split.h"

namespace hwkv {

// Instantiated in the per-format sources.
extern template hipError_t launch_decode_shared_fmt<HWKV_KV_BF16>(int, const SharedArgs &, hipStream_t);
extern template hipError_t launch_decode_shared_fmt<HWKV_KV_F16>(int, const SharedArgs &, hipStream_t);
extern template hipError_t launch_decode_shared_fmt<HWKV_KV_FP8_E4M3>(int, const SharedArgs &, hipStream_t);
extern template hipError_t launch_decode_shared_fmt<HWKV_KV_I8>(int, const SharedArgs &, hipStream_t);

namespace {

// Workgroup j of n of turn `turn`, among all of a block's.
__device__ __forceinline__ int block_wg(int j, int turn, int n, int turns) {
  return (j & ~7) * turns + turn * min(8, n - (j & ~7)) + (j & 7);
}

// One workgroup per (sequence, q head): rows of D / 4 lanes take every R-th part, a
// lane 4 channels, and meet in LDS.
template <int D>
__global__ __launch_bounds__(512) void shared_merge(SharedArgs a) {
  constexpr int LPR = D / 4, R = 512 / LPR;
  constexpr int U = 4;                           // parts per round, loads in flight
  __shared__ __attribute__((aligned(16))) f32x4_t acc_s[512];
  __shared__ float m_s[R], l_s[R];
  const int i = blockIdx.x, rank = blockIdx.y / a.group, g = blockIdx.y % a.group;
  // parts: of the sequence's block, then its own
  const int width = 16 * a.col_groups;
  int nb = 0, no, own0, step = 1, turns = 1, turn = 0, block0 = 0, col = 0;
  if (rank < a.n_full) {
    const int b = a.seq_block[i];
    if (b != kNoBlock) {
      col = (i - a.block_first[b]) * a.group + g;
      turns = (a.block_count[b] * a.group + width - 1) / width;
      turn = col / width;
      nb = (a.item_begin[b + 1] - a.item_begin[b]) / turns;
      block0 = a.item_begin[b] * a.n_full;
    }
    own0 = a.item_begin[a.n_blocks + i];
    no = a.item_begin[a.n_blocks + i + 1] - own0;
    own0 -= a.block_wgs;
  } else {
    const int tiles = (min(a.len[i], a.head[rank].cap) + 63) / 64;
    no = (tiles + a.tiles_per_wg - 1) / a.tiles_per_wg;
    own0 = i;
    step = a.n_seqs;
  }
  if (nb == 0 && no == 1) return;                // uniform: written whole
  const int n = nb + no;
  const int row = threadIdx.x / LPR, c = threadIdx.x % LPR * 4;
  float M = -FLT_MAX, L = 0.f;
  f32x4_t A = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = row; j0 < n; j0 += U * R) {
    f32x2_t ml[U];
    f32x4_t x[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int j = min(j0 + k * R, n - 1);
      const bool of_block = j < nb;
      const size_t p = of_block ? (size_t)(block0 + block_wg(rank * nb + j, turn, nb * a.n_full, turns)) * width + col % width
                                : (size_t)(a.wg_begin[rank] + own0 + (j - nb) * step) * a.group + g;
      ml[k] = *reinterpret_cast<const f32x2_t *>((of_block ? a.block_ml : a.own_ml) + p * 2);
      x[k] = *reinterpret_cast<const f32x4_t *>((of_block ? a.block_acc : a.own_acc) + p * D + c);
    }
    float Mn = M;
#pragma unroll
    for (int k = 0; k < U; ++k) Mn = fmaxf(Mn, ml[k].x);
    const float f = exp2f(M - Mn);
    L *= f;
    A *= f;
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const float e = j0 + k * R < n ? exp2f(ml[k].x - Mn) : 0.f;
      if (j0 + k * R < n) {
        L += ml[k].y * e;
        A += x[k] * e;
      }
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
  const int rows = min(R, n);                    // those that had a part
  for (int r = 1; r < rows; ++r) M = fmaxf(M, m_s[r]);
  L = 0.f;
  A = f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int r = 0; r < rows; ++r) {
    const float f = exp2f(m_s[r] - M);
    L += l_s[r] * f;
    A += acc_s[r * LPR + threadIdx.x] * f;
  }
  const int64_t to = (int64_t)a.seq[i] * a.n_q_heads + a.head_id[rank] * a.group + g;
  *reinterpret_cast<f32x4_t *>(a.out + to * D + c) = A * (1.0f / L);
}

}  // namespace

hipError_t launch_decode_shared(int fmt, int D, const SharedArgs &a, hipStream_t s) {
  switch (fmt) {
    case HWKV_KV_BF16: return launch_decode_shared_fmt<HWKV_KV_BF16>(D, a, s);
    case HWKV_KV_F16: return launch_decode_shared_fmt<HWKV_KV_F16>(D, a, s);
    case HWKV_KV_FP8_E4M3: return launch_decode_shared_fmt<HWKV_KV_FP8_E4M3>(D, a, s);
    case HWKV_KV_I8: return launch_decode_shared_fmt<HWKV_KV_I8>(D, a, s);
    default: return hipErrorInvalidValue;
  }
}

hipError_t launch_shared_merge(int D, const SharedArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)a.n_seqs, (unsigned)(a.n_heads * a.group));
  switch (D) {
    case 64: hipLaunchKernelGGL(shared_merge<64>, grid, dim3(512), 0, s, a); break;
    case 128: hipLaunchKernelGGL(shared_merge<128>, grid, dim3(512), 0, s, a); break;
    case 256: hipLaunchKernelGGL(shared_merge<256>, grid, dim3(512), 0, s, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace hwkv
