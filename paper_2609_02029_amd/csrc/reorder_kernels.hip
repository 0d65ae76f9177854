// reorder_kernels.hip -- rows and pages of whole sequences copied (gfx950): a
// cache's sequences reordered in place, or a cache taken into another buffer.
//
// Nothing is computed: 16-byte chunks are read and written as they lie, so one
// kernel serves every format and head_dim.  What bounds it: HBM where there is much
// to copy, the launch where there is little.
#include <algorithm>

#include "hwkv_internal.h"

namespace hwkv {
namespace {

typedef uint32_t chunk_t __attribute__((ext_vector_type(4)));

constexpr int64_t kWgChunks = (int64_t)kMoveChunks * 256;
constexpr int kPageParts = 8;        // workgroups that copy a page

__host__ __device__ constexpr int64_t whole_tiles(int64_t rows) {
  return (rows + kTile - 1) / kTile * kTile;
}
// Chunks of 16 bytes of `rows` rows of K (whole tiles), V and the scale pairs.
__host__ __device__ constexpr int64_t part_chunks(int part, int64_t rows, int row_bytes, int pair_bytes) {
  return part == 0 ? whole_tiles(rows) * row_bytes / 16
                   : part == 1 ? rows * row_bytes / 16 : (rows * pair_bytes + 15) / 16;
}

// Every thread holds its chunks of all sequences, so that a permutation in place
// needs no order between threads: a chunk's sources are read before any of its
// destinations is written, within a round by the registers, from round to round by
// the order of the moves (host).  A round is a read and a write of memory in a row, about
// 3.7 us: rounds that touch other sequences are parts of their own, side by side (56
// sequences of 5 rows, 7 rounds: 26.6 us in one part, 7.1 in seven).  32 beams of 1,500
// to 6,000 tokens, 48 units with windows of 1,024: 980 MB in 201 us, 4.9 TB/s, the rate
// of a copy.
template <bool ONE, int M>
__device__ __forceinline__ void move_rows_of(const MoveArgsOf<M> &a, int block, int part_of_moves) {
  const int lane = threadIdx.x & 63;
  const int u = __builtin_amdgcn_readfirstlane(__popcll(__ballot(a.wg_begin[lane] <= block)) - 1);
  const MoveUnit &unit = a.unit[u];
  // the part (K, V, pairs) of this workgroup, by the most rows any move has
  int64_t wg = block - a.wg_begin[u];
  int part = 0;
  for (; part < 2; ++part) {
    const int64_t wgs =
        (part_chunks(part, min(a.most, unit.cap), a.row_bytes, a.pair_bytes) + kWgChunks - 1) / kWgChunks;
    if (wg < wgs) break;
    wg -= wgs;
  }
  const int64_t at = part == 0 ? unit.k_off : part == 1 ? unit.v_off : unit.s_off;
  const int64_t stride = (int64_t)unit.cap_pad * (part == 2 ? a.pair_bytes : a.row_bytes);
  const int64_t first = wg * kWgChunks;
  chunk_t carry[kMoveChunks] = {};
  // (ONE: every part is one round, which needs no carry: 68 registers, not 87, and 203
  // MB in 44 us, not 50)
  const int r0 = a.part[part_of_moves] * kMoveRound;
  const int r1 = ONE ? r0 + kMoveRound : a.part[part_of_moves + 1] * kMoveRound;
  for (int r = r0; r < r1; r += kMoveRound) {
    chunk_t x[kMoveRound][kMoveChunks];
    bool has[kMoveRound][kMoveChunks];
#pragma unroll
    for (int i = 0; i < kMoveRound; ++i) {
      const int src = a.src[r + i];
      // (uniform: the chunks that are left, and where they begin)
      const int n = (int)min(part_chunks(part, min(a.n[r + i], unit.cap), a.row_bytes, a.pair_bytes) - first, kWgChunks);
      const chunk_t *const from = reinterpret_cast<const chunk_t *>(a.from + at + src * stride) + first;
#pragma unroll
      for (int j = 0; j < kMoveChunks; ++j) {
        has[i][j] = (int)threadIdx.x + j * 256 < n;
        if (!ONE && src == kMoveCarry)
          x[i][j] = carry[j];
        else if (has[i][j])
          x[i][j] = from[threadIdx.x + j * 256];
      }
    }
#pragma unroll
    for (int i = 0; i < kMoveRound; ++i) {
      const int dst = a.dst[r + i];
      chunk_t *const to = reinterpret_cast<chunk_t *>(a.to + at + dst * stride) + first;
#pragma unroll
      for (int j = 0; j < kMoveChunks; ++j) {
        if (!has[i][j]) continue;
        if (!ONE && dst == kMoveCarry)
          carry[j] = x[i][j];
        else
          to[threadIdx.x + j * 256] = x[i][j];
      }
    }
  }
}

template <bool ONE>
__global__ __launch_bounds__(256) void move_rows(MoveArgs a) {
  move_rows_of<ONE>(a, blockIdx.x, blockIdx.y);
}

// Part `part` of kPageParts of a page's first `rows` rows.
__device__ __forceinline__ void copy_page(const uint8_t *from, uint8_t *to, int part, int rows, int row_bytes,
                                          int pair_bytes) {
  const int k = (int)part_chunks(0, rows, row_bytes, pair_bytes);
  const int v = (int)part_chunks(1, rows, row_bytes, pair_bytes);
  const int all = k + v + (int)part_chunks(2, rows, row_bytes, pair_bytes);
  const int v_at = kPageTokens * row_bytes / 16, s_at = 2 * v_at;
  const chunk_t *const src = reinterpret_cast<const chunk_t *>(from);
  chunk_t *const dst = reinterpret_cast<chunk_t *>(to);
  constexpr int step = kPageParts * 256;
  for (int c = part * 256 + (int)threadIdx.x; c < all; c += 4 * step) {
    chunk_t x[4];
    int at[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int ci = c + i * step;
      at[i] = ci < k ? ci : ci < k + v ? v_at + ci - k : s_at + ci - k - v;
      if (ci < all) x[i] = src[at[i]];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c + i * step < all) dst[at[i]] = x[i];
  }
}

__host__ __device__ constexpr int64_t page_bytes(int row_bytes, int pair_bytes) {
  return (int64_t)kPageTokens * (2 * row_bytes + pair_bytes);
}

// kPageParts workgroups a copy, and one that installs the entries.
template <int N, int E>
__device__ __forceinline__ void pages_of(const PageCopyArgsOf<N, E> &a, int block) {
  const int i = block / kPageParts;
  if (i == a.n_copies) {
    for (int e = threadIdx.x; e < a.n_entries; e += 256) a.table[a.idx[e]] = a.page[e];
    for (int e = threadIdx.x; e < a.n_copies; e += 256) a.table[a.at[e]] = a.dst[e];
    return;
  }
  const int64_t page = page_bytes(a.row_bytes, a.pair_bytes);
  copy_page(a.pool + a.src[i] * page, a.pool + a.dst[i] * page, block % kPageParts, a.rows[i], a.row_bytes,
            a.pair_bytes);
}
__global__ __launch_bounds__(256) void page_copy(PageCopyArgs a) { pages_of(a, blockIdx.x); }

// As move_rows, for the page table: a thread holds entry j of every row of a unit.  Grid:
// (entries / 256, units, parts).
__global__ __launch_bounds__(256) void table_move(TableMoveArgs a) {
  const int j = blockIdx.x * 256 + threadIdx.x;
  int32_t *const rows = a.table + (int64_t)blockIdx.y * a.batch * a.max_pages + j;
  int32_t carry = 0;
  for (int r = a.part[blockIdx.z] * kMoveRound; r < a.part[blockIdx.z + 1] * kMoveRound; r += kMoveRound) {
    int32_t x[kMoveRound] = {};
#pragma unroll
    for (int i = 0; i < kMoveRound; ++i) {
      const int src = a.src[r + i];
      if (j < a.pages[r + i]) x[i] = src == kMoveCarry ? carry : rows[(int64_t)src * a.max_pages];
    }
#pragma unroll
    for (int i = 0; i < kMoveRound; ++i) {
      const int dst = a.dst[r + i];
      if (j >= a.pages[r + i]) continue;
      if (dst == kMoveCarry)
        carry = x[i];
      else
        rows[(int64_t)dst * a.max_pages] = x[i];
    }
  }
}

// kPageParts workgroups a page.
template <int N>
__device__ __forceinline__ void pages_of(const PageMoveArgsOf<N> &a, int block) {
  const int lane = threadIdx.x & 63, p = block / kPageParts, part = block % kPageParts;
  int run = -1;
  for (int i = 0; i < N; i += 64) run += __popcll(__ballot(i + lane < N && a.run[min(i + lane, N - 1)].begin <= p));
  const PageRun r = a.run[__builtin_amdgcn_readfirstlane(run)];
  const int j = p - r.begin, dst = r.dst0 + j;
  const int src = a.from_table[r.pto + r.j0 + j];
  if (part == 0 && threadIdx.x == 0) a.to_table[r.pto + r.j0 + j] = dst;
  if (!r.copy) return;
  const int64_t page = page_bytes(a.row_bytes, a.pair_bytes);
  copy_page(a.from_pool + src * page, a.to_pool + dst * page, part, kPageTokens, a.row_bytes, a.pair_bytes);
}
__global__ __launch_bounds__(256) void page_move(PageMoveArgs a) { pages_of(a, blockIdx.x); }

// Few moves and few pages: a launch of its own for the pages is 3 us of a call of 11.
template <bool ONE, typename Pages>
__global__ __launch_bounds__(256) void few(FewMoves m, Pages p, int wgs) {
  const int rows = wgs * m.n_parts;
  if ((int)blockIdx.x < rows) move_rows_of<ONE>(m, blockIdx.x % wgs, blockIdx.x / wgs);
  else pages_of(p, blockIdx.x - rows);
}

int page_wgs(const FewPageCopies &p) { return p.n_copies * kPageParts + 1; }
int page_wgs(const FewPageMoves &p) { return p.n_pages * kPageParts; }

template <int N>
int last_wg(const MoveArgsOf<N> &a) {
  int n = 0;
  while (n < kMaxItems && a.wg_begin[n + 1] != INT32_MAX) ++n;
  return a.wg_begin[n];
}

template <typename Pages>
hipError_t launch_few_of(const FewMoves &m, const Pages &p, hipStream_t s) {
  const int wgs = last_wg(m);
  const dim3 grid((unsigned)(wgs * m.n_parts + page_wgs(p)));
  if (m.part[m.n_parts] == m.n_parts) hipLaunchKernelGGL((few<true, Pages>), grid, dim3(256), 0, s, m, p, wgs);
  else hipLaunchKernelGGL((few<false, Pages>), grid, dim3(256), 0, s, m, p, wgs);
  return hipGetLastError();
}

}  // namespace

int64_t move_workgroups(int64_t rows, int32_t row_bytes, int32_t pair_bytes) {
  int64_t n = 0;
  for (int part = 0; part < 3; ++part)
    n += (part_chunks(part, rows, row_bytes, pair_bytes) + kWgChunks - 1) / kWgChunks;
  return n;
}

hipError_t launch_move_rows(const MoveArgs &a, hipStream_t s) {
  const int n = last_wg(a);
  if (n == 0) return hipSuccess;
  const dim3 grid((unsigned)n, (unsigned)a.n_parts);
  if (a.part[a.n_parts] == a.n_parts) hipLaunchKernelGGL(move_rows<true>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(move_rows<false>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_few(const FewMoves &m, const FewPageCopies &p, hipStream_t s) { return launch_few_of(m, p, s); }
hipError_t launch_few(const FewMoves &m, const FewPageMoves &p, hipStream_t s) { return launch_few_of(m, p, s); }

hipError_t launch_table_move(const TableMoveArgs &a, int n_units, hipStream_t s) {
  hipLaunchKernelGGL(table_move, dim3((unsigned)((a.most + 255) / 256), (unsigned)n_units, (unsigned)a.n_parts),
                     dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_page_copy(const PageCopyArgs &a, hipStream_t s) {
  const int wgs = a.n_copies * kPageParts + 1;
  hipLaunchKernelGGL(page_copy, dim3((unsigned)wgs), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_page_move(const PageMoveArgs &a, hipStream_t s) {
  if (a.n_pages == 0) return hipSuccess;
  hipLaunchKernelGGL(page_move, dim3((unsigned)(a.n_pages * kPageParts)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace hwkv
