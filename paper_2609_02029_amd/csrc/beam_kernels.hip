// beam_kernels.hip -- beam search's choice over beams and vocabulary (gfx950).
//
// With the logits x[b, t] of a group's beams b and their running scores s[b],
//     lse[b] = log sum_t e^x[b, t],   score(b, t) = s[b] + (x[b, t] - lse[b]),
// the n largest scores of a group, falling, ties to the lowest b * vocab + t.
//
// Two launches.  beam_scan reads every logit once, with several workgroups a row,
// and leaves the row's partial sums of e^x and the largest logit of each block of
// 64 chunks of 16 bytes.
// beam_pick, a workgroup per group, joins the sums and finds the n largest from
// the blocks' maxima: the blocks in the order (score of the largest falling, place
// rising), an element of a block behind the n-th has n elements before it, the
// largest of each of the n blocks.  So n blocks are read again, and no others.
//
// Sums and scores are 64-bit: two beams' tokens are ordered by scores that differ
// by their lse, and an fp32 sum (off by 1e-7) would swap near ones.  2^f is a
// polynomial of degree 8, 1.1e-12 off, on [-1/2, 1/2], and the power of two goes
// into the exponent's bits: 14 64-bit operations a logit, at the rate of fp32's.
#include <algorithm>

#include "hwkv.h"
#include "hwkv_internal.h"

namespace hwkv {
namespace {

constexpr int kScanWaves = 4, kScanDeep = 4;   // waves; blocks a wave has in flight
constexpr double kLog2e = 0x1.71547652b82fep+0;
constexpr float kInf = __builtin_inff();

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef u32x4_t __attribute__((aligned(2))) chunk_t;

template <int T>
constexpr int kBytes = T == HWKV_LOGITS_F32 ? 4 : 2;
template <int T>
constexpr int kPerChunk = 16 / kBytes<T>;

// Element e of a chunk.
template <int T>
__device__ __forceinline__ float element(const u32x4_t &c, int e) {
  if constexpr (T == HWKV_LOGITS_F32) {
    return __uint_as_float(c[e]);
  } else {
    const uint32_t u = c[e / 2] >> (e % 2 * 16);
    if constexpr (T == HWKV_LOGITS_BF16) return __uint_as_float(u << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)u);
  }
}

// A row's chunks of 16 bytes, from its first logit on.  (Rows of an odd vocabulary
// start anywhere: the loads need not be aligned, and equal rows are then summed in
// equal order wherever they lie, so that equal scores are equal in all their bits.)
template <int T>
struct Row {
  const uint8_t *at;
  __device__ __forceinline__ Row(const BeamArgs &a, int64_t row)
      : at(static_cast<const uint8_t *>(a.logits) + row * a.stride * kBytes<T>) {}
  // Chunk c; minus infinity past the row's end (nothing there is read).
  __device__ __forceinline__ u32x4_t load(int c, int vocab) const {
    constexpr int N = kPerChunk<T>;
    constexpr uint32_t none = T == HWKV_LOGITS_F32 ? 0xff800000u : T == HWKV_LOGITS_BF16 ? 0xff80ff80u : 0xfc00fc00u;
    const int left = vocab - c * N;
    const uint8_t *const from = at + (int64_t)c * 16;
    u32x4_t v = {none, none, none, none};
    if (left >= N) {
      v = *reinterpret_cast<const chunk_t *>(from);
    } else {
#pragma unroll
      for (int e = 0; e < N - 1; ++e) {
        if (e >= left) continue;
        if constexpr (T == HWKV_LOGITS_F32) {
          v[e] = reinterpret_cast<const uint32_t *>(from)[e];
        } else {
          const uint32_t u = reinterpret_cast<const uint16_t *>(from)[e];
          v[e / 2] = e % 2 ? (v[e / 2] & 0xffffu) | u << 16 : (v[e / 2] & 0xffff0000u) | u;
        }
      }
    }
    return v;
  }
};

// The larger, NaN if either is.
__device__ __forceinline__ float most(float x, float y) { return __builtin_elementwise_maximum(x, y); }

template <int CTRL>
__device__ __forceinline__ float most_dpp(float x) {
  return most(x, __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), CTRL, 0xf, 0xf, true)));
}

// The largest over the wavefront, in every lane (NaN if any is).
__device__ __forceinline__ float wave_most(float x) {
  x = most_dpp<0xb1>(x);                     // lanes 1 apart,
  x = most_dpp<0x4e>(x);                     // 2,
  x = most_dpp<0x141>(x);                    // a half row's mirror,
  x = most_dpp<0x140>(x);                    // the row's
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t y = __float_as_uint(most(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const auto b = __builtin_amdgcn_permlane32_swap(y, y, false, false);
  return most(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
  return x;
}

// 2^f on [-1/2, 1/2].
__device__ __forceinline__ double exp2_small(double f) {
  double p = 0x1.63d1363930791p-20;
  p = __builtin_fma(p, f, 0x1.00dc4a53395d3p-16);
  p = __builtin_fma(p, f, 0x1.4308ac85a7718p-13);
  p = __builtin_fma(p, f, 0x1.5d8745a72831bp-10);
  p = __builtin_fma(p, f, 0x1.3b2ab7181b778p-7);
  p = __builtin_fma(p, f, 0x1.c6b08dd6fd236p-5);
  p = __builtin_fma(p, f, 0x1.ebfbdff823cedp-3);
  p = __builtin_fma(p, f, 0x1.62e42fef84cf0p-1);
  return __builtin_fma(p, f, 1.0);
}

// A sum of e^x as sum * e^base, base a logit (kNone where there is none).  Held so, and
// a score as s + ((x - base) - log sum), rows far from zero lose nothing.
constexpr double kNone = -0x1p1000;
struct Sum {
  double sum, base;
};

// Grid: n_splits workgroups a row.  Wave w of split i takes blocks 4 i + w, and so
// on in steps of 4 n_splits.  What bounds it: HBM, and the 64-bit sums beside it.
template <int T>
__global__ __launch_bounds__(kScanWaves * 64) void beam_scan(BeamArgs a) {
  constexpr int N = kPerChunk<T>;
  const int64_t row = blockIdx.x / a.n_splits;
  const int split = blockIdx.x % a.n_splits;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const Row<T> r(a, row);
  float *const block_max = a.block_max + row * a.n_blocks;
  const int step = kScanWaves * a.n_splits;
  // e^(x - base), summed; the base is the largest logit of the first block that has
  // one, and of a block whose largest passes it by 600.  A logit more than 690 below
  // it counts as that (e^-690).
  double sum = 0.0, base = kNone;
  for (int b0 = split * kScanWaves + wave; b0 < a.n_blocks; b0 += kScanDeep * step) {
    u32x4_t c[kScanDeep];
#pragma unroll
    for (int i = 0; i < kScanDeep; ++i) c[i] = r.load((b0 + i * step) * 64 + lane, a.vocab);
#pragma unroll
    for (int i = 0; i < kScanDeep; ++i) {
      const int b = b0 + i * step;
      if (b >= a.n_blocks) break;
      float x[N];
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = element<T>(c[i], e);
      float top = x[0];
#pragma unroll
      for (int e = 1; e < N; ++e) top = most(top, x[e]);
      top = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(wave_most(top))));
      if (lane == 0) block_max[b] = top;
      if (top == -kInf) continue;
      if (!(top < kInf)) {                   // an infinity or NaN: the row has no sum
        sum = __builtin_nan("");
        continue;
      }
      if ((double)top > base + 600.0) {
        sum *= exp(base - (double)top);
        base = (double)top;
      }
#pragma unroll
      for (int e = 0; e < N; ++e) {
        // with 1.5 * 2^52 added, the low word is the whole part of d log2 e
        const double d = fmax((double)x[e] - base, -690.0);
        const double y = __builtin_fma(d, kLog2e, 0x1.8p52);
        const double p = exp2_small(__builtin_fma(d, kLog2e, -(y - 0x1.8p52)));
        sum += __hiloint2double(__double2hiint(p) + (__double2loint(y) << 20), __double2loint(p));
      }
    }
  }
  sum = wave_sum(sum);
  __shared__ Sum parts[kScanWaves];
  if (lane == 0) parts[wave] = {sum, base};
  __syncthreads();
  if (threadIdx.x > 0) return;
  double top = kNone, all = 0.0;
  for (int i = 0; i < kScanWaves; ++i) top = fmax(top, parts[i].base);
  for (int i = 0; i < kScanWaves; ++i) all += parts[i].sum * exp(parts[i].base - top);
  a.part[(row * a.n_splits + split) * 2] = all;
  a.part[(row * a.n_splits + split) * 2 + 1] = top;
}

// Scores as whole numbers in their order; 0: no candidate.
__device__ __forceinline__ uint64_t order_key(double score) {
  const uint64_t u = __double_as_longlong(score + 0.0);
  return score > -__builtin_inf() ? u ^ (u >> 63 ? ~0ull : 1ull << 63) : 0;
}
__device__ __forceinline__ float key_score(uint64_t key) {
  return (float)__longlong_as_double(key >> 63 ? key ^ 1ull << 63 : ~key);
}

constexpr int kPickWaves = 4, kListed = 1024;

struct Candidate {
  uint64_t key;
  uint32_t at;
};
struct PickShared {
  double s[kMaxBeams], base[kMaxBeams];
  double log_sum[kMaxBeams];                 // NaN: a beam without candidates
  uint64_t key[kListed];
  uint32_t at[kListed];
  uint64_t lane_key[kPickWaves][64];
  uint64_t best_key[kMaxSelected];
  uint32_t best_at[kMaxSelected];
  uint64_t least;
  int listed, count[kPickWaves];
};

// Items of the workgroup for which f holds; `visit` calls its argument with every
// (key, place) of the thread.
template <typename V, typename F>
__device__ __forceinline__ int count_items(PickShared &sh, V visit, F f) {
  int n = 0;
  visit([&](uint64_t key, uint32_t at) { n += f(key, at) ? 1 : 0; });
#pragma unroll
  for (int d = 1; d < 64; d *= 2) n += __shfl_xor(n, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.count[threadIdx.x >> 6] = n;
  __syncthreads();
  n = 0;
  for (int w = 0; w < kPickWaves; ++w) n += sh.count[w];
  return n;
}

// The n first items in the order (key falling, place rising) of those that `visit`
// gives, into best_key / best_at; returns how many there are.  `least`: a key that at
// least n items reach (or 1).  The items from there on are listed and counted
// against each other.  Where the list does not hold them (long runs of equal or
// rising logits), the n-th key and then the n-th item's place are found bit by bit
// first.
template <typename V>
__device__ __forceinline__ int pick(PickShared &sh, int n, uint64_t least, V visit) {
  uint32_t last = 0xffffffffu;               // the last place of items with key `least`
  for (int round = 0;; ++round) {
    if (threadIdx.x == 0) sh.listed = 0;
    __syncthreads();
    visit([&](uint64_t key, uint32_t at) {
      if (key > least || (key == least && at <= last)) {
        const int i = atomicAdd(&sh.listed, 1);
        if (i < kListed) {
          sh.key[i] = key;
          sh.at[i] = at;
        }
      }
    });
    __syncthreads();
    if (sh.listed <= kListed || round == 1) break;
    least = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t k = least | 1ull << bit;
      if (count_items(sh, visit, [&](uint64_t key, uint32_t) { return key >= k; }) >= n) least = k;
    }
    const int more = n - count_items(sh, visit, [&](uint64_t key, uint32_t) { return key > least; });
    last = 0;
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t p = last | 1u << bit;
      if (count_items(sh, visit, [&](uint64_t key, uint32_t at) { return key == least && at < p; }) < more) last = p;
    }
  }
  const int all = min(sh.listed, kListed);
  for (int i = threadIdx.x; i < all; i += kPickWaves * 64) {
    const uint64_t key = sh.key[i];
    const uint32_t at = sh.at[i];
    int before = 0;
    for (int j = 0; j < all; ++j) before += sh.key[j] > key || (sh.key[j] == key && sh.at[j] < at) ? 1 : 0;
    if (before < n) {
      sh.best_key[before] = key;
      sh.best_at[before] = at;
    }
  }
  __syncthreads();
  return min(all, n);
}

// Grid: one workgroup a group.  What bounds it: latency, a chain of two reads and
// four short searches.
template <int T>
__global__ __launch_bounds__(kPickWaves * 64) void beam_pick(BeamArgs a) {
  constexpr int N = kPerChunk<T>;
  __shared__ PickShared sh;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t row0 = (int64_t)blockIdx.x * a.n_beams;
  const int n = a.n_out;

  for (int b = wave; b < a.n_beams; b += kPickWaves) {
    const double *const part = a.part + ((row0 + b) * a.n_splits + lane) * 2;
    const double sum = lane < a.n_splits ? part[0] : 0.0, base = lane < a.n_splits ? part[1] : kNone;
    double top = base;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) top = fmax(top, __shfl_xor(top, d));
    const double all = wave_sum(sum * exp(base - top));
    const double s = (double)a.scores[row0 + b];
    const bool some = all > 0.0 && all < __builtin_inf() && __builtin_fabs(s) < __builtin_inf();
    if (lane == 0) {
      sh.s[b] = some ? s : 0.0;
      sh.base[b] = top;
      sh.log_sum[b] = some ? log(all) : __builtin_nan("");
    }
  }
  __syncthreads();
  // (the key of a logit, 0 in a beam without candidates: its score is NaN)
  auto key_of = [&](int b, float x) { return order_key(sh.s[b] + (((double)x - sh.base[b]) - sh.log_sum[b])); };

  // the n-th largest of 64 sets' largest block maxima: n blocks reach it
  auto blocks = [&](auto f) {
    for (int b = wave; b < a.n_beams; b += kPickWaves) {
      if (sh.log_sum[b] != sh.log_sum[b]) continue;
      const float *const m = a.block_max + (row0 + b) * a.n_blocks;
      for (int j = lane; j < a.n_blocks; j += 64) f(key_of(b, m[j]), (uint32_t)(b * a.n_blocks + j));
    }
  };
  uint64_t top = 0;
  blocks([&](uint64_t key, uint32_t) { top = key > top ? key : top; });
  sh.lane_key[wave][lane] = top;
  __syncthreads();
  if (wave == 0) {
    for (int w = 1; w < kPickWaves; ++w) top = sh.lane_key[w][lane] > top ? sh.lane_key[w][lane] : top;
    sh.lane_key[0][lane] = top;
  }
  __syncthreads();
  if (wave == 0) {
    int above = 0;
    for (int j = 0; j < 64; ++j) above += sh.lane_key[0][j] > top ? 1 : 0;
    // the least of those that fewer than n lie above
    uint64_t least = above < n ? top : ~0ull;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint64_t o = __shfl_xor(least, d);
      least = o < least ? o : least;
    }
    if (lane == 0) sh.least = least > 1 ? least : 1;
  }
  __syncthreads();
  const int n_best = pick(sh, n, sh.least, blocks);
  // every element of these blocks from the last one's largest on
  uint32_t mine[kMaxSelected / kPickWaves];
#pragma unroll
  for (int i = 0; i < kMaxSelected / kPickWaves; ++i) {
    const int q = i * kPickWaves + wave;
    mine[i] = q < n_best ? sh.best_at[q] : 0;
  }
  const uint64_t least = n_best == n ? sh.best_key[n - 1] : 1;
  __syncthreads();
  auto elements = [&](auto f) {
#pragma unroll 4
    for (int i = 0; i < kMaxSelected / kPickWaves; ++i) {
      if (i * kPickWaves + wave >= n_best) break;
      const int b = mine[i] / a.n_blocks, c = (mine[i] - b * a.n_blocks) * 64 + lane;
      const Row<T> r(a, row0 + b);
      const u32x4_t v = r.load(c, a.vocab);
#pragma unroll
      for (int e = 0; e < N; ++e)
        f(key_of(b, element<T>(v, e)), (uint32_t)b * (uint32_t)a.vocab + (uint32_t)(c * N + e));
    }
  };
  const int found = n_best > 0 ? pick(sh, n, least, elements) : 0;
  if (threadIdx.x < n) {
    const int i = threadIdx.x;
    const int64_t o = (int64_t)blockIdx.x * n + i;
    const bool some = i < found;
    const uint32_t at = some ? sh.best_at[i] : 0;
    a.out_scores[o] = some ? key_score(sh.best_key[i]) : -kInf;
    a.out_parents[o] = some ? (int32_t)(row0 + at / a.vocab) : -1;
    a.out_tokens[o] = some ? (int32_t)(at % a.vocab) : -1;
  }
}

template <int T>
hipError_t launch(const BeamArgs &a, int64_t n_groups, hipStream_t s) {
  hipLaunchKernelGGL(beam_scan<T>, dim3((unsigned)(n_groups * a.n_beams * a.n_splits)), dim3(kScanWaves * 64), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(beam_pick<T>, dim3((unsigned)n_groups), dim3(kPickWaves * 64), 0, s, a);
  return hipGetLastError();
}

}  // namespace

int32_t beam_blocks(int32_t type, int32_t vocab) {
  const int n = 64 * (type == HWKV_LOGITS_F32 ? 4 : 8);
  return (vocab + n - 1) / n;
}

// Workgroups a row: enough for every CU, each with a block or more for every wave.
int32_t beam_splits(int64_t n_rows, int32_t n_blocks) {
  const int64_t most = std::min((n_blocks + kScanWaves - 1) / kScanWaves, 64);
  return (int32_t)std::max<int64_t>(1, std::min<int64_t>(most, (kScanTarget + n_rows - 1) / n_rows));
}

hipError_t launch_beam_select(int32_t type, const BeamArgs &a, int64_t n_groups, hipStream_t s) {
  switch (type) {
    case HWKV_LOGITS_BF16: return launch<HWKV_LOGITS_BF16>(a, n_groups, s);
    case HWKV_LOGITS_F16: return launch<HWKV_LOGITS_F16>(a, n_groups, s);
    case HWKV_LOGITS_F32: return launch<HWKV_LOGITS_F32>(a, n_groups, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace hwkv
