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

constexpr int kScanWaves = 4;
constexpr int kBlock = 512;          // logits of a block: 8 a lane
constexpr double kLog2e = 0x1.71547652b82fep+0;
constexpr float kInf = __builtin_inff();

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef u32x4_t __attribute__((aligned(2))) chunk_t;

template <int T>
constexpr int kBytes = T == HWKV_LOGITS_F32 ? 4 : 2;
template <int T>
constexpr int kPerChunk = 16 / kBytes<T>;
template <int T>
constexpr int kBlockChunks = kBlock / 64 / kPerChunk<T>;   // a lane's

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

// op(x, y) over the wavefront, in every lane: lanes 1 and 2 apart, a half row's
// mirror, a row's, and the rows, two and two (registers only, where a shuffle goes
// through LDS).  Words: 32-bit parts of the value.
template <int CTRL>
__device__ __forceinline__ uint32_t from_dpp(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xf, 0xf, true);
}
template <typename V, typename F>
__device__ __forceinline__ V over_wave(V x, F op) {
  constexpr int W = sizeof(V) / 4;
  struct Words {
    uint32_t w[W];
  };
  auto step = [&](auto f) {
    Words a = __builtin_bit_cast(Words, x), b;
#pragma unroll
    for (int i = 0; i < W; ++i) b.w[i] = f(a.w[i]);
    x = op(x, __builtin_bit_cast(V, b));
  };
  step([](uint32_t u) { return from_dpp<0xb1>(u); });
  step([](uint32_t u) { return from_dpp<0x4e>(u); });
  step([](uint32_t u) { return from_dpp<0x141>(u); });
  step([](uint32_t u) { return from_dpp<0x140>(u); });
  auto rows = [&](auto swap) {
    Words a = __builtin_bit_cast(Words, x), b;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const auto r = swap(a.w[i]);
      a.w[i] = r[0];
      b.w[i] = r[1];
    }
    x = op(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b));
  };
  rows([](uint32_t u) { return __builtin_amdgcn_permlane16_swap(u, u, false, false); });
  rows([](uint32_t u) { return __builtin_amdgcn_permlane32_swap(u, u, false, false); });
  return x;
}
__device__ __forceinline__ float wave_max(float x) {
  return over_wave(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ double wave_sum(double x) {
  return over_wave(x, [](double a, double b) { return a + b; });
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

// A sum of e^x as sum * e^base, base a logit (kNone where there is none): x - base is
// exact, also far from zero.
constexpr double kNone = -0x1p1000;
struct Sum {
  double sum, base;
};

// Grid: n_splits workgroups a row.  Wave w of split i takes blocks 4 i + w, and so
// on in steps of 4 n_splits, DEEP at a time.  What bounds it: HBM, and the 64-bit sums
// beside it.
template <int T, int DEEP>
__global__ __launch_bounds__(kScanWaves * 64) void beam_scan(BeamArgs a) {
  constexpr int N = kPerChunk<T>, C = kBlockChunks<T>;
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
  for (int b0 = split * kScanWaves + wave; b0 < a.n_blocks; b0 += DEEP * step) {
    u32x4_t v[DEEP][C];
#pragma unroll
    for (int i = 0; i < DEEP; ++i)
#pragma unroll
      for (int c = 0; c < C; ++c) v[i][c] = r.load(((b0 + i * step) * C + c) * 64 + lane, a.vocab);
#pragma unroll
    for (int i = 0; i < DEEP; ++i) {
      const int b = b0 + i * step;
      if (b >= a.n_blocks) break;
      float x[C * N];
#pragma unroll
      for (int e = 0; e < C * N; ++e) x[e] = element<T>(v[i][e / N], e % N);
      float top = x[0];
#pragma unroll
      for (int e = 1; e < C * N; ++e) top = __builtin_elementwise_maximum(top, x[e]);   // (NaN if any is)
      top = top == top ? top : kInf;
      top = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(wave_max(top))));
      if (lane == 0) block_max[b] = top;
      if (top == -kInf) continue;
      if (top == kInf) {                     // an infinity or NaN: the row has no sum
        sum = __builtin_nan("");
        continue;
      }
      if ((double)top > base + 600.0) {
        sum *= exp(base - (double)top);
        base = (double)top;
      }
#pragma unroll
      for (int e = 0; e < C * N; ++e) {
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
__device__ __forceinline__ double key_score(uint64_t key) {
  return __longlong_as_double(key >> 63 ? key ^ 1ull << 63 : ~key);
}

constexpr int kPickThreads = 512, kListed = 1024;
constexpr int kHeldMax = 8192;       // block maxima that a workgroup keeps in LDS,
constexpr int kHeldBlocks = 16;      //   and blocks of logits

struct PickShared {
  double s[kMaxBeams], lse[kMaxBeams];       // lse NaN: a beam without candidates
  float bound[kMaxBeams];                    // below every logit of the beam that is asked for
  uint64_t key[kListed];
  uint32_t at[kListed];
  uint32_t lane_key[kPickThreads / 64][64];
  uint64_t best_key[kMaxSelected];
  uint32_t best_at[kMaxSelected];
  uint16_t block_beam[kMaxSelected];         // of the blocks whose logits are read
  uint16_t block_in[kMaxSelected];
  uint64_t least;
  int listed, hits[kPickThreads / 64];
  union {
    float max[kHeldMax];
    u32x4_t logits[kHeldBlocks * kBlock / 4];
  };
};

// The n first items in the order (key falling, place rising) of those that `visit`
// gives (its argument is called with a beam, a logit and a place), into best_key /
// best_at; returns how many there are.  `least`: a key that at least n items reach (or
// 1).  The items from there on are listed and counted against each other; a bound for
// the beam's logits keeps all others out with one comparison.  Where the list does not
// hold them (long runs of equal or rising logits), the n-th key, how many lie above it
// and then the n-th item's place are found bit by bit first.
//
// (One visit in a loop, whatever it is for: the kernel runs through its code once.
// With a visit for each purpose, unrolled, it took 13 to 23 us; so 11 to 24, of which
// half went into the keys of logits that the bound now keeps out.)
template <typename V>
__device__ __forceinline__ int pick(PickShared &sh, int n, int n_beams, uint64_t least, V visit) {
  enum { kList, kKey, kAbove, kPlace, kLast };
  int mode = kList, bit = 0, more = 0;
  uint32_t last = 0xffffffffu;               // the last place of items with key `least`
  for (;;) {
    // items above `over`, and those at `equal` up to place `upto`
    uint64_t over = least, equal = least;
    uint32_t upto = last;
    if (mode == kKey) over = least | 1ull << bit, equal = over, upto = 0xffffffffu;
    if (mode == kAbove) equal = ~0ull;
    if (mode == kPlace) over = ~0ull, upto = (last | 1u << bit) - 1;
    const bool listing = mode == kList || mode == kLast;
    if (threadIdx.x < n_beams) {
      // score >= that of `least`: x >= score - s + lse, less what fp64 and fp32 round
      float bound = -kInf;
      if (listing && least > 1) {
        const int b = threadIdx.x;
        const double t = key_score(least), at = t - sh.s[b] + sh.lse[b];
        const double off = (__builtin_fabs(t) + __builtin_fabs(sh.s[b]) + __builtin_fabs(sh.lse[b])) * 0x1p-48 +
                           __builtin_fabs(at) * 0x1p-22;
        bound = (float)(at - off);
      }
      sh.bound[threadIdx.x] = bound;
    }
    if (listing && threadIdx.x == 0) sh.listed = 0;
    __syncthreads();
    int hits = 0;
    visit([&](int b, float x, uint32_t at) {
      if (x < sh.bound[b]) return;
      const uint64_t key = order_key(sh.s[b] + ((double)x - sh.lse[b]));
      if (!(key > over || (key == equal && at <= upto))) return;
      ++hits;
      if (!listing) return;
      const int i = atomicAdd(&sh.listed, 1);
      if (i < kListed) {
        sh.key[i] = key;
        sh.at[i] = at;
      }
    });
    if (!listing) {
      hits = over_wave(hits, [](int a, int b) { return a + b; });
      if ((threadIdx.x & 63) == 0) sh.hits[threadIdx.x >> 6] = hits;
    }
    __syncthreads();
    if (listing) {
      if (sh.listed <= kListed || mode == kLast) break;
      mode = kKey;
      bit = 63;
      least = 0;
      __syncthreads();
      continue;
    }
    hits = 0;
    for (int w = 0; w < kPickThreads / 64; ++w) hits += sh.hits[w];
    if (mode == kKey) {
      if (hits >= n) least = over;
      if (--bit < 0) mode = kAbove;
    } else if (mode == kAbove) {
      more = n - hits;                       // items at `least` that are taken
      mode = kPlace;
      bit = 31;
      last = 0;
    } else {
      if (hits < more) last |= 1u << bit;
      if (--bit < 0) mode = kLast;
    }
  }
  const int all = min(sh.listed, kListed);
  for (int i = threadIdx.x; i < all; i += kPickThreads) {
    const uint64_t key = sh.key[i];
    const uint32_t at = sh.at[i];
    int before = 0;
#pragma unroll 4
    for (int j = 0; j < all; ++j) before += sh.key[j] > key || (sh.key[j] == key && sh.at[j] < at) ? 1 : 0;
    if (before < n) {
      sh.best_key[before] = key;
      sh.best_at[before] = at;
    }
  }
  __syncthreads();
  return min(all, n);
}

// Grid: one workgroup a group.  What bounds it: latency, a chain of two reads (each
// whole into LDS first, as far as it fits) and four short searches.
template <int T>
__global__ __launch_bounds__(kPickThreads) void beam_pick(BeamArgs a) {
  constexpr int N = kPerChunk<T>, CHUNKS = kBlock / N, WAVES = kPickThreads / 64;
  __shared__ __attribute__((aligned(16))) PickShared sh;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t row0 = (int64_t)blockIdx.x * a.n_beams;
  const int n = a.n_out;

  const float *const maxima = a.block_max + row0 * a.n_blocks;
  const int n_max = a.n_beams * a.n_blocks;
  const bool max_held = n_max <= kHeldMax;
#pragma unroll 4
  for (int i = threadIdx.x; i < n_max && max_held; i += kPickThreads) sh.max[i] = maxima[i];
  for (int b = wave; b < a.n_beams; b += WAVES) {
    const double *const part = a.part + ((row0 + b) * a.n_splits + lane) * 2;
    const double sum = lane < a.n_splits ? part[0] : 0.0, base = lane < a.n_splits ? part[1] : kNone;
    const double s = (double)a.scores[row0 + b];
    const double top = over_wave(base, [](double x, double y) { return fmax(x, y); });
    const double all = wave_sum(sum * exp(base - top));
    const bool some = all > 0.0 && all < __builtin_inf() && __builtin_fabs(s) < __builtin_inf();
    if (lane == 0) {
      sh.s[b] = some ? s : 0.0;
      sh.lse[b] = some ? top + log(all) : __builtin_nan("");
    }
  }
  __syncthreads();

  // The n-th largest of 64 sets' largest block maxima: n blocks reach it.  By the upper
  // half of the keys, which is enough for a key that they reach.
  auto blocks = [&](auto f) {
    int b = 0, j = threadIdx.x;
    for (int i = threadIdx.x; i < n_max; i += kPickThreads, j += kPickThreads) {
      for (; j >= a.n_blocks; j -= a.n_blocks) ++b;
      f(b, max_held ? sh.max[i] : maxima[i], (uint32_t)i);
    }
  };
  uint32_t top = 0;
  blocks([&](int b, float x, uint32_t) {
    top = max(top, (uint32_t)(order_key(sh.s[b] + ((double)x - sh.lse[b])) >> 32));
  });
  sh.lane_key[wave][lane] = top;
  __syncthreads();
  if (wave == 0) {
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top = max(top, sh.lane_key[w][lane]);
    uint32_t least = 0;                      // the largest value that n lanes reach
#pragma unroll 4
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t t = least | 1u << bit;
      if (__popcll(__ballot(top >= t)) >= n) least = t;
    }
    if (lane == 0) sh.least = least > 0 ? (uint64_t)least << 32 : 1;
  }
  __syncthreads();
  const int n_best = pick(sh, n, a.n_beams, sh.least, blocks);
  // every logit of these blocks from the last one's largest on
  const int n_chunks = n_best * CHUNKS;
  const bool logits_held = n_best <= kHeldBlocks;
  const uint64_t least = n_best == n ? sh.best_key[n - 1] : 1;
  if (threadIdx.x < n_best) {
    const int at = sh.best_at[threadIdx.x];
    sh.block_beam[threadIdx.x] = (uint16_t)(at / a.n_blocks);
    sh.block_in[threadIdx.x] = (uint16_t)(at % a.n_blocks);
  }
  __syncthreads();
  const auto load = [&](int i) {
    const int q = i / CHUNKS;
    return Row<T>(a, row0 + sh.block_beam[q]).load(sh.block_in[q] * CHUNKS + i % CHUNKS, a.vocab);
  };
#pragma unroll 4
  for (int i = threadIdx.x; i < n_chunks && logits_held; i += kPickThreads) sh.logits[i] = load(i);
  // (a thread reads what it has written)
  auto elements = [&](auto f) {
    for (int i = threadIdx.x; i < n_chunks; i += kPickThreads) {
      const u32x4_t v = logits_held ? sh.logits[i] : load(i);
      const int q = i / CHUNKS, b = sh.block_beam[q];
      const uint32_t place = (uint32_t)b * (uint32_t)a.vocab + (uint32_t)(sh.block_in[q] * kBlock + i % CHUNKS * N);
      
#pragma unroll
      for (int e = 0; e < N; ++e) f(b, element<T>(v, e), place + e);
    }
  };
  const int found = n_best > 0 ? pick(sh, n, a.n_beams, least, elements) : 0;
  if (threadIdx.x < n) {
    const int i = threadIdx.x;
    const int64_t o = (int64_t)blockIdx.x * n + i;
    const bool some = i < found;
    const uint32_t at = some ? sh.best_at[i] : 0;
    a.out_scores[o] = some ? (float)key_score(sh.best_key[i]) : -kInf;
    a.out_parents[o] = some ? (int32_t)(row0 + at / a.vocab) : -1;
    a.out_tokens[o] = some ? (int32_t)(at % a.vocab) : -1;
  }
}

template <int T>
hipError_t launch(const BeamArgs &a, int64_t n_groups, hipStream_t s) {
  const dim3 grid((unsigned)(n_groups * a.n_beams * a.n_splits)), threads(kScanWaves * 64);
  hipLaunchKernelGGL((beam_scan<T, 4 / kBlockChunks<T>>), grid, threads, 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(beam_pick<T>, dim3((unsigned)n_groups), dim3(kPickThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

int32_t beam_blocks(int32_t vocab) { return (vocab + kBlock - 1) / kBlock; }

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
