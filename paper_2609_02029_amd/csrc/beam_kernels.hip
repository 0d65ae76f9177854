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
// polynomial of degree 7, 5.5e-11 off, on [-1/2, 1/2], and the power of two goes
// into the exponent's bits: 11 64-bit operations a logit, at the rate of fp32's.
#include <algorithm>

#include "hwkv.h"
#include "hwkv_internal.h"

namespace hwkv {
namespace {

constexpr int kScanWaves = 4;
constexpr int kBlock = 512;          // logits of a block: 8 a lane
constexpr double kLog2e = 0x1.71547652b82fep+0, kLn2 = 0x1.62e42fefa39efp-1;
constexpr float kInf = __builtin_inff();

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
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
__device__ __forceinline__ float most(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float wave_max(float x) {
  return over_wave(x, [](float a, float b) { return most(a, b); });
}
__device__ __forceinline__ double wave_sum(double x) {
  return over_wave(x, [](double a, double b) { return a + b; });
}

// 2^f on [-1/2, 1/2].
__device__ __forceinline__ double exp2_small(double f) {
  double p = 0x1.00c0e4e155dc0p-16;
  p = __builtin_fma(p, f, 0x1.446c79efd4eb1p-13);
  p = __builtin_fma(p, f, 0x1.5d8775983506fp-10);
  p = __builtin_fma(p, f, 0x1.3b29d8bb0b975p-7);
  p = __builtin_fma(p, f, 0x1.c6b08da70cce3p-5);
  p = __builtin_fma(p, f, 0x1.ebfbe0aa03df0p-3);
  p = __builtin_fma(p, f, 0x1.62e42fef9cc69p-1);
  return __builtin_fma(p, f, 0x1.ffffffffa7135p-1);
}

__host__ __device__ constexpr int whole_quads(int n) { return (n + 3) & ~3; }

// A sum of e^x as sum * e^base (base kNone where there is none).
constexpr double kNone = -0x1p1000;
struct Sum {
  double sum, base;
};

// Grid: n_splits workgroups a row.  Wave w of split i takes blocks 4 i + w, and so
// on in steps of 4 n_splits, DEEP at a time.  What bounds it: HBM and the 64-bit sums
// beside it, 22 vector instructions a logit in all.  512 rows of 131,072 fp32 logits (268
// MB): 51 us, 5.2 TB/s; 528 rows of 161,840 bf16 logits (171 MB): 63 us, three quarters
// of which the vector units are busy.  (Registers for eight workgroups a CU: spills; for
// seven: as fast.)
template <int T, int DEEP>
__global__ __launch_bounds__(kScanWaves * 64) void beam_scan(BeamArgs a) {
  constexpr int N = kPerChunk<T>, C = kBlockChunks<T>;
  const int64_t row = blockIdx.x / a.n_splits;
  const int split = blockIdx.x % a.n_splits;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const Row<T> r(a, row);
  float *const block_max = a.block_max + row * whole_quads(a.n_blocks);
  const int step = kScanWaves * a.n_splits;
  // (rows of maxima are whole quads)
  if (split == 0 && (int)threadIdx.x < whole_quads(a.n_blocks) - a.n_blocks) block_max[a.n_blocks + threadIdx.x] = -kInf;
  // e^(x - base), summed; the base is set by the largest logit of the first block that
  // has one, and of a block whose largest passes it by 500, and a logit more than 690
  // below it counts as that (e^-690).  Logits up to 2^16 take base = shift ln 2 with a
  // whole shift, so that x log2 e needs no difference first; others a logit as their
  // base, from which they differ exactly.
  double sum = 0.0, base = kNone, shift = 0.0;
  float lowest = 0.0f, over = -kInf;         // base - 690, base + 500 (no base yet: any logit
                                             //   is over it, the lowest one too)
  double magic = 0.0;                        // 1.5 * 2^52 - shift: added, the low word is the
                                             //   whole part less the shift
  bool near = true;
  for (int b0 = split * kScanWaves + wave; b0 < a.n_blocks; b0 += DEEP * step) {
    u32x4_t v[DEEP][C];
    if ((b0 + (DEEP - 1) * step + 1) * kBlock <= a.vocab) {    // uniform: whole blocks
      const uint8_t *const from = r.at + (int64_t)b0 * (kBlock * kBytes<T>);
#pragma unroll
      for (int i = 0; i < DEEP; ++i)
#pragma unroll
        for (int c = 0; c < C; ++c)
          v[i][c] = reinterpret_cast<const chunk_t *>(from + (int64_t)i * step * (kBlock * kBytes<T>))[c * 64 + lane];
    } else {
#pragma unroll
      for (int i = 0; i < DEEP; ++i)
#pragma unroll
        for (int c = 0; c < C; ++c) v[i][c] = r.load(((b0 + i * step) * C + c) * 64 + lane, a.vocab);
    }
#pragma unroll
    for (int i = 0; i < DEEP; ++i) {
      const int b = b0 + i * step;
      if (b >= a.n_blocks) break;
      float x[C * N];
#pragma unroll
      for (int e = 0; e < C * N; ++e) x[e] = element<T>(v[i][e / N], e % N);
      float top = x[0], low = x[0];
#pragma unroll
      for (int e = 1; e < C * N; ++e) {
        top = most(top, x[e]);               // (NaN if any is)
        low = __builtin_elementwise_minimum(low, x[e]);
      }
      top = top == top ? top : kInf;
      top = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(wave_max(top))));
      if (lane == 0) block_max[b] = top;
      if (top == -kInf) continue;
      if (top == kInf) {                     // an infinity or NaN: the row has no sum
        sum = __builtin_nan("");
        continue;
      }
      if (top > over) {
        const double before = base;
        near = __builtin_fabsf(top) <= 0x1p16f;
        shift = rint((double)top * kLog2e);
        base = near ? shift * kLn2 : (double)top;
        lowest = (float)(base - 690.0);
        // (in fp32's steps 512 above a large base at most: half a step of 1,024 is not reached)
        over = (float)(base + 500.0);
        magic = 0x1.8p52 - shift;
        sum *= exp(before - base);
      }
      const auto add = [&](float xe) {
        const double d = (double)xe, y = __builtin_fma(d, kLog2e, magic);
        const double p = exp2_small(__builtin_fma(d, kLog2e, -(y - magic)));
        sum += __hiloint2double(__double2hiint(p) + (__double2loint(y) << 20), __double2loint(p));
      };
      if (near && !__any(low < lowest)) {
#pragma unroll
        for (int e = 0; e < C * N; ++e) add(x[e]);
      } else if (near) {
#pragma unroll
        for (int e = 0; e < C * N; ++e) add(fmaxf(x[e], lowest));
      } else {
#pragma unroll
        for (int e = 0; e < C * N; ++e) {
          const double d = fmax((double)x[e] - base, -690.0), y = __builtin_fma(d, kLog2e, 0x1.8p52);
          const double p = exp2_small(__builtin_fma(d, kLog2e, -(y - 0x1.8p52)));
          sum += __hiloint2double(__double2hiint(p) + (__double2loint(y) << 20), __double2loint(p));
        }
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

// Scores as whole numbers in their order; above 0.
__device__ __forceinline__ uint64_t order_key(double score) {
  const uint64_t u = __double_as_longlong(score + 0.0);
  return u ^ (u >> 63 ? ~0ull : 1ull << 63);
}
__device__ __forceinline__ double key_score(uint64_t key) {
  return __longlong_as_double(key >> 63 ? key ^ 1ull << 63 : ~key);
}

constexpr int kPickThreads = 512, kListed = 1024;
constexpr int kHeld = 8192, kHeldMost = 32768;   // values that a workgroup keeps in LDS
static_assert(kHeldMost >= kMaxSelected * kBlock, "the blocks of a second search");
constexpr int kRanked = 96;          // listed items that are counted against each other as they are

// A run of a search's list: consecutive places of one beam.
struct Run {
  uint32_t beam, place;
  float bound;                       // below every logit that is asked for (NaN: none is)
  uint32_t unused;
  double s, lse;                     // the beam's (lse NaN: one without candidates), or, where
                                     //   lse would lose log sum e^(x - base), s less that, and base
  __device__ __forceinline__ double score(float x) const { return s + ((double)x - lse); }
};

// Grid: one workgroup a group.  Two searches for the n first of a list, in the order
// (score falling, place rising): of the beams' block maxima, then of the logits of the
// n blocks found; each list goes into LDS, as far as it fits, in quads.  A score that n
// items reach is known before a search (the n-th largest of 64 sets' largest maxima; the
// n-th block's largest), so one comparison of logits with a bound keeps nearly all out,
// and what passes is listed, given its 64-bit key, and counted against each other (of
// many, those that a second such score leaves).
// Where a row has few blocks, the n-th is far below the best, and too many logits pass
// it: with fewer blocks than are chosen, or where the list overflows, the bound is that
// of 64 sets of logits (2 groups of 16 beams, 1,100 logits, 30 chosen: 19 us, after an
// overflow 24, without it 380; 4 groups, 2,165 logits, 18 chosen: 16.5, not 19.3, and
// 27.8 where 302 are counted against each other).  Where that does not hold them either
// (long runs of equal or rising logits), the n-th key, how many lie above it and then
// the n-th item's place are found bit by bit first.
//
// What bounds it: latency, of two reads of what other XCDs wrote or left in memory
// (about 1.5 us each) and some twenty steps through LDS: 7 us for 24 groups of 4 beams,
// 131,072 logits.
template <int T, int HELD>
__global__ __launch_bounds__(kPickThreads) void beam_pick(BeamArgs a) {
  constexpr int N = kPerChunk<T>, WAVES = kPickThreads / 64;
  __shared__ __attribute__((aligned(16))) Run run_s[2][kMaxBeams];   // of each search
  __shared__ uint32_t at_s[kListed];
  __shared__ uint64_t key_s[kListed], kept_key[kListed];
  __shared__ uint32_t kept_at[kListed];
  __shared__ float lane_top[WAVES][64];
  __shared__ double floor_s;
  __shared__ int listed, kept, hits_s[WAVES];
  __shared__ __attribute__((aligned(16))) float value_s[HELD];
  static_assert(kMaxSelected <= kMaxBeams, "a run per beam, or per block");

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t row0 = (int64_t)blockIdx.x * a.n_beams;
  const int n = a.n_out;

  // sums and block maxima
  int runs = a.n_beams;              // of the list,
  int quads = whole_quads(a.n_blocks) / 4;   // and the quads of each
  bool held = runs * quads * 4 <= HELD;
  const f32x4_t *const maxima = reinterpret_cast<const f32x4_t *>(a.block_max) + row0 * quads;
  struct Part {
    double sum, base, s;
  };
  const auto load_part = [&](int b) -> Part {
    Part p = {0.0, kNone, 0.0};
    if (b >= a.n_beams) return p;
    const double *const part = a.part + ((row0 + b) * a.n_splits + lane) * 2;
    if (lane < a.n_splits) p.sum = part[0], p.base = part[1];
    p.s = (double)a.scores[row0 + b];
    return p;
  };
  Part next = load_part(wave);
  if (held) {
#pragma unroll 4
    for (int i = threadIdx.x; i < runs * quads; i += kPickThreads)
      reinterpret_cast<f32x4_t *>(value_s)[i] = maxima[i];
  }
  for (int b = wave; b < a.n_beams; b += WAVES) {
    const Part p = next;
    next = load_part(b + WAVES);
    const double top = over_wave(p.base, [](double x, double y) { return fmax(x, y); });
    const double all = wave_sum(p.sum * exp(p.base - top)), rest = log(all);
    const bool some = all > 0.0 && all < __builtin_inf() && __builtin_fabs(p.s) < __builtin_inf();
    // A row at a type's lowest value, -3.4e38, is uniform: in top + rest nothing of rest is
    // left.  So rows from 2^19 on keep them apart, rest in the steps that lse has there, 2^-34
    // (3e-11 off): s less that is exact, and scores of two beams that are equal stay so.
    const bool near = __builtin_fabs(top) < 0x1p19;
    if (lane == 0)
      run_s[0][b] = {(uint32_t)b, (uint32_t)(b * quads * 4), 0.f, 0u,
                     !some ? 0.0 : near ? p.s : p.s - rint(rest * 0x1p34) * 0x1p-34,
                     !some ? __builtin_nan("") : near ? top + rest : top};
  }
  __syncthreads();

  for (int search = 0, sets = 1;;) {
    Run *const run_of = run_s[search];
    const auto quad = [&](int i) -> f32x4_t { return held ? reinterpret_cast<const f32x4_t *>(value_s)[i] : maxima[i]; };
    // A score that n items reach, from fp32 roundings: the n-th largest of 64 sets'
    // largest (minus infinity: fewer have one).
    if (sets) {
      float top = -kInf;
#pragma unroll 2
      for (int i = threadIdx.x; i < runs * quads; i += kPickThreads) {
        const int r = i / quads;
        const f32x4_t v = quad(i);
        // (fmaxf passes over the NaN of a beam without candidates)
        top = fmaxf(top, (float)run_of[r].score(fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w))));
      }
      lane_top[wave][lane] = top;
      __syncthreads();
      if (wave == 0) {
#pragma unroll
        for (int w = 1; w < WAVES; ++w) top = fmaxf(top, lane_top[w][lane]);
        int above = 0;
#pragma unroll
        for (int l = 0; l < 64; ++l)
          above += __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(top), l)) > top ? 1 : 0;
        const float least = over_wave(above < n ? top : kInf, [](float x, float y) { return fminf(x, y); });
        // (rounded: less a step)
        const double reached = (double)least - __builtin_fabs((double)least) * 0x1p-23;
        if (lane == 0) floor_s = search == 0 ? reached : fmax(reached, floor_s);
      }
      __syncthreads();
    }
    const double floor = floor_s;
    // score >= floor: x >= floor - s + lse, less what fp64 and fp32 round
    const auto set_bounds = [&](bool any) {
      if (threadIdx.x < runs) {
        const double s = run_of[threadIdx.x].s, lse = run_of[threadIdx.x].lse, x = floor - s + lse;
        const double off = (__builtin_fabs(floor) + __builtin_fabs(s) + __builtin_fabs(lse)) * 0x1p-48 +
                           __builtin_fabs(x) * 0x1p-22;
        // Of a beam without candidates nothing passes (a NaN: its logits may be +infinity),
        // of a floor of minus infinity all, but never a logit of minus infinity: every
        // item that is listed has a score.
        const float least = any || floor == -__builtin_inf() ? -__FLT_MAX__ : fmaxf((float)(x - off), -__FLT_MAX__);
        run_of[threadIdx.x].bound = lse != lse ? __builtin_nanf("") : least;
      }
      if (threadIdx.x == 0) listed = 0;
      __syncthreads();
    };
    // every item that its run's bound lets pass
    const auto visit = [&](auto f) {
      for (int i = threadIdx.x; i < runs * quads; i += kPickThreads) {
        const int r = search == 0 ? i / quads : i / (kBlock / 4), j = 4 * (i - r * quads);
        const Run run = run_of[r];
        const f32x4_t v = quad(i);
        if (!(fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)) >= run.bound)) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (v[e] >= run.bound) f(order_key(run.score(v[e])), run.place + j + e);
      }
    };
    const auto list = [&](uint64_t key, uint32_t at) {
      const int l = atomicAdd(&listed, 1);
      if (l < kListed) {
        key_s[l] = key;
        at_s[l] = at;
      }
    };
    set_bounds(false);
    visit(list);
    __syncthreads();
    if (listed > kListed && !sets) {
      __syncthreads();
      sets = 1;                        // once more, above the sets' bound
      continue;
    }
    if (listed > kListed) {
      // the n-th key `least`, then the place `last` of the n-th item
      __syncthreads();
      set_bounds(true);
      uint64_t least = 0;
      uint32_t last = 0;
      int more = 0;
      for (int step = 0; step < 64 + 1 + 32; ++step) {
        // items above `over`, and those at `equal` below place `upto`
        uint64_t over = least, equal = ~0ull;
        uint32_t upto = 0;
        if (step < 64) over = (least | 1ull << (63 - step)) - 1;
        if (step > 64) over = ~0ull, equal = least, upto = last | 1u << (96 - step);
        int hits = 0;
        visit([&](uint64_t key, uint32_t at) {
          hits += key > over || (key == equal && at < upto) ? 1 : 0;
        });
        hits = over_wave(hits, [](int x, int y) { return x + y; });
        __syncthreads();
        if (lane == 0) hits_s[wave] = hits;
        __syncthreads();
        hits = 0;
        for (int w = 0; w < WAVES; ++w) hits += hits_s[w];
        if (step < 64) least = hits >= n ? over + 1 : least;
        else if (step == 64) more = n - hits;          // items at `least` that are taken
        else last = hits < more ? upto : last;
      }
      visit([&](uint64_t key, uint32_t at) {
        if (key > least || (key == least && at <= last)) list(key, at);
      });
      __syncthreads();
    }
    int all = min(listed, kListed);
    const uint64_t *key = key_s;
    const uint32_t *place = at_s;
    if (all > kRanked) {
      // too many to count against each other: those that the n-th largest of 64 sets'
      // largest keeps out go first (every wave finds it for itself)
      uint64_t top = 0;
      for (int i = lane; i < all; i += 64) top = max(top, key_s[i]);
      int above = 0;
#pragma unroll 8
      for (int l = 0; l < 64; ++l) {
        const uint64_t k = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(top >> 32), l) << 32 |
                           (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)top, l);
        above += k > top ? 1 : 0;
      }
      const uint64_t least =
          over_wave(above < n ? top : ~0ull, [](uint64_t x, uint64_t y) { return x < y ? x : y; });
      if (threadIdx.x == 0) kept = 0;
      __syncthreads();
      for (int i = threadIdx.x; i < all; i += kPickThreads)
        if (key_s[i] >= least) {
          const int l = atomicAdd(&kept, 1);
          kept_key[l] = key_s[i];
          kept_at[l] = at_s[i];
        }
      __syncthreads();
      all = kept;
      key = kept_key;
      place = kept_at;
    }
    for (int i = threadIdx.x; i < all; i += kPickThreads) {
      const uint64_t mine = key[i];
      const uint32_t at = place[i];
      int before = 0;
#pragma unroll 4
      for (int j = 0; j < all; ++j) {
        const uint64_t k = key[j];
        const uint32_t p = place[j];
        before += (k > mine) | ((k == mine) & (p < at));
      }
      if (before >= n) continue;
      if (search == 0) {
        // its block's logits are a run of the next list, from the n-th's largest on
        const uint32_t row_items = 4 * quads, b = at / row_items;
        run_s[1][before] = {b, b * (uint32_t)a.vocab + (at - b * row_items) * kBlock, 0.f, 0u,
                            run_s[0][b].s, run_s[0][b].lse};
        if (before == n - 1) floor_s = key_score(mine);
      } else {
        const int64_t o = (int64_t)blockIdx.x * n + before;
        a.out_scores[o] = (float)key_score(mine);
        a.out_parents[o] = (int32_t)(row0 + at / a.vocab);
        a.out_tokens[o] = (int32_t)(at % a.vocab);
      }
    }
    const int found = min(all, n);
    if (search == 1 || found == 0) {
      if ((int)threadIdx.x >= found && (int)threadIdx.x < n) {
        const int64_t o = (int64_t)blockIdx.x * n + threadIdx.x;
        a.out_scores[o] = -kInf;
        a.out_parents[o] = a.out_tokens[o] = -1;
      }
      return;
    }
    if (threadIdx.x == 0 && found < n) floor_s = -__builtin_inf();
    __syncthreads();
    search = 1;
    sets = a.n_blocks < n ? 1 : 0;     // (a beam's blocks alone do not reach the n-th)
    runs = found;
    quads = kBlock / 4;
    held = true;                       // (n_out blocks at most: launch)
#pragma unroll 4
    for (int i = threadIdx.x; i < runs * (kBlock / N); i += kPickThreads) {
      const Run run = run_s[1][i / (kBlock / N)];
      const u32x4_t v = Row<T>(a, row0 + run.beam)
                            .load((int)(run.place - run.beam * (uint32_t)a.vocab) / N + i % (kBlock / N), a.vocab);
#pragma unroll
      for (int e = 0; e < N; ++e) value_s[i * N + e] = element<T>(v, e);
    }
    __syncthreads();
  }
}

template <int T>
hipError_t launch(const BeamArgs &a, int64_t n_groups, hipStream_t s) {
  const dim3 grid((unsigned)(n_groups * a.n_beams * a.n_splits)), threads(kScanWaves * 64);
  hipLaunchKernelGGL((beam_scan<T, 4 / kBlockChunks<T>>), grid, threads, 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // (with more in LDS one workgroup fits a CU, not two; without it 28 of 161,840 x 16 logits
  // took 75.2 us for 33 groups, not 73.5, and 64 of 200,000 x 64 58.6, not 52.9.)
  const int64_t values = std::max<int64_t>((int64_t)a.n_beams * whole_quads(a.n_blocks), a.n_out * kBlock);
  if (values <= kHeld) hipLaunchKernelGGL((beam_pick<T, kHeld>), dim3((unsigned)n_groups), dim3(kPickThreads), 0, s, a);
  else hipLaunchKernelGGL((beam_pick<T, kHeldMost>), dim3((unsigned)n_groups), dim3(kPickThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

int32_t beam_blocks(int32_t vocab) { return (vocab + kBlock - 1) / kBlock; }
int64_t beam_maxima(int32_t n_blocks) { return whole_quads(n_blocks); }

// Workgroups a row: those of all rows run at once (six fit a CU), or, where every wave
// still has eight blocks or more, in two rounds, which even the CUs out; each with a block
// or more for every wave, and no fewer blocks for some waves than need be.  (One round
// against two: 96 rows of 131,072 bf16 logits 12.3 and 14.8 us, of 232,019 20.5 and 19.9;
// 528 of 161,840 73 and 63; four rounds 19.8, 23.5 and 62.8.)
int32_t beam_splits(int64_t n_rows, int32_t n_blocks) {
  const int64_t quads = (n_blocks + kScanWaves - 1) / kScanWaves;
  const auto most = [&](int64_t target) {
    return std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(quads, 64), target / n_rows));
  };
  const int64_t splits = quads / most(2 * kScanTarget) >= 8 ? most(2 * kScanTarget) : most(kScanTarget);
  const int64_t per_wave = (quads + splits - 1) / splits;
  return (int32_t)((quads + per_wave - 1) / per_wave);
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
