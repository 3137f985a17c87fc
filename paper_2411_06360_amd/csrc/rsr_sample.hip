// A token for every row of scores (include/rsr_decode.h).
//
// With the scores in order, the highest first, everything that is asked for is a place in one running sum: of tokens (top-k), of
// weights (top-p, the token itself), or a score (min-p).  No row is sorted for that; a look at some thousand of its scores comes first.
//   Where few tokens can be kept (a small top_k, or min_p without top_p) it says above which score all of them lie, and enough, and one pass
// gathers those in LDS, where they are sorted and the places found.
//   Else one pass counts the scores in some thousand steps between those that were looked at (the few above go into a list).  Counts
// times the weights of the steps' middles tell every sum of weights to some hundredths of a percent, and so in which steps the places are.  A
// second pass adds up what lies before these, in 64 bits, and gathers what is in them.  It computes a weight for every score, which
// takes longer than reading it, and several workgroups share it.
//   If too many tokens are there, they are most often equal (16-bit scores far from zero): then the second pass counts them in parts of the steps, and
// a place is a number among equal ones.  If that does not hold either the slow way is taken: a histogram with count and weight of each bin, 2048
// bins of 1/32 of an octave of weight, and place after place with finer ones of what is left.
//
// Where there are as many rows as CUs a row is one workgroup's, of sixteen wavefronts; few long rows are shared by several, in either pass, and
// the last one that comes goes on.  What all sixteen compute alike costs four times what one of them takes, so one alone plans and finds, and the
// others wait.  Every function is part of its kernel: a single call anywhere gives every launch a stack, which takes 1 to 13 us more (256 rows of 131072 with
// top_k 50 52 us, and 46 without it; with min_p 0.1 72 and 60); what is left are two to four registers that 16-bit scores spill, 12 to 20 bytes a lane.  There is one copy of each pass for that, and no more scores on their way than a pass needs: a kernel has to
// stay below what a short branch reaches (42 and 52 us then).
//
// What bounds it: with few rows the steps behind each other.  16 rows of 131072 with top_p 0.9, 37 us from call to call: a look 2.3, counts of 16384 scores 4.2,
// handing them on and adding them up 7.3, the plan 4.8, until the second launch is at work 3.0, weights of 8192 scores 4.5, handing on 3.4, sorting 2.4, finding 1.4.
// With many rows the second pass, some 14 operations in 64 bits for a score: 256 rows, 88 us, of which 20 are for counting and 40 for weighing (at a
// copy's rate two reads of all scores would be 53; nothing was counted that says where the second one comes from).  Other figures: one row of 131072 32 us; with top_k 50 one row takes 20, 16 rows 23, 256 rows 42; the highest
// score of each of 256 rows 29; 256 rows that all ask for something else 82 to 84.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <string>

#include "../../include/rsr_decode.h"

#include "rsr_cache_check.h"

namespace {

using rsr_internal::set_error;

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 2 * kThreads;  // two for each thread
constexpr int kPerOctave = 32;       // bins
constexpr int kList = 2 * kThreads;  // tokens that are sorted at once
constexpr int kSteps = 8 * kThreads;  // of counted scores; the first has what is above all others
constexpr int kPeaks = 2 * kThreads;  // scores above the steps
// top_k up to here is looked up in one pass: 16 rows of 131072 take 23 us with top_k 50 (counted in steps: 32), 25 with 512 (32), 53 with 900 (32); 256
// rows 42 (65), 56 (65), some 90 (65).
constexpr int kBounded = 512;
constexpr int kGroups = 256;          // workgroups of a launch: one for each CU
// Scores of a workgroup at least, where several have a row.  The second pass: one row of 131072 takes 32 us, with 8192 a microsecond more, with 16384 four.
constexpr int kLeastPiece = 4096;
constexpr int kMostRows = 1024;       // of a launch
constexpr int64_t kMostFew = UINT32_MAX / kThreads;  // of one for short rows: a launch has fewer than 2^32 threads
// The first pass hands 16 KB of counts on for each piece: four to eight pieces or one.  16 rows of 131072 take 37 us (in one piece 46; one row in eight
// pieces 32, in one 41, in 16 or 64 a microsecond more), 32768 scores in two pieces 30.7 us (in one 28.4), 128 rows of 131072 in two 72 (69.5).
constexpr int kLeastCounted = 1 << 14, kFewestCounts = 4, kMostCounts = 8;
// Tokens that are rather gathered from the first one on than counted: 256 rows of 131072 with top_k 900 take 65 us (with a prefix of 64 some 90).
constexpr int kPrefix = 1024;

// What a bin adds up in one word: for each token a one above, and below how much less than the bin's most its weight is, in units of
// 2^-34 of that.  A bin is 1/46 of its most wide at least (2^(1/32)): below 2^29 of them, and 2^17 tokens fit.
constexpr int kUnit = 34, kCountAt = 46, kChunk = 1 << 17;

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;

struct Args {
  const void* logits;
  const float *temperature, *top_p, *min_p, *uniform;
  const int32_t* top_k;
  int32_t* token;
  float* probability;
  int32_t* kept;
  int64_t stride;
  int32_t columns, log2_columns;  // log2_columns: bits of a column's number
};

constexpr int kMostRuns = 4;

// The step of a place, with the sums up to it and up to and with it.
struct Mark {
  int bin;
  uint32_t before, count;
  float mass_before, mass;
};

// Scores to steps, the higher ones first: 0 for what is above the first of the others, the last but one for what is below them.  (A
// difference of halves, which is not beyond the range of float, times the steps of half a unit.)
struct Steps {
  float from, half, per;
  __device__ __forceinline__ float down(float x) const { return fmaf(-0.5f, x, half) * per; }
  __device__ __forceinline__ float score(int step) const { return 2.f * (half - (float)step / per); }  // at about the end of a step
  static __device__ __forceinline__ int step(float down) { return down < 0.f ? 0 : 1 + (int)__builtin_amdgcn_fmed3f(down, 0.f, (float)(kSteps - 3)); }
  // The bounds of `down` from step lo to step hi, both included.
  static __device__ __forceinline__ float first_of(int lo) { return lo ? (float)(lo - 1) : -INFINITY; }
  static __device__ __forceinline__ float last_of(int hi) { return hi >= kSteps - 2 ? INFINITY : hi ? __uint_as_float(__float_as_uint((float)hi) - 1) : -FLT_MIN; }
};

// Tokens of neighbouring steps that lie in the list, one run behind the other.
struct Run {
  int b0, b1;                     // steps
  uint32_t start, count, before;  // where it begins in the list, how many there are, and before them in the row
  int shift;                      // how far apart its buckets are, for sorting; kEven: as many for each step
  float from, each;               // for kEven: where it begins, and buckets of a step
  u64 code;                       // about that of the first
  double mass_before;             // the weight of those before

  // As many buckets as tokens, or half as many, from one code to another.  Codes are dense where scores are near zero: if these lie on both
  // sides of it, the buckets are even in the scores.
  static constexpr int kEven = -1;
  __device__ __forceinline__ void span(u64 from, u64 to) {
    code = from;
    shift = max(0, __clz((int)count) + 33 - __clzll((long long)(to > from ? to - from : 1)));
  }
  __device__ __forceinline__ void span_even(float down_first, float down_last) {
    shift = kEven, from = down_first, each = (float)count / (down_last - down_first);
  }
  __device__ __forceinline__ uint32_t bucket(u64 x, float down) const {
    if (shift == kEven) return start + (uint32_t)__builtin_amdgcn_fmed3f((down - from) * each, 0.f, (float)(count - 1));
    return start + (x < code ? 0 : (uint32_t)min((x - code) >> shift, (u64)(count - 1)));
  }
};

// What the second pass has to do.
struct Plan {
  Run run[kMostRuns];
  int n;            // runs
  int near;         // the run up to this step has the last token that min_p keeps; -1: min_p keeps all
  uint32_t tokens;  // of all runs
  uint32_t all;     // of the row
  int weighed;      // it adds up weights
  int behind;       // the place of top_p is taken to be behind what min_p keeps
  int ends;         // the last run has the row's last token
  int shift;        // of the unit in which weights are added up
  int slow;         // kMany: too many tokens for the list; kSlow: too many above the steps, or no steps
};
constexpr int kMany = 1, kSlow = 2;
// (Not 1, so that a workspace that was not cleared, whose rows are never planned, leads nowhere.)
constexpr int32_t kPlanned = 0x706c616e;

// What a row is asked for.
struct Ask {
  double factor;   // octaves of weight in a unit of scores
  double top_p;    // 2: all
  double far;      // the distance of the last that min_p keeps, or infinity
  double u;
  uint32_t top_k;  // 0: all
};

// What is known of a row before the second pass.
struct Head {
  int32_t planned;  // kPlanned: the second pass has something to do
  float top;
  Steps steps;
  Ask ask;
  Plan plan;
};

// For sums over the wavefronts of a workgroup, and what one of them tells the others.
struct Waves {
  double mass[kWaves];
  uint32_t count[kWaves];
  u64 best[kWaves];
  float low[kWaves], high[kWaves];
  Head head;
  uint32_t arrived, sure;
};

// Of a workgroup that counts scores.
struct Counts {
  uint32_t steps[kSteps + 64];
  float peaks[kPeaks];  // scores above the steps
  float looked[kThreads];
  float bound;
  Mark mark[2 * kMostRuns];
  uint32_t before[2];
  uint32_t listed, all_count;
  uint32_t first_steps;  // tokens of the first 128 steps
  float all_mass;
};

// Of one that gathers tokens.
struct Lists {
  u64 list[kList];                                // tokens, sorted
  double upto[kList];                             // weight up to and with each
  uint32_t part_count[kBins + 1];                 // of a finer histogram, or where buckets begin
  union { u64 part_sum[kBins]; double part_mass[kBins]; u64 bucketed[kList]; };
  uint32_t count[kBins];                          // of the slow way: up to and with the bin
  union {
    u64 sum[kBins];  // packed as above; then
    double mass[kBins];  // the weight up to and with the bin
    struct { uint32_t least[kBins], most[kBins]; };  // keys, where equal scores are counted
  };
  u64 weight[kMostRuns + 1];                      // before each run, and of all
  uint32_t listed, first;
};

// ---- scores -----------------------------------------------------------------------------------------------
// A score as a whole number, ascending for descending scores, both zeros alike, without the bits that its type does not have.
template <typename T> struct Key {
  static constexpr int kDrop = sizeof(T) == 4 ? 0 : __is_same(T, __bf16) ? 16 : 13;
  static __device__ uint32_t of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u >> 31 ? u : ~u & 0x7fffffffu) >> kDrop;
  }
  static __device__ float score(uint32_t key) {
    const uint32_t k = key << kDrop;
    return __uint_as_float(k >> 31 ? k : ~(k | ((1u << kDrop) - 1)) & 0x7fffffffu);
  }
};

// f(scores, column of the first) for 16 bytes of `count` scores of a row from column `first` on at a time, by all threads of the
// workgroup, each in ascending order, wherever the row begins; SCORES of a thread are on their way while as many are looked at.  What sticks out at
// the ends is read by itself and comes with minus infinity behind it.
template <int SCORES = 16, typename T, typename F> __device__ __forceinline__ void for_pieces(const T* row, int first, int count, F f) {
  typedef const __attribute__((address_space(1))) T* Scores;
  typedef const __attribute__((address_space(1))) u4* Pieces;
  constexpr int kWide = 16 / sizeof(T), kAtOnce = SCORES / kWide;
  const Scores from = (Scores)(row + first);
  const int head = min(count, (int)((16 - (reinterpret_cast<uintptr_t>(row + first) & 15)) & 15) / (int)sizeof(T));
  const int pieces = (count - head) / kWide, tail = head + pieces * kWide, tid = threadIdx.x;
  auto alone = [&](int at) {
    float x[kWide] = {(float)from[at]};
#pragma unroll
    for (int j = 1; j < kWide; ++j) x[j] = -INFINITY;
    f(x, first + at);
  };
  if (tid < head) alone(tid);
  const Pieces body = (Pieces)(from + head);
  auto load = [&](u4 (&v)[kAtOnce], int p0) {
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) v[i] = body[min(p0 + i * kThreads, pieces - 1)];
  };
  auto use = [&](const u4 (&v)[kAtOnce], int p0) {
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int p = p0 + i * kThreads;
      if (p >= pieces) break;
      float x[kWide];
      if constexpr (kWide == 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = __uint_as_float(v[i][j]);
      } else {
        typedef T t8 __attribute__((ext_vector_type(8)));
        const t8 t = __builtin_bit_cast(t8, v[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (float)t[j];
      }
      f(x, first + head + p * kWide);
    }
  };
  constexpr int kStep = kThreads * kAtOnce;
  if (pieces > 0) {
    u4 v[2][kAtOnce];
    load(v[0], tid);
    for (int p0 = tid; p0 < pieces; p0 += 2 * kStep) {
      load(v[1], p0 + kStep);
      use(v[0], p0);
      if (p0 + kStep >= pieces) break;
      load(v[0], p0 + 2 * kStep);
      use(v[1], p0 + kStep);
    }
  }
  if (tid < count - tail) alone(tail + tid);
}
// f(score, column) for each score.
template <typename T, typename F> __device__ __forceinline__ void for_each(const T* row, int first, int count, F f) {
  for_pieces<8>(row, first, count, [&](const float (&x)[16 / sizeof(T)], int column) {
#pragma unroll
    for (int j = 0; j < 16 / (int)sizeof(T); ++j) f(x[j], column + j);
  });
}

// The same in any order, score by score, with little code: for what is seldom or little to do.
template <int AT_ONCE = 2, typename T, typename F> __device__ __forceinline__ void for_each_seldom(const T* row, int first, int count, F f) {
  typedef const __attribute__((address_space(1))) T* Scores;
  const Scores from = (Scores)(row + first);
  for (int i0 = threadIdx.x; i0 < count; i0 += AT_ONCE * kThreads) {
    T x[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) x[j] = from[min(i0 + j * kThreads, count - 1)];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j)
      if (i0 + j * kThreads < count) f((float)x[j], first + i0 + j * kThreads);
  }
}

// ---- weights ----------------------------------------------------------------------------------------------
// A score's distance below the highest, in octaves of its weight: the weight is 2^-distance, 1 exactly for the highest.
struct Scale {
  float top;
  double factor;
  __device__ __forceinline__ double distance(float x) const { return x == top ? 0.0 : ((double)top - (double)x) * factor; }
  // `one` + 2^f - 1, f from -1/2 to 1/2: 2^f is the polynomial that has its values at nine Chebyshev nodes, off by 2^-39 of it.  (A thousand
  // octaves down nothing is left of a weight.)
  static __device__ __forceinline__ double power(double f, double one) {
    return one + f * (0.6931471805459335 + f * (0.2402265069581299 + f * (0.05550410941205934 + f * (0.009618129159402607 + f * (0.0013333450567999429 +
           f * (0.00015403455852420792 + f * (1.5310079402541085e-05 + f * 1.3255224885567153e-06)))))));
  }
  __device__ __forceinline__ double weight(float x) const {
    const double d = fmin(distance(x), 1000.0), n = rint(d);
    return power(n - d, 1.0) * __builtin_bit_cast(double, (u64)((uint32_t)(1023 - (int)n) << 20) << 32);
  }
};
__device__ __forceinline__ int bin_of(double distance) { return (int)fmin(distance * kPerOctave, (double)(kBins - 1)); }

// Sums of weights in whole numbers, so that no order of additions matters, in units of 2^-62 of the highest's shifted up by as much as
// keeps the sum of all below 2^64.  What is cut off is less than a unit for each: at most 2^-40 of the sum for 2^22 scores, 2^-45 for 2^17.  (In units
// that are the same for all rows, 2^-40, a tail of 2^17 equal scores was off by a thousand of them.)  2 + 2^f has the bits of 2^f / 2 behind its point.
struct Weights {
  double top, factor;
  int shift;
  __device__ __forceinline__ u64 of(float x) const {
    const double d = fmin((top - (double)x) * factor, 62.25 - shift), n = rint(d);  // (2^-62.25 is nothing)
    return __builtin_bit_cast(u64, Scale::power(n - d, 3.0)) << 12 >> ((int)n + shift + 1);
  }
  static __device__ __forceinline__ double sum(u64 units, int shift) { return (double)units * __builtin_bit_cast(double, (u64)(1023 - 62 + shift) << 52); }
  // The shift for weights that together are less than `most`.
  static __device__ __forceinline__ int shift_of(float most) { return max(0, __builtin_amdgcn_frexp_expf(most) - 2); }
};

// 2^34 times 1 - 2^-(f / 32) for f from 0 to 1, as a sum of powers of f ln 2 / 32 (the sixth adds less than 2^-42).  Of the last bin,
// which has all that is 64 octaves down and more, nothing is weighed.
__device__ __forceinline__ uint32_t below_most(double distance, int bin) {
  constexpr double l = 0.021660849392498290, u = (double)(1ull << kUnit);
  const double f = distance * kPerOctave - bin;
  const double q = f * (u * l + f * (-u * l * l / 2 + f * (u * l * l * l / 6 + f * (-u * l * l * l * l / 24 + f * (u * l * l * l * l * l / 120)))));
  return bin == kBins - 1 ? 0u : (uint32_t)(q + 0.5);
}
__device__ __forceinline__ u64 packed(double distance, int bin) { return (u64)1 << kCountAt | below_most(distance, bin); }
__device__ __forceinline__ uint32_t count_in(u64 sum) { return (uint32_t)(sum >> kCountAt); }
__device__ __forceinline__ double mass_in(u64 sum, int bin) {
  if (bin == kBins - 1) return 0.0;
  const u64 less = sum & (((u64)1 << kCountAt) - 1);
  return (double)(((u64)count_in(sum) << kUnit) - less) * exp2(-(double)bin / kPerOctave - kUnit);
}

// ---- sums over a workgroup ---------------------------------------------------------------------------------
template <int CTRL, int ROWS, typename T> __device__ __forceinline__ T moved(T x) {  // 0 where there is no other lane
  if constexpr (sizeof(T) == 8) {
    const u64 v = __builtin_bit_cast(u64, x);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false), hi = __builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROWS, 0xf, false);
    return __builtin_bit_cast(T, (u64)hi << 32 | lo);
  } else {
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, ROWS, 0xf, false));
  }
}
// Sums of the lanes up to and with the own one: of 16 lanes, and of all.
template <typename T> __device__ __forceinline__ T sum_of_16(T x) {
  x += moved<0x111, 0xf>(x);
  x += moved<0x112, 0xf>(x);
  x += moved<0x114, 0xf>(x);
  return x + moved<0x118, 0xf>(x);
}
template <typename T> __device__ __forceinline__ T sum_of_lanes(T x) {
  x = sum_of_16(x);
  x += moved<0x142, 0xa>(x);
  return x + moved<0x143, 0xc>(x);
}
template <typename T> __device__ __forceinline__ T of_lane(T x, int lane) {
  if constexpr (sizeof(T) == 8) {
    const u64 v = __builtin_bit_cast(u64, x);
    return __builtin_bit_cast(T, (u64)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane));
  } else {
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
  }
}

// The largest of the lanes of 16, and of all; of what the wavefronts wrote down.
template <int CTRL, int ROWS> __device__ __forceinline__ float largest_step(float x) {
  return fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), CTRL, ROWS, 0xf, false)));
}
__device__ __forceinline__ float largest_of_16(float x) { return largest_step<0x118, 0xf>(largest_step<0x114, 0xf>(largest_step<0x112, 0xf>(largest_step<0x111, 0xf>(x)))); }
__device__ __forceinline__ float largest(float x) { return of_lane(largest_step<0x143, 0xc>(largest_step<0x142, 0xa>(largest_of_16(x))), 63); }
__device__ __forceinline__ float largest_of_waves(const float* x) { return of_lane(largest_of_16(x[threadIdx.x & 15]), 15); }

// Running sums of two entries per thread, in their order, and what is before them.
template <typename M> struct Sums {
  uint32_t c[2], c_before;
  M m[2], m_before;

  __device__ __forceinline__ void scan(Waves& waves, uint32_t c0, M m0) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t cs = sum_of_lanes(c[0] + c[1]);
    const M ms = sum_of_lanes(m[0] + m[1]);
    __syncthreads();
    if (lane == 63) waves.count[wave] = cs, waves.mass[wave] = ms;
    __syncthreads();
    const uint32_t cw = sum_of_16(waves.count[lane & 15]);
    const M mw = sum_of_16((M)waves.mass[lane & 15]);
    c_before = c0, m_before = m0;
    if (wave) c_before += of_lane(cw, wave - 1), m_before += of_lane(mw, wave - 1);
    c_before += moved<0x138, 0xf>(cs), m_before += moved<0x138, 0xf>(ms);  // (of the lane before)
    c[0] += c_before, m[0] += m_before, c[1] += c[0], m[1] += m[0];
  }
};

// ---- places -----------------------------------------------------------------------------------------------
// The place where a running sum reaches what is asked for.
template <typename M> struct Place {
  bool of_count, strict;  // a sum of tokens (at least `count`), or of weights: at least `mass`, or more than that
  uint32_t count;
  M mass;
  __device__ __forceinline__ bool reached(uint32_t c, M m) const { return of_count ? c >= count : strict ? m > mass : m >= mass; }
  static __device__ __forceinline__ Place tokens(uint32_t n) { return {true, false, n, 0}; }
  static __device__ __forceinline__ Place weight(M m, bool more) { return {false, more, 0, m}; }
};
typedef Place<double> At;

// The first of n running sums that reaches the place; the last one if none does.
__device__ __forceinline__ int first_at(const At& p, const uint32_t* count, const double* mass, int n) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (p.reached(count ? count[mid] : 0, mass[mid])) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

struct Found {
  u64 code;
  double share;  // of the weight of what is kept
  uint32_t kept;
  bool sure;
};

template <typename T> struct Row {
  const T* row;
  int columns, log2_columns;
  Scale scale;

  __device__ __forceinline__ u64 code(float x, int column) const { return (u64)Key<T>::of(x) << log2_columns | (uint32_t)column; }
  __device__ float score(u64 code) const { return Key<T>::score((uint32_t)(code >> log2_columns)); }
  __device__ int column(u64 code) const { return (int)(code & (((u64)1 << log2_columns) - 1)); }

  // Tokens that are wanted, into the list in any order; how many there are (they may be more than fit).
  template <typename W> __device__ __forceinline__ uint32_t gather(Lists& lds, W wanted) const {
    __syncthreads();
    if (threadIdx.x == 0) lds.listed = 0;
    __syncthreads();
    for_each_seldom(row, 0, columns, [&](float x, int column) {
      if (x == -INFINITY || !wanted(x, column)) return;
      const uint32_t at = atomicAdd(&lds.listed, 1u);
      if (at < kList) lds.list[at] = code(x, column);
    });
    __syncthreads();
    return lds.listed;
  }

  // Sorts the list and adds up its weights.  Codes are dealt into buckets, as many for each run as it has tokens, and each finds its
  // place among those of its bucket.  (What lies outside the bounds of its run lands in a bucket at the end, still in order.)
  __device__ __forceinline__ void sort(Waves& waves, Lists& lds, const Plan& plan, const Steps& steps) const {
    const int tid = threadIdx.x;
    const uint32_t n = plan.tokens;
    u64 x[2];
    uint32_t bucket[2], slot[2];
    lds.part_count[2 * tid] = lds.part_count[2 * tid + 1] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t i = tid + j * kThreads;
      if (i >= n) continue;
      x[j] = lds.list[i];
      const float down = steps.down(score(x[j]));
      bucket[j] = plan.run[0].bucket(x[j], down);
#pragma unroll
      for (int k = 1; k < kMostRuns; ++k)
        if (k < plan.n && x[j] >= plan.run[k].code) bucket[j] = plan.run[k].bucket(x[j], down);
      slot[j] = atomicAdd(&lds.part_count[bucket[j]], 1u);
    }
    __syncthreads();
    Sums<double> s;
#pragma unroll
    for (int j = 0; j < 2; ++j) s.c[j] = lds.part_count[2 * tid + j], s.m[j] = 0.0;
    s.scan(waves, 0, 0.0);
    lds.part_count[2 * tid] = s.c_before, lds.part_count[2 * tid + 1] = s.c[0];
    if (tid == kThreads - 1) lds.part_count[kBins] = s.c[1];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (tid + j * kThreads < n) lds.bucketed[lds.part_count[bucket[j]] + slot[j]] = x[j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (tid + j * kThreads >= n) continue;
      const uint32_t end = lds.part_count[bucket[j] + 1];
      uint32_t at = lds.part_count[bucket[j]];
      for (uint32_t i = at; i < end; ++i) at += lds.bucketed[i] < x[j];
      lds.list[at] = x[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j) s.c[j] = 0, s.m[j] = 2 * tid + j < n ? scale.weight(score(lds.list[2 * tid + j])) : 0.0;
    s.scan(waves, 0, 0.0);
    lds.upto[2 * tid] = s.m[0], lds.upto[2 * tid + 1] = s.m[1];
    __syncthreads();
  }

  // ---- places in the list
  static __device__ double mass_at(const Lists& lds, const Run& r, uint32_t i) { return r.mass_before + (lds.upto[i] - (r.start ? lds.upto[r.start - 1] : 0.0)); }
  // The first token of the list at the place, and its run.  (Loops over runs are unrolled: they stay in registers.)
  static __device__ __forceinline__ uint32_t seek(const Lists& lds, const Plan& plan, At p, Run& r) {
    r = plan.run[0];
#pragma unroll
    for (int i = 1; i < kMostRuns; ++i)
      if (i < plan.n && !p.reached(r.before + r.count, mass_at(lds, r, r.start + r.count - 1))) r = plan.run[i];
    if (p.of_count) return r.start + min(max(p.count, r.before + 1) - r.before, r.count) - 1;
    p.mass -= r.mass_before - (r.start ? lds.upto[r.start - 1] : 0.0);
    return r.start + first_at(p, nullptr, lds.upto + r.start, r.count);
  }

  // Whether the place that seek found is where the sum reaches it: not before its run, and not behind.
  static __device__ bool sure(const Lists& lds, const At& p, const Run& r, uint32_t all) {
    return (!r.before || !p.reached(r.before, r.mass_before)) && (r.before + r.count == all || p.reached(r.before + r.count, mass_at(lds, r, r.start + r.count - 1)));
  }

  // The answer, where the list has all places.  `kept`, `mass`: all tokens and their weight (if a place or the token needs it).  Nothing
  // is `sure` if a place is in none of the runs.
  __device__ __forceinline__ Found solve(const Lists& lds, const Ask& ask, const Plan& plan, uint32_t kept, double mass) const {
    Run r;
    bool is_sure = true;
    const uint32_t all = kept;
    if (ask.top_k && ask.top_k < kept) {
      const At p = At::tokens(ask.top_k);
      const uint32_t at = seek(lds, plan, p, r);
      is_sure &= sure(lds, p, r, all);
      kept = ask.top_k, mass = mass_at(lds, r, at);
    }
    if (ask.top_p < 1.0 && !plan.behind) {
      const At p = At::weight(ask.top_p * mass, false);
      const uint32_t at = seek(lds, plan, p, r), n = r.before + at - r.start + 1;
      is_sure &= sure(lds, p, r, all);
      if (n < kept) kept = n, mass = mass_at(lds, r, at);
      // (min_p was left out because its place is behind: the last one is near enough then)
      if (plan.near < 0 && ask.far < INFINITY) is_sure &= scale.distance(score(lds.list[at])) <= ask.far;
    }
    if (plan.near >= 0) {
      r = plan.run[0];
#pragma unroll
      for (int i = 1; i < kMostRuns; ++i)
        if (i < plan.n && plan.run[i].b0 <= plan.near) r = plan.run[i];
      uint32_t lo = 0, hi = r.count;  // how many are near enough
      while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (scale.distance(score(lds.list[r.start + mid])) <= ask.far) lo = mid + 1;
        else hi = mid;
      }
      is_sure &= lo < r.count || r.before + r.count >= kept;
      // (top_p's place is behind them if the sum without the last of them is below it; without any of the run, with the last one)
      if (plan.behind) is_sure &= !At::weight(ask.top_p * mass, false).reached(0, lo > 1 ? mass_at(lds, r, r.start + lo - 2) : r.mass_before);
      if (r.before + lo < kept) kept = r.before + lo, mass = lo ? mass_at(lds, r, r.start + lo - 1) : r.mass_before;
    }
    const At p = At::weight(ask.u * mass, true);
    const uint32_t at = seek(lds, plan, p, r);
    return {lds.list[at], scale.weight(score(lds.list[at])) / mass, kept, is_sure && sure(lds, p, r, all)};
  }

  // ---- place after place (a list for each), where there are too many tokens for one list
  // The run of tokens in which the place is.
  __device__ __forceinline__ Run run_at(Waves& waves, Lists& lds, const At& p) const {
    const int tid = threadIdx.x;
    int b = first_at(p, lds.count, lds.mass, kBins);
    while (b && lds.count[b] == lds.count[b - 1]) --b;  // (what rounding puts behind the last token is the last token's)
    uint32_t before = b ? lds.count[b - 1] : 0, count = lds.count[b] - before;
    double mass_before = b ? lds.mass[b - 1] : 0.0;
    u64 lo = 0, hi = ((u64)1 << (32 + log2_columns)) - 1;
    while (count > kList) {
      const int shift = max(0, 64 - __clzll((long long)(hi - lo)) - 11);
      Sums<double> s{{0, 0}, 0, {0.0, 0.0}, 0.0};
      for (int first = 0; first < columns; first += kChunk) {
        __syncthreads();
        lds.part_sum[2 * tid] = lds.part_sum[2 * tid + 1] = 0;
        __syncthreads();
        for_each_seldom(row, first, min(kChunk, columns - first), [&](float x, int column) {
          if (x == -INFINITY) return;
          const double d = scale.distance(x);
          const u64 c = code(x, column);
          if (bin_of(d) == b && c >= lo && c <= hi) atomicAdd(&lds.part_sum[(c - lo) >> shift], packed(d, b));
        });
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 2; ++j) s.c[j] += count_in(lds.part_sum[2 * tid + j]), s.m[j] += mass_in(lds.part_sum[2 * tid + j], b);
      }
      s.scan(waves, before, mass_before);
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 2; ++j) lds.part_count[2 * tid + j] = s.c[j], lds.part_mass[2 * tid + j] = s.m[j];
      __syncthreads();
      int part = first_at(p, lds.part_count, lds.part_mass, kBins);
      while (part && lds.part_count[part] == lds.part_count[part - 1]) --part;
      while (lds.part_count[part] == before) ++part;  // (or before the first one)
      if (part) before = lds.part_count[part - 1], mass_before = lds.part_mass[part - 1];
      count = lds.part_count[part] - before;
      lo += (u64)part << shift;
      hi = min(hi, lo + ((u64)1 << shift) - 1);
    }
    gather(lds, [&](float x, int column) {
      const u64 c = code(x, column);
      return bin_of(scale.distance(x)) == b && c >= lo && c <= hi;
    });
    Plan plan;
    plan.n = 1, plan.near = -1, plan.tokens = count;
    Run& r = plan.run[0];
    r = {b, b, 0, count, before, 0, 0.f, 0.f, 0, mass_before};
    if (!lo && scale.top < INFINITY)  // (the bin's ends, or what is left of it)
      lo = code((float)((double)scale.top - b / (kPerOctave * scale.factor)), 0), hi = code((float)((double)scale.top - (b + 1) / (kPerOctave * scale.factor)), 0);
    r.span(lo, hi);
    sort(waves, lds, plan, waves.head.steps);
    return r;
  }

  __device__ __forceinline__ Found solve_slowly(Waves& waves, Lists& lds, const Ask& ask) const {
    uint32_t kept = lds.count[kBins - 1];
    double mass = lds.mass[kBins - 1];
    Plan plan{};
    Run r;
    uint32_t at = 0;
    // top_k's place, top_p's, and the token's: a loop, for one copy of the code
#pragma unroll 1
    for (int place = 0; place < 3; ++place) {
      if (place == 0 && !(ask.top_k && ask.top_k < kept)) continue;
      if (place == 1 && !(ask.top_p < 1.0)) continue;
      if (place == 2 && ask.far < INFINITY) {
        const int b = bin_of(ask.far);
        const uint32_t before = b ? lds.count[b - 1] : 0;
        if (before < kept) {
          // (a count and a sum over all that is near enough in its bin)
          double sum = 0.0;
          uint32_t n = 0;
          for (int first = 0; first < columns; first += kChunk) {
            __syncthreads();
            if (threadIdx.x == 0) lds.part_sum[0] = 0;
            __syncthreads();
            for_each_seldom(row, first, min(kChunk, columns - first), [&](float x, int) {
              if (x == -INFINITY) return;
              const double d = scale.distance(x);
              if (d <= ask.far && bin_of(d) == b) atomicAdd(&lds.part_sum[0], packed(d, b));
            });
            __syncthreads();
            n += count_in(lds.part_sum[0]), sum += mass_in(lds.part_sum[0], b);
          }
          if (before + n < kept) kept = before + n, mass = (b ? lds.mass[b - 1] : 0.0) + sum;
        }
      }
      const At p = place == 0 ? At::tokens(ask.top_k) : place == 1 ? At::weight(ask.top_p * mass, false) : At::weight(ask.u * mass, true);
      const Run& have = plan.run[0];
      const bool here = plan.n && !p.reached(have.before, have.mass_before) && p.reached(have.before + have.count, mass_at(lds, have, have.count - 1));
      if (!here) plan.run[0] = run_at(waves, lds, p), plan.n = 1;
      at = seek(lds, plan, p, r);
      if (place == 0) kept = ask.top_k, mass = mass_at(lds, r, at);
      const uint32_t n = r.before + at + 1;
      if (place == 1 && n < kept) kept = n, mass = mass_at(lds, r, at);
    }
    return {lds.list[at], scale.weight(score(lds.list[at])) / mass, kept, true};
  }
};

// ---- a look at a row --------------------------------------------------------------------------------------
__device__ __forceinline__ float parameter(const float* p, int64_t r, float without) { return p ? p[r] : without; }

__device__ __forceinline__ Ask ask_of(const Args& a, int64_t r, float temperature) {
  const float top_p = parameter(a.top_p, r, 1.f), min_p = parameter(a.min_p, r, 0.f), uniform = a.uniform[r];
  const int top_k = a.top_k ? a.top_k[r] : 0;
  // (0 times infinity is NaN)
  return {fmax(1.4426950408889634 / (double)temperature, 1e-300), top_p < 1.f ? fmax((double)top_p, 0.0) : 2.0,
          min_p > 0.f ? min_p >= 1.f ? 0.0 : -log2((double)min_p) : INFINITY, uniform > 0.f ? fmin((double)uniform, 1.0 - 0x1p-24) : 0.0,
          top_k > 0 && top_k < a.columns ? (uint32_t)top_k : 0u};
}

// Steps from one of the highest of some thousand scores of a row down to the lowest, or to the last that has any weight, and a bound
// above which lie the tokens that can be kept, if they are few (else NaN): where top_k is small, the score of which so many are above
// among the highest of four to eight that enough of the row's are, and some hundred more; with min_p alone, the least that it may come to.
template <typename T> __device__ __forceinline__ void look(const Args& a, int64_t r, const T* row, float temperature, Waves& waves, Counts& lds) {
  constexpr int kWide = 16 / sizeof(T);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / (int)sizeof(T), pieces = (a.columns - head) / kWide, looked = min(pieces, kThreads);
  float high = -INFINITY, low = INFINITY;
  if (tid < looked) {
    const u4 v = *reinterpret_cast<const u4*>(row + head + (int64_t)((int64_t)tid * pieces / looked) * kWide);
    T x[kWide];
    __builtin_memcpy(x, &v, 16);
#pragma unroll
    for (int j = 0; j < kWide; ++j) {
      const float f = (float)x[j];
      if (f > -INFINITY && f < INFINITY) high = fmaxf(high, f), low = fminf(low, f);
    }
  }
  Ask ask;
  if (wave == 0) ask = ask_of(a, r, temperature);
  lds.looked[tid] = high;
  high = largest(high), low = largest(-low);
  if (lane == 0) waves.high[wave] = high, waves.low[wave] = low;
  __syncthreads();
  if (wave == 0) {
    low = -largest_of_waves(waves.low);
    const float mine = waves.high[lane & (kWaves - 1)];
    high = of_lane(largest_of_16(mine), 15);
    // above the first step are some hundred scores: those above the `rank`-th of the wavefronts' highest
    const int with = __popcll(__ballot(mine > -INFINITY) & 0xffff), rank = max(1, min(with / 2, (kWaves / 2 << 17) / a.columns));
    int higher = 0;
    for (int w = 0; w < kWaves; ++w) {
      const float other = of_lane(mine, w);
      higher += other > mine || (other == mine && w < (lane & (kWaves - 1)));
    }
    const float from = of_lane(mine, __builtin_ctzll(__ballot(higher == rank - 1)));
    Steps steps{-FLT_MAX, -FLT_MAX / 2, 1.f};
    if (from > -INFINITY) {
      // (but no finer than 2^-33 of the scores, so that those above are some steps away and not infinitely many)
      const double range = fmax(fmin((double)from - (double)low, 48.0 / ask.factor), fmax(fabs((double)from) * 0x1p-20, 1e-20));
      steps = {from, 0.5f * from, (float)fmin(2.0 * (kSteps - 3) / range, (double)FLT_MAX)};
    }
    float bound = NAN;
    if (ask.top_k && ask.top_k <= kBounded) {
      const float share = (float)ask.top_k * (float)(looked * kWide) / (float)a.columns;
      const int wanted = (int)(share + 5.f * sqrtf(share) + 8.f);
      float down[kThreads / 64];
#pragma unroll
      for (int j = 0; j < kThreads / 64; ++j) down[j] = steps.down(lds.looked[j * 64 + lane]);
      int least = 0, most = kSteps;
      while (most - least > 4) {
        const int mid = (least + most) / 2;
        int n = 0;
#pragma unroll
        for (int j = 0; j < kThreads / 64; ++j) n += __popcll(__ballot(down[j] <= (float)mid));
        if (n >= wanted) most = mid;
        else least = mid;
      }
      bound = most >= kSteps - 4 ? INFINITY : (float)most;
    } else if (ask.far < INFINITY && ask.top_p >= 1.0) {
      const float x = (float)fmax((double)high - ask.far / ask.factor, -(double)FLT_MAX);
      bound = high > -INFINITY ? fmaxf(steps.down(x), 0.f) + 1.f : NAN;
      // Not if it leaves sixteen thousand tokens or more, as the share of the looked at pieces with such a score says.
      const float share = (float)(8 * kList) / (float)a.columns;
      int n = 0;
      for (int j = 0; j < kThreads / 64; ++j) n += __popcll(__ballot(steps.down(lds.looked[j * 64 + lane]) <= bound));
      if (share < 1.f && (float)n > (float)looked * (1.f - __builtin_amdgcn_exp2f(kWide * __builtin_amdgcn_logf(1.f - share)))) bound = NAN;
    }
    if (lane == 0) waves.head.ask = ask, waves.head.steps = steps, lds.bound = bound;
  }
}

// The first pass: the highest score, whether one is NaN, and the tokens above the bound, or else all scores counted in steps and those above
// the steps in a list.
template <typename T> __device__ __forceinline__ float gather_above(Waves& waves, Lists& lds, const Row<T>& row, const Steps& steps, int first, int count, float bound, bool& nan) {
  constexpr int kWide = 16 / sizeof(T);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) lds.listed = 0;
  __syncthreads();
  float high = -INFINITY;
  for_pieces<sizeof(T) == 2 ? 8 : 16>(row.row, first, count, [&](const float (&x)[kWide], int column) {
    bool some = false;
#pragma unroll
    for (int j = 0; j < kWide; ++j) {
      high = __builtin_elementwise_maximum(high, x[j]);  // (NaN stays)
      some |= steps.down(x[j]) <= bound;
    }
    if (some)
#pragma unroll
      for (int j = 0; j < kWide; ++j)
        if (steps.down(x[j]) <= bound && x[j] > -INFINITY) {
          const uint32_t at = atomicAdd(&lds.listed, 1u);
          if (at < kList) lds.list[at] = row.code(x[j], column + j);
        }
  });
  nan = __syncthreads_or(high != high);
  high = largest(high);
  if (lane == 0) waves.high[wave] = high;
  __syncthreads();
  return largest_of_waves(waves.high);
}

template <typename T> __device__ __forceinline__ float count_steps(Waves& waves, Counts& lds, const Row<T>& row, const Steps& steps, int first, int count, bool& nan) {
  constexpr int kWide = 16 / sizeof(T);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, aside = kSteps + lane;
  u4* const zero = reinterpret_cast<u4*>(lds.steps);
  for (int i = tid; i < kSteps / 4; i += kThreads) zero[i] = u4{0, 0, 0, 0};
  if (tid == 0) lds.listed = 0;
  __syncthreads();
  float high = -INFINITY;
  for_pieces<8>(row.row, first, count, [&](const float (&x)[kWide], int) {
    float least = 0.f;
#pragma unroll
    for (int j = 0; j < kWide; ++j) {
      const float down = steps.down(x[j]);
      high = __builtin_elementwise_maximum(high, x[j]);  // (NaN stays)
      least = __builtin_elementwise_minimum(least, down);
      // what is not counted is added somewhere else, so that there is no branch
      const int step = 1 + (int)__builtin_amdgcn_fmed3f(down, 0.f, (float)(kSteps - 3));
      atomicAdd(&lds.steps[down >= 0.f && x[j] > -INFINITY ? step : aside], 1u);
    }
    if (!(least >= 0.f))  // (seldom; NaN comes here too, and is none of them)
#pragma unroll
      for (int j = 0; j < kWide; ++j)
        if (steps.down(x[j]) < 0.f) {
          const uint32_t at = atomicAdd(&lds.listed, 1u);
          if (at < kPeaks) lds.peaks[at] = x[j];
        }
  });
  nan = __syncthreads_or(high != high);
  high = largest(high);
  if (lane == 0) waves.high[wave] = high;
  __syncthreads();
  return largest_of_waves(waves.high);
}

// In which steps the places may be, and so which tokens are gathered.  The scores above the steps are weighed one by one, a step as its
// count times the weight in its middle.  Where a step's scores lie in it is not known: it is off by its weight times its width (in
// ln 2 octaves) over the root of 12, as if they all lay at one place of which any is as likely, and the sums of all are off by the root of the
// squares of that; four and a half times as much is allowed for.  That is no bound: scores near the same end of all steps are off by more.  Whether it was
// enough is seen in the end, for a place that is looked up as for one that is left out because another comes before it.
__device__ __forceinline__ void plan_row(Waves& waves, Counts& lds, const Scale& scale) {
  constexpr int kEach = kSteps / kThreads;
  constexpr float kRounded = 2e-6f;  // of a sum: what some twenty roundings come to, and more
  static_assert(kEach == 8);
  typedef Place<float> About;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const Ask& ask = waves.head.ask;
  const Steps steps = waves.head.steps;
  const uint32_t peaks = lds.listed;
  const double wide = 2.0 * scale.factor / steps.per, above = ((double)scale.top - (double)steps.from) * scale.factor - 0.5 * wide;
  // (steps wider than half an octave of scores next to zero tell nothing; of others, all of a step are equal then)
  if (peaks > kPeaks || scale.top == INFINITY || (wide > 0.5 && fabsf(steps.from) < 1e-14f)) {
    if (tid == 0) waves.head.plan.slow = kSlow;
    __syncthreads();
    return;
  }
  const Weights weights{scale.top, scale.factor, Weights::shift_of(kPeaks)};
  u64 high = 0;  // (they lie in any order, so their sum is one of whole numbers)
#pragma unroll
  for (int j = 0; j < 2; ++j)
    if ((uint32_t)(tid + j * kThreads) < peaks) high += weights.of(lds.peaks[tid + j * kThreads]);
  high = sum_of_lanes(high);
  if (lane == 63) waves.best[wave] = high;
  if (tid == 0) lds.steps[0] = peaks;
  if (tid < 2 * kMostRuns) lds.mark[tid].bin = kSteps;
  __syncthreads();
  const float peak = (float)Weights::sum(of_lane(sum_of_16(waves.best[lane & 15]), 15), weights.shift);

  // the sums of each thread's steps
  const float octaves = (float)wide;
  auto weight_of = [&](uint32_t n, int step) { return step ? (float)n * __builtin_amdgcn_exp2f(-fmaxf((float)(above + step * wide), 0.f)) : peak; };
  const float first = (float)(above + tid * kEach * wide);
  float squares = 0.f;
  Sums<float> s{{0, 0}, 0, {0.f, 0.f}, 0.f};
#pragma unroll
  for (int j = 0; j < kEach / 4; ++j) {
    const u4 n = reinterpret_cast<const u4*>(lds.steps)[tid * (kEach / 4) + j];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float w = (float)n[i] * __builtin_amdgcn_exp2f(-fmaxf(fmaf((float)(4 * j + i), octaves, first), 0.f));
      if (i == 0 && j == 0) w = tid ? w : 0.f;
      s.c[0] += n[i], s.m[0] += w, squares = fmaf(w, w, squares);
    }
  }
  if (tid == 0) s.m[0] += peak;
  squares = sum_of_lanes(squares);
  if (lane == 63) waves.high[wave] = squares;
  s.scan(waves, 0, 0.f);
  if (tid == kThreads - 1) lds.all_count = s.c[0], lds.all_mass = s.m[0];
  if (tid == 128 / kEach) lds.first_steps = s.c_before;
  // The step of a place: the wavefront in which a thread's sums reach it adds up the steps of that thread, a lane each.
  auto mark = [&](int place, const About& p) {
    const u64 here = __ballot(s.c[0] > s.c_before && p.reached(s.c[0], s.m[0]) && (!s.c_before || !p.reached(s.c_before, s.m_before)));
    if (!here) return;
    const int thread = __builtin_ctzll(here), step = ((wave << 6) + thread) * kEach + (lane & (kEach - 1));
    const uint32_t n = lane < kEach ? lds.steps[step] : 0, c = of_lane(s.c_before, thread) + sum_of_16(n);
    const float w = lane < kEach ? weight_of(n, step) : 0.f, m = of_lane(s.m_before, thread) + sum_of_16(w);
    const u64 some = __ballot(n != 0), at = __ballot(n && p.reached(c, m));
    if (lane == (at ? __builtin_ctzll(at) : 63 - __builtin_clzll(some))) lds.mark[place] = {step, c - n, c, m - w, m};
  };
  const bool far = ask.far < INFINITY;
  if (far) {
    // tokens before the step before that of the last score that is kept, and before the one behind it
    const int step = Steps::step(steps.down((float)((double)scale.top - ask.far / scale.factor)));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = i ? min(step + 1, kSteps - 1) : max(step - 1, 0);
      if (tid != at / kEach) continue;
      uint32_t c = s.c_before;
      for (int j = 0; j < at % kEach; ++j) c += lds.steps[tid * kEach + j];
      lds.before[i] = c;
    }
  }
  __syncthreads();
  const uint32_t all = lds.all_count;
  const float total = lds.all_mass;
  const float off = 0.9004245f * octaves * sqrtf(of_lane(sum_of_16(waves.high[lane & 15]), 15)) + kRounded * total +  // (4.5 ln 2 / sqrt 12)
                    weight_of(lds.steps[kSteps - 2], kSteps - 2);  // (what is below all that were looked at may have no weight at all)
  const bool k = ask.top_k && ask.top_k < all, p = ask.top_p < 1.0;
  mark(0, About::tokens(all));
  if (k) mark(1, About::tokens(ask.top_k));
  if (far) mark(4, About::tokens(lds.before[0] + 1)), mark(5, About::tokens(lds.before[1] + 1));
  __syncthreads();
  // What is kept ends at `end` at the latest; its weight is between `least` and `most`.
  auto marked = [&](int place, const Mark& end) { return lds.mark[place].bin < end.bin ? lds.mark[place] : end; };
  Mark end = lds.mark[0];
  int lo[kMostRuns], hi[kMostRuns];             // of top_k, top_p, min_p, and the token
  uint32_t before[kMostRuns], upto[kMostRuns];  // tokens before, and up to and with
#pragma unroll
  for (int i = 0; i < kMostRuns; ++i) lo[i] = hi[i] = kSteps, before[i] = upto[i] = 0;  // none
  float least = total - off, most = total + off;
  if (k) {
    end = lds.mark[1];
    lo[0] = hi[0] = end.bin, before[0] = end.before, upto[0] = end.count;
    least = end.mass_before - off, most = end.mass + off;
  }
  if (p) {
    mark(2, About::weight((float)ask.top_p * least - off, false)), mark(3, About::weight((float)ask.top_p * most + off, false));
    __syncthreads();
    const Mark a = marked(2, end);
    end = marked(3, end);
    lo[1] = a.bin, before[1] = a.before, hi[1] = end.bin, upto[1] = end.count;
    least = fminf(least, a.mass_before - off), most = fminf(most, end.mass + off);
  }
  const Mark weight_end = end;
  const bool m = far && lds.mark[4].bin <= end.bin;
  if (m) {
    const Mark a = lds.mark[4];
    end = marked(5, end);
    lo[2] = a.bin, before[2] = a.before, hi[2] = end.bin, upto[2] = end.count;
    least = fminf(least, a.mass_before - off), most = fminf(most, end.mass + off);
  }
  const int near = m ? end.bin : -1;
  const bool behind = m && p && end.bin < lo[1];
  if (behind) lo[1] = hi[1] = kSteps, before[1] = upto[1] = 0;
  const Mark last = k ? lds.mark[1] : p && !behind ? weight_end : end;  // (the weight of the first top_k is asked for, and top_p's place looked up)
  const bool prefix = last.count <= kPrefix;
  if (!prefix) mark(6, About::weight((float)ask.u * least - off, true)), mark(7, About::weight((float)ask.u * most + off, true));
  __syncthreads();
  if (wave == 0) {
    Plan plan;
    plan.near = near, plan.all = all, plan.behind = behind;
    // (A step's weights are less than 2^(1/4) of what is in its middle.  Of wider ones, those behind the first 128 have no weight.)
    plan.shift = Weights::shift_of(octaves <= 0.5f ? fminf(1.25f * total, (float)all) : (float)lds.first_steps);
    if (prefix) {
      lo[0] = 0, hi[0] = last.bin, before[0] = 0, upto[0] = last.count;
#pragma unroll
      for (int i = 1; i < kMostRuns; ++i) lo[i] = hi[i] = kSteps;
      plan.weighed = last.count < all && !k && (p || !m);
    } else {
      const Mark a = marked(6, end), b = marked(7, end);
      lo[3] = a.bin, before[3] = a.before, hi[3] = b.bin, upto[3] = b.count;
      plan.weighed = true;
      // in order
      auto order = [&](int i, int j) {
        if (lo[j] < lo[i]) {
          const int l = lo[i], h = hi[i];
          const uint32_t x = before[i], y = upto[i];
          lo[i] = lo[j], hi[i] = hi[j], before[i] = before[j], upto[i] = upto[j];
          lo[j] = l, hi[j] = h, before[j] = x, upto[j] = y;
        }
      };
      order(0, 1), order(2, 3), order(0, 2), order(1, 3), order(1, 2);
      // What meets is one: those that do are taken into the one before, and the others move up.
#pragma unroll
      for (int i = 1; i < kMostRuns; ++i)
        if (lo[i] < kSteps) hi[i] = max(hi[i], hi[i - 1]), upto[i] = max(upto[i], upto[i - 1]);
#pragma unroll
      for (int i = kMostRuns - 1; i; --i)
        if (lo[i] < kSteps && lo[i] <= hi[i - 1] + 1) {
          hi[i - 1] = hi[i], upto[i - 1] = upto[i];
#pragma unroll
          for (int j = i; j < kMostRuns; ++j) {
            const bool more = j + 1 < kMostRuns;
            lo[j] = more ? lo[(j + 1) % kMostRuns] : kSteps, hi[j] = more ? hi[(j + 1) % kMostRuns] : kSteps;
            before[j] = more ? before[(j + 1) % kMostRuns] : 0, upto[j] = more ? upto[(j + 1) % kMostRuns] : 0;
          }
        }
    }
    plan.n = 0, plan.tokens = 0, plan.ends = 0;
#pragma unroll
    for (int i = 0; i < kMostRuns; ++i) {
      const bool there = lo[i] < kSteps;
      plan.run[i] = {lo[i], hi[i], plan.tokens, there ? upto[i] - before[i] : 0, before[i], 0, 0.f, 0.f, 0, 0.0};
      plan.tokens += plan.run[i].count, plan.n += there, plan.ends |= there && upto[i] == all;
    }
    plan.slow = plan.tokens > kList ? kMany : 0;
    if (lane == 0) waves.head.plan = plan;
  }
  __syncthreads();
}

// ---- the second pass --------------------------------------------------------------------------------------
// Gathers the tokens of the plan's runs among `count` scores from `first` on.  RUNS: adds up the weights before each of so many runs too, and
// of all.  0: there is one run, from the first token on.  EQUAL: does not list tokens, but counts them, each run's in kEach parts, with the least and
// the most of their keys.
constexpr int kEach = kBins / kMostRuns;
template <int RUNS, bool EQUAL, typename T> __device__ __forceinline__ void gather_runs(const Plan& plan, Lists& lds, const Row<T>& row, const Steps& steps, int first, int count) {
  constexpr int kWide = 16 / sizeof(T), kRuns = RUNS ? RUNS : 1;
  if (threadIdx.x == 0) lds.listed = 0;
  if (threadIdx.x <= kMostRuns) lds.weight[threadIdx.x] = 0;
  if constexpr (EQUAL)
    for (int i = threadIdx.x; i < kBins; i += kThreads) lds.count[i] = lds.most[i] = 0, lds.least[i] = ~0u;
  __syncthreads();
  const Weights weights{row.scale.top, row.scale.factor, plan.shift};
  float lo[kRuns], hi[kRuns], from[kRuns], per[kRuns];
  u64 before[kRuns], all = 0;
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    const bool there = i < plan.n;
    lo[i] = there ? Steps::first_of(plan.run[i].b0) : INFINITY, hi[i] = there ? Steps::last_of(plan.run[i].b1) : -INFINITY, before[i] = 0;
    if constexpr (EQUAL) from[i] = there && plan.run[i].b0 ? lo[i] : steps.down(row.scale.top), per[i] = kEach / ((float)plan.run[i].b1 - from[i]);
  }
  auto wanted = [&](float down) {
    bool in = false;
#pragma unroll
    for (int i = 0; i < kRuns; ++i) in |= down >= lo[i] && down <= hi[i];
    return in;
  };
  // (Few on their way are enough where each is weighed; more would take more registers, and code than a kernel may have.)
  for_pieces<RUNS == 4 ? kWide : RUNS || sizeof(T) == 2 ? 8 : 16>(row.row, first, count, [&](const float (&x)[kWide], int column) {
    bool some = false;
#pragma unroll
    for (int j = 0; j < kWide; ++j) {
      const float down = steps.down(x[j]);
      some |= wanted(down);
      if constexpr (RUNS) {
        const u64 w = weights.of(x[j]);
        all += w;
#pragma unroll
        for (int i = 0; i < kRuns; ++i) before[i] += down < lo[i] ? w : 0;
      }
    }
    if (some)
#pragma unroll
      for (int j = 0; j < kWide; ++j)
        if (wanted(steps.down(x[j])) && x[j] > -INFINITY) {
          if constexpr (EQUAL) {
            const float down = steps.down(x[j]);
            int part = 0;
#pragma unroll
            for (int i = 0; i < kRuns; ++i)
              if (down >= lo[i] && down <= hi[i]) part = i * kEach + (int)__builtin_amdgcn_fmed3f((down - from[i]) * per[i], 0.f, (float)(kEach - 1));
            const uint32_t key = Key<T>::of(x[j]);
            atomicAdd(&lds.count[part], 1u), atomicMin(&lds.least[part], key), atomicMax(&lds.most[part], key);
            continue;
          }
          const uint32_t at = atomicAdd(&lds.listed, 1u);
          if (at < kList) lds.list[at] = row.code(x[j], column + j);
        }
  });
  if constexpr (RUNS) {
    auto give = [&](u64 sum, u64* to) {
      sum = sum_of_lanes(sum);
      if ((threadIdx.x & 63) == 63) atomicAdd(to, sum);
    };
#pragma unroll
    for (int i = 0; i < kRuns; ++i) give(before[i], &lds.weight[i]);
    give(all, &lds.weight[kMostRuns]);
  }
  __syncthreads();
}

template <typename T> __device__ __forceinline__ void gather_plan(const Plan& plan, Lists& lds, const Row<T>& row, const Steps& steps, int first, int count) {
  if (plan.slow) gather_runs<4, true>(plan, lds, row, steps, first, count);
  else if (!plan.weighed) gather_runs<0, false>(plan, lds, row, steps, first, count);
  else if (plan.n == 1 && sizeof(T) == 4) gather_runs<sizeof(T) == 4 ? 1 : 2, false>(plan, lds, row, steps, first, count);  // (16-bit scores: no room for its code)
  else if (plan.n <= 2) gather_runs<2, false>(plan, lds, row, steps, first, count);
  else gather_runs<4, false>(plan, lds, row, steps, first, count);
}

// ---- answers ----------------------------------------------------------------------------------------------
__device__ __forceinline__ void answer(const Args& a, int64_t r, int token, float probability, uint32_t kept) {
  if (threadIdx.x) return;
  a.token[r] = token;
  if (a.probability) a.probability[r] = probability;
  if (a.kept) a.kept[r] = (int32_t)kept;
}

// True if the row is answered with what is known of its highest score.
template <typename T> __device__ __forceinline__ bool is_answered(const Args& a, int64_t r, const Row<T>& row, u64 best, bool nan, bool greedy) {
  if (nan) answer(a, r, -1, NAN, 0);
  else if (best == ~(u64)0) answer(a, r, -1, 0.f, 0);
  else if (greedy) answer(a, r, row.column(best), 1.f, 1);
  else return false;
  return true;
}

// The first of the highest scores, as a code (all ones: there is none), and the lowest.
template <typename T> __device__ __forceinline__ u64 best_of(Waves& lds, const Row<T>& row, int first, int count, float& low, bool& nan) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float high = -INFINITY;
  int at = 0;
  nan = false, low = INFINITY;
  for_each(row.row, first, count, [&](float x, int column) {
    nan |= x != x;
    low = x > -INFINITY ? fminf(low, x) : low;
    const bool more = x > high;
    high = more ? x : high, at = more ? column : at;
  });
  u64 best = high > -INFINITY ? row.code(high, at) : ~(u64)0;
  low = largest(-low);
#pragma unroll
  for (int d = 32; d; d >>= 1) best = min(best, (u64)__shfl_xor((long long)best, d));
  if (lane == 0) lds.best[wave] = best, lds.low[wave] = low;
  nan = __syncthreads_or(nan);
  for (int w = 0; w < kWaves; ++w) best = min(best, lds.best[w]);
  low = -largest_of_waves(lds.low);
  return best;
}

// The tokens of the plan are in the list, and the weights before its runs are known: the answer, if it is sure.
// SPANNED: its run's codes are too.
template <bool SPANNED, typename T> __device__ __forceinline__ bool find(const Args& a, int64_t r, const Row<T>& row, Waves& waves, Lists& lds) {
  Plan& plan = waves.head.plan;
  if (lds.listed != plan.tokens) return false;
  const Steps steps = waves.head.steps;
  const int tid = threadIdx.x;
  if (!SPANNED && tid < kMostRuns) {
    Run run = plan.run[tid];
    run.mass_before = plan.weighed ? Weights::sum(lds.weight[tid], plan.shift) : 0.0;
    if (tid < plan.n) {
      const float first = run.b0 ? steps.score(run.b0 - 1) : row.scale.top, last = steps.score(min(run.b1, kSteps - 2));
      run.span(row.code(first, 0), row.code(last, row.columns - 1));
      if (first > 0.f && last < 0.f) run.span_even(steps.down(first), steps.down(last));
    }
    plan.run[tid] = run;
  }
  __syncthreads();
  row.sort(waves, lds, plan, steps);
  if (tid < 64) {
    // (where the last run ends the row, its sum of all is that of the places in it)
    double mass = lds.upto[plan.tokens - 1];
    if (plan.weighed) mass = plan.ends ? row.mass_at(lds, plan.run[plan.n - 1], plan.tokens - 1) : Weights::sum(lds.weight[kMostRuns], plan.shift);
    const Found f = row.solve(lds, waves.head.ask, plan, plan.all, mass);
    if (f.sure) answer(a, r, row.column(f.code), (float)f.share, f.kept);
    if (tid == 0) waves.sure = f.sure;
  }
  __syncthreads();
  return waves.sure;
}

// The runs have more tokens than the list, but they are counted, and in every part all are equal: the answer, if that holds and it is sure.
// Among equal tokens a place is a number, and the token itself is looked for.
template <typename T> __device__ __forceinline__ bool find_equal(const Args& a, int64_t r, const Row<T>& row, Waves& waves, Lists& lds) {
  const Plan& plan = waves.head.plan;
  const Ask& ask = waves.head.ask;
  const int tid = threadIdx.x;
  int near = 0;
  for (int i = 1; i < kMostRuns; ++i)
    if (i < plan.n && plan.run[i].b0 <= plan.near) near = i;
  if (tid == 0) lds.first = 0;
  Sums<double> s;
  bool mixed = false, is_near[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int part = 2 * tid + j;
    const uint32_t n = lds.count[part];
    const float x = Key<T>::score(n ? lds.least[part] : 0);
    mixed |= n && lds.least[part] != lds.most[part];
    is_near[j] = n && plan.near >= 0 && part / kEach == near && row.scale.distance(x) <= ask.far;
    s.c[j] = n, s.m[j] = n ? n * row.scale.weight(x) : 0.0;
  }
  if (__syncthreads_or(mixed)) return false;
  s.scan(waves, 0, 0.0);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    lds.part_count[2 * tid + j] = s.c[j], lds.upto[2 * tid + j] = s.m[j];
    if (is_near[j]) atomicMax(&lds.first, (uint32_t)(2 * tid + j + 1));
  }
  __syncthreads();
  if (lds.part_count[kBins - 1] != plan.tokens) return false;

  if (tid < 64) {
    uint32_t kept = plan.all, before, count, nth;
    double mass_before, upto;
    int part;
    bool is_sure = true;
    // a run's sums up to and with a part
    auto counted = [&](int i, int at) { return plan.run[i].before + lds.part_count[at] - (i ? lds.part_count[i * kEach - 1] : 0); };
    auto weighed = [&](int i, int at) { return Weights::sum(lds.weight[i], plan.shift) + (lds.upto[at] - (i ? lds.upto[i * kEach - 1] : 0.0)); };
    const int end = plan.n - 1;  // (as in find)
    double mass = plan.ends ? weighed(end, end * kEach + kEach - 1) : Weights::sum(lds.weight[kMostRuns], plan.shift);
    auto seek = [&](const At& p) {
      int i = 0;
      while (i + 1 < plan.n && !p.reached(counted(i, i * kEach + kEach - 1), weighed(i, i * kEach + kEach - 1))) ++i;
      int lo = i * kEach, hi = lo + kEach - 1;
      const bool behind = p.reached(counted(i, hi), weighed(i, hi));
      is_sure &= (!plan.run[i].before || !p.reached(plan.run[i].before, Weights::sum(lds.weight[i], plan.shift))) && (behind || counted(i, hi) == plan.all);
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (p.reached(counted(i, mid), weighed(i, mid))) hi = mid;
        else lo = mid + 1;
      }
      auto size = [&](int at) { return lds.part_count[at] - (at ? lds.part_count[at - 1] : 0); };
      while (!size(lo) && lo < i * kEach + kEach - 1) ++lo;  // (what is reached before the first one is the first one's)
      while (!size(lo)) --lo;                                // (and what rounding puts behind the last is the last one's)
      part = lo;
      const uint32_t n = size(part);
      const double weight = row.scale.weight(Key<T>::score(lds.least[part]));
      before = counted(i, part) - n, mass_before = weighed(i, part) - n * weight;
      const double of = fmin(fmax((p.mass - mass_before) / weight, 0.0), (double)n);
      nth = min(max(p.of_count ? p.count - before : p.strict ? (uint32_t)floor(of) + 1 : (uint32_t)ceil(of), 1u), n);
      count = before + nth, upto = mass_before + nth * weight;
    };
    // top_k's place, top_p's, and the token's: a loop, for one copy of the code
#pragma unroll 1
    for (int place = 0; place < 3; ++place) {
      if (place == 0 && !(ask.top_k && ask.top_k < kept)) continue;
      if (place == 1 && !(ask.top_p < 1.0 && !plan.behind)) continue;
      if (place == 2 && plan.near >= 0) {
        const int last = (int)lds.first - 1;
        const uint32_t n = last < 0 ? plan.run[near].before : counted(near, last), end = plan.run[near].before + plan.run[near].count;
        is_sure &= n < end || end >= kept;
        const double upto_last = last < 0 ? Weights::sum(lds.weight[near], plan.shift) : weighed(near, last);
        // (as in Row::solve)
        if (plan.behind) is_sure &= !At::weight(ask.top_p * mass, false).reached(0, last < 0 ? upto_last : upto_last - row.scale.weight(Key<T>::score(lds.least[last])));
        if (n < kept) kept = n, mass = upto_last;
      }
      seek(place == 0 ? At::tokens(ask.top_k) : place == 1 ? At::weight(ask.top_p * mass, false) : At::weight(ask.u * mass, true));
      if (place == 0) kept = ask.top_k, mass = upto;
      if (place == 1 && count < kept) kept = count, mass = upto;
      if (place == 1 && plan.near < 0 && ask.far < INFINITY) is_sure &= row.scale.distance(Key<T>::score(lds.least[part])) <= ask.far;
    }
    if (tid == 0) waves.sure = is_sure, waves.count[0] = lds.least[part], waves.count[1] = nth, waves.count[2] = kept, waves.mass[0] = mass;
  }
  __syncthreads();
  if (!waves.sure) return false;
  const float x = Key<T>::score(waves.count[0]);
  const uint32_t number = waves.count[1], kept = waves.count[2];
  const double mass = waves.mass[0];

  // the token: a count of the equal ones in 2048 parts of the row, then one part
  const int shift = max(0, row.log2_columns - 11);
  __syncthreads();
  lds.part_count[2 * tid] = lds.part_count[2 * tid + 1] = 0;
  __syncthreads();
  for_each_seldom<16>(row.row, 0, row.columns, [&](float y, int column) {
    if (y == x) atomicAdd(&lds.part_count[column >> shift], 1u);
  });
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 2; ++j) s.c[j] = lds.part_count[2 * tid + j], s.m[j] = 0.0;
  s.scan(waves, 0, 0.0);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t c = j ? s.c[0] : s.c_before;
    if (c < number && s.c[j] >= number) lds.first = 2 * tid + j, lds.listed = number - c;
  }
  __syncthreads();
  const int column = ((int)lds.first << shift) + 2 * tid, end = min(((int)lds.first + 1) << shift, row.columns);
  const uint32_t wanted = lds.listed;
#pragma unroll
  for (int j = 0; j < 2; ++j) s.c[j] = column + j < end && (float)row.row[min(column + j, row.columns - 1)] == x, s.m[j] = 0.0;
  s.scan(waves, 0, 0.0);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t c = j ? s.c[0] : s.c_before;
    if (c < wanted && s.c[j] >= wanted) lds.first = column + j;
  }
  __syncthreads();
  answer(a, r, (int)lds.first, (float)(row.scale.weight(x) / mass), kept);
  return true;
}

// A plan of one run that has all tokens that matter, `n` of them.
__device__ __forceinline__ void plan_all(Waves& waves, uint32_t n, int last) {
  if (threadIdx.x) return;
  Plan& plan = waves.head.plan;
  plan.run[0] = {0, last, 0, n, 0, 0, 0.f, 0.f, 0, 0.0};
  plan.n = 1, plan.near = waves.head.ask.far < INFINITY ? 0 : -1, plan.tokens = plan.all = n, plan.weighed = plan.behind = plan.slow = 0;
}

template <typename T> __device__ __forceinline__ void find_slowly(const Args& a, int64_t r, const Row<T>& row, Waves& waves, Lists& lds) {
  const int tid = threadIdx.x;
  Sums<double> s{{0, 0}, 0, {0.0, 0.0}, 0.0};
  for (int at = 0; at < a.columns; at += kChunk) {
    __syncthreads();
    lds.sum[2 * tid] = lds.sum[2 * tid + 1] = 0;
    __syncthreads();
    for_each_seldom(row.row, at, min(kChunk, a.columns - at), [&](float x, int) {
      if (x == -INFINITY) return;
      const double d = row.scale.distance(x);
      const int bin = bin_of(d);
      atomicAdd(&lds.sum[bin], packed(d, bin));
    });
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j) s.c[j] += count_in(lds.sum[2 * tid + j]), s.m[j] += mass_in(lds.sum[2 * tid + j], 2 * tid + j);
  }
  s.scan(waves, 0, 0.0);
#pragma unroll
  for (int j = 0; j < 2; ++j) lds.count[2 * tid + j] = s.c[j], lds.mass[2 * tid + j] = s.m[j];
  __syncthreads();
  const Found f = row.solve_slowly(waves, lds, waves.head.ask);
  answer(a, r, row.column(f.code), (float)f.share, f.kept);
}

// ---- kernels ----------------------------------------------------------------------------------------------
// The workspace: of a launch's first rows, which several workgroups share, the only words that have to be zero before a call, and are
// behind it; what the second pass has to know of each row, and what each piece of a row has given the first.
struct Counter {
  uint32_t arrived, listed;
};
constexpr int kSharedRows = kGroups / 2, kCounterBytes = kSharedRows * sizeof(Counter);
static_assert(kCounterBytes % 256 == 0);
struct alignas(256) State {
  Head head;
  u64 weight[kMostRuns + 1];
  uint32_t listed, arrived;
  union {
    u64 list[kList];
    struct { uint32_t count[kBins], least[kBins]; };
  };
  uint32_t most[kBins];
};
struct alignas(256) Part {
  u64 best, high;  // `high` with flags above: a NaN, too many of a step
  u64 steps[kSteps / 4];
};
struct Workspace {
  Counter* counters;
  State* states;
  Part* parts;
};
constexpr int kHeadWords = sizeof(Head) / 4;
static_assert(sizeof(Head) % 4 == 0 && kHeadWords <= kThreads);

template <typename T> __device__ __forceinline__ T read_through(const T* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename T> __device__ __forceinline__ void write_through(T* p, T x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename T> __device__ __forceinline__ T add_through(T* p, T x) { return __hip_atomic_fetch_add(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Whether this workgroup is the last of a row's.  What the others have written past the caches is there then: every wavefront waits until
// its writes are done, then the workgroup counts itself.
__device__ __forceinline__ bool all_arrived(Waves& waves, uint32_t* counter, uint32_t workgroups) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) waves.arrived = add_through(counter, 1u);
  __syncthreads();
  return waves.arrived == workgroups - 1;
}

// Rows that fit in the list: sorted whole.  16 rows of 2048 take 11 us, with steps 16.
template <typename T> __global__ void __launch_bounds__(kThreads) few_kernel(Args a, int64_t row0) {
  __shared__ Waves waves;
  __shared__ Lists lds;
  const int64_t r = row0 + blockIdx.x;
  const float temperature = parameter(a.temperature, r, 1.f);
  Row<T> row{static_cast<const T*>(a.logits) + r * a.stride, a.columns, a.log2_columns, {0.f, 0.0}};
  if (threadIdx.x < 64) waves.head.ask = ask_of(a, r, temperature);  // (all lanes write the same)
  bool nan;
  float low;
  const u64 best = best_of(waves, row, 0, a.columns, low, nan);
  if (is_answered(a, r, row, best, nan, !(temperature > 0.f))) return;
  row.scale = {row.score(best), waves.head.ask.factor};
  const uint32_t n = row.gather(lds, [&](float, int) { return true; });
  plan_all(waves, n, kSteps);
  if (threadIdx.x == 0) {
    const float top = row.scale.top;
    waves.head.plan.run[0].span(best, row.code(low, a.columns - 1)), waves.head.steps = {top, 0.5f * top, 1.f};
    if (top > 0.f && low < 0.f && top < INFINITY) waves.head.plan.run[0].span_even(0.f, waves.head.steps.down(low));
  }
  __syncthreads();
  find<true>(a, r, row, waves, lds);
}

// The scores of a row's piece.
__device__ __forceinline__ void piece_of(int columns, int pieces, int piece, int& first, int& count) {
  const int each = ((columns + pieces - 1) / pieces + 15) / 16 * 16;
  first = min(each * piece, columns), count = min(each, columns - first);
}

// What a workgroup has found in its piece goes past the caches: counts, and the list behind what others have listed.
__device__ __forceinline__ void give(Lists& lists, const Counts& counts, bool counted, u64 best, float high, bool nan, int count, State* state, Counter* counter,
                                     Part* part) {
  const int tid = threadIdx.x;
  bool too_many = false;
  if (counted) {
    u64 packed[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t n = counts.steps[tid * 8 + j];
      too_many |= n > 0xffff;
      packed[j / 4] |= (u64)(n & 0xffff) << 16 * (j % 4);
    }
    write_through(&part->steps[2 * tid], packed[0]), write_through(&part->steps[2 * tid + 1], packed[1]);
    if (count > 0xffff) too_many = __syncthreads_or(too_many);
  }
  if (tid == 0) {
    write_through(&part->best, best);
    write_through(&part->high, (u64)(nan ? 1 : 0) << 32 | (u64)(too_many ? 2 : 0) << 32 | __float_as_uint(high));
  }
  const uint32_t listed = counted ? counts.listed : lists.listed;
  if (listed) {
    if (tid == 0) lists.first = add_through(&counter->listed, listed);
    __syncthreads();
    const uint32_t first = lists.first;
    for (uint32_t i = tid; i < min(listed, (uint32_t)kList) && first + i < kList; i += kThreads)
      write_through(&state->list[first + i], counted ? (u64)__float_as_uint(counts.peaks[i]) : lists.list[i]);
  }
}
// All that others have found, by the last of them.  The row's counters are zero then.
__device__ __forceinline__ void take(Waves& waves, Lists& lists, Counts& counts, bool counted, u64& best, float& high, bool& nan, bool& too_many, State* state, Counter* counter, const Part* part, int pieces) {
  const int tid = threadIdx.x, lane = tid & 63;
  if (tid < 64) {
    u64 b = ~(u64)0;
    uint32_t flags = 0;
    float h = -INFINITY;
    for (int i = lane; i < pieces; i += 64) {
      const u64 x = read_through(&part[i].high);
      b = min(b, read_through(&part[i].best)), flags |= (uint32_t)(x >> 32), h = fmaxf(h, __uint_as_float((uint32_t)x));
    }
    const u64 any_nan = __ballot(flags & 1), any_many = __ballot(flags & 2);
#pragma unroll
    for (int d = 32; d; d >>= 1) b = min(b, (u64)__shfl_xor((long long)b, d));
    h = largest(h);
    if (tid == 0) waves.best[0] = b, waves.high[0] = h, waves.sure = (any_nan ? 1 : 0) | (any_many ? 2 : 0);
  }
  const uint32_t listed = read_through(&counter->listed);
  if (counted) {
    uint32_t n[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int i0 = 0; i0 < pieces; i0 += 8) {
      u64 x[8][2];
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) x[i][j] = read_through(&part[min(i0 + i, pieces - 1)].steps[2 * tid + j]);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i0 + i < pieces)
#pragma unroll
          for (int j = 0; j < 8; ++j) n[j] += (uint32_t)(x[i][j / 4] >> 16 * (j % 4)) & 0xffff;
    }
    for (int j = 0; j < 8; ++j) counts.steps[8 * tid + j] = n[j];
    for (uint32_t i = tid; i < min(listed, (uint32_t)kPeaks); i += kThreads) counts.peaks[i] = __uint_as_float((uint32_t)read_through(&state->list[i]));
  } else {
    for (uint32_t i = tid; i < min(listed, (uint32_t)kList); i += kThreads) lists.list[i] = read_through(&state->list[i]);
  }
  __syncthreads();
  if (tid == 0) {
    lists.listed = counts.listed = listed;
    write_through(&counter->arrived, 0u), write_through(&counter->listed, 0u);
  }
  best = waves.best[0], high = waves.high[0], nan = waves.sure & 1, too_many = waves.sure & 2;
  __syncthreads();
}

// The first pass over a longer row; SECOND: and all the rest, by one workgroup.  Else several share it, and the last of them goes on.
template <typename T, bool SECOND> __global__ void __launch_bounds__(kThreads) row_kernel(Args a, int64_t row0, Workspace w, int pieces) {
  __shared__ Waves waves;
  __shared__ Lists lists;
  __shared__ Counts counts;
  const int tid = threadIdx.x, slot = SECOND ? blockIdx.x : blockIdx.x / pieces, piece = SECOND ? 0 : blockIdx.x % pieces;
  const int64_t r = row0 + slot;
  State* const state = w.states + slot;
  Counter* const counter = w.counters + slot;
  Part* const parts = w.parts + (int64_t)slot * pieces;
  const float temperature = parameter(a.temperature, r, 1.f);
  const bool greedy = !(temperature > 0.f);
  Row<T> row{static_cast<const T*>(a.logits) + r * a.stride, a.columns, a.log2_columns, {0.f, 0.0}};
  bool nan = false, too_many = false;
  int first = 0, count = a.columns;
  if (!SECOND) piece_of(a.columns, pieces, piece, first, count);
  bool shared = !SECOND && pieces > 1;
  u64 best = ~(u64)0;
  float high = -INFINITY;
  // A piece of the row is done: true if others go on.  What all have found is here then.
  auto is_others = [&](bool counted) {
    if (!shared) return false;
    give(lists, counts, counted, best, high, nan, count, state, counter, parts + piece);
    if (!all_arrived(waves, &counter->arrived, pieces)) return true;
    take(waves, lists, counts, counted, best, high, nan, too_many, state, counter, parts, pieces);
    shared = false, first = 0, count = a.columns;
    return false;
  };
  if (!SECOND && !shared && tid == 0) state->head.planned = 0;
  if (greedy) {
    best = best_of(waves, row, first, count, high, nan);
    if (tid == 0) lists.listed = 0;
    __syncthreads();
    if (is_others(false)) return;
    if (!SECOND && tid == 0) state->head.planned = 0;
    is_answered(a, r, row, best, nan, true);
    return;
  }
  look(a, r, row.row, temperature, waves, counts);
  __syncthreads();
  float bound = counts.bound;
  row.scale.factor = waves.head.ask.factor;
  const Steps steps = waves.head.steps;
  if (bound == bound) {
    const uint32_t top_k = waves.head.ask.top_k;
#pragma unroll 1
    for (int turn = 0;; ++turn) {
      high = gather_above(waves, lists, row, steps, first, count, bound, nan);
      if (is_others(false)) return;
      if (turn || lists.listed <= kList || (top_k && top_k <= kBounded)) break;
      // (min_p alone: with the highest score known the bound is what it has to be)
      bound = fmaxf(steps.down((float)fmax((double)high - waves.head.ask.far / row.scale.factor, -(double)FLT_MAX)), 0.f) + 1.f;
      __syncthreads();
    }
    if (!SECOND && tid == 0) state->head.planned = 0;
    if (is_answered(a, r, row, high > -INFINITY ? 0 : ~(u64)0, nan, false)) return;
    const uint32_t n = lists.listed;
    if (n && n <= kList && (n >= top_k || bound == INFINITY)) {
      row.scale.top = high;
      plan_all(waves, n, bound < kSteps - 4 ? (int)bound : kSteps - 2);
      __syncthreads();
      if (find<false>(a, r, row, waves, lists)) return;
    }
    __syncthreads();
  }
#pragma unroll 1
  do {
    high = count_steps(waves, counts, row, steps, first, count, nan);
    too_many = false;
    if (is_others(true)) return;
  } while (too_many);
  if (!SECOND && tid == 0) state->head.planned = 0;
  if (is_answered(a, r, row, high > -INFINITY ? 0 : ~(u64)0, nan, false)) return;
  row.scale.top = high;
  plan_row(waves, counts, row.scale);
  if constexpr (SECOND) {
    if (waves.head.plan.slow != kSlow) {
      gather_plan(waves.head.plan, lists, row, steps, 0, a.columns);
      if (waves.head.plan.slow ? find_equal(a, r, row, waves, lists) : find<false>(a, r, row, waves, lists)) return;
    }
    find_slowly(a, r, row, waves, lists);
  } else {
    if (tid == 0) waves.head.planned = kPlanned, waves.head.top = high, state->listed = state->arrived = 0;
    if (tid <= kMostRuns) state->weight[tid] = 0;
    if (waves.head.plan.slow)
      for (int i = tid; i < kBins; i += kThreads) state->count[i] = state->most[i] = 0, state->least[i] = ~0u;
    __syncthreads();
    if (tid < kHeadWords) reinterpret_cast<uint32_t*>(&state->head)[tid] = reinterpret_cast<const uint32_t*>(&waves.head)[tid];
  }
}

// The second pass over a row, by several workgroups; the last of them does the rest.
template <typename T> __global__ void __launch_bounds__(kThreads) gather_kernel(Args a, int64_t row0, Workspace w, int pieces) {
  __shared__ Waves waves;
  __shared__ Lists lds;
  const int tid = threadIdx.x, slot = blockIdx.x / pieces, piece = blockIdx.x % pieces;
  const int64_t r = row0 + slot;
  State* const state = w.states + slot;
  if (state->head.planned != kPlanned) return;
  if (tid < kHeadWords) reinterpret_cast<uint32_t*>(&waves.head)[tid] = reinterpret_cast<const uint32_t*>(&state->head)[tid];
  __syncthreads();
  const Row<T> row{static_cast<const T*>(a.logits) + r * a.stride, a.columns, a.log2_columns, {waves.head.top, waves.head.ask.factor}};
  const int slow = waves.head.plan.slow;
  if (slow == kSlow) {
    if (piece) return;
  } else {
    int first, count;
    piece_of(a.columns, pieces, piece, first, count);
    gather_plan(waves.head.plan, lds, row, waves.head.steps, first, count);
    if (tid <= kMostRuns && lds.weight[tid]) add_through(&state->weight[tid], lds.weight[tid]);
    if (slow) {
      for (int i = tid; i < kBins; i += kThreads) {
        if (!lds.count[i]) continue;
        add_through(&state->count[i], lds.count[i]);
        __hip_atomic_fetch_min(&state->least[i], lds.least[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_fetch_max(&state->most[i], lds.most[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    } else {
      const uint32_t listed = lds.listed;
      if (tid == 0) lds.first = listed ? add_through(&state->listed, listed) : 0;
      __syncthreads();
      for (uint32_t i = tid; i < min(listed, (uint32_t)kList) && lds.first + i < kList; i += kThreads) write_through(&state->list[lds.first + i], lds.list[i]);
    }
    if (!all_arrived(waves, &state->arrived, pieces)) return;
    if (tid <= kMostRuns) lds.weight[tid] = read_through(&state->weight[tid]);
    if (slow) {
      for (int i = tid; i < kBins; i += kThreads) lds.count[i] = read_through(&state->count[i]), lds.least[i] = read_through(&state->least[i]), lds.most[i] = read_through(&state->most[i]);
    } else {
      for (uint32_t i = tid; i < waves.head.plan.tokens; i += kThreads) lds.list[i] = read_through(&state->list[i]);
      if (tid == 0) lds.listed = read_through(&state->listed);
    }
    __syncthreads();
    if (slow ? find_equal(a, r, row, waves, lds) : find<false>(a, r, row, waves, lds)) return;
  }
  find_slowly(a, r, row, waves, lds);
}

int64_t states_of(int64_t rows) { return std::max<int64_t>(1, std::min<int64_t>(rows, kSharedRows)); }

template <typename T> void launch(const Args& a, int64_t rows, void* workspace, hipStream_t stream) {
  if (a.columns <= kList) {
    for (int64_t row0 = 0; row0 < rows; row0 += kMostFew)
      hipLaunchKernelGGL(few_kernel<T>, dim3((unsigned)std::min(rows - row0, kMostFew)), dim3(kThreads), 0, stream, a, row0);
    return;
  }
  Workspace w{static_cast<Counter*>(workspace), reinterpret_cast<State*>(static_cast<char*>(workspace) + kCounterBytes), nullptr};
  w.parts = reinterpret_cast<Part*>(w.states + states_of(rows));
  for (int64_t row0 = 0; row0 < rows; row0 += kMostRows) {
    const int n = (int)std::min<int64_t>(rows - row0, kMostRows), pieces = std::min(kGroups / n, a.columns / kLeastPiece);
    if (pieces < 2) {
      hipLaunchKernelGGL((row_kernel<T, true>), dim3((unsigned)n), dim3(kThreads), 0, stream, a, row0, w, 1);
    } else {
      int counted = std::min({kGroups / n, a.columns / kLeastCounted, kMostCounts});
      if (counted < kFewestCounts) counted = 1;
      hipLaunchKernelGGL((row_kernel<T, false>), dim3((unsigned)(n * counted)), dim3(kThreads), 0, stream, a, row0, w, counted);
      hipLaunchKernelGGL(gather_kernel<T>, dim3((unsigned)(n * pieces)), dim3(kThreads), 0, stream, a, row0, w, pieces);
    }
  }
}

}  // namespace

extern "C" {

int64_t rsr_sample_workspace(int64_t rows, int64_t columns) {
  if (rows < 0 || rows > 1 << 24) return set_error(RSR_ERR_INVALID_ARGUMENT, "rows must be in 0..2^24");
  if (columns < 1 || columns > 1 << 22) return set_error(RSR_ERR_INVALID_ARGUMENT, "columns must be in 1..2^22");
  const int64_t parts = std::min<int64_t>(kGroups, std::min<int64_t>(rows, kMostRows) * (columns / kLeastCounted));
  return kCounterBytes + states_of(rows) * (int64_t)sizeof(State) + parts * (int64_t)sizeof(Part);
}

int rsr_sample(const void* logits, int64_t rows, int64_t columns, int64_t stride, int dtype, const float* temperature, const int32_t* top_k,
               const float* top_p, const float* min_p, const float* uniform, int32_t* token, float* probability, int32_t* kept, void* workspace,
               int64_t workspace_bytes, void* stream) {
  const int64_t need = rsr_sample_workspace(rows, columns);
  if (need < 0) return (int)need;
  if (dtype != RSR_F32 && dtype != RSR_F16 && dtype != RSR_BF16) return set_error(RSR_ERR_INVALID_ARGUMENT, "dtype must be RSR_F32, RSR_F16 or RSR_BF16");
  if (stride < columns) return set_error(RSR_ERR_INVALID_ARGUMENT, "a stride is shorter than a row");
  if (rows == 0) return RSR_OK;
  if (!logits || !uniform || !token) return set_error(RSR_ERR_INVALID_ARGUMENT, "null pointer");
  const void* const outputs[] = {token, probability, kept};
  const void* const inputs[] = {logits, temperature, top_k, top_p, min_p, uniform, workspace};
  for (int i = 0; i < 3; ++i) {
    bool twice = false;
    for (const void* p : inputs) twice |= outputs[i] == p;
    for (int j = 0; j < i; ++j) twice |= outputs[i] == outputs[j];
    if (outputs[i] && twice) return set_error(RSR_ERR_INVALID_ARGUMENT, "an output must not be an input, the workspace or another output");
  }
  if (!rsr_internal::aligned(logits, rsr_internal::size_of(dtype))) return set_error(RSR_ERR_INVALID_ARGUMENT, "logits must be aligned as their elements");
  if (!workspace || !rsr_internal::aligned(workspace, 256) || workspace_bytes < need)
    return set_error(RSR_ERR_INVALID_ARGUMENT, "the workspace is missing, too small or not 256-byte aligned");
  Args a{logits, temperature, top_p, min_p, uniform, top_k, token, probability, kept, stride, (int32_t)columns, 1};
  while ((int64_t)1 << a.log2_columns < columns) ++a.log2_columns;
  (dtype == RSR_F32 ? launch<float> : dtype == RSR_F16 ? launch<_Float16> : launch<__bf16>)(a, rows, workspace, static_cast<hipStream_t>(stream));
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(RSR_ERR_HIP, std::string("rsr_sample: ") + hipGetErrorString(e));
  return RSR_OK;
}

}  // extern "C"
