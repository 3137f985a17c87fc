// A token for every row of scores (include/rsr_decode.h).
//
// With the scores in order, the highest first, everything that is asked for is a place in one running sum: of tokens (top-k), of
// weights (top-p, the token itself), or a score (min-p).  No row is sorted for that.
//   1. One pass finds the highest score and counts the scores in 16383 steps between the lowest and the highest of some of
//      them (those above go into a list).  Counts times the weights at a step's ends bound every sum of weights from both sides, by some
//      hundredths or tenths of a percent, and so the steps in which the places can be.
//   2. A second pass adds up what lies before these steps, in 64 bits, and gathers what is in them in LDS, where it is sorted and the
//      places are found.
// If too many tokens are there (thousands of equal scores, say), the slow way is taken: a histogram with count and weight of each bin, 2048
// bins of 1/32 of an octave of weight, and place after place with finer ones of what is left.
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
constexpr int kSteps = 16 * kThreads;  // of counted scores; the first has what is above all others
constexpr int kPeaks = 2 * kThreads;   // scores above the steps
constexpr int kPrefix = 1024;        // tokens that are rather gathered from the first one on than counted

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

constexpr int kPlaces = 7, kMostRuns = 4;

// The bin or step of a place, with the sums up to it and up to and with it.
struct Mark {
  int bin;
  uint32_t before, count;
  double mass_before, mass;
};

struct Lds {
  union {
    uint32_t steps[kSteps];                     // counted scores
    struct {
      u64 list[kList];                          // tokens, sorted
      double upto[kList];                       // weight up to and with each
      uint32_t count[kBins];                    // up to and with the bin
      union { u64 sum[kBins]; double mass[kBins]; };  // packed as above; then the weight up to and with the bin
      uint32_t part_count[kBins + 1];           // of a finer histogram, or where buckets begin
      union { u64 part_sum[kBins]; double part_mass[kBins]; u64 bucketed[kList]; };
    };
  };
  float peaks[kPeaks];
  u64 weight[kMostRuns + 1];  // before each run, and of all
  Mark mark[2 * kMostRuns + 1];
  double wave_mass[kWaves];
  uint32_t wave_count[kWaves];
  u64 wave_best[kWaves];
  float wave_low[kWaves], wave_high[kWaves];
  uint32_t place[kPlaces];  // bins of places
  uint32_t listed, all_count;
  double all_mass;
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

// f(scores, column of the first) for pieces of `count` scores of a row from column `first` on, by all threads of the workgroup, each in
// ascending order.  Reads are 16 bytes wide wherever the row begins, 16 scores on their way while 16 are looked at; what sticks out at the ends is read by
// itself and comes with minus infinity behind it.
template <typename T, typename F> __device__ __forceinline__ void for_pieces(const T* row, int first, int count, F f) {
  typedef const __attribute__((address_space(1))) T* Scores;
  typedef const __attribute__((address_space(1))) u4* Pieces;
  constexpr int kWide = 16 / sizeof(T), kAtOnce = sizeof(T) == 4 ? 4 : 2;
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
  for_pieces(row, first, count, [&](const float (&x)[16 / sizeof(T)], int column) {
#pragma unroll
    for (int j = 0; j < 16 / (int)sizeof(T); ++j) f(x[j], column + j);
  });
}

// ---- weights ----------------------------------------------------------------------------------------------
// A score's distance below the highest, in octaves of its weight: the weight is 2^-distance, 1 exactly for the highest.
struct Scale {
  float top;
  double factor;
  __device__ double distance(float x) const { return x == top ? 0.0 : ((double)top - (double)x) * factor; }
  __device__ double weight(float x) const { return exp2(-distance(x)); }
};

// Sums of weights in units of 2^-40 of the highest's, in whole numbers, so that no order of additions matters.  2^f, f from -1/2 to 1/2,
// is the polynomial that has its values at nine Chebyshev nodes (off by 2^-39 of it); a weight is added to 2^12, where 2^-40 is the last
// bit, and the bits of that are added up.
struct Weights {
  double top, factor;
  static constexpr double kAbove = 0x1p12;
  __device__ __forceinline__ u64 of(float x) const {
    const double d = fmin((top - (double)x) * factor, 1000.0), n = rint(d), f = n - d;  // (nothing is left of the weight there)
    const double p = 1.0 + f * (0.6931471805459335 + f * (0.2402265069581299 + f * (0.05550410941205934 + f * (0.009618129159402607 + f * (0.0013333450567999429 +
                     f * (0.00015403455852420792 + f * (1.5310079402541085e-05 + f * 1.3255224885567153e-06)))))));
    const uint32_t power = (uint32_t)(1023 - (int)n) << 20;
    return __builtin_bit_cast(u64, fma(p, __builtin_bit_cast(double, (u64)power << 32), kAbove));
  }
  static __device__ __forceinline__ u64 none() { return __builtin_bit_cast(u64, kAbove); }
};
__device__ __forceinline__ int bin_of(double distance) { return (int)fmin(distance * kPerOctave, (double)(kBins - 1)); }

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

// Running sums of two entries per thread, in their order, and what is before them.
struct Sums {
  uint32_t c[2], c_before;
  double m[2], m_before;

  __device__ __forceinline__ void scan(Lds& lds, uint32_t c0, double m0) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t cs = sum_of_lanes(c[0] + c[1]);
    const double ms = sum_of_lanes(m[0] + m[1]);
    __syncthreads();
    if (lane == 63) lds.wave_count[wave] = cs, lds.wave_mass[wave] = ms;
    __syncthreads();
    const uint32_t cw = sum_of_16(lds.wave_count[lane & 15]);
    const double mw = sum_of_16(lds.wave_mass[lane & 15]);
    c_before = c0, m_before = m0;
    if (wave) c_before += of_lane(cw, wave - 1), m_before += of_lane(mw, wave - 1);
    c_before += moved<0x138, 0xf>(cs), m_before += moved<0x138, 0xf>(ms);  // (of the lane before)
    c[0] += c_before, m[0] += m_before, c[1] += c[0], m[1] += m[0];
  }
};

// ---- places -----------------------------------------------------------------------------------------------
// The place where a running sum reaches what is asked for.
struct Place {
  bool of_count, strict;  // a sum of tokens (at least `count`), or of weights: at least `mass`, or more than that
  uint32_t count;
  double mass;
  __device__ bool reached(uint32_t c, double m) const { return of_count ? c >= count : strict ? m > mass : m >= mass; }
  static __device__ Place tokens(uint32_t n) { return {true, false, n, 0.0}; }
  static __device__ Place weight(double m, bool more) { return {false, more, 0, m}; }
};

// The first of n running sums that reaches the place; the last one if none does.
__device__ __forceinline__ int first_at(const Place& p, const uint32_t* count, const double* mass, int n) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (p.reached(count ? count[mid] : 0, mass[mid])) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

// Tokens of neighbouring steps that lie in the list, one run behind the other.
struct Run {
  int b0, b1;                     // steps
  uint32_t start, count, before;  // where it begins in the list, how many there are, and before them in the row
  double mass_before;             // and the weight of those
  u64 code;                       // about that of the first, for sorting
  int shift;                      // and how far apart its buckets are

  // as many buckets as tokens, or half as many, from one code to another
  __device__ __forceinline__ void span(u64 from, u64 to) {
    code = from;
    shift = max(0, __clz((int)count) + 33 - __clzll((long long)(to > from ? to - from : 1)));
  }
  __device__ __forceinline__ uint32_t bucket(u64 x) const { return start + (x < code ? 0 : (uint32_t)min((x - code) >> shift, (u64)(count - 1))); }
};
struct Runs {
  static constexpr int kMost = kMostRuns;
  Run run[kMost];
  int n;
  int near;         // the run up to this step has the last token that min_p keeps; -1: min_p keeps all
  uint32_t tokens;  // of all runs
};

// What a row is asked for.
struct Ask {
  uint32_t top_k;  // 0: all
  double top_p;    // 2: all
  double far;      // the distance of the last that min_p keeps, or infinity
  double u;
};

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
  template <typename W> __device__ __forceinline__ uint32_t gather(Lds& lds, W wanted) const {
    __syncthreads();
    if (threadIdx.x == 0) lds.listed = 0;
    __syncthreads();
    for_each(row, 0, columns, [&](float x, int column) {
      if (x == -INFINITY || !wanted(x, column)) return;
      const uint32_t at = atomicAdd(&lds.listed, 1u);
      if (at < kList) lds.list[at] = code(x, column);
    });
    __syncthreads();
    return lds.listed;
  }

  // Sorts the list and adds up its weights.  Codes are dealt into buckets, as many for each run as it has tokens, and each finds its
  // place among those of its bucket.  (What lies outside the bounds of its run lands in a bucket at the end, still in order.)
  __device__ __forceinline__ void sort(Lds& lds, const Runs& runs) const {
    const int tid = threadIdx.x;
    const uint32_t n = runs.tokens;
    u64 x[2];
    uint32_t bucket[2], slot[2];
    lds.part_count[2 * tid] = lds.part_count[2 * tid + 1] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t i = tid + j * kThreads;
      if (i >= n) continue;
      x[j] = lds.list[i];
      bucket[j] = runs.run[0].bucket(x[j]);
#pragma unroll
      for (int k = 1; k < Runs::kMost; ++k)
        if (k < runs.n && x[j] >= runs.run[k].code) bucket[j] = runs.run[k].bucket(x[j]);
      slot[j] = atomicAdd(&lds.part_count[bucket[j]], 1u);
    }
    __syncthreads();
    Sums s;
#pragma unroll
    for (int j = 0; j < 2; ++j) s.c[j] = lds.part_count[2 * tid + j], s.m[j] = 0.0;
    s.scan(lds, 0, 0.0);
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
    s.scan(lds, 0, 0.0);
    lds.upto[2 * tid] = s.m[0], lds.upto[2 * tid + 1] = s.m[1];
    __syncthreads();
  }

  // ---- places in the list
  static __device__ double mass_at(const Lds& lds, const Run& r, uint32_t i) { return r.mass_before + (lds.upto[i] - (r.start ? lds.upto[r.start - 1] : 0.0)); }
  // The first token of the list at the place, and its run.  (Loops over runs are unrolled: they stay in registers.)
  static __device__ __forceinline__ uint32_t seek(const Lds& lds, const Runs& runs, Place p, Run& r) {
    r = runs.run[0];
#pragma unroll
    for (int i = 1; i < Runs::kMost; ++i)
      if (i < runs.n && !p.reached(r.before + r.count, mass_at(lds, r, r.start + r.count - 1))) r = runs.run[i];
    if (p.of_count) return r.start + min(max(p.count, r.before + 1) - r.before, r.count) - 1;
    p.mass -= r.mass_before - (r.start ? lds.upto[r.start - 1] : 0.0);
    return r.start + first_at(p, nullptr, lds.upto + r.start, r.count);
  }

  // Whether the place that seek found is where the sum reaches it: not before its run, and not behind.
  static __device__ bool sure(const Lds& lds, const Place& p, const Run& r, uint32_t all) {
    return (!r.before || !p.reached(r.before, r.mass_before)) && (r.before + r.count == all || p.reached(r.before + r.count, mass_at(lds, r, r.start + r.count - 1)));
  }

  // The answer, where the list has all places.  `kept`, `mass`: all tokens and their weight (if a place or the token needs it).  Nothing
  // is `sure` if a place is in none of the runs.
  __device__ __forceinline__ Found solve(const Lds& lds, const Ask& ask, const Runs& runs, uint32_t kept, double mass) const {
    Run r;
    bool is_sure = true;
    const uint32_t all = kept;
    if (ask.top_k && ask.top_k < kept) {
      const Place p = Place::tokens(ask.top_k);
      const uint32_t at = seek(lds, runs, p, r);
      is_sure &= sure(lds, p, r, all);
      kept = ask.top_k, mass = mass_at(lds, r, at);
    }
    if (ask.top_p < 1.0) {
      const Place p = Place::weight(ask.top_p * mass, false);
      const uint32_t at = seek(lds, runs, p, r), n = r.before + at - r.start + 1;
      is_sure &= sure(lds, p, r, all);
      if (n < kept) kept = n, mass = mass_at(lds, r, at);
    }
    if (runs.near >= 0) {
      r = runs.run[0];
#pragma unroll
      for (int i = 1; i < Runs::kMost; ++i)
        if (i < runs.n && runs.run[i].b0 <= runs.near) r = runs.run[i];
      uint32_t lo = 0, hi = r.count;  // how many are near enough
      while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (scale.distance(score(lds.list[r.start + mid])) <= ask.far) lo = mid + 1;
        else hi = mid;
      }
      is_sure &= lo < r.count || r.before + r.count >= kept;
      if (r.before + lo < kept) kept = r.before + lo, mass = lo ? mass_at(lds, r, r.start + lo - 1) : r.mass_before;
    }
    const Place p = Place::weight(ask.u * mass, true);
    const uint32_t at = seek(lds, runs, p, r);
    return {lds.list[at], scale.weight(score(lds.list[at])) / mass, kept, is_sure && sure(lds, p, r, all)};
  }

  // ---- place after place (a list for each), where there are too many tokens for one list
  // The run of tokens in which the place is.
  __device__ __attribute__((noinline)) Run run_at(Lds& lds, const Place& p) const {
    const int tid = threadIdx.x;
    int b = first_at(p, lds.count, lds.mass, kBins);
    while (b && lds.count[b] == lds.count[b - 1]) --b;  // (what rounding puts behind the last token is the last token's)
    uint32_t before = b ? lds.count[b - 1] : 0, count = lds.count[b] - before;
    double mass_before = b ? lds.mass[b - 1] : 0.0;
    u64 lo = 0, hi = ((u64)1 << (32 + log2_columns)) - 1;
    while (count > kList) {
      const int shift = max(0, 64 - __clzll((long long)(hi - lo)) - 11);
      Sums s{{0, 0}, 0, {0.0, 0.0}, 0.0};
      for (int first = 0; first < columns; first += kChunk) {
        __syncthreads();
        lds.part_sum[2 * tid] = lds.part_sum[2 * tid + 1] = 0;
        __syncthreads();
        for_each(row, first, min(kChunk, columns - first), [&](float x, int column) {
          if (x == -INFINITY) return;
          const double d = scale.distance(x);
          const u64 c = code(x, column);
          if (bin_of(d) == b && c >= lo && c <= hi) atomicAdd(&lds.part_sum[(c - lo) >> shift], packed(d, b));
        });
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 2; ++j) s.c[j] += count_in(lds.part_sum[2 * tid + j]), s.m[j] += mass_in(lds.part_sum[2 * tid + j], b);
      }
      s.scan(lds, before, mass_before);
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
    Runs runs;
    runs.n = 1, runs.near = -1, runs.tokens = count;
    Run& r = runs.run[0];
    r = {b, b, 0, count, before, mass_before, 0, 0};
    if (!lo && scale.top < INFINITY)  // (the bin's ends, or what is left of it)
      lo = code((float)((double)scale.top - b / (kPerOctave * scale.factor)), 0), hi = code((float)((double)scale.top - (b + 1) / (kPerOctave * scale.factor)), 0);
    r.span(lo, hi);
    sort(lds, runs);
    return r;
  }

  __device__ __attribute__((noinline)) Found solve_slowly(Lds& lds, const Ask& ask) const {
    uint32_t kept = lds.count[kBins - 1];
    double mass = lds.mass[kBins - 1];
    Runs runs{};
    Run r;
    uint32_t at;
    auto find = [&](const Place& p) {
      const Run& have = runs.run[0];
      const bool here = runs.n && !p.reached(have.before, have.mass_before) && p.reached(have.before + have.count, mass_at(lds, have, have.count - 1));
      if (!here) runs.run[0] = run_at(lds, p), runs.n = 1;
      at = seek(lds, runs, p, r);
    };
    if (ask.top_k && ask.top_k < kept) {
      find(Place::tokens(ask.top_k));
      kept = ask.top_k, mass = mass_at(lds, r, at);
    }
    if (ask.top_p < 1.0) {
      find(Place::weight(ask.top_p * mass, false));
      const uint32_t n = r.before + at + 1;
      if (n < kept) kept = n, mass = mass_at(lds, r, at);
    }
    if (ask.far < INFINITY) {
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
          for_each(row, first, min(kChunk, columns - first), [&](float x, int) {
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
    find(Place::weight(ask.u * mass, true));
    return {lds.list[at], scale.weight(score(lds.list[at])) / mass, kept, true};
  }
};

// ---- steps ------------------------------------------------------------------------------------------------
// Scores to steps, the higher ones first: 0 for what is above the first of the others, the last but one for what is below them.  (A
// difference of halves, which is not beyond the range of float, times the steps of half a unit.)
struct Steps {
  float from, half, per;
  __device__ __forceinline__ float down(float x) const { return fmaf(-0.5f, x, half) * per; }
  __device__ __forceinline__ float score(int step) const { return 2.f * (half - (float)step / per); }  // at about the end of a step
  static __device__ __forceinline__ int step(float down) { return down < 0.f ? 0 : 1 + (int)min((uint32_t)down, (uint32_t)(kSteps - 3)); }
  // The bounds of `down` from step lo to step hi, both included.
  static __device__ __forceinline__ float first_of(int lo) { return lo ? (float)(lo - 1) : -INFINITY; }
  static __device__ __forceinline__ float last_of(int hi) { return hi >= kSteps - 2 ? INFINITY : hi ? __uint_as_float(__float_as_uint((float)hi) - 1) : -FLT_MIN; }
};

__device__ __forceinline__ void over_lanes_max(float& x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
}

// Steps from the highest of some thousand scores of a row down to the lowest, or to the last that has any weight.
template <typename T> __device__ __forceinline__ Steps look(Lds& lds, const Row<T>& row, double factor) {
  constexpr int kWide = 16 / sizeof(T);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int head = (int)((16 - (reinterpret_cast<uintptr_t>(row.row) & 15)) & 15) / (int)sizeof(T), pieces = (row.columns - head) / kWide;
  const u4 v = *reinterpret_cast<const u4*>(row.row + head + (int64_t)((int64_t)tid * pieces / kThreads) * kWide);
  T x[kWide];
  __builtin_memcpy(x, &v, 16);
  float high = -INFINITY, low = INFINITY;
#pragma unroll
  for (int j = 0; j < kWide; ++j) {
    const float f = (float)x[j];
    if (f > -INFINITY && f < INFINITY) high = fmaxf(high, f), low = fminf(low, f);
  }
  low = -low;
  over_lanes_max(high), over_lanes_max(low);
  if (lane == 0) lds.wave_high[wave] = high, lds.wave_low[wave] = low;
  __syncthreads();
  // Above the first step are some hundred scores: those above the `rank`-th of the wavefronts' highest.
  const int rank = max(1, min(kWaves / 4, (kWaves / 4 << 17) / row.columns));
  const float mine = lds.wave_high[lane & (kWaves - 1)];
  int higher = 0;
  for (int w = 0; w < kWaves; ++w) {
    const float other = lds.wave_high[w];
    higher += other > mine || (other == mine && w < (lane & (kWaves - 1)));
    low = fmaxf(low, lds.wave_low[w]);
  }
  high = of_lane(mine, __builtin_ctzll(__ballot(higher == rank - 1)));
  low = -low;
  if (!(high > -INFINITY)) return {-FLT_MAX, -FLT_MAX / 2, 1.f};
  const double range = fmin((double)high - (double)low, 48.0 / factor);
  return {high, 0.5f * high, (float)fmin(2.0 * (kSteps - 3) / range, (double)FLT_MAX)};
}

// Counts scores in steps, lists those above them; the highest score, and whether one is NaN.
template <typename T> __device__ __forceinline__ float count_steps(Lds& lds, const Row<T>& row, const Steps& steps, int first, int count, bool& nan) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  u4* const zero = reinterpret_cast<u4*>(lds.steps);
  for (int i = tid; i < kSteps / 4; i += kThreads) zero[i] = u4{0, 0, 0, 0};
  if (tid == 0) lds.listed = 0;
  __syncthreads();
  float high = -INFINITY;
  for_pieces(row.row, first, count, [&](const float (&x)[16 / sizeof(T)], int) {
    bool above = false;
#pragma unroll
    for (int j = 0; j < 16 / (int)sizeof(T); ++j) {
      high = __builtin_elementwise_maximum(high, x[j]);  // (NaN stays)
      const float down = steps.down(x[j]);
      above |= down < 0.f;
      if (down >= 0.f && x[j] > -INFINITY) atomicAdd(&lds.steps[1 + min((uint32_t)down, (uint32_t)(kSteps - 3))], 1u);
    }
    if (above)  // (seldom)
#pragma unroll
      for (int j = 0; j < 16 / (int)sizeof(T); ++j)
        if (steps.down(x[j]) < 0.f) {
          const uint32_t at = atomicAdd(&lds.listed, 1u);
          if (at < kPeaks) lds.peaks[at] = x[j];
        }
  });
  nan = __syncthreads_or(high != high);
  over_lanes_max(high);
  if (lane == 0) lds.wave_high[wave] = high;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) high = fmaxf(high, lds.wave_high[w]);
  return high;
}

struct Plan {
  Runs runs;
  uint32_t all;   // tokens
  bool weighed;   // the second pass adds up weights
  bool slow;      // too many tokens
};

// In which steps the places may be, and so which tokens are gathered.  The scores above the steps are weighed one by one, a step as its
// count times the weight in its middle.  Where a step's scores lie in it is not known: it is off by its weight times its width (in
// ln 2 octaves) over the root of 12, as if they all lay at one place of which any is as likely, and the sums of all are off by the root of the
// squares of that; six times as much is allowed for.  (Whether that was enough is seen in the end.)
__device__ __forceinline__ Plan plan_of(Lds& lds, const Scale& scale, const Steps& steps, const Ask& ask) {
  constexpr int kEach = kSteps / kThreads;
  constexpr double kRounded = 1e-5;  // of a sum: what weights are rounded by here, and more
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  static_assert(kEach == 16);
  const uint32_t peaks = lds.listed;
  Plan plan;
  plan.slow = peaks > kPeaks || scale.top == INFINITY;
  if (plan.slow) return plan;
  double peak = 0.0;
#pragma unroll
  for (int j = 0; j < 2; ++j)
    if ((uint32_t)(tid + j * kThreads) < peaks) peak += scale.weight(lds.peaks[tid + j * kThreads]);
  peak = sum_of_lanes(peak);
  if (lane == 63) lds.wave_mass[wave] = peak;
  if (tid == 0) lds.steps[0] = peaks;
  if (tid < 2 * kMostRuns) lds.mark[tid].bin = kSteps;
  __syncthreads();
  peak = 0.0;
  for (int w = 0; w < kWaves; ++w) peak += lds.wave_mass[w];

  // the sums of each thread's steps
  const double octaves = 2.0 * scale.factor / steps.per, above = ((double)scale.top - (double)steps.from) * scale.factor - 0.5 * octaves;
  auto weight_of = [&](uint32_t n, int step) { return step ? n * (double)__builtin_amdgcn_exp2f(-fmaxf((float)(above + step * octaves), 0.f)) : peak; };
  float squares = 0.f;
  Sums s{{0, 0}, 0, {0.0, 0.0}, 0.0};
#pragma unroll
  for (int j = 0; j < kEach / 4; ++j) {
    const u4 n = reinterpret_cast<const u4*>(lds.steps)[tid * (kEach / 4) + j];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int step = tid * kEach + 4 * j + i;
      const double w = weight_of(n[i], step);
      s.c[0] += n[i], s.m[0] += w;
      squares += step ? (float)(w * w) : 0.f;
    }
  }
  s.scan(lds, 0, 0.0);
  squares = sum_of_lanes(squares);
  if (lane == 63) lds.wave_low[wave] = squares;
  if (tid == kThreads - 1) lds.all_count = s.c[0], lds.all_mass = s.m[0];
  // The step of a place: the wavefront in which a thread's sums reach it adds up the steps of that thread, a lane each.
  auto mark = [&](int place, auto reached) {
    const u64 here = __ballot(s.c[0] > s.c_before && reached(s.c[0], s.m[0]) && (!s.c_before || !reached(s.c_before, s.m_before)));
    if (!here) return;
    const int thread = __builtin_ctzll(here), step = ((wave << 6) + thread) * kEach + (lane & (kEach - 1));
    const uint32_t n = lds.steps[step], c = of_lane(s.c_before, thread) + sum_of_16(n);
    const double w = weight_of(n, step), m = of_lane(s.m_before, thread) + sum_of_16(w);
    const u64 some = __ballot(lane < kEach && n), at = __ballot(lane < kEach && n && reached(c, m));
    if (lane == (at ? __builtin_ctzll(at) : 63 - __builtin_clzll(some))) lds.mark[place] = {step, c - n, c, m - w, m};
  };
  auto up_to = [&](double mass, bool more) { return [=](uint32_t, double m) { return more ? m > mass : m >= mass; }; };
  auto tokens = [&](uint32_t count) { return [=](uint32_t c, double) { return c >= count; }; };

  __syncthreads();
  const uint32_t all = lds.all_count;
  const double total = lds.all_mass;
  squares = 0.f;
  for (int w = 0; w < kWaves; ++w) squares += lds.wave_low[w];
  const double off = 6.0 * 0.6931471805599453 / 3.4641016151377544 * octaves * sqrt((double)squares) + kRounded * total;
  const bool k = ask.top_k && ask.top_k < all, p = ask.top_p < 1.0;
  bool m = ask.far < INFINITY;
  mark(0, tokens(all));
  if (k) mark(1, tokens(ask.top_k));
  if (m) {
    // the first tokens from the step before that of the last score that is kept on, and from the one behind it on
    const int step = Steps::step(steps.down((float)((double)scale.top - ask.far / scale.factor)));
    const int at[2] = {max(step - 1, 0), min(step + 1, kSteps - 1)};
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (tid == at[i] / kEach) {
        uint32_t c = s.c_before;
        for (int j = 0; j < at[i] % kEach; ++j) c += lds.steps[tid * kEach + j];
        lds.place[i] = c;
      }
    __syncthreads();
    mark(4, tokens(lds.place[0] + 1)), mark(5, tokens(lds.place[1] + 1));
  }
  __syncthreads();
  auto marked = [&](int place, const Mark& end) { return lds.mark[place].bin < end.bin ? lds.mark[place] : end; };
  Mark end = lds.mark[0];
  int lo[Runs::kMost], hi[Runs::kMost];             // of top_k, top_p, min_p, and the token
  uint32_t before[Runs::kMost], upto[Runs::kMost];  // tokens before, and up to and with
#pragma unroll
  for (int i = 0; i < Runs::kMost; ++i) lo[i] = hi[i] = kSteps, before[i] = upto[i] = 0;  // none
  double least = total - off, most = total + off;
  if (k) {
    end = lds.mark[1];
    lo[0] = hi[0] = end.bin, before[0] = end.before, upto[0] = end.count;
    least = end.mass_before - off, most = end.mass + off;
  }
  if (p) {
    mark(2, up_to(ask.top_p * least - off, false)), mark(3, up_to(ask.top_p * most + off, false));
    __syncthreads();
    const Mark a = marked(2, end);
    end = marked(3, end);
    lo[1] = a.bin, before[1] = a.before, hi[1] = end.bin, upto[1] = end.count;
    least = fmin(least, a.mass_before - off), most = fmin(most, end.mass + off);
  }
  plan.runs.near = -1;
  m = m && lds.mark[4].bin <= end.bin;
  if (m) {
    const Mark a = lds.mark[4];
    end = marked(5, end);
    lo[2] = a.bin, before[2] = a.before, hi[2] = end.bin, upto[2] = end.count;
    least = fmin(least, a.mass_before - off), most = fmin(most, end.mass + off);
    plan.runs.near = end.bin;
  }
  const Mark last = all <= kList ? lds.mark[0] : k ? lds.mark[1] : end;  // (the weight of the first top_k is asked for)
  if (last.count <= kPrefix || all <= kList) {
    plan.runs.n = 1, plan.runs.tokens = last.count, plan.runs.run[0] = {0, last.bin, 0, last.count, 0, 0.0, 0, 0};
#pragma unroll
    for (int i = 1; i < Runs::kMost; ++i) plan.runs.run[i] = {kSteps, kSteps, 0, 0, 0, 0.0, 0, 0};
    plan.all = all, plan.weighed = last.count < all && !k && (p || !m);
    __syncthreads();
    return plan;
  }
  mark(6, up_to(ask.u * least - off, true)), mark(7, up_to(ask.u * most + off, true));
  __syncthreads();
  {
    const Mark a = marked(6, end), b = marked(7, end);
    lo[3] = a.bin, before[3] = a.before, hi[3] = b.bin, upto[3] = b.count;
  }
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
  for (int i = 1; i < Runs::kMost; ++i)
    if (lo[i] < kSteps) hi[i] = max(hi[i], hi[i - 1]), upto[i] = max(upto[i], upto[i - 1]);
#pragma unroll
  for (int i = Runs::kMost - 1; i; --i)
    if (lo[i] < kSteps && lo[i] <= hi[i - 1] + 1) {
      hi[i - 1] = hi[i], upto[i - 1] = upto[i];
#pragma unroll
      for (int j = i; j < Runs::kMost; ++j) {
        const bool more = j + 1 < Runs::kMost;
        lo[j] = more ? lo[(j + 1) % Runs::kMost] : kSteps, hi[j] = more ? hi[(j + 1) % Runs::kMost] : kSteps;
        before[j] = more ? before[(j + 1) % Runs::kMost] : 0, upto[j] = more ? upto[(j + 1) % Runs::kMost] : 0;
      }
    }
  plan.runs.n = 0, plan.runs.tokens = 0;
#pragma unroll
  for (int i = 0; i < Runs::kMost; ++i) {
    plan.runs.run[i] = {lo[i], hi[i], plan.runs.tokens, upto[i] - before[i], before[i], 0.0, 0, 0};
    plan.runs.tokens += upto[i] - before[i], plan.runs.n += lo[i] < kSteps;
  }
  plan.all = all, plan.weighed = true, plan.slow = plan.runs.tokens > kList;
  __syncthreads();
  return plan;
}

// Gathers the tokens of the plan's runs among `count` scores from `first` on.  RUNS: adds up the weights before each of so many runs too, and
// of all, in units of 2^-40: a thread's sums of them are exact, and so are those of all threads.  0: there is one run, from the first
// token on.
template <int RUNS, typename T> __device__ __forceinline__ void gather_runs(Lds& lds, const Row<T>& row, const Steps& steps, const Runs& runs, int first, int count) {
  constexpr int kWide = 16 / sizeof(T), kRuns = RUNS ? RUNS : 1;
  if (threadIdx.x == 0) lds.listed = 0;
  if (threadIdx.x <= kMostRuns) lds.weight[threadIdx.x] = 0;
  __syncthreads();
  const Weights weights{row.scale.top, row.scale.factor};
  float lo[kRuns], hi[kRuns];
  u64 before[kRuns], all = 0;
  uint32_t pieces = 0;
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    const bool there = i < runs.n;
    lo[i] = there ? Steps::first_of(runs.run[i].b0) : INFINITY, hi[i] = there ? Steps::last_of(runs.run[i].b1) : -INFINITY, before[i] = 0;
  }
  auto wanted = [&](float down) {
    bool in = false;
#pragma unroll
    for (int i = 0; i < kRuns; ++i) in |= down >= lo[i] && down <= hi[i];
    return in;
  };
  for_pieces(row.row, first, count, [&](const float (&x)[kWide], int column) {
    bool some = false;
#pragma unroll
    for (int j = 0; j < kWide; ++j) {
      const float down = steps.down(x[j]);
      some |= wanted(down);
      if constexpr (RUNS) {
        const u64 w = weights.of(x[j]);
        all += w;
#pragma unroll
        for (int i = 0; i < kRuns; ++i) before[i] += down < lo[i] ? w : Weights::none();
      }
    }
    ++pieces;
    if (some) {
#pragma unroll
      for (int j = 0; j < kWide; ++j)
        if (wanted(steps.down(x[j])) && x[j] > -INFINITY) {
          const uint32_t at = atomicAdd(&lds.listed, 1u);
          if (at < kList) lds.list[at] = row.code(x[j], column + j);
        }
    }
  });
  if constexpr (RUNS) {
    const u64 none = (u64)pieces * kWide * Weights::none();
    auto give = [&](u64 sum, u64* to) {
      sum = sum_of_lanes(sum - none);
      if ((threadIdx.x & 63) == 63) atomicAdd(to, sum);
    };
#pragma unroll
    for (int i = 0; i < kRuns; ++i) give(before[i], &lds.weight[i]);
    give(all, &lds.weight[kMostRuns]);
  }
  __syncthreads();
}

__device__ __forceinline__ float parameter(const float* p, int64_t r, float without) { return p ? p[r] : without; }

template <typename T> __global__ void __launch_bounds__(kThreads) sample_kernel(Args a) {
  __shared__ Lds lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t r = blockIdx.x;
  Row<T> row{static_cast<const T*>(a.logits) + r * a.stride, a.columns, a.log2_columns, {0.f, 0.0}};
  auto answer = [&](int token, float probability, uint32_t kept) {
    if (tid) return;
    a.token[r] = token;
    if (a.probability) a.probability[r] = probability;
    if (a.kept) a.kept[r] = (int32_t)kept;
  };
  const float temperature = parameter(a.temperature, r, 1.f), top_p = parameter(a.top_p, r, 1.f), min_p = parameter(a.min_p, r, 0.f), uniform = a.uniform[r];
  const int top_k = a.top_k ? a.top_k[r] : 0;
  const Ask ask{top_k > 0 && top_k < a.columns ? (uint32_t)top_k : 0u, top_p < 1.f ? fmax((double)top_p, 0.0) : 2.0,
                min_p > 0.f ? min_p >= 1.f ? 0.0 : -log2((double)min_p) : INFINITY, uniform > 0.f ? fmin((double)uniform, 1.0 - 0x1p-24) : 0.0};
  row.scale.factor = fmax(1.4426950408889634 / (double)temperature, 1e-300);  // (0 times infinity is NaN)
  auto give = [&](const Found& f) { answer(row.column(f.code), (float)f.share, f.kept); };

  if (!(temperature > 0.f) || a.columns <= kList) {
    // ---- the highest score, and few
    float high = -INFINITY, low = INFINITY;
    int at = 0;
    bool nan = false;
    for_each(row.row, 0, a.columns, [&](float x, int column) {
      nan |= x != x;
      low = x > -INFINITY ? fminf(low, x) : low;
      const bool more = x > high;
      high = more ? x : high, at = more ? column : at;
    });
    u64 best = high > -INFINITY ? row.code(high, at) : ~(u64)0;
    low = -low;
#pragma unroll
    for (int d = 32; d; d >>= 1) best = min(best, (u64)__shfl_xor((long long)best, d));
    over_lanes_max(low);
    if (lane == 0) lds.wave_best[wave] = best, lds.wave_low[wave] = low;
    nan = __syncthreads_or(nan);
    for (int w = 0; w < kWaves; ++w) best = min(best, lds.wave_best[w]), low = fmaxf(low, lds.wave_low[w]);
    if (nan) return answer(-1, NAN, 0);
    if (best == ~(u64)0) return answer(-1, 0.f, 0);
    if (!(temperature > 0.f)) return answer(row.column(best), 1.f, 1);
    row.scale.top = row.score(best);
    const uint32_t n = row.gather(lds, [&](float, int) { return true; });
    Runs runs;
    runs.n = 1, runs.run[0] = {0, kSteps, 0, n, 0, 0.0, 0, 0}, runs.tokens = n, runs.near = ask.far < INFINITY ? 0 : -1;
    runs.run[0].span(best, row.code(-low, row.columns - 1));
    row.sort(lds, runs);
    return give(row.solve(lds, ask, runs, n, lds.upto[n - 1]));
  }

  bool nan;
  const Steps steps = look(lds, row, row.scale.factor);
  row.scale.top = count_steps(lds, row, steps, 0, a.columns, nan);
  if (nan) return answer(-1, NAN, 0);
  if (row.scale.top == -INFINITY) return answer(-1, 0.f, 0);
  Plan plan = plan_of(lds, row.scale, steps, ask);
  if (!plan.slow) {
    const Runs& runs = plan.runs;
    if (!plan.weighed) gather_runs<0>(lds, row, steps, runs, 0, a.columns);
    else if (runs.n == 1) gather_runs<1>(lds, row, steps, runs, 0, a.columns);
    else if (runs.n == 2) gather_runs<2>(lds, row, steps, runs, 0, a.columns);
    else gather_runs<4>(lds, row, steps, runs, 0, a.columns);
#pragma unroll
    for (int i = 0; i < Runs::kMost; ++i) {
      Run& run = plan.runs.run[i];
      run.mass_before = plan.weighed ? (double)lds.weight[i] * 0x1p-40 : 0.0;
      if (i < runs.n) run.span(row.code(run.b0 ? steps.score(run.b0 - 1) : row.scale.top, 0), row.code(steps.score(run.b1), row.columns - 1));
    }
    row.sort(lds, runs);
    const Found f = row.solve(lds, ask, plan.runs, plan.all, plan.weighed ? (double)lds.weight[kMostRuns] * 0x1p-40 : lds.upto[plan.runs.tokens - 1]);
    if (f.sure && lds.listed == runs.tokens) return give(f);
  }

  // ---- the slow way
  Sums s{{0, 0}, 0, {0.0, 0.0}, 0.0};
  for (int first = 0; first < a.columns; first += kChunk) {
    __syncthreads();
    lds.sum[2 * tid] = lds.sum[2 * tid + 1] = 0;
    __syncthreads();
    for_each(row.row, first, min(kChunk, a.columns - first), [&](float x, int) {
      if (x == -INFINITY) return;
      const double d = row.scale.distance(x);
      const int bin = bin_of(d);
      atomicAdd(&lds.sum[bin], packed(d, bin));
    });
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j) s.c[j] += count_in(lds.sum[2 * tid + j]), s.m[j] += mass_in(lds.sum[2 * tid + j], 2 * tid + j);
  }
  s.scan(lds, 0, 0.0);
#pragma unroll
  for (int j = 0; j < 2; ++j) lds.count[2 * tid + j] = s.c[j], lds.mass[2 * tid + j] = s.m[j];
  __syncthreads();
  give(row.solve_slowly(lds, ask));
}

constexpr int64_t kWorkspace = 256;

}  // namespace

extern "C" {

int64_t rsr_sample_workspace(int64_t rows, int64_t columns) {
  if (rows < 0 || rows > 1 << 24) return set_error(RSR_ERR_INVALID_ARGUMENT, "rows must be in 0..2^24");
  if (columns < 1 || columns > 1 << 22) return set_error(RSR_ERR_INVALID_ARGUMENT, "columns must be in 1..2^22");
  return kWorkspace;
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
  if (!rsr_internal::aligned(logits, rsr_internal::size_of(dtype))) return set_error(RSR_ERR_INVALID_ARGUMENT, "logits must be aligned as their elements");
  if (!workspace || !rsr_internal::aligned(workspace, 256) || workspace_bytes < need)
    return set_error(RSR_ERR_INVALID_ARGUMENT, "the workspace is missing, too small or not 256-byte aligned");
  Args a{logits, temperature, top_p, min_p, uniform, top_k, token, probability, kept, stride, (int32_t)columns, 1};
  while ((int64_t)1 << a.log2_columns < columns) ++a.log2_columns;
  auto kern = dtype == RSR_F32 ? sample_kernel<float> : dtype == RSR_F16 ? sample_kernel<_Float16> : sample_kernel<__bf16>;
  hipLaunchKernelGGL(kern, dim3((unsigned)rows), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(RSR_ERR_HIP, std::string("rsr_sample: ") + hipGetErrorString(e));
  return RSR_OK;
}

}  // extern "C"
