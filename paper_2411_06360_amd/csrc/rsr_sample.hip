// A token for every row of scores (include/rsr_decode.h).
//
// With the scores in order, the highest first, everything that is asked for is a place in one running sum: of tokens (top-k), of
// weights (top-p, the token itself), or a score (min-p).  No row is sorted for that.  A histogram of the scores, 2048 bins of 1/32 of an
// octave of weight below the highest, with count and weight of each bin, says in which bin a place is; the tokens of the bins up to
// there (or, if these are too many, of that bin; or, if these are too many too, of a part of it that a finer histogram
// finds) are gathered in LDS and sorted, and there the place is found.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "../../include/rsr_decode.h"

#include "rsr_cache_check.h"

namespace {

using rsr_internal::set_error;

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 2048;         // two for each thread
constexpr int kPerOctave = 32;      // bins
constexpr int kList = 2048;         // tokens that are sorted at once
constexpr int kFixed = 40;          // bits behind the point of summed weights

typedef uint32_t u4 __attribute__((ext_vector_type(4)));

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

struct Lds {
  uint32_t count[kBins];                                  // then: up to and with the bin
  union { unsigned long long sum[kBins]; double mass[kBins]; };  // the same of weights
  uint32_t part_count[kBins];                             // of a finer histogram
  union { unsigned long long part_sum[kBins]; double part_mass[kBins]; };
  unsigned long long list[kList];                         // tokens, sorted
  double upto[kList];                                     // weight up to and with each
  double wave_mass[kWaves];
  uint32_t wave_count[kWaves];
  uint32_t listed;
};

// ---- scores -----------------------------------------------------------------------------------------------
// Ascending for descending scores; both zeros alike.
__device__ inline uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u >> 31 ? u : ~u & 0x7fffffffu;
}
__device__ inline float score_of(uint32_t key) { return __uint_as_float(key >> 31 ? key : ~key & 0x7fffffffu); }

// f(score, column) for all scores of a row, by all threads of the workgroup.  Reads are 16 bytes wide wherever the row begins; what
// sticks out at the ends is read by itself.
template <typename T, typename F> __device__ inline void for_each(const T* row, int columns, F f) {
  constexpr int kWide = 16 / sizeof(T), kAtOnce = 4;
  const int lead = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
  const int64_t pieces = ((int64_t)columns + lead + kWide - 1) / kWide;
  const T* const from = row - lead;
  for (int64_t p0 = threadIdx.x; p0 < pieces; p0 += kThreads * kAtOnce) {
    T x[kAtOnce][kWide];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int64_t p = p0 + (int64_t)i * kThreads, at = p * kWide - lead;
      if (at >= 0 && at + kWide <= columns) {
        const u4 v = *reinterpret_cast<const u4*>(from + p * kWide);
        __builtin_memcpy(x[i], &v, 16);
      } else {
#pragma unroll
        for (int j = 0; j < kWide; ++j) x[i][j] = at + j >= 0 && at + j < columns ? row[at + j] : (T)-INFINITY;
      }
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int64_t at = (p0 + (int64_t)i * kThreads) * kWide - lead;
#pragma unroll
      for (int j = 0; j < kWide; ++j) f((float)x[i][j], (int)(at + j));
    }
  }
}

// ---- weights ----------------------------------------------------------------------------------------------
// A score's distance below the highest, in octaves of its weight: the weight is 2^-distance, 1 exactly for the highest.
struct Scale {
  float top;
  double factor;
  __device__ double distance(float x) const { return x == top ? 0.0 : ((double)top - (double)x) * factor; }
  __device__ double weight(float x) const { return exp2(-distance(x)); }
};
__device__ inline int bin_of(double distance) { return (int)fmin(distance * kPerOctave, (double)(kBins - 1)); }
// The weight within its bin as a whole number: 2^(bin / 32 - distance) in units of 2^-40.
__device__ inline unsigned long long in_bin(double distance, int bin) { return (unsigned long long)(exp2((double)bin / kPerOctave - distance) * (double)(1ull << kFixed) + 0.5); }
__device__ inline double of_bin(unsigned long long sum, int bin) { return (double)sum * exp2(-(double)bin / kPerOctave - kFixed); }

// ---- sums over a workgroup ---------------------------------------------------------------------------------
// Running sums of two bins per thread, in their order.
__device__ inline void scan(Lds& lds, uint32_t (&c)[2], double (&m)[2], uint32_t c0, double m0) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  c[1] += c[0], m[1] += m[0];
  uint32_t cs = c[1];
  double ms = m[1];
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t cu = __shfl_up(cs, d);
    const double mu = __shfl_up(ms, d);
    if (lane >= d) cs += cu, ms += mu;
  }
  __syncthreads();
  if (lane == 63) lds.wave_count[wave] = cs, lds.wave_mass[wave] = ms;
  __syncthreads();
  uint32_t cb = c0;
  double mb = m0;
  for (int w = 0; w < wave; ++w) cb += lds.wave_count[w], mb += lds.wave_mass[w];
  const uint32_t cl = __shfl_up(cs, 1);
  const double ml = __shfl_up(ms, 1);
  if (lane) cb += cl, mb += ml;
  c[0] += cb, c[1] += cb, m[0] += mb, m[1] += mb;
}

// ---- places -----------------------------------------------------------------------------------------------
// The place where a running sum reaches what is asked for.
struct Place {
  bool of_count, strict;  // a sum of tokens (at least `count`), or of weights: at least `mass`, or more than that
  uint32_t count;
  double mass;
  __device__ bool reached(uint32_t c, double m) const { return of_count ? c >= count : strict ? m > mass : m >= mass; }
};

// The first entry of n running sums that reaches the place; the last one if none does.
__device__ inline int first_at(const Place& p, const uint32_t* count, const double* mass, int n) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (p.reached(count ? count[mid] : 0, mass[mid])) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

// A run of tokens in their order, sorted in LDS.
struct Run {
  uint32_t before;     // tokens before it
  double mass_before;  // and their weight
  uint32_t count;
};

template <typename T> struct Row {
  const T* row;
  int columns, log2_columns;
  Scale scale;

  __device__ unsigned long long code(float x, int column) const { return (unsigned long long)key_of(x) << log2_columns | (uint32_t)column; }
  __device__ float score(unsigned long long code) const { return score_of((uint32_t)(code >> log2_columns)); }

  // Tokens of the bins b0 .. b1 whose codes are within c0 .. c1, sorted, with their running weights.
  __device__ Run gather(Lds& lds, int b0, int b1, unsigned long long c0, unsigned long long c1, uint32_t before, double mass_before) const {
    const int tid = threadIdx.x;
    __syncthreads();
    if (tid == 0) lds.listed = 0;
    __syncthreads();
    for_each(row, columns, [&](float x, int column) {
      if (x == -INFINITY) return;
      const int bin = bin_of(scale.distance(x));
      const unsigned long long c = code(x, column);
      if (bin < b0 || bin > b1 || c < c0 || c > c1) return;
      const uint32_t at = atomicAdd(&lds.listed, 1u);
      if (at < kList) lds.list[at] = c;
    });
    __syncthreads();
    const uint32_t n = min(lds.listed, (uint32_t)kList);
    uint32_t size = 2;
    while (size < n) size *= 2;
    for (uint32_t i = n + tid; i < size; i += kThreads) lds.list[i] = ~0ull;
    __syncthreads();
    for (uint32_t k = 2; k <= size; k *= 2)
      for (uint32_t j = k / 2; j; j /= 2) {
        for (uint32_t i = tid; i < size / 2; i += kThreads) {
          const uint32_t lo = 2 * i - (i & (j - 1)), hi = lo + j;
          const unsigned long long x = lds.list[lo], y = lds.list[hi];
          if ((x > y) == ((lo & k) == 0)) lds.list[lo] = y, lds.list[hi] = x;
        }
        __syncthreads();
      }
    uint32_t c[2];
    double m[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t i = 2 * tid + j;
      c[j] = 0, m[j] = i < n ? scale.weight(score(lds.list[i])) : 0.0;
    }
    scan(lds, c, m, 0, mass_before);
    lds.upto[2 * tid] = m[0], lds.upto[2 * tid + 1] = m[1];
    __syncthreads();
    return {before, mass_before, n};
  }

  // The run of tokens in which the place is.
  __device__ Run seek(Lds& lds, const Place& p) const {
    const int tid = threadIdx.x;
    int b = first_at(p, lds.count, lds.mass, kBins);
    while (b && lds.count[b] == lds.count[b - 1]) --b;  // (what rounding puts behind the last token is the last token's)
    if (lds.count[b] <= kList) return gather(lds, 0, b, 0, ~0ull, 0, 0.0);
    uint32_t before = b ? lds.count[b - 1] : 0, count = lds.count[b] - before;
    double mass_before = b ? lds.mass[b - 1] : 0.0;
    unsigned long long lo = 0, hi = (1ull << (32 + log2_columns)) - 1;
    while (count > kList) {
      const int shift = max(0, 64 - __clzll((long long)(hi - lo)) - 11);
      __syncthreads();
      for (int i = tid; i < kBins; i += kThreads) lds.part_count[i] = 0, lds.part_sum[i] = 0;
      __syncthreads();
      for_each(row, columns, [&](float x, int column) {
        if (x == -INFINITY) return;
        const double d = scale.distance(x);
        const unsigned long long c = code(x, column);
        if (bin_of(d) != b || c < lo || c > hi) return;
        const int part = (int)((c - lo) >> shift);
        atomicAdd(&lds.part_count[part], 1u);
        atomicAdd(&lds.part_sum[part], in_bin(d, b));
      });
      __syncthreads();
      uint32_t c[2];
      double m[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) c[j] = lds.part_count[2 * tid + j], m[j] = of_bin(lds.part_sum[2 * tid + j], b);
      scan(lds, c, m, before, mass_before);
#pragma unroll
      for (int j = 0; j < 2; ++j) lds.part_count[2 * tid + j] = c[j], lds.part_mass[2 * tid + j] = m[j];
      __syncthreads();
      int part = first_at(p, lds.part_count, lds.part_mass, kBins);
      while (part && lds.part_count[part] == lds.part_count[part - 1]) --part;
      while (lds.part_count[part] == before) ++part;  // (or before the first one)
      if (part) before = lds.part_count[part - 1], mass_before = lds.part_mass[part - 1];
      count = lds.part_count[part] - before;
      lo += (unsigned long long)part << shift;
      hi = min(hi, lo + (1ull << shift) - 1);
    }
    return gather(lds, b, b, lo, hi, before, mass_before);
  }

  __device__ bool holds(const Lds& lds, const Run& run, const Place& p) const {
    return run.count && !p.reached(run.before, run.mass_before) && p.reached(run.before + run.count, lds.upto[run.count - 1]);
  }
  // Which token of the run is at the place.
  __device__ uint32_t at(const Lds& lds, const Run& run, const Place& p) const {
    if (p.of_count) return min(max(p.count, run.before + 1) - run.before, run.count) - 1;
    return first_at(p, nullptr, lds.upto, run.count);
  }

  // How many scores are at most that far below the highest, and their weight.
  __device__ void tally(Lds& lds, double far, uint32_t& count, double& mass) const {
    __syncthreads();
    if (threadIdx.x == 0) lds.part_count[0] = 0, lds.part_sum[0] = 0;
    __syncthreads();
    uint32_t n = 0;
    unsigned long long sum = 0;
    for_each(row, columns, [&](float x, int) {
      if (x == -INFINITY) return;
      const double d = scale.distance(x);
      if (d <= far) ++n, sum += in_bin(d, 0);
    });
    atomicAdd(&lds.part_count[0], n), atomicAdd(&lds.part_sum[0], sum);
    __syncthreads();
    count = lds.part_count[0], mass = of_bin(lds.part_sum[0], 0);
  }
};

__device__ inline float parameter(const float* p, int64_t r, float without) { return p ? p[r] : without; }

template <typename T> __global__ void __launch_bounds__(kThreads) sample_kernel(Args a) {
  __shared__ Lds lds;
  __shared__ unsigned long long best[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t r = blockIdx.x;
  Row<T> row{static_cast<const T*>(a.logits) + r * a.stride, a.columns, a.log2_columns, {0.f, 0.0}};
  auto answer = [&](int token, float probability, uint32_t kept) {
    if (tid) return;
    a.token[r] = token;
    if (a.probability) a.probability[r] = probability;
    if (a.kept) a.kept[r] = (int32_t)kept;
  };

  // ---- the highest score
  unsigned long long first = ~0ull;
  bool nan = false;
  for_each(row.row, a.columns, [&](float x, int column) {
    nan |= x != x;
    if (x > -INFINITY) first = min(first, row.code(x, column));
  });
#pragma unroll
  for (int d = 32; d; d >>= 1) first = min(first, (unsigned long long)__shfl_xor((long long)first, d));
  if (lane == 0) best[wave] = first;
  nan = __syncthreads_or(nan);
  for (int w = 0; w < kWaves; ++w) first = min(first, best[w]);
  if (nan) return answer(-1, NAN, 0);
  if (first == ~0ull) return answer(-1, 0.f, 0);
  const float temperature = parameter(a.temperature, r, 1.f);
  const int token0 = (int)(first & ((1ull << a.log2_columns) - 1));
  if (!(temperature > 0.f)) return answer(token0, 1.f, 1);
  row.scale = {row.score(first), fmax(1.4426950408889634 / (double)temperature, 1e-300)};  // (0 times infinity is NaN)

  // ---- the histogram
  for (int i = tid; i < kBins; i += kThreads) lds.count[i] = 0, lds.sum[i] = 0;
  __syncthreads();
  for_each(row.row, a.columns, [&](float x, int) {
    if (x == -INFINITY) return;
    const double d = row.scale.distance(x);
    const int bin = bin_of(d);
    atomicAdd(&lds.count[bin], 1u);
    atomicAdd(&lds.sum[bin], in_bin(d, bin));
  });
  __syncthreads();
  uint32_t c[2];
  double m[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) c[j] = lds.count[2 * tid + j], m[j] = of_bin(lds.sum[2 * tid + j], 2 * tid + j);
  scan(lds, c, m, 0, 0.0);
#pragma unroll
  for (int j = 0; j < 2; ++j) lds.count[2 * tid + j] = c[j], lds.mass[2 * tid + j] = m[j];
  __syncthreads();

  // ---- how many are kept, and their weight
  uint32_t kept = lds.count[kBins - 1];
  double mass = lds.mass[kBins - 1];
  Run run{0, 0.0, 0};
  auto find = [&](const Place& p) {
    if (!row.holds(lds, run, p)) run = row.seek(lds, p);
    return row.at(lds, run, p);
  };
  const int top_k = a.top_k ? a.top_k[r] : 0;
  if (top_k > 0 && (uint32_t)top_k < kept) {
    const uint32_t i = find({true, false, (uint32_t)top_k, 0.0});
    kept = top_k, mass = lds.upto[i];
  }
  const float top_p = parameter(a.top_p, r, 1.f);
  if (top_p < 1.f) {
    const uint32_t i = find({false, false, 0, fmax((double)top_p, 0.0) * mass}), n = run.before + i + 1;
    if (n < kept) kept = n, mass = lds.upto[i];
  }
  const float min_p = parameter(a.min_p, r, 0.f);
  if (min_p > 0.f) {
    const double far = min_p >= 1.f ? 0.0 : -log2((double)min_p);
    const int b = bin_of(far);
    if ((b ? lds.count[b - 1] : 0) < kept) {
      uint32_t n;
      double within;
      row.tally(lds, far, n, within);
      if (n < kept) kept = n, mass = within;
    }
  }

  // ---- the token
  const float uniform = a.uniform[r];
  const double u = uniform > 0.f ? fmin((double)uniform, 1.0 - 0x1p-24) : 0.0;
  uint32_t i = find({false, true, 0, u * mass});
  i = min(i, kept > run.before ? kept - 1 - run.before : 0u);
  const float x = row.score(lds.list[i]);
  answer((int)(lds.list[i] & ((1ull << a.log2_columns) - 1)), (float)(row.scale.weight(x) / mass), kept);
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
