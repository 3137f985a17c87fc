// Norms and rotation of heads, and the kept path of drafted trees (include/rsr_decode.h).  Sampling is in rsr_sample.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "../../include/rsr_decode.h"

#include "rsr_cache_check.h"

namespace {

using rsr_internal::set_error;

int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(RSR_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
  return RSR_OK;
}

// ---- norms and rotation ------------------------------------------------------------------------------------
// A lane has eight dimensions of a head: four from dimension `lo` on and four from `hi` on, of the rotated part's first and second half
// (or of the rest's), so that with either pairing both of a pair are its own.  As many lanes as the next power of two above
// head_dim / 8 make a head, and a wavefront turns from head to head of one token, whose angles it works out once.  Values are rounded once,
// where they are written; the norm's sums are held in 32 bits.
//
// Bound by memory: 16384 tokens of 25 heads of 128, float to bfloat16, take 62.2 us, 5.06 TB/s, what a large copy reaches.  What that took: the
// next heads are on their way while some are worked on (two, three and four of them at once take as long there, and 2048 tokens 9.8, 11.2 and 12.0 us
// instead of 8.5), and the norm's sum is one of 32 bits by moves between lanes (in 64 bits, at half the rate: 77 us).  Loads and stores past the caches were as
// fast, and the attention that reads the results would not find them there.
constexpr int kRotateThreads = 256;
constexpr int64_t kRotateTokens = UINT32_MAX / kRotateThreads * (kRotateThreads / 64);  // of a launch, which has fewer than 2^32 threads

typedef float f4 __attribute__((ext_vector_type(4)));

struct RotateArgs {
  const void *q, *k;
  void *q_out, *k_out;
  const double* frequency;
  const float *q_weight, *k_weight;
  const int32_t* position;
  int64_t q_stride, k_stride, q_out_stride, k_out_stride, tokens;
  int32_t heads, kv_heads, dim, rotated;
  int32_t log2_lanes;  // lanes of a head
  int32_t share;       // wavefronts of a token
  float eps;
  float share_of_one;  // 1 / dim
  bool norm, pairs;
};

template <typename T> struct Four {
  typedef T type __attribute__((ext_vector_type(4)));
  static __device__ inline type load(const T* p) { return *reinterpret_cast<const type*>(p); }
  static __device__ inline f4 wide(type x) { return f4{(float)x[0], (float)x[1], (float)x[2], (float)x[3]}; }
  static __device__ inline void store(T* p, f4 x) { *reinterpret_cast<type*>(p) = type{(T)x[0], (T)x[1], (T)x[2], (T)x[3]}; }
};

// (the norm's weights may lie anywhere)
__device__ inline f4 load4_anywhere(const float* p) { return f4{p[0], p[1], p[2], p[3]}; }

// position * frequency in whole turns, less the whole ones: the product in two doubles, and the quotient by 2 pi as a product with two.
__device__ inline float turn_of(int position, double frequency) {
  constexpr double kTurn = 0.15915494309189535, kTurnRest = -9.8393358101206405e-18;  // 1 / (2 pi)
  const double each = frequency * kTurn, each_rest = fma(frequency, kTurn, -each) + frequency * kTurnRest;
  const double p = position, turns = p * each, rest = fma(p, each, -turns) + p * each_rest;
  return (float)((turns - rint(turns)) + rest);
}

// The sum over the lanes of a head, in each of them.
template <int CTRL> __device__ inline float and_moved(float x) {
  return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
__device__ inline float over_head(float x, int log2_lanes) {
  if (log2_lanes >= 1) x = and_moved<0xb1>(x);   // the neighbour
  if (log2_lanes >= 2) x = and_moved<0x4e>(x);   // the other two of four
  if (log2_lanes >= 3) x = and_moved<0x141>(x);  // of eight, backwards
  if (log2_lanes >= 4) x = and_moved<0x140>(x);  // of sixteen, backwards
  return log2_lanes >= 5 ? x + __shfl_xor(x, 16) : x;
}

template <typename IN, typename OUT> __global__ void __launch_bounds__(kRotateThreads) rotate_kernel(RotateArgs a) {
  const int lane = threadIdx.x & 63, lanes = 1 << a.log2_lanes, in_head = lane & (lanes - 1), part = lane >> a.log2_lanes;
  const int64_t wave = (int64_t)blockIdx.x * (kRotateThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), token = wave / a.share;
  if (token >= a.tokens) return;
  const int all = a.heads + a.kv_heads, each = 64 >> a.log2_lanes, step = a.share * each;
  const bool there = in_head < a.dim / 8, turns = in_head < a.rotated / 8;
  const int rest = in_head - a.rotated / 8;
  const int lo = there ? turns ? 4 * in_head : a.rotated + 4 * rest : 0, hi = there ? turns ? a.rotated / 2 + lo : (a.dim - a.rotated) / 2 + lo : 0;
  const IN* const q = static_cast<const IN*>(a.q) + token * a.q_stride;
  const IN* const k = static_cast<const IN*>(a.k) + token * a.k_stride;
  OUT* const q_out = static_cast<OUT*>(a.q_out) + token * a.q_out_stride;
  OUT* const k_out = static_cast<OUT*>(a.k_out) + token * a.k_out_stride;
  const int first = (int)(wave - token * a.share) * each;
  // The heads that are next are on their way while some are worked on, the first ones while the angles are.
  typedef typename Four<IN>::type Raw;
  Raw next[2];
  auto load = [&](int head0) {
    const int head = min(head0 + part, all - 1);  // (the last one again instead of none)
    const IN* const from = head < a.heads ? q + head * a.dim : k + (head - a.heads) * a.dim;
    next[0] = Four<IN>::load(from + lo), next[1] = Four<IN>::load(from + hi);
  };
  load(first);
  f4 q_weight[2]{{1, 1, 1, 1}, {1, 1, 1, 1}}, k_weight[2]{{1, 1, 1, 1}, {1, 1, 1, 1}};
  if (a.norm && a.q_weight) q_weight[0] = load4_anywhere(a.q_weight + lo), q_weight[1] = load4_anywhere(a.q_weight + hi);
  if (a.norm && a.k_weight) k_weight[0] = load4_anywhere(a.k_weight + lo), k_weight[1] = load4_anywhere(a.k_weight + hi);
  f4 sin{0, 0, 0, 0}, cos{1, 1, 1, 1};
  if (there && turns) {
    const int position = a.position[token];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int pair = !a.pairs ? lo + j : j < 2 ? lo / 2 + j : hi / 2 + j - 2;
      float s, c;
      sincospif(2.f * turn_of(position, a.frequency[pair]), &s, &c);
      sin[j] = s, cos[j] = c;
    }
  }
  for (int head0 = first; head0 < all; head0 += step) {
    f4 x[2] = {Four<IN>::wide(next[0]), Four<IN>::wide(next[1])};
    if (head0 + step < all) load(head0 + step);  // (in place too: another turn's heads are others)
    const int head = head0 + part;
    const bool is_there = there && head < all;
    if (a.norm) {
      if (!there) x[0] = x[1] = f4{0, 0, 0, 0};
      f4 s = x[0] * x[0];
      s = x[1] * x[1] + s;
      const float mean = over_head((s[0] + s[1]) + (s[2] + s[3]), a.log2_lanes) * a.share_of_one;
      const float m = mean + a.eps, near = __builtin_amdgcn_rsqf(m), by = fmaf(0.5f * near, fmaf(-m * near, near, 1.f), near);
      const bool odd = is_there && !(mean < 1e30f && m > 1e-30f);
      f4 w[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) w[j] = head < a.heads ? q_weight[j] : k_weight[j];
      if (!__ballot(odd)) {
        x[0] = x[0] * by * w[0], x[1] = x[1] * by * w[1];
      } else {
        // (seldom: squares beyond the range of float, or what does not count in it; of these heads alone)
        double sum = 0;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) sum = fma((double)x[j][e], (double)x[j][e], sum);
        for (int d = lanes / 2; d; d >>= 1) sum += __shfl_xor(sum, d);
        const double exact = 1.0 / sqrt(sum / a.dim + (double)a.eps);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) x[j][e] = (odd ? (float)((double)x[j][e] * exact) : x[j][e] * by) * w[j][e];
      }
    }
    if (!is_there) continue;
    if (turns) {
      const f4 u = x[0], v = x[1];
      if (!a.pairs) {
        x[0] = u * cos - v * sin, x[1] = u * sin + v * cos;
      } else {
        x[0] = f4{u[0] * cos[0] - u[1] * sin[0], u[0] * sin[0] + u[1] * cos[0], u[2] * cos[1] - u[3] * sin[1], u[2] * sin[1] + u[3] * cos[1]};
        x[1] = f4{v[0] * cos[2] - v[1] * sin[2], v[0] * sin[2] + v[1] * cos[2], v[2] * cos[3] - v[3] * sin[3], v[2] * sin[3] + v[3] * cos[3]};
      }
    }
    OUT* const to = head < a.heads ? q_out + head * a.dim : k_out + (head - a.heads) * a.dim;
    Four<OUT>::store(to + lo, x[0]), Four<OUT>::store(to + hi, x[1]);
  }
}

template <typename IN> void (*rotate_to(int out_dtype))(RotateArgs) {
  return out_dtype == RSR_F32 ? rotate_kernel<IN, float> : out_dtype == RSR_F16 ? rotate_kernel<IN, _Float16> : rotate_kernel<IN, __bf16>;
}

bool is_dtype(int dtype) { return dtype == RSR_F32 || dtype == RSR_F16 || dtype == RSR_BF16; }

// ---- the kept path of drafted trees ------------------------------------------------------------------------
// One wavefront walks a tree, a lane per token: from the token that it is at, the first lane that hangs on it and has what was chosen
// behind it is next.  A path's tokens come in the order of their numbers, so the path is a mask.  Bound by latency: in a graph one request takes
// 2.8 us, 64 take 6.9 (one launch; with a launch for counts and one for paths one request took 5.7), 512 trees of up to 64 tokens 7.0, 4096 of up
// to 16 8.4.
constexpr int kKeepThreads = 1024, kKeepWaves = kKeepThreads / 64;

struct KeepArgs {
  const int32_t *drafted, *chosen, *parent, *start;
  int32_t *rows, *found, *add, *first;
  int32_t requests, tokens;
};

struct Path {
  int64_t first;     // row of the request's first token
  uint64_t on;       // tokens on the path
  int32_t chosen;    // behind the lane's token
};

__device__ inline Path path_of(const KeepArgs& a, int r, int lane) {
  Path p{a.start[r], 0, -1};
  const int64_t end = min((int64_t)a.start[r + 1], (int64_t)a.tokens);
  if (p.first < 0 || p.first >= end) return p;
  const int n = (int)min(end - p.first, (int64_t)64);
  const int64_t row = p.first + min(lane, n - 1);
  p.chosen = a.chosen[row];
  const int drafted = a.drafted[row], up = a.parent ? a.parent[row] : lane - 1;
  const bool hangs = lane < n && up >= 0 && up < lane;
  p.on = 1;
  for (int at = 0;;) {
    const int next = __builtin_amdgcn_readlane(p.chosen, at);
    const uint64_t found = __ballot(hangs && up == at && drafted == next);
    if (next < 0 || !found) break;
    at = __builtin_ctzll(found);
    p.on |= 1ull << at;
  }
  return p;
}

// What the requests add.
__global__ void __launch_bounds__(kKeepThreads) count_kernel(KeepArgs a) {
  const int r = blockIdx.x * kKeepWaves + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= a.requests) return;
  const Path p = path_of(a, r, lane);
  if (lane == 0) a.add[r] = __popcll(p.on);
}

__device__ inline void write_path(const KeepArgs& a, int r, int lane, const Path& p, int64_t at) {
  if (lane == 0) a.first[r] = (int32_t)min(at, (int64_t)a.tokens);
  at += __popcll(p.on & ((1ull << lane) - 1));
  if (p.on >> lane & 1 && at < a.tokens) a.rows[at] = (int32_t)(p.first + lane), a.found[at] = p.chosen;
}

// The paths, one behind the other, with what is behind the last.  ALONE: of at most kAlone requests, which one workgroup walks, some for
// each wavefront.  Else `add` is known, a workgroup has `each` requests, adds up what all before them add, and walks its own again (a
// place to keep the paths in between would be as long as all trees).
constexpr int kRounds = 4, kAlone = kRounds * kKeepWaves;

template <bool ALONE> __global__ void __launch_bounds__(kKeepThreads) paths_kernel(KeepArgs a, int each) {
  __shared__ int64_t before_sum[kKeepWaves], all_sum[kKeepWaves];
  __shared__ int32_t adds[kAlone];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int64_t before = 0, all = 0;
  if constexpr (ALONE) {
    Path p[kRounds];
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      const int r = i * kKeepWaves + wave;
      if (r >= a.requests) continue;
      p[i] = path_of(a, r, lane);
      if (lane == 0) a.add[r] = adds[r] = __popcll(p[i].on);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      const int r = i * kKeepWaves + wave;
      if (r >= a.requests) continue;
      int64_t at = lane < r ? adds[lane] : 0;
      for (int d = 32; d; d >>= 1) at += __shfl_xor(at, d);
      write_path(a, r, lane, p[i], at);
    }
    all = lane < a.requests ? adds[lane] : 0;
    for (int d = 32; d; d >>= 1) all += __shfl_xor(all, d);
  } else {
    const int r0 = blockIdx.x * each, r1 = min(r0 + each, a.requests);
    for (int r = tid; r < a.requests; r += kKeepThreads) {
      const int add = a.add[r];
      all += add, before += r < r0 ? add : 0;
    }
    for (int d = 32; d; d >>= 1) before += __shfl_xor(before, d), all += __shfl_xor(all, d);
    if (lane == 0) before_sum[wave] = before, all_sum[wave] = all;
    __syncthreads();
    before = all = 0;
    for (int w = 0; w < kKeepWaves; ++w) before += before_sum[w], all += all_sum[w];
    for (int r = r0 + wave; r < r1; r += kKeepWaves) {
      const Path p = path_of(a, r, lane);
      int64_t at = 0;
      for (int s = r0 + lane; s < r; s += 64) at += a.add[s];
      for (int d = 32; d; d >>= 1) at += __shfl_xor(at, d);
      write_path(a, r, lane, p, before + at);
    }
  }
  if (blockIdx.x == 0 && tid == 0) a.first[a.requests] = (int32_t)min(all, (int64_t)a.tokens);
  for (int64_t i = all + (int64_t)blockIdx.x * kKeepThreads + tid; i < a.tokens; i += (int64_t)gridDim.x * kKeepThreads) a.rows[i] = a.found[i] = -1;
}
static_assert(kAlone <= 64);

}  // namespace

extern "C" {

int rsr_head_rotate(const rsr_rotary_t* rotary, const void* q, int64_t q_stride, int heads, const void* k, int64_t k_stride, int kv_heads, int dtype,
                    const int32_t* position, int64_t tokens, void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride, int out_dtype,
                    void* stream) {
  const char* fault = nullptr;
  if (!rotary) fault = "null pointer";
  else if (rotary->head_dim < 8 || rotary->head_dim > 256 || rotary->head_dim % 8) fault = "head_dim must be a multiple of 8 in 8..256";
  else if (rotary->rotated < 0 || rotary->rotated > rotary->head_dim || rotary->rotated % 8) fault = "rotated must be a multiple of 8 in 0..head_dim";
  else if ((rotary->norm | 1) != 1 || (rotary->pairs | 1) != 1) fault = "norm and pairs must be 0 or 1";
  else if (rotary->norm && !(rotary->eps >= 0.f && std::isfinite(rotary->eps))) fault = "eps must be finite and not negative";
  else if (!is_dtype(dtype) || !is_dtype(out_dtype)) fault = "dtype and out_dtype must be RSR_F32, RSR_F16 or RSR_BF16";
  else if (heads < 0 || heads > 65535 || kv_heads < 0 || kv_heads > 65535 || heads + kv_heads == 0) fault = "heads and kv_heads must be in 0..65535, not both 0";
  else if (tokens < 0 || tokens > INT32_MAX) fault = "tokens must be in 0..2^31-1";
  if (fault) return set_error(RSR_ERR_INVALID_ARGUMENT, fault);
  if (tokens == 0) return RSR_OK;
  const int64_t width = (int64_t)heads * rotary->head_dim, kv_width = (int64_t)kv_heads * rotary->head_dim;
  if (heads) fault = rsr_internal::fault_of_rows(q, q_stride, width, dtype);
  if (heads && !fault) fault = rsr_internal::fault_of_rows(q_out, q_out_stride, width, out_dtype);
  if (kv_heads && !fault) fault = rsr_internal::fault_of_rows(k, k_stride, kv_width, dtype);
  if (kv_heads && !fault) fault = rsr_internal::fault_of_rows(k_out, k_out_stride, kv_width, out_dtype);
  if (!fault && rotary->rotated && (!position || !rotary->frequency)) fault = "null pointer";
  if (!fault && ((heads && q_out == q && (q_out_stride != q_stride || out_dtype != dtype)) || (kv_heads && k_out == k && (k_out_stride != k_stride || out_dtype != dtype))))
    fault = "an output that is an input must have its stride and type";
  if (!fault && ((heads && kv_heads && q_out == k_out) || (heads && kv_heads && (q_out == k || k_out == q)))) fault = "an output must not be another input or output";
  if (fault) return set_error(RSR_ERR_INVALID_ARGUMENT, fault);
  RotateArgs a{q, k, q_out, k_out, rotary->frequency, rotary->q_weight, rotary->k_weight, position, q_stride, k_stride, q_out_stride, k_out_stride, tokens,
               heads, kv_heads, rotary->head_dim, rotary->rotated, 0, 1, rotary->eps, 1.f / (float)rotary->head_dim, rotary->norm != 0, rotary->pairs != 0};
  while (8 << a.log2_lanes < a.dim) ++a.log2_lanes;
  // A wavefront for each token, or as many as its heads keep busy where that leaves the chip idle: 25 heads of 1 .. 512 tokens take 2.9 .. 4.7 us
  // (kernels alone, in a graph) instead of 5.6 .. 7.2 with one, 2048 tokens 8.4 instead of 9.0; with up to 16384 wavefronts these take 11.7.
  const int each = 64 >> a.log2_lanes;
  const int64_t most = (heads + kv_heads + each - 1) / each;
  a.share = (int32_t)std::min(most, std::max<int64_t>(1, 4096 / tokens));
  auto kern = dtype == RSR_F32 ? rotate_to<float>(out_dtype) : dtype == RSR_F16 ? rotate_to<_Float16>(out_dtype) : rotate_to<__bf16>(out_dtype);
  auto behind = [](const void* p, int64_t stride, int type) { return static_cast<const char*>(p) + kRotateTokens * stride * rsr_internal::size_of(type); };
  for (;;) {
    a.tokens = std::min(tokens, kRotateTokens);
    const int64_t groups = (a.tokens * a.share + kRotateThreads / 64 - 1) / (kRotateThreads / 64);
    hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3(kRotateThreads), 0, static_cast<hipStream_t>(stream), a);
    if ((tokens -= a.tokens) == 0) return launched("rsr_head_rotate");
    if (heads) a.q = behind(a.q, q_stride, dtype), a.q_out = const_cast<char*>(behind(a.q_out, q_out_stride, out_dtype));
    if (kv_heads) a.k = behind(a.k, k_stride, dtype), a.k_out = const_cast<char*>(behind(a.k_out, k_out_stride, out_dtype));
    if (position) a.position += kRotateTokens;
  }
}

int rsr_tree_keep(const int32_t* drafted, const int32_t* chosen, const int32_t* parent, const int32_t* start, int requests, int tokens, int32_t* rows,
                  int32_t* found, int32_t* add, int32_t* first, void* stream) {
  if (requests < 0 || requests > 65535) return set_error(RSR_ERR_INVALID_ARGUMENT, "requests must be in 0..65535");
  if (tokens < 0) return set_error(RSR_ERR_INVALID_ARGUMENT, "tokens must not be negative");
  if (!first || (requests && (!start || !add)) || (tokens && (!rows || !found || (requests && (!drafted || !chosen)))))
    return set_error(RSR_ERR_INVALID_ARGUMENT, "null pointer");
  const void* const outputs[] = {rows, found, add, first};
  const void* const inputs[] = {drafted, chosen, parent, start};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 4; ++j)
      if (outputs[i] && (outputs[i] == inputs[j] || (j < i && outputs[i] == outputs[j]))) return set_error(RSR_ERR_INVALID_ARGUMENT, "an output must not be an input or another output");
  }
  const KeepArgs a{drafted, chosen, parent, start, rows, found, add, first, requests, tokens};
  if (requests <= kAlone) {
    hipLaunchKernelGGL(paths_kernel<true>, dim3(1), dim3(kKeepThreads), 0, static_cast<hipStream_t>(stream), a, 0);
    return launched("rsr_tree_keep");
  }
  const int each = std::max(kKeepWaves, (requests + 255) / 256);
  hipLaunchKernelGGL(count_kernel, dim3((requests + kKeepWaves - 1) / kKeepWaves), dim3(kKeepThreads), 0, static_cast<hipStream_t>(stream), a);
  hipLaunchKernelGGL(paths_kernel<false>, dim3((requests + each - 1) / each), dim3(kKeepThreads), 0, static_cast<hipStream_t>(stream), a, each);
  return launched("rsr_tree_keep");
}

}  // extern "C"
