// Attention of a step's new tokens over the paged cache and over each other (include/rsr_cache.h).
//
// The definition, one workgroup per new token and query head: a running maximum m and sum l of the weights, positions 256
// at a time, a lane per position for the scores and a lane per dimension for the values.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <string>

#include "rsr_cache_check.h"

namespace {

using rsr_internal::set_error;

constexpr int kThreads = 256;

struct Args {
  const void *q, *k, *v;
  void* out;
  const uint16_t *cache_k, *cache_v;
  const int32_t *table, *held, *start;
  const uint64_t* mask;
  int64_t q_stride, kv_stride, out_stride, page_stride, head_stride, token_stride;
  int32_t requests, tokens, max_new, max_pages, log2_page, pages, heads, kv_heads, dim;
  float scale;
};

template <typename T> __device__ inline float widened(uint16_t x) { return (float)__builtin_bit_cast(T, x); }

// element i of activations, rounded to the cache's type if ROUND
template <typename CT, bool FLOAT, bool ROUND> __device__ inline float activation(const void* p, int64_t i) {
  if (!FLOAT) return widened<CT>(static_cast<const uint16_t*>(p)[i]);
  const float x = static_cast<const float*>(p)[i];
  return ROUND ? (float)(CT)x : x;
}

template <typename CT, bool FLOAT>
__global__ void __launch_bounds__(kThreads) attend_kernel(Args a) {
  __shared__ float query[256], weight[kThreads], reduced[kThreads];
  const int r = blockIdx.z, i = blockIdx.y, head = blockIdx.x, tid = threadIdx.x;
  const int64_t first = a.start[r], fresh = min((int64_t)a.max_new, min((int64_t)a.start[r + 1], (int64_t)a.tokens) - first);
  if (first < 0 || i >= fresh) return;
  const int64_t size = int64_t(1) << a.log2_page, held = min((int64_t)max(a.held[r], 0), a.max_pages * size), row = first + i;
  const int kv = head / (a.heads / a.kv_heads);
  const uint64_t mask = a.mask ? a.mask[row] : 0;
  if (tid < a.dim) query[tid] = activation<CT, FLOAT, false>(a.q, row * a.q_stride + head * a.dim + tid);
  float m = -INFINITY, l = 0.f, acc = 0.f;
  const int64_t total = held + fresh;
  for (int64_t p0 = 0; p0 < total; p0 += kThreads) {
    __syncthreads();
    const int64_t p = p0 + tid;
    float s = -INFINITY;
    const uint16_t* cached = nullptr;
    if (p < held) {
      const int page = a.table[(int64_t)r * a.max_pages + (p >> a.log2_page)];
      if (page >= 0 && page < a.pages) cached = a.cache_k + page * a.page_stride + kv * a.head_stride + (p & (size - 1)) * a.token_stride;
    }
    const bool seen = p < held ? cached != nullptr : p < total && (a.mask ? (mask >> (p - held)) & 1 : p - held <= i);
    if (seen) {
      float dot = 0.f;
      for (int d = 0; d < a.dim; ++d)
        dot += query[d] * (cached ? widened<CT>(cached[d]) : activation<CT, FLOAT, true>(a.k, (first + p - held) * a.kv_stride + kv * a.dim + d));
      s = dot * a.scale;
    }
    reduced[tid] = s;
    __syncthreads();
    for (int d = kThreads / 2; d > 0; d >>= 1) {
      if (tid < d) reduced[tid] = fmaxf(reduced[tid], reduced[tid + d]);
      __syncthreads();
    }
    const float top = fmaxf(m, reduced[0]), base = top == -INFINITY ? 0.f : top;
    const float back = expf(m - base);
    const float w = seen ? expf(s - base) : 0.f;
    __syncthreads();
    weight[tid] = seen ? w : -1.f;  // (a weight is never negative: what is not seen is not touched)
    reduced[tid] = w;
    __syncthreads();
    for (int d = kThreads / 2; d > 0; d >>= 1) {
      if (tid < d) reduced[tid] += reduced[tid + d];
      __syncthreads();
    }
    l = l * back + reduced[0];
    m = top;
    if (tid < a.dim) {
      float part = 0.f;  // of these positions: short sums of their own, so that a long cache is no long chain of additions
      for (int j = 0; j < kThreads && p0 + j < total; ++j) {
        const float wj = weight[j];
        if (wj == -1.f) continue;
        const int64_t pj = p0 + j;
        float x;
        if (pj < held) {
          const int page = a.table[(int64_t)r * a.max_pages + (pj >> a.log2_page)];
          x = widened<CT>(a.cache_v[page * a.page_stride + kv * a.head_stride + (pj & (size - 1)) * a.token_stride + tid]);
        } else {
          x = activation<CT, FLOAT, true>(a.v, (first + pj - held) * a.kv_stride + kv * a.dim + tid);
        }
        part += wj * x;
      }
      acc = acc * back + part;
    }
  }
  if (tid < a.dim) {
    const float o = l == 0.f ? 0.f : acc / l;
    const int64_t to = row * a.out_stride + head * a.dim + tid;
    if (FLOAT) static_cast<float*>(a.out)[to] = o;
    else static_cast<CT*>(a.out)[to] = (CT)o;
  }
}

const char* fault_of(const rsr_cache_t* cache, const rsr_step_t* step, int heads) {
  if (const char* fault = rsr_internal::fault_of(cache)) return fault;
  if (!step) return "null pointer";
  if (step->requests < 0 || step->requests > 65535) return "requests must be in 0..65535";
  if (step->tokens < 0) return "tokens must not be negative";
  if (step->max_new < 1 || step->max_new > 65535 || (step->mask && step->max_new > 64)) return "max_new must be in 1..65535, and at most 64 with a mask";
  if (step->max_pages < 1) return "max_pages must be at least 1";
  if (heads < 1 || heads % cache->kv_heads || heads / cache->kv_heads > 64) return "heads must be a multiple of kv_heads, at most 64 times as many";
  if (step->requests && (!step->table || !step->held || !step->start)) return "null pointer";
  return nullptr;
}

}  // namespace

extern "C" {

int64_t rsr_tree_attention_workspace(const rsr_cache_t* cache, const rsr_step_t* step, int heads) {
  if (const char* fault = fault_of(cache, step, heads)) return set_error(RSR_ERR_INVALID_ARGUMENT, fault);
  return 256;
}

int rsr_tree_attention(const rsr_cache_t* cache, const rsr_step_t* step, const void* q, int64_t q_stride, const void* k, const void* v,
                       int64_t kv_stride, void* out, int64_t out_stride, int dtype, int heads, float scale, void* workspace, int64_t workspace_bytes,
                       void* stream) {
  const char* fault = fault_of(cache, step, heads);
  if (!fault && dtype != RSR_F32 && dtype != cache->dtype) fault = "dtype must be RSR_F32 or the cache's";
  if (!fault && !std::isfinite(scale)) fault = "scale must be finite";
  if (fault) return set_error(RSR_ERR_INVALID_ARGUMENT, fault);
  if (step->requests == 0 || step->tokens == 0) return RSR_OK;
  const int64_t width = (int64_t)heads * cache->head_dim, kv_width = (int64_t)cache->kv_heads * cache->head_dim;
  fault = rsr_internal::fault_of_rows(q, q_stride, width, dtype);
  if (!fault) fault = rsr_internal::fault_of_rows(k, kv_stride, kv_width, dtype);
  if (!fault) fault = rsr_internal::fault_of_rows(v, kv_stride, kv_width, dtype);
  if (!fault) fault = rsr_internal::fault_of_rows(out, out_stride, width, dtype);
  if (!fault && (!workspace || !rsr_internal::aligned(workspace, 256) || workspace_bytes < rsr_tree_attention_workspace(cache, step, heads)))
    fault = "the workspace is missing, too small or not 256-byte aligned";
  if (fault) return set_error(RSR_ERR_INVALID_ARGUMENT, fault);
  const Args a{q, k, v, out, static_cast<const uint16_t*>(cache->k), static_cast<const uint16_t*>(cache->v), step->table, step->held, step->start, step->mask,
               q_stride, kv_stride, out_stride, cache->page_stride, cache->head_stride, cache->token_stride, step->requests, step->tokens, step->max_new,
               step->max_pages, rsr_internal::log2_of(cache->page_size), cache->pages, heads, cache->kv_heads, cache->head_dim, scale};
  auto kern = cache->dtype == RSR_F16 ? (dtype == RSR_F32 ? attend_kernel<_Float16, true> : attend_kernel<_Float16, false>)
                                      : (dtype == RSR_F32 ? attend_kernel<__bf16, true> : attend_kernel<__bf16, false>);
  hipLaunchKernelGGL(kern, dim3(heads, step->max_new, step->requests), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(RSR_ERR_HIP, std::string("rsr_tree_attention: ") + hipGetErrorString(e));
  return RSR_OK;
}

}  // extern "C"
