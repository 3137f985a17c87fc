// The cache's own operators (include/rsr_cache.h): slots and block tables from lengths, the write of kept tokens, and
// the masks of drafted trees.  The attention over the cache is in rsr_attend.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <string>

#include "rsr_cache_check.h"

namespace {

using rsr_internal::set_error;

int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(RSR_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
  return RSR_OK;
}

// ---- slots and block tables --------------------------------------------------------------------------------
// With before_r = ceil(held_r / page) and after_r = ceil((held_r + add_r) / page), both at most the length of a table's
// row, request r takes the free pages number F_r .. F_r + after_r - before_r - 1 from the end of the list, and its
// slots are the entries S_r .. S_r + add_r - 1 of the map; F and S are running sums over the requests before it.
// Every workgroup adds up all requests by itself, a batch at a time (a batch is read from L2 and costs two barriers, less
// than a second launch would), and then fills its share of the entries: an entry finds its request by halving the batch's
// running sums.  No workgroup waits for another: a slot on a new page takes it from the list, not from the table.
// Bound by latency: 6.0 us for 256 requests of up to 8 tokens, 7.2 for 64 prompts with 600 000 slots (2.4 MB; 10.5
// with 8 slots per lane instead of 2).
constexpr int kSlotThreads = 256;
constexpr int kPerThread = 4;
constexpr int kBatch = kSlotThreads * kPerThread;

struct SlotsArgs {
  const int32_t *held, *add, *free_pages, *free_count;
  int32_t *table, *free_left, *slots, *start, *now;
  int64_t max_free, max_slots;
  int32_t requests, max_pages, log2_page;
};

// Index of the first of n ascending sums that is above x (there is one).
__device__ inline int above(const int64_t* sums, int n, int64_t x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] > x) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

__global__ void __launch_bounds__(kSlotThreads) slots_kernel(SlotsArgs a) {
  __shared__ int64_t slot_end[kBatch], page_end[kBatch];  // running sums, own entry included, over all requests so far
  __shared__ int32_t first_token[kBatch], first_page[kBatch];
  __shared__ int64_t wave_slots[kSlotThreads / 64], wave_pages[kSlotThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t every = (int64_t)gridDim.x * kSlotThreads, mine = (int64_t)blockIdx.x * kSlotThreads + tid;
  const int64_t size = int64_t(1) << a.log2_page, width = a.max_pages, most_start = min(a.max_slots, (int64_t)INT32_MAX);
  const int64_t count = min((int64_t)max(a.free_count[0], 0), a.max_free);
  int64_t slots0 = 0, pages0 = 0;
  for (int r0 = 0; r0 < a.requests; r0 += kBatch) {
    const int n = min(kBatch, a.requests - r0);
    int64_t added[kPerThread], held[kPerThread], before[kPerThread], need[kPerThread], s = 0, p = 0;
#pragma unroll
    for (int j = 0; j < kPerThread; ++j) {
      const int r = tid * kPerThread + j;
      held[j] = r < n ? max(a.held[r0 + r], 0) : 0;
      added[j] = r < n ? max(a.add[r0 + r], 0) : 0;
      before[j] = min((held[j] + size - 1) >> a.log2_page, width);
      need[j] = min((held[j] + added[j] + size - 1) >> a.log2_page, width) - before[j];
      s += added[j];
      p += need[j];
    }
    int64_t s_in = s, p_in = p;  // sums over this thread and those before it
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t us = __shfl_up(s_in, d), up = __shfl_up(p_in, d);
      if (lane >= d) s_in += us, p_in += up;
    }
    if (lane == 63) wave_slots[wave] = s_in, wave_pages[wave] = p_in;
    __syncthreads();
    int64_t s_at = slots0 + s_in - s, p_at = pages0 + p_in - p;
    for (int w = 0; w < wave; ++w) s_at += wave_slots[w], p_at += wave_pages[w];
    const bool writes = (r0 / kBatch) % (int)gridDim.x == (int)blockIdx.x;
#pragma unroll
    for (int j = 0; j < kPerThread; ++j) {
      const int r = tid * kPerThread + j;
      if (writes && r < n) {
        a.start[r0 + r] = (int32_t)min(s_at, most_start);
        const int64_t granted = min(max(count - p_at, int64_t(0)), need[j]);
        a.now[r0 + r] = (int32_t)min(max(held[j], min(held[j] + added[j], (before[j] + granted) << a.log2_page)), (int64_t)INT32_MAX);
      }
      s_at += added[j];
      p_at += need[j];
      if (r < n) {
        slot_end[r] = s_at, page_end[r] = p_at;
        first_token[r] = (int32_t)held[j], first_page[r] = (int32_t)before[j];
      }
    }
    __syncthreads();
    const int64_t slots1 = slot_end[n - 1], pages1 = page_end[n - 1], most = min(slots1, a.max_slots);
    for (int64_t i = mine + (slots0 > mine ? (slots0 - mine + every - 1) / every * every : 0); i < most; i += every) {
      const int r = above(slot_end, n, i);
      const int64_t at = first_token[r] + i - (r ? slot_end[r - 1] : slots0), page_at = at >> a.log2_page;
      int64_t page = -1;
      if (page_at < first_page[r]) {
        page = a.table[(int64_t)(r0 + r) * width + page_at];
      } else if (page_at < width) {
        const int64_t taken = (r ? page_end[r - 1] : pages0) + page_at - first_page[r];
        if (taken < count) page = a.free_pages[count - 1 - taken];
      }
      const int64_t slot = (page << a.log2_page) + (at & (size - 1));
      a.slots[i] = page < 0 || slot > INT32_MAX ? -1 : (int32_t)slot;
    }
    for (int64_t i = mine + (pages0 > mine ? (pages0 - mine + every - 1) / every * every : 0); i < pages1; i += every) {
      const int r = above(page_end, n, i);
      a.table[(int64_t)(r0 + r) * width + first_page[r] + i - (r ? page_end[r - 1] : pages0)] = i < count ? a.free_pages[count - 1 - i] : -1;
    }
    __syncthreads();  // the next batch overwrites the sums
    slots0 = slots1, pages0 = pages1;
  }
  for (int64_t i = mine + (slots0 > mine ? (slots0 - mine + every - 1) / every * every : 0); i < a.max_slots; i += every) a.slots[i] = -1;
  if (mine == 0) {
    a.start[a.requests] = (int32_t)min(slots0, most_start);
    a.free_left[0] = (int32_t)max(count - pages0, (int64_t)INT32_MIN);
  }
}

// ---- the write of kept tokens ------------------------------------------------------------------------------
// One lane moves eight values of a key or a value: 16 bytes into the cache.  The eights of a workgroup's tokens are numbered
// through, keys and values one behind the other, so that a row of any width fills the lanes.  Bound by the bytes: 84 MB of 16384
// tokens with 5 heads of 128 in 13 to 15 us (part of it from the last-level cache), 3.1 us for the kept path of a tree.
constexpr int kAppendThreads = 256;

struct AppendArgs {
  const void *k, *v;
  const int32_t *rows, *slots;
  uint16_t *cache_k, *cache_v;
  int64_t stride, nrows, page_stride, head_stride, token_stride, count;
  int32_t log2_page, pages, eights, eights_per_head;  // eights: of a row (keys only)
  int32_t tokens_per_group;
};

template <typename T> __device__ inline uint32_t pair_of(float lo, float hi);
template <> __device__ inline uint32_t pair_of<_Float16>(float lo, float hi) {
  typedef _Float16 h2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, h2{(_Float16)lo, (_Float16)hi});
}
template <> __device__ inline uint32_t pair_of<__bf16>(float lo, float hi) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, b2{(__bf16)lo, (__bf16)hi});
}

// CT: the cache's type; FLOAT: the activations are float, otherwise of the cache's type
template <typename CT, bool FLOAT>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(AppendArgs a) {
  const int64_t token0 = (int64_t)blockIdx.x * a.tokens_per_group;
  const int tokens = (int)min((int64_t)a.tokens_per_group, a.count - token0);
  const uint32_t per_token = 2u * a.eights, items = per_token * tokens;
  for (uint32_t i = threadIdx.x; i < items; i += kAppendThreads) {
    const uint32_t t = i / per_token, e = i - t * per_token;
    const int64_t slot = a.slots[token0 + t], row = a.rows ? (int64_t)a.rows[token0 + t] : token0 + t;
    const int64_t page = slot >> a.log2_page;
    if (slot < 0 || page >= a.pages || row < 0 || row >= a.nrows) continue;
    const bool value = e >= (uint32_t)a.eights;
    const uint32_t at = value ? e - a.eights : e, head = at / a.eights_per_head, d8 = at - head * a.eights_per_head;
    const int64_t from = row * a.stride + (int64_t)at * 8;
    const int64_t to = page * a.page_stride + head * a.head_stride + (slot & ((int64_t(1) << a.log2_page) - 1)) * a.token_stride + d8 * 8;
    uint4 x;
    if (FLOAT) {
      const float4* f = reinterpret_cast<const float4*>(static_cast<const float*>(value ? a.v : a.k) + from);
      const float4 lo = f[0], hi = f[1];
      x = {pair_of<CT>(lo.x, lo.y), pair_of<CT>(lo.z, lo.w), pair_of<CT>(hi.x, hi.y), pair_of<CT>(hi.z, hi.w)};
    } else {
      x = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(value ? a.v : a.k) + from);
    }
    *reinterpret_cast<uint4*>((value ? a.cache_v : a.cache_k) + to) = x;
  }
}

// ---- masks of drafted trees --------------------------------------------------------------------------------
// One wavefront per tree, a lane per token.  mask_i = bit i | mask of the parent: every round a lane takes over what the
// last token that it has reached has reached, so that the links double and six rounds reach through 64 tokens.  Bound by the
// latency of a launch: 1.4 us for one tree, 2.8 for 512.
constexpr int kMaskThreads = 256;

__global__ void __launch_bounds__(kMaskThreads) masks_kernel(const int32_t* __restrict__ parent, const int32_t* __restrict__ start, int requests,
                                                             int tokens, uint64_t* __restrict__ mask, int32_t* __restrict__ depth) {
  const int r = blockIdx.x * (kMaskThreads / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= requests) return;
  const int64_t first = start[r], end = min(start[r + 1], tokens);
  if (first < 0) return;
  const int64_t n = end - first;
  const int up = lane < n ? parent[first + lane] : -1;
  int to = up >= 0 && up < lane ? up : lane;
  uint64_t seen = 1ull << lane;
  for (;;) {
    const int next = __shfl(to, to);  // (a token that hangs on none points to itself)
    if (!__ballot(next != to)) break;
    seen |= __shfl(seen, to);
    to = next;
  }
  seen |= __shfl(seen, to);
  if (lane < n) {
    mask[first + lane] = seen;
    depth[first + lane] = __popcll(seen) - 1;
  }
  for (int64_t i = 64 + lane; i < n; i += 64) mask[first + i] = 0, depth[first + i] = -1;
}

}  // namespace

extern "C" {

int rsr_cache_slots_bounded(const int32_t* held, const int32_t* add, int requests, int32_t* table, int max_pages, int page_size,
                            const int32_t* free_pages, int64_t max_free, const int32_t* free_count, int32_t* free_left, int32_t* slots, int64_t max_slots,
                            int32_t* start, int32_t* now, void* stream) {
  if (requests < 0 || requests > 65535) return set_error(RSR_ERR_INVALID_ARGUMENT, "requests must be in 0..65535");
  if (max_slots < 0 || max_free < 0 || max_pages < 1)
    return set_error(RSR_ERR_INVALID_ARGUMENT, "max_slots and max_free must be at least 0 and max_pages at least 1");
  if (!rsr_internal::is_page_size(page_size)) return set_error(RSR_ERR_INVALID_ARGUMENT, "page_size must be a power of two in 8..1024");
  if (!free_count || !free_left || !start || (max_slots && !slots) || (requests && (!held || !add || !table || (max_free && !free_pages) || !now)))
    return set_error(RSR_ERR_INVALID_ARGUMENT, "null pointer");
  if (free_left == free_count || (requests && (now == held || now == add || start == held || start == add)))
    return set_error(RSR_ERR_INVALID_ARGUMENT, "an output must not be an input");
  const SlotsArgs a{held,     add,       free_pages, free_count, table,     free_left, slots, start, now,
                    max_free, max_slots, requests,   max_pages,  rsr_internal::log2_of(page_size)};
  // two slots per lane: each is a search and two reads one after the other, and adding up the requests anew costs less than a third
  const int64_t groups = (max_slots + 2 * kSlotThreads - 1) / (2 * kSlotThreads);
  hipLaunchKernelGGL(slots_kernel, dim3((unsigned)(groups < 1 ? 1 : groups > 1024 ? 1024 : groups)), dim3(kSlotThreads), 0, static_cast<hipStream_t>(stream), a);
  return launched("rsr_cache_slots");
}

int rsr_cache_slots(const int32_t* held, const int32_t* add, int requests, int32_t* table, int max_pages, int page_size, const int32_t* free_pages,
                    const int32_t* free_count, int32_t* free_left, int32_t* slots, int64_t max_slots, int32_t* start, int32_t* now, void* stream) {
  return rsr_cache_slots_bounded(held, add, requests, table, max_pages, page_size, free_pages, INT32_MAX, free_count, free_left, slots, max_slots, start, now,
                                 stream);
}

int rsr_cache_append(const rsr_cache_t* cache, const void* k, const void* v, int64_t stride, int64_t nrows, int dtype, const int32_t* rows,
                     const int32_t* slots, int64_t count, void* stream) {
  if (const char* fault = rsr_internal::fault_of(cache)) return set_error(RSR_ERR_INVALID_ARGUMENT, fault);
  if (dtype != RSR_F32 && dtype != cache->dtype) return set_error(RSR_ERR_INVALID_ARGUMENT, "dtype must be RSR_F32 or the cache's");
  if (count < 0 || nrows < 0) return set_error(RSR_ERR_INVALID_ARGUMENT, "count and nrows must not be negative");
  if (count == 0 || nrows == 0) return RSR_OK;
  const int64_t width = (int64_t)cache->kv_heads * cache->head_dim;
  const char* fault = rsr_internal::fault_of_rows(k, stride, width, dtype);
  if (!fault) fault = rsr_internal::fault_of_rows(v, stride, width, dtype);
  if (!fault && !slots) fault = "null pointer";
  if (fault) return set_error(RSR_ERR_INVALID_ARGUMENT, fault);
  AppendArgs a{k, v, rows, slots, static_cast<uint16_t*>(cache->k), static_cast<uint16_t*>(cache->v), stride, nrows, cache->page_stride, cache->head_stride,
               cache->token_stride, count, rsr_internal::log2_of(cache->page_size), cache->pages, (int32_t)(width / 8), cache->head_dim / 8, 1};
  // as many tokens per workgroup as give its lanes an eight or two each, or, if that made more lanes than a launch may have, as many as
  // do not (their eights are numbered in 32 bits)
  const int64_t most_groups = UINT32_MAX / kAppendThreads, few = 2 * a.eights >= 2 * kAppendThreads ? 1 : 2 * kAppendThreads / (2 * a.eights);
  const int64_t tokens = std::max(few, (count - 1) / most_groups + 1);
  if (tokens > UINT32_MAX / (2 * a.eights)) return set_error(RSR_ERR_INVALID_ARGUMENT, "count is too large");
  a.tokens_per_group = (int32_t)tokens;
  const int64_t groups = (count - 1) / tokens + 1;
  auto kern = cache->dtype == RSR_F16 ? (dtype == RSR_F32 ? append_kernel<_Float16, true> : append_kernel<_Float16, false>)
                                      : (dtype == RSR_F32 ? append_kernel<__bf16, true> : append_kernel<__bf16, false>);
  hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3(kAppendThreads), 0, static_cast<hipStream_t>(stream), a);
  return launched("rsr_cache_append");
}

int rsr_tree_masks(const int32_t* parent, const int32_t* start, int requests, int tokens, uint64_t* mask, int32_t* depth, void* stream) {
  if (requests < 0 || requests > 65535) return set_error(RSR_ERR_INVALID_ARGUMENT, "requests must be in 0..65535");
  if (tokens < 0) return set_error(RSR_ERR_INVALID_ARGUMENT, "tokens must not be negative");
  if (requests == 0 || tokens == 0) return RSR_OK;
  if (!parent || !start || !mask || !depth) return set_error(RSR_ERR_INVALID_ARGUMENT, "null pointer");
  const int groups = (requests + kMaskThreads / 64 - 1) / (kMaskThreads / 64);
  hipLaunchKernelGGL(masks_kernel, dim3(groups), dim3(kMaskThreads), 0, static_cast<hipStream_t>(stream), parent, start, requests, tokens, mask, depth);
  return launched("rsr_tree_masks");
}

}  // extern "C"
