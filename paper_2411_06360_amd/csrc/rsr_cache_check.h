// Shared by the units behind include/rsr_cache.h: checks of the descriptors, and conversions.
#ifndef RSR_CACHE_CHECK_H_
#define RSR_CACHE_CHECK_H_

#include <cstdint>

#include "../../include/rsr_cache.h"

#include "rsr_internal.h"

namespace rsr_internal {

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline bool is_page_size(int64_t n) { return n >= 8 && n <= 1024 && (n & (n - 1)) == 0; }
inline int log2_of(int n) { return __builtin_ctz((unsigned)n); }
inline int size_of(int dtype) { return dtype == RSR_F32 ? 4 : 2; }

// What is wrong with a cache, or null.
inline const char* fault_of(const rsr_cache_t* c) {
  if (!c || !c->k || !c->v) return "null pointer";
  if (c->dtype != RSR_F16 && c->dtype != RSR_BF16) return "the cache's dtype must be RSR_F16 or RSR_BF16";
  if (!is_page_size(c->page_size)) return "page_size must be a power of two in 8..1024";
  if (c->pages < 1 || (int64_t)c->pages * c->page_size >= (int64_t(1) << 31)) return "pages * page_size must be in 1..2^31-1";
  if (c->kv_heads < 1 || c->kv_heads > 1024) return "kv_heads must be in 1..1024";
  if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8) return "head_dim must be a multiple of 8 in 8..256";
  if ((c->page_stride | c->head_stride | c->token_stride) & 7) return "the cache's strides must be multiples of 8";
  if (c->page_stride < 0 || c->head_stride < 0 || c->token_stride < 0) return "the cache's strides must not be negative";
  if (c->page_stride >> 31 || c->token_stride >> 24) return "the cache's page_stride must be below 2^31, its token_stride below 2^24";
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return "the cache must be 16-byte aligned";
  return nullptr;
}

// What is wrong with the rows of activations at p, or null.
inline const char* fault_of_rows(const void* p, int64_t stride, int64_t width, int dtype) {
  if (!p) return "null pointer";
  if (stride < width) return "a stride is shorter than a row";
  if (!aligned(p, 16) || stride * size_of(dtype) % 16) return "rows must be 16-byte aligned";
  return nullptr;
}

}  // namespace rsr_internal
#endif  // RSR_CACHE_CHECK_H_
