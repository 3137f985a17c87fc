// Attention of a step's new tokens over the paged cache and over each other (include/rsr_cache.h).
//
// The scores of 16 query rows (a row: one new token, one query head) and 32 positions are S^T = K Q^T on the matrix cores, the
// result is O^T += V^T P^T with P = 2^(S - m), and a running maximum m and sum l per row (one pass over the cache).
// Transposed, because the positions of a score tile then lie along a lane's registers: what S^T leaves in a lane, eight
// consecutive positions of one row, is the operand that V^T P^T wants there.  Keys and values go from the cache straight into
// registers (a wavefront reads whole rows of 16 or 32 tokens, no two wavefronts read the same), values change their two halves
// of dwords with v_perm_b32; LDS serves to join the four wavefronts of a workgroup at the end.
//
// Position order.  Lane (n, g) = (lane & 15, lane >> 4) holds of S^T the rows 4g .. 4g+3 of two tiles of 16 keys.  With key
// 8 (x >> 2) + (x & 3) in row x of the first tile and that plus 4 in the second, these are the positions 8g .. 8g+7.
//
// Work split.  The positions of a request (tiles of 32: first the cached ones, then the new ones) are cut into as many pieces
// as keep the chip busy; a workgroup takes a piece for the rows of one key head, its wavefronts a quarter of the piece each.
// The pieces of a row meet in the workspace, where the workgroup that comes last joins them in their order.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "rsr_cache_check.h"

namespace {

using rsr_internal::set_error;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kTile = 32;        // positions of a tile
constexpr int kLeastTiles = 4;   // of a piece: one for each wavefront
constexpr float kBias = 7.f;     // weights are 2^(s - m + 7): as float16 they keep their bits down to 2^-21 of the largest
constexpr float kSlack = 8.f;    // m follows the maximum when it is left behind by more: weights stay below 2^15

typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));

struct Args {
  const void *q, *k, *v;
  void* out;
  const uint16_t *cache_k, *cache_v;
  const int32_t *table, *held, *start;
  const uint64_t* mask;
  uint32_t* counters;
  float* partial;
  int64_t q_stride, kv_stride, out_stride, page_stride, head_stride, token_stride;
  int32_t requests, tokens, max_new, max_pages, log2_page, pages, kv_heads, dim, group, target;
  float scale;
};

// ---- the cache's types on the matrix cores -----------------------------------------------------------------
template <typename CT> struct Half;
template <> struct Half<_Float16> {
  typedef _Float16 v8 __attribute__((ext_vector_type(8)));
  typedef _Float16 v2 __attribute__((ext_vector_type(2)));
  static constexpr int kTerms = 2;  // of a float: 22 bits
  static __device__ f4 mfma(u4 a, u4 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
};
template <> struct Half<__bf16> {
  typedef __bf16 v8 __attribute__((ext_vector_type(8)));
  typedef __bf16 v2 __attribute__((ext_vector_type(2)));
  static constexpr int kTerms = 3;  // of a float: all 24 bits
  static __device__ f4 mfma(u4 a, u4 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
};

// Eight floats as the sum of TERMS operands, each the rounding of what the ones before leave.
template <typename CT, int TERMS> __device__ inline void split(const float (&x)[8], u4 (&t)[TERMS]) {
  float rest[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) rest[j] = x[j];
#pragma unroll
  for (int k = 0; k < TERMS; ++k)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const typename Half<CT>::v2 h{(CT)rest[2 * j], (CT)rest[2 * j + 1]};
      t[k][j] = __builtin_bit_cast(uint32_t, h);
      if (k + 1 < TERMS) rest[2 * j] -= (float)h[0], rest[2 * j + 1] -= (float)h[1];
    }
}

// The largest / the sum over the four lanes n, n + 16, n + 32, n + 48.
__device__ inline float over_groups_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float over_groups_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// ---- which piece of work ------------------------------------------------------------------------------------
struct Request {
  int64_t first;  // row of its first new token
  int32_t fresh;  // new tokens
  int32_t held;   // cached tokens
};

__device__ inline Request request_of(const Args& a, int r) {
  const int64_t first = a.start[r], end = min((int64_t)a.start[r + 1], (int64_t)a.tokens);
  const int64_t fresh = first < 0 ? 0 : max(min(end - first, (int64_t)a.max_new), (int64_t)0);
  const int64_t held = min((int64_t)max(a.held[r], 0), (int64_t)a.max_pages << a.log2_page);
  return {first, (int32_t)fresh, (int32_t)min(held, (int64_t)INT32_MAX - 1024)};
}

__device__ inline int tiles_of(int n) { return (n + kTile - 1) / kTile; }

struct Counts {
  int64_t units;           // pieces
  int32_t slots, groups;   // pieces of rows that are cut, and such sets of rows
};

// Pieces of a request when a piece is `most` tiles at most.
__device__ inline Counts counts_of(const Request& q, int rows_per_unit, int group, int kv_heads, int64_t most, int* blocks, int* pieces) {
  *blocks = (int)(((int64_t)q.fresh * group + rows_per_unit - 1) / rows_per_unit);
  const int64_t tiles = tiles_of(q.held) + tiles_of(q.fresh);
  *pieces = (int)((tiles + most - 1) / most);
  const int64_t sets = (int64_t)*blocks * kv_heads;
  if (*pieces < 2) return {sets * *pieces, 0, 0};
  return {sets * *pieces, (int32_t)(sets * *pieces), (int32_t)sets};
}

template <int DP> constexpr int stride_of_partial() { return DP + 4; }

template <typename CT, bool FLOAT, int DP, int MT>
__global__ void __launch_bounds__(kThreads) attend_kernel(Args a) {
  constexpr int kTerms = FLOAT ? Half<CT>::kTerms : 1;
  constexpr int kRows = 16 * MT;                   // rows of a unit
  constexpr int kSteps = DP / 32;                  // of a score's sum
  constexpr int kEach = DP / 16 < 8 ? DP / 16 : 8; // neighbouring dimensions of a lane's piece of a value
  constexpr int kParts = DP / (16 * kEach);        // such pieces
  constexpr int kLine = DP + 4;                    // floats between rows in LDS

  __shared__ int64_t unit_end[kThreads];
  __shared__ int32_t slot_end[kThreads], group_end[kThreads];
  __shared__ int64_t sums[kWaves];
  __shared__ int32_t more[kWaves][2];
  __shared__ float row_m[kWaves][kRows], row_l[kWaves][kRows];
  __shared__ __align__(16) float joined[kWaves][16][kLine];
  __shared__ uint32_t arrived;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;

  // -- every workgroup counts the pieces of all requests, a run of requests per thread
  const int run = (a.requests + kThreads - 1) / kThreads, run0 = min(tid * run, a.requests), run1 = min(run0 + run, a.requests);
  int64_t work = 0;
  for (int r = run0; r < run1; ++r) {
    const Request q = request_of(a, r);
    work += (((int64_t)q.fresh * a.group + kRows - 1) / kRows) * a.kv_heads * (tiles_of(q.held) + tiles_of(q.fresh));
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) work += __shfl_xor(work, d);
  if (lane == 0) sums[wave] = work;
  __syncthreads();
  work = sums[0] + sums[1] + sums[2] + sums[3];
  const int64_t most = max((work + a.target - 1) / a.target, (int64_t)kLeastTiles);
  Counts mine{0, 0, 0};
  for (int r = run0; r < run1; ++r) {
    int blocks, pieces;
    const Counts c = counts_of(request_of(a, r), kRows, a.group, a.kv_heads, most, &blocks, &pieces);
    mine.units += c.units, mine.slots += c.slots, mine.groups += c.groups;
  }
  const Counts own = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t u = __shfl_up(mine.units, d);
    const int s = __shfl_up(mine.slots, d), o = __shfl_up(mine.groups, d);
    if (lane >= d) mine.units += u, mine.slots += s, mine.groups += o;
  }
  __syncthreads();
  if (lane == 63) sums[wave] = mine.units, more[wave][0] = mine.slots, more[wave][1] = mine.groups;
  __syncthreads();
  for (int w = 0; w < wave; ++w) mine.units += sums[w], mine.slots += more[w][0], mine.groups += more[w][1];
  unit_end[tid] = mine.units, slot_end[tid] = mine.slots - own.slots, group_end[tid] = mine.groups - own.groups;
  __syncthreads();
  const int64_t units = unit_end[kThreads - 1];

  // consecutive pieces (the same cached tokens for other rows) go to workgroups of one XCD (blockIdx % 8)
  const int grid = gridDim.x, eighth = grid / 8;
  const int64_t first_unit = grid % 8 ? blockIdx.x : (int64_t)(blockIdx.x % 8) * eighth + blockIdx.x / 8;

  for (int64_t unit = first_unit; unit < units; unit += grid) {
    // -- which request, key head, piece and rows
    int lo = 0, hi = kThreads - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (unit_end[mid] > unit) hi = mid;
      else lo = mid + 1;
    }
    int64_t at = unit - (lo ? unit_end[lo - 1] : 0);
    int r = lo * run, blocks, pieces, slot = slot_end[lo], set = group_end[lo];
    Request q;
    for (;; ++r) {
      q = request_of(a, r);
      const Counts c = counts_of(q, kRows, a.group, a.kv_heads, most, &blocks, &pieces);
      if (at < c.units) break;
      at -= c.units, slot += c.slots, set += c.groups;
    }
    const int block = (int)(at % blocks), piece = (int)(at / blocks % pieces), head = (int)(at / blocks / pieces);
    set += head * blocks + block;
    slot += (head * blocks + block) * pieces + piece;
    const int row0 = block * kRows, rows = min(kRows, q.fresh * a.group - row0);
    const int cached = tiles_of(q.held);
    const int last_token = (row0 + rows - 1) / a.group;
    const int tiles = cached + (a.mask ? tiles_of(q.fresh) : tiles_of(last_token + 1));
    const int begin = (int)((int64_t)tiles * piece / pieces), end = (int)((int64_t)tiles * (piece + 1) / pieces);
    const int t0 = begin + (end - begin) * wave / kWaves, t1 = begin + (end - begin) * (wave + 1) / kWaves;

    // -- queries: operand B of the scores, zeros behind the last dimension and the last row
    u4 query[MT][kSteps][kTerms];
    float factor[MT];  // of a score to its exponent of two
    int token[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int row = row0 + mt * 16 + n;
      const bool there = mt * 16 + n < rows;
      token[mt] = there ? row / a.group : 0;
      const int64_t from = (q.first + token[mt]) * a.q_stride + (int64_t)(head * a.group + (there ? row - token[mt] * a.group : 0)) * a.dim;
      factor[mt] = a.scale * 1.44269504088896341f;
      if constexpr (!FLOAT) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          const int d = 32 * s + 8 * g;
          u4 x{0, 0, 0, 0};
          if (there && d < a.dim) x = *reinterpret_cast<const u4*>(static_cast<const uint16_t*>(a.q) + from + d);
          query[mt][s][0] = x;
        }
      } else {
        float x[kSteps][8];
        float top = 0.f;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          const int d = 32 * s + 8 * g;
          f4 lo4{0, 0, 0, 0}, hi4{0, 0, 0, 0};
          if (there && d < a.dim) {
            const f4* p = reinterpret_cast<const f4*>(static_cast<const float*>(a.q) + from + d);
            lo4 = p[0], hi4 = p[1];
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            x[s][j] = lo4[j], x[s][4 + j] = hi4[j];
            top = fmaxf(top, fmaxf(fabsf(lo4[j]), fabsf(hi4[j])));
          }
        }
        if constexpr (sizeof(CT) == 2 && Half<CT>::kTerms == 2) {
          // float16 has not the range of float: the row's largest query becomes 2^14 (exact, taken back by the factor)
          top = over_groups_max(top);
          const int e = top > 0.f && top < INFINITY ? 15 - __builtin_amdgcn_frexp_expf(top) : 0;
#pragma unroll
          for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int j = 0; j < 8; ++j) x[s][j] = ldexpf(x[s][j], e);
          factor[mt] = ldexpf(factor[mt], -e);
        }
#pragma unroll
        for (int s = 0; s < kSteps; ++s) split<CT, kTerms>(x[s], query[mt][s]);
      }
    }

    f4 acc[MT][kParts * kEach];
    float m[MT], base[MT], l[MT];  // base: what is taken off an exponent
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      m[mt] = -INFINITY, base[mt] = 0.f, l[mt] = 0.f;
#pragma unroll
      for (int j = 0; j < kParts * kEach; ++j) acc[mt][j] = f4{0, 0, 0, 0};
    }

    u4 key[2][kSteps];
    uint32_t value[kParts][8][kEach / 2];  // [token][pair of dimensions]

    auto scores = [&](int mt, float (&s)[8]) {
      f4 x[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
      for (int k = 0; k < kSteps; ++k)
#pragma unroll
        for (int t = kTerms - 1; t >= 0; --t)
#pragma unroll
          for (int h = 0; h < 2; ++h) x[h] = Half<CT>::mfma(key[h][k], query[mt][k][t], x[h]);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = x[j >> 2][j & 3] * factor[mt];
    };
    // m follows the maximum of the row where it is left behind
    auto follow = [&](int mt, const float (&s)[8]) {
      float top = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
      if (__ballot(top > m[mt] + kSlack)) {
        top = over_groups_max(top);
        if (top > m[mt] + kSlack) {
          const float back = exp2f(m[mt] - top);  // (0 at first)
          m[mt] = top, base[mt] = top - kBias;
          l[mt] *= back;
#pragma unroll
          for (int j = 0; j < kParts * kEach; ++j) acc[mt][j] *= back;
        }
      }
    };
    auto weights = [&](int mt, float (&s)[8]) {
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = __builtin_amdgcn_exp2f(s[j] - base[mt]);
      l[mt] += ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
    };
    // operand A of the result: of eight tokens the dimension that is number j of the lane's piece
    auto transposed = [&](int part, int j) {
      u4 x;
#pragma unroll
      for (int t = 0; t < 4; ++t)
        x[t] = __builtin_amdgcn_perm(value[part][2 * t + 1][j >> 1], value[part][2 * t][j >> 1], j & 1 ? 0x07060302u : 0x05040100u);
      return x;
    };
    auto add_values = [&](const u4 (&p)[MT][kTerms]) {
#pragma unroll
      for (int part = 0; part < kParts; ++part)
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
          const u4 x = transposed(part, j);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int t = kTerms - 1; t >= 0; --t) acc[mt][part * kEach + j] = Half<CT>::mfma(x, p[mt][t], acc[mt][part * kEach + j]);
        }
    };

    // ---- cached tokens
    const int c1 = min(t1, cached);
    if (t0 < c1) {
      const int last_page = (q.held - 1) >> a.log2_page;
      const int32_t* table = a.table + (int64_t)r * a.max_pages;
      int window = (t0 * kTile) >> a.log2_page;  // the lanes hold the entries of the table from here on, and the 64 after those
      auto entry = [&](int at) { return at <= last_page ? table[at] : -1; };
      int now = entry(window + lane), next = entry(window + 64 + lane);
      const int64_t head_at = (int64_t)head * a.head_stride, in_page = (int64_t(1) << a.log2_page) - 1;
      auto page_for = [&](int position) { return __shfl(now, (position >> a.log2_page) - window); };
      auto advance = [&](int tile) {
        if (((tile * kTile + kTile - 1) >> a.log2_page) - window >= 64) {
          window += 64;  // (a tile that begins inside the window ends inside it: both begin at a multiple of a tile's pages)
          now = next;
          next = entry(window + 64 + lane);
        }
      };
      auto load_keys = [&](int tile) {
        const int position = tile * kTile + 8 * (n >> 2) + (n & 3);
        const int page = page_for(position);
        const uint16_t* p = a.cache_k + ((uint32_t)page < (uint32_t)a.pages ? page : 0) * a.page_stride + head_at + (position & in_page) * a.token_stride;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int k = 0; k < kSteps; ++k) key[h][k] = *reinterpret_cast<const u4*>(p + 4 * h * a.token_stride + min(32 * k + 8 * g, a.dim - 8));
      };
      auto load_values = [&](int tile, int& seen) {
        const int position = tile * kTile + 8 * g;
        const int page = page_for(position);
        const bool there = (uint32_t)page < (uint32_t)a.pages;
        seen = there ? (1 << max(min(q.held - position, 8), 0)) - 1 : 0;
        const uint16_t* p = a.cache_v + (there ? page : 0) * a.page_stride + head_at + (position & in_page) * a.token_stride;
#pragma unroll
        for (int part = 0; part < kParts; ++part)
#pragma unroll
          for (int t = 0; t < 8; ++t) {
            const uint16_t* from = p + t * a.token_stride + min(part * 16 * kEach + kEach * n, a.dim - kEach);
            if constexpr (kEach == 8) {
              const u4 x = *reinterpret_cast<const u4*>(from);
#pragma unroll
              for (int j = 0; j < 4; ++j) value[part][t][j] = x[j];
            } else {
              const u2 x = *reinterpret_cast<const u2*>(from);
              value[part][t][0] = x[0], value[part][t][1] = x[1];
            }
          }
      };
      int seen;
      advance(t0);
      load_keys(t0);
      load_values(t0, seen);
      for (int tile = t0; tile < c1; ++tile) {
        const bool whole = __ballot(seen != 255) == 0;
        u4 p[MT][kTerms];
        float s[MT][8];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) scores(mt, s[mt]);
        if (tile + 1 < c1) {
          advance(tile + 1);
          load_keys(tile + 1);
        }
        if (!whole) {
#pragma unroll
          for (int t = 0; t < 8; ++t) {
            const bool is = seen >> t & 1;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) s[mt][t] = is ? s[mt][t] : -INFINITY;
#pragma unroll
            for (int part = 0; part < kParts; ++part)
#pragma unroll
              for (int j = 0; j < kEach / 2; ++j) value[part][t][j] = is ? value[part][t][j] : 0u;
          }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          follow(mt, s[mt]);
          weights(mt, s[mt]);
          split<CT, kTerms>(s[mt], p[mt]);
        }
        add_values(p);
        if (tile + 1 < c1) load_values(tile + 1, seen);
      }
    }

    // ---- new tokens
    for (int tile = max(t0, cached); tile < t1; ++tile) {
      const int j0 = (tile - cached) * kTile;
      const int64_t kv_at = (int64_t)head * a.dim;
      auto load8 = [&](const void* p, int64_t at) {
        if constexpr (!FLOAT) return *reinterpret_cast<const u4*>(static_cast<const uint16_t*>(p) + at);
        else {
          const f4* f = reinterpret_cast<const f4*>(static_cast<const float*>(p) + at);
          const f4 lo4 = f[0], hi4 = f[1];
          const float x[8] = {lo4[0], lo4[1], lo4[2], lo4[3], hi4[0], hi4[1], hi4[2], hi4[3]};
          u4 t[1];
          split<CT, 1>(x, t);
          return t[0];
        }
      };
      const int j_key = j0 + 8 * (n >> 2) + (n & 3), j_value = j0 + 8 * g;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t from = (q.first + min(j_key + 4 * h, q.fresh - 1)) * a.kv_stride + kv_at;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) key[h][k] = load8(a.k, from + min(32 * k + 8 * g, a.dim - 8));
      }
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const bool there = j_value + t < q.fresh;
        const int64_t from = (q.first + min(j_value + t, q.fresh - 1)) * a.kv_stride + kv_at;
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
          if constexpr (kEach == 8) {
            const u4 x = load8(a.v, from + min(part * 128 + 8 * n, a.dim - 8));
#pragma unroll
            for (int j = 0; j < 4; ++j) value[part][t][j] = there ? x[j] : 0u;
          } else {
            const int d = min(4 * n, a.dim - 4);  // (eight from a multiple of eight, of which this lane takes its four)
            const u4 x = load8(a.v, from + (d & ~7));
#pragma unroll
            for (int j = 0; j < 2; ++j) value[part][t][j] = there ? (d & 4 ? x[2 + j] : x[j]) : 0u;
          }
        }
      }
      u4 p[MT][kTerms];
      float s[MT][8];
      int seen[MT];
      bool whole = true;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        if (a.mask) {
          const uint64_t bits = mt * 16 + n < rows ? a.mask[q.first + token[mt]] : ~0ull;
          seen[mt] = (int)(bits >> j_value) & 255;  // (j_value < 64: with a mask there are at most two tiles)
        } else {
          seen[mt] = mt * 16 + n < rows ? (1 << max(min(token[mt] + 1 - j_value, 8), 0)) - 1 : 255;
        }
        seen[mt] &= (1 << max(min(q.fresh - j_value, 8), 0)) - 1;
        whole &= seen[mt] == 255;
        scores(mt, s[mt]);
      }
      const bool partly = __ballot(!whole) != 0;
      // A value that is not finite must not reach the rows that do not see it (0 times infinity is NaN): it is left out
      // of the product and added to the rows that see it by itself.
      uint32_t odd = 0;
      if (partly) {
        constexpr uint32_t kExponent = Half<CT>::kTerms == 2 ? 0x7c00u : 0x7f80u;
#pragma unroll
        for (int t = 0; t < 8; ++t)
#pragma unroll
          for (int part = 0; part < kParts; ++part)
#pragma unroll
            for (int j = 0; j < kEach / 2; ++j) {
              uint32_t& x = value[part][t][j];
              const bool lo_odd = (x & kExponent) == kExponent, hi_odd = ((x >> 16) & kExponent) == kExponent;
              odd |= (lo_odd || hi_odd) ? 1u << t : 0u;
              x &= (lo_odd ? 0xffff0000u : ~0u) & (hi_odd ? 0x0000ffffu : ~0u);
            }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int t = 0; t < 8; ++t) s[mt][t] = seen[mt] >> t & 1 ? s[mt][t] : -INFINITY;
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        follow(mt, s[mt]);
        weights(mt, s[mt]);
        split<CT, kTerms>(s[mt], p[mt]);
      }
      add_values(p);
      if (__ballot(odd)) {
        for (int t = 0; t < kTile; ++t) {
          const int from_group = t >> 3;
          if (!(__ballot(odd >> (t & 7) & 1) >> (16 * from_group) & 0xffff)) continue;
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            float w = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) w = (t & 7) == j ? s[mt][j] : w;
            w = __shfl(w, 16 * from_group + n);
            const bool sees = __shfl(seen[mt], 16 * from_group + n) >> (t & 7) & 1;
            const int64_t from = (q.first + min(j0 + t, q.fresh - 1)) * a.kv_stride + kv_at;
#pragma unroll
            for (int part = 0; part < kParts; ++part)
#pragma unroll
              for (int j = 0; j < kEach; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const int d = part * 16 * kEach + kEach * (4 * g + i) + j;
                  if (sees && d < a.dim) {
                    float x;
                    if constexpr (FLOAT) x = (float)(CT)static_cast<const float*>(a.v)[from + d];
                    else x = (float)static_cast<const CT*>(a.v)[from + d];
                    if (!(fabsf(x) < INFINITY)) acc[mt][part * kEach + j][i] += w * x;
                  }
                }
          }
        }
      }
    }

    // ---- the four wavefronts of the workgroup
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      l[mt] = over_groups_sum(l[mt]);
      if (g == 0) row_m[wave][mt * 16 + n] = m[mt], row_l[wave][mt * 16 + n] = l[mt];
    }
    __syncthreads();
    float* const mine_out = a.partial + (int64_t)slot * kRows * stride_of_partial<DP>();
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      if (mt * 16 < rows) {
        const int row = mt * 16 + n;
        const float top = fmaxf(fmaxf(row_m[0][row], row_m[1][row]), fmaxf(row_m[2][row], row_m[3][row]));
        const float mine_scale = m[mt] == -INFINITY ? 0.f : exp2f(m[mt] - top);
#pragma unroll
        for (int part = 0; part < kParts; ++part)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < kEach; j += 4) {
              const f4 x{acc[mt][part * kEach + j][i], acc[mt][part * kEach + j + 1][i], acc[mt][part * kEach + j + 2][i], acc[mt][part * kEach + j + 3][i]};
              *reinterpret_cast<f4*>(&joined[wave][n][part * 16 * kEach + kEach * (4 * g + i) + j]) = x * mine_scale;
            }
      }
      __syncthreads();
      for (int e = tid; e < 16 * (DP / 4); e += kThreads) {
        const int row = e / (DP / 4), d = e % (DP / 4) * 4, of = mt * 16 + row;
        if (of >= rows || d >= a.dim) continue;
        const f4 x = (*reinterpret_cast<const f4*>(&joined[0][row][d]) + *reinterpret_cast<const f4*>(&joined[1][row][d])) +
                     (*reinterpret_cast<const f4*>(&joined[2][row][d]) + *reinterpret_cast<const f4*>(&joined[3][row][d]));
        const float top = fmaxf(fmaxf(row_m[0][of], row_m[1][of]), fmaxf(row_m[2][of], row_m[3][of]));
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) total += row_m[w][of] == -INFINITY ? row_l[w][of] : row_l[w][of] * exp2f(row_m[w][of] - top);
        if (pieces == 1) {
          const int id = row0 + of, tok = id / a.group;
          const int64_t to = (q.first + tok) * a.out_stride + (int64_t)(head * a.group + id - tok * a.group) * a.dim + d;
          const f4 o = total == 0.f ? f4{0, 0, 0, 0} : x / total;
          if constexpr (FLOAT) {
            *reinterpret_cast<f4*>(static_cast<float*>(a.out) + to) = o;
          } else {
            const typename Half<CT>::v2 lo2{(CT)o[0], (CT)o[1]}, hi2{(CT)o[2], (CT)o[3]};
            *reinterpret_cast<u2*>(static_cast<uint16_t*>(a.out) + to) = u2{__builtin_bit_cast(uint32_t, lo2), __builtin_bit_cast(uint32_t, hi2)};
          }
        } else {
          float* to = mine_out + of * stride_of_partial<DP>();
          *reinterpret_cast<f4*>(to + d) = x;
          if (d == 0) to[DP] = top, to[DP + 1] = total;
        }
      }
      __syncthreads();
    }
    if (pieces == 1) continue;

    // ---- the pieces of these rows: the workgroup that comes last joins them
    __threadfence();
    __syncthreads();
    if (tid == 0) arrived = __hip_atomic_fetch_add(&a.counters[set], 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    const bool last = arrived == (uint32_t)pieces - 1;
    __syncthreads();
    if (!last) continue;
    __threadfence();
    if (tid == 0) __hip_atomic_store(&a.counters[set], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const float* const all = a.partial + (int64_t)(slot - piece) * kRows * stride_of_partial<DP>();
    constexpr int kPiece = kRows * stride_of_partial<DP>();
    for (int e = tid; e < kRows * (DP / 4); e += kThreads) {
      const int of = e / (DP / 4), d = e % (DP / 4) * 4;
      if (of >= rows || d >= a.dim) continue;
      const float* from = all + of * stride_of_partial<DP>();
      float top = -INFINITY, total = 0.f;
#pragma unroll 4
      for (int c = 0; c < pieces; ++c) top = fmaxf(top, from[(int64_t)c * kPiece + DP]);
      f4 x{0, 0, 0, 0};
#pragma unroll 4
      for (int c = 0; c < pieces; ++c) {
        const float* p = from + (int64_t)c * kPiece;
        const float w = p[DP] == -INFINITY ? 0.f : exp2f(p[DP] - top), lc = p[DP + 1];
        const f4 xc = *reinterpret_cast<const f4*>(p + d);
        total += p[DP] == -INFINITY ? lc : lc * w;
        x += xc * w;
      }
      const int id = row0 + of, tok = id / a.group;
      const int64_t to = (q.first + tok) * a.out_stride + (int64_t)(head * a.group + id - tok * a.group) * a.dim + d;
      const f4 o = total == 0.f ? f4{0, 0, 0, 0} : x / total;
      if constexpr (FLOAT) {
        *reinterpret_cast<f4*>(static_cast<float*>(a.out) + to) = o;
      } else {
        const typename Half<CT>::v2 lo2{(CT)o[0], (CT)o[1]}, hi2{(CT)o[2], (CT)o[3]};
        *reinterpret_cast<u2*>(static_cast<uint16_t*>(a.out) + to) = u2{__builtin_bit_cast(uint32_t, lo2), __builtin_bit_cast(uint32_t, hi2)};
      }
    }
  }
}

// ---- host ---------------------------------------------------------------------------------------------------
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

// The kernel for a call, and how it is launched.
struct Shape {
  int dims;         // head_dim, padded
  int row_tiles;    // tiles of 16 rows that a wavefront carries
  int target;       // pieces of work that are aimed at
  int64_t counters_bytes, bytes;  // of the workspace
};

// `floats`: the activations are float, whose queries and weights take several operands each
Shape shape_of(const rsr_cache_t* cache, const rsr_step_t* step, int heads, bool floats) {
  Shape s;
  s.dims = cache->head_dim <= 64 ? 64 : cache->head_dim <= 128 ? 128 : 256;
  const int64_t rows = (int64_t)step->max_new * (heads / cache->kv_heads);
  s.row_tiles = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  if (s.dims == 256 && s.row_tiles > 2) s.row_tiles = 2;
  if (floats && s.dims == 256) s.row_tiles = 1;
  if (floats && s.dims == 128 && s.row_tiles > 2) s.row_tiles = 2;
  s.target = 512;
  s.counters_bytes = (int64_t)s.target * 4;
  s.bytes = s.counters_bytes + (int64_t)2 * s.target * 16 * s.row_tiles * (s.dims + 4) * 4;
  return s;
}

template <typename CT, bool FLOAT> void (*kernel_of(const Shape& s))(Args) {
  if (s.dims == 64) return s.row_tiles == 1 ? attend_kernel<CT, FLOAT, 64, 1> : s.row_tiles == 2 ? attend_kernel<CT, FLOAT, 64, 2> : attend_kernel<CT, FLOAT, 64, 4>;
  if constexpr (FLOAT) {
    if (s.dims == 128) return s.row_tiles == 1 ? attend_kernel<CT, FLOAT, 128, 1> : attend_kernel<CT, FLOAT, 128, 2>;
    return attend_kernel<CT, FLOAT, 256, 1>;
  } else {
    if (s.dims == 128) return s.row_tiles == 1 ? attend_kernel<CT, FLOAT, 128, 1> : s.row_tiles == 2 ? attend_kernel<CT, FLOAT, 128, 2> : attend_kernel<CT, FLOAT, 128, 4>;
    return s.row_tiles == 1 ? attend_kernel<CT, FLOAT, 256, 1> : attend_kernel<CT, FLOAT, 256, 2>;
  }
}

}  // namespace

extern "C" {

int64_t rsr_tree_attention_workspace(const rsr_cache_t* cache, const rsr_step_t* step, int heads) {
  if (const char* fault = fault_of(cache, step, heads)) return set_error(RSR_ERR_INVALID_ARGUMENT, fault);
  return std::max(shape_of(cache, step, heads, false).bytes, shape_of(cache, step, heads, true).bytes);
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
  const bool floats = dtype == RSR_F32;
  const Shape s = shape_of(cache, step, heads, floats);
  fault = rsr_internal::fault_of_rows(q, q_stride, width, dtype);
  if (!fault) fault = rsr_internal::fault_of_rows(k, kv_stride, kv_width, dtype);
  if (!fault) fault = rsr_internal::fault_of_rows(v, kv_stride, kv_width, dtype);
  if (!fault) fault = rsr_internal::fault_of_rows(out, out_stride, width, dtype);
  if (!fault && (!workspace || !rsr_internal::aligned(workspace, 256) || workspace_bytes < s.bytes))
    fault = "the workspace is missing, too small or not 256-byte aligned";
  if (fault) return set_error(RSR_ERR_INVALID_ARGUMENT, fault);
  const Args a{q, k, v, out, static_cast<const uint16_t*>(cache->k), static_cast<const uint16_t*>(cache->v), step->table, step->held, step->start, step->mask,
               static_cast<uint32_t*>(workspace), reinterpret_cast<float*>(static_cast<char*>(workspace) + s.counters_bytes),
               q_stride, kv_stride, out_stride, cache->page_stride, cache->head_stride, cache->token_stride, step->requests, step->tokens, step->max_new,
               step->max_pages, rsr_internal::log2_of(cache->page_size), cache->pages, cache->kv_heads, cache->head_dim, heads / cache->kv_heads, s.target, scale};
  auto kern = cache->dtype == RSR_F16 ? (floats ? kernel_of<_Float16, true>(s) : kernel_of<_Float16, false>(s))
                                      : (floats ? kernel_of<__bf16, true>(s) : kernel_of<__bf16, false>(s));
  // no more workgroups than there can be pieces
  const int64_t blocks = ((int64_t)step->max_new * (heads / cache->kv_heads) + 16 * s.row_tiles - 1) / (16 * s.row_tiles);
  const int64_t tiles = (((int64_t)step->max_pages * cache->page_size) + kTile - 1) / kTile + (step->max_new + kTile - 1) / kTile;
  const int64_t units = step->requests * (int64_t)cache->kv_heads * blocks * ((tiles + kLeastTiles - 1) / kLeastTiles);
  hipLaunchKernelGGL(kern, dim3((unsigned)std::min(units, (int64_t)s.target)), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(RSR_ERR_HIP, std::string("rsr_tree_attention: ") + hipGetErrorString(e));
  return RSR_OK;
}

}  // extern "C"
