// Attention of a step's new tokens over the paged cache and over each other (include/rsr_cache.h).
//
// The scores of 16 query rows (a row: one new token, one query head) and 32 positions are S^T = K Q^T on the matrix cores, the
// result is O^T += V^T P^T with P = 2^(S - m), and a running maximum m and sum l per row: one pass over the cache.
// Transposed, because the positions of a score tile then lie along a lane's registers: what S^T leaves in a lane, eight
// consecutive positions of one row, is the operand that V^T P^T wants there, and P never leaves its registers.  l is one more
// row of the result, with ones for values.
//
// Position order.  Lane (n, g) = (lane & 15, lane >> 4) holds of S^T the rows 4g .. 4g+3 of two tiles of 16 keys.  With key
// 8 (x >> 2) + (x & 3) in row x of the first tile and that plus 4 in the second, these are the positions 8g .. 8g+7.
// Values: the lane reads eight dimensions of each of these positions (whole rows side by side) and has, after exchanging halves
// of dwords with v_perm_b32, eight positions of each dimension, the other operand.
//
// Two kernels, by the rows that a key head has (new tokens times query heads of the group):
//   attend_split  up to 16: the wavefronts of a workgroup take the same rows and different positions, keys and values go
//                 from the cache straight into registers, LDS serves to join the wavefronts at the end
//   attend_shared more: the wavefronts take different rows and the same positions, which come through LDS
// The positions (tiles of 32: first a request's cached ones, then its new ones) are cut into equal pieces, or, if these were more
// than the workgroups that the chip runs at once, dealt out evenly to those (32 ragged requests of up to 8192: 138 us, with pieces
// of one length 181).  The pieces of a row meet in the workspace, where the workgroup that comes last joins them in their order.
//
// Measured on one MI355X, whole calls (a large copy moves 4.8 TB/s there, a sum reads 4.0, a large product does 1.23 PFLOP/s with
// 16-bit operands): 32 requests of one token, 20 heads of 128, 8192 cached tokens each: 453 us, 5.9 TB/s of cache, bound by memory.
// 16 drafted tokens over 4096, the same heads: 18 us for 42.6 MB; a token over 500: 12 us for 5.2 MB, a chain of latencies (lengths,
// table, tiles, the join).  64 drafted tokens with four query heads per key head, 4 requests over 131072: 0.47 to 0.49 ms, 0.7 PFLOP/s;
// one request over 2000: 21 us.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <string>

#include "rsr_cache_check.h"

namespace {

using rsr_internal::set_error;

constexpr int kTile = 32;        // positions of a tile
constexpr int kLeastTiles = 16;  // of a workgroup of attend_split, about (a set may have fewer)
constexpr int kLeastShared = 4;  // and of attend_shared
constexpr float kBias = 7.f;     // weights are 2^(s - m + 7): as float16 they keep their bits down to 2^-21 of the largest
constexpr float kUnseen = -FLT_MAX;  // the exponent of what a row does not see: a weight of 0, and not a maximum
constexpr float kLimit = 15.f;   // m follows the maximum when a weight would pass 2^15, so that it seldom does

typedef float f2 __attribute__((ext_vector_type(2)));
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
  int64_t head_stride;
  uint32_t q_stride, kv_stride, out_stride, page_stride, token_stride;
  int32_t requests, tokens, max_new, max_pages, log2_page, pages, kv_heads, dim, group;
  uint32_t group_inverse;  // ceil(2^32 / group), 0 for 1
  float scale;
};

// ---- the cache's types on the matrix cores -----------------------------------------------------------------
template <typename CT> struct Half;
template <> struct Half<_Float16> {
  typedef _Float16 v8 __attribute__((ext_vector_type(8)));
  typedef _Float16 v2 __attribute__((ext_vector_type(2)));
  static constexpr int kTerms = 2;  // of a float: 22 bits
  static constexpr uint32_t kExponent = 0x7c00, kOnes = 0x3c003c00;
  static __device__ f4 mfma(u4 a, u4 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
};
template <> struct Half<__bf16> {
  typedef __bf16 v8 __attribute__((ext_vector_type(8)));
  typedef __bf16 v2 __attribute__((ext_vector_type(2)));
  static constexpr int kTerms = 3;  // of a float: all 24 bits
  static constexpr uint32_t kExponent = 0x7f80, kOnes = 0x3f803f80;
  static __device__ f4 mfma(u4 a, u4 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
};

template <typename CT> __device__ inline uint32_t pair_of(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, typename Half<CT>::v2{(CT)lo, (CT)hi});
}

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

// Eight activations in the cache's type, from eight in memory.
template <typename CT, bool FLOAT> struct Eight {
  u4 raw[FLOAT ? 2 : 1];
  __device__ void load(const void* p, int64_t at) {
    const u4* from = reinterpret_cast<const u4*>(static_cast<const char*>(p) + at * (FLOAT ? 4 : 2));
    raw[0] = from[0];
    if constexpr (FLOAT) raw[1] = from[1];
  }
  __device__ u4 rounded() const {
    if constexpr (!FLOAT) return raw[0];
    else {
      const f4 lo = __builtin_bit_cast(f4, raw[0]), hi = __builtin_bit_cast(f4, raw[1]);
      return u4{pair_of<CT>(lo[0], lo[1]), pair_of<CT>(lo[2], lo[3]), pair_of<CT>(hi[0], hi[1]), pair_of<CT>(hi[2], hi[3])};
    }
  }
};

// x, of which the compiler knows nothing more: what follows from a lane's number is then worked out where it is used and does not
// fill registers through the loops before.
__device__ inline int hidden(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// The largest over the four lanes n, n + 16, n + 32, n + 48.
__device__ inline float over_groups_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

__device__ inline float max3(float x, float y, float z) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(x), "v"(y), "v"(z));
  return r;
}

__device__ inline float min3(float x, float y, float z) {
  float r;
  asm("v_min3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(x), "v"(y), "v"(z));
  return r;
}

// Where the elements of row `row` of activations begin.
__device__ inline int64_t row_at(int row, uint32_t stride) { return (int64_t)((uint64_t)(uint32_t)row * stride); }

__device__ inline int eight_bits(int count) { return (1 << max(min(count, 8), 0)) - 1; }  // the lowest `count`

// ---- which piece of work ------------------------------------------------------------------------------------
__device__ inline int tiles_of(int n) { return (n + kTile - 1) / kTile; }

struct Request {
  int32_t first;  // row of its first new token
  int32_t fresh;  // new tokens
  int32_t held;   // cached tokens
};

__device__ inline Request request_of(const Args& a, int r) {
  const int64_t first = a.start[r], end = min((int64_t)a.start[r + 1], (int64_t)a.tokens);
  const int64_t fresh = first < 0 ? 0 : max(min(end - first, (int64_t)a.max_new), (int64_t)0);
  const int64_t held = min((int64_t)max(a.held[r], 0), (int64_t)a.max_pages << a.log2_page);
  return {(int32_t)first, (int32_t)fresh, (int32_t)min(held, (int64_t)INT32_MAX - 65536 - 1024)};
}

template <typename T> __device__ inline T from_lane(T x, int lane) {
  if constexpr (sizeof(T) == 8) {
    const uint64_t v = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)v, lane), hi = __builtin_amdgcn_readlane((int)(v >> 32), lane);
    return __builtin_bit_cast(T, (uint64_t)hi << 32 | lo);
  } else {
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
  }
}

__device__ inline int token_of(const Args& a, int row) { return a.group_inverse ? (int)__umulhi((uint32_t)row, a.group_inverse) : row; }

// A set: the rows of a key head that a workgroup takes together.  A workgroup has one piece of a set, or, where the tiles of all
// sets are dealt out, the end of one set, whole sets, and the beginning of another.
struct Unit {
  Request q;
  int32_t r, head, row0, rows;   // request, key head, first row and rows
  int32_t piece, pieces;         // of the set
  int32_t slot0, counter;        // where its pieces lie in the workspace, and where they are counted
  int32_t tile0, tile1, cached;  // its tiles; tiles of cached tokens (those behind hold new ones)
  __device__ int slot(int c) const { return slot0 + 2 * c - (c > 0); }
};

// Quotients in floating point that are off by one at most, and put right: n / d where that is below 2^20; x / y for x below 2^51
// (rsr_tree_attention sees to that).  (A workgroup waits for some of these before its first load.)
__device__ inline int quotient(int n, int d) {
  const int q = (int)((float)n * __builtin_amdgcn_rcpf((float)d)), left = n - q * d;
  return q + (left >= d) - (left < 0);
}
__device__ inline int64_t divided(int64_t x, int64_t y) {
  if (x < (1 << 20)) return quotient((int)x, (int)min(y, (int64_t)1 << 20));
  int64_t q = (int64_t)((double)x / (double)y);
  const int64_t left = x - q * y;
  return q + (left >= y) - (left < 0);
}

// Every wavefront adds up the tiles of all requests by itself, a run of requests per lane, without a barrier.
//
// Where the chip has room for that many workgroups, each set is cut into as many equal pieces as suit it, a workgroup each.  A
// workgroup of attend_split has some 16 tiles, four or two for a wavefront.  In attend_shared n pieces of T tiles take the time of
// T / n tiles and then of n pieces taken up, each that of one and a half tiles (float: of three quarters), least with n = sqrt(T /
// 1.5).  (Sets of 64 rows and 62 tiles: 21 us with pieces of 8, 24 of 16, 28 of 5; 130 tiles: 26 us with 16, 36 with 8, 41 with 5;
// 16 tiles: 17 us with 8, 25 with 16.)  With more work the tiles of all sets, one set behind the other, are dealt out in equal
// runs.  (Seven ragged requests of 13 tokens over up to 3001: 28 us cut, 34 dealt out.)
template <int ROWS, bool SPLIT, bool FLOAT> struct Plan {
  int64_t end, work;        // tiles up to the lane's last request; of all
  Request q;                // the lane's first request
  int32_t run, groups;      // requests per lane; workgroups with work
  int32_t pieces_end;       // pieces up to the lane's last request, if the sets are cut
  bool cut;
  static constexpr int kMany = 1 << 24;  // more sets or pieces than a chip has workgroups

  static __device__ int blocks_of(const Args& a, const Request& q) { return (q.fresh * a.group + ROWS - 1) / ROWS; }
  static __device__ int tiles_in(const Request& q) { return tiles_of(q.held) + tiles_of(q.fresh); }
  static __device__ int64_t sets_of(const Args& a, const Request& q) { return (int64_t)blocks_of(a, q) * a.kv_heads; }
  static __device__ int pieces_of(const Request& q) {
    const int tiles = tiles_in(q);
    if constexpr (SPLIT) return max((tiles + kLeastTiles / 2) / kLeastTiles, 1);
    else return max(min((int)(sqrtf((float)tiles * (FLOAT ? 4.f / 3 : 2.f / 3)) + 0.5f), tiles / kLeastShared), 1);
  }

  __device__ explicit Plan(const Args& a, int lane) {
    run = (a.requests + 63) / 64;
    const int r0 = min(lane * run, a.requests), r1 = min(r0 + run, a.requests);
    int sets = 0;
    end = 0, pieces_end = 0;
    q = {0, 0, 0};
    for (int r = r1 - 1; r >= r0; --r) {
      q = request_of(a, r);
      const int64_t more = sets_of(a, q);
      end += more * tiles_in(q);
      sets = (int)min(sets + more, (int64_t)kMany);
      pieces_end = (int)min(pieces_end + more * pieces_of(q), (int64_t)kMany);
    }
    if (a.requests > 1) {
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int64_t u = __shfl_up(end, d);
        const int v = __shfl_up(sets, d), w = __shfl_up(pieces_end, d);
        if (lane >= d) end += u, sets += v, pieces_end += w;
      }
      work = from_lane(end, 63), sets = from_lane(sets, 63), groups = from_lane(pieces_end, 63);
    } else {
      work = end = from_lane(end, 0), sets = from_lane(sets, 0), groups = pieces_end = from_lane(pieces_end, 0);
    }
    cut = groups <= (int)gridDim.x;
    if (!cut) {
      groups = gridDim.x;
      // as many for each set, if few are lost by it: sets of one length are then cut alike and no workgroup has parts of two
      if (sets && sets <= groups && groups % sets <= groups / 8) groups -= groups % sets;
    }
  }

  // Where a workgroup begins: a piece, or a tile of all.
  __device__ int64_t begin_of(int group) const { return cut ? group : divided(work * group, groups); }
  __device__ int group_of(int64_t tile) const { return (int)divided((tile + 1) * groups - 1, work); }  // whose run it is in

  // The piece that begins at `at` and, if it is a tile, ends at `stop` at the latest; `at` moves on behind it.
  __device__ Unit next(const Args& a, int64_t& at, int64_t stop) const {
    Unit u;
    const int lane = __builtin_amdgcn_readfirstlane(__builtin_ctzll(__ballot(cut ? pieces_end > at : end > at)));
    int64_t before = !lane ? 0 : cut ? from_lane(pieces_end, lane - 1) : from_lane(end, lane - 1);
    u.r = lane * run;
    if (run == 1) {
      u.q = {from_lane(q.first, lane), from_lane(q.fresh, lane), from_lane(q.held, lane)};
    } else {
      for (;; ++u.r) {
        const Request q = request_of(a, u.r);
        u.q = {from_lane(q.first, 0), from_lane(q.fresh, 0), from_lane(q.held, 0)};
        const int64_t here = sets_of(a, u.q) * (cut ? pieces_of(u.q) : tiles_in(u.q));
        if (at < before + here) break;
        before += here;
      }
    }
    const int all = tiles_in(u.q), blocks = blocks_of(a, u.q);
    int set;
    if (cut) {
      // (512 pieces at most, and so fewer than 2^19 tiles)
      const int in = (int)(at - before);
      u.pieces = __builtin_amdgcn_readfirstlane(pieces_of(u.q));
      set = quotient(in, u.pieces);
      u.piece = in - set * u.pieces, u.counter = (int)at - u.piece;
      u.tile0 = quotient(all * u.piece, u.pieces), u.tile1 = quotient(all * (u.piece + 1), u.pieces);
      u.head = blocks == 1 ? set : quotient(set, blocks);
      at += 1;
    } else {
      set = (int)divided(at - before, all);
      const int64_t from = before + (int64_t)set * all, last = min(from + all, stop);
      u.tile0 = (int)(at - from), u.tile1 = (int)(last - from);
      u.pieces = 1, u.piece = 0, u.counter = 0;
      if (at > from || last < from + all) {
        u.counter = group_of(from);
        u.pieces = group_of(from + all - 1) - u.counter + 1, u.piece = group_of(at) - u.counter;
      }
      u.head = blocks == 1 ? set : (int)divided(set, blocks);
      at = last;
    }
    u.slot0 = 2 * u.counter + 1;  // the first workgroup's last run; of the others their first: 2 (first + c)
    // (long and short blocks of a chain in turn: a run of tiles has some of both)
    const int in = set - u.head * blocks, block = in & 1 ? blocks - 1 - (in >> 1) : in >> 1;
    u.row0 = block * ROWS, u.rows = min(ROWS, u.q.fresh * a.group - u.row0);
    u.cached = tiles_of(u.q.held);
    if (!a.mask) {  // a chain's rows see no further than themselves: a share of fewer tiles
      const int tiles = u.cached + tiles_of(token_of(a, u.row0 + u.rows - 1) + 1);
      if (tiles < all) u.tile0 = (int)divided((int64_t)u.tile0 * tiles, all), u.tile1 = (int)divided((int64_t)u.tile1 * tiles, all);
    }
    return u;
  }
};

// Runs that follow each other (the same cached tokens for other rows) go to workgroups of one XCD (blockIdx % 8), as many to
// each.  (The grid is a multiple of eight.)  -1: none is left for this one.
__device__ inline int group_index(int groups) {
  const int each = (groups + 7) / 8, in = blockIdx.x / 8, group = blockIdx.x % 8 * each + in;
  return in < each && group < groups ? group : -1;
}

// The first of `count` dimensions: where the head ends before them the last ones it has (they meet zeros of the query, or a
// result that nobody wants).  FULL: the head has as many dimensions as the kernel.
template <bool FULL> __device__ inline int within(const Args& a, int d, int count) { return FULL ? d : min(d, a.dim - count); }

// ---- the rows of a wavefront --------------------------------------------------------------------------------
template <typename CT, bool FLOAT, int DP> struct Rows {
  static constexpr int kTerms = FLOAT ? Half<CT>::kTerms : 1;
  static constexpr int kSteps = DP / 32;                   // of a score's sum
  static constexpr int kEach = DP / 16 < 8 ? DP / 16 : 8;  // neighbouring dimensions of a lane's piece of a value
  static constexpr int kParts = DP / (16 * kEach);         // such pieces

  f4 acc[kParts * kEach];
  f4 sum;        // four times the same for finite scores
  float factor;  // of a score to its exponent of two
  float base;    // taken off the exponents: m - kBias
  float limit;   // of an exponent: kLimit, and kUnseen before the row has seen anything
  uint64_t sees;  // new tokens, a bit each; in a chain how many

  // Queries of the 16 rows from `first` on: operand B of the scores, zeros behind the last dimension and the last row.
  __device__ void begin(const Args& a, const Unit& u, int first, int n, int g, u4 (&query)[kSteps][kTerms]) {
    const int in = first + n, row = u.row0 + in;
    const bool there = in < u.rows;
    const int token = there ? token_of(a, row) : 0;
    const int64_t from = row_at(u.q.first + token, a.q_stride) + (u.head * a.group + (there ? row - token * a.group : 0)) * a.dim;
    // (a row that is not there sees all: it must not make a tile one that has to be masked)
    sees = a.mask ? there ? a.mask[u.q.first + token] : ~0ull : there ? token + 1 : a.max_new;
    factor = a.scale * 1.44269504088896341f;
    base = 0.f, limit = kUnseen;
    sum = f4{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < kParts * kEach; ++j) acc[j] = f4{0, 0, 0, 0};
    if constexpr (!FLOAT) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int d = 32 * s + 8 * g;
        u4 x{0, 0, 0, 0};
        if (there && d < a.dim) x = *reinterpret_cast<const u4*>(static_cast<const uint16_t*>(a.q) + from + d);
        query[s][0] = x;
      }
    } else {
      float x[kSteps][8];
      float top = 0.f;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int d = 32 * s + 8 * g;
        f4 lo{0, 0, 0, 0}, hi{0, 0, 0, 0};
        if (there && d < a.dim) {
          const f4* p = reinterpret_cast<const f4*>(static_cast<const float*>(a.q) + from + d);
          lo = p[0], hi = p[1];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[s][j] = lo[j], x[s][4 + j] = hi[j];
          top = fmaxf(top, fmaxf(fabsf(lo[j]), fabsf(hi[j])));
        }
      }
      if constexpr (Half<CT>::kTerms == 2) {
        // float16 has not the range of float: the row's largest query becomes 2^14 (exact, taken back by the factor)
        top = over_groups_max(top);
        const int e = top > 0.f && top < INFINITY ? 15 - __builtin_amdgcn_frexp_expf(top) : 0;
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
          for (int j = 0; j < 8; ++j) x[s][j] = ldexpf(x[s][j], e);
        factor = ldexpf(factor, -e);
      }
#pragma unroll
      for (int s = 0; s < kSteps; ++s) split<CT, kTerms>(x[s], query[s]);
    }
  }

  // Scores of two tiles of 16 keys, a step of 32 dimensions.
  static __device__ void add_score(u4 lo, u4 hi, const u4 (&query)[kTerms], f4 (&x)[2]) {
#pragma unroll
    for (int t = kTerms - 1; t >= 0; --t) {
      x[0] = Half<CT>::mfma(lo, query[t], x[0]);
      x[1] = Half<CT>::mfma(hi, query[t], x[1]);
    }
  }

  __device__ void exponents(const f4 (&x)[2], float (&s)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = fmaf(x[j >> 2][j & 3], factor, -base);
  }

  // Exponents to weights and to operand B of the result.  With 16-bit rows a weight is one operand of that type, 8 or 11 bits, and the
  // sum is that of the rounded weights: the error is 1.4 times that of rounding the result.  (The rest as a second operand takes that
  // away and costs twice the matrix instructions of the result: 4 x 64 tokens over 131072 762 us instead of 482, spilling in the loop;
  // chains of 512 over 2048 110 instead of 79; with one tile of rows 1 to 7 % more.)
  //
  // A score of minus infinity (a key that is not finite, products beyond the range of float) would drop out with a weight of 0, and a
  // row of such scores would look like one that sees nothing.  Zero times the lowest exponent is NaN there and 0 else, and goes into
  // one of a lane's four sums, which finish() looks at: five instructions a tile, no register and no branch (4 x 64 tokens over 131072
  // 472 us, without it 467; with a branch 723, with the lowest exponent in a register of its own 631).
  __device__ void weigh(float (&s)[8], u4 (&p)[kTerms]) {
    sum[1] = fmaf(min3(min3(s[0], s[1], s[2]), min3(s[3], s[4], s[5]), min3(s[6], s[7], s[7])), 0.f, sum[1]);
    float top = max3(max3(max3(s[0], s[1], s[2]), s[3], s[4]), max3(s[5], s[6], s[7]), -INFINITY);
    if (__ballot(top > limit)) {
      // the maximum follows where it is left behind: a row's matter alone, so that no other row's scores move it
      top = over_groups_max(top);
      if (top > limit) {
        const float up = top - kBias, back = limit == kLimit ? exp2f(-up) : 0.f;
        base += up;
        limit = kLimit;
        sum *= back;
#pragma unroll
        for (int j = 0; j < kParts * kEach; ++j) acc[j] *= back;
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] -= up;
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = __builtin_amdgcn_exp2f(s[j]);
    split<CT, kTerms>(s, p);
    const u4 ones{Half<CT>::kOnes, Half<CT>::kOnes, Half<CT>::kOnes, Half<CT>::kOnes};
#pragma unroll
    for (int t = kTerms - 1; t >= 0; --t) sum = Half<CT>::mfma(ones, p[t], sum);
  }

  // Behind the last tile.
  __device__ void finish() {
    float x = sum[1] + __shfl_xor(sum[1], 16);
    x += __shfl_xor(x, 32);
    if (x != x) sum[0] = x;
  }

  // Of eight positions the dimension that is number j of the lane's piece.
  static __device__ u4 column(const uint32_t (&value)[8][kEach / 2], int j) {
    u4 x;
#pragma unroll
    for (int t = 0; t < 4; ++t) x[t] = __builtin_amdgcn_perm(value[2 * t + 1][j >> 1], value[2 * t][j >> 1], j & 1 ? 0x07060302u : 0x05040100u);
    return x;
  }
  __device__ void add_column(int at, u4 x, const u4 (&p)[kTerms]) {
#pragma unroll
    for (int t = kTerms - 1; t >= 0; --t) acc[at] = Half<CT>::mfma(x, p[t], acc[at]);
  }
  // Values of part `part`: [position][pair of dimensions].
  __device__ void add_values(int part, const uint32_t (&value)[8][kEach / 2], const u4 (&p)[kTerms]) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) add_column(part * kEach + j, column(value, j), p);
  }

  // Which of eight new tokens from number j0 on the row sees, a bit each.
  __device__ int seen_new(const Args& a, const Unit& u, int j0) const {
    return (a.mask ? (int)(sees >> min(j0, 63)) & 255 : eight_bits((int)sees - j0)) & eight_bits(u.q.fresh - j0);
  }

  // Which of the lane's eight positions have a value that is not finite?
  static __device__ uint32_t odd_positions(const uint32_t (&value)[8][kEach / 2]) {
    typedef uint16_t us2 __attribute__((ext_vector_type(2)));
    uint32_t odd = 0;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      us2 most{0, 0};
#pragma unroll
      for (int j = 0; j < kEach / 2; ++j) most = __builtin_elementwise_max(most, __builtin_bit_cast(us2, value[t][j] & 0x7fff7fffu));
      odd |= most.x >= Half<CT>::kExponent || most.y >= Half<CT>::kExponent ? 1u << t : 0u;
    }
    return odd;
  }
  // What is not finite becomes zero, in positions that have such a value.
  static __device__ void take_out(uint32_t (&value)[8][kEach / 2], uint32_t odd) {
#pragma unroll
    for (int t = 0; t < 8; ++t)
#pragma unroll
      for (int j = 0; j < kEach / 2; ++j) {
        const uint32_t x = value[t][j], e = Half<CT>::kExponent;
        value[t][j] = odd >> t & 1 ? x & ((x & e) == e ? 0xffff0000u : ~0u) & ((x >> 16 & e) == e ? 0xffffu : ~0u) : x;
      }
  }
  static __device__ void leave_out(uint32_t (&value)[8][kEach / 2], uint32_t positions) {
#pragma unroll
    for (int t = 0; t < 8; ++t)
#pragma unroll
      for (int j = 0; j < kEach / 2; ++j) value[t][j] = positions >> t & 1 ? 0u : value[t][j];
  }

  __device__ float maximum() const { return limit == kLimit ? base + kBias : -INFINITY; }
  // Four dimensions from dimension 16 * kEach * part + kEach * (4 * g + i) + j on.
  __device__ f4 four(int part, int i, int j) const {
    return f4{acc[part * kEach + j][i], acc[part * kEach + j + 1][i], acc[part * kEach + j + 2][i], acc[part * kEach + j + 3][i]};
  }
};

// ---- results ------------------------------------------------------------------------------------------------
template <typename CT, bool FLOAT> __device__ inline void store(const Args& a, const Unit& u, int in, int d, f4 x, float total) {
  const int row = u.row0 + in, token = token_of(a, row);
  const int64_t to = row_at(u.q.first + token, a.out_stride) + (u.head * a.group + row - token * a.group) * a.dim + d;
  const f4 o = total == 0.f ? f4{0, 0, 0, 0} : x * (1.f / total);
  if constexpr (FLOAT) *reinterpret_cast<f4*>(static_cast<float*>(a.out) + to) = o;
  else *reinterpret_cast<u2*>(static_cast<uint16_t*>(a.out) + to) = u2{pair_of<CT>(o[0], o[1]), pair_of<CT>(o[2], o[3])};
}

// A piece in the workspace: its values in the order in which lanes hold them, so that a wavefront writes and reads whole lines (pairs
// of floats, 512 bytes for 64 lanes), then a maximum and a sum of weights for every row.  (In the order of the rows, scattered writes
// of eight bytes: 32 ragged requests 138 us instead of 88, 4 x 64 tokens over 131072 0.57 ms instead of 0.49.)
//   SPLIT  lane e % (16 * DP / 4) of attend_split has the four values e of rows of DP / 4
//   else   a wavefront of attend_shared has 16 rows as in Rows: pair r of lane (n, g) are the values i and i + 1 of acc[r / 2]
template <int DP, int ROWS, bool SPLIT> struct Partial {
  static constexpr int kPiece = ROWS * (DP + 2);
  static __device__ float* of(const Args& a, int slot) { return a.partial + (int64_t)slot * kPiece; }
  static __device__ float* fours(float* piece, int e, int half) { return piece + (half * (ROWS * DP / 4) + e) * 2; }
  static __device__ float* pair(float* piece, int tile, int r, int lane) { return piece + ((tile * (DP / 8) + r) * 64 + lane) * 2; }
  static __device__ float* sums(float* piece, int in) { return piece + ROWS * DP + 2 * in; }
  static __device__ float* value(float* piece, int in, int d) {
    if constexpr (SPLIT) return fours(piece, in * (DP / 4) + d / 4, d >> 1 & 1) + (d & 1);
    constexpr int kEach = DP / 16 < 8 ? DP / 16 : 8;
    const int part = d / (16 * kEach), rest = d % (16 * kEach), j = rest % kEach, i = rest / kEach % 4, g = rest / kEach / 4;
    return pair(piece, in / 16, (part * kEach + j) * 2 + i / 2, in % 16 + 16 * g) + (i & 1);
  }
};

// Writes of a piece go past the L2 of the XCD, to where all XCDs read: no write-back of a whole L2 has to follow them.
__device__ inline void write_through(float* to, float x, float y) {
  __hip_atomic_store(reinterpret_cast<uint64_t*>(to), __builtin_bit_cast(uint64_t, f2{x, y}), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// And they are read past the caches, which may hold what was there before.
__device__ inline f2 read_through(const float* from) {
  const uint64_t x = __hip_atomic_load(reinterpret_cast<const uint64_t*>(from), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return __builtin_bit_cast(f2, x);
}

// 2^(m - top) for a maximum that may be that of nothing
__device__ inline float behind(float m, float top) { return m == -INFINITY ? 0.f : exp2f(m - top); }

// The workgroup that comes last joins the pieces of its rows, in their order.  What the others wrote is there: every wavefront
// waits until its writes, which go through all caches, are done, then the workgroup counts itself.  (A release and an acquire
// instead would write back and drop a whole L2 each, 0.1 and 0.3 us for every workgroup, one after the other.)  Bound by the
// latency of these reads: a lane has eight pieces of its four values under way at once (sixteen were 1 us slower), and lanes that
// are left over take a share of the pieces.  Three to four microseconds for up to 26 pieces.
__device__ inline bool all_arrived(const Args& a, const Unit& u, uint32_t& arrived) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    arrived = __hip_atomic_fetch_add(&a.counters[u.counter], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (arrived == (uint32_t)u.pieces - 1) __hip_atomic_store(&a.counters[u.counter], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  return arrived == (uint32_t)u.pieces - 1;
}

// attend_split: a lane has four values of a row.
template <int THREADS> struct Joint {
  f4 part[THREADS];
  float m[THREADS], l[THREADS];
  uint32_t arrived;
};

template <typename CT, bool FLOAT, int DP, int ROWS, int THREADS> __device__ inline void join(const Args& a, const Unit& u, Joint<THREADS>& lds) {
  constexpr int kAtOnce = 8;
  if (!all_arrived(a, u, lds.arrived)) return;
  typedef Partial<DP, ROWS, true> P;
  const int tid = hidden(threadIdx.x), items = u.rows * (DP / 4), shares = items < THREADS ? THREADS / items : 1;
  for (int e0 = 0; e0 < items; e0 += THREADS) {
    const int share = shares > 1 ? tid / items : 0, e = e0 + tid - share * items, in = e / (DP / 4), d = e % (DP / 4) * 4;
    const bool there = e < items && d < a.dim && share < shares;
    f4 x{0, 0, 0, 0};
    float m = -INFINITY, l = 0.f;
    if (there) {
      for (int c0 = share; c0 < u.pieces; c0 += kAtOnce * shares) {
        f4 xc[kAtOnce];
        f2 mlc[kAtOnce];
        float top = m;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
          float* const piece = P::of(a, u.slot(min(c0 + k * shares, u.pieces - 1)));
          const f2 lo = read_through(P::fours(piece, e, 0)), hi = read_through(P::fours(piece, e, 1));
          xc[k] = f4{lo[0], lo[1], hi[0], hi[1]}, mlc[k] = read_through(P::sums(piece, in));
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
          if (c0 + k * shares >= u.pieces) mlc[k] = f2{-INFINITY, 0.f}, xc[k] = f4{0, 0, 0, 0};  // (0 times an infinite value is NaN)
          top = fmaxf(top, mlc[k][0]);
        }
        const float back = behind(m, top);
        x *= back, l = m == -INFINITY ? l : l * back;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
          const float w = behind(mlc[k][0], top);
          x += xc[k] * w, l += mlc[k][0] == -INFINITY ? mlc[k][1] : mlc[k][1] * w;  // (without a maximum: 0, or NaN)
        }
        m = top;
      }
    }
    if (shares > 1) {
      lds.part[tid] = x, lds.m[tid] = m, lds.l[tid] = l;
      __syncthreads();
      if (tid < items) {
        float top = m;
        for (int w = 1; w < shares; ++w) top = fmaxf(top, lds.m[w * items + tid]);
        const float back = behind(m, top);
        x *= back, l = m == -INFINITY ? l : l * back;
        for (int w = 1; w < shares; ++w) {
          const int at = w * items + tid;
          const float mw = lds.m[at], lw = lds.l[at], by = behind(mw, top);
          x += lds.part[at] * by, l += mw == -INFINITY ? lw : lw * by;
        }
      }
    }
    if (there && share == 0) store<CT, FLOAT>(a, u, in, d, x, l);
  }
}

// A value that is not finite must not reach the rows that do not see it, and a product would bring it there (0 times infinity is
// NaN).  In tiles of new tokens that some rows see in part it is taken out of the products, and added here, with whatever weight,
// to the rows that do see it: to what the workgroup has written of them, for the new tokens number j0 .. j1-1.
template <typename CT, bool FLOAT, int DP, int ROWS, bool SPLIT> __device__ inline void add_odd_values(const Args& a, const Unit& u, int threads) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  const int j0 = max(u.tile0 - u.cached, 0) * kTile, j1 = min((u.tile1 - u.cached) * kTile, u.q.fresh), quarters = a.dim / 4;
  for (int e = hidden(threadIdx.x); e < u.rows * quarters; e += threads) {
    const int in = e / quarters, d = (e - in * quarters) * 4, row = u.row0 + in, token = token_of(a, row);
    const uint64_t mask = a.mask ? a.mask[u.q.first + token] : 0;
    f4 add{0, 0, 0, 0};
    for (int j = j0; j < j1; ++j) {
      if (!(a.mask ? mask >> j & 1 : j <= token)) continue;
      const int64_t from = row_at(u.q.first + j, a.kv_stride) + u.head * a.dim + d;
      for (int i = 0; i < 4; ++i) {
        float x;
        if constexpr (FLOAT) x = (float)(CT)static_cast<const float*>(a.v)[from + i];
        else x = (float)static_cast<const CT*>(a.v)[from + i];
        if (!(fabsf(x) < INFINITY)) add[i] += x;
      }
    }
    if (u.pieces > 1) {
      for (int i = 0; i < 4; ++i) {
        float* const to = Partial<DP, ROWS, SPLIT>::value(Partial<DP, ROWS, SPLIT>::of(a, u.slot(u.piece)), in, d + i);
        const float x = __hip_atomic_load(to, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(to, x + add[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    } else {
      const int64_t to = row_at(u.q.first + token, a.out_stride) + (u.head * a.group + row - token * a.group) * a.dim + d;
      for (int i = 0; i < 4; ++i) {
        if constexpr (FLOAT) static_cast<float*>(a.out)[to + i] += add[i];
        else static_cast<CT*>(a.out)[to + i] = (CT)((float)static_cast<CT*>(a.out)[to + i] + add[i]);
      }
    }
  }
}

// ---- few rows: the wavefronts split the positions -----------------------------------------------------------
// A wavefront has the whole of its 16 rows' result in registers and reads each key and value of its positions once, as the operand
// itself: no LDS and no barrier between tiles, a tile of keys and one of values on their way while one is computed.  With enough
// tiles bound by memory (5.9 TB/s with 8192 cached tokens for each of 640 key heads, 5.4 with 65536 for each of 20), with few by
// the latencies behind each other: about 1.2 us until a workgroup knows its piece, 2 until the first keys are there, 1.2 to 1.6
// per tile, and the join.
template <typename CT, bool FLOAT, int DP, int WAVES, bool FULL>
__global__ void __launch_bounds__(64 * WAVES, 2) attend_split(Args a) {
  constexpr int kWaves = WAVES, kThreads = 64 * WAVES;
  typedef Rows<CT, FLOAT, DP> R;
  constexpr int kRows = 16, kSteps = R::kSteps, kEach = R::kEach, kParts = R::kParts, kTerms = R::kTerms;
  constexpr int kLine = DP + 4;  // floats between rows in LDS
  typedef Partial<DP, kRows, true> P;
  __shared__ float row_m[kWaves][kRows], row_l[kWaves][kRows], all_m[kRows], all_l[kRows];
  __shared__ __align__(16) float joined[kWaves][16][kLine];
  __shared__ __align__(16) u4 queries[FLOAT ? kSteps : 1][FLOAT ? kTerms : 1][64];  // the operands of floats fill too many registers
  __shared__ Joint<kThreads> joint;
  __shared__ uint32_t any_odd;  // a value that is not finite was taken out of a product
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Plan<kRows, true, FLOAT> plan(a, threadIdx.x & 63);

  const int group = group_index(plan.groups);
  if (group < 0) return;
  int64_t at_tile = plan.begin_of(group);
  const int64_t stop = plan.begin_of(group + 1);
  while (at_tile < stop) {
    const int tid = hidden(threadIdx.x), lane = tid & 63, n = lane & 15, g = lane >> 4;
    const Unit u = plan.next(a, at_tile, stop);
    if (tid == 0) any_odd = 0;
    __syncthreads();
    const int t0 = u.tile0 + (u.tile1 - u.tile0) * wave / kWaves, t1 = u.tile0 + (u.tile1 - u.tile0) * (wave + 1) / kWaves;
    R rows;
    u4 query[kSteps][kTerms];
    rows.begin(a, u, 0, n, g, query);
    if constexpr (FLOAT) {
      // (all wavefronts have the same rows, and write the same)
#pragma unroll
      for (int k = 0; k < kSteps; ++k)
#pragma unroll
        for (int t = 0; t < kTerms; ++t) queries[k][t][lane] = query[k][t];
      asm volatile("" ::: "memory");
    }
    u4 key[2][kSteps];
    uint32_t value[kParts][8][kEach / 2];
    auto scores = [&](f4 (&x)[2]) {
      x[0] = x[1] = f4{0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        if constexpr (FLOAT) {
          u4 q[kTerms];
#pragma unroll
          for (int t = 0; t < kTerms; ++t) q[t] = queries[k][t][lane];
          R::add_score(key[0][k], key[1][k], q, x);
        } else {
          R::add_score(key[0][k], key[1][k], query[k], x);
        }
      }
    };

    // The new tokens of the wavefront's first such tile are asked for now, a line per lane, and come from L2 when it is their turn.
    constexpr int kAsked = FLOAT ? 4 : 2;  // loads: keys and values, 64 dimensions of 16 bits or 32 floats in a line
    uint32_t asked[kAsked];
    if (t1 > u.cached) {
      const int j = min((max(t0, u.cached) - u.cached) * kTile + (lane >> 1), u.q.fresh - 1);
      const int64_t from = row_at(u.q.first + j, a.kv_stride) + u.head * a.dim;
#pragma unroll
      for (int i = 0; i < kAsked; ++i) {
        const int64_t at = from + min((lane & 1) * (FLOAT ? 32 : 64) + i / 2 * 64, a.dim - 2);
        asked[i] = *reinterpret_cast<const uint32_t*>(static_cast<const char*>(i & 1 ? a.v : a.k) + at * (FLOAT ? 4 : 2));
      }
    }

    // ---- cached tokens.  Loads run ahead by a tile, their pages by two; the last ones are loaded again instead of none,
    // so that the order of loads is the same in every turn and none waits for a later one.
    const int c1 = min(t1, u.cached);
    if (t0 < c1) {
      const int last_page = (u.q.held - 1) >> a.log2_page, in_page = (1 << a.log2_page) - 1;
      const int32_t* table = a.table + (int64_t)u.r * a.max_pages;
      const int key_at = 8 * (n >> 2), value_at = 8 * g;  // (eight positions from a multiple of eight lie on one page)
      auto page = [&](int tile, int at) { return table[min((tile * kTile + at) >> a.log2_page, last_page)]; };
      // a tile's first position on its page times the stride; the lane's own part is the same for all tiles
      auto row_of = [&](const uint16_t* cache, int tile, int page, uint32_t lane_part) {
        const uint16_t* p = cache + (int64_t)u.head * a.head_stride + (int64_t)((tile * kTile) & in_page) * a.token_stride;
        return p + (uint64_t)((uint32_t)page < (uint32_t)a.pages ? (uint32_t)page : 0u) * a.page_stride + lane_part;
      };
      const uint32_t key_lane = ((key_at & in_page) + (n & 3)) * a.token_stride, value_lane = (value_at & in_page) * a.token_stride;
      auto load_keys = [&](int tile, int page) {
        const uint16_t* p = row_of(a.cache_k, tile, page, key_lane);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int k = 0; k < kSteps; ++k) key[h][k] = *reinterpret_cast<const u4*>(p + 4 * h * a.token_stride + within<FULL>(a, 32 * k + 8 * g, 8));
      };
      auto load_values = [&](int tile, int page) {
        const uint16_t* p = row_of(a.cache_v, tile, page, value_lane);
#pragma unroll
        for (int part = 0; part < kParts; ++part)
#pragma unroll
          for (int t = 0; t < 8; ++t) {
            const uint16_t* from = p + t * a.token_stride + within<FULL>(a, part * 16 * kEach + kEach * n, kEach);
            if constexpr (kEach == 8) {
              const u4 x = *reinterpret_cast<const u4*>(from);
#pragma unroll
              for (int j = 0; j < 4; ++j) value[part][t][j] = x[j];
            } else {
              const u2 x = *reinterpret_cast<const u2*>(from);
              value[part][t][0] = x[0], value[part][t][1] = x[1];
            }
          }
        return (uint32_t)page < (uint32_t)a.pages ? eight_bits(u.q.held - tile * kTile - value_at) : 0;
      };
      int key_page = page(t0, key_at), value_page = page(t0, value_at);
      int next_key_page = page(min(t0 + 1, c1 - 1), key_at), next_value_page = page(min(t0 + 1, c1 - 1), value_at);
      load_keys(t0, key_page);
      int seen = load_values(t0, value_page);
      for (int tile = t0; tile < c1; ++tile) {
        f4 x[2];
        scores(x);
        key_page = next_key_page, value_page = next_value_page;
        next_key_page = page(min(tile + 2, c1 - 1), key_at), next_value_page = page(min(tile + 2, c1 - 1), value_at);
        load_keys(min(tile + 1, c1 - 1), key_page);
        float s[8];
        u4 p[kTerms];
        rows.exponents(x, s);
        if (__ballot(seen != 255)) {
#pragma unroll
          for (int t = 0; t < 8; ++t) s[t] = seen >> t & 1 ? s[t] : kUnseen;
#pragma unroll
          for (int part = 0; part < kParts; ++part) R::leave_out(value[part], ~seen);  // (what lies on a page behind the last token)
        }
        rows.weigh(s, p);
#pragma unroll
        for (int part = 0; part < kParts; ++part) rows.add_values(part, value[part], p);
        seen = load_values(min(tile + 1, c1 - 1), value_page);
      }
    }

    // ---- new tokens
    if (t1 > u.cached) {
#pragma unroll
      for (int i = 0; i < kAsked; ++i) asm volatile("" ::"v"(asked[i]));
    }
    for (int tile = max(t0, u.cached); tile < t1; ++tile) {
      const int j0 = (tile - u.cached) * kTile;
      const int in_row = u.head * a.dim;
      Eight<CT, FLOAT> e;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t from = row_at(u.q.first + min(j0 + 8 * (n >> 2) + (n & 3) + 4 * h, u.q.fresh - 1), a.kv_stride) + in_row;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          e.load(a.k, from + within<FULL>(a, 32 * k + 8 * g, 8));
          key[h][k] = e.rounded();
        }
      }
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        // (behind the last token the last one again: its values meet weights of 0)
        const int64_t from = row_at(u.q.first + min(j0 + 8 * g + t, u.q.fresh - 1), a.kv_stride) + in_row;
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
          const int d = within<FULL>(a, part * 16 * kEach + kEach * n, kEach);
          e.load(a.v, from + (d & ~7));  // (of eight dimensions the lane may take four)
          const u4 x = e.rounded();
#pragma unroll
          for (int j = 0; j < kEach / 2; ++j) value[part][t][j] = kEach == 4 && d & 4 ? x[2 + j] : x[j];
        }
      }
      f4 x[2];
      scores(x);
      float s[8];
      u4 p[kTerms];
      rows.exponents(x, s);
      const int seen = rows.seen_new(a, u, j0 + 8 * g);
      const bool partly = __ballot(seen != 255) != 0;
      if (partly) {
#pragma unroll
        for (int t = 0; t < 8; ++t) s[t] = seen >> t & 1 ? s[t] : kUnseen;
      }
      rows.weigh(s, p);
#pragma unroll
      for (int part = 0; part < kParts; ++part) {
        if (partly) {
          const uint32_t odd = R::odd_positions(value[part]);
          if (__ballot(odd)) {
            R::take_out(value[part], odd);
            any_odd = 1;
          }
        }
        rows.add_values(part, value[part], p);
      }
    }

    // ---- the wavefronts
    rows.finish();
    if (g == 0) row_m[wave][n] = rows.maximum(), row_l[wave][n] = rows.sum[0];
    __syncthreads();
    float top = row_m[0][n];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, row_m[w][n]);
    const float back = behind(rows.maximum(), top);
#pragma unroll
    for (int part = 0; part < kParts; ++part)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < kEach; j += 4)
          *reinterpret_cast<f4*>(&joined[wave][n][part * 16 * kEach + kEach * (4 * g + i) + j]) = rows.four(part, i, j) * back;
    if (wave == 0 && g == 0) {
      float total = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) total += row_m[w][n] == -INFINITY ? row_l[w][n] : row_l[w][n] * exp2f(row_m[w][n] - top);
      all_m[n] = top, all_l[n] = total;
    }
    __syncthreads();
    for (int e = tid; e < u.rows * (DP / 4); e += kThreads) {
      const int in = e / (DP / 4), d = e % (DP / 4) * 4;
      if (!FULL && d >= a.dim) continue;
      f4 x = *reinterpret_cast<const f4*>(&joined[0][in][d]);
#pragma unroll
      for (int w = 1; w < kWaves; ++w) x += *reinterpret_cast<const f4*>(&joined[w][in][d]);
      if (u.pieces == 1) {
        store<CT, FLOAT>(a, u, in, d, x, all_l[in]);
      } else {
        float* const piece = P::of(a, u.slot(u.piece));
        write_through(P::fours(piece, e, 0), x[0], x[1]);
        write_through(P::fours(piece, e, 1), x[2], x[3]);
        if (d == 0) write_through(P::sums(piece, in), all_m[in], all_l[in]);
      }
    }
    if (any_odd) add_odd_values<CT, FLOAT, DP, kRows, true>(a, u, kThreads);
    if (u.pieces > 1) join<CT, FLOAT, DP, kRows, kThreads>(a, u, joint);
    __syncthreads();
  }
}

// ---- many rows: the wavefronts share the positions ----------------------------------------------------------
// A tile is fetched by all wavefronts, a share each, as the 16 bytes that every lane will want of it (keys: fragment (h, k) of the
// lane; values: one position's eight dimensions), straight into LDS, where it lies in that order, a kilobyte per fragment without
// bank conflicts, and is read by all of them.  kAhead tiles are on their way while one is computed: the cache answers after one to
// two microseconds, a tile's products take a third of that. Counted with 4 requests of 64 tokens, four query heads per key head,
// over 131072 (0.47 to 0.49 ms with pages of 64): the matrix cores work a third of the time, vector instructions (the weights, and turning
// values) take two fifths, and between barriers all wavefronts want the same of the two at once; no bank conflicts.  Two tiles of rows
// of 128 dimensions spill 30 to 40 registers, with full heads and eight wavefronts none of them inside the loop over tiles, else one or
// two a tile; one reload there waits for all tiles that are on their way (4 x 64 over 131072: 700 us).  Float rows have two or three
// operands for each query and weight: 3 matrix instructions of bfloat16 where 16-bit rows have one, and 4 to 20 registers spilled, none
// inside the loop.  Chains of up to 512 tokens over up to 2048, 4 requests: 145 us, of which a large product would need 63 us for these
// (bfloat16 rows 79 us of 21); new float tokens are converted on their way to LDS, which nothing hides.
constexpr int kWindow = 512;  // entries of a request's table in LDS

// 16 bytes per lane from memory to the kilobyte of LDS at `to`, a place that nothing reads before wait_for_all_but has waited.  (The
// compiler is not told that LDS changes: every read of LDS would wait for all such loads.)
__device__ inline void to_lds(const void* from, uint32_t to) {
  uint32_t m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\ts_mov_b32 m0, %0"
               : "=&s"(m0)
               : "v"(from), "s"(__builtin_amdgcn_readfirstlane(to)));
}
// Until all but the last LOADS loads of the wavefront are done, and what it reads from and writes to LDS; then all wavefronts.
template <int LOADS> __device__ inline void wait_for_all_but() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LOADS) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// MT: tiles of 16 rows of a wavefront.
template <typename CT, bool FLOAT, int DP, int WAVES, int MT, bool FULL>
__global__ void __launch_bounds__(64 * WAVES, DP == 256 ? 1 : 2) attend_shared(Args a) {
  typedef Rows<CT, FLOAT, DP> R;
  constexpr int kSteps = R::kSteps, kEach = R::kEach, kParts = R::kParts, kTerms = R::kTerms;
  constexpr int kRows = 16 * MT * WAVES;
  constexpr int kKeys = 2 * kSteps, kValues = DP == 64 ? 4 : 8 * kParts;   // fragments of a tile
  constexpr int kFragments = kKeys + kValues, kMine = kFragments / WAVES;  // that a wavefront fetches
  // Eight wavefronts take two tiles between barriers: they lose less to each other (four, whose other workgroup fills in, lose
  // registers).
  constexpr int kBuffers = 4, kTogether = WAVES == 8 ? 2 : 1, kAhead = kBuffers - kTogether;
  constexpr bool kEarly = !(FLOAT && DP == 128);  // values are read from LDS while scores are worked out, where registers allow it
  static_assert(kFragments % WAVES == 0);
  struct Lds {
    u4 stage[kBuffers][kFragments][64];
    int32_t seen[kBuffers][4];  // which of eight positions there are
    int32_t pages[kWindow];
    uint32_t arrived;
    uint32_t any_odd;  // a value that is not finite was taken out of a product
  };
  __shared__ __align__(1024) Lds lds;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Plan<kRows, false, FLOAT> plan(a, threadIdx.x & 63);
  // The wavefronts of the first half fetch keys, the others values (there are as many of both).
  constexpr int kHalf = WAVES / 2;
  const bool keys = wave < kHalf;
  const int fragment0 = (keys ? wave : wave - kHalf) * kMine;

  const int group = group_index(plan.groups);
  if (group < 0) return;
  int64_t at_tile = plan.begin_of(group);
  const int64_t stop = plan.begin_of(group + 1);
  while (at_tile < stop) {
    const int tid = hidden(threadIdx.x), lane = tid & 63, n = lane & 15, g = lane >> 4;
    const Unit u = plan.next(a, at_tile, stop);
    // Fragment f of the keys: step f % kSteps of the 16 keys f / kSteps; of the values: part f % kParts of position f / kParts of the
    // lane's eight (heads of up to 64: positions 2 f and 2 f + 1, half a row of lanes each).
    const int at = keys ? 8 * (n >> 2) : 8 * g;  // eight positions that lie on one page
    auto position = [&](int f) { return keys ? (n & 3) + 4 * (f / kSteps) : kEach == 8 ? f / kParts : 2 * f + (n >> 3); };
    auto dimension = [&](int f) { return within<FULL>(a, keys ? 32 * (f % kSteps) + 8 * g : kEach == 8 ? 128 * (f % kParts) + 8 * n : 8 * (n & 7), 8); };
    R rows[MT];
    u4 query[MT][kSteps][kTerms];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      rows[mt].begin(a, u, 16 * (MT * wave + mt), n, g, query[mt]);
      // (in registers now: a wait for these loads inside the loop would be one for all tiles that are on their way)
#pragma unroll
      for (int k = 0; k < kSteps; ++k)
#pragma unroll
        for (int t = 0; t < kTerms; ++t) asm volatile("" : "+v"(query[mt][k][t]));
      asm volatile("" : "+v"(rows[mt].sees));
    }
    const bool idle = 16 * MT * wave >= u.rows;  // no rows: fetches only

    const int last_page = max(u.q.held - 1, 0) >> a.log2_page, in_page = (1 << a.log2_page) - 1, end = u.tile1, last = max(end - 1, 0);
    const int32_t* table = a.table + (int64_t)u.r * a.max_pages;
    const uint16_t* const cache = (keys ? a.cache_k : a.cache_v) + (int64_t)u.head * a.head_stride;
    const void* const fresh = keys ? a.k : a.v;
    const uint32_t lane_part = (at & in_page) * a.token_stride;
    int window = (min(u.tile0, last) * kTile) >> a.log2_page;  // the entry that pages[0] holds
    auto fill_window = [&] {
      for (int i = tid; i < kWindow; i += 64 * WAVES) lds.pages[i] = table[min(window + i, last_page)];
    };
    const uint32_t stage_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) u4*)&lds.stage[0][keys ? fragment0 : kKeys + fragment0][0];
    auto fetch = [&](int tile, int buffer) {
      const uint32_t to = stage_at + buffer * (kFragments * 1024);
      if (tile < u.cached) {
        const int page = lds.pages[min((tile * kTile + at) >> a.log2_page, last_page) - window];
        const bool there = (uint32_t)page < (uint32_t)a.pages;
        const uint16_t* p = cache + (int64_t)((tile * kTile) & in_page) * a.token_stride + (uint64_t)(there ? (uint32_t)page : 0u) * a.page_stride + lane_part;
#pragma unroll
        for (int i = 0; i < kMine; ++i) to_lds(p + position(fragment0 + i) * a.token_stride + dimension(fragment0 + i), to + i * 1024);
        if (wave == WAVES - 1 && n == 0) lds.seen[buffer][g] = there ? eight_bits(u.q.held - tile * kTile - at) : 0;
      } else {
        const int j0 = (tile - u.cached) * kTile + at;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
          const int64_t from = row_at(u.q.first + min(j0 + position(fragment0 + i), u.q.fresh - 1), a.kv_stride) + u.head * a.dim + dimension(fragment0 + i);
          if constexpr (FLOAT) {
            // (these loads the compiler waits for, and with them for all that were made before)
            Eight<CT, FLOAT> e;
            e.load(fresh, from);
            lds.stage[buffer][(keys ? 0 : kKeys) + fragment0 + i][lane] = e.rounded();
          } else {
            to_lds(static_cast<const uint16_t*>(fresh) + from, to + i * 1024);
          }
        }
        if (wave == WAVES - 1 && n == 0) lds.seen[buffer][g] = eight_bits(u.q.fresh - j0);
      }
    };
    // the values of part `part`, as R takes them
    auto read_values = [&](int buffer, int part, uint32_t (&value)[8][kEach / 2]) {
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        if constexpr (kEach == 8) {
          const u4 x = lds.stage[buffer][kKeys + t * kParts + part][lane];
#pragma unroll
          for (int j = 0; j < 4; ++j) value[t][j] = x[j];
        } else {
          const u2 x = reinterpret_cast<const u2*>(&lds.stage[buffer][kKeys + t / 2][16 * g + (t % 2) * 8 + (n >> 1)])[n & 1];
          value[t][0] = x[0], value[t][1] = x[1];
        }
      }
    };

    fill_window();
    if (tid == 0) lds.any_odd = 0;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // from here on only tiles are on their way
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kAhead; ++i) fetch(min(u.tile0 + i, last), i);  // (the last tile again instead of none: the count of loads stays)
    for (int first = u.tile0; first < end; first += kTogether) {
      wait_for_all_but<(kAhead - kTogether) * kMine>();  // these tiles are there, and all are done with those before
      const int next = min(first + kAhead, last);
      if (next < u.cached && ((min(next + kTogether, u.cached) * kTile - 1) >> a.log2_page) - window >= kWindow) {
        window = (next * kTile) >> a.log2_page;
        fill_window();
        __syncthreads();
      }
#pragma unroll
      for (int i = 0; i < kTogether; ++i) fetch(min(next + i, last), (first - u.tile0 + kAhead + i) % kBuffers);
      for (int tile = first; tile < min(first + kTogether, end) && !idle; ++tile) {
        const int buffer = (tile - u.tile0) % kBuffers;
        f4 x[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) x[mt][0] = x[mt][1] = f4{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          const u4 lo = lds.stage[buffer][k][lane], hi = lds.stage[buffer][kSteps + k][lane];
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) R::add_score(lo, hi, query[mt][k], x[mt]);
        }
        const bool is_new = tile >= u.cached;
        const int there = lds.seen[buffer][g];
        uint32_t value[8][kEach / 2];
        if constexpr (kEarly) read_values(buffer, 0, value);
        float s[MT][8];
        u4 p[MT][kTerms];
        bool whole = there == 255;
        int seen[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          rows[mt].exponents(x[mt], s[mt]);
          seen[mt] = is_new ? rows[mt].seen_new(a, u, (tile - u.cached) * kTile + 8 * g) : there;
          whole &= seen[mt] == 255;
        }
        const bool partly = __ballot(!whole) != 0;
        if (partly) {
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int t = 0; t < 8; ++t) s[mt][t] = seen[mt] >> t & 1 ? s[mt][t] : kUnseen;
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) rows[mt].weigh(s[mt], p[mt]);
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
          if (part || !kEarly) read_values(buffer, part, value);
          if (partly) {
            if (is_new) {
              const uint32_t odd = R::odd_positions(value);
              if (__ballot(odd)) {
                R::take_out(value, odd);
                lds.any_odd = 1;
              }
            } else {
              R::leave_out(value, ~there);  // (what lies on a page behind the last token)
            }
          }
#pragma unroll
          for (int j = 0; j < kEach; ++j) {
            const u4 v = R::column(value, j);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) rows[mt].add_column(part * kEach + j, v, p[mt]);
          }
        }
      }
    }
    wait_for_all_but<0>();
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) rows[mt].finish();

    auto store_rows = [&] {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const int in = 16 * (MT * wave + mt) + n;
        if (in >= u.rows) continue;
#pragma unroll
        for (int part = 0; part < kParts; ++part)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < kEach; j += 4) {
              const int d = part * 16 * kEach + kEach * (4 * g + i) + j;
              if (FULL || d < a.dim) store<CT, FLOAT>(a, u, in, d, rows[mt].four(part, i, j), rows[mt].sum[0]);
            }
      }
    };
    typedef Partial<DP, kRows, false> P;
    if (u.pieces == 1) {
      store_rows();
    } else if (!idle) {
      float* const piece = P::of(a, u.slot(u.piece));
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        if (g == 0) write_through(P::sums(piece, 16 * (MT * wave + mt) + n), rows[mt].maximum(), rows[mt].sum[0]);
#pragma unroll
        for (int r = 0; r < DP / 8; ++r) write_through(P::pair(piece, MT * wave + mt, r, lane), rows[mt].acc[r / 2][r % 2 * 2], rows[mt].acc[r / 2][r % 2 * 2 + 1]);
      }
    }
    if (lds.any_odd) add_odd_values<CT, FLOAT, DP, kRows, false>(a, u, 64 * WAVES);
    if (u.pieces > 1 && all_arrived(a, u, lds.arrived) && !idle) {
      // A lane takes up the pieces of the values that it has itself, several at once where registers allow it: bound by the
      // latency of these reads, and by what a CU can have under way.
      constexpr int kAtOnce = WAVES == 4 ? 2 : 1;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const int tile = MT * wave + mt;
        float m = -INFINITY, l = 0.f;
#pragma unroll
        for (int j = 0; j < kParts * kEach; ++j) rows[mt].acc[j] = f4{0, 0, 0, 0};
        for (int c0 = 0; c0 < u.pieces; c0 += kAtOnce) {
          f2 ml[kAtOnce], x[kAtOnce][DP / 8];
          float top = m;
#pragma unroll
          for (int c = 0; c < kAtOnce; ++c) {
            float* const from = P::of(a, u.slot(min(c0 + c, u.pieces - 1)));
            ml[c] = read_through(P::sums(from, 16 * tile + n));
#pragma unroll
            for (int r = 0; r < DP / 8; ++r) x[c][r] = read_through(P::pair(from, tile, r, lane));
          }
#pragma unroll
          for (int c = 0; c < kAtOnce; ++c) {
            if (c0 + c >= u.pieces) ml[c] = f2{-INFINITY, 0.f};
            top = fmaxf(top, ml[c][0]);
          }
          const float back = behind(m, top);
          l = m == -INFINITY ? l : l * back;
          m = top;
#pragma unroll
          for (int j = 0; j < kParts * kEach; ++j) rows[mt].acc[j] *= back;
#pragma unroll
          for (int c = 0; c < kAtOnce; ++c) {
            if (c0 + c >= u.pieces) break;  // (0 times an infinite value is NaN)
            const float by = behind(ml[c][0], top);
            l += ml[c][0] == -INFINITY ? ml[c][1] : ml[c][1] * by;  // (without a maximum: 0, or NaN)
#pragma unroll
            for (int r = 0; r < DP / 8; ++r)
#pragma unroll
              for (int i = 0; i < 2; ++i) rows[mt].acc[r / 2][r % 2 * 2 + i] += x[c][r][i] * by;
          }
        }
        rows[mt].sum[0] = l;
      }
      store_rows();
    }
    __syncthreads();
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

// The counters come first, at one place for calls of all shapes: what one leaves behind them no other takes for a count.
constexpr int kMostGroups = 512, kCountersBytes = kMostGroups * 4;
constexpr int64_t kMuch = 1 << 15;  // tiles of 64 rows: some 64 for each workgroup

// The kernel for a call, and how it is launched.
struct Shape {
  int dims;         // head_dim, padded
  bool shared;      // attend_shared
  int waves;        // of a workgroup
  int row_tiles;    // of a wavefront of attend_shared
  int rows;         // of a workgroup
  int target;       // workgroups at most: those that the chip runs at once
  int64_t bytes;    // of the workspace

  // of a workspace with room for so many workgroups' pieces
  int64_t bytes_for(int groups) const { return kCountersBytes + (int64_t)2 * groups * rows * (dims + 2) * 4; }
};

// of a request: as many as its row of the table can name, and the new ones
int64_t most_tiles(const rsr_cache_t* cache, const rsr_step_t* step) {
  return ((int64_t)step->max_pages * cache->page_size + kTile - 1) / kTile + (step->max_new + kTile - 1) / kTile;
}

// The kernels multiply the tiles of all sets (of 16 rows at least) by the number of a workgroup in floating point, exactly below
// 2^51.
constexpr char kTooMany[] = "the tables could name more tokens than the kernels count";
bool can_be_counted(const rsr_cache_t* cache, const rsr_step_t* step, int heads) {
  const int64_t blocks = ((int64_t)step->max_new * (heads / cache->kv_heads) + 15) / 16;
  return (double)step->requests * cache->kv_heads * blocks * most_tiles(cache, step) < 0x1p42;
}

Shape shape_of(const rsr_cache_t* cache, const rsr_step_t* step, int heads, bool floats) {
  Shape s;
  s.dims = cache->head_dim <= 64 ? 64 : cache->head_dim <= 128 ? 128 : 256;
  const int64_t rows = (int64_t)step->max_new * (heads / cache->kv_heads);
  // (keys and values of 256 dimensions do not fit in the registers beside a result, nor do two tiles of rows of that many, or of
  // float)
  s.shared = rows > 16 || s.dims == 256;
  const int64_t sets = (int64_t)step->requests * cache->kv_heads, tiles = most_tiles(cache, step);
  // attend_shared: workgroups of 64 rows; with much work of 128, or, where there are as many, 256, two tiles of rows per
  // wavefront.  A fragment is then read from LDS once for both and a tile fetched once for all, but there are fewer workgroups for
  // a set's rows, and more to join for each.  (256 rows per key head: 4 x 131072 cached tokens 0.54 ms, with 64 rows 0.72; 8 x
  // 8000 89 us against 106; 8 x 4000 61 against 60; 2000 41 against 22; a chain of 512 over 2048 48 against 42.  128 rows: 4 x 131072
  // 352 us against 435, 8 x 16000 114 against 107.)  The work is what the tables could name: the host knows no lengths, and a table for 131072
  // tokens takes the 41 us where 2000 are held.
  const bool much = s.shared && !floats && s.dims < 256 && rows > 64 && sets * ((rows + 63) / 64) * tiles >= kMuch;
  s.row_tiles = much ? 2 : 1;
  // attend_split: four wavefronts, of which two workgroups per CU hide each other's waits.  Eight, one workgroup per CU, where few
  // sets have so many tiles that they are cut into more pieces than there are CUs: half as many to join (20 heads of 128, 16
  // tokens: 41 against 50 us over 16384 cached ones, but 19.1 against 17.5 us over 4096).
  if (s.shared) s.waves = much && rows > 128 ? 8 : 4;
  else s.waves = sets < 128 && sets * tiles > kMostGroups / 2 * kLeastTiles ? 8 : 4;
  s.rows = s.shared ? 16 * s.waves * s.row_tiles : 16;
  // two workgroups of four wavefronts per CU, one of eight (their LDS and registers allow no more)
  s.target = s.waves == 4 && s.dims < 256 ? kMostGroups : kMostGroups / 2;
  s.bytes = s.bytes_for(s.target);
  return s;
}

template <typename CT, bool FLOAT, bool FULL> void (*kernel_of(const Shape& s))(Args) {
  if (s.dims == 256) return attend_shared<CT, FLOAT, 256, 4, 1, FULL>;
  if (!s.shared) {
    if (s.waves == 8) return s.dims == 64 ? attend_split<CT, FLOAT, 64, 8, FULL> : attend_split<CT, FLOAT, 128, 8, FULL>;
    return s.dims == 64 ? attend_split<CT, FLOAT, 64, 4, FULL> : attend_split<CT, FLOAT, 128, 4, FULL>;
  }
  if constexpr (!FLOAT) {
    if (s.row_tiles == 2) {
      if (s.dims == 64) return s.waves == 4 ? attend_shared<CT, FLOAT, 64, 4, 2, FULL> : attend_shared<CT, FLOAT, 64, 8, 2, FULL>;
      return s.waves == 4 ? attend_shared<CT, FLOAT, 128, 4, 2, FULL> : attend_shared<CT, FLOAT, 128, 8, 2, FULL>;
    }
  }
  return s.dims == 64 ? attend_shared<CT, FLOAT, 64, 4, 1, FULL> : attend_shared<CT, FLOAT, 128, 4, 1, FULL>;
}

template <typename CT> void (*kernel_of(const Shape& s, bool floats, bool full))(Args) {
  if (floats) return full ? kernel_of<CT, true, true>(s) : kernel_of<CT, true, false>(s);
  return full ? kernel_of<CT, false, true>(s) : kernel_of<CT, false, false>(s);
}

}  // namespace

extern "C" {

int64_t rsr_tree_attention_workspace(const rsr_cache_t* cache, const rsr_step_t* step, int heads) {
  if (const char* fault = fault_of(cache, step, heads)) return set_error(RSR_ERR_INVALID_ARGUMENT, fault);
  if (!can_be_counted(cache, step, heads)) return set_error(RSR_ERR_UNSUPPORTED, kTooMany);
  // Not less for more work, so that a workspace for a program's largest step does for all: attend_split with eight wavefronts itself needs
  // half as much as with four.
  int64_t bytes = 0;
  for (const bool floats : {false, true}) {
    const Shape s = shape_of(cache, step, heads, floats);
    bytes = std::max(bytes, s.shared ? s.bytes : s.bytes_for(kMostGroups));
  }
  return bytes;
}

int rsr_tree_attention(const rsr_cache_t* cache, const rsr_step_t* step, const void* q, int64_t q_stride, const void* k, const void* v,
                       int64_t kv_stride, void* out, int64_t out_stride, int dtype, int heads, float scale, void* workspace, int64_t workspace_bytes,
                       void* stream) {
  const char* fault = fault_of(cache, step, heads);
  if (!fault && dtype != RSR_F32 && dtype != cache->dtype) fault = "dtype must be RSR_F32 or the cache's";
  if (!fault && !std::isfinite(scale)) fault = "scale must be finite";
  if (fault) return set_error(RSR_ERR_INVALID_ARGUMENT, fault);
  if (step->requests == 0 || step->tokens == 0) return RSR_OK;
  if (!can_be_counted(cache, step, heads)) return set_error(RSR_ERR_UNSUPPORTED, kTooMany);
  const int64_t width = (int64_t)heads * cache->head_dim, kv_width = (int64_t)cache->kv_heads * cache->head_dim;
  const bool floats = dtype == RSR_F32;
  const Shape s = shape_of(cache, step, heads, floats);
  fault = rsr_internal::fault_of_rows(q, q_stride, width, dtype);
  if (!fault) fault = rsr_internal::fault_of_rows(k, kv_stride, kv_width, dtype);
  if (!fault) fault = rsr_internal::fault_of_rows(v, kv_stride, kv_width, dtype);
  if (!fault) fault = rsr_internal::fault_of_rows(out, out_stride, width, dtype);
  if (!fault && (q_stride >> 31 || kv_stride >> 31 || out_stride >> 31)) fault = "strides must be below 2^31";
  if (!fault && (!workspace || !rsr_internal::aligned(workspace, 256) || workspace_bytes < s.bytes))
    fault = "the workspace is missing, too small or not 256-byte aligned";
  if (fault) return set_error(RSR_ERR_INVALID_ARGUMENT, fault);
  const int group = heads / cache->kv_heads;
  const Args a{q, k, v, out, static_cast<const uint16_t*>(cache->k), static_cast<const uint16_t*>(cache->v), step->table, step->held, step->start, step->mask,
               static_cast<uint32_t*>(workspace), reinterpret_cast<float*>(static_cast<char*>(workspace) + kCountersBytes),
               cache->head_stride, (uint32_t)q_stride, (uint32_t)kv_stride, (uint32_t)out_stride, (uint32_t)cache->page_stride,
               (uint32_t)cache->token_stride, step->requests, step->tokens,
               step->max_new, step->max_pages, rsr_internal::log2_of(cache->page_size), cache->pages, cache->kv_heads, cache->head_dim, group,
               group == 1 ? 0u : (uint32_t)(((uint64_t(1) << 32) + group - 1) / group), scale};
  const bool full = cache->head_dim == s.dims;
  auto kern = cache->dtype == RSR_F16 ? kernel_of<_Float16>(s, floats, full) : kernel_of<__bf16>(s, floats, full);
  // no more workgroups than there can be pieces
  const int64_t blocks = ((int64_t)step->max_new * group + s.rows - 1) / s.rows;
  const int64_t least = s.shared ? kLeastShared : kLeastTiles, pieces = (most_tiles(cache, step) + least - 1) / least;
  const int64_t most = std::min((int64_t)s.target, (step->requests * cache->kv_heads * blocks * pieces + 7) / 8 * 8);
  hipLaunchKernelGGL(kern, dim3((unsigned)most), dim3(64 * s.waves), 0, static_cast<hipStream_t>(stream), a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(RSR_ERR_HIP, std::string("rsr_tree_attention: ") + hipGetErrorString(e));
  return RSR_OK;
}

}  // extern "C"
