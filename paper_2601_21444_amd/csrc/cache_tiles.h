// The cache's keys as the attention kernels see them (device code): requests, the axis that all their tiles lie on, and the
// 16-key blocks of a tile.
#pragma once
#include "attention_tiles.h"
#include "cache.h"

namespace apbv {
namespace {

#define APBV_CONST(T) const __attribute__((address_space(4))) T*     // read through the scalar cache
__device__ __forceinline__ int scalar_load(const int32_t* p, int64_t i) { return ((APBV_CONST(int32_t))p)[i]; }

// The query that a row (query x head of the group, below 2^30) is of.  (row + 1/2) / group is no nearer to a whole number than 1 /
// (2 group), the double's error is below 2^-20: three instructions where the division of integers has twenty.
__device__ __forceinline__ int query_of(const CacheAttnParams& p, int row) { return (int)(((double)row + 0.5) * p.per_group); }

struct Request {
  int first, rows, len;      // first query, rows (query x head of the group), keys
  int tiles;                 // 64-key tiles of each of its row tiles; 0: none
};

__device__ __forceinline__ int clip(int x, int hi) { return x < 0 ? 0 : (x > hi ? hi : x); }
__device__ __forceinline__ Request request_of(const CacheAttnParams& p, int first, int past, int len) {
  Request r;
  r.first = clip(first, p.n_rows);
  past = clip(past, p.n_rows);
  r.rows = (past > r.first ? past - r.first : 0) * p.group;
  r.len = clip(len, p.max_len);
  r.tiles = r.rows > 0 ? (r.len + kCacheKeyTile - 1) / kCacheKeyTile : 0;
  return r;
}
// Inclusive sums over the lanes of a wave, on the DPP path.
__device__ __forceinline__ uint32_t add_sat(uint32_t x, uint32_t y) { return __builtin_elementwise_add_sat(x, y); }
template <int kCtrl, int kRows>
__device__ __forceinline__ uint32_t dpp_add(uint32_t x) {
  return add_sat(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kCtrl, kRows, 0xf, false));
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  x = dpp_add<0x111, 0xf>(x);      // row_shr 1, 2, 4, 8: within sixteen lanes
  x = dpp_add<0x112, 0xf>(x);
  x = dpp_add<0x114, 0xf>(x);
  x = dpp_add<0x118, 0xf>(x);
  x = dpp_add<0x142, 0xa>(x);      // row_bcast 15: lane 15 to the second sixteen, lane 47 to the fourth
  x = dpp_add<0x143, 0xc>(x);      // row_bcast 31: lane 31 to the upper half
  return x;
}

// Natural logarithm of l * 2^m: the result is held to what float32 holds, whatever the sizes of m and l.
__device__ __forceinline__ float log_sum(float m, float l) {
  if (!(l > 0.f)) return -INFINITY;
  const double x = (double)m + (double)__builtin_amdgcn_frexp_expf(l) + (double)__builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(l));
  return (float)(x * 0.69314718055994530942);
}
// Statistics of the parts of a workgroup that begin a row tile (slot 1) or go on with one (slot 0): maxima, sums, exact sums.
__device__ __forceinline__ float* part_stats(const CacheAttnParams& p, int slot, int R, int D) {
  return p.parts + (int64_t)p.workgroups * 2 * (R * D) + (int64_t)slot * (3 * R) * p.workgroups;
}

// The axis of tiles: its length, and where the requests lie on it.  A wave holds a window of 64 consecutive requests, one a
// lane, handed from lane to lane as they are needed; with more than 64 it first adds up 64 groups of `per` (at most 64).
// The host has seen that the tiles of requests which do not overlap fit 32 bits; sums stop at the largest number otherwise.
template <int R>
struct Axis {
  uint32_t total;
  int base;                  // the window: request base + lane is `mine`
  uint32_t base_begin;       // where the window begins on the axis
  Request mine;
  uint32_t past;             // where `mine` ends
  int per, group_first;      // this lane's group: its first query row (RowsOnly) ...
  uint32_t group_past;       // ... and where it ends

  __device__ __forceinline__ static uint32_t top(uint32_t x) { return x < 0x7fff0000u ? x : 0x7fff0000u; }
  __device__ __forceinline__ static uint32_t tiles(const CacheAttnParams& p, const Request& r) {
    return (uint32_t)((r.rows + R - 1) / R * p.hkv) * (uint32_t)r.tiles;
  }
  __device__ __forceinline__ static Request load(const CacheAttnParams& p, int b) {
    const int first = p.starts ? p.starts[b] : b * p.each, past_row = p.starts ? p.starts[b + 1] : (b + 1) * p.each;
    return request_of(p, first, past_row, p.lengths[b]);
  }
  __device__ __forceinline__ void window(const CacheAttnParams& p, int from, uint32_t begin) {
    base = from;
    base_begin = begin;
    mine = Request{0x7fffffff, 0, 0, 0};
    const int b = from + (int)(threadIdx.x & 63);
    if (b < p.n_requests) mine = load(p, b);
    past = add_sat(begin, wave_scan(tiles(p, mine)));
  }
  __device__ __forceinline__ Axis(const CacheAttnParams& p) {
    if (p.n_requests <= 64) {
      window(p, 0, 0);
      total = top(__builtin_amdgcn_readlane(past, 63));
      return;
    }
    const int lane = threadIdx.x & 63;
    per = (p.n_requests + 63) / 64;
    uint32_t sum = 0;
    for (int u = 0; u < per; u += 4) {
      Request r[4];
#pragma unroll
      for (int v = 0; v < 4; ++v) {                        // (four at a time on their way)
        const int b = lane * per + u + v;
        r[v] = load(p, b < p.n_requests ? b : p.n_requests - 1);
        if (u + v >= per || b >= p.n_requests) r[v].rows = 0;
      }
#pragma unroll
      for (int v = 0; v < 4; ++v) sum = add_sat(sum, tiles(p, r[v]));
    }
    group_past = wave_scan(sum);
    total = top(__builtin_amdgcn_readlane(group_past, 63));
  }
  // Of the rows alone, for find_row: whoever takes a request's first tile leaves word of where it begins.
  struct RowsOnly {};
  __device__ __forceinline__ Axis(const CacheAttnParams& p, RowsOnly) {
    if (p.n_requests <= 64) {
      window(p, 0, 0);
      total = top(__builtin_amdgcn_readlane(past, 63));
      return;
    }
    per = (p.n_requests + 63) / 64;
    const int b = (int)(threadIdx.x & 63) * per;
    group_first = 0x7fffffff;
    if (b < p.n_requests) group_first = clip(p.starts ? p.starts[b] : b * p.each, p.n_rows);
    group_past = 0;
  }
  __device__ __forceinline__ void leave_word(const CacheAttnParams& p, int b, uint32_t begin, uint32_t share) const {
    if (p.n_requests > 64 && (threadIdx.x & 63) == 0) {
      p.begins[1 + b] = begin;
      if (begin == 0) p.begins[0] = share;
    }
  }
  __device__ __forceinline__ void group_window(const CacheAttnParams& p, int group) {
    window(p, group * per, group > 0 ? __builtin_amdgcn_readlane(group_past, group - 1) : 0);
  }
  __device__ __forceinline__ uint32_t begin_of(int b) const {                   // b of the window
    return b > base ? __builtin_amdgcn_readlane(past, b - base - 1) : base_begin;
  }
  __device__ __forceinline__ Request at(const CacheAttnParams& p, int b) {     // b uniform
    if ((unsigned)(b - base) >= 64u) window(p, b, 0);      // (a walk that leaves the window knows where it is)
    Request r;
    r.first = __builtin_amdgcn_readlane(mine.first, b - base);
    r.rows = __builtin_amdgcn_readlane(mine.rows, b - base);
    r.len = __builtin_amdgcn_readlane(mine.len, b - base);
    r.tiles = __builtin_amdgcn_readlane(mine.tiles, b - base);
    return r;
  }
  // Length of a workgroup's share.
  __device__ __forceinline__ uint32_t share(const CacheAttnParams& p) const {
    return cache_share(total, (uint32_t)p.workgroups, (uint32_t)p.short_tiles, (uint32_t)p.least_tiles, (uint32_t)p.share_step);
  }
  // The share of this workgroup, or -1: consecutive shares on one XCD (row tiles of a head read the same keys), which a launch
  // gives its workgroups in turn.
  __device__ __forceinline__ int my_share(uint32_t share) const {
    const int n = (int)((total + share - 1) / share), per_xcd = (n + kXcds - 1) / kXcds;
    const int x = (int)blockIdx.x / kXcds, wg = (int)(blockIdx.x % kXcds) * per_xcd + x;
    return x < per_xcd && wg < n ? wg : -1;
  }
  // The request that holds tile `pos` < total.
  __device__ __forceinline__ int find(const CacheAttnParams& p, uint32_t pos) {
    if (p.n_requests > 64) group_window(p, __builtin_ctzll(__builtin_amdgcn_ballot_w64(group_past > pos)));
    return base + __builtin_ctzll(__builtin_amdgcn_ballot_w64(past > pos));
  }
  // The last request that begins at or before this query row (the first one if there is none).
  __device__ __forceinline__ int find_row(const CacheAttnParams& p, int row) {
    if (p.n_requests > 64) {
      const uint64_t before = __builtin_amdgcn_ballot_w64(group_first <= row);
      group_window(p, before ? 63 - __builtin_clzll(before) : 0);
    }
    const uint64_t before = __builtin_amdgcn_ballot_w64(mine.first <= row);
    return base + (before ? 63 - __builtin_clzll(before) : 0);
  }
};

// A 16-key block's codes (16 bytes a lane at head_dim 128, 8 at 64) and scale byte.
template <int D>
struct Codes {
  static constexpr int kWords = D / 32;
  uint32_t w[kWords];
  uint32_t scale;
  // uniform bases, and how far behind them the block lies; this lane's key li of it, quarter lg
  __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* scales, int code_step, int scale_step, int li, int lg) {
    if constexpr (D == 128) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(codes + (uint32_t)(li * 64 + lg * 16) + code_step);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = x[i];
      scale = scales[(uint32_t)(li * 4 + lg) + scale_step];
    } else {
      const u32x2 x = *reinterpret_cast<const u32x2*>(codes + (uint32_t)(li * 32 + lg * 8) + code_step);
      w[0] = x[0];
      w[1] = x[1];
      scale = scales[(uint32_t)(li * 2 + (lg >> 1)) + scale_step];
    }
  }
  // eight elements as bf16
  __device__ __forceinline__ u32x4 values(int i) const {
    const float s = __uint_as_float(scale << 23);
    u32x4 x;
    x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], s, 0));
    x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], s, 1));
    x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], s, 2));
    x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], s, 3));
    return x;
  }
};

// Where the four 16-key blocks of a tile lie, as byte offsets into the codes and the scales of K and of V, and which blocks are
// not there.  A page of 64 tokens or more holds a whole tile: one lookup, uniform, and the blocks follow one another.
template <int D, bool kOnePage>
struct Blocks {
  int64_t codes, scales;
  int absent;                // the page is out of range, or no key of the request lies in it
  __device__ __forceinline__ void find(const CacheAttnParams& p, const int32_t* table_row, int head, int len, int tile) {
    const int token = tile * kCacheKeyTile, at = token < len ? token : len - 1;      // (a table entry that the request has)
    const int page = scalar_load(table_row, at >> p.cache.page_log2);
    const bool there = token < len && (unsigned)page < (unsigned)p.cache.n_pages;
    absent = there ? 0 : 1;
    const int pg = there ? page : 0;
    const int row = (head << p.cache.page_log2) + (token & ((1 << p.cache.page_log2) - 1));
    codes = (int64_t)((uint64_t)(uint32_t)pg * (uint32_t)p.cache.stride_codes) + (uint32_t)row * (uint32_t)(D / 2);
    scales = (int64_t)((uint64_t)(uint32_t)pg * (uint32_t)p.cache.stride_scales) + (uint32_t)row * (uint32_t)(D / 32);
  }
  __device__ __forceinline__ bool gone(int) const { return absent != 0; }
  // this lane's pieces of the four blocks of K or of V
  __device__ __forceinline__ void load(Codes<D> (&x)[4], const uint8_t* code_base, const uint8_t* scale_base, int li, int lg) const {
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) x[kb].load(code_base + codes, scale_base + scales, kb * 16 * (D / 2), kb * 16 * (D / 32), li, lg);
  }
};
// Smaller pages: lane n of every four has the n-th block's place, and looks its page up a tile before it is needed (us, four times
// in scalar instructions / so: one query over 700 keys, 2 / 1 heads of 64, pages of 16 7.5 / 6.7; 256 requests of 65 to 2048 keys,
// 8 / 2 heads of 64, pages of 32 15.4 / 14.7).
template <int D>
struct Blocks<D, false> {
  int64_t codes, scales;
  int absent;                // bit i: of block i, uniform
  __device__ __forceinline__ static int token_of(int tile) { return tile * kCacheKeyTile + 16 * (int)(threadIdx.x & 3); }
  __device__ __forceinline__ static int look_up(const CacheAttnParams& p, const int32_t* table_row, int len, int tile) {
    const int token = token_of(tile);
    return table_row[(token < len ? token : len - 1) >> p.cache.page_log2];
  }
  __device__ __forceinline__ void place(const CacheAttnParams& p, int head, int len, int tile, int page) {
    const int token = token_of(tile);
    const bool there = token < len && (unsigned)page < (unsigned)p.cache.n_pages;
    absent = (int)(~__builtin_amdgcn_ballot_w64(there) & 15);
    const int pg = there ? page : 0;
    const int row = (head << p.cache.page_log2) + (token & ((1 << p.cache.page_log2) - 1));
    codes = (int64_t)((uint64_t)(uint32_t)pg * (uint32_t)p.cache.stride_codes) + (uint32_t)row * (uint32_t)(D / 2);
    scales = (int64_t)((uint64_t)(uint32_t)pg * (uint32_t)p.cache.stride_scales) + (uint32_t)row * (uint32_t)(D / 32);
  }
  __device__ __forceinline__ bool gone(int kb) const { return (absent >> kb & 1) != 0; }
  __device__ __forceinline__ static int64_t of_block(int64_t x, int kb) {
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)x, kb), hi = __builtin_amdgcn_readlane((uint32_t)((uint64_t)x >> 32), kb);
    return (int64_t)((uint64_t)hi << 32 | lo);
  }
  __device__ __forceinline__ void load(Codes<D> (&x)[4], const uint8_t* code_base, const uint8_t* scale_base, int li, int lg) const {
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) x[kb].load(code_base + of_block(codes, kb), scale_base + of_block(scales, kb), 0, 0, li, lg);
  }
};

}  // namespace
}  // namespace apbv
