// Attention over the key/value cache held in 4 bits (include/apbv_cache.h), for gfx950.
//
// Rows.  As in query_attention.hip the G query heads of a KV head are G rows of one problem: row r = i * G + g of a request is
// its query i of head kvh * G + g.  A row tile is 16 or 32 of them.
//
// Cut.  Only the device knows the lengths.  Every workgroup adds up the requests' tiles (a wave's lanes take a request each)
// and takes an equal share of the axis that all (request, KV head, row tile) lie on one after the other, 64 keys a tile, and
// every wave an equal part of that: a batch of unequal lengths fills the chip as an equal one does, and so does one request.
// A wave finishes the row tiles that lie in its part by itself; the pieces of others are put together in LDS at the end, and
// what a workgroup shares with its neighbours is left in the workspace in float32 (O, maxima, row sums), where a second launch
// joins it.  (All waves on one row tile at a time: 256 requests of 65 to 2048 keys 24.2 us instead of 16.9, 64 requests of 512 to
// 32768 53.7 instead of 47.8, one of 133120 14.4 instead of 14.8.)
//
// Keys.  A lane of the matrix instruction's A operand needs eight elements of one key, and which elements go with which k-step
// is free as long as K and Q agree: lane (key li, quarter lg) takes the quarter's 16 bytes of codes, one load, all of one
// scale block, and converts eight of them a k-step.  No LDS.  V is needed transposed: a lane converts its quarter of a key's
// row, writes it to the wave's own LDS tile as bf16, and the transposing LDS read does the rest.
#include "attention_tiles.h"
#include "cache.h"

namespace apbv {
namespace {

#define APBV_CONST(T) const __attribute__((address_space(4))) T*     // read through the scalar cache
__device__ __forceinline__ int scalar_load(const int32_t* p, int64_t i) { return ((APBV_CONST(int32_t))p)[i]; }

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
__device__ __forceinline__ int64_t readlane64(int64_t x, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)x, lane), hi = __builtin_amdgcn_readlane((uint32_t)((uint64_t)x >> 32), lane);
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

// x / y for 0 <= x, 0 < y; almost always within 32 bits, where it takes a fifth of the instructions.
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t y) {
  if (((uint64_t)x | (uint64_t)y) >> 32 == 0) return (int64_t)((uint32_t)x / (uint32_t)y);
  return x / y;
}

// Inclusive sums over the lanes of a wave, on the DPP path.
template <int kCtrl, int kRows>
__device__ __forceinline__ int64_t dpp64(int64_t x) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, kCtrl, kRows, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)((uint64_t)x >> 32), kCtrl, kRows, 0xf, false);
  return (int64_t)(((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ int64_t wave_scan(int64_t x) {
  x += dpp64<0x111, 0xf>(x);      // row_shr 1, 2, 4, 8: within sixteen lanes
  x += dpp64<0x112, 0xf>(x);
  x += dpp64<0x114, 0xf>(x);
  x += dpp64<0x118, 0xf>(x);
  x += dpp64<0x142, 0xa>(x);      // row_bcast 15: lane 15 to the second sixteen, lane 47 to the fourth
  x += dpp64<0x143, 0xc>(x);      // row_bcast 31: lane 31 to the upper half
  return x;
}

// The axis of tiles: its length, and where the requests lie on it.  A wave holds a window of 64 consecutive requests, one a
// lane, handed from lane to lane as they are needed; with more than 64 it first adds up 64 groups of `per` (at most 64).
template <int R>
struct Axis {
  int64_t total;
  int base;                  // the window: request base + lane is `mine`
  int64_t base_begin;        // where the window begins on the axis
  Request mine;
  int64_t past;              // where `mine` ends
  int per, group_first;      // this lane's group: its first query row ...
  int64_t group_past;        // ... and where it ends

  __device__ __forceinline__ static int64_t tiles(const CacheAttnParams& p, const Request& r) {
    return (int64_t)((r.rows + R - 1) / R) * p.hkv * r.tiles;
  }
  __device__ __forceinline__ static Request load(const CacheAttnParams& p, int b) {
    const int first = p.starts ? p.starts[b] : b * p.each, past_row = p.starts ? p.starts[b + 1] : (b + 1) * p.each;
    return request_of(p, first, past_row, p.lengths[b]);
  }
  __device__ __forceinline__ void window(const CacheAttnParams& p, int from, int64_t begin) {
    base = from;
    base_begin = begin;
    mine = Request{0x7fffffff, 0, 0, 0};
    const int b = from + (int)(threadIdx.x & 63);
    if (b < p.n_requests) mine = load(p, b);
    past = begin + wave_scan(tiles(p, mine));
  }
  __device__ __forceinline__ Axis(const CacheAttnParams& p) {
    if (p.n_requests <= 64) {
      window(p, 0, 0);
      total = readlane64(past, 63);
      return;
    }
    const int lane = threadIdx.x & 63;
    per = (p.n_requests + 63) / 64;
    group_first = 0x7fffffff;
    int64_t sum = 0;
    for (int u = 0; u < per; u += 4) {
      Request r[4];
#pragma unroll
      for (int v = 0; v < 4; ++v) {                        // (four at a time on their way)
        const int b = lane * per + u + v;
        r[v] = load(p, b < p.n_requests ? b : p.n_requests - 1);
        if (u + v >= per || b >= p.n_requests) r[v].rows = 0;
        else if (u + v == 0) group_first = r[v].first;
      }
#pragma unroll
      for (int v = 0; v < 4; ++v) sum += tiles(p, r[v]);
    }
    group_past = wave_scan(sum);
    total = readlane64(group_past, 63);
  }
  __device__ __forceinline__ void group_window(const CacheAttnParams& p, int group) {
    window(p, group * per, group > 0 ? readlane64(group_past, group - 1) : 0);
  }
  __device__ __forceinline__ int64_t begin_of(int b) const {                   // b of the window
    return b > base ? readlane64(past, b - base - 1) : base_begin;
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
  __device__ __forceinline__ int64_t share(const CacheAttnParams& p) const {
    const int64_t q = quotient(total + p.workgroups - 1, p.workgroups);
    return q > p.least_tiles ? q : p.least_tiles;
  }
  // The request that holds tile `pos` < total.
  __device__ __forceinline__ int find(const CacheAttnParams& p, int64_t pos) {
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

enum : int { kHead = 1, kTail = 2, kSpan = 4 };            // what a wave keeps of row tiles that are not its own alone

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

// Where the four 16-key blocks of a tile lie (uniform), as byte offsets into the codes and the scales of K and of V, and which
// blocks are not there.  A page of 64 tokens or more holds a whole tile: one lookup, and the blocks follow one another.
template <int D, bool kOnePage>
struct Blocks {
  static constexpr int kLookups = kOnePage ? 1 : 4;
  int64_t codes[kLookups], scales[kLookups];
  int absent;                // bit i: the page of lookup i is out of range, or no key of the request lies in it
  __device__ __forceinline__ void find(const CacheAttnParams& p, const int32_t* table_row, int head, int len, int tile) {
    absent = 0;
#pragma unroll
    for (int i = 0; i < kLookups; ++i) {
      const int token = tile * kCacheKeyTile + 16 * i;
      const int at = token < len ? token : len - 1;                      // (a table entry that the request has)
      const int page = scalar_load(table_row, at >> p.cache.page_log2);
      const bool there = token < len && (unsigned)page < (unsigned)p.cache.n_pages;
      absent |= there ? 0 : 1 << i;
      const int pg = there ? page : 0;
      const int row = (head << p.cache.page_log2) + (token & ((1 << p.cache.page_log2) - 1));
      codes[i] = (int64_t)((uint64_t)(uint32_t)pg * (uint32_t)p.cache.stride_codes) + (uint32_t)row * (uint32_t)(D / 2);
      scales[i] = (int64_t)((uint64_t)(uint32_t)pg * (uint32_t)p.cache.stride_scales) + (uint32_t)row * (uint32_t)(D / 32);
    }
  }
  __device__ __forceinline__ bool gone(int kb) const { return (absent >> (kOnePage ? 0 : kb) & 1) != 0; }
  // this lane's pieces of the four blocks of K or of V
  __device__ __forceinline__ void load(Codes<D> (&x)[4], const uint8_t* code_base, const uint8_t* scale_base, int li, int lg) const {
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      constexpr int kCodeStep = kOnePage ? 16 * (D / 2) : 0, kScaleStep = kOnePage ? 16 * (D / 32) : 0;
      x[kb].load(code_base + codes[kOnePage ? 0 : kb], scale_base + scales[kOnePage ? 0 : kb], kb * kCodeStep, kb * kScaleStep, li, lg);
    }
  }
};

template <int D, int NQ, bool kOnePage>
__global__ __launch_bounds__(64 * kCacheWaves, 2) void cache_attention_kernel(const CacheAttnParams p) {
  using T = Tile<D, 1>;
  constexpr int W = kCacheWaves, R = 16 * NQ;
  // a wave's V tile, later its last piece's O; its first piece's O where it goes on to others (two blocks of rows leave no room
  // for it in LDS: in the workspace)
  constexpr int kWaveLds = T::TILE_BYTES > R * D * 4 ? T::TILE_BYTES : R * D * 4;
  constexpr bool kHeadsInLds = NQ == 1;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kHeadsInLds ? 2 : 1][W][kWaveLds];      // [tails, heads]
  __shared__ float stat[2][W][2][R];                       // [tails, heads][wave][maximum, row sum]
  __shared__ __attribute__((aligned(16))) int kept[W], place[2][W][4];       // place: first query, rows, KV head, first row

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int li = lane & 15, lg = lane >> 4;
  Axis<R> axis(p);
  const int64_t share = axis.share(p);
  // consecutive shares on one XCD: row tiles of a head read the same keys
  const int wg = p.workgroups % kXcds == 0 ? (int)(blockIdx.x % kXcds) * (p.workgroups / kXcds) + (int)(blockIdx.x / kXcds) : (int)blockIdx.x;
  const int64_t wg_begin = wg * share;
  const int64_t wg_end = wg_begin + share < axis.total ? wg_begin + share : axis.total;
  if (wg_begin >= wg_end) return;
  // a wave's part of the share
  const int64_t wave_share = (wg_end - wg_begin + W - 1) / W;
  int64_t pos = wg_begin + wave * wave_share;
  const int64_t end = pos + wave_share < wg_end ? pos + wave_share : wg_end;
  int keeps = 0;

  // per-lane LDS offsets: V rows as written, and as the A operand of O^T (query_attention.hip)
  constexpr int kPieces = D / 64 * 2;                      // 16-byte chunks of a lane's quarter row
  int v_put[kPieces], v_off[T::DBN];
#pragma unroll
  for (int x = 0; x < kPieces; ++x) v_put[x] = li * T::ROW_BYTES + (((lg * kPieces + x) ^ T::fv(li)) << 4);
  {
    const int row = 4 * lg + (li >> 2);
#pragma unroll
    for (int d = 0; d < T::DBN; ++d) v_off[d] = row * T::ROW_BYTES + (((2 * d + ((li & 3) >> 1)) ^ T::fv(row)) << 4) + (li & 1) * 8;
  }
  constexpr int kChunks = D / 4;                           // 16-byte chunks of a kept row of O, swizzled by the row
  float* head_global = p.parts + (int64_t)p.workgroups * 2 * (R * (D + 2)) + (int64_t)wg * W * (R * D);
  unsigned char* vbuf = lds[0][wave];
  const float inv_scale_log2 = 1.0f / p.scale_log2;

  int b = 0;
  int64_t begin = 0;
  if (pos < end) {
    b = axis.find(p, pos);
    begin = axis.begin_of(b);
  }
#pragma unroll 1
  while (pos < end) {
    const Request rq = axis.at(p, b);
    const int row_tiles = (rq.rows + R - 1) / R;
    const int64_t of_request = (int64_t)row_tiles * p.hkv * rq.tiles;
    if (pos >= begin + of_request) {                       // (or a request with nothing to do)
      begin += of_request;
      ++b;
      continue;
    }
    const int64_t rel = pos - begin;
    const int64_t item = quotient(rel, rq.tiles);
    const int head = (int)quotient(item, row_tiles), rt = (int)(item - (int64_t)head * row_tiles);
    const int t0 = (int)(rel - item * rq.tiles);
    const int t1 = end - pos < rq.tiles - t0 ? t0 + (int)(end - pos) : rq.tiles;
    pos += t1 - t0;

    // ---- the row tile's rows: keys each sees, and Q^T fragments (k-step c of lane lg: elements lg * D / 4 + 8 c ...)
    const int r0 = rt * R;
    const int queries = rq.rows / p.group;
    bf16x8 qf[T::KSD][NQ];
    int jlast[NQ];
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      const int r = r0 + 16 * nq + li < rq.rows ? r0 + 16 * nq + li : rq.rows - 1;
      const int i = r / p.group;
      jlast[nq] = p.causal ? rq.len - queries + i : rq.len - 1;
      const bf16_t* qrow = p.q.ptr + (int64_t)(rq.first + i) * p.q.st + (int64_t)(head * p.group + r % p.group) * p.q.sh + lg * (D / 4);
#pragma unroll
      for (int c = 0; c < T::KSD; ++c) qf[c][nq] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qrow + 8 * c));
    }
    // keys that every row sees, keys that some row sees
    const int all = p.causal ? rq.len - queries + r0 / p.group + 1 : rq.len;
    const int last_row = r0 + R < rq.rows ? r0 + R - 1 : rq.rows - 1;
    const int some = p.causal ? rq.len - queries + last_row / p.group + 1 : rq.len;
    const int t_end = some <= 0 ? 0 : (t1 * kCacheKeyTile < some ? t1 : (some + kCacheKeyTile - 1) / kCacheKeyTile);

    f32x4 o[T::DBN][NQ];
    float m_ref[NQ], m_sub[NQ], s_far[NQ], l_run[NQ];
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
#pragma unroll
      for (int d = 0; d < T::DBN; ++d) o[d][nq] = f32x4{0.f, 0.f, 0.f, 0.f};
      m_ref[nq] = s_far[nq] = -INFINITY;
      m_sub[nq] = l_run[nq] = 0.f;
    }

    const int32_t* table_row = p.table + (int64_t)b * p.table_stride;
    // With one block of rows two tiles are on their way while one is worked on: in a long request a wave has only a few, and
    // what takes time is how often it waits for memory.  (With two there are no registers for it.)
    constexpr int kAhead = NQ == 1 ? 2 : 1;
    Codes<D> kc[kAhead][4], vc[kAhead][4];
    Blocks<D, kOnePage> at[kAhead];
    auto find = [&](auto& x, int t) { x.find(p, table_row, head, rq.len, t < t_end ? t : t_end - 1); };      // (the last tile again)
    auto load_k = [&](const auto& x, Codes<D> (&to)[4]) { x.load(to, p.cache.k_codes, p.cache.k_scales, li, lg); };
    auto load_v = [&](const auto& x, Codes<D> (&to)[4]) { x.load(to, p.cache.v_codes, p.cache.v_scales, li, lg); };
    auto work = [&](int t, Blocks<D, kOnePage>& here, Codes<D> (&kc)[4], Codes<D> (&vc)[4]) {
      const Blocks<D, kOnePage> now = here;
      find(here, t + kAhead);

      // ---- S^T = K Q^T, lane: keys 16 kb + 4 lg + e of row li
      f32x4 s[4][NQ];
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int c = 0; c < T::KSD; ++c) {
          const bf16x8 a = __builtin_bit_cast(bf16x8, kc[kb].values(c));
#pragma unroll
          for (int nq = 0; nq < NQ; ++nq)
            s[kb][nq] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[c][nq], c == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[kb][nq], 0, 0, 0);
        }
      load_k(here, kc);

      // ---- hidden keys: out of sight of a row, or not there at all, whose values may be anything
      if ((t + 1) * kCacheKeyTile > all || now.absent != 0) {
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
          const int j = t * kCacheKeyTile + 16 * kb;
          const bool gone = now.gone(kb);
          vc[kb].scale = gone || j + li >= rq.len ? 0u : vc[kb].scale;
#pragma unroll
          for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (gone || j + 4 * lg + e > jlast[nq]) s[kb][nq][e] = -INFINITY;
        }
      }

      // ---- the reference maxima move when a logit lies far above (attention.hip)
      float lm[NQ];
      bool far = false;
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) {
        float mx = s[0][nq][0];
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
          for (int e = 0; e < 4; ++e) mx = __builtin_fmaxf(mx, s[kb][nq][e]);
        lm[nq] = mx;
        far = far || mx > s_far[nq];
      }
      if (__builtin_amdgcn_ballot_w64(far) != 0) {
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
          float mx = lm[nq];
          {
            auto sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
          }
          {
            auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
          }
          const float m_new = fmaxf(m_ref[nq], mx * p.scale_log2);
          const float alpha = m_new > -INFINITY ? __builtin_amdgcn_exp2f(m_ref[nq] - m_new) : 1.f;
          m_ref[nq] = m_new;
          m_sub[nq] = m_new > -INFINITY ? m_new : 0.f;
          s_far[nq] = (m_new + kRescaleThreshold) * inv_scale_log2;
          l_run[nq] *= alpha;
#pragma unroll
          for (int d = 0; d < T::DBN; ++d) o[d][nq] *= alpha;
        }
      }

      // ---- O^T += V^T P^T, 32 keys at a time through the wave's LDS tile (LDS operations of a wave are in order)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int mb = 0; mb < 2; ++mb)
#pragma unroll
          for (int x = 0; x < kPieces; ++x)
            *reinterpret_cast<u32x4*>(vbuf + mb * 16 * T::ROW_BYTES + v_put[x]) = vc[2 * half + mb].values(x);
        u32x4 pw[NQ];
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
          for (int mb = 0; mb < 2; ++mb)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
              const f32x4& y = s[2 * half + mb][nq];
              const f32x2 xy = {__builtin_amdgcn_exp2f(__builtin_fmaf(y[e], p.scale_log2, -m_sub[nq])),
                                __builtin_amdgcn_exp2f(__builtin_fmaf(y[e + 1], p.scale_log2, -m_sub[nq]))};
              const bf16x2 c = __builtin_convertvector(xy, bf16x2);
              l_run[nq] = __builtin_amdgcn_fdot2_f32_bf16(c, bf16x2{(__bf16)1.0f, (__bf16)1.0f}, l_run[nq], false);
              pw[nq][2 * mb + (e >> 1)] = __builtin_bit_cast(uint32_t, c);
            }
#pragma unroll
        for (int d = 0; d < T::DBN; ++d) {
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((APBV_LDS(s16x4))(vbuf + v_off[d]));
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((APBV_LDS(s16x4))(vbuf + 16 * T::ROW_BYTES + v_off[d]));
          const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
          for (int nq = 0; nq < NQ; ++nq)
            o[d][nq] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, pw[nq]), o[d][nq], 0, 0, 0);
        }
      }
      load_v(here, vc);
    };
    int t = t0;
    if (t < t_end) {
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        find(at[a], t + a);
        load_k(at[a], kc[a]);
        load_v(at[a], vc[a]);
      }
#pragma unroll 1
      for (;;) {
        work(t, at[0], kc[0], vc[0]);
        if (++t >= t_end) break;
        if constexpr (kAhead > 1) {
          work(t, at[1], kc[1], vc[1]);
          if (++t >= t_end) break;
        }
      }
    }

    // ---- a piece that is a whole row tile is done; others are kept for the waves' pieces to be put together below
    float l_tot[NQ];
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      float x = l_run[nq];
      {
        auto sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
      }
      {
        auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
      }
      l_tot[nq] = x;
    }
    if (t0 == 0 && t1 == rq.tiles) {
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) {
        const int row = r0 + 16 * nq + li;
        if (row >= rq.rows) continue;
        const int i = row / p.group, h = head * p.group + row % p.group;
        const float inv = l_tot[nq] > 0.f ? 1.0f / l_tot[nq] : 0.f;
        bf16_t* dst = p.out + ((int64_t)(rq.first + i) * p.hq + h) * D + 4 * lg;
#pragma unroll
        for (int d = 0; d < T::DBN; ++d) {
          const f32x4 x = o[d][nq] * inv;
          u32x2 y;
          y.x = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x.x, x.y}), bf16x2));
          y.y = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x.z, x.w}), bf16x2));
          *reinterpret_cast<u32x2*>(dst + 16 * d) = y;
        }
        if (p.lse != nullptr && lg == 0)
          p.lse[(int64_t)h * p.n_rows + rq.first + i] = l_tot[nq] > 0.f ? (m_ref[nq] + __builtin_amdgcn_logf(l_tot[nq])) * 0.6931471805599453f : -INFINITY;
      }
    } else {
      // (a row tile that ends here but began before is a head; one that goes on, a tail or, of one that began before, a span)
      const int is_head = t1 == rq.tiles ? 1 : 0;
      auto keep = [&](f32x4* to) {
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
          for (int d = 0; d < T::DBN; ++d) to[(16 * nq + li) * kChunks + ((4 * d + lg) ^ li)] = o[d][nq];
      };
      if constexpr (kHeadsInLds)
        keep(reinterpret_cast<f32x4*>(lds[is_head][wave]));
      else if (is_head)
        keep(reinterpret_cast<f32x4*>(head_global + (int64_t)wave * (R * D)));
      else
        keep(reinterpret_cast<f32x4*>(lds[0][wave]));
      if (lg == 0) {
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
          stat[is_head][wave][0][16 * nq + li] = m_ref[nq];
          stat[is_head][wave][1][16 * nq + li] = l_tot[nq];
        }
      }
      keeps |= is_head ? kHead : (t0 == 0 ? kTail : kSpan);
      if (lane == 0) {
        place[is_head][wave][0] = rq.first;
        place[is_head][wave][1] = rq.rows;
        place[is_head][wave][2] = head;
        place[is_head][wave][3] = r0;
      }
    }
  }
  if (lane == 0) kept[wave] = keeps;
  __syncthreads();

  // ---- the pieces of a row tile that lie in consecutive waves, one chain of them after the other: chain 0 goes on with a row
  // tile that began before this workgroup, chain c begins with the tail of wave c - 1
  int heads = 0, tails = 0, spans = 0;                     // a bit a wave
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const int k = __builtin_amdgcn_readfirstlane(kept[w]);
    heads |= (k & kHead ? 1 : 0) << w;
    tails |= (k & kTail ? 1 : 0) << w;
    spans |= (k & kSpan ? 1 : 0) << w;
  }
#pragma unroll 1
  for (int chain = 0; chain <= W; ++chain) {
    const int from = chain == 0 ? 0 : chain - 1;
    if (((chain == 0 ? heads | spans : tails) >> from & 1) == 0) continue;
    int to = from;                                         // its last wave
    bool ends = chain == 0 && (heads & 1);
    while (!ends && to + 1 < W) {
      if (heads >> (to + 1) & 1) ends = true;
      else if ((spans >> (to + 1) & 1) == 0) break;        // a wave without a share: the workgroup ends here
      ++to;
    }
    const bool whole = chain > 0 && ends;
    const int* at = place[ends && to == from ? 1 : 0][from];
    const int first = at[0], rows = at[1], head = at[2], r0 = at[3];
    const int slot = chain > 0 ? 1 : 0;                    // a part that begins a row tile, or one that goes on with it
    float* part = p.parts + ((int64_t)wg * 2 + slot) * (R * D);
    float* part_stat = p.parts + (int64_t)p.workgroups * 2 * (R * D) + (int64_t)slot * (2 * R) * p.workgroups + wg;
    for (int x = threadIdx.x; x < R * (D / 8); x += 64 * W) {
      const int row = x / (D / 8), c = x % (D / 8);
      if (r0 + row >= rows) break;
      float m = -INFINITY, l = 0.f;
      for (int w = from; w <= to; ++w) m = fmaxf(m, stat[w == to && ends ? 1 : 0][w][0][row]);
      const float m0 = m > -INFINITY ? m : 0.f;
      f32x4 x0 = {0.f, 0.f, 0.f, 0.f}, x1 = {0.f, 0.f, 0.f, 0.f};
      for (int w = from; w <= to; ++w) {
        const int is_head = w == to && ends ? 1 : 0;
        const float weight = __builtin_amdgcn_exp2f(stat[is_head][w][0][row] - m0);
        l = __builtin_fmaf(stat[is_head][w][1][row], weight, l);
        auto add = [&](const f32x4* src) {
          src += row * kChunks;
          x0 += weight * src[(2 * c) ^ (row & 15)];
          x1 += weight * src[(2 * c + 1) ^ (row & 15)];
        };
        if constexpr (kHeadsInLds)
          add(reinterpret_cast<const f32x4*>(lds[is_head][w]));
        else if (is_head)
          add(reinterpret_cast<const f32x4*>(head_global + (int64_t)w * (R * D)));
        else
          add(reinterpret_cast<const f32x4*>(lds[0][w]));
      }
      if (whole) {
        const float inv = l > 0.f ? 1.0f / l : 0.f;
        x0 *= inv;
        x1 *= inv;
        u32x4 y;
        y.x = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x0.x, x0.y}), bf16x2));
        y.y = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x0.z, x0.w}), bf16x2));
        y.z = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x1.x, x1.y}), bf16x2));
        y.w = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x1.z, x1.w}), bf16x2));
        const int i = (r0 + row) / p.group, h = head * p.group + (r0 + row) % p.group;
        *reinterpret_cast<u32x4*>(p.out + ((int64_t)(first + i) * p.hq + h) * D + 8 * c) = y;
        if (p.lse != nullptr && c == 0)
          p.lse[(int64_t)h * p.n_rows + first + i] = l > 0.f ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : -INFINITY;
      } else {
        f32x4* dst = reinterpret_cast<f32x4*>(part + row * D + 8 * c);
        dst[0] = x0;
        dst[1] = x1;
        if (c == 0) {
          part_stat[(int64_t)row * p.workgroups] = m;
          part_stat[(int64_t)(R + row) * p.workgroups] = l;
        }
      }
    }
  }
}

// kJoin waves per (row of q, head): joins the parts of rows that several workgroups share, and clears the rows without a key.
// A row has as many parts as workgroups share its keys: a few in a batch, a hundred and more in one long request, where the
// waves take them in turn.  Maxima and row sums of a row lie side by side over the workgroups.
template <int D, int R, int kJoin>
__global__ __launch_bounds__(kJoin == 1 ? 256 : 64 * kJoin) void cache_join_kernel(const CacheAttnParams p) {
  constexpr int kRowsPerGroup = kJoin == 1 ? 4 : 1;
  __shared__ float shared_max[kJoin], shared_sum[kJoin];
  __shared__ f32x4 shared_acc[kJoin][D / 4];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t job = (int64_t)blockIdx.x * kRowsPerGroup + (kJoin == 1 ? wave : 0);
  if (job >= (int64_t)p.n_rows * p.hq) return;
  const int row = (int)(job / p.hq), h = (int)(job % p.hq);
  Axis<R> axis(p);
  const int b = axis.find_row(p, row);
  const Request rq = axis.at(p, b);
  const int i = row - rq.first;
  if (i < 0 || i * p.group >= rq.rows) return;             // a row of no request
  constexpr int kLanes = D / 4;                            // lanes that hold a row, four elements each
  constexpr int kAtOnce = 64 / kLanes;
  const int sub = lane / kLanes, c = lane % kLanes;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  if (rq.tiles > 0) {
    const int64_t share = axis.share(p);
    const int r = i * p.group + h % p.group, rt = r / R, row_tiles = (rq.rows + R - 1) / R;
    const int64_t from = axis.begin_of(b) + ((int64_t)(h / p.group) * row_tiles + rt) * rq.tiles;
    const int first = (int)quotient(from, share), last = (int)quotient(from + rq.tiles - 1, share);
    if (first == last) return;                             // written by its only workgroup
    const float* stat = p.parts + (int64_t)p.workgroups * 2 * (R * D) + (int64_t)(r % R) * p.workgroups;
    const float* rows = p.parts + (r % R) * D + 4 * c;
    // a wave's equal share of the parts, kAtOnce * kLoads at a time: lane n holds the n-th's maximum and row sum, and the rows
    // are on their way while the weights are found
    constexpr int kLoads = 8, kChunk = kAtOnce * kLoads;
    const int each = kJoin == 1 ? last - first + 1 : (last - first + kJoin) / kJoin;
    const int from_part = first + (kJoin == 1 ? 0 : wave * each);
    const int past_part = from_part + each <= last ? from_part + each : last + 1;
    for (int base = from_part; base < past_part; base += kChunk) {
      const int w = base + lane;
      const bool mine = lane < kChunk && w < past_part;
      const float* s = stat + (w == first ? (int64_t)(2 * R) * p.workgroups : 0) + w;
      const float m_part = mine ? s[0] : -INFINITY, l_part = mine ? s[(int64_t)R * p.workgroups] : 0.f;
      f32x4 x[kLoads];
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        const int y = base + u * kAtOnce + sub;
        x[u] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (y < past_part) x[u] = *reinterpret_cast<const f32x4*>(rows + ((int64_t)y * 2 + (y == first ? 1 : 0)) * (R * D));
      }
      float top = m_part;
#pragma unroll
      for (int d = 1; d < kChunk; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
      top = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(fmaxf(top, m))));
      const float m0 = top > -INFINITY ? top : 0.f;
      const float old = __builtin_amdgcn_exp2f(m - m0), weight = __builtin_amdgcn_exp2f(m_part - m0);
      m = top;
      l = __builtin_fmaf(l, old, weight * l_part);         // (this lane's parts; the lanes are added up below)
      acc *= old;
#pragma unroll
      for (int u = 0; u < kLoads; ++u) acc += __shfl(weight, u * kAtOnce + sub) * x[u];
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) l += __shfl_xor(l, d);
#pragma unroll
    for (int d = kLanes; d < 64; d *= 2)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], d);
  }
  if constexpr (kJoin > 1) {
    if (lane == 0) shared_max[wave] = m, shared_sum[wave] = l;
    if (sub == 0) shared_acc[wave][c] = acc;
    __syncthreads();
    if (wave != 0) return;
    m = -INFINITY;
#pragma unroll
    for (int w = 0; w < kJoin; ++w) m = fmaxf(m, shared_max[w]);
    const float m0 = m > -INFINITY ? m : 0.f;
    l = 0.f;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kJoin; ++w) {
      const float weight = __builtin_amdgcn_exp2f(shared_max[w] - m0);
      l = __builtin_fmaf(shared_sum[w], weight, l);
      acc += weight * shared_acc[w][c];
    }
  }
  if (sub != 0) return;
  const float inv = l > 0.f ? 1.0f / l : 0.f;
  u32x2 y;
  y.x = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{acc.x * inv, acc.y * inv}), bf16x2));
  y.y = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{acc.z * inv, acc.w * inv}), bf16x2));
  *reinterpret_cast<u32x2*>(p.out + job * D + 4 * c) = y;
  if (p.lse != nullptr && lane == 0) p.lse[(int64_t)h * p.n_rows + row] = l > 0.f ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : -INFINITY;
}

template <int D, int NQ, bool kOnePage>
apbv_status launch_variant(const CacheAttnParams& p, hipStream_t stream) {
  const int64_t rows = (int64_t)p.n_rows * p.hq;
  if (rows > 0x7fffffff) return APBV_ERR_UNSUPPORTED;
  Launcher launch(stream);
  launch(cache_attention_kernel<D, NQ, kOnePage>, dim3((unsigned)p.workgroups), dim3(64 * kCacheWaves), 0, p);
  if (rows <= kCacheJoinRows)
    launch(cache_join_kernel<D, 16 * NQ, 16>, dim3((unsigned)rows), dim3(1024), 0, p);
  else
    launch(cache_join_kernel<D, 16 * NQ, 1>, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, p);
  return launch.status();
}
template <int D, int NQ>
apbv_status launch_rows(const CacheAttnParams& p, hipStream_t stream) {
  return (1 << p.cache.page_log2) >= kCacheKeyTile ? launch_variant<D, NQ, true>(p, stream) : launch_variant<D, NQ, false>(p, stream);
}

}  // namespace

apbv_status launch_cache_attention(const CacheAttnParams& p, const CachePlan& plan, int head_dim, hipStream_t stream) {
  if (head_dim == 128) return plan.rows == 16 ? launch_rows<128, 1>(p, stream) : launch_rows<128, 2>(p, stream);
  return plan.rows == 16 ? launch_rows<64, 1>(p, stream) : launch_rows<64, 2>(p, stream);
}

}  // namespace apbv
