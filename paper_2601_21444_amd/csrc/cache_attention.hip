// Attention over the key/value cache held in 4 bits (include/apbv_cache.h), for gfx950.
//
// Rows.  As in query_attention.hip the G query heads of a KV head are G rows of one problem: row r = i * G + g of a request is
// its query i of head kvh * G + g.  A row tile is 16 or 32 of them.
//
// Cut.  Only the device knows the lengths.  Every workgroup adds up the requests' tiles (a wave's lanes take a request each)
// and takes an equal share of the axis that all (request, KV head, row tile) lie on one after the other, 64 keys a tile: a
// batch of unequal lengths fills the chip as an equal one does, and so does one request.  A share that begins or ends inside
// a (request, head, row tile) leaves O, the maxima and the row sums of its part in the workspace in float32; a second launch
// joins the parts.
//
// Keys.  A lane of the matrix instruction's A operand needs eight elements of one key, and which elements go with which k-step
// is free as long as K and Q agree: lane (key li, quarter lg) takes the quarter's 16 bytes of codes, one load, all of one
// scale block, and converts eight of them a k-step.  No LDS.  V is needed transposed: a lane converts its quarter of a key's
// row, writes it to the wave's own LDS tile as bf16, and the transposing LDS read does the rest.  The waves of a workgroup take
// a share's tiles in turn, with no barrier, and are joined in LDS at its end.
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
__device__ __forceinline__ Request request(const CacheAttnParams& p, int b) {                  // b uniform
  const int first = p.starts ? scalar_load(p.starts, b) : b * p.each;
  const int past = p.starts ? scalar_load(p.starts, b + 1) : (b + 1) * p.each;
  return request_of(p, first, past, scalar_load(p.lengths, b));
}

__device__ __forceinline__ int64_t uniform64(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)x >> 32));
  return (int64_t)(((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ int64_t readlane64(int64_t x, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)x, lane), hi = __builtin_amdgcn_readlane((uint32_t)((uint64_t)x >> 32), lane);
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

// The axis of tiles: its length, and where the requests lie on it.  Lane l of a wave holds requests l * per to (l + 1) * per - 1.
template <int R>
struct Axis {
  int per;
  int64_t past;              // where this lane's requests end
  int64_t total;
  __device__ __forceinline__ static int64_t tiles(const CacheAttnParams& p, const Request& r) {
    return (int64_t)((r.rows + R - 1) / R) * p.hkv * r.tiles;
  }
  __device__ __forceinline__ Axis(const CacheAttnParams& p) {
    const int lane = threadIdx.x & 63;
    per = (p.n_requests + 63) / 64;
    int64_t sum = 0;
    for (int u = 0; u < per; ++u) {
      const int b = lane * per + u;
      if (b >= p.n_requests) break;
      const int first = p.starts ? p.starts[b] : b * p.each, past_row = p.starts ? p.starts[b + 1] : (b + 1) * p.each;
      sum += tiles(p, request_of(p, first, past_row, p.lengths[b]));
    }
    past = sum;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int64_t x = __shfl_up(past, d);
      if (lane >= d) past += x;
    }
    total = readlane64(past, 63);
  }
  // Length of a workgroup's share.
  __device__ __forceinline__ int64_t share(const CacheAttnParams& p) const {
    const int64_t q = (total + p.workgroups - 1) / p.workgroups;
    return q > p.least_tiles ? q : p.least_tiles;
  }
  // The request that holds tile `pos` < total, and where it begins.
  __device__ __forceinline__ int find(const CacheAttnParams& p, int64_t pos, int64_t& begin) const {
    const uint64_t behind = __builtin_amdgcn_ballot_w64(past > pos);
    const int lane = __builtin_ctzll(behind);
    int b = lane * per;
    begin = lane > 0 ? readlane64(past, lane - 1) : 0;
    for (;; ++b) {
      const int64_t t = tiles(p, request(p, b));
      if (pos < begin + t) return b;
      begin += t;
    }
  }
  // Where request b (uniform) begins.
  __device__ __forceinline__ int64_t begin_of(const CacheAttnParams& p, int b) const {
    const int lane = b / per;
    int64_t begin = lane > 0 ? readlane64(past, lane - 1) : 0;
    for (int i = lane * per; i < b; ++i) begin += tiles(p, request(p, i));
    return begin;
  }
};

constexpr int kCacheWaves = 4;

// A 16-key block's codes (16 bytes a lane at head_dim 128, 8 at 64) and scale byte.
template <int D>
struct Codes {
  static constexpr int kWords = D / 32;
  uint32_t w[kWords];
  uint32_t scale;
  // row: of the page, this lane's key; lg: its quarter
  __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* scales, int li, int lg) {
    if constexpr (D == 128) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(codes + (uint32_t)(li * 64 + lg * 16));
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = x[i];
      scale = scales[(uint32_t)(li * 4 + lg)];
    } else {
      const u32x2 x = *reinterpret_cast<const u32x2*>(codes + (uint32_t)(li * 32 + lg * 8));
      w[0] = x[0];
      w[1] = x[1];
      scale = scales[(uint32_t)(li * 2 + (lg >> 1))];
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

// Where the four 16-key blocks of a tile lie (uniform): row offsets, pages, and which are not there.
struct Blocks {
  int page[4];
  int row[4];
  int absent;                // bit kb: block kb's page is out of range, or no key of the request lies in it
  __device__ __forceinline__ void find(const CacheAttnParams& p, const int32_t* table_row, int head, int len, int tile) {
    absent = 0;
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      const int token = tile * kCacheKeyTile + 16 * kb;
      const int at = token < len ? token : len - 1;                      // (a table entry that the request has)
      const int pg = scalar_load(table_row, at >> p.cache.page_log2);
      const bool there = token < len && (unsigned)pg < (unsigned)p.cache.n_pages;
      absent |= there ? 0 : 1 << kb;
      page[kb] = there ? pg : 0;
      row[kb] = (head << p.cache.page_log2) + (there ? token & ((1 << p.cache.page_log2) - 1) : 0);
    }
  }
};

template <int D, int NQ>
__global__ __launch_bounds__(64 * kCacheWaves, 2) void cache_attention_kernel(const CacheAttnParams p) {
  using T = Tile<D, 1>;
  constexpr int W = kCacheWaves, R = 16 * NQ;
  constexpr int kWaveLds = T::TILE_BYTES > R * D * 4 ? T::TILE_BYTES : R * D * 4;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[W][kWaveLds];
  __shared__ float stat[W][2][R];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int li = lane & 15, lg = lane >> 4;
  const Axis<R> axis(p);
  const int64_t share = axis.share(p);
  // consecutive shares on one XCD: row tiles of a head read the same keys
  const int wg = p.workgroups % kXcds == 0 ? (int)(blockIdx.x % kXcds) * (p.workgroups / kXcds) + (int)(blockIdx.x / kXcds) : (int)blockIdx.x;
  int64_t pos = wg * share;
  const int64_t end = pos + share < axis.total ? pos + share : axis.total;
  if (pos >= end) return;
  int64_t begin;
  int b = axis.find(p, pos, begin);

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
  unsigned char* vbuf = lds[wave];
  const float inv_scale_log2 = 1.0f / p.scale_log2;

#pragma unroll 1
  while (pos < end) {
    const Request rq = request(p, b);
    const int row_tiles = (rq.rows + R - 1) / R;
    const int64_t of_request = (int64_t)row_tiles * p.hkv * rq.tiles;
    if (pos >= begin + of_request) {                       // (or a request with nothing to do)
      begin += of_request;
      ++b;
      continue;
    }
    const int64_t rel = pos - begin;
    const int64_t item = rel / rq.tiles;
    const int head = (int)(item / row_tiles), rt = (int)(item % row_tiles);
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
    Codes<D> kc[4], vc[4];
    Blocks at;
    auto load_k = [&](const Blocks& x) {
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
        kc[kb].load(p.cache.k_codes + (int64_t)x.page[kb] * p.cache.stride_codes + (int64_t)x.row[kb] * (D / 2),
                    p.cache.k_scales + (int64_t)x.page[kb] * p.cache.stride_scales + (int64_t)x.row[kb] * (D / 32), li, lg);
    };
    auto load_v = [&](const Blocks& x) {
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
        vc[kb].load(p.cache.v_codes + (int64_t)x.page[kb] * p.cache.stride_codes + (int64_t)x.row[kb] * (D / 2),
                    p.cache.v_scales + (int64_t)x.page[kb] * p.cache.stride_scales + (int64_t)x.row[kb] * (D / 32), li, lg);
    };
    int t = t0 + wave;
    if (t < t_end) {
      at.find(p, table_row, head, rq.len, t);
      load_k(at);
      load_v(at);
    }
#pragma unroll 1
    for (; t < t_end; t += W) {
      const int absent = at.absent;
      const int tn = t + W < t_end ? t + W : t;            // (the last tile is requested again)
      at.find(p, table_row, head, rq.len, tn);

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
      load_k(at);

      // ---- hidden keys: out of sight of a row, or not there at all, whose values may be anything
      if ((t + 1) * kCacheKeyTile > all || absent != 0) {
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
          const int j = t * kCacheKeyTile + 16 * kb;
          const bool gone = (absent >> kb & 1) != 0;
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
      load_v(at);
    }

    // ---- the waves' results together: O scaled to the rows' maximum over the waves, in LDS as float32, chunks of a row
    // swizzled by the row
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
      if (lg == 0) {
        stat[wave][0][16 * nq + li] = m_ref[nq];
        stat[wave][1][16 * nq + li] = x;
      }
    }
    __syncthreads();
    constexpr int kChunks = D / 4;
    const bool whole = t0 == 0 && t1 == rq.tiles;
    float* part = p.parts + ((int64_t)wg * 2 + (t0 == 0 ? 1 : 0)) * (R * (D + 2));
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      const int row = 16 * nq + li;
      float m = -INFINITY, l = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) m = fmaxf(m, stat[w][0][row]);
      const float m0 = m > -INFINITY ? m : 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) l = __builtin_fmaf(stat[w][1][row], __builtin_amdgcn_exp2f(stat[w][0][row] - m0), l);
      float factor = __builtin_amdgcn_exp2f(m_ref[nq] - m0);
      if (whole) factor = l > 0.f ? factor / l : 0.f;
      f32x4* mine = reinterpret_cast<f32x4*>(lds[wave]);
#pragma unroll
      for (int d = 0; d < T::DBN; ++d) mine[row * kChunks + ((4 * d + lg) ^ li)] = o[d][nq] * factor;
      if (wave == 0 && lg == 0) {
        if (!whole) {
          part[R * D + row] = m;
          part[R * D + R + row] = l;
        } else if (p.lse != nullptr && r0 + row < rq.rows) {
          const int i = (r0 + row) / p.group, h = head * p.group + (r0 + row) % p.group;
          p.lse[(int64_t)h * p.n_rows + rq.first + i] = l > 0.f ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : -INFINITY;
        }
      }
    }
    __syncthreads();
    for (int x = threadIdx.x; x < R * (D / 8); x += 64 * W) {
      const int row = x / (D / 8), c = x % (D / 8);
      if (r0 + row >= rq.rows) break;
      f32x4 x0 = {0.f, 0.f, 0.f, 0.f}, x1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const f32x4* src = reinterpret_cast<const f32x4*>(lds[w]) + row * kChunks;
        x0 += src[(2 * c) ^ (row & 15)];
        x1 += src[(2 * c + 1) ^ (row & 15)];
      }
      if (whole) {
        u32x4 y;
        y.x = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x0.x, x0.y}), bf16x2));
        y.y = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x0.z, x0.w}), bf16x2));
        y.z = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x1.x, x1.y}), bf16x2));
        y.w = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x1.z, x1.w}), bf16x2));
        const int i = (r0 + row) / p.group, h = head * p.group + (r0 + row) % p.group;
        *reinterpret_cast<u32x4*>(p.out + ((int64_t)(rq.first + i) * p.hq + h) * D + 8 * c) = y;
      } else {
        f32x4* dst = reinterpret_cast<f32x4*>(part + row * D + 8 * c);
        dst[0] = x0;
        dst[1] = x1;
      }
    }
    __syncthreads();                                       // LDS is free again
  }
}

// One wave per (row of q, head): joins the parts of rows that several workgroups share, and clears the rows without a key.
template <int D, int R>
__global__ __launch_bounds__(256) void cache_join_kernel(const CacheAttnParams p) {
  const int lane = threadIdx.x & 63;
  const int64_t job = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (job >= (int64_t)p.n_rows * p.hq) return;
  const int row = (int)(job / p.hq), h = (int)(job % p.hq);
  const Axis<R> axis(p);
  // the request of this row: the last that begins at or before it
  int b;
  if (p.starts == nullptr) {
    b = row / p.each;
  } else {
    int lo = 0, hi = p.n_requests;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (scalar_load(p.starts, mid) <= row) lo = mid; else hi = mid;
    }
    b = lo;
  }
  const Request rq = request(p, b);
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
    const int64_t from = axis.begin_of(p, b) + ((int64_t)(h / p.group) * row_tiles + rt) * rq.tiles;
    const int first = (int)(from / share), last = (int)((from + rq.tiles - 1) / share);
    if (first == last) return;                             // written by its only workgroup
    auto part = [&](int w) { return p.parts + ((int64_t)w * 2 + (w == first ? 1 : 0)) * (R * (D + 2)); };
    for (int w = first + lane; w <= last; w += 64) m = fmaxf(m, part(w)[R * D + r % R]);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
    if (m > -INFINITY) {
      for (int w = first + sub; w <= last; w += kAtOnce) {
        const float* x = part(w);
        const float weight = __builtin_amdgcn_exp2f(x[R * D + r % R] - m);
        l = __builtin_fmaf(weight, x[R * D + R + r % R], l);
        acc += weight * *reinterpret_cast<const f32x4*>(x + (r % R) * D + 4 * c);
      }
#pragma unroll
      for (int d = kLanes; d < 64; d *= 2) {
        l += __shfl_xor(l, d);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], d);
      }
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

template <int D, int NQ>
apbv_status launch_variant(const CacheAttnParams& p, hipStream_t stream) {
  const int64_t blocks = ((int64_t)p.n_rows * p.hq + 3) / 4;
  if (blocks > 0x7fffffff) return APBV_ERR_UNSUPPORTED;
  Launcher launch(stream);
  launch(cache_attention_kernel<D, NQ>, dim3((unsigned)p.workgroups), dim3(64 * kCacheWaves), 0, p);
  launch(cache_join_kernel<D, 16 * NQ>, dim3((unsigned)blocks), dim3(256), 0, p);
  return launch.status();
}

}  // namespace

apbv_status launch_cache_attention(const CacheAttnParams& p, const CachePlan& plan, int head_dim, hipStream_t stream) {
  if (head_dim == 128) return plan.rows == 16 ? launch_variant<128, 1>(p, stream) : launch_variant<128, 2>(p, stream);
  return plan.rows == 16 ? launch_variant<64, 1>(p, stream) : launch_variant<64, 2>(p, stream);
}

}  // namespace apbv
