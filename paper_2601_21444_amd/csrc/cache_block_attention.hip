// Attention over the 4-bit cache for query blocks and chunks of prompts (more than 32 rows per KV head of a request): the
// operation, the axis of tiles and its equal shares are those of cache_attention.hip; what differs is who converts the keys.
//
// A workgroup works on one row tile of 128 rows at a time, 32 rows a wave, and its waves share the keys: a tile of 64 keys is
// converted once, 16 keys a wave and a quarter of a row a lane, into bf16 tiles of K and V in LDS, beside the matrix
// instructions of the tiles before it; codes are asked for a tile before they are converted.  One barrier a tile.  Every wave
// owns its rows, so a piece of a row tile needs no joining inside the workgroup.  Matrix instruction and operands are those of
// packed_attention.hip: with one workgroup a unit a wave has its SIMD to itself, where vector instructions are free beside
// 32x32x16 and not beside 16x16x32.  Weights are rounded to bf16 for the product with V, as in all attention here
// (cache_attention.hip).
//
// Chunks of prompts, two waves a SIMD, are bound by what a SIMD issues: matrix instructions are under way in 49 % of the cycles, vector
// instructions (exponentials, conversions of keys and of weights, maxima) in 41 % more, and little of the one runs beside the other
// (1020 TFLOP/s at 2.03 GHz; a kernel of 16x16x32 instructions, and one whose waves took K from memory each for itself, which convert
// as much or more, run at the same rate to a percent: 4 x 512 queries of 28 / 4 heads of 128 over 20000 keys 568, 568, 574 us).
// Every row tile of a head converts its keys again.  Short blocks are bound by their start (4 us), the end (3 us) and 3000 cycles a
// tile of a lone wave, of which 1024 are matrix instructions.
#include "cache_tiles.h"

namespace apbv {
namespace {

__device__ __forceinline__ f32x16 mfma32(const bf16x8 a, const bf16x8 b, const f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// A barrier that orders LDS alone: __syncthreads() also waits for the codes that are on their way to registers.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <int D, bool kLse>                                // kLse: as in cache_attention.hip
__global__ __launch_bounds__(64 * kCacheWaves, 2) void cache_block_attention_kernel(const CacheAttnParams p) {
  using T = Tile<D, 1, true>;
  constexpr int W = kCacheWaves, R = kCacheBlockRows;
  static_assert(R == 32 * W, "a wave owns 32 rows");
  constexpr int KS = D / 16;                               // matrix instructions of S^T of 32 keys
  constexpr int DB = D / 32;                               // 32-row blocks of O^T, two matrix instructions each
  constexpr int kHalf = T::TILE_BYTES;                     // 32 keys
  __shared__ __attribute__((aligned(1024))) unsigned char k_lds[2][2 * kHalf], v_lds[2][2 * kHalf];
  __shared__ __attribute__((aligned(16))) int gone_lds[4][W];                           // 16-key blocks that are not there, of a tile modulo 4

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, hh = lane >> 5;
  Axis<R> axis(p);
  const uint32_t share = axis.share(p);
  const int wg = axis.my_share(share);
  if (wg < 0) return;
  uint32_t pos = wg * share;
  const uint32_t end = share < axis.total - pos ? pos + share : axis.total;
  int b = axis.find(p, pos);
  uint32_t begin = axis.begin_of(b);

  // Per-lane LDS offsets: of K a lane converts quarter `cq` of key `ck` of its wave's 16-key block, of V quarter `vq` of key `vk`;
  // the matrix operands are read as in packed_attention.hip.  16-byte chunks of a row are swizzled by the row so that the
  // writes, too, spread over the banks: K by the row, V by its bits 0, 1 (upper) and 2, 3 (lower half of the chunk's number;
  // head_dim 64: bit 1, and 2, 3).  Rows eight further on then have the lower half differ in bit 1.
  constexpr int kPieces = D / 32;                          // 16-byte chunks of a lane's quarter row, as bf16
  auto fv = [](int r) { return (D == 128 ? (r & 3) << 2 : (r >> 1 & 1) << 2) | (r >> 2 & 3); };
  const int ck = lane >> 2, cq = lane & 3, vk = lane & 15, vq = lane >> 4;
  int k_off[KS], v_off[2][DB];
  const int k_put = (16 * wave + ck) * T::ROW_BYTES + (((cq * kPieces) ^ T::fk((16 * wave + ck) & 31)) << 4);      // ^ 16 x: chunk x
  const int v_put = (16 * wave + vk) * T::ROW_BYTES + (((vq * kPieces) ^ fv(vk)) << 4);
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) k_off[kk] = c * T::ROW_BYTES + (((2 * kk + hh) ^ T::fk(c)) << 4);
  {
    const int s = lane & 15, vrow = 4 * hh + (s >> 2);
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const int chunk = 4 * db + 2 * ((lane >> 4) & 1) + ((s & 3) >> 1);
      v_off[0][db] = vrow * T::ROW_BYTES + ((chunk ^ fv(vrow)) << 4) + (s & 1) * 8;
      v_off[1][db] = (v_off[0][db] ^ 32) + 8 * T::ROW_BYTES;
    }
  }
  const float inv_scale_log2 = 1.0f / p.scale_log2;

#pragma unroll 1
  while (pos < end) {
    const Request rq = axis.at(p, b);
    const int row_tiles = (rq.rows + R - 1) / R;
    const uint32_t of_request = (uint32_t)(row_tiles * p.hkv) * (uint32_t)rq.tiles;
    if (pos >= begin + of_request) {                       // (or a request with nothing to do)
      begin += of_request;
      ++b;
      continue;
    }
    const uint32_t rel = pos - begin, item = rel / (uint32_t)rq.tiles;
    const int head = (int)(item / (uint32_t)row_tiles), rt = (int)(item - (uint32_t)head * row_tiles);
    const int t0 = (int)(rel - item * (uint32_t)rq.tiles);
    if (rel == 0 && wave == 0) axis.leave_word(p, b, begin, share);
    const int t1 = end - pos < (uint32_t)(rq.tiles - t0) ? t0 + (int)(end - pos) : rq.tiles;
    pos += t1 - t0;

    // ---- keys that every row of the wave sees, that this lane's row sees last, that some row of the workgroup sees
    const int r_tile = rt * R, rw = r_tile + 32 * wave;
    const int queries = query_of(p, rq.rows);
    const int row = rw + c < rq.rows ? rw + c : rq.rows - 1, qi = query_of(p, row);
    const int jlast = p.causal ? rq.len - queries + qi : rq.len - 1;
    const int r_first = rw < rq.rows ? rw : rq.rows - 1;
    const int all = p.causal ? rq.len - queries + query_of(p, r_first) + 1 : rq.len;
    const int r_last = r_tile + R < rq.rows ? r_tile + R - 1 : rq.rows - 1;
    const int some = p.causal ? rq.len - queries + query_of(p, r_last) + 1 : rq.len;
    const int t_end = some <= 0 ? 0 : (t1 * kCacheKeyTile < some ? t1 : (some + kCacheKeyTile - 1) / kCacheKeyTile);

    // ---- this wave's 16 keys of a tile (past the last tile: of the last one, again).  The page is looked up a tile before its
    // codes are asked for, as the loads would wait for it.
    const int32_t* table_row = p.table + (int64_t)b * p.table_stride;
    auto token_of = [&](int t) { return (t < t_end ? t : t_end - 1) * kCacheKeyTile + 16 * wave; };
    auto look_up = [&](int t) {
      const int token = token_of(t);
      // (a vector load: a scalar one in flight turns every wait for LDS into a wait for all of them and for it)
      int at = (token < rq.len ? token : rq.len - 1) >> p.cache.page_log2;
      asm("" : "+v"(at));
      return table_row[at];
    };
    struct Place {                                         // byte offsets, and whether this lane's key, the block's first one are there
      int64_t codes, scales;
      int key_here, here;
    };
    auto locate = [&](int t, int looked_up) {
      const int page = __builtin_amdgcn_readfirstlane(looked_up);
      const int token = token_of(t);
      Place x;
      x.here = token < rq.len && (unsigned)page < (unsigned)p.cache.n_pages;
      x.key_here = rq.len - token;                         // keys of the block
      const int pg = x.here ? page : 0;
      const uint32_t at = (uint32_t)((head << p.cache.page_log2) + (token & ((1 << p.cache.page_log2) - 1)));
      x.codes = (int64_t)((uint64_t)(uint32_t)pg * (uint32_t)p.cache.stride_codes) + at * (uint32_t)(D / 2);
      x.scales = (int64_t)((uint64_t)(uint32_t)pg * (uint32_t)p.cache.stride_scales) + at * (uint32_t)(D / 32);
      return x;
    };
    Codes<D> kc, vc;
    int k_gone = 0;
    bool v_here = true;
    auto load_k = [&](const Place& x) {
      kc.load(p.cache.k_codes + x.codes, p.cache.k_scales + x.scales, 0, 0, ck, cq);
      k_gone = x.here ? 0 : 1;
    };
    auto load_v = [&](const Place& x) {
      vc.load(p.cache.v_codes + x.codes, p.cache.v_scales + x.scales, 0, 0, vk, vq);
      v_here = x.here && vk < x.key_here;
    };
    // (values of keys that are not there may be anything, and a weight of zero would not make them nothing)
    auto settle_v = [&]() { vc.scale = v_here ? vc.scale : 0u; };
    auto put_k = [&](int slot, int x) { *reinterpret_cast<u32x4*>(k_lds[slot] + (k_put ^ (x << 4))) = kc.values(x); };
    auto put_v = [&](int slot, int x) { *reinterpret_cast<u32x4*>(v_lds[slot] + (v_put ^ (x << 4))) = vc.values(x); };
    auto note_k = [&](int t) { gone_lds[t & 3][wave] = k_gone; };

    bf16x8 qf[KS];
    f32x16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
    float m_ref = -INFINITY, m_sub = 0.f, s_far = -INFINITY, l_run = 0.f, e_run = 0.f;
    const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};

    bf16x8 kf[KS];
    auto read_k = [&](int slot, int half, int kk) {
      kf[kk] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(k_lds[slot] + half * kHalf + k_off[kk]));
    };
    // the largest logit of the lane's row among 32 keys
    auto lane_max = [&](const f32x16& s) {
      float mx = __builtin_fmaxf(s[0], s[1]);
#pragma unroll
      for (int i = 2; i < 16; ++i) mx = __builtin_fmaxf(mx, s[i]);
      return mx;
    };
    // hidden keys among 32 of tile t; the largest logit again
    auto hide = [&](f32x16& s, float& lm, int t, int half, int absent) {
      if ((t + 1) * kCacheKeyTile > all || absent != 0) {
        asm volatile("" ::: "memory");                     // (a branch: as selects in every step these cost a seventh of the time)
        const int jrel = jlast - t * kCacheKeyTile - 32 * half;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (8 * (i / 4) + 4 * hh + i % 4 > jrel || (absent >> (2 * half + i / 8) & 1)) s[i] = -INFINITY;
        lm = lane_max(s);
      }
    };
    auto gone_of = [&](int t) { return *reinterpret_cast<const u32x4*>(gone_lds[t & 3]); };
    auto absent_of = [&](const u32x4& g) { return (int)__builtin_amdgcn_readfirstlane(g.x | g.y << 1 | g.z << 2 | g.w << 3); };
    // the reference maximum moves when a logit lies far above (attention.hip); the lane halves hold disjoint keys
    auto advance_reference = [&](float lm) {
      if (__builtin_amdgcn_ballot_w64(lm > s_far) != 0) {
        auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(lm), __float_as_uint(lm), false, false);
        const float mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
        const float m_new = fmaxf(m_ref, mx * p.scale_log2);
        const float alpha = m_new > -INFINITY ? __builtin_amdgcn_exp2f(m_ref - m_new) : 1.f;
        m_ref = m_new;
        m_sub = m_new > -INFINITY ? m_new : 0.f;
        s_far = (m_new + kRescaleThreshold) * inv_scale_log2;
        l_run *= alpha;
        if constexpr (kLse) e_run *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
      }
    };

    // ---- 32 keys: finishes them (S^T in sc, V in half `half` of slot `vs`) while S^T of the next 32 is formed into sn from the
    // K fragments in registers, whose successors are read from half `half` of slot `ks`.  First the KS matrix instructions of
    // S^T, then DB of O^T for the first 16 keys and DB for the second.  The exponentials run beside the first two groups, the
    // conversion of a coming tile (`convert`, a 16-byte chunk each) and the new logits' maximum beside the last, and the loads of
    // codes (`ask`) beside the first; the fences keep every instruction beside the matrix instruction it is written at.
    auto step = [&](auto ks_, auto vs_, auto half_, const f32x16& sc, f32x16& sn, float& lm, auto&& ask, auto&& convert) {
      constexpr int ks = decltype(ks_)::value, vs = decltype(vs_)::value, half = decltype(half_)::value;
      constexpr int kMfma = KS + 2 * DB, kExp = KS + DB;   // (DB chunks of a lane's quarter row)
      float xf[8][2];
      uint32_t cw[8];
      u32x4 pw[2];
      s16x4 vf[2][DB][2];
      const unsigned char* vt = v_lds[vs] + half * kHalf;
      auto stage_f = [&](int pi) {
        xf[pi][0] = __builtin_fmaf(sc[2 * pi], p.scale_log2, -m_sub);
        xf[pi][1] = __builtin_fmaf(sc[2 * pi + 1], p.scale_log2, -m_sub);
      };
      auto stage_e = [&](int pi) {
        xf[pi][0] = __builtin_amdgcn_exp2f(xf[pi][0]);
        xf[pi][1] = __builtin_amdgcn_exp2f(xf[pi][1]);
      };
      auto stage_c = [&](int pi) {
        const f32x2 xy = {xf[pi][0], xf[pi][1]};
        if constexpr (kLse) e_run += xy.x + xy.y;
        cw[pi] = __builtin_bit_cast(uint32_t, __builtin_convertvector(xy, bf16x2));
        pw[pi >> 2][pi & 3] = cw[pi];
      };
      auto stage_d = [&](int pi) {
        l_run = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, cw[pi]), bf16x2{(__bf16)1.0f, (__bf16)1.0f}, l_run, false);
      };
      static_for<kMfma>([&](auto I) {
        constexpr int i = I;
        if constexpr (i < KS) {
          sn = mfma32(kf[i], qf[i], i == 0 ? zero : sn);
          constexpr int v0 = (4 * DB * i) / KS, v1 = (4 * DB * (i + 1)) / KS;
          static_for<v1 - v0>([&](auto J) {
            constexpr int r = v0 + J, m = r / (2 * DB), db = r / 2 % DB, h = r % 2;
            vf[m][db][h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((APBV_LDS(s16x4))(vt + 16 * m * T::ROW_BYTES + v_off[h][db]));
          });
        } else {
          constexpr int m = (i - KS) / DB, db = (i - KS) % DB;
          const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(vf[m][db][0], vf[m][db][1], 0, 1, 2, 3, 4, 5, 6, 7));
          o[db] = mfma32(a, __builtin_bit_cast(bf16x8, pw[m]), o[db]);
          constexpr int k0 = (KS * (i - KS)) / (2 * DB), k1 = (KS * (i - KS + 1)) / (2 * DB);
          static_for<k1 - k0>([&](auto J) { read_k(ks, half, k0 + J); });
        }
        if constexpr (i < kExp) {
          constexpr int s0 = (16 * i) / kExp, s1 = (16 * (i + 1)) / kExp;
          static_for<s1 - s0>([&](auto J) {
            constexpr int sl = s0 + J, pi = sl / 2;
            if constexpr (sl % 2 == 0) {
              stage_f(pi);
              if constexpr (pi > 0) stage_c(pi - 1);
            } else {
              stage_e(pi);
              if constexpr (pi > 0) stage_d(pi - 1);
            }
          });
          if constexpr (i == kExp - 1) {
            stage_c(7);
            stage_d(7);
          }
        }
        if constexpr (i == 1) ask();
        if constexpr (i >= kExp) {
          convert(i - kExp);
          constexpr int m0 = (8 * (i - kExp)) / DB, m1 = (8 * (i - kExp + 1)) / DB;
          static_for<m1 - m0>([&](auto J) {
            constexpr int m = m0 + J;
            lm = m == 0 ? __builtin_fmaxf(sn[0], sn[1]) : __builtin_fmaxf(lm, __builtin_fmaxf(sn[2 * m], sn[2 * m + 1]));
          });
        }
        __builtin_amdgcn_sched_barrier(0);
      });
    };

    // ---- Tile j's body, behind a barrier in front of which K(j + 1) and V(j) have been written: the first half is finished
    // beside S^T of the second, the second beside S^T of the first half of tile j + 1; K(j + 2) and V(j + 1) go into the slots
    // that everyone has left, and the codes of K(j + 3) and V(j + 2) are asked for.  Fragments of K are read one step ahead.
    f32x16 s_a, s_b;
    int absent = 0;                                        // of the tile being worked on
    int page_k = 0;
    Place next_v;                                          // of tile t + 2, whose K is on its way
    auto body = [&](int t, auto slot_) {
      constexpr int slot = decltype(slot_)::value;
      std::integral_constant<int, slot> here;
      std::integral_constant<int, slot ^ 1> other;
      std::integral_constant<int, 0> first;
      std::integral_constant<int, 1> second;
      float lm;
      Place coming;
      lds_barrier();
      const u32x4 gone_next = gone_of(t + 1);
      step(other, here, first, s_a, s_b, lm, []() {}, [&](int x) {
        if (x == 0) note_k(t + 2);
        put_k(slot, x);
      });
      hide(s_b, lm, t, 1, absent);
      advance_reference(lm);
      step(other, here, second, s_b, s_a, lm, [&]() {
        coming = locate(t + 3, page_k);
        load_k(coming);
        page_k = look_up(t + 4);
      }, [&](int x) {
        if (x == 0) settle_v();
        put_v(slot ^ 1, x);
      });
      load_v(next_v);
      next_v = coming;
      absent = absent_of(gone_next);
      if (t + 1 < t_end) {
        hide(s_a, lm, t + 1, 0, absent);
        advance_reference(lm);
      }
    };
    if (t0 < t_end) {
      const int page0 = look_up(t0), page1 = look_up(t0 + 1), page2 = look_up(t0 + 2);
      page_k = look_up(t0 + 3);
      lds_barrier();                                       // everyone has left the last piece's tiles
      const Place place0 = locate(t0, page0), place1 = locate(t0 + 1, page1);
      load_k(place0);
      load_v(place0);
      Codes<D> next;
      next.load(p.cache.k_codes + place1.codes, p.cache.k_scales + place1.scales, 0, 0, ck, cq);
      {
        const bf16_t* qrow = p.q.ptr + (int64_t)(rq.first + qi) * p.q.st + (int64_t)(head * p.group + row - qi * p.group) * p.q.sh + 8 * hh;
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) qf[kk] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qrow + 16 * kk));
      }
      settle_v();
#pragma unroll
      for (int x = 0; x < kPieces; ++x) {
        put_k(t0 & 1, x);
        put_v(t0 & 1, x);
      }
      note_k(t0);
      kc = next;
      k_gone = place1.here ? 0 : 1;
#pragma unroll
      for (int x = 0; x < kPieces; ++x) put_k((t0 & 1) ^ 1, x);
      note_k(t0 + 1);
      next_v = locate(t0 + 2, page2);
      load_k(next_v);
      load_v(place1);
      lds_barrier();
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) read_k(t0 & 1, 0, kk);
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) s_a = mfma32(kf[kk], qf[kk], kk == 0 ? zero : s_a);
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) read_k(t0 & 1, 1, kk);
      absent = absent_of(gone_of(t0));
      float lm = lane_max(s_a);
      hide(s_a, lm, t0, 0, absent);
      advance_reference(lm);
      int t = t0;
      if (t & 1) {
        body(t, std::integral_constant<int, 1>{});
        ++t;
      }
#pragma unroll 1
      while (t < t_end) {
        body(t, std::integral_constant<int, 0>{});
        if (++t >= t_end) break;
        body(t, std::integral_constant<int, 1>{});
        ++t;
      }
    }

    // ---- the rows are done, or this workgroup's part of them: a part that begins the row tile, or one that goes on with it
    const bool whole = t0 == 0 && t1 == rq.tiles;
    const int part_slot = t0 == 0 ? 1 : 0;
    float* part = p.parts + ((int64_t)wg * 2 + part_slot) * (R * D);
    float* part_stat = part_stats(p, part_slot, R, D) + wg;
    {
      auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run), false, false);
      l_run = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    }
    if constexpr (kLse) {
      auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(e_run), __float_as_uint(e_run), false, false);
      e_run = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    }
    if (rw + c >= rq.rows) continue;
    if (whole) {
      const int h = head * p.group + row - qi * p.group;
      const float inv = l_run > 0.f ? 1.0f / l_run : 0.f;
      bf16_t* dst = p.out + ((int64_t)(rq.first + qi) * p.hq + h) * D + 4 * hh;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          u32x2 y;
          y.x = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{o[db][4 * q] * inv, o[db][4 * q + 1] * inv}), bf16x2));
          y.y = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{o[db][4 * q + 2] * inv, o[db][4 * q + 3] * inv}), bf16x2));
          *reinterpret_cast<u32x2*>(dst + 32 * db + 8 * q) = y;
        }
      if (kLse && hh == 0) p.lse[(int64_t)h * p.n_rows + rq.first + qi] = log_sum(m_ref, e_run);
    } else {
      const int in_tile = 32 * wave + c;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<f32x4*>(part + in_tile * D + 32 * db + 8 * q + 4 * hh) = f32x4{o[db][4 * q], o[db][4 * q + 1], o[db][4 * q + 2], o[db][4 * q + 3]};
      if (hh == 0) {
        part_stat[(int64_t)in_tile * p.workgroups] = m_ref;
        part_stat[(int64_t)(R + in_tile) * p.workgroups] = l_run;
        if (kLse) part_stat[(int64_t)(2 * R + in_tile) * p.workgroups] = e_run;
      }
    }
  }
}

}  // namespace

apbv_status launch_cache_block_attention(const CacheAttnParams& p, int head_dim, hipStream_t stream) {
  Launcher launch(stream);
  auto kernel = head_dim == 128 ? (p.lse ? cache_block_attention_kernel<128, true> : cache_block_attention_kernel<128, false>)
                                : (p.lse ? cache_block_attention_kernel<64, true> : cache_block_attention_kernel<64, false>);
  launch(kernel, dim3((unsigned)p.workgroups), dim3(64 * kCacheWaves), 0, p);
  return launch.status();
}

}  // namespace apbv
