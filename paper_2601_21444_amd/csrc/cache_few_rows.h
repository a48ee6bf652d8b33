// Few rows of many requests over the cache (device code): the work of a workgroup of cache_attention.hip, where the operation and
// what bounds it are described, and of shared_attention.hip.
#pragma once
#include "cache_tiles.h"

namespace apbv {
namespace {

enum : int { kHead = 1, kTail = 2, kSpan = 4 };            // what a wave keeps of row tiles that are not its own alone

// kCut: shares of the axis; kWhole: a workgroup takes one whole (request, KV head, row tile), its waves a quarter of the keys each, and
// nothing is left to join; kKept: shares of the axis, and whole row tiles are kept in float32 as well (CacheAttnParams::kept).
enum class Form { kCut, kWhole, kKept };

template <int D, int NQ, bool kWhole>
struct FewRowsLds {
  static constexpr int W = kCacheWaves, R = 16 * NQ;
  // a wave's V tile, later its last piece's O; its first piece's O where it goes on to others (two blocks of rows leave no room
  // for it in LDS: in the workspace)
  static constexpr int kWave = Tile<D, 1>::TILE_BYTES > R * D * 4 ? Tile<D, 1>::TILE_BYTES : R * D * 4;
  __attribute__((aligned(1024))) unsigned char lds[NQ == 1 && !kWhole ? 2 : 1][W][kWave];      // [tails, heads]
  float stat[2][W][3][R];                                  // [tails, heads][wave][maximum, row sum, exact row sum]
  __attribute__((aligned(16))) int kept[W], place[2][W][4];                 // place: first query, rows, KV head, first row
};

// kLse: the log-sum-exp is wanted, and the weights are added up before they are rounded, too: their rounded sum, which the
// output is divided by, would leave it with errors of 2^-9 over the square root of the number of keys.
// `block`: which share; kKept: of this cut, which has it.
template <int D, int NQ, bool kOnePage, bool kLse, Form kForm, bool kGroups = false, typename P>
__device__ __forceinline__ void attend_few_rows(const P& p, FewRowsLds<D, NQ, kForm == Form::kWhole>& shared, uint32_t block,
                                                const AxisCut& cut, const Request& of_lane) {
  using T = Tile<D, 1>;
  constexpr int W = kCacheWaves, R = 16 * NQ;
  constexpr bool kWhole = kForm == Form::kWhole, kKept = kForm == Form::kKept;
  constexpr bool kHeadsInLds = NQ == 1 || kWhole;          // (a whole row tile's last piece is its wave's only one)
  auto& lds = shared.lds;
  auto& stat = shared.stat;
  auto& kept = shared.kept;
  auto& place = shared.place;

  int lane = threadIdx.x & 63;
  if constexpr (kKept) asm volatile("" : "+v"(lane));       // (what follows from it is not kept in registers across the work of the other axis)
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int li = lane & 15, lg = lane >> 4, thread = kKept ? 64 * wave + lane : (int)threadIdx.x;
  int keeps = 0, wg = 0;

  // per-lane LDS offsets: V rows as written, and as the A operand of O^T (query_attention.hip)
  constexpr int kPieces = D / 64 * 2;                      // 16-byte chunks of a lane's quarter row
  // (the lowest bit spreads the writes: of eight rows, which go together, over eight chunks of 128 bytes, of sixteen over all)
  auto fv = [](int r) { return T::fv(r) | (((D == 128 ? r >> 2 : r) ^ r >> 3) & 1); };
  int v_put[kPieces], v_off[T::DBN];
#pragma unroll
  for (int x = 0; x < kPieces; ++x) v_put[x] = li * T::ROW_BYTES + (((lg * kPieces + x) ^ fv(li)) << 4);
  {
    const int row = 4 * lg + (li >> 2);
#pragma unroll
    for (int d = 0; d < T::DBN; ++d) v_off[d] = row * T::ROW_BYTES + (((2 * d + ((li & 3) >> 1)) ^ fv(row)) << 4) + (li & 1) * 8;
  }
  constexpr int kChunks = D / 4;                           // 16-byte chunks of a kept row of O, swizzled by the row
  unsigned char* vbuf = lds[0][wave];
  const float inv_scale_log2 = 1.0f / p.scale_log2;

  auto head_global = [&]() { return p.parts + (int64_t)p.workgroups * 2 * (R * (D + 3)) + (int64_t)wg * W * (R * D); };
  // Where a wave keeps O of a piece.
  auto with_kept = [&](int is_head, int w, auto&& f) {
    if constexpr (kHeadsInLds)
      f(reinterpret_cast<f32x4*>(lds[kWhole ? 0 : is_head][w]));
    else if (is_head)
      f(reinterpret_cast<f32x4*>(head_global() + (int64_t)w * (R * D)));
    else
      f(reinterpret_cast<f32x4*>(lds[0][w]));
  };

  // ---- tiles t0 to t1 - 1 of row tile rt of a request and KV head, by this wave
  auto piece = [&](const Request& rq, int b, int head, int rt, int t0, int t1) {
    // ---- the row tile's rows: keys each sees, and Q^T fragments (k-step c of lane lg: elements lg * D / 4 + 8 c ...)
    const int r0 = rt * R;
    const int queries = query_of(p, rq.rows);
    bf16x8 qf[T::KSD][NQ];
    int jlast[NQ];
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      const int r = r0 + 16 * nq + li < rq.rows ? r0 + 16 * nq + li : rq.rows - 1;
      const int i = query_of(p, r);
      jlast[nq] = p.causal ? rq.len - queries + i : rq.len - 1;
      const bf16_t* qrow = p.q.ptr + (int64_t)(rq.first + i) * p.q.st + (int64_t)(head * p.group + r - i * p.group) * p.q.sh + lg * (D / 4);
#pragma unroll
      for (int c = 0; c < T::KSD; ++c) qf[c][nq] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qrow + 8 * c));
    }
    // keys that every row sees, keys that some row sees
    const int all = p.causal ? rq.len - queries + query_of(p, r0) + 1 : rq.len;
    const int last_row = r0 + R < rq.rows ? r0 + R - 1 : rq.rows - 1;
    const int some = p.causal ? rq.len - queries + query_of(p, last_row) + 1 : rq.len;
    const int t_end = some <= 0 ? 0 : (t1 * kCacheKeyTile < some ? t1 : (some + kCacheKeyTile - 1) / kCacheKeyTile);

    f32x4 o[T::DBN][NQ];
    float m_ref[NQ], m_sub[NQ], s_far[NQ], l_run[NQ], e_run[NQ];
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
#pragma unroll
      for (int d = 0; d < T::DBN; ++d) o[d][nq] = f32x4{0.f, 0.f, 0.f, 0.f};
      m_ref[nq] = s_far[nq] = -INFINITY;
      m_sub[nq] = l_run[nq] = e_run[nq] = 0.f;
    }

    const int32_t* table_row = p.table + (int64_t)b * p.table_stride;
    // One tile is on its way while one is worked on.  (Two, us, with / without: one query over 133120 keys, 16 / 2 heads of 128 18.5 /
    // 17.9; 64 requests of 512 to 32768, 28 / 4 heads 51.0 / 48.9; 256 of 65 to 1200 24.2 / 21.5; 256 of 65 to 2048, 8 / 2 heads of 64,
    // pages of 32 14.7 / 13.6; 64 of 2048, pages of 64 10.9 / 10.9.)
    Codes<D> kc[4], vc[4];
    Blocks<D, kOnePage> here;
    auto tile = [&](int t) { return t < t_end ? t : t_end - 1; };          // (the last tile again)
    int next_page = 0;                                     // of smaller pages: looked up for the next tile to find
    auto find = [&](int t) {
      if constexpr (kOnePage) {
        here.find(p, table_row, head, rq.len, tile(t));
      } else {
        here.place(p, head, rq.len, tile(t), next_page);
        next_page = here.look_up(p, table_row, rq.len, tile(t + 1));
      }
    };
    auto load_k = [&]() { here.load(kc, p.cache.k_codes, p.cache.k_scales, li, lg); };
    auto load_v = [&]() { here.load(vc, p.cache.v_codes, p.cache.v_scales, li, lg); };
    if (t0 < t_end) {
      if constexpr (!kOnePage) next_page = here.look_up(p, table_row, rq.len, t0);
      find(t0);
      load_k();
      load_v();
    }
#pragma unroll 1
    for (int t = t0; t < t_end; ++t) {
      const Blocks<D, kOnePage> now = here;
      find(t + 1);

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
      load_k();

      // ---- hidden keys: out of sight of a row, or not there at all, whose values may be anything
      if ((t + 1) * kCacheKeyTile > all || now.absent != 0) {
        asm volatile("" ::: "memory");                     // (a branch, not selects in every tile)
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
          if constexpr (kLse) e_run[nq] *= alpha;
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
              if constexpr (kLse) e_run[nq] += xy.x + xy.y;
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
      load_v();
    }

    // ---- a piece that is a whole row tile is done; others are kept for the waves' pieces to be put together below
    auto over_quarters = [](float x) {
      {
        auto sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
      }
      {
        auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
      }
      return x;
    };
    float l_tot[NQ], e_tot[NQ];
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      l_tot[nq] = over_quarters(l_run[nq]);
      e_tot[nq] = kLse ? over_quarters(e_run[nq]) : 0.f;
    }
    if (t0 == 0 && t1 == rq.tiles) {
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) {
        const int row = r0 + 16 * nq + li;
        if (row >= rq.rows) continue;
        const int i = query_of(p, row), h = head * p.group + row - i * p.group;
        if constexpr (kKept) {
          const int64_t at = (int64_t)(rq.first + i) * p.hq + h;
#pragma unroll
          for (int d = 0; d < T::DBN; ++d) *reinterpret_cast<f32x4*>(p.kept + at * D + 16 * d + 4 * lg) = o[d][nq];
          if (lg == 0) keep_stats<D, kLse>(p, at, m_ref[nq], l_tot[nq], e_tot[nq]);
          continue;
        }
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
        if (kLse && lg == 0) p.lse[(int64_t)h * p.n_rows + rq.first + i] = log_sum(m_ref[nq], e_tot[nq]);
      }
    } else {
      // (a row tile that ends here but began before is a head; one that goes on, a tail or, of one that began before, a span)
      const int is_head = t1 == rq.tiles ? 1 : 0;
      with_kept(is_head, wave, [&](f32x4* to) {
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
          for (int d = 0; d < T::DBN; ++d) to[(16 * nq + li) * kChunks + ((4 * d + lg) ^ li)] = o[d][nq];
      });
      if (lg == 0) {
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
          stat[is_head][wave][0][16 * nq + li] = m_ref[nq];
          stat[is_head][wave][1][16 * nq + li] = l_tot[nq];
          if (kLse) stat[is_head][wave][2][16 * nq + li] = e_tot[nq];
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
  };

  // ---- the pieces of a row tile that lie in consecutive waves, one chain of them after the other: chain 0 goes on with a row
  // tile that began before this workgroup, chain c begins with the tail of wave c - 1
  auto put_together = [&]() {
    if (lane == 0) kept[wave] = keeps;
    __syncthreads();
    int heads = 0, tails = 0, spans = 0;                     // a bit a wave
  #pragma unroll
    for (int w = 0; w < W; ++w) {
      const int k = __builtin_amdgcn_readfirstlane(kept[w]);
      heads |= (k & kHead ? 1 : 0) << w;
      tails |= (k & kTail ? 1 : 0) << w;
      spans |= (k & kSpan ? 1 : 0) << w;
    }
  #pragma unroll 1
    for (int chain = kWhole ? 1 : 0; chain <= (kWhole ? 1 : W); ++chain) {
      const int from = chain == 0 ? 0 : chain - 1;
      if (((chain == 0 ? heads | spans : tails) >> from & 1) == 0) continue;
      int to = from;                                         // its last wave
      bool ends = chain == 0 && (heads & 1);
      while (!ends && to + 1 < W) {
        if (heads >> (to + 1) & 1) ends = true;
        else if ((spans >> (to + 1) & 1) == 0) break;        // a wave without a share: the workgroup ends here
        ++to;
      }
      const bool whole = kWhole || (chain > 0 && ends);
      const int* at = place[ends && to == from ? 1 : 0][from];
      const int first = at[0], rows = at[1], head = at[2], r0 = at[3];
      const int slot = chain > 0 ? 1 : 0;                    // a part that begins a row tile, or one that goes on with it
      float* part = p.parts + ((int64_t)wg * 2 + slot) * (R * D);
      float* part_stat = part_stats(p, slot, R, D) + wg;
      for (int x = thread; x < R * (D / 8); x += 64 * W) {
        const int row = x / (D / 8), c = x % (D / 8);
        if (r0 + row >= rows) break;
        // (all waves' statistics, then all waves' rows, are read at once, those of others than the chain's left out)
        float m_of[W], l = 0.f, exact = 0.f, m = -INFINITY;
  #pragma unroll
        for (int w = 0; w < W; ++w) {
          m_of[w] = stat[w == to && ends ? 1 : 0][w][0][row];
          m_of[w] = w >= from && w <= to ? m_of[w] : -INFINITY;
          m = fmaxf(m, m_of[w]);
        }
        const float m0 = m > -INFINITY ? m : 0.f;
        f32x4 x0 = {0.f, 0.f, 0.f, 0.f}, x1 = {0.f, 0.f, 0.f, 0.f};
  #pragma unroll
        for (int w = 0; w < W; ++w) {
          if (w < from || w > to) continue;
          const int is_head = w == to && ends ? 1 : 0;
          const float weight = __builtin_amdgcn_exp2f(m_of[w] - m0);
          l = __builtin_fmaf(stat[is_head][w][1][row], weight, l);
          if (kLse) exact = __builtin_fmaf(stat[is_head][w][2][row], weight, exact);
          with_kept(is_head, w, [&](const f32x4* src) {
            src += row * kChunks;
            x0 += weight * src[(2 * c) ^ (row & 15)];
            x1 += weight * src[(2 * c + 1) ^ (row & 15)];
          });
        }
        if (kKept && whole) {
          const int i = query_of(p, r0 + row), h = head * p.group + r0 + row - i * p.group;
          const int64_t at = (int64_t)(first + i) * p.hq + h;
          *reinterpret_cast<f32x4*>(p.kept + at * D + 8 * c) = x0;
          *reinterpret_cast<f32x4*>(p.kept + at * D + 8 * c + 4) = x1;
          if (c == 0) keep_stats<D, kLse>(p, at, m, l, exact);
        } else if (whole) {
          const float inv = l > 0.f ? 1.0f / l : 0.f;
          x0 *= inv;
          x1 *= inv;
          u32x4 y;
          y.x = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x0.x, x0.y}), bf16x2));
          y.y = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x0.z, x0.w}), bf16x2));
          y.z = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x1.x, x1.y}), bf16x2));
          y.w = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x1.z, x1.w}), bf16x2));
          const int i = query_of(p, r0 + row), h = head * p.group + r0 + row - i * p.group;
          *reinterpret_cast<u32x4*>(p.out + ((int64_t)(first + i) * p.hq + h) * D + 8 * c) = y;
          if (kLse && c == 0) p.lse[(int64_t)h * p.n_rows + first + i] = log_sum(m, exact);
        } else {
          f32x4* dst = reinterpret_cast<f32x4*>(part + row * D + 8 * c);
          dst[0] = x0;
          dst[1] = x1;
          if (c == 0) {
            part_stat[(int64_t)row * p.workgroups] = m;
            part_stat[(int64_t)(R + row) * p.workgroups] = l;
            if (kLse) part_stat[(int64_t)(2 * R + row) * p.workgroups] = exact;
          }
        }
      }
    }
  };

  if constexpr (kWhole) {
    const int head = (int)(block % (uint32_t)p.hkv), rest = (int)(block / (uint32_t)p.hkv), b = rest / p.row_tiles;
    const int first = p.starts ? scalar_load(p.starts, b) : b * p.each, past = p.starts ? scalar_load(p.starts, b + 1) : (b + 1) * p.each;
    const Request rq = request_of(p, first, past, scalar_load(p.lengths, b));
    const int per_wave = (rq.tiles + W - 1) / W, t0 = wave * per_wave, t1 = t0 + per_wave < rq.tiles ? t0 + per_wave : rq.tiles;
#pragma unroll 1
    for (int rt = rest % p.row_tiles; rt * R < rq.rows; rt += p.row_tiles) {       // (one, unless max_q is too small)
      keeps = 0;
      if (t0 < t1) piece(rq, b, head, rt, t0, t1);
      put_together();
      if (rq.tiles == 0)
        for (int x = thread; x < R * (D / 8); x += 64 * W) {
          const int row = rt * R + x / (D / 8), c = x % (D / 8);
          if (row >= rq.rows) break;
          const int i = query_of(p, row), h = head * p.group + row - i * p.group;
          *reinterpret_cast<u32x4*>(p.out + ((int64_t)(rq.first + i) * p.hq + h) * D + 8 * c) = u32x4{0u, 0u, 0u, 0u};
          if (kLse && c == 0) p.lse[(int64_t)h * p.n_rows + rq.first + i] = -INFINITY;
        }
      __syncthreads();                                     // LDS is free again
    }
  } else {
    typedef Axis<R, kGroups> A;
    A axis = kKept ? A(p, of_lane) : A(p);
    uint32_t wg_begin, wg_end, share = 0;
    if constexpr (kKept) {
      const uint32_t die = block % kCutDies, x = block / kCutDies, past = cut_end(cut, die, x);
      wg_begin = cut_begin(cut, die, x);
      wg_end = past < axis.total ? past : axis.total;
      if (wg_begin >= wg_end) return;
      wg = (int)(die * cut.used + x);
    } else {
      share = axis.share(p);
      wg = axis.my_share(share, block);
      if (wg < 0) return;
      wg_begin = wg * share;
      wg_end = share < axis.total - wg_begin ? wg_begin + share : axis.total;
    }
    // a wave's part of the share
    const uint32_t wave_share = (wg_end - wg_begin + W - 1) / W;
    uint32_t pos = wg_begin + wave * wave_share;
    const uint32_t end = pos + wave_share < wg_end ? pos + wave_share : wg_end;
    int b = 0;
    uint32_t begin = 0;
    if (pos < end) {
      b = axis.find(p, pos);
      begin = axis.begin_of(b);
    }
#pragma unroll 1
    while (pos < end) {
      const Request rq = axis.at(p, b);
      const int row_tiles = (rq.rows + R - 1) / R;
      const uint32_t of_request = (uint32_t)(row_tiles * p.hkv) * (uint32_t)rq.tiles;
      if (pos >= begin + of_request) {                     // (or a request with nothing to do)
        begin += of_request;
        ++b;
        continue;
      }
      const uint32_t rel = pos - begin, item = rel / (uint32_t)rq.tiles;
      const int head = (int)(item / (uint32_t)row_tiles), rt = (int)(item - (uint32_t)head * row_tiles);
      const int t0 = (int)(rel - item * (uint32_t)rq.tiles);
      if (rel == 0) {
        if constexpr (kKept)
          axis.leave_word(p, b, begin, cut);
        else
          axis.leave_word(p, b, begin, share);
      }
      const int t1 = end - pos < (uint32_t)(rq.tiles - t0) ? t0 + (int)(end - pos) : rq.tiles;
      pos += t1 - t0;
      piece(rq, b, head, rt, t0, t1);
    }
    put_together();
  }
}

}  // namespace
}  // namespace apbv
