// Attention behind short shared prefixes in one launch (include/apbv_shared.h; the operation and its launch for long ones are in
// shared_attention.hip).
//
// A workgroup takes 16 rows (query x head of the KV group) of a group and a KV head, and all the keys that they see: the prefix' tiles and
// behind them those of the own keys of every request that has one of the rows, hidden from the others.  That is one list of tiles,
// of which each wave takes an equal part; a wave goes from one segment to the next without a pause, as the next tile is on its way while one is
// worked on.  A tile is worked on as in cache_few_rows.h.  Nothing is cut, so nothing is left to join: bound by the chain of launch, starts,
// lengths, pages and codes, and a microsecond a tile of a wave (2 requests of 2 / 1 heads of 64 behind 700 keys, two tiles a wave, 8.0 us).  The
// rule when it is taken, and how many waves there are, stands in shared_validation.h.
//
// No workgroup has more than one row tile, and none walks over requests that are not near its rows: both are found by a search 64 ways over the
// starts, twice where there are more than 62 groups (us, with a loop over row tiles, as many workgroups for every group as the average needs, and
// over requests / so: 4096 requests of 8 / 8 heads of 128 behind 1000 prefixes of 256 keys, 3097 of them behind one, 5124 / 149, 4096 behind one 174 / 70;
// 4096 behind as many prefixes of 64 keys, ten of them with a row, 45.5 / 6.6).  The search costs a small call 0.3 us, one of 64 groups of one
// request 0.9 (6.1 / 7.0).
#include "cache_few_rows.h"
#include "shared.h"

namespace apbv {
namespace {

template <int D, bool kOnePage, bool kLse, int W>
__global__ __launch_bounds__(64 * W, 2) void shared_short_kernel(const SharedParams p) {
  using T = Tile<D, 1>;
  constexpr int R = 16;
  constexpr int kWaveLds = T::TILE_BYTES > R * D * 4 ? T::TILE_BYTES : R * D * 4;      // a wave's V tile, later its O
  __shared__ __attribute__((aligned(1024))) unsigned char lds[W][kWaveLds];
  __shared__ float stat[W][3][R];

  const CacheAttnParams& own = p.own;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int li = lane & 15, lg = lane >> 4;
  // per-lane LDS offsets: V rows as written, and as the A operand of O^T (cache_few_rows.h)
  constexpr int kPieces = D / 64 * 2;
  auto fv = [](int r) { return T::fv(r) | (((D == 128 ? r >> 2 : r) ^ r >> 3) & 1); };
  int v_put[kPieces], v_off[T::DBN];
#pragma unroll
  for (int x = 0; x < kPieces; ++x) v_put[x] = li * T::ROW_BYTES + (((lg * kPieces + x) ^ fv(li)) << 4);
  {
    const int row = 4 * lg + (li >> 2);
#pragma unroll
    for (int d = 0; d < T::DBN; ++d) v_off[d] = row * T::ROW_BYTES + (((2 * d + ((li & 3) >> 1)) ^ fv(row)) << 4) + (li & 1) * 8;
  }
  constexpr int kChunks = D / 4;
  unsigned char* vbuf = lds[wave];
  const float inv_scale_log2 = 1.0f / own.scale_log2;

  // ---- the group, or the requests in front of all groups or behind them, which have no prefix, and the row tile
  const int head = (int)(blockIdx.x % (uint32_t)own.hkv), slot = (int)(blockIdx.x / (uint32_t)own.hkv);
  const bool listed = p.prefix.members != nullptr;
  auto start_of = [&](int b) { return clip(own.starts ? scalar_load(own.starts, b) : b * own.each, own.n_rows); };
  int g, rt, from, to, first, past;                        // g: -1 in front of the groups, n_requests behind them; its requests, its queries
  if (!listed && own.starts == nullptr) {
    g = slot / p.prefix.row_tiles;
    rt = slot - g * p.prefix.row_tiles;
    from = g * p.prefix.members_each;
    to = from + p.prefix.members_each;
    first = start_of(from);
    past = start_of(to);
  } else {
    // the last that begins at or before the slot.  A wave's lanes look at where 64 of them begin, or every step-th; the last entry is where all end
    const int n = p.prefix.n_requests + (listed ? 2 : 0);
    int e = 0, top = n, step = (n + 64) / 64, begin;
#pragma unroll 1
    for (;;) {
      const int x = e + lane * step < top ? e + lane * step : top;
      const int b = !listed ? x * p.prefix.members_each : x == 0 ? 0 : x == n ? own.n_requests : clip(p.prefix.members[x - 1], own.n_requests);
      const int q = clip(own.starts ? own.starts[b] : b * own.each, own.n_rows);
      const int its_begin = first_slot(q, own.group, x);
      const uint64_t before = __builtin_amdgcn_ballot_w64(e + lane * step < top && its_begin <= slot);
      if (before == 0) return;
      const int at = 63 - __builtin_clzll(before);
      e += at * step;
      if (step == 1) {
        from = __builtin_amdgcn_readlane(b, at);
        to = __builtin_amdgcn_readlane(b, at + 1);
        first = __builtin_amdgcn_readlane(q, at);
        past = __builtin_amdgcn_readlane(q, at + 1);
        begin = __builtin_amdgcn_readlane(its_begin, at);
        break;
      }
      top = e + step < n ? e + step : n;
      step = (step + 64) / 64;
    }
    rt = slot - begin;
    g = listed ? e - 1 : e;
  }
  const int rows = (past > first ? past - first : 0) * own.group, r0 = rt * R;
  if (from >= to || r0 >= rows) return;                    // (a slot that is left over)
  const bool grouped = g >= 0 && g < p.prefix.n_requests;
  const int prefix_len = grouped ? clip(scalar_load(p.prefix.lengths, g), p.prefix.max_len) : 0;
  const int prefix_tiles = (prefix_len + kCacheKeyTile - 1) / kCacheKeyTile;
  const int32_t* prefix_row = p.prefix.table + (int64_t)(grouped ? g : 0) * p.prefix.table_stride;

  const int r = r0 + li < rows ? r0 + li : rows - 1;
  const int i = query_of(own, r), query = first + i;     // this lane's
  const int query_lo = first + query_of(own, r0), query_hi = first + query_of(own, r0 + R < rows ? r0 + R - 1 : rows - 1);
  bf16x8 qf[T::KSD];
  {
    const bf16_t* qrow = own.q.ptr + (int64_t)query * own.q.st + (int64_t)(head * own.group + r - i * own.group) * own.q.sh + lg * (D / 4);
#pragma unroll
    for (int c = 0; c < T::KSD; ++c) qf[c] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qrow + 8 * c));
  }

  // ---- requests with rows among these, a window of 64 at a time, one a lane: first query, past the last, keys, tiles.  Of more than 64 the
  // windows begin with one that begins at or before the first row (those in front of it have ended by then).
  int near = from;
  if (to - from > 64) {
    const int per = (to - from + 63) / 64, x = from + lane * per;
    const uint64_t before = __builtin_amdgcn_ballot_w64(x < to && clip(own.starts ? own.starts[x < to ? x : from] : x * own.each, own.n_rows) <= query_lo);
    near = before ? from + (63 - __builtin_clzll(before)) * per : from;
  }
  int base = near, w_first = 0, w_past = 0, w_len = 0, w_tiles = 0;
  auto window = [&](int b) {
    base = b;
    w_first = 0x7fffffff;
    w_past = w_len = w_tiles = 0;
    if (b + lane < to) {
      w_first = clip(own.starts ? own.starts[b + lane] : (b + lane) * own.each, own.n_rows);
      w_past = clip(own.starts ? own.starts[b + lane + 1] : (b + lane + 1) * own.each, own.n_rows);
      w_len = clip(own.lengths[b + lane], own.max_len);
      w_tiles = w_first < w_past && w_past > query_lo && w_first <= query_hi ? (w_len + kCacheKeyTile - 1) / kCacheKeyTile : 0;
    }
  };
  // how many tiles there are: in the windows from there to the last that begins at or before the last row
  int total = prefix_tiles;
  for (int b = near;; b += 64) {
    window(b);
    total += (int)__builtin_amdgcn_readlane(wave_scan((uint32_t)w_tiles), 63);
    if (b + 64 >= to || (int)__builtin_amdgcn_readlane(w_first, 63) > query_hi) break;
  }
  const int each = (total + W - 1) / W, u0 = wave * each < total ? wave * each : total, u1 = u0 + each < total ? u0 + each : total;

  // ---- a place in the list: request (before the first: the prefix) and tile
  struct Place {
    int b, tile, tiles, len;
  };
  auto seek = [&](Place& at, int b) {                    // to the first tile of request b, or of the next one that has any
    for (;;) {
      if (b >= to) b = to - 1;                           // (not reached: there are as many tiles as were counted)
      if ((unsigned)(b - base) >= 64u) window(near + (b - near) / 64 * 64);
      const uint64_t any = __builtin_amdgcn_ballot_w64(w_tiles > 0 && base + lane >= b);
      if (any != 0) {
        const int l = __builtin_ctzll(any);
        at.b = base + l;
        at.tile = 0;
        at.tiles = __builtin_amdgcn_readlane(w_tiles, l);
        at.len = __builtin_amdgcn_readlane(w_len, l);
        return;
      }
      b = base + 64;
      if (b >= to) {                                     // nothing left: the place stays what it was
        at.tile = at.tiles - 1;
        return;
      }
    }
  };
  auto next = [&](Place& at) {
    if (++at.tile >= at.tiles) seek(at, at.b < from ? near : at.b + 1);
  };
  auto table_of = [&](const Place& at) { return at.b < from ? prefix_row : own.table + (int64_t)at.b * own.table_stride; };

  f32x4 o[T::DBN];
#pragma unroll
  for (int d = 0; d < T::DBN; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_ref = -INFINITY, m_sub = 0.f, s_far = -INFINITY, l_run = 0.f, e_run = 0.f;

  if (u0 < u1) {
    Place here_at = {from - 1, 0, prefix_tiles, prefix_len};
    if (u0 < prefix_tiles) {
      here_at.tile = u0;
    } else {
      int skip = u0 - prefix_tiles;
      here_at.tiles = 0;
      seek(here_at, near);
      while (skip >= here_at.tiles) {
        skip -= here_at.tiles;
        seek(here_at, here_at.b + 1);
      }
      here_at.tile = skip;
    }
    Codes<D> kc[4], vc[4];
    Blocks<D, kOnePage> here;
    Place coming = here_at;                              // of smaller pages: the tile whose pages are looked up
    int next_page = 0;
    int u_find = u0;                                     // (the last tile again at the end)
    auto find = [&]() {
      if constexpr (kOnePage) {
        here.find(own, table_of(here_at), head, here_at.len, here_at.tile);
      } else {
        here.place(own, head, here_at.len, here_at.tile, next_page);
        if (u_find + 1 < u1) next(coming);
        next_page = here.look_up(own, table_of(coming), coming.len, coming.tile);
      }
    };
    auto load_k = [&]() { here.load(kc, own.cache.k_codes, own.cache.k_scales, li, lg); };
    auto load_v = [&]() { here.load(vc, own.cache.v_codes, own.cache.v_scales, li, lg); };
    if constexpr (!kOnePage) next_page = here.look_up(own, table_of(here_at), here_at.len, here_at.tile);
    find();
    load_k();
    load_v();
#pragma unroll 1
    for (int u = u0; u < u1; ++u) {
      const Blocks<D, kOnePage> now = here;
      const Place now_at = here_at;
      if (u + 1 < u1) {
        next(here_at);
        u_find = u + 1;
      }
      find();

      // ---- S^T = K Q^T, lane: keys 16 kb + 4 lg + e of row li
      f32x4 s[4];
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int c = 0; c < T::KSD; ++c)
          s[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kc[kb].values(c)), qf[c],
                                                          c == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[kb], 0, 0, 0);
      load_k();

      // ---- hidden keys: of another request than the row's, out of its sight, or not there at all, whose values may be anything
      const bool is_own = now_at.b >= from;
      if (is_own || (now_at.tile + 1) * kCacheKeyTile > now_at.len || now.absent != 0) {
        asm volatile("" ::: "memory");                   // (a branch, not selects in every tile)
        int jlast = now_at.len - 1;
        if (is_own) {
          const int b_first = start_of(now_at.b), b_past = start_of(now_at.b + 1);
          jlast = query < b_first || query >= b_past ? -1 : (own.causal ? now_at.len - b_past + query : jlast);
        }
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
          const int j = now_at.tile * kCacheKeyTile + 16 * kb;
          const bool gone = now.gone(kb);
          vc[kb].scale = gone || j + li >= now_at.len ? 0u : vc[kb].scale;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (gone || j + 4 * lg + e > jlast) s[kb][e] = -INFINITY;
        }
      }

      // ---- the reference maxima move when a logit lies far above (attention.hip)
      float mx = s[0][0];
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = __builtin_fmaxf(mx, s[kb][e]);
      if (__builtin_amdgcn_ballot_w64(mx > s_far) != 0) {
        {
          auto sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
          mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
        }
        {
          auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
          mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
        }
        const float m_new = fmaxf(m_ref, mx * own.scale_log2);
        const float alpha = m_new > -INFINITY ? __builtin_amdgcn_exp2f(m_ref - m_new) : 1.f;
        m_ref = m_new;
        m_sub = m_new > -INFINITY ? m_new : 0.f;
        s_far = (m_new + kRescaleThreshold) * inv_scale_log2;
        l_run *= alpha;
        if constexpr (kLse) e_run *= alpha;
#pragma unroll
        for (int d = 0; d < T::DBN; ++d) o[d] *= alpha;
      }

      // ---- O^T += V^T P^T, 32 keys at a time through the wave's LDS tile (LDS operations of a wave are in order)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int mb = 0; mb < 2; ++mb)
#pragma unroll
          for (int x = 0; x < kPieces; ++x)
            *reinterpret_cast<u32x4*>(vbuf + mb * 16 * T::ROW_BYTES + v_put[x]) = vc[2 * half + mb].values(x);
        u32x4 pw;
#pragma unroll
        for (int mb = 0; mb < 2; ++mb)
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            const f32x4& y = s[2 * half + mb];
            const f32x2 xy = {__builtin_amdgcn_exp2f(__builtin_fmaf(y[e], own.scale_log2, -m_sub)),
                              __builtin_amdgcn_exp2f(__builtin_fmaf(y[e + 1], own.scale_log2, -m_sub))};
            if constexpr (kLse) e_run += xy.x + xy.y;
            const bf16x2 c = __builtin_convertvector(xy, bf16x2);
            l_run = __builtin_amdgcn_fdot2_f32_bf16(c, bf16x2{(__bf16)1.0f, (__bf16)1.0f}, l_run, false);
            pw[2 * mb + (e >> 1)] = __builtin_bit_cast(uint32_t, c);
          }
        // (two reads ahead of the matrix instruction, and kept there: left to itself the compiler waits for each by itself where it has registers to save
        // for a third wave of a SIMD, 16 requests of 8 / 8 heads of 128 behind 192 keys, 64 of their own, 13.0 / 12.3 us)
        auto of_v = [&](int d) {
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((APBV_LDS(s16x4))(vbuf + v_off[d]));
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((APBV_LDS(s16x4))(vbuf + 16 * T::ROW_BYTES + v_off[d]));
          return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        };
        bf16x8 a[2] = {of_v(0), of_v(1)};
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int d = 0; d < T::DBN; ++d) {
          o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[d % 2], __builtin_bit_cast(bf16x8, pw), o[d], 0, 0, 0);
          if (d + 2 < T::DBN) a[d % 2] = of_v(d + 2);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      load_v();
    }
  }

  // ---- the waves' parts are put together
  auto over_lanes = [](float x) {
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
  const float l_tot = over_lanes(l_run), e_tot = kLse ? over_lanes(e_run) : 0.f;
  f32x4* to_lds = reinterpret_cast<f32x4*>(lds[wave]);
#pragma unroll
  for (int d = 0; d < T::DBN; ++d) to_lds[li * kChunks + ((4 * d + lg) ^ li)] = o[d];
  if (lg == 0) {
    stat[wave][0][li] = m_ref;
    stat[wave][1][li] = l_tot;
    if (kLse) stat[wave][2][li] = e_tot;
  }
  __syncthreads();
  for (int x = threadIdx.x; x < R * (D / 8); x += 64 * W) {
    const int row = x / (D / 8), c = x % (D / 8);
    if (r0 + row >= rows) break;
    float m = stat[0][0][row], l = 0.f, exact = 0.f;
#pragma unroll
    for (int w = 1; w < W; ++w) m = fmaxf(m, stat[w][0][row]);
    const float m0 = m > -INFINITY ? m : 0.f;
    f32x4 x0 = {0.f, 0.f, 0.f, 0.f}, x1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float weight = __builtin_amdgcn_exp2f(stat[w][0][row] - m0);
      l = __builtin_fmaf(stat[w][1][row], weight, l);
      if (kLse) exact = __builtin_fmaf(stat[w][2][row], weight, exact);
      const f32x4* src = reinterpret_cast<const f32x4*>(lds[w]) + row * kChunks;
      x0 += weight * src[(2 * c) ^ (row & 15)];
      x1 += weight * src[(2 * c + 1) ^ (row & 15)];
    }
    const float inv = l > 0.f ? 1.0f / l : 0.f;
    x0 *= inv;
    x1 *= inv;
    u32x4 y;
    y.x = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x0.x, x0.y}), bf16x2));
    y.y = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x0.z, x0.w}), bf16x2));
    y.z = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x1.x, x1.y}), bf16x2));
    y.w = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x1.z, x1.w}), bf16x2));
    const int q = query_of(own, r0 + row), h = head * own.group + r0 + row - q * own.group;
    *reinterpret_cast<u32x4*>(own.out + ((int64_t)(first + q) * own.hq + h) * D + 8 * c) = y;
    if (kLse && c == 0) own.lse[(int64_t)h * own.n_rows + first + q] = log_sum(m, exact);
  }
}

template <int D, int W>
auto short_kernel(const SharedParams& p) {
  if ((1 << p.own.cache.page_log2) >= kCacheKeyTile) return p.own.lse ? shared_short_kernel<D, true, true, W> : shared_short_kernel<D, true, false, W>;
  return p.own.lse ? shared_short_kernel<D, false, true, W> : shared_short_kernel<D, false, false, W>;
}

}  // namespace

apbv_status launch_shared_short(const SharedParams& p, const SharedPlan& plan, int head_dim, hipStream_t stream) {
  Launcher launch(stream);
  const int waves = plan.short_waves;
  auto kernel = waves == 8 ? (head_dim == 128 ? short_kernel<128, 8>(p) : short_kernel<64, 8>(p)) : (head_dim == 128 ? short_kernel<128, 4>(p) : short_kernel<64, 4>(p));
  launch(kernel, dim3((unsigned)(plan.slots * p.own.hkv)), dim3(64 * waves), 0, p);
  return launch.status();
}

}  // namespace apbv
