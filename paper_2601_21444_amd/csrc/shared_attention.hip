// Attention of requests that share cached prefixes (include/apbv_shared.h), for gfx950.
//
// The rows of a group are one problem over its prefix, as many rows as its requests have together: the prefix is read and converted once
// for up to 128 of them, and what it costs is matrix instructions, not bytes.  The rows of a request over its own keys are the problem of
// cache_attention.hip.  Both lie on axes of tiles of their own, cut into shares, in one launch.  A row's parts, of either
// axis, are left in float32 and joined by a second launch.
//
// Bound, behind long prefixes, by what a SIMD issues (cache_block_attention.hip): 64 questions of 16 / 2 heads of 128 behind 133120 keys
// take 90 us from a graph.  In a trace, which times each launch from its own start, the first is 84 (70 GFLOP, 835 TFLOP/s: matrix instructions
// under way in 42 % of the cycles, vector instructions in 37 % more, little of the one beside the other) and the second, which reads 34 MB of
// parts, 10; the same 64 rows as one request of apbv_cache_attention, without own keys, take 88.  256 requests of 28 / 4 heads behind 32768 keys,
// 65 to 2048 of their own 152 to 156 (122 GFLOP and 75 MB of own keys), as one request without them 132.  One launch holds two bodies, and at head_dim
// 128 the compiler spills 26 to 40 registers in the instances with row tiles of 32 or 128, where a piece begins and ends, none in the loop over
// tiles: 14 MB written beside the parts of the first call.  Tried and not kept (us, so / then): waves of 64 rows, one a SIMD
// with 512 registers, which read half of the LDS bytes, 90 / 99 and 136 / 144 (a lone wave's matrix and vector instructions do not
// overlap either, and 90 moves between the register files come with every 32 keys); workgroups for the one axis or the other by
// what they cost 205 / 238 (300 requests behind 40000 keys, up to 300 of their own); parts in the order in which lanes store them, 90.4 / 92.1.
//
// Weights are rounded to bf16 for the product with V (cache_attention.hip): outputs lie 1.9 to 2.4e-3 from those of 64 bits, root mean square,
// where float32 weights leave 1.5 to 1.7e-3, the rounding of the output alone.
//
// Behind shorter prefixes it is bound by its start, the end of the longest share and the join, 12 us with row tiles of 16 rows (shared_validation.h).
#include "cache_block_rows.h"
#include "cache_few_rows.h"
#include "shared.h"

namespace apbv {
namespace {

template <int D, int R>
struct LdsOf {
  typedef FewRowsLds<D, R / 16, false> type;
};
template <int D>
struct LdsOf<D, kCacheBlockRows> {
  typedef BlockRowsLds<D> type;
};

template <int D, int R, bool kOnePage, bool kLse, bool kGroups, typename P>
__device__ __forceinline__ void attend(const P& p, typename LdsOf<D, R>::type& lds, uint32_t block, const AxisCut& cut,
                                       const Request& of_lane) {
  if constexpr (R == kCacheBlockRows)
    attend_block_rows<D, kLse, true, kGroups>(p, lds, block, cut, of_lane);
  else
    attend_few_rows<D, R / 16, kOnePage, kLse, Form::kKept, kGroups>(p, lds, block, cut, of_lane);
}

__device__ __forceinline__ AxisCut uniform(const AxisCut& c) {       // (whole-number divisions leave the scalar registers)
  auto u = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane(x); };
  return AxisCut{u(c.stretch), u(c.share), u(c.rest), u(c.full), u(c.used)};
}

// What a share of `tiles` tiles of own keys costs, in tiles of a prefix: its start, and 64 keys of 16 rows or of a row tile.
template <int RP, int RO>
constexpr uint32_t own_cost(uint32_t tiles) {
  if (RO == kCacheBlockRows) return 2 + tiles;
  return RP == kCacheBlockRows ? 2 + tiles / 7 : 4 + tiles;
}

// Every workgroup has a share of either axis, or of one of them where they are short: those of the prefixes are dealt from each die's first
// workgroup on, those of the own keys from the last, and a workgroup that has own keys takes as much less of the prefixes as they cost
// (5 requests of 28 / 4 heads behind 10185 keys 21.4 -> 19.0 us, 64 of 16 / 2 behind 133120 92.8 -> 91.5).  Half of the workgroups begin
// with the one and half with the other (all with the own keys, 1.00 of the time over 19 calls; all with the prefixes, 1.00).
template <int D, int RP, int RO, bool kOnePage, bool kLse>
__global__ __launch_bounds__(64 * kCacheWaves, 2) void shared_attention_kernel(const SharedParams) {
  __shared__ union Lds {
    typename LdsOf<D, RP>::type prefix;
    typename LdsOf<D, RO>::type own;
    __device__ Lds() {}
  } lds;
  // (arguments are read from where they lie, when they are needed: there are too many for the scalar registers)
  typedef APBV_CONST(SharedParams) Arguments;
  Arguments args = (Arguments)__builtin_amdgcn_kernarg_segment_ptr();
  constexpr uint32_t workgroups = kSharedWorkgroups;
  AxisCut of_own, of_prefix;
  // (in LDS, where all waves write the same, until it is this axis' turn: registers are what there is least of)
  __shared__ Request of_lanes[2][64];
  const int lane = threadIdx.x & 63;
  {
    typedef Axis<RO> Own;
    typedef Axis<RP, true> Prefix;
    uint32_t own_total, prefix_total;
    if (args->own.n_requests <= 64) {                      // (there are no more groups than requests)
      const Request prefix_group = Prefix::lane_request(args->prefix), own_request = Own::lane_request(args->own);
      of_lanes[0][lane] = own_request;
      of_lanes[1][lane] = prefix_group;
      own_total = Own(args->own, own_request).total;
      prefix_total = Prefix(args->prefix, prefix_group).total;
    } else {
      const Own own_axis(args->own);
      const Prefix prefix_axis(args->prefix);
      of_lanes[0][lane] = own_axis.of_lane(args->own);
      of_lanes[1][lane] = prefix_axis.of_lane(args->prefix);
      own_total = own_axis.total;
      prefix_total = prefix_axis.total;
    }
    of_own = uniform(shared_cut(own_total, workgroups, (uint32_t)args->own.short_tiles, (uint32_t)args->own.least_tiles, 0, 0));
    of_prefix = uniform(shared_cut(prefix_total, workgroups, (uint32_t)args->prefix.short_tiles, (uint32_t)args->prefix.least_tiles,
                           own_total > 0 ? of_own.used : 0, own_cost<RP, RO>(of_own.share)));
  }
  const int begins_with = blockIdx.x < workgroups / 2 ? 1 : 0;
#pragma unroll 1
  for (int turn = 0; turn < 2; ++turn) {
    const bool on_prefix = (turn ^ begins_with) != 0;
    const uint32_t block = on_prefix ? blockIdx.x : workgroups - 1 - blockIdx.x;
    if (turn > 0) __syncthreads();                         // LDS is free again
    const AxisCut cut = {on_prefix ? of_prefix.stretch : of_own.stretch, on_prefix ? of_prefix.share : of_own.share, on_prefix ? of_prefix.rest : of_own.rest,
                         on_prefix ? of_prefix.full : of_own.full, on_prefix ? of_prefix.used : of_own.used};
    if (block / kCutDies < cut.used) {
      Arguments now = args;
      asm volatile("" : "+s"(now));
      if constexpr (RP == RO)                              // (one body for both)
        attend<D, RP, kOnePage, kLse, true>(on_prefix ? now->prefix : now->own, lds.prefix, block, cut, of_lanes[on_prefix ? 1 : 0][lane]);
      else if (on_prefix)
        attend<D, RP, kOnePage, kLse, true>(now->prefix, lds.prefix, block, cut, of_lanes[1][lane]);
      else
        attend<D, RO, kOnePage, kLse, false>(now->own, lds.own, block, cut, of_lanes[0][lane]);
    }
  }
}

// Where the parts of a row over one axis lie: of the workgroups `first` to `last`, each of which has a part of the row tile, or the row
// that one has kept whole.
struct Parts {
  int first, count;                // none: 0
  bool whole, of_axis;             // of_axis: the row is one of a request (or of a group)
  const float *rows, *stat;        // of workgroup 0 in slot 0, or of the row
  int64_t stat_step;
};
// kFew: there are 64 at most, and nothing is asked for behind a branch, so that the lookups on two axes are under way together.
template <int D, int R, bool kGroups, bool kFew>
__device__ __forceinline__ Parts parts_of(const CacheAttnParams& p, int row, int h) {
  typedef Axis<R, kGroups> A;
  const int lane = threadIdx.x & 63;
  int base = 0;
  if (!kFew && p.n_requests > 64) {                        // the last 64th of them that begins at or before the row
    const int per = (p.n_requests + 63) / 64, b = lane * per;
    const uint64_t before = __builtin_amdgcn_ballot_w64(b < p.n_requests && clip(A::first_row(p, b), p.n_rows) <= row);
    base = before ? (63 - __builtin_clzll(before)) * per : 0;
  }
  // (a window of requests, and where each begins on the axis, asked for together)
  const int mine = base + lane;
  Request rq = {0x7fffffff, 0, 0, 0};
  uint32_t begin = 0;
  const auto* left = (APBV_CONST(CutWord))p.begins;        // (through the scalar cache)
  const CutWord word = {{left->cut.stretch, left->cut.share, left->cut.rest, left->cut.full, left->cut.used}, 0, left->per_stretch, left->per_share, left->per_rest};
  if constexpr (kFew) {
    begin = p.begins[kCutWords + (mine < p.n_requests ? mine : p.n_requests - 1)];
    rq = A::lane_request(p);
  } else if (mine < p.n_requests) {
    begin = p.begins[kCutWords + mine];
    rq = A::load(p, mine);
  }
  const uint64_t before = __builtin_amdgcn_ballot_w64(rq.first <= row);
  const int at = before ? 63 - __builtin_clzll(before) : 0;
  const int first_row = __builtin_amdgcn_readlane(rq.first, at), rows = __builtin_amdgcn_readlane(rq.rows, at), tiles = __builtin_amdgcn_readlane(rq.tiles, at);
  const uint32_t its_begin = __builtin_amdgcn_readlane(begin, at);
  const int i = row - first_row;
  Parts x;
  x.of_axis = i >= 0 && i * p.group < rows;
  const int r = i * p.group + h % p.group, rt = r / R, row_tiles = (rows + R - 1) / R;
  const uint32_t from = its_begin + (uint32_t)(h / p.group * row_tiles + rt) * (uint32_t)tiles;
  // (requests that overlap, against the contract, may have left no word: whatever it says, reads stay inside the workspace)
  const uint32_t top = (uint32_t)p.workgroups - 1, first = cut_share_of(word, from), last = cut_share_of(word, from + (uint32_t)tiles - 1);
  x.first = (int)(first < top ? first : top);
  x.count = x.of_axis && tiles > 0 && last >= first ? (int)(last < top ? last : top) - x.first + 1 : 0;
  x.whole = x.count == 1;
  if (x.whole) {
    const int64_t row_at = (int64_t)row * p.hq + h, n = (int64_t)p.n_rows * p.hq;
    x.rows = p.kept + row_at * D;
    x.stat = p.kept + n * D + row_at;
    x.stat_step = n;
  } else {
    x.rows = p.parts + (x.of_axis ? r % R : 0) * D;
    x.stat = part_stats(p, 0, R, D) + (int64_t)(x.of_axis ? r % R : 0) * p.workgroups;
    x.stat_step = (int64_t)R * p.workgroups;
  }
  return x;
}

// kJoin waves per (row, head): joins the parts of the row over its prefix and over its own keys, one list, as cache_join_kernel
// those over one axis.
template <int D, int RP, int RO, int kJoin>
__global__ __launch_bounds__(256) void shared_join_kernel(const SharedParams p) {
  constexpr int kLanes = D / 4;                            // lanes that hold a row, four elements each
  constexpr int kAtOnce = 64 / kLanes;
  constexpr int kLoads = 8, kChunk = kAtOnce * kLoads;
  __shared__ float shared_max[kJoin], shared_sum[kJoin], shared_exact[kJoin];
  __shared__ f32x4 shared_acc[kJoin][kLanes];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t job = kJoin == 1 ? (int64_t)blockIdx.x * 4 + wave : (int64_t)blockIdx.x;
  if (job >= (int64_t)p.own.n_rows * p.own.hq) return;
  const int row = (int)(job / p.own.hq), h = (int)(job % p.own.hq);
  Parts a, b;
  if (p.own.n_requests <= 64) {                            // (there are no more groups than requests)
    a = parts_of<D, RP, true, true>(p.prefix, row, h);
    b = parts_of<D, RO, false, true>(p.own, row, h);
  } else {
    a = parts_of<D, RP, true, false>(p.prefix, row, h);
    b = parts_of<D, RO, false, false>(p.own, row, h);
  }
  if (!b.of_axis) return;                                  // a row of no request
  const int sub = lane / kLanes, c = lane % kLanes;
  const bool with_lse = p.own.lse != nullptr;
  // part n of the list: its statistics, and its row
  auto stat_of = [&](int n, int64_t& step) {
    const bool own = n >= a.count;
    const int w = own ? b.first + n - a.count : a.first + n;
    const bool whole = own ? b.whole : a.whole, begins = n == 0 || n == a.count;
    const int64_t slot = (int64_t)(3 * (own ? RO : RP)) * p.own.workgroups;
    step = own ? b.stat_step : a.stat_step;
    return (own ? b.stat : a.stat) + (whole ? 0 : w + (begins ? slot : 0));
  };
  auto row_of = [&](int n) {
    const bool own = n >= a.count;
    const int w = own ? b.first + n - a.count : a.first + n;
    const bool whole = own ? b.whole : a.whole, begins = n == 0 || n == a.count;
    return (own ? b.rows : a.rows) + (whole ? 0 : (2 * (int64_t)w + (begins ? 1 : 0)) * ((own ? RO : RP) * D));
  };
  const int count = a.count + b.count, each = (count + kJoin - 1) / kJoin;
  const int from_part = kJoin == 1 ? 0 : wave * each, past_part = from_part + each < count ? from_part + each : count;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f, exact = 0.f;
  for (int base = from_part; base < past_part; base += kChunk) {
    const bool mine = lane < kChunk && base + lane < past_part;
    int64_t step;
    const float* s = stat_of(mine ? base + lane : base, step);
    const float m_part = mine ? s[0] : -INFINITY, l_part = mine ? s[step] : 0.f;
    const float exact_part = mine && with_lse ? s[2 * step] : 0.f;
    f32x4 x[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int n = base + u * kAtOnce + sub;
      x[u] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (n < past_part) x[u] = *reinterpret_cast<const f32x4*>(row_of(n) + 4 * c);
    }
    float top = m_part;
#pragma unroll
    for (int d = 1; d < kChunk; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    top = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(fmaxf(top, m))));
    const float m0 = top > -INFINITY ? top : 0.f;
    const float old = __builtin_amdgcn_exp2f(m - m0), weight = __builtin_amdgcn_exp2f(m_part - m0);
    m = top;
    l = __builtin_fmaf(l, old, weight * l_part);           // (this lane's parts; the lanes are added up below)
    exact = __builtin_fmaf(exact, old, weight * exact_part);
    acc *= old;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) acc += __shfl(weight, u * kAtOnce + sub) * x[u];
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) l += __shfl_xor(l, d);
  if (with_lse)
#pragma unroll
    for (int d = 1; d < 64; d *= 2) exact += __shfl_xor(exact, d);
#pragma unroll
  for (int d = kLanes; d < 64; d *= 2)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], d);
  if constexpr (kJoin > 1) {
    if (lane == 0) shared_max[wave] = m, shared_sum[wave] = l, shared_exact[wave] = exact;
    if (sub == 0) shared_acc[wave][c] = acc;
    __syncthreads();
    if (wave != 0) return;
    m = -INFINITY;
#pragma unroll
    for (int w = 0; w < kJoin; ++w) m = fmaxf(m, shared_max[w]);
    const float m0 = m > -INFINITY ? m : 0.f;
    l = exact = 0.f;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kJoin; ++w) {
      const float weight = __builtin_amdgcn_exp2f(shared_max[w] - m0);
      l = __builtin_fmaf(shared_sum[w], weight, l);
      exact = __builtin_fmaf(shared_exact[w], weight, exact);
      acc += weight * shared_acc[w][c];
    }
  }
  if (sub != 0) return;
  const float inv = l > 0.f ? 1.0f / l : 0.f;
  u32x2 y;
  y.x = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{acc.x * inv, acc.y * inv}), bf16x2));
  y.y = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{acc.z * inv, acc.w * inv}), bf16x2));
  *reinterpret_cast<u32x2*>(p.own.out + job * D + 4 * c) = y;
  if (with_lse && lane == 0) p.own.lse[(int64_t)h * p.own.n_rows + row] = log_sum(m, exact);
}

template <int D, int RP, int RO>
void launch_rows(Launcher& launch, const SharedParams& p, int waves) {
  const bool one_page = (1 << p.own.cache.page_log2) >= kCacheKeyTile, lse = p.own.lse != nullptr;
  auto kernel = one_page ? (lse ? shared_attention_kernel<D, RP, RO, true, true> : shared_attention_kernel<D, RP, RO, true, false>)
                         : (lse ? shared_attention_kernel<D, RP, RO, false, true> : shared_attention_kernel<D, RP, RO, false, false>);
  launch(kernel, dim3(kSharedWorkgroups), dim3(64 * kCacheWaves), 0, p);
  const int64_t rows = (int64_t)p.own.n_rows * p.own.hq;
  if (waves == 4)
    launch(shared_join_kernel<D, RP, RO, 4>, dim3((unsigned)rows), dim3(256), 0, p);
  else
    launch(shared_join_kernel<D, RP, RO, 1>, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, p);
}
template <int D>
apbv_status launch_dim(const SharedParams& p, const SharedPlan& plan, hipStream_t stream) {
  Launcher launch(stream);
  if (plan.prefix.rows == 16)
    launch_rows<D, 16, 16>(launch, p, plan.join_waves);
  else if (plan.prefix.rows == 32)
    launch_rows<D, 32, 16>(launch, p, plan.join_waves);
  else if (plan.own.rows == 16)
    launch_rows<D, kCacheBlockRows, 16>(launch, p, plan.join_waves);
  else
    launch_rows<D, kCacheBlockRows, kCacheBlockRows>(launch, p, plan.join_waves);
  return launch.status();
}

}  // namespace

apbv_status launch_shared_attention(const SharedParams& p, const SharedPlan& plan, int head_dim, hipStream_t stream) {
  if (plan.whole) return launch_shared_short(p, plan, head_dim, stream);
  return head_dim == 128 ? launch_dim<128>(p, plan, stream) : launch_dim<64>(p, plan, stream);
}

}  // namespace apbv
