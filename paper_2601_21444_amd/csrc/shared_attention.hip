// Attention of requests that share cached prefixes (include/apbv_shared.h), for gfx950.
//
// The rows of a group are one problem over its prefix, as many rows as its requests have together: the prefix is read and converted once
// for up to 128 of them, and what it costs is matrix instructions, not bytes.  The rows of a request over its own keys are the problem of
// cache_attention.hip.  Both lie on axes of tiles of their own, cut into equal shares, and run in one launch: as many workgroups
// as their tiles cost take shares of the one axis and the others of the other, so that what is bound by matrix instructions runs beside
// what is bound by memory.  A row's parts, of either axis, are left in float32 and joined by a second launch.
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

template <int D, int R, bool kOnePage, bool kLse, bool kGroups>
__device__ __forceinline__ void attend(const CacheAttnParams& p, typename LdsOf<D, R>::type& lds, uint32_t block, uint32_t workgroups) {
  if constexpr (R == kCacheBlockRows)
    attend_block_rows<D, kLse, true, kGroups>(p, lds, block, workgroups);
  else
    attend_few_rows<D, R / 16, kOnePage, kLse, Form::kKept, kGroups>(p, lds, block, workgroups);
}

// What a tile of 64 keys costs, R rows.
constexpr uint64_t tile_cost(int rows) { return rows == kCacheBlockRows ? 3 : 1; }

template <int D, int RP, int RO, bool kOnePage, bool kLse>
__global__ __launch_bounds__(64 * kCacheWaves, 2) void shared_attention_kernel(const SharedParams p) {
  __shared__ union Lds {
    typename LdsOf<D, RP>::type prefix;
    typename LdsOf<D, RO>::type own;
    __device__ Lds() {}
  } lds;
  const uint32_t workgroups = (uint32_t)p.own.workgroups;
  const uint64_t prefix_cost = Axis<RP, true>(p.prefix).total * tile_cost(RP), own_cost = Axis<RO>(p.own).total * tile_cost(RO);
  const uint32_t of_prefix = shared_split(workgroups, prefix_cost, own_cost);
  if constexpr (RP == RO) {
    const bool on_prefix = blockIdx.x < of_prefix;         // (one body for both)
    attend<D, RP, kOnePage, kLse, true>(on_prefix ? p.prefix : p.own, lds.prefix, on_prefix ? blockIdx.x : blockIdx.x - of_prefix,
                                        on_prefix ? of_prefix : workgroups - of_prefix);
  } else if (blockIdx.x < of_prefix)
    attend<D, RP, kOnePage, kLse, true>(p.prefix, lds.prefix, blockIdx.x, of_prefix);
  else
    attend<D, RO, kOnePage, kLse, false>(p.own, lds.own, blockIdx.x - of_prefix, workgroups - of_prefix);
}

// Where the parts of a row over one axis lie: workgroups `first` to `last`, each with a part of the row tile, or the row kept whole.
struct Parts {
  int first, last;                 // last < first: none
  bool whole;
  const float *rows, *stat;        // of workgroup 0 in slot 0, or of the row
  int64_t stat_step, slot_rows, slot_stat;
};
template <int D, int R, bool kGroups>
__device__ __forceinline__ Parts parts_of(const CacheAttnParams& p, int row, int h) {
  Parts x;
  x.first = 0;
  x.last = -1;
  x.whole = false;
  Axis<R, kGroups> axis(p, typename Axis<R, kGroups>::RowsOnly{});
  const int b = axis.find_row(p, row);
  const Request rq = axis.at(p, b);
  const int i = row - rq.first;
  if (i < 0 || i * p.group >= rq.rows || rq.tiles == 0) return x;
  const uint32_t share = (uint32_t)scalar_load(reinterpret_cast<const int32_t*>(p.begins), 0);
  const uint32_t begin = (uint32_t)scalar_load(reinterpret_cast<const int32_t*>(p.begins), 1 + b);
  const int r = i * p.group + h % p.group, rt = r / R, row_tiles = (rq.rows + R - 1) / R;
  const uint32_t from = begin + (uint32_t)(h / p.group * row_tiles + rt) * (uint32_t)rq.tiles;
  // (requests that overlap, against the contract, may have left no word: whatever it says, reads stay inside the workspace)
  const uint32_t each = share > 0 ? share : 1, top = (uint32_t)p.workgroups - 1;
  const uint32_t first = from / each, last = (from + (uint32_t)rq.tiles - 1) / each;
  x.first = (int)(first < top ? first : top);
  x.last = (int)(last < top ? last : top);
  x.whole = x.first == x.last;
  if (x.whole) {
    const int64_t at = (int64_t)row * p.hq + h, n = (int64_t)p.n_rows * p.hq;
    x.rows = p.kept + at * D;
    x.stat = p.kept + n * D + at;
    x.stat_step = n;
  } else {
    x.rows = p.parts + (r % R) * D;
    x.stat = part_stats(p, 0, R, D) + (int64_t)(r % R) * p.workgroups;
    x.stat_step = (int64_t)R * p.workgroups;
  }
  x.slot_rows = R * D;
  x.slot_stat = (int64_t)(3 * R) * p.workgroups;
  return x;
}

// A wave per (row, head), four a workgroup: joins the parts of the row over its prefix and over its own keys, as cache_join_kernel
// those over one.
template <int D, int RP, int RO>
__global__ __launch_bounds__(256) void shared_join_kernel(const SharedParams p) {
  constexpr int kLanes = D / 4;                            // lanes that hold a row, four elements each
  constexpr int kAtOnce = 64 / kLanes;
  const int lane = threadIdx.x & 63;
  const int64_t job = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (job >= (int64_t)p.own.n_rows * p.own.hq) return;
  const int row = (int)(job / p.own.hq), h = (int)(job % p.own.hq);
  {                                                        // a row of no request?
    Axis<RO> axis(p.own, typename Axis<RO>::RowsOnly{});
    const Request rq = axis.at(p.own, axis.find_row(p.own, row));
    if (row < rq.first || (row - rq.first) * p.own.group >= rq.rows) return;
  }
  const int sub = lane / kLanes, c = lane % kLanes;
  const bool with_lse = p.own.lse != nullptr;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f, exact = 0.f;
  auto add = [&](const Parts& x) {
    constexpr int kLoads = 8, kChunk = kAtOnce * kLoads;
    for (int base = x.first; base <= x.last; base += kChunk) {
      const int w = base + lane;
      const bool mine = lane < kChunk && w <= x.last;
      const float* s = x.stat + (x.whole ? 0 : w + (w == x.first ? x.slot_stat : 0));
      const float m_part = mine ? s[0] : -INFINITY, l_part = mine ? s[x.stat_step] : 0.f;
      const float exact_part = mine && with_lse ? s[2 * x.stat_step] : 0.f;
      f32x4 y[kLoads];
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        const int v = base + u * kAtOnce + sub;
        y[u] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (v <= x.last) y[u] = *reinterpret_cast<const f32x4*>(x.rows + 4 * c + (x.whole ? 0 : (2 * (int64_t)v + (v == x.first ? 1 : 0)) * x.slot_rows));
      }
      float top = m_part;
#pragma unroll
      for (int d = 1; d < kChunk; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
      top = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(fmaxf(top, m))));
      const float m0 = top > -INFINITY ? top : 0.f;
      const float old = __builtin_amdgcn_exp2f(m - m0), weight = __builtin_amdgcn_exp2f(m_part - m0);
      m = top;
      l = __builtin_fmaf(l, old, weight * l_part);         // (this lane's parts; the lanes are added up below)
      exact = __builtin_fmaf(exact, old, weight * exact_part);
      acc *= old;
#pragma unroll
      for (int u = 0; u < kLoads; ++u) acc += __shfl(weight, u * kAtOnce + sub) * y[u];
    }
  };
  const Parts of_prefix = parts_of<D, RP, true>(p.prefix, row, h), of_own = parts_of<D, RO, false>(p.own, row, h);
  add(of_prefix);
  add(of_own);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) l += __shfl_xor(l, d);
  if (with_lse)
#pragma unroll
    for (int d = 1; d < 64; d *= 2) exact += __shfl_xor(exact, d);
#pragma unroll
  for (int d = kLanes; d < 64; d *= 2)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], d);
  if (sub != 0) return;
  const float inv = l > 0.f ? 1.0f / l : 0.f;
  u32x2 y;
  y.x = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{acc.x * inv, acc.y * inv}), bf16x2));
  y.y = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{acc.z * inv, acc.w * inv}), bf16x2));
  *reinterpret_cast<u32x2*>(p.own.out + job * D + 4 * c) = y;
  if (with_lse && lane == 0) p.own.lse[(int64_t)h * p.own.n_rows + row] = log_sum(m, exact);
}

template <int D, int RP, int RO>
void launch_rows(Launcher& launch, const SharedParams& p) {
  const bool one_page = (1 << p.own.cache.page_log2) >= kCacheKeyTile, lse = p.own.lse != nullptr;
  auto kernel = one_page ? (lse ? shared_attention_kernel<D, RP, RO, true, true> : shared_attention_kernel<D, RP, RO, true, false>)
                         : (lse ? shared_attention_kernel<D, RP, RO, false, true> : shared_attention_kernel<D, RP, RO, false, false>);
  launch(kernel, dim3((unsigned)p.own.workgroups), dim3(64 * kCacheWaves), 0, p);
  const int64_t rows = (int64_t)p.own.n_rows * p.own.hq;
  launch(shared_join_kernel<D, RP, RO>, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, p);
}
template <int D>
apbv_status launch_dim(const SharedParams& p, const SharedPlan& plan, hipStream_t stream) {
  Launcher launch(stream);
  if (plan.prefix.rows == 16)
    launch_rows<D, 16, 16>(launch, p);
  else if (plan.prefix.rows == 32)
    launch_rows<D, 32, 16>(launch, p);
  else if (plan.own.rows == 16)
    launch_rows<D, kCacheBlockRows, 16>(launch, p);
  else
    launch_rows<D, kCacheBlockRows, kCacheBlockRows>(launch, p);
  return launch.status();
}

}  // namespace

apbv_status launch_shared_attention(const SharedParams& p, const SharedPlan& plan, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? launch_dim<128>(p, plan, stream) : launch_dim<64>(p, plan, stream);
}

}  // namespace apbv
