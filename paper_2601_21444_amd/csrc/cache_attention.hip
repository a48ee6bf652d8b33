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
// joins it.  (All waves on one row tile at a time took 53.7 us instead of 47.8 for 64 requests of 512 to 32768 keys, 24.2 instead
// of 16.9 for 256 of 65 to 2048, 14.4 instead of 14.8 for one of 133120.)
//
// Bound by memory in batches and long requests (called again and again, whose keys are partly in the last-level cache): 64 requests,
// 28 / 4 heads of 128, 251 MB in 44.0 us (5.7 TB/s; the join 4.8 more); of one request every 8192 keys of 16 / 2 heads of 128 cost
// 0.33 us more (6.8 TB/s); 133120 keys, 36 MB in 12.3 us, of which the start (lengths, page, codes, one after the other) takes 3 and
// the end 2, the join 4.8.
//
// Weights are rounded to bf16 for the product with V, which keeps the bf16 matrix instruction at one product a key: half a step each,
// 2^-8 at most and 1.7e-3 in root mean square.  Outputs lie 2.3e-3 from those of 64 bits where the rounding of the output alone leaves
// 1.65e-3; two products of a weight's halves would take that away for as many matrix instructions again.
//
// Keys.  A lane of the matrix instruction's A operand needs eight elements of one key, and which elements go with which k-step
// is free as long as K and Q agree: lane (key li, quarter lg) takes the quarter's 16 bytes of codes, one load, all of one
// scale block, and converts eight of them a k-step.  No LDS.  V is needed transposed: a lane converts its quarter of a key's
// row, writes it to the wave's own LDS tile as bf16, and the transposing LDS read does the rest.
#include "cache_few_rows.h"

namespace apbv {
namespace {

template <int D, int NQ, bool kOnePage, bool kLse, bool kWhole>
__global__ __launch_bounds__(64 * kCacheWaves, 2) void cache_attention_kernel(const CacheAttnParams p) {
  __shared__ FewRowsLds<D, NQ, kWhole> lds;
  attend_few_rows<D, NQ, kOnePage, kLse, kWhole ? Form::kWhole : Form::kCut>(p, lds, blockIdx.x, AxisCut{}, Request{});
}

// kJoin waves per (row of q, head): joins the parts of rows that several workgroups share, and clears the rows without a key.
// A row has as many parts as workgroups share its keys: a few in a batch, a hundred and more in one long request, where the
// waves take them in turn.  Maxima and row sums of a row lie side by side over the workgroups.
template <int D, int R, int kJoin>
__global__ __launch_bounds__(kJoin == 1 ? 256 : 64 * kJoin) void cache_join_kernel(const CacheAttnParams p) {
  constexpr int kRowsPerGroup = kJoin == 1 ? 4 : 1;
  __shared__ float shared_max[kJoin], shared_sum[kJoin], shared_exact[kJoin];
  __shared__ f32x4 shared_acc[kJoin][D / 4];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t job = (int64_t)blockIdx.x * kRowsPerGroup + (kJoin == 1 ? wave : 0);
  if (job >= (int64_t)p.n_rows * p.hq) return;
  const int row = (int)(job / p.hq), h = (int)(job % p.hq);
  Axis<R> axis(p, typename Axis<R>::RowsOnly{});
  const int b = axis.find_row(p, row);
  const Request rq = axis.at(p, b);
  const int i = row - rq.first;
  if (i < 0 || i * p.group >= rq.rows) return;             // a row of no request
  constexpr int kLanes = D / 4;                            // lanes that hold a row, four elements each
  constexpr int kAtOnce = 64 / kLanes;
  const int sub = lane / kLanes, c = lane % kLanes;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f, exact = 0.f;               // exact: of the weights before they were rounded, for the log-sum-exp
  const bool with_lse = p.lse != nullptr;
  if (rq.tiles > 0) {
    const bool few = p.n_requests <= 64;
    const uint32_t share = few ? axis.share(p) : (uint32_t)scalar_load(reinterpret_cast<const int32_t*>(p.begins), 0);
    const uint32_t begin = few ? axis.begin_of(b) : (uint32_t)scalar_load(reinterpret_cast<const int32_t*>(p.begins), 1 + b);
    const int r = i * p.group + h % p.group, rt = r / R, row_tiles = (rq.rows + R - 1) / R;
    const uint32_t from = begin + (uint32_t)(h / p.group * row_tiles + rt) * (uint32_t)rq.tiles;
    const int first = (int)(from / share);
    int last = (int)((from + rq.tiles - 1) / share);
    last = last < p.workgroups ? last : p.workgroups - 1;
    if (first == last) return;                             // written by its only workgroup
    const float* stat = part_stats(p, 0, R, D) + (int64_t)(r % R) * p.workgroups;
    const float* rows = p.parts + (r % R) * D + 4 * c;
    // a wave's equal share of the parts, kAtOnce * kLoads at a time: lane n holds the n-th's maximum and row sum, and the rows
    // are on their way while the weights are found (32 at a time where four waves join: one request of 133120 keys has 30 for each)
    constexpr int kLoads = kJoin == 1 ? 8 : 32 / kAtOnce, kChunk = kAtOnce * kLoads;
    const int each = kJoin == 1 ? last - first + 1 : (last - first + kJoin) / kJoin;
    const int from_part = first + (kJoin == 1 ? 0 : wave * each);
    const int past_part = from_part + each <= last ? from_part + each : last + 1;
    for (int base = from_part; base < past_part; base += kChunk) {
      const int w = base + lane;
      const bool mine = lane < kChunk && w < past_part;
      const float* s = stat + (w == first ? (int64_t)(3 * R) * p.workgroups : 0) + w;
      const float m_part = mine ? s[0] : -INFINITY, l_part = mine ? s[(int64_t)R * p.workgroups] : 0.f;
      const float exact_part = mine && with_lse ? s[(int64_t)(2 * R) * p.workgroups] : 0.f;
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
  }
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
  *reinterpret_cast<u32x2*>(p.out + job * D + 4 * c) = y;
  if (with_lse && lane == 0) p.lse[(int64_t)h * p.n_rows + row] = log_sum(m, exact);
}

template <int D, int R>
void launch_join(Launcher& launch, const CacheAttnParams& p, int waves) {
  const int64_t rows = (int64_t)p.n_rows * p.hq;
  if (waves == 4)
    launch(cache_join_kernel<D, R, 4>, dim3((unsigned)rows), dim3(256), 0, p);
  else
    launch(cache_join_kernel<D, R, 1>, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, p);
}
template <int D, int NQ, bool kWhole>
auto few_rows_kernel(const CacheAttnParams& p) {
  if ((1 << p.cache.page_log2) >= kCacheKeyTile) return p.lse ? cache_attention_kernel<D, NQ, true, true, kWhole> : cache_attention_kernel<D, NQ, true, false, kWhole>;
  return p.lse ? cache_attention_kernel<D, NQ, false, true, kWhole> : cache_attention_kernel<D, NQ, false, false, kWhole>;
}
template <int D, int NQ>
void launch_few_rows(Launcher& launch, const CacheAttnParams& p, const CachePlan& plan) {
  if (plan.whole) {
    launch(few_rows_kernel<D, NQ, true>(p), dim3((unsigned)(p.n_requests * p.hkv * p.row_tiles)), dim3(64 * kCacheWaves), 0, p);
    return;
  }
  launch(few_rows_kernel<D, NQ, false>(p), dim3((unsigned)p.workgroups), dim3(64 * kCacheWaves), 0, p);
  launch_join<D, 16 * NQ>(launch, p, plan.join_waves);
}
template <int D>
apbv_status launch_dim(const CacheAttnParams& p, const CachePlan& plan, hipStream_t stream) {
  Launcher launch(stream);
  if (plan.rows == 16) {
    launch_few_rows<D, 1>(launch, p, plan);
  } else if (plan.rows == 32) {
    launch_few_rows<D, 2>(launch, p, plan);
  } else {
    const apbv_status st = launch_cache_block_attention(p, D, stream);
    if (st != APBV_OK) return st;
    launch_join<D, kCacheBlockRows>(launch, p, plan.join_waves);
  }
  return launch.status();
}

}  // namespace

apbv_status launch_cache_attention(const CacheAttnParams& p, const CachePlan& plan, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? launch_dim<128>(p, plan, stream) : launch_dim<64>(p, plan, stream);
}

}  // namespace apbv
