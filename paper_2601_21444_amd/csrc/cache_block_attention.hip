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
// Chunks of prompts, two waves a SIMD, are bound by what a SIMD issues: matrix instructions are under way in 53 % of the cycles, vector
// instructions (exponentials, conversions of keys and of weights, maxima) in 43 % more, and little of the one runs beside the other
// (1030 TFLOP/s at 1.89 GHz; a kernel of 16x16x32 instructions, and one whose waves took K from memory each for itself, which convert
// as much or more, run at the same rate to a percent: 4 x 512 queries of 28 / 4 heads of 128 over 20000 keys 568, 568, 574 us).
// A turn of the loop is two tiles without a way out between them, holds the scales as bytes and keeps the maxima where they are written: else the
// compiler waits for codes that have just been asked for, and forms the maxima behind the last matrix instruction (4 x 1 to 512 queries over
// 9000 to 40000 keys 292.8 / 282.6 us, both in one run).  Every row tile of a head converts its keys again.  Short blocks are bound by their start
// (4 us), the end (3 us) and 3000 cycles a tile of a lone wave, of which 1024 are matrix instructions.  At head_dim 128 19 registers are spilled
// (25 with lse), where a piece begins and ends, none in the loop.
#include "cache_block_rows.h"

namespace apbv {
namespace {

template <int D, bool kLse>                                // kLse: as in cache_attention.hip
__global__ __launch_bounds__(64 * kCacheWaves, 2) void cache_block_attention_kernel(const CacheAttnParams p) {
  __shared__ BlockRowsLds<D> lds;
  attend_block_rows<D, kLse>(p, lds, blockIdx.x, AxisCut{}, Request{});
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
