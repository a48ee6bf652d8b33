// Positions of queries and keys (include/apbv_positions.h): norm and rotation of rows, to bf16 or, of keys, to the codes of the cache.
//
// Angles.  A position times a frequency reaches far beyond a turn, where float32 holds nothing of the angle's fraction (position
// 200000 leaves 2^-7 of a radian), so the product is float64 and is reduced to an eighth of a turn with 2 / pi in two parts; sine and
// cosine are the Taylor polynomials there, whose first term left out is below 2^-53.  A workgroup forms them once for its tokens, in LDS, for all
// its heads.
//
// Queries (and keys that go to bf16).  A lane holds two times eight elements of a row that belong together: elements 8 c and rot / 2 + 8 c
// on, so that nothing is exchanged but the norm's sum.
//
// Keys for the cache.  A code is a whole number that a rounding decides, so everything in front of it is float64 (which issues as
// fast as float32 does here): codes are those of the exact value, whatever the order of the arithmetic.  The 21 leading bits and a
// bit for all that lie behind them are what a float32 is given, which rounds to the same code.
#include "cache_rows.h"
#include "positions.h"

namespace apbv {
namespace {

struct Turn {
  double c, s;
};
__device__ __forceinline__ Turn turn_of(int position, float inv_freq) {
  const double x = (double)position * (double)inv_freq;
  constexpr double kHi = 0x1.45f306dc9c883p-1, kLo = -0x1.6b01ec5417056p-55;       // 2 / pi
  const double t = x * kHi, n = __builtin_rint(t);
  const double r = ((t - n) + __builtin_fma(x, kLo, __builtin_fma(x, kHi, -t))) * 1.5707963267948966;
  const double z = r * r;
  double s = -1.0 / 1307674368000.0, c = 1.0 / 20922789888000.0;                   // 15!, 16!
  s = __builtin_fma(s, z, 1.0 / 6227020800.0);
  c = __builtin_fma(c, z, -1.0 / 87178291200.0);
  s = __builtin_fma(s, z, -1.0 / 39916800.0);
  c = __builtin_fma(c, z, 1.0 / 479001600.0);
  s = __builtin_fma(s, z, 1.0 / 362880.0);
  c = __builtin_fma(c, z, -1.0 / 3628800.0);
  s = __builtin_fma(s, z, -1.0 / 5040.0);
  c = __builtin_fma(c, z, 1.0 / 40320.0);
  s = __builtin_fma(s, z, 1.0 / 120.0);
  c = __builtin_fma(c, z, -1.0 / 720.0);
  s = __builtin_fma(s, z, -1.0 / 6.0);
  c = __builtin_fma(c, z, 1.0 / 24.0);
  s = __builtin_fma(s * z, r, r);
  c = __builtin_fma(c, z, -0.5);
  c = __builtin_fma(c, z, 1.0);
  // quarter turns (beyond 2^53 of them nothing of the angle is left, and any will do)
  const int quarter = (int)(n - 4.0 * __builtin_floor(n * 0.25));
  Turn y;
  y.c = quarter & 1 ? s : c;
  y.s = quarter & 1 ? c : s;
  y.c = quarter == 1 || quarter == 2 ? -y.c : y.c;
  y.s = quarter >= 2 ? -y.s : y.s;
  return y;
}
__device__ __forceinline__ Turn turn_at(const Rotation& r, int64_t token, int pair) {
  return turn_of(r.positions[r.axis[pair] * r.position_stride + token], r.inv_freq[pair]);
}

__device__ __forceinline__ float low(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float high(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }
__device__ __forceinline__ uint32_t to_pair(float x, float y) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), bf16x2));
}
template <int kCtrl>
__device__ __forceinline__ double dpp_add(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, kCtrl, 0xf, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), kCtrl, 0xf, 0xf, false);
  return x + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// Sums over groups of 4, 8 or 16 consecutive lanes.
template <int kLanes>
__device__ __forceinline__ double group_sum(double x) {
  x = dpp_add<0xB1>(x);                                    // quad_perm [1,0,3,2], [2,3,0,1]
  x = dpp_add<0x4E>(x);
  if constexpr (kLanes >= 8) x = dpp_add<0x141>(x);        // row_half_mirror
  if constexpr (kLanes >= 16) x = dpp_add<0x140>(x);       // row_mirror
  return x;
}

// The cosines and sines of a workgroup's tokens: float32 [token][2][pair] of rows that go to bf16, Turn [token][pair] of keys for the cache.
extern __shared__ __attribute__((aligned(16))) float angles[];
constexpr size_t turn_lds_bytes(const TurnParams& p) { return (size_t)p.tile_tokens * p.rot.rot * sizeof(float); }
constexpr size_t append_lds_bytes(int d, int rot) { return (size_t)(2048 / d) * (rot / 2) * sizeof(Turn); }

// The rows of token tile and head tile `group`, kRows a thread.
template <int D, int kRows>
__device__ __forceinline__ void turn_rows_of(const TurnParams& p, uint32_t group, float* lds) {
  constexpr int L = D / 16, kAtOnce = 256 / L;             // lanes of a row
  const int heads = p.hq + p.hkv, half = p.rot.rot >> 1;
  const uint32_t tt = group / (uint32_t)p.head_tiles;
  const int64_t t0 = (int64_t)tt * p.tile_tokens;
  const int h0 = (int)(group - tt * (uint32_t)p.head_tiles) * p.tile_heads;
  const int c = threadIdx.x % L;
  // this lane's two times eight elements: of pairs, or elements that stay
  const bool turned = c < p.rot.rot / 16;
  const int e0 = turned ? 8 * c : 16 * c, e1 = turned ? half + 8 * c : 16 * c + 8;      // (16 c = rot + 16 (c - rot / 16))

  int token[kRows], head[kRows];
  bool live[kRows];
  u32x4 x[kRows][2];
  {
    const int row = threadIdx.x / L;
    int t = row / p.tile_heads, h = row - t * p.tile_heads;
    const int step_t = kAtOnce / p.tile_heads, step_h = kAtOnce - step_t * p.tile_heads;
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      token[u] = t;
      head[u] = h0 + h;
      live[u] = t < p.tile_tokens && t0 + t < p.tokens && h0 + h < heads;
      const bool is_q = head[u] < p.hq;
      const View& v = is_q ? p.q : p.k;
      if (live[u]) {
        const bf16_t* from = v.ptr + (t0 + t) * v.st + (int64_t)(is_q ? head[u] : head[u] - p.hq) * v.sh;
        x[u][0] = *reinterpret_cast<const u32x4*>(from + e0);
        x[u][1] = *reinterpret_cast<const u32x4*>(from + e1);
      } else {
        x[u][0] = x[u][1] = u32x4{0u, 0u, 0u, 0u};
      }
      t += step_t;
      h += step_h;
      if (h >= p.tile_heads) h -= p.tile_heads, ++t;
    }
  }

  // cosines and sines [token][2][half]
  const int n = (int)(p.tokens - t0 < p.tile_tokens ? p.tokens - t0 : p.tile_tokens) * half;
  for (int i = threadIdx.x; i < n; i += 256) {
    const int t = i / half, pair = i - t * half;
    const Turn y = turn_at(p.rot, t0 + t, pair);
    lds[t * 2 * half + pair] = (float)y.c;
    lds[(t * 2 + 1) * half + pair] = (float)y.s;
  }
  __syncthreads();

#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    const bool is_q = head[u] < p.hq;
    float y[2][8];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        y[s][2 * i] = low(x[u][s][i]);
        y[s][2 * i + 1] = high(x[u][s][i]);
      }
    const bf16_t* weight = is_q ? p.rot.q_weight : p.rot.k_weight;
    if (weight != nullptr) {
      const u32x4 w0 = *reinterpret_cast<const u32x4*>(weight + e0), w1 = *reinterpret_cast<const u32x4*>(weight + e1);
      double sum = 0.0;
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = __builtin_fma((double)y[s][i], (double)y[s][i], sum);
      sum = group_sum<L>(sum);
      const float scale = (float)(1.0 / __builtin_sqrt(sum / D + p.rot.eps));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        y[0][2 * i] *= scale * low(w0[i]);
        y[0][2 * i + 1] *= scale * high(w0[i]);
        y[1][2 * i] *= scale * low(w1[i]);
        y[1][2 * i + 1] *= scale * high(w1[i]);
      }
    }
    if (turned) {
      const float* table = lds + (live[u] ? token[u] : 0) * 2 * half;
      if (p.rot.adjacent) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const f32x4 cs = *reinterpret_cast<const f32x4*>(table + (s ? e1 : e0) / 2), sn = *reinterpret_cast<const f32x4*>(table + half + (s ? e1 : e0) / 2);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float a = y[s][2 * i], b = y[s][2 * i + 1];
            y[s][2 * i] = a * cs[i] - b * sn[i];
            y[s][2 * i + 1] = b * cs[i] + a * sn[i];
          }
        }
      } else {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const f32x4 cs = *reinterpret_cast<const f32x4*>(table + e0 + 4 * s), sn = *reinterpret_cast<const f32x4*>(table + half + e0 + 4 * s);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float a = y[0][4 * s + i], b = y[1][4 * s + i];
            y[0][4 * s + i] = a * cs[i] - b * sn[i];
            y[1][4 * s + i] = b * cs[i] + a * sn[i];
          }
        }
      }
    }
    if (live[u]) {
      bf16_t* to = (is_q ? p.q_out + ((t0 + token[u]) * p.hq + head[u]) * D : p.k_out + ((t0 + token[u]) * p.hkv + head[u] - p.hq) * D);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        u32x4 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = to_pair(y[s][2 * i], y[s][2 * i + 1]);
        *reinterpret_cast<u32x4*>(to + (s ? e1 : e0)) = o;
      }
    }
  }
}

template <int D, int kRows>
__global__ __launch_bounds__(256) void rotate_kernel(const TurnParams p) {
  turn_rows_of<D, kRows>(p, blockIdx.x, angles);
}

// ---- keys and values for the cache: eight elements a lane, as cache_store_kernel

// float64 elements of a block (its other lanes hold the rest) -> eight codes, and the block's scale byte.
__device__ __forceinline__ uint32_t encode64(const double (&x)[8], uint32_t& scale) {
  constexpr uint64_t kAbs = ~(1ull << 63), kInf = 0x7ff0000000000000ull, kLargest = 0x47efe00000000000ull;      // the largest finite bf16
  uint64_t u[8], m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    u[i] = __builtin_bit_cast(uint64_t, x[i]);
    const uint64_t a = u[i] & kAbs;
    u[i] = a > kInf ? 0ull : (a > kLargest ? (u[i] & ~kAbs) | kLargest : u[i]);
    const uint64_t b = u[i] & kAbs;
    m = m > b ? m : b;
  }
  auto over_quad = [&](auto ctrl) {
    constexpr int kCtrl = decltype(ctrl)::value;
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)m, kCtrl, 0xf, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(m >> 32), kCtrl, 0xf, 0xf, false);
    const uint64_t y = (uint64_t)hi << 32 | lo;
    m = m > y ? m : y;
  };
  over_quad(std::integral_constant<int, 0xB1>{});
  over_quad(std::integral_constant<int, 0x4E>{});
  int e = (int)(m >> 52) - 1023 + 127 - 2 + ((m & 0xfffffffffffffull) > 0xc000000000000ull ? 1 : 0);      // one more from 1.75 * 2^n on
  e = e < 2 ? 2 : (e > 252 ? 252 : e);
  scale = (uint32_t)e;
  const float s = __uint_as_float((uint32_t)e << 23);
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t hi = (uint32_t)(u[i] >> 32) | ((uint32_t)u[i] != 0u ? 1u : 0u);
    f[i] = (float)__builtin_bit_cast(double, (uint64_t)hi << 32);
  }
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[0], f[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[2], f[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[4], f[5], s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[6], f[7], s, 3);
  return c;
}

// One head of 256 / (D / 8) consecutive tokens; the neighbour takes the next head of them.
template <int D>
__device__ __forceinline__ void append_rows(const AppendParams& p, uint32_t group, Turn* lds) {
  constexpr int kPieces = D / 8, kTokens = 256 / kPieces;
  const Rotation& r = p.turn.rot;
  const int64_t tokens = p.turn.tokens, t0 = (int64_t)(group / (uint32_t)p.hkv) * kTokens;
  const int head = (int)(group % (uint32_t)p.hkv), piece = threadIdx.x % kPieces, t = threadIdx.x / kPieces, half = r.rot >> 1;
  const bool live = t0 + t < tokens;
  const int64_t token = live ? t0 + t : tokens - 1;
  const int e0 = 8 * piece;
  const bool turned = e0 < r.rot, upper = !r.adjacent && e0 >= half;
  const int slot = p.slots[token];
  const bf16_t* row = p.k.ptr + token * p.k.st + (int64_t)head * p.k.sh;
  const u32x4 k = *reinterpret_cast<const u32x4*>(row + e0);
  const int with = !turned || r.adjacent ? e0 : (upper ? e0 - half : e0 + half);
  const u32x4 k_with = *reinterpret_cast<const u32x4*>(row + with);      // the elements that these turn with
  const u32x4 v = *reinterpret_cast<const u32x4*>(p.v.ptr + token * p.v.st + (int64_t)head * p.v.sh + e0);

  // [token][pair]
  const int n = (int)(tokens - t0 < kTokens ? tokens - t0 : kTokens) * half;
  for (int i = threadIdx.x; i < n; i += 256) {
    const int at = i / half;
    lds[i] = turn_at(r, t0 + at, i - at * half);
  }
  __syncthreads();

  double x[8], y[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = low(k[i]), x[2 * i + 1] = high(k[i]);
    y[2 * i] = low(k_with[i]), y[2 * i + 1] = high(k_with[i]);
  }
  if (r.k_weight != nullptr) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(r.k_weight + e0), w_with = *reinterpret_cast<const u32x4*>(r.k_weight + with);
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = __builtin_fma(x[i], x[i], sum);
    sum = group_sum<kPieces>(sum);
    const double scale = 1.0 / __builtin_sqrt(sum / D + r.eps);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] *= scale * low(w[i]), x[2 * i + 1] *= scale * high(w[i]);
      y[2 * i] *= scale * low(w_with[i]), y[2 * i + 1] *= scale * high(w_with[i]);
    }
  }
  if (turned) {
    const Turn* table = lds + (live ? t : 0) * half;
    if (r.adjacent) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const Turn a = table[e0 / 2 + i];
        const double one = x[2 * i], two = x[2 * i + 1];
        x[2 * i] = one * a.c - two * a.s;
        x[2 * i + 1] = two * a.c + one * a.s;
      }
    } else {
      const int pair = upper ? e0 - half : e0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const Turn a = table[pair + i];
        x[i] = x[i] * a.c + y[i] * (upper ? a.s : -a.s);
      }
    }
  }
  uint32_t ks, vs;
  const uint32_t kc = encode64(x, ks), vc = encode(v, vs);
  const RowPlace place(p.cache, slot, head);
  if (!live || !place.held) return;
  const int64_t codes = place.page * p.cache.stride_codes + (int64_t)place.row * (D / 2) + 4 * piece;
  *reinterpret_cast<uint32_t*>(p.cache.k_codes + codes) = kc;
  *reinterpret_cast<uint32_t*>(p.cache.v_codes + codes) = vc;
  if (piece % 4 == 0) {
    const int64_t scales = place.page * p.cache.stride_scales + (int64_t)place.row * (D / 32) + piece / 4;
    p.cache.k_scales[scales] = (uint8_t)ks;
    p.cache.v_scales[scales] = (uint8_t)vs;
  }
}

template <int D, int kRows>
__global__ __launch_bounds__(256) void cache_append_kernel(const AppendParams p) {
  if (blockIdx.x < (uint32_t)p.query_groups)
    turn_rows_of<D, kRows>(p.turn, blockIdx.x, angles);
  else
    append_rows<D>(p, blockIdx.x - (uint32_t)p.query_groups, reinterpret_cast<Turn*>(angles));
}

// Fills in how the rows are dealt; the number of workgroups.
int64_t deal_rows(TurnParams& p, int64_t rows, int d) {
  const TurnPlan plan = turn_plan(p.tokens, p.hq + p.hkv, turn_rows(rows, d));
  p.tile_tokens = plan.tokens;
  p.tile_heads = plan.heads;
  p.head_tiles = (int)plan.head_tiles;
  return plan.workgroups();
}

}  // namespace

apbv_status launch_rotate(TurnParams& p, int d, hipStream_t stream) {
  const int64_t rows = p.tokens * (p.hq + p.hkv), groups = deal_rows(p, rows, d);
  auto kernel = turn_rows(rows, d) > 4096 / d ? (d == 128 ? rotate_kernel<128, 4> : rotate_kernel<64, 4>)
                                              : (d == 128 ? rotate_kernel<128, 1> : rotate_kernel<64, 1>);
  Launcher launch(stream);
  launch(kernel, dim3((unsigned)groups), dim3(256), turn_lds_bytes(p), p);
  return launch.status();
}

apbv_status launch_cache_append(AppendParams& p, int d, hipStream_t stream) {
  const int64_t rows = p.turn.tokens * p.turn.hq;
  p.query_groups = p.turn.hq > 0 ? (int)deal_rows(p.turn, rows, d) : 0;
  auto kernel = turn_rows(rows, d) > 4096 / d ? (d == 128 ? cache_append_kernel<128, 4> : cache_append_kernel<64, 4>)
                                              : (d == 128 ? cache_append_kernel<128, 1> : cache_append_kernel<64, 1>);
  const size_t of_keys = append_lds_bytes(d, p.turn.rot.rot), of_queries = p.query_groups > 0 ? turn_lds_bytes(p.turn) : 0;
  Launcher launch(stream);
  launch(kernel, dim3((unsigned)(p.query_groups + cache_row_groups(p.turn.tokens, p.hkv, d))), dim3(256), of_keys > of_queries ? of_keys : of_queries, p);
  return launch.status();
}

}  // namespace apbv
