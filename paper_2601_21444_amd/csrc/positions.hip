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
//
// Bound.  Rows that go to bf16, by HBM: 16384 tokens of 16 + 2 heads of 128 (151 MB) 25.9 us, 5.8 TB/s; 32768 of 28 + 4, normed (537 MB)
// 93 us, 5.8 TB/s; a copy of 1 GiB reaches 5.2.  Few tokens by the launch and a chain of position, angle, row: 2.5 us.  Rows that are bound for the
// cache by float64 arithmetic: keys and values of 16384 tokens of 2 heads of 128 12.2 us, where cache_store_kernel takes 5.6; with 16 heads of
// queries beside them 34.8 (157 MB, 4.5 TB/s).  Loads that pass the caches by 28.6 / 25.2 us and 94.3 / 96.6 (with / without, of the first two);
// five waves a SIMD 43.5 / 35.1 (the third); workgroups of keys among those of the queries 37.8 / 36.2.
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
// f(token, pair, its turn) for the pairs of `tokens` tokens from t0 on, dealt to 256 threads.
template <int D, typename F>
__device__ __forceinline__ void for_turns(const Rotation& r, int64_t t0, int tokens, F&& f) {
  constexpr int kPairs = D / 2;
  const int pair = threadIdx.x % kPairs;
  if (2 * pair >= r.rot) return;
  const int axis = (int)((pair < 32 ? r.axis[0] : r.axis[1]) >> (2 * (pair % 32))) & 3;
  const int32_t* positions = r.positions + axis * r.position_stride + t0;
  const float inv_freq = r.inv_freq[pair];
  for (int t = threadIdx.x / kPairs; t < tokens; t += 256 / kPairs) f(t, pair, turn_of(positions[t], inv_freq));
}
// 1 / sqrt(x): the instruction's 24 bits, doubled by a Newton step for each that is asked for; of infinity, which a step would make
// infinity times zero, zero.
template <int kSteps>
__device__ __forceinline__ double inv_sqrt(double x) {
  double y = __builtin_amdgcn_rsq(x);
#pragma unroll
  for (int i = 0; i < kSteps; ++i) y = __builtin_fma(y * 0.5, __builtin_fma(-x * y, y, 1.0), y);
  return x == __builtin_inf() ? 0.0 : y;
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
constexpr size_t append_lds_bytes(const AppendParams& p) { return (size_t)p.tile_tokens * (p.turn.rot.rot / 2) * sizeof(Turn); }

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
  u32x4 x[kRows][2], wq[2], wk[2];
  const bool q_normed = p.rot.q_weight != nullptr, k_normed = p.rot.k_weight != nullptr;
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
    if (q_normed) wq[0] = *reinterpret_cast<const u32x4*>(p.rot.q_weight + e0), wq[1] = *reinterpret_cast<const u32x4*>(p.rot.q_weight + e1);
    if (k_normed) wk[0] = *reinterpret_cast<const u32x4*>(p.rot.k_weight + e0), wk[1] = *reinterpret_cast<const u32x4*>(p.rot.k_weight + e1);
  }

  // cosines and sines [token][2][half]
  for_turns<D>(p.rot, t0, (int)(p.tokens - t0 < p.tile_tokens ? p.tokens - t0 : p.tile_tokens), [&](int t, int pair, const Turn& y) {
    lds[t * 2 * half + pair] = (float)y.c;
    lds[(t * 2 + 1) * half + pair] = (float)y.s;
  });
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
    if (is_q ? q_normed : k_normed) {
      double sum = 0.0;
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = __builtin_fma((double)y[s][i], (double)y[s][i], sum);
      sum = group_sum<L>(sum);
      const double inv = inv_sqrt<1>(__builtin_fma(sum, 1.0 / D, p.rot.eps));
      const float scale = (float)inv;
      auto weight = [&](int s, int i) { return is_q ? wq[s][i] : wk[s][i]; };
      if (scale > 0x1p-60f && scale < 0x1p60f) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t w = weight(s, i);
            y[s][2 * i] *= scale * low(w);
            y[s][2 * i + 1] *= scale * high(w);
          }
      } else {                                             // rows near the ends of bf16's range, in float64: the scale, or
                                                           // its product with a weight, may be no normal float32
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t w = weight(s, i);
            y[s][2 * i] = (float)(y[s][2 * i] * (inv * low(w)));
            y[s][2 * i + 1] = (float)(y[s][2 * i + 1] * (inv * high(w)));
          }
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
        u32x4* dst = reinterpret_cast<u32x4*>(to + (s ? e1 : e0));
        // (of many rows past the caches' write-back, which leaves the rows that are read their room: 16384 tokens of 16 + 2 heads of 128
        // 35.1 -> 25.2 us a call, 32768 of 28 + 4 105.2 -> 96.6; reads past the caches, too: 28.6 and 94.3; with apbv_compress_kv, which
        // reads the keys, behind it 52.3 -> 44.2)
        if constexpr (kRows > 1)
          __builtin_nontemporal_store(o, dst);
        else
          *dst = o;
      }
    }
  }
}

template <int D, int kRows>
__global__ __launch_bounds__(256) void rotate_kernel(const TurnParams p) {
  turn_rows_of<D, kRows>(p, blockIdx.x, angles);
}

// ---- keys and values for the cache: eight elements a lane, as cache_store_kernel

// float64 elements of a block (its other lanes hold the rest) -> eight codes, and the block's scale byte.  The upper word of an element, with
// its last bit set where anything lies behind it, is on the same side of every border (all have zeros there) as the element.
__device__ __forceinline__ uint32_t encode64(const double (&x)[8], uint32_t& scale) {
  constexpr uint32_t kSign = 0x80000000u, kInf = 0x7ff00000u, kLargest = 0x47efe000u;      // the largest finite bf16
  uint32_t u[8], m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, x[i]);
    const uint32_t hi = (uint32_t)(bits >> 32) | ((uint32_t)bits != 0u ? 1u : 0u);
    uint32_t a = hi & ~kSign;
    a = a > kInf ? 0u : a;                                 // (not a number: zero)
    a = a < kLargest ? a : kLargest;
    m = m > a ? m : a;
    u[i] = (hi & kSign) | a;
  }
  m = quad_max(m);
  int e = (int)(m >> 20) - 1023 + 127 - 2 + ((m & 0xfffffu) > 0xc0000u ? 1 : 0);      // one more from 1.75 * 2^n on
  e = e < 2 ? 2 : (e > 252 ? 252 : e);
  scale = (uint32_t)e;
  const float s = __uint_as_float((uint32_t)e << 23);
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = (float)__builtin_bit_cast(double, (uint64_t)u[i] << 32);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[0], f[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[2], f[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[4], f[5], s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[6], f[7], s, 3);
  return c;
}

// 256 / (D / 8) rows: a few heads of consecutive tokens, which share the angles; the tokens of a head follow one another in a page, and
// their codes are written in whole lines.
template <int D>
__device__ __forceinline__ void append_rows(const AppendParams& p, uint32_t group, Turn* lds) {
  constexpr int kPieces = D / 8;
  const Rotation& r = p.turn.rot;
  const uint32_t tt = group / (uint32_t)p.head_tiles;
  const int64_t tokens = p.turn.tokens, t0 = (int64_t)tt * p.tile_tokens;
  const int row = threadIdx.x / kPieces, piece = threadIdx.x % kPieces, half = r.rot >> 1;
  const int h = row / p.tile_tokens, t = row - h * p.tile_tokens;
  const int h0 = (int)(group - tt * (uint32_t)p.head_tiles) * p.tile_heads;
  const bool live = h < p.tile_heads && h0 + h < p.hkv && t0 + t < tokens;
  const int head = live ? h0 + h : h0;
  const int64_t token = live ? t0 + t : t0;
  const int e0 = 8 * piece;
  const bool turned = e0 < r.rot, upper = !r.adjacent && e0 >= half;
  const int slot = p.slots[token];
  const bf16_t* from = p.k.ptr + token * p.k.st + (int64_t)head * p.k.sh;
  const u32x4 k = *reinterpret_cast<const u32x4*>(from + e0);
  const int with = !turned || r.adjacent ? e0 : (upper ? e0 - half : e0 + half);
  const u32x4 k_with = *reinterpret_cast<const u32x4*>(from + with);      // the elements that these turn with
  const u32x4 v = *reinterpret_cast<const u32x4*>(p.v.ptr + token * p.v.st + (int64_t)head * p.v.sh + e0);
  u32x4 w, w_with;
  if (r.k_weight != nullptr) w = *reinterpret_cast<const u32x4*>(r.k_weight + e0), w_with = *reinterpret_cast<const u32x4*>(r.k_weight + with);

  // [token][pair]
  for_turns<D>(r, t0, (int)(tokens - t0 < p.tile_tokens ? tokens - t0 : p.tile_tokens), [&](int at, int pair, const Turn& y) { lds[at * half + pair] = y; });
  __syncthreads();

  double x[8], y[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = low(k[i]), x[2 * i + 1] = high(k[i]);
    y[2 * i] = low(k_with[i]), y[2 * i + 1] = high(k_with[i]);
  }
  if (r.k_weight != nullptr) {
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = __builtin_fma(x[i], x[i], sum);
    sum = group_sum<kPieces>(sum);
    const double scale = inv_sqrt<2>(__builtin_fma(sum, 1.0 / D, r.eps));
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
  if (blockIdx.x < (uint32_t)p.row_groups)
    append_rows<D>(p, blockIdx.x, reinterpret_cast<Turn*>(angles));
  else
    turn_rows_of<D, kRows>(p.turn, blockIdx.x - (uint32_t)p.row_groups, angles);
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
  const int64_t rows = p.turn.tokens * p.turn.hq, query_groups = p.turn.hq > 0 ? deal_rows(p.turn, rows, d) : 0;
  const TurnPlan plan = append_plan(p.turn.tokens, p.hkv, d);
  p.tile_tokens = plan.tokens;
  p.tile_heads = plan.heads;
  p.head_tiles = (int)plan.head_tiles;
  p.row_groups = (int)plan.workgroups();
  auto kernel = turn_rows(rows, d) > 4096 / d ? (d == 128 ? cache_append_kernel<128, 4> : cache_append_kernel<64, 4>)
                                              : (d == 128 ? cache_append_kernel<128, 1> : cache_append_kernel<64, 1>);
  const size_t of_keys = append_lds_bytes(p), of_queries = query_groups > 0 ? turn_lds_bytes(p.turn) : 0;
  Launcher launch(stream);
  launch(kernel, dim3((unsigned)(p.row_groups + query_groups)), dim3(256), of_keys > of_queries ? of_keys : of_queries, p);
  return launch.status();
}

}  // namespace apbv
