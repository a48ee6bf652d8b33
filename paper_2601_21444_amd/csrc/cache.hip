// The key/value cache held in 4 bits (include/apbv_cache.h): rows written and read back, and the block tables, slots and free
// pages of a step.
//
// Rows.  Four lanes share a block of 32 elements, eight each: 16 bytes of bf16 against 4 bytes of codes, for K and V at once.
// The block's maximum is taken on the absolute bit patterns (bf16 of one sign order as integers), so its exponent field gives
// the scale without arithmetic; the conversions are the hardware's own for this format (round to nearest even, saturating).
// Both directions move bytes and are bound by them.
//
// Tables.  The lengths are few thousand integers: one workgroup takes their prefix sums and does what depends on the order of
// the requests (pages given back, pages taken).  The slots of a step's few tokens are found by the same workgroup; those of
// prompts, of which there may be a hundred thousand, by a second launch over the tokens.
#include "cache.h"

namespace apbv {
namespace {

// ---- rows

// Absolute value of a bf16 pattern as it is held: NaN counts as zero, infinity as the largest finite value.
__device__ __forceinline__ uint32_t held(uint32_t x) {
  const uint32_t a = x & 0x7fffu;
  return a > 0x7f80u ? 0u : (a == 0x7f80u ? (x & 0x8000u) | 0x7f7fu : x);
}
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, false);      // quad_perm [1,0,3,2]
  x = x > y ? x : y;
  const uint32_t z = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, false);      // quad_perm [2,3,0,1]
  return x > z ? x : z;
}

// Eight elements of a block (its other lanes hold the rest) -> eight codes, and the block's scale byte.
__device__ __forceinline__ uint32_t encode(u32x4 x, uint32_t& scale) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = held(x[i] & 0xffffu), hi = held(x[i] >> 16);
    x[i] = lo | (hi << 16);
    const uint32_t a = lo & 0x7fffu, b = hi & 0x7fffu;
    m = m > a ? m : a;
    m = m > b ? m : b;
  }
  m = quad_max(m);
  int e = (int)(m >> 7) - 2 + ((m & 0x7fu) > 0x60u ? 1 : 0);       // one more from 1.75 * 2^n (fraction 0x60 of 0x80) on
  e = e < 2 ? 2 : (e > 252 ? 252 : e);
  scale = (uint32_t)e;
  const float s = __uint_as_float((uint32_t)e << 23);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)x[0]), s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)x[1]), s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)x[2]), s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)x[3]), s, 3);
  return c;
}
__device__ __forceinline__ u32x4 decode(uint32_t c, uint32_t scale) {
  const float s = __uint_as_float(scale << 23);
  u32x4 x;
  x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0));
  x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1));
  x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2));
  x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3));
  return x;
}

// Thread -> (token, head, eight elements); the tokens' slots are checked against the pool.
template <int D>
struct RowPiece {
  static constexpr int kPieces = D / 8;
  int64_t token;
  int head, piece, slot;
  bool live, held;
  __device__ __forceinline__ RowPiece(const CacheRowsParams& p) {
    const int64_t row = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) / kPieces;
    piece = threadIdx.x % kPieces;
    live = row < p.tokens * p.hkv;
    token = live ? row / p.hkv : p.tokens - 1;
    head = live ? (int)(row % p.hkv) : 0;
    slot = p.slots[token];
    held = slot >= 0 && (slot >> p.cache.page_log2) < p.cache.n_pages;
  }
  // offset of the row in the codes and in the scales, in rows of the page, and the page
  __device__ __forceinline__ int64_t page(const CacheRowsParams& p) const { return slot >> p.cache.page_log2; }
  __device__ __forceinline__ int64_t in_page(const CacheRowsParams& p) const {
    return ((int64_t)head << p.cache.page_log2) + (slot & ((1 << p.cache.page_log2) - 1));
  }
};

template <int D>
__global__ __launch_bounds__(256) void cache_store_kernel(const CacheRowsParams p) {
  const RowPiece<D> r(p);
  if (!r.live || !r.held) return;                          // (the lanes of a block go together)
  const int64_t at = r.token, h = r.head;
  const u32x4 k = *reinterpret_cast<const u32x4*>(p.k.ptr + at * p.k.st + h * p.k.sh + 8 * r.piece);
  const u32x4 v = *reinterpret_cast<const u32x4*>(p.v.ptr + at * p.v.st + h * p.v.sh + 8 * r.piece);
  uint32_t ks, vs;
  const uint32_t kc = encode(k, ks), vc = encode(v, vs);
  const int64_t codes = r.page(p) * p.cache.stride_codes + r.in_page(p) * (D / 2) + 4 * r.piece;
  *reinterpret_cast<uint32_t*>(p.cache.k_codes + codes) = kc;
  *reinterpret_cast<uint32_t*>(p.cache.v_codes + codes) = vc;
  if (r.piece % 4 == 0) {
    const int64_t scales = r.page(p) * p.cache.stride_scales + r.in_page(p) * (D / 32) + r.piece / 4;
    p.cache.k_scales[scales] = (uint8_t)ks;
    p.cache.v_scales[scales] = (uint8_t)vs;
  }
}

template <int D>
__global__ __launch_bounds__(256) void cache_load_kernel(const CacheRowsParams p) {
  const RowPiece<D> r(p);
  if (!r.live) return;
  u32x4 k = {0u, 0u, 0u, 0u}, v = {0u, 0u, 0u, 0u};
  if (r.held) {
    const int64_t codes = r.page(p) * p.cache.stride_codes + r.in_page(p) * (D / 2) + 4 * r.piece;
    const int64_t scales = r.page(p) * p.cache.stride_scales + r.in_page(p) * (D / 32) + r.piece / 4;
    k = decode(*reinterpret_cast<const uint32_t*>(p.cache.k_codes + codes), p.cache.k_scales[scales]);
    v = decode(*reinterpret_cast<const uint32_t*>(p.cache.v_codes + codes), p.cache.v_scales[scales]);
  }
  const int64_t to = (r.token * p.hkv + r.head) * D + 8 * r.piece;
  *reinterpret_cast<u32x4*>(p.k_out + to) = k;
  *reinterpret_cast<u32x4*>(p.v_out + to) = v;
}

template <int D>
apbv_status launch_rows(const CacheRowsParams& p, bool store, hipStream_t stream) {
  const int64_t blocks = (p.tokens * p.hkv * (D / 8) + 255) / 256;
  if (blocks > 0x7fffffff) return APBV_ERR_UNSUPPORTED;
  Launcher launch(stream);
  launch(store ? cache_store_kernel<D> : cache_load_kernel<D>, dim3((unsigned)blocks), dim3(256), 0, p);
  return launch.status();
}

// ---- tables

constexpr int kMapThreads = 1024;
constexpr int kMapSlots = 8192;             // new tokens up to which the one workgroup finds the slots too
constexpr int kMapPerThread = (APBV_CACHE_MAX_REQUESTS + kMapThreads - 1) / kMapThreads;

__device__ __forceinline__ int clamp_int(int64_t x, int lo, int hi) { return (int)(x < lo ? lo : (x > hi ? hi : x)); }

// Inclusive sums over the workgroup of three numbers a thread.
struct Three {
  int64_t a, b, c;
};
__device__ __forceinline__ Three workgroup_scan(Three x, Three* wave_sum) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t a = __shfl_up(x.a, d), b = __shfl_up(x.b, d), c = __shfl_up(x.c, d);
    if (lane >= d) x.a += a, x.b += b, x.c += c;
  }
  if (lane == 63) wave_sum[wave] = x;
  __syncthreads();
  for (int w = 0; w < wave; ++w) x.a += wave_sum[w].a, x.b += wave_sum[w].b, x.c += wave_sum[w].c;
  return x;
}

// The last b with first[b] <= x among n + 1 ascending entries, first[0] = 0 <= x < first[n].
__device__ __forceinline__ int owner(const int* first, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// The slot of position pos, whose block lies on this page; -1 where no slot has that number.
__device__ __forceinline__ int slot_of(int page, int pos, int page_log2) {
  if (page < 0 || page > (0x7fffffff >> page_log2)) return -1;
  return (page << page_log2) + (pos & ((1 << page_log2) - 1));
}

// What a request asks for.
struct Change {
  int had, want;           // lengths; the same where the new length cannot be taken at all
  int64_t grown;           // new tokens
  __device__ __forceinline__ Change(const CacheMapParams& p, int b) {
    had = clamp_int(p.old_lengths[b], 0, p.cap);
    const int n = p.new_lengths[b];
    grown = (int64_t)n > had ? (int64_t)n - had : 0;
    want = n < 0 || n > p.cap ? had : n;
  }
  __device__ __forceinline__ int blocks(const CacheMapParams& p, int length) const { return (int)(((int64_t)length + (1 << p.page_log2) - 1) >> p.page_log2); }
};

__global__ __launch_bounds__(kMapThreads) void cache_map_kernel(const CacheMapParams p, const int with_slots) {
  // first new token, first page taken and first page given back of every request, cut off at 2^31 - 1
  __shared__ int first_token[APBV_CACHE_MAX_REQUESTS + 1], first_taken[APBV_CACHE_MAX_REQUESTS + 1], first_back[APBV_CACHE_MAX_REQUESTS + 1];
  __shared__ Three wave_sum[kMapThreads / 64];
  __shared__ int n_taken;
  const int n = p.n_requests, per = (n + kMapThreads - 1) / kMapThreads;
  if (threadIdx.x == 0) n_taken = 0;

  Three mine = {0, 0, 0};
  for (int u = 0; u < per; ++u) {
    const int b = threadIdx.x * per + u;
    if (b >= n) break;
    const Change c(p, b);
    const int up = c.blocks(p, c.want) - c.blocks(p, c.had);
    mine.a += c.grown;
    mine.b += up > 0 ? up : 0;
    mine.c += up < 0 ? -up : 0;
  }
  Three at = workgroup_scan(mine, wave_sum);
  at.a -= mine.a, at.b -= mine.b, at.c -= mine.c;
  constexpr int kTop = 0x7fffffff;
  for (int u = 0; u <= per; ++u) {
    const int b = threadIdx.x * per + u;
    if (b > n || (u == per && b != n)) break;              // (the last thread's entry behind its own: the totals)
    first_token[b] = clamp_int(at.a, 0, kTop);
    first_taken[b] = clamp_int(at.b, 0, kTop);
    first_back[b] = clamp_int(at.c, 0, kTop);
    if (b == n) break;
    const Change c(p, b);
    const int up = c.blocks(p, c.want) - c.blocks(p, c.had);
    at.a += c.grown;
    at.b += up > 0 ? up : 0;
    at.c += up < 0 ? -up : 0;
  }
  __syncthreads();
  const int held = clamp_int(*p.free_count, 0, p.free_capacity);
  const int n_back = first_back[n];

  // pages given back, behind the free ones
  for (int i = threadIdx.x; i < n_back && i < p.free_capacity - held; i += kMapThreads) {
    const int b = owner(first_back, n, i);
    const Change c(p, b);
    p.free_pages[held + i] = p.table[(int64_t)b * p.table_stride + c.blocks(p, c.want) + (i - first_back[b])];
  }
  const int free = clamp_int((int64_t)held + n_back, 0, p.free_capacity);
  // Refused for want of pages or room: what is asked for up to a request only grows, so that the pages taken are a prefix
  // of those asked for.
  auto granted = [&](int b, const Change& c) {
    if (p.new_lengths[b] != c.want) return false;
    if (c.grown == 0) return true;
    return first_token[b + 1] <= p.max_new && (first_taken[b + 1] == first_taken[b] || first_taken[b + 1] <= free);
  };
  for (int b = threadIdx.x; b < n; b += kMapThreads) {
    const Change c(p, b);
    if (granted(b, c) && c.grown > 0) atomicMax(&n_taken, first_taken[b + 1] <= free ? first_taken[b + 1] : 0);
  }
  __syncthreads();                                         // ... and the free pages written above can be read
  const int taken = n_taken;
  for (int i = threadIdx.x; i < taken; i += kMapThreads) {
    const int b = owner(first_taken, n, i);
    const Change c(p, b);
    p.table[(int64_t)b * p.table_stride + c.blocks(p, c.had) + (i - first_taken[b])] = p.free_pages[free - 1 - i];
  }
  for (int b = threadIdx.x; b <= n; b += kMapThreads) p.starts_out[b] = first_token[b] < p.max_new ? first_token[b] : p.max_new;
  __syncthreads();                                         // the table is complete
  if (with_slots) {
    const int total = first_token[n];
    for (int t = threadIdx.x; t < p.max_new; t += kMapThreads) {
      int slot = -1;
      if (t < total) {
        const int b = owner(first_token, n, t);
        const Change c(p, b);
        if (granted(b, c)) {
          const int pos = c.had + (t - first_token[b]);
          slot = slot_of(p.table[(int64_t)b * p.table_stride + (pos >> p.page_log2)], pos, p.page_log2);
        }
      }
      p.slots_out[t] = slot;
    }
    __syncthreads();                                       // (lengths_out may be old_lengths)
  }
  if (threadIdx.x == 0) *p.free_count_out = free - taken;
  // (a request's lengths are read by the thread that writes its result, and by no other any more)
  for (int b = threadIdx.x; b < n; b += kMapThreads) {
    const Change c(p, b);
    p.lengths_out[b] = granted(b, c) ? c.want : c.had;
  }
}

// The slots of many new tokens, from what the first launch wrote: a request that was refused kept another length than it
// asked for.
constexpr int kSlotsPerThread = 4;
__global__ __launch_bounds__(256) void cache_slots_kernel(const CacheMapParams p) {
  __shared__ int first[APBV_CACHE_MAX_REQUESTS + 1];
  const int n = p.n_requests;
  for (int b = threadIdx.x; b <= n; b += 256) first[b] = p.starts_out[b];
  __syncthreads();
  const int total = first[n];
#pragma unroll
  for (int u = 0; u < kSlotsPerThread; ++u) {
    const int t = (blockIdx.x * kSlotsPerThread + u) * 256 + threadIdx.x;
    if (t >= p.max_new) break;
    int slot = -1;
    if (t < total) {
      const int b = owner(first, n, t);
      const int now = p.lengths_out[b];
      if (now == p.new_lengths[b]) {
        const int pos = now - (first[b + 1] - t);
        slot = slot_of(p.table[(int64_t)b * p.table_stride + (pos >> p.page_log2)], pos, p.page_log2);
      }
    }
    p.slots_out[t] = slot;
  }
}

}  // namespace

apbv_status launch_cache_store(const CacheRowsParams& p, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? launch_rows<128>(p, true, stream) : launch_rows<64>(p, true, stream);
}
apbv_status launch_cache_load(const CacheRowsParams& p, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? launch_rows<128>(p, false, stream) : launch_rows<64>(p, false, stream);
}

apbv_status launch_cache_map(const CacheMapParams& p, hipStream_t stream) {
  Launcher launch(stream);
  const int with_slots = p.max_new <= kMapSlots;
  launch(cache_map_kernel, dim3(1), dim3(kMapThreads), 0, p, with_slots);
  if (!with_slots) {
    const unsigned per = 256 * kSlotsPerThread;
    launch(cache_slots_kernel, dim3(((unsigned)p.max_new + per - 1) / per), dim3(256), 0, p);
  }
  return launch.status();
}

}  // namespace apbv
