// The key/value cache held in 4 bits (include/apbv_cache.h): rows written and read back, and the block tables, slots and free
// pages of a step.
//
// Rows.  Four lanes share a block of 32 elements, eight each: 16 bytes of bf16 against 4 bytes of codes, for K and V at once.
// The block's maximum is taken on the absolute bit patterns (bf16 of one sign order as integers), so its exponent field gives
// the scale without arithmetic; the conversions are the hardware's own for this format (round to nearest even, saturating).
// Both directions move bytes and are bound by them: 16384 tokens of 4 heads of 128 are written in 9.7 us (4.4 TB/s) and read
// back in 7.4 (5.8 TB/s); of 64 tokens a launch's 2.5 us are all.
//
// Tables.  The lengths are few thousand integers: a workgroup takes their prefix sums, finds which requests are granted, and then
// deals tokens and pages to its threads.  A hundred thousand tokens of prompts are dealt to as many workgroups as they fill, each
// of which takes the sums for itself; in place, where one would write what another has yet to read, one workgroup does all but
// the slots, which a second launch finds.  Bound by the chain of launch, lengths, prefix sums and pages: 64 requests of one token
// 3.9 us, of which a launch that only reads and writes takes 2.5; 48 prompts of 80000 tokens 6.6, in place 12.0 (pages taken, slots and
// pages given back each wait for memory by themselves).
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

// A workgroup takes one head of 256 / (D / 8) consecutive tokens, its neighbour the next head of them: rows are read in whole
// tokens, and the codes of a head's tokens, which follow one another in a page, are written in whole lines.
template <int D>
struct RowPiece {
  static constexpr int kPieces = D / 8, kTokens = 256 / kPieces;
  int head, piece;
  int64_t token;
  bool live;
  __device__ __forceinline__ RowPiece(const CacheRowsParams& p) {
    head = (int)(blockIdx.x % (uint32_t)p.hkv);
    piece = threadIdx.x % kPieces;
    token = (int64_t)(blockIdx.x / (uint32_t)p.hkv) * kTokens + threadIdx.x / kPieces;
    live = token < p.tokens;
    if (!live) token = p.tokens - 1;
  }
};
// A row's place: offsets of its codes and scales, or not in the pool.
struct RowPlace {
  int64_t page;
  int row;
  bool held;
  __device__ __forceinline__ RowPlace(const CacheView& c, int slot, int head) {
    page = slot >> c.page_log2;
    held = slot >= 0 && page < c.n_pages;
    row = (head << c.page_log2) + (slot & ((1 << c.page_log2) - 1));
  }
};

template <int D>
__global__ __launch_bounds__(256) void cache_store_kernel(const CacheRowsParams p) {
  const RowPiece<D> r(p);
  const int slot = p.slots[r.token];                       // (the rows do not wait for their slots)
  const int64_t at = r.token, h = r.head;
  const u32x4 k = *reinterpret_cast<const u32x4*>(p.k.ptr + at * p.k.st + h * p.k.sh + 8 * r.piece);
  const u32x4 v = *reinterpret_cast<const u32x4*>(p.v.ptr + at * p.v.st + h * p.v.sh + 8 * r.piece);
  uint32_t ks, vs;
  const uint32_t kc = encode(k, ks), vc = encode(v, vs);
  const RowPlace place(p.cache, slot, r.head);
  if (!r.live || !place.held) return;
  const int64_t codes = place.page * p.cache.stride_codes + (int64_t)place.row * (D / 2) + 4 * r.piece;
  *reinterpret_cast<uint32_t*>(p.cache.k_codes + codes) = kc;
  *reinterpret_cast<uint32_t*>(p.cache.v_codes + codes) = vc;
  if (r.piece % 4 == 0) {
    const int64_t scales = place.page * p.cache.stride_scales + (int64_t)place.row * (D / 32) + r.piece / 4;
    p.cache.k_scales[scales] = (uint8_t)ks;
    p.cache.v_scales[scales] = (uint8_t)vs;
  }
}

template <int D>
__global__ __launch_bounds__(256) void cache_load_kernel(const CacheRowsParams p) {
  const RowPiece<D> r(p);
  if (!r.live) return;
  const RowPlace place(p.cache, p.slots[r.token], r.head);
  u32x4 k = {0u, 0u, 0u, 0u}, v = {0u, 0u, 0u, 0u};
  if (place.held) {
    const int64_t codes = place.page * p.cache.stride_codes + (int64_t)place.row * (D / 2) + 4 * r.piece;
    const int64_t scales = place.page * p.cache.stride_scales + (int64_t)place.row * (D / 32) + r.piece / 4;
    k = decode(*reinterpret_cast<const uint32_t*>(p.cache.k_codes + codes), p.cache.k_scales[scales]);
    v = decode(*reinterpret_cast<const uint32_t*>(p.cache.v_codes + codes), p.cache.v_scales[scales]);
  }
  // (past the caches' write-back: 131072 tokens of 4 heads of 128, 268 MB out of 71, 65 -> 50 us, 6.8 TB/s)
  const int64_t to = (r.token * p.hkv + r.head) * D + 8 * r.piece;
  __builtin_nontemporal_store(k, reinterpret_cast<u32x4*>(p.k_out + to));
  __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p.v_out + to));
}

template <int D>
apbv_status launch_rows(const CacheRowsParams& p, bool store, hipStream_t stream) {
  static_assert(RowPiece<D>::kTokens == 2048 / D, "cache_row_groups");
  const int64_t blocks = cache_row_groups(p.tokens, p.hkv, D);
  Launcher launch(stream);
  launch(store ? cache_store_kernel<D> : cache_load_kernel<D>, dim3((unsigned)blocks), dim3(256), 0, p);
  return launch.status();
}

// ---- tables

constexpr int kMapThreads = 1024;
constexpr int kMapSlots = 8192;             // new tokens up to which one workgroup finds the slots too, in place
constexpr int kTop = 0x7fffffff;

__device__ __forceinline__ int clamp_int(int64_t x, int lo, int hi) { return (int)(x < lo ? lo : (x > hi ? hi : x)); }

// Sums that stop at kTop, over the lanes of a wave (inclusive) on the DPP path.
__device__ __forceinline__ int add_stop(int x, int y) { return (int)__builtin_elementwise_min(__builtin_elementwise_add_sat((uint32_t)x, (uint32_t)y), (uint32_t)kTop); }
template <int kCtrl, int kRows>
__device__ __forceinline__ int dpp_add(int x) { return add_stop(x, __builtin_amdgcn_update_dpp(0, x, kCtrl, kRows, 0xf, false)); }
__device__ __forceinline__ int wave_scan(int x) {
  x = dpp_add<0x111, 0xf>(x);      // row_shr 1, 2, 4, 8; row_bcast 15, 31
  x = dpp_add<0x112, 0xf>(x);
  x = dpp_add<0x114, 0xf>(x);
  x = dpp_add<0x118, 0xf>(x);
  x = dpp_add<0x142, 0xa>(x);
  return dpp_add<0x143, 0xc>(x);
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
  if (page < 0 || page > (kTop >> page_log2)) return -1;
  return (page << page_log2) + (pos & ((1 << page_log2) - 1));
}

// One workgroup, or several where nothing that they write is read by another: where the outputs are not the inputs.  All find
// the same sums; the first writes what there is one of a request, tokens and pages are dealt to the threads of all.
// A thread holds kPer consecutive requests in registers and knows, after the prefix sums, where their tokens and
// pages lie.  In a decoding step, where no request grows by more than kFew tokens, that is all it takes: every thread serves
// its own requests.  Otherwise, and for pages given back, tokens and pages are dealt to the threads, which find the request of
// each in LDS, in a loop for the pages taken, one for the slots and one for the pages given back.  Pages are taken from where the list
// has them or will have them, so that nothing written here is read here: in a decoding step two waits for memory, for the lengths and
// for the pages (and one more if pages are given back), otherwise one for the lengths and one or more in each loop.
template <int kPer>
__global__ __launch_bounds__(kMapThreads) void cache_map_kernel(const CacheMapParams p, const int with_slots) {
  constexpr int kMost = kPer * kMapThreads, kWaves = kMapThreads / 64;
  constexpr int kFew = 4;                      // fewer than a page: at most one page is taken
  // first new token, first page taken and first page given back of every request (sums that stop at kTop), and its old length,
  // with the upper bit set where it is granted
  __shared__ int first_token[kMost + 1], first_taken[kMost + 1], first_back[kMost + 1];
  __shared__ uint32_t had_granted[kMost];
  __shared__ int wave_sum[kWaves][4];          // the three sums, and whether a request grows by many tokens
  __shared__ int n_taken;
  const int n = p.n_requests, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b0 = threadIdx.x * kPer;
  const int of_all = blockIdx.x * kMapThreads + threadIdx.x, all = gridDim.x * kMapThreads;
  auto blocks = [&](int length) { return (int)(((uint32_t)length + (1u << p.page_log2) - 1) >> p.page_log2); };
  auto table_at = [&](int b, int block) -> int32_t* { return p.table + (int64_t)b * p.table_stride + block; };

  const int held = clamp_int(*p.free_count, 0, p.free_capacity);
  int had[kPer], want[kPer], grown[kPer];      // want: as asked for; the old length where that cannot be taken at all
  bool possible[kPer];
  int sum[3] = {0, 0, 0};
  bool many = false;
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int b = b0 + u < n ? b0 + u : n - 1;
    had[u] = p.old_lengths[b];
    want[u] = p.new_lengths[b];
  }
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const bool real = b0 + u < n;
    had[u] = clamp_int(had[u], 0, p.cap);
    grown[u] = real && want[u] > had[u] ? want[u] - had[u] : 0;
    many = many || grown[u] > kFew;
    possible[u] = want[u] >= 0 && want[u] <= p.cap;
    if (!possible[u] || !real) want[u] = had[u];
    const int up = blocks(want[u]) - blocks(had[u]);
    sum[0] = add_stop(sum[0], grown[u]);
    sum[1] = add_stop(sum[1], up > 0 ? up : 0);
    sum[2] = add_stop(sum[2], up < 0 ? -up : 0);
  }
  int at[3];                                   // behind this thread's requests, then before each of them
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    at[k] = wave_scan(sum[k]);
    if (lane == 63) wave_sum[wave][k] = at[k];
  }
  const bool wave_many = __builtin_amdgcn_ballot_w64(many) != 0;
  if (lane == 63) wave_sum[wave][3] = wave_many;
  if (threadIdx.x == 0) n_taken = 0;
  __syncthreads();
  // (exclusive over the wave's lanes: the inclusive sum of the lane before, as sums that stop cannot be taken back)
  int total[4] = {0, 0, 0, 0}, before[3];
  const int waves = (n + 64 * kPer - 1) / (64 * kPer);     // those that hold requests
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    before[k] = __shfl_up(at[k], 1);
    before[k] = lane == 0 ? 0 : before[k];
  }
  for (int w = 0; w < waves; ++w) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int x = wave_sum[w][k];
      if (k < 3 && w < wave) before[k < 3 ? k : 0] = add_stop(before[k < 3 ? k : 0], x);
      total[k] = add_stop(total[k], x);
    }
  }
  const int n_back = total[2];
  const bool own = total[3] == 0;              // every thread serves its own requests
  const int free = clamp_int((int64_t)held + n_back, 0, p.free_capacity);

  // Refused for want of pages or room: what is asked for up to a request only grows, so that the pages taken are a prefix of
  // those asked for.
  int first[3][kPer];
  bool granted[kPer];
  int last_taken = 0;
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int b = b0 + u, up = blocks(want[u]) - blocks(had[u]);
#pragma unroll
    for (int k = 0; k < 3; ++k) first[k][u] = before[k];
    before[0] = add_stop(before[0], grown[u]);
    before[1] = add_stop(before[1], up > 0 ? up : 0);
    before[2] = add_stop(before[2], up < 0 ? -up : 0);
    granted[u] = possible[u] && (grown[u] == 0 || (before[0] <= p.max_new && (up == 0 || before[1] <= free)));
    if (granted[u] && up > 0) last_taken = before[1];
    if (b < n && blockIdx.x == 0) {
      p.lengths_out[b] = granted[u] ? want[u] : had[u];
      p.starts_out[b] = first[0][u] < p.max_new ? first[0][u] : p.max_new;
    }
  }
  if (of_all == 0) p.starts_out[n] = total[0] < p.max_new ? total[0] : p.max_new;
  if (last_taken > 0) atomicMax(&n_taken, last_taken);
  if (!own || n_back > 0) {
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int b = b0 + u;
      if (b > n) continue;
      first_token[b] = first[0][u];
      first_taken[b] = first[1][u];
      first_back[b] = first[2][u];
      if (b < n) had_granted[b] = (uint32_t)had[u] | (granted[u] ? 0x80000000u : 0u);
    }
    if (threadIdx.x == 0) first_token[n] = total[0], first_taken[n] = total[1], first_back[n] = total[2];
  }
  __syncthreads();
  if (of_all == 0) *p.free_count_out = free - n_taken;

  // a page given back, the i-th: one of the last blocks its request had; entry i of the list as it stands then
  auto back = [&](int i) -> const int32_t* {
    const int b = owner(first_back, n, i);
    return table_at(b, blocks((int)(had_granted[b] & kTop)) - (first_back[b + 1] - i));
  };
  auto entry = [&](int i) -> const int32_t* { return i < held ? p.free_pages + i : back(i - held); };

  if (own) {
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int b = b0 + u, old = blocks(had[u]), up = blocks(want[u]) - old;
      if (b >= n || grown[u] == 0 || blockIdx.x != 0) continue;
      int page_old = -1, page_new = -1;
      if (granted[u]) {
        if ((had[u] & ((1 << p.page_log2) - 1)) != 0) page_old = *table_at(b, old - 1);
        if (up > 0) page_new = *entry(free - 1 - first[1][u]);
        if (up > 0) *table_at(b, old) = page_new;
      }
      if (with_slots)
        for (int j = 0; j < grown[u]; ++j) {
          const int pos = had[u] + j;
          if (first[0][u] + j < p.max_new)
            p.slots_out[first[0][u] + j] = granted[u] ? slot_of(pos >> p.page_log2 < old ? page_old : page_new, pos, p.page_log2) : -1;
        }
    }
    if (with_slots)
      for (int64_t t = (int64_t)total[0] + of_all; t < p.max_new; t += all) p.slots_out[t] = -1;
  } else {
    const int taken = n_taken;
    for (int i = of_all; i < taken; i += all) {
      const int b = owner(first_taken, n, i);
      *table_at(b, blocks((int)(had_granted[b] & kTop)) + (i - first_taken[b])) = *entry(free - 1 - i);
    }
    if (with_slots)
      for (int t = of_all; t < p.max_new; t += all) {
        int slot = -1;
        if (t < total[0]) {
          const int b = owner(first_token, n, t);
          if (had_granted[b] >> 31) {
            const int old = (int)(had_granted[b] & kTop), pos = old + (t - first_token[b]), block = pos >> p.page_log2, fresh = block - blocks(old);
            slot = slot_of(fresh >= 0 ? *entry(free - 1 - first_taken[b] - fresh) : *table_at(b, block), pos, p.page_log2);
          }
        }
        p.slots_out[t] = slot;
      }
  }
  for (int i = of_all; i < n_back && i < p.free_capacity - held; i += all) p.free_pages[held + i] = *back(i);
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
  // (each step for all of a thread's tokens before the next: three waits for memory, not three a token)
  int t[kSlotsPerThread], owner_of[kSlotsPerThread], now[kSlotsPerThread], asked[kSlotsPerThread], slot[kSlotsPerThread];
#pragma unroll
  for (int u = 0; u < kSlotsPerThread; ++u) {
    t[u] = (blockIdx.x * kSlotsPerThread + u) * 256 + threadIdx.x;
    owner_of[u] = t[u] < total ? owner(first, n, t[u]) : 0;
    now[u] = p.lengths_out[owner_of[u]];
    asked[u] = p.new_lengths[owner_of[u]];
  }
#pragma unroll
  for (int u = 0; u < kSlotsPerThread; ++u) {
    const bool granted = t[u] < total && now[u] == asked[u];
    const int pos = granted ? now[u] - (first[owner_of[u] + 1] - t[u]) : 0;
    now[u] = pos;
    slot[u] = granted ? p.table[(int64_t)owner_of[u] * p.table_stride + (pos >> p.page_log2)] : -1;
  }
#pragma unroll
  for (int u = 0; u < kSlotsPerThread; ++u)
    if (t[u] < p.max_new) p.slots_out[t[u]] = slot_of(slot[u], now[u], p.page_log2);
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
  // in place, one workgroup and, for many tokens, a second launch; otherwise a workgroup for 1024 tokens, two a compute unit at most
  const bool in_place = p.lengths_out == p.old_lengths || p.free_count_out == p.free_count;
  const int with_slots = !in_place || p.max_new <= kMapSlots;
  const int groups = in_place ? 1 : p.max_new <= kMapThreads ? 1 : p.max_new < 512 * kMapThreads ? (p.max_new + kMapThreads - 1) / kMapThreads : 512;
  static_assert(4 * kMapThreads == APBV_CACHE_MAX_REQUESTS, "a thread's requests");
  launch(p.n_requests <= kMapThreads ? cache_map_kernel<1> : cache_map_kernel<4>, dim3(groups), dim3(kMapThreads), 0, p, with_slots);
  if (!with_slots) {
    const unsigned per = 256 * kSlotsPerThread;
    launch(cache_slots_kernel, dim3(((unsigned)p.max_new + per - 1) / per), dim3(256), 0, p);
  }
  return launch.status();
}

}  // namespace apbv
