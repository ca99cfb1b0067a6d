// The paged context cache: the handle, the pages and slots of every request
// from its lengths, and the write of new keys and values into the pages.
//
// The cache is caller-owned, k_cache and v_cache [n_pages][n_kv][P][head_dim]
// each: a page of one KV head is one contiguous run (4 KB at 16 keys of 128
// bf16), so that the attention reads whole runs, and a token's write touches one
// row of every head's run.
//
// Writes and reads are bound by memory: 16384 rows of 8 heads read back from 4 bits (85 MB)
// 17.4 to 18.7 us, 4.7 TB/s; 2048 rows of 8 heads written in 4 bits (10.6 MB) 4.4 us.
// A thread has 8 values (16 bytes) of the bf16 side, so that its accesses are whole lines a
// wave; with 4 bits the other side is 4 bytes a thread, and a quad of threads has a block.
#include <stdarg.h>
#include <stdio.h>

#include <algorithm>
#include <new>
#include <string>

#include "xp_kv.h"

namespace xp {

struct KvMap {
  int n, logP, cols, n_pages, max_slots;
  const int32_t* lens;
  const int32_t* add;
  int32_t* table;
  int64_t ld;
  int32_t* held;
  int32_t* pool;
  int32_t* pool_n;
  int32_t* cu;
  int32_t* kv_len;
  int32_t* slots;
  int32_t *take, *old, *acu, *len, *top;   // for k_kv_slots, which may run with kv_len in lens's place
  uint32_t* err;
};

// The pool's page number k from its top, given `top` free pages.
__device__ __forceinline__ int pool_page(const int32_t* pool, int top, int k) { return pool[top - 1 - k]; }

// Slot of token t: its request b (from lo, before hi), its position's page from the
// table or, where this call takes it, from the pool.
__device__ __forceinline__ int slot_of(const KvMap& d, int t, const int* acu, const int* take,
                                       const int32_t* old, const int32_t* len, int top,
                                       uint32_t& bad, int lo, int hi) {
  if (t >= acu[d.n]) return -1;
  const int b = kv_owner(acu, lo, hi, t);
  const int pos = len[b] + t - acu[b], col = pos >> d.logP, h = old[b];
  if (take[b + 1] > take[b] && take[b + 1] > top) return -1;     // not served
  const int page = col < h ? d.table[b * d.ld + col] : pool_page(d.pool, top, take[b] + col - h);
  if ((uint32_t)page >= (uint32_t)d.n_pages) {
    bad |= XP_DEVERR_PAGE;
    return -1;
  }
  return (page << d.logP) + (pos & ((1 << d.logP) - 1));
}

// the k-th page that the call takes, to its request's table
__device__ __forceinline__ void take_page(const KvMap& d, int k, const int* take,
                                          const int32_t* old, int top) {
  const int b = kv_owner(take, d.n, k);
  d.table[b * d.ld + old[b] + k - take[b]] = pool_page(d.pool, top, k);
}

// One workgroup: what every request releases, takes and adds, with the sums
// over the requests before it; the releases, the tables' new lengths and the
// pool's; with ALL also the pages taken and the slots.  Bound by latency: three
// block scans over the requests, then one search per page and slot (8 requests with
// blocks of 17: 5.2 us, 4.5 at best; 512 without slots 5.4).
constexpr int kMapThreads = 1024;
// Slots up to which one launch does all: 4096 of 64 requests 6.6 us in one, 7.5 in two;
// 8192 9.6 and 7.6, 32768 27.7 and 7.6.
constexpr int kMapOneLaunch = 5120;
template <bool ALL>
__global__ __launch_bounds__(kMapThreads) void k_kv_map(const KvMap d) {
  __shared__ int rel[kKvMaxBatch + 1], take[kKvMaxBatch + 1], acu[kKvMaxBatch + 1];
  __shared__ int old[kKvMaxBatch], len[kKvMaxBatch];   // len: -1 where it was left alone
  __shared__ int64_t red[3][kMapThreads / kWave];
  __shared__ int taken;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t bad = 0;
  int64_t sum[3] = {0, 0, 0};
  int free0 = d.pool_n[0];
  auto sat = [](int64_t x) { return (int)(x < 0x7fffffff ? x : 0x7fffffff); };
  if (tid == 0) taken = 0;
  for (int b0 = 0; b0 < d.n; b0 += kMapThreads) {
    const int b = b0 + tid;
    int v[3] = {0, 0, 0};                         // released, taken, added
    if (b < d.n) {
      const int x = d.lens[b], a = d.add[b], h = d.held[b];
      old[b] = h;
      len[b] = x;
      const int64_t total = (int64_t)x + a;
      if (x < 0 || a < 0 || h < 0 || h > d.cols || total > (int64_t)d.cols << d.logP) {
        bad |= XP_DEVERR_LENGTH;                  // left as it is
        old[b] = h < 0 ? 0 : (h > d.cols ? d.cols : h);
        len[b] = -1;
      } else {
        const int need = (int)((total + (1 << d.logP) - 1) >> d.logP);
        v[0] = need < h ? h - need : 0;
        v[1] = need > h ? need - h : 0;
        v[2] = a;
      }
    }
    // only the waves that have requests: with all sixteen at it their exchanges, one
    // LDS for all, were most of a small call's time
    const int left = d.n - b0, waves = left < kMapThreads ? (left + kWave - 1) / kWave : kMapThreads / kWave;
    int64_t in[3] = {0, 0, 0};
    if (wave < waves) {
#pragma unroll
      for (int q = 0; q < 3; ++q) {
        in[q] = v[q];
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
          const int64_t y = __shfl_up((long long)in[q], o, kWave);
          if (lane >= o) in[q] += y;
        }
        if (lane == kWave - 1) red[q][wave] = in[q];
      }
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      int64_t before = sum[q];
      for (int w = 0; w < waves; ++w) {
        const int64_t t = red[q][w];
        before += w < wave ? t : 0;
        sum[q] += t;
      }
      in[q] += before - v[q];
    }
    if (b < d.n) {
      rel[b] = (int)in[0];
      take[b] = (int)in[1];
      acu[b] = sat(in[2]);
    }
    __syncthreads();
  }
  if (tid == 0) {
    rel[d.n] = (int)sum[0];
    take[d.n] = (int)sum[1];
    acu[d.n] = sat(sum[2]);
  }
  __syncthreads();
  const int R = (int)sum[0];
  if (free0 < 0 || free0 > d.n_pages - R) {  // more pages than there are
    bad |= XP_DEVERR_POOL;
    free0 = free0 < 0 ? 0 : (free0 > d.n_pages ? d.n_pages : free0);
  }
  int top = free0 + R;
  // A wave returns kBack * 64 neighbouring pages at a time: one search finds the
  // requests of every 64th, and each page's lies between those of its 64 (a search
  // per page kept one workgroup's shared memory busy: 32000 pages 35 us, now 15).
  constexpr int kBack = 16;
  for (int i0 = wave * kBack * kWave; i0 < R; i0 += kBack * kMapThreads) {
    const int mark = i0 + lane * kWave;
    const int own = kv_owner(rel, d.n, mark < R ? mark : R - 1);   // lanes 0 .. kBack
    int32_t* at[kBack];
    int32_t page[kBack];
#pragma unroll
    for (int u = 0; u < kBack; ++u) {
      const int i = i0 + u * kWave + lane < R ? i0 + u * kWave + lane : R - 1;
      const int b = kv_owner(rel, __builtin_amdgcn_readlane(own, u),
                             __builtin_amdgcn_readlane(own, u + 1) + 1, i);
      at[u] = d.table + b * d.ld + old[b] - (rel[b + 1] - i);
      page[u] = *at[u];
    }
#pragma unroll
    for (int u = 0; u < kBack; ++u) {
      const int i = i0 + u * kWave + lane;
      if (i >= R) continue;
      if (top - 1 - i < d.n_pages) d.pool[top - 1 - i] = page[u];
      *at[u] = -1;
    }
  }
  top = top < d.n_pages ? top : d.n_pages;
  __syncthreads();                                // the pool holds them
  for (int b = tid; b < d.n; b += kMapThreads) {
    const int tk = take[b + 1] - take[b], rl = rel[b + 1] - rel[b];
    const bool ok = tk == 0 || take[b + 1] <= top;
    if (!ok) bad |= XP_DEVERR_POOL;
    else if (tk > 0) atomicMax(&taken, take[b + 1]);
    if (ok && tk + rl > 0) d.held[b] = old[b] + tk - rl;
    if (d.cu) d.cu[b] = acu[b];
    // a request that was left as it is has no keys to speak of
    const int x = len[b];
    if (d.kv_len) d.kv_len[b] = x < 0 ? 0 : (ok ? x + d.add[b] : x);
    if (!ALL) {
      d.take[b] = take[b];
      d.old[b] = old[b];
      d.acu[b] = acu[b];
      d.len[b] = len[b];
    }
  }
  __syncthreads();
  const int T = taken;
  if (tid == 0) {
    if (d.cu) d.cu[d.n] = acu[d.n];
    d.pool_n[0] = top - T;
    if (d.slots && acu[d.n] > d.max_slots) bad |= XP_DEVERR_SLOT;
    if (!ALL) {
      d.take[d.n] = take[d.n];
      d.acu[d.n] = acu[d.n];
      d.top[0] = top;
      d.top[1] = T;
    }
  }
  if constexpr (ALL) {
    for (int k = tid; k < T; k += kMapThreads) take_page(d, k, take, old, top);
    if (d.slots)
      for (int t = tid; t < d.max_slots; t += kMapThreads)
        d.slots[t] = slot_of(d, t, acu, take, old, len, top, bad, 0, d.n);
  }
  if (bad) atomicOr(d.err, bad);
}

// The pages taken and the slots of a large call, over many workgroups (a slot's
// page comes from the pool where this call takes it, so that no workgroup waits
// for another's table entries).  524000 slots: 6.8 us.
__global__ __launch_bounds__(256) void k_kv_slots(const KvMap d) {
  __shared__ int take[kKvMaxBatch + 1], acu[kKvMaxBatch + 1];
  for (int b = threadIdx.x; b <= d.n; b += 256) {
    take[b] = d.take[b];
    acu[b] = d.acu[b];
  }
  __syncthreads();
  const int top = d.top[0], T = d.top[1], step = gridDim.x * 256;
  uint32_t bad = 0;
  for (int k = blockIdx.x * 256 + threadIdx.x; k < T; k += step) take_page(d, k, take, d.old, top);
  // a wave takes 256 neighbouring slots: one search for the requests of every 64th
  constexpr int kU = 4;
  const int lane = threadIdx.x & 63, last = acu[d.n] - 1;
  for (int64_t i0 = ((int64_t)blockIdx.x * 256 + (threadIdx.x & ~63)) * kU; i0 < d.max_slots;
       i0 += (int64_t)step * kU) {
    const int64_t mark = i0 + lane * kWave;
    const int own = last < 0 ? 0 : kv_owner(acu, d.n, (int)(mark < last ? mark : last));
    int slot[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int64_t t = i0 + u * kWave + lane;
      slot[u] = t < d.max_slots
          ? slot_of(d, (int)t, acu, take, d.old, d.len, top, bad,
                    __builtin_amdgcn_readlane(own, u), __builtin_amdgcn_readlane(own, u + 1) + 1)
          : 0;
    }
#pragma unroll
    for (int u = 0; u < kU; ++u)
      if (i0 + u * kWave + lane < d.max_slots) d.slots[i0 + u * kWave + lane] = slot[u];
  }
  if (bad) atomicOr(d.err, bad);
}

// ---------------------------------------------------------------------------
// The write.  A thread moves VE values of one head of one token: 16 bytes of
// the cache.  Bound by memory: 2048 tokens of 8 x 128 (17 MB read and written) 4.4 us;
// 16397 to an 8-bit cache 23 us, 4.2 TB/s (the quotients' 20 instructions a value
// beside it).
// ---------------------------------------------------------------------------
// x / s (inv = 1 / s) to e4m3, the quotient rounded once: an fp32 quotient less
// than one step from the true one, to odd where it is not exact (an even one moves
// one step towards the truth), so that no middle between two e4m3 values lies
// between it and the truth; then to nearest even in the conversion.  Saturates at
// 448; NaN stays.
__device__ __forceinline__ float f8_quotient(float x, float s, float inv) {
  // beyond 448 by far: no rounding to decide, and no overflow below
  float q = x * inv;
  if (fabsf(q) < 1024.f) {
    q = fmaf(fmaf(-q, s, x), inv, q);             // one step of Newton's
    const float r = fmaf(-q, s, x);               // the exact rest
    const uint32_t u = __float_as_uint(q);
    const uint32_t up = (u ^ __float_as_uint(r) ^ __float_as_uint(s)) >> 31 ? u - 1u : u + 1u;
    q = ((r != 0.f) & (q != 0.f) & !(u & 1u)) ? __uint_as_float(up) : q;
  }
  return q > 448.f ? 448.f : (q < -448.f ? -448.f : q);
}

// a thread's item where a grid's x holds 2^22 workgroups (its threads are counted in 32 bits)
constexpr int kKvGridX = 1 << 22;
__device__ __forceinline__ int64_t kv_item() {
  return ((int64_t)blockIdx.z * kKvGridX + blockIdx.x) * 256 + threadIdx.x;
}
static dim3 kv_items_grid(int64_t items, unsigned y) {
  const int64_t wgs = (items + 255) / 256;
  return dim3((unsigned)std::min<int64_t>(wgs, kKvGridX), y, (unsigned)((wgs + kKvGridX - 1) / kKvGridX));
}

struct KvWrite {
  const uint16_t *k, *v;
  int64_t k_ld, v_ld;
  int64_t items;                     // tokens * n_kv * chunks
  int nkv, logP, n_pages;
  const int32_t* slots;              // NULL: by position
  const int32_t* table;
  int64_t table_ld;
  int cols;
  const int32_t* len;
  int B;
  char *kc, *vc;
  const float *ks, *vs;
  uint32_t* err;
};

// by value: a cast of a vector's element itself reads the first one
__device__ __forceinline__ xp_bf16x2 as_bf16x2(uint32_t x) { return __builtin_bit_cast(xp_bf16x2, x); }
// the greatest of a quad's four
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  const uint32_t y = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true));
  return max(y, (uint32_t)__builtin_amdgcn_mov_dpp((int)y, 0x4E, 0xF, 0xF, true));
}
// where row `slot` of KV head g begins; of a 4-bit cache its codes
template <int HD, int FMT>
__device__ __forceinline__ int64_t kv_row_at(int64_t slot, int g, int nkv, int logP) {
  const int64_t head = (slot >> logP) * nkv + g;
  const int r = (int)slot & ((1 << logP) - 1);
  if constexpr (FMT == XP_MXFP4) return (head << logP) * kv_row_bytes(FMT, HD) + r * (HD / 2);
  else return ((head << logP) + r) * kv_row_bytes(FMT, HD);
}
// from a 4-bit row's codes to its exponents
template <int HD>
__device__ __forceinline__ int64_t kv_exp_at(int64_t slot, int logP) {
  const int r = (int)slot & ((1 << logP) - 1);
  return ((int64_t)(HD / 2) << logP) - r * (HD / 2) + r * (HD / 32);
}

template <int HD, int FMT>
__global__ __launch_bounds__(256) void k_kv_write(const KvWrite d) {
  constexpr bool F8 = FMT == XP_E4M3, F4 = FMT == XP_MXFP4;
  constexpr int VE = F8 ? 16 : 8, CH = HD / VE;   // values, chunks of a row
  const int64_t i = kv_item();
  if (i >= d.items) return;
  const bool isv = blockIdx.y == 1;
  const int c = (int)(i % CH);
  const int64_t row = i / CH;
  const int64_t t = row / d.nkv;
  const int g = (int)(row - t * d.nkv);
  int slot;
  if (d.slots != nullptr) {
    slot = d.slots[t];
    if (slot == -1) return;                       // a token without a place
    if ((uint32_t)slot >= (uint32_t)d.n_pages << d.logP) {
      if (g == 0 && c == 0) atomicOr(d.err, XP_DEVERR_SLOT);
      return;
    }
  } else {
    const int b = (int)(t / d.B), x = d.len[b];
    const int64_t pos = (int64_t)x + (t - (int64_t)b * d.B);
    const bool in = x >= 0 && pos < (int64_t)d.cols << d.logP;
    const int page = in ? d.table[b * d.table_ld + (pos >> d.logP)] : -1;
    if ((uint32_t)page >= (uint32_t)d.n_pages) {
      if (g == 0 && c == 0) atomicOr(d.err, in ? XP_DEVERR_PAGE : XP_DEVERR_LENGTH);
      return;
    }
    slot = (page << d.logP) + (int)(pos & ((1 << d.logP) - 1));
  }
  const uint16_t* src = (isv ? d.v + t * d.v_ld : d.k + t * d.k_ld) + g * HD + c * VE;
  char* dst = (isv ? d.vc : d.kc) + kv_row_at<HD, FMT>(slot, g, d.nkv, d.logP) + (F4 ? 4 : 16) * c;
  const u32x4 a = ld16(src);
  if constexpr (F4) {
    // A quad of lanes has a block.  With its greatest magnitude m 2^k (1 <= m < 2) the
    // exponent is k - 2 where m <= 1.75 and k - 1 above: 31 units of the last place more
    // carry into the bf16 exponent exactly then.
    typedef unsigned short us2 __attribute__((ext_vector_type(2)));
    us2 m = __builtin_bit_cast(us2, a[0] & 0x7fff7fffu);
#pragma unroll
    for (int q = 1; q < 4; ++q)
      m = __builtin_elementwise_max(m, __builtin_bit_cast(us2, a[q] & 0x7fff7fffu));
    const uint32_t top = quad_max(m[0] > m[1] ? m[0] : m[1]);
    const bool num = top < 0x7f80u;
    const int e = min(max((int)((top + 31) >> 7) - 2, 2), 252);
    const float s = __uint_as_float((uint32_t)e << 23);
    uint32_t y = 0;
    y = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(y, as_bf16x2(a[0]), s, 0);
    y = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(y, as_bf16x2(a[1]), s, 1);
    y = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(y, as_bf16x2(a[2]), s, 2);
    y = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(y, as_bf16x2(a[3]), s, 3);
    *reinterpret_cast<uint32_t*>(dst) = num ? y : 0u;
    if ((c & 3) == 0)
      *reinterpret_cast<uint8_t*>(dst - 4 * c + kv_exp_at<HD>(slot, d.logP) + c / 4) =
          (uint8_t)(num ? e : 255);
  } else if constexpr (!F8) {
    *reinterpret_cast<u32x4*>(dst) = a;
  } else {
    const u32x4 b = ld16(src + 8);
    const float* sp = isv ? d.vs : d.ks;
    const float s = sp != nullptr ? sp[g] : 1.f, inv = __fdiv_rn(1.f, s);
    u32x4 y;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t w0 = q < 2 ? a[2 * q] : b[2 * q - 4], w1 = q < 2 ? a[2 * q + 1] : b[2 * q - 3];
      int z = __builtin_amdgcn_cvt_pk_fp8_f32(f8_quotient(__uint_as_float(w0 << 16), s, inv),
                                              f8_quotient(__uint_as_float(w0 & 0xffff0000u), s, inv), 0,
                                              false);
      z = __builtin_amdgcn_cvt_pk_fp8_f32(f8_quotient(__uint_as_float(w1 << 16), s, inv),
                                          f8_quotient(__uint_as_float(w1 & 0xffff0000u), s, inv), z, true);
      y[q] = (uint32_t)z;
    }
    *reinterpret_cast<u32x4*>(dst) = y;
  }
}

struct KvRead {
  const int32_t* slots;
  int64_t items;                     // tokens * n_kv * chunks of 8 values
  int nkv, logP, n_pages;
  const char *kc, *vc;
  const float *ks, *vs;
  uint16_t *k, *v;
  int64_t k_ld, v_ld;
  uint32_t* err;
};

// x s rounded once to bf16: the fp32 product moves off the middle between two bf16
// values where its own rounding put it there
__device__ __forceinline__ float product_for_bf16(float x, float s) {
  const float p = x * s, e = fmaf(x, s, -p);
  uint32_t u = __float_as_uint(p);
  if ((u & 0xffffu) == 0x8000u && e != 0.f) u += (e > 0.f) == (p > 0.f) ? 1u : -1u;
  return __uint_as_float(u);
}

// 8 values (16 bytes of the result) a thread
template <int HD, int FMT>
__global__ __launch_bounds__(256) void k_kv_read(const KvRead d) {
  constexpr int CH = HD / 8;
  const int64_t i = kv_item();
  if (i >= d.items) return;
  const bool isv = blockIdx.y == 1 || d.k == nullptr;
  const int c = (int)(i % CH);
  const int64_t row = i / CH;
  const int64_t t = row / d.nkv;
  const int g = (int)(row - t * d.nkv);
  const int slot = d.slots[t];
  const bool in = (uint32_t)slot < (uint32_t)d.n_pages << d.logP;
  if (!in && slot != -1 && g == 0 && c == 0) atomicOr(d.err, XP_DEVERR_SLOT);
  u32x4 y{0u, 0u, 0u, 0u};
  if (in) {
    const char* src = (isv ? d.vc : d.kc) + kv_row_at<HD, FMT>(slot, g, d.nkv, d.logP) +
                      c * (FMT == XP_BF16 ? 16 : (FMT == XP_E4M3 ? 8 : 4));
    if constexpr (FMT == XP_BF16) {
      y = ld16(src);
    } else if constexpr (FMT == XP_E4M3) {
      const uint2 x = *reinterpret_cast<const uint2*>(src);
      const float* sp = isv ? d.vs : d.ks;
      const float s = sp != nullptr ? sp[g] : 1.f;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const xp_f32x2 f = q % 2 == 0 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)(q < 2 ? x.x : x.y), false)
                                      : __builtin_amdgcn_cvt_pk_f32_fp8((int)(q < 2 ? x.x : x.y), true);
        y[q] = pk_bf16(product_for_bf16(f[0], s), product_for_bf16(f[1], s));
      }
    } else {
      const uint32_t x = *reinterpret_cast<const uint32_t*>(src);
      const uint8_t e =
          *reinterpret_cast<const uint8_t*>(src - 4 * c + kv_exp_at<HD>(slot, d.logP) + c / 4);
      const float s = __uint_as_float((e > 252 ? 255u : (uint32_t)e) << 23);
      y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, s, 0));
      y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, s, 1));
      y[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, s, 2));
      y[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, s, 3));
    }
  }
  *reinterpret_cast<u32x4*>((isv ? d.v + t * d.v_ld : d.k + t * d.k_ld) + g * HD + 8 * c) = y;
}

__global__ void k_kv_clear_err(uint32_t* err) {
  if (threadIdx.x == 0) *err = 0u;
}

bool kv_units_fit(const xp_kv* kv, int64_t tokens, int64_t n, int groups, int64_t table_ld,
                  int64_t max_q) {
  const int64_t keys = std::min<int64_t>(kv->max_pages, table_ld) * kv->P;
  const int64_t ent = (tokens * kv->grp / kv_least(kv, max_q * kv->grp) + n) * (groups > 0 ? 2 : 1);
  return ent * (keys / kKvTile + 8) * kv->nkv < ((int64_t)1 << 31);
}

hipError_t launch_kv_write(const xp_kv* kv, int tokens, const uint16_t* k, const uint16_t* v,
                           int64_t k_ld, int64_t v_ld, const int32_t* slots, const int32_t* table,
                           int64_t table_ld, const int32_t* len, int B, void* kc, void* vc,
                           const float* k_scale, const float* v_scale, hipStream_t st) {
  KvWrite d{};
  d.k = k;
  d.v = v;
  d.k_ld = k_ld;
  d.v_ld = v_ld;
  d.nkv = kv->nkv;
  d.items = (int64_t)tokens * kv->nkv * (kv->hd / (kv->dtype == XP_E4M3 ? 16 : 8));
  d.logP = kv->logP;
  d.n_pages = kv->n_pages;
  d.slots = slots;
  d.table = table;
  d.table_ld = table_ld;
  d.cols = (int)std::min<int64_t>(kv->max_pages, table_ld);
  d.len = len;
  d.B = B;
  d.kc = (char*)kc;
  d.vc = (char*)vc;
  d.ks = k_scale;
  d.vs = v_scale;
  d.err = kv->err;
  const dim3 grid = kv_items_grid(d.items, 2);
#define XP_KV(HD_, FMT_) hipLaunchKernelGGL((k_kv_write<HD_, FMT_>), grid, dim3(256), 0, st, d)
  if (kv->hd == 128) {
    if (kv->dtype == XP_BF16) XP_KV(128, XP_BF16);
    else if (kv->dtype == XP_E4M3) XP_KV(128, XP_E4M3);
    else XP_KV(128, XP_MXFP4);
  } else {
    if (kv->dtype == XP_BF16) XP_KV(64, XP_BF16);
    else if (kv->dtype == XP_E4M3) XP_KV(64, XP_E4M3);
    else XP_KV(64, XP_MXFP4);
  }
#undef XP_KV
  return hipGetLastError();
}

hipError_t launch_kv_read(const xp_kv* kv, int tokens, const int32_t* slots, const void* kc,
                          const void* vc, const float* k_scale, const float* v_scale, uint16_t* k,
                          uint16_t* v, int64_t k_ld, int64_t v_ld, hipStream_t st) {
  KvRead d{};
  d.slots = slots;
  d.items = (int64_t)tokens * kv->nkv * (kv->hd / 8);
  d.nkv = kv->nkv;
  d.logP = kv->logP;
  d.n_pages = kv->n_pages;
  d.kc = (const char*)kc;
  d.vc = (const char*)vc;
  d.ks = k_scale;
  d.vs = v_scale;
  d.k = k;
  d.v = v;
  d.k_ld = k_ld;
  d.v_ld = v_ld;
  d.err = kv->err;
  const dim3 grid = kv_items_grid(d.items, k != nullptr && v != nullptr ? 2 : 1);
#define XP_KV(HD_, FMT_) hipLaunchKernelGGL((k_kv_read<HD_, FMT_>), grid, dim3(256), 0, st, d)
  if (kv->hd == 128) {
    if (kv->dtype == XP_BF16) XP_KV(128, XP_BF16);
    else if (kv->dtype == XP_E4M3) XP_KV(128, XP_E4M3);
    else XP_KV(128, XP_MXFP4);
  } else {
    if (kv->dtype == XP_BF16) XP_KV(64, XP_BF16);
    else if (kv->dtype == XP_E4M3) XP_KV(64, XP_E4M3);
    else XP_KV(64, XP_MXFP4);
  }
#undef XP_KV
  return hipGetLastError();
}

}  // namespace xp

using namespace xp;

// Message of the last failed xp_kv_create of this thread.
static thread_local std::string g_kv_err;

static xp_status kv_fail(xp_kv* kv, xp_status s, const char* fmt, ...)
    __attribute__((format(printf, 3, 4)));
static xp_status kv_fail(xp_kv* kv, xp_status s, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  (kv ? kv->msg : g_kv_err) = buf;
  return s;
}

extern "C" const char* xp_kv_last_error(const xp_kv* kv) {
  return kv ? kv->msg.c_str() : g_kv_err.c_str();
}

extern "C" xp_status xp_kv_create(const xp_kv_shape* s, int32_t max_batch, int32_t max_tokens,
                                  int32_t max_len, int32_t shared, xp_kv** out) {
  g_kv_err.clear();
  if (out == nullptr) return kv_fail(nullptr, XP_EINVAL, "out is NULL");
  *out = nullptr;
  if (s == nullptr) return kv_fail(nullptr, XP_EINVAL, "shape is NULL");
  if (s->n_heads < 1 || s->n_kv < 1 || s->head_dim < 1 || s->page_size < 1 || s->n_pages < 1)
    return kv_fail(nullptr, XP_EINVAL,
                   "sizes must be positive (heads=%d kv=%d head_dim=%d page_size=%d n_pages=%d)",
                   s->n_heads, s->n_kv, s->head_dim, s->page_size, s->n_pages);
  if (s->dtype != XP_BF16 && s->dtype != XP_E4M3 && s->dtype != XP_MXFP4)
    return kv_fail(nullptr, XP_EINVAL, "dtype %d is not XP_BF16, XP_E4M3 or XP_MXFP4", s->dtype);
  if (max_batch < 1 || max_batch > kKvMaxBatch || max_tokens < 1 || max_tokens > (1 << 20) ||
      max_len < 1 || max_len > kKvMaxLen || (shared != 0 && shared != 1))
    return kv_fail(nullptr, XP_EINVAL,
                   "max_batch=%d (1..%d), max_tokens=%d (1..2^20), max_len=%d (1..2^22) or "
                   "shared=%d (0, 1) out of range", max_batch, kKvMaxBatch, max_tokens, max_len,
                   shared);
  const int P = s->page_size, hd = s->head_dim;
  if ((hd != 64 && hd != 128) || s->n_heads % s->n_kv != 0 || s->n_heads / s->n_kv > 64 ||
      s->n_heads > 1024 || P < 16 || P > 256 || (P & (P - 1)) != 0 ||
      (int64_t)s->n_pages * P >= ((int64_t)1 << 31))
    return kv_fail(nullptr, XP_EUNSUPPORTED,
                   "shape not built: head_dim %d (64, 128), heads/kv %d/%d (a whole group up to 64, "
                   "up to 1024 heads), page_size %d (16, 32, 64, 128, 256), n_pages * page_size %lld "
                   "(below 2^31)", hd, s->n_heads, s->n_kv, P, (long long)s->n_pages * P);
  xp_kv* kv = new (std::nothrow) xp_kv();
  if (kv == nullptr) return kv_fail(nullptr, XP_ENOMEM, "host allocation failed");
  kv->nh = s->n_heads;
  kv->nkv = s->n_kv;
  kv->grp = s->n_heads / s->n_kv;
  kv->hd = hd;
  kv->P = P;
  kv->logP = __builtin_ctz((unsigned)P);
  kv->n_pages = s->n_pages;
  kv->dtype = s->dtype;
  kv->max_batch = max_batch;
  kv->max_tokens = max_tokens;
  kv->max_len = max_len;
  kv->max_pages = (max_len + P - 1) / P;
  kv->shared = shared;
  hipError_t e = hipGetDevice(&kv->device);
  if (e == hipSuccess)
    e = hipDeviceGetAttribute(&kv->cus, hipDeviceAttributeMultiprocessorCount, kv->device);
  if (e != hipSuccess) {
    delete kv;
    return kv_fail(nullptr, XP_EHIP, "device query failed: %s", hipGetErrorString(e));
  }
  kv->cus = kv->cus > 0 ? kv->cus : 256;
  int shares = 0;
  kv_attn_sizes(kv, &kv->rows, &kv->entries, &shares);
  const size_t lists = shared ? 2 : 1, nb = (size_t)max_batch;
  const size_t prows = lists * kv->rows + (shared ? (size_t)2 * max_tokens * kv->nh : 0);
  // slices of the workspace
  KvList &l0 = kv->a.list[0], &l1 = kv->a.list[1];
  struct Slice { void** at; size_t bytes; };
  char* zero = nullptr;
  int32_t *acu = nullptr, *len = nullptr;
  const Slice slices[] = {
      {(void**)&zero, 256},
      {(void**)&kv->err, 256},
      {(void**)&kv->top, 256},
      {(void**)&kv->take, (nb + 1) * 4},
      {(void**)&kv->old, nb * 4},
      {(void**)&acu, (nb + 1) * 4},
      {(void**)&len, nb * 4},
      {(void**)&kv->a.dump, 512},
      {(void**)&l0.hdr, 256},
      {(void**)&l0.share, ((size_t)shares + 1) * sizeof(KvShare)},
      {(void**)&l0.ent, lists * kv->entries * sizeof(KvEntry)},
      {(void**)&l0.cum, (lists * kv->entries + 1) * 4},
      {(void**)&l1.hdr, (size_t)(shared ? 256 : 0)},
      {(void**)&l1.share, shared ? ((size_t)shares + 1) * sizeof(KvShare) : 0},
      {(void**)&l1.ent, shared ? (size_t)kv->entries * sizeof(KvEntry) : 0},
      {(void**)&l1.cum, shared ? ((size_t)kv->entries + 1) * 4 : 0},
      {(void**)&kv->a.pos, shared ? (size_t)max_tokens * 4 : 0},
      {(void**)&kv->a.row[0], shared ? (size_t)max_tokens * 8 : 0},
      {(void**)&kv->a.row[1], shared ? (size_t)max_tokens * 8 : 0},
      {(void**)&kv->a.ml, prows * 8},
      {(void**)&kv->a.part, prows * hd * 4},
  };
  size_t total = 0;
  for (const Slice& sl : slices) total += (sl.bytes + 255) / 256 * 256;
  e = hipMalloc(&kv->ws, total);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    delete kv;
    return kv_fail(nullptr, XP_ENOMEM, "workspace of %zu bytes: %s", total, hipGetErrorString(e));
  }
  char* at = static_cast<char*>(kv->ws);
  for (const Slice& sl : slices) {
    *sl.at = at;
    at += (sl.bytes + 255) / 256 * 256;
  }
  kv->a.zero = zero;
  kv->acu = acu;
  kv->len = len;
  // the zero row and the device error word; done before the call returns
  e = hipMemset(kv->ws, 0, 512);
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e != hipSuccess) {
    (void)hipFree(kv->ws);
    delete kv;
    return kv_fail(nullptr, XP_EHIP, "workspace: %s", hipGetErrorString(e));
  }
  *out = kv;
  return XP_OK;
}

extern "C" void xp_kv_destroy(xp_kv* kv) {
  if (kv == nullptr) return;
  (void)hipDeviceSynchronize();
  if (kv->ws) (void)hipFree(kv->ws);
  delete kv;
}

// The workspace lives on the handle's device: a call from another one would
// launch there.
static xp_status kv_device(xp_kv* kv) {
  int dev = -1;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return kv_fail(kv, XP_EHIP, "device query failed: %s", hipGetErrorString(e));
  if (dev != kv->device)
    return kv_fail(kv, XP_EINVAL, "the current device is %d, the handle's %d", dev, kv->device);
  return XP_OK;
}

static bool misaligned(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 != 0; }

extern "C" xp_status xp_kv_map(xp_kv* kv, int32_t n, const int32_t* lens, const int32_t* add,
                               int32_t* table, int64_t table_ld, int32_t* held, int32_t* pool,
                               int32_t* pool_n, int32_t* cu, int32_t* kv_len, int32_t* slots,
                               int32_t max_slots, void* stream) {
  if (kv == nullptr) return XP_EINVAL;
  if (n < 0 || n > kv->max_batch)
    return kv_fail(kv, XP_EINVAL, "n=%d out of range 0..%d", n, kv->max_batch);
  if (lens == nullptr || add == nullptr || table == nullptr || held == nullptr ||
      pool == nullptr || pool_n == nullptr)
    return kv_fail(kv, XP_EINVAL, "lens, add, table, held, pool and pool_n are required");
  if (table_ld < 1 || max_slots < 0)
    return kv_fail(kv, XP_EINVAL, "table_ld=%lld (>= 1) or max_slots=%d (>= 0) out of range",
                   (long long)table_ld, max_slots);
  const xp_status ds = kv_device(kv);
  if (ds != XP_OK) return ds;
  KvMap d{};
  d.n = n;
  d.logP = kv->logP;
  d.cols = (int)std::min<int64_t>(kv->max_pages, table_ld);
  d.n_pages = kv->n_pages;
  d.max_slots = slots ? max_slots : 0;
  d.lens = lens;
  d.add = add;
  d.table = table;
  d.ld = table_ld;
  d.held = held;
  d.pool = pool;
  d.pool_n = pool_n;
  d.cu = cu;
  d.kv_len = kv_len;
  d.slots = slots;
  d.take = kv->take;
  d.old = kv->old;
  d.acu = kv->acu;
  d.len = kv->len;
  d.top = kv->top;
  d.err = kv->err;
  hipStream_t st = (hipStream_t)stream;
  hipError_t e;
  if (d.max_slots <= kMapOneLaunch) {
    hipLaunchKernelGGL(k_kv_map<true>, dim3(1), dim3(kMapThreads), 0, st, d);
    e = hipGetLastError();
  } else {
    hipLaunchKernelGGL(k_kv_map<false>, dim3(1), dim3(kMapThreads), 0, st, d);
    if ((e = hipGetLastError()) == hipSuccess) {
      const int wgs = (int)std::min<int64_t>(((int64_t)d.max_slots + 1023) / 1024, 1024);
      hipLaunchKernelGGL(k_kv_slots, dim3(wgs), dim3(256), 0, st, d);
      e = hipGetLastError();
    }
  }
  if (e != hipSuccess) return kv_fail(kv, XP_EHIP, "map launch failed: %s", hipGetErrorString(e));
  return XP_OK;
}

// Checks of the cache's buffers, shared by the entry points that touch them.
static xp_status kv_cache_args(xp_kv* kv, const void* kc, const void* vc, const float* ks,
                               const float* vs) {
  if (kc == nullptr || vc == nullptr || misaligned(kc) || misaligned(vc))
    return kv_fail(kv, XP_EINVAL, "k_cache or v_cache is NULL or not 16-byte aligned");
  if (kv->dtype != XP_E4M3 && (ks != nullptr || vs != nullptr))
    return kv_fail(kv, XP_EINVAL, "only an 8-bit cache has scales of the caller's");
  return XP_OK;
}

extern "C" xp_status xp_kv_write(xp_kv* kv, int32_t tokens, const void* k, int64_t k_ld,
                                 const void* v, int64_t v_ld, const int32_t* slots, void* k_cache,
                                 void* v_cache, const float* k_scale, const float* v_scale,
                                 void* stream) {
  if (kv == nullptr) return XP_EINVAL;
  if (tokens < 0 || tokens > kv->max_tokens)
    return kv_fail(kv, XP_EINVAL, "tokens=%d out of range 0..%d", tokens, kv->max_tokens);
  const int64_t row = (int64_t)kv->nkv * kv->hd;
  if (k == nullptr || v == nullptr || slots == nullptr || misaligned(k) || misaligned(v) ||
      k_ld < row || v_ld < row || k_ld % 8 != 0 || v_ld % 8 != 0)
    return kv_fail(kv, XP_EINVAL,
                   "k, v (16-byte aligned) and slots are required, k_ld=%lld and v_ld=%lld at least "
                   "n_kv*head_dim=%lld and multiples of 8", (long long)k_ld, (long long)v_ld,
                   (long long)row);
  xp_status s = kv_cache_args(kv, k_cache, v_cache, k_scale, v_scale);
  if (s == XP_OK) s = kv_device(kv);
  if (s != XP_OK || tokens == 0) return s;
  const hipError_t e = launch_kv_write(kv, tokens, (const uint16_t*)k, (const uint16_t*)v, k_ld,
                                       v_ld, slots, nullptr, 0, nullptr, 0, k_cache, v_cache,
                                       k_scale, v_scale, (hipStream_t)stream);
  if (e != hipSuccess) return kv_fail(kv, XP_EHIP, "write launch failed: %s", hipGetErrorString(e));
  return XP_OK;
}

extern "C" xp_status xp_kv_read(xp_kv* kv, int32_t tokens, const int32_t* slots,
                                const void* k_cache, const void* v_cache, const float* k_scale,
                                const float* v_scale, void* k, int64_t k_ld, void* v, int64_t v_ld,
                                void* stream) {
  if (kv == nullptr) return XP_EINVAL;
  if (tokens < 0 || tokens > kv->max_tokens)
    return kv_fail(kv, XP_EINVAL, "tokens=%d out of range 0..%d", tokens, kv->max_tokens);
  const int64_t row = (int64_t)kv->nkv * kv->hd;
  if ((k == nullptr && v == nullptr) || slots == nullptr || misaligned(k) || misaligned(v) ||
      (k != nullptr && (k_ld < row || k_ld % 8 != 0)) ||
      (v != nullptr && (v_ld < row || v_ld % 8 != 0)))
    return kv_fail(kv, XP_EINVAL,
                   "slots and one of k and v (16-byte aligned) are required, k_ld=%lld and v_ld=%lld "
                   "at least n_kv*head_dim=%lld and multiples of 8", (long long)k_ld,
                   (long long)v_ld, (long long)row);
  xp_status s = kv_cache_args(kv, k_cache, v_cache, k_scale, v_scale);
  if (s == XP_OK) s = kv_device(kv);
  if (s != XP_OK || tokens == 0) return s;
  const hipError_t e = launch_kv_read(kv, tokens, slots, k_cache, v_cache, k_scale, v_scale,
                                      (uint16_t*)k, (uint16_t*)v, k_ld, v_ld, (hipStream_t)stream);
  if (e != hipSuccess) return kv_fail(kv, XP_EHIP, "read launch failed: %s", hipGetErrorString(e));
  return XP_OK;
}

static xp_status kv_attn(xp_kv* kv, const KvAttnArgs& a, void* stream) {
  if (a.n < 0 || a.n > kv->max_batch || a.total_q < 0 || a.total_q > kv->max_tokens ||
      a.max_q < 0 || a.max_q > kv->max_tokens)
    return kv_fail(kv, XP_EINVAL,
                   "n=%d (0..%d), tokens=%d (0..%d) or max_q=%d (0..%d) out of range", a.n,
                   kv->max_batch, a.total_q, kv->max_tokens, a.max_q, kv->max_tokens);
  if (a.cu_q == nullptr && (int64_t)a.n * a.max_q != a.total_q)
    return kv_fail(kv, XP_EINVAL, "without cu_q, tokens=%d must be n=%d times max_q=%d", a.total_q,
                   a.n, a.max_q);
  if (a.q == nullptr || a.out == nullptr || a.kv_len == nullptr || a.table == nullptr ||
      misaligned(a.q) || misaligned(a.out))
    return kv_fail(kv, XP_EINVAL,
                   "q, out (16-byte aligned), kv_len and table are required");
  const int64_t row = (int64_t)kv->nh * kv->hd;
  if (a.q_ld < row || a.out_ld < row || a.q_ld % 8 != 0 || a.out_ld % 8 != 0 || a.table_ld < 1)
    return kv_fail(kv, XP_EINVAL,
                   "q_ld=%lld and out_ld=%lld must be at least n_heads*head_dim=%lld and multiples "
                   "of 8, table_ld=%lld at least 1", (long long)a.q_ld, (long long)a.out_ld,
                   (long long)row, (long long)a.table_ld);
  if ((a.causal != 0 && a.causal != 1) || a.window < 0 || a.window > kKvMaxLen || a.sinks < 0 ||
      a.sinks > kKvMaxLen || !(a.scale == 0.f || (a.scale >= 0x1p-60f && a.scale <= 0x1p60f)))
    return kv_fail(kv, XP_EINVAL,
                   "causal=%d (0, 1), window=%d, sinks=%d (0..2^22) or scale=%g (0, 2^-60..2^60) out "
                   "of range", a.causal, a.window, a.sinks, (double)a.scale);
  const xp_status s = kv_cache_args(kv, a.kc, a.vc, a.k_scale, a.v_scale);
  if (s != XP_OK) return s;
  if (!kv_units_fit(kv, a.total_q, a.n, a.groups, a.table_ld, a.max_q))
    return kv_fail(kv, XP_EINVAL, "the call's tokens and max_len reach 2^31 key tiles");
  const xp_status ds = kv_device(kv);
  if (ds != XP_OK || a.n == 0 || a.total_q == 0) return ds;
  const hipError_t e = launch_kv_attn(kv, a, (hipStream_t)stream);
  if (e != hipSuccess)
    return kv_fail(kv, XP_EHIP, "attention launch failed: %s", hipGetErrorString(e));
  return XP_OK;
}

extern "C" xp_status xp_kv_attn(xp_kv* kv, int32_t n, int32_t tokens, int32_t max_q, const void* q,
                                int64_t q_ld, const int32_t* cu_q, const int32_t* kv_len,
                                const int32_t* table, int64_t table_ld, const void* k_cache,
                                const void* v_cache, const float* k_scale, const float* v_scale,
                                int32_t causal, int32_t window, int32_t sinks, float scale,
                                void* out, int64_t out_ld, float* lse, void* stream) {
  if (kv == nullptr) return XP_EINVAL;
  KvAttnArgs a{};
  a.n = n;
  a.total_q = tokens;
  a.max_q = max_q;
  a.cu_q = cu_q;
  a.kv_len = kv_len;
  a.table = table;
  a.table_ld = table_ld;
  a.q = (const uint16_t*)q;
  a.q_ld = q_ld;
  a.kc = k_cache;
  a.vc = v_cache;
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.causal = causal;
  a.window = window;
  a.sinks = sinks;
  a.scale = scale;
  a.out = (uint16_t*)out;
  a.out_ld = out_ld;
  a.lse = lse;
  return kv_attn(kv, a, stream);
}

extern "C" xp_status xp_kv_attn_shared(xp_kv* kv, int32_t n, int32_t tokens, int32_t max_q,
                                       int32_t groups, const int32_t* group_start,
                                       const int32_t* shared_len, const void* q, int64_t q_ld,
                                       const int32_t* cu_q, const int32_t* kv_len,
                                       const int32_t* table, int64_t table_ld, const void* k_cache,
                                       const void* v_cache, const float* k_scale,
                                       const float* v_scale, int32_t causal, int32_t window,
                                       int32_t sinks, float scale, void* out, int64_t out_ld,
                                       float* lse, void* stream) {
  if (kv == nullptr) return XP_EINVAL;
  if (!kv->shared) return kv_fail(kv, XP_EINVAL, "the handle was created without shared prefixes");
  if (groups < 1 || groups > n || group_start == nullptr || shared_len == nullptr)
    return kv_fail(kv, XP_EINVAL, "groups=%d out of range 1..n=%d, or group_start or shared_len is "
                   "NULL", groups, n);
  KvAttnArgs a{};
  a.n = n;
  a.total_q = tokens;
  a.max_q = max_q;
  a.cu_q = cu_q;
  a.kv_len = kv_len;
  a.table = table;
  a.table_ld = table_ld;
  a.q = (const uint16_t*)q;
  a.q_ld = q_ld;
  a.kc = k_cache;
  a.vc = v_cache;
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.causal = causal;
  a.window = window;
  a.sinks = sinks;
  a.scale = scale;
  a.out = (uint16_t*)out;
  a.out_ld = out_ld;
  a.lse = lse;
  a.groups = groups;
  a.group_start = group_start;
  a.shared_len = shared_len;
  return kv_attn(kv, a, stream);
}

extern "C" xp_status xp_kv_device_errors(xp_kv* kv, uint32_t* out, void* stream) {
  if (kv == nullptr) return XP_EINVAL;
  if (out == nullptr) return kv_fail(kv, XP_EINVAL, "out is NULL");
  const xp_status s = kv_device(kv);
  if (s != XP_OK) return s;
  hipStream_t st = (hipStream_t)stream;
  hipError_t e = hipMemcpyAsync(out, kv->err, sizeof(uint32_t), hipMemcpyDeviceToHost, st);
  if (e == hipSuccess) {
    hipLaunchKernelGGL(k_kv_clear_err, dim3(1), dim3(64), 0, st, kv->err);
    e = hipGetLastError();
  }
  if (e == hipSuccess) e = hipStreamSynchronize(st);
  if (e != hipSuccess) return kv_fail(kv, XP_EHIP, "device errors: %s", hipGetErrorString(e));
  return XP_OK;
}
