// Attention over the paged context cache: single tokens, drafted blocks and
// prompts, with an optional sliding window and first keys that stay visible,
// and with prefixes that several sequences share.
//
// Row (token i of sequence b, head h) has position p = kv_len[b] - q_len[b] + i
// and sees key j iff
//   j < kv_len[b]  and  (not causal or j <= p)  and
//   (window == 0 or j > p - window or j < sinks);
// o = sum_j softmax_j(scale q.k_j) v_j over these, 0 if there are none (and 0 / 0 if
// every score is -inf).
//
// Work list (k_kv_plan, plan_own).  The rows of a KV head's group, (token, head) pairs,
// are cut into tiles of up to R rows; a tile walks the 64-key tiles that any of
// its rows sees.  (row tile, KV head, key tile) in this order is a list of units
// that k_kv_attn cuts into equal shares, one a workgroup, whatever the lengths:
// long and short contexts, prompts beside single tokens, causal triangles and
// windows all carry the same load.  A share that begins or ends inside a (row
// tile, KV head) segment leaves a partial (O, reference maximum, sum), and
// k_kv_join adds the parts of every cut segment in order; a segment inside one
// share is written at once.  The same call gives the same bits.
//
// With shared prefixes a group's prefix keys are segments of their own, whose
// rows are all tokens of the group, so that they are read once for all of them, and
// each sequence's own segments begin behind the prefix.  k_kv_join_rows adds both
// results of every row.
#include <algorithm>
#include <cmath>

#include "xp_kv.h"

namespace xp {

typedef float floatx16 __attribute__((ext_vector_type(16)));
// read-only data at wave-uniform addresses: scalar loads
#define XP_AS4 __attribute__((address_space(4)))
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef const XP_AS4 int32_t* scalar_i32;

__device__ __forceinline__ scalar_i32 as_scalar(const void* p) {
  return (scalar_i32)(uintptr_t)p;
}
__device__ __forceinline__ float fsum_xor32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float fsum_xor16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ uint32_t umax_xor16(uint32_t x) {
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return max(r[0], r[1]);
}
__device__ __forceinline__ uint32_t umax_xor32(uint32_t x) {
  const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return max(r[0], r[1]);
}
__device__ __forceinline__ int imin(int a, int b) { return a < b ? a : b; }
__device__ __forceinline__ int imax(int a, int b) { return a > b ? a : b; }

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return imin(imax(x, lo), hi); }

// What the work lists follow from.
struct KvPlan {
  int n, total_q, max_q, kv_add, cap, grp, nkv, causal, window, sinks, groups;
  int entries;                       // that a list holds at most
  int R[2], shares[2];               // of each list
  const int32_t* cu_q;
  const int32_t* kv_len;
  const int32_t* group_start;
  const int32_t* shared_len;
};

// What the attention's kernels read of a call.
struct KvDev {
  const uint16_t* q;
  int64_t q_ld;
  uint16_t* out;
  int64_t out_ld;
  float* lse;
  const char* kc;
  const char* vc;
  const float* k_scale;
  const float* v_scale;
  const int32_t* table;
  int64_t table_ld;
  int nh, nkv, grp, logP, n_pages, cols;
  int causal, window, sinks;
  float scale2;                      // scale log2(e)
  int total_q, groups;
  KvPlan p;
  KvList list;                       // the work
  int64_t part0, row0;               // first partial row of its cut segments; of whole ones
  KvAttnWs w;
  uint32_t* err;
};

// ---------------------------------------------------------------------------
// The work lists, one workgroup each.  Items of the first are the sequences (with
// their keys behind a shared prefix, if they have one); the groups (their prefixes)
// follow them or are the items of a second list.  The items' row tiles, the entries'
// key ranges, the sums of both, and where each share begins.  Bound by latency, a few
// block scans and one search per entry and share: 64 sequences 7.2 us, 60 behind
// five prefixes 9.7.  (Small calls: plan_own.)
// ---------------------------------------------------------------------------
constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kPlanCum = 4096;       // entries whose sums stay in LDS
// Units that a segment counts beside its key tiles, for its rows' loads, its first
// tile's latency and its results: without them the shares at the beginnings of
// prompts, many segments of a few tiles, ran 1.65 ms where the others took 1.0.
constexpr int kSegUnits = 3;
// A share has one unit at least: small calls spread over all workgroups, a tile each,
// and leave the parts to the join (one token over 180 .. 500 keys: 14.3 .. 14.8 us,
// with shares of two units 16.3 .. 16.5, of five 18.6 .. 20.5).
constexpr int kPlanMinShare = 1;

// exclusive sum over the workgroup of each thread's v, 0 from thread `count` on (whose
// waves stay out of it); *total their sum
__device__ __forceinline__ int block_scan(int v, int count, int* lds, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int waves = imin((count + kWave - 1) / kWave, kPlanWaves);
  int x = v;
  if (wave < waves) {
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int y = __shfl_up(x, o, kWave);
      if (lane >= o) x += y;
    }
  }
  __syncthreads();
  if (wave < waves && lane == kWave - 1) lds[wave] = x;
  __syncthreads();
  int before = 0, all = 0;
  for (int w = 0; w < waves; ++w) {
    const int t = lds[w];
    before += w < wave ? t : 0;
    all += t;
  }
  *total = all;
  return before + x - v;
}

// first token of sequence b
__device__ __forceinline__ int plan_first(const KvPlan& d, int b) {
  return d.cu_q != nullptr ? clampi(d.cu_q[b], 0, d.total_q) : imin(b * d.max_q, d.total_q);
}
// its keys
__device__ __forceinline__ int plan_keys(const KvPlan& d, int b, uint32_t& bad) {
  const int x = d.kv_len[b];
  if (x < 0 || x > d.cap - d.kv_add) bad |= XP_DEVERR_LENGTH;
  return clampi(x, 0, imax(d.cap - d.kv_add, 0)) + imin(d.kv_add, d.cap);
}
// the key tiles of an entry whose tokens have positions pa .. pb
__device__ __forceinline__ void plan_tiles(const KvPlan& d, KvEntry& x, int pa, int pb) {
  x.hi = d.causal ? imin(x.ceil, pb + 1) : x.ceil;
  x.lo = d.window > 0 ? imax(pa - d.window + 1, x.floor) : x.floor;
  x.s = d.window > 0 ? imax(imin(d.sinks, x.hi), x.floor) : x.floor;
  const bool sink = x.s > x.floor;
  const int fl = x.floor / kKvTile;
  x.a0 = sink ? fl : x.lo / kKvTile;
  const int a1 = sink ? (x.s + kKvTile - 1) / kKvTile : x.a0;
  x.n1 = a1 - x.a0;
  x.b0 = imax(x.lo / kKvTile, a1);
  const int b1 = x.hi > x.lo ? (x.hi + kKvTile - 1) / kKvTile : 0;
  // no row sees a key: one tile, wholly masked, writes the zeros
  x.tiles = imax(x.n1 + imax(b1 - x.b0, 0), 1);
}
// the entry of the rows from x.row0 on of sequence i, its tk tokens from t0 on
__device__ __forceinline__ void plan_rows(const KvPlan& d, KvEntry& x, int i, int t0, int tk,
                                          int keys, int floor, int R) {
  x.tok0 = t0;
  x.seq = i;
  x.nrows = imin(tk * d.grp - x.row0, R);
  x.ceil = keys;
  x.p0 = keys - tk;
  x.floor = floor;
  plan_tiles(d, x, x.p0 + x.row0 / d.grp, x.p0 + (x.row0 + x.nrows - 1) / d.grp);
}

template <bool SHARED>
__global__ __launch_bounds__(kPlanThreads) void k_kv_plan(const KvPlan d, const KvAttnWs w,
                                                                uint32_t* __restrict__ err) {
  __shared__ int off[(SHARED ? 2 : 1) * kKvMaxBatch + 1];   // entries before each item
  __shared__ int floors[SHARED ? kKvMaxBatch : 1];   // keys of the sequence that its prefix holds
  __shared__ int gmin[SHARED ? kKvMaxBatch : 1];  // a group's positions: least and greatest
  __shared__ int gmax[SHARED ? kKvMaxBatch : 1];
  __shared__ int glen[SHARED ? kKvMaxBatch : 1];  // and its prefix keys
  __shared__ int gseq[SHARED ? kKvMaxBatch : 1];  // its first request that has tokens
  __shared__ int cums[kPlanCum];
  __shared__ int red[kPlanWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = d.n;
  const bool second = SHARED && blockIdx.x == 1;
  const int ns = second ? 0 : n;                  // items that are sequences
  const int items = ns + (SHARED && (second || gridDim.x == 1) ? d.groups : 0);
  const int R = d.R[second], shares = d.shares[second];
  const KvList out = w.list[second];
  uint32_t bad = 0;
  auto first = [&](int b) { return plan_first(d, b); };
  auto keys = [&](int b) { return plan_keys(d, b, bad); };
  auto tokens = [&](int b, int t0) { return imax(first(b + 1) - t0, 0); };
  auto members = [&](int g, int& s0, int& s1) {
    s0 = clampi(d.group_start[g], 0, n);
    s1 = clampi(d.group_start[g + 1], s0, n);
  };
  if constexpr (SHARED) {
    for (int b = tid; b < n; b += kPlanThreads) floors[b] = 0;
    for (int t = tid; t < d.total_q; t += kPlanThreads) {   // tokens of no sequence, of no group
      if (!second) w.row[0][t] = int2{-1, 0};
      if (items > ns) w.row[1][t] = int2{-1, 0};
    }
    // Groups that run backwards could hold a request twice: then none is shared.  Every
    // wave looks through all of them (an or over the workgroup took 0.3 us longer).
    bool back = false;
    for (int g = lane; g < d.groups; g += kWave) {
      const int s0 = d.group_start[g], s1 = d.group_start[g + 1];
      back |= s1 < s0;
      bad |= (s1 < s0) | (s0 < 0) | (s1 > n) ? XP_DEVERR_LENGTH : 0u;
    }
    const bool apart = __ballot(back) != 0;
    __syncthreads();
    // a wave per group: its members' positions, and a prefix that none is shorter than
    for (int g = wave; g < d.groups; g += kPlanWaves) {
      int s0, s1;
      members(g, s0, s1);
      int pmin = 0x7fffffff, pmax = -0x7fffffff, kmin = d.cap, smin = n;
      for (int b = s0 + lane; b < s1; b += kWave) {
        const int t0 = first(b), ql = tokens(b, t0), kv = keys(b);
        if (ql == 0) continue;
        pmin = imin(pmin, kv - ql);
        pmax = imax(pmax, kv - 1);
        kmin = imin(kmin, kv);
        smin = imin(smin, b);
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        pmin = imin(pmin, __shfl_xor(pmin, o, kWave));
        pmax = imax(pmax, __shfl_xor(pmax, o, kWave));
        kmin = imin(kmin, __shfl_xor(kmin, o, kWave));
        smin = imin(smin, __shfl_xor(smin, o, kWave));
      }
      const int want = d.shared_len[g], len = apart ? 0 : clampi(want, 0, kmin);
      if (want != len) bad |= XP_DEVERR_LENGTH;
      for (int b = s0 + lane; b < s1; b += kWave) floors[b] = len;
      if (lane == 0) {
        gmin[g] = pmin;
        gmax[g] = pmax;
        glen[g] = len;
        gseq[g] = smin;
      }
    }
    __syncthreads();
  }
  // entries of each item; where token ranges overlap, as many as the tokens could have
  const int most = (items > n ? 2 : 1) * d.entries;
  int T = 0;
  for (int i0 = 0; i0 < items; i0 += kPlanThreads) {
    const int i = i0 + tid;
    int nt = 0;
    if (i < items) {
      int tk;
      if (i < ns) {
        tk = tokens(i, first(i));
      } else {
        int s0, s1;
        members(i - ns, s0, s1);
        tk = glen[i - ns] > 0 ? imax(first(s1) - first(s0), 0) : 0;
      }
      nt = (int)(((int64_t)tk * d.grp + R - 1) / R);
    }
    int all;
    const int before = block_scan(nt, items - i0, red, &all);
    if (i < items) off[i] = T + before;
    T = T > most ? T : T + all;                   // stays far below 2^31
  }
  if (tid == 0) off[items] = T;
  if (T > most) {
    T = most;
    bad |= XP_DEVERR_LENGTH;
  }
  __syncthreads();
  if constexpr (SHARED) {                         // a wave per item: where its tokens' rows are
    if (!second)
      for (int b = wave; b < n; b += kPlanWaves) {
        const int t0 = first(b), ql = tokens(b, t0), p0 = keys(b) - ql;
        for (int i = lane; i < ql; i += kWave) {
          w.pos[t0 + i] = p0 + i;
          w.row[0][t0 + i] = int2{i * d.grp, off[b]};
        }
      }
    for (int g = wave; g < items - ns; g += kPlanWaves) {
      int s0, s1;
      members(g, s0, s1);
      const int t0 = first(s0), ql = glen[g] > 0 ? first(s1) - t0 : 0;
      for (int i = lane; i < ql; i += kWave) w.row[1][t0 + i] = int2{i * d.grp, off[ns + g]};
    }
  }
  // their key ranges
  int W = 0;
  for (int e0 = 0; e0 < T; e0 += kPlanThreads) {
    const int e = e0 + tid;
    int units = 0;
    if (e < T) {
      const int i = kv_owner((const int*)off, items, e);
      KvEntry x{};
      x.row0 = (e - off[i]) * R;
      int pa, pb;                                 // positions of the tile's tokens
      if (i < ns) {
        const int t0 = first(i);
        plan_rows(d, x, i, t0, tokens(i, t0), keys(i), SHARED ? floors[i] : 0, R);
      } else {
        int s0, s1;
        members(i - ns, s0, s1);
        x.tok0 = first(s0);
        x.seq = imin(gseq[i - ns], n - 1);
        x.nrows = imin((first(s1) - x.tok0) * d.grp - x.row0, R);
        x.prefix = 1;
        x.ceil = glen[i - ns];
        x.p0 = gmin[i - ns];
        x.p1 = gmax[i - ns];
        plan_tiles(d, x, x.p0, x.p1);
      }
      out.ent[e] = x;
      units = (x.tiles + kSegUnits) * d.nkv;
    }
    int all;
    const int before = block_scan(units, T - e0, red, &all);
    if (e < T) {
      if (e < kPlanCum) cums[e] = W + before;
      out.cum[e] = W + before;
    }
    W += all;
  }
  const int S = imax((W + shares - 1) / shares, kPlanMinShare);
  if (tid == 0) {
    out.cum[T] = W;
    out.hdr[0] = W;
    out.hdr[1] = S;
    out.hdr[2] = T;
  }
  __syncthreads();                                // also the entries, for this workgroup
  for (int s = tid; s <= shares; s += kPlanThreads) {
    KvShare r{};
    r.f = (int64_t)s * S < W ? s * S : W;
    if (r.f < W) {
      r.e = T <= kPlanCum ? kv_owner((const int*)cums, T, r.f)
                          : kv_owner((const int32_t*)out.cum, T, r.f);
      const int units = out.ent[r.e].tiles + kSegUnits;
      const int in = r.f - (T <= kPlanCum ? cums[r.e] : out.cum[r.e]);
      r.kvh = in / units;
      r.j = in - r.kvh * units - kSegUnits;       // negative: before the first tile
    }
    out.share[s] = r;
  }
  if (bad) atomicOr(err, bad);
}

// ---------------------------------------------------------------------------
// The attention.
// ---------------------------------------------------------------------------
// Layout of a stage: a tile's 64 K rows, then its 64 V rows, of RB bytes; the
// 16-byte chunk c of row r at position c ^ swz(r), so that neither the K reads
// (16 rows, one chunk) nor the transposing V reads (4 or 8 rows, 4 or 2 chunks)
// meet in a bank.
template <int HD, bool F8>
struct KvRows {
  static constexpr int RB = HD * (F8 ? 1 : 2);
  static constexpr int CPR = RB / 16;
  static constexpr int kHalf = kKvTile * CPR;     // 16-byte slots of K, of V
  static constexpr int kStage = 2 * kHalf;
  static constexpr int IPG = CPR / 4;             // 1 KB loads of 16 rows
  __device__ static __forceinline__ int swz(int r) {
    if constexpr (CPR == 16) return ((r & 3) << 2) | ((r >> 2) & 3);
    else if constexpr (CPR == 8 && !F8) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    else if constexpr (CPR == 8)
      return (((r >> 1) & 1) << 2) | (((r >> 3) & 1) << 1) | ((r >> 2) & 1);
    else return (((r >> 3) & 1) << 1) | ((r >> 2) & 1);
  }
};

// the same of K's codes in 4 bits: 16-byte chunk c of row r at position c ^ swz4(r)
template <int HD>
__device__ __forceinline__ int kv_swz4(int r) { return HD == 128 ? (r >> 2) & 3 : (r >> 3) & 1; }

__device__ __forceinline__ floatx16 mma32(u32x4 a, u32x4 b, floatx16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// the same of P and V: fp16 over an 8-bit cache
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
template <bool F8>
__device__ __forceinline__ floatx16 mma32_pv(u32x4 a, u32x4 b, floatx16 c) {
  if constexpr (F8)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a),
                                                  __builtin_bit_cast(half8, b), c, 0, 0, 0);
  else return mma32(a, b, c);
}
template <bool F8>
__device__ __forceinline__ uint32_t pk_p(float a, float b) {
  if constexpr (F8)
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(xp_f32x2{a, b}, half2v));
  else return pk_bf16(a, b);
}
// 8 e4m3 values to fp16 (exact)
__device__ __forceinline__ u32x4 f8_f16x8(uint32_t a, uint32_t b) {
  return u32x4{
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, false)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, true)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, false)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, true))};
}
// 8 e4m3 values to bf16 (exact)
__device__ __forceinline__ u32x4 f8_bf16x8(uint32_t a, uint32_t b) {
  return u32x4{
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true))};
}
// 8 e2m1 codes times a power of two to bf16 (exact; NaN for the exponent 255)
__device__ __forceinline__ u32x4 f4_bf16x8(uint32_t a, float s) {
  return u32x4{
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a, s, 0)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a, s, 1)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a, s, 2)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a, s, 3))};
}
__device__ __forceinline__ uint32_t lds_byte(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

// V operands of two 16-key steps (OFF bytes into the lane's addresses, the second
// 16 rows of RB bytes further) for ND blocks of 32 dims, with the wait for the
// reads: a[] the lane's part of each block, b[] (+ 8 RB) the same of the keys 8
// further (8-bit rows: one read brings both groups of four keys).  Written out
// because the compiler takes its transposing-read builtin for a use of the
// global-to-LDS loads in flight and waits for all of them.
template <int ND, bool F8, int OFF, int RB>
__device__ __forceinline__ void lds_v(const uint32_t* a, const uint32_t* b, u32x4 (&v)[2][ND]) {
  constexpr int ON = OFF + 16 * RB, OB = OFF + 8 * RB, ONB = OFF + 24 * RB;
  if constexpr (!F8 && ND == 4) {
    uint2 r[16];
    asm volatile(
        "ds_read_b64_tr_b16 %0, %16 offset:%24\n\t"
        "ds_read_b64_tr_b16 %1, %20 offset:%25\n\t"
        "ds_read_b64_tr_b16 %2, %17 offset:%24\n\t"
        "ds_read_b64_tr_b16 %3, %21 offset:%25\n\t"
        "ds_read_b64_tr_b16 %4, %18 offset:%24\n\t"
        "ds_read_b64_tr_b16 %5, %22 offset:%25\n\t"
        "ds_read_b64_tr_b16 %6, %19 offset:%24\n\t"
        "ds_read_b64_tr_b16 %7, %23 offset:%25\n\t"
        "ds_read_b64_tr_b16 %8, %16 offset:%26\n\t"
        "ds_read_b64_tr_b16 %9, %20 offset:%27\n\t"
        "ds_read_b64_tr_b16 %10, %17 offset:%26\n\t"
        "ds_read_b64_tr_b16 %11, %21 offset:%27\n\t"
        "ds_read_b64_tr_b16 %12, %18 offset:%26\n\t"
        "ds_read_b64_tr_b16 %13, %22 offset:%27\n\t"
        "ds_read_b64_tr_b16 %14, %19 offset:%26\n\t"
        "ds_read_b64_tr_b16 %15, %23 offset:%27\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]),
          "=&v"(r[6]), "=&v"(r[7]), "=&v"(r[8]), "=&v"(r[9]), "=&v"(r[10]),
          "=&v"(r[11]), "=&v"(r[12]), "=&v"(r[13]), "=&v"(r[14]), "=&v"(r[15])
        : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]),
          "n"(OFF), "n"(OB), "n"(ON), "n"(ONB)
        : "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i)
      v[i / ND][i % ND] = u32x4{r[2 * i].x, r[2 * i].y, r[2 * i + 1].x, r[2 * i + 1].y};
  } else if constexpr (!F8) {
    uint2 r[8];
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8 offset:%12\n\t"
        "ds_read_b64_tr_b16 %1, %10 offset:%13\n\t"
        "ds_read_b64_tr_b16 %2, %9 offset:%12\n\t"
        "ds_read_b64_tr_b16 %3, %11 offset:%13\n\t"
        "ds_read_b64_tr_b16 %4, %8 offset:%14\n\t"
        "ds_read_b64_tr_b16 %5, %10 offset:%15\n\t"
        "ds_read_b64_tr_b16 %6, %9 offset:%14\n\t"
        "ds_read_b64_tr_b16 %7, %11 offset:%15\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]),
          "=&v"(r[6]), "=&v"(r[7])
        : "v"(a[0]), "v"(a[1]), "v"(b[0]), "v"(b[1]),
          "n"(OFF), "n"(OB), "n"(ON), "n"(ONB)
        : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[i / ND][i % ND] = u32x4{r[2 * i].x, r[2 * i].y, r[2 * i + 1].x, r[2 * i + 1].y};
  } else if constexpr (ND == 4) {
    uint2 r[8];
    asm volatile(
        "ds_read_b64_tr_b8 %0, %8 offset:%12\n\t"
        "ds_read_b64_tr_b8 %1, %9 offset:%12\n\t"
        "ds_read_b64_tr_b8 %2, %10 offset:%12\n\t"
        "ds_read_b64_tr_b8 %3, %11 offset:%12\n\t"
        "ds_read_b64_tr_b8 %4, %8 offset:%13\n\t"
        "ds_read_b64_tr_b8 %5, %9 offset:%13\n\t"
        "ds_read_b64_tr_b8 %6, %10 offset:%13\n\t"
        "ds_read_b64_tr_b8 %7, %11 offset:%13\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]),
          "=&v"(r[6]), "=&v"(r[7])
        : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]),
          "n"(OFF), "n"(ON)
        : "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i / ND][i % ND] = f8_f16x8(r[i].x, r[i].y);
  } else {
    uint2 r[4];
    asm volatile(
        "ds_read_b64_tr_b8 %0, %4 offset:%6\n\t"
        "ds_read_b64_tr_b8 %1, %5 offset:%6\n\t"
        "ds_read_b64_tr_b8 %2, %4 offset:%7\n\t"
        "ds_read_b64_tr_b8 %3, %5 offset:%7\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3])
        : "v"(a[0]), "v"(a[1]),
          "n"(OFF), "n"(ON)
        : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i / ND][i % ND] = f8_f16x8(r[i].x, r[i].y);
  }
}

// Infinities and NaN among 16-bit (8-bit) values: the largest magnitudes so far (the
// bytes all of whose low bits were ones).
typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
template <bool F8>
struct KvOdd {
  uint32_t acc = 0;
  __device__ __forceinline__ void add(u32x4 x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (F8) {
        const uint32_t y = ~x[i] & 0x7f7f7f7fu;   // a byte 0: all seven bits are ones
        acc |= (y - 0x01010101u) & ~y;
      } else {
        const ushort2v m = __builtin_elementwise_max(
            __builtin_bit_cast(ushort2v, acc), __builtin_bit_cast(ushort2v, x[i] & 0x7fff7fffu));
        acc = __builtin_bit_cast(uint32_t, m);
      }
    }
  }
  __device__ __forceinline__ bool any() const {
    if constexpr (F8) return (acc & 0x80808080u) != 0u;
    else return (acc >= 0x7f800000u) | ((acc & 0xffffu) >= 0x7f80u);
  }
};

// the exponent's bits of V's operand: bf16, fp16 over an 8-bit cache
template <bool F8>
constexpr uint32_t kOddExp = F8 ? 0x7c00u : 0x7f80u;
// ones over each of the two values of x that is an infinity or NaN
template <bool F8>
__device__ __forceinline__ uint32_t nonfinite_mask(uint32_t x) {
  constexpr uint32_t E = kOddExp<F8>;
  return ((x & (E << 16)) == E << 16 ? 0xffff0000u : 0u) | ((x & E) == E ? 0xffffu : 0u);
}

// 1 where the value x is an infinity (c = 0), a negative one (1) or NaN (2)
template <bool F8>
__device__ __forceinline__ uint32_t ones_of(int c, uint32_t x) {
  constexpr uint32_t E = kOddExp<F8>;
  const bool is = c == 0 ? x == E : (c == 1 ? x == (E | 0x8000u) : (x & 0x7fffu) > E);
  return is ? (F8 ? 0x3c00u : 0x3f80u) : 0u;
}

// n KB of a page into LDS, 1 KB a load; a load's immediate offset counts for the
// memory and the LDS address alike.  The second with the non-temporal hint, for keys
// that one row tile streams: 48 single tokens over 4096 keys 157 -> 139 us (5.1 ->
// 5.8 TB/s), 32 blocks of 16 over 8192 225 -> 209; from 128 rows on no change.
__device__ __forceinline__ void kv_dma(const char* base, uint32_t lp, uint32_t x, int n, u32x4* dst) {
  const uint64_t b = (uint64_t)(uintptr_t)base;
  __builtin_amdgcn_global_load_lds((const void*)(uintptr_t)(b + lp), dst, 16, 0, 0);
  if (n > 1) __builtin_amdgcn_global_load_lds((const void*)(uintptr_t)(b + (lp ^ x)), dst, 16, 1 * 1024, 0);
  if (n > 2) {
    __builtin_amdgcn_global_load_lds((const void*)(uintptr_t)(b + (lp ^ (2 * x))), dst, 16, 2 * 1024, 0);
    __builtin_amdgcn_global_load_lds((const void*)(uintptr_t)(b + (lp ^ (3 * x))), dst, 16, 3 * 1024, 0);
  }
}

__device__ __forceinline__ void kv_dma_nt(const char* base, uint32_t lp, uint32_t x, int n, u32x4* dst) {
  const uint64_t b = (uint64_t)(uintptr_t)base;
  __builtin_amdgcn_global_load_lds((const void*)(uintptr_t)(b + lp), dst, 16, 0, 2);
  if (n > 1) __builtin_amdgcn_global_load_lds((const void*)(uintptr_t)(b + (lp ^ x)), dst, 16, 1 * 1024, 2);
  if (n > 2) {
    __builtin_amdgcn_global_load_lds((const void*)(uintptr_t)(b + (lp ^ (2 * x))), dst, 16, 2 * 1024, 2);
    __builtin_amdgcn_global_load_lds((const void*)(uintptr_t)(b + (lp ^ (3 * x))), dst, 16, 3 * 1024, 2);
  }
}

// the upper 32 lanes of a and the lower ones of b change places
__device__ __forceinline__ void swap_halves(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}

// A row's view of the keys: [lo, lo + n) and [floor, floor + s).
struct KvSees {
  int lo, floor;
  uint32_t n, s;
};

// a token at position p of a sequence of `keys` keys sees one of them
__device__ __forceinline__ bool sees_some(const KvDev& d, int p, int keys) {
  const int hi = d.causal ? imin(p + 1, keys) : keys;
  return (hi > 0) & ((d.window == 0) | (hi > p - d.window + 1) | (d.sinks > 0));
}

// inclusive sum over the wave
__device__ __forceinline__ int wave_scan(int v, int lane) {
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int y = __shfl_up(v, o, kWave);
    v += lane >= o ? y : 0;
  }
  return v;
}

// A work list of at most 64 entries of at most 64 sequences, made by one wave of every
// workgroup for itself, a lane per sequence and then per entry: small calls spare a launch
// and the way of the list through memory (one token over 100 keys 17.2 -> 14.6 us, 48 in a
// window 72.5 -> 70.8).  Entries to ent, the share's beginning to sh[0..3] (and its global
// copy, for k_kv_join) and its end to sh[4].
constexpr int kOwnEntries = kWave;
__device__ __forceinline__ void plan_own(const KvDev& d, int R, int shares, int sidx, KvEntry* ent,
                                         int32_t* sh) {
  const KvPlan& p = d.p;
  const int lane = threadIdx.x & 63, b = imin(lane, p.n - 1);
  uint32_t bad = 0;
  const int t0 = plan_first(p, b), t1 = plan_first(p, b + 1), keys = plan_keys(p, b, bad);
  const int tk = lane < p.n ? imax(t1 - t0, 0) : 0;
  const int nt = (tk * p.grp + R - 1) / R;
  const int upto = wave_scan(nt, lane), off = upto - nt, all = __shfl(upto, kWave - 1, kWave);
  bad |= all > p.entries ? XP_DEVERR_LENGTH : 0u;   // token ranges that overlap
  const int T = imin(all, p.entries);
  const int me = imin(lane, imax(T - 1, 0));
  int i = 0;                                      // the last sequence whose entries begin at most at me
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) {
    const int at = __shfl(off, imin(i + o, kWave - 1), kWave);
    i += ((i + o < p.n) & (at <= me)) ? o : 0;
  }
  KvEntry x{};
  x.row0 = (me - __shfl(off, i, kWave)) * R;
  plan_rows(p, x, i, __shfl(t0, i, kWave), __shfl(tk, i, kWave), __shfl(keys, i, kWave), 0, R);
  const int units = lane < T ? (x.tiles + kSegUnits) * p.nkv : 0;
  const int sum = wave_scan(units, lane), cum = sum - units, W = __shfl(sum, kWave - 1, kWave);
  // k_kv_few's waves take a share's tiles side by side: one request's shares have a tile a
  // wave, for fewer parts to join (4000 keys 21.4 -> 17.8 us, 1000 14.7 -> 13.1, 100 the
  // same); of several requests such shares reach over segments (8 of 500 keys 14 -> 16 us)
  const int least = R <= 16 && T == 1 ? 4 : kPlanMinShare;
  const int S = imax((W + shares - 1) / shares, least);
  const int f = (int)(((int64_t)sidx * S) < W ? sidx * S : W);
  const int f1 = (int)(((int64_t)sidx + 1) * S < W ? (sidx + 1) * S : W);
  const uint64_t before = __ballot((lane < T) & (cum <= f));
  const int e = before != 0 ? 63 - __builtin_clzll(before) : 0;
  const int seg = __shfl(x.tiles, e, kWave) + kSegUnits, in = f - __shfl(cum, e, kWave);
  const KvShare r{f, e, in / seg, in % seg - kSegUnits};
  ent[lane] = x;
  sh[0] = r.f;                                    // every lane the same
  sh[1] = r.e;
  sh[2] = r.kvh;
  sh[3] = r.j;
  sh[4] = f1;
  d.list.share[sidx] = r;
  if (blockIdx.x == 0) {                          // the list, for k_kv_join
    KvEntry* to = lane < T ? d.list.ent + lane : (KvEntry*)d.w.dump;
    *to = x;
    d.list.hdr[0] = W;
    d.list.hdr[1] = S;
    d.list.hdr[2] = T;
    if (__ballot(bad != 0) != 0) atomicOr(d.err, XP_DEVERR_LENGTH);
  }
}

// waves of a SIMD: two (256 registers each), or three where half the head leaves room
constexpr int kv_waves(int hd, int wr, int wk) { return hd == 64 && wr == 4 && wk == 1 ? 3 : 2; }

// WR x WK waves: wave (wr, wk) takes rows 32 wr .. + 31 of the tile and the wk-th
// part of each tile's keys, in blocks of 32.  S^T = K Q^T and O^T =
// V^T P^T on v_mfma_f32_32x32x16_bf16: a lane holds one query row (l % 32) in both,
// so the softmax's statistics are the lane's own but for one exchange with lane l ^
// 32, and the numerators go from the accumulators of S straight into the B operand
// (its k order is that of the keys 16 t + 4 (l / 32) + 0..3 and + 8, which the
// transposing reads of V follow).  Scores are kept in base 2.  A row's reference
// maximum moves only when a score exceeds it by more than 2^8, so most blocks
// rescale nothing.
// Numerators enter P V as PARTS bf16 parts, two (16 significant bits) or one (8).  One
// where more than 64 rows make the second part's products cost time: 64 blocks of 32 over
// 512 .. 16384 keys 487 us with one, 574 with two; prompts of 1 .. 8191 995 and 1252; a
// shared prefix of 8192 48 and 55.  The results' error is then 2.2e-3 of their rms in
// place of 1.65e-3, the bf16 output's own rounding.
// Over an 8-bit cache, whose values are exact in fp16, as one fp16 part of 11 bits: the
// row's reference lies 2^7 below its maximum, so that numerators reach 2^15 (with the
// 2^8 above), and those of 2^-21 of the greatest still have all 11 bits; the smaller
// ones are off by at most 2^-25, where the sum is 2^7 at least.  Error 1.67e-3, where one
// bf16 part had 2.2e-3 in 0 to 2% less time, two 1.66e-3 in 5 to 30% more.
// Over a 4-bit cache, whose values span more than fp16 does, two bf16 parts up to 32 rows and
// one above: memory bounds those calls no longer (32 blocks of 16 over 8192 keys 130 us with
// one part, 163 with two).  K lies in LDS as in memory and becomes an operand behind it, V is
// expanded on its way there: with both expanded, whose writes (64 bytes a cycle) and reads
// are four times as long, the same 155 and 175 us.
// Tiles wait in an LDS ring of NST stages filled by global_load_lds; the keys
// that no row of the tile sees are loaded as zeros, whatever lies there.
// Matrix pipe and vector pipe work side by side only if one wave's instructions
// alternate (two waves of a SIMD run in step, held by the tiles' barriers), and a
// product that follows the one it adds to waits for it.  So block n's numerators
// are formed between the products of block n + 1's scores and of block n - 1's P V,
// in turn.
// Bound by memory up to 128 rows (48 single tokens over 4096 keys 138 us, 5.8 TB/s; 32
// blocks of 16 over 8192 182 us, 5.9; 64 of 32 445 us, 4.9 TB/s and 620 TFLOP/s), by
// the loop's vector instructions beside the products above (4096 tokens x 8192 keys:
// 560 us, 980 TFLOP/s; head_dim 64, with as many exponentials to half the products,
// 410 us, 670).  A segment's beginning and end take about 10000 cycles, 2 to 3 tiles:
// four causal prompts of 4096 668 us, 822 TFLOP/s.
template <int HD, int FMT, int WR, int WK, int NST, int PARTS, bool OWN>
__global__ __launch_bounds__(WR* WK* kWave, kv_waves(HD, WR, WK)) void k_kv_attn(const KvDev d) {
  constexpr bool F8 = FMT == XP_E4M3, F4 = FMT == XP_MXFP4;
  using SH = KvRows<HD, F8>;
  constexpr int NW = WR * WK, R = 32 * WR, NB = 2 / WK, ND = HD / 32, NKS = HD / 16;
  constexpr int RB = SH::RB, CPR = SH::CPR, IPG = SH::IPG;
  static_assert(!F8 || PARTS == 1, "one fp16 part");
  // fp16 numerators reach up to 2^15 (see below), so that those of far smaller scores
  // keep their bits
  constexpr float kAbove = F8 ? 7.f : 0.f;
  constexpr int NG = 8 / NW;                      // groups of 16 rows that a wave loads
  static_assert(NG * NW == 8 && NB * WK == 2, "waves");
  constexpr int PER = NG * IPG;                   // loads of a wave for a stage
  static_assert(F4 || (NST - 1) * PER < 64, "vmcnt field");
  // 4 bits: K as in memory (codes, then exponents), V expanded to bf16
  static_assert(!F4 || NST == 3, "4-bit: the tile at work, the next, the one being stored");
  constexpr int kCodes = HD / 2, kExps = HD / 32; // bytes of a row
  constexpr int kK4 = kKvTile * (kCodes + kExps) / 16, kV0 = NST * kK4;   // K of a tile; V's beginning
  constexpr int kMerge = (HD / 2 + 2) * kWave;    // floats that a wave hands over
  constexpr int kRing = F4 ? kV0 + NST * SH::kHalf : NST * SH::kStage;
  static_assert(F4 || WK == 1 || WR * kMerge * 4 <= kRing * 16, "merge in LDS");
  constexpr int kMerges = WK == 2 ? WR * kMerge / 4 : 0;
  __shared__ __align__(256) u32x4 lds[kRing > kMerges ? kRing : kMerges];
  auto v_rows = [&](int stage, int r) { return lds + (F4 ? kV0 + stage * SH::kHalf : stage * SH::kStage + SH::kHalf) + r * CPR; };
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave % WR, wk = wave / WR;
  const int h = lane >> 5, li = lane & 31;
  // neighbouring shares on one XCD: they read the same sequence's keys
  const int sidx = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
  __shared__ KvEntry own_ent[OWN ? kOwnEntries : 1];
  __shared__ int32_t own_sh[8];
  if constexpr (OWN) {
    if (wave == 0) plan_own(d, R, gridDim.x, sidx, own_ent, own_sh);
    __syncthreads();
  }
  auto share = [&](int i) {
    if constexpr (OWN) return __builtin_amdgcn_readfirstlane(own_sh[i]);
    else return as_scalar(d.list.share + sidx)[i];
  };
  int f = share(0), e = share(1), kvh = share(2), j = share(3);
  const int f1 = share(4);
  if (f >= f1) return;                            // whole workgroup
  // The lane's byte addresses within 16 rows being loaded, and within a stage's K
  // and V: one register each.  The others follow by an exclusive or in the bits of
  // the chunk, load i (1 KB each): 1024 i + (lp ^ kLoadX i); K's 16-byte chunk 2 ks +
  // h: ka ^ 32 ks; block db of 32 dims of V: va ^ kVX db, its keys 8 further: ^ 32,
  // 8 rows on.
  constexpr int kLoadX = CPR == 16 ? 16 : 32, kVX = F8 ? 32 : 64;
  uint32_t lp, ka, va;
  {
    const int r = lane / CPR;
    lp = (uint32_t)(r * RB + 16 * ((lane % CPR) ^ SH::swz(r)));
    if constexpr (F4) ka = (uint32_t)(li * kCodes + 16 * (HD == 128 ? 2 * h ^ kv_swz4<HD>(li) : h ^ kv_swz4<HD>(li)));
    else ka = (uint32_t)(li * RB + 16 * (h ^ SH::swz(li)));
    const int rv = F8 ? 4 * h + ((lane >> 1) & 3) + 8 * ((lane >> 3) & 1) : 4 * h + ((lane & 15) >> 2);
    const int cv = F8 ? (lane >> 4) & 1 : 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    va = (uint32_t)(rv * RB + 16 * (cv ^ SH::swz(rv)) + 8 * (lane & 1));
  }
  const int P1 = (1 << d.logP) - 1;
  for (;;) {
  int en[kKvEntryInts];
#pragma unroll
  for (int i = 0; i < kKvEntryInts; ++i) {
    if constexpr (OWN) en[i] = __builtin_amdgcn_readfirstlane(reinterpret_cast<const int32_t*>(own_ent + e)[i]);
    else en[i] = as_scalar(d.list.ent + e)[i];
  }
  const int tok0 = en[0], row0 = en[1], nrows = en[2], seq = en[3], p0 = en[4], prefix = en[5];
  const int kfloor = en[6], kceil = en[7], ks_ = en[8], klo = en[9], khi = en[10], tiles = en[11];
  const int a0 = en[12], n1 = en[13], b0 = en[14];
  // the part's tiles [j, j + nj); its first kSegUnits units are none
  const int left = f1 - f + imin(j, 0);           // units of the share from tile max(j, 0) on
  f += tiles - j;                                 // the segment's end
  j = imax(j, 0);
  const int nj = imin(tiles - j, left);
  if (nj <= 0) return;                            // whole workgroup: the share ends before a tile
  const bool whole = nj == tiles;
  auto tile_key = [&](int t) { return kKvTile * (t < n1 ? a0 + t : b0 + t - n1); };

  // ---- the wave's query rows (B operand): row li of its 32 ----
  const bool live = 32 * wr < nrows;              // wave-uniform
  const int rr = 32 * wr + li;
  const bool rv = rr < nrows;
  u32x4 qf[NKS];
  KvSees sees;
  {
    const int row = row0 + (rv ? rr : 0), tk = row / d.grp;
    const int64_t tok = tok0 + tk;
    const uint16_t* qs = d.q + tok * d.q_ld + (int64_t)(kvh * d.grp + (row - tk * d.grp)) * HD;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks)
      qf[ks] = ld16(qs + (F8 ? 32 * (ks >> 1) + 16 * h + 8 * (ks & 1)
                             : (F4 ? HD / 2 * h + 8 * ks : 16 * ks + 8 * h)));
    const int p = prefix ? d.w.pos[tok] : p0 + tk;
    const int hi = rv ? (d.causal ? imin(p + 1, kceil) : kceil) : kfloor;
    const int lo = d.window > 0 ? imax(p - d.window + 1, kfloor) : kfloor;
    sees = KvSees{lo, kfloor, (uint32_t)imax(hi - lo, 0),
                  d.window > 0 ? (uint32_t)imax(imin(d.sinks, hi) - kfloor, 0) : 0u};
  }
  // keys that every row of the wave sees: [kfloor or wlo, whi), and [kfloor, wsink);
  // rows of several sequences: that every one of the group's does
  const int pmin = p0 + (prefix ? 0 : (row0 + 32 * wr) / d.grp);
  const int pmax = prefix ? en[15] : p0 + (row0 + imin(32 * wr + 31, nrows - 1)) / d.grp;
  const int whi = d.causal ? imin(pmin + 1, kceil) : kceil;
  const int wlo = d.window > 0 ? imax(pmax - d.window + 1, kfloor) : kfloor;
  const int wsink = d.window > 0 ? d.sinks : 0;
  const float scale2 = d.scale2 * (F8 && d.k_scale != nullptr ? d.k_scale[kvh] : 1.f);

  // ---- loads ----
  const scalar_i32 tb = as_scalar(d.table + (int64_t)seq * d.table_ld);
  // the first page's rows of this KV head, and the bytes from page to page
  constexpr int RBM = kv_row_bytes(FMT, HD);      // bytes of a row in memory
  const int64_t head0 = ((int64_t)kvh << d.logP) * RBM;
  const char* heads = (wave < NW / 2 ? d.kc : d.vc) + head0;
  const uint32_t page_bytes = (uint32_t)(d.nkv * RBM) << d.logP;
  const int kin = imax(klo, kfloor);              // from here to khi, or to ks_, some row sees all
  uint32_t bad = 0;                               // a page outside the cache was asked for
  // 4 bits: a lane's units of a tile, 16 or 8 bytes of codes, 16 or 8 rows of a wave each
  constexpr int kUnit = HD == 128 && NW <= 4 ? 16 : 8, kUnits = kKvTile * kCodes / (NW * kWave * kUnit);
  constexpr int kUPR = kCodes / kUnit, kURows = kWave / kUPR;   // units of a row, rows of a wave
  static_assert(!F4 || (kUnits >= 1 && kURows <= 16), "units");
  auto row4 = [&](int u) { return (u * NW + wave) * kURows; };
  constexpr int NPG = F4 ? kUnits : NG;
  auto pages = [&](int t, int (&pg)[NPG]) {       // page ids of the wave's rows of tile t
#pragma unroll
    for (int g = 0; g < NPG; ++g)
      pg[g] = tb[imin((tile_key(t) + (F4 ? row4(g) : 16 * ((wave * NG + g) & 3))) >> d.logP, d.cols - 1)];
  };
  // tile t to a slot; a segment's first tiles by the general way alone (a tile all of
  // whose keys some row sees needs no test of its keys, but costs a copy of the code)
  auto issue = [&](auto first, int t, int slot, const int (&pg)[NPG]) __attribute__((always_inline)) {
    const int k0 = tile_key(t);
    const bool inner = !decltype(first)::value &&
        (((k0 >= kin) & (k0 + kKvTile <= khi)) | ((k0 >= kfloor) & (k0 + kKvTile <= ks_)));
    u32x4* stage = lds + slot * SH::kStage + wave * (NG * 16 * CPR);   // its rows of K, then V
    if (inner) {
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const uint32_t page = (uint32_t)pg[g];
        const bool ok = page < (uint32_t)d.n_pages;
        bad |= ok ? 0u : XP_DEVERR_PAGE;
        const char* base = heads + (uint64_t)(ok ? page : 0u) * page_bytes +
                           ((k0 + 16 * ((wave * NG + g) & 3)) & P1) * RB;
        // a load's offset counts for both addresses
        if constexpr (R <= 64) kv_dma_nt(base, lp, kLoadX, IPG, stage + 16 * g * CPR);
        else kv_dma(base, lp, kLoadX, IPG, stage + 16 * g * CPR);
      }
    } else {
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const int g0 = k0 + 16 * ((wave * NG + g) & 3);
        const uint32_t page = (uint32_t)pg[g];
        const bool ok = page < (uint32_t)d.n_pages;
        const int from = imax(g0, kfloor), to = imin(g0 + 16, khi);
        bad |= (!ok & (from < to) & ((to > klo) | (from < ks_))) ? XP_DEVERR_PAGE : 0u;
        const char* base = heads + (uint64_t)(ok ? page : 0u) * page_bytes + (g0 & P1) * RB;
#pragma unroll
        for (int i = 0; i < IPG; ++i) {
          const int key = g0 + i * (kWave / CPR) + lane / CPR;
          const bool any = (key >= kfloor) & (key < khi) & ((key >= klo) | (key < ks_));
          const uint64_t at = (uint64_t)(uintptr_t)base + 1024 * i + (lp ^ (kLoadX * i));
          const uint64_t none = (uint64_t)(uintptr_t)d.w.zero + 16 * (lane & 15);
          lds_dma16((const void*)(uintptr_t)(any ? at : none), stage + 16 * g * CPR + 64 * i);
        }
      }
    }
  };
  // The scores of a block of keys are formed while the block before it goes through
  // its softmax, so K is needed a block ahead of V.  With one block a tile (WK = 2)
  // K of tile t is done with when iteration t begins, and the waves that load K run
  // one tile ahead: before it they have brought tiles up to t + NST - 1, else, as the
  // waves that load V, up to t + NST - 2.  Tile i lies in stage i % NST.
  const int is_k = wave < NW / 2 ? 1 : 0, ahead = NB == 1 ? is_k : 0;
  // loads still under way when iteration t has what it needs: K of tile t + 1, V of t
  constexpr int kWaitV = (NST - 2) * PER, kWaitK = (NB == 1 ? NST - 2 : NST - 3) * PER;
  static_assert(F4 || kWaitK >= 0, "stages");
  // A 4-bit cache's tiles come through registers: K's codes and exponents go to LDS as
  // they are and become bf16 operands behind it, V is expanded to bf16 (both exactly) on
  // its way there.  In iteration t every wave stores its part of tile t + 2 and has tile
  // t + 3 under way.  Keys that no row sees come like the others: their scores are masked
  // and their V is looked through for NaN, as where only some row does not see them.
  struct Held {
    u32x4 k[kUnits], v[kUnits];
    uint32_t ke[kUnits], ve[kUnits];
  };
  const int ur = lane / kUPR, uc = lane % kUPR;   // the lane's row and unit of a wave's
  const int ub = uc * kUnit / 16;                 // its block of 32
  const uint32_t xo = ur * kCodes + kUnit * uc, eo = ur * kExps + ub;
  auto fetch = [&](int t, const int (&pg)[NPG], Held& to) __attribute__((always_inline)) {
    const int k0 = tile_key(t);
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int g0 = k0 + row4(u), r = g0 & P1;
      uint32_t page = (uint32_t)pg[u];
      if (page >= (uint32_t)d.n_pages) {          // wave-uniform
        const int from = imax(g0, kfloor), upto = imin(g0 + kURows, khi);
        bad |= ((from < upto) & ((upto > klo) | (from < ks_))) ? XP_DEVERR_PAGE : 0u;
        page = 0;
      }
      // wave-uniform addresses: scalar registers and the lane's bytes
      const uint64_t at = (uint64_t)head0 + (uint64_t)page * page_bytes + (uint32_t)(r * kCodes);
      const uint64_t ex = at + ((uint32_t)kCodes << d.logP) - (uint32_t)(r * (kCodes - kExps));
      uint64_t kx = (uint64_t)(uintptr_t)d.kc + at, vx = (uint64_t)(uintptr_t)d.vc + at;
      uint64_t ke = (uint64_t)(uintptr_t)d.kc + ex, ve = (uint64_t)(uintptr_t)d.vc + ex;
      asm volatile("" : "+s"(kx), "+s"(vx), "+s"(ke), "+s"(ve));
      if constexpr (kUnit == 16) {
        to.k[u] = ld16((const char*)(uintptr_t)kx + xo);
        to.v[u] = ld16((const char*)(uintptr_t)vx + xo);
      } else {
        const uint2 y = *reinterpret_cast<const uint2*>((const char*)(uintptr_t)kx + xo);
        const uint2 z = *reinterpret_cast<const uint2*>((const char*)(uintptr_t)vx + xo);
        to.k[u] = u32x4{y.x, y.y, 0u, 0u};
        to.v[u] = u32x4{z.x, z.y, 0u, 0u};
      }
      to.ke[u] = *reinterpret_cast<const uint8_t*>((const char*)(uintptr_t)ke + eo);
      to.ve[u] = *reinterpret_cast<const uint8_t*>((const char*)(uintptr_t)ve + eo);
    }
  };
  auto put = [&](int slot, const Held& from) __attribute__((always_inline)) {
    char* kst = reinterpret_cast<char*>(lds + slot * kK4);
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int r = row4(u) + ur;
      const u32x4 x = from.k[u];
      if constexpr (kUnit == 16)
        *reinterpret_cast<u32x4*>(kst + r * kCodes + 16 * (uc ^ kv_swz4<HD>(r))) = x;
      else
        *reinterpret_cast<uint2*>(kst + r * kCodes + 16 * ((uc >> 1) ^ kv_swz4<HD>(r)) + 8 * (uc & 1)) = uint2{x[0], x[1]};
      // exponents above 252 are NaN
      kst[kKvTile * kCodes + r * kExps + ub] = (char)(from.ke[u] > 252u ? 255u : from.ke[u]);
      const float s = __uint_as_float((from.ve[u] > 252u ? 255u : from.ve[u]) << 23);
      u32x4* row = v_rows(slot, r);
#pragma unroll
      for (int i = 0; i < kUnit / 4; ++i)
        row[(kUnit / 4 * uc + i) ^ SH::swz(r)] = f4_bf16x8(from.v[u][i], s);
    }
  };
  Held held;
  constexpr int NFST = F4 ? 2 : NST;              // tiles whose pages are asked for at once
  int pg[NPG], pg0[NFST][NPG];
#pragma unroll
  for (int t = 0; t < NFST; ++t) pages(j + imin(t, nj - 1), pg0[t]);
  pages(j + imin(F4 ? 2 : NST - 1 + ahead, nj - 1), pg);
  // The query rows are waited for here: with loads to LDS under way the compiler waits
  // for all of them before it uses a register that was loaded.
#pragma unroll
  for (int ks = 0; ks < NKS; ++ks) asm volatile("" : "+v"(qf[ks]));
  if constexpr (F4) {
    Held first;
    fetch(j, pg0[0], first);
    fetch(j + imin(1, nj - 1), pg0[1], held);
    put(0, first);
    put(1, held);
    fetch(j + imin(2, nj - 1), pg, held);
    pages(j + imin(3, nj - 1), pg);
  } else {
#pragma unroll
    for (int t = 0; t < NST; ++t)
      if (t < nj && t < NST - 1 + ahead) issue(std::true_type{}, j + t, t, pg0[t]);   // whole wave
  }

  float m_run = -INFINITY, l_run = 0.f;           // the row's; l of this half's keys
  floatx16 o[ND];
#pragma unroll
  for (int db = 0; db < ND; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;

  // every row of the wave sees every key of the block that begins at k0
  auto all_seen = [&](int k0) {
    return k0 >= kfloor && k0 + 32 <= whi && (k0 >= wlo || k0 + 32 <= wsink);
  };
  // K operands of the block at row r of a stage
  u32x4 kf[NKS];
  float kscale[2] = {};
  auto k_read = [&](int stage, int r) __attribute__((always_inline)) {
    if constexpr (F4) {
      uint32_t kx = ka + lds_byte(lds + stage * kK4) + r * kCodes;
      uint32_t ex = lds_byte(lds + stage * kK4) + kKvTile * kCodes + (r + li) * kExps;
      asm volatile("" : "+v"(kx), "+v"(ex));
      kf[0] = *(const lds_u32x4*)(uintptr_t)kx;
      if constexpr (HD == 128) {
        kf[1] = *(const lds_u32x4*)(uintptr_t)(kx ^ 16);
        const uint32_t y = *(const __attribute__((address_space(3))) uint32_t*)(uintptr_t)ex >> (16 * h);
        kscale[0] = __uint_as_float(y << 23 & 0x7f800000u);
        kscale[1] = __uint_as_float(y << 15 & 0x7f800000u);
      } else {
        const uint32_t y = *(const __attribute__((address_space(3))) uint16_t*)(uintptr_t)ex >> (8 * h);
        kscale[0] = __uint_as_float(y << 23 & 0x7f800000u);
      }
      __builtin_amdgcn_sched_barrier(0);
      return;
    }
    uint32_t kx = ka + lds_byte(lds + stage * SH::kStage + r * CPR);
    asm volatile("" : "+v"(kx));                  // opaque: no address is kept for the next block
#pragma unroll
    for (int i = 0; i < (F8 ? NKS / 2 : NKS); ++i)
      kf[F8 ? 2 * i : i] = *(const lds_u32x4*)(uintptr_t)(kx ^ (32 * i));
    __builtin_amdgcn_sched_barrier(0);
  };
  auto k_operand = [&](int i) {                   // in order: an even i leaves i + 1 behind
    if constexpr (F8) {
      if (i % 2 == 0) {
        const u32x4 x = kf[i];
        kf[i + 1] = f8_bf16x8(x.z, x.w);
        return f8_bf16x8(x.x, x.y);
      }
    }
    if constexpr (F4) return f4_bf16x8(kf[i / 4][i % 4], kscale[i / 4]);
    else return kf[i];
  };
  // V operands of a block, and the numerators (as bf16 parts) of this one and the next
  u32x4 v[2][ND], ph[2][2], pl[2][2];
  auto v_read = [&](int stage, int r) __attribute__((always_inline)) {
    uint32_t vx = va + lds_byte(v_rows(stage, r));
    asm volatile("" : "+v"(vx));
    uint32_t xa[ND], xb[ND];
#pragma unroll
    for (int db = 0; db < ND; ++db) {
      xa[db] = vx ^ (kVX * db);
      xb[db] = xa[db] ^ 32;
    }
    lds_v<ND, F8, 0, RB>(xa, xb, v);
  };
  auto v_product = [&](int x, const u32x4 (&a)[2], const u32x4 (&b)[2])
      __attribute__((always_inline)) {
    const int u = x / ND, db = x % ND;
    if constexpr (PARTS == 2) o[db] = mma32(v[u][db], b[u], o[db]);
    o[db] = mma32_pv<F8>(v[u][db], a[u], o[db]);
  };
  // infinities or NaN among the block's V
  auto odd_values = [&](int stage, int r) __attribute__((always_inline)) {
    const u32x4* Vs = v_rows(stage, r);
    constexpr int N = 32 * CPR / kWave, U = N < 4 ? N : 4;   // reads of a lane, at a time
    KvOdd<F8> odd;
#pragma unroll 1
    for (int i = 0; i < N; i += U) {
      u32x4 x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = Vs[kWave * (i + u) + lane];
#pragma unroll
      for (int u = 0; u < U; ++u) odd.add(x[u]);
    }
    return __ballot(odd.any()) != 0;
  };
  // Rows must not meet the infinities and NaN of keys that they do not see (0 times
  // one is no number): those values leave the operands, and the rows with a
  // numerator for one get it from a product with ones in its places.  Only blocks on
  // the border of some row's view come here, and only if they hold such values.
  auto take_odd = [&](const u32x4 (&a)[2]) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int db = 0; db < ND; ++db) {
#pragma unroll 1
        for (int c = 0; c < 3; ++c) {             // inf, -inf, NaN
          u32x4 one;
#pragma unroll
          for (int w = 0; w < 4; ++w)
            one[w] = ones_of<F8>(c, v[u][db][w] & 0xffffu) | ones_of<F8>(c, v[u][db][w] >> 16) << 16;
          const float val = c == 0 ? INFINITY : (c == 1 ? -INFINITY : NAN);
          floatx16 y;
#pragma unroll
          for (int i = 0; i < 16; ++i) y[i] = 0.f;
          y = mma32_pv<F8>(one, a[u], y);
#pragma unroll
          for (int i = 0; i < 16; ++i) o[db][i] += y[i] > 0.f ? val : 0.f;
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) v[u][db][w] &= ~nonfinite_mask<F8>(v[u][db][w]);
      }
  };
  constexpr int EP = 16 / NKS;                    // numerators beside a product of S
  // a pair of them, and l, which sums them in fp32
  auto pack = [&](const floatx16& s, int x, u32x4 (&a)[2], u32x4 (&b)[2])
      __attribute__((always_inline)) {
    const int u = x / 8, i = x % 8 / 2;
    const float e0 = s[x], e1 = s[x + 1];
    l_run += e0;
    l_run += e1;
    uint32_t y = pk_p<F8>(e0, e1);
    asm volatile("" : "+v"(y), "+v"(l_run));      // here, not where it is used
    a[u][i] = y;
    if constexpr (PARTS == 2) {
      y = pk_bf16(e0 - __uint_as_float(y << 16), e1 - __uint_as_float(y & 0xFFFF0000u));
      asm volatile("" : "+v"(y));
      b[u][i] = y;
    }
  };
  // Block n at row r of a stage (first key k0, scores in s), numerators to set PAR;
  // nx takes the scores of block n + 1 (at row rn of stage sn; where there is none,
  // of whatever lies there).
  auto block = [&](auto par, int k0, int stage, int r, floatx16& s, int sn, int rn, floatx16& nx)
      __attribute__((always_inline)) {
    constexpr int PAR = decltype(par)::value;
    k_read(sn, rn);
    bool odd = false;
    if (!all_seen(k0)) {
      uint32_t a = (uint32_t)(k0 + 4 * h - sees.lo), b = (uint32_t)(k0 + 4 * h - sees.floor);
      asm volatile("" : "+v"(a), "+v"(b));        // opaque: no key is kept in a register
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t c = 8 * (i / 4) + i % 4;
        s[i] = ((a + c < sees.n) | (b + c < sees.s)) ? s[i] : -INFINITY;
      }
      odd = odd_values(stage, r);
    }
    constexpr float kLazy = 8.f;
    float mt = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mt = fmaxf(mt, s[i]);
    mt = fmax_xor32(mt) * scale2 - kAbove;
    const bool grow = __ballot(mt > m_run + kLazy) != 0;   // wave-uniform
    float alpha = 1.f;
    if (grow) {
      const float mref = fmaxf(m_run, mt);
      alpha = __builtin_amdgcn_exp2f(m_run - (mref == -INFINITY ? 0.f : mref));
      l_run *= alpha;
      m_run = mref;
    }
    // with no visible key yet (m = -inf) every exponent below is -inf: 0
    const float ref = m_run == -INFINITY ? 0.f : m_run;
    floatx16 c0;
#pragma unroll
    for (int y = 0; y < 16; ++y) c0[y] = 0.f;
    // Beside each product of S: EP numerators, the packing of the EP before them, and
    // the products of P V of block n - 1 (relative to the reference before it grew).
    // The order is fixed: the compiler's own is all products, then everything else.
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < NKS; ++i) {
#pragma unroll
      for (int x = EP * i; x < EP * (i + 1); ++x) {
        float y = __builtin_amdgcn_exp2f(fmaf(s[x], scale2, -ref));
        asm volatile("" : "+v"(y));
        s[x] = y;
      }
      if (i > 0) {
#pragma unroll
        for (int x = EP * (i - 1); x < EP * i; x += 2) pack(s, x, ph[PAR], pl[PAR]);
      }
      nx = mma32(k_operand(i), qf[i], i == 0 ? c0 : nx);
#pragma unroll
      for (int x = 2 * ND * i / NKS; x < 2 * ND * (i + 1) / NKS; ++x)
        v_product(x, ph[1 - PAR], pl[1 - PAR]);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int x = 16 - EP; x < 16; x += 2) pack(s, x, ph[PAR], pl[PAR]);
    if (grow) {
#pragma unroll
      for (int db = 0; db < ND; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
    }
    uint32_t some = 0;                            // numerators above 0; fp16 rounds small ones to it
    if constexpr (F8) {
      if (__builtin_expect(odd, 0)) {
#pragma unroll
        for (int x = 0; x < 16; ++x) some |= s[x] > 0.f ? 1u << x : 0u;
      }
    }
    v_read(stage, r);
    if (__builtin_expect(odd, 0)) {
      if constexpr (F8) {
        u32x4 a[2];
#pragma unroll
        for (int x = 0; x < 16; x += 2)
          a[x / 8][x % 8 / 2] = ((some >> x) & 1u) * 0x3c00u | ((some >> (x + 1)) & 1u) * 0x3c000000u;
        take_odd(a);
      } else {
        take_odd(ph[PAR]);
      }
    }
  };
  auto after = [](int stage) { return stage + 1 == NST ? 0 : stage + 1; };
  // The beginning of iteration t: K of tile t + 1 and V of tile t landed (every
  // wave's loads), and every wave is done with what the next loads replace.
  auto begin = [&](int t, int stage) __attribute__((always_inline)) {
    if constexpr (F4) {
      lds_barrier();
      if (t + 2 < nj) put(stage == 0 ? NST - 1 : stage - 1, held);
      if (t + 3 < nj) {
        fetch(j + t + 3, pg, held);
        pages(j + imin(t + 4, nj - 1), pg);
      }
      return;
    }
    asm volatile("" ::: "memory");
    if (t + NST - 2 + ahead < nj) {
      if (is_k) __builtin_amdgcn_s_waitcnt(0x0070 | (kWaitK & 15) | ((kWaitK >> 4) << 14));
      else __builtin_amdgcn_s_waitcnt(0x0070 | (kWaitV & 15) | ((kWaitV >> 4) << 14));
    } else {
      __builtin_amdgcn_s_waitcnt(0x0070);
    }
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (t + NST - 1 + ahead < nj) {
      issue(std::false_type{}, j + t + NST - 1 + ahead, ahead ? stage : (stage == 0 ? NST - 1 : stage - 1), pg);
      pages(j + imin(t + NST + ahead, nj - 1), pg);
    }
  };
  // K of the first tile landed
  if constexpr (F4) {
    lds_barrier();
  } else {
    asm volatile("" ::: "memory");
    if (is_k) {
      constexpr int kFirst = (NST - 2 + (NB == 1 ? 1 : 0)) * PER;
      if (NST - 1 + ahead <= nj) __builtin_amdgcn_s_waitcnt(0x0070 | (kFirst & 15) | ((kFirst >> 4) << 14));
      else __builtin_amdgcn_s_waitcnt(0x0070);
    }
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  }
  floatx16 sa, sb;
  constexpr std::integral_constant<int, 0> even{};
  constexpr std::integral_constant<int, 1> uneven{};
  if (live) {                                     // the first block's scores
    k_read(0, 32 * wk);
    floatx16 c0;
#pragma unroll
    for (int y = 0; y < 16; ++y) c0[y] = 0.f;
#pragma unroll
    for (int i = 0; i < NKS; ++i) sa = mma32(k_operand(i), qf[i], i == 0 ? c0 : sa);
  }
#pragma unroll
  for (int u = 0; u < 2; ++u) {                   // and nothing for the block before it
    ph[1][u] = u32x4{0u, 0u, 0u, 0u};
    if constexpr (PARTS == 2) pl[1][u] = ph[1][u];
#pragma unroll
    for (int db = 0; db < ND; ++db) v[u][db] = u32x4{0u, 0u, 0u, 0u};
  }
  int stage = 0;
  bool last_even = false;                         // the last block's numerators are set 0
#pragma unroll 1
  for (int t = 0; t < nj; ++t) {
    begin(t, stage);
    int k0 = tile_key(j + t) + 32 * wk;
    if constexpr (NB == 2) {
      if (live) {
        block(even, k0, stage, 0, sa, stage, 32, sb);
        block(uneven, k0 + 32, stage, 32, sb, after(stage), 0, sa);
      }
    } else {                                      // two tiles: the scores change places
      if (live) block(even, k0, stage, 32 * wk, sa, after(stage), 32 * wk, sb);
      stage = after(stage);
      if (++t == nj) {                            // whole workgroup
        last_even = true;
        break;
      }
      begin(t, stage);
      k0 = tile_key(j + t) + 32 * wk;
      if (live) block(uneven, k0, stage, 32 * wk, sb, after(stage), 32 * wk, sa);
    }
    stage = after(stage);
  }
  if (live) {                                     // P V of the last block
    if (NB == 1 && last_even) {
#pragma unroll
      for (int x = 0; x < 2 * ND; ++x) v_product(x, ph[0], pl[0]);
    } else {
#pragma unroll
      for (int x = 0; x < 2 * ND; ++x) v_product(x, ph[1], pl[1]);
    }
  }
  l_run = fsum_xor32(l_run);
  if constexpr (WK == 2) {
    // the second key half hands (m, l, O) to the first through the ring's LDS:
    // O = 2^(m0 - M) O0 + 2^(m1 - M) O1, l likewise, M = max(m0, m1)
    __syncthreads();                              // every wave's reads of the ring done
    float* mg = reinterpret_cast<float*>(lds) + wr * kMerge + lane;
    floatx4* mo = reinterpret_cast<floatx4*>(mg - lane + 2 * kWave) + lane;
    if (wk == 1) {
#pragma unroll
      for (int db = 0; db < ND; ++db)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          mo[(4 * db + i / 4) * kWave] = floatx4{o[db][i], o[db][i + 1], o[db][i + 2], o[db][i + 3]};
      mg[0] = m_run;
      mg[kWave] = l_run;
    }
    __syncthreads();
    if (wk == 0) {
      const float m1 = mg[0], l1 = mg[kWave];
      const float M = fmaxf(m_run, m1), Ms = M == -INFINITY ? 0.f : M;
      const float w0 = __builtin_amdgcn_exp2f(m_run - Ms), w1 = __builtin_amdgcn_exp2f(m1 - Ms);
      m_run = M;
      l_run = w0 * l_run + w1 * l1;
#pragma unroll
      for (int db = 0; db < ND; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] = w0 * o[db][i] + w1 * mo[(4 * db + i / 4) * kWave][i % 4];
    }
  }
  // ---- results: the rows themselves, or what k_kv_join(_rows) adds up ----
  // Lanes without a row write to a row that no one reads: with branches of single
  // lanes here this compiler brought registers back under the narrower mask.
  if (wk == 0) {
    const int row = row0 + rr, tk = row / d.grp;
    const int64_t tok = tok0 + tk;
    const int head = kvh * d.grp + (row - tk * d.grp);
    if (whole && d.groups == 0) {
      const float inv = l_run == 0.f
          ? (sees_some(d, p0 + tk, kceil) ? NAN : 0.f)
          : (F8 && d.v_scale != nullptr ? d.v_scale[kvh] : 1.f) / l_run;
      uint16_t* op = (rv ? d.out + tok * d.out_ld + (int64_t)head * HD : (uint16_t*)d.w.dump) + 8 * h;
#pragma unroll
      for (int db = 0; db < ND; ++db)
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          const floatx16& y = o[db];
          uint32_t w[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) w[k] = pk_bf16(y[4 * i + 2 * k] * inv, y[4 * i + 2 * k + 1] * inv);
          // 16 bytes a lane: dims 8 i + 0..7 here, 8 (i + 1) + 0..7 in lane + 32
          swap_halves(w[0], w[2]);
          swap_halves(w[1], w[3]);
          *reinterpret_cast<u32x4*>(op + 32 * db + 8 * i) = u32x4{w[0], w[1], w[2], w[3]};
        }
      if (d.lse != nullptr) {
        const float y = l_run == 0.f
            ? -INFINITY : (m_run + __builtin_amdgcn_logf(l_run)) * 0.69314718055994531f;
        *(rv ? d.lse + tok * d.nh + head : (float*)d.w.dump) = y;
      }
    } else {
      const int64_t prow = whole ? d.row0 + ((int64_t)prefix * d.total_q + tok) * d.nh + head
                                 : d.part0 + (int64_t)(2 * sidx + (j == 0 ? 1 : 0)) * R + rr;
      float* op = (rv ? d.w.part + prow * HD : (float*)d.w.dump) + 4 * h;
#pragma unroll
      for (int db = 0; db < ND; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const floatx16& y = o[db];
          *reinterpret_cast<floatx4*>(op + 32 * db + 8 * i) =
              floatx4{y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]};
        }
      *reinterpret_cast<float2*>(rv ? d.w.ml + 2 * prow : (float*)d.w.dump) =
          float2{m_run, l_run};
    }
  }
  if (bad != 0) atomicOr(d.err, bad);
  // ---- on to the next segment of the share ----
  if (f >= f1) return;                            // whole workgroup
  j = -kSegUnits;
  if (++kvh == d.nkv) {
    kvh = 0;
    ++e;
  }
  __syncthreads();                                // the ring is read, the merge done
  }
}

// ---------------------------------------------------------------------------
// Few rows over a 4-bit cache: up to 8 or 16 of a tile (single tokens, short blocks).
// A cache of 68 bytes a key (head_dim 128) leaves a third of the time a key that 8 bits
// leave, so nothing may be done for rows that are not there, and little a key:
//
// * S^T = K Q^T on v_mfma_scale_f32_16x16x128_f8f6f4: its fp4 operand is a lane's 32
//   codes of one block as they lie in memory, with the block's power of two, so K goes
//   from the load into the product.  The queries are its e4m3 operand, in two parts: a
//   row's largest element lies in [2^7, 2^8), the first part takes 4 bits, the second the
//   next 4: all that bf16 has, for elements down to 2^-14 of the largest.
// * Where a row of the tile has smaller ones (beside a key whose block for the largest is
//   as small, they are the score), K is expanded to bf16 in registers and the queries come
//   as they are, through LDS: 6% of such tiles of 4 normal rows, which take a tenth longer
//   (a third fp8 part instead: registers that the loads need, 16 rows 2 to 5% slower).
// * V's power of two differs from key to key, the dimension that P V sums over, where
//   the instruction takes one for 32: V is expanded to bf16 (exactly) on its way into
//   the wave's LDS and comes back by transposing reads.
// * O^T = V^T P^T on v_mfma_f32_16x16x32_bf16, P in two bf16 parts.  A lane has one
//   column of S and of O; its numerators are the next product's operand.
// * Up to 8 rows: a column is a row and a part, so that one product has the first two
//   parts of Q, and one both parts of P (its 16 x 16 take 30 cycles whatever they hold).
//
// NW waves take a share's tiles of 64 keys in turn, each with its own statistics and
// no barrier, the next tile on its way while one is worked on; at a segment's end their
// results are added through LDS.  A wave issues an instruction in 8 cycles at best, a SIMD
// in 4.3: three waves of 168 registers (two, each with two tiles under way, 107 to 118 us
// where three take 94; 1 or 2 waves a workgroup the same, 3, 6, 8 and 12 take 110 to 150).
// 48 single tokens over 512 .. 16384 keys, 439 MB: 91 to 95 us, 4.6 to 4.8 TB/s; the 32-row
// engine above took 225.  Bound by memory, by the vector instructions (V's expansion and
// its way through LDS, exponentials) and by 384 segments' beginnings and ends.
// ---------------------------------------------------------------------------
typedef int intx8 __attribute__((ext_vector_type(8)));
constexpr int kFewRows = 16;         // the larger row tile (kv_least)
constexpr int kFewSimd = 3;          // waves of a SIMD

__device__ __forceinline__ floatx4 mma16_bf16(u32x4 a, u32x4 b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// 32 e2m1 codes of A times 2^(ea - 127), 32 e4m3 values of B times 2^(eb - 127)
__device__ __forceinline__ floatx4 mma16_f4f8(u32x4 a, intx8 b, floatx4 c, int ea, int eb) {
  const intx8 x{(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, b, c, 4, 0, 0, ea, 0, eb);
}
// 4 keys of the lane's dim: 16 lanes read 4 rows of 16 dims
__device__ __forceinline__ uint2 lds_tr16(uint32_t at) {
  typedef short short4v __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) short4v lds_short4;
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(uintptr_t)at));
}

// of the column 8 further in the lane's 16
__device__ __forceinline__ float other_half(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), 0x128, 0xF, 0xF, true));
}

template <int HD, int R, int NW, bool OWN>
__global__ __launch_bounds__(NW* kWave, kFewSimd) void k_kv_few(const KvDev d) {
  // rows of V in LDS, 16 bytes apart from the next: neither the 16-byte writes of 16 rows
  // nor the transposing reads meet in a bank, and every address is one register and an
  // offset
  constexpr int NT = HD / 16, RB = 2 * HD + 16;
  constexpr bool HALF = R == 8;                   // a column is a row and a part
  constexpr int QM = HALF || HD == 64 ? 1 : 2;    // products of the queries' two parts
  constexpr int kDeepest = 14;                    // binades that the parts hold
  constexpr int RBM = kv_row_bytes(XP_MXFP4, HD);
  constexpr int kMerge = (4 * NT + 2) * kWave;    // floats that a wave hands over
  constexpr int kRing = kMerge * 4 > 32 * RB ? kMerge * 4 : 32 * RB;   // its LDS: V of half a tile
  static_assert(kRing % 256 == 0, "a wave's LDS");
  __shared__ __align__(256) char lds[NW * kRing];
  // the queries, where parts do not hold them: 16 bytes behind every row of V, where that is
  // enough (4 KB of their own cost 2% of a call's time)
  constexpr bool kBehind = R * HD / 8 <= 32 * NW;
  __shared__ __align__(16) u32x4 own_q[kBehind ? 1 : R * HD / 8];
  __shared__ KvEntry own_ent[OWN ? kOwnEntries : 1];
  __shared__ int32_t own_sh[8];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int li = lane & 15, g = lane >> 4, ri = li & (R - 1);   // column, its keys; its row
  const int sidx = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
  if constexpr (OWN) {
    if (wave == 0) plan_own(d, R, gridDim.x, sidx, own_ent, own_sh);
    __syncthreads();
  }
  auto share = [&](int i) {
    if constexpr (OWN) return __builtin_amdgcn_readfirstlane(own_sh[i]);
    else return as_scalar(d.list.share + sidx)[i];
  };
  int f = share(0), e = share(1), kvh = share(2), j = share(3);
  const int f1 = share(4);
  if (f >= f1) return;                            // whole workgroup
  // the lane's bytes within 16 rows: K a block of 32 codes (head_dim 64: the lanes of the
  // second half have them again, for the second part of Q), V HD / 4 codes
  const uint32_t ko = li * (HD / 2) + 16 * (HD == 128 ? g : g & 1);
  const uint32_t keo = li * (HD / 32) + (HD == 128 ? g : g & 1);
  const uint32_t vo = li * (HD / 2) + (HD / 8) * g;
  const uint32_t veo = li * (HD / 32) + (HD == 128 ? g : g >> 1);
  char* ring = lds + wave * kRing;
  // V into LDS: row 16 n + li, 16 bytes HD / 32 g + i; back: rows 4 g + li / 4, dims
  // 16 u + 4 (li % 4) + 0..3 of the row, which make the lane's dim 16 u + li
  const uint32_t vw = lds_byte(ring) + li * RB + HD / 2 * g;
  const uint32_t vr = lds_byte(ring) + (4 * g + (li >> 2)) * RB + 8 * (li & 3);
  const int P1 = (1 << d.logP) - 1;
  const uint32_t exps = (uint32_t)(HD / 2) << d.logP;      // from a page's codes to its exponents
  for (;;) {
  int en[kKvEntryInts];
#pragma unroll
  for (int i = 0; i < kKvEntryInts; ++i) {
    if constexpr (OWN) en[i] = __builtin_amdgcn_readfirstlane(reinterpret_cast<const int32_t*>(own_ent + e)[i]);
    else en[i] = as_scalar(d.list.ent + e)[i];
  }
  const int tok0 = en[0], row0 = en[1], nrows = en[2], seq = en[3], p0 = en[4], prefix = en[5];
  const int kfloor = en[6], kceil = en[7], ks_ = en[8], klo = en[9], khi = en[10], tiles = en[11];
  const int a0 = en[12], n1 = en[13], b0 = en[14];
  const int left = f1 - f + imin(j, 0);           // units of the share from tile max(j, 0) on
  f += tiles - j;                                 // the segment's end
  j = imax(j, 0);
  const int nj = imin(tiles - j, left);
  if (nj <= 0) return;                            // whole workgroup: the share ends before a tile
  const bool whole = nj == tiles;
  auto tile_key = [&](int t) { return kKvTile * (t < n1 ? a0 + t : b0 + t - n1); };

  // ---- loads of a tile: 4 groups of 16 keys, wherever their pages lie ----
  // Keys that no row sees are loaded like the others: their scores are masked, and blocks
  // of V that are NaN leave the product where a row may not see their key.
  const scalar_i32 tb = as_scalar(d.table + (int64_t)seq * d.table_ld);
  const uint64_t head = (uint64_t)((int64_t)kvh << d.logP) * RBM;
  const uint32_t page_bytes = (uint32_t)(d.nkv * RBM) << d.logP;
  uint32_t bad = 0;
  u32x4 kx[4], vx[4];
  uint32_t ke[4], ve[4];
  int pg[4];                                      // the next tile's pages
  auto pages = [&](int t) __attribute__((always_inline)) {
    const int k0 = tile_key(t);
#pragma unroll
    for (int n = 0; n < 4; ++n) pg[n] = tb[imin((k0 + 16 * n) >> d.logP, d.cols - 1)];
  };
  auto fetch = [&](auto isv, int t, u32x4 (&x)[4], uint32_t (&ex)[4]) __attribute__((always_inline)) {
    constexpr bool V = decltype(isv)::value;
    const char* const base = (V ? d.vc : d.kc) + head;
    const uint32_t xo = V ? vo : ko, eo = V ? veo : keo;
    const int k0 = tile_key(t);
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int g0 = k0 + 16 * n, r = g0 & P1;
      uint32_t page = (uint32_t)pg[n];
      if (page >= (uint32_t)d.n_pages) {          // wave-uniform
        const int from = imax(g0, kfloor), to = imin(g0 + 16, khi);
        bad |= ((from < to) & ((to > klo) | (from < ks_))) ? XP_DEVERR_PAGE : 0u;
        page = 0;
      }
      // wave-uniform addresses: scalar registers and the lane's bytes
      uint64_t codes = (uint64_t)(uintptr_t)base + (uint64_t)page * page_bytes + (uint32_t)(r * (HD / 2));
      uint64_t ep = codes + exps - (uint32_t)(r * (HD / 2 - HD / 32));
      asm volatile("" : "+s"(codes), "+s"(ep));
      if constexpr (HD == 128 || !V) {
        x[n] = ld16_nt((const char*)(uintptr_t)codes + xo);
      } else {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        const u32x2 y = __builtin_nontemporal_load(
            reinterpret_cast<const u32x2*>((const char*)(uintptr_t)codes + xo));
        x[n] = u32x4{y[0], y[1], 0u, 0u};
      }
      ex[n] = *reinterpret_cast<const uint8_t*>((const char*)(uintptr_t)ep + eo);
    }
  };
  constexpr std::integral_constant<bool, false> isk{};
  constexpr std::integral_constant<bool, true> isv{};
  if (wave < nj) {
    pages(j + wave);
    fetch(isk, j + wave, kx, ke);
    fetch(isv, j + wave, vx, ve);
    pages(j + imin(wave + NW, nj - 1));
  }

  // ---- the query rows ----
  const bool rv = ri < nrows;
  KvSees sees;
  // dims 8 c .. 8 c + 7 of row ri, as they are
  auto raw_q = [&](int c) __attribute__((always_inline)) {
    c += ri * (HD / 8);
    if constexpr (kBehind)
      return reinterpret_cast<u32x4*>(lds + c / 32 * kRing + c % 32 * RB + 2 * HD);
    else
      return own_q + c;
  };
  intx8 qp[QM];
  int qs[QM];
  bool raw = false;                               // some row has elements that are in no part
  {
    const int row = row0 + (rv ? ri : 0), tk = row / d.grp;
    const int64_t tok = tok0 + tk;
    const uint16_t* q = d.q + tok * d.q_ld + (int64_t)(kvh * d.grp + (row - tk * d.grp)) * HD;
    constexpr int NQ = HD / 64;                   // pieces of 16 dims: 16 g, and 64 + 16 g
    uint32_t x[NQ][8];
    uint32_t top = 0;                             // the greatest magnitudes, two of 16 bits,
    ushort2v low = {0xffff, 0xffff};              // the least but 0, less 1
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const u32x4 y = ld16(q + 64 * n + 16 * g + 8 * c);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[n][4 * c + i] = y[i];
          top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(
              __builtin_bit_cast(ushort2v, top), __builtin_bit_cast(ushort2v, y[i] & 0x7fff7fffu)));
          low = __builtin_elementwise_min(
              low, __builtin_bit_cast(ushort2v, y[i] & 0x7fff7fffu) - ushort2v{1, 1});
        }
      }
    const uint32_t most = umax_xor32(umax_xor16(max(top >> 16, top & 0xffffu)));
    // 2^7 <= x < 2^8 for the largest; an infinity or NaN makes the row's scores NaN
    const bool odd = most >= 0x7f80u;
    const int eb = imax((int)(most >> 7), kDeepest + 1);
    const int s0 = eb - 7, s1 = s0 - 5;
    const float up = __uint_as_float((uint32_t)(261 - imin(eb, 254)) << 23);
    raw = __ballot((int)min(low[0], low[1]) + 1 < (eb - kDeepest) << 7) != 0;
    if (__builtin_expect(raw, 0)) {               // wave-uniform; every wave writes the same
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c)
          if (li < R)
            *raw_q(8 * n + 2 * g + c) = u32x4{x[n][4 * c], x[n][4 * c + 1], x[n][4 * c + 2], x[n][4 * c + 3]};
      wave_lds_order();
    }
    intx8 part[2];
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t w = odd ? 0u : x[n][2 * c + i / 2];
          y[i] = __uint_as_float(i % 2 == 0 ? w << 16 : w & 0xffff0000u) * up;
        }
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
          w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
          part[p][4 * n + c] = w;
          if (p == 0) {                           // 5 binades to the next
            const xp_f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
            const xp_f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
            y[0] = (y[0] - lo[0]) * 0x1p5f;
            y[1] = (y[1] - lo[1]) * 0x1p5f;
            y[2] = (y[2] - hi[0]) * 0x1p5f;
            y[3] = (y[3] - hi[1]) * 0x1p5f;
          }
        }
      }
    const bool second = HALF && li >= 8;          // the columns of second parts
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      if constexpr (HD == 128 && !HALF) {
        qp[0][c] = part[0][c];
        qp[1][c] = part[1][c];
      } else if constexpr (HD == 128) {
        qp[0][c] = second ? part[1][c] : part[0][c];
      } else {                                    // both parts, 64 dims each
        qp[0][c] = second ? 0 : part[c / 4][c % 4];
      }
    }
    if constexpr (HD == 128 && !HALF) {
      qs[0] = s0;
      qs[1] = s1;
    } else if constexpr (HD == 128) {
      qs[0] = second ? s1 : s0;
    } else {
      qs[0] = g < 2 ? s0 : s1;
    }
#pragma unroll
    for (int i = 0; i < QM; ++i) qs[i] = odd ? 255 : qs[i];
    const int p = prefix ? d.w.pos[tok] : p0 + tk;
    const int hi = rv ? (d.causal ? imin(p + 1, kceil) : kceil) : kfloor;
    const int lo = d.window > 0 ? imax(p - d.window + 1, kfloor) : kfloor;
    sees = KvSees{lo, kfloor, (uint32_t)imax(hi - lo, 0),
                  d.window > 0 ? (uint32_t)imax(imin(d.sinks, hi) - kfloor, 0) : 0u};
  }
  const int pmin = p0 + (prefix ? 0 : row0 / d.grp);
  const int pmax = prefix ? en[15] : p0 + (row0 + nrows - 1) / d.grp;
  const int whi = d.causal ? imin(pmin + 1, kceil) : kceil;
  const int wlo = d.window > 0 ? imax(pmax - d.window + 1, kfloor) : kfloor;
  const int wsink = d.window > 0 ? d.sinks : 0;

  float m_run = -INFINITY, l_run = 0.f;           // the row's; l of this lane's keys
  floatx4 o[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) o[t] = floatx4{0.f, 0.f, 0.f, 0.f};

  auto v_write = [&](int h) __attribute__((always_inline)) {   // V of half a tile to LDS
    wave_lds_order();
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const float s = __uint_as_float(ve[2 * h + n] << 23);
#pragma unroll
      for (int i = 0; i < HD / 32; ++i)
        *(lds_u32x4*)(uintptr_t)(vw + 16 * n * RB + 16 * i) = f4_bf16x8(vx[2 * h + n][i], s);
    }
    wave_lds_order();
  };
#pragma unroll 1
  for (int t = wave; t < nj; t += NW) {
    const int k0 = tile_key(j + t);
    const bool more = t + NW < nj;
    // every row sees every key of the tile
    const bool seen = k0 >= kfloor && k0 + kKvTile <= whi && (k0 >= wlo || k0 + kKvTile <= wsink);
    // exponents above 252 are NaN; rarely there, so all are looked at together
    if (__builtin_expect(__ballot(max(max(ke[0], ke[1]), max(ke[2], ke[3])) > 252u) != 0, 0)) {
#pragma unroll
      for (int n = 0; n < 4; ++n) ke[n] = ke[n] > 252u ? 255u : ke[n];
    }
    // ---- scores ----
    floatx4 s[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) s[n] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int p = QM - 1; p >= 0; --p)
#pragma unroll
      for (int n = 0; n < 4; ++n) s[n] = mma16_f4f8(kx[n], qp[p], s[n], (int)ke[n], qs[p]);
    if (__builtin_expect(raw, 0)) {               // wave-uniform: in their place
#pragma unroll
      for (int n = 0; n < 4; ++n) s[n] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const u32x4 x = *raw_q(4 * (g & (HD / 32 - 1)) + t);
        const u32x4 y = li < R && g < HD / 32 ? x : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int n = 0; n < 4; ++n)
          s[n] = mma16_bf16(f4_bf16x8(kx[n][t], __uint_as_float(ke[n] << 23)), y, s[n]);
      }
    }
    if constexpr (HALF) {                         // a row's parts
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][i] += other_half(s[n][i]);
    }
    if (!seen) {
      uint32_t a = (uint32_t)(k0 + 4 * g - sees.lo), b = (uint32_t)(k0 + 4 * g - sees.floor);
      asm volatile("" : "+v"(a), "+v"(b));        // a branch of its own
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          s[n][i] = ((a + 16 * n + i < sees.n) | (b + 16 * n + i < sees.s)) ? s[n][i] : -INFINITY;
    }
    if (more) fetch(isk, j + t + NW, kx, ke);
    // ---- softmax ----
    constexpr float kLazy = 8.f;
    float mt = s[0][0];
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) mt = fmaxf(mt, s[n][i]);
    mt = fmax_xor32(fmax_xor16(mt)) * d.scale2;
    if (__ballot(mt > m_run + kLazy) != 0) {      // wave-uniform
      const float mref = fmaxf(m_run, mt);
      const float alpha = __builtin_amdgcn_exp2f(m_run - (mref == -INFINITY ? 0.f : mref));
      l_run *= alpha;
      m_run = mref;
#pragma unroll
      for (int u = 0; u < NT; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[u][i] *= alpha;
    }
    const float ref = m_run == -INFINITY ? 0.f : m_run;
    u32x4 ph[2], pl[2];                           // the column's part; both parts
#pragma unroll
    for (int n = 0; n < 4; ++n) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[n][i] = __builtin_amdgcn_exp2f(fmaf(s[n][i], d.scale2, -ref));
        l_run += s[n][i];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float e0 = s[n][2 * i], e1 = s[n][2 * i + 1];
        const uint32_t y = pk_bf16(e0, e1);
        const uint32_t z = pk_bf16(e0 - __uint_as_float(y << 16), e1 - __uint_as_float(y & 0xFFFF0000u));
        ph[n / 2][2 * (n % 2) + i] = HALF && li >= 8 ? z : y;
        if constexpr (!HALF) pl[n / 2][2 * (n % 2) + i] = z;
      }
    }
    if (__builtin_expect(__ballot(max(max(ve[0], ve[1]), max(ve[2], ve[3])) > 252u) != 0, 0)) {
      uint32_t odd = 0;                           // a bit a group: the lane's block is NaN
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        if (ve[n] > 252u) {
          // where a row may not see the key its NaN leaves the product
          odd |= seen ? 0u : 1u << n;
          ve[n] = seen ? 255u : 0u;
          vx[n] = seen ? vx[n] : u32x4{0u, 0u, 0u, 0u};
        }
      }
      // Rows with a numerator for a key whose block is NaN are NaN in its dims.  Key li of
      // group n, the dims of lane (li, g): the key's numerator is element li % 4 of s[n] in
      // the lanes 16 (li / 4) + row.
      uint32_t some = 0;
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) some |= s[n][i] > 0.f ? 1u << (4 * n + i) : 0u;
#pragma unroll 1
      for (int n = 0; n < 4; ++n) {
        uint64_t who = __ballot((odd >> n) & 1u);
        while (who != 0) {                        // wave-uniform
          const int src = __builtin_ctzll(who), key = src & 15, part = src >> 4;
          who &= who - 1;
          const uint32_t has = (uint32_t)__shfl((int)some, 16 * (key / 4) + li, kWave);
          const bool hit = (has >> (4 * n + key % 4)) & 1u;
#pragma unroll
          for (int u = 0; u < NT; ++u)
            if ((16 * u) / (HD / 4) == part && hit)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[u][i] = NAN;
        }
      }
    }
    // ---- P V, 32 keys at a time ----
    v_write(0);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      constexpr int NB = NT / 2;                  // blocks of dims at a time
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        u32x4 v[NB];
#pragma unroll
        for (int u = 0; u < NB; ++u) {
          const uint2 lo = lds_tr16(vr + 32 * (c * NB + u)), hi = lds_tr16(vr + 32 * (c * NB + u) + 16 * RB);
          v[u] = u32x4{lo.x, lo.y, hi.x, hi.y};
        }
        if (h == 0 && c == 1) {
          v_write(1);
          if (more) {
            fetch(isv, j + t + NW, vx, ve);
            pages(j + imin(t + 2 * NW, nj - 1));
          }
        }
        if constexpr (!HALF) {
#pragma unroll
          for (int u = 0; u < NB; ++u) o[c * NB + u] = mma16_bf16(v[u], pl[h], o[c * NB + u]);
        }
#pragma unroll
        for (int u = 0; u < NB; ++u) o[c * NB + u] = mma16_bf16(v[u], ph[h], o[c * NB + u]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  // ---- the waves' results ----
  if constexpr (HALF) {                           // a row's parts
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[u][i] += other_half(o[u][i]);
  }
  l_run = fsum_xor32(fsum_xor16(l_run));
  __syncthreads();                                // every wave's reads of its ring done
  float* mg = reinterpret_cast<float*>(lds) + wave * (kRing / 4) + lane;
  mg[0] = m_run;
  mg[kWave] = l_run;
  floatx4* mo = reinterpret_cast<floatx4*>(ring + 2 * kWave * 4) + lane;
#pragma unroll
  for (int u = 0; u < NT; ++u) mo[u * kWave] = o[u];
  __syncthreads();
  // wave w adds the blocks w, w + NW, .. of 16 dims
  {
    float M = -INFINITY, wt[NW], l = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      wt[w] = reinterpret_cast<const float*>(lds)[w * (kRing / 4) + lane];
      M = fmaxf(M, wt[w]);
    }
    const float Ms = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      wt[w] = __builtin_amdgcn_exp2f(wt[w] - Ms);
      l += wt[w] * reinterpret_cast<const float*>(lds)[w * (kRing / 4) + kWave + lane];
    }
    const bool mine = li < imin(nrows, R);
    const int row = row0 + (mine ? li : 0), tk = row / d.grp;
    const int64_t tok = tok0 + tk;
    const int hd_ = kvh * d.grp + (row - tk * d.grp);
    const bool done = whole && d.groups == 0;
    const int64_t prow = whole ? d.row0 + ((int64_t)prefix * d.total_q + tok) * d.nh + hd_
                               : d.part0 + (int64_t)(2 * sidx + (j == 0 ? 1 : 0)) * R + li;
    const float inv = l == 0.f ? (sees_some(d, p0 + tk, kceil) ? NAN : 0.f) : 1.f / l;
#pragma unroll
    for (int u0 = 0; u0 < NT; u0 += NW) {
      const int u = u0 + wave;
      if (NT % NW != 0 && u >= NT) break;         // whole wave
      floatx4 y{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const floatx4 x = reinterpret_cast<const floatx4*>(lds + w * kRing + 2 * kWave * 4)[u * kWave + lane];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] += wt[w] * x[i];
      }
      if (mine && done) {
        *reinterpret_cast<uint2*>(d.out + tok * d.out_ld + (int64_t)hd_ * HD + 16 * u + 4 * g) =
            uint2{pk_bf16(y[0] * inv, y[1] * inv), pk_bf16(y[2] * inv, y[3] * inv)};
      } else if (mine) {
        *reinterpret_cast<floatx4*>(d.w.part + prow * HD + 16 * u + 4 * g) = y;
      }
    }
    if (mine && wave == 0 && g == 0) {
      if (!done) {
        *reinterpret_cast<float2*>(d.w.ml + 2 * prow) = float2{M, l};
      } else if (d.lse != nullptr) {
        d.lse[tok * d.nh + hd_] =
            l == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
      }
    }
  }
  if (bad != 0) atomicOr(d.err, bad);
  // ---- on to the next segment of the share ----
  if (f >= f1) return;                            // whole workgroup
  j = -kSegUnits;
  if (++kvh == d.nkv) {
    kvh = 0;
    ++e;
  }
  __syncthreads();                                // the merge is read
  }
}

// ---------------------------------------------------------------------------
// Joining.  Part (m_i, l_i, O_i) of a row: O = sum 2^(m_i - M) O_i, l likewise,
// M = max m_i, parts in order.  A workgroup per share and 1024 / head_dim rows, most of
// which find nothing cut: 4 us, 12 to 17 with a tile of 128 or 256 rows for every
// share; every row of 960 tokens with a prefix 21 us (reads of the parts from memory).
// ---------------------------------------------------------------------------
struct KvSum {
  float m = -INFINITY, l = 0.f;
  floatx4 o{0.f, 0.f, 0.f, 0.f};
  __device__ __forceinline__ void add(float m1, float l1, floatx4 o1) {
    const float M = fmaxf(m, m1), Ms = M == -INFINITY ? 0.f : M;
    const float w0 = __builtin_amdgcn_exp2f(m - Ms), w1 = __builtin_amdgcn_exp2f(m1 - Ms);
    m = M;
    l = w0 * l + w1 * l1;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = w0 * o[i] + w1 * o1[i];
  }
};

// U parts from share s on, their loads in flight together; those behind share s1 are
// not added (the last one is read again)
template <int HD, int U>
__device__ __forceinline__ void add_some(const KvDev& d, int64_t part0, int R, int s, int s0, int s1,
                                         int rr, int c, KvSum& x) {
  float2 ml[U];
  floatx4 o[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int su = imin(s + u, s1);
    const int64_t prow = part0 + (int64_t)(2 * su + (su == s0 ? 1 : 0)) * R + rr;
    ml[u] = *reinterpret_cast<const float2*>(d.w.ml + 2 * prow);
    o[u] = *reinterpret_cast<const floatx4*>(d.w.part + prow * HD + c);
  }
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (s + u <= s1) x.add(ml[u].x, ml[u].y, o[u]);
}

// the parts of row rr of the segment whose tiles are units [a, a + tiles), cut at
// multiples of S: the first at the end of share a / S, the others at the beginning of
// theirs.  Eight at a time where a long prefix has many (32 x 8192 keys in 26 parts:
// 7.5 us against 11 us by fours), four for the few of ordinary ones (19 against 24 us)
template <int HD>
__device__ __forceinline__ void add_parts(const KvDev& d, int64_t part0, int R, int a, int tiles,
                                          int S, int rr, int c, KvSum& x) {
  const int s0 = a / S, s1 = (a + tiles - 1) / S;
  int s = s0;
  for (; s + 3 < s1; s += 8) add_some<HD, 8>(d, part0, R, s, s0, s1, rr, c, x);
  if (s <= s1) add_some<HD, 4>(d, part0, R, s, s0, s1, rr, c, x);
}

// p: the token's position, keys: its sequence's
template <int HD>
__device__ __forceinline__ void write_row(const KvDev& d, int64_t tok, int head, int c,
                                          const KvSum& x, int p, int keys) {
  const int kvh = head / d.grp;
  const float inv = x.l == 0.f ? (sees_some(d, p, keys) ? NAN : 0.f)
                               : (d.v_scale != nullptr ? d.v_scale[kvh] : 1.f) / x.l;
  *reinterpret_cast<uint2*>(d.out + tok * d.out_ld + (int64_t)head * HD + c) =
      uint2{pk_bf16(x.o[0] * inv, x.o[1] * inv), pk_bf16(x.o[2] * inv, x.o[3] * inv)};
  if (d.lse != nullptr && c == 0)
    d.lse[tok * d.nh + head] = x.l == 0.f
        ? -INFINITY : (x.m + __builtin_amdgcn_logf(x.l)) * 0.69314718055994531f;
}

// Workgroup (s, y): the segment that share s begins inside of, if no share
// before s does; rows HD / 4 threads each.
template <int HD>
__global__ __launch_bounds__(256) void k_kv_join(const KvDev d, int R) {
  constexpr int TPR = HD / 4, RPB = 256 / TPR;
  const int s = blockIdx.x + 1;
  const scalar_i32 sh = as_scalar(d.list.share + s), hd = as_scalar(d.list.hdr);
  const int f = sh[0], e = sh[1], kvh = sh[2], j = sh[3], S = hd[1];
  if (f >= hd[0] || j <= 0) return;               // past the end, or nothing is cut here
  const int a = f - j;                            // the unit of the segment's first tile
  if (a < f - S) return;                          // cut before: an earlier workgroup's
  const scalar_i32 en = as_scalar(d.list.ent + e);
  const int tok0 = en[0], row0 = en[1], nrows = en[2], p0 = en[4], keys = en[7], tiles = en[11];
  const int rr = blockIdx.y * RPB + threadIdx.x / TPR, c = 4 * (threadIdx.x % TPR);
  if (rr >= nrows) return;
  KvSum x;
  add_parts<HD>(d, d.part0, R, a, tiles, S, rr, c, x);
  const int row = row0 + rr, tk = row / d.grp;
  write_row<HD>(d, tok0 + tk, kvh * d.grp + (row - tk * d.grp), c, x, p0 + tk, keys);
}

// Calls with shared prefixes: every row, its prefix's result and its own.
struct KvJoin {
  int R[2];                          // row tiles of the sequences, of the groups
  int64_t part0;                     // first partial row of the groups' list
  int one;                           // both are in one list, the groups behind the sequences
};
template <int HD>
__global__ __launch_bounds__(256) void k_kv_join_rows(const KvDev d, const KvJoin jn) {
  constexpr int TPR = HD / 4, RPB = 256 / TPR;
  const int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
  const int c = 4 * (threadIdx.x % TPR);
  if (row >= (int64_t)d.total_q * d.nh) return;
  const int tok = (int)(row / d.nh), head = (int)(row - (int64_t)tok * d.nh);
  const int kvh = head / d.grp, hg = head - kvh * d.grp;
  const int2 at[2] = {d.w.row[0][tok], d.w.row[1][tok]};
  if (at[0].x < 0) return;                        // behind the last sequence
  int lr[2], c0[2], c1[2], S[2];                  // row, units before and behind its entry
  const KvEntry* own = nullptr;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const KvList& l = d.w.list[jn.one ? 0 : k];
    lr[k] = at[k].x + hg;
    const int e = at[k].y + lr[k] / jn.R[k];
    const bool has = (at[k].x >= 0) & (e < l.hdr[2]);   // past it: token ranges that overlap
    S[k] = l.hdr[1];
    c0[k] = l.cum[has ? e : 0];
    c1[k] = has ? l.cum[e + 1] : 0;
    if (k == 0) own = l.ent + (has ? e : 0);
  }
  KvSum x;
#pragma unroll
  for (int k = 1; k >= 0; --k) {                  // the prefix, then the sequence's own keys
    if (c1[k] == 0) continue;
    const int seg = (c1[k] - c0[k]) / d.nkv, tiles = seg - kSegUnits;
    const int a = c0[k] + kvh * seg + kSegUnits;
    if (a / S[k] == (a + tiles - 1) / S[k]) {
      const int64_t prow = d.row0 + ((int64_t)k * d.total_q + tok) * d.nh + head;
      const float2 ml = *reinterpret_cast<const float2*>(d.w.ml + 2 * prow);
      x.add(ml.x, ml.y, *reinterpret_cast<const floatx4*>(d.w.part + prow * HD + c));
    } else {
      add_parts<HD>(d, k == 1 ? jn.part0 : 0, jn.R[k], a, tiles, S[k], lr[k] % jn.R[k], c, x);
    }
  }
  write_row<HD>(d, tok, head, c, x, d.w.pos[tok], own->ceil);
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
// Rows of a workgroup by the rows that a sequence of max_q tokens (a group of
// sequences) brings: the fewest waves that hold them, so that short ones leave room for
// a second workgroup and its loads.  Where many rows let the products bound the call:
// 8 waves of 32 rows at head_dim 128 (a CU's ring holds no second workgroup's), at 64
// three workgroups of 4, whose tiles waste less of ragged sequences (24 of 1 .. 513
// tokens 255 -> 232 us; 4096 x 8192 415 either way).
static int kv_most(const xp_kv* kv) { return kv->hd == 64 ? 128 : 256; }
static int kv_rows(const xp_kv* kv, int64_t rows) {
  const int most = kv_most(kv);
  if (kv_least(kv, rows) < 32) return kv_least(kv, rows);   // k_kv_few
  return rows <= 32 ? 32 : rows <= 64 ? 64 : rows <= 128 ? 128 : most;
}
constexpr int kFewWaves = 4;
// Workgroups of a CU: 8 waves (12, see above), or as many as the rings leave room for (a
// ring of two 32 KB stages twice).  128 rows over an 8-bit cache as two workgroups of 4
// waves: 64 blocks of 32 over 8192 keys 405 us as one of 8, 378 so; 256 rows as two
// tiles of them 3 to 7% slower.
static int kv_wgs(const xp_kv* kv, int R) {
  if (R <= kFewRows) return 4 * kFewSimd / kFewWaves;
  if (kv->hd == 64) return R >= 128 ? 3 : (R == 64 ? 2 : 4);
  const bool f8 = kv->dtype == XP_E4M3;
  return R >= 128 ? (f8 && R == 128 ? 2 : 1) : (f8 && R == 32 ? 4 : 2);
}
static int kv_shares(const xp_kv* kv, int R) { return std::max(8, kv->cus * kv_wgs(kv, R) / 8 * 8); }

void kv_attn_sizes(const xp_kv* kv, int64_t* rows, int* entries, int* shares) {
  const int64_t all = (int64_t)kv->max_tokens * kv->grp;
  const int R = kv_rows(kv, all);
  *rows = 0;
  const int least = kv_least(kv);
  for (int r = least; r <= R; r *= 2) *rows = std::max(*rows, (int64_t)2 * kv_shares(kv, r) * r);
  // every sequence (group) rounds its rows up to whole tiles
  *entries = (int)((all + least - 1) / least + kv->max_batch);
  *shares = 0;
  for (int r = least; r <= R; r *= 2) *shares = std::max(*shares, kv_shares(kv, r));
}

// one list's attention, in tiles of R rows
static hipError_t launch_list(const xp_kv* kv, int R, bool own, const KvDev& d, hipStream_t st) {
  const int shares = kv_shares(kv, R);
#define XP_KV(HD_, FMT_, WR_, WK_, NST_, PARTS_)                                                 \
  do {                                                                                           \
    if (own)                                                                                     \
      hipLaunchKernelGGL((k_kv_attn<HD_, FMT_, WR_, WK_, NST_, PARTS_, true>), dim3(shares),     \
                         dim3((WR_) * (WK_) * kWave), 0, st, d);                                 \
    else                                                                                         \
      hipLaunchKernelGGL((k_kv_attn<HD_, FMT_, WR_, WK_, NST_, PARTS_, false>), dim3(shares),    \
                         dim3((WR_) * (WK_) * kWave), 0, st, d);                                 \
  } while (0)
  const int fmt = kv->dtype;
  if (R <= kFewRows) {
#define XP_FEW(HD_, R_)                                                                         \
  do {                                                                                           \
    const dim3 grid(shares), block(kFewWaves * kWave);                                           \
    if (own) hipLaunchKernelGGL((k_kv_few<HD_, R_, kFewWaves, true>), grid, block, 0, st, d);    \
    else hipLaunchKernelGGL((k_kv_few<HD_, R_, kFewWaves, false>), grid, block, 0, st, d);       \
  } while (0)
    if (kv->hd == 128 && R == 8) XP_FEW(128, 8);
    else if (kv->hd == 128) XP_FEW(128, 16);
    else if (R == 8) XP_FEW(64, 8);
    else XP_FEW(64, 16);
#undef XP_FEW
  } else if (kv->hd == 128 && fmt == XP_BF16) {
    if (R == 32) XP_KV(128, XP_BF16, 1, 2, 2, 2);
    else if (R == 64) XP_KV(128, XP_BF16, 2, 2, 2, 2);
    else if (R == 128) XP_KV(128, XP_BF16, 4, 2, 4, 1);
    else XP_KV(128, XP_BF16, 8, 1, 4, 1);
  } else if (kv->hd == 128 && fmt == XP_E4M3) {
    if (R == 32) XP_KV(128, XP_E4M3, 1, 2, 2, 1);
    else if (R == 64) XP_KV(128, XP_E4M3, 2, 2, 4, 1);
    else if (R == 128) XP_KV(128, XP_E4M3, 4, 1, 4, 1);
    else XP_KV(128, XP_E4M3, 8, 1, 8, 1);
  } else if (kv->hd == 128) {
    if (R == 32) XP_KV(128, XP_MXFP4, 1, 2, 3, 2);
    else if (R == 64) XP_KV(128, XP_MXFP4, 2, 2, 3, 1);
    else if (R == 128) XP_KV(128, XP_MXFP4, 4, 2, 3, 1);
    else XP_KV(128, XP_MXFP4, 8, 1, 3, 1);
  } else if (fmt == XP_BF16) {
    if (R == 32) XP_KV(64, XP_BF16, 1, 2, 2, 2);
    else if (R == 64) XP_KV(64, XP_BF16, 2, 2, 4, 2);
    else XP_KV(64, XP_BF16, 4, 1, 3, 1);
  } else if (fmt == XP_E4M3) {
    if (R == 32) XP_KV(64, XP_E4M3, 1, 2, 2, 1);
    else if (R == 64) XP_KV(64, XP_E4M3, 2, 2, 4, 1);
    else XP_KV(64, XP_E4M3, 4, 1, 6, 1);
  } else {
    if (R == 32) XP_KV(64, XP_MXFP4, 1, 2, 3, 2);
    else if (R == 64) XP_KV(64, XP_MXFP4, 2, 2, 3, 1);
    else XP_KV(64, XP_MXFP4, 4, 1, 3, 1);
  }
#undef XP_KV
  return hipGetLastError();
}

hipError_t launch_kv_attn(const xp_kv* kv, const KvAttnArgs& a, hipStream_t st) {
  // row tiles of the sequences, and of the groups.  One list for both unless the
  // groups' are the largest, where products bound the call: a short sequence's
  // rows in such tiles cost more than a second launch.  32 single tokens behind 8192 keys
  // (tiles of 128 rows): one list 53 us, two 61; 60 blocks of 16 behind 500 .. 12000
  // (tiles of 256): 239 and 218.
  const int64_t rows = (int64_t)a.max_q * kv->grp;
  int R[2] = {kv_rows(kv, rows), 0};
  if (a.groups > 0) R[1] = kv_rows(kv, std::max(rows, (int64_t)a.total_q / a.groups * kv->grp));
  const int lists = R[1] == kv_most(kv) && R[0] < R[1] ? 2 : 1;
  if (lists == 1 && a.groups > 0) R[0] = R[1];
  const int cols = (int)std::min<int64_t>(kv->max_pages, a.table_ld);
  KvPlan p{};
  p.n = a.n;
  p.total_q = a.total_q;
  p.max_q = a.max_q;
  p.kv_add = a.kv_add;
  p.cap = (int)std::min<int64_t>((int64_t)cols << kv->logP, kKvMaxLen);
  p.grp = kv->grp;
  p.nkv = kv->nkv;
  p.causal = a.causal;
  p.window = a.window;
  p.sinks = a.sinks;
  p.groups = a.groups;
  p.entries = (int)((int64_t)a.total_q * kv->grp / kv_least(kv, rows) + a.n);   // of a list: no more fit the tokens
  for (int k = 0; k < lists; ++k) {
    p.R[k] = R[k];
    p.shares[k] = kv_shares(kv, R[k]);
  }
  p.cu_q = a.cu_q;
  p.kv_len = a.kv_len;
  p.group_start = a.group_start;
  p.shared_len = a.shared_len;
  int64_t most = (int64_t)a.total_q * kv->grp / R[0] + a.n;
  // few rows: a tile has a token at least, so that 64 single tokens make their list themselves
  if (R[0] <= kFewRows && kv->grp <= R[0]) most = std::min<int64_t>(most, a.total_q);
  // plan_own has a lane for a request and one for an entry: requests without tokens have a
  // lane, but no entry
  const bool own = a.groups == 0 && a.n <= kOwnEntries && most <= kOwnEntries;
  if (own) p.entries = (int)most;
  hipError_t e;
  if (!own) {
    if (a.groups > 0)
      hipLaunchKernelGGL(k_kv_plan<true>, dim3(lists), dim3(kPlanThreads), 0, st, p, kv->a, kv->err);
    else
      hipLaunchKernelGGL(k_kv_plan<false>, dim3(1), dim3(kPlanThreads), 0, st, p, kv->a, kv->err);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }

  KvDev d{};
  d.q = a.q;
  d.q_ld = a.q_ld;
  d.out = a.out;
  d.out_ld = a.out_ld;
  d.lse = a.lse;
  d.kc = (const char*)a.kc;
  d.vc = (const char*)a.vc;
  d.k_scale = a.k_scale;
  d.v_scale = a.v_scale;
  d.table = a.table;
  d.table_ld = a.table_ld;
  d.nh = kv->nh;
  d.nkv = kv->nkv;
  d.grp = kv->grp;
  d.logP = kv->logP;
  d.n_pages = kv->n_pages;
  d.cols = cols;
  d.causal = a.causal;
  d.window = a.window;
  d.sinks = a.sinks;
  d.scale2 = (a.scale > 0.f ? a.scale : 1.f / std::sqrt((float)kv->hd)) * 1.4426950408889634f;
  d.total_q = a.total_q;
  d.groups = a.groups;
  d.row0 = 2 * kv->rows;
  d.p = p;
  d.w = kv->a;
  d.err = kv->err;
  const bool wide = kv->hd == 128;
  if (a.groups == 0) {
    d.list = kv->a.list[0];
    if ((e = launch_list(kv, R[0], own, d, st)) != hipSuccess) return e;
    const dim3 grid(kv_shares(kv, R[0]) - 1, (R[0] * kv->hd + 1023) / 1024);
    if (wide) hipLaunchKernelGGL(k_kv_join<128>, grid, dim3(256), 0, st, d, R[0]);
    else hipLaunchKernelGGL(k_kv_join<64>, grid, dim3(256), 0, st, d, R[0]);
    return hipGetLastError();
  }
  for (int k = lists - 1; k >= 0; --k) {          // the prefixes, then the sequences' own keys
    d.list = kv->a.list[k];
    d.part0 = k * kv->rows;
    if ((e = launch_list(kv, R[k], false, d, st)) != hipSuccess) return e;
  }
  KvJoin jn{};
  jn.R[0] = R[0];
  jn.R[1] = R[1];
  jn.part0 = lists == 2 ? kv->rows : 0;
  jn.one = lists == 1;
  const int rpb = 1024 / kv->hd;
  const dim3 grid((unsigned)(((int64_t)a.total_q * kv->nh + rpb - 1) / rpb));
  if (wide) hipLaunchKernelGGL(k_kv_join_rows<128>, grid, dim3(256), 0, st, d, jn);
  else hipLaunchKernelGGL(k_kv_join_rows<64>, grid, dim3(256), 0, st, d, jn);
  return hipGetLastError();
}

}  // namespace xp
