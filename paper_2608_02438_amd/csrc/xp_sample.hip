// Tokens from logits: temperature, top-k, top-p and min-p, from given uniforms.
//
// With m = max l, the weight of token v is e^{(l_v - m) / T}.  Top-k and top-p keep
// what lies above a threshold of l (top-p also cuts through equal logits, lowest index
// first), min-p what is heavy enough, and the sample is the first token in index order
// with sum of the kept weights up to it > u times their sum.
//
// A sample hangs on where u falls between sums over the vocabulary, so the weights are
// formed in 64 bits and then held as integers, 2^45 for the largest: sums of up to 2^18
// of them are 2^63 at most and exact, the same whatever their order.  They are compared
// with p or u times another sum in fp64: from 2^53 on (256 tokens of the largest weight)
// both sides are rounded, by 2^-53 of themselves, which never puts sums out of order, so
// that exactly one token passes.  What that, and 2^-46 of the largest weight, can move is
// far below the 2^-24 by which uniforms differ.
//
// Four launches: the largest logits; weights or a histogram of them; the tokens in the bin
// where the threshold falls (or down to it); thresholds and the draw.  Each reads the row
// once, from the caches after the first, and what bounds them is what each does before its
// first and after its last token (settings, bins, scans, barriers): one row of 151936 logits
// 3.5 + 5.5 + 8 + 6 us, 64 rows with every kind of filter 7.5 + 19 + 15 + 21.  The weights of
// all tokens of 64 rows take 7 us.  With fewer registers (118 to 128) more workgroups would
// run at once, but spill (74 to 148 us in all in place of 64); by half chunks, in 82 to 92
// and without spilling, 66.5.
#include <stdarg.h>
#include <stdio.h>

#include <algorithm>
#include <new>
#include <string>

#include "xp_internal.h"

namespace xp {

constexpr int kSmpMaxV = 1 << 18;
constexpr int kSmpChunk = 4096;                    // tokens of a chunk
constexpr int kSmpChunks = kSmpMaxV / kSmpChunk;
constexpr int kSmpBatch = 128;                     // rows that go through the launches together
// passes over the vocabulary: a workgroup has some chunks of a row, a thread 16 tokens of each
constexpr int kSmpThreads = 256;
constexpr int kSmpPer = kSmpChunk / kSmpThreads;
constexpr int kSmpHist = 512;                      // bins of 1 / 16 in (m - l) / T
constexpr int kSmpCap = 16384;                     // candidates of a row
// the last launch: a workgroup a row
constexpr int kRowThreads = 1024;
constexpr int kRowWaves = kRowThreads / kWave;
constexpr int kRowBins = 2048;
static_assert(kSmpChunk == 4 * kRowThreads, "a thread of the row has 4 tokens of a chunk");

// What a row's launches leave for each other.
struct SmpRec {
  int32_t mode, edge;                // SmpMode; the last bin that counts
  uint32_t n, pad;                   // candidates
  uint64_t above, all;               // of the bins before the edge, of all: tokens where
                                     // top-k decides, else weight
};
enum SmpMode {
  kSmpPlain = 0,                     // no threshold of l: the chunks' sums are final
  kSmpList = 1,                      // the candidates are all tokens that can stay
  kSmpEdge = 2,                      // tokens before the edge's bin stay, those of it are candidates
  kSmpSlow = 3                       // too many candidates, no bins, or top-p among fewer than k
                                     // tokens with a weight: the row by radix selection
};

struct Smp {
  const void* logits;
  int64_t ld;
  int V;
  const uint8_t* temp;
  const float *temperature, *top_p, *min_p, *u;
  const int32_t* top_k;
  int32_t* ids;
  float* logprob;
  uint32_t* err;
  // of the batch's rows
  int64_t row0;
  int chunks, per_wg;                // of a row, of a workgroup
  uint64_t* best;                    // [rows][kSmpChunks] the largest key, lowest index
  uint64_t* sums;                    // [rows][kSmpChunks] kept weights
  uint64_t* hist;                    // [rows][kSmpHist] tokens (top-k) or weights of a bin
  uint64_t* part;                    // [rows][kSmpChunks][kSmpHist] weights of every chunk's bins
  SmpRec* rec;                       // [rows]
  uint64_t* list;                    // [rows][kSmpCap] key, index
};

// order-preserving image of a logit; 0 for NaN and -inf, which no one draws
__device__ __forceinline__ uint32_t smp_key(float l) {
  uint32_t u = __float_as_uint(l);
  if (u == 0x80000000u) u = 0u;                    // -0 is +0
  return l > -INFINITY ? ((u & 0x80000000u) ? ~u : (u | 0x80000000u)) : 0u;
}
__device__ __forceinline__ float smp_value(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? (key & 0x7FFFFFFFu) : ~key);
}

// A row's temperature and largest logit; x(l) = (l - m) / T, weights from it.
struct SmpRow {
  double inv_t, top;
  uint32_t top_key;
  float top_f, bin_t;
  __device__ __forceinline__ SmpRow(float t, uint32_t key)
      : inv_t(1.0 / (double)t), top((double)smp_value(key)), top_key(key), top_f(smp_value(key)),
        bin_t(16.f / t) {}
  __device__ __forceinline__ double xl(float l) const {
    return l == top_f ? 0.0 : ((double)l - top) * inv_t;
  }
  __device__ __forceinline__ double x(uint32_t key) const { return xl(smp_value(key)); }
  // e^x 2^45 to the nearest integer: 2^k e^f with |f| <= ln 2 / 2, e^f by its series up
  // to f^11 (2^-47 off), the integer from the sum with 2^52
  __device__ __forceinline__ uint64_t weight_at(double y) const {
    const double k = rint(y * 1.4426950408889634);
    const double f = fma(-k, 0.69314718055994531, y);
    double e = 1.0 / 39916800;
    e = fma(e, f, 1.0 / 3628800);
    e = fma(e, f, 1.0 / 362880);
    e = fma(e, f, 1.0 / 40320);
    e = fma(e, f, 1.0 / 5040);
    e = fma(e, f, 1.0 / 720);
    e = fma(e, f, 1.0 / 120);
    e = fma(e, f, 1.0 / 24);
    e = fma(e, f, 1.0 / 6);
    e = fma(e, f, 0.5);
    e = fma(e, f, 1.0);
    e = fma(e, f, 1.0);
    const int up = (int)k + 45;
    const double v = __hiloint2double(__double2hiint(e) + (up << 20), __double2loint(e));
    const uint64_t w = (uint64_t)__double_as_longlong(v + 0x1p52) & 0xfffffffffffffull;
    return y > -32.0 ? w : 0u;
  }
  __device__ __forceinline__ uint64_t weight(uint32_t key) const {
    return key != 0u ? weight_at(x(key)) : 0u;
  }
  // Bins of l from the largest down, 1 / 16 of (m - l) / T each: differences, products and
  // truncation in fp32 never fall where l falls, which is all that bins have to do.  From
  // kSmpHist on (and for -inf and NaN) there is no weight.
  __device__ __forceinline__ int bin(float l) const {
    const float b = l == top_f ? 0.f : (top_f - l) * bin_t;
    return b < (float)kSmpHist ? (int)b : kSmpHist;
  }
};

// What the sum of the kept weights is to exceed: u Z, not below 0 (else it would before
// the first token); NaN is never exceeded.
__device__ __forceinline__ double smp_goal(const Smp& d, int64_t r, uint64_t Z) {
  const float u = d.u[r];
  return u < 0.f ? 0.0 : (double)u * (double)Z;
}

// A sampled row's settings, replaced where they are out of range.
struct SmpSet {
  float t, p, mp;
  int k;
  uint32_t bad;
  __device__ __forceinline__ SmpSet(const Smp& d, int64_t r) {
    bad = 0;
    t = d.temperature ? d.temperature[r] : 1.f;
    if (!(t > 0.f && t < INFINITY)) {
      bad |= XP_DEVERR_TEMPERATURE;
      t = 1.f;
    }
    k = d.top_k ? d.top_k[r] : 0;
    p = d.top_p ? d.top_p[r] : 1.f;
    mp = d.min_p ? d.min_p[r] : 0.f;
    if (k < 0 || !(p > 0.f) || !(mp >= 0.f && mp <= 1.f)) {
      bad |= XP_DEVERR_FILTER;
      k = max(k, 0);
      p = p > 0.f ? p : 1.f;
      mp = mp >= 0.f && mp <= 1.f ? mp : 0.f;
    }
    k = k < d.V ? k : 0;
  }
  __device__ __forceinline__ bool cuts() const { return k > 0 || p < 1.f; }
  // the bins' fp32 holds 16 / t, and every difference of logits that has a weight
  __device__ __forceinline__ bool bins() const { return t >= 0x1p-120f && t <= 0x1p120f; }
  __device__ __forceinline__ double log_min() const { return mp > 0.f ? log((double)mp) : -INFINITY; }
};

__device__ __forceinline__ uint64_t wave_sum_u64(uint64_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += shfl_xor_u64(v, o);
  return v;
}
__device__ __forceinline__ uint64_t shfl_u64(uint64_t v, int lane) {
  return ((uint64_t)(uint32_t)__shfl((int)(v >> 32), lane, kWave) << 32) |
         (uint32_t)__shfl((int)v, lane, kWave);
}
__device__ __forceinline__ uint64_t wave_max_u64(uint64_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = umax64(v, shfl_xor_u64(v, o));
  return v;
}
// sums of this and lower lanes
__device__ __forceinline__ uint64_t wave_scan_u64(uint64_t v, int lane) {
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const uint32_t lo = __shfl_up((uint32_t)v, o, kWave), hi = __shfl_up((uint32_t)(v >> 32), o, kWave);
    v += lane >= o ? ((uint64_t)hi << 32) | lo : 0u;
  }
  return v;
}

// four tokens' logits from index i0 on; -inf past the vocabulary
template <typename T>
__device__ __forceinline__ void smp_logits(const Smp& d, const T* row, bool wide, int i0, float (&l)[4]) {
  if (wide && i0 + 4 <= d.V) {
    if constexpr (sizeof(T) == 2) {
      const uint2 x = *reinterpret_cast<const uint2*>(row + i0);
      l[0] = __uint_as_float(x.x << 16);
      l[1] = __uint_as_float(x.x & 0xffff0000u);
      l[2] = __uint_as_float(x.y << 16);
      l[3] = __uint_as_float(x.y & 0xffff0000u);
    } else {
      const floatx4 x = *reinterpret_cast<const floatx4*>(row + i0);
#pragma unroll
      for (int q = 0; q < 4; ++q) l[q] = x[q];
    }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) l[q] = i0 + q < d.V ? to_f32<T>(row[i0 + q]) : -INFINITY;
  }
}
template <typename T>
__device__ __forceinline__ void smp_load(const Smp& d, const T* row, bool wide, int i0,
                                         uint32_t (&key)[4]) {
  float l[4];
  smp_logits(d, row, wide, i0, l);
#pragma unroll
  for (int q = 0; q < 4; ++q) key[q] = smp_key(l[q]);
}

// the row's token and its log probability, Z the sum of the kept weights
template <typename T>
__device__ __forceinline__ void smp_out(const Smp& d, int64_t r, const T* row, const SmpRow& w, int id,
                                        uint64_t Z) {
  id = min(max(id, 0), d.V - 1);                   // an index of the row, whatever was found
  d.ids[r] = id;
  if (d.logprob)
    d.logprob[r] = (float)(w.x(smp_key(to_f32<T>(row[id]))) -
                           (log((double)Z) - 45.0 * 0.69314718055994531));
}

// ---------------------------------------------------------------------------
// The passes over the vocabulary.
// ---------------------------------------------------------------------------
struct SmpPlace {
  int64_t r, row;                    // the row in the batch, in the call
  int c0, c1;                        // its chunks
};
__device__ __forceinline__ SmpPlace smp_place(const Smp& d) {
  const int groups = (d.chunks + d.per_wg - 1) / d.per_wg;
  const int64_t r = blockIdx.x / groups;
  const int g = (int)(blockIdx.x - r * groups);
  return SmpPlace{r, d.row0 + r, g * d.per_wg, min((g + 1) * d.per_wg, d.chunks)};
}
// index of token q of the thread's i-th four in a chunk
__device__ __forceinline__ int smp_index(int chunk, int i) {
  return chunk * kSmpChunk + i * 4 * kSmpThreads + 4 * (int)threadIdx.x;
}
template <typename T>
__device__ __forceinline__ void smp_chunk(const Smp& d, const T* row, bool wide, int chunk,
                                          float (&l)[kSmpPer]) {
#pragma unroll
  for (int i = 0; i < kSmpPer / 4; ++i) {
    float x[4];
    smp_logits(d, row, wide, smp_index(chunk, i), x);
#pragma unroll
    for (int q = 0; q < 4; ++q) l[4 * i + q] = x[q];
  }
}
// the row's largest key and its lowest index, from the chunks' (every wave for itself)
__device__ __forceinline__ uint64_t smp_best(const Smp& d, int64_t r) {
  const int lane = threadIdx.x & 63;
  return wave_max_u64(lane < d.chunks ? d.best[r * kSmpChunks + lane] : 0u);
}

// The largest logit of every chunk; clears the row's histogram for the next launch.
template <typename T>
__global__ __launch_bounds__(kSmpThreads) void k_smp_max(const Smp d) {
  __shared__ uint64_t red[kSmpThreads / kWave];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const SmpPlace at = smp_place(d);
  const T* row = static_cast<const T*>(d.logits) + at.row * d.ld;
  const bool wide = reinterpret_cast<uintptr_t>(row) % (4 * sizeof(T)) == 0;
  if (at.c0 == 0 && d.temp != nullptr) {
    for (int b = tid; b < kSmpHist; b += kSmpThreads) d.hist[at.r * kSmpHist + b] = 0;
    if (tid == 0) d.rec[at.r] = SmpRec{};
  }
  for (int c = at.c0; c < at.c1; ++c) {
    float l[kSmpPer];
    smp_chunk(d, row, wide, c, l);
    float top = -INFINITY;
    int at_i = 0;
#pragma unroll
    for (int i = 0; i < kSmpPer; ++i) {            // indices ascend; NaN is never more
      const bool more = l[i] > top;
      top = more ? l[i] : top;
      at_i = more ? i : at_i;
    }
    const int idx = smp_index(c, at_i / 4) + at_i % 4;
    const uint64_t best = wave_max_u64(((uint64_t)smp_key(top) << 32) | (uint32_t)~idx);
    if (lane == 0) red[wave] = best;
    __syncthreads();
    if (tid == 0) {
      uint64_t x = red[0];
      for (int w = 1; w < kSmpThreads / kWave; ++w) x = umax64(x, red[w]);
      d.best[at.r * kSmpChunks + c] = x;
    }
    __syncthreads();
  }
}

// The weights: every chunk's sum where no threshold of l is to be found; else the row's
// histogram, of tokens where top-k decides and of weights for top-p alone.
template <typename T>
__global__ __launch_bounds__(kSmpThreads) void k_smp_mass(const Smp d) {
  __shared__ uint64_t hist[kSmpHist];
  __shared__ uint64_t red[kSmpThreads / kWave];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const SmpPlace at = smp_place(d);
  if (d.temp[at.row] == 0) return;
  const T* row = static_cast<const T*>(d.logits) + at.row * d.ld;
  const bool wide = reinterpret_cast<uintptr_t>(row) % (4 * sizeof(T)) == 0;
  float next[kSmpPer];                             // the next chunk's, on their way
  smp_chunk(d, row, wide, at.c0, next);
  const SmpSet set(d, at.row);
  const uint32_t top_key = (uint32_t)(smp_best(d, at.r) >> 32);
  if (top_key == 0u) return;
  const SmpRow w(set.t, top_key);
  const bool cuts = set.cuts(), tokens = set.k > 0;
  const double log_mp = set.log_min();
  for (int c = at.c0; c < at.c1; ++c) {
    float l[kSmpPer];
#pragma unroll
    for (int i = 0; i < kSmpPer; ++i) l[i] = next[i];
    if (c + 1 < at.c1) smp_chunk(d, row, wide, c + 1, next);
    if (!cuts) {
      uint64_t sum = 0;
#pragma unroll
      for (int i = 0; i < kSmpPer; ++i) {
        const double y = w.xl(l[i]);               // NaN for NaN: no weight
        sum += y >= log_mp ? w.weight_at(y) : 0u;
      }
      sum = wave_sum_u64(sum);
      if (lane == 0) red[wave] = sum;
      lds_barrier();
      if (tid == 0) {
        for (int x = 1; x < kSmpThreads / kWave; ++x) sum += red[x];
        d.sums[at.r * kSmpChunks + c] = sum;
      }
      lds_barrier();
      continue;
    }
    for (int b = tid; b < kSmpHist; b += kSmpThreads) hist[b] = 0;
    lds_barrier();
#pragma unroll
    for (int i = 0; i < kSmpPer; ++i) {
      const int b = w.bin(l[i]);
      if (b < kSmpHist)
        atomicAdd((unsigned long long*)&hist[b],
                  (unsigned long long)(tokens ? 1u : w.weight_at(w.xl(l[i]))));
    }
    lds_barrier();
    for (int b = tid; b < kSmpHist; b += kSmpThreads) {
      const uint64_t v = hist[b];
      if (v != 0u) atomicAdd((unsigned long long*)&d.hist[at.r * kSmpHist + b], (unsigned long long)v);
      if (!tokens) d.part[(at.r * kSmpChunks + c) * kSmpHist + b] = v;
    }
  }
}

// What the histogram says: the bin in which the threshold lies (whole workgroup, two bins
// a thread; by every wave for itself 0.7 us more).
struct SmpDecide {
  uint64_t red[kSmpThreads / kWave];
  SmpRec rec;
};
__device__ __forceinline__ SmpRec smp_decide(const Smp& d, int64_t r, const SmpSet& set, SmpDecide& s) {
  static_assert(kSmpHist == 2 * kSmpThreads, "two bins a thread");
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool by_k = set.k > 0;
  SmpRec x{};
  if (!set.bins()) {
    x.mode = kSmpSlow;
    return x;
  }
  const uint64_t* bins = d.hist + r * kSmpHist + 2 * tid;
  const uint64_t v[2] = {bins[0], bins[1]};
  uint64_t before = wave_scan_u64(v[0] + v[1], lane);
  if (lane == 63) s.red[wave] = before;
  if (tid == 0) {
    // where no bin reaches it, top-k leaves every token that has a weight: the bins' all, or
    // what top-p cuts of them
    x.mode = set.p >= 1.f ? kSmpEdge : kSmpSlow;
    x.edge = kSmpHist;
    s.rec = x;
  }
  lds_barrier();
  before -= v[0] + v[1];
  for (int w = 0; w < kSmpThreads / kWave; ++w) {
    x.all += s.red[w];
    before += w < wave ? s.red[w] : 0u;
  }
  const double want = (double)set.p * (double)x.all;
#pragma unroll
  for (int i = 0; i < 2; ++i) {                    // one bin of all hits
    const uint64_t upto = before + v[i];
    if (by_k ? before < (uint64_t)set.k && upto >= (uint64_t)set.k
             : (double)before < want && (double)upto >= want) {
      x.edge = 2 * tid + i;
      x.above = before;
      // top-p alone: whether the candidates are too many shows when they are counted
      x.mode = !by_k ? kSmpEdge
                     : (upto <= (uint64_t)kSmpCap ? kSmpList
                        : (v[i] <= (uint64_t)kSmpCap && set.p >= 1.f ? kSmpEdge : kSmpSlow));
      s.rec = x;
    }
    before = upto;
  }
  lds_barrier();
  return s.rec;
}

// Rows with a threshold of l: the candidates, and the sums of what stays before them.
template <typename T>
__global__ __launch_bounds__(kSmpThreads) void k_smp_list(const Smp d) {
  __shared__ uint64_t red[kSmpThreads / kWave];
  __shared__ uint32_t num[kSmpThreads / kWave], base;
  __shared__ SmpDecide dec;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const SmpPlace at = smp_place(d);
  if (d.temp[at.row] == 0) return;
  const SmpSet set(d, at.row);
  if (!set.cuts()) return;
  const T* row = static_cast<const T*>(d.logits) + at.row * d.ld;
  const bool wide = reinterpret_cast<uintptr_t>(row) % (4 * sizeof(T)) == 0;
  float next[kSmpPer];                             // the next chunk's, on their way
  smp_chunk(d, row, wide, at.c0, next);
  const uint32_t top_key = (uint32_t)(smp_best(d, at.r) >> 32);
  if (top_key == 0u) return;
  const SmpRec rec = smp_decide(d, at.r, set, dec);
  if (at.c0 == 0 && tid == 0) {
    SmpRec* to = d.rec + at.r;                     // rec.n counts meanwhile
    to->mode = rec.mode;
    to->edge = rec.edge;
    to->above = rec.above;
    to->all = rec.all;
  }
  if (rec.mode == kSmpSlow) return;
  const SmpRow w(set.t, top_key);
  const double log_mp = set.log_min();
  // the chunks' bins hold the weights before the edge, unless min-p may take some of them
  const bool held = set.k == 0 && !(set.mp > 0.f);
  for (int c = at.c0; c < at.c1; ++c) {
    float l[kSmpPer];
#pragma unroll
    for (int i = 0; i < kSmpPer; ++i) l[i] = next[i];
    if (c + 1 < at.c1) smp_chunk(d, row, wide, c + 1, next);
    uint64_t sum = 0;
    uint32_t pick = 0;                             // a bit a candidate
    if (rec.mode == kSmpEdge && held)
      for (int b = tid; b < rec.edge; b += kSmpThreads)
        sum += d.part[(at.r * kSmpChunks + c) * kSmpHist + b];
#pragma unroll
    for (int i = 0; i < kSmpPer; ++i) {
      const int b = w.bin(l[i]);
      const bool cand = rec.mode == kSmpList ? b <= rec.edge : b == rec.edge;
      pick |= cand && b < kSmpHist ? 1u << i : 0u;
      if (rec.mode == kSmpEdge && !held && b < rec.edge) {
        const double y = w.xl(l[i]);
        sum += y >= log_mp ? w.weight_at(y) : 0u;
      }
    }
    const uint32_t n = __popc(pick);
    uint32_t upto = n;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const uint32_t x = __shfl_up(upto, o, kWave);
      upto += lane >= o ? x : 0u;
    }
    sum = wave_sum_u64(sum);
    if (lane == 63) num[wave] = upto;
    if (lane == 0) red[wave] = sum;
    lds_barrier();
    if (tid == 0) {
      uint32_t all = 0;
      for (int x = 0; x < kSmpThreads / kWave; ++x) all += num[x];
      base = all != 0u ? atomicAdd(&d.rec[at.r].n, all) : 0u;
      for (int x = 1; x < kSmpThreads / kWave; ++x) sum += red[x];
      d.sums[at.r * kSmpChunks + c] = sum;
    }
    lds_barrier();
    uint32_t to = base + upto - n;
    for (int x = 0; x < wave; ++x) to += num[x];
#pragma unroll
    for (int i = 0; i < kSmpPer; ++i)
      if (((pick >> i) & 1u) && to < (uint32_t)kSmpCap)
        d.list[at.r * kSmpCap + to++] =
            ((uint64_t)smp_key(l[i]) << 32) | (uint32_t)(smp_index(c, i / 4) + i % 4);
    lds_barrier();
  }
}

// ---------------------------------------------------------------------------
// The last launch: thresholds and the draw, a workgroup a row.
// ---------------------------------------------------------------------------
struct RowShared {
  uint64_t bins[kRowBins];
  uint64_t part[kSmpChunks * kRowWaves];
  uint64_t red[kRowWaves];
  uint64_t out[4];
};

__device__ __forceinline__ uint64_t row_sum(RowShared& s, uint64_t v) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = wave_sum_u64(v);
  __syncthreads();                                 // the last sum's reads
  if (lane == 0) s.red[wave] = v;
  __syncthreads();
  v = 0;
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) v += s.red[w];
  return v;
}

__device__ __forceinline__ uint64_t row_max(RowShared& s, uint64_t v) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = wave_max_u64(v);
  __syncthreads();
  if (lane == 0) s.red[wave] = v;
  __syncthreads();
  for (int w = 0; w < kRowWaves; ++w) v = umax64(v, s.red[w]);
  return v;
}
// sum of this and lower threads' v; all: the workgroup's
__device__ __forceinline__ uint64_t row_scan(RowShared& s, uint64_t v, uint64_t& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t x = wave_scan_u64(v, lane);
  __syncthreads();
  if (lane == 63) s.red[wave] = x;
  __syncthreads();
  all = 0;
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) {
    x += w < wave ? s.red[w] : 0u;
    all += s.red[w];
  }
  return x;
}
// thread `at`'s x (whole workgroup)
__device__ __forceinline__ uint64_t row_get(RowShared& s, uint64_t x, int at) {
  __syncthreads();
  if ((int)threadIdx.x == at) s.out[2] = x;
  __syncthreads();
  return s.out[2];
}
// The threads' x in falling order, n of them at most other than 0: bitonic, in as many
// threads as n needs, within a wave by lane exchanges.
__device__ __forceinline__ uint64_t row_sort(RowShared& s, uint64_t x, int n) {
  const int tid = threadIdx.x;
  int size = kWave;
  while (size < n) size *= 2;
  for (int m = 2; m <= size; m *= 2)
    for (int o = m / 2; o > 0; o /= 2) {
      uint64_t y;
      if (o >= kWave) {                            // whole workgroup
        __syncthreads();
        s.bins[tid] = x;
        __syncthreads();
        y = s.bins[tid ^ o];
      } else {
        y = shfl_xor_u64(x, o);
      }
      const bool first = (tid & o) == 0, falls = (tid & m) == 0 || m == size;
      x = first == falls ? umax64(x, y) : (x < y ? x : y);
    }
  return tid < size ? x : 0u;
}

// The same of a wave's 64.
__device__ __forceinline__ uint64_t wave_sort(uint64_t x, int lane) {
#pragma unroll
  for (int m = 2; m <= kWave; m *= 2)
#pragma unroll
    for (int o = m / 2; o > 0; o /= 2) {
      const uint64_t y = shfl_xor_u64(x, o);
      const bool first = (lane & o) == 0, falls = (lane & m) == 0 || m == kWave;
      x = first == falls ? umax64(x, y) : (x < y ? x : y);
    }
  return x;
}

// The first of the bins, from the top one down, at which the sum passes.
template <typename F>
__device__ __forceinline__ int row_find(RowShared& s, F reach, uint64_t& before) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b0 = kRowBins - 1 - 2 * tid, b1 = b0 - 1;
  const uint64_t v0 = s.bins[b0], v1 = s.bins[b1];
  const uint64_t inc = wave_scan_u64(v0 + v1, lane);
  if (lane == 63) s.red[wave] = inc;
  if (tid == 0) s.out[0] = ~0ull;
  __syncthreads();
  uint64_t x = inc - v0 - v1;
  for (int w = 0; w < wave; ++w) x += s.red[w];
  if (v0 > 0 && !reach(x) && reach(x + v0)) {
    s.out[0] = b0;
    s.out[1] = x;
  } else if (v1 > 0 && !reach(x + v0) && reach(x + v0 + v1)) {
    s.out[0] = b1;
    s.out[1] = x + v0;
  }
  __syncthreads();
  const int bin = (int)s.out[0];
  before = s.out[1];
  return bin;
}

// Radix selection among keys of so many bits, 11 a round: the key at which the sum of
// values, from the largest key down, passes; what lies before it, and at it alone (0
// where it never does).  each(f) calls f(key, value) for the thread's elements.
template <typename E, typename F>
__device__ __forceinline__ uint32_t row_select(RowShared& s, int bits, E each, F reach,
                                               uint64_t& before, uint64_t& at) {
  uint32_t prefix = 0, mask = 0;
  before = 0;
  at = 0;
  for (int shift = bits > 11 ? bits - 11 : 0;; shift = shift > 11 ? shift - 11 : 0) {
    // the round's bits: those below the ones that are known
    const uint32_t field = ~mask & ((bits < 32 ? 1u << bits : 0u) - 1u) & ~((1u << shift) - 1u);
    __syncthreads();
    for (int b = threadIdx.x; b < kRowBins; b += kRowThreads) s.bins[b] = 0;
    __syncthreads();
    each([&](uint32_t key, uint64_t v) {
      if ((key & mask) == prefix && v != 0u)
        atomicAdd((unsigned long long*)&s.bins[(key & field) >> shift], (unsigned long long)v);
    });
    __syncthreads();
    uint64_t in;
    const uint64_t base = before;
    const int bin = row_find(s, [&](uint64_t x) { return reach(base + x); }, in);
    if (bin < 0) {                                 // whole workgroup
      at = 0;
      return 0u;
    }
    before = base + in;
    at = s.bins[bin];
    prefix |= (uint32_t)bin << shift;
    mask |= field;
    if (shift == 0) return prefix;
  }
}

// How many of n equal weights stay where the sum reaches `want` among them: those before
// which less lies.
__device__ __forceinline__ uint64_t row_ties(double want, uint64_t before, uint64_t each, uint64_t n) {
  uint64_t c = (uint64_t)fmax((want - (double)before) / (double)each, 0.0);
  c = c < n ? c : n;
  while (c > 0 && (double)(before + (c - 1) * each) >= want) --c;
  while (c < n && (double)(before + c * each) < want) ++c;
  return c;
}

constexpr uint32_t kIndexTop = kSmpMaxV - 1;        // indices in falling order: kIndexTop - i

// The draw from the chunks' sums: the chunk in which they pass u times their sum, and
// the token within it; kept(key, index) is a token's weight.  The last token with a
// weight where none passes.
template <typename T, typename K>
__device__ __forceinline__ void row_draw(const Smp& d, RowShared& s, int64_t r, const T* row, bool wide,
                                         const SmpRow& w, const uint64_t* sums, K kept) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint64_t mine = lane < d.chunks ? sums[lane] : 0u;
  const uint64_t upto = wave_scan_u64(mine, lane);
  const uint64_t Z = shfl_u64(upto, 63);
  const double goal = smp_goal(d, r, Z);
  auto over = [&](uint64_t x) { return (double)x > goal; };
  const uint64_t hit = __ballot(mine > 0 && over(upto)), some = __ballot(mine > 0);
  const bool none = hit == 0;                      // u is no number below 1
  const int c = none ? 63 - __builtin_clzll(some | 1u) : __builtin_ctzll(hit);
  const uint64_t b = upto - mine;
  const uint64_t before = shfl_u64(b, c);
  const int i0 = c * kSmpChunk + 4 * tid;
  uint32_t key[4];
  uint64_t wt[4], n = 0;
  smp_load(d, row, wide, i0, key);
#pragma unroll
  for (int q = 0; q < 4; ++q) n += wt[q] = kept(key[q], i0 + q);
  const uint64_t inc = wave_scan_u64(n, lane);
  __syncthreads();
  if (lane == 63) s.red[wave] = inc;
  __syncthreads();
  uint64_t x = before + inc - n;
  for (int v = 0; v < wave; ++v) x += s.red[v];
  int pick = -1;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const bool was = over(x);
    x += wt[q];
    // the one token at which the sum passes; else the last of this thread's
    if (wt[q] > 0 && (none || (!was && over(x)))) pick = i0 + q;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) pick = max(pick, __shfl_xor(pick, o, kWave));
  __syncthreads();
  if (lane == 0) s.red[wave] = (uint32_t)pick;
  __syncthreads();
  if (tid == 0) {
    for (int v = 0; v < kRowWaves; ++v) pick = max(pick, (int)(uint32_t)s.red[v]);
    smp_out(d, r, row, w, pick, Z);
  }
}

// Rows with more candidates than the list holds (many equal logits, or top-k of tens of
// thousands with top-p), with top-p where fewer than k tokens have a weight (within 32 T of
// the largest logit: peaked rows), or a temperature past the bins' fp32: radix selection over
// the row, which one workgroup walks about eight times.
template <typename T>
__device__ __forceinline__ void row_slow(const Smp& d, RowShared& s, int64_t r, const T* row, bool wide,
                                      const SmpRow& w, const SmpSet& set) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto walk = [&](auto f) {
    for (int c = 0; c < d.chunks; ++c) {
      uint32_t key[4];
      smp_load(d, row, wide, c * kSmpChunk + 4 * tid, key);
#pragma unroll
      for (int q = 0; q < 4; ++q) f(c, c * kSmpChunk + 4 * tid + q, key[q]);
    }
  };
  uint32_t cut = 1u;                               // keys from here on stay
  uint32_t tie_end = ~0u;                          // of those at the cut, indices before this one
  uint64_t before, at;
  if (set.k > 0)
    cut = max(cut, row_select(s, 32, [&](auto f) {
            walk([&](int, int, uint32_t key) { f(key, key != 0u ? 1u : 0u); });
          }, [&](uint64_t x) { return x >= (uint64_t)set.k; }, before, at));
  if (set.p < 1.f) {
    uint64_t sum = 0;                              // of what top-k left
    walk([&](int, int, uint32_t key) { sum += key >= cut ? w.weight(key) : 0u; });
    sum = row_sum(s, sum);
    const double want = (double)set.p * (double)sum;
    const uint32_t key = row_select(s, 32, [&](auto f) {
      walk([&](int, int, uint32_t key) {
        if (key >= cut) f(key, w.weight(key));
      });
    }, [&](uint64_t x) { return (double)x >= want; }, before, at);
    if (key != 0u) {
      cut = key;
      const uint64_t one = w.weight(key), n = at / one, stay = row_ties(want, before, one, n);
      if (stay < n)
        tie_end = kIndexTop + 1 - row_select(s, 18, [&](auto f) {
          walk([&](int, int i, uint32_t key) {
            if (key == cut) f(kIndexTop - (uint32_t)i, 1u);
          });
        }, [&](uint64_t x) { return x >= stay; }, before, at);
    }
  }
  const double log_mp = set.log_min();
  auto kept = [&](uint32_t key, int i) -> uint64_t {
    if (key < cut || (key == cut && (uint32_t)i >= tie_end)) return 0u;
    return w.x(key) >= log_mp ? w.weight(key) : 0u;
  };
  for (int c = 0; c < d.chunks; ++c) {
    uint32_t key[4];
    const int i0 = c * kSmpChunk + 4 * tid;
    smp_load(d, row, wide, i0, key);
    uint64_t sum = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) sum += kept(key[q], i0 + q);
    sum = wave_sum_u64(sum);
    if (lane == 0) s.part[c * kRowWaves + wave] = sum;
  }
  __syncthreads();
  if (wave == 0) {
    uint64_t sum = 0;
    if (lane < d.chunks)
      for (int v = 0; v < kRowWaves; ++v) sum += s.part[lane * kRowWaves + v];
    s.bins[lane] = sum;
  }
  __syncthreads();
  row_draw(d, s, r, row, wide, w, s.bins, kept);
}

template <typename T>
__global__ __launch_bounds__(kRowThreads) void k_smp_row(const Smp d) {
  __shared__ RowShared s;
  __shared__ uint64_t cand[kSmpCap];               // key, index; 0: none
  const int tid = threadIdx.x;
  const int64_t rb = blockIdx.x, r = d.row0 + rb;
  const uint64_t best = smp_best(d, rb);
  const uint32_t top_key = (uint32_t)(best >> 32);
  const bool sampled = d.temp != nullptr && d.temp[r] != 0;
  if (top_key == 0u || !sampled) {                 // whole workgroup
    if (tid == 0) {
      d.ids[r] = top_key == 0u ? -1 : (int)~(uint32_t)best;
      if (d.logprob) d.logprob[r] = top_key == 0u ? -INFINITY : 0.f;
      if (top_key == 0u) atomicOr(d.err, XP_DEVERR_EMPTY);
    }
    return;
  }
  const T* row = static_cast<const T*>(d.logits) + r * d.ld;
  const bool wide = reinterpret_cast<uintptr_t>(row) % (4 * sizeof(T)) == 0;
  const SmpSet set(d, r);
  if (set.bad && tid == 0) atomicOr(d.err, set.bad);
  const SmpRow w(set.t, top_key);
  const double log_mp = set.log_min();
  const uint64_t* sums = d.sums + rb * kSmpChunks;
  auto heavy = [&](uint32_t key) -> uint64_t { return w.x(key) >= log_mp ? w.weight(key) : 0u; };
  if (!set.cuts()) {
    row_draw(d, s, r, row, wide, w, sums,
             [&](uint32_t key, int) -> uint64_t { return key != 0u ? heavy(key) : 0u; });
    return;
  }
  const SmpRec rec = d.rec[rb];
  if (rec.mode == kSmpSlow || rec.n > (uint32_t)kSmpCap) {
    row_slow(d, s, r, row, wide, w, set);
    return;
  }
  // ---- the candidates that stay: down to the key `cut`, of those at it the ones whose
  // index lies before tie_end ----
  const int n = (int)rec.n;
  const uint64_t* list = d.list + rb * kSmpCap;
  // the edge's bin lies behind tokens that stay; a list begins at the top
  const uint64_t num_above = rec.mode == kSmpEdge && set.k > 0 ? rec.above : 0u;
  const uint64_t mass_above = rec.mode == kSmpEdge && set.k == 0 ? rec.above : 0u;
  uint32_t cut = 1u, tie_end = ~0u;
  auto kept = [&](uint32_t k, uint32_t i) { return !(k < cut || (k == cut && i >= tie_end)); };
  auto stays = [&](uint32_t k, uint32_t i) -> uint64_t { return kept(k, i) ? heavy(k) : 0u; };
  if (rec.mode == kSmpList && n <= kWave) {
    // a wave has them all, and needs no barrier (12 -> 5.2 us): top-k decides, as in every list
    if (tid >= kWave) return;
    uint64_t x = tid < n ? list[tid] : 0u;
    x = wave_sort(x != 0u ? (x & ~0xffffffffull) | (uint32_t)~(uint32_t)x : 0u, tid);
    const uint32_t key = (uint32_t)(x >> 32), idx = ~(uint32_t)x;
    const uint32_t kth = set.k <= n ? __shfl(key, set.k - 1, kWave) : 1u;
    bool in = key != 0u && key >= kth;             // what ties with the k-th stays
    const uint64_t v = in ? w.weight(key) : 0u;
    uint64_t upto = wave_scan_u64(v, tid);
    const double want = (double)set.p * (double)shfl_u64(upto, 63);
    in = in && (set.p >= 1.f || (double)(upto - v) < want) && w.x(key) >= log_mp;
    // by index, the lowest first
    x = wave_sort(in ? ((uint64_t)(kIndexTop + 1 - idx) << 32) | key : 0u, tid);
    const uint64_t mine = x != 0u ? w.weight((uint32_t)x) : 0u;
    upto = wave_scan_u64(mine, tid);
    const uint64_t Z = shfl_u64(upto, 63);
    const double goal = smp_goal(d, r, Z);
    const bool none = !((double)Z > goal);
    const bool hit = mine > 0 && (none ? upto == Z : (double)upto > goal && !((double)(upto - mine) > goal));
    if (hit) smp_out(d, r, row, w, (int)(kIndexTop + 1 - (uint32_t)(x >> 32)), Z);
    return;
  }
  // In order, a thread each, what lies before a candidate is a prefix sum: two sorts, where
  // radix selection takes two rounds for every threshold and two for the draw.  64 rows of
  // 200 candidates 17 us against 19, of 400 20.5 against 19, of 800 24.5 against 20; with
  // both thresholds 25.8 against 28.9.
  if (n <= (set.k > 0 && set.p < 1.f ? kRowThreads : kRowThreads / 4)) {
    uint64_t x = tid < n ? list[tid] : 0u;
    x = row_sort(s, x != 0u ? (x & ~0xffffffffull) | (uint32_t)~(uint32_t)x : 0u, n);
    const uint32_t key = (uint32_t)(x >> 32), idx = ~(uint32_t)x;
    bool in = key != 0u;
    if (set.k > 0) {
      const int64_t last = set.k - 1 - (int64_t)num_above;   // of the k, among the candidates
      const uint32_t kth = last < n ? (uint32_t)(row_get(s, x, (int)last) >> 32) : 1u;
      in = in && key >= kth;                       // what ties with it stays
    }
    const uint64_t v = in ? w.weight(key) : 0u;
    if (set.p < 1.f) {
      uint64_t sum;
      const uint64_t upto = row_scan(s, v, sum);
      sum = set.k > 0 ? sum : rec.all;             // what top-k leaves
      in = in && (double)(mass_above + upto - v) < (double)set.p * (double)sum;
    }
    const int stay = (int)row_sum(s, in ? 1u : 0u);
    if (rec.mode == kSmpList) {
      // the draw among them: by index, the lowest first
      const bool take = in && w.x(key) >= log_mp;
      x = row_sort(s, take ? ((uint64_t)(kIndexTop + 1 - idx) << 32) | key : 0u, n);
      const uint64_t mine = x != 0u ? w.weight((uint32_t)x) : 0u;
      uint64_t Z;
      const uint64_t upto = row_scan(s, mine, Z);
      const double goal = smp_goal(d, r, Z);
      const bool none = !((double)Z > goal);       // the last one with a weight then
      const bool hit = mine > 0 && (none ? upto == Z : (double)upto > goal && !((double)(upto - mine) > goal));
      if (hit) smp_out(d, r, row, w, (int)(kIndexTop + 1 - (uint32_t)(x >> 32)), Z);
      return;
    }
    if (stay > 0) {
      const uint64_t y = row_get(s, x, stay - 1);
      cut = (uint32_t)(y >> 32);
      tie_end = ~(uint32_t)y + 1;
    } else {
      cut = ~0u;                                   // no candidate stays
    }
  } else {
    uint32_t hi = 0, lo = ~0u;
    for (int i = tid; i < n; i += kRowThreads) {   // its own ones from here on
      const uint64_t x = list[i];
      cand[i] = x;
      hi = max(hi, (uint32_t)(x >> 32));
      lo = min(lo, (uint32_t)(x >> 32));
    }
    // the bits in which the keys differ
    hi = (uint32_t)row_max(s, hi);
    lo = ~(uint32_t)row_max(s, (uint32_t)~lo);
    const int bits = hi > lo ? 32 - __builtin_clz(hi - lo) : 1;
    auto each = [&](auto f) {
      for (int i = tid; i < n; i += kRowThreads) f((uint32_t)(cand[i] >> 32), (uint32_t)cand[i]);
    };
    uint64_t before, at, sum = rec.all;            // what top-k leaves
    if (set.k > 0) {
      const uint32_t x = row_select(s, bits, [&](auto f) {
        each([&](uint32_t k, uint32_t) { f(k - lo, 1u); });
      }, [&](uint64_t x) { return num_above + x >= (uint64_t)set.k; }, before, at);
      if (at != 0u) cut = lo + x;
      sum = 0;
      each([&](uint32_t k, uint32_t) { sum += k >= cut ? w.weight(k) : 0u; });
      sum = row_sum(s, sum);
    }
    if (set.p < 1.f) {
      const double want = (double)set.p * (double)sum;
      const uint32_t x = row_select(s, bits, [&](auto f) {
        each([&](uint32_t k, uint32_t) {
          if (k >= cut) f(k - lo, w.weight(k));
        });
      }, [&](uint64_t x) { return (double)(mass_above + x) >= want; }, before, at);
      if (at != 0u) {
        cut = lo + x;
        const uint64_t one = w.weight(cut), m = at / one;
        const uint64_t stay = row_ties(want, mass_above + before, one, m);
        if (stay < m)
          tie_end = kIndexTop + 1 - row_select(s, 18, [&](auto f) {
            each([&](uint32_t k, uint32_t i) {
              if (k == cut) f(kIndexTop - i, 1u);
            });
          }, [&](uint64_t x) { return x >= stay; }, before, at);
      }
    }
    if (rec.mode == kSmpList) {
      uint64_t Z = 0;
      each([&](uint32_t k, uint32_t i) { Z += stays(k, i); });
      Z = row_sum(s, Z);
      const double goal = smp_goal(d, r, Z);
      // a sum that is to exceed the goal, or, where none does, to be whole
      const bool none = !((double)Z > goal);
      const uint32_t x = row_select(s, 18, [&](auto f) {
        each([&](uint32_t k, uint32_t i) { f(kIndexTop - i, stays(k, i)); });
      }, [&](uint64_t x) { return none ? x >= Z : (double)x > goal; }, before, at);
      if (tid == 0) smp_out(d, r, row, w, (int)(kIndexTop - x), Z);
      return;
    }
  }
  // ---- the chunks' sums with the candidates that stay, and the draw ----
  __syncthreads();
  if (tid < kSmpChunks) s.bins[tid] = tid < d.chunks ? sums[tid] : 0u;
  __syncthreads();
  for (int i = tid; i < n; i += kRowThreads) {
    const uint64_t x = list[i], v = stays((uint32_t)(x >> 32), (uint32_t)x);
    if (v != 0u)
      atomicAdd((unsigned long long*)&s.bins[(uint32_t)x / kSmpChunk], (unsigned long long)v);
  }
  __syncthreads();
  row_draw(d, s, r, row, wide, w, s.bins, [&](uint32_t k, int i) -> uint64_t {
    const int b = w.bin(smp_value(k));
    return b < kSmpHist && (b < rec.edge || (b == rec.edge && kept(k, (uint32_t)i))) ? heavy(k) : 0u;
  });
}

__global__ void k_smp_clear_err(uint32_t* err) {
  if (threadIdx.x == 0) *err = 0u;
}

template <typename T>
static hipError_t launch_sample(Smp d, int rows, int cus, hipStream_t st) {
  // as many chunks a workgroup as leave four workgroups a CU: 64 rows of 38 chunks in 1216
  // workgroups of two took 7 + 18 + 15 us, of one 7 + 18 + 18, in 832 of three 8 + 21 + 18
  d.per_wg = std::max(1, std::min(d.chunks, rows * d.chunks / (4 * cus)));
  const dim3 grid(rows * ((d.chunks + d.per_wg - 1) / d.per_wg)), block(kSmpThreads);
  hipError_t e;
  hipLaunchKernelGGL(k_smp_max<T>, grid, block, 0, st, d);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (d.temp != nullptr) {
    hipLaunchKernelGGL(k_smp_mass<T>, grid, block, 0, st, d);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (d.top_k != nullptr || d.top_p != nullptr) {
      hipLaunchKernelGGL(k_smp_list<T>, grid, block, 0, st, d);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  hipLaunchKernelGGL(k_smp_row<T>, dim3(rows), dim3(kRowThreads), 0, st, d);
  return hipGetLastError();
}

}  // namespace xp

using namespace xp;

struct xp_sampler {
  int device = 0, cus = 0, V = 0, max_rows = 0;
  void* ws = nullptr;
  Smp d{};                           // the workspace's slices
  std::string msg;
};

// Message of the last failed xp_sampler_create of this thread.
static thread_local std::string g_smp_err;

static xp_status smp_fail(xp_sampler* s, xp_status st, const char* fmt, ...)
    __attribute__((format(printf, 3, 4)));
static xp_status smp_fail(xp_sampler* s, xp_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  (s ? s->msg : g_smp_err) = buf;
  return st;
}

extern "C" const char* xp_sampler_last_error(const xp_sampler* s) {
  return s ? s->msg.c_str() : g_smp_err.c_str();
}

extern "C" xp_status xp_sampler_create(int32_t V, int32_t max_rows, xp_sampler** out) {
  g_smp_err.clear();
  if (out == nullptr) return smp_fail(nullptr, XP_EINVAL, "out is NULL");
  *out = nullptr;
  if (V < 1 || max_rows < 1 || max_rows > 65536)
    return smp_fail(nullptr, XP_EINVAL, "V=%d (>= 1) or max_rows=%d (1..65536) out of range", V, max_rows);
  if (V > kSmpMaxV) return smp_fail(nullptr, XP_EUNSUPPORTED, "V=%d is not built (up to 2^18)", V);
  xp_sampler* s = new (std::nothrow) xp_sampler();
  if (s == nullptr) return smp_fail(nullptr, XP_ENOMEM, "host allocation failed");
  s->V = V;
  s->max_rows = max_rows;
  hipError_t e = hipGetDevice(&s->device);
  if (e == hipSuccess)
    e = hipDeviceGetAttribute(&s->cus, hipDeviceAttributeMultiprocessorCount, s->device);
  if (e != hipSuccess) {
    delete s;
    return smp_fail(nullptr, XP_EHIP, "device query failed: %s", hipGetErrorString(e));
  }
  s->cus = s->cus > 0 ? s->cus : 256;
  const size_t nb = (size_t)std::min(max_rows, kSmpBatch);
  struct Slice { void** at; size_t bytes; };
  const Slice slices[] = {
      {(void**)&s->d.err, 256},
      {(void**)&s->d.best, nb * kSmpChunks * 8},
      {(void**)&s->d.sums, nb * kSmpChunks * 8},
      {(void**)&s->d.hist, nb * kSmpHist * 8},
      {(void**)&s->d.part, nb * kSmpChunks * kSmpHist * 8},
      {(void**)&s->d.rec, nb * sizeof(SmpRec)},
      {(void**)&s->d.list, nb * kSmpCap * 8},
  };
  size_t total = 0;
  for (const Slice& sl : slices) total += (sl.bytes + 255) / 256 * 256;
  e = hipMalloc(&s->ws, total);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    delete s;
    return smp_fail(nullptr, XP_ENOMEM, "workspace of %zu bytes: %s", total, hipGetErrorString(e));
  }
  char* at = static_cast<char*>(s->ws);
  for (const Slice& sl : slices) {
    *sl.at = at;
    at += (sl.bytes + 255) / 256 * 256;
  }
  e = hipMemset(s->ws, 0, 256);                    // the device error word
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e != hipSuccess) {
    (void)hipFree(s->ws);
    delete s;
    return smp_fail(nullptr, XP_EHIP, "workspace: %s", hipGetErrorString(e));
  }
  *out = s;
  return XP_OK;
}

extern "C" void xp_sampler_destroy(xp_sampler* s) {
  if (s == nullptr) return;
  (void)hipDeviceSynchronize();
  if (s->ws) (void)hipFree(s->ws);
  delete s;
}

static xp_status smp_device(xp_sampler* s) {
  int dev = -1;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return smp_fail(s, XP_EHIP, "device query failed: %s", hipGetErrorString(e));
  if (dev != s->device)
    return smp_fail(s, XP_EINVAL, "the current device is %d, the sampler's %d", dev, s->device);
  return XP_OK;
}

extern "C" xp_status xp_sample(xp_sampler* s, int32_t rows, int32_t dtype, const void* logits,
                               int64_t ld, const uint8_t* temp, const float* temperature,
                               const int32_t* top_k, const float* top_p, const float* min_p,
                               const float* u, int32_t* out_ids, float* out_logprob,
                               void* stream) {
  if (s == nullptr) return XP_EINVAL;
  if (rows < 0 || rows > s->max_rows)
    return smp_fail(s, XP_EINVAL, "rows=%d out of range 0..%d", rows, s->max_rows);
  if (dtype != XP_F32 && dtype != XP_BF16)
    return smp_fail(s, XP_EINVAL, "dtype %d is not XP_F32 or XP_BF16", dtype);
  const size_t es = dtype == XP_F32 ? 4 : 2;
  if (logits == nullptr || out_ids == nullptr || reinterpret_cast<uintptr_t>(logits) % es != 0 ||
      ld < s->V)
    return smp_fail(s, XP_EINVAL, "logits (aligned to its type) and out_ids are required, ld=%lld at "
                    "least V=%d", (long long)ld, s->V);
  if (temp == nullptr && (temperature || top_k || top_p || min_p))
    return smp_fail(s, XP_EINVAL, "temperature, top_k, top_p and min_p need temp");
  if ((temp != nullptr) != (u != nullptr))
    return smp_fail(s, XP_EINVAL, "u is required with temp, and only with it");
  const xp_status ds = smp_device(s);
  if (ds != XP_OK || rows == 0) return ds;
  Smp d = s->d;
  d.logits = logits;
  d.ld = ld;
  d.V = s->V;
  d.temp = temp;
  d.temperature = temperature;
  d.top_k = top_k;
  d.top_p = top_p;
  d.min_p = min_p;
  d.u = u;
  d.ids = out_ids;
  d.logprob = out_logprob;
  d.chunks = (s->V + kSmpChunk - 1) / kSmpChunk;
  hipError_t e = hipSuccess;
  for (int32_t r0 = 0; r0 < rows && e == hipSuccess; r0 += kSmpBatch) {
    d.row0 = r0;
    const int n = std::min(rows - r0, (int32_t)kSmpBatch);
    e = dtype == XP_F32 ? launch_sample<float>(d, n, s->cus, (hipStream_t)stream)
                        : launch_sample<uint16_t>(d, n, s->cus, (hipStream_t)stream);
  }
  if (e != hipSuccess) return smp_fail(s, XP_EHIP, "launch failed: %s", hipGetErrorString(e));
  return XP_OK;
}

extern "C" xp_status xp_sampler_device_errors(xp_sampler* s, uint32_t* out, void* stream) {
  if (s == nullptr) return XP_EINVAL;
  if (out == nullptr) return smp_fail(s, XP_EINVAL, "out is NULL");
  const xp_status ds = smp_device(s);
  if (ds != XP_OK) return ds;
  hipStream_t st = (hipStream_t)stream;
  hipError_t e = hipMemcpyAsync(out, s->d.err, sizeof(uint32_t), hipMemcpyDeviceToHost, st);
  if (e == hipSuccess) {
    hipLaunchKernelGGL(k_smp_clear_err, dim3(1), dim3(64), 0, st, s->d.err);
    e = hipGetLastError();
  }
  if (e == hipSuccess) e = hipStreamSynchronize(st);
  if (e != hipSuccess) return smp_fail(s, XP_EHIP, "device errors: %s", hipGetErrorString(e));
  return XP_OK;
}
