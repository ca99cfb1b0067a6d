// Tokens from logits: temperature, top-k, top-p and min-p, from given uniforms.
//
// With m = max l, the weight of token v is e^{(l_v - m) / T}.  Top-k and top-p keep
// what lies above a threshold of l (top-p also cuts through equal logits, lowest index
// first), min-p what is heavy enough, and the sample is the first token in index order
// with sum of the kept weights up to it > u times their sum.
//
// A sample hangs on where u falls between sums over the vocabulary, so the weights are
// formed in 64 bits and then held as integers, 2^45 for the largest: sums of up to 2^18
// of them fit 63 bits and are exact, the same whatever their order, and of any two sums
// that are compared neither is rounded.  What 2^-46 of the largest weight can move is
// far below the 2^-24 by which uniforms differ.
#include <stdarg.h>
#include <stdio.h>

#include <new>
#include <string>

#include "xp_internal.h"

namespace xp {

constexpr int kSmpMaxV = 1 << 18;
constexpr int kSmpThreads = 1024;
constexpr int kSmpWaves = kSmpThreads / kWave;
constexpr int kSmpSeg = kSmpThreads * 4;           // tokens of a segment, 4 a thread
constexpr int kSmpSegs = kSmpMaxV / kSmpSeg;
constexpr int kSmpBins = 2048;

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
  __device__ __forceinline__ double x(uint32_t key) const {
    return key == top_key ? 0.0 : ((double)smp_value(key) - top) * inv_t;
  }
  __device__ __forceinline__ uint64_t weight(uint32_t key) const {
    if (key == 0u) return 0u;
    const double y = x(key);
    return y > -32.0 ? (uint64_t)rint(exp(y) * 0x1p45) : 0u;
  }
};

__device__ __forceinline__ uint64_t wave_sum_u64(uint64_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += shfl_xor_u64(v, o);
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

// four tokens' keys from index i0 on; 0 past the vocabulary
template <typename T>
__device__ __forceinline__ void smp_load(const Smp& d, const T* row, bool wide, int i0,
                                         uint32_t (&key)[4]) {
  float l[4];
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
#pragma unroll
  for (int q = 0; q < 4; ++q) key[q] = smp_key(l[q]);
}

struct SmpShared {
  uint64_t mass[kSmpBins];
  uint32_t count[kSmpBins];
  uint64_t part[kSmpSegs * kSmpWaves];
  uint64_t red[kSmpWaves + 1];
  uint64_t out[4];
};

// What a radix round finds, counted from the largest key down: the bin in which
// `before + bin` reaches the target, and what lies before it.
struct SmpBin {
  int bin;
  uint64_t before;
};
// the first bin from the top at which the sum passes: reach(before, upto)
template <typename F>
__device__ __forceinline__ SmpBin smp_find(SmpShared& s, const uint64_t* val64, const uint32_t* val32,
                                           F reach) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b0 = kSmpBins - 1 - 2 * tid, b1 = b0 - 1;
  const uint64_t v0 = val64 ? val64[b0] : val32[b0], v1 = val64 ? val64[b1] : val32[b1];
  const uint64_t inc = wave_scan_u64(v0 + v1, lane);
  if (lane == 63) s.red[wave] = inc;
  if (tid == 0) {
    s.out[0] = ~0ull;
    s.out[1] = 0;
  }
  __syncthreads();
  uint64_t before = inc - v0 - v1;
  for (int w = 0; w < wave; ++w) before += s.red[w];
  const bool at0 = v0 > 0 && !reach(before) && reach(before + v0);
  const bool at1 = v1 > 0 && !reach(before + v0) && reach(before + v0 + v1);
  if (at0) {
    s.out[0] = b0;
    s.out[1] = before;
  } else if (at1) {
    s.out[0] = b1;
    s.out[1] = before + v0;
  }
  __syncthreads();
  const SmpBin r{(int)s.out[0], s.out[1]};
  __syncthreads();
  return r;
}

// A row by one workgroup.  Thresholds by radix selection on the keys, 11 bits a round.
template <typename T>
__global__ __launch_bounds__(kSmpThreads) void k_sample_row(const Smp d) {
  __shared__ SmpShared s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t r = blockIdx.x;
  const T* row = static_cast<const T*>(d.logits) + r * d.ld;
  const bool wide = reinterpret_cast<uintptr_t>(row) % (4 * sizeof(T)) == 0;
  const int segs = (d.V + kSmpSeg - 1) / kSmpSeg;
  // ---- the largest logit, lowest index first ----
  uint64_t best = 0;
  for (int g = 0; g < segs; ++g) {
    const int i0 = g * kSmpSeg + 4 * tid;
    uint32_t key[4];
    smp_load(d, row, wide, i0, key);
#pragma unroll
    for (int q = 0; q < 4; ++q) best = umax64(best, ((uint64_t)key[q] << 32) | (uint32_t)~(i0 + q));
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) best = umax64(best, shfl_xor_u64(best, o));
  if (lane == 0) s.red[wave] = best;
  __syncthreads();
  for (int w = 0; w < kSmpWaves; ++w) best = umax64(best, s.red[w]);
  __syncthreads();
  const uint32_t top_key = (uint32_t)(best >> 32);
  const bool sampled = d.temp != nullptr && d.temp[r] != 0;
  if (top_key == 0u || !sampled) {
    if (tid == 0) {
      d.ids[r] = top_key == 0u ? -1 : (int)~(uint32_t)best;
      if (d.logprob) d.logprob[r] = top_key == 0u ? -INFINITY : 0.f;
      if (top_key == 0u) atomicOr(d.err, XP_DEVERR_EMPTY);
    }
    return;
  }
  // ---- the row's settings ----
  uint32_t bad = 0;
  float t = d.temperature ? d.temperature[r] : 1.f;
  if (!(t > 0.f && t < INFINITY)) {
    bad |= XP_DEVERR_TEMPERATURE;
    t = 1.f;
  }
  int k = d.top_k ? d.top_k[r] : 0;
  float p = d.top_p ? d.top_p[r] : 1.f, mp = d.min_p ? d.min_p[r] : 0.f;
  if (k < 0) {
    bad |= XP_DEVERR_FILTER;
    k = 0;
  }
  if (!(p > 0.f)) {
    bad |= XP_DEVERR_FILTER;
    p = 1.f;
  }
  if (!(mp >= 0.f && mp <= 1.f)) {
    bad |= XP_DEVERR_FILTER;
    mp = 0.f;
  }
  if (bad && tid == 0) atomicOr(d.err, bad);
  const SmpRow w{1.0 / (double)t, (double)smp_value(top_key), top_key};
  const double log_mp = mp > 0.f ? log((double)mp) : -INFINITY;
  // one radix selection; lo: keys below do not count.  Returns the key at which the sum
  // passes, what lies before it, and the sum at that key alone.
  auto select = [&](bool by_mass, uint32_t lo, auto reach, uint64_t& before, uint64_t& at) {
    uint32_t prefix = 0, mask = 0;
    before = 0;
    for (int shift = 21; shift >= 0; shift = shift == 21 ? 10 : (shift == 10 ? 0 : -1)) {
      const uint32_t field = shift == 0 ? 1023u : 2047u;
      for (int b = tid; b < kSmpBins; b += kSmpThreads) {
        s.mass[b] = 0;
        s.count[b] = 0;
      }
      __syncthreads();
      for (int g = 0; g < segs; ++g) {
        uint32_t key[4];
        smp_load(d, row, wide, g * kSmpSeg + 4 * tid, key);
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (key[q] != 0u && key[q] >= lo && (key[q] & mask) == prefix) {
            const uint32_t b = (key[q] >> shift) & field;
            if (by_mass) atomicAdd((unsigned long long*)&s.mass[b], (unsigned long long)w.weight(key[q]));
            else atomicAdd(&s.count[b], 1u);
          }
      }
      __syncthreads();
      const uint64_t base = before;
      const SmpBin f = smp_find(s, by_mass ? s.mass : nullptr, s.count,
                                [&](uint64_t x) { return reach(base + x); });
      if (f.bin < 0) return 0u;                    // the sum never passes: all keys count
      before = base + f.before;
      at = by_mass ? s.mass[f.bin] : s.count[f.bin];
      prefix |= (uint32_t)f.bin << shift;
      mask |= field << shift;
      __syncthreads();
    }
    return prefix;
  };
  // ---- thresholds ----
  uint32_t cut = 1u;                               // keys from here on stay
  uint64_t ties = ~0ull;                           // of those at the cut, the first so many
  if (k > 0 && k < d.V) {
    uint64_t before, at;
    const uint32_t key = select(false, 1u, [&](uint64_t x) { return x >= (uint64_t)k; }, before, at);
    if (key > cut) cut = key;
  }
  if (p < 1.f) {
    // the mass of what top-k left
    uint64_t sum = 0;
    for (int g = 0; g < segs; ++g) {
      uint32_t key[4];
      smp_load(d, row, wide, g * kSmpSeg + 4 * tid, key);
#pragma unroll
      for (int q = 0; q < 4; ++q) sum += key[q] >= cut ? w.weight(key[q]) : 0u;
    }
    sum = wave_sum_u64(sum);
    if (lane == 0) s.red[wave] = sum;
    __syncthreads();
    sum = 0;
    for (int x = 0; x < kSmpWaves; ++x) sum += s.red[x];
    __syncthreads();
    const double want = (double)p * (double)sum;
    uint64_t before, at = 0;
    const uint32_t key = select(true, cut, [&](uint64_t x) { return (double)x >= want; }, before, at);
    if (key != 0u) {
      cut = key;
      const uint64_t each = w.weight(key);
      const uint64_t n = at / each;                // ties; of them those with before + i each < want
      uint64_t c = (uint64_t)((want - (double)before) / (double)each);
      while (c > 0 && (double)(before + (c - 1) * each) >= want) --c;
      while (c < n && (double)(before + c * each) < want) ++c;
      ties = c < n ? c : ~0ull;
    }
  }
  // ---- where the ties end ----
  int tie_end = d.V;                               // tokens at the cut stay before this index
  if (ties != ~0ull) {
    for (int g = 0; g < segs; ++g) {
      uint32_t key[4];
      smp_load(d, row, wide, g * kSmpSeg + 4 * tid, key);
      uint64_t n = 0;
#pragma unroll
      for (int q = 0; q < 4; ++q) n += key[q] == cut ? 1u : 0u;
      n = wave_sum_u64(n);
      if (lane == 0) s.part[g * kSmpWaves + wave] = n;
    }
    __syncthreads();
    uint64_t before = 0;
    int at = 0;
    while (before + s.part[at] < ties) before += s.part[at++];   // ties is below their number
    uint32_t key[4];
    const int i0 = (at / kSmpWaves) * kSmpSeg + (at % kSmpWaves) * 256 + 4 * lane;
    smp_load(d, row, wide, i0, key);
    uint64_t n = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) n += key[q] == cut ? 1u : 0u;
    uint64_t x = before + wave_scan_u64(n, lane) - n;
    int end = -1;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (key[q] == cut && ++x == ties) end = i0 + q + 1;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) end = max(end, __shfl_xor(end, o, kWave));
    tie_end = end;
    __syncthreads();
  }
  auto kept = [&](uint32_t key, int i) -> uint64_t {
    if (key < cut || (key == cut && i >= tie_end)) return 0u;
    if (mp > 0.f && !(w.x(key) >= log_mp)) return 0u;
    return w.weight(key);
  };
  // ---- the kept weights of each 256 tokens, their sum, and where u falls ----
  for (int g = 0; g < segs; ++g) {
    const int i0 = g * kSmpSeg + 4 * tid;
    uint32_t key[4];
    smp_load(d, row, wide, i0, key);
    uint64_t sum = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) sum += kept(key[q], i0 + q);
    sum = wave_sum_u64(sum);
    if (lane == 0) s.part[g * kSmpWaves + wave] = sum;
  }
  __syncthreads();
  if (wave != 0) return;
  uint64_t Z = 0;
  for (int i = lane; i < segs * kSmpWaves; i += kWave) Z += s.part[i];
  Z = wave_sum_u64(Z);
  const double goal = (double)d.u[r] * (double)Z;
  auto over = [&](uint64_t x) { return (double)x > goal; };
  // the first 256 tokens whose sum passes, or the last with any weight
  int at = -1, last = 0;
  uint64_t before = 0, run = 0;
  for (int i = 0; i < segs * kSmpWaves; ++i) {
    const uint64_t x = s.part[i];
    if (x > 0) last = i;
    if (over(run + x) && x > 0) {
      at = i;
      before = run;
      break;
    }
    run += x;
  }
  const bool none = at < 0;                        // u is no number below 1
  if (none) at = last;
  const int i0 = (at / kSmpWaves) * kSmpSeg + (at % kSmpWaves) * 256 + 4 * lane;
  uint32_t key[4];
  uint64_t wt[4], n = 0;
  smp_load(d, row, wide, i0, key);
#pragma unroll
  for (int q = 0; q < 4; ++q) n += wt[q] = kept(key[q], i0 + q);
  uint64_t x = before + wave_scan_u64(n, lane) - n;
  int pick = none ? -1 : 0x7fffffff;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    x += wt[q];
    if (wt[q] > 0) {
      if (none) pick = i0 + q;
      else if (over(x) && pick == 0x7fffffff) pick = i0 + q;
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const int y = __shfl_xor(pick, o, kWave);
    pick = none ? max(pick, y) : min(pick, y);
  }
  if (lane == 0) {
    d.ids[r] = pick;
    if (d.logprob)
      d.logprob[r] = (float)(w.x(smp_key(to_f32<T>(row[pick]))) - (log((double)Z) - 45.0 * 0.69314718055994531));
  }
}

__global__ void k_smp_clear_err(uint32_t* err) {
  if (threadIdx.x == 0) *err = 0u;
}

}  // namespace xp

using namespace xp;

struct xp_sampler {
  int device = 0, V = 0, max_rows = 0;
  void* ws = nullptr;
  uint32_t* err = nullptr;
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
  if (e == hipSuccess) {
    const size_t total = 256;
    e = hipMalloc(&s->ws, total);
    if (e != hipSuccess) {
      (void)hipGetLastError();
      delete s;
      return smp_fail(nullptr, XP_ENOMEM, "workspace of %zu bytes: %s", total, hipGetErrorString(e));
    }
    s->err = static_cast<uint32_t*>(s->ws);
    e = hipMemset(s->ws, 0, 256);
    if (e == hipSuccess) e = hipDeviceSynchronize();
  }
  if (e != hipSuccess) {
    if (s->ws) (void)hipFree(s->ws);
    delete s;
    return smp_fail(nullptr, XP_EHIP, "sampler: %s", hipGetErrorString(e));
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
  Smp d{};
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
  d.err = s->err;
  hipStream_t st = (hipStream_t)stream;
  if (dtype == XP_F32) hipLaunchKernelGGL(k_sample_row<float>, dim3(rows), dim3(kSmpThreads), 0, st, d);
  else hipLaunchKernelGGL(k_sample_row<uint16_t>, dim3(rows), dim3(kSmpThreads), 0, st, d);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return smp_fail(s, XP_EHIP, "launch failed: %s", hipGetErrorString(e));
  return XP_OK;
}

extern "C" xp_status xp_sampler_device_errors(xp_sampler* s, uint32_t* out, void* stream) {
  if (s == nullptr) return XP_EINVAL;
  if (out == nullptr) return smp_fail(s, XP_EINVAL, "out is NULL");
  const xp_status ds = smp_device(s);
  if (ds != XP_OK) return ds;
  hipStream_t st = (hipStream_t)stream;
  hipError_t e = hipMemcpyAsync(out, s->err, sizeof(uint32_t), hipMemcpyDeviceToHost, st);
  if (e == hipSuccess) {
    hipLaunchKernelGGL(k_smp_clear_err, dim3(1), dim3(64), 0, st, s->err);
    e = hipGetLastError();
  }
  if (e == hipSuccess) e = hipStreamSynchronize(st);
  if (e != hipSuccess) return smp_fail(s, XP_EHIP, "device errors: %s", hipGetErrorString(e));
  return XP_OK;
}
