// Rotary positions of one or several axes for the rows of queries and keys, with the
// RMSNorm over a head in front of them: what the rows of a paged cache and of its
// queries go through before PagedKV.write and .attend.
//
// Pair j of a head is (x[j], x[j + rot / 2]); with the position p on the pair's axis
// its angle is p theta^(-2 j / rot):
//   y[j] = x[j] cos - x[j + rot/2] sin,  y[j + rot/2] = x[j + rot/2] cos + x[j] sin;
// dims from rot on pass.  Angles are formed in 64 bits, in half turns, and only their
// part within (-1, 1] goes to 32: far positions lose nothing.
//
// A wave has a token (a part of its heads where there are few tokens): its lanes form
// the token's cosines and sines once, a pair each, and hand them round through LDS.
// A head is HD / 16 lanes of 16 values: 8 of the pairs' first halves and their 8
// partners, so that no value changes lanes.  Bound by memory where there are many tokens:
// 8191 tokens of 40 heads, three axes (168 MB), 37 to 41 us where the inputs alternate, 4.1 to
// 4.5 TB/s, 29 where the caches still hold some of them; one token 2.9 us.  Tokens split among
// more waves, each with fewer heads, took 49 to 52 us (the sines again).
#include <algorithm>
#include <cmath>

#include "xp_internal.h"

namespace xp {

constexpr int kRopeThreads = 256;
constexpr int kRopeWaves = kRopeThreads / kWave;
constexpr int kRopeMaxPairs = 128;
// waves that fill the chip, 4 a SIMD: below, a token's heads are split among waves
constexpr int kRopeFill = 4096;
constexpr int kRopeGrid = 1024;      // workgroups that run at once; their waves take token after token

// results that the caches (4 MB a die) would not keep go past them: 84 MB (8191 tokens of 40
// heads) 40.5 -> 36.9 us; smaller ones are read next by the cache write and the attention
constexpr int64_t kRopeCached = 32 << 20;

struct RopeRows {
  const void* x;
  void* y;
  const void* g;                     // gains of the norm; NULL: none
  int64_t x_ld, y_ld;
  int heads;
};
struct Rope {
  RopeRows r[2];                     // queries, keys
  const int32_t* pos;
  int64_t pos_ld;
  int64_t tokens;
  int half, split;                   // pairs; waves of a token
  double log2_theta;
  float eps;
  int past;                          // results go past the caches
  uint64_t axis[kRopeMaxPairs / 32]; // two bits a pair
};

template <typename T>
__device__ __forceinline__ void ld8(const T* p, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const u32x4 a = ld16(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(a[i] << 16);
      x[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
  } else {
    const floatx4 a = *reinterpret_cast<const floatx4*>(p), b = *reinterpret_cast<const floatx4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = a[i];
      x[i + 4] = b[i];
    }
  }
}
template <typename V>
__device__ __forceinline__ void st16(V* p, V x, bool past) {
  if (past) __builtin_nontemporal_store(x, p);     // wave-uniform
  else *p = x;
}
template <typename T>
__device__ __forceinline__ void st8(T* p, const float (&x)[8], bool past) {
  if constexpr (sizeof(T) == 2) {
    u32x4 a;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = pk_bf16(x[2 * i], x[2 * i + 1]);
    st16(reinterpret_cast<u32x4*>(p), a, past);
  } else {
    st16(reinterpret_cast<floatx4*>(p), floatx4{x[0], x[1], x[2], x[3]}, past);
    st16(reinterpret_cast<floatx4*>(p + 4), floatx4{x[4], x[5], x[6], x[7]}, past);
  }
}

template <typename T, int HD>
__global__ __launch_bounds__(kRopeThreads) void k_rope(const Rope d) {
  constexpr int L = HD / 16, HPW = kWave / L;      // lanes of a head, heads of a wave
  __shared__ __align__(16) float2 cs[kRopeWaves][kRopeMaxPairs];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = lane % L, hw = lane / L;
  const bool rot = 16 * c < 2 * d.half;            // the lane's chunks are pairs, or pass
  const int a0 = rot ? 8 * c : 16 * c, b0 = rot ? d.half + 8 * c : 16 * c + 8;
  const int all = d.r[0].heads + d.r[1].heads;
  const int64_t waves = (int64_t)gridDim.x * kRopeWaves;
  // the lane's pairs: their axes, and half turns a position
  constexpr int NP = HD / 128 > 0 ? HD / 128 : 1;
  double f[NP];
  int axis[NP];
#pragma unroll
  for (int n = 0; n < NP; ++n) {
    const int j = lane + kWave * n;
    axis[n] = (int)(d.axis[j >> 5] >> (2 * (j & 31))) & 3;
    f[n] = exp2(-d.log2_theta * j / d.half) * 0.31830988618379067154;
  }
  for (int64_t w = (int64_t)blockIdx.x * kRopeWaves + wave; w < d.tokens * d.split; w += waves) {
    const int64_t t = w / d.split;
    const int part = (int)(w - t * d.split);
    wave_lds_order();                              // the last token's reads
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      double turn = (double)d.pos[axis[n] * d.pos_ld + t] * f[n];
      turn -= 2.0 * rint(0.5 * turn);
      float sn, co;
      sincospif((float)turn, &sn, &co);
      cs[wave][lane + kWave * n] = float2{co, sn};
    }
    wave_lds_order();
    float co[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 x = cs[wave][rot ? 8 * c + i : 0];
      co[i] = rot ? x.x : 1.f;
      sn[i] = rot ? x.y : 0.f;
    }
    for (int h = part * HPW + hw; h < all; h += d.split * HPW) {
      const bool key = h >= d.r[0].heads;
      const RopeRows& r = d.r[key];
      const int64_t head = (int64_t)(key ? h - d.r[0].heads : h) * HD;
      const T* x = static_cast<const T*>(r.x) + t * r.x_ld + head;
      T* y = static_cast<T*>(r.y) + t * r.y_ld + head;
      float a[8], b[8];
      ld8(x + a0, a);
      ld8(x + b0, b);
      if (r.g != nullptr) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(a[i], a[i], fmaf(b[i], b[i], s));
#pragma unroll
        for (int o = 1; o < L; o <<= 1) s += __shfl_xor(s, o, kWave);
        const float inv = 1.f / sqrtf(s / HD + d.eps);
        float ga[8], gb[8];
        ld8(static_cast<const T*>(r.g) + a0, ga);
        ld8(static_cast<const T*>(r.g) + b0, gb);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          a[i] *= inv * ga[i];
          b[i] *= inv * gb[i];
        }
      }
      float ya[8], yb[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        ya[i] = rot ? a[i] * co[i] - b[i] * sn[i] : a[i];
        yb[i] = rot ? b[i] * co[i] + a[i] * sn[i] : b[i];
      }
      st8(y + a0, ya, d.past);
      st8(y + b0, yb, d.past);
    }
  }
}

}  // namespace xp

using namespace xp;

static bool rope_rows_ok(const RopeRows& r, int hd, int es) {
  if (r.heads == 0) return true;
  const auto odd = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 != 0; };
  const int64_t row = (int64_t)r.heads * hd;
  return r.x != nullptr && r.y != nullptr && !odd(r.x) && !odd(r.y) && !odd(r.g) && r.x_ld >= row &&
         r.y_ld >= row && r.x_ld * es % 16 == 0 && r.y_ld * es % 16 == 0 &&
         (r.x != r.y || r.x_ld == r.y_ld);
}

extern "C" xp_status xp_rope(const xp_rope_shape* s, int32_t tokens, const int32_t* pos,
                             int64_t pos_ld, const void* q, int64_t q_ld, int32_t n_heads,
                             const void* g_q, void* q_out, int64_t q_out_ld, const void* k,
                             int64_t k_ld, int32_t n_kv, const void* g_k, void* k_out,
                             int64_t k_out_ld, void* stream) {
  if (s == nullptr || tokens < 0 || n_heads < 0 || n_kv < 0 || n_heads + (int64_t)n_kv < 1 ||
      n_heads > 65536 || n_kv > 65536 || (s->dtype != XP_F32 && s->dtype != XP_BF16) ||
      s->head_dim < 1 || s->rot_dim < 16 || s->rot_dim > s->head_dim || s->rot_dim % 16 != 0 ||
      s->axes < 1 || s->axes > 4 || (s->interleaved != 0 && s->interleaved != 1) ||
      !(s->theta >= 1.f && s->theta <= 0x1p60f) || !(s->eps >= 0.f && s->eps <= 0x1p60f))
    return XP_EINVAL;
  if (s->head_dim != 64 && s->head_dim != 128 && s->head_dim != 256) return XP_EUNSUPPORTED;
  Rope d{};
  d.half = s->rot_dim / 2;
  int sum = 0;
  for (int a = 0; a < s->axes; ++a) {
    if (s->sections[a] < 0 || s->sections[a] > d.half) return XP_EINVAL;
    sum += s->sections[a];
    // in turn, the pairs of an axis but the first are a, a + axes, ..
    if (s->interleaved && a > 0 && s->sections[a] > 0 &&
        a + s->axes * (s->sections[a] - 1) >= d.half)
      return XP_EINVAL;
  }
  if (sum != d.half) return XP_EINVAL;
  for (int j = 0, a = 0, end = s->sections[0]; j < d.half; ++j) {
    int ax;
    if (s->interleaved) {
      ax = j % s->axes;
      if (j / s->axes >= s->sections[ax]) ax = 0;
    } else {
      while (j >= end) end += s->sections[++a];
      ax = a;
    }
    d.axis[j >> 5] |= (uint64_t)ax << (2 * (j & 31));
  }
  const int es = s->dtype == XP_BF16 ? 2 : 4;
  d.r[0] = RopeRows{q, q_out, g_q, q_ld, q_out_ld, n_heads};
  d.r[1] = RopeRows{k, k_out, g_k, k_ld, k_out_ld, n_kv};
  if (pos == nullptr || pos_ld < tokens || !rope_rows_ok(d.r[0], s->head_dim, es) ||
      !rope_rows_ok(d.r[1], s->head_dim, es))
    return XP_EINVAL;
  if (tokens == 0) return XP_OK;
  d.pos = pos;
  d.pos_ld = pos_ld;
  d.tokens = tokens;
  d.log2_theta = std::log2((double)s->theta);
  d.eps = s->eps;
  d.past = (int64_t)tokens * (n_heads + n_kv) * s->head_dim * es > kRopeCached;
  const int hpw = kWave / (s->head_dim / 16), groups = (n_heads + n_kv + hpw - 1) / hpw;
  d.split = (int)std::min<int64_t>(groups, (kRopeFill + tokens - 1) / tokens);
  const int64_t wgs = ((int64_t)tokens * d.split + kRopeWaves - 1) / kRopeWaves;
  const dim3 grid((unsigned)std::min<int64_t>(wgs, kRopeGrid)), block(kRopeThreads);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
#define XP_ROPE(T_, HD_) hipLaunchKernelGGL((k_rope<T_, HD_>), grid, block, 0, st, d)
  if (s->dtype == XP_BF16) {
    if (s->head_dim == 64) XP_ROPE(uint16_t, 64);
    else if (s->head_dim == 128) XP_ROPE(uint16_t, 128);
    else XP_ROPE(uint16_t, 256);
  } else {
    if (s->head_dim == 64) XP_ROPE(float, 64);
    else if (s->head_dim == 128) XP_ROPE(float, 128);
    else XP_ROPE(float, 256);
  }
#undef XP_ROPE
  return hipGetLastError() == hipSuccess ? XP_OK : XP_EHIP;
}
