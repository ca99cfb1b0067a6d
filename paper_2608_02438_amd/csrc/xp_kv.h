// The paged context cache: its handle and what the kernels of xp_kv.hip and
// xp_kv_attn.hip share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <string>

#include "../../include/xpress.h"
#include "xp_device.h"

namespace xp {

constexpr int kKvTile = 64;          // keys of an attention tile
constexpr int kKvMaxBatch = 4096;    // sequences of a call
constexpr int kKvMaxLen = 1 << 22;   // keys of a sequence

// the last index in [lo, hi) whose a[] is at most x (a[lo] <= x, a non-decreasing)
template <typename P>
__device__ __forceinline__ int kv_owner(P a, int lo, int hi, int x) {
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (a[m] <= x) lo = m;
    else hi = m;
  }
  return lo;
}
template <typename P>
__device__ __forceinline__ int kv_owner(P a, int n, int x) { return kv_owner(a, 0, n, x); }

// One row tile of the attention's work list: up to R query rows of one
// sequence (or of the sequences of one group, for a shared prefix), and the
// key tiles they walk.  Row r of the tile is row row0 + r of the tokens from
// tok0 on, counted (token, head of the KV head's group).  The keys are [floor,
// ceil) (a prefix, or what lies behind one); of these some row sees those of
// [floor, s) and of [lo, hi).  Tile j starts at key 64 (j < n1 ? a0 + j :
// b0 + j - n1).
struct KvEntry {
  int32_t tok0, row0, nrows, seq;    // seq: the row of the block table
  int32_t p0;                        // position of token tok0; of several sequences the least
  int32_t prefix;                    // 1: rows of several sequences, positions from pos[]
  int32_t floor, ceil;
  int32_t s, lo, hi, tiles;
  int32_t a0, n1, b0;
  int32_t p1;                        // the greatest position of several sequences
};
constexpr int kKvEntryInts = sizeof(KvEntry) / 4;

// where share s of the work begins: unit f, at tile j of (entry e, KV head kvh), or
// -j units before its first
struct KvShare {
  int32_t f, e, kvh, j;
};

// A work list (device pointers).
struct KvList {
  int32_t* hdr = nullptr;            // [0] units, [1] units of a share, [2] entries
  KvShare* share = nullptr;          // [shares + 1]
  KvEntry* ent = nullptr;            // [entries]
  int32_t* cum = nullptr;            // [entries + 1] units before each entry
};

// Workspace of the attention (device pointers).
struct KvAttnWs {
  KvList list[2];                    // the sequences' own keys (and prefixes); the prefixes
  float* part = nullptr;             // [rows][head_dim] partial O of each list's cut segments,
                                     // then of rows (own keys, prefix)
  float* ml = nullptr;               // [rows][2] their reference maximum (base 2) and sum
  // calls with shared prefixes
  int32_t* pos = nullptr;            // [tokens] position of every token
  int2* row[2] = {};                 // [tokens] first row among its sequence's (group's; -1:
                                     // none), and their first entry
  char* dump = nullptr;              // a row of 128 floats that takes what no one reads
  const char* zero = nullptr;        // 256 bytes of zeros: a key row that no one sees
};

// Arguments of the attention's kernels.
struct KvAttnArgs {
  int n, total_q, max_q;             // max_q: tokens of the longest sequence; of each without cu_q
  const int32_t* cu_q;
  const int32_t* kv_len;
  int kv_add;                        // added to every kv_len (the layer's own block)
  const int32_t* table;
  int64_t table_ld;
  const uint16_t* q;
  int64_t q_ld;
  const void* kc;
  const void* vc;
  const float* k_scale;
  const float* v_scale;
  int causal, window, sinks;
  float scale;
  uint16_t* out;
  int64_t out_ld;
  float* lse;
  int groups;                        // 0: no shared prefixes
  const int32_t* group_start;
  const int32_t* shared_len;
};

}  // namespace xp

struct xp_kv {
  int device = 0, cus = 0;
  int nh = 0, nkv = 0, grp = 1, hd = 0, P = 0, logP = 0, n_pages = 0, dtype = 0;
  int max_batch = 0, max_tokens = 0, max_len = 0, max_pages = 0, shared = 0;
  int entries = 0;                   // entries the workspace holds
  int64_t rows = 0;                  // partial rows of a list's cut segments
  void* ws = nullptr;
  xp::KvAttnWs a;
  int32_t* take = nullptr;           // [max_batch + 1] pages taken before each request
  int32_t* old = nullptr;            // [max_batch] pages held before the call
  int32_t* acu = nullptr;            // [max_batch + 1] new tokens before each request
  int32_t* len = nullptr;            // [max_batch] tokens before the call (-1: left alone)
  int32_t* top = nullptr;            // [2] free pages after the releases, pages taken
  uint32_t* err = nullptr;
  std::string msg;
};

namespace xp {

// The attention's launch sequence; sizes and pointers were checked.
hipError_t launch_kv_attn(const xp_kv* kv, const KvAttnArgs& a, hipStream_t st);
// k, v rows [tokens][n_kv][head_dim] (strides in elements) to their slots, or,
// with slots NULL, to positions len[b] + i of the block table (B tokens a sequence)
hipError_t launch_kv_write(const xp_kv* kv, int tokens, const uint16_t* k, const uint16_t* v,
                           int64_t k_ld, int64_t v_ld, const int32_t* slots, const int32_t* table,
                           int64_t table_ld, const int32_t* len, int B, void* kc, void* vc,
                           const float* k_scale, const float* v_scale, hipStream_t st);
// the units of the attention's work list, counted in 32 bits, for n sequences of
// `tokens` tokens and tables of table_ld pages
bool kv_units_fit(const xp_kv* kv, int64_t tokens, int64_t n, int groups, int64_t table_ld);
// rows of partials and entries a handle needs
void kv_attn_sizes(const xp_kv* kv, int64_t* rows, int* entries, int* shares);

}  // namespace xp
