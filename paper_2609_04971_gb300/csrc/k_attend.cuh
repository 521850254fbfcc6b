// Work layout of the attention kernels: row blocks of query rows against key
// tiles, and the workspace that carries partial results between the kernels.
//
// A *source* is a set of caches that queries read: the sequences' own caches,
// or the shared prefixes.  Source instance e has R * m query rows: the R = G *
// n_q rows (query head, query) of its KV head in each of m sequences (m = 1 for
// a sequence's own cache).  They are cut into row blocks of at most N rows, mb
// sequences x rr rows; an *item* is one row block of one instance, and its keys
// are walked in tiles of 128.  All tiles of all items, in item order, are split
// evenly over the grid, so a CTA works through a run of *segments*: consecutive
// tiles of one item.
#pragma once

#include "bkv_device.cuh"
#include "bkv_internal.h"

namespace bkv {

constexpr int kAtTile = 128;  // keys per tile

struct AtGeo {
  int I;          // instances
  int n_kv;       // KV heads: instance e is KV head e % n_kv of sequence group e / n_kv
  int m;          // sequences per instance
  int R, rr, mb;  // rows per sequence; a row block's rows per sequence and sequences
  int nr, nrb;    // row blocks along the rows of a sequence; row blocks per instance
  int n_q;
  int causal;     // own caches: row i of n_q sees length - n_q + 1 + i keys; prefixes: every row sees all
  int cap;        // rows allocated per instance
  const int* len; // own: one per instance; prefix: one per sequence group
  int len_div;    // instance e has length len[e / len_div]
};

// Rows of a row block and the row it starts at.
struct AtBlock {
  int b0, r0;
};

__host__ __device__ inline AtBlock at_block(const AtGeo& g, int rb) { return {rb / g.nr * g.mb, rb % g.nr * g.rr}; }

// Instance length; out of range counts as 0 (the caller reports it).
__device__ __forceinline__ int at_len(const AtGeo& g, int e) {
  const int n = __ldg(g.len + e / g.len_div);
  return n >= 0 && n <= g.cap ? n : 0;
}

// Keys that the last and the first row (in causal order) of rows [r0, r0 + rr) see.
__device__ __forceinline__ int at_limit_max(const AtGeo& g, int len, int r0) {
  if (!g.causal) return len;
  const int r1 = min(g.R, r0 + g.rr) - 1;
  const int i = r1 / g.n_q > r0 / g.n_q ? g.n_q - 1 : r1 % g.n_q;
  return max(0, len - g.n_q + 1 + i);
}
__device__ __forceinline__ int at_limit_min(const AtGeo& g, int len, int r0) {
  if (!g.causal) return len;
  const int r1 = min(g.R, r0 + g.rr) - 1;
  const int i = r1 / g.n_q > r0 / g.n_q ? 0 : r0 % g.n_q;
  return max(0, len - g.n_q + 1 + i);
}

// Tiles of an item: an item without keys still has one, all masked, that writes its empty rows.
__device__ __forceinline__ int at_tiles(int limit) { return max(1, (limit + kAtTile - 1) / kAtTile); }

__device__ __forceinline__ long long at_inst_tiles(const AtGeo& g, int e) {
  const int len = at_len(g, e);
  if (!g.causal || g.n_q == 1) return static_cast<long long>(g.nrb) * at_tiles(len);
  long long n = 0;  // m == 1 here: every row block starts at another row
  for (int rb = 0; rb < g.nrb; ++rb) n += at_tiles(at_limit_max(g, len, at_block(g, rb).r0));
  return n;
}

// Row of q, o and lse that column c of a row block stands for, or -1.
__device__ __forceinline__ long long at_row(const AtGeo& g, int e, AtBlock blk, int c) {
  const int bi = c / g.rr, r = blk.r0 + c % g.rr;
  if (bi >= g.mb || blk.b0 + bi >= g.m || r >= g.R) return -1;
  const long long seq = static_cast<long long>(e / g.n_kv) * g.m + blk.b0 + bi;
  return (seq * g.n_kv + e % g.n_kv) * g.R + r;
}

// Where one source's kernel leaves what the merge needs.  Segment `cta + item` is the part of an
// item that a CTA worked on: both rise along the run of all segments, one of them by at least 1 from
// each segment to the next, so the numbers differ.
struct AtParts {
  float* o = nullptr;           // [segment][N rows][D] sums of p v
  float2* ml = nullptr;         // [segment][N rows] (reference, sum of p), base 2
  long long* u0 = nullptr;      // [item] number of its first tile in the run of all tiles
  long long* per = nullptr;     // [1] tiles per CTA
  int rows = 0;                 // rows per segment in o and ml
};

// Parts of an item: CTAs first .. last worked on it.
struct AtSpan {
  int first, last;
};
__device__ __forceinline__ AtSpan at_span(const AtParts& p, long long item, int tiles) {
  const long long u = p.u0[item], per = *p.per;
  return {static_cast<int>(u / per), static_cast<int>((u + tiles - 1) / per)};
}

// One source's launch plan, made on the host.
struct AtPlan {
  AtGeo geo;
  int n_cols;   // template columns: 16, 32, 64 or 128
  int grid;
  long long items;
  size_t off_o, off_ml, off_u0, off_per;  // byte offsets in the workspace
  AtParts parts(unsigned char* ws) const {
    AtParts p;
    p.o = reinterpret_cast<float*>(ws + off_o);
    p.ml = reinterpret_cast<float2*>(ws + off_ml);
    p.u0 = reinterpret_cast<long long*>(ws + off_u0);
    p.per = reinterpret_cast<long long*>(ws + off_per);
    p.rows = geo.mb * geo.rr;
    return p;
  }
};

// The whole call: own caches, the prefix if there is one, and what the weights need.
struct AtLayout {
  AtPlan own, prefix;
  bool has_prefix = false;
  bool logits = false;     // the own kernel stores its logits for the weights
  size_t off_lse2 = 0;     // fp32 [rows]: log2 normalisers
  size_t off_logits = 0;   // fp32 [rows][cap]
  size_t bytes = 0;
};
AtLayout attend_layout(const Shape& s, int n_q, int groups, int pcap, bool weights);

// Arguments of the attention kernel.
struct AtKernelArgs {
  AtGeo geo;
  AtParts parts;
  int whole_is_final;  // an item that one CTA finished writes o and lse itself (no other source)
  int reuse;           // several row blocks read the same keys: let them stay in L2
  float sc;
  __nv_bfloat16* o;
  float* lse;
  float* lse2;
  float* logits;       // [rows][cap] or nullptr
  int* err;
};
cudaError_t launch_attend_tiles(int d, const AtPlan& p, const CUtensorMap& qmap, const CUtensorMap& kmap,
                                const CUtensorMap& vmap, const AtKernelArgs& a, cudaStream_t st);

}  // namespace bkv
