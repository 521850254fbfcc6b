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
#include "k_launch.cuh"

namespace bkv {

constexpr int kAtTile = 128;             // keys per tile
constexpr uint32_t kAtBox = 128 * 128;   // [128 rows][64 bf16] swizzled box
constexpr int kMaxRows = 256;            // query rows per row block
constexpr int kBlockRows4 = 16;          // the same over 4-bit caches
// Query rows per KV head up to which a 4-bit cache is read code by code, 16 rows at a time, which takes time by the
// row; beyond, its rows are unpacked to fp16 first, which does not.  A call in us, by codes and unpacked:
//   without weights       32 rows     64 rows     80 rows     96 rows     128 rows
//   128 x 4224          81, 176    131, 177    156, 177    182, 178    230, 181
//   8 x 32768           51, 100     73, 101     83, 101     95, 101    117, 102
//   32 x 1024            25, 25      31, 26      36, 25      43, 27      44, 27
//   128 x 4224, d 64    60, 102     93, 102    110, 102    128, 102    160, 103
//   with weights          16 rows     32 rows     48 rows     64 rows      96 rows
//   128 x 4224          66, 225    116, 226    160, 225    204, 227    290, 230
//   8 x 32768           47, 128     66, 130     91, 128    113, 129    163, 131
//   32 x 1024            27, 37      36, 32      48, 32      55, 33      72, 37
// From 16 to 24 rows on bkv_attend over bf16 caches of the same keys is faster than either.
constexpr int kRows4[2] = {80, 96};  // head_dim 64, 128
constexpr int kLogitRows4 = 48;      // the same with weights
// Query rows per KV head up to which the logits are kept for the weights, 4 bytes a row and key written and
// read once more, row by row by the merge; beyond, the weights are recomputed from the keys by two more launches.
// A call in us, kept and recomputed, by the number of caches and their keys:
//   head_dim 128        4 rows       16 rows      24 rows      32 rows      44 rows       64 rows
//   56 x 1088       15.0, 22.7   21.0, 23.3   25.9, 24.2   29.1, 24.2   35.9, 25.1   48.2, 26.5
//   8 x 32768       30.2, 50.0   36.0, 50.7   40.8, 51.9   45.9, 52.5   53.7, 53.5   71.8, 54.5
//   128 x 4224      52.5, 81.6   62.2, 82.7   73.4, 83.9   89.9, 84.4    111, 85.2    144, 85.9
// (head_dim 64 crosses at the same rows.)  32 rows gain a seventh where the keys are many and the logits stay in L2
// and lose a fifth on short caches; 24 rows gain a fifth or an eighth, or lose a twelfth.
constexpr int kLogitRows = 32;
constexpr float kMaxAbove = 32.f;        // log2 of how far p may exceed 1 before its reference moves
constexpr float kRefFloor = -1e30f;

// mbar_wait in few instructions: the attention kernels wait in many places, and a short kernel pays for
// the instructions it has to fetch.  Gives up after limit_ns (below 2^32), or once *abort is set.
__device__ __forceinline__ uint32_t globaltimer_lo() {
  uint32_t t;
  asm volatile("mov.u32 %0, %%globaltimer_lo;" : "=r"(t));
  return t;
}
__device__ __forceinline__ bool at_wait_for(uint64_t* bar, uint32_t parity, volatile int* abort, int* err, int code,
                                            uint32_t limit_ns) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint32_t t0 = globaltimer_lo();
#pragma unroll 1
  while (!mbar_try_wait_sleep(bar, parity)) {
    if (abort && *abort) return false;
    if (globaltimer_lo() - t0 > limit_ns) {
      if (abort) *abort = 1;
      record_error(err, code);
      return false;
    }
  }
  return true;
}
constexpr uint32_t kAtWaitNs = static_cast<uint32_t>(kWaitLimitNs);
__device__ __forceinline__ bool at_wait(uint64_t* bar, uint32_t parity, volatile int* abort, int* err, int code) {
  return at_wait_for(bar, parity, abort, err, code, kAtWaitNs);
}
// The same for a barrier that arrives whatever the abort flag says (limit_s: at most 4).
__device__ __forceinline__ void at_wait_always(uint64_t* bar, uint32_t parity, int* err, int code, int limit_s) {
  at_wait_for(bar, parity, nullptr, err, code, limit_s * kAtWaitNs);
}

// Division of numbers below 2^31 by a number fixed on the host.
struct FastDiv {
  uint32_t d, mul, shift;
  FastDiv() = default;
  explicit FastDiv(uint32_t n) : d(n), mul(0), shift(0) {
    while ((1ull << shift) < n) ++shift;
    mul = static_cast<uint32_t>(((1ull << 32) * ((1ull << shift) - n)) / n + 1);
  }
  // x / d and x % d
  __device__ __forceinline__ int div(int x) const {
    return static_cast<int>((__umulhi(static_cast<uint32_t>(x), mul) + static_cast<uint32_t>(x)) >> shift);
  }
  __device__ __forceinline__ int mod(int x, int& quotient) const {
    quotient = div(x);
    return x - quotient * static_cast<int>(d);
  }
  __device__ __forceinline__ int mod(int x) const {
    int q;
    return mod(x, q);
  }
};

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
  // With a window a row of limit n sees the keys j < n with j >= n - window or j < n_sink (bkv_attend_window).
  int window, n_sink;
  int whole;  // with a window: CTA b takes item b and nothing else
  FastDiv by_n_kv, by_m, by_rr, by_mb, by_nr, by_nrb, by_n_q, by_len_div;
};

// Rows of a row block and the row it starts at.
struct AtBlock {
  int b0, r0;
};

__device__ __forceinline__ AtBlock at_block(const AtGeo& g, int rb) {
  int q;
  const int r = g.by_nr.mod(rb, q);
  return {q * g.mb, r * g.rr};
}

// Instance length; out of range counts as 0 (the caller reports it).
__device__ __forceinline__ int at_raw_len(const AtGeo& g, int e) { return __ldg(g.len + g.by_len_div.div(e)); }
__device__ __forceinline__ int at_valid_len(const AtGeo& g, int n) { return n >= 0 && n <= g.cap ? n : 0; }
__device__ __forceinline__ int at_len(const AtGeo& g, int e) { return at_valid_len(g, at_raw_len(g, e)); }

// Keys that the last and the first row (in causal order) of rows [r0, r0 + rr) see.
__device__ __forceinline__ int at_limit_max(const AtGeo& g, int len, int r0) {
  if (!g.causal) return len;
  const int r1 = min(g.R, r0 + g.rr) - 1;
  int h1;
  const int i1 = g.by_n_q.mod(r1, h1), i = h1 > g.by_n_q.div(r0) ? g.n_q - 1 : i1;
  return max(0, len - g.n_q + 1 + i);
}
__device__ __forceinline__ int at_limit_min(const AtGeo& g, int len, int r0) {
  if (!g.causal) return len;
  const int r1 = min(g.R, r0 + g.rr) - 1;
  int h0;
  const int i0 = g.by_n_q.mod(r0, h0), i = g.by_n_q.div(r1) > h0 ? 0 : i0;
  return max(0, len - g.n_q + 1 + i);
}

// Keys that column c of a row block sees.
__device__ __forceinline__ int at_limit(const AtGeo& g, int len, int r0, int c) {
  return g.causal ? max(0, len - g.n_q + 1 + g.by_n_q.mod(r0 + g.by_rr.mod(c))) : len;
}

// Tiles of an item: an item without keys still has one, all masked, that writes its empty rows.
__device__ __forceinline__ int at_tiles(int limit) { return max(1, (limit + kAtTile - 1) / kAtTile); }

// Where the tiles of an item lie.  Without a window one run from key 0.  With one, `ts` tiles of the first ns keys
// and then a run from key w0, the first that a row's window reaches; one run from key 0 where the two would meet.
struct AtRuns {
  int ts, ns, w0, T;
};
template <bool WIN>
__device__ __forceinline__ AtRuns at_runs(const AtGeo& g, int len, int r0) {
  const int limit = at_limit_max(g, len, r0);
  if (!WIN) return {0, 0, 0, at_tiles(limit)};
  const int lo = at_limit_min(g, len, r0) - g.window, ns = min(g.n_sink, limit);
  const int ts = (ns + kAtTile - 1) / kAtTile;
  if (lo <= ts * kAtTile) return {0, ns, 0, at_tiles(limit)};
  return {ts, ns, lo, ts + at_tiles(limit - lo)};
}

// Row of q, o and lse (there are fewer than 2^27) that column c of a row block stands for, or -1.
__device__ __forceinline__ int at_row(const AtGeo& g, int e, AtBlock blk, int c) {
  int bi, group;
  const int r = blk.r0 + g.by_rr.mod(c, bi), kv = g.by_n_kv.mod(e, group);
  if (bi >= g.mb || blk.b0 + bi >= g.m || r >= g.R) return -1;
  const int seq = group * g.m + blk.b0 + bi;
  return (seq * g.n_kv + kv) * g.R + r;
}

// ---------------------------------------------------------------- an even split of a run of units
// Units of all items in order, cut into equal shares: where this CTA's share starts.  There are n groups
// of items; `count(x)` is the number of units of group x, and `find(x, u)` turns unit u of group x into
// the unit's place.  Called by the whole block; ends with a barrier.
struct AtPlace {
  int e, k, t;  // instance, item of it, unit of that
};
struct AtShare {
  AtPlace at;
  int left, u;  // units of this CTA; number of the first one (there are fewer than 2^31 of them)
  int per;      // units of a full share
};

template <int THREADS, typename Count, typename Find>
__device__ __forceinline__ void at_split(int n, Count&& count, Find&& find, int* scan, AtShare* out) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int chunk = (n + THREADS - 1) / THREADS;
  const int x0 = min(n, tid * chunk), x1 = min(n, x0 + chunk);
  int mine = 0;
#pragma unroll 1
  for (int x = x0; x < x1; ++x) mine += count(x);
  int incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  if (lane == 31) scan[warp] = incl;
  __syncthreads();
  constexpr int kWarps = THREADS / 32;
  int w = lane < kWarps ? scan[lane] : 0;  // every warp scans the warps' totals
#pragma unroll
  for (int o = 1; o < kWarps; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += v;
  }
  const int total = __shfl_sync(0xffffffffu, w, kWarps - 1);
  const int before = __shfl_sync(0xffffffffu, w, warp) - __shfl_sync(0xffffffffu, incl, 31) + incl - mine;
  const int per = max(1u, (static_cast<uint32_t>(total) + gridDim.x - 1) / gridDim.x);
  const int u0 = static_cast<int>(min(static_cast<uint32_t>(total), blockIdx.x * static_cast<uint32_t>(per)));
  if (u0 == total) {
    if (tid == 0) *out = {{0, 0, 0}, 0, u0, per};
  } else if (u0 >= before && u0 < before + mine) {  // the start lies in this thread's groups
    int u = before, x = x0;
#pragma unroll 1
    for (;; ++x) {
      const int c = count(x);
      if (u0 < u + c) break;
      u += c;
    }
    *out = {find(x, u0 - u), min(per, total - u0), u0, per};
  }
  __syncthreads();
}

// The split of a source's tiles: by instances where all row blocks of one have the same tiles, else by
// row blocks; or an item to a CTA.
template <int THREADS, bool WIN = false>
__device__ __forceinline__ void at_split_tiles(const AtGeo& g, int* scan, AtShare* out) {
  if (WIN && g.whole) {
    int e;
    const int rb = g.by_nrb.mod(blockIdx.x, e), n = at_runs<WIN>(g, at_len(g, e), at_block(g, rb).r0).T;
    if (threadIdx.x == 0) *out = {{e, rb, 0}, n, 0, n};
    __syncthreads();
    return;
  }
  const bool even = !g.causal || g.n_q == 1;
  auto tiles = [&](int x) {
    const int e = even ? x : g.by_nrb.div(x), len = at_len(g, e);
    if (WIN) return at_runs<true>(g, len, even ? 0 : at_block(g, x - e * g.nrb).r0).T;
    return at_tiles(even ? len : at_limit_max(g, len, at_block(g, x - e * g.nrb).r0));
  };
  at_split<THREADS>(
      even ? g.I : g.I * g.nrb, [&](int x) { return tiles(x) * (even ? g.nrb : 1); },
      [&](int x, int u) {
        const int n = tiles(x);
        if (even) return AtPlace{x, u / n, u % n};
        int e;
        const int rb = g.by_nrb.mod(x, e);
        return AtPlace{e, rb, u};
      },
      scan, out);
}

// Reports lengths out of range; by the threads of one CTA.
template <int THREADS>
__device__ __forceinline__ void at_check_lengths(const AtGeo& g, int* err) {
  for (int e = threadIdx.x; e < g.I; e += THREADS) {
    const int n = __ldg(g.len + g.by_len_div.div(e));
    if (n < 0 || n > g.cap) record_error(err, kDevBadLength);
  }
}

// CTAs of `ctas` that an item of n >= 1 units was split over, where its first unit has number u and a full share
// `per` units: first .. last.  False where one CTA had it all, and for numbers that no split makes: a CTA that
// gave up a wait leaves u of its later items unwritten.
__host__ __device__ inline bool at_split_over(uint32_t u, uint32_t n, uint32_t per, uint32_t ctas, uint32_t& first,
                                              uint32_t& last) {
  if (per == 0) return false;
  first = u / per;
  last = (u + n - 1) / per;
  return first < last && last < ctas;  // a sum that wraps is below u
}

// One segment of a CTA's run.
struct AtSeg {
  int e, rb, t0, t1, T, len, r0, b0;
  int item, u;  // u: number of tile t0 in the run of all tiles
  int ts, ns, w0;  // with a window
};

// With a window: whether no row of [r0, r0 + n) sees a key of tile t, whose first key is k0.
__device__ __forceinline__ bool at_unseen(const AtGeo& g, const AtSeg& s, int r0, int n, int k0) {
  const int r1 = min(min(s.r0 + g.rr, g.R), r0 + n) - 1;
  if (r1 < r0) return true;
  int h0, h1;
  const int i0 = g.by_n_q.mod(r0, h0), i1 = g.by_n_q.mod(r1, h1);  // rows of several heads: all queries
  const int most = s.len - g.n_q + 1 + (h1 > h0 ? g.n_q - 1 : i1), least = s.len - g.n_q + 1 + (h1 > h0 ? 0 : i0);
  return k0 >= most || (k0 + kAtTile <= least - g.window && k0 >= g.n_sink);
}

// The first key of tile t of a segment's item.
template <bool WIN>
__device__ __forceinline__ int at_key0(const AtSeg& s, int t) {
  return WIN && t >= s.ts ? s.w0 + (t - s.ts) * kAtTile : t * kAtTile;
}

// With a window: the first key from `from` on that a row of limit n sees, or -1.  In a run that begins there the row
// sees none before.
__device__ __forceinline__ int at_first_seen(const AtGeo& g, int n, int from) {
  const int j = from < g.n_sink ? from : max(from, n - g.window);
  return j < n ? j : -1;
}

// Walks the CTA's segments; every role has its own.
template <bool WIN>
struct AtWalkOf {
  int e, rb, t, left, u;
  int raw, raw_ahead;  // lengths of instances e and e + 1; the latter is under way until it is needed
  __device__ __forceinline__ void look(const AtGeo& g) { raw_ahead = at_raw_len(g, min(e + 1, g.I - 1)); }
  __device__ __forceinline__ AtWalkOf(const AtGeo& g, const AtShare& s)
      : e(s.at.e), rb(s.at.k), t(s.at.t), left(s.left), u(s.u), raw(at_raw_len(g, s.at.e)) {
    look(g);
  }
  __device__ __forceinline__ bool next(const AtGeo& g, AtSeg& s) {
    if (left <= 0 || e >= g.I) return false;
    const AtBlock blk = at_block(g, rb);
    s.e = e;
    s.rb = rb;
    s.b0 = blk.b0;
    s.r0 = blk.r0;
    s.len = at_valid_len(g, raw);
    const AtRuns runs = at_runs<WIN>(g, s.len, blk.r0);
    s.T = runs.T;
    s.ts = runs.ts;
    s.ns = runs.ns;
    s.w0 = runs.w0;
    s.t0 = t;
    s.t1 = min(s.T, t + left);
    s.item = e * g.nrb + rb;
    s.u = u;
    u += s.t1 - s.t0;
    left -= s.t1 - s.t0;
    t = s.t1;
    if (t == s.T) {
      t = 0;
      if (++rb == g.nrb) {
        rb = 0;
        ++e;
        raw = raw_ahead;
        look(g);
      }
    }
    return true;
  }
};

using AtWalk = AtWalkOf<false>;

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// 2^k for any k (0 below the normal range).
__device__ __forceinline__ float pow2i(int k) {
  return k < -126 ? 0.f : __uint_as_float(static_cast<uint32_t>(min(k, 127) + 127) << 23);
}

// Where one source's kernel leaves what the merge needs.  Segment `cta + item` is the part of an
// item that a CTA worked on: both rise along the run of all segments, one of them by at least 1 from
// each segment to the next, so the numbers differ.
struct AtParts {
  float* o = nullptr;           // [segment][N rows][D] sums of p v
  float2* ml = nullptr;         // [segment][N rows] (reference, sum of p), base 2
  int2* span = nullptr;         // [item] first and last CTA that worked on it
  int2* cut = nullptr;          // [CTA] the item that the CTA began and left to others to finish (or -1), and
                                // the last CTA that worked on it
  int rows = 0;                 // rows per segment in o and ml
};

// What a CTA notes of its segments for the merge; `per` is the number of tiles of a full share.
__device__ __forceinline__ void at_note(const AtParts& p, const AtSeg& s, bool last_segment, int per) {
  const int last = static_cast<uint32_t>(s.u - s.t0 + s.T - 1) / static_cast<uint32_t>(per);
  if (s.t0 == 0) p.span[s.item] = make_int2(blockIdx.x, last);
  if (last_segment) p.cut[blockIdx.x] = make_int2(s.t0 == 0 && s.t1 < s.T ? s.item : -1, last);
}

// One source's launch plan, made on the host.
struct AtPlan {
  AtGeo geo;
  int grid;
  long long items;
  size_t off_o, off_ml, off_span, off_cut;  // byte offsets in the workspace
  AtParts parts(unsigned char* ws) const {
    AtParts p;
    p.o = reinterpret_cast<float*>(ws + off_o);
    p.ml = reinterpret_cast<float2*>(ws + off_ml);
    p.span = reinterpret_cast<int2*>(ws + off_span);
    p.cut = reinterpret_cast<int2*>(ws + off_cut);
    p.rows = geo.mb * geo.rr;
    return p;
  }
};

// The whole call: own caches, the prefix if there is one, and what the weights need.
struct AtLayout {
  AtPlan own, prefix;
  bool has_prefix = false;
  bool four = false;       // the caches are in 4 bits and the own kernel is that of k_attend4.cu
  bool unpacked = false;   // they are unpacked into the workspace as fp16 numbers, for the rows kernel
  size_t off_k = 0, off_k_rest = 0, off_v = 0, off_q = 0;  // fp16 [batch][n_kv][cap][d], and q
  size_t off_row_sc = 0;   // fp32 [rows]
  bool logits = false;     // the own kernel stores its logits for the weights
  size_t off_lse2 = 0;     // fp32 [rows]: log2 normalisers
  size_t off_logits = 0;   // fp32 [rows][cap]
  size_t off_wpart = 0, off_wu0 = 0;  // weights recomputed from the keys: [2 CTAs][128] partial sums, and the
                                      // [items + 1] unit numbers of their merge
  size_t bytes = 0;
  bool too_large = false;  // 2^31 tiles or more
  int sms = 0;             // of the current device: one CTA of the attention kernels each
};
// The workspace does not depend on pcap.
AtLayout attend_layout(const Shape& s, int n_q, int groups, int pcap, bool weights);
AtLayout attend4_layout(const Shape& s, int n_q, bool weights);
// Bytes that serve every call with at most n_q queries: more queries can need less (beyond kLogitRows rows no
// logits are kept), but beyond kMaxRows of them the need only grows.
size_t attend_workspace(const Shape& s, int n_q, int groups, bool weights);
size_t attend4_workspace(const Shape& s, int n_q, bool weights);

// Tiles of keys that the recomputed weights are made for.
inline long long weights_items(const Shape& s) {
  return 1ll * s.batch * s.n_kv * ((s.cap + kAtTile - 1) / kAtTile);
}

// In this order on one stream: tiles, merge (with the weights where the logits were kept), and with
// weights but no logits the weights, recomputed from the keys.
cudaError_t launch_attend(const Shape& s, const AttendArgs& a, const AtLayout& l, cudaStream_t st);
cudaError_t launch_attend_merge(const Shape& s, const AttendArgs& a, const AtLayout& l, cudaStream_t st);
cudaError_t launch_attend_weights(const Shape& s, const AttendArgs& a, const AtLayout& l, cudaStream_t st);

// The tiles of 4-bit caches, l.four set; the merge follows as above.
cudaError_t launch_attend4(const Shape& s, const Attend4Args& a, const AtLayout& l, cudaStream_t st);

// Arguments of the attention kernel.
struct AtKernelArgs {
  AtGeo geo;
  AtParts parts;
  int whole_is_final;  // an item that one CTA finished writes o and lse itself (no other source)
  int after_prefix;    // launched to overlap the prefix's kernel, which its own work does not need
  float sc;
  const float* row_sc;  // of fp16 operands: [rows], instead of sc
  __nv_bfloat16* o;
  float* lse;
  float* lse2;
  float* logits;       // [rows][cap] or nullptr
  int* err;
};
// With a window, boxes of kSinkRows rows of the keys and values, for the first keys.
constexpr int kSinkRows = 16;
template <bool WIN>
struct AtSinkMaps {
  CUtensorMap k, v;
};
template <>
struct AtSinkMaps<false> {};
// Row blocks of up to 128 rows (k_attend_tiles.cuh, one translation unit per head_dim), and of up to
// 256 (k_attend_rows.cuh); each once without and once with a window.
cudaError_t launch_attend_rows(int d, const AtPlan& p, const CUtensorMap& qmap, const CUtensorMap& kmap,
                               const CUtensorMap& vmap, const AtKernelArgs& a, cudaStream_t st);
// Over fp16 numbers, the keys in two terms.
cudaError_t launch_attend_rows_split(int d, const AtPlan& p, const CUtensorMap& qmap, const CUtensorMap& kmap,
                                     const CUtensorMap& restmap, const CUtensorMap& vmap, const AtKernelArgs& a,
                                     cudaStream_t st);
cudaError_t launch_attend_rows_window(int d, const AtPlan& p, const CUtensorMap& qmap, const CUtensorMap& kmap,
                                      const CUtensorMap& vmap, const AtKernelArgs& a, cudaStream_t st);
cudaError_t launch_attend_window_64(const AtPlan& p, const CUtensorMap& qmap, const CUtensorMap& kmap,
                                    const CUtensorMap& vmap, const AtSinkMaps<true>& sink, const AtKernelArgs& a,
                                    cudaStream_t st);
cudaError_t launch_attend_window_128(const AtPlan& p, const CUtensorMap& qmap, const CUtensorMap& kmap,
                                     const CUtensorMap& vmap, const AtSinkMaps<true>& sink, const AtKernelArgs& a,
                                     cudaStream_t st);
cudaError_t launch_attend_tiles_64(const AtPlan& p, const CUtensorMap& qmap, const CUtensorMap& kmap,
                                   const CUtensorMap& vmap, const AtKernelArgs& a, cudaStream_t st);
cudaError_t launch_attend_tiles_128(const AtPlan& p, const CUtensorMap& qmap, const CUtensorMap& kmap,
                                    const CUtensorMap& vmap, const AtKernelArgs& a, cudaStream_t st);

}  // namespace bkv
