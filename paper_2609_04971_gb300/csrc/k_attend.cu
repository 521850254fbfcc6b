// Attention of the newest queries over a sequence's cache and, with a shared
// prefix, over the prefix of its group (include/bkv.h, bkv_attend): the plan of
// a call, its workspace, and the merge of the partial results.
//
// The attention kernels (k_attend_tiles.cuh, k_attend_rows.cu) leave, for every part
// of an item that one CTA worked on, the sums O_p = sum p v and l_p = sum p of each
// row against a reference m_p (p = 2^(y - m_p), y the base-2 logits), all in fp32.  A
// row's result over all its parts is
//   lse2 = log2 sum_p l_p 2^(m_p),   o = sum_p O_p 2^(m_p - lse2),
// taken in the parts' order, a warp to a row: the order of the GPU's blocks does not
// show.  A row that one CTA finished is already written, so without a prefix the
// merge goes by the CTAs: each leaves one unfinished item at most.  The same launch
// adds the attention weights where the logits were kept, a thread to a key:
// weights[j] += sum over rows of 2^(y - lse2), rows in order.
//
// Bound by latency: it starts while the attention kernel ends (its launch overlaps),
// and then reads a row's references, its parts and its weights one after the other.
// Cold: one token, 128 caches of 4224 keys 7.7 us (11 MB of parts and logits); 8 caches
// of 32768 keys 8 us; 16 samples of a prefix of 32768 keys 9.8 us; merge_rows_kernel, a prompt
// of 4096 tokens, 32 heads, 152 split blocks of 256 rows, 10.8 us for 35 MB of parts.
#include <algorithm>
#include <type_traits>

#include "k_attend.cuh"

namespace bkv {
namespace {

constexpr int kMergeThreads = 256, kMergeRows = kMergeThreads / 32;  // rows per block
constexpr int kMergeWarpRows = 4;  // rows per warp of merge_rows_kernel
constexpr int kMergeKeys = 1024;   // keys per block of the weights' part

size_t align_up(size_t n) { return (n + 255) / 256 * 256; }

// Row blocks of m sequences x R rows: all rows of an instance in one block while there are at most 128
// of them (keys as lanes, k_attend_tiles.cuh), else blocks of at most 256, as even as 16-row steps allow (rows
// as lanes, k_attend_rows.cu).  Both sides of the 128, head_dim 128, 128 caches of 4224 keys: 80 rows 51 and 59 us,
// 128 rows 60 and 63 us; 144 rows (two blocks, and one) 90 and 64 us, 256 rows 105 and 72 us; 8 caches of 32768 keys:
// 80 rows 35 and 40, 128 rows 42.5 and 42.5, 144 rows 52 and 43 us.
AtPlan make_plan(const Shape& s, int I, int m, int R, int n_q, bool causal, int cap, int len_div, int sms,
                 bool& too_large, int most4 = 0) {
  AtPlan p{};
  AtGeo& g = p.geo;
  g.I = I;
  g.n_kv = s.n_kv;
  g.m = m;
  g.R = R;
  g.n_q = n_q;
  g.causal = causal;
  g.cap = cap;
  g.len_div = len_div;
  const int most_rows = 1ll * R * m <= kAtTile ? kAtTile : kMaxRows;
  if (most4) {  // blocks of up to that many rows, as even as they can be
    g.mb = 1;
    g.nr = (R + most4 - 1) / most4;
    g.rr = (R + g.nr - 1) / g.nr;
    g.nr = (R + g.rr - 1) / g.rr;
  } else if (R <= most_rows) {
    const int most = most_rows / R, nb = (m + most - 1) / most;
    g.rr = R;
    g.mb = (m + nb - 1) / nb;
    g.nr = 1;
  } else {
    const int nr = (R + kMaxRows - 1) / kMaxRows;
    g.rr = ((R + nr - 1) / nr + 15) / 16 * 16;
    g.mb = 1;
    g.nr = (R + g.rr - 1) / g.rr;
  }
  g.nrb = (m + g.mb - 1) / g.mb * g.nr;
  g.by_n_kv = FastDiv(g.n_kv);
  g.by_m = FastDiv(m);
  g.by_rr = FastDiv(g.rr);
  g.by_mb = FastDiv(g.mb);
  g.by_nr = FastDiv(g.nr);
  g.by_nrb = FastDiv(g.nrb);
  g.by_n_q = FastDiv(n_q);
  g.by_len_div = FastDiv(len_div);
  p.items = static_cast<long long>(I) * g.nrb;
  const long long most = p.items * ((cap + kAtTile - 1) / kAtTile);
  too_large |= most >= (1ll << 31) - sms;
  p.grid = static_cast<int>(most < sms ? most : sms);
  return p;
}

size_t place_parts(AtPlan& p, int d, int sms, size_t at) {
  const AtGeo& g = p.geo;
  size_t parts = static_cast<size_t>(p.items) + sms, rows = static_cast<size_t>(g.mb) * g.rr;
  if (g.R > kMaxRows) {  // room that only grows with the rows, whatever their split rounds to
    rows = kMaxRows;
    parts = static_cast<size_t>(g.I) * g.m * ((g.R + kMaxRows - 1) / kMaxRows) + sms;
  }
  p.off_o = at;
  at = align_up(at + parts * rows * d * sizeof(float));
  p.off_ml = at;
  at = align_up(at + parts * rows * sizeof(float2));
  p.off_span = at;
  at = align_up(at + static_cast<size_t>(p.items) * sizeof(int2));
  p.off_cut = at;
  return align_up(at + static_cast<size_t>(sms) * sizeof(int2));
}

// What the weights need that are recomputed from the keys.
size_t place_weights(AtLayout& l, const Shape& s, size_t at) {
  l.off_wpart = at;
  at = align_up(at + static_cast<size_t>(2 * l.sms) * kAtTile * sizeof(float));
  l.off_wu0 = at;
  return align_up(at + static_cast<size_t>(weights_items(s) + 1) * sizeof(int));
}

struct MergeArgs {
  AtGeo own, pre;
  AtParts own_parts, pre_parts;
  int has_prefix;
  int row_blocks;
  float sc;
  __nv_bfloat16* o;
  float* lse;
  float* lse2;
  const float* logits;
  float* weights;
  FastDiv by_row_blocks, by_key_blocks;  // blocks per item, and blocks of kMergeKeys keys per instance
  int own_items, own_ctas, pre_ctas;     // what items and CTAs that device data names are checked against
  int* err;
};

// The run of a row's parts in one source: n of them, `step` segments' rows apart in ml and o.
struct Run {
  const float2* ml;
  const float* o;
  int n, rows;
};

__device__ __forceinline__ Run make_run(const AtParts& p, int2 span, int item, int c, int d, int ctas, int* err) {
  if (!in_bounds(span.x, ctas, err) || !in_bounds(span.y, ctas, err) || !in_bounds(span.y - span.x, ctas, err))
    return {nullptr, nullptr, 0, 0};
  const size_t at = static_cast<size_t>(span.x + item) * p.rows + c;
  return {p.ml + at, p.o + at * d, span.y - span.x + 1, p.rows};
}

// Row r of own instance e in the prefix; no parts where there is none.
__device__ __forceinline__ Run prefix_run(const MergeArgs& a, int e, int r, int d) {
  if (!a.has_prefix) return {nullptr, nullptr, 0, 0};
  const AtGeo& q = a.pre;
  int b, group, bq, rb;
  const int kv = q.by_n_kv.mod(e, b), bb = q.by_m.mod(b, group), pe = group * q.n_kv + kv;
  const int bi = q.by_mb.mod(bb, bq), c = q.by_rr.mod(r, rb), item = pe * q.nrb + bq * q.nr + rb;
  return make_run(a.pre_parts, a.pre_parts.span[item], item, bi * q.rr + c, d, a.pre_ctas, a.err);
}

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Part i of a row, counting the prefix's parts first: its (reference, sum of p); l = 0 past the last.
__device__ __forceinline__ float2 part_ml(const Run& pre, const Run& own, int i) {
  const float2* at = i < pre.n ? pre.ml + static_cast<size_t>(i) * pre.rows
                               : own.ml + static_cast<size_t>(i - pre.n) * own.rows;
  return i < pre.n + own.n ? __ldcg(at) : make_float2(0.f, 0.f);
}

// log2 of the sum of the parts' l 2^m; -inf when no part saw a key.  The whole warp; `mine` is part
// `lane`, the parts past the 32nd are read here.
__device__ __noinline__ float merged_lse2(Run pre, Run own, float2 mine, int lane) {
  const int n = pre.n + own.n;
  float top = mine.y != 0.f ? mine.x : -INFINITY;
#pragma unroll 1
  for (int i = 32 + lane; i - lane < n; i += 32) {
    const float2 v = part_ml(pre, own, i);
    if (v.y != 0.f) top = fmaxf(top, v.x);
  }
  top = warp_max(top);
  if (top == -INFINITY) top = 0.f;
  float sum = mine.y != 0.f ? mine.y * ex2_approx(mine.x - top) : 0.f;
#pragma unroll 1
  for (int i = 32 + lane; i - lane < n; i += 32) {
    const float2 v = part_ml(pre, own, i);
    if (v.y != 0.f) sum += v.y * ex2_approx(v.x - top);
  }
  sum = warp_sum(sum);
  return sum == 0.f ? -INFINITY : top + log2f(sum);
}

template <int D>
__global__ void __launch_bounds__(kMergeThreads, 4) merge_kernel(MergeArgs a) {
  constexpr int kPer = D / 32, U = 4;  // parts of O under way at a time
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const AtGeo& g = a.own;
  grid_dependents_go();
  grid_dependency_wait();
  if (static_cast<int>(blockIdx.x) < a.row_blocks) {
    // kMergeRows rows of an item of the own caches to a block, one to a warp: of every item where there is a
    // prefix, else of those that a CTA began and did not finish
    int x;
    const int c = a.by_row_blocks.mod(blockIdx.x, x) * kMergeRows + warp;
    const int2 cut = a.has_prefix ? make_int2(x, 0) : a.own_parts.cut[x];
    if (cut.x < 0 || !in_bounds(cut.x, a.own_items, a.err)) return;
    int e;
    const int r = g.by_nrb.mod(cut.x, e) * g.rr + c;
    if (c >= g.rr || r >= g.R) return;
    const Run own = make_run(a.own_parts, a.has_prefix ? a.own_parts.span[x] : make_int2(x, cut.y), cut.x, c, D,
                             a.own_ctas, a.err);
    const Run pre = prefix_run(a, e, r, D);
    const int n = pre.n + own.n;
    float2 mine = part_ml(pre, own, lane);
    const float lse2 = merged_lse2(pre, own, mine, lane);
    float o[kPer] = {};
#pragma unroll 1
    for (int base = 0; base < n; base += 32) {
      if (base > 0) mine = part_ml(pre, own, base + lane);
      const float w = mine.y == 0.f || lse2 == -INFINITY ? 0.f : ex2_approx(mine.x - lse2);
#pragma unroll 1
      for (int i = base; i < min(n, base + 32); i += U) {
        float f[U][kPer];
#pragma unroll
        for (int y = 0; y < U; ++y) {
          const int j = i + y;
          const float* src = lane + (j < pre.n ? pre.o + static_cast<size_t>(j) * pre.rows * D
                                               : own.o + static_cast<size_t>(j - pre.n) * own.rows * D);
#pragma unroll
          for (int z = 0; z < kPer; ++z) f[y][z] = j < n ? __ldcg(src + z * 32) : 0.f;
        }
#pragma unroll
        for (int y = 0; y < U; ++y) {
          const float wi = __shfl_sync(0xffffffffu, w, (i + y) & 31);
#pragma unroll
          for (int z = 0; z < kPer; ++z) o[z] = i + y < n && wi != 0.f ? fmaf(f[y][z], wi, o[z]) : o[z];
        }
      }
    }
    const size_t row = static_cast<size_t>(e) * g.R + r;
#pragma unroll
    for (int z = 0; z < kPer; ++z) a.o[row * D + z * 32 + lane] = __float2bfloat16(o[z]);
    if (lane == 0) {
      a.lse2[row] = lse2;
      if (a.lse) a.lse[row] = lse2 * 0.69314718055994531f;
    }
    return;
  }
  // ---- weights from the kept logits: one block per instance and run of keys
  constexpr int kMostRows = kLogitRows > kLogitRows4 ? kLogitRows : kLogitRows4;
  __shared__ float lse2_sh[kMostRows];
  __shared__ int seen_sh[kMostRows];
  int e;
  const int j0 = a.by_key_blocks.mod(blockIdx.x - a.row_blocks, e) * kMergeKeys + tid;
  // loads that need no normaliser, under way while it is computed: the first kAhead rows
  constexpr int kKeys = kMergeKeys / kMergeThreads, kAhead = 4;
  const float* y = a.logits + static_cast<size_t>(e) * g.R * g.cap;
  float* weights = a.weights + static_cast<size_t>(e) * g.cap;
  float sum[kKeys], ahead[kAhead][kKeys];
#pragma unroll
  for (int x = 0; x < kKeys; ++x) {
    const int j = j0 + x * kMergeThreads;
    sum[x] = j < g.cap ? weights[j] : 0.f;
#pragma unroll
    for (int r = 0; r < kAhead; ++r)
      ahead[r][x] = j < g.cap && r < g.R ? __ldcg(y + static_cast<size_t>(r) * g.cap + j) : 0.f;
  }
  const int len = at_len(g, e);
  if (j0 - tid >= len) return;
#pragma unroll 1
  for (int r = warp; r < g.R; r += kMergeThreads / 32) {
    int rb;
    const int c = g.by_rr.mod(r, rb), item = e * g.nrb + rb;  // one sequence to a block
    const Run own = make_run(a.own_parts, a.own_parts.span[item], item, c, D, a.own_ctas, a.err),
              pre = prefix_run(a, e, r, D);
    const float v = pre.n + own.n > 1 || a.has_prefix ? merged_lse2(pre, own, part_ml(pre, own, lane), lane)
                                                      : a.lse2[static_cast<size_t>(e) * g.R + r];
    if (lane == 0) {
      lse2_sh[r] = v;
      seen_sh[r] = min(len, len - g.n_q + 1 + g.by_n_q.mod(r));
    }
  }
  __syncthreads();
  float add[kKeys] = {};
#pragma unroll
  for (int r = 0; r < kAhead; ++r) {
    if (r < g.R) {
      const float lse2 = lse2_sh[r];
      const int seen = seen_sh[r];
#pragma unroll
      for (int x = 0; x < kKeys; ++x)
        if (j0 + x * kMergeThreads < seen) add[x] += ex2_approx(fmaf(ahead[r][x], a.sc, -lse2));
    }
  }
#pragma unroll 1
  for (int r0 = kAhead; r0 < g.R; r0 += kAhead) {  // as many rows' loads under way again
    float next[kAhead][kKeys];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int x = 0; x < kKeys; ++x) {
        const int r = r0 + u, j = j0 + x * kMergeThreads;
        next[u][x] = r < g.R && j < g.cap ? __ldcg(y + static_cast<size_t>(r) * g.cap + j) : 0.f;
      }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (r0 + u < g.R) {
        const float lse2 = lse2_sh[r0 + u];
        const int seen = seen_sh[r0 + u];
#pragma unroll
        for (int x = 0; x < kKeys; ++x)
          if (j0 + x * kMergeThreads < seen) add[x] += ex2_approx(fmaf(next[u][x], a.sc, -lse2));
      }
    }
  }
#pragma unroll
  for (int x = 0; x < kKeys; ++x) {
    const int j = j0 + x * kMergeThreads;
    if (j < len) weights[j] = sum[x] + add[x];
  }
}

// The same for many rows in few parts, without a prefix or kept logits: four rows of an unfinished item to a
// warp, eight lanes for the parts of each while the normalisers are computed, all lanes along D for the sums.
template <int D>
__global__ void __launch_bounds__(kMergeThreads, 3) merge_rows_kernel(MergeArgs a) {
  constexpr int RW = kMergeWarpRows, P = 32 / RW, kPer = D / 32, U = 2;
  using Vec = std::conditional_t<kPer == 4, float4, float2>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane / P, slot = lane % P;
  const AtGeo& g = a.own;
  grid_dependents_go();
  grid_dependency_wait();
  int x;
  const int c0 = (a.by_row_blocks.mod(blockIdx.x, x) * (kMergeThreads / 32) + warp) * RW, c = c0 + sub;
  const int2 cut = a.own_parts.cut[x];
  if (cut.x < 0 || !in_bounds(cut.x, a.own_items, a.err)) return;
  int e;
  const int r0 = g.by_nrb.mod(cut.x, e) * g.rr, rows = min(g.rr, g.R - r0);  // of the row block
  if (c0 >= rows) return;
  const Run run = make_run(a.own_parts, make_int2(x, cut.y), cut.x, c0, D, a.own_ctas, a.err);
  const int n = run.n, part = run.rows;
  const bool mine = c < rows;
  auto ml = [&](int i) {
    return mine && i < n ? __ldcg(run.ml + static_cast<size_t>(i) * part + sub) : make_float2(0.f, 0.f);
  };
  const float2 v0 = ml(slot);
  float top = v0.y != 0.f ? v0.x : -INFINITY;
#pragma unroll 1
  for (int i = P + slot; i - slot < n; i += P) {
    const float2 v = ml(i);
    if (v.y != 0.f) top = fmaxf(top, v.x);
  }
#pragma unroll
  for (int o = P / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (top == -INFINITY) top = 0.f;
  float sum = v0.y != 0.f ? v0.y * ex2_approx(v0.x - top) : 0.f;
#pragma unroll 1
  for (int i = P + slot; i - slot < n; i += P) {
    const float2 v = ml(i);
    if (v.y != 0.f) sum += v.y * ex2_approx(v.x - top);
  }
#pragma unroll
  for (int o = P / 2; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  const float lse2 = sum == 0.f ? -INFINITY : top + log2f(sum);
  const size_t row0 = static_cast<size_t>(e) * g.R + r0 + c0;
  if (mine && slot == 0) {
    a.lse2[row0 + sub] = lse2;
    if (a.lse) a.lse[row0 + sub] = lse2 * 0.69314718055994531f;
  }
  float o[RW][kPer] = {};
  float w = 0.f;
  const Vec* src = reinterpret_cast<const Vec*>(run.o) + lane;
#pragma unroll 1
  for (int i = 0; i < n; i += U) {
    if (i % P == 0) {
      const float2 v = i == 0 ? v0 : ml(i + slot);
      w = v.y == 0.f || lse2 == -INFINITY ? 0.f : ex2_approx(v.x - lse2);
    }
    Vec f[U][RW];
#pragma unroll
    for (int y = 0; y < U; ++y)
#pragma unroll
      for (int k = 0; k < RW; ++k)
        if (i + y < n && c0 + k < rows) f[y][k] = __ldcg(src + (static_cast<size_t>(i + y) * part + k) * (D / kPer));
#pragma unroll
    for (int y = 0; y < U; ++y) {
#pragma unroll
      for (int k = 0; k < RW; ++k) {
        const float wi = __shfl_sync(0xffffffffu, w, k * P + (i + y) % P);
        if (i + y < n && wi != 0.f) {
          const float* v = reinterpret_cast<const float*>(&f[y][k]);
#pragma unroll
          for (int z = 0; z < kPer; ++z) o[k][z] = fmaf(v[z], wi, o[k][z]);
        }
      }
    }
  }
#pragma unroll
  for (int k = 0; k < RW; ++k) {
    if (c0 + k < rows) {
      uint32_t* dst = reinterpret_cast<uint32_t*>(a.o + (row0 + k) * D) + lane * (kPer / 2);
#pragma unroll
      for (int z = 0; z < kPer; z += 2) dst[z / 2] = pack_bf16(o[k][z], o[k][z + 1]);
    }
  }
}

}  // namespace

size_t attend4_workspace(const Shape& s, int n_q, bool weights) {
  size_t most = attend4_layout(s, n_q, weights).bytes;
  for (int n = 1; n < n_q && n <= kMaxRows; ++n) most = std::max(most, attend4_layout(s, n, weights).bytes);
  return most;
}

size_t attend_workspace(const Shape& s, int n_q, int groups, bool weights) {
  size_t most = attend_layout(s, n_q, groups, 1, weights).bytes;
  for (int n = 1; n < n_q && n <= kMaxRows; ++n) most = std::max(most, attend_layout(s, n, groups, 1, weights).bytes);
  return most;
}

AtLayout attend_layout(const Shape& s, int n_q, int groups, int pcap, bool weights) {
  AtLayout l;
  const int sms = l.sms = device_sms();
  const int R = s.G * n_q;
  l.own = make_plan(s, s.batch * s.n_kv, 1, R, n_q, true, s.cap, 1, sms, l.too_large);
  size_t at = place_parts(l.own, s.d, sms, 0);
  l.has_prefix = groups > 0;
  if (l.has_prefix) {
    l.prefix = make_plan(s, groups * s.n_kv, s.batch / groups, R, n_q, false, pcap, s.n_kv, sms,
                         l.too_large);
    at = place_parts(l.prefix, s.d, sms, at);
  }
  const size_t rows = static_cast<size_t>(s.batch) * s.n_kv * R;
  l.off_lse2 = at;
  at = align_up(at + rows * sizeof(float));
  l.logits = weights && R <= kLogitRows;
  l.off_logits = at;
  if (l.logits) at = align_up(at + rows * s.cap * sizeof(float));
  if (weights && !l.logits) at = place_weights(l, s, at);
  l.bytes = at;
  return l;
}

AtLayout attend4_layout(const Shape& s, int n_q, bool weights) {
  AtLayout l;
  const int sms = l.sms = device_sms();
  const int R = s.G * n_q;
  const size_t rows = static_cast<size_t>(s.batch) * s.n_kv * R;
  if (R > (weights ? kLogitRows4 : kRows4[s.d == 128])) {
    l.unpacked = true;
    // the rows kernel of k_attend_rows.cuh, whatever the rows
    l.own = make_plan(s, s.batch * s.n_kv, 1, R, n_q, true, s.cap, 1, sms, l.too_large, R <= kMaxRows ? kMaxRows : 0);
    size_t at = place_parts(l.own, s.d, sms, 0);
    l.off_lse2 = at;
    at = align_up(at + rows * sizeof(float));
    if (weights) at = place_weights(l, s, at);
    const size_t cache = align_up(static_cast<size_t>(s.batch) * s.n_kv * s.cap * s.d * 2);
    l.off_k = at;
    l.off_k_rest = l.off_k + cache;
    l.off_v = l.off_k_rest + cache;
    l.off_q = l.off_v + cache;
    l.off_row_sc = align_up(l.off_q + rows * s.d * 2);
    l.bytes = align_up(l.off_row_sc + rows * sizeof(float));
    return l;
  }
  l.four = true;
  l.own = make_plan(s, s.batch * s.n_kv, 1, R, n_q, true, s.cap, 1, sms, l.too_large, kBlockRows4);
  size_t at = place_parts(l.own, s.d, sms, 0);
  l.off_lse2 = at;
  at = align_up(at + rows * sizeof(float));
  l.logits = weights;
  l.off_logits = at;
  if (l.logits) at = align_up(at + rows * s.cap * sizeof(float));
  l.bytes = at;
  return l;
}

namespace {

// With a window: whether every item is one CTA's, which writes its rows' results, with no merge after it.  An even
// split shares the tiles among all SMs, and then costs a second launch that joins the parts.  Where `lost` counts the
// tiles by which an item is longer than an even share, a call over long caches, head_dim 128, even and whole: lost 1.6
// (128 items, window 1024) 4 rows 26.7 and 22.5 us; 2.6 (96 items, window 512) 8 rows 22.5 and 16.4, 128 rows 41.0 and
// 32.8 us; 2.8 (8 items, window 128) 4 rows 14.4 and 12.3; 3.2 (32 items, window 128) 64 rows 19.5 and 20.4, 128 rows
// 22.5 and 27.6; 9.5 (8 items, window 1024) 8 rows 16.4 and 18.4 us.  Sequences much shorter than the window would make
// an even share smaller than what is known here, so windows of many tiles are split as well.
constexpr int kWholeTiles = 12, kWholeLost = 3;
bool whole_items(const AttendArgs& a, const AtLayout& l) {
  const AtPlan& p = l.own;
  if (a.window <= 0 || p.items > l.sms) return false;
  const int span = std::min(p.geo.n_q, p.geo.rr);  // queries of a row block
  const int tiles = (std::min(a.n_sink, p.geo.cap) + kAtTile - 1) / kAtTile + (a.window + span + kAtTile - 2) / kAtTile;
  return tiles <= kWholeTiles && tiles * (l.sms - p.items) <= kWholeLost * l.sms;
}

}  // namespace

cudaError_t launch_attend(const Shape& s, const AttendArgs& a, const AtLayout& l, cudaStream_t st) {
  float* lse2 = reinterpret_cast<float*>(a.ws + l.off_lse2);
  float* logits = l.logits ? reinterpret_cast<float*>(a.ws + l.off_logits) : nullptr;
  const bool whole = whole_items(a, l);
  auto tiles = [&](AtPlan p, const __nv_bfloat16* K, const __nv_bfloat16* V, const int* len, bool own) {
    CUtensorMap qmap, kmap, vmap;
    const AtGeo& g = p.geo;
    const uint64_t rows = static_cast<uint64_t>(g.I) * g.cap;
    if (encode_queries_bf16(&qmap, a.q, s.batch, s.n_kv, g.R, s.d, g.mb, g.rr) != CUDA_SUCCESS ||
        encode_rows_bf16(&kmap, K, rows, s.d, kAtTile) != CUDA_SUCCESS ||
        encode_rows_bf16(&vmap, V, rows, s.d, kAtTile) != CUDA_SUCCESS)
      return cudaErrorInvalidValue;
    AtKernelArgs k{};
    k.geo = g;
    k.geo.len = len;
    k.parts = p.parts(a.ws);
    k.whole_is_final = !l.has_prefix;
    k.sc = a.sc;
    k.o = a.o;
    k.lse = a.lse;
    k.lse2 = lse2;
    k.logits = own ? logits : nullptr;
    k.err = a.err;
    k.after_prefix = own && l.has_prefix;
    if (a.K_rest) {
      k.row_sc = a.row_sc;
      CUtensorMap restmap;
      if (encode_rows_bf16(&restmap, a.K_rest, rows, s.d, kAtTile) != CUDA_SUCCESS) return cudaErrorInvalidValue;
      return launch_attend_rows_split(s.d, p, qmap, kmap, restmap, vmap, k, st);
    }
    if (a.window > 0) {
      if (whole) p.grid = static_cast<int>(p.items);
      k.geo.whole = whole;
      k.geo.window = a.window;
      k.geo.n_sink = a.n_sink;
      if (g.mb * g.rr > kAtTile) return launch_attend_rows_window(s.d, p, qmap, kmap, vmap, k, st);
      AtSinkMaps<true> sink;
      if (encode_rows_bf16(&sink.k, K, rows, s.d, kSinkRows) != CUDA_SUCCESS ||
          encode_rows_bf16(&sink.v, V, rows, s.d, kSinkRows) != CUDA_SUCCESS)
        return cudaErrorInvalidValue;
      return s.d == 128 ? launch_attend_window_128(p, qmap, kmap, vmap, sink, k, st)
                        : launch_attend_window_64(p, qmap, kmap, vmap, sink, k, st);
    }
    if (g.mb * g.rr > kAtTile) return launch_attend_rows(s.d, p, qmap, kmap, vmap, k, st);
    return s.d == 128 ? launch_attend_tiles_128(p, qmap, kmap, vmap, k, st)
                      : launch_attend_tiles_64(p, qmap, kmap, vmap, k, st);
  };
  cudaError_t e = cudaSuccess;
  if (l.has_prefix && (e = tiles(l.prefix, a.Kp, a.Vp, a.plen, false)) != cudaSuccess) return e;
  if ((e = tiles(l.own, a.K, a.V, a.len, true)) != cudaSuccess) return e;
  return cudaSuccess;
}

cudaError_t launch_attend_merge(const Shape& s, const AttendArgs& a, const AtLayout& l, cudaStream_t st) {
  if (whole_items(a, l)) return cudaSuccess;  // nothing to join
  MergeArgs m{};
  m.own = l.own.geo;
  m.own.len = a.len;
  m.own_parts = l.own.parts(a.ws);
  m.has_prefix = l.has_prefix;
  if (l.has_prefix) {
    m.pre = l.prefix.geo;
    m.pre.len = a.plen;
    m.pre_parts = l.prefix.parts(a.ws);
    m.pre_ctas = l.prefix.grid;
  }
  m.own_items = static_cast<int>(l.own.items);
  m.own_ctas = l.own.grid;
  m.err = a.err;
  // Many rows in few parts are bound by the instructions of a row, few rows in many parts by the latency of a
  // part; with merge_rows_kernel an item has 8 parts at most on average.  A call with it and with merge_kernel,
  // head_dim 128: a prompt of 4096 tokens, 32 heads 143 and 153 us; 128 caches of 4224 keys, 256 rows 72 and 82,
  // 128 rows 60 and 64, 44 rows 50 and 51 us; 32 caches of 8320 keys, 256 rows 46 and 50, 128 rows 41 and 42 us; 24
  // of them, 256 rows 40.5 and 43.5, 128 rows 37 and 37 us; 16 caches of 16384 keys, 256 rows 48 and 49, 128 rows 43
  // and 41 us; 8 caches of 32768 keys, 256 rows 53 and 49, 128 rows 47 and 42, 44 rows 33.5 and 33 us.
  const bool many_rows = !l.has_prefix && !l.logits && 8 * l.own.items >= l.own.grid && l.own.geo.rr > kLogitRows;
  const int block_rows = many_rows ? kMergeRows * kMergeWarpRows : kMergeRows;
  const int per_item = (l.own.geo.rr + block_rows - 1) / block_rows;
  m.by_row_blocks = FastDiv(per_item);
  m.row_blocks = static_cast<int>((l.has_prefix ? l.own.items : l.own.grid) * per_item);
  m.sc = a.sc;
  m.o = a.o;
  m.lse = a.lse;
  m.lse2 = reinterpret_cast<float*>(a.ws + l.off_lse2);
  unsigned blocks = static_cast<unsigned>(m.row_blocks);
  if (l.logits) {
    m.logits = reinterpret_cast<const float*>(a.ws + l.off_logits);
    m.weights = a.weights;
    const int key_blocks = (s.cap + kMergeKeys - 1) / kMergeKeys;
    m.by_key_blocks = FastDiv(key_blocks);
    blocks += static_cast<unsigned>(l.own.geo.I) * key_blocks;
  }
  const auto kernel = many_rows ? (s.d == 128 ? merge_rows_kernel<128> : merge_rows_kernel<64>)
                                : (s.d == 128 ? merge_kernel<128> : merge_kernel<64>);
  return launch_after(kernel, blocks, kMergeThreads, 0, st, m);
}

}  // namespace bkv
