// Attention of the newest queries over a sequence's cache and, with a shared
// prefix, over the prefix of its group (include/bkv.h, bkv_attend): the plan of
// a call, its workspace, and the merge of the partial results.
//
// k_attend_tiles.cu leaves, for every part of an item that one CTA worked on, the
// sums O_p = sum p v and l_p = sum p of each row against a reference m_p (p = 2^(y -
// m_p), y the base-2 logits).  A row's result over all its parts is
//   lse2 = log2 sum_p l_p 2^(m_p),   o = sum_p O_p 2^(m_p - lse2),
// taken in the parts' order, a warp to a row.  A row that one CTA finished is
// already written.  The same launch adds the attention weights where the logits
// were kept: weights[j] += sum over rows of 2^(y - lse2).
#include "k_attend.cuh"

namespace bkv {
namespace {

constexpr int kMergeThreads = 256;
constexpr int kMergeKeys = 1024;   // keys per block of the weights' part
constexpr int kLogitRows = 16;      // rows per instance up to which logits are kept for the weights

size_t align_up(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

static int attend_sms() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
      n < 1) {
    cudaGetLastError();
    return 152;
  }
  return n;
}

namespace {

// Row blocks of m sequences x R rows: all rows of an instance in one block while there are at most 128
// of them, else blocks of at most 256, as even as 16-row steps allow.
AtPlan make_plan(const Shape& s, int I, int m, int R, int n_q, bool causal, int cap, int len_div, int sms,
                 bool& too_large) {
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
  const int most_rows = 1ll * R * m <= 128 ? 128 : 256;
  if (R <= most_rows) {
    const int most = most_rows / R, nb = (m + most - 1) / most;
    g.rr = R;
    g.mb = (m + nb - 1) / nb;
    g.nr = 1;
  } else {
    const int nr = (R + 255) / 256;
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
  const size_t parts = static_cast<size_t>(p.items) + sms, rows = static_cast<size_t>(p.geo.mb) * p.geo.rr;
  p.off_o = at;
  at = align_up(at + parts * rows * d * sizeof(float));
  p.off_ml = at;
  at = align_up(at + parts * rows * sizeof(float2));
  p.off_span = at;
  at = align_up(at + static_cast<size_t>(p.items) * sizeof(int2));
  p.off_cut = at;
  return align_up(at + static_cast<size_t>(sms) * sizeof(int));
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
};

// The run of a row's parts in one source: n of them, `step` segments' rows apart in ml and o.
struct Run {
  const float2* ml;
  const float* o;
  int n, rows;
};

__device__ __forceinline__ Run make_run(const AtParts& p, int2 span, int item, int c, int d) {
  const size_t at = static_cast<size_t>(span.x + item) * p.rows + c;
  return {p.ml + at, p.o + at * d, span.y - span.x + 1, p.rows};
}

// Row r of own instance e in the own caches, and in the prefix.
__device__ __forceinline__ Run own_run(const MergeArgs& a, int e, int r, int d) {
  int rb;
  const int c = a.own.by_rr.mod(r, rb), item = e * a.own.nrb + rb;
  return make_run(a.own_parts, a.own_parts.span[item], item, c, d);
}
__device__ __forceinline__ Run prefix_run(const MergeArgs& a, int e, int r, int d) {
  const AtGeo& q = a.pre;
  int b, group, bq, rb;
  const int kv = q.by_n_kv.mod(e, b), bb = q.by_m.mod(b, group), pe = group * q.n_kv + kv;
  const int bi = q.by_mb.mod(bb, bq), c = q.by_rr.mod(r, rb), item = pe * q.nrb + bq * q.nr + rb;
  return make_run(a.pre_parts, a.pre_parts.span[item], item, bi * q.rr + c, d);
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

__device__ __forceinline__ float2 part_ml(const Run& u, int i) {
  return i < u.n ? __ldcg(u.ml + static_cast<size_t>(i) * u.rows) : make_float2(0.f, 0.f);
}

// Parts of a row that a lane holds: part `lane` of its run in each source; l = 0 stands for none.
struct Held {
  float2 own, pre;
};
__device__ __forceinline__ float held_top(float2 v) { return v.y != 0.f ? v.x : -INFINITY; }
__device__ __forceinline__ float held_sum(float2 v, float top) { return v.y != 0.f ? v.y * ex2_approx(v.x - top) : 0.f; }

// log2 of the sum of the parts' l 2^m; -inf when no part saw a key.  The whole warp, a part to a lane;
// `h` holds the first 32 parts of each run, and `pre` has no parts where there is no prefix.
__device__ __forceinline__ float merged_lse2(const Held& h, const Run& own, const Run& pre, int lane) {
  const int n = max(own.n, pre.n);
  float top = fmaxf(held_top(h.own), held_top(h.pre));
#pragma unroll 1
  for (int i = 32 + lane; i - lane < n; i += 32) top = fmaxf(top, fmaxf(held_top(part_ml(own, i)), held_top(part_ml(pre, i))));
  top = warp_max(top);
  if (top == -INFINITY) top = 0.f;
  float sum = held_sum(h.own, top) + held_sum(h.pre, top);
#pragma unroll 1
  for (int i = 32 + lane; i - lane < n; i += 32) sum += held_sum(part_ml(own, i), top) + held_sum(part_ml(pre, i), top);
  sum = warp_sum(sum);
  return sum == 0.f ? -INFINITY : top + log2f(sum);
}

// RPW rows to a warp, U parts of each under way at a time.
template <int D, int RPW, int U>
__global__ void __launch_bounds__(kMergeThreads, 4) merge_kernel(MergeArgs a) {
  constexpr int kPer = D / 32, kRowsPerWarp = RPW, kMergeRows = kMergeThreads / 32 * RPW;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const AtGeo& g = a.own;
  grid_dependents_go();
  grid_dependency_wait();
  if (static_cast<int>(blockIdx.x) < a.row_blocks) {
    // kMergeRows rows of an item of the own caches to a block, kRowsPerWarp to a warp: of every item where
    // there is a prefix, else of those that a CTA began and did not finish
    int x;
    const int c0 = a.by_row_blocks.mod(blockIdx.x, x) * kMergeRows + warp;
    const int item = a.has_prefix ? x : a.own_parts.cut[x];
    if (item < 0) return;
    int e;
    const int r0 = g.by_nrb.mod(item, e) * g.rr;
    Run own[kRowsPerWarp], pre[kRowsPerWarp];
    Held held[kRowsPerWarp];
    float lse2[kRowsPerWarp], o[kRowsPerWarp][kPer] = {};
    int row[kRowsPerWarp], n_own = 0, n_pre = 0;
#pragma unroll
    for (int y = 0; y < kRowsPerWarp; ++y) {  // the rows' loads are under way together
      const int c = c0 + y * (kMergeThreads / 32), r = r0 + c;
      const bool there = c < g.rr && r < g.R;
      row[y] = there ? e * g.R + r : -1;
      own[y] = own_run(a, e, there ? r : r0, D);
      if (a.has_prefix) pre[y] = prefix_run(a, e, there ? r : r0, D);
      else pre[y] = Run{own[y].ml, own[y].o, 0, 0};
      held[y] = {part_ml(own[y], lane), part_ml(pre[y], lane)};
      n_own = max(n_own, own[y].n);
      n_pre = max(n_pre, pre[y].n);
    }
#pragma unroll
    for (int y = 0; y < kRowsPerWarp; ++y) lse2[y] = merged_lse2(held[y], own[y], pre[y], lane);
    // O of the parts, in order: the prefix's, then the own ones
    auto add = [&](const Run(&u)[kRowsPerWarp], int n, bool is_own) {
#pragma unroll 1
      for (int base = 0; base < n; base += 32) {
        float w[kRowsPerWarp];
#pragma unroll
        for (int y = 0; y < kRowsPerWarp; ++y) {
          const float2 v = base == 0 ? (is_own ? held[y].own : held[y].pre) : part_ml(u[y], base + lane);
          w[y] = v.y == 0.f || lse2[y] == -INFINITY ? 0.f : ex2_approx(v.x - lse2[y]);
        }
        const int here = min(32, n - base);
#pragma unroll 1
        for (int i = 0; i < here; i += U) {
          float f[U][kRowsPerWarp][kPer];
#pragma unroll
          for (int v = 0; v < U; ++v)
#pragma unroll
            for (int y = 0; y < kRowsPerWarp; ++y) {
              const bool some = i + v < here && base + i + v < u[y].n;
              const float* src = u[y].o + static_cast<size_t>(base + i + v) * u[y].rows * D + lane;
#pragma unroll
              for (int z = 0; z < kPer; ++z) f[v][y][z] = some ? __ldcg(src + z * 32) : 0.f;
            }
#pragma unroll
          for (int v = 0; v < U; ++v)
#pragma unroll
            for (int y = 0; y < kRowsPerWarp; ++y) {
              const float wi = __shfl_sync(0xffffffffu, w[y], (i + v) & 31);
#pragma unroll
              for (int z = 0; z < kPer; ++z)
                o[y][z] = i + v < here && wi != 0.f ? fmaf(f[v][y][z], wi, o[y][z]) : o[y][z];
            }
        }
      }
    };
    add(pre, n_pre, false);
    add(own, n_own, true);
#pragma unroll
    for (int y = 0; y < kRowsPerWarp; ++y) {
      if (row[y] < 0) continue;
#pragma unroll
      for (int z = 0; z < kPer; ++z) a.o[static_cast<size_t>(row[y]) * D + z * 32 + lane] = __float2bfloat16(o[y][z]);
      if (lane == 0) {
        a.lse2[row[y]] = lse2[y];
        if (a.lse) a.lse[row[y]] = lse2[y] * 0.69314718055994531f;
      }
    }
    return;
  }
  // ---- weights from the kept logits: one block per instance and run of keys
  __shared__ float lse2_sh[kLogitRows];
  __shared__ int seen_sh[kLogitRows];
  int e;
  const int j0 = a.by_key_blocks.mod(blockIdx.x - a.row_blocks, e) * kMergeKeys;
  const int len = at_len(g, e);
  // loads that need no normaliser, under way while it is computed
  constexpr int kKeys = kMergeKeys / kMergeThreads, kAhead = 4;
  const float* y = a.logits + static_cast<size_t>(e) * g.R * g.cap;
  float sum[kKeys], ahead[kAhead][kKeys];
#pragma unroll
  for (int x = 0; x < kKeys; ++x) {
    const int j = j0 + x * kMergeThreads + tid;
    sum[x] = j < g.cap ? a.weights[static_cast<size_t>(e) * g.cap + j] : 0.f;
#pragma unroll
    for (int r = 0; r < kAhead; ++r)
      ahead[r][x] = j < g.cap && r < g.R ? __ldcg(y + static_cast<size_t>(r) * g.cap + j) : 0.f;
  }
  if (j0 >= len) return;
#pragma unroll 1
  for (int r = warp; r < g.R; r += kMergeThreads / 32) {
    const Run own = own_run(a, e, r, D);
    const Run pre = a.has_prefix ? prefix_run(a, e, r, D) : Run{own.ml, own.o, 0, 0};
    const float v = a.has_prefix || own.n > 1 ? merged_lse2({part_ml(own, lane), part_ml(pre, lane)}, own, pre, lane)
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
        if (j0 + x * kMergeThreads + tid < seen) add[x] += ex2_approx(fmaf(ahead[r][x], a.sc, -lse2));
    }
  }
#pragma unroll 1
  for (int r = kAhead; r < g.R; ++r) {
    const float lse2 = lse2_sh[r];
    const int seen = seen_sh[r];
#pragma unroll
    for (int x = 0; x < kKeys; ++x) {
      const int j = j0 + x * kMergeThreads + tid;
      if (j < seen) add[x] += ex2_approx(fmaf(__ldcg(y + static_cast<size_t>(r) * g.cap + j), a.sc, -lse2));
    }
  }
#pragma unroll
  for (int x = 0; x < kKeys; ++x) {
    const int j = j0 + x * kMergeThreads + tid;
    if (j < len) a.weights[static_cast<size_t>(e) * g.cap + j] = sum[x] + add[x];
  }
}

}  // namespace

AtLayout attend_layout(const Shape& s, int n_q, int groups, int pcap, bool weights) {
  AtLayout l;
  const int sms = l.sms = attend_sms();
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
  if (weights && !l.logits) {
    l.off_wpart = at;
    at = align_up(at + static_cast<size_t>(2 * sms) * kAtTile * sizeof(float));
    l.off_wu0 = at;
    at = align_up(at + static_cast<size_t>(weights_items(s) + 1) * sizeof(int));
  }
  l.bytes = at;
  return l;
}

cudaError_t launch_attend(const Shape& s, const AttendArgs& a, const AtLayout& l, cudaStream_t st) {
  float* lse2 = reinterpret_cast<float*>(a.ws + l.off_lse2);
  float* logits = l.logits ? reinterpret_cast<float*>(a.ws + l.off_logits) : nullptr;
  auto tiles = [&](const AtPlan& p, const __nv_bfloat16* K, const __nv_bfloat16* V, const int* len, bool own) {
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
    k.reuse = g.nrb > 1;
    k.sc = a.sc;
    k.o = a.o;
    k.lse = a.lse;
    k.lse2 = lse2;
    k.logits = own ? logits : nullptr;
    k.err = a.err;
    k.after_prefix = own && l.has_prefix;
    if (g.mb * g.rr > 128) return launch_attend_rows(s.d, p, qmap, kmap, vmap, k, st);
    return s.d == 128 ? launch_attend_tiles_128(p, qmap, kmap, vmap, k, st)
                      : launch_attend_tiles_64(p, qmap, kmap, vmap, k, st);
  };
  cudaError_t e = cudaSuccess;
  if (l.has_prefix && (e = tiles(l.prefix, a.Kp, a.Vp, a.plen, false)) != cudaSuccess) return e;
  if ((e = tiles(l.own, a.K, a.V, a.len, true)) != cudaSuccess) return e;
  return cudaSuccess;
}

cudaError_t launch_attend_merge(const Shape& s, const AttendArgs& a, const AtLayout& l, cudaStream_t st) {
  MergeArgs m{};
  m.own = l.own.geo;
  m.own.len = a.len;
  m.own_parts = l.own.parts(a.ws);
  m.has_prefix = l.has_prefix;
  if (l.has_prefix) {
    m.pre = l.prefix.geo;
    m.pre.len = a.plen;
    m.pre_parts = l.prefix.parts(a.ws);
  }
  // Few items are cut into many parts each, of few rows; many items into two or three parts, of many rows.
  const bool many_rows = !l.has_prefix && l.own.items >= l.own.grid;
  const int rows = kMergeThreads / 32 * (many_rows ? 2 : 1);
  const int per_item = (l.own.geo.rr + rows - 1) / rows;
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
  const auto kernel = s.d == 128 ? (many_rows ? merge_kernel<128, 2, 2> : merge_kernel<128, 1, 4>)
                                 : (many_rows ? merge_kernel<64, 2, 2> : merge_kernel<64, 1, 4>);
  return launch_after(kernel, blocks, kMergeThreads, 0, st, m);
}

}  // namespace bkv
