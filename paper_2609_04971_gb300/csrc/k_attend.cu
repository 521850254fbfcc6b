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
constexpr int kMergeRows = 32;      // rows per block: four per warp
constexpr int kMergeKeys = 512;    // keys per block of the weights' part
constexpr int kLogitRows = 16;      // rows per instance up to which logits are kept for the weights

size_t align_up(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

int attend_sms() {
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
AtPlan make_plan(const Shape& s, int I, int m, int R, int n_q, bool causal, int cap, int len_div, int sms) {
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
  p.items = static_cast<long long>(I) * g.nrb;
  const long long most = p.items * ((cap + kAtTile - 1) / kAtTile);
  p.grid = static_cast<int>(most < sms ? most : sms);
  return p;
}

size_t place_parts(AtPlan& p, int d, int sms, size_t at) {
  const size_t parts = static_cast<size_t>(p.items) + sms, rows = static_cast<size_t>(p.geo.mb) * p.geo.rr;
  p.off_o = at;
  at = align_up(at + parts * rows * d * sizeof(float));
  p.off_ml = at;
  at = align_up(at + parts * rows * sizeof(float2));
  p.off_u0 = at;
  at = align_up(at + static_cast<size_t>(p.items) * sizeof(long long));
  p.off_per = at;
  at = align_up(at + sizeof(long long));
  p.off_cut = at;
  return align_up(at + static_cast<size_t>(sms) * sizeof(long long));
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
  int key_blocks;  // blocks of kMergeKeys keys per instance
};

// The parts of one row: own instance e, row r of R.
struct RowParts {
  AtSpan own, pre;
  long long own_item, pre_item;
  int own_c, pre_c;
  bool split;  // more than one part
};

__device__ __forceinline__ RowParts row_parts(const MergeArgs& a, int e, int r) {
  RowParts p;
  const AtGeo& g = a.own;
  const int rb = r / g.rr;
  p.own_item = static_cast<long long>(e) * g.nrb + rb;
  p.own_c = r % g.rr;
  p.own = at_span(a.own_parts, p.own_item, at_tiles(at_limit_max(g, at_len(g, e), rb * g.rr)));
  p.pre = {0, -1};
  p.pre_item = 0;
  p.pre_c = 0;
  if (a.has_prefix) {
    const AtGeo& q = a.pre;
    const int b = e / g.n_kv, bb = b % q.m, pe = b / q.m * g.n_kv + e % g.n_kv;
    p.pre_item = static_cast<long long>(pe) * q.nrb + bb / q.mb * q.nr + r / q.rr;
    p.pre_c = bb % q.mb * q.rr + r % q.rr;
    p.pre = at_span(a.pre_parts, p.pre_item, at_tiles(at_len(q, pe)));
  }
  p.split = a.has_prefix || p.own.first != p.own.last;
  return p;
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

// The parts of a row, a warp at a time: lane x holds part base + x.
struct WarpParts {
  int n_pre, n;
  __device__ __forceinline__ explicit WarpParts(const RowParts& p)
      : n_pre(p.pre.last - p.pre.first + 1), n(n_pre + p.own.last - p.own.first + 1) {}
  // Index of part i in ml, and whether it is the prefix's.
  __device__ __forceinline__ long long at(const MergeArgs& a, const RowParts& p, int i, bool& pre) const {
    pre = i < n_pre;
    return pre ? (p.pre.first + i + p.pre_item) * a.pre_parts.rows + p.pre_c
               : (p.own.first + i - n_pre + p.own_item) * a.own_parts.rows + p.own_c;
  }
  __device__ __forceinline__ float2 ml(const MergeArgs& a, const RowParts& p, int i) const {
    if (i >= n) return make_float2(0.f, 0.f);
    bool pre;
    const long long x = at(a, p, i, pre);
    return pre ? a.pre_parts.ml[x] : a.own_parts.ml[x];
  }
};

// log2 of the sum of the parts' l 2^m; -inf when no part saw a key.  The whole warp.
__device__ __forceinline__ float merged_lse2(const MergeArgs& a, const RowParts& p, const WarpParts& wp, int lane) {
  const float2 mine = wp.ml(a, p, lane);
  float top = mine.y != 0.f ? mine.x : -INFINITY;
  for (int i = 32 + lane; i - lane < wp.n; i += 32) {
    const float2 v = wp.ml(a, p, i);
    if (v.y != 0.f) top = fmaxf(top, v.x);
  }
  top = warp_max(top);
  if (top == -INFINITY) top = 0.f;
  float sum = mine.y != 0.f ? mine.y * exp2f(mine.x - top) : 0.f;
  for (int i = 32 + lane; i - lane < wp.n; i += 32) {
    const float2 v = wp.ml(a, p, i);
    if (v.y != 0.f) sum += v.y * exp2f(v.x - top);
  }
  sum = warp_sum(sum);
  return sum == 0.f ? -INFINITY : top + log2f(sum);
}

template <int D>
__global__ void __launch_bounds__(kMergeThreads, 4) merge_kernel(MergeArgs a) {
  constexpr int kPer = D / 32;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  grid_dependents_go();
  grid_dependency_wait();
  if (static_cast<int>(blockIdx.x) < a.row_blocks) {
    // kMergeRows rows of an item of the own caches to a block: of every item where there is a prefix, else
    // of those that a CTA began and did not finish
    const AtGeo& g = a.own;
    const int per_item = (g.rr + kMergeRows - 1) / kMergeRows;
    const long long x = blockIdx.x / per_item, item = a.has_prefix ? x : a.own_parts.cut[x];
    if (item < 0) return;
    const int e = static_cast<int>(item / g.nrb), r0 = static_cast<int>(item % g.nrb) * g.rr, c1 = min(g.rr, g.R - r0);
    for (int c = blockIdx.x % per_item * kMergeRows + warp, n = 0; c < c1 && n < kMergeRows / 8; c += 8, ++n) {
      const int r = r0 + c;
      const long long row = static_cast<long long>(e) * g.R + r;
      const RowParts p = row_parts(a, e, r);
      const WarpParts wp(p);
      const float lse2 = merged_lse2(a, p, wp, lane);
      float o[kPer] = {};
      // parts in runs of consecutive places, four loads of O under way at a time
      auto run = [&](const AtParts& parts, long long item, int c, int first, int n) {
        const float2* ml = parts.ml + (first + item) * parts.rows + c;
        const float* src = parts.o + ((first + item) * parts.rows + c) * D + lane;
        const size_t step = static_cast<size_t>(parts.rows) * D;
        for (int base = 0; base < n; base += 32) {
          float w = 0.f;
          if (base + lane < n) {
            const float2 v = ml[static_cast<size_t>(base + lane) * parts.rows];
            w = v.y == 0.f || lse2 == -INFINITY ? 0.f : exp2f(v.x - lse2);
          }
          const int here = min(32, n - base);
          for (int i = 0; i < here; i += 4) {
            float v[4][kPer];
#pragma unroll
            for (int y = 0; y < 4; ++y)
#pragma unroll
              for (int x = 0; x < kPer; ++x) v[y][x] = i + y < here ? src[(base + i + y) * step + x * 32] : 0.f;
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const float wi = __shfl_sync(0xffffffffu, w, (i + y) & 31);
#pragma unroll
              for (int x = 0; x < kPer; ++x) o[x] = i + y < here && wi != 0.f ? fmaf(v[y][x], wi, o[x]) : o[x];
            }
          }
        }
      };
      if (a.has_prefix) run(a.pre_parts, p.pre_item, p.pre_c, p.pre.first, p.pre.last - p.pre.first + 1);
      run(a.own_parts, p.own_item, p.own_c, p.own.first, p.own.last - p.own.first + 1);
#pragma unroll
      for (int x = 0; x < kPer; ++x) a.o[row * D + x * 32 + lane] = __float2bfloat16(o[x]);
      if (lane == 0) {
        a.lse2[row] = lse2;
        if (a.lse) a.lse[row] = lse2 * 0.69314718055994531f;
      }
    }
    return;
  }
  // ---- weights from the kept logits: one block per instance and run of keys
  __shared__ float lse2_sh[kLogitRows];
  const int w = blockIdx.x - a.row_blocks;
  const int e = w / a.key_blocks, j0 = w % a.key_blocks * kMergeKeys;
  const AtGeo& g = a.own;
  const int len = at_len(g, e);
  if (j0 >= len) return;
  constexpr int kKeys = kMergeKeys / kMergeThreads, kAhead = 4;
  const float* y = a.logits + static_cast<size_t>(e) * g.R * g.cap;
  float sum[kKeys], ahead[kAhead][kKeys];  // loads that need no normaliser, under way while it is computed
#pragma unroll
  for (int x = 0; x < kKeys; ++x) {
    const int j = j0 + x * kMergeThreads + tid;
    sum[x] = j < len ? a.weights[static_cast<size_t>(e) * g.cap + j] : 0.f;
#pragma unroll
    for (int r = 0; r < kAhead; ++r)
      ahead[r][x] = j < len && r < g.R ? __ldcg(y + static_cast<size_t>(r) * g.cap + j) : 0.f;
  }
  for (int r = warp; r < g.R; r += kMergeThreads / 32) {
    const RowParts p = row_parts(a, e, r);
    const float v = p.split ? merged_lse2(a, p, WarpParts(p), lane) : a.lse2[static_cast<long long>(e) * g.R + r];
    if (lane == 0) lse2_sh[r] = v;
  }
  __syncthreads();
  float add[kKeys] = {};
  auto term = [&](int x, int r, float logit) {
    const int j = j0 + x * kMergeThreads + tid;
    if (j < min(len, len - g.n_q + 1 + r % g.n_q)) add[x] += exp2f(fmaf(logit, a.sc, -lse2_sh[r]));
  };
#pragma unroll
  for (int r = 0; r < kAhead; ++r) {
    if (r < g.R) {
#pragma unroll
      for (int x = 0; x < kKeys; ++x) term(x, r, ahead[r][x]);
    }
  }
  for (int r = kAhead; r < g.R; ++r) {
#pragma unroll
    for (int x = 0; x < kKeys; ++x) {
      const int j = j0 + x * kMergeThreads + tid;
      if (j < len) term(x, r, __ldcg(y + static_cast<size_t>(r) * g.cap + j));
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
  const int sms = attend_sms();
  const int R = s.G * n_q;
  l.own = make_plan(s, s.batch * s.n_kv, 1, R, n_q, true, s.cap, 1, sms);
  size_t at = place_parts(l.own, s.d, sms, 0);
  l.has_prefix = groups > 0;
  if (l.has_prefix) {
    l.prefix = make_plan(s, groups * s.n_kv, s.batch / groups, R, n_q, false, pcap, s.n_kv, sms);
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
    at = align_up(at + static_cast<size_t>(weights_items(s) + 1) * sizeof(long long));
  }
  l.bytes = at;
  return l;
}

bool attend_recomputes_weights(const Shape& s, int n_q) { return s.G * n_q > kLogitRows; }

size_t attend_workspace(const Shape& s, int n_q, int groups, bool weights) {
  return n_q < 1 ? 0 : attend_layout(s, n_q, groups, 1, weights).bytes;
}

cudaError_t launch_attend(const Shape& s, const AttendArgs& a, cudaStream_t st) {
  const AtLayout l = attend_layout(s, a.n_q, a.groups, a.pcap, a.weights != nullptr);
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

cudaError_t launch_attend_merge(const Shape& s, const AttendArgs& a, cudaStream_t st) {
  const AtLayout l = attend_layout(s, a.n_q, a.groups, a.pcap, a.weights != nullptr);
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
  m.row_blocks = static_cast<int>((l.has_prefix ? l.own.items : l.own.grid) *
                                  ((l.own.geo.rr + kMergeRows - 1) / kMergeRows));
  m.sc = a.sc;
  m.o = a.o;
  m.lse = a.lse;
  m.lse2 = reinterpret_cast<float*>(a.ws + l.off_lse2);
  unsigned blocks = static_cast<unsigned>(m.row_blocks);
  if (l.logits) {
    m.logits = reinterpret_cast<const float*>(a.ws + l.off_logits);
    m.weights = a.weights;
    m.key_blocks = (s.cap + kMergeKeys - 1) / kMergeKeys;
    blocks += static_cast<unsigned>(l.own.geo.I) * m.key_blocks;
  }
  return s.d == 128 ? launch_after(merge_kernel<128>, blocks, kMergeThreads, 0, st, m)
                    : launch_after(merge_kernel<64>, blocks, kMergeThreads, 0, st, m);
}

}  // namespace bkv
