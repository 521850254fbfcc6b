// Attention of the newest queries over a sequence's cache and, with a shared
// prefix, over the prefix of its group (include/bkv.h, bkv_attend): the plan of
// a call, its workspace, and the merge of the partial results.
//
// k_attend_tiles.cu leaves, for every part of an item that one CTA worked on, the
// sums O_p = sum p v and l_p = sum p of each row against a reference m_p (p = 2^(y -
// m_p), y the base-2 logits).  A row's result over all its parts is
//   lse2 = log2 sum_p l_p 2^(m_p),   o = sum_p O_p 2^(m_p - lse2),
// taken in the parts' order, one warp per row.  A row that one CTA finished is
// already written.  The same launch adds the attention weights where the logits
// were kept: weights[j] += sum over rows of 2^(y - lse2).
#include "k_attend.cuh"

namespace bkv {
namespace {

constexpr int kMergeThreads = 256;
constexpr int kMergeKeys = 1024;    // keys per block of the weights' part
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

// Row blocks of m sequences x R rows with at most 128 rows each, as even as 16-row steps allow.
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
  if (R <= 128) {
    const int most = 128 / R, nb = (m + most - 1) / most;
    g.rr = R;
    g.mb = (m + nb - 1) / nb;
    g.nr = 1;
  } else {
    const int nr = (R + 127) / 128;
    g.rr = ((R + nr - 1) / nr + 15) / 16 * 16;
    g.mb = 1;
    g.nr = (R + g.rr - 1) / g.rr;
  }
  g.nrb = (m + g.mb - 1) / g.mb * g.nr;
  const int rows = g.mb * g.rr;
  p.n_cols = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
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
  return align_up(at + sizeof(long long));
}

struct MergeArgs {
  AtGeo own, pre;
  AtParts own_parts, pre_parts;
  int has_prefix;
  long long rows;
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

// f(reference, sum of p, partial o or its place) over the parts of a row, in order.
template <typename F>
__device__ __forceinline__ void each_part(const MergeArgs& a, const RowParts& p, F&& f) {
  for (int c = p.pre.first; c <= p.pre.last; ++c) {
    const long long at = (c + p.pre_item) * a.pre_parts.rows + p.pre_c;
    f(a.pre_parts.ml[at], a.pre_parts.o, at);
  }
  for (int c = p.own.first; c <= p.own.last; ++c) {
    const long long at = (c + p.own_item) * a.own_parts.rows + p.own_c;
    f(a.own_parts.ml[at], a.own_parts.o, at);
  }
}

// log2 of the sum of the parts' l 2^m; -inf when no part saw a key.
__device__ __forceinline__ float merged_lse2(const MergeArgs& a, const RowParts& p) {
  float top = -INFINITY;
  each_part(a, p, [&](float2 ml, const float*, long long) {
    if (ml.y != 0.f) top = fmaxf(top, ml.x);
  });
  if (top == -INFINITY) top = 0.f;
  float sum = 0.f;
  each_part(a, p, [&](float2 ml, const float*, long long) {
    if (ml.y != 0.f) sum += ml.y * exp2f(ml.x - top);
  });
  return sum == 0.f ? -INFINITY : top + log2f(sum);
}

template <int D>
__global__ void __launch_bounds__(kMergeThreads) merge_kernel(MergeArgs a) {
  constexpr int kPer = D / 32;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (static_cast<int>(blockIdx.x) < a.row_blocks) {
    const long long row = static_cast<long long>(blockIdx.x) * (kMergeThreads / 32) + warp;
    if (row >= a.rows) return;
    const RowParts p = row_parts(a, static_cast<int>(row / a.own.R), static_cast<int>(row % a.own.R));
    if (!p.split) return;
    const float lse2 = merged_lse2(a, p);
    float o[kPer] = {};
    if (lse2 != -INFINITY) {
      each_part(a, p, [&](float2 ml, const float* src, long long at) {
        if (ml.y == 0.f) return;
        const float w = exp2f(ml.x - lse2);
#pragma unroll
        for (int x = 0; x < kPer; ++x) o[x] = fmaf(src[at * D + x * 32 + lane], w, o[x]);
      });
    }
#pragma unroll
    for (int x = 0; x < kPer; ++x) a.o[row * D + x * 32 + lane] = __float2bfloat16(o[x]);
    if (lane == 0) {
      a.lse2[row] = lse2;
      if (a.lse) a.lse[row] = lse2 * 0.69314718055994531f;
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
  for (int r = warp; r < g.R; r += kMergeThreads / 32) {
    const RowParts p = row_parts(a, e, r);
    const float v = p.split ? merged_lse2(a, p) : a.lse2[static_cast<long long>(e) * g.R + r];
    if (lane == 0) lse2_sh[r] = v;
  }
  __syncthreads();
  const float* y = a.logits + static_cast<size_t>(e) * g.R * g.cap;
#pragma unroll
  for (int x = 0; x < kMergeKeys / kMergeThreads; ++x) {
    const int j = j0 + x * kMergeThreads + tid;
    if (j >= len) break;
    float sum = 0.f;
    for (int r = 0; r < g.R; ++r)
      if (j < len - g.n_q + 1 + r % g.n_q) sum += exp2f(fmaf(__ldcg(y + static_cast<size_t>(r) * g.cap + j), a.sc, -lse2_sh[r]));
    a.weights[static_cast<size_t>(e) * g.cap + j] += sum;
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
    return launch_attend_tiles(s.d, p, qmap, kmap, vmap, k, st);
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
  m.rows = static_cast<long long>(l.own.geo.I) * l.own.geo.R;
  m.row_blocks = static_cast<int>((m.rows + kMergeThreads / 32 - 1) / (kMergeThreads / 32));
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
  if (s.d == 128)
    merge_kernel<128><<<blocks, kMergeThreads, 0, st>>>(m);
  else
    merge_kernel<64><<<blocks, kMergeThreads, 0, st>>>(m);
  return cudaGetLastError();
}

}  // namespace bkv
