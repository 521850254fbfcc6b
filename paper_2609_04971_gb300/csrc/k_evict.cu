// Eviction by accumulated attention weight: selection of the kept rows and
// compaction of K, V and the weights, one CTA per instance.
//
// Selection.  Each warp owns a contiguous run of rows, 32 at a time across its
// lanes.  Up to a capacity of 10240 their keys stay in registers; longer caches
// are read again in each of the five passes, from L1 and L2, which leaves room for
// four CTAs per SM.
// A three-pass radix select (digits of 12, 10 and 10 bits from the top, one
// shared histogram) finds the key T of the last row that is kept by weight and
// how many rows equal to T are needed.  A 12-bit first digit splits an octave
// into 8 bins: weights that span a few octaves, as softmax sums do, then spread
// over enough bins that the histogram's atomics seldom meet.  Kept rows are
// numbered in index order by ballots inside each warp and one scan of the warps'
// totals; rows equal to T are taken in index order.
//
// Compaction.  Row i receives row kept[i] >= i.  Into other buffers the rows are
// independent.  In place they are taken in ascending chunks: all loads of a
// chunk are issued before the barrier that precedes its stores, and they touch
// only rows that no earlier chunk writes; rows before the first evicted one
// already stand where they belong.  The weights move with the rows.
//
// Into other buffers an instance may be worked on by several CTAs, each of which
// repeats the selection and moves its share of the rows.  That fills the GPU when
// there are few instances, and evens out what a last wave of CTAs leaves idle.
//
// Bound by HBM: the kept rows are read and written once (8 d bytes a row), the
// weights read (4 bytes a cached row) and written.
#include "bkv_device.cuh"
#include "bkv_internal.h"

namespace bkv {
namespace {

constexpr int kEvBins = 4096;

// Weights in descending order are keys in descending order; -0 equals 0 and NaN is the largest.
__device__ __forceinline__ uint32_t weight_key(float w) {
  return w != w ? 0xFFFFFFFFu : float_order_key(w + 0.f);
}

// Exclusive sum of v over the block's threads in order; the block's total in `total`.
template <int THREADS>
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* wsum, uint32_t& total) {
  constexpr int kWarps = THREADS / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t n = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += n;
  }
  if (lane == 31) wsum[warp] = incl;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const uint32_t c = wsum[w];
    before += w < warp ? c : 0;
    all += c;
  }
  total = all;
  __syncthreads();  // wsum may be written again
  return before + incl - v;
}

// The rows of one warp: row0 + 32 i + lane for i < n, with their keys in registers (KPT > 0) or read
// again on every use (KPT = 0).
template <int KPT>
struct WarpRows {
  uint32_t key[KPT > 0 ? KPT : 1];
  const float* w;
  int row0, n, L, lane;
  __device__ __forceinline__ int row(int i) const { return row0 + i * 32 + lane; }
  __device__ __forceinline__ void init() {
    if constexpr (KPT > 0) {
#pragma unroll
      for (int i = 0; i < KPT; ++i) key[i] = i < n && row(i) < L ? weight_key(w[row(i)]) : 0;
    }
  }
  // f(row, key) for every i, also where the row is not below L (every lane takes part).
  template <typename F>
  __device__ __forceinline__ void each(F&& f) const {
    if constexpr (KPT > 0) {
#pragma unroll
      for (int i = 0; i < KPT; ++i)
        if (i < n) f(row(i), key[i]);
    } else {
      constexpr int kBatch = 8;  // loads in flight
      for (int i0 = 0; i0 < n; i0 += kBatch) {
        uint32_t k[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int j = row(i0 + u);
          k[u] = i0 + u < n && j < L ? weight_key(w[j]) : 0;
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
          if (i0 + u < n) f(row(i0 + u), k[u]);
      }
    }
  }
};

// One digit of the radix select: among the candidates [c_lo, c_hi) that match `prefix` under `mask`,
// finds the digit that holds the k-th largest (k >= 1, at most the number of matches) and what is left
// of k inside it.  Called by the whole block; the result is the same in every thread.
template <int THREADS, int KPT, int BITS>
__device__ __forceinline__ void select_digit(const WarpRows<KPT>& rows, int c_lo, int c_hi, int shift, uint32_t& prefix,
                                             uint32_t& mask, uint32_t& k, uint32_t* hist, uint32_t* wsum,
                                             uint32_t* found) {
  constexpr int kBins = 1 << BITS;
  constexpr int kPer = (kBins + THREADS - 1) / THREADS;
  const int tid = threadIdx.x;
  for (int i = tid; i < kBins; i += THREADS) hist[i] = 0;
  __syncthreads();
  rows.each([&](int j, uint32_t key) {
    if (j >= c_lo && j < c_hi && (key & mask) == prefix) atomicAdd(&hist[(key >> shift) & (kBins - 1)], 1u);
  });
  __syncthreads();
  uint32_t loc[kPer], sum = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int b = kBins - 1 - (tid * kPer + i);  // descending digits
    loc[i] = b >= 0 ? hist[b] : 0;
    sum += loc[i];
  }
  uint32_t total;
  uint32_t above = block_scan<THREADS>(sum, wsum, total);
  if (above < k && k <= above + sum) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (above < k && k <= above + loc[i]) {
        found[0] = static_cast<uint32_t>(kBins - 1 - (tid * kPer + i));
        found[1] = k - above;
      }
      above += loc[i];
    }
  }
  __syncthreads();
  prefix |= found[0] << shift;
  mask |= static_cast<uint32_t>(kBins - 1) << shift;
  k = found[1];
  __syncthreads();
}

// KPT > 0: at most KPT * THREADS rows per instance.
template <int D, int THREADS, int KPT, int MINB>
__global__ void __launch_bounds__(THREADS, MINB) evict_kernel(Shape s, EvictArgs a, int shares) {
  constexpr int kWarps = THREADS / 32;
  extern __shared__ __align__(16) uint16_t kept_s[];  // [min(budget, cap)] kept rows (cap <= 32768)
  __shared__ uint32_t hist[kEvBins];
  __shared__ uint32_t wsum[kWarps], found[2];
  __shared__ uint32_t w_tie[kWarps], w_keep[kWarps];
  __shared__ int first_sh;

  const int e = blockIdx.x / shares, share = blockIdx.x % shares;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int L = a.L[e];  // len_out may be L itself, but then the instance has one CTA
  int* kept_e = a.kept + static_cast<size_t>(e) * a.budget;
  if (L < 0 || L > s.cap) {  // the whole block
    if (share == 0)
      for (int i = tid; i < a.budget; i += THREADS) kept_e[i] = -1;
    __syncthreads();
    if (tid == 0 && share == 0) {
      record_error(a.err, kDevBadLength);
      if (a.len_out) a.len_out[e] = 0;
    }
    return;
  }
  const bool in_place = a.K_out == a.K;
  const float* w_in = a.weights + static_cast<size_t>(e) * s.cap;
  float* w_out = a.weights_out + static_cast<size_t>(e) * a.cap_out;
  const int n_keep = min(L, a.budget);

  WarpRows<KPT> rows;
  rows.n = (L + kWarps * 32 - 1) / (kWarps * 32);
  rows.row0 = warp * rows.n * 32;
  rows.w = w_in;
  rows.L = L;
  rows.lane = lane;
  rows.init();
  if (tid == 0) first_sh = n_keep;
  uint32_t T = 0, ties = 0;
  const int c_lo = s.n_prefix, c_hi = L - s.W;
  const bool all = L <= a.budget;
  const int k_sel = a.budget - s.n_prefix - s.W;
  if (!all && k_sel > 0) {
    uint32_t prefix = 0, mask = 0, k = static_cast<uint32_t>(k_sel);
    select_digit<THREADS, KPT, 12>(rows, c_lo, c_hi, 20, prefix, mask, k, hist, wsum, found);
    select_digit<THREADS, KPT, 10>(rows, c_lo, c_hi, 10, prefix, mask, k, hist, wsum, found);
    select_digit<THREADS, KPT, 10>(rows, c_lo, c_hi, 0, prefix, mask, k, hist, wsum, found);
    T = prefix;
    ties = k;
  }
  // 0: not kept, 1: kept, 2: kept if it is among the first `ties` rows equal to T
  auto kind = [&](int j, uint32_t key) -> int {
    if (j >= L) return 0;
    if (all || j < c_lo || j >= c_hi) return 1;
    if (k_sel <= 0) return 0;
    return key > T ? 1 : (key == T ? 2 : 0);
  };
  uint32_t n_tie = 0, n_sure = 0;
  rows.each([&](int j, uint32_t key) {
    const int c = kind(j, key);
    n_tie += __popc(__ballot_sync(0xffffffffu, c == 2));
    n_sure += __popc(__ballot_sync(0xffffffffu, c == 1));
  });
  if (lane == 0) {
    w_tie[warp] = n_tie;
    w_keep[warp] = n_sure;
  }
  __syncthreads();
  uint32_t tie_at = 0, at = 0;
  for (int v = 0; v < warp; ++v) {
    const uint32_t t = w_tie[v];
    at += w_keep[v] + min(t, ties > tie_at ? ties - tie_at : 0u);
    tie_at += t;
  }
  const uint32_t below = (1u << lane) - 1u;
  rows.each([&](int j, uint32_t key) {
    const int c = kind(j, key);
    const uint32_t tie_mask = __ballot_sync(0xffffffffu, c == 2);
    const bool keep = c == 1 || (c == 2 && tie_at + __popc(tie_mask & below) < ties);
    const uint32_t keep_mask = __ballot_sync(0xffffffffu, keep);
    const int pos = static_cast<int>(at + __popc(keep_mask & below));
    if (keep && in_bounds(pos, n_keep, a.err)) {
      kept_s[pos] = static_cast<uint16_t>(j);
      if (share == 0) kept_e[pos] = j;
      if (pos != j) atomicMin(&first_sh, pos);  // rows before it stand where they belong
    }
    tie_at += __popc(tie_mask);
    at += __popc(keep_mask);
  });
  if (share == 0)
    for (int i = n_keep + tid; i < a.budget; i += THREADS) kept_e[i] = -1;
  __syncthreads();
  if (tid == 0 && share == 0 && a.len_out) a.len_out[e] = n_keep;

  // ---------------------------------------------------------------- gather
  constexpr int kVpr = D * 2 / 16;    // 16-byte vectors per row of one tensor
  constexpr int kRowVec = 2 * kVpr;   // K row, then V row
  constexpr int kPer = MINB > 1 ? 4 : 8;  // vectors per thread and chunk
  constexpr int kRowsPerPass = THREADS / kRowVec;
  constexpr int kChunkRows = kRowsPerPass * kPer;
  static_assert(kChunkRows <= THREADS, "one weight per thread and chunk");
  const int col = tid % kRowVec, r0 = tid / kRowVec;
  const int vcol = col < kVpr ? col : col - kVpr;
  const uint4* src = reinterpret_cast<const uint4*>((col < kVpr ? a.K : a.V) + static_cast<size_t>(e) * s.cap * D) + vcol;
  uint4* dst = reinterpret_cast<uint4*>((col < kVpr ? a.K_out : a.V_out) + static_cast<size_t>(e) * a.cap_out * D) + vcol;
  const int first = in_place ? first_sh : static_cast<int>(static_cast<long long>(n_keep) * share / shares);
  const int end = in_place ? n_keep : static_cast<int>(static_cast<long long>(n_keep) * (share + 1) / shares);

  uint4 cur[kPer], nxt[kPer];
  float w_cur = 0.f, w_nxt = 0.f;
  auto load_chunk = [&](int i0, uint4 (&R)[kPer], float& w) {
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int row = i0 + r0 + kRowsPerPass * u;
      if (row < end) {
        int from = kept_s[row];
        if (!in_bounds(from - row, L - row, a.err)) from = row;  // row <= kept[row] < L
        R[u] = __ldcg(src + static_cast<size_t>(from) * kVpr);
      }
    }
    if (tid < kChunkRows && i0 + tid < end) {
      int from = kept_s[i0 + tid];
      if (!in_bounds(from, L, a.err)) from = i0 + tid;
      w = __ldcg(w_in + from);
    }
  };
  if (first < end) load_chunk(first, cur, w_cur);
  for (int i0 = first; i0 < end; i0 += kChunkRows) {
    if (in_place) __syncthreads();  // every load of this chunk was issued before any of its stores
    const int i1 = i0 + kChunkRows;
    if (i1 < end) load_chunk(i1, nxt, w_nxt);
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int row = i0 + r0 + kRowsPerPass * u;
      if (row < end) dst[static_cast<size_t>(row) * kVpr] = cur[u];
    }
    if (tid < kChunkRows && i0 + tid < end) w_out[i0 + tid] = w_cur;
#pragma unroll
    for (int u = 0; u < kPer; ++u) cur[u] = nxt[u];
    w_cur = w_nxt;
  }
  if (in_place) __syncthreads();  // the last kept weights have been read
  for (int i = n_keep + share * THREADS + tid; i < a.cap_out; i += shares * THREADS) w_out[i] = 0.f;
}

template <int D, int THREADS, int KPT, int MINB>
cudaError_t launch(const Shape& s, const EvictArgs& a, cudaStream_t st) {
  const int kept = a.budget < s.cap ? a.budget : s.cap;
  const int smem = kept * static_cast<int>(sizeof(uint16_t));
  const cudaError_t e = cudaFuncSetAttribute(evict_kernel<D, THREADS, KPT, MINB>,
                                             cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  // Shares of an instance into other buffers: as many as bring the grid to kShareGrid CTAs, with rows
  // enough for each (a selection costs what a few hundred rows do).
  int shares = 1;
  if (a.K_out != a.K && a.len_out != a.L) {
    constexpr int kShareGrid = 304, kShareRows = 64;
    shares = (kShareGrid + s.n_inst - 1) / s.n_inst;
    if (shares > (kept + kShareRows - 1) / kShareRows) shares = (kept + kShareRows - 1) / kShareRows;
  }
  evict_kernel<D, THREADS, KPT, MINB><<<s.n_inst * shares, THREADS, smem, st>>>(s, a, shares);
  return cudaGetLastError();
}

// The capacity decides whether a CTA can hold an instance's keys in registers.
template <int D>
cudaError_t launch_d(const Shape& s, const EvictArgs& a, cudaStream_t st) {
  if (s.cap <= 256 * 8) return launch<D, 256, 8, 1>(s, a, st);
  if (s.cap <= 512 * 20) return launch<D, 512, 20, 1>(s, a, st);
  return launch<D, 512, 0, 2>(s, a, st);
}

}  // namespace

cudaError_t launch_evict(const Shape& s, const EvictArgs& a, cudaStream_t st) {
  return s.d == 128 ? launch_d<128>(s, a, st) : launch_d<64>(s, a, st);
}

}  // namespace bkv
