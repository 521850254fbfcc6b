// Eviction by accumulated attention weight: selection of the kept rows and
// compaction of K, V and the weights, one CTA per instance.
//
// Selection.  Each warp owns a contiguous run of rows, 32 at a time across its
// lanes, and holds their weights in registers, so the weights are read once.
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
// already stand where they belong.
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

// One digit of the radix select: among the candidates that match `prefix` under `mask`, finds the
// digit that holds the k-th largest (k >= 1, at most the number of matches) and what is left of k
// inside it.  Called by the whole block; the result is the same in every thread.
template <int THREADS, int KPT, int BITS>
__device__ __forceinline__ void select_digit(const uint32_t (&key)[KPT], int c_lo, int c_hi, int row0, int rpw, int shift,
                                             uint32_t& prefix, uint32_t& mask, uint32_t& k, uint32_t* hist,
                                             uint32_t* wsum, uint32_t* found) {
  constexpr int kBins = 1 << BITS;
  constexpr int kPer = (kBins + THREADS - 1) / THREADS;
  const int tid = threadIdx.x, lane = tid & 31;
  for (int i = tid; i < kBins; i += THREADS) hist[i] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < KPT; ++i) {
    const int j = row0 + i * 32 + lane;
    if (i * 32 < rpw && j >= c_lo && j < c_hi && (key[i] & mask) == prefix)
      atomicAdd(&hist[(key[i] >> shift) & (kBins - 1)], 1u);
  }
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

// KPT * THREADS rows at most per instance.
template <int D, int THREADS, int KPT>
__global__ void __launch_bounds__(THREADS) evict_kernel(Shape s, EvictArgs a) {
  constexpr int kWarps = THREADS / 32;
  extern __shared__ __align__(16) uint16_t kept_s[];  // [min(budget, cap)] kept rows (cap <= 32768)
  __shared__ uint32_t hist[kEvBins];
  __shared__ uint32_t wsum[kWarps], found[2];
  __shared__ uint32_t w_tie[kWarps], w_keep[kWarps];
  __shared__ int first_sh;

  const int e = blockIdx.x;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  int L = a.L[e];
  int* kept_e = a.kept + static_cast<size_t>(e) * a.budget;
  if (L < 0 || L > s.cap) {  // the whole block
    for (int i = tid; i < a.budget; i += THREADS) kept_e[i] = -1;
    __syncthreads();  // len_out may be L itself
    if (tid == 0) {
      record_error(a.err, kDevBadLength);
      if (a.len_out) a.len_out[e] = 0;
    }
    return;
  }
  const bool in_place = a.K_out == a.K;
  const float* w_in = a.weights + static_cast<size_t>(e) * s.cap;
  float* w_out = a.weights_out + static_cast<size_t>(e) * a.cap_out;
  const int n_keep = min(L, a.budget);

  // this warp's rows: row0 + 32 i + lane, rpw of them (a multiple of 32)
  const int rpw = (L + kWarps * 32 - 1) / (kWarps * 32) * 32;
  const int row0 = warp * rpw;
  float w[KPT];
  uint32_t key[KPT];
#pragma unroll
  for (int i = 0; i < KPT; ++i) {
    const int j = row0 + i * 32 + lane;
    w[i] = i * 32 < rpw && j < L ? w_in[j] : 0.f;
    key[i] = weight_key(w[i]);
  }
  if (tid == 0) first_sh = n_keep;
  uint32_t T = 0, ties = 0;
  const int c_lo = s.n_prefix, c_hi = L - s.W;
  const bool all = L <= a.budget;
  const int k_sel = a.budget - s.n_prefix - s.W;
  if (!all && k_sel > 0) {
    uint32_t prefix = 0, mask = 0, k = static_cast<uint32_t>(k_sel);
    select_digit<THREADS, KPT, 12>(key, c_lo, c_hi, row0, rpw, 20, prefix, mask, k, hist, wsum, found);
    select_digit<THREADS, KPT, 10>(key, c_lo, c_hi, row0, rpw, 10, prefix, mask, k, hist, wsum, found);
    select_digit<THREADS, KPT, 10>(key, c_lo, c_hi, row0, rpw, 0, prefix, mask, k, hist, wsum, found);
    T = prefix;
    ties = k;
  }
  // 0: not kept, 1: kept, 2: kept if it is among the first `ties` rows equal to T
  auto kind = [&](int i) -> int {
    const int j = row0 + i * 32 + lane;
    if (i * 32 >= rpw || j >= L) return 0;
    if (all || j < c_lo || j >= c_hi) return 1;
    if (k_sel <= 0) return 0;
    return key[i] > T ? 1 : (key[i] == T ? 2 : 0);
  };
  uint32_t n_tie = 0, n_sure = 0;
#pragma unroll
  for (int i = 0; i < KPT; ++i) {
    const int c = kind(i);
    n_tie += __popc(__ballot_sync(0xffffffffu, c == 2));
    n_sure += __popc(__ballot_sync(0xffffffffu, c == 1));
  }
  if (lane == 0) {
    w_tie[warp] = n_tie;
    w_keep[warp] = n_sure;
  }
  __syncthreads();  // every weight has been read: the outputs may be the inputs
  uint32_t tie_at = 0, at = 0;
  for (int v = 0; v < warp; ++v) {
    const uint32_t t = w_tie[v];
    at += w_keep[v] + min(t, ties > tie_at ? ties - tie_at : 0u);
    tie_at += t;
  }
  const uint32_t below = (1u << lane) - 1u;
#pragma unroll
  for (int i = 0; i < KPT; ++i) {
    const int c = kind(i);
    const uint32_t tie_mask = __ballot_sync(0xffffffffu, c == 2);
    const bool keep = c == 1 || (c == 2 && tie_at + __popc(tie_mask & below) < ties);
    const uint32_t keep_mask = __ballot_sync(0xffffffffu, keep);
    const int j = row0 + i * 32 + lane;
    const int pos = static_cast<int>(at + __popc(keep_mask & below));
    if (keep && in_bounds(pos, n_keep, a.err)) {
      kept_s[pos] = static_cast<uint16_t>(j);
      kept_e[pos] = j;
      w_out[pos] = w[i];
      if (pos != j) atomicMin(&first_sh, pos);  // rows before it stand where they belong
    }
    tie_at += __popc(tie_mask);
    at += __popc(keep_mask);
  }
  for (int i = n_keep + tid; i < a.budget; i += THREADS) kept_e[i] = -1;
  for (int i = n_keep + tid; i < a.cap_out; i += THREADS) w_out[i] = 0.f;
  __syncthreads();
  if (tid == 0 && a.len_out) a.len_out[e] = n_keep;

  // ---------------------------------------------------------------- gather
  constexpr int kVpr = D * 2 / 16;    // 16-byte vectors per row of one tensor
  constexpr int kRowVec = 2 * kVpr;   // K row, then V row
  constexpr int kPer = 8;             // vectors per thread and chunk
  constexpr int kRowsPerPass = THREADS / kRowVec;
  constexpr int kChunkRows = kRowsPerPass * kPer;
  const int col = tid % kRowVec, r0 = tid / kRowVec;
  const int vcol = col < kVpr ? col : col - kVpr;
  const uint4* src = reinterpret_cast<const uint4*>((col < kVpr ? a.K : a.V) + static_cast<size_t>(e) * s.cap * D) + vcol;
  uint4* dst = reinterpret_cast<uint4*>((col < kVpr ? a.K_out : a.V_out) + static_cast<size_t>(e) * a.cap_out * D) + vcol;
  const int first = in_place ? first_sh : 0;

  uint4 cur[kPer], nxt[kPer];
  auto load_chunk = [&](int i0, uint4 (&R)[kPer]) {
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int row = i0 + r0 + kRowsPerPass * u;
      if (row < n_keep) {
        int from = kept_s[row];
        if (!in_bounds(from - row, L - row, a.err)) from = row;  // row <= kept[row] < L
        R[u] = __ldcg(src + static_cast<size_t>(from) * kVpr);
      }
    }
  };
  if (first < n_keep) load_chunk(first, cur);
  for (int i0 = first; i0 < n_keep; i0 += kChunkRows) {
    if (in_place) __syncthreads();  // every load of this chunk was issued before any of its stores
    const int i1 = i0 + kChunkRows;
    if (i1 < n_keep) load_chunk(i1, nxt);
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int row = i0 + r0 + kRowsPerPass * u;
      if (row < n_keep) dst[static_cast<size_t>(row) * kVpr] = cur[u];
    }
#pragma unroll
    for (int u = 0; u < kPer; ++u) cur[u] = nxt[u];
  }
}

template <int D, int THREADS, int KPT>
cudaError_t launch(const Shape& s, const EvictArgs& a, cudaStream_t st) {
  const int smem = (a.budget < s.cap ? a.budget : s.cap) * static_cast<int>(sizeof(uint16_t));
  const cudaError_t e = cudaFuncSetAttribute(evict_kernel<D, THREADS, KPT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  evict_kernel<D, THREADS, KPT><<<s.n_inst, THREADS, smem, st>>>(s, a);
  return cudaGetLastError();
}

// The capacity decides how many rows a CTA must be able to hold in registers.
template <int D>
cudaError_t launch_d(const Shape& s, const EvictArgs& a, cudaStream_t st) {
  if (s.cap <= 256 * 8) return launch<D, 256, 8>(s, a, st);
  if (s.cap <= 512 * 20) return launch<D, 512, 20>(s, a, st);
  static_assert(kMaxCapacity <= 1024 * 32, "rows of the largest capacity in registers");
  return launch<D, 1024, 32>(s, a, st);
}

}  // namespace

cudaError_t launch_evict(const Shape& s, const EvictArgs& a, cudaStream_t st) {
  return s.d == 128 ? launch_d<128>(s, a, st) : launch_d<64>(s, a, st);
}

}  // namespace bkv
