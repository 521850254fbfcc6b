// Eviction by accumulated attention weight: selection of the kept rows and
// compaction of K, V and the weights.
//
// Selection, one CTA per instance.  Each warp owns a contiguous run of rows, 32 at
// a time across its lanes; the keys stay in shared memory (in registers the passes
// would have to be unrolled, and a short kernel pays for every instruction that it
// fetches).  A three-pass radix select (digits of 12, 10 and 10 bits from the top, one shared histogram) finds the
// key T of the last row that is kept by weight and how many rows equal to T are needed.
// A 12-bit first digit splits an octave into 8 bins: weights that span a few octaves,
// as softmax sums do, then spread over enough bins that the histogram's atomics seldom
// meet.  Kept rows are numbered in index order by ballots inside each warp and one scan
// of the warps' totals; rows equal to T are taken in index order.
//
// Compaction, a launch of its own.  Row i receives row kept[i] >= i.  Into other
// buffers the rows are independent and move in small blocks spread over all SMs.  In
// place an instance has one CTA, which takes its rows in ascending chunks: all loads of
// a chunk are issued before the barrier that precedes its stores, and they touch only
// rows that no earlier chunk writes; rows before the first evicted one already stand
// where they belong.  The weights move with the rows.
//
// Bound by HBM: the kept rows are read and written once (8 d bytes a row), the
// weights read (4 bytes a cached row) and written.  head_dim 128, cold: 1024 instances of
// 4224 rows to 4096, selection 35.5 us, rows 604 us, 4.3 GB at 7.1 TB/s (1.05 of the measured copy
// rate), in place 701 us for the whole call; 320 instances of 1..32768 rows to 2048, 47.5 and
// 95.5 us (the selection there is one CTA of 1024 threads to an SM, in 2.1 waves).
#include "bkv_device.cuh"
#include "bkv_internal.h"
#include "k_launch.cuh"

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
  uint32_t w = lane < kWarps ? wsum[lane] : 0;  // every warp scans the warps' totals
#pragma unroll
  for (int o = 1; o < kWarps; o <<= 1) {
    const uint32_t n = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += n;
  }
  total = __shfl_sync(0xffffffffu, w, kWarps - 1);
  const uint32_t upto = __shfl_sync(0xffffffffu, w, warp);  // this warp's total among them
  const uint32_t before = upto - __shfl_sync(0xffffffffu, incl, 31);
  __syncthreads();  // wsum may be written again
  return before + incl - v;
}

// The rows of one warp: row0 + 32 i + lane for i < n, and their keys in shared memory.
struct WarpRows {
  uint32_t* key;
  int row0, n, lane, L;
  __device__ __forceinline__ void init(const float* w) {
    constexpr int kBatch = 8;  // loads under way
#pragma unroll 1
    for (int i0 = 0; i0 < n; i0 += kBatch) {
      float v[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int j = row0 + (i0 + u) * 32 + lane;
        v[u] = j < L ? w[j] : 0.f;
      }
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int j = row0 + (i0 + u) * 32 + lane;
        if (i0 + u < n && j < L) key[j] = weight_key(v[u]);
      }
    }
    __syncwarp();
  }
  // inner(row, key) for 32 rows that are all candidates, [c_lo, c_hi); edge(row, key) for the others, also
  // where a row is not below L (every lane takes part).
  template <typename F, typename G>
  __device__ __forceinline__ void each(int c_lo, int c_hi, F&& inner, G&& edge) const {
#pragma unroll 2
    for (int i = 0; i < n; ++i) {
      const int j = row0 + i * 32;
      if (j >= c_lo && j + 32 <= c_hi) inner(j + lane, key[j + lane]);
      else edge(j + lane, j + lane < L ? key[j + lane] : 0u);
    }
  }
};

// One digit of the radix select: among the candidates [c_lo, c_hi) that match `prefix` under `mask`,
// finds the digit that holds the k-th largest (k >= 1, at most the number of matches) and what is left
// of k inside it.  Called by the whole block; the result is the same in every thread.
template <int THREADS, int BITS>
__device__ __forceinline__ void select_digit(const WarpRows& rows, int c_lo, int c_hi, int shift, uint32_t& prefix,
                                             uint32_t& mask, uint32_t& k, uint32_t* hist, uint32_t* wsum,
                                             uint32_t* found) {
  constexpr int kBins = 1 << BITS;
  constexpr int kPer = kBins / THREADS >= 4 ? kBins / THREADS : 4;  // bins per thread, from the top
  const int tid = threadIdx.x;
  for (int i = tid; i < kBins; i += THREADS) hist[i] = 0;
  __syncthreads();
  auto count = [&](uint32_t key) {
    if ((key & mask) == prefix) atomicAdd(&hist[(key >> shift) & (kBins - 1)], 1u);
  };
  rows.each(c_lo, c_hi, [&](int, uint32_t key) { count(key); },
            [&](int j, uint32_t key) {
              if (j >= c_lo && j < c_hi) count(key);
            });
  __syncthreads();
  uint32_t loc[kPer], sum = 0;
#pragma unroll
  for (int i = 0; i < kPer; i += 4) {
    const int b = kBins - 4 - (tid * kPer + i);  // descending digits, four at a time
    const uint4 v = b >= 0 ? *reinterpret_cast<const uint4*>(hist + b) : make_uint4(0, 0, 0, 0);
    loc[i] = v.w;
    loc[i + 1] = v.z;
    loc[i + 2] = v.y;
    loc[i + 3] = v.x;
    sum += v.x + v.y + v.z + v.w;
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

// Selection: kept, len_out, into other buffers the zeros of weights_out, and in `plan` the number of kept
// rows (-1 for a length out of range) and the first of them that has to move.
template <int THREADS>
__global__ void __launch_bounds__(THREADS, 2048 / THREADS) evict_select_kernel(Shape s, EvictArgs a) {
  extern __shared__ uint32_t keys[];  // [cap]
  constexpr int kWarps = THREADS / 32;
  __shared__ __align__(16) uint32_t hist[kEvBins];
  __shared__ uint32_t wsum[kWarps], found[2];
  __shared__ uint32_t w_tie[kWarps], w_keep[kWarps];
  __shared__ int first_sh;
  const int e = blockIdx.x;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  grid_dependents_go();
  const int L = a.L[e];
  int* kept_e = a.kept + static_cast<size_t>(e) * a.budget;
  if (L < 0 || L > s.cap) {  // the whole block
    for (int i = tid; i < a.budget; i += THREADS) kept_e[i] = -1;
    __syncthreads();  // len_out may be L itself
    if (tid == 0) {
      record_error(a.err, kDevBadLength);
      if (a.len_out) a.len_out[e] = 0;
      a.plan[e] = make_int2(-1, 0);
    }
    return;
  }
  const bool in_place = a.K_out == a.K;
  const float* w_in = a.weights + static_cast<size_t>(e) * s.cap;
  float* w_out = a.weights_out + static_cast<size_t>(e) * a.cap_out;
  const int n_keep = min(L, a.budget);

  WarpRows rows;
  rows.key = keys;
  rows.L = L;
  rows.n = (L + kWarps * 32 - 1) / (kWarps * 32);
  rows.row0 = warp * rows.n * 32;
  rows.lane = lane;
  rows.init(w_in);
  if (tid == 0) first_sh = n_keep;
  uint32_t T = 0, ties = 0;
  const int c_lo = s.n_prefix, c_hi = L - s.W;
  const bool all = L <= a.budget;
  const int k_sel = a.budget - s.n_prefix - s.W;
  if (!all && k_sel > 0) {
    uint32_t prefix = 0, mask = 0, k = static_cast<uint32_t>(k_sel);
    select_digit<THREADS, 12>(rows, c_lo, c_hi, 20, prefix, mask, k, hist, wsum, found);
    select_digit<THREADS, 10>(rows, c_lo, c_hi, 10, prefix, mask, k, hist, wsum, found);
    select_digit<THREADS, 10>(rows, c_lo, c_hi, 0, prefix, mask, k, hist, wsum, found);
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
  const int in_lo = all || k_sel <= 0 ? L : c_lo;  // no inner rows where nothing is selected by weight
  rows.each(in_lo, c_hi,
            [&](int, uint32_t key) {
              n_tie += key == T;
              n_sure += key > T;
            },
            [&](int j, uint32_t key) {
              const int c = kind(j, key);
              n_tie += c == 2;
              n_sure += c == 1;
            });
  n_tie = __reduce_add_sync(0xffffffffu, n_tie);
  n_sure = __reduce_add_sync(0xffffffffu, n_sure);
  if (lane == 0) {
    w_tie[warp] = n_tie;
    w_keep[warp] = n_sure;
  }
  __syncthreads();
  uint32_t tie_at = 0, at = 0;
#pragma unroll 1
  for (int v = 0; v < warp; ++v) {
    const uint32_t t = w_tie[v];
    at += w_keep[v] + min(t, ties > tie_at ? ties - tie_at : 0u);
    tie_at += t;
  }
  const uint32_t below = (1u << lane) - 1u;
  bool moves = false;  // a row of this warp that has to move was seen
  auto put = [&](int j, bool sure, bool tie) {
    bool keep = sure;
    if (n_tie) {
      const uint32_t tie_mask = __ballot_sync(0xffffffffu, tie);
      keep = sure || (tie && tie_at + __popc(tie_mask & below) < ties);
      tie_at += __popc(tie_mask);
    }
    const uint32_t keep_mask = __ballot_sync(0xffffffffu, keep);
    const int pos = static_cast<int>(at + __popc(keep_mask & below));
    if (keep && in_bounds(pos, n_keep, a.err)) kept_e[pos] = j;
    if (!moves) {  // rows before the first one that moves stand where they belong
      const uint32_t m = __ballot_sync(0xffffffffu, keep && pos != j);
      if (m) {
        moves = true;
        if (lane == __ffs(m) - 1) atomicMin(&first_sh, pos);
      }
    }
    at += __popc(keep_mask);
  };
  rows.each(in_lo, c_hi, [&](int j, uint32_t key) { put(j, key > T, key == T); },
            [&](int j, uint32_t key) {
              const int c = kind(j, key);
              put(j, c == 1, c == 2);
            });
  for (int i = n_keep + tid; i < a.budget; i += THREADS) kept_e[i] = -1;
  if (!in_place)
    for (int i = n_keep + tid; i < a.cap_out; i += THREADS) w_out[i] = 0.f;
  __syncthreads();
  if (tid == 0) {
    if (a.len_out) a.len_out[e] = n_keep;
    a.plan[e] = make_int2(n_keep, first_sh);
  }
}

// Compaction in place: one CTA per instance, the next chunk under way while one is written.
template <int D, int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) evict_move_in_place_kernel(Shape s, EvictArgs a) {
  constexpr int kVpr = D * 2 / 16;    // 16-byte vectors per row of one tensor
  constexpr int kRowVec = 2 * kVpr;   // K row, then V row
  constexpr int kPer = 4;             // vectors per thread and chunk, one chunk ahead
  constexpr int kRowsPerPass = kThreads / kRowVec;
  constexpr int kChunkRows = kRowsPerPass * kPer;
  static_assert(kChunkRows <= kThreads, "one weight per thread and chunk");
  const int e = blockIdx.x, tid = threadIdx.x;
  grid_dependency_wait();
  const int2 plan = a.plan[e];
  if (plan.x < 0 || !in_bounds(plan.x, min(a.budget, s.cap) + 1, a.err) || !in_bounds(plan.y, plan.x + 1, a.err)) return;
  const int first = plan.y, end = plan.x;
  const int* kept = a.kept + static_cast<size_t>(e) * a.budget;
  const int col = tid % kRowVec, r0 = tid / kRowVec;
  const int vcol = col < kVpr ? col : col - kVpr;
  uint4* base = reinterpret_cast<uint4*>((col < kVpr ? a.K_out : a.V_out) + static_cast<size_t>(e) * s.cap * D) + vcol;
  float* weights = a.weights_out + static_cast<size_t>(e) * s.cap;

  uint4 cur[kPer], nxt[kPer];
  float w_cur = 0.f, w_nxt = 0.f;
  auto load_chunk = [&](int i0, uint4 (&R)[kPer], float& w) {
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int row = i0 + r0 + kRowsPerPass * u;
      if (row < end) {
        int j = __ldcg(kept + row);
        if (!in_bounds(j - row, s.cap - row, a.err)) j = row;  // row <= kept[row] < cap
        R[u] = __ldcg(base + static_cast<size_t>(j) * kVpr);
      }
    }
    if (tid < kChunkRows && i0 + tid < end) {
      int j = __ldcg(kept + i0 + tid);
      if (!in_bounds(j, s.cap, a.err)) j = i0 + tid;
      w = __ldcg(weights + j);
    }
  };
  if (first < end) load_chunk(first, cur, w_cur);
  for (int i0 = first; i0 < end; i0 += kChunkRows) {
    __syncthreads();  // every load of this chunk was issued before any of its stores
    const int i1 = i0 + kChunkRows;
    if (i1 < end) load_chunk(i1, nxt, w_nxt);
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int row = i0 + r0 + kRowsPerPass * u;
      if (row < end) base[static_cast<size_t>(row) * kVpr] = cur[u];
    }
    if (tid < kChunkRows && i0 + tid < end) weights[i0 + tid] = w_cur;
#pragma unroll
    for (int u = 0; u < kPer; ++u) cur[u] = nxt[u];
    w_cur = w_nxt;
  }
  __syncthreads();  // the last kept weights have been read
  for (int i = end + tid; i < s.cap; i += kThreads) weights[i] = 0.f;
}

// Compaction into other buffers: kMoveRows rows of an instance to a block.
constexpr int kMoveRows = 64, kMoveThreads = 256;
template <int D>
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(Shape s, EvictArgs a, int chunks) {
  constexpr int kVpr = D * 2 / 16, kRowVec = 2 * kVpr, kPer = kMoveRows * kRowVec / kMoveThreads;
  __shared__ int rows[kMoveRows];
  const int e = blockIdx.x / chunks, i0 = blockIdx.x % chunks * kMoveRows;
  const int tid = threadIdx.x;
  grid_dependency_wait();
  const int kept = a.plan[e].x;
  if (kept >= 0 && !in_bounds(kept, min(a.budget, s.cap) + 1, a.err)) return;
  const int n = min(kMoveRows, kept - i0);
  if (tid < kMoveRows) rows[tid] = tid < n ? __ldcg(a.kept + static_cast<size_t>(e) * a.budget + i0 + tid) : 0;
  if (n <= 0) return;
  __syncthreads();
  const int col = tid % kRowVec, r0 = tid / kRowVec;
  const int vcol = col < kVpr ? col : col - kVpr;
  const uint4* src = reinterpret_cast<const uint4*>((col < kVpr ? a.K : a.V) + static_cast<size_t>(e) * s.cap * D) + vcol;
  uint4* dst = reinterpret_cast<uint4*>((col < kVpr ? a.K_out : a.V_out) +
                                        (static_cast<size_t>(e) * a.cap_out + i0) * D) + vcol;
  const bool mine = tid < n;  // one weight per thread
  float w = 0.f;
  if (mine) {
    int j = rows[tid];
    if (!in_bounds(j, s.cap, a.err)) j = i0 + tid;
    w = a.weights[static_cast<size_t>(e) * s.cap + j];
  }
  uint4 R[kPer];
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int r = r0 + u * (kMoveThreads / kRowVec);
    if (r < n) {
      int j = rows[r];
      if (!in_bounds(j, s.cap, a.err)) j = i0 + r;
      R[u] = __ldcg(src + static_cast<size_t>(j) * kVpr);
    }
  }
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int r = r0 + u * (kMoveThreads / kRowVec);
    if (r < n) dst[static_cast<size_t>(r) * kVpr] = R[u];
  }
  if (mine) a.weights_out[static_cast<size_t>(e) * a.cap_out + i0 + tid] = w;
}

// More threads for more rows.  A call with 256, 512 and 1024 threads, 4.3 M rows in all: instances of 1088 rows
// 51, 63 and 94 us; of 2048 rows 45, 46 and 60; of 4224 rows 47, 45 and 52; of 10240 rows 50, 44 and 45 us;
// 2.1 M rows, instances of 16384 rows 58, 46 and 41 us, of 32768 rows 86, 62 and 50 us.
template <int THREADS>
cudaError_t select(const Shape& s, const EvictArgs& a, cudaStream_t st) {
  const size_t smem = sizeof(uint32_t) * s.cap;
  if (smem > 30 * 1024) {  // with the static 17 KB past the 48 KB that need no opt-in
    const cudaError_t e = allow_smem<evict_select_kernel<THREADS>>(sizeof(uint32_t) * kMaxCapacity);
    if (e != cudaSuccess) return e;
  }
  evict_select_kernel<THREADS><<<s.n_inst, THREADS, smem, st>>>(s, a);
  return cudaGetLastError();
}

template <int D>
cudaError_t launch_d(const Shape& s, const EvictArgs& a, cudaStream_t st) {
  const cudaError_t e = s.cap <= 2048    ? select<256>(s, a, st)
                        : s.cap <= 10240 ? select<512>(s, a, st)
                                         : select<1024>(s, a, st);
  if (e != cudaSuccess) return e;
  if (a.K_out == a.K) {
    // An instance's rows move in order, so its block has as many threads as still let the blocks of all
    // instances be on the SMs at once, 1024 threads of 64 registers on each.  A call with blocks of 512 threads,
    // and of this rule's: 16 instances, 32768 rows to 2048, 73 and 60 us; 4224 rows to 4096, 128 instances 138 and
    // 110 us, 384 instances 343 and 318, 1024 instances 762 and 701, 4608 instances 3216 and 3095 us.
    const int sms = device_sms();
    const auto move = [&](auto kernel, int threads) { return launch_after(kernel, s.n_inst, threads, 0, st, s, a); };
    return s.n_inst <= sms       ? move(evict_move_in_place_kernel<D, 1024>, 1024)
           : s.n_inst <= 2 * sms ? move(evict_move_in_place_kernel<D, 512>, 512)
           : s.n_inst <= 4 * sms ? move(evict_move_in_place_kernel<D, 256>, 256)
                                 : move(evict_move_in_place_kernel<D, 128>, 128);
  }
  const int kept = a.budget < s.cap ? a.budget : s.cap, chunks = (kept + kMoveRows - 1) / kMoveRows;
  return launch_after(evict_move_kernel<D>, static_cast<unsigned>(s.n_inst) * chunks, kMoveThreads, 0, st, s, a, chunks);
}

}  // namespace

cudaError_t launch_evict(const Shape& s, const EvictArgs& a, cudaStream_t st) {
  return s.d == 128 ? launch_d<128>(s, a, st) : launch_d<64>(s, a, st);
}

}  // namespace bkv
