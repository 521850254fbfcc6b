// Eviction by accumulated attention weight: selection of the kept rows and
// compaction of K, V and the weights.
//
// Selection, one CTA per instance.  Each warp owns a contiguous run of rows, four to a lane.  A radix select finds the
// key T of the last row that is kept by weight and how many rows equal to T are needed: one pass over the
// weights counts their first digits, a second one marks the rows that these decide, four bits to four rows, and lists
// those that share the first digit of T.  The list is short, so that it alone is searched for the other digits and
// corrects the marks; weights of which more share a digit than the list holds are read in two more
// passes.  A first digit of 12 bits splits an octave into 8 bins: weights that span a few octaves,
// as softmax sums do, then spread over enough bins that the histogram's atomics seldom
// meet.  The marked rows are numbered in index order by scans inside each warp and one scan of the warps' totals;
// rows equal to T are taken in index order.  Bound by instruction issue (2.5 a clock on each SM that has a block).
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
// 4224 rows to 4096, selection 32 us, rows 607 us, 4.3 GB at 7.1 TB/s (1.05 of the measured copy
// rate), in place 684 us for the whole call; 320 instances of 1..32768 rows to 2048, 30.5 and
// 99 us.  4-bit caches (1.25 d bytes a row, moved in vectors of K, V and scales): the same selections, rows 207 us
// (1.34 GB, 6.5 TB/s) and 41.5 us.
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

// The rows of one warp, four to a lane: row0 + 128 i + c for i < n and c < 4, in order over the lanes.  each(f) calls
// f(first row, keys) for them, every lane together; candidates are the rows of [c_lo, c_hi).  The weights are read
// again in every pass: the first one leaves them in L1 and L2, and without a copy in shared memory a block of 1024
// threads has a second one beside it.
struct WarpRows {
  const float* w;
  int row0, n, L, c_lo, c_hi;
  bool aligned;  // to 16 bytes, and an instance's rows a multiple of four
  __device__ __forceinline__ float4 load(int j) const {
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (aligned) {
      if (j < L) v = __ldg(reinterpret_cast<const float4*>(w + j));
    } else {
      if (j < L) v.x = __ldg(w + j);
      if (j + 1 < L) v.y = __ldg(w + j + 1);
      if (j + 2 < L) v.z = __ldg(w + j + 2);
      if (j + 3 < L) v.w = __ldg(w + j + 3);
    }
    return v;
  }
  template <typename F>
  __device__ __forceinline__ void each(F&& f) const {
    float4 next = load(row0);
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
      const int j = row0 + i * 128;
      const float4 v = next;
      if (i + 1 < n) next = load(j + 128);
      const uint32_t key[4] = {weight_key(v.x), weight_key(v.y), weight_key(v.z), weight_key(v.w)};
      f(j, key);
    }
  }
  // One bit to a row of j .. j + 3: which are below `end`, and which are candidates.
  static __device__ __forceinline__ uint32_t below(int j, int end) { return 15u >> min(max(j + 4 - end, 0), 4); }
  __device__ __forceinline__ uint32_t candidates(int j) const { return below(j, c_hi) & ~below(j, c_lo); }
};

// Set bits of the lower lanes' words, and of all lanes'.
__device__ __forceinline__ uint32_t before_lane(uint32_t bits, uint32_t& all) {
  const uint32_t own = __popc(bits);
  uint32_t incl = own;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t n = __shfl_up_sync(0xffffffffu, incl, o);
    if (static_cast<int>(threadIdx.x & 31) >= o) incl += n;
  }
  all = __shfl_sync(0xffffffffu, incl, 31);
  return incl - own;
}

// One digit of the radix select: count(add) calls add(key) for the keys that it may lie in, of which those that match
// `prefix` under `mask` are counted; finds the digit that holds the k-th largest of them (k >= 1, at most
// their number), what is left of k inside it, and how many keys share it.  Called by the whole block; the
// results are the same in every thread.
template <int THREADS, int BITS, typename F>
__device__ __forceinline__ void select_digit(F&& count, int shift, uint32_t& prefix, uint32_t& mask, uint32_t& k,
                                             uint32_t& shared, uint32_t* hist, uint32_t* wsum, uint32_t* found) {
  constexpr int kBins = 1 << BITS;
  constexpr int kPer = kBins / THREADS >= 4 ? kBins / THREADS : 4;  // bins per thread, from the top
  const int tid = threadIdx.x;
  for (int i = 4 * tid; i < kBins; i += 4 * THREADS) *reinterpret_cast<uint4*>(hist + i) = make_uint4(0, 0, 0, 0);
  __syncthreads();
  count([&](uint32_t key) {
    if ((key & mask) == prefix) atomicAdd(&hist[(key >> shift) & (kBins - 1)], 1u);
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
        found[2] = loc[i];
      }
      above += loc[i];
    }
  }
  __syncthreads();
  prefix |= found[0] << shift;
  mask |= static_cast<uint32_t>(kBins - 1) << shift;
  k = found[1];
  shared = found[2];
  __syncthreads();
}

// Rows of an instance that a block has room for: 8 runs of 128 rows to a warp.
template <int THREADS>
constexpr int kMostRows = 32 * THREADS;

// Selection: kept, len_out, into other buffers the zeros of weights_out, and in `plan` the number of kept
// rows (-1 for a length out of range) and the first of them that has to move.
template <int THREADS>
__global__ void __launch_bounds__(THREADS, 2048 / THREADS) evict_select_kernel(Shape s, EvictArgs a) {
  constexpr int kWarps = THREADS / 32, kList = 5 * THREADS / 2;
  constexpr int kLow = 20;  // bits of a key below its first digit
  constexpr uint32_t kLowMask = (1u << kLow) - 1u;
  constexpr uint32_t kRanked = 128;  // keys that are compared with one another
  __shared__ __align__(16) uint32_t hist[kEvBins];
  __shared__ uint32_t list[kList];  // keys with the first digit of T, without it
  __shared__ uint16_t list_row[kList];
  __shared__ __align__(4) uint8_t kinds[kMostRows<THREADS> / 4];  // of rows 4 i .. 4 i + 3: bits kept, bits equal to T
  __shared__ uint32_t wsum[kWarps], found[3], n_list;
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
  const int n_keep = min(L, a.budget);
  if (tid == 0) {
    first_sh = n_keep;
    n_list = 0;
  }
  if (L <= a.budget) {
    for (int j = tid; j < L; j += THREADS) kept_e[j] = j;
  } else {
    WarpRows rows;
    rows.w = a.weights + static_cast<size_t>(e) * s.cap;
    rows.n = (L + kWarps * 128 - 1) / (kWarps * 128);
    rows.row0 = warp * rows.n * 128 + lane * 4;
    rows.L = L;
    rows.aligned = (reinterpret_cast<uintptr_t>(a.weights) & 15) == 0 && (s.cap & 3) == 0;
    rows.c_lo = s.n_prefix;
    rows.c_hi = L - s.W;
    // Of the candidates those above T are kept, and the first `ties` of those equal to it.
    uint32_t T = 0xFFFFFFFFu, ties = 0, in_list = 0;
    uint32_t top = T, low = T;  // keys above top are kept, those from low to top depend on the digits to come
    const int k_sel = a.budget - s.n_prefix - s.W;
    const auto count_rows = [&](auto&& add) {
      rows.each([&](int j, const uint32_t (&key)[4]) {
        const uint32_t candidates = rows.candidates(j);
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (candidates >> c & 1) add(key[c]);
      });
    };
    uint32_t prefix = 0, mask = 0, k = static_cast<uint32_t>(k_sel), shared;
    if (k_sel > 0) {
      static_assert(kLow == 20, "digits of 12, 10 and 10 bits");
      select_digit<THREADS, 12>(count_rows, kLow, prefix, mask, k, shared, hist, wsum, found);
      if (shared <= kList) {
        in_list = shared;
        low = prefix;
        top = prefix | kLowMask;
      } else {
#pragma unroll 1
        for (int shift = 10; shift >= 0; shift -= 10)
          select_digit<THREADS, 10>(count_rows, shift, prefix, mask, k, shared, hist, wsum, found);
        low = top = T = prefix;
        ties = k;
      }
    }
    uint32_t n_tie = 0, n_sure = 0;
    rows.each([&](int j, const uint32_t (&key)[4]) {
      uint32_t above = 0, from = 0;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        above |= static_cast<uint32_t>(key[c] > top) << c;
        from |= static_cast<uint32_t>(key[c] >= low) << c;
      }
      const uint32_t candidates = rows.candidates(j), open = from & ~above & candidates;
      const uint32_t sure = (above & candidates) | (WarpRows::below(j, L) & ~candidates);
      n_sure += __popc(sure);
      kinds[j >> 2] = static_cast<uint8_t>(sure | (in_list ? 0u : open << 4));
      if (open) {
        n_tie += __popc(open);
        if (in_list) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            if (open >> c & 1) {
              const uint32_t at = atomicAdd(&n_list, 1u);
              if (at < kList) {
                list[at] = key[c] & kLowMask;
                list_row[at] = static_cast<uint16_t>(j + c);
              }
            }
          }
        }
      }
    });
    n_tie = __reduce_add_sync(0xffffffffu, n_tie);
    n_sure = __reduce_add_sync(0xffffffffu, n_sure);
    if (lane == 0) {
      w_tie[warp] = in_list ? 0 : n_tie;
      w_keep[warp] = n_sure;
    }
    __syncthreads();
    if (in_list) {
      const uint32_t digit = prefix;
      if (in_list <= kRanked) {
        for (uint32_t i = tid; i < in_list; i += THREADS) {
          const uint32_t mine = list[i];
          uint32_t above = 0, equal = 0;
#pragma unroll 4
          for (uint32_t u = 0; u < in_list; ++u) {
            above += list[u] > mine;
            equal += list[u] == mine;
          }
          if (above < k && k <= above + equal) {
            found[0] = mine;
            found[1] = k - above;
          }
        }
        __syncthreads();
        T = digit | found[0];
        ties = found[1];
      } else {
        const auto count_list = [&](auto&& add) {
          for (uint32_t i = tid; i < in_list; i += THREADS) add(digit | list[i]);
        };
#pragma unroll 1
        for (int shift = 10; shift >= 0; shift -= 10)
          select_digit<THREADS, 10>(count_list, shift, prefix, mask, k, shared, hist, wsum, found);
        T = prefix;
        ties = k;
      }
      const uint32_t run = static_cast<uint32_t>(rows.n) * 128u;
      for (uint32_t i = tid; i < in_list; i += THREADS) {
        const uint32_t key = digit | list[i], row = list_row[i] % kMostRows<THREADS>;
        if (key >= T) {
          const uint32_t bit = (row >> 2 & 3u) * 8u + (row & 3u) + (key > T ? 0u : 4u);
          atomicOr(reinterpret_cast<uint32_t*>(kinds) + (row >> 4), 1u << bit);
          atomicAdd((key > T ? w_keep : w_tie) + min(row / run, kWarps - 1u), 1u);
        }
      }
      __syncthreads();
    }
    // this warp's first place among the kept rows, and the ties before it
    const uint32_t t = lane < kWarps ? w_tie[lane] : 0u;
    uint32_t tie_at = t, at = 0;
#pragma unroll
    for (int o = 1; o < kWarps; o <<= 1) {
      const uint32_t n = __shfl_up_sync(0xffffffffu, tie_at, o);
      if (lane >= o) tie_at += n;
    }
    tie_at -= t;
    const uint32_t kept_w = lane < kWarps ? w_keep[lane] + min(t, ties > tie_at ? ties - tie_at : 0u) : 0u;
    at = __reduce_add_sync(0xffffffffu, lane < warp ? kept_w : 0u);
    tie_at = __shfl_sync(0xffffffffu, tie_at, warp);
    n_tie = __shfl_sync(0xffffffffu, t, warp);

    bool moves = false;  // a row of this warp that has to move was seen
#pragma unroll 1
    for (int i = 0; i < rows.n; ++i) {
      const int j = rows.row0 + i * 128;
      const uint32_t kind = kinds[j >> 2], tie = kind >> 4;
      uint32_t keep = kind & 15u;
      if (n_tie && __any_sync(0xffffffffu, tie)) {
        uint32_t all;
        uint32_t t_at = tie_at + before_lane(tie, all);
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (tie >> c & 1) keep |= static_cast<uint32_t>(t_at++ < ties) << c;
        tie_at += all;
      }
      uint32_t all;
      const int pos = static_cast<int>(at + before_lane(keep, all));
      if (keep && in_bounds(pos + __popc(keep), n_keep + 1, a.err)) {
        int to = pos;
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (keep >> c & 1) kept_e[to++] = j + c;
      }
      if (!moves) {  // rows before the first one that moves stand where they belong
        int first = n_keep, to = pos;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          if (keep >> c & 1) {
            if (to != j + c) first = min(first, to);
            ++to;
          }
        }
        const uint32_t m = __ballot_sync(0xffffffffu, first < n_keep);
        if (m) {
          moves = true;
          if (lane == __ffs(m) - 1) atomicMin(&first_sh, first);
        }
      }
      at += all;
    }
  }
  for (int i = n_keep + tid; i < a.budget; i += THREADS) kept_e[i] = -1;
  if (a.K_out != a.K) {
    float* w_out = a.weights_out + static_cast<size_t>(e) * a.cap_out;
    for (int i = n_keep + tid; i < a.cap_out; i += THREADS) w_out[i] = 0.f;
  }
  __syncthreads();
  if (tid == 0) {
    if (a.len_out) a.len_out[e] = n_keep;
    a.plan[e] = make_int2(n_keep, first_sh);
  }
}

// What a row consists of: vectors of 16 bytes of K, V and, in a 4-bit cache, of the scales.
template <int D, bool FOUR>
struct RowOf {
  static constexpr int kK = FOUR ? D / 32 : D / 8, kS = FOUR ? D / 64 : 0, kVec = 2 * kK + kS;
  // a thread's vector: where it lies in row 0 of instance e's rows, and how many vectors on the next row lies
  template <typename T>
  static __device__ __forceinline__ T* at(T* K, T* V, T* S, int col, size_t row, int& stride) {
    const int c = col < kK ? col : col < 2 * kK ? col - kK : col - 2 * kK;
    stride = FOUR && col >= 2 * kK ? kS : kK;
    return (col < kK ? K : !FOUR || col < 2 * kK ? V : S) + row * stride + c;
  }
};

// 16 bytes of a row, from L2, which fetches 64 bytes with them and not the 128 of its default: a row of a 4-bit cache
// has pieces of 64 and 32 bytes, and what lies beside them may not be kept.  320 instances of 1..32768 rows to 2048,
// 4-bit caches of head_dim 128: 140 MB read and 41.5 us, with the default 228 MB and 51 us.
__device__ __forceinline__ uint4 load_piece(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.cg.L2::64B.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p)
               : "memory");
  return v;
}

// Compaction in place: one CTA per instance, the next chunk under way while one is written.
template <int D, bool FOUR, int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) evict_move_in_place_kernel(Shape s, EvictArgs a) {
  using Row = RowOf<D, FOUR>;
  constexpr int kRowVec = Row::kVec;
  constexpr int kPer = 4;             // vectors per thread and chunk, one chunk ahead
  constexpr int kRowsPerPass = kThreads / kRowVec;  // a rest of the threads may have no rows
  constexpr int kChunkRows = kRowsPerPass * kPer;
  static_assert(kChunkRows <= kThreads, "one weight per thread and chunk");
  const int e = blockIdx.x, tid = threadIdx.x;
  grid_dependency_wait();
  const int2 plan = a.plan[e];
  if (plan.x < 0 || !in_bounds(plan.x, min(a.budget, s.cap) + 1, a.err) || !in_bounds(plan.y, plan.x + 1, a.err)) return;
  const int first = plan.y, end = plan.x;
  const int* kept = a.kept + static_cast<size_t>(e) * a.budget;
  const int col = tid % kRowVec, r0 = tid / kRowVec;
  const int n_rows = r0 < kRowsPerPass ? end : 0;  // rows below it are this thread's to move
  int stride;
  uint4* base = Row::at(static_cast<uint4*>(a.K_out), static_cast<uint4*>(a.V_out), static_cast<uint4*>(a.S_out), col,
                        static_cast<size_t>(e) * s.cap, stride);
  float* weights = a.weights_out + static_cast<size_t>(e) * s.cap;

  uint4 cur[kPer], nxt[kPer];
  float w_cur = 0.f, w_nxt = 0.f;
  auto load_chunk = [&](int i0, uint4 (&R)[kPer], float& w) {
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int row = i0 + r0 + kRowsPerPass * u;
      if (row < n_rows) {
        int j = __ldcg(kept + row);
        if (!in_bounds(j - row, s.cap - row, a.err)) j = row;  // row <= kept[row] < cap
        R[u] = load_piece(base + static_cast<size_t>(j) * stride);
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
      if (row < n_rows) base[static_cast<size_t>(row) * stride] = cur[u];
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
template <int D, bool FOUR>
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(Shape s, EvictArgs a, int chunks) {
  using Row = RowOf<D, FOUR>;
  constexpr int kRowVec = Row::kVec, kPass = kMoveThreads / kRowVec, kPer = (kMoveRows + kPass - 1) / kPass;
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
  const int n_rows = r0 < kPass ? n : 0;
  int stride;
  const uint4* src = Row::at(static_cast<const uint4*>(a.K), static_cast<const uint4*>(a.V),
                             static_cast<const uint4*>(a.S), col, static_cast<size_t>(e) * s.cap, stride);
  uint4* dst = Row::at(static_cast<uint4*>(a.K_out), static_cast<uint4*>(a.V_out), static_cast<uint4*>(a.S_out), col,
                       static_cast<size_t>(e) * a.cap_out + i0, stride);
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
    const int r = r0 + u * kPass;
    if (r < n_rows) {
      int j = rows[r];
      if (!in_bounds(j, s.cap, a.err)) j = i0 + r;
      R[u] = load_piece(src + static_cast<size_t>(j) * stride);
    }
  }
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int r = r0 + u * kPass;
    if (r < n_rows) dst[static_cast<size_t>(r) * stride] = R[u];
  }
  if (mine) a.weights_out[static_cast<size_t>(e) * a.cap_out + i0 + tid] = w;
}

// More threads for more rows.  A call with 256, 512 and 1024 threads, 4-bit caches of head_dim 64, half or more of the
// rows evicted, 4.5 M rows in all: instances of 1088 rows 146, 156 and 212 us; of 2048 rows 125, 130 and 157; of 4224
// rows 122, 123 and 138 (16 instances 21, 18 and 18); of 10240 rows 82 us with 512 and 87 with 1024; 128 instances of
// 16384 rows 43 and 40 us.
template <int THREADS>
cudaError_t select(const Shape& s, const EvictArgs& a, cudaStream_t st) {
  if (s.cap > kMostRows<THREADS>) return cudaErrorInvalidValue;
  evict_select_kernel<THREADS><<<s.n_inst, THREADS, 0, st>>>(s, a);
  return cudaGetLastError();
}

template <int D, bool FOUR>
cudaError_t launch_d(const Shape& s, const EvictArgs& a, cudaStream_t st) {
  const cudaError_t e = s.cap <= 2048    ? select<256>(s, a, st)
                        : s.cap <= 10240 ? select<512>(s, a, st)
                                         : select<1024>(s, a, st);
  if (e != cudaSuccess) return e;
  if (a.K_out == a.K) {
    // An instance's rows move in order, so its block has as many threads as still let the blocks of all
    // instances be on the SMs at once, 1024 threads of 64 registers on each.  A call with blocks of 512 threads,
    // and of this rule's: 16 instances, 32768 rows to 2048, 73 and 60 us; 4224 rows to 4096, 128 instances 138 and
    // 110 us, 384 instances 343 and 318, 1024 instances 762 and 701, 4608 instances 3216 and 3095 us (with a slower
    // selection; now 59, 108, 313, 684 and 2977 us).
    const int sms = device_sms();
    const auto move = [&](auto kernel, int threads) { return launch_after(kernel, s.n_inst, threads, 0, st, s, a); };
    return s.n_inst <= sms       ? move(evict_move_in_place_kernel<D, FOUR, 1024>, 1024)
           : s.n_inst <= 2 * sms ? move(evict_move_in_place_kernel<D, FOUR, 512>, 512)
           : s.n_inst <= 4 * sms ? move(evict_move_in_place_kernel<D, FOUR, 256>, 256)
                                 : move(evict_move_in_place_kernel<D, FOUR, 128>, 128);
  }
  const int kept = a.budget < s.cap ? a.budget : s.cap, chunks = (kept + kMoveRows - 1) / kMoveRows;
  return launch_after(evict_move_kernel<D, FOUR>, static_cast<unsigned>(s.n_inst) * chunks, kMoveThreads, 0, st, s, a, chunks);
}

}  // namespace

cudaError_t launch_evict(const Shape& s, const EvictArgs& a, cudaStream_t st) {
  if (a.four) return s.d == 128 ? launch_d<128, true>(s, a, st) : launch_d<64, true>(s, a, st);
  return s.d == 128 ? launch_d<128, false>(s, a, st) : launch_d<64, false>(s, a, st);
}

}  // namespace bkv
