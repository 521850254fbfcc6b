// Accumulated attention weights (include/bkv.h, bkv_attend) of many query rows:
// the logits are computed again from the keys, and
//   weights[j] += sum over rows of 2^(scale2 q.k_j - lse2_row)
// is a sum along the rows of S^T = K_tile Q^T, whose lanes are the keys: every
// thread owns a key and adds its columns, no reduction over lanes is needed.
//
// Persistent, one CTA per SM.  An item is one tile of 128 keys of an instance, a
// unit is one block of up to 128 query rows that sees some of its keys; with
// more than 64 queries per head a block lies in one head and starts at the first
// query that sees the tile, so what the causal mask hides is not computed.  All
// units in item order are split evenly over the grid.  An item that one CTA
// finished is added to the weights there; the parts of a split one go to the
// workspace (a CTA has two at most: its first and its last) and a second launch
// adds them in order.
//
// Warp roles: warp 0 TMA producer, warp 1 MMA issue, warp 2 describes the units (the
// columns' normalisers and limits, what is masked, where an item ends) in a ring in
// shared memory, warps 4..11 exponentials: two groups take the units in turn, so that
// one computes while the other waits for its next unit (with both on every unit, half
// of the columns each, they waited and computed together).
//
// Per unit of 128 rows and head_dim 128 the matrix product takes 512 clocks and the exponentials,
// 32 per clock and SM, as long; the hand-overs between the warps bring it to some 1400.
// Cold: a prompt of 4096 tokens, 32 heads, 88 us, 780 TFLOP/s of the causal pairs
// (tensor pipe busy 0.32 of the time); 56 caches of at most 2171 keys, 44 rows, head_dim 64, 9 us.
// The merge of split items: 4.5 and 3.6 us.
//
// Sums and exponentials are fp32; the normalisers are those of the attention kernel.
#include "k_attend.cuh"

namespace bkv {
namespace {

constexpr int kSmWarps = 8, kGroups = kSmWarps / 4;  // two groups of four warps take the units in turn
constexpr int kThreads = 32 * (4 + kSmWarps);
constexpr int kDescs = 4;  // units described ahead
constexpr uint32_t kBox = 128 * 128;
constexpr int kCols = 128, kHalf = 64;
constexpr int kBufs = kDescs;  // of S in tensor memory: a unit described is a unit whose buffer is free
constexpr uint32_t kTmem = kBufs * kCols;

struct WArgs {
  int I, n_kv, G, R, n_q, cap;
  FastDiv by_n_kv, by_n_q, by_tiles;
  int hp, brow;     // heads per block (1: blocks within a head); rows of a Q box
  const int* len;
  float sc;
  const float* lse2;
  float* weights;
  float* parts;     // [2 grid][128]
  int* u0;          // [I * tiles]: number of an item's first unit; [I * tiles]: units per CTA
  int tiles;        // tiles of the capacity
  int ctas;         // of weights_kernel
  int* err;
};

__device__ __forceinline__ int w_len(const WArgs& a, int e) {
  const int n = __ldg(a.len + e);
  return n >= 0 && n <= a.cap ? n : 0;
}

// First query that sees a key of tile t, and units of the item.
__device__ __forceinline__ int w_first(const WArgs& a, int len, int t) { return max(0, t * kAtTile - len + a.n_q); }
__device__ __forceinline__ int w_units(const WArgs& a, int len, int t) {
  if (t * kAtTile >= len) return 0;
  if (a.hp > 1) return (a.G + a.hp - 1) / a.hp;
  return a.G * ((a.n_q - w_first(a, len, t) + kCols - 1) / kCols);
}

// Units of the tiles before tile t (at most the tiles in use): whole runs of query blocks for the tiles
// that every query sees, then one block less from tile to tile.
__device__ __forceinline__ int w_units_before(const WArgs& a, int len, int t) {
  if (a.hp > 1) return t * ((a.G + a.hp - 1) / a.hp);
  const int tiles = (len + kAtTile - 1) / kAtTile;
  const int t1 = len >= a.n_q ? (len - a.n_q) / kAtTile + 1 : 0;
  const int full = min(t, t1), m = max(0, t - t1), last = tiles - t1;  // m tiles of last, last - 1, ... blocks
  return a.G * (full * ((a.n_q + kCols - 1) / kCols) + m * last - m * (m - 1) / 2);
}

struct Unit {
  int e, t, k, n, len;  // unit k of the n of item (e, t)
  int head, blk, per_head, first;  // hp == 1: its head, block of the head's rows from query `first` on
  int r0, i0, cols;     // its rows r0 .. r0 + cols - 1; the query of the first
  __device__ __forceinline__ void place(const WArgs& a) {
    if (a.hp > 1) {
      r0 = k * a.hp * a.n_q;
      i0 = 0;
      cols = min(a.hp, a.G - k * a.hp) * a.n_q;
    } else {
      i0 = first + blk * kCols;
      r0 = head * a.n_q + i0;
      cols = min(kCols, a.n_q - i0);
    }
  }
  __device__ __forceinline__ void item(const WArgs& a) {
    n = w_units(a, len, t);
    first = w_first(a, len, t);
    per_head = (a.n_q - first + kCols - 1) / kCols;
    head = blk = 0;
  }
  __device__ __forceinline__ void start(const WArgs& a, const AtShare& s) {
    e = s.at.e;
    t = s.at.k;
    k = s.at.t;
    len = w_len(a, e);
    item(a);
    if (a.hp == 1) {
      head = k / per_head;
      blk = k % per_head;
    }
    place(a);
  }
  // The next unit; call it only while there is one.
  __device__ __forceinline__ void next(const WArgs& a) {
    if (++blk == per_head) {
      blk = 0;
      ++head;
    }
    if (++k == n) {
      k = 0;
      do {
        if (++t >= a.tiles || t * kAtTile >= len) {
          t = 0;
          ++e;
          len = w_len(a, e);
        }
        item(a);
      } while (n == 0);
    }
    place(a);
  }
};

// What the exponentials need to know of a unit.
struct Desc {
  int e, j0, len, cols;
  int plain;  // every column is a row that sees every key of the tile
  int ends;   // the item's last unit in this CTA: 1: all its units were here, 2: a part of them; + 4: it had this
              // one here only, and the other group has nothing to do with it
  int part;   // slot of the part
  int ends_cols;  // ends << 16 | cols
  int prev_e, prev_j0, prev_len, prev_ends, prev_part;  // the same of the unit before, which the other group had;
                                                        // prev_ends = 0 where that group needs no help
};

template <int D>
struct WCfg {
  static constexpr int kBoxes = D / 64;
  static constexpr uint32_t kTileBytes = kBoxes * kBox;
  static constexpr int kStages = D == 128 ? 4 : 8;
  static constexpr size_t kSmem = 1024 + (2 + kStages) * static_cast<size_t>(kTileBytes);
};

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    weights_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap, WArgs a) {
  using C = WCfg<D>;
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) uint64_t full_bar[C::kStages], empty_bar[C::kStages];
  __shared__ __align__(8) uint64_t kfull_bar[2], kempty_bar[2], sfull_bar[kBufs], meet_bar, drain_bar;
  __shared__ uint32_t tmem_base_sh;
  __shared__ int abort_sh;
  __shared__ int scan_sh[kThreads / 32];
  __shared__ AtShare share_sh;
  __shared__ __align__(16) float lse_sh[kDescs][kCols];
  __shared__ __align__(16) int lim_sh[kDescs][kCols];
  __shared__ Desc desc_sh[kDescs];
  __shared__ __align__(8) uint64_t dfull_bar[kDescs], dempty_bar[kDescs];
  __shared__ float sum_sh[kGroups][kAtTile];

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  unsigned char* base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  unsigned char* k_smem = base;
  unsigned char* q_smem = base + 2 * C::kTileBytes;
  volatile int* abort_flag = &abort_sh;

  if (tid == 0) {
    for (int i = 0; i < C::kStages; ++i) {
      mbar_init(&full_bar[i], 1);
      mbar_init(&empty_bar[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&kfull_bar[i], 1);
      mbar_init(&kempty_bar[i], 1);
    }
    for (int i = 0; i < kBufs; ++i) {
      mbar_init(&sfull_bar[i], 1);
    }
    for (int i = 0; i < kDescs; ++i) {
      mbar_init(&dfull_bar[i], 1);
      mbar_init(&dempty_bar[i], 4);
    }
    mbar_init(&drain_bar, 1);
    mbar_init(&meet_bar, kSmWarps);
    abort_sh = 0;
    fence_mbar_init();
  }
  grid_dependents_go();
  if (warp == 1) {
    tmem_alloc(&tmem_base_sh, kTmem);
    tmem_relinquish();
  }
  tc_fence_before();
  at_split<kThreads>(
      a.I,
      [&](int e) {
        const int len = w_len(a, e);
        return w_units_before(a, len, (len + kAtTile - 1) / kAtTile);
      },
      [&](int e, int u) {
        const int len = w_len(a, e);
        int lo = 0, hi = (len + kAtTile - 1) / kAtTile - 1;  // the last tile that begins at or before unit u
        while (lo < hi) {
          const int mid = (lo + hi + 1) / 2;
          if (w_units_before(a, len, mid) <= u) lo = mid;
          else hi = mid - 1;
        }
        return AtPlace{e, lo, static_cast<int>(u - w_units_before(a, len, lo))};
      },
      scan_sh, &share_sh);
  tc_fence_after();
  grid_dependency_wait();  // the normalisers; what came before reads len, q and K only
  const uint32_t tmem = tmem_base_sh;
  const AtShare share = share_sh;
  const int n_units = share.left;
  if (blockIdx.x == 0 && tid == 0) a.u0[static_cast<size_t>(a.I) * a.tiles] = share.per;

  if (warp == 0) {
    // ---------------------------------------------------------------- producer
    if (lane == 0 && n_units > 0) {
      const uint64_t pol = l2_policy_evict_last();
      prefetch_tmap(&qmap);
      prefetch_tmap(&kmap);
      Unit u;
      u.start(a, share);
      bool ok = true;
      int n_k = 0, i = 0;
      for (; ok && i < n_units; ++i) {
        if (i > 0) u.next(a);
        if (i == 0 || u.k == 0) {  // a new tile of keys
          const int kb = n_k & 1;
          if (n_k >= 2 && !at_wait(&kempty_bar[kb], ((n_k >> 1) - 1) & 1, abort_flag, a.err, kDevTimeoutProducer)) break;
          mbar_arrive_expect_tx(&kfull_bar[kb], C::kTileBytes);
          for (int b = 0; b < C::kBoxes; ++b)
            tma_load_2d(k_smem + kb * C::kTileBytes + b * kBox, &kmap, &kfull_bar[kb], b * 64,
                        u.e * a.cap + u.t * kAtTile, pol);
          ++n_k;
        }
        const int st = i % C::kStages;
        if (i >= C::kStages &&
            !at_wait(&empty_bar[st], ((i / C::kStages) - 1) & 1, abort_flag, a.err, kDevTimeoutProducer)) {
          ok = false;
          break;
        }
        mbar_arrive_expect_tx(&full_bar[st], static_cast<uint32_t>(a.brow) * D * 2);
        int b_kv;
        const int kv = a.by_n_kv.mod(u.e, b_kv);
        for (int b = 0; b < C::kBoxes; ++b)
          tma_load_4d(q_smem + st * C::kTileBytes + b * kBox, &qmap, &full_bar[st], b * 64, u.r0, kv, b_kv, pol);
      }
      if (i < n_units || *abort_flag) {  // let every copy already issued land before the CTA exits
        for (int p = max(0, n_k - 2); p < n_k; ++p)
          at_wait_always(&kfull_bar[p & 1], (p >> 1) & 1, a.err, kDevTimeoutDrain, 1);
        for (int p = max(0, i - C::kStages); p < i; ++p)
          at_wait_always(&full_bar[p % C::kStages], (p / C::kStages) & 1, a.err, kDevTimeoutDrain, 1);
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issuer
    // The whole warp walks along and one lane issues, so that descriptors stay in uniform registers.
    const uint32_t k_addr = smem_u32(k_smem), q_addr = smem_u32(q_smem);
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    bool ok = true;
    auto await = [&](uint64_t* bar, uint32_t parity) {
      if (ok) ok = __all_sync(0xffffffffu, at_wait(bar, parity, abort_flag, a.err, kDevTimeoutMma));
    };
    if (n_units > 0) {
      int n_k = 0;
      await(&kfull_bar[0], 0);
      for (int i = 0; ok && i < n_units; ++i) {
        const int st = i % C::kStages, buf = i % kBufs, x = i % kDescs;
        await(&dfull_bar[x], (i / kDescs) & 1);
        await(&full_bar[st], (i / C::kStages) & 1);
        if (!ok) break;
        // The description's slot was free, so the exponentials of the unit that had it, and with it this
        // buffer of S, are done.  It stays until those of this unit are.
        const int cols = __shfl_sync(0xffffffffu, desc_sh[x].ends_cols, 0), ends = cols >> 16;
        tc_fence_after();
        const uint32_t idesc = idesc_bf16_f32(128, ((cols & 0xFFFF) + 15) / 16 * 16);
        const uint64_t k = sdesc_kmajor_sw128(k_addr + (n_k & 1) * C::kTileBytes);
        const uint64_t q = sdesc_kmajor_sw128(q_addr + st * C::kTileBytes);
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)
            mma_bf16_ss(tm + buf * kCols, k + (((kk >> 2) * kBox + (kk & 3) * 32) >> 4),
                        q + (((kk >> 2) * kBox + (kk & 3) * 32) >> 4), idesc, kk > 0);
          mma_commit(&empty_bar[st]);
          mma_commit(&sfull_bar[buf]);
          if (ends) mma_commit(&kempty_bar[n_k & 1]);
        }
        __syncwarp();
        if (ends && i + 1 < n_units) {
          ++n_k;
          await(&kfull_bar[n_k & 1], (n_k >> 1) & 1);
        }
      }
    }
    if (elect_one()) mma_commit(&drain_bar);
    __syncwarp();
    at_wait_always(&drain_bar, 0, a.err, kDevTimeoutDrain, 1);
    __syncwarp();
  } else if (warp == 2) {
    // ---------------------------------------------------------------- descriptions
    if (n_units > 0) {
      Unit u;
      u.start(a, share);
      bool from_start = u.k == 0;  // this CTA has the item's units from its first one on
      int began = 0;               // unit of the CTA at which the item began
      Desc d;
      d.e = d.j0 = d.len = d.ends = d.part = 0;
      float lse[kCols / 32], lse_next[kCols / 32];
      auto fetch = [&](const Unit& v, float(&out)[kCols / 32]) {
#pragma unroll
        for (int y = 0; y < kCols / 32; ++y) {
          const int c = y * 32 + lane;
          out[y] = c < v.cols ? a.lse2[static_cast<size_t>(v.e) * a.R + v.r0 + c] : 0.f;
        }
      };
      fetch(u, lse);
      for (int i = 0; i < n_units; ++i) {
        const int x = i % kDescs;
        Unit v = u;
        if (i + 1 < n_units) {  // the next unit's normalisers are under way while this one is described
          v.next(a);
          fetch(v, lse_next);
        }
        if (from_start && u.k == 0 && lane == 0) a.u0[static_cast<size_t>(u.e) * a.tiles + u.t] = share.u + i;
        if (i >= kDescs &&
            !__all_sync(0xffffffffu,
                        at_wait(&dempty_bar[x], ((i / kDescs) - 1) & 1, abort_flag, a.err, kDevTimeoutProducer)))
          break;
#pragma unroll
        for (int y = 0; y < kCols / 32; ++y) {
          const int c = y * 32 + lane;
          // a row that sees nothing has -inf, and its columns are masked: any finite number will do
          lse_sh[x][c] = lse[y] == -INFINITY ? 0.f : -lse[y];
          // columns without a row see nothing
          lim_sh[x][c] = c < u.cols ? u.len - a.n_q + 1 + (a.hp > 1 ? a.by_n_q.mod(c) : u.i0 + c) : 0;
        }
        const bool ends = i + 1 == n_units || u.k + 1 == u.n, whole = from_start && u.k + 1 == u.n;
        const int how = ends ? (whole ? 1 : 2) + (i == began ? 4 : 0) : 0;
        d = {u.e, u.t * kAtTile, u.len, u.cols,
             u.cols == kCols && (u.t + 1) * kAtTile <= u.len - a.n_q + 1 + u.i0, how,
             // an item that began here after the CTA's first unit leaves part 1; else part 0
             static_cast<int>(blockIdx.x) * 2 + (from_start && began > 0), how << 16 | u.cols, d.e, d.j0, d.len,
             d.ends & 4 ? 0 : d.ends, d.part};
        if (lane == 0) desc_sh[x] = d;
        __syncwarp();
        if (lane == 0) mbar_arrive(&dfull_bar[x]);
        if (v.k == 0) {
          from_start = true;
          began = i + 1;
        }
        u = v;
#pragma unroll
        for (int y = 0; y < kCols / 32; ++y) lse[y] = lse_next[y];
      }
    }
  } else if (warp >= 4) {
    // ---------------------------------------------------------------- weights
    const int grp = (warp - 4) >> 2;
    const int quarter = warp & 3, key_lane = quarter * 32 + lane;
    const uint32_t lane_addr = static_cast<uint32_t>(quarter * 32) << 16;
    const float sc = a.sc;
    bool ok = true;  // after an expired wait the warp leaves: its descriptions cannot be trusted
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      if (ok) ok = __all_sync(0xffffffffu, at_wait(bar, parity, abort_flag, a.err, kDevTimeoutEpilogue));
    };
    uint32_t meetings = 0;
    auto meet = [&] {  // all eight warps; a barrier whose wait is bounded
      __syncwarp();
      if (lane == 0) mbar_arrive(&meet_bar);
      wait(&meet_bar, meetings++ & 1);
    };
    float acc = 0.f;
    // An item's sum.  A weight is added to once in a call, so the order of the additions cannot matter, and
    // nobody waits for the old value.
    auto write = [&](int e, int j0, int len, int ends, int part, float sum) {
      const int j = j0 + key_lane;
      if (ends & 2) a.parts[static_cast<size_t>(part) * kAtTile + key_lane] = sum;
      else if (j < len) atomicAdd(a.weights + static_cast<size_t>(e) * a.cap + j, sum);
    };
    // The sums of an item that both groups had units of, by both after their last unit of it: the one that
    // had its last unit then, the other before its next unit.
    auto finish = [&](int e, int j0, int len, int ends, int part) {
      sum_sh[grp][key_lane] = acc;
      acc = 0.f;
      meet();
      if (grp == 0 && ok) write(e, j0, len, ends, part, sum_sh[0][key_lane] + sum_sh[1][key_lane]);
      meet();
    };
#pragma unroll 1
    for (int i = grp; ok && i < n_units + 1; i += kGroups) {
      // past the last unit only its item is left to finish, by the group that did not have it
      const bool have = i < n_units;
      const int buf = i % kBufs, x = (have ? i : n_units - 1) % kDescs;
      if (!have && n_units == 0) break;
      wait(&dfull_bar[x], ((have ? i : n_units - 1) / kDescs) & 1);
      if (!ok) break;
      const Desc u = desc_sh[x];
      if (have ? u.prev_ends : u.ends) {
        if (have) finish(u.prev_e, u.prev_j0, u.prev_len, u.prev_ends, u.prev_part);
        else if (!(u.ends & 4)) finish(u.e, u.j0, u.len, u.ends, u.part);
      }
      if (!have) break;
      wait(&sfull_bar[buf], (i / kBufs) & 1);
      if (!ok) break;
      tc_fence_after();
      const int j = u.j0 + key_lane;
      float2 s0 = make_float2(0.f, 0.f), s1 = s0;
      auto add4 = [&](const float* y, int c) {
        const float4 l = *reinterpret_cast<const float4*>(&lse_sh[x][c]);  // minus the normalisers
        const float2 sc2 = make_float2(sc, sc);
        const float2 a0 = fma2(make_float2(y[0], y[1]), sc2, make_float2(l.x, l.y));
        const float2 a1 = fma2(make_float2(y[2], y[3]), sc2, make_float2(l.z, l.w));
        s0 = add2(s0, make_float2(ex2_approx(a0.x), ex2_approx(a0.y)));
        s1 = add2(s1, make_float2(ex2_approx(a1.x), ex2_approx(a1.y)));
      };
      const uint32_t at = tmem + buf * kCols + lane_addr;
      const int end = (u.cols + kHalf - 1) & ~(kHalf - 1);
#pragma unroll 1
      for (int h = 0; h < end; h += kHalf) {
        float y[kHalf];
#pragma unroll
        for (int c = 0; c < kHalf; c += 32) tmem_ld32(at + h + c, *reinterpret_cast<float(*)[32]>(y + c));
        tmem_wait_ld();
        if (!u.plain) {  // what a key's lane does not see, or no row, adds nothing
#pragma unroll
          for (int c = 0; c < kHalf; c += 4) {
            const int4 m = *reinterpret_cast<const int4*>(&lim_sh[x][h + c]);
            y[c] = j < m.x ? y[c] : -INFINITY;
            y[c + 1] = j < m.y ? y[c + 1] : -INFINITY;
            y[c + 2] = j < m.z ? y[c + 2] : -INFINITY;
            y[c + 3] = j < m.w ? y[c + 3] : -INFINITY;
          }
        }
#pragma unroll
        for (int c = 0; c < kHalf; c += 4) add4(y + c, h + c);
      }
      s0 = add2(s0, s1);
      acc += s0.x + s0.y;
      tc_fence_before();  // also gives back the buffer of S
      __syncwarp();
      if (lane == 0) mbar_arrive(&dempty_bar[x]);
      if (u.ends & 4) {
        write(u.e, u.j0, u.len, u.ends, u.part, acc);
        acc = 0.f;
      } else if (u.ends) {
        finish(u.e, u.j0, u.len, u.ends, u.part);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, kTmem);
}

// Parts of split items, in order: one thread per key.
__global__ void __launch_bounds__(kAtTile) weights_merge_kernel(WArgs a) {
  grid_dependency_wait();
  int e;
  const int t = a.by_tiles.mod(blockIdx.x, e);
  const int len = w_len(a, e), n = w_units(a, len, t);
  if (n == 0) return;
  const uint32_t per = a.u0[static_cast<size_t>(a.I) * a.tiles], u = a.u0[static_cast<size_t>(e) * a.tiles + t];
  const int j = t * kAtTile + threadIdx.x;
  if (!in_bounds(static_cast<long long>(u) + n - 1, static_cast<long long>(per) * a.ctas, a.err)) return;
  uint32_t first, last;
  if (!at_split_over(u, n, per, a.ctas, first, last) || j >= len) return;
  float sum = 0.f;
  for (uint32_t c = first; c <= last; ++c)
    sum += a.parts[(static_cast<size_t>(c) * 2 + (c == first && u != c * per)) * kAtTile + threadIdx.x];
  a.weights[static_cast<size_t>(e) * a.cap + j] += sum;
}

template <int D>
cudaError_t launch(const CUtensorMap& qmap, const CUtensorMap& kmap, const WArgs& a, cudaStream_t st) {
  const cudaError_t e = allow_smem<weights_kernel<D>>(WCfg<D>::kSmem);
  if (e != cudaSuccess) return e;
  const cudaError_t w = launch_after(weights_kernel<D>, a.ctas, kThreads, WCfg<D>::kSmem, st, qmap, kmap, a);
  if (w != cudaSuccess) return w;
  return launch_after(weights_merge_kernel, static_cast<unsigned>(a.I) * a.tiles, kAtTile, 0, st, a);
}

}  // namespace

cudaError_t launch_attend_weights(const Shape& s, const AttendArgs& a, const AtLayout& l, cudaStream_t st) {
  WArgs w{};
  w.I = s.batch * s.n_kv;
  w.n_kv = s.n_kv;
  w.G = s.G;
  w.R = s.G * a.n_q;
  w.n_q = a.n_q;
  w.cap = s.cap;
  // Several whole heads to a block while that halves the number of blocks at least: 128 caches of 4224 keys,
  // 4 heads of 11 queries 87 us (one to a block 128), of 32 queries 104 (144), of 64 queries 132 us (159).
  w.hp = a.n_q <= kCols / 2 ? kCols / a.n_q : 1;
  if (w.hp > s.G) w.hp = s.G;
  w.brow = w.hp > 1 ? w.hp * a.n_q : (a.n_q < kCols ? a.n_q : kCols);
  w.len = a.len;
  w.sc = a.sc;
  w.lse2 = reinterpret_cast<const float*>(a.ws + l.off_lse2);
  w.weights = a.weights;
  w.parts = reinterpret_cast<float*>(a.ws + l.off_wpart);
  w.u0 = reinterpret_cast<int*>(a.ws + l.off_wu0);
  w.tiles = (s.cap + kAtTile - 1) / kAtTile;
  w.ctas = l.sms;
  w.err = a.err;
  w.by_n_kv = FastDiv(w.n_kv);
  w.by_n_q = FastDiv(w.n_q);
  w.by_tiles = FastDiv(w.tiles);
  CUtensorMap qmap, kmap;
  if (encode_queries_bf16(&qmap, a.q, s.batch, s.n_kv, w.R, s.d, 1, w.brow) != CUDA_SUCCESS ||
      encode_rows_bf16(&kmap, a.K, static_cast<uint64_t>(w.I) * s.cap, s.d, kAtTile) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  return s.d == 128 ? launch<128>(qmap, kmap, w, st) : launch<64>(qmap, kmap, w, st);
}

}  // namespace bkv
