// The attention kernel: softmax(Q K^T) V over key tiles on the tensor cores.
//
// Persistent, one CTA per SM.  For every key tile the keys are the 128 rows of
// the matrix product and the query rows its N columns, so a decode step's few
// queries fill the tensor cores' narrow dimension and every key costs one lane:
//   S^T [128 keys x N]  = K_tile Q^T          (K and Q from shared memory, K-major)
//   P^T [128 keys x N]  = 2^(scale S^T - ref)  (registers, rounded to bf16)
//   O^T [D x N]        += V_tile^T P           (V and P from shared memory, MN-major)
// S^T is double buffered in tensor memory, and O^T too, so that a segment's
// result is read out while the next one accumulates; up to 64 columns P and Q are
// double buffered in shared memory.  A softmax thread owns one key and half of the
// columns: the sum of p over the keys is a register per column, reduced over lanes
// once per segment.
//
// The reference of a column is the logit of the first key of the segment, not
// the maximum: p and its sum are fp32 and P is bf16, whose exponent range is as
// wide, so p may be large without losing precision.  Only when a logit exceeds
// the reference by more than 2^32 the reference moves to the tile's maximum, and
// the sums and O^T are scaled once.  That takes the reduction of the maximum over
// the lanes off the path: what is left of it is a vote of a group's four warps,
// under way on a barrier while they compute their exponentials.  With causal rows a
// column whose first key is masked is masked throughout the segment (rows see a
// prefix of the keys).
//
// Roundings: P to bf16 for the tensor cores, u = 2^-8 of each weight.  With 8 rows
// or fewer half of the columns are free and take the rest of each p, rounded to bf16
// again: the weights then carry 16 bits, the output is as exact as one of fp32
// weights (error 0.0017 of the output's size, its own rounding, against 0.0022), and
// the products cost the same (a step of 128 caches 53.4 us either way).
//
// Warp roles: warp 0 TMA producer, warp 1 MMA issue, warps 2 and 3 none, warps 4..11
// softmax (two groups of four warps, each with half of the columns).  K and V tiles share one
// ring of stages in the order in which they are used: S of the next tile is
// issued before O of this one, so the softmax of one tile overlaps both products.
//
// Rows of V past the last key of an item are zeroed in shared memory before they
// are used (0 * NaN would spread); rows of K need nothing, a key only reaches its
// own lane.
//
// Every wait, product and copy has one place in the code: a CTA runs through it 28 to
// 110 times, and before that the instructions come from memory (the same kernel with
// its loops peeled was twice as long and 5 us slower on one token).
//
// Bound by HBM, and in short calls by start and end.  head_dim 128, cold: 128 caches
// of 4097..4224 keys, 4 rows: 48 us, 277 MB, 5.8 TB/s (0.85 of the measured copy rate);
// 8 caches of 32768 keys: 27 us, 134 MB, 5.0 TB/s; 8 prefixes of 32768 keys, 64 rows:
// 28 us.  About 4.5 us pass until the first tile is there and 2 us after the last.
#pragma once

#include "k_attend.cuh"

namespace bkv {
namespace {

constexpr int kSmWarps = 8;
constexpr int kAtThreads = 32 * (4 + kSmWarps);
// Registers: 168 a thread at launch; the first four warps give back what the softmax warps take, 88 + 2 x 208
// of 3 x 168 per scheduler.
constexpr int kRegsFew = 88, kRegsMany = 208;
constexpr int kAtMaxStages = 12;
constexpr size_t kAtSmem = 218 * 1024;       // dynamic shared memory, next to up to 8 KB of static

// U: 8-column units per softmax group; N = 16 U columns.
template <int D, int U>
struct AtCfg {
  static constexpr int N = 16 * U;
  static constexpr int kBoxes = D / 64;
  static constexpr uint32_t kTileBytes = kBoxes * kAtBox;
  static constexpr uint32_t kQBox = N * 128;
  static constexpr int kQBufs = N <= 64 ? 2 : 1;
  static constexpr uint32_t kQBytes = kBoxes * kQBox;
  static constexpr int kPBoxes = N > 64 ? 2 : 1;
  static constexpr uint32_t kPBytes = kPBoxes * kAtBox;
  static constexpr int kPBufs = N <= 64 ? 2 : 1;
  static constexpr int kFit = static_cast<int>((kAtSmem - 1024 - kQBufs * kQBytes - kPBufs * kPBytes) / kTileBytes);
  static constexpr int kStages = kFit < kAtMaxStages ? kFit : kAtMaxStages;
  static constexpr size_t kSmem = 1024 + kQBufs * kQBytes + kPBufs * kPBytes + static_cast<size_t>(kStages) * kTileBytes;
  static constexpr int kNC = N / 2;  // columns of a softmax group
  static constexpr uint32_t kTmem = U <= 1 ? 64 : U <= 2 ? 128 : U <= 4 ? 256 : 512;  // S, S, O, O of N columns
  static_assert(kStages >= 3, "K of the next tile, V of this one, and one in flight");
};

// NC column sums of each lane, summed over the warp: the totals of columns first .. first + n - 1 end up
// in v[0 .. n - 1]; one lane per block of columns has `writer` set.  Halves the columns a lane holds
// while their number is even.
template <int NC>
__device__ __forceinline__ int warp_sum_columns(float (&v)[NC], int lane, bool& writer) {
  int first = 0, cols = NC;
  writer = true;
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) {
    if (cols % 2 == 0) {
      const int half = cols / 2;
      const bool upper = (lane & o) != 0;
#pragma unroll
      for (int i = 0; i < NC / 2; ++i) {
        if (i < half) {
          const float send = upper ? v[i] : v[i + half];
          const float keep = upper ? v[i + half] : v[i];
          v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
        }
      }
      if (upper) first += half;
      cols = half;
    } else {
#pragma unroll
      for (int i = 0; i < NC; ++i)
        if (i < cols) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
      if (lane & o) writer = false;
    }
  }
  return first;
}
// Columns that a lane holds after warp_sum_columns.
__host__ __device__ constexpr int held_columns(int cols) {
  for (int o = 16; o >= 1; o >>= 1)
    if (cols % 2 == 0) cols /= 2;
  return cols;
}

// The 8 U columns of this thread's lane, few loads.
template <int U>
__device__ __forceinline__ void tmem_ld_units(uint32_t taddr, float (&v)[8 * U]) {
  constexpr int n32 = U / 4 * 32;
#pragma unroll
  for (int c = 0; c < n32; c += 32) tmem_ld32(taddr + c, *reinterpret_cast<float(*)[32]>(v + c));
  if constexpr (U & 2) tmem_ld16(taddr + n32, v + n32);
  if constexpr (U & 1) tmem_ld8(taddr + 8 * U - 8, v + 8 * U - 8);
}

// What is left of (lo, hi) beside the bf16 pair `p` that they were rounded to.
__device__ __forceinline__ uint32_t pack_rest(uint32_t p, float lo, float hi) {
  return pack_bf16(lo - __uint_as_float(p << 16), hi - __uint_as_float(p & 0xFFFF0000u));
}

template <int D, int U>
__global__ void __launch_bounds__(kAtThreads, 1)
    attend_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                  const __grid_constant__ CUtensorMap vmap, AtKernelArgs a) {
  using C = AtCfg<D, U>;
  constexpr int N = C::N, NC = C::kNC;
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) uint64_t full_bar[kAtMaxStages], empty_bar[kAtMaxStages];
  __shared__ __align__(8) uint64_t qfull_bar[2], qempty_bar[2], sfull_bar[2], sfree_bar[2], pfull_bar[2], pfree_bar[2];
  __shared__ __align__(8) uint64_t ofull_bar[2], ofree_bar[2], vote_bar[2], drain_bar;
  __shared__ uint32_t tmem_base_sh;
  __shared__ int abort_sh;
  __shared__ int scan_sh[kAtThreads / 32];
  __shared__ AtShare share_sh;
  __shared__ __align__(16) float ref_sh[2][N];   // minus the reference of a column, by segment parity
  __shared__ __align__(16) int lim_sh[2][N];
  __shared__ int row_sh[2][N];  // row of q, o and lse (below 2^27), or -1
  __shared__ float red_sh[kSmWarps][NC];
  __shared__ float fac_sh[N];
  __shared__ float inv_sh[2][N];  // 1 / sum of p, by segment parity
  __shared__ int high_sh[2];  // tile (counted from 1) in which the group last found a logit far above its reference

  const AtGeo& g = a.geo;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  unsigned char* base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  unsigned char* q_smem = base;
  unsigned char* p_smem = q_smem + C::kQBufs * C::kQBytes;
  unsigned char* kv_smem = p_smem + C::kPBufs * C::kPBytes;
  volatile int* abort_flag = &abort_sh;

  if (tid == 32) {
    prefetch_tmap(&qmap);
    prefetch_tmap(&kmap);
    prefetch_tmap(&vmap);
  }
  if (tid == 0) {
    for (int i = 0; i < C::kStages; ++i) {
      mbar_init(&full_bar[i], 1);
      mbar_init(&empty_bar[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&qfull_bar[i], 1);
      mbar_init(&qempty_bar[i], 1);
      mbar_init(&sfull_bar[i], 1);
      mbar_init(&sfree_bar[i], kSmWarps);
      mbar_init(&pfull_bar[i], kSmWarps);
      mbar_init(&pfree_bar[i], 1);
      mbar_init(&ofull_bar[i], 1);
      mbar_init(&ofree_bar[i], kSmWarps);
      mbar_init(&vote_bar[i], 4);
      high_sh[i] = 0;
    }
    mbar_init(&drain_bar, 1);
    abort_sh = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&tmem_base_sh, C::kTmem);
    tmem_relinquish();
  }
  // rows of a Q buffer that no load fills are columns whose results are not used: zero, so that they
  // do not move references
  for (uint32_t i = tid * 16; i < C::kQBufs * C::kQBytes; i += kAtThreads * 16)
    *reinterpret_cast<uint4*>(q_smem + i) = make_uint4(0, 0, 0, 0);
  fence_async_smem();

  if (!a.after_prefix) grid_dependency_wait();  // whatever came before may have written the inputs
  grid_dependents_go();
  if (blockIdx.x == 0) at_check_lengths<kAtThreads>(g, a.err);
  tc_fence_before();
  at_split_tiles<kAtThreads>(g, scan_sh, &share_sh);
  tc_fence_after();
  if (tid == 0 && share_sh.left == 0) a.parts.cut[blockIdx.x] = make_int2(-1, -1);
  const uint32_t tmem = tmem_base_sh;
  AtWalk walk(g, share_sh);
  const int n_tiles = share_sh.left;  // tiles of this CTA (below 2^31)

  // Ring positions.  Tile i of the CTA: K(0); then for each i: K(i + 1), V(i), but V(i) first where
  // K(i + 1) needs a Q buffer that is still in use (one buffer, next segment) and at the end.
  if (warp < 4) {
    set_max_regs_dec<kRegsFew>();
    if (warp == 0) {
      // ---------------------------------------------------------------- producer
      if (lane == 0 && n_tiles > 0) {
        // Every key is read once (all rows of an instance are one block); kept in L2 the keys would push the
        // partial results out: a step of 128 caches 55.3 us, like this 53.4 us.
        const uint64_t pol = l2_policy_evict_first();
        const uint64_t pol_q = l2_policy_evict_last();
        int pos = 0, n_seg = 0;
        bool ok = true;
        auto load = [&](const CUtensorMap* map, int row) {
          const int st = pos % C::kStages;
          if (pos >= C::kStages &&
              !at_wait(&empty_bar[st], ((pos / C::kStages) - 1) & 1, abort_flag, a.err, kDevTimeoutProducer)) {
            ok = false;
            return;
          }
          mbar_arrive_expect_tx(&full_bar[st], C::kTileBytes);
          for (int b = 0; b < C::kBoxes; ++b)
            tma_load_2d(kv_smem + st * C::kTileBytes + b * kAtBox, map, &full_bar[st], b * 64, row, pol);
          ++pos;
        };
        auto load_q = [&](const AtSeg& s) {
          const int qb = n_seg % C::kQBufs;
          if (n_seg >= C::kQBufs &&
              !at_wait(&qempty_bar[qb], (n_seg / C::kQBufs - 1) & 1, abort_flag, a.err, kDevTimeoutProducer)) {
            ok = false;
            return;
          }
          mbar_arrive_expect_tx(&qfull_bar[qb], static_cast<uint32_t>(g.mb * g.rr) * D * 2);
          int group;
          const int kv = g.by_n_kv.mod(s.e, group);
          for (int b = 0; b < C::kBoxes; ++b)
            tma_load_4d(q_smem + qb * C::kQBytes + b * C::kQBox, &qmap, &qfull_bar[qb], b * 64, s.r0, kv,
                        group * g.m + s.b0, pol_q);
          ++n_seg;
        };
        AtSeg s;
        int t = 0, k_row = 0, v_row = 0;
        s.t1 = 0;
        for (int i = 0; ok && i <= n_tiles; ++i) {  // K(i) and V(i - 1)
          const bool turn = t == s.t1;              // tile i begins a segment
          const bool v_first = turn && C::kQBufs == 1;
          if (i < n_tiles) {
            if (turn) {
              walk.next(g, s);
              t = s.t0;
            }
            k_row = s.e * g.cap + t * kAtTile;
            ++t;
          }
#pragma unroll 1
          for (int h = 0; ok && h < 2; ++h) {
            const bool is_k = (h == 0) != v_first;
            if (is_k ? i == n_tiles : i == 0) continue;
            if (is_k && turn) load_q(s);
            if (ok) load(is_k ? &kmap : &vmap, is_k ? k_row : v_row);
          }
          v_row = k_row;
        }
        if (!ok || *abort_flag) {  // let every copy already issued land before the CTA exits
          for (int p = max(0, n_seg - C::kQBufs); p < n_seg; ++p)
            at_wait_always(&qfull_bar[p % C::kQBufs], (p / C::kQBufs) & 1, a.err, kDevTimeoutDrain, 1);
          for (int p = max(0, pos - C::kStages); p < pos; ++p)
            at_wait_always(&full_bar[p % C::kStages], (p / C::kStages) & 1, a.err, kDevTimeoutDrain, 1);
        }
      }
      __syncwarp();
    } else if (warp == 1) {
      // ---------------------------------------------------------------- MMA issuer
      // The whole warp walks along and one lane issues, so that descriptors stay in uniform registers.
      const uint32_t idesc_s = idesc_bf16_f32(128, N);
      const uint32_t idesc_o = idesc_s | kIdescMnMajorA | kIdescMnMajorB;
      const uint32_t v_box = C::kBoxes > 1 ? kAtBox : 0;  // head_dim 64: lanes 64 .. 127 repeat 0 .. 63
      const uint32_t kv_addr = smem_u32(kv_smem), q_addr = smem_u32(q_smem), p_addr = smem_u32(p_smem);
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
      int pos = 0;
      bool ok = true;
      auto await = [&](uint64_t* bar, uint32_t parity) {
        if (ok) ok = __all_sync(0xffffffffu, at_wait(bar, parity, abort_flag, a.err, kDevTimeoutMma));
      };
      auto issue_s = [&](int i, int seg, bool first, bool last_of_seg) {
        const int st = pos % C::kStages, buf = i & 1, qb = seg % C::kQBufs;
        if (first) await(&qfull_bar[qb], (seg / C::kQBufs) & 1);
        await(&full_bar[st], (pos / C::kStages) & 1);
        if (i >= 2) await(&sfree_bar[buf], ((i >> 1) - 1) & 1);
        if (!ok) return;
        tc_fence_after();
        const uint64_t k = sdesc_kmajor_sw128(kv_addr + st * C::kTileBytes);
        const uint64_t q = sdesc_kmajor_sw128(q_addr + qb * C::kQBytes);
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)
            mma_bf16_ss(tm + buf * N, k + (((kk >> 2) * kAtBox + (kk & 3) * 32) >> 4),
                        q + (((kk >> 2) * C::kQBox + (kk & 3) * 32) >> 4), idesc_s, kk > 0);
          mma_commit(&empty_bar[st]);
          mma_commit(&sfull_bar[buf]);
          if (last_of_seg) mma_commit(&qempty_bar[qb]);
        }
        __syncwarp();
        ++pos;
      };
      auto issue_o = [&](int i, int seg, bool first, bool last_of_seg) {
        const int st = pos % C::kStages, pb = i % C::kPBufs, ob = seg & 1;
        await(&full_bar[st], (pos / C::kStages) & 1);
        await(&pfull_bar[pb], (i / C::kPBufs) & 1);
        if (first && seg >= 2) await(&ofree_bar[ob], ((seg >> 1) - 1) & 1);
        if (!ok) return;
        tc_fence_after();
        const uint64_t v = sdesc_mnmajor_sw128(kv_addr + st * C::kTileBytes, v_box);
        const uint64_t p = sdesc_mnmajor_sw128(p_addr + pb * C::kPBytes, kAtBox);
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < kAtTile / 16; ++kk)
            mma_bf16_ss(tm + (2 + ob) * N, v + kk * (2048 >> 4), p + kk * (2048 >> 4), idesc_o, !first || kk > 0);
          mma_commit(&empty_bar[st]);
          mma_commit(&pfree_bar[pb]);
          if (last_of_seg) mma_commit(&ofull_bar[ob]);
        }
        __syncwarp();
        ++pos;
      };
      AtSeg s;
      int t = 0, seg = -1;
      bool o_first = false, o_last = false;  // tile i - 1 begins, ends its segment
      s.t1 = 0;
      for (int i = 0; ok && i <= n_tiles; ++i) {  // S(i) and O(i - 1)
        const bool turn = t == s.t1;
        const bool o_before = turn && C::kQBufs == 1;
        const int seg_o = seg;
        if (i < n_tiles) {
          if (turn) {
            walk.next(g, s);
            t = s.t0;
            ++seg;
          }
          ++t;
        }
        const bool first = o_first, last = o_last;
        o_first = turn;
        o_last = t == s.t1;
#pragma unroll 1
        for (int h = 0; ok && h < 2; ++h) {
          if ((h == 0) != o_before) {
            if (i < n_tiles) issue_s(i, seg, turn, t == s.t1);
          } else if (i > 0) {
            issue_o(i - 1, seg_o, first, last);
          }
        }
      }
      if (elect_one()) mma_commit(&drain_bar);  // every MMA issued above has finished once this arrives
      __syncwarp();
      at_wait_always(&drain_bar, 0, a.err, kDevTimeoutDrain, 1);
      __syncwarp();
    }
  } else {
    set_max_regs_inc<kRegsMany>();
    // ---------------------------------------------------------------- softmax
    const int grp = (warp - 4) >> 2, wt = tid & 127;  // column group; thread of the group
    const int quarter = warp & 3, key_lane = quarter * 32 + lane;
    const uint32_t lane_addr = static_cast<uint32_t>(quarter * 32) << 16;
    const uint32_t bar_id = 1 + grp;
    const int cols = g.mb * g.rr;
    const int c0 = grp * NC;
    const bool active = c0 < cols;  // the group has columns in use
    // The second group's columns of P and O carry what rounding the first group's P to bf16 leaves.
    const bool two_term = U == 1 && cols <= 8;
    const float sc = a.sc;
    auto wait = [&](uint64_t* bar, uint32_t parity) {  // after an abort every wait returns at once
      at_wait(bar, parity, abort_flag, a.err, kDevTimeoutEpilogue);
      __syncwarp();
    };
    // A finished segment's O^T is read out after the next segment's first tile: by then its last
    // product is complete.
    int out_seg = -1;
    size_t out_part = 0;
    bool out_final = false;
    auto read_out = [&] {
      wait(&ofull_bar[out_seg & 1], (out_seg >> 1) & 1);
      tc_fence_after();
      if (active) {
        const int* rows = row_sh[out_seg & 1] + c0;
        float o[NC];
        const uint32_t at = tmem + (2 + (out_seg & 1)) * N + c0 + lane_addr;
        tmem_ld_units<U>(at, o);
        if constexpr (U == 1) {
          if (two_term) {
            float low[8];
            tmem_ld8(at + 8, low);
            tmem_wait_ld();
#pragma unroll
            for (int c = 0; c < 8; ++c) o[c] += low[c];
          }
        }
        tmem_wait_ld();
        if (key_lane < D) {
          if (out_final) {
            const float* inv = inv_sh[out_seg & 1] + c0;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
              const int row = rows[c];
              if (row >= 0) a.o[static_cast<size_t>(row) * D + key_lane] = __float2bfloat16(o[c] * inv[c]);
            }
          } else {
            float* dst = a.parts.o + (out_part * a.parts.rows + c0) * D + key_lane;
#pragma unroll
            for (int c = 0; c < NC; ++c)
              if (rows[c] >= 0) dst[c * D] = o[c];
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ofree_bar[out_seg & 1]);
    };
    AtSeg s, next;
    int i = 0;  // tile of the CTA
    bool more = false;
    for (int seg = -1;; ++seg) {  // each segment is looked up one ahead
      const bool have = more;     // after the last one there is only its result to read out
      s = next;
      more = walk.next(g, next);
      if (seg < 0) continue;
      if (!have && out_seg < 0) break;
      float* ref = ref_sh[seg & 1] + c0;
      int* lim = lim_sh[seg & 1] + c0;
      int* rows = row_sh[seg & 1] + c0;
      int limit_min = 0, limit_max = 0, t = 0, t_end = 1;
      if (have) {
        limit_min = at_limit_min(g, s.len, s.r0);
        limit_max = at_limit_max(g, s.len, s.r0);
        t = s.t0;
        t_end = s.t1;
        if (tid == 128) at_note(a.parts, s, !more, share_sh.per);
      }
      if (have && wt < NC) {
        const int c = c0 + wt;
        rows[wt] = c < cols ? at_row(g, s.e, {s.b0, s.r0}, c) : -1;
        lim[wt] = at_limit(g, s.len, s.r0, c);
      }
      named_barrier(bar_id, 128);
      float l[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) l[c] = 0.f;
      for (bool first = true; t < t_end; ++t, first = false) {
        if (have) {
          const int buf = i & 1, k0 = t * kAtTile, j = k0 + key_lane;
          wait(&sfull_bar[buf], (i >> 1) & 1);
          tc_fence_after();
          const int pb = i % C::kPBufs;
          if (active) {
            float y[NC];
            // logits to base 2, less the references; masked ones to -inf
            auto load = [&] {
              tmem_ld_units<U>(tmem + buf * N + c0 + lane_addr, y);
              tmem_wait_ld();
            };
            auto shift = [&] {
#pragma unroll
              for (int c = 0; c < NC; c += 4) {
                const float4 r = *reinterpret_cast<const float4*>(ref + c);
                const float2 sc2 = make_float2(sc, sc);
                const float2 a0 = fma2(make_float2(y[c], y[c + 1]), sc2, make_float2(r.x, r.y));
                const float2 a1 = fma2(make_float2(y[c + 2], y[c + 3]), sc2, make_float2(r.z, r.w));
                y[c] = a0.x;
                y[c + 1] = a0.y;
                y[c + 2] = a1.x;
                y[c + 3] = a1.y;
              }
              if (k0 + kAtTile > limit_min) {  // some row does not see all keys of the tile
#pragma unroll
                for (int c = 0; c < NC; c += 4) {
                  const int4 m = *reinterpret_cast<const int4*>(lim + c);
                  y[c] = j < m.x ? y[c] : -INFINITY;
                  y[c + 1] = j < m.y ? y[c + 1] : -INFINITY;
                  y[c + 2] = j < m.z ? y[c + 2] : -INFINITY;
                  y[c + 3] = j < m.w ? y[c + 3] : -INFINITY;
                }
              }
            };
            load();
            if constexpr (16 * U <= kLogitRows) {
              // rows of an instance with so few of them are one block: consecutive
              if (a.logits && j < s.len) {
                float* dst = a.logits + (static_cast<size_t>(s.e) * g.R + c0) * g.cap + j;
#pragma unroll
                for (int c = 0; c < NC; ++c)
                  if (c0 + c < cols) dst[static_cast<size_t>(c) * g.cap] = y[c];
              }
            }
            if (t == s.t0) {
              if (key_lane == 0) {
#pragma unroll
                for (int c = 0; c < NC; ++c) ref[c] = k0 < lim[c] ? -fmaxf(y[c] * sc, kRefFloor) : 0.f;
              }
              named_barrier(bar_id, 128);
            }
            shift();
            float top0 = y[0], top1 = y[1], top2 = y[2], top3 = y[3];
#pragma unroll
            for (int c = 4; c < NC; c += 4) {
              top0 = fmaxf(top0, y[c]);
              top1 = fmaxf(top1, y[c + 1]);
              top2 = fmaxf(top2, y[c + 2]);
              top3 = fmaxf(top3, y[c + 3]);
            }
            // the group's vote is under way while the exponentials are computed
            const bool high = __any_sync(0xffffffffu, fmaxf(fmaxf(top0, top1), fmaxf(top2, top3)) > kMaxAbove);
            if (lane == 0) {
              if (high) *reinterpret_cast<volatile int*>(&high_sh[grp]) = i + 1;
              mbar_arrive(&vote_bar[grp]);
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) y[c] = ex2_approx(y[c]);
            // Not given up after an abort: the four warps must agree on the path below, which has barriers,
            // and each of them arrives after waits that are bounded.
            if (!mbar_try_wait(&vote_bar[grp], i & 1)) {
              at_wait_always(&vote_bar[grp], i & 1, a.err, kDevTimeoutEpilogue, 4);
            }
            __syncwarp();
            if (*reinterpret_cast<volatile int*>(&high_sh[grp]) == i + 1) {
              // move the references up to the tile's maxima; the logits are still in tensor memory
              load();
              shift();
#pragma unroll
              for (int c = 0; c < NC; ++c) {
                float v = y[c];
#pragma unroll
                for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
                if (lane == 0) red_sh[warp - 4][c] = v;
              }
              named_barrier(bar_id, 128);
              if (wt < NC) {
                float v = 0.f;
                for (int w = 0; w < 4; ++w) v = fmaxf(v, red_sh[grp * 4 + w][wt]);
                ref[wt] -= v;
                fac_sh[c0 + wt] = v;
              }
              named_barrier(bar_id, 128);
#pragma unroll
              for (int c = 0; c < NC; ++c) {
                const float v = fac_sh[c0 + c];
                y[c] = ex2_approx(y[c] - v);
                l[c] *= ex2_approx(-v);
              }
              if (t > s.t0) {  // O^T of the tiles before this one, complete once the last of them is
                wait(&pfree_bar[(i - 1) % C::kPBufs], ((i - 1) / C::kPBufs) & 1);
                tc_fence_after();
                const int units = two_term ? 2 : U;
#pragma unroll 1
                for (int u = 0; u < units; ++u) {
                  float o8[8];
                  const uint32_t at = tmem + (2 + (seg & 1)) * N + c0 + u * 8 + lane_addr;
                  tmem_ld8(at, o8);
                  tmem_wait_ld();
#pragma unroll
                  for (int c = 0; c < 8; ++c) o8[c] *= ex2_approx(-fac_sh[c0 + (two_term ? 0 : u * 8) + c]);
                  tmem_st8(at, o8);
                }
                tmem_wait_st();
              }
              named_barrier(bar_id, 128);  // fac_sh and red_sh may be written again
            }
            tc_fence_before();
            if (lane == 0) mbar_arrive(&sfree_bar[buf]);
            uint4 packed[U];
            uint4 low = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
              const float* p = y + u * 8;
#pragma unroll
              for (int c = 0; c < 8; c += 2) {
                const float2 v = add2(make_float2(l[u * 8 + c], l[u * 8 + c + 1]), make_float2(p[c], p[c + 1]));
                l[u * 8 + c] = v.x;
                l[u * 8 + c + 1] = v.y;
              }
              packed[u] = make_uint4(pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]),
                                     pack_bf16(p[6], p[7]));
            }
            if (two_term)
              low = make_uint4(pack_rest(packed[0].x, y[0], y[1]), pack_rest(packed[0].y, y[2], y[3]),
                               pack_rest(packed[0].z, y[4], y[5]), pack_rest(packed[0].w, y[6], y[7]));
            if (i >= C::kPBufs) wait(&pfree_bar[pb], (i / C::kPBufs - 1) & 1);
            unsigned char* p_row = p_smem + pb * C::kPBytes + key_lane * 128;
#pragma unroll
            for (int u = 0; u < U; ++u) {
              const int unit = grp * U + u;  // 16-byte unit of the key's row; 8 units to a box
              *reinterpret_cast<uint4*>(p_row + (unit >> 3) * kAtBox + (((unit ^ key_lane) & 7) * 16)) = packed[u];
            }
            if (two_term) *reinterpret_cast<uint4*>(p_row + ((1 ^ key_lane) & 7) * 16) = low;
          } else if (lane == 0) {
            mbar_arrive(&sfree_bar[buf]);
          }
          if (grp == 0 && k0 + kAtTile > limit_max && j >= limit_max) {
            // rows of V that no row of the item sees
            const bool last = i + 1 == n_tiles, turn = t + 1 == s.t1;
            const int vpos = 2 * i + (last || (turn && C::kQBufs == 1) ? 1 : 2);
            const int st = vpos % C::kStages;
            at_wait(&full_bar[st], (vpos / C::kStages) & 1, abort_flag, a.err, kDevTimeoutEpilogue);
#pragma unroll
            for (int b = 0; b < C::kBoxes; ++b)
#pragma unroll
              for (int x = 0; x < 8; ++x)
                *reinterpret_cast<uint4*>(kv_smem + st * C::kTileBytes + b * kAtBox + key_lane * 128 + x * 16) =
                    make_uint4(0, 0, 0, 0);
          }
          fence_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(&pfull_bar[pb]);
          ++i;
        }
        if (first && out_seg >= 0) read_out();
      }
      if (!have) break;
      // ---- the segment's sums
      out_seg = seg;
      out_final = a.whole_is_final && s.t0 == 0 && s.t1 == s.T;
      out_part = blockIdx.x + s.item;
      if (active) {
        bool writer;
        const int first = warp_sum_columns<NC>(l, lane, writer);
#pragma unroll
        for (int c = 0; c < held_columns(NC); ++c)
          if (writer) red_sh[warp - 4][first + c] = l[c];
        named_barrier(bar_id, 128);
        if (wt < NC && rows[wt] >= 0) {
          float sum = 0.f;
          for (int w = 0; w < 4; ++w) sum += red_sh[grp * 4 + w][wt];
          const bool some = sum != 0.f;  // a NaN stays one
          if (out_final) {
            inv_sh[seg & 1][c0 + wt] = some ? 1.f / sum : 0.f;
            const float y2 = some ? log2f(sum) - ref[wt] : -INFINITY;
            a.lse2[rows[wt]] = y2;
            if (a.lse) a.lse[rows[wt]] = y2 * 0.69314718055994531f;
          } else {
            a.parts.ml[out_part * a.parts.rows + c0 + wt] = make_float2(-ref[wt], sum);
          }
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, C::kTmem);
  if (a.after_prefix) grid_dependency_wait();  // what follows this kernel needs the prefix's results too
}

template <int D, int U>
cudaError_t launch(const AtPlan& p, const CUtensorMap& qmap, const CUtensorMap& kmap, const CUtensorMap& vmap,
                   const AtKernelArgs& a, cudaStream_t st) {
  using C = AtCfg<D, U>;
  const cudaError_t e = allow_smem<attend_kernel<D, U>>(C::kSmem);
  if (e != cudaSuccess) return e;
  return launch_after(attend_kernel<D, U>, p.grid, kAtThreads, C::kSmem, st, qmap, kmap, vmap, a);
}

}  // namespace

template <int D>
cudaError_t launch_attend_tiles_d(const AtPlan& p, const CUtensorMap& qmap, const CUtensorMap& kmap,
                                  const CUtensorMap& vmap, const AtKernelArgs& a, cudaStream_t st) {
  switch ((p.geo.mb * p.geo.rr + 15) / 16) {
    case 1: return launch<D, 1>(p, qmap, kmap, vmap, a, st);
    case 2: return launch<D, 2>(p, qmap, kmap, vmap, a, st);
    case 3: return launch<D, 3>(p, qmap, kmap, vmap, a, st);
    case 4: return launch<D, 4>(p, qmap, kmap, vmap, a, st);
    case 5: return launch<D, 5>(p, qmap, kmap, vmap, a, st);
    case 6: return launch<D, 6>(p, qmap, kmap, vmap, a, st);
    case 7: return launch<D, 7>(p, qmap, kmap, vmap, a, st);
    default: return launch<D, 8>(p, qmap, kmap, vmap, a, st);
  }
}

}  // namespace bkv
