// The attention kernel: softmax(Q K^T) V over key tiles on the tensor cores.
//
// Persistent, one CTA per SM.  For every key tile the keys are the 128 rows of
// the matrix product and the query rows its N columns, so a decode step's few
// queries fill the tensor cores' narrow dimension and every key costs one lane:
//   S^T [128 keys x N]  = K_tile Q^T          (K and Q from shared memory, K-major)
//   P^T [128 keys x N]  = 2^(scale S^T - ref)  (registers, rounded to bf16)
//   O^T [D x N]        += V_tile^T P           (V and P from shared memory, MN-major)
// S^T is double buffered in tensor memory, and O^T too, so that a segment's
// result is read out while the next one accumulates.  An softmax thread owns one
// key and half of the columns: the sum of p over the keys is a register per
// column, reduced over lanes once per segment.
//
// The reference of a column is the logit of the first key of the segment, not
// the maximum: p and its sum are fp32 and P is bf16, whose exponent range is as
// wide, so p may be large without losing precision.  Only when a logit exceeds
// the reference by more than 2^32 the reference moves to the tile's maximum, and
// the sums and O^T are scaled once.  That takes the reduction of the maximum over
// the lanes off the path.  With causal rows a column whose first key is masked is
// masked throughout the segment (rows see a prefix of the keys).
//
// Warp roles: warp 0 TMA producer, warp 1 MMA issue, warps 2..9 softmax (two
// groups of four warps, each with half of the columns).  K and V tiles share one
// ring of stages in the order in which they are used: S of the next tile is
// issued before O of this one, so the softmax of one tile overlaps both products.
//
// Rows of V past the last key of an item are zeroed in shared memory before they
// are used (0 * NaN would spread); rows of K need nothing, a key only reaches its
// own lane.
#include "k_attend.cuh"

namespace bkv {
namespace {

constexpr int kSmWarps = 8;
constexpr int kAtThreads = 32 * (2 + kSmWarps);
constexpr uint32_t kAtBox = 128 * 128;       // [128 rows][64 bf16]
constexpr int kAtMaxStages = 12;
constexpr size_t kAtSmem = 218 * 1024;       // dynamic shared memory, next to up to 8 KB of static
constexpr float kMaxAbove = 32.f;            // log2 of how far p may exceed 1
constexpr float kRefFloor = -1e30f;

template <int D, int N>
struct AtCfg {
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
  static constexpr uint32_t kTmem = 4 * N < 32 ? 32 : 4 * N;  // S, S, O, O
  static_assert(kStages >= 3, "K of the next tile, V of this one, and one in flight");
};

struct Seg {
  int e, rb, t0, t1, T, len, r0, b0;
  long long item, u;  // u: number of tile t0 in the run of all tiles
};

// Walks the CTA's segments; every role has its own.
struct Walk {
  int e, rb, t;
  long long left, u;
  __device__ __forceinline__ bool next(const AtGeo& g, Seg& s) {
    if (left <= 0 || e >= g.I) return false;
    const AtBlock blk = at_block(g, rb);
    s.e = e;
    s.rb = rb;
    s.b0 = blk.b0;
    s.r0 = blk.r0;
    s.len = at_len(g, e);
    s.T = at_tiles(at_limit_max(g, s.len, blk.r0));
    s.t0 = t;
    s.t1 = static_cast<int>(min(static_cast<long long>(s.T), t + left));
    s.item = static_cast<long long>(e) * g.nrb + rb;
    s.u = u;
    u += s.t1 - s.t0;
    left -= s.t1 - s.t0;
    t = s.t1;
    if (t == s.T) {
      t = 0;
      if (++rb == g.nrb) {
        rb = 0;
        ++e;
      }
    }
    return true;
  }
};

// NC column sums of each lane, summed over the warp: the totals of columns first .. first + n - 1 end
// up in v[0 .. n - 1] of a lane; n = max(1, NC / 32).  Halves the columns while there are several.
template <int NC>
__device__ __forceinline__ int warp_sum_columns(float (&v)[NC], int lane) {
  int first = 0;
#pragma unroll
  for (int o = 16, cols = NC; o >= 1; o >>= 1) {
    if (cols > 1) {
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
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    }
  }
  return first;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

template <int D, int N>
__global__ void __launch_bounds__(kAtThreads, 1)
    attend_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                  const __grid_constant__ CUtensorMap vmap, AtKernelArgs a) {
  using C = AtCfg<D, N>;
  constexpr int NC = C::kNC;
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) uint64_t full_bar[kAtMaxStages], empty_bar[kAtMaxStages];
  __shared__ __align__(8) uint64_t qfull_bar[2], qempty_bar[2], sfull_bar[2], sfree_bar[2], pfull_bar[2], pfree_bar[2];
  __shared__ __align__(8) uint64_t ofull_bar[2], ofree_bar[2], drain_bar;
  __shared__ uint32_t tmem_base_sh;
  __shared__ int abort_sh;
  __shared__ long long scan_sh[kAtThreads / 32];
  __shared__ AtShare share_sh;
  __shared__ __align__(16) float ref_sh[2][N];   // minus the reference of a column, by segment parity
  __shared__ __align__(16) int lim_sh[2][N];
  __shared__ int row_sh[2][N];  // row of q, o and lse (below 2^27), or -1
  __shared__ float red_sh[kSmWarps][NC];
  __shared__ float fac_sh[N];

  const AtGeo& g = a.geo;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  unsigned char* base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  unsigned char* q_smem = base;
  unsigned char* p_smem = q_smem + C::kQBufs * C::kQBytes;
  unsigned char* kv_smem = p_smem + C::kPBufs * C::kPBytes;
  volatile int* abort_flag = &abort_sh;

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

  if (blockIdx.x == 0) {
    for (int e = tid; e < g.I; e += kAtThreads) {
      const int n = __ldg(g.len + e / g.len_div);
      if (n < 0 || n > g.cap) record_error(a.err, kDevBadLength);
    }
  }
  tc_fence_before();
  at_split<kAtThreads>(
      g.I, [&](int e) { return at_inst_tiles(g, e); },
      [&](int e, int rb) { return at_tiles(at_limit_max(g, at_len(g, e), at_block(g, rb).r0)); }, scan_sh, &share_sh);
  tc_fence_after();
  if (blockIdx.x == 0 && tid == 0) *a.parts.per = share_sh.per;
  const uint32_t tmem = tmem_base_sh;
  Walk walk{share_sh.e, share_sh.k, share_sh.t, share_sh.left, share_sh.u};
  const int n_tiles = static_cast<int>(share_sh.left);  // tiles of this CTA (below 2^31)

  // Ring positions.  Tile i of the CTA: K(0); then for each i: K(i + 1), V(i), but V(i) first where
  // K(i + 1) needs a Q buffer that is still in use (one buffer, next segment) and at the end.
  if (warp == 0) {
    // ---------------------------------------------------------------- producer
    if (lane == 0 && n_tiles > 0) {
      const uint64_t pol = a.reuse ? l2_policy_evict_last() : l2_policy_evict_first();
      const uint64_t pol_q = l2_policy_evict_last();
      prefetch_tmap(&qmap);
      prefetch_tmap(&kmap);
      prefetch_tmap(&vmap);
      int pos = 0, n_seg = 0;
      bool ok = true;
      auto load = [&](const CUtensorMap* map, int row) {
        const int st = pos % C::kStages;
        if (pos >= C::kStages &&
            !mbar_wait(&empty_bar[st], ((pos / C::kStages) - 1) & 1, abort_flag, a.err, kDevTimeoutProducer)) {
          ok = false;
          return;
        }
        mbar_arrive_expect_tx(&full_bar[st], C::kTileBytes);
        for (int b = 0; b < C::kBoxes; ++b)
          tma_load_2d(kv_smem + st * C::kTileBytes + b * kAtBox, map, &full_bar[st], b * 64, row, pol);
        ++pos;
      };
      auto load_q = [&](const Seg& s) {
        const int qb = n_seg % C::kQBufs;
        if (n_seg >= C::kQBufs &&
            !mbar_wait(&qempty_bar[qb], (n_seg / C::kQBufs - 1) & 1, abort_flag, a.err, kDevTimeoutProducer)) {
          ok = false;
          return;
        }
        mbar_arrive_expect_tx(&qfull_bar[qb], static_cast<uint32_t>(g.mb * g.rr) * D * 2);
        for (int b = 0; b < C::kBoxes; ++b)
          tma_load_4d(q_smem + qb * C::kQBytes + b * C::kQBox, &qmap, &qfull_bar[qb], b * 64, s.r0, s.e % g.n_kv,
                      s.e / g.n_kv * g.m + s.b0, pol_q);
        ++n_seg;
      };
      Seg s;
      walk.next(g, s);
      load_q(s);
      if (ok) load(&kmap, s.e * g.cap + s.t0 * kAtTile);
      int t = s.t0;
      for (int i = 0; ok && i < n_tiles; ++i) {
        const int v_row = s.e * g.cap + t * kAtTile;
        const bool last = i + 1 == n_tiles, turn = t + 1 == s.t1;
        const bool v_first = last || (turn && C::kQBufs == 1);
        if (v_first) load(&vmap, v_row);
        if (!last && ok) {
          ++t;
          if (turn) {
            walk.next(g, s);
            t = s.t0;
            load_q(s);
          }
          if (ok) load(&kmap, s.e * g.cap + t * kAtTile);
        }
        if (!v_first && ok) load(&vmap, v_row);
      }
      if (!ok || *abort_flag) {  // let every copy already issued land before the CTA exits
        int never = 0;
        for (int p = max(0, n_seg - C::kQBufs); p < n_seg; ++p)
          mbar_wait(&qfull_bar[p % C::kQBufs], (p / C::kQBufs) & 1, &never, a.err, kDevTimeoutDrain);
        for (int p = max(0, pos - C::kStages); p < pos; ++p)
          mbar_wait(&full_bar[p % C::kStages], (p / C::kStages) & 1, &never, a.err, kDevTimeoutDrain);
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issuer
    if (lane == 0) {
      const int cols = (g.mb * g.rr + 15) / 16 * 16;
      const uint32_t idesc_s = idesc_bf16_f32(128, cols);
      const uint32_t idesc_o = idesc_s | kIdescMnMajorA | kIdescMnMajorB;
      const uint32_t v_box = C::kBoxes > 1 ? kAtBox : 0;  // head_dim 64: lanes 64 .. 127 repeat 0 .. 63
      int pos = 0;
      bool ok = true;
      auto issue_s = [&](int i, int seg, bool first, bool last_of_seg) {
        const int st = pos % C::kStages, buf = i & 1, qb = seg % C::kQBufs;
        if (first) ok = ok && mbar_wait(&qfull_bar[qb], (seg / C::kQBufs) & 1, abort_flag, a.err, kDevTimeoutMma);
        ok = ok && mbar_wait(&full_bar[st], (pos / C::kStages) & 1, abort_flag, a.err, kDevTimeoutMma);
        if (i >= 2) ok = ok && mbar_wait(&sfree_bar[buf], ((i >> 1) - 1) & 1, abort_flag, a.err, kDevTimeoutMma);
        if (!ok) return;
        tc_fence_after();
        const uint32_t k_addr = smem_u32(kv_smem + st * C::kTileBytes), q_addr = smem_u32(q_smem + qb * C::kQBytes);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          mma_bf16_ss(tmem + buf * N, sdesc_kmajor_sw128(k_addr + (kk >> 2) * kAtBox + (kk & 3) * 32),
                      sdesc_kmajor_sw128(q_addr + (kk >> 2) * C::kQBox + (kk & 3) * 32), idesc_s, kk > 0);
        mma_commit(&empty_bar[st]);
        mma_commit(&sfull_bar[buf]);
        if (last_of_seg) mma_commit(&qempty_bar[qb]);
        ++pos;
      };
      auto issue_o = [&](int i, int seg, bool first, bool last_of_seg) {
        const int st = pos % C::kStages, pb = i % C::kPBufs, ob = seg & 1;
        ok = ok && mbar_wait(&full_bar[st], (pos / C::kStages) & 1, abort_flag, a.err, kDevTimeoutMma);
        ok = ok && mbar_wait(&pfull_bar[pb], (i / C::kPBufs) & 1, abort_flag, a.err, kDevTimeoutMma);
        if (first && seg >= 2)
          ok = ok && mbar_wait(&ofree_bar[ob], ((seg >> 1) - 1) & 1, abort_flag, a.err, kDevTimeoutMma);
        if (!ok) return;
        tc_fence_after();
        const uint32_t v_addr = smem_u32(kv_smem + st * C::kTileBytes), p_addr = smem_u32(p_smem + pb * C::kPBytes);
#pragma unroll
        for (int kk = 0; kk < kAtTile / 16; ++kk)
          mma_bf16_ss(tmem + (2 + ob) * N, sdesc_mnmajor_sw128(v_addr + kk * 2048, v_box),
                      sdesc_mnmajor_sw128(p_addr + kk * 2048, kAtBox), idesc_o, !first || kk > 0);
        mma_commit(&empty_bar[st]);
        mma_commit(&pfree_bar[pb]);
        if (last_of_seg) mma_commit(&ofull_bar[ob]);
        ++pos;
      };
      if (n_tiles > 0) {
        Seg s;
        walk.next(g, s);
        int t = s.t0, seg = 0;
        issue_s(0, 0, true, s.t1 - s.t0 == 1);
        for (int i = 0; ok && i < n_tiles; ++i) {
          const bool last = i + 1 == n_tiles, first = t == s.t0, turn = t + 1 == s.t1;
          const int seg_o = seg;
          const bool v_first = last || (turn && C::kQBufs == 1);
          if (v_first) issue_o(i, seg_o, first, turn);
          if (!last && ok) {
            ++t;
            if (turn) {
              walk.next(g, s);
              t = s.t0;
              ++seg;
            }
            issue_s(i + 1, seg, t == s.t0, t + 1 == s.t1);
          }
          if (!v_first && ok) issue_o(i, seg_o, first, turn);
        }
      }
      mma_commit(&drain_bar);  // every MMA issued above has finished once this arrives
      int never = 0;
      mbar_wait(&drain_bar, 0, &never, a.err, kDevTimeoutDrain);
    }
    __syncwarp();
  } else {
    // ---------------------------------------------------------------- softmax
    const int grp = (warp - 2) >> 2, wt = (tid - 64) & 127;  // column group; thread of the group
    const int quarter = warp & 3, key_lane = quarter * 32 + lane;
    const uint32_t lane_addr = static_cast<uint32_t>(quarter * 32) << 16;
    const uint32_t bar_id = 1 + grp;
    const int cols = g.mb * g.rr;
    const int half = (cols + 15) / 16 * 8;          // columns of the first group, at most NC
    const int c0 = grp * half;
    const int ncw = max(0, min(half, cols - c0));   // columns in use in this group
    const float sc = a.sc;
    auto wait = [&](uint64_t* bar, uint32_t parity) {  // after an abort every wait returns at once
      if (!*abort_flag) mbar_wait(bar, parity, abort_flag, a.err, kDevTimeoutEpilogue);
      __syncwarp();
    };
    Seg s;
    int i = 0;  // tile of the CTA
    for (int seg = 0; walk.next(g, s); ++seg) {
      float* ref = ref_sh[seg & 1] + c0;
      int* lim = lim_sh[seg & 1] + c0;
      int* rows = row_sh[seg & 1] + c0;
      const int limit_min = at_limit_min(g, s.len, s.r0), limit_max = at_limit_max(g, s.len, s.r0);
      if (wt < half) {
        const int c = c0 + wt;
        rows[wt] = c < cols ? static_cast<int>(at_row(g, s.e, {s.b0, s.r0}, c)) : -1;
        lim[wt] = g.causal ? max(0, s.len - g.n_q + 1 + (s.r0 + c % g.rr) % g.n_q) : s.len;
      }
      if (wt == 0 && grp == 0 && s.t0 == 0) a.parts.u0[s.item] = s.u;
      named_barrier(bar_id, 128);
      float l[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) l[c] = 0.f;
      for (int t = s.t0; t < s.t1; ++t, ++i) {
        const int buf = i & 1, k0 = t * kAtTile, j = k0 + key_lane;
        wait(&sfull_bar[buf], (i >> 1) & 1);
        tc_fence_after();
        float y[NC];
#pragma unroll
        for (int u = 0; u < NC / 8; ++u)
          if (u * 8 < ncw) tmem_ld8(tmem + buf * N + c0 + u * 8 + lane_addr, y + u * 8);
        tmem_wait_ld();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sfree_bar[buf]);
        if (ncw > 0) {
          if (a.logits && j < s.len) {
#pragma unroll
            for (int c = 0; c < NC; ++c)
              if (c < ncw && rows[c] >= 0) a.logits[static_cast<size_t>(rows[c]) * g.cap + j] = y[c];
          }
          const bool masked = k0 + kAtTile > limit_min;
          if (t == s.t0) {
            if (key_lane == 0) {
#pragma unroll
              for (int c = 0; c < NC; ++c)
                if (c < ncw) ref[c] = k0 < lim[c] ? -fmaxf(y[c] * sc, kRefFloor) : 0.f;
            }
            named_barrier(bar_id, 128);
          }
          float top = -INFINITY;
#pragma unroll
          for (int c = 0; c < NC; c += 4) {
            if (c / 8 * 8 < ncw) {
              const float4 r = *reinterpret_cast<const float4*>(ref + c);
              y[c] = fmaf(y[c], sc, r.x);
              y[c + 1] = fmaf(y[c + 1], sc, r.y);
              y[c + 2] = fmaf(y[c + 2], sc, r.z);
              y[c + 3] = fmaf(y[c + 3], sc, r.w);
              if (masked) {
                const int4 m = *reinterpret_cast<const int4*>(lim + c);
                y[c] = j < m.x ? y[c] : -INFINITY;
                y[c + 1] = j < m.y ? y[c + 1] : -INFINITY;
                y[c + 2] = j < m.z ? y[c + 2] : -INFINITY;
                y[c + 3] = j < m.w ? y[c + 3] : -INFINITY;
              }
              top = fmaxf(fmaxf(top, fmaxf(y[c], y[c + 1])), fmaxf(y[c + 2], y[c + 3]));
            }
          }
          if (named_barrier_any(bar_id, 128, top > kMaxAbove)) {
            // move the references up to the tile's maxima
#pragma unroll
            for (int c = 0; c < NC; ++c) {
              if (c < ncw) {
                float v = y[c];
#pragma unroll
                for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
                if (lane == 0) red_sh[warp - 2][c] = v;
              }
            }
            named_barrier(bar_id, 128);
            if (wt < ncw) {
              float v = 0.f;
              for (int w = 0; w < 4; ++w) v = fmaxf(v, red_sh[grp * 4 + w][wt]);
              ref[wt] -= v;
              fac_sh[c0 + wt] = v;
            }
            named_barrier(bar_id, 128);
#pragma unroll
            for (int c = 0; c < NC; ++c) {
              if (c < ncw) {
                const float v = fac_sh[c0 + c];
                y[c] -= v;
                l[c] *= ex2_approx(-v);
              }
            }
            if (t > s.t0) {  // O^T of the tiles before this one, complete once the last of them is
              wait(&pfree_bar[(i - 1) % C::kPBufs], ((i - 1) / C::kPBufs) & 1);
              tc_fence_after();
#pragma unroll 1
              for (int u = 0; u * 8 < ncw; ++u) {
                float o8[8];
                const uint32_t at = tmem + (2 + (seg & 1)) * N + c0 + u * 8 + lane_addr;
                tmem_ld8(at, o8);
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < 8; ++c)
                  if (u * 8 + c < ncw) o8[c] *= ex2_approx(-fac_sh[c0 + u * 8 + c]);
                tmem_st8(at, o8);
              }
              tmem_wait_st();
              tc_fence_before();
            }
            named_barrier(bar_id, 128);  // fac_sh and red_sh may be written again
          }
        }
        uint4 packed[NC / 8];
#pragma unroll
        for (int u = 0; u < NC / 8; ++u) {
          if (u * 8 < ncw) {
            float* p = y + u * 8;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
              p[c] = ex2_approx(p[c]);
              l[u * 8 + c] += p[c];
            }
            packed[u] = make_uint4(pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]),
                                   pack_bf16(p[6], p[7]));
          }
        }
        const int pb = i % C::kPBufs;
        if (i >= C::kPBufs) wait(&pfree_bar[pb], (i / C::kPBufs - 1) & 1);
        unsigned char* p_row = p_smem + pb * C::kPBytes + key_lane * 128;
#pragma unroll
        for (int u = 0; u < NC / 8; ++u) {
          if (u * 8 < ncw) {
            const int unit = c0 / 8 + u;  // 16-byte unit of the key's row; 8 units to a box
            *reinterpret_cast<uint4*>(p_row + (unit >> 3) * kAtBox + (((unit ^ key_lane) & 7) * 16)) = packed[u];
          }
        }
        if (grp == 0 && k0 + kAtTile > limit_max && j >= limit_max) {
          // rows of V that no row of the item sees
          const bool last = i + 1 == n_tiles, turn = t + 1 == s.t1;
          const int vpos = 2 * i + (last || (turn && C::kQBufs == 1) ? 1 : 2);
          const int st = vpos % C::kStages;
          if (!*abort_flag) mbar_wait(&full_bar[st], (vpos / C::kStages) & 1, abort_flag, a.err, kDevTimeoutEpilogue);
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
      }
      // ---- the segment's result
      const int first = warp_sum_columns<NC>(l, lane);
      constexpr int kHeld = NC >= 32 ? NC / 32 : 1;
#pragma unroll
      for (int c = 0; c < kHeld; ++c)
        if (NC >= 32 || (lane & (32 / NC - 1)) == 0) red_sh[warp - 2][first + c] = l[c];
      named_barrier(bar_id, 128);
      const bool final_rows = a.whole_is_final && s.t0 == 0 && s.t1 == s.T;
      const long long part = blockIdx.x + s.item;
      if (wt < ncw && rows[wt] >= 0) {
        float sum = 0.f;
        for (int w = 0; w < 4; ++w) sum += red_sh[grp * 4 + w][wt];
        fac_sh[c0 + wt] = sum > 0.f || sum != sum ? 1.f / sum : 0.f;  // NaN stays NaN
        if (final_rows) {
          const float y2 = sum > 0.f || sum != sum ? log2f(sum) - ref[wt] : -INFINITY;
          a.lse2[rows[wt]] = y2;
          if (a.lse) a.lse[rows[wt]] = y2 * 0.69314718055994531f;
        } else {
          a.parts.ml[part * a.parts.rows + c0 + wt] = make_float2(-ref[wt], sum);
        }
      }
      named_barrier(bar_id, 128);
      wait(&ofull_bar[seg & 1], (seg >> 1) & 1);
      tc_fence_after();
      const bool d_lane = key_lane < D;
#pragma unroll
      for (int u = 0; u < NC / 8; ++u) {
        if (u * 8 < ncw) {
          float o8[8];
          tmem_ld8(tmem + (2 + (seg & 1)) * N + c0 + u * 8 + lane_addr, o8);
          tmem_wait_ld();
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            const int col = u * 8 + c;
            if (col < ncw && d_lane && rows[col] >= 0) {
              if (final_rows)
                a.o[static_cast<size_t>(rows[col]) * D + key_lane] = __float2bfloat16(o8[c] * fac_sh[c0 + col]);
              else
                a.parts.o[(part * a.parts.rows + c0 + col) * D + key_lane] = o8[c];
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ofree_bar[seg & 1]);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, C::kTmem);
}

template <int D, int N>
cudaError_t launch(const AtPlan& p, const CUtensorMap& qmap, const CUtensorMap& kmap, const CUtensorMap& vmap,
                   const AtKernelArgs& a, cudaStream_t st) {
  using C = AtCfg<D, N>;
  const cudaError_t e = cudaFuncSetAttribute(attend_kernel<D, N>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             static_cast<int>(C::kSmem));
  if (e != cudaSuccess) return e;
  attend_kernel<D, N><<<p.grid, kAtThreads, C::kSmem, st>>>(qmap, kmap, vmap, a);
  return cudaGetLastError();
}

template <int D>
cudaError_t launch_d(const AtPlan& p, const CUtensorMap& qmap, const CUtensorMap& kmap, const CUtensorMap& vmap,
                     const AtKernelArgs& a, cudaStream_t st) {
  switch (p.n_cols) {
    case 16: return launch<D, 16>(p, qmap, kmap, vmap, a, st);
    case 32: return launch<D, 32>(p, qmap, kmap, vmap, a, st);
    case 64: return launch<D, 64>(p, qmap, kmap, vmap, a, st);
    default: return launch<D, 128>(p, qmap, kmap, vmap, a, st);
  }
}

}  // namespace

cudaError_t launch_attend_tiles(int d, const AtPlan& p, const CUtensorMap& qmap, const CUtensorMap& kmap,
                                const CUtensorMap& vmap, const AtKernelArgs& a, cudaStream_t st) {
  return d == 128 ? launch_d<128>(p, qmap, kmap, vmap, a, st) : launch_d<64>(p, qmap, kmap, vmap, a, st);
}

}  // namespace bkv
