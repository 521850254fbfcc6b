// The attention kernel for row blocks of more than 128 query rows (whole prompts,
// prefixes that many sequences share): compute bound, so the query rows are the
// lanes.
//
// Persistent, one CTA per SM, the work split into segments as in k_attend.cuh.  A
// row block is two row tiles of 128 that share every tile of keys and values:
//   S_w [128 rows x 128 keys] = Q_w K_tile^T     (both from shared memory, K-major)
//   P_w = 2^(scale S_w - ref)                    (registers; bf16, into tensor memory
//                                                 in place of S_w)
//   O_w [128 rows x D] += P_w V_tile             (P from tensor memory, V MN-major)
// Each softmax group (four warps, one thread per row) has one of the row tiles to
// itself: sum and reference are one register each, nothing is reduced across
// lanes, and P takes no shared-memory traffic.  While one group computes
// exponentials the tensor cores work for the other.
//
// The reference of a row is the logit of the segment's first key; only when a
// logit of a tile exceeds it by more than 2^32, or their sum does, the warp moves its references to
// the tile's maxima and scales its sums and its lanes of O (fp32 sums and bf16 P
// have the exponent range for that).  S_w stays in tensor memory until the tile's P is
// known to stand, so the exponentials need not wait for a maximum.  P is rounded to bf16 for
// the tensor cores, its sum is taken in fp32 before.
//
// Per 256 x 128 tile with head_dim 128 the products take 2048 clocks, as do the shared
// memory's reads for them and the copies into it (256 KB), and the exponentials, 32 per
// clock and SM, 1024; the two groups overlap them to some 3400.  A prompt of 4096
// tokens, 32 heads, cold: 128 us, 1.07 PFLOP/s of the causal pairs (0.57 of the measured
// rate of a large product); some 2 us at the end of each of a CTA's four segments are its
// results' way out, in which the tensor cores wait.  Steps of 64 keys, with S of both halves under way, were slower
// (a call of this prompt 196 us instead of 152): a product of half the columns takes more than
// half the time, and there are twice as many hand-overs.  So were two issuing warps.
#include "k_attend.cuh"

namespace bkv {
namespace {

constexpr int kThreads = 384;  // producer, MMA, two idle warps; two groups of four
constexpr int kRegsFew = 88, kRegsMany = 208;  // 88 + 2 x 208 of the 3 x 168 per scheduler at launch
constexpr int kRows = 128;     // rows of a row tile
constexpr float kSumAbove = 4294967296.f;  // 2^kMaxAbove

template <int D>
struct RowsCfg {
  static constexpr int kBoxes = D / 64;
  static constexpr uint32_t kTileBytes = kBoxes * kAtBox;
  static constexpr uint32_t kQBox = 2 * kAtBox;  // 256 rows of 64 columns
  static constexpr uint32_t kQBytes = kBoxes * kQBox;
  static constexpr int kStages = D == 128 ? 5 : 10;
  static constexpr size_t kSmem = 1024 + kQBytes + static_cast<size_t>(kStages) * kTileBytes;
  // tensor memory: S_0, S_1 (P in their first 64 columns), O_0, O_1
  static constexpr uint32_t kO = 2 * kAtTile;
  static constexpr uint32_t kTmem = 512;
};

// 32 bytes to an address aligned to them.  A thread writes a row, so a store of a warp touches 32 lines, and
// takes as long for 16 bytes of each as for 32: a prompt of 4096 tokens 136 us, its output by 16 bytes 141 us.
__device__ __forceinline__ void store_sector(void* dst, const uint32_t* v) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(dst), "r"(v[0]), "r"(v[1]), "r"(v[2]),
               "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    rows_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                const __grid_constant__ CUtensorMap vmap, AtKernelArgs a) {
  using C = RowsCfg<D>;
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) uint64_t full_bar[C::kStages], empty_bar[C::kStages];
  __shared__ __align__(8) uint64_t qfull_bar, qempty_bar, sfull_bar[2], pfull_bar[2];
  __shared__ __align__(8) uint64_t ofull_bar[2], ofree_bar[2], drain_bar;
  __shared__ uint32_t tmem_base_sh;
  __shared__ int abort_sh;
  __shared__ int scan_sh[kThreads / 32];
  __shared__ AtShare share_sh;

  const AtGeo& g = a.geo;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  unsigned char* base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  unsigned char* q_smem = base;
  unsigned char* kv_smem = base + C::kQBytes;
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
    mbar_init(&qfull_bar, 1);
    mbar_init(&qempty_bar, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sfull_bar[i], 1);
      mbar_init(&pfull_bar[i], 4);
      mbar_init(&ofull_bar[i], 1);
      mbar_init(&ofree_bar[i], 4);
    }
    mbar_init(&drain_bar, 1);
    abort_sh = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&tmem_base_sh, C::kTmem);
    tmem_relinquish();
  }
  // rows of the Q buffer that no load fills are rows whose results are not used
  for (uint32_t i = tid * 16; i < C::kQBytes; i += kThreads * 16)
    *reinterpret_cast<uint4*>(q_smem + i) = make_uint4(0, 0, 0, 0);
  fence_async_smem();

  if (!a.after_prefix) grid_dependency_wait();  // whatever came before may have written the inputs
  grid_dependents_go();
  if (blockIdx.x == 0) at_check_lengths<kThreads>(g, a.err);
  tc_fence_before();
  at_split_tiles<kThreads>(g, scan_sh, &share_sh);
  tc_fence_after();
  if (tid == 0 && share_sh.left == 0) a.parts.cut[blockIdx.x] = make_int2(-1, -1);
  const uint32_t tmem = tmem_base_sh;
  AtWalk walk(g, share_sh);
  const int n_tiles = share_sh.left;  // key tiles of this CTA

  // Ring of stages: K(0), then for each tile i: V(i), K(i + 1).
  if (warp < 4) {
    set_max_regs_dec<kRegsFew>();
    if (warp == 0) {
      // -------------------------------------------------------------- producer
      if (lane == 0 && n_tiles > 0) {
        const uint64_t pol = l2_policy_evict_last();
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
          if (n_seg >= 1 && !at_wait(&qempty_bar, (n_seg - 1) & 1, abort_flag, a.err, kDevTimeoutProducer)) {
            ok = false;
            return;
          }
          mbar_arrive_expect_tx(&qfull_bar, static_cast<uint32_t>(g.mb * g.rr) * D * 2);
          int group;
          const int kv = g.by_n_kv.mod(s.e, group);
          for (int b = 0; b < C::kBoxes; ++b)
            tma_load_4d(q_smem + b * C::kQBox, &qmap, &qfull_bar, b * 64, s.r0, kv, group * g.m + s.b0,
                        pol);
          ++n_seg;
        };
        AtSeg s;
        int t = 0, v_row = 0;
        s.t1 = 0;
        for (int i = 0; ok && i <= n_tiles; ++i) {  // V(i - 1), then K(i) and with a new segment its Q
          const bool turn = t == s.t1;
          int k_row = 0;
          if (i < n_tiles) {
            if (turn) {
              walk.next(g, s);
              t = s.t0;
            }
            k_row = s.e * g.cap + t * kAtTile;
            ++t;
          }
#pragma unroll 1
          for (int h = 0; ok && h < 2; ++h)
            if (h == 0 ? i > 0 : i < n_tiles) load(h == 0 ? &vmap : &kmap, h == 0 ? v_row : k_row);
          if (ok && turn && i < n_tiles) load_q(s);
          v_row = k_row;
        }
        if (!ok || *abort_flag) {  // let every copy already issued land before the CTA exits
          if (n_seg > 0) at_wait_always(&qfull_bar, (n_seg - 1) & 1, a.err, kDevTimeoutDrain, 1);
          for (int p = max(0, pos - C::kStages); p < pos; ++p)
            at_wait_always(&full_bar[p % C::kStages], (p / C::kStages) & 1, a.err, kDevTimeoutDrain, 1);
        }
      }
      __syncwarp();
    } else if (warp == 1) {
      // -------------------------------------------------------------- MMA issuer
      // Products run in the order in which they are issued, so S_w of the next tile may follow O_w of
      // this one at once although it overwrites its P.
      // The whole warp walks along and one lane issues, so that descriptors stay in uniform registers.
      const uint32_t idesc_s = idesc_bf16_f32(kRows, kAtTile), idesc_o = idesc_bf16_f32(kRows, D) | kIdescMnMajorB;
      const uint32_t kv_addr = smem_u32(kv_smem), q_addr = smem_u32(q_smem);
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
      bool ok = true;
      auto await = [&](uint64_t* bar, uint32_t parity) {
        if (ok) ok = __all_sync(0xffffffffu, at_wait(bar, parity, abort_flag, a.err, kDevTimeoutMma));
      };
      auto issue_s = [&](int w, int st, bool done, bool last_of_seg) {
        if (!ok) return;
        tc_fence_after();
        const uint64_t q = sdesc_kmajor_sw128(q_addr + w * kAtBox), k = sdesc_kmajor_sw128(kv_addr + st * C::kTileBytes);
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)
            mma_bf16_ss(tm + w * kAtTile, q + (((kk >> 2) * C::kQBox + (kk & 3) * 32) >> 4),
                        k + (((kk >> 2) * kAtBox + (kk & 3) * 32) >> 4), idesc_s, kk > 0);
          mma_commit(&sfull_bar[w]);
          if (done) mma_commit(&empty_bar[st]);
          if (done && last_of_seg) mma_commit(&qempty_bar);
        }
        __syncwarp();
      };
      auto issue_o = [&](int w, int i, int st, int seg, bool first, bool last_of_seg, bool done) {
        await(&pfull_bar[w], i & 1);
        if (first && seg >= 1) await(&ofree_bar[w], (seg - 1) & 1);
        if (!ok) return;
        tc_fence_after();
        const uint64_t v = sdesc_mnmajor_sw128(kv_addr + st * C::kTileBytes, kAtBox);
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < kAtTile / 16; ++kk)
            mma_bf16_ts(tm + C::kO + w * D, tm + w * kAtTile + kk * 8, v + kk * (2048 >> 4), idesc_o, !first || kk > 0);
          if (last_of_seg) mma_commit(&ofull_bar[w]);
          if (done) mma_commit(&empty_bar[st]);
        }
        __syncwarp();
      };
      AtSeg s;
      int t = 0, seg = -1;
      bool o_first = false, o_last = false;  // tile i - 1 begins, ends its segment
      s.t1 = 0;
      for (int i = 0; ok && i <= n_tiles; ++i) {  // for each row tile O(i - 1), then S(i)
        const bool turn = t == s.t1, more = i < n_tiles;
        const int seg_o = seg, v_pos = 2 * i - 1, k_pos = 2 * i;
        const int v_st = i > 0 ? v_pos % C::kStages : 0, k_st = k_pos % C::kStages;
        if (more) {
          if (turn) {
            walk.next(g, s);
            t = s.t0;
            ++seg;
          }
          ++t;
        }
        const bool first = o_first, last = o_last, last_s = t == s.t1;
        o_first = turn;
        o_last = last_s;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          if (i > 0) {
            if (w == 0) await(&full_bar[v_st], (v_pos / C::kStages) & 1);
            issue_o(w, i - 1, v_st, seg_o, first, last, w == 1);
          }
          if (more) {
            if (w == 0 && turn) await(&qfull_bar, seg & 1);
            if (w == 0) await(&full_bar[k_st], (k_pos / C::kStages) & 1);
            issue_s(w, k_st, w == 1, last_s);
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
    const int w = (warp - 4) >> 2;                       // row tile of the group
    const int lane_row = (warp & 3) * 32 + lane;         // row of it (tensor-memory lane)
    const uint32_t lane_addr = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_addr = tmem + w * kAtTile + lane_addr, o_addr = tmem + C::kO + w * D + lane_addr;
    const int c = w * kRows + lane_row, cols = g.mb * g.rr;  // row of the block
    const float sc = a.sc;
    const bool wide = (reinterpret_cast<uintptr_t>(a.o) & 31) == 0;  // the caller's o is aligned to 16 bytes at least
    auto wait = [&](uint64_t* bar, uint32_t parity) {  // after an abort every wait returns at once
      at_wait(bar, parity, abort_flag, a.err, kDevTimeoutEpilogue);
      __syncwarp();
    };
    AtSeg s, next;
    int i = 0;  // tile of the CTA
    bool more = false;
    for (int seg = -1;; ++seg) {  // each segment is looked up one ahead
      const bool have = more;
      s = next;
      more = walk.next(g, next);
      if (seg < 0) continue;
      if (!have) break;
      const int row = c < cols ? at_row(g, s.e, {s.b0, s.r0}, c) : -1;
      const int lim = row < 0 ? 0 : at_limit(g, s.len, s.r0, c);
      const int lim_min = __reduce_min_sync(0xffffffffu, row < 0 ? 0x7fffffff : lim);  // of the warp's rows
      const int limit_max = at_limit_max(g, s.len, s.r0);
      if (tid == 128) at_note(a.parts, s, !more, share_sh.per);
      float ref = 0.f, l = 0.f;  // ref: minus the reference
      for (int t = s.t0; t < s.t1; ++t, ++i) {
        const int k0 = t * kAtTile, seen = lim - k0;  // keys of the tile that the row sees
        const bool masked = k0 + kAtTile > lim_min;
        wait(&sfull_bar[w], i & 1);
        tc_fence_after();
        uint32_t p[kAtTile / 2];
        float sum = 0.f;
        // a quarter of the tile's logits, as exponents against the reference
        auto shift = [&](float(&v)[32], int q) {
          const float2 sc2 = make_float2(sc, sc), ref2 = make_float2(ref, ref);
#pragma unroll
          for (int x = 0; x < 32; x += 2) {
            const float2 y = fma2(make_float2(v[x], v[x + 1]), sc2, ref2);
            v[x] = y.x;
            v[x + 1] = y.y;
          }
          if (masked) {
#pragma unroll
            for (int x = 0; x < 32; ++x) v[x] = q * 32 + x < seen ? v[x] : -INFINITY;
          }
        };
        // the tile's weights against the present reference, and their sum
        auto weigh = [&](bool first) {
          float2 s0 = make_float2(0.f, 0.f), s1 = s0;
          float y[2][32];
          tmem_ld32(s_addr, y[0]);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float(&v)[32] = y[q & 1];
            tmem_wait_ld();
            if (q < 3) tmem_ld32(s_addr + (q + 1) * 32, y[(q + 1) & 1]);
            // A lane that sees nothing of the segment, or stands for no row but holds one of the next group, has
            // p = 0 whatever its logits are, so that they cannot ask for a move of the references.
            if (q == 0 && first) ref = seen > 0 ? -fmaxf(v[0] * sc, kRefFloor) : -INFINITY;
            shift(v, q);
#pragma unroll
            for (int x = 0; x < 32; x += 4) {
              const float2 e0 = make_float2(ex2_approx(v[x]), ex2_approx(v[x + 1]));
              const float2 e1 = make_float2(ex2_approx(v[x + 2]), ex2_approx(v[x + 3]));
              s0 = add2(s0, e0);
              s1 = add2(s1, e1);
              p[q * 16 + x / 2] = pack_bf16(e0.x, e0.y);
              p[q * 16 + x / 2 + 1] = pack_bf16(e1.x, e1.y);
            }
          }
          s0 = add2(s0, s1);
          sum = s0.x + s0.y;
        };
#pragma unroll 1
        for (int pass = 0;; ++pass) {
          weigh(pass == 0 && t == s.t0);
          // a weight above 2^32 shows in the sum, so no maximum is kept
          if (pass > 0 || !__any_sync(0xffffffffu, sum > kSumAbove)) break;
          // Move the references up to the tile's maxima.  The products of the tiles before are complete:
          // the barrier of this tile's S was waited for, and they were issued before it.
          float up = 0.f;
#pragma unroll 1
          for (int q = 0; q < 4; ++q) {
            float v[32];
            tmem_ld32(s_addr + q * 32, v);
            tmem_wait_ld();
            shift(v, 0);
#pragma unroll
            for (int x = 0; x < 32; ++x) up = fmaxf(up, q * 32 + x < seen ? v[x] : 0.f);
          }
          const float f = ex2_approx(-up);
          ref -= up;
          l *= f;
          if (t > s.t0) {
#pragma unroll 1
            for (int x = 0; x < D; x += 8) {
              float o8[8];
              tmem_ld8(o_addr + x, o8);
              tmem_wait_ld();
#pragma unroll
              for (int z = 0; z < 8; ++z) o8[z] *= f;
              tmem_st8(o_addr + x, o8);
            }
            tmem_wait_st();
          }
        }
        l += sum;
        tmem_st32(s_addr, p);
        tmem_st32(s_addr + 32, p + 32);
        tmem_wait_st();
        if (w == 0 && k0 + kAtTile > limit_max && k0 + lane_row >= limit_max) {
          // rows of V that no row of the item sees must not hold what 0 times it is not 0
          const int v_pos = 2 * i + 1, st = v_pos % C::kStages;
          at_wait(&full_bar[st], (v_pos / C::kStages) & 1, abort_flag, a.err, kDevTimeoutEpilogue);
#pragma unroll
          for (int b = 0; b < C::kBoxes; ++b)
#pragma unroll
            for (int x = 0; x < 8; ++x)
              *reinterpret_cast<uint4*>(kv_smem + st * C::kTileBytes + b * kAtBox + lane_row * 128 + x * 16) =
                  make_uint4(0, 0, 0, 0);
          fence_async_smem();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&pfull_bar[w]);
      }
      // ---- the segment's result
      const bool final_rows = a.whole_is_final && s.t0 == 0 && s.t1 == s.T;
      const size_t part = blockIdx.x + s.item;
      const bool some = l != 0.f;  // a NaN stays one
      if (row >= 0) {
        if (final_rows) {
          const float y2 = some ? log2f(l) - ref : -INFINITY;
          a.lse2[row] = y2;
          if (a.lse) a.lse[row] = y2 * 0.69314718055994531f;
        } else {
          a.parts.ml[part * a.parts.rows + c] = make_float2(-ref, l);
        }
      }
      const float inv = some ? 1.f / l : 0.f;
      wait(&ofull_bar[w], seg & 1);
      tc_fence_after();
      float* dst = a.parts.o + (part * a.parts.rows + c) * D;
#pragma unroll 1
      for (int x = 0; x < D; x += 32) {
        float o[32];
        tmem_ld32(o_addr + x, o);
        tmem_wait_ld();
        if (row >= 0) {
          if (final_rows) {
            __nv_bfloat16* out = a.o + static_cast<size_t>(row) * D + x;
#pragma unroll
            for (int z = 0; z < 32; z += 16) {
              uint32_t v[8];
#pragma unroll
              for (int y = 0; y < 8; ++y) v[y] = pack_bf16(o[z + 2 * y] * inv, o[z + 2 * y + 1] * inv);
              if (wide) {
                store_sector(out + z, v);
              } else {
                *reinterpret_cast<uint4*>(out + z) = make_uint4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<uint4*>(out + z + 8) = make_uint4(v[4], v[5], v[6], v[7]);
              }
            }
          } else {
#pragma unroll
            for (int z = 0; z < 32; z += 8) {
              uint32_t v[8];
#pragma unroll
              for (int y = 0; y < 8; ++y) v[y] = __float_as_uint(o[z + y]);
              store_sector(dst + x + z, v);
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ofree_bar[w]);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, C::kTmem);
  if (a.after_prefix) grid_dependency_wait();  // what follows this kernel needs the prefix's results too
}

template <int D>
cudaError_t launch(const AtPlan& p, const CUtensorMap& qmap, const CUtensorMap& kmap, const CUtensorMap& vmap,
                   const AtKernelArgs& a, cudaStream_t st) {
  using C = RowsCfg<D>;
  const cudaError_t e = allow_smem<rows_kernel<D>>(C::kSmem);
  if (e != cudaSuccess) return e;
  return launch_after(rows_kernel<D>, p.grid, kThreads, C::kSmem, st, qmap, kmap, vmap, a);
}

}  // namespace

cudaError_t launch_attend_rows(int d, const AtPlan& p, const CUtensorMap& qmap, const CUtensorMap& kmap,
                               const CUtensorMap& vmap, const AtKernelArgs& a, cudaStream_t st) {
  return d == 128 ? launch<128>(p, qmap, kmap, vmap, a, st) : launch<64>(p, qmap, kmap, vmap, a, st);
}

}  // namespace bkv
