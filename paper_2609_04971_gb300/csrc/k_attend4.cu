// Attention of a few newest queries over caches held in 4 bits (include/bkv.h,
// bkv_attend4), for up to kRows4 query rows per KV head; more rows take the unpacked
// path of bkv_attend_api.cu.
//
// A key is low_g + step_g n in each group g of 32 elements, so with the codes n as the
// matrix product's left operand and the queries as its right one
//   q . k_j = sum_g step_jg (sum_{i in g} q_i n_ji) + low_jg (sum_{i in g} q_i),
// where each group's inner sum is exact up to fp32 addition, and for the values
//   o_i = sum_j (p_j step_jg(i)) n_ji + sum_j p_j low_jg(i).
// No element is ever scaled or rounded by itself.  A code in the lowest bits of an fp16 number is the
// number n 2^-24 (a subnormal, or in bits 4..7 16 n 2^-24: up to 2047 the bits of fp16 count linearly), so one
// AND makes two operands of a tensor-core product; a shift every second.  The queries, scaled to 2^11 by a
// power of two of each row, are exact in fp16 down to 2^-24 of the row's largest element; p and p step are rounded to
// fp16 (2^-11 of themselves each).
//
// Warps, not the tcgen05 unit, hold the operands: m16n8k16 products take the unpacked codes from the registers
// they are unpacked in, where tcgen05 would need 16-bit copies of every code in shared memory, four times the
// bytes that come from HBM, written and read again.
//
// Persistent, one CTA per SM, the work split into segments as in k_attend.cuh.  A warp takes slices
// of 16 keys: S [16 keys x 8 rows] per block of 8 query rows, P transposed in registers (movmatrix), and
// O^T [D x 8 rows] += V^T P.  The lows' share of a logit is a product too, of a key's lows and the queries' sums as
// three fp16 terms (33 bits), and so is their share of the output.  Each warp has its own reference m of a row's
// logits (base 2), which moves up when a logit exceeds it by more than 4.  p stands as 2^(y - m + 11), which fp16 holds
// down to 2^-36 of p = 1.  Where all steps of a slice's values lie in 2^-11 .. 1, as those of values of ordinary size
// do, or are 0, p step is a product of fp16 numbers, which loses what is below 2^-25 of p = 1 for the smallest of them.
// Other steps are multiplied in fp32, and the sums of a group of elements then have a power of two of their own that
// follows the slice's largest p step: neither large steps whose p is small nor small steps take digits from the rest.
//
// Warp roles: three load tiles of 128 keys into a ring, K, V and scales each (linear copies, 20 KB a tile at
// head_dim 128), one prepares the queries of the next segment as operands and joins the warps' sums of the last one,
// twelve (eight with two blocks of rows, whose accumulators need the registers) take steps of 32 keys in turn
// (k_ring4.cuh: what a step waits for).
//
// Bound by HBM on long caches and by start and end on short ones; 310 instructions a slice, half of them on the
// integer pipe, which unpacks, leave it there.  head_dim 128, cold: 128 caches of 4097..4224 keys, 4 rows 27.1 us,
// 88 MB; of 16896 keys 72 us, 346 MB, 4.8 TB/s; from 4224 to 16896 keys 6.0 TB/s (0.90 of the measured copy rate), so
// some 14 us do not depend on the bytes: 2.7 until the first load leaves (the lengths, the split), 2 until it is there,
// 2 to 3 after the last step; what makes up the rest was not measured.  8 rows cost 3 us more than 4; 16 rows 49 us,
// 32 rows 76 us: eight warps of long dependent chains.  When these took 45 and 70 us, blocks of 8 rows took 51 and
// 80, twelve warps for two blocks, their operands read from shared memory each time, 52 and 79 (head_dim 64, operands in
// registers: 32 rows 52 us instead of 55, but 28 rows of 7 sequences with weights 57 instead of 53).  A decode step over
// 128 caches spends 0.4 us on the waits for a slot's last tile and 0.4 on the look at the steps of V; where these are
// not the ordinary ones, a call over 128 caches of 4224 keys with weights takes 42 us instead of 36.
#include <cuda_fp16.h>

#include <type_traits>

#include "k_attend.cuh"
#include "k_ring4.cuh"

namespace bkv {
namespace {

constexpr int kSlice = 16, kStep = 2 * kSlice;  // keys of a product, of a warp's step
constexpr float kAbove4 = 4.f;                  // log2 of how far p may exceed 1
constexpr float kUp = 11.f;                     // p stands as p 2^kUp, at most 2^15
constexpr uint32_t kLeastStep = 0x1000, kMostStep = 0x3C00;  // 2^-11 and 1 as fp16: p step is an fp16 product
constexpr int kProductTop = 14, kProductLow = 8;  // exponents that the largest scaled p step of a slice may have
constexpr int kLeastScale = -26;                // p step below 2^-51 is nothing beside steps of at least 2^-24
constexpr float kCodeUnit = 16777216.f;         // a code n stands as n / 2^24
constexpr float kSumUnit = 64.f;                // sums of queries as fp16 terms are divided by it

// A B + C: A [16 x 16] and B [16 x 8] of fp16, fragments by lane as PTX defines them for m16n8k16.
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                              uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// The transpose of an 8 x 8 matrix of 16-bit numbers, a row to four lanes.
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ float half_lo(uint32_t v) { return __low2float(*reinterpret_cast<__half2*>(&v)); }
// Both numbers of `a` times the lower one of `b`.
__device__ __forceinline__ uint32_t mul_lo(uint32_t a, uint32_t b) {
  const __half2 m = __hmul2(*reinterpret_cast<__half2*>(&a), __low2half2(*reinterpret_cast<__half2*>(&b)));
  return *reinterpret_cast<const uint32_t*>(&m);
}
// The groups' exponents, a byte each.
__device__ __forceinline__ int scale_of(int exps, int i) { return static_cast<int8_t>(exps >> (8 * i)); }

// The exponent of a finite x >= 0 (of the smallest normal number below that).
__device__ __forceinline__ int exponent(float x) {
  return max(1, static_cast<int>(__float_as_uint(x) >> 23)) - 127;
}

struct Kernel4Args {
  AtGeo geo;
  AtParts parts;
  float sc;
  const __nv_bfloat16* q;
  const uint32_t *K4, *V4, *S4;
  __nv_bfloat16* o;
  float* lse;
  float* lse2;
  float* logits;  // [rows][cap] or nullptr
  int* err;
};

template <int D, int NB>
struct Cfg4 {
  // Warps at work on slices, behind three loading ones and one that joins.  Registers: 128 a thread at launch for
  // 16 warps (168 for 12), of which the first four give back what the others take.
  using Ring = Ring4<D, NB>;
  static constexpr int kWarps = Ring::kWarps, kFirst = 4;
  static constexpr int kThreads = 32 * (kFirst + kWarps);
  static constexpr int kRegsFew = NB == 1 ? 80 : 88, kRegsMany = NB == 1 ? 144 : 208;
  static constexpr int kRow = D + 4;  // floats of a joined row, so that a warp's stores meet no bank twice
  static constexpr size_t kJoin = sizeof(float) * kWarps * 8 * NB * kRow;
  // a slot of the ring: a tile's rows of K, V and scales, kPart steps
  static constexpr uint32_t kCodes = kAtTile * D / 2, kScales = kAtTile * D / 4, kSlot = 2 * kCodes + kScales;
  static constexpr int kPart = Ring::kPart, kSlots = Ring::kSlots;
  static_assert(kPart == kAtTile / kStep, "a tile's steps");
  static constexpr size_t kSmem = kJoin + static_cast<size_t>(kSlots) * kSlot;
};

// A row block's right operands, by lane: of every group the queries, then the terms of their sums; what a logit of
// columns 2 t and 2 t + 1 counts in, and how many keys they see.
template <int D, int NB>
struct Queries4 {
  uint4 qb[NB][D / 32][32];
  uint2 qs[NB][32];
  float2 unit[NB][32];
  int2 lim[NB][32];
};

template <int N>
__device__ __forceinline__ void load_words(uint32_t (&w)[N], const void* p) {
  if constexpr (N == 4) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    w[0] = x.x;
    w[1] = x.y;
    w[2] = x.z;
    w[3] = x.w;
  } else if constexpr (N == 2) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    w[0] = x.x;
    w[1] = x.y;
  } else {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}

// Linear copy of `bytes` (a multiple of 16, both ends 16-byte aligned) into shared memory.
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1], %2, [%3], %4;" ::"r"(smem_u32(dst)),
      "l"(src), "r"(bytes), "r"(smem_u32(bar)), "l"(policy)
      : "memory");
}

// The right operands of the block of rows [row0, row0 + cols), by one warp.
template <int D, int NB>
__device__ __forceinline__ void prepare_queries(Queries4<D, NB>& out, const Kernel4Args& a, size_t row0, int cols,
                                                const AtSeg& s, int lane) {
  constexpr int kG = D / 32;
  const int lg = lane >> 2, lt = lane & 3;
#pragma unroll 1
  for (int b = 0; b < NB; ++b) {
    const int c = b * 8 + lg;
    const uint4* src = reinterpret_cast<const uint4*>(a.q + (row0 + c) * D + 8 * lt);
    uint4 r[kG];
    uint32_t top2 = 0;  // the largest magnitude, as bf16
#pragma unroll
    for (int i = 0; i < kG; ++i) {
      r[i] = c < cols ? __ldg(src + 4 * i) : make_uint4(0, 0, 0, 0);
      const uint32_t w[4] = {r[i].x, r[i].y, r[i].z, r[i].w};
#pragma unroll
      for (int y = 0; y < 4; ++y) top2 = __vmaxu2(top2, w[y] & 0x7FFF7FFFu);
    }
    top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, 1));
    top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, 2));
    const float top = fmaxf(__uint_as_float(top2 << 16), __uint_as_float(top2 & 0x7FFF0000u));
    const int ex = top == 0.f ? 0 : max(exponent(top), -115);
    const float up = pow2i(11 - ex);
    float term[kG][3];
#pragma unroll
    for (int i = 0; i < kG; ++i) {
      const uint32_t w[4] = {r[i].x, r[i].y, r[i].z, r[i].w};
      float lo[4], hi[4], sum = 0.f;  // elements 2 y and 2 y + 1
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        lo[y] = __uint_as_float(w[y] << 16) * up;
        hi[y] = __uint_as_float(w[y] & 0xFFFF0000u) * up;
        sum += lo[y] + hi[y];
      }
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      sum *= 1.f / kSumUnit;
#pragma unroll
      for (int z = 0; z < 3; ++z) {
        term[i][z] = __half2float(__float2half_rn(sum));
        sum -= term[i][z];
      }
      // codes 2 y and 2 y + 1 of a byte: the second stands 16 times as high
      out.qb[b][i][lane] = make_uint4(pack_f16(lo[0], lo[2]), pack_f16(hi[0] * 0.0625f, hi[2] * 0.0625f),
                                      pack_f16(lo[1], lo[3]), pack_f16(hi[1] * 0.0625f, hi[3] * 0.0625f));
    }
    // Products with the keys' lows: k = 2 t, 2 t + 1 are a pair of groups and a term, k = 2 t + 8, 2 t + 9 too.
    uint2 qs;
    if constexpr (D == 128) {
      const bool odd = lt & 1;
      const float h0 = odd ? term[2][0] : term[0][0], h1 = odd ? term[3][0] : term[1][0];
      const float m0 = odd ? term[2][1] : term[0][1], m1 = odd ? term[3][1] : term[1][1];
      const float l0 = odd ? term[2][2] : term[0][2], l1 = odd ? term[3][2] : term[1][2];
      qs = make_uint2(lt < 2 ? pack_f16(h0, h1) : pack_f16(m0, m1), lt < 2 ? pack_f16(l0, l1) : 0u);
    } else {
      qs = make_uint2(lt == 0   ? pack_f16(term[0][0], term[1][0])
                      : lt == 1 ? pack_f16(term[0][1], term[1][1])
                      : lt == 2 ? pack_f16(term[0][2], term[1][2])
                                : 0u,
                      0u);
    }
    out.qs[b][lane] = qs;
    // columns 2 t and 2 t + 1 are the rows of lanes 8 t and 8 t + 4
    float unit[2];
    int lim[2];
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      unit[y] = pow2i(__shfl_sync(0xffffffffu, ex, 8 * lt + 4 * y) + 13);
      const int cc = b * 8 + 2 * lt + y;
      lim[y] = cc < cols ? at_limit(a.geo, s.len, s.r0, cc) : 0;
    }
    out.unit[b][lane] = make_float2(unit[0], unit[1]);
    out.lim[b][lane] = make_int2(lim[0], lim[1]);
  }
}

// Steps of a segment: of 32 keys each.
__device__ __forceinline__ int steps_of(const AtGeo& g, const AtSeg& s) {
  return max(0, (min(s.t1 * kAtTile, at_limit_max(g, s.len, s.r0)) - s.t0 * kAtTile + kStep - 1) / kStep);
}

template <int D, int NB>
__global__ void __launch_bounds__(Cfg4<D, NB>::kThreads, 1) attend4_kernel(Kernel4Args a) {
  using C = Cfg4<D, NB>;
  constexpr int kWarps = C::kWarps;
  constexpr int kG = D / 32;   // groups of a row
  constexpr int kMt = D / 16;             // tiles of 16 elements of o
  extern __shared__ __align__(128) unsigned char smem4[];
  float* join = reinterpret_cast<float*>(smem4);  // [warp][8 NB rows][kRow]
  unsigned char* ring = smem4 + C::kJoin;
  __shared__ __align__(16) Queries4<D, NB> queries_sh[2];
  __shared__ __align__(8) uint64_t full_bar[C::kSlots], empty_bar[C::kSlots];
  __shared__ __align__(8) uint64_t qfull_bar[2], qempty_bar[2], jfull_bar, jempty_bar;
  __shared__ float ref_sh[kWarps][8 * NB], sum_sh[kWarps][8 * NB];
  __shared__ int scan_sh[C::kThreads / 32];
  __shared__ AtShare share_sh;
  __shared__ int abort_sh;

  const AtGeo& g = a.geo;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, lg = lane >> 2, lt = lane & 3;
  volatile int* abort_flag = &abort_sh;
  if (tid < C::kSlots) {
    mbar_init(&full_bar[tid], 3);
    mbar_init(&empty_bar[tid], C::kPart);
  }
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&qfull_bar[i], 1);
      mbar_init(&qempty_bar[i], kWarps);
    }
    mbar_init(&jfull_bar, kWarps);
    mbar_init(&jempty_bar, 1);
    abort_sh = 0;
  }
  fence_mbar_init();
  grid_dependency_wait();
  grid_dependents_go();
  if (blockIdx.x == 0) at_check_lengths<C::kThreads>(g, a.err);
  at_split_tiles<C::kThreads>(g, scan_sh, &share_sh);
  if (tid == 0 && share_sh.left == 0) a.parts.cut[blockIdx.x] = make_int2(-1, -1);
  AtWalk walk(g, share_sh);
  AtSeg s;
  auto wait = [&](uint64_t* bar, uint32_t parity) {  // after an abort every wait returns at once
    at_wait(bar, parity, abort_flag, a.err, kDevTimeoutEpilogue);
    __syncwarp();
  };

  if (warp < C::kFirst) set_max_regs_dec<C::kRegsFew>();
  if (warp < C::kFirst && warp != 1) {
    // ---------------------------------------------------------------- loads: K, V and the scales by a warp each
    // (one warp for all three took 660 clocks for three copies, and a step of 128 caches 49.8 us)
    if (lane == 0) {
      // with one row block to an instance every key is read once
      const uint64_t pol = g.nrb == 1 ? l2_policy_evict_first() : l2_policy_evict_last();
      const unsigned char* src =
          reinterpret_cast<const unsigned char*>(warp == 0 ? a.K4 : warp == 2 ? a.V4 : a.S4);
      const uint32_t row_bytes = warp == 3 ? D / 4 : D / 2;
      unsigned char* dst = ring + (warp == 0 ? 0 : warp == 2 ? C::kCodes : 2 * C::kCodes);
      int slot = 0, turn = 0;  // slots are taken in order; turns of the ring so far
      bool ok = true;
      while (ok && walk.next(g, s)) {
        const int steps = steps_of(g, s);
        const int left = s.len - s.t0 * kAtTile;
        const unsigned char* at = src + (static_cast<size_t>(s.e) * g.cap + s.t0 * kAtTile) * row_bytes;
#pragma unroll 1
        for (int i = 0; i < steps; i += C::kPart) {
          if (turn > 0 && !at_wait(&empty_bar[slot], (turn - 1) & 1, abort_flag, a.err, kDevTimeoutProducer)) {
            ok = false;
            break;
          }
          const uint32_t bytes = min(kAtTile, left - i * kStep) * row_bytes;
          mbar_arrive_expect_tx(&full_bar[slot], bytes);
          bulk_load(dst + slot * C::kSlot, at, bytes, &full_bar[slot], pol);
          if (warp == 0)  // parts of the tile that no warp takes
            for (int x = steps - i; x < C::kPart; ++x) mbar_arrive(&empty_bar[slot]);
          at += kAtTile * row_bytes;
          if (++slot == C::kSlots) {
            slot = 0;
            ++turn;
          }
        }
      }
      if (!ok || *abort_flag) {
        // Let every copy already issued land before the CTA exits.  Where another loading warp gave up earlier a
        // barrier does not complete, and the wait ends by its limit.
        for (int i = 0; i < C::kSlots; ++i) {
          const int fills = turn + (i < slot);
          if (fills > 0) at_wait_always(&full_bar[i], (fills - 1) & 1, a.err, kDevTimeoutDrain, 1);
        }
      }
    }
    __syncwarp();
    return;
  }
  if (warp == 1) {
    // ---------------------------------------------------------------- queries, and the join of the warps' sums
    AtSeg done;
    bool have = false;
    for (int seg = 0;; ++seg) {  // the queries of segment seg, then the sums of the one before
      const bool more = walk.next(g, s);
      if (more) {
        if (seg >= 2) wait(&qempty_bar[seg & 1], ((seg >> 1) - 1) & 1);
        prepare_queries<D, NB>(queries_sh[seg & 1], a, static_cast<size_t>(s.e) * g.R + s.r0, min(g.rr, g.R - s.r0), s,
                               lane);
        __syncwarp();
        if (lane == 0) mbar_arrive(&qfull_bar[seg & 1]);
      }
      if (have) {
        if (lane == 0) at_note(a.parts, done, !more, share_sh.per);
        wait(&jfull_bar, (seg - 1) & 1);
        const int cols = min(g.rr, g.R - done.r0);
        const size_t row0 = static_cast<size_t>(done.e) * g.R + done.r0;
        int whole = done.t0 == 0 && done.t1 == done.T;
        const size_t part = (static_cast<size_t>(blockIdx.x) + done.item) * a.parts.rows;
#pragma unroll 1
        for (int c = 0; c < cols; ++c) {
          constexpr int kPer = D / 32;
          const float l = lane < kWarps ? sum_sh[lane][c] : 0.f;
          // a warp that took no step has no reference either
          const float ref = l != 0.f ? ref_sh[lane][c] : kRefFloor;
          float m = ref;
#pragma unroll
          for (int x = 16; x; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
          const float f = ex2_approx(ref - m);
          float sum = l * f;
#pragma unroll
          for (int x = 16; x; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
          float v[kPer] = {};
#pragma unroll
          for (int w = 0; w < kWarps; ++w) {
            const float fw = __shfl_sync(0xffffffffu, f, w);
            uint32_t r[kPer];
            load_words(r, join + (w * 8 * NB + c) * C::kRow + lane * kPer);
#pragma unroll
            for (int y = 0; y < kPer; ++y) v[y] = fmaf(__uint_as_float(r[y]), fw, v[y]);
          }
          const float inv = sum != 0.f ? 1.f / sum : 0.f;
          asm volatile("" : "+r"(whole));  // not two copies of the loop
          if (whole) {
            uint32_t* dst = reinterpret_cast<uint32_t*>(a.o + (row0 + c) * D) + lane * (kPer / 2);
#pragma unroll
            for (int y = 0; y < kPer; y += 2) dst[y / 2] = pack_bf16(v[y] * inv, v[y + 1] * inv);
          } else {
            float* dst = a.parts.o + (part + c) * D + lane * kPer;
#pragma unroll
            for (int y = 0; y < kPer; ++y) dst[y] = v[y];
          }
          if (lane == 0) {
            if (whole) {
              const float y2 = sum != 0.f ? m + log2f(sum) : -INFINITY;
              a.lse2[row0 + c] = y2;
              if (a.lse) a.lse[row0 + c] = y2 * 0.69314718055994531f;
            } else {
              a.parts.ml[part + c] = make_float2(m, sum);
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&jempty_bar);
      }
      if (!more) break;
      done = s;
      have = true;
    }
    return;
  }

  // ------------------------------------------------------------------ products
  set_max_regs_inc<C::kRegsMany>();
  const int mine = warp - C::kFirst;
  RingWalk<typename C::Ring> ring_at(mine);
  for (int seg = 0; walk.next(g, s); ++seg) {
    const int cols = min(g.rr, g.R - s.r0);       // rows of this block
    const int limit_min = at_limit_min(g, s.len, s.r0), n_steps = steps_of(g, s), len = s.len;
    float* logits = a.logits;
    if (logits) logits += (static_cast<size_t>(s.e) * g.R + s.r0) * g.cap;
    uint32_t qb[NB][kG][4], qs[NB][2];
    float unit[NB][2];
    int lim[NB][2];
    wait(&qfull_bar[seg & 1], (seg >> 1) & 1);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const Queries4<D, NB>& in = queries_sh[seg & 1];
#pragma unroll
      for (int i = 0; i < kG; ++i) load_words(qb[b][i], &in.qb[b][i][lane]);
      load_words(qs[b], &in.qs[b][lane]);
      const float2 u = in.unit[b][lane];
      const int2 m = in.lim[b][lane];
      unit[b][0] = u.x;
      unit[b][1] = u.y;
      lim[b][0] = m.x;
      lim[b][1] = m.y;
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&qempty_bar[seg & 1]);

    // p = 2^(y - ref): ref is the reference of the column less kUp
    float o[NB][kMt][4] = {}, low[NB][4] = {}, l[NB][2] = {}, ref[NB][2];
    int exps = 0;              // o of group i is times 2^-scale_of(i)
    float most_y = -INFINITY;  // what y - ref may be; no reference yet
    auto rescale = [&](int now) {
#pragma unroll
      for (int i = 0; i < kG; ++i) {
        const float f = pow2i(scale_of(exps, i) - scale_of(now, i));
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int m = i * (kMt / kG); m < (i + 1) * (kMt / kG); ++m)
#pragma unroll
            for (int z = 0; z < 4; ++z) o[b][m][z] *= f;
      }
      exps = now;
    };
#pragma unroll
    for (int b = 0; b < NB; ++b) ref[b][0] = ref[b][1] = 0.f;

    ring_at.begin();
#pragma unroll 1
    for (; ring_at.step < n_steps; ring_at.next()) {
      const int j0 = s.t0 * kAtTile + ring_at.step * kStep, slot = ring_at.slot;
      if (!ring_at.there([&](int i, int parity) { return mbar_try_wait(&empty_bar[i], parity); },
                         [&](int i, int parity) { return mbar_try_wait(&full_bar[i], parity); }))
        ring_at.await(
            [&](int i, int parity) { at_wait(&empty_bar[i], parity, abort_flag, a.err, kDevTimeoutEpilogue); },
            [&](int i, int parity) { at_wait(&full_bar[i], parity, abort_flag, a.err, kDevTimeoutEpilogue); });
      __syncwarp();
      const int row = ring_at.step % C::kPart * kStep;  // of the tile
      const unsigned char* at = ring + slot * C::kSlot + row * (D / 2);
      unsigned char* scales = ring + slot * C::kSlot + 2 * C::kCodes + row * (D / 4);
      const int left = len - j0;
      if (left < kStep) {  // rows past the length hold anything: their steps and lows become 0
        if (lane >= left) {
#pragma unroll
          for (int i = 0; i < D / 4; i += 16) *reinterpret_cast<uint4*>(scales + lane * (D / 4) + i) = uint4{};
        }
        fence_async_smem();  // the slot is loaded again
        __syncwarp();
      }
      bool any_wide;  // a step of the values, lane's row by lane, that is none of the ordinary ones
      {
        uint32_t w[kG], most = 0, least = 0xFFFFFFFFu;
        load_words(w, scales + lane * (D / 4) + kG * 4);
#pragma unroll
        for (int i = 0; i < kG; ++i) {
          most = max(most, w[i] << 16);
          least = min(least, (w[i] << 16) - 0x10000u);  // 0 is the largest
        }
        any_wide = __any_sync(0xffffffffu, most > kMostStep << 16 || least < (kLeastStep - 1) << 16);
      }
#pragma unroll 1
      for (int r0 = 0; r0 < kStep; r0 += kSlice) {  // rolled: what a short call waits for is instructions
        // ---- logits, in the columns' units
        float y[NB][4];
        {
          uint32_t k[2][kG], ks[2][kG], lows[2];  // lows of a pair of groups of keys g and g + 8
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int r = r0 + lg + 8 * h;
            load_words(k[h], at + r * (D / 2) + lt * (kG * 4));
            load_words(ks[h], scales + r * (D / 4));
            uint32_t pair[2];
            load_words(pair, scales + r * (D / 4) + (D == 128 ? (lt & 1) * 8 : 0));
            lows[h] = __byte_perm(pair[0], pair[1], 0x7632);
          }
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            float c[4];
            mma_f16_first(c, lows[0], lows[1], lows[0], lows[1], qs[b][0], qs[b][1]);
#pragma unroll
            for (int z = 0; z < 4; ++z) y[b][z] = c[z] * (kSumUnit / kCodeUnit);
          }
#pragma unroll
          for (int i = 0; i < kG; ++i) {
            uint32_t f[2][4];  // codes (0, 4), (1, 5), (2, 6), (3, 7) of the word
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t w = k[h][i], w8 = w >> 8;
              f[h][0] = w & 0x000F000Fu;
              f[h][1] = w & 0x00F000F0u;
              f[h][2] = w8 & 0x000F000Fu;
              f[h][3] = w8 & 0x00F000F0u;
            }
            const float s0 = half_lo(ks[0][i]), s1 = half_lo(ks[1][i]);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
              float c[4];
              mma_f16_first(c, f[0][0], f[1][0], f[0][1], f[1][1], qb[b][i][0], qb[b][i][1]);
              mma_f16(c, f[0][2], f[1][2], f[0][3], f[1][3], qb[b][i][2], qb[b][i][3]);
              y[b][0] = fmaf(s0, c[0], y[b][0]);
              y[b][1] = fmaf(s0, c[1], y[b][1]);
              y[b][2] = fmaf(s1, c[2], y[b][2]);
              y[b][3] = fmaf(s1, c[3], y[b][3]);
            }
          }
        }
        asm volatile("" : "+l"(logits));  // not two copies of the loop
        if (logits) {
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int z = 0; z < 4; ++z) {
              const int c = b * 8 + 2 * lt + (z & 1), r = r0 + lg + 8 * (z >> 1);
              if (c < cols && r < left) logits[static_cast<size_t>(c) * g.cap + j0 + r] = y[b][z] * unit[b][z & 1];
            }
        }
        uint32_t vs[2][kG];  // (step, low) of V of keys g and g + 8
#pragma unroll
        for (int h = 0; h < 2; ++h) load_words(vs[h], scales + (r0 + lg + 8 * h) * (D / 4) + kG * 4);
        uint32_t lv[2];  // lows of group g of keys 2 t, 2 t + 1 and 2 t + 8, 2 t + 9
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t w[2];
#pragma unroll
          for (int z = 0; z < 2; ++z)
            w[z] = *reinterpret_cast<const uint32_t*>(scales + (r0 + 8 * h + 2 * lt + z) * (D / 4) + kG * 4 +
                                                      (lg & (kG - 1)) * 4);
          lv[h] = __byte_perm(w[0], w[1], 0x7632);
        }
        // ---- to base 2, against the references
        float above = -INFINITY;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int z = 0; z < 4; ++z) y[b][z] = fmaf(y[b][z], unit[b][z & 1] * a.sc, -ref[b][z & 1]);
        if (j0 + r0 + kSlice > limit_min) {
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int z = 0; z < 4; ++z)
              if (j0 + r0 + lg + 8 * (z >> 1) >= lim[b][z & 1]) y[b][z] = -INFINITY;
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int z = 0; z < 4; ++z) above = fmaxf(above, y[b][z]);
        if (__any_sync(0xffffffffu, above > most_y)) {
          // Move the references to the slice's maxima.  A column that sees nothing of the slice of a warp's first
          // reference sees nothing after it either: it stays at the floor.
          const bool begins = most_y == -INFINITY;
          const float back = begins ? kRefFloor : kUp;
          most_y = kAbove4 + kUp;
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              float v = fmaxf(y[b][z], y[b][z + 2]);
#pragma unroll
              for (int m = 4; m < 32; m <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, m));
              // relative to ref: the reference was at `back`; it moves up to v
              const float by = fmaxf(v, back) - kUp;
              const float fac = begins ? 0.f : ex2_approx(-by);
              ref[b][z] += by;
              l[b][z] *= fac;
              low[b][z] *= fac;
              y[b][z] -= by;
              y[b][z + 2] -= by;
#pragma unroll
              for (int m = 0; m < kMt; ++m) {
                o[b][m][z] *= fac;
                o[b][m][z + 2] *= fac;
              }
            }
        }
        // ---- weights
        uint32_t pb[NB][kG][2];
        auto weigh = [&](auto ordinary) {  // p, its sums, and p step; one piece of code to a case
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            float(&p)[4] = y[b];
#pragma unroll
            for (int z = 0; z < 4; ++z) p[z] = ex2_approx(p[z]);
            l[b][0] += p[0] + p[2];
            l[b][1] += p[1] + p[3];
            const uint32_t p0 = pack_f16(p[0], p[1]), p1 = pack_f16(p[2], p[3]);
            if constexpr (ordinary.value) {
#pragma unroll
              for (int i = 0; i < kG; ++i) {
                pb[b][i][0] = transpose8(mul_lo(p0, vs[0][i]));
                pb[b][i][1] = transpose8(mul_lo(p1, vs[1][i]));
              }
            }
            mma_f16(low[b], lv[0], 0u, lv[1], 0u, transpose8(p0), transpose8(p1));
          }
        };
        if (!any_wide && exps == 0) {
          weigh(std::true_type{});
        } else {
          weigh(std::false_type{});
          int now = 0;
#pragma unroll
          for (int i = 0; i < kG; ++i) {
            const float s0 = half_lo(vs[0][i]), s1 = half_lo(vs[1][i]);
            float m = 0.f;  // a NaN is its column's own matter, and columns without a row are nobody's
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
              for (int z = 0; z < 2; ++z)
                if (b * 8 + 2 * lt + z < cols) m = fmaxf(m, fmaxf(y[b][z] * s0, y[b][z + 2] * s1));
            const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(m));
            int scale = any_wide ? scale_of(exps, i) : 0;
            const int ex = exponent(__uint_as_float(top));
            if (any_wide && top != 0 && (ex - scale > kProductTop || ex - scale < kProductLow))
              scale = max(kLeastScale, ex - kProductTop);
            now |= (scale & 255) << (8 * i);
            const float f0 = s0 * pow2i(-scale), f1 = s1 * pow2i(-scale);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
              pb[b][i][0] = transpose8(pack_f16(y[b][0] * f0, y[b][1] * f0));
              pb[b][i][1] = transpose8(pack_f16(y[b][2] * f1, y[b][3] * f1));
            }
          }
          if (now != exps) rescale(now);
        }
        // ---- values
        uint32_t v[4][D / 64];  // words g D / 64 .. of keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9
#pragma unroll
        for (int h = 0; h < 4; ++h)
          load_words(v[h], at + C::kCodes + (r0 + 2 * lt + (h & 1) + 8 * (h >> 1)) * (D / 2) + lg * (D / 16));
#pragma unroll
        for (int m = 0; m < 4; ++m) {  // byte m of the words: codes 2 m and 2 m + 1
          uint32_t f[D / 64][2];       // [word][keys 2 t.., 2 t + 8..]: that byte of both keys
#pragma unroll
          for (int w = 0; w < D / 64; ++w)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              f[w][h] = __byte_perm(v[2 * h][w], v[2 * h + 1][w], m | (m << 4) | ((4 + m) << 8) | ((4 + m) << 12));
          constexpr uint32_t kLo = 0x000F000Fu, kHi = 0x00F000F0u;
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            if constexpr (D == 128) {  // rows g and g + 8: words 2 g and 2 g + 1, one code of each
              mma_f16(o[b][2 * m], f[0][0] & kLo, f[1][0] & kLo, f[0][1] & kLo, f[1][1] & kLo, pb[b][m][0],
                      pb[b][m][1]);
              mma_f16(o[b][2 * m + 1], f[0][0] & kHi, f[1][0] & kHi, f[0][1] & kHi, f[1][1] & kHi, pb[b][m][0],
                      pb[b][m][1]);
            } else {  // rows g and g + 8: both codes of word g
              mma_f16(o[b][m], f[0][0] & kLo, f[0][0] & kHi, f[0][1] & kLo, f[0][1] & kHi, pb[b][m >> 1][0],
                      pb[b][m >> 1][1]);
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&empty_bar[slot]);
    }
    ring_at.end(n_steps);

    if (exps != 0) rescale(0);
    // ---- the warp's sums, for the join
    if (seg >= 1) wait(&jempty_bar, (seg - 1) & 1);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int z = 0; z < 2; ++z) {
#pragma unroll
        for (int m = 4; m < 32; m <<= 1) l[b][z] += __shfl_xor_sync(0xffffffffu, l[b][z], m);
        float lo[kG];  // the lanes of row g hold the sums of group g
#pragma unroll
        for (int i = 0; i < kG; ++i) lo[i] = __shfl_sync(0xffffffffu, low[b][z], 4 * i + lt);
        const int c = b * 8 + 2 * lt + z;
        if (lg == 0) {
          ref_sh[mine][c] = ref[b][z];
          sum_sh[mine][c] = l[b][z];
        }
        float* dst = join + (mine * 8 * NB + c) * C::kRow;
#pragma unroll
        for (int m = 0; m < kMt; ++m) {
          constexpr float f0 = kCodeUnit, f1 = kCodeUnit / 16.f;
          if constexpr (D == 128) {
            const float f = m & 1 ? f1 : f0;
            *reinterpret_cast<float2*>(dst + 16 * m + 2 * lg) =
                make_float2(fmaf(o[b][m][z], f, lo[m / 2]), fmaf(o[b][m][2 + z], f, lo[m / 2]));
          } else {
            dst[16 * m + lg] = fmaf(o[b][m][z], f0, lo[m / 2]);
            dst[16 * m + 8 + lg] = fmaf(o[b][m][2 + z], f1, lo[m / 2]);
          }
        }
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&jfull_bar);
  }
}

template <int D, int NB>
cudaError_t launch(const AtPlan& p, const Kernel4Args& k, cudaStream_t st) {
  using C = Cfg4<D, NB>;
  const cudaError_t e = allow_smem<attend4_kernel<D, NB>>(C::kSmem);
  if (e != cudaSuccess) return e;
  return launch_after(attend4_kernel<D, NB>, p.grid, C::kThreads, C::kSmem, st, k);
}

}  // namespace

cudaError_t launch_attend4(const Shape& s, const Attend4Args& a, const AtLayout& l, cudaStream_t st) {
  const AtPlan& p = l.own;
  Kernel4Args k{};
  k.geo = p.geo;
  k.geo.len = a.len;
  k.parts = p.parts(a.ws);
  k.sc = a.sc;
  k.q = a.q;
  k.K4 = a.K4;
  k.V4 = a.V4;
  k.S4 = a.S4;
  k.o = a.o;
  k.lse = a.lse;
  k.lse2 = reinterpret_cast<float*>(a.ws + l.off_lse2);
  k.logits = l.logits ? reinterpret_cast<float*>(a.ws + l.off_logits) : nullptr;
  k.err = a.err;
  const bool wide = p.geo.rr > 8;
  if (s.d == 128) return wide ? launch<128, 2>(p, k, st) : launch<128, 1>(p, k, st);
  return wide ? launch<64, 2>(p, k, st) : launch<64, 1>(p, k, st);
}

}  // namespace bkv
