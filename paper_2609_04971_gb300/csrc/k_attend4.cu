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
// power of two of each row, are exact in fp16 down to 2^-24 of the row's largest element; p step is rounded to fp16 once
// (2^-11 of itself; below some 2^-31 of the largest it becomes 0).
//
// Warps, not the tcgen05 unit, hold the operands: m16n8k16 products take the unpacked codes from the registers
// they are unpacked in, where tcgen05 would need 16-bit copies of every code in shared memory, four times the
// bytes that come from HBM, written and read again.
//
// Persistent, one CTA per SM, the work split into segments as in k_attend.cuh.  A warp takes slices
// of 16 keys: S [16 keys x 8 rows] per block of 8 query rows, P transposed in registers (movmatrix), and
// O^T [D x 8 rows] += V^T P.  Each warp has its own reference m of a row's logits (base 2): it moves up
// when a logit exceeds it by more than 4, and p = 2^(y - m) stays below 2^4.  The steps are scaled by a
// power of two 2^E, which moves likewise, so that p step 2^E fits fp16.  The warps' sums are joined in shared
// memory at a segment's end.
#include <cuda_fp16.h>

#include "k_attend.cuh"

namespace bkv {
namespace {

constexpr int kSlice = 16, kStep = 2 * kSlice;  // keys of a product, of a warp's step
constexpr float kAbove4 = 4.f;                  // log2 of how far p may exceed 2^E
constexpr float kStepTop = 2048.f;              // step 2^E stays at or below it
constexpr int kMostUp = 11;                     // E stays at or below it
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
__device__ __forceinline__ uint32_t max_f16x2(uint32_t a, uint32_t b) {
  const __half2 m = __hmax2(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&m);
}

// 2^k for any k (0 below the normal range).
__device__ __forceinline__ float pow2i(int k) {
  return k < -126 ? 0.f : __uint_as_float(static_cast<uint32_t>(min(k, 127) + 127) << 23);
}
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
  static constexpr int kWarps = NB == 1 ? 12 : 8, kThreads = 32 * kWarps;
  static constexpr int kRow = D + 4;  // floats of a joined row, so that a warp's stores meet no bank twice
  static constexpr size_t kJoin = sizeof(float) * kWarps * 8 * NB * kRow;
  // a slot of a warp's ring: a step's rows of K, V and scales
  static constexpr uint32_t kCodes = kStep * D / 2, kScales = kStep * D / 4, kSlot = 2 * kCodes + kScales;
  static constexpr int kDepth = (D == 128 ? 2 : 4) + (NB > 1);
  static constexpr size_t kSmem = kJoin + static_cast<size_t>(kWarps) * kDepth * kSlot;
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

// The steps of a warp in the order in which it takes them, ahead of the warp itself.
template <int WARPS>
struct Ahead4 {
  AtWalk walk;
  size_t row;  // of the caches: the present instance's first
  int j, j_end, len;
  __device__ __forceinline__ Ahead4(const AtGeo& g, const AtShare& s) : walk(g, s), row(0), j(0), j_end(0), len(0) {}
  // Moves to a step there is, if one is left.
  __device__ __forceinline__ bool find(const AtGeo& g, int warp) {
    while (j >= j_end) {
      AtSeg s;
      if (!walk.next(g, s)) return false;
      row = static_cast<size_t>(s.e) * g.cap;
      len = s.len;
      j = s.t0 * kAtTile + warp * kStep;
      j_end = min(s.t1 * kAtTile, at_limit_max(g, s.len, s.r0));
    }
    return true;
  }
};

// Linear copy of `bytes` (a multiple of 16, both ends 16-byte aligned) into shared memory.
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(
          smem_u32(dst)),
      "l"(src), "r"(bytes), "r"(smem_u32(bar)), "l"(policy)
      : "memory");
}

template <int D, int NB>
__global__ void __launch_bounds__(Cfg4<D, NB>::kThreads, 1) attend4_kernel(Kernel4Args a) {
  using C = Cfg4<D, NB>;
  constexpr int kWarps = C::kWarps;
  constexpr int kG = D / 32, kW = D / 8;  // groups, words of a row
  constexpr int kMt = D / 16;             // tiles of 16 elements of o
  extern __shared__ __align__(128) unsigned char smem4[];
  float* join = reinterpret_cast<float*>(smem4);  // [warp][8 NB rows][kRow]
  __shared__ __align__(8) uint64_t full_bar[kWarps][C::kDepth];
  __shared__ float ref_sh[kWarps][8 * NB], sum_sh[kWarps][8 * NB];
  __shared__ int scan_sh[kWarps];
  __shared__ AtShare share_sh;

  const AtGeo& g = a.geo;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, lg = lane >> 2, lt = lane & 3;
  if (lane == 0) {
    for (int i = 0; i < C::kDepth; ++i) mbar_init(&full_bar[warp][i], 1);
    fence_mbar_init();
  }
  grid_dependency_wait();
  grid_dependents_go();
  if (blockIdx.x == 0) at_check_lengths<C::kThreads>(g, a.err);
  at_split_tiles<C::kThreads>(g, scan_sh, &share_sh);
  if (tid == 0 && share_sh.left == 0) a.parts.cut[blockIdx.x] = make_int2(-1, -1);
  AtWalk walk(g, share_sh);

  // Every warp has a ring of its own, filled by its first lane: what the warp has read it may overwrite.
  unsigned char* ring = smem4 + C::kJoin + warp * (C::kDepth * C::kSlot);
  // with one row block to an instance every key is read once
  const uint64_t pol = g.nrb == 1 ? l2_policy_evict_first() : l2_policy_evict_last();
  Ahead4<kWarps> ahead(g, share_sh);
  int slot = 0, phase = 0;  // of the step to come
  int under_way = 0;        // steps loaded and not yet taken
  bool ok = true;           // false once a wait expired: nothing is loaded any more
  auto load_next = [&](int to) {
    if (!ahead.find(g, warp)) return;
    if (lane == 0) {
      const uint32_t n = min(kStep, ahead.len - ahead.j);
      const size_t row = ahead.row + ahead.j;
      unsigned char* dst = ring + to * C::kSlot;
      uint64_t* bar = &full_bar[warp][to];
      mbar_arrive_expect_tx(bar, n * (D + D / 4));
      bulk_load(dst, a.K4 + row * kW, n * (D / 2), bar, pol);
      bulk_load(dst + 2 * C::kCodes, a.S4 + row * (2 * kG), n * (D / 4), bar, pol);
      bulk_load(dst + C::kCodes, a.V4 + row * kW, n * (D / 2), bar, pol);
    }
    ahead.j += kWarps * kStep;
    ++under_way;
  };
#pragma unroll 1
  for (int i = 0; i < C::kDepth; ++i) load_next(i);

  AtSeg s, next;
  bool more = walk.next(g, next);
  while (more) {
    s = next;
    more = walk.next(g, next);
    if (tid == 0) at_note(a.parts, s, !more, share_sh.per);
    const int cols = min(g.rr, g.R - s.r0);       // rows of this block
    const int limit_max = at_limit_max(g, s.len, s.r0), limit_min = at_limit_min(g, s.len, s.r0);
    const size_t row0 = static_cast<size_t>(s.e) * g.R + s.r0;  // of q, o and lse

    // ---- the block's queries: right operands, and their sums over groups as three fp16 terms
    uint32_t qb[NB][kG][4], qs[NB][2];
    float unit[NB][2];  // columns 2 t, 2 t + 1: what a logit counts in
    int lim[NB][2];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int c = b * 8 + lg;
      float x[kG][8], top = 0.f;
#pragma unroll
      for (int i = 0; i < kG; ++i) {
        uint4 r = make_uint4(0, 0, 0, 0);
        if (c < cols) r = __ldg(reinterpret_cast<const uint4*>(a.q + (row0 + c) * D + 32 * i + 8 * lt));
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          x[i][2 * y] = __uint_as_float(w[y] << 16);
          x[i][2 * y + 1] = __uint_as_float(w[y] & 0xFFFF0000u);
          top = fmaxf(top, fmaxf(fabsf(x[i][2 * y]), fabsf(x[i][2 * y + 1])));
        }
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int ex = top == 0.f ? 0 : max(exponent(top), -115);
      const float up = pow2i(11 - ex);
      float term[kG][3];
#pragma unroll
      for (int i = 0; i < kG; ++i) {
        float sum = 0.f;
#pragma unroll
        for (int y = 0; y < 8; ++y) sum += x[i][y] *= up;
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        sum *= 1.f / kSumUnit;
#pragma unroll
        for (int z = 0; z < 3; ++z) {
          term[i][z] = __half2float(__float2half_rn(sum));
          sum -= term[i][z];
        }
        // codes 2 y and 2 y + 1 of a byte: the second stands 16 times as high
        qb[b][i][0] = pack_f16(x[i][0], x[i][4]);
        qb[b][i][1] = pack_f16(x[i][1] * 0.0625f, x[i][5] * 0.0625f);
        qb[b][i][2] = pack_f16(x[i][2], x[i][6]);
        qb[b][i][3] = pack_f16(x[i][3] * 0.0625f, x[i][7] * 0.0625f);
      }
      // Products with the keys' lows: k = 2 t, 2 t + 1 are a pair of groups and a term, k = 2 t + 8, 2 t + 9 too.
      if constexpr (D == 128) {
        const bool odd = lt & 1;
        const float h0 = odd ? term[2][0] : term[0][0], h1 = odd ? term[3][0] : term[1][0];
        const float m0 = odd ? term[2][1] : term[0][1], m1 = odd ? term[3][1] : term[1][1];
        const float l0 = odd ? term[2][2] : term[0][2], l1 = odd ? term[3][2] : term[1][2];
        qs[b][0] = lt < 2 ? pack_f16(h0, h1) : pack_f16(m0, m1);
        qs[b][1] = lt < 2 ? pack_f16(l0, l1) : 0u;
      } else {
        qs[b][0] = lt == 0   ? pack_f16(term[0][0], term[1][0])
                   : lt == 1 ? pack_f16(term[0][1], term[1][1])
                   : lt == 2 ? pack_f16(term[0][2], term[1][2])
                             : 0u;
        qs[b][1] = 0u;
      }
      // columns 2 t and 2 t + 1 are the rows of lanes 8 t and 8 t + 4
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        unit[b][y] = pow2i(__shfl_sync(0xffffffffu, ex, 8 * lt + 4 * y) + 13);
        const int cc = b * 8 + 2 * lt + y;
        lim[b][y] = cc < cols ? at_limit(g, s.len, s.r0, cc) : 0;
      }
    }

    // p = 2^(y - ref): ref is the reference of the column less E
    float o[NB][kMt][4] = {}, low[NB][4] = {}, l[NB][2] = {}, ref[NB][2];
    int up = -1000;  // E; none yet
#pragma unroll
    for (int b = 0; b < NB; ++b) ref[b][0] = ref[b][1] = 0.f;

    const int j_end = min(s.t1 * kAtTile, limit_max);
#pragma unroll 1
    for (int j0 = s.t0 * kAtTile + warp * kStep; j0 < j_end; j0 += kWarps * kStep) {
      ok = ok && __all_sync(0xffffffffu, at_wait(&full_bar[warp][slot], phase, nullptr, a.err, kDevTimeoutProducer));
      if (!ok) break;  // an expired wait: the outputs are invalid, the barriers below are still met
      const unsigned char* at = ring + slot * C::kSlot;
      const unsigned char* scales = at + 2 * C::kCodes;
      const bool tail = j0 + kStep > s.len;  // rows past the length hold anything
      // ---- logits, in the columns' units
      float y[2][NB][4];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        uint32_t k[2][kG], ks[2][kG];
        uint32_t lows[2];  // of a pair of groups of keys g and g + 8
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = u * kSlice + lg + 8 * h;
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
          for (int z = 0; z < 4; ++z) y[u][b][z] = c[z] * (kSumUnit / kCodeUnit);
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
            y[u][b][0] = fmaf(s0, c[0], y[u][b][0]);
            y[u][b][1] = fmaf(s0, c[1], y[u][b][1]);
            y[u][b][2] = fmaf(s1, c[2], y[u][b][2]);
            y[u][b][3] = fmaf(s1, c[3], y[u][b][3]);
          }
        }
      }
      if (a.logits) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            const int c = b * 8 + 2 * lt + z;
            if (c < cols) {
              float* dst = a.logits + (row0 + c) * g.cap + j0 + lg;
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if (!tail || j0 + lg + 8 * r < s.len) dst[8 * r] = y[r >> 1][b][z + 2 * (r & 1)] * unit[b][z];
            }
          }
      }
      // the largest step of V
      auto v_scales = [&](int u, int h, uint32_t(&w)[kG]) {  // (step, low) of keys g and g + 8 of a product
        const int r = u * kSlice + lg + 8 * h;
        load_words(w, scales + r * (D / 4) + kG * 4);
        if (tail && j0 + r >= s.len) {
#pragma unroll
          for (int i = 0; i < kG; ++i) w[i] = 0;
        }
      };
      uint32_t top2 = 0;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        uint32_t w[kG];
        v_scales(x >> 1, x & 1, w);
#pragma unroll
        for (int i = 0; i < kG; ++i) top2 = max_f16x2(top2, w[i]);
      }
      // ---- to base 2, against the references
      const float step = half_lo(top2), most = 16.f * pow2i(up);  // p 2^-E may be 2^4
      float above = -INFINITY;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          const float f = unit[b][z & 1] * a.sc;
          y[0][b][z] = fmaf(y[0][b][z], f, -ref[b][z & 1]);
          y[1][b][z] = fmaf(y[1][b][z], f, -ref[b][z & 1]);
        }
      if (j0 + kStep > limit_min) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int z = 0; z < 4; ++z)
              if (j0 + u * kSlice + lg + 8 * (z >> 1) >= lim[b][z & 1]) y[u][b][z] = -INFINITY;
      }
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int z = 0; z < 4; ++z) above = fmaxf(above, fmaxf(y[0][b][z], y[1][b][z]));
      if (__any_sync(0xffffffffu, above > kAbove4 + up || step * most > 16.f * kStepTop || up < -999)) {
        // Move the references to the step's maxima, and the steps' scale.  A column that sees nothing of a warp's
        // first step sees nothing after it either: it stays at the floor.
        float top = step;
#pragma unroll
        for (int m = 1; m < 32; m <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
        const int now = up < -999 || top * most > 16.f * kStepTop ? min(kMostUp, 7 - exponent(top)) : up;
        const bool begins = up < -999;
        const float back = begins ? kRefFloor : static_cast<float>(up);
        up = now;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            float v = fmaxf(fmaxf(y[0][b][z], y[0][b][z + 2]), fmaxf(y[1][b][z], y[1][b][z + 2]));
#pragma unroll
            for (int m = 4; m < 32; m <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, m));
            // relative to ref: the reference was at `back`; it moves up to v, and 2^E moves to `now`
            const float by = fmaxf(v, back) - static_cast<float>(now);
            const float fac = begins ? 0.f : ex2_approx(-by);
            ref[b][z] += by;
            l[b][z] *= fac;
            low[b][z] *= fac;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              y[u][b][z] -= by;
              y[u][b][z + 2] -= by;
            }
#pragma unroll
            for (int m = 0; m < kMt; ++m) {
              o[b][m][z] *= fac;
              o[b][m][z + 2] *= fac;
            }
          }
      }
      // ---- weights and values
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        uint32_t vs[2][kG], lv[2];  // lv: lows of group g of keys 2 t, 2 t + 1 and 2 t + 8, 2 t + 9
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          v_scales(u, h, vs[h]);
          uint32_t w[2];
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            const int r = u * kSlice + 8 * h + 2 * lt + z;
            w[z] = *reinterpret_cast<const uint32_t*>(scales + r * (D / 4) + kG * 4 + (lg & (kG - 1)) * 4);
            if (tail && j0 + r >= s.len) w[z] = 0;
          }
          lv[h] = __byte_perm(w[0], w[1], 0x7632);
        }
        uint32_t pb[NB][kG][2];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          float p[4];
#pragma unroll
          for (int z = 0; z < 4; ++z) p[z] = ex2_approx(y[u][b][z]);
          l[b][0] += p[0] + p[2];
          l[b][1] += p[1] + p[3];
#pragma unroll
          for (int i = 0; i < kG; ++i) {
            const float s0 = half_lo(vs[0][i]), s1 = half_lo(vs[1][i]);
            pb[b][i][0] = transpose8(pack_f16(p[0] * s0, p[1] * s0));
            pb[b][i][1] = transpose8(pack_f16(p[2] * s1, p[3] * s1));
          }
          mma_f16(low[b], lv[0], 0u, lv[1], 0u, transpose8(pack_f16(p[0], p[1])),
                  transpose8(pack_f16(p[2], p[3])));
        }
        uint32_t v[4][D / 64];  // words g D / 64 .. of keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9
#pragma unroll
        for (int h = 0; h < 4; ++h)
          load_words(v[h], at + C::kCodes + (u * kSlice + 2 * lt + (h & 1) + 8 * (h >> 1)) * (D / 2) + lg * (D / 16));
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
      --under_way;
      load_next(slot);
      if (++slot == C::kDepth) {
        slot = 0;
        phase ^= 1;
      }
    }

    // ---- join the warps
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
          ref_sh[warp][c] = ref[b][z];
          sum_sh[warp][c] = l[b][z];
        }
        float* dst = join + (warp * 8 * NB + c) * C::kRow;
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
    __syncthreads();
    const bool whole = s.t0 == 0 && s.t1 == s.T;
    const size_t part = (static_cast<size_t>(blockIdx.x) + s.item) * a.parts.rows;
    for (int c = warp; c < cols; c += kWarps) {
      float m = kRefFloor, sum = 0.f, f[kWarps];
#pragma unroll
      for (int w = 0; w < kWarps; ++w) m = fmaxf(m, ref_sh[w][c]);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        f[w] = ex2_approx(ref_sh[w][c] - m);
        sum = fmaf(sum_sh[w][c], f[w], sum);
      }
      const float inv = sum != 0.f ? 1.f / sum : 0.f;
      for (int d = lane; d < D; d += 32) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) v = fmaf(join[(w * 8 * NB + c) * C::kRow + d], f[w], v);
        if (whole) a.o[(row0 + c) * D + d] = __float2bfloat16(v * inv);
        else a.parts.o[(part + c) * D + d] = v;
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
    __syncthreads();
  }
  if (!ok) {  // let every copy already issued land before the CTA exits
    for (; under_way > 0; --under_way) {
      at_wait_always(&full_bar[warp][slot], phase, a.err, kDevTimeoutDrain, 1);
      if (++slot == C::kDepth) {
        slot = 0;
        phase ^= 1;
      }
    }
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
