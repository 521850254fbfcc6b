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

constexpr int kWarps4 = 8, kThreads4 = 32 * kWarps4;
constexpr int kSlice = 16;                 // keys of a warp's step
constexpr float kAbove4 = 4.f;             // log2 of how far p may exceed 1
constexpr float kStepTop = 2048.f;         // step 2^E stays at or below it
constexpr float kCodeUnit = 16777216.f;    // a code n stands as n / 2^24

// D += A B: A [16 x 16] and B [16 x 8] of fp16, fragments by lane as PTX defines them for m16n8k16.
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The transpose of an 8 x 8 matrix of 16-bit numbers, a row to four lanes.
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ float2 unpack_f16(uint32_t v) { return __half22float2(*reinterpret_cast<__half2*>(&v)); }

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

// What a warp loads of a slice; a thread's lane is 4 g + t.
template <int D>
struct Slice4 {
  static constexpr int kG = D / 32;
  uint32_t k[2][kG];         // K: words t kG .. of keys g and g + 8, one for each group
  uint32_t v[4][D / 64];     // V: words g D / 64 .. of keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9
  uint32_t ks[2][kG], vs[2][kG];  // (step, low) of keys g and g + 8
};

template <int D, int NB>
struct Cfg4 {
  static constexpr int kRow = D + 4;  // floats of a joined row, so that a warp's stores meet no bank twice
  static constexpr size_t kJoin = sizeof(float) * kWarps4 * 8 * NB * kRow;
  // a slot of a warp's ring: a slice's rows of K, V and scales
  static constexpr uint32_t kCodes = kSlice * D / 2, kScales = kSlice * D / 4, kSlot = 2 * kCodes + kScales;
  static constexpr int kDepth = (D == 128 ? 8 : 16) / NB + (NB > 1 ? 2 : 0);
  static constexpr size_t kSmem = kJoin + static_cast<size_t>(kWarps4) * kDepth * kSlot;
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

// The slices of a warp in the order in which it takes them, ahead of the warp itself.
struct Ahead4 {
  AtWalk walk;
  size_t row;  // of the caches: the present instance's first
  int j, j_end, len;
  __device__ __forceinline__ Ahead4(const AtGeo& g, const AtShare& s) : walk(g, s), row(0), j(0), j_end(0), len(0) {}
  // Moves to a slice there is, if one is left.
  __device__ __forceinline__ bool find(const AtGeo& g, int warp) {
    while (j >= j_end) {
      AtSeg s;
      if (!walk.next(g, s)) return false;
      row = static_cast<size_t>(s.e) * g.cap;
      len = s.len;
      j = s.t0 * kAtTile + warp * kSlice;
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
__global__ void __launch_bounds__(kThreads4, 1) attend4_kernel(Kernel4Args a) {
  using C = Cfg4<D, NB>;
  constexpr int kG = D / 32, kW = D / 8;  // groups, words of a row
  constexpr int kMt = D / 16;             // tiles of 16 elements of o
  extern __shared__ __align__(128) unsigned char smem4[];
  float* join = reinterpret_cast<float*>(smem4);  // [warp][8 NB rows][kRow]
  __shared__ __align__(8) uint64_t full_bar[kWarps4][C::kDepth];
  __shared__ float ref_sh[kWarps4][8 * NB], sum_sh[kWarps4][8 * NB];
  __shared__ int scan_sh[kThreads4 / 32];
  __shared__ AtShare share_sh;

  const AtGeo& g = a.geo;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, lg = lane >> 2, lt = lane & 3;
  if (lane == 0) {
    for (int i = 0; i < C::kDepth; ++i) mbar_init(&full_bar[warp][i], 1);
    fence_mbar_init();
  }
  grid_dependency_wait();
  grid_dependents_go();
  if (blockIdx.x == 0) at_check_lengths<kThreads4>(g, a.err);
  at_split_tiles<kThreads4>(g, scan_sh, &share_sh);
  if (tid == 0 && share_sh.left == 0) a.parts.cut[blockIdx.x] = make_int2(-1, -1);
  AtWalk walk(g, share_sh);

  // Every warp has a ring of its own, filled by its first lane: what the warp has read it may overwrite.
  unsigned char* ring = smem4 + C::kJoin + warp * (C::kDepth * C::kSlot);
  // with one row block to an instance every key is read once
  const uint64_t pol = g.nrb == 1 ? l2_policy_evict_first() : l2_policy_evict_last();
  Ahead4 ahead(g, share_sh);
  int slot = 0, phase = 0;  // of the slice to come
  int under_way = 0;        // slices loaded and not yet taken
  bool ok = true;           // false once a wait expired: nothing is loaded any more
  auto load_next = [&](int to) {
    if (!ahead.find(g, warp)) return;
    if (lane == 0) {
      const uint32_t n = min(kSlice, ahead.len - ahead.j);
      const size_t row = ahead.row + ahead.j;
      unsigned char* dst = ring + to * C::kSlot;
      uint64_t* bar = &full_bar[warp][to];
      mbar_arrive_expect_tx(bar, n * (D + D / 4));
      bulk_load(dst, a.K4 + row * kW, n * (D / 2), bar, pol);
      bulk_load(dst + 2 * C::kCodes, a.S4 + row * (2 * kG), n * (D / 4), bar, pol);
      bulk_load(dst + C::kCodes, a.V4 + row * kW, n * (D / 2), bar, pol);
    }
    ahead.j += kWarps4 * kSlice;
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

    // ---- the block's queries: right operands, and their sums over groups
    uint32_t qb[NB][kG][4];
    float qs[NB][kG][2], unit[NB][2];  // columns 2 t, 2 t + 1
    int lim[NB][2];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int c = b * 8 + lg;
      const bool there = c < cols;
      float x[kG][8], top = 0.f;
#pragma unroll
      for (int i = 0; i < kG; ++i) {
        uint4 r = make_uint4(0, 0, 0, 0);
        if (there) r = __ldg(reinterpret_cast<const uint4*>(a.q + (row0 + c) * D + 32 * i + 8 * lt));
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
      const int ex = max(exponent(top), -115);
      const float up = pow2i(11 - ex);
      float sums[kG];
#pragma unroll
      for (int i = 0; i < kG; ++i) {
        float sum = 0.f;
#pragma unroll
        for (int y = 0; y < 8; ++y) sum += x[i][y] *= up;
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        sums[i] = sum * (1.f / kCodeUnit);
        // codes 2 y and 2 y + 1 of a byte: the second stands 16 times as high
        qb[b][i][0] = pack_f16(x[i][0], x[i][4]);
        qb[b][i][1] = pack_f16(x[i][1] * 0.0625f, x[i][5] * 0.0625f);
        qb[b][i][2] = pack_f16(x[i][2], x[i][6]);
        qb[b][i][3] = pack_f16(x[i][3] * 0.0625f, x[i][7] * 0.0625f);
      }
      // columns 2 t and 2 t + 1 are the rows of lanes 8 t and 8 t + 4
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int from = 8 * lt + 4 * y;
#pragma unroll
        for (int i = 0; i < kG; ++i) qs[b][i][y] = __shfl_sync(0xffffffffu, sums[i], from);
        unit[b][y] = pow2i(__shfl_sync(0xffffffffu, ex, from) + 13);
        const int cc = b * 8 + 2 * lt + y;
        lim[b][y] = cc < cols ? at_limit(g, s.len, s.r0, cc) : 0;
      }
    }

    float o[NB][kMt][4] = {}, ol[NB][kG][2] = {}, l[NB][2] = {}, ref[NB][2];
#pragma unroll
    for (int b = 0; b < NB; ++b) ref[b][0] = ref[b][1] = kRefFloor;
    float grow = 0.f;  // 2^E

    const int j_end = min(s.t1 * kAtTile, limit_max);
    for (int j0 = s.t0 * kAtTile + warp * kSlice; j0 < j_end; j0 += kWarps4 * kSlice) {
      Slice4<D> x;
      ok = ok && __all_sync(0xffffffffu, at_wait(&full_bar[warp][slot], phase, nullptr, a.err, kDevTimeoutProducer));
      if (!ok) break;  // an expired wait: the outputs are invalid, the barriers below are still met
      const unsigned char* at = ring + slot * C::kSlot;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = lg + 8 * h;
        load_words(x.k[h], at + r * (D / 2) + lt * (kG * 4));
        load_words(x.ks[h], at + 2 * C::kCodes + r * (D / 4));
        load_words(x.vs[h], at + 2 * C::kCodes + r * (D / 4) + kG * 4);
      }
#pragma unroll
      for (int h = 0; h < 4; ++h)
        load_words(x.v[h], at + C::kCodes + (2 * lt + (h & 1) + 8 * (h >> 1)) * (D / 2) + lg * (D / 16));
      if (j0 + kSlice > s.len) {  // rows past the length hold anything
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < kG; ++i)
            if (j0 + lg + 8 * h >= s.len) x.vs[h][i] = 0;
      }
      __syncwarp();
      --under_way;
      load_next(slot);
      if (++slot == C::kDepth) {
        slot = 0;
        phase ^= 1;
      }
      // ---- logits
      float y[NB][4] = {};
#pragma unroll
      for (int i = 0; i < kG; ++i) {
        uint32_t f[2][4];  // codes (0, 4), (1, 5), (2, 6), (3, 7) of the word
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t w = x.k[h][i], w8 = w >> 8;
          f[h][0] = w & 0x000F000Fu;
          f[h][1] = w & 0x00F000F0u;
          f[h][2] = w8 & 0x000F000Fu;
          f[h][3] = w8 & 0x00F000F0u;
        }
        const float2 s0 = unpack_f16(x.ks[0][i]), s1 = unpack_f16(x.ks[1][i]);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          float c[4] = {};
          mma_f16(c, f[0][0], f[1][0], f[0][1], f[1][1], qb[b][i][0], qb[b][i][1]);
          mma_f16(c, f[0][2], f[1][2], f[0][3], f[1][3], qb[b][i][2], qb[b][i][3]);
          y[b][0] = fmaf(s0.x, c[0], fmaf(s0.y, qs[b][i][0], y[b][0]));
          y[b][1] = fmaf(s0.x, c[1], fmaf(s0.y, qs[b][i][1], y[b][1]));
          y[b][2] = fmaf(s1.x, c[2], fmaf(s1.y, qs[b][i][0], y[b][2]));
          y[b][3] = fmaf(s1.x, c[3], fmaf(s1.y, qs[b][i][1], y[b][3]));
        }
      }
      // ---- to base 2, against the references
      float above = -INFINITY;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          y[b][z] *= unit[b][z & 1];
          const int j = j0 + lg + 8 * (z >> 1), c = b * 8 + 2 * lt + (z & 1);
          if (a.logits && c < cols && j < s.len) a.logits[(row0 + c) * g.cap + j] = y[b][z];
          y[b][z] *= a.sc;
          if (j0 + kSlice > limit_min) y[b][z] = j < lim[b][z & 1] ? y[b][z] : -INFINITY;
          above = fmaxf(above, y[b][z] - ref[b][z & 1]);
        }
      }
      float2 vs[2][kG];
      float step = 0.f;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < kG; ++i) {
          vs[h][i] = unpack_f16(x.vs[h][i]);
          step = fmaxf(step, vs[h][i].x);
        }
      if (__any_sync(0xffffffffu, above > kAbove4 || step * grow > kStepTop || grow == 0.f)) {
        // move the references to the slice's maxima, and the steps' scale
        float fac[NB][2];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            float v = fmaxf(y[b][z], y[b][z + 2]);
#pragma unroll
            for (int m = 4; m < 32; m <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, m));
            v = fmaxf(v, ref[b][z]);
            fac[b][z] = ex2_approx(ref[b][z] - v);
            ref[b][z] = v;
            l[b][z] *= fac[b][z];
#pragma unroll
            for (int i = 0; i < kG; ++i) ol[b][i][z] *= fac[b][z];
          }
#pragma unroll
        for (int m = 1; m < 32; m <<= 1) step = fmaxf(step, __shfl_xor_sync(0xffffffffu, step, m));
        float regrow = 1.f;
        if (step * grow > kStepTop || grow == 0.f) {
          const float now = pow2i(7 - exponent(step));
          regrow = grow == 0.f ? 0.f : now / grow;
          grow = now;
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int m = 0; m < kMt; ++m)
#pragma unroll
            for (int z = 0; z < 4; ++z) o[b][m][z] *= fac[b][z & 1] * regrow;
      }
      // ---- weights
      uint32_t pb[NB][kG][2];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        float p[4];
#pragma unroll
        for (int z = 0; z < 4; ++z) p[z] = ex2_approx(y[b][z] - ref[b][z & 1]);
        l[b][0] += p[0] + p[2];
        l[b][1] += p[1] + p[3];
#pragma unroll
        for (int i = 0; i < kG; ++i) {
          ol[b][i][0] = fmaf(p[0], vs[0][i].y, fmaf(p[2], vs[1][i].y, ol[b][i][0]));
          ol[b][i][1] = fmaf(p[1], vs[0][i].y, fmaf(p[3], vs[1][i].y, ol[b][i][1]));
          const float s0 = vs[0][i].x * grow, s1 = vs[1][i].x * grow;
          pb[b][i][0] = transpose8(pack_f16(p[0] * s0, p[1] * s0));
          pb[b][i][1] = transpose8(pack_f16(p[2] * s1, p[3] * s1));
        }
      }
      // ---- values
#pragma unroll
      for (int m = 0; m < 4; ++m) {  // byte m of the words: codes 2 m and 2 m + 1
        uint32_t f[D / 64][2];       // [word][keys 2 t.., 2 t + 8..]: that byte of both keys
#pragma unroll
        for (int w = 0; w < D / 64; ++w)
#pragma unroll
          for (int h = 0; h < 2; ++h)
            f[w][h] = __byte_perm(x.v[2 * h][w], x.v[2 * h + 1][w], m | (m << 4) | ((4 + m) << 8) | ((4 + m) << 12));
        constexpr uint32_t kLo = 0x000F000Fu, kHi = 0x00F000F0u;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          if constexpr (D == 128) {  // rows g and g + 8: words 2 g and 2 g + 1, one code of each
            mma_f16(o[b][2 * m], f[0][0] & kLo, f[1][0] & kLo, f[0][1] & kLo, f[1][1] & kLo, pb[b][m][0], pb[b][m][1]);
            mma_f16(o[b][2 * m + 1], f[0][0] & kHi, f[1][0] & kHi, f[0][1] & kHi, f[1][1] & kHi, pb[b][m][0],
                    pb[b][m][1]);
          } else {  // rows g and g + 8: both codes of word g
            mma_f16(o[b][m], f[0][0] & kLo, f[0][0] & kHi, f[0][1] & kLo, f[0][1] & kHi, pb[b][m >> 1][0],
                    pb[b][m >> 1][1]);
          }
        }
      }
    }

    // ---- join the warps
    const float shrink = grow == 0.f ? 0.f : kCodeUnit / grow;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int z = 0; z < 2; ++z) {
#pragma unroll
        for (int m = 4; m < 32; m <<= 1) {
          l[b][z] += __shfl_xor_sync(0xffffffffu, l[b][z], m);
#pragma unroll
          for (int i = 0; i < kG; ++i) ol[b][i][z] += __shfl_xor_sync(0xffffffffu, ol[b][i][z], m);
        }
        const int c = b * 8 + 2 * lt + z;
        if (lg == 0) {
          ref_sh[warp][c] = ref[b][z];
          sum_sh[warp][c] = l[b][z];
        }
        float* dst = join + (warp * 8 * NB + c) * C::kRow;
#pragma unroll
        for (int m = 0; m < kMt; ++m) {
          const float lo = ol[b][m / 2][z];
          if constexpr (D == 128) {
            const float f = m & 1 ? shrink * 0.0625f : shrink;
            *reinterpret_cast<float2*>(dst + 16 * m + 2 * lg) =
                make_float2(fmaf(o[b][m][z], f, lo), fmaf(o[b][m][2 + z], f, lo));
          } else {
            dst[16 * m + lg] = fmaf(o[b][m][z], shrink, lo);
            dst[16 * m + 8 + lg] = fmaf(o[b][m][2 + z], shrink * 0.0625f, lo);
          }
        }
      }
    }
    __syncthreads();
    const bool whole = s.t0 == 0 && s.t1 == s.T;
    const size_t part = (static_cast<size_t>(blockIdx.x) + s.item) * a.parts.rows;
    for (int c = warp; c < cols; c += kWarps4) {
      float m = kRefFloor, sum = 0.f, f[kWarps4];
#pragma unroll
      for (int w = 0; w < kWarps4; ++w) m = fmaxf(m, ref_sh[w][c]);
#pragma unroll
      for (int w = 0; w < kWarps4; ++w) {
        f[w] = ex2_approx(ref_sh[w][c] - m);
        sum = fmaf(sum_sh[w][c], f[w], sum);
      }
      const float inv = sum != 0.f ? 1.f / sum : 0.f;
      for (int d = lane; d < D; d += 32) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps4; ++w) v = fmaf(join[(w * 8 * NB + c) * C::kRow + d], f[w], v);
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
  return launch_after(attend4_kernel<D, NB>, p.grid, kThreads4, C::kSmem, st, k);
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
