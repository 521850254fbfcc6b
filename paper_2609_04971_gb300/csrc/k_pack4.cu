// Rows of K and V into and out of caches held in 4 bits (include/bkv.h, bkv_pack4
// and bkv_unpack4).
//
// A group of 32 elements x keeps low = fp16(min x), step = fp16((max x - low) / 15) and the codes
// n = rint((x - low) / step) in 0..15; it stands for low + step n.  Each of the three is the rounding of the
// exact quotient or difference, so that the codes do not depend on how they are computed: the step's
// quotient is rounded to odd in fp32 before fp16 (a second rounding to nearest would decide ties wrongly), and a
// code whose quotient comes close to a tie is decided by the exact sign of the difference from it.
//
// One thread to eight elements of a row of K and the same of V; a group is four threads.  A row of
// K stores a thread's eight codes as one word.  A row of V stores in one word what the attention's
// products need of eight of their rows, which eight threads hold: a transpose in three exchanges.
//
// Bound by HBM: 4 d bytes of bf16 and 1.25 d bytes of codes and scales a row.  295 thousand rows of head_dim 128,
// cold: packed in 58.5 us (199 MB, 3.4 TB/s; some 140 instructions to eight elements), read back in 35 us (5.6 TB/s).
#include <cuda_fp16.h>

#include <cfloat>

#include "bkv_device.cuh"
#include "bkv_internal.h"
#include "k_attend.cuh"
#include "k_launch.cuh"

namespace bkv {
namespace {

constexpr int kPackThreads = 256, kBatch = 4;
constexpr float kHalfMax = 65504.f;

// Rows of a new block that instance e takes: cache rows first .. first + n.
struct Span4 {
  int first, n;
};
__device__ __forceinline__ Span4 span4(const Pack4Args& a, int e, bool report) {
  const int len = __ldg(a.len + e), first = a.first ? __ldg(a.first + e) : 0;
  if (len < 0 || len > a.cap || first < 0 || first > len) {
    if (report) record_error(a.err, kDevBadLength);
    return {0, 0};
  }
  return {first, min(a.n_rows, len - first)};
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// The code of x by the exact sign of x - low - (n + 1/2) step, where the quotient f may lie on the wrong side of a tie.
__device__ __forceinline__ int code_near_tie(float x, float low, float step, float f) {
  const int n = min(14, max(0, static_cast<int>(floorf(f))));
  const float edge = (static_cast<float>(n) + 0.5f) * step;  // at most 16 significant bits
  const float s = x - low, bb = s - x;                        // s + err = x - low exactly
  const float err = (x - (s - bb)) + (-low - bb);
  const float t = (s - edge) + err;
  return t > 0.f || (t == 0.f && (n & 1)) ? n + 1 : n;
}
__device__ __forceinline__ uint32_t min_bf16x2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 m = __hmin2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&m);
}

// Codes of eight elements of a group that four neighbouring threads share, as a word, and the group's (step, low).
__device__ __forceinline__ uint32_t quantise(const uint4& raw, uint32_t& scale) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
  constexpr uint32_t kSigns = 0x80008000u;
  uint32_t lo2 = min_bf16x2(min_bf16x2(w[0], w[1]), min_bf16x2(w[2], w[3]));
  uint32_t hi2 = min_bf16x2(min_bf16x2(w[0] ^ kSigns, w[1] ^ kSigns), min_bf16x2(w[2] ^ kSigns, w[3] ^ kSigns));
  // (smallest, minus the largest) of this thread, then of the group
  uint32_t ends = min_bf16x2(__byte_perm(lo2, hi2, 0x5410), __byte_perm(lo2, hi2, 0x7632));
#pragma unroll
  for (int o = 1; o <= 2; o <<= 1) ends = min_bf16x2(ends, __shfl_xor_sync(0xffffffffu, ends, o));
  const float lo = bf16_lo(ends), hi = -bf16_hi(ends);
  const __half low16 = __float2half_rn(fminf(fmaxf(lo, -kHalfMax), kHalfMax));
  const float low = __half2float(low16);
  const float range = fmaxf(0.f, __fsub_rd(hi, low));
  // range / 15 with its last bit set where it is not exact; what is left of range tells on which side q lies
  constexpr float kBy15 = 1.f / 15.f;
  float q = range * kBy15;
  q = fmaf(fmaf(-15.f, q, range), kBy15, q);
  const float rest = fmaf(-15.f, q, range);
  uint32_t bits = __float_as_uint(q);
  if (rest < 0.f) --bits;
  if (rest != 0.f || __fsub_ru(hi, low) != range) bits |= 1u;
  const __half step16 = __float2half_rn(range < 15.f * kHalfMax ? __uint_as_float(bits) : kHalfMax);
  const float step = __half2float(step16), inv = step > 0.f ? __fdividef(kBy15, step) : 0.f;
  scale = static_cast<uint32_t>(__half_as_ushort(step16)) | (static_cast<uint32_t>(__half_as_ushort(low16)) << 16);
  // n = rint(f), f = 15 clamp((x - low) / (15 step)) to 1e-5: what is added and taken away leaves no fraction in fp32.
  // Where f is as near to a tie n may be wrong: 1 element in 2000 of random rows, most of them ties to the bit.
  constexpr float kRound = 12582912.f;  // 1.5 2^23
  float n[8];
  uint32_t near = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = i & 1 ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]);
    const float f = __saturatef((x - low) * inv);
    n[i] = fmaf(f, 15.f, kRound) - kRound;
    if (fabsf(fmaf(f, 15.f, -n[i])) > 0.49998f) near |= 1u << i;
  }
  const float a = fmaf(n[3], 4096.f, fmaf(n[2], 256.f, fmaf(n[1], 16.f, n[0])));
  const float b = fmaf(n[7], 4096.f, fmaf(n[6], 256.f, fmaf(n[5], 16.f, n[4])));
  uint32_t word = __byte_perm(__float_as_uint(a + 8388608.f), __float_as_uint(b + 8388608.f), 0x5410);  // below 2^16
#pragma unroll 1
  while (near) {
    const int i = __ffs(near) - 1;
    near &= near - 1;
    const uint32_t pair = i < 4 ? (i < 2 ? w[0] : w[1]) : (i < 6 ? w[2] : w[3]);
    const float x = i & 1 ? bf16_hi(pair) : bf16_lo(pair);
    const uint32_t code = code_near_tie(x, low, step, fminf(15.f, fmaxf(0.f, (x - low) * (15.f * inv))));
    word = (word & ~(15u << (4 * i))) | code << (4 * i);
  }
  return word;
}

// A row of V stores the transpose of its codes: eight threads whose words hold codes r = 0 .. 7 of elements 8 i + r end
// with one word each of code r = their number among the eight, in three exchanges of halves.  The threads are
// `apart` lanes from one another; x is the thread's number.  The transpose is its own inverse.
template <int APART>
__device__ __forceinline__ uint32_t transpose_codes(uint32_t w, int x) {
#pragma unroll
  for (int b = 0; b < 3; ++b) {
    const uint32_t low = b == 0 ? 0x0F0F0F0Fu : b == 1 ? 0x00FF00FFu : 0x0000FFFFu;
    const bool up = x >> b & 1;
    const uint32_t p = __shfl_xor_sync(0xffffffffu, w, APART << b);
    const uint32_t take = up ? low : ~low;  // codes that come from the other thread
    w = (w & ~take) | (__funnelshift_l(p, p, up ? 32 - (4 << b) : 4 << b) & take);
  }
  return w;
}
// Of a row's D / 8 threads, thread i holds codes of elements 8 i .. 8 i + 7, and after the transpose word v_word(i).
template <int D>
__device__ __forceinline__ int v_word(int i) {
  return D == 128 ? 8 * (i & 1) + (i >> 1) : i;
}
template <int D>
__device__ __forceinline__ uint32_t transpose_row(uint32_t w, int i) {
  return D == 128 ? transpose_codes<2>(w, i >> 1) : transpose_codes<1>(w, i);
}

__device__ __forceinline__ uint4 values(uint32_t codes, uint32_t scale) {
  const float step = __half2float(__ushort_as_half(static_cast<unsigned short>(scale & 0xFFFFu))),
              low = __half2float(__ushort_as_half(static_cast<unsigned short>(scale >> 16)));
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = fmaf(step, static_cast<float>((codes >> (4 * i)) & 15u), low);
  return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}

// kBatch rows to a thread, their loads under way together: 295 thousand rows of head_dim 128, with one row to a thread,
// 71 us to pack and 43 us to read back; with four 61 and 36 us (launches timed by events).
template <int D, bool PACK>
__global__ void __launch_bounds__(kPackThreads) pack4_kernel(Pack4Args a, FastDiv by_blocks) {
  constexpr int T = D / 8, kRows = kPackThreads / T;  // threads per row, rows of a pass
  constexpr int kGroups = D / 32;
  grid_dependency_wait();
  grid_dependents_go();
  int e;
  const int i0 = by_blocks.mod(blockIdx.x, e) * (kRows * kBatch);
  const Span4 span = span4(a, e, i0 == 0 && threadIdx.x == 0);
  if (i0 >= span.n) return;
  const int i = threadIdx.x % T, r0 = i0 + threadIdx.x / T;
  const int grp = i >> 2, t = i & 3;
  const size_t in = (static_cast<size_t>(e) * a.n_rows + r0) * T + i;
  const size_t row = static_cast<size_t>(e) * a.cap + span.first + r0;
  uint32_t* k4 = a.K4 + row * T + t * kGroups + grp;
  uint32_t* v4 = a.V4 + row * T + v_word<D>(i);
  uint32_t* s4 = a.S4 + row * (2 * kGroups) + grp;
  if (PACK) {
    uint4 k[kBatch], v[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const bool mine = r0 + u * kRows < span.n;
      k[u] = mine ? __ldcs(a.K + in + u * (kRows * T)) : make_uint4(0, 0, 0, 0);
      v[u] = mine ? __ldcs(a.V + in + u * (kRows * T)) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (i0 + u * kRows >= span.n) return;  // the whole block
      uint32_t ks, vs;
      const uint32_t kw = quantise(k[u], ks), vw = transpose_row<D>(quantise(v[u], vs), i);
      if (r0 + u * kRows < span.n) {
        k4[u * (kRows * T)] = kw;
        v4[u * (kRows * T)] = vw;
        if (t == 0) s4[u * (kRows * 2 * kGroups)] = ks;
        if (t == 1) s4[u * (kRows * 2 * kGroups) + kGroups] = vs;
      }
    }
  } else {
    uint32_t kw[kBatch], vw[kBatch], ks[kBatch], vs[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const bool mine = r0 + u * kRows < span.n;
      kw[u] = mine ? __ldg(k4 + u * (kRows * T)) : 0u;
      vw[u] = mine ? __ldg(v4 + u * (kRows * T)) : 0u;
      ks[u] = mine ? __ldg(s4 + u * (kRows * 2 * kGroups)) : 0u;
      vs[u] = mine ? __ldg(s4 + u * (kRows * 2 * kGroups) + kGroups) : 0u;
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (i0 + u * kRows >= span.n) return;  // the whole block
      const uint32_t vc = transpose_row<D>(vw[u], i);
      if (r0 + u * kRows < span.n) {
        a.K[in + u * (kRows * T)] = values(kw[u], ks[u]);
        a.V[in + u * (kRows * T)] = values(vc, vs[u]);
      }
    }
  }
}

// For the attention of many rows: its operands are fp16 numbers, and a key, of up to 15 significant bits beside low's
// 11, is a sum of two.
constexpr int kQueryTop = 14, kLeastQuery = -112;  // exponents of a scaled row's largest element, of the least one's
__device__ __forceinline__ float to_f16_range(float v) { return fminf(fmaxf(v, -kHalfMax), kHalfMax); }
__device__ __forceinline__ void values16(uint32_t codes, uint32_t scale, uint4& hi, uint4& rest) {
  const float step = __half2float(__ushort_as_half(static_cast<unsigned short>(scale & 0xFFFFu))),
              low = __half2float(__ushort_as_half(static_cast<unsigned short>(scale >> 16)));
  uint32_t h[4], r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = to_f16_range(fmaf(step, static_cast<float>((codes >> (8 * i)) & 15u), low)),
                b = to_f16_range(fmaf(step, static_cast<float>((codes >> (8 * i + 4)) & 15u), low));
    h[i] = pack_f16(a, b);
    const float2 back = __half22float2(*reinterpret_cast<__half2*>(&h[i]));
    r[i] = pack_f16(a - back.x, b - back.y);
  }
  hi = make_uint4(h[0], h[1], h[2], h[3]);
  rest = make_uint4(r[0], r[1], r[2], r[3]);
}

template <int D>
__global__ void __launch_bounds__(kPackThreads) unpack16_kernel(Unpack16Args a, FastDiv by_blocks, int row_blocks) {
  constexpr int T = D / 8, kRows = kPackThreads / T, kGroups = D / 32;
  grid_dependency_wait();
  grid_dependents_go();
  if (static_cast<int>(blockIdx.x) >= row_blocks) {
    // Queries: T threads to a row, which is scaled by a power of two that brings its largest element to
    // 2^14 .. 2^15.  Elements down to 2^-31 of that are exact, smaller ones off by 2^-39 of it at most.
    const size_t i = static_cast<size_t>(blockIdx.x - row_blocks) * kPackThreads + threadIdx.x;
    const bool mine = i < a.q_vecs;  // a row's threads all or none
    const uint4 v = mine ? __ldg(a.q + i) : make_uint4(0, 0, 0, 0);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t top2 = 0;  // the largest magnitude, as bf16
#pragma unroll
    for (int y = 0; y < 4; ++y) top2 = __vmaxu2(top2, w[y] & 0x7FFF7FFFu);
#pragma unroll
    for (int x = 1; x < T; x <<= 1) top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, x));
    if (!mine) return;
    const int top = static_cast<int>(max(top2 & 0xFFFFu, top2 >> 16));
    const int ex = top == 0 ? 0 : max((top >> 7) - 127, kLeastQuery);
    const float up = pow2i(kQueryTop - ex);
    uint32_t h[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) h[y] = pack_f16(bf16_lo(w[y]) * up, bf16_hi(w[y]) * up);
    a.q16[i] = make_uint4(h[0], h[1], h[2], h[3]);
    // positive and finite, whatever the scale: a factor of 0 would make a hidden key's -inf a NaN
    if (i % T == 0) a.row_sc[i / T] = fminf(fmaxf(a.sc * pow2i(ex - kQueryTop), FLT_MIN), FLT_MAX);
    return;
  }
  int e;
  const int i0 = by_blocks.mod(blockIdx.x, e) * kRows;
  int len = __ldg(a.len + e);
  if (len > a.cap) len = 0;  // the attention reports it
  if (i0 >= len) return;
  const int i = threadIdx.x % T, r = i0 + threadIdx.x / T;
  const bool mine = r < len;
  const int grp = i >> 2, t = i & 3;
  const size_t row = static_cast<size_t>(e) * a.cap + r;
  const uint32_t kw = mine ? __ldg(a.K4 + row * T + t * kGroups + grp) : 0u,
                 vw = mine ? __ldg(a.V4 + row * T + v_word<D>(i)) : 0u;
  const uint32_t ks = mine ? __ldg(a.S4 + row * (2 * kGroups) + grp) : 0u,
                 vs = mine ? __ldg(a.S4 + row * (2 * kGroups) + kGroups + grp) : 0u;
  const uint32_t vc = transpose_row<D>(vw, i);
  if (!mine) return;
  uint4 hi, rest, none;
  values16(kw, ks, hi, rest);
  a.K[row * T + i] = hi;
  a.K_rest[row * T + i] = rest;
  values16(vc, vs, hi, none);
  a.V[row * T + i] = hi;
}

template <bool PACK>
cudaError_t launch(int d, const Pack4Args& a, cudaStream_t st) {
  const int rows = kPackThreads / (d / 8) * kBatch, blocks = (a.n_rows + rows - 1) / rows;
  return launch_after(d == 128 ? pack4_kernel<128, PACK> : pack4_kernel<64, PACK>,
                      static_cast<unsigned>(a.n_inst) * blocks, kPackThreads, 0, st, a, FastDiv(blocks));
}

}  // namespace

cudaError_t launch_unpack16(int d, const Unpack16Args& a, cudaStream_t st) {
  const int rows = kPackThreads / (d / 8), blocks = (a.cap + rows - 1) / rows, row_blocks = a.n_inst * blocks;
  const unsigned q_blocks = static_cast<unsigned>((a.q_vecs + kPackThreads - 1) / kPackThreads);
  return launch_after(d == 128 ? unpack16_kernel<128> : unpack16_kernel<64>, row_blocks + q_blocks, kPackThreads, 0, st,
                      a, FastDiv(blocks), row_blocks);
}
cudaError_t launch_pack4(int d, const Pack4Args& a, cudaStream_t st) { return launch<true>(d, a, st); }
cudaError_t launch_unpack4(int d, const Pack4Args& a, cudaStream_t st) { return launch<false>(d, a, st); }

}  // namespace bkv
