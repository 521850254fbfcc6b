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
// products need of eight of their rows, which eight threads hold: eight shuffles.
//
// Bound by HBM: 4 d bytes of bf16 and 1.25 d bytes of codes and scales a row.
#include <cuda_fp16.h>

#include "bkv_device.cuh"
#include "bkv_internal.h"
#include "k_attend.cuh"
#include "k_launch.cuh"

namespace bkv {
namespace {

constexpr int kPackThreads = 256;
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

// The code of x where the quotient f is within 1e-4 of a tie: by the exact sign of x - low - (n + 1/2) step.
__device__ __noinline__ int code_near_tie(float x, float low, float step, float f) {
  const int n = min(14, max(0, static_cast<int>(floorf(f))));
  const float edge = (static_cast<float>(n) + 0.5f) * step;  // at most 16 significant bits
  const float s = x - low, bb = s - x;                        // s + err = x - low exactly
  const float err = (x - (s - bb)) + (-low - bb);
  const float t = (s - edge) + err;
  return t > 0.f || (t == 0.f && (n & 1)) ? n + 1 : n;
}

// Codes of eight elements of a group that four neighbouring threads share, as a word, and the group's (step, low).
__device__ __forceinline__ uint32_t quantise(const uint4& raw, uint32_t& scale) {
  float x[8] = {bf16_lo(raw.x), bf16_hi(raw.x), bf16_lo(raw.y), bf16_hi(raw.y),
                bf16_lo(raw.z), bf16_hi(raw.z), bf16_lo(raw.w), bf16_hi(raw.w)};
  float lo = x[0], hi = x[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    lo = fminf(lo, x[i]);
    hi = fmaxf(hi, x[i]);
  }
#pragma unroll
  for (int o = 1; o <= 2; o <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  const __half low16 = __float2half_rn(fminf(fmaxf(lo, -kHalfMax), kHalfMax));
  const float low = __half2float(low16);
  const float range = fmaxf(0.f, __fsub_rd(hi, low));
  float q = fminf(kHalfMax, __fdiv_rz(range, 15.f));
  if (range > 0.f && (fmaf(-15.f, q, range) != 0.f || __fsub_ru(hi, low) != range))
    q = __uint_as_float(__float_as_uint(q) | 1u);
  const __half step16 = __float2half_rn(q);
  const float step = __half2float(step16), inv = step > 0.f ? 1.f / step : 0.f;
  uint32_t word = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float f = fminf(15.f, fmaxf(0.f, (x[i] - low) * inv)), r = rintf(f);
    int n = static_cast<int>(r);
    if (fabsf(fabsf(f - r) - 0.5f) < 1e-4f) n = code_near_tie(x[i], low, step, f);
    word |= static_cast<uint32_t>(n) << (4 * i);
  }
  scale = static_cast<uint32_t>(__half_as_ushort(step16)) | (static_cast<uint32_t>(__half_as_ushort(low16)) << 16);
  return word;
}

// Word i of a row of V from every thread's eight consecutive codes, and back (each is its own kind of transpose
// among the D / 8 threads of the row); `row0` is the row's first lane.
template <int D>
__device__ __forceinline__ uint32_t words_of_v(uint32_t codes, int i, int row0) {
  constexpr int W = D / 8;
  uint32_t word = 0;
#pragma unroll
  for (int x = 0; x < 8; ++x) {  // element i + x W
    const uint32_t c = __shfl_sync(0xffffffffu, codes, row0 + (x * W + i) / 8);
    word |= ((c >> (4 * (i & 7))) & 15u) << (4 * x);  // W is a multiple of 8
  }
  return word;
}
template <int D>
__device__ __forceinline__ uint32_t codes_of_v(uint32_t word, int i, int row0) {
  constexpr int W = D / 8;
  uint32_t codes = 0;
#pragma unroll
  for (int r = 0; r < 8; ++r) {  // element 8 i + r
    const uint32_t w = __shfl_sync(0xffffffffu, word, row0 + (8 * i) % W + r);
    codes |= ((w >> (4 * ((8 * i) / W))) & 15u) << (4 * r);
  }
  return codes;
}

__device__ __forceinline__ uint4 values(uint32_t codes, uint32_t scale) {
  const float step = __half2float(__ushort_as_half(static_cast<unsigned short>(scale & 0xFFFFu))),
              low = __half2float(__ushort_as_half(static_cast<unsigned short>(scale >> 16)));
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = fmaf(step, static_cast<float>((codes >> (4 * i)) & 15u), low);
  return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}

template <int D, bool PACK>
__global__ void __launch_bounds__(kPackThreads) pack4_kernel(Pack4Args a, FastDiv by_blocks) {
  constexpr int T = D / 8, kRows = kPackThreads / T;  // threads per row, rows per block
  constexpr int kGroups = D / 32;
  grid_dependency_wait();
  grid_dependents_go();
  int e;
  const int i0 = by_blocks.mod(blockIdx.x, e) * kRows;
  const Span4 span = span4(a, e, i0 == 0 && threadIdx.x == 0);
  if (i0 >= span.n) return;
  const int i = threadIdx.x % T, r = i0 + threadIdx.x / T, row0 = (threadIdx.x & 31) / T * T;
  const bool mine = r < span.n;
  const int grp = i >> 2, t = i & 3;
  const size_t in = (static_cast<size_t>(e) * a.n_rows + r) * T + i;
  const size_t row = static_cast<size_t>(e) * a.cap + span.first + r;
  uint32_t* k4 = a.K4 + row * T + t * kGroups + grp;
  uint32_t* v4 = a.V4 + row * T + i;
  uint32_t* s4 = a.S4 + row * (2 * kGroups) + grp;
  if (PACK) {
    const uint4 zero = make_uint4(0, 0, 0, 0);
    const uint4 k = mine ? __ldcs(a.K + in) : zero, v = mine ? __ldcs(a.V + in) : zero;
    uint32_t ks, vs;
    const uint32_t kw = quantise(k, ks), vw = words_of_v<D>(quantise(v, vs), i, row0);
    if (!mine) return;
    *k4 = kw;
    *v4 = vw;
    if (t == 0) s4[0] = ks;
    if (t == 1) s4[kGroups] = vs;
  } else {
    const uint32_t kw = mine ? __ldg(k4) : 0u, vw = mine ? __ldg(v4) : 0u;
    const uint32_t ks = mine ? __ldg(s4) : 0u, vs = mine ? __ldg(s4 + kGroups) : 0u;
    const uint32_t vc = codes_of_v<D>(vw, i, row0);
    if (!mine) return;
    a.K[in] = values(kw, ks);
    a.V[in] = values(vc, vs);
  }
}

// For the attention of many rows: its operands are fp16 numbers, and a key, of up to 15 significant bits beside low's
// 11, is a sum of two.
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
  if (static_cast<int>(blockIdx.x) >= row_blocks) {  // queries
    const size_t i = static_cast<size_t>(blockIdx.x - row_blocks) * kPackThreads + threadIdx.x;
    if (i >= a.q_vecs) return;
    const uint4 v = __ldg(a.q + i);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t h[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) h[y] = pack_f16(to_f16_range(bf16_lo(w[y])), to_f16_range(bf16_hi(w[y])));
    a.q16[i] = make_uint4(h[0], h[1], h[2], h[3]);
    return;
  }
  int e;
  const int i0 = by_blocks.mod(blockIdx.x, e) * kRows;
  int len = __ldg(a.len + e);
  if (len > a.cap) len = 0;  // the attention reports it
  if (i0 >= len) return;
  const int i = threadIdx.x % T, r = i0 + threadIdx.x / T, row0 = (threadIdx.x & 31) / T * T;
  const bool mine = r < len;
  const int grp = i >> 2, t = i & 3;
  const size_t row = static_cast<size_t>(e) * a.cap + r;
  const uint32_t kw = mine ? __ldg(a.K4 + row * T + t * kGroups + grp) : 0u, vw = mine ? __ldg(a.V4 + row * T + i) : 0u;
  const uint32_t ks = mine ? __ldg(a.S4 + row * (2 * kGroups) + grp) : 0u,
                 vs = mine ? __ldg(a.S4 + row * (2 * kGroups) + kGroups + grp) : 0u;
  const uint32_t vc = codes_of_v<D>(vw, i, row0);
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
  const int rows = kPackThreads / (d / 8), blocks = (a.n_rows + rows - 1) / rows;
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
