// Attention of the newest queries over a sequence's cache and, with a shared
// prefix, over the prefix of its group (include/bkv.h, bkv_attend).
//
// One warp per output row (query head, query): lanes split head_dim, keys one
// after another with a running maximum and sum in base 2.
#include "bkv_device.cuh"
#include "bkv_internal.h"

namespace bkv {
namespace {

constexpr int kThreads = 128;

// A cache length from device memory: out of range counts as 0 and is reported.
__device__ __forceinline__ int checked_len(int n, int cap, int* err) {
  if (n >= 0 && n <= cap) return n;
  record_error(err, kDevBadLength);
  return 0;
}

template <int D>
struct Row {
  float q[D / 32], o[D / 32], m = -INFINITY, l = 0.f;
  __device__ void keys(const __nv_bfloat16* K, const __nv_bfloat16* V, int n, float sc, int lane) {
    for (int j = 0; j < n; ++j) {
      float dot = 0.f;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) dot = fmaf(q[i], __bfloat162float(K[static_cast<size_t>(j) * D + i * 32 + lane]), dot);
#pragma unroll
      for (int x = 16; x; x >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, x);
      const float y = dot * sc, top = fmaxf(m, y);
      const float scale = exp2f(m - top), p = exp2f(y - top);
      m = top;
      l = l * scale + p;
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
        o[i] = o[i] * scale + p * __bfloat162float(V[static_cast<size_t>(j) * D + i * 32 + lane]);
    }
  }
};

template <int D>
__global__ void __launch_bounds__(kThreads) attend_kernel(Shape s, AttendArgs a, float* lse2) {
  const int lane = threadIdx.x & 31;
  const long long row = (blockIdx.x * static_cast<long long>(kThreads) + threadIdx.x) / 32;
  const int hq = s.n_kv * s.G;
  if (row >= 1LL * s.batch * hq * a.n_q) return;
  const int i = static_cast<int>(row % a.n_q), h = static_cast<int>(row / a.n_q % hq), b = static_cast<int>(row / a.n_q / hq);
  const int kv = h / s.G;
  Row<D> r;
#pragma unroll
  for (int x = 0; x < D / 32; ++x) {
    r.q[x] = __bfloat162float(a.q[row * D + x * 32 + lane]);
    r.o[x] = 0.f;
  }
  if (a.groups) {
    const int g = b / (s.batch / a.groups);
    const size_t at = (static_cast<size_t>(g) * s.n_kv + kv) * a.pcap * D;
    r.keys(a.Kp + at, a.Vp + at, checked_len(a.plen[g], a.pcap, a.err), a.sc, lane);
  }
  const int e = b * s.n_kv + kv;
  const int n = checked_len(a.len[e], s.cap, a.err) - a.n_q + 1 + i;
  r.keys(a.K + static_cast<size_t>(e) * s.cap * D, a.V + static_cast<size_t>(e) * s.cap * D, n, a.sc, lane);
  const float y = r.l > 0.f ? r.m + log2f(r.l) : -INFINITY;
#pragma unroll
  for (int x = 0; x < D / 32; ++x)
    a.o[row * D + x * 32 + lane] = __float2bfloat16(r.l > 0.f ? r.o[x] / r.l : 0.f);
  if (lane == 0) {
    lse2[row] = y;
    if (a.lse) a.lse[row] = y * 0.69314718055994531f;
  }
}

}  // namespace

size_t attend_workspace(const Shape& s, int n_q, int, bool) {
  return sizeof(float) * static_cast<size_t>(s.batch) * s.n_kv * s.G * n_q;
}

cudaError_t launch_attend(const Shape& s, const AttendArgs& a, cudaStream_t st) {
  const long long rows = 1LL * s.batch * s.n_kv * s.G * a.n_q;
  const unsigned blocks = static_cast<unsigned>((rows * 32 + kThreads - 1) / kThreads);
  if (s.d == 128)
    attend_kernel<128><<<blocks, kThreads, 0, st>>>(s, a, reinterpret_cast<float*>(a.ws));
  else
    attend_kernel<64><<<blocks, kThreads, 0, st>>>(s, a, reinterpret_cast<float*>(a.ws));
  return cudaGetLastError();
}

}  // namespace bkv
