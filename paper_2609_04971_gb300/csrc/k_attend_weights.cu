// Accumulated attention weights (include/bkv.h, bkv_attend): one warp per
// cached key adds the weights of the queries of its group, in row order.
#include "k_attend.cuh"

namespace bkv {
namespace {

constexpr int kThreads = 128;

template <int D>
__global__ void __launch_bounds__(kThreads) weights_kernel(Shape s, AttendArgs a, const float* lse2) {
  const int lane = threadIdx.x & 31;
  const long long key = (blockIdx.x * static_cast<long long>(kThreads) + threadIdx.x) / 32;
  const int j = static_cast<int>(key % s.cap), e = static_cast<int>(key / s.cap);
  if (e >= s.batch * s.n_kv) return;
  const int len = a.len[e];
  if (len < 0 || len > s.cap || j >= len) return;
  float k[D / 32];
#pragma unroll
  for (int x = 0; x < D / 32; ++x) k[x] = __bfloat162float(a.K[key * D + x * 32 + lane]);
  float sum = 0.f;
  for (int r = 0; r < s.G * a.n_q; ++r) {
    const long long row = static_cast<long long>(e) * s.G * a.n_q + r;
    if (j >= len - a.n_q + 1 + r % a.n_q) continue;
    float dot = 0.f;
#pragma unroll
    for (int x = 0; x < D / 32; ++x) dot = fmaf(k[x], __bfloat162float(a.q[row * D + x * 32 + lane]), dot);
#pragma unroll
    for (int x = 16; x; x >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, x);
    sum += exp2f(dot * a.sc - lse2[row]);
  }
  if (lane == 0) a.weights[key] += sum;
}

}  // namespace

cudaError_t launch_attend_weights(const Shape& s, const AttendArgs& a, cudaStream_t st) {
  const float* lse2 = reinterpret_cast<const float*>(a.ws + attend_layout(s, a.n_q, a.groups, a.pcap, true).off_lse2);
  const long long keys = 1LL * s.batch * s.n_kv * s.cap;
  const unsigned blocks = static_cast<unsigned>((keys * 32 + kThreads - 1) / kThreads);
  if (s.d == 128)
    weights_kernel<128><<<blocks, kThreads, 0, st>>>(s, a, lse2);
  else
    weights_kernel<64><<<blocks, kThreads, 0, st>>>(s, a, lse2);
  return cudaGetLastError();
}

}  // namespace bkv
