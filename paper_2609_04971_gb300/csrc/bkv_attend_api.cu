// C ABI of the attention over compacted caches and of the eviction by
// accumulated weight (declared in include/bkv.h): argument validation,
// workspace, and kernel launches on the context's stream.

#include <algorithm>
#include <cmath>
#include <new>

#include "bkv.h"
#include "bkv_ctx.h"
#include "bkv_device.cuh"
#include "bkv_internal.h"
#include "k_attend.cuh"

using bkv::aligned16;
using bkv::cuda_fail;
using bkv::fail;
using bkv::ProfScope;
using bkv::Shape;

namespace {

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Bytes of an argument; none for one that is not given.
struct Range {
  const void* p;
  size_t n;
  bool overlaps(const Range& o) const {
    const uintptr_t x = reinterpret_cast<uintptr_t>(p), y = reinterpret_cast<uintptr_t>(o.p);
    return p && o.p && x < y + o.n && y < x + n;
  }
};

// Whether an output shares a byte with an input or with another output.
template <int IN, int OUT>
bool overlap(const Range (&in)[IN], const Range (&out)[OUT]) {
  for (int i = 0; i < OUT; ++i) {
    for (const Range& r : in)
      if (out[i].overlaps(r)) return true;
    for (int j = 0; j < i; ++j)
      if (out[i].overlaps(out[j])) return true;
  }
  return false;
}

// Limits shared by the calls and the reservation: 32-bit row counts everywhere.
int check_attend_shape(bkv_ctx* c, int32_t n_q, int32_t n_groups) {
  const Shape& s = c->shape;
  if (n_q < 0) return fail(c, BKV_EINVAL, "n_q must be >= 0");
  if (n_groups < 0 || (n_groups > 0 && s.batch % n_groups != 0))
    return fail(c, BKV_EINVAL, "n_groups = %d must divide the batch (%d)", n_groups, s.batch);
  if (1LL * s.batch * s.n_kv * s.G * n_q >= (1LL << 27))
    return fail(c, BKV_EINVAL, "batch * n_q_heads * n_q must be below 2^27");
  return BKV_OK;
}

int attend(bkv_ctx* ctx, bkv::AttendArgs& a, double scale) {
  const Shape& s = ctx->shape;
  if (!a.q || !a.K || !a.V || !a.len || !a.o) return fail(ctx, BKV_EINVAL, "q, K, V, len and o must be non-NULL");
  if (!aligned16(a.q) || !aligned16(a.K) || !aligned16(a.V) || !aligned16(a.o))
    return fail(ctx, BKV_EINVAL, "q, K, V and o must be 16-byte aligned");
  if (!aligned4(a.len) || !aligned4(a.lse) || !aligned4(a.weights))
    return fail(ctx, BKV_EINVAL, "len, lse_out and weights must be 4-byte aligned");
  if (!std::isfinite(scale) || scale < 0.0) return fail(ctx, BKV_EINVAL, "scale must be finite and >= 0");
  a.sc = static_cast<float>(1.4426950408889634 * (scale == 0.0 ? 1.0 / std::sqrt(static_cast<double>(s.d)) : scale));
  if (!std::isfinite(a.sc) || a.sc < 1.17549435e-38f)
    return fail(ctx, BKV_EINVAL, "scale is out of the range of fp32");
  // Outputs are written while other blocks and the kernels that follow still read the inputs.
  const size_t rows = static_cast<size_t>(s.batch) * s.n_kv * s.G * a.n_q, lens = static_cast<size_t>(s.batch) * s.n_kv,
               kv = lens * s.cap, kvp = static_cast<size_t>(a.groups) * s.n_kv * a.pcap;
  const Range in[] = {{a.q, rows * s.d * 2},
                      {a.K, kv * s.d * 2},
                      {a.V, kv * s.d * 2},
                      {a.Kp, kvp * s.d * 2},
                      {a.Vp, kvp * s.d * 2},
                      {a.len, lens * 4},
                      {a.plen, static_cast<size_t>(a.groups) * 4}},
              out[] = {{a.o, rows * s.d * 2}, {a.lse, rows * 4}, {a.weights, kv * 4}};
  if (overlap(in, out)) return fail(ctx, BKV_EINVAL, "o, lse_out or weights overlaps an input or another output");
  const bkv::AtLayout l = bkv::attend_layout(s, a.n_q, a.groups, a.pcap, a.weights != nullptr);
  if (l.too_large) return fail(ctx, BKV_EINVAL, "row blocks times key tiles must be below 2^31");
  if (l.bytes > ctx->attend_ws_bytes)
    return fail(ctx, BKV_ESTATE, "this call needs %zu bytes of workspace, bkv_attend_reserve made %zu", l.bytes,
                ctx->attend_ws_bytes);
  a.ws = ctx->attend_ws;
  if (!ctx->attend_ws_captured) {
    cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
    // on an error the launches report what is wrong with the stream
    if (cudaStreamIsCapturing(ctx->stream, &status) != cudaSuccess) cudaGetLastError();
    ctx->attend_ws_captured = status != cudaStreamCaptureStatusNone;
  }
  a.err = ctx->err;
  cudaError_t e;
  {
    ProfScope ps(ctx, BKV_K_ATTEND);
    e = bkv::launch_attend(s, a, l, ctx->stream);
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "attend launch");
  {
    ProfScope ps(ctx, BKV_K_ATTEND_MERGE);
    e = bkv::launch_attend_merge(s, a, l, ctx->stream);
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "attend merge launch");
  if (a.weights && !l.logits) {
    ProfScope ps(ctx, BKV_K_ATTEND_WEIGHTS);
    e = bkv::launch_attend_weights(s, a, l, ctx->stream);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "attend weights launch");
  }
  return BKV_OK;
}

}  // namespace

extern "C" {

int bkv_attend_reserve(bkv_ctx* ctx, int32_t n_q, int32_t n_groups, int weights) {
  if (!ctx) return BKV_EINVAL;
  const int rc = check_attend_shape(ctx, n_q, n_groups);
  if (rc != BKV_OK) return rc;
  const size_t need = n_q == 0 ? 0 : bkv::attend_workspace(ctx->shape, n_q, n_groups, weights != 0);
  if (need <= ctx->attend_ws_bytes) return BKV_OK;
  // the new workspace exists before the old one goes, so that a failure changes nothing
  unsigned char* ws = nullptr;
  cudaError_t e = bkv::fail_this_alloc() ? cudaErrorMemoryAllocation : cudaMalloc(reinterpret_cast<void**>(&ws), need);
  if (e != cudaSuccess) {
    cudaGetLastError();
    if (e == cudaErrorMemoryAllocation) return fail(ctx, BKV_ENOMEM, "no room for %zu bytes of workspace", need);
    return cuda_fail(ctx, e, "workspace allocation");
  }
  e = cudaStreamSynchronize(ctx->stream);
  if (e != cudaSuccess) {
    cudaFree(ws);
    return cuda_fail(ctx, e, "stream synchronize");
  }
  if (ctx->attend_ws_captured) {
    auto* old = new (std::nothrow) bkv_ctx::Workspace{ctx->attend_ws, ctx->attend_ws_old};
    if (!old) {
      cudaFree(ws);
      return fail(ctx, BKV_ENOMEM, "no host memory");
    }
    ctx->attend_ws_old = old;
    ctx->attend_ws_captured = false;
  } else {
    cudaFree(ctx->attend_ws);
  }
  ctx->attend_ws = ws;
  ctx->attend_ws_bytes = need;
  return BKV_OK;
}

int bkv_attend(bkv_ctx* ctx, const void* q, int32_t n_q, const void* K, const void* V, const int32_t* len, double scale,
               void* o, float* lse_out, float* weights) {
  if (!ctx) return BKV_EINVAL;
  const int rc = check_attend_shape(ctx, n_q, 0);
  if (rc != BKV_OK || n_q == 0) return rc;
  bkv::AttendArgs a;
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.K = static_cast<const __nv_bfloat16*>(K);
  a.V = static_cast<const __nv_bfloat16*>(V);
  a.len = len;
  a.n_q = n_q;
  a.o = static_cast<__nv_bfloat16*>(o);
  a.lse = lse_out;
  a.weights = weights;
  return attend(ctx, a, scale);
}

int bkv_attend_shared(bkv_ctx* ctx, const void* q, int32_t n_q, const void* Kp, const void* Vp, const int32_t* prefix_len,
                      int32_t n_groups, int32_t prefix_capacity, const void* K, const void* V, const int32_t* len,
                      double scale, void* o, float* lse_out, float* weights) {
  if (!ctx) return BKV_EINVAL;
  const Shape& s = ctx->shape;
  if (n_groups < 1) return fail(ctx, BKV_EINVAL, "n_groups must be >= 1");
  const int rc = check_attend_shape(ctx, n_q, n_groups);
  if (rc != BKV_OK) return rc;
  if (prefix_capacity < 1 || 1LL * n_groups * s.n_kv * prefix_capacity >= (1LL << 31) ||
      prefix_capacity >= (1 << 30))
    return fail(ctx, BKV_EINVAL, "prefix_capacity must be >= 1 and n_groups * n_kv_heads * prefix_capacity below 2^31");
  if (n_q == 0) return BKV_OK;
  if (!Kp || !Vp || !prefix_len || !aligned16(Kp) || !aligned16(Vp) || !aligned4(prefix_len))
    return fail(ctx, BKV_EINVAL, "Kp and Vp (16-byte aligned) and prefix_len are required");
  bkv::AttendArgs a;
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.K = static_cast<const __nv_bfloat16*>(K);
  a.V = static_cast<const __nv_bfloat16*>(V);
  a.Kp = static_cast<const __nv_bfloat16*>(Kp);
  a.Vp = static_cast<const __nv_bfloat16*>(Vp);
  a.len = len;
  a.plen = prefix_len;
  a.n_q = n_q;
  a.groups = n_groups;
  a.pcap = prefix_capacity;
  a.o = static_cast<__nv_bfloat16*>(o);
  a.lse = lse_out;
  a.weights = weights;
  return attend(ctx, a, scale);
}

int bkv_evict(bkv_ctx* ctx, const void* K, const void* V, const float* weights, const int32_t* L, int32_t budget,
              void* K_out, void* V_out, float* weights_out, int32_t capacity_out, int32_t* kept_idx_out,
              int32_t* len_out) {
  if (!ctx) return BKV_EINVAL;
  const Shape& s = ctx->shape;
  if (!K || !V || !weights || !L || !K_out || !V_out || !weights_out || !kept_idx_out)
    return fail(ctx, BKV_EINVAL, "K, V, weights, L, their outputs and kept_idx_out must be non-NULL");
  if (!aligned16(K) || !aligned16(V) || !aligned16(K_out) || !aligned16(V_out))
    return fail(ctx, BKV_EINVAL, "K, V, K_out and V_out must be 16-byte aligned");
  if (!aligned4(weights) || !aligned4(weights_out) || !aligned4(L) || !aligned4(kept_idx_out) || !aligned4(len_out))
    return fail(ctx, BKV_EINVAL, "weights, L and the index outputs must be 4-byte aligned");
  if (budget < 1 || budget < s.n_prefix + s.W)
    return fail(ctx, BKV_EINVAL, "budget = %d must be >= max(1, n_prefix + window = %d)", budget, s.n_prefix + s.W);
  if (1LL * s.n_inst * budget >= (1LL << 31)) return fail(ctx, BKV_EINVAL, "budget too large");
  if (capacity_out < std::min(budget, s.cap))
    return fail(ctx, BKV_EINVAL, "capacity_out = %d is below min(budget, capacity) = %d", capacity_out,
                std::min(budget, s.cap));
  if (1LL * s.n_inst * capacity_out >= (1LL << 31)) return fail(ctx, BKV_EINVAL, "capacity_out too large");
  const bool in_place = K_out == K && V_out == V && weights_out == weights;
  const size_t rows = static_cast<size_t>(s.n_inst) * s.cap, rows_out = static_cast<size_t>(s.n_inst) * capacity_out;
  const size_t kv = rows * s.d * 2, kv_out = rows_out * s.d * 2, lens = sizeof(int32_t) * s.n_inst;
  if (in_place && capacity_out != s.cap)
    return fail(ctx, BKV_EINVAL, "in place, capacity_out = %d must be the capacity (%d)", capacity_out, s.cap);
  // The rows are moved by kept_idx_out, so a row number must not be written over either.
  const Range in[] = {{in_place ? nullptr : K, kv},
                      {in_place ? nullptr : V, kv},
                      {in_place ? nullptr : weights, rows * 4},
                      {len_out == L ? nullptr : L, lens}},
              out[] = {{K_out, kv_out},
                       {V_out, kv_out},
                       {weights_out, rows_out * 4},
                       {kept_idx_out, sizeof(int32_t) * s.n_inst * budget},
                       {len_out, lens}};
  if (overlap(in, out))
    return fail(ctx, BKV_EINVAL, "an output overlaps an input or another output (K, V and weights may be their own "
                "outputs, all three, and L may be len_out)");
  bkv::EvictArgs a;
  a.K = static_cast<const __nv_bfloat16*>(K);
  a.V = static_cast<const __nv_bfloat16*>(V);
  a.weights = weights;
  a.L = L;
  a.budget = budget;
  a.cap_out = capacity_out;
  a.K_out = static_cast<__nv_bfloat16*>(K_out);
  a.V_out = static_cast<__nv_bfloat16*>(V_out);
  a.weights_out = weights_out;
  a.kept = kept_idx_out;
  a.len_out = len_out;
  a.plan = reinterpret_cast<int2*>(ctx->valid);  // scratch of a compress, 16 bytes per instance
  a.err = ctx->err;
  ProfScope ps(ctx, BKV_K_EVICT);
  const cudaError_t e = bkv::launch_evict(s, a, ctx->stream);
  return e == cudaSuccess ? BKV_OK : cuda_fail(ctx, e, "evict launch");
}

}  // extern "C"
