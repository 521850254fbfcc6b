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

// Bytes of a row of K (and of V), and of the scales of a row of a 4-bit cache.
size_t row_bytes(const Shape& s, bool four) { return four ? s.d / 2 : 2 * static_cast<size_t>(s.d); }
size_t scale_bytes(const Shape& s, bool four) { return four ? s.d / 4 : 0; }

// The scale of the logits, to base 2.
int check_scale(bkv_ctx* ctx, double scale, float& sc) {
  if (!std::isfinite(scale) || scale < 0.0) return fail(ctx, BKV_EINVAL, "scale must be finite and >= 0");
  const double by_dim = 1.0 / std::sqrt(static_cast<double>(ctx->shape.d));
  sc = static_cast<float>(1.4426950408889634 * (scale == 0.0 ? by_dim : scale));
  if (!std::isfinite(sc) || sc < 1.17549435e-38f)
    return fail(ctx, BKV_EINVAL, "scale is out of the range of fp32");
  return BKV_OK;
}

// The workspace of a call laid out as `l`.
int take_workspace(bkv_ctx* ctx, const bkv::AtLayout& l, const char* reserve, unsigned char*& ws) {
  if (l.too_large) return fail(ctx, BKV_EINVAL, "row blocks times key tiles must be below 2^31");
  if (l.bytes > ctx->attend_ws_bytes)
    return fail(ctx, BKV_ESTATE, "this call needs %zu bytes of workspace, %s made %zu", l.bytes, reserve,
                ctx->attend_ws_bytes);
  ws = ctx->attend_ws;
  if (!ctx->attend_ws_captured) {
    cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
    // on an error the launches report what is wrong with the stream
    if (cudaStreamIsCapturing(ctx->stream, &status) != cudaSuccess) cudaGetLastError();
    ctx->attend_ws_captured = status != cudaStreamCaptureStatusNone;
  }
  return BKV_OK;
}

int launch_merge(bkv_ctx* ctx, const bkv::AttendArgs& a, const bkv::AtLayout& l) {
  ProfScope ps(ctx, BKV_K_ATTEND_MERGE);
  const cudaError_t e = bkv::launch_attend_merge(ctx->shape, a, l, ctx->stream);
  return e == cudaSuccess ? BKV_OK : cuda_fail(ctx, e, "attend merge launch");
}

int launch_attend_kernels(bkv_ctx* ctx, const bkv::AttendArgs& a, const bkv::AtLayout& l) {
  const Shape& s = ctx->shape;
  cudaError_t e;
  {
    ProfScope ps(ctx, BKV_K_ATTEND);
    e = bkv::launch_attend(s, a, l, ctx->stream);
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "attend launch");
  const int rc = launch_merge(ctx, a, l);
  if (rc != BKV_OK) return rc;
  if (a.weights && !l.logits) {
    ProfScope ps(ctx, BKV_K_ATTEND_WEIGHTS);
    e = bkv::launch_attend_weights(s, a, l, ctx->stream);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "attend weights launch");
  }
  return BKV_OK;
}

int attend(bkv_ctx* ctx, bkv::AttendArgs& a, double scale) {
  const Shape& s = ctx->shape;
  if (!a.q || !a.K || !a.V || !a.len || !a.o) return fail(ctx, BKV_EINVAL, "q, K, V, len and o must be non-NULL");
  if (!aligned16(a.q) || !aligned16(a.K) || !aligned16(a.V) || !aligned16(a.o))
    return fail(ctx, BKV_EINVAL, "q, K, V and o must be 16-byte aligned");
  if (!aligned4(a.len) || !aligned4(a.lse) || !aligned4(a.weights))
    return fail(ctx, BKV_EINVAL, "len, lse_out and weights must be 4-byte aligned");
  int rc = check_scale(ctx, scale, a.sc);
  if (rc != BKV_OK) return rc;
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
  rc = take_workspace(ctx, l, "bkv_attend_reserve", a.ws);
  if (rc != BKV_OK) return rc;
  a.err = ctx->err;
  return launch_attend_kernels(ctx, a, l);
}

// Grows the attention workspace to `need` bytes.
int reserve(bkv_ctx* ctx, size_t need) {
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

// Rows of K and V into (pack) or out of one layer's 4-bit caches.
int pack4(bkv_ctx* ctx, bool pack, bkv::Pack4Args& a) {
  const Shape& s = ctx->shape;
  if (a.n_rows < 0) return fail(ctx, BKV_EINVAL, "n_rows must be >= 0");
  a.n_inst = s.batch * s.n_kv;
  a.cap = s.cap;
  if (1LL * a.n_inst * a.n_rows >= (1LL << 31))
    return fail(ctx, BKV_EINVAL, "batch * n_kv_heads * n_rows must be below 2^31");
  if (a.n_rows == 0) return BKV_OK;
  if (!a.K || !a.V || !a.K4 || !a.V4 || !a.S4 || !a.len)
    return fail(ctx, BKV_EINVAL, "K, V, K4, V4, S4 and len must be non-NULL");
  if (!aligned16(a.K) || !aligned16(a.V) || !aligned16(a.K4) || !aligned16(a.V4) || !aligned16(a.S4))
    return fail(ctx, BKV_EINVAL, "K, V, K4, V4 and S4 must be 16-byte aligned");
  if (!aligned4(a.first) || !aligned4(a.len)) return fail(ctx, BKV_EINVAL, "first and len must be 4-byte aligned");
  const size_t lens = static_cast<size_t>(a.n_inst) * 4, rows = static_cast<size_t>(a.n_inst) * a.n_rows * s.d * 2,
               caches = static_cast<size_t>(a.n_inst) * s.cap;
  const Range K{a.K, rows}, V{a.V, rows}, K4{a.K4, caches * row_bytes(s, true)}, V4{a.V4, caches * row_bytes(s, true)},
      S4{a.S4, caches * scale_bytes(s, true)}, first{a.first, lens}, len{a.len, lens}, none{nullptr, 0};
  bool bad;
  if (pack) {
    const Range in[] = {K, V, first, len}, out[] = {K4, V4, S4};
    bad = overlap(in, out);
  } else {
    const Range in[] = {K4, V4, S4, first, len}, out[] = {K, V, none};
    bad = overlap(in, out);
  }
  if (bad) return fail(ctx, BKV_EINVAL, "an output overlaps an input or another output");
  a.err = ctx->err;
  ProfScope ps(ctx, pack ? BKV_K_PACK4 : BKV_K_UNPACK4);
  const cudaError_t e = pack ? bkv::launch_pack4(s.d, a, ctx->stream) : bkv::launch_unpack4(s.d, a, ctx->stream);
  return e == cudaSuccess ? BKV_OK : cuda_fail(ctx, e, pack ? "pack launch" : "unpack launch");
}

int attend4(bkv_ctx* ctx, bkv::Attend4Args& a, double scale) {
  const Shape& s = ctx->shape;
  if (!a.q || !a.K4 || !a.V4 || !a.S4 || !a.len || !a.o)
    return fail(ctx, BKV_EINVAL, "q, K4, V4, S4, len and o must be non-NULL");
  if (!aligned16(a.q) || !aligned16(a.K4) || !aligned16(a.V4) || !aligned16(a.S4) || !aligned16(a.o))
    return fail(ctx, BKV_EINVAL, "q, K4, V4, S4 and o must be 16-byte aligned");
  if (!aligned4(a.len) || !aligned4(a.lse) || !aligned4(a.weights))
    return fail(ctx, BKV_EINVAL, "len, lse_out and weights must be 4-byte aligned");
  int rc = check_scale(ctx, scale, a.sc);
  if (rc != BKV_OK) return rc;
  const size_t rows = static_cast<size_t>(s.batch) * s.n_kv * s.G * a.n_q, lens = static_cast<size_t>(s.batch) * s.n_kv,
               kv = lens * s.cap;
  const Range in[] = {{a.q, rows * s.d * 2},
                      {a.K4, kv * row_bytes(s, true)},
                      {a.V4, kv * row_bytes(s, true)},
                      {a.S4, kv * scale_bytes(s, true)},
                      {a.len, lens * 4}},
              out[] = {{a.o, rows * s.d * 2}, {a.lse, rows * 4}, {a.weights, kv * 4}};
  if (overlap(in, out)) return fail(ctx, BKV_EINVAL, "o, lse_out or weights overlaps an input or another output");
  const bkv::AtLayout l = bkv::attend4_layout(s, a.n_q, a.weights != nullptr);
  rc = take_workspace(ctx, l, "bkv_attend4_reserve", a.ws);
  if (rc != BKV_OK) return rc;
  a.err = ctx->err;
  bkv::AttendArgs b;
  b.q = a.q;
  b.len = a.len;
  b.n_q = a.n_q;
  b.sc = a.sc;
  b.o = a.o;
  b.lse = a.lse;
  b.weights = a.weights;
  b.ws = a.ws;
  b.err = a.err;
  if (l.unpacked) {
    bkv::Unpack16Args u;
    u.K = reinterpret_cast<uint4*>(a.ws + l.off_k);
    u.K_rest = reinterpret_cast<uint4*>(a.ws + l.off_k_rest);
    u.V = reinterpret_cast<uint4*>(a.ws + l.off_v);
    u.K4 = a.K4;
    u.V4 = a.V4;
    u.S4 = a.S4;
    u.len = a.len;
    u.n_inst = s.batch * s.n_kv;
    u.cap = s.cap;
    u.q = reinterpret_cast<const uint4*>(a.q);
    u.q16 = reinterpret_cast<uint4*>(a.ws + l.off_q);
    u.q_vecs = rows * s.d / 8;
    u.sc = a.sc;
    u.row_sc = reinterpret_cast<float*>(a.ws + l.off_row_sc);
    b.q = reinterpret_cast<const __nv_bfloat16*>(u.q16);
    b.K = reinterpret_cast<const __nv_bfloat16*>(u.K);
    b.K_rest = u.K_rest;
    b.row_sc = u.row_sc;
    b.V = reinterpret_cast<const __nv_bfloat16*>(u.V);
    cudaError_t e;
    {
      ProfScope ps(ctx, BKV_K_UNPACK4);
      e = bkv::launch_unpack16(s.d, u, ctx->stream);
    }
    if (e != cudaSuccess) return cuda_fail(ctx, e, "unpack launch");
    return launch_attend_kernels(ctx, b, l);
  }
  cudaError_t e;
  {
    ProfScope ps(ctx, BKV_K_ATTEND4);
    e = bkv::launch_attend4(s, a, l, ctx->stream);
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "attend4 launch");
  return launch_merge(ctx, b, l);
}

int evict(bkv_ctx* ctx, bkv::EvictArgs& a) {
  const Shape& s = ctx->shape;
  if (!a.K || !a.V || !a.weights || !a.L || !a.K_out || !a.V_out || !a.weights_out || !a.kept ||
      (a.four && (!a.S || !a.S_out)))
    return fail(ctx, BKV_EINVAL, "the caches, weights, L, their outputs and kept_idx_out must be non-NULL");
  if (!aligned16(a.K) || !aligned16(a.V) || !aligned16(a.S) || !aligned16(a.K_out) || !aligned16(a.V_out) ||
      !aligned16(a.S_out))
    return fail(ctx, BKV_EINVAL, "the caches and their outputs must be 16-byte aligned");
  if (!aligned4(a.weights) || !aligned4(a.weights_out) || !aligned4(a.L) || !aligned4(a.kept) || !aligned4(a.len_out))
    return fail(ctx, BKV_EINVAL, "weights, L and the index outputs must be 4-byte aligned");
  if (a.budget < 1 || a.budget < s.n_prefix + s.W)
    return fail(ctx, BKV_EINVAL, "budget = %d must be >= max(1, n_prefix + window = %d)", a.budget, s.n_prefix + s.W);
  if (1LL * s.n_inst * a.budget >= (1LL << 31)) return fail(ctx, BKV_EINVAL, "budget too large");
  if (a.cap_out < std::min(a.budget, s.cap))
    return fail(ctx, BKV_EINVAL, "capacity_out = %d is below min(budget, capacity) = %d", a.cap_out,
                std::min(a.budget, s.cap));
  if (1LL * s.n_inst * a.cap_out >= (1LL << 31)) return fail(ctx, BKV_EINVAL, "capacity_out too large");
  const bool in_place = a.K_out == a.K && a.V_out == a.V && a.S_out == a.S && a.weights_out == a.weights;
  const size_t rows = static_cast<size_t>(s.n_inst) * s.cap, rows_out = static_cast<size_t>(s.n_inst) * a.cap_out;
  const size_t kv = row_bytes(s, a.four), sc = scale_bytes(s, a.four), lens = sizeof(int32_t) * s.n_inst;
  if (in_place && a.cap_out != s.cap)
    return fail(ctx, BKV_EINVAL, "in place, capacity_out = %d must be the capacity (%d)", a.cap_out, s.cap);
  // The rows are moved by kept_idx_out, so a row number must not be written over either.
  const Range in[] = {{in_place ? nullptr : a.K, rows * kv},
                      {in_place ? nullptr : a.V, rows * kv},
                      {in_place ? nullptr : a.S, rows * sc},
                      {in_place ? nullptr : a.weights, rows * 4},
                      {a.len_out == a.L ? nullptr : a.L, lens}},
              out[] = {{a.K_out, rows_out * kv},
                       {a.V_out, rows_out * kv},
                       {a.S_out, rows_out * sc},
                       {a.weights_out, rows_out * 4},
                       {a.kept, sizeof(int32_t) * s.n_inst * a.budget},
                       {a.len_out, lens}};
  if (overlap(in, out))
    return fail(ctx, BKV_EINVAL, "an output overlaps an input or another output (the caches and weights may be their "
                "own outputs, all of them, and L may be len_out)");
  a.plan = reinterpret_cast<int2*>(ctx->valid);  // scratch of a compress, 16 bytes per instance
  a.err = ctx->err;
  ProfScope ps(ctx, BKV_K_EVICT);
  const cudaError_t e = bkv::launch_evict(s, a, ctx->stream);
  return e == cudaSuccess ? BKV_OK : cuda_fail(ctx, e, "evict launch");
}

}  // namespace

extern "C" {

int bkv_attend_reserve(bkv_ctx* ctx, int32_t n_q, int32_t n_groups, int weights) {
  if (!ctx) return BKV_EINVAL;
  const int rc = check_attend_shape(ctx, n_q, n_groups);
  if (rc != BKV_OK) return rc;
  return reserve(ctx, n_q == 0 ? 0 : bkv::attend_workspace(ctx->shape, n_q, n_groups, weights != 0));
}

int bkv_attend4_reserve(bkv_ctx* ctx, int32_t n_q, int weights) {
  if (!ctx) return BKV_EINVAL;
  const int rc = check_attend_shape(ctx, n_q, 0);
  if (rc != BKV_OK) return rc;
  return reserve(ctx, n_q == 0 ? 0 : bkv::attend4_workspace(ctx->shape, n_q, weights != 0));
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

int bkv_attend_window(bkv_ctx* ctx, const void* q, int32_t n_q, const void* K, const void* V, const int32_t* len,
                      int32_t window, int32_t n_sink, double scale, void* o, float* lse_out) {
  if (!ctx) return BKV_EINVAL;
  const int rc = check_attend_shape(ctx, n_q, 0);
  if (rc != BKV_OK) return rc;
  if (window < 1 || n_sink < 0) return fail(ctx, BKV_EINVAL, "window must be >= 1 and n_sink >= 0");
  if (n_q == 0) return BKV_OK;
  bkv::AttendArgs a;
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.K = static_cast<const __nv_bfloat16*>(K);
  a.V = static_cast<const __nv_bfloat16*>(V);
  a.len = len;
  a.n_q = n_q;
  a.window = std::min(window, ctx->shape.cap);  // no row sees more than the capacity
  a.n_sink = std::min(n_sink, ctx->shape.cap);
  a.o = static_cast<__nv_bfloat16*>(o);
  a.lse = lse_out;
  return attend(ctx, a, scale);
}

int bkv_pack4(bkv_ctx* ctx, const void* K, const void* V, int32_t n_rows, const int32_t* first, const int32_t* len,
              void* K4, void* V4, void* S4) {
  if (!ctx) return BKV_EINVAL;
  bkv::Pack4Args a;
  a.K = static_cast<uint4*>(const_cast<void*>(K));
  a.V = static_cast<uint4*>(const_cast<void*>(V));
  a.K4 = static_cast<uint32_t*>(K4);
  a.V4 = static_cast<uint32_t*>(V4);
  a.S4 = static_cast<uint32_t*>(S4);
  a.first = first;
  a.len = len;
  a.n_rows = n_rows;
  return pack4(ctx, true, a);
}

int bkv_unpack4(bkv_ctx* ctx, const void* K4, const void* V4, const void* S4, int32_t n_rows, const int32_t* first,
                const int32_t* len, void* K, void* V) {
  if (!ctx) return BKV_EINVAL;
  bkv::Pack4Args a;
  a.K = static_cast<uint4*>(K);
  a.V = static_cast<uint4*>(V);
  a.K4 = static_cast<uint32_t*>(const_cast<void*>(K4));
  a.V4 = static_cast<uint32_t*>(const_cast<void*>(V4));
  a.S4 = static_cast<uint32_t*>(const_cast<void*>(S4));
  a.first = first;
  a.len = len;
  a.n_rows = n_rows;
  return pack4(ctx, false, a);
}

int bkv_attend4(bkv_ctx* ctx, const void* q, int32_t n_q, const void* K4, const void* V4, const void* S4,
                const int32_t* len, double scale, void* o, float* lse_out, float* weights) {
  if (!ctx) return BKV_EINVAL;
  const int rc = check_attend_shape(ctx, n_q, 0);
  if (rc != BKV_OK || n_q == 0) return rc;
  bkv::Attend4Args a;
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.K4 = static_cast<const uint32_t*>(K4);
  a.V4 = static_cast<const uint32_t*>(V4);
  a.S4 = static_cast<const uint32_t*>(S4);
  a.len = len;
  a.n_q = n_q;
  a.o = static_cast<__nv_bfloat16*>(o);
  a.lse = lse_out;
  a.weights = weights;
  return attend4(ctx, a, scale);
}

int bkv_evict4(bkv_ctx* ctx, const void* K4, const void* V4, const void* S4, const float* weights, const int32_t* L,
               int32_t budget, void* K4_out, void* V4_out, void* S4_out, float* weights_out, int32_t capacity_out,
               int32_t* kept_idx_out, int32_t* len_out) {
  if (!ctx) return BKV_EINVAL;
  bkv::EvictArgs a;
  a.four = true;
  a.K = K4;
  a.V = V4;
  a.S = S4;
  a.weights = weights;
  a.L = L;
  a.budget = budget;
  a.cap_out = capacity_out;
  a.K_out = K4_out;
  a.V_out = V4_out;
  a.S_out = S4_out;
  a.weights_out = weights_out;
  a.kept = kept_idx_out;
  a.len_out = len_out;
  return evict(ctx, a);
}

int bkv_evict(bkv_ctx* ctx, const void* K, const void* V, const float* weights, const int32_t* L, int32_t budget,
              void* K_out, void* V_out, float* weights_out, int32_t capacity_out, int32_t* kept_idx_out,
              int32_t* len_out) {
  if (!ctx) return BKV_EINVAL;
  bkv::EvictArgs a;
  a.K = K;
  a.V = V;
  a.weights = weights;
  a.L = L;
  a.budget = budget;
  a.cap_out = capacity_out;
  a.K_out = K_out;
  a.V_out = V_out;
  a.weights_out = weights_out;
  a.kept = kept_idx_out;
  a.len_out = len_out;
  return evict(ctx, a);
}

}  // extern "C"
