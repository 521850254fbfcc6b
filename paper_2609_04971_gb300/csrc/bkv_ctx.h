// The context behind the C ABI and the small helpers that its entry points share.
#pragma once

#include <cstdarg>
#include <cstdio>
#include <string>
#include <vector>

#include "bkv.h"
#include "bkv_internal.h"

struct bkv_ctx {
  bkv_config cfg{};
  bkv::Shape shape{};
  cudaStream_t stream = nullptr;
  int device = 0;
  // beacon state
  float* cent = nullptr;
  double* sums = nullptr;
  long long* counts = nullptr;
  bool state_ready = false;
  // Continual FPS (BKV_F_CONTINUAL_FPS): per-query-head buffers; cent / counts then hold each
  // compress's beacons ([n_inst][G * n_beacons] rows, count 1 or 0) for the scoring-query build
  bool cfps = false;
  int b_min = 0, b_max = 0, n_heads = 0;
  __nv_bfloat16* cbuf = nullptr;  // [n_heads][b_max][d]
  int* csize = nullptr;           // [n_heads]
  // scratch
  __nv_bfloat16* qobs = nullptr;  // [n_inst][n_obs_pad][d]
  uint32_t* valid = nullptr;      // [n_inst][4]
  float* rscore = nullptr;        // [n_inst][cap]
  double2* rope = nullptr;        // [W + 1][d / 2] fp64 (cos, sin), then the same table in fp32
  int* err = nullptr;             // device error word
  // pinned host staging of the rotary table, a ring of kRopeSlots: a compress fills the next slot,
  // a kernel on the stream copies it to `rope` through the slot's device mapping, and the slot is
  // refilled only after that copy's event completed
  static constexpr int kRopeSlots = 4;
  double2* rope_pinned[kRopeSlots] = {};
  void* rope_mapped[kRopeSlots] = {};  // device address of rope_pinned[i]
  cudaEvent_t rope_ev[kRopeSlots] = {};
  bool rope_used[kRopeSlots] = {};
  int rope_next = 0;
  // per-instance lengths (bkv_compress_ragged): the instances a compress evicts from, and a rotary
  // table per batch row followed by the causal gaps [batch][W] (int32), staged like `rope`
  int* work = nullptr;            // [n_inst]
  int* n_work = nullptr;          // [1]
  unsigned char* rag = nullptr;   // device copy of the per-row tables and gaps
  size_t rag_bytes = 0, rag_row = 0, rag_gaps_off = 0;  // total bytes; one row's table (double2 units); gaps offset
  void* rag_pinned[kRopeSlots] = {};
  void* rag_mapped[kRopeSlots] = {};
  cudaEvent_t rag_ev[kRopeSlots] = {};
  bool rag_used[kRopeSlots] = {};
  int rag_next = 0;
  // attention (bkv_attend_reserve): partial results, logits and normalisers of one call
  unsigned char* attend_ws = nullptr;
  size_t attend_ws_bytes = 0;
  bool attend_ws_captured = false;  // a graph may hold its address
  // workspaces that a larger one replaced while a graph may hold their address; freed with the context
  struct Workspace {
    unsigned char* p;
    Workspace* next;
  };
  Workspace* attend_ws_old = nullptr;
  cudaEvent_t switch_ev = nullptr;  // orders a new stream after the previous one (bkv_set_stream)
  std::string last_error;
  // per-kernel timing
  struct Rec {
    cudaEvent_t start, stop;
    int kernel;
  };
  bool prof = false;
  std::vector<Rec> pending;
  std::vector<cudaEvent_t> spare;
  double prof_ms[BKV_NUM_KERNELS] = {};
  long long prof_n[BKV_NUM_KERNELS] = {};
};

namespace bkv {


inline int fail(bkv_ctx* c, int code, const char* fmt, ...) {
  if (c) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    c->last_error = buf;
  }
  return code;
}

inline int cuda_fail(bkv_ctx* c, cudaError_t e, const char* what) {
  return fail(c, BKV_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline cudaEvent_t take_event(bkv_ctx* c) {
  if (!c->spare.empty()) {
    cudaEvent_t ev = c->spare.back();
    c->spare.pop_back();
    return ev;
  }
  cudaEvent_t ev = nullptr;
  cudaEventCreate(&ev);
  return ev;
}

// Brackets one kernel launch with events when timing is enabled.
struct ProfScope {
  bkv_ctx* c;
  int kernel;
  cudaEvent_t start = nullptr;
  ProfScope(bkv_ctx* ctx, int k) : c(ctx), kernel(k) {
    if (c->prof && (start = take_event(c))) cudaEventRecord(start, c->stream);
  }
  ~ProfScope() {
    if (!start) return;
    cudaEvent_t stop = take_event(c);
    if (!stop) return;
    cudaEventRecord(stop, c->stream);
    c->pending.push_back({start, stop, kernel});
  }
};

// True when the allocation-failure hook wants this allocation to fail (bkv_api.cu).
bool fail_this_alloc();

}  // namespace bkv
