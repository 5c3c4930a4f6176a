// What the C entry points of the library share: the context, the plan upload, error mapping and per-launch timing.
// Internal to the library.
#ifndef OTAS_CONTEXT_H_
#define OTAS_CONTEXT_H_

#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "../../include/otas.h"
#include "kernels.h"

namespace otas {

constexpr size_t kAlign = 256;
constexpr size_t kPlanInts = (size_t)1 << 20;  // capacity of the device plan buffer (int32 entries)
constexpr int kStageSlots = 32;
constexpr size_t kSlotInts = kPlanInts / kStageSlots;
constexpr int kMaxLanes = 8;

inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

}  // namespace otas

struct otas_ctx {
  otas_model_desc desc;
  std::vector<otas_layer_weights> layers;
  hipStream_t stream;
  int device;
  int32_t* d_plan;        // device plan buffer [kPlanInts]
  int32_t* d_scratch;     // this device's copy of the static scratch array (otas_token_merge_static)
  // Pinned host staging for the plan: a ring of kStageSlots slots of kSlotInts entries, so that the host
  // can enqueue that many calls ahead of the device (a host thread that is descheduled for tens of
  // milliseconds then costs nothing as long as the queue holds work).  Slot i may be overwritten once
  // h_done[i] has completed.  A plan larger than a slot uses the whole buffer and waits for the copy.
  int32_t* h_plan;
  hipEvent_t h_done[otas::kStageSlots];
  bool h_used[otas::kStageSlots];
  int h_next;
  // The merge plan of a layer needs only that layer's keys (the QKV projection), so it runs on a
  // second stream next to attention and the output projection: forked after the QKV GEMM, joined
  // before merge-apply.
  // A forward pass may also be cut into lanes (contiguous query ranges) that run side by side on
  // streams of their own, so that one lane's launch gaps, partial waves and latency-bound small
  // kernels overlap another lane's work.  Lane 0 runs on the caller's stream.
  struct Lane {
    hipStream_t main, side;
    hipEvent_t ev_fork, ev_join, ev_done;
  };
  Lane lane[8];
  hipEvent_t ev_begin;
  int lanes;   // requested lane count, 0 = chosen from the batch size
  int lanes_ready;   // lanes whose streams and events exist
  // optional per-launch timing (otas_timing_enable): one event pair per launch, summed per kind
  bool timing;
  float ev_overhead_ms;   // what an event pair reads around an empty launch (subtracted from every record)
  std::vector<hipEvent_t> ev_pool;
  std::vector<int> ev_kind;   // kind of the launch bracketed by ev_pool[2i], ev_pool[2i+1]
  // optional shader-clock probe (otas_clock_probe_start): its own stream and sample buffer, made at first use
  hipStream_t probe_stream;
  uint32_t* d_probe;      // [kProbeMaxSamples]
  int32_t probe_samples;  // samples of the probe in flight or finished and unread, 0 = none
};

namespace otas {

inline size_t elem_size(int dtype) { return dtype == OTAS_F32 ? 4 : 2; }

inline bool offsets_ok(const int32_t* off, int B) {
  if (off[0] != 0) return false;
  for (int q = 0; q < B; ++q)
    if (off[q + 1] < off[q]) return false;
  return true;
}

// Copies `count` ints to the device plan buffer at entry `at` through pinned staging.
inline otas_status upload_plan(otas_ctx* c, const int32_t* host, size_t count) {
  if (count > kPlanInts) return OTAS_ENOMEM;
  const size_t bytes = count * sizeof(int32_t);
  if (count > kSlotInts) {
    for (int j = 0; j < kStageSlots; ++j) {
      if (c->h_used[j] && hipEventSynchronize(c->h_done[j]) != hipSuccess) return OTAS_EDEVICE;
      c->h_used[j] = false;
    }
    std::memcpy(c->h_plan, host, bytes);
    if (hipMemcpyAsync(c->d_plan, c->h_plan, bytes, hipMemcpyHostToDevice, c->stream) != hipSuccess ||
        hipStreamSynchronize(c->stream) != hipSuccess)
      return OTAS_EDEVICE;
    return OTAS_OK;
  }
  const int i = c->h_next;
  c->h_next = (c->h_next + 1) % kStageSlots;
  if (c->h_used[i] && hipEventSynchronize(c->h_done[i]) != hipSuccess) return OTAS_EDEVICE;
  int32_t* slot = c->h_plan + (size_t)i * kSlotInts;
  std::memcpy(slot, host, bytes);
  if (hipMemcpyAsync(c->d_plan, slot, bytes, hipMemcpyHostToDevice, c->stream) != hipSuccess) return OTAS_EDEVICE;
  if (hipEventRecord(c->h_done[i], c->stream) != hipSuccess) return OTAS_EDEVICE;
  c->h_used[i] = true;
  return OTAS_OK;
}
inline otas_status upload_plan(otas_ctx* c, const std::vector<int32_t>& host) {
  return upload_plan(c, host.data(), host.size());
}

// A failing HIP call maps to OTAS_EDEVICE; with OTAS_DEBUG set in the environment it is also named
// on stderr.
inline bool hip_ok(hipError_t e, const char* what) {
  if (e == hipSuccess) return true;
  static const bool verbose = std::getenv("OTAS_DEBUG") != nullptr;
  if (verbose) std::fprintf(stderr, "otas: %s -> %s\n", what, hipGetErrorString(e));
  return false;
}
#define OTAS_HIP(expr)                              \
  do {                                              \
    if (!hip_ok((expr), #expr)) return OTAS_EDEVICE; \
  } while (0)

enum Kind { K_PREPEND = 0, K_LN, K_QKV, K_ATTN, K_PROJ, K_PLAN, K_APPLY, K_FC1, K_FC2, K_REDUCE, K_MISC, K_COUNT };
inline const char* const kKindNames[K_COUNT] = {"prompt_prepend", "layer_norm", "gemm_qkv", "attention", "gemm_proj",
                                         "merge_plan", "merge_apply", "gemm_fc1", "gemm_fc2", "splitk_reduce_ln",
                                         "misc"};

// Brackets one launch with an event pair when timing is on.
struct LaunchTimer {
  otas_ctx* c;
  bool on;
  hipStream_t st;
  LaunchTimer(otas_ctx* ctx, int kind, hipStream_t stream) : c(ctx), on(ctx->timing), st(stream) {
    if (!on) return;
    const size_t i = c->ev_kind.size();
    while (c->ev_pool.size() < 2 * (i + 1)) {
      hipEvent_t e;
      if (hipEventCreate(&e) != hipSuccess) { on = false; return; }
      c->ev_pool.push_back(e);
    }
    c->ev_kind.push_back(kind);
    idx = i;
    (void)hipEventRecord(c->ev_pool[2 * i], st);
  }
  ~LaunchTimer() {
    if (on) (void)hipEventRecord(c->ev_pool[2 * idx + 1], st);
  }
  size_t idx = 0;
};
#define OTAS_LAUNCH_ON(kind, stream, expr) \
  do {                                     \
    LaunchTimer _t(c, kind, stream);       \
    OTAS_HIP(expr);                        \
  } while (0)
#define OTAS_LAUNCH(kind, expr) OTAS_LAUNCH_ON(kind, c->stream, expr)

}  // namespace otas
#endif  // OTAS_CONTEXT_H_
