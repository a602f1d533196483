// The context behind every entry point: device, stream, cached plan and scratch, with the helpers
// that the files implementing the C ABI share (device switch, named ranges, logging, error codes,
// growing scratch).
#pragma once

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <new>

#if defined(__has_include)
#if __has_include(<nvtx3/nvToolsExt.h>)
#include <nvtx3/nvToolsExt.h>
#define QV2_HAVE_NVTX 1
#endif
#endif

#include "qv2_common.cuh"

namespace qv2 {
constexpr int kCodeRing = 4;     // pinned staging areas for the per-call table of code pointers
constexpr uint64_t kDefaultChunkBytes = 48ull << 20;
}  // namespace qv2

struct qv2_ctx {
  int device = 0;
  cudaStream_t stream = nullptr;
  int sm_count = 1;
  qv2::GridCaps caps;               // largest useful grid of each persistent kernel on this device
  int last_cuda = 0;
  uint64_t launches = 0;
  uint64_t syncs = 0;          // host-side stream synchronisations this context has performed
  uint32_t live_graphs = 0;    // captured passes that hold addresses of this context's scratch
  bool log = false;            // QV2_LOG=1: one line per call on stderr
  uint32_t schedule = QV2_SCHEDULE_PHASE_MAJOR;
  uint64_t chunk_bytes = qv2::kDefaultChunkBytes;
  uint32_t fold_mode = QV2_FOLD_AUTO;
  bool dependent_launch = true;   // kernels of a pass are launched as programmatic dependents of one another

  // cached plan: rebuilt only when the descriptor bytes or the schedule change
  qv2::HostPlan plan;
  std::vector<uint8_t> plan_key;
  bool plan_valid = false;

  // device scratch
  qv2::TensorRec* d_tensors = nullptr; size_t cap_tensors = 0;
  qv2::Tile* d_tiles = nullptr;        size_t cap_tiles = 0;
  qv2::Tile* d_hist_tiles = nullptr;   size_t cap_hist_tiles = 0;
  qv2::Tile* d_ghist_tiles = nullptr;  size_t cap_ghist_tiles = 0;   // per-group histogram mode
  uint32_t* d_ghist_owner = nullptr; size_t cap_ghist_owner = 0;
  unsigned long long* d_ghist = nullptr; size_t cap_ghist = 0;  // used when the caller passes no group_hist
  double2* d_partials = nullptr;  size_t cap_slots = 0;
  uint2* d_rslots = nullptr;      size_t cap_rslots = 0;
  double* d_partials_xe = nullptr; size_t cap_slots_xe = 0;   // sum x*e slots, cosine only
  unsigned long long* d_kl_hist = nullptr; size_t cap_kl_hist = 0;   // used when the caller passes no hists
  float* d_tensor_absmax = nullptr; size_t cap_absmax = 0;
  // accumulators that are zero between passes (cleared when a plan is made resident, and by the
  // CTA that consumes them afterwards)
  uint32_t* d_keys = nullptr;     size_t cap_keys = 0;         // kmin then kmax, total_groups each
  unsigned long long* d_nf_acc = nullptr; size_t cap_nf = 0;   // per tensor
  unsigned long long* d_hist_acc = nullptr; size_t cap_hist_acc = 0;   // 2048 per percentile tensor
  uint32_t* d_tickets = nullptr;  size_t cap_tickets = 0;      // 3 per tensor: range, histogram, metrics
  uint8_t** d_codes = nullptr;    size_t cap_codes = 0;        // per-tensor code buffers of the current call
  double* d_rank = nullptr;                                    // 2 * kMaxRankLayers doubles
  // qv2_mx_linear: the activations of the current call in packed form
  uint8_t* d_mx_codes = nullptr;  size_t cap_mx_codes = 0;  bool mx_codes_captured = false;
  uint8_t* d_mx_scales = nullptr; size_t cap_mx_scales = 0; bool mx_scales_captured = false;
  std::vector<void*> kept;        // outgrown blocks whose addresses a graph of the caller's may hold; freed with the context
  uint32_t* h_fault = nullptr;    // host-mapped word and its device address: a kernel that gave up waiting sets it
  uint32_t* d_fault = nullptr;
  // pinned host staging for the plan upload
  uint8_t* h_pinned = nullptr;    size_t cap_pinned = 0;
  // pinned ring for the code-pointer table: a call fills the next area and copies it on the
  // stream; the area's event tells when it may be refilled
  uint8_t** h_codes[qv2::kCodeRing] = {}; size_t cap_h_codes = 0;
  cudaEvent_t code_ev[qv2::kCodeRing] = {};
  uint32_t code_next = 0;
  // qv2_set_phase_timing: events around the range and histogram phases of qv2_calibrate
  bool phase_timing = false;
  bool phase_marks_valid = false;
  cudaEvent_t phase_ev[3] = {};
};

namespace qv2 {

struct DeviceGuard {
  int prev = -1;
  bool switched = false;
  explicit DeviceGuard(int dev) {
    if (cudaGetDevice(&prev) == cudaSuccess && prev != dev) switched = cudaSetDevice(dev) == cudaSuccess;
  }
  ~DeviceGuard() { if (switched) cudaSetDevice(prev); }
};

// A named range around each entry point for timeline tools; compiled out without the NVTX headers.
struct TraceRange {
#ifdef QV2_HAVE_NVTX
  explicit TraceRange(const char* name) { nvtxRangePushA(name); }
  ~TraceRange() { nvtxRangePop(); }
#else
  explicit TraceRange(const char*) {}
#endif
};

// QV2_LOG=1: one line per call on stderr (host side only; nothing is read back from the device).
inline void log_call(const qv2_ctx* c, const char* call, uint32_t n_tensors, uint64_t launches_before, int status) {
  if (!c->log) return;
  std::fprintf(stderr, "qv2: %s tensors=%u tiles=%zu stages=%zu launches=%llu status=%d (%s)\n", call, n_tensors,
               c->plan_valid ? c->plan.tiles.size() : (size_t)0, c->plan_valid ? c->plan.stages.size() : (size_t)0,
               (unsigned long long)(c->launches - launches_before), status, qv2_status_string(status));
}

inline int cuda_fail(qv2_ctx* c, cudaError_t e) {
  c->last_cuda = (int)e;
  c->plan_valid = false;          // a pass that stopped half-way may leave accumulators dirty: start over
  return e == cudaErrorMemoryAllocation ? QV2_ERR_NOMEM : QV2_ERR_CUDA;
}

#define QV2_CUDA(c, expr)                              \
  do {                                                 \
    cudaError_t e__ = (expr);                          \
    if (e__ != cudaSuccess) return cuda_fail((c), e__);\
  } while (0)

// graph_held: a captured pass may hold the address of this buffer, so it must not move while one
// is alive.
template <class T>
int grow(qv2_ctx* c, T** p, size_t* cap, size_t need, bool graph_held = true) {
  if (need <= *cap) return QV2_OK;
  if (graph_held && c->live_graphs) return QV2_ERR_UNSUPPORTED;
  size_t want = need + need / 4 + 16;
  if (*p) { QV2_CUDA(c, cudaFree(*p)); *p = nullptr; *cap = 0; }
  QV2_CUDA(c, cudaMalloc((void**)p, want * sizeof(T)));
  *cap = want;
  return QV2_OK;
}

// The same for a buffer whose address calls may leave in a graph that the caller captures (*captured: one has).  Such a
// block is kept until the context ends, since nothing tells when the graph is gone; while the stream is capturing the buffer
// cannot grow at all.
inline int grow_capturable(qv2_ctx* c, uint8_t** p, size_t* cap, size_t need, bool capturing, bool* captured) {
  if (need > *cap) {
    if (capturing) return QV2_ERR_UNSUPPORTED;
    if (*captured) {
      try { c->kept.push_back(*p); } catch (const std::bad_alloc&) { return QV2_ERR_NOMEM; }
      *p = nullptr; *cap = 0; *captured = false;
    }
    if (int st = grow(c, p, cap, need, false)) return st;
  }
  if (capturing) *captured = true;
  return QV2_OK;
}

}  // namespace qv2
