// The context behind a kb_ctx handle and the host-side helpers that every entry point uses:
// error text, device guard, guarded allocations.  Shared by the translation units of the library.
#pragma once

#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <vector>

#include <nvtx3/nvToolsExt.h>

#include "kb_common.cuh"

struct kb_ctx {
  int device = 0;
  int sm_count = 0;
  // Workspace for ws_cap_K candidates: [accumulators, set 0 | accumulators, set 1 | pointer table |
  // accumulators of the binary64 gate]; no offset depends on a call's K.
  unsigned char* ws = nullptr;
  size_t ws_bytes = 0;
  uint32_t ws_cap_K = 0;
  bool ws_fixed = false;            // the workspace is not ours to grow or free (kb_screen_static)
  // The binary32 gate keeps two sets of accumulators and counters.  A call works on set
  // `ws_parity`, which is zero on entry, and its lead kernel zeroes the other set (as far as the
  // last call on it got: `used_K`) for the next call.  `ws_dirty`: that may not hold (fresh
  // memory, a call that failed half-way or ran out of time, a call captured into a graph, a path
  // without a lead launch): the next call zeroes both sets with memsets first.
  int ws_parity = 0;
  uint32_t used_K[2] = {0, 0};
  bool ws_dirty = true;
  // Choice between the instantiations of the streaming kernel.  The plain one reports, in a
  // host-visible word, the share of its warp steps that took a fruitless second look: one byte
  // for looks taken while the candidate was lean, one for looks (and exact paths) beyond the lean
  // bound that changed nothing.  When the last report says a quarter or more, the next calls use
  // the sharp instantiation (first byte) or the by-definition one (second byte), and every so
  // often one of them probes the plain one again.
  unsigned int* h_hint = nullptr;   // pinned, mapped
  unsigned int* d_hint = nullptr;   // its device address
  int filter_mode = 0;              // 0 automatic, 1 plain, 2 sharp, 3 by definition
  int alt_mode = 1;                 // the instantiation the automatic choice currently alternates with: 1 or 3
  int sharp_left = 0;
  bool sharp_probe_next = false, sharp_probed = false;
  int last_mode = 0;                // instantiation of the last streaming launch: 0 plain, 1 sharp, 3 by definition
  float call_steps = 0.0f;          // warp steps of the current call's plain streaming launch (0: none)
  float steps_hist[2] = {0.0f, 0.0f};   // the same for the last call on each accumulator set
  // [0] status, [1..3] counters of the binary64 gate, [4] effective K of an indexed call,
  // [8..10] and [16..18] the two counter sets of the binary32 gate, [20..23] two 64-bit sums of
  // fruitless second looks on their way to the host, [60] probe sink
  unsigned int* d_status = nullptr;
  uint32_t forced_grid = 0;
  unsigned char* small_ws = nullptr; // single-launch path: [tickets 4 KB | partial records 384 KB]
  bool small_on = true;
  int wins_algo = 0;                // 0 auto, 1 direct comparison, 2 binary search on sorted rows,
                                    // 3 lane-per-row merge of sorted rows
  float* srt = nullptr;             // [K][S] sorted timings (binary-search win count)
  size_t srt_bytes = 0;
  char err[512] = {0};
  // staging owned for kb_screen_host
  unsigned char* st_ref = nullptr;
  size_t st_ref_bytes = 0;
  unsigned char* st_batch[2] = {nullptr, nullptr};
  size_t st_batch_bytes[2] = {0, 0};
  kb_screen_result* st_out = nullptr;
  size_t st_out_bytes = 0;
  cudaStream_t copy_stream = nullptr;
  cudaEvent_t ev_copied[2] = {nullptr, nullptr};
  cudaEvent_t ev_done[2] = {nullptr, nullptr};
  uint32_t skip_allocs = 0;         // test hook: let this many device allocations through, ...
  uint32_t fail_allocs = 0;         // ... then refuse this many
  // Every buffer the context owns sits between two 256-byte guard bands filled with kGuardByte;
  // kb_ctx_check_guards counts the band bytes that no longer hold it (an out-of-bounds write).
  struct Guarded { unsigned char* raw; size_t bytes; };
  std::vector<Guarded> guarded;
  // A launch that is captured into a graph keeps the addresses it was given: from the first such call on,
  // workspaces that are outgrown stay allocated until the context goes.
  bool captured = false;
  std::vector<void*> outgrown;
  // instrumentation
  uint64_t launches = 0;
  bool timing = false;
  bool dependent_launch = true;     // streaming kernel as a programmatic dependent of the lead kernel
  static constexpr int kTimers = 2, kPool = 256;
  cudaEvent_t tm_beg[kTimers][kPool] = {};
  cudaEvent_t tm_end[kTimers][kPool] = {};
  uint32_t tm_used[kTimers] = {0, 0};
  // model operators (kb_ops.h)
  unsigned char* ops_ws = nullptr;  // partial sums of the norm's parameter gradients
  size_t ops_ws_bytes = 0;
  void* encode_tiled = nullptr;     // the driver's tensor-map encoder, looked up at first use
  int cluster_room[9] = {};         // clusters of n CTAs, one CTA per SM, that run at the same time
  bool ops_ready = false;           // shared-memory limits of the operators' kernels are raised
  uint32_t product_rows = 0, product_splits = 0;   // of the last product's launch: rows of A per tile, CTAs per tile
};

namespace kb {

inline kb_status fail(kb_ctx* ctx, kb_status st, const char* fmt, ...) {
  if (ctx) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(ctx->err, sizeof ctx->err, fmt, ap);
    va_end(ap);
  }
  return st;
}

struct DeviceGuard {
  int prev = -1;
  bool changed = false;
  explicit DeviceGuard(int dev) {
    if (cudaGetDevice(&prev) == cudaSuccess && prev != dev) changed = cudaSetDevice(dev) == cudaSuccess;
  }
  ~DeviceGuard() {
    if (changed) cudaSetDevice(prev);
  }
};

#define KB_CUDA(ctx, call)                                                              \
  do {                                                                                  \
    cudaError_t e_ = (call);                                                            \
    if (e_ != cudaSuccess)                                                              \
      return fail((ctx), KB_ERR_CUDA, "%s failed: %s", #call, cudaGetErrorString(e_));  \
  } while (0)

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
inline int elem_bytes(kb_dtype dt) { return dt == KB_F32 ? 4 : (dt == KB_F8E4M3 || dt == KB_F8E5M2) ? 1 : 2; }
inline bool known_dtype(int dt) { return dt >= KB_F32 && dt <= KB_F8E5M2; }

// A named range around an entry point's host work, for a timeline tool that is attached
// (the header-only NVTX v3 calls do nothing otherwise).
struct TraceRange {
  explicit TraceRange(const char* name) { nvtxRangePushA(name); }
  ~TraceRange() { nvtxRangePop(); }
  TraceRange(const TraceRange&) = delete;
  TraceRange& operator=(const TraceRange&) = delete;
};

// Every device allocation of a context goes through here: a test can make it fail
// (kb_ctx_fail_next_allocs) without exhausting a GPU's memory, and every buffer gets guard
// bands (compute-sanitizer's stand-in for out-of-bounds writes; see kb_ctx_check_guards).
constexpr size_t kGuardBytes = 256;
constexpr int kGuardByte = 0xA5;
inline cudaError_t ctx_malloc(kb_ctx* ctx, void** p, size_t bytes) {
  *p = nullptr;
  if (ctx->skip_allocs) {
    --ctx->skip_allocs;
  } else if (ctx->fail_allocs) {
    --ctx->fail_allocs;
    return cudaErrorMemoryAllocation;
  }
  unsigned char* raw = nullptr;
  const size_t body = round_up(bytes, 256);
  cudaError_t e = cudaMalloc(reinterpret_cast<void**>(&raw), body + 2 * kGuardBytes);
  if (e == cudaSuccess) e = cudaMemset(raw, kGuardByte, kGuardBytes);
  if (e == cudaSuccess) e = cudaMemset(raw + kGuardBytes + body, kGuardByte, kGuardBytes);
  if (e != cudaSuccess) {
    if (raw) cudaFree(raw);
    cudaGetLastError();
    return e;
  }
  try {
    ctx->guarded.push_back({raw, body});
  } catch (...) {   // no host memory for the entry: nothing may be thrown across the C boundary
    cudaFree(raw);
    return cudaErrorMemoryAllocation;
  }
  *p = raw + kGuardBytes;
  return cudaSuccess;
}
inline void ctx_free(kb_ctx* ctx, void* p) {
  if (!p) return;
  unsigned char* raw = static_cast<unsigned char*>(p) - kGuardBytes;
  for (size_t i = 0; i < ctx->guarded.size(); ++i)
    if (ctx->guarded[i].raw == raw) {
      ctx->guarded.erase(ctx->guarded.begin() + (long)i);
      break;
    }
  cudaFree(raw);   // waits for enqueued work that still uses the buffer
}

// Grow *buf to at least `need` bytes.  The new buffer is allocated BEFORE the old one is
// released, and pointer and size change together: after a failure the context still holds
// its old, valid (pointer, size) pair and a later, smaller call works as before.
template <typename T>
inline kb_status ensure_buf(kb_ctx* ctx, T** buf, size_t* have, size_t need, const char* what = "device staging") {
  if (need <= *have) return KB_OK;
  void* fresh = nullptr;
  if (ctx_malloc(ctx, &fresh, need) != cudaSuccess)
    return fail(ctx, KB_ERR_WORKSPACE, "cannot allocate %zu bytes of %s", need, what);
  ctx_free(ctx, *buf);
  *buf = static_cast<T*>(fresh);
  *have = need;
  return KB_OK;
}

// Whether launches on `st` go into a graph (asked about the default stream while another one is
// captured, the runtime answers with an error: nothing may be allocated then either).
inline bool is_capturing(cudaStream_t st) {
  cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
  if (cudaStreamIsCapturing(st, &status) != cudaSuccess) {
    cudaGetLastError();
    return true;
  }
  return status != cudaStreamCaptureStatusNone;
}
// The same for a workspace that kernels on `st` are given the address of.  Growing is refused while the
// stream is captured; what a graph may use is kept.  Callers set ctx->captured for calls that are captured.
template <typename T>
inline kb_status ensure_workspace(kb_ctx* ctx, T** buf, size_t* have, size_t need, cudaStream_t st, const char* what) {
  if (need <= *have) return KB_OK;
  if (is_capturing(st))
    return fail(ctx, KB_ERR_WORKSPACE, "%s: %zu bytes cannot be allocated while a stream is captured; make such a call "
                "(or reserve) before the capture", what, need);
  if (!ctx->captured || !*buf) return ensure_buf(ctx, buf, have, need, what);
  try {
    ctx->outgrown.reserve(ctx->outgrown.size() + 1);
  } catch (...) {   // nothing may be thrown across the C boundary
    return fail(ctx, KB_ERR_WORKSPACE, "%s: no host memory to keep an outgrown buffer", what);
  }
  T* old = *buf;
  *buf = nullptr;
  const kb_status rc = ensure_buf(ctx, buf, have, need, what);
  if (rc == KB_OK)
    ctx->outgrown.push_back(old);
  else
    *buf = old;
  return rc;
}

}  // namespace kb
