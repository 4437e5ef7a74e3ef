// Host-side helpers shared by the files that implement the C ABI.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>

#include <cstdint>

#include "compresskv.h"

namespace ckv {
// In api.cu: the checks that every entry point makes of a problem description;
// the address under which the device reads K or V; the SMs that kernels on the
// stream may use (after the current device's one-time set-up); a map over
// `rows` rows of 64 bytes for boxes of `box_rows`, 64-byte swizzle.
int check_problem(const ckv_problem* p);
int device_readable(const void* ptr, const void** dev);
int usable_sms(cudaStream_t stream, int* sms);
int make_row64_map(const void* base, unsigned long long rows, unsigned box_rows, CUtensorMap* map);
}  // namespace ckv

namespace {

// A named range around each entry point for profilers (NVTX; nothing happens
// unless a profiling tool is attached to the process).
struct NvtxRange {
  explicit NvtxRange(const char* name) { nvtxRangePushA(name); }
  ~NvtxRange() { nvtxRangePop(); }
  NvtxRange(const NvtxRange&) = delete;
  NvtxRange& operator=(const NvtxRange&) = delete;
};

inline bool aligned16(const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & 15u) == 0; }

// ------------------------------------------------------------------ tracing
// Records the caller's trace events around each launch.  A failed record
// (for example a null event handle) is reported as CKV_ERR_INVALID_ARG and
// the runtime's last-error state is cleared.
struct Tracer {
  ckv_trace* t;
  cudaStream_t s;
  int slot = -1;
  int begin(int kind) {
    slot = -1;
    if (!t) return CKV_OK;
    if (t->count < t->capacity && t->events) {
      slot = t->count++;
      if (t->kinds) t->kinds[slot] = kind;
      return record(static_cast<cudaEvent_t>(t->events[2 * slot]));
    }
    return CKV_OK;
  }
  int end() {
    if (!t) return CKV_OK;
    ++t->launches;
    if (slot >= 0) return record(static_cast<cudaEvent_t>(t->events[2 * slot + 1]));
    return CKV_OK;
  }
  int record(cudaEvent_t e) {
    if (!e) return CKV_ERR_INVALID_ARG;
    cudaStreamCaptureStatus cs = cudaStreamCaptureStatusNone;
    cudaError_t err = cudaStreamIsCapturing(s, &cs);
    if (err == cudaSuccess) {
      err = cs == cudaStreamCaptureStatusActive
                ? cudaEventRecordWithFlags(e, s, cudaEventRecordExternal)
                : cudaEventRecord(e, s);
    }
    if (err != cudaSuccess) {
      cudaGetLastError();
      return CKV_ERR_INVALID_ARG;
    }
    return CKV_OK;
  }
};

// Launch `fn` bracketed by the trace: trace errors win over a clean launch.
template <class F>
int traced(Tracer& tr, int kind, F&& fn) {
  int rc = tr.begin(kind);
  if (rc != CKV_OK) return rc;
  const cudaError_t e = fn();
  const int rc2 = tr.end();
  if (e != cudaSuccess) return CKV_ERR_CUDA;
  return rc2;
}

}  // namespace
