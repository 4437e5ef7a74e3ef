// Host-side helpers shared by the files that implement the C ABI.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>

#include <algorithm>
#include <cstdint>

#include "ckv_params.h"
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
// A map over f16 / bf16 rows of 128 channels in `rank` - 1 dimensions (strides in
// elements), for boxes of 64 channels, 128-byte swizzle.
int make_rows_map(const void* base, bool bf16, int rank, const unsigned long long* dims, const long long* strides,
                  const unsigned* box, CUtensorMap* map);
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

// Whether two rows of kHeadDim elements share one, in a layout of n[i] rows at
// strides[i] (0 .. kMaxStride) in each of three dimensions.  They do not where
// every stride holds what the smaller ones span; otherwise they do exactly
// where the indices' differences, not all zero, come to less than a row.
constexpr int64_t kMaxStride = 1LL << 44;  // (32 TB: products of strides and indices stay in 64 bits)
inline bool rows_overlap(const int64_t (&strides)[3], const int (&n)[3]) {
  int order[3] = {0, 1, 2};
  std::sort(order, order + 3, [&](int a, int b) { return strides[a] < strides[b]; });
  int64_t span = ckv::kHeadDim;
  bool nested = true;
  for (int d : order) {
    if (n[d] == 1) continue;
    nested = nested && strides[d] >= span;
    span += strides[d] * (n[d] - 1);  // (a dimension of one row has no stride)
  }
  if (nested) return false;
  // the dimension of most rows is solved for
  const int a = static_cast<int>(std::max_element(n, n + 3) - n), b = (a + 1) % 3, c = (a + 2) % 3;
  const int64_t s = strides[a], most = n[a] - 1;
  if (most > 0 && s < ckv::kHeadDim) return true;
  for (int64_t j = 0; j < n[b]; ++j)
    for (int64_t k = j ? 1 - n[c] : 1; k < n[c]; ++k) {
      const int64_t rest = j * strides[b] + k * strides[c], near = most ? -rest / s : 0;
      for (int64_t i = near - 1; i <= near + 1; ++i) {
        const int64_t at = rest + std::min(std::max(i, -most), most) * s;
        if (at < ckv::kHeadDim && at > -ckv::kHeadDim) return true;
      }
    }
  return false;
}

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
