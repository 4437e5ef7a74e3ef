// Rows of a paged cache, packed.
//
// Memory is the bound: a row is read once and written once.  A warp takes one
// token -- its page is looked up once -- and moves the rows of its heads, of K
// and V, with all of a lane's loads in flight at a time.
#include "ckv_device.cuh"
#include "paged_params.h"
#include "q4_params.h"

namespace ckv {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kUnroll = 8;  // 16-byte pieces of a lane in flight
constexpr int kPieces = kHeadDim * 2 / 16;

__global__ void __launch_bounds__(kThreads) paged_gather_kernel(const __grid_constant__ PagedGatherParams p, int of) {
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const long long task = static_cast<long long>(blockIdx.x) * kWarps + threadIdx.x / 32;
  const int row = static_cast<int>(task / of), w = static_cast<int>(task - static_cast<long long>(row) * of);
  if (row >= p.rows) return;
  int seq = 0, index = row;
  if (p.rows_per_seq >= 0) {
    seq = row / p.rows_per_seq;
    index = row - seq * p.rows_per_seq;
  } else {
    int hi = p.c.batch;  // cu_rows[seq] <= row < cu_rows[hi]
    while (hi - seq > 1) {
      const int mid = (seq + hi) / 2;
      if (p.cu_rows[mid] <= row)
        seq = mid;
      else
        hi = mid;
    }
    index = row - p.cu_rows[seq];
  }
  const int first = p.start ? p.start[seq] : 0, length = min(p.c.lengths[seq], p.c.capacity);
  if (first < 0 || length < 0) return;
  const long long slot = static_cast<long long>(first) + index;
  int page = -1;
  if (slot < length) page = p.c.table[seq * p.c.table_stride + (slot >> p.c.page_shift)];
  if (page < 0 || page >= p.c.num_pages) {
    if (lane == 0 && w == 0 && p.status) atomicCAS(p.status, 0, CKV_DEV_ERR_INDEX);
    return;
  }
  const long long at = page * p.c.page_stride + (slot & ((1 << p.c.page_shift) - 1)) * p.c.slot_stride;
  const long long to = static_cast<long long>(row) * p.c.num_kv_heads * kHeadDim;
  const int each = p.c.num_kv_heads * kPieces;              // pieces of the row in K, and in V
  const int lo = p.out[0] ? 0 : each, hi = p.out[1] ? 2 * each : each;
  for (int i0 = lo + w * 32 + lane; i0 < hi; i0 += 32 * of * kUnroll) {
    uint4 x[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int i = i0 + u * 32 * of;
      if (i < hi) {
        const int part = i >= each, j = i - part * each;
        x[u] = *reinterpret_cast<const uint4*>(p.c.pages[part] + at + (j / kPieces) * p.c.head_stride +
                                               (j % kPieces) * 8);
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int i = i0 + u * 32 * of;
      if (i < hi) {
        const int part = i >= each, j = i - part * each;
        *reinterpret_cast<uint4*>(p.out[part] + to + j * 8) = x[u];
      }
    }
  }
}

}  // namespace

cudaError_t launch_paged_gather(const PagedGatherParams& p, cudaStream_t stream) {
  const int pieces = p.c.num_kv_heads * kPieces * ((p.out[0] != nullptr) + (p.out[1] != nullptr));
  const int most = (pieces + 31) / 32;
  int of = (4864 + p.rows - 1) / p.rows;
  of = of < 1 ? 1 : of > most ? most : of;
  const long long ctas = (static_cast<long long>(p.rows) * of + kWarps - 1) / kWarps;
  return launch_dependent(paged_gather_kernel, dim3(static_cast<unsigned>(ctas)), kThreads, 0, stream, p, of);
}

}  // namespace ckv
