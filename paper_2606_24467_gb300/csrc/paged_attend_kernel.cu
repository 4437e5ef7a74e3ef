// Attention of chunks of query tokens over a paged cache.
//
// One pass over the slots with each row's running maximum m and sum l: a tile's
// logits z raise m to m', and l and the output are scaled by 2^(m - m') before
// 2^(z - m') is added.  A row is one head of one query token; 16 rows of a KV
// group share the tiles of 32 slots.
#include "ckv_device.cuh"
#include "paged_params.h"
#include "q4_params.h"

namespace ckv {
namespace {

constexpr int kRows = 16, kSlots = 32, kThreads = 128;

template <bool kBf16>
__device__ __forceinline__ float value(uint16_t w) {
  if (kBf16) return __uint_as_float(static_cast<uint32_t>(w) << 16);
  float r;
  asm("{\n\t.reg .f16 h;\n\tmov.b16 h, %1;\n\tcvt.f32.f16 %0, h;\n\t}" : "=f"(r) : "h"(w));
  return r;
}
template <bool kBf16>
__device__ __forceinline__ uint16_t rounded(float x) {
  uint32_t r;
  if (kBf16)
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(0.f), "f"(x));
  else
    r = pack_half2(x, 0.f);
  return static_cast<uint16_t>(r);
}

template <bool kBf16>
__global__ void __launch_bounds__(kThreads) paged_attend_kernel(const __grid_constant__ PagedAttendParams p) {
  pdl_wait();
  __shared__ float q[kRows][kHeadDim], kv[kSlots][kHeadDim + 1], z[kRows][kSlots + 1];
  __shared__ float m[kRows], l[kRows], rescale[kRows];
  const int seq = blockIdx.z, head = blockIdx.y, tid = threadIdx.x;
  const int row0 = p.rows_per_seq >= 0 ? seq * p.rows_per_seq : p.cu_rows[seq];
  const int n = p.rows_per_seq >= 0 ? p.rows_per_seq : p.cu_rows[seq + 1] - row0;
  const int r0 = blockIdx.x * kRows;
  if (r0 >= n * p.group) return;
  const int length = max(min(p.c.lengths[seq], p.c.capacity), 0);
  const long long start = p.start ? p.start[seq] : static_cast<long long>(length) - n;
  auto token = [&](int r) { return (r0 + r) / p.group; };
  auto q_head = [&](int r) { return head * p.group + (r0 + r) % p.group; };
  for (int r = 0; r < kRows; ++r)
    q[r][tid] = token(r) < n ? value<kBf16>(p.q[(row0 + token(r)) * p.q_token + q_head(r) * p.q_head + tid]) : 0.f;
  if (tid < kRows) {
    m[tid] = -INFINITY;
    l[tid] = 0.f;
  }
  float o[kRows] = {};
  long long end = length;
  if (p.causal) end = min(end, start + min(token(kRows - 1), n - 1) + 1);
  for (int s0 = 0; s0 < end; s0 += kSlots) {
    long long at[2];
    __syncthreads();
    for (int j = 0; j < kSlots; ++j) {
      const int slot = s0 + j;
      int page = -1;
      if (slot < length) {
        page = p.c.table[seq * p.c.table_stride + (slot >> p.c.page_shift)];
        if (page < 0 || page >= p.c.num_pages) {
          page = -1;
          if (tid == 0) atomicCAS(p.status, 0, CKV_DEV_ERR_INDEX);
        }
      }
      at[0] = page * p.c.page_stride + (slot & ((1 << p.c.page_shift) - 1)) * p.c.slot_stride + head * p.c.head_stride;
      kv[j][tid] = page >= 0 ? value<kBf16>(p.c.pages[0][at[0] + tid]) : 0.f;
    }
    __syncthreads();
    for (int i = tid; i < kRows * kSlots; i += kThreads) {
      const int r = i / kSlots, j = i % kSlots;
      float x = 0.f;
      for (int c = 0; c < kHeadDim; ++c) x = fmaf(q[r][c], kv[j][c], x);
      const bool seen = s0 + j < length && (!p.causal || s0 + j <= start + token(r));
      z[r][j] = seen ? x * p.scale_log2 : -INFINITY;
    }
    __syncthreads();
    if (tid < kRows) {
      float top = m[tid];
      for (int j = 0; j < kSlots; ++j) top = fmaxf(top, z[tid][j]);
      const float ref = top == -INFINITY ? 0.f : top;
      float sum = 0.f;
      for (int j = 0; j < kSlots; ++j) {
        z[tid][j] = exp2f(z[tid][j] - ref);
        sum += z[tid][j];
      }
      rescale[tid] = exp2f(m[tid] - ref);
      l[tid] = l[tid] * rescale[tid] + sum;
      m[tid] = top;
    }
    __syncthreads();
    for (int r = 0; r < kRows; ++r) o[r] *= rescale[r];
    for (int j = 0; j < kSlots; ++j) {
      const int slot = s0 + j;
      if (slot >= length) break;
      const int page = p.c.table[seq * p.c.table_stride + (slot >> p.c.page_shift)];
      if (page < 0 || page >= p.c.num_pages) continue;
      at[1] = page * p.c.page_stride + (slot & ((1 << p.c.page_shift) - 1)) * p.c.slot_stride + head * p.c.head_stride;
      const float v = value<kBf16>(p.c.pages[1][at[1] + tid]);
      for (int r = 0; r < kRows; ++r)
        if (!p.causal || slot <= start + token(r)) o[r] = fmaf(z[r][j], v, o[r]);
    }
  }
  __syncthreads();
  for (int r = 0; r < kRows; ++r)
    if (token(r) < n) {
      const float x = l[r] == 0.f ? 0.f : o[r] / l[r];  // (a NaN row has a sum, NaN)
      p.out[(row0 + token(r)) * p.o_token + q_head(r) * p.o_head + tid] = rounded<kBf16>(x);
      if (p.lse && tid == 0)
        p.lse[static_cast<long long>(q_head(r)) * p.rows + row0 + token(r)] =
            l[r] == 0.f ? -INFINITY : (m[r] + log2f(l[r])) * 0.6931471805599453f;
    }
}

}  // namespace

cudaError_t launch_paged_attend(const PagedAttendParams& p, cudaStream_t stream) {
  int most = p.rows_per_seq;
  if (most < 0)
    for (int s = 0; s < p.c.batch; ++s) most = max(most, p.cu_rows[s + 1] - p.cu_rows[s]);
  const dim3 grid((most * p.group + kRows - 1) / kRows, p.c.num_kv_heads, p.c.batch);
  return p.is_bf16 ? launch_dependent(paged_attend_kernel<true>, grid, kThreads, 0, stream, p)
                   : launch_dependent(paged_attend_kernel<false>, grid, kThreads, 0, stream, p);
}

}  // namespace ckv
