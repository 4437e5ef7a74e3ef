// Eviction from the 4-bit cache by accumulated attention weight, in place.
//
// A unit with n slots in use and a budget b < n keeps the b slots with the
// largest (forced, weight), ties to the lower slot; forced are positions below
// `sinks` and the `recent` newest positions.  Slot order means nothing to the
// attention, so only rows move that have to: the j-th evicted slot below b
// receives the j-th kept slot at or above b.  Sources and destinations are
// disjoint, so the copies need no order.
//
// One CTA takes a unit: the b-th largest key by four passes of a radix
// selection (8 bits each, most significant first), then one ordered pass that
// ranks the ties and lists the holes and the rows that fill them.
#include <cuda_runtime.h>

#include "ckv_device.cuh"
#include "q4_params.h"

namespace ckv {

namespace {

constexpr int kEvictThreads = 512;

// Order-preserving key of a weight: larger weight, larger key; -0 and +0 are
// one, NaN lies below everything.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Exclusive prefix of `v` over the CTA and the total (two syncs).
__device__ __forceinline__ int2 block_scan(int v, int* s_warp) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) s_warp[warp] = x;
  __syncthreads();
  int before = 0, total = 0;
  for (int w = 0; w < kEvictThreads / 32; ++w) {
    const int t = s_warp[w];
    if (w < warp) before += t;
    total += t;
  }
  __syncthreads();
  return make_int2(before + x - v, total);
}

__global__ void __launch_bounds__(kEvictThreads) evict_kernel(const __grid_constant__ Q4EvictParams p) {
  __shared__ int s_hist[256], s_warp[kEvictThreads / 32], s_newest, s_pick[2];
  const int unit = blockIdx.x, tid = threadIdx.x;
  const int n = min(max(p.c.lengths[unit], 0), p.c.capacity);
  const int b = p.budgets ? p.budgets[unit] : p.budget;
  if (b < 0 || b >= n) return;
  const long long base = static_cast<long long>(unit) * p.c.capacity;
  const int32_t* pos = p.c.positions + base;
  const float* wt = p.c.weights + base;
  if (tid == 0) s_newest = -0x7fffffff - 1;
  __syncthreads();
  int newest = -0x7fffffff - 1;
  for (int j = tid; j < n; j += kEvictThreads) newest = max(newest, pos[j]);
  atomicMax(&s_newest, newest);
  __syncthreads();
  newest = s_newest;
  auto key_of = [&](int j) -> uint32_t {
    const int at = pos[j];
    const bool forced = at < p.sinks || static_cast<long long>(at) > static_cast<long long>(newest) - p.recent;
    return forced ? 0xffffffffu : weight_key(wt[j]);
  };
  // threshold: the b-th largest key; `need` slots equal to it are kept
  uint32_t prefix = 0;
  int need = b;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += kEvictThreads) s_hist[i] = 0;
    __syncthreads();
    const uint32_t mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
    for (int j = tid; j < n; j += kEvictThreads) {
      const uint32_t k = key_of(j);
      if ((k & mask) == prefix) atomicAdd(&s_hist[(k >> shift) & 255u], 1);
    }
    __syncthreads();
    if (tid == 0) {
      int d = 255, left = need;
      while (d > 0 && s_hist[d] < left) left -= s_hist[d--];
      s_pick[0] = d;
      s_pick[1] = left;
    }
    __syncthreads();
    prefix |= static_cast<uint32_t>(s_pick[0]) << shift;
    need = s_pick[1];
    __syncthreads();
  }
  // holes below b and rows at or above b, both in slot order
  int32_t* holes = p.lists + base;
  int32_t* rows = holes + p.c.capacity / 2;
  int ties = 0, nh = 0, nr = 0;
  for (int j0 = 0; j0 < n; j0 += kEvictThreads) {
    const int j = j0 + tid;
    const uint32_t k = j < n ? key_of(j) : 0u;
    const bool tie = j < n && k == prefix;
    const int2 t = block_scan(tie, s_warp);
    const bool keep = j < n && (k > prefix || (tie && ties + t.x < need));
    ties += t.y;
    const bool hole = j < b && !keep, row = j >= b && keep;
    const int2 h = block_scan(hole, s_warp), r = block_scan(row, s_warp);
    if (hole) holes[nh + h.x] = j;
    if (row) rows[nr + r.x] = j;
    nh += h.y;
    nr += r.y;
  }
  __syncthreads();
  const int lane = tid & 31;
  for (int i = tid >> 5; i < nh; i += kEvictThreads / 32) {
    const long long to = base + holes[i], from = base + rows[i];
    if (lane < 10) {  // 4 + 4 pieces of codes, 1 + 1 of params
      const int part = lane < 8 ? lane >> 2 : lane - 8;
      uint8_t* a = lane < 8 ? p.c.codes[part] : p.c.params[part];
      const int bytes = lane < 8 ? kQ4CodeBytes : kQ4ParamBytes, at = lane < 8 ? (lane & 3) * 16 : 0;
      *reinterpret_cast<uint4*>(a + to * bytes + at) = *reinterpret_cast<const uint4*>(a + from * bytes + at);
    } else if (lane == 10) {
      p.c.positions[to] = p.c.positions[from];
    } else if (lane == 11) {
      p.c.weights[to] = p.c.weights[from];
    }
  }
  if (tid == 0) p.c.lengths[unit] = b;
}

}  // namespace

cudaError_t launch_q4_evict(const Q4EvictParams& p, cudaStream_t stream) {
  evict_kernel<<<p.c.batch * p.c.num_kv_heads, kEvictThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace ckv
