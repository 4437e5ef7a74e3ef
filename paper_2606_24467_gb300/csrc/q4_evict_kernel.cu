// Eviction from the 4-bit cache by accumulated attention weight, in place.
//
// A unit with n slots in use and a budget b < n keeps the b slots with the
// largest (forced, weight), ties to the lower slot; forced are positions below
// `sinks` and the `recent` newest positions.  Slot order means nothing to the
// attention, so only rows move that have to: the j-th evicted slot below b
// receives the j-th kept slot at or above b.  Sources and destinations are
// disjoint, so the copies need no order.
//
// A CTA, or a cluster of up to eight, takes a unit.  Weights and positions are
// read once into shared memory as order-preserving 32-bit keys; the b-th
// largest key comes from at most four passes of a radix selection (8 bits each,
// most significant first), whose histograms the CTAs of a cluster add up from
// one another's shared memory.  Then warps count, in slot order, the ties, the
// holes below b and the kept rows behind it, list the latter two, and copy.
// Bound by latency: a handful of barriers and two dependent trips to memory
// against 8 bytes a slot and 344 a moved row.
#include <cuda_runtime.h>

#include "ckv_device.cuh"
#include "q4_params.h"

namespace ckv {

namespace {

constexpr int kBins = 256;

// Order-preserving key of a weight: larger weight, larger key; -0 and +0 are
// one, NaN lies below everything.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// The 32-bit word at this CTA's shared address `addr`, in CTA `rank`.
__device__ __forceinline__ int remote_word(uint32_t addr, uint32_t rank) {
  int v;
  asm volatile(
      "{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.s32 %0, [a];\n\t}"
      : "=r"(v)
      : "r"(addr), "r"(rank)
      : "memory");
  return v;
}
template <bool kCluster>
__device__ __forceinline__ void unit_sync() {
  if (kCluster) {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
  } else {
    __syncthreads();
  }
}

// kCluster: more CTAs than one a unit; kShared: keys and positions fit shared
// memory (else they are read again wherever they are needed).
template <int kThreads, bool kCluster, bool kShared>
__global__ void __launch_bounds__(kThreads) evict_kernel(const __grid_constant__ Q4EvictParams p) {
  constexpr int kWarps = kThreads / 32;
  extern __shared__ uint32_t s_keys[];  // [slice] keys, then [slice] positions (later the lists)
  __shared__ int s_hist[4][kBins];
  __shared__ int s_newest, s_pick[3], s_ties[kWarps], s_holes[kWarps], s_rows[kWarps], s_sums[kBins / 32];
  const uint32_t ranks = kCluster ? p.cluster : 1, rank = kCluster ? cluster_rank() : 0;
  const int unit = blockIdx.x / ranks, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int n = min(max(p.c.lengths[unit], 0), p.c.capacity);
  const int b = p.budgets ? p.budgets[unit] : p.budget;
  if (b < 0 || b >= n) return;  // (for every CTA of the unit)
  const long long base = static_cast<long long>(unit) * p.c.capacity;
  const int32_t* pos = p.c.positions + base;
  const float* wt = p.c.weights + base;
  const int slice = ((n + static_cast<int>(ranks) - 1) / static_cast<int>(ranks) + 31) & ~31;
  const int s0 = min(static_cast<int>(rank) * slice, n), s1 = min(s0 + slice, n);
  int32_t* s_pos = reinterpret_cast<int32_t*>(s_keys + slice);

  for (int i = tid; i < 4 * kBins; i += kThreads) (&s_hist[0][0])[i] = 0;
  if (tid == 0) s_newest = -0x7fffffff - 1;
  __syncthreads();
  int newest = -0x7fffffff - 1;
#pragma unroll 4
  for (int j = s0 + tid; j < s1; j += kThreads) {
    const int at = pos[j];
    newest = max(newest, at);
    if (kShared) {
      s_pos[j - s0] = at;
      s_keys[j - s0] = weight_key(wt[j]);
    }
  }
  newest = __reduce_max_sync(0xffffffffu, newest);
  if (lane == 0) atomicMax(&s_newest, newest);
  unit_sync<kCluster>();
  newest = s_newest;
  if (kCluster)
    for (uint32_t r = 0; r < ranks; ++r) newest = max(newest, remote_word(smem_u32(&s_newest), r));
  auto forced = [&](int at) {
    return at < p.sinks || static_cast<long long>(at) > static_cast<long long>(newest) - p.recent;
  };
  // (the keys of forced slots are put in place in the first pass)
  auto key_at = [&](int j) -> uint32_t {
    if (kShared) return s_keys[j - s0];
    return forced(pos[j]) ? 0xffffffffu : weight_key(wt[j]);
  };

  // ---- threshold: the b-th largest key; `need` slots equal to it are kept
  uint32_t top = 0;
  int need = b;
#pragma unroll 1
  for (int pass = 0; pass < 4; ++pass) {
    const int shift = 24 - 8 * pass;
    const uint32_t mask = pass == 0 ? 0u : 0xffffffffu << (shift + 8);
#pragma unroll 4
    for (int j = s0 + tid; j < s1; j += kThreads) {
      uint32_t k;
      if (kShared && pass == 0) {
        k = forced(s_pos[j - s0]) ? 0xffffffffu : s_keys[j - s0];
        s_keys[j - s0] = k;
      } else {
        k = key_at(j);
      }
      if ((k & mask) == top) atomicAdd(&s_hist[pass][(k >> shift) & 255u], 1);
    }
    unit_sync<kCluster>();
    // threads 0.. take the bins from the largest down
    int count = 0, incl = 0;
    if (tid < kBins) {
      const int bin = kBins - 1 - tid;
      if (kCluster) {
        for (uint32_t r = 0; r < ranks; ++r) count += remote_word(smem_u32(&s_hist[pass][bin]), r);
      } else {
        count = s_hist[pass][bin];
      }
      incl = count;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
      }
      if (lane == 31) s_sums[warp] = incl;
    }
    __syncthreads();
    if (tid < kBins) {
      for (int w = 0; w < warp; ++w) incl += s_sums[w];
      // need = 0 takes the first bin
      if ((incl - count < need && need <= incl) || (need == 0 && tid == 0)) {
        s_pick[0] = kBins - 1 - tid;
        s_pick[1] = need - (incl - count);
        s_pick[2] = count;
      }
    }
    __syncthreads();
    top |= static_cast<uint32_t>(s_pick[0]) << shift;
    need = s_pick[1];
    if (need == s_pick[2] && top != 0) {  // the whole bin is kept
      top -= 1;
      need = 0;
      break;
    }
    __syncthreads();
  }

  // ---- ranks in slot order: warps take neighbouring runs of slots
  const int run = ((s1 - s0 + kWarps - 1) / kWarps + 31) & ~31;
  const int w0 = min(s0 + warp * run, s1), w1 = min(w0 + run, s1);
  // counts of the warps before this one, in this CTA and the ones before it
  auto before = [&](const int (&counts)[kWarps]) {
    int sum = lane < warp ? counts[lane] : 0;
    if (kCluster && lane < kWarps)
      for (uint32_t r = 0; r + 1 <= rank; ++r) sum += remote_word(smem_u32(&counts[lane]), r);
    return static_cast<int>(__reduce_add_sync(0xffffffffu, sum));
  };
  int ties = 0;
  if (need > 0) {
    for (int j = w0; j < w1; j += 32)
      ties += __popc(__ballot_sync(0xffffffffu, j + lane < w1 && key_at(j + lane) == top));
    if (lane == 0) s_ties[warp] = ties;
    unit_sync<kCluster>();
    ties = before(s_ties);
  }
  const int first_tie = ties;
  auto kept = [&](int j) {  // of the 32 slots from j, ties counted on
    const uint32_t k = j + lane < w1 ? key_at(j + lane) : 0u;
    bool keep = j + lane < w1 && k > top;
    if (need > 0) {
      const unsigned t = __ballot_sync(0xffffffffu, j + lane < w1 && k == top);
      if (j + lane < w1 && k == top) keep = ties + __popc(t & ((1u << lane) - 1u)) < need;
      ties += __popc(t);
    }
    return keep;
  };
  int holes = 0, rows = 0;
  for (int j = w0; j < w1; j += 32) {
    const bool keep = kept(j);
    holes += __popc(__ballot_sync(0xffffffffu, j + lane < w1 && j + lane < b && !keep));
    rows += __popc(__ballot_sync(0xffffffffu, j + lane >= b && keep));
  }
  if (lane == 0) {
    s_holes[warp] = holes;
    s_rows[warp] = rows;
  }
  unit_sync<kCluster>();  // (and the positions in shared memory are done with)
  holes = before(s_holes);
  rows = before(s_rows);
  ties = first_tie;
  const bool local = kShared && !kCluster;  // the lists have room in place of the positions
  int32_t* to = local ? s_pos : p.lists + base;
  int32_t* from = to + (local ? slice : p.c.capacity) / 2;
  for (int j = w0; j < w1; j += 32) {
    const bool keep = kept(j);
    const unsigned below = (1u << lane) - 1u;
    const bool hole = j + lane < w1 && j + lane < b && !keep, row = j + lane >= b && keep;
    const unsigned hb = __ballot_sync(0xffffffffu, hole), rb = __ballot_sync(0xffffffffu, row);
    if (hole) to[holes + __popc(hb & below)] = j + lane;
    if (row) from[rows + __popc(rb & below)] = j + lane;
    holes += __popc(hb);
    rows += __popc(rb);
  }
  // every hole of the unit: what its last warp has counted
  if (warp == kWarps - 1 && lane == 0) s_pick[0] = holes;
  unit_sync<kCluster>();
  const int moves = kCluster ? remote_word(smem_u32(&s_pick[0]), ranks - 1) : s_pick[0];

  // ---- copies: half a warp a row, 4 + 4 pieces of codes, 1 + 1 of params
  const int l = lane & 15;
  const int part = l < 8 ? l >> 2 : l & 1;
  const bool code = l < 8;
  uint8_t* a = code ? p.c.codes[part] : p.c.params[part];
  const long long bytes = code ? kQ4CodeBytes : kQ4ParamBytes;
  a += base * bytes + (code ? (l & 3) * 16 : 0);
  uint32_t* word = reinterpret_cast<uint32_t*>(p.c.positions) + base;
  if (l == 11) word = reinterpret_cast<uint32_t*>(p.c.weights) + base;
  const int step = static_cast<int>(ranks) * kWarps * 2;
#pragma unroll 2
  for (int i = (static_cast<int>(rank) * kWarps + warp) * 2 + (lane >> 4); i < moves; i += step) {
    const long long dst = to[i], src = from[i];
    if (l < 10) *reinterpret_cast<uint4*>(a + dst * bytes) = *reinterpret_cast<const uint4*>(a + src * bytes);
    else if (l < 12) word[dst] = word[src];
  }
  if (rank == 0 && tid == 0) p.c.lengths[unit] = b;
  if (kCluster) unit_sync<true>();  // no CTA leaves while another reads its words
}

template <int kThreads, bool kCluster, bool kShared>
cudaError_t launch(const Q4EvictParams& p, size_t smem, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(p.c.batch * p.c.num_kv_heads) * p.cluster);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {static_cast<unsigned>(p.cluster), 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = kCluster ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, evict_kernel<kThreads, kCluster, kShared>, p);
}

constexpr size_t kSharedMost = 200 * 1024;  // 25600 slots a CTA

}  // namespace

cudaError_t q4_evict_set_smem_limit() {
  cudaError_t e = cudaSuccess;
  auto set = [&](auto* f) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedMost);
  };
  set(evict_kernel<256, false, true>);
  set(evict_kernel<1024, false, true>);
  set(evict_kernel<1024, true, true>);
  return e;
}

cudaError_t launch_q4_evict(const Q4EvictParams& params, int sms, cudaStream_t stream) {
  Q4EvictParams p = params;
  const long long units = static_cast<long long>(p.c.batch) * p.c.num_kv_heads;
  // long units share the SMs that there are no other units for
  p.cluster = 1;
  while (p.cluster < 8 && units * p.cluster * 2 <= sms && p.c.capacity / p.cluster >= 4096) p.cluster *= 2;
  const int slice = ((p.c.capacity + p.cluster - 1) / p.cluster + 31) & ~31;
  const size_t smem = static_cast<size_t>(slice) * 8;
  if (smem > kSharedMost)
    return p.cluster > 1 ? launch<1024, true, false>(p, 0, stream) : launch<1024, false, false>(p, 0, stream);
  if (p.cluster > 1) return launch<1024, true, true>(p, smem, stream);
  return slice <= 4096 ? launch<256, false, true>(p, smem, stream) : launch<1024, false, true>(p, smem, stream);
}

}  // namespace ckv
