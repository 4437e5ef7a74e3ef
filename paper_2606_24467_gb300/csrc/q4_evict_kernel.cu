// Eviction from the 4-bit cache by accumulated attention weight, in place.
//
// A unit with n slots in use and a budget b < n keeps the b slots with the
// largest (forced, weight), ties to the lower slot; forced are positions below
// `sinks` and the `recent` newest positions.  Slot order means nothing to the
// attention, so only rows move that have to: the j-th evicted slot below b
// receives the j-th kept slot at or above b.  Sources and destinations are
// disjoint, so the copies need no order.
//
// A CTA, or a cluster of up to eight, takes a unit, and every warp a run of
// its slots, whose weights it holds in registers as order-preserving 32-bit
// keys (units beyond 131072 slots are read again for every sweep).  A radix
// selection of 8 bits a pass, whose histograms the CTAs of a cluster add up
// from one another's shared memory, goes on until at most 64 slots can be the
// last one kept: those are ranked by (key, slot) directly, which settles ties
// too.  More equal weights than that are counted in slot order instead.  Then
// the warps count the holes below b and the kept rows behind it, list both in
// slot order, and copy.
// Bound by latency and instructions: a dozen barriers and three dependent trips
// to memory against 8 bytes a slot and 336 a moved row.  Measured: 64 units of
// 1025 slots that lose one 6 us; 2048 units of 1100 to 1200 that lose a tenth 36
// us, where the bytes need 14.8 and the sectors they lie in 21 (the moved rows
// are pieces of 16 and 64 bytes all over the cache).
#include <cuda_runtime.h>

#include "ckv_device.cuh"
#include "q4_params.h"

namespace ckv {

namespace {

constexpr int kBins = 256;
constexpr int kRanked = 64;  // slots that are ranked directly
constexpr int kItems = 16;   // keys a lane holds at most
constexpr int kShortItems = 5;  // ... in CTAs for short units

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

__device__ __forceinline__ int4 remote_words(uint32_t addr, uint32_t rank) {
  int4 v;
  asm volatile(
      "{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %4, %5;\n\t"
      "ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [a];\n\t}"
      : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
      : "r"(addr), "r"(rank)
      : "memory");
  return v;
}

// kHold: keys a lane holds (0: none, they are read again).
template <int kThreads, int kHold, bool kCluster>
__global__ void __launch_bounds__(kThreads, kHold && kHold <= 8 ? 1536 / kThreads : 1) evict_kernel(const __grid_constant__ Q4EvictParams p) {
  constexpr int kWarps = kThreads / 32;
  constexpr int kHists = kCluster ? 4 : 1;  // one a pass where other CTAs read it
  extern __shared__ int32_t s_lists[];      // a single CTA's holes and rows
  __shared__ __align__(16) int s_hist[kHists][kBins];
  __shared__ uint32_t s_key[kRanked], s_all_key[kCluster ? kRanked : 1];
  __shared__ int s_slot[kRanked], s_all_slot[kCluster ? kRanked : 1], s_ranked, s_newest, s_pick[3];
  __shared__ uint32_t s_last[2];
  __shared__ int s_ties[kWarps], s_holes[kWarps], s_rows[kWarps];
  const uint32_t ranks = kCluster ? p.cluster : 1, rank = kCluster ? cluster_rank() : 0;
  const int unit = blockIdx.x / ranks, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  const long long base = static_cast<long long>(unit) * p.c.capacity;
  const int32_t* pos = p.c.positions + base;
  const float* wt = p.c.weights + base;
  // this warp's run of slots.  Short units are cut by their capacity, so that
  // their loads need not wait for the length.
  constexpr bool kEarly = kHold == kShortItems;
  const int parts = static_cast<int>(ranks) * kWarps;
  const int order = static_cast<int>(rank) * kWarps + warp;
  int run = ((p.c.capacity + parts - 1) / parts + 31) & ~31;
  uint32_t held[kHold ? kHold : 1];
  int at[kHold ? kHold : 1];
  constexpr int kNone = -0x7fffffff - 1;
  int newest = kNone;
  if (kEarly) {
#pragma unroll
    for (int i = 0; i < kHold; ++i) {
      const int j = order * run + 32 * i + lane;
      at[i] = kNone;
      held[i] = 0u;
      if (32 * i < run && j < p.c.capacity) {
        at[i] = pos[j];
        held[i] = __float_as_uint(wt[j]);
      }
    }
  }
  const int n = min(max(p.c.lengths[unit], 0), p.c.capacity);
  const int b = p.budgets ? p.budgets[unit] : p.budget;
  if (b < 0 || b >= n) return;  // (for every CTA of the unit)
  if (!kEarly) run = ((n + parts - 1) / parts + 31) & ~31;
  const int w0 = min(order * run, n), w1 = min(w0 + run, n);

  for (int i = tid; i < kHists * kBins; i += kThreads) (&s_hist[0][0])[i] = 0;
  if (tid == 0) {
    s_newest = kNone;
    s_ranked = 0;
  }
  if (kHold) {
#pragma unroll
    for (int i = 0; i < kHold; ++i) {
      const int j = w0 + 32 * i + lane;
      if (!kEarly) {
        at[i] = kNone;
        held[i] = 0u;
        if (j < w1) {
          at[i] = pos[j];
          held[i] = __float_as_uint(wt[j]);
        }
      } else if (j >= w1) {
        at[i] = kNone;
      }
    }
#pragma unroll
    for (int i = 0; i < kHold; ++i) held[i] = weight_key(__uint_as_float(held[i]));
#pragma unroll
    for (int i = 0; i < kHold; ++i) newest = max(newest, at[i]);
  } else {
    for (int j = w0 + lane; j < w1; j += 32) newest = max(newest, pos[j]);
  }
  __syncthreads();
  newest = __reduce_max_sync(0xffffffffu, newest);
  if (lane == 0) atomicMax(&s_newest, newest);
  unit_sync<kCluster>();
  newest = s_newest;
  if (kCluster)
    for (uint32_t r = 0; r < ranks; ++r) newest = max(newest, remote_word(smem_u32(&s_newest), r));
  auto forced = [&](int at) {
    return at < p.sinks || static_cast<long long>(at) > static_cast<long long>(newest) - p.recent;
  };
  if (kHold) {
#pragma unroll
    for (int i = 0; i < kHold; ++i)
      if (forced(at[i])) held[i] = 0xffffffffu;
  }
  // f(slot, key) for every slot of this lane's share of the run (all lanes of
  // the warp together; slots at or behind w1 are no slots)
  auto sweep = [&](auto&& f) {
    if (kHold) {
#pragma unroll
      for (int i = 0; i < kHold; ++i)
        if (w0 + 32 * i < w1) f(w0 + 32 * i + lane, held[i]);
    } else {
      for (int j0 = w0; j0 < w1; j0 += 32) {
        const int j = j0 + lane;
        f(j, j < w1 ? (forced(pos[j]) ? 0xffffffffu : weight_key(wt[j])) : 0u);
      }
    }
  };

  // ---- the last key kept, and the last slot that is kept with it
  uint32_t top = b == 0 ? 0xffffffffu : 0u;
  int need = b;           // slots to keep of those that start with the bits of `top`
  int last_slot = -1;     // of the slots with key `top`, the last one kept
  bool count_ties = false;
#pragma unroll 1
  for (int pass = 0; pass < 4 && b > 0; ++pass) {
    const int shift = 24 - 8 * pass;
    const uint32_t mask = pass == 0 ? 0u : 0xffffffffu << (shift + 8);
    int* hist = s_hist[kCluster ? pass : 0];
    sweep([&](int j, uint32_t k) {
      const int bin = j < w1 && (k & mask) == top ? static_cast<int>((k >> shift) & 255u) : -1;
      if (pass == 0) {
        // signs and exponents: few bins, so a warp adds each once
        const unsigned same = __match_any_sync(0xffffffffu, bin);
        if (bin >= 0 && lane == __ffs(same) - 1) atomicAdd(&hist[bin], __popc(same));
      } else if (bin >= 0) {
        atomicAdd(&hist[bin], 1);
      }
    });
    unit_sync<kCluster>();
    if (warp == 0) {  // lane l: bins 255 - 8 l and the seven below
      int4 hi = make_int4(0, 0, 0, 0), lo = hi;
      int4* mine = reinterpret_cast<int4*>(hist + kBins - 8 - 8 * lane);
      if (kCluster) {
        for (uint32_t r = 0; r < ranks; ++r) {
          const int4 x = remote_words(smem_u32(mine), r), y = remote_words(smem_u32(mine + 1), r);
          lo.x += x.x; lo.y += x.y; lo.z += x.z; lo.w += x.w;
          hi.x += y.x; hi.y += y.y; hi.z += y.z; hi.w += y.w;
        }
      } else {
        lo = mine[0];
        hi = mine[1];
        mine[0] = mine[1] = make_int4(0, 0, 0, 0);  // for the next pass
      }
      const int count[8] = {hi.w, hi.z, hi.y, hi.x, lo.w, lo.z, lo.y, lo.x};
      int sum = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += count[i];
      int incl = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
      }
      int before = incl - sum;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (before < need && need <= before + count[i]) {
          s_pick[0] = kBins - 1 - (8 * lane + i);
          s_pick[1] = need - before;
          s_pick[2] = count[i];
        }
        before += count[i];
      }
    }
    __syncthreads();
    const int count = s_pick[2];
    top |= static_cast<uint32_t>(s_pick[0]) << shift;
    need = s_pick[1];
    if (need == count && top != 0) {  // the whole bin is kept
      top -= 1;
      last_slot = -1;
      break;
    }
    if (count <= kRanked) {
      // rank the candidates by (key, slot); a cluster's lists are read by all
      const uint32_t prefix = 0xffffffffu << shift;
      sweep([&](int j, uint32_t k) {
        if (j < w1 && (k & prefix) == top) {
          const int i = atomicAdd(&s_ranked, 1);
          s_key[i] = k;
          s_slot[i] = j;
        }
      });
      unit_sync<kCluster>();
      if (kCluster) {  // every candidate of the unit
        int x = tid, r = 0;
        for (; r < static_cast<int>(ranks); ++r) {
          const int m = remote_word(smem_u32(&s_ranked), r);
          if (x < m) break;
          x -= m;
        }
        if (tid < count) {
          s_all_key[tid] = static_cast<uint32_t>(remote_word(smem_u32(&s_key[x]), r));
          s_all_slot[tid] = remote_word(smem_u32(&s_slot[x]), r);
        }
        __syncthreads();
      }
      if (tid < count) {
        const uint32_t* keys = kCluster ? s_all_key : s_key;
        const int* slots = kCluster ? s_all_slot : s_slot;
        const uint32_t key = keys[tid];
        const int slot = slots[tid];
        int larger = 0;
#pragma unroll 8
        for (int c = 0; c < count; ++c) {
          const uint32_t k = keys[c];
          larger += k > key || (k == key && slots[c] < slot);
        }
        if (larger == need - 1) {
          s_last[0] = key;
          s_last[1] = static_cast<uint32_t>(slot);
        }
      }
      __syncthreads();
      top = s_last[0];
      last_slot = static_cast<int>(s_last[1]);
      break;
    }
    count_ties = pass == 3;  // (equal keys, more than are ranked)
    __syncthreads();
  }

  // counts of the warps before this one, in this CTA and the ones before it
  auto before = [&](const int (&counts)[kWarps]) {
    int sum = lane < warp ? counts[lane] : 0;
    if (kCluster && lane < kWarps)
      for (uint32_t r = 0; r + 1 <= rank; ++r) sum += remote_word(smem_u32(&counts[lane]), r);
    return static_cast<int>(__reduce_add_sync(0xffffffffu, sum));
  };
  if (count_ties) {
    int ties = 0;
    sweep([&](int j, uint32_t k) { ties += __popc(__ballot_sync(0xffffffffu, j < w1 && k == top)); });
    if (lane == 0) s_ties[warp] = ties;
    unit_sync<kCluster>();
    ties = before(s_ties);
    // the last tie that is kept is in one warp's run: all before it are kept
    last_slot = 0x7fffffff;
    if (ties >= need) last_slot = -1;
    else
      sweep([&](int j, uint32_t k) {
        const unsigned t = __ballot_sync(0xffffffffu, j < w1 && k == top);
        if (ties < need && ties + __popc(t) >= need)
          last_slot = (j & ~31) + static_cast<int>(__fns(t, 0, need - ties));
        ties += __popc(t);
      });
  }
  auto kept = [&](int j, uint32_t k) { return j < w1 && (k > top || (k == top && j <= last_slot)); };

  // ---- holes and rows in slot order
  int holes = 0, rows = 0;
  sweep([&](int j, uint32_t k) {
    const bool keep = kept(j, k);
    holes += __popc(__ballot_sync(0xffffffffu, j < w1 && j < b && !keep));
    rows += __popc(__ballot_sync(0xffffffffu, j >= b && keep));
  });
  if (lane == 0) {
    s_holes[warp] = holes;
    s_rows[warp] = rows;
  }
  unit_sync<kCluster>();
  holes = before(s_holes);
  rows = before(s_rows);
  int32_t* to = kCluster || !kHold ? p.lists + base : s_lists;
  int32_t* from = to + (kCluster || !kHold ? p.c.capacity / 2 : kThreads * kHold / 2);
  sweep([&](int j, uint32_t k) {
    const bool keep = kept(j, k);
    const unsigned below = (1u << lane) - 1u;
    const bool hole = j < w1 && j < b && !keep, row = j >= b && keep;
    const unsigned hb = __ballot_sync(0xffffffffu, hole), rb = __ballot_sync(0xffffffffu, row);
    if (hole) to[holes + __popc(hb & below)] = j;
    if (row) from[rows + __popc(rb & below)] = j;
    holes += __popc(hb);
    rows += __popc(rb);
  });
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
  for (int i0 = (static_cast<int>(rank) * kWarps + warp) * 2 + (lane >> 4); i0 < moves; i0 += 4 * step) {
    uint4 v[4];
    uint32_t x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i0 + k * step < moves) {
        const long long src = from[i0 + k * step];
        if (l < 10) v[k] = *reinterpret_cast<const uint4*>(a + src * bytes);
        else if (l < 12) x[k] = word[src];
      }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i0 + k * step < moves) {
        const long long dst = to[i0 + k * step];
        if (l < 10) *reinterpret_cast<uint4*>(a + dst * bytes) = v[k];
        else if (l < 12) word[dst] = x[k];
      }
  }
  if (rank == 0 && tid == 0) p.c.lengths[unit] = b;
  if (kCluster) unit_sync<true>();  // no CTA leaves while another reads its words
}

template <int kThreads, int kHold, bool kCluster>
cudaError_t launch(const Q4EvictParams& p, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(p.c.batch * p.c.num_kv_heads) * p.cluster);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kCluster ? 0 : kThreads * kHold * sizeof(int32_t);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {static_cast<unsigned>(p.cluster), 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = kCluster ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, evict_kernel<kThreads, kHold, kCluster>, p);
}

}  // namespace

cudaError_t q4_evict_set_smem_limit() {
  return cudaFuncSetAttribute(evict_kernel<1024, kItems, false>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              1024 * kItems * static_cast<int>(sizeof(int32_t)));
}

cudaError_t launch_q4_evict(const Q4EvictParams& params, int sms, cudaStream_t stream) {
  Q4EvictParams p = params;
  const long long units = static_cast<long long>(p.c.batch) * p.c.num_kv_heads;
  // (All by the capacity: the host does not know the lengths.  256 units of 1100
  // slots that lose 76 take 7.7 us in a cache of 1152 slots each, 23 in one of 16K
  // and 124 in one of 64K.)
  const int cap = p.c.capacity;
  // Long units share the SMs that there are no other units for, and those that
  // no CTA holds: 8 units of 8000, 16000 and 32000 slots 18.4, 19.7 and 24.3 us,
  // and 19.1, 28.5 and 41.0 with clusters only where a CTA cannot hold a unit.
  p.cluster = 1;
  while (p.cluster < 8 && (cap > 1024 * kItems * p.cluster ||
                           (units * p.cluster * 2 <= sms && cap >= 4096 * p.cluster)))
    p.cluster *= 2;
  if (cap > 1024 * kItems * p.cluster) return launch<1024, 0, true>(p, stream);
  if (p.cluster > 1)
    return cap <= 8192 * p.cluster ? launch<1024, 8, true>(p, stream) : launch<1024, kItems, true>(p, stream);
  // The smallest CTA whose lanes hold the unit in few keys, so that an SM holds
  // several: 2048 units of 1025 slots 39 us, and 72 with up to 16 keys a lane; 1024 of
  // 2000 slots 37, and 58 with 256 threads of 16 keys; 512 of 4000 slots 45, and 66
  // with 1024 threads of 16 keys; 512 of 6000 slots 82, and 89.
  if (cap <= 256 * kShortItems) return launch<256, kShortItems, false>(p, stream);
  if (cap <= 512 * kShortItems) return launch<512, kShortItems, false>(p, stream);
  if (cap <= 512 * 8) return launch<512, 8, false>(p, stream);
  if (cap <= 1024 * 8) return launch<1024, 8, false>(p, stream);
  return launch<1024, kItems, false>(p, stream);
}

}  // namespace ckv
