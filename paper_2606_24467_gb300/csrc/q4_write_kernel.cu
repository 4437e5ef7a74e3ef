// Rows of K and V into the 4-bit cache: appended (decode tokens, prompt
// chunks) or gathered by index lists (the retained rows of a compression).
//
// A group of 32 channels x_c becomes 4-bit codes n_c with a bf16 minimum m and
// a bf16 scale s:
//   m = min x, rounded down to bf16;   t = fl32(max x - m)
//   s = the smallest bf16 number with 15 s >= t
//   n_c = rint(fl32(x_c - m) / s), ties to even;   value s n_c + m
// Rounding m down and s up keeps every n_c within 0..15 without a clamp, and
// costs at most 2^-8 of the range.  bf16 holds the range of both 16-bit input
// types; since the codes are taken against the stored m and s, their rounding
// adds no error of its own.  The quotient d / s is exact: with 1/s rounded
// down, d * (1/s) rounded to an integer gives n or, where d / s is at or within
// an ulp above n + 1/2, stays one below; the remainder d - n s (one fused
// multiply-add, exact there) tells, and ties then go to the even code.  About
// every other row of bf16 numbers has a tie, so they are put right in place.
// A group that holds a NaN or an infinity (or whose spread overflows) gets
// s = m = NaN.
//
// Half a warp takes one row of K, the other half the same row of V: 8
// channels a lane, so a group is four lanes.  Minimum and maximum are taken in
// the rows' 16-bit type, two numbers an instruction, and cross lanes together
// as (min, -max).  One pass, bound by memory: 512 bytes read and 160 written a
// row (1184 with the values); long calls give a warp four rows, whose loads are
// in flight together.
#include <cuda_runtime.h>

#include "ckv_device.cuh"
#include "q4_params.h"

namespace ckv {

namespace {

constexpr int kWriteThreads = 256;
constexpr int kSmallRows = 64;  // appends of up to this many rows a sequence: one CTA a unit

// The two numbers of a word.
template <bool kBf16>
__device__ __forceinline__ float2 word_floats(uint32_t w) {
  if (kBf16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  float2 f;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}"
      : "=f"(f.x), "=f"(f.y)
      : "r"(w));
  return f;
}
template <bool kBf16>
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {
  uint32_t r;
  if (kBf16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Smaller of each half; NaN if either is.
template <bool kBf16>
__device__ __forceinline__ uint32_t min_pair(uint32_t a, uint32_t b) {
  uint32_t r;
  if (kBf16) asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

constexpr float kMagic = 12582912.0f;  // 1.5 * 2^23: adding it rounds to an integer

// Quantises this half-warp's row (8 channels a lane) into the cache row `dst`
// and, where asked for, writes the values it stands for.
template <bool kBf16>
__device__ __forceinline__ void quantise(const Q4Cache& c, int part, long long dst, uint4 raw,
                                         uint16_t* values) {
  const int l = threadIdx.x & 15;
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
  constexpr uint32_t kSign = 0x80008000u;
  uint32_t lo2 = min_pair<kBf16>(min_pair<kBf16>(w[0], w[1]), min_pair<kBf16>(w[2], w[3]));
  uint32_t hi2 = min_pair<kBf16>(min_pair<kBf16>(w[0] ^ kSign, w[1] ^ kSign),
                                 min_pair<kBf16>(w[2] ^ kSign, w[3] ^ kSign));
  // (min, -max) of this lane, then of the group's four
  uint32_t both = min_pair<kBf16>(__byte_perm(lo2, hi2, 0x5410), __byte_perm(lo2, hi2, 0x7632));
  both = min_pair<kBf16>(both, __shfl_xor_sync(0xffffffffu, both, 1));
  both = min_pair<kBf16>(both, __shfl_xor_sync(0xffffffffu, both, 2));
  const float2 ends = word_floats<kBf16>(both);
  const float lo = ends.x, hi = -ends.y;
  uint32_t mb = __float_as_uint(lo) & 0xffff0000u;
  if (!kBf16 && lo < 0.f && mb != __float_as_uint(lo)) mb += 0x10000u;  // away from zero: down
  float m = __uint_as_float(mb);
  const float spread = hi - m;
  float s = __uint_as_float(__float_as_uint(spread * (1.0f / 15.0f)) & 0xffff0000u);
  // the truncated quotient is at most two bf16 steps below the scale
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (15.0f * s < spread) s = __uint_as_float(__float_as_uint(s) + 0x10000u);
  const bool bad = !(spread <= 3.4028235e38f);  // NaN, infinite
  if (bad) s = m = __uint_as_float(0x7fc00000u);
  // the smallest scales are lifted by 2^64 (exact), so that 1 / s is finite
  const float lift = s < 8.67e-19f ? 18446744073709551616.0f : 1.0f;
  const float sl = s * lift, half = 0.5f * sl;
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(sl));
  inv *= 1.0f - 0x1p-22f;  // (rcp is within 2^-23: now below 1 / s)
  float t[8], r[8], most = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 x = word_floats<kBf16>(w[i >> 1]);
    const float d = ((i & 1 ? x.y : x.x) - m) * lift;
    t[i] = fmaf(d, inv, kMagic);
    r[i] = fmaf(kMagic - t[i], sl, d);
    most = fmaxf(most, r[i]);
  }
  if (most >= half) {
    const float above = __uint_as_float(__float_as_uint(half) + 1u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t n = __float_as_uint(t[i]);
      if (r[i] >= (n & 1u ? half : above)) t[i] = __uint_as_float(n + 1u);
    }
  }
  uint32_t code = 0;
  float val[8];
#pragma unroll
  for (int i = 7; i >= 0; --i) {
    code = (code << 4) + __float_as_uint(t[i]);
    val[i] = fmaf(t[i] - kMagic, s, m);
  }
  code -= 0x4b400000u * 0x11111111u;  // each t has the bits of kMagic above its code
  if (!(s > 0.f)) {  // one value, or NaN
    code = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) val[i] = m;
  }
  reinterpret_cast<uint32_t*>(c.codes[part] + dst * kQ4CodeBytes)[l] = code;
  if ((l & 3) == 0) {
    uint16_t* pr = reinterpret_cast<uint16_t*>(c.params[part] + dst * kQ4ParamBytes);
    pr[l >> 2] = static_cast<uint16_t>(__float_as_uint(s) >> 16);
    pr[kQ4Groups + (l >> 2)] = static_cast<uint16_t>(__float_as_uint(m) >> 16);
  }
  if (values) {
    uint4 o;
    o.x = pack_pair<kBf16>(val[0], val[1]);
    o.y = pack_pair<kBf16>(val[2], val[3]);
    o.z = pack_pair<kBf16>(val[4], val[5]);
    o.w = pack_pair<kBf16>(val[6], val[7]);
    reinterpret_cast<uint4*>(values)[l] = o;
  }
}

// First row of sequence s, and its number of rows.
__device__ __forceinline__ int2 rows_of(const Q4AppendParams& p, int s) {
  if (p.rows_per_seq >= 0) return make_int2(s * p.rows_per_seq, p.rows_per_seq);
  return make_int2(p.cu_rows[s], p.cu_rows[s + 1] - p.cu_rows[s]);
}

// This lane's 16 bytes of a source row, and the row into the cache.
template <int kTable>
__device__ __forceinline__ uint4 load_row(const Q4WriteParams<kTable>& p, long long row, int g) {
  const uint16_t* src = p.src[(threadIdx.x >> 4) & 1] + row * p.tok_stride + static_cast<long long>(g) * p.head_stride;
  return __ldg(reinterpret_cast<const uint4*>(src) + (threadIdx.x & 15));
}
template <bool kBf16, int kTable>
__device__ __forceinline__ void store_row(const Q4WriteParams<kTable>& p, uint4 raw, long long dst,
                                          long long value_row, int position, float weight) {
  const int lane = threadIdx.x & 31, part = lane >> 4;
  quantise<kBf16>(p.c, part, dst, raw, p.values[part] ? p.values[part] + value_row * kHeadDim : nullptr);
  if (lane == 0) p.c.positions[dst] = position;
  if (lane == 16 && p.c.weights) p.c.weights[dst] = weight;
}

// The slot from which a unit's rows go, or -1 where it is outside the unit.
__device__ __forceinline__ int first_slot(const Q4AppendParams& p, int unit) {
  const int at = p.start ? p.start[unit] : p.c.lengths[unit];
  return at >= 0 && at <= p.c.capacity ? at : -1;
}

// Length of a unit after `used` rows from slot `at`, as far as there is room.
__device__ __forceinline__ void set_length(const Q4AppendParams& p, int unit, int at, int used) {
  if (at < 0 || used > p.c.capacity - at) {
    if (p.status) atomicCAS(p.status, 0, CKV_DEV_ERR_INDEX);
    if (at < 0) return;
    used = p.c.capacity - at;
  }
  p.c.lengths[unit] = at + used;
}

// Few rows a sequence: a CTA takes a unit, so the length can be read by all
// of its warps and then be written.  A warp's first row is loaded before it is
// known where it goes.
template <bool kBf16>
__global__ void __launch_bounds__(kWriteThreads) append_unit_kernel(const __grid_constant__ Q4AppendParams p) {
  const int unit = blockIdx.x;
  const int s = unit / p.c.num_kv_heads, g = unit - s * p.c.num_kv_heads;
  const int2 r = rows_of(p, s);
  const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5, lane = threadIdx.x & 31;
  uint4 raw = make_uint4(0u, 0u, 0u, 0u);
  if (warp < r.y) raw = load_row(p, r.x + warp, g);
  const int at = first_slot(p, unit);
  int used = r.y;  // rows before the first negative position
  for (int i = 0; i < r.y; i += 32) {
    const unsigned pad = __ballot_sync(0xffffffffu, i + lane < r.y && p.positions[r.x + i + lane] < 0);
    if (pad) {
      used = i + __ffs(pad) - 1;
      break;
    }
  }
  const long long base = static_cast<long long>(unit) * p.c.capacity;
  if (at >= 0)
    for (int i = warp; i < used && i < p.c.capacity - at; i += warps) {
      if (i != warp) raw = load_row(p, r.x + i, g);
      store_row<kBf16>(p, raw, base + at + i, static_cast<long long>(r.x + i) * p.c.num_kv_heads + g,
                       p.positions[r.x + i], 0.f);
    }
  __syncthreads();
  if (threadIdx.x == 0) set_length(p, unit, at, used);
}

// Many rows: a warp takes kRows neighbouring (row, group) pairs, all their
// loads first; the lengths follow in a launch of their own.
template <bool kBf16, int kRows>
__global__ void __launch_bounds__(kWriteThreads) append_rows_kernel(const __grid_constant__ Q4AppendParams p) {
  pdl_launch_dependents();
  const int H = p.c.num_kv_heads;
  const long long tasks = static_cast<long long>(p.rows) * H;
  const long long task0 = (static_cast<long long>(blockIdx.x) * (kWriteThreads / 32) + (threadIdx.x >> 5)) * kRows;
  if (task0 >= tasks) return;
  int row = static_cast<int>(task0 / H), g = static_cast<int>(task0 - static_cast<long long>(row) * H);
  int s;
  if (p.rows_per_seq >= 0) {
    s = row / p.rows_per_seq;
  } else {
    int lo = 0, hi = p.c.batch;  // cu_rows[s] <= row < cu_rows[s + 1]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (p.cu_rows[mid] <= row) lo = mid; else hi = mid;
    }
    s = lo;
  }
  int2 r = rows_of(p, s);
  uint4 raw[kRows];
  long long dst[kRows];
  int at[kRows], position[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    dst[k] = -1;
    if (task0 + k < tasks) {
      raw[k] = load_row(p, row, g);
      at[k] = first_slot(p, s * H + g);
      position[k] = p.positions[row];
      const int i = row - r.x;
      if (at[k] >= 0 && i < p.c.capacity - at[k] && position[k] >= 0)
        dst[k] = static_cast<long long>(s * H + g) * p.c.capacity + at[k] + i;
      if (++g == H) {
        g = 0;
        ++row;
        while (row >= r.x + r.y && s + 1 < p.c.batch) r = rows_of(p, ++s);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < kRows; ++k)
    if (dst[k] >= 0) store_row<kBf16>(p, raw[k], dst[k], task0 + k, position[k], 0.f);
}

// A CTA a sequence: the first of its rows with a negative position.
__global__ void __launch_bounds__(kWriteThreads) append_lengths_kernel(const __grid_constant__ Q4AppendParams p) {
  __shared__ int s_used;
  const int s = blockIdx.x, H = p.c.num_kv_heads;
  const int2 r = rows_of(p, s);
  if (threadIdx.x == 0) s_used = r.y;
  __syncthreads();
  int used = r.y;
#pragma unroll 4
  for (int i = threadIdx.x; i < r.y; i += kWriteThreads)
    if (p.positions[r.x + i] < 0) used = min(used, i);
  if (used < r.y) atomicMin(&s_used, used);
  __syncthreads();
  pdl_wait();  // the rows' kernel has read the lengths
  for (int g = threadIdx.x; g < H; g += kWriteThreads)
    set_length(p, s * H + g, first_slot(p, s * H + g), s_used);
}

// A warp takes kRows neighbouring retained rows and groups; further warps
// write the units' lengths.
template <bool kBf16, int kRows, class P>
__global__ void __launch_bounds__(kWriteThreads) gather_q4_kernel(const __grid_constant__ P p) {
  const int H = p.c.num_kv_heads, B = p.c.batch, lane = threadIdx.x & 31;
  const long long tasks = p.group_major ? p.rows : static_cast<long long>(p.rows) * H;
  const long long warps = (tasks + kRows - 1) / kRows;
  const long long warp = static_cast<long long>(blockIdx.x) * (kWriteThreads / 32) + (threadIdx.x >> 5);
  if (warp >= warps) {
    const long long unit = (warp - warps) * 32 + lane;
    if (unit < static_cast<long long>(B) * H) {
      const int s = static_cast<int>(unit / H), g = static_cast<int>(unit - static_cast<long long>(s) * H);
      const int* cu = p.cu_rows + (p.group_major ? g * (B + 1) : 0);
      p.c.lengths[unit] = cu[s + 1] - cu[s];
    }
    return;
  }
  const long long task0 = warp * kRows;
  int row, g;
  if (p.group_major) {
    row = static_cast<int>(task0);
    g = 0;
    while (g + 1 < H && p.cu_rows[(g + 1) * (B + 1)] <= row) ++g;
  } else {
    row = static_cast<int>(task0 / H);
    g = static_cast<int>(task0 - static_cast<long long>(row) * H);
  }
  const int* cu = p.cu_rows + (p.group_major ? g * (B + 1) : 0);
  int lo = 0, hi = B;  // cu[s] <= row < cu[s + 1]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] <= row) lo = mid; else hi = mid;
  }
  int s = lo;
  int idx[kRows];
  long long at[kRows];  // of the row in K, V; -1: an index outside
  long long dst[kRows];
  int head[kRows], seq[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    at[k] = -1;
    if (task0 + k < tasks) {
      idx[k] = p.indices[p.group_major ? row : static_cast<long long>(g) * p.rows + row];
      dst[k] = static_cast<long long>(s * H + g) * p.c.capacity + (row - cu[s]);
      head[k] = g;
      seq[k] = s;
      at[k] = p.cu_seqlens[s];
      // the next pair
      if (p.group_major || ++g == H) {
        ++row;
        if (!p.group_major) g = 0;
        while (row >= cu[s + 1]) {
          if (s + 1 < B) {
            ++s;
          } else if (p.group_major && g + 1 < H) {
            ++g;
            cu += B + 1;
            s = 0;
          } else {
            break;
          }
        }
      }
    }
  }
  uint4 raw[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k)
    if (at[k] >= 0) {
      const int L = p.cu_seqlens[seq[k] + 1] - p.cu_seqlens[seq[k]];
      if (idx[k] < 0 || idx[k] >= L) {
        if (lane == 0 && p.status) atomicCAS(p.status, 0, CKV_DEV_ERR_INDEX);
        at[k] = -1;
      } else {
        raw[k] = load_row(p, at[k] + idx[k], head[k]);
      }
    }
#pragma unroll
  for (int k = 0; k < kRows; ++k)
    if (at[k] >= 0) {
      const int L = p.cu_seqlens[seq[k] + 1] - p.cu_seqlens[seq[k]];
      float weight = 0.f;
      if (p.raw && idx[k] < L - p.window)
        weight = p.raw[static_cast<long long>(head[k]) * p.p_total + p.cu_prefix[seq[k]] + idx[k]];
      store_row<kBf16>(p, raw[k], dst[k], task0 + k, idx[k], weight);
    }
}

// Rows a warp takes: four once every SM has more warps than it holds at once.
constexpr long long kManyTasks = 152 * 64;

template <bool kBf16, int kRows, class P>
cudaError_t launch_gather_rows(const P& p, long long tasks, cudaStream_t stream) {
  const long long units = static_cast<long long>(p.c.batch) * p.c.num_kv_heads;
  const long long warps = (tasks + kRows - 1) / kRows + (units + 31) / 32;
  constexpr int kPer = kWriteThreads / 32;
  gather_q4_kernel<kBf16, kRows, P><<<static_cast<unsigned>((warps + kPer - 1) / kPer), kWriteThreads, 0, stream>>>(p);
  return cudaGetLastError();
}
template <class P>
cudaError_t launch_gather_any(const P& p, cudaStream_t stream) {
  const long long tasks = p.group_major ? p.rows : static_cast<long long>(p.rows) * p.c.num_kv_heads;
  if (tasks <= kManyTasks)
    return p.is_bf16 ? launch_gather_rows<true, 1>(p, tasks, stream) : launch_gather_rows<false, 1>(p, tasks, stream);
  return p.is_bf16 ? launch_gather_rows<true, 4>(p, tasks, stream) : launch_gather_rows<false, 4>(p, tasks, stream);
}

template <bool kBf16, int kRows>
cudaError_t launch_append_rows(const Q4AppendParams& p, long long tasks, cudaStream_t stream) {
  constexpr long long kPer = static_cast<long long>(kWriteThreads / 32) * kRows;
  append_rows_kernel<kBf16, kRows>
      <<<static_cast<unsigned>((tasks + kPer - 1) / kPer), kWriteThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_q4_append(const Q4AppendParams& p, int max_rows, cudaStream_t stream) {
  const int units = p.c.batch * p.c.num_kv_heads;
  if (max_rows <= kSmallRows) {
    constexpr int kMost = kWriteThreads / 32;
    const int warps = max_rows < 1 ? 1 : max_rows < kMost ? max_rows : kMost;
    if (p.is_bf16) append_unit_kernel<true><<<units, warps * 32, 0, stream>>>(p);
    else append_unit_kernel<false><<<units, warps * 32, 0, stream>>>(p);
    return cudaGetLastError();
  }
  const long long tasks = static_cast<long long>(p.rows) * p.c.num_kv_heads;
  cudaError_t e;
  if (tasks <= kManyTasks)
    e = p.is_bf16 ? launch_append_rows<true, 1>(p, tasks, stream) : launch_append_rows<false, 1>(p, tasks, stream);
  else
    e = p.is_bf16 ? launch_append_rows<true, 4>(p, tasks, stream) : launch_append_rows<false, 4>(p, tasks, stream);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.c.batch);
  cfg.blockDim = dim3(kWriteThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, append_lengths_kernel, p);
}

cudaError_t launch_q4_gather(const Q4GatherParams& p, cudaStream_t stream) {
  return launch_gather_any(p, stream);
}
cudaError_t launch_q4_gather(const Q4GatherUnitParams& p, cudaStream_t stream) {
  return launch_gather_any(p, stream);
}

}  // namespace ckv
