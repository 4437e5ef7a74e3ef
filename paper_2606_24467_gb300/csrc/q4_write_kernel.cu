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
// adds no error of its own.  The quotient is exact: d * (1/s) is rounded to an
// integer n, and the remainder d - n s (one fused multiply-add, exact near a
// tie) decides where it lies within an ulp of a tie.
// A group that holds a NaN or an infinity (or whose spread overflows) gets
// s = m = NaN.
//
// Half a warp takes one row of K, the other half the same row of V: 8
// channels a lane, so a group is four lanes and two shuffle steps.  One pass,
// bound by memory: 512 bytes read and 160 written a row (1184 with the values).
#include <cuda_runtime.h>

#include "ckv_device.cuh"
#include "q4_params.h"

namespace ckv {

namespace {

constexpr int kWriteThreads = 256;
constexpr int kSmallRows = 64;  // appends of up to this many rows a sequence: one CTA a unit

__device__ __forceinline__ float bits_to_float(uint32_t h, bool bf16) {
  if (bf16) return __uint_as_float(h << 16);
  float f;
  asm("{\n\t.reg .b16 t;\n\tcvt.u16.u32 t, %1;\n\tcvt.f32.f16 %0, t;\n\t}" : "=f"(f) : "r"(h));
  return f;
}
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi, bool bf16) {
  uint32_t r;
  if (bf16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Quantises this half-warp's row (8 channels a lane) into the cache row `dst`
// and, where asked for, writes the values it stands for.
__device__ __forceinline__ void quantise_row(const Q4Cache& c, int part, long long dst, uint4 raw,
                                             bool bf16, uint16_t* values) {
  const int l = threadIdx.x & 15;
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
  float x[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = bits_to_float(w[i] & 0xffffu, bf16);
    x[2 * i + 1] = bits_to_float(w[i] >> 16, bf16);
  }
  float lo = x[0], hi = x[0];
  uint32_t top_bits = __float_as_uint(x[0]) & 0x7fffffffu;
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    lo = fminf(lo, x[i]);
    hi = fmaxf(hi, x[i]);
    top_bits = max(top_bits, __float_as_uint(x[i]) & 0x7fffffffu);
  }
#pragma unroll
  for (int o = 1; o <= 2; o <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    top_bits = max(top_bits, __shfl_xor_sync(0xffffffffu, top_bits, o));
  }
  uint32_t mb = __float_as_uint(lo) & 0xffff0000u;
  if (lo < 0.f && mb != __float_as_uint(lo)) mb += 0x10000u;  // away from zero: down
  float m = __uint_as_float(mb);
  const float spread = hi - m;
  float s = __uint_as_float(__float_as_uint(spread * (1.0f / 15.0f)) & 0xffff0000u);
  // the truncated quotient is at most two bf16 steps below the scale
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (15.0f * s < spread) s = __uint_as_float(__float_as_uint(s) + 0x10000u);
  if (top_bits >= 0x7f800000u || !(spread <= 3.4028235e38f)) s = m = __uint_as_float(0x7fc00000u);
  // 1/s of the smallest scales overflows: scale both by 2^64 (exact)
  const float lift = s < 8.67e-19f ? 18446744073709551616.0f : 1.0f;
  const float sl = s * lift, half = 0.5f * sl;
  const float inv = sl > 0.f ? __frcp_rn(sl) : 0.f;
  constexpr float kMagic = 12582912.0f;  // 1.5 * 2^23: adding it rounds to an integer
  uint32_t code = 0;
  float val[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float d = (x[i] - m) * lift;
    float n = fmaf(d, inv, kMagic) - kMagic;
    const float r = fmaf(-n, sl, d);
    if (fabsf(r) >= half) {
      const bool odd = (static_cast<int>(n) & 1) != 0;
      if (fabsf(r) > half || odd) n += r > 0.f ? 1.0f : -1.0f;
    }
    if (!(n >= 0.f)) n = 0.f;  // a group of NaN, or of one value
    code |= static_cast<uint32_t>(n) << (4 * i);
    val[i] = fmaf(n, s, m);
  }
  reinterpret_cast<uint32_t*>(c.codes[part] + dst * kQ4CodeBytes)[l] = code;
  if ((l & 3) == 0) {
    uint16_t* pr = reinterpret_cast<uint16_t*>(c.params[part] + dst * kQ4ParamBytes);
    pr[l >> 2] = static_cast<uint16_t>(__float_as_uint(s) >> 16);
    pr[kQ4Groups + (l >> 2)] = static_cast<uint16_t>(__float_as_uint(m) >> 16);
  }
  if (values) {
    uint4 o;
    o.x = pack_pair(val[0], val[1], bf16);
    o.y = pack_pair(val[2], val[3], bf16);
    o.z = pack_pair(val[4], val[5], bf16);
    o.w = pack_pair(val[6], val[7], bf16);
    reinterpret_cast<uint4*>(values)[l] = o;
  }
}

// First row of sequence s, and its number of rows.
__device__ __forceinline__ int2 rows_of(const Q4AppendParams& p, int s) {
  if (p.rows_per_seq >= 0) return make_int2(s * p.rows_per_seq, p.rows_per_seq);
  return make_int2(p.cu_rows[s], p.cu_rows[s + 1] - p.cu_rows[s]);
}

// One row of one unit.
__device__ __forceinline__ void append_row(const Q4AppendParams& p, int s, int g, int row, int slot) {
  const int lane = threadIdx.x & 31, part = lane >> 4;
  const uint16_t* src = p.src[part] + static_cast<long long>(row) * p.tok_stride +
                        static_cast<long long>(g) * p.head_stride;
  const uint4 raw = __ldg(reinterpret_cast<const uint4*>(src) + (lane & 15));
  const long long dst =
      static_cast<long long>(s * p.c.num_kv_heads + g) * p.c.capacity + slot;
  uint16_t* values =
      p.values[part] ? p.values[part] + (static_cast<long long>(row) * p.c.num_kv_heads + g) * kHeadDim
                     : nullptr;
  quantise_row(p.c, part, dst, raw, p.is_bf16 != 0, values);
  if (lane == 0) p.c.positions[dst] = p.positions[row];
  if (lane == 16 && p.c.weights) p.c.weights[dst] = 0.f;
}

// The slot from which a unit's rows go, or -1 where it is outside the unit.
__device__ __forceinline__ int first_slot(const Q4AppendParams& p, int unit) {
  const int at = p.start ? p.start[unit] : p.c.lengths[unit];
  return at >= 0 && at <= p.c.capacity ? at : -1;
}

// Length of a unit after the call, by one warp: `n` rows from slot `at`, up
// to the first one with a negative position, as far as there is room.
__device__ __forceinline__ void set_length(const Q4AppendParams& p, int unit, int at, int row, int n) {
  const int lane = threadIdx.x & 31;
  if (at < 0) {
    if (lane == 0 && p.status) atomicCAS(p.status, 0, CKV_DEV_ERR_INDEX);
    return;
  }
  int used = n;
  for (int i = 0; i < n; i += 32) {
    const unsigned pad =
        __ballot_sync(0xffffffffu, i + lane < n && p.positions[row + i + lane] < 0);
    if (pad) {
      used = i + __ffs(pad) - 1;
      break;
    }
  }
  if (lane == 0) {
    if (used > p.c.capacity - at) {
      used = p.c.capacity - at;
      if (p.status) atomicCAS(p.status, 0, CKV_DEV_ERR_INDEX);
    }
    p.c.lengths[unit] = at + used;
  }
}

// Few rows a sequence: a CTA takes a unit, so the length can be read by all
// of its warps and then be written.
__global__ void __launch_bounds__(kWriteThreads) append_unit_kernel(const __grid_constant__ Q4AppendParams p) {
  const int unit = blockIdx.x;
  const int s = unit / p.c.num_kv_heads, g = unit - s * p.c.num_kv_heads;
  const int2 r = rows_of(p, s);
  const int at = first_slot(p, unit);
  const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  if (at >= 0)
    for (int i = warp; i < r.y && i < p.c.capacity - at; i += warps)
      if (p.positions[r.x + i] >= 0) append_row(p, s, g, r.x + i, at + i);
  __syncthreads();
  if (warp == 0) set_length(p, unit, at, r.x, r.y);
}

// Many rows: a warp a row and group; the lengths follow in a launch of their own.
__global__ void __launch_bounds__(kWriteThreads) append_rows_kernel(const __grid_constant__ Q4AppendParams p) {
  const long long task = static_cast<long long>(blockIdx.x) * (kWriteThreads / 32) + (threadIdx.x >> 5);
  if (task >= static_cast<long long>(p.rows) * p.c.num_kv_heads) return;
  const int row = static_cast<int>(task / p.c.num_kv_heads);
  const int g = static_cast<int>(task - static_cast<long long>(row) * p.c.num_kv_heads);
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
  const int at = first_slot(p, s * p.c.num_kv_heads + g);
  const int i = row - rows_of(p, s).x;
  if (at < 0 || i >= p.c.capacity - at || p.positions[row] < 0) return;
  append_row(p, s, g, row, at + i);
}

__global__ void __launch_bounds__(kWriteThreads) append_lengths_kernel(const __grid_constant__ Q4AppendParams p) {
  const int unit = blockIdx.x * (kWriteThreads / 32) + (threadIdx.x >> 5);
  if (unit >= p.c.batch * p.c.num_kv_heads) return;
  const int2 r = rows_of(p, unit / p.c.num_kv_heads);
  set_length(p, unit, first_slot(p, unit), r.x, r.y);
}

// A warp a retained row and group, and one for each unit's length.
template <class P>
__global__ void __launch_bounds__(kWriteThreads) gather_q4_kernel(const __grid_constant__ P p) {
  const int H = p.c.num_kv_heads, B = p.c.batch, lane = threadIdx.x & 31;
  const long long rows = p.group_major ? p.rows : static_cast<long long>(p.rows) * H;
  const long long task = static_cast<long long>(blockIdx.x) * (kWriteThreads / 32) + (threadIdx.x >> 5);
  if (task >= rows) {
    const long long unit = task - rows;
    if (unit < static_cast<long long>(B) * H && lane == 0) {
      const int s = static_cast<int>(unit / H), g = static_cast<int>(unit - static_cast<long long>(s) * H);
      const int* cu = p.cu_rows + (p.group_major ? g * (B + 1) : 0);
      p.c.lengths[unit] = cu[s + 1] - cu[s];
    }
    return;
  }
  int row, g;
  if (p.group_major) {
    row = static_cast<int>(task);
    g = 0;
    while (g + 1 < H && p.cu_rows[(g + 1) * (B + 1)] <= row) ++g;
  } else {
    row = static_cast<int>(task / H);
    g = static_cast<int>(task - static_cast<long long>(row) * H);
  }
  const int* cu = p.cu_rows + (p.group_major ? g * (B + 1) : 0);
  int lo = 0, hi = B;  // cu[s] <= row < cu[s + 1]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] <= row) lo = mid; else hi = mid;
  }
  const int s = lo, L = p.cu_seqlens[s + 1] - p.cu_seqlens[s];
  const int idx = p.indices[p.group_major ? row : static_cast<long long>(g) * p.rows + row];
  if (idx < 0 || idx >= L) {
    if (lane == 0 && p.status) atomicCAS(p.status, 0, CKV_DEV_ERR_INDEX);
    return;
  }
  const int part = lane >> 4;
  const uint16_t* src = p.src[part] + static_cast<long long>(p.cu_seqlens[s] + idx) * p.tok_stride +
                        static_cast<long long>(g) * p.head_stride;
  const uint4 raw = __ldg(reinterpret_cast<const uint4*>(src) + (lane & 15));
  const long long dst = static_cast<long long>(s * H + g) * p.c.capacity + (row - cu[s]);
  quantise_row(p.c, part, dst, raw, p.is_bf16 != 0,
               p.values[part] ? p.values[part] + task * kHeadDim : nullptr);
  if (lane == 0) p.c.positions[dst] = idx;
  if (lane == 16 && p.c.weights)
    p.c.weights[dst] = p.raw && idx < L - p.window
                           ? p.raw[static_cast<long long>(g) * p.p_total + p.cu_prefix[s] + idx]
                           : 0.f;
}

template <class P>
cudaError_t launch_gather_any(const P& p, cudaStream_t stream) {
  const long long units = static_cast<long long>(p.c.batch) * p.c.num_kv_heads;
  const long long tasks = units + (p.group_major ? p.rows : static_cast<long long>(p.rows) * p.c.num_kv_heads);
  constexpr int kPer = kWriteThreads / 32;
  gather_q4_kernel<<<static_cast<unsigned>((tasks + kPer - 1) / kPer), kWriteThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_q4_append(const Q4AppendParams& p, int max_rows, cudaStream_t stream) {
  const int units = p.c.batch * p.c.num_kv_heads;
  constexpr int kPer = kWriteThreads / 32;
  if (max_rows <= kSmallRows) {
    const int warps = max_rows < 1 ? 1 : max_rows < kPer ? max_rows : kPer;
    append_unit_kernel<<<units, warps * 32, 0, stream>>>(p);
    return cudaGetLastError();
  }
  const long long tasks = static_cast<long long>(p.rows) * p.c.num_kv_heads;
  append_rows_kernel<<<static_cast<unsigned>((tasks + kPer - 1) / kPer), kWriteThreads, 0, stream>>>(p);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  append_lengths_kernel<<<(units + kPer - 1) / kPer, kWriteThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_q4_gather(const Q4GatherParams& p, cudaStream_t stream) {
  return launch_gather_any(p, stream);
}
cudaError_t launch_q4_gather(const Q4GatherUnitParams& p, cudaStream_t stream) {
  return launch_gather_any(p, stream);
}

}  // namespace ckv
