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
// as (min, -max).  One pass: 512 bytes read and 160 written a row (1184 with the
// values); long calls give a warp four rows, whose loads are in flight together.
// Measured, with the values: the retained rows of 32 layers (256 units of 917 of
// 32768 rows) 62.7 us, 4.5 TB/s of the 6.78 that a copy reaches; 8191 rows of 4
// heads appended 11.3 us, where the bytes need 5.8 (two launches).  Bound by
// instructions: 212 a row of K and V, issued in 66 % of the cycles.
#include <cuda_runtime.h>

#include "ckv_device.cuh"
#include "q4_params.h"

namespace ckv {

namespace {

constexpr int kWriteThreads = 256;
// Appends of up to this many rows a sequence take one launch, a CTA a unit;
// longer ones one for the rows and one for the lengths.  One sequence of 16, 32
// and 64 rows: 2.6, 3.8 and 6.6 us against 3.3, 3.2 and 3.4; sixteen: 2.7, 3.9
// and 6.6 against 3.7, 4.1 and 5.5; sixty-four: 4.0, 6.4 and 11.1 against 5.5,
// 7.1 and 10.3.
constexpr int kSmallRows = 32;

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

// Two fp32 operations an instruction.
__device__ __forceinline__ float2 both2(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
      "add.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

constexpr float kMagic = 12582912.0f;  // 1.5 * 2^23: adding it rounds to an integer

// Quantises this half-warp's row (8 channels a lane) into the cache row `dst`
// and, where asked for, writes the values it stands for.
template <bool kBf16>
__device__ __forceinline__ void quantise(const Q4Cache& c, int part, int dst, uint4 raw,
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
  const float half = 0.5f * s;
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
  inv *= 1.0f - 0x1p-22f;  // (rcp is within 2^-23: now below 1 / s)
  float2 t[4], r[4], val[4];
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 d = add2(word_floats<kBf16>(w[i]), both2(-m));
    t[i] = fma2(d, both2(inv), both2(kMagic));
    const float2 minus_n = fma2(t[i], both2(-1.0f), both2(kMagic));
    r[i] = fma2(minus_n, both2(s), d);
    val[i] = fma2(minus_n, both2(-s), both2(m));
    most = fmaxf(most, fmaxf(r[i].x, r[i].y));
  }
  if (s < 8.67e-19f && s > 0.f) {  // 1 / s may not be finite: all times 2^64 (exact)
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s * 0x1p64f));
    inv *= 1.0f - 0x1p-22f;
    most = half;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 d = add2(word_floats<kBf16>(w[i]), both2(-m));
      t[i] = make_float2(fmaf(d.x * 0x1p64f, inv, kMagic), fmaf(d.y * 0x1p64f, inv, kMagic));
      r[i] = make_float2(fmaf(kMagic - t[i].x, s, d.x), fmaf(kMagic - t[i].y, s, d.y));
    }
  }
  if (most >= half) {
    // above a tie, or a tie of an odd code (numbers >= 0 compare like their bits)
    auto put = [&](float& t, float r) {
      const int n = __float_as_int(t);
      if (__float_as_int(r) + (n & 1) > __float_as_int(half)) t = __int_as_float(n + 1);
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      put(t[i].x, r[i].x);
      put(t[i].y, r[i].y);
      val[i] = fma2(add2(t[i], both2(-kMagic)), both2(s), both2(m));
    }
  }
  uint32_t code = 0;
#pragma unroll
  for (int i = 3; i >= 0; --i) {
    code = (code << 4) + __float_as_uint(t[i].y);
    code = (code << 4) + __float_as_uint(t[i].x);
  }
  code -= 0x4b400000u * 0x11111111u;  // each t has the bits of kMagic above its code
  if (!(s > 0.f)) {  // one value, or NaN
    code = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) val[i] = both2(m);
  }
  reinterpret_cast<uint32_t*>(c.codes[part] + static_cast<size_t>(dst) * kQ4CodeBytes)[l] = code;
  if ((l & 3) == 0) {
    uint16_t* pr = reinterpret_cast<uint16_t*>(c.params[part] + static_cast<size_t>(dst) * kQ4ParamBytes);
    pr[l >> 2] = static_cast<uint16_t>(__float_as_uint(s) >> 16);
    pr[kQ4Groups + (l >> 2)] = static_cast<uint16_t>(__float_as_uint(m) >> 16);
  }
  if (values) {
    uint4 o;
    o.x = pack_pair<kBf16>(val[0].x, val[0].y);
    o.y = pack_pair<kBf16>(val[1].x, val[1].y);
    o.z = pack_pair<kBf16>(val[2].x, val[2].y);
    o.w = pack_pair<kBf16>(val[3].x, val[3].y);
    reinterpret_cast<uint4*>(values)[l] = o;
  }
}

// First row of sequence s, and its number of rows.
__device__ __forceinline__ int2 rows_of(const Q4AppendParams& p, int s) {
  if (p.rows_per_seq >= 0) return make_int2(s * p.rows_per_seq, p.rows_per_seq);
  return make_int2(p.cu_rows[s], p.cu_rows[s + 1] - p.cu_rows[s]);
}

// This lane's 16 bytes of a source row, and the row into the cache.  (An
// ordinary load: a gather that lets its successor start early may write the row.)
template <int kTable>
__device__ __forceinline__ uint4 load_row(const Q4WriteParams<kTable>& p, int row, int g) {
  const uint16_t* src = p.src[(threadIdx.x >> 4) & 1] + row * p.tok_stride + g * p.head_stride;
  return reinterpret_cast<const uint4*>(src)[threadIdx.x & 15];
}
template <bool kBf16, int kTable>
__device__ __forceinline__ void store_row(const Q4WriteParams<kTable>& p, uint4 raw, int dst, int value_row,
                                          int position, float weight) {
  const int lane = threadIdx.x & 31, part = lane >> 4;
  quantise<kBf16>(p.c, part, dst, raw, p.values[part] ? p.values[part] + static_cast<size_t>(value_row) * kHeadDim : nullptr);
  if (lane == 0) p.c.positions[dst] = position;
  if (lane == 16 && p.c.weights) p.c.weights[dst] = weight;
}

// The slot from which a unit's rows go, or -1 where a given one is outside the
// unit.  (A length outside it counts as the nearer end.)
__device__ __forceinline__ int first_slot(const Q4AppendParams& p, int unit) {
  if (!p.start) return min(max(p.c.lengths[unit], 0), p.c.capacity);
  const int at = p.start[unit];
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
  pdl_wait();
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
  const int base = unit * p.c.capacity;
  if (at >= 0)
    for (int i = warp; i < used && i < p.c.capacity - at; i += warps) {
      if (i != warp) raw = load_row(p, r.x + i, g);
      store_row<kBf16>(p, raw, base + at + i, (r.x + i) * p.c.num_kv_heads + g,
                       p.positions[r.x + i], 0.f);
    }
  __syncthreads();
  if (threadIdx.x == 0) set_length(p, unit, at, used);
}

// Where a lane's row and group come from and go to.
struct Move {
  int row = 0, head = 0;  // of K, V
  int dst = -1;           // slot row of the cache; -1: nothing to do
  int position = 0;
  float weight = 0.f;
};

// The warp's tasks task0 .. task0 + count - 1 (count <= kTasks), whose moves
// its first lanes hold: four rows in flight at a time.
template <bool kBf16, int kTasks, int kTable>
__device__ __forceinline__ void move_rows(const Q4WriteParams<kTable>& p, const Move& mine, int task0) {
  constexpr int kBatch = kTasks < 4 ? kTasks : 4;
  const int lane = threadIdx.x & 31, part = lane >> 4;
  if (lane < kTasks && mine.dst >= 0) {
    p.c.positions[mine.dst] = mine.position;
    if (p.c.weights) p.c.weights[mine.dst] = mine.weight;
  }
#pragma unroll 1
  for (int t = 0; t < kTasks; t += kBatch) {
    uint4 raw[kBatch];
    int dst[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      dst[k] = __shfl_sync(0xffffffffu, mine.dst, t + k);
      const int row = __shfl_sync(0xffffffffu, mine.row, t + k);
      const int head = __shfl_sync(0xffffffffu, mine.head, t + k);
      if (dst[k] >= 0) raw[k] = load_row(p, row, head);
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (dst[k] >= 0)
        quantise<kBf16>(p.c, part, dst[k], raw[k],
                        p.values[part] ? p.values[part] + static_cast<size_t>(task0 + t + k) * kHeadDim : nullptr);
  }
}

// Many rows: a warp takes kTasks neighbouring (row, group) pairs; the lengths
// follow in a launch of their own.
template <bool kBf16, int kTasks>
__global__ void __launch_bounds__(kWriteThreads, 4) append_rows_kernel(const __grid_constant__ Q4AppendParams p) {
  pdl_wait();
  pdl_launch_dependents();  // the lengths' kernel, which waits for this one
  const int H = p.c.num_kv_heads;
  // (the host bounds the tasks by 2^31 - 1, and the slots)
  const unsigned tasks = static_cast<unsigned>(p.rows) * H;
  const unsigned task0 = (blockIdx.x * (kWriteThreads / 32) + (threadIdx.x >> 5)) * kTasks;
  if (task0 >= tasks) return;
  const unsigned task = task0 + (threadIdx.x & 31);
  Move m;
  if ((threadIdx.x & 31) < kTasks && task < tasks) {
    m.row = static_cast<int>(task / H);
    m.head = static_cast<int>(task) - m.row * H;
    int s;
    if (p.rows_per_seq >= 0) {
      s = m.row / p.rows_per_seq;
    } else {
      int lo = 0, hi = p.c.batch;  // cu_rows[s] <= row < cu_rows[s + 1]
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.cu_rows[mid] <= m.row) lo = mid; else hi = mid;
      }
      s = lo;
    }
    const int at = first_slot(p, s * H + m.head), i = m.row - rows_of(p, s).x;
    m.position = p.positions[m.row];
    if (at >= 0 && i < p.c.capacity - at && m.position >= 0) m.dst = (s * H + m.head) * p.c.capacity + at + i;
  }
  move_rows<kBf16, kTasks>(p, m, static_cast<int>(task0));
}

// A CTA a sequence: the first of its rows with a negative position.
constexpr int kLengthThreads = 1024;
__global__ void __launch_bounds__(kLengthThreads) append_lengths_kernel(const __grid_constant__ Q4AppendParams p) {
  pdl_wait();  // the rows' kernel has read the lengths
  __shared__ int s_used;
  const int s = blockIdx.x, H = p.c.num_kv_heads;
  const int2 r = rows_of(p, s);
  if (threadIdx.x == 0) s_used = r.y;
  __syncthreads();
  int used = r.y;
#pragma unroll 8
  for (int i = threadIdx.x; i < r.y; i += kLengthThreads)
    used = p.positions[r.x + i] < 0 ? min(used, i) : used;
  if (used < r.y) atomicMin(&s_used, used);
  __syncthreads();
  for (int g = threadIdx.x; g < H; g += kLengthThreads)
    set_length(p, s * H + g, first_slot(p, s * H + g), s_used);
}

// A warp takes kTasks neighbouring retained rows and groups; further warps
// write the units' lengths.
template <bool kBf16, int kTasks, class P>
__global__ void __launch_bounds__(kWriteThreads, 4) gather_q4_kernel(const __grid_constant__ P p) {
  pdl_wait();
  const int H = p.c.num_kv_heads, B = p.c.batch, lane = threadIdx.x & 31;
  const unsigned tasks = p.group_major ? p.rows : static_cast<unsigned>(p.rows) * H;
  const unsigned warps = (tasks + kTasks - 1) / kTasks;
  const unsigned warp = blockIdx.x * (kWriteThreads / 32) + (threadIdx.x >> 5);
  if (warp >= warps) {
    const int unit = static_cast<int>(warp - warps) * 32 + lane;
    if (unit < B * H) {
      const int s = unit / H, g = unit - s * H;
      const int* cu = p.cu_rows + (p.group_major ? g * (B + 1) : 0);
      p.c.lengths[unit] = cu[s + 1] - cu[s];
    }
    return;
  }
  const unsigned task = warp * kTasks + lane;
  Move m;
  if (lane < kTasks && task < tasks) {
    int row = static_cast<int>(task);
    if (p.group_major) {
      while (m.head + 1 < H && p.cu_rows[(m.head + 1) * (B + 1)] <= row) ++m.head;
    } else {
      row = static_cast<int>(task / H);
      m.head = static_cast<int>(task) - row * H;
    }
    const int* cu = p.cu_rows + (p.group_major ? m.head * (B + 1) : 0);
    int s = 0, hi = B;  // cu[s] <= row < cu[s + 1]
    while (hi - s > 1) {
      const int mid = (s + hi) >> 1;
      if (cu[mid] <= row) s = mid; else hi = mid;
    }
    const int idx = p.indices[p.group_major ? row : static_cast<long long>(m.head) * p.rows + row];
    const int first = p.cu_seqlens[s], L = p.cu_seqlens[s + 1] - first;
    if (idx < 0 || idx >= L) {
      if (p.status) atomicCAS(p.status, 0, CKV_DEV_ERR_INDEX);
    } else {
      m.row = first + idx;
      m.dst = (s * H + m.head) * p.c.capacity + (row - cu[s]);
      m.position = idx;
      if (p.raw && idx < L - p.window)
        m.weight = p.raw[static_cast<long long>(m.head) * p.p_total + p.cu_prefix[s] + idx];
    }
  }
  move_rows<kBf16, kTasks>(p, m, static_cast<int>(warp * kTasks));
}

// Tasks a warp takes: four once every SM has more warps than it holds.  600,
// 1024, 2048 and 8192 rows of eight heads appended: 4.0, 5.6, 8.1 and 24.0 us by
// single tasks, 4.4, 5.4, 7.2 and 18.1 by four.
constexpr long long kManyTasks = 152 * 64;
constexpr int kMostTasks = 4;

template <bool kBf16, int kTasks, class P>
cudaError_t launch_gather_rows(const P& p, long long tasks, cudaStream_t stream) {
  const long long units = static_cast<long long>(p.c.batch) * p.c.num_kv_heads;
  const long long warps = (tasks + kTasks - 1) / kTasks + (units + 31) / 32;
  constexpr int kPer = kWriteThreads / 32;
  return launch_dependent(gather_q4_kernel<kBf16, kTasks, P>, dim3(static_cast<unsigned>((warps + kPer - 1) / kPer)),
                          kWriteThreads, 0, stream, p);
}
template <class P>
cudaError_t launch_gather_any(const P& p, cudaStream_t stream) {
  const long long tasks = p.group_major ? p.rows : static_cast<long long>(p.rows) * p.c.num_kv_heads;
  if (tasks <= kManyTasks)
    return p.is_bf16 ? launch_gather_rows<true, 1>(p, tasks, stream) : launch_gather_rows<false, 1>(p, tasks, stream);
  return p.is_bf16 ? launch_gather_rows<true, kMostTasks>(p, tasks, stream)
                   : launch_gather_rows<false, kMostTasks>(p, tasks, stream);
}

template <bool kBf16, int kTasks>
cudaError_t launch_append_rows(const Q4AppendParams& p, long long tasks, cudaStream_t stream) {
  constexpr long long kPer = static_cast<long long>(kWriteThreads / 32) * kTasks;
  return launch_dependent(append_rows_kernel<kBf16, kTasks>, dim3(static_cast<unsigned>((tasks + kPer - 1) / kPer)),
                          kWriteThreads, 0, stream, p);
}

}  // namespace

cudaError_t launch_q4_append(const Q4AppendParams& p, int max_rows, cudaStream_t stream) {
  const int units = p.c.batch * p.c.num_kv_heads;
  if (max_rows <= kSmallRows) {
    constexpr int kMost = kWriteThreads / 32;
    const int warps = max_rows < 1 ? 1 : max_rows < kMost ? max_rows : kMost;
    return launch_dependent(p.is_bf16 ? append_unit_kernel<true> : append_unit_kernel<false>, dim3(units), warps * 32,
                            0, stream, p);
  }
  const long long tasks = static_cast<long long>(p.rows) * p.c.num_kv_heads;
  cudaError_t e;
  if (tasks <= kManyTasks)
    e = p.is_bf16 ? launch_append_rows<true, 1>(p, tasks, stream) : launch_append_rows<false, 1>(p, tasks, stream);
  else
    e = p.is_bf16 ? launch_append_rows<true, kMostTasks>(p, tasks, stream) : launch_append_rows<false, kMostTasks>(p, tasks, stream);
  if (e != cudaSuccess) return e;
  return launch_dependent(append_lengths_kernel, dim3(p.c.batch), kLengthThreads, 0, stream, p);
}

cudaError_t launch_q4_gather(const Q4GatherParams& p, cudaStream_t stream) {
  return launch_gather_any(p, stream);
}
cudaError_t launch_q4_gather(const Q4GatherUnitParams& p, cudaStream_t stream) {
  return launch_gather_any(p, stream);
}

}  // namespace ckv
