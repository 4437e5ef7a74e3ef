// Attention of a few query tokens a sequence over the 4-bit cache.
//
//   z[r,j] = scale * sum_c q[r,c] (s n[j,c] + m),   p = softmax over the visible slots
//   out[r] = sum_j p[r,j] (s n[j,:] + m),   lse[r] = log sum_j exp z[r,j]
//   weight[j] += sum_r p[r,j]   (where asked for)
//
// A CTA takes one row r of one unit; its warps take every eighth slot with a
// running maximum and sum each, and are joined at the end.
#include <cuda_runtime.h>

#include "ckv_device.cuh"
#include "q4_params.h"

namespace ckv {

namespace {

constexpr int kAttendThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float to_float(uint32_t h, bool bf16) {
  if (bf16) return __uint_as_float(h << 16);
  float f;
  asm("{\n\t.reg .b16 t;\n\tcvt.u16.u32 t, %1;\n\tcvt.f32.f16 %0, t;\n\t}" : "=f"(f) : "r"(h));
  return f;
}
__device__ __forceinline__ uint16_t from_float(float x, bool bf16) {
  uint32_t r;
  if (bf16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(0.f), "f"(x));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(0.f), "f"(x));
  return static_cast<uint16_t>(r);
}

__device__ __forceinline__ int length_of(const Q4Cache& c, int unit) {
  return min(max(c.lengths[unit], 0), c.capacity);
}

// The four channels 4 * lane .. of a cache row.
__device__ __forceinline__ void row_values(const Q4Cache& c, int part, long long at, int lane,
                                           float (&x)[4]) {
  const uint32_t w = reinterpret_cast<const uint16_t*>(c.codes[part] + at * kQ4CodeBytes)[lane];
  const uint16_t* pr = reinterpret_cast<const uint16_t*>(c.params[part] + at * kQ4ParamBytes);
  const float s = to_float(pr[lane >> 3], true), m = to_float(pr[kQ4Groups + (lane >> 3)], true);
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = fmaf(static_cast<float>((w >> (4 * i)) & 15u), s, m);
}

__global__ void __launch_bounds__(kAttendThreads) attend_kernel(const __grid_constant__ Q4AttendParams p) {
  __shared__ float s_m[kAttendThreads / 32], s_l[kAttendThreads / 32];
  __shared__ float s_o[kAttendThreads / 32][kHeadDim];
  const int rows = p.group * p.num_queries;
  const int unit = blockIdx.x / rows, r = blockIdx.x - unit * rows;
  const int b = unit / p.c.num_kv_heads, g = unit - b * p.c.num_kv_heads;
  const int h = g * p.group + r / p.num_queries, qi = r % p.num_queries;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const bool bf16 = p.is_bf16 != 0;
  const uint16_t* qp = p.q + b * p.q_bs + h * p.q_hs + qi * p.q_qs + 4 * lane;
  float q[4], o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < 4; ++i) q[i] = to_float(qp[i], bf16);
  const int n = length_of(p.c, unit);
  const long long base = static_cast<long long>(unit) * p.c.capacity;
  const int at_most = p.q_positions ? p.q_positions[b * p.num_queries + qi] : 0x7fffffff;
  float m = -INFINITY, l = 0.f;
  for (int j = warp; j < n; j += kAttendThreads / 32) {
    float z = -INFINITY;
    const bool seen = !p.q_positions || p.c.positions[base + j] <= at_most;
    if (seen) {
      float k[4];
      row_values(p.c, 0, base + j, lane, k);
      z = fmaf(q[0], k[0], fmaf(q[1], k[1], fmaf(q[2], k[2], q[3] * k[3])));
      for (int d = 16; d; d >>= 1) z += __shfl_xor_sync(0xffffffffu, z, d);
      z *= p.scale * kLog2e;
    }
    if (p.accumulate && lane == 0) p.z[(static_cast<long long>(unit) * rows + r) * p.c.capacity + j] = z;
    if (!seen) continue;
    const float top = fmaxf(m, z), ref = top == -INFINITY ? 0.f : top;
    const float f = exp2f(m - ref), e = exp2f(z - ref);
    float v[4];
    row_values(p.c, 1, base + j, lane, v);
    for (int i = 0; i < 4; ++i) o[i] = fmaf(o[i], f, e * v[i]);
    l = fmaf(l, f, e);
    m = top;
  }
  for (int i = 0; i < 4; ++i) s_o[warp][4 * lane + i] = o[i];
  if (lane == 0) {
    s_m[warp] = m;
    s_l[warp] = l;
  }
  __syncthreads();
  if (threadIdx.x < kHeadDim) {
    float top = -INFINITY, sum = 0.f, x = 0.f;
    for (int w = 0; w < kAttendThreads / 32; ++w) top = fmaxf(top, s_m[w]);
    const float ref = top == -INFINITY ? 0.f : top;
    for (int w = 0; w < kAttendThreads / 32; ++w) {
      const float f = exp2f(s_m[w] - ref);
      sum = fmaf(s_l[w], f, sum);
      x = fmaf(s_o[w][threadIdx.x], f, x);
    }
    const float y = sum == 0.f ? 0.f : x / sum;
    p.out[b * p.o_bs + h * p.o_hs + qi * p.o_qs + threadIdx.x] = from_float(y, bf16);
    if (threadIdx.x == 0) {
      const float l2 = ref + log2f(sum);
      p.lse_ws[static_cast<long long>(unit) * rows + r] = l2;
      if (p.lse) p.lse[(static_cast<long long>(b) * p.num_q_heads + h) * p.num_queries + qi] = l2 / kLog2e;
    }
  }
}

__global__ void __launch_bounds__(kAttendThreads) weights_kernel(const __grid_constant__ Q4AttendParams p) {
  const int rows = p.group * p.num_queries;
  const int unit = blockIdx.y;
  const int j = blockIdx.x * kAttendThreads + threadIdx.x;
  if (j >= length_of(p.c, unit)) return;
  float add = 0.f;
  for (int r = 0; r < rows; ++r) {
    const long long row = static_cast<long long>(unit) * rows + r;
    const float z = p.z[row * p.c.capacity + j];
    if (z != -INFINITY) add += exp2f(z - p.lse_ws[row]);
  }
  p.c.weights[static_cast<long long>(unit) * p.c.capacity + j] += add;
}

}  // namespace

cudaError_t launch_q4_attend(const Q4AttendParams& p, cudaStream_t stream) {
  const unsigned ctas = static_cast<unsigned>(p.c.batch * p.c.num_kv_heads) * p.group * p.num_queries;
  attend_kernel<<<ctas, kAttendThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_q4_weights(const Q4AttendParams& p, cudaStream_t stream) {
  const dim3 grid((p.c.capacity + kAttendThreads - 1) / kAttendThreads, p.c.batch * p.c.num_kv_heads);
  weights_kernel<<<grid, kAttendThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace ckv
