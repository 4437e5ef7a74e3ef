// Attention of a few query tokens a sequence over the 4-bit cache.
//
//   z[r,j] = scale * sum_c q[r,c] (s n[j,c] + m),   p = softmax over the visible slots
//   out[r] = sum_j p[r,j] (s n[j,:] + m),   lse[r] = log sum_j exp z[r,j]
//   weight[j] += sum_r p[r,j]   (where asked for)
//
// Bound by memory: 160 bytes a slot against at most a few thousand operations,
// so the kernel is built around a steady stream of slots and few instructions
// a code.  Warps are independent workers: each takes a run of tiles of 32
// slots (see Q4AttendParams), keeps two or three in flight with TMA into its
// own part of shared memory, and leaves the softmax reference, sum and outputs
// of each row block it touched; a second kernel joins them.
//
// Codes enter the tensor cores as they are.  A nibble n masked out of a word is
// the fp16 subnormal n * 2^-24 (one in bits 4-7 is 16 n * 2^-24), exact in a
// product with fp32 sums, so five instructions make eight operands and neither
// scale, minimum nor an offset is applied to a code.  mma.sync takes operands
// from registers: with 8 or 16 query rows a unit's products are far below the
// tensor cores' rate, while tcgen05 would want the operands expanded to 16 bits
// in shared memory, four times the bytes of the codes.
//
//   S^T = K Q^T: A = codes of 16 slots, B = 8 query rows (as fp16, scaled by a
//     power of two a row so that the largest element is in [2^14, 2^15): exact
//     but for elements below 2^-34 of it); the four groups are summed apart and
//     scaled by their s in fp32.  The minima's term sum_J m_J (sum of q over J)
//     is one more product: the group sums as three bf16 parts (24 bits), m in bf16.
//   O^T = V^T P^T: A = codes of 16 channels, B = P^T, which movmatrix makes of
//     the result layout of S^T.  With p in fp16 (relative error 2^-12) the weights
//     of group J's codes are p s_J (rounded once more), those of its minimum p; the
//     minima's term is a product of its own.  Scales and minima are fp16 too,
//     exact against a power of two that follows the largest of both: 2^-21 of it
//     and above for scales, 2^-22 for minima.
// Eight lanes of a warp need the same slot's scales, so one lane a slot converts
// them for all (K: times the softmax scale in fp32; V: fp16 pairs of slots) and
// leaves them in shared memory.
// Softmax references are raised only when a logit passes them by 2^8, so the
// outputs are hardly ever rescaled.
#include <cuda_runtime.h>

#include "ckv_device.cuh"
#include "q4_params.h"

namespace ckv {

namespace {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kRaise = 8.0f;         // references lag behind the largest logit by at most this
constexpr float kLift = 3.0f;          // probabilities are held times 2^3: at most 2^11
constexpr int kTopExp = 7;             // scales become < 2^4, minima < 2^8: p s < 2^15
constexpr int kMinScaleExp = -110;     // smaller scales and minima share this reference

// Shared memory of a worker's stage: codes of K and V (swizzled), then params
// and positions.
constexpr int kCodeTile = kQ4TileSlots * kQ4CodeBytes;    // 2048
constexpr int kParamTile = kQ4TileSlots * kQ4ParamBytes;  // 512
constexpr int kPosTile = kQ4TileSlots * 4;                // 128
constexpr int kSideBytes = 2 * kParamTile + kPosTile;     // 1152
constexpr int kScaleTile = kQ4TileSlots * 16;             // K's scales of the tile at hand, fp32

#ifndef Q4W1
#define Q4W1 12
#define Q4S1 2
#define Q4W2 8
#define Q4S2 4
#endif
template <int NB>
struct Shape {
  static constexpr int kWarps = NB == 1 ? Q4W1 : Q4W2;
  static constexpr int kStages = NB == 1 ? Q4S1 : Q4S2;
  static constexpr int kThreads = kWarps * 32;
  static constexpr int kCodes = kWarps * kStages * 2 * kCodeTile;
  static constexpr int kSide = kWarps * kStages * kSideBytes;
  static constexpr int kScales = kWarps * kScaleTile;
  static constexpr int kSmem = 1024 + kCodes + kSide + kScales + kWarps * kStages * 8;
};

__device__ __forceinline__ float to_float(uint32_t h, bool bf16) {
  if (bf16) return __uint_as_float(h << 16);
  float f;
  asm("{\n\t.reg .b16 t;\n\tcvt.u16.u32 t, %1;\n\tcvt.f32.f16 %0, t;\n\t}" : "=f"(f) : "r"(h));
  return f;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ float pow2(int e) {  // -126 <= e <= 127
  return __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
}

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                        uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                         uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t mul_half2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// Transpose of an 8x8 matrix of 16-bit numbers: lane (g, t) gives row g,
// columns 2t and 2t + 1, and receives those of column g.
__device__ __forceinline__ uint32_t transpose8(uint32_t a) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
  return r;
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldmatrix4_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(a)
               : "memory");
  return v;
}
__device__ __forceinline__ void sts128(uint32_t a, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
               : "memory");
}
__device__ __forceinline__ void tma_rows(uint32_t dst, const CUtensorMap* map, uint32_t bar, int row) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], "
      "[%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(0), "r"(row)
      : "memory");
}
__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
      "l"(src), "r"(bytes), "r"(bar)
      : "memory");
}

__device__ __forceinline__ int length_of(const Q4Cache& c, int unit) {
  return min(max(__ldg(c.lengths + unit), 0), c.capacity);
}
__device__ __forceinline__ int tiles_of(const Q4Cache& c, int unit) {
  return (length_of(c, unit) + kQ4TileSlots - 1) / kQ4TileSlots;
}

// A tile's place in the sequence of tiles.
struct Place {
  int unit, block;
  int row;    // slot row of the cache: unit * capacity + first slot
  int valid;  // slots in use from there on
  // The next tile; past the end of a row block the next one that has tiles
  // (the caller knows that there is one).
  __device__ __forceinline__ void next(const Q4AttendParams& p) {
    row += kQ4TileSlots;
    valid -= kQ4TileSlots;
    if (valid > 0) return;
    if (++block == p.blocks) {
      block = 0;
      ++unit;
    }
    while ((valid = length_of(p.c, unit)) == 0) ++unit;
    row = unit * p.c.capacity;
  }
};

// Sum over the CTA of one number a thread: the exclusive prefix, and the total.
template <int kThreads>
__device__ __forceinline__ long long cta_scan(long long v, long long* s_sums, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) s_sums[warp] = x;
  __syncthreads();
  long long before = 0, all = 0;
  for (int w = 0; w < kThreads / 32; ++w) {
    const long long t = s_sums[w];
    if (w < warp) before += t;
    all += t;
  }
  *total = all;
  return before + x - v;
}

// The largest of 16 s and |m| of a params row, as the bits of a float (whose
// order is that of the numbers; NaN above all).
__device__ __forceinline__ uint32_t top_of(uint4 w) {
  const uint32_t s = max(max(w.x << 16, w.x & 0xffff0000u), max(w.y << 16, w.y & 0xffff0000u)) + (4u << 23);
  const uint32_t z = max((w.z << 16) & 0x7fff0000u, w.z & 0x7fff0000u);
  return max(s, max(z, max((w.w << 16) & 0x7fff0000u, w.w & 0x7fff0000u)));
}

// The query rows of a row block as operands: row lane/4 of each 8.
template <int NB>
struct Queries {
  uint32_t b[NB][8][2];      // [8 rows][4 groups x 2 steps][k half]
  uint32_t sum[NB][2];       // group sums as three bf16 parts, scaled like the codes' products
  // of rows 2 (lane % 4) and the next, the columns of a result:
  float f2[NB][2];           // z = products * f2 (K's scales carry the softmax scale)
  int limit[NB][2];          // q_position
};

template <int NB>
__device__ __forceinline__ void load_queries(const Q4AttendParams& p, int unit, int block, Queries<NB>& Q) {
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int b = unit / p.c.num_kv_heads, kv = unit - b * p.c.num_kv_heads;
  const bool bf16 = p.is_bf16 != 0;
  const float f1 = p.scale_log2 * 1024.0f;  // codes carry 2^-24, queries 2^14
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int r = block * (8 * NB) + nb * 8 + g;
    float x[4][8];
    uint32_t top = 0;
    int limit = 0x7fffffff;
    if (r < p.rows) {
      const int h = kv * p.group + r / p.num_queries, qi = r % p.num_queries;
      const uint16_t* src = p.q + b * p.q_bs + h * p.q_hs + qi * p.q_qs + 8 * t;
      if (p.q_positions) limit = __ldg(p.q_positions + b * p.num_queries + qi);
#pragma unroll
      for (int J = 0; J < 4; ++J) {
        const uint4 w = __ldg(reinterpret_cast<const uint4*>(src + 32 * J));
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[J][i] = to_float(i & 1 ? u[i >> 1] >> 16 : u[i >> 1] & 0xffffu, bf16);
          top = max(top, __float_as_uint(x[J][i]) & 0x7fffffffu);
        }
      }
    } else {
#pragma unroll
      for (int J = 0; J < 4; ++J)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[J][i] = 0.f;
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    // exponent of the largest element; a row of zeros, NaN or infinities as it is
    int e = top >= 0x7f800000u || top == 0 ? 14 : static_cast<int>(top >> 23) - 127;
    e = max(e, -110);  // smaller rows (bf16) scale by no more than 2^124
    const float up = pow2(14 - e);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      Q.f2[nb][j] = __shfl_sync(0xffffffffu, pow2(e), 8 * t + 4 * j);
      Q.limit[nb][j] = __shfl_sync(0xffffffffu, limit, 8 * t + 4 * j);
    }
    float part[4];
#pragma unroll
    for (int J = 0; J < 4; ++J) {
      part[J] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[J][i] *= up;
        part[J] += x[J][i];
      }
      part[J] += __shfl_xor_sync(0xffffffffu, part[J], 1);
      part[J] += __shfl_xor_sync(0xffffffffu, part[J], 2);
      part[J] *= 5.9604644775390625e-8f * f1;  // 2^-24
      // nibbles (0, 4), (1, 5), (2, 6), (3, 7) of a word; the odd ones count 16-fold
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        Q.b[nb][2 * J + st][0] = pack_half2(x[J][2 * st], x[J][2 * st + 4]);
        Q.b[nb][2 * J + st][1] = pack_half2(x[J][2 * st + 1] * 0.0625f, x[J][2 * st + 5] * 0.0625f);
      }
    }
    // k index J + 4 * part: this lane's pairs are groups 2 (t & 1), 2 (t & 1) + 1
    const float s0 = t & 1 ? part[2] : part[0], s1 = t & 1 ? part[3] : part[1];
    const uint32_t hi = pack_bf16(s0, s1);
    const float m0 = s0 - bf_lo(hi), m1 = s1 - bf_hi(hi);
    const uint32_t mid = pack_bf16(m0, m1);
    const uint32_t lo = pack_bf16(m0 - bf_lo(mid), m1 - bf_hi(mid));
    Q.sum[nb][0] = t < 2 ? hi : mid;
    Q.sum[nb][1] = t < 2 ? lo : 0u;
  }
}

template <int NB, bool kPos>
__global__ void __launch_bounds__(Shape<NB>::kThreads, 1)
    attend_kernel(const __grid_constant__ Q4AttendParams p) {
  using S = Shape<NB>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ long long s_sums[S::kWarps], s_before[S::kWarps];
  __shared__ int s_unit[S::kWarps], s_abort;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, t = lane & 3;
  const uint32_t codes = base + warp * S::kStages * 2 * kCodeTile;
  const uint32_t side = base + S::kCodes + warp * S::kStages * kSideBytes;
  const uint32_t scales = base + S::kCodes + S::kSide + warp * kScaleTile;
  const uint32_t bars = base + S::kCodes + S::kSide + S::kScales + warp * S::kStages * 8;
  if (lane == 0)
    for (int i = 0; i < S::kStages; ++i) mbar_init(bars + 8 * i, 1);
  if (threadIdx.x == 0) s_abort = 0;
  if (threadIdx.x == 0) {
    tma_prefetch_map(&p.map_k);
    tma_prefetch_map(&p.map_v);
  }
  fence_mbar_init();

  // ---- this worker's tiles
  const int units = p.c.batch * p.c.num_kv_heads;
  const int span = (units + S::kThreads - 1) / S::kThreads;  // units a thread adds up
  const int u0 = min(static_cast<int>(threadIdx.x) * span, units), u1 = min(u0 + span, units);
  long long mine = 0, total = 0;
  for (int u = u0; u < u1; ++u) mine += tiles_of(p.c, u);
  const long long before = cta_scan<S::kThreads>(mine, s_sums, &total);
  if (blockIdx.x == 0) {
    long long at = before;
    for (int u = u0; u < u1; ++u) {
      p.first_tile[u] = at;
      at += tiles_of(p.c, u);
    }
    if (threadIdx.x == 0) p.first_tile[units] = total;
  }
  total *= p.blocks;
  const long long chunk = (total + p.workers - 1) / p.workers;
  // neighbouring workers sit on different SMs
  const int worker = warp * gridDim.x + blockIdx.x;
  // the worker's first unit: the thread whose units hold it, then that unit
  for (int w = 0; w < S::kWarps; ++w) {
    const long long at = (static_cast<long long>(w) * gridDim.x + blockIdx.x) * chunk;
    if (at >= before * p.blocks && at < (before + mine) * p.blocks) {
      s_unit[w] = u0;
      s_before[w] = before * p.blocks;
    }
  }
  __syncthreads();
  const long long from = worker * chunk;
  int left = static_cast<int>(min(chunk, total - from));  // tiles of this worker
  if (chunk == 0 || left <= 0) return;
  Place c;
  {
    int u = s_unit[warp];
    long long at = s_before[warp];
    int n;
    while (at + static_cast<long long>(n = tiles_of(p.c, u)) * p.blocks <= from) {
      at += static_cast<long long>(n) * p.blocks;
      ++u;
    }
    const long long in = from - at;
    c.unit = u;
    c.block = static_cast<int>(in / n);
    const int slot = static_cast<int>(in - static_cast<long long>(c.block) * n) * kQ4TileSlots;
    c.row = u * p.c.capacity + slot;
    c.valid = length_of(p.c, u) - slot;
  }

  constexpr uint32_t kBytes = 2 * kCodeTile + 2 * kParamTile + (kPos ? kPosTile : 0);
  Place ahead = c;
  int to_issue = left;
  auto issue = [&](int stage) {
    if (lane == 0) {
      const uint32_t bar = bars + 8 * stage, cd = codes + stage * 2 * kCodeTile, sd = side + stage * kSideBytes;
      mbar_arrive_expect_tx(bar, kBytes);
      tma_rows(cd, &p.map_k, bar, ahead.row);
      tma_rows(cd + kCodeTile, &p.map_v, bar, ahead.row);
      const size_t row = static_cast<size_t>(ahead.row);
      bulk_copy(sd, p.c.params[0] + row * kQ4ParamBytes, kParamTile, bar);
      bulk_copy(sd + kParamTile, p.c.params[1] + row * kQ4ParamBytes, kParamTile, bar);
      if (kPos) bulk_copy(sd + 2 * kParamTile, p.c.positions + row, kPosTile, bar);
    }
    if (--to_issue > 0) ahead.next(p);
  };
  for (int i = 0; i < S::kStages && to_issue > 0; ++i) issue(i);

  // ldmatrix row of this lane: slot lane & 7, piece lane >> 3 of its 64 bytes,
  // stored at piece ^ (slot / 2) by the 64-byte swizzle
  const uint32_t mat = (lane & 7) * kQ4CodeBytes + (((lane >> 3) ^ ((lane >> 1) & 3)) << 4);

  const float f1 = p.scale_log2 * 1024.0f;
  Queries<NB> Q;
  float o[NB][4][2][4];   // [8 rows][group][step][channel, row pair]
  float om[NB][4];        // minima's term (lanes of g >= 4)
  float ref[NB][2], l[NB][2];  // rows 2t, 2t + 1
  int vexp = kMinScaleExp;
  bool fresh = true;
  uint32_t phase = 0;
  int stage = 0;
  bool failed = false;

  for (; left > 0; --left) {
    if (fresh) {
      load_queries<NB>(p, c.unit, c.block, Q);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        ref[nb][0] = ref[nb][1] = -INFINITY;
        l[nb][0] = l[nb][1] = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) om[nb][i] = 0.f;
#pragma unroll
        for (int J = 0; J < 4; ++J)
#pragma unroll
          for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[nb][J][st][i] = 0.f;
      }
      vexp = kMinScaleExp;
      fresh = false;
    }
    if (!mbar_wait_bounded(bars + 8 * stage, phase, &s_abort, p.status)) {
      failed = true;
      break;
    }
    __syncwarp();
    const uint32_t cd = codes + stage * 2 * kCodeTile, sd = side + stage * kSideBytes;
    const int valid = c.valid;

    // ---- scales: one lane a slot.  Slots behind the length and groups that
    // hold a NaN count nothing in V's products
    uint32_t nan_groups = 0;  // of this lane's slot
    bool special;
    {
      const uint2 kw = lds64(sd + lane * kQ4ParamBytes);
      uint4 w = lds128(sd + kParamTile + lane * kQ4ParamBytes);
      if (lane >= valid) w = make_uint4(0u, 0u, 0u, 0u);
      sts128(scales + lane * 16,
             make_uint4(__float_as_uint(bf_lo(kw.x) * f1), __float_as_uint(bf_hi(kw.x) * f1),
                        __float_as_uint(bf_lo(kw.y) * f1), __float_as_uint(bf_hi(kw.y) * f1)));
      uint32_t all = __reduce_max_sync(0xffffffffu, top_of(w));
      special = all >= 0x7f800000u;
      if (special) {
        uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int J = 0; J < 4; ++J) {
          const uint32_t half = 0xffffu << (16 * (J & 1)), inf = 0x7f807f80u & half;
          if ((x[J >> 1] & inf) == inf || (x[2 + (J >> 1)] & inf) == inf) {
            nan_groups |= 1u << J;
            x[J >> 1] &= ~half;
            x[2 + (J >> 1)] &= ~half;
          }
        }
        w = make_uint4(x[0], x[1], x[2], x[3]);
        all = min(__reduce_max_sync(0xffffffffu, top_of(w)), 0x7f000000u);
      }
      const int k = max(static_cast<int>(all >> 23) - 127, kMinScaleExp);
      if (k > vexp) {  // the sums go to the new power of two
        const float f = pow2(max(vexp - k, -126));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          om[nb][0] *= f;
          om[nb][1] *= f;
#pragma unroll
          for (int J = 0; J < 4; ++J)
#pragma unroll
            for (int st = 0; st < 2; ++st)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[nb][J][st][i] *= f;
        }
        vexp = k;
      }
      const float f = pow2(kTopExp - vexp);
      const uint32_t s01 = pack_half2(bf_lo(w.x) * f, bf_hi(w.x) * f);
      const uint32_t s23 = pack_half2(bf_lo(w.y) * f, bf_hi(w.y) * f);
      // an even lane keeps groups 0 and 1 of its pair of slots, an odd one 2 and 3
      const uint32_t got = __shfl_xor_sync(0xffffffffu, lane & 1 ? s01 : s23, 1);
      const uint32_t a = lane & 1 ? got : s01, b = lane & 1 ? s23 : got;
      sts128(sd + kParamTile + lane * kQ4ParamBytes,
             make_uint4(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632),
                        pack_half2(bf_lo(w.z) * f, bf_hi(w.z) * f),
                        pack_half2(bf_lo(w.w) * f, bf_hi(w.w) * f)));
      __syncwarp();
    }

    // ---- logits: twice 16 slots; slots g and g + 8 of rows 2t and 2t + 1
    float z[NB][2][4];  // [8 rows][16 slots][slot half, row]
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int s16 = h * 16;
      uint32_t wa[4], wb[4];
      ldmatrix4(wa, cd + s16 * kQ4CodeBytes + mat);
      ldmatrix4(wb, cd + (s16 + 8) * kQ4CodeBytes + mat);
      const uint32_t ma = lds32(sd + (s16 + g) * kQ4ParamBytes + 8 + (t & 1) * 4);
      const uint32_t mb = lds32(sd + (s16 + 8 + g) * kQ4ParamBytes + 8 + (t & 1) * 4);
      const uint4 sa = lds128(scales + (s16 + g) * 16), sb = lds128(scales + (s16 + 8 + g) * 16);
      const uint32_t ka[4] = {sa.x, sa.y, sa.z, sa.w}, kb[4] = {sb.x, sb.y, sb.z, sb.w};
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
        for (int i = 0; i < 4; ++i) z[nb][h][i] = 0.f;
        mma_bf16(z[nb][h], ma, mb, ma, mb, Q.sum[nb][0], Q.sum[nb][1]);
      }
#pragma unroll
      for (int J = 0; J < 4; ++J) {
        const uint32_t ha = wa[J] >> 8, hb = wb[J] >> 8;
        const uint32_t a0 = wa[J] & 0x000f000fu, a1 = wb[J] & 0x000f000fu;
        const uint32_t a2 = wa[J] & 0x00f000f0u, a3 = wb[J] & 0x00f000f0u;
        const uint32_t b0 = ha & 0x000f000fu, b1 = hb & 0x000f000fu;
        const uint32_t b2 = ha & 0x00f000f0u, b3 = hb & 0x00f000f0u;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          float x[4] = {0.f, 0.f, 0.f, 0.f};
          mma_f16(x, a0, a1, a2, a3, Q.b[nb][2 * J][0], Q.b[nb][2 * J][1]);
          mma_f16(x, b0, b1, b2, b3, Q.b[nb][2 * J + 1][0], Q.b[nb][2 * J + 1][1]);
          z[nb][h][0] = fmaf(x[0], __uint_as_float(ka[J]), z[nb][h][0]);
          z[nb][h][1] = fmaf(x[1], __uint_as_float(ka[J]), z[nb][h][1]);
          z[nb][h][2] = fmaf(x[2], __uint_as_float(kb[J]), z[nb][h][2]);
          z[nb][h][3] = fmaf(x[3], __uint_as_float(kb[J]), z[nb][h][3]);
        }
      }
      if (kPos) {
        const int at0 = static_cast<int>(lds32(sd + 2 * kParamTile + (s16 + g) * 4));
        const int at1 = static_cast<int>(lds32(sd + 2 * kParamTile + (s16 + 8 + g) * 4));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            if (at0 > Q.limit[nb][j]) z[nb][h][j] = -INFINITY;
            if (at1 > Q.limit[nb][j]) z[nb][h][2 + j] = -INFINITY;
          }
      }
    }
    if (valid < kQ4TileSlots) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (h * 16 + (i >> 1) * 8 + g >= valid)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) z[nb][h][i] = -INFINITY;
    }
    if (p.accumulate) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int r = c.block * (8 * NB) + nb * 8 + 2 * t + j;
          if (r < p.rows) {
            float* zp = p.z + (static_cast<long long>(c.unit) * (p.rows - 1) + r) * p.c.capacity + c.row + g;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              zp[h * 16] = z[nb][h][j] * Q.f2[nb][j];
              zp[h * 16 + 8] = z[nb][h][2 + j] * Q.f2[nb][j];
            }
          }
        }
    }

    // ---- references, probabilities (in place of z)
    uint32_t seen_nan[2] = {0u, 0u};
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float top[2];
      bool raise = false;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        top[j] = fmaxf(fmaxf(z[nb][0][j], z[nb][0][2 + j]), fmaxf(z[nb][1][j], z[nb][1][2 + j]));
        top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], 4));
        top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], 8));
        top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], 16)) * Q.f2[nb][j];
        raise |= top[j] > ref[nb][j] + kRaise;
      }
      if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (!(top[j] > ref[nb][j] + kRaise)) continue;
          const float f = ref[nb][j] == -INFINITY ? 0.f : ex2_approx(ref[nb][j] - top[j]);
          ref[nb][j] = top[j];
          l[nb][j] *= f;
          om[nb][j] *= f;
#pragma unroll
          for (int J = 0; J < 4; ++J)
#pragma unroll
            for (int st = 0; st < 2; ++st) {
              o[nb][J][st][j] *= f;
              o[nb][J][st][2 + j] *= f;
            }
        }
      }
      if (special) {
        // rows that see a slot's NaN group
        uint32_t hit[2] = {0u, 0u};
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t m = __shfl_sync(0xffffffffu, nan_groups, h * 16 + (i >> 1) * 8 + g);
            if (z[nb][h][i] != -INFINITY) hit[i & 1] |= m;
          }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          hit[j] |= __shfl_xor_sync(0xffffffffu, hit[j], 4);
          hit[j] |= __shfl_xor_sync(0xffffffffu, hit[j], 8);
          hit[j] |= __shfl_xor_sync(0xffffffffu, hit[j], 16);
          seen_nan[j] |= hit[j] << (4 * nb);
        }
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float r = ref[nb][j] == -INFINITY ? 0.f : ref[nb][j] - kLift;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = j; i < 4; i += 2) {
            z[nb][h][i] = ex2_approx(fmaf(z[nb][h][i], Q.f2[nb][j], -r));
            l[nb][j] += z[nb][h][i];
          }
      }
    }

    // ---- outputs: twice 16 slots
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int s16 = h * 16;
      uint32_t va[4], vb[4], pm[4];
      ldmatrix4_t(va, cd + kCodeTile + s16 * kQ4CodeBytes + mat);
      ldmatrix4_t(vb, cd + kCodeTile + (s16 + 8) * kQ4CodeBytes + mat);
      // rows of [2 pairs of scales, 4 minima]: rows 4-7 of the transposed
      // operand are the minima; rows 8-15 repeat rows 0-7
      ldmatrix4_t(pm, sd + kParamTile + (s16 + (lane & 7) + ((lane & 16) >> 1)) * kQ4ParamBytes);
      const uint2 s0 = lds64(sd + kParamTile + (s16 + 2 * t) * kQ4ParamBytes);
      const uint2 s1 = lds64(sd + kParamTile + (s16 + 2 * t + 1) * kQ4ParamBytes);
      const uint2 s2 = lds64(sd + kParamTile + (s16 + 8 + 2 * t) * kQ4ParamBytes);
      const uint2 s3 = lds64(sd + kParamTile + (s16 + 9 + 2 * t) * kQ4ParamBytes);
      const uint32_t sa[4] = {s0.x, s0.y, s1.x, s1.y}, sb[4] = {s2.x, s2.y, s3.x, s3.y};
      uint32_t p0[NB], p1[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        p0[nb] = transpose8(pack_half2(z[nb][h][0], z[nb][h][1]));
        p1[nb] = transpose8(pack_half2(z[nb][h][2], z[nb][h][3]));
        mma_f16(om[nb], pm[0], pm[1], pm[2], pm[3], p0[nb], p1[nb]);
      }
#pragma unroll
      for (int J = 0; J < 4; ++J) {
        const uint32_t ah = va[J] >> 8, bh = vb[J] >> 8;
        const uint32_t a0 = va[J] & 0x000f000fu, a1 = va[J] & 0x00f000f0u;
        const uint32_t a2 = vb[J] & 0x000f000fu, a3 = vb[J] & 0x00f000f0u;
        const uint32_t b0 = ah & 0x000f000fu, b1 = ah & 0x00f000f0u;
        const uint32_t b2 = bh & 0x000f000fu, b3 = bh & 0x00f000f0u;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const uint32_t q0 = mul_half2(p0[nb], sa[J]), q1 = mul_half2(p1[nb], sb[J]);
          mma_f16(o[nb][J][0], a0, a1, a2, a3, q0, q1);
          mma_f16(o[nb][J][1], b0, b1, b2, b3, q0, q1);
        }
      }
    }
    if (special) {
      const float bad = __uint_as_float(0x7fc00000u);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
        for (int J = 0; J < 4; ++J)
#pragma unroll
          for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if ((seen_nan[i & 1] >> (4 * nb + J)) & 1u) o[nb][J][st][i] = bad;
      }
    }
    fence_proxy_async_smem();  // (the scales were written into the stage)
    __syncwarp();  // every lane is done with the stage
    if (to_issue > 0) issue(stage);
    if (++stage == S::kStages) {
      stage = 0;
      phase ^= 1u;
    }

    // ---- the row block ends here, or this worker's share of it
    const int unit = c.unit, block = c.block;
    if (left > 1) c.next(p);
    if (left == 1 || c.unit != unit || c.block != block) {
      const long long part = static_cast<long long>(worker) + static_cast<long long>(unit) * p.blocks + block;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float sum = l[nb][j];
          sum += __shfl_xor_sync(0xffffffffu, sum, 4);
          sum += __shfl_xor_sync(0xffffffffu, sum, 8);
          sum += __shfl_xor_sync(0xffffffffu, sum, 16);
          if (g == 0) p.part_ml[part * (8 * NB) + nb * 8 + 2 * t + j] = make_float2(ref[nb][j] - kLift, sum);
        }
        const float f = pow2(vexp - kTopExp);  // codes' sums: * 2^24, and 1/16 for the odd channels
        float* dst = p.part_o + (part * (8 * NB) + nb * 8) * kHeadDim;
#pragma unroll
        for (int J = 0; J < 4; ++J) {
          const float m0 = __shfl_sync(0xffffffffu, om[nb][0], (4 + J) * 4 + t);
          const float m1 = __shfl_sync(0xffffffffu, om[nb][1], (4 + J) * 4 + t);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float m = i ? m1 : m0;
            float4 v;
            v.x = fmaf(o[nb][J][0][i], 16777216.0f, m) * f;
            v.y = fmaf(o[nb][J][0][2 + i], 1048576.0f, m) * f;
            v.z = fmaf(o[nb][J][1][i], 16777216.0f, m) * f;
            v.w = fmaf(o[nb][J][1][2 + i], 1048576.0f, m) * f;
            if (block * (8 * NB) + nb * 8 + 2 * t + i < p.rows)
              *reinterpret_cast<float4*>(dst + (2 * t + i) * kHeadDim + 32 * J + 4 * g) = v;
          }
        }
      }
      fresh = true;
    }
  }
  if (failed) {
    // copies in flight end before the shared memory does (or their wait runs out)
    for (int i = 0; i < S::kStages; ++i) {
      const uint64_t t0 = globaltimer_ns();
      while (!mbar_test_wait(bars + 8 * i, phase) && globaltimer_ns() - t0 < 100000000ull) {
      }
    }
  }
}

// ---------------------------------------------------------------- joining
// A CTA takes one query row of a unit: its parts' references and sums, then
// their outputs, a warp a part.
constexpr int kCombineThreads = 256;

__global__ void __launch_bounds__(kCombineThreads) combine_kernel(const __grid_constant__ Q4AttendParams p) {
  __shared__ float s_red[kCombineThreads / 32];
  __shared__ float4 s_o[kCombineThreads / 32][32];
  const int unit = blockIdx.x, r = blockIdx.y;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int units = p.c.batch * p.c.num_kv_heads;
  const int brows = p.rows <= 8 ? 8 : 16;
  const int block = r / brows, rb = r - block * brows;
  const long long total = p.first_tile[units] * p.blocks;
  const long long chunk = (total + p.workers - 1) / p.workers;
  const long long before = p.first_tile[unit], n = p.first_tile[unit + 1] - before;
  const long long from = before * p.blocks + block * n;
  const int b = unit / p.c.num_kv_heads, h = (unit - b * p.c.num_kv_heads) * p.group + r / p.num_queries;
  const int qi = r % p.num_queries;
  int first = 0, count = 0;
  if (n > 0) {
    first = static_cast<int>(from / chunk);
    count = static_cast<int>((from + n - 1) / chunk) - first + 1;
  }
  const long long part0 = static_cast<long long>(first) + static_cast<long long>(unit) * p.blocks + block;
  const float2* ml = p.part_ml + part0 * brows + rb;
  float top = -INFINITY;
  for (int i = threadIdx.x; i < count; i += kCombineThreads) top = fmaxf(top, ml[static_cast<long long>(i) * brows].x);
#pragma unroll
  for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (lane == 0) s_red[warp] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kCombineThreads / 32; ++w) top = fmaxf(top, s_red[w]);
  const float ref = top == -INFINITY ? 0.f : top;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float sum = 0.f;
  for (int i = warp; i < count; i += kCombineThreads / 32) {
    const float2 x = ml[static_cast<long long>(i) * brows];
    const float f = ex2_approx(x.x - ref);
    const float4 v = reinterpret_cast<const float4*>(p.part_o + ((part0 + i) * brows + rb) * kHeadDim)[lane];
    sum = fmaf(x.y, f, sum);
    acc.x = fmaf(v.x, f, acc.x);
    acc.y = fmaf(v.y, f, acc.y);
    acc.z = fmaf(v.z, f, acc.z);
    acc.w = fmaf(v.w, f, acc.w);
  }
  s_o[warp][lane] = acc;
  __syncthreads();
  if (lane == 0) s_red[warp] = sum;
  __syncthreads();
  if (warp != 0) return;
  sum = 0.f;
  acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int w = 0; w < kCombineThreads / 32; ++w) {
    sum += s_red[w];
    const float4 v = s_o[w][lane];
    acc.x += v.x;
    acc.y += v.y;
    acc.z += v.z;
    acc.w += v.w;
  }
  const float f = sum == 0.f ? 0.f : 1.0f / sum;
  uint2 y;
  if (p.is_bf16) {
    y.x = pack_bf16(acc.x * f, acc.y * f);
    y.y = pack_bf16(acc.z * f, acc.w * f);
  } else {
    y.x = pack_half2(acc.x * f, acc.y * f);
    y.y = pack_half2(acc.z * f, acc.w * f);
  }
  *reinterpret_cast<uint2*>(p.out + b * p.o_bs + h * p.o_hs + qi * p.o_qs + 4 * lane) = y;
  if (lane == 0) {
    const float l2 = ref + log2f(sum);
    p.lse_ws[static_cast<long long>(unit) * p.rows + r] = l2;
    if (p.lse) p.lse[(static_cast<long long>(b) * p.num_q_heads + h) * p.num_queries + qi] = l2 * kLn2;
  }
}

// ---------------------------------------------------------------- weights
constexpr int kWeightThreads = 256;

__global__ void __launch_bounds__(kWeightThreads) weights_kernel(const __grid_constant__ Q4AttendParams p) {
  const int unit = blockIdx.y;
  const int j = blockIdx.x * kWeightThreads + threadIdx.x;
  if (j >= length_of(p.c, unit)) return;
  float add = 0.f;
  for (int r = 0; r < p.rows; ++r) {
    const long long row = static_cast<long long>(unit) * p.rows + r;
    const float z = p.z[row * p.c.capacity + j];
    if (z != -INFINITY) add += ex2_approx(z - p.lse_ws[row]);
  }
  p.c.weights[static_cast<long long>(unit) * p.c.capacity + j] += add;
}

template <int NB>
cudaError_t launch(const Q4AttendParams& p, int sms, cudaStream_t stream) {
  using S = Shape<NB>;
  if (p.q_positions) attend_kernel<NB, true><<<sms, S::kThreads, S::kSmem, stream>>>(p);
  else attend_kernel<NB, false><<<sms, S::kThreads, S::kSmem, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace

int q4_attend_workers(int rows, int sms) { return sms * (rows <= 8 ? Shape<1>::kWarps : Shape<2>::kWarps); }

cudaError_t q4_attend_set_smem_limit() {
  cudaError_t e = cudaSuccess;
  auto set = [&](auto* f, int bytes) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  };
  set(attend_kernel<1, false>, Shape<1>::kSmem);
  set(attend_kernel<1, true>, Shape<1>::kSmem);
  set(attend_kernel<2, false>, Shape<2>::kSmem);
  set(attend_kernel<2, true>, Shape<2>::kSmem);
  return e;
}

cudaError_t launch_q4_attend(const Q4AttendParams& p, int sms, cudaStream_t stream) {
  return p.rows <= 8 ? launch<1>(p, sms, stream) : launch<2>(p, sms, stream);
}

cudaError_t launch_q4_combine(const Q4AttendParams& p, cudaStream_t stream) {
  const dim3 grid(p.c.batch * p.c.num_kv_heads, p.rows);
  combine_kernel<<<grid, kCombineThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_q4_weights(const Q4AttendParams& p, cudaStream_t stream) {
  const dim3 grid((p.c.capacity + kWeightThreads - 1) / kWeightThreads, p.c.batch * p.c.num_kv_heads);
  weights_kernel<<<grid, kWeightThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace ckv
