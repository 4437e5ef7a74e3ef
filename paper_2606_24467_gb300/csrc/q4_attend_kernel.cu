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
//   S = Q K^T: A = q rows (16-bit queries as fp16, scaled by a power of two a
//     row so that the largest is in [2^14, 2^15): exact but for elements below
//     2^-34 of it), B = codes of 8 slots; the four groups are summed apart and
//     scaled by their s in fp32.  The minima's term sum_J m_J (sum of q over J)
//     is one more product: the group sums as three bf16 parts (24 bits), m in bf16.
//   O^T = V^T P^T: the result layout of S is the operand layout of P^T, so no
//     value changes lanes.  The weights of group J's codes are p s_J, in fp16
//     (relative error 2^-12, independent for each slot) against a power of two
//     that follows the largest s seen: 20 binades below the largest p s_J keep
//     that precision.  The minima's term sum_j p m_J is one more product with
//     p as two bf16 parts.
// Softmax references are raised only when a logit passes them by 2^8, so the
// outputs are hardly ever rescaled.
#include <cuda_runtime.h>

#include "ckv_device.cuh"
#include "q4_params.h"

namespace ckv {

namespace {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kRaise = 8.0f;         // references lag behind the largest logit by at most this
constexpr int kTopExp = 14 - 8;        // p s_J <= 2^8 * 2^(k+1) becomes < 2^15
constexpr int kMinScaleExp = -110;     // smaller scales share this reference

// Shared memory of a worker's stage: codes of K and V (swizzled), then params
// and positions.
constexpr int kCodeTile = kQ4TileSlots * kQ4CodeBytes;    // 2048
constexpr int kParamTile = kQ4TileSlots * kQ4ParamBytes;  // 512
constexpr int kPosTile = kQ4TileSlots * 4;                // 128
constexpr int kSideBytes = 2 * kParamTile + kPosTile;     // 1152

template <int NB>
struct Shape {
  static constexpr int kWarps = NB == 1 ? 16 : 12;
  static constexpr int kStages = NB == 1 ? 2 : 3;
  static constexpr int kThreads = kWarps * 32;
  static constexpr int kCodes = kWarps * kStages * 2 * kCodeTile;
  static constexpr int kSide = kWarps * kStages * kSideBytes;
  static constexpr int kSmem = 1024 + kCodes + kSide + kWarps * kStages * 8;
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

// A place in the sequence of tiles.
struct Place {
  int unit, block, tile, len;  // len: slots in use of the unit
  __device__ __forceinline__ int tiles() const { return (len + kQ4TileSlots - 1) / kQ4TileSlots; }
  // The next tile; past the end of a row block the next one that has tiles
  // (or unit = units).
  __device__ __forceinline__ void next(const Q4AttendParams& p, int units) {
    if (++tile < tiles()) return;
    tile = 0;
    if (++block < p.blocks) return;
    block = 0;
    do {
      ++unit;
      len = unit < units ? length_of(p.c, unit) : 0;
    } while (unit < units && len == 0);
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

// The query rows of a row block as operands: row lane/4 (and 8 more).
template <int NB>
struct Queries {
  uint32_t a[NB][2][8];      // [8 rows][k half][4 groups x 2 steps]
  uint32_t sum[NB][2];       // group sums * 2^-24 as three bf16 parts
  float f1, f2[NB];          // z = (products * f1) * f2
  int limit[NB];             // q_position
};

template <int NB>
__device__ __forceinline__ void load_queries(const Q4AttendParams& p, int unit, int block, Queries<NB>& Q) {
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int b = unit / p.c.num_kv_heads, kv = unit - b * p.c.num_kv_heads;
  const bool bf16 = p.is_bf16 != 0;
  Q.f1 = p.scale_log2 * 1024.0f;  // codes carry 2^-24, queries 2^14
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int r = block * (8 * NB) + nb * 8 + g;
    float x[4][8];
    uint32_t top = 0;
    Q.limit[nb] = 0x7fffffff;
    if (r < p.rows) {
      const int h = kv * p.group + r / p.num_queries, qi = r % p.num_queries;
      const uint16_t* src = p.q + b * p.q_bs + h * p.q_hs + qi * p.q_qs + 8 * t;
      if (p.q_positions) Q.limit[nb] = __ldg(p.q_positions + b * p.num_queries + qi);
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
    Q.f2[nb] = pow2(max(e, -126));
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
      part[J] *= 5.9604644775390625e-8f;  // 2^-24
      // nibbles (0, 4), (1, 5), (2, 6), (3, 7) of a word; the odd ones count 16-fold
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        Q.a[nb][0][2 * J + st] = pack_half2(x[J][2 * st], x[J][2 * st + 4]);
        Q.a[nb][1][2 * J + st] = pack_half2(x[J][2 * st + 1] * 0.0625f, x[J][2 * st + 5] * 0.0625f);
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
  const uint32_t bars = base + S::kCodes + S::kSide + warp * S::kStages * 8;
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
  long long left = min(chunk, total - from);  // tiles of this worker
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
    c.unit = u;
    c.len = length_of(p.c, u);
    const long long in = from - at;
    c.block = static_cast<int>(in / n);
    c.tile = static_cast<int>(in - static_cast<long long>(c.block) * n);
  }

  constexpr uint32_t kBytes = 2 * kCodeTile + 2 * kParamTile + (kPos ? kPosTile : 0);
  Place ahead = c;
  long long to_issue = left;
  auto issue = [&](int stage) {
    if (lane == 0) {
      const uint32_t bar = bars + 8 * stage, cd = codes + stage * 2 * kCodeTile, sd = side + stage * kSideBytes;
      const long long row = static_cast<long long>(ahead.unit) * p.c.capacity + ahead.tile * kQ4TileSlots;
      mbar_arrive_expect_tx(bar, kBytes);
      tma_rows(cd, &p.map_k, bar, static_cast<int>(row));
      tma_rows(cd + kCodeTile, &p.map_v, bar, static_cast<int>(row));
      bulk_copy(sd, p.c.params[0] + row * kQ4ParamBytes, kParamTile, bar);
      bulk_copy(sd + kParamTile, p.c.params[1] + row * kQ4ParamBytes, kParamTile, bar);
      if (kPos) bulk_copy(sd + 2 * kParamTile, p.c.positions + row, kPosTile, bar);
    }
    --to_issue;
    if (to_issue > 0) ahead.next(p, units);
  };
  for (int i = 0; i < S::kStages && to_issue > 0; ++i) issue(i);

  // ldmatrix row of this lane: slot lane & 7, piece lane >> 3 of its 64 bytes,
  // stored at piece ^ (slot / 2) by the 64-byte swizzle
  const uint32_t mat = (lane & 7) * kQ4CodeBytes + (((lane >> 3) ^ ((lane >> 1) & 3)) << 4);

  Queries<NB> Q;
  float o[NB][4][2][4];   // [8 rows][group][step][channel, row pair]
  float om[NB][4];        // minima's term (lanes of g >= 4)
  float ref[NB], l[NB];
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
        ref[nb] = -INFINITY;
        l[nb] = 0.f;
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
    const int slot0 = c.tile * kQ4TileSlots, valid = c.len - slot0;

    // ---- scales of V: the largest of the tile; NaN groups and slots behind
    // the length are taken out (their codes then count nothing)
    uint32_t nan_groups = 0;  // lane = slot: groups that hold a NaN
    uint32_t special = 0;
    {
      uint4 w = lds128(sd + kParamTile + lane * kQ4ParamBytes);
      uint32_t top = max(max(w.x << 16, w.x & 0xffff0000u), max(w.y << 16, w.y & 0xffff0000u));
      const uint32_t mz = w.z & 0x7fff7fffu, mw = w.w & 0x7fff7fffu;
      const uint32_t mtop = max(max(mz << 16, mz & 0xffff0000u), max(mw << 16, mw & 0xffff0000u));
      uint32_t both = max(top, mtop);
      if (lane >= valid) both = 0xffffffffu;
      special = __any_sync(0xffffffffu, both >= 0x7f800000u);
      if (special) {
        uint32_t s[4] = {w.x & 0xffffu, w.x >> 16, w.y & 0xffffu, w.y >> 16};
        uint32_t m[4] = {w.z & 0xffffu, w.z >> 16, w.w & 0xffffu, w.w >> 16};
        top = 0;
#pragma unroll
        for (int J = 0; J < 4; ++J) {
          const bool bad = (s[J] & 0x7fffu) >= 0x7f80u || (m[J] & 0x7fffu) >= 0x7f80u;
          if (bad && lane < valid) nan_groups |= 1u << J;
          if (bad || lane >= valid) s[J] = m[J] = 0u;
          top = max(top, s[J] << 16);
        }
        w = make_uint4(s[0] | s[1] << 16, s[2] | s[3] << 16, m[0] | m[1] << 16, m[2] | m[3] << 16);
        sts128(sd + kParamTile + lane * kQ4ParamBytes, w);
        __syncwarp();
      }
      const int k = max(static_cast<int>(__reduce_max_sync(0xffffffffu, top) >> 23) - 127, kMinScaleExp);
      if (k > vexp) {  // the codes' sums go to the new power of two
        const float f = pow2(max(vexp - k, -126));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int J = 0; J < 4; ++J)
#pragma unroll
            for (int st = 0; st < 2; ++st)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[nb][J][st][i] *= f;
        vexp = k;
      }
    }

    // ---- logits: four times 8 slots
    float z[NB][4][2];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      uint32_t w[4];
      ldmatrix4(w, cd + n * 8 * kQ4CodeBytes + mat);
      const uint32_t mins = lds32(sd + (n * 8 + g) * kQ4ParamBytes + 8 + (t & 1) * 4);
      float acc[4] = {0.f, 0.f, 0.f, 0.f};
      mma_bf16(acc, Q.sum[0][0], NB > 1 ? Q.sum[NB - 1][0] : 0u, Q.sum[0][1],
               NB > 1 ? Q.sum[NB - 1][1] : 0u, mins, mins);
      const uint2 sa = lds64(sd + (n * 8 + 2 * t) * kQ4ParamBytes);
      const uint2 sb = lds64(sd + (n * 8 + 2 * t + 1) * kQ4ParamBytes);
#pragma unroll
      for (int J = 0; J < 4; ++J) {
        float x[4] = {0.f, 0.f, 0.f, 0.f};
        const uint32_t hi = w[J] >> 8;
        mma_f16(x, Q.a[0][0][2 * J], NB > 1 ? Q.a[NB - 1][0][2 * J] : 0u, Q.a[0][1][2 * J],
                NB > 1 ? Q.a[NB - 1][1][2 * J] : 0u, w[J] & 0x000f000fu, w[J] & 0x00f000f0u);
        mma_f16(x, Q.a[0][0][2 * J + 1], NB > 1 ? Q.a[NB - 1][0][2 * J + 1] : 0u, Q.a[0][1][2 * J + 1],
                NB > 1 ? Q.a[NB - 1][1][2 * J + 1] : 0u, hi & 0x000f000fu, hi & 0x00f000f0u);
        const uint32_t wa = J < 2 ? sa.x : sa.y, wb = J < 2 ? sb.x : sb.y;
        const float s0 = J & 1 ? bf_hi(wa) : bf_lo(wa), s1 = J & 1 ? bf_hi(wb) : bf_lo(wb);
        acc[0] = fmaf(x[0], s0, acc[0]);
        acc[1] = fmaf(x[1], s1, acc[1]);
        if (NB > 1) {
          acc[2] = fmaf(x[2], s0, acc[2]);
          acc[3] = fmaf(x[3], s1, acc[3]);
        }
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        z[nb][n][0] = acc[2 * nb] * Q.f1 * Q.f2[nb];
        z[nb][n][1] = acc[2 * nb + 1] * Q.f1 * Q.f2[nb];
      }
      if (kPos) {
        const uint2 at = lds64(sd + 2 * kParamTile + (n * 8 + 2 * t) * 4);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          if (static_cast<int>(at.x) > Q.limit[nb]) z[nb][n][0] = -INFINITY;
          if (static_cast<int>(at.y) > Q.limit[nb]) z[nb][n][1] = -INFINITY;
        }
      }
    }
    if (valid < kQ4TileSlots) {
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (n * 8 + 2 * t + i >= valid)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) z[nb][n][i] = -INFINITY;
    }
    if (p.accumulate) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int r = c.block * (8 * NB) + nb * 8 + g;
        if (r < p.rows) {
          float2* zp = reinterpret_cast<float2*>(
              p.z + (static_cast<long long>(c.unit) * p.rows + r) * p.c.capacity + slot0 + 2 * t);
#pragma unroll
          for (int n = 0; n < 4; ++n) zp[n * 4] = make_float2(z[nb][n][0], z[nb][n][1]);
        }
      }
    }

    // ---- references, probabilities (in place of z)
    uint32_t seen_nan = 0;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float top = -INFINITY;
#pragma unroll
      for (int n = 0; n < 4; ++n) top = fmaxf(top, fmaxf(z[nb][n][0], z[nb][n][1]));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const bool raise = top > ref[nb] + kRaise;
      if (__any_sync(0xffffffffu, raise)) {
        const float f = raise ? (ref[nb] == -INFINITY ? 0.f : ex2_approx(ref[nb] - top)) : 1.0f;
        if (raise) ref[nb] = top;
        l[nb] *= f;
        // rows 2t and 2t + 1 are this lane's columns of the outputs
        const float f0 = __shfl_sync(0xffffffffu, f, 8 * t), f1 = __shfl_sync(0xffffffffu, f, 8 * t + 4);
#pragma unroll
        for (int J = 0; J < 4; ++J)
#pragma unroll
          for (int st = 0; st < 2; ++st) {
            o[nb][J][st][0] *= f0;
            o[nb][J][st][1] *= f1;
            o[nb][J][st][2] *= f0;
            o[nb][J][st][3] *= f1;
          }
        om[nb][0] *= f0;
        om[nb][1] *= f1;
      }
      if (special) {
        // rows that see a slot's NaN group
        uint32_t hit = 0;
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t m = __shfl_sync(0xffffffffu, nan_groups, n * 8 + 2 * t + i);
            if (z[nb][n][i] != -INFINITY) hit |= m;
          }
        hit |= __shfl_xor_sync(0xffffffffu, hit, 1);
        hit |= __shfl_xor_sync(0xffffffffu, hit, 2);
        seen_nan |= hit << (4 * nb);
      }
      const float r = ref[nb] == -INFINITY ? 0.f : ref[nb];
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          z[nb][n][i] = ex2_approx(z[nb][n][i] - r);
          l[nb] += z[nb][n][i];
        }
    }

    // ---- outputs: twice 16 slots
    const float inv = pow2(kTopExp - vexp);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int s16 = h * 16;
      uint32_t va[4], vb[4], pm[4];
      ldmatrix4_t(va, cd + kCodeTile + s16 * kQ4CodeBytes + mat);
      ldmatrix4_t(vb, cd + kCodeTile + (s16 + 8) * kQ4CodeBytes + mat);
      // params as 8x8 matrices of slots x (scales, minima): rows 4-7 of the
      // transposed operand are the minima (lanes 16-31 repeat the addresses)
      ldmatrix4_t(pm, sd + kParamTile + (s16 + (lane & 15)) * kQ4ParamBytes);
      const uint2 s0 = lds64(sd + kParamTile + (s16 + 2 * t) * kQ4ParamBytes);
      const uint2 s1 = lds64(sd + kParamTile + (s16 + 2 * t + 1) * kQ4ParamBytes);
      const uint2 s2 = lds64(sd + kParamTile + (s16 + 8 + 2 * t) * kQ4ParamBytes);
      const uint2 s3 = lds64(sd + kParamTile + (s16 + 9 + 2 * t) * kQ4ParamBytes);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const float p0 = z[nb][2 * h][0], p1 = z[nb][2 * h][1];
        const float p2 = z[nb][2 * h + 1][0], p3 = z[nb][2 * h + 1][1];
        const uint32_t h0 = pack_bf16(p0, p1), h1 = pack_bf16(p2, p3);
        mma_bf16(om[nb], pm[0], 0u, pm[1], 0u, h0, h1);
        mma_bf16(om[nb], pm[0], 0u, pm[1], 0u, pack_bf16(p0 - bf_lo(h0), p1 - bf_hi(h0)),
                 pack_bf16(p2 - bf_lo(h1), p3 - bf_hi(h1)));
        const float q0 = p0 * inv, q1 = p1 * inv, q2 = p2 * inv, q3 = p3 * inv;
#pragma unroll
        for (int J = 0; J < 4; ++J) {
          const uint32_t w0 = J < 2 ? s0.x : s0.y, w1 = J < 2 ? s1.x : s1.y;
          const uint32_t w2 = J < 2 ? s2.x : s2.y, w3 = J < 2 ? s3.x : s3.y;
          const uint32_t b0 = J & 1 ? pack_half2(q0 * bf_hi(w0), q1 * bf_hi(w1))
                                    : pack_half2(q0 * bf_lo(w0), q1 * bf_lo(w1));
          const uint32_t b1 = J & 1 ? pack_half2(q2 * bf_hi(w2), q3 * bf_hi(w3))
                                    : pack_half2(q2 * bf_lo(w2), q3 * bf_lo(w3));
          const uint32_t ah = va[J] >> 8, bh = vb[J] >> 8;
          mma_f16(o[nb][J][0], va[J] & 0x000f000fu, va[J] & 0x00f000f0u, vb[J] & 0x000f000fu,
                  vb[J] & 0x00f000f0u, b0, b1);
          mma_f16(o[nb][J][1], ah & 0x000f000fu, ah & 0x00f000f0u, bh & 0x000f000fu, bh & 0x00f000f0u,
                  b0, b1);
        }
      }
    }
    if (special) {
      const float bad = __uint_as_float(0x7fc00000u);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const uint32_t h0 = __shfl_sync(0xffffffffu, seen_nan, 8 * t) >> (4 * nb);
        const uint32_t h1 = __shfl_sync(0xffffffffu, seen_nan, 8 * t + 4) >> (4 * nb);
#pragma unroll
        for (int J = 0; J < 4; ++J)
#pragma unroll
          for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (((i & 1 ? h1 : h0) >> J) & 1u) o[nb][J][st][i] = bad;
      }
    }
    if (special) fence_proxy_async_smem();  // (it wrote to the stage)
    __syncwarp();  // every lane is done with the stage
    if (to_issue > 0) issue(stage);
    if (++stage == S::kStages) {
      stage = 0;
      phase ^= 1u;
    }

    // ---- the row block ends here, or this worker's share of it
    const int unit = c.unit, block = c.block;
    if (left > 1) c.next(p, units);
    if (left == 1 || c.unit != unit || c.block != block) {
      const long long part = static_cast<long long>(worker) + static_cast<long long>(unit) * p.blocks + block;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float sum = l[nb];
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        if (t == 0) p.part_ml[part * (8 * NB) + nb * 8 + g] = make_float2(ref[nb], sum);
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
            v.x = fmaf(o[nb][J][0][i] * 16777216.0f, f, m);
            v.y = fmaf(o[nb][J][0][2 + i] * 1048576.0f, f, m);
            v.z = fmaf(o[nb][J][1][i] * 16777216.0f, f, m);
            v.w = fmaf(o[nb][J][1][2 + i] * 1048576.0f, f, m);
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
