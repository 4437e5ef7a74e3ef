// Attention of a few query tokens a sequence over the 4-bit cache.
//
//   z[r,j] = scale * sum_c q[r,c] (s n[j,c] + m),   p = softmax over the visible slots
//   out[r] = sum_j p[r,j] (s n[j,:] + m),   lse[r] = log sum_j exp z[r,j]
//   weight[j] += sum_r p[r,j]   (where asked for)
//
// 160 bytes a slot against at most a few thousand operations, so the kernel is
// built around a steady stream of slots and few instructions a code.  Every
// warp takes a run of tiles of 64 slots (see Q4AttendParams) and keeps two in
// flight with TMA into its own part of shared memory.  A row block that lies in
// its run it finishes itself; of others it leaves the softmax reference, sum and
// outputs, which its CTA joins, and for row blocks that several CTAs share the
// last of them to come, always in slot order.
//
// Measured, in a graph of 20 calls: four sequences of 128K slots, 8 groups of 4
// heads, 134 us, 5.0 TB/s of the 6.78 that a copy reaches (the loads alone
// take 108): two warps a scheduler issue in 46 % of the cycles, the tensor cores
// are busy in 30 %.  One sequence of 32K slots 18.9 us and of 777 10.3, where
// fixed latencies add up: the scan of the lengths (1 us), the first copies and
// the queries (2), the first tile with no instruction cached (2), the joins in a
// CTA and over CTAs (2 to 5).  64 sequences of 1000 to 8000 slots, 8 groups of 8
// heads, f16, with weights, 125 us against 56 for the bytes: instructions.
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
//     power of two a row so that the largest element is in [2^14, 2^15), odd
//     channels by 1/16 of it: bf16 elements are exact down to 2^-31 of the largest
//     (even channels) and 2^-27 (odd ones), f16 ones to 2^-28 and 2^-24, and smaller
//     ones off by at most 2^-39 and 2^-35 of it); the four groups are summed apart and
//     scaled by their s in fp32.  The minima's term sum_J m_J (sum of q over J)
//     is one more product: the group sums as three bf16 parts (24 bits), m in bf16.
//   O^T = V^T P^T: A = codes of 16 channels, B = P^T, which movmatrix makes of
//     the result layout of S^T.  With c = n - 7.5 and the group's middle
//     m + 7.5 s, out = sum p s c + sum p (m + 7.5 s): both terms stay as small as
//     the output does where many slots share the attention.  (With n and m they
//     grow with sum p; the tensor cores truncate their sums, so that at 128K slots
//     3 % of the output were lost.)  The 7.5 comes off once a tile, as 7.5 sum p s.
//     p is fp16 (off by at most 2^-11 of itself), the weights of group J's codes are
//     p s_J, rounded once more, whose sum is a product with ones; the middles' term
//     is a product of its own, with p, whose operand has rows to spare: what rounding
//     a middle to fp16 left is in the second eight.  (Where one channel is 30 or 100
//     times wider than the others, the middles are large against the output: rounded
//     once they cost f16 outputs 2 to 9 times their own rounding, bf16 1.3 to 2.4.)
//     For f16 outputs (kFine) what rounding p and p s left is a second operand; sum
//     p s is then exact and comes with the middles' product before the codes', so
//     that it comes off half way, where the truncation before and after it cancels.
//     Error 2.1e-4 of the output, all of it the output's own rounding (2.7e-4 at
//     128K slots), where one rounding of p s gave 3.0e-4 and two 3.6e-4.  bf16
//     outputs, whose rounding is eight times that, keep single roundings: second
//     operands took 153 us for 133 at 128K x 4 slots, and the error is within 2 % of
//     the output's own rounding (15 % where a channel is 100 times wider).
//     Scales (exactly) and middles enter fp16 against a power of
//     two 2^e of the slot's own, which goes to the weights: p 2^e, times a power of
//     two of the row's (its gain) that follows the largest of them.  What a row does
//     not see, or hardly attends to, then costs the rest no bits, however large
//     it is.  A weight below 2^-16 of the row's largest is off by 2^-27 of that one,
//     and a scale below 2^-20 of the largest magnitude in its row of V loses bits.
// Eight lanes of a warp need the same slot's scales, so one lane converts them
// for all (K: times the softmax scale in fp32; V: fp16 pairs of slots) and
// leaves them in shared memory.
// Softmax references are raised only when a logit passes them by 2^8, so the
// outputs are hardly ever rescaled.
#include <cuda_runtime.h>

#include <type_traits>

#include "ckv_device.cuh"
#include "q4_params.h"
#include "q4_ring.h"

namespace ckv {

namespace {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kRaise = 8.0f;         // references lag behind the largest logit by at most this
constexpr float kLift = 3.0f;          // probabilities are held times 2^3: at most 2^11
constexpr int kTopExp = 3;             // a slot's scales become < 1, its middles < 2^5
constexpr uint32_t kOnes = 0x3c003c00u;  // fp16, twice
constexpr float kMiddle = 7.5f / 16777216.0f;  // of the codes, as they are held
constexpr int kMinScaleExp = -110;     // rows of smaller scales and minima share this exponent
constexpr float kTopWeight = 32768.0f; // of weights p 2^e: w s < 2^15
constexpr int kExpOff = 12;            // a slot's 2^e is held as 2^(e - 12): p 2^(e - 12) < 2^127
constexpr int kMaxGain = 122;          // weights are p 2^(e - 12) times 2^gain

// A row block of up to two tiles a warp is one CTA's; longer ones are shared,
// by CTAs of at least four tiles.  Joining over CTAs costs about 3 us, a warp's
// further tile 2.5.  Eight units of 777 slots (two tiles a warp): 10.4 us, and
// 11.2 shared; of 2048 slots (four): 16.0 on one CTA each, 11.2 shared; of 4096
// slots by CTAs of 2, 4, 8 and 16 tiles: 11.4, 11.3, 12.0 and 14.5 us.  64 units of
// 2048 slots: 14.7 us shared, 16.7 on one CTA each.
constexpr int kMinTiles = 4;
constexpr int kSoloTiles = 2;

// Eight warps of 64 slots a step with the next 64 on their way: 183 KB a CTA.
// More warps of fewer slots issue more instructions a slot: measured when V's
// exponents were not yet a slot's own, for four sequences of 128K slots 127.5 us,
// and 147 with 12 warps of 32, 140 with 16 and 175 with 8; for one of 777 slots
// 9.8, and 10.1, 10.8 and 11.4.
// A warp's stage holds the codes of K and V (swizzled); their params and the
// positions lie in an area of their own.
template <int NB>
struct Shape {
  static constexpr int kTile = kQ4Tile;
  static constexpr int kWarps = kQ4Warps;
  static constexpr int kStages = 2;
  static constexpr int kThreads = kWarps * 32;
  static constexpr int kSteps = kTile / 16;
  static constexpr int kCodeTile = kTile * kQ4CodeBytes;
  static constexpr int kParamTile = kTile * kQ4ParamBytes;
  static constexpr int kSideBytes = 2 * kParamTile + kTile * 4;
  static constexpr int kScaleTile = kTile * 16;  // K's scales of the tile at hand, fp32
  static constexpr int kCodes = kWarps * kStages * 2 * kCodeTile;
  static constexpr int kSide = kWarps * kStages * kSideBytes;
  static constexpr int kPairTile = kTile * 16;   // V's scales by pairs of slots, rests of its middles, fp16
  static constexpr int kExpTile = kTile * 4;     // 2^(e - 12) of its slots, fp32
  static constexpr int kScales = kWarps * (kScaleTile + kPairTile + kExpTile);
  static constexpr int kSmem = 1024 + kCodes + kSide + kScales + kWarps * kStages * 8 + 8;
  static constexpr int kLane = (kTile + 31) / 32;  // slots a lane prepares
  static_assert(kTile % 16 == 0, "steps");
  static_assert(kCodeTile % 512 == 0, "swizzle");
  static_assert(kStages * 2 * kCodeTile >= 8 * NB * kHeadDim * 4, "a warp's outputs fit its stages");
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
// 1 / x of a sum of probabilities; 0 where there are none.
__device__ __forceinline__ float inverse(float x) { return x == 0.f ? 0.f : 1.0f / x; }
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
// What rounding a and b to the pair h of fp16 numbers left, as another pair.
__device__ __forceinline__ uint32_t half_rest(float a, float b, uint32_t h) {
  return pack_half2(a - to_float(h & 0xffffu, false), b - to_float(h >> 16, false));
}
__device__ __forceinline__ uint32_t mul_half2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t fma_half2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
// a *= x, b *= y in one instruction.
__device__ __forceinline__ void mul_pair(float& a, float& b, float x, float y) {
  asm("{\n\t.reg .b64 s, t;\n\tmov.b64 s, {%0, %1};\n\tmov.b64 t, {%2, %3};\n\t"
      "mul.rn.f32x2 s, s, t;\n\tmov.b64 {%0, %1}, s;\n\t}"
      : "+f"(a), "+f"(b)
      : "f"(x), "f"(y));
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
__device__ __forceinline__ void sts32(uint32_t a, uint32_t x) {
  asm volatile("st.shared.b32 [%0], %1;" ::"r"(a), "r"(x) : "memory");
}
__device__ __forceinline__ void tma_rows(uint32_t dst, const CUtensorMap* map, uint32_t bar, int row,
                                         uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], "
      "[%1, {%3, %4}], [%2], %5;" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(0), "r"(row), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar,
                                          uint64_t policy) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(
          dst),
      "l"(src), "r"(bytes), "r"(bar), "l"(policy)
      : "memory");
}
__device__ __forceinline__ uint64_t l2_policy_normal() {
  uint64_t p;
  asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(p));
  return p;
}

// (An ordinary load: the read-only path is for what nobody writes while the
// kernel is there, and this one may be brought up while the append still runs.)
__device__ __forceinline__ int length_of(const Q4Cache& c, int unit) {
  return min(max(c.lengths[unit], 0), c.capacity);
}
template <int kTile>
__device__ __forceinline__ int tiles_of(const Q4Cache& c, int unit) {
  return (length_of(c, unit) + kTile - 1) / kTile;
}

// A tile's place in the sequence of tiles.
struct Place {
  int unit, block;
  int row;    // slot row of the cache: unit * capacity + first slot
  int valid;  // slots in use from there on
  // The next tile; past the end of a row block the next one that has tiles
  // (the caller knows that there is one).
  template <int kTile>
  __device__ __forceinline__ void next(const Q4AttendParams& p) {
    row += kTile;
    valid -= kTile;
    if (valid > 0) return;
    if (++block == p.blocks) {
      block = 0;
      ++unit;
    }
    // (never past the last unit, whatever the lengths become meanwhile)
    const int last = p.c.batch * p.c.num_kv_heads - 1;
    unit = min(unit, last);
    while ((valid = length_of(p.c, unit)) == 0 && unit < last) ++unit;
    row = unit * p.c.capacity;
  }
};

// Inclusive prefix over a warp.
__device__ __forceinline__ int warp_prefix(int x, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  return x;
}

// The largest of 16 s and |m| of a params row, as the bits of a float (whose
// order is that of the numbers; NaN above all).
__device__ __forceinline__ uint32_t top_of(uint4 w) {
  const uint32_t s = max(max(w.x << 16, w.x & 0xffff0000u), max(w.y << 16, w.y & 0xffff0000u)) + (4u << 23);
  const uint32_t z = max((w.z << 16) & 0x7fff0000u, w.z & 0x7fff0000u);
  return max(s, max(z, max((w.w << 16) & 0x7fff0000u, w.w & 0x7fff0000u)));
}

// What a warp leaves of a row block that it shares with others.
struct Part {
  int block;        // unit * blocks + row block, or -1
  int count;        // tiles of the row block
  int first;        // its first tile
  bool starts, ends;
};

__device__ __forceinline__ void write_row(const Q4AttendParams& p, int unit, int row, int lane, float4 v,
                                          float ref, float sum);

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
    uint4 raw[4];
    int limit = 0x7fffffff;
    uint32_t abs2 = 0;  // largest magnitudes of the low and of the high halves
    if (r < p.rows) {
      const int h = kv * p.group + r / p.num_queries, qi = r % p.num_queries;
      const uint16_t* src = p.q + b * p.q_bs + h * p.q_hs + qi * p.q_qs + 8 * t;
      if (p.q_positions) limit = __ldg(p.q_positions + b * p.num_queries + qi);
#pragma unroll
      for (int J = 0; J < 4; ++J) raw[J] = __ldg(reinterpret_cast<const uint4*>(src + 32 * J));
    } else {
#pragma unroll
      for (int J = 0; J < 4; ++J) raw[J] = make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int J = 0; J < 4; ++J) {
      // (magnitudes compare like their bits, NaN above all)
      abs2 = __vmaxu2(abs2, __vmaxu2(raw[J].x & 0x7fff7fffu, raw[J].y & 0x7fff7fffu));
      abs2 = __vmaxu2(abs2, __vmaxu2(raw[J].z & 0x7fff7fffu, raw[J].w & 0x7fff7fffu));
    }
    abs2 = __vmaxu2(abs2, __shfl_xor_sync(0xffffffffu, abs2, 1));
    abs2 = __vmaxu2(abs2, __shfl_xor_sync(0xffffffffu, abs2, 2));
    const uint32_t top = __float_as_uint(to_float(max(abs2 & 0xffffu, abs2 >> 16), bf16));
    // exponent of the largest element; a row of zeros, NaN or infinities as it is
    int e = top >= 0x7f800000u || top == 0 ? 14 : static_cast<int>(top >> 23) - 127;
    e = max(e, -110);  // smaller rows (bf16) scale by no more than 2^124
    const float up = pow2(14 - e), up16 = up * 0.0625f;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      Q.f2[nb][j] = __shfl_sync(0xffffffffu, pow2(e), 8 * t + 4 * j);
      Q.limit[nb][j] = __shfl_sync(0xffffffffu, limit, 8 * t + 4 * j);
    }
    float part[4];
#pragma unroll
    for (int J = 0; J < 4; ++J) {
      const uint32_t w[4] = {raw[J].x, raw[J].y, raw[J].z, raw[J].w};
      float even = 0.f, odd = 0.f;
      // nibbles (0, 4), (1, 5), (2, 6), (3, 7) of a word; the odd ones count 16-fold
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const float a0 = to_float(w[st] & 0xffffu, bf16) * up, a1 = to_float(w[st + 2] & 0xffffu, bf16) * up;
        const float b0 = to_float(w[st] >> 16, bf16) * up16, b1 = to_float(w[st + 2] >> 16, bf16) * up16;
        Q.b[nb][2 * J + st][0] = pack_half2(a0, a1);
        Q.b[nb][2 * J + st][1] = pack_half2(b0, b1);
        even += a0 + a1;
        odd += b0 + b1;
      }
      part[J] = fmaf(odd, 16.0f, even);
      part[J] += __shfl_xor_sync(0xffffffffu, part[J], 1);
      part[J] += __shfl_xor_sync(0xffffffffu, part[J], 2);
      part[J] *= 5.9604644775390625e-8f * f1;  // 2^-24
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

// kPos: slots are seen by position.  kFine: f16 outputs, whose rounding is as
// small as that of the weights, which then have a second part.
template <int NB, bool kPos, bool kFine>
__global__ void __launch_bounds__(Shape<NB>::kThreads, 1)
    attend_kernel(const __grid_constant__ Q4AttendParams p) {
  using S = Shape<NB>;
  constexpr int kRows = 8 * NB;
  constexpr int kTile = S::kTile, kSteps = S::kSteps;
  constexpr int kCodeTile = S::kCodeTile, kParamTile = S::kParamTile, kSideBytes = S::kSideBytes;
  constexpr int kScaleTile = S::kScaleTile, kPairTile = S::kPairTile, kExpTile = S::kExpTile, kLane = S::kLane;
  extern __shared__ uint8_t smem_raw[];
  __shared__ int s_sums[S::kWarps], s_unit[S::kWarps], s_at[S::kWarps], s_abort;
  __shared__ float2 s_ml[S::kWarps][kRows];
  __shared__ Part s_tail[S::kWarps], s_head[S::kWarps];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, t = lane & 3;
  const uint32_t codes = base + warp * S::kStages * 2 * kCodeTile;
  const uint32_t side = base + S::kCodes + warp * S::kStages * kSideBytes;
  const uint32_t scales = base + S::kCodes + S::kSide + warp * (kScaleTile + kPairTile + kExpTile);
  const uint32_t pairs = scales + kScaleTile, exps = pairs + kPairTile;
  const uint32_t bars = base + S::kCodes + S::kSide + S::kScales + warp * S::kStages * 8;
  const uint32_t never = base + S::kSmem - 1024 - 8;  // the test hook's stall waits for it
  if (lane == 0) {
    for (int i = 0; i < S::kStages; ++i) mbar_init(bars + 8 * i, 1);
    s_tail[warp].block = s_head[warp].block = -1;
  }
  if (threadIdx.x == 0) {
    s_abort = 0;
    mbar_init(never, 1);
    tma_prefetch_map(&p.map_k);
    tma_prefetch_map(&p.map_v);
  }
  fence_mbar_init();
  __syncthreads();  // (the others' parts and the abort flag)
  pdl_wait();  // everything before is of this launch alone
  if (p.accumulate) pdl_launch_dependents();  // the weights' kernel, which waits for this one

  // ---- this CTA's tiles, and this warp's share of them.  (The host bounds the
  // tiles by 2^30.)
  const int units = p.c.batch * p.c.num_kv_heads, ctas = gridDim.x;
  int chunk = 0, tile = 0, left = 0;  // tiles of a CTA; this warp's first tile, and how many
  int unit0 = 0, at = 0;              // the unit that holds it, and that unit's first tile
  int own0 = -1;                      // first of the CTAs that have a row block to themselves
  auto share_out = [&](int from, int count) {
    const int share = (chunk + S::kWarps - 1) / S::kWarps;
    tile = from + warp * share;
    left = max(0, min(share, count - warp * share));
  };
  // CTAs take equal runs of the whole sequence of tiles, at least kMinTiles
  auto even_chunk = [&](int total) { return max((total + ctas - 1) / ctas, kMinTiles); };
  constexpr int kPer = 4;
  if (units <= 32 * kPer) {
    // every warp for itself: kPer units a lane
    int n[kPer], mine = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int u = lane * kPer + k;
      n[k] = u < units ? tiles_of<kTile>(p.c, u) : 0;
      mine += n[k];
    }
    const int incl = warp_prefix(mine, lane), total = __shfl_sync(0xffffffffu, incl, 31) * p.blocks;
    chunk = even_chunk(total);
    // Where the row blocks come out about even over whole CTAs, each has its
    // own: one where it is short, else in proportion.  No CTA then joins the end
    // of one row block and the start of another (8 units of 300 slots: 7.7 us, and
    // 10.4 in equal runs; of 32K slots 19.1 and 22.7).
    // (Quotients in fp32: every warp takes the same ones, near enough.)
    int own[kPer], own_mine = 0, own_chunk = 0;
    const float rate = __fdividef(static_cast<float>(ctas), static_cast<float>(total));
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int share = min(static_cast<int>(fmaf(n[k], rate, 1e-3f)), (n[k] + kMinTiles - 1) / kMinTiles);
      own[k] = n[k] <= kSoloTiles * S::kWarps ? min(n[k], 1) : max(1, share);
      own_mine += own[k] * p.blocks;
      if (own[k]) own_chunk = max(own_chunk, static_cast<int>(__fdividef(n[k], own[k])));
    }
    const int own_incl = warp_prefix(own_mine, lane);
    own_chunk = __reduce_max_sync(0xffffffffu, own_chunk);
    if (__shfl_sync(0xffffffffu, own_incl, 31) <= ctas &&
        own_chunk <= max(kSoloTiles * S::kWarps, chunk + chunk / 8 + 1)) {
      const unsigned holds = __ballot_sync(0xffffffffu, own_incl > static_cast<int>(blockIdx.x));
      int u = 0, rest = static_cast<int>(blockIdx.x) - (own_incl - own_mine), before = incl - mine, c = 0, count = 0;
      bool found = false;
#pragma unroll
      for (int k = 0; k < kPer; ++k)
        if (!found) {
          if (rest < own[k] * p.blocks) {
            found = true;
            u = lane * kPer + k;
            c = own[k];
            count = n[k];
          } else {
            rest -= own[k] * p.blocks;
            before += n[k];
          }
        }
      const int src = holds ? __ffs(holds) - 1 : 0;
      unit0 = __shfl_sync(0xffffffffu, u, src);
      rest = __shfl_sync(0xffffffffu, rest, src);
      c = __shfl_sync(0xffffffffu, c, src);
      count = __shfl_sync(0xffffffffu, count, src);
      at = __shfl_sync(0xffffffffu, before, src) * p.blocks;
      chunk = 1;
      if (holds && c > 0) {
        const int block = rest / c, index = rest - block * c;
        chunk = (count + c - 1) / c;
        own0 = static_cast<int>(blockIdx.x) - index;
        share_out(at + block * count + index * chunk, min(chunk, count - index * chunk));
      }
    } else {
      const int from = static_cast<int>(blockIdx.x) * chunk;
      share_out(from, min(chunk, total - from));
      // the lane that holds the first tile, then the unit of that lane
      const unsigned holds = __ballot_sync(0xffffffffu, incl * p.blocks > tile);
      int before = incl - mine, u = lane * kPer;
#pragma unroll
      for (int k = 0; k < kPer - 1; ++k)
        if (u == lane * kPer + k && (before + n[k]) * p.blocks <= tile) {
          before += n[k];
          ++u;
        }
      const int src = holds ? __ffs(holds) - 1 : 0;
      unit0 = __shfl_sync(0xffffffffu, u, src);
      at = __shfl_sync(0xffffffffu, before, src) * p.blocks;
    }
  } else {
    const int span = (units + S::kThreads - 1) / S::kThreads;  // units a thread adds up
    const int u0 = min(static_cast<int>(threadIdx.x) * span, units), u1 = min(u0 + span, units);
    int mine = 0;
    for (int u = u0; u < u1; ++u) mine += tiles_of<kTile>(p.c, u);
    int incl = warp_prefix(mine, lane);
    if (lane == 31) s_sums[warp] = incl;
    __syncthreads();
    int total = 0;
    for (int w = 0; w < S::kWarps; ++w) {
      if (w < warp) incl += s_sums[w];
      total += s_sums[w];
    }
    const int before = (incl - mine) * p.blocks;
    total *= p.blocks;
    chunk = even_chunk(total);
    const int from = static_cast<int>(blockIdx.x) * chunk;
    share_out(from, min(chunk, total - from));
    // the thread that holds a warp's first tile
    const int share = (chunk + S::kWarps - 1) / S::kWarps;
    const int first = tile - warp * share;
    for (int w = 0; w < S::kWarps; ++w)
      if (first + w * share >= before && first + w * share < before + mine * p.blocks) {
        s_unit[w] = u0;
        s_at[w] = before;
      }
    __syncthreads();
    if (left > 0) {
      unit0 = s_unit[warp];
      at = s_at[warp];
      int n;
      while (at + (n = tiles_of<kTile>(p.c, unit0)) * p.blocks <= tile && unit0 < units - 1) {
        at += n * p.blocks;
        ++unit0;
      }
    }
  }
  Place c = {};
  if (left > 0) {
    unit0 = min(unit0, units - 1);
    const int len = length_of(p.c, unit0), n = max(1, (len + kTile - 1) / kTile);
    c.unit = unit0;
    c.block = min((tile - at) / n, p.blocks - 1);
    const int slot = min(tile - at - c.block * n, n - 1) * kTile;
    c.row = unit0 * p.c.capacity + slot;
    c.valid = len - slot;
  }

  // logits that are read again stay in L2 in preference to the cache's rows
  const uint64_t policy = p.accumulate ? l2_policy_evict_first() : l2_policy_normal();
  Place ahead = c;
  int to_issue = left;
  auto issue = [&](int stage) {
    if (lane == 0) {
      const uint32_t bar = bars + 8 * stage, cd = codes + stage * 2 * kCodeTile, sd = side + stage * kSideBytes;
      // the capacity may end in the middle of the tile; codes of the next unit
      // (or zeros, behind the last one) then come along and count nothing
      const int slots = min(kTile, (ahead.unit + 1) * p.c.capacity - ahead.row);
      mbar_arrive_expect_tx(bar, 2 * kCodeTile + slots * (2 * kQ4ParamBytes + (kPos ? 4 : 0)));
      tma_rows(cd, &p.map_k, bar, ahead.row, policy);
      tma_rows(cd + kCodeTile, &p.map_v, bar, ahead.row, policy);
      const size_t row = static_cast<size_t>(ahead.row);
      bulk_copy(sd, p.c.params[0] + row * kQ4ParamBytes, slots * kQ4ParamBytes, bar, policy);
      bulk_copy(sd + kParamTile, p.c.params[1] + row * kQ4ParamBytes, slots * kQ4ParamBytes, bar, policy);
      if (kPos) bulk_copy(sd + 2 * kParamTile, p.c.positions + row, slots * 4, bar, policy);
    }
    if (--to_issue > 0) ahead.template next<S::kTile>(p);
  };
  for (int i = 0; i < S::kStages && to_issue > 0; ++i) issue(i);


  // ldmatrix row of this lane: slot lane & 7, piece lane >> 3 of its 64 bytes,
  // stored at piece ^ (slot / 2) by the 64-byte swizzle
  const uint32_t mat = (lane & 7) * kQ4CodeBytes + (((lane >> 3) ^ ((lane >> 1) & 3)) << 4);
  // ... and for one group of 32 slots: slot lane, piece 0 (others by exclusive or)
  const uint32_t group_mat = lane * kQ4CodeBytes + (((lane >> 1) & 3) << 4);

  const float f1 = p.scale_log2 * 1024.0f;
  Queries<NB> Q;
  float o[NB][4][2][4];   // [8 rows][group][step][channel, row pair]
  float om[NB][2];        // middles' term (lanes of g >= 4)
  float ref[NB][2], l[NB][2];  // rows 2t, 2t + 1
  int gain[NB][2];
  bool fresh = true;
  int seg_tiles = 0;  // tiles of the row block so far
  TileRing<S::kStages> ring;
  // the sums of row j of eight go from one gain to another, at most as large
  auto scale_outputs = [&](int nb, int j, int& from, int to) {
    const float f = pow2(max(to - from, -126));
    from = to;
    om[nb][j] *= f;
#pragma unroll
    for (int J = 0; J < 4; ++J)
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        o[nb][J][st][j] *= f;
        o[nb][J][st][2 + j] *= f;
      }
  };
  bool failed = p.stall_ns && blockIdx.x == 0 && warp == 0 && left > 0 &&
                !mbar_wait_bounded(never, 0, &s_abort, p.status, p.stall_ns);

  for (; left > 0 && !failed; --left) {
    if (fresh) {
      seg_tiles = 0;
      load_queries<NB>(p, c.unit, c.block, Q);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        ref[nb][0] = ref[nb][1] = -INFINITY;
        l[nb][0] = l[nb][1] = 0.f;
        gain[nb][0] = gain[nb][1] = kMaxGain;
#pragma unroll
        for (int i = 0; i < 2; ++i) om[nb][i] = 0.f;
#pragma unroll
        for (int J = 0; J < 4; ++J)
#pragma unroll
          for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[nb][J][st][i] = 0.f;
      }
      fresh = false;
    }
    // (all lanes go on, or none: another warp's abort may reach some lanes only)
    const bool landed = mbar_wait_bounded(bars + 8 * ring.stage, ring.phase, &s_abort, p.status);
    if (!__all_sync(0xffffffffu, landed)) {
      failed = true;
      break;
    }
    ++seg_tiles;
    const uint32_t cd = codes + ring.stage * 2 * kCodeTile, sd = side + ring.stage * kSideBytes;
    const int valid = c.valid;

    // ---- scales: one or two slots a lane.  Slots behind the length and groups that
    // hold a NaN count nothing in V's products
    uint32_t nan_groups[kLane] = {};  // of this lane's slots
    bool special;
    float largest;  // of the slots' 2^(e - 12)
    {
      uint4 w[kLane];
#pragma unroll
      for (int i = 0; i < kLane; ++i) {
        const int slot = lane + 32 * i;
        w[i] = make_uint4(0u, 0u, 0u, 0u);
        if (slot >= kTile) continue;
        const uint2 kw = lds64(sd + slot * kQ4ParamBytes);
        if (slot < valid) w[i] = lds128(sd + kParamTile + slot * kQ4ParamBytes);
        sts128(scales + slot * 16,
               make_uint4(__float_as_uint(bf_lo(kw.x) * f1), __float_as_uint(bf_hi(kw.x) * f1),
                          __float_as_uint(bf_lo(kw.y) * f1), __float_as_uint(bf_hi(kw.y) * f1)));
      }
      uint32_t top[kLane], all = 0;
#pragma unroll
      for (int i = 0; i < kLane; ++i) {
        top[i] = top_of(w[i]);
        all = max(all, top[i]);
      }
      all = __reduce_max_sync(0xffffffffu, all);
      special = all >= 0x7f800000u;
      if (special) {
        all = 0;
#pragma unroll
        for (int i = 0; i < kLane; ++i) {
          uint32_t x[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
          for (int J = 0; J < 4; ++J) {
            const uint32_t half = 0xffffu << (16 * (J & 1)), inf = 0x7f807f80u & half;
            if ((x[J >> 1] & inf) == inf || (x[2 + (J >> 1)] & inf) == inf) {
              nan_groups[i] |= 1u << J;
              x[J >> 1] &= ~half;
              x[2 + (J >> 1)] &= ~half;
            }
          }
          w[i] = make_uint4(x[0], x[1], x[2], x[3]);
          top[i] = min(top_of(w[i]), 0x7f000000u);
          all = max(all, top[i]);
        }
        all = __reduce_max_sync(0xffffffffu, all);
      }
      largest = pow2(max(static_cast<int>(all >> 23) - 127, kMinScaleExp) - kExpOff);
#pragma unroll
      for (int i = 0; i < kLane; ++i) {
        const int e = max(static_cast<int>(top[i] >> 23) - 127, kMinScaleExp);
        const float f = pow2(kTopExp - e);
        const float s0 = bf_lo(w[i].x) * f, s1 = bf_hi(w[i].x) * f, s2 = bf_lo(w[i].y) * f, s3 = bf_hi(w[i].y) * f;
        // middles: m + 7.5 s
        const float m0 = fmaf(s0, 7.5f, bf_lo(w[i].z) * f), m1 = fmaf(s1, 7.5f, bf_hi(w[i].z) * f);
        const float m2 = fmaf(s2, 7.5f, bf_lo(w[i].w) * f), m3 = fmaf(s3, 7.5f, bf_hi(w[i].w) * f);
        const uint32_t m01 = pack_half2(m0, m1), m23 = pack_half2(m2, m3);
        // an even lane keeps groups 0 and 1 of its pair of slots, an odd one 2 and 3
        const uint32_t s01 = pack_half2(s0, s1), s23 = pack_half2(s2, s3);
        const uint32_t got = __shfl_xor_sync(0xffffffffu, lane & 1 ? s01 : s23, 1);
        const uint32_t a = lane & 1 ? got : s01, b = lane & 1 ? s23 : got;
        if (lane + 32 * i < kTile) {
          const uint32_t even = __byte_perm(a, b, 0x5410), odd = __byte_perm(a, b, 0x7632);
          sts128(sd + kParamTile + (lane + 32 * i) * kQ4ParamBytes, make_uint4(s01, s23, m01, m23));
          sts128(pairs + (lane + 32 * i) * 16, make_uint4(even, odd, half_rest(m0, m1, m01), half_rest(m2, m3, m23)));
          sts32(exps + (lane + 32 * i) * 4, __float_as_uint(pow2(e - kExpOff)));
        }
      }
      __syncwarp();
    }

    // ---- logits: 16 slots a step; slots g and g + 8 of rows 2t and 2t + 1
    float z[NB][kSteps][4];  // [8 rows][16 slots][slot half, row]
#pragma unroll
    for (int h = 0; h < kSteps; ++h) {
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
    if (valid < kTile) {
#pragma unroll
      for (int h = 0; h < kSteps; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (h * 16 + (i >> 1) * 8 + g >= valid)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) z[nb][h][i] = -INFINITY;
    }
    if (p.accumulate) {
      // [slot][rows]: a lane's two rows are neighbours.  (Behind the length
      // there may be the next unit.)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int r = c.block * kRows + nb * 8 + 2 * t;
        float* zp = p.z + static_cast<size_t>(c.row + g) * p.z_stride + r;
#pragma unroll
        for (int h = 0; h < kSteps; ++h)
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (r < p.rows && h * 16 + 8 * i + g < valid)
              *reinterpret_cast<float2*>(zp + (h * 16 + 8 * i) * p.z_stride) =
                  make_float2(z[nb][h][2 * i] * Q.f2[nb][0], z[nb][h][2 * i + 1] * Q.f2[nb][1]);
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
        top[j] = fmaxf(z[nb][0][j], z[nb][0][2 + j]);
#pragma unroll
        for (int h = 1; h < kSteps; ++h) top[j] = fmaxf(top[j], fmaxf(z[nb][h][j], z[nb][h][2 + j]));
        top[j] *= Q.f2[nb][j];
        raise |= top[j] > ref[nb][j] + kRaise;
      }
      if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], 4));
          top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], 8));
          top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], 16));
          if (!(top[j] > ref[nb][j] + kRaise)) continue;
          // (references are whole numbers; while there is none, nothing is summed yet)
          const float up = ceilf(top[j]);
          const int more = ref[nb][j] == -INFINITY ? 0 : static_cast<int>(fminf(up - ref[nb][j], 1000.f));
          ref[nb][j] = up;
          l[nb][j] *= pow2(max(-more, -126));
          // probabilities shrink by 2^more, so the gain of the outputs' weights grows
          gain[nb][j] += more;
          if (gain[nb][j] > kMaxGain) scale_outputs(nb, j, gain[nb][j], kMaxGain);
        }
      }
      if (special) {
        // rows that see a slot's NaN group
        uint32_t hit[2] = {0u, 0u};
#pragma unroll
        for (int h = 0; h < kSteps; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t m = __shfl_sync(0xffffffffu, nan_groups[h >> 1], (h & 1) * 16 + (i >> 1) * 8 + g);
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
        for (int h = 0; h < kSteps; ++h)
#pragma unroll
          for (int i = j; i < 4; i += 2) {
            z[nb][h][i] = ex2_approx(fmaf(z[nb][h][i], Q.f2[nb][j], -r));
            l[nb][j] += z[nb][h][i];
          }
      }
    }
    // ---- weights of the slots' rows of V: probabilities times 2^e, and the row's gain
    int high = gain[0][0];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) high = max(high, max(gain[nb][0], gain[nb][1]));
#pragma unroll
    for (int h = 0; h < kSteps; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float x = __uint_as_float(lds32(exps + (h * 16 + 8 * i + g) * 4));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) mul_pair(z[nb][h][2 * i], z[nb][h][2 * i + 1], x, x);
      }
    // (probabilities are at most 2^11: no need to look where no slot of the tile is
    // beyond 2^4 in any row's terms)
    if (__any_sync(0xffffffffu, largest * pow2(high) > kTopWeight / 2048.0f)) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float most = 0.f;
#pragma unroll
          for (int h = 0; h < kSteps; ++h) most = fmaxf(most, fmaxf(z[nb][h][j], z[nb][h][2 + j]));
          most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 4));
          most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 8));
          most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 16));
          // the largest of the tile becomes 2^2 .. 2^3
          if (most * pow2(gain[nb][j]) > kTopWeight)
            scale_outputs(nb, j, gain[nb][j], max(129 - static_cast<int>(__float_as_uint(most) >> 23), -122));
        }
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const float x0 = pow2(gain[nb][0]), x1 = pow2(gain[nb][1]);
#pragma unroll
      for (int h = 0; h < kSteps; ++h)
#pragma unroll
        for (int i = 0; i < 4; i += 2) mul_pair(z[nb][h][i], z[nb][h][i + 1], x0, x1);
    }

    // ---- outputs: the sums of p s and p m', then the codes group by group
    // (lanes of g >= 4: p m' of group g - 4, of both parts; of g < 4: p s of group g)
    float sums[NB][4];
    uint32_t p0[NB][kSteps], p1[NB][kSteps];
    uint32_t r0[kFine ? NB : 1][kSteps], r1[kFine ? NB : 1][kSteps];  // what their rounding left
#pragma unroll
    for (int h = 0; h < kSteps; ++h) {
      uint32_t pm[4];
      // rows of [4 scales, 4 middles], transposed, and as rows 8-15 of the operand
      // of [2 pairs of scales, 4 rests of middles]
      ldmatrix4_t(pm, (lane & 8 ? pairs : sd + kParamTile) + (h * 16 + (lane & 7) + ((lane & 16) >> 1)) * 16);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const uint32_t lo = pack_half2(z[nb][h][0], z[nb][h][1]), hi = pack_half2(z[nb][h][2], z[nb][h][3]);
        p0[nb][h] = transpose8(lo);
        p1[nb][h] = transpose8(hi);
        if (h == 0) sums[nb][0] = sums[nb][1] = sums[nb][2] = sums[nb][3] = 0.f;
        mma_f16(sums[nb], pm[0], pm[1], pm[2], pm[3], p0[nb][h], p1[nb][h]);
        if (kFine) {
          r0[nb][h] = transpose8(half_rest(z[nb][h][0], z[nb][h][1], lo));
          r1[nb][h] = transpose8(half_rest(z[nb][h][2], z[nb][h][3], hi));
          mma_f16(sums[nb], pm[0], pm[1], pm[2], pm[3], r0[nb][h], r1[nb][h]);
        }
      }
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      om[nb][0] += sums[nb][0] + sums[nb][2];
      om[nb][1] += sums[nb][1] + sums[nb][3];
    }
#pragma unroll
    for (int J = 0; J < 4; ++J) {
      uint32_t v[kTile / 8];  // group J of 8 slots each
#pragma unroll
      for (int i = 0; i < kTile / 32; ++i)
        ldmatrix4_t(*reinterpret_cast<uint32_t (*)[4]>(v + 4 * i),
                    cd + kCodeTile + i * 32 * kQ4CodeBytes + (group_mat ^ (J << 4)));
      // sum of p s; where p s is rounded, of the rounded ones
      float mass[NB][4];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          mass[nb][i] = kFine ? __shfl_sync(0xffffffffu, sums[nb][i & 1], 4 * J + t) : 0.f;
      auto take_off = [&] {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              o[nb][J][st][i] = fmaf(mass[nb][i], -kMiddle, o[nb][J][st][i]);
              o[nb][J][st][2 + i] = fmaf(mass[nb][i], -16.0f * kMiddle, o[nb][J][st][2 + i]);
            }
      };
#pragma unroll
      for (int h = 0; h < kSteps; ++h) {
        // (half way, where it is known: what the sums' truncation takes before, it
        // gives after)
        if (kFine && h == kSteps / 2) take_off();
        // scales of two pairs of slots
        const uint32_t pair = pairs + (h * 16 + 2 * t + (J >> 1)) * 16 + (J & 1) * 4;
        const uint32_t sa = lds32(pair), sb = lds32(pair + 8 * 16);
        const uint32_t x = v[2 * h], y = v[2 * h + 1], xh = x >> 8, yh = y >> 8;
        const uint32_t a0 = x & 0x000f000fu, a1 = x & 0x00f000f0u, a2 = y & 0x000f000fu, a3 = y & 0x00f000f0u;
        const uint32_t b0 = xh & 0x000f000fu, b1 = xh & 0x00f000f0u, b2 = yh & 0x000f000fu, b3 = yh & 0x00f000f0u;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          uint32_t q0 = mul_half2(p0[nb][h], sa), q1 = mul_half2(p1[nb][h], sb);
          mma_f16(o[nb][J][0], a0, a1, a2, a3, q0, q1);
          mma_f16(o[nb][J][1], b0, b1, b2, b3, q0, q1);
          if (!kFine) {
            mma_f16(mass[nb], kOnes, kOnes, kOnes, kOnes, q0, q1);
          } else {
            q0 = fma_half2(r0[nb][h], sa, fma_half2(p0[nb][h], sa, q0 ^ 0x80008000u));
            q1 = fma_half2(r1[nb][h], sb, fma_half2(p1[nb][h], sb, q1 ^ 0x80008000u));
            mma_f16(o[nb][J][0], a0, a1, a2, a3, q0, q1);
            mma_f16(o[nb][J][1], b0, b1, b2, b3, q0, q1);
          }
        }
      }
      if (!kFine) take_off();
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
    if (to_issue > 0) issue(ring.stage);
    ring.advance();

    // ---- the row block ends here, or this warp's share of it
    const int unit = c.unit, block = c.block, done = c.row - c.unit * p.c.capacity;
    const int len = done + c.valid;
    ++tile;
    const bool ends = c.valid <= kTile;
    if (left > 1) c.template next<S::kTile>(p);
    if (left == 1 || ends) {
      const int count = (len + kTile - 1) / kTile;
      const bool starts = seg_tiles > done / kTile;
      const bool whole = starts && ends, tail = left == 1;
      if (!whole && lane == 0) {
        Part& part = tail ? s_tail[warp] : s_head[warp];
        part.block = unit * p.blocks + block;
        part.count = count;
        part.first = tile - 1 - done / kTile;
        part.starts = starts;
        part.ends = ends;
      }
      // sums of the codes' products: * 2^24, and 1/16 for a byte's second channel
      float* head = p.head_o + static_cast<size_t>(blockIdx.x * S::kWarps + warp) * kRows * kHeadDim;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float sum[2], norm[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          sum[j] = l[nb][j];
          sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 4);
          sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 8);
          sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 16);
          // 2^(kExpOff - kTopExp - gain) / sum
          norm[j] = pow2(1 - gain[nb][j]) * (256.0f * inverse(sum[j]));
          if (!whole && g == 0) {
            const float2 ml = make_float2(ref[nb][j] - kLift, sum[j]);
            const int r = nb * 8 + 2 * t + j;
            if (tail) s_ml[warp][r] = ml;
            else p.head_ml[(blockIdx.x * S::kWarps + warp) * kRows + r] = ml;
          }
        }
#pragma unroll
        for (int J = 0; J < 4; ++J) {
          const float m0 = __shfl_sync(0xffffffffu, om[nb][0], (4 + J) * 4 + t);
          const float m1 = __shfl_sync(0xffffffffu, om[nb][1], (4 + J) * 4 + t);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float m = i ? m1 : m0;
            const int r = nb * 8 + 2 * t + i, row = block * kRows + r;
            float4 v;
            v.x = fmaf(o[nb][J][0][i], 16777216.0f, m) * norm[i];
            v.y = fmaf(o[nb][J][0][2 + i], 1048576.0f, m) * norm[i];
            v.z = fmaf(o[nb][J][1][i], 16777216.0f, m) * norm[i];
            v.w = fmaf(o[nb][J][1][2 + i], 1048576.0f, m) * norm[i];
            if (row >= p.rows) continue;
            if (whole) write_row(p, unit, row, 8 * J + g, v, ref[nb][i] - kLift, sum[i]);
            else if (tail) sts128(codes + r * (kHeadDim * 4) + (8 * J + g) * 16,
                                  make_uint4(__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z),
                                             __float_as_uint(v.w)));
            else reinterpret_cast<float4*>(head + r * kHeadDim)[8 * J + g] = v;
          }
        }
      }
      fresh = true;
    }
  }
  if (failed) {
    if (lane == 0) *reinterpret_cast<volatile int*>(p.stopped) = 1;
    // copies in flight end before the shared memory does (or their wait runs out)
    for (int k = 0; k < ring.in_flight(left); ++k) {
      const uint64_t t0 = globaltimer_ns();
      while (!mbar_test_wait(bars + 8 * ring.stage_of(k), ring.phase_of(k)) && globaltimer_ns() - t0 < 100000000ull) {
      }
    }
  }
  // ---- units that hold nothing
  for (int u = blockIdx.x + ctas * warp; u < units; u += ctas * S::kWarps)
    if (length_of(p.c, u) == 0)
      for (int r = 0; r < p.rows; ++r)
        write_row(p, u, r, lane, make_float4(0.f, 0.f, 0.f, 0.f), -INFINITY, 0.f);

  // ---- row blocks that this CTA's warps share: joined in slot order
  __syncthreads();
  if (s_abort) return;
  // A part is a softmax reference, a sum and the outputs over that part alone:
  // averages of averages stay within V's range.  Gives the weight f of each
  // part (lane i has the reference and sum of part i) and the sum over all, and
  // returns their common reference.
  auto weigh = [&](float2 ml, float* f, float* sum) {
    float top = ml.x;
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    *f = ex2_approx(ml.x - (top == -INFINITY ? 0.f : top));
    const float mine = ml.y * *f;
    float x = mine;
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    *sum = x;
    *f = mine * inverse(x);
    return top;
  };
  auto add = [](float4& acc, float4 v, float f) {
    acc.x = fmaf(v.x, f, acc.x);
    acc.y = fmaf(v.y, f, acc.y);
    acc.z = fmaf(v.z, f, acc.z);
    acc.w = fmaf(v.w, f, acc.w);
  };
  int shared[2] = {-2, -2};  // (-1: the head of the first) warp whose part begins the row block shared with CTAs before, behind
  {
    const int tb = lane < S::kWarps ? s_tail[lane].block : -1;
    const int hb = lane < S::kWarps ? s_head[lane].block : -1;
    const int prev = __shfl_up_sync(0xffffffffu, tb, 1);
    // a row block's first part here: the first warp's head, or a tail unlike
    // the one before it
    unsigned todo = __ballot_sync(0xffffffffu, tb >= 0 && (lane == 0 || tb != prev)) << 1;
    if (__shfl_sync(0xffffffffu, hb, 0) >= 0) todo |= 1u;
    while (todo) {
      const int w = __ffs(todo) - 2;  // -1: the head
      todo &= todo - 1;
      const int vu = __shfl_sync(0xffffffffu, w < 0 ? hb : tb, max(w, 0));
      const int tails = w < 0 ? 0 : __popc(__ballot_sync(0xffffffffu, tb == vu));
      const unsigned heads = __ballot_sync(0xffffffffu, hb == vu);
      const int first = max(w, 0), head = heads ? __ffs(heads) - 1 : -1;
      const bool starts = w < 0 ? s_head[0].starts : s_tail[first].starts;
      const bool ends = heads ? s_head[head].ends : s_tail[first + tails - 1].ends;
      const bool whole = starts && ends;
      if (!whole) shared[starts] = w;
      const int unit = vu / p.blocks, row0 = (vu - unit * p.blocks) * kRows;
      for (int r = warp; r < kRows && row0 + r < p.rows; r += S::kWarps) {
        const size_t hr = static_cast<size_t>(blockIdx.x * S::kWarps + head) * kRows + r;
        float2 ml = make_float2(-INFINITY, 0.f);
        float4 hv = make_float4(0.f, 0.f, 0.f, 0.f);
        if (lane < tails) ml = s_ml[first + lane][r];
        if (heads) {
          if (lane == tails) ml = p.head_ml[hr];
          hv = reinterpret_cast<const float4*>(p.head_o + hr * kHeadDim)[lane];
        }
        float f, sum;
        const float top = weigh(ml, &f, &sum);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int k = 0; k < tails; ++k) {
          const uint4 v = lds128(base + (first + k) * S::kStages * 2 * kCodeTile + r * (kHeadDim * 4) + lane * 16);
          add(acc, make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z),
                               __uint_as_float(v.w)),
              __shfl_sync(0xffffffffu, f, k));
        }
        if (heads) add(acc, hv, __shfl_sync(0xffffffffu, f, tails));
        if (whole) {
          write_row(p, unit, row0 + r, lane, acc, top, sum);
        } else {
          const size_t to = static_cast<size_t>(blockIdx.x * 2 + starts) * kRows + r;
          reinterpret_cast<float4*>(p.cta_o + to * kHeadDim)[lane] = acc;
          if (lane == 0) p.cta_ml[to] = make_float2(top, sum);
        }
      }
    }
  }
  if (shared[0] < -1 && shared[1] < -1) return;

  // ---- row blocks that CTAs share: the last one to come joins them, in order
  auto first_cta = [&](const Part& x) { return own0 >= 0 ? own0 : x.first / chunk; };
  auto last_cta = [&](const Part& x) {
    return own0 >= 0 ? own0 + (x.count - 1) / chunk : (x.first + x.count - 1) / chunk;
  };
  fence_acq_rel_gpu();
  __syncthreads();
  __shared__ int s_last[2];
  if (threadIdx.x < 2) {
    const int w = shared[threadIdx.x];
    int last = 0;
    if (w >= -1) {
      const Part& part = w < 0 ? s_head[0] : s_tail[w];
      const int c0 = first_cta(part), c1 = last_cta(part);
      if (atomicAdd(p.tickets + c0, 1) == c1 - c0) {
        p.tickets[c0] = 0;  // for the next call
        last = 1;
      }
      fence_acq_rel_gpu();
    }
    s_last[threadIdx.x] = last;
  }
  __syncthreads();
  // The parts of a row are summed by several warps where there are fewer rows,
  // of both row blocks at once.
  const int both = s_last[0] + s_last[1];
  if (both == 0) return;
  float4* s_acc = reinterpret_cast<float4*>(smem_raw + (base - smem_u32(smem_raw)));
  const int which = both == 2 ? warp & 1 : s_last[1];
  const int warps = S::kWarps / both, mine = warp / both;
  const Part part = shared[which] < 0 ? s_head[0] : s_tail[shared[which]];
  const int c0 = first_cta(part), c1 = last_cta(part);
  const int unit = part.block / p.blocks, row0 = (part.block - unit * p.blocks) * kRows;
  const int rows = min(kRows, p.rows - row0);
  // (rounds as many as the row block with more rows takes: every warp is at
  // every barrier)
  const int rounds = (min(kRows, p.rows) + warps - 1) / warps;
  for (int round = 0; round < rounds; ++round) {
    const int r0 = round * warps, rn = max(1, min(rows - r0, warps)), split = warps / rn;
    const int r = r0 + mine % rn, k = mine / rn;
    float top = -INFINITY, sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r < rows && k < split) {
      constexpr int kBatch = 8;
      for (int c = c0 + k; c <= c1; c += kBatch * split) {
        float2 ml[kBatch];
        float4 v[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          const int x = c + i * split;
          ml[i] = make_float2(-INFINITY, 0.f);
          v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (x <= c1) {
            const size_t from = static_cast<size_t>(x * 2 + (x == c0)) * kRows + r;
            ml[i] = __ldcg(&p.cta_ml[from]);
            v[i] = __ldcg(reinterpret_cast<const float4*>(p.cta_o + from * kHeadDim) + lane);
          }
        }
        float t = top;
#pragma unroll
        for (int i = 0; i < kBatch; ++i) t = fmaxf(t, ml[i].x);
        const float ref0 = t == -INFINITY ? 0.f : t, old = sum * ex2_approx(top - ref0);
        sum = old;
        top = t;
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          ml[i].y *= ex2_approx(ml[i].x - ref0);
          sum += ml[i].y;
        }
        const float inv = inverse(sum), keep = old * inv;
        acc = make_float4(acc.x * keep, acc.y * keep, acc.z * keep, acc.w * keep);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) add(acc, v[i], ml[i].y * inv);
      }
    }
    __syncthreads();
    s_acc[warp * 32 + lane] = acc;
    if (lane == 0) s_ml[warp][0] = make_float2(top, sum);
    __syncthreads();
    if (r < rows && k == 0) {
      float2 ml = make_float2(-INFINITY, 0.f);
      if (lane < split) ml = s_ml[warp + lane * rn * both][0];
      float f;
      top = weigh(ml, &f, &sum);
      acc = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int i = 0; i < split; ++i)
        add(acc, s_acc[(warp + i * rn * both) * 32 + lane], __shfl_sync(0xffffffffu, f, i));
      write_row(p, unit, row0 + r, lane, acc, top, sum);
    }
  }
}

// Four channels (4 * lane ..) of a query row's output v, whose `sum` is that of
// 2^(logit - ref); the first lane writes the log-sum-exp.
__device__ __forceinline__ void write_row(const Q4AttendParams& p, int unit, int row, int lane, float4 v,
                                          float ref, float sum) {
  const int b = unit / p.c.num_kv_heads;
  const int hg = row / p.num_queries, qi = row - hg * p.num_queries;
  const int h = (unit - b * p.c.num_kv_heads) * p.group + hg;
  uint2 y;
  if (p.is_bf16) {
    y.x = pack_bf16(v.x, v.y);
    y.y = pack_bf16(v.z, v.w);
  } else {
    y.x = pack_half2(v.x, v.y);
    y.y = pack_half2(v.z, v.w);
  }
  *reinterpret_cast<uint2*>(p.out + b * p.o_bs + h * p.o_hs + qi * p.o_qs + 4 * lane) = y;
  if (lane == 0) {
    const float l2 = ref + log2f(sum);
    p.lse_ws[static_cast<long long>(unit) * p.rows + row] = l2;
    if (p.lse) p.lse[(static_cast<long long>(b) * p.num_q_heads + h) * p.num_queries + qi] = l2 * kLn2;
  }
}

// ---------------------------------------------------------------- weights
// A thread takes a slot, whose logits lie side by side: kWide of them a read,
// four where the rows are a multiple of four (28 rows of 32 units of 1000 to
// 8000 slots, attention and weights: 47.7 us, and 52.2 in pairs; 8 rows of 64
// units: 28.4 and 28.8).  (Groups of lanes that share a slot, or several slots a
// thread, took half as long again: more instructions, and more lines at once than
// L1 holds.)  Bound by L2, which holds the logits of some 30 MB: 21 us for 2.3
// million slots of 8 rows, whose logits and weights are 92 MB.
constexpr int kWeightThreads = 256;

template <int kWide>
__global__ void __launch_bounds__(kWeightThreads) weights_kernel(const __grid_constant__ Q4AttendParams p) {
  __shared__ float s_lse[kMaxQRows + 2];
  pdl_wait();
  const int unit = blockIdx.y, len = length_of(p.c, unit);
  const int j = blockIdx.x * kWeightThreads + threadIdx.x;
  if (j - static_cast<int>(threadIdx.x) >= len) return;
  const size_t slot = static_cast<size_t>(unit) * p.c.capacity + j;
  // An attention that stopped early leaves logits and sums of earlier calls.
  // (Read through L1: 16000 CTAs that all asked L2 for this word took 20 us.)
  const int stopped = *p.stopped;
  const float old = j < len ? p.c.weights[slot] : 0.f;
  for (int r = threadIdx.x; r < p.rows; r += kWeightThreads)
    s_lse[r] = p.lse_ws[static_cast<size_t>(unit) * p.rows + r];
  __syncthreads();
  if (j >= len) return;
  const float* z = p.z + slot * p.z_stride;
  float add = 0.f;
  // (a row that does not see the slot has -inf there; of an odd number of rows
  // the last read holds one more, which is none)
#pragma unroll 2
  for (int r = 0; r < p.rows; r += kWide) {
    float x[kWide];
    if (kWide == 4) {
      const float4 v = *reinterpret_cast<const float4*>(z + r);
      x[0] = v.x, x[1] = v.y, x[kWide - 2] = v.z, x[kWide - 1] = v.w;
    } else {
      const float2 v = *reinterpret_cast<const float2*>(z + r);
      x[0] = v.x, x[1] = v.y;
    }
#pragma unroll
    for (int i = 0; i < kWide; ++i)
      if (r + i < p.rows && x[i] != -INFINITY) add += ex2_approx(x[i] - s_lse[r + i]);
  }
  if (!stopped) p.c.weights[slot] = old + add;
}

template <int NB, bool kPos, bool kFine>
cudaError_t launch(const Q4AttendParams& p, int sms, cudaStream_t stream) {
  return launch_dependent(attend_kernel<NB, kPos, kFine>, dim3(sms), Shape<NB>::kThreads, Shape<NB>::kSmem, stream, p);
}

}  // namespace

cudaError_t q4_attend_set_smem_limit() {
  cudaError_t e = cudaSuccess;
  auto set = [&](auto* f, int bytes) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  };
  set(attend_kernel<1, false, false>, Shape<1>::kSmem);
  set(attend_kernel<1, false, true>, Shape<1>::kSmem);
  set(attend_kernel<1, true, false>, Shape<1>::kSmem);
  set(attend_kernel<1, true, true>, Shape<1>::kSmem);
  set(attend_kernel<2, false, false>, Shape<2>::kSmem);
  set(attend_kernel<2, false, true>, Shape<2>::kSmem);
  set(attend_kernel<2, true, false>, Shape<2>::kSmem);
  set(attend_kernel<2, true, true>, Shape<2>::kSmem);
  return e;
}

cudaError_t launch_q4_attend(const Q4AttendParams& p, int sms, cudaStream_t stream) {
  auto choose = [&](auto positions, auto fine) {
    return p.block_rows == 8 ? launch<1, decltype(positions)::value, decltype(fine)::value>(p, sms, stream)
                             : launch<2, decltype(positions)::value, decltype(fine)::value>(p, sms, stream);
  };
  using Yes = std::true_type;
  using No = std::false_type;
  if (p.is_bf16) return p.q_positions ? choose(Yes{}, No{}) : choose(No{}, No{});
  return p.q_positions ? choose(Yes{}, Yes{}) : choose(No{}, Yes{});
}

cudaError_t launch_q4_weights(const Q4AttendParams& p, cudaStream_t stream) {
  const dim3 grid((p.c.capacity + kWeightThreads - 1) / kWeightThreads, p.c.batch * p.c.num_kv_heads);
  return launch_dependent(p.z_stride % 4 ? weights_kernel<2> : weights_kernel<4>, grid, kWeightThreads, 0, stream, p);
}

}  // namespace ckv
