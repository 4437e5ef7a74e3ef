// Rotary positions of Q and K rows, alone or on the way into a paged cache.
//
// A pair (a, b) of a row turns by its position m times its frequency:
//   a' = a cos t - b sin t,  b' = a sin t + b cos t,  t = 2 pi frac(m T),
// with T the turns a position.  m T is taken modulo one as a 64-bit integer
// product, so that far positions lose nothing; its upper 32 bits, as a signed
// number in half turns, are what sincospif takes.  The gradient turns by -t.
//
// Memory is the bound: a row is read once and written once.  Eight lanes hold a
// head's row, eight pairs each (two 16-byte pieces), and a warp four heads at a
// time, all of one token, so that the cosines and sines of a token are computed
// once for all of its heads.
#include "ckv_device.cuh"
#include "paged_params.h"
#include "q4_params.h"

namespace ckv {
namespace {

constexpr int kThreads = 256;
constexpr int kBlocks = 4;                      // CTAs of an SM, at least
constexpr int kWarps = kThreads / 32;
constexpr int kLanes = 8;                       // lanes of a head
constexpr int kPairsLane = kRopePairs / kLanes; // 8
constexpr int kUnroll = 2;                      // heads of a lane in flight
constexpr int kFill = 2432;                     // warps that the GPU is to have where there is enough for them
// Rows of a sequence that one CTA appends where the start is the length itself; more take
// a second launch for the lengths.  In a graph, 32 + 8 heads with Q, 1 / 8 / 64 sequences
// of one row: 3.3 / 3.6 / 3.5 us so, 4.1 / 4.5 / 4.3 in two launches; of two rows: 5.0 / 5.1 /
// 5.1 and 4.3 / 4.2 / 4.9; of 16 rows: 25 / 25 / 26 and 4.5 / 4.9 / 8.2.
constexpr int kFewRows = 1;

// Where a lane's eight pairs are.
enum Layout {
  kHalves,      // channels i and i + rot_dim / 2, rot_dim a multiple of 16: two pieces
  kNeighbours,  // channels 2i and 2i + 1: two pieces side by side
  kOddHalves    // as kHalves, any rot_dim: single channels
};

template <bool kBf16>
__device__ __forceinline__ float2 unpack(uint32_t w) {
  if (kBf16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  float2 r;
  asm("{\n\t.reg .f16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, h;\n\t}"
      : "=f"(r.x), "=f"(r.y)
      : "r"(w));
  return r;
}
template <bool kBf16>
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  if (!kBf16) return pack_half2(lo, hi);
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

struct Angles {
  float c[kPairsLane], s[kPairsLane];
};

template <int kLayout>
__device__ __forceinline__ int pair_of(int l, int i) {
  return kLayout == kOddHalves ? l + kLanes * i : kPairsLane * l + i;
}

// The four lanes that hold the same pairs, of four heads, compute two of their
// angles each and hand them on.  (8191 tokens of 28 and 4 heads: 23.7 us, with loads
// that start before the angles; 29.6 before both.)
template <int kLayout>
__device__ __forceinline__ void angles_at(const RopeTable& r, int position, bool backward, int lane, Angles& a) {
  constexpr int kEach = kPairsLane * kLanes / 32;  // 2
  const int l = lane % kLanes;
  float c[kEach], s[kEach];
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    c[e] = 1.f;
    s[e] = 0.f;
    const int pair = pair_of<kLayout>(l, lane / kLanes * kEach + e);
    if (pair < r.pairs) {
      const unsigned long long t = r.turns[pair] * static_cast<unsigned long long>(static_cast<long long>(position));
      const float half_turns = static_cast<float>(static_cast<int>(t >> 32)) * 0x1p-31f;
      sincospif(half_turns, &s[e], &c[e]);
      c[e] *= r.scale;
      s[e] *= backward ? -r.scale : r.scale;
    }
  }
#pragma unroll
  for (int i = 0; i < kPairsLane; ++i) {
    const int from = l + kLanes * (i / kEach);
    a.c[i] = __shfl_sync(0xffffffffu, c[i % kEach], from);
    a.s[i] = __shfl_sync(0xffffffffu, s[i % kEach], from);
  }
}

// A lane's sixteen channels.  Pieces: the words of its two pieces; single
// channels: word i holds the pair's two.
struct Piece {
  uint32_t w[8];
};

template <int kLayout>
__device__ __forceinline__ int offset_of(int l, int pairs, int piece) {
  if (kLayout == kHalves && kPairsLane * l < pairs) return kPairsLane * l + piece * pairs;
  return 16 * l + 8 * piece;  // (behind the halves, too: 2 pairs + 2 (8 l - pairs))
}
// The two channels of a pair, or of a copied one.
__device__ __forceinline__ int2 channels_of(int pair, int pairs) {
  return pair < pairs ? make_int2(pair, pair + pairs) : make_int2(2 * pair, 2 * pair + 1);
}

template <int kLayout>
__device__ __forceinline__ void load(const uint16_t* row, int l, int pairs, Piece& x) {
  if (kLayout == kOddHalves) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int2 c = channels_of(pair_of<kLayout>(l, i), pairs);
      x.w[i] = row[c.x] | static_cast<uint32_t>(row[c.y]) << 16;
    }
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint4 v = *reinterpret_cast<const uint4*>(row + offset_of<kLayout>(l, pairs, h));
      x.w[4 * h] = v.x, x.w[4 * h + 1] = v.y, x.w[4 * h + 2] = v.z, x.w[4 * h + 3] = v.w;
    }
  }
}
template <int kLayout>
__device__ __forceinline__ void store(uint16_t* row, int l, int pairs, const Piece& x) {
  if (kLayout == kOddHalves) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int2 c = channels_of(pair_of<kLayout>(l, i), pairs);
      row[c.x] = static_cast<uint16_t>(x.w[i]);
      row[c.y] = static_cast<uint16_t>(x.w[i] >> 16);
    }
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      *reinterpret_cast<uint4*>(row + offset_of<kLayout>(l, pairs, h)) =
          make_uint4(x.w[4 * h], x.w[4 * h + 1], x.w[4 * h + 2], x.w[4 * h + 3]);
  }
}

template <bool kBf16, int kLayout>
__device__ __forceinline__ void turn(const Angles& t, int l, int pairs, Piece& x) {
  if (kLayout == kHalves) {
    if (kPairsLane * l >= pairs) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 a = unpack<kBf16>(x.w[j]), b = unpack<kBf16>(x.w[4 + j]);
      const float c0 = t.c[2 * j], s0 = t.s[2 * j], c1 = t.c[2 * j + 1], s1 = t.s[2 * j + 1];
      x.w[j] = pack<kBf16>(a.x * c0 - b.x * s0, a.y * c1 - b.y * s1);
      x.w[4 + j] = pack<kBf16>(a.x * s0 + b.x * c0, a.y * s1 + b.y * c1);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 a = unpack<kBf16>(x.w[i]);
      const uint32_t y = pack<kBf16>(a.x * t.c[i] - a.y * t.s[i], a.x * t.s[i] + a.y * t.c[i]);
      if (pair_of<kLayout>(l, i) < pairs) x.w[i] = y;
    }
  }
}

struct Place {
  int seq, index, rows;  // row `index` of the `rows` of sequence `seq`
};
template <class P>
__device__ __forceinline__ Place place_of(const P& p, int row) {
  if (p.rows_per_seq >= 0) {
    const int s = row / p.rows_per_seq;
    return {s, row - s * p.rows_per_seq, p.rows_per_seq};
  }
  int lo = 0, hi = p.c.batch;  // cu_rows[lo] <= row < cu_rows[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (p.cu_rows[mid] <= row)
      lo = mid;
    else
      hi = mid;
  }
  return {lo, row - p.cu_rows[lo], p.cu_rows[lo + 1] - p.cu_rows[lo]};
}

// The first slot of a sequence's rows (negative: it is not there).
__device__ __forceinline__ int first_slot(const RopeParams& p, int seq) {
  return min((p.start ? p.start : p.c.lengths)[seq], p.c.capacity);
}

// Heads w, w + of, ... (in fours) of one row.  `paged`: K and V go to slot
// `slot` of sequence `seq`.
template <bool kBf16, int kLayout>
__device__ __forceinline__ void row_heads(const RopeParams& p, int row, int position, int w, int of, int seq,
                                          long long slot) {
  const int lane = threadIdx.x & 31, l = lane & (kLanes - 1);
  const int heads = p.num_q + p.num_k * (p.paged ? 2 : 1);
  const int pairs = p.rope.pairs;
  long long at = -1;  // the slot's element offset in the pool
  if (p.paged) {
    int page = -1;
    if (slot < p.c.capacity) page = p.c.table[seq * p.c.table_stride + (slot >> p.c.page_shift)];
    if (page >= 0 && page < p.c.num_pages)
      at = page * p.c.page_stride + (slot & ((1 << p.c.page_shift) - 1)) * p.c.slot_stride;
    else if (w == 0 && lane == 0 && p.status)
      atomicCAS(p.status, 0, CKV_DEV_ERR_INDEX);
  }
  const int fours = (heads + 3) / 4;
  // (the first rows are on their way while the angles are computed)
  Piece x[kUnroll];
  uint16_t* to[kUnroll];
  bool turned[kUnroll];
  auto fetch = [&](int f0) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      int h = (f0 + u * of) * 4 + lane / kLanes;
      to[u] = nullptr;
      turned[u] = false;
      if (h < heads) {
        const uint16_t* from;
        if (h < p.num_q) {
          from = p.q.in + row * p.q.in_token + h * p.q.in_head;
          to[u] = p.q.out + row * p.q.out_token + h * p.q.out_head;
          turned[u] = true;
        } else {
          h -= p.num_q;
          const bool value = h >= p.num_k;
          if (value) h -= p.num_k;
          const RowSet& r = value ? p.v : p.k;
          from = r.in + row * r.in_token + h * r.in_head;
          turned[u] = !value;
          if (!p.paged)
            to[u] = r.out + row * r.out_token + h * r.out_head;
          else if (at >= 0)
            to[u] = p.c.pages[value] + at + h * p.c.head_stride;
        }
        if (to[u]) load<kLayout>(from, l, pairs, x[u]);
      }
    }
  };
  fetch(w);
  Angles t;
  angles_at<kLayout>(p.rope, position, p.backward != 0, lane, t);
  for (int f0 = w;;) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (to[u]) {
        if (turned[u]) turn<kBf16, kLayout>(t, l, pairs, x[u]);
        store<kLayout>(to[u], l, pairs, x[u]);
      }
    f0 += of * kUnroll;
    if (f0 >= fours) break;
    fetch(f0);
  }
}

// A paged row: where it goes, and its position.
template <bool kBf16, int kLayout>
__device__ __forceinline__ void paged_row(const RopeParams& p, int row, const Place& at, int first, int w, int of) {
  const long long slot = static_cast<long long>(first) + at.index;
  const int position = p.positions ? p.positions[row] : static_cast<int>(slot);
  row_heads<kBf16, kLayout>(p, row, position, w, of, at.seq, slot);
}

__device__ __forceinline__ int rows_of(const RopeParams& p, int seq) {
  return p.rows_per_seq >= 0 ? p.rows_per_seq : p.cu_rows[seq + 1] - p.cu_rows[seq];
}
__device__ __forceinline__ void set_length(const RopeParams& p, int seq, int first) {
  if (first >= 0)
    p.c.lengths[seq] = static_cast<int>(min(static_cast<long long>(first) + rows_of(p, seq),
                                            static_cast<long long>(p.c.capacity)));
}

// Warp w of a row's `of` warps.
template <bool kBf16, int kLayout>
__global__ void __launch_bounds__(kThreads, kBlocks) rope_rows_kernel(const __grid_constant__ RopeParams p, int of) {
  if (p.paged && !p.start) pdl_launch_dependents();  // the kernel that sets the lengths follows
  pdl_wait();
  const long long task = static_cast<long long>(blockIdx.x) * kWarps + threadIdx.x / 32;
  const int row = static_cast<int>(task / of), w = static_cast<int>(task - static_cast<long long>(row) * of);
  if (row < p.rows) {
    if (!p.paged) {
      row_heads<kBf16, kLayout>(p, row, p.positions[row], w, of, 0, 0);
    } else {
      const Place at = place_of(p, row);
      const int first = first_slot(p, at.seq);
      if (first >= 0) paged_row<kBf16, kLayout>(p, row, at, first, w, of);
    }
  }
  if (p.paged && p.start && blockIdx.x == 0)  // (nothing reads the lengths then)
    for (int s = threadIdx.x; s < p.c.batch; s += kThreads) set_length(p, s, first_slot(p, s));
}

// A sequence to a CTA, which reads its length before it writes it.
template <bool kBf16, int kLayout>
__global__ void __launch_bounds__(kThreads, kBlocks) append_sequence_kernel(const __grid_constant__ RopeParams p, int of) {
  pdl_wait();
  const int seq = blockIdx.x, first = first_slot(p, seq), rows = rows_of(p, seq);
  const int row0 = p.rows_per_seq >= 0 ? seq * p.rows_per_seq : p.cu_rows[seq];
  __syncthreads();
  if (first < 0) return;
  if (threadIdx.x == 0) set_length(p, seq, first);
  for (int task = threadIdx.x / 32; task < rows * of; task += kWarps) {
    const int i = task / of;
    paged_row<kBf16, kLayout>(p, row0 + i, Place{seq, i, rows}, first, task - i * of, of);
  }
}

__global__ void append_lengths_kernel(const __grid_constant__ RopeParams p) {
  pdl_wait();
  for (int s = threadIdx.x; s < p.c.batch; s += blockDim.x) set_length(p, s, first_slot(p, s));
}

template <bool kBf16, int kLayout>
cudaError_t launch(const RopeParams& p, int most_rows, cudaStream_t stream) {
  const int fours = (p.num_q + p.num_k * (p.paged ? 2 : 1) + 3) / 4;
  if (p.paged && !p.start && most_rows <= kFewRows) {
    const int of = fours < kWarps ? fours : kWarps;
    return launch_dependent(append_sequence_kernel<kBf16, kLayout>, dim3(p.c.batch), kThreads, 0, stream, p, of);
  }
  // a warp a row fills the GPU from some thousands of rows on
  int of = p.rows > 0 ? (kFill + p.rows - 1) / p.rows : 1;
  of = of < 1 ? 1 : of > fours ? fours : of;
  const long long ctas = (static_cast<long long>(p.rows) * of + kWarps - 1) / kWarps;
  const cudaError_t e = launch_dependent(rope_rows_kernel<kBf16, kLayout>, dim3(static_cast<unsigned>(ctas > 0 ? ctas : 1)),
                                         kThreads, 0, stream, p, of);
  if (e != cudaSuccess || !p.paged || p.start) return e;
  return launch_dependent(append_lengths_kernel, dim3(1), 512, 0, stream, p);
}

template <bool kBf16>
cudaError_t launch_layout(const RopeParams& p, int most_rows, cudaStream_t stream) {
  if (p.rope.interleaved) return launch<kBf16, kNeighbours>(p, most_rows, stream);
  if (p.rope.pairs % kPairsLane == 0) return launch<kBf16, kHalves>(p, most_rows, stream);
  return launch<kBf16, kOddHalves>(p, most_rows, stream);
}

}  // namespace

cudaError_t launch_rope(const RopeParams& p, cudaStream_t stream) {
  return p.is_bf16 ? launch_layout<true>(p, 0, stream) : launch_layout<false>(p, 0, stream);
}
cudaError_t launch_paged_append(const RopeParams& p, int most_rows, cudaStream_t stream) {
  return p.is_bf16 ? launch_layout<true>(p, most_rows, stream) : launch_layout<false>(p, most_rows, stream);
}

}  // namespace ckv
