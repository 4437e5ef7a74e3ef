// Attention of chunks of query tokens over a paged cache.
//
// A row is one head of one query token.  For the rows of a KV group, over the
// slots j that a row sees,
//   z_j = q . K_j,  p_j = 2^(c z_j - c m),  l = sum p_j,  out = sum p_j V_j / l,
// in one pass: m is the largest logit so far, and when it has grown by more than
// 2^8 in p, l and the output so far are scaled by 2^(c (m_old - m)).  (Until then
// m stays: p is at most 2^8, which fp32 sums and the 16-bit types hold as well as
// 1.)  Logits and output are products on the tensor cores (tcgen05), 128 rows by
// 128 slots at a time, with fp32 accumulators in tensor memory; p enters the
// second product rounded to the 16-bit type, from tensor memory, while l sums it
// unrounded.
//
// One CTA per SM, in roles: four warps a 128-row tile for the softmax, one lane of
// them a row; a warp that finds the work and moves Q, K and V by TMA; one a
// tile that issues the products; and one that makes V fit for tiles of which some
// rows see only a part.  Two forms:
//  * kPair, for chunks: two 128-row tiles of the same KV group and sequence share
//    each tile of K and V, and while the tensor cores work for one, the other's
//    softmax runs.  An item is two tiles of rows; where there are few items for
//    the SMs, all their tiles are shared in equal runs, else items are taken by
//    ticket, so that CTAs that run together read the same K and V, and only the
//    last ones are shared in runs.
//  * single, where 128 rows hold all query tokens of a sequence (decode): the
//    bytes of K and V bound it.  The tiles of all units form one sequence, of which
//    each CTA takes an equal run; logits of the next tile are made while the
//    softmax of this one runs.
// What the pieces of an item leave in the workspace (output, reference and sum in
// fp32) is joined by whichever CTA finishes the last of them, in the order of the
// slots.
#include "ckv_device.cuh"
#include "paged_params.h"
#include "q4_params.h"

namespace ckv {
namespace {

constexpr int kTile = kPagedTile;
constexpr int kThreads = 384;
constexpr int kMmaWarp = 0, kLoadWarp = 1, kFixWarp = 2;    // (kPair: 3 issues for the second tile)
constexpr int kSoftWarp = 4;                                // 4 .. 7 and 8 .. 11: softmax of a tile of rows
constexpr int kHalf = kTile * 128;                          // 64 channels of a tile, bytes
constexpr int kTileBytes2 = 2 * kHalf;                      // K, V or Q: 32 KB
constexpr int kRing = 4;                                    // piece descriptors
constexpr int kAhead = 4;                                   // tiles to load when the next piece is found,
constexpr int kTicketAhead = 2;                             // and more when its ticket is taken
constexpr int kDiagTiles = 3;                               // tiles that an item's rows see in part, at most
constexpr float kGrowth = 8.f;                              // log2 of how far p may pass 1
constexpr float kFar = 0x1p18f;                             // references from where fp32's steps in them count

// A part of an item's slots, as the roles get it.
struct Piece {
  int go;                 // 0: no more pieces
  int first;              // of the call
  int seq, head;
  int row0;               // packed row of the item's first token
  int tokens;             // of the item
  int pos0;               // slot of its first token
  int length;             // slots in use
  int tile0;              // first tile
  int tiles[2];           // of each 128-row tile (its rows see none behind); 0: not there
  int pieces[2];          // of the item, for each 128-row tile; 1: the piece is all of it
  int slot;               // where the piece's results go
  // CTA (kPair: run) that has the item's first tile.  The others' are those behind
  // it; its own piece begins the item, so its slot is 2 base + 1, theirs 2 (base + k).
  int base;
  __device__ long long slot_of(int k) const { return k == 0 ? 2 * base + 1 : 2 * (base + k); }
};

template <bool kPair>
struct Shape {
  static constexpr int kQTiles = kPair ? 2 : 1;
  static constexpr int kStages = kPair ? 5 : 6;
  static constexpr int kConsumers = kPair ? 11 : 10;  // warps that read a piece
};

struct Misc {
  // a piece's first K; V of a tile with K of the next; stages free again; V fixed
  uint64_t kfull[kRing], full[kRing], empty[6], vready[kRing];
  uint64_t qfull[4], qempty[4], sfull[2], pready[2][2], odone[2], oempty[2];
  uint64_t sready[2], oready[2], stored;  // single: a piece's references and sums, output, and output in memory
  uint64_t pfull[kRing], pempty[kRing], drain[2], turn[2];
  Piece ring[kRing];
  uint32_t poison[kRing][kDiagTiles][4];  // slots whose V holds what is not finite,
  uint32_t found[kRing];                  // and whether there are any
  float2 sums[2][kTile];
  uint32_t tmem;
  int abort;
};
constexpr int kOperandBytes = 7 * kTileBytes2;  // (2 + 5 or 1 + 6)
constexpr int kSmemBytes = kOperandBytes + static_cast<int>(sizeof(Misc));
static_assert(kSmemBytes <= 232448, "shared memory");

__device__ __forceinline__ uint64_t l2_policy_evict_normal() {
  uint64_t p;
  asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(p));
  return p;
}

// ------------------------------------------------------------------- numbers
template <bool kBf16>
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  if (!kBf16) return pack_half2(lo, hi);
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <bool kBf16>
__device__ __forceinline__ float value(uint32_t w) {  // of the low half
  if (kBf16) return __uint_as_float(w << 16);
  float r;
  asm("{\n\t.reg .f16 h, g;\n\tmov.b32 {h, g}, %1;\n\tcvt.f32.f16 %0, h;\n\t}" : "=f"(r) : "r"(w));
  return r;
}
__device__ __forceinline__ uint64_t pair_of(float x, float y) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ float2 split_of(uint64_t p) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(p));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// ------------------------------------------------------------- tensor memory
__device__ __forceinline__ void tmem_store16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t taddr, uint32_t (&r)[16]) {  // and waits
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
// The product of an operand in tensor memory (rows in lanes, two numbers of K to
// a column) and one in shared memory.
__device__ __forceinline__ void umma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc,
                                            uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// V as the right operand: rows of slots, 64 channels (128 bytes, swizzled) to a
// row; groups of 8 rows 1024 bytes apart, the other 64 channels kHalf further.
__device__ __forceinline__ uint64_t v_desc(uint32_t saddr) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr >> 4) & 0x3FFFu);
  d |= static_cast<uint64_t>(kHalf >> 4) << 16;  // between the two groups of 64 channels
  d |= static_cast<uint64_t>(1024 >> 4) << 32;   // between groups of 8 slots
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(2) << 61;           // 128-byte swizzle
  return d;
}

// One lane of a converged warp; the compiler then knows that no other runs what
// follows.
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}

// The rest of a wait, out of line: the roles' loops run from the instruction
// caches, and code that hardly ever runs between them costs every pass over it.
__device__ __noinline__ bool wait_on(uint32_t bar, uint32_t parity, volatile int* abort, int* status, int* stopped,
                                     uint64_t ns) {
  const bool ok = mbar_wait_bounded(bar, parity, abort, status, ns);
  if (!ok) atomicExch(stopped, 1);
  return ok;
}

// ------------------------------------------------------------------- the call
struct Cta {
  const PagedAttendParams& p;
  Misc* m;
  uint32_t smem;  // of the operands: Q tiles, then the stages
  // Bounded wait on a phase; false: this CTA stops.
  __device__ __forceinline__ bool wait(uint64_t& bar, uint32_t parity) const {
    const uint32_t at = smem_u32(&bar);
    return mbar_try_wait(at, parity) || wait_on(at, parity, &m->abort, p.status, p.stopped, kWaitTimeoutNs);
  }
  __device__ __forceinline__ bool wait_warp(uint64_t& bar, uint32_t parity) const {
    return __all_sync(0xffffffffu, wait(bar, parity));
  }
  // (without a call: the softmax's registers are full)
  __device__ __forceinline__ bool wait_here(uint64_t& bar, uint32_t parity) const {
    const bool ok = mbar_wait_bounded(smem_u32(&bar), parity, &m->abort, p.status);
    if (!ok) atomicExch(p.stopped, 1);
    return __all_sync(0xffffffffu, ok);
  }
  __device__ __forceinline__ bool stopped() const { return *reinterpret_cast<volatile int*>(&m->abort) != 0; }
};

// A piece from the ring, for a whole warp; the last use of it is followed by done().
struct Reader {
  const Cta& c;
  int at = 0;
  __device__ __forceinline__ const Piece* next() {
    if (!c.wait_here(c.m->pfull[at % kRing], (at / kRing) & 1)) return nullptr;
    const Piece* x = &c.m->ring[at % kRing];
    return x->go ? x : nullptr;
  }
  __device__ __forceinline__ void done() {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&c.m->pempty[at % kRing]));
    ++at;
  }
};

__device__ __forceinline__ int clamp_to(long long x, int lo, int hi) {
  return static_cast<int>(x < lo ? lo : x > hi ? hi : x);
}
// Slots that the token at slot `pos` sees.
__device__ __forceinline__ int limit_of(const PagedAttendParams& p, int pos, int length) {
  return p.causal ? min(max(pos + 1, 0), length) : length;
}
__device__ __forceinline__ int tiles_of(int limit) { return max((limit + kTile - 1) / kTile, 1); }

// p enters the product with V times 2^-down, and the output leaves it times 2^down.
// bf16: a sum of p V (2^8 in each of `length` slots, at most) would pass fp32's range
// where V is large and the output is not; V below 2^(down - 126) may be lost for it.
// f16: its V is small enough for any sum, and its p has room above: 2^8 times 2^7 is
// half of its largest number.  Without that, p below 2^-14 of the reference had fewer
// bits and below 2^-25 none: what 32K slots, each 18 nats below a sink, add up to was
// off by 42 % (2-norm; 0.4 % so), and slots 16 +- 1 below it by 4 % (0.1 %).
constexpr float kDownF16 = -7.f;
static_assert(kGrowth - kDownF16 < 16.f, "p is below 2^16 in f16");
template <bool kBf16>
__device__ __forceinline__ float down_of(int length) {
  return kBf16 ? static_cast<float>(static_cast<int>(kGrowth) + 32 - __clz(length)) : kDownF16;
}
template <bool kBf16>
__device__ __forceinline__ float up_of(int length) {  // 2^down
  return kBf16 ? __int_as_float((127 + static_cast<int>(kGrowth) + 32 - __clz(length)) << 23)
               : __int_as_float((127 + static_cast<int>(kDownF16)) << 23);
}

// A sequence, as a lane of the work-finding warp sees it.
struct Sequence {
  int rows, row0, length, start;
  __device__ void load(const PagedAttendParams& p, int s) {
    rows = row0 = length = start = 0;
    if (s >= p.c.batch) return;
    row0 = p.rows_per_seq >= 0 ? s * p.rows_per_seq : p.cu_rows[s];
    rows = p.rows_per_seq >= 0 ? p.rows_per_seq : p.cu_rows[s + 1] - row0;
    length = max(min(p.c.lengths[s], p.c.capacity), 0);
    // (far beyond any slot or token all positions are alike)
    start = p.start ? clamp_to(p.start[s], -(1 << 28), 1 << 28) : length - rows;
  }
  // Tiles that tokens first .. last - 1 see together.
  __device__ int tiles(const PagedAttendParams& p, int last) const {
    return tiles_of(limit_of(p, start + last - 1, length));
  }
};

__device__ __forceinline__ int warp_prefix(int x, int lane) {  // inclusive
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  return x;
}

__device__ __forceinline__ long long warp_prefix(long long x, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  return x;
}
// (64-bit divisions take some hundred instructions, 32-bit ones far fewer)
__device__ __forceinline__ long long quotient(long long a, long long b) {
  return (a | b) >> 32 ? a / b : static_cast<long long>(static_cast<uint32_t>(a) / static_cast<uint32_t>(b));
}

// kPair: the items of a sequence and head, those that see most first, on the line of
// all work: an item takes its tiles and kPagedPiece.  (As if they grew evenly, so
// that a position is found by arithmetic; what an item has beyond or short of that
// makes a piece a tile longer or shorter.)
struct Items {
  int count, low, high;  // tiles of the item that sees least, and most
  __device__ void load(const PagedAttendParams& p, const Sequence& x) {
    count = low = high = 0;
    if (x.rows <= 0) return;
    count = (x.rows + p.item_tokens - 1) / p.item_tokens;
    low = x.tiles(p, min(p.item_tokens, x.rows));
    high = x.tiles(p, x.rows);
  }
  __device__ long long before(int n) const {  // of the first n
    if (n == 0) return 0;
    const long long steps = static_cast<long long>(n) * (n - 1) * (high - low);
    return static_cast<long long>(n) * (high + kPagedPiece) - quotient(steps, 2 * max(count - 1, 1));
  }
};

// Finds the pieces of this CTA, a warp together.
template <bool kPair>
struct Finder {
  const PagedAttendParams& p;
  int lane;
  // the 32 sequences that the lanes hold, and what came before them
  int group = -1;
  Sequence s;
  // kPair: items, and work, before what the lane holds and with it
  Items it;
  int items_upto = 0, items_before = 0;
  long long work_upto = 0, work_before = 0;
  int whole = 0, runs = 0;     // items that are a piece, and runs of the work behind them
  long long body = 0;          // work of the former
  bool taken = false;          // a ticket that is still to be used:
  int ticket = 0, run = 0;     // of lane 0, and run at hand (negative: an item)
  long long all = 0, at = 0, end = 0;  // work, and this CTA's next
  // single
  int ctas = 0;
  int mine = 0, upto = 0;      // tiles of a head; and prefix, inclusive
  int before = 0;
  // (K and V of chunks are read by many CTAs; single's once)
  uint64_t policy = kPair ? l2_policy_evict_last() : l2_policy_evict_normal();

  __device__ void hold(int g) {
    group = g;
    s.load(p, g * 32 + lane);
    if (kPair) {
      const int heads = p.c.num_kv_heads;
      it.load(p, s);
      work_upto = warp_prefix(it.before(it.count) * heads, lane);
      items_upto = warp_prefix(it.count * heads, lane);
    } else {
      mine = s.rows > 0 ? s.tiles(p, s.rows) : 0;
      upto = warp_prefix(mine, lane);
    }
  }
  __device__ bool advance() {  // to the next 32
    if ((group + 1) * 32 >= p.c.batch) return false;
    if (kPair) {
      items_before += __shfl_sync(0xffffffffu, items_upto, 31);
      work_before += __shfl_sync(0xffffffffu, work_upto, 31);
    } else {
      before += __shfl_sync(0xffffffffu, upto, 31);
    }
    hold(group + 1);
    return true;
  }
  __device__ void rewind() {
    if (group == 0) return;
    before = items_before = 0;
    work_before = 0;
    hold(0);
  }
  __device__ int groups() const { return (p.c.batch + 31) / 32; }

  // kPair: an item of the line: its sequence, head and number, and where it begins.
  struct Place {
    int src, head, number;
    Sequence q;
    Items it;
    long long from;  // (found by position)
  };
  // By its number on the line, or by a position in it (neither goes back).
  template <bool kNumber>
  __device__ Place locate(long long want) {
    while (want >= (kNumber ? items_before + __shfl_sync(0xffffffffu, items_upto, 31)
                            : work_before + __shfl_sync(0xffffffffu, work_upto, 31)))
      if (!advance()) break;
    const long long to = kNumber ? items_before + items_upto : work_before + work_upto;
    const int src = max(__ffs(__ballot_sync(0xffffffffu, to > want)) - 1, 0);
    Place y;
    y.src = src;
    y.q.rows = __shfl_sync(0xffffffffu, s.rows, src);
    y.q.row0 = __shfl_sync(0xffffffffu, s.row0, src);
    y.q.length = __shfl_sync(0xffffffffu, s.length, src);
    y.q.start = __shfl_sync(0xffffffffu, s.start, src);
    y.it.count = __shfl_sync(0xffffffffu, it.count, src);
    y.it.low = __shfl_sync(0xffffffffu, it.low, src);
    y.it.high = __shfl_sync(0xffffffffu, it.high, src);
    if (kNumber) {
      const int in = static_cast<int>(want) - (items_before + __shfl_sync(0xffffffffu, items_upto, src) -
                                               y.it.count * p.c.num_kv_heads);
      y.head = in / y.it.count;
      y.number = in - y.head * y.it.count;
      y.from = 0;
    } else {
      const long long work = y.it.before(y.it.count);
      const long long first = work_before + __shfl_sync(0xffffffffu, work_upto, src) - work * p.c.num_kv_heads;
      y.head = static_cast<int>(quotient(want - first, work));
      const long long in = want - first - y.head * work;
      int at = 0, n = y.it.count;  // it is one of these
      while (n > 1) {
        const int step = (n + 31) / 32, mine = at + step * lane;
        const unsigned ok = __ballot_sync(0xffffffffu, step * lane < n && y.it.before(mine) <= in);
        const int k = 31 - __clz(ok);
        at += step * k;
        n = min(step, n - step * k);
      }
      y.number = at;
      y.from = first + y.head * work + y.it.before(at);
    }
    return y;
  }
  // The tile of an item of n at which a run that ends `in` behind the item's
  // beginning ends.  (No pieces of a few tiles.)
  static __device__ int tile_at(long long in, int n) {
    const long long k = in - kPagedPiece;
    return k < kPagedLeast ? 0 : n - k < kPagedLeast ? n : static_cast<int>(k);
  }

  // kPair: where items are many, each is a piece, taken in turn, but for the last ones:
  // that work, or where items are few all, is shared in equal runs.
  __device__ void plan() {
    const int grid = static_cast<int>(gridDim.x);
    hold(0);
    int longest = it.high;
    while (advance()) longest = max(longest, it.high);
    longest = __reduce_max_sync(0xffffffffu, longest);
    all = work_before + __shfl_sync(0xffffffffu, work_upto, 31);
    const int items = items_before + __shfl_sync(0xffffffffu, items_upto, 31);
    rewind();
    if (all == 0) return;
    runs = grid;
    if (static_cast<long long>(kPagedFew) * longest * grid <= all) {
      // An eighth of the longest item a CTA; of items that are nearly alike all behind
      // the last full round, if that leaves many CTAs without one.
      const long long most = longest + kPagedPiece;
      long long tail = (grid * most + 7) / 8;
      const int left = items % grid;
      if (8 * all >= 7 * most * items && 4 * left < 3 * grid) tail = max(tail, left * most);
      const Place y = locate<false>(max(all - tail, 0LL));
      whole = items_before + __shfl_sync(0xffffffffu, items_upto, y.src) - (p.c.num_kv_heads - y.head) * y.it.count +
              y.number;
      body = y.from;
      runs = kPagedRuns * grid;
      rewind();
    }
    runs = clamp_to((all - body) / kPagedShare, 1, min(runs, kPagedSlots / 2));
  }

  // kPair: a ticket for find(), which need not wait for it then.
  __device__ void take() {
    if (!kPair || taken || at < end) return;
    if (lane == 0) ticket = atomicAdd(p.next, 1);
    taken = true;
  }
  __device__ void start() {
    if (kPair) {
      take();
      plan();
    } else {
      hold(0);
      int n = __shfl_sync(0xffffffffu, upto, 31);
      while (advance()) n += __shfl_sync(0xffffffffu, upto, 31);
      all = static_cast<long long>(n) * p.c.num_kv_heads;
      ctas = static_cast<int>(min(static_cast<long long>(gridDim.x), all));
      if (blockIdx.x < ctas) {
        at = quotient(all * blockIdx.x, ctas);
        end = quotient(all * (blockIdx.x + 1), ctas);
      }
      rewind();
    }
  }

  // Into *x by lane 0; false: there is none.
  __device__ bool find(Piece* x) { return kPair ? find_chunk(x) : find_single(x); }

  __device__ bool find_chunk(Piece* x) {
    Piece y;
    Place i;
    int from, to, most[2];  // tiles of the item
    long long next = 0;  // where on the line the item after it begins
    for (;;) {
      y.first = 0;
      if (at >= end) {
        take();
        const int n = __shfl_sync(0xffffffffu, ticket, 0);
        taken = false;
        if (n >= whole + runs) return false;
        y.first = n == 0;
        run = n - whole;
        if (run >= 0) {
          at = body + quotient((all - body) * run, runs);
          end = body + quotient((all - body) * (run + 1), runs);
        }
      }
      i = run < 0 ? locate<true>(whole + run) : locate<false>(at);
      const int token = (i.it.count - 1 - i.number) * p.item_tokens;
      y.row0 = i.q.row0 + token;
      y.tokens = min(p.item_tokens, i.q.rows - token);
      y.pos0 = i.q.start + token;
      const int tokens_a = min(p.item_tokens / 2, y.tokens);
      most[0] = i.q.tiles(p, token + tokens_a);
      most[1] = i.q.tiles(p, token + y.tokens);
      from = 0;
      to = most[1];
      if (run >= 0) {
        next = i.from + i.it.before(i.number + 1) - i.it.before(i.number);
        from = tile_at(at - i.from, most[1]);
        if (end < next) to = tile_at(end - i.from, most[1]);
        at = min(end, next);
      }
      if (from < to) break;
    }
    y.go = 1;
    y.seq = group * 32 + i.src;
    y.head = i.head;
    y.length = i.q.length;
    y.tile0 = from;
    y.tiles[0] = max(min(most[0], to) - from, 0);
    y.tiles[1] = y.tokens > p.item_tokens / 2 ? to - from : 0;
    y.pieces[0] = y.pieces[1] = 1;
    y.base = y.slot = 0;
    if (run >= 0) {
      // the runs that begin inside the item are consecutive: from tile kPagedLeast on,
      // before the last kPagedLeast (and before the last that the first 128 rows see)
      auto begun = [&](long long x) { return quotient((x - body) * runs + all - body - 1, all - body); };
      const long long tile = i.from + kPagedPiece;
      const long long past = min(tile + most[1] - kPagedLeast + 1, next);
      const long long first = begun(tile + kPagedLeast);
      const int inside = static_cast<int>(max(begun(past) - first, 0LL));
      y.pieces[1] = inside + 1;
      y.pieces[0] = min(static_cast<int>(max(begun(min(past, tile + most[0])) - first, 0LL)), inside) + 1;
      y.base = inside ? static_cast<int>(first) - 1 : run;
      y.slot = 2 * run + (from == 0);
    }
    if (lane == 0) *x = y;
    return true;
  }

  __device__ bool find_single(Piece* x) {
    const int heads = p.c.num_kv_heads;  // that `mine` counts one of
    if (at >= end) return false;
    while (at >= static_cast<long long>(before + __shfl_sync(0xffffffffu, upto, 31)) * heads)
      if (!advance()) return false;
    const unsigned over = __ballot_sync(0xffffffffu, static_cast<long long>(before + upto) * heads > at);
    const int src = __ffs(over) - 1;
    const int count = __shfl_sync(0xffffffffu, mine, src);
    const long long first = static_cast<long long>(before + __shfl_sync(0xffffffffu, upto, src) - count) * heads;
    const int in_seq = static_cast<int>(at - first);
    const int head = in_seq / count, rest = in_seq - head * count;
    Piece y;
    y.go = 1;
    y.first = at == 0;
    y.seq = group * 32 + src;
    y.length = __shfl_sync(0xffffffffu, s.length, src);
    y.head = head;
    y.row0 = __shfl_sync(0xffffffffu, s.row0, src);
    y.tokens = __shfl_sync(0xffffffffu, s.rows, src);
    y.pos0 = __shfl_sync(0xffffffffu, s.start, src);
    y.tile0 = rest;
    const int n = static_cast<int>(min(static_cast<long long>(count - rest), end - at));
    y.tiles[0] = n;
    y.tiles[1] = 0;
    const long long u0 = first + static_cast<long long>(head) * count;  // the unit's first tile
    auto owner = [&](long long tile) { return static_cast<int>(quotient((tile + 1) * ctas - 1, all)); };
    y.base = owner(u0);
    y.pieces[0] = y.pieces[1] = owner(u0 + count - 1) - y.base + 1;
    y.slot = 2 * static_cast<int>(blockIdx.x) + (rest == 0);
    at += n;
    if (lane == 0) *x = y;
    return true;
  }
};

// ---------------------------------------------------------------- TMA warp
// Waits for a phase whether the CTA stops or not.
__device__ void settle(uint64_t& bar, uint32_t parity, uint64_t ns) {
  const uint64_t t0 = globaltimer_ns();
  while (!mbar_try_wait(smem_u32(&bar), parity) && globaltimer_ns() - t0 < ns) {
  }
}

template <bool kPair>
__device__ void load_role(const Cta& c) {
  using S = Shape<kPair>;
  const PagedAttendParams& p = c.p;
  const int lane = threadIdx.x & 31;
  const int page = 1 << p.c.page_shift, box = min(page, kTile), copies = 2 * (kTile / box);
  // a call that stopped may have left tickets behind: nothing runs until the
  // workspace is set up again
  const bool go = *reinterpret_cast<volatile int*>(p.stopped) == 0;
  Finder<kPair> f{p, lane};
  f.start();
  int pos = 0, pieces = 0, count = 0;  // stages filled; pieces and tiles begun
  // kPair: a Q buffer for each tile of rows; single: as many, for pieces to come, as
  // their rows leave room for (a tile's rows behind them are whatever lies there)
  const int q_step = kPair ? kTileBytes2 : kHalf / p.q_buffers;
  uint32_t q_used = 0, q_phase = 0;  // a bit for each buffer
  // this lane's page of a tile (not yet checked)
  auto look_up = [&](const Piece& x, int tile) {
    const int slot = tile * kTile + (lane >> 1) * box;
    if (lane >= copies || slot >= x.length) return p.c.num_pages;
    const int e = p.c.table[x.seq * p.c.table_stride + (slot >> p.c.page_shift)];
    return e;
  };
  // `arm`: bytes that the barrier is to wait for from here on
  auto load_tile = [&](const Piece& x, const CUtensorMap& map, int tile, int entry, uint64_t& full, uint32_t arm) {
    const int st = pos % S::kStages;
    if (!c.wait_warp(c.m->empty[st], ((pos / S::kStages) & 1) ^ 1)) return false;
    const uint32_t bar = smem_u32(&full);
    if (lane == 0 && arm) mbar_arrive_expect_tx(bar, arm);
    __syncwarp();
    ++pos;
    if (lane < copies) {
      const int half = lane & 1, part = lane >> 1;
      if (entry < 0 || entry > p.c.num_pages ||
          (entry == p.c.num_pages && tile * kTile + part * box < x.length)) {
        atomicCAS(p.status, 0, CKV_DEV_ERR_INDEX);
        entry = p.c.num_pages;
      }
      // (a page behind the pool, as behind the length, is read as zeros)
      tma_load_4d(c.smem + (S::kQTiles + st) * kTileBytes2 + half * kHalf + part * box * 128, &map, bar, half * 64,
                  x.head, (tile * kTile) & (page - 1), entry, f.policy);
    }
    return true;
  };
  auto load_q = [&](const Piece& x, int t, int buffer) {
    if (!c.wait_warp(c.m->qempty[buffer], ((q_phase >> buffer) & 1) ^ 1)) return false;
    if (lane == 0) {
      const uint32_t bar = smem_u32(&c.m->qfull[buffer]);
      mbar_arrive_expect_tx(bar, p.q_box_bytes * 2);
      for (int half = 0; half < 2; ++half)
        tma_load_3d(c.smem + buffer * q_step + half * kHalf, &p.map_q, bar, half * 64, x.head * p.group,
                    x.row0 + t * p.tile_tokens, f.policy);
    }
    __syncwarp();
    q_used |= 1u << buffer;
    q_phase ^= 1u << buffer;
    return true;
  };
  bool found = false;
  auto find = [&](int n) {
    if (!c.wait_warp(c.m->pempty[n % kRing], ((n / kRing) & 1) ^ 1)) return false;
    Piece& x = c.m->ring[n % kRing];
    found = go && f.find(&x);
    if (!found && lane == 0) x.go = 0;
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&c.m->pfull[n % kRing]));
    return true;
  };
  bool ok = find(0);
  for (int n = 0; ok && found; ++n) {
    const Piece& x = c.m->ring[n % kRing];
    const int tiles = max(x.tiles[0], x.tiles[1]), first = x.tile0;
    int now = look_up(x, first), next = tiles > 1 ? look_up(x, first + 1) : 0;
    ok = load_tile(x, p.map_k, first, now, c.m->kfull[n % kRing], kTileBytes2);
    pieces += ok;
    for (int t = 0; ok && t < S::kQTiles; ++t)
      if (x.tiles[t]) ok = load_q(x, t, kPair ? t : n % p.q_buffers);
    for (int j = 0; ok && j < tiles; ++j) {
      if (j == max(tiles - kAhead - kTicketAhead, 0)) f.take();
      const int after = j + 2 < tiles ? look_up(x, first + j + 2) : 0;
      const bool more = j + 1 < tiles;
      uint64_t& full = c.m->full[count % kRing];
      if (more) {
        ok = load_tile(x, p.map_k, first + j + 1, next, full, 2 * kTileBytes2);
        count += ok;
      }
      if (ok) ok = load_tile(x, p.map_v, first + j, now, full, more ? 0 : kTileBytes2);
      count += ok && !more;
      now = next;
      next = after;
      // (kPair: so early that the piece's first tiles are not late, so late that the
      // CTA that is through first takes it)
      if (kPair && ok && j == max(tiles - 1 - kAhead, 0)) ok = find(n + 1);
    }
    if (!kPair && ok) ok = find(n + 1);
  }
  // No copy, and no arrival that a stage or Q tile is free again, may come after
  // this CTA has ended.  (A stopped CTA has only its copies to wait for.)
  const bool all = !c.stopped();
  if (all) {
    for (int i = max(pos - S::kStages, 0); i < pos; ++i)
      c.wait_warp(c.m->empty[i % S::kStages], (i / S::kStages) & 1);
  } else {
    for (int i = max(pieces - kRing, 0); i < pieces; ++i)
      settle(c.m->kfull[i % kRing], (i / kRing) & 1, 100000000ull);
    for (int i = max(count - kRing, 0); i < count; ++i)
      settle(c.m->full[i % kRing], (i / kRing) & 1, 100000000ull);
  }
  for (int i = 0; i < kRing; ++i)
    if ((q_used >> i) & 1) {
      if (all)
        c.wait_warp(c.m->qempty[i], ((q_phase >> i) & 1) ^ 1);
      else
        settle(c.m->qfull[i], ((q_phase >> i) & 1) ^ 1, 100000000ull);
    }
}

// ---------------------------------------------------------------- products
// One lane does a tile's products (a wait of a whole warp costs 110 to 150 cycles
// even where there is nothing to wait for).  With kPair two lanes of two warps take
// turns, so that one tile's softmax runs beside the other's products, and each
// waits for its operands while the other issues: one lane for both spent 2600 of a
// tile's 2048 cycles of products, and two without turns fell into step, both
// softmaxes at a time and then all products.
template <bool kBf16, bool kPair>
__device__ void product_role(const Cta& c, uint32_t tmem, int t) {
  using S = Shape<kPair>;
  constexpr uint32_t kQk = umma_idesc_f16(kTile, kTile, kBf16);
  constexpr uint32_t kPv = kQk | 1u << 16;  // V: channels, not slots, are contiguous
  const uint32_t stages = c.smem + S::kQTiles * kTileBytes2;
  auto bar = [&](uint64_t& b) { return smem_u32(&b); };
  const int q_step = kPair ? kTileBytes2 : kHalf / c.p.q_buffers;
  auto logits = [&](int q, int buffer, int st) {
    const uint64_t a = smem_desc_sw128(c.smem + q * q_step);
    const uint64_t b = smem_desc_sw128(stages + st * kTileBytes2);
#pragma unroll
    for (int i = 0; i < kHeadDim / 16; ++i) {
      const uint64_t step = (i / 4) * (kHalf >> 4) + (i % 4) * 2;
      umma_f16(tmem + buffer * kTile, a + step, b + step, kQk, i > 0);
    }
  };
  auto output = [&](int o, int buffer, int st, bool more, int i0, int i1) {
    const uint64_t b = v_desc(stages + st * kTileBytes2);
#pragma unroll
    for (int i = i0; i < i1; ++i)
      umma_f16_ts(tmem + (2 + o) * kTile, tmem + buffer * kTile + i * 8, b + i * (2048 >> 4), kPv, more || i > 0);
  };
  int at = 0, count = 0;  // the next stage; tiles
  auto step = [&] {
    const int st = at;
    at = at + 1 == S::kStages ? 0 : at + 1;
    return st;
  };
  uint32_t v_phase = 0, q_phase = 0, o_phase = 3;  // bits: of the ring, of Q buffers, of outputs
  int done = 0;                                    // tiles with products
  uint32_t turn = t ^ 1;
  // A lane's turn to issue.
  auto begin = [&] {
    const bool ok = !kPair || c.wait(c.m->turn[t], turn);
    turn ^= 1;
    return ok;
  };
  auto end = [&] {
    if (kPair) mbar_arrive(bar(c.m->turn[t ^ 1]));
  };
  auto drop = [&](int st) { mbar_arrive(bar(c.m->empty[st])); };  // a stage that this tile's rows do not need
  bool ok = true;
  for (int piece = 0; ok; ++piece) {
    if (!(ok = c.wait(c.m->pfull[piece % kRing], (piece / kRing) & 1))) break;
    const Piece& x = c.m->ring[piece % kRing];
    if (!x.go) break;
    const int n = x.tiles[t], tiles = kPair ? max(n, x.tiles[t ^ 1]) : n;
    const bool stall = c.p.stall_ns != 0 && x.first;
    const int in_part = limit_of(c.p, x.pos0, x.length) / kTile - x.tile0;  // first tile that not all rows see whole
    mbar_arrive(bar(c.m->pempty[piece % kRing]));
    if (!(ok = c.wait(c.m->kfull[piece % kRing], (piece / kRing) & 1))) break;
    const int k0 = step(), q = kPair ? t : piece % c.p.q_buffers, o = kPair ? t : piece & 1;
    if (n) {
      ok = c.wait(c.m->qfull[q], (q_phase >> q) & 1) && begin();
      q_phase ^= 1u << q;
      if (!ok) break;
      const int buffer = kPair ? t : done & 1;
      tc_fence_after();
      logits(q, buffer, k0);
      end();
      umma_commit(bar(c.m->sfull[buffer]));
      umma_commit(bar(c.m->empty[k0]));
      if (n == 1) umma_commit(bar(c.m->qempty[q]));
    } else {
      if (!(ok = begin())) break;
      end();
      drop(k0);
    }
    if (stall) {  // test hook: a wait for what nothing completes
      wait_on(bar(c.m->drain[t]), 0, &c.m->abort, c.p.status, c.p.stopped, c.p.stall_ns);
      break;
    }
#pragma unroll 1
    for (int j = 0; ok && j < tiles; ++j) {
      const bool more = j + 1 < tiles;
      const int k = more ? step() : 0, v = step(), slot = count % kRing;
      ok = c.wait(c.m->full[slot], (count / kRing) & 1);
      ++count;
      if (ok && j >= in_part) {
        ok = c.wait(c.m->vready[slot], (v_phase >> slot) & 1);
        v_phase ^= 1u << slot;
      }
      if (!ok) break;
      if (j >= n) {
        if (!(ok = begin())) break;
        end();
        drop(v);
        if (more) drop(k);
        continue;
      }
      const int buffer = kPair ? t : done & 1, phase = (kPair ? done : done >> 1) & 1;
      ++done;
      if (!kPair && more) {  // the next tile's logits beside this one's softmax
        tc_fence_after();
        logits(q, buffer ^ 1, k);
        umma_commit(bar(c.m->sfull[buffer ^ 1]));
        umma_commit(bar(c.m->empty[k]));
        if (j + 2 == n) umma_commit(bar(c.m->qempty[q]));
      }
      if (j == 0) {
        ok = c.wait(c.m->oempty[o], (o_phase >> o) & 1);
        o_phase ^= 1u << o;
      }
      if (!(ok = ok && c.wait(c.m->pready[buffer][0], phase) && begin())) break;
      tc_fence_after();
      output(o, buffer, v, j > 0, 0, kTile / 32);
      if (!(ok = c.wait(c.m->pready[buffer][1], phase))) break;
      tc_fence_after();
      output(o, buffer, v, true, kTile / 32, kTile / 16);
      if (kPair && j + 1 < n) {
        logits(t, t, k);
        end();
        umma_commit(bar(c.m->sfull[t]));
        umma_commit(bar(c.m->empty[v]));
        umma_commit(bar(c.m->empty[k]));
        if (j + 2 == n) umma_commit(bar(c.m->qempty[t]));
      } else {
        end();
        umma_commit(bar(c.m->odone[t]));
        if (!kPair && !more) umma_commit(bar(c.m->oready[o]));
        umma_commit(bar(c.m->empty[v]));
        if (kPair && more) drop(k);
      }
    }
  }
  // every product, and every arrival that waits for one, is over before the
  // tensor memory is given back
  umma_commit(bar(c.m->drain[t]));
  settle(c.m->drain[t], 0, 1000000000ull);
}

// ---------------------------------------------------------------- V of tiles that rows see in part
// A hidden slot has p = 0, but 0 times what is not finite is not 0.  In tiles that
// the item's first token does not see whole, rows of slots behind the length
// become zero, and what is not finite in slots that other tokens see: those slots
// are noted, and the rows that do see them get it added to their output.
// (Eight slots at a time.  x times 0 is 0, or NaN where x is not
// finite: a multiply-add a pair of channels finds the few that need a closer look.
// Looking at each exponent took up to 8700 cycles a tile.)
template <bool kBf16>
__device__ __forceinline__ uint32_t add_zeros(uint32_t x, uint32_t sum) {
  if (kBf16)
    asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(x), "r"(0));
  else
    asm("fma.rn.f16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(x), "r"(0));
  return sum;
}

template <bool kBf16, bool kPair>
__device__ void fix_role(const Cta& c) {
  using S = Shape<kPair>;
  const PagedAttendParams& p = c.p;
  const int lane = threadIdx.x & 31;
  constexpr uint32_t kTop = kBf16 ? 0x7f807f80u : 0x7c007c00u;  // exponents of all ones
  Reader reader{c};
  int pos = 0, count = 0;
  while (const Piece* x = reader.next()) {
    uint32_t& found = c.m->found[reader.at % kRing];
    uint32_t(*poison)[4] = c.m->poison[reader.at % kRing];
    if (lane < 4 * kDiagTiles) poison[lane >> 2][lane & 3] = 0;
    if (lane == 0) found = 0;
    __syncwarp();
    const int tiles = max(x->tiles[0], x->tiles[1]), tile0 = x->tile0, length = x->length;
    const int whole = limit_of(p, x->pos0, length);  // slots that all rows see
    bool ok = true;
    auto pass = [&](int at) {  // a stage is not free before this warp is past it
      if (lane == 0) mbar_arrive(smem_u32(&c.m->empty[at % S::kStages]));
    };
    for (int j = 0; j < tiles; ++j, ++count) {
      // (of every tile, or the phase of a later one could be taken for it)
      if (!(ok = c.wait_warp(c.m->full[count % kRing], (count / kRing) & 1))) break;
      if (j == 0) pass(pos++);             // the first K
      if (j + 1 < tiles) pass(pos++);      // the next K
      const int st = pos++ % S::kStages;
      const int base = (tile0 + j) * kTile;
      if (base + kTile > whole) {
        char* v = reinterpret_cast<char*>(c.m) - kOperandBytes + (S::kQTiles + st) * kTileBytes2;
        const int diag = tile0 + j - whole / kTile;
        // 16 pieces of 16 bytes a slot
        for (int i = max(whole - base, 0) & ~7; i < kTile; i += 8) {
          uint4* at = reinterpret_cast<uint4*>(v + ((lane >> 3) & 1) * kHalf + (i + (lane >> 4)) * 128) + (lane & 7);
          const int slot = base + i + (lane >> 4);
          uint32_t sum = 0;
          if (base + i < length) {
            uint4 w[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) w[u] = at[16 * u];
#pragma unroll
            for (int u = 0; u < 4; ++u)
              if (slot + 2 * u < length)
                sum = add_zeros<kBf16>(w[u].x, add_zeros<kBf16>(w[u].y, add_zeros<kBf16>(w[u].z, add_zeros<kBf16>(w[u].w, sum))));
          }
#pragma unroll
          for (int u = 0; u < 4; ++u)
            if (slot + 2 * u >= length) at[16 * u] = make_uint4(0, 0, 0, 0);
          if ((sum & 0x7fff7fffu) == 0) continue;
#pragma unroll 1
          for (int u = 0; u < 4; ++u) {
            const int s = slot + 2 * u;
            if (s >= length || s < whole) continue;
            bool any = false;
            uint32_t* word = reinterpret_cast<uint32_t*>(at + 16 * u);
#pragma unroll 1
            for (int k = 0; k < 4; ++k) {
              uint32_t y = word[k];
              if ((y & kTop & 0xffffu) == (kTop & 0xffffu)) y &= 0xffff0000u, any = true;
              if ((y & kTop & 0xffff0000u) == (kTop & 0xffff0000u)) y &= 0xffffu, any = true;
              word[k] = y;
            }
            if (any && diag < kDiagTiles) {
              atomicOr(&poison[diag][(s - base) >> 5], 1u << ((s - base) & 31));
              found = 1;
            }
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&c.m->vready[count % kRing]));
      }
      pass(st);
    }
    if (!ok) return;
    reader.done();
  }
}

// ---------------------------------------------------------------- softmax
// 32 channels of a row's output, over the sum of its exponentials (`up`: up_of()).
// `none`: the row sees no slot.  (One that does may have a sum of 0 or NaN, and gives
// NaN.)
template <bool kBf16, int kN>
__device__ __forceinline__ void write_channels(const PagedAttendParams& p, uint16_t* to, bool none, float l, float up,
                                               const uint32_t (&o)[kN]) {
  const float inv = up / l;
#pragma unroll
  for (int i = 0; i < kN / 16; ++i) {
    uint32_t w[8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      w[k] = none ? 0u
                  : pack<kBf16>(__uint_as_float(o[16 * i + 2 * k]) * inv, __uint_as_float(o[16 * i + 2 * k + 1]) * inv);
    // (32 bytes at a time where rows are aligned to that: a warp's rows are far
    // apart, and each of its stores takes as many steps as it has rows)
    if (p.wide_rows) {
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to + 16 * i), "r"(w[0]), "r"(w[1]),
                   "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                   : "memory");
    } else {
      reinterpret_cast<uint4*>(to)[2 * i] = make_uint4(w[0], w[1], w[2], w[3]);
      reinterpret_cast<uint4*>(to)[2 * i + 1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
  }
}
// A row's log-sum-exp, of base-2 reference `ref` and sum `l`.
__device__ __forceinline__ void write_lse(const PagedAttendParams& p, long long row, int head, float ref, float l) {
  if (p.lse)
    p.lse[static_cast<long long>(head) * p.rows + row] = l == 0.f ? -INFINITY : (ref + log2f(l)) * 0.6931471805599453f;
}

// The results of an item's pieces for this warp's rows, joined: the weights of the
// pieces are 2^(their reference - the largest), over the sum.  kPair: rows by
// lanes, as they were computed; four channels of consecutive rows are side by side
// (rows by the warp, in order, as below: a split item of 256 rows took 35 us more).
// 32 channels of four pieces at a time are under way.
template <bool kBf16>
__device__ __forceinline__ void join_rows(const PagedAttendParams& p, const Piece& x, int tile, int row, int token,
                                          int head, bool valid) {
  const int pieces = x.pieces[tile];
  auto read = [&](int k) {
    return k < pieces ? __ldcg(p.part_ml + x.slot_of(k) * p.part_rows + row) : make_float2(0.f, 0.f);
  };
  // (equal infinities: 1, so that they and NaN go on into the sum)
  auto weight = [](float2 ml, float top) { return ml.y == 0.f ? 0.f : ml.x == top ? 1.f : exp2f(ml.x - top); };
  float top = -INFINITY, sum = 0.f;
#pragma unroll 1
  for (int k0 = 0; k0 < pieces; k0 += 4) {
    float2 ml[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) ml[u] = read(k0 + u);
    // (the largest so far may grow: the sum follows)
    float now = top;
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (ml[u].y != 0.f) now = fmaxf(now, ml[u].x);
    sum *= now == top ? 1.f : exp2f(top - now);
    top = now;
#pragma unroll
    for (int u = 0; u < 4; ++u) sum += ml[u].y == 0.f ? 0.f : ml[u].y * weight(ml[u], top);
  }
  uint16_t* to = p.out + (x.row0 + token) * p.o_token + head * p.o_head;
  const bool none = limit_of(p, x.pos0 + token, x.length) == 0;
  // 32 channels, two pieces at a time (four, or the next on their way meanwhile: registers
  // spill, or code that runs once is longer; both slower)
  const float4* rows = reinterpret_cast<const float4*>(p.part_o) + row;
#pragma unroll 1
  for (int part = 0; part < 4; ++part) {
    uint32_t o[32] = {};
#pragma unroll 1
    for (int k0 = 0; k0 < pieces; k0 += 2) {
      float2 ml[2];
      float4 v[2][8];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        ml[u] = read(k0 + u);
        const float4* from = rows + (x.slot_of(min(k0 + u, pieces - 1)) * 32 + 8 * part) * p.part_rows;
#pragma unroll
        for (int c = 0; c < 8; ++c) v[u][c] = __ldcg(from + c * p.part_rows);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float w = weight(ml[u], top);
        if (k0 + u < pieces)  // (a weight of 0 too: times what is not finite it is not 0)
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            o[4 * c] = __float_as_uint(fmaf(w, v[u][c].x, __uint_as_float(o[4 * c])));
            o[4 * c + 1] = __float_as_uint(fmaf(w, v[u][c].y, __uint_as_float(o[4 * c + 1])));
            o[4 * c + 2] = __float_as_uint(fmaf(w, v[u][c].z, __uint_as_float(o[4 * c + 2])));
            o[4 * c + 3] = __float_as_uint(fmaf(w, v[u][c].w, __uint_as_float(o[4 * c + 3])));
          }
      }
    }
    if (valid) write_channels<kBf16>(p, to + 32 * part, none, sum, up_of<kBf16>(x.length), o);
  }
  if (valid) write_lse(p, x.row0 + token, head, top, sum);
}

// Counts a piece of an item (whose results this warp has written, or seen written);
// true for the last one, which finds the others' in memory.
__device__ __forceinline__ bool take_ticket(int* ticket, int pieces) {
  int before = 0;
  if ((threadIdx.x & 31) == 0) before = atomicAdd(ticket, 1);
  before = __shfl_sync(0xffffffffu, before, 0);
  if (before != pieces - 1) return false;
  __threadfence();
  if ((threadIdx.x & 31) == 0) *ticket = 0;
  return true;
}

// Single: rows first, first + 4, .. of few, of many pieces: a row by the warp.  (This
// runs once, from instructions that no cache holds: unrolled over four rows it
// took 15500 cycles, of which memory's answers are some 3000.)
template <bool kBf16>
__device__ __forceinline__ void join(const PagedAttendParams& p, const Piece& x, int first, int rows) {
  const int lane = threadIdx.x & 31, pieces = x.pieces[0];
#pragma unroll 1
  for (int row = first; row < rows; row += 4) {
    auto read = [&](int k) {
      return k < pieces ? __ldcg(p.part_ml + x.slot_of(k) * p.part_rows + row) : make_float2(0.f, 0.f);
    };
    float top = -INFINITY, sum = 0.f;
#pragma unroll 1
    for (int k0 = 0; k0 < pieces; k0 += 32) {
      const float2 ml = read(k0 + lane);
      if (ml.y != 0.f) top = fmaxf(top, ml.x);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int k0 = 0; k0 < pieces; k0 += 32) {
      const float2 ml = read(k0 + lane);
      const float w = ml.y == 0.f ? 0.f : ml.x == top ? 1.f : exp2f(ml.x - top);  // (as in join_rows)
      float l = ml.y == 0.f ? 0.f : ml.y * w;
#pragma unroll
      for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
      sum += l;
      const int count = min(32, pieces - k0);
#pragma unroll 1
      for (int k = 0; k < count; k += 8) {
        float4 v[8];
        float f[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          f[u] = __shfl_sync(0xffffffffu, w, (k + u) & 31);
          v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (k + u < count)  // (whatever its weight, as in join_rows)
            v[u] = __ldcg(reinterpret_cast<const float4*>(p.part_o) + (x.slot_of(k0 + k + u) * p.part_rows + row) * 32 + lane);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          acc.x = fmaf(f[u], v[u].x, acc.x);
          acc.y = fmaf(f[u], v[u].y, acc.y);
          acc.z = fmaf(f[u], v[u].z, acc.z);
          acc.w = fmaf(f[u], v[u].w, acc.w);
        }
      }
    }
    const int token = row / p.group, head = x.head * p.group + row - token * p.group;
    const bool none = limit_of(p, x.pos0 + token, x.length) == 0;
    const float inv = up_of<kBf16>(x.length) / sum;
    const long long row_at = x.row0 + token;
    reinterpret_cast<uint2*>(p.out + row_at * p.o_token + head * p.o_head)[lane] =
        none ? make_uint2(0u, 0u)
             : make_uint2(pack<kBf16>(acc.x * inv, acc.y * inv), pack<kBf16>(acc.z * inv, acc.w * inv));
    if (p.lse && lane == 0)
      p.lse[static_cast<long long>(head) * p.rows + row_at] =
          sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
  }
}

// A lane's row of a piece.
struct Row {
  int in_tile, token, head, limit;  // row of the tile; token of the item; query head; slots that it sees
  bool valid;
  unsigned rows;                    // of the warp that are
  __device__ __forceinline__ Row(const PagedAttendParams& p, const Piece& x, int tile, int warp, int lane) {
    in_tile = warp * 32 + lane;
    const int at = in_tile / p.group;
    token = tile * p.tile_tokens + at;
    head = x.head * p.group + in_tile - at * p.group;
    valid = at < p.tile_tokens && token < x.tokens;
    limit = valid ? limit_of(p, x.pos0 + token, x.length) : 0x7fffffff;
    rows = __ballot_sync(0xffffffffu, valid);
  }
};

// The output of a piece's rows (of reference `ref` and sum `l`), from tensor memory
// to where it goes.
template <bool kBf16, bool kPair>
__device__ __forceinline__ void finish(const Cta& c, Reader& reader, const Piece& x, int tile, uint32_t o_addr,
                                       uint64_t& oempty, const Row& row, float ref, float l) {
  const PagedAttendParams& p = c.p;
  const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) & 3;
  const Piece y = x;
  const bool all = y.pieces[tile] == 1;
  const int at = tile * kTile + row.in_tile;
  uint16_t* to = p.out + (y.row0 + row.token) * p.o_token + row.head * p.o_head;
  float4* part_o = reinterpret_cast<float4*>(p.part_o) + static_cast<long long>(y.slot) * p.part_rows * 32 +
                   (kPair ? at : at * 32);
  const int step = kPair ? p.part_rows : 1;
  const bool found = c.m->found[reader.at % kRing] != 0;
  tc_fence_after();
  // (32 channels at a time: this runs once a piece, from instructions that no cache
  // holds; all at once took 5000 cycles)
#pragma unroll 1
  for (int part = 0; part < 4; ++part) {
    uint32_t o[32];
    tmem_load32_async(o_addr + 32 * part, o);
    tmem_wait_ld(o);
    if (found) {
      const int whole = limit_of(p, y.pos0, y.length);
#pragma unroll 1
      for (int d = 0; d < 4 * kDiagTiles; ++d)
        for (uint32_t bits = c.m->poison[reader.at % kRing][d / 4][d % 4]; bits; bits &= bits - 1) {
          const int slot = whole / kTile * kTile + 32 * d + __ffs(bits) - 1;
          if (slot >= row.limit || !row.valid) continue;
          const int page = p.c.table[y.seq * p.c.table_stride + (slot >> p.c.page_shift)];
          if (page < 0 || page >= p.c.num_pages) continue;
          const uint16_t* v = p.c.pages[1] + page * p.c.page_stride +
                              (slot & ((1 << p.c.page_shift) - 1)) * p.c.slot_stride + y.head * p.c.head_stride +
                              32 * part;
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const float f = value<kBf16>(v[i]);
            if (!(fabsf(f) < INFINITY)) o[i] = __float_as_uint(__uint_as_float(o[i]) + f);
          }
        }
    }
    if (row.valid) {
      if (all) {
        write_channels<kBf16>(p, to + 32 * part, row.limit == 0, l, up_of<kBf16>(y.length), o);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          part_o[(8 * part + i) * step] = make_float4(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1]),
                                                      __uint_as_float(o[4 * i + 2]), __uint_as_float(o[4 * i + 3]));
      }
    }
  }
  tc_fence_before();
  __syncwarp();
  if (lane == 0) mbar_arrive(smem_u32(&oempty));
  reader.done();
  if (all) {
    if (row.valid) write_lse(p, y.row0 + row.token, row.head, ref, l);
    return;
  }
  if (kPair && !row.rows) return;
  if (row.valid) p.part_ml[static_cast<long long>(y.slot) * p.part_rows + at] = make_float2(ref, l);
  __threadfence();
  __syncwarp();
  if (kPair && take_ticket(p.tickets + (y.base * 2 + tile) * 4 + warp, y.pieces[tile]))
    join_rows<kBf16>(p, y, tile, at, row.token, row.head, row.valid);
}

// Whether a row's reference is so far from zero that logits are taken relative to it.
__device__ __forceinline__ bool far_off(float m, float scale) {
  return m > -INFINITY && fabsf(m * scale) > kFar;
}

template <bool kBf16, bool kPair>
__device__ void softmax_role(const Cta& c, uint32_t tmem, int tile) {
  const PagedAttendParams& p = c.p;
  const int warp = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31, r = warp * 32 + lane;
  const uint32_t lanes = tmem + (static_cast<uint32_t>(warp * 32) << 16);
  const float scale = p.scale_log2;
  const uint64_t scale2 = pair_of(scale, scale);
  Reader reader{c};
  int count = 0, o_count = 0;  // tiles and pieces done
  while (const Piece* x = reader.next()) {
    const int n = x->tiles[tile];
    if (n == 0) {
      reader.done();
      continue;
    }
    const Row row(p, *x, tile, warp, lane);
    const int tile0 = x->tile0, limit = row.limit, least = __reduce_min_sync(0xffffffffu, limit);
    // (single: two outputs in turns)
    const uint32_t o_addr = lanes + (2 + (kPair ? tile : reader.at & 1)) * kTile;
    const float down = down_of<kBf16>(x->length), up = up_of<kBf16>(x->length);
    float m = -INFINITY, l = 0.f;
    bool far = false;  // (not for rows that are none, which may hold anything)
    for (int j = 0; j < n; ++j, ++count) {
      const int buffer = kPair ? tile : count & 1;
      if (!c.wait_here(c.m->sfull[buffer], (kPair ? count : count >> 1) & 1)) return;
      const uint32_t s_addr = lanes + buffer * kTile;
      if (row.rows) {
        tc_fence_after();
        uint32_t s[4][32];
#pragma unroll
        for (int k = 0; k < 4; ++k) tmem_load32_async(s_addr + 32 * k, s[k]);
        tmem_wait_ld(s[0]);
#pragma unroll
        for (int k = 1; k < 4; ++k) tmem_order_after_wait(s[k]);
        const int base = (tile0 + j) * kTile;
        if (base + kTile > least) {
          const int see = limit - base;
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (32 * k + i >= see) s[k][i] = 0xff800000u;
        }
        // The first 32 probabilities are made with the old reference while the
        // largest logit is found, and again in the few cases where that has grown.
        uint64_t sum[4] = {};
        auto exponentials = [&](int k, uint32_t (&w)[16], float ref) {
          const uint64_t ref2 = pair_of(ref, ref);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float2 e = split_of(
                fma2(pair_of(__uint_as_float(s[k][2 * i]), __uint_as_float(s[k][2 * i + 1])), scale2, ref2));
            const float a = ex2_approx(e.x), b = ex2_approx(e.y);
            sum[i & 3] = add2(sum[i & 3], pair_of(a, b));
            w[i] = pack<kBf16>(a, b);
          }
        };
        uint32_t w[16];
        auto reference = [&] { return -((m == -INFINITY ? 0.f : m * scale) + down); };
        float ref = reference();
        exponentials(0, w, ref);
        float top[4] = {m, m, m, m};
#pragma unroll
        for (int i = 0; i < 32; i += 2)
#pragma unroll
          for (int k = 0; k < 4; ++k) top[k] = max3(top[k], __uint_as_float(s[k][i]), __uint_as_float(s[k][i + 1]));
        const float now = fmaxf(max3(top[0], top[1], top[2]), top[3]);
        if (!kPair && j > 0 && !c.wait_here(c.m->odone[0], (count - 1) & 1)) return;
        const bool grown = now > m && (m == -INFINITY || (now - m) * scale > kGrowth);
        if (__any_sync(0xffffffffu, grown || far)) {
          const float f = grown ? ex2_approx((m - now) * scale) : 1.f;
          if (grown) m = now;
          far = row.valid && far_off(m, scale);
          l *= f;
          if (j > 0) {
            tc_fence_after();
            const uint64_t f2 = pair_of(f, f);
#pragma unroll 1
            for (int k = 0; k < 8; ++k) {
              uint32_t o[16];
              tmem_load16(o_addr + 16 * k, o);
#pragma unroll
              for (int i = 0; i < 16; i += 2) {
                const float2 y = split_of(mul2(pair_of(__uint_as_float(o[i]), __uint_as_float(o[i + 1])), f2));
                o[i] = __float_as_uint(y.x);
                o[i + 1] = __float_as_uint(y.y);
              }
              tmem_store16(o_addr + 16 * k, o);
            }
          }
          ref = far ? -down : reference();
          // c z - c m with c m rounded is off by half of fp32's step in c m, the same for all
          // of a row: nothing, until it takes p out of its type's range.  Far from zero p
          // is made from z - m.
          if (__any_sync(0xffffffffu, far)) {
            const float by = far ? m : 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
              for (int i = 0; i < 32; ++i) s[k][i] = __float_as_uint(__uint_as_float(s[k][i]) - by);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[i] = 0;
          exponentials(0, w, ref);
        }
        tmem_store16(s_addr, w);
#pragma unroll
        for (int k = 1; k < 4; ++k) {
          exponentials(k, w, ref);
          tmem_store16(s_addr + 16 * k, w);
          if (k == 1) {  // the product with the first half of the slots can begin
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&c.m->pready[buffer][0]));
          }
        }
        const float2 total = split_of(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])));
        l += (total.x + total.y) * up;
        tmem_wait_st();
        tc_fence_before();
      } else {
        if (!kPair && j > 0 && !c.wait_here(c.m->odone[0], (count - 1) & 1)) return;
        if (lane == 0) mbar_arrive(smem_u32(&c.m->pready[buffer][0]));
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&c.m->pready[buffer][1]));
    }
    // (the reference as it entered, rounded beside `down`)
    const float ref = far ? m * scale : ((m == -INFINITY ? 0.f : m * scale) + down) - down;
    if (kPair) {
      if (!c.wait_here(c.m->odone[tile], o_count++ & 1)) return;
      finish<kBf16, true>(c, reader, *x, tile, o_addr, c.m->oempty[tile], row, ref, l);
    } else {  // the other warps take it from here
      const int o = reader.at & 1;
      if (!c.wait_here(c.m->oempty[o], ((reader.at >> 1) & 1) ^ 1)) return;  // (they have read the one before)
      c.m->sums[o][r] = make_float2(ref, l);
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&c.m->sready[o]));
      reader.done();
    }
  }
}

// Single: the pieces' outputs, while the softmax goes on with the next piece.
template <bool kBf16>
__device__ void output_role(const Cta& c, uint32_t tmem) {
  const int warp = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31;
  uint32_t stored = 0;
  Reader reader{c};
  while (const Piece* x = reader.next()) {
    const int o = reader.at & 1, phase = (reader.at >> 1) & 1;
    const Row row(c.p, *x, 0, warp, lane);
    if (!c.wait_here(c.m->sready[o], phase) || !c.wait_here(c.m->oready[o], phase)) return;
    const float2 sums = c.m->sums[o][warp * 32 + lane];
    const Piece y = *x;
    finish<kBf16, false>(c, reader, *x, 0, tmem + (static_cast<uint32_t>(warp * 32) << 16) + (2 + o) * kTile,
                         c.m->oempty[o], row, sums.x, sums.y);
    if (y.pieces[0] > 1) {  // each warp counts the CTA's rows, and joins some of them
      if (lane == 0) mbar_arrive(smem_u32(&c.m->stored));
      if (!c.wait_here(c.m->stored, stored)) return;
      stored ^= 1;
      __threadfence();
      if (take_ticket(c.p.tickets + y.base * 8 + warp, y.pieces[0])) join<kBf16>(c.p, y, warp, y.tokens * c.p.group);
    }
  }
}

template <bool kBf16, bool kPair>
__global__ void __launch_bounds__(kThreads, 1) paged_attend_kernel(const __grid_constant__ PagedAttendParams p) {
  using S = Shape<kPair>;
  extern __shared__ __align__(1024) unsigned char smem[];
  Misc* m = reinterpret_cast<Misc*>(smem + kOperandBytes);
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const Cta c{p, m, smem_u32(smem)};
  // The warp that moves tiles sets the barriers up and goes on; the others wait for
  // them, and for tensor memory.
  constexpr int kReady = 1;  // named barrier
  if (warp == kLoadWarp) {
    if (lane == 0) {
      for (int i = 0; i < S::kStages; ++i) mbar_init(smem_u32(&m->empty[i]), 1 + S::kQTiles);
#pragma unroll 1
      for (int i = 0; i < 2; ++i) {
        mbar_init(smem_u32(&m->sfull[i]), 1);
        mbar_init(smem_u32(&m->pready[i][0]), 4);
        mbar_init(smem_u32(&m->pready[i][1]), 4);
        mbar_init(smem_u32(&m->odone[i]), 1);
        mbar_init(smem_u32(&m->oempty[i]), 4);
        mbar_init(smem_u32(&m->sready[i]), 4);
        mbar_init(smem_u32(&m->oready[i]), 1);
        mbar_init(smem_u32(&m->drain[i]), 1);
        mbar_init(smem_u32(&m->turn[i]), 1);
      }
#pragma unroll 1
      for (int i = 0; i < kRing; ++i) {
        mbar_init(smem_u32(&m->qfull[i]), 1);
        mbar_init(smem_u32(&m->qempty[i]), 1);
        mbar_init(smem_u32(&m->kfull[i]), 1);
        mbar_init(smem_u32(&m->full[i]), 1);
        mbar_init(smem_u32(&m->vready[i]), 1);
        mbar_init(smem_u32(&m->pfull[i]), 1);
        mbar_init(smem_u32(&m->pempty[i]), S::kConsumers);
      }
      mbar_init(smem_u32(&m->stored), 4);
      m->abort = 0;
      fence_mbar_init();
    }
    __syncwarp();
    asm volatile("bar.arrive %0, %1;" ::"n"(kReady), "n"(kThreads) : "memory");
  } else {
    if (warp == kMmaWarp) {
      tmem_alloc(smem_u32(&m->tmem), 512);
      tmem_relinquish();
      tc_fence_before();
    }
    named_bar_sync(kReady, kThreads);
    tc_fence_after();
  }
  pdl_wait();
  const uint32_t tmem = warp == kLoadWarp ? 0 : m->tmem;
  if (warp >= kSoftWarp && warp < kSoftWarp + 8) {
    // registers for the softmax, which holds a row of logits: of the launch's 384 x
    // 168 kPair 256 x 200 and 128 x 104 (finding pieces spills with 88: 3 % of a
    // prompt), single 256 x 208 and 128 x 88
    if constexpr (kPair)
      asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    else
      asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    if (kPair || warp < kSoftWarp + 4)
      softmax_role<kBf16, kPair>(c, tmem, (warp - kSoftWarp) / 4);
    else
      output_role<kBf16>(c, tmem);
  } else {
    if constexpr (kPair)
      asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    else
      asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == kLoadWarp)
      load_role<kPair>(c);
    else if (warp == kFixWarp)
      fix_role<kBf16, kPair>(c);
    else if ((kPair || warp == kMmaWarp) && elect_one())
      product_role<kBf16, kPair>(c, tmem, warp != kMmaWarp);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
  if (kPair && threadIdx.x == 0 && atomicAdd(p.done, 1) == static_cast<int>(gridDim.x) - 1) {
    *p.next = 0;  // every CTA has taken its last ticket
    *p.done = 0;
  }
}

template <bool kBf16, bool kPair>
cudaError_t set_limit() {
  return cudaFuncSetAttribute(paged_attend_kernel<kBf16, kPair>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              kSmemBytes);
}

}  // namespace

cudaError_t paged_attend_set_smem_limit() {
  cudaError_t e = set_limit<true, true>();
  if (e == cudaSuccess) e = set_limit<true, false>();
  if (e == cudaSuccess) e = set_limit<false, true>();
  if (e == cudaSuccess) e = set_limit<false, false>();
  return e;
}

cudaError_t launch_paged_attend(const PagedAttendParams& p, int ctas, cudaStream_t stream) {
  const dim3 grid(static_cast<unsigned>(ctas));
  if (p.pair)
    return p.is_bf16 ? launch_dependent(paged_attend_kernel<true, true>, grid, kThreads, kSmemBytes, stream, p)
                     : launch_dependent(paged_attend_kernel<false, true>, grid, kThreads, kSmemBytes, stream, p);
  return p.is_bf16 ? launch_dependent(paged_attend_kernel<true, false>, grid, kThreads, kSmemBytes, stream, p)
                   : launch_dependent(paged_attend_kernel<false, false>, grid, kThreads, kSmemBytes, stream, p);
}

}  // namespace ckv
