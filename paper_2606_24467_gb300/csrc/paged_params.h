// Parameter blocks of the rotary and paged-cache kernels, shared by their host
// side and the kernels.  They travel by value like the others (ckv_params.h).
#pragma once

#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>

#include "ckv_params.h"

namespace ckv {

constexpr int kRopePairs = kHeadDim / 2;

struct RopeTable {
  unsigned long long turns[kRopePairs];  // turns a position, in units of 2^-64
  float scale;
  int pairs;                             // rotated; 0: rows are copied
  int interleaved;
};

// The cache as the kernels see it; strides in elements.
struct PagedCache {
  uint16_t* pages[2];          // K, V
  const int32_t* table;
  int32_t* lengths;
  long long page_stride, slot_stride, head_stride, table_stride;
  int batch, num_kv_heads, num_pages, table_width;
  int page_shift;              // log2 of a page's slots
  int capacity;                // slots that a table row holds
};

// Rows of heads from and to; strides in elements.
struct RowSet {
  const uint16_t* in;
  uint16_t* out;
  long long in_token, in_head, out_token, out_head;
};

// Rotary rows, and rows into a paged cache.  A row's heads are num_q query
// heads, then num_k key heads, then (paged) as many value heads.
struct RopeParams {
  RopeTable rope;
  RowSet q, k, v;              // paged: k and v have no `out`
  const int32_t* positions;    // [rows]; null (paged): the slots
  const int32_t* start;        // paged: first slot of each sequence; null: its length
  int* status;                 // may be null
  PagedCache c;
  int rows, num_q, num_k, is_bf16, backward, paged;
  int rows_per_seq;            // negative: by cu_rows
  int cu_rows[kMaxBatch + 1];
};

struct PagedGatherParams {
  PagedCache c;
  uint16_t* out[2];            // K, V; either may be null
  const int32_t* start;
  int* status;
  int rows, rows_per_seq;
  int cu_rows[kMaxBatch + 1];
};

cudaError_t launch_rope(const RopeParams& p, cudaStream_t s);
cudaError_t launch_paged_append(const RopeParams& p, int most_rows, cudaStream_t s);
cudaError_t launch_paged_gather(const PagedGatherParams& p, cudaStream_t s);

constexpr int kPagedTile = 128;  // slots of a K or V tile, and rows of a tile of queries
constexpr int kPagedMaxCtas = 160;
// Chunks.  All work is a line, an item (two tiles of rows of a KV head) after another;
// each takes its tiles and kPagedPiece, what its beginning and end cost.  Where that is
// less than kPagedFew of the longest items an SM, the line is cut into equal runs, one an
// SM: 501 tokens after 9000 to 16000 take 147 us so, 170 with items whole but for the
// last; 777 after 3000 to 20000, four times, 480 and 580.  Else items are whole and taken
// in turn, as CTAs that run together then read the same tiles, but for the last ones, in
// kPagedRuns runs an SM: 4096 tokens after 128K take 4980 us so, 5840 all in runs; eight
// times 2000 from the first on 270 and 350; 8191 once 365 and 373.  (Each side by side on
// one GPU, L2 flushed; from one GPU to another these times differ by 5 %.)
// No piece has fewer than kPagedLeast tiles of an item that has more (16: 160 us for the
// first), no run less than kPagedShare of the line.  The results of at most kPagedSlots
// pieces, two a run, wait to be joined.
constexpr int kPagedFew = 2;
constexpr int kPagedPiece = 4;
constexpr int kPagedLeast = 4;
constexpr int kPagedShare = 12;
constexpr int kPagedRuns = 2;
constexpr int kPagedSlots = 608;
static_assert(kPagedShare > kPagedPiece + kPagedLeast, "a run has a piece");
// Workspace header: status word, the word that says that a call has stopped, the
// next ticket and the CTAs done; behind it the counters of items in pieces, one
// for each 32 rows.  Every call leaves them zero.
constexpr int kPagedTickets = 256;  // bytes
constexpr int kPagedHeaderBytes = kPagedTickets + kPagedSlots * 8 * 4 + 256 - (kPagedSlots * 32) % 256;
static_assert(kPagedHeaderBytes % 256 == 0 && kPagedMaxCtas <= kPagedSlots, "header");

struct PagedAttendParams {
  CUtensorMap map_q;           // [rows][heads][128]: boxes of a KV group's heads, some tokens, 64 channels
  CUtensorMap map_k, map_v;    // [pages][slots][heads][128]: boxes of up to 128 slots, 64 channels
  PagedCache c;
  uint16_t* out;
  float* lse;                  // optional, [num_q_heads][rows]
  const int32_t* start;        // optional, [batch]
  long long o_token, o_head;
  float scale_log2;
  int rows, group, causal, is_bf16;
  int pair;                    // two tiles of rows to an item
  int wide_rows;               // rows of `out` are aligned to 32 bytes
  int tile_tokens;             // query tokens of 128 rows
  int item_tokens;             // of an item
  int q_box_bytes;             // of 64 channels of a tile
  int q_buffers;               // single: Q of 1, 2 or 4 pieces at a time
  // workspace
  int* status;
  int* stopped;
  int* next;
  int* done;
  int* tickets;
  float2* part_ml;             // [slots][part_rows]: base-2 reference and sum of a piece's rows,
  float* part_o;               //   [128]: and output
  int part_rows;
  unsigned long long stall_ns; // test hook: the CTA of the first piece waits this long for what nothing sets; 0: not
  int rows_per_seq;
  int cu_rows[kMaxBatch + 1];
};

cudaError_t paged_attend_set_smem_limit();
cudaError_t launch_paged_attend(const PagedAttendParams& p, int ctas, cudaStream_t s);

}  // namespace ckv
