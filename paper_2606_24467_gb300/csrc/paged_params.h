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

constexpr int kPagedTile = 128;          // slots of a K or V tile
constexpr int kPagedHeaderBytes = 1024;  // workspace: status word, the word that says that a call has stopped

struct PagedAttendParams {
  CUtensorMap map_q, map_k, map_v;
  PagedCache c;
  const uint16_t* q;
  uint16_t* out;
  float* lse;                  // optional, [num_q_heads][rows]
  const int32_t* start;        // optional, [batch]
  long long q_token, q_head, o_token, o_head;
  float scale_log2;
  int rows, num_q_heads, group, causal, is_bf16;
  int* status;
  int* stopped;
  int rows_per_seq;
  int cu_rows[kMaxBatch + 1];
};

cudaError_t launch_paged_attend(const PagedAttendParams& p, cudaStream_t s);

}  // namespace ckv
