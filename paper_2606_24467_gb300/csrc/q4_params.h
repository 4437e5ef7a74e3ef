// Parameter blocks of the 4-bit cache's kernels (append / gather, attention,
// eviction), shared by their host side and the kernels.  They travel by value
// like the others (ckv_params.h).
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "ckv_params.h"

namespace ckv {

constexpr int kQ4GroupDim = 32;                         // channels that share a scale
constexpr int kQ4Groups = kHeadDim / kQ4GroupDim;       // 4
constexpr int kQ4CodeBytes = kHeadDim / 2;              // codes of one K or V row
constexpr int kQ4ParamBytes = 4 * kQ4Groups;            // 4 bf16 scales, 4 bf16 minima
constexpr int kQ4SlotStep = 32;                         // capacity is a multiple of this
constexpr int kQ4MaxUnits = 65535;                      // (sequence, KV group) pairs of a cache
constexpr int kQ4MaxQueries = 16;                       // query tokens a sequence and call
constexpr int kQ4MaxCtas = 160;                         // of the attention
constexpr int kQ4HeaderBytes = 1024;                    // workspace: status word, tickets

// The cache as the kernels see it; unit u = sequence * num_kv_heads + group,
// slot row = u * capacity + slot.
struct Q4Cache {
  uint8_t* codes[2];     // K, V: [units][capacity][64]
  uint8_t* params[2];    // K, V: [units][capacity][16]
  int32_t* positions;    // [units][capacity]
  float* weights;        // [units][capacity], or null
  int32_t* lengths;      // [units]
  int capacity, num_kv_heads, batch;
};

// Rows into the cache.  Table: per sequence [batch + 1] first rows, or per
// unit (group-major: [num_kv_heads][batch + 1]) where a unit has its own rows.
template <int kTable>
struct Q4WriteParams {
  Q4Cache c;
  const uint16_t* src[2];      // K, V rows (f16 / bf16 bits)
  uint16_t* values[2];         // optional: the values that the codes stand for
  long long tok_stride, head_stride;          // of src, elements
  const int32_t* positions;    // append: [rows]
  const int32_t* start;        // append: first slot of each unit, or null (lengths)
  const int32_t* indices;      // gather: [num_kv_heads][rows] (or [rows], group-major)
  const float* raw;            // gather: optional raw scores, score layout
  int* status;                 // may be null
  int is_bf16, rows, rows_per_seq;            // append: rows_per_seq < 0: by the table
  int group_major, window, p_total;
  int cu_seqlens[kTable ? kMaxBatch + 1 : 1]; // gather: first source row of each sequence
  int cu_prefix[kTable ? kMaxBatch + 1 : 1];
  int cu_rows[kTable ? kTable : kMaxBatch + 1];
};
constexpr int kQ4SeqTable = kMaxBatch + 1;
constexpr int kQ4UnitTable = kMaxBudgetUnits + kMaxKvHeads;
using Q4AppendParams = Q4WriteParams<0>;
using Q4GatherParams = Q4WriteParams<kQ4SeqTable>;
using Q4GatherUnitParams = Q4WriteParams<kQ4UnitTable>;

constexpr int kQ4Tile = 64;  // attention: slots of a tile,
constexpr int kQ4Warps = 8;  // warps of a CTA (there is one an SM),
// query rows of a row block.  16 rows share the work on their codes, but leave
// fewer tiles to a warp and take every register: 16 rows a unit (bf16) take 37.5
// us in blocks of 16 and 32.6 in blocks of 8 at 64 units of 1000 to 8000 slots,
// at four of 777 14.7 and 10.4, but 16 rows of 32 units of 128K slots 205 and 254,
// 20 of 512 units of 1000 to 8000 (with weights) 327 and 374.  `slots`: the
// capacity of all units, as the host does not know the lengths.
constexpr int q4_block_rows(int rows, long long slots) { return rows <= 8 || slots <= 1 << 20 ? 8 : 16; }

// Attention.  The tiles of all row blocks -- some query rows of a unit -- form one sequence, of which every CTA takes an equal run, and every
// warp of it a run of that; or, where they come out about even that way, each row
// block has CTAs of its own.
struct Q4AttendParams {
  CUtensorMap map_k, map_v;    // codes: [units * capacity] rows of 64 bytes, boxes of kQ4Tile rows
  Q4Cache c;
  const uint16_t* q;           // f16 / bf16 bits
  uint16_t* out;
  float* lse;                  // optional, [batch][num_q_heads][num_queries]
  const int32_t* q_positions;  // optional, [batch][num_queries]
  long long q_bs, q_hs, q_qs, o_bs, o_hs, o_qs;  // elements
  float scale_log2;            // softmax scale * log2(e)
  int num_q_heads, group, num_queries, is_bf16, accumulate;
  int rows, block_rows, blocks;  // query rows of a unit, of a row block, and row blocks of a unit
  int* status;
  // workspace
  int* stopped;                // 1 once a wait has run out, until the workspace is set up again
  int* tickets;                // [CTAs]: CTAs done with the row block that starts in one and goes on
  float* head_o;               // [warps]: the end of a row block that another warp began,
  float2* head_ml;             //   [block rows][128], and its softmax reference and sum
  float* cta_o;                // [CTAs][2]: likewise of row blocks from before, and going on
  float2* cta_ml;
  float* lse_ws;               // [units][rows]: base-2 log-sum-exp
  float* z;                    // accumulate: [units][capacity][z_stride] base-2 logits of the rows
  int z_stride;                // rows, made even
  unsigned long long stall_ns; // test hook: CTA 0's first warp waits this long for what nothing sets; 0: not
};

struct Q4EvictParams {
  Q4Cache c;
  const int32_t* budgets;      // optional, [units]
  int budget;                  // where `budgets` is null
  int sinks, recent;
  int cluster;                 // CTAs a unit (set at the launch)
  int32_t* lists;              // workspace: [units][capacity]: the holes, from capacity / 2 on the rows
  int* status;
};

// Launches a kernel that may be brought up while the one before it in the
// stream ends (its first act is then to wait for that one's results).  Only a
// kernel that another of the same call follows lets its successor start before
// its own end: whatever comes after a call finds its outputs complete.
template <class... A>
cudaError_t launch_dependent(void (*kernel)(A...), dim3 grid, int threads, size_t smem, cudaStream_t stream,
                             const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(static_cast<unsigned>(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

cudaError_t launch_q4_append(const Q4AppendParams& p, int max_rows, cudaStream_t s);
cudaError_t launch_q4_gather(const Q4GatherParams& p, cudaStream_t s);
cudaError_t launch_q4_gather(const Q4GatherUnitParams& p, cudaStream_t s);
cudaError_t q4_attend_set_smem_limit();
cudaError_t launch_q4_attend(const Q4AttendParams& p, int sms, cudaStream_t s);
cudaError_t launch_q4_weights(const Q4AttendParams& p, cudaStream_t s);
cudaError_t q4_evict_set_smem_limit();
cudaError_t launch_q4_evict(const Q4EvictParams& p, int sms, cudaStream_t s);

}  // namespace ckv
