// Host side of the rotary and paged-cache entry points (include/compresskv.h):
// argument checks, workspace and launches.  Nothing here allocates device
// memory or waits for a stream.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>

#include "compresskv.h"
#include "host_common.h"
#include "paged_params.h"

using namespace ckv;

namespace {

constexpr int kMaxPagedCapacity = 1 << 24;
constexpr float kMaxScale = 0x1p96f;
constexpr int64_t kMaxQueryRows = 1 << 26;  // query tokens times heads (items and pieces count in 32 bits)

// Test hook: how long the next attention stalls on purpose (0: not).
std::atomic<long long> g_stall_attend_ns{0};

// The attention's area behind the workspace header: results of pieces.  Where a
// tile holds all rows of a unit, each CTA has at most two units in part.
struct AttendArea {
  size_t ml = 0, o = 0, bytes = 0;
  int rows = 0;
};
AttendArea attend_area(long long rows) {
  AttendArea a;
  const bool pair = rows > kPagedTile;
  a.rows = pair ? 2 * kPagedTile : static_cast<int>(rows);
  const size_t all = static_cast<size_t>(pair ? kPagedSlots : 2 * kPagedMaxCtas) * a.rows;
  a.ml = kPagedHeaderBytes;
  a.o = a.ml + (all * sizeof(float2) + 255) / 256 * 256;
  a.bytes = a.o + all * kHeadDim * sizeof(float);
  return a;
}

bool dtype_ok(int dtype) { return dtype == CKV_DTYPE_F16 || dtype == CKV_DTYPE_BF16; }

bool strides_ok(int64_t token, int64_t head) {
  return token >= 0 && head >= 0 && token % 8 == 0 && head % 8 == 0 && std::max(token, head) <= kMaxStride;
}

// Whether [a, a + na) and [b, b + nb) share a byte.
bool share(const void* a, uint64_t na, const void* b, uint64_t nb) {
  const uint64_t x = reinterpret_cast<uint64_t>(a), y = reinterpret_cast<uint64_t>(b);
  return na && nb && x < y + nb && y < x + na;
}

// Elements from the first row's start to the last row's end.
uint64_t span_of(int rows, int heads, int64_t token, int64_t head) {
  return static_cast<uint64_t>(rows - 1) * token + static_cast<uint64_t>(heads - 1) * head + kHeadDim;
}

// Rows [rows][heads][128] from `in` to `out`, at least one of each.
int check_rows(int rows, int heads, const void* in, int64_t in_token, int64_t in_head, const void* out,
               int64_t out_token, int64_t out_head) {
  if (!in || !out || !aligned16(in) || !aligned16(out)) return CKV_ERR_INVALID_ARG;
  if (!strides_ok(in_token, in_head) || !strides_ok(out_token, out_head)) return CKV_ERR_INVALID_ARG;
  const int64_t strides[3] = {out_token, out_head, 0};
  const int dims[3] = {rows, heads, 1};
  if (rows_overlap(strides, dims)) return CKV_ERR_INVALID_ARG;
  const bool in_place = in == out && (rows == 1 || in_token == out_token) && (heads == 1 || in_head == out_head);
  if (!in_place && share(in, 2 * span_of(rows, heads, in_token, in_head), out,
                         2 * span_of(rows, heads, out_token, out_head)))
    return CKV_ERR_INVALID_ARG;
  return CKV_OK;
}

// Whether a row of one set of rows ([rows][heads][128]) shares an element with one of
// another.  (With token strides that differ: not told.)
bool rows_meet(int rows, const void* a, int heads_a, int64_t token_a, int64_t head_a, const void* b, int heads_b,
               int64_t token_b, int64_t head_b) {
  if (heads_a == 0 || heads_b == 0) return false;
  const int64_t span_a = static_cast<int64_t>(span_of(1, heads_a, 0, head_a));
  const int64_t span_b = static_cast<int64_t>(span_of(1, heads_b, 0, head_b));
  if (!share(a, 2 * span_of(rows, heads_a, token_a, head_a), b, 2 * span_of(rows, heads_b, token_b, head_b)))
    return false;
  if (rows > 1 && token_a != token_b) return false;
  const int64_t off = (static_cast<int64_t>(reinterpret_cast<uintptr_t>(b)) -
                       static_cast<int64_t>(reinterpret_cast<uintptr_t>(a))) / 2;
  const int64_t most = rows - 1, token = most ? token_a : 0;
  if (token > 0) {  // side by side within a token, as in a fused projection
    const int64_t at = (off % token + token) % token;
    if (at >= span_a && at + span_b <= token) return false;
  }
  // of two heads x apart: whether some tokens' rows meet
  auto near = [&](int64_t x) {
    const int64_t at = token ? -x / token : 0;
    for (int64_t d = at - 1; d <= at + 1; ++d) {
      const int64_t gap = x + std::min(std::max(d, -most), most) * token;
      if (gap < kHeadDim && gap > -kHeadDim) return true;
    }
    return false;
  };
  if (head_a == head_b) {
    for (int i = 1 - heads_a; i < heads_b; ++i)
      if (near(off + i * head_a)) return true;
    return false;
  }
  for (int i = 0; i < heads_a; ++i)
    for (int j = 0; j < heads_b; ++j)
      if (near(off + j * head_b - i * head_a)) return true;
  return false;
}

RowSet row_set(const void* in, int64_t in_token, int64_t in_head, void* out, int64_t out_token, int64_t out_head) {
  return {static_cast<const uint16_t*>(in), static_cast<uint16_t*>(out), in_token, in_head, out_token, out_head};
}

int check_rope(const ckv_rope* r) {
  if (!r || r->rot_dim < 2 || r->rot_dim > kHeadDim || r->rot_dim % 2 || !std::isfinite(r->scale))
    return CKV_ERR_INVALID_ARG;
  return CKV_OK;
}

RopeTable rope_table(const ckv_rope* r) {
  RopeTable t;
  std::memcpy(t.turns, r->turns, sizeof(t.turns));
  t.scale = r->scale;
  t.pairs = r->rot_dim / 2;
  t.interleaved = r->interleaved != 0;
  return t;
}

int check_cache(const ckv_paged_cache* c, bool pointers = true) {
  if (!c || c->batch < 1 || c->num_kv_heads < 1 || c->num_pages < 1 || c->table_width < 1 || !dtype_ok(c->dtype))
    return CKV_ERR_INVALID_ARG;
  if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1))) return CKV_ERR_INVALID_ARG;
  if (c->batch > kMaxBatch || c->head_dim != kHeadDim || c->num_kv_heads > kMaxKvHeads ||
      static_cast<int64_t>(c->table_width) * c->page_size > kMaxPagedCapacity)
    return CKV_ERR_UNSUPPORTED;
  if (!pointers) return CKV_OK;
  if (!c->k_pages || !c->v_pages || !c->table || !c->lengths || !aligned16(c->k_pages) || !aligned16(c->v_pages))
    return CKV_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(c->table) & 3u) || (reinterpret_cast<uintptr_t>(c->lengths) & 3u) ||
      c->table_stride < c->table_width)
    return CKV_ERR_INVALID_ARG;
  if (!strides_ok(c->page_stride, c->slot_stride) || !strides_ok(0, c->head_stride)) return CKV_ERR_INVALID_ARG;
  const int64_t strides[3] = {c->page_stride, c->slot_stride, c->head_stride};
  const int dims[3] = {c->num_pages, c->page_size, c->num_kv_heads};
  return rows_overlap(strides, dims) ? CKV_ERR_INVALID_ARG : CKV_OK;
}

PagedCache device_cache(const ckv_paged_cache* c) {
  PagedCache d;
  d.pages[0] = static_cast<uint16_t*>(c->k_pages);
  d.pages[1] = static_cast<uint16_t*>(c->v_pages);
  d.table = c->table;
  d.lengths = c->lengths;
  d.page_stride = c->page_stride;
  d.slot_stride = c->slot_stride;
  d.head_stride = c->head_stride;
  d.table_stride = c->table_stride;
  d.batch = c->batch;
  d.num_kv_heads = c->num_kv_heads;
  d.num_pages = c->num_pages;
  d.table_width = c->table_width;
  d.page_shift = 0;
  while ((1 << d.page_shift) < c->page_size) ++d.page_shift;
  d.capacity = c->table_width * c->page_size;
  return d;
}

// The rows of each sequence, into a parameter block.
int take_rows(const ckv_paged_cache* c, const int32_t* cu, int32_t rows_per_seq, int* to, int* per_seq, int* rows,
              int* most) {
  long long all = 0;
  *most = 0;
  if (cu) {
    if (cu[0] != 0) return CKV_ERR_INVALID_ARG;
    for (int s = 0; s < c->batch; ++s) {
      if (cu[s + 1] < cu[s]) return CKV_ERR_INVALID_ARG;
      *most = std::max(*most, cu[s + 1] - cu[s]);
    }
    std::copy(cu, cu + c->batch + 1, to);
    all = cu[c->batch];
    *per_seq = -1;
  } else {
    if (rows_per_seq < 0) return CKV_ERR_INVALID_ARG;
    *per_seq = *most = rows_per_seq;
    all = static_cast<long long>(rows_per_seq) * c->batch;
  }
  if (all > (1LL << 31) - 1) return CKV_ERR_UNSUPPORTED;
  *rows = static_cast<int>(all);
  return CKV_OK;
}

int check_index(const int32_t* ptr) { return reinterpret_cast<uintptr_t>(ptr) & 3u ? CKV_ERR_INVALID_ARG : CKV_OK; }

int check_workspace(const void* ws, size_t have, size_t need) {
  if (!ws || have < need || (reinterpret_cast<uintptr_t>(ws) & 255u)) return CKV_ERR_WORKSPACE;
  return CKV_OK;
}

int check_heads(const ckv_paged_cache* c, int num_q_heads) {
  if (num_q_heads < 1 || num_q_heads % c->num_kv_heads) return CKV_ERR_INVALID_ARG;
  if (num_q_heads > kMaxQHeads || num_q_heads / c->num_kv_heads > kPagedTile) return CKV_ERR_UNSUPPORTED;
  return CKV_OK;
}

}  // namespace

extern "C" {

int compresskv_rope_apply(const ckv_rope* r, const ckv_rope_rows* x, const int32_t* positions, const void* q,
                          const void* k, void* q_out, void* k_out, void* stream) {
  NvtxRange nvtx_range(__func__);
  int rc = check_rope(r);
  if (rc != CKV_OK) return rc;
  if (!x || x->rows < 0 || x->num_q_heads < 0 || x->num_k_heads < 0 || !dtype_ok(x->dtype))
    return CKV_ERR_INVALID_ARG;
  if (x->num_q_heads > kMaxQHeads || x->num_k_heads > kMaxQHeads) return CKV_ERR_UNSUPPORTED;
  if (x->num_q_heads == 0 ? (q || q_out) : x->num_k_heads == 0 && (k || k_out)) return CKV_ERR_INVALID_ARG;
  if (x->num_k_heads == 0 && (k || k_out)) return CKV_ERR_INVALID_ARG;
  if (x->rows == 0 || x->num_q_heads + x->num_k_heads == 0) return CKV_OK;
  if (!positions || (rc = check_index(positions)) != CKV_OK) return CKV_ERR_INVALID_ARG;
  if (x->num_q_heads && (rc = check_rows(x->rows, x->num_q_heads, q, x->q_token_stride, x->q_head_stride, q_out,
                                         x->q_out_token_stride, x->q_out_head_stride)) != CKV_OK)
    return rc;
  if (x->num_k_heads && (rc = check_rows(x->rows, x->num_k_heads, k, x->k_token_stride, x->k_head_stride, k_out,
                                         x->k_out_token_stride, x->k_out_head_stride)) != CKV_OK)
    return rc;
  if (rows_meet(x->rows, q_out, x->num_q_heads, x->q_out_token_stride, x->q_out_head_stride, k, x->num_k_heads,
                x->k_token_stride, x->k_head_stride) ||
      rows_meet(x->rows, q_out, x->num_q_heads, x->q_out_token_stride, x->q_out_head_stride, k_out, x->num_k_heads,
                x->k_out_token_stride, x->k_out_head_stride) ||
      rows_meet(x->rows, k_out, x->num_k_heads, x->k_out_token_stride, x->k_out_head_stride, q, x->num_q_heads,
                x->q_token_stride, x->q_head_stride))
    return CKV_ERR_INVALID_ARG;
  static thread_local RopeParams P;
  std::memset(&P, 0, sizeof(P));
  P.rope = rope_table(r);
  P.q = row_set(q, x->q_token_stride, x->q_head_stride, q_out, x->q_out_token_stride, x->q_out_head_stride);
  P.k = row_set(k, x->k_token_stride, x->k_head_stride, k_out, x->k_out_token_stride, x->k_out_head_stride);
  P.positions = positions;
  P.rows = x->rows;
  P.num_q = x->num_q_heads;
  P.num_k = x->num_k_heads;
  P.is_bf16 = x->dtype == CKV_DTYPE_BF16;
  P.backward = x->backward != 0;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  Tracer tr{x->trace, st};
  return traced(tr, CKV_KERNEL_ROPE, [&] { return launch_rope(P, st); });
}

int compresskv_paged_append(const ckv_paged_cache* c, const ckv_paged_rows* r, const void* k, const void* v,
                            const int32_t* start, const ckv_rope* rope, const int32_t* positions, const void* q,
                            void* q_out, int32_t* device_status, void* stream) {
  NvtxRange nvtx_range(__func__);
  int rc = check_cache(c);
  if (rc != CKV_OK) return rc;
  if (!r || r->num_q_heads < 0) return CKV_ERR_INVALID_ARG;
  if (r->num_q_heads > kMaxQHeads) return CKV_ERR_UNSUPPORTED;
  if (rope ? (rc = check_rope(rope)) != CKV_OK : r->num_q_heads > 0) return CKV_ERR_INVALID_ARG;
  if (r->num_q_heads == 0 && (q || q_out)) return CKV_ERR_INVALID_ARG;
  if (check_index(start) != CKV_OK || check_index(positions) != CKV_OK || check_index(device_status) != CKV_OK)
    return CKV_ERR_INVALID_ARG;
  if (start == c->lengths) start = nullptr;
  const uint64_t word = sizeof(int32_t) * static_cast<uint64_t>(c->batch);
  if (start && share(start, word, c->lengths, word)) return CKV_ERR_INVALID_ARG;
  static thread_local RopeParams P;
  std::memset(&P, 0, sizeof(P));
  int most = 0;
  if ((rc = take_rows(c, r->cu_rows, r->rows_per_seq, P.cu_rows, &P.rows_per_seq, &P.rows, &most)) != CKV_OK)
    return rc;
  if (P.rows == 0 && !start) return CKV_OK;  // no row, and every length stays
  if (P.rows > 0) {
    if (!k || !v || !aligned16(k) || !aligned16(v) || !strides_ok(r->kv_token_stride, r->kv_head_stride))
      return CKV_ERR_INVALID_ARG;
    if (r->num_q_heads && (rc = check_rows(P.rows, r->num_q_heads, q, r->q_token_stride, r->q_head_stride, q_out,
                                           r->q_out_token_stride, r->q_out_head_stride)) != CKV_OK)
      return rc;
    for (const void* from : {k, v})
      if (rows_meet(P.rows, q_out, r->num_q_heads, r->q_out_token_stride, r->q_out_head_stride, from,
                    c->num_kv_heads, r->kv_token_stride, r->kv_head_stride))
        return CKV_ERR_INVALID_ARG;
  }
  P.c = device_cache(c);
  if (rope)
    P.rope = rope_table(rope);
  P.q = row_set(q, r->q_token_stride, r->q_head_stride, q_out, r->q_out_token_stride, r->q_out_head_stride);
  P.k = row_set(k, r->kv_token_stride, r->kv_head_stride, nullptr, 0, 0);
  P.v = row_set(v, r->kv_token_stride, r->kv_head_stride, nullptr, 0, 0);
  P.positions = positions;
  P.start = start;
  P.status = device_status;
  P.num_q = r->num_q_heads;
  P.num_k = c->num_kv_heads;
  P.is_bf16 = c->dtype == CKV_DTYPE_BF16;
  P.paged = 1;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  Tracer tr{c->trace, st};
  return traced(tr, CKV_KERNEL_PAGED_WRITE, [&] { return launch_paged_append(P, most, st); });
}

int compresskv_paged_gather(const ckv_paged_cache* c, const int32_t* cu_rows, int32_t rows_per_seq,
                            const int32_t* start, void* k_out, void* v_out, int32_t* device_status, void* stream) {
  NvtxRange nvtx_range(__func__);
  int rc = check_cache(c);
  if (rc != CKV_OK) return rc;
  if (check_index(start) != CKV_OK || check_index(device_status) != CKV_OK || !aligned16(k_out) || !aligned16(v_out))
    return CKV_ERR_INVALID_ARG;
  static thread_local PagedGatherParams P;
  std::memset(&P, 0, sizeof(P));
  int most = 0;
  if ((rc = take_rows(c, cu_rows, rows_per_seq, P.cu_rows, &P.rows_per_seq, &P.rows, &most)) != CKV_OK) return rc;
  if (P.rows == 0 || (!k_out && !v_out)) return CKV_OK;
  P.c = device_cache(c);
  P.out[0] = static_cast<uint16_t*>(k_out);
  P.out[1] = static_cast<uint16_t*>(v_out);
  P.start = start;
  P.status = device_status;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  Tracer tr{c->trace, st};
  return traced(tr, CKV_KERNEL_PAGED_GATHER, [&] { return launch_paged_gather(P, st); });
}

int compresskv_debug_stall_next_paged_attend(long long wait_ns) {
  if (wait_ns < 0 || (wait_ns > 0 && (wait_ns < 100000 || wait_ns > 2000000000ll)))
    return CKV_ERR_INVALID_ARG;
  g_stall_attend_ns.store(wait_ns);
  return CKV_OK;
}

size_t compresskv_paged_workspace_size(const ckv_paged_cache* c, int32_t num_q_heads, int32_t num_queries) {
  if (check_cache(c, false) != CKV_OK || num_queries < 0 || check_heads(c, num_q_heads) != CKV_OK) return 0;
  const long long rows = static_cast<long long>(num_queries) * (num_q_heads / c->num_kv_heads);
  size_t n = attend_area(std::min<long long>(rows, kPagedTile)).bytes;
  if (rows > kPagedTile) n = std::max(n, attend_area(rows).bytes);
  return n;
}

int compresskv_paged_workspace_init(void* workspace, size_t workspace_bytes, void* stream) {
  NvtxRange nvtx_range(__func__);
  const int rc = check_workspace(workspace, workspace_bytes, kPagedHeaderBytes);
  if (rc != CKV_OK) return rc;
  return cudaMemsetAsync(workspace, 0, kPagedHeaderBytes, static_cast<cudaStream_t>(stream)) == cudaSuccess
             ? CKV_OK
             : CKV_ERR_CUDA;
}

int compresskv_paged_attend(const ckv_paged_cache* c, const ckv_paged_queries* a, const void* q,
                            const int32_t* start, void* out, float* lse, void* workspace, size_t workspace_bytes,
                            void* stream) {
  NvtxRange nvtx_range(__func__);
  int rc = check_cache(c);
  if (rc != CKV_OK) return rc;
  if (!a) return CKV_ERR_INVALID_ARG;
  if ((rc = check_heads(c, a->num_q_heads)) != CKV_OK) return rc;
  if (!(a->scale >= 0.f && a->scale <= kMaxScale)) return CKV_ERR_INVALID_ARG;  // (NaN too)
  if (check_index(start) != CKV_OK || (reinterpret_cast<uintptr_t>(lse) & 3u)) return CKV_ERR_INVALID_ARG;
  static thread_local PagedAttendParams P;
  std::memset(&P, 0, sizeof(P));
  int most = 0;
  if ((rc = take_rows(c, a->cu_rows, a->rows_per_seq, P.cu_rows, &P.rows_per_seq, &P.rows, &most)) != CKV_OK)
    return rc;
  if (P.rows > 0) {
    if ((rc = check_rows(P.rows, a->num_q_heads, q, a->q_token_stride, a->q_head_stride, out, a->out_token_stride,
                         a->out_head_stride)) != CKV_OK)
      return rc;
    if ((P.rows > 1 && a->q_token_stride == 0) || (a->num_q_heads > 1 && a->q_head_stride == 0))
      return CKV_ERR_INVALID_ARG;
    if (share(q, 2 * span_of(P.rows, a->num_q_heads, a->q_token_stride, a->q_head_stride), out,
              2 * span_of(P.rows, a->num_q_heads, a->out_token_stride, a->out_head_stride)))
      return CKV_ERR_INVALID_ARG;  // (a row of q is read after another's output is written)
    if (static_cast<int64_t>(P.rows) * a->num_q_heads > kMaxQueryRows) return CKV_ERR_UNSUPPORTED;
  }
  if ((rc = check_workspace(workspace, workspace_bytes,
                            compresskv_paged_workspace_size(c, a->num_q_heads, most))) != CKV_OK)
    return rc;
  if (P.rows == 0) return CKV_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int sms = 0;
  if ((rc = usable_sms(st, &sms)) != CKV_OK) return rc;
  const bool bf16 = c->dtype == CKV_DTYPE_BF16;
  P.group = a->num_q_heads / c->num_kv_heads;
  const long long unit_rows = static_cast<long long>(most) * P.group;
  P.pair = unit_rows > kPagedTile;
  P.tile_tokens = kPagedTile / P.group;
  P.item_tokens = P.pair ? 2 * P.tile_tokens : P.tile_tokens;
  const int box_tokens = std::min(P.tile_tokens, most);
  P.q_box_bytes = box_tokens * P.group * 64 * 2;
  P.q_buffers = box_tokens * P.group <= 32 ? 4 : box_tokens * P.group <= 64 ? 2 : 1;
  {
    const unsigned long long dims[2] = {static_cast<unsigned long long>(a->num_q_heads),
                                        static_cast<unsigned long long>(P.rows)};
    // (a dimension of one element has a stride that means nothing)
    const long long strides[2] = {a->num_q_heads > 1 ? a->q_head_stride : kHeadDim,
                                  P.rows > 1 ? a->q_token_stride : kHeadDim};
    const unsigned box[2] = {static_cast<unsigned>(P.group), static_cast<unsigned>(box_tokens)};
    if ((rc = make_rows_map(q, bf16, 3, dims, strides, box, &P.map_q)) != CKV_OK) return rc;
  }
  {
    const unsigned long long dims[3] = {static_cast<unsigned long long>(c->num_kv_heads),
                                        static_cast<unsigned long long>(c->page_size),
                                        static_cast<unsigned long long>(c->num_pages)};
    const long long strides[3] = {c->num_kv_heads > 1 ? c->head_stride : kHeadDim, c->slot_stride,
                                  c->num_pages > 1 ? c->page_stride : kHeadDim};
    const unsigned box[3] = {1u, static_cast<unsigned>(std::min(c->page_size, kPagedTile)), 1u};
    if ((rc = make_rows_map(c->k_pages, bf16, 4, dims, strides, box, &P.map_k)) != CKV_OK) return rc;
    if ((rc = make_rows_map(c->v_pages, bf16, 4, dims, strides, box, &P.map_v)) != CKV_OK) return rc;
  }
  P.c = device_cache(c);
  P.out = static_cast<uint16_t*>(out);
  P.lse = lse;
  P.start = start;
  P.o_token = a->out_token_stride;
  P.o_head = a->out_head_stride;
  const double scale = a->scale > 0.f ? a->scale : 1.0 / std::sqrt(static_cast<double>(kHeadDim));
  P.scale_log2 = static_cast<float>(scale * 1.4426950408889634);
  P.causal = a->causal != 0;
  P.wide_rows = (reinterpret_cast<uintptr_t>(out) & 31u) == 0 && a->out_token_stride % 16 == 0 && a->out_head_stride % 16 == 0;
  P.is_bf16 = bf16;
  P.status = static_cast<int*>(workspace);
  P.stopped = P.status + 1;
  P.next = P.status + 2;
  P.done = P.status + 3;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  P.tickets = reinterpret_cast<int*>(ws + kPagedTickets);
  const AttendArea area = attend_area(unit_rows);
  P.part_ml = reinterpret_cast<float2*>(ws + area.ml);
  P.part_o = reinterpret_cast<float*>(ws + area.o);
  P.part_rows = area.rows;
  P.stall_ns = static_cast<unsigned long long>(g_stall_attend_ns.exchange(0));
  // no more CTAs than there can be tiles
  const long long items = std::max<long long>((P.rows + P.item_tokens - 1) / P.item_tokens, 1) + c->batch;
  const long long tiles = items * c->num_kv_heads * ((c->table_width * static_cast<long long>(c->page_size) + kPagedTile - 1) / kPagedTile);
  const int ctas = static_cast<int>(std::min<long long>({sms, kPagedMaxCtas, tiles}));
  Tracer tr{c->trace, st};
  return traced(tr, CKV_KERNEL_PAGED_ATTEND, [&] { return launch_paged_attend(P, ctas, st); });
}

}  // extern "C"
