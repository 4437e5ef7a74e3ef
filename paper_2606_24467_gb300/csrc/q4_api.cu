// Host side of the 4-bit cache's entry points (include/compresskv.h):
// argument checks, workspace and launches.  Nothing here allocates device
// memory or waits for a stream.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>
#include <new>

#include "compresskv.h"
#include "host_common.h"
#include "q4_params.h"

using namespace ckv;

namespace {

constexpr int kMaxCapacity = 1 << 24;
constexpr float kMaxScale = 0x1p96f;

// Test hook: how long the next attention stalls on purpose (0: not).
std::atomic<long long> g_stall_attend_ns{0};

size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

// The cache's shape (and, with `pointers`, its buffers).
int check_cache(const ckv_q4_cache* c, bool pointers = true) {
  if (!c || c->batch < 1 || c->num_kv_heads < 1 || c->capacity < 1) return CKV_ERR_INVALID_ARG;
  if (c->capacity % kQ4SlotStep) return CKV_ERR_INVALID_ARG;
  if (c->head_dim != kHeadDim || c->num_kv_heads > kMaxKvHeads || c->capacity > kMaxCapacity)
    return CKV_ERR_UNSUPPORTED;
  const long long units = static_cast<long long>(c->batch) * c->num_kv_heads;
  if (units > kQ4MaxUnits || units * c->capacity > (1LL << 31) - 1) return CKV_ERR_UNSUPPORTED;
  if (!pointers) return CKV_OK;
  if (!c->k_codes || !c->v_codes || !c->k_params || !c->v_params || !c->positions || !c->lengths)
    return CKV_ERR_INVALID_ARG;
  for (const void* ptr : {static_cast<const void*>(c->k_codes), static_cast<const void*>(c->v_codes),
                          static_cast<const void*>(c->k_params), static_cast<const void*>(c->v_params),
                          static_cast<const void*>(c->positions), static_cast<const void*>(c->weights)})
    if (!aligned16(ptr)) return CKV_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(c->lengths) & 3u) return CKV_ERR_INVALID_ARG;
  return CKV_OK;
}

int units_of(const ckv_q4_cache* c) { return c->batch * c->num_kv_heads; }
long long slots_of(const ckv_q4_cache* c) { return static_cast<long long>(units_of(c)) * c->capacity; }

Q4Cache device_cache(const ckv_q4_cache* c) {
  Q4Cache d;
  d.codes[0] = static_cast<uint8_t*>(c->k_codes);
  d.codes[1] = static_cast<uint8_t*>(c->v_codes);
  d.params[0] = static_cast<uint8_t*>(c->k_params);
  d.params[1] = static_cast<uint8_t*>(c->v_params);
  d.positions = c->positions;
  d.weights = c->weights;
  d.lengths = c->lengths;
  d.capacity = c->capacity;
  d.num_kv_heads = c->num_kv_heads;
  d.batch = c->batch;
  return d;
}

bool row_strides_ok(int64_t token, int64_t head) {
  return token > 0 && head > 0 && token % 8 == 0 && head % 8 == 0;
}

int check_values(const void* k, const void* v) {
  return aligned16(k) && aligned16(v) ? CKV_OK : CKV_ERR_INVALID_ARG;
}

// The attention's area behind the workspace header (status word at its start,
// the word that says that a call has stopped behind it, the tickets from
// kTicketBytes on).
constexpr size_t kTicketBytes = 256;
static_assert(kTicketBytes + kQ4MaxCtas * sizeof(int) <= kQ4HeaderBytes, "tickets");
struct AttendArea {
  size_t head_ml = 0, head_o = 0, cta_ml = 0, cta_o = 0, lse = 0, z = 0, bytes = 0;
};
AttendArea attend_area(const ckv_q4_cache* c, int num_q_heads, int num_queries, bool accumulate) {
  const size_t rows = static_cast<size_t>(num_q_heads / c->num_kv_heads) * num_queries;
  const size_t brows = q4_block_rows(static_cast<int>(rows), slots_of(c));
  const size_t heads = kQ4MaxCtas * kQ4Warps * brows;
  const size_t ctas = kQ4MaxCtas * 2 * brows;
  AttendArea a;
  a.head_ml = kQ4HeaderBytes;
  a.head_o = a.head_ml + align256(heads * sizeof(float2));
  a.cta_ml = a.head_o + align256(heads * kHeadDim * sizeof(float));
  a.cta_o = a.cta_ml + align256(ctas * sizeof(float2));
  a.lse = a.cta_o + align256(ctas * kHeadDim * sizeof(float));
  a.z = a.lse + align256(units_of(c) * rows * sizeof(float));
  a.bytes = a.z + (accumulate ? align256(units_of(c) * (rows + rows % 2) * c->capacity * sizeof(float)) : 0);
  return a;
}
size_t evict_bytes(const ckv_q4_cache* c) {
  return kQ4HeaderBytes + align256(static_cast<size_t>(units_of(c)) * c->capacity * sizeof(int32_t));
}

int check_workspace(const void* ws, size_t have, size_t need) {
  if (!ws || have < need || (reinterpret_cast<uintptr_t>(ws) & 255u)) return CKV_ERR_WORKSPACE;
  return CKV_OK;
}

int check_heads(const ckv_q4_cache* c, int num_q_heads, int num_queries) {
  if (num_q_heads < 1 || num_queries < 1 || num_q_heads % c->num_kv_heads) return CKV_ERR_INVALID_ARG;
  if (num_q_heads > kMaxQHeads || num_queries > kQ4MaxQueries) return CKV_ERR_UNSUPPORTED;
  if (num_q_heads / c->num_kv_heads * num_queries > kMaxQRows) return CKV_ERR_UNSUPPORTED;
  return CKV_OK;
}

// Whether two rows of kHeadDim elements share one, in a layout of n[i] rows at
// strides[i] (0 .. kMaxStride) in each of three dimensions.  They do not where
// every stride holds what the smaller ones span; otherwise they do exactly
// where the indices' differences, not all zero, come to less than a row.
constexpr int64_t kMaxStride = 1LL << 44;  // (32 TB: products of strides and indices stay in 64 bits)
bool rows_overlap(const int64_t (&strides)[3], const int (&n)[3]) {
  int order[3] = {0, 1, 2};
  std::sort(order, order + 3, [&](int a, int b) { return strides[a] < strides[b]; });
  int64_t span = kHeadDim;
  bool nested = true;
  for (int d : order) {
    if (n[d] == 1) continue;
    nested = nested && strides[d] >= span;
    span += strides[d] * (n[d] - 1);  // (a dimension of one row has no stride)
  }
  if (nested) return false;
  // the dimension of most rows is solved for
  const int a = static_cast<int>(std::max_element(n, n + 3) - n), b = (a + 1) % 3, c = (a + 2) % 3;
  const int64_t s = strides[a], most = n[a] - 1;
  if (most > 0 && s < kHeadDim) return true;
  for (int64_t j = 0; j < n[b]; ++j)
    for (int64_t k = j ? 1 - n[c] : 1; k < n[c]; ++k) {
      const int64_t rest = j * strides[b] + k * strides[c], near = most ? -rest / s : 0;
      for (int64_t i = near - 1; i <= near + 1; ++i) {
        const int64_t at = rest + std::min(std::max(i, -most), most) * s;
        if (at < kHeadDim && at > -kHeadDim) return true;
      }
    }
  return false;
}

template <class P>
int gather(P& P_, const ckv_problem* p, int group_major, const ckv_q4_cache* c, const int32_t* indices,
           const int32_t* cu_out, const void* k, const void* v, const float* raw, void* k_values,
           void* v_values, void* workspace, cudaStream_t stream) {
  const int tables = group_major ? c->num_kv_heads : 1;
  std::memset(&P_, 0, sizeof(P_));
  int prefix = 0;
  for (int s = 0; s <= c->batch; ++s) {
    P_.cu_seqlens[s] = p->cu_seqlens[s];
    P_.cu_prefix[s] = prefix;
    if (s < c->batch) prefix += std::max(p->cu_seqlens[s + 1] - p->cu_seqlens[s] - p->window, 0);
  }
  int at = 0;
  for (int t = 0; t < tables; ++t)
    for (int s = 0; s <= c->batch; ++s) {
      const int i = t * (c->batch + 1) + s;
      const long long kept = s ? static_cast<long long>(cu_out[i]) - cu_out[i - 1] : 0;
      if (s ? (kept < 0 || kept > p->cu_seqlens[s] - p->cu_seqlens[s - 1] || kept > c->capacity)
            : cu_out[i] != at)
        return CKV_ERR_INVALID_ARG;
      P_.cu_rows[i] = at = cu_out[i];
    }
  const long long rows = group_major ? at : static_cast<long long>(at) * c->num_kv_heads;
  if (rows > (1LL << 31) - 1) return CKV_ERR_UNSUPPORTED;
  if (rows > 0) {
    if (!indices || !k || !v || !aligned16(k) || !aligned16(v)) return CKV_ERR_INVALID_ARG;
    const int rv = device_readable(v, &v);
    if (rv != CKV_OK) return rv;
  }
  if (check_values(k_values, v_values) != CKV_OK) return CKV_ERR_INVALID_ARG;
  P_.c = device_cache(c);
  P_.src[0] = static_cast<const uint16_t*>(k);
  P_.src[1] = static_cast<const uint16_t*>(v);
  P_.values[0] = static_cast<uint16_t*>(k_values);
  P_.values[1] = static_cast<uint16_t*>(v_values);
  P_.tok_stride = p->kv_token_stride;
  P_.head_stride = p->kv_head_stride;
  P_.indices = indices;
  P_.raw = raw;
  P_.status = static_cast<int*>(workspace);
  P_.is_bf16 = p->dtype == CKV_DTYPE_BF16;
  P_.rows = at;
  P_.group_major = group_major;
  P_.window = p->window;
  P_.p_total = prefix;
  Tracer tr{p->trace, stream};
  return traced(tr, CKV_KERNEL_Q4_WRITE, [&] { return launch_q4_gather(P_, stream); });
}

}  // namespace

extern "C" {

int compresskv_debug_stall_next_q4_attend(long long wait_ns) {
  if (wait_ns < 0 || (wait_ns > 0 && (wait_ns < 100000 || wait_ns > 2000000000ll)))
    return CKV_ERR_INVALID_ARG;
  g_stall_attend_ns.store(wait_ns);
  return CKV_OK;
}

size_t compresskv_q4_workspace_size(const ckv_q4_cache* c, int32_t num_q_heads, int32_t num_queries) {
  if (check_cache(c, false) != CKV_OK) return 0;
  size_t n = evict_bytes(c);
  if (num_q_heads != 0 || num_queries != 0) {
    if (check_heads(c, num_q_heads, num_queries) != CKV_OK) return 0;
    const bool weights = c->weights != nullptr;
    n = std::max(n, attend_area(c, num_q_heads, num_queries, weights).bytes);
  }
  return n;
}

int compresskv_q4_workspace_init(void* workspace, size_t workspace_bytes, void* stream) {
  NvtxRange nvtx_range(__func__);
  const int rc = check_workspace(workspace, workspace_bytes, kQ4HeaderBytes);
  if (rc != CKV_OK) return rc;
  return cudaMemsetAsync(workspace, 0, kQ4HeaderBytes, static_cast<cudaStream_t>(stream)) == cudaSuccess
             ? CKV_OK
             : CKV_ERR_CUDA;
}

int compresskv_q4_append(const ckv_q4_cache* c, const ckv_q4_rows* r, const void* k, const void* v,
                         const int32_t* positions, const int32_t* start, void* k_values, void* v_values,
                         int32_t* device_status, void* stream) {
  NvtxRange nvtx_range(__func__);
  int rc = check_cache(c);
  if (rc != CKV_OK) return rc;
  if (!r || (r->dtype != CKV_DTYPE_F16 && r->dtype != CKV_DTYPE_BF16)) return CKV_ERR_INVALID_ARG;
  if (!row_strides_ok(r->token_stride, r->head_stride)) return CKV_ERR_INVALID_ARG;
  static thread_local Q4AppendParams P;
  std::memset(&P, 0, sizeof(P));
  int most = 0;
  long long rows = 0;
  if (r->cu_rows) {
    if (c->batch > kMaxBatch) return CKV_ERR_UNSUPPORTED;
    if (r->cu_rows[0] != 0) return CKV_ERR_INVALID_ARG;
    for (int s = 0; s < c->batch; ++s) {
      if (r->cu_rows[s + 1] < r->cu_rows[s]) return CKV_ERR_INVALID_ARG;
      most = std::max(most, r->cu_rows[s + 1] - r->cu_rows[s]);
    }
    std::copy(r->cu_rows, r->cu_rows + c->batch + 1, P.cu_rows);
    rows = r->cu_rows[c->batch];
    P.rows_per_seq = -1;
  } else {
    if (r->rows_per_seq < 0) return CKV_ERR_INVALID_ARG;
    most = P.rows_per_seq = r->rows_per_seq;
    rows = static_cast<long long>(most) * c->batch;
  }
  if (rows * c->num_kv_heads > (1LL << 31) - 1) return CKV_ERR_UNSUPPORTED;
  if (rows == 0 && !start) return CKV_OK;  // no row, and every length stays
  if (rows > 0) {
    if (!k || !v || !positions || !aligned16(k) || !aligned16(v)) return CKV_ERR_INVALID_ARG;
    if ((rc = device_readable(v, &v)) != CKV_OK) return rc;
  }
  if ((rc = check_values(k_values, v_values)) != CKV_OK) return rc;
  P.c = device_cache(c);
  P.src[0] = static_cast<const uint16_t*>(k);
  P.src[1] = static_cast<const uint16_t*>(v);
  P.values[0] = static_cast<uint16_t*>(k_values);
  P.values[1] = static_cast<uint16_t*>(v_values);
  P.tok_stride = r->token_stride;
  P.head_stride = r->head_stride;
  P.positions = positions;
  P.start = start;
  P.status = device_status;
  P.is_bf16 = r->dtype == CKV_DTYPE_BF16;
  P.rows = static_cast<int>(rows);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  Tracer tr{c->trace, st};
  return traced(tr, CKV_KERNEL_Q4_WRITE, [&] { return launch_q4_append(P, most, st); });
}

int compresskv_q4_gather(const ckv_problem* p, const ckv_q4_cache* c, int32_t group_major,
                         const int32_t* indices, const int32_t* cu_out, const void* k, const void* v,
                         const float* raw_scores, void* k_values, void* v_values, void* workspace,
                         void* stream) {
  NvtxRange nvtx_range(__func__);
  try {
    int rc = check_problem(p);
    if (rc == CKV_OK) rc = check_cache(c);
    if (rc != CKV_OK) return rc;
    if (!cu_out || p->batch != c->batch || p->num_kv_heads != c->num_kv_heads) return CKV_ERR_INVALID_ARG;
    if (workspace && (reinterpret_cast<uintptr_t>(workspace) & 255u)) return CKV_ERR_WORKSPACE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (group_major) {
      if (units_of(c) > kMaxBudgetUnits) return CKV_ERR_UNSUPPORTED;
      static thread_local Q4GatherUnitParams P;
      return gather(P, p, 1, c, indices, cu_out, k, v, raw_scores, k_values, v_values, workspace, st);
    }
    static thread_local Q4GatherParams P;
    return gather(P, p, 0, c, indices, cu_out, k, v, raw_scores, k_values, v_values, workspace, st);
  } catch (const std::bad_alloc&) {
    return CKV_ERR_CUDA;
  }
}

int compresskv_q4_attend(const ckv_q4_cache* c, const ckv_q4_queries* a, const void* q,
                         const int32_t* q_positions, void* out, float* lse, void* workspace,
                         size_t workspace_bytes, void* stream) {
  NvtxRange nvtx_range(__func__);
  int rc = check_cache(c);
  if (rc != CKV_OK) return rc;
  if (!a || (a->dtype != CKV_DTYPE_F16 && a->dtype != CKV_DTYPE_BF16)) return CKV_ERR_INVALID_ARG;
  if ((rc = check_heads(c, a->num_q_heads, a->num_queries)) != CKV_OK) return rc;
  // (NaN too; the kernel holds it times 2^10 log2 e)
  if (!(a->scale >= 0.f && a->scale <= kMaxScale)) return CKV_ERR_INVALID_ARG;
  if (a->accumulate && !c->weights) return CKV_ERR_INVALID_ARG;
  if (!q || !out || !aligned16(q) || !aligned16(out)) return CKV_ERR_INVALID_ARG;
  const int64_t in[3] = {a->q_batch_stride, a->q_head_stride, a->q_query_stride};
  const int64_t to[3] = {a->out_batch_stride, a->out_head_stride, a->out_query_stride};
  const int dims[3] = {c->batch, a->num_q_heads, a->num_queries};
  for (int i = 0; i < 3; ++i)
    if (in[i] < 0 || in[i] % 8 || to[i] < 0 || to[i] % 8 || (dims[i] > 1 && std::max(in[i], to[i]) > kMaxStride))
      return CKV_ERR_INVALID_ARG;
  if (rows_overlap(to, dims)) return CKV_ERR_INVALID_ARG;
  const AttendArea area = attend_area(c, a->num_q_heads, a->num_queries, a->accumulate != 0);
  if ((rc = check_workspace(workspace, workspace_bytes, area.bytes)) != CKV_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int sms = 0;
  if ((rc = usable_sms(st, &sms)) != CKV_OK) return rc;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  Q4AttendParams P;
  std::memset(&P, 0, sizeof(P));
  P.group = a->num_q_heads / c->num_kv_heads;
  P.num_queries = a->num_queries;
  P.rows = P.group * P.num_queries;
  P.block_rows = q4_block_rows(P.rows, slots_of(c));
  P.blocks = (P.rows + P.block_rows - 1) / P.block_rows;
  if ((rc = make_row64_map(c->k_codes, slots_of(c), kQ4Tile, &P.map_k)) != CKV_OK) return rc;
  if ((rc = make_row64_map(c->v_codes, slots_of(c), kQ4Tile, &P.map_v)) != CKV_OK) return rc;
  P.c = device_cache(c);
  P.q = static_cast<const uint16_t*>(q);
  P.out = static_cast<uint16_t*>(out);
  P.lse = lse;
  P.q_positions = q_positions;
  P.q_bs = in[0];
  P.q_hs = in[1];
  P.q_qs = in[2];
  P.o_bs = to[0];
  P.o_hs = to[1];
  P.o_qs = to[2];
  const double scale = a->scale > 0.f ? a->scale : 1.0 / std::sqrt(static_cast<double>(kHeadDim));
  P.scale_log2 = static_cast<float>(scale * 1.4426950408889634);
  P.num_q_heads = a->num_q_heads;
  P.is_bf16 = a->dtype == CKV_DTYPE_BF16;
  P.accumulate = a->accumulate != 0;
  P.status = static_cast<int*>(workspace);
  // no more CTAs than there can be tiles
  const long long tiles = static_cast<long long>(units_of(c)) * ((c->capacity + kQ4Tile - 1) / kQ4Tile) * P.blocks;
  sms = static_cast<int>(std::min<long long>({sms, kQ4MaxCtas, tiles}));
  P.stopped = P.status + 1;
  P.tickets = reinterpret_cast<int*>(ws + kTicketBytes);
  P.head_ml = reinterpret_cast<float2*>(ws + area.head_ml);
  P.head_o = reinterpret_cast<float*>(ws + area.head_o);
  P.cta_ml = reinterpret_cast<float2*>(ws + area.cta_ml);
  P.cta_o = reinterpret_cast<float*>(ws + area.cta_o);
  P.lse_ws = reinterpret_cast<float*>(ws + area.lse);
  P.z = reinterpret_cast<float*>(ws + area.z);
  P.z_stride = P.rows + P.rows % 2;
  P.stall_ns = static_cast<unsigned long long>(g_stall_attend_ns.exchange(0));
  Tracer tr{c->trace, st};
  rc = traced(tr, CKV_KERNEL_Q4_ATTEND, [&] { return launch_q4_attend(P, sms, st); });
  if (rc != CKV_OK || !P.accumulate) return rc;
  return traced(tr, CKV_KERNEL_Q4_ATTEND, [&] { return launch_q4_weights(P, st); });
}

int compresskv_q4_evict(const ckv_q4_cache* c, int32_t budget, const int32_t* budgets, int32_t sinks,
                        int32_t recent, void* workspace, size_t workspace_bytes, void* stream) {
  NvtxRange nvtx_range(__func__);
  int rc = check_cache(c);
  if (rc != CKV_OK) return rc;
  if (!c->weights || sinks < 0 || recent < 0) return CKV_ERR_INVALID_ARG;
  if (!budgets) {
    if (budget < 0) return CKV_ERR_INVALID_ARG;
    if (budget < static_cast<int64_t>(sinks) + recent) return CKV_ERR_BUDGET;
  }
  if ((rc = check_workspace(workspace, workspace_bytes, evict_bytes(c))) != CKV_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int sms = 0;
  if ((rc = usable_sms(st, &sms)) != CKV_OK) return rc;
  Q4EvictParams P;
  std::memset(&P, 0, sizeof(P));
  P.c = device_cache(c);
  P.budgets = budgets;
  P.budget = budget;
  P.sinks = sinks;
  P.recent = recent;
  P.status = static_cast<int*>(workspace);
  P.lists = reinterpret_cast<int32_t*>(static_cast<uint8_t*>(workspace) + kQ4HeaderBytes);
  Tracer tr{c->trace, st};
  return traced(tr, CKV_KERNEL_Q4_EVICT, [&] { return launch_q4_evict(P, sms, st); });
}

}  // extern "C"
