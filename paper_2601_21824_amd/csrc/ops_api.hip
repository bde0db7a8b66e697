// ops_api.hip -- the C ABI of the variable-length operators (include/dash.h):
// argument checks, workspace layout and launches.  Host code only; the kernels
// live in kv_append.hip, attn_decode.hip and attn_packed_*.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "api.h"
#include "dash.h"
#include "ops.h"
#include "packed_order.h"
#include "page_index.h"

namespace {

using dash::api::device_info;
using dash::api::DeviceInfo;
using dash::api::fail;
using dash::api::hip_fail;

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

constexpr int64_t kMaxRowStride = 1 << 22;
constexpr int kMaxBatch = 1 << 20, kMaxHeads = 1 << 12, kMaxRows = 1 << 28;

int check_heads(int batch, int heads_q, int heads_kv, int d) {
  if (batch < 0 || batch > kMaxBatch) return fail(DASH_ERR_INVALID_ARG, "batch must be in 0 .. 2^20");
  if (heads_kv < 1 || heads_q < 1 || heads_q > kMaxHeads || heads_q % heads_kv)
    return fail(DASH_ERR_INVALID_ARG, "heads_kv must divide heads_q, heads_q at most 4096");
  if (d != 64 && d != 128 && d != 256) return fail(DASH_ERR_INVALID_ARG, "head dim d must be 64, 128 or 256");
  return DASH_OK;
}

// whether elements d apart along up to three strided dimensions can meet: each
// stride, from the smallest, has to pass what lies inside it
struct Dim {
  int64_t n, stride;
};
bool overlap(Dim a, Dim b, Dim c, int d) {
  Dim t[3] = {a, b, c};
  std::sort(t, t + 3, [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
  int64_t span = d;
  for (const Dim& x : t) {
    if (x.n <= 1) continue;
    if (x.stride < span) return true;
    span += (x.n - 1) * x.stride;
  }
  return false;
}

// a tensor of rows x heads x d elements: aligned, in reach of the kernels' 32-bit
// offsets inside a tile, and, where the call writes it, no element twice
int check_tensor(const char* name, const void* p, int64_t rows, int heads, int d, int64_t row, int64_t head, int unit,
                 bool written) {
  if (!p) return fail(DASH_ERR_INVALID_ARG, std::string(name) + ": null pointer");
  if (rows <= 1) row = 0;  // (the stride of a single row or head means nothing)
  if (heads <= 1) head = 0;
  if (((uintptr_t)p & 15) != 0) return fail(DASH_ERR_INVALID_ARG, std::string(name) + ": must be 16-byte aligned");
  if (row < 0 || head < 0 || row % unit || head % unit)
    return fail(DASH_ERR_INVALID_ARG, std::string(name) + ": strides must be multiples of 16 bytes, and not negative");
  if (rows > 1 && (row < d || row > kMaxRowStride))
    return fail(DASH_ERR_INVALID_ARG, std::string(name) + ": the row stride must be in d .. 2^22");
  if (head > ((int64_t)1 << 40)) return fail(DASH_ERR_INVALID_ARG, std::string(name) + ": head stride too large");
  if (written && overlap({rows, row}, {heads, head}, {1, 0}, d))
    return fail(DASH_ERR_INVALID_ARG, std::string(name) + ": the strides make elements overlap");
  return DASH_OK;
}

int check_cache(const dash_paged_cache_t* c, bool written) {
  if (!c) return fail(DASH_ERR_INVALID_ARG, "null cache");
  int rc = check_heads(c->batch, c->heads_q, c->heads_kv, c->d);
  if (rc) return rc;
  if (c->cache_type != DASH_CACHE_BF16 && c->cache_type != DASH_CACHE_E4M3)
    return fail(DASH_ERR_INVALID_ARG, "unknown cache_type");
  if (c->cache_type == DASH_CACHE_BF16 && (c->k_scale || c->v_scale))
    return fail(DASH_ERR_INVALID_ARG, "k_scale and v_scale are for E4M3 caches");
  if (c->page_size < 16 || c->page_size % 16 || c->page_size > 65536)
    return fail(DASH_ERR_INVALID_ARG, "page_size must be a multiple of 16, at most 65536");
  if (c->table_width < 0 || (int64_t)c->table_width * c->page_size > dash::kMaxKeys)
    return fail(DASH_ERR_INVALID_ARG, "table_width must be >= 0 and table_width * page_size below 2^31 - 255");
  if (c->batch == 0) return DASH_OK;
  if (c->pages < 1) return fail(DASH_ERR_INVALID_ARG, "pages must be >= 1");
  if (!c->lens || (!c->block_table && c->table_width > 0)) return fail(DASH_ERR_INVALID_ARG, "null lens or block_table");
  if (c->table_stride < c->table_width && c->batch > 1) return fail(DASH_ERR_INVALID_ARG, "table_stride is below table_width");
  const int unit = c->cache_type == DASH_CACHE_E4M3 ? 16 : 8;
  const struct {
    const char* name;
    const void* p;
    int64_t page, head, row;
  } t[2] = {{"k_cache", c->k_cache, c->k_page_stride, c->k_head_stride, c->k_row_stride},
            {"v_cache", c->v_cache, c->v_page_stride, c->v_head_stride, c->v_row_stride}};
  for (const auto& x : t) {
    if ((rc = check_tensor(x.name, x.p, c->page_size, c->heads_kv, c->d, x.row, x.head, unit, written))) return rc;
    if (x.page < 0 || x.page % unit || x.page > ((int64_t)1 << 40))
      return fail(DASH_ERR_INVALID_ARG, std::string(x.name) + ": page stride must be a multiple of 16 bytes in 0 .. 2^40");
    if (written && overlap({c->page_size, x.row}, {c->heads_kv, x.head}, {c->pages, x.page}, c->d))
      return fail(DASH_ERR_INVALID_ARG, std::string(x.name) + ": the strides make pages overlap");
  }
  return DASH_OK;
}

dash::CacheArgs cache_args(const dash_paged_cache_t* c, int* status) {
  return {c->batch, c->heads_q, c->heads_kv, c->d, c->pages, c->page_size, c->table_width, c->cache_type == DASH_CACHE_E4M3,
          c->k_cache, c->v_cache, c->k_page_stride, c->k_head_stride, c->k_row_stride, c->v_page_stride, c->v_head_stride,
          c->v_row_stride, c->block_table, c->table_stride, c->lens, c->k_scale, c->v_scale, status};
}

struct DecodeLayout {
  int slots;
  size_t part_o, part_m, base, total;
};
DecodeLayout decode_layout(int batch, int heads_q, int heads_kv, int d, int tokens) {
  DecodeLayout L;
  L.slots = dash::decode_slots(batch, heads_q, heads_kv, d, tokens);
  size_t off = 0;
  L.part_o = off;
  off += align256((size_t)L.slots * heads_q * d * sizeof(float));
  L.part_m = off;
  off += align256((size_t)L.slots * heads_q * 2 * sizeof(float));
  L.base = off;
  off += align256((size_t)batch * 2 * sizeof(int));
  L.total = off;
  return L;
}

int check_scale(float* scale, int d) {
  if (*scale == 0.f) *scale = 1.0f / std::sqrt((float)d);
  if (!(*scale > 0.f) || !std::isfinite(*scale)) return fail(DASH_ERR_INVALID_ARG, "scale must be finite and > 0");
  return DASH_OK;
}

int kv_append(const dash_paged_cache_t* c, const dash_append_t* x, int* status, void* stream) {
  int rc = check_cache(c, true);
  if (rc) return rc;
  if (!x) return fail(DASH_ERR_INVALID_ARG, "null tokens");
  if (x->tokens < 0) return fail(DASH_ERR_INVALID_ARG, "tokens must be >= 0");
  if (x->inv_freq && (x->rotary_dim < 16 || x->rotary_dim % 16 || x->rotary_dim > c->d))
    return fail(DASH_ERR_INVALID_ARG, "rotary_dim must be a multiple of 16, at most d");
  if (!x->cu && x->tokens != c->batch) return fail(DASH_ERR_INVALID_ARG, "without cu, tokens must be batch");
  if (x->tokens == 0 || c->batch == 0) return DASH_OK;
  if ((rc = check_tensor("k", x->k, x->tokens, c->heads_kv, c->d, x->k_row_stride, x->k_head_stride, 8, false))) return rc;
  if ((rc = check_tensor("v", x->v, x->tokens, c->heads_kv, c->d, x->v_row_stride, x->v_head_stride, 8, false))) return rc;
  if (!x->q != !x->q_out) return fail(DASH_ERR_INVALID_ARG, "q and q_out come together");
  if (x->q) {
    if ((rc = check_tensor("q", x->q, x->tokens, c->heads_q, c->d, x->q_row_stride, x->q_head_stride, 8, false))) return rc;
    if ((rc = check_tensor("q_out", x->q_out, x->tokens, c->heads_q, c->d, x->q_out_row_stride, x->q_out_head_stride, 8, true)))
      return rc;
  }
  if (x->k_out &&
      (rc = check_tensor("k_out", x->k_out, x->tokens, c->heads_kv, c->d, x->k_out_row_stride, x->k_out_head_stride, 8, true)))
    return rc;
  const dash::AppendArgs a{cache_args(c, status), x->tokens, x->cu, x->k, x->v, x->q, x->q_out, x->k_out,
                           {x->k_row_stride, x->k_head_stride}, {x->v_row_stride, x->v_head_stride},
                           {x->q_row_stride, x->q_head_stride}, {x->q_out_row_stride, x->q_out_head_stride},
                           {x->k_out_row_stride, x->k_out_head_stride}, x->inv_freq, x->rotary_dim, x->interleaved ? 1 : 0};
  if (dash::append_waves(a) > dash::kMaxWaves) return fail(DASH_ERR_UNSUPPORTED, "too many tokens for one call");
  DeviceInfo di;
  if ((rc = device_info(&di))) return rc;
  const hipError_t e = dash::launch_kv_append(a, (hipStream_t)stream);
  return e == hipSuccess ? DASH_OK : hip_fail(e, "append launch");
}

int attn_decode(const dash_paged_cache_t* c, const void* q, int64_t q_row, int64_t q_head, void* o, int64_t o_row,
                int64_t o_head, float* lse, float scale, void* workspace, size_t ws_bytes, int* status, void* stream) {
  int rc = check_cache(c, false);
  if (rc) return rc;
  if ((rc = check_scale(&scale, c->d))) return rc;
  if (c->batch == 0) return DASH_OK;
  if ((rc = check_tensor("q", q, c->batch, c->heads_q, c->d, q_row, q_head, 8, false))) return rc;
  if ((rc = check_tensor("o", o, c->batch, c->heads_q, c->d, o_row, o_head, 8, true))) return rc;
  const DecodeLayout L = decode_layout(c->batch, c->heads_q, c->heads_kv, c->d, c->table_width * c->page_size);
  if (!workspace || ws_bytes < L.total)
    return fail(DASH_ERR_INVALID_ARG, "workspace missing or smaller than dash_decode_workspace_size()");
  if (((uintptr_t)workspace & 255) != 0) return fail(DASH_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  char* ws = (char*)workspace;
  const dash::DecodeArgs a{cache_args(c, status), q, o, lse, {q_row, q_head}, {o_row, o_head}, scale,
                           dash::decode_workers(c->heads_q, c->heads_kv, c->d, c->table_width * c->page_size), L.slots, (float*)(ws + L.part_o),
                           (float*)(ws + L.part_m), (int*)(ws + L.base)};
  if (dash::decode_waves(a) > dash::kMaxWaves) return fail(DASH_ERR_UNSUPPORTED, "batch * heads_q too large for one call");
  DeviceInfo di;
  if ((rc = device_info(&di))) return rc;
  const hipError_t e = dash::launch_decode(a, (hipStream_t)stream);
  return e == hipSuccess ? DASH_OK : hip_fail(e, "decode launch");
}

// what both directions of a packed call need; false in *work: nothing to compute
int check_packed(const dash_packed_t* p, float* scale, const void* q, const void* k, const void* v, const void* o, bool o_written,
                 const float* lse, bool* work) {
  if (!p) return fail(DASH_ERR_INVALID_ARG, "null problem");
  int rc = check_heads(p->batch, p->heads_q, p->heads_kv, p->d);
  if (rc) return rc;
  *scale = p->scale;
  if ((rc = check_scale(scale, p->d))) return rc;
  if (p->total_q < 0 || p->total_k < 0 || p->total_q > kMaxRows || p->total_k > kMaxRows)
    return fail(DASH_ERR_INVALID_ARG, "total_q and total_k must be in 0 .. 2^28");
  if ((int64_t)(p->total_q / 64 + p->batch) * p->heads_q >= (1 << 24))
    return fail(DASH_ERR_UNSUPPORTED, "(total_q / 64 + batch) * heads_q must be below 2^24");
  if ((int64_t)(p->total_k / 128 + p->batch) * p->heads_q >= (1 << 30))
    return fail(DASH_ERR_UNSUPPORTED, "(total_k / 128 + batch) * heads_q must be below 2^30");
  *work = p->batch > 0 && (p->total_q > 0 || p->total_k > 0);
  if (!*work) return DASH_OK;
  if (!p->cu_q) return fail(DASH_ERR_INVALID_ARG, "null cu_q");
  if (!p->cu_k && p->total_k != p->total_q) return fail(DASH_ERR_INVALID_ARG, "without cu_k, total_k must be total_q");
  const int64_t nq = p->total_q, nk = p->total_k;
  if (nq && (rc = check_tensor("q", q, nq, p->heads_q, p->d, p->q_row_stride, p->q_head_stride, 8, false))) return rc;
  if (nk && (rc = check_tensor("k", k, nk, p->heads_kv, p->d, p->k_row_stride, p->k_head_stride, 8, false))) return rc;
  if (nk && (rc = check_tensor("v", v, nk, p->heads_kv, p->d, p->v_row_stride, p->v_head_stride, 8, false))) return rc;
  if (nq && (rc = check_tensor("o", o, nq, p->heads_q, p->d, p->o_row_stride, p->o_head_stride, 8, o_written))) return rc;
  if (nq && !lse) return fail(DASH_ERR_INVALID_ARG, "lse: null pointer");
  return DASH_OK;
}

// The stride of a single row means nothing (a broadcast's is 0), but the kernels find the
// end of a tensor's rows by it.
int64_t row_stride(int64_t stride, int rows, int d) { return rows > 1 ? stride : d; }

dash::PackedArgs packed_args(const dash_packed_t* p, float scale, const void* q, const void* k, const void* v, void* o, float* lse) {
  const auto row_q = [&](int64_t s) { return row_stride(s, p->total_q, p->d); };
  const auto row_k = [&](int64_t s) { return row_stride(s, p->total_k, p->d); };
  return {q, k, v, o, lse, p->cu_q, p->cu_k ? p->cu_k : p->cu_q, p->batch, p->heads_q, p->heads_kv, p->total_q, p->total_k,
          p->causal ? 1 : 0, scale, {row_q(p->q_row_stride), p->q_head_stride}, {row_k(p->k_row_stride), p->k_head_stride},
          {row_k(p->v_row_stride), p->v_head_stride}, {row_q(p->o_row_stride), p->o_head_stride}, 1, nullptr, nullptr};
}

struct FwdLayout {
  int splits;
  size_t part_o, part_l, total;
};
FwdLayout fwd_layout(int batch, int total_q, int total_k, int heads_q, int d, int causal) {
  FwdLayout L;
  L.splits = batch > 0 ? dash::packed_splits(d, total_q, total_k, batch, heads_q, causal) : 1;
  const size_t rows = dash::packed_part_rows(total_q, batch, heads_q, L.splits);
  L.part_o = 0;
  L.part_l = rows * d * sizeof(float);
  L.total = L.part_l + align256(rows * 2 * sizeof(float));
  return L;
}

int attn_packed_fwd(const dash_packed_t* p, const void* q, const void* k, const void* v, void* o, float* lse, void* workspace,
                    size_t ws_bytes, void* stream) {
  bool work = false;
  float scale = 0.f;
  int rc = check_packed(p, &scale, q, k, v, o, true, lse, &work);
  if (rc || !work || p->total_q == 0) return rc;
  dash::PackedArgs a = packed_args(p, scale, q, k, v, o, lse);
  const FwdLayout L = fwd_layout(p->batch, p->total_q, p->total_k, p->heads_q, p->d, a.causal);
  if (L.splits > 1 && workspace) {
    if (ws_bytes < dash_packed_fwd_workspace_size(p->batch, p->total_q, p->total_k, p->heads_q, p->heads_kv, p->d))
      return fail(DASH_ERR_INVALID_ARG, "workspace smaller than dash_packed_fwd_workspace_size()");
    if (((uintptr_t)workspace & 255) != 0) return fail(DASH_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    a.splits = L.splits;
    a.part_o = (float*)((char*)workspace + L.part_o);
    a.part_l = (float*)((char*)workspace + L.part_l);
  }
  DeviceInfo di;
  if ((rc = device_info(&di))) return rc;
  const hipError_t e = dash::launch_packed_fwd(a, p->d, (hipStream_t)stream);
  return e == hipSuccess ? DASH_OK : hip_fail(e, "packed forward launch");
}

struct PackedLayout {
  int bc, slots_q, slots_k, split_room;
  size_t ctrl, dqacc, dvec, lse2, counters, order, dkv_part, total;
};
// ctrl first, where dash_bwd_check looks; bc: rows of the KV tiles
PackedLayout packed_layout(int batch, int total_q, int total_k, int heads_q, int heads_kv, int d, int bc) {
  PackedLayout L;
  L.bc = bc;
  L.slots_q = total_q / dash::kBlockRows + batch;
  L.slots_k = total_k / L.bc + batch;
  L.split_room = heads_q == heads_kv ? 0 : dash::split_room(L.slots_k, heads_q);
  const size_t blocks = (size_t)L.slots_q * heads_q, rows = (size_t)total_q * heads_q;
  size_t off = 0;
  L.ctrl = off;
  off += dash::kCtrlBytes;
  L.dqacc = off;
  off += align256(blocks * dash::kBlockRows * d * sizeof(float));
  L.dvec = off;
  off += align256(rows * sizeof(float));
  L.lse2 = off;
  off += align256(rows * sizeof(float));
  L.counters = off;
  off += align256(blocks * dash::kCtrStride * sizeof(int));
  L.order = off;
  off += align256((size_t)L.slots_k * 2 * sizeof(int));
  L.dkv_part = off;
  off += (size_t)L.split_room * 2 * L.bc * d * sizeof(float);
  L.total = off;
  return L;
}

int attn_packed_bwd(const dash_packed_t* p, const void* q, const void* k, const void* v, const void* o, const void* dO,
                    const float* lse, void* dq, void* dk, void* dv, void* workspace, size_t ws_bytes, int* status, void* stream) {
  bool work = false;
  float scale = 0.f;
  int rc = check_packed(p, &scale, q, k, v, o, false, lse, &work);
  if (rc) return rc;
  if (!work) {
    int* flag = workspace && ws_bytes >= dash::kCtrlBytes ? (int*)workspace + dash::kCtrlError : nullptr;
    return dash::api::clear_flags(flag, status, stream);
  }
  const int64_t nq = p->total_q, nk = p->total_k;
  if (nq && (rc = check_tensor("dO", dO, nq, p->heads_q, p->d, p->do_row_stride, p->do_head_stride, 8, false))) return rc;
  if (nq && (rc = check_tensor("dq", dq, nq, p->heads_q, p->d, p->dq_row_stride, p->dq_head_stride, 8, true))) return rc;
  if (nk && (rc = check_tensor("dk", dk, nk, p->heads_kv, p->d, p->dk_row_stride, p->dk_head_stride, 8, true))) return rc;
  if (nk && (rc = check_tensor("dv", dv, nk, p->heads_kv, p->d, p->dv_row_stride, p->dv_head_stride, 8, true))) return rc;
  const PackedLayout L = packed_layout(p->batch, p->total_q, p->total_k, p->heads_q, p->heads_kv, p->d,
                                       dash::packed_tile_rows(p->d, p->total_k, p->batch, p->heads_q, p->causal != 0));
  if (!workspace || ws_bytes < dash_packed_workspace_size(p->batch, p->total_q, p->total_k, p->heads_q, p->heads_kv, p->d))
    return fail(DASH_ERR_INVALID_ARG, "workspace missing or smaller than dash_packed_workspace_size()");
  if (((uintptr_t)workspace & 255) != 0) return fail(DASH_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  DeviceInfo di;
  if ((rc = device_info(&di))) return rc;
  char* ws = (char*)workspace;
  dash::PackedBwdArgs a{};
  a.p = packed_args(p, scale, q, k, v, const_cast<void*>(o), const_cast<float*>(lse));
  a.q = q;
  a.k = k;
  a.v = v;
  a.o = o;
  a.dO = dO;
  a.lse = lse;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  a.dqacc = (float*)(ws + L.dqacc);
  a.dvec = (float*)(ws + L.dvec);
  a.lse2 = (float*)(ws + L.lse2);
  a.counters = (int*)(ws + L.counters);
  a.ctrl = (int*)(ws + L.ctrl);
  a.order = (int*)(ws + L.order);
  a.bh = 1;
  a.nblk = L.slots_q * p->heads_q;  // counters
  a.scale = scale;
  a.spin_limit = 1 << 24;
  a.status = status;
  a.dos = {row_stride(p->do_row_stride, p->total_q, p->d), p->do_head_stride};
  a.dqs = {row_stride(p->dq_row_stride, p->total_q, p->d), p->dq_head_stride};
  a.dks = {row_stride(p->dk_row_stride, p->total_k, p->d), p->dk_head_stride};
  a.dvs = {row_stride(p->dv_row_stride, p->total_k, p->d), p->dv_head_stride};
  a.bc = L.bc;
  a.slots_q = L.slots_q;
  a.slots_k = L.slots_k;
  a.split_room = L.split_room;
  a.dkv_part = (float*)(ws + L.dkv_part);
  const hipError_t e = dash::launch_packed_bwd(a, p->d, di.cus, (hipStream_t)stream);
  return e == hipSuccess ? DASH_OK : hip_fail(e, "packed backward launch");
}

// no C++ exception (an error message that finds no memory) crosses the interface
template <typename F>
int guarded(F&& f) {
  try {
    return f();
  } catch (...) {
    return DASH_ERR_HIP;
  }
}

}  // namespace

extern "C" {

int dash_kv_append(const dash_paged_cache_t* cache, const dash_append_t* x, int* status, void* stream) {
  return guarded([&] { return kv_append(cache, x, status, stream); });
}

size_t dash_decode_workspace_size(int batch, int heads_q, int heads_kv, int d, int page_size, int table_width) {
  size_t bytes = 0;
  guarded([&] {
    if (check_heads(batch, heads_q, heads_kv, d) == DASH_OK && page_size >= 16 && page_size % 16 == 0 && page_size <= 65536 &&
        table_width >= 0 && (int64_t)table_width * page_size <= dash::kMaxKeys)
      bytes = decode_layout(batch, heads_q, heads_kv, d, table_width * page_size).total;
    return 0;
  });
  return bytes;
}

int dash_attn_decode(const dash_paged_cache_t* cache, const void* q, int64_t q_row_stride, int64_t q_head_stride, void* o,
                     int64_t o_row_stride, int64_t o_head_stride, float* lse, float scale, void* workspace, size_t ws_bytes,
                     int* status, void* stream) {
  return guarded([&] {
    return attn_decode(cache, q, q_row_stride, q_head_stride, o, o_row_stride, o_head_stride, lse, scale, workspace, ws_bytes,
                       status, stream);
  });
}

size_t dash_packed_fwd_workspace_size(int batch, int total_q, int total_k, int heads_q, int heads_kv, int d) {
  size_t bytes = 0;
  guarded([&] {
    if (check_heads(batch, heads_q, heads_kv, d) == DASH_OK && total_q >= 0 && total_k >= 0 && total_q <= kMaxRows && total_k <= kMaxRows)
      bytes = std::max(fwd_layout(batch, total_q, total_k, heads_q, d, 0).total, fwd_layout(batch, total_q, total_k, heads_q, d, 1).total);
    return 0;
  });
  return bytes;
}

int dash_attn_packed_fwd(const dash_packed_t* p, const void* q, const void* k, const void* v, void* o, float* lse, void* workspace,
                         size_t ws_bytes, void* stream) {
  return guarded([&] { return attn_packed_fwd(p, q, k, v, o, lse, workspace, ws_bytes, stream); });
}

size_t dash_packed_workspace_size(int batch, int total_q, int total_k, int heads_q, int heads_kv, int d) {
  size_t bytes = 0;
  guarded([&] {
    if (check_heads(batch, heads_q, heads_kv, d) == DASH_OK && total_q >= 0 && total_k >= 0 && total_q <= kMaxRows && total_k <= kMaxRows)
      for (int causal = 0; causal < 2; ++causal)  // either mask
        bytes = std::max(bytes, packed_layout(batch, total_q, total_k, heads_q, heads_kv, d,
                                              dash::packed_tile_rows(d, total_k, batch, heads_q, causal)).total);
    return 0;
  });
  return bytes;
}

int dash_attn_packed_bwd(const dash_packed_t* p, const void* q, const void* k, const void* v, const void* o, const void* dO,
                         const float* lse, void* dq, void* dk, void* dv, void* workspace, size_t ws_bytes, int* status, void* stream) {
  return guarded([&] { return attn_packed_bwd(p, q, k, v, o, dO, lse, dq, dk, dv, workspace, ws_bytes, status, stream); });
}

}  // extern "C"
