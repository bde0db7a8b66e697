// ops.h -- interface between the C ABI layer and the kernels of the
// variable-length operators: the paged key-value cache (append, one-token
// attention) and attention over packed sequences.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"

namespace dash {

// strides in elements
struct Strides {
  int64_t row, head;
};

// ---------------------------------------------------------------- paged cache
struct CacheArgs {
  int batch, heads_q, heads_kv, d;
  int pages, page_size, table_width;
  int e4m3;  // element type: 0 bf16, 1 e4m3
  void* k;
  void* v;
  int64_t k_page, k_head, k_row, v_page, v_head, v_row;  // strides in elements
  const int32_t* table;
  int64_t table_stride;
  const int32_t* lens;
  const float* k_scale;  // null: 1
  const float* v_scale;
  int* status;  // null, or set to 1 by a bad page or length
};

struct AppendArgs {
  CacheArgs c;
  int tokens;
  const int32_t* cu;
  const void *k, *v, *q;
  void *q_out, *k_out;
  Strides ks, vs, qs, qos, kos;
  const float* inv_freq;
  int rotary, interleaved;
};
hipError_t launch_kv_append(const AppendArgs& a, hipStream_t stream);

struct DecodeArgs {
  CacheArgs c;
  const void* q;
  void* o;
  float* lse;  // null, or [batch][heads_q]
  Strides qs, os;  // row: from sequence to sequence
  float scale;
  int workers;    // chunks aimed at (decode_workers)
  int slots;      // chunks at most (decode_slots)
  float* part_o;  // [slots][heads_q][d]
  float* part_m;  // [slots][heads_q][2]: maximum (log2 domain), sum
  int* base;      // [batch][2]: first slot of a sequence, its chunks
};
int decode_workers(int heads_q, int heads_kv);
int decode_slots(int batch, int heads_q, int heads_kv, int table_tokens);
hipError_t launch_decode(const DecodeArgs& a, hipStream_t stream);

// ---------------------------------------------------------------- packed sequences
struct PackedArgs {
  const void *q, *k, *v;
  void* o;
  float* lse;  // [heads_q][total_q]
  const int32_t *cu_q, *cu_k;
  int batch, heads_q, heads_kv, total_q, total_k, causal;
  float scale;
  Strides qs, ks, vs, os;
};
hipError_t launch_packed_fwd(const PackedArgs& a, int d, hipStream_t stream);

}  // namespace dash
