// ops.h -- interface between the C ABI layer and the kernels of the
// variable-length operators: the paged key-value cache (append, one-token
// attention) and attention over packed sequences.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"

namespace dash {

// A launch takes fewer than 2^32 threads.
constexpr int64_t kMaxWaves = ((int64_t)1 << 26) - 8;  // (whole workgroups of at most eight waves)

// strides in elements
struct Strides {
  int64_t row, head;
};

// ---------------------------------------------------------------- paged cache
enum CacheType { kBf16 = 0, kE4m3 = 1, kMx8 = 2, kMx4 = 3 };
struct CacheArgs {
  int batch, heads_q, heads_kv, d;
  int pages, page_size, table_width;
  int type;  // CacheType
  void* k;
  void* v;
  int64_t k_page, k_head, k_row, v_page, v_head, v_row;  // strides in elements
  const int32_t* table;
  int64_t table_stride;
  const int32_t* lens;
  const float* k_scale;  // null: 1
  const float* v_scale;
  int* status;  // null, or set to 1 by a bad page or length
  uint8_t *k_mx, *v_mx;  // scale bytes [pages][heads_kv][page_size][d / 32]
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
// waves of the launch
int64_t append_waves(const AppendArgs& a);
hipError_t launch_kv_append(const AppendArgs& a, hipStream_t stream);

struct ReadArgs {
  CacheArgs c;
  int rows;
  const int32_t *cu, *first;  // first null: 0
  void *k_out, *v_out;        // either may be null
  Strides ks, vs;
};
// waves of the launch
int64_t read_waves(const ReadArgs& a);
hipError_t launch_kv_read(const ReadArgs& a, hipStream_t stream);

// ---------------------------------------------------------------- rotary positions
struct RotaryArgs {
  int rows, heads_q, heads_k, d, batch;
  const int32_t *positions, *cu, *start;  // positions, or cu and (null: 0) start
  const void *q, *k;
  void *q_out, *k_out;
  Strides qs, ks, qos, kos;
  const float* inv_freq;
  int rotary, interleaved, back;
  float amplitude;
  int* status;
};
// waves of the launch
int64_t rotary_waves(const RotaryArgs& a);
hipError_t launch_rotary(const RotaryArgs& a, hipStream_t stream);

// ---------------------------------------------------------------- one new token
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
  // behind a shared prefix
  const int32_t* prefix_table;
  const int32_t* prefix_len;
  int prefix_width;
  bool few;  // as in PrefixPlan
  int splits, min_run;
  float* prefix_o;  // [splits][batch][heads_q][d], each over its own sum
  float* prefix_m;  // [splits][batch][heads_q][2]
};
int decode_workers(int heads_q, int heads_kv, int d, int table_tokens);
int decode_slots(int batch, int table_tokens, int workers);
// waves of the larger launch
int64_t decode_waves(const DecodeArgs& a);
hipError_t launch_decode(const DecodeArgs& a, hipStream_t stream);
// workgroups of the chunks
int64_t decode_blocks(const DecodeArgs& a);
// attention behind a shared prefix (attn_prefix.hip)
struct PrefixPlan {
  bool few;     // 16 rows a workgroup, or 128 by the forward's kernel
  int splits;   // runs that the prefix is cut into at most,
  int min_run;  // of so many keys at least
};
PrefixPlan prefix_plan(int batch, int heads_q, int heads_kv, int d, int prefix_tokens);
int prefix_workers(int heads_q, int heads_kv);
int64_t prefix_waves(const DecodeArgs& a);
hipError_t launch_prefix(const DecodeArgs& a, hipStream_t stream);

// ---------------------------------------------------------------- packed sequences
struct PackedArgs {
  const void *q, *k, *v;
  void* o;
  float* lse;  // [heads_q][total_q]
  const int32_t *cu_q, *cu_k;
  int batch, heads_q, heads_kv, total_q, total_k, causal;
  float scale;
  Strides qs, ks, vs, os;
  // the forward's split over the keys: runs at most, and their O, maxima and sums (packed_part_rows)
  int splits;
  float* part_o;
  float* part_l;
};
int packed_splits(int d, int total_q, int total_k, int batch, int heads_q, int causal);
// rows of part_l (maximum in the log2 domain, sum), and of d columns of part_o
size_t packed_part_rows(int total_q, int batch, int heads_q, int splits);
hipError_t launch_packed_fwd(const PackedArgs& a, int d, hipStream_t stream);

// The backward's main kernels run on BwdArgs; of those, a packed call uses q, k, v, o,
// dO, lse, dq, dk, dv, dqacc, dvec and lse2 ([heads_q][total_q]), counters (one per 64-row
// slot and query head), ctrl, order (start order -> sequence, KV tile), scale,
// spin_limit and status.
struct PackedBwdArgs : BwdArgs {
  PackedArgs p;
  Strides dos, dqs, dks, dvs;
  int bc;               // rows of a KV tile
  int slots_q, slots_k;  // 64-row query slots, KV-tile slots
  int split_room;        // parts that dkv_part has room for
  float* dkv_part;       // split tiles: [place][K/V head][part][dK, dV][bc][d]
};
constexpr int kCtrlItems = 48;  // ctrl[] slot: KV tiles of all sequences
constexpr int kCtrlLong = 49;   // ctrl[] slot: how many of them, from the first on, are split
constexpr int kCtrlHeads = 50;  // ctrl[] slot: query heads of a part of those
// rows of a KV tile for a packed call
int packed_tile_rows(int d, int total_k, int batch, int heads_q, int causal);
hipError_t launch_packed_bwd(const PackedBwdArgs& a, int d, int cus, hipStream_t stream);
hipError_t launch_packed_main64(const PackedBwdArgs& a, int grid, hipStream_t stream);   // attn_bwd_d64.hip
hipError_t launch_packed_main64w(const PackedBwdArgs& a, int grid, hipStream_t stream);  // attn_bwd64w.hip
hipError_t launch_packed_main128(const PackedBwdArgs& a, int grid, hipStream_t stream);  // attn_bwd.hip
hipError_t launch_packed_mainw(const PackedBwdArgs& a, int d, int grid, hipStream_t stream);  // attn_bwdw.hip

}  // namespace dash
