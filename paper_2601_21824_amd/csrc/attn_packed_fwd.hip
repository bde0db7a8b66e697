// attn_packed_fwd.hip -- the forward over packed sequences of different lengths, with
// grouped heads and strided tensors: the kernel of fwd_main.h on another view of
// its rows.
//
// A workgroup takes 128 query rows of one sequence and head.  The slots of 128
// rows are found from cu_q on the device (first_slot), so that nothing has to be
// prepared and a captured call follows its offsets; at most `batch` slots a head are empty
// and end at once.  Tensors are addressed from a tile's first row on: 64-bit
// bases, 32-bit offsets inside a tile.  Buffer bounds end at the sequence's last
// row, so that a tile that reaches past it reads zeros, never a neighbour.
//
// Calls with few rows for the GPU split the keys as well (packed_splits): a
// workgroup takes an equal run of the tiles that its rows see and leaves, of those keys
// alone and in fp32, O and each row's maximum m_i (log2 domain) and sum s_i; join_kernel adds
// the runs in order, weighted by s_i 2^(m_i - m).  (Not by exp(L_i - L): an L far from 0
// holds log s_i in few bits or none.)
//
// Bound, as the dense forward, by the issue of the MFMAs and of the softmax beside them.
// Measured, causal, 32 heads over 8 of 128: one sequence of 8192 550-615 us, 890-1000 TFLOP/s; 12
// of 8192 in all (1 to 1761) 119-138 us, whose diagonal tiles are half masked.
#include "fwd_main.h"
#include "ops.h"
#include "paged.h"

namespace dash {
namespace {

constexpr int kRows = 128;  // query rows of a workgroup

// A workgroup's run of keys: the tiles of KT keys that its rows see, cut into n equal
// runs of kMinRun keys at least (half of that where they are cut unevenly: more than
// a workgroup's rows, so that under a causal mask every row sees a key of every run).
constexpr int kMinRun = 512;
struct Run {
  int first, keys, n;  // its first key, its keys (end: of all runs), the runs
};
template <int KT>
__device__ inline Run run_of(int kv_end, int splits, int i) {
  const int tiles = (kv_end + KT - 1) / KT;
  int n = kv_end / kMinRun;
  n = n < splits ? n : splits;
  n = n > 1 ? n : 1;
  const int a = (int)((int64_t)tiles * i / n), b = (int)((int64_t)tiles * (i + 1) / n);
  return {a * KT, (b * KT < kv_end ? b * KT : kv_end) - a * KT, n};
}

// The rows of a slot: first row q0 and their number (<= 0: none), the keys that they
// see at most.
struct Rows {
  int q0, n, kv_end;
  Span q, k;
};
__device__ inline Rows rows_of(const PackedArgs& a, int slot, int l) {
  Rows r;
  const int s = __builtin_amdgcn_readfirstlane(
      find_last(a.batch, slot, l, [&](int x) { return first_slot(a.cu_q, x, a.total_q, kRows); }));
  r.q = span_of(a.cu_q, s, a.total_q);
  r.k = span_of(a.cu_k, s, a.total_k);
  r.q0 = (slot - first_slot(a.cu_q, s, a.total_q, kRows)) * kRows;
  r.n = r.q0 < 0 ? 0 : r.q.len - r.q0 < kRows ? r.q.len - r.q0 : kRows;
  r.kv_end = r.k.len;
  if (a.causal) {
    const int end = r.q0 + kRows + r.k.len - r.q.len;
    r.kv_end = end < r.kv_end ? end : r.kv_end;
  }
  return r;
}

template <int D>
struct PackedView {
  static constexpr bool kPacked = true;
  const PackedArgs& a;
  int h, hk, q0;
  int nq, nk, off_;  // nk, off_: as the run counts its keys
  int qstart, kstart;
  int64_t part;  // number of the run's partial result; -1: the rows have one run, which is the result
  __device__ int off() const { return off_; }
  __device__ __amdgpu_buffer_rsrc_t q() const { return strided_rows<D>(a.q, (int64_t)qstart + q0, a.qs, h, nq - q0, kRows); }
  __device__ __amdgpu_buffer_rsrc_t k(int k0) const { return strided_rows<D>(a.k, (int64_t)kstart + k0, a.ks, hk, nk - k0, 64); }
  __device__ __amdgpu_buffer_rsrc_t v(int k0) const { return strided_rows<D>(a.v, (int64_t)kstart + k0, a.vs, hk, nk - k0, 64); }
  __device__ uint32_t q_at(int row, int col) const { return (uint32_t)(row - q0) * (uint32_t)a.qs.row * 2 + col * 2; }
  __device__ uint32_t k_at(int, int row, int col) const { return (uint32_t)row * (uint32_t)a.ks.row * 2 + col * 2; }
  __device__ uint32_t v_at(int, int row, int col) const { return (uint32_t)row * (uint32_t)a.vs.row * 2 + col * 2; }
  __device__ __amdgpu_buffer_rsrc_t o() const {
    if (part >= 0) return make_rsrc(a.part_o + part * (kRows * D), kRows * D * 4);
    return strided_rows<D>(a.o, (int64_t)qstart + q0, a.os, h, nq - q0, kRows);
  }
  __device__ __amdgpu_buffer_rsrc_t lse() const {
    if (part >= 0) return make_rsrc(a.part_l + part * (2 * kRows), kRows * 8);
    const int n = nq - q0;
    return make_rsrc(a.lse + (int64_t)h * a.total_q + qstart + q0, (uint32_t)(n < kRows ? n : kRows) * 4);
  }
  __device__ uint32_t l_at(int row) const { return (uint32_t)(row - q0) * 4; }
  __device__ void put_l(__amdgpu_buffer_rsrc_t r, int row, float m, float sum) const {
    if (part >= 0) st8(r, (uint32_t)(row - q0) * 8, u32x2{__builtin_bit_cast(unsigned, m), __builtin_bit_cast(unsigned, sum)});
    else st4f(r, l_at(row), (m + __log2f(sum)) * kLn2);
  }
  __device__ void put_o(__amdgpu_buffer_rsrc_t r, int row, int col, float a0, float a1, float a2, float a3) const {
    if (part >= 0) st16(r, (uint32_t)((row - q0) * D + col) * 4, __builtin_bit_cast(u32x4, f32x4{a0, a1, a2, a3}));
    else st8(r, (uint32_t)(row - q0) * (uint32_t)a.os.row * 2 + col * 2, u32x2{pack_bf16(a0, a1), pack_bf16(a2, a3)});
  }
};

template <int D, int WPS>
__global__ __launch_bounds__(256, WPS) void packed_fwd_kernel(PackedArgs a) {
  constexpr int KT = D == 256 ? 32 : 64;
  const int tid = threadIdx.x;
  // Workgroup -> (K/V head, run of keys, slot, query head of the group).  Consecutive
  // workgroups go to the 8 XCDs in turn; each XCD takes a contiguous run, so that
  // the workgroups sharing an XCD's L2 read the same K and V.
  const int G = a.heads_q / a.heads_kv;
  const int slots = a.total_q / kRows + a.batch;
  const int items = slots * a.heads_q * a.splits;
  const int per = (items + 7) >> 3;
  const int item = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || item >= items) return;
  const int hk = item / (slots * G * a.splits), in = item % (slots * G * a.splits);
  const int split = in / (slots * G);
  int slot = in / G % slots;
  // causal: a sequence's longest blocks (last rows) first; where a run ends inside a
  // head, from both ends in turn, so that every run holds like work.  (Longest first over
  // all sequences, found by a search, costs more than the tail that it saves: 16 sequences of
  // 512 67 -> 73 us, 12 of 8192 in all 111 -> 112.)
  if (a.causal) slot = (a.heads_kv & 7) == 0 ? slots - 1 - slot : (slot & 1) ? slot >> 1 : slots - 1 - (slot >> 1);
  const Rows r = rows_of(a, slot, tid & 63);
  if (r.n <= 0) return;
  const int h = hk * G + in % G;
  Run run = {0, 0, 1};
  if (r.kv_end > 0) run = run_of<KT>(r.kv_end, a.splits, split);
  if (split >= run.n) return;
  const int64_t part = run.n > 1 ? ((int64_t)slot * a.heads_q + h) * a.splits + split : -1;
  const PackedView<D> view{a, h, hk, r.q0, r.q.len, run.keys, r.k.len - r.q.len - run.first, r.q.start, r.k.start + run.first, part};
  if (r.kv_end <= 0) {  // no row sees a key
    const auto ro = view.o(), rl = view.lse();
    for (int e = tid; e < kRows * (D / 4); e += 256) view.put_o(ro, r.q0 + e / (D / 4), 4 * (e % (D / 4)), 0.f, 0.f, 0.f, 0.f);
    if (tid < kRows) st4f(rl, view.l_at(r.q0 + tid), -INFINITY);
    return;
  }
  attn_fwd_rows<D, 1>(view, a.causal, a.scale, r.q0);
}

// The runs of a slot's rows, in order: one workgroup per two passes of rows and head, D / 4
// lanes a row: 1301 and 199 rows of 8 heads of 256 in two runs 7.6 us (8 passes a workgroup, one
// after the other, 12.9).
template <int D>
__global__ __launch_bounds__(256) void join_kernel(PackedArgs a) {
  constexpr int KT = D == 256 ? 32 : 64, RPP = 1024 / D, RWG = 2 * RPP;  // rows a pass, rows a workgroup
  const int tid = threadIdx.x;
  const int x = (int)blockIdx.x / (kRows / RWG), r0 = (int)blockIdx.x % (kRows / RWG) * RWG;
  const int slot = x / a.heads_q, h = x % a.heads_q;
  const Rows r = rows_of(a, slot, tid & 63);
  if (r0 >= r.n || r.kv_end <= 0) return;
  const int n = run_of<KT>(r.kv_end, a.splits, 0).n;
  if (n == 1) return;  // the result is there
  const int64_t part = ((int64_t)slot * a.heads_q + h) * a.splits;
  const int c = tid % (D / 4) * 4;
  for (int row = r0 + tid / (D / 4); row < r0 + RWG && row < r.n; row += RPP) {
    const float2* stat = (const float2*)a.part_l;  // m, sum
    float top = -INFINITY;
    for (int i = 0; i < n; ++i) top = fmaxf(top, stat[(part + i) * kRows + row].x);
    const float at = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < n; ++i) {
      const float2 x = stat[(part + i) * kRows + row];
      const float w = x.y * __builtin_amdgcn_exp2f(x.x - at);
      sum += w;
      o += w * *(const f32x4*)(a.part_o + (part + i) * (kRows * D) + row * D + c);
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;  // (nothing but -inf: O 0)
    *(u32x2*)((__bf16*)a.o + ((int64_t)r.q.start + r.q0 + row) * a.os.row + h * a.os.head + c) =
        u32x2{pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
    if (c == 0) a.lse[(int64_t)h * a.total_q + r.q.start + r.q0 + row] = sum == 0.f ? -INFINITY : (top + __log2f(sum)) * kLn2;
  }
}

template <int D, int WPS>
void launch(const PackedArgs& a, hipStream_t stream) {
  const long blocks = (long)(a.total_q / kRows + a.batch) * a.heads_q, items = blocks * a.splits;
  hipLaunchKernelGGL((packed_fwd_kernel<D, WPS>), dim3((unsigned)((items + 7) / 8 * 8)), dim3(256), 0, stream, a);
  if (a.splits > 1) hipLaunchKernelGGL((join_kernel<D>), dim3((unsigned)(blocks * (kRows / (2048 / D)))), dim3(256), 0, stream, a);
}

}  // namespace

// Runs of keys a workgroup's rows are split into at most.  Measured (us, whole / in s
// runs): 1 query on 8192 keys, 32 heads over 8 of 128, 132 / 30 (16); 700 on 4096, 8 heads of 256,
// 152 / 92 (5); 1301 and 199 on 5397 and 4295, 8 heads of 256, 200 / 123 (2; 131 in 4, 156 in 5: the
// last round is short); causal prompts, heads of 128: 8192 4 heads 184 / 121 (4), 4096 8 heads
// 88 / 73 (4), 2048 16 heads 48 / 46 (4), but 8192 8 heads 193 / 184 and 4096 16 heads of 64
// 68 / 71 in 2; 4096 8 heads of 256 155 / 127 (2).
int packed_splits(int d, int total_q, int total_k, int batch, int heads_q, int causal) {
  // workgroups with rows: whole slots, and one at least for each sequence
  const long rows = (total_q + 127) / 128 > batch ? (total_q + 127) / 128 : batch < total_q ? batch : total_q;
  const long blocks = rows * heads_q;
  // workgroups that run at once on 256 CUs: one a CU, or two (at d = 64, where three fit, two
  // as well: the figures above were taken with this rule)
  const long fit = d == 256 ? 256 : 512;
  // with as many queries as keys a causal block's work goes from one tile to all: runs
  // for two rounds level it, where two workgroups share a CU from three runs on
  const bool triangle = causal && total_k < 2L * total_q;
  // of a sequence of the average length: the host knows no other, so that one long sequence among
  // many short ones is split less than alone, or not at all
  const long most = (long)total_k / batch / kMinRun;
  long s = blocks > 0 ? (triangle ? 2 : 1) * fit / blocks : 1;
  s = s < most ? s : most;
  if (triangle && d < 256 && s < 3) s = 1;
  // Partial results have room for every slot: with far more sequences than queries (most of
  // them empty) for nearly nothing but empty ones, so that their number is bounded (1.1 GB at d = 256;
  // up to 2048 where batch <= total_q)
  const long room = 8192 / ((total_q / 128 + (long)batch) * heads_q);
  s = s < room ? s : room;
  return (int)(s < 1 ? 1 : s > 64 ? 64 : s);
}
size_t packed_part_rows(int total_q, int batch, int heads_q, int splits) {
  return splits > 1 ? (size_t)(total_q / 128 + batch) * heads_q * splits * 128 : 0;
}

hipError_t launch_packed_fwd(const PackedArgs& a, int d, hipStream_t stream) {
  if (d == 64) launch<64, 3>(a, stream);
  else if (d == 128) launch<128, 2>(a, stream);
  else launch<256, 1>(a, stream);
  return hipGetLastError();
}

}  // namespace dash
