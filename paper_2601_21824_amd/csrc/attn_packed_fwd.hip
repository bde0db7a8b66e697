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
#include "fwd_main.h"
#include "ops.h"
#include "paged.h"

namespace dash {
namespace {

template <int D, int QROWS>
struct PackedView {
  static constexpr bool kPacked = true;
  const PackedArgs& a;
  int h, hk, q0;
  int nq, nk;
  int qstart, kstart;
  __device__ int off() const { return nk - nq; }
  // a resource over at most `most` rows of the n behind row r0
  __device__ static __amdgpu_buffer_rsrc_t rows(const void* p, int64_t first, const Strides& s, int head, int n, int most) {
    const int r = n < most ? n : most;
    const uint32_t bytes = r > 0 ? (uint32_t)(r - 1) * (uint32_t)s.row * 2 + D * 2 : 0;
    return make_rsrc((const __bf16*)p + first * s.row + head * s.head, bytes);
  }
  __device__ __amdgpu_buffer_rsrc_t q() const { return rows(a.q, (int64_t)qstart + q0, a.qs, h, nq - q0, QROWS); }
  __device__ __amdgpu_buffer_rsrc_t o() const { return rows(a.o, (int64_t)qstart + q0, a.os, h, nq - q0, QROWS); }
  __device__ __amdgpu_buffer_rsrc_t k(int k0) const { return rows(a.k, (int64_t)kstart + k0, a.ks, hk, nk - k0, 64); }
  __device__ __amdgpu_buffer_rsrc_t v(int k0) const { return rows(a.v, (int64_t)kstart + k0, a.vs, hk, nk - k0, 64); }
  __device__ __amdgpu_buffer_rsrc_t lse() const { return make_rsrc(a.lse + (int64_t)h * a.total_q + qstart, (uint32_t)nq * 4); }
  __device__ uint32_t q_at(int row, int col) const { return (uint32_t)(row - q0) * (uint32_t)a.qs.row * 2 + col * 2; }
  __device__ uint32_t o_at(int row, int col) const { return (uint32_t)(row - q0) * (uint32_t)a.os.row * 2 + col * 2; }
  __device__ uint32_t k_at(int, int row, int col) const { return (uint32_t)row * (uint32_t)a.ks.row * 2 + col * 2; }
  __device__ uint32_t v_at(int, int row, int col) const { return (uint32_t)row * (uint32_t)a.vs.row * 2 + col * 2; }
};

template <int D, int QG, int WPS>
__global__ __launch_bounds__(256, WPS) void packed_fwd_kernel(PackedArgs a) {
  constexpr int QROWS = 128 * QG;
  const int tid = threadIdx.x;
  // Workgroup -> (K/V head, slot, query head of the group).  Consecutive
  // workgroups go to the 8 XCDs in turn; each XCD takes a contiguous run, so that
  // the workgroups sharing an XCD's L2 read the same K and V.
  const int G = a.heads_q / a.heads_kv;
  const int slots = a.total_q / QROWS + a.batch;
  const int items = slots * a.heads_q;
  const int per = (items + 7) >> 3;
  const int item = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || item >= items) return;
  const int hk = item / (slots * G), in = item % (slots * G);
  int slot = in / G;
  // causal: a sequence's longest blocks (last rows) first; where a run ends inside a
  // head, from both ends in turn, so that every run holds like work
  if (a.causal) slot = (a.heads_kv & 7) == 0 ? slots - 1 - slot : (slot & 1) ? slot >> 1 : slots - 1 - (slot >> 1);
  const int s = __builtin_amdgcn_readfirstlane(
      find_last(a.batch, slot, tid & 63, [&](int x) { return first_slot(a.cu_q, x, a.total_q, QROWS); }));
  const Span sq = span_of(a.cu_q, s, a.total_q), sk = span_of(a.cu_k, s, a.total_k);
  const int q0 = (slot - first_slot(a.cu_q, s, a.total_q, QROWS)) * QROWS;
  if (q0 < 0 || q0 >= sq.len) return;
  const PackedView<D, QROWS> view{a, hk * G + in % G, hk, q0, sq.len, sk.len, sq.start, sk.start};
  if (sk.len == 0 || (a.causal && q0 + QROWS + view.off() <= 0)) {  // no row sees a key
    const auto ro = view.o(), rl = view.lse();
    for (int e = tid; e < QROWS * (D / 8); e += 256) st16(ro, view.o_at(q0 + e / (D / 8), 8 * (e % (D / 8))), u32x4{0, 0, 0, 0});
    if (tid < QROWS) st4f(rl, (uint32_t)(q0 + tid) * 4, -INFINITY);
    return;
  }
  attn_fwd_rows<D, QG>(view, a.causal, a.scale, q0);
}

template <int D, int QG, int WPS>
void launch(const PackedArgs& a, hipStream_t stream) {
  const long items = (long)(a.total_q / (128 * QG) + a.batch) * a.heads_q;
  hipLaunchKernelGGL((packed_fwd_kernel<D, QG, WPS>), dim3((unsigned)((items + 7) / 8 * 8)), dim3(256), 0, stream, a);
}

}  // namespace

hipError_t launch_packed_fwd(const PackedArgs& a, int d, hipStream_t stream) {
  if (d == 64) launch<64, 1, 3>(a, stream);
  else if (d == 128) launch<128, 1, 2>(a, stream);
  else launch<256, 1, 1>(a, stream);
  return hipGetLastError();
}

}  // namespace dash
