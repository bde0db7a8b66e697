// packed_chain.h -- one KV tile's chain over a packed sequence, as the backward main
// kernels run it: buffer resources and offsets of its tensors.  64-bit bases at a
// tile's or block's first row, 32-bit offsets inside; bounds end at the
// sequence's last row, so that rows past it read zeros and are not written.
#pragma once
#include "common.h"
#include "kernels.h"
#include "ops.h"
#include "packed_order.h"
#include "paged.h"

namespace dash {

// a 64-row query block of one query head of the group
struct PackedBlk {
  int pb, h;
  int x;  // number of its accumulator and ordering counter
};

struct NoChain {
  template <typename A>
  __device__ explicit NoChain(const A&) {}
};

template <int D, int BC>
struct PackedChain {
  const PackedBwdArgs& a;
  SeqGeom sg;
  int j, hk, G;
  int place;                  // the tile's place in the order
  int h0, hn;                 // the chain's query heads of the group: all, or a part's of a split tile
  bool split;
  int part;                   // the part's number
  int qstart, kstart, slot0;  // slot0: the sequence's first accumulator slot
  int pb0;                    // the chain's last (lowest) block

  __device__ explicit PackedChain(const PackedBwdArgs& args) : a(args) {}
  // the work item's chain; false: no such chain (an order table that cu does not match)
  __device__ bool init(int item) {
    G = a.p.heads_q / a.p.heads_kv;
    const int n_long = __builtin_amdgcn_readfirstlane(a.ctrl[kCtrlLong]);
    const int per = __builtin_amdgcn_readfirstlane(a.ctrl[kCtrlHeads]), parts = split_parts(G, per);
    const int of_long = n_long * a.p.heads_kv * parts;
    split = item < of_long;
    h0 = 0, hn = G;
    part = item;
    if (split) {
      place = item / (a.p.heads_kv * parts);
      const int x = item - place * (a.p.heads_kv * parts);
      hk = x / parts;
      h0 = (x - hk * parts) * per;
      hn = h0 + per < G ? per : G - h0;
    } else {
      place = (item - of_long) / a.p.heads_kv;
      hk = item - of_long - place * a.p.heads_kv;
      place += n_long;
    }
    const int s = __builtin_amdgcn_readfirstlane(a.order[2 * place]);
    j = __builtin_amdgcn_readfirstlane(a.order[2 * place + 1]);
    if ((unsigned)s >= (unsigned)a.p.batch) return false;
    const Span q = span_of(a.p.cu_q, s, a.p.total_q), k = span_of(a.p.cu_k, s, a.p.total_k);
    qstart = __builtin_amdgcn_readfirstlane(q.start);
    kstart = __builtin_amdgcn_readfirstlane(k.start);
    sg = SeqGeom{__builtin_amdgcn_readfirstlane(q.len), __builtin_amdgcn_readfirstlane(k.len), a.p.causal != 0, BC};
    slot0 = qstart / kBlockRows + s;
    if ((unsigned)j >= (unsigned)sg.tiles()) return false;
    pb0 = sg.first_block(j);
    return true;
  }
  // items of the call
  __device__ static int items(const PackedBwdArgs& a) {
    const int n = a.ctrl[kCtrlItems], n_long = a.ctrl[kCtrlLong];
    const int parts = split_parts(a.p.heads_q / a.p.heads_kv, a.ctrl[kCtrlHeads]);
    return (n_long * parts + n - n_long) * a.p.heads_kv;
  }
  __device__ int steps() const { return (sg.blocks() - pb0) * hn; }
  __device__ PackedBlk first() const {
    const int pb = sg.blocks() - 1, h = h0 + hn - 1;
    return {pb, h, (slot0 + pb) * a.p.heads_q + hk * G + h};
  }
  __device__ PackedBlk next(PackedBlk b) const {
    return b.h > h0 ? PackedBlk{b.pb, b.h - 1, b.x - 1} : PackedBlk{b.pb - 1, h0 + hn - 1, b.x - a.p.heads_q + hn - 1};
  }
  // a part's fp32 partials: dK (0) or dV (1), BC rows of D
  __device__ __amdgpu_buffer_rsrc_t partial(int which) const {
    return make_rsrc(a.dkv_part + ((size_t)part * 2 + which) * (BC * D), BC * D * 4);
  }
  __device__ bool last(PackedBlk b) const { return sg.last_tile(b.pb) == j; }

  __device__ __amdgpu_buffer_rsrc_t acc(PackedBlk b, bool on = true) const {
    return make_rsrc(a.dqacc + (size_t)b.x * (kBlockRows * D), on ? kBlockRows * D * 4 : 0);
  }

  __device__ static uint32_t at(const Strides& s, int row, int col) { return (uint32_t)row * (uint32_t)s.row * 2 + (uint32_t)col * 2; }
  __device__ __amdgpu_buffer_rsrc_t block(const void* p, const Strides& s, PackedBlk b) const {
    return strided_rows<D>(p, (int64_t)qstart + b.pb * kBlockRows, s, hk * G + b.h, sg.nq - b.pb * kBlockRows, kBlockRows);
  }
  __device__ __amdgpu_buffer_rsrc_t q(PackedBlk b) const { return block(a.q, a.p.qs, b); }
  __device__ __amdgpu_buffer_rsrc_t dO(PackedBlk b) const { return block(a.dO, a.dos, b); }
  __device__ __amdgpu_buffer_rsrc_t dq(PackedBlk b) const { return block(a.dq, a.dqs, b); }
  // one fp32 per row of the block: L * log2(e), D
  __device__ __amdgpu_buffer_rsrc_t vec(const float* p, PackedBlk b) const {
    const int n = sg.nq - b.pb * kBlockRows;
    return make_rsrc(p + (int64_t)(hk * G + b.h) * a.p.total_q + qstart + b.pb * kBlockRows, (uint32_t)(n < kBlockRows ? n : kBlockRows) * 4);
  }
  __device__ __amdgpu_buffer_rsrc_t tile(const void* p, const Strides& s) const {
    return strided_rows<D>(p, (int64_t)kstart + j * BC, s, hk, sg.nk - j * BC, BC);
  }
};

}  // namespace dash
