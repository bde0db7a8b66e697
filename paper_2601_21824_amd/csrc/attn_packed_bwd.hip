// attn_packed_bwd.hip -- the deterministic backward over packed sequences: the kernel
// before the main kernel, and the launch sequence of a call.  The main kernels are
// bwd_main.h (128-row KV tiles at d = 64 and 128), attn_bwd64w.hip (256 rows at d = 64) and
// attn_bwdw.hip (256 rows at d = 128, 128 at d = 256) on the chains of packed_chain.h, with the ordered dQ reduction
// of the dense calls in Descending order.  As there, P and dS are rounded to bf16, the MFMAs' operand
// type, before the products that make dV, and dK and dQ (2^-8 of each term at most, as much as the
// results' own rounding); scores, dP, D, L and every sum, the split chains' partials among them,
// stay in fp32.
//
// packed_pre: D = rowsum(dO o O) and L log2(e) (+inf for a row that sees nothing, so that
// its P is 0) for every row and head, of no sequence too; the ordering counters; dQ = 0
// where no KV tile sees a 64-row block; and the KV tiles' chains in the order in which
// they start (packed_order.h): longest first over all sequences, each sequence's own in
// ascending order.  Workgroups of three kinds, by blockIdx, the rows' last.  Memory-bound,
// as bwd_pre, O and dO once: 8192 rows of 32 heads of 128 35 us, 134 MB, 3.9 TB/s (a bare copy
// 5.0).
//
// Measured, causal, 32 heads over 8: one sequence of 8192, d = 128, 1.81 ms (pre 35 us, main
// 1740, the sum of partials 34), 760 TFLOP/s of the five products, the dense Descending call
// of as many heads 1.72-1.83 ms; d = 64 1.19 ms; 12 sequences of 8192 in all (1 to 1761), d =
// 128, 421 us (40, 374, 24).  Bound, as the dense wide kernel, by the issue of one wave a SIMD.
#include "common.h"
#include "ops.h"
#include "packed_order.h"
#include "paged.h"

namespace dash {
namespace {

constexpr int BM = kBlockRows;

// H query heads of 64 rows a workgroup, their bytes side by side in a packed layout.
template <int D, int H>
__global__ __launch_bounds__(256) void packed_pre_kernel(PackedBwdArgs a) {
  constexpr int TPR = D / 8;           // threads per row and head, 8 elements each
  constexpr int RPP = 256 / TPR / H;   // rows per pass
  constexpr int U = BM / RPP < 4 ? BM / RPP : 4;  // passes whose loads are in flight together
  static_assert(RPP >= 1 && BM % (RPP * U) == 0, "passes");
  const PackedArgs& p = a.p;
  const int tid = threadIdx.x, l = tid & 63;
  const bool causal = p.causal != 0;
  const int groups = p.heads_q / H, order = (a.slots_k + 3) / 4;
  int x = (int)blockIdx.x;
  if (x < order) {  // ---- one wave per KV-tile slot; first, as one of them counts longest
    const int slot = __builtin_amdgcn_readfirstlane(x * 4 + (tid >> 6));
    if (slot >= a.slots_k) return;
    const int s = __builtin_amdgcn_readfirstlane(
        find_last(p.batch, slot, l, [&](int x) { return first_slot(p.cu_k, x, p.total_k, a.bc); }));
    auto geom = [&](int x) {
      return SeqGeom{span_of(p.cu_q, x, p.total_q).len, span_of(p.cu_k, x, p.total_k).len, causal, a.bc};
    };
    const SeqGeom g = geom(s);
    const int j = slot - first_slot(p.cu_k, s, p.total_k, a.bc);
    const int length = g.chain(j);
    int place = 0, total = 0;
    long steps = 0;
    for (int b = 0; b < p.batch; b += 64) {
      const int o = b + l;
      if (o < p.batch) {
        const SeqGeom og = geom(o);
        place += order_part(og, o, s, j, length);
        total += og.tiles();
        steps += og.steps();
      }
    }
    place = wave_sum(place);
    if (slot == 0) {  // the wave of the first slot counts, and looks the offsets over
      bool bad = false;
      for (int b = l; b < p.batch; b += 64)
        bad |= p.cu_q[b] < 0 || p.cu_q[b + 1] < p.cu_q[b] || p.cu_q[b + 1] > p.total_q || p.cu_k[b] < 0 ||
               p.cu_k[b + 1] < p.cu_k[b] || p.cu_k[b + 1] > p.total_k;
      bad = __any(bad);
      total = wave_sum(total);
      total = total < a.slots_k ? total : a.slots_k;
      steps = ((long)wave_sum((int)(steps >> 20)) << 20) + wave_sum((int)(steps & 0xfffff));
      // the cheapest split: lane l weighs limit l % 8 with parts l / 8
      const int group = p.heads_q / p.heads_kv;
      int n_long = 0, heads = group;
      if (group > 1) {
        const long share = steps * p.heads_q / kSplitWorkers;
        int longest = 0, mine = 0;
#pragma unroll
        for (int i = 0; i < kSplitLimits; ++i) {
          const long above = split_above(share, group, i);
          const int from = above < (1 << 30) ? (int)above + 1 : 1 << 30;
          int n = 0;
          for (int b = 0; b < p.batch; b += 64)
            if (b + l < p.batch) n += geom(b + l).tiles_from(from);
          n = wave_sum(n);
          mine = (l & 7) == i ? n : mine;
        }
        for (int b = 0; b < p.batch; b += 64)
          if (b + l < p.batch) {
            const SeqGeom og = geom(b + l);
            const int x = og.tiles() > 0 ? og.chain(0) : 0;
            longest = x > longest ? x : longest;
          }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
          const int x = __shfl_xor(longest, o);
          longest = x > longest ? x : longest;
        }
        const int per = split_heads(group, l >> 3);
        long cost = split_cost(share, longest, split_above(share, group, l & 7), mine, per, group, p.heads_kv);
        if (per < group && (long)mine * p.heads_kv * split_parts(group, per) > a.split_room) cost = 1L << 48;
        cost = cost << 6 | l;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
          const long x = __shfl_xor(cost, o);
          cost = x < cost ? x : cost;
        }
        const int best = (int)(cost & 63);
        heads = split_heads(group, best >> 3);
        n_long = __shfl(mine, best);
        if (heads >= group) n_long = 0;
        n_long = n_long < total ? n_long : total;
      }
      if (l == 0) {
        a.ctrl[kCtrlTicket] = 0;
        a.ctrl[kCtrlError] = bad ? 1 : 0;
        if (a.status) *a.status = bad ? 1 : 0;
        // chains of sequences that overlap would wait for one another in vain
        if (bad) total = n_long = 0;
        a.ctrl[kCtrlItems] = total;
        a.ctrl[kCtrlLong] = n_long;
        a.ctrl[kCtrlHeads] = heads;
      }
    }
    if (l != 0) return;
    if (j >= 0 && j < g.tiles() && (unsigned)place < (unsigned)a.slots_k) {
      a.order[2 * (size_t)place] = s;
      a.order[2 * (size_t)place + 1] = j;
    }
    return;
  }
  x -= order;
  if (x < a.slots_q) {  // ---- a slot's counters, and dQ where nothing else writes it
    for (int h = tid; h < p.heads_q; h += 256) a.counters[((size_t)x * p.heads_q + h) * kCtrStride] = 0;
    const int s = __builtin_amdgcn_readfirstlane(
        find_last(p.batch, x, l, [&](int i) { return first_slot(p.cu_q, i, p.total_q, BM); }));
    const Span q = span_of(p.cu_q, s, p.total_q), k = span_of(p.cu_k, s, p.total_k);
    const int pb = x - first_slot(p.cu_q, s, p.total_q, BM);
    if (pb < 0 || pb * BM >= q.len) return;
    const SeqGeom g{q.len, k.len, causal, a.bc};
    if (g.last_tile(pb) >= 0) return;
    const int rows = q.len - pb * BM < BM ? q.len - pb * BM : BM;
    for (int e = tid; e < rows * p.heads_q * TPR; e += 256) {
      const int r = e / (p.heads_q * TPR), h = e / TPR % p.heads_q;
      *(u32x4*)((__bf16*)a.dq + ((int64_t)q.start + pb * BM + r) * a.dqs.row + h * a.dqs.head + 8 * (e % TPR)) = u32x4{0, 0, 0, 0};
    }
    return;
  }
  x -= a.slots_q;
  // ---- D and L of 64 rows
  const int row0 = x / groups * BM, hg = x % groups * H;
  const int rows = p.total_q - row0 < BM ? p.total_q - row0 : BM;
  const int c = tid % TPR, h = hg + tid / TPR % H, r0 = tid / (TPR * H);
  const int64_t vec = (int64_t)h * p.total_q + row0;
  const __bf16* dO = (const __bf16*)a.dO + row0 * a.dos.row + h * a.dos.head + 8 * c;
  const __bf16* O = (const __bf16*)a.o + row0 * p.os.row + h * p.os.head + 8 * c;
  for (int b = r0; b < rows; b += RPP * U) {
    u32x4 u0[U], u1[U];
    float L[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      int r = b + u * RPP;
      r = r < rows ? r : rows - 1;  // (read, not written)
      u0[u] = *(const u32x4*)(dO + r * a.dos.row);
      u1[u] = __builtin_nontemporal_load((const u32x4*)(O + r * p.os.row));  // (nothing reads O again)
      L[u] = p.lse[vec + r];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float acc = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float xf = bf16_to_f32((unsigned short)(u0[u][e >> 1] >> (16 * (e & 1))));
        const float yf = bf16_to_f32((unsigned short)(u1[u][e >> 1] >> (16 * (e & 1))));
        acc = __builtin_fmaf(xf, yf, acc);
      }
      // butterfly over the TPR lanes of a row, as in bwd_pre
#pragma unroll
      for (int o = 1; o < TPR; o <<= 1) acc += __shfl_xor(acc, o);
      const int r = b + u * RPP;
      if (c == 0 && r < rows) {
        a.dvec[vec + r] = acc;
        a.lse2[vec + r] = L[u] == -INFINITY ? INFINITY : L[u] * kLog2e;
      }
    }
  }
}

// dK, dV of the split tiles: the parts' partials, in order.  A thread sums 8 columns of
// a row, a workgroup 2048 / D rows of a tile, K/V head and tensor; eight parts' loads are
// in flight at once.  A fixed grid takes the pieces in turn, as their number is only
// known on the device.  Memory-bound: 8192 keys of 8 heads of 128 in two parts 34 us, 168 MB,
// 4.9 TB/s.
template <int D>
__global__ __launch_bounds__(256) void packed_sum_kernel(PackedBwdArgs a) {
  constexpr int RPW = 2048 / D;
  const PackedArgs& p = a.p;
  const int tid = threadIdx.x, pieces = a.bc / RPW;
  const int n_long = a.ctrl[kCtrlLong], parts = split_parts(p.heads_q / p.heads_kv, a.ctrl[kCtrlHeads]);
  const long todo = (long)n_long * p.heads_kv * 2 * pieces;
  for (long x = blockIdx.x; x < todo; x += gridDim.x) {
    const int piece = (int)(x % pieces), which = (int)(x / pieces) & 1;  // 0: dK, 1: dV
    const int tile = (int)(x / (2 * pieces)), hk = tile % p.heads_kv, place = tile / p.heads_kv;
    const int s = a.order[2 * (size_t)place], j = a.order[2 * (size_t)place + 1];
    if ((unsigned)s >= (unsigned)p.batch) continue;
    const Span k = span_of(p.cu_k, s, p.total_k);
    const int r = piece * RPW + tid / (D / 8), c = tid % (D / 8) * 8;  // row of the tile, first column
    if (j < 0 || j * a.bc + r >= k.len) continue;
    const size_t step = (size_t)a.bc * D;
    const float* src = a.dkv_part + ((size_t)tile * parts * 2 + which) * step + (size_t)r * D + c;
    f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
    int g = 0;
    for (; g + 8 <= parts; g += 8) {
      f32x4 x0[8], x1[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x0[i] = *(const f32x4*)(src + (g + i) * (2 * step));
        x1[i] = *(const f32x4*)(src + (g + i) * (2 * step) + 4);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) lo += x0[i], hi += x1[i];
    }
    for (; g < parts; ++g) {
      lo += *(const f32x4*)(src + g * (2 * step));
      hi += *(const f32x4*)(src + g * (2 * step) + 4);
    }
    const float scale = which ? 1.f : a.scale;
    lo *= scale, hi *= scale;
    const Strides& st = which ? a.dvs : a.dks;
    __bf16* out = (__bf16*)(which ? a.dv : a.dk) + ((int64_t)k.start + j * a.bc + r) * st.row + hk * st.head + c;
    *(u32x4*)out = u32x4{pack_bf16(lo[0], lo[1]), pack_bf16(lo[2], lo[3]), pack_bf16(hi[0], hi[1]), pack_bf16(hi[2], hi[3])};
  }
}

template <int D>
hipError_t launch(const PackedBwdArgs& a, int cus, hipStream_t stream) {
  // several heads a workgroup where that leaves workgroups enough
  const int rows = (a.p.total_q + BM - 1) / BM, rest = a.slots_q + (a.slots_k + 3) / 4;
  constexpr int H = D == 256 ? 2 : 4;
  if (a.p.heads_q % H == 0 && (long)rows * a.p.heads_q >= 4096)
    hipLaunchKernelGGL((packed_pre_kernel<D, H>), dim3((unsigned)(rows * (a.p.heads_q / H) + rest)), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((packed_pre_kernel<D, 1>), dim3((unsigned)(rows * a.p.heads_q + rest)), dim3(256), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // persistent workgroups: as many as stay resident (two per CU at d = 64 and 128 rows, else one).
  // A chain waits only on chains that took an earlier ticket, so any count is safe.
  const long items = (long)a.slots_k * a.p.heads_q, cap = (long)cus * (D == 64 && a.bc == 128 ? 2 : 1);
  const int g = (int)(items < cap ? items : cap);
  if constexpr (D == 64) e = a.bc == 256 ? launch_packed_main64w(a, g, stream) : launch_packed_main64(a, g, stream);
  else if constexpr (D == 256) e = launch_packed_mainw(a, D, g, stream);
  else e = a.bc == 256 ? launch_packed_mainw(a, D, g, stream) : launch_packed_main128(a, g, stream);
  if (e != hipSuccess || a.p.heads_q == a.p.heads_kv) return e;
  const long most = (long)a.split_room * 2 * (a.bc / (2048 / D));  // (2 parts at least to a sum)
  const unsigned sums = (unsigned)(most / 2 < 8L * cus ? most / 2 : 8L * cus);
  hipLaunchKernelGGL(packed_sum_kernel<D>, dim3(sums), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

// d = 64 and 128 have both tiles.  Wide ones at d = 128 need chains enough for 256 CUs (split by query
// head, total_k / 256 times heads_q; longer ones weigh more under a causal mask) and
// sequences that fill them.  Measured (us, narrow / wide; heads_q over heads_kv):
//   causal  352 chains of one of 3000 385 / 348, 384 (4096, 24 over 8) 511 / 466, 512 (2048
//           64 over 8) 360 / 312; 256 (4096, 16 over 16) 345 / 367, (8192, 8 over 1) 673 / 721,
//           (2 of 1024, 32 over 8) 136 / 138
//   full    192 (2048, 24 over 24) 303 / 258, 256 (4096, 16 over 4) 674 / 525; 128 (4096, 8 over 8,
//           causal) 264 / 363
//   length  1024 chains of 16 of 512 292 / 272; 24 of 384 233 / 314, 32 of 256 159 / 226, 10 of 409
//           on average 180 / 200
// d = 64 likewise, for longer causal sequences:
//   causal  512 chains (4096, 32 over 8) 421 / 354, 384 (2048, 48 over 8) 192 / 172, 380 (5000, 20 over 4)
//           408 / 354; 320 (4096, 20 over 4) 285 / 313, 256 (8192, 8 over 1) 463 / 541
//   full    176 (3000, 16 over 4) 285 / 260, 256 (2048, 32 over 32) 202 / 175; 128 (4096, 8 over 8) 265 / 329
//   length  causal 8 of 1024 255 / 219, 4 of 2048 414 / 360; 11 of 768 202 / 228, 14 of 600 180 / 203 (but 13
//           of 640, 32 over 32, 201 / 183); full 32 of 256 122 / 98, 24 of 341 on average 279 / 262, 40 of 200
//           158 / 161 (but 16 of 520 313 / 328)
int packed_tile_rows(int d, int total_k, int batch, int heads_q, int causal) {
  const long chains = (long)(total_k / 256) * heads_q;
  if (d == 128) return chains >= (causal ? 320 : 160) && total_k >= 480L * batch ? 256 : 128;
  if (d == 64) return chains >= (causal ? 352 : 160) && total_k >= (causal ? 800L : 256L) * batch ? 256 : 128;
  return 128;
}

hipError_t launch_packed_bwd(const PackedBwdArgs& a, int d, int cus, hipStream_t stream) {
  if (d == 64) return launch<64>(a, cus, stream);
  if (d == 128) return launch<128>(a, cus, stream);
  return launch<256>(a, cus, stream);
}

}  // namespace dash
