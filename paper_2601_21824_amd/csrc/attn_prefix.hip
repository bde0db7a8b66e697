// attn_prefix.hip -- attention of one new token per sequence for a batch that shares a long
// prefix of its keys, which are read and multiplied once for all of its sequences.
//
//   o = (sum_j e^(s_j - m) v_j) / (sum_j e^(s_j - m)),  j over the prefix's runs and the sequence's own keys
//
// The prefix is a matrix product like a prompt's: every query head of every sequence is a
// row.  prefix_kernel runs the forward of fwd_main.h on another view of its rows: a
// workgroup takes 128 rows of one K/V head (sequence r / G, query head r % G) and a run of
// the prefix's keys, and leaves O, maximum and sum in fp32.  Few rows are not worth a tile of that size:
// prefix_few_kernel takes 16, with the one-token step of decode_main.h.  Further workgroups of the same
// launch take each sequence's own keys by that step, and prefix_join_kernel adds the parts in order.
//
// A sequence shorter than the prefix does without it: all of its keys are its own.  (A row either sees
// a whole run or is left out of it, so that nothing behind a sequence's last key reaches it.)
//
// K and V come from the cache's pages, tile by tile, each wave its quarter of the rows, which
// lie in one page: bf16 by direct copies into LDS; the 8-bit and 4-bit types through
// registers, widened to bf16 (exactly) on the way to LDS.  The next tile's page numbers are
// read a tile ahead.  Rows past the run read zeros.
//
// Bound by the issue of four waves a CU where the batch is large, 4 d operations a row and key: 64 sequences of 32
// heads over 8 of 128 behind 32768 shared bf16 keys and with 256 of their own on average, 35 GFLOP, 70 us, 500 TFLOP/s (a prompt's
// forward, with eight waves, 980).  Smaller ones by the launch and the search of 800 to 960 workgroups, most of which
// find no own keys (6.2 us with nothing to attend to), and by dependent tiles: 24 sequences behind 16384 keys in MXFP8, eight tiles
// of 64 keys a workgroup at 1.7 us each (they go through registers, of which one instantiation, d = 128 in MXFP8, has three
// too few), 24 us; by 16 rows, 8 of 16 heads over 4 of 256 behind 9001 keys in MXFP4, two or three tiles a wave, 13.7, of which a first tile
// is 1.9, the others 4.8 and own keys 0.9; 3 of 8 over 2 of 64 behind 700 keys 5.8.
#include "decode_main.h"
#include "fwd_main.h"
#include "mx.h"
#include "ops.h"
#include "page_index.h"
#include "paged.h"

namespace dash {
namespace {

constexpr int kRows = 128;  // rows of a workgroup, if they are many

// The forward masks and takes maxima before it multiplies by the softmax scale, which so has to be above 0: K's scale
// of an e4m3 head may be anything, and its sign, or 0, goes into Q.  (The product in decode_main.h's order: equal scores
// 2^24 and more from 0 would otherwise differ by a rounding that moves weights.)
struct ScoreScale {
  float c2, q;  // q: 1, -1 or 0 (times which an infinity is NaN, as it is for the other kernels)
};
__device__ inline ScoreScale score_scale(float scale, float k_scale) {
  const float c2 = scale * kLog2e, s = c2 * k_scale;
  return {s == 0.f ? c2 : __builtin_fabsf(s), s == 0.f ? 0.f : s < 0.f ? -1.f : 1.f};
}

// The prefix's runs: whole kUnit keys, cut into n equal runs of min_run keys at least.
constexpr int kUnit = 128;
struct Run {
  int first, keys, n;
};
__device__ inline Run run_of(const DecodeArgs& a, int keys, int i) {
  const int units = (keys + kUnit - 1) / kUnit;
  int n = keys / a.min_run;
  n = n < a.splits ? n : a.splits;
  n = n > 1 ? n : 1;
  const int from = (int)((int64_t)units * i / n), to = (int)((int64_t)units * (i + 1) / n);
  return {from * kUnit, (to * kUnit < keys ? to * kUnit : keys) - from * kUnit, keys > 0 ? n : 0};
}
// Item -> K/V head, run, tile of rows
struct Item {
  int hk, split, q0;
};
__device__ inline Item item_of(const DecodeArgs& a, int item, int rows) {
  const int tiles = (a.c.batch * (a.c.heads_q / a.c.heads_kv) + rows - 1) / rows;
  return {item / (a.splits * tiles), item / tiles % a.splits, item % tiles * rows};
}

template <int D, int TYPE>
struct PrefixView {
  static constexpr bool kPacked = true, kPaged = true;
  static constexpr int KT = D == 256 ? 32 : 64;
  static constexpr int BITS = TYPE == kBf16 ? 16 : TYPE == kMx4 ? 4 : 8;
  static constexpr bool kStaged = TYPE != kBf16, MX = TYPE >= kMx8;
  static constexpr int SZ = TYPE == kBf16 ? 2 : 1;          // bytes of a stride's unit
  static constexpr int PE = kStaged ? 16 : 8;               // components of a lane's piece
  static constexpr int PPR = D / PE;                        // pieces of a row
  static constexpr int RW = KT / 4, RL = 64 / PPR;          // rows of a wave, in one page; rows of one load
  static constexpr int PARTS = RW / RL;
  static_assert(RW % RL == 0 && 16 % RW == 0);
  static constexpr int PW = PE * BITS / 32;                 // words of a piece
  static constexpr int SB = D / kMxBlock;
  const DecodeArgs& a;
  int hk, nq, nk, first, w, last_page;
  const __bf16* q;   // of the lane's row
  bool sees;         // whether its sequence has the prefix (else it is computed on zeros and left out)
  int64_t part;      // its number in prefix_o and prefix_m, -1: there is no such row
  float v_scale, q_scale;
  mutable int at, row, id;  // the next tile's place: page index and row, and page, of this wave's rows
  mutable unsigned kx[PARTS][PW], vx[PARTS][PW], kb[PARTS], vb[PARTS];
  mutable bool bad;

  __device__ PrefixView(const DecodeArgs& a_, const Item& it, int prefix, const Run& run, int w_, float q_scale_)
      : a(a_), hk(it.hk), nk(run.keys), first(run.first), w(w_), last_page((prefix - 1) / a_.c.page_size), q_scale(q_scale_), bad(false) {
    const int key = first + w * RW;
    at = key / a.c.page_size;
    row = key - at * a.c.page_size;
    look();
    const int G = a.c.heads_q / a.c.heads_kv, r = it.q0 + 32 * w + (threadIdx.x & 31);
    nq = a.c.batch * G;
    const int s = r < nq ? r / G : 0, h = hk * G + r % G;
    sees = r < nq && has_prefix(a.c, s, prefix);
    part = r < nq ? ((int64_t)it.split * a.c.batch + s) * a.c.heads_q + h : -1;
    q = (const __bf16*)a.q + s * a.qs.row + h * a.qs.head;
    v_scale = TYPE == kE4m3 && a.c.v_scale ? a.c.v_scale[hk] : 1.f;
  }
  __device__ void look() const { id = table_entry(a.prefix_table, at < last_page ? at : last_page); }

  __device__ static constexpr int off() { return 0; }

  // ---- tiles
  __device__ __amdgpu_buffer_rsrc_t rows(const void* p, int64_t page, int64_t head, int64_t stride, int i, int n) const {
    const uint32_t bytes = n > 0 ? (uint32_t)(n - 1) * (uint32_t)stride * SZ + D * BITS / 8 : 0;
    return make_rsrc((const char*)p + (i * page + hk * head + row * stride) * SZ, bytes);
  }
  __device__ __amdgpu_buffer_rsrc_t scales(const uint8_t* p, int i, int n) const {
    return make_rsrc(p + (((int64_t)i * a.c.heads_kv + hk) * a.c.page_size + row) * SB, n > 0 ? n * SB : 0);
  }
  __device__ void request(int k0, uint32_t k_lds, uint32_t v_lds) const {
    const CacheArgs& c = a.c;
    const int l = threadIdx.x & 63, lr = l / PPR;
    int n = nk - (k0 + w * RW);  // rows that the wave has here
    n = n < RW ? n : RW;
    int i = id;
    if (!page_ok(i, c.pages)) bad = true, i = 0;
    const auto rk = rows(c.k, c.k_page, c.k_head, c.k_row, i, n), rv = rows(c.v, c.v_page, c.v_head, c.v_row, i, n);
    const auto sk = MX ? scales(c.k_mx, i, n) : rk, sv = MX ? scales(c.v_mx, i, n) : rv;
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      const int r = p * RL + lr;  // this lane's row among the wave's
      if constexpr (!kStaged) {
        const int ch = (l % PPR) ^ tile_swz<D>(w * RW + r);
        const uint32_t to = (uint32_t)(w * RW * D * 2 + 1024 * p);
        dma16(rk, k_lds + to, (uint32_t)r * (uint32_t)c.k_row * 2 + ch * 16);
        dma16(rv, v_lds + to, (uint32_t)r * (uint32_t)c.v_row * 2 + ch * 16);
      } else {
        load(kx[p], rk, (uint32_t)r * (uint32_t)c.k_row + l % PPR * (PW * 4));
        load(vx[p], rv, (uint32_t)r * (uint32_t)c.v_row + l % PPR * (PW * 4));
        if constexpr (MX) {
          const uint32_t o = r * SB + l % PPR * PE / kMxBlock;
          kb[p] = __builtin_amdgcn_raw_buffer_load_b8(sk, o, 0, 0);
          vb[p] = __builtin_amdgcn_raw_buffer_load_b8(sv, o, 0, 0);
        }
      }
    }
    at += KT / c.page_size;
    row += KT % c.page_size;
    if (row >= c.page_size) row -= c.page_size, ++at;
    look();
  }
  __device__ static void load(unsigned (&x)[PW], __amdgpu_buffer_rsrc_t r, uint32_t off) {
    if constexpr (PW == 4) {
      const u32x4 y = ld16(r, off);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = y[i];
    } else {
      const u32x2 y = __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0);
      x[0] = y[0], x[1] = y[1];
    }
  }
  // 8 components of a piece as bf16
  __device__ static u32x4 chunk(const unsigned* x, unsigned byte) {
    if constexpr (TYPE == kMx4) {
      const float s = mx_scale(byte);
      return u32x4{mx_pair<true>(x[0], 0, s), mx_pair<true>(x[0], 1, s), mx_pair<true>(x[0], 2, s), mx_pair<true>(x[0], 3, s)};
    } else {
      const float s = MX ? mx_scale(byte) : 1.f;
      return u32x4{mx_pair<false>(x[0], 0, s), mx_pair<false>(x[0], 1, s), mx_pair<false>(x[1], 0, s), mx_pair<false>(x[1], 1, s)};
    }
  }
  __device__ void store(uint32_t k_lds, uint32_t v_lds) const {
    if constexpr (kStaged) {
      const int l = threadIdx.x & 63, piece = l % PPR;
#pragma unroll
      for (int p = 0; p < PARTS; ++p) {
        const int r = w * RW + p * RL + l / PPR;
        // which of its two chunks a lane writes first: 16 lanes' chunks lie in distinct banks
        const bool odd = D == 256 ? piece >= 8 : D == 128 ? r & 1 : false;
        put(k_lds, r, piece, odd, kx[p], kb[p]);
        put(v_lds, r, piece, odd, vx[p], vb[p]);
      }
    }
  }
  __device__ static void put(uint32_t lds, int r, int piece, bool odd, const unsigned* x, unsigned byte) {
    const u32x4 a = chunk(x, byte), b = chunk(x + PW / 2, byte);
    u32x4 p, q;
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = odd ? b[i] : a[i], q[i] = odd ? a[i] : b[i];
    typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
    const uint32_t base = lds + r * (D * 2);
    *(lds_u32x4*)(base + (((2 * piece + odd) ^ tile_swz<D>(r)) << 4)) = p;
    *(lds_u32x4*)(base + (((2 * piece + !odd) ^ tile_swz<D>(r)) << 4)) = q;
  }

  // ---- single rows, for far_rows: key (of the run), component
  __device__ const char* place(const void* p, int64_t page, int64_t head, int64_t stride, int key, int col, int64_t* mx) const {
    const int j = first + (key < nk ? key : 0), pg = j / a.c.page_size, r = j - pg * a.c.page_size;
    const int i = page_ok(a.prefix_table[pg], a.c.pages) ? a.prefix_table[pg] : 0;
    *mx = (((int64_t)i * a.c.heads_kv + hk) * a.c.page_size + r) * SB + col / kMxBlock;
    return (const char*)p + (i * page + hk * head + r * stride) * SZ + col * BITS / 8;
  }
  __device__ u32x4 eight(const void* p, const uint8_t* bytes, int64_t page, int64_t head, int64_t stride, int key, int col) const {
    int64_t mx;
    const unsigned* x = (const unsigned*)place(p, page, head, stride, key, col, &mx);
    u32x4 y;
    if constexpr (TYPE == kBf16) y = *(const u32x4*)x;
    else y = chunk(x, MX ? bytes[mx] : 0);
    return key < nk ? y : u32x4{0, 0, 0, 0};
  }
  __device__ bf16x8 k8(int key, int col) const { return as_bf16x8(eight(a.c.k, a.c.k_mx, a.c.k_page, a.c.k_head, a.c.k_row, key, col)); }
  __device__ unsigned v1(int key, int col) const {
    const u32x4 y = eight(a.c.v, a.c.v_mx, a.c.v_page, a.c.v_head, a.c.v_row, key, col & ~7);
    const unsigned lo = col & 4 ? y[2] : y[0], hi = col & 4 ? y[3] : y[1], x = col & 2 ? hi : lo;
    return col & 1 ? x >> 16 : x & 0xffffu;
  }

  // ---- query rows: a lane has one, q0 + 32 w + l % 32, whose place is found once
  __device__ bf16x8 q8(int, int col) const {
    u32x4 x = {0, 0, 0, 0};
    if (sees) x = *(const u32x4*)(q + col);
    if constexpr (TYPE == kE4m3) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        x[i] = pack_bf16(__builtin_bit_cast(float, x[i] << 16) * q_scale, __builtin_bit_cast(float, x[i] & 0xffff0000u) * q_scale);
    }
    return as_bf16x8(x);
  }
  __device__ int o() const { return 0; }
  __device__ int lse() const { return 0; }
  __device__ void put_o(int, int, int col, float a0, float a1, float a2, float a3) const {
    f32x4 x = {a0 * v_scale, a1 * v_scale, a2 * v_scale, a3 * v_scale};
    if (!sees) x = f32x4{0.f, 0.f, 0.f, 0.f};
    if (part >= 0) *(f32x4*)(a.prefix_o + part * D + col) = x;
  }
  __device__ void put_l(int, int, float m, float sum) const {
    if (part >= 0) *(float2*)(a.prefix_m + 2 * part) = sees ? make_float2(m, sum) : make_float2(-INFINITY, 0.f);
  }
};

// Workgroup -> item, each XCD a contiguous share: the row tiles of a run read its keys from
// one L2.  Those behind the prefix's take the sequences' own keys.
__device__ inline int own_block(const DecodeArgs& a, int items, int* item) {
  const int per = (items + 7) >> 3, x = (int)blockIdx.x;
  *item = x < 8 * per ? (x & 7) * per + (x >> 3) : items;
  return x - 8 * per;
}

template <int D, int TYPE, int WPS>
__global__ __launch_bounds__(256, WPS) void prefix_kernel(DecodeArgs a, int items) {
  const CacheArgs& c = a.c;
  int item;
  const int own = own_block(a, items, &item);
  __shared__ __attribute__((aligned(1024))) union Space {
    FwdTiles<D> tiles;
    JoinSpace<D, 4> join;
    __device__ Space() {}
  } space;
  if (own >= 0) return decode_part<D, TYPE, 4, true>(a, own, space.join);
  if (item >= items) return;
  const Item it = item_of(a, item, kRows);
  const int prefix = __builtin_amdgcn_readfirstlane(prefix_of(a));
  if (item == 0 && threadIdx.x == 0 && c.status && *a.prefix_len != prefix) *c.status = 1;
  const Run run = run_of(a, prefix, it.split);
  if (it.split >= run.n) return;
  const ScoreScale score = score_scale(a.scale, TYPE == kE4m3 && c.k_scale ? c.k_scale[it.hk] : 1.f);
  const PrefixView<D, TYPE> view(a, it, prefix, run, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), score.q);
  attn_fwd_rows<D, 1>(view, 0, score.c2, it.q0, space.tiles);
  if (view.bad && (threadIdx.x & 63) == 0 && c.status) *c.status = 1;
}

// Few rows: 16 of a K/V head's a workgroup, whose four waves take every fourth 32 keys of the run each.
template <int D, int TYPE>
__global__ __launch_bounds__(256, 2) void prefix_few_kernel(DecodeArgs a, int items) {
  __shared__ JoinSpace<D, 4> space;
  const CacheArgs& c = a.c;
  int item;
  const int own = own_block(a, items, &item);
  if (own >= 0) return decode_part<D, TYPE, 4, true>(a, own, space);
  if (item >= items) return;
  const Item it = item_of(a, item, kQ);
  const int prefix = __builtin_amdgcn_readfirstlane(prefix_of(a));
  if (item == 0 && threadIdx.x == 0 && c.status && *a.prefix_len != prefix) *c.status = 1;
  const Run run = run_of(a, prefix, it.split);
  if (it.split >= run.n) return;
  const int tid = threadIdx.x, l = tid & 63, g = l >> 4, lq = l & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = c.heads_q / c.heads_kv, nq = c.batch * G, to = run.first + run.keys;
  // row q0 + l % 16: its sequence and query head
  const int r = it.q0 + lq, s = r < nq ? r / G : 0, h = it.hk * G + (r < nq ? r % G : 0);
  const bool sees = r < nq && has_prefix(c, s, prefix);
  Rows<D> rows;
#pragma unroll
  for (int ks = 0; ks < D / 32; ++ks) {
    const u32x4 x = *(const u32x4*)((const __bf16*)a.q + s * a.qs.row + h * a.qs.head + Tile<D, TYPE>::first(ks, g));
    rows.q[ks] = as_bf16x8(sees ? x : u32x4{0, 0, 0, 0});
  }
  rows.clear();
  const float c2 = a.scale * kLog2e * (TYPE == kE4m3 && c.k_scale ? c.k_scale[it.hk] : 1.f);
  if (run.first + 32 * w < to) {
    KeyRows<D, TYPE, false> keys(c, a.prefix_table, it.hk, prefix, run.first + 32 * w, 32 * 4, l);
    for (int kb = run.first + 32 * w; kb < to; kb += 32 * 4) {
      Tile<D, TYPE> t;
      keys.load(t);
      keys.look();
      rows.add(t, c2, kb, 0, to, lq, g);
    }
    if (keys.bad && l == 0 && c.status) *c.status = 1;
  }
  const float vs = TYPE == kE4m3 && c.v_scale ? c.v_scale[it.hk] : 1.f;
  join_waves<D, 4>(space, rows.o, rows.m, rows.sum, w, nq - it.q0 < kQ ? nq - it.q0 : kQ, [&](int i, int d0, float top, float den, f32x4 out) {
    const int r = it.q0 + i;
    const int64_t at = ((int64_t)it.split * c.batch + r / G) * c.heads_q + it.hk * G + r % G;
    const bool sees = has_prefix(c, r / G, prefix);
    const float inv = sees && (den > 0.f || den != den) ? vs / den : 0.f;
    *(f32x4*)(a.prefix_o + at * D + d0) = sees ? out * inv : f32x4{0.f, 0.f, 0.f, 0.f};
    if (d0 == 0) *(float2*)(a.prefix_m + 2 * at) = sees ? make_float2(top, den) : make_float2(-INFINITY, 0.f);
  });
}

// The parts of one sequence and query head, the prefix's first, each in order: thread groups of
// D / 4 lanes take every NG-th part with a running maximum and are added in order of the group.  Bound by
// latency, three dependent loads: 4 us for a few rows (finding the maximum first, one load more, 4.7), and for 2048 rows
// of 18 parts by the parts' 19 MB, 8 us (9.8).
template <int D>
__global__ __launch_bounds__(256) void prefix_join_kernel(DecodeArgs a) {
  constexpr int NG = 256 / (D / 4), U = 8;  // U parts' loads in flight together
  __shared__ f32x4 acc[NG][D / 4];
  __shared__ float dens[NG], tops[NG];
  const int hq = a.c.heads_q, s = (int)blockIdx.x / hq, h = (int)blockIdx.x % hq;
  const int np = run_of(a, prefix_of(a), 0).n;
  const int first = a.base[2 * s], n = np + a.base[2 * s + 1];
  const int tid = threadIdx.x, grp = tid / (D / 4), d4 = tid % (D / 4);
  float top = -INFINITY, den = 0.f;
  f32x4 out = {0.f, 0.f, 0.f, 0.f};
  for (int i = grp; i < n; i += U * NG) {
    float2 m[U];
    f32x4 o[U];
    float mx = top;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int iu = i + u * NG < n ? i + u * NG : i;  // (read again, not added)
      // part iu: its row of prefix_o and prefix_m, or of part_o and part_m
      const int64_t at = iu < np ? ((int64_t)iu * a.c.batch + s) * hq + h : (int64_t)(first + iu - np) * hq + h;
      m[u] = *(const float2*)((iu < np ? a.prefix_m : a.part_m) + 2 * at);
      o[u] = *(const f32x4*)((iu < np ? a.prefix_o : a.part_o) + at * D + 4 * d4);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) mx = fmaxf(mx, m[u].x);
    const float mm = mx == -INFINITY ? 0.f : mx, alpha = __builtin_amdgcn_exp2f(top - mm);
    top = mx;
    den *= alpha;
    out *= alpha;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * NG < n) {
        const float f = __builtin_amdgcn_exp2f(m[u].x - mm), e = f * m[u].y;
        den += e;
        out += (i + u * NG < np ? e : f) * o[u];  // (a prefix's part is over its sum already)
      }
  }
  acc[grp][d4] = out;
  if (d4 == 0) dens[grp] = den, tops[grp] = top;
  __syncthreads();
  if (grp != 0) return;
#pragma unroll
  for (int i = 1; i < NG; ++i) top = fmaxf(top, tops[i]);
  const float mm = top == -INFINITY ? 0.f : top;
  den = 0.f;
  out = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < NG; ++i) {
    const float f = __builtin_amdgcn_exp2f(tops[i] - mm);
    den += f * dens[i];
    out += f * acc[i][d4];
  }
  const float inv = den > 0.f || den != den ? 1.f / den : 0.f;
  *(u32x2*)((__bf16*)a.o + s * a.os.row + h * a.os.head + 4 * d4) =
      u32x2{pack_bf16(out[0] * inv, out[1] * inv), pack_bf16(out[2] * inv, out[3] * inv)};
  if (a.lse && d4 == 0) a.lse[(size_t)s * hq + h] = den == 0.f ? -INFINITY : (top + __log2f(den)) * kLn2;
}

int64_t items_of(int batch, int heads_q, int heads_kv, int rows) {  // without the runs
  return heads_kv * (((int64_t)batch * (heads_q / heads_kv) + rows - 1) / rows);
}
int64_t items_of(const DecodeArgs& a) { return a.splits * items_of(a.c.batch, a.c.heads_q, a.c.heads_kv, a.few ? kQ : kRows); }
// whole rounds of the XCDs, and the sequences' own chunks behind them
int64_t blocks_of(const DecodeArgs& a) { return (items_of(a) + 7) / 8 * 8 + decode_blocks(a); }

template <int D, int TYPE>
auto kernel_of(const DecodeArgs& a) {
  // (at d = 64 the types that go through registers have no room for a third workgroup's)
  constexpr int kWps = D == 256 ? 1 : D == 64 && TYPE == kBf16 ? 3 : 2;
  return a.few ? prefix_few_kernel<D, TYPE> : prefix_kernel<D, TYPE, kWps>;
}

template <int D>
void launch(const DecodeArgs& a, hipStream_t stream) {
  const auto kernel = a.c.type == kBf16   ? kernel_of<D, kBf16>(a)
                      : a.c.type == kE4m3 ? kernel_of<D, kE4m3>(a)
                      : a.c.type == kMx8  ? kernel_of<D, kMx8>(a)
                                          : kernel_of<D, kMx4>(a);
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks_of(a)), dim3(256), 0, stream, a, (int)items_of(a));
  hipLaunchKernelGGL(prefix_join_kernel<D>, dim3((unsigned)(a.c.batch * a.c.heads_q)), dim3(256), 0, stream, a);
}

}  // namespace

// How the prefix is cut.  16 rows a workgroup read K and V once for every 16, with 16 waves a CU and no
// barrier; 128 rows once for all of them, at the price of a longer start (us of the whole call, 16 / 128 rows a
// workgroup, 16384 shared keys, 8 K/V heads: 32 rows of 128 components 25.7 / 27.2, 64 rows 32 / 30, 128 rows 55 / 36;
// 4 K/V heads of 256: 32 rows 22 / 32, 64 rows 28 / 41, 128 rows 55 / 54).
// Runs: with the K/V heads and the tiles of rows 256 workgroups, one a CU, or two where a run keeps 2048
// keys all the same (at d = 64, where three fit, always): each run leaves its rows' O in fp32 to be read again
// (64 sequences of 32 heads of 128 behind 32768 keys: 81 in 256 workgroups, 86 in 512; behind 65536, the kernel alone, 134 and 116).
PrefixPlan prefix_plan(int batch, int heads_q, int heads_kv, int d, int prefix_tokens) {
  const int64_t rows = (int64_t)batch * (heads_q / heads_kv);
  PrefixPlan p;
  p.few = rows <= (d == 256 ? 96 : 32);
  p.min_run = p.few ? 128 : 256;
  const int64_t blocks = items_of(batch, heads_q, heads_kv, p.few ? kQ : kRows), most = prefix_tokens / p.min_run;
  const int64_t fit = d == 64 || (!p.few && blocks * prefix_tokens >= 512 * 2048) ? 512 : 256;
  int64_t s = fit / blocks;
  s = s < most ? s : most;
  // (64 runs at most: a bound on the parts that the join reads.  One K/V head and few rows leave CUs idle with it: more was not measured.)
  p.splits = (int)(s < 1 ? 1 : s > 64 ? 64 : s);
  return p;
}

// Chunks aimed at for the sequences' own keys: with the K/V heads (and further groups of 16 query heads) 512
// workgroups, two for each of 256 CUs, as many as run at once beside the prefix's.
int prefix_workers(int heads_q, int heads_kv) {
  const int units = heads_kv * ((heads_q / heads_kv + kQ - 1) / kQ);
  const int w = 512 / units;
  return w > 1 ? w : 1;
}

int64_t prefix_waves(const DecodeArgs& a) {
  const int64_t main = blocks_of(a) * 4, join = (int64_t)a.c.batch * a.c.heads_q * 4;
  return main > join ? main : join;
}

hipError_t launch_prefix(const DecodeArgs& a, hipStream_t stream) {
  if (a.c.d == 64) launch<64>(a, stream);
  else if (a.c.d == 128) launch<128>(a, stream);
  else launch<256>(a, stream);
  return hipGetLastError();
}

}  // namespace dash
