// attn_prefix.hip -- attention of one new token per sequence for a batch that shares a long
// prefix of its keys, which are read and multiplied once for all of its sequences.
//
//   o = (sum_j e^(s_j - m) v_j) / (sum_j e^(s_j - m)),  j over the prefix's runs and the sequence's own keys
//
// The prefix is a matrix product like a prompt's: every query head of every sequence is a
// row.  prefix_kernel runs the forward of fwd_main.h on another view of its rows: a
// workgroup takes 128 rows of one K/V head (sequence r / G, query head r % G) and a run of
// the prefix's keys, and leaves O, maximum and sum in fp32.  decode_kernel does the same
// for each sequence's own keys, 16 rows at a time, and join_kernel adds the parts in order.
//
// K and V come from the cache's pages, tile by tile: bf16 by direct copies into LDS, each wave
// from the one page that its rows of a part lie in; the 8-bit and 4-bit types through
// registers, widened to bf16 (exactly) on the way to LDS.  The next tile's page numbers are
// read a tile ahead.  Rows past the run read zeros.
#include "fwd_main.h"
#include "mx.h"
#include "ops.h"
#include "page_index.h"
#include "paged.h"

namespace dash {
namespace {

constexpr int kRows = 128;  // rows of a workgroup

// The prefix's runs: tiles of KT keys, cut into n equal runs of kMinRun keys at least.
constexpr int kMinRun = 256;
struct Run {
  int first, keys, n;
};
template <int D>
__device__ inline Run run_of(int keys, int splits, int i) {
  constexpr int KT = D == 256 ? 32 : 64;
  const int tiles = (keys + KT - 1) / KT;
  int n = keys / kMinRun;
  n = n < splits ? n : splits;
  n = n > 1 ? n : 1;
  const int a = (int)((int64_t)tiles * i / n), b = (int)((int64_t)tiles * (i + 1) / n);
  return {a * KT, (b * KT < keys ? b * KT : keys) - a * KT, keys > 0 ? n : 0};
}

template <int D, int TYPE>
struct PrefixView {
  static constexpr bool kPacked = true, kPaged = true;
  static constexpr int KT = D == 256 ? 32 : 64;
  static constexpr int BITS = TYPE == kBf16 ? 16 : TYPE == kMx4 ? 4 : 8;
  static constexpr bool kStaged = TYPE != kBf16, MX = TYPE >= kMx8;
  static constexpr int SZ = TYPE == kBf16 ? 2 : 1;          // bytes of a stride's unit
  static constexpr int PE = kStaged ? 16 : 8;               // components of a thread's piece
  static constexpr int PPR = D / PE;                        // pieces of a row
  static constexpr int RP = 256 / PPR, RW = RP / 4;         // rows of a part, and of a wave in it (16 at most: one page)
  static constexpr int PARTS = KT / RP;
  static constexpr int PW = PE * BITS / 32;                 // words of a piece
  static constexpr int SB = D / kMxBlock;
  const DecodeArgs& a;
  int hk, G, nq, nk, first, prefix, split, w, last_page;
  // the next tile's places: page index and row, and page, of this wave's rows in each part
  mutable int at[PARTS], row[PARTS], id[PARTS];
  mutable unsigned kx[PARTS][PW], vx[PARTS][PW], kb[PARTS], vb[PARTS];
  mutable bool bad;

  __device__ PrefixView(const DecodeArgs& a_, int hk_, int prefix_, const Run& run, int split_, int w_)
      : a(a_), hk(hk_), G(a_.c.heads_q / a_.c.heads_kv), nq(a_.c.batch * (a_.c.heads_q / a_.c.heads_kv)), nk(run.keys), first(run.first),
        prefix(prefix_), split(split_), w(w_), last_page((prefix_ - 1) / a_.c.page_size), bad(false) {
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      const int key = first + p * RP + w * RW;
      at[p] = key / a.c.page_size;
      row[p] = key - at[p] * a.c.page_size;
      look(p);
    }
  }
  __device__ void look(int p) const { id[p] = __builtin_amdgcn_readfirstlane(a.prefix_table[at[p] < last_page ? at[p] : last_page]); }

  __device__ static constexpr int off() { return 0; }

  // ---- tiles
  __device__ __amdgpu_buffer_rsrc_t rows(const void* p, int64_t page, int64_t head, int64_t stride, int i, int r, int n) const {
    const uint32_t bytes = n > 0 ? (uint32_t)(n - 1) * (uint32_t)stride * SZ + D * BITS / 8 : 0;
    return make_rsrc((const char*)p + (i * page + hk * head + r * stride) * SZ, bytes);
  }
  __device__ __amdgpu_buffer_rsrc_t scales(const uint8_t* p, int i, int r, int n) const {
    return make_rsrc(p + (((int64_t)i * a.c.heads_kv + hk) * a.c.page_size + r) * SB, n > 0 ? n * SB : 0);
  }
  __device__ void request(int k0, uint32_t k_lds, uint32_t v_lds) const {
    const CacheArgs& c = a.c;
    const int tid = threadIdx.x, lr = tid % 64 / PPR;  // row of this lane among the wave's
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      int n = nk - (k0 + p * RP + w * RW);  // rows that the wave has here
      n = n < RW ? n : RW;
      int i = id[p];
      if (!page_ok(i, c.pages)) bad = true, i = 0;
      const auto rk = rows(c.k, c.k_page, c.k_head, c.k_row, i, row[p], n), rv = rows(c.v, c.v_page, c.v_head, c.v_row, i, row[p], n);
      if constexpr (!kStaged) {
        const int ch = (tid % PPR) ^ tile_swz<D>(p * RP + tid / PPR);
        const uint32_t to = 1024u * w + 4096u * p;
        dma16(rk, k_lds + to, (uint32_t)lr * (uint32_t)c.k_row * 2 + ch * 16);
        dma16(rv, v_lds + to, (uint32_t)lr * (uint32_t)c.v_row * 2 + ch * 16);
      } else {
        load(kx[p], rk, (uint32_t)lr * (uint32_t)c.k_row + tid % PPR * (PW * 4));
        load(vx[p], rv, (uint32_t)lr * (uint32_t)c.v_row + tid % PPR * (PW * 4));
        if constexpr (MX) {
          const uint32_t o = lr * SB + tid % PPR * PE / kMxBlock;
          kb[p] = __builtin_amdgcn_raw_buffer_load_b8(scales(c.k_mx, i, row[p], n), o, 0, 0);
          vb[p] = __builtin_amdgcn_raw_buffer_load_b8(scales(c.v_mx, i, row[p], n), o, 0, 0);
        }
      }
      at[p] += KT / c.page_size;
      row[p] += KT % c.page_size;
      if (row[p] >= c.page_size) row[p] -= c.page_size, ++at[p];
      look(p);
    }
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
      const int tid = threadIdx.x, piece = tid % PPR;
#pragma unroll
      for (int p = 0; p < PARTS; ++p) {
        const int r = p * RP + tid / PPR;
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

  // ---- query rows
  __device__ int sequence(int r) const { return r / G; }
  // keys of the prefix that row r's sequence has, less those of earlier runs
  __device__ int seen(int r) const {
    const int n = clamp_len(a.c.lens[sequence(r)], a.c.table_width, a.c.page_size);
    return (n < prefix ? n : prefix) - first;
  }
  __device__ bool alive(int r) const { return r < nq && seen(r) > 0; }
  __device__ int limit(int r) const {
    if (!alive(r)) return nk;
    const int n = seen(r);
    return n < nk ? n : nk;
  }
  __device__ int least(int x) const {
    if (!__any(x < nk)) return nk;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x = min(x, __shfl_xor(x, o));
    return __builtin_amdgcn_readfirstlane(x);
  }
  __device__ bf16x8 q8(int r, int col) const {
    u32x4 x = {0, 0, 0, 0};
    if (alive(r)) x = *(const u32x4*)((const __bf16*)a.q + sequence(r) * a.qs.row + (hk * G + r % G) * a.qs.head + col);
    return as_bf16x8(x);
  }
  __device__ int o() const { return 0; }
  __device__ int lse() const { return 0; }
  __device__ int64_t part(int r) const { return ((int64_t)split * a.c.batch + sequence(r)) * a.c.heads_q + hk * G + r % G; }
  __device__ void put_o(int, int r, int col, float a0, float a1, float a2, float a3) const {
    if (r >= nq) return;
    const float f = TYPE == kE4m3 && a.c.v_scale ? a.c.v_scale[hk] : 1.f;
    f32x4 x = {a0 * f, a1 * f, a2 * f, a3 * f};
    if (!alive(r)) x = f32x4{0.f, 0.f, 0.f, 0.f};
    *(f32x4*)(a.prefix_o + part(r) * D + col) = x;
  }
  __device__ void put_l(int, int r, float m, float sum) const {
    if (r >= nq) return;
    const bool on = alive(r);
    *(float2*)(a.prefix_m + 2 * part(r)) = make_float2(on ? m : -INFINITY, on ? sum : 0.f);
  }
};

template <int D, int TYPE, int WPS>
__global__ __launch_bounds__(256, WPS) void prefix_kernel(DecodeArgs a) {
  // Workgroup -> (K/V head, run, tile of rows), each XCD a contiguous share: the row tiles
  // of a run read its keys from one L2
  const CacheArgs& c = a.c;
  const int tiles = (c.batch * (c.heads_q / c.heads_kv) + kRows - 1) / kRows;
  const int items = c.heads_kv * a.splits * tiles, per = (items + 7) >> 3;
  const int item = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || item >= items) return;
  const int hk = item / (a.splits * tiles), split = item / tiles % a.splits, q0 = item % tiles * kRows;
  const int prefix = __builtin_amdgcn_readfirstlane(prefix_of(a));
  if (item == 0 && threadIdx.x == 0 && c.status && *a.prefix_len != prefix) *c.status = 1;
  const Run run = run_of<D>(prefix, a.splits, split);
  if (split >= run.n) return;
  const PrefixView<D, TYPE> view(a, hk, prefix, run, split, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
  const float scale = a.scale * (TYPE == kE4m3 && c.k_scale ? c.k_scale[hk] : 1.f);
  attn_fwd_rows<D, 1>(view, 0, scale, q0);
  if (view.bad && (threadIdx.x & 63) == 0 && c.status) *c.status = 1;
}

// The parts of one sequence and query head, the prefix's first, each in order: thread groups of
// D / 4 lanes take every NG-th part and are added in order of the group.
template <int D>
__global__ __launch_bounds__(256) void prefix_join_kernel(DecodeArgs a) {
  constexpr int NG = 256 / (D / 4), U = 8;  // U parts' loads in flight together
  __shared__ f32x4 acc[NG][D / 4];
  __shared__ float dens[NG];
  const int hq = a.c.heads_q, s = (int)blockIdx.x / hq, h = (int)blockIdx.x % hq;
  const int np = run_of<D>(prefix_of(a), a.splits, 0).n;
  const int first = a.base[2 * s], n = np + a.base[2 * s + 1];
  const int tid = threadIdx.x, l = tid & 63, grp = tid / (D / 4), d4 = tid % (D / 4);
  // part i: its row of prefix_o and prefix_m, or of part_o and part_m
  const auto at = [&](int i) { return i < np ? ((int64_t)i * a.c.batch + s) * hq + h : (int64_t)(first + i - np) * hq + h; };
  const auto stat = [&](int i) { return *(const float2*)((i < np ? a.prefix_m : a.part_m) + 2 * at(i)); };
  float top = -INFINITY;
  for (int i = l; i < n; i += 64) top = fmaxf(top, stat(i).x);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  const float mm = top == -INFINITY ? 0.f : top;
  float den = 0.f;
  f32x4 out = {0.f, 0.f, 0.f, 0.f};
  for (int i = grp; i < n; i += U * NG) {
    float2 m[U];
    f32x4 o[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int iu = i + u * NG < n ? i + u * NG : i;  // (read again, not added)
      m[u] = stat(iu);
      o[u] = *(const f32x4*)((iu < np ? a.prefix_o : a.part_o) + at(iu) * D + 4 * d4);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * NG < n) {
        const float f = __builtin_amdgcn_exp2f(m[u].x - mm), e = f * m[u].y;
        den += e;
        out += (i + u * NG < np ? e : f) * o[u];  // (a prefix's part is over its sum already)
      }
  }
  acc[grp][d4] = out;
  if (d4 == 0) dens[grp] = den;
  __syncthreads();
  if (grp != 0) return;
#pragma unroll
  for (int i = 1; i < NG; ++i) out += acc[i][d4], den += dens[i];
  const float inv = den > 0.f || den != den ? 1.f / den : 0.f;
  *(u32x2*)((__bf16*)a.o + s * a.os.row + h * a.os.head + 4 * d4) =
      u32x2{pack_bf16(out[0] * inv, out[1] * inv), pack_bf16(out[2] * inv, out[3] * inv)};
  if (a.lse && d4 == 0) a.lse[(size_t)s * hq + h] = den == 0.f ? -INFINITY : (top + __log2f(den)) * kLn2;
}

int row_tiles(int batch, int heads_q, int heads_kv) { return (int)(((int64_t)batch * (heads_q / heads_kv) + kRows - 1) / kRows); }

template <int D, int WPS>
void launch(const DecodeArgs& a, hipStream_t stream) {
  const int64_t items = (int64_t)a.c.heads_kv * a.splits * row_tiles(a.c.batch, a.c.heads_q, a.c.heads_kv);
  const auto kernel = a.c.type == kBf16   ? prefix_kernel<D, kBf16, WPS>
                      : a.c.type == kE4m3 ? prefix_kernel<D, kE4m3, WPS>
                      : a.c.type == kMx8  ? prefix_kernel<D, kMx8, WPS>
                                          : prefix_kernel<D, kMx4, WPS>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((items + 7) / 8 * 8)), dim3(256), 0, stream, a);
  (void)launch_decode_tail(a, stream);
  hipLaunchKernelGGL(prefix_join_kernel<D>, dim3((unsigned)(a.c.batch * a.c.heads_q)), dim3(256), 0, stream, a);
}

}  // namespace

// Runs of the prefix at most: with the K/V heads and the tiles of rows, the workgroups that
// run at once on 256 CUs (two a CU, one at d = 256).
int prefix_splits(int batch, int heads_q, int heads_kv, int d, int prefix_tokens) {
  const int64_t blocks = (int64_t)heads_kv * row_tiles(batch, heads_q, heads_kv), fit = d == 256 ? 256 : 512;
  const int64_t most = prefix_tokens / kMinRun;
  int64_t s = blocks > 0 ? fit / blocks : 1;
  s = s < most ? s : most;
  return (int)(s < 1 ? 1 : s > 64 ? 64 : s);
}

int64_t prefix_waves(const DecodeArgs& a) {
  const int64_t main = ((int64_t)a.c.heads_kv * a.splits * row_tiles(a.c.batch, a.c.heads_q, a.c.heads_kv) + 8) * 4;
  const int64_t join = (int64_t)a.c.batch * a.c.heads_q * 4, tail = decode_waves(a);
  const int64_t most = main > join ? main : join;
  return most > tail ? most : tail;
}

hipError_t launch_prefix(const DecodeArgs& a, hipStream_t stream) {
  if (a.c.d == 64) launch<64, 3>(a, stream);
  else if (a.c.d == 128) launch<128, 2>(a, stream);
  else launch<256, 1>(a, stream);
  return hipGetLastError();
}

}  // namespace dash
