// decode_main.h -- the step of the one-token attention kernels: 32 keys of a paged cache
// against up to 16 query rows, by one wave, with no LDS.
//   S^T = K Q^T   (MFMA 16x16x32, twice 16 keys) A = K rows, loaded in the operand's own layout
//   P = exp(S - m), in the C layout: one query a lane, keys 4g .. 4g+3 and 16 + 4g .. +3
//   O^T += V^T P^T   B = those 8 probabilities as they are; A = V^T: lane l loads rows
//                 4g .. and 16 + 4g .. of V, D/16 columns each, and picks column by column
// (g = l / 16).  The columns of V that one lane holds are D/16 neighbours, so that
// 16 lanes read one whole row; O^T's rows come out in that order.
// P goes into that product rounded to bf16, the MFMA's operand type: each weight by 2^-8 at most, as
// much as O itself at the end.  Its sum takes it unrounded; sums, maxima and all that is
// joined stay in fp32.
// An e4m3 cache is widened to bf16, which holds every e4m3 value exactly; a microscaled one as well,
// its scales included (mx.h).
#pragma once
#include "common.h"
#include "mx.h"
#include "ops.h"
#include "page_index.h"
#include "paged.h"

namespace dash {

constexpr int kQ = 16;  // query rows of an MFMA
constexpr int kWholeWaves = 8;  // waves of a workgroup where every sequence is one chunk (workers 0); else four

// two e4m3 values of a word (its low or high half) as the upper halves of two floats
template <bool HI>
__device__ inline u32x2 widen2(unsigned x) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 f = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, HI);
  return __builtin_bit_cast(u32x2, f);
}
__device__ inline unsigned tops(unsigned a, unsigned b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ inline bf16x8 widen8(unsigned a, unsigned b) {
  const u32x2 p = widen2<false>(a), q = widen2<true>(a), r = widen2<false>(b), t = widen2<true>(b);
  return as_bf16x8(u32x4{tops(p[0], p[1]), tops(q[0], q[1]), tops(r[0], r[1]), tops(t[0], t[1])});
}

// BYTES bytes at p, in loads as wide as they allow
template <int BYTES, bool PAST>
__device__ inline void load_words(unsigned* to, const char* p) {
  if constexpr (BYTES == 2) to[0] = PAST ? __builtin_nontemporal_load((const uint16_t*)p) : *(const uint16_t*)p;
  else if constexpr (BYTES == 4) to[0] = PAST ? __builtin_nontemporal_load((const unsigned*)p) : *(const unsigned*)p;
  else if constexpr (BYTES == 8) *(u32x2*)to = PAST ? __builtin_nontemporal_load((const u32x2*)p) : *(const u32x2*)p;
  else
#pragma unroll
    for (int y = 0; y < BYTES / 4; y += 4) *(u32x4*)(to + y) = PAST ? __builtin_nontemporal_load((const u32x4*)(p + 4 * y)) : *(const u32x4*)(p + 4 * y);
}

// the scale bytes of row r of four: 1
template <int SB>
__device__ inline void unit_scale(unsigned* w, int r) {
  if constexpr (SB == 2) w[r >> 1] = r & 1 ? (w[r >> 1] & 0xffffu) | 0x7f7f0000u : (w[r >> 1] & 0xffff0000u) | 0x7f7fu;
  else
#pragma unroll
    for (int i = 0; i < SB / 4; ++i) w[r * (SB / 4) + i] = 0x7f7f7f7fu;
}

// A tile's 32 keys, as one lane holds them.  K: `PE` neighbouring components of a row at a
// time; V: VE = D / 16 columns of eight rows.
template <int D, int TYPE>
struct Tile {
  static constexpr int BITS = TYPE == kBf16 ? 16 : TYPE == kMx4 ? 4 : 8;  // of a component
  static constexpr bool MX = TYPE >= kMx8;
  static constexpr int PE = TYPE == kMx4 && D == 64 ? 16 : 128 / BITS;  // (4 PE at most a row)
  static constexpr int NK = D / (4 * PE);          // pieces of a K row per lane
  static constexpr int KW = PE * BITS / 32;        // words of a piece
  static constexpr int VB = D / 16 * BITS / 8;     // bytes of a V row per lane
  static constexpr int VW = VB < 4 ? 1 : VB / 4;
  static constexpr int SB = D / kMxBlock;          // scale bytes of a row
  unsigned k[2][NK][KW];
  unsigned v[8][VW];
  unsigned ks[MX ? 2 : 1][SB < 4 ? 1 : SB / 4];     // the scale bytes of this lane's K rows
  unsigned vs[MX ? 2 : 1][MX ? SB : 1];             // and of its V rows 4g .. 4g + 3 (SB words)

  // the component of a row at which k-step ks of lane group g begins, in K's order of d
  __device__ static int first(int ks, int g) { return 4 * PE * (ks / (PE / 8)) + PE * g + 8 * (ks % (PE / 8)); }
  // 8 components of K's rows 16 tt + l % 16, as the A operand of k-step ks
  __device__ bf16x8 key(int tt, int ks, int g) const {
    constexpr int PK = PE / 8;  // k-steps of a piece
    const unsigned* kw = k[tt][ks / PK] + ks % PK * (BITS / 4);
    if constexpr (TYPE == kE4m3) {
      return widen8(kw[0], kw[1]);
    } else if constexpr (MX) {
      // the byte of the block that this lane's components of piece ks / PK lie in
      const int blk = (4 * PE * (ks / PK) + PE * g) / kMxBlock;
      const float s = mx_scale(SB <= 4 ? ks_word(tt, 0) >> (8 * blk) & 255 : ks_word(tt, ks / PK * (4 * PE / kMxBlock) >> 2) >> (8 * (blk & 3)) & 255);
      if constexpr (TYPE == kMx4) return as_bf16x8(u32x4{mx_pair<true>(kw[0], 0, s), mx_pair<true>(kw[0], 1, s), mx_pair<true>(kw[0], 2, s), mx_pair<true>(kw[0], 3, s)});
      else return as_bf16x8(u32x4{mx_pair<false>(kw[0], 0, s), mx_pair<false>(kw[0], 1, s), mx_pair<false>(kw[1], 0, s), mx_pair<false>(kw[1], 1, s)});
    } else {
      return as_bf16x8(u32x4{kw[0], kw[1], kw[2], kw[3]});
    }
  }
  __device__ unsigned ks_word(int tt, int i) const { return this->ks[tt][i]; }
  // V's row e (of this lane's eight) reads 0
  __device__ void hide(int e) {
#pragma unroll
    for (int y = 0; y < VW; ++y) v[e][y] = 0;
    if constexpr (MX) unit_scale<SB>(vs[e >> 2], e & 3);
  }
  // f(y, column VE (l % 16) + y of the 32 rows as the A operand) for y = 0 .. VE - 1
  template <typename F>
  __device__ void columns(int lq, F&& f) const {
    constexpr int VE = D / 16;
    if constexpr (MX) {
      float scale[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {  // the byte of columns VE lq .. of row e
        const int byte = (e & 3) * SB + VE * lq / kMxBlock;  // (SB > 4: of two words, by the lane)
        unsigned word = vs[e >> 2][(e & 3) * SB >> 2];
        if constexpr (SB == 8) word = lq < 8 ? word : vs[e >> 2][2 * (e & 3) + 1];
        scale[e] = mx_scale(word >> (8 * (byte & 3)) & 255);
      }
#pragma unroll
      for (int y = 0; y < VE; y += 2) {
        constexpr int PW = 16 / BITS;  // pairs of columns in a word
        unsigned x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = mx_pair<TYPE == kMx4>(v[e][y / 2 / PW], y / 2 % PW, scale[e]);
#pragma unroll
        for (int z = 0; z < 2; ++z) f(y + z, as_bf16x8(u32x4{pick16(x[0], x[1], z), pick16(x[2], x[3], z), pick16(x[4], x[5], z), pick16(x[6], x[7], z)}));
      }
    } else if constexpr (TYPE == kE4m3) {
#pragma unroll
      for (int y = 0; y < VE; y += 2) {
        u32x2 x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (y & 2) ? widen2<true>(v[e][y >> 2]) : widen2<false>(v[e][y >> 2]);
#pragma unroll
        for (int z = 0; z < 2; ++z) f(y + z, as_bf16x8(u32x4{tops(x[0][z], x[1][z]), tops(x[2][z], x[3][z]), tops(x[4][z], x[5][z]), tops(x[6][z], x[7][z])}));
      }
    } else {
#pragma unroll
      for (int y = 0; y < VE; ++y)
        f(y, as_bf16x8(u32x4{pick16(v[0][y >> 1], v[1][y >> 1], y & 1), pick16(v[2][y >> 1], v[3][y >> 1], y & 1),
                             pick16(v[4][y >> 1], v[5][y >> 1], y & 1), pick16(v[6][y >> 1], v[7][y >> 1], y & 1)}));
    }
  }
};

// Where a wave's tiles come from: the rows of one K/V head in the pages of `table`, every `step` keys from
// `from` on (multiples of 16).  PAST: V's rows are not read again soon (a load takes a row whole): past the caches.
template <int D, int TYPE, bool PAST>
struct KeyRows {
  using T = Tile<D, TYPE>;
  static constexpr int SZ = TYPE == kBf16 ? 2 : 1;  // bytes of a stride's unit
  const CacheArgs& c;
  const int32_t* table;
  int last_page;
  // K/V head hk's first row of page 0; bytes from page to page and row to row; the scales alike
  const char *k0, *v0, *k_mx, *v_mx;
  uint64_t k_page, v_page;
  uint32_t k_row, v_row, mx_page;
  uint32_t k_lane, v_lane, ks_lane, vs_lane;  // this lane's part of a tile's rows
  int next, next_row, step_pages, step_rows;  // the place in the table of the tile after the next
  int id[2], row[2];                          // pages and rows of the next tile's two halves
  bool bad = false;
  // keys: the last one's number and one more, as the table counts
  __device__ KeyRows(const CacheArgs& c_, const int32_t* table_, int hk, int keys, int from, int step, int l)
      : c(c_), table(table_), last_page(keys > 0 ? (keys - 1) / c_.page_size : 0), k0((const char*)c_.k + hk * c_.k_head * SZ),
        v0((const char*)c_.v + hk * c_.v_head * SZ), k_page(c_.k_page * SZ), v_page(c_.v_page * SZ), k_row((uint32_t)c_.k_row * SZ),
        v_row((uint32_t)c_.v_row * SZ), k_lane((l & 15) * k_row + 4 * T::KW * (l >> 4)), v_lane(4 * (l >> 4) * v_row + (l & 15) * T::VB),
        next(from / c_.page_size), next_row(from % c_.page_size), step_pages(step / c_.page_size), step_rows(step % c_.page_size) {
    if constexpr (T::MX) {
      const int64_t head = (int64_t)hk * c.page_size * T::SB;
      k_mx = (const char*)c.k_mx + head, v_mx = (const char*)c.v_mx + head;
      mx_page = (uint32_t)c.heads_kv * c.page_size * T::SB;  // (at most 2^12 2^16 2^3)
      ks_lane = (l & 15) * T::SB, vs_lane = (l >> 4) * (4 * T::SB);
    }
    look();
  }
  // The next tile's pages, read a tile ahead: their latency is not the loads'.  (Past the last key some page
  // of the sequence, whose keys are masked.)
  __device__ void look() {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      int p = next, r = next_row + 16 * tt;
      if (tt && r >= c.page_size) r -= c.page_size, ++p;
      row[tt] = r;
      id[tt] = table_entry(table, p < last_page ? p : last_page);
    }
    next += step_pages;
    next_row += step_rows;
    if (next_row >= c.page_size) next_row -= c.page_size, ++next;
  }
  __device__ void load(T& t) {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const uint32_t r = row[tt];
      uint32_t i = id[tt];
      if (!page_ok(i, c.pages)) bad = true, i = 0;
      const char* kp = k0 + (i * k_page + (uint64_t)r * k_row);
      const char* vp = v0 + (i * v_page + (uint64_t)r * v_row);
#pragma unroll
      for (int x = 0; x < T::NK; ++x) load_words<4 * T::KW, false>(t.k[tt][x], kp + k_lane + 16 * T::KW * x);
#pragma unroll
      for (int x = 0; x < 4; ++x) load_words<T::VB, PAST>(t.v[4 * tt + x], vp + v_lane + x * v_row);
      if constexpr (T::MX) {
        const uint64_t at = (uint64_t)i * mx_page + r * T::SB;
        load_words<T::SB, false>(t.ks[tt], k_mx + at + ks_lane);
        load_words<4 * T::SB, false>(t.vs[tt], v_mx + at + vs_lane);
      }
    }
  }
};

// The running result of 16 query rows, row l % 16 in this lane.  o[y][r]: column
// VE (4g + r) + y of O^T; sum: over this lane's keys.
template <int D>
struct Rows {
  static constexpr int KS = D / 32, VE = D / 16;  // MFMA k-steps over d; columns of V per lane
  bf16x8 q[KS];
  f32x4 o[VE];
  float m, sum;
  __device__ void clear() {
#pragma unroll
    for (int y = 0; y < VE; ++y) o[y] = f32x4{0.f, 0.f, 0.f, 0.f};
    m = -INFINITY;
    sum = 0.f;
  }
  // The 32 keys of t, whose first is kb: those from `from` to `to` - 1.
  template <int TYPE>
  __device__ void add(Tile<D, TYPE>& t, float c2, int kb, int from, int to, int lq, int g) {
    f32x4 sc[2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      sc[tt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) sc[tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(t.key(tt, ks, g), q[ks], sc[tt], 0, 0, 0);
    }
    // S in the log2 domain, rounded before the maximum is taken off, so that the
    // largest gives exactly 1 however far from 0 it is
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = sc[e >> 2][e & 3] * c2;
      asm("" : "+v"(x[e]));
    }
    if (kb + 32 > to || kb < from) {  // other keys: no weight, and whatever V holds there is not touched
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int key = kb + 16 * (e >> 2) + 4 * g + (e & 3);
        if (key >= to || key < from) {
          x[e] = -INFINITY;
          t.hide(e);
        }
      }
    }
    float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    mx = quad_max(mx);
    if (__any(mx > m)) {
      const float mn = fmaxf(m, mx);
      const float alpha = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      sum *= alpha;
#pragma unroll
      for (int y = 0; y < VE; ++y) o[y] *= alpha;
    }
    const float mm = m == -INFINITY ? 0.f : m;  // (nothing but -inf so far: P = 0)
    float p[8], add = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) add += p[e] = __builtin_amdgcn_exp2f(x[e] - mm);
    sum += add;
    const bf16x8 pb = as_bf16x8(u32x4{pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7])});
    t.columns(lq, [&](int y, bf16x8 vt) { o[y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, pb, o[y], 0, 0, 0); });
  }
};

template <int D, int NW>
struct JoinSpace {
  float o[NW][kQ][D + 4];  // (rows padded)
  float m[NW][kQ], sum[NW][kQ];
};
// The waves' results of 16 rows: put(row, first of four columns, maximum, sum, O) for rows 0 .. nq - 1.
// o[y][r] is column VE (4g + r) + y of row l % 16.
template <int D, int NW, typename F>
__device__ inline void join_waves(JoinSpace<D, NW>& s, const f32x4 (&o)[D / 16], float m, float sum, int w, int nq, F&& put) {
  constexpr int VE = D / 16;
  const int tid = threadIdx.x, l = tid & 63, g = l >> 4, lq = l & 15;
  sum = quad_sum(sum);
  if (g == 0) s.m[w][lq] = m, s.sum[w][lq] = sum;
#pragma unroll
  for (int y = 0; y < VE; ++y)
#pragma unroll
    for (int r = 0; r < 4; ++r) s.o[w][lq][VE * (4 * g + r) + y] = o[y][r];
  __syncthreads();
  for (int e = tid; e < nq * (D / 4); e += 64 * NW) {
    const int q = e / (D / 4), d0 = e % (D / 4) * 4;
    float top = s.m[0][q];
#pragma unroll
    for (int x = 1; x < NW; ++x) top = fmaxf(top, s.m[x][q]);
    const float mm = top == -INFINITY ? 0.f : top;
    float den = 0.f;
    f32x4 out = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < NW; ++x) {
      const float f = __builtin_amdgcn_exp2f(s.m[x][q] - mm);
      den += f * s.sum[x][q];
      out += f * *(const f32x4*)&s.o[x][q][d0];
    }
    put(q, d0, top, den, out);
  }
}

// One workgroup's chunk of one sequence's keys, for one K/V head and up to 16 of its query heads.
// TYPE: of the cache.  TAIL: the keys behind a shared prefix alone, whose result is always
// left as a part, to be joined with the prefix's.
template <int D, int TYPE, int NW, bool TAIL>
__device__ inline void decode_part(const DecodeArgs& a, int block, JoinSpace<D, NW>& space) {
  constexpr bool F8 = TYPE == kE4m3;
  constexpr int KS = D / 32;        // MFMA k-steps over d
  const CacheArgs& c = a.c;
  const int tid = threadIdx.x, l = tid & 63, g = l >> 4, lq = l & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = c.heads_q / c.heads_kv, qtiles = (G + kQ - 1) / kQ;
  const int units = c.heads_kv * qtiles;
  const int slot = block / units, unit = block % units;
  const int hk = unit / qtiles, q0 = unit % qtiles * kQ;
  const int nq = G - q0 < kQ ? G - q0 : kQ;  // query heads h0 .. h0 + nq - 1
  const int h0 = hk * G + q0;

  // TAIL: keys from the prefix's end on, counted from the 16 that it lies in (none: none, not the prefix's last few, for which
  // a sequence need not have a page); a sequence that is shorter does without the prefix
  const int prefix = TAIL ? prefix_of(a) : 0;
  const auto keys_in = [&](int length) {
    const int n = clamp_len(length, c.table_width, c.page_size);
    return !TAIL || n < prefix ? n : n > prefix ? n - (prefix & ~15) : 0;
  };
  const auto keys_of = [&](int b) { return keys_in(c.lens[b]); };

  // ---- the workgroup's sequence s, its chunk number i of n, and where the sequence's parts begin.  First all chunks of at
  // least half the size, then the shorter rests of sequences: what starts late is short (32 heads over 8 of 128, us,
  // in the sequences' order / so / whole chunks first: 64 sequences of 131072 keys in bf16 106 / 100 / 106 and in MXFP8
  // 68 / 61 / 65, of 66000 38 / 37 / 39, 128 of 131072 73 / 70 / 74, 65 of 66000 38.4 / 39.8 / 40.5).
  // (Sequences that are one chunk each: the workgroup's number, without a search: one of 28 keys, 8 heads over 2 of 64, 3.7 us and
  // 400 of 100 keys 9.0; with a search over all lengths 4.3 and 17.)
  int s = slot, i = 0, n = 1, base = slot, chunk = kMaxKeys, len = 0;
  if constexpr (NW == kWholeWaves) {
    len = keys_of(slot);
  } else {
    s = base = 0;
    len = l < c.batch ? keys_of(l) : 0;
    long sum = len;
#pragma unroll 8
    for (int b = l + 64; b < c.batch; b += 64) sum += keys_of(b);
    const long total = wave_sum((int)(sum >> 24)) * (1l << 24) + wave_sum((int)(sum & 0xffffff));  // (a table's keys: below 2^54)
    chunk = __builtin_amdgcn_readfirstlane(chunk_size(total, a.workers));
    // Among `count` sequences from s on, each lane takes a 64th of them, in order; the lane that holds the chunk
    // leaves its share to the next round (one round up to 64 sequences, two up to 4096).
    int want = slot;
    bool rest = false;
    for (int count = c.batch;;) {
      const int per = (count + 63) >> 6;
      int mine = 0, first = 0;  // chunks of this lane's share, and those among them that come first
      const auto add = [&](int keys) {
        const int m = chunks_of(keys, chunk);
        mine += m, first += m - ((unsigned)m * (unsigned)chunk - (unsigned)keys > (unsigned)chunk / 2);  // (32 bits, as chunks_of)
      };
      if (per == 1) {
        if (c.batch > 64) len = keys_of(s + (l < count ? l : 0));
        if (l < count) add(len);
      } else {
        // four neighbours a load (the batch's last four where fewer follow): the lanes' shares lie a line or more apart
        // (4096 sequences of 100 keys, 8 heads over 2 of 64, us: one a load 523, four 233)
        typedef int lens4 __attribute__((ext_vector_type(4), aligned(4)));
        const int from = s + l * per, to = s + (l * per + per < count ? l * per + per : count);
#pragma unroll 1
        for (int j = from; j < from + per; j += 4) {
          const int p = j < c.batch - 4 ? j : c.batch - 4;
          const lens4 x = *(const lens4*)(c.lens + p);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (p + e >= j && p + e < to) add(keys_in(x[e]));
        }
      }
      const int mines = wave_scan(mine), firsts = wave_scan(first);
      if (count == c.batch) {
        const int all = __builtin_amdgcn_readlane(firsts, 63);
        rest = slot >= all;
        want = rest ? slot - all : slot;
      }
      const int own = rest ? mine - first : first, upto = rest ? mines - firsts : firsts;
      const unsigned long long here = __ballot(upto > want);
      if (!here) return;  // (in the first round: no such chunk)
      const int at = __builtin_ctzll(here);
      want -= __builtin_amdgcn_readlane(upto - own, at);
      base += __builtin_amdgcn_readlane(mines - mine, at);
      s += at * per;
      if (per == 1) {
        n = __builtin_amdgcn_readlane(mine, at);
        i = rest ? __builtin_amdgcn_readlane(first, at) : want;
        len = __builtin_amdgcn_readlane(len, at);
        break;
      }
      count = count - at * per < per ? count - at * per : per;
    }
  }
  s = __builtin_amdgcn_readfirstlane(s);  // wave-uniform: tables are read and addresses made by the scalar unit
  n = __builtin_amdgcn_readfirstlane(n);
  i = __builtin_amdgcn_readfirstlane(i);
  len = __builtin_amdgcn_readfirstlane(len);
  base = __builtin_amdgcn_readfirstlane(base);
  const int skip = TAIL && has_prefix(c, s, prefix) ? __builtin_amdgcn_readfirstlane(prefix) : 0, skip16 = skip & ~15;
  const int k0 = skip16 + i * chunk, k1 = skip16 + (len - i * chunk < chunk ? len : i * chunk + chunk);
  if (unit == 0 && i == 0 && tid == 0) {
    a.base[2 * s] = base;
    a.base[2 * s + 1] = n;
    if (c.status && c.lens[s] != (TAIL ? clamp_len(c.lens[s], c.table_width, c.page_size) : len)) *c.status = 1;
  }

  // ---- Q: lane l holds query head h0 + l % 16 (zero past the group), in K's order of d
  Rows<D> rows;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const u32x4 x = *(const u32x4*)((const __bf16*)a.q + s * a.qs.row + (h0 + (lq < nq ? lq : 0)) * a.qs.head + Tile<D, TYPE>::first(ks, g));
    rows.q[ks] = as_bf16x8(lq < nq ? x : u32x4{0, 0, 0, 0});
  }
  rows.clear();
  const float c2 = a.scale * kLog2e * (F8 && c.k_scale ? c.k_scale[hk] : 1.f);

  // ---- tiles of 32 keys (those of further 16 query heads read the same keys again, V from memory)
  if (k0 + 32 * w < k1) {
    KeyRows<D, TYPE, true> keys(c, c.table + (int64_t)s * c.table_stride, hk, skip16 + len, k0 + 32 * w, 32 * NW, l);
    for (int kb = k0 + 32 * w; kb < k1; kb += 32 * NW) {
      Tile<D, TYPE> t;
      keys.load(t);
      keys.look();
      rows.add(t, c2, kb, skip, k1, lq, g);
    }
    if (keys.bad && l == 0 && c.status) *c.status = 1;
  }

  const float vs = F8 && c.v_scale ? c.v_scale[hk] : 1.f;
  join_waves<D, NW>(space, rows.o, rows.m, rows.sum, w, nq, [&](int q, int d0, float top, float den, f32x4 out) {
    if (!TAIL && n == 1) {
      const float inv = den > 0.f || den != den ? vs / den : 0.f;
      *(u32x2*)((__bf16*)a.o + s * a.os.row + (h0 + q) * a.os.head + d0) =
          u32x2{pack_bf16(out[0] * inv, out[1] * inv), pack_bf16(out[2] * inv, out[3] * inv)};
      if (a.lse && d0 == 0) a.lse[(size_t)s * c.heads_q + h0 + q] = den == 0.f ? -INFINITY : (top + __log2f(den)) * kLn2;
    } else {
      const size_t at = (size_t)(base + i) * c.heads_q + h0 + q;
      *(f32x4*)(a.part_o + at * D + d0) = out * vs;
      if (d0 == 0) a.part_m[2 * at] = top, a.part_m[2 * at + 1] = den;
    }
  });
}

}  // namespace dash
