// attn_decode.hip -- attention of one new token per sequence over a paged
// key-value cache, split over the cache's length and joined.
//
//   o_h = sum_j softmax_j(scale q_h . k_j) v_j over the lens[s] cached keys
//
// Bound by memory: K and V are read once for every 16 query heads of a K/V head (with more,
// each 16 are a workgroup of their own), 4 d bytes a key and head (2 d in e4m3),
// for 4 d G operations, G query heads to a K/V head.  So the kernel's business is
// to keep loads in flight.  One workgroup takes a chunk of one sequence's keys for
// one K/V head and up to 16 of its query heads; each of its four waves takes every
// fourth tile of 32 keys by itself, with its own running maximum and sum; the other
// waves' loads are in flight meanwhile (8 to 16 waves a CU, 16 KB each at d = 128; a
// second tile ahead in registers leaves fewer waves and gains nothing: 538 MB 111 us with it
// and without).  Nothing goes through LDS until the four waves are joined:
//   S^T = K Q^T   (MFMA 16x16x32, twice 16 keys) A = K rows, loaded in the operand's own layout
//   P = exp(S - m), in the C layout: one query a lane, keys 4g .. 4g+3 and 16 + 4g .. +3
//   O^T += V^T P^T   B = those 8 probabilities as they are; A = V^T: lane l loads rows
//                 4g .. and 16 + 4g .. of V, D/16 columns each, and picks column by column
// (g = l / 16).  The columns of V that one lane holds are D/16 neighbours, so that
// 16 lanes read one whole row; O^T's rows come out in that order.
// P goes into that product rounded to bf16, the MFMA's operand type: each weight by 2^-8 at most, as
// much as O itself at the end.  Its sum takes it unrounded; sums, maxima and all that is
// joined stay in fp32.
// An e4m3 cache is widened to bf16, which holds every e4m3 value exactly; K's scale goes into
// the softmax scale and V's into the output.
//
// The keys of all sequences are cut into chunks of one size, found on the device
// from lens (so that a captured call follows them): the sum over `workers`.  A sequence of one chunk is written at once; the others' chunks leave
// (m, sum, O) in fp32 and join_kernel adds them in order.  The chunk size, and so
// the order of the sums, is fixed by lens and the call's shape, never by timing.
// (Chunks of at least 128 keys: one tile for each wave.)
//
// Measured, 32 heads over 8 of 128: 131072 keys of 64 sequences in bf16 97 us, 5.5 TB/s,
// and 5 us of joins; of one sequence in e4m3 43 us, 6.2 TB/s, and 6.4; 901 keys, 8 heads over 2 of
// 64, whole, 8.9 us (four tiles a wave, one after the other).
#include "common.h"
#include "mx.h"
#include "ops.h"
#include "page_index.h"
#include "paged.h"

namespace dash {
namespace {

constexpr int kQ = 16;      // query heads of a workgroup

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
};
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

// TYPE: of the cache.  TAIL: the keys behind a shared prefix alone, whose result is always
// left as a part, to be joined with the prefix's.
template <int D, int TYPE, int NW, bool TAIL>
__global__ __launch_bounds__(64 * NW, 2) void decode_kernel(DecodeArgs a) {
  using T = Tile<D, TYPE>;
  constexpr bool F8 = TYPE == kE4m3;
  constexpr int KS = D / 32;        // MFMA k-steps over d
  constexpr int VE = D / 16;        // columns of V per lane = 16-row blocks of O^T
  constexpr int SZ = TYPE == kBf16 ? 2 : 1;  // bytes of a stride's unit
  constexpr int OP = D + 4;         // padded row of the join buffer
  __shared__ float so[NW][kQ][OP];
  __shared__ float sm[NW][kQ], sl[NW][kQ];
  const CacheArgs& c = a.c;
  const int tid = threadIdx.x, l = tid & 63, g = l >> 4, lq = l & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = c.heads_q / c.heads_kv, qtiles = (G + kQ - 1) / kQ;
  const int units = c.heads_kv * qtiles;
  const int slot = (int)blockIdx.x / units, unit = (int)blockIdx.x % units;
  const int hk = unit / qtiles, q0 = unit % qtiles * kQ;
  const int nq = G - q0 < kQ ? G - q0 : kQ;  // query heads h0 .. h0 + nq - 1
  const int h0 = hk * G + q0;

  // the first key that this call does itself, and the 16 keys that it lies in
  const int skip = TAIL ? prefix_of(a) : 0, skip16 = skip & ~15;
  const auto keys_of = [&](int b) {
    const int n = clamp_len(c.lens[b], c.table_width, c.page_size);
    return TAIL ? (n > skip16 ? n - skip16 : 0) : n;
  };

  // ---- the slot's sequence s, its chunk number i of n
  long total = 0;
  int len = 0;
  for (int b = 0; b < c.batch; b += 64) {
    len = b + l < c.batch ? keys_of(b + l) : 0;
    total += wave_sum(len >> 12) * 4096l + wave_sum(len & 4095);
  }
  const int chunk = __builtin_amdgcn_readfirstlane(chunk_size(total, a.workers));
  int s = -1, i = 0, n = 0;
  for (int b = 0, before = 0; b < c.batch; b += 64) {
    if (c.batch > 64) len = b + l < c.batch ? keys_of(b + l) : 0;
    const int mine = b + l < c.batch ? chunks_of(len, chunk) : 0;
    const int upto = wave_scan(mine);
    const unsigned long long here = __ballot(before + upto > slot);
    if (here) {
      const int at = __builtin_ctzll(here);
      s = b + at;
      n = __builtin_amdgcn_readlane(mine, at);
      i = slot - (before + __builtin_amdgcn_readlane(upto, at) - n);
      len = __builtin_amdgcn_readlane(len, at);
      break;
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  if (s < 0) return;
  s = __builtin_amdgcn_readfirstlane(s);  // wave-uniform: tables are read and addresses made by the scalar unit
  n = __builtin_amdgcn_readfirstlane(n);
  i = __builtin_amdgcn_readfirstlane(i);
  len = __builtin_amdgcn_readfirstlane(len);
  const int k0 = skip16 + i * chunk, k1 = skip16 + (len - i * chunk < chunk ? len : i * chunk + chunk);
  if (unit == 0 && i == 0 && tid == 0) {
    a.base[2 * s] = slot;
    a.base[2 * s + 1] = n;
    if (c.status && c.lens[s] != (TAIL ? clamp_len(c.lens[s], c.table_width, c.page_size) : len)) *c.status = 1;
  }

  // ---- Q: lane l holds query head h0 + l % 16 (zero past the group), in K's order of d
  bf16x8 qf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const int d0 = 4 * T::PE * (ks / (T::PE / 8)) + T::PE * g + 8 * (ks % (T::PE / 8));
    const u32x4 x = *(const u32x4*)((const __bf16*)a.q + s * a.qs.row + (h0 + (lq < nq ? lq : 0)) * a.qs.head + d0);
    qf[ks] = as_bf16x8(lq < nq ? x : u32x4{0, 0, 0, 0});
  }
  const float c2 = a.scale * kLog2e * (F8 && c.k_scale ? c.k_scale[hk] : 1.f);

  // ---- tiles of 32 keys
  const int32_t* table = c.table + (int64_t)s * c.table_stride;
  const int last_page = len > 0 ? (skip16 + len - 1) / c.page_size : 0;
  const char* kbase = (const char*)c.k + hk * c.k_head * SZ;
  const char* vbase = (const char*)c.v + hk * c.v_head * SZ;
  const uint32_t k_lane = (uint32_t)(lq * (int)c.k_row * SZ + 4 * T::KW * g);
  const uint32_t v_lane = (uint32_t)(4 * g * (int)c.v_row * SZ + lq * T::VB);
  bool bad = false;
  auto load = [&](T& t, int kb) {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const int key = kb + 16 * tt;
      int p = key / c.page_size;
      const int r = key - p * c.page_size;
      p = p < last_page ? p : last_page;  // (keys behind the last are masked)
      int id = table[p];
      if (!page_ok(id, c.pages)) bad = true, id = 0;
      const char* kp = kbase + (id * c.k_page + r * c.k_row) * SZ;
      const char* vp = vbase + (id * c.v_page + r * c.v_row) * SZ;
#pragma unroll
      for (int x = 0; x < T::NK; ++x) load_words<4 * T::KW, false>(t.k[tt][x], kp + k_lane + 16 * T::KW * x);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const char* at = vp + v_lane + x * (uint32_t)((int)c.v_row * SZ);
        unsigned* v = t.v[4 * tt + x];
        // this workgroup does not read V's rows again (those of further 16 query heads do, from
        // memory), and one load takes a row whole: past the caches
        load_words<T::VB, true>(v, at);
      }
      if constexpr (T::MX) {
        const int64_t row = ((int64_t)id * c.heads_kv + hk) * c.page_size + r;
        load_words<T::SB, false>(t.ks[tt], (const char*)c.k_mx + (row + lq) * T::SB);
        load_words<4 * T::SB, false>(t.vs[tt], (const char*)c.v_mx + (row + 4 * g) * T::SB);
      }
    }
  };
  f32x4 o[VE];
#pragma unroll
  for (int x = 0; x < VE; ++x) o[x] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, sum = 0.f;  // of this lane's query; sum: over this lane's keys
  auto compute = [&](T& t, int kb) {
    f32x4 sc[2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      sc[tt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        constexpr int PK = T::PE / 8;  // k-steps of a piece
        const unsigned* kw = t.k[tt][ks / PK] + ks % PK * (T::BITS / 4);
        bf16x8 kf;
        if constexpr (F8) {
          kf = widen8(kw[0], kw[1]);
        } else if constexpr (T::MX) {
          // the byte of the block that this lane's components of piece ks / PK lie in
          const int blk = (4 * T::PE * (ks / PK) + T::PE * g) / kMxBlock;
          const float sc8 = mx_scale(T::SB <= 4 ? t.ks[tt][0] >> (8 * blk) & 255 : t.ks[tt][ks / PK * (4 * T::PE / kMxBlock) >> 2] >> (8 * (blk & 3)) & 255);
          if constexpr (TYPE == kMx4) kf = as_bf16x8(u32x4{mx_pair<true>(kw[0], 0, sc8), mx_pair<true>(kw[0], 1, sc8), mx_pair<true>(kw[0], 2, sc8), mx_pair<true>(kw[0], 3, sc8)});
          else kf = as_bf16x8(u32x4{mx_pair<false>(kw[0], 0, sc8), mx_pair<false>(kw[0], 1, sc8), mx_pair<false>(kw[1], 0, sc8), mx_pair<false>(kw[1], 1, sc8)});
        } else {
          kf = as_bf16x8(u32x4{kw[0], kw[1], kw[2], kw[3]});
        }
        sc[tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[ks], sc[tt], 0, 0, 0);
      }
    }
    // S in the log2 domain, rounded before the maximum is taken off, so that the
    // largest gives exactly 1 however far from 0 it is
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = sc[e >> 2][e & 3] * c2;
      asm("" : "+v"(x[e]));
    }
    if (kb + 32 > k1 || (TAIL && kb < skip)) {  // keys behind the chunk's last: no weight, and whatever V holds there is not touched
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int key = kb + 16 * (e >> 2) + 4 * g + (e & 3);
        if (key >= k1 || (TAIL && key < skip)) {
          x[e] = -INFINITY;
#pragma unroll
          for (int y = 0; y < T::VW; ++y) t.v[e][y] = 0;
          if constexpr (T::MX) unit_scale<T::SB>(t.vs[e >> 2], e & 3);
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
    if constexpr (T::MX) {
      float vsc[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {  // the byte of columns VE lq .. of row e
        const int byte = (e & 3) * T::SB + VE * lq / kMxBlock;  // (SB > 4: of two words, by the lane)
        unsigned word = t.vs[e >> 2][(e & 3) * T::SB >> 2];
        if constexpr (T::SB == 8) word = lq < 8 ? word : t.vs[e >> 2][2 * (e & 3) + 1];
        vsc[e] = mx_scale(word >> (8 * (byte & 3)) & 255);
      }
#pragma unroll
      for (int y = 0; y < VE; y += 2) {
        constexpr int PW = 16 / T::BITS;  // pairs of columns in a word
        unsigned f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = mx_pair<TYPE == kMx4>(t.v[e][y / 2 / PW], y / 2 % PW, vsc[e]);
#pragma unroll
        for (int z = 0; z < 2; ++z)
          o[y + z] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              as_bf16x8(u32x4{pick16(f[0], f[1], z), pick16(f[2], f[3], z), pick16(f[4], f[5], z), pick16(f[6], f[7], z)}), pb, o[y + z], 0, 0, 0);
      }
    } else if constexpr (!F8) {
#pragma unroll
      for (int y = 0; y < VE; ++y)
        o[y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            as_bf16x8(u32x4{pick16(t.v[0][y >> 1], t.v[1][y >> 1], y & 1), pick16(t.v[2][y >> 1], t.v[3][y >> 1], y & 1),
                            pick16(t.v[4][y >> 1], t.v[5][y >> 1], y & 1), pick16(t.v[6][y >> 1], t.v[7][y >> 1], y & 1)}),
            pb, o[y], 0, 0, 0);
    } else {
#pragma unroll
      for (int y = 0; y < VE; y += 2) {
        u32x2 f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (y & 2) ? widen2<true>(t.v[e][y >> 2]) : widen2<false>(t.v[e][y >> 2]);
#pragma unroll
        for (int z = 0; z < 2; ++z)
          o[y + z] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              as_bf16x8(u32x4{tops(f[0][z], f[1][z]), tops(f[2][z], f[3][z]), tops(f[4][z], f[5][z]), tops(f[6][z], f[7][z])}),
              pb, o[y + z], 0, 0, 0);
      }
    }
  };
  for (int kb = k0 + 32 * w; kb < k1; kb += 32 * NW) {
    T t;
    load(t, kb);
    compute(t, kb);
  }
  if (bad && l == 0 && c.status) *c.status = 1;

  // ---- join the waves: o[y][r] is column VE (4g + r) + y of query l % 16
  sum = quad_sum(sum);
  if (g == 0) sm[w][lq] = m, sl[w][lq] = sum;
#pragma unroll
  for (int y = 0; y < VE; ++y)
#pragma unroll
    for (int r = 0; r < 4; ++r) so[w][lq][VE * (4 * g + r) + y] = o[y][r];
  __syncthreads();
  const float vs = F8 && c.v_scale ? c.v_scale[hk] : 1.f;
  for (int e = tid; e < nq * (D / 4); e += 64 * NW) {
    const int q = e / (D / 4), d0 = e % (D / 4) * 4;
    float top = sm[0][q];
#pragma unroll
    for (int x = 1; x < NW; ++x) top = fmaxf(top, sm[x][q]);
    const float mm = top == -INFINITY ? 0.f : top;
    float den = 0.f;
    f32x4 out = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < NW; ++x) {
      const float f = __builtin_amdgcn_exp2f(sm[x][q] - mm);
      den += f * sl[x][q];
      out += f * *(const f32x4*)&so[x][q][d0];
    }
    if (!TAIL && n == 1) {
      const float inv = den > 0.f || den != den ? vs / den : 0.f;
      *(u32x2*)((__bf16*)a.o + s * a.os.row + (h0 + q) * a.os.head + d0) =
          u32x2{pack_bf16(out[0] * inv, out[1] * inv), pack_bf16(out[2] * inv, out[3] * inv)};
      if (a.lse && d0 == 0) a.lse[(size_t)s * c.heads_q + h0 + q] = den == 0.f ? -INFINITY : (top + __log2f(den)) * kLn2;
    } else {
      const size_t at = (size_t)slot * c.heads_q + h0 + q;
      *(f32x4*)(a.part_o + at * D + d0) = out * vs;
      if (d0 == 0) a.part_m[2 * at] = top, a.part_m[2 * at + 1] = den;
    }
  }
}

// The chunks of one sequence and query head, in order: thread groups of D/4 lanes
// take every NG-th chunk and are added in order of the group.  Bound by latency: 128 chunks
// of 32 heads 8.6 us with one chunk's loads in flight, 6.7 with four, 6.4 with eight.
template <int D>
__global__ __launch_bounds__(256) void join_kernel(DecodeArgs a) {
  constexpr int NG = 256 / (D / 4), U = 8;  // U chunks' loads in flight together
  __shared__ f32x4 acc[NG][D / 4];
  __shared__ float dens[NG];
  const int hq = a.c.heads_q, s = (int)blockIdx.x / hq, h = (int)blockIdx.x % hq;
  const int first = a.base[2 * s], n = a.base[2 * s + 1];
  if (n == 1) return;  // decode_kernel has written it
  const int tid = threadIdx.x, l = tid & 63, grp = tid / (D / 4), d4 = tid % (D / 4);
  const float* pm = a.part_m + 2 * ((size_t)first * hq + h);
  float top = -INFINITY;
  for (int i = l; i < n; i += 64) top = fmaxf(top, pm[2 * (size_t)i * hq]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  const float mm = top == -INFINITY ? 0.f : top;
  float den = 0.f;
  f32x4 out = {0.f, 0.f, 0.f, 0.f};
  for (int i = grp; i < n; i += U * NG) {
    float m[U], e[U];
    f32x4 o[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int iu = i + u * NG < n ? i + u * NG : i;  // (read again, not added)
      m[u] = pm[2 * (size_t)iu * hq];
      e[u] = pm[2 * (size_t)iu * hq + 1];
      o[u] = *(const f32x4*)(a.part_o + ((size_t)(first + iu) * hq + h) * D + 4 * d4);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * NG < n) {
        const float f = __builtin_amdgcn_exp2f(m[u] - mm);
        den += f * e[u];
        out += f * o[u];
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

template <int D, int NW, bool TAIL>
void launch_main(const DecodeArgs& a, hipStream_t stream) {
  const int G = a.c.heads_q / a.c.heads_kv;
  const unsigned grid = (unsigned)a.slots * a.c.heads_kv * ((G + kQ - 1) / kQ);
  const auto kernel = a.c.type == kBf16   ? decode_kernel<D, kBf16, NW, TAIL>
                      : a.c.type == kE4m3 ? decode_kernel<D, kE4m3, NW, TAIL>
                      : a.c.type == kMx8  ? decode_kernel<D, kMx8, NW, TAIL>
                                          : decode_kernel<D, kMx4, NW, TAIL>;
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(64 * NW), 0, stream, a);
}

template <int D>
void launch(const DecodeArgs& a, hipStream_t stream) {
  if (a.workers == 0) return launch_main<D, 8, false>(a, stream);
  launch_main<D, 4, false>(a, stream);
  if (a.slots > a.c.batch)  // (else no sequence can have two chunks)
    hipLaunchKernelGGL(join_kernel<D>, dim3((unsigned)(a.c.batch * a.c.heads_q)), dim3(256), 0, stream, a);
}

template <int D>
void launch_tail(const DecodeArgs& a, hipStream_t stream) {
  if (a.workers == 0) launch_main<D, 8, true>(a, stream);
  else launch_main<D, 4, true>(a, stream);
}

}  // namespace

// Chunks aimed at, over all sequences: with the K/V heads (and further groups of
// 16 query heads) about 1024 workgroups, four for each of 256 CUs.
// 0: each sequence is one chunk of eight waves, written at once -- tables of up to
// 65536 / d keys, for which the second kernel costs more than the waves' further tiles
// (us with the host's part, whole / cut: 1 sequence of 1000, 2 heads of 64, 10.9 / 12.0; 8 of 500, 8 heads
// of 128, 10.2 / 11.7, in e4m3 9.9 / 12.2; 4 of 200, 4 heads of 256, 10.0 / 11.9; but 1 of 1000, 8 heads
// of 128, 13.6 / 12.0, 8 of 1000 in e4m3 14.1 / 12.2, 4 of 500, 4 heads of 256, 17.8 / 11.7).
int decode_workers(int heads_q, int heads_kv, int d, int table_tokens) {
  if (table_tokens <= 65536 / d) return 0;
  const int units = heads_kv * ((heads_q / heads_kv + kQ - 1) / kQ);
  return units < 1024 ? 1024 / units : 1;
}
int decode_slots(int batch, int heads_q, int heads_kv, int d, int table_tokens) {
  const long most = table_tokens > kMinChunk ? (long)batch * ((table_tokens + kMinChunk - 1) / kMinChunk) : batch;
  const long s = (long)decode_workers(heads_q, heads_kv, d, table_tokens) + batch;
  return (int)(s < most ? s : most);
}

int64_t decode_waves(const DecodeArgs& a) {
  const int64_t G = a.c.heads_q / a.c.heads_kv, main = (int64_t)a.slots * a.c.heads_kv * ((G + kQ - 1) / kQ) * (a.workers == 0 ? 8 : 4);
  const int64_t join = a.slots > a.c.batch ? (int64_t)a.c.batch * a.c.heads_q * 4 : 0;
  return main > join ? main : join;
}

hipError_t launch_decode_tail(const DecodeArgs& a, hipStream_t stream) {
  if (a.c.d == 64) launch_tail<64>(a, stream);
  else if (a.c.d == 128) launch_tail<128>(a, stream);
  else launch_tail<256>(a, stream);
  return hipGetLastError();
}

hipError_t launch_decode(const DecodeArgs& a, hipStream_t stream) {
  if (a.c.d == 64) launch<64>(a, stream);
  else if (a.c.d == 128) launch<128>(a, stream);
  else launch<256>(a, stream);
  return hipGetLastError();
}

}  // namespace dash
