// kv_append.hip -- new keys and values into a paged cache, keys (and queries)
// rotated by their position on the way.
//
// Token t of sequence s stands at place p = lens[s] + (t - cu[s]).  Pair i of a
// head's first `rotary` components turns by the angle p f_i:
//   (x, y) -> (x cos - y sin, x sin + y cos),
// pairs being (i, i + rotary / 2), or (2i, 2i + 1) when interleaved.  The angle is
// reduced in 64 bits: at p = 10^5 a product in 32 bits is off by 2^-24 10^5 = 0.006
// radians, more than a bf16 rounding.  The rest is 32 bits with one rounding at the
// store (bf16, or value / scale[head] in e4m3).  Keys for a microscaled cache are rotated in 64 bits and
// stored with their block's scale byte (mx.h), found from the largest of four chunks through LDS.
//
// Bound by memory for prompts (q, k, v in, q and the cache rows out) and by the
// launch for single tokens.  One wave per token: it takes sine and cosine of every
// pair once (through LDS, for all heads), then 64 items a round: two 16-byte chunks of
// a head that hold 8 whole pairs, so that a lane never needs another lane's data and
// q_out may be q.  Calls with few
// tokens give each wave one round only, and the waves of a token redo its sines.
//
// Measured, heads of 128, 32 over 8: 8192 tokens into an e4m3 cache 40 us, 101 MB in and 84
// out, 4.6 TB/s, and into an MXFP8 cache 40.7 us, 101 MB and 85; 3001 tokens into an MXFP4 cache 17.6 us, 37 MB and
// 28; one token of each of 64 sequences, bf16, 4.4 us (1.6 MB).
#include <type_traits>

#include "common.h"
#include "ops.h"
#include "page_index.h"
#include "mx.h"
#include "paged.h"
#include "rotate.h"

namespace dash {
namespace {

constexpr int kWaves = 4;

// 4 values -> e4m3, saturated at 448 (a NaN stays one)
__device__ inline unsigned pack_e4m3(const float* x) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = x[i] != x[i] ? x[i] : __builtin_amdgcn_fmed3f(x[i], -448.f, 448.f);
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], r, true);
}

// ONCE: inputs larger than the last-level cache can hold behind the kernel that made
// them are read past the caches (and, MX, its rotated rows written past them).  MX: the cache is
// microscaled, 1 in 8 bits and 2 in 4 (0: bf16 or e4m3).
template <int D, bool ONCE, int MX>
__global__ __launch_bounds__(64 * kWaves) void kv_append_kernel(AppendArgs a, int rounds) {
  using T = std::conditional_t<MX != 0, double, float>;
  constexpr int IPH = D / 16;    // items per head
  constexpr int HPR = 64 / IPH;  // heads per round
  __shared__ Turn<T> turn[kWaves][D / 2];
  __shared__ __attribute__((aligned(16))) unsigned most[MX ? kWaves : 1][MX ? 128 : 1];  // of each 8 components of a round's heads
  const CacheArgs& c = a.c;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63;
  const int hq = a.q ? c.heads_q : 0, heads = hq + 2 * c.heads_kv;
  const int total_rounds = (heads + HPR - 1) / HPR;
  const int per_token = (total_rounds + rounds - 1) / rounds;  // waves
  const long wave = (long)blockIdx.x * kWaves + w;
  const int t = (int)(wave / per_token);
  if (t >= a.tokens) return;
  const int first = (int)(wave % per_token) * rounds;

  int s = t, place = 0;
  if (a.cu) {
    s = find_sequence(a.cu, c.batch, t, l);
    if (s < 0) return;  // before the first sequence or behind the last
    const int start = a.cu[s], end = a.cu[s + 1];
    if (start < 0 || t < start || t >= end) {  // offsets that do not rise from 0 on: nobody's row
      if (l == 0 && c.status) *c.status = 1;
      return;
    }
    place = t - start;
  }
  const int old = c.lens[s];
  const int64_t at_place = (int64_t)place + old;

  const int pairs = a.inv_freq ? a.rotary >> 1 : 0;
  fill_turns(turn[w], a.inv_freq, pairs, at_place, l);

  // the token's cache row
  const PageRow to = page_row(c.table + s * c.table_stride, c.table_width, c.page_size, c.pages, old < 0 ? -1 : at_place);
  if (!to.ok && l == 0 && c.status) *c.status = 1;

  const RotaryItem<D, float> item(turn[w], l % IPH, pairs, a.interleaved);
  const int e0 = item.e0, e1 = item.e1;
  for (int r = first; r < first + rounds; ++r) {
    const int h = r * HPR + l / IPH;
    if (h >= heads) return;
    const int kind = h < hq ? 0 : h < hq + c.heads_kv ? 1 : 2;  // q, k, v
    const int hk = kind == 1 ? h - hq : h - hq - c.heads_kv;    // head of the cache
    const __bf16* src = kind == 0   ? (const __bf16*)a.q + t * a.qs.row + h * a.qs.head
                        : kind == 1 ? (const __bf16*)a.k + t * a.ks.row + hk * a.ks.head
                                    : (const __bf16*)a.v + t * a.vs.row + hk * a.vs.head;
    u32x4 x0 = ONCE ? __builtin_nontemporal_load((const u32x4*)(src + e0)) : *(const u32x4*)(src + e0);
    u32x4 x1 = ONCE ? __builtin_nontemporal_load((const u32x4*)(src + e1)) : *(const u32x4*)(src + e1);
    float y0[8], y1[8];
    unpack8(x0, y0);
    unpack8(x1, y1);
    if (kind != 2 && item.on0) {
      // a key for a microscaled cache in 64 bits: what is stored follows from the rotated value, not from an
      // order of roundings
      if (MX && kind == 1) {
        if constexpr (MX) item.turn_wide(turn[w], y0, y1);
      } else {
        item.turn(y0, y1);
      }
      x0 = pack8_bf16(y0);
      if (item.on1) x1 = pack8_bf16(y1);
    }
    __bf16* out = kind == 0                ? (__bf16*)a.q_out + t * a.qos.row + h * a.qos.head
                  : kind == 1 && a.k_out   ? (__bf16*)a.k_out + t * a.kos.row + hk * a.kos.head
                                           : nullptr;
    if (out && ONCE && MX) {
      __builtin_nontemporal_store(x0, (u32x4*)(out + e0));
      __builtin_nontemporal_store(x1, (u32x4*)(out + e1));
    } else if (out) {
      *(u32x4*)(out + e0) = x0;
      *(u32x4*)(out + e1) = x1;
    }
    if (kind == 0 || !to.ok) continue;
    const int64_t at = kind == 1 ? to.page * c.k_page + hk * c.k_head + to.row * c.k_row : to.page * c.v_page + hk * c.v_head + to.row * c.v_row;
    if constexpr (MX) {
      // a block's largest value: four chunks, which lie with lanes of this head in any order
      unsigned* of = most[w] + l / IPH * (D / 8);
      of[e0 / 8] = mx_most(y0);
      of[e1 / 8] = mx_most(y1);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      const u32x4 m0 = *(const u32x4*)(of + (e0 / 32) * 4), m1 = *(const u32x4*)(of + (e1 / 32) * 4);
      const auto top = [](u32x4 m) {
        const unsigned a = m[0] > m[1] ? m[0] : m[1], b = m[2] > m[3] ? m[2] : m[3];
        return a > b ? a : b;
      };
      const int b0 = mx_byte<MX == 2>(top(m0)), b1 = mx_byte<MX == 2>(top(m1));
      const u32x2 p0 = mx_pack<MX == 2>(y0, b0), p1 = mx_pack<MX == 2>(y1, b1);
      uint8_t* dst = (uint8_t*)(kind == 1 ? c.k : c.v) + at;
      if constexpr (MX == 1) {
        *(u32x2*)(dst + e0) = p0;
        *(u32x2*)(dst + e1) = p1;
      } else {
        *(unsigned*)(dst + e0 / 2) = p0[0];
        *(unsigned*)(dst + e1 / 2) = p1[0];
      }
      uint8_t* bytes = (kind == 1 ? c.k_mx : c.v_mx) + (((int64_t)to.page * c.heads_kv + hk) * c.page_size + to.row) * (D / 32);
      if (e0 % 32 == 0) bytes[e0 / 32] = (uint8_t)b0;
      if (e1 % 32 == 0) bytes[e1 / 32] = (uint8_t)b1;
      asm volatile("" ::: "memory");  // (the next round's maxima behind this one's reads)
    } else if (c.type == kBf16) {
      __bf16* dst = (__bf16*)(kind == 1 ? c.k : c.v) + at;
      *(u32x4*)(dst + e0) = x0;
      *(u32x4*)(dst + e1) = x1;
    } else {
      const float* sc = kind == 1 ? c.k_scale : c.v_scale;
      if (sc) {
        const float scale = sc[hk];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          y0[i] /= scale;
          y1[i] /= scale;
        }
      }
      uint8_t* dst = (uint8_t*)(kind == 1 ? c.k : c.v) + at;
      *(u32x2*)(dst + e0) = u32x2{pack_e4m3(y0), pack_e4m3(y0 + 4)};
      *(u32x2*)(dst + e1) = u32x2{pack_e4m3(y1), pack_e4m3(y1 + 4)};
    }
  }
}

// waves a token and their rounds
struct Split {
  int rounds, waves;
};
Split split_of(const AppendArgs& a) {
  const int hpr = 64 / (a.c.d / 16), heads = (a.q ? a.c.heads_q : 0) + 2 * a.c.heads_kv;
  const int total = (heads + hpr - 1) / hpr;
  // one round per wave until the waves fill the GPU (256 CUs of 16), then as many
  // rounds as a token has
  const int rounds = (long)a.tokens * total <= 4096 ? 1 : total;
  return {rounds, (total + rounds - 1) / rounds};
}

template <int D>
void launch(const AppendArgs& a, hipStream_t stream) {
  const int heads = (a.q ? a.c.heads_q : 0) + 2 * a.c.heads_kv, rounds = split_of(a).rounds;
  const dim3 grid((unsigned)((append_waves(a) + kWaves - 1) / kWaves));
  // past the caches from 64 MB of q, k and v on (us, through / past them: 8192 tokens, 32 heads
  // over 8 of 128, 100 MB, 44.2 / 40.3; 16 over 4 of 64, 25 MB, where the cache still holds them, 14.0 / 17.5)
  // (microscaled from 32 MB on: 3001 tokens of 32 heads over 8, 37 MB, and 19385 rows read back behind them 41.2 / 35.8; with packed
  // attention behind them, and 640 MB of other data through the caches before each pass, the two are even within 1%: 4096 MXFP8 tokens
  // 347 / 347, 6000 391 / 395, 8192 442 / 444, 10000 505 / 497)
  const bool once = (long)a.tokens * heads * D * 2 >= (a.c.type >= kMx8 ? 32L : 64L) << 20;
  const auto kernel = a.c.type == kMx8   ? once ? kv_append_kernel<D, true, 1> : kv_append_kernel<D, false, 1>
                      : a.c.type == kMx4 ? once ? kv_append_kernel<D, true, 2> : kv_append_kernel<D, false, 2>
                                         : once ? kv_append_kernel<D, true, 0> : kv_append_kernel<D, false, 0>;
  hipLaunchKernelGGL(kernel, grid, dim3(64 * kWaves), 0, stream, a, rounds);
}

}  // namespace

int64_t append_waves(const AppendArgs& a) { return (int64_t)a.tokens * split_of(a).waves; }

hipError_t launch_kv_append(const AppendArgs& a, hipStream_t stream) {
  if (a.c.d == 64) launch<64>(a, stream);
  else if (a.c.d == 128) launch<128>(a, stream);
  else launch<256>(a, stream);
  return hipGetLastError();
}

}  // namespace dash
