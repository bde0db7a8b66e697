// kv_append.hip -- new keys and values into a paged cache, keys (and queries)
// rotated by their position on the way.
//
// Token t of sequence s stands at place p = lens[s] + (t - cu[s]).  Pair i of a
// head's first `rotary` components turns by the angle p f_i:
//   (x, y) -> (x cos - y sin, x sin + y cos),
// pairs being (i, i + rotary / 2), or (2i, 2i + 1) when interleaved.  The angle is
// reduced in 64 bits: at p = 10^5 a product in 32 bits is off by 2^-24 10^5 = 0.006
// radians, more than a bf16 rounding.  The rest is 32 bits with one rounding at the
// store (bf16, or value / scale[head] in e4m3).
//
// Bound by memory for prompts (q, k, v in, q and the cache rows out) and by the
// launch for single tokens.  One wave per token: it takes sine and cosine of every
// pair once (through LDS, for all heads), then 64 items a round: two 16-byte chunks of
// a head that hold 8 whole pairs, so that a lane never needs another lane's data and
// q_out may be q.  Calls with few
// tokens give each wave one round only, and the waves of a token redo its sines.
//
// Measured, heads of 128, 32 over 8: 8192 tokens into an e4m3 cache 40 us, 101 MB in and 84
// out, 4.6 TB/s; one token of each of 64 sequences, bf16, 4.4 us (1.6 MB).
#include "common.h"
#include "ops.h"
#include "page_index.h"
#include "paged.h"

namespace dash {
namespace {

constexpr int kWaves = 4;

__device__ inline float bf_lo(unsigned x) { return __builtin_bit_cast(float, x << 16); }
__device__ inline float bf_hi(unsigned x) { return __builtin_bit_cast(float, x & 0xffff0000u); }

// 4 values -> e4m3, saturated at 448 (a NaN stays one)
__device__ inline unsigned pack_e4m3(const float* x) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = x[i] != x[i] ? x[i] : __builtin_amdgcn_fmed3f(x[i], -448.f, 448.f);
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], r, true);
}

// ONCE: inputs larger than the last-level cache can hold behind the kernel that made
// them are read past the caches.
template <int D, bool ONCE>
__global__ __launch_bounds__(64 * kWaves) void kv_append_kernel(AppendArgs a, int rounds) {
  constexpr int IPH = D / 16;    // items per head
  constexpr int HPR = 64 / IPH;  // heads per round
  __shared__ float2 turn[kWaves][D / 2];
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

  // sine and cosine of pair i = l, l + 64: whole turns are taken off in 64 bits
  const int pairs = a.inv_freq ? a.rotary >> 1 : 0;
  for (int i = l; i < pairs; i += 64) {
    const double turns = (double)at_place * (double)a.inv_freq[i] * 0.15915494309189535;
    const float part = (float)(2.0 * (turns - rint(turns)));  // half turns, -1 .. 1
    float sn, cs;
    sincospif(part, &sn, &cs);
    turn[w][i] = make_float2(cs, sn);
  }
  // (a wave's own LDS writes and reads are in order)
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");

  // the token's cache row
  const PageRow to = page_row(c.table + s * c.table_stride, c.table_width, c.page_size, c.pages, old < 0 ? -1 : at_place);
  if (!to.ok && l == 0 && c.status) *c.status = 1;

  // The item's two 16-byte chunks (element offsets e0, e1) and their sines: neighbouring
  // lanes hold neighbouring chunks, so that a load is whole lines
  const int j = l % IPH, rot = 2 * pairs;
  const bool split = !a.interleaved && 16 * j < rot;  // chunks of the two halves of 8 pairs
  int e0 = 8 * j, e1 = 8 * j + D / 2;
  if (split) {
    e1 = 8 * j + pairs;
  } else if (!a.interleaved) {  // components that are not rotated
    e0 = rot + 8 * (j - rot / 16);
    e1 = e0 + (D - rot) / 2;
  }
  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    // split: pairs 8j .. 8j+7; interleaved: the four of chunk e0 and the four of e1
    const int at = split ? 8 * j + i : (i < 4 ? e0 : e1) / 2 + (i & 3);
    const bool on = split || (a.interleaved && (i < 4 ? e0 : e1) < rot);
    const float2 x = on ? turn[w][at] : make_float2(1.f, 0.f);
    cs[i] = x.x;
    sn[i] = x.y;
  }
  // whether each chunk is rotated; one that is not keeps its bits (x cos 0 - y sin 0 makes NaN
  // beside an infinity, and +0 of -0)
  const bool turned0 = split || (a.interleaved && e0 < rot), turned1 = split || (a.interleaved && e1 < rot);
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
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y0[2 * i] = bf_lo(x0[i]);
      y0[2 * i + 1] = bf_hi(x0[i]);
      y1[2 * i] = bf_lo(x1[i]);
      y1[2 * i + 1] = bf_hi(x1[i]);
    }
    if (kind != 2 && turned0) {  // (e1 < rot only if e0 is)
      if (split) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = y0[i], y = y1[i];
          y0[i] = x * cs[i] - y * sn[i];
          y1[i] = x * sn[i] + y * cs[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = y0[2 * i], y = y0[2 * i + 1];
          y0[2 * i] = x * cs[i] - y * sn[i];
          y0[2 * i + 1] = x * sn[i] + y * cs[i];
        }
        if (turned1) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float x = y1[2 * i], y = y1[2 * i + 1];
            y1[2 * i] = x * cs[4 + i] - y * sn[4 + i];
            y1[2 * i + 1] = x * sn[4 + i] + y * cs[4 + i];
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x0[i] = pack_bf16(y0[2 * i], y0[2 * i + 1]);
        if (turned1) x1[i] = pack_bf16(y1[2 * i], y1[2 * i + 1]);
      }
    }
    __bf16* out = kind == 0                ? (__bf16*)a.q_out + t * a.qos.row + h * a.qos.head
                  : kind == 1 && a.k_out   ? (__bf16*)a.k_out + t * a.kos.row + hk * a.kos.head
                                           : nullptr;
    if (out) {
      *(u32x4*)(out + e0) = x0;
      *(u32x4*)(out + e1) = x1;
    }
    if (kind == 0 || !to.ok) continue;
    const int64_t at = kind == 1 ? to.page * c.k_page + hk * c.k_head + to.row * c.k_row : to.page * c.v_page + hk * c.v_head + to.row * c.v_row;
    if (!c.e4m3) {
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
  if ((long)a.tokens * heads * D * 2 >= 64L << 20)
    hipLaunchKernelGGL((kv_append_kernel<D, true>), grid, dim3(64 * kWaves), 0, stream, a, rounds);
  else
    hipLaunchKernelGGL((kv_append_kernel<D, false>), grid, dim3(64 * kWaves), 0, stream, a, rounds);
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
