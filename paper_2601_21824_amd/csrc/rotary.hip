// rotary.hip -- queries and keys of packed rows turned by their positions, and their
// gradients turned back.
//
//   y = a R(p f) x    backward: dx = a R(-p f) dy, the transpose
//
// R turns each pair (rotate.h); a, the amplitude, scales what is rotated.  Sine and cosine
// are fp32 times a, the products fp32, with one rounding at the store.  Components
// behind rotary_dim keep their bits, and are copied where q_out is not q.
//
// Bound by memory (q and k in and out), by the launch for single rows.  One wave per
// row takes sine and cosine of every pair once, for all heads of q and k, then 64 items
// a round (two 16-byte chunks of a head each), the loads of two rounds in flight.  Calls
// of few rows give each wave one round, and the waves of a row redo its sines.
//
// Measured: 8192 rows of 32 and 8 heads of 128 33.6 us, 84 MB in and 84 out, 5.0 TB/s, a copy's rate; 5001 rows
// of 16 and 4 heads of 256, 128 components rotated, 18.8 us, 102 MB; 64 rows 3.7 us.
#include "common.h"
#include "ops.h"
#include "paged.h"
#include "rotate.h"

namespace dash {
namespace {

constexpr int kWaves = 4;

// PAST: large outputs are written past the caches (1), and larger inputs read past them too (2).
template <int D, int PAST>
__global__ __launch_bounds__(64 * kWaves) void rotary_kernel(RotaryArgs a, int rounds) {
  constexpr int IPH = D / 16;    // items per head
  constexpr int HPR = 64 / IPH;  // heads per round
  __shared__ Turn<float> turn[kWaves][D / 2];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63;
  const int hq = a.q ? a.heads_q : 0, heads = hq + (a.k ? a.heads_k : 0);
  const int total_rounds = (heads + HPR - 1) / HPR;
  const int per_row = (total_rounds + rounds - 1) / rounds;  // waves
  const long wave = (long)blockIdx.x * kWaves + w;
  const int t = (int)(wave / per_row);
  if (t >= a.rows) return;
  const int first = (int)(wave % per_row) * rounds;

  int64_t place;
  if (a.positions) {
    place = a.positions[t];
  } else {
    const int s = find_sequence(a.cu, a.batch, t, l);
    if (s < 0) return;  // before the first sequence or behind the last
    const int start = a.cu[s], end = a.cu[s + 1];
    if (start < 0 || t < start || t >= end) {  // offsets that do not rise from 0 on: nobody's row
      if (l == 0 && a.status) *a.status = 1;
      return;
    }
    place = (int64_t)(t - start) + (a.start ? a.start[s] : 0);
  }
  const int pairs = a.rotary >> 1;
  fill_turns(turn[w], a.inv_freq, pairs, place, l);
  RotaryItem<D, float> item(turn[w], l % IPH, pairs, a.interleaved);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    item.cs[i] *= a.amplitude;
    item.sn[i] *= a.back ? -a.amplitude : a.amplitude;
  }

  constexpr int U = 2;
  for (int r0 = first; r0 < first + rounds && r0 < total_rounds; r0 += U) {
    u32x4 x[U][2];
    __bf16* out[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = (r0 + u) * HPR + l / IPH;
      out[u] = nullptr;
      if (r0 + u >= first + rounds || h >= heads) continue;
      const bool q = h < hq;
      const __bf16* src = q ? (const __bf16*)a.q + t * a.qs.row + h * a.qs.head : (const __bf16*)a.k + t * a.ks.row + (h - hq) * a.ks.head;
      out[u] = q ? (__bf16*)a.q_out + t * a.qos.row + h * a.qos.head : (__bf16*)a.k_out + t * a.kos.row + (h - hq) * a.kos.head;
      x[u][0] = PAST == 2 ? __builtin_nontemporal_load((const u32x4*)(src + item.e0)) : *(const u32x4*)(src + item.e0);
      x[u][1] = PAST == 2 ? __builtin_nontemporal_load((const u32x4*)(src + item.e1)) : *(const u32x4*)(src + item.e1);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!out[u]) continue;
      if (item.on0) {
        float y0[8], y1[8];
        unpack8(x[u][0], y0);
        unpack8(x[u][1], y1);
        item.turn(y0, y1);
        x[u][0] = pack8_bf16(y0);
        if (item.on1) x[u][1] = pack8_bf16(y1);
      }
      if (PAST) {
        __builtin_nontemporal_store(x[u][0], (u32x4*)(out[u] + item.e0));
        __builtin_nontemporal_store(x[u][1], (u32x4*)(out[u] + item.e1));
      } else {
        *(u32x4*)(out[u] + item.e0) = x[u][0];
        *(u32x4*)(out[u] + item.e1) = x[u][1];
      }
    }
  }
}

// waves a row and their rounds
struct Split {
  int rounds, waves;
};
Split split_of(const RotaryArgs& a) {
  const int hpr = 64 / (a.d / 16), heads = (a.q ? a.heads_q : 0) + (a.k ? a.heads_k : 0);
  const int total = (heads + hpr - 1) / hpr;
  // one round per wave until the waves fill the GPU (256 CUs of 16), then as many as a row has
  const int rounds = (long)a.rows * total <= 4096 ? 1 : total;
  return {rounds, (total + rounds - 1) / rounds};
}

template <int D>
void launch(const RotaryArgs& a, hipStream_t stream) {
  const int heads = (a.q ? a.heads_q : 0) + (a.k ? a.heads_k : 0), rounds = split_of(a).rounds;
  const dim3 grid((unsigned)((rotary_waves(a) + kWaves - 1) / kWaves));
  // The call itself, us, through the caches / outputs / both past them, with inputs and outputs that no cache holds: 5001 rows of 16
  // and 4 heads of 256, 51 MB each way, 25.9 / 22.6 / 21.3, and 21.2 / 18.5 / 21.2 where a cache holds a part; 8192 of 32 and 8 heads
  // of 128, 84 MB, 39 / - / 33.5, inputs alone past them 36.1.  With the packed attention behind it, and 640 MB of other data through the
  // caches before each pass, it is even within 1%: 32 and 8 heads of 128, 4096 rows 342 / 344 / 342, 6000 383 / 386 / 386, 8192
  // 436 / 435 / 436, 12000 559 / 553 / 552 (in a loop of the two calls alone 72 / 76 / 76, 117 / 121 / 121, 174 / 174 / 175, 300 / 294 / 294).
  const long bytes = (long)a.rows * heads * D * 2;
  const auto kernel = bytes >= 64L << 20 ? rotary_kernel<D, 2> : bytes >= 32L << 20 ? rotary_kernel<D, 1> : rotary_kernel<D, 0>;
  hipLaunchKernelGGL(kernel, grid, dim3(64 * kWaves), 0, stream, a, rounds);
}

}  // namespace

int64_t rotary_waves(const RotaryArgs& a) { return (int64_t)a.rows * split_of(a).waves; }

hipError_t launch_rotary(const RotaryArgs& a, hipStream_t stream) {
  if (a.d == 64) launch<64>(a, stream);
  else if (a.d == 128) launch<128>(a, stream);
  else launch<256>(a, stream);
  return hipGetLastError();
}

}  // namespace dash
