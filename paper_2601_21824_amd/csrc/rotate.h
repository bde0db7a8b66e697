// rotate.h -- rotary positions: what one wave turns of a row, and by how much.
//
// Pair i of a head's first `rotary` components turns by the angle p f_i at place p,
//   (x, y) -> (x cos - y sin, x sin + y cos),
// pairs being (i, i + rotary / 2), or (2i, 2i + 1) when interleaved.  The angle is
// reduced in 64 bits: at p = 10^5 a product in 32 bits is off by 2^-24 10^5 = 0.006
// radians, more than a bf16 rounding.
//
// A lane holds two 16-byte chunks of a head that make 8 whole pairs, so that it never
// needs another lane's data; neighbouring lanes hold neighbouring chunks, so that a
// load is whole lines.
#pragma once
#include "common.h"

namespace dash {

__device__ inline float bf_lo(unsigned x) { return __builtin_bit_cast(float, x << 16); }
__device__ inline float bf_hi(unsigned x) { return __builtin_bit_cast(float, x & 0xffff0000u); }

template <typename T>
struct Turn {
  T c, s;
};

__device__ inline void sin_cos_pi(float x, float* s, float* c) { sincospif(x, s, c); }
__device__ inline void sin_cos_pi(double x, double* s, double* c) { sincospi(x, s, c); }

// Sine and cosine of every pair at place p, by one wave into turn[0 .. pairs - 1] of
// its LDS (its own reads behind this see them).
template <typename T>
__device__ inline void fill_turns(Turn<T>* turn, const float* inv_freq, int pairs, int64_t place, int l) {
  for (int i = l; i < pairs; i += 64) {
    const double turns = (double)place * (double)inv_freq[i] * 0.15915494309189535;
    const T part = (T)(2.0 * (turns - rint(turns)));  // half turns, -1 .. 1: whole turns are taken off in 64 bits
    T sn, cs;
    sin_cos_pi(part, &sn, &cs);
    turn[i] = {cs, sn};
  }
  // (a wave's own LDS writes and reads are in order)
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// The chunks (first elements e0, e1) of item j = 0 .. D / 16 - 1 of a head, and their turns.
template <int D, typename T>
struct RotaryItem {
  int e0, e1;
  bool split;     // chunks of the two halves of 8 pairs
  bool on0, on1;  // whether each chunk is rotated (e1 only if e0 is)
  T cs[8], sn[8];

  template <typename S>  // (turns of 64 bits are rounded to 32 for an item of those)
  __device__ RotaryItem(const Turn<S>* turn, int j, int pairs, int interleaved) {
    const int rot = 2 * pairs;
    e0 = 8 * j, e1 = 8 * j + D / 2;
    split = !interleaved && 16 * j < rot;
    if (split) {
      e1 = 8 * j + pairs;
    } else if (!interleaved) {  // components that are not rotated
      e0 = rot + 8 * (j - rot / 16);
      e1 = e0 + (D - rot) / 2;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // split: pairs 8j .. 8j+7; interleaved: the four of chunk e0 and the four of e1
      const int at = split ? 8 * j + i : (i < 4 ? e0 : e1) / 2 + (i & 3);
      const bool on = split || (interleaved && (i < 4 ? e0 : e1) < rot);
      const Turn<S> x = on ? turn[at] : Turn<S>{1, 0};
      cs[i] = (T)x.c;
      sn[i] = (T)x.s;
    }
    // a chunk that is not rotated keeps its bits (x cos 0 - y sin 0 makes NaN beside an
    // infinity, and +0 of -0)
    on0 = split || (interleaved && e0 < rot);
    on1 = split || (interleaved && e1 < rot);
  }

  // the chunks' values turned in 64 bits, by turns of 64 bits from LDS, and rounded to 32 (where on0 says so)
  __device__ void turn_wide(const Turn<double>* turn, float (&y0)[8], float (&y1)[8]) const {
    if (split) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const Turn<double> t = turn[e0 + i];  // (e0 is 8 j, the item's first pair)
        const double x = y0[i], y = y1[i];
        y0[i] = (float)(x * t.c - y * t.s);
        y1[i] = (float)(x * t.s + y * t.c);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float(&z)[8] = i < 4 ? y0 : y1;
        if (i >= 4 && !on1) continue;
        const Turn<double> t = turn[(i < 4 ? e0 : e1) / 2 + (i & 3)];
        const double x = z[2 * (i & 3)], y = z[2 * (i & 3) + 1];
        z[2 * (i & 3)] = (float)(x * t.c - y * t.s);
        z[2 * (i & 3) + 1] = (float)(x * t.s + y * t.c);
      }
    }
  }
  // the chunks' values, turned (where on0 says so)
  __device__ void turn(T (&y0)[8], T (&y1)[8]) const {
    if (split) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const T x = y0[i], y = y1[i];
        y0[i] = x * cs[i] - y * sn[i];
        y1[i] = x * sn[i] + y * cs[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const T x = y0[2 * i], y = y0[2 * i + 1];
        y0[2 * i] = x * cs[i] - y * sn[i];
        y0[2 * i + 1] = x * sn[i] + y * cs[i];
      }
      if (on1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const T x = y1[2 * i], y = y1[2 * i + 1];
          y1[2 * i] = x * cs[4 + i] - y * sn[4 + i];
          y1[2 * i + 1] = x * sn[4 + i] + y * cs[4 + i];
        }
      }
    }
  }
};

template <typename T>
__device__ inline void unpack8(u32x4 x, T (&y)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[2 * i] = bf_lo(x[i]);
    y[2 * i + 1] = bf_hi(x[i]);
  }
}
__device__ inline u32x4 pack8_bf16(const float (&y)[8]) {
  return u32x4{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])};
}

}  // namespace dash
