// paged.h -- device pieces shared by the variable-length operators: which
// sequence a row belongs to, its resource, and reductions over the wave.
#pragma once
#include "common.h"
#include "ops.h"

namespace dash {

// The last s in 0 .. n-1 with key(s) <= t (0 if there is none), for keys that rise.
// A search with 64 samples a step (one key per lane): two steps up to 4096.
// Wave-uniform, all lanes active.  Keys that do not rise give some s in 0 .. n-1.
template <typename Key>
__device__ inline int find_last(int n, int t, int l, Key&& key) {
  int lo = 0;  // the answer is in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 63) / 64;
    const int at = l * step;
    const bool below = at < n && key(lo + at) <= t;
    const int c = __builtin_popcountll(__ballot(below));  // samples at or below t: a prefix
    const int k = c > 0 ? c - 1 : 0;
    lo += k * step;
    n = n - k * step < step ? n - k * step : step;
  }
  return lo;
}

// The sequence that row t lies in, -1 where t is before cu[0] or at or behind cu[batch].
// Offsets that do not rise give some sequence, which need not hold t.
__device__ inline int find_sequence(const int32_t* cu, int batch, int t, int l) {
  if (t < cu[0] || t >= cu[batch]) return -1;
  return find_last(batch, t, l, [&](int s) { return cu[s]; });
}

// Rows of sequence s among `total`: offsets outside 0 .. total are clamped, and an
// end before its start makes an empty sequence.
struct Span {
  int start, len;
};
__device__ inline int clamp_row(int x, int total) { return x < 0 ? 0 : x > total ? total : x; }
__device__ inline Span span_of(const int32_t* cu, int s, int total) {
  const int b = clamp_row(cu[s], total), e = clamp_row(cu[s + 1], total);
  return {b, e > b ? e - b : 0};
}

// Blocks of `rows` rows, numbered so that no prefix sum is needed: those of
// sequence s begin at start / rows + s.  (A sequence of n rows has at most
// (start + n) / rows - start / rows + 1 of them.)  At most total / rows + batch slots;
// those between two sequences' blocks are empty.
__device__ inline int first_slot(const int32_t* cu, int s, int total, int rows) { return clamp_row(cu[s], total) / rows + s; }

// a resource over at most `most` of n rows from row `first` on: what lies past them reads 0 and
// is not written
template <int D>
__device__ inline __amdgpu_buffer_rsrc_t strided_rows(const void* p, int64_t first, const Strides& s, int head, int n, int most) {
  const int r = n < most ? n : most;
  const uint32_t bytes = r > 0 ? (uint32_t)(r - 1) * (uint32_t)s.row * 2 + D * 2 : 0;
  return make_rsrc((const __bf16*)p + first * s.row + head * s.head, bytes);
}

// x plus the lanes before it: four shifts inside rows of 16 lanes, then the last lane
// of a row, and of the lower half, to those behind it.  All lanes active.
__device__ inline int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);   // row_shr:2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);   // row_shr:4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);   // row_shr:8
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31 into rows 2 and 3
  return x;
}
// sum over the 64 lanes, wave-uniform
__device__ inline int wave_sum(int x) { return __builtin_amdgcn_readlane(wave_scan(x), 63); }

// Over the four lanes l % 16 + 16 i.  The swaps exchange the upper half (every odd
// row of 16) of one register with the lower half (even row) of another, here two
// copies of x: afterwards the two hold x of both partners.
template <typename Op>
__device__ inline float quad_reduce(float x, Op&& op) {
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const unsigned p0 = p[0], p1 = p[1];  // (a bit cast of p[1] itself would take p[0])
  const float y = op(__builtin_bit_cast(float, p0), __builtin_bit_cast(float, p1));
  const unsigned v = __builtin_bit_cast(unsigned, y);
  const auto q = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  const unsigned q0 = q[0], q1 = q[1];
  return op(__builtin_bit_cast(float, q0), __builtin_bit_cast(float, q1));
}
__device__ inline float quad_max(float x) {
  return quad_reduce(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ inline float quad_sum(float x) {
  return quad_reduce(x, [](float a, float b) { return a + b; });
}

}  // namespace dash
