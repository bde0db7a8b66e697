// kv_read.hip -- rows of a paged cache read back as packed bf16 rows, what attention over
// packed sequences takes for the keys and values that earlier calls have stored.
//
// Row cu[s] + i receives key first[s] + i of sequence s: the cached value itself (bf16),
// times its head's scale and rounded (e4m3), or times its block's power of two, which is exact.
//
// Bound by memory: the rows in, two bytes a component out.  A wave takes 16 rows of one
// head, K and V: its lanes find the rows' pages first, one row each, then all loads are
// in flight together, 8 components a lane.  Rows of one head are neighbours in a page, so the
// reads are whole lines; a row's 2 d bytes are, in the output.
//
// Measured, 8 heads of 128: 8192 rows in MXFP8 11.0 us, 18 MB that the append before has left in the caches and 34 out;
// 19385 rows in MXFP4 19.4 us, 24 MB in and 79 out, 5.3 TB/s; 64 rows 7.1 us, the searches and dependent loads.
#include <type_traits>

#include "common.h"
#include "mx.h"
#include "ops.h"
#include "page_index.h"
#include "paged.h"

namespace dash {
namespace {

constexpr int kWaves = 4, kRows = 16;

// 8 components of a cached row as bf16
template <int TYPE>
struct Piece {
  using Raw = std::conditional_t<TYPE == kBf16, u32x4, std::conditional_t<TYPE == kMx4, unsigned, u32x2>>;
  Raw x;
  unsigned byte;
};
template <int TYPE>
__device__ inline u32x4 values(const Piece<TYPE>& p, float scale) {
  if constexpr (TYPE == kBf16) {
    return p.x;
  } else if constexpr (TYPE == kE4m3) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x2 f = i & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)p.x[i >> 1], true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)p.x[i >> 1], false);
      r[i] = pack_bf16(f[0] * scale, f[1] * scale);
    }
    return r;
  } else if constexpr (TYPE == kMx8) {
    const float s = mx_scale(p.byte);
    return u32x4{mx_pair<false>(p.x[0], 0, s), mx_pair<false>(p.x[0], 1, s), mx_pair<false>(p.x[1], 0, s), mx_pair<false>(p.x[1], 1, s)};
  } else {
    const float s = mx_scale(p.byte);
    return u32x4{mx_pair<true>(p.x, 0, s), mx_pair<true>(p.x, 1, s), mx_pair<true>(p.x, 2, s), mx_pair<true>(p.x, 3, s)};
  }
}

template <bool PAST>
__device__ inline void put(void* p, int64_t at, u32x4 x) {
  if (PAST) __builtin_nontemporal_store(x, (u32x4*)((__bf16*)p + at));
  else *(u32x4*)((__bf16*)p + at) = x;
}

// PAST: large outputs are written past the caches.
template <int D, int TYPE, bool PAST>
__global__ __launch_bounds__(64 * kWaves) void kv_read_kernel(ReadArgs a) {
  constexpr int LPR = D / 8;       // lanes a row
  constexpr int RPI = 64 / LPR;    // rows of one load
  constexpr int NI = kRows / RPI;  // loads
  using P = Piece<TYPE>;
  const CacheArgs& c = a.c;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63;
  const long wave = (long)blockIdx.x * kWaves + w;
  const int hk = (int)(wave % c.heads_kv);
  const int t0 = (int)(wave / c.heads_kv) * kRows;
  if (t0 >= a.rows) return;

  // ---- lane l (of 16) finds row t0 + l: -1 where it is nobody's, or has no key
  const int end = a.cu[c.batch], begin = a.cu[0];
  const int t1 = t0 + kRows - 1 < a.rows - 1 ? t0 + kRows - 1 : a.rows - 1;
  int lo = find_last(c.batch, t0, l, [&](int s) { return a.cu[s]; });
  int hi = find_last(c.batch, t1, l, [&](int s) { return a.cu[s]; });
  int page = -1, row = 0;
  const int t = t0 + l;
  if (l < kRows && t <= t1 && t >= begin && t < end) {
    while (lo < hi) {  // the last s of lo .. hi with cu[s] <= t
      const int mid = (lo + hi + 1) >> 1;
      if (a.cu[mid] <= t) lo = mid;
      else hi = mid - 1;
    }
    const int start = a.cu[lo];
    bool ok = start >= 0 && t >= start && t < a.cu[lo + 1];  // (else offsets that do not rise from 0 on)
    if (ok) {
      const int64_t from = a.first ? a.first[lo] : 0, place = from + (t - start);
      const PageRow r = page_row(c.table + lo * c.table_stride, c.table_width, c.page_size, c.pages, from < 0 ? -1 : place);
      ok = r.ok && place < c.lens[lo];
      if (ok) page = r.page, row = r.row;
    }
    if (!ok && c.status) *c.status = 1;
  }

  const int col = l % LPR * 8;
  const bool has_k = a.k_out != nullptr, has_v = a.v_out != nullptr;
  P k[NI], v[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int r = i * RPI + l / LPR, id = __shfl(page, r), at = __shfl(row, r);
    if (id < 0) continue;
    constexpr int kBits = TYPE == kBf16 ? 16 : TYPE == kMx4 ? 4 : 8;  // of a component
    constexpr int kUnit = TYPE == kBf16 ? 2 : 1;                      // bytes of a stride's unit
    const int64_t blk = (((int64_t)id * c.heads_kv + hk) * c.page_size + at) * (D / 32) + col / 32;
    if (has_k) {
      k[i].x = *(const typename P::Raw*)((const char*)c.k + (id * c.k_page + hk * c.k_head + at * c.k_row) * kUnit + col * kBits / 8);
      if constexpr (TYPE >= kMx8) k[i].byte = c.k_mx[blk];
    }
    if (has_v) {
      v[i].x = *(const typename P::Raw*)((const char*)c.v + (id * c.v_page + hk * c.v_head + at * c.v_row) * kUnit + col * kBits / 8);
      if constexpr (TYPE >= kMx8) v[i].byte = c.v_mx[blk];
    }
  }
  const float ks = TYPE == kE4m3 && c.k_scale ? c.k_scale[hk] : 1.f, vs = TYPE == kE4m3 && c.v_scale ? c.v_scale[hk] : 1.f;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int r = i * RPI + l / LPR;
    if (__shfl(page, r) < 0) continue;
    const int64_t to = t0 + r;
    if (has_k) put<PAST>(a.k_out, to * a.ks.row + hk * a.ks.head + col, values<TYPE>(k[i], ks));
    if (has_v) put<PAST>(a.v_out, to * a.vs.row + hk * a.vs.head + col, values<TYPE>(v[i], vs));
  }
}

template <int D, int TYPE>
void launch(const ReadArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)((read_waves(a) + kWaves - 1) / kWaves));
  // The call itself, among calls whose data no cache holds together, us, through / past the caches: 19385 rows of 8 heads of 128 in
  // MXFP4, 79 MB out, 31 / 19.4; 8192 in MXFP8, 34 MB, 12.2 / 11.1.  With the packed attention that reads them, and 640 MB of other
  // data through the caches before each pass, it is even up to about 80 MB: those 19385 rows and 3001 queries 489.0 / 488.7, 16684
  // rows and 300 queries 336 / 338 (in a loop of the two calls alone 63 / 69); larger reads lose up to 1% (51001 bf16 rows 968 / 980).
  const bool past = (int64_t)a.rows * a.c.heads_kv * D * 2 * ((a.k_out != nullptr) + (a.v_out != nullptr)) >= 32L << 20;
  hipLaunchKernelGGL((past ? kv_read_kernel<D, TYPE, true> : kv_read_kernel<D, TYPE, false>), grid, dim3(64 * kWaves), 0, stream, a);
}
template <int D>
void launch(const ReadArgs& a, hipStream_t stream) {
  if (a.c.type == kBf16) launch<D, kBf16>(a, stream);
  else if (a.c.type == kE4m3) launch<D, kE4m3>(a, stream);
  else if (a.c.type == kMx8) launch<D, kMx8>(a, stream);
  else launch<D, kMx4>(a, stream);
}

}  // namespace

int64_t read_waves(const ReadArgs& a) { return (int64_t)((a.rows + kRows - 1) / kRows) * a.c.heads_kv; }

hipError_t launch_kv_read(const ReadArgs& a, hipStream_t stream) {
  if (a.c.d == 64) launch<64>(a, stream);
  else if (a.c.d == 128) launch<128>(a, stream);
  else launch<256>(a, stream);
  return hipGetLastError();
}

}  // namespace dash
