// attn_fwd.hip -- the forward of dense batches (fwd_main.h): which workgroup takes
// which query rows, and the choice of the rows per wave.
#include "fwd_main.h"

namespace dash {

template <int D, int QG, int WPS>
__global__ __launch_bounds__(256, WPS) void attn_fwd_kernel(FwdArgs a) {
  constexpr int QROWS = 128 * QG;
  const int N = a.n;
  const int nqb = (N + QROWS - 1) / QROWS;
  // Workgroup -> (head, query block).  Consecutive workgroups go to the 8
  // XCDs in turn; each XCD takes a contiguous run of the head-major order, so
  // that the workgroups sharing an XCD's L2 read the same K and V.
  const int items = nqb * a.bh;
  const int per = (items + 7) >> 3;
  const int item = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || item >= items) return;
  const int bh = item / nqb;
  int qb_i = item % nqb;
  // causal: the longest query blocks (last rows) first; where a run ends inside
  // a head, long and short ones alternate instead so that every run holds the
  // same work
  if (a.causal) qb_i = (a.bh & 7) == 0 ? nqb - 1 - qb_i : (qb_i & 1) ? qb_i >> 1 : nqb - 1 - (qb_i >> 1);
  attn_fwd_rows<D, QG>(DenseView<D>(a, bh), a.causal, a.scale, qb_i * QROWS);
}

template <int D, int QG, int WPS>
void launch_fwd(const FwdArgs& a, hipStream_t stream) {
  const long items = (long)((a.n + 128 * QG - 1) / (128 * QG)) * a.bh;
  hipLaunchKernelGGL((attn_fwd_kernel<D, QG, WPS>), dim3((unsigned)((items + 7) / 8 * 8)), dim3(256), 0, stream, a);
}

hipError_t launch_attn_fwd(const FwdArgs& a, int d, hipStream_t stream) {
  // Two query groups per wave halve the LDS reads per MFMA, but need 256-row
  // workgroups enough for two per CU, and under a causal mask leave half of a
  // diagonal workgroup's waves waiting.  At d = 64, full mask, 512 to 4096
  // such workgroups: 0-11% faster (16 heads of 8192: 291 against 322 us), with
  // 256 and fewer 1-33% slower, causal 3-34% slower below N = 16384.  A head of at most 128 rows
  // leaves two of the four waves without any: 600 heads of 100 13.8 us against
  // 9.1, 2048 of 128 34.2 against 29.7, 8192 of 33 61.8 against 37.1.  At d = 128 two
  // groups leave room for one wave per SIMD only: -13% to +4% at 512 workgroups
  // and more, so it is not built.
  const long wide = (long)((a.n + 255) / 256) * a.bh;
  if (d == 64) {
    if (!a.causal && a.n > 128 && wide >= 512) launch_fwd<64, 2, 2>(a, stream);
    else launch_fwd<64, 1, 3>(a, stream);
  } else if (d == 128) {
    launch_fwd<128, 1, 2>(a, stream);
  } else {
    launch_fwd<256, 1, 1>(a, stream);
  }
  return hipGetLastError();
}

}  // namespace dash
