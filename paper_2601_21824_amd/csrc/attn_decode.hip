// attn_decode.hip -- attention of one new token per sequence over a paged
// key-value cache, split over the cache's length and joined.
//
//   o_h = sum_j softmax_j(scale q_h . k_j) v_j over the lens[s] cached keys
//
// Bound by memory in bf16 and e4m3: K and V are read once for every 16 query heads of a K/V head
// (with more, each 16 are a workgroup of their own), 4 d bytes a key and head (2 d in e4m3 and MXFP8 and d
// in MXFP4, d / 16 of scale bytes), for 4 d G operations, G query heads to a K/V head.  So the kernel's
// business is to keep loads in flight.  One workgroup takes a chunk of one sequence's keys for
// one K/V head and up to 16 of its query heads; each of its four waves takes every
// fourth tile of 32 keys by itself, with its own running maximum and sum (decode_main.h); the other
// waves' loads are in flight meanwhile (8 to 16 waves a CU, 16 KB each at d = 128 in bf16; a
// second tile ahead in registers leaves fewer waves and gains nothing: 538 MB 111 us with it
// and without).  Only the tiles' page numbers are read a tile ahead.  Nothing goes through LDS until the
// four waves are joined.  K's scale of an e4m3 cache goes into the softmax scale and V's into the output.
//
// The keys of all sequences are cut into chunks of one size, found on the device
// from lens (so that a captured call follows them): the sum over `workers`.  A sequence of one chunk is written at once; the others' chunks leave
// (m, sum, O) in fp32 and join_kernel adds them in order.  The chunk size, and so
// the order of the sums, is fixed by lens and the call's shape, never by timing.
// (Chunks of at least 128 keys: one tile for each wave.)
//
// Measured, 32 heads over 8 of 128: 131072 keys of 64 sequences in bf16 90 us, 6.0 TB/s,
// and 5 us of joins, and in MXFP8 47 us, 6.2 TB/s; of one sequence in e4m3 42 us, 6.3 TB/s, and 5.4, and in MXFP4 27 us, 5.3 TB/s, bound by the vector instructions that widen
// it; 901 keys, 8 heads over 2 of 64, whole, 8.1 us (four tiles a wave, one after the other).
#include "common.h"
#include "decode_main.h"
#include "ops.h"
#include "page_index.h"
#include "paged.h"

namespace dash {
namespace {

template <int D, int TYPE, int NW>
__global__ __launch_bounds__(64 * NW, 2) void decode_kernel(DecodeArgs a) {
  __shared__ JoinSpace<D, NW> space;
  decode_part<D, TYPE, NW, false>(a, (int)blockIdx.x, space);
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

template <int D, int NW>
void launch_main(const DecodeArgs& a, hipStream_t stream) {
  const auto kernel = a.c.type == kBf16   ? decode_kernel<D, kBf16, NW>
                      : a.c.type == kE4m3 ? decode_kernel<D, kE4m3, NW>
                      : a.c.type == kMx8  ? decode_kernel<D, kMx8, NW>
                                          : decode_kernel<D, kMx4, NW>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)decode_blocks(a)), dim3(64 * NW), 0, stream, a);
}

template <int D>
void launch(const DecodeArgs& a, hipStream_t stream) {
  if (a.workers == 0) return launch_main<D, kWholeWaves>(a, stream);
  launch_main<D, 4>(a, stream);
  if (a.slots > a.c.batch)  // (else no sequence can have two chunks)
    hipLaunchKernelGGL(join_kernel<D>, dim3((unsigned)(a.c.batch * a.c.heads_q)), dim3(256), 0, stream, a);
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
int decode_slots(int batch, int table_tokens, int workers) {
  const long most = table_tokens > kMinChunk ? (long)batch * ((table_tokens + kMinChunk - 1) / kMinChunk) : batch;
  const long s = (long)workers + batch;
  return (int)(s < most ? s : most);
}

int64_t decode_blocks(const DecodeArgs& a) {
  const int64_t G = a.c.heads_q / a.c.heads_kv;
  return (int64_t)a.slots * a.c.heads_kv * ((G + kQ - 1) / kQ);
}
int64_t decode_waves(const DecodeArgs& a) {
  const int64_t main = decode_blocks(a) * (a.workers == 0 ? kWholeWaves : 4);
  const int64_t join = a.slots > a.c.batch ? (int64_t)a.c.batch * a.c.heads_q * 4 : 0;
  return main > join ? main : join;
}

hipError_t launch_decode(const DecodeArgs& a, hipStream_t stream) {
  if (a.c.d == 64) launch<64>(a, stream);
  else if (a.c.d == 128) launch<128>(a, stream);
  else launch<256>(a, stream);
  return hipGetLastError();
}

}  // namespace dash
