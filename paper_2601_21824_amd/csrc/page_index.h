// page_index.h -- where a paged cache's rows are, and how a call's keys are cut into
// chunks.  Usable on host and device, so that a host test can run it over tables
// that hold anything.
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#define DASH_PAGE_HD __host__ __device__ inline
#else
#define DASH_PAGE_HD inline
#endif

namespace dash {

// a page that may be read or written
DASH_PAGE_HD bool page_ok(int id, int pages) { return (unsigned)id < (unsigned)pages; }

// Place `place` of a sequence whose pages are table[0 .. width-1].
struct PageRow {
  int page, row;
  bool ok;  // false: there is no such place, or its page does not exist (page is then 0)
};
DASH_PAGE_HD PageRow page_row(const int32_t* table, int width, int page_size, int pages, int64_t place) {
  if (place < 0 || place >= (int64_t)width * page_size) return {0, 0, false};
  const int id = table[place / page_size];
  const bool ok = page_ok(id, pages);
  return {ok ? id : 0, (int)(place % page_size), ok};
}

// a sequence's length, in what its table can hold
DASH_PAGE_HD int clamp_len(int len, int width, int page_size) {
  const int64_t cap = (int64_t)width * page_size;
  return len < 0 ? 0 : len > cap ? (int)cap : len;
}

// Keys of a chunk: `total` over the chunks aimed at, in whole rounds of the four
// waves' 32 keys.  With it, all sequences have at most workers + batch chunks
// (an empty sequence has one): sum ceil(len / chunk) <= total / chunk + batch.
constexpr int kMinChunk = 128;
DASH_PAGE_HD int64_t chunk_keys(int64_t total, int workers) {
  const int64_t per = (total + workers - 1) / workers;
  const int64_t c = (per + kMinChunk - 1) / kMinChunk * kMinChunk;
  return c < kMinChunk ? kMinChunk : c;
}
// What a call takes: no table holds more than kMaxKeys, so a chunk of as many is any
// sequence whole, and the bound holds for longer ones as well.  workers 0: all whole.
constexpr int kMaxKeys = 0x7fffff00;
DASH_PAGE_HD int chunk_size(int64_t total, int workers) {
  const int64_t c = workers > 0 ? chunk_keys(total, workers) : kMaxKeys;
  return c < kMaxKeys ? (int)c : kMaxKeys;
}
DASH_PAGE_HD int chunks_of(int len, int64_t chunk) { return len > 0 ? (int)((len + chunk - 1) / chunk) : 1; }

}  // namespace dash
