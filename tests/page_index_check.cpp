// Host check of page_index.h: every place of a sequence maps to its page and
// row, places and pages that do not exist are refused whatever the table holds, and
// the chunks of any set of lengths fit the slots the host provides.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "page_index.h"

static int bad = 0;
#define CHECK(x) \
  if (!(x)) std::printf("line %d: %s\n", __LINE__, #x), ++bad

int main() {
  using namespace dash;
  std::mt19937 rng(1);
  for (int page : {16, 32, 48, 64, 65536}) {
    const int width = 5, pages = 7;
    std::vector<int32_t> t = {3, 0, 6, 7, -1};  // the last two do not exist
    for (int64_t p = 0; p < (int64_t)width * page; ++p) {
      const PageRow r = page_row(t.data(), width, page, pages, p);
      const bool ok = p < 3 * (int64_t)page;
      CHECK(r.ok == ok && r.page == (ok ? t[p / page] : 0) && r.row == p % page);
    }
    for (int64_t p : {(int64_t)-1, (int64_t)width * page, (int64_t)1 << 31, (int64_t)1 << 40, -((int64_t)1 << 40)}) {
      const PageRow r = page_row(t.data(), width, page, pages, p);
      CHECK(!r.ok && r.page == 0 && r.row == 0);
    }
    for (int32_t id : {7, -1, 1 << 30, -2147483647 - 1, 2147483647}) {
      t[0] = id;
      CHECK(!page_row(t.data(), width, page, pages, 5).ok && page_row(t.data(), width, page, pages, 5).page == 0);
    }
  }
  CHECK(!page_row(nullptr, 0, 16, 4, 0).ok);
  CHECK(clamp_len(-5, 4, 16) == 0 && clamp_len(64, 4, 16) == 64 && clamp_len(65, 4, 16) == 64 && clamp_len(2147483647, 0, 16) == 0);
  for (int trial = 0; trial < 20000; ++trial) {
    const int batch = 1 + (int)(rng() % 70), workers = 1 + (int)(rng() % 1024);
    const int top = 1 << (rng() % 21);
    std::vector<int> len(batch);
    int64_t total = 0;
    for (int& n : len) total += n = (int)(rng() % top);
    const int64_t chunk = chunk_keys(total, workers);
    CHECK(chunk % 128 == 0 && chunk >= kMinChunk);
    int64_t slots = 0;
    for (int n : len) {
      const int c = chunks_of(n, chunk);
      CHECK(c >= 1 && (int64_t)c * chunk >= n && (n == 0 || (int64_t)(c - 1) * chunk < n));
      CHECK(c <= (n + kMinChunk - 1) / kMinChunk || c == 1);
      slots += c;
    }
    CHECK(slots <= (int64_t)workers + batch);
  }
  CHECK(chunk_keys((int64_t)1 << 50, 1) == (int64_t)1 << 50);
  // sequences as long as a table can hold (they may share pages): the slots still suffice
  for (int batch : {1, 3, 70, 200})
    for (int workers : {0, 1, 2, 128, 1024}) {
      const int len = kMaxKeys - batch % 3;
      const int chunk = chunk_size((int64_t)batch * len, workers);
      CHECK(chunk % 128 == 0);
      CHECK((int64_t)batch * chunks_of(len, chunk) <= (int64_t)workers + batch);
    }
  CHECK(chunk_size(1000, 4) == chunk_keys(1000, 4) && chunk_size((int64_t)1 << 50, 1) == kMaxKeys);
  std::printf("%s\n", bad ? "FAILED" : "ok");
  return bad != 0;
}
