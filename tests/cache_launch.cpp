// Checks that every write and read that the growing cache accepts has a grid whose threads
// (256 a workgroup) a launch counts in 32 bits: around each limit of tokens, requests and
// heads, and where the row kernel gives way to the tiles; and what a batch's bound on its chunks
// is where none is given.
// Usage: cache_launch; prints "ok <calls checked>".
#include <cstdio>
#include <initializer_list>

#include "cache_index.hpp"

using namespace c2kv;

#define CHECK(c) do { if (!(c)) { std::printf("FAIL %s line %d: %lld tokens, %lld requests, %lld heads\n", \
    #c, __LINE__, (long long)n, (long long)b, (long long)h); return 1; } } while (0)

int main() {
  const int64_t kThreads = 1ll << 32;
  long checked = 0;
  bool rows = false, tiles = false, refused = false;
  for (int64_t h : {1, 2, 3, 5, 8, 64, 65535})
    for (int64_t n0 : {int64_t(1), int64_t(2048) / h, int64_t(1 << 26) / h, int64_t(1) << 29,
                       (int64_t(1) << 31) / h})
      for (int64_t n = n0 - 9; n <= n0 + 9; ++n)
        for (int64_t b : {int64_t(1), int64_t(1) << 20, (int64_t(1) << 22) - 1, int64_t(1) << 22})
          for (int max_chunk : {1, 8, 9}) {
            // (query heads are as many at least)
            if (n < 1 || n > 1 << 29 || n * h > (1ll << 31) - 1) continue;
            if (most_chunk_tiles(n, b) > kMostGroups) {
              refused = true;
              continue;
            }
            CHECK(most_chunk_tiles(n, b) * 256 < kThreads);
            if (write_by_rows(n, h, max_chunk)) {
              CHECK(row_groups(n, h) * 256 < kThreads && row_groups(n, h) * 4 >= n * h);
              rows = true;
            } else {
              tiles = true;
            }
            ++checked;
          }
  const int64_t n = 0, b = 0, h = 0;
  // the bound, at most all tokens; without one, a step is a token of each request
  CHECK(longest_chunk(5, 100, 3) == 5 && longest_chunk(500, 100, 3) == 100);
  CHECK(longest_chunk(0, 100, 99) == 100 && longest_chunk(0, 100, 100) == 1);
  CHECK(longest_chunk(7, 100, 100) == 7 && longest_chunk(3, 0, 9) == 1);
  CHECK(write_by_rows(512, 8, longest_chunk(0, 512, 512)));
  CHECK(!write_by_rows(512, 8, longest_chunk(0, 512, 511)));
  CHECK(rows && tiles && refused);
  std::printf("ok %ld\n", checked);
  return 0;
}
