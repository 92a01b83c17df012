// Checks the index rules of the growing cache (cache_index.hpp) for garbage in the device
// arrays: every row is one of the n_tokens rows, every slot of a tile lies in it, every
// tile in the block-table row, no two units of a well-formed batch share a slot, and the
// units of a batch are as many as the launches provide for.
// Usage: cache_index <iterations> <seed>; prints "ok <tiles checked>".
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <limits>
#include <random>
#include <set>
#include <vector>
#include "cache_index.hpp"
using namespace c2kv;
#define CHECK(c) do { if (!(c)) { std::printf("FAIL %s line %d iter %d\n", #c, __LINE__, it); return 1; } } while (0)

int main(int argc, char** argv) {
  const int iters = argc > 1 ? std::atoi(argv[1]) : 1000;
  std::mt19937_64 rng(argc > 2 ? std::atoi(argv[2]) : 1);
  auto pick = [&](int lo, int hi) { return int(lo + int64_t(rng() % uint64_t(int64_t(hi) - lo + 1))); };
  const int wild[] = {std::numeric_limits<int>::min(), -1, 0, 1, 63, 64, 65, 1 << 30,
                      std::numeric_limits<int>::max()};
  long checked = 0;
  for (int it = 0; it < iters; ++it) {
    const bool good = it % 2 == 0;
    const int B = pick(1, 9), PS = 64 * pick(1, 4);
    const int max_pages = it % 7 == 0 ? (1 << 30) / PS : pick(1, 9);
    const int limit = max_pages * PS;
    std::vector<int> off(B + 1), len(B);
    for (int b = 0; b <= B; ++b) off[b] = b ? off[b - 1] + pick(0, 3) * pick(0, 90) : pick(0, 5);
    int n_tokens = off[B] + pick(0, 5);
    for (int b = 0; b < B; ++b) len[b] = pick(0, 700);
    if (!good) {
      n_tokens = pick(0, 300);
      for (int& x : off) if (rng() % 2) x = rng() % 2 ? wild[rng() % 9] : pick(-50, 400);
      for (int& x : len) if (rng() % 2) x = wild[rng() % 9];
    }
    std::set<std::pair<int, int>> seen;          // (request, cache index)
    std::vector<int> rows(size_t(n_tokens) + 1);
    long tiles = 0, covered = 0, expected = 0;
    for (int b = 0; b < B; ++b) {
      const Req r = clamp_req(off[b], off[b + 1], len[b], n_tokens);
      CHECK(r.first >= 0 && r.n >= 0 && r.first + r.n <= n_tokens);
      CHECK(int64_t(r.base) + r.n == std::max(len[b], 0));
      const Tiles t = chunk_tiles(r, limit);
      tiles += t.n;
      for (int i = 0; i < r.n; ++i) {
        const int64_t j = int64_t(r.base) + i;
        if (j >= 0 && j < limit) ++expected;
      }
      for (int i = t.t0; i < t.t0 + t.n; ++i) {
        CHECK(i >= 0 && int64_t(i + 1) * kSlotTile <= limit);
        const TileSlots s = tile_slots(r, i);
        CHECK(s.lo >= 0 && s.lo < s.hi && s.hi <= kSlotTile);
        CHECK(s.row0 + s.lo >= r.first && s.row0 + s.hi <= r.first + r.n);
        for (int k = s.lo; k < s.hi; ++k) {
          CHECK(seen.insert({b, i * kSlotTile + k}).second);
          CHECK(i * kSlotTile + k == r.base + (s.row0 + k - r.first));
          if (good) CHECK(rows[s.row0 + k]++ == 0);
          ++covered;
        }
        ++checked;
      }
    }
    CHECK(covered == expected);
    // ---- attention: the shares of all workgroups hold every tile of every unit once, a
    // unit's pieces lie in consecutive workgroups, and only a workgroup's first piece may
    // continue a unit and only its last be continued
    const int G = pick(1, 9), rb = 16 << pick(0, 4), Hkv = pick(1, 3), W = pick(1, 40);
    int64_t total = 0;
    std::vector<int64_t> ends;                   // of the units, along the line
    for (int b = 0; b < B; ++b) {
      const Req r = clamp_req(off[b], off[b + 1], len[b], n_tokens);
      CHECK(r.n > 0 || row_blocks(r, G, rb) == 0);
      for (int g = 0; g < Hkv; ++g)
        for (int i = 0; i < row_blocks(r, G, rb); ++i) {
          const int t = unit_tiles(r, G, rb, i, limit), keys = unit_keys(r, G, rb, i, limit);
          CHECK(t >= 1 && keys >= 0 && keys <= limit && int64_t(t) * kSlotTile >= keys);
          CHECK(t == 1 || int64_t(t - 1) * kSlotTile < keys);
          // no row of the block sees more
          const int last = std::min((i + 1) * rb, r.n * G) - 1;
          CHECK(keys == std::min(std::max(0, r.base + last / G + 1), limit));
          total += t;
          ends.push_back(total);
        }
      if (Hkv == 1) CHECK(head_tiles(r, G, rb, limit) ==
                          (ends.empty() ? 0 : total - [&] {
                            const int n = row_blocks(r, G, rb);
                            return int(ends.size()) > n ? ends[ends.size() - n - 1] : int64_t(0);
                          }()));
    }
    if (good) CHECK(total <= most_tiles(n_tokens, B, G, Hkv, rb, limit));
    if (total > 0 && total < (int64_t(1) << 31)) {
      const Shares sh = make_shares(unsigned(total), unsigned(W));
      CHECK(sh.begin(0) == 0 && sh.begin(W) == total);
      for (int w = 0; w < W; ++w) {
        const unsigned p0 = sh.begin(w), p1 = sh.begin(w + 1);
        CHECK(p0 <= p1 && p1 - p0 <= total / W + 1);
        if (p0 == p1) continue;
        CHECK(sh.of(p0) == unsigned(w) && sh.of(p1 - 1) == unsigned(w));
      }
      for (int64_t e : ends) {
        const unsigned w = sh.of(unsigned(e - 1));
        CHECK(w < unsigned(W) && sh.begin(w) <= e - 1 && e - 1 < sh.begin(w + 1));
      }
    }
  }
  const int it = -1;
  CHECK(valid_page(-1, 5) == -1 && valid_page(5, 5) == -1 && valid_page(4, 5) == 4);
  CHECK(valid_page(std::numeric_limits<int>::min(), 5) == -1 && valid_page(0, 0) == -1);
  std::printf("ok %ld\n", checked);
  return 0;
}
